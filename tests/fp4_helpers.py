"""Shared pieces of the tests of 4-bit rows."""
import numpy as np

from oracle import entmtp_oracle as orc
from oracle import fp4_oracle as fo
from paper_2606_27550_amd import synth
from tests.paged_helpers import TREES, block_table, row_offsets

D = 128


def quantize_fast(x):
    """fo.quantize for large arrays of finite numbers (tests/test_oracle_fp4.py holds it against that)."""
    g = np.asarray(x, np.float64).reshape(-1, 32)
    m = np.abs(g).max(1)
    e = np.frexp(m)[1] - 1
    e = e + (m >= 1.75 * 2.0 ** e)
    s = np.where(m > 0, np.clip(e - 2 + 127, 2, 252), 2)
    a = np.abs(g) / 2.0 ** (s[:, None] - 127.0)
    c = sum((a > t if k % 2 == 0 else a >= t).astype(np.uint8) for k, t in enumerate((.25, .75, 1.25, 1.75, 2.5, 3.5, 5)))
    c = (c + 8 * np.signbit(g)).astype(np.uint8).reshape(*x.shape)
    return c[..., 0::2] | c[..., 1::2] << 4, s.astype(np.uint8).reshape(*x.shape[:-1], -1)


def pool_bits(pool):
    """4-bit pages as bf16 bits [.., page, 128] (exact)."""
    return orc.f64_to_bf16_bits(fo.pool_values(pool))


def random_pool(g, n_pages, Hkv, page):
    return fo.join(*quantize_fast(orc.bf16_to_f64(synth.normal_bf16(g, (n_pages, Hkv, page, D)))))


def make(seed, topo, lens, Hq, Hkv, page, spare=3, behind=0):
    """Inputs of a batch over 4-bit pools; topo -1: an unused place."""
    g = np.random.default_rng(seed)
    use = [t if 0 <= t < len(TREES) else 0 for t in topo]
    table, n_pages = block_table(g, use, [max(0, L) for L in lens], page, spare)
    off = row_offsets(topo)
    rows = int(off[-1]) + behind
    return dict(topo=np.asarray(topo, np.int32), lens=np.asarray(lens, np.int32), table=table, page=page, n_pages=n_pages,
                off=off, rows=rows, Hq=Hq, Hkv=Hkv, q=synth.normal_bf16(g, (rows, Hq, D)),
                kp=random_pool(g, n_pages, Hkv, page), vp=random_pool(g, n_pages, Hkv, page),
                status=np.array([0 if 0 <= t < len(TREES) else 1 for t in topo], np.int32))


def tree_rows(pool_b, table, L, T, page):
    """bf16 bits [T, Hkv, d] of the rows at positions L .. L + T - 1."""
    return np.stack([pool_b[table[(L + i) // page], :, (L + i) % page] for i in range(T)])
