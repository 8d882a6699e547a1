"""GPU: compaction of the accepted paths in the page pool, bit for bit."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import entmtp_oracle as orc  # noqa: E402
from oracle import paged_oracle as po  # noqa: E402
from tests.paged_helpers import TREES, bits, block_table, i32, row_offsets, say, unbits  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_27550_amd import api as _api
    return _api


def case(seed, B, page, path_cap):
    g = np.random.default_rng(seed)
    topo = g.integers(0, len(TREES), B)
    lens = g.integers(0, 90, B)
    table, n_pages = block_table(g, topo, lens, page)
    off = row_offsets(topo)
    slots = np.concatenate([[table[b, (L + i) // page] * page + (L + i) % page for i in range(len(TREES[t]))]
                            for b, (t, L) in enumerate(zip(topo, lens))]).astype(np.int32)
    path = np.full((B, path_cap), -1, np.int32)
    a = np.zeros(B, np.int32)
    for b, t in enumerate(topo):
        chain = orc.ancestors_or_self(TREES[t], int(g.integers(0, len(TREES[t]))))[:path_cap]
        path[b, :len(chain)] = chain
        a[b] = len(chain) - 1
    return g, path, a, off, slots, n_pages


def pools(g, layers, n_pages, Hkv, page, d):
    return [g.integers(0, 2 ** 16, (layers, n_pages, Hkv, page, d), dtype=np.uint16) for _ in range(2)]


@pytest.mark.parametrize("B,page,path_cap,layers,Hkv,d", [
    (1, 16, 32, 1, 8, 128), (4, 32, 32, 3, 2, 128), (9, 256, 16, 2, 1, 64), (3, 16, 7, 1, 5, 8), (2, 64, 32, 1, 3, 256),
    (40, 16, 5, 2, 4, 128), (2, 128, 1, 1, 2, 128), (3, 16, 40, 2, 8, 128)])
def test_against_the_oracle(api, B, page, path_cap, layers, Hkv, d):
    say("kv_compact_paged", B, page, path_cap, layers, Hkv, d)
    g, path, a, off, slots, n_pages = case(B + page, B, page, path_cap)
    k, v = pools(g, layers, n_pages, Hkv, page, d)
    kd, vd = bits(k), bits(v)
    args = (i32(path), i32(a), i32(off), i32(slots))
    api.kv_compact_paged(*args, kd if layers > 1 else kd[0], vd if layers > 1 else vd[0])
    np.testing.assert_array_equal(unbits(kd), po.kv_compact_paged(k, path, a, off, slots))
    np.testing.assert_array_equal(unbits(vd), po.kv_compact_paged(v, path, a, off, slots))


def test_arbitrary_paths_read_before_they_write(api):
    """Any order of nodes: a source that is another row's destination still holds the old row."""
    g, path, a, off, slots, n_pages = case(3, 2, 16, 8)
    path[0], a[0] = [2, 0, 1, 4, 3, 6, 5, 0], 7
    off = np.array([0, 26, 33], np.int32)
    slots = g.permutation(n_pages * 16)[:33].astype(np.int32)
    k, v = pools(g, 1, n_pages, 4, 16, 128)
    kd, vd = bits(k), bits(v)
    api.kv_compact_paged(i32(path), i32(a), i32(off), i32(slots), kd[0], vd[0])
    np.testing.assert_array_equal(unbits(kd), po.kv_compact_paged(k, path, a, off, slots))
    np.testing.assert_array_equal(unbits(vd), po.kv_compact_paged(v, path, a, off, slots))


def test_what_cannot_move_stays(api):
    """Not verified, not mapped, nodes outside the sequence's rows, slots
    outside the pool, accept lengths past the path."""
    g = np.random.default_rng(4)
    B, page, n_pages = 7, 16, 12
    off = np.array([0, 8, 16, 24, 32, 40, 48, 2 ** 31 - 1], np.int32)
    slots = g.permutation(n_pages * page)[:56].astype(np.int32)
    path = np.tile(np.array([0, 3, 5, 7], np.int32), (B, 1))
    a = np.array([-1, 3, 3, 3, 2 ** 31 - 1, 3, 3], np.int32)
    slots[8:16] = -1                    # 1: not mapped
    path[2] = [0, 8, 2 ** 31 - 1, -7]   # 2: no row moves
    slots[24 + 3], slots[24 + 2] = n_pages * page, 2 ** 31 - 1    # 3: one source, one destination outside
    off[6] = -3                         # 5 ends below its start, 6 starts below zero
    k, v = pools(g, 2, n_pages, 2, page, 128)
    kd, vd = bits(k), bits(v)
    api.kv_compact_paged(i32(path), i32(a), i32(off), i32(slots), kd, vd)
    good = path.copy()
    good[2] = -1
    keep = a.copy()
    keep[[0, 1, 5, 6]] = -1
    safe = off.copy()
    safe[6:] = 48
    want = po.kv_compact_paged(k, good, keep, safe, slots)
    np.testing.assert_array_equal(unbits(kd), want)
    np.testing.assert_array_equal(unbits(vd), po.kv_compact_paged(v, good, keep, safe, slots))
