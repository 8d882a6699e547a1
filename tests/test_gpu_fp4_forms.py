"""GPU: what each of the three forms of the attention over 4-bit pages (at most 16
query rows of a KV head, at most 64, more) does with queries whose values differ
much in size, with groups that are no numbers and with bytes that a window hides.

Bounds.  A query's value of at least 2^-13 of the largest of its 32 enters the
products as it is; a smaller one is off by at most 2^-21 of that largest.  The
sum of 128 products is off by at most 2^-15 of the sum of their magnitudes (the
matrix instruction aligns them before it adds), the scaling in fp32 by less.  So a
score is off by at most d_k = scale (2^-15 sum |q_c k_c| + 2^-21 sum over its
groups of the largest times the |k_c| of the small ones), all of a row's by at
most D, and with it the output by at most (e^(2 D) - 1) sum p |v - out|.  The
weights are rounded to bf16 (2^-8 sum p |v|), a split's partial to fp16 (2^-11 sum
p |v|), the output to bf16 (2^-8 |out|).  A cap bends a score by at most one and
is off by 2^-21 of itself.
"""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import entmtp_oracle as orc  # noqa: E402
from oracle import fp4_oracle as fo  # noqa: E402
from tests.fp4_helpers import D, make, pool_bits  # noqa: E402
from tests.paged_helpers import TREES, say, unbits  # noqa: E402
from tests.test_gpu_fp4_attn import SCALE, launch, nan_row  # noqa: E402

pytestmark = pytest.mark.gpu
FORMS = [(0, 8, 2), (1, 4, 2), (2, 4, 2), (1, 16, 2), (4, 8, 2)]   # 4, 14, 52, 56, 256 rows
APART = (5, 45, 64, 127)   # a channel of each group of 32, in either half


@pytest.fixture(scope="module")
def api():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_27550_amd import api as _api
    return _api


def reference(c, b=0, softcap=0.0, window=0, slopes=None):
    """Sequence b in 64 bits: out [T, Hq, d] and its bound."""
    t, L = int(c["topo"][b]), int(c["lens"][b])
    T, Hq, group = len(TREES[t]), c["Hq"], c["Hq"] // c["Hkv"]
    row = lambda p: np.concatenate([p[c["table"][b][j]] for j in range(-(-(L + T) // c["page"]))], 1)[:, :L + T]   # noqa: E731
    k, v = (orc.bf16_to_f64(row(pool_bits(c[n]))) for n in ("kp", "vp"))
    q = orc.bf16_to_f64(c["q"][int(c["off"][b]):int(c["off"][b]) + T])
    depth = np.array(orc.depths(TREES[t]))
    pos = np.concatenate([np.arange(L), L + depth])
    out, room = np.zeros((T, Hq, D)), np.zeros((T, Hq, D))
    for i in range(T):
        see = np.concatenate([np.ones(L, bool), np.isin(np.arange(T), orc.ancestors_or_self(TREES[t], i))])
        dist = L + depth[i] - pos
        if window:
            see &= dist < window
        for h in range(Hq):
            kk, vv = k[h // group][see], v[h // group][see]
            z = kk @ q[i, h] * SCALE
            if softcap:
                z = softcap * np.tanh(z / softcap)
            if slopes is not None:
                z = z - slopes[h] * dist[see]
            p = np.exp(z - z.max())
            p /= p.sum()
            o = p @ vv
            a = np.abs(q[i, h])
            top = np.repeat(a.reshape(4, 32).max(1), 32)
            off = 2.0 ** -15 * (np.abs(kk) @ a) + 2.0 ** -21 * (np.abs(kk) @ np.where(a < 2.0 ** -13 * top, top, 0.0))
            most = SCALE * float(off.max()) + softcap * 2.0 ** -21
            out[i, h] = o
            room[i, h] = (2.0 ** -8 + 2.0 ** -11) * (p @ np.abs(vv)) + 2.0 ** -8 * np.abs(o) + math.expm1(2 * most) * (p @ np.abs(vv - o))
    return out, room


def apart(c, by):
    """A channel of every group of the queries by times the others, where all keys are zero."""
    c = dict(c, q=c["q"].copy(), kp=c["kp"].copy())
    codes, scales = fo.planes(c["kp"])
    codes = codes.copy()
    for ch in APART:
        codes[..., ch // 2] &= 0xF0 if ch % 2 == 0 else 0x0F
        x = orc.bf16_to_f64(c["q"][..., ch]) * by
        c["q"][..., ch] = orc.f64_to_bf16_bits(x)
    c["kp"] = fo.join(codes, scales)
    return c


@pytest.mark.parametrize("t,Hq,Hkv", FORMS)
@pytest.mark.parametrize("by", [1, 64, 1024, 8192])
@pytest.mark.parametrize("L", [0, 21, 470])
def test_channels_that_stand_out(api, t, Hq, Hkv, by, L):
    """One channel of a group far above the others costs the others nothing (down to 2^-13 of it)."""
    say("fp4 outliers", t, Hq, Hkv, by, L)
    c = apart(make(51 + t + L, [t], [L], Hq, Hkv, 16), by)
    ref, room = reference(c)
    got = orc.bf16_to_f64(unbits(launch(api, c)["out"]))[:len(ref)]
    err = np.abs(got - ref)
    assert (err <= room).all(), float((err / room).max())


@pytest.mark.parametrize("t,Hq,Hkv", FORMS)
@pytest.mark.parametrize("opt", [dict(softcap=5.0), dict(window=40), dict(softcap=9.0, window=17, slopes=True)])
def test_channels_that_stand_out_with_caps_windows_and_biases(api, t, Hq, Hkv, opt):
    say("fp4 outliers", t, Hq, Hkv, opt)
    opt = dict(opt)
    if opt.get("slopes"):
        opt["slopes"] = [2.0 ** (-h) for h in range(Hq)]
    c = apart(make(57 + t, [t], [90], Hq, Hkv, 32), 1024)
    ref, room = reference(c, **opt)
    got = orc.bf16_to_f64(unbits(launch(api, c, **opt)["out"]))[:len(ref)]
    err = np.abs(got - ref)
    assert (err <= room).all(), float((err / room).max())


@pytest.mark.parametrize("t,Hq,Hkv", FORMS[:1] + FORMS[2:3] + FORMS[4:])
@pytest.mark.parametrize("size", [-90, 100])
def test_queries_of_extreme_size(api, t, Hq, Hkv, size):
    """Queries near 2^100 against keys near 2^-100, and the other way round: the scores are ordinary."""
    say("fp4 sizes", t, Hq, Hkv, size)
    c = make(61, [t], [50], Hq, Hkv, 16)
    x = orc.bf16_to_f64(c["q"]) * 2.0 ** size
    codes, scales = fo.planes(c["kp"])
    c["q"] = orc.f64_to_bf16_bits(x)
    c["kp"] = fo.join(codes, np.maximum(scales.astype(int) - size, 2).astype(np.uint8))
    ref, room = reference(c)
    got = orc.bf16_to_f64(unbits(launch(api, c)["out"]))[:len(ref)]
    err = np.abs(got - ref)
    assert (err <= room).all(), float((err / room).max())


@pytest.mark.parametrize("t,Hq,Hkv", [(1, 2, 2), (1, 4, 2), (2, 8, 4), (4, 8, 2), (4, 4, 2)])
@pytest.mark.parametrize("pool", ["kp", "vp"])
def test_groups_that_are_no_numbers_in_every_form(api, t, Hq, Hkv, pool):
    """A bad group makes NaN of the rows that see its key, whole, and of no others, whichever half or block it lies in."""
    L, T, group = 300, len(TREES[t]), Hq // Hkv
    say("fp4 no numbers", t, Hq, Hkv, pool)
    c = make(71 + t, [t], [L], Hq, Hkv, 16)
    ref = orc.bf16_to_f64(unbits(launch(api, c)["out"]))
    clean = c[pool].copy()
    # (at 300: the block of 32 keys from 288 on holds prefix and tree; a node in its second half, others in later blocks)
    nodes = sorted({0, 1, T // 2, T - 1} | {n for n in (4, 20, 36) if n < T})
    for k, node in enumerate(nodes):
        c[pool] = clean.copy()
        nan_row(c, pool, 0, L + node, k % Hkv, group=k % 4)
        got = orc.bf16_to_f64(unbits(launch(api, c)["out"]))
        want = np.zeros((T, Hq), bool)
        heirs = [i for i in range(T) if node in orc.ancestors_or_self(TREES[t], i)]
        want[heirs, (k % Hkv) * group:(k % Hkv + 1) * group] = True
        np.testing.assert_array_equal(np.isnan(got).any(2), want)
        assert np.isnan(got[want]).all()
        np.testing.assert_array_equal(got[~want], ref[~want])
    # several at once, in one block and in neighbouring ones, beside a prefix key of another head
    c[pool] = clean.copy()
    want = np.zeros((T, Hq), bool)
    for k, node in enumerate(nodes):
        nan_row(c, pool, 0, L + node, 0, group=k % 4)
        want[[i for i in range(T) if node in orc.ancestors_or_self(TREES[t], i)], :group] = True
    for pos in (0, 17, 31, 32, 150):
        nan_row(c, pool, 0, pos, 1, group=3)
    want[:, group:2 * group] = True
    got = orc.bf16_to_f64(unbits(launch(api, c)["out"]))
    np.testing.assert_array_equal(np.isnan(got).any(2), want)
    assert np.isnan(got[want]).all()
    np.testing.assert_array_equal(got[~want], ref[~want])


@pytest.mark.parametrize("t,Hq,Hkv,L,window", [(0, 8, 2, 301, 20), (0, 4, 4, 1000, 64), (1, 4, 2, 700, 33), (1, 2, 1, 90, 1)])
@pytest.mark.parametrize("pool", ["kp", "vp"])
def test_bytes_before_a_window_of_few_rows(api, t, Hq, Hkv, L, window, pool):
    """Slots before every row's window hold any bytes, in the window's own blocks too; the outputs are the same bits."""
    say("fp4 window bytes", t, Hq, Hkv, L, window, pool)
    c, g = make(81 + L, [t], [L], Hq, Hkv, 16), np.random.default_rng(L)
    want = unbits(launch(api, c, window=window)["out"])
    codes, scales = (x.copy() for x in fo.planes(c[pool]))
    for pos in range(L - window + 1):
        at = (c["table"][0, pos // 16], slice(None), pos % 16)
        codes[at] = g.integers(0, 256, codes[at].shape)
        scales[at] = g.choice([0, 1, 127, 252, 253, 254, 255], scales[at].shape)
    c[pool] = fo.join(codes, scales)
    got = unbits(launch(api, c, window=window)["out"])
    assert np.isfinite(orc.bf16_to_f64(want)).all()
    np.testing.assert_array_equal(got, want)
