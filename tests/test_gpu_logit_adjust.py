"""GPU: penalties, biases and grammar masks on the logits of tree rows, and the
statistics of the result, against 64 bits.

Tolerances.  A logit takes at most five fp32 roundings (division or product,
freq * c, two differences, the bias), each at most 2^-24 of the largest
magnitude on the way: 5 * 2^-24 * (|z'| + |freq c| + |pres| + |bias|).  The
statistics are held against those of the kernel's own logits: with t = (z -
max) inv_temp, an exponential is off by (3 |t| + 2) 2^-24 of itself (two
roundings of t, one of the base-2 exponent, the instruction's ulp), a sum over
a thread's 16 entries, 64 lanes and the slices adds up to 40 roundings; so Z is
off by 2^-24 (3 E|t| + 42) of itself, S / Z by 2^-24 E[3 t^2 + 42 |t|], and ln
and the division add a few roundings of their results.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import paged_oracle as po  # noqa: E402
from tests.paged_helpers import TREES, dev, host, i32, row_offsets, say  # noqa: E402

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def api():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_27550_amd import api as _api
    return _api


def make(seed, topo, V, history=True, bias=True, mask=True, neutral=(), behind=0):
    g = np.random.default_rng(seed)
    B, off = len(topo), row_offsets(topo)
    rows = int(off[-1]) + behind
    c = dict(topo=np.asarray(topo, np.int32), off=off, V=V, rows=rows,
             z=(g.standard_normal((rows, V)) * 3).astype(np.float32), tok=g.integers(-1, V + 1, rows).astype(np.int32),
             params=np.stack([1 + g.random(B), g.random(B) - 0.3, g.random(B) - 0.3, 0.5 + g.random(B)], 1).astype(np.float32),
             history=None, bias=None, bias_idx=None, mask=None, mask_idx=None)
    for b in neutral:
        c["params"][b] = [1, 0, 0, 1]
    if history:
        h = np.where(g.random((B, V)) < 0.1, g.integers(1, 5, (B, V)), 0)
        c["history"] = (h | np.where(g.random((B, V)) < 0.1, po.SEEN, 0)).astype(np.int32)
    if bias:
        c["bias"] = (g.standard_normal((2, V)) * (g.random((2, V)) < 0.2)).astype(np.float32)
        c["bias_idx"] = np.resize(np.array([1, -1, 0, 2, 2 ** 31 - 1], np.int32), B)
    if mask:
        c["mask"] = g.integers(-2 ** 31, 2 ** 31, (3, (V + 31) // 32 + 1)).astype(np.int32)
        c["mask"][1] = 0
        c["mask"][2] = -1
        c["mask_idx"] = np.resize(np.array([0, -1, 2, 0, 1, 3, -2 ** 31], np.int32), rows)
    return c


def launch(api, c, in_place=False, out=True, stats=True, trees=TREES, stream=None, bank=None):
    d = {k: (None if v is None else dev(v)) for k, v in c.items() if k not in ("V", "rows")}
    rows, V = c["rows"], c["V"]
    d["out"] = d["z"] if in_place else (torch.full((rows, V), 7.0, device="cuda") if out else None)
    d["H"], d["p1"] = (torch.full((rows,), 7.0, device="cuda") if stats else None for _ in range(2))
    d["am"] = torch.full((rows,), 7, dtype=torch.int32, device="cuda") if stats else None
    ws = torch.empty(api.logit_adjust_workspace(rows, V), dtype=torch.uint8, device="cuda") if stats else None
    d["bank"] = bank or api.Bank(trees)
    d["go"] = lambda: api.logit_adjust(d["bank"], d["topo"], d["off"], d["tok"], d["z"], d["params"], d["out"], d["H"], d["p1"],
                                       d["am"], ws, history=d["history"], bias=d["bias"], bias_idx=d["bias_idx"],
                                       mask=d["mask"], mask_idx=d["mask_idx"], stream=stream)
    d["go"]()
    torch.cuda.synchronize()
    return d


def expected(c, trees=TREES):
    """Per row: (adjusted logits in 64 bits, tolerance), or None for a row of no sequence."""
    rows = [None] * c["rows"]
    for b, t in enumerate(c["topo"]):
        if not 0 <= t < len(trees):
            continue
        r0 = int(c["off"][b])
        tok = c["tok"][r0:r0 + len(trees[t])]
        bi = None if c["bias"] is None else int(c["bias_idx"][b])
        bias = c["bias"][bi].astype(np.float64) if bi is not None and 0 <= bi < len(c["bias"]) else None
        for i in range(len(trees[t])):
            allowed = None
            if c["mask"] is not None and 0 <= c["mask_idx"][r0 + i] < len(c["mask"]):
                w = c["mask"][c["mask_idx"][r0 + i]].view(np.uint32)
                v = np.arange(c["V"])
                allowed = (w[v >> 5] >> (v & 31).astype(np.uint32)) & 1 == 1
            h = None if c["history"] is None else c["history"][b]
            args = (c["z"][r0 + i], trees[t], i, tok, c["params"][b], h)
            z = po.adjusted_row(*args, bias, allowed)
            raw = po.adjusted_row(*args, None, None)
            said = np.abs(np.nan_to_num(raw)) + abs(c["params"][b][1]) * 40 + abs(c["params"][b][2])
            if bias is not None:
                said = said + np.abs(bias)
            rows[r0 + i] = (z, 5 * U * said, float(c["params"][b][3]))
    return rows


def check_stats(z, it, H, p1, am, what):
    """The statistics of the kernel's own row of logits (fp32 values in 64 bits)."""
    rH, rp, ram = po.row_stats(z, it)
    assert am == ram, what
    if np.isnan(rH):
        assert np.isnan(H) and np.isnan(p1), what
        return
    if ram < 0:
        assert H == 0 and p1 == 0, what
        return
    t = (z[z > -np.inf] - z.max()) * it
    p = np.exp(t) / np.exp(t).sum()
    a = np.abs(t)
    assert abs(p1 - rp) <= rp * U * (3 * (p * a).sum() + 42), what
    assert abs(H - rH) <= U * ((p * (3 * a * a + 42 * a)).sum() + 3 * (p * a).sum() + 42 + 8 * (abs(rH) + np.log(z.size) + 1)), what


def check(c, d, trees=TREES):
    want = expected(c, trees)
    out = None if d["out"] is None else host(d["out"])
    H, p1, am = (None if d[k] is None else host(d[k]) for k in ("H", "p1", "am"))
    for r, w in enumerate(want):
        if w is None:
            if out is not None:
                np.testing.assert_array_equal(out[r], c["z"][r] if d["out"] is d["z"] else np.full(c["V"], 7, np.float32))
            if H is not None:
                assert H[r] == 7 and p1[r] == 7 and am[r] == 7
            continue
        z, tol, it = w
        if out is not None:
            got = out[r].astype(np.float64)
            fin = np.isfinite(z)
            np.testing.assert_array_equal(np.isfinite(got), fin)
            np.testing.assert_array_equal(got[~fin], z[~fin])
            assert (np.abs(got[fin] - z[fin]) <= tol[fin]).all(), r
        if H is not None and out is not None:
            check_stats(out[r].astype(np.float64), it, H[r], p1[r], am[r], r)
    return want


@pytest.mark.parametrize("topo,V", [
    ([0], 1), ([1], 3), ([2], 32), ([0, 1, 2], 4095), ([1, 0], 4096), ([2, 1], 4097), ([6], 12300), ([3, 2, 1], 8202),
    ([1, 3], 50257), ([2], 128256)])
def test_against_64_bits(api, topo, V):
    say("logit_adjust", topo, V)
    c = make(V, topo, V, behind=3)
    check(c, launch(api, c))


@pytest.mark.parametrize("V", [50, 64])
def test_many_rows(api, V):
    """32 trees of 256 nodes: the form that takes four rows a workgroup, across sequences."""
    topo = [5, -1] * 3 + [5] * 29 + [1, 0, 0, 1]
    say("logit_adjust many rows", V)
    c = make(V, topo, V, neutral=(4, 9), behind=1)
    assert c["rows"] >= 8192
    check(c, launch(api, c))


def test_many_slices_and_rows(api):
    c = make(5, [4, 5, 2], 102400, bias=False)
    assert c["rows"] * (102400 // 4096) >= 8192
    say("logit_adjust", c["rows"], "rows of 102400")
    check(c, launch(api, c))


@pytest.mark.parametrize("history,bias,mask", [(False, False, False), (True, False, False), (False, True, False),
                                               (False, False, True), (False, True, True)])
def test_parts_alone(api, history, bias, mask):
    c = make(6, [2, 1, 0], 5000, history=history, bias=bias, mask=mask, neutral=(1,))
    check(c, launch(api, c))


def test_in_place_no_logits_no_statistics(api):
    c = make(7, [2, 1, -1, 0], 9001, behind=2)
    ref = launch(api, c)
    d = launch(api, c, in_place=True)
    check(c, d)
    np.testing.assert_array_equal(host(d["out"])[:-2], host(ref["out"])[:-2])
    only = launch(api, c, out=False)
    for k in ("H", "p1", "am"):
        np.testing.assert_array_equal(host(only[k]), host(ref[k]))
    bare = launch(api, c, stats=False)
    np.testing.assert_array_equal(host(bare["out"]), host(ref["out"]))
    launch(api, c, out=False, stats=False)


def test_values_that_are_not_finite(api):
    """Hidden by a mask they are gone; else NaN and +inf show, -inf counts for nothing."""
    V = 9000
    c = make(8, [2], V, history=False, bias=False)
    c["params"][0] = [1.2, 0.1, 0.1, 0.8]
    c["mask_idx"][:] = -1
    for r, bad in enumerate([np.nan, np.inf, -np.inf]):
        c["z"][r, [0, 4095, 4096, V - 1]] = bad
        c["z"][3 + r, [0, 4095, 4096, V - 1]] = bad
        c["mask_idx"][3 + r] = 0
    c["mask"][0] = -1
    for v in (0, 4095, 4096, V - 1):
        w = c["mask"][0].view(np.uint32)
        w[v >> 5] &= np.uint32(0xFFFFFFFF) ^ np.uint32(1 << (v & 31))
    c["z"][6] = -np.inf
    c["z"][7] = np.nan
    c["z"][8, :] = -np.inf
    c["z"][8, 5000] = np.nan
    c["tok"][:] = -1
    d = launch(api, c)
    H, p1, am, out = (host(d[k]) for k in ("H", "p1", "am", "out"))
    assert np.isnan(H[[0, 1, 7, 8]]).all() and np.isnan(p1[[0, 1, 7, 8]]).all()
    assert am[1] == 0 and am[7] == -1 and am[8] == -1
    assert am[0] == np.argmax(np.nan_to_num(c["z"][0], nan=-np.inf))
    assert (H[6], p1[6], am[6]) == (0, 0, -1)
    for r in (2, 3, 4, 5):
        assert (out[r, [0, 4095, 4096, V - 1]] == -np.inf).all()
        check_stats(out[r].astype(np.float64), 0.8, H[r], p1[r], am[r], r)


def test_a_mask_that_allows_nothing_and_one_token(api):
    c = make(9, [1, 1], 4100)
    c["mask_idx"][:] = 1                                     # nothing
    c["mask"][0] = 0
    c["mask"][0, 4099 >> 5] = np.int32(1 << (4099 & 31))      # the last token alone
    c["mask_idx"][3] = 0
    d = launch(api, c)
    H, p1, am = (host(d[k]) for k in ("H", "p1", "am"))
    for r in range(c["rows"]):
        assert (H[r], p1[r], am[r]) == ((0, 1, 4099) if r == 3 else (0, 0, -1))
    check(c, d)


def test_the_lowest_index_wins_a_tie(api):
    c = make(10, [1], 20000, history=False, bias=False, mask=False)
    c["tok"][:] = -1
    c["z"][:] = 0.5
    d = launch(api, c)
    assert (host(d["am"]) == 0).all()
    c["z"][:, 100] = c["z"][:, 4096] = c["z"][:, 19999] = 3
    d = launch(api, c)
    assert (host(d["am"]) == 100).all()


def test_one_token_drafted_along_a_whole_path(api):
    """32 nodes that all draft token 3: node i's row counts it i times."""
    c = make(11, [3], 8, history=False, bias=False, mask=False)
    c["tok"][:] = 3
    c["params"][0] = [1, 0.25, 0, 1]
    c["z"][:] = 1
    d = launch(api, c)
    out = host(d["out"])
    np.testing.assert_array_equal(out[:, 3], 1 - 0.25 * np.arange(32, dtype=np.float32))
    assert (np.delete(out, 3, 1) == 1).all()


def test_entries_the_host_cannot_check(api):
    """Row offsets and tree indexes that fit nothing: those rows are left alone."""
    c = make(12, [1, 2, 1], 300)
    good = launch(api, c)
    for off, topo in (([0, 7, 33, 40], [1, 2 ** 31 - 1, 1]), ([0, 7, 33, 40], [-2 ** 31, 2, 1]),
                      ([3, 10, 36, 40], [1, 2, 1]), ([0, 2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1], [1, 2, 1]),
                      ([-5, -5, -5, -5], [1, 2, 1]), ([30, 20, 10, 0], [1, 2, 1])):
        k = dict(c, off=np.array(off, np.int32), topo=np.array(topo, np.int32))
        d = launch(api, k)
        out = host(d["out"])
        assert np.isfinite(host(d["H"])).all()
        if off[0] == 0 and off[1] == 7:
            for b in range(3):
                rows = slice(off[b], off[b + 1])
                if 0 <= topo[b] < len(TREES):
                    np.testing.assert_array_equal(out[rows], host(good["out"])[rows])
                else:
                    assert (out[rows] == 7).all()
        if off[0] == 3:
            assert (out[:3] == 7).all()


def test_streams_and_graph(api):
    c = make(13, [2, 1], 6000)
    ref = launch(api, c)
    s = torch.cuda.Stream()
    d = launch(api, c, stream=s, bank=ref["bank"])
    np.testing.assert_array_equal(host(d["out"]), host(ref["out"]))
    g = launch(api, c, bank=ref["bank"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g["go"]()
    for k in range(3):
        g["out"].fill_(5)
        g["z"].add_(0.5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        now = dict(c, z=host(g["z"]).copy())
        check(now, g)


def test_refusals(api):
    c = make(14, [1], 64)
    d = launch(api, c)
    for bad in (dict(z=d["z"][:, ::2]), dict(tok=d["tok"][:-1]), dict(params=d["params"][:, :3].contiguous()),
                dict(history=d["history"][:, :-1].contiguous()), dict(bias_idx=None), dict(mask_idx=None),
                dict(off=d["off"][:-1]), dict(topo=d["topo"].long()), dict(out=d["out"].double())):
        a = {**d, **bad}
        with pytest.raises(ValueError):
            api.logit_adjust(d["bank"], a["topo"], a["off"], a["tok"], a["z"], a["params"], a["out"], a["H"], a["p1"], a["am"],
                             torch.empty(1 << 20, dtype=torch.uint8, device="cuda"), history=a["history"], bias=a["bias"],
                             bias_idx=a["bias_idx"], mask=a["mask"], mask_idx=a["mask_idx"])
    with pytest.raises(api.EntmtpError):
        api.logit_adjust(d["bank"], d["topo"], d["off"], d["tok"], d["z"], d["params"], d["out"], d["H"], d["p1"], d["am"], None)
    with pytest.raises(api.EntmtpError):
        api.logit_adjust(api.Bank(TREES, device=None), d["topo"], d["off"], d["tok"], d["z"], d["params"], d["out"], None, None,
                         None, None)
    assert i32 is not None
