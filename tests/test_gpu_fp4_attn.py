"""GPU: tree attention over 4-bit pages against 64 bits.

The pages' numbers are exact in bf16, so the oracle's attention over bf16 pages
applies, with its bounds: per element roundings to bf16 (weights, a split's
partial, the output: 2^-8 of the value each, and the query's) pushed through the
softmax; over a whole output 2^-7 in the 2-norm as for bf16 pages.  A partial is
fp16 here, which is less.  A query enters as three 6-bit numbers: the first leaves
1/16 of a step in which the largest of its 32 numbers is 3.75 to 7.5 (below 2; up to
1/4 above), the others 2^-3 of that each, so that it is off by at most 2^-10 steps,
2^-10 / 3.75 of the largest.  The oracle allows it 2^-8 of every number; the check
asserts that this moves no row's scores by more.
"""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import entmtp_oracle as orc  # noqa: E402
from oracle import fp4_oracle as fo  # noqa: E402
from oracle import paged_oracle as po  # noqa: E402
from tests.fp4_helpers import D, make, pool_bits, tree_rows  # noqa: E402
from tests.paged_helpers import TREES, bits, dev, host, i32, say, unbits  # noqa: E402
from tests.test_gpu_paged_attn import CASES  # noqa: E402

pytestmark = pytest.mark.gpu
SCALE = 1 / math.sqrt(D)


@pytest.fixture(scope="module")
def api():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_27550_amd import api as _api
    return _api


def launch(api, c, softcap=0.0, window=0, slopes=None, bank=None, stream=None, plan_window=None, run=True):
    B, rows = len(c["topo"]), c["rows"]
    d = {k: i32(c[k]) for k in ("topo", "lens", "table", "off", "status")}
    d.update(q=bits(c["q"]), kp=dev(c["kp"]), vp=dev(c["vp"]), bank=bank or api.Bank(TREES))
    d["out"] = torch.full((rows, c["Hq"], D), 7.0, dtype=torch.bfloat16, device="cuda")
    d["bad"] = torch.full((B,), 9, dtype=torch.int32, device="cuda")
    d["slopes"] = None if slopes is None else dev(np.asarray(slopes, np.float32))
    shape = (rows, c["Hq"], c["Hkv"])
    mp = c["table"].shape[1]
    d["plan"] = torch.empty(api.tree_attn_paged_fp4_plan_bytes(d["bank"], B, *shape, mp, c["page"]), dtype=torch.uint8,
                            device="cuda")
    ws = api.tree_attn_paged_fp4_workspace(d["bank"], B, *shape, D, mp, c["page"])
    d["ws"] = torch.empty(ws, dtype=torch.uint8, device="cuda") if ws else None

    def plan():
        api.tree_attn_paged_fp4_plan(d["bank"], d["topo"], d["lens"], d["off"], d["status"], d["table"], c["page"],
                                     c["n_pages"], *shape, d["plan"], window=window if plan_window is None else plan_window,
                                     bad=d["bad"], stream=stream)

    def attend():
        api.tree_attn_paged_fp4(d["bank"], d["plan"], d["q"], d["kp"], d["vp"], d["table"], SCALE, d["out"], d["ws"],
                                softcap=softcap, window=window, slopes=d["slopes"], stream=stream)
    d["plan_call"], d["attend"] = plan, attend
    if run:
        plan()
        attend()
        torch.cuda.synchronize()
    return d


def check(c, out, idle=(), nan=(), softcap=0.0, window=0, slopes=None):
    """Every sequence against the oracle; those in idle (and rows of none) untouched; rows in nan NaN."""
    got = orc.bf16_to_f64(out)
    kp, vp = pool_bits(c["kp"]), pool_bits(c["vp"])
    left = np.ones(c["rows"], bool)
    e2, n2 = 0.0, 0.0
    for b, (t, L) in enumerate(zip(c["topo"], c["lens"])):
        if not 0 <= t < len(TREES) or b in idle:
            continue
        T, r0 = len(TREES[t]), int(c["off"][b])
        r = slice(r0, r0 + T)
        rows = [tree_rows(p, c["table"][b], int(L), T, c["page"]) for p in (kp, vp)]
        ref, _, off = po.tree_attention_paged(c["q"][r], *rows, kp, vp, c["table"][b], int(L), TREES[t], SCALE, 0.0, softcap,
                                              window, slopes)
        left[r] = False
        keys = orc.bf16_to_f64(np.concatenate([kp[c["table"][b][j]] for j in range(-(-(L + T) // c["page"]))], 1))[:, :L + T]
        q = np.abs(orc.bf16_to_f64(c["q"][r]))
        q[~np.isfinite(q)] = 0
        top = np.repeat(q.reshape(T, c["Hq"], 4, 32).max(3), 32, 2)
        for g in range(c["Hkv"]):
            of = slice(g * c["Hq"] // c["Hkv"], (g + 1) * c["Hq"] // c["Hkv"])
            k = np.nan_to_num(np.abs(keys[g])).T
            assert ((top[:, of] @ k).max(-1) * 2.0 ** -10 / 3.75 <= (q[:, of] @ k).max(-1) * 2.0 ** -8).all()
        fine = np.array([i not in nan for i in range(r0, r0 + T)])
        assert np.isnan(got[r][~fine]).all()
        err = np.abs(got[r] - ref)[fine]
        assert (err <= off[fine]).all(), (b, t, L, float((err / off[fine]).max()))
        e2 += float((err ** 2).sum())
        n2 += float((ref[fine] ** 2).sum())
    assert e2 <= (2.0 ** -7) ** 2 * n2, math.sqrt(e2 / n2)
    assert (out[left] == 0x40E0).all()


@pytest.mark.parametrize("topo,lens,Hq,Hkv,page", CASES)
def test_against_64_bits(api, topo, lens, Hq, Hkv, page):
    say("tree_attn_paged_fp4", topo, lens, Hq, Hkv, page)
    c = make(len(topo) + lens[0], topo, lens, Hq, Hkv, page, behind=2)
    d = launch(api, c)
    assert (host(d["bad"]) == 0).all()
    check(c, unbits(d["out"]))
    np.testing.assert_array_equal(host(d["kp"]), c["kp"])   # (read only)
    np.testing.assert_array_equal(host(d["vp"]), c["vp"])


OPTIONS = [dict(softcap=3.0), dict(softcap=1024.0), dict(softcap=0.01), dict(window=1), dict(window=2), dict(window=5),
           dict(window=33), dict(window=64), dict(window=500), dict(window=2 ** 31 - 1), dict(slopes=True),
           dict(softcap=30.0, window=40), dict(softcap=2.0, window=100, slopes=True)]


@pytest.mark.parametrize("opt", OPTIONS)
def test_caps_windows_and_biases(api, opt):
    say("tree_attn_paged_fp4", opt)
    opt = dict(opt)
    if opt.get("slopes"):
        opt["slopes"] = [2.0 ** (-h) for h in range(8)]
    c = make(7, [2, 0, 3, 6, 1], [700, 40, 90, 333, 0], 8, 2, 16, behind=1)
    d = launch(api, c, **opt)
    check(c, unbits(d["out"]), **opt)


def test_head_groups(api):
    """A KV head's rows in one tile, two, three, more than four: the wavefronts share them differently."""
    for t, Hq, Hkv in ((1, 4, 1), (2, 2, 1), (2, 3, 1), (4, 1, 1), (4, 2, 1), (5, 1, 1), (2, 32, 1)):
        say("tree_attn_paged_fp4 groups", t, Hq, Hkv)
        c = make(t + Hq, [t, t], [450, 77], Hq, Hkv, 32)
        check(c, unbits(launch(api, c)["out"]))


def test_split_and_whole_agree(api):
    """The same sequence alone (split over the chip) and in a batch that leaves it whole."""
    c1 = make(21, [2], [900], 8, 2, 16)
    one = orc.bf16_to_f64(unbits(launch(api, c1)["out"]))
    c2 = make(21, [2] * 120, [900] * 120, 8, 2, 16)
    n = c1["n_pages"]
    for k in ("kp", "vp"):
        c2[k][:n] = c1[k]
    c2["table"][:] = c1["table"][0][None, :c2["table"].shape[1]]
    c2["q"] = np.tile(c1["q"], (120, 1, 1))
    many = orc.bf16_to_f64(unbits(launch(api, c2)["out"])).reshape(120, 26, 8, D)
    assert (many == many[:1]).all()
    # (each is off by at most its own roundings)
    assert np.linalg.norm(many[0] - one) <= 2 * 2.0 ** -7 * np.linalg.norm(one)


def test_repeats_are_the_same(api):
    c = make(23, [2, 4, 0], [1200, 333, 4000], 8, 2, 16)
    d = launch(api, c)
    first = unbits(d["out"])
    for _ in range(5):
        d["out"].fill_(3)
        d["attend"]()
        torch.cuda.synchronize()
        np.testing.assert_array_equal(unbits(d["out"]), first)


def test_bad_pages_and_unmapped_sequences(api):
    """A page outside the pool (of the prefix or of the tree), a status, no room: no work, and the others have theirs."""
    c = make(25, [1, 2, 1, 4, 0], [100, 64, 40, 30, 700], 8, 2, 16)
    c["table"][0, 3] = c["n_pages"]
    c["table"][2, 2] = -1            # the tree's page (positions 32 .. 47)
    c["status"][3] = po.FULL
    d = launch(api, c)
    assert host(d["bad"]).tolist() == [1, 0, 1, 0, 0]
    assert host(api.tree_attn_paged_topo(d["plan"], 5)).tolist() == [-1, 2, -1, -1, 0]
    check(c, unbits(d["out"]), idle=(0, 2, 3))


def test_pages_that_change_after_the_plan(api):
    """They read as zeros (never out of bounds), and only their sequence's rows change."""
    c = make(27, [0, 1], [200, 90], 4, 2, 16)
    d = launch(api, c, run=False)
    d["plan_call"]()
    d["table"][1, 1:4] = i32([-5, c["n_pages"], 2 ** 31 - 1])
    d["attend"]()
    torch.cuda.synchronize()
    got = unbits(d["out"])
    kp, vp = (p.copy() for p in (c["kp"], c["vp"]))
    zero = np.zeros((1, *kp.shape[1:]), np.uint8)
    codes, scales = fo.planes(zero)
    scales = scales + 127
    zero = fo.join(codes, scales.astype(np.uint8))
    c2 = dict(c, kp=np.concatenate([kp, zero]), vp=np.concatenate([vp, zero]), table=c["table"].copy())
    c2["table"][1, 1:4] = c["n_pages"]
    check(c2, got)


def test_another_plan_does_nothing(api):
    c = make(29, [1], [40], 4, 2, 16)
    d = launch(api, c, run=False, plan_window=9)
    d["plan_call"]()
    d["attend"]()                     # a plan of another window
    torch.cuda.synchronize()
    assert (unbits(d["out"]) == 0x40E0).all()
    shape = (c["rows"], 4, 2)         # a bf16 pool's plan
    api.tree_attn_paged_plan(d["bank"], d["topo"], d["lens"], d["off"], d["status"], d["table"], 16, c["n_pages"], *shape,
                             d["plan"])
    d["attend"]()
    torch.cuda.synchronize()
    assert (unbits(d["out"]) == 0x40E0).all()


def nan_row(c, pool, b, pos, g, group=1):
    page = c["page"]
    slot = c["table"][b, pos // page]
    c[pool][slot, g, page * 64 + (pos % page) * 4 + group] = 255


@pytest.mark.parametrize("pool", ["kp", "vp"])
def test_groups_that_are_no_numbers(api, pool):
    """Rows that see their key become NaN, the others keep their values: of the prefix every row of the KV head's, of the
    tree the node's own line, of what a window hides, of slots past the tree, none."""
    t, L, W = 2, 300, 64
    T = len(TREES[t])
    c = make(31, [t], [L], 4, 2, 16)
    clean = c[pool].copy()
    node = 7
    heirs = [i for i in range(T) if node in orc.ancestors_or_self(TREES[t], i)]
    assert 0 < len(heirs) < T
    nan_row(c, pool, 0, L + node, 0)
    last = (L + T - 1) % 16
    if last < 15:                     # a slot behind the tree's last row
        nan_row(c, pool, 0, L + T, 0)
        nan_row(c, pool, 0, L + T, 1)
    d = launch(api, c)
    got = orc.bf16_to_f64(unbits(d["out"]))
    is_nan = np.isnan(got).all(2)
    assert (is_nan == np.isnan(got).any(2)).all()
    want = np.zeros((T, 4), bool)
    want[heirs, :2] = True            # (query heads 0, 1 share KV head 0)
    np.testing.assert_array_equal(is_nan, want)
    plain = dict(c, **{pool: clean})
    ref = orc.bf16_to_f64(unbits(launch(api, plain)["out"]))
    np.testing.assert_array_equal(got[~want], ref[~want])
    # hidden by a window from all rows, and from some
    depth = np.array(orc.depths(TREES[t]))
    for pos in (L - W - 3, L - W + 2, 10):
        c = dict(plain, **{pool: clean.copy()})
        nan_row(c, pool, 0, pos, 1, group=3)
        got = orc.bf16_to_f64(unbits(launch(api, c, window=W)["out"]))
        ref = orc.bf16_to_f64(unbits(launch(api, plain, window=W)["out"]))
        sees = np.zeros((T, 4), bool)
        sees[L + depth - pos < W, 2:] = True
        np.testing.assert_array_equal(np.isnan(got).any(2), sees)
        np.testing.assert_array_equal(got[~sees], ref[~sees])


@pytest.mark.parametrize("t,Hq,Hkv,page,L,window", [(0, 8, 2, 16, 37, 0), (2, 4, 2, 64, 300, 0), (2, 8, 2, 16, 700, 100),
                                                    (4, 8, 2, 16, 301, 0), (4, 16, 2, 64, 1000, 200), (0, 4, 4, 256, 0, 0)])
def test_bytes_that_no_row_sees(api, t, Hq, Hkv, page, L, window):
    """Slots behind the tree, before the window and of other pages hold any bytes, those of infinities and NaN included;
    the outputs are the same bits."""
    say("fp4 bytes unseen", t, Hq, Hkv, page, L, window)
    T, g = len(TREES[t]), np.random.default_rng(t + L)
    c = make(41, [t], [L], Hq, Hkv, page)
    seen = np.zeros((c["n_pages"], page), bool)
    for pos in range(max(0, L - window + 1) if window else 0, L + T):
        seen[c["table"][0, pos // page], pos % page] = True
    assert not seen.all()
    junk = dict(c)
    for pool in ("kp", "vp"):
        codes, scales = fo.planes(c[pool])
        codes, scales = codes.copy(), scales.copy()
        where = ~np.broadcast_to(seen[:, None], codes.shape[:3])
        codes[where] = g.integers(0, 256, codes[where].shape)
        scales[where] = g.choice([0, 1, 127, 252, 253, 254, 255], scales[where].shape)
        junk[pool] = fo.join(codes, scales)
    want, got = (unbits(launch(api, x, window=window)["out"]) for x in (c, junk))
    assert np.isfinite(orc.bf16_to_f64(want)).all()
    np.testing.assert_array_equal(got, want)


@pytest.mark.parametrize("t,Hq", [(0, 8), (2, 4), (4, 8)])
@pytest.mark.parametrize("byte", [253, 254])
def test_values_beyond_bf16(api, t, Hq, byte):
    """A group of values with a scale byte above 252 counts as no number, whatever its codes."""
    T = len(TREES[t])
    c = make(43, [t], [90], Hq, 2, 16)
    clean = unbits(launch(api, c)["out"])
    c["vp"] = c["vp"].copy()
    slot = c["table"][0, 33 // 16]
    c["vp"][slot, 1, (33 % 16) * 64:(33 % 16) * 64 + 64] = 0x11
    c["vp"][slot, 1, 16 * 64 + 4 * (33 % 16) + 2] = byte
    got = unbits(launch(api, c)["out"])
    assert np.isnan(orc.bf16_to_f64(got[:T, Hq // 2:])).all()
    np.testing.assert_array_equal(got[:, :Hq // 2], clean[:, :Hq // 2])


def test_large_and_small_scores(api):
    """Queries of very different sizes within a row, zeros, and one that is not finite."""
    c = make(33, [1, 1], [64, 500], 2, 1, 16)
    q = c["q"].copy()
    q[0] = 0
    q[1, :, ::3] = (q[1, :, ::3] & 0x807F) | (0x7F - 20 << 7)     # about 2^-20 beside ordinary ones
    q[2] = (q[2] & 0x807F) | 0x0100
    q[3] = (q[3] & 0x807F) | (0x7F + 3 << 7)
    c["q"] = q
    check(c, unbits(launch(api, c)["out"]))
    q = c["q"].copy()
    q[4, 0, 5] = 0x7F80
    got = orc.bf16_to_f64(unbits(launch(api, dict(c, q=q))["out"]))
    ref = orc.bf16_to_f64(unbits(launch(api, c)["out"]))
    assert np.isnan(got[4, 0]).all()
    got[4, 0] = ref[4, 0]
    np.testing.assert_array_equal(got, ref)


def test_two_streams_and_a_graph(api):
    """Captured on a stream of its own and replayed with other queries; a second graph shares the workspace, in order."""
    c = make(35, [2, 0], [700, 5000], 8, 2, 16)
    d = launch(api, c)
    graphs = []
    for k in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            d["plan_call"]()
            d["attend"]()
        graphs.append(g)
    rng = np.random.default_rng(1)
    for k in range(4):
        q = c["q"][rng.permutation(c["rows"])]
        d["q"].copy_(bits(q))
        d["out"].fill_(7)
        torch.cuda.synchronize()
        graphs[k % 2].replay()
        torch.cuda.synchronize()
        check(dict(c, q=q), unbits(d["out"]))
    side = torch.cuda.Stream()
    d["q"].copy_(bits(c["q"]))
    d["out"].fill_(7)
    torch.cuda.synchronize()
    d2 = launch(api, c, stream=side, run=False)
    torch.cuda.synchronize()
    d2["plan_call"]()
    d2["attend"]()
    side.synchronize()
    check(c, unbits(d2["out"]))
