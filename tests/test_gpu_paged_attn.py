"""GPU: tree attention over the page pool against 64 bits.

Per element the bound is the oracle's: roundings to bf16 are off by at most
2^-8 of the rounded value (weights, a split's partial, the rotated query, the
output), pushed through the softmax.  Over a whole output the roundings are
independent, each of root mean square at most 2^-8 / sqrt(3), and the four of
them (the query's as large as the others at these score spreads) add up in
squares to 2^-7 / sqrt(3): the 2-norm bound is 2^-7.
"""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import entmtp_oracle as orc  # noqa: E402
from oracle import paged_oracle as po  # noqa: E402
from paper_2606_27550_amd import synth  # noqa: E402
from tests.paged_helpers import TREES, bits, block_table, dev, host, i32, row_offsets, say, unbits  # noqa: E402

pytestmark = pytest.mark.gpu
D = 128
SCALE = 1 / math.sqrt(D)


@pytest.fixture(scope="module")
def api():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_27550_amd import api as _api
    return _api


def make(seed, topo, lens, Hq, Hkv, page, spare=3, behind=0):
    """Inputs of a batch as bf16 bits; topo -1: an unused place."""
    g = np.random.default_rng(seed)
    use = [t if 0 <= t < len(TREES) else 0 for t in topo]
    table, n_pages = block_table(g, use, [max(0, L) for L in lens], page, spare)
    off = row_offsets(topo)
    rows = int(off[-1]) + behind
    normal = lambda *s: synth.normal_bf16(g, s)   # noqa: E731
    c = dict(topo=np.asarray(topo, np.int32), lens=np.asarray(lens, np.int32), table=table, page=page, n_pages=n_pages,
             off=off, rows=rows, Hq=Hq, Hkv=Hkv, q=normal(rows, Hq, D), kt=normal(rows, Hkv, D), vt=normal(rows, Hkv, D),
             kp=normal(n_pages, Hkv, page, D), vp=normal(n_pages, Hkv, page, D), status=np.zeros(len(topo), np.int32),
             slots=np.full(rows, -1, np.int32))
    for b, (t, L) in enumerate(zip(topo, lens)):
        if not 0 <= t < len(TREES):
            c["status"][b] = po.NONE
            continue
        for i in range(len(TREES[t])):
            c["slots"][off[b] + i] = table[b, (L + i) // page] * page + (L + i) % page
    return c


def launch(api, c, theta=1e4, softcap=0.0, window=0, slopes=None, bank=None, stream=None, plan_window=None, run=True):
    B, rows = len(c["topo"]), c["rows"]
    d = {k: i32(c[k]) for k in ("topo", "lens", "table", "off", "status", "slots")}
    d.update({k: bits(c[k]) for k in ("q", "kt", "vt", "kp", "vp")})
    d["bank"] = bank or api.Bank(TREES)
    d["out"] = torch.full((rows, c["Hq"], D), 7.0, dtype=torch.bfloat16, device="cuda")
    d["bad"] = torch.full((B,), 9, dtype=torch.int32, device="cuda")
    d["slopes"] = None if slopes is None else dev(np.asarray(slopes, np.float32))
    shape = (rows, c["Hq"], c["Hkv"])
    mp = c["table"].shape[1]
    d["plan"] = torch.empty(api.tree_attn_paged_plan_bytes(d["bank"], B, *shape, mp, c["page"]), dtype=torch.uint8, device="cuda")
    ws = api.tree_attn_paged_workspace(d["bank"], B, *shape, D, mp, c["page"])
    d["ws"] = torch.empty(ws, dtype=torch.uint8, device="cuda") if ws else None

    def plan():
        api.tree_attn_paged_plan(d["bank"], d["topo"], d["lens"], d["off"], d["status"], d["table"], c["page"], c["n_pages"],
                                 *shape, d["plan"], window=window if plan_window is None else plan_window, bad=d["bad"],
                                 stream=stream)

    def attend():
        api.tree_attn_paged(d["bank"], d["plan"], d["q"], d["kt"], d["vt"], d["kp"], d["vp"], d["table"], d["slots"], SCALE,
                            theta, d["out"], d["ws"], softcap=softcap, window=window, slopes=d["slopes"], stream=stream)
    d["plan_call"], d["attend"] = plan, attend
    if run:
        plan()
        attend()
        torch.cuda.synchronize()
    return d


def check(c, d, idle=(), theta=1e4, softcap=0.0, window=0, slopes=None):
    """Every sequence against the oracle; those in idle (and rows of none) untouched."""
    out = unbits(d["out"])
    got = orc.bf16_to_f64(out)
    kp, vp = c["kp"].copy(), c["vp"].copy()
    left = np.ones(c["rows"], bool)
    page, e2, n2 = c["page"], 0.0, 0.0
    for b, (t, L) in enumerate(zip(c["topo"], c["lens"])):
        if not 0 <= t < len(TREES) or b in idle:
            continue
        T, r0 = len(TREES[t]), int(c["off"][b])
        r = slice(r0, r0 + T)
        ref, keys, off = po.tree_attention_paged(c["q"][r], c["kt"][r], c["vt"][r], c["kp"], c["vp"], c["table"][b], int(L),
                                                 TREES[t], SCALE, theta, softcap, window, slopes)
        err = np.abs(got[r] - ref)
        assert (err <= off).all(), (b, t, L, float((err / off).max()))
        e2 += float((err ** 2).sum())
        n2 += float((ref ** 2).sum())
        left[r] = False
        for i in range(T):
            s = c["slots"][r0 + i]
            kp[s // page, :, s % page], vp[s // page, :, s % page] = keys[i], c["vt"][r0 + i]
    assert e2 <= (2.0 ** -7) ** 2 * n2, math.sqrt(e2 / n2)
    assert (out[left] == 0x40E0).all()
    np.testing.assert_array_equal(unbits(d["kp"]), kp)
    np.testing.assert_array_equal(unbits(d["vp"]), vp)


CASES = [
    ([0], [0], 1, 1, 16), ([0], [1], 4, 1, 16), ([0], [15], 8, 8, 16), ([1], [16], 8, 2, 16), ([1], [31], 4, 4, 32),
    ([2], [32], 8, 2, 32), ([2], [33], 8, 1, 64), ([3], [0], 2, 2, 16), ([4], [63], 8, 2, 16), ([5], [100], 8, 2, 128),
    ([6], [130], 4, 1, 16), ([0], [400], 8, 2, 16), ([2], [353], 8, 2, 16), ([4], [1000], 8, 2, 64), ([0], [6001], 4, 2, 16),
    ([5], [700], 8, 1, 256), ([2], [5000], 32, 1, 16), ([6], [2047], 2, 2, 32),
    ([0, 1, 2, 3, 4, 5, 6], [17, 0, 300, 64, 900, 5, 1500], 8, 2, 16),
    ([0] * 40, [(37 * i) % 700 for i in range(40)], 8, 4, 32),
    ([1, -1, 2, 99, 0], [40, 0, 70, 10, 800], 8, 2, 16)]


@pytest.mark.parametrize("topo,lens,Hq,Hkv,page", CASES)
def test_against_64_bits(api, topo, lens, Hq, Hkv, page):
    say("tree_attn_paged", topo, lens, Hq, Hkv, page)
    c = make(len(topo) + lens[0], topo, lens, Hq, Hkv, page, behind=2)
    d = launch(api, c)
    assert (host(d["bad"]) == 0).all()
    check(c, d)


OPTIONS = [dict(softcap=3.0), dict(softcap=1024.0), dict(softcap=0.01), dict(window=1), dict(window=2),
           dict(window=5), dict(window=33), dict(window=64), dict(window=500), dict(window=2 ** 31 - 1),
           dict(slopes=True), dict(softcap=30.0, window=40), dict(softcap=2.0, window=100, slopes=True),
           dict(theta=0.0), dict(theta=0.0, softcap=5.0, window=7), dict(theta=0.5), dict(theta=0.5, window=90)]


@pytest.mark.parametrize("opt", OPTIONS)
def test_caps_windows_and_biases(api, opt):
    opt = dict(opt)
    topo, lens, Hq = [2, 0, 6, 1, 4], [50, 1000, 31, 0, 640], 8
    c = make(77, topo, lens, Hq, 2, 16)
    if opt.get("slopes"):
        opt["slopes"] = np.float32(0.5) ** np.arange(1, Hq + 1)
    say("tree_attn_paged", opt)
    check(c, launch(api, c, **opt), **opt)


def test_many_sequences(api):
    """256 sequences, the most a call takes, decoding token by token."""
    g = np.random.default_rng(8)
    topo = [int(t) for t in g.choice([0, 0, 0, 1, -1], 256)]
    lens = [int(n) for n in g.integers(0, 200, 256)]
    lens[17] = 3000
    topo[17] = 0
    c = make(8, topo, lens, 4, 2, 16, behind=5)
    say("tree_attn_paged 256 sequences")
    check(c, launch(api, c))


def test_equals_the_dense_attention(api):
    """The same keys and values in a dense cache give the same output (other splits: within two roundings)."""
    for t, L, Hq, Hkv, page in ((2, 300, 8, 2, 16), (4, 2000, 16, 16, 64), (5, 31, 8, 2, 256)):
        c = make(t, [t], [L], Hq, Hkv, page)
        d = launch(api, c)
        T = len(TREES[t])
        n = -(-(L + T) // page)
        flat = lambda p: bits(np.concatenate([c[p][k] for k in c["table"][0, :n]], axis=1))   # noqa: E731
        kc, vc = flat("kp"), flat("vp")
        out = torch.empty_like(d["out"])
        ws = torch.empty(api.tree_attn_workspace(T, Hq, Hkv, D, L), dtype=torch.uint8, device="cuda")
        api.tree_attn(d["bank"], t, d["q"], d["kt"], d["vt"], kc, vc, L, SCALE, 1e4, out, ws)
        x, y = out.double(), d["out"].double()
        assert float((x - y).norm() / x.norm()) <= 2.0 ** -7
        got = torch.cat([d["kp"][int(k)] for k in c["table"][0, :n]], dim=1)
        np.testing.assert_array_equal(unbits(got)[:, :L + T], unbits(kc)[:, :L + T])


def test_shared_prefix_pages(api):
    """Four sequences whose prefixes lie in the same pages."""
    c = make(9, [2, 1, 2, 0], [64, 64, 64, 48], 8, 2, 16)
    c["table"][1:, :3] = c["table"][0, :3]
    c["table"][1:3, 3] = c["table"][0, 3]
    check(c, launch(api, c))


def test_sequences_that_cannot_run_are_left_alone(api):
    """A status, a prefix page outside the pool, rows that do not fit: no output, no append; the others run."""
    c = make(10, [2, 1, 2, 0, 4, 1, 0], [100, 50, 40, 33, 500, 20, 90], 8, 2, 16)
    c["status"][1] = po.FULL
    c["table"][2, 1] = -1
    c["table"][4, 20] = c["n_pages"]
    c["off"] = c["off"].copy()
    d = launch(api, c)
    assert host(d["bad"]).tolist() == [0, 0, 1, 0, 1, 0, 0]
    check(c, d, idle=(1, 2, 4))
    # lengths and trees that fit nothing, row ranges shorter than the tree
    for k, b, v in (("lens", 0, -1), ("lens", 0, 2 ** 31 - 1), ("lens", 0, c["table"].shape[1] * 16 - 25), ("topo", 0, 99),
                    ("topo", 0, -2 ** 31), ("off", 1, 25), ("off", 0, -1), ("off", 0, 2 ** 31 - 1)):
        e = dict(c, **{k: c[k].copy()})
        e[k][b] = v
        d = launch(api, e)
        assert (unbits(d["out"])[:26] == 0x40E0).all(), (k, v)
        e = dict(c, topo=c["topo"].copy())
        e["topo"][0] = -1
        e["lens"] = np.maximum(c["lens"], 0)
        check(e, d, idle=(1, 2, 4))


def test_a_page_that_goes_after_the_plan_reads_as_zeros(api):
    """(In bounds whatever the table says when the attention runs.)"""
    c = make(11, [2], [200], 8, 2, 16)
    d = launch(api, c, run=False)
    d["plan_call"]()
    d["table"][0, 3] = -7
    d["table"][0, 4] = 2 ** 31 - 1
    d["attend"]()
    for k in ("kp", "vp"):
        c[k][c["table"][0, [3, 4]]] = 0
        d[k][torch.from_numpy(c["table"][0, [3, 4]]).long().cuda()] = 0
    check(c, d)


def test_slots_outside_the_pool_are_not_written(api):
    c = make(12, [2], [60], 8, 2, 16)
    d = launch(api, c, run=False)
    d["plan_call"]()
    d["slots"][4] = -1
    d["slots"][5] = c["n_pages"] * 16
    d["slots"][6] = 2 ** 31 - 1
    d["attend"]()
    keep = c["slots"].copy()
    for p in ("kp", "vp"):
        for i in (4, 5, 6):
            s = keep[i]
            np.testing.assert_array_equal(unbits(d[p])[s // 16, :, s % 16], c[p][s // 16, :, s % 16])
    for p, src in (("kp", None), ("vp", "vt")):
        if src:
            s = keep[7]
            np.testing.assert_array_equal(unbits(d[p])[s // 16, :, s % 16], c[src][7])


def test_a_plan_of_something_else_does_nothing(api):
    c = make(13, [2, 1], [100, 90], 8, 2, 16)
    for kw in (dict(plan_window=50), dict(window=50, plan_window=0)):
        d = launch(api, c, **kw)
        assert (unbits(d["out"]) == 0x40E0).all()
        np.testing.assert_array_equal(unbits(d["kp"]), c["kp"])
    d = launch(api, c, run=False)
    d["plan"].zero_()
    d["attend"]()
    assert (unbits(d["out"]) == 0x40E0).all()
    other = api.Bank(TREES)
    d["plan_call"]()
    api.tree_attn_paged(other, d["plan"], d["q"], d["kt"], d["vt"], d["kp"], d["vp"], d["table"], d["slots"], SCALE, 1e4,
                        d["out"], d["ws"])
    assert (unbits(d["out"]) == 0x40E0).all()


def test_pages_before_the_window_may_be_gone(api):
    """Entries wholly before the root's window are missing, and the slots there hold NaN."""
    for window, L in ((40, 300), (16, 77), (33, 64), (500, 2000), (3, 400)):
        c = make(window, [2, 0], [L, L + 5], 8, 2, 16)
        for b, n in enumerate((L, L + 5)):
            first = n + 1 - window
            gone = first // 16
            c["kp"][c["table"][b, :gone]] = 0x7FC0
            c["vp"][c["table"][b, :gone]] = 0x7F80
            c["kp"][c["table"][b, gone], :, :first % 16] = 0x7FC0     # the part of a held page before it
            c["vp"][c["table"][b, gone], :, :first % 16] = 0x7FC0
            c["table"][b, :gone] = [-1, c["n_pages"], 2 ** 31 - 1, -2 ** 31][b % 4]
        d = launch(api, c, window=window)
        assert (host(d["bad"]) == 0).all()
        # (the oracle takes a product with what it does not see out of the sum)
        e = dict(c, kp=np.where((c["kp"] & 0x7F80) == 0x7F80, 0, c["kp"]).astype(np.uint16),
                 vp=np.where((c["vp"] & 0x7F80) == 0x7F80, 0, c["vp"]).astype(np.uint16), table=np.where(
                     (c["table"] < 0) | (c["table"] >= c["n_pages"]), 0, c["table"]))
        kp, vp = unbits(d["kp"]), unbits(d["vp"])
        d["kp"], d["vp"] = (bits(np.where((x & 0x7F80) == 0x7F80, 0, x).astype(np.uint16)) for x in (kp, vp))
        check(e, d, window=window)


@pytest.mark.parametrize("bad", [0x7FC0, 0x7F80, 0xFF80])
@pytest.mark.parametrize("which", ["vt", "kt"])
def test_what_is_not_finite_reaches_the_rows_that_see_it(api, bad, which):
    """A node's key or value that is NaN or infinite: its descendants' rows show it, nothing else does."""
    t, L = 4, 45
    c = make(14, [t, 1], [L, 20], 8, 2, 16)
    node = 5
    sees = [node in orc.ancestors_or_self(TREES[t], i) for i in range(len(TREES[t]))]
    assert any(sees) and not all(sees)
    clean = launch(api, c)
    c[which] = c[which].copy()
    c[which][node, :, 9] = bad
    d = launch(api, c)
    got, ref = d["out"].float().cpu().numpy(), clean["out"].float().cpu().numpy()
    hidden = ~np.array(sees)
    np.testing.assert_array_equal(got[:64][hidden], ref[:64][hidden])
    np.testing.assert_array_equal(got[64:], ref[64:])
    if which == "vt":
        assert np.isnan(got[:64][np.array(sees)]).all()
    elif bad == 0x7FC0:
        assert np.isnan(got[:64][np.array(sees)]).all()
    s = c["slots"][node]
    assert (unbits(d["vp" if which == "vt" else "kp"])[s // 16, :, s % 16, 9] != c["vp" if which == "vt" else "kp"][
        s // 16, :, s % 16, 9]).any()


@pytest.mark.parametrize("bad", [0x7FC0, 0x7F80, 0xFF80])
@pytest.mark.parametrize("which", ["vp", "kp"])
def test_what_is_not_finite_at_the_windows_edge(api, bad, which):
    """A prefix key or value within the root's window and before its descendants': only rows that see it show it."""
    t, L, window = 4, 700, 300
    depth = orc.depths(TREES[t])
    for pos in (L + 1 - window, L + 2 - window, L + int(max(depth)) - window):
        c = make(22, [t, 1], [L, 20], 8, 2, 16)
        sees = np.array([L + d - pos < window for d in depth])
        assert sees.any() and not sees.all()
        clean = launch(api, c, window=window)
        c[which] = c[which].copy()
        c[which][c["table"][0, pos // 16], :, pos % 16, 9] = bad
        d = launch(api, c, window=window)
        got, ref = d["out"].float().cpu().numpy(), clean["out"].float().cpu().numpy()
        np.testing.assert_array_equal(got[:64][~sees], ref[:64][~sees])
        np.testing.assert_array_equal(got[64:], ref[64:])
        if which == "vp" or bad == 0x7FC0:
            assert np.isnan(got[:64][sees]).all()


@pytest.mark.parametrize("t,Hq,Hkv,L", [(2, 32, 8, 5000), (4, 32, 8, 1500), (0, 8, 8, 3333)])
def test_an_infinite_value_of_the_prefix_is_one_in_its_column(api, t, Hq, Hkv, L):
    """Also from the last of a prefix's splits, and however many heads a merge takes."""
    c = make(27, [t], [L], Hq, Hkv, 16)
    clean = launch(api, c)["out"].float().cpu().numpy()
    for pos in (3, L - 40):
        e = dict(c, vp=c["vp"].copy())
        e["vp"][c["table"][0, pos // 16], 0, pos % 16, 9] = 0x7F80
        got = launch(api, e)["out"].float().cpu().numpy()
        G = Hq // Hkv
        assert np.isposinf(got[:, :G, 9]).all()
        got[:, :G, 9] = clean[:, :G, 9]
        np.testing.assert_array_equal(got, clean)


def test_streams_graphs_and_two_at_once(api):
    """A captured plan and attention follow the lengths they find; two batches on two streams, each with its workspace."""
    c = make(15, [2, 0, 1, 4], [0, 0, 0, 0], 8, 2, 16)
    mp = 60
    g = np.random.default_rng(15)
    c["n_pages"] = 4 * mp
    c["table"] = g.permutation(4 * mp).reshape(4, mp).astype(np.int32)
    c["kp"], c["vp"] = (synth.normal_bf16(g, (4 * mp, 2, 16, D)) for _ in range(2))
    d = launch(api, c, run=False)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        d["plan_call"]()
        d["attend"]()
    for lens in ([0, 0, 0, 0], [100, 3, 17, 500], [800, 850, 3, 64], [16, 32, 48, 31]):
        now = dict(c, lens=np.array(lens, np.int32), kp=unbits(d["kp"]).copy(), vp=unbits(d["vp"]).copy(),
                   slots=c["slots"].copy())
        for b, L in enumerate(lens):
            for i in range(len(TREES[c["topo"][b]])):
                now["slots"][c["off"][b] + i] = c["table"][b, (L + i) // 16] * 16 + (L + i) % 16
        d["lens"].copy_(i32(lens))
        d["slots"].copy_(i32(now["slots"]))
        d["out"].fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        check(now, d)
    one, two = make(16, [4, 2], [900, 300], 8, 2, 16), make(17, [5, 0], [400, 2000], 8, 4, 32)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    a, b = launch(api, one, stream=s1, run=False), launch(api, two, stream=s2, window=300, run=False)
    torch.cuda.synchronize()
    for _ in range(3):
        for x in (a, b):
            x["plan_call"]()
            x["attend"]()
    torch.cuda.synchronize()
    check(one, a)
    check(two, b, window=300)


def test_two_graphs_of_one_workspace(api):
    """Two captured batches share a workspace and replay in turn, an eager call of a third between them."""
    cs = [make(24, [4, 2], [900, 300], 8, 2, 16), make(25, [5, 0, 1], [400, 2000, 0], 8, 4, 32), make(26, [6], [3000], 4, 2, 64)]
    ds = [launch(api, c, run=False) for c in cs]
    ws = torch.empty(max(d["ws"].numel() for d in ds), dtype=torch.uint8, device="cuda")
    graphs = []
    for d in ds:
        d["ws"] = ws
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            d["plan_call"]()
            d["attend"]()
    for order in ((0, 1, 1, 0), (1, 0, 0, 1)):
        for d in ds:
            d["out"].fill_(7)
        for k in order:
            graphs[k].replay()
            ds[2]["plan_call"]()
            ds[2]["attend"]()
        torch.cuda.synchronize()
        for c, d in zip(cs, ds):
            check(c, d)


def test_results_do_not_depend_on_the_run(api):
    c = make(18, [4, 2, 0, 5], [900, 30, 5000, 111], 8, 2, 16)
    ref = unbits(launch(api, c)["out"])
    for _ in range(3):
        np.testing.assert_array_equal(unbits(launch(api, c)["out"]), ref)


def test_offsets_past_32_bits(api):
    """A pool of more than 2^32 bytes and 2^31 elements a side, pages at its end."""
    Hkv, page = 8, 256
    n_pages = 2 ** 31 // (Hkv * page * D) + 40
    c = make(19, [2, 0], [600, 5000], 16, Hkv, page)
    d = launch(api, c, run=False)
    big = {}
    for k in ("kp", "vp"):
        big[k] = torch.empty((n_pages, Hkv, page, D), dtype=torch.bfloat16, device="cuda")
        big[k][-c["n_pages"]:] = d[k]
    shift = n_pages - c["n_pages"]
    table = torch.where(d["table"] >= 0, d["table"] + shift, d["table"])
    slots = d["slots"] + shift * page
    api.tree_attn_paged_plan(d["bank"], d["topo"], d["lens"], d["off"], d["status"], table, page, n_pages, c["rows"], 16, Hkv,
                             d["plan"])
    api.tree_attn_paged(d["bank"], d["plan"], d["q"], d["kt"], d["vt"], big["kp"], big["vp"], table, slots, SCALE, 1e4, d["out"],
                        d["ws"])
    for k in ("kp", "vp"):
        d[k] = big[k][-c["n_pages"]:]
    check(c, d)
    # and its compaction
    path, a = i32([[0, 3, 7, 9, 25], [0, -1, -1, -1, -1]]), i32([4, 0])
    want = {k: po.kv_compact_paged(unbits(d[k])[None].copy(), host(path), host(a), c["off"], c["slots"])[0] for k in big}
    api.kv_compact_paged(path, a, d["off"], slots, big["kp"], big["vp"])
    for k in big:
        np.testing.assert_array_equal(unbits(big[k][-c["n_pages"]:]), want[k])


def test_positions_near_31_bits(api):
    """With a window and no rotation a sequence far along gives what it gives early on; so do its slots."""
    c = make(23, [2], [700], 8, 2, 256)
    T, window = len(TREES[2]), 300
    near = launch(api, c, theta=0.0, window=window)
    pages = (2 ** 31 - 1 - 1024) // 256      # the most there may be
    shift = pages - 4                        # (the tree lies in pages 2 .. 3 of the table)
    table = torch.full((1, pages), -1, dtype=torch.int32, device="cuda")
    table[0, shift:shift + 3] = i32(c["table"][0, :3])
    d = launch(api, c, run=False)
    L, bank = i32([700 + 256 * shift]), d["bank"]
    off, slots, status = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (2, T, 1))
    say("tree_attn_paged at position", int(L))
    api.page_map(bank, d["topo"], L, table, 256, c["n_pages"], off, slots, status)
    assert host(status)[0] == po.OK
    np.testing.assert_array_equal(host(slots), c["slots"])
    shape = (T, 8, 2)
    plan = torch.empty(api.tree_attn_paged_plan_bytes(bank, 1, *shape, pages, 256), dtype=torch.uint8, device="cuda")
    ws = torch.empty(api.tree_attn_paged_workspace(bank, 1, *shape, D, pages, 256), dtype=torch.uint8, device="cuda")
    api.tree_attn_paged_plan(bank, d["topo"], L, off, status, table, 256, c["n_pages"], *shape, plan, window=window,
                             bad=d["bad"])
    api.tree_attn_paged(bank, plan, d["q"], d["kt"], d["vt"], d["kp"], d["vp"], table, slots, SCALE, 0.0, d["out"], ws,
                        window=window)
    assert host(d["bad"])[0] == 0
    for k in ("out", "kp", "vp"):
        np.testing.assert_array_equal(unbits(d[k]), unbits(near[k]))
    # every position there can be, in one page: the work list's ranges (the attention is not run)
    table.zero_()
    api.tree_attn_paged_plan(bank, d["topo"], L, off, status, table, 256, 1, *shape, plan, bad=d["bad"])
    assert host(d["bad"])[0] == 0


def test_refusals(api):
    c = make(20, [1], [20], 8, 2, 16)
    d = launch(api, c)
    ok = (d["bank"], d["plan"], d["q"], d["kt"], d["vt"], d["kp"], d["vp"], d["table"], d["slots"], SCALE, 1e4, d["out"], d["ws"])
    for at, bad in ((2, d["q"].float()), (2, d["q"].transpose(0, 1)), (3, d["kt"][:-1]), (5, d["kp"][0]), (6, d["vp"][:-1]),
                    (7, d["table"].long()), (8, d["slots"][:-1]), (11, d["out"][:-1]), (12, d["table"].cpu()), (1, None)):
        args = list(ok)
        args[at] = bad
        with pytest.raises(ValueError):
            api.tree_attn_paged(*args)
    with pytest.raises(ValueError):
        api.tree_attn_paged(*ok, slopes=torch.zeros(4, device="cuda"))
    args = list(ok)
    args[1] = d["plan"][:64]
    with pytest.raises(api.EntmtpError):
        api.tree_attn_paged(*args)
    long = make(21, [1], [900], 8, 2, 16)
    e = launch(api, long)
    args = [e["bank"], e["plan"], e["q"], e["kt"], e["vt"], e["kp"], e["vp"], e["table"], e["slots"], SCALE, 1e4, e["out"], None]
    with pytest.raises(api.EntmtpError):
        api.tree_attn_paged(*args)
