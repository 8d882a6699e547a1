"""GPU: sequences that a step could not serve -- no free page, a page outside the
pool, a length that does not fit -- in a captured step of 20 sequences (two
calls of the acceptance): nothing of theirs changes, nothing is accepted for
them, and the step that finds them mended is the oracle's."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import entmtp_oracle as orc  # noqa: E402
from oracle import paged_oracle as po  # noqa: E402
from paper_2606_27550_amd import synth  # noqa: E402
from tests.paged_helpers import TREES, bits, dev, host, i32, row_offsets, say, unbits  # noqa: E402
from tests.test_gpu_logit_adjust import U  # noqa: E402

pytestmark = pytest.mark.gpu
D, SCALE, THETA = 128, 1 / math.sqrt(128), 1e4


@pytest.fixture(scope="module")
def api():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_27550_amd import api as _api
    return _api


def test_the_plans_trees(api):
    """topo[b] where a sequence has work, -1 elsewhere; a plan made from another's trees has no more work than that one."""
    bank, page, n_pages = api.Bank(TREES), 16, 40
    topo = [2, 1, -1, 99, 0, 1, 2, 0]
    lens = [40, 20, 0, 0, 100, -3, 7, 64]
    B, off = len(topo), row_offsets(topo)
    table = np.full((B, 12), -1, np.int32)
    for b in range(B):
        table[b, :9] = np.arange(9) + 2 * b
    table[0, 1] = -1                       # a prefix page is missing
    table[4, 0] = n_pages                  # and one outside the pool, behind a window of 40
    status = [0, 0, 1, 1, 0, 2, 3, 0]
    args = [i32(x) for x in (lens, off, status, table)]
    rows = int(off[-1])
    plan, other = (torch.empty(api.tree_attn_paged_plan_bytes(bank, B, rows, 8, 2, 12, page), dtype=torch.uint8, device="cuda")
                   for _ in range(2))
    run, second = api.tree_attn_paged_topo(plan, B), api.tree_attn_paged_topo(other, B)
    bad = i32([9] * B)
    say("tree_attn_paged_plan of unmapped sequences")
    api.tree_attn_paged_plan(bank, i32(topo), *args, page, n_pages, rows, 8, 2, plan, bad=bad)
    assert host(bad).tolist() == [1, 0, 0, 0, 1, 0, 0, 0]
    assert host(run).tolist() == [-1, 1, -1, -1, -1, -1, -1, 0]
    api.tree_attn_paged_plan(bank, i32(topo), *args, page, n_pages, rows, 8, 2, other, window=40)
    assert host(second).tolist() == [-1, 1, -1, -1, 0, -1, -1, 0]
    api.tree_attn_paged_plan(bank, run, *args, page, n_pages, rows, 8, 2, other, window=40)
    assert host(second).tolist() == [-1, 1, -1, -1, -1, -1, -1, 0]
    with pytest.raises(api.EntmtpError):
        api.tree_attn_paged_plan(bank, second, *args, page, n_pages, rows, 8, 2, other, window=40)


def test_steps_with_unmapped_sequences(api):
    g = np.random.default_rng(61)
    B, Hq, Hkv, page, layers, V, hid, window, cap_path = 20, 4, 2, 16, 2, 149, 64, 24, 32
    max_pages, n_pages, rows = 12, 120, 240
    topo = np.array([1, 0, 2, 1, 1, 2, 0, 1, 0, -1, 1, 2, 0, 1, 1, 0, 2, 1, 0, 2], np.int32)
    lens = np.array([20, 5, 31, 46, 0, 100, 33, 12, 17, 0, 64, 40, 3, 9, 80, 16, 30, 30, 48, 48], np.int32)
    T = [len(TREES[t]) if t >= 0 else 0 for t in topo]
    assert sum(T) <= rows
    bank = api.Bank(TREES)
    table, used = np.full((B, max_pages), -1, np.int32), 0
    for b, L in enumerate(lens):
        n = -(-int(L) // page)
        table[b, :n] = np.arange(used, used + n)
        used += n
    # what keeps a sequence from being mapped, and what mends it before the second step
    mended_table, mended_lens = table.copy(), lens.copy()
    table[5, 1] = -1                                  # a prefix page gone (only the list without a window reads it)
    table[14, 0] = n_pages                            # a prefix page outside the pool, likewise
    table[17, 1] = n_pages + 7                        # the tree's first page outside the pool
    table[11, 2] = -1                                 # the page that holds the prefix's last slots
    lens[7] = -1
    lens[13] = max_pages * page - 3
    # the stack: enough for the others up to sequence 18, none for 19
    _, _, _, status, left = po.page_map(TREES, topo, lens, table, page, n_pages, rows, np.arange(used, n_pages, dtype=np.int32),
                                        n_pages - used)
    assert status[19] == po.OK and left >= 0
    need19 = -(-(48 + T[19]) // page) - 3
    free = g.permutation(np.arange(used, n_pages)).astype(np.int32)
    first = n_pages - used - left - need19            # pages the others take
    stack = np.concatenate([free[first + 1:], free[:first + 1]]).astype(np.int32)   # (its top is the end)
    n_free = first + 1                                # one left over, sequence 19 needs two
    assert need19 == 2 and stack.size >= n_free
    low = np.zeros_like(stack)
    low[:n_free] = stack[-n_free:]
    unmapped = {5: po.OK, 7: po.RANGE, 11: po.BAD, 13: po.RANGE, 14: po.OK, 17: po.BAD, 19: po.FULL}
    pools = [synth.normal_bf16(g, (layers, n_pages, Hkv, page, D)) for _ in range(2)]
    history = g.integers(0, 3, (B, V)).astype(np.int32)
    w = synth.lm_head_weight(61, V, hid, std=0.3)
    params = np.stack([1 + g.random(B) * 0.3, g.random(B) * 0.2, g.random(B) * 0.2, 0.5 + g.random(B)], 1).astype(np.float32)
    z = lambda *s, dt=torch.int32: torch.zeros(s, dtype=dt, device="cuda")   # noqa: E731
    bf, f32 = torch.bfloat16, torch.float32
    d = dict(topo=i32(topo), lens=i32(lens), table=i32(table), free=i32(low), n=i32([n_free]), off=z(B + 1), slots=z(rows),
             status=z(B), bad=z(B), kp=bits(pools[0]), vp=bits(pools[1]), history=i32(history), w=bits(w), params=dev(params),
             tok=z(rows), q=z(layers, rows, Hq, D, dt=bf), kt=z(layers, rows, Hkv, D, dt=bf), vt=z(layers, rows, Hkv, D, dt=bf),
             out=z(layers, rows, Hq, D, dt=bf), x=z(rows, hid, dt=bf), z=z(rows, V, dt=f32), H=z(rows, dt=f32),
             p1=z(rows, dt=f32), am=z(rows), a=z(B), path=z(B, cap_path), bonus=z(B), best=z(B, dt=f32), adj=z(rows, V, dt=f32))
    byte = lambda n: torch.empty(max(n, 64), dtype=torch.uint8, device="cuda")   # noqa: E731
    shape = (rows, Hq, Hkv)
    plans = [byte(api.tree_attn_paged_plan_bytes(bank, B, *shape, max_pages, page)) for _ in range(2)]
    runs = [api.tree_attn_paged_topo(p, B) for p in plans]
    ws = byte(api.tree_attn_paged_workspace(bank, B, *shape, D, max_pages, page))
    aws = byte(api.logit_adjust_workspace(rows, V))

    def step():
        api.page_map(bank, d["topo"], d["lens"], d["table"], page, n_pages, d["off"], d["slots"], d["status"], d["free"], d["n"])
        for plan, of, win, bad in zip(plans, (d["topo"], runs[0]), (0, window), (d["bad"], None)):
            api.tree_attn_paged_plan(bank, of, d["lens"], d["off"], d["status"], d["table"], page, n_pages, *shape, plan,
                                     window=win, bad=bad)
        for layer, win in ((0, 0), (1, window)):
            api.tree_attn_paged(bank, plans[layer], d["q"][layer], d["kt"][layer], d["vt"][layer], d["kp"][layer], d["vp"][layer],
                                d["table"], d["slots"], SCALE, THETA, d["out"][layer], ws, window=win)
        run = runs[-1]
        api.verify_logits(d["x"], d["w"], d["z"])
        api.logit_adjust(bank, run, d["off"], d["tok"], d["z"], d["params"], d["adj"], d["H"], d["p1"], d["am"], aws,
                         history=d["history"])
        for k in range(0, B, 16):
            e = min(B, k + 16)
            api.accept_batched_device(bank, run[k:e], d["off"][k:e + 1], d["tok"], d["am"], d["p1"], d["a"][k:e], d["path"][k:e],
                                      d["bonus"][k:e], d["best"][k:e])
        api.kv_compact_paged(d["path"], d["a"], d["off"], d["slots"], d["kp"], d["vp"])
        api.token_history_accept(d["off"], d["tok"], d["path"], d["a"], d["bonus"], d["history"])
        d["lens"].add_(d["a"] + 1)

    def fill():
        s = dict(q=synth.normal_bf16(g, (layers, rows, Hq, D)), kt=synth.normal_bf16(g, (layers, rows, Hkv, D)),
                 vt=synth.normal_bf16(g, (layers, rows, Hkv, D)), x=synth.normal_bf16(g, (rows, hid)),
                 tok=g.integers(0, V, rows).astype(np.int32))
        raw, r0 = orc.verify_logits(s["x"], w), 0
        for b, t in enumerate(topo):
            for i in range(1, T[b]):
                if g.random() < 0.7:
                    p = TREES[t][i]
                    y = po.adjusted_row(raw[r0 + p], TREES[t], p, s["tok"][r0:r0 + T[b]], params[b], history[b], None, None)
                    s["tok"][r0 + i] = int(np.argmax(y))
            r0 += T[b]
        for k in ("q", "kt", "vt", "x"):
            d[k].copy_(bits(s[k]))
        d["tok"].copy_(i32(s["tok"]))
        for k in ("out", "adj", "H", "p1", "am", "a", "bonus"):
            d[k].fill_(7)
        return s

    def reset(tab, ln, stack_now, n_now):
        for k, v in (("lens", ln), ("table", tab), ("n", [n_now]), ("free", stack_now)):
            d[k].copy_(i32(v))

    step()          # (the first calls, eager)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    reset(table, lens, low, n_free)
    d["history"].copy_(i32(history))
    for k, src in (("kp", pools[0]), ("vp", pools[1])):
        d[k].copy_(bits(src))
    accepted = 0
    for n in range(4):
        idle = set(unmapped) if n == 0 else set()
        s = fill()
        torch.cuda.synchronize()
        say("serving step", n, "lens", lens.tolist(), "unmapped", sorted(idle))
        graph.replay()
        torch.cuda.synchronize()
        table, row_off, slots, status, n_free = po.page_map(TREES, topo, lens, table, page, n_pages, rows, low, n_free)
        assert {b: status[b] for b in idle} == {b: unmapped[b] for b in idle}
        assert all(status[b] == (po.OK if topo[b] >= 0 else po.NONE) for b in range(B) if b not in idle)
        assert host(d["bad"]).tolist() == [int(n == 0 and b in (5, 14)) for b in range(B)]
        for k, want in (("table", table), ("off", row_off), ("status", status)):
            np.testing.assert_array_equal(host(d[k]), want)
        np.testing.assert_array_equal(host(d["slots"])[:slots.size], slots)
        assert int(d["n"]) == n_free
        out, adj, am, zl, H = (host(d[k]) if k != "out" else orc.bf16_to_f64(unbits(d[k])) for k in ("out", "adj", "am", "z", "H"))
        a, path = np.full(B, -1, np.int32), np.full((B, cap_path), -1, np.int32)
        bonus = np.full(B, -1, np.int32)
        for b, t in enumerate(topo):
            if t < 0:
                continue
            r = slice(int(row_off[b]), int(row_off[b + 1]))
            if b in idle:      # nothing of its rows is written
                assert (out[:, r] == 7).all() and (adj[r] == 7).all() and (am[r] == 7).all() and (H[r] == 7).all()
                continue
            for layer, win in ((0, 0), (1, window)):
                ref, keys, tol = po.tree_attention_paged(s["q"][layer][r], s["kt"][layer][r], s["vt"][layer][r], pools[0][layer],
                                                         pools[1][layer], table[b], int(lens[b]), TREES[t], SCALE, THETA, 0.0, win)
                assert (np.abs(out[layer][r] - ref) <= tol).all(), (n, b, layer)
                for i in range(T[b]):
                    sl = slots[r.start + i]
                    pools[0][layer, sl // page, :, sl % page] = keys[i]
                    pools[1][layer, sl // page, :, sl % page] = s["vt"][layer][r.start + i]
            for i in range(T[b]):
                y = po.adjusted_row(zl[r.start + i], TREES[t], i, s["tok"][r], params[b], history[b], None, None)
                got = adj[r.start + i].astype(np.float64)
                assert (np.abs(got - y) <= 5 * U * (np.abs(y) + 40)).all()
                assert am[r.start + i] == np.argmax(got)
            a[b], chain, bonus[b], _ = orc.accept(TREES[t], s["tok"][r], am[r])
            path[b, :len(chain)] = chain
        np.testing.assert_array_equal(host(d["a"]), a)
        np.testing.assert_array_equal(host(d["bonus"]), bonus)
        for k, pool in (("kp", 0), ("vp", 1)):
            pools[pool] = po.kv_compact_paged(pools[pool], path, a, row_off, slots)
            np.testing.assert_array_equal(unbits(d[k]), pools[pool])
        history = po.history_accept(history, row_off, s["tok"], path, a, bonus)
        np.testing.assert_array_equal(host(d["history"]), history)
        lens = lens + a + 1
        np.testing.assert_array_equal(host(d["lens"]), lens)
        accepted += int(a[a > 0].sum())
        if n == 0:
            assert all(a[b] == -1 for b in idle) and (a[[b for b in range(B) if b not in idle and topo[b] >= 0]] >= 0).all()
            for b in (5, 14, 17, 11):        # the pages come back, the lengths are put right, the stack is filled
                table[b, :mended_table.shape[1]] = np.where(mended_table[b] >= 0, mended_table[b], -1)
            lens[[7, 13]] = mended_lens[[7, 13]]
            held = set(table[table >= 0].tolist())
            spare = [p for p in range(n_pages) if p not in held]
            low[:] = 0
            n_free = min(len(spare), low.size)
            low[:n_free] = spare[:n_free]
            reset(table, lens, low, n_free)
    assert accepted > 10
