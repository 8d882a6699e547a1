"""GPU: the 4-bit operators together, as a serving loop runs them: a prompt on
its way into the pages, then a step captured into one graph (page map, plan,
positions, two layers of append and attention, LM head, statistics, acceptance,
compaction, prefix lengths) and replayed, every replay held against the oracle."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import entmtp_oracle as orc  # noqa: E402
from oracle import fp4_oracle as fo  # noqa: E402
from oracle import paged_oracle as po  # noqa: E402
from paper_2606_27550_amd import synth  # noqa: E402
from tests.fp4_helpers import pool_bits, quantize_fast, tree_rows  # noqa: E402
from tests.paged_helpers import TREES, bits, dev, host, i32, say, unbits  # noqa: E402
from tests.test_gpu_fp4_rows import to_bf16  # noqa: E402

pytestmark = pytest.mark.gpu
D, SCALE, THETA, EPS = 128, 1 / math.sqrt(128), 1e4, 1e-5


@pytest.fixture(scope="module")
def api():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_27550_amd import api as _api
    return _api


def store(pool, slot, page, row):
    """A row's 64-bit numbers [Hkv, d] (bf16 ones) into a layer's 4-bit pages."""
    codes, scales = quantize_fast(row)
    i = slot % page
    pool[slot // page, :, 64 * i:64 * i + 64] = codes
    pool[slot // page, :, 64 * page + 4 * i:64 * page + 4 * i + 4] = scales


def test_captured_steps(api):
    g = np.random.default_rng(41)
    B, Hq, Hkv, page, layers, V, hid, window = 5, 8, 2, 16, 2, 301, 96, 48
    max_pages, n_pages, rows, cap_path = 30, 90, 240, 32
    topo = np.array([2, 1, -1, 4, 3], np.int32)              # one unused place
    lens = np.array([37, 0, 0, 150, 16], np.int32)
    T = [len(TREES[t]) if t >= 0 else 0 for t in topo]
    bank = api.Bank(TREES)
    table = np.full((B, max_pages), -1, np.int32)
    used = 0
    for b, L in enumerate(lens):
        n = -(-int(L) // page)
        table[b, :n] = np.arange(used, used + n)
        used += n
    # the last sequence finds its tree's pages missing (the stack runs dry before it) until some are given back
    need = sum(-(-int(L + t) // page) - -(-int(L) // page) for L, t in zip(lens[:4], T[:4]))
    free = g.permutation(np.arange(used, n_pages)).astype(np.int32)
    n_free = need
    wq, wk = (synth.normal_bf16(g, (D,)) for _ in range(2))
    codes, scales = quantize_fast(orc.bf16_to_f64(synth.lm_head_weight(31, V, hid, std=0.3)))
    w64 = fo.values(codes, scales)

    z = lambda *s, dt=torch.int32: torch.zeros(s, dtype=dt, device="cuda")   # noqa: E731
    bf, f32, u8 = torch.bfloat16, torch.float32, torch.uint8
    size = page * 68
    pools = [np.zeros((layers, n_pages, Hkv, size), np.uint8) for _ in "kv"]
    d = dict(topo=i32(topo), lens=i32(lens), table=i32(table), free=i32(free), n=i32([n_free]), off=z(B + 1), slots=z(rows),
             status=z(B), kp=z(layers, n_pages, Hkv, size, dt=u8), vp=z(layers, n_pages, Hkv, size, dt=u8), codes=dev(codes),
             scales=dev(scales), tok=z(rows), qkv=z(layers, rows, Hq + 2 * Hkv, D, dt=bf), q=z(layers, rows, Hq, D, dt=bf),
             out=z(layers, rows, Hq, D, dt=bf), x=z(rows, hid, dt=bf), z=z(rows, V, dt=f32), H=z(rows, dt=f32), p1=z(rows, dt=f32),
             am=z(rows), a=z(B), path=z(B, cap_path), bonus=z(B), best=z(B, dt=f32), pos=z(rows), wq=bits(wq), wk=bits(wk))
    byte = lambda n: torch.empty(max(n, 64), dtype=torch.uint8, device="cuda")   # noqa: E731
    shape = (rows, Hq, Hkv)
    plans = [byte(api.tree_attn_paged_fp4_plan_bytes(bank, B, *shape, max_pages, page)) for _ in range(2)]
    ws = byte(api.tree_attn_paged_fp4_workspace(bank, B, *shape, D, max_pages, page))
    first = api.tree_attn_paged_topo(plans[0], B)
    runs = api.tree_attn_paged_topo(plans[1], B)

    def key(x, pos):
        return orc.bf16_to_f64(to_bf16(fo.norm_turn(orc.bf16_to_f64(x), int(pos), orc.bf16_to_f64(wk), EPS, THETA)))

    # the prompts, all sequences' rows in one call a layer
    where = [(b, p) for b, L in enumerate(lens) for p in range(L)]
    slots = np.array([table[b, p // page] * page + p % page for b, p in where], np.int32)
    for layer in range(layers):
        qkv = synth.normal_bf16(g, (len(where), Hq + 2 * Hkv, D))
        t = bits(qkv)
        api.kv_append_paged_fp4(None, t[:, Hq:Hq + Hkv], t[:, Hq + Hkv:], i32([p for _, p in where]), i32(slots), THETA, None,
                                d["kp"][layer], d["vp"][layer], k_norm=d["wk"], eps=EPS)
        for r, (b, p) in enumerate(where):
            store(pools[0][layer], slots[r], page, key(qkv[r, Hq:Hq + Hkv], p))
            store(pools[1][layer], slots[r], page, orc.bf16_to_f64(qkv[r, Hq + Hkv:]))
    torch.cuda.synchronize()
    np.testing.assert_array_equal(host(d["kp"]), pools[0])
    np.testing.assert_array_equal(host(d["vp"]), pools[1])

    def step():
        api.page_map(bank, d["topo"], d["lens"], d["table"], page, n_pages, d["off"], d["slots"], d["status"], d["free"], d["n"])
        api.tree_attn_paged_fp4_plan(bank, d["topo"], d["lens"], d["off"], d["status"], d["table"], page, n_pages, *shape,
                                     plans[0])
        api.tree_attn_paged_fp4_plan(bank, first, d["lens"], d["off"], d["status"], d["table"], page, n_pages, *shape, plans[1],
                                     window=window)
        api.tree_positions(bank, runs, d["lens"], d["off"], d["pos"])
        for layer, win in ((0, 0), (1, window)):
            qkv = d["qkv"][layer]
            api.kv_append_paged_fp4(qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:], d["pos"], d["slots"], THETA,
                                    d["q"][layer], d["kp"][layer], d["vp"][layer], q_norm=d["wq"], k_norm=d["wk"], eps=EPS)
            api.tree_attn_paged_fp4(bank, plans[layer], d["q"][layer], d["kp"][layer], d["vp"][layer], d["table"], SCALE,
                                    d["out"][layer], ws, window=win, softcap=20.0 * layer)
        api.verify_logits_fp4(d["x"], d["codes"], d["scales"], d["z"])
        api.logit_stats(d["z"], 1.0, d["H"], d["p1"], d["am"])
        api.accept_batched_device(bank, runs, d["off"], d["tok"], d["am"], d["p1"], d["a"], d["path"], d["bonus"], d["best"])
        api.kv_compact_paged_fp4(d["path"], d["a"], d["off"], d["slots"], d["kp"], d["vp"])
        d["lens"].add_(d["a"] + 1)

    def fill():
        s = dict(qkv=synth.normal_bf16(g, (layers, rows, Hq + 2 * Hkv, D)), x=synth.normal_bf16(g, (rows, hid)),
                 tok=g.integers(0, V, rows).astype(np.int32))
        raw = orc.bf16_to_f64(s["x"]) @ w64.T
        r0 = 0
        for b, t in enumerate(topo):
            for i in range(1, T[b]):
                if g.random() < 0.8:
                    s["tok"][r0 + i] = int(np.argmax(raw[r0 + TREES[t][i]]))
            r0 += T[b]
        d["qkv"].copy_(bits(s["qkv"]))
        d["x"].copy_(bits(s["x"]))
        d["tok"].copy_(i32(s["tok"]))
        d["out"].fill_(7)
        return s

    fill()
    step()          # (the first calls, eager)
    torch.cuda.synchronize()
    for k, v in (("lens", lens), ("table", table), ("n", [n_free])):
        d[k].copy_(i32(v))
    for k, v in (("kp", pools[0]), ("vp", pools[1])):
        d[k].copy_(dev(v))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    accepted = 0
    for n in range(5):
        s = fill()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        say("4-bit serving step", n, "lens", lens.tolist())
        table, row_off, slots, status, n_free = po.page_map(TREES, topo, lens, table, page, n_pages, rows, free, n_free)
        served = [status[b] == po.OK for b in range(B)]
        if n == 0:
            assert status.tolist() == [0, 0, po.NONE, 0, po.FULL]
        np.testing.assert_array_equal(host(d["table"]), table)
        np.testing.assert_array_equal(host(d["slots"])[:slots.size], slots)
        assert host(runs).tolist() == [int(t) if ok else -1 for t, ok in zip(topo, served)]
        pos = np.full(rows, -1, np.int32)
        out, q = orc.bf16_to_f64(unbits(d["out"])), unbits(d["q"])
        am, zl = host(d["am"]), host(d["z"])
        xf = orc.bf16_to_f64(s["x"])
        room = 64 * 2.0 ** -23 * (np.abs(xf) @ np.abs(w64).T)
        assert (np.abs(zl - xf @ w64.T) <= room).all()
        np.testing.assert_array_equal(am, zl.argmax(1))
        a, path = np.full(B, -1, np.int32), np.full((B, cap_path), -1, np.int32)
        bonus = np.full(B, -1, np.int32)
        for b, t in enumerate(topo):
            if not served[b]:
                continue
            r0, L = int(row_off[b]), int(lens[b])
            r = slice(r0, r0 + T[b])
            pos[r] = L + np.array(orc.depths(TREES[t]))
            for layer, win in ((0, 0), (1, window)):
                for i in range(T[b]):
                    x = s["qkv"][layer, r0 + i]
                    store(pools[0][layer], slots[r0 + i], page, key(x[Hq:Hq + Hkv], pos[r0 + i]))
                    store(pools[1][layer], slots[r0 + i], page, orc.bf16_to_f64(x[Hq + Hkv:]))
                    want = fo.norm_turn(orc.bf16_to_f64(x[:Hq]), int(pos[r0 + i]), orc.bf16_to_f64(wq), EPS, THETA)
                    err = np.abs(orc.bf16_to_f64(q[layer][r0 + i]) - want)
                    assert (err <= 2.0 ** -8 * np.abs(want) + 1e-4).all()
                kb, vb = pool_bits(pools[0][layer]), pool_bits(pools[1][layer])
                ref, _, off = po.tree_attention_paged(q[layer][r], tree_rows(kb, table[b], L, T[b], page),
                                                      tree_rows(vb, table[b], L, T[b], page), kb, vb, table[b], L, TREES[t], SCALE,
                                                      0.0, 20.0 * layer, win)
                assert (np.abs(out[layer][r] - ref) <= off).all(), (n, b, layer)
            a[b], chain, bonus[b], _ = orc.accept(TREES[t], s["tok"][r], am[r])
            path[b, :len(chain)] = chain
        np.testing.assert_array_equal(host(d["pos"]), pos)
        idle = pos < 0
        assert (out[:, idle] == 7).all()
        np.testing.assert_array_equal(host(d["a"]), a)
        np.testing.assert_array_equal(host(d["bonus"]), bonus)
        for k, name in enumerate(("kp", "vp")):
            parts = [po.kv_compact_paged(x, path, a, row_off, slots) for x in fo.planes(pools[k])]
            pools[k] = fo.join(*parts)
            np.testing.assert_array_equal(host(d[name]), pools[k])
        lens = lens + a + 1
        np.testing.assert_array_equal(host(d["lens"]), lens)
        accepted += int(a[a > 0].sum())
        if n == 1:      # pages come back: the sequence that waited is run again
            free = g.permutation([p for p in range(n_pages) if p not in set(table[table >= 0].tolist())]).astype(np.int32)
            n_free = free.size
            d["free"][:free.size].copy_(i32(free))
            d["n"].copy_(i32([n_free]))
    assert accepted > 10 and served[4]
