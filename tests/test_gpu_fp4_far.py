"""GPU: 4-bit pools and weights beyond 4 GiB, and scale bytes at odd addresses.

Offsets into a pool or weights pass 32 bits there; the outputs are the same bits
as those of the same rows in small ones (what other rows hold does not matter).
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import entmtp_oracle as orc  # noqa: E402
from oracle import fp4_oracle as fo  # noqa: E402
from paper_2606_27550_amd import synth  # noqa: E402
from tests.fp4_helpers import D, make, quantize_fast  # noqa: E402
from tests.paged_helpers import TREES, bits, dev, host, i32, say, unbits  # noqa: E402
from tests.test_gpu_fp4_attn import launch  # noqa: E402

pytestmark = pytest.mark.gpu
FAR = 33000   # pages of 8 heads of 256 rows: 4.6e9 bytes


@pytest.fixture(scope="module")
def api():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_27550_amd import api as _api
    return _api


@pytest.mark.parametrize("t", [0, 2, 4])
def test_attention_and_append(api, t):
    say("4-bit pool of", FAR, "pages, tree", t)
    page, Hkv, Hq, L, T = 256, 8, 32, 700, len(TREES[t])
    c = make(51, [t], [L], Hq, Hkv, page)
    near = launch(api, c, run=False)
    far = {k: torch.empty((FAR, Hkv, page * 68), dtype=torch.uint8, device="cuda") for k in ("kp", "vp")}
    move = FAR - c["n_pages"]
    for k, pool in far.items():
        pool[move:].copy_(near[k])
    table, n = i32(c["table"] + move), c["n_pages"]
    g = np.random.default_rng(t)
    k, v = (bits(synth.normal_bf16(g, (T, Hkv, D))) for _ in "kv")
    pos = i32(L + np.arange(T))
    slots = np.array([c["table"][0, (L + i) // page] * page + (L + i) % page for i in range(T)])
    outs = []
    for pools, tab, first, pages in (((near["kp"], near["vp"]), near["table"], 0, n), ((far["kp"], far["vp"]), table, move, FAR)):
        api.kv_append_paged_fp4(None, k, v, pos, i32(slots + first * page), 10000.0, None, *pools)
        api.tree_attn_paged_fp4_plan(near["bank"], near["topo"], near["lens"], near["off"], near["status"], tab, page, pages,
                                     T, Hq, Hkv, near["plan"])
        api.tree_attn_paged_fp4(near["bank"], near["plan"], near["q"], *pools, tab, 0.09, near["out"], near["ws"])
        outs.append(unbits(near["out"]).copy())
    assert np.isfinite(orc.bf16_to_f64(outs[0])).all()
    np.testing.assert_array_equal(outs[1], outs[0])
    for k in ("kp", "vp"):
        assert torch.equal(far[k][move:], near[k])
    # the last tree row moves to the first one's slot
    if T > 1:
        for pools, first in (((near["kp"], near["vp"]), 0), ((far["kp"], far["vp"]), move)):
            api.kv_compact_paged_fp4(i32([[0, T - 1]]), i32([1]), i32([0, T]), i32(slots + first * page), *pools)
        codes, scales = fo.planes(host(near["kp"]))
        a, b = ((slots[i] // page, slice(None), slots[i] % page) for i in (T - 1, 1))
        np.testing.assert_array_equal(codes[a], codes[b])
        for k in ("kp", "vp"):
            assert torch.equal(far[k][move:], near[k])


@pytest.mark.parametrize("T", [1, 20])
def test_logits_of_large_weights(api, T):
    V, hid, n = 2_200_003, 4096, 1000
    say("4-bit weights", V, hid, T)
    g = np.random.default_rng(5)
    small = [dev(a) for a in quantize_fast(orc.bf16_to_f64(synth.normal_bf16(g, (n, hid))))]
    codes = torch.zeros((V, hid // 2), dtype=torch.uint8, device="cuda")
    scales = torch.full((V, hid // 32), 127, dtype=torch.uint8, device="cuda")
    codes[-n:].copy_(small[0])
    scales[-n:].copy_(small[1])
    x = bits(synth.normal_bf16(g, (T, hid)))
    want, got = torch.empty((T, n), device="cuda"), torch.empty((T, V), device="cuda")
    api.verify_logits_fp4(x, *small, want)
    api.verify_logits_fp4(x, codes, scales, got)
    np.testing.assert_array_equal(host(got[:, -n:]), host(want))
    assert (got[:, :-n] == 0).all()


@pytest.mark.parametrize("T,hid", [(1, 1024), (20, 1024), (40, 1024), (3, 896)])
def test_scale_bytes_at_odd_addresses(api, T, hid):
    V = 301
    g = np.random.default_rng(T)
    w = synth.normal_bf16(g, (V, hid))
    c, s = quantize_fast(orc.bf16_to_f64(w))
    x = synth.normal_bf16(g, (T, hid))
    codes = torch.empty((V, hid // 2), dtype=torch.uint8, device="cuda")
    room = torch.full((V * hid // 32 + 2,), 9, dtype=torch.uint8, device="cuda")
    scales = room[1:-1].view(V, hid // 32)
    out = torch.empty((T, V), device="cuda")
    api.quantize_fp4(bits(w), codes, scales)
    assert int(room[0]) == 9 and int(room[-1]) == 9
    np.testing.assert_array_equal(host(scales), s)
    api.verify_logits_fp4(bits(x), codes, scales, out)
    xf, wf = orc.bf16_to_f64(x), fo.values(c, s)
    # (the bound of the sums in the tests of aligned weights)
    room = (44 + hid / 256 + 8) * 2.0 ** -23 * (np.abs(xf) @ np.abs(wf).T)
    assert (np.abs(host(out).astype(np.float64) - xf @ wf.T) <= room).all()
