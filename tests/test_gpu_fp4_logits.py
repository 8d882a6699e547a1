"""GPU: LM-head logits from 4-bit weights against 64 bits.

The products of a bf16 number and a 4-bit one are exact, so a logit is a sum of
hid exact numbers in fp32: however it is ordered in groups of 32 that a matrix
instruction adds up (at most 32 roundings, or truncations: 2^-23 each), the
groups of a wavefront one after another (hid / 256 + 4 at most) and the eight
wavefronts, its error is at most (32 + hid / 256 + 4 + 8 + passes) 2^-23 sum |x w|.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import entmtp_oracle as orc  # noqa: E402
from oracle import fp4_oracle as fo  # noqa: E402
from paper_2606_27550_amd import synth  # noqa: E402
from tests.fp4_helpers import quantize_fast  # noqa: E402
from tests.paged_helpers import bits, dev, host, say  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_27550_amd import api as _api
    return _api


def weights(seed, V, hid):
    g = np.random.default_rng(seed)
    w = orc.bf16_to_f64(synth.normal_bf16(g, (V, hid))) * 2.0 ** g.integers(-9, -3, (V, 1))
    return quantize_fast(w)


def check(x, codes, scales, got, rows=None):
    hid = x.shape[1]
    xf, w = orc.bf16_to_f64(x), fo.values(codes, scales)
    ref, size = xf @ w.T, np.abs(xf) @ np.abs(w).T
    room = (44 + hid / 256 + 8) * 2.0 ** -23 * size
    err = np.abs(got.astype(np.float64) - ref)
    assert (err <= room).all(), float((err / room).max())


@pytest.mark.parametrize("T,hid,V", [
    (1, 32, 1), (1, 4096, 4096), (2, 64, 17), (1, 1056, 999), (5, 160, 3001), (16, 2048, 515), (17, 4096, 260), (27, 5120, 1000),
    (31, 96, 64), (32, 8192, 130), (33, 1024, 777), (48, 4096, 300), (64, 2048, 1025), (65, 320, 515), (100, 4096, 400),
    (128, 5120, 513), (129, 1024, 64), (200, 544, 130), (256, 2048, 1000), (300, 128, 48), (1, 12288, 50), (3, 65536, 20),
    (40, 20000, 33), (130, 16384, 40),
    (33, 128, 129), (64, 256, 127), (65, 384, 1), (128, 512, 300), (129, 4096, 131), (700, 128, 257), (50, 5120, 2100),
    (5, 8320, 40), (40, 5248, 100), (1, 3584, 300), (27, 2688, 401), (100, 1536, 77), (20, 4992, 33)])
def test_against_64_bits(api, T, hid, V):
    say("verify_logits_fp4", T, hid, V)
    codes, scales = weights(T + V, V, hid)
    x = synth.normal_bf16(np.random.default_rng(T), (T, hid))
    out = torch.full((T + 1, V), 7.0, device="cuda")
    api.verify_logits_fp4(bits(x), dev(codes), dev(scales), out[:T])
    check(x, codes, scales, host(out)[:T])
    assert (host(out)[T] == 7).all()


def test_rows_do_not_depend_on_each_other(api):
    """A row's logits, among others and (where the same kernel takes it) alone; repeats are the same bits."""
    codes, scales = (dev(a) for a in weights(3, 2500, 1024))
    x = bits(synth.normal_bf16(np.random.default_rng(3), (150, 1024)))
    def logits(x):
        out = torch.empty((x.shape[0], 2500), device="cuda")
        api.verify_logits_fp4(x, codes, scales, out)
        return host(out)
    all_ = logits(x)
    np.testing.assert_array_equal(logits(x), all_)
    y = x.clone()
    y[10:] = 0
    np.testing.assert_array_equal(logits(y)[:10], all_[:10])
    np.testing.assert_array_equal(logits(x[:9].clone()), logits(x[:12].clone())[:9])


def test_values_that_are_not_finite(api):
    """A weight group that is no number takes its vocabulary entry with it, a hidden value its row; nothing else."""
    T, hid, V = 20, 4160, 300
    codes, scales = weights(5, V, hid)
    x = synth.normal_bf16(np.random.default_rng(5), (T, hid))
    clean = torch.empty((T, V), device="cuda")
    api.verify_logits_fp4(bits(x), dev(codes), dev(scales), clean)
    clean = host(clean)
    for at in (0, hid // 32 - 1):     # (the last group: of a step that the row does not fill)
        s, y = scales.copy(), x.copy()
        s[7, at] = 255
        y[3, 32 * at] = 0x7FC0
        out = torch.empty((T, V), device="cuda")
        api.verify_logits_fp4(bits(y), dev(codes), dev(s), out)
        got = host(out)
        assert np.isnan(got[:, 7]).all() and np.isnan(got[3]).all()
        keep = np.ones((T, V), bool)
        keep[3], keep[:, 7] = False, False
        np.testing.assert_array_equal(got[keep], clean[keep])


def test_wide_range(api):
    """Hidden values and scales over many binades."""
    T, hid, V = 12, 512, 200
    g = np.random.default_rng(7)
    codes, scales = weights(7, V, hid)
    scales = (scales + g.integers(-30, 30, scales.shape)).astype(np.uint8)
    x = synth.normal_bf16(g, (T, hid))
    x = (x & 0x807F) | (g.integers(97, 157, (T, hid)) << 7).astype(np.uint16)
    out = torch.empty((T, V), device="cuda")
    api.verify_logits_fp4(bits(x), dev(codes), dev(scales), out)
    check(x, codes, scales, host(out))


@pytest.mark.parametrize("hid", [512, 1024])
def test_largest_scales(api, hid):
    """Scale bytes up to 254 where the values are bf16 numbers, small hidden values."""
    T, V = 3, 40
    g = np.random.default_rng(8)
    scales = g.integers(240, 255, (V, hid // 32)).astype(np.uint8)
    most = np.where(scales == 254, 3, np.where(scales == 253, 5, 7))        # codes below: 1 and a half, 3, 6 steps
    code = g.integers(0, 1 << 30, (V, hid)) % (np.repeat(most, 32, 1) + 1) | g.integers(0, 2, (V, hid)) << 3
    codes = (code[:, ::2] | code[:, 1::2] << 4).astype(np.uint8)
    x = synth.normal_bf16(g, (T, hid))
    x = (x & 0x807F) | (g.integers(60, 90, (T, hid)) << 7).astype(np.uint16)
    out = torch.empty((T, V), device="cuda")
    api.verify_logits_fp4(bits(x), dev(codes), dev(scales), out)
    check(x, codes, scales, host(out))


def test_with_the_quantizer(api):
    """Weights laid out by quantize_fp4, then the statistics of the logits."""
    T, hid, V = 27, 512, 1000
    g = np.random.default_rng(9)
    w, x = synth.normal_bf16(g, (V, hid)), synth.normal_bf16(g, (T, hid))
    codes = torch.empty((V, hid // 2), dtype=torch.uint8, device="cuda")
    scales = torch.empty((V, hid // 32), dtype=torch.uint8, device="cuda")
    out = torch.empty((T, V), device="cuda")
    H, p1 = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    am = torch.empty(T, dtype=torch.int32, device="cuda")
    api.quantize_fp4(bits(w), codes, scales)
    api.verify_logits_fp4(bits(x), codes, scales, out)
    api.logit_stats(out, 1.0, H, p1, am)
    c, s = quantize_fast(orc.bf16_to_f64(w))
    np.testing.assert_array_equal(host(codes), c)
    np.testing.assert_array_equal(host(scales), s)
    check(x, c, s, host(out))
    np.testing.assert_array_equal(host(am), host(out).argmax(1))


def test_captured(api):
    """Replayed with other hidden states, eager work between."""
    codes, scales = weights(11, 700, 2048)
    dc, ds = dev(codes), dev(scales)
    for T in (3, 80):
        x = torch.zeros((T, 2048), dtype=torch.bfloat16, device="cuda")
        out = torch.empty((T, 700), device="cuda")
        api.verify_logits_fp4(x, dc, ds, out)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            api.verify_logits_fp4(x, dc, ds, out)
        for k in range(3):
            xs = synth.normal_bf16(np.random.default_rng(k), (T, 2048))
            x.copy_(bits(xs))
            out.fill_(0)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            check(xs, codes, scales, host(out))
