"""GPU: the paged attention where the caller has rotated queries and keys already
(rope_theta 0).  Such a query is exact in bf16, so only the softmax weights, a
split's partial and the output are rounded: 2^-8 of the value each."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import entmtp_oracle as orc  # noqa: E402
from tests.paged_helpers import say, unbits  # noqa: E402
from tests.test_gpu_paged_attn import SCALE, api, launch, make  # noqa: E402,F401

pytestmark = pytest.mark.gpu
D = 128


def bf16(x):
    """Bits of a value that bf16 holds."""
    b = orc.f64_to_bf16_bits(np.asarray(x, np.float64))
    assert (orc.bf16_to_f64(b) == x).all()
    return b


def worst_pair():
    """Two bf16 values whose products with scale * log2(e) rounding to bf16 moves furthest apart."""
    c = SCALE * math.log2(math.e)
    x = 1 + np.arange(128) / 128
    off = orc.bf16_to_f64(orc.f64_to_bf16_bits(x * c)) / (x * c) - 1
    a, b = x[np.argmax(off)], x[np.argmin(off)]
    assert off.max() - off.min() > 0.004
    return float(a), float(b)


OPTIONS = [dict(), dict(window=2 ** 31 - 1), dict(softcap=1024.0), dict(slopes=True), dict(softcap=1024.0, window=2 ** 30, slopes=True)]


@pytest.mark.parametrize("opt", OPTIONS)
@pytest.mark.parametrize("L,Hq,Hkv", [(1, 4, 1), (31, 8, 8), (200, 8, 2), (3000, 8, 2)])
def test_equal_scores_stay_equal(api, L, Hq, Hkv, opt):
    """Keys of two kinds, one along each half of the query, whose products with it are equal and exact in fp32 whatever the
    order (about 240 once scaled): every key weighs the same, so the output is the share of keys of value one."""
    opt = dict(opt)
    if opt.get("slopes"):
        opt["slopes"] = np.zeros(Hq, np.float32)
    a, b = worst_pair()
    c = make(L, [0], [L], Hq, Hkv, 16)
    half = np.arange(D) < D // 2
    c["q"][:] = bf16(np.where(half, a, b))
    # a (16 b) = b (16 a): the two kinds of key, values one and zero
    first, second = bf16(np.where(half, 16 * b, 0.0)), bf16(np.where(half, 0.0, 16 * a))
    kind = np.random.default_rng(L).random(L + 1) < 0.5
    kind[-1] = not kind[0]
    for p in range(L):
        page, at = c["table"][0, p // 16], p % 16
        c["kp"][page, :, at] = first if kind[p] else second
        c["vp"][page, :, at] = bf16(1.0 if kind[p] else 0.0)
    c["kt"][0] = first if kind[L] else second
    c["vt"][0] = bf16(1.0 if kind[L] else 0.0)
    say("tree_attn_paged without rotation", L, Hq, Hkv, sorted(opt))
    got = orc.bf16_to_f64(unbits(launch(api, c, theta=0.0, **opt)["out"]))[0]
    share = float(kind.mean())
    # weights of one sum, each 1 / (L + 1) within 2^-24 or so; three roundings of at most 2^-8 of the share
    assert (np.abs(got - share) <= 3 * 2.0 ** -8 * share + 1e-5).all(), (float(np.abs(got - share).max()), share)
