"""GPU: the repetition factor's division and product, bit for bit what fp32 gives,
over every size a logit or a factor can have."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import paged_oracle as po  # noqa: E402
from tests.paged_helpers import TREES, dev, host, i32, say  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_27550_amd import api as _api
    return _api


def floats(g, n, lo, hi):
    """Positive floats of random significands, exponents in [lo, hi] (below -126: subnormal)."""
    with np.errstate(under="ignore"):
        x = np.ldexp((1 + g.integers(0, 1 << 23, n) / 2.0 ** 23), g.integers(lo, hi + 1, n)).astype(np.float32)
    return np.where(x > 0, x, np.float32(2.0 ** -149))


@pytest.mark.parametrize("V", [1 << 16, (1 << 16) + 3])
@pytest.mark.parametrize("reps", ["ordinary", "any", "edges", "beyond"])
def test_a_seen_logit_is_divided_as_fp32_divides(api, V, reps):
    g = np.random.default_rng(V + len(reps))
    B = 16
    rep = {"ordinary": 1 + g.random(B).astype(np.float32), "any": floats(g, B, -149, 127),
           "edges": np.array([2.0 ** -40, np.nextafter(np.float32(2.0 ** -40), np.float32(0)), 2.0 ** 40,
                              np.nextafter(np.float32(2.0 ** 40), np.float32(np.inf)), 2.0 ** -149, 2.0 ** -127, 2.0 ** -126,
                              3.4028234e38, 2.0 ** 126, 2.0 ** 127, np.nextafter(np.float32(1), np.float32(2)),
                              np.nextafter(np.float32(1), np.float32(0)), np.nextafter(np.float32(2), np.float32(0)), 1.5,
                              1.1754942e-38, 1e-39]),
           "beyond": np.resize(np.array([np.inf, 0.0, -1.5, -1e-39]), B)}[reps].astype(np.float32)   # (not asked for)
    z = np.concatenate([floats(g, V // 2, -6, 6), floats(g, V // 4, -149, 127), floats(g, V - V // 2 - V // 4, -64, -56)])
    z = (z * g.choice(np.array([1, 1, 1, -1], np.float32), V)).astype(np.float32)
    z[:6] = [0.0, -0.0, np.inf, -np.inf, 2.0 ** -60, 2.0 ** 60]
    if reps == "beyond":
        z[2:4] = 1.0
    z = np.tile(z, (B, 1))
    for b in range(B):
        g.shuffle(z[b])
    hist = np.full((B, V), po.SEEN, np.int32)      # (in the prompt, never said: the factor alone)
    hist[:, ::5] = 0
    params = np.zeros((B, 4), np.float32)
    params[:, 0], params[:, 3] = rep, 1
    bank, out = api.Bank(TREES), torch.zeros((B, V), device="cuda")
    say("logit_adjust division", V, reps)
    api.logit_adjust(bank, i32([0] * B), i32(np.arange(B + 1)), i32([-1] * B), dev(z), dev(params), out, None, None, None, None,
                     history=dev(hist))
    with np.errstate(all="ignore"):
        want = np.where(z > 0, z / rep[:, None], z * rep[:, None]).astype(np.float32)
    want = np.where(hist != 0, want, z)
    got = host(out)
    nan = np.isnan(want)
    np.testing.assert_array_equal(np.isnan(got), nan)
    np.testing.assert_array_equal(np.where(nan, 0, got).view(np.int32), np.where(nan, np.float32(0), want).view(np.int32))
