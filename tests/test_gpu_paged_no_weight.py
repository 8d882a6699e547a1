"""GPU: a row that sees no key of any weight -- every visible score is minus
infinity -- is NaN, as the softmax of such a row, whether or not its prefix is
split; with a score cap the scores are finite and every key weighs the same."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import entmtp_oracle as orc  # noqa: E402
from tests.paged_helpers import say, unbits  # noqa: E402
from tests.test_gpu_paged_attn import api, launch, make  # noqa: E402,F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("L", [0, 1, 40, 300, 3000])
def test_every_score_minus_infinity(api, L):
    c = make(L + 91, [0, 0], [L, 20], 8, 2, 16)
    c["q"] &= 0x7FFF                                  # (positive)
    n = -(-L // 16)
    mine = c["table"][0, :n]
    c["kp"][mine, :, :, 9] = 0xFF80                   # all keys of the first sequence
    c["kt"][0, :, 9] = 0xFF80
    for kw in (dict(), dict(window=2 ** 30), dict(slopes=[0.0] * 8)):
        say("tree_attn_paged without weight", L, sorted(kw))
        got = orc.bf16_to_f64(unbits(launch(api, c, theta=0.0, **kw)["out"]))
        assert np.isnan(got[0]).all() and np.isfinite(got[1]).all()
    got = orc.bf16_to_f64(unbits(launch(api, c, theta=0.0, softcap=30.0)["out"]))
    v = orc.bf16_to_f64(c["vp"])
    for h in range(8):
        rows = np.concatenate([np.concatenate([v[p, h // 4] for p in mine])[:L] if L else np.zeros((0, 128)),
                               orc.bf16_to_f64(c["vt"])[:1, h // 4]])
        ref = rows.mean(0)
        # a split's partial and the output are rounded to bf16, weights of one sum exactly
        assert (np.abs(got[0, h] - ref) <= 2.0 ** -8 * (np.abs(rows).mean(0) + np.abs(ref)) + 1e-5).all()
