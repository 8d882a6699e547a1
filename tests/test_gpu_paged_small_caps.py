"""GPU: the smallest score caps there may be: every score is plus or minus next to
nothing, so that all keys weigh the same."""
import pytest

torch = pytest.importorskip("torch")

from tests.paged_helpers import say  # noqa: E402
from tests.test_gpu_paged_attn import SCALE, api, check, launch, make  # noqa: E402,F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("theta", [1e4, 0.0])
@pytest.mark.parametrize("softcap", [SCALE * 2.0 ** -64, 2.0 ** -40])
def test_smallest_caps(api, softcap, theta):
    c = make(81, [2, 0, 1], [300, 2000, 0], 8, 2, 16)
    say("tree_attn_paged", softcap, theta)
    d = launch(api, c, softcap=softcap, theta=theta)
    check(c, d, softcap=softcap, theta=theta)
