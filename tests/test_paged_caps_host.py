"""Score caps so small that the query they are folded into could overflow are
refused on the host (no GPU)."""
import pytest

from paper_2606_27550_amd import api
from tests.test_paged_host import ATTN, bank, call, refused  # noqa: F401


@pytest.mark.parametrize("scale,softcap,fits", [(1.0, 2.0 ** -64, True), (1.0, 2.0 ** -65, False), (0.1, 1e-25, False),
                                                (2.0 ** 70, 64.0, True), (2.0 ** 71, 64.0, False), (1e30, 1024.0, False),
                                                (0.1, 2.0 ** -60, True)])
def test_caps_against_the_scale(bank, scale, softcap, fits):  # noqa: F811
    # (a call whose cap fits is refused for its bank, which has no device arena)
    refused(call("entmtp_tree_attn_paged", ATTN, bank=bank.handle, scale=scale, softcap=softcap), api.EINVAL)
    assert ("softcap" in api.last_error()) == (not fits)
