"""Host side of the trees that a plan hands to the rest of a step (no GPU)."""
import pytest

torch = pytest.importorskip("torch")

from paper_2606_27550_amd import api  # noqa: E402

P = 1 << 20


def test_topo_is_a_view_into_the_plan():
    bank = api.Bank([[-1, 0, 0], [-1]], device=None)
    for B in (1, 2, 17, 256):
        plan = torch.full((api.tree_attn_paged_plan_bytes(bank, B, 3 * B, 8, 2, 8, 16),), 255, dtype=torch.uint8)
        run = api.tree_attn_paged_topo(plan, B)
        assert run.dtype == torch.int32 and tuple(run.shape) == (B,) and run.is_contiguous()
        at = run.data_ptr() - plan.data_ptr()
        assert 64 <= at <= plan.numel() - 4 * B and at % 16 == 0 and (run == -1).all()
        plan.zero_()
        assert (run == 0).all()
        assert api.tree_attn_paged_topo(plan.view(torch.int64), B).data_ptr() == run.data_ptr()


def test_refusals():
    for B in (0, -1, 257):
        assert not api.lib.entmtp_tree_attn_paged_topo(P, B)
    assert not api.lib.entmtp_tree_attn_paged_topo(None, 2)
    plan = torch.zeros(4096, dtype=torch.uint8)
    for args in ((plan, 0), (plan, 257), (plan[:64], 2), (plan[::2], 2), (None, 2)):
        with pytest.raises(ValueError):
            api.tree_attn_paged_topo(*args)
