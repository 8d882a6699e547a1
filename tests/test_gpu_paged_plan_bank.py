"""GPU: a plan belongs to the bank it was made for, also where the next bank lies
in the same memory."""
import ctypes
import types

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests.paged_helpers import TREES, say, unbits  # noqa: E402
from tests.test_gpu_paged_attn import api, check, launch, make  # noqa: E402,F401

pytestmark = pytest.mark.gpu


def build(api, trees, arena):
    """A bank whose arena the caller brings."""
    parents = np.ascontiguousarray(np.concatenate([np.asarray(t, np.int32) for t in trees]))
    sizes = np.array([len(t) for t in trees], np.int32)
    need, handle = ctypes.c_size_t(0), ctypes.c_void_p(None)
    ptr = lambda a: a.ctypes.data_as(ctypes.c_void_p)   # noqa: E731
    rc = api.lib.entmtp_bank_build(ptr(parents), ptr(sizes), len(trees), arena.data_ptr(), arena.numel(), ctypes.byref(need),
                                   torch.cuda.current_stream().cuda_stream, ctypes.byref(handle))
    assert rc == api.OK, api.last_error()
    return types.SimpleNamespace(handle=handle)


def test_a_plan_of_the_bank_before_does_nothing(api):
    arena = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    old = build(api, TREES, arena)
    c = make(71, [2, 1], [100, 300], 8, 2, 16)
    d = launch(api, c, bank=old)
    check(c, d)
    assert api.lib.entmtp_bank_destroy(old.handle) == api.OK
    new = build(api, TREES[::-1], arena)
    d["out"].fill_(7)
    keys = unbits(d["kp"]).copy()
    say("tree_attn_paged with the plan of a bank that is gone")
    api.tree_attn_paged(new, d["plan"], d["q"], d["kt"], d["vt"], d["kp"], d["vp"], d["table"], d["slots"], 128 ** -0.5, 1e4,
                        d["out"], d["ws"])
    assert (unbits(d["out"]) == 0x40E0).all()
    np.testing.assert_array_equal(unbits(d["kp"]), keys)
    assert api.lib.entmtp_bank_destroy(new.handle) == api.OK
    # (and the same trees in a third bank: its own plan runs)
    check(c, launch(api, c, bank=build(api, TREES, arena)))
