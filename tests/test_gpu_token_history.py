"""GPU: the token history of a batch, from prompts and from accepted paths (exact)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import entmtp_oracle as orc  # noqa: E402
from oracle import paged_oracle as po  # noqa: E402
from tests.paged_helpers import TREES, host, i32, row_offsets, say  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_27550_amd import api as _api
    return _api


@pytest.mark.parametrize("B,V,most", [(1, 1, 3), (3, 50257, 400), (256, 1000, 60), (2, 7, 5000), (5, 128256, 70000)])
def test_prompts(api, B, V, most):
    g = np.random.default_rng(B)
    n = g.integers(0, most, B)
    n[0] = 0 if B > 1 else 2
    off = (np.concatenate([[0], np.cumsum(n)]) + 5).astype(np.int32)    # (the first five tokens are nobody's)
    tok = (g.random(off[-1] + 3) ** 3 * V).astype(np.int32)
    tok[::11] = -1
    tok[5::13] = V
    h = g.integers(0, 3, (B, V)).astype(np.int32)
    say("token_history_prompt", B, V, tok.size)
    hd = i32(h)
    api.token_history_prompt(i32(tok), i32(off), hd)
    want = po.history_prompt(h, tok, off)
    np.testing.assert_array_equal(host(hd), want)
    api.token_history_prompt(i32(tok), i32(off), hd)      # (once more changes nothing)
    np.testing.assert_array_equal(host(hd), want)


def test_no_tokens(api):
    h = torch.ones((2, 9), dtype=torch.int32, device="cuda")
    api.token_history_prompt(torch.zeros(0, dtype=torch.int32, device="cuda"), i32([0, 0, 0]), h)
    assert (host(h) == 1).all()


@pytest.mark.parametrize("B,V,path_cap", [(1, 3, 32), (4, 32000, 32), (256, 50257, 6), (3, 5, 1), (2, 11, 64)])
def test_accepted_paths(api, B, V, path_cap):
    g = np.random.default_rng(B + V)
    topo = g.integers(0, len(TREES), B)
    off = row_offsets(topo)
    tok = g.integers(-1, V + 1, off[-1]).astype(np.int32)
    path = np.full((B, path_cap), -1, np.int32)
    a = np.zeros(B, np.int32)
    for b, t in enumerate(topo):
        chain = orc.ancestors_or_self(TREES[t], int(g.integers(0, len(TREES[t]))))[:path_cap]
        path[b, :len(chain)] = chain
        a[b] = len(chain) - 1
    if B > 2:
        a[1] = -1
        path[2, 0:path_cap] = 2 ** 31 - 1
        a[2] = 2 ** 31 - 1
    bonus = g.integers(-1, V + 1, B).astype(np.int32)
    h = (g.integers(0, 3, (B, V)) | np.where(g.random((B, V)) < 0.3, po.SEEN, 0)).astype(np.int32)
    say("token_history_accept", B, V, path_cap)
    hd = i32(h)
    for _ in range(3):
        api.token_history_accept(i32(off), i32(tok), i32(path), i32(a), i32(bonus), hd)
        h = po.history_accept(h, off, tok, path, a, bonus)
    np.testing.assert_array_equal(host(hd), h)


def test_one_token_all_along_a_path(api):
    off, path = np.array([0, 32], np.int32), np.arange(32, dtype=np.int32)[None]
    h = torch.zeros((1, 4), dtype=torch.int32, device="cuda")
    api.token_history_accept(i32(off), i32(np.full(32, 2)), i32(path), i32([31]), i32([2]), h)
    assert host(h).tolist() == [[0, 0, 32, 0]]
