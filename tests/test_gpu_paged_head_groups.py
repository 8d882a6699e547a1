"""GPU: tree attention over the page pool with head counts that divide nothing
evenly -- query groups that are no power of two (rows of several heads share a
32-row tile), KV heads that are no multiple of eight (padded work lists),
heads that a merge's workgroups do not divide -- against 64 bits, with the
bounds of test_gpu_paged_attn.py."""
import pytest

torch = pytest.importorskip("torch")

from tests.paged_helpers import say  # noqa: E402
from tests.test_gpu_paged_attn import api, check, launch, make  # noqa: E402,F401

pytestmark = pytest.mark.gpu

HEADS = [(40, 8), (28, 4), (32, 32), (12, 12), (24, 12), (15, 5), (9, 3), (33, 11), (7, 1), (31, 1)]


@pytest.mark.parametrize("Hq,Hkv", HEADS)
def test_lone_sequences(api, Hq, Hkv):
    """One sequence, short (not split) and long (split), few rows (a merge of a wavefront a head) and many."""
    for t, L, page in ((0, 63, 16), (2, 40, 16), (0, 3000, 32), (2, 1200, 16), (4, 900, 64)):
        say("tree_attn_paged", Hq, Hkv, t, L, page)
        c = make(Hq + t, [t], [L], Hq, Hkv, page, behind=1)
        check(c, launch(api, c))


@pytest.mark.parametrize("Hq,Hkv", HEADS)
def test_batches(api, Hq, Hkv):
    """Several sequences, split and not, an unused place among them; then with a window and a cap, then with a bias."""
    topo, lens = [2, 0, -1, 1, 0, 4], [700, 45, 0, 31, 2500, 5]
    c = make(Hq, topo, lens, Hq, Hkv, 16, behind=3)
    for kw in (dict(), dict(window=100, softcap=20.0), dict(slopes=[2.0 ** -(1 + h % 8) for h in range(Hq)])):
        say("tree_attn_paged", Hq, Hkv, sorted(kw))
        check(c, launch(api, c, **kw), **kw)


@pytest.mark.parametrize("Hq,Hkv,rows", [(40, 8, 25), (40, 8, 26), (28, 4, 36), (28, 4, 37), (12, 12, 85), (12, 12, 86)])
def test_both_sides_of_the_merges_forms(api, Hq, Hkv, rows):
    """Rows x heads at and past the count up to which a wavefront takes a head (four a compute unit: 1024 of 256 units)."""
    topo, lens = [0, 0, 1], [2000, 400, 1100]
    c = make(rows, topo, lens, Hq, Hkv, 16, behind=rows - 9)
    assert c["rows"] == rows
    say("tree_attn_paged", Hq, Hkv, rows)
    check(c, launch(api, c))
