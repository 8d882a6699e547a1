"""GPU: positions of tree rows where offsets leave the ordinary (whole numbers, compared as they are)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import entmtp_oracle as orc  # noqa: E402
from tests.paged_helpers import TREES, host, i32, say  # noqa: E402

pytestmark = pytest.mark.gpu
LOW, HIGH = -2 ** 31, 2 ** 31 - 1


@pytest.fixture(scope="module")
def api():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_27550_amd import api as _api
    return _api


def positions(topo, lens, off, rows):
    """The definition: a row's sequence is the one whose range holds it."""
    want = np.full(rows, -1, np.int64)
    for b, (t, L) in enumerate(zip(topo, lens)):
        if not 0 <= t < len(TREES) or off[b] < 0 or not 0 <= L <= HIGH - 256:
            continue
        T = len(TREES[t])
        if off[b] + T <= min(off[b + 1], rows):
            want[off[b]:off[b] + T] = L + np.array(orc.depths(TREES[t]))
    return want


@pytest.mark.parametrize("topo,lens,off", [
    ([1], [9], [-3, 5]), ([1], [9], [-3, 30]), ([1], [9], [LOW, HIGH]), ([1], [9], [LOW, 0]), ([1], [9], [LOW, 12]),
    ([1], [9], [7, LOW]), ([1], [9], [HIGH, LOW]), ([1], [9], [HIGH, HIGH]), ([1], [9], [LOW, LOW]), ([1], [9], [33, HIGH]),
    ([1], [9], [34, HIGH]), ([0, 1], [4, 9], [-5, 6, 20]), ([0, 1, 0], [4, 9, 2], [-9, -1, 3, 4]),
    ([1, 0], [9, 4], [2, 9, 40]),
    # falling offsets: a sequence without rows between, before and behind those that have some
    ([0, 1], [4, 9], [12, 3, 11]), ([1, 0], [9, 4], [0, 20, 10]), ([0], [4], [20, 0]), ([1, 0, 1], [9, 4, 2], [20, 30, 1, 8])])
def test_positions_at_any_offsets(api, topo, lens, off):
    """-1 in every row of [0, rows) that no served sequence holds, whatever was there; nothing behind."""
    say("tree_positions", topo, lens, off)
    room = torch.full((400,), 77, dtype=torch.int32, device="cuda")
    api.tree_positions(api.Bank(TREES), i32(topo), i32(lens), i32(off), room[:40])
    got = host(room)
    np.testing.assert_array_equal(got[:40], positions(topo, lens, off, 40))
    assert (got[40:] == 77).all()


def test_positions_of_a_full_batch(api):
    """256 sequences, one of them at a negative offset, one with a range that falls."""
    g = np.random.default_rng(5)
    topo, lens = g.integers(0, 3, 256), g.integers(0, 5000, 256)
    off = np.concatenate([[0], np.cumsum([len(TREES[t]) for t in topo])])
    rows = int(off[-1]) + 50
    for change in ({}, {0: -4}, {256: int(off[255]) - 30}):
        o = off.copy()
        for k, v in change.items():
            o[k] = v
        pos = torch.full((rows,), 77, dtype=torch.int32, device="cuda")
        api.tree_positions(api.Bank(TREES), i32(topo), i32(lens), i32(o), pos)
        want = positions(topo, lens, o, rows)
        np.testing.assert_array_equal(host(pos), want)
