"""GPU: the page map against the oracle (exact): rows, slots, pages taken,
statuses of the sequences it cannot map."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import paged_oracle as po  # noqa: E402
from tests.paged_helpers import TREES, dev, host, i32, row_offsets, say  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_27550_amd import api as _api
    return _api


@pytest.fixture(scope="module")
def bank(api):
    return api.Bank(TREES)


def run(api, bank, topo, lens, table, page, n_pages, rows_cap, free, n_free, stream=None):
    B = len(topo)
    d = dict(table=i32(table), off=torch.full((B + 1,), -9, dtype=torch.int32, device="cuda"),
             slots=torch.full((rows_cap,), -9, dtype=torch.int32, device="cuda"),
             status=torch.full((B,), -9, dtype=torch.int32, device="cuda"),
             free=None if free is None else i32(free), n=None if free is None else i32([n_free]),
             topo=i32(topo), lens=i32(lens))

    def go():
        api.page_map(bank, d["topo"], d["lens"], d["table"], page, n_pages, d["off"], d["slots"], d["status"],
                     free_pages=d["free"], n_free=d["n"], stream=stream)
    return d, go


def check(d, want, rows_cap):
    table, off, slots, status, left = want
    np.testing.assert_array_equal(host(d["status"]), status)
    np.testing.assert_array_equal(host(d["off"]), off)
    np.testing.assert_array_equal(host(d["slots"])[:len(slots)], slots)
    assert (host(d["slots"])[len(slots):] == -9).all()
    np.testing.assert_array_equal(host(d["table"]), table)
    if d["n"] is not None:
        assert int(d["n"]) == left


@pytest.mark.parametrize("B,page,seed", [(1, 16, 0), (2, 256, 1), (5, 32, 2), (17, 64, 3), (64, 16, 4), (65, 128, 5),
                                         (255, 16, 6), (256, 32, 7)])
def test_against_the_oracle(api, bank, B, page, seed):
    """Batches with every kind of entry: unused places, lengths that do not fit,
    missing and foreign pages, a stack that runs out."""
    g = np.random.default_rng(seed)
    for trial in range(4):
        max_pages = int(g.integers(1, 40))
        topo = g.integers(-1 if trial else 0, len(TREES) + (1 if trial else 0), B)
        lens = g.integers(0, max(1, max_pages * page - (0 if trial > 1 else 256)), B)
        if trial == 3:
            lens[g.integers(0, B)] = -5
            lens[g.integers(0, B)] = 2 ** 31 - 1
            topo[g.integers(0, B)] = -2 ** 31
        n_pages = B * max_pages + 7
        table = g.permutation(n_pages)[:B * max_pages].reshape(B, max_pages).astype(np.int32)
        for b in range(B):   # what the prefix does not need is missing (mostly)
            keep = -(-max(0, int(lens[b])) // page) + int(g.integers(0, 2))
            table[b, keep:] = g.integers(-3, 0)
        if trial > 1:
            table[g.integers(0, B), :] = [n_pages, 2 ** 31 - 1][trial - 2]
            table[g.integers(0, B), :] = -1
        free = g.permutation(n_pages)[:max(1, B * 3)].astype(np.int32)
        if trial == 2:
            free[g.integers(0, free.size)] = n_pages
        n_free = [free.size, free.size // 2, free.size + 100, free.size][trial]
        rows = int(row_offsets(topo)[-1])
        rows_cap = max(1, [rows, rows + 11, rows - 40, rows][trial])
        say("page_map", B, page, trial, "rows", rows, rows_cap)
        want = po.page_map(TREES, topo, lens, table, page, n_pages, rows_cap, free, n_free)
        d, go = run(api, bank, topo, lens, table, page, n_pages, rows_cap, free, n_free)
        go()
        check(d, want, rows_cap)
        # once more: the pages are there
        want = po.page_map(TREES, topo, lens, want[0], page, n_pages, rows_cap, free, want[4])
        go()
        check(d, want, rows_cap)


@pytest.mark.parametrize("n_free", [0, -4])
def test_without_free_pages(api, bank, n_free):
    topo, lens, page = [2, 0, 1], [31, 16, 32], 16
    table = np.array([[5, 3, 7, 1], [2, -1, -1, -1], [0, 6, 4, -1]], np.int32)
    for free in (None, np.arange(3, dtype=np.int32)):
        want = po.page_map(TREES, topo, lens, table, page, 8, 60, free, n_free)
        assert want[3].tolist() == [po.OK, po.FULL, po.OK]
        d, go = run(api, bank, topo, lens, table, page, 8, 60, free, n_free)
        go()
        check(d, want, 60)


def test_empty_prefix_takes_every_page(api, bank):
    topo, lens, page = [5, 3, 0], [0, 0, 0], 16
    table = np.full((3, 16), -1, np.int32)
    free = np.arange(40, dtype=np.int32)[::-1].copy()
    want = po.page_map(TREES, topo, lens, table, page, 40, 300, free, 40)
    assert want[4] == 40 - 16 - 2 - 1
    d, go = run(api, bank, topo, lens, table, page, 40, 300, free, 40)
    go()
    check(d, want, 300)


def test_captured_and_on_another_stream(api, bank):
    """A graph of the call takes pages for whatever lengths it finds at each replay."""
    g = np.random.default_rng(9)
    topo, page, n_pages = [2, 1, -1, 4], 16, 64
    table = np.full((4, 12), -1, np.int32)
    free = g.permutation(n_pages).astype(np.int32)
    s = torch.cuda.Stream()
    d, go = run(api, bank, topo, [0, 0, 0, 0], table, page, n_pages, 120, free, n_pages)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        go()
    left = n_pages
    for lens in ([0, 0, 0, 0], [5, 1, 9, 3], [40, 2, 9, 70], [90, 30, 9, 100]):
        d["lens"].copy_(i32(lens))
        d["slots"].fill_(-9)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = po.page_map(TREES, topo, lens, table, page, n_pages, 120, free, left)
        check(d, want, 120)
        table, left = want[0], want[4]


def test_host_bank_and_shapes_are_refused(api, bank):
    z = torch.zeros(2, dtype=torch.int32, device="cuda")
    t = torch.zeros((2, 4), dtype=torch.int32, device="cuda")
    off = torch.zeros(3, dtype=torch.int32, device="cuda")
    with pytest.raises(api.EntmtpError):
        api.page_map(api.Bank(TREES, device=None), z, z, t, 16, 4, off, z, z)
    for bad in (dict(topo=z.long()), dict(lens=z[:1]), dict(table=t[:1]), dict(table=t.t()), dict(off=z), dict(status=off),
                dict(free=z), dict(n=z[:1]), dict(free=z, n=z)):
        a = {**dict(topo=z, lens=z, table=t, off=off, status=z, free=None, n=None), **bad}
        with pytest.raises(ValueError):
            api.page_map(bank, a["topo"], a["lens"], a["table"], 16, 4, a["off"], z, a["status"], free_pages=a["free"],
                         n_free=a["n"])
    with pytest.raises(api.EntmtpError):
        api.page_map(bank, z, z, t, 20, 4, off, z, z)
    assert dev is not None
