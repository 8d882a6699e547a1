"""GPU: rows to 4 bits, rows appended to the pages, positions of tree rows and
compaction of 4-bit pages, against the oracle.

Codes, scale bytes and keys are held bit for bit.  A query is computed in fp32
and rounded once: of a head's 128 squares the sum is off by at most 128 roundings
(2^-24 each, half of that after the root), a dozen more roundings follow, and the
turn adds two products, so the error is at most 2^-8 |q| (the rounding to bf16)
plus 80 x 2^-24 (|y_c| + |y_{c + d/2}|).
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import entmtp_oracle as orc  # noqa: E402
from oracle import fp4_oracle as fo  # noqa: E402
from oracle import paged_oracle as po  # noqa: E402
from paper_2606_27550_amd import synth  # noqa: E402
from tests.fp4_helpers import D, quantize_fast  # noqa: E402
from tests.paged_helpers import TREES, bits, dev, host, i32, say, unbits  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_27550_amd import api as _api
    return _api


def u8(*shape, fill=0):
    return torch.full(shape, fill, dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("rows,n", [(1, 32), (3, 64), (7, 4096), (501, 160), (2, 8192)])
def test_quantize(api, rows, n):
    say("quantize_fp4", rows, n)
    x = synth.normal_bf16(np.random.default_rng(rows), (rows, n))
    codes, scales = u8(rows, n // 2), u8(rows, n // 32)
    api.quantize_fp4(bits(x), codes, scales)
    c, s = quantize_fast(orc.bf16_to_f64(x))
    np.testing.assert_array_equal(host(codes), c)
    np.testing.assert_array_equal(host(scales), s)


def test_quantize_every_bf16_number(api):
    """All 65536 patterns, each beside the largest of its group: a scale of its own, one of its neighbour's, zeros, infinities."""
    every = np.arange(65536, dtype=np.uint16)
    for top in (0x0000, 0x3F80, 0x3FE0, 0x0003, 0x7F7F, 0x7F80):
        x = np.full((65536 // 31 + 1, 32), top, np.uint16)
        x[:, 1:].flat[:65536] = every
        codes, scales = u8(*x.shape[:1], 16), u8(*x.shape[:1], 1)
        api.quantize_fp4(bits(x), codes, scales)
        with np.errstate(invalid="ignore"):
            c, s = fo.quantize(orc.bf16_to_f64(x))
        np.testing.assert_array_equal(host(codes), c)
        np.testing.assert_array_equal(host(scales), s)


def to_bf16(x):
    """64-bit numbers to fp32 and then to bf16 bits."""
    return orc.f64_to_bf16_bits(x.astype(np.float32).astype(np.float64))


def append_case(seed, rows, Hq, Hkv, page, fp4, norm, theta, strided, far=0):
    g = np.random.default_rng(seed)
    n_pages = -(-rows // page) + 3
    qkv = synth.normal_bf16(g, (rows, Hq + 2 * Hkv, D))
    c = dict(qkv=qkv, q=qkv[:, :Hq], k=qkv[:, Hq:Hq + Hkv], v=qkv[:, Hq + Hkv:],
             pos=(g.integers(0, 5000, rows) + far).astype(np.int32), slots=g.permutation(n_pages * page)[:rows].astype(np.int32),
             w=synth.normal_bf16(g, (2, D)) if norm else None, n_pages=n_pages, page=page, Hq=Hq, Hkv=Hkv, fp4=fp4, theta=theta)
    t = bits(qkv)
    part = (lambda a, b: t[:, a:b]) if strided else (lambda a, b: t[:, a:b].contiguous())
    c["dq"], c["dk"], c["dv"] = part(0, Hq), part(Hq, Hq + Hkv), part(Hq + Hkv, Hq + 2 * Hkv)
    c["dw"] = (None, None) if not norm else (bits(c["w"][0]), bits(c["w"][1]))
    if fp4:
        c["kp"], c["vp"] = (g.integers(0, 256, (n_pages, Hkv, page * 68), dtype=np.uint8) for _ in "kv")
        c["dkp"], c["dvp"] = dev(c["kp"]), dev(c["vp"])
    else:
        c["kp"], c["vp"] = (synth.normal_bf16(g, (n_pages, Hkv, page, D)) for _ in "kv")
        c["dkp"], c["dvp"] = bits(c["kp"]), bits(c["vp"])
    for n, H in (("qo", Hq), ("ko", Hkv), ("vo", Hkv)):
        c[n] = torch.full((rows, H, D), 7.0, dtype=torch.bfloat16, device="cuda")
    return c


def append(api, c, eps=1e-6, stream=None, q=True, held=True):
    f = api.kv_append_paged_fp4 if c["fp4"] else api.kv_append_paged
    f(c["dq"] if q else None, c["dk"], c["dv"], i32(c["pos"]), i32(c["slots"]), c["theta"], c["qo"] if q else None, c["dkp"],
      c["dvp"], q_norm=c["dw"][0] if q else None, k_norm=c["dw"][1], eps=eps, k_out=c["ko"] if held else None,
      v_out=c["vo"] if held else None, stream=stream)


def check_append(c, eps=1e-6, q=True, held=True):
    qo, ko, vo = unbits(c["qo"]), unbits(c["ko"]), unbits(c["vo"])
    kp, vp = c["kp"].copy(), c["vp"].copy()
    n_slots, page = c["n_pages"] * c["page"], c["page"]
    wq, wk = (None, None) if c["w"] is None else orc.bf16_to_f64(c["w"])
    planes = {id(p): fo.planes(p) for p in (kp, vp)} if c["fp4"] else None
    for r, (pos, slot) in enumerate(zip(c["pos"], c["slots"])):
        if pos < 0:
            assert (qo[r] == 0x40E0).all() and (ko[r] == 0x40E0).all() and (vo[r] == 0x40E0).all()
            continue
        x = orc.bf16_to_f64(c["q"][r])
        ref = fo.norm_turn(x, int(pos), wq, eps, c["theta"])
        y = np.abs(fo.norm_turn(x, 0, wq, eps, 0.0))
        if q:
            room = 2.0 ** -8 * np.abs(ref) + 80 * 2.0 ** -24 * (y + np.roll(y, D // 2, -1))
            assert (np.abs(orc.bf16_to_f64(qo[r]) - ref) <= room).all(), r
        else:
            assert (qo[r] == 0x40E0).all()
        key = to_bf16(fo.norm_turn(orc.bf16_to_f64(c["k"][r]), int(pos), wk, eps, c["theta"]))
        for row, out, pool in ((key, ko, kp), (c["v"][r], vo, vp)):
            codes = None
            if c["fp4"]:
                codes, scales = quantize_fast(orc.bf16_to_f64(row))
                row = orc.f64_to_bf16_bits(fo.values(codes, scales))
            if held:
                zero = orc.bf16_to_f64(row) == 0
                np.testing.assert_array_equal(out[r][~zero], row[~zero])
                assert (out[r][zero] & 0x7FFF == 0).all()   # (the oracle keeps no sign of a zero)
            if not 0 <= slot < n_slots:
                continue
            if c["fp4"]:
                planes[id(pool)][0][slot // page, :, slot % page] = codes
                planes[id(pool)][1][slot // page, :, slot % page] = scales
            else:
                pool[slot // page, :, slot % page] = row
    if c["fp4"]:
        np.testing.assert_array_equal(host(c["dkp"]), fo.join(*planes[id(kp)]))
        np.testing.assert_array_equal(host(c["dvp"]), fo.join(*planes[id(vp)]))
    else:
        np.testing.assert_array_equal(unbits(c["dkp"]), kp)
        np.testing.assert_array_equal(unbits(c["dvp"]), vp)


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("rows,Hq,Hkv,page,norm,theta,strided", [
    (1, 1, 1, 16, True, 1e4, False), (1, 32, 8, 64, True, 1e4, True), (3, 7, 7, 16, True, 5e5, True), (26, 32, 8, 32, False, 1e4, True),
    (17, 9, 3, 128, True, 0.0, False), (5, 8, 1, 256, False, 0.0, True), (33, 28, 4, 16, True, 0.5, True),
    (130, 5, 5, 16, True, 1e4, False), (700, 4, 2, 32, True, 1e4, True)])
def test_append(api, fp4, rows, Hq, Hkv, page, norm, theta, strided):
    say("kv_append", fp4, rows, Hq, Hkv, page, norm, theta, strided)
    c = append_case(rows + Hq, rows, Hq, Hkv, page, fp4, norm, theta, strided)
    append(api, c)
    check_append(c)


@pytest.mark.parametrize("fp4", [False, True])
def test_many_rows(api, fp4):
    """More rows than wavefronts that are in flight together: each takes all groups of a row."""
    say("kv_append many rows", fp4)
    c = append_case(5, 4300, 3, 1, 64, fp4, True, 1e4, True)
    append(api, c)
    check_append(c)


@pytest.mark.parametrize("fp4", [False, True])
def test_rows_without_place(api, fp4):
    """Rows without a position are left alone; slots outside the pool are not written, their outputs are."""
    say("kv_append without place", fp4)
    c = append_case(9, 40, 8, 2, 16, fp4, True, 1e4, True)
    c["pos"][::3] = -1
    c["pos"][1] = -2 ** 31
    c["slots"][5:30:4] = [-1, c["n_pages"] * 16, 2 ** 31 - 1, -2 ** 31, -7, c["n_pages"] * 16 + 5, -1]
    append(api, c)
    check_append(c)


@pytest.mark.parametrize("fp4", [False, True])
def test_far_positions_and_no_queries(api, fp4):
    say("kv_append far", fp4)
    c = append_case(11, 20, 8, 2, 16, fp4, True, 1e4, True, far=2 ** 31 - 5001)
    append(api, c, q=False, held=False)
    check_append(c, q=False, held=False)


@pytest.mark.parametrize("fp4", [False, True])
def test_in_place(api, fp4):
    """Outputs may be the inputs where those are dense."""
    say("kv_append in place", fp4)
    c = append_case(13, 29, 8, 2, 16, fp4, True, 1e4, False)
    c["qo"], c["ko"], c["vo"] = c["dq"], c["dk"], c["dv"]
    append(api, c)
    check_append(c)


def test_values_that_are_not_finite(api):
    """A group with one is no number; the others of its row, and other heads, are what they were."""
    c = append_case(15, 4, 2, 2, 16, True, False, 0.0, False)
    k, v = c["qkv"][:, 2:4].copy(), c["qkv"][:, 4:].copy()
    k[1, 0, 40], v[2, 1, 127] = 0x7F80, 0x7FC0
    c["dk"], c["dv"] = bits(k), bits(v)
    append(api, c)
    for x, pool, out in ((k, c["dkp"], c["ko"]), (v, c["dvp"], c["vo"])):
        with np.errstate(invalid="ignore"):
            codes, scales = fo.quantize(orc.bf16_to_f64(x))
        pc, ps = fo.planes(host(pool))
        for r, s in enumerate(c["slots"]):
            np.testing.assert_array_equal(pc[s // 16, :, s % 16], codes[r])
            np.testing.assert_array_equal(ps[s // 16, :, s % 16], scales[r])
        np.testing.assert_array_equal(orc.bf16_to_f64(unbits(out)), fo.values(codes, scales))
    assert (fo.planes(host(c["dkp"]))[1] == 255).sum() >= 1


def test_small_and_large_norms(api):
    """Heads near the ends of bf16's range: the norm's sum of squares stays finite in fp64, zeros give zeros."""
    c = append_case(17, 6, 2, 2, 16, True, True, 1e4, False)
    k = c["qkv"][:, 2:4].copy()
    k[0] = 0
    k[1] = (k[1] & 0x807F) | 0x7E80           # about 2^126
    k[2] = (k[2] & 0x807F) | 0x0100           # about 2^-125
    c["k"], c["dk"] = k, bits(k)
    append(api, c)
    check_append(c)


@pytest.mark.parametrize("topo,lens,behind", [([0], [0], 0), ([2, 1, 4], [5, 0, 70000], 3), ([5, -1, 6, 99, 3], [1, 2, 3, 4, 5], 300),
                                              ([1, 2], [-1, 2 ** 31 - 1], 0)])
def test_positions(api, topo, lens, behind):
    say("tree_positions", topo, lens)
    T = [len(TREES[t]) if 0 <= t < len(TREES) else 0 for t in topo]
    off = np.concatenate([[0], np.cumsum(T)]).astype(np.int32)
    pos = torch.full((int(off[-1]) + behind,), 77, dtype=torch.int32, device="cuda")
    bank = api.Bank(TREES)
    api.tree_positions(bank, i32(topo), i32(lens), i32(off), pos)
    want = np.full(pos.numel(), -1, np.int32)
    for b, t in enumerate(topo):
        if T[b] and 0 <= lens[b] <= 2 ** 31 - 257:
            want[off[b]:off[b] + T[b]] = lens[b] + np.array(orc.depths(TREES[t]))
    np.testing.assert_array_equal(host(pos), want)


def test_positions_of_sequences_without_work(api):
    """With the plan's trees (-1: none) a sequence keeps its rows, without positions; rows past the end are not written."""
    bank = api.Bank(TREES)
    off = np.array([0, 26, 33, 33, 97], np.int32)
    pos = torch.full((60,), 77, dtype=torch.int32, device="cuda")
    api.tree_positions(bank, i32([2, -1, 0, 4]), i32([3, 4, 5, 6]), i32(off), pos)
    want = np.full(60, -1)
    want[:26] = 3 + np.array(orc.depths(TREES[2]))
    np.testing.assert_array_equal(host(pos), want)   # (the last tree does not fit its rows)


def test_positions_with_rows_before_and_wild_offsets(api):
    """Rows before the first sequence's have no position; offsets outside the rows, down to the lowest number, write nothing."""
    bank = api.Bank(TREES)
    pos = torch.full((40,), 77, dtype=torch.int32, device="cuda")
    api.tree_positions(bank, i32([0, 0]), i32([9, 4]), i32([5, 6, 7]), pos)
    want = np.full(40, -1)
    want[5], want[6] = 9, 4
    np.testing.assert_array_equal(host(pos), want)
    low, high = -2 ** 31, 2 ** 31 - 1
    for off in ([7, low], [low, high], [high, low], [high, high], [-3, 5]):
        room = torch.full((400,), 77, dtype=torch.int32, device="cuda")
        api.tree_positions(bank, i32([2]), i32([9]), i32(off), room[:40])
        assert (host(room)[40:] == 77).all() and (host(room)[:40] <= 0).sum() + (host(room)[:40] == 77).sum() == 40


@pytest.mark.parametrize("off", [[7, -2 ** 31], [-2 ** 31, 2 ** 31 - 1], [2 ** 31 - 1, -2 ** 31], [-1, 9]])
def test_compact_with_wild_offsets(api, off):
    pools = [np.random.default_rng(3).integers(0, 256, (4, 2, 16 * 68), dtype=np.uint8) for _ in "kv"]
    d = [dev(p) for p in pools]
    api.kv_compact_paged_fp4(i32([[0, 2, 3]]), i32([2]), i32(off), i32(np.arange(20)), *d)
    for p, t in zip(pools, d):
        np.testing.assert_array_equal(host(t), p)


@pytest.mark.parametrize("layers,page,cap", [(1, 16, 32), (3, 64, 5), (2, 256, 17)])
def test_compact(api, layers, page, cap):
    say("kv_compact_paged_fp4", layers, page, cap)
    g = np.random.default_rng(layers)
    topo, Hkv, n_pages = [4, 2, 3, 1], 3, 40
    off = np.concatenate([[0], np.cumsum([len(TREES[t]) for t in topo])]).astype(np.int32)
    slots = g.permutation(n_pages * page)[:off[-1]].astype(np.int32)
    slots[3] = -1
    slots[off[1] + 1] = n_pages * page
    path, a = np.full((4, cap), -1, np.int32), np.zeros(4, np.int32)
    for b, t in enumerate(topo):
        chain = orc.ancestors_or_self(TREES[t], len(TREES[t]) - 1)
        chain = list(chain)[:cap]
        path[b, :len(chain)], a[b] = chain, len(chain) - 1
    a[3] = -1
    a[2] = 1000   # (clamped)
    pools = [g.integers(0, 256, (layers, n_pages, Hkv, page * 68), dtype=np.uint8) for _ in "kv"]
    d = [dev(p if layers > 1 else p[0]) for p in pools]
    api.kv_compact_paged_fp4(i32(path), i32(a), i32(off), i32(slots), *d)
    for p, t in zip(pools, d):
        parts = [po.kv_compact_paged(x, path, a, off, slots) for x in fo.planes(p)]
        np.testing.assert_array_equal(host(t).reshape(p.shape), fo.join(*parts))


def test_streams(api):
    """On a stream of its own, behind work that makes the inputs there."""
    c = append_case(19, 33, 8, 2, 16, True, True, 1e4, True)
    side = torch.cuda.Stream()
    pos, slots = i32(c["pos"]), i32(c["slots"])
    src = [t.clone() for t in (c["dq"], c["dk"], c["dv"])]
    into = [torch.zeros_like(t) for t in src]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            for a, b in zip(into, src):
                a.copy_(b)
        api.kv_append_paged_fp4(*into, pos, slots, 1e4, c["qo"], c["dkp"], c["dvp"], q_norm=c["dw"][0], k_norm=c["dw"][1],
                                eps=1e-6, k_out=c["ko"], v_out=c["vo"])
    side.synchronize()
    check_append(c)
