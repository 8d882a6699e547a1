"""GPU: positions and appended rows where offsets, sizes and values leave the ordinary.

Positions are whole numbers and compared as they are.  A query is computed in
fp64 from angles and sums in fp64, rounded to fp32 and then to bf16: by at most
2^-8 + 2^-24 of its value; the fp64 before it is off by less than 2^-40 of the
two numbers that a turn adds.  Keys are held bit for bit.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import entmtp_oracle as orc  # noqa: E402
from oracle import fp4_oracle as fo  # noqa: E402
from tests.fp4_helpers import D  # noqa: E402
from tests.paged_helpers import TREES, bits, host, i32, say, unbits  # noqa: E402
from tests.test_gpu_fp4_rows import append, append_case  # noqa: E402

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


def to_bf16(x):
    """64-bit numbers to fp32 and then to bf16 bits, subnormal ones too (the oracle's bits cut those short)."""
    return torch.from_numpy(x).to(torch.float32).to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)


def with_heads(c, q=None, k=None):
    """The case with other queries or keys on both sides."""
    if q is not None:
        c["q"], c["dq"] = q, bits(q)
    if k is not None:
        c["k"], c["dk"] = k, bits(k)
    return c


def check_queries(c, eps):
    got = orc.bf16_to_f64(unbits(c["qo"]))
    w = None if c["w"] is None else orc.bf16_to_f64(c["w"])[0]
    for r, pos in enumerate(c["pos"]):
        x = orc.bf16_to_f64(c["q"][r])
        ref = fo.norm_turn(x, int(pos), w, eps, c["theta"])
        y = np.abs(fo.norm_turn(x, 0, w, eps, 0.0))
        room = (2.0 ** -8 + 2.0 ** -24) * np.abs(ref) + 2.0 ** -40 * (y + np.roll(y, D // 2, -1)) + 2.0 ** -133
        err = np.abs(got[r] - ref)
        assert (err <= room).all(), (r, float((err / room).max()))


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("eps", [0.0, 1e-6])
def test_queries_and_keys_of_any_size_are_normed(api, fp4, eps):
    """Heads near both ends of bf16's range, queries as well as keys: their squares pass fp32's range on either side."""
    say("kv_append sizes", fp4, eps)
    c = append_case(21, 8, 4, 2, 16, fp4, True, 1e4, False)
    def sized(x):
        x = x.copy()
        x[0] = (x[0] & 0x807F) | (0x7F + 126 << 7)              # about 2^126
        x[1] = (x[1] & 0x807F) | (0x7F + 61 << 7)               # 2^61: 128 squares pass 2^128
        x[2, :, 77] = (0x7F + 64 << 7) | 0x8011                 # one of 2^64
        x[3] = (x[3] & 0x807F) | (0x7F - 100 << 7)              # 2^-100: squares below fp32
        x[4] = (x[4] & 0x807F) | 0x0080                         # 2^-126
        x[5] = x[5] & 0x803F | 1                                # subnormal
        x[6, :, ::2] = 0x7F7F                                   # the largest number beside ordinary ones
        return x
    with_heads(c, sized(c["q"]), sized(c["k"]))
    append(api, c, eps=eps)
    check_queries(c, eps)
    wk = orc.bf16_to_f64(c["w"])[1]
    kout = unbits(c["ko"])
    for r, pos in enumerate(c["pos"]):
        key = to_bf16(fo.norm_turn(orc.bf16_to_f64(c["k"][r]), int(pos), wk, eps, c["theta"]))
        if fp4:
            key = orc.f64_to_bf16_bits(fo.values(*fo.quantize(orc.bf16_to_f64(key))))
        zero = orc.bf16_to_f64(key) == 0
        np.testing.assert_array_equal(kout[r][~zero], key[~zero])
        assert (kout[r][zero] & 0x7FFF == 0).all()


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("theta", [0.0, 0.5, 1e4])
@pytest.mark.parametrize("odd", [0x7F80, 0xFF80, 0x7FC0])
def test_heads_that_are_not_finite_are_no_numbers_under_a_norm(api, fp4, theta, odd):
    """One infinity or NaN: the whole head is NaN, in the pool and the outputs; all others are what they were."""
    say("kv_append not finite", fp4, theta, hex(odd))
    c = append_case(23, 6, 9, 3, 16, fp4, True, theta, False)
    clean_q, clean_k = c["q"].copy(), c["k"].copy()
    append(api, c)
    want = {n: unbits(c[n]).copy() for n in ("qo", "ko", "vo")}
    pools = [host(c[n]).copy() if fp4 else unbits(c[n]).copy() for n in ("dkp", "dvp")]
    q, k = clean_q.copy(), clean_k.copy()
    q[1, 0, 3], q[2, 8, 127], k[3, 0, 64], k[4, 2, 31] = odd, odd, odd, odd
    with_heads(c, q, k)
    append(api, c)
    got = {n: orc.bf16_to_f64(unbits(c[n])) for n in ("qo", "ko", "vo")}
    for n, H, heads in (("qo", 9, [(1, 0), (2, 8)]), ("ko", 3, [(3, 0), (4, 2)]), ("vo", 3, [])):
        bad = np.zeros((6, H), bool)
        for at in heads:
            bad[at] = True
        assert np.isnan(got[n][bad]).all()
        np.testing.assert_array_equal(unbits(c[n])[~bad], want[n][~bad])
    now = [host(c[n]) if fp4 else unbits(c[n]) for n in ("dkp", "dvp")]
    np.testing.assert_array_equal(now[1], pools[1])
    hit = np.zeros((c["n_pages"], 16, 3), bool)
    for r, g in ((3, 0), (4, 2)):
        hit[c["slots"][r] // 16, c["slots"][r] % 16, g] = True
    hit = hit.transpose(0, 2, 1)
    if fp4:
        (codes, scales), (oc, os_) = fo.planes(now[0]), fo.planes(pools[0])
        assert (codes[hit] == 0).all() and (scales[hit] == 255).all()
        np.testing.assert_array_equal(codes[~hit], oc[~hit])
        np.testing.assert_array_equal(scales[~hit], os_[~hit])
    else:
        assert np.isnan(orc.bf16_to_f64(now[0][hit])).all()
        np.testing.assert_array_equal(now[0][~hit], pools[0][~hit])
