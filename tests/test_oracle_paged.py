"""Pins of the oracle of the page-pool operators: hand-worked cases, and
agreement with the oracle of the dense operators."""
import numpy as np

from oracle import entmtp_oracle as orc
from oracle import paged_oracle as po
from paper_2606_27550_amd import synth


def test_page_map_by_hand():
    trees = [[-1], [-1, 0, 0]]
    table = np.array([[4, -1, -1], [-1, -1, -1], [2, 0, -1], [1, -1, -1]], np.int32)
    # sequence 0: positions 15..17 (page 4, one new), 1: unused, 2: 20, 3: 14..16 (one new)
    got = po.page_map(trees, [1, -1, 0, 1], [15, 0, 20, 14], table, 16, 9, 20, np.array([7, 5, 8]), 3)
    assert got[0].tolist() == [[4, 8, -1], [-1] * 3, [2, 0, -1], [1, 5, -1]]
    assert got[1].tolist() == [0, 3, 3, 4, 7]
    assert got[2].tolist() == [79, 128, 129, 4, 30, 31, 80]
    assert got[3].tolist() == [po.OK, po.NONE, po.OK, po.OK] and got[4] == 1
    # one free page: the first takes it, the last goes without
    got = po.page_map(trees, [1, -1, 0, 1], [15, 0, 20, 14], table, 16, 9, 20, np.array([7, 5, 8]), 1)
    assert got[3].tolist() == [po.OK, po.NONE, po.OK, po.FULL] and got[4] == 0
    assert got[0][0, 1] == 7 and got[2][4:].tolist() == [-1] * 3


def test_page_map_statuses():
    trees = [[-1, 0]]
    table = np.array([[0, 9], [-1, 1], [2, -1], [3, 4]], np.int32)
    got = po.page_map(trees, [0, 0, 0, 0], [15, 3, 31, -1], table, 16, 9, 6, np.array([5]), 1)
    assert got[3].tolist() == [po.BAD, po.BAD, po.RANGE, po.RANGE] and got[1].tolist() == [0, 2, 4, 6, 6]


def test_compact_equals_the_dense_oracle():
    g = np.random.default_rng(1)
    Hkv, d, L, page = 2, 8, 21, 16
    tree = synth.uniform_attach_tree(5, 12, 4)
    dense = g.integers(0, 2 ** 16, (2, Hkv, 48, d)).astype(np.uint16)
    table = np.array([5, 1, 3])
    pool = np.zeros((2, 6, Hkv, page, d), np.uint16)
    for i, pg in enumerate(table):
        pool[:, pg] = dense[:, :, i * page:(i + 1) * page]
    slots = np.array([table[(L + i) // page] * page + (L + i) % page for i in range(12)])
    path = orc.ancestors_or_self(tree, 11)
    k, v = dense[0].copy(), dense[1].copy()
    orc_k, orc_v = orc.kv_compact(k, v, L, path)
    got = po.kv_compact_paged(pool, np.array([path]), [len(path) - 1], [0, 12], slots)
    for ref, layer in ((orc_k, 0), (orc_v, 1)):
        flat = np.concatenate([got[layer, p] for p in table], axis=1)
        np.testing.assert_array_equal(flat[:, :L + len(path)], ref[:, :L + len(path)])


def test_attention_equals_the_dense_oracle():
    tree = synth.uniform_attach_tree(6, 9, 3)
    L, page, cap = 37, 16, 48
    inp = synth.attn_inputs(6, 9, 4, 2, 128, L, cap)
    ref, rk, _ = orc.tree_attention(inp.q, inp.k_tree, inp.v_tree, inp.k_cache, inp.v_cache, L, tree, 0.1, 10000.0)
    table = [4, 0, 2]
    kp, vp = np.zeros((5, 2, page, 128), np.uint16), np.zeros((5, 2, page, 128), np.uint16)
    for i, pg in enumerate(table):
        kp[pg], vp[pg] = inp.k_cache[:, i * page:(i + 1) * page], inp.v_cache[:, i * page:(i + 1) * page]
    out, keys, off = po.tree_attention_paged(inp.q, inp.k_tree, inp.v_tree, kp, vp, table, L, tree, 0.1, 10000.0)
    np.testing.assert_allclose(out, ref, rtol=0, atol=1e-12)
    np.testing.assert_array_equal(keys.transpose(1, 0, 2), rk[:, L:L + 9])
    assert (off > 0).all()
    # a wide window, a huge cap and no slope change nothing
    same = po.tree_attention_paged(inp.q, inp.k_tree, inp.v_tree, kp, vp, table, L, tree, 0.1, 10000.0, softcap=1e6,
                                   window=L + 9, slopes=np.zeros(4))[0]
    np.testing.assert_allclose(same, ref, rtol=0, atol=1e-9)


def test_attention_options_by_hand():
    """A window of one leaves the node itself; a steep slope too; a tiny cap makes every score alike."""
    tree = [-1, 0, 0]
    inp = synth.attn_inputs(7, 3, 2, 1, 128, 5, 16)
    kp, vp = inp.k_cache[None, :, :16], inp.v_cache[None, :, :16]
    args = (inp.q, inp.k_tree, inp.v_tree, kp, vp, [0], 5, tree, 0.1, 0.0)
    own = orc.bf16_to_f64(inp.v_tree)[:, 0]
    for kw in (dict(window=1), dict(slopes=np.array([1e4, 1e4]))):
        out = po.tree_attention_paged(*args, **kw)[0]
        for h in range(2):
            np.testing.assert_allclose(out[:, h], own, atol=1e-12)
    out = po.tree_attention_paged(*args, softcap=1e-9)[0]
    pre = orc.bf16_to_f64(inp.v_cache)[0, :5]
    np.testing.assert_allclose(out[2, 0], np.concatenate([pre, own[[0, 2]]]).mean(0), atol=1e-6)


def test_adjusted_row_by_hand():
    z = np.array([2.0, -2.0, 1.0, 3.0, 0.0])
    h = np.array([1, po.SEEN, 0, 0, 2], np.int64).astype(np.int32)
    tree, tok = [-1, 0, 1], [9, 2, 2]
    got = po.adjusted_row(z, tree, 2, tok, [2.0, 0.5, 0.25, 1.0], h, np.array([0, 0, 0, 1.0, 0]), np.array([1, 1, 1, 1, 0], bool))
    # 0: said once; 1: in the prompt only; 2: drafted twice on the path; 3: a bias; 4: forbidden
    np.testing.assert_allclose(got, [1 - 0.5 - 0.25, -4, 0.5 - 1 - 0.25, 4, -np.inf])
    assert po.row_stats(got, 1.0)[2] == 3
    assert po.row_stats(np.full(3, -np.inf), 1.0) == (0.0, 0.0, -1)


def test_history_by_hand():
    h = np.zeros((2, 5), np.int32)
    h = po.history_prompt(h, np.array([9, 4, 4, -1, 2]), [1, 4, 5])
    assert (h < 0).tolist() == [[False] * 4 + [True], [False, False, True, False, False]]
    h = po.history_accept(h, [0, 3, 4], np.array([0, 4, 4, 1]), np.array([[0, 1, 2], [0, -1, -1]]), [2, -1], [4, 0])
    assert (h & 0x7FFFFFFF).tolist() == [[0, 0, 0, 0, 3], [0] * 5]
