"""Shared pieces of the tests of the page-pool operators."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2606_27550_amd import synth  # noqa: E402

TREES = [[-1], synth.uniform_attach_tree(71, 7, 3), synth.uniform_attach_tree(72, 26, 4),
         synth.chain_tree(32), synth.uniform_attach_tree(73, 64, 5), synth.star_tree(256),
         synth.chain_tree(32) + [(7 * i) % 31 for i in range(98)]]


def say(*a):
    print("[gpu-test]", *a, flush=True)


def dev(a, dtype=None):
    a = np.ascontiguousarray(a if dtype is None else np.asarray(a, dtype))
    return torch.from_numpy(a).cuda()


def i32(a):
    return dev(a, np.int32)


def host(t):
    return t.detach().cpu().numpy()


def bits(a):
    """bf16 bit patterns on the GPU as a bf16 tensor."""
    return dev(np.asarray(a, np.uint16).view(np.int16)).view(torch.bfloat16)


def unbits(t):
    return host(t.view(torch.int16)).view(np.uint16)


def row_offsets(topo, trees=TREES):
    return np.concatenate([[0], np.cumsum([len(trees[t]) if 0 <= t < len(trees) else 0 for t in topo])]).astype(np.int32)


def block_table(g, topo, lens, page, spare=3, extra=2, trees=TREES):
    """Random pages for every prefix and tree: (table, pages in the pool)."""
    need = [-(-(L + len(trees[t])) // page) for t, L in zip(topo, lens)]
    order = g.permutation(sum(need) + spare).astype(np.int32)
    table = np.full((len(topo), max(need) + extra), -1, np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, sum(need) + spare
