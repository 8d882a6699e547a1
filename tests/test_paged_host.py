"""Host-side refusals of the operators over a page pool (no GPU): every bad
size, missing pointer or unsupported shape comes back as the documented status
before anything is launched."""
import ctypes

import pytest

from paper_2606_27550_amd import api

P = 1 << 20            # a non-NULL, aligned address that no refused call touches
ODD = P + 4


@pytest.fixture(scope="module")
def bank():
    return api.Bank([[-1, 0, 0], [-1]], device=None)


def refused(rc, code):
    assert rc == code, (rc, api.last_error())
    assert api.last_error()


def call(name, base, **change):
    args = dict(base, **change)
    return getattr(api.lib, name)(*args.values())


MAP = dict(bank=None, B=2, topo=P, prefix_len=P, table=P, max_pages=8, page=16, n_pages=4, free=P, free_cap=4,
           n_free=P, rows_cap=9, row_off=P, slot_map=P, status=P, stream=None)


@pytest.mark.parametrize("change,code", [
    (dict(B=0), api.EINVAL), (dict(B=257), api.EINVAL), (dict(topo=None), api.EINVAL),
    (dict(prefix_len=None), api.EINVAL), (dict(table=None), api.EINVAL), (dict(row_off=None), api.EINVAL),
    (dict(slot_map=None), api.EINVAL), (dict(status=None), api.EINVAL), (dict(free=None), api.EINVAL),
    (dict(n_free=None), api.EINVAL), (dict(free_cap=0), api.EINVAL), (dict(rows_cap=0), api.EINVAL),
    (dict(page=8), api.EINVAL), (dict(page=24), api.EINVAL), (dict(page=512), api.EINVAL),
    (dict(page=0), api.EINVAL), (dict(n_pages=0), api.EINVAL), (dict(n_pages=1 << 27), api.ERANGE),
    (dict(max_pages=0), api.ERANGE), (dict(max_pages=1 << 27), api.ERANGE), (dict(), api.EINVAL)])
def test_page_map_refusals(bank, change, code):
    # (the last one: a bank without a device arena)
    refused(call("entmtp_page_map", MAP, **{"bank": bank.handle, **change}), code)


def test_page_map_needs_a_bank():
    refused(call("entmtp_page_map", MAP), api.EINVAL)


COMPACT = dict(B=2, path=P, path_cap=5, accept_len=P, row_off=P, slot_map=P, rows=9, k=P, v=P, layers=2,
               stride=4 * 2 * 16 * 128, n_pages=4, Hkv=2, page=16, d=128, stream=None)


@pytest.mark.parametrize("change,code", [
    (dict(B=0), api.EINVAL), (dict(B=300), api.EINVAL), (dict(path=None), api.EINVAL),
    (dict(accept_len=None), api.EINVAL), (dict(row_off=None), api.EINVAL), (dict(slot_map=None), api.EINVAL),
    (dict(k=None), api.EINVAL), (dict(v=None), api.EINVAL), (dict(path_cap=0), api.EINVAL),
    (dict(rows=0), api.EINVAL), (dict(layers=0), api.EINVAL), (dict(Hkv=0), api.EINVAL), (dict(d=0), api.EINVAL),
    (dict(d=12), api.EINVAL), (dict(d=264), api.EINVAL), (dict(page=48), api.EINVAL), (dict(n_pages=0), api.EINVAL),
    (dict(n_pages=1 << 28), api.ERANGE), (dict(stride=4 * 2 * 16 * 128 - 8), api.EINVAL),
    (dict(layers=1, stride=4), api.EINVAL), (dict(k=ODD), api.EINVAL), (dict(v=ODD), api.EINVAL)])
def test_compact_refusals(change, code):
    refused(call("entmtp_kv_compact_paged", COMPACT, **change), code)


ADJUST = dict(bank=None, B=2, topo=P, row_off=P, rows=9, tok=P, logits=P, V=100, params=P, history=P, bias=P,
              n_bias=1, bias_idx=P, mask=P, n_masks=1, words=4, mask_idx=P, out=P, entropy=P, top1p=P, argmax=P,
              ws=P, ws_bytes=1 << 20, stream=None)


@pytest.mark.parametrize("change,code", [
    (dict(B=0), api.EINVAL), (dict(B=257), api.EINVAL), (dict(topo=None), api.EINVAL), (dict(row_off=None), api.EINVAL),
    (dict(tok=None), api.EINVAL), (dict(logits=None), api.EINVAL), (dict(params=None), api.EINVAL),
    (dict(rows=0), api.EINVAL), (dict(V=0), api.EINVAL), (dict(V=2 ** 31 - 1), api.ERANGE),
    (dict(bias=None), api.EINVAL), (dict(bias_idx=None), api.EINVAL), (dict(n_bias=0), api.EINVAL),
    (dict(mask=None), api.EINVAL), (dict(mask_idx=None), api.EINVAL), (dict(n_masks=0), api.EINVAL),
    (dict(words=3), api.EINVAL), (dict(logits=ODD), api.EINVAL), (dict(out=ODD), api.EINVAL),
    (dict(history=ODD), api.EINVAL), (dict(params=ODD), api.EINVAL), (dict(ws=None), api.EINVAL),
    (dict(ws_bytes=0), api.ENOSPC), (dict(), api.EINVAL)])
def test_adjust_refusals(bank, change, code):
    refused(call("entmtp_logit_adjust", ADJUST, **{"bank": bank.handle, **change}), code)


def test_adjust_workspace():
    assert api.logit_adjust_workspace(0, 10) == 0 and api.logit_adjust_workspace(10, 0) == 0
    for rows, V in ((1, 1), (26, 32000), (1024, 128256)):
        need = api.logit_adjust_workspace(rows, V)
        assert need >= 16 * rows
        refused(call("entmtp_logit_adjust", ADJUST, rows=rows, V=V, words=V // 32 + 1, ws_bytes=need - 1), api.ENOSPC)


PROMPT = dict(tokens=P, n=10, off=P, B=2, V=100, history=P, stream=None)
ACCEPT = dict(B=2, row_off=P, tok=P, rows=9, path=P, path_cap=5, accept_len=P, bonus=P, V=100, history=P, stream=None)


@pytest.mark.parametrize("name,base,change", [
    ("prompt", PROMPT, c) for c in (dict(B=0), dict(B=257), dict(off=None), dict(history=None), dict(tokens=None),
                                    dict(n=-1), dict(n=2 ** 31 - 1), dict(V=0))] + [
    ("accept", ACCEPT, c) for c in (dict(B=0), dict(B=257), dict(row_off=None), dict(tok=None), dict(path=None),
                                    dict(accept_len=None), dict(bonus=None), dict(history=None), dict(rows=0),
                                    dict(V=0), dict(path_cap=0))])
def test_history_refusals(name, base, change):
    refused(call("entmtp_token_history_" + name, base, **change), api.EINVAL)


def test_no_prompt_tokens_is_no_launch():
    assert call("entmtp_token_history_prompt", PROMPT, tokens=None, n=0) == api.OK


def test_binding_refuses_host_tensors(bank):
    torch = pytest.importorskip("torch")
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        api.page_map(bank, i, i, i[None], 16, 4, i, i, i)
    with pytest.raises(ValueError):
        api.token_history_prompt(i, i, i[None])
    with pytest.raises(ValueError):
        api.kv_compact_paged(i[None], i, i, i, i, i)
    with pytest.raises(ValueError):
        api.logit_adjust(bank, i, i, i, i, i, i, i, i, i, i)


def test_statuses_match_the_header():
    import os
    import re
    from tests.conftest import ROOT
    text = open(os.path.join(ROOT, "include", "entmtp.h")).read()
    for name in ("OK", "NONE", "RANGE", "FULL", "BAD"):
        assert int(re.search(rf"#define ENTMTP_PAGE_{name}\s+(\d+)", text)[1]) == getattr(api, "PAGE_" + name)
    assert int(re.search(r"#define ENTMTP_PAGED_B_MAX (\d+)", text)[1]) == api.PAGED_B_MAX
    assert ctypes.sizeof(ctypes.c_void_p) == 8


PLAN = dict(bank=None, B=2, topo=P, prefix_len=P, row_off=P, status=P, table=P, max_pages=8, page=16, n_pages=4,
            rows_cap=9, Hq=8, Hkv=2, window=0, bad=None, plan=P, plan_bytes=1 << 30, stream=None)
ATTN = dict(bank=None, B=2, plan=P, plan_bytes=1 << 30, q=P, kt=P, vt=P, kp=P, vp=P, n_pages=4, page=16, table=P,
            max_pages=8, slots=P, rows_cap=9, Hq=8, Hkv=2, d=128, scale=0.1, theta=1e4, softcap=0.0, window=0,
            slopes=None, out=P, ws=P, ws_bytes=1 << 30, stream=None)
BATCH = [(dict(B=0), api.EINVAL), (dict(B=257), api.EINVAL), (dict(rows_cap=0), api.EINVAL), (dict(Hq=0), api.EINVAL),
         (dict(Hkv=0), api.EINVAL), (dict(Hq=9), api.ERANGE), (dict(Hq=66, Hkv=2), api.ERANGE),
         (dict(Hq=257, Hkv=257), api.ERANGE), (dict(page=8), api.EINVAL), (dict(n_pages=0), api.EINVAL),
         (dict(n_pages=1 << 27), api.ERANGE), (dict(max_pages=0), api.ERANGE),
         (dict(max_pages=(1 << 27) - 1), api.ERANGE), (dict(window=-1), api.EINVAL), (dict(plan=None), api.EINVAL),
         (dict(plan=P + 16), api.EINVAL), (dict(table=None), api.EINVAL), (dict(), api.EINVAL)]


@pytest.mark.parametrize("change,code", BATCH + [(dict([(k, None)]), api.EINVAL) for k in
                                                 ("topo", "prefix_len", "row_off", "status")])
def test_plan_refusals(bank, change, code):
    refused(call("entmtp_tree_attn_paged_plan", PLAN, **{"bank": bank.handle, **change}), code)


@pytest.mark.parametrize("change,code", BATCH + [(dict([(k, v)]), api.EINVAL) for v in (None, ODD) for k in
                                                 ("q", "kt", "vt", "kp", "vp", "out")] + [
    (dict(slots=None), api.EINVAL), (dict(ws=ODD), api.EINVAL), (dict(d=64), api.EINVAL), (dict(scale=0.0), api.EINVAL),
    (dict(scale=float("nan")), api.EINVAL), (dict(scale=float("inf")), api.EINVAL), (dict(theta=-1.0), api.EINVAL),
    (dict(theta=float("inf")), api.EINVAL), (dict(softcap=-1.0), api.EINVAL), (dict(softcap=float("nan")), api.EINVAL),
    (dict(softcap=float("inf")), api.EINVAL), (dict(softcap=1e-42, scale=1.0), api.EINVAL),
    (dict(softcap=1025.0), api.EINVAL)])
def test_paged_attention_refusals(bank, change, code):
    refused(call("entmtp_tree_attn_paged", ATTN, **{"bank": bank.handle, **change}), code)


def test_paged_sizes(bank):
    size = lambda **c: (api.tree_attn_paged_plan_bytes(bank, *{**dict(B=2, rows=9, Hq=8, Hkv=2, mp=8, page=16), **c}.values()),  # noqa: E731
                        api.tree_attn_paged_workspace(bank, *{**dict(B=2, rows=9, Hq=8, Hkv=2, d=128, mp=8, page=16), **c}.values()))
    plan, ws = size()
    assert plan > 0 and ws == 0                       # 128 positions: never split
    assert size(mp=64)[1] > 0
    for bad in (dict(B=0), dict(B=257), dict(rows=0), dict(Hq=7), dict(Hkv=0), dict(mp=0), dict(page=17), dict(mp=1 << 27)):
        assert size(**bad) == (0, 0)
    assert api.tree_attn_paged_workspace(bank, 2, 9, 8, 2, 64, 64, 16) == 0
