"""Host-side refusals of the 4-bit operators and the append (no GPU)."""
import pytest

from paper_2606_27550_amd import api
from tests.test_paged_host import P, ODD, call, refused


@pytest.fixture(scope="module")
def bank():
    return api.Bank([[-1, 0, 0], [-1]], device=None)


QUANT = dict(x=P, rows=4, n=64, codes=P, scales=P, stream=None)


@pytest.mark.parametrize("change", [dict(x=None), dict(codes=None), dict(scales=None), dict(rows=0), dict(n=0), dict(n=48),
                                    dict(n=-32), dict(rows=1 << 60), dict(x=ODD), dict(codes=P + 2)])
def test_quantize_refusals(change):
    refused(call("entmtp_quantize_fp4", QUANT, **change), api.EINVAL)


POS = dict(bank=None, B=2, topo=P, prefix_len=P, row_off=P, rows=9, pos=P, stream=None)


@pytest.mark.parametrize("change", [dict(B=0), dict(B=257), dict(topo=None), dict(prefix_len=None), dict(row_off=None),
                                    dict(rows=0), dict(pos=None), dict(), dict(bank=None)])
def test_positions_refusals(bank, change):
    # (the last but one: a bank without a device arena)
    refused(call("entmtp_tree_positions", POS, **{"bank": bank.handle, **change}), api.EINVAL)


APPEND = dict(q=P, qs=1024, k=P, ks=256, v=P, vs=256, rows=5, Hq=8, Hkv=2, d=128, pos=P, slot_map=P, q_norm=P, k_norm=P,
              eps=1e-6, theta=1e4, q_out=P, kp=P, vp=P, n_pages=4, page=16, k_out=P, v_out=P, stream=None)


@pytest.mark.parametrize("name", ["entmtp_kv_append_paged", "entmtp_kv_append_paged_fp4"])
@pytest.mark.parametrize("change,code", [
    (dict(k=None), api.EINVAL), (dict(v=None), api.EINVAL), (dict(pos=None), api.EINVAL), (dict(slot_map=None), api.EINVAL),
    (dict(kp=None), api.EINVAL), (dict(vp=None), api.EINVAL), (dict(q=None), api.EINVAL), (dict(q_out=None), api.EINVAL),
    (dict(q=None, q_out=None), api.EINVAL), (dict(rows=0), api.EINVAL), (dict(Hq=0), api.EINVAL), (dict(Hkv=0), api.EINVAL),
    (dict(d=64), api.EINVAL), (dict(page=8), api.EINVAL), (dict(page=40), api.EINVAL), (dict(n_pages=0), api.EINVAL),
    (dict(n_pages=1 << 27), api.ERANGE), (dict(eps=-1.0), api.EINVAL), (dict(eps=float("nan")), api.EINVAL),
    (dict(theta=-1.0), api.EINVAL), (dict(theta=float("inf")), api.EINVAL), (dict(qs=1016), api.EINVAL),
    (dict(ks=252), api.EINVAL), (dict(ks=248), api.EINVAL), (dict(vs=0), api.EINVAL), (dict(vs=260), api.EINVAL),
    (dict(vs=1 << 41), api.EINVAL), (dict(Hq=1 << 20, qs=1 << 27), api.ERANGE)] +
    [({n: ODD}, api.EINVAL) for n in ("q", "k", "v", "q_norm", "k_norm", "q_out", "kp", "vp", "k_out", "v_out")])
def test_append_refusals(name, change, code):
    refused(call(name, APPEND, **change), code)


PLAN = dict(bank=None, B=2, topo=P, prefix_len=P, row_off=P, status=P, table=P, max_pages=8, page=16, n_pages=4, rows_cap=9,
            Hq=8, Hkv=2, window=0, bad=P, plan=P, plan_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("change,code", [
    (dict(B=0), api.EINVAL), (dict(B=257), api.EINVAL), (dict(topo=None), api.EINVAL), (dict(prefix_len=None), api.EINVAL),
    (dict(row_off=None), api.EINVAL), (dict(status=None), api.EINVAL), (dict(table=None), api.EINVAL),
    (dict(plan=None), api.EINVAL), (dict(plan=P + 16), api.EINVAL), (dict(page=8), api.EINVAL), (dict(n_pages=0), api.EINVAL),
    (dict(max_pages=0), api.ERANGE), (dict(rows_cap=0), api.EINVAL), (dict(Hq=9), api.ERANGE), (dict(Hq=66), api.ERANGE),
    (dict(Hkv=0), api.EINVAL), (dict(window=-1), api.EINVAL), (dict(), api.EINVAL)])
def test_plan_refusals(bank, change, code):
    refused(call("entmtp_tree_attn_paged_fp4_plan", PLAN, **{"bank": bank.handle, **change}), code)


ATTN = dict(bank=None, B=2, plan=P, plan_bytes=1 << 30, q=P, kp=P, vp=P, n_pages=4, page=16, table=P, max_pages=8, rows_cap=9,
            Hq=8, Hkv=2, d=128, scale=0.1, softcap=0.0, window=0, slopes=P, out=P, ws=P, ws_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("change,code", [
    (dict(B=0), api.EINVAL), (dict(plan=None), api.EINVAL), (dict(q=None), api.EINVAL), (dict(kp=None), api.EINVAL),
    (dict(vp=None), api.EINVAL), (dict(table=None), api.EINVAL), (dict(out=None), api.EINVAL), (dict(d=64), api.EINVAL),
    (dict(scale=0.0), api.EINVAL), (dict(scale=float("inf")), api.EINVAL), (dict(softcap=-1.0), api.EINVAL),
    (dict(softcap=1025.0), api.EINVAL), (dict(softcap=1e-30), api.EINVAL), (dict(window=-1), api.EINVAL),
    (dict(plan=P + 16), api.EINVAL), (dict(q=ODD), api.EINVAL), (dict(kp=ODD), api.EINVAL), (dict(vp=ODD), api.EINVAL),
    (dict(out=ODD), api.EINVAL), (dict(ws=ODD), api.EINVAL), (dict(Hq=9), api.ERANGE), (dict(page=24), api.EINVAL),
    (dict(max_pages=1 << 28), api.ERANGE), (dict(), api.EINVAL)])
def test_attention_refusals(bank, change, code):
    refused(call("entmtp_tree_attn_paged_fp4", ATTN, **{"bank": bank.handle, **change}), code)


def test_sizes(bank):
    for f in (api.tree_attn_paged_fp4_plan_bytes, lambda *a: api.tree_attn_paged_fp4_workspace(*a[:5], 128, *a[5:])):
        assert f(bank, 2, 9, 8, 2, 64, 16) > 0
        assert f(bank, 0, 9, 8, 2, 64, 16) == 0 and f(bank, 2, 9, 9, 2, 64, 16) == 0 and f(bank, 2, 9, 8, 2, 64, 20) == 0


COMPACT = dict(B=2, path=P, path_cap=5, accept_len=P, row_off=P, slot_map=P, rows=9, k=P, v=P, layers=2,
               stride=4 * 2 * 16 * 68, n_pages=4, Hkv=2, page=16, d=128, stream=None)


@pytest.mark.parametrize("change,code", [
    (dict(B=0), api.EINVAL), (dict(path=None), api.EINVAL), (dict(accept_len=None), api.EINVAL), (dict(row_off=None), api.EINVAL),
    (dict(slot_map=None), api.EINVAL), (dict(k=None), api.EINVAL), (dict(v=None), api.EINVAL), (dict(path_cap=0), api.EINVAL),
    (dict(rows=0), api.EINVAL), (dict(layers=0), api.EINVAL), (dict(Hkv=0), api.EINVAL), (dict(d=64), api.EINVAL),
    (dict(page=48), api.EINVAL), (dict(n_pages=1 << 28), api.ERANGE), (dict(stride=4 * 2 * 16 * 68 - 16), api.EINVAL),
    (dict(layers=1, stride=8), api.EINVAL), (dict(k=ODD), api.EINVAL), (dict(v=ODD), api.EINVAL), (dict(Hkv=1 << 17), api.ERANGE)])
def test_compact_refusals(change, code):
    refused(call("entmtp_kv_compact_paged_fp4", COMPACT, **change), code)


LOGITS = dict(hidden=P, codes=P, scales=P, T=3, hid=64, V=100, logits=P, stream=None)


@pytest.mark.parametrize("change", [dict(hidden=None), dict(codes=None), dict(scales=None), dict(logits=None), dict(T=0),
                                    dict(T=4097), dict(hid=0), dict(hid=48), dict(hid=65568), dict(V=0), dict(V=2 ** 31 - 1),
                                    dict(hidden=ODD), dict(codes=ODD), dict(logits=ODD)])
def test_logits_refusals(change):
    refused(call("entmtp_verify_logits_fp4", LOGITS, **change), api.EINVAL)


def test_binding_refuses_host_tensors(bank):
    torch = pytest.importorskip("torch")
    i = torch.zeros(4, dtype=torch.int32)
    bf, u8 = torch.zeros(4, 2, 128, dtype=torch.bfloat16), torch.zeros(4, 2, 16 * 68, dtype=torch.uint8)
    for f in (lambda: api.quantize_fp4(bf.view(8, 128), u8, u8), lambda: api.tree_positions(bank, i, i, i, i),
              lambda: api.kv_append_paged_fp4(bf, bf, bf, i, i, 1e4, bf, u8, u8),
              lambda: api.kv_append_paged(bf, bf, bf, i, i, 1e4, bf, bf, bf),
              lambda: api.tree_attn_paged_fp4(bank, u8, bf, u8, u8, i.view(2, 2), 0.1, bf, u8),
              lambda: api.kv_compact_paged_fp4(i.view(2, 2), i, i, i, u8, u8),
              lambda: api.verify_logits_fp4(bf.view(8, 128), u8.view(8, -1), u8, bf)):
        with pytest.raises(ValueError):
            f()
