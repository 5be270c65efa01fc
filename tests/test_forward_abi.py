"""Refusals of the calls around the forward (append, attention, logits): every
host-visible fault is reported before anything reaches a GPU, and nothing is
written.  Dummy addresses, never dereferenced, on hosts without a GPU only."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def sd():
    if torch.cuda.is_available():
        pytest.skip("error paths with dummy pointers run on CPU-only hosts")
    from paper_2510_22876_amd import specdec
    return specdec


A = 0x10000


def _a(i):
    return A + ((i + 1) << 24)


KV, QKV, QN, KN, IF, IDX, TAB, OUT, WS, ST, S, DR, BG, LN, PR, RP, PS, FQ, BI, BV, MK = (_a(i) for i in range(21))


def _kv(sd, data=KV, L=2, B=3, H=2, D=16, cap=64):
    return sd.KV(data, L, B, H, D, cap)


def _append(sd, paged, kv=None, **over):
    a = dict(qkv=QKV, dtype=1, T=4, Hq=4, q_norm=QN, k_norm=KN, eps=1e-6, inv_freq=IF, n_freq=8, adjacent=0, kv=kv or _kv(sd),
             layer=1, idx=(60, IDX), q_out=OUT, status=ST)
    if paged:
        a["idx"], a["B"] = (TAB, 4, IDX), 3
    a.update(over)
    head = (a["qkv"], a["dtype"]) + ((a["B"],) if paged else ())
    return (sd.lib.specdec_append_paged if paged else sd.lib.specdec_append_window)(
        *head, a["T"], a["Hq"], a["q_norm"], a["k_norm"], a["eps"], a["inv_freq"], a["n_freq"], a["adjacent"],
        ctypes.byref(a["kv"]) if a["kv"] != "none" else None, a["layer"], *a["idx"], a["q_out"], a["status"], None)


def _attend(sd, paged, kv=None, **over):
    a = dict(q=QKV, T=4, Hq=4, scale=0.25, kv=kv or _kv(sd), layer=0, idx=(60, IDX), out=OUT, ws=WS, ws_bytes=1 << 22, status=ST)
    if paged:
        a["idx"], a["B"] = (TAB, 4, IDX, 100), 3
    a.update(over)
    head = (a["q"],) + ((a["B"],) if paged else ())
    return (sd.lib.specdec_attend_paged if paged else sd.lib.specdec_attend_window)(
        *head, a["T"], a["Hq"], a["scale"], ctypes.byref(a["kv"]) if a["kv"] != "none" else None, a["layer"], *a["idx"],
        a["out"], a["ws"], a["ws_bytes"], a["status"], None)


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("call", [_append, _attend])
def test_cache_side_refusals(sd, call, paged):
    k = lambda **kw: _kv(sd, **kw)   # noqa: E731
    for over, code in [
            (dict(kv="none"), 1), (dict(T=0), 1), (dict(T=66), 1), (dict(layer=-1), 1), (dict(layer=2), 1), (dict(Hq=0), 1),
            (dict(Hq=3), 1), (dict(Hq=-2), 1), (dict(kv=k(D=264, cap=64)), 2), (dict(kv=k(D=12)), 2), (dict(kv=k(data=KV + 8)), 2),
            (dict(kv=k(data=None)), 1), (dict(kv=k(H=0)), 1), (dict(kv=k(cap=0)), 1), (dict(status=ST + 2), 2),
            (dict(status=KV + 64), 1)]:
        assert call(sd, paged, **over) == code, over
        assert sd.lib.specdec_last_error().decode() != ""
    if paged:
        idx = [((None, 4, IDX), 1), ((TAB, 0, IDX), 1), ((TAB, 1 << 25, IDX), 1), ((TAB, 4, None), 1), ((TAB + 2, 4, IDX), 2),
               ((TAB, 4, IDX + 1), 2)]
        if call is _attend:
            idx = [(i + (100,), code) for i, code in idx]
            idx += [((TAB, 4, IDX, 3), 1), ((TAB, 4, IDX, 257), 1), ((TAB, 4, IDX, 0), 1), ((TAB, 4, IDX, -1), 1)]
        else:
            assert call(sd, True, kv=k(cap=3), idx=(TAB, 1, IDX)) == 1     # the table holds less than the window
        for over, code in idx:
            assert call(sd, True, idx=over) == code, over
        for B, code in ((-1, 1), (65537, 1)):
            assert call(sd, True, B=B) == code
        assert call(sd, True, B=65536, T=17) == 1                          # B*T
        assert call(sd, True, B=0) == 0
    else:
        for over, code in [((3, IDX), 1), ((65, IDX), 1), ((1 << 25, IDX), 1), ((60, None), 1), ((60, IDX + 2), 2)]:
            assert call(sd, False, idx=over) == code, over
        assert call(sd, False, kv=k(B=0)) == 0


@pytest.mark.parametrize("paged", [False, True])
def test_append_refusals(sd, paged):
    for over, code in [
            (dict(dtype=5), 2), (dict(eps=-1.0), 1), (dict(eps=float("nan")), 1), (dict(eps=float("inf")), 1), (dict(n_freq=-1), 1),
            (dict(n_freq=9), 1), (dict(adjacent=2), 1), (dict(qkv=None), 1), (dict(q_out=None), 1), (dict(inv_freq=None), 1),
            (dict(qkv=QKV + 8), 2), (dict(q_out=OUT + 4), 2), (dict(q_norm=QN + 1), 2), (dict(k_norm=KN + 1), 2), (dict(inv_freq=IF + 2), 2),
            (dict(q_out=QKV + 256), 1), (dict(q_out=KV + 256), 1), (dict(qkv=KV + 256), 1), (dict(q_norm=OUT), 1),
            (dict(inv_freq=KV), 1)]:
        assert _append(sd, paged, **over) == code, over
    over = dict(idx=(TAB, 4, KV)) if paged else dict(idx=(60, KV))
    assert _append(sd, paged, **over) == 1                                 # the index tensor inside the cache
    if paged:
        assert _append(sd, True, idx=(OUT, 4, IDX)) == 1                   # the table inside q_out


@pytest.mark.parametrize("paged", [False, True])
def test_attend_refusals(sd, paged):
    for over, code in [
            (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1), (dict(q=None), 1), (dict(out=None), 1), (dict(q=QKV + 8), 2),
            (dict(out=OUT + 8), 2), (dict(out=QKV), 1), (dict(out=KV), 1), (dict(ws=None), 4), (dict(ws=WS + 8), 4),
            (dict(ws_bytes=0), 4), (dict(ws=OUT), 1), (dict(ws=KV), 1), (dict(ws=QKV), 1)]:
        assert _attend(sd, paged, **over) == code, over


def test_attend_workspace_bytes(sd):
    f = sd.attend_workspace_bytes
    assert f(1, 1, 32, 8, 128, 1000) > 0 and f(0, 1, 32, 8, 128, 1000) > 0
    for bad in [(-1, 1, 32, 8, 128, 1000), (1, 0, 32, 8, 128, 1000), (1, 66, 32, 8, 128, 1000), (1, 1, 31, 8, 128, 1000),
                (1, 1, 32, 0, 128, 1000), (1, 1, 32, 8, 4, 1000), (1, 1, 32, 8, 264, 1000), (1, 1, 32, 8, 100, 1000),
                (1, 4, 32, 8, 128, 3), (1, 1, 32, 8, 128, 1 << 25), (65537, 1, 32, 8, 128, 1000), (65536, 17, 4, 4, 64, 100)]:
        assert f(*bad) == 0, bad


def _logits(sd, **over):
    a = dict(logits=QKV, out=OUT, dtype=1, B=2, k=3, V=100, s=S, s_stride=20, width=15, draft=DR, begin=BG, lens=None, prompt=PR,
             rep=RP, pres=PS, freq=FQ, bias_ids=BI, bias=BV, n_bias=4, mask=MK, mask_stride=4, status=ST, stream=None)
    a.update(over)
    return sd.lib.specdec_process_logits(*a.values())


def test_logits_refusals(sd):
    for over, code in [
            (dict(B=-1), 1), (dict(B=65537), 1), (dict(k=-1), 1), (dict(k=65), 1), (dict(V=0), 1), (dict(dtype=3), 2),
            (dict(B=65536, k=63), 1), (dict(n_bias=-1), 1), (dict(n_bias=1025), 1), (dict(s_stride=0), 1), (dict(width=20), 1),
            (dict(width=-1), 1), (dict(mask_stride=3), 1), (dict(logits=None), 1), (dict(out=None), 1), (dict(s=None), 1),
            (dict(draft=None), 1), (dict(bias_ids=None), 1), (dict(bias=None), 1), (dict(logits=QKV + 1), 2), (dict(out=OUT + 1), 2),
            (dict(dtype=0, out=OUT + 2), 2), (dict(s=S + 2), 2), (dict(mask=MK + 1), 2), (dict(prompt=PR + 2), 2), (dict(status=ST + 1), 2),
            (dict(out=QKV + 2), 1), (dict(out=S), 1), (dict(out=MK), 1), (dict(out=BV), 1), (dict(status=OUT + 4), 1),
            (dict(status=RP), 1)]:
        assert _logits(sd, **over) == code, over
        assert sd.lib.specdec_last_error().decode() != ""
    assert _logits(sd, B=0) == 0


def test_wrappers_refuse_host_tensors(sd):
    kv = torch.zeros((1, 2, 1, 1, 16, 8), dtype=torch.bfloat16)
    i32 = torch.zeros(1, dtype=torch.int32)
    q = torch.zeros((1, 1, 1, 8), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        sd.specdec_append_window(torch.zeros((1, 1, 3, 8)), kv, 0, 4, i32, q)
    with pytest.raises(ValueError):
        sd.specdec_append_paged(torch.zeros((1, 1, 3, 8)), kv, 0, i32[None], i32, q)
    with pytest.raises(ValueError):
        sd.specdec_attend_window(q, kv, 0, 4, i32, q.clone(), i32)
    with pytest.raises(ValueError):
        sd.specdec_attend_paged(q, kv, 0, i32[None], i32, 4, q.clone(), i32)
    with pytest.raises(ValueError):
        sd.specdec_process_logits(torch.zeros((1, 1, 5)), torch.zeros((1, 1, 5)))


def test_attend_workspace_serves_smaller_calls(sd):
    """The bytes never fall as a batch, a window or a length grows: one workspace lasts a whole run, though a smaller
    batch may be cut into more pieces than a larger one."""
    f = sd.attend_workspace_bytes
    lens = [65, 300, 640, 641, 1030, 1536, 1537, 8192, 1 << 24]
    for Hq, H, D in [(32, 32, 128), (32, 8, 128), (28, 4, 128), (4, 1, 128), (4, 2, 16), (12, 12, 80), (8, 2, 256), (96, 1, 200)]:
        for T in (1, 5, 12, 13, 65):
            for most in lens:
                sizes = [f(B, T, Hq, H, D, most) for B in (1, 2, 3, 8, 16, 17, 32, 33, 64, 128, 129, 512, 1024, 1025, 4097)]
                assert sizes == sorted(sizes) and sizes[0] > 0, (Hq, H, D, T, most)
        for B in (1, 8, 33, 64, 1025):
            for most in lens:
                sizes = [f(B, T, Hq, H, D, most) for T in range(1, 66)]
                assert sizes == sorted(sizes), (Hq, H, D, B, most)
            for T in (1, 6, 65):
                sizes = [f(B, T, Hq, H, D, most) for most in lens]
                assert sizes == sorted(sizes), (Hq, H, D, B, T)
