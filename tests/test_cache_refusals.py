"""What the shared-prefix, cross-attention, weighing and eviction calls refuse, before any HIP call
(CPU only: every call here fails its checks, so nothing is launched)."""
import pytest
import torch

from paper_2405_19261_amd import spc
from test_ops_refusals import BAD_CACHES, INF, NAN, OK, cache


def shared(c, **kw):
    a = dict(shared=20, st=OK, q=OK, dtype=spc.SPC_BF16, qs=1024, heads=8, rows=6, start=None, most=0,
             scale=0.1, window=0, out=OK, os=1024, ws=None, n=0)
    a.update(kw)
    return spc.lib().spc_kv_attend_shared(c, a["shared"], a["st"], a["q"], a["dtype"], a["qs"],
                                          a["heads"], a["rows"], a["start"], a["most"], a["scale"],
                                          a["window"], a["out"], a["os"], a["ws"], a["n"], None)


def cross(c, **kw):
    a = dict(q=OK, dtype=spc.SPC_BF16, qs=1024, heads=8, rows=6, start=None, most=0, scale=0.1, mask=OK,
             ms=64, mw=64, out=OK, os=1024, ws=None, n=0)
    a.update(kw)
    return spc.lib().spc_cross_attend(c, a["q"], a["dtype"], a["qs"], a["heads"], a["rows"], a["start"],
                                      a["most"], a["scale"], a["mask"], a["ms"], a["mw"], a["out"],
                                      a["os"], a["ws"], a["n"], None)


def weigh(c, **kw):
    a = dict(q=OK, dtype=spc.SPC_BF16, qs=1024, heads=8, rows=6, start=None, most=0, scale=0.1, window=0,
             w=OK, out=OK, ld=64, length=64, ws=None, n=0)
    a.update(kw)
    return spc.lib().spc_kv_weigh(c, a["q"], a["dtype"], a["qs"], a["heads"], a["rows"], a["start"],
                                  a["most"], a["scale"], a["window"], a["w"], a["out"], a["ld"],
                                  a["length"], a["ws"], a["n"], None)


def evict(c, **kw):
    a = dict(w=OK, ld=64, length=64, keep=32, first=4, recent=8, table=OK, width=2, n=OK + 4096, index=OK,
             out_w=OK + 8192, out_ld=32)
    a.update(kw)
    return spc.lib().spc_kv_evict(c, a["w"], a["ld"], a["length"], a["keep"], a["first"], a["recent"],
                                  a["table"], a["width"], a["n"], a["index"], a["out_w"], a["out_ld"],
                                  None)


@pytest.mark.parametrize("kw,status", BAD_CACHES)
def test_cache_refusals(kw, status):
    for call in (shared, cross, weigh, evict):
        assert call(cache(**kw)) == status
        assert spc.spc_last_error() != ""


BAD_QUERIES = [(dict(q=None), -1), (dict(out=None), -1), (dict(dtype=spc.SPC_F32), -4), (dict(heads=7), -2),
               (dict(heads=0), -2), (dict(qs=1023), -2), (dict(rows=0), -2), (dict(rows=7), -2),
               (dict(rows=(1 << 24) + 1, start=OK, most=1), -2), (dict(start=OK, most=0), -2),
               (dict(scale=NAN), -4), (dict(scale=INF), -4), (dict(q=OK + 1), -5),
               (dict(ws=OK, n=16), -6), (dict(ws=OK + 8, n=1 << 30), -6)]


@pytest.mark.parametrize("kw,status", BAD_QUERIES)
def test_query_refusals(kw, status):
    # (tables that give the workspace a use)
    wide = dict(table_width=64, B=3)
    for call in (shared, cross, weigh):
        assert call(cache(**wide), **kw) == status
        assert spc.spc_last_error() != ""


@pytest.mark.parametrize("call,kw,status", [
    (shared, dict(st=None), -1), (shared, dict(st=OK + 2), -5), (shared, dict(shared=-1), -2),
    (shared, dict(shared=(1 << 30) + 1), -2), (shared, dict(window=-1), -4), (shared, dict(os=1023), -2),
    (shared, dict(out=OK + 4), -5), (shared, dict(os=1026), -5),
    (shared, dict(rows=1 << 24, start=OK, most=1, heads=4096, qs=1 << 20, os=1 << 20), -2),
    # (two parts that one launch could not hold, each of which alone it could)
    (shared, dict(rows=2620000, start=OK, most=2620000, heads=128, qs=1 << 14, os=1 << 14), -2),
    (cross, dict(mw=0), -2), (cross, dict(ms=-1), -2), (cross, dict(os=1023), -2),
    (cross, dict(out=OK + 4), -5),
    (weigh, dict(window=-1), -4), (weigh, dict(length=0), -2), (weigh, dict(length=(1 << 26) + 1, ld=1 << 27), -2),
    (weigh, dict(ld=63), -2), (weigh, dict(out=OK + 2), -5), (weigh, dict(w=OK + 1), -5),
    (evict, dict(w=None), -1), (evict, dict(table=None), -1), (evict, dict(n=None), -1),
    (evict, dict(index=None), -1), (evict, dict(length=0), -2), (evict, dict(ld=63), -2),
    (evict, dict(keep=0), -2), (evict, dict(keep=(1 << 26) + 1, width=1 << 25), -2),
    (evict, dict(keep=33), -2), (evict, dict(width=0), -2), (evict, dict(out_ld=31), -2),
    (evict, dict(first=-1), -4), (evict, dict(recent=-1), -4), (evict, dict(first=25), -4),
    (evict, dict(first=2 ** 31 - 1, recent=2 ** 31 - 1), -4), (evict, dict(w=OK + 2), -5),
    (evict, dict(table=OK + 1), -5), (evict, dict(index=OK + 2), -5), (evict, dict(n=OK + 1), -5),
    (evict, dict(out_w=OK + 3), -5), (evict, dict(n=OK), -4), (evict, dict(out_w=OK), -4),
])
def test_refusals(call, kw, status):
    assert call(cache(), **kw) == status
    assert spc.spc_last_error() != ""


def test_workspace_queries():
    """Sizes that no call takes give 0; others what a call of them asks for."""
    L = spc.lib()
    for f in (lambda c, h, r, m: L.spc_kv_shared_workspace_bytes(c, 100, h, r, m),
              L.spc_kv_weigh_workspace_bytes, L.spc_cross_workspace_bytes):
        assert f(cache(table_width=64), 8, 6, 0) > 0
        for bad in (dict(B=0), dict(page_size=8), dict(head_dim=96), dict(dtype=0), dict(kv_heads=0)):
            assert f(cache(**bad), 8, 6, 0) == 0
        for h, r, m in ((7, 6, 0), (0, 6, 0), (8, 0, 0), (8, 7, 0), (8, 6, -1), (8, (1 << 24) + 1, 2)):
            assert f(cache(), h, r, m) == 0
        assert f(None, 8, 6, 0) == 0
    for s in (-1, (1 << 30) + 1):
        assert L.spc_kv_shared_workspace_bytes(cache(), s, 8, 6, 0) == 0
    assert L.spc_kv_shared_workspace_bytes(cache(), 0, 8, 6, 0) == L.spc_kv_workspace_bytes(cache(), 8, 6, 0)
    # a workspace of that size passes its check (the call then stops at nothing else: it is not made)
    c = cache(table_width=64)
    need = L.spc_kv_weigh_workspace_bytes(c, 8, 6, 0)
    assert weigh(c, ws=OK, n=need - 1) == -6
    need = L.spc_kv_shared_workspace_bytes(c, 20, 8, 6, 0)
    assert shared(c, ws=OK, n=need - 1) == -6
    need = L.spc_cross_workspace_bytes(c, 8, 6, 0)
    assert cross(c, ws=OK, n=need - 1) == -6


def tensors(B=2, H=2, S=16, D=64, width=4, pages=12):
    k = torch.zeros((pages, H, S, D), dtype=torch.bfloat16)
    v = torch.zeros((pages, H, D, S), dtype=torch.bfloat16)
    return k, v, torch.zeros((B, width), dtype=torch.int32), torch.zeros(B, dtype=torch.int32)


def test_binding_refusals():
    a = tensors()
    q = torch.zeros((2, 1, 4, 64), dtype=torch.bfloat16)
    w = torch.zeros((2, 2, 64))
    t = torch.zeros((2, 2), dtype=torch.int32)
    for bad in (lambda: spc.spc_kv_attend_shared(q, *a, 65),                     # the table holds 64
                lambda: spc.spc_kv_attend_shared(q, *a, 17, shared_table=a[2][0, :1]),
                lambda: spc.spc_kv_attend_shared(q, *a, 2 ** 31),
                lambda: spc.spc_kv_attend_shared(q, *a, 20, shared_table=a[2]),
                lambda: spc.spc_kv_attend_shared(q, *a, 20, out=q[:1]),
                lambda: spc.spc_cross_attend(q, *a, key_mask=torch.ones((1, 9), dtype=torch.bool)),
                lambda: spc.spc_cross_attend(q, *a, key_mask=torch.ones((9, 2), dtype=torch.bool).t()),
                lambda: spc.spc_cross_attend(q[:, :, :, :32], *a),
                lambda: spc.spc_kv_weigh(q, *a, w[:1]),
                lambda: spc.spc_kv_weigh(q, *a, w, out=torch.zeros((2, 2, 63))),
                lambda: spc.spc_kv_weigh(q, *a, w, out=torch.zeros((2, 2, 70))[..., :64]),
                lambda: spc.spc_kv_weigh(q, *a, w.transpose(0, 1)),
                lambda: spc.spc_kv_weigh(q[:, :0], *a, w),
                lambda: spc.spc_kv_evict(*a, w, 0, t), lambda: spc.spc_kv_evict(*a, w, 8, t[0]),
                lambda: spc.spc_kv_evict(*a, w, 8, t[:1]),
                lambda: spc.spc_kv_evict(*a, w, 8, t, out_index=torch.zeros((2, 2, 9), dtype=torch.int32)),
                lambda: spc.spc_kv_evict(*a, w, 8, t, out_weights=torch.zeros((2, 2, 9))),
                # on the CPU
                lambda: spc.spc_kv_attend_shared(q, *a, 20), lambda: spc.spc_cross_attend(q, *a),
                lambda: spc.spc_kv_weigh(q, *a, w), lambda: spc.spc_kv_evict(*a, w, 8, t)):
        with pytest.raises((ValueError, RuntimeError, AssertionError)):
            bad()
    for bad in (lambda: spc.spc_kv_attend_shared(q.float(), *a, 20),
                lambda: spc.spc_kv_attend_shared(q, *a, 20, shared_table=a[2][0].long()),
                lambda: spc.spc_cross_attend(q, *a, key_mask=torch.ones((2, 9))),
                lambda: spc.spc_kv_weigh(q, *a, w.double()),
                lambda: spc.spc_kv_evict(*a, w.half(), 8, t),
                lambda: spc.spc_kv_evict(*a, w, 8, t.long())):
        with pytest.raises(TypeError):
            bad()
