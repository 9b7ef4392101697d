"""What the truncation and cache calls refuse, before any HIP call (CPU only:
every call here fails its checks, so nothing is launched)."""
import ctypes

import pytest
import torch

from paper_2405_19261_amd import spc

OK = 0x10000   # an aligned address, never dereferenced
NAN, INF = float("nan"), float("inf")


def cut(**kw):
    a = dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, temp_per_seq=None, top_k_per_seq=None,
             top_p_per_seq=None, min_p_per_seq=None)
    a.update(kw)
    return spc.Truncation(**a)


def sample(**kw):
    t = kw.pop("cut", cut())
    a = dict(z=OK, dtype=spc.SPC_BF16, B=4, V=1000, ld=1000, u=OK, tok=OK, lp=None, kept=None,
             ws=None, n=0)
    a.update(kw)
    return spc.lib().spc_sample(a["z"], a["dtype"], a["B"], a["V"], a["ld"],
                                None if t is None else ctypes.byref(t), a["u"], a["tok"], a["lp"],
                                a["kept"], a["ws"], a["n"], None)


def truncate(**kw):
    t = kw.pop("cut", cut())
    a = dict(z=OK, dtype=spc.SPC_F32, B=4, rows=3, V=1000, out=OK, ws=None, n=0)
    a.update(kw)
    return spc.lib().spc_truncate(a["z"], a["dtype"], a["B"], a["rows"], a["V"],
                                  None if t is None else ctypes.byref(t), a["out"], a["ws"], a["n"],
                                  None)


BAD_CUTS = [dict(temperature=-1.0), dict(temperature=NAN), dict(temperature=INF), dict(top_k=-1),
            dict(top_p=0.0), dict(top_p=1.0001), dict(top_p=NAN), dict(min_p=-0.1), dict(min_p=1.1),
            dict(min_p=NAN)]


@pytest.mark.parametrize("kw,status", [
    (dict(z=None), -1), (dict(tok=None), -1), (dict(u=None), -1), (dict(cut=None), -1),
    (dict(u=None, cut=cut(temperature=0.0, temp_per_seq=OK)), -1),
    (dict(B=0), -2), (dict(V=1), -2), (dict(ld=999), -2), (dict(dtype=2), -4), (dict(z=OK + 1), -5),
    (dict(dtype=spc.SPC_F32, z=OK + 2), -5),
] + [(dict(cut=cut(**c)), -4) for c in BAD_CUTS])
def test_sample_refusals(kw, status):
    assert sample(**kw) == status
    assert spc.spc_last_error() != ""


@pytest.mark.parametrize("kw,status", [
    (dict(z=None), -1), (dict(out=None), -1), (dict(cut=None), -1), (dict(B=0), -2),
    (dict(rows=0), -2), (dict(V=1), -2), (dict(dtype=-1), -4), (dict(out=OK + 2), -5),
    (dict(out=OK + 4), -4), (dict(out=OK - 47996), -4),  # overlapping, not the same
] + [(dict(cut=cut(**c)), -4) for c in BAD_CUTS])
def test_truncate_refusals(kw, status):
    assert truncate(**kw) == status
    assert spc.spc_last_error() != ""


def test_arrays_stand_in_for_bad_scalars():
    """A scalar that its array replaces is not looked at (the call stops at the alignment)."""
    for name, bad in (("temp", dict(temperature=NAN)), ("top_k", dict(top_k=-3)),
                      ("top_p", dict(top_p=7.0)), ("min_p", dict(min_p=NAN))):
        assert sample(z=OK + 1, cut=cut(**{name + "_per_seq": OK}, **bad)) == -5
    assert sample(z=OK + 1, u=None, cut=cut(temperature=0.0)) == -5


def cache(**kw):
    a = dict(k_pages=OK, v_pages=OK, k_scale=None, v_scale=None, dtype=spc.SPC_BF16, num_pages=8,
             page_size=16, kv_heads=2, head_dim=128, page_table=OK, table_width=4, kv_len=OK, B=3)
    a.update(kw)
    return spc.KvCache(**a)


BAD_CACHES = [
    (dict(k_pages=None), -1), (dict(v_pages=None), -1), (dict(page_table=None), -1),
    (dict(kv_len=None), -1), (dict(dtype=spc.SPC_E4M3), -1),
    (dict(dtype=spc.SPC_E4M3, k_scale=OK), -1), (dict(dtype=0), -4), (dict(dtype=3), -4),
    (dict(B=0), -2), (dict(B=65536), -2), (dict(num_pages=0), -2), (dict(table_width=0), -2),
    (dict(table_width=(1 << 26) + 1), -2), (dict(kv_heads=0), -2), (dict(page_size=8), -2), (dict(page_size=24), -2),
    (dict(page_size=2048), -2), (dict(page_size=0), -2), (dict(head_dim=96), -2),
    (dict(head_dim=0), -2), (dict(k_pages=OK + 8), -5), (dict(v_pages=OK + 2), -5),
    (dict(page_table=OK + 2), -5), (dict(kv_len=OK + 1), -5),
    (dict(dtype=spc.SPC_E4M3, k_scale=OK, v_scale=OK + 4), -5)]


def write(c, **kw):
    a = dict(k=OK, v=OK, dtype=spc.SPC_F32, ks=256, vs=256, rows=6, start=None)
    a.update(kw)
    return spc.lib().spc_kv_write(c, a["k"], a["v"], a["dtype"], a["ks"], a["vs"], a["rows"],
                                  a["start"], None)


def read(c, **kw):
    a = dict(k=OK, v=OK, dtype=spc.SPC_F32, n=6)
    a.update(kw)
    return spc.lib().spc_kv_read(c, a["k"], a["v"], a["dtype"], a["n"], None)


def attend(c, **kw):
    a = dict(q=OK, dtype=spc.SPC_BF16, qs=1024, heads=8, rows=6, start=None, most=0, scale=0.1,
             window=0, out=OK, os=1024, ws=None, n=0)
    a.update(kw)
    return spc.lib().spc_kv_attend(c, a["q"], a["dtype"], a["qs"], a["heads"], a["rows"], a["start"],
                                   a["most"], a["scale"], a["window"], a["out"], a["os"], a["ws"],
                                   a["n"], None)


@pytest.mark.parametrize("kw,status", BAD_CACHES)
def test_cache_refusals(kw, status):
    for call in (write, read, attend):
        assert call(cache(**kw)) == status
        assert spc.spc_last_error() != ""


@pytest.mark.parametrize("call,kw,status", [
    (write, dict(k=None), -1), (write, dict(v=None), -1), (write, dict(dtype=2), -4),
    (write, dict(ks=255), -2), (write, dict(vs=0), -2), (write, dict(rows=0), -2),
    (write, dict(rows=7), -2), (write, dict(rows=(1 << 24) + 1, start=OK), -2),
    (write, dict(k=OK + 2), -5), (write, dict(dtype=spc.SPC_BF16, v=OK + 1), -5),
    (read, dict(k=None), -1), (read, dict(v=None), -1), (read, dict(dtype=2), -4),
    (read, dict(n=0), -2), (read, dict(n=(1 << 26) + 1), -2), (read, dict(v=OK + 4), -5),
    (attend, dict(q=None), -1), (attend, dict(out=None), -1), (attend, dict(dtype=spc.SPC_F32), -4),
    (attend, dict(heads=7), -2), (attend, dict(heads=0), -2), (attend, dict(qs=1023), -2),
    (attend, dict(os=1000), -2), (attend, dict(rows=5), -2), (attend, dict(start=OK, most=0), -2),
    (attend, dict(scale=NAN), -4), (attend, dict(scale=INF), -4), (attend, dict(window=-1), -4),
    (attend, dict(rows=1 << 24, start=OK, most=1 << 24, heads=64, qs=8192, os=8192), -2),
    (attend, dict(q=OK + 1), -5), (attend, dict(out=OK + 4), -5), (attend, dict(os=1026), -5),
])
def test_cache_call_refusals(call, kw, status):
    assert call(cache(), **kw) == status
    assert spc.spc_last_error() != ""


# ------------------------------------------------------------------ the binding
def pages(dt=torch.bfloat16, n=4, H=2, S=16, D=64):
    return torch.zeros((n, H, S, D), dtype=dt), torch.zeros((n, H, D, S), dtype=dt)


def test_binding_refuses_shapes_types_and_layouts():
    """The binding raises before the library is called (host tensors: a call
    that got through would fail on its device, which no case here reaches)."""
    z, u = torch.zeros(3, 50), torch.zeros(3)
    for bad in (torch.zeros(50), torch.zeros(2, 3, 50), torch.zeros(50, 3).t(),
                torch.zeros(1, 50).expand(3, 50)):
        with pytest.raises(ValueError):
            spc.spc_sample(bad, u)
    with pytest.raises(TypeError):
        spc.spc_sample(z.half(), u)
    with pytest.raises(TypeError):
        spc.spc_sample(z, u.double())
    with pytest.raises(ValueError):
        spc.spc_sample(z, torch.zeros(4))
    with pytest.raises(TypeError):
        spc.spc_sample(z, u, top_k_per_seq=torch.zeros(3, dtype=torch.int64))
    with pytest.raises(ValueError):
        spc.spc_sample(z, u, out_kept=torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        spc.spc_truncate(torch.zeros(3, 2, 50)[:, :1])
    with pytest.raises(TypeError):
        spc.spc_truncate(z, out=torch.zeros(3, 50, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        spc.spc_truncate(z, out=torch.zeros(3, 49))

    k, v = pages()
    table, n = torch.zeros((3, 2), dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    new = torch.zeros((3, 2, 2, 64))
    q = torch.zeros((3, 2, 4, 64), dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        spc.spc_kv_write(new, new, k.float(), v.float(), table, n)
    with pytest.raises(ValueError):
        spc.spc_kv_write(new, new, k, k, table, n)          # values not transposed
    with pytest.raises(ValueError):
        spc.spc_kv_write(new, new, *pages(torch.float8_e4m3fn), table, n)  # no scales
    with pytest.raises(ValueError):
        spc.spc_kv_write(new, new, k, v, table, n, k_scale=torch.zeros(4, 2, 16),
                         v_scale=torch.zeros(4, 2, 16))
    with pytest.raises(TypeError):
        spc.spc_kv_write(new, new, k, v, table.long(), n)
    with pytest.raises(ValueError):
        spc.spc_kv_write(new, new, k, v, table, torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        spc.spc_kv_write(new, new[:, :1], k, v, table, n)
    with pytest.raises(ValueError):
        spc.spc_kv_write(new.transpose(1, 2), new, k, v, table, n)
    with pytest.raises(ValueError):
        spc.spc_kv_write(new[:2], new[:2], k, v, table, n)
    with pytest.raises(ValueError):
        spc.spc_kv_write(new, new, k, v, table, n, q_start=torch.zeros(4, dtype=torch.int32))
    with pytest.raises(TypeError):
        spc.spc_kv_attend(q.float(), k, v, table, n)
    with pytest.raises(ValueError):
        spc.spc_kv_attend(q[..., :32], k, v, table, n)
    with pytest.raises(ValueError):
        spc.spc_kv_attend(q, k, v, table, n, out=q[:, :1])
    with pytest.raises(ValueError):
        spc.spc_kv_attend(torch.zeros((3, 5, 4, 64), dtype=torch.bfloat16)[:, :2], k, v, table, n)
    with pytest.raises(ValueError):
        spc.spc_kv_read(k, v, table, n)                     # neither length nor out
    with pytest.raises(ValueError):
        spc.spc_kv_read(k, v, table, n, 5, out=(new, new))


def test_binding_refuses_host_tensors():
    """Nothing of the host's reaches a kernel."""
    z, u = torch.zeros(3, 50), torch.zeros(3)
    k, v = pages()
    table, n = torch.zeros((3, 2), dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    new = torch.zeros((3, 2, 2, 64))
    for call in (lambda: spc.spc_sample(z, u), lambda: spc.spc_truncate(z, top_k=3),
                 lambda: spc.spc_kv_write(new, new, k, v, table, n),
                 lambda: spc.spc_kv_read(k, v, table, n, 5),
                 lambda: spc.spc_kv_attend(new.bfloat16(), k, v, table, n)):
        with pytest.raises(ValueError, match="current HIP device"):
            call()


def test_binding_takes_empty_chunks():
    """No rows: nothing to do, and nothing launched."""
    k, v = pages()
    table, n = torch.zeros((3, 2), dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    none = torch.zeros((3, 0, 2, 64))
    spc.spc_kv_write(none, none, k, v, table, n)
    q = torch.zeros((3, 0, 4, 64), dtype=torch.bfloat16)
    assert spc.spc_kv_attend(q, k, v, table, n).shape == q.shape
    ko, vo = spc.spc_kv_read(k, v, table, n, 0)
    assert ko.shape == (3, 0, 2, 64) == vo.shape
