"""Sizes of the cache calls' workspaces (CPU: sizes only, nothing is launched).
Calls run in a child process where they might end it."""
import subprocess
import sys

import pytest
import torch

from paper_2405_19261_amd import spc

OK = 0x10000   # an aligned address, never dereferenced


def cache(**kw):
    a = dict(dtype=spc.SPC_BF16, num_pages=8, page_size=16, kv_heads=2, head_dim=128,
             table_width=4000, B=4)
    a.update(kw)
    return spc.KvCache(**a)


def query(c, heads=4, rows=8, max_rows=0):
    return spc.lib().spc_kv_workspace_bytes(c, heads, rows, max_rows)


def test_fewer_rows_than_sequences_are_no_error_of_the_process():
    code = ("import sys; sys.path.insert(0, 'tests'); import test_kv_workspace as t; "
            "print([t.query(t.cache(), rows=r) for r in (1, 2, 3)])")
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "[0, 0, 0]", (r.returncode, r.stderr)


@pytest.mark.parametrize("bad", [
    dict(B=0), dict(B=65536), dict(num_pages=0), dict(kv_heads=0), dict(kv_heads=65536),
    dict(page_size=8), dict(page_size=24), dict(page_size=1 << 30), dict(head_dim=0),
    dict(head_dim=96), dict(head_dim=-64), dict(table_width=0), dict(table_width=(1 << 26) + 1),
    dict(dtype=spc.SPC_F32), dict(dtype=7)])
def test_sizes_of_no_cache_need_no_workspace(bad):
    heads = bad.get("kv_heads", 2) or 2
    assert query(cache(**bad), heads=heads, rows=65536 if "B" in bad else 8) == 0


@pytest.mark.parametrize("kw", [dict(rows=0), dict(rows=-1), dict(rows=(1 << 24) + 1, max_rows=1),
                                dict(rows=9), dict(max_rows=-1), dict(heads=0), dict(heads=3),
                                dict(heads=-2)])
def test_sizes_of_no_call_need_no_workspace(kw):
    assert query(cache(), **kw) == 0


@pytest.mark.parametrize("dtype", [spc.SPC_BF16, spc.SPC_E4M3])
@pytest.mark.parametrize("rows,max_rows", [(1, 1), (3, 1), (3, 3), (4, 0), (8, 0), (9, 5), (9, 100),
                                           (400, 0), (401, 100), (1 << 24, 7)])
def test_the_query_and_the_call_agree(rows, max_rows, dtype):
    """A workspace one byte short of the query's is what the call refuses, and it
    says how many it needs."""
    c = cache(k_pages=OK, v_pages=OK, page_table=OK, kv_len=OK, k_scale=OK, v_scale=OK, dtype=dtype)
    n = query(c, rows=rows, max_rows=max_rows)
    assert n > 0  # (a call that needs none would be launched)
    status = spc.lib().spc_kv_attend(c, OK, spc.SPC_BF16, 512, 4, rows, OK if max_rows else None,
                                     max_rows, 0.1, 0, OK, 512, OK, n - 1, None)
    assert status == -6 and f"need {n}," in spc.spc_last_error()


def test_the_binding_asks_for_what_its_call_needs(monkeypatch):
    """With the same q_start and max_q (defaults too) the query gives the size
    that spc_kv_attend lays out."""
    B, H, S, D, width, heads = 4, 2, 16, 64, 1000, 8
    k = torch.zeros((8, H, S, D), dtype=torch.bfloat16)
    v = torch.zeros((8, H, D, S), dtype=torch.bfloat16)
    args = (k, v, torch.zeros((B, width), dtype=torch.int32), torch.zeros(B, dtype=torch.int32))
    short = torch.zeros(4096, dtype=torch.uint8)[:1]  # (no call gets past its check of the workspace)
    start = torch.zeros(B + 1, dtype=torch.int32)
    monkeypatch.setattr(spc, "_on_current_device", lambda t: None)
    monkeypatch.setattr(spc, "_stream", lambda s: None)
    for rows, q_start, max_q in ((8, None, None), (9, start, None), (9, start, 3), (3, start, 3),
                                 (3, start, None), (400, start, None), (400, None, None)):
        lead = (rows,) if q_start is not None else (B, rows // B)
        q = torch.zeros(lead + (heads, D), dtype=torch.bfloat16)
        n = spc.spc_kv_workspace_bytes(*args, heads, rows, max_q, q_start=q_start)
        assert n > 0
        with pytest.raises(spc.SpcError, match=f"need {n},"):
            spc.spc_kv_attend(q, *args, q_start=q_start, max_q=max_q, workspace=short)
    # a size alone is that of even rows, or with max_q of a call with q_start
    assert spc.spc_kv_workspace_bytes(*args, heads, 3) == 0
    assert (spc.spc_kv_workspace_bytes(*args, heads, 9, 3) ==
            spc.spc_kv_workspace_bytes(*args, heads, 9, 3, q_start=start) > 0)
