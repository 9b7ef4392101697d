"""Pages whose places pass 32 bits: a cache of more than 2^32 bytes of keys, its last pages used
by every operator of the cache's attention, weights and eviction, against the same tokens in a
small cache."""
import pytest
import torch

import ops_oracle
from cache_oracle import i32, randn
from paper_2405_19261_amd import spc

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


@pytest.mark.parametrize("f8", [False, True])
def test_pages_past_32_bits(f8):
    H, D, S, B = 2, 128, 64, 2
    dt = torch.float8_e4m3fn if f8 else torch.bfloat16
    n = (1 << 32) // (H * S * D * (1 if f8 else 2)) + 64
    k = torch.empty((n, H, S, D), dtype=dt, device=DEV)
    v = torch.empty((n, H, D, S), dtype=dt, device=DEV)
    ks = [torch.empty((n, H, S), device=DEV) if f8 else None for _ in range(2)]
    far = dict(k_scale=ks[0], v_scale=ks[1])
    small = ops_oracle.Cache(B, 4, H, D, S, f8, DEV, spare=16)
    last = torch.arange(n - 8, n, dtype=torch.int32, device=DEV).view(2, 4)
    lens = i32([250, 200])
    ref = (small.k, small.v, small.table, lens)
    big = (k, v, last, lens)
    for m in (250, 3):  # (the prompt, then a chunk over its end again)
        knew, vnew = randn((B, m, H, D), m).to(DEV), randn((B, m, H, D), m + 1).to(DEV)
        spc.spc_kv_write(knew, vnew, *ref, **small.scales())
        spc.spc_kv_write(knew, vnew, *big, **far)
    for rows in (1, 5, 80):
        q = randn((B, rows, 4, D), rows).to(DEV)
        for call in (spc.spc_kv_attend, spc.spc_cross_attend, spc.spc_kv_weigh):
            assert torch.equal(call(q, *big, **far), call(q, *ref, **small.scales())), (call, rows)
        a = spc.spc_kv_attend_shared(q, *big, 100, shared_table=last[0], **far)
        b = spc.spc_kv_attend_shared(q, *ref, 100, shared_table=small.table[0].contiguous(),
                                     **small.scales())
        assert torch.equal(a, b)
    w = torch.rand((B, H, 256), device=DEV)
    used = set(small.table.flatten().tolist())
    free = i32([p for p in range(small.pages) if p not in used][:4]).view(2, 2)
    out_far = torch.arange(n - 12, n - 8, dtype=torch.int32, device=DEV).view(2, 2)
    a = spc.spc_kv_evict(*big, w, 100, out_far, recent=7, **far)
    b = spc.spc_kv_evict(*ref, w, 100, free, recent=7, **small.scales())
    for x, y in zip(a, b):
        assert torch.equal(x, y)
    q = randn((B, 1, 4, D), 9).to(DEV)
    assert torch.equal(spc.spc_kv_attend(q, k, v, out_far, a[0], **far),
                       spc.spc_kv_attend(q, small.k, small.v, free, b[0], **small.scales()))
