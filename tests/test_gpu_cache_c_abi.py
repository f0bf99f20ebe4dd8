"""Calls of include/mars_cache.h that the Python binding does not make."""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2601_15498_amd import cache as C
from tests.cache_util import Filled, rounded

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,P,dtype", [(1, 64, "bf16"), (9, 16, "bf16"), (40, 64, "bf16"), (3, 16, "f32")])
def test_requests_beyond_the_sequences_have_rows_of_zeros(N, P, dtype):
    """No sequence numbers are given: request b is sequence b, and those from `sequences` on are outside the cache."""
    print("beyond", N, P, dtype, flush=True)
    rng = np.random.default_rng(N)
    D, heads, group, B = 128, 2, 4, 70
    f = Filled(rng, (40, 9), N, heads, D, P)
    d = f.to()
    q, _ = rounded(rng.standard_normal((B, N, heads * group, D)), dtype)
    q = q.cuda()
    out, lse = torch.full_like(q, 5.0), torch.full((B, N, heads * group), 5.0, device="cuda")
    want, want_lse = torch.empty_like(q), torch.empty_like(lse)
    seqs = torch.tensor([0, 1] + [-1] * (B - 2), dtype=torch.int32, device="cuda")
    C.mars_kv_attention(d["pool"], d["table"], d["lens"], q, seqs=seqs, out=want, lse=want_lse)
    work = C.alloc_attention_workspace(d["pool"], d["table"], q)
    c = C.CacheStruct(d["pool"].data_ptr(), d["table"].data_ptr(), d["lens"].data_ptr(), None, None, 1, f.pool.shape[1], heads, D, P, 2, f.width)
    rows = lambda t: C.RowsStruct(t.data_ptr(), t.stride(0), t.stride(1), t.stride(2))  # noqa: E731
    qr, outr = rows(q), rows(out)
    torch.cuda.synchronize()
    rc = C.lib().mars_kv_attention(ctypes.byref(c), 0, None, ctypes.byref(qr), 1 if dtype == "bf16" else 0, heads * group, None, None, 1 / math.sqrt(D), 0,
                                   ctypes.byref(outr), lse.data_ptr(), B, N, work.data_ptr(), work.numel(), C._stream())
    assert rc == 0
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, want_lse) and torch.isfinite(lse[:2]).all()
    assert (out[2:] == 0).all() and (lse[2:] == -math.inf).all()
