"""Attention of bf16 rows over the 4-bit cache against a bound that one wrong key does not hide below.

Bound, derived: the probability p_j of a key is rounded to bf16 in front of the product with the values, by d_j p_j with |d_j| <= u = 2^-8.  With scores that
spread over several powers of two the d_j are as good as independent and of mean zero; then (Hoeffding's inequality for sums of terms within
[-u p_j |v_j|, u p_j |v_j|]) the sum of d_j p_j v_j is beyond 7 u sqrt(sum p_j^2 v_j^2) with a probability of 2 exp(-49 / 2) = 5e-11, of a few million elements
here.  The result's own rounding adds u |o|, fp32 arithmetic what tests/test_gpu_cache_attention.py derives.  That bound grows with the root of the number of keys where the
worst case grows with the number; every case also shows that the value of one key of at least average probability in some row, with the other sign, would be found (planted in the
oracle).
"""
import math

import numpy as np
import pytest
import torch

from paper_2601_15498_amd import cache as C
from tests.test_gpu_cache_attention import U, bounds
from tests.test_gpu_cache_attention_deal import Bytes

pytestmark = pytest.mark.gpu

CASES = [  # D, P, heads, group, lens, N
    (128, 64, 2, 4, (900, 100, 333), 1),     # 4 rows
    (128, 16, 1, 5, (700, 65), 3),           # 15
    (64, 8, 1, 4, (800, 17), 4),             # 16
    (256, 64, 1, 4, (600, 90), 4),
    (128, 64, 1, 4, (900, 100), 7),          # 28 rows, 32 at a time
    (64, 16, 1, 7, (500, 40), 4),
    (256, 32, 1, 8, (700, 31), 3),
    (128, 64, 1, 4, (800, 90), 20),          # 80 rows, four waves
    (64, 32, 1, 2, (700, 3), 50),
    (256, 64, 1, 4, (500, 128), 40),
    (128, 16, 1, 8, (600, 70), 36),          # 288 rows, three blocks
    (128, 64, 2, 4, (900, 200), 60),         # 240 rows, eight waves
    (64, 64, 1, 4, (900, 130), 60),
    (128, 16, 1, 4, (800, 5), 55),
    (128, 64, 1, 4, (300, 0), 400),          # a prompt
]


@pytest.mark.parametrize("D,P,heads,group,lens,N", CASES)
def test_one_wrong_key_would_show(D, P, heads, group, lens, N):
    print("spread", D, P, heads, group, lens, N, flush=True)
    rng = np.random.default_rng(D + P + N + group)
    f = Bytes(D * 3 + N, lens, N, heads, D, P)
    q = torch.from_numpy(rng.standard_normal((len(lens), N, heads * group, D)).astype(np.float32)).bfloat16().cuda()
    out, _ = C.mars_kv_attention(f.pool, f.table, f.lens, q)
    scale, share = 1.0 / math.sqrt(D), 0.0
    for b, length in enumerate(lens):
        T = length + N
        sees = torch.arange(T, device="cuda")[None] <= length + torch.arange(N, device="cuda")[:, None]
        for h in range(heads):
            k, v = f.rows(b, T, h)
            planted, j, found = None, None, False
            for i in range(h * group, (h + 1) * group):
                x = q[b, :, i].double()
                z = torch.where(sees, scale * (x @ k.T), -math.inf)
                p = torch.softmax(z, 1)
                if planted is None:
                    j = int(rng.choice(torch.nonzero(p[0] >= 1 / (length + 1)).flatten().cpu().numpy()))   # (node 0 sees the committed tokens and itself, as all do)
                    planted = v.clone()
                    planted[j] = -v[j]
                worst = torch.where(sees, scale * (x.abs() @ k.abs().T), 0.0).amax(1)
                want = p @ v
                arithmetic, _ = bounds("f32", D, T, want.cpu().numpy(), torch.logsumexp(z, 1).cpu().numpy(), (p @ v.abs()).cpu().numpy(), worst.cpu().numpy())
                bound = torch.from_numpy(arithmetic).cuda() + 1.01 * U * (want.abs() + 7 * ((p * p) @ (v * v)).sqrt())
                got = out[b, :, i].double()
                off = (got - want).abs()
                assert (off <= bound).all(), (b, i, float((off / bound).max()))
                share = max(share, float((off / bound).max()))
                found |= bool(((got - p @ planted).abs() > bound).any())
            assert found, (b, h, j)
    print("largest share of the bound:", share, flush=True)
