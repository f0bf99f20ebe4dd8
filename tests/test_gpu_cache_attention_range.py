"""Attention over the 4-bit cache where scores reach the ends of fp32's range."""
import math

import numpy as np
import pytest
import torch

from paper_2601_15498_amd import cache as C
from tests.cache_util import DTYPES, Filled

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,group", [(1, 4), (7, 4), (40, 4)])
def test_scores_near_the_least_number(dtype, N, group):
    """All of a row's scores lie between -3.4e38 and -3e38: they are numbers like others, and the row is no row that sees nothing."""
    print("least", dtype, N, group, flush=True)
    D, P, n = 64, 16, 300
    rng = np.random.default_rng(N)
    f = Filled(rng, (n,), N, 1, D, P, rows=False)
    k, v = np.zeros((n + N, 1, D)), rng.choice([-2.0, -1.0, 0.5, 1.0, 3.0], (n + N, 1, D))   # (codes of one scale: the cache holds them as they are)
    v[..., ::32] = 6.0
    k[:, 0, 0] = -2.0
    f.k, f.v = [k], [v]
    f.write(0, range(n + N))
    d = f.to()
    q = torch.zeros((1, N, group, D), dtype=DTYPES[dtype], device="cuda")
    q[..., 0] = 1.25 * 2.0 ** 126                    # (a bf16 number) scores of -2.5 * 2^126 = -2.13e38 each,
    scale = 1.5 * math.log(2.0)                      # times 1.5: -3.19e38 powers of two
    mask = torch.zeros((1, N, (N + 63) // 64), dtype=torch.int64, device="cuda")
    out, lse = torch.empty_like(q), torch.empty((1, N, group), device="cuda")
    C.mars_kv_attention(d["pool"], d["table"], d["lens"], q, seqs=d["seqs"], mask=mask, scale=scale, out=out, lse=lse)
    # all weights are equal: the mean of the committed values, whose sums of halves are exact; the division and (bf16) the rounding are not
    want = torch.from_numpy(v[:n, 0].mean(0)).cuda()
    mass = torch.from_numpy(np.abs(v[:n, 0]).mean(0)).cuda()
    unit = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -23
    assert ((out[0].double() - want).abs() <= 1.01 * unit * want.abs() + 2 * (n + 8) * 2.0 ** -24 * mass).all()
    # log(300) is far below half a unit of the last place of 1e38
    assert ((lse.double() / (scale * -2.5 * 2.0 ** 126) - 1).abs() <= 2.0 ** -21).all()


def large_scores(size, N, group, dtype, D, P, lens):
    rng = np.random.default_rng(N)
    f = Filled(rng, lens, N, 1, D, P, rows=False)
    f.k, f.v = [], []
    for n in lens:
        k, v = np.zeros((n + N, 1, D)), rng.choice([-2.0, -1.0, 0.5, 1.0, 3.0], (n + N, 1, D))
        v[..., ::32] = 6.0
        k[:, 0, 0], k[:, 0, 1] = rng.choice([-6.0, -3.0, 0.5, 2.0, 4.0, 6.0], n + N), 6.0   # (channel 1 keeps the scale at 1)
        f.k.append(k)
        f.v.append(v)
        f.write(len(f.k) - 1, range(n + N))
    d = f.to()
    heads = torch.tensor([1.0, -1.0, 1.375, -0.6875], dtype=torch.float64)
    q = torch.zeros((2, N, group, D), dtype=DTYPES[dtype], device="cuda")
    q[..., 0] = (heads * size).to(DTYPES[dtype]).cuda()
    scale = 0.3
    mask = torch.zeros((2, N, (N + 63) // 64), dtype=torch.int64, device="cuda")
    out, lse = torch.empty_like(q), torch.empty((2, N, group), device="cuda")
    C.mars_kv_attention(d["pool"], d["table"], d["lens"], q, seqs=d["seqs"], mask=mask, scale=scale, out=out, lse=lse)
    for b, n in enumerate(lens):
        for h in range(group):
            s = f.k[b][:n, 0, 0] * float(heads[h]) * size
            top = s == s.max()
            want = torch.from_numpy(f.v[b][:n, 0][top].mean(0)).cuda()
            mass = torch.from_numpy(np.abs(f.v[b][:n, 0][top]).mean(0)).cuda()
            unit = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -23   # the result's rounding; equal weights are equal in bf16 too
            bound = 1.01 * unit * want.abs() + 2 * (n + 8) * 2.0 ** -24 * mass   # and two sums of n terms in fp32
            assert ((out[b, :, h].double() - want).abs() <= bound).all(), (b, h)
            want_lse = float(np.float32(scale)) * s.max() + math.log(top.sum())
            assert ((lse[b, :, h].double() - want_lse).abs() <= 2.0 ** -20 * abs(want_lse)).all(), (b, h)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,group", [(1, 4), (7, 4), (26, 4), (60, 4)])
@pytest.mark.parametrize("size", [2.0 ** 12, 2.0 ** 25, 2.0 ** 33, 2.0 ** 64, 2.0 ** 120])
def test_large_scores(size, N, group, dtype):
    """Scores are exact (one channel), the largest of a row are equal: their values' mean is the result, however large they are."""
    print("large", size, N, group, dtype, flush=True)
    large_scores(size, N, group, dtype, 64, 16, (700, 40))


@pytest.mark.parametrize("dtype,D,P,N", [("bf16", 128, 64, 1), ("bf16", 256, 32, 2), ("bf16", 128, 16, 7), ("bf16", 64, 64, 40), ("bf16", 128, 64, 60), ("f32", 128, 8, 3),
                                         ("f32", 64, 64, 30)])
def test_large_scores_of_pieces_that_are_joined(dtype, D, P, N):
    print("large, joined", dtype, D, P, N, flush=True)
    for size in (2.0 ** 12, 2.0 ** 40):
        large_scores(size, N, 4, dtype, D, P, (2600, 1500))
