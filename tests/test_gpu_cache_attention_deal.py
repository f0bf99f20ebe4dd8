"""Attention over the 4-bit cache where the work is cut between work-groups and joined again: long and uneven lengths, many requests, blocks of rows
of every kind.  Against the definition in 64 bits, computed from the cache's bytes; the bounds are those of the tests beside this file."""
import math

import numpy as np
import pytest
import torch

from oracle import cache_ref as R
from paper_2601_15498_amd import cache as C
from tests.cache_util import DTYPES
from tests.test_gpu_cache_attention import bounds

pytestmark = pytest.mark.gpu


class Bytes:
    """Random bytes in pages dealt out at random; what no token owns decodes to NaN."""

    def __init__(self, seed, lens, room, heads, D, P):
        g = torch.Generator("cuda").manual_seed(seed)
        self.D, self.P = D, P
        held = [-(-(n + room) // P) for n in lens]
        pages = sum(held) + 3
        order = torch.randperm(pages, device="cuda", generator=g).int()
        self.table = torch.full((len(lens), max(held) + 2), -1, dtype=torch.int32, device="cuda")
        self.pool = torch.randint(0, 256, (1, pages, heads, P * (D + D // 16)), dtype=torch.uint8, device="cuda", generator=g)
        self.pool[..., P * D:] = torch.randint(123, 128, self.pool[..., P * D:].shape, dtype=torch.uint8, device="cuda", generator=g)
        at = 0
        free = torch.ones(pages, dtype=torch.bool, device="cuda")
        for b, (n, h) in enumerate(zip(lens, held)):
            own = order[at: at + h]
            self.table[b, :h] = own
            free[own.long()] = False
            at += h
            for t in range(n + room, h * P):
                page, i = int(own[t // P]), t % P
                self.pool[0, page, :, P * D + i * (D // 32): P * D + (i + 1) * (D // 32)] = 255
                v = P * D + P * D // 32 + i // 8 * (D // 4) + i % 8
                self.pool[0, page, :, v: v + D // 4: 8] = 255
        self.pool[0, free] = 255
        self.lens = torch.tensor(lens, dtype=torch.int32, device="cuda")

    def rows(self, b, n, head):
        """Keys and values [n, D] of sequence b."""
        D, P = self.D, self.P
        t, c = torch.arange(n, device="cuda"), torch.arange(D, device="cuda")
        part = self.pool[0, self.table[b, t // P].long(), head]
        t = t % P
        grid = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64, device="cuda")

        def values(code_at, scale_at):
            byte = part.gather(1, code_at).int()
            return grid[torch.where(c % 2 == 1, byte >> 4, byte & 15).long()] * torch.exp2(part.gather(1, scale_at).double() - 127)

        k = values(t[:, None] * (D // 2) + c // 2, P * D + t[:, None] * (D // 32) + c // 32)
        v = values(P * D // 2 + (t[:, None] // 8) * 4 * D + (c // 8) * 32 + (t[:, None] % 8) * 4 + c % 8 // 2,
                   P * D + P * D // 32 + (t[:, None] // 8) * (D // 4) + c // 32 * 8 + t[:, None] % 8)
        return k, v


def check(cache, lens, n_new, q, sees_of, out, lse, scale, dtype, group):
    q = q.cuda().double()
    for b, (n, length) in enumerate(zip(n_new, lens)):
        assert (out[b, n:] == 0).all() and (lse[b, n:] == -math.inf).all(), b
        if n == 0:
            continue
        sees = torch.cat([torch.ones((n, length), dtype=torch.bool, device="cuda"), torch.from_numpy(sees_of(b)[:n, :n]).cuda()], 1)
        for h in range(cache.pool.shape[2]):
            k, v = cache.rows(b, length + n, h)
            for i in range(h * group, (h + 1) * group):
                z = scale * (q[b, :n, i] @ k.T)
                z[~sees] = -math.inf
                want_lse = torch.logsumexp(z, 1)
                some = torch.isfinite(want_lse)
                p = torch.where(some[:, None], torch.softmax(z, 1), 0.0)
                worst = torch.where(sees, scale * (q[b, :n, i].abs() @ k.abs().T), 0.0).amax(1)
                want, mass, worst, base = ((p @ v).cpu().numpy(), (p @ v.abs()).cpu().numpy(), worst.cpu().numpy(), want_lse.cpu().numpy())
                bo, bl = bounds(dtype, cache.D, length + n, want, base, mass, worst)
                got, got_lse = out[b, :n, i].double().cpu().numpy(), lse[b, :n, i].double().cpu().numpy()
                fine = np.isfinite(base)
                assert (got[~fine] == 0).all() and (got_lse[~fine] == -np.inf).all(), (b, i)
                off, off_lse = np.abs(got - want), np.abs(got_lse[fine] - base[fine])
                assert (off <= bo).all(), (b, i, float((off / bo).max()))
                assert (off_lse <= bl[fine]).all(), (b, i, float((off_lse / bl[fine]).max()))


MANY = tuple(int(x) for x in np.random.default_rng(3).integers(0, 1700, 130))
CASES = [  # D, P, heads, group, lens, N, dtype, mask, extras
    (128, 64, 2, 4, (3000, 10, 1500), 1, "bf16", None, {}),                 # every unit with another work-group
    (128, 16, 1, 5, (2049, 0, 1023), 3, "bf16", None, {}),                  # 15 rows
    (256, 32, 1, 4, (1800, 1), 6, "bf16", "tree", {}),                      # 24 rows
    (64, 8, 1, 7, (1500, 129), 4, "bf16", "tree", {"ragged": True}),        # 28 rows
    (128, 64, 1, 4, MANY, 1, "bf16", None, {}),                             # more requests than lanes
    (64, 64, 2, 1, MANY[:70], 5, "bf16", "tree", {"ragged": True}),
    (64, 32, 1, 2, MANY[:66], 7, "f32", None, {"ragged": True}),
    (128, 64, 1, 4, (2500, 700, 0), 16, "bf16", "tree", {}),                # 64 rows, four waves
    (128, 16, 1, 4, (2500, 0), 60, "bf16", "tree", {"ragged": True}),       # 240 rows, eight waves
    (64, 64, 1, 4, (1100, 2100), 60, "bf16", "tree", {}),
    (256, 64, 1, 2, (1300,), 60, "bf16", "tree", {}),
    (256, 16, 1, 3, (1200, 40), 30, "f32", "tree", {}),                     # 90 rows
    (128, 64, 1, 4, (2000, 5), 30, "f32", "tree", {"ragged": True}),
    (128, 32, 1, 4, (1300, 1400), 12, "f32", None, {}),                     # three blocks of 16 rows
    (64, 16, 1, 40, (1500, 0), 1, "f32", None, {}),                         # a node's heads fill no block of 16
    (128, 64, 1, 40, (1500, 77), 1, "bf16", None, {}),
    (128, 64, 1, 64, (1100, 300), 3, "bf16", "tree", {}),
    (128, 64, 1, 4, (700, 0, 2500), 300, "bf16", None, {"ragged": True}),   # chains, pairs of blocks are cut
    (128, 64, 1, 3, (1200,), 200, "f32", None, {}),
    (64, 128, 1, 24, (900, 1500), 30, "bf16", None, {}),                    # blocks of 240 rows in 256
    (128, 64, 1, 4, (1500, 33), 130, "bf16", "any", {"ragged": True}),      # three words of mask, rows that see nothing new
    (128, 64, 1, 4, (2000, 900), 1, "bf16", None, {"max_len": 100}),        # the hint is no promise
    (128, 64, 1, 4, (2000, 900), 50, "bf16", None, {"max_len": 1}),
    (128, 64, 2, 4, (900, 5, 1000), 1, "bf16", None, {"max_len": 1000}),    # whole blocks, one work-group each
]


@pytest.mark.parametrize("D,P,heads,group,lens,N,dtype,mask,extras", CASES)
def test_work_that_is_cut(D, P, heads, group, lens, N, dtype, mask, extras):
    print("deal", D, P, heads, group, lens[:4], len(lens), N, dtype, mask, extras, flush=True)
    rng = np.random.default_rng(D + P + N + group)
    B = len(lens)
    f = Bytes(D + N, lens, N, heads, D, P)
    n_new = rng.integers(0, N + 1, B) if extras.get("ragged") else np.full(B, N)
    q = torch.from_numpy(rng.standard_normal((B, N, heads * group, D)).astype(np.float32)).to(DTYPES[dtype])
    count = torch.from_numpy(n_new.astype(np.int32)).cuda() if extras.get("ragged") else None
    words = None
    if mask == "tree":
        parent = np.array([[-1] + [int(rng.integers(max(0, i - 9), i)) for i in range(1, N)] for _ in range(B)], np.int32)
        words = C.mars_tree_mask(torch.from_numpy(parent).cuda(), n_new=count)
        sees_of = lambda b: R.tree_sees(parent[b].tolist(), int(n_new[b]))[0]  # noqa: E731
    elif mask == "any":
        every = rng.random((B, N, N)) < 0.3
        every[:, 1::5] = False
        words = torch.from_numpy(R.words_of(every)).cuda()
        sees_of = lambda b: every[b]  # noqa: E731
    else:
        sees_of = lambda b: np.tril(np.ones((N, N), bool))  # noqa: E731
    out, lse = torch.full_like(q, 5.0, device="cuda"), torch.full((B, N, heads * group), 5.0, device="cuda")
    C.mars_kv_attention(f.pool, f.table, f.lens, q.cuda(), mask=words, n_new=count, max_len=extras.get("max_len", 0), out=out, lse=lse)
    check(f, lens, n_new, q, sees_of, out, lse, 1.0 / math.sqrt(D), dtype, group)
    again, lse2 = torch.empty_like(out), torch.empty_like(lse)
    C.mars_kv_attention(f.pool, f.table, f.lens, q.cuda(), mask=words, n_new=count, max_len=extras.get("max_len", 0), out=again, lse=lse2)
    assert torch.equal(again, out) and torch.equal(lse2, lse)


def test_logarithms_of_the_sums_are_exact_to_32_bits():
    """One key, queries and a key whose channels span eight powers of two: the sum's logarithm is the score, a sum of products that are exact in fp32.
    Each of the D additions and the shift rounds once: (D + 8) 2^-24 of the largest partial sum, which is at most sum |q k|, scaled."""
    print("exact", flush=True)
    for D, N, group in ((64, 1, 4), (128, 1, 4), (256, 1, 4), (128, 7, 4), (128, 16, 4), (64, 60, 4), (128, 60, 4), (256, 60, 1)):
        f = Bytes(D, (1, 1), N, 1, D, 64)
        g = torch.Generator("cuda").manual_seed(D + N)
        q = (torch.randn((2, N, group, D), device="cuda", generator=g) * torch.exp2(torch.randint(-8, 1, (D,), device="cuda", generator=g).float())).bfloat16()
        mask = torch.zeros((2, N, 1), dtype=torch.int64, device="cuda")
        lse = torch.empty((2, N, group), device="cuda")
        C.mars_kv_attention(f.pool, f.table, f.lens, q, mask=mask, lse=lse, scale=1.0)
        for b in range(2):
            k, _ = f.rows(b, 1, 0)
            want, size = q[b].double() @ k[0], q[b].double().abs() @ k[0].abs()
            assert ((lse[b].double() - want).abs() <= (D + 8) * 2.0 ** -24 * size + 2.0 ** -22 * want.abs()).all(), (D, N)
