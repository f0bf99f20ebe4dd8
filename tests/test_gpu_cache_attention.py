"""Attention over the 4-bit cache against the oracle in 64 bits.

Bounds, derived: u = 2^-8 is the unit roundoff of bf16 (eight significant bits: 1 + 2^-8 lies
halfway between 1 and its neighbour 1 + 2^-7).  For bf16 rows every probability is rounded once (u p_j, so u sum p |v| in the
result) and the result once (u |o|).  Beside that, for both types, fp32 arithmetic: a score is a sum of D exact products (three per product
for fp32 rows: their split is exact to 2^-24 of the query), off by at most (D + 8) 2^-24 scale sum |q k|; the exponent of a probability is off by
that and by the rounding of the shifted score (2^-22 |s| covers the product with log2 e and the difference); a power of two is good to 2^-22,
sums of T terms to T 2^-24 of their magnitude.  A probability's relative error moves the result by at most twice that times sum p |v|.
"""
import math

import numpy as np
import pytest
import torch

from oracle import cache_ref as R
from paper_2601_15498_amd import cache as C
from tests.cache_util import DTYPES, Filled, rounded

pytestmark = pytest.mark.gpu
U = 2.0 ** -8


def bounds(dtype, D, T, out, lse, mass, worst):
    score = (D + 8) * 2.0 ** -24 * worst + 2.0 ** -22 * (worst + np.abs(np.where(np.isfinite(lse), lse, 0))) + 2.0 ** -22 + T * 2.0 ** -24
    of_out = 2.2 * score[:, None] * mass + 1e-30
    if dtype == "bf16":
        of_out = of_out + 1.01 * U * (mass + np.abs(out))
    return of_out, 1.1 * score + 2.0 ** -22 * (1 + np.abs(np.where(np.isfinite(lse), lse, 0)))


def check(f, lens, n_new, q64, sees_of, out, lse, scale, dtype, group):
    """sees_of(b): [n, n] among the nodes, or [N, N]."""
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    B, N, Hq, D = out.shape
    worst_of = 0.0
    for b in range(B):
        n = n_new[b]
        assert (out[b, n:] == 0).all() and (lse[b, n:] == -np.inf).all()
        if n == 0:
            continue
        sees = np.concatenate([np.ones((n, lens[b]), bool), sees_of(b)[:n, :n]], 1)
        for h in range(f.heads):
            k, v = f.values(b, lens[b] + n, h)
            for g in range(group):
                want, want_lse, mass, most = R.attention(q64[b, :n, h * group + g], k, v, sees, scale)
                got, got_lse = out[b, :n, h * group + g], lse[b, :n, h * group + g]
                bo, bl = bounds(dtype, D, sees.shape[1], want, want_lse, mass, most)
                assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isnan(got_lse), np.isnan(want_lse)), (b, h, g)
                assert np.array_equal(np.isneginf(got_lse), np.isneginf(want_lse)), (b, h, g)
                fine = np.isfinite(want_lse)
                off, off_lse = np.abs(got - want)[fine], np.abs(got_lse - want_lse)[fine]
                assert (off <= bo[fine]).all(), (b, h, g, float((off / bo[fine]).max()))
                assert (off_lse <= bl[fine]).all(), (b, h, g, float((off_lse / bl[fine]).max()))
                assert (got[np.isneginf(want_lse)] == 0).all()
                if fine.any():
                    worst_of = max(worst_of, float((off / bo[fine]).max()))
    return worst_of


CASES = [  # D, P, heads, group, lens, N, dtype, mask, extras
    (128, 64, 2, 4, (0, 1, 31, 32, 33, 127, 128, 129, 300), 1, "bf16", None, {}),
    (128, 64, 1, 7, (0, 5, 200), 1, "f32", None, {}),
    (64, 8, 2, 4, (0, 3, 77, 130), 3, "bf16", None, {}),
    (128, 16, 3, 1, (0, 16, 90, 257), 7, "f32", None, {}),
    (256, 32, 1, 2, (0, 40, 100), 9, "bf16", "tree", {}),
    (256, 16, 1, 3, (0, 70), 11, "f32", "tree", {}),
    (128, 64, 2, 4, (0, 1, 100, 391), 9, "bf16", "tree", {}),           # 36 rows
    (128, 64, 1, 8, (3, 250), 4, "bf16", "tree", {"ragged": True}),     # 32 rows
    (128, 64, 2, 4, (0, 70, 300), 60, "bf16", "tree", {"ragged": True}),  # 240 rows
    (64, 16, 1, 3, (0, 30, 150), 26, "f32", "tree", {"ragged": True}),
    (256, 8, 1, 4, (0, 50, 90), 60, "bf16", "tree", {}),
    (128, 32, 1, 2, (5, 60), 130, "bf16", "tree", {"ragged": True}),    # three words of mask
    (128, 64, 1, 5, (0, 33, 64), 50, "bf16", "any", {"ragged": True}),  # any mask, rows that see nothing
    (64, 8, 1, 1, (0, 0, 9), 70, "f32", "any", {}),
    (128, 64, 1, 4, (0, 77), 200, "bf16", None, {}),                    # a prompt
    (64, 128, 1, 4, (0, 100), 150, "bf16", None, {"ragged": True}),
    (256, 64, 1, 1, (30,), 140, "bf16", None, {}),
    (128, 16, 1, 2, (50, 0), 80, "f32", None, {"ragged": True}),
]


@pytest.mark.parametrize("D,P,heads,group,lens,N,dtype,mask,extras", CASES)
def test_attention(D, P, heads, group, lens, N, dtype, mask, extras):
    print("attention", D, P, heads, group, lens, N, dtype, mask, extras, flush=True)
    rng = np.random.default_rng(D * 7 + P + N + group)
    B = len(lens)
    f = Filled(rng, lens, N, heads, D, P, layers=2, layer=1, sequences=B + 2)
    d = f.to()
    n_new = rng.integers(0, N + 1, B) if extras.get("ragged") else np.full(B, N)
    q, q64 = rounded(rng.standard_normal((B, N, heads * group, D)), dtype)
    words = None
    if mask == "tree":
        parent = np.array([[-1] + [int(rng.integers(max(0, i - 9), i)) for i in range(1, N)] for _ in range(B)], np.int32)
        nd = torch.from_numpy(n_new.astype(np.int32)).cuda()
        words = C.mars_tree_mask(torch.from_numpy(parent).cuda(), n_new=nd)
        sees_of = lambda b: R.tree_sees(parent[b].tolist(), int(n_new[b]))[0]  # noqa: E731
    elif mask == "any":
        every = rng.random((B, N, N)) < 0.3
        every[:, 1::5] = False
        words = torch.from_numpy(R.words_of(every)).cuda()
        sees_of = lambda b: every[b]  # noqa: E731
    else:
        sees_of = lambda b: np.tril(np.ones((N, N), bool))  # noqa: E731
    scale = 1.0 / math.sqrt(D)
    out, lse = torch.full_like(q, 5.0, device="cuda"), torch.full((B, N, heads * group), 5.0, device="cuda")
    kw = dict(layer=1, seqs=d["seqs"], mask=words, n_new=torch.from_numpy(n_new.astype(np.int32)).cuda() if extras.get("ragged") else None)
    C.mars_kv_attention(d["pool"], d["table"], d["lens"], q.cuda(), out=out, lse=lse, **kw)
    share = check(f, lens, n_new, q64, sees_of, out, lse, scale, dtype, group)
    print("largest share of the bound:", share, flush=True)
    # the same bits again, and from rows that lie apart
    wide = torch.zeros((B, heads * group, N, 2 * D), dtype=q.dtype, device="cuda")
    wide[..., :D] = q.cuda().transpose(1, 2)
    out2 = torch.full((B, heads * group, N, 2 * D), 7.0, dtype=q.dtype, device="cuda")
    lse2 = torch.empty_like(lse)
    C.mars_kv_attention(d["pool"], d["table"], d["lens"], wide[..., :D].transpose(1, 2), out=out2[..., D:].transpose(1, 2), lse=lse2, **kw)
    assert torch.equal(out2[..., D:].transpose(1, 2), out) and torch.equal(lse2, lse) and (out2[..., :D] == 7).all()


@pytest.mark.parametrize("dtype,N,group", [("bf16", 12, 2), ("f32", 12, 1), ("bf16", 30, 4)])
def test_a_row_that_is_not_finite_is_seen_by_its_descendants_alone(dtype, N, group):
    print("poison", dtype, N, flush=True)
    rng = np.random.default_rng(5)
    D, P, heads, lens = 128, 16, 2, (40, 9, 0)
    f = Filled(rng, lens, N, heads, D, P)
    d = f.to()
    k = [rng.standard_normal((3, N, heads, D)) for _ in range(2)]
    k[0][0, 4, 1, 7] = np.nan           # a node's key, of one head
    k[1][1, 2, 0, 100] = np.inf         # a node's value
    k[1][2, 0, 0, 0] = -np.inf          # the root's
    (kt, k64), (vt, v64) = rounded(k[0], dtype), rounded(k[1], dtype)
    C.mars_kv_append(d["pool"], d["table"], d["lens"], kt.cuda(), vt.cuda(), seqs=d["seqs"])
    f.pool = d["pool"].cpu().numpy()
    parent = np.array([[-1] + [int(rng.integers(0, i)) for i in range(1, N)] for _ in range(3)], np.int32)
    words = C.mars_tree_mask(torch.from_numpy(parent).cuda())
    q, q64 = rounded(rng.standard_normal((3, N, heads * group, D)), dtype)
    out, lse = torch.empty_like(q, device="cuda"), torch.empty((3, N, heads * group), device="cuda")
    C.mars_kv_attention(d["pool"], d["table"], d["lens"], q.cuda(), seqs=d["seqs"], mask=words, out=out, lse=lse)
    sees_of = lambda b: R.tree_sees(parent[b].tolist(), N)[0]  # noqa: E731
    check(f, lens, [N] * 3, q64, sees_of, out, lse, 1.0 / math.sqrt(D), dtype, group)
    sick = torch.isnan(out[0, :, group:]).all(-1).all(-1).cpu().numpy()
    assert np.array_equal(sick, sees_of(0)[:, 4]) and sick.any() and not sick.all()
    assert not torch.isnan(out[0, :, :group]).any() and torch.isnan(out[2, :, :group]).all()


def test_sequences_and_pages_outside_the_cache():
    print("outside", flush=True)
    rng = np.random.default_rng(6)
    f = Filled(rng, (100, 50), 1, 1, 64, 8, sequences=2)
    f.table[f.seqs[1], 3] = 10 ** 6
    d = f.to()
    seqs = torch.tensor([f.seqs[0], f.seqs[1], -1, 2], dtype=torch.int32, device="cuda")
    q, q64 = rounded(rng.standard_normal((4, 1, 2, 64)), "bf16")
    out, lse = torch.full_like(q, 3.0, device="cuda"), torch.empty((4, 1, 2), device="cuda")
    C.mars_kv_attention(d["pool"], d["table"], d["lens"], q.cuda(), seqs=seqs, out=out, lse=lse)
    assert torch.isnan(out[1]).all() and torch.isnan(lse[1]).all()
    assert (out[2:] == 0).all() and (lse[2:] == -math.inf).all()
    check(f, (100,), [1], q64, lambda b: np.ones((1, 1), bool), out[:1], lse[:1], 0.125, "bf16", 2)
    # a length past the table: the keys that cannot be there are NaN
    d["lens"][int(f.seqs[0])] = 10 ** 9
    C.mars_kv_attention(d["pool"], d["table"], d["lens"], q[:1].cuda(), seqs=seqs[:1].contiguous(), out=out[:1], lse=lse[:1])
    assert torch.isnan(out[0]).all()


@pytest.mark.parametrize("scale,size", [(1.0, 30.0), (0.01, 1.0), (3.0, 10.0)])
def test_scores_far_from_each_other(scale, size):
    """Scores that grow along the sequence (the reference moves all the time) or fall, from probabilities near one to none."""
    print("scores", scale, size, flush=True)
    rng = np.random.default_rng(8)
    D, P, lens, N = 128, 64, (700, 700), 2
    f = Filled(rng, lens, N, 1, D, P, rows=False)
    f.k, f.v = [], []
    for b in range(2):
        ramp = np.linspace(0, size, 702) if b == 0 else np.linspace(size, 0, 702)
        k = rng.standard_normal((702, 1, D)) * 0.1
        k[:, 0, 0] = ramp
        f.k.append(k)
        f.v.append(rng.standard_normal((702, 1, D)))
        f.write(b, range(702))
    d = f.to()
    for dtype in ("bf16", "f32"):
        x = rng.standard_normal((2, N, 4, D))
        x[..., 0] = np.abs(x[..., 0]) + 1
        x[:, :, 3, 0] *= -1
        q, q64 = rounded(x, dtype)
        out, lse = torch.empty_like(q, device="cuda"), torch.empty((2, N, 4), device="cuda")
        C.mars_kv_attention(d["pool"], d["table"], d["lens"], q.cuda(), seqs=d["seqs"], scale=scale, out=out, lse=lse)
        check(f, lens, [N] * 2, q64, lambda b: np.tril(np.ones((N, N), bool)), out, lse, scale, dtype, 4)


def plain(pool, table, n, q, D, P, scale):
    """One request on the GPU in 64 bits, from the bytes: q [R, D], committed tokens only."""
    t = torch.arange(n, device="cuda")
    part = pool[table[t // P].long()][:, 0]
    t = t % P
    c = torch.arange(D, device="cuda")
    grid = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64, device="cuda")

    def values(code_at, scale_at):
        byte = part.gather(1, code_at).int()
        return grid[torch.where(c % 2 == 1, byte >> 4, byte & 15).long()] * torch.exp2(part.gather(1, scale_at).double() - 127)

    k = values(t[:, None] * (D // 2) + c // 2, P * D + t[:, None] * (D // 32) + c // 32)
    v = values(P * D // 2 + (t[:, None] // 8) * 4 * D + (c // 8) * 32 + (t[:, None] % 8) * 4 + c % 8 // 2,
               P * D + P * D // 32 + (t[:, None] // 8) * (D // 4) + c // 32 * 8 + t[:, None] % 8)
    z = scale * (q.double() @ k.T)
    p = torch.softmax(z, 1)
    return p @ v, torch.logsumexp(z, 1), p @ v.abs(), (scale * (q.double().abs() @ k.abs().T)).amax(1)


@pytest.mark.parametrize("dtype,N", [("bf16", 1), ("bf16", 26), ("f32", 1)])
def test_a_long_sequence_far_into_the_pool(dtype, N):
    """100 003 tokens whose rows lie more than 4 GiB into the pool, in pages in no order."""
    print("long", dtype, N, flush=True)
    D, P, n = 128, 64, 100003
    layers, pages = 3, 200000
    g = torch.Generator("cuda").manual_seed(N)
    pool = torch.empty((layers, pages, 1, P * (D + D // 16)), dtype=torch.uint8, device="cuda")
    assert pool[2].data_ptr() - pool.data_ptr() > 1 << 31 and pool.numel() > 1 << 32
    W = -(-(n + N) // P)
    table = (torch.randperm(pages - 150000, device="cuda", generator=g)[:W] + 150000).int()[None].contiguous()
    part = torch.randint(0, 256, (W, 1, P * (D + D // 16)), dtype=torch.uint8, device="cuda", generator=g)
    part[:, :, P * D:] = torch.randint(124, 128, (W, 1, P * (D // 16)), dtype=torch.uint8, device="cuda", generator=g)
    pool[2, table[0].long()] = part
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    mask = torch.zeros((1, N, 1), dtype=torch.int64, device="cuda")     # committed tokens alone
    q = torch.randn((1, N, 4, D), device="cuda", generator=g).to(DTYPES[dtype])
    out, lse = C.mars_kv_attention(pool, table, lens, q, layer=2, mask=mask, lse=torch.empty((1, N, 4), device="cuda"))
    scale = 1 / math.sqrt(D)
    want, want_lse, mass, worst = (x.cpu().numpy() for x in plain(pool[2], table[0], n, q[0].reshape(N * 4, D), D, P, scale))
    bo, bl = bounds(dtype, D, n, want, want_lse, mass, worst)
    assert (np.abs(out[0].reshape(N * 4, D).double().cpu().numpy() - want) <= bo).all()
    assert (np.abs(lse[0].reshape(-1).double().cpu().numpy() - want_lse) <= bl).all()


def test_on_another_stream_and_in_a_graph():
    print("graph", flush=True)
    rng = np.random.default_rng(9)
    f = Filled(rng, (200, 90, 3), 8, 2, 128, 16)
    d = f.to()
    parent = torch.from_numpy(np.array([[-1, 0, 0, 1, 1, 2, 5]] * 3, np.int32)).cuda()
    k, _ = rounded(rng.standard_normal((3, 7, 2, 128)), "bf16")
    k = k.cuda()
    q = rounded(rng.standard_normal((3, 7, 8, 128)), "bf16")[0].cuda()
    mask = torch.empty((3, 7, 1), dtype=torch.int64, device="cuda")
    out, lse = torch.empty_like(q), torch.empty((3, 7, 8), device="cuda")
    work = C.alloc_attention_workspace(d["pool"], d["table"], q)
    accept, path = torch.tensor([2, 0, 1], dtype=torch.int32, device="cuda"), torch.full((3, 7), -1, dtype=torch.int32, device="cuda")
    path[0, :2], path[2, 0] = torch.tensor([2, 5]), 1
    new = torch.empty_like(d["lens"])
    room = C.alloc_reserve_workspace(d["pool"], 3)
    status = torch.empty(3, dtype=torch.int32, device="cuda")

    def step():
        C.mars_kv_reserve(d["pool"], d["table"], d["lens"], d["held"], d["refs"], 7, page_size=16, seqs=d["seqs"], status=status, workspace=room)
        C.mars_tree_mask(parent, mask=mask)
        C.mars_kv_append(d["pool"], d["table"], d["lens"], k, k, seqs=d["seqs"])
        C.mars_kv_attention(d["pool"], d["table"], d["lens"], q, seqs=d["seqs"], mask=mask, out=out, lse=lse, workspace=work)
        C.mars_kv_commit(d["pool"], d["table"], d["lens"], accept, path, page_size=16, seqs=d["seqs"], new_lens=new)

    start = d["pool"].clone()
    step()
    torch.cuda.synchronize()
    want = [x.clone() for x in (out, lse, new, d["pool"])]
    stream = torch.cuda.Stream()
    for x in (d["pool"], out, lse):
        x.fill_(0) if x is not d["pool"] else x.copy_(start)
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    stream.synchronize()
    for x, y in zip((out, lse, new, d["pool"]), want):
        assert torch.equal(x, y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        d["pool"].copy_(start)
        out.fill_(i)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip((out, lse, new, d["pool"]), want):
            assert torch.equal(x, y), i
        torch.mm(torch.randn(64, 64, device="cuda"), torch.randn(64, 64, device="cuda"))
