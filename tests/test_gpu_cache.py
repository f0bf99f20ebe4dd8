"""Rows into the 4-bit cache and out of it, and its pages, against the oracle: everything here is exact."""
import numpy as np
import pytest
import torch

from oracle import cache_ref as R
from paper_2601_15498_amd import cache as C
from tests.cache_util import DTYPES, Filled, rounded

pytestmark = pytest.mark.gpu


def report(*a):
    print(*a, flush=True)


ROWS = [  # D, P, heads, lens, N, dtype, ragged, strided
    (128, 64, 8, (0, 1, 63, 64, 65), 1, "bf16", False, False),
    (128, 64, 2, (0, 7, 8, 60, 129), 60, "bf16", True, True),
    (128, 16, 3, (5, 16, 0), 33, "f32", True, False),
    (64, 8, 5, (0, 3, 8, 15), 9, "bf16", True, True),
    (64, 256, 1, (255, 1), 2, "f32", False, True),
    (256, 32, 2, (0, 31, 40), 17, "bf16", True, False),
    (256, 128, 1, (126,), 5, "f32", False, True),
]


@pytest.mark.parametrize("D,P,heads,lens,N,dtype,ragged,strided", ROWS)
def test_rows_appended_and_read_back(D, P, heads, lens, N, dtype, ragged, strided):
    report("append", D, P, heads, lens, N, dtype)
    rng = np.random.default_rng(D + P + N)
    f = Filled(rng, lens, N, heads, D, P, layers=2, layer=1, sequences=len(lens) + 2)
    B = len(lens)
    n_new = rng.integers(0, N + 1, B) if ragged else np.full(B, N)
    scale = 2.0 ** rng.integers(-30, 30, (B, N, heads, 1))
    k, k64 = rounded(rng.standard_normal((B, N, heads, D)) * scale, dtype)
    v, v64 = rounded(rng.standard_normal((B, N, heads, D)), dtype)
    d = f.to()
    if strided:    # a slice of a projection's output, heads in front of nodes
        both = torch.zeros((B, 3 * heads, N, D), dtype=DTYPES[dtype], device="cuda")
        both[:, heads:2 * heads], both[:, 2 * heads:] = k.transpose(1, 2).cuda(), v.transpose(1, 2).cuda()
        kd, vd = both[:, heads:2 * heads].transpose(1, 2), both[:, 2 * heads:].transpose(1, 2)
    else:
        kd, vd = k.cuda(), v.cuda()
    status = torch.full((B,), 77, dtype=torch.int32, device="cuda")
    C.mars_kv_append(d["pool"], d["table"], d["lens"], kd, vd, layer=1, seqs=d["seqs"],
                     n_new=torch.from_numpy(n_new.astype(np.int32)).cuda() if ragged else None, status=status)
    for b in range(B):
        for i in range(n_new[b]):
            f.k[b][lens[b] + i], f.v[b][lens[b] + i] = k64[b, i], v64[b, i]
        f.write(b, range(lens[b], lens[b] + n_new[b]))
    assert status.tolist() == [0] * B
    assert np.array_equal(d["pool"].cpu().numpy(), f.pool)
    # read across everything that the sequences hold and past it
    first = np.array([max(-3, n - 11) for n in lens], np.int32)
    count = N + 11 + P
    rk, rv = C.mars_kv_read(d["pool"], d["table"], d["held"], layer=1, seqs=d["seqs"], first=torch.from_numpy(first).cuda(), N=count, head_dim=D,
                            dtype=DTYPES[dtype])
    want = np.zeros((2, B, count, heads, D))
    for b in range(B):
        s = f.seqs[b]
        for i in range(count):
            t = first[b] + i
            if 0 <= t < f.held[s] * P:
                for h in range(heads):
                    want[0, b, i, h], want[1, b, i, h] = R.row(f.pool, 1, f.table[s, t // P], h, D, P, t % P)
    assert np.array_equal(rk.double().cpu().numpy(), want[0], equal_nan=True)
    assert np.array_equal(rv.double().cpu().numpy(), want[1], equal_nan=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_edges_of_the_format(dtype):
    report("edges", dtype)
    D, P = 128, 8
    x = np.zeros((10, D), np.float32)
    x[0, :8] = [6, -0.25, 0.75, 1.25, -1.75, 2.5, 3.5, 5]               # ties
    x[1, 32] = 7.0
    x[2, 64:67] = [6.96875, -7, 0.4375]
    x[3] = 2.0 ** -126                                                 # the smallest scale
    x[4, 1] = 1.5 * 2.0 ** -127                                        # below it
    x[5] = 3.0e38
    x[5, ::2] = -1.0e37
    x[6, 5] = np.nan
    x[7, 127] = np.inf
    x[8] = -0.0
    x[9, ::3] = np.linspace(-9, 9, 43)
    t, x64 = rounded(x, dtype)
    f = Filled(np.random.default_rng(0), (0,), 12, 1, D, P)
    d = f.to()
    one = torch.ones_like(t)
    C.mars_kv_append(d["pool"], d["table"], d["lens"], t.view(1, 10, 1, D).cuda(), one.view(1, 10, 1, D).cuda())
    f.k[0][:10, 0], f.v[0][:10, 0] = x64, 1.0
    f.write(0, range(10))
    assert np.array_equal(d["pool"].cpu().numpy(), f.pool)
    k, v = C.mars_kv_read(d["pool"], d["table"], N=10, head_dim=D, dtype=torch.float32)
    assert torch.isnan(v[0, 6:8]).all() and torch.isnan(k[0, 6:8]).all() and (v[0, [0, 1, 2, 3, 4, 5, 8, 9]] == 1).all()


def test_append_says_where_it_could_not_write():
    report("append status")
    f = Filled(np.random.default_rng(1), (5, 14, 3), 2, 2, 64, 8, sequences=3, rows=False, stale=0)
    d = f.to()
    seqs = torch.tensor([f.seqs[0], -1, f.seqs[2], 3], dtype=torch.int32, device="cuda")
    k = torch.ones((4, 6, 2, 64), device="cuda")
    status = torch.empty(4, dtype=torch.int32, device="cuda")
    C.mars_kv_append(d["pool"], d["table"], d["lens"], k, k, seqs=seqs, status=status)
    # request 0 holds one page: 3 of its 6 rows have none; request 2 (3 + 6 of 8) misses the last
    assert status.tolist() == [C.MARS_KV_NO_PAGES, C.MARS_KV_BAD_SEQUENCE, C.MARS_KV_NO_PAGES, C.MARS_KV_BAD_SEQUENCE]
    k0, _ = C.mars_kv_read(d["pool"], d["table"], seqs=seqs, N=9, head_dim=64)
    assert (k0[0, 5:8] == 1).all() and (k0[0, 8] == 0).all() and (k0[2, 3:8] == 1).all() and (k0[1] == 0).all() and (k0[3] == 0).all()


@pytest.mark.parametrize("N", [1, 2, 60, 64, 65, 200, 1024])
def test_tree_masks(N):
    report("mask", N)
    rng = np.random.default_rng(N)
    B = 6
    parent = np.array([[-1] + [rng.integers(max(0, i - 9), i) for i in range(1, N)] for _ in range(B)], np.int32)
    parent[1] = np.arange(-1, N - 1)                                   # a chain
    n = np.array([N, N, N // 2, 0, N, N], np.int32)
    if N > 2:
        parent[4, N - 1] = N - 1
        parent[5, 0] = 0
    mask = torch.full((B, N, (N + 63) // 64), -1, dtype=torch.int64, device="cuda")
    status = torch.empty(B, dtype=torch.int32, device="cuda")
    C.mars_tree_mask(torch.from_numpy(parent).cuda(), n_new=torch.from_numpy(n).cuda(), mask=mask, status=status)
    got = mask.cpu().numpy()
    for b in range(B):
        sees, good = R.tree_sees(parent[b].tolist(), int(n[b]))
        assert status[b].item() == (0 if good else 1)
        assert np.array_equal(got[b], R.words_of(sees)), b


@pytest.mark.parametrize("D,P,heads,layers,N,alias", [(128, 64, 8, 3, 60, False), (64, 8, 3, 2, 9, True), (256, 16, 2, 1, 26, True),
                                                      (128, 8, 5, 2, 200, False)])
def test_accepted_rows_move_up(D, P, heads, layers, N, alias):
    report("commit", D, P, heads, layers, N)
    rng = np.random.default_rng(N)
    lens = (0, 1, 7, 8, 63, 64, 130, 20, 33)
    B = len(lens)
    f = Filled(rng, lens, N, heads, D, P, layers=layers, sequences=B + 1, rows=False)
    f.pool[:] = rng.integers(0, 256, f.pool.shape)
    accept = np.minimum([0, 1, 2, 3, 7, N - 1, N - 1, 4, 3], N - 1).astype(np.int32)
    path = np.full((B, N), -1, np.int32)
    for b in range(B):
        path[b, : accept[b]] = np.sort(rng.choice(np.arange(1, N), accept[b], replace=False))
    path[7, : accept[7]] = np.arange(1, accept[7] + 1)                  # a chain: nothing moves
    path[8, :3] = [2, 2, 5]                                             # no path
    seqs = f.seqs.copy()
    d = f.to()
    status = torch.empty(B, dtype=torch.int32, device="cuda")
    new = d["lens"] if alias else torch.full_like(d["lens"], -5)
    C.mars_kv_commit(d["pool"], d["table"], d["lens"], torch.from_numpy(accept).cuda(), torch.from_numpy(path).cuda(), page_size=P,
                     seqs=torch.from_numpy(seqs).cuda(), new_lens=None if alias else new, status=status)
    want = f.pool.copy()
    want_lens = f.lens.copy() if alias else np.full(B + 1, -5, np.int32)
    for b in range(B):
        s = seqs[b]
        want_lens[s] = f.lens[s]
        if b == 8:
            continue
        want_lens[s] = f.lens[s] + 1 + accept[b]
        for i in range(accept[b]):
            a, z = f.lens[s] + path[b, i], f.lens[s] + 1 + i
            at, to = np.concatenate(R.place(D, P, a % P)), np.concatenate(R.place(D, P, z % P))
            want[:, f.table[s, z // P], :, to] = f.pool[:, f.table[s, a // P], :, at]
    assert status.tolist() == [0] * 8 + [C.MARS_KV_BAD_PATH]
    assert np.array_equal(new.cpu().numpy(), want_lens)
    assert np.array_equal(d["pool"].cpu().numpy(), want)


def test_commit_refuses_what_is_no_path_or_has_no_page():
    report("commit status")
    f = Filled(np.random.default_rng(2), (4, 4, 4, 4, 4), 3, 1, 64, 8, sequences=5, rows=False, stale=3)
    d = f.to()
    seqs = torch.from_numpy(f.seqs).cuda()
    seqs[4] = 9
    accept = torch.tensor([3, -1, 6, 2, 1], dtype=torch.int32, device="cuda")     # (every sequence has one page, 8 tokens)
    path = torch.tensor([[1, 2, 5, -1, -1, -1]] * 5, dtype=torch.int32, device="cuda")
    path[3, 1] = 6
    status = torch.empty(5, dtype=torch.int32, device="cuda")
    before = d["pool"].clone()
    C.mars_kv_commit(d["pool"], d["table"], d["lens"], accept, path, page_size=8, seqs=seqs, status=status)
    assert status.tolist() == [C.MARS_KV_NO_PAGES, C.MARS_KV_BAD_PATH, C.MARS_KV_BAD_PATH, C.MARS_KV_BAD_PATH, C.MARS_KV_BAD_SEQUENCE]
    assert torch.equal(d["pool"], before) and d["lens"].tolist() == [4] * 5


def contents(t, pool, s):
    """Bytes of the committed tokens of a sequence: [layers, tokens, ...] page by page."""
    return pool[:, t.table[s, : -(-t.lens[s] // t.P)]]


@pytest.mark.parametrize("pages,P,sequences,width,layers,seed", [(40, 8, 12, 6, 2, 0), (5000, 16, 64, 100, 1, 1), (9000, 8, 40, 300, 1, 2), (17, 64, 9, 3, 3, 3)])
def test_pages_over_many_steps(pages, P, sequences, width, layers, seed):
    """A few dozen random steps: the tables follow the oracle's, and what a sequence has committed stays as it was."""
    report("pages", pages, P, sequences)
    rng = np.random.default_rng(seed)
    D, heads = 64, 1
    t = R.Tables(pages, sequences, width, P)
    pool = torch.from_numpy(rng.integers(0, 256, (layers, pages, heads, P * (D + D // 16)), dtype=np.uint8)).cuda()
    table, lens, held, refs = (torch.from_numpy(x.copy()).cuda() for x in (t.table, t.lens, t.held, t.refs))

    def same(what):
        for name, x, y in (("table", table, t.table), ("lens", lens, t.lens), ("held", held, t.held), ("refs", refs, t.refs)):
            assert np.array_equal(x.cpu().numpy(), y), (what, name)

    to = lambda x: torch.tensor(list(x), dtype=torch.int32, device="cuda")  # noqa: E731
    for step in range(40):
        kind = rng.choice(["reserve", "reserve", "reserve", "fork", "release"])
        status = torch.full((sequences,), 99, dtype=torch.int32, device="cuda")
        if kind == "reserve":
            seqs = [int(s) for s in rng.permutation(sequences)[: rng.integers(1, sequences + 1)]]
            if step % 7 == 3:
                seqs[0] = sequences if step % 2 else -1
            n = [int(x) for x in rng.integers(0, 3 * P, len(seqs))]
            before = pool.clone()
            want, copied = t.reserve(seqs, n)
            C.mars_kv_reserve(pool, table, lens, held, refs, to(n), page_size=P, seqs=to(seqs), status=status[: len(seqs)])
            assert status[: len(seqs)].tolist() == want
            for a, z in copied:
                before[:, z] = before[:, a]
            assert torch.equal(pool, before)
            # some of it is written and committed
            for s, m, ok in zip(seqs, n, want):
                if ok == 0 and m:
                    used = int(rng.integers(0, m + 1))
                    for i in range(t.lens[s] // P, -(-(t.lens[s] + m) // P)):
                        assert t.refs[t.table[s, i]] == 1
                    t.lens[s] += used
            lens.copy_(torch.from_numpy(t.lens))
        elif kind == "fork":
            empty = [s for s in range(sequences) if t.held[s] == 0]
            full = [s for s in range(sequences) if t.held[s]]
            if not empty or not full:
                continue
            dst = [int(s) for s in rng.permutation(empty)[: rng.integers(1, len(empty) + 1)]]
            src = [int(s) for s in rng.choice(full, len(dst))]
            if len(full) > 1 and step % 3 == 0:
                dst[0] = next(s for s in full if s not in src) if len(set(src)) < len(full) else dst[0]
            want = t.fork(src, dst)
            C.mars_kv_fork(table, lens, held, refs, to(src), to(dst), page_size=P, status=status[: len(src)])
            assert status[: len(src)].tolist() == want
        else:
            seqs = [int(s) for s in rng.permutation(sequences)[: rng.integers(1, max(2, sequences // 3))]]
            t.release(seqs)
            C.mars_kv_release(table, lens, held, refs, to(seqs + [-7]), status=status[: len(seqs) + 1])
            assert status[: len(seqs) + 1].tolist() == [0] * len(seqs) + [C.MARS_KV_BAD_SEQUENCE]
        same((step, kind))
    assert np.array_equal(np.bincount(t.table[t.table >= 0], minlength=pages), t.refs)


def test_reserve_of_more_requests_than_a_work_group_has_threads():
    report("reserve, 1500 requests")
    P, sequences, pages = 8, 1500, 4000
    t = R.Tables(pages, sequences, 4, P)
    t.reserve(range(0, 1400), [5] * 1400)
    t.lens[:1400] = 5
    t.fork(range(0, 100), range(1400, 1500))
    table, lens, held, refs = (torch.from_numpy(x.copy()).cuda() for x in (t.table, t.lens, t.held, t.refs))
    pool = torch.randint(0, 256, (1, pages, 1, P * 68), dtype=torch.uint8, device="cuda")
    before = pool.clone()
    want, copied = t.reserve(range(1500), [20] * 1500)
    status = C.mars_kv_reserve(pool, table, lens, held, refs, 20, page_size=P)
    assert status.tolist() == want and 1 in want and len(copied) == 100
    for a, z in copied:
        before[:, z] = before[:, a]
    assert torch.equal(pool, before)
    for x, y in ((table, t.table), (held, t.held), (refs, t.refs)):
        assert np.array_equal(x.cpu().numpy(), y)


def test_copied_pages():
    report("copy")
    pool = torch.randint(0, 256, (3, 20, 5, 64 * 136), dtype=torch.uint8, device="cuda")
    want = pool.clone()
    src, dst = torch.tensor([3, 3, 19, -1, 4, 5], dtype=torch.int32), torch.tensor([0, 7, 1, 2, 20, 6], dtype=torch.int32)
    for a, z in zip(src.tolist(), dst.tolist()):
        if 0 <= a < 20 and 0 <= z < 20:
            want[:, z] = pool[:, a]
    C.mars_kv_copy_pages(pool, src.cuda(), dst.cuda())
    assert torch.equal(pool, want)
