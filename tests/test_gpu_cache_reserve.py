"""mars_kv_reserve where a sequence goes on from an earlier token, and what its holders see of a page that one of them writes."""
import numpy as np
import pytest
import torch

from oracle import cache_ref as R
from paper_2601_15498_amd import cache as C

pytestmark = pytest.mark.gpu
D, HEADS = 64, 2


def tensors(t, pool):
    return [torch.from_numpy(x.copy()).cuda() for x in (pool, t.table, t.lens, t.held, t.refs)]


def ints(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


def rows_of(pool, table, held, n, seqs, layer=0):
    """Keys and values that sequences hold at their first n positions."""
    return torch.stack(C.mars_kv_read(pool, table, held, layer=layer, seqs=ints(seqs), N=n, head_dim=D, dtype=torch.float32))


@pytest.mark.parametrize("cut", [8, 16, 4, 13, 19, 20, 0])
@pytest.mark.parametrize("n", [8, 1, 30])
def test_a_branch_at_an_earlier_token_leaves_the_other_sequence_as_it_was(cut, n):
    """Sequence 1 is a copy of sequence 0's 20 tokens, cut at a page's border or inside a page, and goes on with rows of its own."""
    print("cut", cut, n, flush=True)
    P, pages = 8, 16
    t = R.Tables(pages, 2, 8, P)
    pool, table, lens, held, refs = tensors(t, np.full((2, pages, HEADS, P * (D + D // 16)), 0xFF, np.uint8))
    status = C.mars_kv_reserve(pool, table, lens, held, refs, 20, page_size=P, seqs=ints([0]))
    assert status.tolist() == [0]
    g = torch.Generator("cuda").manual_seed(cut)
    k = torch.randn((1, 20, HEADS, D), device="cuda", generator=g)
    for layer in range(2):
        C.mars_kv_append(pool, table, lens, k + layer, -k, layer=layer, seqs=ints([0]))
    lens[0] = 20
    C.mars_kv_fork(table, lens, held, refs, ints([0]), ints([1]), page_size=P)
    before = [rows_of(pool, table, held, 20, [0], layer) for layer in range(2)]
    assert not any(torch.isnan(x).any() for x in before)
    lens[1] = cut
    status = C.mars_kv_reserve(pool, table, lens, held, refs, n, page_size=P, seqs=ints([1]))
    assert status.tolist() == [0]
    own = torch.full((1, n, HEADS, D), 6.0, device="cuda")   # (a code of the format)
    for layer in range(2):
        C.mars_kv_append(pool, table, lens, own, own, layer=layer, seqs=ints([1]))
    for layer in range(2):
        assert torch.equal(rows_of(pool, table, held, 20, [0], layer), before[layer]), "the other sequence's tokens"
        mine = rows_of(pool, table, held, cut + n, [1], layer)
        assert torch.equal(mine[:, :, :cut], before[layer][:, :, :cut]), "the tokens in front of the cut"
        assert (mine[:, :, cut:] == 6).all()
    counts = np.bincount(table.cpu().numpy()[table.cpu().numpy() >= 0], minlength=pages)
    assert np.array_equal(counts, refs.cpu().numpy())


def write_rows(t, rng, pool, marks, stamp, s, begin, end):
    """Overwrites positions begin .. end - 1 of sequence s with bytes of their own, noted in `marks`."""
    for i in range(begin, end):
        page, at = t.table[s, i // t.P], np.concatenate(R.place(D, t.P, i % t.P))
        assert t.refs[page] == 1, (s, i)
        pool[:, page, :, at] = stamp[0] % 251
        marks[s, i] = stamp[0] % 251
        stamp[0] += 1


@pytest.mark.parametrize("pages,P,sequences,width,most,seed", [(150, 8, 12, 20, 5, 0), (2500, 8, 25, 150, 70, 1), (900, 16, 300, 20, 5, 2),
                                                               (33000, 8, 30, 90, 40, 3), (90, 32, 20, 7, 3, 4),
                                                               (150, 8, 12, 40, 30, 5), (60, 8, 8, 30, 20, 6)])
def test_committed_tokens_over_many_steps_with_lengths_that_fall(pages, P, sequences, width, most, seed):
    """Random steps; every row that a sequence has committed keeps its bytes, whatever the others do, and the tables follow the oracle's."""
    print("steps", pages, P, sequences, flush=True)
    rng = np.random.default_rng(seed)
    t = R.Tables(pages, sequences, width, P)
    pool, marks, stamp = np.zeros((1, pages, 1, P * (D + D // 16)), np.uint8), {}, [0]
    reserves = several = refused = 0
    for step in range(60):
        kind = rng.choice(["reserve", "reserve", "reserve", "fork", "fall", "release"], p=[0.15, 0.15, 0.15, 0.25, 0.22, 0.08])
        if kind == "reserve":
            few = rng.random() < 0.5
            seqs = [int(s) for s in rng.permutation(sequences)[: rng.integers(1, max(2, sequences // 4 if few else sequences) + 1)]]
            n = [int(x) for x in rng.integers(0, (2 if few else most) * P, len(seqs))]
            dev = tensors(t, pool)
            several += sum(len([j for j in t.written(s, m) if t.refs[t.table[s, j]] > 1]) > 1 for s, m in zip(seqs, n))
            want, copied = t.reserve(seqs, n)
            refused += R.Tables.NO_PAGES in want
            reserves += 1
            status = C.mars_kv_reserve(*dev, ints(n), page_size=P, seqs=ints(seqs))
            assert status.tolist() == want, step
            for a, z in copied:
                pool[:, z] = pool[:, a]
            for x, y, name in zip(dev, (pool, t.table, t.lens, t.held, t.refs), ("pool", "table", "lens", "held", "refs")):
                assert np.array_equal(x.cpu().numpy(), y), (step, name)
            for s, m, ok in zip(seqs, n, want):
                if ok == 0 and m:
                    write_rows(t, rng, pool, marks, stamp, s, t.lens[s], t.lens[s] + m)
                    t.lens[s] += int(rng.integers(0, m + 1))
        elif kind == "fork":
            empty, full = [s for s in range(sequences) if t.held[s] == 0], [s for s in range(sequences) if t.lens[s]]
            if not empty or not full:
                continue
            dst = [int(s) for s in rng.permutation(empty)[: rng.integers(1, len(empty) + 1)]]
            src = [int(s) for s in rng.choice(full, len(dst))]
            t.fork(src, dst)
            for a, z in zip(src, dst):
                marks.update({(z, i): marks[a, i] for i in range(t.lens[a])})
        elif kind == "fall":
            for s in rng.permutation(sequences)[: max(1, sequences // 3)]:
                t.lens[s] = rng.integers(0, t.lens[s] + 1)
                if rng.random() < 0.5:
                    t.lens[s] -= t.lens[s] % P
        else:
            t.release([int(s) for s in rng.permutation(sequences)[: max(1, sequences // 4)]])
        for s in range(sequences):
            for i in range(t.lens[s]):
                assert (pool[:, t.table[s, i // P], :, np.concatenate(R.place(D, P, i % P))] == marks[s, i]).all(), (step, kind, s, i)
    assert reserves and several, "no request had several shared pages to write: the case shows nothing"
    print(reserves, "reserves,", several, "requests with several shared pages,", refused, "calls that ran out of pages", flush=True)


def test_all_holders_of_several_pages_ask_for_room():
    print("all holders", flush=True)
    P = 8
    t = R.Tables(12, 3, 6, P)
    t.reserve([0], [30])
    t.lens[0] = 30
    t.fork([0, 0], [1, 2])
    assert t.refs[:4].tolist() == [3] * 4
    t.lens[:] = 10                                   # inside the second page; all three write into pages 1 and 2
    pool = np.random.default_rng(0).integers(0, 256, (1, 12, 1, P * (D + D // 16)), dtype=np.uint8)
    dev = tensors(t, pool)
    want, copied = t.reserve([2, 0, 1], [12, 9, 14])
    assert want == [0, 0, 0] and copied == [(1, 4), (1, 6)]
    assert t.table[:, :4].tolist() == [[0, 6, 7, 3], [0, 1, 2, 3], [0, 4, 5, 3]] and t.refs.tolist() == [3, 1, 1, 3, 1, 1, 1, 1, 0, 0, 0, 0]
    status = C.mars_kv_reserve(*dev, ints([12, 9, 14]), page_size=P, seqs=ints([2, 0, 1]))
    assert status.tolist() == want
    for a, z in copied:
        pool[:, z] = pool[:, a]
    for x, y in zip(dev, (pool, t.table, t.lens, t.held, t.refs)):
        assert np.array_equal(x.cpu().numpy(), y)
