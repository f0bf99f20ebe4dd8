"""Caches filled row by row by the oracle, for the tests of the 4-bit cache."""
import numpy as np
import torch

from oracle import cache_ref as R

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def rounded(x, dtype):
    """x as the device gets it (a tensor on the CPU) and as numbers."""
    t = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(DTYPES[dtype])
    return t, t.double().numpy()


class Filled:
    """Sequences of the given lengths (with room for `room` tokens each) in pages dealt out at random; bytes that no row owns are `stale`."""

    def __init__(self, rng, lens, room, heads, D, P, *, layers=1, layer=0, spare=2, sequences=None, stale=0xFF, width=None, rows=True):
        self.D, self.P, self.heads, self.layer = D, P, heads, layer
        slots = rng.permutation(sequences or len(lens))[: len(lens)]
        held = [-(-(n + room) // P) for n in lens]
        pages = sum(held) + spare
        order = rng.permutation(pages)
        self.width = width or max(held) + 1
        S = sequences or len(lens)
        self.seqs = slots.astype(np.int32)
        self.table = np.full((S, self.width), -1, np.int32)
        self.lens, self.held = np.zeros(S, np.int32), np.zeros(S, np.int32)
        self.refs = np.zeros(pages, np.int32)
        at = 0
        for s, n, h in zip(slots, lens, held):
            self.table[s, :h] = order[at: at + h]
            self.refs[order[at: at + h]] = 1
            self.lens[s], self.held[s] = n, h
            at += h
        self.pool = np.full((layers, pages, heads, P * (D + D // 16)), stale, np.uint8)
        if rows:
            self.k = [rng.standard_normal((n + room, heads, D)) * (1 + 3 * (np.arange(D) % 16 == 5)) for n in lens]
            self.v = [rng.standard_normal((n + room, heads, D)) for n in lens]
            for b, s in enumerate(slots):
                self.write(b, range(len(self.k[b])))

    def write(self, b, tokens):
        for t in tokens:
            for h in range(self.heads):
                R.write(self.pool, self.layer, self.table[self.seqs[b], t // self.P], h, self.D, self.P, t % self.P, self.k[b][t, h], self.v[b][t, h])

    def values(self, b, count, head):
        """Keys and values [count, D] of a request, out of the pool."""
        s = self.seqs[b]
        rows = [R.row(self.pool, self.layer, self.table[s, t // self.P], head, self.D, self.P, t % self.P) for t in range(count)]
        return (np.array([r[0] for r in rows]).reshape(count, self.D), np.array([r[1] for r in rows]).reshape(count, self.D))

    def to(self, device="cuda"):
        return {n: torch.from_numpy(getattr(self, n)).to(device) for n in ("pool", "table", "lens", "held", "refs", "seqs")}
