"""Plain implementation of the paged 4-bit cache in 64 bits, written from include/mars_cache.h's text; test infrastructure only.

Rows are kept as codes and scales by (layer, page, head, token); their bytes in the pool's layout come from one function, ``place``.
"""
import numpy as np

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
NAN_SCALE = 255


def encode(x):
    """Codes (0 .. 15) and scale bytes of rows x [..., D], finite."""
    x = np.asarray(x, np.float64)
    blocks = x.reshape(*x.shape[:-1], -1, 32)
    top = np.abs(blocks).max(-1)
    e = np.full(top.shape, 1)
    for byte in range(1, 253):                    # the least at which the largest magnitude is below 7 scales
        e = np.where(top >= 7 * 2.0 ** (byte - 127), byte + 1, e)
    e = np.minimum(e, 252)
    y = np.abs(blocks) / 2.0 ** (e[..., None] - 127)
    off = np.abs(y[..., None] - GRID)
    least = off.min(-1, keepdims=True)
    near = off == least
    even = near & (np.arange(8) % 2 == 0)
    code = np.where(even.any(-1), even.argmax(-1), near.argmax(-1))
    code = np.where(np.signbit(blocks), code + 8, code)
    return code.reshape(x.shape).astype(np.uint8), e.astype(np.uint8)


def decode(code, byte):
    v = GRID[code & 7] * np.where(code >= 8, -1.0, 1.0)
    scale = np.where(byte == NAN_SCALE, np.nan, 2.0 ** (byte.astype(np.float64) - 127))
    return (v.reshape(*v.shape[:-1], -1, 32) * scale[..., None]).reshape(v.shape)


def stored(k, v):
    """What the cache holds of rows k, v [..., D] of one head: (codes, bytes) of both, poisoned where either is not finite."""
    bad = ~(np.isfinite(k).all(-1) & np.isfinite(v).all(-1))
    (ck, bk), (cv, bv) = (encode(np.where(bad[..., None], 0, x)) for x in (k, v))
    bk = np.where(bad[..., None], NAN_SCALE, bk).astype(np.uint8)
    return (ck, bk), (cv, bv)


def read_back(k, v):
    """Values that rows k, v read back as."""
    (ck, bk), (cv, bv) = stored(k, v)
    kk, vv = decode(ck, bk), decode(cv, bv)
    return kk, np.where(np.isnan(kk).any(-1, keepdims=True), np.nan, vv)


def place(D, P, t):
    """Offsets of token t's bytes in a head's part of a page: keys' codes, values' codes, keys' scales, values' scales."""
    i, s = np.arange(D // 2), np.arange(D // 32)
    key = t * (D // 2) + i
    value = P * D // 2 + (((t // 8) * (D // 8) + i // 4) * 8 + t % 8) * 4 + i % 4
    return key, value, P * D + t * (D // 32) + s, P * D + P * D // 32 + ((t // 8) * (D // 32) + s) * 8 + t % 8


def write(pool, layer, page, head, D, P, t, k, v):
    """One token's row into a pool of bytes [layers, pages, heads, blk]."""
    (ck, bk), (cv, bv) = stored(k, v)
    at = place(D, P, t)
    part = pool[layer, page, head]
    part[at[0]] = ck[0::2] | ck[1::2] << 4
    part[at[1]] = cv[0::2] | cv[1::2] << 4
    part[at[2]], part[at[3]] = bk, bv


def row(pool, layer, page, head, D, P, t):
    """Values of one token: (k, v)."""
    part = pool[layer, page, head]
    at = place(D, P, t)
    out = []
    for codes, scales in ((part[at[0]], part[at[2]]), (part[at[1]], part[at[3]])):
        code = np.empty(D, np.uint8)
        code[0::2], code[1::2] = codes & 15, codes >> 4
        out.append(decode(code, scales))
    if np.isnan(out[0]).any():
        out[1] = np.full(D, np.nan)
    return out


def tree_sees(parent, n):
    """[N, N]: row i sees node j; None for a malformed tree (then the root alone sees itself)."""
    N = len(parent)
    sees = np.zeros((N, N), bool)
    good = n == 0 or (parent[0] == -1 and all(0 <= parent[i] < i for i in range(1, n)))
    for i in range(n):
        if good or i == 0:
            j = i
            while j >= 0:
                sees[i, j] = True
                j = parent[j] if j else -1
    return sees, good


def words_of(sees):
    N = sees.shape[-1]
    W = (N + 63) // 64
    bits = np.zeros((*sees.shape[:-1], W), np.uint64)
    for j in range(N):
        bits[..., j // 64] |= np.where(sees[..., j], np.uint64(1) << np.uint64(j % 64), np.uint64(0))
    return bits.view(np.int64)


def attention(q, k, v, sees, scale):
    """Rows q [R, D] over keys and values [T, D] under sees [R, T]: (out, lse, sum of p |v|, largest of scale * sum |q_d k_d|).  A key that is NaN
    makes the rows that see it NaN."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    bad = np.isnan(k).any(-1) | np.isnan(v).any(-1)
    k, v = np.where(bad[:, None], 0, k), np.where(bad[:, None], 0, v)
    s = scale * (q @ k.T)
    s = np.where(sees, s, -np.inf)
    top = s.max(-1, keepdims=True) if s.shape[1] else np.full((len(q), 1), -np.inf)
    p = np.exp(s - np.where(np.isfinite(top), top, 0))
    total = p.sum(-1, keepdims=True)
    with np.errstate(divide="ignore", invalid="ignore"):
        p = np.where(total > 0, p / total, 0)
        lse = (top + np.log(total))[:, 0]
    out, mass = p @ v, p @ np.abs(v)
    worst = np.where(sees, scale * (np.abs(q) @ np.abs(k).T), 0).max(-1) if s.shape[1] else np.zeros(len(q))
    sick = (sees & bad).any(-1)
    out[sick], lse[sick] = np.nan, np.nan
    return out, lse, mass, worst


class Tables:
    """Page table, lengths and counts, one request after the other.  ``copied``: (from, to) pages."""
    OK, NO_PAGES, TOO_LONG, BAD_SEQUENCE, BAD_PATH, NOT_EMPTY = range(6)

    def __init__(self, pages, sequences, width, P):
        self.P, self.width = P, width
        self.table = np.full((sequences, width), -1, np.int32)
        self.lens, self.held = np.zeros(sequences, np.int32), np.zeros(sequences, np.int32)
        self.refs = np.zeros(pages, np.int32)

    def written(self, s, m):
        """Places in its row of the pages held by s that m new tokens go into."""
        return range(self.lens[s] // self.P, min(self.held[s], -(-(self.lens[s] + m) // self.P))) if m > 0 else range(0)

    def reserve(self, seqs, n):
        status, copied = [], []
        wants, into, asks = [], [], {}
        for i, (s, m) in enumerate(zip(seqs, n)):
            status.append(self.OK)
            into.append(range(0))
            wants.append(0)
            if not 0 <= s < len(self.lens):
                status[-1] = self.BAD_SEQUENCE
                continue
            need = -(-(self.lens[s] + m) // self.P)
            if need > self.width:
                status[-1] = self.TOO_LONG
                continue
            wants[-1] = max(0, need - self.held[s])
            into[-1] = self.written(s, m)
            for j in into[-1]:
                asks.setdefault(int(self.table[s, j]), []).append(i)
        # a page that others hold too is given up, but not by the last of its holders where all of them are here
        given = [[j for j in js if self.refs[self.table[seqs[i], j]] > 1
                  and (asks[self.table[seqs[i], j]][-1] != i or len(asks[self.table[seqs[i], j]]) < self.refs[self.table[seqs[i], j]])]
                 for i, js in enumerate(into)]
        free = [p for p in range(len(self.refs)) if self.refs[p] == 0]
        out = False
        for i, s in enumerate(seqs):
            k = wants[i] + len(given[i])
            if k == 0:
                continue
            out |= k > len(free)
            if out:
                status[i] = self.NO_PAGES
                continue
            got, free = free[:k], free[k:]
            self.refs[got] = 1
            for j, page in zip(given[i], got):
                old, self.table[s, j] = self.table[s, j], page
                self.refs[old] -= 1
                if j * self.P < self.lens[s]:        # committed tokens are in it
                    copied.append((old, page))
            for page in got[len(given[i]):]:
                self.table[s, self.held[s]] = page
                self.held[s] += 1
        for i, js in enumerate(into):                # the last holder, where an earlier one went without a page of its own
            if status[i] == self.OK and any(self.refs[self.table[seqs[i], j]] > 1 for j in js):
                status[i] = self.NO_PAGES
        return status, copied

    def fork(self, src, dst):
        status = []
        for a, z in zip(src, dst):
            if not (0 <= a < len(self.lens) and 0 <= z < len(self.lens)) or a == z:
                status.append(self.BAD_SEQUENCE)
            elif self.held[z]:
                status.append(self.NOT_EMPTY)
            else:
                status.append(self.OK)
                n = min(self.held[a], -(-self.lens[a] // self.P))
                self.table[z] = -1
                self.table[z, :n] = self.table[a, :n]
                self.refs[self.table[z, :n]] += 1
                self.lens[z], self.held[z] = self.lens[a], n
        return status

    def release(self, seqs):
        for s in seqs:
            if 0 <= s < len(self.lens):
                for i in range(self.held[s]):
                    self.refs[self.table[s, i]] -= 1
                    self.table[s, i] = -1
                self.lens[s] = self.held[s] = 0
