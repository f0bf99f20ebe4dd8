"""The paged 4-bit cache around a verification step, as cases that can be timed and compared.

A serving step of speculative decoding, layer by layer: the keys and values of the drafted nodes go into the cache
(``mars_kv_append``), every node attends the committed tokens and its own ancestors there (``mars_tree_mask``,
``mars_kv_attention``); then, once the logits are verified, the accepted path's rows move up behind the committed ones
(``mars_kv_commit``).  Requests that branch share their pages until one of them writes (``mars_kv_fork``,
``mars_kv_reserve``), and give them back (``mars_kv_release``).

The cache.  ``pool`` [layers, pages, kv heads, bytes]; a page holds P tokens, and of a head P * (D + D/16) bytes: its
keys' codes [P][D/2], its values' codes [P/8][D/8][8][4] (eight tokens' codes of the same eight channels beside each
other), its keys' scales [P][D/32], its values' scales [P/8][D/32][8].  A code is 4 bits (sign, two bits of exponent, one of
mantissa: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives), the even channel in the low half of a byte; 32 channels of a
token share a scale 2^(byte - 127).  ``page_table`` [sequences, width] (-1: none), ``lens`` (committed tokens), ``held``
(pages) and ``refs`` [pages] (sequences that hold a page; 0: free), all int32.

Head layouts are those of the target models the workloads stand for: 32 query heads over 8 of the cache, 64 over 8, 40
over 40, and a few others in drawn cases; node counts those of the benchmark's trees and chains.
"""
import math

import torch

own = False          # which side `run` is: the plain form, or the framework's operators

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------------------------------------------------- cases

def _attention(B, N, Hq, Hkv, D, P, lo, hi, *, tree=False, dtype="bf16", L=1):
    return dict(op="attention", B=B, N=N, Hq=Hq, Hkv=Hkv, D=D, P=P, lo=lo, hi=hi, tree=tree, dtype=dtype, L=L)


def _append(B, N, Hkv, D, P, lo, hi, *, ragged=False, dtype="bf16"):
    return dict(op="append", B=B, N=N, Hkv=Hkv, D=D, P=P, lo=lo, hi=hi, ragged=ragged, dtype=dtype, L=1)


def _commit(B, N, Hkv, D, P, lo, hi, L):
    return dict(op="commit", B=B, N=N, Hkv=Hkv, D=D, P=P, lo=lo, hi=hi, L=L)


def _fork(B, children, room, Hkv, D, P, lo, hi, L):
    return dict(op="fork", B=B, children=children, N=room, Hkv=Hkv, D=D, P=P, lo=lo, hi=hi, L=L)


def listed():
    return [
        # One user, one token over a thousand cached ones: launches and latency.
        dict(_attention(1, 1, 32, 8, 128, 64, 1021, 1021), name="attend_one"),
        # Ordinary decoding of 64 users, lengths all over the place: the cache is streamed.
        dict(_attention(64, 1, 32, 8, 128, 64, 500, 8192), name="attend_tokens"),
        # The benchmark's batch of drafted trees: 16 requests of 60 nodes.
        dict(_attention(16, 60, 32, 8, 128, 64, 1024, 8191, tree=True), name="attend_trees"),
        # Long contexts, the last of eight layers (rows lie more than 4 GB into the pool), a wider group of query heads.
        dict(_attention(4, 26, 64, 8, 128, 64, 60001, 131071, tree=True, L=8), name="attend_long"),
        # A part of a prompt, with what was cached before it.
        dict(_attention(2, 2048, 32, 8, 128, 64, 1000, 2047), name="attend_prompt"),
        # Chains of six drafts in 32 bits, a head of the cache for every query head, short pages.
        dict(_attention(8, 7, 40, 40, 128, 16, 3, 2000, dtype="f32"), name="attend_chains_f32"),
        # A step's nodes into one layer's cache, ...
        dict(_append(16, 60, 8, 128, 64, 1024, 8191), name="append_trees"),
        # ... and prompts of different lengths.
        dict(_append(8, 8192, 8, 128, 64, 0, 100, ragged=True), name="append_prompts"),
        # The accepted paths of the benchmark's batch, in all 32 layers, ...
        dict(_commit(16, 60, 8, 128, 64, 300, 1000, 32), name="commit_trees"),
        # ... and of the largest batch of trees, with short pages.
        dict(_commit(256, 26, 8, 128, 16, 20, 150, 32), name="commit_many"),
        # One request is sampled twice: its children drop what they had, share its pages, get room for a step.
        dict(_fork(1, 2, 60, 8, 128, 64, 1000, 1000, 32), name="fork_one"),
        # 16 requests with eight children each.
        dict(_fork(16, 8, 60, 8, 128, 64, 500, 3000, 32), name="fork_many"),
    ]


def _spread(rng, lo, hi):
    """A whole number of lo .. hi; over its logarithm where that spans more than a factor of ten."""
    if hi > 10 * lo:
        return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))
    return rng.randint(lo, hi)


_HEADS = ((32, 8), (64, 8), (40, 40), (64, 4), (16, 8), (12, 4), (8, 1), (28, 4))


def _cost(c):
    w = work(c)
    return w["bytes"] / 8e12 + w["flops"] / 4e14


def draw(rng):
    op = rng.choice(("attention", "attention", "attention", "append", "commit", "fork"))
    most = max(_cost(c) for c in listed() if c["op"] == op)
    while True:
        Hq, Hkv = rng.choice(_HEADS)
        D = rng.choice((64, 128, 128, 128, 256))
        P = rng.choice((8, 16, 32, 64, 64, 128))
        if op == "attention":
            kind = rng.choice(("token", "chain", "tree", "tree", "prompt"))
            B = _spread(rng, 1, 64) if kind != "prompt" else rng.randint(1, 4)
            N = {"token": 1, "chain": rng.randint(2, 16), "tree": rng.randint(2, 64), "prompt": _spread(rng, 65, 2048)}[kind]
            hi = _spread(rng, 1, 131071)
            c = _attention(B, N, Hq, Hkv, D, P, rng.randint(hi // 8, hi), hi, tree=kind == "tree",
                           dtype="f32" if kind != "prompt" and rng.random() < 0.25 else "bf16", L=rng.choice((1, 1, 2)))
            # (the plain form widens the cache and keeps its scores)
            if B * (hi + N) * Hkv * D > 5.5e8 or B * Hq * N * (hi + N) > 9e8:
                continue
        elif op == "append":
            N, hi = _spread(rng, 1, 8192), _spread(rng, 1, 8192)
            c = _append(_spread(rng, 1, 64), N, Hkv, D, P, rng.randint(0, hi), hi, ragged=rng.random() < 0.5,
                        dtype="f32" if rng.random() < 0.25 else "bf16")
        elif op == "commit":
            hi = _spread(rng, 1, 1000)
            c = _commit(_spread(rng, 1, 256), rng.randint(2, 64), Hkv, D, P, rng.randint(0, hi), hi, rng.randint(1, 36))
        else:
            hi = _spread(rng, 1, 3000)
            c = _fork(_spread(rng, 1, 16), rng.randint(1, 8), rng.randint(1, 64), Hkv, D, P, rng.randint(0, hi), hi, rng.randint(1, 36))
        if c["op"] in ("commit", "fork", "append"):
            if c["L"] * _pages(c) * _page_bytes(c) > 6e9:
                continue
        if _cost(c) <= most:
            return c


# ---------------------------------------------------------------------------------------------------------- sizes

def _lengths(case):
    """Committed tokens of every request: lo .. hi, unevenly spread, the first one the longest."""
    lo, hi, B = case["lo"], case["hi"], case["B"]
    return [hi - int((hi - lo) * ((0.618034 * b) % 1.0)) for b in range(B)]


def _new(case):
    """Tokens that come behind them."""
    N, B = case["N"], case["B"]
    if not case.get("ragged"):
        return [N] * B
    return [max(1, N - int(N * 0.9 * ((0.382 * b) % 1.0))) for b in range(B)]


def _width(case):
    return -(-(case["hi"] + case["N"]) // case["P"])


def _blk(case):
    """Bytes of a head in a page."""
    return case["P"] * (case["D"] + case["D"] // 16)


def _page_bytes(case):
    return case["Hkv"] * _blk(case)


def _held(case):
    P = case["P"]
    if case["op"] == "fork":      # what is committed; the children get their room in the pass
        return [-(-n // P) for n in _lengths(case)]
    return [-(-(n + m) // P) for n, m in zip(_lengths(case), _new(case))]


def _pages(case):
    pages = sum(_held(case))
    if case["op"] == "fork":
        pages += case["B"] * (case["children"] + 1) * (2 + case["N"] // case["P"]) + 5
    return pages + 3


def _accepted(case):
    """Accepted drafts of every request: none to seven."""
    return [min(case["N"] - 1, (5 * b + 3) % 8) for b in range(case["B"])]


def work(case):
    B, N, Hkv, D, P, L = (case[k] for k in ("B", "N", "Hkv", "D", "P", "L"))
    record = D + D // 16                               # bytes of a token and head, keys and values
    lens = _lengths(case)
    if case["op"] == "attention":
        elt = 2 if case["dtype"] == "bf16" else 4
        seen = sum(N * n + (N * (N + 1) // 2 if not case["tree"] else N) for n in lens)      # (a tree's node: itself at least)
        rows = B * N * case["Hq"]
        return {"bytes": sum(n + N for n in lens) * Hkv * record + rows * (2 * D * elt + 4), "flops": 4 * D * case["Hq"] * seen}
    if case["op"] == "append":
        elt = 2 if case["dtype"] == "bf16" else 4
        new = sum(_new(case)) * Hkv                    # rows in, codes out, and read back
        return {"bytes": new * (2 * D * elt + 2 * record) + B * N * Hkv * 2 * D * elt, "flops": 0}
    if case["op"] == "commit":
        return {"bytes": sum(_accepted(case)) * 2 * record * Hkv * L + 8 * B * N, "flops": 0}
    copied = sum(case["children"] for n in lens if n % P)      # a child whose last page is shared gets one of its own
    return {"bytes": copied * 2 * _page_bytes(case) * L + 4 * _pages(case) + 4 * sum(_held(case)) * (1 + case["children"]), "flops": 0}


# ------------------------------------------------------------------------------------------------ 4 bits, plainly

def _quantised(x):
    """Codes [..., D] (0 .. 15) and scales' bytes [..., D/32] of values [..., D]."""
    x = x.float().unflatten(-1, (-1, 32))
    top = x.abs().amax(-1)
    # 2^e with the largest value at most 7 of them (and over 3.5): no value is further off than half a step
    byte = (((top.view(torch.int32) + 0x200000) >> 23) - 2).clamp(1, 252)
    y = x * ((254 - byte) << 23).view(torch.float32)[..., None]
    a = y.abs()
    code = ((a > 0.25).int() + (a >= 0.75).int() + (a > 1.25).int() + (a >= 1.75).int() + (a > 2.5).int() + (a >= 3.5).int()
            + (a > 5.0).int())                         # to the nearest, ties to the even code
    code = torch.where(torch.signbit(y), code + 8, code).flatten(-2)
    return code.to(torch.uint8), byte.to(torch.uint8)


def _values(code, byte):
    """What codes [..., D] and scales [..., D/32] stand for, in 32 bits."""
    m = (code & 7).int()
    a = torch.where(m < 2, 0.5 * m, (((m >> 1) + 126 << 23) | ((m & 1) << 22)).view(torch.float32))
    a = torch.where(code >= 8, -a, a).unflatten(-1, (-1, 32))
    return (a * (byte.int() << 23).view(torch.float32)[..., None]).flatten(-2)


def _packed(code):
    return code[..., 0::2] | (code[..., 1::2] << 4)


def _unpacked(byte):
    return torch.stack((byte & 15, byte >> 4), -1).flatten(-2)


def _record_places(P, D, device):
    """Where in a head's part of a page the bytes of a token lie: [P, D + D/16] (codes of key and value, scales of both)."""
    t = torch.arange(P, device=device)[:, None]
    i, s = torch.arange(D // 2, device=device)[None], torch.arange(D // 32, device=device)[None]
    at_k = t * (D // 2) + i
    at_v = P * (D // 2) + ((t // 8) * (D // 8) + i // 4) * 32 + (t % 8) * 4 + i % 4
    scale_k = P * D + t * (D // 32) + s
    scale_v = P * D + P * (D // 32) + ((t // 8) * (D // 32) + s) * 8 + t % 8
    return torch.cat((at_k, at_v, scale_k, scale_v), 1)


def _token_places(table, position, P, D, Hkv, pages, layer):
    """Places in the pool of the bytes of tokens at position [B, n] of sequences with page table rows [B, W]: [B, n, Hkv, D + D/16]."""
    blk = P * (D + D // 16)
    page = table.long().gather(1, (position // P).clamp(max=table.shape[1] - 1))
    first = ((layer * pages + page)[..., None] * Hkv + torch.arange(Hkv, device=table.device)) * blk
    return first[..., None] + _record_places(P, D, table.device)[position % P][:, :, None, :]


def _halves(record, D):
    """Values of key and value from a token's bytes [..., D + D/16]."""
    k, v, sk, sv = record.split((D // 2, D // 2, D // 32, D // 32), -1)
    return _values(_unpacked(k), sk), _values(_unpacked(v), sv)


def _heads_pages(s, layer):
    """Keys and values [B, Hkv, T, D] of the whole page table of a layer."""
    P, D, Hkv = s["P"], s["D"], s["Hkv"]
    part = s["pool"][layer][s["page_table"].clamp(min=0).long()]              # [B, W, Hkv, blk]
    B, W = part.shape[:2]
    k, v, sk, sv = part.split((P * D // 2, P * D // 2, P * (D // 32), P * (D // 32)), -1)
    k = _values(_unpacked(k.unflatten(-1, (P, D // 2))), sk.unflatten(-1, (P, D // 32)))
    v = v.unflatten(-1, (P // 8, D // 8, 8, 4)).transpose(-3, -2).reshape(B, W, Hkv, P, D // 2)
    sv = sv.unflatten(-1, (P // 8, D // 32, 8)).transpose(-2, -1).reshape(B, W, Hkv, P, D // 32)
    v = _values(_unpacked(v), sv)
    return [x.transpose(1, 2).reshape(B, Hkv, W * P, D) for x in (k, v)]


# -------------------------------------------------------------------------------------------------------- inputs

def _fill_pages(pool, P, D, g):
    """Pages of one layer [pages, Hkv, blk] filled as a model would: some channels of the keys are far larger than the others."""
    loud = 1.0 + 3.0 * (torch.arange(D, device=pool.device) % 16 == 5)
    for part in pool.split(max(1, (1 << 27) // (pool.shape[1] * P * D))):
        shape = (*part.shape[:2], P, D)
        k, sk = _quantised(torch.randn(shape, device=pool.device, generator=g) * loud)
        v, sv = _quantised(torch.randn(shape, device=pool.device, generator=g))
        v = _packed(v).unflatten(-1, (D // 8, 4)).unflatten(2, (P // 8, 8)).transpose(-3, -2)
        sv = sv.unflatten(2, (P // 8, 8)).transpose(-2, -1)
        part.copy_(torch.cat([x.flatten(2) for x in (_packed(k), v, sk, sv)], -1))


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(dev).manual_seed(seed)
    B, N, Hkv, D, P, L = (case[k] for k in ("B", "N", "Hkv", "D", "P", "L"))
    pages, W = _pages(case), _width(case)
    lens, held = _lengths(case), _held(case)
    s = dict(case, layer=L - 1)
    slots = B * (1 + case.get("children", 0))
    s["lens"] = torch.zeros(slots, dtype=torch.int32, device=dev)
    s["lens"][:B] = torch.tensor(lens, dtype=torch.int32)
    s["held"] = torch.zeros(slots, dtype=torch.int32, device=dev)
    s["held"][:B] = torch.tensor(held, dtype=torch.int32)
    # pages in no particular order, as they are after some hours
    order = torch.randperm(pages, device=dev, generator=g).int()
    width = torch.arange(W, device=dev)[None]
    mine = width < s["held"][:, None]
    rank = (torch.cumsum(s["held"], 0) - s["held"])[:, None] + width
    s["page_table"] = torch.where(mine, order[rank.clamp(max=pages - 1)], -1).int().contiguous()
    s["refs"] = torch.zeros(pages, dtype=torch.int32, device=dev)
    s["refs"][s["page_table"][mine].long()] = 1
    s["pool"] = torch.empty((L, pages, Hkv, _blk(case)), dtype=torch.uint8, device=dev)
    if case["op"] == "attention":
        _fill_pages(s["pool"][s["layer"]], P, D, g)
        dtype = TYPES[case["dtype"]]
        s["q"] = torch.randn((B, N, case["Hq"], D), device=dev, generator=g).to(dtype)
        s["out"], s["lse"] = torch.empty_like(s["q"]), torch.empty((B, N, case["Hq"]), device=dev)
        if case["tree"]:
            u = torch.rand((B, N), device=dev, generator=g)
            node = torch.arange(N, device=dev)
            s["tree_parent"] = torch.minimum((u * node).int(), (node - 1).int()).int()      # the root's is -1
            s["mask"] = torch.zeros((B, N, (N + 63) // 64), dtype=torch.int64, device=dev)
    else:
        s["pool"].random_(generator=g)                   # (what the pages hold does not matter to who moves them)
    if case["op"] == "append":
        _fill_pages(s["pool"][0], P, D, g)
        dtype = TYPES[case["dtype"]]
        # (a slice of the projection's output: queries, keys and values of a token lie beside each other)
        loud = 1.0 + 3.0 * (torch.arange(D, device=dev) % 16 == 5)
        qkv = torch.empty((B, N, 4 * Hkv, D), dtype=dtype, device=dev)
        for b in range(B):
            qkv[b] = torch.randn((N, 4 * Hkv, D), device=dev, generator=g) * loud
        s["k"], s["v"] = qkv[:, :, 2 * Hkv:3 * Hkv], qkv[:, :, 3 * Hkv:]
        s["n_new"] = torch.tensor(_new(case), dtype=torch.int32, device=dev)
        s["read_k"], s["read_v"] = (torch.empty((B, N, Hkv, D), dtype=dtype, device=dev) for _ in range(2))
    if case["op"] == "commit":
        s["accept_len"] = torch.tensor(_accepted(case), dtype=torch.int32, device=dev)
        most = max(_accepted(case))
        nodes = torch.rand((B, N - 1), device=dev, generator=g).topk(most, dim=1).indices if N > 1 else torch.zeros((B, 0), device=dev)
        depth = torch.arange(most, device=dev)[None]
        taken = depth < s["accept_len"][:, None]
        nodes = torch.where(taken, nodes + 1, N + depth).sort(1).values
        s["path_idx"] = torch.full((B, N), -1, dtype=torch.int32, device=dev)
        s["path_idx"][:, :most] = torch.where(taken, nodes, -1).int()
        s["new_lens"] = torch.empty_like(s["lens"])
    if case["op"] == "fork":
        child = torch.arange(B * case["children"], dtype=torch.int32, device=dev)
        s["dst"] = child + B
        s["src"] = (child // case["children"]).int()
        s["every"] = torch.cat((torch.arange(B, dtype=torch.int32, device=dev), s["dst"]))
        s["status"] = torch.empty(slots, dtype=torch.int32, device=dev)
    return s


# ------------------------------------------------------------------------------------------------------- one pass

def _ancestors(parent):
    """[B, N, N]: whether node i is node j or one of its descendants."""
    N = parent.shape[1]
    node = torch.arange(N, device=parent.device)
    up = (parent[..., None] == node).float() + torch.eye(N, device=parent.device)
    return torch.linalg.matrix_power(up, N) > 0


def _plain_attention(s):
    q, B, N, Hkv, D = s["q"], s["B"], s["N"], s["Hkv"], s["D"]
    k, v = _heads_pages(s, s["layer"])
    T = k.shape[2]
    dev = q.device
    at, node = torch.arange(T, device=dev), torch.arange(N, device=dev)
    own_place = (at[None] - s["lens"][:, None].long())                        # [B, T]: which node, < 0 committed
    inside = (own_place >= 0) & (own_place < N)
    if s["tree"]:
        sees = _ancestors(s["tree_parent"])
        bit = torch.ones((), dtype=torch.int64, device=dev) << node
        mask = torch.where(sees, bit, 0).sum(-1, keepdim=True) if N <= 64 else None
        sees = sees.gather(2, own_place.clamp(0, N - 1)[:, None].expand(B, N, T))
    else:
        sees = own_place[:, None] <= node[None, :, None]
        mask = None
    sees = (own_place < 0)[:, None] | (sees & inside[:, None])                 # [B, N, T]
    group = s["Hq"] // Hkv
    x = q.float().unflatten(2, (Hkv, group)).permute(0, 2, 1, 3, 4).reshape(B, Hkv, N * group, D)
    scores = (x @ k.transpose(2, 3)) * (1.0 / math.sqrt(D))
    del k
    # (written over: the scores are the largest thing here)
    scores.view(B, Hkv, N, group, T).masked_fill_(~sees[:, None, :, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    scores.sub_(torch.where(top == -math.inf, 0, top)).exp_()
    total = scores.sum(-1, keepdim=True)
    out = torch.where(total > 0, (scores @ v) / total, 0)
    lse = (top + torch.log(total)).squeeze(-1)
    out = out.unflatten(2, (N, group)).permute(0, 2, 1, 3, 4).reshape(q.shape).to(q.dtype)
    lse = lse.unflatten(2, (N, group)).permute(0, 2, 1, 3).reshape(B, N, s["Hq"])
    return (out, lse) if mask is None else (out, lse, mask)


def _plain_append(s):
    P, D, Hkv, B, N = s["P"], s["D"], s["Hkv"], s["B"], s["N"]
    pages = s["pool"].shape[1]
    (ck, bk), (cv, bv) = _quantised(s["k"]), _quantised(s["v"])
    record = torch.cat((_packed(ck), _packed(cv), bk, bv), -1)
    node = torch.arange(N, device=ck.device)[None]
    position = s["lens"][:, None].long() + node
    places = _token_places(s["page_table"], position, P, D, Hkv, pages, s["layer"])
    flat = s["pool"].view(-1)
    there = (node < s["n_new"][:, None])
    flat[places[there]] = record[there]
    # read back; what lies beyond a sequence's pages is zero
    k, v = _halves(flat[places], D)
    room = (position < (s["held"][:, None] * P))[:, :, None, None]
    return torch.where(room, k, 0).to(s["k"].dtype), torch.where(room, v, 0).to(s["v"].dtype)


def _plain_commit(s):
    P, D, Hkv, B, N, L = s["P"], s["D"], s["Hkv"], s["B"], s["N"], s["L"]
    pages = s["pool"].shape[1]
    most = max(1, min(N - 1, 7))
    depth = torch.arange(most, device=s["lens"].device)[None]
    path = s["path_idx"][:, :most].long()
    moves = depth < s["accept_len"][:, None]
    first = s["lens"][:, None].long()
    source = _token_places(s["page_table"], first + torch.where(moves, path, 0), P, D, Hkv, pages, 0)
    target = _token_places(s["page_table"], first + 1 + torch.where(moves, depth, 0), P, D, Hkv, pages, 0)
    layers = s["pool"].view(L, -1)
    layers[:, target[moves]] = layers[:, source[moves]]
    torch.add(s["lens"], s["accept_len"] + 1, out=s["new_lens"])
    return s["pool"], s["new_lens"]


def _plain_fork(s):
    P, W = s["P"], s["page_table"].shape[1]
    table, lens, held, refs, src, dst, every = (s[k] for k in ("page_table", "lens", "held", "refs", "src", "dst", "every"))
    at = torch.arange(W, device=table.device)[None]
    lose, keep = dst.long(), src.long()
    # the children give back what they hold
    gone = table[lose]
    refs.index_add_(0, gone[gone >= 0].long(), torch.full_like(gone[gone >= 0], -1))
    # and share their parents' committed pages
    shared = -(-lens[keep] // P)
    row = torch.where(at < shared[:, None], table[keep], -1)
    refs.index_add_(0, row[row >= 0].long(), torch.ones_like(row[row >= 0]))
    table[lose], lens[lose], held[lose] = row, lens[keep], shared
    # room for the step: a shared page that would be written is replaced by a copy, in all but the last of its holders where nobody else holds it
    n, have = lens[every.long()], held[every.long()]
    need = -(-(n + s["N"]) // P)
    last = table[every.long()].gather(1, (n // P).clamp(max=W - 1).long()[:, None])[:, 0]
    writes = (n % P != 0) & (n // P < have)
    held_by = torch.where(writes, refs[last.clamp(min=0).long()], 0)
    same = (last[:, None] == last[None]) & writes[:, None] & writes[None]
    later = torch.triu(same, 1).sum(1)
    others = held_by - same.sum(1)                       # holders that do not write now
    copies = writes & (held_by > 1) & ((later > 0) | (others > 0))
    wants = (need - have).clamp(min=0) + copies.int()
    begin = torch.cumsum(wants, 0) - wants
    free = torch.nonzero(refs == 0)[:, 0].int()          # the lowest first
    fits = begin + wants <= free.numel()
    fresh = torch.where(copies, free[begin.clamp(max=free.numel() - 1)], last)
    rows = table[every.long()]
    k = at - have[:, None]
    new = free[(begin[:, None] + copies[:, None] + k).clamp(0, free.numel() - 1)]
    rows = torch.where((k >= 0) & (at < need[:, None]), new, rows)
    rows = torch.where((at == (n // P)[:, None]) & copies[:, None], fresh[:, None], rows)
    pool = s["pool"]
    pool[:, fresh[copies].long()] = pool[:, last[copies].long()]
    refs.index_add_(0, last[copies].long(), torch.full_like(last[copies], -1))
    refs[free[: int(wants.sum())].long()] = 1
    table[every.long()], held[every.long()] = rows, torch.maximum(have, need)
    s["status"].copy_(torch.where(fits, 0, 1))
    return pool, table, lens, held, refs, s["status"]


def run(s):
    if not own:
        return {"attention": _plain_attention, "append": _plain_append, "commit": _plain_commit, "fork": _plain_fork}[s["op"]](s)
    from paper_2601_15498_amd import cache
    pool, table, lens = s["pool"], s["page_table"], s["lens"]
    if s["op"] == "attention":
        if "workspace" not in s:                         # kept from step to step, as a serving loop does
            s["workspace"] = cache.alloc_attention_workspace(pool, table, s["q"])
        if not s["tree"]:
            return cache.mars_kv_attention(pool, table, lens, s["q"], layer=s["layer"], max_len=s["hi"], out=s["out"], lse=s["lse"],
                                           workspace=s["workspace"])
        mask = cache.mars_tree_mask(s["tree_parent"], mask=s["mask"])
        out, lse = cache.mars_kv_attention(pool, table, lens, s["q"], layer=s["layer"], mask=mask, max_len=s["hi"], out=s["out"],
                                           lse=s["lse"], workspace=s["workspace"])
        return out, lse, mask
    if s["op"] == "append":
        cache.mars_kv_append(pool, table, lens, s["k"], s["v"], layer=s["layer"], n_new=s["n_new"])
        return cache.mars_kv_read(pool, table, s["held"], first=lens, layer=s["layer"], out=(s["read_k"], s["read_v"]))
    if s["op"] == "commit":
        cache.mars_kv_commit(pool, table, lens, s["accept_len"], s["path_idx"], page_size=s["P"], new_lens=s["new_lens"])
        return pool, s["new_lens"]
    if "workspace" not in s:
        s["workspace"] = cache.alloc_reserve_workspace(pool, s["every"].numel())
    cache.mars_kv_release(table, lens, s["held"], s["refs"], s["dst"])
    cache.mars_kv_fork(table, lens, s["held"], s["refs"], s["src"], s["dst"], page_size=s["P"])
    cache.mars_kv_reserve(pool, table, lens, s["held"], s["refs"], s["N"], seqs=s["every"], page_size=s["P"], status=s["status"],
                          workspace=s["workspace"])
    return pool, table, lens, s["held"], s["refs"], s["status"]


# ------------------------------------------------------------------------------------------- in 64 bits, once more

_GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _grid(device):
    return torch.tensor(_GRID + tuple(-x for x in _GRID), dtype=torch.float64, device=device)


def _exact_rounded(x):
    """The values a row of the cache would hold for x [..., D], from the definition: the nearest multiples, ties to the even code."""
    x = x.double().unflatten(-1, (-1, 32))
    top = x.abs().amax(-1, keepdim=True)
    exponent = torch.floor(torch.log2(top.clamp(min=2.0 ** -149))) - 2
    exponent = exponent + (top >= 7 * torch.exp2(exponent)).double() - (top < 3.5 * torch.exp2(exponent)).double()
    step = torch.exp2(exponent.clamp(-126, 125))
    places = torch.tensor(_GRID, dtype=torch.float64, device=x.device)
    a = (x.abs() / step).clamp(max=6.0)
    best, best_off = torch.zeros_like(a), a.clone()
    for code in (2, 4, 6, 1, 3, 5, 7):                   # the even ones first: an odd one has to be nearer
        off = (a - places[code]).abs()
        nearer = off < best_off
        best, best_off = torch.where(nearer, places[code], best), torch.where(nearer, off, best_off)
    return (best * step * torch.sign(x)).flatten(-2)


def _exact_sequence(s, b, T):
    """Keys and values [Hkv, T, D] of request b, byte by byte."""
    P, D, Hkv = s["P"], s["D"], s["Hkv"]
    dev = s["pool"].device
    t = torch.arange(T, device=dev)
    head = s["pool"][s["layer"]][s["page_table"][b].clamp(min=0).long()[t // P]]      # [T, Hkv, blk]
    t = t % P
    d = torch.arange(D, device=dev)
    grid = _grid(dev)

    def part(code_at, scale_at):
        byte = head.gather(2, code_at[:, None].expand(T, Hkv, D)).int()
        code = torch.where(d % 2 == 1, byte >> 4, byte & 15)
        scale = head.gather(2, scale_at[:, None].expand(T, Hkv, D)).double()
        return (grid[code.long()] * torch.exp2(scale - 127)).transpose(0, 1)

    k = part(t[:, None] * (D // 2) + d // 2, P * D + t[:, None] * (D // 32) + d // 32)
    v = part(P * D // 2 + (t[:, None] // 8) * 4 * D + (d // 8) * 32 + (t[:, None] % 8) * 4 + (d % 8) // 2,
             P * D + P * D // 32 + (t[:, None] // 8) * (D // 4) + (d // 32) * 8 + t[:, None] % 8)
    return k, v


def exact(case, seed):
    if case["op"] in ("commit", "fork"):
        return None                                      # bytes and whole numbers: they are moved, not computed
    s = prepare(case, seed)
    if case["op"] == "append":
        both = [torch.zeros(s["k"].shape, dtype=torch.float64, device="cuda") for _ in range(2)]
        for b, (n, new, held) in enumerate(zip(_lengths(case), _new(case), _held(case))):
            room = held * case["P"]
            for x, fresh, before in zip(both, (s["k"], s["v"]), _exact_sequence(s, b, room)):
                got = min(case["N"], room - n)            # (behind a short request's last token: what the pages held before)
                x[b, :got] = before.transpose(0, 1)[n:n + got]
                x[b, :new] = _exact_rounded(fresh[b, :new])
        return both
    B, N, Hq, Hkv, D = (case[k] for k in ("B", "N", "Hq", "Hkv", "D"))
    out, lse = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda"), torch.empty((B, N, Hq), dtype=torch.float64, device="cuda")
    lens = _lengths(case)
    for b in range(B):
        n = lens[b]
        sees = torch.zeros((N, n + N), dtype=torch.bool, device="cuda")
        sees[:, :n] = True
        if case["tree"]:
            parent = s["tree_parent"][b].tolist()
            for i in range(N):
                j = i
                while j >= 0:
                    sees[i, n + j] = True
                    j = parent[j]
        else:
            sees[:, n:] = torch.ones((N, N), dtype=torch.bool, device="cuda").tril()
        k, v = _exact_sequence(s, b, n + N)
        for h in range(Hq):
            z = s["q"][b, :, h].double() @ k[h * Hkv // Hq].T / math.sqrt(D)
            z = z.masked_fill(~sees, -math.inf)
            lse[b, :, h] = torch.logsumexp(z, 1)
            out[b, :, h] = torch.softmax(z, 1) @ v[h * Hkv // Hq]
    return (out, lse) if not case["tree"] else (out, lse, None)
