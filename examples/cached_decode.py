"""Speculative decoding of a small random model over the paged 4-bit cache: prompts into the cache, drafted trees attended and verified, accepted paths
committed, one request branched into two.

    python examples/cached_decode.py

The model is a few layers of random weights (projections are plain torch products); the "draft model" is told what the target will say and errs on
purpose, so that paths of all lengths are accepted.  With strict verification every committed token is the target's own choice, whatever is
drafted: at the end the whole text is scored once more as a prompt.  (Where the two largest logits are a rounding apart that choice can differ between
two ways of computing it, so the texts of two runs need not be the same to the end.)
"""
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2601_15498_amd import binding as mars  # noqa: E402
from paper_2601_15498_amd import cache as kv  # noqa: E402

LAYERS, HIDDEN, HEADS, KV_HEADS, HEAD_DIM, VOCAB, PAGE = 3, 512, 8, 2, 128, 2000, 16
STRICT = 2.0   # a logit ratio is never above 1: nothing is relaxed


class Model:
    """Weights, and what a step keeps beside them."""

    def __init__(self, seed=0, device="cuda"):
        g = torch.Generator(device).manual_seed(seed)
        w = lambda *shape, scale=1.0: (torch.randn(shape, device=device, generator=g) * scale / shape[-1] ** 0.5).bfloat16()  # noqa: E731
        self.embed = w(VOCAB, HIDDEN, scale=HIDDEN ** 0.5)
        self.qkv = [w((HEADS + 2 * KV_HEADS) * HEAD_DIM, HIDDEN) for _ in range(LAYERS)]
        self.out = [w(HIDDEN, HEADS * HEAD_DIM, scale=2.0) for _ in range(LAYERS)]
        self.head = w(VOCAB, HIDDEN, scale=3.0)

    def hidden(self, c, tokens, seqs, mask=None):
        """Last hidden states [B, N, HIDDEN] of `tokens` behind what sequences `seqs` have committed; their rows go into the cache."""
        B, N = tokens.shape
        x = self.embed[tokens.long()]
        a = work = None                                  # (one of each for all layers: calls that are given both go through the binding's native part)
        for layer in range(LAYERS):
            rows = (x @ self.qkv[layer].T).view(B, N, HEADS + 2 * KV_HEADS, HEAD_DIM)
            q, k, v = rows.split((HEADS, KV_HEADS, KV_HEADS), 2)
            kv.mars_kv_append(c.pool, c.page_table, c.lens, k, v, layer=layer, seqs=seqs)
            if work is None:
                a, work = torch.empty(q.shape, dtype=q.dtype, device=q.device), kv.alloc_attention_workspace(c.pool, c.page_table, q)
            kv.mars_kv_attention(c.pool, c.page_table, c.lens, q, layer=layer, seqs=seqs, mask=mask, out=a, workspace=work)
            x = x + a.reshape(B, N, -1) @ self.out[layer].T
            x = x * torch.rsqrt(x.float().square().mean(-1, keepdim=True)).bfloat16()
        return x


def room(c, n, seqs):
    status = kv.mars_kv_reserve(c.pool, c.page_table, c.lens, c.held, c.refs, n, page_size=PAGE, seqs=seqs)
    if bool((status != kv.MARS_KV_OK).any()):
        raise RuntimeError(f"no room: {status.tolist()}")


def prefill(model, c, prompts, seqs):
    """Prompts [B, N] into empty sequences; returns the token after each."""
    room(c, prompts.shape[1], seqs)
    h = model.hidden(c, prompts, seqs)
    c.lens[seqs.long()] += prompts.shape[1]
    return (h[:, -1].float() @ model.head.float().T).argmax(-1).int()


def step(model, c, roots, drafts, parents, seqs, theta=STRICT):
    """One step: node 0 of every request is its last token (not in the cache yet), `drafts` [B, N] with parents [B, N] hang below it.
    Returns the verification's outputs; the cache holds the accepted path."""
    B, N = drafts.shape
    tokens = drafts.clone()
    tokens[:, 0] = roots
    room(c, N, seqs)
    h = model.hidden(c, tokens, seqs, kv.mars_tree_mask(parents))
    out = mars.mars_lmhead_verify(h, model.head, tokens, parents, torch.full((B,), theta, device=h.device), want_commit=True)
    kv.mars_kv_commit(c.pool, c.page_table, c.lens, out.accept_len, out.path_idx, page_size=PAGE, seqs=seqs)
    return out


def one_by_one(model, prompts, count):
    """[B, count] tokens, each with a step of its own."""
    B = prompts.shape[0]
    c = kv.KVCache(LAYERS, 64 * B, KV_HEADS, HEAD_DIM, PAGE, B, 512)
    seqs = torch.arange(B, dtype=torch.int32, device="cuda")
    roots = prefill(model, c, prompts, seqs)
    parents = torch.full((B, 1), -1, dtype=torch.int32, device="cuda")
    got = [roots]
    while len(got) < count:
        got.append(step(model, c, got[-1], got[-1][:, None], parents, seqs).bonus_token)
    return torch.stack(got, 1)


def drafted(will, at, n_chain, wrong, g):
    """A tree per request: a chain of what the target will say from position at[b] on, wrong from depth `wrong[b]`, and beside every node of it another child."""
    B = will.shape[0]
    N = 1 + 2 * n_chain
    tokens = torch.randint(0, VOCAB, (B, N), generator=g, dtype=torch.int32)
    parents = torch.empty((B, N), dtype=torch.int32)
    parents[:, 0] = -1
    for d in range(n_chain):
        decoy, node = 1 + 2 * d, 2 + 2 * d           # (the decoy comes first: accepted rows have to move)
        parents[:, decoy] = parents[:, node] = 0 if d == 0 else node - 2
        for b in range(B):
            if d < wrong[b] and at[b] + d < will.shape[1]:
                tokens[b, node] = will[b, at[b] + d]
    return tokens.cuda(), parents.cuda()


def shortfalls(model, prompts, got):
    """For every committed token: how far its logit is below the largest, when the whole text goes through the model as a prompt."""
    requests, n = prompts.shape
    short = []
    for b, tokens in enumerate(got):
        text = torch.cat((prompts[b if b < requests else 0], torch.tensor(tokens[:-1], dtype=torch.int32, device="cuda")))[None]
        c = kv.KVCache(LAYERS, 64, KV_HEADS, HEAD_DIM, PAGE, 1, 512)
        seqs = torch.zeros(1, dtype=torch.int32, device="cuda")
        room(c, text.shape[1], seqs)
        logits = model.hidden(c, text, seqs)[0, n - 1:].float() @ model.head.float().T
        own = logits.gather(1, torch.tensor(tokens, device="cuda")[:, None])[:, 0]
        short.append((logits.amax(1) - own).tolist())
    return short


def main(requests=3, count=40, seed=0, say=print):
    g = torch.Generator().manual_seed(seed)
    model = Model(seed)
    prompts = torch.randint(0, VOCAB, (requests, 37), generator=g, dtype=torch.int32).cuda()
    will = one_by_one(model, prompts, count + 10).cpu()

    slots = requests + 1
    c = kv.KVCache(LAYERS, 64 * slots, KV_HEADS, HEAD_DIM, PAGE, slots, 512)
    seqs = torch.arange(requests, dtype=torch.int32, device="cuda")
    roots = prefill(model, c, prompts, seqs)
    # request 0 is sampled twice: its copy shares the prompt's pages until one of them writes
    kv.mars_kv_fork(c.page_table, c.lens, c.held, c.refs, seqs[:1], torch.tensor([requests], dtype=torch.int32, device="cuda"), page_size=PAGE)
    seqs = torch.arange(slots, dtype=torch.int32, device="cuda")
    roots, will = torch.cat((roots, roots[:1])), torch.cat((will, will[:1]))
    got = [[int(r)] for r in roots]
    taken = []
    while min(len(x) for x in got) < count:
        at = [len(x) for x in got]
        wrong = torch.randint(0, 6, (slots,), generator=g).tolist()
        tokens, parents = drafted(will, at, 5, wrong, g)
        out = step(model, c, roots, tokens, parents, seqs)
        roots = out.bonus_token
        for b, (new, n) in enumerate(zip(out.out_tokens.tolist(), out.out_len.tolist())):
            got[b] += new[:n]
            taken.append(n)
    short = shortfalls(model, prompts, got)
    for b in range(slots):
        same = next((i for i, (x, y) in enumerate(zip(got[b], will[b].tolist())) if x != y), len(got[b]))
        say(f"sequence {b}: {len(got[b])} tokens, the first {same} those of decoding one at a time; scored again as a prompt, "
            f"none is more than {max(short[b]):.3f} below the largest logit")
    say(f"{sum(taken) / len(taken):.2f} tokens per step and sequence; pages held: {int(c.held.sum())}, of which shared: {int((c.refs > 1).sum())}")
    kv.mars_kv_release(c.page_table, c.lens, c.held, c.refs, seqs)
    say(f"pages in use at the end: {int((c.refs != 0).sum())}")
    return got, short, c


if __name__ == "__main__":
    main()
