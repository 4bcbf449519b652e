"""A worker answering a batch of queries: the executor's calls as they follow each other.

    python examples/answer_queries.py [--queries 6] [--tokens 16]

The queries of one application have its prompt in front of them, which is in the cache once.  A small decoder with random
weights stands for the variant; everything but its products is the executor's: each layer appends the step's keys and
values to its cache (rotated on the way) and attends over it, and behind the last layer a token of every query is drawn.
The first step reads the prompts, the steps after it take a token of each query.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1905_13348_amd import Executor  # noqa: E402


class Variant:
    """A decoder's sizes and weights, on the device."""

    def __init__(self, layers=2, heads=8, kv_heads=2, head_dim=64, hidden=256, vocab=5_000, seed=0):
        g = torch.Generator().manual_seed(seed)
        w = lambda *shape: (torch.randn(shape, generator=g) * shape[0] ** -0.5).bfloat16().cuda()
        self.layers, self.heads, self.kv_heads, self.head_dim, self.hidden, self.vocab = layers, heads, kv_heads, head_dim, hidden, vocab
        self.embed = torch.randn((vocab, hidden), generator=g).bfloat16().cuda()
        self.qkv = [w(hidden, (heads + 2 * kv_heads) * head_dim) for _ in range(layers)]
        self.proj = [w(heads * head_dim, hidden) for _ in range(layers)]
        self.up = [w(hidden, 4 * hidden) for _ in range(layers)]
        self.down = [w(4 * hidden, hidden) for _ in range(layers)]
        self.head = w(hidden, vocab) * 4
        self.freq = 10000.0 ** (-torch.arange(head_dim // 2, dtype=torch.float64) / (head_dim // 2)).cuda()


def norm(x):
    y = x.float()
    return (y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype)


def answer(variant, prompt, queries, tokens, temperature=0.8, top_k=50, top_p=0.95, seed=0, page=16):
    """prompt: token numbers that all queries share; queries: token numbers of each (one at least).  Returns the tokens
    drawn, [queries, tokens], and the logits they were drawn from, [tokens, queries, vocab]."""
    v, S, shared = variant, len(queries), len(prompt)
    i32 = lambda a: torch.as_tensor(a, dtype=torch.int32).cuda()
    ex = Executor()

    # pages: whole pages of the prompt belong to the first query's row of the table and to all others'
    own = [len(q) + tokens for q in queries]
    whole = shared // page
    width = -(-(shared + max(own)) // page)
    table, at = torch.zeros((S, width), dtype=torch.int32), whole
    for s in range(S):
        need = -(-(shared + own[s]) // page) - whole
        table[s, :whole] = torch.arange(whole)
        table[s, whole:whole + need] = torch.arange(at, at + need)
        at += need
    pools = [[torch.zeros((at, page, v.kv_heads, v.head_dim), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
             for _ in range(v.layers)]
    caches = [ex.cache(k, w) for k, w in pools]
    table = table.cuda()

    def batch_of(new, start, length, pos, group):
        """`new` tokens of every sequence, whose keys end at `length`."""
        seq = [s for s, n in enumerate(new) for _ in range(n)]
        groups = dict(group_start=i32([0, S]), shared_len=i32([group])) if group else {}
        b = ex.batch(caches[0], v.heads, token_seq=i32(seq), token_pos=pos, seq_start=i32(start), seq_len=length, page_table=table,
                     max_len=shared + max(own), **groups)
        ex.reserve(caches[0], b)
        return b

    def step(x, batch):
        """Hidden states of the batch's tokens, through all layers."""
        ex.plan(batch)
        n = x.shape[0]
        out = torch.empty((n, v.heads, v.head_dim), dtype=x.dtype, device="cuda")
        for i, cache in enumerate(caches):
            qkv = (norm(x) @ v.qkv[i]).view(n, v.heads + 2 * v.kv_heads, v.head_dim)
            q, k, w = qkv.split([v.heads, v.kv_heads, v.kv_heads], dim=1)
            ex.append(cache, batch, q, k, w, q, v.freq)      # (queries in place)
            ex.attend(cache, batch, q, out)
            x = x + out.flatten(1) @ v.proj[i]
            x = x + torch.relu(norm(x) @ v.up[i]) @ v.down[i]
        return x

    # The prompt is read by the first query alone: its whole pages are then there for all, and what it has on the page where it
    # ends, and beyond, the others read for themselves.
    done = whole * page
    if done:
        step(v.embed[i32(prompt[:done]).long()], batch_of([done] + [0] * (S - 1), [0] + [done] * S, i32([done] + [0] * (S - 1)),
                                                          i32(range(done)), 0))
    rest = [list(prompt[done:]) + list(q) for q in queries]
    new = [len(r) for r in rest]
    start = [sum(new[:s]) for s in range(S + 1)]
    pos = i32([done + j for n in new for j in range(n)])
    x = step(v.embed[i32(sum(rest, [])).long()], batch_of(new, start, i32([done + n for n in new]), pos, done))
    x = x[torch.tensor(start[1:], device="cuda") - 1]

    # a token of every query at a time; positions and lengths move on the device
    pos, length = i32([done + n - 1 for n in new]), i32([done + n for n in new])
    batch = batch_of([1] * S, list(range(S + 1)), length, pos, done)
    draws = torch.rand((tokens, S), generator=torch.Generator().manual_seed(seed)).clamp_max(1 - 2.0 ** -24).cuda()
    full = lambda value, dtype: torch.full((S,), value, dtype=dtype, device="cuda")
    limits = dict(temperature=full(temperature, torch.float32), top_k=full(top_k, torch.int32), top_p=full(top_p, torch.float32))
    drawn, all_logits = [], []
    for t in range(tokens):
        logits = norm(x) @ v.head
        token, prob = full(-1, torch.int32), full(0, torch.float32)
        ex.sample(logits, draws[t], token, prob, **limits)
        drawn.append(token)
        all_logits.append(logits)
        if t + 1 < tokens:
            pos += 1
            length += 1
            x = step(v.embed[token.long()], batch)
    result = torch.stack(drawn, dim=1), torch.stack(all_logits)
    torch.cuda.synchronize()
    ex.destroy()
    return result


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--queries", type=int, default=6)
    p.add_argument("--tokens", type=int, default=16)
    a = p.parse_args()
    variant = Variant()
    g = torch.Generator().manual_seed(1)
    prompt = torch.randint(0, variant.vocab, (100,), generator=g).tolist()
    queries = [torch.randint(0, variant.vocab, (3 + 5 * s,), generator=g).tolist() for s in range(a.queries)]
    tokens, _ = answer(variant, prompt, queries, a.tokens)
    for s, row in enumerate(tokens.tolist()):
        print(f"query {s}: {row}")


if __name__ == "__main__":
    main()
