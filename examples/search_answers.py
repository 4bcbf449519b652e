"""A worker searching for the best answers: the executor's calls of beam search as they follow each other.

    python examples/search_answers.py [--queries 3] [--beams 4] [--tokens 12] [--bits 8]

Every query has some beams, each a sequence of the worker's table.  A step picks the best continuations of all beams of a query,
lets the sequences go on from the beams that they continue (pages are shared, a page that is not full is copied), and appends and
attends over a cache of 8 or 16 bits.  Lengths, pages and the batch's arrays stay on the device; a beam that has ended takes no
more tokens and keeps its score, and one for which a query has no continuation left is empty until the query has enough again.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from answer_queries import Variant, norm  # noqa: E402
from paper_1905_13348_amd import Executor  # noqa: E402


def make_cache(ex, variant, pages, page, bits, block):
    v = variant
    shape = (pages, page, v.kv_heads, v.head_dim)
    if bits == 16:
        return ex.cache(*(torch.zeros(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2)))
    zeros = lambda *s: torch.zeros(s, dtype=torch.uint8, device="cuda")
    scales = [zeros(pages, page // block, v.kv_heads).view(torch.float8_e8m0fnu) for _ in range(2)]
    return ex.cache(*(zeros(*shape).view(torch.float8_e4m3fn) for _ in range(2)), k_scale=scales[0], v_scale=scales[1])


def search(variant, queries, tokens, beams=4, end_token=1, bits=8, alpha=0.7, page=16, block=8):
    """queries: token numbers of each (one at least).  Returns the beams' tokens [queries, beams, tokens] (-1 and a score of minus
    infinity where there were fewer answers than beams), their scores, and of every step what was picked from what."""
    v, Q, W = variant, len(queries), beams
    S, longest, all_new = Q * W, max(len(q) for q in queries) + tokens, sum(len(q) for q in queries)
    i32 = lambda a: torch.as_tensor(a, dtype=torch.int32).cuda()
    ex = Executor()
    width = -(-longest // page)
    pages = S * (width + 1)
    table = ex.table(S, width, page, pages, max(S, all_new))
    caches = [make_cache(ex, v, pages, page, bits, block) for _ in range(v.layers)]

    def batch_of(n):
        """The first n tokens of the table's step."""
        arrays = table.arrays()
        b = ex.batch(caches[0], v.heads, token_seq=arrays.pop("token_seq")[:n], token_pos=arrays.pop("token_pos")[:n], **arrays)
        ex.reserve(caches[0], b)
        return b

    def step(x, batch):
        """Hidden states of the batch's tokens, through all layers."""
        ex.plan(batch)
        n = x.shape[0]
        out = torch.empty((n, v.heads, v.head_dim), dtype=x.dtype, device="cuda")
        for i, cache in enumerate(caches):
            ex.copy(cache, table)
            qkv = (norm(x) @ v.qkv[i]).view(n, v.heads + 2 * v.kv_heads, v.head_dim)
            q, k, w = qkv.split([v.heads, v.kv_heads, v.kv_heads], dim=1)
            ex.append(cache, batch, q, k, w, q, v.freq)      # (queries in place)
            ex.attend(cache, batch, q, out)
            x = x + out.flatten(1) @ v.proj[i]
            x = x + torch.relu(norm(x) @ v.up[i]) @ v.down[i]
        return norm(x) @ v.head

    # the queries are read by the first beam of each; the others go on from it in the first step of the search
    new = torch.zeros((Q, W), dtype=torch.int32)
    new[:, 0] = torch.tensor([len(q) for q in queries])
    ex.advance(table, new.view(-1).cuda())
    logits = step(v.embed[i32(sum(queries, [])).long()], batch_of(all_new))
    last = (table.seq_start[1:].view(Q, W)[:, :1] - 1).expand(Q, W).reshape(-1)
    logits = logits[last.long()]

    scores = torch.full((Q, W), float("-inf"), device="cuda")
    scores[:, 0] = 0
    ended = torch.zeros((Q, W), dtype=torch.int32, device="cuda")
    length = torch.ones((Q, W), device="cuda")
    history = torch.zeros((S, 0), dtype=torch.int32, device="cuda")
    batch, picked = batch_of(S), []
    refused = torch.zeros((), dtype=torch.int64, device="cuda")
    for t in range(tokens):
        parent, token = (torch.empty((Q, W), dtype=torch.int32, device="cuda") for _ in range(2))
        best = torch.empty((Q, W), device="cuda")
        factor = length ** -alpha
        ex.beam(logits, scores, parent, token, best, ended=ended, factor=factor, end_token=end_token)
        picked.append(dict(logits=logits, scores=scores, ended=ended, factor=factor, parent=parent, token=token, best=best, history=history))
        # (a pick of -1: the query had fewer continuations than beams; its score of minus infinity keeps it from going on)
        none = parent.view(-1) < 0
        go = parent.view(-1).clamp_min(0).long()
        was = ended.view(-1)[go].view(Q, W)
        length = length.view(-1)[go].view(Q, W) + (1 - was)
        ended, scores = ((token == end_token) | (token < 0)).int(), best
        history = torch.cat([history[go], token.view(-1, 1)], dim=1).masked_fill(none[:, None], -1)
        if t + 1 < tokens:
            new = (1 - ended).view(-1)
            ex.advance(table, new, parent.view(-1))
            refused += (table.taken != new).sum()
            x = v.embed[token.view(-1)[table.token_seq[:S].clamp_min(0).long()].clamp_min(0).long()]
            logits = step(x, batch)[table.seq_start[:-1].clamp_max(S - 1).long()]
    torch.cuda.synchronize()
    if refused:      # (whose logits would be another beam's)
        raise RuntimeError(f"{int(refused)} steps of beams for which no pages were left")
    ex.destroy()
    return history.view(Q, W, tokens), scores, picked


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--queries", type=int, default=3)
    p.add_argument("--beams", type=int, default=4)
    p.add_argument("--tokens", type=int, default=12)
    p.add_argument("--bits", type=int, default=8, choices=(8, 16))
    a = p.parse_args()
    variant = Variant()
    g = torch.Generator().manual_seed(1)
    queries = [torch.randint(0, variant.vocab, (5 + 9 * s,), generator=g).tolist() for s in range(a.queries)]
    history, scores, _ = search(variant, queries, a.tokens, a.beams, bits=a.bits)
    for q in range(a.queries):
        for w in range(a.beams):
            print(f"query {q}, score {scores[q, w]:.3f}: {history[q, w].tolist()}")


if __name__ == "__main__":
    main()
