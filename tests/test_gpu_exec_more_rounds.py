"""More work than a launch's grid has workgroups for: read, beam search, the table's rows and tokens.  Workgroups go on with the next."""
import numpy as np
import pytest
import torch

import paper_1905_13348_amd as pkg

pytestmark = pytest.mark.gpu

i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


@pytest.mark.parametrize("coded", [False, True])
def test_read(coded):
    """2^26 pieces of sixteen dimensions and more: tokens that name the keys of a short cache over and over."""
    n, keys, kv, dim, page = 530_001, 1000, 8, 128, 16
    gen = torch.Generator(device="cuda").manual_seed(1)
    pages = -(-keys // page)
    shape = (pages, page, kv, dim)
    x = [torch.randn(shape, generator=gen, device="cuda") for _ in range(2)]
    ex = pkg.Executor()
    if coded:
        codes = [(y * 100).clamp(-448, 448).to(torch.float8_e4m3fn) for y in x]
        e = [torch.randint(115, 130, (pages, page // 4, kv), generator=gen, device="cuda", dtype=torch.uint8) for _ in range(2)]
        cache = ex.cache(*codes, k_scale=e[0].view(torch.float8_e8m0fnu), v_scale=e[1].view(torch.float8_e8m0fnu))
        x = [(c.float() * torch.exp2(s.float() - 127).repeat_interleave(4, dim=1)[..., None]).bfloat16() for c, s in zip(codes, e)]
    else:
        x = [y.bfloat16() for y in x]
        cache = ex.cache(*x)
    order = torch.randperm(pages, generator=gen, device="cuda")
    pos = (torch.arange(n, device="cuda") * 7 % (keys + 1)).int()      # (there is no key number `keys`: zeros)
    batch = ex.batch(cache, kv, token_seq=torch.zeros(n, dtype=torch.int32, device="cuda"), token_pos=pos, seq_start=i32([0, n]), seq_len=i32([keys]),
                     page_table=order.int().view(1, -1), max_len=keys)
    k, v = (torch.full((n, kv, dim), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    print(f"read: {n} tokens", flush=True)
    ex.read(cache, batch, k, v)
    for got, y in ((k, x[0]), (v, x[1])):
        of_key = torch.cat([y[order].flatten(0, 1)[:keys], torch.zeros((1, kv, dim), dtype=torch.bfloat16, device="cuda")])
        assert torch.equal(got, of_key[pos.long()])
    ex.destroy()


@pytest.mark.parametrize("picks", [4, 20])
def test_beam(picks):
    """More than 2^20 parts and 2^16 queries, with beams that have ended and dead ones between them.  Every row has the same eight logits in
    an order of its own, so the sum of its weights is the same, and scores are multiples of 1/4 for a beam's tokens and of 1/64 for the
    beams: continuations are 1/64 apart at the least, but those of beams that have ended, whose distance is asserted."""
    Q, W, V = 270_000, 4, 8
    gen = torch.Generator(device="cuda").manual_seed(2)
    x = torch.rand((Q * W, V), generator=gen, device="cuda").argsort(dim=1).float() / 4
    scores = -torch.randint(0, 40, (Q, W), generator=gen, device="cuda").float() / 4 - torch.arange(W, device="cuda") / 64
    kind = torch.randint(0, 8, (Q, W), generator=gen, device="cuda")
    ended = (kind == 0).int()
    scores[kind == 1] = float("-inf")
    ex = pkg.Executor()
    out = [torch.full((Q, picks), -7, dtype=d, device="cuda") for d in (torch.int32, torch.int32, torch.float32)]
    print(f"beam: {Q} queries", flush=True)
    ex.beam(x, scores, *out, ended=ended, end_token=3)
    s, lse = scores.double()[:, :, None], torch.logsumexp(torch.arange(V).double() / 4, 0).item()
    rank = s + x.double().view(Q, W, V) - lse
    alone = torch.full_like(rank, -np.inf)
    alone[:, :, 3] = s[:, :, 0]
    rank = torch.where(ended[:, :, None] != 0, alone, rank).flatten(1)
    best, which = torch.sort(rank, dim=1, descending=True, stable=True)
    gap = best[:, :-1] - best[:, 1:]
    assert gap[best[:, 1:] > -np.inf].min() > 1e-4
    best, which = best[:, :picks], which[:, :picks]
    there = best > -np.inf
    parent = torch.where(there, torch.arange(Q, device="cuda")[:, None] * W + which // V, -1)
    assert torch.equal(out[0], parent.int()) and torch.equal(out[1], torch.where(there, which % V, -1).int())
    # (scores up to 16: half a step of 32 bits; of weights in 32 bits 14 roundings each and 2.5 of an exponent up to 1.75)
    assert torch.equal(torch.isinf(out[2]), ~there)
    assert ((out[2].double() - best)[there].abs() <= 16 * 2.0 ** -24 + 19 * 2.0 ** -24).all()
    ex.destroy()


def test_rows_of_a_wide_table():
    """4096 sequences on rows of 8200 pages, more columns than workgroups take at once: every row goes on from another."""
    S, W, P, pages, used = 4096, 8200, 2, 40_000, 5
    rng = np.random.default_rng(3)
    length = np.zeros(S, dtype=np.int64)
    length[:used] = [W * P, W * P - 3, 9000, 1, 0]
    table = np.full((S, W), -1)
    free = rng.permutation(pages)
    for s in range(used):
        need = -(-length[s] // P)
        table[s, :need], free = free[:need], free[need:]
    refs = np.bincount(table[table >= 0], minlength=pages)
    parent = np.where(np.arange(S) < 16, (np.arange(S) * 3 + 1) % used, -1)
    parent[S - 1] = 0
    ex = pkg.Executor()
    t = ex.table(S, W, P, pages, 64)
    t.page_table.copy_(i32(table)), t.seq_len.copy_(i32(length)), t.page_refs.copy_(i32(refs))
    print(f"advance: {S} sequences on rows of {W} pages", flush=True)
    ex.advance(t, i32(np.zeros(S)), i32(parent))
    there = parent >= 0
    want = np.where(there[:, None], table[np.maximum(parent, 0)], -1)
    assert np.array_equal(t.page_table.cpu().numpy(), want)
    assert np.array_equal(t.seq_len.cpu().numpy(), np.where(there, length[np.maximum(parent, 0)], 0))
    assert np.array_equal(t.page_refs.cpu().numpy(), np.bincount(want[want >= 0], minlength=pages))
    assert (t.taken == 0).all() and (t.token_seq == -1).all() and (t.copies == -1).all()
    ex.destroy()


def test_many_tokens():
    """A step of more tokens than the workgroups that write them have threads."""
    S, P, room = 300, 1024, 300_001
    rng = np.random.default_rng(4)
    new = rng.integers(0, 1900, S)
    total = int(new.sum())
    assert 262_144 < total < room
    ex = pkg.Executor()
    t = ex.table(S, 4, P, 4 * S, room)
    print(f"advance: {total} tokens", flush=True)
    for first in (0, 1):
        if first:
            ex.advance(t, i32(np.full(S, -5000)))
            ex.advance(t, i32(np.ones(S)))
        ex.advance(t, i32(new))
        start = np.concatenate([[0], np.cumsum(new)])
        seq = np.repeat(np.arange(S), new)
        assert np.array_equal(t.taken.cpu().numpy(), new) and np.array_equal(t.seq_start.cpu().numpy(), start)
        assert np.array_equal(t.token_seq.cpu().numpy(), np.concatenate([seq, np.full(room - total, -1)]))
        assert np.array_equal(t.token_pos.cpu().numpy(), np.concatenate([first + np.arange(total) - start[seq], np.full(room - total, -1)]))
    ex.destroy()
