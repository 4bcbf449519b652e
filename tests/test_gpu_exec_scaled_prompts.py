"""Appending whole prompts to a cache of 8 bits: many heads, long blocks, columns shared among workgroups, more blocks than workgroups.
The definition is computed in 64 bits on the device."""
import numpy as np
import pytest
import torch

import paper_1905_13348_amd as pkg

pytestmark = pytest.mark.gpu

i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()
BF16, FP16 = torch.bfloat16, torch.float16
CODES, SCALES = torch.float8_e4m3fn, torch.float8_e8m0fnu


def rounded(x):
    """x in 64 bits to the nearest number of e4m3 (of up to 448): three bits behind the first one, steps of 2^-9 at the least."""
    step = torch.exp2(torch.frexp(x)[1].clamp_min(-5).double() - 4)
    return torch.round(x / step) * step


def need(top):
    """The least e >= 1 with top <= 448 * 2^(e - 127)."""
    fraction, power = torch.frexp(top)
    return torch.where(top == 0, 1, (power.long() - 9 + (fraction > 0.875).long() + 127).clamp_min(1))


def rotated(x, pos, freq, interleaved):
    x = x.double()
    if freq is None:
        return x
    half = freq.numel()
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    angle = pos.double()[:, None] * freq[None, :]
    cos, sin = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    y = x.clone()
    y[..., a], y[..., b] = x[..., a] * cos - x[..., b] * sin, x[..., b] * cos + x[..., a] * sin
    return y


def check(first, new, heads, kv, dim, page, block, rot, layout="token", dtype=BF16, interleaved=False, fused=False, seed=0):
    """Keys of sequences that have `first` and get `new`.  Values and their scales have to be the definition's bit by bit.  A rotated
    number is off by `off`, of products in 32 bits (sine and cosine 2^-24 each, three roundings of the larger of a pair), so that a
    scale is that of a largest number as far off, and a code is off by half a step and that."""
    first, new = np.asarray(first, dtype=np.int64), np.asarray(new, dtype=np.int64)
    S, n = len(first), int(new.sum())
    print(f"append: {n} tokens of {S} sequences, {heads} + 2 x {kv} heads of {dim}, pages {page}, blocks {block}, rotated {rot}", flush=True)
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    start = np.concatenate([[0], np.cumsum(new)])
    seq = np.repeat(np.arange(S), new)
    pos = first[seq] + np.arange(n) - start[seq]
    used = -(-(first + new) // page)
    width, total = int(used.max()), int(used.sum()) + 1
    table = np.full((S, width), -1, dtype=np.int64)
    table[np.arange(width)[None, :] < used[:, None]] = rng.permutation(total)[:int(used.sum())]
    randn = lambda *shape: torch.randn(shape, generator=gen, device="cuda")
    loud = torch.exp(0.7 * randn(n, 1, 1))
    if fused:
        qkv = (randn(n, heads + 2 * kv, dim) * loud).to(dtype)
        q, k, v = qkv[:, :heads], qkv[:, heads:heads + kv], qkv[:, heads + kv:]
    else:
        q, k, v = ((randn(n, h, dim) * loud).to(dtype) for h in (heads, kv, kv))
    pools = [(randn(total, page, kv, dim) * 100).clamp(-448, 448).to(CODES) for _ in range(2)]
    scales = [torch.randint(116, 122, (total, page // block, kv), generator=gen, device="cuda", dtype=torch.uint8) for _ in range(2)]
    turn = lambda t: t.view(torch.uint8).transpose(1, 2).contiguous() if layout == "head" else t.view(torch.uint8)
    before = [(p.float().double(), s.long()) for p, s in zip(pools, scales)]
    dev = [(turn(p).clone(), turn(s).clone()) for p, s in zip(pools, scales)]
    freq = torch.from_numpy(10000.0 ** (-np.arange(rot // 2) / max(1, rot // 2))).cuda() if rot else None
    ex = pkg.Executor()
    cache = ex.cache(*(p.view(CODES) for p, _ in dev), layout=layout, k_scale=dev[0][1].view(SCALES), v_scale=dev[1][1].view(SCALES), dtype=dtype)
    batch = ex.batch(cache, heads, token_seq=i32(seq), token_pos=i32(pos), seq_start=i32(start), seq_len=i32(first + new), page_table=i32(table))
    out = torch.full((n, heads, dim), float("nan"), dtype=dtype, device="cuda")
    ex.append(cache, batch, q, k, v, out, freq, interleaved=interleaved)
    torch.cuda.synchronize()

    where = torch.from_numpy(pos).cuda()
    # of products in 32 bits, in units of 2^-24 of the larger number: sine and cosine, two products, the sum (0 where nothing turns)
    off_of = lambda x: (8 * 2.0 ** -24 if rot else 0.0) * x.double().abs().amax(dim=2)
    want = rotated(q, where, freq, interleaved)
    assert ((out.double() - want).abs() <= torch.finfo(dtype).eps / 2 * want.abs() + 2.0 ** -25 * (dtype == FP16) + off_of(q)[..., None]).all()

    at, slot = torch.from_numpy(table[seq, pos // page]).cuda(), where % page
    edge = np.flatnonzero(np.concatenate([[True], (seq[1:] != seq[:-1]) | (pos[1:] // block != pos[:-1] // block)]))
    count = np.diff(np.append(edge, n))
    run = torch.from_numpy(np.repeat(np.arange(len(edge)), count)).cuda()
    lead = torch.from_numpy(edge).cuda()
    p0, b0, s0 = at[lead], slot[lead] // block, slot[lead] % block
    for i, (x, off) in enumerate(((rotated(k, where, freq, interleaved), off_of(k)), (v.double(), torch.zeros((n, kv), dtype=torch.float64, device="cuda")))):
        got, e = (turn(t).view(t.dtype) for t in dev[i])      # (of "head" pages: back to tokens in front)
        got, e = got.view(CODES).float().double(), e.long()
        old_code, old_e = before[i]
        amax = x.abs().amax(dim=2)
        high, low = (torch.zeros((len(edge), kv), dtype=torch.float64, device="cuda").scatter_reduce(0, run[:, None].expand(-1, kv), y, "amax")
                     for y in (amax + off, (amax - off).clamp_min(0)))
        least, most = need(low), need(high)
        stays = torch.where((s0 == 0)[:, None], 1, old_e[p0, b0])
        least, most = torch.maximum(least, stays), torch.maximum(most, stays)
        now = e[p0, b0]
        assert ((now >= least) & (now <= most)).all()
        # the step's own codes
        power = torch.exp2((now[run] - 127).double())[..., None]
        code = got[at, slot]
        if i == 1 or not rot:
            assert torch.equal(code, rounded(x / power))
        else:
            assert ((code * power - x).abs() <= torch.maximum(2.0 ** -4 * x.abs(), 2.0 ** -10 * power) + 2 * off[..., None]).all()
        # what the blocks held in front of them, and everything else, which stays
        block_of = old_code.unflatten(1, (page // block, block)).clone()
        held = block_of[p0, b0]
        down = rounded(held * torch.exp2((old_e[p0, b0] - now).clamp_max(0).double())[:, None, :, None])
        rose = (now > old_e[p0, b0])[:, None, :, None] & (torch.arange(block, device="cuda")[None, :] < s0[:, None])[:, :, None, None]
        block_of[p0, b0] = torch.where(rose, down, held)
        expected = block_of.flatten(1, 2)
        expected[at, slot] = code
        assert torch.equal(got, expected)
        rest = old_e.clone()
        rest[p0, b0] = now
        assert torch.equal(e, rest)
    ex.destroy()


@pytest.mark.parametrize("dim", [128, 256])
@pytest.mark.parametrize("layout, interleaved", [("token", False), ("head", True)])
@pytest.mark.parametrize("kv", [8, 5])
def test_prompts(dim, layout, interleaved, kv):
    """Chunks of several tokens, four tokens' queries to a workgroup, a block's columns shared among workgroups."""
    check([0, 40, 7], [1300, 900, 103], 2 * kv, kv, dim, 32, 32, dim, layout, FP16 if interleaved else BF16, interleaved, fused=kv == 8, seed=dim + kv)


@pytest.mark.parametrize("kv, dim, tokens", [(8, 256, 5000), (8, 256, 9001), (16, 128, 9001), (5, 256, 9001), (32, 64, 9001)])
def test_columns_one_after_the_other(kv, dim, tokens):
    """So many blocks that a workgroup takes several columns in a row, with the sines and cosines of the first."""
    check([3], [tokens], kv, kv, dim, 16, 4, dim, seed=kv)
    check([3], [tokens], kv, kv, dim, 16, 4, dim // 2, "head", FP16, True, seed=kv)


@pytest.mark.parametrize("block, dim, rot", [(128, 128, 128), (512, 256, 256), (256, 64, 32), (1024, 128, 64)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_blocks_longer_than_a_wave_holds(block, dim, rot, interleaved):
    """Sines and cosines come in several turns, for the block's largest and again for its codes, for several columns."""
    check([0, 100, 700], [2100, 37, 1500], 4, 4, dim, block, block, rot, "head" if interleaved else "token", BF16, interleaved, seed=block)


def test_a_block_of_many_columns():
    """The same for columns one after the other: as many chunks as leave a workgroup several, of blocks that are longer than it holds."""
    check([1] * 40, [3500 + 17 * i for i in range(40)], 8, 8, 256, 64, 64, 256, seed=3)


def test_short_runs_in_a_chunk():
    """Sequences of some tokens beside long ones: several blocks begin within a chunk."""
    rng = np.random.default_rng(4)
    new = np.where(rng.random(700) < 0.97, rng.integers(1, 9, 700), rng.integers(50, 200, 700))
    check(rng.integers(0, 50, 700), new, 16, 8, 128, 16, 16, 128, seed=5)
    check(rng.integers(0, 50, 700), new, 8, 8, 128, 16, 16, 64, "head", FP16, True, seed=6)


def test_more_blocks_than_a_grid_has_workgroups():
    """Tokens with a scale each, and the queries of so many tokens: workgroups go on with others."""
    check([0, 5, 2], [140_000, 130_001, 3], 1, 1, 64, 256, 1, 16, seed=7)
