"""A cache of 8 bits against its definition in 64 bits: what append leaves, what read gives, what attend computes."""
import numpy as np
import pytest
import torch

import exec_ref
from exec_ref import attend_tolerance
import paper_1905_13348_amd as pkg
import scaled_ref
from scaled_ref import Scene, need, numbers, rounded

pytestmark = pytest.mark.gpu

i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()
BF16, FP16 = torch.bfloat16, torch.float16


# ---- append and read ------------------------------------------------------------------------------------------

class Cache:
    """A cache of 8 bits on the device, with the host's idea of it."""

    def __init__(self, pages, kv, dim, page, block, layout="token", dtype=BF16, seed=0):
        rng = np.random.default_rng(seed)
        self.page, self.block, self.layout, self.dtype = page, block, layout, dtype
        self.code = [rounded(rng.standard_normal((pages, page, kv, dim)) * 100) for _ in range(2)]
        self.e = [rng.integers(116, 122, (pages, page // block, kv)) for _ in range(2)]
        turn = (lambda t: t.view(torch.uint8).transpose(1, 2).contiguous().view(t.dtype)) if layout == "head" else lambda t: t
        self.pools = [turn(scaled_ref.codes(c)).cuda() for c in self.code]
        self.scales = [turn(scaled_ref.scales(e)).cuda() for e in self.e]

    def on(self, ex):
        return ex.cache(*self.pools, layout=self.layout, k_scale=self.scales[0], v_scale=self.scales[1], dtype=self.dtype)

    def get(self, i):
        """Codes (as numbers) and scales (as bytes) of keys or values, from the device."""
        p, s = self.pools[i].float().cpu().double().numpy(), self.scales[i].view(torch.uint8).cpu().numpy().astype(int)
        return (p.transpose(0, 2, 1, 3), s.transpose(0, 2, 1)) if self.layout == "head" else (p, s)

    def append(self, i, x, at, written):
        """By the definition: x [n][kv][dim], at [n] = (sequence, position, page or None, begins the step in its block?)."""
        code, e = self.code[i], self.e[i]
        blocks = {}
        for t, (s, pos, page) in enumerate(at):
            if t in written:
                blocks.setdefault((s, page, pos % self.page // self.block), []).append(t)
        for (s, page, b), ts in blocks.items():
            offset = at[ts[0]][1] % self.block
            for h in range(x.shape[1]):
                v = np.abs(x[ts, h])
                top = need(np.max(v[np.isfinite(v)], initial=0.0))
                new = top if offset == 0 else max(top, e[page, b, h])
                if offset and new > e[page, b, h]:
                    rows = slice(b * self.block, b * self.block + offset)
                    code[page, rows, h] = rounded(code[page, rows, h] * 2.0 ** (e[page, b, h] - new))
                e[page, b, h] = new
                for t in ts:
                    code[page, at[t][1] % self.page, h] = rounded(x[t, h] * 2.0 ** (127 - new))


def _append(first, new, kv=2, heads=4, dim=64, page=16, block=8, layout="token", dtype=BF16, rot=0, interleaved=False, seed=0,
            loud=1.0, spoil=None, fused=False, with_q=True, values=None, missing=()):
    """Appends to sequences that have `first` keys; the whole cache by the definition, queries too."""
    ex = pkg.Executor()
    rng = np.random.default_rng(seed)
    S, n = len(first), int(sum(new))
    start = np.concatenate([[0], np.cumsum(new)]).astype(int)
    seq = np.repeat(np.arange(S), new)
    pos = np.array(first)[seq] + np.arange(n) - start[seq]
    width = int(max(f + m for f, m in zip(first, new)) // page + 1)
    table = rng.permutation(S * width + 2)[:S * width].reshape(S, width)
    for s, j in missing:
        table[s, j] = -1 if j % 2 else S * width + 2
    c = Cache(S * width + 2, kv, dim, page, block, layout, dtype, seed)
    scale = np.exp(loud * rng.standard_normal((n, 1, 1)))
    if fused:
        qkv = torch.from_numpy(rng.standard_normal((n, heads + 2 * kv, dim)) * scale).to(dtype).cuda()
        q, k, v = qkv[:, :heads], qkv[:, heads:heads + kv], qkv[:, heads + kv:]
    else:
        q, k, v = (torch.from_numpy(rng.standard_normal((n, h, dim)) * scale).to(dtype).cuda() for h in (heads, kv, kv))
    if values is not None:
        values(k, v)
    freq = 10000.0 ** (-np.arange(rot // 2) / max(1, rot // 2))
    pos_in, seq_in = pos.copy(), seq.copy()
    if spoil:
        spoil(pos_in, seq_in)
    cache = c.on(ex)
    b = ex.batch(cache, heads, token_seq=i32(seq_in), token_pos=i32(pos_in), seq_start=i32(start),
                 seq_len=i32(np.array(first) + np.array(new)), page_table=i32(table))
    out = torch.full((n, heads, dim), float("nan"), dtype=dtype, device="cuda")
    kd, vd, qd = (t.double().cpu().numpy() for t in (k, v, q))
    ex.append(cache, b, q if with_q else None, k, v, out if with_q else None, torch.from_numpy(freq).cuda() if rot else None,
              interleaved=interleaved)
    torch.cuda.synchronize()
    at = [(int(s), int(p), int(table[s, p // page])) for s, p in zip(seq, pos)]
    written = {t for t in range(n) if pos_in[t] == pos[t] and seq_in[t] == seq[t] and 0 <= at[t][2] < S * width + 2
               and pos_in[start[seq[t]]] == first[seq[t]]}
    return ex, c, cache, dict(k=kd, v=vd, q=qd, pos=pos, pos_in=pos_in, at=at, written=written, out=out, freq=freq if rot else [],
                              seq=seq, start=start, table=table)


def _exact(c, i, x, r):
    c.append(i, x, r["at"], r["written"])
    code, e = c.get(i)
    assert np.array_equal(e, c.e[i])
    assert np.array_equal(np.isnan(code), np.isnan(c.code[i]))
    bad = ~np.isnan(code) & (code != c.code[i])
    assert not bad.any(), f"{bad.sum()} of {bad.size}, first {np.argwhere(bad)[:3].tolist()}"


def _check_queries(r, interleaved):
    want = exec_ref.rotate(r["q"], r["pos_in"], r["freq"], interleaved)
    got = r["out"].double().cpu().numpy()
    tol = torch.finfo(r["out"].dtype).eps / 2 * np.abs(want) + 8 * 2.0 ** -24 * 2 * np.abs(r["q"]).max(axis=2, keepdims=True)
    assert (np.abs(got - want) <= tol).all()


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("layout", ["token", "head"])
@pytest.mark.parametrize("block", [1, 4, 16])
def test_append_without_rotation(dim, dtype, layout, block):
    """Every code and every scale, bit by bit: tokens that begin blocks, go on in them, and both."""
    ex, c, _, r = _append([0, 5, 16, 31, 3], [1, 40, 2, 1, 13], dim=dim, dtype=dtype, layout=layout, block=block, seed=dim + block,
                          fused=block == 4)
    _exact(c, 0, r["k"], r)
    _exact(c, 1, r["v"], r)
    assert torch.equal(r["out"].double().cpu(), torch.from_numpy(r["q"]))
    ex.destroy()


@pytest.mark.parametrize("page, block", [(1, 1), (2, 2), (8, 2), (64, 64), (128, 32), (512, 512), (256, 1)])
def test_append_pages_and_blocks(page, block):
    ex, c, _, r = _append([0, 70, 600, 3], [130, 200, 1, 70], page=page, block=block, seed=page + block, kv=1)
    _exact(c, 0, r["k"], r)
    _exact(c, 1, r["v"], r)
    ex.destroy()


@pytest.mark.parametrize("dim, rot", [(64, 64), (128, 32), (128, 128), (256, 256)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_append_rotated(dim, rot, interleaved):
    """Values exactly; a rotated key's code is off by half a step of e4m3 and the products in 32 bits, of which there are three
    roundings of at most |x| each and 2 ulp of the sine; a scale is that of a largest number as far off."""
    first, new = [0, 5, 16, 2000], [1, 40, 2, 17]
    ex, c, _, r = _append(first, new, dim=dim, rot=rot, interleaved=interleaved, block=4, seed=rot, fused=True)
    _exact(c, 1, r["v"], r)
    _check_queries(r, interleaved)
    keys = exec_ref.rotate(r["k"], r["pos"], r["freq"], interleaved)
    off = 8 * 2.0 ** -24 * 2 * np.abs(r["k"]).max(axis=2, keepdims=True)
    before = [a.copy() for a in (c.code[0], c.e[0])]
    code, e = c.get(0)
    for s in range(len(first)):
        for b in range(first[s] // 4, (first[s] + new[s] - 1) // 4 + 1):
            ts = [t for t in range(len(r["seq"])) if r["seq"][t] == s and r["pos"][t] // 4 == b]
            page, slot = r["at"][ts[0]][2], b * 4 % 16
            offset = r["pos"][ts[0]] % 4
            for h in range(2):
                got = e[page, slot // 4, h]
                top = np.abs(keys[ts, h]).max()
                low, high = need(top - off[ts, h].max()), need(top + off[ts, h].max())
                if offset:
                    low, high = max(low, before[1][page, slot // 4, h]), max(high, before[1][page, slot // 4, h])
                assert low <= got <= high
                step = 2.0 ** (got - 127)
                for t in ts:
                    x, y = keys[t, h], code[page, r["pos"][t] % 16, h] * step
                    assert (np.abs(x - y) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * step) + 2 * off[t, h]).all()
                rows = slice(slot, slot + offset)
                assert np.array_equal(code[page, rows, h], rounded(before[0][page, rows, h] * 2.0 ** (min(0, before[1][page, slot // 4, h] - got))))
    ex.destroy()


def test_append_step_by_step():
    """Tokens one at a time end as the definition says, not as all at once would: earlier codes are rounded again whenever a
    scale rises."""
    ex = pkg.Executor()
    rng = np.random.default_rng(9)
    c = Cache(3, 2, 64, 32, 16, seed=9)
    cache = c.on(ex)
    for t in range(40):
        x = torch.from_numpy(rng.standard_normal((2, 1, 2, 64)) * np.exp(t / 8)).to(BF16).cuda()
        b = ex.batch(cache, 2, token_seq=i32([0]), token_pos=i32([t]), seq_start=i32([0, 1]), seq_len=i32([t + 1]), page_table=i32([[2, 0]]))
        ex.append(cache, b, None, x[0], x[1], None)
        for i in range(2):
            c.append(i, x[i].double().cpu().numpy(), [(0, t, (2, 0)[t // 32])], {0})
            code, e = c.get(i)
            assert np.array_equal(code, c.code[i]) and np.array_equal(e, c.e[i]), t
    ex.destroy()


def test_append_numbers():
    """Zeros, the type's largest and smallest numbers, infinities, NaN: finite ones decide the scale, the others become NaN."""
    def values(k, v):
        k[0] = 0
        k[1, 0, :5] = torch.tensor([float("inf"), float("-inf"), float("nan"), 1.0, -2.5])
        k[2, 0] = float("nan")
        v[0, :, 0] = 3.0e38
        v[1, :, 3] = 1e-40
        v[3] = -0.0
        v[4] = 2.0 ** -130
        v[5, 0, 1] = float("-inf")
    for first in ([0, 0, 0, 0, 0, 0], [3, 3, 3, 3, 3, 3]):
        ex, c, _, r = _append(first, [1] * 6, values=values, seed=2)
        _exact(c, 0, r["k"], r)
        _exact(c, 1, r["v"], r)
        ex.destroy()


def test_append_borders_of_a_scale():
    """A largest number of exactly 448 times a power of two takes that power, the next one above twice as much."""
    def values(k, v):
        k[:] = 0.001
        v[:] = 0.001
        for t in range(8):
            k[t, 0, 7] = 448 * 2.0 ** (t - 6)
            v[t, 0, 9] = 450 * 2.0 ** (t - 6)
    ex, c, _, r = _append([0] * 8, [1] * 8, values=values, seed=3)
    _exact(c, 0, r["k"], r)
    _exact(c, 1, r["v"], r)
    _, e = c.get(0)
    assert {int(e[r["at"][t][2], 0, 0]) for t in range(8)} == {t - 6 + 127 for t in range(8)}
    _, e = c.get(1)
    assert {int(e[r["at"][t][2], 0, 0]) for t in range(8)} == {t - 5 + 127 for t in range(8)}
    ex.destroy()


def test_append_scales_at_the_ends():
    """Blocks that go on with scales of 0 (2^-127), 254 and 255 (NaN, which stays)."""
    for old in (0, 1, 254, 255):
        ex = pkg.Executor()
        c = Cache(2, 1, 64, 8, 8, seed=4)
        for i in range(2):
            c.e[i][:] = old
            c.scales[i].view(torch.uint8).fill_(old)
        cache = c.on(ex)
        x = torch.full((2, 1, 1, 64), 1.5, dtype=BF16, device="cuda")
        x[1, 0, 0, 3] = 2.9e38
        b = ex.batch(cache, 1, token_seq=i32([0]), token_pos=i32([5]), seq_start=i32([0, 1]), seq_len=i32([6]), page_table=i32([[1]]))
        ex.append(cache, b, None, x[0], x[1], None)
        for i in range(2):
            code, e = c.get(i)
            if old == 255:
                assert (e[1] == 255).all()
                continue
            c.append(i, x[i].double().cpu().numpy(), [(0, 5, 1)], {0})
            assert np.array_equal(code, c.code[i]) and np.array_equal(e, c.e[i])
        ex.destroy()


@pytest.mark.parametrize("case", ["padding behind", "padding in front", "a block of padding", "a gap", "backwards", "another sequence", "no page", "beyond"])
def test_append_what_is_not_written(case):
    """Tokens out of their sequence's order, padding and positions without a page leave the cache as it is."""
    spoil, missing = None, ()
    if case == "padding behind":
        def spoil(pos, seq): pos[18:20] = -1
    elif case == "padding in front":
        def spoil(pos, seq): pos[0] = -1
    elif case == "a block of padding":
        def spoil(pos, seq): pos[11:20], pos[29:32] = -1, -1
    elif case == "a gap":
        def spoil(pos, seq): pos[5:9] += 3
    elif case == "backwards":
        def spoil(pos, seq): pos[3], pos[4] = pos[4], pos[3]
    elif case == "another sequence":
        def spoil(pos, seq): seq[6], seq[7], seq[21] = 1, -1, 7
    elif case == "no page":
        missing = [(0, 0), (1, 1)]
    else:
        def spoil(pos, seq): pos[19] = 1 << 30
    ex, c, _, r = _append([2, 9], [20, 12], rot=32, spoil=spoil, missing=missing, seed=5, dim=64)
    _exact(c, 1, r["v"], r)
    assert len(r["written"]) < 32
    _check_queries(r, False)
    ex.destroy()


def test_append_without_queries_and_in_place():
    ex, c, _, r = _append([2, 9], [20, 12], rot=0, with_q=False, seed=6)
    _exact(c, 0, r["k"], r)
    _exact(c, 1, r["v"], r)
    assert torch.isnan(r["out"]).all()
    ex.destroy()


def test_append_many():
    """More blocks than a grid's limit allows workgroups for, through chunks of tokens, to the end."""
    ex, c, _, r = _append([0, 7], [3000, 70_001], kv=1, heads=1, dim=64, page=64, block=64, seed=7)
    _exact(c, 0, r["k"], r)
    _exact(c, 1, r["v"], r)
    ex.destroy()


@pytest.mark.parametrize("coded", [False, True])
@pytest.mark.parametrize("layout", ["token", "head"])
@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_read(coded, layout, dtype, dim):
    """Every number of a cache, exactly; zeros where there is none; strided results leave what is between them."""
    ex = pkg.Executor()
    kw = dict(seqs=[(70, 1), (3, 1), (0, 0), (129, 1)], dim=dim, dtype=dtype, layout=layout, seed=8, page=32)
    sc = Scene(block=8, low=90, high=140, **kw) if coded else exec_ref.Scene(**kw)
    cache = sc.cache(ex) if coded else ex.cache(sc.k_pool, sc.v_pool, layout=layout)
    seq = np.repeat(np.arange(4), sc.length)
    start = np.concatenate([[0], np.cumsum(sc.length)])
    pos = np.arange(len(seq)) - start[seq]
    pos[10], pos[75], seq[100] = -1, 100_000, 4
    b = ex.batch(cache, 8, token_seq=i32(seq), token_pos=i32(pos), seq_start=i32(start), seq_len=i32(sc.length), page_table=i32(sc.table))
    wide = torch.full((len(seq), 3, 2, dim), 7.0, dtype=dtype, device="cuda")
    ex.read(cache, b, wide[:, 0], wide[:, 2])
    got = wide.double().cpu().numpy()
    for i, j in ((0, 0), (1, 2)):
        want = np.concatenate([f[:n] for f, n in zip(sc.full[i], sc.length)])
        want[[10, 75, 100]] = 0
        assert np.array_equal(got[:, j], want)
    assert (got[:, 1] == 7).all()
    ex.destroy()


# ---- attend ---------------------------------------------------------------------------------------------------

def _attend(ex, sc, scale=None, batch=None, cache=None):
    cache = sc.cache(ex) if cache is None else cache
    batch = sc.batch(ex, cache) if batch is None else batch
    out = torch.full((sc.n, sc.heads, sc.dim), 7.0, dtype=sc.dtype, device="cuda")
    ex.plan(batch)
    ex.attend(cache, batch, sc.q, out, scale)
    torch.cuda.synchronize()
    return out.double().cpu().numpy()


def _check(sc, scale=None, limits=None, got=None):
    ex = pkg.Executor()
    got = _attend(ex, sc, scale) if got is None else got
    want, weighted, top = sc.reference(sc.dim ** -0.5 if scale is None else scale, limits)
    tol = attend_tolerance(want, weighted, top, sc.dtype, sc.length.max())
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), f"{bad.sum()} of {bad.size} off, first {np.argwhere(bad)[:3].tolist()}, worst {np.nanmax(np.abs(got - want) / tol)}"
    ex.destroy()


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("layout", ["token", "head"])
@pytest.mark.parametrize("new", ["one", "some"])
def test_attend_types_and_layouts(dim, dtype, layout, new):
    seqs = [(1, 1), (31, 1), (64, 1), (65, 1), (200, 1)] if new == "one" else [(5, 5), (70, 3), (130, 40), (64, 64), (33, 1)]
    _check(Scene(seqs, dim=dim, dtype=dtype, layout=layout, seed=dim, block=4))


@pytest.mark.parametrize("length", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 127, 128, 129, 255, 256, 257, 511, 513, 1000])
def test_attend_lengths(length):
    _check(Scene([(length, 1), (length + 1, 2)], heads=4, kv_heads=1, dim=64, seed=length))


@pytest.mark.parametrize("heads, kv", [(1, 1), (2, 2), (3, 1), (8, 1), (16, 1), (17, 1), (40, 8), (64, 2), (128, 1), (60, 4), (36, 12)])
def test_attend_head_counts(heads, kv):
    _check(Scene([(50, 1), (130, 9), (200, 1)], heads=heads, kv_heads=kv, dim=64, seed=heads))
    _check(Scene([(300, 1), (77, 1)], heads=heads, kv_heads=kv, dim=128, seed=heads))


@pytest.mark.parametrize("page, block", [(1, 1), (2, 1), (8, 8), (32, 2), (128, 128), (128, 16), (1024, 64)])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_attend_pages_and_blocks(page, block, dim):
    _check(Scene([(100, 1), (300, 2), (7, 7), (260, 1)], page=page, block=block, dim=dim, layout="head" if page == 8 else "token", seed=page))


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("shared", [1, 16, 40, 64, 333])
def test_attend_shared_prefix(dim, shared):
    seqs = [(shared + 30, 1), (shared + 1, 1), (shared + 200, 1), (shared + 77, 1), (shared, 1)]
    _check(Scene(seqs, groups=[0, 5], shared=[shared], dim=dim, seed=shared))


@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_attend_many_in_a_group(dtype):
    rng = np.random.default_rng(3)
    seqs = [(300 + int(x), 1) for x in rng.integers(1, 60, 70)]
    _check(Scene(seqs, groups=[0, 70], shared=[300], heads=8, kv_heads=2, dim=64, seed=4, dtype=dtype))


def test_attend_groups_side_by_side():
    seqs = [(90, 1), (80, 2), (40, 1), (41, 1), (500, 1), (70, 30), (65, 1)]
    _check(Scene(seqs, groups=[0, 2, 4, 5, 5, 7], shared=[60, 0, 400, 10, 33], dim=128, dtype=FP16, seed=5))


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_attend_long(dim):
    """Items of many tiles, several of them to a sequence."""
    _check(Scene([(9001, 1), (5000, 1)], heads=8, kv_heads=2, dim=dim, page=64, block=32, seed=6))


@pytest.mark.parametrize("low, high", [(100, 127), (127, 150), (60, 61)])
def test_attend_scales_apart(low, high):
    """Blocks of very different magnitudes side by side (bf16 has all of their numbers)."""
    _check(Scene([(200, 1), (77, 3)], dim=128, block=4, low=low, high=high, seed=low), scale=2.0 ** -9 if high < 130 else 2.0 ** -30)


@pytest.mark.parametrize("new", [1, 5])
def test_attend_numbers_that_are_none(new):
    """NaN codes and NaN scales behind what a token sees do not reach it; what it sees makes it NaN."""
    def spoil(which, code, e):
        page = sc0.table[0, 90 // 16]
        code[page, 90 % 16:] = np.nan                       # sequence 0 from its key 90 on
        if which == 1:
            e[sc0.table[1, 3]] = 255                        # sequence 1's values from its key 48 on
    seqs = [(90 + new, new), (60, 1), (33, 1)]
    sc0 = exec_ref.Scene(seqs, seed=11)
    sc = Scene(seqs, seed=11, block=16, spoil=spoil)
    ex = pkg.Executor()
    got = _attend(ex, sc)
    assert np.isnan(got[:new]).all() and np.isnan(got[new]).all() and np.isfinite(got[new + 1]).all()
    pos = sc.pos.copy()
    pos[:new] = 89
    pos[new] = 47
    cache = sc.cache(ex)
    got = _attend(ex, sc, cache=cache, batch=sc.batch(ex, cache, pos=pos))
    limits = [np.arange(int(sc.length[s])) <= p for s, p in zip(sc.seq, pos)]
    want, weighted, top = sc.reference(sc.dim ** -0.5, limits)
    assert (np.abs(got - want) <= attend_tolerance(want, weighted, top, sc.dtype, 95)).all()
    ex.destroy()


def test_attend_rows_that_see_nothing():
    """Padding, sequences without keys, pages that are not there: zeros."""
    sc = Scene([(40, 1), (0, 0), (70, 2), (20, 1)], seed=12)
    ex = pkg.Executor()
    cache = sc.cache(ex)
    table = sc.table.copy()
    table[3] = [-1, 10 ** 6] + [-1] * (table.shape[1] - 2)
    pos = sc.pos.copy()
    pos[0] = -1
    got = _attend(ex, sc, cache=cache, batch=sc.batch(ex, cache, pos=pos, table=table))
    assert (got[0] == 0).all() and (got[3] == 0).all()
    want, weighted, top = sc.reference(sc.dim ** -0.5)
    assert (np.abs(got - want) <= attend_tolerance(want, weighted, top, sc.dtype, 70))[1:3].all()
    ex.destroy()


def test_attend_as_over_numbers():
    """The same as over a cache of 16 bits with the same numbers, up to the order of sums (two results, each within its tolerance)."""
    sc = Scene([(700, 1), (90, 4), (333, 1)], groups=[0, 3], shared=[50], seed=13, dim=128)
    ex = pkg.Executor()
    cache = sc.cache(ex)
    batch = sc.batch(ex, cache)
    got = _attend(ex, sc, cache=cache, batch=batch)
    pools = [torch.from_numpy(numbers(c, np.repeat(e, sc.block, axis=1)[..., None], BF16)).to(BF16).cuda() for c, e in zip(sc.code, sc.e)]
    wide = ex.cache(*pools)
    out = torch.empty((sc.n, sc.heads, sc.dim), dtype=BF16, device="cuda")
    ex.attend(wide, batch, sc.q, out)      # (the batch and its plan go with caches of either width)
    want, weighted, top = sc.reference(sc.dim ** -0.5)
    assert (np.abs(got - out.double().cpu().numpy()) <= 2 * attend_tolerance(want, weighted, top, BF16, 700)).all()
    ex.destroy()


def test_attend_is_reproducible():
    sc = Scene([(700, 1), (90, 4), (3000, 1)], seed=14, dim=128)
    ex = pkg.Executor()
    first = _attend(ex, sc)
    for _ in range(3):
        assert np.array_equal(_attend(ex, sc), first)
    ex.destroy()


# ---- together ---------------------------------------------------------------------------------------------------

def test_steps_in_a_graph():
    """Append and attend of a step, recorded once and replayed with other numbers, positions and lengths; beside eager work."""
    ex = pkg.Executor()
    rng = np.random.default_rng(15)
    S, H, kv, D, P, B, steps = 3, 4, 2, 64, 16, 8, 40
    table = rng.permutation(S * 4).reshape(S, 4)
    def make():
        c = Cache(S * 4, kv, D, P, B, seed=15)
        return c, c.on(ex)
    (c1, cache1), (c2, cache2) = make(), make()
    pos, length = i32(np.zeros(S)), i32(np.ones(S))
    batch = ex.batch(cache1, H, token_seq=i32(np.arange(S)), token_pos=pos, seq_start=i32(np.arange(S + 1)), seq_len=length, page_table=i32(table))
    ex.reserve(cache1, batch)
    qkv = torch.zeros((S, H + 2 * kv, D), dtype=BF16, device="cuda")
    out = torch.zeros((S, H, D), dtype=BF16, device="cuda")
    freq = torch.from_numpy(10000.0 ** (-np.arange(D // 2) / (D // 2))).cuda()
    def step(cache):
        ex.plan(batch)
        ex.append(cache, batch, qkv[:, :H], qkv[:, H:H + kv], qkv[:, H + kv:], qkv[:, :H], freq)
        ex.attend(cache, batch, qkv[:, :H], out)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(cache1)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(cache1)
    for t in range(steps):
        x = torch.from_numpy(rng.standard_normal((S, H + 2 * kv, D)) * np.exp(rng.standard_normal((S, 1, 1)))).to(BF16).cuda()
        pos.fill_(t)
        length.fill_(t + 1)
        qkv.copy_(x)
        g.replay()
        got = out.clone()
        qkv.copy_(x)
        step(cache2)
        torch.cuda.synchronize()
        assert torch.equal(got, out), t
        for i in range(2):
            # (the first block of the recording's own run is begun again)
            assert torch.equal(c1.pools[i].view(torch.uint8), c2.pools[i].view(torch.uint8)) and \
                torch.equal(c1.scales[i].view(torch.uint8), c2.scales[i].view(torch.uint8)), t
    ex.destroy()


def test_on_another_stream():
    sc = Scene([(700, 1), (90, 4)], seed=16, dim=128)
    ex = pkg.Executor()
    want = _attend(ex, sc)
    cache = sc.cache(ex)
    batch = sc.batch(ex, cache)
    out = torch.zeros((sc.n, sc.heads, sc.dim), dtype=sc.dtype, device="cuda")
    k = torch.zeros((sc.n, sc.kv_heads, sc.dim), dtype=sc.dtype, device="cuda")
    v = torch.zeros_like(k)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ex.plan(batch, stream=side)
    ex.attend(cache, batch, sc.q, out, stream=side)
    ex.read(cache, batch, k, v, stream=side)
    side.synchronize()
    assert np.array_equal(out.double().cpu().numpy(), want)
    own = np.concatenate([sc.full[0][s][n - m:] for s, (n, m) in enumerate(zip(sc.length, sc.new))])
    assert np.array_equal(k.double().cpu().numpy(), own)
    ex.destroy()
