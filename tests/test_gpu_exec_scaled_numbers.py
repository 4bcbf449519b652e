"""What a cache of 8 bits keeps of its numbers: sines and cosines on the way in, weights and infinite values on the way out."""
import numpy as np
import pytest
import torch

import paper_1905_13348_amd as pkg
from scaled_ref import Scene

pytestmark = pytest.mark.gpu

i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()
BF16, FP16 = torch.bfloat16, torch.float16


def last_place(x):
    return np.exp2(np.floor(np.log2(np.abs(x))) - 23)


@pytest.mark.parametrize("interleaved", [False, True])
def test_sines_and_cosines(interleaved):
    """Pairs (a, b) of powers of two that an angle turns to next to nothing: a cos t - b sin t, of which the products are exact in 32
    bits, shows the errors of sine and cosine a thousand times larger than the rounding to fp16.  These are 0.6 of a last place of the
    cosine and 0.76 of the sine where the angle is an eighth of a turn at most, and the other way round in every other quarter, so
    0.76 of either; the difference is rounded once to 32 bits and once to fp16, and an angle in 64 bits is off by three roundings."""
    rng = np.random.default_rng(1)
    ex = pkg.Executor()
    pools = [torch.zeros((1, 16, 1, 256), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2)]
    scales = [torch.zeros((1, 1, 1), dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu) for _ in range(2)]
    cache = ex.cache(*pools, k_scale=scales[0], v_scale=scales[1], dtype=FP16)
    worst = 0.0
    for call in range(24):
        pos = (1, 3, 11)[call % 3]
        j, quarter = rng.integers(-5, 6, 128), rng.integers(0, 200, 128)
        off = np.exp(rng.uniform(np.log(1e-7), np.log(3e-5), 128)) * rng.choice((-1, 1), 128)
        freq = (np.arctan(2.0 ** j) + quarter * (np.pi / 2) + off) / pos
        t = np.longdouble(pos) * freq.astype(np.longdouble)
        cos, sin = np.cos(t), np.sin(t)
        # a / b is near the tangent, a power of two
        tangent = np.sign(sin * cos) * np.where(quarter % 2 == 0, 2.0 ** j, 2.0 ** -j)
        b = np.where(np.abs(tangent) > 1, 1024 / np.abs(tangent), 1024.0).astype(np.float64)
        a = (b * tangent).astype(np.float64)
        q = np.zeros((1, 1, 256))
        first, second = (slice(0, 256, 2), slice(1, 256, 2)) if interleaved else (slice(0, 128), slice(128, 256))
        q[0, 0, first], q[0, 0, second] = a, b
        dev = torch.from_numpy(q).to(FP16).cuda()
        assert np.array_equal(dev.double().cpu().numpy(), q)
        kv = torch.zeros((1, 1, 256), dtype=FP16, device="cuda")
        out = torch.empty_like(dev)
        batch = ex.batch(cache, 1, token_seq=i32([0]), token_pos=i32([pos]), seq_start=i32([0, 1]), seq_len=i32([pos + 1]), page_table=i32([[0]]))
        ex.append(cache, batch, dev, kv, kv, out, torch.from_numpy(freq).cuda(), interleaved=interleaved)
        got = out.double().cpu().numpy()[0, 0, first]
        want = (a * cos - b * sin).astype(np.float64)
        assert (np.abs(want) < 0.1).all()
        tol = 0.76 * (np.abs(a) * last_place(cos.astype(np.float64)) + np.abs(b) * last_place(sin.astype(np.float64)))
        tol = tol + np.abs(want) * (2.0 ** -11 + 2.0 ** -24) * 1.01 + 2.0 ** -25 + 2048 * 3 * t.astype(np.float64) * 2.0 ** -53
        worst = max(worst, float((np.abs(got - want) / tol).max()))
    assert worst <= 1, worst
    ex.destroy()


@pytest.mark.parametrize("dim, heads, new", [(64, 2, 1), (64, 8, 1), (64, 64, 1), (128, 2, 1), (128, 8, 1), (128, 32, 2), (256, 2, 1), (256, 32, 1)])
@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_weights_keep_their_bits(dim, heads, new, dtype):
    """Up to 32 rows (16 of 256 dimensions) to a KV head.  A query has one dimension, so that scores are exact; of n keys, relative to
    sum p |v|: what is left of a weight behind its two numbers (half a step of half a step), two sums of n in 32 bits, of the exponent
    16 and of its power, the division and the joining 8 roundings; and half a step of the result, and of fp16 weights below
    their normal range 2^-25 where the greatest is 2^7 at least."""
    seqs = [(n, min(n, new)) for n in (1, 2, 3, 4, 5, 6, 7, 8, 8, 9, 20, 33, 64)]
    sc = Scene(seqs, heads=heads, kv_heads=2, dim=dim, dtype=dtype, block=4, low=119, high=121, seed=dim + heads)
    rng = np.random.default_rng(2)
    sc.q_host = np.where(np.arange(dim) == rng.integers(0, dim, (sc.n, heads))[..., None], rng.choice((-4.0, 4.0, 2.0), (sc.n, heads, 1)), 0.0)
    sc.q = torch.from_numpy(sc.q_host).to(dtype).cuda()
    ex = pkg.Executor()
    cache = sc.cache(ex)
    batch = sc.batch(ex, cache)
    out = torch.empty((sc.n, heads, dim), dtype=dtype, device="cuda")
    ex.plan(batch)
    ex.attend(cache, batch, sc.q, out, 0.25)
    want, weighted, top = sc.reference(0.25)
    half = torch.finfo(dtype).eps / 2
    n = sc.length[sc.seq][:, None, None]
    tol = half * np.abs(want) + (half ** 2 + (2 * n + 24) * 2.0 ** -24) * weighted + n * 2.0 ** -32 * top
    off = np.abs(out.double().cpu().numpy() - want)
    assert (off <= tol).all(), (int((off > tol).sum()), off.size, float((off / tol).max()))
    ex.destroy()


@pytest.mark.parametrize("new", [1, 3, 40])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype, e", [(FP16, 135), (FP16, 140), (BF16, 247), (BF16, 250)])
def test_infinite_values(new, dim, dtype, e):
    """Codes that are infinite as numbers of the type, with signs: what sees them is infinite, or NaN where both signs meet; what does not
    see them is as without, whether all rows of an item see them or some.  (In bf16 beside zeros: sums of weights times values of 2^120
    and more end beyond 32 bits.)"""
    seqs = [(300, new), (45, min(new, 45)), (70, 1)]

    def spoil(which, code, scale):
        if which == 1:
            scale[sc0.table[0, 3], 0, 0] = e           # sequence 0's keys 48 to 55 of head 0
            scale[sc0.table[0, 18], 1, 1] = e          # 296 to 299 of head 1
            scale[sc0.table[1, 2], 1, 0] = e           # sequence 1's 40 to 44
            code[sc0.table[0, 3], :, 0, :dim // 4] = np.abs(code[sc0.table[0, 3], :, 0, :dim // 4])
            if dtype == BF16:
                high = np.repeat(scale, 8, axis=1)[..., None] == e
                code[:] = np.where(high & (np.abs(code) * 2.0 ** (e - 247) < 256), 0, code)

    sc0 = Scene(seqs, dim=dim, dtype=dtype, block=8, seed=21)
    sc = Scene(seqs, dim=dim, dtype=dtype, block=8, seed=21, spoil=spoil)
    ex = pkg.Executor()
    cache = sc.cache(ex)
    batch = sc.batch(ex, cache)
    out = torch.empty((sc.n, sc.heads, dim), dtype=dtype, device="cuda")
    ex.plan(batch)
    ex.attend(cache, batch, sc.q, out)
    got = out.double().cpu().numpy()
    with np.errstate(invalid="ignore"):
        want, weighted, top = sc.reference(dim ** -0.5)
        # (the result is of the type, too)
        want_t = torch.from_numpy(want).to(dtype).double().numpy()
    assert np.isinf(want).any() and np.isnan(want).any() and np.isfinite(want).any()
    assert np.array_equal(np.isnan(got), np.isnan(want))
    infinite = np.isinf(want)
    assert np.array_equal(got[infinite], want[infinite])
    finite = np.isfinite(want) & np.isfinite(want_t)
    half = torch.finfo(dtype).eps / 2
    with np.errstate(invalid="ignore"):
        tol = half * np.abs(want) + (half + 2.0 ** -11) * weighted + (300 * 2.0 ** -25 * top if dtype == FP16 else 0) + 1e-30
        assert (np.abs(got - want) <= tol)[finite].all()
    ex.destroy()
