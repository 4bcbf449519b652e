"""Attention where numbers end: keys that are no numbers and are seen, scores of minus infinity, scores beyond what 32 bits
tell apart, weights below the normal range of fp16, rows that see nothing beside rows that do."""
import numpy as np
import pytest
import torch

import exec_history
from exec_history import History, tolerance
import paper_1905_13348_amd as pkg

pytestmark = pytest.mark.gpu


def _normal(shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def _run(h, q, scale, length, raised=0, **kw):
    """(result, the definition's, tolerance, items)"""
    ex = pkg.Executor()
    cache = ex.cache(*h.pools)
    batch, limit = h.batch(ex, cache, q.shape[1], length, **kw)
    got = exec_history.attend(ex, cache, batch, q, scale)
    items = exec_history.plan_of(batch)[1]
    ex.destroy()
    want, weighted = h.reference(q, limit, scale, kw.get("missing", ()))
    top = float(torch.nan_to_num(h.v.double().abs(), 0, 0, 0).max())
    return got, want, tolerance(np.nan_to_num(want), np.nan_to_num(weighted), q.dtype, int(np.max(limit)), top, raised), items


@pytest.mark.parametrize("keys", [slice(0, 64), slice(64, 128), slice(960, 1000), slice(70, 71), slice(0, 1000), slice(130, 260)])
@pytest.mark.parametrize("shared", [None, 64, 200])
def test_keys_that_are_no_numbers_and_are_seen(keys, shared):
    """The result of every row that sees them is NaN, wherever the plan cuts (into items of a tile here, so that whole items
    have no score that is a number) and in whichever order the parts are joined; other heads' are as ever."""
    dtype = torch.bfloat16
    k, v = _normal((1000, 2, 64), dtype, 1), _normal((1000, 2, 64), dtype, 2)
    k[keys, 1, 5] = torch.nan
    q = _normal((3, 4, 64), dtype, 3)
    got, want, tol, items = _run(History(k, v), q, 0.125, [1000, 990, 40], shared=shared)
    seen = [keys.start < n for n in (1000, 990, 40)]
    for t in range(3):
        assert np.isnan(want[t, 2:]).all() == seen[t]
        assert np.isnan(got[t, 2:]).all() == seen[t], t
    fine = np.isfinite(want)
    assert (np.abs(got[fine] - want[fine]) <= tol[fine]).all() and (items[:, 3] - items[:, 2]).max() == 64


def test_keys_that_are_no_numbers_in_one_item():
    """The same where nothing is split."""
    dtype = torch.float16
    k, v = _normal((60, 1, 128), dtype, 4), _normal((60, 1, 128), dtype, 5)
    k[:30, 0, 0] = torch.nan
    got, want, tol, items = _run(History(k, v), _normal((2, 2, 128), dtype, 6), 0.1, [60, 20])
    assert len(items) == 2 and np.isnan(got).all() and np.isnan(want).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("shared", [None, 64])
@pytest.mark.parametrize("which", ["all", "first", "last", "one", "prefix"])
def test_scores_of_minus_infinity(which, shared, dtype):
    """Keys that take every score to minus infinity: weights of 0 beside others, NaN (0 by 0) where a row sees nothing else;
    not the zeros of a row that sees no key."""
    k, v = _normal((500, 2, 64), dtype, 7), _normal((500, 2, 64), dtype, 8)
    q = _normal((5, 4, 64), dtype, 9)
    q[:, :, 0] = 1
    cut = {"all": slice(0, 500), "first": slice(0, 64), "last": slice(448, 500), "one": slice(0, 1), "prefix": slice(0, 200)}[which]
    k[cut, :, 0] = -torch.inf
    length = [500, 300, 64, 1, 200]
    got, want, tol, _ = _run(History(k, v), q, 0.125, length, shared=shared)
    for t, n in enumerate(length):
        only = cut.start == 0 and n <= cut.stop
        assert np.isnan(want[t]).all() == only
        assert np.isnan(got[t]).all() == only, t
    fine = np.isfinite(want)
    assert (np.abs(got[fine] - want[fine]) <= tol[fine]).all()


def test_scores_of_minus_infinity_on_pages_that_are_not_there():
    """Keys on missing pages are not seen: a row that sees none beside them has zeros, a row that sees one of minus infinity
    has NaN."""
    k, v = _normal((320, 1, 64), torch.bfloat16, 10), _normal((320, 1, 64), torch.bfloat16, 11)
    k[:, :, 0] = -torch.inf
    q = torch.ones((4, 2, 64), dtype=torch.bfloat16, device="cuda")
    h = History(k, v)
    got, want, _, _ = _run(h, q, 0.125, [32, 33, 320, 5], missing=(0, 1))
    assert (got[[0, 3]] == 0).all() and (want[[0, 3]] == 0).all()
    assert np.isnan(got[[1, 2]]).all() and np.isnan(want[[1, 2]]).all()


@pytest.mark.parametrize("new", [3, 100])
def test_a_prompt_whose_first_key_takes_scores_to_minus_infinity(new):
    """The first token sees nothing else: NaN; the second has the second value."""
    k, v = _normal((new, 1, 128), torch.float16, 12), _normal((new, 1, 128), torch.float16, 13)
    q = _normal((new, 3, 128), torch.float16, 14)
    q[:, :, 7] = 0.5
    k[0, 0, 7] = -torch.inf
    got, want, tol, _ = _run(History(k, v), q, 0.1, [new], new=[new])
    assert np.isnan(got[0]).all() and np.isnan(want[0]).all()
    assert np.array_equal(got[1], np.broadcast_to(v[1].double().cpu().numpy(), got[1].shape))
    assert (np.abs(got - want)[1:] <= tol[1:]).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("S", [3, 512])
def test_scores_beyond_32_bits(S, dim, dtype):
    """Scores of 2^5 to 2^40 of either sign, further apart than they are rounded: the greatest takes all, at every size.
    (S = 512: an item has the whole history, so that its maximum moves from tile to tile.)"""
    rng = np.random.default_rng(dim)
    keys = 400
    # every row's scores are its factor times the keys', which are 1% apart, in no order
    level = np.linspace(0.02, 1, keys) * rng.choice([-1, 1])
    level = torch.from_numpy(rng.permutation(level) * (60000.0 if dtype == torch.float16 else 3e5)).to(dtype)
    assert len(set(level.tolist())) > 100
    k = level.cuda()[:, None, None].expand(keys, 1, dim).contiguous()
    v = _normal((keys, 1, dim), dtype, 15)
    q = torch.from_numpy(np.exp(rng.uniform(np.log(1e-3), np.log(6e4), S)) * rng.choice([-1, 1], S)).to(dtype).cuda()
    q = q[:, None, None].expand(S, 2, dim).contiguous()
    scale = 0.3
    got, want, tol, items = _run(History(k, v), q, scale, [keys] * S)
    # the oracle's own weights are exact at these scores: some rows' greatest is there twice or more (rounded levels)
    assert np.isfinite(want).all()
    steps = torch.mm(q[:, 0, :1].double(), level.double().cuda()[None, :]) * dim * scale
    two = torch.topk(torch.unique(level.double()).cuda()[None, :] * q[:, 0, :1].double() * dim * scale, 2, dim=1).values
    # 32 bits err by dim * 2^-24 of the score in the sum, and the next score is further away than that and 20 more
    clear = (two[:, 0] - two[:, 1] > 20 + dim * 2.0 ** -23 * steps.abs().amax(dim=1)).cpu().numpy()
    assert clear.sum() >= S // 3
    bad = ~(np.abs(got - want) <= tol)[clear]
    assert not bad.any(), (bad.sum(), bad.size, got[clear][bad][:4], want[clear][bad][:4])
    if S == 512:
        assert (items[:, 3] - items[:, 2]).min() == keys


def test_small_weights_in_fp16():
    """One key 25.5 halvings above 131,071 others: together these have 0.28% of the weight, each of them 2^-25.5.  (512
    sequences of one history: an item has all of it.)"""
    keys, S = 131_072, 512
    k = torch.zeros((keys, 1, 64), dtype=torch.float16, device="cuda")
    v = torch.ones((keys, 1, 64), dtype=torch.float16, device="cuda")
    k[0, 0, 0], v[0] = 1, 0
    q = torch.zeros((S, 1, 64), dtype=torch.float16, device="cuda")
    q[:, 0, 0] = 1
    ex = pkg.Executor()
    h = History(k, v, page=1024)
    cache = ex.cache(*h.pools)
    batch, _ = h.batch(ex, cache, 1, [keys] * S)
    got = exec_history.attend(ex, cache, batch, q, 25.5 * float(np.log(2)))
    items = exec_history.plan_of(batch)[1]
    ex.destroy()
    assert (items[:, 3] - items[:, 2]).min() > keys // 2
    rest = (keys - 1) * 2.0 ** -25.5
    want = np.full(got.shape, rest / (1 + rest))
    tol = tolerance(want, want, torch.float16, keys, 1.0, raised=7)
    assert (np.abs(got - want) <= tol).all(), (got.min(), got.max(), want[0, 0, 0])


def _time(f, n=5):
    """Least of some calls, us."""
    f()
    best = 1e30
    for _ in range(n):
        a, b = torch.cuda.Event(True), torch.cuda.Event(True)
        a.record()
        f()
        b.record()
        b.synchronize()
        best = min(best, a.elapsed_time(b) * 1e3)
    return best


@pytest.mark.parametrize("odd", [False, True])
def test_padding_beside_rows_that_see_a_prefix(odd):
    """A token of padding in a group: its own result is zeros, also where what the others see is no number, and the others'
    tiles take the time that they take without it (within twice)."""
    S, keys = 64, 16_384
    k, v = _normal((keys, 2, 128), torch.bfloat16, 16), _normal((keys, 2, 128), torch.bfloat16, 17)
    if odd:
        v[11, 0, 3], v[5_000, 1, 4] = torch.inf, torch.nan
    q = _normal((S, 8, 128), torch.bfloat16, 18)
    h = History(k, v)
    ex = pkg.Executor()
    cache = ex.cache(*h.pools)
    length = [keys] * S
    pos = np.full(S, keys - 1)
    batch, limit = h.batch(ex, cache, 8, length, shared=keys - 100, pos=pos)
    pos[9] = -1
    padded, padded_limit = h.batch(ex, cache, 8, length, shared=keys - 100, pos=pos)
    for b, lim in ((batch, limit), (padded, padded_limit)):
        got = exec_history.attend(ex, cache, b, q, 0.1)
        want, weighted = h.reference(q, lim, 0.1)
        fine = np.isfinite(want)
        assert np.array_equal(got[~fine], want[~fine], equal_nan=True)
        tol = tolerance(np.nan_to_num(want), weighted, torch.bfloat16, keys, 8.0)
        assert (np.abs(got[fine] - want[fine]) <= tol[fine]).all()
    assert (got[9] == 0).all()
    out = torch.empty_like(q)
    times = []
    for b in (batch, padded):
        ex.plan(b)
        times.append(_time(lambda: ex.attend(cache, b, q, out, 0.1)))
    ex.destroy()
    print(times)
    assert times[1] <= 2 * times[0], times


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_rows_that_see_nothing_of_an_item(dim):
    """Sequences that end inside their group's prefix, and padding, beside others, with values that are no numbers behind
    the end: each row has what it has alone."""
    keys = 700
    k, v = _normal((keys, 1, dim), torch.float16, 19), _normal((keys, 1, dim), torch.float16, 20)
    k[600, 0, 1], v[300, 0, 2], v[650, 0, 3] = torch.nan, torch.inf, torch.nan
    q = _normal((9, 2, dim), torch.float16, 21)
    length = [700, 64, 1, 300, 301, 128, 129, 599, 600]
    pos = [699, 63, 0, 299, 300, -1, 128, 598, 599]
    got, want, tol, _ = _run(History(k, v), q, 0.1, length, pos=pos, shared=650)
    ex = pkg.Executor()
    h = History(k, v)
    cache = ex.cache(*h.pools)
    for t, n in enumerate(length):
        if pos[t] < 0:
            assert (got[t] == 0).all()
            continue
        one, _ = h.batch(ex, cache, 2, [n])
        alone = exec_history.attend(ex, cache, one, q[t:t + 1], 0.1)[0]
        fine = np.isfinite(want[t])
        for x in (got[t], alone):
            assert np.array_equal(x[~fine], want[t][~fine], equal_nan=True), t
            assert (np.abs(x[fine] - want[t][fine]) <= tol[t][fine]).all(), t
    ex.destroy()
