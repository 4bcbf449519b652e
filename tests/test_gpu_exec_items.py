"""Attention by what a plan makes of a batch: items of several tiles, more items than workgroups, many rows to merge, prompts
of thousands of tokens.  Each test asserts from the plan that it has what it is there for."""
import numpy as np
import pytest
import torch

import exec_history
from exec_history import History, tolerance
import paper_1905_13348_amd as pkg

pytestmark = pytest.mark.gpu

DTYPES = [torch.bfloat16, torch.float16]


def _normal(shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def _check(h, q, scale, length, **kw):
    ex = pkg.Executor()
    cache = ex.cache(*h.pools)
    batch, limit = h.batch(ex, cache, q.shape[1], length, **kw)
    got = exec_history.attend(ex, cache, batch, q, scale)
    header, items = exec_history.plan_of(batch)
    ex.destroy()
    want, weighted = h.reference(q, limit, scale, kw.get("missing", ()))
    top = float(h.v.double().abs().nan_to_num(0, 0, 0).max())
    fine = np.isfinite(want)
    assert np.array_equal(got[~fine], want[~fine], equal_nan=True)
    tol = tolerance(np.nan_to_num(want), weighted, q.dtype, int(np.max(limit)), top)
    bad = np.abs(got[fine] - want[fine]) > tol[fine]
    assert not bad.any(), (bad.sum(), bad.size, np.argwhere(~(np.abs(np.nan_to_num(got) - np.nan_to_num(want)) <= tol))[:4])
    return header, items, fine


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("keys, chunk", [(1_000, 192), (2_000, 320)])
@pytest.mark.parametrize("what", ["plain", "rising", "falling", "missing", "odd"])
def test_items_of_several_tiles(what, keys, chunk, dim, dtype):
    """40 ragged sequences: an item is three tiles or five (six or ten of 32 keys), so both of its buffers and all four slots of
    the lookup are used and used again, the end is ragged, and the maximum moves on within an item (by some 60 halvings over
    the keys, up or down)."""
    rng = np.random.default_rng(keys + dim)
    S, new = 40, 3 if what == "odd" else 1
    length = rng.integers(int(0.7 * keys), keys + 1, S)
    length[3], length[7] = keys, keys - 1
    k, v = _normal((keys, 2, dim), dtype, 1), _normal((keys, 2, dim), dtype, 2)
    q = _normal((S * new, 6, dim), dtype, 3)
    scale = dim ** -0.5
    kw = {}
    if what in ("rising", "falling"):
        ramp = torch.linspace(0, 40, keys).cuda()[:, None]
        q[:, :, 0] = 1
        k[:, :, 0] = ((ramp if what == "rising" else 40 - ramp) / scale).to(dtype)
    elif what == "missing":
        kw["missing"] = (0, 5, 6, 7, 8, 9, 10, 23, 24, 40, keys // 16 - 3)
    elif what == "odd":
        kw["new"] = [new] * S
        for i, s in enumerate((0, 3, 5, 7)):      # (the last keys of some, so that their tokens differ in what they see)
            v[int(length[s]) - 1 - i % 2, i % 2, 3 * i] = (np.inf, -np.inf, np.nan, np.inf)[i]
    header, items, fine = _check(History(k, v), q, scale, length, **kw)
    sizes = items[:, 3] - items[:, 2]
    assert sizes.max() == chunk and chunk > 2 * (32 if dim == 256 else 64)
    assert len(set(sizes.tolist())) > 5 and (what != "odd" or not fine.all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("S", [992, 993])
def test_many_rows_to_merge(S, dim, dtype):
    """33 query heads on one KV head and 992 or 993 tokens: 32,736 and 32,769 rows, on both sides of where the merge takes
    several rows to a workgroup (and no multiple of how many).  Some tokens behind prefixes, some with one part of their own (so
    nothing to merge), some with several."""
    rng = np.random.default_rng(S + dim)
    keys = 2_000
    length = rng.integers(1, 300, S)
    length[rng.choice(S, 20, replace=False)] = rng.integers(1_500, keys + 1, 20)
    k, v = _normal((keys, 1, dim), dtype, 4), _normal((keys, 1, dim), dtype, 5)
    q = _normal((S, 33, dim), dtype, 6)
    pos = length - 1
    pos[5::97] = -1
    header, items, _ = _check(History(k, v), q, dim ** -0.5, length, pos=pos, groups=[0, 300, 301, 500], shared=[100, 40, 250])
    own = items[items[:, 2] > 0]
    assert (items[:, 6] == -1).sum() > 200 and len(own) > 50


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_more_items_than_workgroups(dim, dtype):
    """300 short sequences of 8 KV heads: workgroups take a second item, and behind one from which values that are no numbers were
    taken out an ordinary one."""
    rng = np.random.default_rng(dim)
    S, keys = 300, 90
    length = rng.integers(3, keys + 1, S)
    new = rng.integers(1, 4, S)
    k, v = _normal((keys, 8, dim), dtype, 7), _normal((keys, 8, dim), dtype, 8)
    for i in range(8):
        v[40 + 5 * i, i, 7 * i] = (np.inf, -np.inf, np.nan)[i % 3]
    header, items, fine = _check(History(k, v), _normal((int(new.sum()), 8, dim), dtype, 9), dim ** -0.5, length, new=new)
    starts = header[12:30].reshape(2, 9)
    assert np.diff(starts, axis=1).sum(axis=0).min() > 2048 // 8 + 1 and len(items) > 2100
    assert fine.mean() > 0.9 and not fine.all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dim, heads, kv", [(64, 32, 8), (128, 16, 2), (256, 8, 8)])
@pytest.mark.parametrize("new", [[2_000], [700, 1_100, 64, 513]])
def test_prompts_alone(new, dim, heads, kv, dtype):
    """Prompts without anything in front of them: several parts to a tile of tokens, of which early tokens see only the first."""
    keys = max(new)
    k, v = _normal((keys, kv, dim), dtype, 10), _normal((keys, kv, dim), dtype, 11)
    header, items, _ = _check(History(k, v), _normal((sum(new), heads, dim), dtype, 12), dim ** -0.5, new, new=new)
    per_tile = 128 // (heads // kv)
    tiles = [items[(items[:, 5] == 0) & (items[:, 0] == t)] for t in range(0, new[0], per_tile)]
    assert all(len(t) == len(tiles[0]) for t in tiles) and len(tiles[0]) > 1 and len(tiles) > 2


@pytest.mark.parametrize("dtype", DTYPES)
def test_prompts_that_go_on(dtype):
    """Chunks of 600 tokens of prompts that are partly in the cache, with pages missing and values that are no numbers."""
    keys = 1_500
    k, v = _normal((keys, 4, 128), dtype, 13), _normal((keys, 4, 128), dtype, 14)
    v[1_000, 0, 5], v[1_203, 1, 6], v[1_499, 3, 127], v[30, 2, 1] = np.inf, np.nan, -np.inf, np.inf
    new, length = [600, 300], [1_500, 1_205]
    header, items, fine = _check(History(k, v, page=64), _normal((900, 8, 128), dtype, 15), 0.09, length, new=new, missing=(2, 17, 18))
    assert not fine.all()
