"""Attention where numbers end."""
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
    assert (np.abs(got - want)[fine] <= tol[fine]).all() and (items[:, 3] - items[:, 2]).max() == 64


def test_keys_that_are_no_numbers_in_one_item():
    """The same where nothing is split."""
    dtype = torch.float16
    k, v = _normal((60, 1, 128), dtype, 4), _normal((60, 1, 128), dtype, 5)
    k[:30, 0, 0] = torch.nan
    got, want, tol, items = _run(History(k, v), _normal((2, 2, 128), dtype, 6), 0.1, [60, 20])
    assert len(items) == 2 and np.isnan(got).all() and np.isnan(want).all()
