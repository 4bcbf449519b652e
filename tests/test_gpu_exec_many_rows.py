"""Batches whose rows are more than a launch's grid can hold."""
import numpy as np
import pytest
import torch

import exec_history
import paper_1905_13348_amd as pkg

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [(1 << 16) - 1, (1 << 16) + 1, (1 << 22) + 5])
def test_draws_of_many_rows(rows):
    """A workgroup of 1024 threads to a row: 2^22 rows are 2^32 threads.  Three tokens to a row; the second or, by the row's
    number, the third has all the weight."""
    logits = torch.full((rows, 3), -200.0, device="cuda")
    which = 1 + torch.arange(rows, device="cuda") % 2
    logits.scatter_(1, which[:, None], 0.0)
    token = torch.full((rows,), -9, dtype=torch.int32, device="cuda")
    prob = torch.zeros(rows, device="cuda")
    ex = pkg.Executor()
    ex.sample(logits, torch.full((rows,), 0.5, device="cuda"), token, prob)
    torch.cuda.synchronize()
    ex.destroy()
    assert torch.equal(token.long(), which) and bool((prob == 1).all())


def test_attention_of_many_rows():
    """8200 tokens of 128 heads behind a short prefix: 1,049,600 rows to merge, more than 65,536 workgroups of 16."""
    tokens, heads, dim, dtype = 8_200, 128, 64, torch.bfloat16
    normal = lambda shape, seed: torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()
    h = exec_history.History(normal((40, 1, dim), 1), normal((40, 1, dim), 2))
    q = normal((tokens, heads, dim), 3)
    length = 1 + np.arange(tokens) % 40
    ex = pkg.Executor()
    cache = ex.cache(*h.pools)
    batch, limit = h.batch(ex, cache, heads, length, shared=7)
    got = exec_history.attend(ex, cache, batch, q, 0.125)
    ex.destroy()
    want, weighted = h.reference(q, limit, 0.125)
    assert (np.abs(got - want) <= exec_history.tolerance(want, weighted, dtype, 40, 6.0)).all()
