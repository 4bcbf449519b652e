"""Batches whose rows are more than a launch's grid can hold."""
import pytest
import torch

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
