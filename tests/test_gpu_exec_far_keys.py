"""Keys numbered up to what 32 bits hold: every loop over them ends, and what is counted is what the header says."""
import numpy as np
import pytest
import torch

import exec_history
from exec_history import i32
import paper_1905_13348_amd as pkg

pytestmark = pytest.mark.gpu

PAGE, WIDTH, MOST = 1 << 16, 1 << 15, 2 ** 31 - 256


def _sparse(ex, dim, tokens, pos):
    """One sequence of 2^31 - 1 keys, of which only those on its first and last page are there; the keys from 2^31 - 256 on
    are NaN."""
    pools = [torch.randn((2, PAGE, 1, dim), generator=torch.Generator().manual_seed(i)).to(torch.bfloat16).cuda() for i in (1, 2)]
    for p in pools:
        p[1, PAGE - 256:] = torch.nan
    table = np.full((1, WIDTH), -1)
    table[0, 0], table[0, -1] = 0, 1
    cache = ex.cache(*pools)
    batch = ex.batch(cache, 2, token_seq=i32([0] * tokens), token_pos=i32(pos), seq_start=i32([0, tokens]), seq_len=i32([2 ** 31 - 1]),
                     page_table=i32(table))
    return pools, cache, batch


@pytest.mark.parametrize("dim", [64, 256])
def test_a_sequence_of_all_keys(dim):
    ex = pkg.Executor()
    pos = [2 ** 31 - 1, MOST, MOST - 1, 2 ** 31 - PAGE - 1, 7]
    pools, cache, batch = _sparse(ex, dim, len(pos), pos)
    q = torch.randn((len(pos), 2, dim), generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).cuda()
    got = exec_history.attend(ex, cache, batch, q, 0.1)
    header, items = exec_history.plan_of(batch)
    assert items[:, 3].max() == MOST
    k, v = (p.view(2 * PAGE, dim).double() for p in pools)
    for t, seen in enumerate((2 * PAGE - 256, 2 * PAGE - 256, 2 * PAGE - 256, PAGE, 8)):
        w = torch.softmax(torch.mm(q[t].double(), k[:seen].t().contiguous()) * 0.1, dim=1)
        want, weighted = (torch.mm(w, x).cpu().numpy() for x in (v[:seen], v[:seen].abs()))
        tol = exec_history.tolerance(want, weighted, torch.bfloat16, seen, 6.0)
        assert (np.abs(got[t] - want) <= tol).all(), t
    ex.destroy()


def test_keys_that_far_are_written_up_to_the_same_border():
    ex = pkg.Executor()
    pos = [MOST - 1, MOST, 2 ** 31 - 1, 0]
    pools, cache, batch = _sparse(ex, 64, 4, pos)
    before = [p.clone() for p in pools]
    k, v = (torch.randn((4, 1, 64), generator=torch.Generator().manual_seed(i)).to(torch.bfloat16).cuda() for i in (4, 5))
    ex.append(cache, batch, None, k, v, None)
    torch.cuda.synchronize()
    for pool, old, new in zip(pools, before, (k, v)):
        old[1, PAGE - 257], old[0, 0] = new[0], new[3]
        assert torch.equal(pool.nan_to_num(9), old.nan_to_num(9))
    ex.destroy()
