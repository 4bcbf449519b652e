"""A cache of 8 bits with keys numbered up to what 32 bits hold, and pools beyond 2^31 elements."""
import numpy as np
import pytest
import torch

import exec_history
from exec_history import i32
import paper_1905_13348_amd as pkg
import scaled_ref

pytestmark = pytest.mark.gpu

PAGE, WIDTH, MOST = 1 << 16, 1 << 15, 2 ** 31 - 256
E8 = torch.float8_e8m0fnu


def _sparse(ex, dim, tokens, pos):
    """One sequence of 2^31 - 1 keys, of which only those on its first and last page are there; the keys from 2^31 - 256 on
    are NaN."""
    codes, scales = [], []
    for i in (1, 2):
        # (beyond 464 the conversion would make NaN of them)
        x = (torch.randn((2, PAGE, 1, dim), generator=torch.Generator().manual_seed(i)) * 100).clamp_(-448, 448)
        x[1, PAGE - 256:] = torch.nan
        codes.append(x.to(torch.float8_e4m3fn).cuda())
        scales.append(torch.randint(118, 122, (2, PAGE // 64, 1), generator=torch.Generator().manual_seed(i), dtype=torch.uint8).cuda())
    table = np.full((1, WIDTH), -1)
    table[0, 0], table[0, -1] = 0, 1
    cache = ex.cache(*codes, k_scale=scales[0].view(E8), v_scale=scales[1].view(E8))
    batch = ex.batch(cache, 2, token_seq=i32([0] * tokens), token_pos=i32(pos), seq_start=i32([0, tokens]), seq_len=i32([2 ** 31 - 1]),
                     page_table=i32(table))
    return codes, scales, cache, batch


@pytest.mark.parametrize("dim", [64, 256])
@pytest.mark.parametrize("copies", [1, 9])
def test_a_sequence_of_all_keys(dim, copies):
    """Few rows to an item, and more than its waves take side by side."""
    ex = pkg.Executor()
    pos = [2 ** 31 - 1, MOST, MOST - 1, 2 ** 31 - PAGE - 1, 7] * copies
    codes, scales, cache, batch = _sparse(ex, dim, len(pos), pos)
    q = torch.randn((len(pos), 2, dim), generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).cuda()
    got = exec_history.attend(ex, cache, batch, q, 0.1)
    numbers = [(c.float().double() * torch.exp2(s.double() - 127).repeat_interleave(64, dim=1)[..., None]).view(2 * PAGE, dim) for c, s in zip(codes, scales)]
    for t in range(len(pos)):
        seen = (2 * PAGE - 256, 2 * PAGE - 256, 2 * PAGE - 256, PAGE, 8)[t % 5]
        k, v = (x[:seen] for x in numbers)
        w = torch.softmax(torch.mm(q[t].double(), k.t().contiguous()) * 0.1, dim=1)
        want, weighted = (torch.mm(w, x).cpu().numpy() for x in (v, v.abs()))
        tol = exec_history.tolerance(want, weighted, torch.bfloat16, seen, float(v.abs().max()))
        assert (np.abs(got[t] - want) <= tol).all(), t
    ex.destroy()


def test_keys_that_far_are_written_up_to_the_same_border():
    ex = pkg.Executor()
    pos = [MOST - 2, MOST - 1, MOST, 2 ** 31 - 1]
    codes, scales, cache, batch = _sparse(ex, 64, 4, pos)
    before = [c.float() for c in codes]
    k, v = (torch.randn((4, 1, 64), generator=torch.Generator().manual_seed(i)).to(torch.bfloat16).cuda() for i in (4, 5))
    ex.append(cache, batch, None, k, v, None)
    for code, scale, old, new in zip(codes, scales, before, (k, v)):
        e = int(scale[1, (PAGE - 258) // 64, 0])
        want = scaled_ref.rounded(new[:2].double().cpu().numpy() * 2.0 ** (127 - e))
        assert np.array_equal(code[1, PAGE - 258:PAGE - 256].float().double().cpu().numpy(), want)
        assert torch.isnan(code[1, PAGE - 256:].float()).all()
        assert torch.equal(code[0].float(), old[0]) and torch.equal(code[1, :PAGE - 320].float(), old[1, :PAGE - 320])
    got = [torch.full((4, 1, 64), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    ex.read(cache, batch, *got)
    assert (got[0][2:] == 0).all() and (got[1][2:] == 0).all() and (got[0][:2] != 0).any()
    ex.destroy()


def test_pools_beyond_32_bits():
    """A pool of 2^31 codes and more: the last page is as good as any."""
    ex = pkg.Executor()
    pages, page, kv, dim = (1 << 31) // (64 * 8 * 128) + 70, 64, 8, 128
    pools = [torch.zeros((pages, page, kv, dim), dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.full((pages, page, kv), 127, dtype=torch.uint8, device="cuda") for _ in range(2)]      # (a scale for each key)
    cache = ex.cache(*(p.view(torch.float8_e4m3fn) for p in pools), k_scale=scales[0].view(E8), v_scale=scales[1].view(E8))
    n, last = 50, pages - 1
    batch = ex.batch(cache, 32, token_seq=i32([0] * n), token_pos=i32(range(n)), seq_start=i32([0, n]), seq_len=i32([n]), page_table=i32([[last]]))
    q, k, v = (torch.randn((n, h, dim), generator=torch.Generator().manual_seed(h + i)).to(torch.bfloat16).cuda() for i, h in enumerate((32, kv, kv)))
    out = torch.empty_like(q)
    ex.append(cache, batch, None, k, v, None)
    ex.plan(batch)
    ex.attend(cache, batch, q, out)
    got = [torch.empty_like(k) for _ in range(2)]
    ex.read(cache, batch, *got)
    for x, y in zip(got, (k, v)):
        assert ((x.double() - y.double()).abs() <= 2.0 ** -4 * y.double().abs() + 2.0 ** -10 * 2.0 ** -6).all()
    table = ex.table(1, 1, page, pages, 1)
    table.copies.copy_(i32([[last, pages - 2, n]]))
    ex.copy(cache, table)
    for x in pools + scales:
        assert torch.equal(x[last, :n], x[pages - 2, :n])
    kd, vd = (x.double().cpu().numpy() for x in got)
    for t in (0, 49):
        s = kd[:t + 1, 3] @ q[t, 13].double().cpu().numpy() * dim ** -0.5
        w = np.exp(s - s.max())
        w /= w.sum()
        x, y = w @ vd[:t + 1, 3], out[t, 13].double().cpu().numpy()
        assert (np.abs(x - y) <= 2.0 ** -8 * np.abs(x) + (2.0 ** -8 + 2.0 ** -11) * (w @ np.abs(vd[:t + 1, 3])) + 1e-30).all()
    ex.destroy()
