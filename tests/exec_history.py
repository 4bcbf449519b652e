"""Many sequences over the pages of one history, so that a batch is as large as a test wants while its reference stays one
matrix product, in 64 bits; and what a plan holds."""
import numpy as np
import torch

HEADER_INTS, HEADER_BYTES, TOKEN_BYTES, UNIT_BYTES, ITEM_INTS = 32, 128, 32, 32, 8


def i32(a):
    return torch.as_tensor(np.ascontiguousarray(a, dtype=np.int32)).cuda()


class History:
    """k, v: [keys, kv_heads, dim] on the device.  Every sequence of a batch has these keys, up to a length of its own."""

    def __init__(self, k, v, page=16):
        self.k, self.v, self.page = k, v, page
        keys, self.kv_heads, self.dim = k.shape
        pages = -(-keys // page)
        self.pools = []
        for x in (k, v):
            pool = torch.full((pages * page, self.kv_heads, self.dim), float("nan"), dtype=k.dtype, device="cuda")
            pool[:keys] = x
            # (in another order, and one page more that nothing names)
            order = np.random.default_rng(keys).permutation(pages + 1)[:pages]
            mixed = torch.full((pages + 1, page, self.kv_heads, self.dim), float("nan"), dtype=k.dtype, device="cuda")
            mixed[torch.from_numpy(order).cuda()] = pool.view(pages, page, self.kv_heads, self.dim)
            self.pools.append(mixed)
        self.row = order

    def batch(self, ex, cache, heads, length, new=None, pos=None, missing=(), shared=None, groups=None, max_len=None):
        """A token to every sequence (or `new` of them), the last of its keys; `missing`: pages (of the history) that are not
        there; `shared`: keys that all of them share as a group, or with `groups` (first sequences and the end) each group."""
        S = len(length)
        length = np.asarray(length, dtype=np.int64)
        new = np.ones(S, dtype=np.int64) if new is None else np.asarray(new)
        start = np.concatenate([[0], np.cumsum(new)])
        seq = np.repeat(np.arange(S), new)
        if pos is None:
            pos = (length - new)[seq] + np.arange(len(seq)) - start[seq]
        row = self.row.copy()
        row[list(missing)] = -1
        if shared is not None and groups is None:
            groups, shared = [0, S], [shared]
        groups = {} if shared is None else dict(group_start=i32(groups), shared_len=i32(shared))
        batch = ex.batch(cache, heads, token_seq=i32(seq), token_pos=i32(pos), seq_start=i32(start), seq_len=i32(length),
                         page_table=i32(np.tile(row, (S, 1))), max_len=int(length.max()) if max_len is None else max_len, **groups)
        return batch, np.minimum(np.asarray(pos) + 1, length[seq])

    def reference(self, q, limit, scale, missing=()):
        """[tokens, heads, dim] in 64 bits, with sum p |v|, which rounding goes by.  Keys from `limit` on are not seen; nor
        what is on missing pages; a token that sees none has zeros."""
        n, H, D = q.shape
        G, keys = H // self.kv_heads, self.k.shape[0]
        seen = torch.arange(keys, device="cuda")[None, :] < torch.as_tensor(np.asarray(limit)).cuda()[:, None]
        for p in missing:
            seen[:, p * self.page:(p + 1) * self.page] = False
        out, weighted = (torch.zeros((n, H, D), dtype=torch.float64, device="cuda") for _ in range(2))
        for h in range(self.kv_heads):
            k, v = self.k[:, h].double(), self.v[:, h].double()
            odd = (~v.isfinite()).nonzero().tolist()      # (added where they are seen; 0 times them would be NaN)
            odd = [(key, d, float(v[key, d])) for key, d in odd]
            v = v.nan_to_num(0, 0, 0)
            for j in range(h * G, (h + 1) * G):
                s = (torch.mm(q[:, j].double(), k.t().contiguous()) * scale).masked_fill(~seen, -torch.inf)
                p = torch.softmax(s, dim=1)
                p[~seen.any(dim=1)] = 0
                out[:, j] = torch.mm(p, v)
                for key, d, x in odd:
                    out[:, j, d] += torch.where(seen[:, key], x, 0.0)
                weighted[:, j] = torch.mm(p, v.abs())
        return out.cpu().numpy(), weighted.cpu().numpy()


def attend(ex, cache, batch, q, scale, out=None):
    out = torch.full_like(q, 7.0) if out is None else out
    ex.plan(batch)
    ex.attend(cache, batch, q, out, scale)
    torch.cuda.synchronize()
    return out.double().cpu().numpy()


def plan_of(batch):
    """(header, items): items as rows of first token, tokens, first key, end of the keys, sequence, KV head, row, -."""
    mem = batch.plan_memory.cpu().numpy()
    c = batch._c
    at = (HEADER_BYTES + c.num_tokens * TOKEN_BYTES + (c.num_seqs + c.num_groups) * UNIT_BYTES) // 4
    n = int(mem[10])
    return mem[:HEADER_INTS], mem[at:at + n * ITEM_INTS].reshape(n, ITEM_INTS)


def tolerance(want, weighted, dtype, keys, top, raised=0):
    """Half a step of the result; of the rounded weights half a step each and 2^-11 for the scores' products in 32 bits, both
    of sum p |v|; in fp16 half of the smallest step, 2^-25, of every value of a key whose weight is below the normal range
    (`raised`: halvings that the greatest weight is above 1)."""
    half = torch.finfo(dtype).eps / 2
    low = keys * 2.0 ** (-25 - raised) * top if dtype == torch.float16 else 0
    return half * np.abs(want) + (half + 2.0 ** -11) * weighted + low + 1e-30
