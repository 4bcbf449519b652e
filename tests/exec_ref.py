"""The executor's operators by their definitions, in 64 bits on the host (numpy), and inputs for their tests."""
import numpy as np
import torch


def rotate(x, pos, freq, interleaved):
    """x [n, heads, dim] float64, the first 2 * len(freq) dimensions rotated by pos * freq."""
    half = len(freq)
    if half == 0:
        return x.copy()
    ang = np.asarray(pos, dtype=np.float64)[:, None] * freq[None, :]
    cos, sin = np.cos(ang)[:, None], np.sin(ang)[:, None]
    y = x.copy()
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    y[..., a], y[..., b] = x[..., a] * cos - x[..., b] * sin, x[..., b] * cos + x[..., a] * sin
    return y


def attend(q, k_of, v_of, limits, scale):
    """q [n, heads, dim]; k_of(t) and v_of(t): keys and values [len, kv_heads, dim] that token t may see, with the truth
    values of which it does in limits[t].  Returns the result and, for the tolerance, sum p |v| and max |v|."""
    n, H, D = q.shape
    out, scale_of, top = np.zeros(q.shape), np.zeros(q.shape), np.zeros((n, H, 1))
    for t in range(n):
        k, v, seen = k_of(t), v_of(t), limits[t]
        k, v = k[seen], v[seen]
        if not len(k):
            continue
        G = H // k.shape[1]
        for h in range(H):
            s = k[:, h // G] @ q[t, h] * scale
            p = np.exp(s - s.max())
            p /= p.sum()
            out[t, h] = p @ v[:, h // G]
            scale_of[t, h] = p @ np.abs(v[:, h // G])
            top[t, h] = np.abs(v[:, h // G]).max()
    return out, scale_of, top


def sample(row, t=1.0, k=0, top_p=1.0, min_p=0.0, draw=0.0):
    """(token, probability) of one row, logits as float64."""
    row = np.where(np.isnan(row), -np.inf, row)
    top = row.max()
    if top == -np.inf:
        return -1, 0.0
    if not t > 0 or min_p > 1:
        return int(row.argmax()), 1.0
    with np.errstate(invalid="ignore", over="ignore"):
        w = (row == np.inf).astype(np.float64) if top == np.inf else np.exp(np.where(row == -np.inf, -np.inf, (row - top) / t))
    order = np.argsort(-row, kind="stable")
    order = order[row[order] > -np.inf]
    if k > 0:
        order = order[:k]
    if top_p < 1:
        cum = np.cumsum(w[order])
        order = order[:1 + int((cum[:-1] < top_p * cum[-1]).sum())]
    order = np.sort(order[w[order] >= min_p]) if min_p > 0 else np.sort(order)
    cum = np.cumsum(w[order])
    i = min(int(np.searchsorted(cum, draw * cum[-1], side="right")), len(order) - 1)
    while w[order[i]] == 0:
        i -= 1
    return int(order[i]), float(w[order[i]] / cum[-1])


class Scene:
    """A ragged batch over a paged cache, on the device and on the host.  seqs: (length, new tokens); groups: first
    sequence of every group and the end; shared: their shared lengths.  Unused slots of the pools hold NaN."""

    def __init__(self, seqs, groups=None, shared=None, heads=8, kv_heads=2, dim=128, page=16, layout="token",
                 dtype=torch.bfloat16, seed=0, joined=False):
        rng = np.random.default_rng(seed)
        S = len(seqs)
        self.heads, self.kv_heads, self.dim, self.page, self.dtype = heads, kv_heads, dim, page, dtype
        self.length = np.array([s[0] for s in seqs], dtype=np.int64).reshape(S)
        self.new = np.array([s[1] for s in seqs], dtype=np.int64).reshape(S)
        self.start = np.concatenate([[0], np.cumsum(self.new)]).astype(np.int64)
        self.n = int(self.start[-1])
        self.seq = np.repeat(np.arange(S), self.new)
        self.pos = self.length[self.seq] - self.new[self.seq] + np.arange(self.n) - self.start[self.seq]
        self.group_start, self.shared = groups, shared
        width = max(1, int(-(-self.length.max() // page))) + 1
        total = S * width + 3
        self.table = rng.permutation(total)[:S * width].reshape(S, width)
        # logical keys and values; a group's shared ones are its first sequence's
        shape = (total, page, kv_heads, dim)
        self.pools = []
        self.full = []
        for _ in range(2):
            pool = np.full(shape, np.nan)
            full = []
            for s in range(S):
                x = rng.standard_normal((int(self.length[s]), kv_heads, dim))
                x = torch.from_numpy(x).to(dtype).double().numpy()
                j = np.arange(len(x))
                pool[self.table[s, j // page], j % page] = x
                full.append(x)
            for g in range(len(shared) if shared is not None else 0):
                a = groups[g]
                for s in range(groups[g], groups[g + 1]):
                    m = min(shared[g], len(full[s]))
                    if s != a:
                        full[s] = np.concatenate([full[a][:m], full[s][m:]])
            self.pools.append(pool)
            self.full.append(full)
        dev = []
        for pool in self.pools:
            t = torch.from_numpy(pool).to(dtype)
            dev.append(t if layout == "token" else t.transpose(1, 2).contiguous())
        if joined:      # both pools in one allocation, pages side by side
            both = torch.stack(dev, dim=1).cuda()
            self.k_pool, self.v_pool = both[:, 0], both[:, 1]
        else:
            self.k_pool, self.v_pool = (t.cuda() for t in dev)
        self.layout = layout
        q = torch.from_numpy(rng.standard_normal((self.n, heads, dim))).to(dtype)
        self.q_host, self.q = q.double().numpy(), q.cuda()

    def batch(self, ex, cache, max_len=None, pos=None, length=None, table=None):
        i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()
        groups = {} if self.shared is None else dict(group_start=i32(self.group_start), shared_len=i32(self.shared))
        return ex.batch(cache, self.heads, token_seq=i32(self.seq), token_pos=i32(self.pos if pos is None else pos),
                        seq_start=i32(self.start), seq_len=i32(self.length if length is None else length),
                        page_table=i32(self.table if table is None else table), max_len=max_len, **groups)

    def limits(self):
        return [np.arange(int(self.length[s])) <= p for s, p in zip(self.seq, self.pos)]

    def reference(self, scale, limits=None):
        return attend(self.q_host, lambda t: self.full[0][self.seq[t]], lambda t: self.full[1][self.seq[t]],
                      self.limits() if limits is None else limits, scale)


def attend_tolerance(want, weighted, top, dtype, keys):
    """Of a result rounded to dtype: half a step of itself; of the rounded weights half a step each, and 2^-11 for the
    scores' products in 32 bits (their error moves a weight by its own share), both of sum p |v|; and the smallest step of
    fp16 weights below its normal range, 2^-25, of every value."""
    half = torch.finfo(dtype).eps / 2
    return half * np.abs(want) + (half + 2.0 ** -11) * weighted + (keys * 2.0 ** -25 * top if dtype == torch.float16 else 0) + 1e-30
