"""Caches of 8 bits for tests: codes of e4m3 by their definition in 64 bits (numpy), and scenes of exec_ref over them."""
import numpy as np
import torch

import exec_ref


def rounded(x):
    """x to the nearest number of e4m3, ties to even: three bits behind the first one, steps of 2^-9 at the least.  Beyond 464
    and for what is no number: NaN."""
    x = np.asarray(x, dtype=np.float64)
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        step = np.exp2(np.maximum(np.floor(np.log2(np.abs(x))), -6) - 3)
        step = np.where(np.isfinite(step) & (step > 0), step, 2.0 ** -9)
        y = np.rint(x / step) * step
        return np.where(np.abs(y) <= 448, y, np.nan)


def need(top):
    """The least e >= 1 with top <= 448 * 2^(e - 127)."""
    e = 1
    while top > 448 * 2.0 ** (e - 127):
        e += 1
    return e


def codes(x):
    """Numbers of e4m3 as a tensor of them."""
    return torch.from_numpy(np.ascontiguousarray(x)).float().to(torch.float8_e4m3fn)


def scales(e):
    return torch.from_numpy(np.ascontiguousarray(e).astype(np.uint8)).view(torch.float8_e8m0fnu)


def numbers(code, e, dtype):
    """What code and scale stand for, as numbers of a type: float64 arrays in and out (e: bytes)."""
    with np.errstate(invalid="ignore", over="ignore"):
        x = code * np.where(e == 255, np.nan, np.exp2(np.asarray(e, dtype=np.float64) - 127))
    return torch.from_numpy(x).to(dtype).double().numpy()


class Scene(exec_ref.Scene):
    """exec_ref.Scene over codes: its numbers rounded to codes, by scales drawn for each block and head."""

    def __init__(self, seqs, *args, block=16, low=118, high=124, spoil=None, **kw):
        super().__init__(seqs, *args, **kw)
        rng = np.random.default_rng(kw.get("seed", 0) + 1000)
        P, self.block = self.page, min(block, self.page)
        self.code, self.e, dev = [], [], []
        for pool in self.pools:      # [page][slot][head][dim]
            total, _, H, D = pool.shape
            e = rng.integers(low, high + 1, (total, P // self.block, H))
            per_slot = np.repeat(e, self.block, axis=1)[..., None]
            code = rounded(np.clip(pool / np.exp2(per_slot - 127.0), -448, 448))
            if spoil:
                spoil(len(self.code), code, e)
            self.code.append(code)
            self.e.append(e)
        self.full = [[numbers(c[self.table[s, np.arange(n) // P], np.arange(n) % P],
                              e[self.table[s, np.arange(n) // P], np.arange(n) % P // self.block][..., None], self.dtype)
                      for s, n in enumerate(self.length)] for c, e in zip(self.code, self.e)]
        for full in self.full:
            for g in range(len(self.shared) if self.shared is not None else 0):
                a = self.group_start[g]
                for s in range(a, self.group_start[g + 1]):
                    m = min(self.shared[g], len(full[s]))
                    if s != a:
                        full[s] = np.concatenate([full[a][:m], full[s][m:]])
        for code, e in zip(self.code, self.e):
            c, e = codes(code), scales(e)
            if self.layout == "head":
                c, e = (t.view(torch.uint8).transpose(1, 2).contiguous().view(t.dtype) for t in (c, e))
            dev.append((c.cuda(), e.cuda()))
        (self.k_pool, self.k_scale), (self.v_pool, self.v_scale) = dev

    def cache(self, ex):
        return ex.cache(self.k_pool, self.v_pool, layout=self.layout, k_scale=self.k_scale, v_scale=self.v_scale, dtype=self.dtype)
