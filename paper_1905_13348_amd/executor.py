"""What a worker does with the queries sent to it: the executor's calls of include/infaas_sel.h on torch tensors.

    ex = Executor()
    cache = ex.cache(k_pool, v_pool)                     # one layer's pools of pages
    batch = ex.batch(cache, heads, token_seq=..., ...)   # the step's tokens and the sequences' pages
    ex.plan(batch)                                       # once a step, for all layers
    ex.append(cache, batch, q, k, v, q_out, freq)        # each layer
    ex.attend(cache, batch, q_out, out, scale)
    ex.sample(logits, draws, token, prob, top_p=...)     # behind the last layer

Argument marshalling only, like ``Selector``: shapes and types are checked here, values in the library.  A cache and a
batch keep references to their tensors; the tensors' contents may change from step to step.  There is no backward pass:
inputs that require a gradient are refused where gradients are recorded.
"""
from __future__ import annotations

import ctypes
from typing import Optional

from .binding import InfaasSelError, _AppendArgs, _Batch, _Cache, _stream_ptr, _use_torch, load_library

_TYPES = None        # torch type -> INFAAS_SEL_TYPE_*


_tensor_class = None


def _tensor():
    global _tensor_class
    if _tensor_class is None:
        _tensor_class = _use_torch().Tensor
    return _tensor_class


def _types():
    global _TYPES
    if _TYPES is None:
        torch = _use_torch()
        _TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
    return _TYPES


def _check(status: int) -> None:
    if status != 0:
        lib = load_library()
        text = lib.infaas_sel_strerror(status).decode()
        if status in (-1, -4):
            text += " [" + lib.infaas_sel_last_error().decode() + "]"
        raise InfaasSelError(status, text)


def _i32(value: int, name: str) -> int:
    """A size as the library takes it (ctypes would cut it to 32 bits without a word)."""
    if not -2 ** 31 <= value < 2 ** 31:
        raise ValueError(f"{name}: {value} is beyond 32 bits")
    return value


def _vector(t, dtype, name: str, device: int, size: Optional[int] = None) -> int:
    """Raw pointer of a contiguous tensor of one dimension on a device."""
    if not isinstance(t, _tensor()) or t.dtype is not dtype or t.get_device() != device or not t.is_contiguous() or t.dim() != 1 \
            or (size is not None and t.numel() != size):
        raise TypeError(f"{name}: contiguous {dtype} tensor [{'any' if size is None else size}] on device {device} expected")
    return t.data_ptr()


def _no_gradient(t, name: str) -> None:
    """The calls write to tensors that they are given, and what they compute has no backward: as with torch's own outputs that
    are given, an input that needs a gradient would lose it without a word."""
    if t.requires_grad and _use_torch().is_grad_enabled():
        raise RuntimeError(f"{name} requires a gradient and the executor's calls have none: call them under torch.no_grad()")


class PagedCache:
    """One layer's pools of pages (infaas_sel_cache): ``layout`` "token" for [page][slot][head][dim], "head" for
    [page][head][slot][dim]; both pools have the same shape and strides, the last dimension consecutive."""

    def __init__(self, k_pool, v_pool, layout: str = "token"):
        torch = _use_torch()
        if layout not in ("token", "head"):
            raise ValueError(f"layout {layout!r}: 'token' or 'head'")
        if not all(isinstance(p, torch.Tensor) and p.is_cuda and p.dim() == 4 for p in (k_pool, v_pool)):
            raise TypeError("device tensors of four dimensions expected")
        # (a dimension of one element has a stride of no meaning)
        st, vst = ([0 if n == 1 else x for n, x in zip(p.shape, p.stride())] for p in (k_pool, v_pool))
        if k_pool.dtype not in (torch.bfloat16, torch.float16) or v_pool.dtype != k_pool.dtype \
                or v_pool.shape != k_pool.shape or st != vst or k_pool.stride(3) != 1:
            raise TypeError("pools of one type (bfloat16 or float16), shape and strides expected, the last one 1")
        if k_pool.get_device() != v_pool.get_device():
            raise TypeError("pools on one device expected")
        _no_gradient(k_pool, "k_pool")
        _no_gradient(v_pool, "v_pool")
        slot, head = (1, 2) if layout == "token" else (2, 1)
        self.k_pool, self.v_pool, self.layout, self.dtype = k_pool, v_pool, layout, k_pool.dtype
        self.device = k_pool.get_device()
        self.kv_heads, self.head_dim = k_pool.shape[head], k_pool.shape[3]
        self.page_size, self.num_pages = k_pool.shape[slot], k_pool.shape[0]
        self._c = _Cache(d_k=k_pool.data_ptr(), d_v=v_pool.data_ptr(), type=_types()[k_pool.dtype], kv_heads=_i32(self.kv_heads, "KV heads"),
                         head_dim=_i32(self.head_dim, "head dimension"), page_size=_i32(self.page_size, "page size"), num_pages=self.num_pages,
                         page_stride=st[0], slot_stride=st[slot], head_stride=st[head])
        self._ref = ctypes.byref(self._c)
        self._sizes = (self.kv_heads, self.head_dim, self.page_size)      # what a batch's caches have in common


class Batch:
    """A step's ragged batch (infaas_sel_batch) with the memory of its plan.  That memory is a torch tensor like the arrays:
    it is made and cleared on torch's current stream, so calls on another stream have to wait for that one first, and a batch
    has to be kept until the calls that use it have run."""

    def __init__(self, cache: PagedCache, heads: int, *, token_seq, token_pos, seq_start, seq_len, page_table,
                 group_start=None, shared_len=None, max_len: Optional[int] = None):
        torch = _use_torch()
        i32 = torch.int32
        for name, t in (("token_seq", token_seq), ("seq_len", seq_len)) + ((("shared_len", shared_len),) if shared_len is not None else ()):
            if not isinstance(t, torch.Tensor):
                raise TypeError(f"{name}: a tensor expected, not {type(t).__name__}")
        n, S = token_seq.numel(), seq_len.numel()
        if (group_start is None) != (shared_len is None):
            raise TypeError("group_start and shared_len belong together")
        groups = 0 if shared_len is None else shared_len.numel()
        if not isinstance(page_table, torch.Tensor) or page_table.dim() != 2 or page_table.shape[0] != S \
                or page_table.dtype != i32 or page_table.get_device() != cache.device or not page_table.is_contiguous():
            raise TypeError(f"page_table: contiguous int32 tensor [{S}, pages] on the cache's device {cache.device} expected")
        vector = lambda t, name, size=None: _vector(t, i32, name, cache.device, size)
        width = page_table.shape[1]
        self.num_tokens, self.heads = n, heads
        self._keep = (token_seq, token_pos, seq_start, seq_len, page_table, group_start, shared_len)
        self._c = _Batch(
            num_tokens=_i32(n, "token_seq"), num_seqs=_i32(S, "seq_len"), num_groups=groups, heads=_i32(heads, "heads"),
            max_len=min(width * cache.page_size, 0x7fffffff) if max_len is None else _i32(max_len, "max_len"),
            table_width=_i32(width, "page_table"),
            d_token_seq=vector(token_seq, "token_seq"), d_token_pos=vector(token_pos, "token_pos", n),
            d_seq_start=vector(seq_start, "seq_start", S + 1), d_seq_len=vector(seq_len, "seq_len"),
            d_page_table=page_table.data_ptr(),
            d_group_start=None if not groups else vector(group_start, "group_start", groups + 1),
            d_shared_len=None if not groups else vector(shared_len, "shared_len"))
        self._ref = ctypes.byref(self._c)
        self._q_shape, self._kv_shape = (n, heads, cache.head_dim), (n, cache.kv_heads, cache.head_dim)
        self._cache = cache      # what the plan's sizes go by
        self._sizes = cache._sizes
        size = load_library().infaas_sel_exec_plan_bytes(cache._ref, self._ref)
        if size == 0:
            _check(-1)
        self.plan_memory = torch.zeros((size + 3) // 4, dtype=i32, device=token_seq.device)
        self._c.d_plan, self._c.plan_bytes = self.plan_memory.data_ptr(), size


class Executor:
    """One executor handle of the library (infaas_sel_exec_create ... infaas_sel_exec_destroy)."""

    def __init__(self, device: int = 0):
        self._h = ctypes.c_void_p()
        self._lib = load_library()
        _check(self._lib.infaas_sel_exec_create(_i32(device, "device"), ctypes.byref(self._h)))
        self.device = device

    def cache(self, k_pool, v_pool, layout: str = "token") -> PagedCache:
        return PagedCache(k_pool, v_pool, layout)

    def batch(self, cache: PagedCache, heads: int, **arrays) -> Batch:
        return Batch(cache, heads, **arrays)

    def reserve(self, cache: PagedCache, batch: Batch) -> None:
        self._agree(cache, batch)
        _check(self._lib.infaas_sel_exec_reserve(self._h, cache._ref, batch._ref))

    def plan(self, batch: Batch, stream=None) -> None:
        self._agree(batch._cache, batch)
        _check(self._lib.infaas_sel_exec_plan(self._h, batch._cache._ref, batch._ref, _stream_ptr(stream, self.device)))

    def _agree(self, cache: PagedCache, batch: Batch) -> None:
        if cache is not batch._cache and cache._sizes != batch._sizes:
            raise ValueError(f"a cache of (KV heads, head dimension, page size) {cache._sizes} with a batch made for {batch._sizes}")
        if cache.device != self.device or batch._cache.device != self.device:
            raise ValueError(f"an executor of device {self.device} with a cache on {cache.device} and a batch on {batch._cache.device}")

    @staticmethod
    def _rows(t, cache: PagedCache, batch: Batch, shape, name: str):
        """Pointer and strides of a [tokens][heads][head_dim] tensor."""
        if not isinstance(t, _tensor_class or _tensor()) or t.dtype is not cache.dtype or t.get_device() != cache.device or t.shape != shape:
            raise TypeError(f"{name}: {cache.dtype} tensor {list(shape)} on device {cache.device} expected")
        if t.requires_grad:
            _no_gradient(t, name)
        a, b, c = t.stride()
        if c != 1:
            raise TypeError(f"{name}: the last dimension is not consecutive")
        # (a dimension of one element has a stride of no meaning)
        return t.data_ptr(), a if shape[0] > 1 else 0, b if shape[1] > 1 else 0

    def append(self, cache: PagedCache, batch: Batch, q, k, v, q_out, freq=None, interleaved: bool = False,
               stream=None) -> None:
        """Keys and values into the cache, rotated by the positions; ``freq`` (float64, a frequency per rotated pair) None:
        not rotated; ``q`` and ``q_out`` both None: no queries."""
        if cache is not batch._cache or cache.device != self.device:
            self._agree(cache, batch)
        rows, q_shape, kv_shape = self._rows, batch._q_shape, batch._kv_shape
        qp, qt, qh = (None, 0, 0) if q is None else rows(q, cache, batch, q_shape, "q")
        op, ot, oh = (None, 0, 0) if q_out is None else rows(q_out, cache, batch, q_shape, "q_out")
        kp, kt, kh = rows(k, cache, batch, kv_shape, "k")
        vp, vt, vh = rows(v, cache, batch, kv_shape, "v")
        fp, rot = None, 0
        if freq is not None:
            fp, rot = _vector(freq, _use_torch().float64, "freq", self.device), _i32(2 * freq.numel(), "freq")
            _no_gradient(freq, "freq")
        a = _AppendArgs(qp, kp, vp, op, qt, qh, kt, kh, vt, vh, ot, oh, fp, rot, 1 if interleaved else 0)
        status = self._lib.infaas_sel_exec_append(self._h, cache._ref, batch._ref, a, _stream_ptr(stream, self.device))
        if status:
            _check(status)

    def attend(self, cache: PagedCache, batch: Batch, q, out, scale: Optional[float] = None, stream=None) -> None:
        """Attention of the planned batch's tokens over the cache; ``scale`` None: head_dim ** -0.5."""
        if cache is not batch._cache or cache.device != self.device:
            self._agree(cache, batch)
        shape = batch._q_shape
        status = self._lib.infaas_sel_exec_attend(
            self._h, cache._ref, batch._ref, *self._rows(q, cache, batch, shape, "q"),
            *self._rows(out, cache, batch, shape, "out"), cache.head_dim ** -0.5 if scale is None else scale,
            _stream_ptr(stream, self.device))
        if status:
            _check(status)

    def sample(self, logits, draws, token, prob=None, *, temperature=None, top_k=None, top_p=None, min_p=None,
               stream=None) -> None:
        """A token of every row of logits [rows, vocab]; limits are tensors [rows] or None."""
        torch = _use_torch()
        dev = self.device
        if not isinstance(logits, torch.Tensor) or logits.get_device() != dev or logits.dim() != 2 or logits.dtype not in _types() \
                or (logits.shape[1] > 1 and logits.stride(1) != 1):
            raise TypeError(f"logits: tensor [rows, vocab] on device {dev} expected, the last dimension consecutive")
        _no_gradient(logits, "logits")
        rows, vocab = logits.shape
        f32, i32 = torch.float32, torch.int32
        status = self._lib.infaas_sel_exec_sample(
            self._h, _i32(rows, "rows"), _i32(vocab, "vocab"), _types()[logits.dtype], logits.data_ptr(), logits.stride(0),
            temperature if temperature is None else _vector(temperature, f32, "temperature", dev, rows),
            top_k if top_k is None else _vector(top_k, i32, "top_k", dev, rows),
            top_p if top_p is None else _vector(top_p, f32, "top_p", dev, rows),
            min_p if min_p is None else _vector(min_p, f32, "min_p", dev, rows),
            _vector(draws, f32, "draws", dev, rows), _vector(token, i32, "token", dev, rows),
            prob if prob is None else _vector(prob, f32, "prob", dev, rows), _stream_ptr(stream, self.device))
        if status:
            _check(status)

    def destroy(self) -> None:
        if self._h:
            self._lib.infaas_sel_exec_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass
