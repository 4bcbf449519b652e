"""What a worker does with the queries sent to it: the executor's calls of include/infaas_sel.h on torch tensors.

    ex = Executor()
    cache = ex.cache(k_pool, v_pool)                     # one layer's pools of pages
    batch = ex.batch(cache, heads, token_seq=..., ...)   # the step's tokens and the sequences' pages
    ex.plan(batch)                                       # once a step, for all layers
    ex.append(cache, batch, q, k, v, q_out, freq)        # each layer
    ex.attend(cache, batch, q_out, out, scale)
    ex.sample(logits, draws, token, prob, top_p=...)     # behind the last layer

A cache may be of 8 bits (``ex.cache(..., k_scale=, v_scale=)``), and a batch's arrays may be kept on the device:

    table = ex.table(seqs, width, page_size, pages, max_tokens)
    batch = ex.batch(cache, heads, **table.arrays())
    ex.advance(table, new, parent)                       # once a step: lengths, pages, the batch's arrays
    ex.copy(cache, table)                                # each layer, before its append
    ex.beam(logits, scores, parent, token, score)        # instead of sample: the next step's parents

Argument marshalling only, like ``Selector``: shapes and types are checked here, values in the library.  A cache and a
batch keep references to their tensors; the tensors' contents may change from step to step.  There is no backward pass:
inputs that require a gradient are refused where gradients are recorded.
"""
from __future__ import annotations

import ctypes
from typing import Optional

from .binding import InfaasSelError, _AppendArgs, _Batch, _Cache, _Scales, _stream_ptr, _Table, _use_torch, load_library

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
    [page][head][slot][dim]; both pools have the same shape and strides, the last dimension consecutive.

    With ``k_scale`` and ``v_scale`` a cache of 8 bits (infaas_sel_scales): pools of float8_e4m3fn, scales of float8_e8m0fnu
    [page][block][head] or [page][head][block], page size / blocks keys to a scale; ``dtype`` is then the type of what is
    appended and of queries and results (bfloat16 if not given)."""

    def __init__(self, k_pool, v_pool, layout: str = "token", k_scale=None, v_scale=None, dtype=None):
        torch = _use_torch()
        coded = k_scale is not None or v_scale is not None
        if layout not in ("token", "head"):
            raise ValueError(f"layout {layout!r}: 'token' or 'head'")
        if not all(isinstance(p, torch.Tensor) and p.is_cuda and p.dim() == 4 for p in (k_pool, v_pool)):
            raise TypeError("device tensors of four dimensions expected")
        # (a dimension of one element has a stride of no meaning)
        st, vst = ([0 if n == 1 else x for n, x in zip(p.shape, p.stride())] for p in (k_pool, v_pool))
        types = (torch.float8_e4m3fn,) if coded else (torch.bfloat16, torch.float16)
        if k_pool.dtype not in types or v_pool.dtype != k_pool.dtype or v_pool.shape != k_pool.shape or st != vst or k_pool.stride(3) != 1:
            raise TypeError(f"pools of one type ({'float8_e4m3fn' if coded else 'bfloat16 or float16'}), shape and strides expected, "
                            "the last one 1")
        if k_pool.get_device() != v_pool.get_device():
            raise TypeError("pools on one device expected")
        _no_gradient(k_pool, "k_pool")
        _no_gradient(v_pool, "v_pool")
        slot, head = (1, 2) if layout == "token" else (2, 1)
        if dtype is None:
            dtype = torch.bfloat16 if coded else k_pool.dtype
        if dtype not in (torch.bfloat16, torch.float16) or (not coded and dtype != k_pool.dtype):
            raise TypeError(f"dtype {dtype}: that of the pools, or with scales bfloat16 or float16")
        self.k_pool, self.v_pool, self.layout, self.dtype = k_pool, v_pool, layout, dtype
        self.device = k_pool.get_device()
        self.kv_heads, self.head_dim = k_pool.shape[head], k_pool.shape[3]
        self.page_size, self.num_pages = k_pool.shape[slot], k_pool.shape[0]
        self._c = _Cache(d_k=k_pool.data_ptr(), d_v=v_pool.data_ptr(), type=_types()[dtype], kv_heads=_i32(self.kv_heads, "KV heads"),
                         head_dim=_i32(self.head_dim, "head dimension"), page_size=_i32(self.page_size, "page size"), num_pages=self.num_pages,
                         page_stride=st[0], slot_stride=st[slot], head_stride=st[head])
        self._ref = ctypes.byref(self._c)
        self._sizes = (self.kv_heads, self.head_dim, self.page_size)      # what a batch's caches have in common
        self.k_scale, self.v_scale, self._scales = k_scale, v_scale, None
        if coded:
            self._scales_of(torch, slot, head)

    def _scales_of(self, torch, slot: int, head: int) -> None:
        """The scales' part of the arguments."""
        for name, s in (("k_scale", self.k_scale), ("v_scale", self.v_scale)):
            if not isinstance(s, torch.Tensor) or s.dtype != torch.float8_e8m0fnu or s.dim() != 3 or s.get_device() != self.device:
                raise TypeError(f"{name}: float8_e8m0fnu tensor of three dimensions on device {self.device} expected")
        ks, vs = self.k_scale, self.v_scale
        blocks = ks.shape[slot]
        want = [self.num_pages] * 3
        want[slot], want[head] = blocks, self.kv_heads
        st, vst = ([0 if n == 1 else x for n, x in zip(s.shape, s.stride())] for s in (ks, vs))
        if list(ks.shape) != want or ks.shape != vs.shape or st != vst or blocks < 1 or self.page_size % blocks:
            raise TypeError(f"scales of one shape and strides expected: the pools' without the last dimension, with blocks of keys in the "
                            f"place of {self.page_size} slots, not {list(ks.shape)} and {list(vs.shape)}")
        self._scales = _Scales(d_k_scale=ks.data_ptr(), d_v_scale=vs.data_ptr(), block=self.page_size // blocks,
                               page_stride=st[0], block_stride=st[slot], head_stride=st[head])
        self._scales_ref = ctypes.byref(self._scales)


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


class Table:
    """The pages of a worker's sequences (infaas_sel_table), with all of its arrays: int32 tensors that are made here, empty, on
    torch's current stream.

    State, which ``Executor.advance`` takes a step further: ``page_table`` [sequences, width], ``seq_len`` [sequences],
    ``page_refs`` [pages].  What it writes beside that: ``seq_start``, ``token_seq`` and ``token_pos``, which with the state are the arrays
    of a batch of ``max_tokens`` tokens (``arrays()``), ``taken`` [sequences] and ``copies`` [sequences, 3].

    A batch's work and memory go by its size, padding or not.  Where prompts and single tokens take turns, make a batch of each kind:
    of ``arrays()`` as they are, and with ``token_seq`` and ``token_pos`` cut to the tokens that a step has at the most
    (``token_seq[:num_seqs]`` for one of each sequence)."""

    def __init__(self, num_seqs: int, table_width: int, page_size: int, num_pages: int, max_tokens: int, device: int = 0):
        torch = _use_torch()
        for name, n, most in (("num_seqs", num_seqs, 4096), ("table_width", table_width, 2 ** 31 - 1), ("page_size", page_size, 65536),
                              ("num_pages", num_pages, 2 ** 31 - 1), ("max_tokens", max_tokens, 2 ** 31 - 1)):
            if not 1 <= n <= most:
                raise ValueError(f"{name}: {n} is not within 1 .. {most}")
        if page_size & (page_size - 1):
            raise ValueError(f"page_size: {page_size} is not a power of two")
        full = lambda value, *shape: torch.full(shape, value, dtype=torch.int32, device=torch.device("cuda", device))
        self.num_seqs, self.table_width, self.page_size, self.num_pages, self.max_tokens = num_seqs, table_width, page_size, num_pages, max_tokens
        self.device = device
        self.page_table, self.seq_len, self.page_refs = full(-1, num_seqs, table_width), full(0, num_seqs), full(0, num_pages)
        self.seq_start, self.token_seq, self.token_pos = full(0, num_seqs + 1), full(-1, max_tokens), full(-1, max_tokens)
        self.taken, self.copies = full(0, num_seqs), full(-1, num_seqs, 3)
        self._keep = (self.page_table, self.seq_len, self.page_refs, self.seq_start, self.token_seq, self.token_pos, self.taken, self.copies)
        self._c = _Table(num_seqs, table_width, page_size, num_pages, max_tokens, 0, *(t.data_ptr() for t in self._keep))
        self._ref = ctypes.byref(self._c)

    def arrays(self) -> dict:
        """What ``Executor.batch`` takes."""
        return dict(token_seq=self.token_seq, token_pos=self.token_pos, seq_start=self.seq_start, seq_len=self.seq_len, page_table=self.page_table)


class Executor:
    """One executor handle of the library (infaas_sel_exec_create ... infaas_sel_exec_destroy)."""

    def __init__(self, device: int = 0):
        self._h = ctypes.c_void_p()
        self._lib = load_library()
        _check(self._lib.infaas_sel_exec_create(_i32(device, "device"), ctypes.byref(self._h)))
        self.device = device

    def cache(self, k_pool, v_pool, layout: str = "token", k_scale=None, v_scale=None, dtype=None) -> PagedCache:
        return PagedCache(k_pool, v_pool, layout, k_scale, v_scale, dtype)

    def batch(self, cache: PagedCache, heads: int, **arrays) -> Batch:
        return Batch(cache, heads, **arrays)

    def table(self, num_seqs: int, table_width: int, page_size: int, num_pages: int, max_tokens: int) -> Table:
        return Table(num_seqs, table_width, page_size, num_pages, max_tokens, self.device)

    def advance(self, table: Table, new, parent=None, stream=None) -> None:
        """All sequences a step further: ``new`` tokens of each (below 0: keys that are dropped), going on from ``parent`` (None:
        from itself; a number that is no sequence's: from nothing)."""
        if table.device != self.device:
            raise ValueError(f"an executor of device {self.device} with a table on {table.device}")
        i32 = _use_torch().int32
        status = self._lib.infaas_sel_exec_advance(
            self._h, table._ref, _vector(new, i32, "new", self.device, table.num_seqs),
            None if parent is None else _vector(parent, i32, "parent", self.device, table.num_seqs), _stream_ptr(stream, self.device))
        if status:
            _check(status)

    def copy(self, cache: PagedCache, table: Table, stream=None) -> None:
        """What the table's latest step copies from page to page, in one layer's cache."""
        if table.device != self.device or cache.device != self.device:
            raise ValueError(f"an executor of device {self.device} with a cache on {cache.device} and a table on {table.device}")
        scales = getattr(cache, "_scales", None)
        status = self._lib.infaas_sel_exec_copy(self._h, cache._ref, None if scales is None else cache._scales_ref, table._ref,
                                                _stream_ptr(stream, self.device))
        if status:
            _check(status)

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
        if getattr(cache, "_scales", None) is None:
            status = self._lib.infaas_sel_exec_append(self._h, cache._ref, batch._ref, a, _stream_ptr(stream, self.device))
        else:
            status = self._lib.infaas_sel_exec_append_scaled(self._h, cache._ref, cache._scales_ref, batch._ref, a,
                                                             _stream_ptr(stream, self.device))
        if status:
            _check(status)

    def read(self, cache: PagedCache, batch: Batch, k, v, stream=None) -> None:
        """The cache's keys and values at the batch's tokens' positions into ``k`` and ``v`` [tokens][KV heads][dim]."""
        if cache is not batch._cache or cache.device != self.device:
            self._agree(cache, batch)
        scales = getattr(cache, "_scales", None)
        status = self._lib.infaas_sel_exec_read(
            self._h, cache._ref, None if scales is None else cache._scales_ref, batch._ref,
            *self._rows(k, cache, batch, batch._kv_shape, "k"), *self._rows(v, cache, batch, batch._kv_shape, "v"),
            _stream_ptr(stream, self.device))
        if status:
            _check(status)

    def attend(self, cache: PagedCache, batch: Batch, q, out, scale: Optional[float] = None, stream=None) -> None:
        """Attention of the planned batch's tokens over the cache; ``scale`` None: head_dim ** -0.5."""
        if cache is not batch._cache or cache.device != self.device:
            self._agree(cache, batch)
        shape = batch._q_shape
        rest = (*self._rows(q, cache, batch, shape, "q"), *self._rows(out, cache, batch, shape, "out"),
                cache.head_dim ** -0.5 if scale is None else scale, _stream_ptr(stream, self.device))
        if getattr(cache, "_scales", None) is None:
            status = self._lib.infaas_sel_exec_attend(self._h, cache._ref, batch._ref, *rest)
        else:
            status = self._lib.infaas_sel_exec_attend_scaled(self._h, cache._ref, cache._scales_ref, batch._ref, *rest)
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

    def beam(self, logits, scores, parent, token, score, *, ended=None, factor=None, end_token: int = -1, stream=None) -> None:
        """The best continuations of every query's beams: logits [queries * beams, vocab], ``scores`` [queries, beams], into
        ``parent``, ``token`` and ``score`` [queries, picks].  ``ended`` (int32) and ``factor`` (float32) are [queries, beams] or None."""
        torch = _use_torch()
        dev = self.device
        if not isinstance(logits, torch.Tensor) or logits.get_device() != dev or logits.dim() != 2 or logits.dtype not in _types() \
                or (logits.shape[1] > 1 and logits.stride(1) != 1):
            raise TypeError(f"logits: tensor [rows, vocab] on device {dev} expected, the last dimension consecutive")
        for name, t in (("scores", scores), ("token", token)):
            if not isinstance(t, torch.Tensor) or t.dim() != 2:
                raise TypeError(f"{name}: tensor of two dimensions expected")
        queries, beams = scores.shape
        picks, vocab = token.shape[1], logits.shape[1]
        if logits.shape[0] != queries * beams:
            raise TypeError(f"logits: {queries * beams} rows expected for scores {[queries, beams]}, not {logits.shape[0]}")

        def matrix(t, dtype, name, columns):
            if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.get_device() != dev or not t.is_contiguous() \
                    or tuple(t.shape) != (queries, columns):
                raise TypeError(f"{name}: contiguous {dtype} tensor {[queries, columns]} on device {dev} expected")
            _no_gradient(t, name)
            return t.data_ptr()

        _no_gradient(logits, "logits")
        f32, i32 = torch.float32, torch.int32
        status = self._lib.infaas_sel_exec_beam(
            self._h, _i32(queries, "queries"), _i32(beams, "beams"), _i32(vocab, "vocab"), _i32(picks, "picks"), _types()[logits.dtype],
            logits.data_ptr(), logits.stride(0), matrix(scores, f32, "scores", beams),
            None if ended is None else matrix(ended, i32, "ended", beams), None if factor is None else matrix(factor, f32, "factor", beams),
            _i32(end_token, "end_token"), matrix(parent, i32, "parent", picks), matrix(token, i32, "token", picks),
            matrix(score, f32, "score", picks), _stream_ptr(stream, self.device))
        if status:
            _check(status)

    def reserve_beam(self, queries: int, beams: int, vocab: int, picks: int, dtype) -> None:
        """Scratch memory for ``beam`` with these sizes, for calls that are recorded into a graph."""
        if dtype not in _types():
            raise TypeError(f"dtype {dtype}: float32, bfloat16 or float16")
        _check(self._lib.infaas_sel_exec_reserve_beam(self._h, _i32(queries, "queries"), _i32(beams, "beams"), _i32(vocab, "vocab"),
                                                      _i32(picks, "picks"), _types()[dtype]))

    def destroy(self) -> None:
        if self._h:
            self._lib.infaas_sel_exec_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass
