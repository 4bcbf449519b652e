"""What the calls on a cache of 8 bits refuse, on the host: every pointer here is made up, and no call gets as far as using one."""
import ctypes
import os

import pytest
import torch

import paper_1905_13348_amd as pkg
from paper_1905_13348_amd import binding
from test_exec_refusals import BAD_ARRAYS, BAD_CACHE, BAD_POOLS, BAD_SIZES, P, _batch, _cache, _refused, lib  # noqa: F401

pytestmark = pytest.mark.skipif(not os.path.exists(pkg.library_path()), reason="library not built here")


def _scales(**kw):
    s = dict(d_k_scale=P, d_v_scale=P + 1, block=8, page_stride=4, block_stride=2, head_stride=1)
    s.update(kw)
    return binding._Scales(**s)


def _attend(lib, c, s, b, q=P, scale=0.1):
    return lib.infaas_sel_exec_attend_scaled(lib.h, c, s, b, q, 1024, 128, P, 1024, 128, scale, None)


def _append(lib, c, s, b, **kw):
    a = dict(d_q=P, d_k=P, d_v=P, d_q_out=P, q_token_stride=1024, q_head_stride=128, k_token_stride=256, k_head_stride=128,
             v_token_stride=256, v_head_stride=128, out_token_stride=1024, out_head_stride=128, d_freq=P, rot_dim=128, interleaved=0)
    a.update(kw)
    return lib.infaas_sel_exec_append_scaled(lib.h, c, s, b, binding._AppendArgs(**a), None)


def _read(lib, c, s, b, k=P, v=P, strides=(256, 128, 256, 128)):
    return lib.infaas_sel_exec_read(lib.h, c, s, b, k, strides[0], strides[1], v, strides[2], strides[3], None)


BAD_SCALES = [(dict(d_k_scale=0), "null"), (dict(d_v_scale=0), "null"), (dict(block=0), "block"), (dict(block=-8), "block"), (dict(block=12), "12"),
              (dict(block=32), "32"), (dict(page_stride=-1), "negative"), (dict(block_stride=-1), "negative"), (dict(head_stride=-1), "negative")]


@pytest.mark.parametrize("bad, word", BAD_SCALES)
def test_scales(lib, bad, word):  # noqa: F811
    for call in (_attend, _append, _read):
        _refused(lib, call(lib, _cache(), _scales(**bad), _batch()), "scales", word)


def test_null(lib):  # noqa: F811
    for call in (_attend, _append):
        _refused(lib, call(lib, _cache(), None, _batch()), "scales")
    for call in (_attend, _append, _read):
        _refused(lib, call(lib, None, _scales(), _batch()), "cache")
        _refused(lib, call(lib, _cache(), _scales(), None), "batch")
    c, s, b = _cache(), _scales(), _batch()
    _refused(lib, lib.infaas_sel_exec_attend_scaled(None, c, s, b, P, 0, 0, P, 0, 0, 1.0, None), "null")
    _refused(lib, lib.infaas_sel_exec_append_scaled(None, c, s, b, binding._AppendArgs(), None), "null")
    _refused(lib, lib.infaas_sel_exec_append_scaled(lib.h, c, s, b, None, None), "append")
    _refused(lib, lib.infaas_sel_exec_read(None, c, s, b, P, 0, 0, P, 0, 0, None), "null")


@pytest.mark.parametrize("bad, word", BAD_CACHE + BAD_POOLS + [(dict(page_stride=8), "16"), (dict(slot_stride=136), "16"), (dict(head_stride=8), "16")])
def test_caches(lib, bad, word):  # noqa: F811
    for call in (_attend, _append, _read):
        _refused(lib, call(lib, _cache(**bad), _scales(), _batch()), "cache", word)


@pytest.mark.parametrize("bad, word", BAD_SIZES + BAD_ARRAYS)
def test_batches(lib, bad, word):  # noqa: F811
    for call in (_attend, _append, _read):
        _refused(lib, call(lib, _cache(), _scales(), _batch(**bad)), "batch", word)


def test_rows(lib):  # noqa: F811
    _refused(lib, _append(lib, _cache(), _scales(), _batch(d_seq_start=0)), "batch", "sequence")
    _refused(lib, _append(lib, _cache(), _scales(), _batch(), rot_dim=24), "append", "24")
    _refused(lib, _append(lib, _cache(), _scales(), _batch(), k_token_stride=12), "append", "strides")
    _refused(lib, _attend(lib, _cache(), _scales(), _batch(), q=P + 2), "attend", "aligned")
    _refused(lib, _attend(lib, _cache(), _scales(), _batch(), scale=0.0), "attend", "scale")
    for kw in (dict(k=0), dict(v=0), dict(k=P + 8)):
        _refused(lib, _read(lib, _cache(), _scales(), _batch(), **kw), "read", "aligned")
        _refused(lib, _read(lib, _cache(), None, _batch(), **kw), "read", "aligned")
    for i in range(4):
        strides = [256, 128, 256, 128]
        strides[i] = 12
        _refused(lib, _read(lib, _cache(), None, _batch(), strides=strides), "read", "strides")


def test_batches_without_tokens(lib):  # noqa: F811
    b = _batch(num_tokens=0)
    for call in (_attend, _append, _read):
        assert call(lib, _cache(), _scales(), b) == 0


# ---- the binding ------------------------------------------------------------------------------------------------

class _There(torch.Tensor):
    """A tensor that says that it is on device 0."""
    is_cuda = property(lambda self: True)

    def get_device(self):
        return 0


def _on0(t):
    return t.as_subclass(_There)


def _pools(layout="token", dtype=torch.float8_e4m3fn):
    shape = (3, 16, 2, 64) if layout == "token" else (3, 2, 16, 64)
    return [_on0(torch.zeros(shape, dtype=torch.uint8).view(dtype) if dtype.itemsize == 1 else torch.zeros(shape, dtype=dtype)) for _ in range(2)]


def _scale(*shape, dtype=torch.float8_e8m0fnu):
    return _on0(torch.zeros(shape, dtype=torch.uint8).view(dtype))


def test_a_cache_of_both_layouts():
    c = pkg.PagedCache(*_pools(), k_scale=_scale(3, 4, 2), v_scale=_scale(3, 4, 2))
    assert c.dtype == torch.bfloat16 and c._scales.block == 4 and (c._scales.page_stride, c._scales.block_stride, c._scales.head_stride) == (8, 2, 1)
    c = pkg.PagedCache(*_pools("head"), layout="head", k_scale=_scale(3, 2, 1), v_scale=_scale(3, 2, 1), dtype=torch.float16)
    assert c.dtype == torch.float16 and c._scales.block == 16 and (c._scales.page_stride, c._scales.block_stride, c._scales.head_stride) == (2, 0, 1)


@pytest.mark.parametrize("change", [
    lambda a: a.update(v_scale=None), lambda a: a.update(k_scale=None), lambda a: a.update(k_scale=[1]), lambda a: a.update(k_scale=_scale(3, 4)),
    lambda a: a.update(v_scale=_scale(3, 2, 2)), lambda a: a.update(k_scale=_scale(3, 3, 2), v_scale=_scale(3, 3, 2)),
    lambda a: a.update(k_scale=_scale(2, 4, 2), v_scale=_scale(2, 4, 2)), lambda a: a.update(k_scale=_scale(3, 4, 1), v_scale=_scale(3, 4, 1)),
    lambda a: a.update(k_scale=_scale(3, 0, 2), v_scale=_scale(3, 0, 2)), lambda a: a.update(k_scale=_scale(3, 32, 2), v_scale=_scale(3, 32, 2)),
    lambda a: a.update(k_scale=_scale(3, 4, 2, dtype=torch.uint8)), lambda a: a.update(dtype=torch.float32), lambda a: a.update(dtype=torch.float8_e4m3fn),
    lambda a: a.update(zip(("k_pool", "v_pool"), _pools(dtype=torch.bfloat16))), lambda a: a.update(v_pool=_pools(dtype=torch.float8_e5m2)[0]),
    lambda a: a.update(k_scale=torch.zeros((3, 4, 2), dtype=torch.uint8).view(torch.float8_e8m0fnu)),
    lambda a: a.update(v_scale=_scale(3, 2, 4).transpose(1, 2)), lambda a: (a.pop("k_scale"), a.pop("v_scale"))])
def test_a_cache_that_is_refused(change):
    k, v = _pools()
    a = dict(k_pool=k, v_pool=v, k_scale=_scale(3, 4, 2), v_scale=_scale(3, 4, 2))
    change(a)
    with pytest.raises(TypeError):
        pkg.PagedCache(**a)


def test_a_dtype_that_is_not_the_pools():
    k, v = _pools(dtype=torch.bfloat16)
    assert pkg.PagedCache(k, v, dtype=torch.bfloat16).dtype == torch.bfloat16
    with pytest.raises(TypeError):
        pkg.PagedCache(k, v, dtype=torch.float16)
