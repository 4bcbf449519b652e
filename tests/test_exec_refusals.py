"""What the executor's calls refuse: checked on the host before anything is enqueued, so no GPU is needed (every pointer
here is made up, and no call gets as far as using one)."""
import ctypes
import math
import os

import pytest

import paper_1905_13348_amd as pkg
from paper_1905_13348_amd import binding

pytestmark = pytest.mark.skipif(not os.path.exists(pkg.library_path()), reason="library not built here")

P = 0x10000    # stands for an aligned device pointer


def _cache(**kw):
    c = dict(d_k=P, d_v=P, type=1, kv_heads=2, head_dim=128, page_size=16, num_pages=8, page_stride=16 * 256, slot_stride=256,
             head_stride=128)
    c.update(kw)
    return binding._Cache(**c)


def _batch(**kw):
    b = dict(num_tokens=3, num_seqs=2, num_groups=1, heads=8, max_len=64, table_width=4, d_token_seq=P, d_token_pos=P,
             d_seq_start=P, d_seq_len=P, d_page_table=P, d_group_start=P, d_shared_len=P, d_plan=P, plan_bytes=1 << 30)
    b.update(kw)
    return binding._Batch(**b)


@pytest.fixture()
def lib():
    lib = pkg.load_library()
    h = ctypes.c_void_p()
    assert lib.infaas_sel_exec_create(0, ctypes.byref(h)) == 0 and h.value
    lib.h = h
    yield lib
    lib.infaas_sel_exec_destroy(h)


def _refused(lib, status, *words):
    text = lib.infaas_sel_last_error().decode()
    assert status == -1
    for w in words:
        assert w in text, text


BAD_CACHE = [(dict(type=0), "type"), (dict(type=3), "type"), (dict(kv_heads=0), "KV heads"), (dict(head_dim=96), "96"),
             (dict(page_size=0), "page size"), (dict(page_size=48), "48"), (dict(page_size=1 << 17), "page size")]
BAD_POOLS = [(dict(d_k=0), "pools"), (dict(d_v=P + 8), "pools"), (dict(num_pages=0), "pages"), (dict(slot_stride=132), "strides"),
             (dict(page_stride=1), "strides"), (dict(head_stride=127), "strides")]
BAD_SIZES = [(dict(num_tokens=-1), "negative"), (dict(num_seqs=-1), "negative"), (dict(max_len=-1), "negative"),
             (dict(table_width=-1), "negative"), (dict(num_groups=3), "groups"), (dict(heads=0), "heads"),
             (dict(heads=7), "7"), (dict(heads=2 * 129), "258")]
BAD_ARRAYS = [(dict(d_token_seq=0), "token"), (dict(d_token_pos=0), "token"), (dict(d_page_table=0), "page table")]
BAD_PLAN = [(dict(d_seq_start=0), "sequence"), (dict(d_seq_len=0), "sequence"), (dict(d_group_start=0), "group"),
            (dict(d_shared_len=0), "group"), (dict(d_plan=0), "plan"), (dict(d_plan=P + 4), "plan"), (dict(plan_bytes=100), "100")]


def test_create_and_null_handles(lib):
    h = ctypes.c_void_p()
    _refused(lib, lib.infaas_sel_exec_create(0, None), "null")
    _refused(lib, lib.infaas_sel_exec_create(-1, ctypes.byref(h)), "-1")
    lib.infaas_sel_exec_destroy(None)
    c, b, a = _cache(), _batch(), binding._AppendArgs()
    _refused(lib, lib.infaas_sel_exec_plan(None, c, b, None), "null")
    _refused(lib, lib.infaas_sel_exec_reserve(None, c, b), "null")
    _refused(lib, lib.infaas_sel_exec_append(None, c, b, a, None), "null")
    _refused(lib, lib.infaas_sel_exec_attend(None, c, b, P, 0, 0, P, 0, 0, 1.0, None), "null")
    _refused(lib, lib.infaas_sel_exec_sample(None, 1, 8, 0, P, 8, None, None, None, None, P, P, None, None), "null")


def _attend(lib, c, b, q=P, q_strides=(1024, 128), out=P, out_strides=(1024, 128), scale=0.1):
    return lib.infaas_sel_exec_attend(lib.h, c, b, q, *q_strides, out, *out_strides, scale, None)


def _append(lib, c, b, **kw):
    a = dict(d_q=P, d_k=P, d_v=P, d_q_out=P, q_token_stride=1024, q_head_stride=128, k_token_stride=256, k_head_stride=128,
             v_token_stride=256, v_head_stride=128, out_token_stride=1024, out_head_stride=128, d_freq=P, rot_dim=128, interleaved=0)
    a.update(kw)
    return lib.infaas_sel_exec_append(lib.h, c, b, binding._AppendArgs(**a), None)


@pytest.mark.parametrize("bad, word", BAD_CACHE + BAD_POOLS)
def test_caches(lib, bad, word):
    c = _cache(**bad)
    _refused(lib, _attend(lib, c, _batch()), "cache", word)
    _refused(lib, _append(lib, c, _batch()), "cache", word)
    if (bad, word) in BAD_CACHE:
        _refused(lib, lib.infaas_sel_exec_plan(lib.h, c, _batch(), None), "cache", word)
        assert lib.infaas_sel_exec_plan_bytes(c, _batch()) == 0


@pytest.mark.parametrize("bad, word", BAD_SIZES + BAD_ARRAYS + BAD_PLAN)
def test_batches(lib, bad, word):
    c, b = _cache(), _batch(**bad)
    _refused(lib, _attend(lib, c, b), "batch", word)
    _refused(lib, lib.infaas_sel_exec_plan(lib.h, c, b, None), "batch", word)
    if (bad, word) not in BAD_PLAN:
        _refused(lib, _append(lib, c, b), "batch", word)
    if (bad, word) in BAD_SIZES:
        assert lib.infaas_sel_exec_plan_bytes(c, b) == 0
        _refused(lib, lib.infaas_sel_exec_reserve(lib.h, c, b), "batch", word)


def test_null_structures(lib):
    _refused(lib, _attend(lib, None, _batch()), "cache")
    _refused(lib, _attend(lib, _cache(), None), "batch")
    _refused(lib, lib.infaas_sel_exec_append(lib.h, _cache(), _batch(), None, None), "append")


@pytest.mark.parametrize("kw, word", [(dict(q=0), "null"), (dict(out=0), "null"), (dict(q=P + 2), "aligned"), (dict(out=P + 8), "aligned"),
                                      (dict(q_strides=(1023, 128)), "strides"), (dict(out_strides=(1024, 12)), "strides"),
                                      (dict(scale=0.0), "scale"), (dict(scale=-1.0), "scale"), (dict(scale=math.nan), "scale"),
                                      (dict(scale=math.inf), "scale")])
def test_attend(lib, kw, word):
    _refused(lib, _attend(lib, _cache(), _batch(), **kw), "attend", word)


@pytest.mark.parametrize("kw, word", [(dict(rot_dim=-16), "rotated"), (dict(rot_dim=144), "144"), (dict(rot_dim=24), "24"),
                                      (dict(d_freq=0), "frequencies"), (dict(d_q=0), "output"), (dict(d_q_out=0), "output"),
                                      (dict(d_k=0), "null"), (dict(d_v=P + 2), "aligned"), (dict(d_q=P + 2), "aligned"),
                                      (dict(k_token_stride=257), "strides"), (dict(out_head_stride=4), "strides")])
def test_append(lib, kw, word):
    _refused(lib, _append(lib, _cache(), _batch(), **kw), "append", word)


@pytest.mark.parametrize("kw, word", [(dict(rows=-1), "rows"), (dict(vocab=0), "vocabulary"), (dict(vocab=(1 << 20) + 1), "vocabulary"),
                                      (dict(type=5), "type"), (dict(logits=0), "null"), (dict(draw=0), "null"), (dict(token=0), "null"),
                                      (dict(logits=P + 2), "aligned"), (dict(type=1, logits=P + 1), "aligned")])
def test_sample(lib, kw, word):
    a = dict(rows=2, vocab=100, type=0, logits=P, draw=P, token=P)
    a.update(kw)
    _refused(lib, lib.infaas_sel_exec_sample(lib.h, a["rows"], a["vocab"], a["type"], a["logits"], 100, None, None, None, None,
                                             a["draw"], a["token"], None, None), "sample", word)


def test_too_many_tokens(lib):
    """Partial rows are counted in 32 bits."""
    b = _batch(num_tokens=1 << 29, heads=8)
    assert lib.infaas_sel_exec_plan_bytes(_cache(), b) == 0
    _refused(lib, _attend(lib, _cache(), b), "too many")


def test_empty_calls_are_no_ops(lib):
    """No token, no row: nothing is enqueued (and none of the made-up pointers used)."""
    c, b = _cache(), _batch(num_tokens=0)
    assert lib.infaas_sel_exec_plan(lib.h, c, b, None) == 0
    assert _append(lib, c, b) == 0
    assert _attend(lib, c, b) == 0
    assert lib.infaas_sel_exec_sample(lib.h, 0, 100, 0, None, 100, None, None, None, None, None, None, None, None) == 0


def test_python_side_refuses_shapes_and_types():
    import torch
    x = torch.zeros(2, 16, 2, 128, dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        pkg.PagedCache(x, x)           # not on a device
    with pytest.raises(ValueError):
        pkg.PagedCache(x, x, layout="other")


@pytest.mark.parametrize("name", ["page_stride", "slot_stride", "head_stride"])
def test_negative_strides_of_a_cache(lib, name):
    _refused(lib, _attend(lib, _cache(**{name: -256}), _batch()), "cache", "negative")
    _refused(lib, _append(lib, _cache(**{name: -256}), _batch()), "cache", "negative")


def test_caches_of_other_sizes_than_the_batch():
    """Shapes are checked by the batch's sizes, so the cache of a call has to have them."""
    from types import SimpleNamespace
    ex = pkg.Executor()
    made_for = SimpleNamespace(_sizes=(2, 128, 16), _ref=None)
    batch = SimpleNamespace(_sizes=made_for._sizes, _cache=made_for, _q_shape=(3, 8, 128), _kv_shape=(3, 2, 128), _ref=None)
    for sizes in ((4, 128, 16), (2, 64, 16), (2, 128, 32)):
        cache = SimpleNamespace(_sizes=sizes, _ref=None)
        with pytest.raises(ValueError, match="KV heads"):
            ex.append(cache, batch, None, None, None, None)
        with pytest.raises(ValueError, match="KV heads"):
            ex.attend(cache, batch, None, None)
        with pytest.raises(ValueError, match="KV heads"):
            ex.reserve(cache, batch)
