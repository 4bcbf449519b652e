"""What the executor's Python side refuses before the library is called.  No GPU is needed: host tensors stand for those of
a device (they are on device -1 as torch counts), and a tensor class of another device's number for those of a second one."""
from types import SimpleNamespace

import pytest
import torch

import paper_1905_13348_amd as pkg
from paper_1905_13348_amd import binding


class Elsewhere(torch.Tensor):
    """A tensor that says it is on device 1."""
    is_cuda = property(lambda self: True)

    def get_device(self):
        return 1


def _elsewhere(t):
    return t.as_subclass(Elsewhere)


def _cache(device=-1, heads=2, dim=64):
    c = binding._Cache(d_k=0x10000, d_v=0x10000, type=1, kv_heads=heads, head_dim=dim, page_size=16, num_pages=4, page_stride=16 * heads * dim,
                       slot_stride=heads * dim, head_stride=dim)
    return SimpleNamespace(_c=c, _ref=binding.ctypes.byref(c), _sizes=(heads, dim, 16), kv_heads=heads, head_dim=dim, page_size=16,
                           device=device, dtype=torch.bfloat16)


def _arrays(**kw):
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32)
    a = dict(token_seq=i32(0, 0, 1), token_pos=i32(0, 1, 0), seq_start=i32(0, 2, 3), seq_len=i32(2, 1), page_table=i32(0, 1, 2, 3).view(2, 2),
             group_start=i32(0, 2), shared_len=i32(0))
    a.update(kw)
    return a


def _executor(monkeypatch, device=-1):
    """An executor whose library answers every call with 0 and remembers them."""
    ex = pkg.Executor(0)
    calls = []
    record = lambda name: lambda *a: calls.append((name, a)) or 0
    names = ("reserve", "plan", "append", "attend", "sample")
    ex._lib = SimpleNamespace(**{f"infaas_sel_exec_{n}": record(n) for n in names}, infaas_sel_exec_destroy=ex._lib.infaas_sel_exec_destroy)
    ex.device = device
    binding._use_torch()
    monkeypatch.setattr(binding, "_raw_stream", lambda d: 1000 + d)
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    return ex, calls


def _step(ex, cache, batch, **kw):
    """Every call of a step; tensors of kw instead of the usual ones."""
    t = dict(q=torch.zeros(3, 4, 64, dtype=torch.bfloat16), k=torch.zeros(3, 2, 64, dtype=torch.bfloat16),
             v=torch.zeros(3, 2, 64, dtype=torch.bfloat16), q_out=torch.zeros(3, 4, 64, dtype=torch.bfloat16),
             out=torch.zeros(3, 4, 64, dtype=torch.bfloat16), freq=torch.zeros(32, dtype=torch.float64))
    t.update(kw)
    ex.append(cache, batch, t["q"], t["k"], t["v"], t["q_out"], t["freq"])
    ex.attend(cache, batch, t["q"], t["out"])


LIMITS = {"temperature": torch.float32, "top_k": torch.int32, "top_p": torch.float32, "min_p": torch.float32}


def _sample(ex, **kw):
    t = {"logits": torch.zeros(2, 50), "draws": torch.zeros(2), "token": torch.zeros(2, dtype=torch.int32), "prob": torch.zeros(2)}
    t.update({k: torch.ones(2, dtype=d) for k, d in LIMITS.items()})
    t.update(kw)
    ex.sample(t["logits"], t["draws"], t["token"], t["prob"], **{k: t[k] for k in LIMITS})


def test_calls_that_are_fine(monkeypatch):
    ex, calls = _executor(monkeypatch)
    cache = _cache()
    batch = pkg.Batch(cache, 4, **_arrays())
    ex.reserve(cache, batch)
    ex.plan(batch)
    _step(ex, cache, batch)
    _sample(ex)
    assert [c[0] for c in calls] == ["reserve", "plan", "append", "attend", "sample"]


def test_pools_on_two_devices():
    x = torch.zeros(2, 16, 2, 64, dtype=torch.bfloat16)
    on_device_0 = type("Device0", (Elsewhere,), {"get_device": lambda self: 0})
    with pytest.raises(TypeError, match="one device"):
        pkg.PagedCache(x.as_subclass(on_device_0), _elsewhere(x))
    assert pkg.PagedCache(_elsewhere(x), _elsewhere(x)).device == 1


@pytest.mark.parametrize("name", ["token_seq", "token_pos", "seq_start", "seq_len", "page_table", "group_start", "shared_len"])
def test_arrays_on_another_device_than_the_cache(name):
    with pytest.raises(TypeError, match=name):
        pkg.Batch(_cache(), 4, **_arrays(**{name: _elsewhere(_arrays()[name])}))


def test_a_cache_or_a_batch_of_another_device(monkeypatch):
    ex, calls = _executor(monkeypatch)
    here, there = _cache(), _cache(device=1)
    batch = pkg.Batch(here, 4, **_arrays())
    other = pkg.Batch(there, 4, **{k: _elsewhere(v) for k, v in _arrays().items()})
    for cache, b in ((there, batch), (here, other), (there, other)):
        for call in (lambda: ex.reserve(cache, b), lambda: ex.append(cache, b, None, None, None, None), lambda: ex.attend(cache, b, None, None)):
            with pytest.raises(ValueError, match="device"):
                call()
    with pytest.raises(ValueError, match="device"):
        ex.plan(other)
    assert calls == []


@pytest.mark.parametrize("name", ["q", "k", "v", "q_out", "out", "freq"])
def test_tensors_of_a_step_on_another_device(monkeypatch, name):
    ex, calls = _executor(monkeypatch)
    cache = _cache()
    batch = pkg.Batch(cache, 4, **_arrays())
    shape = (32,) if name == "freq" else (3, 2 if name in "kv" else 4, 64)
    t = torch.zeros(shape, dtype=torch.float64 if name == "freq" else torch.bfloat16)
    with pytest.raises(TypeError, match=name):
        _step(ex, cache, batch, **{name: _elsewhere(t)})
    assert len(calls) == (1 if name == "out" else 0)


@pytest.mark.parametrize("name", ["logits", "draws", "token", "prob", *LIMITS])
def test_tensors_of_a_draw_on_another_device(monkeypatch, name):
    ex, calls = _executor(monkeypatch)
    t = torch.zeros((2, 50) if name == "logits" else 2, dtype=torch.int32 if name == "token" else LIMITS.get(name, torch.float32))
    with pytest.raises(TypeError, match=name):
        _sample(ex, **{name: _elsewhere(t)})
    assert calls == []


def test_streams(monkeypatch):
    """Without a stream a call goes to the current stream of the executor's device, whichever device is current; a stream of
    another device is refused."""
    ex, calls = _executor(monkeypatch)
    monkeypatch.setattr(binding, "_current_device", lambda: 7)
    batch = pkg.Batch(_cache(), 4, **_arrays())
    ex.plan(batch)
    assert calls[-1][1][-1] == 999
    ex.plan(batch, stream=SimpleNamespace(cuda_stream=5, device_index=-1))
    assert calls[-1][1][-1] == 5
    with pytest.raises(ValueError, match="stream of device 1"):
        ex.plan(batch, stream=SimpleNamespace(cuda_stream=5, device_index=1))
    assert len(calls) == 2


@pytest.mark.parametrize("value", [2 ** 32 + 8, 2 ** 31, -2 ** 31 - 8, 2 ** 40])
def test_sizes_beyond_32_bits(monkeypatch, value):
    """They would reach the library cut to 32 bits: 2^32 + 8 query heads as 8."""
    with pytest.raises(ValueError, match="heads"):
        pkg.Batch(_cache(), value, **_arrays())
    with pytest.raises(ValueError, match="max_len"):
        pkg.Batch(_cache(), 4, max_len=value, **_arrays())
    with pytest.raises(ValueError, match="device"):
        pkg.Executor(value)


@pytest.mark.parametrize("size", [2 ** 32 + 8, 2 ** 31])
def test_tensors_of_more_elements_than_32_bits(monkeypatch, size):
    """(Of no memory: what they are refused for is looked at first.)"""
    wide = lambda *shape, dtype=torch.int32: torch.empty(shape, dtype=dtype, device="meta")
    ex, calls = _executor(monkeypatch)
    with pytest.raises(ValueError, match="vocab"):
        _sample(ex, logits=wide(2, size, dtype=torch.float32))
    with pytest.raises(ValueError, match="rows"):
        _sample(ex, logits=wide(size, 50, dtype=torch.float32))
    with pytest.raises(ValueError, match="page_table"):
        pkg.Batch(_cache(), 4, **_arrays(page_table=wide(2, size)))
    with pytest.raises(ValueError, match="token_seq"):
        pkg.Batch(_cache(), 4, **_arrays(token_seq=wide(size)))
    assert calls == []


@pytest.mark.parametrize("name", ["q", "k", "v", "q_out", "out", "freq", "logits", "pool"])
def test_inputs_that_require_a_gradient(monkeypatch, name):
    """Refused where gradients are recorded, by name; taken where they are not."""
    ex, calls = _executor(monkeypatch)
    cache = _cache()
    batch = pkg.Batch(cache, 4, **_arrays())
    if name == "logits":
        t = torch.zeros(2, 50, requires_grad=True)
        call = lambda: _sample(ex, logits=t)
    elif name == "pool":
        t = _elsewhere(torch.zeros(2, 16, 2, 64, dtype=torch.bfloat16)).requires_grad_()
        call = lambda: pkg.PagedCache(t.detach(), t)
    else:
        t = torch.zeros((32,) if name == "freq" else (3, 2 if name in "kv" else 4, 64),
                        dtype=torch.float64 if name == "freq" else torch.bfloat16, requires_grad=True)
        call = lambda: _step(ex, cache, batch, **{name: t})
    with pytest.raises(RuntimeError, match=f"{name}.* requires a gradient"):
        call()
    assert len(calls) == (1 if name == "out" else 0)
    with torch.no_grad():
        call()


@pytest.mark.parametrize("what", [None, [0, 1], 3.0])
def test_what_is_no_tensor(monkeypatch, what):
    """Named, as a wrong type is."""
    ex, calls = _executor(monkeypatch)
    cache = _cache()
    batch = pkg.Batch(cache, 4, **_arrays())
    for name in ("token_seq", "token_pos", "seq_start", "seq_len", "page_table"):
        with pytest.raises(TypeError, match=name):
            pkg.Batch(cache, 4, **_arrays(**{name: what}))
    for name in ("k", "v", "out") + (("q", "q_out", "freq") if what is not None else ()):      # (None: without queries, not rotated)
        calls.clear()
        with pytest.raises(TypeError, match=name):
            _step(ex, cache, batch, **{name: what})
        assert len(calls) == (1 if name == "out" else 0)
    for name in ("logits", "draws", "token"):
        with pytest.raises(TypeError, match=name):
            _sample(ex, **{name: what})
    with pytest.raises(TypeError):
        pkg.PagedCache(what, torch.zeros(2, 16, 2, 64, dtype=torch.bfloat16))
    if what is not None:
        with pytest.raises(TypeError, match="shared_len"):
            pkg.Batch(cache, 4, **_arrays(shared_len=what))


def test_pools_with_dimensions_of_one_element():
    """Their strides mean nothing: neither compared nor asked to be multiples of 8."""
    k = _elsewhere(torch.zeros(1, 16, 1, 64, dtype=torch.bfloat16))
    v = _elsewhere(torch.zeros(16 * 64, dtype=torch.bfloat16).as_strided((1, 16, 1, 64), (5, 64, 3, 1)))
    c = pkg.PagedCache(k, v)._c
    assert (c.page_stride, c.slot_stride, c.head_stride) == (0, 64, 0)
    c = pkg.PagedCache(v, k, layout="head")._c
    assert (c.page_stride, c.slot_stride, c.head_stride) == (0, 0, 64)
    with pytest.raises(TypeError, match="strides"):
        pkg.PagedCache(k, _elsewhere(torch.zeros(2048, dtype=torch.bfloat16).as_strided((1, 16, 1, 64), (5, 72, 3, 1))))
