"""What the Python side of tables, copies, reading and caches of 8 bits refuses, and what reaches the library.  No GPU is needed: host
tensors stand for those of a device, and a library that remembers its calls for the real one."""
from types import SimpleNamespace

import pytest
import torch

import paper_1905_13348_amd as pkg
from paper_1905_13348_amd import binding
from test_exec_binding import _arrays, _cache

i32 = lambda *a: torch.tensor(a, dtype=torch.int32)


@pytest.fixture()
def worker(monkeypatch):
    ex = pkg.Executor(0)
    calls = []
    record = lambda name: lambda *a: calls.append((name, a)) or 0
    names = ("append", "append_scaled", "attend", "attend_scaled", "read", "advance", "copy", "beam", "reserve_beam")
    real = ex._lib
    ex._lib = SimpleNamespace(**{f"infaas_sel_exec_{n}": record(n) for n in names}, infaas_sel_exec_destroy=real.infaas_sel_exec_destroy)
    ex.device = -1
    binding._use_torch()
    monkeypatch.setattr(binding, "_raw_stream", lambda d: 1000 + d)
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    return ex, calls


def _table(device=-1):
    c = binding._Table(num_seqs=2)
    return SimpleNamespace(device=device, num_seqs=2, _c=c, _ref=binding.ctypes.byref(c))


def _coded(device=-1):
    cache = _cache(device)
    cache._scales = binding._Scales(block=4)
    cache._scales_ref = binding.ctypes.byref(cache._scales)
    return cache


def test_advance(worker):
    ex, calls = worker
    ex.advance(_table(), i32(1, -2))
    ex.advance(_table(), i32(1, -2), i32(0, 0), stream=SimpleNamespace(cuda_stream=7))
    assert [c[0] for c in calls] == ["advance"] * 2 and calls[0][1][3] is None and calls[1][1][3]
    for new, parent in ((i32(1), None), (i32(1, 2).long(), None), (None, None), ([1, 2], None), (i32(1, 2, 3, 4)[::2], None), (i32(1, 2), i32(1)),
                        (i32(1, 2), i32(1, 2).float()), (i32(1, 2).view(1, 2), None)):
        with pytest.raises(TypeError):
            ex.advance(_table(), new, parent)
    with pytest.raises(ValueError):
        ex.advance(_table(1), i32(1, 2))
    assert len(calls) == 2


def test_copy(worker):
    ex, calls = worker
    ex.copy(_cache(), _table())
    ex.copy(_coded(), _table())
    assert calls[0][1][2] is None and calls[1][1][2] is not None
    for cache, table in ((_cache(1), _table()), (_cache(), _table(1)), (_coded(1), _table(1))):
        with pytest.raises(ValueError):
            ex.copy(cache, table)
    assert len(calls) == 2


@pytest.mark.parametrize("coded", [False, True])
def test_what_a_cache_is_decides_the_call(worker, coded):
    ex, calls = worker
    cache = _coded() if coded else _cache()
    batch = pkg.Batch(cache, 4, **_arrays())
    q, k = torch.zeros(3, 4, 64, dtype=torch.bfloat16), torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    ex.append(cache, batch, q, k, k, q, torch.zeros(32, dtype=torch.float64))
    ex.attend(cache, batch, q, torch.zeros_like(q))
    ex.read(cache, batch, k, torch.zeros_like(k))
    assert [c[0] for c in calls] == (["append_scaled", "attend_scaled", "read"] if coded else ["append", "attend", "read"])
    assert (calls[2][1][2] is not None) == coded


@pytest.mark.parametrize("name", ["k", "v"])
@pytest.mark.parametrize("change", [lambda t: t.float(), lambda t: t[:2], lambda t: None, lambda t: torch.zeros(3, 64, 2, dtype=t.dtype).transpose(1, 2)])
def test_read(worker, name, change):
    ex, calls = worker
    cache = _coded()
    batch = pkg.Batch(cache, 4, **_arrays())
    t = {n: torch.zeros(3, 2, 64, dtype=torch.bfloat16) for n in ("k", "v")}
    t[name] = change(t[name])
    with pytest.raises(TypeError, match=name):
        ex.read(cache, batch, **t)
    assert not calls


def test_read_with_a_batch_of_another_cache(worker):
    ex, calls = worker
    batch = pkg.Batch(_cache(), 4, **_arrays())
    k = torch.zeros(3, 1, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        ex.read(_cache(heads=1), batch, k, k)
    with pytest.raises(ValueError):
        ex.read(_cache(device=1), batch, k, k)
    assert not calls


def test_read_into_what_needs_a_gradient(worker):
    ex, calls = worker
    batch = pkg.Batch(_cache(), 4, **_arrays())
    k = torch.zeros(3, 2, 64, dtype=torch.bfloat16, requires_grad=True)
    with pytest.raises(RuntimeError, match="gradient"):
        ex.read(batch._cache, batch, k, torch.zeros(3, 2, 64, dtype=torch.bfloat16))
    assert not calls


def test_beam_sizes_beyond_32_bits(worker):
    ex, calls = worker
    wide = torch.empty((2, 2 ** 31), dtype=torch.float32, device="meta")
    out = [torch.zeros((2, 1), dtype=d) for d in (torch.int32, torch.int32, torch.float32)]
    with pytest.raises((ValueError, TypeError)):
        ex.beam(wide, torch.zeros(2, 1), *out)
    with pytest.raises(ValueError):
        ex.reserve_beam(2 ** 31, 1, 10, 1, torch.float32)
    assert not calls
