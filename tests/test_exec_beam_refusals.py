"""What infaas_sel_exec_beam refuses, on the host: every pointer here is made up, and no call gets as far as using one."""
import os

import pytest
import torch

import paper_1905_13348_amd as pkg
from test_exec_refusals import P, _refused, lib  # noqa: F401
from test_exec_scaled_refusals import _on0

pytestmark = pytest.mark.skipif(not os.path.exists(pkg.library_path()), reason="library not built here")

GOOD = dict(queries=2, beams=4, vocab=100, picks=8, type=1, logits=P, stride=100, scores=P, ended=P, factor=P, end=5, parent=P, token=P, score=P)


def _beam(lib, h=True, **kw):
    a = dict(GOOD, **kw)
    return lib.infaas_sel_exec_beam(lib.h if h else None, a["queries"], a["beams"], a["vocab"], a["picks"], a["type"], a["logits"], a["stride"], a["scores"],
                                    a["ended"], a["factor"], a["end"], a["parent"], a["token"], a["score"], None)


SIZES = [(dict(queries=-1), "queries"), (dict(beams=0), "beams"), (dict(beams=65), "65"), (dict(picks=0), "picks"), (dict(picks=65), "65"),
         (dict(vocab=0), "vocabulary"), (dict(vocab=(1 << 20) + 1), "1048577"), (dict(type=3), "type"), (dict(type=-1), "type"),
         (dict(queries=1 << 30), "queries")]


@pytest.mark.parametrize("bad, word", SIZES + [
    (dict(end=-1), "end token"), (dict(end=100), "end token"), (dict(logits=0), "null"), (dict(scores=0), "null"), (dict(parent=0), "null"),
    (dict(token=0), "null"), (dict(score=0), "null"), (dict(logits=P + 1), "aligned"), (dict(logits=P + 2, type=0), "aligned")])
def test_arguments(lib, bad, word):  # noqa: F811
    _refused(lib, _beam(lib, **bad), "beam", word)


@pytest.mark.parametrize("bad, word", SIZES)
def test_reserve(lib, bad, word):  # noqa: F811
    a = dict(GOOD, **bad)
    _refused(lib, lib.infaas_sel_exec_reserve_beam(lib.h, a["queries"], a["beams"], a["vocab"], a["picks"], a["type"]), "beam", word)


def test_null_and_nothing(lib):  # noqa: F811
    _refused(lib, _beam(lib, h=False), "executor")
    _refused(lib, lib.infaas_sel_exec_reserve_beam(None, 1, 1, 1, 1, 0), "executor")
    assert _beam(lib, queries=0) == 0
    assert _beam(lib, queries=0, ended=None, end=-1) == 0


def _arrays():
    z = lambda dtype, *shape: _on0(torch.zeros(shape, dtype=dtype))
    return dict(logits=z(torch.bfloat16, 8, 50), scores=z(torch.float32, 2, 4), parent=z(torch.int32, 2, 6), token=z(torch.int32, 2, 6),
                score=z(torch.float32, 2, 6), ended=z(torch.int32, 2, 4), factor=z(torch.float32, 2, 4))


@pytest.mark.parametrize("name, change", [
    ("logits", lambda t: t.float()[:6]), ("logits", lambda t: t.int()), ("logits", lambda t: t[0]), ("logits", lambda t: _on0(torch.zeros(50, 8)).t()),
    ("logits", lambda t: None), ("logits", lambda t: torch.zeros(8, 50)), ("scores", lambda t: t.double()), ("scores", lambda t: t.view(8)), ("scores", lambda t: 1.0),
    ("parent", lambda t: t[:, :4]), ("parent", lambda t: t.long()), ("token", lambda t: t[:1]), ("token", lambda t: None), ("score", lambda t: t.int()),
    ("ended", lambda t: t.bool()), ("ended", lambda t: t[:, :3]), ("factor", lambda t: t.double()), ("factor", lambda t: _on0(torch.zeros(4, 2)).t())])
def test_binding(name, change):
    a = _arrays()
    a[name] = change(a[name])
    ex = pkg.Executor()
    with pytest.raises(TypeError):
        ex.beam(a.pop("logits"), a.pop("scores"), a.pop("parent"), a.pop("token"), a.pop("score"), **a, end_token=1, stream=0)
    ex.destroy()


@pytest.mark.parametrize("name", ["logits", "scores", "score", "factor"])
def test_gradients(name):
    a = _arrays()
    a[name] = a[name].clone().as_subclass(type(a[name])).requires_grad_()
    ex = pkg.Executor()
    with pytest.raises(RuntimeError, match="gradient"):
        ex.beam(a.pop("logits"), a.pop("scores"), a.pop("parent"), a.pop("token"), a.pop("score"), **a, end_token=1, stream=0)
    ex.destroy()


def test_reserve_of_another_type():
    ex = pkg.Executor()
    with pytest.raises(TypeError):
        ex.reserve_beam(1, 1, 10, 1, torch.float64)
    ex.destroy()
