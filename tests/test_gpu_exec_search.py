"""The executor's calls of beam search together: examples/search_answers.py, its picks against the definition, its logits against
the same decoder in 32 bits without a cache."""
import importlib.util
import os
import sys

import numpy as np
import pytest
import torch

from test_gpu_exec_beam import reference
from test_gpu_exec_example import _dense

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "search_answers.py")


def _example():
    spec = importlib.util.spec_from_file_location("search_answers", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("beams", [1, 3, 5])
def test_search(bits, beams):
    """Each step's picks are the definition's for its logits; the logits are those of the beam's own history.  For 16 bits the
    tolerance is the decoder's (some twenty roundings to bf16: 1%, and twice that); of 8 bits a key's or value's rounding is 2.6%
    rms (2^-4 at the most, by where in a power of two it falls), which moves a weight's logarithm by as much, and the result by both:
    3.7% of a layer's attention, 5.2% of two, and with the roundings three times that."""
    m = _example()
    sys.modules.setdefault("search_answers", m)
    v = m.Variant(vocab=300, hidden=128, heads=4, kv_heads=2)
    g = torch.Generator().manual_seed(3)
    queries = [torch.randint(0, v.vocab, (n,), generator=g).tolist() for n in (1, 14, 20)]
    history, scores, picked = m.search(v, queries, 9, beams, end_token=7, bits=bits, page=8, block=4)
    assert history.shape == (3, beams, 9)
    for t, p in enumerate(picked):
        want = reference(p["logits"].double().cpu().numpy(), p["scores"].double().cpu().numpy(), beams, p["ended"].cpu().numpy(), p["factor"].cpu().numpy(), 7)
        assert np.array_equal(p["parent"].cpu().numpy(), want[0]) and np.array_equal(p["token"].cpu().numpy(), want[1]), t
        for s in range(3 * beams):
            q, w = divmod(s, beams)
            if p["ended"][q, w] or (t == 0 and w):
                continue
            dense = _dense(v, queries[q] + p["history"][s].tolist())[-1]
            got = p["logits"][s].float().cpu()
            assert (got - dense).norm() <= (0.16 if bits == 8 else 0.02) * dense.norm(), (t, s)
    assert torch.equal(scores, picked[-1]["best"])


def test_fewer_continuations_than_beams():
    """A vocabulary smaller than the number of beams, and beams that end: picks of -1 have no tokens, no score and no keys, whatever
    other rows hold, and take part again once there are continuations for them.  The logits' tolerance: 1% rms by the decoder's
    roundings to bf16, as in test_search, of logits of 4 rms (the head's columns have a norm of 4); of the norm of three
    of them four times that, 4 * 0.04 * sqrt(3) = 0.28 (chi-squared of three beyond 48: 2e-10), where another row's are off by 10."""
    m = _example()
    v = m.Variant(vocab=3, hidden=128, heads=4, kv_heads=2)
    queries, beams = [[1], [2, 0, 1, 2, 2, 0, 1], [0, 1, 2]], 5
    history, scores, picked = m.search(v, queries, 5, beams, end_token=2, bits=16, page=4)
    missing = 0
    for t, p in enumerate(picked):
        with np.errstate(invalid="ignore"):
            want = reference(p["logits"].double().cpu().numpy(), p["scores"].double().cpu().numpy(), beams, p["ended"].cpu().numpy(),
                             p["factor"].cpu().numpy(), 2)
        assert np.array_equal(p["parent"].cpu().numpy(), want[0]) and np.array_equal(p["token"].cpu().numpy(), want[1]), t
        after = picked[t + 1]["history"] if t + 1 < len(picked) else history.flatten(0, 1)
        none = p["parent"].view(-1) < 0
        missing += int(none.sum())
        assert (after[none] == -1).all() and (p["best"].view(-1)[none] == float("-inf")).all()
        assert (after[~none] >= 0).all()
        if t + 1 < len(picked):
            assert (picked[t + 1]["ended"].view(-1)[none] == 1).all()
        for s in range(3 * beams):
            q, w = divmod(s, beams)
            if p["ended"][q, w] or (t == 0 and w):
                continue
            dense = _dense(v, queries[q] + p["history"][s].tolist())[-1]
            assert (p["logits"][s].float().cpu() - dense).norm() <= 0.28, (t, s)
    assert missing >= 2 * 3      # (of the first step: three continuations for five beams)
    assert torch.equal(scores, picked[-1]["best"])
