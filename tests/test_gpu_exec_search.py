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
