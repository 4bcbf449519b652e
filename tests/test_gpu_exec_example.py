"""The executor's calls together: examples/answer_queries.py against the same decoder in 32 bits without a cache."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import exec_ref

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "answer_queries.py")


def _example():
    spec = importlib.util.spec_from_file_location("answer_queries", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _dense(v, ids):
    """Logits behind every token of one sequence, in 32 bits on the host."""
    f = lambda w: w.float().cpu()
    x = f(v.embed)[torch.tensor(ids)]
    n = len(ids)
    norm = lambda y: y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6)
    freq = v.freq.cpu().numpy()
    for i in range(v.layers):
        qkv = (norm(x) @ f(v.qkv[i])).view(n, -1, v.head_dim)
        q, k, w = (t.double().numpy() for t in qkv.split([v.heads, v.kv_heads, v.kv_heads], dim=1))
        q, k = (exec_ref.rotate(t, np.arange(n), freq, False) for t in (q, k))
        out, _, _ = exec_ref.attend(q, lambda t: k, lambda t: w, [np.arange(n) <= t for t in range(n)], v.head_dim ** -0.5)
        x = x + torch.from_numpy(out).float().flatten(1) @ f(v.proj[i])
        x = x + torch.relu(norm(x) @ f(v.up[i])) @ f(v.down[i])
    return norm(x) @ f(v.head)


@pytest.mark.parametrize("shared", [0, 5, 16, 39])
def test_answers_of_a_batch(shared):
    """What is drawn goes back into the next step, so the reference takes the tokens as drawn: the logits have to agree, and
    each token has to be the one that the definition draws from them."""
    ex = _example()
    v = ex.Variant(vocab=700, hidden=128, heads=4, kv_heads=2)
    g = torch.Generator().manual_seed(3)
    ids = lambda n: torch.randint(0, v.vocab, (n,), generator=g).tolist()
    prompt, queries, steps = ids(shared), [ids(1), ids(7), ids(20)], 6
    tokens, logits = ex.answer(v, prompt, queries, steps, seed=4)
    draws = torch.rand((steps, 3), generator=torch.Generator().manual_seed(4)).clamp_max(1 - 2.0 ** -24)
    for s, q in enumerate(queries):
        drawn = tokens[s].tolist()
        want = _dense(v, prompt + q + drawn)[shared + len(q) - 1:-1]
        got = logits[:, s].float().cpu()
        # some twenty roundings to bf16 of 2^-9 rms each on the way, independent: 1% of the logits' norm, and twice that
        assert (got - want).norm() <= 0.02 * want.norm(), (s, float((got - want).norm() / want.norm()))
        for t in range(steps):
            token, _ = exec_ref.sample(got[t].double().numpy(), t=float(np.float32(0.8)), k=50, top_p=float(np.float32(0.95)),
                                       draw=float(draws[t, s]))
            assert token == drawn[t], (s, t)
