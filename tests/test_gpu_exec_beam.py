"""infaas_sel_exec_beam against its definition in 64 bits: types, sizes, ties, masks, beams that ended or are dead."""
import numpy as np
import pytest
import torch

import paper_1905_13348_amd as pkg

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def reference(logits, scores, picks, ended=None, factor=None, end=-1):
    """(parent, token, score, tolerance) by the definition; logits float64 [queries * beams, vocab]."""
    Q, W = scores.shape
    parent, token = np.full((Q, picks), -1), np.full((Q, picks), -1)
    score, off = np.full((Q, picks), -np.inf), np.zeros((Q, picks))
    for q in range(Q):
        found = []
        for w in range(W):
            f = 1.0 if factor is None else float(factor[q, w])
            s = float(scores[q, w])
            if not np.isfinite(s) or not (f > 0 and np.isfinite(f)):
                continue
            if ended is not None and ended[q, w]:
                found.append((-s * f, w, end, s, 0.0))
                continue
            x = np.where(np.isnan(logits[q * W + w]), -np.inf, logits[q * W + w])
            top = x.max()
            if top == -np.inf:
                continue
            t = np.where(x == np.inf, 0.0, -np.inf) if top == np.inf else x - top
            weight = np.exp(t)
            lse = np.log(weight.sum())
            # of a weight: two roundings and a constant's of its exponent in 32 bits, which is in two parts (of the row's part, and
            # of that to the row), an ulp of each power (2^-23), and ten roundings of the sums of up to 32 in 32 bits (2^-24 each)
            far = (weight * np.where(weight > 0, np.abs(t), 0) * 2.5 * 2.0 ** -24 + weight * 14 * 2.0 ** -24).sum() / weight.sum()
            for i in np.argsort(-t, kind="stable")[:picks]:
                if t[i] > -np.inf:
                    found.append((-(s + t[i] - lse) * f, w, int(i), s + t[i] - lse, far))
        for k, (_, w, i, s, far) in enumerate(sorted(found)[:picks]):
            parent[q, k], token[q, k], score[q, k], off[q, k] = q * W + w, i, s, far
    return parent, token, score, off


def check(logits, scores, picks, dtype="fp32", ended=None, factor=None, end=-1, shift=0, stride=None, label="", ex=None):
    ex = ex or pkg.Executor()
    scores = np.asarray(scores, dtype=np.float32)
    Q, W = scores.shape
    V = logits.shape[1]
    stride = V if stride is None else stride
    store = torch.full((shift + Q * W * stride + 8,), float("nan"), dtype=TYPES[dtype], device="cuda")
    dev = store[shift:shift + Q * W * stride].view(Q * W, stride)[:, :V]
    dev.copy_(torch.from_numpy(logits))
    out = [torch.full((Q, picks), -7, dtype=d, device="cuda") for d in (torch.int32, torch.int32, torch.float32)]
    to = lambda a, d: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(d).cuda()
    ex.beam(dev, to(scores, torch.float32), *out, ended=to(ended, torch.int32), factor=to(factor, torch.float32), end_token=end)
    parent, token, score = (t.cpu().numpy() for t in out)
    want = reference(dev.double().cpu().numpy(), scores.astype(np.float64), picks, ended, None if factor is None else factor.astype(np.float32), end)
    assert np.array_equal(parent, want[0]) and np.array_equal(token, want[1]), (label, np.argwhere((parent != want[0]) | (token != want[1]))[:5].tolist())
    there = want[0] >= 0
    assert (score[~there] == -np.inf).all()
    tol = want[3] + 2.0 ** -23 * np.abs(want[2])
    assert (np.abs(score - want[2])[there] <= tol[there]).all(), label
    return out


def made(rng, rows, vocab, spread=3.0):
    return rng.standard_normal((rows, vocab)) * spread


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("vocab", [1, 2, 7, 8, 9, 63, 100, 1000, 1021, 8183, 8184, 8185, 8188, 8189, 20_011, 100_003])
def test_types_and_vocabularies(dtype, vocab):
    rng = np.random.default_rng(vocab)
    check(made(rng, 6, vocab), -rng.random((2, 3)) * 3, 5, dtype)


@pytest.mark.parametrize("queries, beams, picks", [(1, 1, 1), (1, 1, 64), (3, 64, 64), (2, 5, 10), (70, 2, 4), (4, 12, 24), (300, 4, 8)])
def test_counts(queries, beams, picks):
    rng = np.random.default_rng(queries + beams)
    check(made(rng, queries * beams, 3001), -np.sort(rng.random((queries, beams)) * 8), picks, "fp32")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shift, stride", [(0, 1003), (1, 1001), (3, 1024), (5, 1007), (7, 1000)])
def test_alignments(dtype, shift, stride):
    rng = np.random.default_rng(shift)
    check(made(rng, 8, 1000), -rng.random((2, 4)), 8, dtype, shift=shift, stride=stride)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("vocab", [999, 20_011])
def test_beams_alike(dtype, vocab):
    """The same logits and scores for all beams, each row at another alignment: equal scores go by beam, then by token."""
    rng = np.random.default_rng(1)
    row = made(rng, 1, vocab)
    check(np.repeat(row, 8, axis=0), np.full((2, 4), -1.5), 16, dtype)


@pytest.mark.parametrize("vocab", [50, 5000, 30_000])
@pytest.mark.parametrize("picks", [1, 6, 64])
def test_logits_alike(vocab, picks):
    """Constant rows, and rows of two values: more equal logits than any list holds."""
    rng = np.random.default_rng(2)
    check(np.zeros((6, vocab)), np.zeros((2, 3)), picks, "bf16")
    check(np.where(rng.random((6, vocab)) < 0.5, 1.0, -1.0), -np.arange(6).reshape(2, 3) / 4, picks, "fp32")
    # masked by a low number but for a few, fewer than are picked among them
    x = np.full((6, vocab), -60_000.0)
    x[:, rng.choice(vocab, 20, replace=False)] = made(rng, 6, 20)
    check(x, -np.arange(6).reshape(2, 3) / 4, picks, "fp16")
    # zeros of both signs are equal
    check(np.where(rng.random((6, vocab)) < 0.5, 0.0, -0.0), np.zeros((2, 3)), picks, "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [1, 150, 600])
def test_parts_of_several_chunks(rows, dtype):
    """Many rows make parts of several chunks: rising and falling logits, equal ones, masks at either end, numbers that are none."""
    rng = np.random.default_rng(rows)
    V = 70_001
    x = np.repeat(made(rng, 3, V), -(-rows // 3), axis=0)[:rows]
    up = np.arange(V) / V * 20
    for r, row in enumerate((up, -up, np.zeros(V), np.where(np.arange(V) < 69_990, -np.inf, 1.0), np.where(np.arange(V) % 9000, -60_000.0, up))):
        x[r % rows] = row
    if rows > 10:
        x[6, 40_000], x[7, 69_999], x[8, [3, 50_000]] = np.nan, np.inf, np.inf
        x[8, 100] = np.nan
    check(x, -rng.random((rows, 1)) * 3, 12, dtype)


def test_many_ties_between_many_beams():
    """More equal continuations than a query's list holds."""
    check(np.zeros((64, 20_000)), np.zeros((1, 64)), 64, "fp32")


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_masks(dtype):
    """Minus infinity, NaN, plus infinity; rows of nothing else; fewer tokens left than picked; the type's lowest number."""
    rng = np.random.default_rng(3)
    x = made(rng, 12, 9001)
    x[0] = -np.inf
    x[1, 5:] = -np.inf
    x[2] = np.nan
    x[3, ::2] = np.nan
    x[4, [7, 8000]] = np.inf
    x[5, 100] = np.inf
    x[5, :50] = np.nan
    x[6, 1:] = -np.inf
    x[7] = float(torch.finfo(TYPES[dtype]).min)
    x[8, :9000] = float(torch.finfo(TYPES[dtype]).min)
    x[9, :8500] = -np.inf
    for picks in (3, 20):
        check(x, -rng.random((3, 4)), picks, dtype)
        check(x, -rng.random((12, 1)), picks, dtype)
        check(x[:1], np.zeros((1, 1)), picks, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("vocab", [700, 20_011, 100_003])
@pytest.mark.parametrize("picks", [1, 8, 33])
def test_finite_masks(dtype, vocab, picks):
    """All of a row but a few logits are one low number, which is picked where there are not enough others; lists fill with it."""
    rng = np.random.default_rng(picks + vocab)
    left = [0, 1, picks - 1, picks, picks + 1, 129]
    x = np.full((len(left), vocab), -60000.0)
    for row, k in zip(x, left):
        at = rng.choice(vocab, k, replace=False)
        row[at] = rng.integers(-20, 20, k) / 4        # (ties among these, too)
    check(x, np.zeros((len(left), 1)), picks, dtype)
    check(x, -rng.random((2, 3)), picks, dtype)


@pytest.mark.parametrize("picks", [2, 4, 12])
def test_beams_that_ended(picks):
    rng = np.random.default_rng(4)
    ended = rng.random((20, 4)) < 0.5
    ended[0], ended[1] = True, False
    factor = rng.random((20, 4)) + 0.2
    scores = -rng.random((20, 4)) * 9
    check(made(rng, 80, 700), scores, picks, "fp32", ended=ended, end=0)
    check(made(rng, 80, 700), scores, picks, "bf16", ended=ended * 7, factor=factor, end=699)
    check(made(rng, 80, 700), scores, picks, "fp16", factor=factor)


def test_beams_that_are_dead():
    rng = np.random.default_rng(5)
    scores = -rng.random((6, 4))
    scores[0, 1:] = -np.inf             # a search that begins
    scores[1] = -np.inf
    scores[2, 0], scores[2, 1] = np.nan, np.inf
    factor = np.ones((6, 4))
    factor[3] = [0.0, -1.0, np.nan, 1.0]
    factor[4] = [np.inf, 0.5, 1e-30, 2.0]
    ended = np.zeros((6, 4))
    ended[1, 0] = ended[3, 0] = ended[5, 3] = 1
    check(made(rng, 24, 300), scores, 4, "fp32", factor=factor, ended=ended, end=3)
    check(made(rng, 24, 300), scores, 4, "fp32")


def test_scores_in_place():
    rng = np.random.default_rng(6)
    ex = pkg.Executor()
    x = torch.from_numpy(made(rng, 24, 5000)).float().cuda()
    scores = torch.from_numpy(-rng.random((6, 4))).float().cuda()
    ended = torch.from_numpy((rng.random((6, 4)) < 0.4).astype(np.int32)).cuda()
    want = reference(x.double().cpu().numpy(), scores.double().cpu().numpy(), 4, ended.cpu().numpy(), None, 9)
    parent, token = (torch.empty((6, 4), dtype=torch.int32, device="cuda") for _ in range(2))
    ex.beam(x, scores, parent, token, scores, ended=ended, end_token=9)
    assert np.array_equal(parent.cpu().numpy(), want[0]) and np.array_equal(token.cpu().numpy(), want[1])
    # many equal ones, which take the other way through the kernel
    zeros, s = torch.zeros((64, 20_000), device="cuda"), torch.zeros((1, 64), device="cuda")
    ends = torch.zeros((1, 64), dtype=torch.int32, device="cuda")
    ends[0, 5] = 1
    parent, token = (torch.empty((1, 64), dtype=torch.int32, device="cuda") for _ in range(2))
    ex.beam(zeros, s, parent, token, s, ended=ends, end_token=9)
    assert parent[0, 0] == 5 and token[0, 0] == 9 and parent[0, 1:].eq(0).all() and token[0, 1:].tolist() == list(range(63))
    ex.destroy()


def test_large():
    """Rows beyond 2^31 elements, 2^20 tokens to a row."""
    ex = pkg.Executor()
    Q, W, V, K = 300, 8, 1 << 20, 4
    x = torch.randn((Q * W, V), dtype=torch.bfloat16, device="cuda")
    scores = -torch.rand((Q, W), device="cuda")
    out = [torch.empty((Q, K), dtype=d, device="cuda") for d in (torch.int32, torch.int32, torch.float32)]
    ex.beam(x, scores, *out)
    for q in (0, 150, 299):
        s = x[q * W:(q + 1) * W].double()
        s = s - s.logsumexp(dim=1, keepdim=True) + scores[q].double()[:, None]
        best = s.flatten().topk(K)
        assert np.allclose(out[2][q].double().cpu().numpy(), best.values.cpu().numpy(), rtol=2e-6)
        got = s[(out[0][q] - q * W).long(), out[1][q].long()]
        assert torch.allclose(got, best.values, rtol=2e-6)
    ex.destroy()


def test_replayed_and_on_another_stream():
    ex = pkg.Executor()
    rng = np.random.default_rng(7)
    ex.reserve_beam(3, 4, 20_000, 8, torch.bfloat16)
    x = torch.zeros((12, 20_000), dtype=torch.bfloat16, device="cuda")
    scores = torch.zeros((3, 4), device="cuda")
    out = [torch.empty((3, 8), dtype=d, device="cuda") for d in (torch.int32, torch.int32, torch.float32)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ex.beam(x, scores, *out)
    side = torch.cuda.Stream()
    other = [torch.empty_like(t) for t in out]
    for t in range(4):
        x.copy_(torch.from_numpy(made(rng, 12, 20_000)))
        scores.copy_(torch.from_numpy(-rng.random((3, 4))))
        graph.replay()
        want = reference(x.double().cpu().numpy(), scores.double().cpu().numpy(), 8)
        side.wait_stream(torch.cuda.current_stream())
        ex.beam(x, scores, *other, stream=side)
        side.synchronize()
        for got in (out, other):
            assert np.array_equal(got[0].cpu().numpy(), want[0]) and np.array_equal(got[1].cpu().numpy(), want[1])
        assert torch.equal(out[2], other[2])
    ex.destroy()


def test_scratch_that_would_have_to_grow_in_a_recording():
    ex = pkg.Executor()
    x, scores = torch.zeros((12, 20_000), device="cuda"), torch.zeros((3, 4), device="cuda")
    out = [torch.empty((3, 8), dtype=d, device="cuda") for d in (torch.int32, torch.int32, torch.float32)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x.add_(0)
        with pytest.raises(pkg.InfaasSelError, match="reserve_beam"):
            ex.beam(x, scores, *out)
    ex.destroy()
