"""infaas_sel_exec_advance and _copy against their definition: every array after every step."""
import numpy as np
import pytest
import torch

import paper_1905_13348_amd as pkg
import table_ref

pytestmark = pytest.mark.gpu

i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


class Both:
    """A table on the device and its definition, taken through the same steps."""

    def __init__(self, S, width, page, pages, most, ex=None):
        self.ex = ex or pkg.Executor()
        self.dev, self.ref = self.ex.table(S, width, page, pages, most), table_ref.Table(S, width, page, pages, most)

    def hold(self, refs):
        """Pages that the caller keeps for itself."""
        self.ref.refs = [a + b for a, b in zip(self.ref.refs, refs)]
        self.dev.page_refs += i32(refs)

    def step(self, new, parent=None, label=""):
        self.ex.advance(self.dev, i32(new), None if parent is None else i32(parent))
        self.check(self.ref.advance(list(new), None if parent is None else list(parent)), label)

    def check(self, want, label=""):
        taken, copies, seq, pos = want
        d, n = self.dev, len(seq)
        got = {k: getattr(d, k).cpu().numpy() for k in ("page_table", "seq_len", "page_refs", "seq_start", "token_seq", "token_pos", "taken", "copies")}
        pad = [-1] * (d.max_tokens - n)
        for name, w in (("taken", taken), ("seq_len", self.ref.length), ("page_table", self.ref.padded()), ("page_refs", self.ref.refs),
                        ("copies", copies), ("seq_start", np.concatenate([[0], np.cumsum(taken)])), ("token_seq", seq + pad),
                        ("token_pos", list(pos) + pad)):
            assert np.array_equal(got[name], np.array(w).reshape(got[name].shape)), f"{label}: {name}"


@pytest.mark.parametrize("S, width, page, pages, most", [
    (1, 1, 1, 1, 1), (1, 3, 4, 5, 20), (5, 4, 16, 30, 100), (64, 8, 4, 300, 400), (70, 5, 2, 200, 300), (300, 7, 8, 2000, 5000), (1025, 3, 16, 2500, 3000),
    (4096, 2, 8, 6000, 9000), (3, 700, 1, 1500, 1000), (16, 40, 64, 40_000, 20_000)])
@pytest.mark.parametrize("seed", [0, 1, 2])
def test_a_life(S, width, page, pages, most, seed):
    """Steps of all kinds: sequences that grow, are cut, begin anew, go on from others, and pages and tokens that run out."""
    rng = np.random.default_rng(S + width + seed * 10_000)
    b = Both(S, width, page, pages, most)
    b.hold((rng.random(pages) < 0.2) * rng.integers(1, 3, pages))
    room = width * page
    for t in range(21):
        kind = t % 7
        new, parent = rng.integers(0, max(2, room // 4), S), None
        if kind == 1:
            new = np.ones(S, dtype=int)
        elif kind == 2:
            new = -rng.integers(0, max(2, room // 3), S)
        elif kind == 3:
            parent = rng.integers(-1, S + 1, S)
            new = rng.integers(0, 3, S)
        elif kind == 4:
            parent, new = np.where(rng.random(S) < 0.3, -1, np.arange(S)), rng.integers(-3, max(4, room // 2), S)
        elif kind == 5:
            parent = np.minimum(np.arange(S) // 4 * 4 + rng.integers(0, 4, S), S - 1)
            new = np.ones(S, dtype=int)
        elif kind == 6:
            parent, new = np.full(S, S // 2), rng.integers(-2, 3, S)
        b.step(new, parent, f"step {t}")


def test_lowest_pages_first_and_back():
    b = Both(3, 4, 4, 12, 64)
    b.step([5, 9, 1])
    assert b.dev.page_table.cpu().tolist() == [[0, 1, -1, -1], [2, 3, 4, -1], [5, -1, -1, -1]]
    b.step([0, -9, 4], None)
    assert b.dev.page_table.cpu().tolist() == [[0, 1, -1, -1], [-1] * 4, [5, 2, -1, -1]]


def test_pages_that_run_out():
    """Who waits for pages is not overtaken by who needs some; who needs none goes on; what was handed out in part goes back."""
    b = Both(5, 8, 4, 6, 100)
    b.step([8, 3, 0, 0, 0])                 # 2 + 1 pages
    b.step([0, 1, 20, 1, 0])                # 5 pages where 3 are free: sequence 2 waits, and 3 behind it
    assert b.dev.taken.cpu().tolist() == [0, 1, 0, 0, 0]
    b.step([-8, 0, 20, 1, 1])               # 5 free: all of them, and none for who comes behind
    assert b.dev.taken.cpu().tolist() == [0, 0, 20, 0, 0]


def test_tokens_that_do_not_fit():
    b = Both(4, 8, 4, 100, 10)
    b.step([4, 7, 1, 5])
    assert b.dev.taken.cpu().tolist() == [4, 0, 0, 0]
    b.step([33, 3, 40, 7])                  # more than a row holds: not counted
    assert b.dev.taken.cpu().tolist() == [0, 3, 0, 7]


def test_a_copy_where_pages_run_out():
    """A shared last page and no page for the copy: the sequence keeps what it has."""
    b = Both(2, 4, 4, 3, 64)
    b.step([6, 0])
    b.step([0, 0], [0, 0])
    b.step([7, 1])                          # 0 asks for 3 (copy + 2) of 1; 1 waits behind it
    assert b.dev.taken.cpu().tolist() == [0, 0] and (b.dev.copies == -1).all()
    b.step([0, 1])
    assert b.dev.copies.cpu().tolist() == [[-1] * 3, [1, 2, 2]]
    b.step([1, 1])                          # both alone on their pages now
    assert (b.dev.copies == -1).all()


def test_lengths_and_pages_that_are_not_there():
    """Lengths and entries out of range count as the nearest length and as no page; nothing is read or written out of range."""
    ex = pkg.Executor()
    t = ex.table(3, 2, 4, 5, 16)
    t.seq_len.copy_(i32([-5, 1 << 30, 3]))
    t.page_table.copy_(i32([[7, 9], [-3, 1 << 30], [5, 0]]))
    ex.advance(t, i32([1, 1, 1]), None)
    assert t.taken.cpu().tolist() == [1, 0, 1] and t.seq_len.cpu().tolist() == [1, 8, 4]
    assert t.page_table.cpu().tolist() == [[0, 9], [-3, 1 << 30], [5, 0]] and t.page_refs.cpu().tolist() == [1, 0, 0, 0, 0]
    ex.advance(t, i32([-(2 ** 31), 2 ** 31 - 1, 0]), i32([2 ** 31 - 1, -(2 ** 31), 1]))
    assert t.seq_len.cpu().tolist() == [0, 0, 8] and t.taken.cpu().tolist() == [0, 0, 0]


@pytest.mark.parametrize("coded", [False, True])
@pytest.mark.parametrize("layout", ["token", "head"])
@pytest.mark.parametrize("page, dim, block", [(16, 64, 4), (128, 256, 16), (4, 128, 4), (1024, 64, 64)])
def test_copy(coded, layout, page, dim, block):
    """The keys below the length, of both pools, and the scales of their blocks; nothing else."""
    ex = pkg.Executor()
    g = torch.Generator().manual_seed(page + dim)
    pages, heads = 9, 3
    t = ex.table(5, 2, page, pages, 8)
    copies = [[0, 3, page - 1], [-1, -1, -1], [2, 5, 1], [1, 9, 2], [7, 8, page // 2 + 1]]
    t.copies.copy_(i32(copies))
    shape = (pages, page, heads, dim) if layout == "token" else (pages, heads, page, dim)
    pools = [torch.randint(0, 256, shape + (1 if coded else 2,), generator=g, dtype=torch.uint8).cuda() for _ in range(2)]
    blocks = (pages, page // block, heads) if layout == "token" else (pages, heads, page // block)
    scales = [torch.randint(0, 256, blocks, generator=g, dtype=torch.uint8).cuda() for _ in range(2)]
    want = [p.cpu().numpy() for p in pools + scales]
    if coded:
        cache = ex.cache(*(p.view(torch.float8_e4m3fn).squeeze(-1) for p in pools), layout=layout, k_scale=scales[0].view(torch.float8_e8m0fnu),
                         v_scale=scales[1].view(torch.float8_e8m0fnu))
    else:
        cache = ex.cache(*(p.view(torch.bfloat16).squeeze(-1) for p in pools), layout=layout)
    ex.copy(cache, t)
    for a, b, n in copies:
        if a >= 0 and b < pages:
            for w in want[:2]:
                w = w if layout == "token" else w.swapaxes(1, 2)
                w[b, :n] = w[a, :n]
            for w in want[2:] if coded else ():
                w = w if layout == "token" else w.swapaxes(1, 2)
                w[b, :-(-n // block)] = w[a, :-(-n // block)]
    for p, w in zip(pools + scales, want):
        assert np.array_equal(p.cpu().numpy(), w)


def test_replayed():
    """Recorded once, replayed through a life with other numbers, with eager work between."""
    b = Both(12, 6, 4, 60, 64)
    rng = np.random.default_rng(5)
    new, parent = i32(np.zeros(12)), i32(np.arange(12))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.ex.advance(b.dev, new, parent)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.ex.advance(b.dev, new, parent)
    for t in range(20):
        m = rng.integers(-4, 9, 12)
        p = np.where(rng.random(12) < 0.3, rng.integers(-1, 12, 12), np.arange(12))
        new.copy_(i32(m))
        parent.copy_(i32(p))
        graph.replay()
        b.check(b.ref.advance(list(m), list(p)), f"replay {t}")
        if t % 3 == 0:
            b.step(np.ones(12, dtype=int), None, f"eager {t}")


def test_steps_of_a_worker():
    """Beams over a cache of 8 bits, all on the device: advance, copy, append, attend; against every beam's own history, read
    back and attended over in 64 bits."""
    ex = pkg.Executor()
    rng = np.random.default_rng(6)
    S, H, kv, D, P, B, pages, most = 6, 4, 2, 64, 8, 4, 80, 40
    t = ex.table(S, 8, P, pages, most)
    zeros = lambda *shape: torch.zeros(shape, dtype=torch.uint8, device="cuda")
    cache = ex.cache(*(zeros(pages, P, kv, D).view(torch.float8_e4m3fn) for _ in range(2)),
                     k_scale=zeros(pages, P // B, kv).view(torch.float8_e8m0fnu), v_scale=zeros(pages, P // B, kv).view(torch.float8_e8m0fnu))
    batch = ex.batch(cache, H, **t.arrays())
    history = [np.zeros((2, 0, kv, D)) for _ in range(S)]
    for step in range(12):
        parent = np.arange(S) if step % 3 else rng.integers(0, S, S)
        new = rng.integers(0, 5, S) if step % 4 else rng.integers(-3, 6, S)
        ex.advance(t, i32(new), i32(parent))
        ex.copy(cache, t)
        ex.plan(batch)
        q, k, v = (torch.from_numpy(rng.standard_normal((most, h, D)) * 3).bfloat16().cuda() for h in (H, kv, kv))
        ex.append(cache, batch, q, k, v, q, None)
        out = torch.full((most, H, D), 5.0, dtype=torch.bfloat16, device="cuda")
        ex.attend(cache, batch, q, out)
        taken, start, length = (getattr(t, n).cpu().numpy() for n in ("taken", "seq_start", "seq_len"))
        kd, vd, qd, od = (x.double().cpu().numpy() for x in (k, v, q, out))
        assert (od[start[-1]:] == 0).all()      # (tokens behind the last sequence)
        before = history
        history = []
        for s in range(S):
            old = before[parent[s]][:, :length[s] - taken[s]]
            own = np.stack([x[start[s]:start[s + 1]] for x in (kd, vd)])
            history.append(np.concatenate([old, own], axis=1))
            assert history[s].shape[1] == length[s]
            # what the cache has: a number of e4m3 for each, by a scale of 2^10 of its block's largest at the most
            n = int(length[s])
            whole = ex.batch(cache, H, token_seq=i32(np.full(n, s)), token_pos=i32(np.arange(n)), seq_start=i32([0] * (s + 1) + [n] * (S - s)),
                             seq_len=t.seq_len, page_table=t.page_table)
            got = [torch.empty((n, kv, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
            ex.read(cache, whole, *got)
            numbers = np.stack([x.double().cpu().numpy() for x in got])
            if n:
                # rounded once, and once more with every rise of its block's scale: half a step of 2^-4, and of the largest
                # number's smallest steps (448 * 2^e is less than twice that number)
                largest = np.abs(history[s]).max()
                assert (np.abs(numbers - history[s]) <= 2 * 2.0 ** -4 * np.abs(history[s]) + 6 * 2.0 ** -10 * largest / 224).all()
            for i in range(taken[s]):
                seen = n - taken[s] + i + 1
                for h in range(H):
                    score = numbers[0, :seen, h // 2] @ qd[start[s] + i, h] * D ** -0.5
                    p = np.exp(score - score.max())
                    p /= p.sum()
                    x, y = p @ numbers[1, :seen, h // 2], od[start[s] + i, h]
                    tol = 2.0 ** -8 * np.abs(x) + (2.0 ** -8 + 2.0 ** -11) * (p @ np.abs(numbers[1, :seen, h // 2])) + 1e-30
                    assert (np.abs(x - y) <= tol).all()
    ex.destroy()
