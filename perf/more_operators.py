"""More operators of a worker that answers in text, as cases that can be timed and compared.

append   keys and values of a step's tokens into a paged cache of 8 bits (e4m3) with a power of two as the scale of every
         block of tokens and head, rotated on the way; the cache is then read back as numbers of the queries' type
attend   attention of a ragged batch over such a cache; what a group of sequences shares at its front is there once
advance  pages handed out, shared, copied and given back from the lengths that sequences ask for, and the arrays of the
         step's batch
beam     the best continuations of every query's beams, over beams and vocabulary

With ``own`` false the operators are elementary torch operations; with ``own`` true they are the calls of
``paper_1905_13348_amd.Executor``.  ``exact`` is the definition in 64 bits.
"""
import math
from types import SimpleNamespace

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
CODES, SCALES = torch.float8_e4m3fn, torch.float8_e8m0fnu
LARGEST = 448.0     # of e4m3
DEVICE = "cuda"


# ---- cases ----------------------------------------------------------------------------------------------------

def _append(tokens, seqs, context, dtype="bf16", heads=32, kv_heads=8, dim=128, rot=128, interleaved=False, page=64,
            block=16, layout="token", fused=True):
    return {"op": "append", "tokens": tokens, "seqs": seqs, "context": context, "dtype": dtype, "heads": heads,
            "kv_heads": kv_heads, "dim": dim, "rot": rot, "interleaved": interleaved, "page": page, "block": block,
            "layout": layout, "fused": fused}


def _attend(seqs, shared, own_most, new, dtype="bf16", heads=32, kv_heads=8, dim=128, page=64, block=16, layout="token",
            groups=1):
    return {"op": "attend", "seqs": seqs, "shared": shared, "own_most": own_most, "new": new, "dtype": dtype,
            "heads": heads, "kv_heads": kv_heads, "dim": dim, "page": page, "block": block, "layout": layout, "groups": groups}


def _advance(what, seqs, most, page, pages, beams=1, used=0.6):
    return {"op": "advance", "what": what, "seqs": seqs, "most": most, "page": page, "pages": pages, "beams": beams,
            "used": used}


def _beam(queries, beams, vocab, picks, dtype, ended=False):
    return {"op": "beam", "queries": queries, "beams": beams, "vocab": vocab, "picks": picks, "dtype": dtype, "ended": ended}


def listed():
    cases = {
        # a decode step of a full batch behind short queries: one token each, straight out of a fused projection; most blocks
        # have tokens already, whose scale may have to rise
        "append_step": _append(200, 200, 60),
        # the prompts of several queries at once: ragged lengths, neighbouring pairs rotated, half of the dimensions, a scale
        # for every page, and a cache that keeps a head's tokens of a page together
        "append_prompts": _append(14_003, 11, 900, "fp16", 32, 8, 128, 64, True, 32, 32, "head", False),
        # a few queries without anything in common, one token each, where latency counts
        "attend_few": _attend(5, 0, 600, 1),
        # one query behind a very long document: the work has to be split along the cache
        "attend_long": _attend(1, 0, 200_003, 1, "bf16", 32, 8, 128, 64, 64, "head"),
        # a full decode step: long own parts behind two applications' prompts (the largest in bytes)
        "attend_full": _attend(192, 8000, 16_000, 1, "bf16", 32, 8, 128, 32, 32, "token", 2),
        # prompts being read behind the application's own, ragged (the largest in operations)
        "attend_prompts": _attend(6, 12_000, 700, 700, "fp16", 32, 4, 128, 16, 16),
        # speculation: every sequence gives back the drafts that were rejected and takes new ones
        "advance_drafts": _advance("drafts", 256, 4000, 16, 65_536),
        # a batch of queries comes in: pages for their prompts, those of the batch before go back
        "advance_prompts": _advance("prompts", 300, 1500, 32, 40_000),
        # beams of one prompt part: whole pages are shared, the page where the prompt ends is copied in a layer's cache
        "advance_beams": _advance("beams", 192, 1200, 16, 9001, 6, 0.2),
        # the beams of one query, where latency counts
        "beam_one": _beam(1, 4, 32_768, 4, "fp32"),
        # a full step of beam search at an odd vocabulary: some beams have ended, lengths differ
        "beam_ended": _beam(24, 8, 100_003, 16, "fp16", True),
        # the largest step
        "beam_full": _beam(128, 4, 128_000, 8, "bf16"),
    }
    return [dict(c, name=name) for name, c in cases.items()]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, uniform in its logarithm."""
    return min(max(int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))))), lo), hi)


def _cost(case):
    w = work(case)
    return w["bytes"] / 4e12 + w["flops"] / 5e14


def draw(rng):
    op = rng.choice(("append", "attend", "attend", "advance", "beam"))
    most = max(_cost(c) for c in listed() if c["op"] == op)
    while True:
        if op == "append":
            seqs = _spread(rng, 1, 200)
            dim, page = rng.choice((64, 128, 256)), rng.choice((16, 32, 64, 128))
            kv = rng.choice((1, 2, 4, 8))
            case = _append(max(seqs, _spread(rng, 1, 14_000)), seqs, _spread(rng, 1, 900), rng.choice(("bf16", "fp16")),
                           kv * rng.choice((1, 3, 4, 8)), kv, dim, rng.choice((dim, dim // 2)), rng.random() < 0.4, page,
                           rng.choice((1, 8, 16, page)), rng.choice(("token", "head")), rng.random() < 0.5)
        elif op == "attend":
            new = rng.choice((1, 1, 1, _spread(rng, 2, 8), _spread(rng, 16, 700)))
            seqs = _spread(rng, 1, 192 if new < 16 else 8)
            kv, page = rng.choice((1, 2, 4, 8)), rng.choice((16, 32, 64, 128))
            case = _attend(seqs, rng.choice((0, _spread(rng, 50, 20_000))),
                           max(new, _spread(rng, 1, 16_000 if seqs > 2 else 200_000)), new, rng.choice(("bf16", "fp16")),
                           kv * rng.choice((1, 3, 4, 8)), kv, rng.choice((64, 128, 128, 256)), page,
                           rng.choice((1, 8, 16, page)), rng.choice(("token", "head")), min(seqs, rng.choice((1, 1, 2, 5))))
            if case["seqs"] * (case["shared"] + case["own_most"]) * kv * case["dim"] > 5e9:
                continue
        elif op == "advance":
            what = rng.choice(("drafts", "prompts", "beams"))
            beams = rng.randint(2, 8) if what == "beams" else 1
            seqs = beams * _spread(rng, 1, 400 // beams)
            most_keys, page = _spread(rng, 20, 4000), rng.choice((1, 16, 32, 64, 128))
            used = rng.choice((0.0, 0.2, 0.6))
            pages = int((seqs * (most_keys + 8) / page + 2 * seqs) / (1 - used) * rng.uniform(1.0, 1.5)) + 8
            if pages > 65_536 or pages * page > 1 << 18:
                continue
            case = _advance(what, seqs, most_keys, page, pages, beams, used)
        else:
            beams = rng.randint(1, 12)
            case = _beam(_spread(rng, 1, 128), beams, _spread(rng, 1000, 160_000), beams * rng.choice((1, 2)),
                         rng.choice(("bf16", "fp16", "fp32")), rng.random() < 0.5)
        if _cost(case) <= most:
            return case


# ---- inputs ---------------------------------------------------------------------------------------------------

def _lengths(case):
    """Of a case, on the host: lengths of the sequences' own parts, their new tokens, their groups and what those share.
    They belong to the case; values, pages and limits go by the seed."""
    rng = np.random.default_rng(78)
    S = case["seqs"]
    if case["op"] == "append":   # every sequence has some tokens in the cache and gets its share of the new ones
        cuts = np.sort(rng.integers(0, case["tokens"] - S + 1, S - 1))
        new = np.diff(np.concatenate([[0], cuts, [case["tokens"] - S]])).astype(int) + 1
        return rng.integers(0, case["context"] + 1, S) + new, new, np.array([0, S]), np.array([0])
    groups = case["groups"]
    own_len = rng.integers(max(1, case["own_most"] // 4), case["own_most"] + 1, S) if S > 1 else np.array([case["own_most"]])
    new = np.full(S, case["new"]) if case["new"] == 1 else rng.integers(max(1, case["new"] // 4), case["new"] + 1, S)
    own_len = np.maximum(own_len, new)
    cut = np.sort(rng.choice(np.arange(1, S), groups - 1, replace=False)) if groups > 1 else np.array([], dtype=int)
    group_start = np.concatenate([[0], cut, [S]]).astype(int)
    shared = np.array([case["shared"] - g * (case["shared"] // (2 * groups)) for g in range(groups)], dtype=int)
    return own_len.astype(int), new.astype(int), group_start, shared


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEVICE)


def _cache_inputs(case, seed):
    rng = np.random.default_rng([seed, 78])
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    t = TYPES[case["dtype"]]
    S, H, Hkv, D, P, B = (case[k] for k in ("seqs", "heads", "kv_heads", "dim", "page", "block"))
    own_len, new, group_start, shared = _lengths(case)
    length = own_len + np.repeat(shared, np.diff(group_start))
    before = length - new
    n = int(new.sum())
    seq = np.repeat(np.arange(S), new)
    start = np.concatenate([[0], np.cumsum(new)])
    pos = before[seq] + np.arange(n) - start[seq]

    # pages in no order at all; whole pages of the shared part are there once, the page where it ends is each sequence's
    # own copy
    need = -(-length // P)
    common = np.repeat(shared // P, np.diff(group_start))
    first = np.repeat(group_start[:-1], np.diff(group_start))
    width = int(need.max())
    total = int(need.sum() - sum(common[s] for s in range(S) if first[s] != s))
    order = rng.permutation(total)
    table = np.zeros((S, width), dtype=np.int64)
    at = 0
    for s in range(S):
        skip = int(common[s]) if first[s] != s else 0
        table[s, :skip] = table[first[s], :skip]
        table[s, skip:need[s]] = order[at:at + need[s] - skip]
        at += int(need[s]) - skip

    # what an append leaves: codes up to the largest, a scale for each block and head
    token_major = case["layout"] == "token"
    shape = (total, P, Hkv, D) if token_major else (total, Hkv, P, D)
    blocks = (total, P // B, Hkv) if token_major else (total, Hkv, P // B)
    x = {"case": case}
    for name in ("k", "v"):
        pool = torch.empty(shape, dtype=CODES, device=DEVICE)
        for part in pool.split(max(1, (1 << 28) // (P * Hkv * D))):
            part.copy_((torch.randn(part.shape, generator=gen, device=DEVICE) * 130).clamp_(-LARGEST, LARGEST))
        x[name + "_pool"] = pool
        # (keys and values of a magnitude of 1 or so, by heads and blocks)
        x[name + "_scale"] = torch.randint(118, 122, blocks, generator=gen, device=DEVICE, dtype=torch.uint8).view(SCALES)
    slots = P // B
    for s in range(S):
        rest = int(shared[np.searchsorted(group_start, s, "right") - 1] % P)
        if first[s] != s and rest:
            a, b, blk = int(table[first[s], common[s]]), int(table[s, common[s]]), min(slots, -(-rest // B))
            for name in ("k", "v"):
                pool, scale = x[name + "_pool"].view(torch.uint8), x[name + "_scale"].view(torch.uint8)
                if token_major:
                    pool[b, :rest], scale[b, :blk] = pool[a, :rest], scale[a, :blk]
                else:
                    pool[b, :, :rest], scale[b, :, :blk] = pool[a, :, :rest], scale[a, :, :blk]
    x.update(table=_i32(table), pos=_i32(pos), seq=_i32(seq), start=_i32(start), length=_i32(length), new=_i32(new),
             group_start=_i32(group_start), shared=_i32(shared), most_new=int(new.max()), most=int(length.max()))
    if case["op"] == "append":
        all_seq = np.repeat(np.arange(S), length)
        all_start = np.concatenate([[0], np.cumsum(length)])
        x.update(all_seq=_i32(all_seq), all_pos=_i32(np.arange(len(all_seq)) - all_start[all_seq]), all_start=_i32(all_start))
        # (some tokens stand out, as they do)
        loud = torch.exp(0.5 * torch.randn((n, 1, 1), generator=gen, device=DEVICE))
        if case["fused"]:
            qkv = (torch.randn((n, H + 2 * Hkv, D), generator=gen, device=DEVICE) * loud).to(t)
            x.update(q=qkv[:, :H], k=qkv[:, H:H + Hkv], v=qkv[:, H + Hkv:])
        else:
            x.update({name: (torch.randn((n, h, D), generator=gen, device=DEVICE) * loud).to(t)
                      for name, h in (("q", H), ("k", Hkv), ("v", Hkv))})
        half = case["rot"] // 2
        x["freq"] = torch.from_numpy(10000.0 ** (-np.arange(half) / half)).to(DEVICE)
    else:
        x["q"] = torch.randn((n, H, D), generator=gen, device=DEVICE, dtype=t)
        x["scale"] = D ** -0.5
    return x


def _advance_inputs(case, seed):
    """The state that a worker's steps have left, and what the next ones ask for."""
    rng = np.random.default_rng([seed, 78])
    S, P, beams, pages = case["seqs"], case["page"], case["beams"], case["pages"]
    width = -(-(case["most"] + 8) // P)
    ask = np.exp(rng.uniform(np.log(max(4, case["most"] // 16)), np.log(case["most"]), S)).astype(int)
    refs, table, length = np.zeros(pages, dtype=np.int64), np.full((S, width), -1), np.zeros(S, dtype=np.int64)
    order = rng.permutation(pages)
    held = int(case["used"] * pages)      # by others than these sequences
    refs[order[:held]] = rng.integers(1, 4, held)
    x = {"case": case}
    if case["what"] == "drafts":
        length = np.maximum(ask, 8)
        at = held
        for s in range(S):
            need = -(-int(length[s]) // P)
            table[s, :need] = order[at:at + need]
            refs[order[at:at + need]] = 1
            at += need
        rejected = rng.integers(1, 5, S)
        x["calls"] = [(_i32(-rejected), None), (_i32(rejected), None)]
    elif case["what"] == "prompts":
        x["calls"] = [(_i32(ask), _i32(np.full(S, -1)))]
    else:
        first = np.arange(S) // beams * beams
        x["calls"] = [(_i32(np.where(np.arange(S) == first, ask, 0)), _i32(np.full(S, -1))), (_i32(np.ones(S)), _i32(first))]
        gen = torch.Generator(device=DEVICE).manual_seed(seed)
        for name in ("k_pool", "v_pool"):
            x[name] = torch.randn((pages, P, 4, 128), generator=gen, device=DEVICE, dtype=torch.bfloat16)
    x["state"] = {"page_table": table, "seq_len": length, "page_refs": refs}
    x["tokens"] = {"drafts": 4 * S, "prompts": S * case["most"], "beams": S // beams * case["most"]}[case["what"]]
    return x


def _beam_inputs(case, seed):
    rng = np.random.default_rng([seed, 78])
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    Q, W, V = case["queries"], case["beams"], case["vocab"]
    # what a model's head gives: a broad bulk, and a few tokens well above it
    logits = torch.randn((Q * W, V), generator=gen, device=DEVICE) * 2.5
    few = torch.randint(0, V, (Q * W, 40), generator=gen, device=DEVICE)
    logits.scatter_add_(1, few, 4 - 4 * torch.log(torch.rand((Q * W, 40), generator=gen, device=DEVICE).clamp_min(1e-9)))
    f32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(DEVICE)
    x = {"case": case, "logits": logits.to(TYPES[case["dtype"]]), "scores": f32(-np.sort(rng.gamma(8, 2, (Q, W)), axis=1)),
         "ended": None, "factor": None, "end": -1}
    if case["ended"]:
        ended = rng.random((Q, W)) < 0.25
        tokens = np.where(ended, rng.integers(5, 40, (Q, W)), 40)
        x.update(ended=_i32(ended), factor=f32(tokens ** -0.7), end=2)
    return x


def prepare(case, seed):
    if case["op"] == "beam":
        x = _beam_inputs(case, seed)
        shape = (case["queries"], case["picks"])
        x["out"] = [torch.empty(shape, dtype=d, device=DEVICE) for d in (torch.int32, torch.int32, torch.float32)]
    elif case["op"] == "advance":
        x = _advance_inputs(case, seed)
    else:
        x = _cache_inputs(case, seed)
        x["out"] = torch.empty((x["q"].shape[0], case["heads"], case["dim"]), dtype=x["q"].dtype, device=DEVICE)
    if own:
        import paper_1905_13348_amd as infaas
        x["worker"] = w = infaas.Executor(device=0)
        if case["op"] == "advance":
            S, width = x["state"]["page_table"].shape
            x["table"] = w.table(S, width, case["page"], case["pages"], x["tokens"])
            if case["what"] == "beams":
                x["cache"] = w.cache(x["k_pool"], x["v_pool"])
        elif case["op"] != "beam":
            x["cache"] = w.cache(x["k_pool"], x["v_pool"], layout=case["layout"], k_scale=x["k_scale"], v_scale=x["v_scale"],
                                 dtype=x["q"].dtype)
            common = dict(seq_len=x["length"], page_table=x["table"], max_len=x["most"])
            x["batch"] = w.batch(x["cache"], case["heads"], token_seq=x["seq"], token_pos=x["pos"], seq_start=x["start"],
                                 group_start=x["group_start"], shared_len=x["shared"], **common)
            if case["op"] == "attend":
                w.plan(x["batch"])      # (once a step, for all layers)
            else:
                x["whole"] = w.batch(x["cache"], case["heads"], token_seq=x["all_seq"], token_pos=x["all_pos"],
                                     seq_start=x["all_start"], **common)
    elif case["op"] == "advance":
        x["table"] = SimpleNamespace()
    if case["op"] == "advance":
        for name, a in x["state"].items():
            if own:
                getattr(x["table"], name).copy_(_i32(a))
            else:
                setattr(x["table"], name, _i32(a))
    elif case["op"] == "append":
        x["read"] = [torch.empty((x["all_seq"].shape[0], case["kv_heads"], case["dim"]), dtype=x["q"].dtype, device=DEVICE)
                     for _ in range(2)]
    return x


# ---- one pass -------------------------------------------------------------------------------------------------

def run(x):
    case = x["case"]
    if case["op"] == "append":
        if own:
            x["worker"].append(x["cache"], x["batch"], x["q"], x["k"], x["v"], x["out"], x["freq"],
                               interleaved=case["interleaved"])
            x["worker"].read(x["cache"], x["whole"], *x["read"])
            return x["out"], *x["read"]
        return _plain_append(x)
    if case["op"] == "attend":
        if own:
            x["worker"].attend(x["cache"], x["batch"], x["q"], x["out"], x["scale"])
            return x["out"]
        return _plain_attend(x)
    if case["op"] == "advance":
        for new, parent in x["calls"]:
            if own:
                x["worker"].advance(x["table"], new, parent)
            else:
                _plain_advance(x, x["table"], new, parent)
        if case["what"] == "beams":
            if own:
                x["worker"].copy(x["cache"], x["table"])
            else:
                _plain_copy(x, x["table"])
        t = x["table"]
        out = {n: getattr(t, n) for n in ("page_table", "seq_len", "page_refs", "seq_start", "token_seq", "token_pos", "taken",
                                          "copies")}
        if case["what"] == "beams":
            out.update(k_pool=x["k_pool"], v_pool=x["v_pool"])
        return out
    if own:
        x["worker"].beam(x["logits"], x["scores"], *x["out"], ended=x["ended"], factor=x["factor"], end_token=x["end"])
        return x["out"]
    return _plain_beam(x)


def _plain_rotate(a, cos, sin, interleaved):
    half = cos.shape[-1]
    y = a.float()
    y = y.clone() if y is a else y
    if interleaved:
        p, q = a[..., 0:2 * half:2].float(), a[..., 1:2 * half:2].float()
        y[..., 0:2 * half:2], y[..., 1:2 * half:2] = p * cos - q * sin, q * cos + p * sin
    else:
        p, q = a[..., :half].float(), a[..., half:2 * half].float()
        y[..., :half], y[..., half:2 * half] = p * cos - q * sin, q * cos + p * sin
    return y


def _power(scale):
    """2 ** (byte - 127) of bytes 1 .. 254, in 32 bits."""
    return (scale.to(torch.int32) << 23).view(torch.float32)


def _plain_append(x):
    case, P, B = x["case"], x["case"]["page"], x["case"]["block"]
    Hkv, D = case["kv_heads"], case["dim"]
    angle = x["pos"].double()[:, None] * x["freq"][None, :]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    out = [_plain_rotate(x["q"], cos, sin, case["interleaved"]).to(x["q"].dtype)]
    page = x["table"][x["seq"].long(), (x["pos"] // P).long()].long()
    slot = (x["pos"] % P).long()
    at = page * (P // B) + slot // B
    all_page = x["table"][x["all_seq"].long(), (x["all_pos"] // P).long()].long()
    all_slot = (x["all_pos"] % P).long()
    for name in ("k", "v"):
        new = _plain_rotate(x["k"], cos, sin, case["interleaved"]) if name == "k" else x["v"].float()
        codes, scale = x[name + "_pool"].view(torch.uint8), x[name + "_scale"].view(torch.uint8)
        if case["layout"] == "head":      # (views, with a page's tokens in front of the heads)
            codes, scale = codes.transpose(1, 2), scale.transpose(1, 2)
        # the least power of two that the block's new tokens need
        most = torch.zeros((scale.shape[0] * scale.shape[1], Hkv), device=DEVICE)
        most = most.scatter_reduce(0, at[:, None].expand(-1, Hkv), new.abs().amax(dim=2), "amax")
        need = (((most.view(torch.int32) + 0x1fffff) >> 23) - 8).clamp_min(1).view(scale.shape)
        # a block that begins with this step has no scale of before
        flags = torch.zeros((2, scale.shape[0] * scale.shape[1]), dtype=torch.bool, device=DEVICE)
        begun = flags[0].index_fill(0, at[slot % B == 0], True).view(scale.shape[:2])[:, :, None]
        touched = flags[1].index_fill(0, at, True).view(scale.shape[:2])[:, :, None]
        old = scale.to(torch.int32)
        now = torch.where(touched, torch.maximum(need, torch.where(begun, 1, old)), old)
        # what the block holds goes down with the scale's rise
        blocks, where = codes.unflatten(1, (P // B, B)), (page, slot // B)
        held = blocks[where].view(CODES).float() * _power(127 + (old - now)[where].clamp_min(-126))[:, None, :, None]
        blocks[where] = held.to(CODES).view(torch.uint8)
        codes[page, slot] = (new / _power(now[where])[:, :, None]).to(CODES).view(torch.uint8)
        scale.copy_(now.to(torch.uint8))
        value = codes[all_page, all_slot].view(CODES).float() * _power(scale[all_page, all_slot // B])[:, :, None]
        out.append(value.to(x["q"].dtype))
    return out


def _gather(x, name):
    """Keys or values of all sequences, [sequence, kv head, key, dim] in 32 bits, rounded to the queries' type."""
    case, B = x["case"], x["case"]["block"]
    pages = x["table"].long()
    codes, power = x[name + "_pool"].view(torch.uint8)[pages].view(CODES).float(), _power(x[name + "_scale"].view(torch.uint8)[pages])
    if case["layout"] == "head":
        codes, power = codes.transpose(2, 3), power.transpose(2, 3)
    codes = codes * power.repeat_interleave(B, dim=2)[..., None]
    return codes.to(x["q"].dtype).float().flatten(1, 2).transpose(1, 2).contiguous()


def _plain_attend(x):
    case = x["case"]
    S, H, Hkv, D = case["seqs"], case["heads"], case["kv_heads"], case["dim"]
    G, most = H // Hkv, x["most_new"]
    seq, row = x["seq"].long(), torch.arange(x["seq"].shape[0], device=DEVICE) - x["start"][x["seq"].long()]
    q = torch.zeros((S, most, H, D), device=DEVICE)
    q[seq, row] = x["q"].float() * x["scale"]
    q = q.view(S, most, Hkv, G, D).transpose(1, 2).reshape(S, Hkv, most * G, D)
    limit = torch.zeros((S, most), dtype=torch.int32, device=DEVICE)
    limit[seq, row] = x["pos"]
    k = _gather(x, "k")
    score = torch.matmul(q, k.transpose(2, 3).contiguous())
    del k
    keys = torch.arange(score.shape[3], device=DEVICE, dtype=torch.int32)
    hidden = keys[None, None, :] > limit.repeat_interleave(G, dim=1)[:, :, None]
    score = score.masked_fill_(hidden[:, None], -math.inf)
    score = torch.exp_(score.sub_(score.amax(dim=3, keepdim=True)))
    v = _gather(x, "v")
    v.masked_fill_((keys[None, :] >= x["length"][:, None])[:, None, :, None], 0)
    o = torch.matmul(score, v) / score.sum(dim=3, keepdim=True)
    o = o.view(S, Hkv, most, G, D).transpose(1, 2).reshape(S, most, H, D)
    return o[seq, row].to(x["q"].dtype)


def _plain_advance(x, t, new, parent):
    P, S, W = x["case"]["page"], *t.page_table.shape
    N, cols, rows = x["case"]["pages"], torch.arange(t.page_table.shape[1], device=DEVICE), torch.arange(S, device=DEVICE)
    pages_of = lambda n: (n + P - 1) // P
    count = lambda table: torch.bincount(table[table >= 0], minlength=N)
    new, length, table, refs = new.long(), t.seq_len.long(), t.page_table.long(), t.page_refs.long()
    refs = refs - count(table)
    if parent is not None:
        there = (parent >= 0) & (parent < S)
        p = torch.where(there, parent, 0).long()
        length, table = torch.where(there, length[p], 0), torch.where(there[:, None], table[p], -1)
    length = (length + new.clamp_max(0)).clamp_min(0)
    table = torch.where(cols < pages_of(length)[:, None], table, -1)
    refs = refs + count(table)
    # what each sequence asks for, and whether there is as much for it and those in front of it
    wants = (new > 0) & (length + new <= W * P)
    last = table[rows, (length // P).clamp_max(W - 1)]
    copy = wants & (length % P > 0) & (refs[last.clamp_min(0)] > 1)
    wants = wants & (torch.cumsum(torch.where(wants, new, 0), 0) <= x["tokens"])
    need = torch.where(wants, pages_of(length + new) - pages_of(length) + copy, 0)
    upto = torch.cumsum(need, 0)
    free = torch.sort((refs != 0).to(torch.int8), stable=True).indices
    served = wants & ((need == 0) | (upto <= (refs == 0).sum()))
    copy = copy & served
    taken = torch.where(served, new, 0)
    base = upto - need
    to = free[base.clamp_max(N - 1)]
    t.copies = torch.where(copy[:, None], torch.stack([last, to, length % P], dim=1), -1).int()
    refs.index_add_(0, last[copy], -torch.ones_like(last[copy]))
    at = base[:, None] + copy[:, None] + cols - pages_of(length)[:, None]
    fresh = (cols >= pages_of(length)[:, None]) & (cols < pages_of(length + taken)[:, None])
    table = torch.where(fresh, free[at.clamp(0, N - 1)], table)
    table = torch.where(copy[:, None] & (cols == (length // P)[:, None]), to[:, None], table)
    refs[table[fresh]] = 1
    refs[to[copy]] = 1
    start = torch.cat([taken.new_zeros(1), torch.cumsum(taken, 0)])
    i = torch.arange(x["tokens"], device=DEVICE)
    seq = torch.searchsorted(start, i, right=True) - 1
    real = seq < S
    seq = torch.where(real, seq, 0)
    t.token_seq = torch.where(real, seq, -1).int()
    t.token_pos = torch.where(real, length[seq] + i - start[seq], -1).int()
    t.seq_start, t.taken, t.seq_len = start.int(), taken.int(), (length + taken).int()
    t.page_table, t.page_refs = table.int(), refs.int()


def _plain_copy(x, t):
    source, to, slots = t.copies[t.copies[:, 0] >= 0].long().unbind(1)
    keep = torch.arange(x["case"]["page"], device=DEVICE)[None, :] >= slots[:, None]
    for pool in (x["k_pool"], x["v_pool"]):
        pool[to] = torch.where(keep[:, :, None, None], pool[to], pool[source])


def _plain_beam(x):
    case = x["case"]
    Q, W, V, K = (case[k] for k in ("queries", "beams", "vocab", "picks"))
    logits = x["logits"].double()
    top = logits.amax(dim=1, keepdim=True)
    score = logits - top - torch.log(torch.exp(logits - top).sum(dim=1, keepdim=True))
    score = score.view(Q, W, V) + x["scores"].double()[:, :, None]
    if x["ended"] is not None:
        alone = torch.full((Q, W, V), -math.inf, dtype=torch.float64, device=DEVICE)
        alone[:, :, x["end"]] = x["scores"].double()
        score = torch.where(x["ended"][:, :, None] != 0, alone, score)
    rank = score if x["factor"] is None else score * x["factor"].double()[:, :, None]
    best = torch.sort(rank.flatten(1), dim=1, descending=True, stable=True).indices[:, :K]
    there = rank.flatten(1).gather(1, best) > -math.inf      # (where beams have ended there may be fewer than were asked for)
    parent = torch.arange(Q, device=DEVICE)[:, None] * W + best // V
    return [torch.where(there, parent, -1).int(), torch.where(there, best % V, -1).int(),
            torch.where(there, score.flatten(1).gather(1, best), -math.inf).float()]


# ---- what a pass cannot do without ------------------------------------------------------------------------------

def work(case):
    if case["op"] == "beam":
        n = case["queries"] * case["beams"] * case["vocab"]
        return {"bytes": n * (4 if case["dtype"] == "fp32" else 2) + 12 * case["queries"] * (case["beams"] + case["picks"]),
                "flops": 4 * n}
    if case["op"] == "advance":
        # counts of all pages, a sequence's length, ask and answers, the entries of pages that come or go, tokens' arrays
        S, P, most = case["seqs"], case["page"], case["most"]
        mean = 0.34 * most                  # of lengths whose logarithm is uniform from most/16 to most
        if case["what"] == "drafts":
            tokens, entries, room, moved = 2.5 * S, 5 * S / P, 4 * S, 0
        elif case["what"] == "prompts":
            tokens, entries, room, moved = S * mean, 2 * S * mean / P, S * most, 0
        else:
            S1 = S // case["beams"]
            tokens, entries, room = S1 * mean + S, 2 * S * mean / P, S1 * most
            moved = 4 * S * (P - 1) / 2 * 4 * 128 * 2
        return {"bytes": 4.0 * case["pages"] + 40.0 * S + 8.0 * entries + 8.0 * room + moved, "flops": tokens + 8 * entries + 20 * S}
    H, Hkv, D = case["heads"], case["kv_heads"], case["dim"]
    own_len, new, group_start, shared = _lengths(case)
    if case["op"] == "append":
        n, whole = case["tokens"], float(own_len.sum())
        return {"bytes": n * D * (4 * H + 6 * Hkv) + 6 * whole * Hkv * D,
                "flops": 3 * n * (H + Hkv) * case["rot"] + 4 * n * Hkv * D + 2 * whole * Hkv * D}
    seqs = np.diff(group_start)
    front = np.repeat(shared, seqs)
    before = own_len - new
    # the shared part is seen by every token, of its own part token i of n sees what came before and itself
    pairs = float((new * front + new * before + new * (new + 1) // 2).sum())
    keys = float(shared.sum() + own_len.sum())
    return {"bytes": 2 * Hkv * keys * (D + 1 / case["block"]) + 4 * float(new.sum()) * H * D, "flops": 4 * pairs * H * D}


# ---- the definition in 64 bits ----------------------------------------------------------------------------------

def exact(case, seed):
    if case["op"] == "beam":
        return _exact_beam(_beam_inputs(case, seed))
    if case["op"] == "advance":
        return _exact_advance(_advance_inputs(case, seed))
    x = _cache_inputs(case, seed)
    return _exact_append(x) if case["op"] == "append" else _exact_attend(x)


def _code(x):
    """x in 64 bits, rounded to the numbers of e4m3: three bits behind the first one, steps of 2^-9 at the least."""
    step = torch.exp2(torch.frexp(x)[1].clamp_min(-5).double() - 4)
    return (torch.round(x / step) * step).clamp(-LARGEST, LARGEST)


def _slots(x, seq, pos):
    """Pages and slots of (sequence, position), on the host."""
    P, table = x["case"]["page"], x["table"].cpu().numpy().astype(np.int64)
    return torch.from_numpy(table[seq, pos // P]).to(DEVICE), torch.from_numpy(pos % P).to(DEVICE)


def _exact_append(x):
    case, P, B, half = x["case"], x["case"]["page"], x["case"]["block"], x["case"]["rot"] // 2
    pos, seq, every, where = (x[n].cpu().numpy().astype(np.int64) for n in ("pos", "seq", "all_pos", "all_seq"))
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEVICE),
                       torch.from_numpy(np.outer(pos, x["freq"].cpu().numpy())).to(DEVICE))[:, None, :]

    def rotated(a):
        a = a.double()
        front = a[..., :2 * half]
        pairs = front.unflatten(-1, (half, 2)) if case["interleaved"] else front.unflatten(-1, (2, half)).transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        z = z if case["interleaved"] else z.transpose(-1, -2)
        return torch.cat([z.flatten(-2), a[..., 2 * half:]], dim=-1)

    # blocks by (sequence, number): the tokens that each gets, and with them its scale
    edge = np.flatnonzero(np.concatenate([[True], (seq[1:] != seq[:-1]) | (pos[1:] // B != pos[:-1] // B), [True]]))
    page, slot = _slots(x, seq, pos)
    page_all, slot_all = _slots(x, where, every)
    run = torch.from_numpy(np.repeat(np.arange(len(edge) - 1), np.diff(edge))).to(DEVICE)
    first = torch.from_numpy(edge[:-1]).to(DEVICE)
    out = [rotated(x["q"])]
    for name in ("k", "v"):
        new = rotated(x["k"]) if name == "k" else x["v"].double()
        codes, scale = x[name + "_pool"].float().double(), x[name + "_scale"].view(torch.uint8).long()
        if case["layout"] == "head":
            codes, scale = codes.transpose(1, 2), scale.transpose(1, 2)
        codes, scale = codes.contiguous(), scale.contiguous()
        high = new.abs().amax(dim=2)
        most = torch.zeros((len(edge) - 1, high.shape[1]), dtype=torch.float64, device=DEVICE)
        most.index_reduce_(0, run, high, "amax")
        # the least e with most <= 448 * 2^e = 0.875 * 2^(e + 9)
        fraction, power = torch.frexp(most)
        need = (power.long() - 9 + (fraction > 0.875).long() + 127).clamp_min(1)
        need = torch.where(most == 0, 1, need)
        p0, b0, s0 = page[first], slot[first] // B, slot[first] % B
        old = scale[p0, b0]
        now = torch.maximum(need, torch.where((s0 == 0)[:, None], 1, old))
        block = codes.unflatten(1, (P // B, B))
        held = block[p0, b0] * torch.exp2((old - now).double())[:, None, :, None]
        before = (torch.arange(B, device=DEVICE)[None, :] < s0[:, None])[:, :, None, None]
        block[p0, b0] = torch.where(before, _code(held), block[p0, b0])
        scale[p0, b0] = now
        codes[page, slot] = _code(new * torch.exp2(127.0 - now[run].double())[:, :, None])
        value = codes[page_all, slot_all] * torch.exp2(scale[page_all, slot_all // B].double() - 127)[:, :, None]
        out.append(value)
    return out


def _exact_attend(x):
    case, P, B = x["case"], x["case"]["page"], x["case"]["block"]
    H, Hkv = case["heads"], case["kv_heads"]
    start, length, pos = (x[n].cpu().numpy().astype(np.int64) for n in ("start", "length", "pos"))
    if 4.0 * H * case["dim"] * float((length * np.diff(start)).sum()) > 2e13:
        return None
    out = torch.empty(x["q"].shape, dtype=torch.float64, device=DEVICE)
    for s in range(case["seqs"]):
        n = int(length[s])
        page, slot = _slots(x, np.full(n, s), np.arange(n))
        tokens = slice(int(start[s]), int(start[s + 1]))
        seen = torch.arange(n, device=DEVICE)[None, :] <= torch.from_numpy(pos[tokens]).to(DEVICE)[:, None]
        k, v = [], []
        for to, name in ((k, "k"), (v, "v")):
            codes, scale = x[name + "_pool"], x[name + "_scale"].view(torch.uint8)
            if case["layout"] == "head":
                codes, scale = codes.transpose(1, 2), scale.transpose(1, 2)
            value = codes.view(torch.uint8)[page, slot].view(CODES).float().double()
            value = value * torch.exp2(scale[page, slot // B].double() - 127)[:, :, None]
            to.append(value.to(x["q"].dtype).double().transpose(0, 1).contiguous())
        q = x["q"][tokens].double().transpose(0, 1).reshape(Hkv, H // Hkv * (tokens.stop - tokens.start), -1).contiguous()
        score = torch.matmul(q, k[0].transpose(1, 2).contiguous()) * x["scale"]
        score.masked_fill_(~seen.repeat(H // Hkv, 1)[None], -math.inf)
        o = torch.matmul(torch.softmax(score, dim=2), v[0])
        out[tokens] = o.reshape(H, tokens.stop - tokens.start, -1).transpose(0, 1)
    return out


def _exact_advance(x):
    case, P = x["case"], x["case"]["page"]
    table = [[int(p) for p in row if p >= 0] for row in x["state"]["page_table"]]
    length, refs = [int(n) for n in x["state"]["seq_len"]], [int(n) for n in x["state"]["page_refs"]]
    S, W, room = len(table), x["state"]["page_table"].shape[1], x["tokens"]
    for new, parent in x["calls"]:
        new = new.tolist()
        old = table
        if parent is not None:
            before = length
            table = [list(old[p]) if 0 <= p < S else [] for p in parent.tolist()]
            length = [before[p] if 0 <= p < S else 0 for p in parent.tolist()]
        else:
            table = [list(row) for row in old]
        for s in range(S):
            length[s] = max(0, length[s] + min(new[s], 0))
            del table[s][-(-length[s] // P):]
        for row in old:
            for p in row:
                refs[p] -= 1
        for row in table:
            for p in row:
                refs[p] += 1
        free = [p for p, r in enumerate(refs) if r == 0]
        left, asked, at = room, 0, 0
        taken, copies, seq, where, leave = [0] * S, [[-1] * 3 for _ in range(S)], [], [], []
        for s in range(S):
            n = new[s]
            if n <= 0 or length[s] + n > W * P:
                continue
            left -= n
            if left < 0:
                continue
            own_copy = length[s] % P > 0 and refs[table[s][-1]] > 1
            need = -(-(length[s] + n) // P) - len(table[s]) + own_copy
            asked += need
            if need and asked > len(free):
                continue
            if own_copy:
                copies[s] = [table[s][-1], free[at], length[s] % P]
                leave.append(table[s][-1])
                table[s][-1] = free[at]
            table[s] += free[at + own_copy:at + need]
            at += need
            seq += [s] * n
            where += range(length[s], length[s] + n)
            taken[s] = n
            length[s] += n
        for p in leave:
            refs[p] -= 1
        for p in free[:at]:
            refs[p] = 1
    i32 = lambda a: np.array(a, dtype=np.int32)
    pad = [-1] * (room - len(seq))
    out = {"page_table": i32([row + [-1] * (W - len(row)) for row in table]), "seq_len": i32(length), "page_refs": i32(refs),
           "seq_start": i32(np.concatenate([[0], np.cumsum(taken)])), "token_seq": i32(seq + pad), "token_pos": i32(where + pad),
           "taken": i32(taken), "copies": i32(copies)}
    if case["what"] == "beams":
        for name in ("k_pool", "v_pool"):
            pool = x[name].double()
            for a, b, n in copies:
                if a >= 0:
                    pool[b, :n] = x[name][a, :n].double()
            out[name] = pool
    return out


def _exact_beam(x):
    case = x["case"]
    Q, W, V, K = (case[k] for k in ("queries", "beams", "vocab", "picks"))
    scores = x["scores"].cpu().numpy().astype(np.float64)
    ended = np.zeros((Q, W), dtype=bool) if x["ended"] is None else x["ended"].cpu().numpy() != 0
    factor = np.ones((Q, W)) if x["factor"] is None else x["factor"].cpu().numpy().astype(np.float64)
    found = []
    for q in range(Q):
        rows = x["logits"][q * W:(q + 1) * W].double().cpu().numpy()
        best = []      # (rank, beam, token, score)
        for w in range(W):
            if ended[q, w]:
                best.append((-scores[q, w] * factor[q, w], w, x["end"], scores[q, w]))
                continue
            row = rows[w]
            norm = row.max() + math.log(np.exp(row - row.max()).sum())
            border = np.partition(row, V - min(K, V))[V - min(K, V)]
            for i in np.flatnonzero(row >= border):
                score = scores[q, w] + row[i] - norm
                best.append((-score * factor[q, w], w, int(i), score))
        best = [(q * W + b[1], b[2], b[3]) for b in sorted(best)[:K]]
        found.append(best + [(-1, -1, -math.inf)] * (K - len(best)))
    columns = [np.array([[f[j] for f in row] for row in found]) for j in range(3)]
    return [columns[0].astype(np.int32), columns[1].astype(np.int32), columns[2]]
