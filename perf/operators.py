"""Operators for serving a transformer at 8 bits: what is timed, and their plain forms.

Three groups that a decoding step uses together: linear layers whose activations are quantized token by token
(`linear`), a paged key/value cache held in int8 with one maximum for each page and head -- written (`append`) and read
by attention (`attention`) -- and the calls that fork sequences and compact the cache (`pages`).

`listed()` holds the cases of fixed size, `draw()` gives further ones of the same ranges, `prepare()` builds what the
caller holds before the call, `run()` makes one pass -- with `own` through the library, without it in elementary torch
operations -- `exact()` states the result in 64 bits, and `work()` what a pass cannot do without.

Codes and scales follow the library's rule: A = max|x|, scale = A / 127 and inverse = 127 / A, one IEEE fp32 division
each (A = 0 gives 1 and 1), code = clamp(round_half_even(fp32(x * inverse)), -127, 127).
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}
QMAX = 127.0


# ------------------------------------------------------------------------------------ the cases

def listed():
    return [
        # a decoding step of 24 sequences through a wide projection: the weights are the traffic
        {"name": "linear_decode", "kind": "linear", "m": 24, "k": 4096, "n": 16384, "dtype": "bf16", "act": "none", "bias": False},
        # a prompt of odd length through a layer of odd sizes: ragged tiles in all three directions
        {"name": "linear_odd", "kind": "linear", "m": 1037, "k": 4001, "n": 2311, "dtype": "fp16", "act": "relu", "bias": True},
        # the first feed-forward layer of a BERT-base block on 32 sequences of 384 tokens
        {"name": "linear_block", "kind": "linear", "m": 32 * 384, "k": 768, "n": 3072, "dtype": "fp32", "act": "gelu", "bias": True},
        # one new token for each of 64 sequences: the smallest writes, some of which raise their page's maximum
        {"name": "append_decode", "kind": "append", "n": 64, "new": 1, "context": 700, "heads": 8, "dim": 128, "page": 64, "dtype": "bf16"},
        # eight prompts of different lengths, some of them behind a context that ends inside a page
        {"name": "append_prompt", "kind": "append", "n": 8, "new": 2000, "context": 300, "heads": 8, "dim": 128, "page": 16, "dtype": "fp32"},
        # a few short chats, where launches and latency are the cost
        {"name": "attention_short", "kind": "attention", "n": 8, "new": 1, "context": 200, "q_heads": 12, "heads": 12, "dim": 64, "page": 16, "dtype": "fp16", "causal": True},
        # a busy decoding batch of ragged lengths with shared heads: the cache is the traffic
        {"name": "attention_batch", "kind": "attention", "n": 64, "new": 1, "context": 8000, "q_heads": 32, "heads": 8, "dim": 128, "page": 64, "dtype": "bf16", "causal": True},
        # one token over one very long context: a single row of work to spread over the GPU
        {"name": "attention_long", "kind": "attention", "n": 1, "new": 1, "context": 131000, "q_heads": 32, "heads": 8, "dim": 128, "page": 64, "dtype": "bf16", "causal": True},
        # chunks of prompts behind contexts of different lengths: the products are the work
        {"name": "attention_prompt", "kind": "attention", "n": 4, "new": 2048, "context": 4000, "q_heads": 32, "heads": 8, "dim": 128, "page": 64, "dtype": "bf16", "causal": True},
        # an encoder's pass over 32 padded sequences of up to 384 tokens, every token seeing all of them
        {"name": "attention_encoder", "kind": "attention", "n": 32, "new": 384, "context": 0, "q_heads": 12, "heads": 12, "dim": 64, "page": 64, "dtype": "fp32", "causal": False},
        # beams: 16 prompts forked four times each, full pages shared and the last page copied
        {"name": "pages_fork", "kind": "fork", "n": 16, "beams": 4, "context": 1500, "heads": 8, "dim": 128, "page": 64},
        # a pool that half of its sequences have left, compacted into its first pages
        {"name": "pages_compact", "kind": "compact", "n": 96, "context": 2600, "heads": 8, "dim": 128, "page": 64},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["linear", "append", "attention", "attention", "fork", "compact"])
    dtype = rng.choice(["fp32", "bf16", "fp16"])
    page = rng.choice([16, 32, 64, 128])
    heads, group = rng.choice([(1, 8), (2, 4), (4, 7), (8, 4), (8, 1), (12, 1), (16, 1)])
    dim = rng.choice([64, 128])
    if kind == "linear":
        while True:
            m, k, n = _log_int(rng, 1, 12000), _log_int(rng, 64, 16000), _log_int(rng, 64, 16000)
            if m * k * n <= 32 * 384 * 768 * 3072 and n * k <= 4096 * 16384:
                break
        return {"kind": kind, "m": m, "k": k, "n": n, "dtype": dtype, "act": rng.choice(["none", "relu", "gelu"]), "bias": rng.random() < 0.5}
    if kind == "append":
        n = _log_int(rng, 1, 200)
        new = _log_int(rng, 1, max(1, 16000 // n))
        context = _log_int(rng, 1, max(2, 60000 // n))
        return {"kind": kind, "n": n, "new": new, "context": context, "heads": heads, "dim": dim, "page": page, "dtype": dtype}
    if kind == "attention":
        n = _log_int(rng, 1, 200)
        new = 1 if rng.random() < 0.5 else _log_int(rng, 2, max(2, 4000 // n))
        context = _log_int(rng, 1, max(2, min(130000, 400000 // n, 10000000 // (n * new))))
        return {"kind": kind, "n": n, "new": new, "context": context, "q_heads": heads * group, "heads": heads, "dim": dim,
                "page": page, "dtype": dtype, "causal": rng.random() < 0.8}
    n = _log_int(rng, 2, 100)
    context = _log_int(rng, 1, 200000 // n)
    if kind == "fork":
        return {"kind": kind, "n": n, "beams": rng.randint(1, 4), "context": context, "heads": heads, "dim": dim, "page": page}
    return {"kind": kind, "n": n, "context": context, "heads": heads, "dim": dim, "page": page}


# ------------------------------------------------------------------------------------ lengths and pages

def _lengths(case):
    """(tokens held before, new tokens) of every sequence, from the case alone: ragged, the first one full."""
    n, context, new = case["n"], case["context"], case.get("new", 0)
    r = random.Random(n * 1000003 + context * 101 + new)
    held = [context] + [r.randint(0, context) for _ in range(n - 1)]
    fresh = [new] + [r.randint(max(1, new // 4), new) if new else 0 for _ in range(n - 1)]
    return held, fresh


def _pages_of(tokens, page):
    return -(-tokens // page)


def _starts(counts):
    s = [0]
    for c in counts:
        s.append(s[-1] + c)
    return s


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _fill(shape, g):
    """Codes as a cache holds them: bell-shaped, the largest near the grid's end."""
    return (torch.randn(shape, generator=g, device="cuda") * 40.0).round_().clamp_(-QMAX, QMAX).to(torch.int8)


def _cache(case, lengths, g, spare, max_seqs=None):
    """Tensors of a pool and one layer's cache whose sequences hold `lengths` tokens in pages handed out at random."""
    page, heads, dim = case["page"], case["heads"], case["dim"]
    need = [_pages_of(t, page) for t in lengths]
    n_pages = max(1, sum(need) + spare)
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32).cpu()
    max_seqs = max_seqs or len(lengths)
    max_pages = max(need) + 1
    table = torch.full((max_seqs, max_pages), -1, dtype=torch.int32)
    refs = torch.zeros(n_pages, dtype=torch.int32)
    at = 0
    for i, c in enumerate(need):
        table[i, :c] = order[at:at + c]
        refs[order[at:at + c].long()] = 1
        at += c
    lens = torch.zeros(max_seqs, dtype=torch.int32)
    lens[:len(lengths)] = torch.tensor(lengths, dtype=torch.int32)
    shape = (n_pages, heads, page, dim)
    state = {"table": table.cuda(), "lens": lens.cuda(), "refs": refs.cuda(), "k": _fill(shape, g), "v": _fill(shape, g)}
    for name in ("k_absmax", "v_absmax"):
        state[name] = torch.exp(torch.randn((n_pages, heads), generator=g, device="cuda") * 0.25 + 1.1)
    return state


def _handles(state, case):
    """With `own`: the library's handles over the same tensors."""
    import paper_2302_01382_b200 as q
    ctx = q.Context(torch.cuda.current_device())
    pool = q.KvPool(ctx, state["refs"].numel(), case["page"], state["table"].shape[0], state["table"].shape[1],
                    table=state["table"], lens=state["lens"], refs=state["refs"])
    cache = q.KvCache(pool, case["heads"], case["dim"], k=state["k"], v=state["v"], k_absmax=state["k_absmax"],
                      v_absmax=state["v_absmax"])
    state.update(ctx=ctx, pool=pool, cache=cache)


# ------------------------------------------------------------------------------------ prepare

def _inputs(case, seed):
    """The tensors of a pass, the same for both sides and for exact()."""
    g = _gen(seed)
    state = {"case": dict(case)}
    kind = case["kind"]
    if kind == "linear":
        m, k, n, dt = case["m"], case["k"], case["n"], DTYPES[case["dtype"]]
        x = torch.randn((m, k), generator=g, device="cuda")
        x *= 1.0 + 15.0 * (torch.rand((1, k), generator=g, device="cuda") < 0.002)      # a few channels are outliers
        state["x"] = x.to(dt)
        ldw = -(-k // 16) * 16
        w = torch.zeros((n, ldw), dtype=torch.int8, device="cuda")
        w[:, :k] = _fill((n, k), g)
        state["w"] = w
        state["scale_w"] = torch.exp(torch.randn(n, generator=g, device="cuda") * 0.2) * (3.0 / (QMAX * math.sqrt(k)))
        state["bias"] = torch.randn(n, generator=g, device="cuda") * 0.1 if case["bias"] else None
        return state
    held, fresh = _lengths(case)
    if kind in ("append", "attention"):
        total = [a + b for a, b in zip(held, fresh)]
        state.update(_cache(case, total, g, spare=7))
        state["seqs"] = _ints(list(range(case["n"])))
        state["starts"] = _ints(_starts(fresh))
        state["tokens"] = sum(fresh)
        if kind == "append":
            shape = (sum(fresh), case["heads"], case["dim"])
            for name in ("k_new", "v_new"):
                state[name] = torch.randn(shape, generator=g, device="cuda").to(DTYPES[case["dtype"]])
            first = [a // case["page"] * case["page"] for a in held]
            state["first"] = _ints(first)
            state["read_starts"] = _ints(_starts([t - f for t, f in zip(total, first)]))
            state["read_tokens"] = sum(total) - sum(first)
        else:
            shape = (sum(fresh), case["q_heads"], case["dim"])
            state["q"] = torch.randn(shape, generator=g, device="cuda").to(DTYPES[case["dtype"]])
            state["max_new"] = max(fresh)
            state["max_len"] = max(total)
        return state
    if kind == "fork":
        n, beams = case["n"], case["beams"]
        state.update(_cache(case, held, g, spare=n * beams + 5, max_seqs=n * (1 + beams)))
        state["parents"] = _ints([i for i in range(n) for _ in range(beams)])
        state["children"] = _ints([n + i for i in range(n * beams)])
        return state
    state.update(_cache(case, held, g, spare=11))
    gone = torch.arange(case["n"], device="cuda") % 2 == 1
    # what a serving loop holds when half of its sequences have left
    table, refs = state["table"], state["refs"]
    left = table[gone]
    refs[left[left >= 0].long()] = 0
    table[gone] = -1
    state["lens"][gone] = 0
    state["table_was"], state["refs_was"] = table.clone(), refs.clone()
    return state


def prepare(case, seed):
    state = _inputs(case, seed)
    if own:
        if case["kind"] == "linear":
            import paper_2302_01382_b200 as q
            state["ctx"] = q.Context(torch.cuda.current_device())
        else:
            _handles(state, case)
    return state


# ------------------------------------------------------------------------------------ one pass

def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"linear": _own_linear, "append": _own_append, "attention": _own_attention, "fork": _own_fork, "compact": _own_compact}[kind](state)
    return {"linear": _plain_linear, "append": _plain_append, "attention": _plain_attention, "fork": _plain_fork, "compact": _plain_compact}[kind](state)


def _own_linear(s):
    import paper_2302_01382_b200 as q
    act = {"none": q.ACT_NONE, "relu": q.ACT_RELU, "gelu": q.ACT_GELU_TANH}[s["case"]["act"]]
    return s["ctx"].linear_i8(s["x"], s["w"], s["scale_w"], bias=s["bias"], act=act)


def _own_append(s):
    s["cache"].append(s["k_new"], s["v_new"], s["seqs"], s["starts"])
    return s["cache"].read(s["seqs"], s["first"], s["read_starts"], s["read_tokens"])


def _own_attention(s):
    return s["cache"].attention(s["q"], s["seqs"], s["starts"], max_new=s["max_new"], max_len=s["max_len"], causal=s["case"]["causal"])


def _own_fork(s):
    s["pool"].free(s["children"])
    src, dst = s["pool"].fork(s["parents"], s["children"])
    s["cache"].copy_pages(src, dst)
    return s["k"], s["v"], s["k_absmax"], s["v_absmax"], s["table"], s["lens"], s["refs"], src, dst


def _own_compact(s):
    s["table"].copy_(s["table_was"])
    s["refs"].copy_(s["refs_was"])
    moved = s["pool"].compact()
    s["cache"].copy_pages(None, moved)
    return s["k"], s["v"], s["k_absmax"], s["v_absmax"], s["table"], s["lens"], s["refs"], moved


# ------------------------------------------------------------------------------------ the plain forms

def _divide(a, b):
    """IEEE fp32 division (a division by a Python number may be turned into a product)."""
    a = a if torch.is_tensor(a) else torch.full_like(b, a)
    b = b if torch.is_tensor(b) else torch.full_like(a, b)
    return a / b


def _scale(absmax):
    return torch.where(absmax == 0, torch.ones_like(absmax), _divide(absmax, QMAX))


def _codes(x, absmax):
    inverse = torch.where(absmax == 0, torch.ones_like(absmax), _divide(QMAX, absmax))
    return torch.round(x * inverse).clamp(-QMAX, QMAX)


def _plain_linear(s):
    x = s["x"].float()
    absmax = x.abs().amax(1, keepdim=True)
    codes = _codes(x, absmax)
    # sums of up to k products of 127 * 127 need more than the 24 bits of an fp32 sum
    acc = codes.double() @ s["w"][:, :x.shape[1]].double().T
    y = acc.float() * (_scale(absmax) * s["scale_w"])
    if s["bias"] is not None:
        y = y + s["bias"]
    if s["case"]["act"] == "relu":
        y = y.clamp_min(0)
    elif s["case"]["act"] == "gelu":
        y = 0.5 * y * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y * y * y)))
    return y.to(s["x"].dtype)


def _token_places(s, starts, n_tokens, first):
    """(sequence, position, page, offset) of every token of a ragged batch; `first`: position of each sequence's first."""
    starts = starts.long()
    at = torch.arange(n_tokens, device="cuda")
    entry = torch.searchsorted(starts, at, right=True) - 1
    pos = first.long()[entry] + at - starts[entry]
    page = s["case"]["page"]
    rows = s["seqs"].long()[entry]
    return rows, pos, s["table"].long()[rows, pos // page], pos % page


def _plain_append(s):
    page = s["case"]["page"]
    starts = s["starts"].long()
    lens = s["lens"].long()[s["seqs"].long()]
    first = lens - (starts[1:] - starts[:-1])                      # where the new tokens begin
    rows, pos, pages, offset = _token_places(s, s["starts"], s["tokens"], first)
    # pages that begin among the new tokens forget what they held
    begun = pages[offset == 0]
    # pages that keep earlier tokens
    cut = first[first % page > 0]
    kept = s["table"].long()[s["seqs"].long()[first % page > 0], cut // page]
    earlier = torch.arange(page, device="cuda")[None, :] < (cut % page)[:, None]         # [kept, page]
    for codes, absmax, new in (("k", "k_absmax", "k_new"), ("v", "v_absmax", "v_new")):
        codes, absmax, x = s[codes], s[absmax], s[new].float()
        absmax[begun] = 0
        old = absmax[kept].clone()
        absmax.index_reduce_(0, pages, x.abs().amax(2), "amax")
        ratio = torch.where(old == 0, torch.ones_like(old), _divide(old, absmax[kept]))
        held = codes[kept]
        again = torch.round(held.float() * ratio[:, :, None, None]).to(torch.int8)
        codes[kept] = torch.where(earlier[:, None, :, None], again, held)
        codes[pages, :, offset] = _codes(x, absmax[pages][:, :, None]).to(torch.int8)
    rows, pos, pages, offset = _token_places(s, s["read_starts"], s["read_tokens"], s["first"])
    return tuple(s[c][pages, :, offset].float() * _scale(s[a][pages])[:, :, None] for c, a in (("k", "k_absmax"), ("v", "v_absmax")))


def _plain_attention(s):
    case = s["case"]
    page, heads, dim = case["page"], case["heads"], case["dim"]
    group = case["q_heads"] // heads
    held, fresh = _lengths(case)
    out = torch.empty_like(s["q"])
    at = 0
    for i, (a, b) in enumerate(zip(held, fresh)):
        length = a + b
        pages = s["table"][i, :_pages_of(length, page)].long()
        k = (s["k"][pages].float() * _scale(s["k_absmax"][pages])[:, :, None, None]).transpose(0, 1).reshape(heads, -1, dim)[:, :length]
        v = (s["v"][pages].float() * _scale(s["v_absmax"][pages])[:, :, None, None]).transpose(0, 1).reshape(heads, -1, dim)[:, :length]
        q = s["q"][at:at + b].float().reshape(b, heads, group, dim).permute(1, 2, 0, 3).reshape(heads, group * b, dim)
        scores = (q @ k.transpose(1, 2) / math.sqrt(dim)).reshape(heads, group, b, length)
        if case["causal"]:
            seen = torch.arange(length, device="cuda")[None, :] <= torch.arange(a, length, device="cuda")[:, None]
            scores = scores.masked_fill(~seen, float("-inf"))
        p = torch.exp(scores - scores.amax(3, keepdim=True))
        p = p / p.sum(3, keepdim=True)
        y = p.reshape(heads, group * b, length) @ v
        out[at:at + b] = y.reshape(heads, group, b, dim).permute(2, 0, 1, 3).reshape(b, heads * group, dim).to(out.dtype)
        at += b
    return out


def _plain_copy(s, src, dst):
    for name in ("k", "v", "k_absmax", "v_absmax"):
        s[name][dst] = s[name][src]


def _plain_fork(s):
    page = s["case"]["page"]
    table, lens, refs = s["table"], s["lens"], s["refs"]
    parents, children = s["parents"].long(), s["children"].long()
    # give the children's pages back
    gone = table[children]
    refs.index_add_(0, gone[gone >= 0].long(), torch.full_like(gone[gone >= 0], -1))
    table[children] = -1
    lens[children] = 0
    # full pages are shared, a page in part is copied into the lowest free one
    lengths = lens[parents]
    full = (lengths // page).long()
    shared = torch.arange(table.shape[1], device="cuda")[None, :] < full[:, None]
    rows = torch.where(shared, table[parents], torch.full_like(table[parents], -1))
    refs.index_add_(0, rows[shared].long(), torch.ones_like(rows[shared]))
    part = torch.nonzero(lengths % page)[:, 0]
    free = torch.nonzero(refs == 0)[:part.numel(), 0]
    src = torch.full_like(s["parents"], -1)
    dst = torch.full_like(s["parents"], -1)
    src[part] = table[parents[part], full[part]]
    dst[part] = free.to(torch.int32)
    rows[part, full[part]] = dst[part]
    refs[free] = 1
    table[children] = rows
    lens[children] = lengths
    _plain_copy(s, src[part].long(), dst[part].long())
    return s["k"], s["v"], s["k_absmax"], s["v_absmax"], table, lens, refs, src, dst


def _plain_compact(s):
    s["table"].copy_(s["table_was"])
    s["refs"].copy_(s["refs_was"])
    table, refs = s["table"], s["refs"]
    live = refs > 0
    count = int(live.sum())
    holes = torch.nonzero(~live[:count])[:, 0]
    movers = torch.nonzero(live[count:])[:, 0] + count
    moved = torch.where(live, torch.arange(refs.numel(), device="cuda"), torch.full_like(refs, -1).long())
    moved[movers] = holes
    refs[holes] = refs[movers]
    refs[movers] = 0
    table.copy_(torch.where(table >= 0, moved[table.clamp_min(0).long()].to(torch.int32), table))
    _plain_copy(s, movers, holes)
    return s["k"], s["v"], s["k_absmax"], s["v_absmax"], table, s["lens"], refs, moved.to(torch.int32)


# ------------------------------------------------------------------------------------ in 64 bits

def exact(case, seed):
    s = _inputs(case, seed)
    return {"linear": _exact_linear, "append": _exact_append, "attention": _exact_attention, "fork": _exact_fork, "compact": _exact_compact}[case["kind"]](s)


def _np_codes(x, absmax):
    """Codes of the rule: the scale and the product before the rounding are fp32 values by definition."""
    absmax = absmax.astype(np.float32)
    with np.errstate(divide="ignore"):
        inverse = np.where(absmax == 0, np.float32(1), np.float32(QMAX) / absmax)
    return np.clip(np.rint((x.astype(np.float32) * inverse).astype(np.float32)).astype(np.float64), -QMAX, QMAX)


def _np_scale(absmax):
    absmax = absmax.astype(np.float32)
    return np.where(absmax == 0, np.float32(1), absmax / np.float32(QMAX)).astype(np.float64)


def _exact_linear(s):
    x = s["x"].float().cpu().numpy()
    absmax = np.abs(x).max(axis=1, keepdims=True)
    codes = torch.from_numpy(_np_codes(x, absmax)).cuda()
    weights = s["w"][:, :x.shape[1]].double()
    y = (codes @ weights.T) * torch.from_numpy(_np_scale(absmax)).cuda() * s["scale_w"].double()[None, :]
    if s["bias"] is not None:
        y += s["bias"].double()
    if s["case"]["act"] == "relu":
        y = torch.where(y > 0, y, torch.zeros_like(y))
    elif s["case"]["act"] == "gelu":
        y = y / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3)))
    return y


def _exact_append(s):
    page = s["case"]["page"]
    held, fresh = _lengths(s["case"])
    table = s["table"].cpu().numpy()
    result = []
    for codes, absmax, new in (("k", "k_absmax", "k_new"), ("v", "v_absmax", "v_new")):
        codes, absmax, x = s[codes].cpu().numpy(), s[absmax].cpu().numpy(), s[new].float().cpu().numpy()
        rows, at = [], 0
        for i, (a, b) in enumerate(zip(held, fresh)):
            for j in range(a // page, _pages_of(a + b, page)):
                lo, hi = max(a, j * page), min(a + b, (j + 1) * page)                    # new tokens of this page
                fresh_rows = x[at + lo - a:at + hi - a].transpose(1, 0, 2)               # [heads, tokens, dim]
                top = np.abs(fresh_rows).max(axis=(1, 2))
                number = table[i, j]
                parts = []
                if lo > j * page:
                    was = absmax[number]
                    top = np.maximum(top, was)
                    with np.errstate(invalid="ignore", divide="ignore"):
                        ratio = np.where(was == 0, np.float32(1), was / top).astype(np.float32)
                    parts.append(np.rint(codes[number, :, :lo - j * page].astype(np.float32) * ratio[:, None, None]).astype(np.float64))
                parts.append(_np_codes(fresh_rows, top[:, None, None]))
                rows.append((np.concatenate(parts, 1) * _np_scale(top)[:, None, None]).transpose(1, 0, 2))
            at += b
        result.append(torch.from_numpy(np.concatenate(rows, 0)))
    return tuple(result)


def _exact_attention(s):
    case = s["case"]
    page, heads, dim = case["page"], case["heads"], case["dim"]
    group = case["q_heads"] // heads
    held, fresh = _lengths(case)
    if sum((a + b) * b for a, b in zip(held, fresh)) * case["q_heads"] > 4e9:
        return None
    table = s["table"].cpu()
    out = torch.zeros(s["q"].shape, dtype=torch.float64)
    at = 0
    for i, (a, b) in enumerate(zip(held, fresh)):
        length = a + b
        pages = table[i, :_pages_of(length, page)].long().cuda()
        past = torch.arange(length, device="cuda")[None, :] > torch.arange(a, length, device="cuda")[:, None]
        for h in range(heads):
            scale = [torch.from_numpy(_np_scale(s[n][pages, h].cpu().numpy())).cuda() for n in ("k_absmax", "v_absmax")]
            k, v = [(s[n][pages, h].double() * c[:, None, None]).reshape(-1, dim)[:length] for n, c in zip(("k", "v"), scale)]
            for j in range(h * group, (h + 1) * group):
                scores = s["q"][at:at + b, j].double() @ k.T / math.sqrt(dim)
                if case["causal"]:
                    scores[past] = -math.inf
                out[at:at + b, j] = (torch.softmax(scores, 1) @ v).cpu()
        at += b
    return out


def _exact_fork(s):
    page, n, beams = s["case"]["page"], s["case"]["n"], s["case"]["beams"]
    table, lens, refs = (s[k].cpu().numpy().copy() for k in ("table", "lens", "refs"))
    src, dst = [-1] * (n * beams), [-1] * (n * beams)
    for f, (parent, child) in enumerate(zip(s["parents"].tolist(), s["children"].tolist())):
        full, rest = divmod(int(lens[parent]), page)
        for j in range(full):
            table[child, j] = table[parent, j]
            refs[table[parent, j]] += 1
        if rest:
            src[f] = int(table[parent, full])
        lens[child] = lens[parent]
    free = iter(np.nonzero(refs == 0)[0])
    for f, child in enumerate(s["children"].tolist()):
        if src[f] >= 0:
            dst[f] = int(next(free))
            refs[dst[f]] = 1
            table[child, lens[child] // page] = dst[f]
    moved = [[torch.from_numpy(a) for a in _np_moved(s, [p for p in src if p >= 0], [p for p in dst if p >= 0])]]
    return (*moved[0], *(torch.from_numpy(a) for a in (table, lens, refs)), torch.tensor(src, dtype=torch.int32), torch.tensor(dst, dtype=torch.int32))


def _np_moved(s, src, dst):
    for name in ("k", "v", "k_absmax", "v_absmax"):
        a = s[name].cpu().numpy().copy()
        for p, d in zip(src, dst):
            a[d] = a[p]
        yield a


def _exact_compact(s):
    table, refs = s["table"].cpu().numpy().copy(), s["refs"].cpu().numpy().copy()
    count = sum(1 for r in refs if r > 0)
    moved = np.array([p if r > 0 else -1 for p, r in enumerate(refs)], dtype=np.int32)
    holes = [p for p in range(count) if refs[p] == 0]
    movers = [p for p in range(count, len(refs)) if refs[p] > 0]
    for p, d in zip(movers, holes):
        moved[p], refs[d], refs[p] = d, refs[p], 0
    for row in table:
        for j, p in enumerate(row):
            if p >= 0:
                row[j] = moved[p]
    codes = [torch.from_numpy(a) for a in _np_moved(s, movers, holes)]
    return (*codes, torch.from_numpy(table), s["lens"].cpu(), torch.from_numpy(refs), torch.from_numpy(moved))


# ------------------------------------------------------------------------------------ the work of a pass

def work(case):
    kind = case["kind"]
    if kind == "linear":
        m, k, n, es = case["m"], case["k"], case["n"], BYTES[case["dtype"]]
        return {"bytes": m * k * es + n * k + 4 * n * (2 if case["bias"] else 1) + m * n * es, "flops": 2 * m * k * n}
    held, fresh = _lengths(case)
    page, heads, dim = case["page"], case["heads"], case["dim"]
    per_page = 2 * heads * (page * dim + 4)
    if kind == "append":
        # new values read, codes written, then codes and maxima of the touched pages read and their values written
        es, row = BYTES[case["dtype"]], 2 * heads * dim
        new = sum(fresh)
        read = sum(a + b - a // page * page for a, b in zip(held, fresh))
        pages = sum(_pages_of(a + b, page) - a // page for a, b in zip(held, fresh))
        return {"bytes": new * row * (es + 1) + read * row * (1 + 4) + 3 * pages * 2 * heads * 4, "flops": 3 * new * row + read * row}
    if kind == "attention":
        es = BYTES[case["dtype"]]
        cached = sum(a + b for a, b in zip(held, fresh))
        pairs = sum(a * b + b * (b + 1) // 2 if case["causal"] else (a + b) * b for a, b in zip(held, fresh))
        pages = sum(_pages_of(a + b, page) for a, b in zip(held, fresh))
        io = 2 * sum(fresh) * case["q_heads"] * dim * es
        return {"bytes": 2 * cached * heads * dim + 8 * pages * heads + 4 * pages + io, "flops": 4 * pairs * case["q_heads"] * dim}
    if kind == "fork":
        parts = case["beams"] * sum(1 for a in held if a % page)
        rows = case["beams"] * sum(_pages_of(a, page) for a in held)
        # parts copied; table rows written (and cleared), counts raised and lowered
        return {"bytes": 2 * parts * per_page + 6 * 4 * rows, "flops": 0}
    live = sum(_pages_of(a, page) for i, a in enumerate(held) if i % 2 == 0)
    pages = sum(_pages_of(a, page) for a in held) + 11
    # pages are handed out at random, so that the share of the live ones behind the first `live` is that of all pages
    movers = int(live * (pages - live) / pages)
    entries = case["n"] * (max(_pages_of(a, page) for a in held) + 1)
    return {"bytes": 2 * movers * per_page + 16 * pages + 16 * entries, "flops": 0}
