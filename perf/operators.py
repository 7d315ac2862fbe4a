"""Cases of the key/value cache and of the attention that reads it, as a program that streams tokens through a model uses them.

Two kinds:

``cache``      new keys and values quantised into a paged cache, and the sequences read back from it
``attention``  the queries of new tokens over the cached keys and values of their sequences: causal, or with a sliding window
               and a few first tokens that stay visible

A case is a dict of plain values.  How long each sequence is follows from the case; keys, values, queries and the order of the pages
are drawn on the GPU from the seed.  Keys have channels with an offset of their own, as trained models have.
"""
from __future__ import annotations

import math
import random

import torch

own = False   # True: the framework's entry points; False: plain torch operations in float32

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
LARGEST = {0: 127, 8: 127, 4: 7}
SMALLEST_ROW = 2.0 ** -100   # rows whose largest magnitude is below this are stored as zeros


def cache(name, **more):
    case = {"name": name, "kind": "cache", "heads": 12, "kv_heads": 12, "d_head": 64, "page": 16, "bits": 8, "io": "f16", "seqs": 1,
            "context": 0, "new": 1, "window": 0, "sinks": 0}
    case.update(more)
    return case


def attention(name, **more):
    return cache(name, **{"kind": "attention", "bits": 16, **more})


def listed():
    return [
        # one token of one short sequence: the smallest write, all launches and host path
        cache("cache_token_4bit", bits=4, context=37),
        # the prompts of a serving batch, quantised as they come in and read back
        cache("cache_prompts_8bit", bits=8, io="bf16", seqs=16, new=384),
        # one token each behind contexts of a few thousand, kept in 16 bits: a cache laid out densely for another program
        cache("cache_tokens_16bit", bits=16, io="bf16", heads=16, kv_heads=16, page=32, seqs=24, context=2000),
        # chunks of long documents in 4 bits, shared key/value heads
        cache("cache_long_4bit", bits=4, heads=32, kv_heads=8, d_head=128, page=64, seqs=4, context=16384, new=512),
        # one token over a short context: the smallest attention, where latency counts
        attention("attend_token_short", context=127),
        # a serving batch generating token by token over an 8-bit cache
        attention("attend_tokens_8bit", bits=8, seqs=32, context=4095),
        # two very long contexts in 4 bits, shared key/value heads
        attention("attend_token_long_4bit", bits=4, io="bf16", heads=32, kv_heads=8, d_head=128, page=64, seqs=2, context=131072),
        # a few tokens at once per sequence (a draft to be checked), many heads per key/value head
        attention("attend_draft_shared_heads", heads=32, kv_heads=4, d_head=128, page=32, seqs=8, context=8192, new=5),
        # chunks of prompts behind what is cached already, ragged
        attention("attend_chunk", io="bf16", heads=16, kv_heads=16, page=32, seqs=4, context=8192, new=512),
        # long prompts over an 8-bit cache: the largest
        attention("attend_prompt_8bit", bits=8, heads=16, kv_heads=4, d_head=128, page=64, seqs=2, context=16384, new=4096),
        # streaming generation: a window of the last thousand tokens and the first four, out of long contexts
        attention("attend_window_tokens", io="bf16", seqs=48, context=16384, window=1024, sinks=4),
        # a long prompt under the same window
        attention("attend_window_prompt", context=0, new=7919, window=512, sinks=4),
    ]


# ---------------------------------------------------------------------------
# More cases of the same ranges
# ---------------------------------------------------------------------------

def log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    while True:
        kind = rng.choice(["cache", "attention", "attention"])
        kv_heads, group = rng.choice([(12, 1), (16, 1), (9, 1), (8, 4), (4, 4), (4, 8), (5, 3), (2, 6)])
        case = {"kind": kind, "heads": kv_heads * group, "kv_heads": kv_heads, "d_head": rng.choice([64, 128]),
                "page": rng.choice([16, 32, 64, 128]), "bits": rng.choice([16, 8, 4]), "io": rng.choice(["f16", "bf16"]),
                "window": 0, "sinks": 0}
        shape = rng.choice(["tokens", "few", "chunk"])
        case["seqs"] = log_int(rng, 1, 48 if shape == "tokens" else 16)
        case["context"] = log_int(rng, 1, 32768)
        case["new"] = {"tokens": 1, "few": log_int(rng, 2, 16), "chunk": log_int(rng, 17, 4096)}[shape]
        if kind == "attention" and rng.random() < 0.35:
            case["window"], case["sinks"] = log_int(rng, 16, 4096), rng.choice([0, 1, 4, 16])
        rows, longest = case["seqs"] * case["new"], case["context"] + case["new"]
        values = case["seqs"] * longest * case["kv_heads"] * case["d_head"]
        # no more than the largest listed case costs: cached values, query-key pairs, products
        if values > 2.5e8 or (kind == "attention" and (rows * case["heads"] * longest > 2.5e9 or
                                                       rows * case["heads"] * longest * case["d_head"] > 3e11)):
            continue
        return case


def sizes(case):
    """[(cached, new)] of each sequence: the first has the full lengths, the others between a quarter of them and all."""
    rng = random.Random(case["seqs"] * 1000003 + case["context"] * 1009 + case["new"])
    got = [(case["context"], case["new"])]
    while len(got) < case["seqs"]:
        got.append((rng.randint(case["context"] // 4, case["context"]), rng.randint((case["new"] + 3) // 4, case["new"])))
    return got


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def codes_of(x, bits):
    """Rows of x quantised: whole numbers (float32) and the scale of each row."""
    most = x.abs().amax(-1, keepdim=True)
    scale = most * (1.0 / LARGEST[bits])
    stored = most >= SMALLEST_ROW
    per_scale = torch.where(stored, torch.reciprocal(scale), torch.zeros_like(scale))
    codes = torch.round(x * per_scale).clamp(-LARGEST[bits], LARGEST[bits])
    scale = torch.where(stored, scale, torch.zeros_like(scale))
    finite = torch.isfinite(most)
    return torch.where(finite, codes, torch.zeros_like(codes)), torch.where(finite, scale, torch.full_like(scale, math.nan))[..., 0]


def stored_of(codes, bits):
    """Whole numbers as the cache holds them: 8 bits each, or two of 4 bits (plus 8) to a byte, the first in its low half."""
    if bits == 8:
        return codes.to(torch.int8)
    c = (codes + 8).to(torch.uint8)
    return c[..., 0::2] | (c[..., 1::2] << 4)


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    rows, page, hkv, d, bits = sizes(case), case["page"], case["kv_heads"], case["d_head"], case["bits"]
    dtype = DTYPES[case["io"]]
    lengths = [c + n for c, n in rows]
    pages = [-(-l // page) for l in lengths]
    n_pages, max_pages = sum(pages) + 8, max(pages)
    order = torch.randperm(n_pages, device=dev, generator=g).to(torch.int32)
    table = torch.full((len(rows), max_pages), -1, dtype=torch.int32, device=dev)
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = order[at:at + n]
        at += n
    offsets = [0]
    for _, n in rows:
        offsets.append(offsets[-1] + n)
    total = offsets[-1]

    def normal(*shape):
        return torch.randn(shape, device=dev, generator=g)

    # what sets one head and one channel apart from the next
    channel = {"k": 1.5 * normal(hkv, 1, d) * (torch.rand(hkv, 1, d, device=dev, generator=g) < 0.1), "v": 0.2 * normal(hkv, 1, d)}
    spread = {"k": 1.0, "v": 0.7}
    state = {"case": dict(case), "table": table, "lengths": torch.tensor(lengths, dtype=torch.int32, device=dev),
             "offsets": torch.tensor(offsets, dtype=torch.int32, device=dev), "total": total, "longest": max(lengths),
             "most_new": max(n for _, n in rows), "keep": {}}
    for name in ("k", "v"):
        pool = normal(n_pages, hkv, page, d).mul_(spread[name]).add_(channel[name])
        if bits == 16:
            state[name] = pool.to(dtype)
            state[name + "_scale"] = None
        else:
            codes, scale = codes_of(pool, bits)
            state[name], state[name + "_scale"] = stored_of(codes, bits), scale.contiguous()
        del pool
        if case["kind"] == "cache":
            state["new_" + name] = (normal(total, hkv, d) * spread[name] + channel[name][:, 0]).to(dtype)
    if case["kind"] == "attention":
        state["q"] = (1.5 * normal(total, case["heads"], d)).to(dtype)
    return state


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def run(state):
    case = state["case"]
    if own:
        return run_own(state)
    return plain_cache(state) if case["kind"] == "cache" else plain_attention(state)


def run_own(state):
    import paper_2207_05022_amd as sti
    case, keep = state["case"], state["keep"]
    if not keep:   # handles and scratch memory, which a program keeps beside its cache
        keep["cache"] = sti.StiCache(state["k"], state["v"], state["k_scale"], state["v_scale"])
        keep["batch"] = sti.StiCacheBatch(state["table"], state["lengths"], state["offsets"], state["total"])
        if case["kind"] == "attention":
            need = sti.sti_cache_attention_workspace_bytes(keep["cache"], keep["batch"], case["heads"], case["window"], case["sinks"])
            keep["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    if case["kind"] == "cache":
        sti.sti_cache_append(keep["cache"], keep["batch"], state["new_k"], state["new_v"])
        shape = (case["seqs"], state["longest"], case["kv_heads"], case["d_head"])
        k = torch.empty(shape, dtype=DTYPES[case["io"]], device="cuda")
        v = torch.empty(shape, dtype=DTYPES[case["io"]], device="cuda")
        sti.sti_cache_read(keep["cache"], keep["batch"], 0, k, v)
        return {"k": k, "v": v}
    out = torch.empty_like(state["q"])
    sti.sti_cache_attention(keep["cache"], keep["batch"], state["q"], out, keep["workspace"], window=case["window"], sinks=case["sinks"])
    return out


def plain_rows(state):
    """For each row of new tokens its sequence, its number there, and its position."""
    offsets, total = state["offsets"].long(), state["total"]
    row = torch.arange(total, device=offsets.device)
    seq = torch.searchsorted(offsets[1:], row, right=True)
    number = row - offsets[seq]
    position = state["lengths"].long()[seq] - (offsets[seq + 1] - offsets[seq]) + number
    return seq, number, position


def plain_read(state, name):
    """[seqs, longest, kv_heads, d_head] in float32, zeros behind a sequence's end."""
    case = state["case"]
    position = torch.arange(state["longest"], device=state["table"].device)
    there = position[None, :] < state["lengths"][:, None]
    page = state["table"].long()[:, position // case["page"]].clamp(min=0)
    slot = (position % case["page"])[None, :].expand_as(page)
    held = state[name][page, :, slot]
    if case["bits"] == 4:
        held = torch.stack((held & 15, held >> 4), -1).flatten(-2).float() - 8
    held = held.float()
    if case["bits"] < 16:
        held = held * state[name + "_scale"][page, :, slot][..., None]
    return torch.where(there[:, :, None, None], held, torch.zeros_like(held))


def plain_cache(state):
    case = state["case"]
    seq, _, position = plain_rows(state)
    page, slot = state["table"].long()[seq, position // case["page"]], position % case["page"]
    out = {}
    for name in ("k", "v"):
        x = state["new_" + name].float()
        if case["bits"] == 16:
            state[name][page, :, slot] = x.to(state[name].dtype)
        else:
            codes, scale = codes_of(x, case["bits"])
            state[name][page, :, slot] = stored_of(codes, case["bits"])
            state[name + "_scale"][page, :, slot] = scale
        out[name] = plain_read(state, name).to(DTYPES[case["io"]])
    return out


def plain_attention(state):
    case = state["case"]
    hkv, d, group = case["kv_heads"], case["d_head"], case["heads"] // case["kv_heads"]
    k = plain_read(state, "k").permute(0, 2, 3, 1).contiguous()   # [seqs, kv_heads, d, longest]
    v = plain_read(state, "v").permute(0, 2, 1, 3).contiguous()   # [seqs, kv_heads, longest, d]
    seq, number, position = plain_rows(state)
    most = state["most_new"]
    q = torch.zeros(case["seqs"], most, case["heads"], d, device=k.device)
    q[seq, number] = state["q"].float()
    q = q.view(case["seqs"], most, hkv, group, d).permute(0, 2, 1, 3, 4).reshape(case["seqs"], hkv, most * group, d)
    at = torch.full((case["seqs"], most), -1, device=k.device)
    at[seq, number] = position
    key = torch.arange(state["longest"], device=k.device)
    seen = key <= at[:, :, None]
    if case["window"]:
        seen &= (key > at[:, :, None] - case["window"]) | (key < case["sinks"])
    scores = torch.matmul(q, k).mul_(1.0 / math.sqrt(d)).view(case["seqs"], hkv, most, group, -1)
    scores.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    top = scores.amax(-1, keepdim=True)
    weight = scores.sub_(torch.where(torch.isinf(top), torch.zeros_like(top), top)).exp_()
    total = weight.sum(-1, keepdim=True)
    o = torch.matmul(weight.view(case["seqs"], hkv, most * group, -1), v).view(case["seqs"], hkv, most, group, d)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    o = o.permute(0, 2, 1, 3, 4).reshape(case["seqs"], most, case["heads"], d)
    return o[seq, number].to(DTYPES[case["io"]])


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    rows = sizes(case)
    d, hkv, heads = case["d_head"], case["kv_heads"], case["heads"]
    held = d * case["bits"] / 8 + (4 if case["bits"] < 16 else 0)   # bytes of one cached row of one head
    new = sum(n for _, n in rows)
    if case["kind"] == "cache":
        longest = max(c + n for c, n in rows)
        moved = 2 * new * hkv * (2 * d + held) + 2 * sum(c for c, _ in rows) * hkv * held + 2 * case["seqs"] * longest * hkv * d * 2
        return {"bytes": moved, "flops": 4.0 * hkv * d * sum(c + n for c, n in rows)}
    pairs = read = 0
    window, sinks = case["window"], case["sinks"]
    for c, n in rows:
        if not window:
            pairs += n * c + n * (n + 1) // 2
            read += c + n
        else:
            for p in range(c, c + n):
                first = max(0, p - window + 1)
                pairs += p + 1 - first + min(sinks, first)
            first = max(0, c - window + 1)
            read += c + n - first + min(sinks, first)
    return {"bytes": 2 * read * hkv * held + 2 * new * heads * d * 2, "flops": 4.0 * d * heads * pairs}


# ---------------------------------------------------------------------------
# The definition in 64 bits, sequence by sequence and head by head
# ---------------------------------------------------------------------------

def exact_row_values(state, name, b, head):
    """What the cache holds for every position of sequence b, in float64 [length, d_head]."""
    case, page = state["case"], state["case"]["page"]
    length = int(state["lengths"][b])
    pages = state["table"][b, :-(-length // page)].long()
    x = state[name][pages, head].reshape(len(pages) * page, -1)[:length]
    if case["bits"] == 4:
        both = x.to(torch.int32)
        values = torch.empty(length, case["d_head"], dtype=torch.float64, device=x.device)
        values[:, 0::2] = (both % 16 - 8).double()
        values[:, 1::2] = (torch.div(both, 16, rounding_mode="floor") - 8).double()
    else:
        values = x.double()
    if case["bits"] < 16:
        values *= state[name + "_scale"][pages, head].reshape(-1)[:length].double()[:, None]
    return values


def exact(case, seed):
    state = prepare(case, seed)
    offsets = [int(x) for x in state["offsets"]]
    heads, hkv, d = case["heads"], case["kv_heads"], case["d_head"]
    if case["kind"] == "cache":
        out = {}
        for name in ("k", "v"):
            dense = torch.zeros(case["seqs"], state["longest"], hkv, d, dtype=torch.float64, device="cuda")
            for b in range(case["seqs"]):
                x = state["new_" + name][offsets[b]:offsets[b + 1]].double()
                if case["bits"] < 16:
                    step = x.abs().max(dim=2, keepdim=True).values / LARGEST[case["bits"]]
                    x = torch.where(step > 0, torch.round(x / step) * step, 0.0)
                length = int(state["lengths"][b])
                for head in range(hkv):
                    dense[b, :length, head] = exact_row_values(state, name, b, head)
                dense[b, length - len(x):length] = x
            out[name] = dense
        return out
    out = torch.zeros(state["total"], heads, d, dtype=torch.float64, device="cuda")
    for b in range(case["seqs"]):
        new, length = offsets[b + 1] - offsets[b], int(state["lengths"][b])
        key = torch.arange(length, device="cuda")
        at = torch.arange(length - new, length, device="cuda")[:, None]
        hidden = key > at
        if case["window"]:
            hidden = hidden | ((key <= at - case["window"]) & (key >= case["sinks"]))
        for kv in range(hkv):
            k, v = (exact_row_values(state, name, b, kv) for name in ("k", "v"))
            kt = k.t().contiguous()
            for head in range(kv * (heads // hkv), (kv + 1) * (heads // hkv)):
                s = state["q"][offsets[b]:offsets[b + 1], head].double() @ kt / math.sqrt(d)
                s[hidden] = -math.inf
                s = torch.softmax(s, dim=1)
                out[offsets[b]:offsets[b + 1], head] = s @ v
    return out
