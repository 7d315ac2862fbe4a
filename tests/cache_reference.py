"""Plain 64-bit reference of the paged key/value cache, and the bound that its attention is held to.

Caches are laid out by numpy code of this file: pages in a shuffled order, slots that were never written filled with whatever the
test asks for."""
import math
from types import SimpleNamespace

import numpy as np
import torch

TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
UNIT = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}     # largest relative error of one rounding to nearest
MOST = {8: 127, 4: 7}


def quantised(x, bits):
    """(codes, scales) of float32 rows x[..., d]: each operation in float32."""
    x = x.astype(np.float32)
    with np.errstate(all="ignore"):
        a = np.max(np.abs(x), axis=-1)
        scale = (a * np.float32(1.0 / MOST[bits])).astype(np.float32)
        stored = a >= np.float32(2.0 ** -100)
        inverse = np.where(stored & np.isfinite(a), np.float32(1) / scale, np.float32(0)).astype(np.float32)
        codes = np.rint((x * inverse[..., None]).astype(np.float32))
        codes = np.clip(codes, -MOST[bits], MOST[bits])
    finite = np.isfinite(a)
    codes = np.where(finite[..., None], codes, 0).astype(np.int64)
    scale = np.where(stored, scale, np.float32(0))
    return codes, np.where(finite, scale, np.float32(np.nan)).astype(np.float32)


def packed(codes, bits):
    if bits == 8:
        return codes.astype(np.int8)
    c = (codes + 8).astype(np.uint8)
    return (c[..., 0::2] | (c[..., 1::2] << 4)).astype(np.uint8)


def unpacked(held, bits):
    if bits == 8:
        return held.astype(np.int64)
    out = np.empty(held.shape[:-1] + (held.shape[-1] * 2,), np.int64)
    out[..., 0::2] = (held & 15).astype(np.int64) - 8
    out[..., 1::2] = (held >> 4).astype(np.int64) - 8
    return out


def make(rng, rows, kv_heads, d, page, bits, io, spare_pages=3, fill=0.0, max_pages=None, spread=1.0, v_spread=1.0):
    """A cache that already holds everything: rows = [(cached, new)]; dense float64 keys and values as stored beside the tensors."""
    lengths = [c + n for c, n in rows]
    pages = [-(-l // page) for l in lengths]
    n_pages = sum(pages) + spare_pages
    most = max(pages + [1]) if max_pages is None else max_pages
    order = rng.permutation(n_pages)
    table = np.full((len(rows), most), -1, np.int32)
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = order[at:at + n]
        at += n
    offsets = np.concatenate([[0], np.cumsum([n for _, n in rows])]).astype(np.int32)
    s = SimpleNamespace(rows=rows, kv_heads=kv_heads, d=d, page=page, bits=bits, io=io, table=table, lengths=np.array(lengths, np.int32),
                        offsets=offsets, total=int(offsets[-1]), n_pages=n_pages, dense={}, pools={}, scales={})
    for name, size in (("k", spread), ("v", v_spread)):
        held = rng.standard_normal((n_pages, kv_heads, page, d)).astype(np.float32) * size
        written = np.zeros((n_pages, page), bool)
        for b, l in enumerate(lengths):
            for p in range(pages[b]):
                written[table[b, p], :min(page, l - p * page)] = True
        if bits == 16:
            t = torch.from_numpy(held).to(TORCH[io])
            t[torch.from_numpy(~written)[:, None, :].expand(-1, kv_heads, -1)] = fill
            s.pools[name], s.scales[name] = t, None
            values = t.double().numpy()
        else:
            codes, scale = quantised(held, bits)
            scale[np.broadcast_to(~written[:, None, :], scale.shape)] = fill
            s.pools[name], s.scales[name] = torch.from_numpy(packed(codes, bits)), torch.from_numpy(scale)
            with np.errstate(invalid="ignore"):
                values = codes.astype(np.float64) * scale.astype(np.float64)[..., None]
        s.dense[name] = [values[table[b, :pages[b]]].transpose(0, 2, 1, 3).reshape(-1, kv_heads, d)[:l] for b, l in enumerate(lengths)]
    return s


def upload(P, s, n_tokens=None):
    """(cache, batch) on the GPU."""
    dev = lambda t: None if t is None else t.cuda()
    cache = P.StiCache(dev(s.pools["k"]), dev(s.pools["v"]), dev(s.scales["k"]), dev(s.scales["v"]))
    batch = P.StiCacheBatch(torch.from_numpy(s.table).cuda(), torch.from_numpy(s.lengths).cuda(), torch.from_numpy(s.offsets).cuda(),
                            s.total if n_tokens is None else n_tokens)
    return cache, batch


def seen_keys(pos, length, window, sinks):
    keys = [j for j in range(max(0, min(pos + 1, length)))]
    if window > 0:
        keys = [j for j in keys if j > pos - window or j < sinks]
    return np.array(keys, np.int64)


def attention(s, q, window=0, sinks=0, scale=None, hide=None):
    """q: float64 [total, heads, d] -> (out float64, bound float64) of the same shape.

    The bound, before any run: one rounding u of the result and one u of each weight, |o| u + u sum_j p_j |v_j|; weights below the
    normal numbers of 16 bits are off by half a step, 2^-25, of the largest value that a weight of 1 can carry; float32 scores, d
    products of relative error 2^-24 each and their sum, move a weight by twice the score's error; float32 sums of n terms."""
    heads, d = q.shape[1], s.d
    group = heads // s.kv_heads
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    out, bound = np.zeros_like(q), np.zeros_like(q)
    u = UNIT[s.io]
    for b in range(len(s.rows)):
        first, end, length = int(s.offsets[b]), int(s.offsets[b + 1]), int(s.lengths[b])
        for r in range(first, end):
            pos = length - (end - r)
            keys = seen_keys(pos, length, window, sinks)
            if hide is not None:
                keys = keys[~hide[b][keys]]
            if not len(keys):
                continue
            for h in range(heads):
                k, v = s.dense["k"][b][keys, h // group], s.dense["v"][b][keys, h // group]
                x = scale * (k @ q[r, h])
                p = np.exp(x - x.max())
                p /= p.sum()
                out[r, h] = p @ v
                mass = p @ np.abs(v)
                score = scale * np.max(np.abs(k) @ np.abs(q[r, h])) * (d + 4) * 2.0 ** -24 + np.abs(x).max() * 2.0 ** -22
                small = len(keys) * 2.0 ** -25 * np.abs(v).max() * p.max()
                bound[r, h] = 1.02 * (u * np.abs(out[r, h]) + u * mass) + (2 * score + (len(keys) + 16) * 2.0 ** -23) * mass + small + 2.0 ** -24
    return out, bound
