"""Refusals of the paged key/value cache: every bad argument is answered with its status before anything is launched."""
import ctypes as C
import math

import pytest

P = None   # the package, loaded by the first test: a library loaded before torch would bring another HIP runtime into runs of the GPU tests


@pytest.fixture(scope="module", autouse=True)
def load():
    global P
    import torch  # noqa: F401
    import paper_2207_05022_amd
    P = paper_2207_05022_amd


FAKE = 0x10000   # aligned, never dereferenced


def cache(**more):
    f = dict(n_kv_heads=4, d_head=64, bits=8, page_tokens=16, n_pages=10, dtype=1, k=FAKE, v=FAKE, k_scale=FAKE, v_scale=FAKE)
    f.update(more)
    return P.StiCacheStruct(*[f[n] for n, _ in P.StiCacheStruct._fields_])


def batch(**more):
    f = dict(n_seqs=2, n_tokens=3, max_pages=5, page_table=FAKE, lengths=FAKE, offsets=FAKE)
    f.update(more)
    return P.StiCacheBatchStruct(*[f[n] for n, _ in P.StiCacheBatchStruct._fields_])


def append(c=None, b=None, k=FAKE, v=FAKE, io=1, ks=256, vs=256):
    return P.lib.sti_cache_append(c and C.byref(c), b and C.byref(b), k, v, io, ks, vs, None)


def read(c=None, b=None, first=0, count=4, k=FAKE, v=FAKE, out=1):
    return P.lib.sti_cache_read(c and C.byref(c), b and C.byref(b), first, count, k, v, out, None)


def attend(c=None, b=None, q=FAKE, out=FAKE, io=1, qs=512, os=512, heads=8, scale=0.0, window=0, sinks=0, ws=None, ws_bytes=0):
    return P.lib.sti_cache_attention(c and C.byref(c), b and C.byref(b), q, out, io, qs, os, heads, scale, window, sinks, ws, ws_bytes, None)


NULL, DIMS, BITS, ALIGN, WORKSPACE, DTYPE, UNSUPPORTED = 1, 2, 3, 5, 6, 7, 9

BAD_CACHES = [
    (dict(bits=5), BITS), (dict(bits=0), BITS), (dict(bits=32), BITS),
    (dict(n_kv_heads=0), DIMS), (dict(n_kv_heads=65), DIMS), (dict(n_kv_heads=-1), DIMS),
    (dict(d_head=32), DIMS), (dict(d_head=96), DIMS), (dict(page_tokens=8), DIMS), (dict(page_tokens=24), DIMS),
    (dict(page_tokens=2048), DIMS), (dict(page_tokens=0), DIMS), (dict(n_pages=-1), DIMS), (dict(n_pages=1 << 26), DIMS),
    (dict(bits=16, dtype=0), DTYPE), (dict(bits=16, dtype=9), DTYPE),
    (dict(k=None), NULL), (dict(v=None), NULL), (dict(k_scale=None), NULL), (dict(bits=4, v_scale=None), NULL),
    (dict(k=FAKE + 8), ALIGN), (dict(v=FAKE + 4), ALIGN), (dict(k_scale=FAKE + 2), ALIGN), (dict(v_scale=FAKE + 1), ALIGN),
]
BAD_BATCHES = [
    (dict(n_seqs=-1), DIMS), (dict(n_tokens=-1), DIMS), (dict(max_pages=-1), DIMS), (dict(n_tokens=(1 << 24) + 1), DIMS),
    (dict(max_pages=(1 << 26) + 1), DIMS), (dict(lengths=None), NULL), (dict(page_table=None), NULL),
    (dict(lengths=FAKE + 2), ALIGN), (dict(page_table=FAKE + 1), ALIGN),
]


@pytest.mark.parametrize("more,status", BAD_CACHES)
def test_caches(more, status):
    for call in (append, read, attend):
        assert call(cache(**more), batch()) == status, call
    if status in (BITS, DIMS, DTYPE):
        c = cache(**more)
        assert P.lib.sti_cache_attention_workspace_bytes(C.byref(c), C.byref(batch(max_pages=5000)), 8, 0, 0) == 0


@pytest.mark.parametrize("more,status", BAD_BATCHES)
def test_batches(more, status):
    for call in (append, read, attend):
        assert call(cache(), batch(**more)) == status, call


def test_offsets_are_needed_for_rows_only():
    for bad, status in ((None, NULL), (FAKE + 2, ALIGN)):
        assert append(cache(), batch(offsets=bad)) == status
        assert attend(cache(), batch(offsets=bad)) == status
    assert read(cache(), batch(offsets=None), k=None) == NULL      # (the outputs': offsets are not looked at)


def test_null_structs():
    for call in (append, read, attend):
        assert call(None, batch()) == NULL and call(cache(), None) == NULL
    assert P.lib.sti_cache_attention_workspace_bytes(None, None, 8, 0, 0) == 0


def test_append_rows():
    c, b = cache(), batch()
    assert append(c, b, k=None) == NULL and append(c, b, v=None) == NULL
    assert append(c, b, ks=255) == DIMS and append(c, b, vs=0) == DIMS and append(c, b, ks=-256) == DIMS
    assert append(c, b, ks=260) == ALIGN and append(c, b, vs=257) == ALIGN and append(c, b, k=FAKE + 2) == ALIGN
    assert append(c, b, io=0, ks=258) == ALIGN
    assert append(c, b, io=3) == DTYPE and append(c, b, io=-1) == DTYPE


def test_read_ranges():
    c, b = cache(), batch()
    assert read(c, b, first=-1) == DIMS and read(c, b, count=-1) == DIMS and read(c, b, first=1 << 30, count=1) == DIMS
    assert read(c, b, k=None) == NULL and read(c, b, v=None) == NULL
    assert read(c, b, k=FAKE + 8) == ALIGN and read(c, b, v=FAKE + 2) == ALIGN and read(c, b, out=5) == DTYPE


def test_attention_arguments():
    c, b = cache(), batch()
    assert attend(c, b, q=None) == NULL and attend(c, b, out=None) == NULL
    assert attend(c, b, heads=0) == DIMS and attend(c, b, heads=6) == DIMS and attend(c, b, heads=516) == DIMS
    assert attend(c, b, qs=511) == DIMS and attend(c, b, os=0) == DIMS
    assert attend(c, b, qs=516) == ALIGN and attend(c, b, os=514) == ALIGN and attend(c, b, q=FAKE + 4) == ALIGN
    assert attend(c, b, io=0) == DTYPE and attend(c, b, io=7) == DTYPE
    assert attend(cache(bits=16, dtype=2), b, io=1) == UNSUPPORTED
    assert attend(c, b, window=-1) == DIMS and attend(c, b, sinks=-1) == DIMS
    for scale in (-1.0, math.inf, math.nan, 3.4e38):
        assert attend(c, b, scale=scale) == DIMS


def test_workspace():
    c, b = cache(), batch(n_seqs=1, n_tokens=1, max_pages=5000)
    need = P.lib.sti_cache_attention_workspace_bytes(C.byref(c), C.byref(b), 8, 0, 0)
    assert need > 0
    assert attend(c, b) == WORKSPACE and attend(c, b, ws=FAKE, ws_bytes=need - 1) == WORKSPACE
    assert attend(c, b, ws=FAKE + 8, ws_bytes=need) == ALIGN
    # a window of few keys needs none
    assert P.lib.sti_cache_attention_workspace_bytes(C.byref(c), C.byref(b), 8, 64, 4) == 0
    for heads, window, sinks in ((7, 0, 0), (8, -1, 0), (8, 0, -1)):
        assert P.lib.sti_cache_attention_workspace_bytes(C.byref(c), C.byref(b), heads, window, sinks) == 0


def test_nothing_to_do():
    """No sequences, no tokens, no positions: done, whatever the pointers."""
    empty = dict(page_table=None, lengths=None, offsets=None)
    for more in (dict(n_seqs=0), dict(n_tokens=0)):
        b = batch(**more, **empty)
        assert append(cache(), b, k=None, v=None, ks=0, vs=0) == 0
        assert attend(cache(), b, q=None, out=None, qs=0, os=0) == 0
    assert read(cache(), batch(n_seqs=0, **empty), k=None, v=None) == 0
    assert read(cache(), batch(**empty), count=0, k=None, v=None) == 0


def test_python_checks():
    import torch
    half = lambda *s: torch.zeros(*s, dtype=torch.float16)
    with pytest.raises(ValueError):
        P.StiCache(torch.zeros(2, 1, 16, 64), torch.zeros(2, 1, 16, 64))
    with pytest.raises(ValueError):
        P.StiCache(half(2, 1, 16, 64), half(2, 1, 32, 64))
    with pytest.raises(ValueError):
        P.StiCache(half(2, 1, 64, 16).transpose(2, 3), half(2, 1, 64, 16).transpose(2, 3))
    codes = torch.zeros(2, 1, 16, 32, dtype=torch.uint8)
    with pytest.raises(ValueError):
        P.StiCache(codes, codes)
    scales = torch.zeros(2, 1, 16)
    c = P.StiCache(codes, codes, scales, scales)
    assert (c.bits, c.d_head, c.page_tokens, c.n_pages) == (4, 64, 16, 2)
    ints = lambda *v: torch.tensor(v, dtype=torch.int32)
    with pytest.raises(ValueError):
        P.StiCacheBatch(ints(0, 1).view(1, 2), ints(3).long(), ints(0, 1), 1)
    with pytest.raises(ValueError):
        P.StiCacheBatch(ints(0, 1).view(1, 2), ints(3), ints(0, 1, 2), 1)
    b = P.StiCacheBatch(ints(0, 1).view(1, 2), ints(3), ints(0, 1), 1)
    with pytest.raises(ValueError):
        P.sti_cache_append(c, b, half(2, 1, 64), half(2, 1, 64))
    with pytest.raises(ValueError):
        P.sti_cache_append(c, b, half(1, 1, 64), torch.zeros(1, 1, 64))
    with pytest.raises(ValueError):
        P.sti_cache_attention(c, b, half(1, 64, 2).transpose(1, 2), half(1, 2, 64))
    with pytest.raises(ValueError):
        P.sti_cache_read(c, b, 0, half(1, 4, 1, 128), half(1, 4, 1, 128))


def test_tensors_of_the_host_are_refused():
    import torch
    half = lambda *s: torch.zeros(*s, dtype=torch.float16)
    ints = lambda *v: torch.tensor(v, dtype=torch.int32)
    c, b = P.StiCache(half(2, 1, 16, 64), half(2, 1, 16, 64)), P.StiCacheBatch(ints(0, 1).view(1, 2), ints(3), ints(0, 1), 1)
    row, back = half(1, 1, 64), half(1, 4, 1, 64)
    for call in (lambda: P.sti_cache_append(c, b, row, row), lambda: P.sti_cache_read(c, b, 0, back, back),
                 lambda: P.sti_cache_attention(c, b, row, row)):
        with pytest.raises(ValueError, match="CUDA"):
            call()
