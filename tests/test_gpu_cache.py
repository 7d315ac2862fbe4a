"""GPU tests of the paged key/value cache: writing and reading back bit for bit, attention against a plain 64-bit form."""
import numpy as np
import pytest

import cache_reference as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    import paper_2207_05022_amd as P
    assert torch.cuda.is_available(), "needs a GPU"
    return torch, P


def queries(torch, rng, s, heads, amp=1.0):
    q = torch.from_numpy((rng.standard_normal((s.total, heads, s.d)) * amp).astype(np.float32)).to(R.TORCH[s.io])
    return q, q.double().numpy()


def attend(torch, P, s, q, heads, window=0, sinks=0, scale=0.0, on=None, n_tokens=None):
    cache, batch = on or R.upload(P, s, n_tokens)
    need = P.sti_cache_attention_workspace_bytes(cache, batch, heads, window, sinks)
    # a workspace of NaN: nothing may be read that this call has not written
    ws = torch.full((need // 4,), float("nan"), device="cuda").view(torch.uint8) if need else None
    out = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda")
    P.sti_cache_attention(cache, batch, q.cuda(), out, ws, scale=scale, window=window, sinks=sinks)
    torch.cuda.synchronize()
    return out.cpu()


def check(got, want, bound):
    got = got.double().numpy()
    assert got.shape == want.shape
    off = np.abs(got - want)
    assert np.isfinite(got).all() and (off <= bound).all(), (np.max(off - bound), np.argwhere(~(off <= bound))[:4])


# ---------------------------------------------------------------------------
# Writing and reading back
# ---------------------------------------------------------------------------

def written(s, name, x, drop=()):
    """The pools after x [total, kv_heads, d] (float32) has been written, from copies of those before."""
    pool = s.pools[name].clone()
    scale = None if s.bits == 16 else s.scales[name].clone()
    import torch
    for b in range(len(s.rows)):
        first, end, length = int(s.offsets[b]), int(s.offsets[b + 1]), int(s.lengths[b])
        for r in range(first, end):
            pos = length - (end - r)
            if pos < 0 or pos >= s.table.shape[1] * s.page:
                continue
            page, slot = int(s.table[b, pos // s.page]), pos % s.page
            if not 0 <= page < s.n_pages:
                continue
            if s.bits == 16:
                pool[page, :, slot] = torch.from_numpy(x[r]).to(pool.dtype)
            else:
                codes, sc = R.quantised(x[r], s.bits)
                pool[page, :, slot] = torch.from_numpy(R.packed(codes, s.bits))
                scale[page, :, slot] = torch.from_numpy(sc)
    return pool, scale


def same(torch, a, b):
    """Equal bits, any NaN equal to any."""
    if a.dtype.is_floating_point:
        return bool(((a == b) | (a.isnan() & b.isnan())).all())
    return torch.equal(a, b)


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("source", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("d,kv_heads,page,rows", [
    (64, 12, 16, [(37, 1)]),
    (64, 1, 16, [(0, 1), (15, 1), (16, 1), (0, 0), (5, 33)]),
    (64, 5, 64, [(63, 2), (0, 65), (200, 7)]),
    (128, 8, 32, [(31, 1), (0, 17), (64, 64)]),
    (128, 3, 1024, [(1000, 30), (0, 1)]),
])
def test_append_leaves_the_bits_of_the_formula(gpu, bits, source, d, kv_heads, page, rows):
    torch, P = gpu
    rng = np.random.default_rng(bits * 1000 + d + page)
    io = "bf16" if page == 32 else "f16"
    s = R.make(rng, rows, kv_heads, d, page, bits, io)
    x = {}
    for name in "kv":
        v = rng.standard_normal((s.total, kv_heads, d)).astype(np.float32) * np.exp(rng.uniform(-6, 6, (s.total, kv_heads, 1)))
        x[name] = torch.from_numpy(v.astype(np.float32)).to(R.TORCH[source])
    x["k"][0, 0] = 0.0                    # a row of zeros
    x["v"][-1, -1, 3] = float("inf")      # and one that is not finite
    x["k"][-1, 0, d - 1] = float("nan")
    if source == "f32":
        x["v"][0, 0] = 1e-33              # below what a scale can carry
    cache, batch = R.upload(P, s)
    P.sti_cache_append(cache, batch, x["k"].cuda(), x["v"].cuda())
    torch.cuda.synchronize()
    for name in "kv":
        pool, scale = written(s, name, x[name].float().numpy())
        assert same(torch, getattr(cache, name).cpu(), pool)
        if bits < 16:
            assert same(torch, getattr(cache, name + "_scale").cpu(), scale)


@pytest.mark.parametrize("bits", [8, 4])
def test_halves_round_to_even_codes(gpu, bits):
    """Values halfway between two codes, and the largest of a row."""
    torch, P = gpu
    rng = np.random.default_rng(3)
    s = R.make(rng, [(0, 4)], 1, 64, 16, bits, "f16")
    most = R.MOST[bits]
    v = np.tile((np.arange(64) % (2 * most + 1) - most + 0.5).astype(np.float32), (4, 1, 1))
    v[:, :, 0] = most
    v[1] *= 2.0 ** -9
    v[2] *= -2.0 ** 5
    v[3] *= np.float32(0.3)
    cache, batch = R.upload(P, s)
    t = torch.from_numpy(v).cuda()
    P.sti_cache_append(cache, batch, t, t)
    pool, scale = written(s, "k", v)
    assert torch.equal(cache.k.cpu(), pool) and torch.equal(cache.k_scale.cpu(), scale)


@pytest.mark.parametrize("bits,d,source", [(16, 64, "bf16"), (8, 64, "f16"), (4, 128, "f32")])
def test_append_takes_slices_of_a_projection(gpu, bits, d, source):
    """Keys and values as columns of one [tokens, 3 heads d] output."""
    torch, P = gpu
    rng = np.random.default_rng(4)
    heads = 6
    s = R.make(rng, [(10, 5), (0, 9)], heads, d, 16, bits, "f16")
    fused = torch.from_numpy(rng.standard_normal((s.total, 3, heads, d)).astype(np.float32)).to(R.TORCH[source])
    cache, batch = R.upload(P, s)
    dev = fused.cuda()
    P.sti_cache_append(cache, batch, dev[:, 1], dev[:, 2])
    for i, name in ((1, "k"), (2, "v")):
        pool, scale = written(s, name, fused[:, i].float().numpy())
        assert torch.equal(getattr(cache, name).cpu(), pool)
        if bits < 16:
            assert torch.equal(getattr(cache, name + "_scale").cpu(), scale)


def test_append_leaves_out_what_has_no_slot(gpu):
    """Positions below zero and behind the table, pages that the table does not name, rows of no sequence, more than 64 sequences."""
    torch, P = gpu
    rng = np.random.default_rng(5)
    rows = [(3, 2)] * 70
    s = R.make(rng, rows, 2, 64, 16, 8, "f16", max_pages=2)
    s.lengths[1] = 1          # two new tokens, a length of one: the first lies below zero
    s.lengths[2] = 33         # behind both pages
    s.lengths[3] = -5
    s.table[4, 0] = s.n_pages
    s.table[5, 0] = -7
    s.offsets[0] = 1          # row 0 belongs to nobody
    s.offsets[70] = s.total - 1
    x = rng.standard_normal((s.total, 2, 64)).astype(np.float32)
    cache, batch = R.upload(P, s)
    t = torch.from_numpy(x).cuda()
    P.sti_cache_append(cache, batch, t, t)
    lengths = s.lengths.copy()
    s.lengths[3] = 0
    pool, scale = written(s, "k", x)
    s.lengths = lengths
    assert torch.equal(cache.k.cpu(), pool) and same(torch, cache.k_scale.cpu(), scale)


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("out", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("d,kv_heads,page,rows,first,count", [
    (64, 12, 16, [(37, 1)], 0, 38),
    (64, 3, 16, [(0, 0), (1, 0), (15, 2), (100, 1)], 5, 61),     # from the middle of a page, past every end
    (128, 7, 64, [(63, 2), (0, 129)], 64, 1),
    (128, 1, 32, [(200, 0)], 0, 500),                            # past the table
])
def test_read_gives_codes_times_scales(gpu, bits, out, d, kv_heads, page, rows, first, count):
    torch, P = gpu
    rng = np.random.default_rng(bits + d + count)
    s = R.make(rng, rows, kv_heads, d, page, bits, "bf16" if d == 128 else "f16", fill=float("nan"))
    if len(rows) == 2:
        s.table[1, 1] = -1    # a page that is not there: zeros
    cache, batch = R.upload(P, s)
    got = [torch.full((len(rows), count, kv_heads, d), float("nan"), dtype=R.TORCH[out], device="cuda") for _ in "kv"]
    P.sti_cache_read(cache, P.StiCacheBatch(batch.page_table, batch.lengths, None, 0), first, *got)
    torch.cuda.synchronize()
    for name, g in zip("kv", got):
        want = torch.zeros(len(rows), count, kv_heads, d)
        for b in range(len(rows)):
            dense = s.dense[name][b].astype(np.float32)     # a code times a scale: one float32 product is the rounded exact one
            for j in range(count):
                if first + j < len(dense) and 0 <= s.table[b, (first + j) // page]:
                    want[b, j] = torch.from_numpy(dense[first + j])
        assert torch.equal(g.cpu(), want.to(R.TORCH[out]))


# ---------------------------------------------------------------------------
# Attention
# ---------------------------------------------------------------------------

SHAPES = [
    # bits, io, d, heads, kv_heads, page, rows, window, sinks
    (16, "f16", 64, 1, 1, 16, [(0, 1)], 0, 0),
    (16, "f16", 64, 12, 12, 16, [(127, 1)], 0, 0),
    (16, "bf16", 64, 12, 12, 16, [(63, 1), (64, 1), (0, 1), (0, 0), (300, 1)], 0, 0),
    (8, "f16", 64, 12, 12, 32, [(1000, 1), (17, 1), (31, 1)], 0, 0),
    (4, "bf16", 128, 16, 4, 64, [(700, 1), (1, 1)], 0, 0),
    (4, "f16", 64, 9, 9, 16, [(33, 1)] * 7, 0, 0),
    (8, "bf16", 128, 6, 2, 128, [(130, 2), (0, 3), (40, 1)], 0, 0),
    (16, "f16", 128, 32, 4, 32, [(400, 5), (3, 5)], 0, 0),
    (16, "bf16", 128, 15, 5, 16, [(100, 9)], 0, 0),
    (4, "f16", 128, 12, 2, 16, [(65, 11), (0, 2)], 0, 0),
    # chunks: around tiles of queries and of keys
    (16, "f16", 64, 2, 2, 16, [(0, 129), (31, 64), (1, 1), (0, 0), (95, 33)], 0, 0),
    (16, "bf16", 128, 4, 1, 16, [(77, 150), (0, 31)], 0, 0),
    (8, "f16", 64, 3, 3, 64, [(200, 130), (0, 65)], 0, 0),
    (8, "bf16", 128, 8, 2, 32, [(33, 127)], 0, 0),
    (4, "f16", 128, 2, 1, 16, [(150, 255), (64, 1)], 0, 0),
    (4, "bf16", 64, 6, 2, 256, [(300, 97)], 0, 0),
    # windows, with and without first tokens
    (16, "f16", 64, 4, 4, 16, [(500, 1), (3, 1), (20, 1)], 17, 4),
    (16, "bf16", 128, 4, 2, 16, [(333, 70), (0, 200)], 33, 5),
    (8, "f16", 64, 2, 2, 16, [(90, 140)], 1, 0),
    (8, "bf16", 64, 2, 1, 32, [(100, 130)], 64, 100),        # more first tokens than the window leaves out
    (4, "f16", 64, 4, 4, 16, [(250, 3), (250, 40)], 128, 1),
    (4, "f16", 128, 2, 2, 64, [(50, 160)], 1000000, 3),      # wider than the sequence
]


@pytest.mark.parametrize("bits,io,d,heads,kv_heads,page,rows,window,sinks", SHAPES)
def test_attention_against_64_bits(gpu, bits, io, d, heads, kv_heads, page, rows, window, sinks):
    torch, P = gpu
    rng = np.random.default_rng(len(rows) * 7919 + bits + d + heads + window)
    # slots that nothing was written to hold NaN
    s = R.make(rng, rows, kv_heads, d, page, bits, io, fill=float("nan"))
    q, exact_q = queries(torch, rng, s, heads, 2.0)
    want, bound = R.attention(s, exact_q, window, sinks)
    check(attend(torch, P, s, q, heads, window, sinks), want, bound)


@pytest.mark.parametrize("bits,new", [(16, 1), (8, 1), (4, 3), (16, 80), (8, 80), (4, 200)])
def test_long_tables_of_short_sequences(gpu, bits, new):
    """Room for 20000 tokens, a few hundred there: parts of the split find nothing to do."""
    torch, P = gpu
    rng = np.random.default_rng(bits + new)
    s = R.make(rng, [(300, new), (0, new), (5, 0)], 2, 64, 16, bits, "f16", max_pages=1250)
    q, exact_q = queries(torch, rng, s, 4)
    check(attend(torch, P, s, q, 4), *R.attention(s, exact_q))


@pytest.mark.parametrize("new,io", [(1, "f16"), (1, "bf16"), (40, "f16")])
def test_long_contexts(gpu, new, io):
    torch, P = gpu
    rng = np.random.default_rng(new)
    for bits in (16, 8, 4):
        s = R.make(rng, [(5000, new)], 1, 64, 64, bits, io)
        q, exact_q = queries(torch, rng, s, 1, 3.0)
        check(attend(torch, P, s, q, 1), *R.attention(s, exact_q))


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("new", [1, 4, 150])
def test_rows_before_the_first_position_see_nothing(gpu, bits, new):
    """More new tokens than the length has: the first of them, all of them, sequences of length zero."""
    torch, P = gpu
    rng = np.random.default_rng(bits * new)
    s = R.make(rng, [(0, new), (20, new), (0, new)], 2, 64, 16, bits, "f16")
    s.lengths[0] = max(0, new - 3)
    s.lengths[2] = 0
    q, exact_q = queries(torch, rng, s, 2)
    s.dense = {n: [s.dense[n][b][:s.lengths[b]] for b in range(3)] for n in "kv"}
    want, bound = R.attention(s, exact_q)
    got = attend(torch, P, s, q, 2)
    check(got, want, bound)
    end = int(s.offsets[3])
    assert (got[end - new:] == 0).all() and (got[:min(3, new)] == 0).all()


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -65504.0])
@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("new,window,sinks", [(1, 40, 3), (3, 40, 3), (100, 40, 3), (100, 0, 0), (5, 0, 0)])
def test_what_a_query_does_not_see_has_no_part_in_it(gpu, value, bits, new, window, sinks):
    """Keys and values at positions that some queries see, others not, and that nobody sees, replaced one after another: queries that do not
    see them keep their bits."""
    torch, P = gpu
    rng = np.random.default_rng(17)
    s = R.make(rng, [(120, new), (64, new)], 2, 64, 16, bits, "f16")
    q, _ = queries(torch, rng, s, 2)
    before = attend(torch, P, s, q, 2, window, sinks)
    assert torch.isfinite(before).all()
    length = 120 + new
    for pos in sorted({0, 3, 50, 80, length - 41, length - 40, length - 2, length - 1}):
        if not 0 <= pos < length:
            continue
        page, slot = int(s.table[0, pos // 16]), pos % 16
        kept = [t.clone() for t in (s.pools["k"], s.pools["v"])] + [None if bits == 16 else s.scales[n].clone() for n in "kv"]
        if bits == 16:
            s.pools["k"][page, :, slot] = value
            s.pools["v"][page, :, slot] = value
        else:
            s.scales["k"][page, :, slot] = value
            s.scales["v"][page, :, slot] = value
        after = attend(torch, P, s, q, 2, window, sinks)
        s.pools["k"], s.pools["v"] = kept[:2]
        s.scales["k"], s.scales["v"] = kept[2:]
        for r in range(s.total):
            at = 120 + r if r < new else None
            seen = at is not None and pos <= at and (window == 0 or pos > at - window or pos < sinks)
            if not seen:
                assert torch.equal(before[r], after[r]), (pos, r)
            elif value != value:
                assert torch.isnan(after[r]).all(), (pos, r)


@pytest.mark.parametrize("bits,new,splits", [(16, 1, False), (4, 1, True), (16, 60, False), (8, 60, False)])
def test_dropped_pages_are_not_seen(gpu, bits, new, splits):
    """Table entries that name no page, where the window has passed and where it has not."""
    torch, P = gpu
    rng = np.random.default_rng(23)
    s = R.make(rng, [(200, new)], 2, 64, 16, bits, "f16", max_pages=1000 if splits else None)
    q, exact_q = queries(torch, rng, s, 2)
    whole = attend(torch, P, s, q, 2, 50, 4)
    kept = s.table.copy()
    s.table[0, 1:9] = [-1, s.n_pages, 2 ** 31 - 1, -2 ** 31, -1, -1, -1, -1]     # positions 16 .. 143: outside every window
    assert torch.equal(whole, attend(torch, P, s, q, 2, 50, 4))
    s.table = kept
    s.table[0, [1, 12]] = -1
    hide = np.zeros(200 + new, bool)
    hide[16:32] = hide[192:208] = True
    check(attend(torch, P, s, q, 2), *R.attention(s, exact_q, hide=[hide]))


@pytest.mark.parametrize("new", [1, 50])
@pytest.mark.parametrize("io", ["f16", "bf16"])
def test_large_scores_and_a_scale(gpu, new, io):
    """Scores of several hundred: one key carries almost everything; and a scale of the caller's."""
    torch, P = gpu
    rng = np.random.default_rng(29)
    for bits in (16, 8):
        s = R.make(rng, [(150, new)], 2, 64, 16, bits, io, spread=6.0)
        q, exact_q = queries(torch, rng, s, 2, 6.0)
        check(attend(torch, P, s, q, 2, scale=0.7), *R.attention(s, exact_q, scale=0.7))


@pytest.mark.parametrize("spread", [1e-6, 3e3])
@pytest.mark.parametrize("new", [1, 70])
def test_values_of_any_size(gpu, spread, new):
    """Scales of values far from 1, and far from one another."""
    torch, P = gpu
    rng = np.random.default_rng(31)
    for bits in (8, 4):
        s = R.make(rng, [(100, new)], 1, 64, 16, bits, "bf16", v_spread=spread)
        s.scales["v"][:, :, ::3] *= 2.0 ** -18
        s.dense["v"] = [R.unpacked(s.pools["v"].numpy(), bits)[s.table[0]].transpose(0, 2, 1, 3).reshape(-1, 1, 64)[:100 + new] *
                        s.scales["v"].double().numpy()[s.table[0]].transpose(0, 2, 1).reshape(-1, 1, 1)[:100 + new]]
        q, exact_q = queries(torch, rng, s, 1)
        check(attend(torch, P, s, q, 1), *R.attention(s, exact_q))


@pytest.mark.parametrize("bits,new", [(16, 1), (8, 3), (16, 90)])
def test_rows_that_lie_apart(gpu, bits, new):
    """q as a slice of a projection's output, out as a slice of a wider matrix whose other columns stay."""
    torch, P = gpu
    rng = np.random.default_rng(37)
    s = R.make(rng, [(33, new), (70, new)], 4, 64, 16, bits, "f16")
    q, _ = queries(torch, rng, s, 4)
    want = attend(torch, P, s, q, 4)
    cache, batch = R.upload(P, s)
    fused = torch.randn(s.total, 3, 4, 64, device="cuda").half()
    fused[:, 1] = q.cuda()
    wide = torch.full((s.total, 2, 4, 64), 7.0, dtype=torch.float16, device="cuda")
    need = P.sti_cache_attention_workspace_bytes(cache, batch, 4)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    P.sti_cache_attention(cache, batch, fused[:, 1], wide[:, 1], ws)
    assert torch.equal(wide[:, 1].cpu(), want) and (wide[:, 0] == 7).all()


@pytest.mark.parametrize("new", [1, 2, 20])
def test_many_sequences_and_rows_of_none(gpu, new):
    """More sequences than lanes; rows before the first offset and behind the last stay as they are."""
    torch, P = gpu
    rng = np.random.default_rng(41)
    rows = [(int(rng.integers(0, 60)), int(rng.integers(0, new + 1))) for _ in range(150)]
    s = R.make(rng, rows, 2, 64, 16, 16, "f16")
    q, exact_q = queries(torch, rng, s, 2)
    want, bound = R.attention(s, exact_q)
    check(attend(torch, P, s, q, 2), want, bound)
    n = s.total + 9
    s.offsets = s.offsets + 4
    wide = torch.zeros(n, 2, 64, dtype=torch.float16)
    wide[4:4 + s.total] = q
    got = attend(torch, P, s, wide, 2, n_tokens=n)
    check(got[4:4 + s.total], want, bound)
    assert torch.isnan(got[:4]).all() and torch.isnan(got[4 + s.total:]).all()


def test_pools_beyond_32_bits(gpu):
    """Rows more than 2^32 bytes into the pool, and behind 2^31 values."""
    torch, P = gpu
    rng = np.random.default_rng(43)
    n_pages, heads, page, d = 300, 64, 1024, 128       # 16 MiB a page
    k = torch.empty(n_pages, heads, page, d, dtype=torch.float16, device="cuda")
    v = torch.empty_like(k)
    cache = P.StiCache(k, v)
    for new in (1, 40):
        s = R.make(rng, [(30, new)], heads, d, page, 16, "f16")
        last = torch.tensor([[n_pages - 1]], dtype=torch.int32, device="cuda")
        total = 30 + new
        everything = P.StiCacheBatch(last, torch.tensor([total], dtype=torch.int32, device="cuda"),
                                     torch.tensor([0, total], dtype=torch.int32, device="cuda"), total)
        dense = {n: torch.from_numpy(np.ascontiguousarray(s.dense[n][0])).half().cuda() for n in "kv"}
        P.sti_cache_append(cache, everything, dense["k"], dense["v"])
        assert torch.equal(k[-1, :, :total], dense["k"].transpose(0, 1)) and torch.equal(v[-1, :, :total], dense["v"].transpose(0, 1))
        back = [torch.empty(1, total, heads, d, dtype=torch.float16, device="cuda") for _ in "kv"]
        P.sti_cache_read(cache, everything, 0, *back)
        assert torch.equal(back[0][0], dense["k"]) and torch.equal(back[1][0], dense["v"])
        q, exact_q = queries(torch, rng, s, heads)
        batch = P.StiCacheBatch(last, everything.lengths, torch.tensor([0, new], dtype=torch.int32, device="cuda"), new)
        check(attend(torch, P, s, q, heads, on=(cache, batch)), *R.attention(s, exact_q))


@pytest.mark.parametrize("bits,new", [(4, 1), (16, 1), (8, 100)])
def test_another_stream_and_the_same_bits_again(gpu, bits, new):
    torch, P = gpu
    rng = np.random.default_rng(47)
    s = R.make(rng, [(3000, new), (10, new)], 2, 64, 16, bits, "f16")
    q, _ = queries(torch, rng, s, 4)
    first = attend(torch, P, s, q, 4)
    for _ in range(3):
        assert torch.equal(first, attend(torch, P, s, q, 4))
    cache, batch = R.upload(P, s)
    need = P.sti_cache_attention_workspace_bytes(cache, batch, 4)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    q = q.cuda()
    out = torch.empty_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    P.sti_cache_attention(cache, batch, q, out, ws, stream=side)
    side.synchronize()
    assert torch.equal(first, out.cpu())


@pytest.mark.parametrize("bits", [16, 8])
def test_a_captured_step_follows_lengths(gpu, bits):
    """Append, attention and reading back captured once; lengths change between the replays, each checked against eager calls."""
    torch, P = gpu
    rng = np.random.default_rng(53)
    s = R.make(rng, [(40, 1), (700, 1), (0, 1)], 2, 64, 16, bits, "f16", max_pages=60)
    s.table[:, :] = rng.permutation(180).reshape(3, 60)
    s.n_pages = 180
    for n in "kv":
        s.pools[n] = torch.zeros(180, 2, 16, s.pools[n].shape[3], dtype=s.pools[n].dtype)
        s.scales[n] = None if bits == 16 else torch.zeros(180, 2, 16)
    cache, batch = R.upload(P, s)
    q = torch.randn(3, 4, 64, device="cuda").half()
    k, v = torch.randn(3, 2, 64, device="cuda").half(), torch.randn(3, 2, 64, device="cuda").half()
    out = torch.zeros_like(q)
    back = [torch.zeros(3, 8, 2, 64, dtype=torch.float16, device="cuda") for _ in "kv"]
    need = P.sti_cache_attention_workspace_bytes(cache, batch, 4, 100, 2)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None

    def step():
        P.sti_cache_append(cache, batch, k, v)
        P.sti_cache_attention(cache, batch, q, out, ws, window=100, sinks=2)
        P.sti_cache_read(cache, batch, 3, *back)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    held = [t.clone() for t in (cache.k, cache.v)]
    scales = [None if t is None else t.clone() for t in (cache.k_scale, cache.v_scale)]
    for lengths in ([1, 1, 1], [41, 701, 1], [17, 900, 960], [0, 5, 2]):
        batch.lengths.copy_(torch.tensor(lengths, dtype=torch.int32))
        k.normal_()
        got = []
        for go in (graph.replay, step):
            cache.k.copy_(held[0]), cache.v.copy_(held[1])
            if bits < 16:
                cache.k_scale.copy_(scales[0]), cache.v_scale.copy_(scales[1])
            out.fill_(float("nan"))
            go()
            torch.cuda.synchronize()
            got.append([t.clone() for t in (out, cache.k, cache.v, *back)])
        assert all(torch.equal(a, b) for a, b in zip(*got))
        assert torch.isfinite(got[0][0]).all()


@pytest.mark.parametrize("bits,new", [(8, 1), (16, 1), (4, 5), (8, 90)])
def test_arrays_of_anything_stay_inside(gpu, bits, new):
    """Offsets that go back or past the rows, lengths and pages of any value: nothing outside the pool and the rows is touched."""
    torch, P = gpu
    rng = np.random.default_rng(67)
    s = R.make(rng, [(600, new)] * 4, 2, 64, 16, bits, "f16")
    q, _ = queries(torch, rng, s, 4)
    for seed in range(6):
        g = np.random.default_rng(seed)
        s.offsets = g.integers(-5, s.total + 9, 5).astype(np.int32)
        s.lengths = g.choice([-2 ** 31, -1, 0, 1, 599, 10 ** 6, 2 ** 31 - 1], 4).astype(np.int32)
        s.table = g.choice([-2 ** 31, -1, 0, 1, s.n_pages - 1, s.n_pages, 2 ** 31 - 1], s.table.shape).astype(np.int32)
        cache, batch = R.upload(P, s)
        need = P.sti_cache_attention_workspace_bytes(cache, batch, 4)
        ws = torch.full((need + 4096,), 7, dtype=torch.uint8, device="cuda")
        wide = torch.full((s.total + 64, 4, 64), 7.0, dtype=torch.float16, device="cuda")
        P.sti_cache_attention(cache, batch, q.cuda(), wide[32:32 + s.total], ws[:need] if need else None)
        k = torch.randn(s.total, 2, 64, device="cuda")
        P.sti_cache_append(cache, batch, k, k)
        back = torch.full((6, 50, 2, 64), 7.0, device="cuda")
        P.sti_cache_read(cache, batch, 590, back[:4], torch.empty_like(back[:4]))
        torch.cuda.synchronize()
        assert (wide[:32] == 7).all() and (wide[32 + s.total:] == 7).all() and (ws[need:] == 7).all() and (back[4:] == 7).all()


@pytest.mark.parametrize("io,value", [("bf16", 1e36), ("bf16", float("inf")), ("f16", float("nan")), ("bf16", 1e25)])
@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("new", [3, 70])
def test_queries_of_any_size_leave_the_others_alone(gpu, io, value, bits, new):
    """One value of one query: the other queries of its tile are within their bound."""
    torch, P = gpu
    rng = np.random.default_rng(71)
    s = R.make(rng, [(50, new)], 2, 64, 16, bits, io)
    q, exact_q = queries(torch, rng, s, 4)
    want, bound = R.attention(s, exact_q)
    q[1, 1, 5] = value
    got = attend(torch, P, s, q, 4).double().numpy()
    rest = np.ones(got.shape[:2], bool)
    rest[1, 1] = False
    assert (np.abs(got - want)[rest] <= bound[rest]).all()


def test_kernels_are_timed(gpu):
    torch, P = gpu
    rng = np.random.default_rng(59)
    s = R.make(rng, [(40, 1)], 2, 64, 16, 8, "f16")
    cache, batch = R.upload(P, s)
    q = torch.randn(1, 2, 64, device="cuda").half()
    P.sti_profile_begin()
    P.sti_cache_append(cache, batch, q, q)
    P.sti_cache_attention(cache, batch, q, torch.empty_like(q))
    P.sti_cache_read(cache, batch, 0, *[torch.empty(1, 4, 2, 64, dtype=torch.float16, device="cuda") for _ in "kv"])
    count = {k: n for k, (n, _) in P.sti_profile_end().items()}
    assert count["convert"] == 2 and count["attention"] == 1 and sum(count.values()) == 3


def test_random_shapes(gpu):
    """Forty small batches of every kind."""
    torch, P = gpu
    rng = np.random.default_rng(61)
    for _ in range(40):
        kv_heads, group = [(1, 1), (3, 1), (2, 2), (1, 3), (2, 4), (1, 7), (1, 16)][rng.integers(7)]
        bits, io, d = [16, 8, 4][rng.integers(3)], ["f16", "bf16"][rng.integers(2)], [64, 128][rng.integers(2)]
        most = [1, 3, 20, 140][rng.integers(4)]
        rows = [(int(rng.integers(0, 260)), int(rng.integers(0, most + 1))) for _ in range(rng.integers(1, 5))]
        if sum(n for _, n in rows) == 0:
            continue
        window, sinks = (0, 0) if rng.integers(2) else (int(rng.integers(1, 90)), int(rng.integers(0, 20)))
        s = R.make(rng, rows, kv_heads, d, int(2 ** rng.integers(4, 8)), bits, io, fill=float("inf"))
        q, exact_q = queries(torch, rng, s, kv_heads * group, 1.5)
        check(attend(torch, P, s, q, kv_heads * group, window, sinks), *R.attention(s, exact_q, window, sinks))


def test_the_streaming_example_runs(gpu, capsys):
    """Chunks and single tokens through layers of shards give what one call gives; fewer bits and a window do what they say."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "streaming_submodel.py")
    spec = importlib.util.spec_from_file_location("streaming_submodel", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    example.main()
    assert capsys.readouterr().out.count("\n") == 4


def test_streaming_against_the_layer_forward(gpu):
    """A sequence of one token sees itself alone, in causal order and without: the example's layers against sti_layer_forward."""
    import importlib.util
    import os
    torch, P = gpu
    import sti_synth as S
    from paper_2207_05022_amd import device as D
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "streaming_submodel.py")
    spec = importlib.util.spec_from_file_location("streaming_submodel", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    wl = S.small_workload(8, S.BERT_BASE, 1, 5, 1, n_absent=4)
    S.make_every_term_matter(wl, 8)
    shards, params, x = D.upload_workload(wl)
    x = x.half()
    model = example.StreamingSubmodel(wl.dims, shards, params, 5, 16)
    got = model.stream(x.view(5, -1), [1] * 5).float()
    y = torch.empty_like(x)
    ws = torch.empty(P.sti_workspace_bytes(wl.dims, 5, 1, P.STI_PREC_F16_MFMA), dtype=torch.uint8, device="cuda")
    P.sti_layer_forward(wl.dims, shards[0], params[0], x, y, P.STI_PREC_F16_MFMA, ws)
    off = (got - y.view(5, -1).float()).norm() / y.float().norm()
    assert off < 3e-3      # a handful of binary16 roundings (2^-11 each) on either side
