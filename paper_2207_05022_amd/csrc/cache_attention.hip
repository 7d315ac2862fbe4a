// Attention of a few queries per sequence over a paged cache: each key and value is read once, by lanes that hold a piece of its row.
//
//   s_j = c q . k_j,   o = sum_j 2^(s_j - m) v_j / sum_j 2^(s_j - m)      (c: scale * log2(e))
//
// A key's row is spread over LPK lanes of 16 bytes (8 values of 16 bits, 16 codes of 8 bits; 8 bytes for 16 codes of 4), so that a wave
// asks for 64 / LPK rows at once and the values arrive as they lie: no transposition, no LDS.  A group of LPK lanes keeps a running maximum, sum
// and result of its own keys; groups and waves are joined once, at the end, and so are the splits of a long sequence over workgroups
// (cache_join_kernel).  All arithmetic is float32 on values or codes as they are stored; a row's scale multiplies its score and its weight.
#include "cache_numbers.hpp"

namespace sti {
namespace {

typedef cache_u32x4 u32x4;
typedef cache_u32x2 u32x2;
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float2v __attribute__((ext_vector_type(2)));

constexpr int kWaves = 4;

template <int BITS>
struct Piece {   // what a lane holds of a row
    static constexpr int VALUES = BITS == 16 ? 8 : 16, BYTES = BITS == 4 ? 8 : 16;
    u32x4 w;
    __device__ inline void load(const uint8_t *p)
    {
        if constexpr (BITS == 4) {
            const u32x2 h = *(const u32x2 *)p;
            w = u32x4{h.x, h.y, 0, 0};
        } else {
            w = *(const u32x4 *)p;
        }
    }
    template <bool BF>
    __device__ inline float value(int i) const
    {
        if constexpr (BITS == 16) {
            const uint32_t h = w[i / 2];
            if constexpr (BF) return __builtin_bit_cast(float, i & 1 ? h & 0xFFFF0000u : h << 16);
            return (float)__builtin_bit_cast(_Float16, (uint16_t)(i & 1 ? h >> 16 : h & 0xFFFF));
        } else if constexpr (BITS == 8) {
            return (float)(int8_t)(w[i / 4] >> (8 * (i % 4)));
        } else {
            return (float)((int)(w[i / 8] >> (4 * (i % 8)) & 15) - 8);
        }
    }
};

template <int LPK>
__device__ inline float piece_sum(float v)   // over the LPK lanes of a key; every lane ends with the same bits
{
    auto moved_by = [](float x, auto ctrl) {
        return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value, 0xf, 0xf, true));
    };
    v += moved_by(v, std::integral_constant<int, 0xB1>());    // lane ^ 1
    v += moved_by(v, std::integral_constant<int, 0x4E>());    // lane ^ 2
    if constexpr (LPK >= 8) v += moved_by(v, std::integral_constant<int, 0x141>());
    if constexpr (LPK >= 16) v += moved_by(v, std::integral_constant<int, 0x140>());
    return v;
}
// over the groups of LPK lanes of the wave: lanes with the same number inside their group
template <int LPK>
__device__ inline float across_groups_max(float v)
{
    v = pair_max(across_32(v));
    v = pair_max(across_16(v));
    if constexpr (LPK <= 8) v = fmaxf(v, rotated<8>(v));
    if constexpr (LPK <= 4) v = fmaxf(v, rotated<4>(v));
    return v;
}
template <int LPK>
__device__ inline float across_groups_sum(float v)
{
    v = pair_sum(across_32(v));
    v = pair_sum(across_16(v));
    if constexpr (LPK <= 8) v += rotated<8>(v);
    if constexpr (LPK <= 4) v += rotated<4>(v);
    return v;
}

__device__ inline float factor(float m, float top) { return m == top ? 1.f : __builtin_amdgcn_exp2f(m - top); }   // (both -inf: 1)

template <bool BF>
__device__ inline uint16_t rounded(float v)
{
    if constexpr (BF) return __builtin_bit_cast(uint16_t, (__bf16)v);
    return __builtin_bit_cast(uint16_t, (_Float16)v);
}

// ROWS (token, head) pairs of one key/value head per workgroup
template <int BITS, bool BF, int D, int ROWS>
__global__ __launch_bounds__(kWaves * 64) void cache_attention_kernel(AttentionCall a, WorkCut cut, Partials partials)
{
    using P = Piece<BITS>;
    constexpr int VALUES = P::VALUES, LPK = D / VALUES, AT_ONCE = 64 / LPK, U = 4, STEP = AT_ONCE * U, ROW_BYTES = D * BITS / 8;
    __shared__ float sums[kWaves][ROWS][D];
    __shared__ float tops[kWaves][ROWS], weights[kWaves][ROWS];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), part = lane % LPK, group_lane = lane / LPK;
    const CacheView &c = a.cache;
    const BatchView &b = a.batch;
    const int from_last = quotient(blockIdx.x, c.heads, cut.heads_recip), head = blockIdx.x - from_last * c.heads;   // blocks in the order (item, head)
    const QueryTile t = find_work(c, b, cut, from_last, head, a.group, a.window, a.sinks);
    if (t.seq < 0) return;

    float q[ROWS][VALUES], o[ROWS][VALUES], top[ROWS], sum[ROWS];
    int pos[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const int row = t.row0 + min(r, t.rows - 1), token = quotient(row, a.group, cut.group_recip);
        pos[r] = t.base + token;
        const uint16_t *src = (const uint16_t *)a.q + (t.first + token) * a.q_stride + (head * a.group + row - token * a.group) * D + part * VALUES;
#pragma unroll
        for (int i = 0; i < VALUES; i += 8) {
            Piece<16> h;
            h.w = *(const u32x4 *)(src + i);
#pragma unroll
            for (int j = 0; j < 8; ++j) q[r][i + j] = h.template value<BF>(j) * a.scale;
        }
#pragma unroll
        for (int i = 0; i < VALUES; ++i) o[r][i] = 0.f;
        top[r] = -INFINITY;
        sum[r] = 0.f;
    }

    const int x_end = t.end;
    for (int x0 = t.begin + wave * STEP; x0 < x_end; x0 += kWaves * STEP) {
        P k[U], v[U];
        float ks[U], vs[U];
        int key[U];
        bool there[U];
        bool plain = x0 + STEP <= x_end;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int x = x0 + u * AT_ONCE + group_lane;
            key[u] = t.keys.key(min(x, x_end - 1));
            const int page = cache_page(b, c, t.seq, key[u]);
            there[u] = x < x_end && is_page(c, page);
            plain &= is_page(c, page);
            const int64_t row = (int64_t)cache_row(c, page_or_0(c, page), head, key[u]);
            k[u].load(c.k + row * ROW_BYTES + part * P::BYTES);
            v[u].load(c.v + row * ROW_BYTES + part * P::BYTES);
            if constexpr (BITS < 16) {
                ks[u] = c.k_scale[row];
                vs[u] = c.v_scale[row];
            }
        }
        // whether every query sees every key of the step
        const int first = t.keys.key(x0), last = t.keys.key(min(x0 + STEP, x_end) - 1);
        plain &= last <= t.first_pos && (a.window <= 0 || first > t.last_pos - a.window || last < a.sinks);
        const bool all = __all(plain);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            float s[U];
            float m = top[r];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float d = 0.f;
#pragma unroll
                for (int i = 0; i < VALUES; ++i) d = fmaf(q[r][i], k[u].template value<BF>(i), d);
                s[u] = piece_sum<LPK>(d);
                if constexpr (BITS < 16) s[u] *= ks[u];
                if (!all && !(there[u] && sees(pos[r], key[u], a.window, a.sinks))) s[u] = -INFINITY;
                m = fmaxf(m, s[u]);
            }
            const float shrink = factor(top[r], m);
            top[r] = m;
            if (m == -INFINITY) m = 0.f;   // nothing seen yet, or scores of minus infinity: weights of zero
            sum[r] *= shrink;
#pragma unroll
            for (int i = 0; i < VALUES; ++i) o[r][i] *= shrink;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const bool seen = all || (there[u] && sees(pos[r], key[u], a.window, a.sinks));
                float p = seen ? __builtin_amdgcn_exp2f(s[u] - m) : 0.f;
                sum[r] += p;
                if constexpr (BITS < 16) p = seen ? p * vs[u] : 0.f;
                if (all) {
#pragma unroll
                    for (int i = 0; i < VALUES; ++i) o[r][i] = fmaf(p, v[u].template value<BF>(i), o[r][i]);
                } else if (seen) {   // (0 x NaN of a value that is not seen)
#pragma unroll
                    for (int i = 0; i < VALUES; ++i) o[r][i] = fmaf(p, v[u].template value<BF>(i), o[r][i]);
                }
            }
        }
    }

    // join the groups of the wave, then the waves
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const float m = across_groups_max<LPK>(top[r]), f = factor(top[r], m);
        const float l = across_groups_sum<LPK>(sum[r] * f);
#pragma unroll
        for (int i = 0; i < VALUES; ++i) {
            const float w = across_groups_sum<LPK>(o[r][i] * f);
            if (group_lane == i % AT_ONCE) sums[wave][r][part * VALUES + i] = w;
        }
        if (lane == 0) {
            tops[wave][r] = m;
            weights[wave][r] = l;
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < ROWS * D; i += kWaves * 64) {
        const int r = i / D, at = i % D;
        if (r >= t.rows) break;
        float m = tops[0][r];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) m = fmaxf(m, tops[w][r]);
        float l = 0.f, w = 0.f;
#pragma unroll
        for (int j = 0; j < kWaves; ++j) {
            const float f = factor(tops[j][r], m);
            l += weights[j][r] * f;
            w += sums[j][r][at] * f;
        }
        const int row = t.row0 + r, token = quotient(row, a.group, cut.group_recip);
        const int q_head = head * a.group + row - token * a.group;
        const int64_t to_row = (int64_t)(t.first + token) * a.heads + q_head, place = (t.slot + (int64_t)t.split * c.heads) * ROWS + r;
        if (t.parts == 1)
            ((uint16_t *)a.out)[(t.first + token) * a.out_stride + q_head * D + at] = rounded<BF>(l > 0.f ? w / l : (l == 0.f ? 0.f : l));
        else
            partials.sums[place * D + at] = w;
        if (cut.slots > 0 && at == 0) {
            partials.top_weight[place * 2] = m;
            partials.top_weight[place * 2 + 1] = l;
            if (t.split == 0) partials.rows[to_row] = {(int32_t)place, t.parts};
        }
    }
}

// The splits' results, each shrunk to the largest maximum.  D / 4 threads of 4 features take a row's splits GROUPS at a time; the groups of a row
// are joined through LDS.
template <bool BF, int D, int GROUPS>
__global__ __launch_bounds__(256) void cache_join_kernel(AttentionCall a, uint32_t heads_recip, int tile_rows, Partials partials)
{
    constexpr int WIDE = D / 4, PER_ROW = WIDE * GROUPS, ROWS = 256 / PER_ROW;
    __shared__ float4v sums[GROUPS > 1 ? GROUPS : 1][WIDE];
    __shared__ float tops[GROUPS], weights[GROUPS];
    const BatchView &b = a.batch;
    const int64_t line = (int64_t)b.n_tokens * a.heads;
    const int row = (int)(blockIdx.x * ROWS + threadIdx.x / PER_ROW), group = threadIdx.x / WIDE % GROUPS, at = threadIdx.x % WIDE;
    if (row >= line) return;   // (rows are whole blocks where groups meet, here and below)
    const int token = quotient(row, a.heads, heads_recip), head = row - token * a.heads;
    const int first = b.offsets[0], end = b.offsets[b.n_seqs];
    const RowShares shares_of = partials.rows[row];
    const int parts = shares_of.parts;
    if (token < first || token >= end || parts == 1) return;   // (of no sequence: no tile has left anything; one share: it has left the result)
    const float2v *ml = (const float2v *)partials.top_weight;
    float m = -INFINITY, l = 0.f;
    float4v w = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int s = group; s < parts; s += GROUPS) {
        const int64_t place = shares_of.place + (int64_t)s * a.cache.heads * tile_rows;
        const float2v theirs = ml[place];
        const float4v x = *(const float4v *)(partials.sums + place * D + at * 4);
        const float t = fmaxf(m, theirs.x), f0 = factor(m, t), f1 = factor(theirs.x, t);
        m = t;
        l = l * f0 + theirs.y * f1;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = w[i] * f0 + x[i] * f1;
    }
    if constexpr (GROUPS > 1) {
        sums[group][at] = w;
        if (at == 0) {
            tops[group] = m;
            weights[group] = l;
        }
        __syncthreads();
        if (group > 0) return;
#pragma unroll
        for (int j = 1; j < GROUPS; ++j) {
            const float theirs = tops[j], t = fmaxf(m, theirs), f0 = factor(m, t), f1 = factor(theirs, t);
            const float4v x = sums[j][at];
            m = t;
            l = l * f0 + weights[j] * f1;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = w[i] * f0 + x[i] * f1;
        }
    }
    const float inv = l > 0.f ? 1.0f / l : (l == 0.f ? 0.f : l);
    const u32x2 out = {cache_pair<BF>(w[0] * inv, w[1] * inv), cache_pair<BF>(w[2] * inv, w[3] * inv)};
    *(u32x2 *)((uint16_t *)a.out + token * a.out_stride + head * D + at * 4) = out;
}

template <int BITS, bool BF, int D>
void launch_rows(const AttentionCall &a, const AttentionCut &cut, const Partials &partials, hipStream_t stream)
{
    launch(cache_attention_kernel<BITS, BF, D, 1>, dim3((uint32_t)cut.blocks), dim3(kWaves * 64), 0, stream, a, cut.work, partials);
}
template <bool BF, int D>
void launch_bits(const AttentionCall &a, const AttentionCut &cut, const Partials &partials, hipStream_t stream)
{
    if (a.bits == 16)
        launch_rows<16, BF, D>(a, cut, partials, stream);
    else if (a.bits == 8)
        launch_rows<8, BF, D>(a, cut, partials, stream);
    else
        launch_rows<4, BF, D>(a, cut, partials, stream);
}

}  // namespace

AttentionCut attention_cut(int64_t n_tokens, int n_seqs, int heads, int kv_heads, int64_t capacity, int window, int sinks)
{
    const int group = heads / kv_heads;
    // rows that share a key/value head in an average sequence
    const int64_t rows = (n_tokens + n_seqs - 1) / n_seqs * group;
    AttentionCut cut;
    WorkCut &w = cut.work;
    w.rows = rows <= 1 ? 1 : rows <= 16 ? 16 : rows <= 64 ? 64 : 128;
    w.token_rows = (w.rows + group - 2) / group + 1;   // (a tile may begin and end inside a token's heads)
    w.group_recip = reciprocal((uint32_t)group);
    w.heads_recip = reciprocal((uint32_t)kv_heads);
    w.least_keys = 256;
    int64_t keys = capacity;   // the most that a tile's queries see
    if (window > 0) keys = std::min(keys, (int64_t)window + sinks + w.token_rows);
    const int64_t tiles = tile_bound(n_tokens, n_seqs, group, w.rows), slots = (w.rows == 1 ? 1024 : 512) / kv_heads;
    w.slots = tiles * kv_heads < 512 && keys >= 2 * w.least_keys ? (int32_t)slots : 0;
    cut.blocks = (w.slots > 0 ? slots : tiles) * kv_heads;
    return cut;
}

hipError_t launch_cache_attention(const AttentionCall &a, const AttentionCut &cut, const Partials &partials, hipStream_t stream)
{
    if (cut.work.rows > 16) return launch_cache_tiles(a, cut, partials, stream);
    if (cut.work.rows > 1) return launch_cache_few(a, cut, partials, stream);
    if (a.d == 64)
        a.bf16 ? launch_bits<true, 64>(a, cut, partials, stream) : launch_bits<false, 64>(a, cut, partials, stream);
    else
        a.bf16 ? launch_bits<true, 128>(a, cut, partials, stream) : launch_bits<false, 128>(a, cut, partials, stream);
    return hipGetLastError();
}

hipError_t launch_cache_join(const AttentionCall &a, const AttentionCut &cut, const Partials &partials, hipStream_t stream)
{
    const int64_t rows = (int64_t)a.batch.n_tokens * a.heads;
    const uint32_t recip = reciprocal((uint32_t)a.heads);
    // many rows: each to D / 4 threads; few (many shares, then): each to a workgroup
    const bool many = rows < 2048;
    const int64_t threads = many ? 256 : a.d / 4;
    const dim3 grid((uint32_t)((rows * threads + 255) / 256));
    auto go = [&](auto kernel) { launch(kernel, grid, dim3(256), 0, stream, a, recip, cut.work.rows, partials); };
    if (a.d == 64) {
        if (a.bf16)
            many ? go(cache_join_kernel<true, 64, 16>) : go(cache_join_kernel<true, 64, 1>);
        else
            many ? go(cache_join_kernel<false, 64, 16>) : go(cache_join_kernel<false, 64, 1>);
    } else {
        if (a.bf16)
            many ? go(cache_join_kernel<true, 128, 8>) : go(cache_join_kernel<true, 128, 1>);
        else
            many ? go(cache_join_kernel<false, 128, 8>) : go(cache_join_kernel<false, 128, 1>);
    }
    return hipGetLastError();
}

}  // namespace sti
