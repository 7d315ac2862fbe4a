// Writing new keys and values into the pages of a cache, quantised to 8 or 4 bits or as they are, and reading positions back.
//
//   scale = a * (1 / t),  a = max |x| of a row of d values, t = 127 or 7;   code = rint(x * (1 / scale))
//
// One scale per token and key/value head: the attention multiplies a score and a weight by it, never a single value.  A row is
// d / 8 lanes of 8 values: one or two 16-byte requests per lane and matrix, the maximum over the lanes by DPP.  Both kernels are bound by
// memory and, for few rows, by the chain offsets -> page -> row.
//
// Measured (kernel alone): one token of 12 heads of 64 in 4 bits 3.7 us to write and 3.0 to read its 38 positions back, start-up and that chain;
// 3953 tokens of 12 heads of 64 in 8 bits, 18 MB, 8.0 us to write; 24 sequences of up to 2001 positions, 16 heads of 64 in 16 bits, 334 MB, 45 us to
// read back, and 4 of up to 16896, 8 heads of 128 in 4 bits, 330 MB, 45 us: 7.4 TB/s (part of the pools comes from the cache in front of memory).
#include "cache_common.hpp"

namespace sti {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

__device__ inline float f32_value(uint32_t bits) { return __builtin_bit_cast(float, bits); }   // (of a vector's element: bit_cast takes the first)
__device__ inline float f16_value(uint32_t bits) { return (float)__builtin_bit_cast(_Float16, (uint16_t)bits); }
__device__ inline float bf16_value(uint32_t bits) { return __builtin_bit_cast(float, bits << 16); }
__device__ inline uint32_t f16_bits(float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); }
__device__ inline uint32_t bf16_bits(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }

template <sti_dtype T>
__device__ inline void load8(const void *p, int64_t at, float (&x)[8])   // 8 values from element `at` on
{
    if constexpr (T == STI_F32) {
        const u32x4 a = *(const u32x4 *)((const float *)p + at), b = *(const u32x4 *)((const float *)p + at + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = f32_value(a[i]);
            x[4 + i] = f32_value(b[i]);
        }
    } else {
        const u32x4 a = *(const u32x4 *)((const uint16_t *)p + at);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = T == STI_F16 ? f16_value(a[i] & 0xFFFF) : bf16_value(a[i] & 0xFFFF);
            x[2 * i + 1] = T == STI_F16 ? f16_value(a[i] >> 16) : bf16_value(a[i] >> 16);
        }
    }
}

template <bool STREAMED>
__device__ inline void put(u32x4 *p, u32x4 v)
{
    if constexpr (STREAMED)
        __builtin_nontemporal_store(v, p);
    else
        *p = v;
}
template <sti_dtype T, bool STREAMED = false>
__device__ inline void store8(void *p, int64_t at, const float (&x)[8])
{
    if constexpr (T == STI_F32) {
        u32x4 a, b;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            a[i] = __builtin_bit_cast(uint32_t, x[i]);
            b[i] = __builtin_bit_cast(uint32_t, x[4 + i]);
        }
        put<STREAMED>((u32x4 *)((float *)p + at), a);
        put<STREAMED>((u32x4 *)((float *)p + at + 4), b);
    } else {
        u32x4 a;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            a[i] = T == STI_F16 ? f16_bits(x[2 * i]) | f16_bits(x[2 * i + 1]) << 16 : bf16_bits(x[2 * i]) | bf16_bits(x[2 * i + 1]) << 16;
        put<STREAMED>((u32x4 *)((uint16_t *)p + at), a);
    }
}

template <int CTRL>
__device__ inline uint32_t max_moved(uint32_t v)
{
    const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
    return v > o ? v : o;
}
// largest of 8 or 16 consecutive lanes
template <int LANES>
__device__ inline uint32_t group_max(uint32_t v)
{
    v = max_moved<0xB1>(v);    // quad_perm: lane ^ 1
    v = max_moved<0x4E>(v);    // lane ^ 2
    v = max_moved<0x141>(v);   // mirrored in each 8: the other four
    if constexpr (LANES == 16) v = max_moved<0x140>(v);   // mirrored in each 16: the other eight
    return v;
}

// 8 values of a row into its slot; every lane of the row's group takes part
template <int BITS, sti_dtype STORED, int D>
__device__ inline void store_row(void *pool, float *scales, int64_t row, int part, const float (&x)[8])
{
    constexpr int LANES = D / 8;
    if constexpr (BITS == 16) {
        store8<STORED>(pool, row * D + part * 8, x);
    } else {
        constexpr float kMost = BITS == 8 ? 127.f : 7.f, kPerMost = (float)(1.0 / (BITS == 8 ? 127.0 : 7.0));
        // magnitudes compare as whole numbers, NaN above infinity above the finite ones
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t m = __builtin_bit_cast(uint32_t, x[i]) & 0x7FFFFFFFu;
            most = m > most ? m : most;
        }
        most = group_max<LANES>(most);
        const bool finite = most < 0x7F800000u, stored = most >= 0x0D800000u;   // 2^-100
        float scale = __builtin_bit_cast(float, most) * kPerMost;
        const float per_scale = finite && stored ? 1.0f / scale : 0.f;
        if (!stored) scale = 0.f;
        if (!finite) scale = __builtin_bit_cast(float, 0x7FC00000u);
        int code[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float c = rintf((finite ? x[i] : 0.f) * per_scale);
            code[i] = (int)fminf(fmaxf(c, -kMost), kMost);
        }
        if constexpr (BITS == 8) {
            u32x2 w;
#pragma unroll
            for (int h = 0; h < 2; ++h)
                w[h] = (code[4 * h] & 0xFF) | (code[4 * h + 1] & 0xFF) << 8 | (code[4 * h + 2] & 0xFF) << 16 | (uint32_t)code[4 * h + 3] << 24;
            *(u32x2 *)((uint8_t *)pool + row * D + part * 8) = w;
        } else {
            uint32_t w = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) w |= (uint32_t)(code[i] + 8) << (4 * i);
            *(uint32_t *)((uint8_t *)pool + row * (D / 2) + part * 4) = w;
        }
        if (part == 0) scales[row] = scale;
    }
}

// Position of each row's token in its sequence, for the rows of a wave (groups of LANES lanes, tokens ascending): a lane per sequence, one count of
// the sequences that end before a token where all rows are of one, a count per row otherwise.
template <int LANES>
__device__ inline void find_slot(const CacheView &c, const BatchView &b, int token, int *seq, int *position)
{
    const int lane = threadIdx.x & 63;
    *seq = -1;
    *position = -1;
    const int first_token = __builtin_amdgcn_readlane(token, 0), last_token = __builtin_amdgcn_readlane(token, 63);
    for (int s0 = 0; s0 < b.n_seqs; s0 += 64) {
        const NewRows r = new_rows(b, min(s0 + lane, b.n_seqs - 1));
        const int end = s0 + lane < b.n_seqs ? r.end : 0x7FFFFFFF;
        // rows of `t`: those among the lanes of this test
        auto take = [&](int t, int n, bool mine) {
            const int l = min(n, 63);
            if (mine && *seq < 0 && n < 64 && s0 + n < b.n_seqs) {
                *seq = s0 + n;
                *position = t >= __builtin_amdgcn_readlane(r.first, l) ? __builtin_amdgcn_readlane(r.length, l) - (__builtin_amdgcn_readlane(r.end, l) - t) : -1;
            }
        };
        const int before_first = __popcll(__ballot(end <= first_token)), before_last = __popcll(__ballot(end <= last_token));
        if (before_first == before_last) {
            take(token, before_first, true);
        } else {
#pragma unroll
            for (int g = 0; g < 64; g += LANES) {
                const int t = __builtin_amdgcn_readlane(token, g);
                take(t, __popcll(__ballot(end <= t)), (lane & ~(LANES - 1)) == g);
            }
        }
        if (before_last < 64) break;
    }
    if (*position >= cache_capacity(c, b)) *position = -1;
    if (*position < 0) *seq = -1;
}

// A row to a group of lanes, keys and values together, so that what a token's slot is found from is read once; the rows are asked for in front of it.
template <int BITS, sti_dtype STORED, sti_dtype IO, int D>
__global__ __launch_bounds__(256) void cache_append_kernel(CacheView c, BatchView b, const void *k, const void *v, int64_t k_stride,
                                                           int64_t v_stride, uint32_t heads_recip)
{
    constexpr int LANES = D / 8, ROWS = 256 / LANES;
    const int part = threadIdx.x % LANES;
    // rows in the order (8 tokens, head, token): the slots of 8 tokens of a sequence lie behind each other in a page (by token and head, whose slots lie
    // a page's row apart: 9.1 us in place of 8.9 for the 3953 tokens above)
    const int row = (int)(blockIdx.x * ROWS + threadIdx.x / LANES);
    const int eight = quotient(row >> 3, c.heads, heads_recip), head = (row >> 3) - eight * c.heads;
    const int token_in = eight * 8 + (row & 7), token = min(token_in, b.n_tokens - 1);
    float xk[8], xv[8];
    load8<IO>(k, token * k_stride + head * D + part * 8, xk);
    load8<IO>(v, token * v_stride + head * D + part * 8, xv);
    int seq, position;
    find_slot<LANES>(c, b, token, &seq, &position);
    const int page = seq >= 0 && token_in < b.n_tokens ? cache_page(b, c, seq, position) : -1;
    if (!is_page(c, page)) return;   // (whole groups of lanes)
    const int64_t at = cache_row(c, page, head, position);
    store_row<BITS, STORED, D>((void *)c.k, (float *)c.k_scale, at, part, xk);
    store_row<BITS, STORED, D>((void *)c.v, (float *)c.v_scale, at, part, xv);
}

template <int BITS, sti_dtype STORED, int D>
__device__ inline void load_row(const void *pool, const float *scales, int64_t row, int part, float (&x)[8])
{
    if constexpr (BITS == 16) {
        load8<STORED>(pool, row * D + part * 8, x);
    } else {
        const float scale = scales[row];
        if constexpr (BITS == 8) {
            const u32x2 w = *(const u32x2 *)((const uint8_t *)pool + row * D + part * 8);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = (float)(int8_t)(w[i / 4] >> (8 * (i % 4))) * scale;
        } else {
            const uint32_t w = *(const uint32_t *)((const uint8_t *)pool + row * (D / 2) + part * 4);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = (float)((int)(w >> (4 * i) & 15) - 8) * scale;
        }
    }
}

// A block takes rows of one sequence in the order (chunk of 16 positions, head, position): the positions of a page and head lie behind each other in
// the pool, whole rows of an output line are 2 D bytes or more.
template <int BITS, sti_dtype STORED, sti_dtype OUT, int D>
__global__ __launch_bounds__(256) void cache_read_kernel(CacheView c, BatchView b, int first, int count, uint32_t heads_recip, void *k_out, void *v_out)
{
    constexpr int LANES = D / 8, ROWS = 256 / LANES;
    const int part = threadIdx.x % LANES, row = blockIdx.x * ROWS + threadIdx.x / LANES;
    const int chunk = quotient(row >> 4, c.heads, heads_recip), head = (row >> 4) - chunk * c.heads, j = chunk * 16 + (row & 15), position = first + j;
    if (j >= count) return;
    for (int seq = blockIdx.y; seq < b.n_seqs; seq += gridDim.y) {
        int page = -1;
        if (position < min(b.lengths[seq], cache_capacity(c, b))) page = cache_page(b, c, seq, position);
        float xk[8] = {}, xv[8] = {};
        if (is_page(c, page)) {
            const int64_t at = cache_row(c, page, head, position);
            load_row<BITS, STORED, D>(c.k, c.k_scale, at, part, xk);
            load_row<BITS, STORED, D>(c.v, c.v_scale, at, part, xv);
        }
        const int64_t to = (((int64_t)seq * count + j) * c.heads + head) * D + part * 8;
        store8<OUT, true>(k_out, to, xk);   // (past the caches: what is read back of long sequences is more than they hold; append and read 84 -> 51 us for 335 MB)
        store8<OUT, true>(v_out, to, xv);
    }
}

// go(a type with constants BITS, STORED, D) for what a cache holds
template <int B, sti_dtype S, int W>
struct Held {
    static constexpr int BITS = B, D = W;
    static constexpr sti_dtype STORED = S;
};
template <int D, typename Go>
inline void with_bits(int bits, sti_dtype stored, Go go)
{
    if (bits == 4)
        go(Held<4, STI_F16, D>());
    else if (bits == 8)
        go(Held<8, STI_F16, D>());
    else if (stored == STI_F16)
        go(Held<16, STI_F16, D>());
    else
        go(Held<16, STI_BF16, D>());
}
template <typename Go>
inline void with_held(int bits, int d, sti_dtype stored, Go go)
{
    if (d == 64)
        with_bits<64>(bits, stored, go);
    else
        with_bits<128>(bits, stored, go);
}

}  // namespace

hipError_t launch_cache_append(const CacheView &c, const BatchView &b, int bits, int d, sti_dtype stored, const void *k, const void *v,
                               sti_dtype io, int64_t k_stride, int64_t v_stride, hipStream_t stream)
{
    const int64_t rows = ((int64_t)b.n_tokens + 7) / 8 * 8 * c.heads, per_block = 256 / (d / 8);
    const dim3 grid((uint32_t)((rows + per_block - 1) / per_block));
    with_held(bits, d, stored, [&](auto h) {
        using H = decltype(h);
        const uint32_t recip = reciprocal((uint32_t)c.heads);
        if (io == STI_F32)
            launch(cache_append_kernel<H::BITS, H::STORED, STI_F32, H::D>, grid, dim3(256), 0, stream, c, b, k, v, k_stride, v_stride, recip);
        else if (io == STI_F16)
            launch(cache_append_kernel<H::BITS, H::STORED, STI_F16, H::D>, grid, dim3(256), 0, stream, c, b, k, v, k_stride, v_stride, recip);
        else
            launch(cache_append_kernel<H::BITS, H::STORED, STI_BF16, H::D>, grid, dim3(256), 0, stream, c, b, k, v, k_stride, v_stride, recip);
    });
    return hipGetLastError();
}

hipError_t launch_cache_read(const CacheView &c, const BatchView &b, int bits, int d, sti_dtype stored, int first, int count, void *k_out,
                             void *v_out, sti_dtype out, hipStream_t stream)
{
    const int64_t rows = ((int64_t)count + 15) / 16 * 16 * c.heads, per_block = 256 / (d / 8);
    const dim3 grid((uint32_t)((rows + per_block - 1) / per_block), (uint32_t)std::min(b.n_seqs, 65535));
    const uint32_t recip = reciprocal((uint32_t)c.heads);
    with_held(bits, d, stored, [&](auto h) {
        using H = decltype(h);
        if (out == STI_F32)
            launch(cache_read_kernel<H::BITS, H::STORED, STI_F32, H::D>, grid, dim3(256), 0, stream, c, b, first, count, recip, k_out, v_out);
        else if (out == STI_F16)
            launch(cache_read_kernel<H::BITS, H::STORED, STI_F16, H::D>, grid, dim3(256), 0, stream, c, b, first, count, recip, k_out, v_out);
        else
            launch(cache_read_kernel<H::BITS, H::STORED, STI_BF16, H::D>, grid, dim3(256), 0, stream, c, b, first, count, recip, k_out, v_out);
    });
    return hipGetLastError();
}

}  // namespace sti
