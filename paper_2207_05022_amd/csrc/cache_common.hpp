// What the kernels of the paged key/value cache share: device views of the caller's structs, where a position's row lies, which
// keys a tile of queries sees, and the launches behind the entry points of cache_api.hip.
#pragma once
#include <algorithm>
#include <type_traits>
#include "sti_internal.hpp"
#include "lane_ops.hpp"

namespace sti {

constexpr int kMaxCacheHeads = 64, kMaxQueryHeads = 512;

struct CacheView {
    const uint8_t *k, *v;
    const float *k_scale, *v_scale;
    int32_t heads;        // key/value heads
    int32_t page_shift;   // log2 of the slots of a page
    int32_t n_pages;
};
struct BatchView {
    const int32_t *table, *lengths, *offsets;
    int32_t n_seqs, n_tokens, max_pages;
};

// The row of (page, head, slot): below 2^32 (the entry points' limit), while its bytes may lie beyond 2^32 in an ordinary pool.
__device__ inline uint32_t cache_row(const CacheView &c, int page, int head, int position)
{
    return (((uint32_t)page * c.heads + head) << c.page_shift) + (position & ((1 << c.page_shift) - 1));
}
// Page of a position (0 <= position < capacity), or -1 where the table names none of the pool's.
__device__ inline int cache_page(const CacheView &c, const BatchView &b, int seq, int position)
{
    const int page = b.table[(int64_t)seq * b.max_pages + (position >> c.page_shift)];
    return (uint32_t)page < (uint32_t)c.n_pages ? page : -1;
}
__device__ inline int cache_capacity(const CacheView &c, const BatchView &b) { return b.max_pages << c.page_shift; }

// A sequence's new rows and its length, inside what the structs promise whatever the caller's arrays hold.  Positions, lengths and windows stay
// within 2^30 + 2^24 of zero (the entry points' limits), so that their sums and differences fit 32 bits.
struct NewRows {
    int first, end, length;
};
__device__ inline NewRows new_rows(const BatchView &b, int seq)
{
    NewRows r;
    r.first = min(max(b.offsets[seq], 0), b.n_tokens);
    r.end = min(max(b.offsets[seq + 1], r.first), b.n_tokens);
    r.length = min(max(b.lengths[seq], 0), 1 << 30);
    return r;
}

// Queries of one key/value head of one sequence, in the order (token, query head of the group), cut into tiles of `rows`; the tiles of
// all sequences one after another, as many as tile_bound() or fewer (how many rows a sequence has is known on the device only).
inline int64_t tile_bound(int64_t n_tokens, int n_seqs, int group, int rows)
{
    const int64_t by_rows = (n_tokens * group) / rows + n_seqs;   // (a sequence adds at most one tile that is not full)
    return std::min(by_rows, n_tokens * group);
}

// What a tile's queries see, as a range of consecutive numbers: first the `sinks` keys 0 .. sinks - 1, then the keys from `low` on.
struct TileKeys {
    int sinks, low, count;
    __device__ inline int key(int x) const { return x < sinks ? x : x - sinks + low; }
};
struct QueryTile {
    int seq;              // -1: none
    int first;            // first row of the sequence's new tokens
    int row0, rows;       // the tile's (token, head of the group) pairs inside the sequence
    int base;             // position of the sequence's first new token (may be negative)
    int first_pos, last_pos;   // positions of the tile's first and last token
    TileKeys keys;
};

__device__ inline int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Tile `index` of the batch, found by one wave: a lane per sequence, sums of their tiles over the lanes.
__device__ inline QueryTile find_tile(const CacheView &c, const BatchView &b, int index, int group, uint32_t group_recip, int tile_rows,
                                      int window, int sinks)
{
    const int lane = threadIdx.x & 63;
    QueryTile t;
    t.seq = -1;
    int before = 0;
    for (int s0 = 0; s0 < b.n_seqs; s0 += 64) {
        const int s = min(s0 + lane, b.n_seqs - 1);
        const NewRows r = new_rows(b, s);
        const int first = r.first, n = r.end - r.first, length = r.length;
        const uint32_t tiles = s0 + lane < b.n_seqs ? (uint32_t)(((int64_t)n * group + tile_rows - 1) / tile_rows) : 0u;
        const uint32_t upto = lane_scan(tiles);
        const uint64_t past = __ballot(upto + (uint32_t)before > (uint32_t)index);
        if (past) {
            const int l = __ffsll((unsigned long long)past) - 1;
            t.seq = s0 + l;
            t.first = __builtin_amdgcn_readlane(first, l);
            const int count = __builtin_amdgcn_readlane(n, l);
            const int len = __builtin_amdgcn_readlane(length, l);
            const int in_seq = index - before - (int)(__builtin_amdgcn_readlane((int)upto, l) - __builtin_amdgcn_readlane((int)tiles, l));
            t.row0 = in_seq * tile_rows;
            t.rows = min(tile_rows, count * group - t.row0);
            t.base = len - count;
            t.first_pos = t.base + quotient(t.row0, group, group_recip);
            t.last_pos = t.base + quotient(t.row0 + t.rows - 1, group, group_recip);
            const int high = max(0, min(min(t.last_pos + 1, len), cache_capacity(c, b)));   // keys below it are seen by some query
            const int low = window > 0 ? min(max(t.first_pos - window + 1, 0), high) : 0;
            t.keys.sinks = window > 0 ? min(sinks, low) : 0;
            t.keys.low = low;
            t.keys.count = t.keys.sinks + high - low;
            return t;
        }
        before += __builtin_amdgcn_readlane((int)upto, 63);
    }
    return t;
}

// Whether a query at `pos` sees `key` (a key below its sequence's length).
__device__ inline bool sees(int pos, int key, int window, int sinks)
{
    return key <= pos && (window <= 0 || key > pos - window || key < sinks);
}

// Bit j of the result: the query at `pos` sees number x0 + j of its tile's keys (below x_end).  Keys grow with their numbers, so that what a query
// sees is the numbers below `sinks` and those from the window's first to its own.
__device__ inline uint64_t bits_below(int n) { return n <= 0 ? 0 : n >= 64 ? ~(uint64_t)0 : ((uint64_t)1 << n) - 1; }
__device__ inline uint64_t seen_keys(const TileKeys &keys, int pos, int window, int sinks, int x0, int x_end)
{
    const int own = pos < keys.low ? min(pos + 1, keys.sinks) : keys.sinks + pos - keys.low + 1;   // numbers of keys up to pos
    uint64_t seen = bits_below(min(own, x_end) - x0);
    if (window > 0) seen &= bits_below(sinks - x0) | ~bits_below(keys.sinks + max(0, pos - window + 1 - keys.low) - x0);
    return seen;
}

// ---- launches (cache_store.hip, cache_attention.hip) ----
hipError_t launch_cache_append(const CacheView &c, const BatchView &b, int bits, int d, sti_dtype stored, const void *k, const void *v,
                               sti_dtype io, int64_t k_stride, int64_t v_stride, hipStream_t stream);
hipError_t launch_cache_read(const CacheView &c, const BatchView &b, int bits, int d, sti_dtype stored, int first, int count, void *k_out,
                             void *v_out, sti_dtype out, hipStream_t stream);

struct AttentionCall {
    CacheView cache;
    BatchView batch;
    int bits, d, heads, group;
    bool bf16;
    float scale;          // includes log2(e)
    int window, sinks;
    const void *q;
    void *out;
    int64_t q_stride, out_stride;
};
// How a call of these sizes is cut: the kernel's rows per tile, and the keys that one workgroup takes of a tile (a multiple of 256).  A tile of
// more keys has several workgroups, at most `splits`; how many is known on the device.
struct AttentionCut {
    int tile_rows, splits, keys;
    int64_t tiles;        // bound
};
AttentionCut attention_cut(int64_t n_tokens, int n_seqs, int heads, int kv_heads, int64_t capacity, int window, int sinks);
// A workgroup's share of its tile's keys: numbers begin .. end - 1.
struct KeyShare {
    int begin, end, parts;   // parts: shares of the tile, 1: the workgroup leaves the result itself
};
__device__ inline KeyShare key_share(const TileKeys &keys, int split, int per_split)
{
    KeyShare s;
    s.parts = max(1, (keys.count + per_split - 1) / per_split);
    s.begin = split * per_split;
    s.end = min(keys.count, s.begin + per_split);
    return s;
}
// Partial results where tiles may have several shares: sums [splits][n_tokens * heads][d], maxima and weights' sums [splits][n_tokens * heads][2],
// and of each row how many shares there are.
inline size_t partial_bytes(int64_t n_tokens, int heads, int d, int splits)
{
    const size_t rows = (size_t)n_tokens * heads;
    return splits > 1 ? rows * splits * (d + 2) * sizeof(float) + rows * sizeof(int32_t) : 0;
}
struct Partials {
    float *sums, *top_weight;
    int32_t *parts;
};
inline Partials partials_at(void *workspace, int64_t n_tokens, int heads, int d, int splits)
{
    const size_t rows = (size_t)n_tokens * heads;
    float *sums = (float *)workspace;
    return Partials{sums, sums + rows * splits * d, (int32_t *)(sums + rows * splits * (d + 2))};
}
hipError_t launch_cache_attention(const AttentionCall &a, const AttentionCut &cut, const Partials &partials, hipStream_t stream);
hipError_t launch_cache_few(const AttentionCall &a, const AttentionCut &cut, const Partials &partials, hipStream_t stream);     // tile_rows 16
hipError_t launch_cache_tiles(const AttentionCall &a, const AttentionCut &cut, const Partials &partials, hipStream_t stream);   // 64 and 128
hipError_t launch_cache_join(const AttentionCall &a, int splits, const Partials &partials, hipStream_t stream);

}  // namespace sti
