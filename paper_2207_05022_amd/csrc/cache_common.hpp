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
// Entry of the table for a position (0 <= position < capacity), and whether it names one of the pool's pages.  (Apart: what is asked for ahead is
// looked at where it is used, or the request is waited for where it is made.)
__device__ inline int cache_page(const BatchView &b, const CacheView &c, int seq, int position)
{
    return b.table[(int64_t)seq * b.max_pages + (position >> c.page_shift)];
}
__device__ inline bool is_page(const CacheView &c, int page) { return (uint32_t)page < (uint32_t)c.n_pages; }
__device__ inline int page_or_0(const CacheView &c, int page) { return is_page(c, page) ? page : 0; }
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

// Queries of one key/value head of one sequence, in the order (token, query head of the group), are cut into tiles of `rows`; the tiles of all
// sequences one after another are as many as tile_bound() or fewer (how many rows a sequence has is known on the device only).
inline int64_t tile_bound(int64_t n_tokens, int n_seqs, int group, int rows)
{
    const int64_t by_rows = (n_tokens * group) / rows + n_seqs;   // (a sequence adds at most one tile that is not full)
    return std::min(by_rows, n_tokens * group);
}

// How a call is cut.  Where its tiles leave compute units idle (slots > 0) the tiles of long sequences go to several workgroups, a share of the
// keys to each: the keys per share are the fewest for which all shares of a key/value head are at most `slots`, found on the device from the
// lengths.
struct WorkCut {
    int32_t rows, slots, least_keys, token_rows;   // rows of a tile; shares per head or 0; a share's least keys; most tokens of a tile
    uint32_t group_recip, heads_recip;
};

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
    int begin, end;       // the workgroup's share of them: numbers begin .. end - 1
    int parts, split;     // shares of the tile (1: the workgroup leaves the result itself), and which this is
    int64_t slot;         // where the share's partial results lie; those of the tile's next share `heads` behind it
};

__device__ inline int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ inline float uniform_float(float v) { return __builtin_bit_cast(float, uniform(__builtin_bit_cast(int, v))); }

// What this lane's sequence (s0 + lane) gives to do.
struct SequenceWork {
    NewRows r;
    int tiles, keys;   // keys: the most that one of its tiles sees
};
__device__ inline SequenceWork sequence_work(const CacheView &c, const BatchView &b, const WorkCut &cut, int s0, int group, int window, int sinks)
{
    const int lane = threadIdx.x & 63;
    SequenceWork w;
    w.r = new_rows(b, min(s0 + lane, b.n_seqs - 1));
    const int n = w.r.end - w.r.first;
    w.tiles = s0 + lane < b.n_seqs ? (int)(((int64_t)n * group + cut.rows - 1) / cut.rows) : 0;
    w.keys = min(w.r.length, cache_capacity(c, b));
    if (window > 0 && window < w.keys) w.keys = min((int64_t)w.keys, (int64_t)window + cut.token_rows + sinks);
    return w;
}
__device__ inline int shares(int keys, float per_keys) { return (int)((float)(keys - 1) * per_keys) + 1; }

// Work item `from_last` of key/value head `head`, counted from the last, found by one wave: a lane per sequence, sums over the lanes.  Items are the
// shares of a tile, tiles and sequences one after another: the later a tile of a sequence, the more keys it has, and the sooner it is begun.
__device__ inline QueryTile find_work(const CacheView &c, const BatchView &b, const WorkCut &cut, int from_last, int head, int group, int window, int sinks)
{
    QueryTile t;
    t.seq = -1;
    SequenceWork w = sequence_work(c, b, cut, 0, group, window, sinks);
    const bool one = b.n_seqs <= 64;
    // sums over all sequences of f(this lane's)
    auto over_all = [&](auto f) {
        float sum = lane_sum<64>(f(w));
        if (!one)
            for (int s0 = 64; s0 < b.n_seqs; s0 += 64) sum += lane_sum<64>(f(sequence_work(c, b, cut, s0, group, window, sinks)));
        return uniform_float(sum);
    };
    float per_keys = 0.f;   // 1 / the keys of a share
    if (cut.slots > 0) {
        const float all_keys = over_all([](const SequenceWork &q) { return (float)q.tiles * (float)q.keys; });
        const float one_round = all_keys * (1.f / 256.f) * (float)c.heads;   // keys of a share with one workgroup on each of the 256 compute units
        float low = fmaxf(all_keys / (float)cut.slots, fminf(fmaxf(one_round, (float)cut.least_keys), 256.f));
        float high = 0x1p31f;   // one share each
        auto fits = [&](float keys) {
            const float per = 1.f / keys;
            return over_all([&](const SequenceWork &q) { return (float)q.tiles * (float)shares(q.keys, per); }) <= (float)cut.slots;
        };
        if (fits(low)) {
            high = low;
        } else {
            // from the ideal share up in steps of an eighth, to twice as much; beyond that one doubling after another
            float step = low * 0.125f;
            for (int i = 0; i < 24; ++i) {
                low += step;
                if (fits(low)) {
                    high = low;
                    break;
                }
                if (i >= 7) step = low;
            }
        }
        per_keys = uniform_float(1.f / high);
    }
    const int items = (int)over_all([&](const SequenceWork &q) { return (float)q.tiles * (float)shares(q.keys, per_keys); });
    int before = 0;
    const int index = items - 1 - from_last;
    if (index < 0 || (cut.slots > 0 && index >= cut.slots)) return t;   // (the latter: offsets that are none; there is no place for its results)
    for (int s0 = 0; s0 < b.n_seqs; s0 += 64) {
        if (s0 > 0) w = sequence_work(c, b, cut, s0, group, window, sinks);
        const uint32_t mine = (uint32_t)(w.tiles * shares(w.keys, per_keys)), upto = lane_scan(mine);
        const uint64_t past = __ballot(upto + (uint32_t)before > (uint32_t)index);
        if (past) {
            const int l = __ffsll((unsigned long long)past) - 1;
            t.seq = s0 + l;
            t.first = __builtin_amdgcn_readlane(w.r.first, l);
            const int count = __builtin_amdgcn_readlane(w.r.end, l) - t.first, len = __builtin_amdgcn_readlane(w.r.length, l);
            const int most = __builtin_amdgcn_readlane(w.keys, l), parts = uniform(shares(most, per_keys));
            const int in_seq = index - before - (int)(__builtin_amdgcn_readlane((int)upto, l) - __builtin_amdgcn_readlane((int)mine, l));
            const int tile = parts == 1 ? in_seq : in_seq / parts;
            t.split = in_seq - tile * parts;
            t.slot = (int64_t)(index - t.split) * c.heads + head;
            t.row0 = tile * cut.rows;
            t.rows = min(cut.rows, count * group - t.row0);
            t.base = len - count;
            t.first_pos = t.base + quotient(t.row0, group, cut.group_recip);
            t.last_pos = t.base + quotient(t.row0 + t.rows - 1, group, cut.group_recip);
            const int high = max(0, min(min(t.last_pos + 1, len), cache_capacity(c, b)));   // keys below it are seen by some query
            const int low = window > 0 ? min(max(t.first_pos - window + 1, 0), high) : 0;
            t.keys.sinks = window > 0 ? min(sinks, low) : 0;
            t.keys.low = low;
            t.keys.count = t.keys.sinks + high - low;
            // shares of whole steps (64 keys); a tile with fewer keys than the sequence's last may have fewer shares
            const int share = parts == 1 ? 0x7FFFFFC0 : ((most + parts - 1) / parts + 63) / 64 * 64;
            t.parts = parts == 1 ? 1 : max(1, (t.keys.count + share - 1) / share);
            if (t.split >= t.parts) t.seq = -1;
            t.begin = t.split * (parts == 1 ? 0 : share);
            t.end = parts == 1 ? t.keys.count : min(t.keys.count, t.begin + share);
            return t;
        }
        before += __builtin_amdgcn_readlane((int)upto, 63);
    }
    return t;
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
// How a call of these sizes is cut, and the workgroups of its launch.
struct AttentionCut {
    WorkCut work;
    int64_t blocks;
};
AttentionCut attention_cut(int64_t n_tokens, int n_seqs, int heads, int kv_heads, int d, int64_t capacity, int window, int sinks);

// Partial results where tiles may have several shares, a place for `rows` of them for each work item of each key/value head: sums [place][d], maxima
// and weights' sums [place][2]; and for each row of the call the place of its first share's and how many shares there are.
struct RowShares {
    int32_t place, parts;
};
struct Partials {
    float *sums, *top_weight;
    RowShares *rows;
};
inline size_t partial_places(const AttentionCut &cut) { return cut.work.slots > 0 ? (size_t)cut.blocks * cut.work.rows : 0; }
inline size_t partial_bytes(const AttentionCut &cut, int64_t n_tokens, int heads, int d)
{
    return cut.work.slots > 0 ? partial_places(cut) * (d + 2) * sizeof(float) + (size_t)n_tokens * heads * sizeof(RowShares) : 0;
}
inline Partials partials_at(void *workspace, const AttentionCut &cut, int d)
{
    float *sums = (float *)workspace;
    const size_t places = partial_places(cut);
    return Partials{sums, sums + places * d, (RowShares *)(sums + places * (d + 2))};
}
hipError_t launch_cache_attention(const AttentionCall &a, const AttentionCut &cut, const Partials &partials, hipStream_t stream);
hipError_t launch_cache_few(const AttentionCall &a, const AttentionCut &cut, const Partials &partials, hipStream_t stream);     // tiles of 16 rows
hipError_t launch_cache_tiles(const AttentionCall &a, const AttentionCut &cut, const Partials &partials, hipStream_t stream);   // 64 and 128
hipError_t launch_cache_join(const AttentionCall &a, const AttentionCut &cut, const Partials &partials, hipStream_t stream);

}  // namespace sti
