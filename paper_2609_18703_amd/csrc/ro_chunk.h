// Shared by the kernels of a model stage's attention: the plan of a chunk,
// 16-bit float types, page addressing and visibility.
#pragma once

#include "ro_device.h"

namespace ro {

// ---- work lists ------------------------------------------------------------------
// The rows of a sequence for one key / value head are its (token, head of the
// group) pairs, token by token: row r is token r / group, head r % group.  An
// item is a tile of rows and a range of the key tiles they see.
constexpr int kKeys = 64;            // positions of a key tile
constexpr int kFewRows = 16;         // rows of a narrow tile, which is a short sequence whole ...
constexpr int kManyRows = 128;       // ... others are cut into wide ones
constexpr int kFewCut = 4;           // key tiles that an item has at least: one for each wave where the rows are few ...
constexpr int kManyCut = 8;          // ... more where they are many
constexpr int kWeighCut = 2;         // the same for items of weights, where rows are few
constexpr int kMaxGroup = 64;        // a token's rows fit a tile of weights
constexpr int kWeighKeys = 256;      // positions that a workgroup adds up weights of, where rows are many
constexpr int kWeighRows = 64;       // rows of a tile there

struct ChunkSeq {
    int32_t q0, n, L;        // first token, new tokens, cached positions (0, 0, 0 if the sequence is invalid)
    int32_t bad;             // 1: invalid because of its offsets
};
struct WorkItem {
    ChunkSeq sq;
    int32_t seq, row0;
    int32_t v0, v1;          // key tiles, counted over those that the rows see
    int32_t part;            // where its partial sums go, in blocks of kFewRows rows; -1: the item is all its rows need
    int32_t part0, parts;    // where those of its rows' first item go, and how many items share them
    int32_t count;           // counts the items that are done, for key / value head 0
};
struct WorkHead {
    int32_t n_few, n_many;
    int32_t n_weigh;         // tiles of kWeighKeys positions of all sequences, or items of few_weigh
    int32_t pad;
    int64_t weigh_cost;      // (token, tile) pairs of all those tiles
};

// A planned chunk, as the kernels see it.  Everything it points to is the
// plan's own memory, checked by the plan: q0 + n <= n_tokens, page ids below
// the planned caches' page count.
struct Chunk {
    ChunkSeq *seq;           // [n_seqs]
    uint32_t *table;         // [n_seqs * cols] page ids of the positions below L
    int64_t cols;
    uint64_t *slot;          // [n_tokens] page << 32 | slot of the token's own position, ~0 if it has none
    uint32_t *tok;           // [n_tokens] the token's sequence, ~0 if it has none
    int32_t n_seqs, n_tokens;
    int32_t q_heads, kv_heads, group, head_dim;
    int32_t page_shift;
    int32_t causal, window, sinks;
    WorkHead *work;
    WorkItem *few, *many;    // [few_cap], [many_cap]
    WorkItem *few_weigh;     // [few_cap] sequences of few rows where weights are added up: v0, v1 are their key tiles
    uint32_t *count;         // [count_cap] items done of rows that several share; 0 between calls
    int32_t *tile_off;       // [n_seqs] first wide tile of every sequence
    int32_t *weigh_off;      // [n_seqs] first of its tiles of positions, and ...
    int64_t *cost_off;       // [n_seqs] ... (token, tile) pairs of the sequences before it
    int64_t few_cap, many_cap, part_cap, count_cap;
    float *part_o;           // [part_cap * kFewRows * 128] sums of p v, and ...
    float2 *part_ml;         // [part_cap * kFewRows] ... maximum and sum of p, per row
    int32_t few_slots, many_slots;   // how many items the work is cut into where there is less
    int32_t max_new;                 // no sequence has more new tokens
    int32_t few_rows;                // a sequence with no more rows than this is one narrow tile: kFewRows, or 0 for none
    int32_t weigh_few;       // weights are added up item by item of few_weigh
};

struct Rows {                // [tokens, heads, head_dim], strides in elements
    void *p;
    int64_t row, head;
};

struct Pages {
    void *k, *v;
    int64_t page, head, slot;
};

struct RotaryArgs {
    const float *freq;
    const int32_t *pos;
    int64_t pos_stride;
    int32_t rot, adjacent;
    uint8_t axis[RO_MAX_ROT / 2];
};

// ---- launchers ---------------------------------------------------------------
hipError_t launch_rope(const Launch &L, const RotaryArgs &r, const Rows &x, const Rows &y, int64_t T, int32_t heads,
                       int32_t D, int32_t dtype, int32_t inverse);
struct PlanArgs {
    const int64_t *q_off;
    const int32_t *kv_len;
    const uint32_t *table;
    int64_t table_stride, n_pages, max_new;
};
hipError_t launch_chunk_plan(const Launch &L, const Chunk &c, const PlanArgs &a);
// r null: no rotation; q.p null: keys and values only
hipError_t launch_append(const Launch &L, const Chunk &c, const Pages &pg, const RotaryArgs *r, const Rows &q,
                         const Rows &k, const Rows &v, const Rows &qo, int32_t dtype);
hipError_t launch_attend(const Launch &L, const Chunk &c, const Pages &pg, const Rows &q, const Rows &out, float *lse,
                         float scale, int32_t dtype);
hipError_t launch_weigh(const Launch &L, const Chunk &c, const Pages &pg, const Rows &q, const float *lse,
                        const float *w_in, float *w_out, int64_t w_stride, float scale, int32_t dtype);
struct EvictArgs {
    const float *weight;
    int64_t w_stride;
    const uint32_t *dst;
    int64_t dst_stride, n_pages;
    int32_t budget, first, last;
    int32_t *new_len, *index;
    float *new_weight;
};
hipError_t launch_evict(const Launch &L, const Chunk &c, const Pages &pg, const EvictArgs &a);

// ---- device side ----------------------------------------------------------------
#ifdef __HIPCC__
using f32x4 = float __attribute__((ext_vector_type(4)));
using f32x16 = float __attribute__((ext_vector_type(16)));
template <typename T>
using Vec8 = T __attribute__((ext_vector_type(8)));
template <typename T>
using Vec4 = T __attribute__((ext_vector_type(4)));

// The key tiles that rows [row0, row0 + rows) of a sequence see: `sink` tiles
// from position 0, then from tile `main` on, `all` in total.
struct Span {
    int32_t p0, p1;          // positions of the first and the last token
    int32_t sink, main, all;
};
__device__ __forceinline__ Span span_of(const Chunk &c, const ChunkSeq &s, int32_t row0, int32_t rows)
{
    Span r;
    const int32_t i0 = row0 / c.group, i1 = min((row0 + rows - 1) / c.group, s.n - 1);
    r.p0 = s.L - s.n + i0;
    r.p1 = s.L - s.n + i1;
    const int32_t hi = c.causal ? max(0, r.p1 + 1) : s.L;
    const int32_t lo = c.window > 0 ? max(0, r.p0 - c.window + 1) : 0;
    r.main = lo / kKeys;
    r.sink = c.window > 0 ? min((min(c.sinks, hi) + kKeys - 1) / kKeys, r.main) : 0;
    r.all = r.sink + (hi > lo ? (hi + kKeys - 1) / kKeys - r.main : 0);
    return r;
}
__device__ __forceinline__ int32_t key_tile(const Span &r, int32_t v) { return v < r.sink ? v : r.main + v - r.sink; }

// Do all tokens of the span see all positions of key tile t?
__device__ __forceinline__ bool tile_whole(const Chunk &c, const Span &r, int32_t L, int32_t t)
{
    const int32_t a = t * kKeys, b = a + kKeys - 1;
    if (b >= L) return false;
    if (!c.causal) return true;
    return b <= r.p0 && (c.window <= 0 || a > r.p1 - c.window || b < c.sinks);
}

// Sum over i < x of kWeighKeys i + a, held to [0, n].
__device__ __forceinline__ int64_t held_sum(int64_t a, int64_t n, int64_t x)
{
    if (n <= 0) return 0;
    const int64_t i1 = min(x, a > 0 ? (int64_t)0 : -a / kWeighKeys + 1);                          // the first above 0 ...
    const int64_t i2 = min(x, a >= n ? (int64_t)0 : (n - a + kWeighKeys - 1) / kWeighKeys);       // ... and at n
    return kWeighKeys / 2 * (i2 * (i2 - 1) - i1 * (i1 - 1)) + a * (i2 - i1) + (x - i2) * n;
}

// How many tokens see something of a sequence's tile of kWeighKeys positions,
// summed over its first x tiles: what adding up their weights costs.
__device__ __forceinline__ int64_t weigh_cost(const Chunk &c, const ChunkSeq &s, int64_t x)
{
    const int64_t n = s.n, past = (int64_t)s.L - n;
    if (!c.causal) return x * n;
    int64_t below = x * n;                        // tokens before the end of who sees a tile
    if (c.window > 0) {
        const int64_t m = min(x, ((int64_t)c.sinks + kWeighKeys - 1) / kWeighKeys), a = kWeighKeys - 1 + (int64_t)c.window - past;
        below = m * n + held_sum(a, n, x) - held_sum(a, n, m);
    }
    return below - held_sum(-past, n, x);         // ... less those before its start
}

__device__ __forceinline__ int64_t page_at(const Chunk &c, const Pages &pg, int32_t s, int32_t j)
{
    const uint32_t page = c.table[(int64_t)s * c.cols + (j >> c.page_shift)];
    return (int64_t)page * pg.page + (int64_t)(j & ((1 << c.page_shift) - 1)) * pg.slot;
}
#endif

}  // namespace ro
