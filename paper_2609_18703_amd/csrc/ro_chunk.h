// Shared by the kernels of a model stage's attention: the plan of a chunk,
// 16-bit float types, page addressing and visibility.
#pragma once

#include "ro_device.h"

namespace ro {

struct ChunkSeq {
    int32_t q0, n, L, pad;   // first token, new tokens, cached positions (0, 0, 0 if the sequence is invalid)
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

// Does a token at position p see position j (of those below L)?
__device__ __forceinline__ bool sees(const Chunk &c, int32_t p, int32_t j)
{
    if (!c.causal) return true;
    return j <= p && (c.window <= 0 || j > p - c.window || j < c.sinks);
}

__device__ __forceinline__ int64_t page_at(const Chunk &c, const Pages &pg, int32_t s, int32_t j)
{
    const uint32_t page = c.table[(int64_t)s * c.cols + (j >> c.page_shift)];
    return (int64_t)page * pg.page + (int64_t)(j & ((1 << c.page_shift) - 1)) * pg.slot;
}
#endif

}  // namespace ro
