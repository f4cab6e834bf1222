// Shared by the kernels of a model stage's step around its attention:
// projections in 8-bit integers, the choice of tokens, pages of a pool.
#pragma once

#include "ro_device.h"

namespace ro {

hipError_t launch_quantize(const Launch &L, const void *x, int64_t x_stride, int64_t n, int64_t dim, int32_t dtype,
                           int8_t *q, int64_t q_stride, float *scale);

struct Product {
    const int8_t *a, *w;         // [m, k] and [n, k]
    int64_t a_stride, w_stride;  // bytes
    const float *a_scale, *w_scale, *bias;
    void *out;
    int64_t out_stride;          // elements
    int64_t m, n;
    int32_t k;
};
hipError_t launch_project(const Launch &L, const Product &p, int32_t dtype);

struct SampleArgs {
    const void *logits;
    int64_t stride;
    int32_t vocab;
    const float *temperature;
    const int32_t *top_k;
    const float *top_p, *min_p;
    const uint32_t *mask;
    int64_t mask_stride;
    const float *u;
    int32_t *token;
    float *logprob;
};
// A part of a row that a workgroup has counted.
struct SampleSlice {
    uint64_t groups;             // of 512 counters: a bit where any is not 0, and they are in memory
    int32_t most, pad;           // its largest key
};
struct SampleSplit {
    SampleSlice *at;             // [rows * slices]
    uint32_t *counters;          // [rows * slices * 32768]
    int32_t slices, pieces;      // of a row; of a slice
};
// How many slices a row is cut into; 1: none.
int32_t sample_slices(int32_t num_cus, int64_t n, int32_t vocab);
hipError_t launch_sample(const Launch &L, const SampleArgs &a, int64_t n, int32_t dtype, SampleSplit split);

// ---- pages ---------------------------------------------------------------------
constexpr int kPageTile = 4096;      // pages whose free ones are counted together: 64 words of 64
constexpr int kSeqTile = 256;        // sequences whose needs are
constexpr int kMaxTables = 16;       // tables of a launch
constexpr int kMaxCaches = 64;       // caches of a launch

struct Tables {
    uint32_t *table;
    int64_t stride;
    int32_t *len;
    int64_t n;
};

// A pool as the kernels see it: the caller's counts, and words that only live
// during a call.
struct Pool {
    int32_t *refs;
    int32_t n_pages, page_shift;
    uint64_t *free;              // [tiles * 64] a bit for every free page
    uint32_t *tile_free;         // [tiles] ... their number
    uint32_t *before;            // [tiles * 64] pages in use before a word
    uint32_t *need;              // [max_seqs] pages that a sequence takes << 2 | kReplace | kLeave
    uint64_t *tile_need;         // [seq tiles] ... their sum
};

hipError_t launch_pages_fork(const Launch &L, const Pool &p, const Tables &from, const int32_t *parent, const Tables &to);
hipError_t launch_pages_grow(const Launch &L, const Pool &p, const Tables &t, const int32_t *add, uint32_t *src,
                             uint32_t *dst, int32_t *slots, int64_t *n_free);
hipError_t launch_pages_release(const Launch &L, const Pool &p, const Tables &t, const int32_t *keep);
hipError_t launch_pages_compact(const Launch &L, const Pool &p, const Tables *tables, int32_t n_tables, uint32_t *src,
                                uint32_t *dst, int64_t *n_moves, int64_t *n_free);

// Caches of one geometry.
struct CopyArgs {
    uint16_t *at[2 * kMaxCaches];    // keys and values in turn
    int64_t page, head, slot;        // strides in elements
    int64_t n_pages, n;
    int32_t n_arrays, heads, page_size, head_dim;
    const uint32_t *src, *dst;
    const int32_t *slots;
    const int64_t *n_dev;
};
hipError_t launch_pages_copy(const Launch &L, const CopyArgs &a);

}  // namespace ro
