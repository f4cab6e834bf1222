// The plan of a chunk.
//
// Copies and checks what the chunk's kernels read again and again: lengths,
// page ids, and for every token the cache position it goes to.  After it no
// kernel has to check an index that came from the caller, and one plan serves
// all layers of a model.
#include "ro_chunk.h"

namespace ro {

// A sequence's tokens and length, or nothing if they are invalid.
__device__ __forceinline__ ChunkSeq read_seq(const Chunk &c, const PlanArgs &a, int64_t s, int &err)
{
    const int64_t q0 = a.q_off[s], q1 = a.q_off[s + 1], L = a.kv_len[s];
    ChunkSeq r = {0, 0, 0, 0};
    if (q0 < 0 || q1 < q0 || q1 > c.n_tokens || (s == 0 && q0 != 0) || (s == c.n_seqs - 1 && q1 != c.n_tokens))
        err = RO_EINVAL;
    else if (q1 - q0 > a.max_new || L < 0 || L > c.cols << c.page_shift || (L > 0 && a.n_pages == 0) ||
             (L + (1 << c.page_shift) - 1) >> c.page_shift > a.table_stride)
        err = RO_ERANGE;
    else
        r = {(int32_t)q0, (int32_t)(q1 - q0), (int32_t)L, 0};
    return r;
}

__global__ __launch_bounds__(kBlock) void k_chunk_plan(Chunk c, PlanArgs a, Ctl *ctl)
{
    const int64_t s = blockIdx.x;
    const int64_t g = (int64_t)blockIdx.y * kBlock + threadIdx.x, step = (int64_t)gridDim.y * kBlock;
    int err = 0;
    if (s < c.n_seqs) {
        const ChunkSeq q = read_seq(c, a, s, err);
        if (blockIdx.y == 0 && threadIdx.x == 0) c.seq[s] = q;
        const int64_t np = (q.L + (1ll << c.page_shift) - 1) >> c.page_shift;
        for (int64_t i = g; i < np; i += step) {
            uint32_t id = a.table[s * a.table_stride + i];
            if (id >= a.n_pages) {
                err = RO_ERANGE;
                id = 0;
            }
            c.table[s * c.cols + i] = id;
        }
    }
    // tokens, spread over all workgroups
    const int64_t all = (int64_t)gridDim.x * step;
    for (int64_t t = s * step + g; t < c.n_tokens; t += all) {
        int64_t lo = 0, hi = c.n_seqs;          // the last sequence that starts at or before t
        while (hi - lo > 1) {
            const int64_t mid = (lo + hi) >> 1;
            if (a.q_off[mid] <= t) lo = mid;
            else hi = mid;
        }
        uint64_t slot = ~0ull;
        uint32_t of = ~0u;
        if (c.n_seqs > 0) {
            int e = 0;
            const ChunkSeq q = read_seq(c, a, lo, e);
            if (t >= q.q0 && t < (int64_t)q.q0 + q.n) {
                of = (uint32_t)lo;
                const int64_t j = (int64_t)q.L - q.n + (t - q.q0);
                if (j >= 0) {
                    const uint32_t id = a.table[lo * a.table_stride + (j >> c.page_shift)];
                    if (id < a.n_pages) slot = (uint64_t)id << 32 | (uint32_t)(j & ((1ll << c.page_shift) - 1));
                }
            }
        }
        c.slot[t] = slot;
        c.tok[t] = of;
    }
    if (err) raise_err(ctl, err);
}

hipError_t launch_chunk_plan(const Launch &L, const Chunk &c, const PlanArgs &a)
{
    const int64_t seqs = c.n_seqs > 0 ? c.n_seqs : 1;
    int64_t y = (c.cols + kBlock * 4 - 1) / (kBlock * 4), yt = (c.n_tokens / seqs + kBlock - 1) / kBlock;
    y = y > yt ? y : yt;
    y = y < 1 ? 1 : (y > 64 ? 64 : y);
    RO_LAUNCH(L, RO_K_CHUNK_PLAN, k_chunk_plan, dim3((unsigned)seqs, (unsigned)y), dim3(kBlock), 0, L.stream, c, a,
              L.ctl);
    return hipGetLastError();
}

}  // namespace ro
