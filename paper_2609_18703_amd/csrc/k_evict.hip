// Eviction from a paged cache by accumulated weight.
//
// k_evict_select: one workgroup per sequence finds the weight of the last
// position that is kept (a radix selection, 8 bits at a time, over keys whose
// unsigned order is the weights' order) and lists the kept positions in
// order; among equal weights the lowest positions stay.
// k_evict_move: copies the kept positions' keys and values to the
// destination pages.
#include "ro_chunk.h"

namespace ro {

constexpr int kSel = 1024;

// Unsigned order of keys = order of weights; -0 equals 0, NaN comes below all.
__device__ __forceinline__ uint32_t weight_key(float w)
{
    if (!(w == w)) return 0;
    const uint32_t b = __float_as_uint(w == 0.0f ? 0.0f : w);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// Exclusive sums of two flags over the workgroup's threads, and their totals.
__device__ __forceinline__ int2 scan2(bool a, bool b, int2 *s_wave, int2 &total)
{
    const uint64_t ma = __ballot(a), mb = __ballot(b);
    const int lane = lane_id(), wave = threadIdx.x >> 6;
    const uint64_t below = (1ull << lane) - 1;
    if (lane == 0) s_wave[wave] = make_int2(__popcll(ma), __popcll(mb));
    __syncthreads();
    int2 r = make_int2(__popcll(ma & below), __popcll(mb & below));
    total = make_int2(0, 0);
    for (int w = 0; w < kSel / 64; ++w) {
        const int2 v = s_wave[w];
        if (w < wave) r = make_int2(r.x + v.x, r.y + v.y);
        total = make_int2(total.x + v.x, total.y + v.y);
    }
    __syncthreads();
    return r;
}

__global__ __launch_bounds__(kSel) void k_evict_select(Chunk c, EvictArgs a, Ctl *ctl)
{
    __shared__ uint32_t hist[256];
    __shared__ uint32_t s_digit, s_need;
    __shared__ int2 s_wave[kSel / 64];
    const int32_t s = blockIdx.x, tid = threadIdx.x;
    const ChunkSeq sq = c.seq[s];
    const int64_t base = (int64_t)s * a.budget;
    if (sq.L > a.w_stride) {
        if (tid == 0) {
            raise_err(ctl, RO_ERANGE);
            a.new_len[s] = 0;
        }
        for (int32_t r = tid; r < a.budget; r += kSel) a.index[base + r] = -1;
        return;
    }
    const float *w = a.weight + (int64_t)s * a.w_stride;
    const int32_t kept = sq.L < a.budget ? sq.L : a.budget;
    const bool all = sq.L <= a.budget;
    const int32_t lo = a.first, hi = sq.L - a.last;      // the positions that compete, if not all are kept
    uint32_t key = 0, need = all ? 0 : (uint32_t)(a.budget - a.first - a.last);
    if (!all && need > 0) {
        for (int shift = 24; shift >= 0; shift -= 8) {
            for (int i = tid; i < 256; i += kSel) hist[i] = 0;
            __syncthreads();
            for (int32_t j = lo + tid; j < hi; j += kSel) {
                const uint32_t k = weight_key(w[j]);
                if (shift == 24 || (k >> (shift + 8)) == (key >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255], 1u);
            }
            __syncthreads();
            if (tid == 0) {
                uint32_t left = need;
                int d = 255;
                while (d > 0 && hist[d] < left) left -= hist[d--];
                s_digit = (uint32_t)d;
                s_need = left;
            }
            __syncthreads();
            key |= s_digit << shift;
            need = s_need;                               // still wanted among the keys with this prefix
            __syncthreads();
        }
    }
    // all keys above `key` stay, and the first `need` that equal it
    int2 run = make_int2(0, 0);
    for (int32_t j0 = 0; j0 < sq.L; j0 += kSel) {
        const int32_t j = j0 + tid;
        bool stay = false, tie = false;
        float x = 0.0f;
        if (j < sq.L) {
            x = w[j];
            stay = all || j < lo || j >= hi;
            if (!stay && a.budget > a.first + a.last) {
                const uint32_t k = weight_key(x);
                stay = k > key;
                tie = k == key;
            }
        }
        int2 total;
        const int2 t = scan2(false, tie, s_wave, total);
        stay = stay || (tie && (uint32_t)(run.y + t.y) < need);
        run.y += total.y;
        const int2 e = scan2(stay, false, s_wave, total);
        if (stay) {
            const int64_t at = base + run.x + e.x;
            a.index[at] = j;
            if (a.new_weight) a.new_weight[at] = x;
        }
        run.x += total.x;
    }
    for (int32_t r = kept + tid; r < a.budget; r += kSel) a.index[base + r] = -1;
    if (tid == 0) a.new_len[s] = kept;
}

__global__ __launch_bounds__(kBlock) void k_evict_move(Chunk c, Pages pg, EvictArgs a, Ctl *ctl)
{
    const int32_t s = blockIdx.x, units = c.head_dim / 8;
    const ChunkSeq sq = c.seq[s];
    if (sq.L > a.w_stride) return;
    const int64_t kept = sq.L < a.budget ? sq.L : a.budget, per = 2ll * c.kv_heads * units;
    const int64_t np = (kept + (1ll << c.page_shift) - 1) >> c.page_shift;
    if (np > a.dst_stride) {
        if (blockIdx.y == 0 && threadIdx.x == 0) raise_err(ctl, RO_ERANGE);
        return;
    }
    for (int64_t i = (int64_t)blockIdx.y * kBlock + threadIdx.x; i < kept * per; i += (int64_t)gridDim.y * kBlock) {
        const int32_t r = (int32_t)(i / per), x = (int32_t)(i % per), u = x % units, h = x / units;
        const int32_t j = a.index[(int64_t)s * a.budget + r];
        const uint32_t page = a.dst[(int64_t)s * a.dst_stride + (r >> c.page_shift)];
        if (page >= a.n_pages) {
            raise_err(ctl, RO_ERANGE);
            continue;
        }
        const bool is_k = h < c.kv_heads;
        uint4 *p = (uint4 *)(is_k ? pg.k : pg.v);
        const int64_t head = (is_k ? h : h - c.kv_heads) * pg.head;
        const int64_t to = (int64_t)page * pg.page + (int64_t)(r & ((1 << c.page_shift) - 1)) * pg.slot;
        p[(to + head) / 8 + u] = p[(page_at(c, pg, s, j) + head) / 8 + u];
    }
}

hipError_t launch_evict(const Launch &L, const Chunk &c, const Pages &pg, const EvictArgs &a)
{
    RO_LAUNCH(L, RO_K_CHUNK_EVICT, k_evict_select, dim3((unsigned)c.n_seqs), dim3(kSel), 0, L.stream, c, a, L.ctl);
    if (hipError_t e = hipGetLastError()) return e;
    RO_LAUNCH(L, RO_K_CHUNK_MOVE, k_evict_move, dim3((unsigned)c.n_seqs, 256), dim3(kBlock), 0, L.stream, c, pg, a,
              L.ctl);
    return hipGetLastError();
}

}  // namespace ro
