// Eviction from a paged cache by accumulated weight.
//
// k_evict_select: one workgroup per sequence finds the weight of the last
// position that is kept, by a radix selection over keys whose unsigned order
// is the weights' order, 11 bits at a time, and lists the kept positions in
// order; among equal weights the lowest positions stay.  Every wave owns a
// run of positions, whose keys stay in registers up to 32,768 positions, so
// that the list needs the waves' counts once and no barrier in between.
// It waits for one pass over the weights after the other: 6.9 us for 1,200
// positions a sequence, 26 us for 32,768.  (Each weight read behind a test of
// its own, so that a lane waited for every one: 37 us.)
//
// k_evict_move: copies the kept positions' keys, values and weights, four
// rows of a wave in flight at a time.  Bound by memory: 381 us, 5.2 TB/s read
// and written, for 16 caches of 16,384 positions that stay.
#include "ro_mfma.h"

namespace ro {

namespace {

constexpr int kSel = 1024, kWaves = kSel / 64;
constexpr int kBins = 2048;

// Unsigned order of keys = order of weights; -0 equals 0, NaN comes below all.
// 0 is no weight's key, nor is kStays.
constexpr uint32_t kStays = 0xffffffffu;
__device__ __forceinline__ uint32_t weight_key(float w)
{
    if (!(w == w)) return 1;
    const uint32_t b = __float_as_uint(w == 0.0f ? 0.0f : w);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// Of bins whose higher ones come first: the bin in which the count reaches
// `need`, and what is still needed in it.
__device__ __forceinline__ uint2 find_bin(const uint32_t *hist, uint32_t need, uint32_t *s_wave, uint2 *s_found)
{
    const int tid = threadIdx.x, wave = tid >> 6;
    const uint32_t hi = hist[kBins - 1 - 2 * tid], lo = hist[kBins - 2 - 2 * tid];
    const uint32_t in = wave_incl_sum(hi + lo);
    if (lane_id() == 63) s_wave[wave] = in;
    __syncthreads();
    uint32_t before = in - hi - lo;
    for (int w = 0; w < wave; ++w) before += s_wave[w];
    if (before < need && need <= before + hi) *s_found = make_uint2(kBins - 1 - 2 * tid, need - before);
    else if (before + hi < need && need <= before + hi + lo) *s_found = make_uint2(kBins - 2 - 2 * tid, need - before - hi);
    __syncthreads();
    return *s_found;
}

}  // namespace

// kPer: rounds of 64 positions a wave that are held in registers; 0: any
// number, read again for every use.  (As many as the sequence needs: nine
// sequences of up to 1,203 positions are selected from in 15.5 us with 32 for
// all, 12.6 with 0, 6.8 so; 16 of up to 32,768 in 26 with 32, 41 with 0.)
template <int kPer>
__device__ __forceinline__ void select(const ChunkSeq &sq, const EvictArgs &a, const float *w, int64_t base, uint32_t *hist,
                                       uint32_t *s_wave, uint2 *s_found)
{
    const int tid = threadIdx.x, lane = lane_id(), wave = uni32(tid >> 6);
    const bool all = sq.L <= a.budget;
    const int32_t lo = a.first, hi = sq.L - a.last;                  // the positions that compete, if not all are kept
    const int32_t rounds = kPer ? kPer : ((sq.L + 63) / 64 + kWaves - 1) / kWaves, from = wave * rounds * 64 + lane;
    // one value says all of a position: its weight's key if it competes, 0 if
    // there is none, kStays if it stays in any case
    auto key_of = [&](int32_t i, float x) -> uint32_t {
        const int32_t j = from + i * 64;
        if (j >= sq.L || i >= rounds) return 0;
        return all || j < lo || j >= hi ? kStays : weight_key(x);
    };
    // kRead loads of a lane are in flight at a time: each reads some position, needed or not
    constexpr int kRead = kPer ? kPer : 8;
    uint32_t held[kRead];
    auto read = [&](int32_t i0) {
        float x[kRead];
#pragma unroll
        for (int i = 0; i < kRead; ++i) x[i] = w[min(from + (i0 + i) * 64, sq.L - 1)];
#pragma unroll
        for (int i = 0; i < kRead; ++i) held[i] = key_of(i0 + i, x[i]);
    };
    if (kPer) read(0);
    auto each = [&](auto f) {
        for (int32_t i0 = 0; i0 < rounds; i0 += kRead) {
            if (!kPer) read(i0);
#pragma unroll
            for (int i = 0; i < kRead; ++i) f(i0 + i, held[i]);
        }
    };

    uint32_t key = kStays - 1, need = all ? 0 : (uint32_t)(a.budget - a.first - a.last);
    if (need > 0) {
        key = 0;
#pragma unroll
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
            hist[tid] = 0;
            hist[tid + kSel] = 0;
            __syncthreads();
            each([&](int32_t, uint32_t k) {
                if (k - 1 < kStays - 1 && (pass == 0 || k >> (shift + bits) == key >> (shift + bits)))
                    atomicAdd(&hist[k >> shift & ((1 << bits) - 1)], 1u);
            });
            __syncthreads();
            const uint2 f = find_bin(hist, need, s_wave, s_found);
            key |= f.x << shift;
            need = f.y;                                              // still wanted among the keys with this prefix
            __syncthreads();
        }
    }
    // what stays: keys above `key`, and the first `need` that equal it
    int32_t n_above = 0, n_equal = 0;
    each([&](int32_t, uint32_t k) {
        n_above += __popcll(__ballot(k > key));
        n_equal += __popcll(__ballot(k == key));
    });
    __shared__ int2 s_count[kWaves];
    if (lane == 0) s_count[wave] = make_int2(n_above, n_equal);
    __syncthreads();
    int32_t at = 0, ties = 0;                                        // of the waves before
    for (int v = 0; v < wave; ++v) {
        const int2 n = s_count[v];
        at += n.x;
        ties += n.y;
    }
    at += min(ties, (int32_t)need);
    int32_t left = max(0, (int32_t)need - ties);                     // of this wave's ties, how many stay
    const uint64_t below = (1ull << lane) - 1;
    each([&](int32_t i, uint32_t k) {
        bool stay = k > key;
        if (left > 0) {
            const uint64_t eq = __ballot(k == key);
            stay = stay || (k == key && (int32_t)__popcll(eq & below) < left);
            left -= min(left, (int32_t)__popcll(eq));
        }
        const uint64_t m = __ballot(stay);
        if (stay) a.index[base + at + __popcll(m & below)] = from + i * 64;
        at += __popcll(m);
    });
}

__global__ __launch_bounds__(kSel) void k_evict_select(Chunk c, EvictArgs a, Ctl *ctl)
{
    __shared__ uint32_t hist[kBins], s_wave[kWaves];
    __shared__ uint2 s_found;
    const int32_t s = blockIdx.x, tid = threadIdx.x;
    const ChunkSeq sq = c.seq[s];
    const int64_t base = (int64_t)s * a.budget;
    const bool bad = sq.L > a.w_stride;
    const int32_t kept = bad ? 0 : min(sq.L, a.budget);
    if (bad && tid == 0) raise_err(ctl, RO_ERANGE);
    for (int32_t r = kept + tid; r < a.budget; r += kSel) a.index[base + r] = -1;
    if (tid == 0) a.new_len[s] = kept;
    if (kept == 0) return;
    const float *w = a.weight + (int64_t)s * a.w_stride;
    if (sq.L <= 2 * kSel) select<2>(sq, a, w, base, hist, s_wave, &s_found);
    else if (sq.L <= 8 * kSel) select<8>(sq, a, w, base, hist, s_wave, &s_found);
    else if (sq.L <= 32 * kSel) select<32>(sq, a, w, base, hist, s_wave, &s_found);
    else select<0>(sq, a, w, base, hist, s_wave, &s_found);
}

constexpr int kMoveRows = 4;         // rows of a wave at a time

__global__ __launch_bounds__(kBlock) void k_evict_move(Chunk c, Pages pg, EvictArgs a, Ctl *ctl)
{
    const int32_t s = blockIdx.x, lane = lane_id(), wave = uni32(threadIdx.x >> 6);
    const int32_t L = scalar_load(&c.seq[s].L);
    if (L > a.w_stride) return;
    const int32_t kept = min(L, a.budget), mask = (1 << c.page_shift) - 1;
    if ((kept + (int64_t)mask) >> c.page_shift > a.dst_stride) {
        if (blockIdx.y == 0 && threadIdx.x == 0) raise_err(ctl, RO_ERANGE);
        return;
    }
    const int ushift = c.head_dim == 128 ? 4 : 3;                    // 16-byte pieces of a head
    const int32_t half = c.kv_heads << ushift;                       // of a position's keys, and of its values
    const int32_t *index = a.index + (int64_t)s * a.budget;
    const uint32_t *src = c.table + (int64_t)s * c.cols, *dst = a.dst + (int64_t)s * a.dst_stride;
    for (int32_t r0 = (blockIdx.y * 4 + wave) * kMoveRows; r0 < kept; r0 += gridDim.y * 4 * kMoveRows) {
        int64_t from[kMoveRows], to[kMoveRows];
        bool ok[kMoveRows];
#pragma unroll
        for (int n = 0; n < kMoveRows; ++n) {
            const int32_t r = min(r0 + n, kept - 1), j = index[r];
            const uint32_t page = dst[r >> c.page_shift];
            ok[n] = r0 + n < kept && page < a.n_pages;
            if (page >= a.n_pages) raise_err(ctl, RO_ERANGE);
            from[n] = (int64_t)src[j >> c.page_shift] * pg.page + (int64_t)(j & mask) * pg.slot;
            to[n] = (int64_t)(ok[n] ? page : 0) * pg.page + (int64_t)(r & mask) * pg.slot;
        }
        if (a.new_weight && lane < kMoveRows && r0 + lane < kept)
            a.new_weight[(int64_t)s * a.budget + r0 + lane] = a.weight[(int64_t)s * a.w_stride + index[r0 + lane]];
        for (int32_t p = lane; p < 2 * half; p += 64) {
            const int32_t q = p < half ? p : p - half;
            const int64_t at = (int64_t)(q >> ushift) * pg.head + (q & ((1 << ushift) - 1)) * 8;
            uint16_t *base = (uint16_t *)(p < half ? pg.k : pg.v) + at;
            u32x4 x[kMoveRows];
#pragma unroll
            for (int n = 0; n < kMoveRows; ++n) x[n] = *reinterpret_cast<const u32x4 *>(base + from[n]);
#pragma unroll
            for (int n = 0; n < kMoveRows; ++n)
                if (ok[n]) *reinterpret_cast<u32x4 *>(base + to[n]) = x[n];
        }
    }
}

hipError_t launch_evict(const Launch &L, const Chunk &c, const Pages &pg, const EvictArgs &a)
{
    RO_LAUNCH(L, RO_K_CHUNK_EVICT, k_evict_select, dim3((unsigned)c.n_seqs), dim3(kSel), 0, L.stream, c, a, L.ctl);
    if (hipError_t e = hipGetLastError()) return e;
    const int64_t most = a.budget < c.cols << c.page_shift ? a.budget : c.cols << c.page_shift;
    int64_t y = (most + 4 * kMoveRows - 1) / (4 * kMoveRows);
    y = y < 1 ? 1 : (y > 65535 ? 65535 : y);
    RO_LAUNCH(L, RO_K_CHUNK_MOVE, k_evict_move, dim3((unsigned)c.n_seqs, (unsigned)y), dim3(kBlock), 0, L.stream, c, pg, a,
              L.ctl);
    return hipGetLastError();
}

}  // namespace ro
