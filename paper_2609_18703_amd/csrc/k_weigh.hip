// The attention that every cached position received.
//
//   w_out[j] = w_in[j] + sum over tokens i that see j, over their heads h, of
//              exp(scale q_ih . k_j - lse_ih)
//
// k_weigh: a workgroup takes 256 positions at a time, 64 to a wave.  Their
// keys stay in registers while tiles of up to 64 rows (a row: a token and a
// head of the keys' group; a tile holds whole tokens) pass through LDS.  With
// S^T = K Q^T a lane has one row and half of its keys, so the row's lse is one
// value, and every key's sum stays in a register until the end, when the
// lanes' sums are added up.  All work, position tile after position tile, is
// one line of (token, tile) pairs that is cut into equal shares, one for each
// workgroup: a tile's sums come from as many workgroups as its tokens take,
// and k_weigh_join adds them in a fixed order.
//
// k_weigh_few: single tokens, at most 16 rows a head.  The keys are the
// traffic, so they stream: a wave takes a head, or a part of the heads, of
// tiles of 64 positions, two halves in LDS, one in flight while the other is
// worked on; all rows lie in LDS from the start.  The waves' sums of a tile
// are added in LDS.
//
// Neither uses atomics: the same call gives the same bits.  All sums are held
// in 32 bits: a key's over all rows of a share in one register of k_weigh, row
// after row, which leaves two to three times the error of sums over short runs
// that are added up (1.6e-7 against 6e-8 for four chunks).
//
// Measured: k_weigh and its join 229 us, 755 TFLOP/s of the products, for four chunks of
// 257 to 2,050 tokens over 1,000 to 9,001 positions, 32 heads of 128.  Of two
// waves' 2,430 cycles a tile the products take 1,022 and the vector
// instructions, mostly one exponential, one addition and one multiply-add a
// weight, 1,540: next to nothing of the two overlaps, since a wave's products
// and its exponentials take turns and two waves a SIMD do not fill the gaps.
// The card runs at 1.87 GHz under it.  Looking for rows whose lse is far or not
// finite takes 1% of it.  k_weigh_few 45 us, 4.5
// TB/s, for 48 single tokens; by k_weigh they would take 67 us.
#include <algorithm>
#include <type_traits>

#include "ro_mfma.h"

namespace ro {

namespace {

// A weight is one multiply-add and an exponential, of scale log2(e) q.k less
// log2(e) lse, up to this size of the lse: its rounding and the product's put
// 2^-11 into the exponent there.  Beyond, the score is formed and rounded as
// the lse was, and their difference multiplied: one that makes up the whole sum
// still has a weight of one.
constexpr float kFar = 4096.0f;
__device__ __forceinline__ float below_lse(float x, float scale, float lse)
{
#pragma clang fp contract(off)
    const float score = x * scale;
    return (score - lse) * kLog2e;
}

// The last of n > 0 places whose value is at most `at`, that of place 0
// being; values rise.  All lanes at once: one round for up to 64 places.
template <typename V, typename F>
__device__ __forceinline__ int32_t last_up_to(int32_t n, V at, F value)
{
    int32_t lo = 0, hi = n;                       // value(lo) <= at, value(hi) > at
    while (hi - lo > 1) {
        const int32_t step = (hi - lo + 63) / 64, i = lo + lane_id() * step;
        const uint64_t le = __ballot(i < hi && value(i) <= at);
        const int32_t k = 63 - __builtin_clzll(le);
        lo = uni32(lo + k * step);
        hi = min(hi, lo + step);
    }
    return lo;
}

// Of two workgroups on a CU the older runs faster (2.05 and 2.6 us a tile of
// rows), and tiles with hidden positions take longer: three shares for each
// that runs at a time even that out, the last positions, where those tiles
// are, first (1, 2, 3, 4 shares: 257, 236, 232, 241 us, 244 with four shares
// of every tile).
constexpr int kShares = 3;

enum { kNone, kUpper, kBoth };                // limits to what a tile's rows see: none, the last position, a window as well

// All pairs in equal shares, none empty: the first pair of share i, and the
// share that has a pair.
struct Shares {
    int64_t all, n;
    __device__ Shares(const Chunk &c) : all(scalar_load(&c.work->weigh_cost)), n(min(all, kShares * (int64_t)c.many_slots)) {}
    __device__ int64_t start(int64_t i) const { return all * i / n; }
    __device__ int64_t of(int64_t pair) const { return ((pair + 1) * n - 1) / all; }
};

}  // namespace

template <typename T, int D>
__global__ __launch_bounds__(256, 2) void k_weigh(Chunk c, Pages pg, Rows q, const float *lse, const float *w_in,
                                                  float *w_out, int64_t w_stride, float scale, Ctl *ctl)
{
    using Load = TileLoad<D>;
    const float sc = scale * kLog2e;
    constexpr int kSteps = D / 16, kB = 2, kKeysWave = 32 * kB;
    constexpr uint32_t kTileBytes = kWeighRows * D * 2, kBuf = kTileBytes + 256;
    const int lane = lane_id(), wave = uni32(threadIdx.x >> 6), col = lane & 31, half = lane >> 5;
    const int row_in = lane / (64 / Load::kRowsAt), piece = lane % (64 / Load::kRowsAt);
    const uint32_t base = lds_base();
    const uint32_t q_at = (uint32_t)(col * D * 2 + ((half ^ Load::key_swizzle(col)) * 16));
    // a tile: as many tokens as have 64 rows at most, so that a lane's rows are
    // the same from the tile's first token on in every tile
    const int32_t tok = kWeighRows / c.group, full = tok * c.group;
    auto row_offset = [&](int n, int32_t rows) {
        const int rr = min(wave * 16 + n * Load::kRowsAt + row_in, rows - 1), i = rr / c.group;
        return (int64_t)i * q.row + (int64_t)(rr - i * c.group) * q.head +
               (piece ^ Load::key_swizzle(wave * 16 + n * Load::kRowsAt + row_in)) * 8;
    };
    auto lse_offset = [&](int32_t rows) {
        const int rr = min(lane, rows - 1), i = rr / c.group;
        return i * c.q_heads + rr - i * c.group;
    };
    int64_t q_from[Load::kLoads];
#pragma unroll
    for (int n = 0; n < Load::kLoads; ++n) q_from[n] = row_offset(n, full);
    const int32_t lse_from = lse_offset(full), token_of[2] = {col / c.group, (col + 32) / c.group};

    const Shares shares(c);
    if ((int64_t)blockIdx.x >= shares.n) return;
    const int64_t me = shares.n - 1 - blockIdx.x;
    const int64_t end = shares.start(me + 1);
    for (int64_t from = shares.start(me), next; from < end; from = next) {
        const int32_t s = last_up_to(c.n_seqs, from, [&](int32_t i) { return c.cost_off[i]; });
        const ChunkSeq sq = {uni32(c.seq[s].q0), uni32(c.seq[s].n), uni32(c.seq[s].L), 0};
        const int64_t in = from - scalar_load(c.cost_off + s);
        const int32_t tile = last_up_to((sq.L + kWeighKeys - 1) / kWeighKeys, in, [&](int32_t i) { return weigh_cost(c, sq, i); });
        const int64_t c0 = weigh_cost(c, sq, tile), c1 = weigh_cost(c, sq, tile + 1);
        const bool starts = in == c0, ends = end - from >= c1 - in;
        next = from + (c1 - in);                  // the next tile's start
        if (sq.L > w_stride) {
            if (threadIdx.x == 0) raise_err(ctl, RO_ERANGE);
            continue;
        }
        const int32_t k0 = tile * kWeighKeys, kw = k0 + wave * kKeysWave, past = sq.L - sq.n;
        // tokens that see any of the tile's positions
        int32_t ia = 0, ib = sq.n;
        if (c.causal) {
            ia = max(0, k0 - past);
            if (c.window > 0 && k0 >= c.sinks) ib = min(ib, max(0, k0 + kWeighKeys - 1 + c.window - past));
        }
        ib = max(ib, ia);
        const int32_t tiles = (ib - ia + tok - 1) / tok;
        // this share's (head, tile of rows) pairs
        const int32_t all = tiles * c.kv_heads;
        const int32_t u0 = (int32_t)((in - c0) * all / (c1 - c0));
        const int32_t u1 = ends ? all : (int32_t)((in + (end - from) - c0) * all / (c1 - c0));

        // (head, first token) to load next, and their place
        int32_t lh = tiles > 0 ? u0 / tiles : 0, lt = ia + (u0 - lh * tiles) * tok, lbuf = 0;
        auto load_next = [&] {
            const uint32_t to = base + lbuf * kBuf;
            const T *from = (const T *)q.p + (int64_t)(sq.q0 + lt) * q.row + (int64_t)(lh * c.group) * q.head;
            const float *z = lse + (int64_t)(sq.q0 + lt) * c.q_heads + lh * c.group;
            // (rows that the tile does not have repeat its last one)
            if (lt + tok <= ib) {
#pragma unroll
                for (int n = 0; n < Load::kLoads; ++n) load_to_lds(from + q_from[n], to + wave * 16 * D * 2 + n * 1024);
                if (wave == 0) load_word_to_lds(z + lse_from, to + kTileBytes);
            } else {
                const int32_t rows = (ib - lt) * c.group;
#pragma unroll
                for (int n = 0; n < Load::kLoads; ++n) load_to_lds(from + row_offset(n, rows), to + wave * 16 * D * 2 + n * 1024);
                if (wave == 0) load_word_to_lds(z + lse_offset(rows), to + kTileBytes);
            }
            lbuf ^= 1;
            if ((lt += tok) >= ib) {
                lt = ia;
                ++lh;
            }
        };

        float sum[kB][16] = {};
        tile_barrier();                           // the last unit's tiles have been read
        int32_t h = lh, t0 = lt, buf = 0;
        if (u0 < u1) load_next();
        for (int32_t u = u0; u < u1; ++h, t0 = ia) {
            Vec8<T> kf[kB][kSteps];
            const T *kp = (const T *)pg.k + (int64_t)h * pg.head;
#pragma unroll
            for (int b = 0; b < kB; ++b) {
                const T *row = kp + page_at(c, pg, s, min(kw + b * 32 + col, sq.L - 1));
#pragma unroll
                for (int k = 0; k < kSteps; ++k) kf[b][k] = *reinterpret_cast<const Vec8<T> *>(row + k * 16 + half * 8);
            }
            // (the compiler's own wait for the keys goes here, not behind the loads that follow)
#pragma unroll
            for (int b = 0; b < kB; ++b)
#pragma unroll
                for (int k = 0; k < kSteps; ++k) asm volatile("" : "+v"(kf[b][k]));
            for (; u < u1 && t0 < ib; ++u, t0 += tok, buf ^= 1) {
                tile_barrier();
                if (u + 1 < u1) load_next();
                if (kw >= sq.L) continue;
                const uint32_t qt = base + buf * kBuf;
                // do all tokens of the tile see all of the wave's positions?
                const int32_t t1 = min(t0 + tok, ib), rows = (t1 - t0) * c.group, ke = kw + kKeysWave - 1;
                const bool whole = ke < sq.L && (!c.causal || (ke <= past + t0 && (c.window <= 0 || kw >= past + t1 - c.window ||
                                                                                  ke < c.sinks)));
                // two blocks of 32 rows: the second's are read behind the
                // exponentials of the first
                auto both = [&](auto mask) {
                    constexpr int kMask = decltype(mask)::value;
                    Vec8<T> qf[2][kSteps];
                    f32x16 x[2][kB];
                    float l[2];
                    bool odd;                     // is an lse far, infinite or NaN?
                    auto read = [&](int cb) {
                        uint32_t lane_at = q_at + qt;
                        asm volatile("" : "+v"(lane_at));
#pragma unroll
                        for (int k = 0; k < kSteps; ++k) {
                            uint32_t at = lane_at ^ (k * 32);
                            asm volatile("" : "+v"(at));
                            qf[cb][k] = lds_vec<T>(at + cb * 32 * D * 2);
                        }
                        if (cb == 0)
#pragma unroll
                            for (int b = 0; b < 2; ++b)
                                l[b] = *(const __attribute__((address_space(3))) float *)(uintptr_t)(qt + kTileBytes + (b * 32 + col) * 4);
                        __builtin_amdgcn_sched_barrier(0);
                    };
                    auto multiply = [&](int cb) {
#pragma unroll
                        for (int k = 0; k < kSteps; ++k)
#pragma unroll
                            for (int b = 0; b < kB; ++b) x[cb][b] = Mma<T>::wide(kf[b][k], qf[cb][k], k ? x[cb][b] : f32x16{});
                    };
                    // (Rows that the tile does not have have a weight of zero, and repeat
                    // one that it has: they see what that sees.  What a row does not see
                    // is not added, whatever its weight comes out as: the row's lse may be
                    // NaN.  Nor is a row whose lse is -inf, whose query may be anything.)
                    auto add = [&](int cb) {
                        if (cb == 0) odd = !__all((fabsf(l[0]) <= kFar) & (fabsf(l[1]) <= kFar));
                        // this row sees the wave's keys from number lo on and up to number hi, and those below `sink`
                        int32_t first = kw + 4 * half;
                        if (kMask != kNone) asm volatile("" : "+v"(first));     // (or 64 comparisons with `sink` are kept in registers)
                        const int32_t p = c.causal ? past + min(t0 + token_of[cb], t1 - 1) : sq.L - 1;
                        const bool idle = l[cb] == -INFINITY;
                        const int32_t hi = idle ? -1 : p - first, lo = (c.window > 0 ? p - c.window : -1) - first, sink = c.sinks - first;
                        float z = cb * 32 + col >= rows ? INFINITY : l[cb] * kLog2e, k = sc;
                        if (odd) {
#pragma unroll
                            for (int b = 0; b < kB; ++b)
#pragma unroll
                                for (int e = 0; e < 16; ++e) x[cb][b][e] = below_lse(x[cb][b][e], scale, l[cb]);
                            z = fabsf(z) == INFINITY ? INFINITY : 0.0f;
                            k = 1.0f;
                        }
                        auto sums = [&](auto some) {
#pragma unroll
                            for (int b = 0; b < kB; ++b)
#pragma unroll
                                for (int e = 0; e < 16; ++e) {
                                    const int32_t n = b * 32 + 8 * (e >> 2) + (e & 3);
                                    const float w = __builtin_amdgcn_exp2f(x[cb][b][e] * k - z);
                                    const bool hidden = kMask == kNone ? idle : (n > hi) | (kMask == kBoth && (n <= lo) & (n >= sink));
                                    sum[b][e] += decltype(some)::value && hidden ? 0.0f : w;
                                }
                        };
                        if (kMask != kNone || odd) sums(std::true_type());
                        else sums(std::false_type());
                    };
                    read(0);
                    __builtin_amdgcn_s_setprio(1);
                    multiply(0);
                    __builtin_amdgcn_s_setprio(0);
                    __builtin_amdgcn_sched_barrier(0);
                    read(1);
                    add(0);
                    __builtin_amdgcn_sched_barrier(0);
                    __builtin_amdgcn_s_setprio(1);
                    multiply(1);
                    __builtin_amdgcn_s_setprio(0);
                    __builtin_amdgcn_sched_barrier(0);
                    add(1);
                    __builtin_amdgcn_sched_barrier(0);
                };
                if (whole) both(std::integral_constant<int, kNone>());
                else if (c.window <= 0) both(std::integral_constant<int, kUpper>());
                else both(std::integral_constant<int, kBoth>());
            }
        }
        // add up the lanes of each half: every step halves the keys a lane
        // holds, and a lane is left with one key of its half
        float v[16 * kB];
#pragma unroll
        for (int b = 0; b < kB; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) v[b * 16 + e] = sum[b][e];
#pragma unroll
        for (int w = 8 * kB; w; w >>= 1) {
            const bool up = lane & w;
#pragma unroll
            for (int e = 0; e < w; ++e) {
                float a = v[e], b = v[e + w];
                asm("" : "+v"(a), "+v"(b));       // values to choose from, not places
                v[e] = (up ? b : a) + __shfl_xor(up ? a : b, w, 64);
            }
        }
        const int at = wave * kKeysWave + (col >> 4) * 32 + ((col & 15) >> 2) * 8 + half * 4 + (col & 3);
        if (!starts || !ends) c.part_o[(me * 2 + starts) * kWeighKeys + at] = v[0];
        else if (k0 + at < sq.L) {
            const int64_t j = (int64_t)s * w_stride + k0 + at;
            w_out[j] = (w_in ? w_in[j] : 0.0f) + v[0];
        }
    }
}

// LDS of k_weigh_few, in bytes from the base, for `rows` rows of queries
template <int D>
struct FewPlace {
    static constexpr uint32_t kHalf = 32 * D * 2;
    uint32_t q, lse, sum, was, end;
    __host__ __device__ FewPlace(uint32_t rows)
    {
        q = 8 * kHalf;                            // after [4 waves][2] halves of keys
        lse = q + rows * D * 2;
        sum = lse + (rows + 63) / 64 * 256;       // [2][4 waves][64] sums of a tile
        was = sum + 2 * 4 * 64 * 4;               // [2][4][64] weights before
        end = was + 2 * 4 * 64 * 4;
    }
};

template <typename T, int D>
__global__ __launch_bounds__(256, 2) void k_weigh_few(Chunk c, Pages pg, Rows q, const float *lse, const float *w_in,
                                                      float *w_out, int64_t w_stride, float scale, uint32_t q_rows, Ctl *ctl)
{
    using Load = TileLoad<D>;
    constexpr int kSteps = D / 32;
    constexpr uint32_t kHalf = FewPlace<D>::kHalf;
    const WorkItem it = scalar_load(c.few_weigh + blockIdx.x);
    if ((int32_t)blockIdx.x >= scalar_load(&c.work->n_weigh)) return;
    const ChunkSeq sq = it.sq;
    if (sq.L > w_stride) {
        if (threadIdx.x == 0) raise_err(ctl, RO_ERANGE);
        return;
    }
    const FewPlace<D> place(q_rows);
    const uint32_t base = lds_base();
    const int lane = lane_id(), wave = uni32(threadIdx.x >> 6), col = lane & 15, quad = lane >> 4;
    // the waves share heads (as many as there are, up to four), then tiles
    const int hw = c.kv_heads >= 4 ? 4 : c.kv_heads >= 2 ? 2 : 1, kw = 4 / hw, hg = wave % hw, kg = wave / hw;
    const int32_t rows = sq.n * c.group, past = sq.L - sq.n, last = sq.L - 1, p0 = past, p1 = past + sq.n - 1;

    // all rows, head by head, and their lse
    const int32_t all = sq.n * c.q_heads;
    constexpr int kAt = Load::kRowsAt;
    auto source = [&](int32_t r, int32_t &t, int32_t &hq) {
        const int32_t h = r / rows, x = r - h * rows, i = x / c.group;
        t = sq.q0 + i;
        hq = h * c.group + (x - i * c.group);
    };
    for (int32_t r0 = wave * kAt; r0 < all; r0 += 4 * kAt) {
        const int32_t r = r0 + lane / (64 / kAt), piece = lane % (64 / kAt);
        int32_t t, hq;
        source(min(r, all - 1), t, hq);
        load_to_lds((const T *)q.p + (int64_t)t * q.row + (int64_t)hq * q.head + (piece ^ Load::key_swizzle(r)) * 8,
                    base + place.q + r0 * D * 2);
    }
    for (int32_t r0 = wave * 64; r0 < all; r0 += 256) {
        int32_t t, hq;
        source(min(r0 + lane, all - 1), t, hq);
        load_word_to_lds(lse + (int64_t)t * c.q_heads + hq, base + place.lse + r0 * 4);
    }

    // steps of this wave: tiles kg, kg + kw, ... that some row sees, its heads, two halves
    const Load load_rows(pg);
    const uint32_t *table = c.table + (int64_t)it.seq * c.cols;
    auto seen = [&](int32_t t) {
        const int32_t a = t * kKeys;
        return rows > 0 && (!c.causal || (a <= p1 && (c.window <= 0 || a + kKeys - 1 > p0 - c.window || a < c.sinks)));
    };
    auto page_of = [&](int32_t j) { return scalar_load(table + (min(j, last) >> c.page_shift)); };
    const uint32_t kb = base + wave * 2 * kHalf;
    int32_t nt = it.v0 + kg, nh = hg, nhalf = 0, n = 0;       // the next step to load, and how many have been
    while (nt < it.v1 && !seen(nt)) nt += kw;
    if (nh >= c.kv_heads) nt = it.v1;
    bool word = false;                                        // did the last loads bring the weights before?
    int32_t words = 0, used = 0;                              // tiles whose weights before were loaded; used, of wave's tiles
    auto load_next = [&] {
        const int32_t j0 = nt * kKeys + nhalf * 32;
        const uint32_t to = kb + (n & 1) * kHalf;
        load_rows.template load<false>(c, pg, nh, page_of(j0), j0, last, to, 0);
        load_rows.template load<false>(c, pg, nh, page_of(j0 + 16), j0 + 16, last, to + 16 * D * 2, 0);
        word = w_in && hg == 0 && nh == 0 && nhalf == 0;
        if (word)
            load_word_to_lds(w_in + (int64_t)it.seq * w_stride + min(j0 + lane, last),
                             base + place.was + (((words++ & 1) * 4 + kg) * 64) * 4);
        ++n;
        nhalf ^= 1;
        if (nhalf == 0 && (nh += hw) >= c.kv_heads) {
            nh = hg;
            do nt += kw;
            while (nt < it.v1 && !seen(nt));
        }
    };
    wait_loads<0>();
    __syncthreads();                                          // the rows are there
    if (nt < it.v1) load_next();
    int32_t done = 0;
    for (int32_t t0 = it.v0; t0 < it.v1; t0 += kw) {
        const int32_t t = t0 + kg, buf = (t0 - it.v0) / kw & 1;
        float sum[16] = {};
        if (t < it.v1 && seen(t)) {
            const int32_t a = t * kKeys;
            const bool whole = a + kKeys <= sq.L &&
                               (!c.causal || (a + kKeys - 1 <= p0 && (c.window <= 0 || a > p1 - c.window || a + kKeys <= c.sinks)));
            for (int32_t h = hg; h < c.kv_heads; h += hw) {
                const int32_t r = h * rows + min(col, rows - 1);
                const uint32_t q_at = base + place.q + r * D * 2 + ((quad ^ Load::key_swizzle(r)) * 16);
                float l = *(const __attribute__((address_space(3))) float *)(uintptr_t)(base + place.lse + r * 4);
                const bool idle = l == -INFINITY;             // adds nothing, whatever its query is
                if (col >= rows || idle) l = INFINITY;
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const uint32_t kt = kb + (done & 1) * kHalf;
                    ++done;
                    if (nt < it.v1) {
                        load_next();
                        if (word) wait_loads<2 * Load::kLoads + 1>();
                        else wait_loads<2 * Load::kLoads>();
                    } else {
                        wait_loads<0>();
                    }
                    const uint32_t k_at = kt + col * D * 2 + ((quad ^ Load::key_swizzle(col)) * 16);
                    f32x4 x[2] = {};
#pragma unroll
                    for (int s = 0; s < kSteps; ++s) {
                        const Vec8<T> qf = lds_vec<T>(q_at ^ (s * 64));
#pragma unroll
                        for (int b = 0; b < 2; ++b) x[b] = Mma<T>::narrow(lds_vec<T>((k_at ^ (s * 64)) + b * 16 * D * 2), qf, x[b]);
                    }
                    // this row sees the lane's keys from number lo on, up to hi, and below sink
                    const int32_t i = min(col, rows - 1) / c.group, first = a + half * 32 + 4 * quad;
                    const int32_t p = col >= rows ? -1 : c.causal ? past + i : last;
                    const int32_t hi = p - first, lo = (c.window > 0 ? p - c.window : -1) - first, sink = c.sinks - first;
#pragma unroll
                    for (int b = 0; b < 2; ++b)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int32_t k = b * 16 + e;
                            const float w = __builtin_amdgcn_exp2f(below_lse(x[b][e], scale, l));
                            const bool hidden = (k > hi) | ((k <= lo) & (k >= sink));
                            sum[half * 8 + b * 4 + e] += idle || (!whole && hidden) ? 0.0f : w;
                        }
                    asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");      // the half may be loaded again
                }
            }
        }
        // the lanes' sums: a lane is left with one of the quad's 16 keys
#pragma unroll
        for (int w = 8; w; w >>= 1) {
            const bool up = lane & w;
#pragma unroll
            for (int e = 0; e < w; ++e) {
                float x = sum[e], y = sum[e + w];
                asm("" : "+v"(x), "+v"(y));
                sum[e] = (up ? y : x) + __shfl_xor(up ? x : y, w, 64);
            }
        }
        auto *sums = (__attribute__((address_space(3))) float *)(uintptr_t)(base + place.sum) + buf * 256;
        sums[wave * 64 + (col >> 3) * 32 + ((col >> 2) & 1) * 16 + 4 * quad + (col & 3)] = sum[0];
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory");
        // The first wave of a tile's heads writes it.  The same wave loads its
        // weights before, so that the loads of the tile after next, to the same
        // place, are issued after this read has returned.
        const int32_t j = t * kKeys + lane;
        if (hg == 0 && t < it.v1 && j < sq.L) {
            float x = 0.0f;
            for (int g = 0; g < hw; ++g) x += sums[(kg * hw + g) * 64 + lane];
            const int64_t at = (int64_t)it.seq * w_stride + j;
            float before = 0.0f;
            if (w_in)
                before = seen(t) ? ((__attribute__((address_space(3))) float *)(uintptr_t)(base + place.was))[((used & 1) * 4 + kg) * 64 + lane]
                                    : w_in[at];
            w_out[at] = before + x;
        }
        used += t < it.v1 && seen(t);
    }
}

// Positions that nothing sees, and those of tiles that several shares have.
// A share keeps sums of at most two such: one that began before it, and one
// that goes on after it.
__global__ __launch_bounds__(kWeighKeys) void k_weigh_join(Chunk c, const float *w_in, float *w_out, int64_t w_stride,
                                                           Ctl *ctl)
{
    const int32_t n = c.work->n_weigh;
    const Shares shares(c);
    for (int32_t f = blockIdx.x; f < n; f += gridDim.x) {
        const int32_t s = last_up_to(c.n_seqs, f, [&](int32_t i) { return c.weigh_off[i]; });
        const ChunkSeq sq = c.seq[s];
        const int32_t tile = f - c.weigh_off[s], j = tile * kWeighKeys + threadIdx.x;
        if (sq.L > w_stride) {
            if (threadIdx.x == 0) raise_err(ctl, RO_ERANGE);
            continue;
        }
        const int64_t c0 = c.cost_off[s] + weigh_cost(c, sq, tile), c1 = c.cost_off[s] + weigh_cost(c, sq, tile + 1);
        float sum = 0.0f;
        if (c1 > c0) {
            const int64_t a = shares.of(c0), b = shares.of(c1 - 1);
            if (a == b) continue;
            const float *part = c.part_o + a * 2 * kWeighKeys + threadIdx.x;
            sum = part[kWeighKeys];               // its first share's, in which it begins
#pragma unroll 8
            for (int32_t i = 1; i <= (int32_t)(b - a); ++i) sum += part[i * 2 * kWeighKeys];
        }
        if (j >= sq.L) continue;
        const int64_t at = (int64_t)s * w_stride + j;
        w_out[at] = (w_in ? w_in[at] : 0.0f) + sum;
    }
}

namespace {

template <typename T, int D>
hipError_t weigh(const Launch &L, const Chunk &c, const Pages &pg, const Rows &q, const float *lse, const float *w_in,
                 float *w_out, int64_t w_stride, float scale)
{
    if (c.weigh_few) {
        const uint32_t rows = (uint32_t)((c.max_new * c.q_heads + 15) / 16 * 16);
        RO_LAUNCH(L, RO_K_CHUNK_WEIGH, (k_weigh_few<T, D>), dim3((unsigned)(c.n_seqs + c.few_slots)), dim3(256),
                  FewPlace<D>(rows).end, L.stream, c, pg, q, lse, w_in, w_out, w_stride, scale, rows, L.ctl);
        return hipGetLastError();
    }
    // the tiles are known on the device alone: a grid that does not hold them takes turns
    const int64_t tiles = c.n_seqs * (((c.cols << c.page_shift) + kWeighKeys - 1) / kWeighKeys);
    const int64_t join = std::max<int64_t>(1, std::min<int64_t>(tiles, 4 * (int64_t)c.many_slots));
    const unsigned lds_bytes = 2 * (kWeighRows * D * 2 + 256);
    RO_LAUNCH(L, RO_K_CHUNK_WEIGH, (k_weigh<T, D>), dim3((unsigned)(kShares * c.many_slots)), dim3(256), lds_bytes, L.stream, c, pg, q, lse, w_in,
              w_out, w_stride, scale, L.ctl);
    RO_LAUNCH(L, RO_K_CHUNK_JOIN, k_weigh_join, dim3((unsigned)join), dim3(kWeighKeys), 0, L.stream, c, w_in, w_out, w_stride,
              L.ctl);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_weigh(const Launch &L, const Chunk &c, const Pages &pg, const Rows &q, const float *lse,
                        const float *w_in, float *w_out, int64_t w_stride, float scale, int32_t dtype)
{
    if (dtype == RO_BF16) return c.head_dim == 128 ? weigh<__bf16, 128>(L, c, pg, q, lse, w_in, w_out, w_stride, scale)
                                                   : weigh<__bf16, 64>(L, c, pg, q, lse, w_in, w_out, w_stride, scale);
    return c.head_dim == 128 ? weigh<_Float16, 128>(L, c, pg, q, lse, w_in, w_out, w_stride, scale)
                             : weigh<_Float16, 64>(L, c, pg, q, lse, w_in, w_out, w_stride, scale);
}

}  // namespace ro
