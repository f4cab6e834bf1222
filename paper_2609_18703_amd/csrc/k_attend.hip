// Attention of a chunk's tokens over a paged cache.
//
//   o = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale q.k_j - m),
//
// over the positions a token sees, in one pass with a running maximum m.  The
// rows of an item are the (token, head) pairs of one sequence that share a
// key / value head, so that a key tile in LDS serves all of them.
//
// Both kernels work on transposed products: S^T = K Q^T has a row of the
// attention in a lane (and its partners that hold the other keys), so the
// softmax needs no exchange but one with the partners for the maximum, and
// the lane's registers of S^T, rounded, are the operand of O^T = V^T P^T as
// they are: the order of keys in that product is free, and V^T is read from
// LDS, transposed by the read, in the order the registers have.
//
// Sums, maxima and outputs are held in 32 bits.  p is rounded to the cache's
// type, which the matrix instructions need: an error of half a unit in the
// last place of each weight, as large as that of the rounded output.
#include <algorithm>
#include <cfloat>
#include <type_traits>

#include "ro_mfma.h"

namespace ro {

namespace {

// Part 0: v with what is not finite replaced by zero.  Parts 1 and 2: one
// where v is +inf or NaN, one where it is -inf or NaN, zero elsewhere.
template <typename T, int kPart>
__device__ __forceinline__ Vec8<T> wild_part(Vec8<T> v)
{
    Vec8<T> y;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float x = (float)v[e];
        const bool fine = x - x == 0.0f;
        if (kPart == 0) y[e] = fine ? v[e] : (T)0.0f;
        else y[e] = (T)(fine || (kPart == 1 ? x < 0.0f : x > 0.0f) ? 0.0f : 1.0f);
    }
    return y;
}

// Eight flags as ones and zeros.
template <typename T>
__device__ __forceinline__ Vec8<T> ones(uint32_t bits)
{
    Vec8<T> y;
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = (T)(float)(bits >> e & 1);
    return y;
}

// Sums taken against another reference.  An infinity is one value's, whatever
// its weight: with kApart it stays where the factor is too small for its type,
// without it becomes a NaN there.
template <bool kApart>
__device__ __forceinline__ f32x4 scaled(f32x4 y, float a)
{
    if (!kApart) return y * a;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = fabsf(y[e]) == INFINITY ? y[e] : y[e] * a;
    return y;
}
__device__ __forceinline__ bool not_a_number(f32x4 y)
{
    return y[0] != y[0] || y[1] != y[1] || y[2] != y[2] || y[3] != y[3];
}

// A maximum that rises by less than this (a factor 2^8 of the weights) does
// not move the reference: the sums need no rescaling, and the weights stay
// below 2^8, far within every type's range and at the same relative precision.
constexpr float kSlack = 8.0f;
// The same, told by a lane's sum of 32 weights: no weight is larger.
constexpr float kOutgrown = 8192.0f;
// The reference is the row's maximum m before the scale.  Up to this size of
// scale * m the weights are formed by one multiply-add less the
// rounded scale * m, which leaves half a unit of its last place, 2^-12, in the
// exponent, as much as the rounding of a score of that size.  Beyond, where the
// rounding alone could be many powers of two, m is taken off the scores first.
constexpr float kFar = 4096.0f;

}  // namespace

// ---- joining what was cut ------------------------------------------------------------
//
// An item that has part of its rows' keys leaves its sums in memory.  The
// last one of the rows to do so adds them all up, in the order of the keys,
// whichever it is: the result does not depend on the order they finish in.
// The sums are written and read past the dies' caches, pair by pair, so that
// no cache has to be written back or emptied for the few lines they fill
// (device-wide fences took 4 us of a 13 us call).
__device__ __forceinline__ void put_pair(float2 *to, float x, float y)
{
    __hip_atomic_store(reinterpret_cast<uint64_t *>(to), (uint64_t)__float_as_uint(y) << 32 | __float_as_uint(x),
                       __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 get_pair(const float2 *from)
{
    const uint64_t v = __hip_atomic_load(reinterpret_cast<const uint64_t *>(from), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return make_float2(__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32)));
}

__device__ __forceinline__ bool last_part(const Chunk &c, const WorkItem &it, int h)
{
    __shared__ uint32_t s_done;
    wait_loads<0>();                              // every wave's sums have arrived ...
    __syncthreads();
    if (threadIdx.x == 0) {                       // ... before the item counts as done
        uint32_t *n = c.count + it.count + h;
        s_done = __hip_atomic_fetch_add(n, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (s_done == (uint32_t)it.parts - 1) __hip_atomic_store(n, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    return s_done == (uint32_t)it.parts - 1;
}

template <typename T, int D, int kRows>
__device__ __forceinline__ void join_parts(const Chunk &c, const WorkItem &it, int h, const Rows &out, float *lse, float sc,
                                           float scale)
{
    const int32_t rows = min(kRows, it.sq.n * c.group - it.row0);
    constexpr int kBlk = kRows / kFewRows;
    const int64_t first = ((int64_t)it.part0 + h * kBlk) * kFewRows, step = (int64_t)c.kv_heads * kBlk * kFewRows;
    for (int u = threadIdx.x; u < rows * (D / 4); u += 256) {
        const int row = u / (D / 4), d = u % (D / 4) * 4;
        const int64_t at = first + row;
        f32x4 y;
        float top, sum;
        // (Eight parts' loads are in flight at a time: one by one, 32 parts of
        // 128 rows took longer to join than to form.)
        constexpr int kAhead = 8;
        auto add = [&](auto apart) {
            constexpr bool kApart = decltype(apart)::value;
            y = f32x4{};
            top = -INFINITY;
            sum = 0.0f;
            for (int k0 = 0; k0 < it.parts; k0 += kAhead) {
                float2 ml[kAhead], lo[kAhead], hi[kAhead];
#pragma unroll
                for (int b = 0; b < kAhead; ++b) {
                    const int64_t from = at + min(k0 + b, it.parts - 1) * step;
                    const float2 *po = reinterpret_cast<const float2 *>(c.part_o + from * D + d);
                    ml[b] = get_pair(c.part_ml + from);
                    lo[b] = get_pair(po);
                    hi[b] = get_pair(po + 1);
                }
#pragma unroll
                for (int b = 0; b < kAhead; ++b) {
                    if (k0 + b >= it.parts || (ml[b].y == 0.0f && ml[b].x == -INFINITY)) continue;
                    // the running maximum moves as it does along the keys
                    const float t = fmaxf(top, ml[b].x), ref = t == -INFINITY ? 0.0f : t;
                    const float was = __builtin_amdgcn_exp2f((top - ref) * sc), is = __builtin_amdgcn_exp2f((ml[b].x - ref) * sc);
                    top = t;
                    sum = sum * was + is * ml[b].y;
                    y = scaled<kApart>(y, was) + scaled<kApart>(f32x4{lo[b].x, lo[b].y, hi[b].x, hi[b].y}, is);
                }
            }
        };
        add(std::false_type());
        if (not_a_number(y)) add(std::true_type());
        const bool none = top == -INFINITY && sum == 0.0f;
        const float inv = none ? 0.0f : 1.0f / sum;
        const int32_t i = (it.row0 + row) / c.group, hh = h * c.group + (it.row0 + row - i * c.group);
        const int64_t t = it.sq.q0 + i;
        Vec4<T> z;
#pragma unroll
        for (int e = 0; e < 4; ++e) z[e] = (T)(y[e] * inv);
        *reinterpret_cast<Vec4<T> *>((T *)out.p + t * out.row + (int64_t)hh * out.head + d) = z;
        if (lse && d == 0) lse[t * c.q_heads + hh] = none ? -INFINITY : top * scale + log2f(sum) * kLn2;
    }
}

// ---- many rows ---------------------------------------------------------------------
//
// Four waves of 32 rows each share a tile of 64 positions, two tiles of keys
// and values in LDS (32 KB each at 128 elements): one is loaded while the
// other is worked on, one barrier a tile.  The two workgroups of a CU fill
// each other's waits.  Bound by the issue of products and of the softmax, one
// exponential, one multiply-add, one addition and half a conversion a weight:
// 3,540 cycles a tile and wave where 64 products alone take 2,048, at the
// 1.85 GHz that the card runs at under it.  870 us, 1.06 PFLOP/s, for 8,000
// tokens over 12,001 positions, 28 heads of 128; 72 us for 13 sequences of up
// to 1,500 tokens, heads of 64 and a window, where an item's 18 tiles take 34
// us and its start and end 8.  Waves that take turns by barriers at products
// and softmax took 930 us, the softmax of one half between the products of
// the other 917.  (At 128 elements 16 registers are kept in memory, and read
// where an item or a pass starts and ends, not between its tiles.)
template <typename T, int D>
__global__ __launch_bounds__(256, D == 64 ? 3 : 2) void k_attend_many(Chunk c, Pages pg, Rows q, Rows out, float *lse, float sc,
                                                        float scale, uint32_t flip)
{
    using Load = TileLoad<D>;
    constexpr int kSteps = D / 16, kBlocks = D / 32;     // of 16 elements of q.k; of 32 elements of o
    constexpr uint32_t kTileBytes = kKeys * D * 2;
    const int item = blockIdx.x / c.kv_heads, h = blockIdx.x % c.kv_heads;
    const WorkItem it = scalar_load(c.many + item);
    if (item >= scalar_load(&c.work->n_many)) return;
    const ChunkSeq sq = it.sq;
    const Span sp = span_of(c, sq, it.row0, kManyRows);
    const int lane = lane_id(), wave = uni32(threadIdx.x >> 6), col = lane & 31, half = lane >> 5;
    const int32_t rows = sq.n * c.group;

    // this lane's row of the attention: a token and a head
    const int32_t wrow = it.row0 + wave * 32, r = min(wrow + col, rows - 1);
    const bool busy = wrow < rows;
    const int32_t i = r / c.group, hq = h * c.group + (r - i * c.group);
    const int32_t p = c.causal ? sq.L - sq.n + i : sq.L - 1;              // sees positions up to p ...
    const int32_t after = c.window > 0 ? p - c.window : -1;               // ... after this one, and below c.sinks
    const Span ws = span_of(c, sq, min(wrow, rows - 1), 32);              // the wave's own rows
    const T *qrow = (const T *)q.p + (int64_t)(sq.q0 + i) * q.row + (int64_t)hq * q.head;
    Vec8<T> qf[kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        u32x4 x = *reinterpret_cast<const u32x4 *>(qrow + s * 16 + half * 8);
        x ^= flip;
        qf[s] = __builtin_bit_cast(Vec8<T>, x);
    }

    // the wave's share of a tile: 16 positions of keys and of values
    const uint32_t base = lds_base();
    Load load_rows(pg);
    const uint32_t *table = c.table + (int64_t)it.seq * c.cols;
    const int32_t last = sq.L - 1;
    auto page_of = [&](int32_t v) { return scalar_load(table + (min(key_tile(sp, v) * kKeys + wave * 16, last) >> c.page_shift)); };
    auto load = [&](int32_t v, uint32_t page, int buf) {
        const uint32_t kt = base + buf * 2 * kTileBytes + wave * 16 * D * 2;
        load_rows.load(c, pg, h, page, key_tile(sp, v) * kKeys + wave * 16, last, kt, kt + kTileBytes);
    };

    // LDS addresses that do not change: keys of this lane's row (piece half of
    // step 0), values of its four rows
    const uint32_t key_at = (uint32_t)(col * D * 2 + ((half ^ Load::key_swizzle(col)) * 16));
    const int vr = (lane & 15) >> 2;
    uint32_t val_at[kBlocks];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) {
        const int pc = 4 * b + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
        val_at[b] = (uint32_t)((4 * half + vr) * D * 2 + (pc ^ Load::value_swizzle(vr)) * 16 + (lane & 1) * 8);
    }

    const float far = fminf(kFar / sc, FLT_MAX);          // of a maximum
    // A weight of zero does not hide a value that is not finite: its product
    // with one is NaN.  If the pass over the keys ends with a NaN, three others
    // follow: over the values with zeros in place of those that are not finite,
    // then over flags of +inf and of -inf (a NaN is both), with weights of one
    // for all that a row sees, which say where infinities are to be added.
    enum { kPlain, kFinite, kUp, kDown };
    for (int mode = kPlain;;) {
        f32x16 o[kBlocks] = {};
        float m = -INFINITY, l = 0.0f;                    // l: of this half's keys
        uint32_t page = 0;
        if (it.v0 < it.v1) {
            load(it.v0, page_of(it.v0), 0);
            page = page_of(min(it.v0 + 1, it.v1 - 1));
        }
        for (int32_t v = it.v0; v < it.v1; ++v) {
            const int buf = (v - it.v0) & 1;
            const uint32_t kt = base + buf * 2 * kTileBytes, vt = kt + kTileBytes;
            tile_barrier();
            if (mode != kPlain) {
                const uint32_t at = vt + wave * (kTileBytes / 4) + lane * 16;     // the wave's share
                for (uint32_t n = 0; n < kTileBytes / 4; n += 1024) {
                    const Vec8<T> x = lds_vec<T>(at + n);
                    *(__attribute__((address_space(3))) Vec8<T> *)(uintptr_t)(at + n) =
                        mode == kFinite ? wild_part<T, 0>(x) : mode == kUp ? wild_part<T, 1>(x) : wild_part<T, 2>(x);
                }
                tile_barrier();
            }
            if (v + 1 < it.v1) {
                load(v + 1, page, buf ^ 1);
                page = page_of(min(v + 2, it.v1 - 1));
            }
            const int32_t t = key_tile(sp, v), j0 = t * kKeys;
            if (!busy || (c.causal && j0 > ws.p1)) continue;

            // LDS reads run half a tile ahead of the products: the first half of
            // the keys, the second, then the first half of the values behind
            // the softmax.  (Left to itself the compiler reads and waits
            // product by product.)
            f32x16 x[2] = {};
            Vec8<T> kf[kSteps][2], vf[4][kBlocks];
            // (Addresses are formed where they are used: kept, they would take 20 registers.)
            auto read_keys = [&](int from, int to) {
                uint32_t lane_at = key_at;
                asm volatile("" : "+v"(lane_at));
#pragma unroll
                for (int s = from; s < to; ++s) {
                    uint32_t at = (lane_at ^ (s * 32)) + kt;
                    asm volatile("" : "+v"(at));
#pragma unroll
                    for (int b = 0; b < 2; ++b) kf[s][b] = lds_vec<T>(at + b * 32 * D * 2);
                }
                __builtin_amdgcn_sched_barrier(0);
            };
            auto multiply_keys = [&](int from, int to) {
#pragma unroll
                for (int s = from; s < to; ++s)
#pragma unroll
                    for (int b = 0; b < 2; ++b) x[b] = Mma<T>::wide(kf[s][b], qf[s], x[b]);
                __builtin_amdgcn_sched_barrier(0);
            };
            auto read_values = [&](int from, int to) {
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) {
                    uint32_t at = vt + val_at[b];
                    asm volatile("" : "+v"(at));
#pragma unroll
                    for (int s = from; s < to; ++s) vf[s][b] = lds_columns<T>(at + s * 16 * D * 2, at + s * 16 * D * 2 + 8 * D * 2);
                }
                __builtin_amdgcn_sched_barrier(0);
            };
            read_keys(0, kSteps / 2);
            read_keys(kSteps / 2, kSteps);
            // (a wave at its products goes before one at its softmax: 2%)
            __builtin_amdgcn_s_setprio(1);
            multiply_keys(0, kSteps / 2);
            read_values(0, 2);
            multiply_keys(kSteps / 2, kSteps);
            __builtin_amdgcn_s_setprio(0);

            if (!tile_whole(c, ws, sq.L, t)) {
                // this row sees the lane's keys from number lo on, up to hi, and below sink
                const int32_t first = j0 + 4 * half, hi = p - first, lo = after - first, sink = c.sinks - first;
                if (c.window <= 0) {
#pragma unroll
                    for (int b = 0; b < 2; ++b)
#pragma unroll
                        for (int e = 0; e < 16; ++e) x[b][e] = b * 32 + 8 * (e >> 2) + (e & 3) > hi ? -INFINITY : x[b][e];
                } else {
#pragma unroll
                    for (int b = 0; b < 2; ++b)
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const int32_t n = b * 32 + 8 * (e >> 2) + (e & 3);
                            x[b][e] = (n > hi) | ((n <= lo) & (n >= sink)) ? -INFINITY : x[b][e];
                        }
                }
            }
            if (mode >= kUp) {                            // the weights below become ones, and zeros for what is hidden
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int e = 0; e < 16; ++e) x[b][e] = x[b][e] == -INFINITY ? -INFINITY : 0.0f;
            }
            // The weights against the reference as it stands.  Only where a
            // sum shows that a row has outgrown it, or has none yet, or has one
            // that is far, is the tile's maximum looked for, and the tile
            // weighed (again) against that: no weight is then above one, or
            // above 2^(2^-12), and none is looked at once more.
            Vec8<T> pf[4];
            float part;
            bool raise = !__all(fabsf(m) <= far), again;
            do {
                float ref = m * sc;
                if (raise) {
                    float mx = x[0][0];
#pragma unroll
                    for (int b = 0; b < 2; ++b)
#pragma unroll
                        for (int e = 0; e < 16; ++e) mx = fmaxf(mx, x[b][e]);
                    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
                    const float top = fmaxf(m, mx), a = top == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((m - top) * sc);
                    m = top;
                    l *= a;
#pragma unroll
                    for (int b = 0; b < kBlocks; ++b) o[b] *= a;
                    const float is = m == -INFINITY ? 0.0f : m;
                    ref = is * sc;
                    if (!__all(fabsf(is) <= far)) {
#pragma unroll
                        for (int b = 0; b < 2; ++b)
#pragma unroll
                            for (int e = 0; e < 16; ++e) x[b][e] -= is;
                        ref = 0.0f;
                    }
                }
                float k = sc;
                asm volatile("" : "+s"(k));               // (or the product is taken out of the loop, and costs as much again)
                float sum[4] = {};
#pragma unroll
                for (int s = 0; s < 4; ++s)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float w = __builtin_amdgcn_exp2f(x[s >> 1][8 * (s & 1) + e] * k - ref);
                        sum[s] += w;
                        pf[s][e] = (T)w;
                    }
                part = (sum[0] + sum[1]) + (sum[2] + sum[3]);
                again = !raise && __any(part > kOutgrown);
                raise = again;
            } while (again);
            l += part;
            __builtin_amdgcn_sched_barrier(0);
            read_values(2, 4);
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int s = 0; s < 4; ++s)
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) o[b] = Mma<T>::wide(vf[s][b], pf[s], o[b]);
            __builtin_amdgcn_s_setprio(0);
        }
        bool wild = false;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) wild |= !(o[b][e] == o[b][e]);
        if (__syncthreads_or(wild) && mode == kPlain) {
            mode = kFinite;
            continue;
        }

        const float inf = mode == kUp ? INFINITY : -INFINITY;
        l += __shfl_xor(l, 32, 64);
        if (it.part >= 0) {
            if (wrow + col < rows) {
                const int64_t at = ((int64_t)it.part + h * (kManyRows / kFewRows)) * kFewRows + wave * 32 + col;
                float *po = c.part_o + at * D;
#pragma unroll
                for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                    for (int e = 0; e < 16; e += 2) {
                        float2 *to = reinterpret_cast<float2 *>(po + b * 32 + 8 * (e >> 2) + 4 * half + (e & 2));
                        if (mode < kUp) put_pair(to, o[b][e], o[b][e + 1]);
                        else if (o[b][e] > 0.0f || o[b][e + 1] > 0.0f) {
                            const float2 was = get_pair(to);
                            put_pair(to, was.x + (o[b][e] > 0.0f ? inf : 0.0f), was.y + (o[b][e + 1] > 0.0f ? inf : 0.0f));
                        }
                    }
                if (half == 0 && mode < kUp) put_pair(c.part_ml + at, m, l);
            }
        } else if (wrow + col < rows) {
            const bool none = m == -INFINITY && l == 0.0f;
            const float inv = none ? 0.0f : 1.0f / l;
            const int64_t t = sq.q0 + i;
            T *orow = (T *)out.p + t * out.row + (int64_t)hq * out.head;
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                for (int e = 0; e < 16; e += 4) {
                    Vec4<T> *to = reinterpret_cast<Vec4<T> *>(orow + b * 32 + 2 * e + 4 * half), y;
                    if (mode < kUp) {
#pragma unroll
                        for (int n = 0; n < 4; ++n) y[n] = (T)(o[b][e + n] * inv);
                    } else {
                        y = *to;
#pragma unroll
                        for (int n = 0; n < 4; ++n)
                            if (o[b][e + n] > 0.0f) y[n] = (T)((float)y[n] + inf);
                    }
                    *to = y;
                }
            if (lse && half == 0 && mode < kUp) lse[t * c.q_heads + hq] = none ? -INFINITY : m * scale + log2f(l) * kLn2;
        }
        if (mode == kPlain || mode == kDown) break;
        ++mode;
        wait_loads<0>();                                  // what this pass wrote is read by the next
    }
    if (it.part >= 0 && last_part(c, it, h)) join_parts<T, D, kManyRows>(c, it, h, out, lse, sc, scale);
}

// ---- few rows -------------------------------------------------------------------------
//
// At most 16 rows: the cache is read once and that is the work.  Every wave
// takes key tiles of its own, halves of 32 positions, two of them in LDS, one
// in flight while the other is worked on, with no barrier between the waves;
// at the end their sums are joined through LDS.  Measured: 748 us, 5.9 TB/s,
// for 64 tokens over caches of 4.4 GB in all, and 8.4 us for 5 over short
// ones, of which a launch and the chain of loads are all (0.2 of it to tell
// far scores and joined infinities); the kernel for many rows takes 850 to 880
// and 15.6 us for them.
template <typename T, int D>
__global__ __launch_bounds__(256, 1) void k_attend_few(Chunk c, Pages pg, Rows q, Rows out, float *lse, float sc,
                                                       float scale, uint32_t flip)
{
    using Load = TileLoad<D>;
    constexpr int kSteps = D / 32, kBlocks = D / 16;     // of 32 elements of q.k; of 16 elements of o
    constexpr uint32_t kHalfBytes = 32 * D * 2, kWaveBytes = 4 * kHalfBytes;
    const int item = blockIdx.x / c.kv_heads, h = blockIdx.x % c.kv_heads;
    const WorkItem it = scalar_load(c.few + item);
    if (item >= scalar_load(&c.work->n_few)) return;
    const ChunkSeq sq = it.sq;
    const Span sp = span_of(c, sq, 0, kFewRows);
    const int lane = lane_id(), wave = uni32(threadIdx.x >> 6), col = lane & 15, quad = lane >> 4;
    const int32_t rows = sq.n * c.group;
    const int32_t r = min(col, rows - 1), i = r / c.group, hq = h * c.group + (r - i * c.group);
    const int32_t p = c.causal ? sq.L - sq.n + i : sq.L - 1, after = c.window > 0 ? p - c.window : -1;
    const T *qrow = (const T *)q.p + (int64_t)(sq.q0 + i) * q.row + (int64_t)hq * q.head;
    Vec8<T> qf[kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        u32x4 x = *reinterpret_cast<const u32x4 *>(qrow + s * 32 + quad * 8);
        x ^= flip;
        qf[s] = __builtin_bit_cast(Vec8<T>, x);
    }

    const uint32_t base = lds_base() + wave * kWaveBytes;
    Load load_rows(pg);
    const uint32_t *table = c.table + (int64_t)it.seq * c.cols;
    const int32_t last = sq.L - 1;
    // the wave's halves: of key tiles v0 + wave, v0 + wave + 4, ...
    const int32_t halves = it.v1 - it.v0 > wave ? 2 * ((it.v1 - it.v0 - wave + 3) / 4) : 0;
    auto first_of = [&](int32_t n) { return key_tile(sp, it.v0 + wave + (n >> 1) * 4) * kKeys + (n & 1) * 32; };
    auto page_of = [&](int32_t j) { return scalar_load(table + (min(j, last) >> c.page_shift)); };
    auto load = [&](int32_t j0, uint32_t p0, uint32_t p1, int buf) {
        const uint32_t kt = base + buf * 2 * kHalfBytes;
#pragma unroll
        for (int g = 0; g < 2; ++g)
            load_rows.load(c, pg, h, g ? p1 : p0, j0 + g * 16, last, kt + g * 16 * D * 2, kt + kHalfBytes + g * 16 * D * 2);
    };
    const uint32_t key_at = (uint32_t)(col * D * 2 + ((quad ^ Load::key_swizzle(col)) * 16));
    const int vr = (lane & 15) >> 2;
    uint32_t val_at[kBlocks];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) {
        const int pc = 2 * b + ((lane & 3) >> 1);
        val_at[b] = (uint32_t)((4 * quad + vr) * D * 2 + (pc ^ Load::value_swizzle(vr)) * 16 + (lane & 1) * 8);
    }

    f32x4 o[kBlocks];
    float m, l;                                           // m: before the scale
    // Where the sums end with a NaN, again, with values that are not finite kept
    // apart from the others: ones in their place, for all that a row sees.  Also
    // again where the reference is far, and then it is taken off the scores first.
    auto pass = [&](auto apart) {
        constexpr bool kApart = decltype(apart)::value;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) o[b] = f32x4{};
        m = -INFINITY;
        l = 0.0f;
        float ms = -INFINITY;                             // scale * m
        uint32_t p0 = 0, p1 = 0;
        if (halves > 0) {
            load(first_of(0), page_of(first_of(0)), page_of(first_of(0) + 16), 0);
            p0 = page_of(first_of(1));
            p1 = page_of(first_of(1) + 16);
        }
        for (int32_t n = 0; n < halves; ++n) {
            const int buf = n & 1;
            const int32_t j0 = first_of(n);
            if (n + 1 < halves) {
                load(first_of(n + 1), p0, p1, buf ^ 1);
                const int32_t jn = first_of(min(n + 2, halves - 1));
                p0 = page_of(jn);
                p1 = page_of(jn + 16);
                wait_loads<4 * Load::kLoads>();
            } else {
                wait_loads<0>();
            }
            const uint32_t kt = base + buf * 2 * kHalfBytes, vt = kt + kHalfBytes;
            f32x4 x[2] = {};
#pragma unroll
            for (int s = 0; s < kSteps; ++s)
#pragma unroll
                for (int b = 0; b < 2; ++b)
                    x[b] = Mma<T>::narrow(lds_vec<T>(kt + (key_at ^ (s * 64)) + b * 16 * D * 2), qf[s], x[b]);
            const bool part = !tile_whole(c, sp, sq.L, j0 / kKeys);
            uint32_t see = ~0u;                           // which weights are not hidden
            if (part) {
                const int32_t first = j0 + 4 * quad, hi = p - first, lo = after - first, sink = c.sinks - first;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int32_t k = 16 * (e >> 2) + (e & 3);
                    const bool hidden = k > hi || (k <= lo && k >= sink);
                    if (hidden) x[e >> 2][e & 3] = -INFINITY;
                    if (kApart && hidden) see &= ~(1u << e);
                }
            }
            float mx = fmaxf(fmaxf(fmaxf(x[0][0], x[0][1]), fmaxf(x[0][2], x[0][3])),
                             fmaxf(fmaxf(x[1][0], x[1][1]), fmaxf(x[1][2], x[1][3])));
            mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
            mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
            if (__any(kApart ? (mx - m) * sc > kSlack : mx * sc > ms + kSlack)) {
                const float top = fmaxf(m, mx), ts = top * sc;
                const float a = top == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(kApart ? (m - top) * sc : ms - ts);
                m = top;
                ms = ts;
                l *= a;
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) o[b] = scaled<kApart>(o[b], a);
            }
            const float ref = m == -INFINITY ? 0.0f : kApart ? m : ms;
            Vec8<T> pf;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float s = x[e >> 2][e & 3], w = __builtin_amdgcn_exp2f(kApart ? (s - ref) * sc : s * sc - ref);
                l += w;
                pf[e] = (T)w;
            }
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) {
                const Vec8<T> val = lds_columns<T>(vt + val_at[b], vt + val_at[b] + 16 * D * 2);
                if (!kApart) {
                    o[b] = Mma<T>::narrow(val, pf, o[b]);
                    continue;
                }
                auto add = [&](auto kind) {
                    constexpr int kKind = decltype(kind)::value;
                    f32x4 y = {};
                    y = Mma<T>::narrow(wild_part<T, kKind>(val), kKind == 0 ? pf : ones<T>(see), y);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        o[b][e] += kKind == 0 ? y[e] : y[e] > 0.0f ? (kKind == 1 ? INFINITY : -INFINITY) : 0.0f;
                };
                add(std::integral_constant<int, 0>());
                add(std::integral_constant<int, 1>());
                add(std::integral_constant<int, 2>());
            }
            // the next load overwrites this half: its reads must have returned
            asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
        }
        bool wild = m != -INFINITY && !(fabsf(ms) <= kFar);
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) wild |= !(o[b][e] == o[b][e]);
        return wild;
    };
    if (__any(pass(std::false_type()))) (void)pass(std::true_type());
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);

    // join the waves: every wave's sums at its reference, in 32 bits
    tile_barrier();
    float *so = (float *)lds;                             // [4][16][D + 4]
    float2 *sml = (float2 *)(lds + 4 * 16 * (D + 4) * 4); // [4][16]
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
        *reinterpret_cast<f32x4 *>(so + (wave * 16 + col) * (D + 4) + b * 16 + 4 * quad) = o[b];
    if (quad == 0) sml[wave * 16 + col] = make_float2(m, l);
    __syncthreads();
    for (int u = threadIdx.x; u < 16 * (D / 4); u += 256) {
        const int row = u / (D / 4), d = u % (D / 4) * 4;
        if (row >= rows) break;
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < 4; ++w) top = fmaxf(top, sml[w * 16 + row].x);
        const float ref = top == -INFINITY ? 0.0f : top;
        f32x4 y;
        float sum;
        auto add = [&](auto apart) {
            y = f32x4{};
            sum = 0.0f;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float2 ml = sml[w * 16 + row];
                const float a = __builtin_amdgcn_exp2f((ml.x - ref) * sc);
                if (ml.y == 0.0f && ml.x == -INFINITY) continue;
                sum += a * ml.y;
                y += scaled<decltype(apart)::value>(*reinterpret_cast<const f32x4 *>(so + (w * 16 + row) * (D + 4) + d), a);
            }
        };
        add(std::false_type());
        if (not_a_number(y)) add(std::true_type());
        if (it.part >= 0) {
            const int64_t at = ((int64_t)it.part + h) * kFewRows + row;
            float2 *po = reinterpret_cast<float2 *>(c.part_o + at * D + d);
            put_pair(po, y[0], y[1]);
            put_pair(po + 1, y[2], y[3]);
            if (d == 0) put_pair(c.part_ml + at, top, sum);
            continue;
        }
        const bool none = top == -INFINITY && sum == 0.0f;
        const float inv = none ? 0.0f : 1.0f / sum;
        const int32_t ti = row / c.group, hh = h * c.group + (row - ti * c.group);
        const int64_t t = sq.q0 + ti;
        Vec4<T> z;
#pragma unroll
        for (int e = 0; e < 4; ++e) z[e] = (T)(y[e] * inv);
        *reinterpret_cast<Vec4<T> *>((T *)out.p + t * out.row + (int64_t)hh * out.head + d) = z;
        if (lse && d == 0) lse[t * c.q_heads + hh] = none ? -INFINITY : top * scale + log2f(sum) * kLn2;
    }
    if (it.part >= 0 && last_part(c, it, h)) join_parts<T, D, kFewRows>(c, it, h, out, lse, sc, scale);
}

namespace {

template <typename T, int D>
hipError_t attend(const Launch &L, const Chunk &c, const Pages &pg, const Rows &q, const Rows &out, float *lse, float scale)
{
    // the maximum is taken before the scale, so that the scale has to be
    // positive: its sign goes to q; and what is hidden, -inf, stays that
    const float sc = std::max(fabsf(scale) * kLog2e, 1e-37f);
    const uint32_t flip = scale < 0.0f ? 0x80008000u : 0u;
    const int64_t rows = (int64_t)c.n_tokens * c.group, most = (int64_t)c.max_new * c.group;
    const int64_t hk = c.kv_heads;
    // grids that hold every item the plan can have made; the rest leave at once
    const int64_t few = (int64_t)c.n_seqs + c.few_slots / hk, many = rows / kManyRows + c.n_seqs + c.many_slots / hk;
    const unsigned few_lds = 4 * 4 * 32 * D * 2, many_lds = 4 * kKeys * D * 2;
    // a launch that no sequence can need is left out
    if (c.few_rows > 0)
        RO_LAUNCH(L, RO_K_CHUNK_ATTEND, (k_attend_few<T, D>), dim3((unsigned)((few + 1) * hk)), dim3(256), few_lds, L.stream,
                  c, pg, q, out, lse, sc, fabsf(scale), flip);
    if (most > kFewRows)
        RO_LAUNCH(L, RO_K_CHUNK_ATTEND, (k_attend_many<T, D>), dim3((unsigned)((many + 1) * hk)), dim3(256), many_lds,
                  L.stream, c, pg, q, out, lse, sc, fabsf(scale), flip);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_attend(const Launch &L, const Chunk &c, const Pages &pg, const Rows &q, const Rows &out, float *lse,
                         float scale, int32_t dtype)
{
    if (dtype == RO_BF16) return c.head_dim == 128 ? attend<__bf16, 128>(L, c, pg, q, out, lse, scale)
                                                   : attend<__bf16, 64>(L, c, pg, q, out, lse, scale);
    return c.head_dim == 128 ? attend<_Float16, 128>(L, c, pg, q, out, lse, scale)
                             : attend<_Float16, 64>(L, c, pg, q, out, lse, scale);
}

}  // namespace ro
