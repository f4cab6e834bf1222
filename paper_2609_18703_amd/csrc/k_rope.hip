// Rotary positions of several axes, alone and on the way into a paged cache.
//
// Pair i of a head turns by angle(t, i) = pos[axis(i), t] * freq(i):
//   (a, b) -> (a cos - b sin, b cos + a sin),
// with sin negated for the rotation back, which is the transpose and so the
// gradient.  Every element is read and written once and nothing else is
// large, so both kernels are bound by memory; the angles of a token are
// formed once, in LDS, and serve all of its heads.  Measured: 102 us, 5.9
// TB/s read and written, for 32,771 tokens of 36 heads of 128; 78 us, 5.5
// TB/s, for 17,600 tokens that enter a cache.  A batch's single tokens take
// 4 us, the time of one small kernel.
#include <algorithm>

#include "ro_chunk.h"

namespace ro {

// cos and sin of a pair's angle.  The product of a 32-bit position and a
// 24-bit frequency is formed and reduced to a part of a turn in 64 bits: in
// 32 bits an angle of 10^5 would be off by 0.004.
__device__ __forceinline__ float2 turn(const RotaryArgs &r, int64_t t, int i, float sign)
{
    const double x = (double)r.pos[(int64_t)r.axis[i] * r.pos_stride + t] * (double)r.freq[i] * 0.15915494309189535;
    float s, c;
    sincospif(2.0f * (float)(x - rint(x)), &s, &c);
    return make_float2(c, sign * s);
}

// One thread's piece of a head: with kVec 8 elements of either half of the
// pairs, or 8 neighbours; without, one pair or one element.  Units below
// rot_units rotate, the others copy.
template <typename T, bool kAdj, bool kVec>
__device__ __forceinline__ void rope_unit(const T *x, T *y, int u, int rot_units, int rot, const float2 *cs, bool turn)
{
    if constexpr (kVec) {
        if (u >= rot_units) {
            const int at = kAdj ? u * 8 : rot + (u - rot_units) * 8;
            *reinterpret_cast<Vec8<T> *>(y + at) = *reinterpret_cast<const Vec8<T> *>(x + at);
        } else if constexpr (kAdj) {
            Vec8<T> a = *reinterpret_cast<const Vec8<T> *>(x + u * 8);
            if (turn)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 w = cs[u * 4 + e];
                    const float p = (float)a[2 * e], q = (float)a[2 * e + 1];
                    a[2 * e] = (T)(p * w.x - q * w.y);
                    a[2 * e + 1] = (T)(q * w.x + p * w.y);
                }
            *reinterpret_cast<Vec8<T> *>(y + u * 8) = a;
        } else {
            const int at = u * 8, half = rot / 2;
            Vec8<T> a = *reinterpret_cast<const Vec8<T> *>(x + at), b = *reinterpret_cast<const Vec8<T> *>(x + half + at);
            if (turn)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float2 w = cs[at + e];
                    const float p = (float)a[e], q = (float)b[e];
                    a[e] = (T)(p * w.x - q * w.y);
                    b[e] = (T)(q * w.x + p * w.y);
                }
            *reinterpret_cast<Vec8<T> *>(y + at) = a;
            *reinterpret_cast<Vec8<T> *>(y + half + at) = b;
        }
    } else {
        if (u >= rot_units) {
            const int at = rot + (u - rot_units);
            y[at] = x[at];
        } else {
            const int i = kAdj ? 2 * u : u, j = kAdj ? 2 * u + 1 : u + rot / 2;
            const T a = x[i], b = x[j];
            const float2 w = turn ? cs[u] : make_float2(1.0f, 0.0f);
            y[i] = turn ? (T)((float)a * w.x - (float)b * w.y) : a;
            y[j] = turn ? (T)((float)b * w.x + (float)a * w.y) : b;
        }
    }
}

// units of a head and how many of them rotate
__host__ __device__ inline void rope_units(int rot, int D, bool adj, bool vec, int &units, int &rot_units)
{
    if (vec) {
        rot_units = adj ? rot / 8 : rot / 16;
        units = rot_units + (D - rot) / 8;
    } else {
        rot_units = rot / 2;
        units = rot_units + (D - rot);
    }
}

template <typename T, bool kAdj, bool kVec>
__global__ __launch_bounds__(kBlock) void k_rope(RotaryArgs r, Rows x, Rows y, int64_t n_tokens, int heads, int D,
                                                 int per, float sign)
{
    extern __shared__ float2 cs[];
    const int pairs = r.rot / 2;
    int units, rot_units;
    rope_units(r.rot, D, kAdj, kVec, units, rot_units);
    for (int64_t t0 = (int64_t)blockIdx.x * per; t0 < n_tokens; t0 += (int64_t)gridDim.x * per) {
        const int nt = (int)min64(per, n_tokens - t0);
        for (int i = threadIdx.x; i < nt * pairs; i += kBlock) cs[i] = turn(r, t0 + i / pairs, i % pairs, sign);
        __syncthreads();
        for (int i = threadIdx.x; i < nt * heads * units; i += kBlock) {
            const int u = i % units, th = i / units, h = th % heads, t = th / heads;
            rope_unit<T, kAdj, kVec>((const T *)x.p + (t0 + t) * x.row + h * x.head,
                                     (T *)y.p + (t0 + t) * y.row + h * y.head, u, rot_units, r.rot, cs + t * pairs, true);
        }
        __syncthreads();
    }
}

template <typename T, bool kAdj, bool kVec>
__global__ __launch_bounds__(kBlock) void k_append(Chunk c, Pages pg, RotaryArgs r, Rows q, Rows k, Rows v, Rows qo,
                                                   int per, Ctl *ctl)
{
    extern __shared__ float2 cs[];
    const int pairs = r.rot / 2, D = c.head_dim;
    int units, rot_units;
    rope_units(r.rot, D, kAdj, kVec, units, rot_units);
    const int qh = q.p ? c.q_heads : 0, heads = qh + 2 * c.kv_heads;
    for (int64_t t0 = (int64_t)blockIdx.x * per; t0 < c.n_tokens; t0 += (int64_t)gridDim.x * per) {
        const int nt = (int)min64(per, c.n_tokens - t0);
        for (int i = threadIdx.x; i < nt * pairs; i += kBlock) cs[i] = turn(r, t0 + i / pairs, i % pairs, 1.0f);
        __syncthreads();
        for (int i = threadIdx.x; i < nt * heads * units; i += kBlock) {
            const int u = i % units, th = i / units, h = th % heads;
            const int64_t t = t0 + th / heads;
            const float2 *w = cs + (th / heads) * pairs;
            if (h < qh) {
                rope_unit<T, kAdj, kVec>((const T *)q.p + t * q.row + h * q.head, (T *)qo.p + t * qo.row + h * qo.head, u,
                                         rot_units, r.rot, w, true);
                continue;
            }
            const uint64_t sl = c.slot[t];
            if (sl == ~0ull) {
                // tokens of an invalid sequence were reported by the plan
                if (c.tok[t] != ~0u) raise_err(ctl, RO_ERANGE);
                continue;
            }
            const bool is_k = h < qh + c.kv_heads;
            const int hh = h - qh - (is_k ? 0 : c.kv_heads);
            const Rows &src = is_k ? k : v;
            T *dst = (T *)(is_k ? pg.k : pg.v) + (int64_t)(sl >> 32) * pg.page + hh * pg.head +
                     (int64_t)(uint32_t)sl * pg.slot;
            rope_unit<T, kAdj, kVec>((const T *)src.p + t * src.row + hh * src.head, dst, u, rot_units, r.rot, w, is_k);
        }
        __syncthreads();
    }
}

namespace {

constexpr int64_t kMostGroups = 1 << 23;        // a launch has fewer than 2^32 threads; more tokens take turns

bool rows_16(const Rows &r) { return (((uintptr_t)r.p) & 15) == 0 && r.row % 8 == 0 && r.head % 8 == 0; }

bool vec_ok(const RotaryArgs &r, int D) { return D % 8 == 0 && r.rot % (r.adjacent ? 8 : 16) == 0; }

// Tokens of a workgroup: as many as give every thread a unit, fewer where
// they would not make four workgroups for every CU.  Threads wait for the
// angles, so that more tokens than that only make them wait together: 1, 2,
// 4, 8 tokens take 78, 81, 88, 99 us where a token has 384 units (append,
// 17,600 tokens), 39, 31, 32, 32 us where it has 80 (40,000 tokens of 16 heads
// of 80 elements), 229, 130, 79, 59 us where it has 16 (300,000 of 4 of 64).
int tokens_per_group(int64_t T, int units, int num_cus)
{
    return (int)std::max<int64_t>(1, std::min<int64_t>({T / (4 * (int64_t)num_cus), kBlock / units, 64}));
}

}  // namespace

hipError_t launch_rope(const Launch &L, const RotaryArgs &r, const Rows &x, const Rows &y, int64_t T, int32_t heads,
                       int32_t D, int32_t dtype, int32_t inverse)
{
    const bool vec = vec_ok(r, D) && rows_16(x) && rows_16(y);
    int units, rot_units;
    rope_units(r.rot, D, r.adjacent, vec, units, rot_units);
    const int per = tokens_per_group(T, heads * units, L.num_cus);
    const dim3 grid((unsigned)std::min<int64_t>((T + per - 1) / per, kMostGroups));
    const size_t lds = (size_t)per * (r.rot / 2) * sizeof(float2);
    const float sign = inverse ? -1.0f : 1.0f;
#define RO_ROPE(T_, A_, V_)                                                                                       \
    RO_LAUNCH(L, RO_K_ROPE, (k_rope<T_, A_, V_>), grid, dim3(kBlock), lds, L.stream, r, x, y, T, heads, D, per, sign)
#define RO_ROPE_T(T_)                                                                  \
    do {                                                                               \
        if (r.adjacent && vec) RO_ROPE(T_, true, true);                                \
        else if (r.adjacent) RO_ROPE(T_, true, false);                                 \
        else if (vec) RO_ROPE(T_, false, true);                                        \
        else RO_ROPE(T_, false, false);                                                \
    } while (0)
    if (dtype == RO_BF16) RO_ROPE_T(__bf16);
    else RO_ROPE_T(_Float16);
    return hipGetLastError();
}

hipError_t launch_append(const Launch &L, const Chunk &c, const Pages &pg, const RotaryArgs *ra, const Rows &q,
                         const Rows &k, const Rows &v, const Rows &qo, int32_t dtype)
{
    RotaryArgs r{};
    if (ra) r = *ra;
    const int D = c.head_dim;
    const bool vec = vec_ok(r, D) && rows_16(k) && rows_16(v) && (!q.p || (rows_16(q) && rows_16(qo)));
    int units, rot_units;
    rope_units(r.rot, D, r.adjacent, vec, units, rot_units);
    const int per = tokens_per_group(c.n_tokens, ((q.p ? c.q_heads : 0) + 2 * c.kv_heads) * units, L.num_cus);
    const dim3 grid((unsigned)std::min<int64_t>((c.n_tokens + per - 1) / per, kMostGroups));
    const size_t lds = (size_t)per * (r.rot / 2) * sizeof(float2);
#define RO_APPEND(T_, A_, V_)                                                                                      \
    RO_LAUNCH(L, RO_K_CHUNK_APPEND, (k_append<T_, A_, V_>), grid, dim3(kBlock), lds, L.stream, c, pg, r, q, k, v, qo, \
              per, L.ctl)
#define RO_APPEND_T(T_)                                                                \
    do {                                                                               \
        if (r.adjacent && vec) RO_APPEND(T_, true, true);                              \
        else if (r.adjacent) RO_APPEND(T_, true, false);                               \
        else if (vec) RO_APPEND(T_, false, true);                                      \
        else RO_APPEND(T_, false, false);                                              \
    } while (0)
    if (dtype == RO_BF16) RO_APPEND_T(__bf16);
    else RO_APPEND_T(_Float16);
    return hipGetLastError();
}

}  // namespace ro
