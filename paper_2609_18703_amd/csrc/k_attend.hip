// Attention of a chunk's tokens over a paged cache.
//
//   o = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale q.k_j - m),
// over the positions a token sees, in one pass with the running maximum m.
//
// One wave per (token, query head): 64 positions at a time, a lane for the
// product of each, then the lanes take the head's elements and add up the
// values.  Positions that are not seen are skipped, not multiplied by zero.
#include "ro_chunk.h"

namespace ro {

template <typename T, int D>
__global__ __launch_bounds__(64) void k_attend(Chunk c, Pages pg, Rows q, Rows out, float *lse, float scale)
{
    __shared__ float s_q[D], s_p[64];
    const int64_t t = blockIdx.x / c.q_heads;
    const int h = blockIdx.x % c.q_heads, hk = h / c.group, lane = lane_id();
    const uint32_t s = c.tok[t];
    constexpr int kPer = D / 64;
    float o[kPer] = {}, m = -INFINITY, l = 0.0f;
    if (s != ~0u) {
        const ChunkSeq sq = c.seq[s];
        const int32_t p = sq.L - sq.n + (int32_t)(t - sq.q0);
        for (int d = lane; d < D; d += 64) s_q[d] = (float)((const T *)q.p)[t * q.row + h * q.head + d] * scale;
        __syncthreads();
        for (int32_t j0 = 0; j0 < sq.L; j0 += 64) {
            const int32_t j = j0 + lane;
            const bool see = j < sq.L && sees(c, p, j);
            if (!__ballot(see)) continue;
            float x = -INFINITY;
            if (see) {
                const Vec8<T> *k = (const Vec8<T> *)((const T *)pg.k + page_at(c, pg, s, j) + hk * pg.head);
                x = 0.0f;
                for (int d = 0; d < D / 8; ++d) {
                    const Vec8<T> a = k[d];
                    for (int e = 0; e < 8; ++e) x += (float)a[e] * s_q[d * 8 + e];
                }
            }
            float mx = x;
            for (int w = 32; w; w >>= 1) mx = fmaxf(mx, __shfl_xor(mx, w, 64));
            mx = fmaxf(mx, m);
            const float base = mx == -INFINITY ? 0.0f : mx;
            const float pr = see ? expf(x - base) : 0.0f, a = expf(m - base);
            m = mx;
            l = l * a + wave_sum(pr);
            for (int e = 0; e < kPer; ++e) o[e] *= a;
            s_p[lane] = pr;
            uint64_t todo = __ballot(see);
            __syncthreads();
            while (todo) {
                const int i = __builtin_ctzll(todo);
                todo &= todo - 1;
                const T *v = (const T *)pg.v + page_at(c, pg, s, j0 + i) + hk * pg.head;
                for (int e = 0; e < kPer; ++e) o[e] += s_p[i] * (float)v[lane + e * 64];
            }
            __syncthreads();
        }
    }
    for (int e = 0; e < kPer; ++e)
        ((T *)out.p)[t * out.row + h * out.head + lane + e * 64] = (T)(m == -INFINITY ? 0.0f : o[e] / l);
    if (lse && lane == 0) lse[t * c.q_heads + h] = m == -INFINITY ? -INFINITY : m + logf(l);
}

hipError_t launch_attend(const Launch &L, const Chunk &c, const Pages &pg, const Rows &q, const Rows &out, float *lse,
                         float scale, int32_t dtype)
{
    const dim3 grid((unsigned)((int64_t)c.n_tokens * c.q_heads));
#define RO_ATTEND(T_, D_)                                                                                            \
    RO_LAUNCH(L, RO_K_CHUNK_ATTEND, (k_attend<T_, D_>), grid, dim3(64), 0, L.stream, c, pg, q, out, lse, scale)
    if (dtype == RO_BF16 && c.head_dim == 128) RO_ATTEND(__bf16, 128);
    else if (dtype == RO_BF16) RO_ATTEND(__bf16, 64);
    else if (c.head_dim == 128) RO_ATTEND(_Float16, 128);
    else RO_ATTEND(_Float16, 64);
    return hipGetLastError();
}

}  // namespace ro
