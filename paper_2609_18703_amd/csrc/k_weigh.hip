// The attention that every cached position received.
//
//   w_out[j] = w_in[j] + sum over tokens i that see j, over their heads h, of
//              exp(scale q_ih . k_j - lse_ih)
//
// A thread owns one position and adds up all that sees it in a fixed order,
// so no atomics are needed and the same call gives the same bits.
#include "ro_chunk.h"

namespace ro {

template <typename T, int D>
__global__ __launch_bounds__(kBlock) void k_weigh(Chunk c, Pages pg, Rows q, const float *lse, const float *w_in,
                                                  float *w_out, int64_t w_stride, float scale, Ctl *ctl)
{
    __shared__ float s_q[D];
    const int32_t s = blockIdx.x;
    const ChunkSeq sq = c.seq[s];
    if (sq.L > w_stride) {
        if (blockIdx.y == 0 && threadIdx.x == 0) raise_err(ctl, RO_ERANGE);
        return;
    }
    for (int32_t j0 = blockIdx.y * kBlock; j0 < sq.L; j0 += gridDim.y * kBlock) {
        const int32_t j = j0 + threadIdx.x;
        float sum = 0.0f;
        for (int h = 0; h < c.q_heads; ++h) {
            Vec8<T> k[D / 8];
            if (j < sq.L) {
                const Vec8<T> *at = (const Vec8<T> *)((const T *)pg.k + page_at(c, pg, s, j) + (h / c.group) * pg.head);
                for (int d = 0; d < D / 8; ++d) k[d] = at[d];
            }
            for (int32_t i = 0; i < sq.n; ++i) {
                const int32_t p = sq.L - sq.n + i;
                const int64_t t = sq.q0 + i;
                __syncthreads();
                if (threadIdx.x < D) s_q[threadIdx.x] = (float)((const T *)q.p)[t * q.row + h * q.head + threadIdx.x] * scale;
                __syncthreads();
                if (j < sq.L && sees(c, p, j)) {
                    float x = 0.0f;
                    for (int d = 0; d < D / 8; ++d)
                        for (int e = 0; e < 8; ++e) x += (float)k[d][e] * s_q[d * 8 + e];
                    sum += expf(x - lse[t * c.q_heads + h]);
                }
            }
        }
        if (j < sq.L) w_out[s * w_stride + j] = (w_in ? w_in[s * w_stride + j] : 0.0f) + sum;
    }
}

hipError_t launch_weigh(const Launch &L, const Chunk &c, const Pages &pg, const Rows &q, const float *lse,
                        const float *w_in, float *w_out, int64_t w_stride, float scale, int32_t dtype)
{
    const int64_t most = (c.cols << c.page_shift);
    int64_t y = (most + kBlock - 1) / kBlock;
    y = y < 1 ? 1 : (y > 1024 ? 1024 : y);
    const dim3 grid((unsigned)c.n_seqs, (unsigned)y);
#define RO_WEIGH(T_, D_)                                                                                               \
    RO_LAUNCH(L, RO_K_CHUNK_WEIGH, (k_weigh<T_, D_>), grid, dim3(kBlock), 0, L.stream, c, pg, q, lse, w_in, w_out, \
              w_stride, scale, L.ctl)
    if (dtype == RO_BF16 && c.head_dim == 128) RO_WEIGH(__bf16, 128);
    else if (dtype == RO_BF16) RO_WEIGH(__bf16, 64);
    else if (c.head_dim == 128) RO_WEIGH(_Float16, 128);
    else RO_WEIGH(_Float16, 64);
    return hipGetLastError();
}

}  // namespace ro
