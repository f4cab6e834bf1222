// The product of 8-bit rows and 8-bit weights, with a scale for each row and
// each channel.
#include "ro_step.h"

namespace ro {

namespace {

using i32x4 = int __attribute__((ext_vector_type(4)));

// out[t, c .. c + 4) of the integer sums, as many as there are channels.
template <typename T>
__device__ __forceinline__ void store_four(const Product &p, int64_t t, int64_t c, const i32x4 &sum, bool wide)
{
    if (t >= p.m || c >= p.n) return;
    const float a = p.a_scale[t];
    const int n = (int)min64(4, p.n - c);
    T *out = (T *)p.out + t * p.out_stride + c;
    T v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (i >= n) break;
        float f = (float)sum[i] * a * p.w_scale[c + i];
        if (p.bias) f += p.bias[c + i];
        v[i] = (T)f;
    }
    (void)wide;
    for (int i = 0; i < n; ++i) out[i] = v[i];
}

}  // namespace

template <typename T>
__global__ void __launch_bounds__(256) k_project(Product p)
{
    const int lane = lane_id(), r = lane & 15, part = lane >> 4;
    const int64_t n0 = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * 16, m0 = (int64_t)blockIdx.y * 16;
    if (n0 >= p.n) return;
    const int8_t *w = p.w + min64(n0 + r, p.n - 1) * p.w_stride, *a = p.a + min64(m0 + r, p.m - 1) * p.a_stride;
    i32x4 sum = {0, 0, 0, 0};
    for (int32_t k = part * 16; k - part * 16 < p.k; k += 64) {
        i32x4 x = {0, 0, 0, 0}, y = {0, 0, 0, 0};
        if (k < p.k) {
            x = *(const i32x4 *)(w + k);
            y = *(const i32x4 *)(a + k);
        }
        sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(x, y, sum, 0, 0, 0);
    }
    store_four<T>(p, m0 + r, n0 + 4 * part, sum, false);
}

hipError_t launch_project(const Launch &L, const Product &p, int32_t dtype)
{
    const dim3 grid((unsigned)((p.n + 63) / 64), (unsigned)((p.m + 15) / 16));
    if (dtype == RO_BF16)
        RO_LAUNCH(L, RO_K_PROJECT, k_project<__bf16>, grid, dim3(256), 0, L.stream, p);
    else if (dtype == RO_F16)
        RO_LAUNCH(L, RO_K_PROJECT, k_project<_Float16>, grid, dim3(256), 0, L.stream, p);
    else
        RO_LAUNCH(L, RO_K_PROJECT, k_project<float>, grid, dim3(256), 0, L.stream, p);
    return hipGetLastError();
}

}  // namespace ro
