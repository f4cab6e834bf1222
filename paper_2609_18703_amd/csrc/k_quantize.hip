// Rows of 16-bit values to 8-bit integers with one scale each.
//
// q = rint(127 x / a), a the row's largest magnitude, as if the quotient were
// exact: 127 x has at most 18 bits, and a quotient of such numbers that is not
// halfway between two integers lies at least 2^-19 of itself away from there,
// far more than the half step (2^-24 of it) by which its 32-bit form is off.
//
// One workgroup a row, which it reads twice, the second time from the cache.
// Bound by memory: 12,001 rows of 4,096 take 35 us, 4.2 TB/s read and written;
// five rows of 3,584 take 3 us, the way to memory and back.
#include "ro_step.h"

namespace ro {

namespace {

constexpr int kQuant = 256;

template <typename T>
using Eight = T __attribute__((ext_vector_type(8)));

// Magnitudes of 16-bit floats are ordered as their bits are; from kInf on they
// are infinite or no numbers.
template <typename T>
constexpr uint32_t kInf = 0x7f80;
template <>
constexpr uint32_t kInf<_Float16> = 0x7c00;

__device__ __forceinline__ uint32_t wave_max(uint32_t v)
{
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, d, 64));
    return v;
}

}  // namespace

template <typename T>
__global__ void __launch_bounds__(kQuant) k_quantize(const T *x, int64_t x_stride, int64_t dim, int8_t *q, int64_t q_stride,
                                                     float *scale, bool wide)
{
    const int64_t t = blockIdx.x;
    const T *row = x + t * x_stride;
    int8_t *out = q + t * q_stride;
    uint32_t most = 0;
    const int64_t whole = wide ? dim / 8 : 0;
    for (int64_t i = threadIdx.x; i < whole; i += kQuant) {
        const Eight<uint16_t> v = ((const Eight<uint16_t> *)row)[i];
#pragma unroll
        for (int j = 0; j < 8; ++j) most = max(most, (uint32_t)(v[j] & 0x7fff));
    }
    for (int64_t i = whole * 8 + threadIdx.x; i < dim; i += kQuant) most = max(most, (uint32_t)(((const uint16_t *)row)[i] & 0x7fff));
    __shared__ uint32_t s_most[kQuant / 64];
    most = wave_max(most);
    if (lane_id() == 0) s_most[threadIdx.x >> 6] = most;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kQuant / 64; ++w) most = max(most, s_most[w]);
    const bool bad = most >= kInf<T>;
    const uint16_t bits = (uint16_t)most;
    float a = (float)__builtin_bit_cast(T, bits);
    if (threadIdx.x == 0) scale[t] = bad ? __builtin_nanf("") : a / 127.0f;
    // 127 times the largest bfloat16 is no 32-bit number
    const float small = a >= 0x1p100f ? 0x1p-20f : 1.0f;
    a *= small;
    auto whole_of = [&](T v) -> int8_t { return bad || a == 0.0f ? 0 : (int8_t)(int)rintf((float)v * small * 127.0f / a); };
    for (int64_t i = threadIdx.x; i < whole; i += kQuant) {
        const Eight<T> v = ((const Eight<T> *)row)[i];
        Eight<int8_t> r;
#pragma unroll
        for (int j = 0; j < 8; ++j) r[j] = whole_of(v[j]);
        ((Eight<int8_t> *)out)[i] = r;
    }
    for (int64_t i = whole * 8 + threadIdx.x; i < dim; i += kQuant) out[i] = whole_of(row[i]);
}

hipError_t launch_quantize(const Launch &L, const void *x, int64_t x_stride, int64_t n, int64_t dim, int32_t dtype,
                           int8_t *q, int64_t q_stride, float *scale)
{
    const bool wide = ((uintptr_t)x & 15) == 0 && x_stride % 8 == 0 && ((uintptr_t)q & 7) == 0 && q_stride % 8 == 0;
    if (dtype == RO_BF16)
        RO_LAUNCH(L, RO_K_QUANTIZE, k_quantize<__bf16>, dim3((unsigned)n), dim3(kQuant), 0, L.stream, (const __bf16 *)x,
                  x_stride, dim, q, q_stride, scale, wide);
    else
        RO_LAUNCH(L, RO_K_QUANTIZE, k_quantize<_Float16>, dim3((unsigned)n), dim3(kQuant), 0, L.stream, (const _Float16 *)x,
                  x_stride, dim, q, q_stride, scale, wide);
    return hipGetLastError();
}

}  // namespace ro
