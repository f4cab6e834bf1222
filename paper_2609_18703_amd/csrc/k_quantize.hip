// Rows of 16-bit values to 8-bit integers with one scale each.
//
// q = rint(127 x / a), a the row's largest magnitude, as if the quotient were
// exact.  127 x has at most 18 bits, and a quotient of such numbers that is not
// halfway between two integers lies at least 2^-19 of itself away from there, far
// more than any error here.  A quotient that is halfway has 8 bits: 127 x times
// the reciprocal of a is off by less than 2^-22 of it, what that leaves of 127 x
// is exact, and added as a part of a it leaves the quotient itself.  (Four
// instructions, where a division takes a dozen.)  Both are taken at a's power
// of two, where neither the products nor the reciprocal leave the range.
//
// One workgroup a row, or one wave where it has 2,048 elements at most (12,001 rows
// of 1,024: 9.7 us, 13.8 in workgroups).  The row is held in registers, but where
// it has more than 16,384 elements or is not aligned, where it is read again (3,000
// rows of 12,288: 28 us so, 21 held).  Bound by memory: 12,001 rows of 4,096 take 24
// us, 6.0 TB/s read and written, part of it in the cache; five rows of 3,584 take
// 2.9 us, the way to memory and back.
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

// kOf: threads of a row, a workgroup or a wave of one.  kHold: pieces of eight
// elements that a thread holds; 0: any number.
template <typename T, int kOf, int kHold>
__global__ void __launch_bounds__(kQuant) k_quantize(const T *x, int64_t x_stride, int64_t n_rows, int64_t dim,
                                                     int8_t *q, int64_t q_stride, float *scale, bool wide)
{
    const int64_t t = kOf == 64 ? blockIdx.x * (int64_t)(kQuant / 64) + uni32(threadIdx.x >> 6) : blockIdx.x;
    const int tid = threadIdx.x % kOf;
    if (kOf == 64 && t >= n_rows) return;
    const T *row = x + t * x_stride;
    int8_t *out = q + t * q_stride;
    uint32_t most = 0;
    const int64_t whole = wide ? dim / 8 : 0;
    Eight<uint16_t> held[kHold ? kHold : 1];
    auto look_at = [&](const Eight<uint16_t> &v) {
#pragma unroll
        for (int j = 0; j < 8; ++j) most = max(most, (uint32_t)(v[j] & 0x7fff));
    };
    if (kHold) {
        // (all on their way at once; a thread without one has the last one again)
#pragma unroll
        for (int i = 0; i < kHold; ++i)
            held[i] = ((const Eight<uint16_t> *)row)[min(tid + i * kOf, (int)whole - 1)];
#pragma unroll
        for (int i = 0; i < kHold; ++i) look_at(held[i]);
    } else {
        for (int64_t i = tid; i < whole; i += kOf) look_at(((const Eight<uint16_t> *)row)[i]);
    }
    for (int64_t i = whole * 8 + tid; i < dim; i += kOf) most = max(most, (uint32_t)(((const uint16_t *)row)[i] & 0x7fff));
    most = wave_max(most);
    if constexpr (kOf > 64) {
        __shared__ uint32_t s_most[kOf / 64];
        if (lane_id() == 0) s_most[threadIdx.x >> 6] = most;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kOf / 64; ++w) most = max(most, s_most[w]);
    }
    const bool bad = most >= kInf<T>;
    const uint16_t bits = (uint16_t)most;
    const float a = (float)__builtin_bit_cast(T, bits);
    if (tid == 0) scale[t] = bad ? __builtin_nanf("") : a / 127.0f;
    int up = 0;
    const float least = bad ? 0.0f : frexpf(a, &up), part = least > 0.0f ? 1.0f / least : 0.0f;
    auto whole_of = [&](T v) -> int8_t {
        const float n = ldexpf((float)v, -up) * 127.0f, about = n * part;
        const float left = __builtin_fmaf(-about, least, n);
        return (int8_t)(int)rintf(__builtin_fmaf(left, part, about));
    };
    auto write = [&](int64_t i, const Eight<uint16_t> &v) {
        Eight<int8_t> r;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint16_t b = v[j];
            r[j] = bad ? 0 : whole_of(__builtin_bit_cast(T, b));
        }
        ((Eight<int8_t> *)out)[i] = r;
    };
    if (kHold) {
#pragma unroll
        for (int i = 0; i < kHold; ++i)
            if (tid + i * kOf < whole) write(tid + i * kOf, held[i]);
    } else {
        for (int64_t i = tid; i < whole; i += kOf) write(i, ((const Eight<uint16_t> *)row)[i]);
    }
    for (int64_t i = whole * 8 + tid; i < dim; i += kOf) out[i] = bad ? 0 : whole_of(row[i]);
}

template <typename T>
hipError_t launch_typed(const Launch &L, const void *x, int64_t x_stride, int64_t n, int64_t dim, int8_t *q, int64_t q_stride,
                        float *scale)
{
    const bool wide = ((uintptr_t)x & 15) == 0 && x_stride % 8 == 0 && ((uintptr_t)q & 7) == 0 && q_stride % 8 == 0;
    const int64_t whole = wide ? dim / 8 : 0;
#define RO_QUANTIZE(kOf, kHold)                                                                                            \
    RO_LAUNCH(L, RO_K_QUANTIZE, (k_quantize<T, kOf, kHold>), dim3((unsigned)((n * kOf + kQuant - 1) / kQuant)), dim3(kQuant), \
              0, L.stream, (const T *)x, x_stride, n, dim, q, q_stride, scale, wide)
    if (whole < 1 || whole > 8 * kQuant) RO_QUANTIZE(kQuant, 0);
    else if (whole <= 64) RO_QUANTIZE(64, 1);
    else if (whole <= 4 * 64) RO_QUANTIZE(64, 4);
    else if (whole <= 2 * kQuant) RO_QUANTIZE(kQuant, 2);
    else if (whole <= 4 * kQuant) RO_QUANTIZE(kQuant, 4);
    else RO_QUANTIZE(kQuant, 8);
#undef RO_QUANTIZE
    return hipGetLastError();
}

hipError_t launch_quantize(const Launch &L, const void *x, int64_t x_stride, int64_t n, int64_t dim, int32_t dtype,
                           int8_t *q, int64_t q_stride, float *scale)
{
    return dtype == RO_BF16 ? launch_typed<__bf16>(L, x, x_stride, n, dim, q, q_stride, scale)
                            : launch_typed<_Float16>(L, x, x_stride, n, dim, q, q_stride, scale);
}

}  // namespace ro
