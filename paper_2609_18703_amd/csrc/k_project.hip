// The product of 8-bit rows and 8-bit weights, with a scale for each row and
// each channel.
//
// A matrix instruction takes weights as its rows and tokens as its columns, so
// that a lane ends with four neighbouring channels of one token.
#include "ro_mfma.h"
#include "ro_step.h"

namespace ro {

namespace {

using i32x4 = int __attribute__((ext_vector_type(4)));
using i32x16 = int __attribute__((ext_vector_type(16)));

constexpr int kStep = 64;            // bytes of every row that a stage holds
constexpr int kStages = 4;

// Piece (16 bytes) p of a stage's row r is kept at piece p ^ swizzle(r): the
// eight rows that LDS hands out at a time then lie in all its banks.
__device__ __forceinline__ int swizzle(int r) { return (r >> 1) & 3; }

template <typename T>
__device__ __forceinline__ T scaled(int sum, float a, float w, float b)
{
    return (T)((float)sum * a * w + b);
}

}  // namespace

// A tile of kN channels and kM tokens; its waves lie kWavesN by kWavesM.
template <typename T, int kN, int kM, int kWavesN, int kWavesM>
__global__ void __launch_bounds__(kWavesN * kWavesM * 64) k_project_tile(Product p, int32_t tiles_n, int32_t tiles_m)
{
    constexpr int kWaves = kWavesN * kWavesM;
    constexpr int kTn = kN / kWavesN / 32, kTm = kM / kWavesM / 32;       // a wave's blocks of 32
    constexpr int kLoadN = kN / 16 / kWaves, kLoadM = kM / 16 / kWaves;   // a wave's loads of a stage
    constexpr int kLoads = kLoadN + kLoadM;
    constexpr uint32_t kStage = (kN + kM) * kStep;
    static_assert(kLoadN * 16 * kWaves == kN && kLoadM * 16 * kWaves == kM, "");
    const int lane = lane_id(), wave = uni32(threadIdx.x >> 6);
    const int wn = wave % kWavesN, wm = wave / kWavesN;
    const int32_t id = blockIdx.x;
    const int64_t n0 = (int64_t)(id % tiles_n) * kN, m0 = (int64_t)(id / tiles_n) * kM;
    const int32_t rows_n = (int32_t)min64(kN, p.n - n0), rows_m = (int32_t)min64(kM, p.m - m0);
    const int8_t *w = p.w + n0 * p.w_stride, *a = p.a + m0 * p.a_stride;

    // where the lane's pieces of a stage come from; rows beyond the last one repeat it
    uint32_t from[kLoads];
    {
        const int r = lane >> 2;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const bool is_w = i < kLoadN;
            const int row = ((is_w ? i : i - kLoadN) * kWaves + wave) * 16 + r;
            const int last = (is_w ? rows_n : rows_m) - 1;
            from[i] = (uint32_t)min(row, last) * (uint32_t)(is_w ? p.w_stride : p.a_stride) + ((lane & 3) ^ swizzle(row)) * 16;
        }
    }
    const uint32_t base = lds_base();
    auto load = [&](int32_t t) {
        const uint32_t to = base + (uint32_t)(t % kStages) * kStage + wave * 1024;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const bool is_w = i < kLoadN;
            load_to_lds((is_w ? w : a) + (int64_t)t * kStep, from[i],
                        to + (is_w ? i * kWaves * 1024 : kN * kStep + (i - kLoadN) * kWaves * 1024));
        }
    };
    // the lane's row of a block of 32, and the two 16-byte pieces of it that a product takes
    const uint32_t own = (uint32_t)(lane & 31) * kStep;
    uint32_t piece[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) piece[s] = own + ((uint32_t)(s * 2 + (lane >> 5)) ^ swizzle(lane & 31)) * 16;
    const uint32_t block_w = base + wn * kTn * 32 * kStep, block_a = base + kN * kStep + wm * kTm * 32 * kStep;
    struct Frags {
        i32x4 w[kTn], a[kTm];
    };
    auto lds_piece = [](uint32_t at) { return *(const __attribute__((address_space(3))) i32x4 *)(uintptr_t)at; };
    auto read = [&](int32_t t, int s, Frags &f) {
        const uint32_t at = (uint32_t)(t % kStages) * kStage + piece[s];
#pragma unroll
        for (int i = 0; i < kTn; ++i) f.w[i] = lds_piece(block_w + at + i * 32 * kStep);
#pragma unroll
        for (int i = 0; i < kTm; ++i) f.a[i] = lds_piece(block_a + at + i * 32 * kStep);
    };
    i32x16 sum[kTn][kTm];
#pragma unroll
    for (int i = 0; i < kTn; ++i)
#pragma unroll
        for (int j = 0; j < kTm; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) sum[i][j][e] = 0;
    auto multiply = [&](const Frags &f) {
#pragma unroll
        for (int i = 0; i < kTn; ++i)
#pragma unroll
            for (int j = 0; j < kTm; ++j) sum[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(f.w[i], f.a[j], sum[i][j], 0, 0, 0);
    };

    const int32_t steps = p.k / kStep;
    if (steps > 0) {
        for (int32_t t = 0; t < min(steps, kStages - 1); ++t) load(t);
        if (steps >= kStages - 1) wait_loads<(kStages - 2) * kLoads>();
        else wait_loads<0>();
        __builtin_amdgcn_s_barrier();
        Frags f0, f1;
        read(0, 0, f0);
        int32_t t = 0;
        for (; t + kStages - 1 < steps; ++t) {
            read(t, 1, f1);
            load(t + kStages - 1);
            multiply(f0);
            // the next stage is there, and all waves have read this one
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"((kStages - 2) * kLoads) : "memory");
            read(t + 1, 0, f0);
            multiply(f1);
        }
        for (; t < steps; ++t) {
            read(t, 1, f1);
            multiply(f0);
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" : : : "memory");
            if (t + 1 < steps) read(t + 1, 0, f0);
            multiply(f1);
        }
    }
    // what the last stage would not be filled by: zeros beyond the rows' end
    for (int32_t k = steps * kStep; k < p.k; k += 32) {
        const int32_t at = k + (lane >> 5) * 16;
        Frags f;
#pragma unroll
        for (int i = 0; i < kTn; ++i) {
            const int32_t row = min((wn * kTn + i) * 32 + (lane & 31), rows_n - 1);
            f.w[i] = i32x4{0, 0, 0, 0};
            if (at < p.k) f.w[i] = *(const i32x4 *)(w + row * p.w_stride + at);
        }
#pragma unroll
        for (int i = 0; i < kTm; ++i) {
            const int32_t row = min((wm * kTm + i) * 32 + (lane & 31), rows_m - 1);
            f.a[i] = i32x4{0, 0, 0, 0};
            if (at < p.k) f.a[i] = *(const i32x4 *)(a + row * p.a_stride + at);
        }
        multiply(f);
    }

    // 32 tokens of the wave's channels at a time go through LDS, so that rows are written in wide pieces
    __syncthreads();
    constexpr int kCols = kTn * 32;
    constexpr int kPer = 16 / (int)sizeof(T);                               // elements of 16 bytes
    constexpr uint32_t kRow = kCols * sizeof(T) + 16;
    char *room = lds + wave * (32 * kRow);
    const int64_t nw = n0 + wn * kCols;
    const int32_t cols = (int32_t)max64(0, min64(kCols, p.n - nw));
    const bool wide = ((uintptr_t)p.out & 15) == 0 && p.out_stride % kPer == 0 && cols == kCols;
    // the wave's channels' scales and biases lie beside them
    float *scales = (float *)(lds + kWaves * (32 * kRow)) + wave * (2 * kCols);
    for (int i = lane; i < kCols; i += 64) {
        const int64_t c = min64(nw + i, p.n - 1);
        scales[i] = p.w_scale[c];
        scales[kCols + i] = p.bias ? p.bias[c] : 0.0f;
    }
#pragma unroll
    for (int j = 0; j < kTm; ++j) {
        const int64_t t0 = m0 + (wm * kTm + j) * 32;
        const float as = p.a_scale[min64(t0 + (lane & 31), p.m - 1)];
#pragma unroll
        for (int i = 0; i < kTn; ++i)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int c = i * 32 + g * 8 + (lane >> 5) * 4;
                const f32x4 ws = *(const f32x4 *)(scales + c), bs = *(const f32x4 *)(scales + kCols + c);
                Vec4<T> v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = scaled<T>(sum[i][j][g * 4 + e], as, ws[e], bs[e]);
                *(Vec4<T> *)(room + (lane & 31) * kRow + c * sizeof(T)) = v;
            }
        // (the wave's own part of LDS: its writes and reads follow one another)
        const int32_t rows = (int32_t)max64(0, min64(32, p.m - t0));
        if (wide) {
            constexpr int kPieces = kCols / kPer;                           // of a row
            for (int32_t i = lane; i < rows * kPieces; i += 64) {
                const int32_t row = i / kPieces, at = i % kPieces * kPer;
                *(u32x4 *)((T *)p.out + (t0 + row) * p.out_stride + nw + at) = *(const u32x4 *)(room + row * kRow + at * sizeof(T));
            }
        } else {
            for (int32_t i = lane; i < rows * kCols; i += 64) {
                const int32_t row = i / kCols, at = i % kCols;
                if (at < cols) ((T *)p.out)[(t0 + row) * p.out_stride + nw + at] = *(const T *)(room + row * kRow + at * sizeof(T));
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
}

template <typename T, int kN, int kM, int kWavesN, int kWavesM>
hipError_t launch_tile(const Launch &L, const Product &p)
{
    const int64_t tn = (p.n + kN - 1) / kN, tm = (p.m + kM - 1) / kM;
    constexpr unsigned stages = kStages * (kN + kM) * kStep;
    constexpr unsigned rows = kWavesN * kWavesM * (32 * (kN / kWavesN * sizeof(T) + 16) + 8 * (kN / kWavesN));
    constexpr unsigned bytes = stages > rows ? stages : rows;
    RO_LAUNCH(L, RO_K_PROJECT, (k_project_tile<T, kN, kM, kWavesN, kWavesM>), dim3((unsigned)(tn * tm)),
              dim3(kWavesN * kWavesM * 64), bytes, L.stream, p, (int32_t)tn, (int32_t)tm);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_typed(const Launch &L, const Product &p)
{
    if (p.m <= 64) return launch_tile<T, 128, 64, 4, 1>(L, p);
    if (p.m <= 1024) return launch_tile<T, 128, 128, 2, 2>(L, p);
    return launch_tile<T, 256, 256, 2, 2>(L, p);
}

hipError_t launch_project(const Launch &L, const Product &p, int32_t dtype)
{
    if (dtype == RO_BF16) return launch_typed<__bf16>(L, p);
    if (dtype == RO_F16) return launch_typed<_Float16>(L, p);
    return launch_typed<float>(L, p);
}

}  // namespace ro
