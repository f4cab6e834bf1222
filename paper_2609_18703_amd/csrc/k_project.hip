// The product of 8-bit rows and 8-bit weights, with a scale for each row and
// each channel.
//
// A matrix instruction takes weights as its rows and tokens as its columns, so
// that a lane ends with four neighbouring channels of one token.  Sums are
// whole numbers in 32 bits: no order of theirs matters.
//
// k_project_tile: stages of every row's next 128 bytes go from memory to LDS
// without a register in between, whole cache lines at a time (half lines: 811
// and not 762 us for 12,001 tokens, 16,384 channels and rows of 4,096), while
// the matrix instructions work on the stage before.  A slice's LDS reads are
// issued before the products of the slice before; a stage's last products run
// behind its only barrier.  There, a tile of 256 x 256 by eight waves reaches
// 2.2 to 2.3 10^15 operations a second (a library's integer product 2.16, without
// scales): the matrix units are busy for 61% of the time, at a clock that
// power holds at 1.6 to 1.7 GHz.  What else a tile costs, its first loads and its way
// out through LDS, is a tenth.
//
// k_project_few: too few tiles to fill the chip, and rows long enough to share among waves.
#include "ro_mfma.h"
#include "ro_step.h"

namespace ro {

namespace {

using i32x4 = int __attribute__((ext_vector_type(4)));
using i32x16 = int __attribute__((ext_vector_type(16)));

constexpr int kStep = 128;               // bytes of every row in a stage: a line

// Piece (16 bytes) p of a stage's row r is kept at piece p ^ swizzle(r): the
// sixteen rows that LDS hands out at a time then lie in all its banks.
__device__ __forceinline__ int swizzle(int r) { return (r >> 1) & 7; }

// What the wave's lanes have written to LDS is there for its other lanes, and what they have read may be written
// again: the hardware keeps a wave's LDS instructions in order, and this the compiler.  (No instruction.)
__device__ __forceinline__ void lanes_in_order()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

template <typename T>
__device__ __forceinline__ T scaled(int sum, float a, float w, float b)
{
    // (alike in every kernel, and everywhere in a tile: a row's result does not depend on the others)
    float r = __builtin_fmaf((float)sum * a, w, b);
    asm("" : "+v"(r));       // (or else some are rounded to 16 bits at once, by an instruction that does both)
    return (T)r;
}

}  // namespace

// A tile of kN channels and kM tokens; its waves lie kWavesN by kWavesM.
// kOnce: there is one tile of tokens, and so the weights are read once.
template <typename T, int kN, int kM, int kWavesN, int kWavesM, int kStages, bool kOnce>
__global__ void __launch_bounds__(kWavesN * kWavesM * 64) k_project_tile(Product p, int32_t tiles_n, int32_t tiles_m)
{
    constexpr int kWaves = kWavesN * kWavesM;
    constexpr int kTn = kN / kWavesN / 32, kTm = kM / kWavesM / 32;       // a wave's blocks of 32
    constexpr int kPieces = kStep / 16, kRows = 64 / kPieces;               // rows that a load of a wave covers
    constexpr int kLoadN = kN / kRows / kWaves, kLoadM = kM / kRows / kWaves;   // a wave's loads of a stage
    constexpr int kLoads = kLoadN + kLoadM;
    constexpr uint32_t kStage = (kN + kM) * kStep;
    static_assert(kLoadN * kRows * kWaves == kN && kLoadM * kRows * kWaves == kM, "whole loads");
    const int lane = lane_id(), wave = uni32(threadIdx.x >> 6);
    const int wn = wave % kWavesN, wm = wave / kWavesN;
    const int32_t id = blockIdx.x;
    const int64_t n0 = (int64_t)(id % tiles_n) * kN, m0 = (int64_t)(id / tiles_n) * kM;
    const int32_t rows_n = (int32_t)min64(kN, p.n - n0), rows_m = (int32_t)min64(kM, p.m - m0);
    const int8_t *w = p.w + n0 * p.w_stride, *a = p.a + m0 * p.a_stride;

    // where the lane's pieces of a stage come from; rows beyond the last one repeat it
    uint32_t from[kLoads];
    {
        const int r = lane / kPieces;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const bool is_w = i < kLoadN;
            const int row = ((is_w ? i : i - kLoadN) * kWaves + wave) * kRows + r;
            const int last = (is_w ? rows_n : rows_m) - 1;
            from[i] = (uint32_t)min(row, last) * (uint32_t)(is_w ? p.w_stride : p.a_stride) + ((lane % kPieces) ^ swizzle(row)) * 16;
        }
    }
    const uint32_t base = lds_base();
    // (read once, every workgroup's weights from another place of their rows on: those of 4,096 bytes, and of many such
    // lengths, lie in the same channels of memory at the same place)
    const int32_t steps = p.k / kStep, turn = kOnce ? id % max(steps, 1) : 0;
    auto load_one = [&](int32_t t, int i) {
        const uint32_t to = base + (uint32_t)(t % kStages) * kStage + wave * 1024;
        const bool is_w = i < kLoadN;
        const int32_t turned = t + turn < steps ? t + turn : t + turn - steps;
        const int8_t *g = (is_w ? w : a) + (int64_t)turned * kStep;
        const uint32_t at = to + (is_w ? i * kWaves * 1024 : kN * kStep + (i - kLoadN) * kWaves * 1024);
        if (kOnce && is_w) load_once_to_lds(g, from[i], at);
        else load_to_lds(g, from[i], at);
    };
    auto load = [&](int32_t t) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) load_one(t, i);
    };
    // the lane's row of a block of 32, and the 16-byte pieces of it that products take
    const uint32_t own = (uint32_t)(lane & 31) * kStep;
    constexpr int kSlices = kStep / 32;
    uint32_t piece[kSlices];
#pragma unroll
    for (int s = 0; s < kSlices; ++s) piece[s] = own + ((uint32_t)(s * 2 + (lane >> 5)) ^ swizzle(lane & 31)) * 16;
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
    // `between` is called after every row of blocks: the compiler keeps this
    // order, so that LDS reads and loads are under way while products run
    auto multiply = [&](const Frags &f, auto between) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < kTn; ++i) {
#pragma unroll
            for (int j = 0; j < kTm; ++j) sum[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(f.w[i], f.a[j], sum[i][j], 0, 0, 0);
            between(i);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto nothing = [](int) {};

    if (steps > 0) {
        for (int32_t t = 0; t < min(steps, kStages); ++t) load(t);
        // (wait and barrier in one, which no LDS read of the first stage may pass)
        if (steps >= kStages) asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" : : "n"((kStages - 1) * kLoads) : "memory");
        else tile_barrier();
        Frags f[2];
        read(0, 0, f[0]);
        auto stage = [&](int32_t t, auto wait, auto next, auto between) {
#pragma unroll
            for (int s = 0; s + 1 < kSlices; ++s) {
                read(t, s + 1, f[(s + 1) & 1]);
                multiply(f[s & 1], nothing);
            }
            wait();          // the next stage is there, and all waves have read this one
            next();
            multiply(f[1], between);
        };
        int32_t t = 0;
        for (; t + kStages < steps; ++t)
            stage(t, [] { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"((kStages - 2) * kLoads) : "memory"); },
                  [&] { read(t + 1, 0, f[0]); },
                  [&](int i) {
#pragma unroll
                      for (int l = i * kLoads / kTn; l < (i + 1) * kLoads / kTn; ++l) load_one(t + kStages, l);
                  });
        for (; t < steps; ++t)
            stage(t, [] { tile_barrier(); }, [&] { if (t + 1 < steps) read(t + 1, 0, f[0]); }, nothing);
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
        multiply(f, nothing);
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
    lanes_in_order();
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
        lanes_in_order();                // (the wave's own part of LDS)
        const int32_t rows = (int32_t)max64(0, min64(32, p.m - t0));
        if (wide) {
            constexpr int kWide = kCols / kPer;                             // of a row
            for (int32_t i = lane; i < rows * kWide; i += 64) {
                const int32_t row = i / kWide, at = i % kWide * kPer;
                *(u32x4 *)((T *)p.out + (t0 + row) * p.out_stride + nw + at) = *(const u32x4 *)(room + row * kRow + at * sizeof(T));
            }
        } else {
            for (int32_t i = lane; i < rows * kCols; i += 64) {
                const int32_t row = i / kCols, at = i % kCols;
                if (at < cols) ((T *)p.out)[(t0 + row) * p.out_stride + nw + at] = *(const T *)(room + row * kRow + at * sizeof(T));
            }
        }
        lanes_in_order();
    }
}

// Few tokens: 16 kBn channels and 16 kBm tokens a workgroup, whose waves share
// the rows' length; their sums, whole numbers, are added in LDS.  Weights go
// from memory to registers, kAhead pieces of a row ahead.
constexpr int kFewWaves = 16;
template <typename T, int kBn, int kBm, int kAhead>
__global__ void __launch_bounds__(kFewWaves * 64) k_project_few(Product p)
{
    __shared__ i32x4 s_sum[kFewWaves][kBn * kBm][64];
    const int lane = lane_id(), wave = uni32(threadIdx.x >> 6), r = lane & 15, part = lane >> 4;
    const int64_t n0 = (int64_t)blockIdx.x * (16 * kBn), m0 = (int64_t)blockIdx.y * (16 * kBm);
    const int8_t *w[kBn], *a[kBm];
#pragma unroll
    for (int i = 0; i < kBn; ++i) w[i] = p.w + min64(n0 + i * 16 + r, p.n - 1) * p.w_stride + part * 16;
#pragma unroll
    for (int j = 0; j < kBm; ++j) a[j] = p.a + min64(m0 + j * 16 + r, p.m - 1) * p.a_stride + part * 16;
    // a wave's steps of 64 bytes follow one another
    const int32_t steps = (p.k + 63) / 64, each = (steps + kFewWaves - 1) / kFewWaves;
    const int32_t first = wave * each, end = min(steps, first + each);
    i32x4 sum[kBn][kBm] = {};
    struct Steps {
        i32x4 w[kAhead][kBn], a[kAhead][kBm];
    };
    auto load = [&](int32_t t0, Steps &f) {
#pragma unroll
        for (int t = 0; t < kAhead; ++t) {
            // (steps behind the wave's last one, and pieces behind the rows' end, are read from their start and count as zeros)
            const int32_t k = (t0 + t) * 64;
            const bool have = t0 + t < end && k + part * 16 < p.k;
            const int32_t at = have ? k : part * 16 < p.k ? 0 : -part * 16;
#pragma unroll
            for (int i = 0; i < kBn; ++i) f.w[t][i] = *(const i32x4 *)(w[i] + at);
#pragma unroll
            for (int j = 0; j < kBm; ++j) {
                f.a[t][j] = *(const i32x4 *)(a[j] + at);
                if (!have) f.a[t][j] = i32x4{0, 0, 0, 0};
            }
        }
    };
    auto multiply = [&](const Steps &f) {
#pragma unroll
        for (int t = 0; t < kAhead; ++t)
#pragma unroll
            for (int i = 0; i < kBn; ++i)
#pragma unroll
                for (int j = 0; j < kBm; ++j)
                    sum[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(f.w[t][i], f.a[t][j], sum[i][j], 0, 0, 0);
    };
    if (first < end) {
        Steps f, g;
        load(first, f);
        for (int32_t t0 = first; t0 < end; t0 += 2 * kAhead) {
            if (t0 + kAhead < end) load(t0 + kAhead, g);
            multiply(f);
            if (t0 + kAhead >= end) break;
            if (t0 + 2 * kAhead < end) load(t0 + 2 * kAhead, f);
            multiply(g);
        }
    }
#pragma unroll
    for (int i = 0; i < kBn; ++i)
#pragma unroll
        for (int j = 0; j < kBm; ++j) s_sum[wave][i * kBm + j][lane] = sum[i][j];
    __syncthreads();
    for (int b = wave; b < kBn * kBm; b += kFewWaves) {
        i32x4 all = s_sum[0][b][lane];
#pragma unroll
        for (int v = 1; v < kFewWaves; ++v) all += s_sum[v][b][lane];
        const int64_t t = m0 + b % kBm * 16 + r, c = n0 + b / kBm * 16 + part * 4;
        if (t >= p.m || c >= p.n) continue;
        const float as = p.a_scale[t];
        T *out = (T *)p.out + t * p.out_stride + c;
        T v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int64_t ce = min64(c + e, p.n - 1);
            v[e] = scaled<T>(all[e], as, p.w_scale[ce], p.bias ? p.bias[ce] : 0.0f);
        }
        if (c + 4 <= p.n && ((uintptr_t)out & (4 * sizeof(T) - 1)) == 0) {
            __builtin_memcpy(__builtin_assume_aligned(out, 4 * sizeof(T)), v, sizeof(v));
        } else {
            for (int e = 0; e < 4 && c + e < p.n; ++e) out[e] = v[e];
        }
    }
}

template <typename T, int kBn, int kBm, int kAhead>
hipError_t launch_few(const Launch &L, const Product &p)
{
    const dim3 grid((unsigned)((p.n + 16 * kBn - 1) / (16 * kBn)), (unsigned)((p.m + 16 * kBm - 1) / (16 * kBm)));
    RO_LAUNCH(L, RO_K_PROJECT, (k_project_few<T, kBn, kBm, kAhead>), grid, dim3(kFewWaves * 64), 0, L.stream, p);
    return hipGetLastError();
}

template <typename T, int kN, int kM, int kWavesN, int kWavesM, int kStages, bool kOnce = false>
hipError_t launch_tile(const Launch &L, const Product &p)
{
    const int64_t tn = (p.n + kN - 1) / kN, tm = (p.m + kM - 1) / kM;
    constexpr unsigned stages = kStages * (kN + kM) * kStep;
    constexpr unsigned rows = kWavesN * kWavesM * (32 * (kN / kWavesN * sizeof(T) + 16) + 8 * (kN / kWavesN));
    constexpr unsigned bytes = stages > rows ? stages : rows;
    if (tn * tm * (kWavesN * kWavesM * 64) >= ((int64_t)1 << 32)) return hipErrorInvalidValue;
    RO_LAUNCH(L, RO_K_PROJECT, (k_project_tile<T, kN, kM, kWavesN, kWavesM, kStages, kOnce>), dim3((unsigned)(tn * tm)),
              dim3(kWavesN * kWavesM * 64), bytes, L.stream, p, (int32_t)tn, (int32_t)tm);
    return hipGetLastError();
}

// Of the tiles, the one whose rounds over the chip should take least.  A round
// is a tile on each of 256 CUs; its time grows with the rows' length alike for
// all, and was measured at 4,096 (us, where every CU has one; of those in pairs
// half of a pair's): 64 channels x 32 tokens 6, 64 x 64 9, 128 x 64 14, 128 x
// 128 20 by eight waves and four stages, 19 by four waves and two stages, of
// which two workgroups fit a CU, 256 x 128 33, 256 x 256 50.  So 777 tokens
// and 4,096 channels take 20.6 us by the rule (128 x 128), 25 to 44 by the
// others; 3,000 take 52 (256 x 256) and 60 to 107; 100 take 8.8 and 9.6 to 42.
// (Of short rows the first loads and the way out, which have nothing beside them, weigh more than
// the rule says: 777, 3,000 and 6,000 tokens of 1,024 onto 28,000 channels take 53, 131 and 241 us, where
// the products alone would take 21, 80 and 159.  Long rows are not split over workgroups: 256 tokens of
// 8,192 onto 2,048 channels take 17 us, four times what the weights' way from memory does.)
template <typename T>
hipError_t launch_typed(const Launch &L, const Product &p)
{
    // Few tokens and channels, so that a round of workgroups has all: 6.2 us for one
    // token and 4,096 channels (64 x 32: 8.4), 6.9 for five and 4,608 of 3,584 (7.8), 6.2 and 9.6 for 8,192 (9 and 13).
    // Behind the limits there are fewer tiles than CUs again: with weights from memory, five tokens and 8,192 channels of
    // 4,096 take 10.3 us, 8,193 11.6, 12,000 12.2 and 16,384 14.5; 4,608 channels are 144 workgroups for 256 CUs.
    if (p.m <= 16 && p.n <= 16 * L.num_cus) return launch_few<T, 1, 1, 4>(L, p);
    if (p.m <= 16 && p.n <= 32 * L.num_cus) return launch_few<T, 2, 1, 2>(L, p);
    // So with more tokens, where rows are long: of 4,096, with weights from memory, 32 tokens and 4,096 channels 8.9 us
    // (64 x 32: 10.9), 64 and 2,048 7.8 (64 x 64: 11.8), 128 and 1,024 7.8 (8.5); of 1,024 5.1 (4.1 to 5.5).
    if (p.m > 16 && p.k >= 1536 && (p.n + 15) / 16 * ((p.m + 31) / 32) <= L.num_cus) return launch_few<T, 1, 2, 2>(L, p);
    // One tile of tokens: the weights are read once, past the caches.  150,001 channels of 4,096 for 16 tokens 110 us,
    // 5.6 TB/s (through the caches 123; tiles of 128 channels 142), for 64 tokens 138 (140; 157).  Not where half of
    // the chip would have no tile: 64 tokens and 8,192 channels of 8,192 take 21.6 us by the rule below, 22.8 so, and
    // 64 and 12,000 of 4,096 14.7 and 13.7.
    // Where tiles of 64 channels are too few, a wave has 32 and eight stages on their way: 32 tokens and 8,000 channels
    // of 4,096 9.8 us (64 x 32: 11.9), 20 and 8,192 of 8,192 16.7 (19.4).  At the limit 20 tokens go from 9.5 us (8,192
    // channels of 4,096) to 12.2 (8,193: 129 tiles of two waves) and 12.6 (12,000).
    if (p.m <= 32 && p.n <= 32 * L.num_cus) return launch_tile<T, 32, 32, 1, 1, 8, true>(L, p);
    if (p.m <= 32) return launch_tile<T, 64, 32, 2, 1, 4, true>(L, p);
    if (p.m <= 64 && (p.n + 63) / 64 > L.num_cus / 2) return launch_tile<T, 64, 64, 2, 2, 4, true>(L, p);
    auto rounds = [&](int64_t n, int64_t m) {
        return ((p.n + n - 1) / n * ((p.m + m - 1) / m) + L.num_cus - 1) / L.num_cus;
    };
    const int64_t pairs = rounds(128, 128);
    const int64_t cost[] = {6 * rounds(64, 32),  9 * rounds(64, 64),   14 * rounds(128, 64),           20 * pairs,
                            pairs > 1 ? 19 * pairs : 23, 33 * rounds(256, 128), 50 * rounds(256, 256)};
    int best = 0;
    for (int i = 1; i < 7; ++i)
        if (cost[i] < cost[best]) best = i;
    switch (best) {
    case 0: return launch_tile<T, 64, 32, 2, 1, 4>(L, p);
    case 1: return launch_tile<T, 64, 64, 2, 2, 4>(L, p);
    case 2: return launch_tile<T, 128, 64, 2, 2, 4>(L, p);
    case 3: return launch_tile<T, 128, 128, 2, 4, 4>(L, p);
    case 4: return launch_tile<T, 128, 128, 2, 2, 2>(L, p);
    case 5: return launch_tile<T, 256, 128, 4, 2, 3>(L, p);
    default: return launch_tile<T, 256, 256, 2, 4, 2>(L, p);
    }
}

hipError_t launch_project(const Launch &L, const Product &p, int32_t dtype)
{
    if (dtype == RO_BF16) return launch_typed<__bf16>(L, p);
    if (dtype == RO_F16) return launch_typed<_Float16>(L, p);
    return launch_typed<float>(L, p);
}

}  // namespace ro
