// Building blocks of the attention kernels: matrix instructions of either
// 16-bit type, asynchronous loads into LDS, transposed reads from it.
#pragma once

#include "ro_chunk.h"

namespace ro {

namespace {

extern __shared__ __attribute__((aligned(1024))) char lds[];

using s16x4 = short __attribute__((ext_vector_type(4)));
using s16x8 = short __attribute__((ext_vector_type(8)));
using u32x4 = uint32_t __attribute__((ext_vector_type(4)));

template <typename T>
struct Mma;
template <>
struct Mma<__bf16> {
    static __device__ __forceinline__ f32x16 wide(Vec8<__bf16> a, Vec8<__bf16> b, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x4 narrow(Vec8<__bf16> a, Vec8<__bf16> b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
};
template <>
struct Mma<_Float16> {
    static __device__ __forceinline__ f32x16 wide(Vec8<_Float16> a, Vec8<_Float16> b, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x4 narrow(Vec8<_Float16> a, Vec8<_Float16> b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
    }
};

__device__ __forceinline__ uint32_t lds_base()
{
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
}

// 16 bytes of every lane from `g` to LDS at `to` + 16 * lane, without a
// register in between.  Asynchronous: counted by vmcnt, which only the
// explicit waits below look at.
__device__ __forceinline__ void load_to_lds(const void *g, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(g), "s"(to) : "memory", "m0");
}

// ... from `g` + `at` bytes, where `g` is the same for all lanes.
__device__ __forceinline__ void load_to_lds(const void *g, uint32_t at, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(at), "s"(g), "s"(to) : "memory", "m0");
}

// 4 bytes of every lane from `g` to LDS at `to` + 4 * lane.
__device__ __forceinline__ void load_word_to_lds(const void *g, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" : : "v"(g), "s"(to) : "memory", "m0");
}

template <int N>
__device__ __forceinline__ void wait_loads()
{
    asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
}

// What the waves have loaded is there, and all are done with what they read.
__device__ __forceinline__ void tile_barrier()
{
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" : : : "memory");
}

// The plan's words are read through the scalar cache: no vector load of the
// compiler's then waits behind the asynchronous ones.
template <typename T>
__device__ __forceinline__ T scalar_load(const T *p)
{
    struct Words {
        uint32_t w[sizeof(T) / 4];
    } x;
    const auto *from = (const __attribute__((address_space(4))) uint32_t *)(uintptr_t)p;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 4); ++i) x.w[i] = from[i];
    return __builtin_bit_cast(T, x);
}

template <typename T>
__device__ __forceinline__ Vec8<T> lds_vec(uint32_t at)
{
    return *(const __attribute__((address_space(3))) Vec8<T> *)(uintptr_t)at;
}

// Four rows of a column from a row-major tile: lane i of 16 gives the address
// of row i / 4's elements 4 (i % 4).., and gets rows 0..3 of column i.
template <typename T>
__device__ __forceinline__ Vec8<T> lds_columns(uint32_t a, uint32_t b)
{
    const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(uintptr_t)a);
    const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(uintptr_t)b);
    return __builtin_bit_cast(Vec8<T>, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Where an item's 16-byte pieces of keys and values come from: the wave's 16
// positions of a key tile lie in one page.  Positions beyond the last one
// repeat it, so that nothing is read that the sequence does not own.
template <int D>
struct TileLoad {
    static constexpr int kRowsAt = 64 * 16 / (D * 2);   // rows that one load of the wave covers
    static constexpr int kLoads = 16 / kRowsAt;
    // Piece (16 bytes) p of row r is kept at piece p ^ swizzle(r) of the row,
    // which spreads the pieces that one LDS read touches over all banks:
    // keys are read as 16 rows' same piece, values as 4 rows' same four pieces.
    static __device__ __forceinline__ int key_swizzle(int r) { return D == 128 ? r & 15 : (r >> 1) & 7; }
    static __device__ __forceinline__ int value_swizzle(int r) { return D == 128 ? 4 * (r & 3) : 4 * ((r >> 1) & 1); }

    // Where the lane's pieces of 16 rows are, in bytes from the first row: the
    // same for every tile but one that the last position ends in.
    uint32_t key_at[kLoads], value_at[kLoads];
    int row_in, piece;
    __device__ __forceinline__ TileLoad(const Pages &pg)
    {
        row_in = lane_id() / (64 / kRowsAt);
        piece = lane_id() % (64 / kRowsAt);
#pragma unroll
        for (int l = 0; l < kLoads; ++l) offsets(pg, l, 15, key_at[l], value_at[l]);
    }
    __device__ __forceinline__ void offsets(const Pages &pg, int l, int most, uint32_t &ka, uint32_t &va) const
    {
        const int r = l * kRowsAt + row_in;
        const uint32_t row = (uint32_t)min(r, most) * (uint32_t)pg.slot * 2;
        ka = row + (piece ^ key_swizzle(r)) * 16;
        va = row + (piece ^ value_swizzle(r)) * 16;
    }
    // Keys of 16 positions from j0 (a multiple of 16) on, in page `page`, to LDS at kt, and with kValues
    // their values to vt; positions beyond `last` repeat it.
    template <bool kValues = true>
    __device__ __forceinline__ void load(const Chunk &c, const Pages &pg, int32_t h, uint32_t page, int32_t j0, int32_t last,
                                         uint32_t kt, uint32_t vt) const
    {
        const int32_t from = min(j0, last & ~15);
        const int64_t at = (int64_t)page * pg.page + (int64_t)h * pg.head + (int64_t)(from & ((1 << c.page_shift) - 1)) * pg.slot;
        const uint16_t *kp = (const uint16_t *)pg.k + at, *vp = (const uint16_t *)pg.v + at;
        if (last - from >= 15) {
#pragma unroll
            for (int l = 0; l < kLoads; ++l) {
                load_to_lds(kp, key_at[l], kt + l * 1024);
                if (kValues) load_to_lds(vp, value_at[l], vt + l * 1024);
            }
        } else {
#pragma unroll
            for (int l = 0; l < kLoads; ++l) {
                uint32_t ka, va;
                offsets(pg, l, last - from, ka, va);
                load_to_lds(kp, ka, kt + l * 1024);
                if (kValues) load_to_lds(vp, va, vt + l * 1024);
            }
        }
    }
};

constexpr float kLn2 = 0.6931471805599453f, kLog2e = 1.4426950408889634f;

}  // namespace

}  // namespace ro
