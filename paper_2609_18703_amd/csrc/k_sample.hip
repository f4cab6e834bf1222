// The next token of every row of logits.
//
// A 16-bit logit is one of 65,536 numbers, so a row is the count of each: a
// histogram in LDS, 16 bits a counter, from which every sum that the choice
// needs follows as count * exp over the distinct values, in 64 bits and in a
// fixed order.  The filters keep a prefix of the candidates' order, and so the
// choice ends at one value and a rank among the row's tokens that have it.
// One workgroup a row, or several that count slices of a long one.
//
// What bounds a row of 128,000 f16 logits in one workgroup (57,000 cycles with
// temperature alone): its way into the registers of one CU, keys and the largest
// (13,000; 27,000 where all CUs read at once), counting, which LDS does for eight
// logits a cycle (17,000: an atomic addition takes eight cycles a wave, whatever
// the bank), the weights' sums (14,000, in bf16 5,000: half as many values lie
// apart), the look for the place by one wave, a chain of sums (8,000; 11,000 for
// the three or four of all filters), and the search for the token (6,000).  1,024
// such rows take 125 to 138 us, 2 TB/s of logits: they come from memory twice, once more for the
// search, 108 us at a copy's rate.  Loops over registers instead of unrolled code: read once,
// the code itself took a third of the time.  A thread has 128 registers at most: with 4 and
// 12 pieces 48 bytes of it are spilled, with 20 84, with 1, 8 and 16 none.
//
// Values so far below the largest that exp leaves less than e^-64 (kReach) are
// not counted: 2^20 of them are less than half a unit in the last place of a
// sum that holds a 1.  They cannot be chosen either by a u below 1, which is so
// by 2^-24 at least; for any other u, which takes the last kept one, all are
// counted.
#include <algorithm>

#include "ro_step.h"

namespace ro {

namespace {

constexpr int kThreads = 1024, kWavesOf = kThreads / 64;
constexpr int kKeys = 8;                 // neighbouring keys that a lane sums up ...
constexpr int kGroup = 64 * kKeys;       // ... and a wave
constexpr int kGroups = 65536 / kGroup, kOwn = kGroups / 64;
constexpr double kReach = 64.0;
constexpr int kTiles = (RO_MAX_VOCAB / 8 / kThreads + 1) * kWavesOf;
constexpr int kHeavy = RO_MAX_VOCAB / 32768;
// Rows of more than kSplitVocab logits are cut where CUs would be idle otherwise,
// into slices of kSliceLogits or more.  16 rows of 150,001 take 25 us so and 31
// uncut, 64 take 27 and 31, 16 of 300,000 27 and 56, 4 of 2^20 31 and 164.  128,000
// fit the registers better and are as fast uncut (25 to 27 us), 49,152 faster (18
// and 25).  Slices of 16,384 are no faster than those of 32,768.  More rows than the
// chip has room for the slices of are whole: of 262,144 logits, 51 rows take 30 us and 52
// 54 (every use reads the row again), 256 76.
constexpr int32_t kSplitVocab = 131072, kSliceLogits = 32768;
constexpr int kMaxSlices = RO_MAX_VOCAB / kSliceLogits;

using s16x2 = short __attribute__((ext_vector_type(2)));
using u32x4 = uint32_t __attribute__((ext_vector_type(4)));
using u32x32 = uint32_t __attribute__((ext_vector_type(32)));

// A key is a logit's magnitude as a whole number, with its sign: keys are
// ordered as the values are, and both zeros are 0.  NaN lie beyond the
// infinities; what is no candidate has the lowest of their keys.
template <typename T>
constexpr int32_t kInfinity = 0x7f80;
template <>
constexpr int32_t kInfinity<_Float16> = 0x7c00;
constexpr int32_t kNone = -32767;
constexpr uint32_t kNoKeys = 0x80018001u;      // two of them

// (a copy first: __builtin_bit_cast of a vector's element takes the first one)
__device__ __forceinline__ s16x2 two_of(uint32_t w) { return __builtin_bit_cast(s16x2, w); }
__device__ __forceinline__ s16x2 keys_of(uint32_t two)
{
    const s16x2 v = __builtin_bit_cast(s16x2, two), sign = v >> 15;
    return ((v & (short)0x7fff) ^ sign) - sign;
}
template <typename T>
__device__ __forceinline__ float value_of(int32_t key)
{
    const uint16_t bits = (uint16_t)(key < 0 ? 0x8000 | -key : key);
    return (float)__builtin_bit_cast(T, bits);
}
template <typename T>
__device__ __forceinline__ int32_t key_of(float f)
{
    const uint16_t bits = __builtin_bit_cast(uint16_t, (T)f);
    return bits & 0x8000 ? -(int32_t)(bits & 0x7fff) : bits;
}

// Counters: a word for keys k >= 0 in its lower half and k - 32,768 in its
// upper one, so that neighbouring keys lie in neighbouring banks.  Groups are
// numbered from the highest keys on.
__device__ __forceinline__ int group_of(int32_t key)
{
    return (key < 0 ? kGroups / 2 : 0) + (kGroups / 2 - 1) - ((key & 0x7fff) / kGroup);
}

// A row in pieces of eight logits that lie 16 bytes apart; the first and the
// last one may not be whole.
struct Row {
    const uint16_t *x;
    const uint8_t *mask;
    int32_t vocab, lead, pieces;         // lead: logits that the first piece lacks
    int32_t from, to;                    // the pieces of this workgroup

    __device__ __forceinline__ Row(const SampleArgs &a, int64_t r)
    {
        x = (const uint16_t *)a.logits + r * a.stride;
        mask = (const uint8_t *)(a.mask ? a.mask + r * a.mask_stride : nullptr);
        vocab = a.vocab;
        lead = (int32_t)((uintptr_t)x >> 1 & 7);
        pieces = (vocab + lead + 7) / 8;
        from = 0;
        to = pieces;
    }
    __device__ __forceinline__ void slice(int32_t i, int32_t each)
    {
        from = min(i * each, pieces);
        to = min(from + each, pieces);
    }
    __device__ __forceinline__ bool whole(int32_t piece) const { return piece * 8 >= lead && piece * 8 - lead + 8 <= vocab; }
    __device__ __forceinline__ bool mine(int32_t piece) const { return piece < to && whole(piece); }
    // A piece's bits, those of NaN where there is no logit.
    __device__ __forceinline__ u32x4 bits(int32_t piece) const
    {
        const int32_t from = piece * 8 - lead;
        if (whole(piece)) return *(const u32x4 *)(x + from);
        u32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int32_t c = from + 2 * i;
            const uint32_t lo = c >= 0 && c < vocab ? x[c] : 0xffffu, hi = c + 1 >= 0 && c + 1 < vocab ? x[c + 1] : 0xffffu;
            v[i] = hi << 16 | lo;
        }
        return v;
    }
    // A bit for each of a piece's tokens that the mask forbids (those of no token exclude what is no logit anyway).
    __device__ __forceinline__ uint32_t forbidden(int32_t piece) const
    {
        const int32_t bit = piece * 8 - lead, at = max(bit, 0) >> 3, from = min(at, (vocab + 31) / 32 * 4 - 2);
        uint16_t two;                    // (at any byte)
        __builtin_memcpy(&two, mask + from, 2);
        return ~((uint32_t)two << max(-bit, 0) >> ((at - from) * 8 + (max(bit, 0) & 7)));
    }
    static __device__ __forceinline__ u32x4 without(u32x4 v, uint32_t no)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            v[i] |= (no >> (2 * i) & 1 ? 0xffffu : 0u) | (no >> (2 * i + 1) & 1 ? 0xffff0000u : 0u);
        return v;
    }
    __device__ __forceinline__ u32x4 allowed(int32_t piece, u32x4 v) const { return without(v, forbidden(piece)); }
};

template <int kCtrl, int kRows>
__device__ __forceinline__ double dpp_of(double v)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, kCtrl, kRows, 0xf, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), kCtrl, kRows, 0xf, false);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// Inclusive sums over the lanes, in a fixed order.
__device__ __forceinline__ double scan_sum(double v)
{
    v += dpp_of<0x111, 0xf>(v);
    v += dpp_of<0x112, 0xf>(v);
    v += dpp_of<0x114, 0xf>(v);
    v += dpp_of<0x118, 0xf>(v);
    v += dpp_of<0x142, 0xa>(v);
    v += dpp_of<0x143, 0xc>(v);
    return v;
}
template <int kCtrl, int kRows>
__device__ __forceinline__ uint32_t dpp_add(uint32_t v)
{
    return v + (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kCtrl, kRows, 0xf, false);
}
__device__ __forceinline__ uint32_t scan_count(uint32_t v)
{
    v = dpp_add<0x111, 0xf>(v);
    v = dpp_add<0x112, 0xf>(v);
    v = dpp_add<0x114, 0xf>(v);
    v = dpp_add<0x118, 0xf>(v);
    v = dpp_add<0x142, 0xa>(v);
    v = dpp_add<0x143, 0xc>(v);
    return v;
}
// The largest of the lanes' values.
template <int kCtrl, int kRows>
__device__ __forceinline__ int32_t dpp_max(int32_t v)
{
    return max(v, __builtin_amdgcn_update_dpp(v, v, kCtrl, kRows, 0xf, false));
}
__device__ __forceinline__ int32_t lanes_max(int32_t v)
{
    v = dpp_max<0x111, 0xf>(v);
    v = dpp_max<0x112, 0xf>(v);
    v = dpp_max<0x114, 0xf>(v);
    v = dpp_max<0x118, 0xf>(v);
    v = dpp_max<0x142, 0xa>(v);
    v = dpp_max<0x143, 0xc>(v);
    return __builtin_amdgcn_readlane(v, 63);
}
// Of the lane before; 0 for the first.
__device__ __forceinline__ double lane_before(double v) { return dpp_of<0x138, 0xf>(v); }
__device__ __forceinline__ uint32_t lane_before(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x138, 0xf, 0xf, false);
}
__device__ __forceinline__ double of_lane(double v, int lane)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)b, lane);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), lane);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ uint32_t of_lane(uint32_t v, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)v, lane); }

// exp(x) for x <= 0: x = n ln 2 + r, |r| <= ln 2 / 2, and the series of exp(r),
// whose first term left out is below 4e-18.  ln 2 is a sum of 24 and of 53 bits,
// off by 2e-25: n times the first is exact, what that leaves of x too, and r is
// off by half a unit in the last place and n 2e-25.  With the series' own
// roundings the result is within 2^-52 of itself.
__device__ __forceinline__ double exp_of(double x)
{
    x = fmax(x, -800.0);                 // 0 from there on
    // (on the GPU long double is double, so that the second part is written out)
    constexpr double kInvLn2 = 1.4426950408889634074, kLn2Hi = 0.693147182464599609375, kLn2Lo = -1.90465429995776787854e-9;
    const double n = __builtin_rint(x * kInvLn2);
    const double r = __builtin_fma(-n, kLn2Lo, __builtin_fma(-n, kLn2Hi, x));
    constexpr double kTerm[] = {1.0, 1.0, 2.0, 6.0, 24.0, 120.0, 720.0, 5040.0, 40320.0, 362880.0, 3628800.0, 39916800.0,
                                479001600.0, 6227020800.0};
    double e = 1.0 / kTerm[13];
#pragma unroll
    for (int i = 12; i >= 0; --i) e = __builtin_fma(e, r, 1.0 / kTerm[i]);
    return __builtin_ldexp(e, (int)n);
}

// The same for x in [-2^-5, 0]; the first term left out is below 2^-55.
__device__ __forceinline__ double exp_near(double x)
{
    constexpr double kTerm[] = {1.0, 1.0, 2.0, 6.0, 24.0, 120.0, 720.0, 5040.0};
    double e = 1.0 / kTerm[7];
#pragma unroll
    for (int i = 6; i >= 0; --i) e = __builtin_fma(e, x, 1.0 / kTerm[i]);
    return e;
}

// A place in the candidates' order: a key, and before it so many candidates
// with such a sum of weights.
struct Place {
    int32_t key;
    uint32_t count, before;  // candidates that have the key
    double weight, sum;      // the key's weight
};

struct Heavy {
    int32_t key;
    uint32_t more;           // beside its counter
};

struct Shared {
    uint32_t hist[32768];                // (first: its offsets are addresses)
    double sum[kGroups];                 // weights of a group
    uint32_t count[kGroups];             // its candidates
    uint32_t tiles[kTiles];
    Heavy heavy[kHeavy];
    uint32_t n_heavy;
    int2 ends[kWavesOf];
    uint32_t above[kWavesOf];
    uint32_t below[64];                  // logits that are not counted, two halves a word
    int32_t key;                         // the choice
    uint32_t rank;
};
static_assert(offsetof(Shared, hist) == 0, "");

// Few long rows: each goes to several workgroups, which count their slices
// (kSlice), and to one that adds the counts up and looks for the choice in them
// (kJoin): the sums are those of kWhole, to the bit.
enum { kWhole, kSlice, kJoin };

// What the solution of a row knows of it.
template <typename T>
struct Solve {
    const Shared &s;
    int32_t most;
    double scale;            // 1 / temperature

    __device__ __forceinline__ double log_weight(int32_t key) const
    {
        return ((double)value_of<T>(key) - (double)value_of<T>(most)) * scale;
    }
    // The weights of a lane's keys, of those that can have candidates.  The values
    // of eight such keys lie evenly: each weight is the one before times the same
    // factor (within 8 half units in the last place).
    __device__ __forceinline__ int32_t first_weight(int32_t key, double &at, double &factor) const
    {
        const int32_t from = min(key, most), next = max(from - 1, -kInfinity<T> + 1);
        // (-800, a factor of 0, also beyond the last number)
        const double gap = fmax(from == kInfinity<T> ? -800.0 : ((double)value_of<T>(next) - (double)value_of<T>(from)) * scale, -800.0);
        at = from == most ? 1.0 : exp_of(log_weight(from));
        factor = __ballot(gap < -0x1p-5) ? exp_of(gap) : exp_near(gap);
        return from;
    }
    __device__ __forceinline__ void weights(int32_t key, double *w) const
    {
        double at, factor;
        const int32_t from = first_weight(key, at, factor);
        if (__ballot(from != key) == 0) {
#pragma unroll
            for (int i = 0; i < kKeys; ++i) {
                w[i] = at;
                at *= factor;
            }
        } else {
#pragma unroll
            for (int i = 0; i < kKeys; ++i) {
                w[i] = at;
                if (key - i <= from) at *= factor;
            }
        }
    }
    // The sum of the weights of a lane's candidates.
    __device__ __forceinline__ double sum_of(int32_t key, const uint32_t *c) const
    {
        double at, factor, sum = 0.0;
        const int32_t from = first_weight(key, at, factor);
        if (__ballot(from != key) == 0) {
#pragma unroll
            for (int i = kKeys - 1; i >= 0; --i) sum = __builtin_fma(sum, factor, (double)c[i]);
            return sum * at;
        }
#pragma unroll
        for (int i = 0; i < kKeys; ++i) {
            sum = __builtin_fma((double)c[i], at, sum);
            if (key - i <= from) at *= factor;
        }
        return sum;
    }
    // The counts of a lane's keys of a group, the highest first, and that one.
    __device__ __forceinline__ int32_t counts(int g, uint32_t *c, uint32_t n_heavy) const
    {
        const bool low = g >= kGroups / 2;
        const int word = (kGroups / 2 - 1 - g % (kGroups / 2)) * kGroup + (63 - lane_id()) * kKeys;
        const int32_t key = (low ? word - 32768 : word) + kKeys - 1;
#pragma unroll
        for (int v = 0; v < kKeys / 4; ++v) {
            const u32x4 w = *(const u32x4 *)&s.hist[word + kKeys - 4 - 4 * v];
#pragma unroll
            for (int i = 0; i < 4; ++i) c[4 * v + i] = low ? w[3 - i] >> 16 : w[3 - i] & 0xffff;
        }
        for (uint32_t h = 0; h < n_heavy; ++h)
#pragma unroll
            for (int i = 0; i < kKeys; ++i)
                if (s.heavy[h].key == key - i) c[i] += s.heavy[h].more;
        return key;
    }
};

}  // namespace

// kPer: pieces that a thread holds; 0: any number, read again for every use.
template <typename T, int kPer, int kMode>
__global__ void __launch_bounds__(kThreads) k_sample(SampleArgs a, SampleSplit split, Ctl *ctl)
{
    __shared__ Shared s;
    const int tid = threadIdx.x, lane = lane_id(), wave = uni32(tid >> 6);
    const int64_t r = kMode == kSlice ? blockIdx.x / split.slices : blockIdx.x;
    Row row(a, r);
    if (kMode == kSlice) row.slice(blockIdx.x % split.slices, split.pieces);
    const SampleSlice *slices = split.at + r * split.slices;
    const uint32_t *counters = split.counters + r * split.slices * 32768;
    int rounds = (row.to - row.from + kThreads - 1) / kThreads;

    // Whole pieces in registers, eight a vector, so that loops over them can be
    // loops: all unrolled, reading the code takes longer than running it.  Threads
    // without one have another whole piece again, which they do not count.  The
    // first and the last piece, if not whole, are apart, with the first two threads.
    // The registers are given up where the keys are counted, and filled again while
    // the first wave looks for the choice.
    constexpr int kVectors = (kPer + 7) / 8;
    u32x32 held[kVectors ? kVectors : 1];
    int32_t first, last;
    auto range = [&]() {
        first = max(row.from, row.lead ? 1 : 0);
        last = min(row.to, (row.vocab + row.lead) / 8) - 1;
    };
    range();
    auto whole_bits = [&](int i) -> u32x4 {
        const int32_t piece = max(first, min(row.from + i * kThreads + tid, last));
        return last >= first ? *(const u32x4 *)(row.x + (piece * 8 - row.lead)) : u32x4{~0u, ~0u, ~0u, ~0u};
    };
    auto load = [&]() {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const u32x4 v = whole_bits(i);
#pragma unroll
            for (int j = 0; j < 4; ++j) held[i / 8][i % 8 * 4 + j] = v[j];
        }
    };
    if (kMode != kJoin) load();
    auto to_keys = [&](int32_t piece, u32x4 v) -> u32x4 {
        if (row.mask) v = row.allowed(piece, v);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const s16x2 k = keys_of(v[j]);
            v[j] = __builtin_bit_cast(uint32_t, k);
        }
        return v;
    };
    int32_t edge_piece;
    bool has_edge;
    auto edges = [&]() {
        edge_piece = tid == 0 ? row.from : row.to - 1;
        has_edge = tid < 2 && row.from < row.to && !row.whole(edge_piece) && (tid == 0 || row.to - row.from > 1);
    };
    edges();
    u32x4 edge = {~0u, ~0u, ~0u, ~0u};
    if (kMode != kJoin && has_edge) edge = row.bits(edge_piece);

    const float temperature = a.temperature ? a.temperature[r] : 1.0f;
    const float top_p = a.top_p ? a.top_p[r] : 1.0f, min_p = a.min_p ? a.min_p[r] : 0.0f;
    const int32_t top_k = a.top_k ? a.top_k[r] : 0;
    const float u = a.u[r];
    auto none = [&](bool bad) {
        if (tid != 0) return;
        if (bad) raise_err(ctl, RO_EINVAL);
        a.token[r] = -1;
        if (a.logprob) a.logprob[r] = -__builtin_inff();
    };
    if (!(temperature >= 0.0f) || temperature == __builtin_inff() || top_p != top_p || min_p != min_p) {
        if (kMode != kSlice) none(true);
        return;
    }
    // (while the logits are on their way)
    for (int i = tid; i < 32768 / 4; i += kThreads) ((u32x4 *)s.hist)[i] = u32x4{0, 0, 0, 0};
    if (tid < kGroups) {
        s.sum[tid] = 0.0;
        s.count[tid] = 0;
    }
    for (int i = tid; i < (kMode == kJoin ? kPer : rounds) * kWavesOf; i += kThreads) s.tiles[i] = 0;
    if (tid < 64) s.below[tid] = 0;
    if (tid < kHeavy) s.heavy[tid].key = kNone;
    if (tid == 0) s.n_heavy = 0;

    bool clean = false;                  // are NaN no candidates yet?
    auto without_nan = [&](uint32_t w) -> uint32_t {
        const s16x2 k = two_of(w);
        const short lo = k[0] > (short)kInfinity<T> ? (short)kNone : k[0], hi = k[1] > (short)kInfinity<T> ? (short)kNone : k[1];
        return (uint32_t)(uint16_t)lo | (uint32_t)(uint16_t)hi << 16;
    };
    // f(v) for every piece of the thread, as keys, read again.
    auto each_read = [&](auto f) {
        for (int i = 0; i < rounds; ++i) {
            const int32_t piece = row.from + i * kThreads + tid;
            u32x4 v = {kNoKeys, kNoKeys, kNoKeys, kNoKeys};
            if (piece < row.to) v = to_keys(piece, row.bits(piece));
            if (clean)
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = without_nan(v[j]);
            f(i, v);
        }
    };
    // the largest key, and the least of the whole pieces
    int32_t fewest = 0;
    s16x2 m, l;
    auto look_at = [&](const u32x4 &v, bool whole) {
        s16x2 p = two_of(v[0]), q = p;
#pragma unroll
        for (int j = 1; j < 4; ++j) {
            p = __builtin_elementwise_min(p, two_of(v[j]));
            q = __builtin_elementwise_max(q, two_of(v[j]));
        }
        if (whole) l = __builtin_elementwise_min(l, p);
        m = __builtin_elementwise_max(m, q);
    };
    auto largest = [&]() -> int32_t {
        int32_t most = lanes_max(max((int32_t)m[0], (int32_t)m[1])), least = -lanes_max(-min((int32_t)l[0], (int32_t)l[1]));
        __syncthreads();
        if (lane == 0) s.ends[wave] = make_int2(most, least);
        __syncthreads();
        const int2 e = s.ends[lane & (kWavesOf - 1)];
        most = lanes_max(e.x);
        least = -lanes_max(-e.y);
        fewest = least;
        return most;
    };
    m = s16x2{(short)kNone, (short)kNone};
    l = s16x2{0x7fff, 0x7fff};
    if (kMode != kJoin) {
        if (has_edge) edge = to_keys(edge_piece, edge);
        else edge = u32x4{kNoKeys, kNoKeys, kNoKeys, kNoKeys};
        look_at(edge, false);
    }
    if (kMode == kJoin) {
    } else if (kPer) {
        if (row.mask) {
            uint32_t no[kPer ? kPer : 1];
#pragma unroll
            for (int i = 0; i < kPer; ++i) no[i] = row.forbidden(max(first, min(row.from + i * kThreads + tid, last)));
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const u32x4 v = Row::without(u32x4{held[i / 8][i % 8 * 4], held[i / 8][i % 8 * 4 + 1], held[i / 8][i % 8 * 4 + 2],
                                                   held[i / 8][i % 8 * 4 + 3]}, no[i]);
#pragma unroll
                for (int j = 0; j < 4; ++j) held[i / 8][i % 8 * 4 + j] = v[j];
            }
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            u32x4 v;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t w = held[i / 8][i % 8 * 4 + j];
                const s16x2 k = keys_of(w);
                held[i / 8][i % 8 * 4 + j] = v[j] = __builtin_bit_cast(uint32_t, k);
            }
            look_at(v, true);
        }
    } else {
        for (int i = 0; i < rounds; ++i) {
            const int32_t piece = max(first, min(row.from + i * kThreads + tid, last));
            look_at(to_keys(piece, whole_bits(i)), true);
        }
    }
    int32_t most;
    if (kMode == kJoin) {
        most = lanes_max(lane < split.slices ? slices[lane].most : kNone);
        __syncthreads();
    } else {
        most = largest();
    }
    if (kMode != kJoin && most > kInfinity<T>) {
        clean = true;
        m = s16x2{(short)kNone, (short)kNone};
        l = s16x2{(short)kNone, (short)kNone};
#pragma unroll
        for (int j = 0; j < 4; ++j) edge[j] = without_nan(edge[j]);
#pragma unroll
        for (int c = 0; c < kVectors; ++c)
#pragma unroll 1
            for (int q = 0; q < (kPer - c * 8 < 8 ? kPer - c * 8 : 8) * 4; ++q) held[c][q] = without_nan(held[c][q]);
        each_read([&](int, const u32x4 &v) { look_at(v, false); });
        most = largest();
    }
    if (kMode != kSlice && most <= -kInfinity<T>) return none(false);

    const double scale = 1.0 / (temperature > 0.0f ? (double)temperature : 1.0);
    // the lowest key that is counted: one too low rather than too high
    int32_t least = most;
    if (!(u < 1.0f)) {
        least = -kInfinity<T> + 1;
    } else if (most != kInfinity<T>) {
        const double low = (double)value_of<T>(most) - kReach * (temperature > 0.0f ? (double)temperature : 1.0);
        least = max(-kInfinity<T> + 1, key_of<T>((float)low) - 1);
    }
    const Solve<T> solve{s, most, scale};
    const bool first_only = temperature == 0.0f || top_k == 1;
    double total = 0.0;                  // (of the first wave)
    Place at{};
    uint32_t rank = 0;
    at.key = most;
    const bool sums = !first_only || a.logprob;
    if (kMode == kSlice && (!sums || most <= -kInfinity<T>)) {
        if (tid == 0) split.at[blockIdx.x] = SampleSlice{0, most, 0};
        return;
    }
    if (sums) {
        auto add = [&](int32_t key) { atomicAdd(&s.hist[key & 0x7fff], key < 0 ? 0x10000u : 1u); };
        // what a key adds: 1 to the lower half of its word, or to the upper one below zero (one
        // instruction after the sign's, where a selection would take a comparison and a wait)
        auto one_of = [](uint32_t negative) -> uint32_t {
            uint32_t v;
            asm("v_mad_u32_u24 %0, %1, %2, 1" : "=v"(v) : "v"(negative), "s"(0xffffu));
            return v;
        };
        auto add_at = [&](uint32_t at, uint32_t negative) { atomicAdd((uint32_t *)((char *)&s + at), one_of(negative)); };
        // (without a branch: what lies below counts in a word of the lane)
        const uint32_t below = (uint32_t)offsetof(Shared, below) + lane * 4;
        auto add_some = [&](const u32x4 &v) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t w = v[j];
                add_at((int16_t)w >= (int16_t)least ? w << 2 & 0x1fffc : below, w >> 15 & 1);
                add_at((int32_t)w >= least * 65536 ? w >> 14 & 0x1fffc : below, w >> 31);
            }
        };
        if (kMode != kJoin && has_edge) add_some(edge);
        auto count_whole = [&](auto add_piece) {
            if (kPer) {
#pragma unroll
                for (int c = 0; c < kVectors; ++c)
#pragma unroll 1
                    for (int q = 0; q < min(kPer - c * 8 < 8 ? kPer - c * 8 : 8, rounds - c * 8); ++q)
                        if (row.mine(row.from + (c * 8 + q) * kThreads + tid))
                            add_piece(u32x4{held[c][q * 4], held[c][q * 4 + 1], held[c][q * 4 + 2], held[c][q * 4 + 3]});
            } else {
                each_read([&](int i, const u32x4 &v) {
                    if (row.mine(row.from + i * kThreads + tid)) add_piece(v);
                });
            }
        };
        if constexpr (kMode == kJoin) {
            // 256 counters of all slices at a time; what a sum has beyond 16 bits is apart
            constexpr int kAtOnce = 8;
            const uint64_t of_slice = lane < split.slices ? slices[lane].groups : 0;
            for (int unit = wave; unit < 32768 / 256; unit += kWavesOf) {
                uint64_t have = __ballot(of_slice >> (unit / 2) & 1);
                if (have == 0) continue;
                const int word = unit * 256 + lane * 4;
                u32x4 lo = {0, 0, 0, 0}, hi = {0, 0, 0, 0};
                while (have) {
                    u32x4 v[kAtOnce];
                    int n = 0, i = 0;
#pragma unroll
                    for (int j = 0; j < kAtOnce; ++j) {
                        if (have) {
                            i = __ffsll((unsigned long long)have) - 1;
                            have &= have - 1;
                            ++n;
                        }
                        v[j] = *(const u32x4 *)(counters + (int64_t)i * 32768 + word);
                    }
#pragma unroll
                    for (int j = 0; j < kAtOnce; ++j) {
                        lo += j < n ? v[j] & 0xffffu : u32x4{0, 0, 0, 0};
                        hi += j < n ? v[j] >> 16 : u32x4{0, 0, 0, 0};
                    }
                }
                u32x4 w;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    // (a slice counts what is in reach of its own largest key)
                    const uint32_t n[2] = {word + j >= least ? lo[j] : 0, word + j - 32768 >= least ? hi[j] : 0};
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        if (n[h] >> 16) s.heavy[atomicAdd(&s.n_heavy, 1u)] = Heavy{word + j - h * 32768, n[h] & ~0xffffu};
                    w[j] = n[1] << 16 | (n[0] & 0xffff);
                }
                *(u32x4 *)&s.hist[word] = w;
            }
        } else if (fewest >= least)              // whole pieces have nothing below
            count_whole([&](const u32x4 &v) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t w = v[j];
                    add_at(w << 2 & 0x1fffc, w >> 15 & 1);
                    add_at(w >> 14 & 0x1fffc, w >> 31);
                }
            });
        else
            count_whole(add_some);
        __syncthreads();
        const uint32_t left_out = s.below[lane];
        uint32_t candidates = (uint32_t)(row.to - row.from) * 8 - of_lane(scan_count((left_out & 0xffff) + (left_out >> 16)), 63);
        if constexpr (kMode == kSlice) {
            // the counters that are not 0, for the workgroup that joins the slices
            uint32_t *out = split.counters + (int64_t)blockIdx.x * 32768;
            uint64_t mine = 0;
#pragma unroll
            for (int i = 0; i < kGroups / 2 / kWavesOf; ++i) {
                const int words = i * kWavesOf + wave, at = words * kGroup + lane * kKeys;
                const u32x4 x = *(const u32x4 *)&s.hist[at], y = *(const u32x4 *)&s.hist[at + 4];
                if (__ballot((x[0] | x[1] | x[2] | x[3] | y[0] | y[1] | y[2] | y[3]) != 0) == 0) continue;
                *(u32x4 *)(out + at) = x;
                *(u32x4 *)(out + at + 4) = y;
                mine |= 1ull << words;
            }
            if (lane == 0) s.sum[wave] = __builtin_bit_cast(double, mine);
            __syncthreads();
            if (tid == 0) {
                for (int w = 1; w < kWavesOf; ++w) mine |= __builtin_bit_cast(uint64_t, s.sum[w]);
                split.at[blockIdx.x] = SampleSlice{mine, most, 0};
            }
            return;
        }
        const int g0 = group_of(most), g1 = group_of(least);
        auto sum_groups = [&](uint32_t n_heavy) {
            uint32_t above = 0;          // candidates that min_p keeps
            // which of the wave's groups have candidates: all read at once
            uint32_t some = 0;
#pragma unroll
            for (int i = 0; i < kGroups / kWavesOf; ++i) {
                const int g = g0 + wave + i * kWavesOf;
                if (g > g1) break;
                const bool low = g >= kGroups / 2;
                const uint32_t *at = &s.hist[(kGroups / 2 - 1 - g % (kGroups / 2)) * kGroup + lane * kKeys];
                const u32x4 x = *(const u32x4 *)at, y = *(const u32x4 *)(at + 4);
                const uint32_t any = x[0] | x[1] | x[2] | x[3] | y[0] | y[1] | y[2] | y[3];
                if (__ballot(any & (low ? 0xffff0000u : 0xffffu))) some |= 1u << i;
            }
            if (n_heavy) some = ~0u;             // (a counter of theirs may be 0)
            while (some) {
                const int g = g0 + wave + (__ffs((int)some) - 1) * kWavesOf;
                some &= some - 1;
                if (g > g1) break;
                uint32_t c[kKeys], n = 0;
                const int32_t key = solve.counts(g, c, n_heavy);
#pragma unroll
                for (int i = 0; i < kKeys; ++i) n += c[i];
                if (__ballot(n != 0) == 0) continue;
                double sum;
                if (min_p > 0.0f) {
                    double w[kKeys];
                    solve.weights(key, w);
                    sum = 0.0;
#pragma unroll
                    for (int i = 0; i < kKeys; ++i) {
                        sum = __builtin_fma((double)c[i], w[i], sum);
                        above += w[i] >= (double)min_p ? c[i] : 0;
                    }
                } else {
                    sum = solve.sum_of(key, c);
                }
                sum = scan_sum(sum);
                n = scan_count(n);
                if (lane == 63) {
                    s.sum[g] = sum;
                    s.count[g] = n;
                }
            }
            above = scan_count(above);
            if (lane == 63) s.above[wave] = above;
            __syncthreads();
        };
        sum_groups(kMode == kJoin ? s.n_heavy : 0);
        // are all there?  (A counter of 16 bits that runs over takes 65,535 or 65,536 from the sum of all.)
        auto counted = [&]() -> uint32_t {
            const uint32_t n = s.count[lane * 2] + s.count[lane * 2 + 1];
            return of_lane(scan_count(n), 63);
        };
        if (kMode == kJoin) {
            candidates = counted();
        } else if (counted() != candidates) {
            // again, at most 2^15 at a time, after which counters that have 2^15 give them up
            __syncthreads();
            for (int i = tid; i < 32768; i += kThreads) s.hist[i] = 0;
            if (tid < kGroups) {
                s.sum[tid] = 0.0;
                s.count[tid] = 0;
            }
            __syncthreads();
            auto spill = [&]() {
                __syncthreads();
                for (int i = tid; i < 32768; i += kThreads) {
                    uint32_t w = s.hist[i];
                    if ((w & 0x80008000u) == 0) continue;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if ((w >> (16 * h + 15) & 1) == 0) continue;
                        const int32_t key = h ? i - 32768 : i;
                        uint32_t e = 0;
                        const uint32_t n = s.n_heavy;
                        while (e < n && s.heavy[e].key != key) ++e;
                        // (a word is one thread's; an entry that another one is writing has its key, or none yet)
                        if (e == n) {
                            e = atomicAdd(&s.n_heavy, 1u);
                            s.heavy[e].key = key;
                            s.heavy[e].more = 0;
                        }
                        s.heavy[e].more += 0x8000;
                        w &= ~(0x8000u << (16 * h));
                    }
                    s.hist[i] = w;
                }
                __syncthreads();
            };
            each_read([&](int i, const u32x4 &v) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const s16x2 k = two_of(v[j]);
                    if (k[0] >= least) add(k[0]);
                    if (k[1] >= least) add(k[1]);
                }
                if (i % 4 == 3 || i == rounds - 1) spill();
            });
            sum_groups(s.n_heavy);
        }
        // The rest is one wave's: places in the order of the candidates.
        if (wave == 0) {
            double in[kOwn];
            uint32_t n_in[kOwn];
            const uint32_t heavy = uni32((int32_t)s.n_heavy);
            uint32_t n_above = 0;
            for (int w = 0; w < kWavesOf; ++w) n_above += s.above[w];
            if (!(min_p > 0.0f)) n_above = candidates;
            // a lane has kOwn groups; sums up to and with each
            double sum = 0.0;
            uint32_t n = 0;
#pragma unroll
            for (int i = 0; i < kOwn; ++i) {
                in[i] = sum += s.sum[lane * kOwn + i];
                n_in[i] = n += s.count[lane * kOwn + i];
            }
            const double up = scan_sum(sum), ex = lane_before(up);
            const uint32_t n_up = scan_count(n), n_ex = lane_before(n_up);
            total = of_lane(up, 63);
#pragma unroll
            for (int i = 0; i < kOwn; ++i) {
                in[i] += ex;
                n_in[i] += n_ex;
            }
            // The first key of the order with which the count exceeds i (kCount), or the sum reaches
            // `want` (kReaches) or exceeds it (kExceeds); or else the last one.
            enum { kCount, kReaches, kExceeds };
            // (The keys of the group it was in last are kept: the next one is often there too.)
            int g_last = -1;
            uint32_t c[kKeys];
            double w[kKeys], lane_sum = 0.0;             // before the lane's keys
            uint32_t lane_n = 0;
            int32_t key = 0;
            auto find = [&](int what, uint32_t i, double want) -> Place {
                // (a sum reaches a number if it exceeds the one before that)
                if (what == kReaches) want = want > 0.0 ? __builtin_bit_cast(double, __builtin_bit_cast(uint64_t, want) - 1) : -1.0;
                auto hit = [&](double upto, uint32_t n) { return what == kCount ? i < n : upto > want; };
                int mine = kOwn, some = -1;
                double b_sum = 0.0, x_sum = 0.0;         // before the group
                uint32_t b_n = 0, x_n = 0;
#pragma unroll
                for (int e = kOwn - 1; e >= 0; --e) {
                    const double g_sum = e ? in[e - 1] : ex;
                    const uint32_t g_n = e ? n_in[e - 1] : n_ex;
                    if (n_in[e] == g_n) continue;
                    if (some < 0) {
                        some = e;
                        x_sum = g_sum;
                        x_n = g_n;
                    }
                    if (hit(in[e], n_in[e])) {
                        mine = e;
                        b_sum = g_sum;
                        b_n = g_n;
                    }
                }
                const uint64_t yes = __ballot(mine < kOwn), have = __ballot(some >= 0);
                const int l = yes ? __ffsll((unsigned long long)yes) - 1 : 63 - __clzll((long long)have);
                const int g = l * kOwn + (int)of_lane((uint32_t)(yes ? mine : some), l);
                b_sum = of_lane(yes ? b_sum : x_sum, l);
                b_n = of_lane(yes ? b_n : x_n, l);
                if (g != g_last) {                       // its keys
                    g_last = g;
                    key = solve.counts(g, c, heavy);
                    solve.weights(key, w);
                    double k_sum = 0.0;
                    uint32_t k_n = 0;
#pragma unroll
                    for (int e = 0; e < kKeys; ++e) {
                        k_sum = __builtin_fma((double)c[e], w[e], k_sum);
                        k_n += c[e];
                    }
                    lane_sum = b_sum + lane_before(scan_sum(k_sum));
                    lane_n = b_n + lane_before(scan_count(k_n));
                }
                double at_sum = lane_sum;
                uint32_t at_n = lane_n;
                // the lane's first key at which it does, or its last one, as a bit
                uint32_t does = 0, has = 0;
                double k_at[kKeys];
#pragma unroll
                for (int e = 0; e < kKeys; ++e) {
                    k_at[e] = at_sum;
                    at_sum = __builtin_fma((double)c[e], w[e], at_sum);
                    at_n += c[e];
                    has |= (c[e] != 0) << e;
                    does |= (c[e] != 0 && hit(at_sum, at_n)) << e;
                }
                const uint64_t hits = __ballot(does != 0), full = __ballot(has != 0);
                const int kl = hits ? __ffsll((unsigned long long)hits) - 1 : 63 - __clzll((long long)full);
                const int ke = (int)of_lane(hits ? (uint32_t)(__ffs((int)does) - 1) : 31u - (uint32_t)__clz((int)has), kl);
                Place p{};
                uint32_t after = 0;                      // the lane's candidates from that key on
#pragma unroll
                for (int e = kKeys - 1; e >= 0; --e) {
                    if (e >= ke) after += c[e];
                    if (e != ke) continue;               // (the same for all lanes)
                    p.count = of_lane(c[e], kl);
                    p.weight = of_lane(w[e], kl);
                    p.sum = of_lane(k_at[e], kl);
                }
                p.key = (int32_t)of_lane((uint32_t)key, kl) - ke;
                p.before = of_lane(at_n - after, kl);
                return p;
            };
            auto sum_with = [](const Place &p, uint32_t i) { return p.sum + (i - p.before + 1.0) * p.weight; };
            // The filters, one after the other, and the choice: each asks for a place or not.
            uint32_t keep = first_only ? 1 : candidates;
            double kept = total;
            Place last{};
            bool have_last = false;
            enum { kTopK, kTopP, kLast, kChoice, kSteps };
#pragma unroll 1
            for (int step = first_only ? (int)kSteps : (int)kTopK; step < kSteps; ++step) {
                int what = kCount;
                uint32_t i = 0;
                double want = 0.0;
                if (step == kTopK) {
                    if (top_k <= 0 || (uint32_t)top_k >= keep) continue;
                    keep = (uint32_t)top_k;
                    i = keep - 1;
                } else if (step == kTopP) {
                    if (!(top_p < 1.0f)) continue;
                    what = kReaches;
                    want = (double)top_p * kept;
                } else if (step == kLast) {
                    if (n_above < keep) {
                        keep = max(1u, n_above);
                        have_last = false;
                    }
                    if (keep == 1) break;
                    if (have_last || (keep == candidates && u < 1.0f)) continue;
                    i = keep - 1;
                } else {
                    if (!(u < 1.0f)) {
                        at = last;
                        rank = keep - 1 - at.before;
                        break;
                    }
                    what = kExceeds;
                    if (keep < candidates) kept = sum_with(last, keep - 1);
                    want = (double)u * kept;
                }
                const Place p = find(what, i, want);
                if (what == kCount) {
                    last = p;
                    have_last = true;
                    kept = sum_with(p, i);
                    continue;
                }
                // the first of the key's candidates with which the sum does (the quotient is rounded)
                const double many = (double)p.count, q = (want - p.sum) / p.weight;
                double j = fmin(fmax(what == kReaches ? ceil(q) - 1.0 : floor(q), 0.0), many - 1.0);
                auto does = [&](double upto) { return what == kReaches ? upto >= want : upto > want; };
                if (j > 0.0 && does(p.sum + j * p.weight)) j -= 1.0;
                else if (j < many - 1.0 && !does(p.sum + (j + 1.0) * p.weight)) j += 1.0;
                i = p.before + (uint32_t)j;
                if (what == kReaches) {
                    if (i + 1 < keep) {
                        keep = i + 1;
                        last = p;
                        have_last = true;
                    }
                } else {
                    at = p;
                    if (i >= keep) {             // (by a rounding; then there are more candidates, and the last kept one is known)
                        i = keep - 1;
                        at = last;
                    }
                    rank = i - at.before;
                }
            }
            if (lane == 0 && a.logprob) a.logprob[r] = (float)((at.key == most ? 0.0 : solve.log_weight(at.key)) - log(total));
        }
    }
    if (kMode != kJoin) load();
    if (tid == 0) {
        s.key = at.key;
        s.rank = rank;
    }
    __syncthreads();

    // the token: of those that have the key, in order, number `rank`
    const int32_t key = uni32(s.key);
    uint32_t left = s.rank;
    if (kMode == kJoin) {                // the slice that has it
        uint32_t n = 0;
        if (lane < split.slices) {
            if (!sums) n = slices[lane].most == key;
            else if (slices[lane].groups >> ((key & 0x7fff) / kGroup) & 1)
                n = counters[(int64_t)lane * 32768 + (key & 0x7fff)] >> (key < 0 ? 16 : 0) & 0xffff;
        }
        const uint32_t upto = scan_count(n);
        const uint64_t yes = __ballot(upto > left);
        const int l = yes ? __ffsll((unsigned long long)yes) - 1 : 0;
        left -= of_lane(upto - n, l);
        row.slice(l, split.pieces);
        range();
        edges();
        rounds = (row.to - row.from + kThreads - 1) / kThreads;
        load();
    }
    // (by its bits, those of both zeros without the sign: other numbers cannot be taken for it)
    const uint32_t sign = key == 0 ? 0x7fff7fffu : ~0u, both = (uint32_t)(key < 0 ? 0x8000 | -key : key) * 0x10001u;
    using u16x2 = uint16_t __attribute__((ext_vector_type(2)));
    // a bit for each of the piece's tokens that have it
    auto same = [&](int32_t piece, u32x4 v) -> uint32_t {
        if (row.mask) v = row.allowed(piece, v);
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t x = (v[j] & sign) ^ both;
            m |= (uint32_t)((x & 0xffff) == 0) << (2 * j) | (uint32_t)(x < 0x10000) << (2 * j + 1);
        }
        return m;
    };
    if (has_edge) {
        const uint32_t n = (uint32_t)__popc(same(edge_piece, row.bits(edge_piece)));
        if (n) atomicAdd(&s.tiles[(edge_piece - row.from) / kThreads * kWavesOf + (edge_piece - row.from) % kThreads / 64], n);
    }
    auto look_for = [&](int i, u32x4 v) {
        const int32_t piece = row.from + i * kThreads + tid;
        if (!row.mine(piece)) return;
        const uint32_t n = (uint32_t)__popc(same(piece, v));
        if (n) atomicAdd(&s.tiles[i * kWavesOf + wave], n);
    };
    if (kPer) {
        // (eight pieces are looked over together: few have it)
#pragma unroll
        for (int c = 0; c < kVectors; ++c) {
            u16x2 least_of = {1, 1};
#pragma unroll
            for (int q = 0; q < (kPer - c * 8 < 8 ? kPer - c * 8 : 8) * 4; ++q) {
                const uint32_t x = (held[c][q] & sign) ^ both;
                least_of = __builtin_elementwise_min(least_of, __builtin_bit_cast(u16x2, x));
            }
            if (__ballot(!(least_of[0] && least_of[1])) == 0) continue;
#pragma unroll 1
            for (int q = 0; q < (kPer - c * 8 < 8 ? kPer - c * 8 : 8); ++q)
                look_for(c * 8 + q, u32x4{held[c][q * 4], held[c][q * 4 + 1], held[c][q * 4 + 2], held[c][q * 4 + 3]});
        }
    } else {
        for (int i = 0; i < rounds; ++i) look_for(i, whole_bits(i));
    }
    __syncthreads();
    const int tiles = rounds * kWavesOf;
    int tile = -1;
    for (int i0 = 0; i0 < tiles; i0 += 64) {
        const uint32_t n = i0 + lane < tiles ? s.tiles[i0 + lane] : 0;
        const uint32_t upto = scan_count(n);
        const uint64_t yes = __ballot(upto > left);
        if (yes) {
            const int l = __ffsll((unsigned long long)yes) - 1;
            left -= of_lane(upto - n, l);
            tile = i0 + l;
            break;
        }
        left -= of_lane(upto, 63);
    }
    if (tile < 0 || tile % kWavesOf != wave) return; // (some tile has it)
    const int32_t piece = row.from + tile / kWavesOf * kThreads + tid;
    uint32_t have = piece < row.to ? same(piece, row.bits(piece)) : 0;
    const uint32_t n = (uint32_t)__popc(have), before = scan_count(n) - n;
    if (before > left || before + n <= left) return;
    for (uint32_t k = before; k < left; ++k) have &= have - 1;
    a.token[r] = piece * 8 - row.lead + (__ffs((int)have) - 1);
}

template <typename T>
hipError_t launch_typed(const Launch &L, const SampleArgs &a, int64_t n, const SampleSplit &split)
{
    const int32_t pieces = (a.vocab + 14) / 8, per = (pieces + kThreads - 1) / kThreads;
#define RO_SAMPLE(kPer, kMode, n)                                                                                          \
    RO_LAUNCH(L, RO_K_SAMPLE, (k_sample<T, kPer, kMode>), dim3((unsigned)(n)), dim3(kThreads), 0, L.stream, a, split, L.ctl)
    if (split.slices > 1) {
        RO_SAMPLE(8, kSlice, n * split.slices);
        RO_SAMPLE(8, kJoin, n);
    } else if (per <= 1) RO_SAMPLE(1, kWhole, n);
    else if (per <= 4) RO_SAMPLE(4, kWhole, n);
    else if (per <= 8) RO_SAMPLE(8, kWhole, n);
    else if (per <= 12) RO_SAMPLE(12, kWhole, n);
    else if (per <= 16) RO_SAMPLE(16, kWhole, n);
    else if (per <= 20) RO_SAMPLE(20, kWhole, n);
    else RO_SAMPLE(0, kWhole, n);
#undef RO_SAMPLE
    return hipGetLastError();
}

int32_t sample_slices(int32_t num_cus, int64_t n, int32_t vocab)
{
    if (vocab <= kSplitVocab) return 1;
    // no counter of 16 bits runs over in a slice
    const int64_t least = (vocab + 65471) / 65472, most = std::min<int64_t>(kMaxSlices, num_cus / n);
    const int64_t s = std::min<int64_t>(most, (vocab + kSliceLogits - 1) / kSliceLogits);
    return s < least || s < 2 ? 1 : (int32_t)s;
}

hipError_t launch_sample(const Launch &L, const SampleArgs &a, int64_t n, int32_t dtype, SampleSplit split)
{
    if (split.slices > 1) split.pieces = ((a.vocab + 14) / 8 + split.slices - 1) / split.slices;
    return dtype == RO_BF16 ? launch_typed<__bf16>(L, a, n, split) : launch_typed<_Float16>(L, a, n, split);
}

}  // namespace ro
