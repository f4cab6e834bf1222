// The next token of every row of logits.
//
// A 16-bit logit is one of 65,536 numbers, so a row is the count of each: a
// histogram in LDS, 16 bits a counter, from which every sum that the choice
// needs follows as count * exp over the distinct values, in 64 bits and in a
// fixed order.  The filters keep a prefix of the candidates' order, and so the
// choice ends at one value and a rank among the row's tokens that have it.
//
// Values so far below the largest that exp leaves less than 2^-92 (kReach) are
// not counted: 2^20 of them are less than half a unit in the last place of a
// sum that holds a 1.  They cannot be chosen either, u being below 1 by
// 2^-24 at least where it is not 0.
#include "ro_step.h"

namespace ro {

namespace {

constexpr int kThreads = 1024, kWavesOf = kThreads / 64;
constexpr int kSegments = 1024;          // runs of 64 neighbouring keys
constexpr double kReach = 64.0;
constexpr int kCountTiles = RO_MAX_VOCAB / 512 + 16;

// Keys are ordered as the values are; -0 has the key of 0.
__device__ __forceinline__ uint32_t key_of(uint32_t bits)
{
    const uint32_t k = bits ^ (bits & 0x8000 ? 0xffffu : 0x8000u);
    return k == 0x7fff ? 0x8000 : k;
}
template <typename T>
__device__ __forceinline__ float value_of(uint32_t key)
{
    const uint16_t bits = (uint16_t)(key ^ (key & 0x8000 ? 0x8000u : 0xffffu));
    return (float)__builtin_bit_cast(T, bits);
}
template <typename T>
constexpr uint32_t kInfinity = 0x7f80;
template <>
constexpr uint32_t kInfinity<_Float16> = 0x7c00;
template <typename T>
constexpr uint32_t kTop = 0x8000 | kInfinity<T>;         // +inf's key; NaN lies above, or below that of -inf
template <typename T>
constexpr uint32_t kBottom = 0x7fff & ~kInfinity<T>;     // -inf's

using u16x8 = uint16_t __attribute__((ext_vector_type(8)));

// A row in pieces of eight logits that lie 16 bytes apart; the first and the
// last one may not be whole.
template <typename T>
struct Row {
    const uint16_t *x;
    const uint32_t *mask;
    int32_t vocab, lead, pieces;         // logits that the first piece lacks

    __device__ __forceinline__ Row(const SampleArgs &a, int64_t r)
    {
        x = (const uint16_t *)a.logits + r * a.stride;
        mask = a.mask ? a.mask + r * a.mask_stride : nullptr;
        vocab = a.vocab;
        lead = (int32_t)((uintptr_t)x >> 1 & 7);
        pieces = (vocab + lead + 7) / 8;
    }
    // The keys of a piece's candidates, 0 for the others.
    __device__ __forceinline__ void keys(int32_t piece, uint32_t *k) const
    {
        const int32_t from = piece * 8 - lead;
        u16x8 v;
        if (from >= 0 && from + 8 <= vocab) {
            v = *(const u16x8 *)(x + from);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = from + i >= 0 && from + i < vocab ? x[from + i] : 0xffff;   // a NaN
        }
        uint32_t allowed = 0xff;
        if (mask) {
            const int32_t lo = max(from, 0) >> 5, hi = min(from + 7, vocab - 1) >> 5;
            const uint64_t w = (uint64_t)mask[hi] << 32 | mask[lo];
            // the piece's bits, the first one lowest
            allowed = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int32_t c = max(0, from + i);
                allowed |= (uint32_t)(w >> ((c & 31) + (c >> 5 > lo ? 32 : 0)) & 1) << i;
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t key = key_of(v[i]);
            k[i] = key > kBottom<T> && key <= kTop<T> && (allowed >> i & 1) ? key : 0;
        }
    }
};

struct Found {
    int32_t key;
    uint32_t rank;           // among the row's tokens of this key
    uint32_t before;         // candidates before them
    double sum, weight;      // their weights' sum; the key's weight
};

struct Shared {
    uint32_t hist[32768];
    double sum[kSegments];               // weights of the segments from the highest on, this one's included
    uint32_t count[kSegments];           // candidates, likewise
    uint32_t bins[64];
    uint16_t tiles[kCountTiles];
    double w_sum[kWavesOf];
    uint32_t w_count[kWavesOf], w_other[kWavesOf];
    uint32_t most;
    int32_t segment;
    Found found;
};

__device__ __forceinline__ double shfl_up_d(double v, int d) { return __shfl_up(v, d, 64); }

}  // namespace

template <typename T>
__global__ void __launch_bounds__(kThreads) k_sample(SampleArgs a, Ctl *ctl)
{
    __shared__ Shared s;
    const int tid = threadIdx.x, lane = lane_id(), wave = uni32(tid >> 6);
    const int64_t r = blockIdx.x;
    const Row<T> row(a, r);
    const float T_r = a.temperature ? a.temperature[r] : 1.0f;
    const float p_r = a.top_p ? a.top_p[r] : 1.0f, m_r = a.min_p ? a.min_p[r] : 0.0f;
    const int32_t k_r = a.top_k ? a.top_k[r] : 0;
    auto none = [&](bool bad) {
        if (tid != 0) return;
        if (bad) raise_err(ctl, RO_EINVAL);
        a.token[r] = -1;
        if (a.logprob) a.logprob[r] = -__builtin_inff();
    };
    if (!(T_r >= 0.0f) || T_r == __builtin_inff() || p_r != p_r || m_r != m_r) return none(true);

    // the largest
    uint32_t most = 0;
    for (int32_t i = tid; i < row.pieces; i += kThreads) {
        uint32_t k[8];
        row.keys(i, k);
#pragma unroll
        for (int j = 0; j < 8; ++j) most = max(most, k[j]);
    }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, d, 64));
    if (lane == 0) s.w_count[wave] = most;
    for (int i = tid; i < 32768; i += kThreads) s.hist[i] = 0;
    s.sum[tid] = 0.0;
    s.count[tid] = 0;
    __syncthreads();
    for (int w = 0; w < kWavesOf; ++w) most = max(most, s.w_count[w]);
    if (most == 0) return none(false);

    const double temp = T_r > 0.0f ? (double)T_r : 1.0;
    const double top = (double)value_of<T>(most) / temp;
    const bool infinite = most == kTop<T>;
    auto weight_log = [&](uint32_t key) -> double { return key == most ? 0.0 : (double)value_of<T>(key) / temp - top; };
    // the lowest key that is counted: found from above, one key too low rather than too high
    uint32_t least = most;
    if (!infinite) {
        const float low = (float)((double)value_of<T>(most) - kReach * temp);
        const T bits = (T)low;
        least = key_of(__builtin_bit_cast(uint16_t, bits));
        least = max(kBottom<T> + 1, least - 1);
    }
    // how many times each occurs
    uint32_t mine = 0;
    for (int32_t i = tid; i < row.pieces; i += kThreads) {
        uint32_t k[8];
        row.keys(i, k);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (k[j] >= least) {
                atomicAdd(&s.hist[k[j] >> 1], k[j] & 1 ? 0x10000u : 1u);
                ++mine;
            }
    }
    __syncthreads();
    // `half` < 0: the counters; else 32 bits each for the upper (1) or lower half of the keys
    auto count_half = [&](int half) {
        __syncthreads();
        for (int i = tid; i < 32768; i += kThreads) s.hist[i] = 0;
        __syncthreads();
        for (int32_t i = tid; i < row.pieces; i += kThreads) {
            uint32_t k[8];
            row.keys(i, k);
            for (int j = 0; j < 8; ++j)
                if (k[j] >= least && (int)(k[j] >> 15) == half) atomicAdd(&s.hist[k[j] & 0x7fff], 1u);
        }
        __syncthreads();
    };
    uint32_t above = 0;                              // candidates whose weight min_p keeps
    auto sum_segments = [&](int lo, int hi, bool wide) {
        for (int g = hi - wave; g >= lo; g -= kWavesOf) {
            const uint32_t key = (uint32_t)g * 64 + (63 - lane);
            const uint32_t c = wide ? s.hist[key & 0x7fff] : s.hist[key >> 1] >> (key & 1 ? 16 : 0) & 0xffff;
            if (__ballot(c != 0) == 0) continue;
            const double w = c ? exp(weight_log(key)) : 0.0;
            if (w >= (double)m_r) above += c;
            double sum = c * w;
            uint32_t n = c;
#pragma unroll
            for (int d = 32; d >= 1; d >>= 1) {
                sum += __shfl_xor(sum, d, 64);
                n += (uint32_t)__shfl_xor((int)n, d, 64);
            }
            if (lane == 0) {
                s.sum[g] = sum;
                s.count[g] = n;
            }
        }
    };
    const int g_lo = (int)(least >> 6), g_hi = (int)(most >> 6);
    sum_segments(g_lo, g_hi, false);
    // are all there?  (A counter of 16 bits that runs over takes 65,535 or
    // 65,536 from the sum of all.)
    auto block_count = [&](uint32_t v, uint32_t *words) -> uint32_t {
        v = wave_sum(v);
        __syncthreads();
        if (lane == 0) words[wave] = v;
        __syncthreads();
        uint32_t t = 0;
        for (int w = 0; w < kWavesOf; ++w) t += words[w];
        return t;
    };
    const uint32_t candidates = block_count(mine, s.w_count);
    const uint32_t got = block_count(s.count[tid], s.w_other);
    const bool wide = got != candidates;
    if (wide) {
        above = 0;
        __syncthreads();
        s.sum[tid] = 0.0;
        s.count[tid] = 0;
        for (int half = 1; half >= 0; --half) {
            count_half(half);
            sum_segments(max(g_lo, half * 512), min(g_hi, half * 512 + 511), true);
        }
    }
    const uint32_t n_above = block_count(above, s.w_count);
    // sums from the highest segment on
    const int g_of = kSegments - 1 - tid;
    double in_sum = s.sum[g_of];
    uint32_t in_count = s.count[g_of];
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const double x = shfl_up_d(in_sum, d);
        const uint32_t y = (uint32_t)__shfl_up((int)in_count, d, 64);
        if (lane >= d) {
            in_sum += x;
            in_count += y;
        }
    }
    __syncthreads();
    if (lane == 63) {
        s.w_sum[wave] = in_sum;
        s.w_count[wave] = in_count;
    }
    __syncthreads();
    double base = 0.0, total = 0.0;
    uint32_t base_count = 0;
    for (int w = 0; w < kWavesOf; ++w) {
        if (w < wave) {
            base += s.w_sum[w];
            base_count += s.w_count[w];
        }
        total += s.w_sum[w];
    }
    in_sum += base;
    in_count += base_count;
    s.sum[g_of] = in_sum;
    s.count[g_of] = in_count;
    __syncthreads();

    // sums before a segment
    auto sum_before = [&](int g) { return g == kSegments - 1 ? 0.0 : s.sum[g + 1]; };
    auto count_before = [&](int g) { return g == kSegments - 1 ? 0u : s.count[g + 1]; };
    // The 64 counts of a segment, the highest key first, one a lane: of all waves alike.
    auto bins_of = [&](int g) -> uint32_t {
        const uint32_t key = (uint32_t)g * 64 + (63 - lane);
        if (!wide) return s.hist[key >> 1] >> (key & 1 ? 16 : 0) & 0xffff;
        __syncthreads();
        if (tid < 64) s.bins[tid] = 0;
        __syncthreads();
        for (int32_t i = tid; i < row.pieces; i += kThreads) {
            uint32_t k[8];
            row.keys(i, k);
            for (int j = 0; j < 8; ++j)
                if (k[j] >= least && (int)(k[j] >> 6) == g) atomicAdd(&s.bins[63 - (k[j] & 63)], 1u);
        }
        __syncthreads();
        return s.bins[lane];
    };
    // Within a segment: the first lane whose key `hit` says yes to (ex: before the key, in: with it).
    auto look = [&](int g, auto hit) -> Found {
        const uint32_t c = bins_of(g);
        const uint32_t key = (uint32_t)g * 64 + (63 - lane);
        const double w = c ? exp(weight_log(key)) : 0.0;
        double in = c * w;
        uint32_t n = c;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const double x = shfl_up_d(in, d);
            const uint32_t y = (uint32_t)__shfl_up((int)n, d, 64);
            if (lane >= d) {
                in += x;
                n += y;
            }
        }
        in += sum_before(g);
        n += count_before(g);
        double ex = shfl_up_d(in, 1);
        if (lane == 0) ex = sum_before(g);
        const uint64_t yes = __ballot(c != 0 && hit(ex, in, n - c, n));
        const uint64_t some = __ballot(c != 0);
        const int at = yes ? __ffsll((unsigned long long)yes) - 1 : 63 - __clzll((long long)some);
        Found f;
        f.key = (int32_t)((uint32_t)g * 64 + (63 - at));
        f.sum = __shfl(ex, at, 64);
        f.weight = __shfl(w, at, 64);
        f.before = (uint32_t)__shfl((int)(n - c), at, 64);
        f.rank = (uint32_t)__shfl((int)c, at, 64);       // for now: how many there are
        return f;
    };
    // The first segment for which `hit` holds, or the last one that has candidates.
    auto segment_of = [&](auto hit) -> int {
        __syncthreads();
        if (tid == 0) s.segment = -1;
        __syncthreads();
        const uint32_t own = s.count[g_of] - count_before(g_of);
        if (own && hit(sum_before(g_of), s.sum[g_of], count_before(g_of), s.count[g_of])) atomicMax(&s.segment, g_of);
        __syncthreads();
        if (s.segment >= 0) return s.segment;
        __syncthreads();
        if (tid == 0) s.segment = kSegments;
        __syncthreads();
        if (own) atomicMin(&s.segment, g_of);
        __syncthreads();
        return s.segment;
    };
    // The item number i < candidates of the order.
    auto item = [&](uint32_t i) -> Found {
        auto hit = [=](double, double, uint32_t, uint32_t in) { return i < in; };
        Found f = look(segment_of(hit), hit);
        f.rank = i - f.before;
        return f;
    };
    auto sum_upto = [&](const Found &f) { return f.sum + (f.rank + 1.0) * f.weight; };

    uint32_t keep = candidates;
    double kept = total;
    Found last{};
    bool have_last = false;
    if (T_r == 0.0f || k_r == 1) {
        keep = 1;
    } else {
        if (k_r > 0 && (uint32_t)k_r < keep) {
            keep = (uint32_t)k_r;
            last = item(keep - 1);
            have_last = true;
            kept = sum_upto(last);
        }
        if (p_r < 1.0f) {
            const double want = (double)p_r * kept;
            // the first item with which the sum reaches it
            auto hit = [=](double, double in, uint32_t, uint32_t) { return in >= want; };
            const Found f = look(segment_of(hit), hit);
            double j = ceil((want - f.sum) / f.weight);
            j = fmin(fmax(j, 1.0), (double)f.rank);
            // (the quotient is rounded)
            if (j > 1.0 && f.sum + (j - 1.0) * f.weight >= want) j -= 1.0;
            else if (j < (double)f.rank && f.sum + j * f.weight < want) j += 1.0;
            const uint32_t upto = f.before + (uint32_t)j;
            if (upto < keep) {
                keep = upto;
                have_last = false;
            }
        }
        if (n_above < keep) {
            keep = max(1u, n_above);
            have_last = false;
        }
    }
    Found f{};
    if (keep == 1) {
        f.key = (int32_t)most;
        f.rank = 0;
    } else {
        if (keep < candidates) {
            if (!have_last) last = item(keep - 1);
            kept = sum_upto(last);
        }
        const float u = a.u[r];
        const double want = (double)u * kept;
        if (u < 1.0f) {
            auto hit = [=](double, double in, uint32_t, uint32_t) { return in > want; };
            f = look(segment_of(hit), hit);
            const double many = (double)f.rank;
            double j = floor((want - f.sum) / f.weight);
            j = fmin(fmax(j, 0.0), many - 1.0);
            if (j > 0.0 && f.sum + j * f.weight > want) j -= 1.0;
            else if (j < many - 1.0 && !(f.sum + (j + 1.0) * f.weight > want)) j += 1.0;
            f.rank = (uint32_t)j;
        }
        if (!(u < 1.0f) || f.before + f.rank >= keep) f = keep < candidates ? last : item(keep - 1);
    }
    if (tid == 0 && a.logprob) a.logprob[r] = (float)(weight_log((uint32_t)f.key) - log(total));

    // the token: of those that have the key, in order, number f.rank
    const int32_t rounds = (row.pieces + kThreads - 1) / kThreads;
    for (int32_t i = 0; i < rounds; ++i) {
        const int32_t piece = i * kThreads + tid;
        uint32_t n = 0;
        if (piece < row.pieces) {
            uint32_t k[8];
            row.keys(piece, k);
#pragma unroll
            for (int j = 0; j < 8; ++j) n += k[j] == (uint32_t)f.key;
        }
        n = wave_sum(n);
        if (lane == 0) s.tiles[i * kWavesOf + wave] = (uint16_t)n;
    }
    __syncthreads();
    if (wave != 0) return;
    const int32_t tiles = rounds * kWavesOf;
    uint32_t left = f.rank;
    int32_t tile = -1;
    for (int32_t i0 = 0; i0 < tiles && tile < 0; i0 += 64) {
        const uint32_t n = i0 + lane < tiles ? s.tiles[i0 + lane] : 0;
        const uint32_t upto = wave_incl_sum(n);
        const uint64_t yes = __ballot(upto > left);
        if (yes) {
            const int at = __ffsll((unsigned long long)yes) - 1;
            left -= (uint32_t)__shfl((int)(upto - n), at, 64);
            tile = i0 + at;
        } else {
            left -= (uint32_t)__shfl((int)upto, 63, 64);
        }
    }
    if (tile < 0) return;                            // (some tile has it)
    const int32_t piece = tile * 64 + lane;
    uint32_t k[8] = {};
    if (piece < row.pieces) row.keys(piece, k);
    uint32_t n = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) n += k[j] == (uint32_t)f.key;
    uint32_t at = wave_incl_sum(n) - n;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (k[j] == (uint32_t)f.key) {
            if (at == left) a.token[r] = piece * 8 - row.lead + j;
            ++at;
        }
}

hipError_t launch_sample(const Launch &L, const SampleArgs &a, int64_t n, int32_t dtype)
{
    if (dtype == RO_BF16)
        RO_LAUNCH(L, RO_K_SAMPLE, k_sample<__bf16>, dim3((unsigned)n), dim3(kThreads), 0, L.stream, a, L.ctl);
    else
        RO_LAUNCH(L, RO_K_SAMPLE, k_sample<_Float16>, dim3((unsigned)n), dim3(kThreads), 0, L.stream, a, L.ctl);
    return hipGetLastError();
}

}  // namespace ro
