// Pages of a pool: shared, taken, given back, moved together, copied.
//
// The pool is its counts alone.  What a call needs besides, a bit for every
// free page and the sums before it, is made from them in the call's first
// launch, so that nothing has to agree with them from call to call.  Taking
// the r-th free page of many is a search in those sums; no order of
// workgroups matters, and counts change by atomic additions only.
//
// Small calls are bound by their launches and by chains of dependent steps: 13 children
// released, forked, grown and copied take 16 to 20 us in four launches (2.8, 3.2, 7.3 and
// 4.0 us on the GPU, and as much of the host), 17 sequences moved together 14.7 in two (7.0
// and 5.5).  Copies are bound by memory: 4.6 GB read and written for
// a pool of 140,600 pages, half of them in use in 907 us, 5.0 TB/s.
#include "ro_step.h"

namespace ro {

namespace {

constexpr uint32_t kReplace = 1, kLeave = 2;    // of Pool::need: the last page is replaced; the row stays as it is
constexpr int64_t kMostPositions = (int64_t)1 << 30;
constexpr int kSmallPages = 32768;              // pages of a pool that one workgroup looks over
constexpr int64_t kSmallSeqs = 64;              // sequences that it grows (13: 7 us, two launches 9; 500: 15 and 14)
constexpr int64_t kSmallEntries = 16384;        // entries of tables that it renumbers (a row costs it 64 at least)

__device__ __forceinline__ int64_t pages_of(const Pool &p, int64_t positions)
{
    return (positions + (1 << p.page_shift) - 1) >> p.page_shift;
}

// Is a row's length one that its entries hold?
__device__ __forceinline__ bool row_ok(const Pool &p, const Tables &t, int32_t len)
{
    return len >= 0 && pages_of(p, len) <= t.stride;
}

__device__ __forceinline__ uint64_t wave_sum64(uint64_t v)
{
    return (uint64_t)__shfl((long long)wave_incl_sum_dpp(v), 63, 64);
}

// The bits of 4,096 pages from tile `tile` on, by a workgroup of 256.
__device__ __forceinline__ void mark_tile(const Pool &p, int64_t tile, uint32_t *s_sum)
{
    const int lane = lane_id(), wave = threadIdx.x >> 6;
    const int64_t from = tile * kPageTile + wave * 1024 + lane;
    int32_t n[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) n[i] = from + i * 64 < p.n_pages ? p.refs[from + i * 64] : 1;
    uint64_t mine = 0;
    uint32_t count = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const uint64_t b = __ballot(n[i] == 0);
        if (lane == i) mine = b;
        count += (uint32_t)__popcll(b);
    }
    if (lane < 16) p.free[tile * 64 + wave * 16 + lane] = mine;
    if (lane == 0) s_sum[wave] = count;
    __syncthreads();
    if (threadIdx.x == 0) p.tile_free[tile] = s_sum[0] + s_sum[1] + s_sum[2] + s_sum[3];
}

// Bit number k (from 0) of those that are set in w.
__device__ __forceinline__ int select_bit(uint64_t w, uint32_t k)
{
    uint32_t x = (uint32_t)w, n = (uint32_t)__popc(x);
    int at = 0;
    if (k >= n) {
        k -= n;
        x = (uint32_t)(w >> 32);
        at = 32;
    }
#pragma unroll
    for (int h = 16; h >= 1; h >>= 1) {
        n = (uint32_t)__popc(x & ((1u << h) - 1));
        if (k >= n) {
            k -= n;
            x >>= h;
            at += h;
        }
    }
    return at;
}

// What a sequence needs: pages << 2 | kReplace | kLeave.
__device__ __forceinline__ uint32_t need_of(const Pool &p, const Tables &t, int64_t s, int32_t len, int32_t more, Ctl *ctl)
{
    const int64_t want = (int64_t)len + more;
    if (!row_ok(p, t, len) || more < 0 || want > kMostPositions) {
        raise_err(ctl, RO_ERANGE);
        return kLeave;
    }
    if (pages_of(p, want) > t.stride) {
        raise_err(ctl, RO_ECAP);
        return kLeave;
    }
    if (more == 0) return 0;
    uint32_t need = (uint32_t)(pages_of(p, want) - pages_of(p, len)), replace = 0;
    if (len & ((1 << p.page_shift) - 1)) {
        const uint32_t last = t.table[s * t.stride + pages_of(p, len) - 1];
        if (last >= (uint32_t)p.n_pages) {
            raise_err(ctl, RO_ERANGE);
            return kLeave;
        }
        const int32_t names = p.refs[last];
        if (names <= 0) {                // (it would be handed out, here or in a later call)
            raise_err(ctl, RO_ESTATE);
            return kLeave;
        }
        if (names > 1) {
            replace = kReplace;
            ++need;
        }
    }
    return min(need, 1u << 25) << 2 | replace;   // (more than any pool has)
}

__device__ __forceinline__ int64_t page_tiles(const Pool &p) { return ((int64_t)p.n_pages + kPageTile - 1) / kPageTile; }

}  // namespace

// One workgroup a row.
__global__ void __launch_bounds__(256) k_pages_fork(Pool p, Tables from, const int32_t *parent, Tables to, Ctl *ctl)
{
    const int64_t i = blockIdx.x;
    const int32_t f = parent[i];
    if (f == -1) return;
    if (f < 0 || f >= from.n) {
        if (threadIdx.x == 0) raise_err(ctl, RO_ERANGE);
        return;
    }
    const int32_t len = from.len[f];
    if (to.len[i] != 0) {
        if (threadIdx.x == 0) raise_err(ctl, RO_ESTATE);
        return;
    }
    if (!row_ok(p, from, len) || pages_of(p, len) > to.stride) {
        if (threadIdx.x == 0) raise_err(ctl, row_ok(p, from, len) ? RO_ECAP : RO_ERANGE);
        return;
    }
    const int64_t n = pages_of(p, len);
    const uint32_t *src = from.table + f * from.stride;
    uint32_t *dst = to.table + i * to.stride;
    bool bad = false;
    for (int64_t c = threadIdx.x; c < n; c += 256) bad |= src[c] >= (uint32_t)p.n_pages;
    if (__syncthreads_or(bad)) {
        if (threadIdx.x == 0) raise_err(ctl, RO_ERANGE);
        return;
    }
    for (int64_t c = threadIdx.x; c < n; c += 256) {
        dst[c] = src[c];
        atomicAdd(&p.refs[src[c]], 1);
    }
    if (threadIdx.x == 0) to.len[i] = len;
}

// One workgroup a row.
__global__ void __launch_bounds__(256) k_pages_release(Pool p, Tables t, const int32_t *keep, Ctl *ctl)
{
    const int64_t s = blockIdx.x;
    const int32_t len = t.len[s], kept = keep ? keep[s] : 0;
    if (!row_ok(p, t, len) || kept < 0) {
        if (threadIdx.x == 0) raise_err(ctl, RO_ERANGE);
        return;
    }
    if (kept >= len) return;
    uint32_t *row = t.table + s * t.stride;
    const int64_t n = pages_of(p, len);
    for (int64_t c = pages_of(p, kept) + threadIdx.x; c < n; c += 256) {
        const uint32_t page = row[c];
        row[c] = (uint32_t)RO_NO_PAGE;
        if (page >= (uint32_t)p.n_pages) {
            raise_err(ctl, RO_ERANGE);
        } else if (atomicAdd(&p.refs[page], -1) <= 0) {
            atomicAdd(&p.refs[page], 1);
            raise_err(ctl, RO_ESTATE);
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) t.len[s] = kept;
}

// Workgroups of tiles of pages, then of sequences.
__global__ void __launch_bounds__(256) k_pages_need(Pool p, Tables t, const int32_t *add, int64_t *n_free, Ctl *ctl)
{
    __shared__ uint32_t s_sum[4];
    __shared__ uint64_t s_need[4];
    const int64_t tiles = page_tiles(p);
    if (blockIdx.x == 0 && threadIdx.x == 0 && n_free) *n_free = 0;
    if (blockIdx.x < tiles) {
        mark_tile(p, blockIdx.x, s_sum);
        return;
    }
    const int64_t tile = blockIdx.x - tiles, s = tile * kSeqTile + threadIdx.x;
    uint64_t need = 0;
    if (s < t.n) {
        const uint32_t word = need_of(p, t, s, t.len[s], add[s], ctl);
        p.need[s] = word;
        need = word >> 2;
    }
    const uint64_t sum = wave_sum64(need);
    if (lane_id() == 0) s_need[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) p.tile_need[tile] = s_need[0] + s_need[1] + s_need[2] + s_need[3];
}

// A wave a sequence, kTakes of them a workgroup: its pages are the free ones
// from as many on as the sequences before it need.
constexpr int kTakes = 4;
__global__ void __launch_bounds__(256) k_pages_take(Pool p, Tables t, const int32_t *add, uint32_t *src, uint32_t *dst,
                                                    int32_t *slots, int64_t *n_free, Ctl *ctl)
{
    __shared__ uint64_t s_a[4], s_b[4], s_c[4];
    const int lane = lane_id(), wave = threadIdx.x >> 6, tid = threadIdx.x;
    const int64_t tiles = page_tiles(p), seq_tiles = (t.n + kSeqTile - 1) / kSeqTile;
    const int64_t s0 = (int64_t)blockIdx.x * kTakes, mine = s0 / kSeqTile;
    // all pages that are free, all that are needed, and those needed before this workgroup's
    uint64_t free = 0, need = 0, before = 0;
    for (int64_t i = tid; i < tiles; i += 256) free += p.tile_free[i];
    for (int64_t i = tid; i < seq_tiles; i += 256) {
        const uint64_t x = p.tile_need[i];
        need += x;
        before += i < mine ? x : 0;
    }
    if (mine * kSeqTile + tid < s0) before += p.need[mine * kSeqTile + tid] >> 2;
    free = wave_sum64(free);
    need = wave_sum64(need);
    before = wave_sum64(before);
    if (lane == 0) {
        s_a[wave] = free;
        s_b[wave] = need;
        s_c[wave] = before;
    }
    __syncthreads();
    free = s_a[0] + s_a[1] + s_a[2] + s_a[3];
    need = s_b[0] + s_b[1] + s_b[2] + s_b[3];
    before = s_c[0] + s_c[1] + s_c[2] + s_c[3];
    const bool enough = need <= free;
    if (blockIdx.x == 0 && tid == 0) {
        if (!enough) raise_err(ctl, RO_ECAP);
        if (n_free) atomicAdd((unsigned long long *)n_free, (unsigned long long)(enough ? free - need : free));
    }
    const int64_t s = s0 + wave;
    if (s >= t.n) return;
    const uint32_t word = p.need[s];
    const int32_t len = t.len[s];
    const bool replace = enough && (word & kReplace);
    uint32_t old = 0;
    int64_t first = 0;
    uint32_t *row = t.table + s * t.stride;
    if (enough && (word & kLeave) == 0) {
        first = pages_of(p, len) - (replace ? 1 : 0);
        if (replace) old = row[first];
    }
    if (lane == 0) {
        src[s] = replace ? old : (uint32_t)RO_NO_PAGE;
        slots[s] = replace ? len & ((1 << p.page_shift) - 1) : 0;
        if (!replace) dst[s] = (uint32_t)RO_NO_PAGE;
    }
    if (!enough || (word & kLeave)) return;
    if (lane == 0) {
        t.len[s] = len + add[s];
        if (replace && atomicAdd(&p.refs[old], -1) == 1 && n_free) atomicAdd((unsigned long long *)n_free, 1ull);
    }
    int64_t left = word >> 2;
    if (left == 0) return;
    for (int w = 0; w < wave; ++w) before += p.need[s0 + w] >> 2;
    // the tile that the first one lies in
    int64_t tile = 0;
    uint64_t skip = before;                              // free pages to pass from the tile's start
    for (int64_t i0 = 0; i0 < tiles; i0 += 64) {
        const uint64_t x = i0 + lane < tiles ? p.tile_free[i0 + lane] : 0;
        const uint64_t upto = wave_incl_sum_dpp(x);
        const uint64_t beyond = __ballot(upto > skip);
        if (beyond) {
            const int at = __ffsll((unsigned long long)beyond) - 1;
            skip -= (uint64_t)__shfl((long long)(upto - x), at, 64);
            tile = i0 + at;
            break;
        }
        skip -= (uint64_t)__shfl((long long)upto, 63, 64);
    }
    int64_t col = first;
    for (; left > 0; ++tile) {                           // (enough are free: it ends before the tiles do)
        uint64_t word_free = p.free[tile * 64 + lane];
        const uint64_t n = (uint64_t)__popcll(word_free);
        const uint64_t upto = wave_incl_sum_dpp(n);
        const int64_t all = __shfl((long long)upto, 63, 64);
        auto take = [&](int64_t rank, uint32_t page) {
            row[col + rank] = page;
            p.refs[page] = 1;
            if (replace && col + rank == first) dst[s] = page;
        };
        if (left <= 128) {                               // a lane a page
            const int64_t most = min64(left, all - (int64_t)skip);
            for (int64_t r0 = 0; r0 < most; r0 += 64) {
                const uint32_t want = (uint32_t)((int64_t)skip + min64(r0 + lane, most - 1));
                int at = 0;                              // the first lane whose sum exceeds it
#pragma unroll
                for (int h = 32; h >= 1; h >>= 1)
                    if ((uint32_t)__shfl((int)(uint32_t)upto, at + h - 1, 64) <= want) at += h;
                const uint32_t with = (uint32_t)__shfl((int)(uint32_t)upto, max(at - 1, 0), 64), before_at = at ? with : 0;
                const uint64_t w = (uint64_t)__shfl((long long)word_free, at, 64);
                if (r0 + lane < most) take(r0 + lane, (uint32_t)(tile * kPageTile + at * 64 + select_bit(w, want - before_at)));
            }
        } else {                                         // a lane a word
            int64_t rank = (int64_t)(upto - n) - (int64_t)skip;
            while (word_free) {
                const int bit = __ffsll((unsigned long long)word_free) - 1;
                word_free &= word_free - 1;
                if (rank >= 0 && rank < left) take(rank, (uint32_t)(tile * kPageTile + lane * 64 + bit));
                ++rank;
            }
        }
        const int64_t took = min64(left, all - (int64_t)skip);
        col += took;
        left -= took;
        skip = 0;
    }
}

__global__ void __launch_bounds__(256) k_pages_mark(Pool p)
{
    __shared__ uint32_t s_sum[4];
    mark_tile(p, blockIdx.x, s_sum);
}

// The lists of pages that move and of those they move to; how many pages in
// use lie before every word.
__global__ void __launch_bounds__(256) k_pages_moves(Pool p, uint32_t *src, uint32_t *dst, int64_t *n_moves, int64_t *n_free)
{
    __shared__ uint64_t s_a[4], s_b[4], s_c[4];
    const int lane = lane_id(), wave = threadIdx.x >> 6, tid = threadIdx.x;
    const int64_t tiles = page_tiles(p), tile = blockIdx.x;
    uint64_t sum = 0, before = 0;
    for (int64_t i = tid; i < tiles; i += 256) {
        const uint64_t x = p.tile_free[i];
        sum += x;
        before += i < tile ? x : 0;
    }
    sum = wave_sum64(sum);
    before = wave_sum64(before);
    if (lane == 0) {
        s_a[wave] = sum;
        s_b[wave] = before;
    }
    __syncthreads();
    const int64_t free = (int64_t)(s_a[0] + s_a[1] + s_a[2] + s_a[3]);
    before = s_b[0] + s_b[1] + s_b[2] + s_b[3];
    const int64_t live = p.n_pages - free;
    // free pages below `live`: as many as pages in use from there on
    const int64_t edge = live / kPageTile;
    uint64_t holes = 0;
    for (int64_t i = tid; i < edge; i += 256) holes += p.tile_free[i];
    if (tid < 64 && live < p.n_pages) {
        const int64_t from = edge * kPageTile + tid * 64;
        const uint64_t w = p.free[edge * 64 + tid];
        holes += from + 64 <= live ? __popcll(w) : from < live ? __popcll(w & ((1ull << (live - from)) - 1)) : 0;
    }
    holes = wave_sum64(holes);
    if (lane == 0) s_c[wave] = holes;
    __syncthreads();
    const int64_t moves = (int64_t)(s_c[0] + s_c[1] + s_c[2] + s_c[3]);
    if (tile == 0 && tid == 0) {
        *n_moves = moves;
        if (n_free) *n_free = free;
    }
    if (wave != 0) return;
    const int64_t at = tile * kPageTile + lane * 64;
    uint64_t w = p.free[tile * 64 + lane];
    const uint64_t n = (uint64_t)__popcll(w);
    int64_t rank = (int64_t)(before + wave_incl_sum_dpp(n) - n);          // free pages before the word
    p.before[tile * 64 + lane] = (uint32_t)(at < p.n_pages ? at - rank : live);
    int64_t used = at - rank - (live - moves);                            // pages in use from `live` on, before the word
    if (at < live) {
        uint64_t below = at + 64 <= live ? w : w & ((1ull << (live - at)) - 1);
        while (below) {
            const int bit = __ffsll((unsigned long long)below) - 1;
            below &= below - 1;
            dst[rank++] = (uint32_t)(at + bit);
        }
    }
    if (at + 64 > live && at < p.n_pages) {
        uint64_t above = ~w;
        if (at + 64 > p.n_pages) above &= (1ull << (p.n_pages - at)) - 1;
        if (at < live) {
            above &= ~((1ull << (live - at)) - 1);
            used = 0;
        }
        while (above) {
            const int bit = __ffsll((unsigned long long)above) - 1;
            above &= above - 1;
            src[used++] = (uint32_t)(at + bit);
        }
    }
}

struct TableList {
    Tables t[kMaxTables];
    int64_t row0[kMaxTables + 1];        // rows of the tables before
    int32_t n;
};

// Workgroups of the moves of counts, then one a row.
__global__ void __launch_bounds__(256) k_pages_renumber(Pool p, TableList tables, const uint32_t *src, const uint32_t *dst,
                                                        const int64_t *n_moves, int32_t move_blocks, Ctl *ctl)
{
    const int64_t moves = *n_moves;
    if ((int32_t)blockIdx.x < move_blocks) {
        for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < moves; i += (int64_t)move_blocks * 256) {
            p.refs[dst[i]] = p.refs[src[i]];
            p.refs[src[i]] = 0;
        }
        return;
    }
    const int64_t r = blockIdx.x - move_blocks;
    int k = 0;
    while (k + 1 < tables.n && r >= tables.row0[k + 1]) ++k;
    const Tables t = tables.t[k];
    const int64_t s = r - tables.row0[k];
    const int32_t len = t.len[s];
    if (!row_ok(p, t, len)) {
        if (threadIdx.x == 0) raise_err(ctl, RO_ERANGE);
        return;
    }
    // pages in use: those before the last tile's end
    const int64_t tiles = page_tiles(p);
    int64_t live = 0;
    if (tiles > 0) {
        live = p.n_pages;
        // (counted here from the last tile on: its first word's sum, and what is in use after it)
        const int64_t w0 = (tiles - 1) * 64;
        live = p.before[w0] + (p.n_pages - w0 * 64) - p.tile_free[tiles - 1];
    }
    uint32_t *row = t.table + s * t.stride;
    for (int64_t c = threadIdx.x; c < pages_of(p, len); c += 256) {
        const uint32_t page = row[c];
        if (page >= (uint32_t)p.n_pages) {
            raise_err(ctl, RO_ERANGE);
            continue;
        }
        const uint64_t w = p.free[page >> 6];
        if (w >> (page & 63) & 1) {
            raise_err(ctl, RO_ESTATE);
            continue;
        }
        if (page < live) continue;
        const int64_t rank = p.before[page >> 6] + __popcll(~w & ((1ull << (page & 63)) - 1)) - (live - moves);
        row[c] = dst[rank];
    }
}

// Small pools: one workgroup does it all, and a launch less, or two, is more
// than what it waits for.
constexpr int kSmall = 1024;
struct SmallPool {
    uint64_t free[kSmallPages / 64];
    uint32_t before[kSmallPages / 64 + 1];       // free pages before a word; all of them
    uint32_t wave[kSmall / 64];
};

// Bits of free pages and the sums before them.
__device__ __forceinline__ void mark_small(const Pool &p, SmallPool &s)
{
    const int lane = lane_id(), wave = threadIdx.x >> 6, words = kSmallPages / 64;
    constexpr int kEach = kSmallPages / kSmall;
    int32_t n[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int32_t page = (wave * kEach + i) * 64 + lane;
        n[i] = page < p.n_pages ? p.refs[page] : 1;
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const uint64_t b = __ballot(n[i] == 0);
        if (lane == 0) s.free[wave * kEach + i] = b;
    }
    __syncthreads();
    const uint32_t count = threadIdx.x < words ? (uint32_t)__popcll(s.free[threadIdx.x]) : 0;
    const uint32_t in = wave_incl_sum(count);
    if (lane == 63) s.wave[wave] = in;
    __syncthreads();
    uint32_t base = 0;
    for (int w = 0; w < wave; ++w) base += s.wave[w];
    if (threadIdx.x < words) s.before[threadIdx.x + 1] = base + in;
    if (threadIdx.x == 0) s.before[0] = 0;
    __syncthreads();
}

// Free page number k, and page in use number k, from 0.
__device__ __forceinline__ uint32_t free_page(const SmallPool &s, uint32_t k)
{
    int at = 0;
#pragma unroll
    for (int h = kSmallPages / 128; h >= 1; h >>= 1)
        if (s.before[at + h] <= k) at += h;
    return (uint32_t)(at * 64 + select_bit(s.free[at], k - s.before[at]));
}
__device__ __forceinline__ uint32_t used_page(const SmallPool &s, uint32_t k)
{
    int at = 0;
#pragma unroll
    for (int h = kSmallPages / 128; h >= 1; h >>= 1)
        if ((at + h) * 64 - s.before[at + h] <= k) at += h;
    return (uint32_t)(at * 64 + select_bit(~s.free[at], k - (at * 64 - s.before[at])));
}

__global__ void __launch_bounds__(kSmall) k_pages_grow_small(Pool p, Tables t, const int32_t *add, uint32_t *src, uint32_t *dst,
                                                             int32_t *slots, int64_t *n_free, Ctl *ctl)
{
    __shared__ SmallPool s;
    __shared__ uint32_t s_off[kSmall + 1], s_first[kSmall], s_wave[kSmall / 64], s_dropped;
    const int tid = threadIdx.x, lane = lane_id(), wave = tid >> 6, n = (int)t.n;
    const int32_t len = tid < n ? t.len[tid] : 0, more = tid < n ? add[tid] : 0;
    const uint32_t word = tid < n ? need_of(p, t, tid, len, more, ctl) : 0;
    mark_small(p, s);
    // (each sum saturates far above a small pool's pages)
    uint32_t need = min(word >> 2, (uint32_t)kSmallPages + 1);
    const uint32_t in = wave_incl_sum(need);
    if (lane == 63) s_wave[wave] = in;
    if (tid == 0) s_dropped = 0;
    __syncthreads();
    uint32_t base = 0, all = 0;
    for (int w = 0; w < kSmall / 64; ++w) {
        base += w < wave ? s_wave[w] : 0;
        all += s_wave[w];
    }
    const uint32_t free = s.before[kSmallPages / 64];
    const bool enough = all <= free, replace = enough && (word & kReplace);
    const bool moves = enough && (word & kLeave) == 0;
    s_off[tid + 1] = base + in;
    if (tid == 0) {
        s_off[0] = 0;
        if (!enough) raise_err(ctl, RO_ECAP);
    }
    const int64_t first = moves ? pages_of(p, len) - (replace ? 1 : 0) : 0;
    s_first[tid] = (uint32_t)first << 1 | (replace ? 1 : 0);
    if (tid < n) {
        const uint32_t old = replace ? t.table[tid * t.stride + first] : (uint32_t)RO_NO_PAGE;
        src[tid] = old;
        slots[tid] = replace ? len & ((1 << p.page_shift) - 1) : 0;
        if (!replace) dst[tid] = (uint32_t)RO_NO_PAGE;
        if (moves) t.len[tid] = len + more;
        if (replace && atomicAdd(&p.refs[old], -1) == 1) atomicAdd(&s_dropped, 1u);
    }
    __syncthreads();
    if (tid == 0 && n_free) *n_free = (int64_t)free - (enough ? all : 0) + s_dropped;
    if (!enough) return;
    for (uint32_t j = tid; j < all; j += kSmall) {
        int q = 0;                               // whose page it is
#pragma unroll
        for (int h = kSmall / 2; h >= 1; h >>= 1)
            if (s_off[q + h] <= j) q += h;
        const uint32_t page = free_page(s, j), nth = j - s_off[q];
        t.table[q * t.stride + (s_first[q] >> 1) + nth] = page;
        p.refs[page] = 1;
        if (nth == 0 && (s_first[q] & 1)) dst[q] = page;
    }
}

__global__ void __launch_bounds__(kSmall) k_pages_compact_small(Pool p, TableList tables, uint32_t *src, uint32_t *dst,
                                                                int64_t *n_moves, int64_t *n_free, Ctl *ctl)
{
    __shared__ SmallPool s;
    mark_small(p, s);
    const int tid = threadIdx.x;
    const uint32_t free = s.before[kSmallPages / 64], live = (uint32_t)p.n_pages - free;
    auto free_before = [&](uint32_t page) -> uint32_t {
        return s.before[page >> 6] + (page & 63 ? (uint32_t)__popcll(s.free[page >> 6] & ((1ull << (page & 63)) - 1)) : 0);
    };
    const uint32_t moves = live < (uint32_t)kSmallPages ? free_before(live) : 0;
    if (tid == 0) {
        *n_moves = moves;
        if (n_free) *n_free = free;
    }
    for (uint32_t i = tid; i < moves; i += kSmall) {
        const uint32_t a = used_page(s, live - moves + i), b = free_page(s, i);
        src[i] = a;
        dst[i] = b;
        p.refs[b] = p.refs[a];
        p.refs[a] = 0;
    }
    // a wave a row
    for (int64_t r = tid >> 6; r < tables.row0[tables.n]; r += kSmall / 64) {
        int k = 0;
        while (k + 1 < tables.n && r >= tables.row0[k + 1]) ++k;
        const Tables t = tables.t[k];
        const int64_t q = r - tables.row0[k];
        const int32_t len = t.len[q];
        if (!row_ok(p, t, len)) {
            if (lane_id() == 0) raise_err(ctl, RO_ERANGE);
            continue;
        }
        for (int64_t c = lane_id(); c < pages_of(p, len); c += 64) {
            const uint32_t page = t.table[q * t.stride + c];
            if (page >= (uint32_t)p.n_pages)
                raise_err(ctl, RO_ERANGE);
            else if (s.free[page >> 6] >> (page & 63) & 1)
                raise_err(ctl, RO_ESTATE);
            else if (page >= live)
                t.table[q * t.stride + c] = free_page(s, page - free_before(page) - (live - moves));
        }
    }
}

// Pages to pages: an item is a page of keys or values.
__global__ void __launch_bounds__(256) k_pages_copy(CopyArgs a, Ctl *ctl)
{
    using u32x4 = uint32_t __attribute__((ext_vector_type(4)));
    int64_t n = a.n;
    if (a.n_dev) n = max64(0, min64(n, *a.n_dev));
    const int32_t lane_pieces = a.head_dim / 8;
    for (int64_t item = blockIdx.x; item < n * a.n_arrays; item += gridDim.x) {
        const int64_t i = item / a.n_arrays;
        const uint32_t from = a.src[i], to = a.dst[i];
        if (from == (uint32_t)RO_NO_PAGE || to == (uint32_t)RO_NO_PAGE) continue;
        const int32_t slots = a.slots ? a.slots[i] : a.page_size;
        if (from >= a.n_pages || to >= a.n_pages || slots < 0 || slots > a.page_size) {
            if (threadIdx.x == 0) raise_err(ctl, RO_ERANGE);
            continue;
        }
        uint16_t *base = a.at[item % a.n_arrays];
        const uint16_t *x = base + (int64_t)from * a.page;
        uint16_t *y = base + (int64_t)to * a.page;
        const int64_t pieces = (int64_t)slots * a.heads * lane_pieces;
        for (int64_t j = threadIdx.x; j < pieces; j += 256) {
            const int64_t row = j / lane_pieces;
            const int64_t at = row / slots * a.head + row % slots * a.slot + j % lane_pieces * 8;
            *(u32x4 *)(y + at) = *(const u32x4 *)(x + at);
        }
    }
}

hipError_t launch_pages_fork(const Launch &L, const Pool &p, const Tables &from, const int32_t *parent, const Tables &to)
{
    RO_LAUNCH(L, RO_K_PAGES, k_pages_fork, dim3((unsigned)to.n), dim3(256), 0, L.stream, p, from, parent, to, L.ctl);
    return hipGetLastError();
}

hipError_t launch_pages_release(const Launch &L, const Pool &p, const Tables &t, const int32_t *keep)
{
    RO_LAUNCH(L, RO_K_PAGES, k_pages_release, dim3((unsigned)t.n), dim3(256), 0, L.stream, p, t, keep, L.ctl);
    return hipGetLastError();
}

static int64_t most(int64_t a, int64_t b) { return a > b ? a : b; }
static int64_t least(int64_t a, int64_t b) { return a < b ? a : b; }
static int64_t tiles_of(const Pool &p) { return ((int64_t)p.n_pages + kPageTile - 1) / kPageTile; }

hipError_t launch_pages_grow(const Launch &L, const Pool &p, const Tables &t, const int32_t *add, uint32_t *src,
                             uint32_t *dst, int32_t *slots, int64_t *n_free)
{
    if (p.n_pages <= kSmallPages && t.n <= kSmallSeqs) {
        RO_LAUNCH(L, RO_K_PAGES, k_pages_grow_small, dim3(1), dim3(kSmall), 0, L.stream, p, t, add, src, dst, slots, n_free,
                  L.ctl);
        return hipGetLastError();
    }
    const int64_t blocks = most(1, tiles_of(p) + (t.n + kSeqTile - 1) / kSeqTile);
    RO_LAUNCH(L, RO_K_PAGES, k_pages_need, dim3((unsigned)blocks), dim3(256), 0, L.stream, p, t, add, n_free, L.ctl);
    RO_LAUNCH(L, RO_K_PAGES, k_pages_take, dim3((unsigned)most(1, (t.n + kTakes - 1) / kTakes)), dim3(256), 0, L.stream, p, t, add,
              src, dst, slots, n_free, L.ctl);
    return hipGetLastError();
}

hipError_t launch_pages_compact(const Launch &L, const Pool &p, const Tables *tables, int32_t n_tables, uint32_t *src,
                                uint32_t *dst, int64_t *n_moves, int64_t *n_free)
{
    TableList list{};
    int64_t entries = 0;
    for (int32_t i = 0; i < n_tables; ++i) {
        list.t[i] = tables[i];
        list.row0[i + 1] = list.row0[i] + tables[i].n;
        entries += tables[i].n * (64 + tables[i].stride);
    }
    list.n = n_tables;
    if (p.n_pages <= kSmallPages && entries <= kSmallEntries) {
        RO_LAUNCH(L, RO_K_PAGES, k_pages_compact_small, dim3(1), dim3(kSmall), 0, L.stream, p, list, src, dst, n_moves, n_free,
                  L.ctl);
        return hipGetLastError();
    }
    const int64_t tiles = most(1, tiles_of(p));
    RO_LAUNCH(L, RO_K_PAGES, k_pages_mark, dim3((unsigned)tiles), dim3(256), 0, L.stream, p);
    RO_LAUNCH(L, RO_K_PAGES, k_pages_moves, dim3((unsigned)tiles), dim3(256), 0, L.stream, p, src, dst, n_moves, n_free);
    const int32_t move_blocks = (int32_t)least(256, ((int64_t)p.n_pages / 2 + 255) / 256 + 1);
    RO_LAUNCH(L, RO_K_PAGES, k_pages_renumber, dim3((unsigned)(move_blocks + list.row0[n_tables])), dim3(256), 0, L.stream,
              p, list, (const uint32_t *)src, (const uint32_t *)dst, (const int64_t *)n_moves, move_blocks, L.ctl);
    return hipGetLastError();
}

hipError_t launch_pages_copy(const Launch &L, const CopyArgs &a)
{
    const int64_t blocks = least(a.n * a.n_arrays, (int64_t)L.num_cus * 8);
    RO_LAUNCH(L, RO_K_PAGES_COPY, k_pages_copy, dim3((unsigned)blocks), dim3(256), 0, L.stream, a, L.ctl);
    return hipGetLastError();
}

}  // namespace ro
