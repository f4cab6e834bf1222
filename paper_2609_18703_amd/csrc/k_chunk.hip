// The plan of a chunk.
//
// Copies and checks what the chunk's kernels read again and again: lengths,
// page ids, and for every token the cache position it goes to.  After it no
// kernel has to check an index that came from the caller, and one plan serves
// all layers of a model.
#include "ro_chunk.h"

namespace ro {

// A sequence's tokens and length, or nothing if they are invalid.
__device__ __forceinline__ ChunkSeq read_seq(const Chunk &c, const PlanArgs &a, int64_t s, int &err)
{
    const int64_t q0 = a.q_off[s], q1 = a.q_off[s + 1], L = a.kv_len[s];
    ChunkSeq r = {0, 0, 0, 0};
    if (q0 < 0 || q1 < q0 || q1 > c.n_tokens || (s == 0 && q0 != 0) || (s == c.n_seqs - 1 && q1 != c.n_tokens)) {
        err = RO_EINVAL;
        r.bad = 1;
    } else if (q1 - q0 > a.max_new || L < 0 || L > c.cols << c.page_shift || (L > 0 && a.n_pages == 0) ||
             (L + (1 << c.page_shift) - 1) >> c.page_shift > a.table_stride)
        err = RO_ERANGE;
    else
        r = {(int32_t)q0, (int32_t)(q1 - q0), (int32_t)L, 0};
    return r;
}

__global__ __launch_bounds__(kBlock) void k_chunk_plan(Chunk c, PlanArgs a, Ctl *ctl)
{
    const int64_t s = blockIdx.x;
    const int64_t g = (int64_t)blockIdx.y * kBlock + threadIdx.x, step = (int64_t)gridDim.y * kBlock;
    int err = 0;
    if (s < c.n_seqs) {
        const ChunkSeq q = read_seq(c, a, s, err);
        if (blockIdx.y == 0 && threadIdx.x == 0) c.seq[s] = q;
        const int64_t np = (q.L + (1ll << c.page_shift) - 1) >> c.page_shift;
        for (int64_t i = g; i < np; i += step) {
            uint32_t id = a.table[s * a.table_stride + i];
            if (id >= a.n_pages) {
                err = RO_ERANGE;
                id = 0;
            }
            c.table[s * c.cols + i] = id;
        }
    }
    // tokens, spread over all workgroups
    const int64_t all = (int64_t)gridDim.x * step;
    for (int64_t t = s * step + g; t < c.n_tokens; t += all) {
        int64_t lo = 0, hi = c.n_seqs;          // the last sequence that starts at or before t
        while (hi - lo > 1) {
            const int64_t mid = (lo + hi) >> 1;
            if (a.q_off[mid] <= t) lo = mid;
            else hi = mid;
        }
        uint64_t slot = ~0ull;
        uint32_t of = ~0u;
        if (c.n_seqs > 0) {
            int e = 0;
            const ChunkSeq q = read_seq(c, a, lo, e);
            if (t >= q.q0 && t < (int64_t)q.q0 + q.n) {
                of = (uint32_t)lo;
                const int64_t j = (int64_t)q.L - q.n + (t - q.q0);
                if (j >= 0) {
                    const uint32_t id = a.table[lo * a.table_stride + (j >> c.page_shift)];
                    if (id < a.n_pages) slot = (uint64_t)id << 32 | (uint32_t)(j & ((1ll << c.page_shift) - 1));
                }
            }
        }
        c.slot[t] = slot;
        c.tok[t] = of;
    }
    if (err) raise_err(ctl, err);
}

constexpr int kPlan = 1024;

// Exclusive sum over the workgroup, and its total.
template <typename T>
__device__ __forceinline__ T plan_scan(T v, T *s_wave, T &total)
{
    const T in = wave_incl_sum(v);
    const int wave = threadIdx.x >> 6;
    if (lane_id() == 63) s_wave[wave] = in;
    __syncthreads();
    T before = 0;
    total = 0;
    for (int w = 0; w < kPlan / 64; ++w) {
        const T x = s_wave[w];
        if (w < wave) before += x;
        total += x;
    }
    __syncthreads();
    return before + in - v;
}
__device__ __forceinline__ int64_t plan_sum(int64_t v, int64_t *s_wave)
{
    v = wave_sum(v);
    if (lane_id() == 0) s_wave[threadIdx.x >> 6] = v;
    __syncthreads();
    int64_t total = 0;
    for (int w = 0; w < kPlan / 64; ++w) total += s_wave[w];
    __syncthreads();
    return total;
}

// Tile f of all wide tiles: its sequence and first row.
__device__ __forceinline__ void wide_tile(const Chunk &c, int32_t f, int32_t &s, int32_t &row0)
{
    int32_t lo = 0, hi = c.n_seqs;              // the last sequence whose tiles start at or before f
    while (hi - lo > 1) {
        const int32_t mid = (lo + hi) >> 1;
        if (c.tile_off[mid] <= f) lo = mid;
        else hi = mid;
    }
    s = lo;
    row0 = (f - c.tile_off[lo]) * kManyRows;
}

// How many key tiles an item has at most: of cuts that make kCuts numbers of
// items where no end of a tile of rows is in the way, the one whose last item
// should end first.
constexpr int kCuts = 4;
struct CutSums {
    int64_t items[kPlan / 64][kCuts];
    int32_t longest[kPlan / 64];
};
// `n` tiles of rows with w key tiles in all, for all key / value heads, in
// items of `least` or more; all_of(i, rows): those of one, or 0, and its rows;
// end_of(items, longest item, parts and rows of the longest tile): when the
// last item should end.
template <typename F, typename G>
__device__ __forceinline__ int32_t choose_cut(const Chunk &c, CutSums *s, int32_t n, int64_t w, int32_t unit, int32_t least,
                                              F all_of, G end_of)
{
    if (w <= (int64_t)least * unit / 2) return least;
    int32_t cut[kCuts], longest = 0;              // longest: key tiles (up to 2^22) << 8 | rows
    int64_t items[kCuts] = {};
#pragma unroll
    for (int m = 0; m < kCuts; ++m)
        cut[m] = (int32_t)min64(1 << 30, max64(m ? least : 2 * least, (w + unit * (m + 1) - 1) / (unit * (m + 1))));
    for (int32_t i = threadIdx.x; i < n; i += kPlan) {
        int32_t rows = 0;
        const int32_t all = all_of(i, rows);
        longest = max(longest, min(all, 1 << 22) << 8 | rows);
#pragma unroll
        for (int m = 0; m < kCuts; ++m) items[m] += (all + cut[m] - 1) / cut[m];
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) longest = max(longest, __shfl_xor(longest, d, 64));
    const int wave = threadIdx.x >> 6;
#pragma unroll
    for (int m = 0; m < kCuts; ++m) {
        const int64_t x = wave_sum(items[m]);
        if (lane_id() == 0) s->items[wave][m] = x;
    }
    if (lane_id() == 0) s->longest[wave] = longest;
    __syncthreads();
    longest = 0;
    for (int v = 0; v < kPlan / 64; ++v) longest = max(longest, s->longest[v]);
    const int32_t rows = longest & 255;
    longest >>= 8;
    int32_t best = 0;
    int64_t ends = 0;
#pragma unroll
    for (int m = 0; m < kCuts; ++m) {
        int64_t sum = 0;
        for (int v = 0; v < kPlan / 64; ++v) sum += s->items[v][m];
        const int64_t end = end_of(sum * c.kv_heads, (int64_t)min(longest, cut[m]), (int64_t)(longest + cut[m] - 1) / cut[m], rows);
        if (m == 0 || end < ends) {
            ends = end;
            best = cut[m];
        }
    }
    __syncthreads();
    return best;
}

// Few rows: the chip holds `slots` items at a time, and each costs kItem tiles
// more than its own, for the chain of loads before and the sums after.  If all
// items run at once the longest ends last; else the last one is half an item
// behind the chip's share of all work.  Where it pays: one, and four items a
// CU, for 32 sequences of 1,000 positions, 8 heads of 128, 23 and 37 us; for
// 100 of 1,500, 4 heads, 53 and 66; but 64 of 700 to 32,768 814 and 744.
constexpr int64_t kItem = 8;
__device__ __forceinline__ int32_t few_cut(const Chunk &c, int64_t w, CutSums *s)
{
    const int32_t cus = c.few_slots / 4, slots = c.head_dim == 64 ? 2 * cus : cus;
    auto all_of = [&](int32_t i, int32_t &rows) {
        const ChunkSeq q = c.seq[i];
        rows = min(q.n * c.group, 255);
        return rows > 0 && rows <= c.few_rows ? max(1, span_of(c, q, 0, kFewRows).all) : 0;
    };
    return choose_cut(c, s, c.n_seqs, w, cus, kFewCut, all_of, [&](int64_t items, int64_t longest, int64_t, int32_t) {
        return items <= slots ? 2 * (longest + kItem) : 2 * (w + items * kItem) / slots + longest + 2 * kItem;      // in half tiles
    });
}

// Many rows: a cut costs more, since up to 64 KB of sums an item go to memory
// and back and one workgroup joins them: ten tiles and one for each part, if
// all rows are there.  A
// workgroup that has its CU alone is a quarter faster.  Two items a CU, and as
// few as this takes: a prompt of 2,000 tokens, 8 heads of 128, 92 and 57 us; a
// chunk of 64 over 30,000 positions 153 and 100; eight of 64 over 1,000 45 and 30.
__device__ __forceinline__ int32_t many_cut(const Chunk &c, int32_t tiles, int64_t w, CutSums *s)
{
    const int32_t cus = c.many_slots / 2, slots = c.head_dim == 64 ? 3 * cus : 2 * cus;
    auto all_of = [&](int32_t i, int32_t &rows) {
        int32_t q, row0;
        wide_tile(c, i, q, row0);
        const ChunkSeq sq = c.seq[q];
        rows = min(sq.n * c.group - row0, kManyRows);
        return max(1, span_of(c, sq, row0, kManyRows).all);
    };
    return choose_cut(c, s, tiles, w, max(1, cus / 2), kManyCut, all_of, [&](int64_t items, int64_t longest, int64_t parts, int32_t rows) {
        const int64_t join = parts > 1 ? 8 + 4 * (8 + parts) * rows / kManyRows : 0;                              // in quarter tiles
        return join + (items <= cus ? 3 * longest : items <= slots ? 4 * longest : 4 * (w + 4 * items) / slots + 2 * longest);
    });
}

// Rows of a sequence whose `all` key tiles are cut into `parts` items, the
// first of which is number `first` of those that are laid out together.
struct Cut {
    int32_t first, seq, row0, all, parts, part, count;
};
// Item i of those that the workgroup's threads have cut; n > 0 items in all.
__device__ __forceinline__ const Cut &cut_of(const Cut *cuts, int32_t i)
{
    int32_t lo = 0, hi = kPlan;                 // the last that starts at or before i: it has parts
    while (hi - lo > 1) {
        const int32_t mid = (lo + hi) >> 1;
        if (cuts[mid].first <= i) lo = mid;
        else hi = mid;
    }
    return cuts[lo];
}

// Lays out the attention's work, in one workgroup.  A tile of rows whose key
// tiles are many for the chip's idle workgroups is cut along them into equal
// items; with enough tiles for all workgroups nothing is cut.  Later rows
// come first: under a causal limit they see most, and the workgroups that
// start last should have the least to do.
__global__ __launch_bounds__(kPlan) void k_chunk_work(Chunk c)
{
    __shared__ int64_t s_sum[kPlan / 64];
    __shared__ int32_t s_scan[kPlan / 64];
    __shared__ Cut s_cut[kPlan];
    __shared__ CutSums s_cuts;
    const int tid = threadIdx.x;
    for (int64_t i = tid; i < c.count_cap; i += kPlan) c.count[i] = 0;
    int32_t tiles = 0, weigh = 0;
    int64_t w_few = 0, w_many = 0, cost = 0, tokens = 0;
    int bad = 0;
    for (int32_t s0 = 0; s0 < c.n_seqs; s0 += kPlan) {
        const int32_t s = s0 + tid;
        int32_t wide = 0, held = 0;
        int64_t costs = 0;
        if (s < c.n_seqs) {
            const ChunkSeq q = c.seq[s];
            tokens += q.n;
            bad |= q.bad;
            held = c.weigh_few ? (q.L + kKeys - 1) / kKeys : (q.L + kWeighKeys - 1) / kWeighKeys;
            if (!c.weigh_few) costs = weigh_cost(c, q, held);
            const int32_t rows = q.n * c.group;
            if (rows > c.few_rows) wide = (rows + kManyRows - 1) / kManyRows;
            else if (rows > 0) w_few += span_of(c, q, 0, kFewRows).all;
        }
        int32_t total;
        const int32_t at = plan_scan(wide, s_scan, total);
        if (s < c.n_seqs) c.tile_off[s] = tiles + at;
        tiles += total;
        const int32_t wat = plan_scan(held, s_scan, total);
        if (s < c.n_seqs) c.weigh_off[s] = weigh + wat;
        weigh += total;
        int64_t sum;
        const int64_t cat = plan_scan(costs, s_sum, sum);
        if (s < c.n_seqs) c.cost_off[s] = cost + cat;
        cost += sum;
    }
    // Offsets that fall can leave sequences that overlap: they were reported, and
    // as their work is not bounded by the tokens there are, none is done.
    if (__syncthreads_or(bad) && plan_sum(tokens, s_sum) > c.n_tokens) {
        for (int32_t s = tid; s < c.n_seqs; s += kPlan) {
            c.seq[s] = {0, 0, 0, 0};
            c.tile_off[s] = c.weigh_off[s] = 0;
            c.cost_off[s] = 0;
        }
        for (int64_t t = tid; t < c.n_tokens; t += kPlan) {
            c.slot[t] = ~0ull;
            c.tok[t] = ~0u;
        }
        tiles = weigh = 0;
        w_few = cost = 0;
        __syncthreads();
    }
    if (!c.weigh_few && tid == 0) {
        c.work->n_weigh = weigh;
        c.work->weigh_cost = cost;
    }
    if (c.weigh_few) {
        // every sequence's key tiles, in items of one size
        const int32_t cut = max(kWeighCut, (weigh + c.few_slots - 1) / c.few_slots);
        int32_t n_items = 0;
        for (int32_t s0 = 0; s0 < c.n_seqs; s0 += kPlan) {
            const int32_t s = s0 + tid;
            ChunkSeq q = {0, 0, 0, 0};
            if (s < c.n_seqs) q = c.seq[s];
            const int32_t all = (q.L + kKeys - 1) / kKeys, parts = (all + cut - 1) / cut;
            int32_t total;
            const int32_t first = plan_scan(parts, s_scan, total);
            s_cut[tid] = {first, s, 0, all, parts, -1, 0};
            __syncthreads();
            for (int32_t i = tid; i < total && n_items + i < c.few_cap; i += kPlan) {
                const Cut &x = cut_of(s_cut, i);
                c.few_weigh[n_items + i] = {c.seq[x.seq], x.seq, 0, (int32_t)((int64_t)x.all * (i - x.first) / x.parts),
                                            (int32_t)((int64_t)x.all * (i - x.first + 1) / x.parts), -1, 0, 0, 0};
            }
            __syncthreads();
            n_items += total;
        }
        if (tid == 0) c.work->n_weigh = (int32_t)min64(n_items, c.few_cap);
    }
    __syncthreads();
    for (int32_t f = tid; f < tiles; f += kPlan) {
        int32_t s, row0;
        wide_tile(c, f, s, row0);
        w_many += span_of(c, c.seq[s], row0, kManyRows).all;
    }
    w_few = plan_sum(w_few, s_sum) * c.kv_heads;
    w_many = plan_sum(w_many, s_sum) * c.kv_heads;
    const int32_t cut_few = few_cut(c, w_few, &s_cuts);
    const int32_t cut_many = many_cut(c, tiles, w_many, &s_cuts);

    int32_t part = 0, n_joins = 0;
    for (int kind = 0; kind < 2; ++kind) {
        const int32_t n = kind ? tiles : c.n_seqs, cut = kind ? cut_many : cut_few;
        const int32_t blocks = (kind ? kManyRows / kFewRows : 1) * c.kv_heads;   // of partial sums, per item
        WorkItem *items = kind ? c.many : c.few;
        const int64_t cap = kind ? c.many_cap : c.few_cap;
        int32_t n_items = 0;
        for (int32_t f0 = 0; f0 < n; f0 += kPlan) {
            const int32_t f = n - 1 - (f0 + tid);
            int32_t s = f, row0 = 0, parts = 0, all = 0;
            if (f >= 0) {
                if (kind) wide_tile(c, f, s, row0);
                const ChunkSeq q = c.seq[s];
                const int32_t rows = q.n * c.group;
                if (kind || (rows > 0 && rows <= c.few_rows)) {
                    all = span_of(c, q, row0, kind ? kManyRows : kFewRows).all;
                    parts = max(1, (all + cut - 1) / cut);
                }
            }
            int32_t total, got;
            int32_t at = part + plan_scan(parts > 1 ? parts * blocks : 0, s_scan, total);
            if (parts > 1 && at + parts * blocks > c.part_cap) parts = 1;        // (what is cut is bounded, so this does not happen)
            part += total;
            const int32_t j = n_joins + plan_scan((int32_t)(parts > 1), s_scan, got);
            n_joins += got;
            const int32_t first = plan_scan(parts, s_scan, got);
            s_cut[tid] = {first, s, row0, all, parts, at, j * c.kv_heads};
            __syncthreads();
            for (int32_t i = tid; i < got && n_items + i < cap; i += kPlan) {
                const Cut &x = cut_of(s_cut, i);
                const int32_t n = i - x.first;
                items[n_items + i] = {c.seq[x.seq], x.seq, x.row0, (int32_t)((int64_t)x.all * n / x.parts),
                                      (int32_t)((int64_t)x.all * (n + 1) / x.parts), x.parts > 1 ? x.part + n * blocks : -1,
                                      x.part, x.parts, x.count};
            }
            __syncthreads();
            n_items += got;
        }
        if (tid == 0) *(kind ? &c.work->n_many : &c.work->n_few) = (int32_t)min64(n_items, cap);
    }
}

hipError_t launch_chunk_plan(const Launch &L, const Chunk &c, const PlanArgs &a)
{
    const int64_t seqs = c.n_seqs > 0 ? c.n_seqs : 1;
    int64_t y = (c.cols + kBlock * 4 - 1) / (kBlock * 4), yt = (c.n_tokens / seqs + kBlock - 1) / kBlock;
    y = y > yt ? y : yt;
    y = y < 1 ? 1 : (y > 64 ? 64 : y);
    RO_LAUNCH(L, RO_K_CHUNK_PLAN, k_chunk_plan, dim3((unsigned)seqs, (unsigned)y), dim3(kBlock), 0, L.stream, c, a,
              L.ctl);
    if (hipError_t e = hipGetLastError()) return e;
    RO_LAUNCH(L, RO_K_CHUNK_PLAN, k_chunk_work, dim3(1), dim3(kPlan), 0, L.stream, c);
    return hipGetLastError();
}

}  // namespace ro
