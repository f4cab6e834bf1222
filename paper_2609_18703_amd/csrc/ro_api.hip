// Host side of the C ABI: contexts, workspace, argument checks, launches.
#include <stdlib.h>
#include <string.h>

#include <vector>

#include "ro_chunk.h"
#include "ro_internal.h"
#include "ro_testing.h"

using namespace ro;

namespace ro {

// Events bracketing every traced launch; recycled after each read.
struct Tracer {
    struct Rec {
        int kind;
        hipEvent_t e0, e1;
    };
    bool on = false;
    std::vector<hipEvent_t> pool;   // all events ever created
    size_t used = 0;                // events handed out since the last read
    std::vector<Rec> recs;
    hipEvent_t next_event()
    {
        if (used == pool.size()) {
            hipEvent_t e = nullptr;
            if (hipEventCreate(&e) != hipSuccess) return nullptr;
            pool.push_back(e);
        }
        return pool[used++];
    }
};

void trace_begin(const Launch &L, int kernel)
{
    Tracer *t = L.tracer;
    if (!t || !t->on) return;
    hipEvent_t e = t->next_event();
    if (e && hipEventRecord(e, L.stream) != hipSuccess) e = nullptr;
    t->recs.push_back({kernel, e, nullptr});
}

void trace_end(const Launch &L, int kernel)
{
    (void)kernel;
    Tracer *t = L.tracer;
    if (!t || !t->on || t->recs.empty()) return;
    hipEvent_t e = t->next_event();
    if (e && hipEventRecord(e, L.stream) != hipSuccess) e = nullptr;
    t->recs.back().e1 = e;
}

}  // namespace ro

struct ro_ctx {
    hipStream_t stream;
    int device;
    int num_cus;
    Ctl *ctl;
    uint64_t *desc;
    int64_t desc_cap;
    Canon *canon;
    int64_t canon_cap;
    int64_t *sub_base;
    int64_t sub_cap;
    uint32_t *cmap;           // coarse child -> parent map used by ro_batch
    int64_t cmap_cap;
    int32_t *cnt;             // [3 * cnt_cap] counters used when the caller passes none
    uint64_t *gkey;           // [cnt_cap] first group failure per parent (gather)
    int64_t cnt_cap;
    int64_t gathers;          // canonical epoch of the next gather (1..2^30-1)
    PbWs pb;                  // parent-bound reservation workspace
    int64_t pb_cap, pb_pcap;  // its queue entries and parents
    void *pb_block;
    Tracer *tracer;
};

struct ro_grains {
    ro_ctx *ctx;
    int64_t n;
    GrainTab tab;
    void *block;              // one device allocation for the table
    uint32_t *scratch;        // [4 * scratch_cap] per report of a commit call: (child, report) by bin; its child; contested reports
    int64_t scratch_cap;
};

struct ro_stream {
    ro_ctx *ctx;
    StreamState st;
    void *block;              // one device allocation for all stream state
};

struct ro_chunk {
    ro_ctx *ctx;
    Chunk tab;                // the planned chunk's view of the block
    int64_t max_seqs, max_tokens, max_pages;
    int64_t n_pages;          // pages of the planned caches
    int32_t page_size;
    bool planned;
    void *block;              // one device allocation for the plan
};

namespace {

int hip_fail(hipError_t e) { return e == hipSuccess ? RO_OK : RO_EHIP; }

// The batch kernels read the queue, mask, offsets and barrier and write the
// tag arrays through restrict-qualified pointers: a tag array that shares
// memory with any of those, or with another tag array, is rejected.
bool batch_outputs_alias(const uint32_t *queue, const uint8_t *keep, int64_t q_len, const int64_t *offsets,
                         int64_t P, const uint8_t *barrier, uint32_t *const outs[3], int64_t out_cap,
                         const void *extra, int64_t extra_bytes)
{
    for (int i = 0; i < 3; ++i) {
        const int64_t nb = out_cap * 4;
        if (overlap(outs[i], nb, queue, q_len * 4) || overlap(outs[i], nb, keep, q_len) ||
            overlap(outs[i], nb, offsets, (P + 1) * 8) || overlap(outs[i], nb, barrier, P) ||
            overlap(outs[i], nb, extra, extra_bytes))
            return true;
        for (int j = i + 1; j < 3; ++j)
            if (overlap(outs[i], nb, outs[j], nb)) return true;
    }
    return false;
}

Launch launch_of(ro_ctx *c)
{
    Launch L;
    L.stream = c->stream;
    L.num_cus = c->num_cus;
    L.ctl = c->ctl;
    L.desc = c->desc;
    L.desc_cap = c->desc_cap;
    L.tracer = c->tracer;
    return L;
}

// A refused allocation is reported by the call that needed it, and not left
// for the next one to find, which may be another library's.
hipError_t dev_block(void **p, size_t bytes)
{
    const hipError_t e = hipMalloc(p, bytes);
    if (e != hipSuccess) (void)hipGetLastError();
    return e;
}

template <typename T>
hipError_t dev_alloc(T **p, int64_t n)
{
    *p = nullptr;
    if (n <= 0) n = 1;
    return dev_block(reinterpret_cast<void **>(p), (size_t)n * sizeof(T));
}

int64_t tiles_for(int64_t n) { return (n + kTile - 1) / kTile + 1; }
// look-back tiles at the smallest tile, 1,024 entries
int64_t scan_tiles_for(int64_t n) { return (n + 4 * kBlock - 1) / (4 * kBlock) + 1; }

// Make sure the look-back descriptors cover `tiles` tiles.
int ensure_desc(ro_ctx *c, int64_t tiles)
{
    if (tiles <= c->desc_cap) return RO_OK;
    if (hipStreamSynchronize(c->stream) != hipSuccess) return RO_EHIP;
    (void)hipFree(c->desc);
    c->desc = nullptr;
    c->desc_cap = 0;
    if (dev_alloc(&c->desc, tiles) != hipSuccess) return RO_EHIP;
    // zeroed on the context's stream: ordered before every later kernel on it
    if (launch_zero_u64(launch_of(c), c->desc, tiles) != hipSuccess) return RO_EHIP;
    c->desc_cap = tiles;
    return RO_OK;
}

int ensure_canon(ro_ctx *c, int64_t children)
{
    if (children <= c->canon_cap && c->canon) return RO_OK;
    if (hipStreamSynchronize(c->stream) != hipSuccess) return RO_EHIP;
    (void)hipFree(c->canon);
    (void)hipFree(c->sub_base);
    (void)hipFree(c->cmap);
    c->canon = nullptr;
    c->sub_base = nullptr;
    c->cmap = nullptr;
    c->canon_cap = 0;
    c->sub_cap = 0;
    c->cmap_cap = 0;
    const int64_t n = children > 0 ? children : 1;
    const int64_t subs = (n / kTile + 2) * (kTile / kGrp);
    const int64_t maps = (n >> 3) + 4;          // coarse map: 8 bytes per 16 to 128 children
    if (dev_alloc(&c->canon, n) != hipSuccess || dev_alloc(&c->sub_base, subs) != hipSuccess ||
        dev_alloc(&c->cmap, maps) != hipSuccess ||
        launch_zero_u64(launch_of(c), reinterpret_cast<uint64_t *>(c->canon),
                        n * (int64_t)(sizeof(Canon) / sizeof(uint64_t))) != hipSuccess) {
        // leave no partial workspace behind: the next call starts from none
        (void)hipStreamSynchronize(c->stream);
        (void)hipFree(c->canon);
        (void)hipFree(c->sub_base);
        (void)hipFree(c->cmap);
        c->canon = nullptr;
        c->sub_base = nullptr;
        c->cmap = nullptr;
        return RO_EHIP;
    }
    c->canon_cap = n;
    c->sub_cap = subs;
    c->cmap_cap = maps;
    return ensure_desc(c, scan_tiles_for(n));
}

int ensure_cnt(ro_ctx *c, int64_t parents)
{
    if (parents <= c->cnt_cap && c->cnt) return RO_OK;
    if (hipStreamSynchronize(c->stream) != hipSuccess) return RO_EHIP;
    (void)hipFree(c->cnt);
    (void)hipFree(c->gkey);
    c->cnt = nullptr;
    c->gkey = nullptr;
    c->cnt_cap = 0;
    const int64_t n = parents > 0 ? parents : 1;
    if (dev_alloc(&c->cnt, 3 * n) != hipSuccess || dev_alloc(&c->gkey, n) != hipSuccess ||
        launch_zero_u64(launch_of(c), c->gkey, n) != hipSuccess) {
        (void)hipStreamSynchronize(c->stream);
        (void)hipFree(c->cnt);
        (void)hipFree(c->gkey);
        c->cnt = nullptr;
        c->gkey = nullptr;
        return RO_EHIP;
    }
    c->cnt_cap = n;
    return RO_OK;
}

// Parent-bound reservation workspace for q queue entries and p parents (one
// allocation, 256-byte aligned arrays).
int ensure_pb(ro_ctx *c, int64_t q, int64_t p)
{
    if (q <= c->pb_cap && p <= c->pb_pcap && c->pb_block) return RO_OK;
    q = q > c->pb_cap ? q : c->pb_cap;
    p = p > c->pb_pcap ? p : c->pb_pcap;
    const int64_t qn = q > 0 ? q : 1, pn = p > 0 ? p : 1;
    const int64_t tiles = (qn + kPbTile * kPbSpan - 1) / (kPbTile * kPbSpan);   // histogram columns
    const size_t sizes[] = {
        (size_t)qn * 4, (size_t)qn * 4, (size_t)qn * 4, (size_t)qn * 8, (size_t)qn * 8,   // kc, k0, k1, v0, v1
        (size_t)qn * 4, (size_t)qn * 4,                                                    // fsize, gslot
        (size_t)pn * 4, (size_t)pn * 4,                                                    // pstart, pend
        (size_t)(kPbMaxBuckets * tiles) * 4, (size_t)(kPbMaxBuckets * tiles + 1) * 8,      // hist, hoff
        (size_t)2 * 8,                                                                     // m
        (size_t)((qn >> 4) + 1) * 16,                                                      // fmark, read 16 bytes at a time
    };
    constexpr int kArrays = (int)(sizeof(sizes) / sizeof(sizes[0]));
    size_t offs[kArrays], total = 0;
    for (int i = 0; i < kArrays; ++i) {
        offs[i] = total;
        total += (sizes[i] + 255) & ~(size_t)255;
    }
    if (hipStreamSynchronize(c->stream) != hipSuccess) return RO_EHIP;
    (void)hipFree(c->pb_block);
    c->pb_block = nullptr;
    c->pb_cap = c->pb_pcap = 0;
    char *b = nullptr;
    if (dev_block((void **)&b, total) != hipSuccess) return RO_EHIP;
    c->pb_block = b;
    c->pb.kc = (uint32_t *)(b + offs[0]);
    c->pb.k[0] = (uint32_t *)(b + offs[1]);
    c->pb.k[1] = (uint32_t *)(b + offs[2]);
    c->pb.v[0] = (uint64_t *)(b + offs[3]);
    c->pb.v[1] = (uint64_t *)(b + offs[4]);
    c->pb.fsize = (uint32_t *)(b + offs[5]);
    c->pb.gslot = (uint32_t *)(b + offs[6]);
    c->pb.pstart = (uint32_t *)(b + offs[7]);
    c->pb.pend = (uint32_t *)(b + offs[8]);
    c->pb.hist = (int32_t *)(b + offs[9]);
    c->pb.hoff = (int64_t *)(b + offs[10]);
    c->pb.m = (int64_t *)(b + offs[11]);
    c->pb.fmark = (uint8_t *)(b + offs[12]);
    c->pb_cap = q;
    c->pb_pcap = p;
    // descriptors: the compaction, the histogram scan and the two-chain group scan
    int64_t need = tiles_for(q);
    need = need > tiles_for(kPbMaxBuckets * tiles) ? need : tiles_for(kPbMaxBuckets * tiles);
    need = need > 2 * tiles_for(q) ? need : 2 * tiles_for(q);
    return ensure_desc(c, need);
}

int before_gather(ro_ctx *c)
{
    if (c->gathers + 1 > (int64_t)kMaxCanonEpoch) {
        if (launch_clear_tags(launch_of(c), c->canon, c->canon_cap) != hipSuccess) return RO_EHIP;
        // group-failure keys carry the same epoch
        if (c->gkey && launch_zero_u64(launch_of(c), c->gkey, c->cnt_cap) != hipSuccess) return RO_EHIP;
        c->gathers = 1;
    }
    c->gathers += 1;
    return RO_OK;
}

// Rows of n tokens x heads x D 16-bit elements that a kernel may read or write.
bool rows_ok(const ro_rows *r)
{
    return r && r->data && r->row_stride >= 0 && r->head_stride >= 0 && ((uintptr_t)r->data & 1) == 0;
}

// ... 16 bytes at a time
bool rows_wide(const ro_rows *r)
{
    return rows_ok(r) && ((uintptr_t)r->data & 15) == 0 && r->row_stride % 8 == 0 && r->head_stride % 8 == 0 &&
           r->row_stride <= INT32_MAX && r->head_stride <= INT32_MAX;
}

int64_t rows_bytes(const ro_rows *r, int64_t n, int64_t heads, int64_t D)
{
    return n <= 0 ? 0 : 2 * ((n - 1) * r->row_stride + (heads - 1) * r->head_stride + D);
}

// Outputs may not be broadcast, nor may their tokens or heads lie inside one another.
bool rows_apart(const ro_rows *r, int64_t n, int64_t heads, int64_t D)
{
    const int64_t a = r->row_stride, b = r->head_stride;
    if (n <= 1 && heads <= 1) return true;
    if (n <= 1) return b >= D;
    if (heads <= 1) return a >= D;
    return (b >= D && a >= (heads - 1) * b + D) || (a >= D && b >= (n - 1) * a + D);
}

// `out` may be `in` itself, element for element, but no other range that overlaps it.
bool rows_clash(const ro_rows *in, const ro_rows *out, int64_t n, int64_t heads, int64_t D, int64_t out_heads = 0)
{
    const bool other = out_heads > 0;             // rows of another operand, with heads of its own: no element in common
    if (!other) out_heads = heads;
    if (!other && in->data == out->data && in->row_stride == out->row_stride && in->head_stride == out->head_stride) return false;
    // interleaved parts of one tensor (a fused projection) overlap as ranges
    // without sharing an element: same row stride, and apart within a row
    if (in->row_stride == out->row_stride && in->row_stride > 0) {
        const int64_t row = 2 * in->row_stride;
        int64_t d = ((const char *)out->data - (const char *)in->data) % row;
        if (d < 0) d += row;
        const int64_t wi = 2 * ((heads - 1) * in->head_stride + D), wo = 2 * ((out_heads - 1) * out->head_stride + D);
        if (d >= wi && d + wo <= row) return false;
    }
    return overlap(in->data, rows_bytes(in, n, heads, D), out->data, rows_bytes(out, n, out_heads, D));
}

bool rotary_ok(const ro_rotary *r, const int32_t *pos, int64_t pos_stride, int64_t n, int32_t D)
{
    if (!r || !r->inv_freq || !r->axis || (n > 0 && !pos) || r->rot_dim < 2 || r->rot_dim > RO_MAX_ROT ||
        (r->rot_dim & 1) || r->rot_dim > D || r->n_axes < 1 || r->n_axes > RO_MAX_AXES ||
        (r->n_axes > 1 && pos_stride < n) || (r->adjacent != 0 && r->adjacent != 1))
        return false;
    for (int i = 0; i < r->rot_dim / 2; ++i)
        if (r->axis[i] >= r->n_axes) return false;
    return true;
}

RotaryArgs rotary_of(const ro_rotary *r, const int32_t *pos, int64_t pos_stride)
{
    RotaryArgs a{};
    a.freq = r->inv_freq;
    a.pos = pos;
    a.pos_stride = pos_stride;
    a.rot = r->rot_dim;
    a.adjacent = r->adjacent;
    memcpy(a.axis, r->axis, (size_t)r->rot_dim / 2);
    return a;
}

Rows rows_of(const ro_rows *r) { return r ? Rows{r->data, r->row_stride, r->head_stride} : Rows{nullptr, 0, 0}; }

bool dtype_ok(int32_t d) { return d == RO_BF16 || d == RO_F16; }

bool cache_ok(const ro_cache *k)
{
    return k && k->n_pages >= 0 && k->n_pages < ((int64_t)1 << 32) && (k->n_pages == 0 || (k->k && k->v)) &&
           k->page_size >= 16 && k->page_size <= 65536 && (k->page_size & (k->page_size - 1)) == 0 && k->n_heads >= 1 &&
           (k->head_dim == 64 || k->head_dim == 128) && dtype_ok(k->dtype) && k->page_stride >= 0 && k->head_stride >= 0 &&
           k->slot_stride >= 0 && (k->page_stride | k->head_stride | k->slot_stride) % 8 == 0 &&
           k->slot_stride <= (1 << 26) &&
           (((uintptr_t)k->k | (uintptr_t)k->v) & 15) == 0;
}

Pages pages_of(const ro_cache *k) { return Pages{k->k, k->v, k->page_stride, k->head_stride, k->slot_stride}; }

// Bytes of keys and values that all sequences together can have cached, from
// which on short sequences beside longer ones are narrow tiles: in a launch of
// their own their caches are read up to 8% faster, but nothing else runs
// beside it.  (Narrow, and wide: 31 tokens beside a chunk of 100, 1,000
// positions each, 46 and 31 us; 8,000 each, 196 and 209; 32,000 each, 687 and
// 744.  60 tokens with 16,000 beside a chunk of 1,000: 155 and 103.)
constexpr int64_t kNarrowBytes = (int64_t)1 << 30;

// A planned chunk of this context, and a cache paged as the plan's was.
bool chunk_ok(const ro_ctx *c, const ro_chunk *h, const ro_cache *k)
{
    return c && h && h->ctx == c && h->planned && cache_ok(k) && k->page_size == h->page_size &&
           k->n_pages >= h->n_pages && k->n_heads == h->tab.kv_heads && k->head_dim == h->tab.head_dim;
}

}  // namespace

extern "C" {

int ro_ctx_create(ro_ctx **out, void *hip_stream)
{
    if (out == nullptr) return RO_EINVAL;
    *out = nullptr;
    ro_ctx *c = (ro_ctx *)calloc(1, sizeof(ro_ctx));
    if (!c) return RO_EINVAL;
    c->tracer = new Tracer();
    c->stream = (hipStream_t)hip_stream;
    if (hipGetDevice(&c->device) != hipSuccess ||
        hipDeviceGetAttribute(&c->num_cus, hipDeviceAttributeMultiprocessorCount, c->device) != hipSuccess ||
        dev_alloc(&c->ctl, 1) != hipSuccess) {
        ro_ctx_destroy(c);
        return RO_EHIP;
    }
    if (c->num_cus <= 0) c->num_cus = 1;
    if (hipMemset(c->ctl, 0, sizeof(Ctl)) != hipSuccess ||
        launch_ctl_init(launch_of(c)) != hipSuccess || hipDeviceSynchronize() != hipSuccess ||
        ensure_desc(c, 64) != RO_OK) {
        ro_ctx_destroy(c);
        return RO_EHIP;
    }
    c->gathers = 1;           // the first gather runs at canonical epoch 1
    *out = c;
    return RO_OK;
}

int ro_ctx_set_stream(ro_ctx *c, void *hip_stream)
{
    if (!c) return RO_EINVAL;
    if (hipStreamSynchronize(c->stream) != hipSuccess) return RO_EHIP;
    c->stream = (hipStream_t)hip_stream;
    return RO_OK;
}

int ro_ctx_reserve(ro_ctx *c, int64_t max_children, int64_t max_parents, int64_t max_queue)
{
    if (!c || max_children < 0 || max_parents < 0 || max_queue < 0) return RO_EINVAL;
    int rc = ensure_canon(c, max_children);
    if (rc) return rc;
    rc = ensure_cnt(c, max_parents);
    if (rc) return rc;
    int64_t m = max_children > max_parents ? max_children : max_parents;
    m = m > max_queue ? m : max_queue;
    return ensure_desc(c, scan_tiles_for(m));
}

int ro_ctx_status(ro_ctx *c)
{
    if (!c) return RO_EINVAL;
    if (hipStreamSynchronize(c->stream) != hipSuccess) return RO_EHIP;
    int32_t err = 0;
    if (hipMemcpy(&err, &c->ctl->err, sizeof(err), hipMemcpyDeviceToHost) != hipSuccess) return RO_EHIP;
    // cleared by a kernel on the context's stream, so that no later kernel of
    // the context can see the old error (a host-to-device copy may still be
    // in flight when it returns)
    if (err != 0 && launch_clear_err(launch_of(c)) != hipSuccess) return RO_EHIP;
    return err;
}

int ro_ctx_destroy(ro_ctx *c)
{
    if (!c) return RO_EINVAL;
    if (c->stream || c->ctl) (void)hipStreamSynchronize(c->stream);
    (void)hipFree(c->ctl);
    (void)hipFree(c->desc);
    (void)hipFree(c->canon);
    (void)hipFree(c->sub_base);
    (void)hipFree(c->cmap);
    (void)hipFree(c->cnt);
    (void)hipFree(c->gkey);
    (void)hipFree(c->pb_block);
    if (c->tracer) {
        for (hipEvent_t e : c->tracer->pool) (void)hipEventDestroy(e);
        delete c->tracer;
    }
    free(c);
    return RO_OK;
}

int ro_ctx_trace(ro_ctx *c, int enable)
{
    if (!c || !c->tracer) return RO_EINVAL;
    c->tracer->on = enable != 0;
    return RO_OK;
}

int ro_ctx_trace_read(ro_ctx *c, int64_t *launches, double *total_ms, int32_t n)
{
    if (!c || !c->tracer || n < 0 || (n > 0 && (!launches || !total_ms))) return RO_EINVAL;
    Tracer *t = c->tracer;
    if (hipStreamSynchronize(c->stream) != hipSuccess) return RO_EHIP;
    for (const Tracer::Rec &r : t->recs) {
        if (r.kind < 0 || r.kind >= n || !r.e0 || !r.e1) continue;
        float ms = 0.f;
        if (hipEventElapsedTime(&ms, r.e0, r.e1) != hipSuccess) continue;
        launches[r.kind] += 1;
        total_ms[r.kind] += (double)ms;
    }
    t->recs.clear();
    t->used = 0;
    return RO_OK;
}

int ro_expand(ro_ctx *c, const int32_t *counts, int64_t n_parents, int64_t *offsets,
              uint32_t *child_parent, uint32_t *child_ordinal, int64_t child_cap)
{
    if (!c || !offsets || n_parents < 0 || child_cap < 0 || (n_parents > 0 && !counts)) return RO_EINVAL;
    int rc = ensure_desc(c, tiles_for(n_parents));
    if (rc) return rc;
    return hip_fail(launch_expand(launch_of(c), counts, n_parents, offsets, child_parent, child_ordinal,
                                  child_cap));
}

int ro_batch(ro_ctx *c, const uint32_t *queue, const uint8_t *keep, int64_t q_len,
             const int64_t *offsets, int64_t n_parents, int32_t batch_size,
             uint32_t *out_child, uint32_t *out_parent, uint32_t *out_ordinal, int64_t out_cap,
             int64_t *n_out_dev, int64_t *n_batches_dev, const uint8_t *barrier)
{
    if (!c || !offsets || q_len < 0 || n_parents < 0 || batch_size <= 0 || out_cap < 0 ||
        (q_len > 0 && !queue))
        return RO_EINVAL;
    uint32_t *const outs[3] = {out_child, out_parent, out_ordinal};
    if (batch_outputs_alias(queue, keep, q_len, offsets, n_parents, barrier, outs, out_cap, nullptr, 0))
        return RO_EINVAL;
    int rc = ensure_desc(c, scan_tiles_for(q_len));
    if (rc) return rc;
    return hip_fail(launch_batch(launch_of(c), queue, keep, q_len, offsets, n_parents, batch_size,
                                 out_child, out_parent, out_ordinal, out_cap, n_out_dev, n_batches_dev,
                                 c->cmap, c->cmap_cap, barrier));
}

int ro_batch_parent(ro_ctx *c, const uint32_t *queue, const uint8_t *keep, int64_t q_len,
                    const int64_t *offsets, int64_t n_parents, int32_t batch_size, uint32_t *out_child,
                    uint32_t *out_parent, uint32_t *out_ordinal, int64_t out_cap, int64_t *batch_off,
                    int64_t batch_cap, int64_t *n_out_dev, int64_t *n_batches_dev, const uint8_t *barrier)
{
    if (!c || !offsets || q_len < 0 || n_parents < 0 || batch_size <= 0 || out_cap < 0 || !batch_off ||
        batch_cap < 1 || (q_len > 0 && !queue))
        return RO_EINVAL;
    if (q_len >= ((int64_t)1 << 32) || n_parents >= ((int64_t)1 << 32)) return RO_EINVAL;
    uint32_t *const outs[3] = {out_child, out_parent, out_ordinal};
    if (batch_outputs_alias(queue, keep, q_len, offsets, n_parents, barrier, outs, out_cap, batch_off,
                            batch_cap * 8) ||
        overlap(batch_off, batch_cap * 8, queue, q_len * 4) || overlap(batch_off, batch_cap * 8, keep, q_len) ||
        overlap(batch_off, batch_cap * 8, offsets, (n_parents + 1) * 8) ||
        overlap(batch_off, batch_cap * 8, barrier, n_parents))
        return RO_EINVAL;
    int rc = ensure_pb(c, q_len, n_parents);
    if (rc) return rc;
    rc = ensure_desc(c, scan_tiles_for(q_len));
    if (rc) return rc;
    return hip_fail(launch_batch_parent(launch_of(c), queue, keep, q_len, offsets, n_parents, batch_size,
                                        out_child, out_parent, out_ordinal, out_cap, batch_off, batch_cap,
                                        n_out_dev, n_batches_dev, c->cmap, c->cmap_cap, barrier, c->pb));
}

int ro_gather(ro_ctx *c, const ro_reports *r, const int64_t *offsets, int64_t n_parents,
              const ro_gather_out *o)
{
    if (!c || !r || !o || !offsets || n_parents < 0 || r->n < 0 || !o->out_off || o->out_cap < 0)
        return RO_EINVAL;
    if (r->n > 0 && (!r->parent || !r->ordinal || !r->state || !r->off)) return RO_EINVAL;
    if (o->out_data != nullptr && r->n > 0 && !r->data) return RO_EINVAL;
    if (o->barrier != nullptr && r->n >= ((int64_t)1 << 32)) return RO_EINVAL;   // report index is 32-bit
    // the canonical workspace must cover the expansion; its size is on the
    // device, so the report count is the host's best lower bound
    int rc = ensure_canon(c, c->canon_cap > r->n ? c->canon_cap : r->n);
    if (rc) return rc;
    rc = ensure_desc(c, scan_tiles_for(c->canon_cap));
    if (rc) return rc;
    GatherArgs a;
    a.rp = r->parent;
    a.ro = r->ordinal;
    a.rs = r->state;
    a.roff = r->off;
    a.data = r->data;
    a.n = r->n;
    a.offsets = offsets;
    a.P = n_parents;
    a.out_off = o->out_off;
    a.out_data = o->out_data;
    a.out_cap = o->out_cap;
    a.ns = o->n_success;
    a.nf = o->n_failed;
    a.nk = o->n_skipped;
    a.complete = o->complete;
    a.pstate = o->parent_state;
    a.cdst = o->child_dst_off;
    a.barrier = o->barrier;
    a.n_rejected = o->n_rejected;
    if (a.barrier && (rc = ensure_cnt(c, n_parents))) return rc;
    if (!a.ns || !a.nf || !a.nk) {
        if ((rc = ensure_cnt(c, n_parents))) return rc;
        if (!a.ns) a.ns = c->cnt;
        if (!a.nf) a.nf = c->cnt + c->cnt_cap;
        if (!a.nk) a.nk = c->cnt + 2 * c->cnt_cap;
    }
    GatherWs w;
    w.canon = c->canon;
    w.canon_cap = c->canon_cap;
    w.sub_base = c->sub_base;
    w.sub_cap = c->sub_cap;
    w.gkey = c->gkey;
    if ((rc = before_gather(c))) return rc;
    return hip_fail(launch_gather(launch_of(c), a, w, (uint32_t)(c->gathers - 1)));
}

int ro_filter(ro_ctx *c, const uint8_t *x_state, const uint8_t *mask_state, const uint8_t *mask, int64_t n,
              uint8_t *out_state)
{
    if (!c || n < 0 || (n > 0 && (!x_state || !mask || !out_state))) return RO_EINVAL;
    if (n == 0) return RO_OK;
    return hip_fail(launch_filter(launch_of(c), x_state, mask_state, mask, n, out_state));
}

int ro_broadcast(ro_ctx *c, const uint32_t *const *maps, const int64_t *map_len, int32_t levels, int64_t n,
                 const uint8_t *x_state, int64_t n_ancestors, const uint8_t *like_state, uint32_t *out_ancestor,
                 uint8_t *out_state)
{
    if (!c || n < 0 || n_ancestors < 0 || levels < 1 || levels > kMaxBroadcastLevels) return RO_EINVAL;
    if (n > 0 && (!maps || !map_len || !x_state || !out_state)) return RO_EINVAL;
    for (int32_t l = 0; n > 0 && l < levels; ++l)
        if (!maps[l] || map_len[l] < 0) return RO_EINVAL;
    if (n == 0) return RO_OK;
    if (map_len[0] < n) return RO_EINVAL;
    return hip_fail(launch_broadcast(launch_of(c), maps, map_len, levels, n, x_state, n_ancestors, like_state,
                                     out_ancestor, out_state));
}

int ro_grains_create(ro_ctx *c, int64_t n_children, ro_grains **out)
{
    if (out) *out = nullptr;
    if (!c || !out || n_children < 0 || n_children >= ((int64_t)1 << 32)) return RO_EINVAL;
    const int64_t n = n_children > 0 ? n_children : 1, w = grain_words(n), n4 = (n + 3) & ~(int64_t)3;
    ro_grains *g = (ro_grains *)calloc(1, sizeof(ro_grains));
    if (!g) return RO_EINVAL;
    uint32_t *b = nullptr;
    if (dev_alloc(&b, 5 * w + 2 * kGrainBins + 64 + 3 * n4) != hipSuccess) {
        free(g);
        return RO_EHIP;
    }
    g->ctx = c;
    g->n = n_children;
    g->block = b;
    g->tab.bits = reinterpret_cast<GrainBits *>(b);
    g->tab.contested = b + 4 * w;
    g->tab.hist = b + 5 * w;
    g->tab.cursor = g->tab.hist + kGrainBins;
    g->tab.n_list = g->tab.cursor + kGrainBins;
    g->tab.first = g->tab.n_list + 64;
    g->tab.gen = g->tab.first + n4;
    g->tab.room = g->tab.gen + n4;
    if (launch_grains_fill(launch_of(c), g->tab, n) != hipSuccess) {
        (void)hipFree(b);
        free(g);
        return RO_EHIP;
    }
    *out = g;
    return RO_OK;
}

int ro_grains_reset(ro_ctx *c, ro_grains *g)
{
    if (!c || !g || g->ctx != c) return RO_EINVAL;
    return hip_fail(launch_grains_fill(launch_of(c), g->tab, g->n > 0 ? g->n : 1));
}

int ro_grains_destroy(ro_grains *g)
{
    if (!g) return RO_EINVAL;
    if (g->ctx) (void)hipStreamSynchronize(g->ctx->stream);
    (void)hipFree(g->block);
    if (g->scratch) (void)hipFree(g->scratch);
    free(g);
    return RO_OK;
}

int ro_grains_read(ro_ctx *c, ro_grains *g, uint32_t *phase, uint32_t *generation)
{
    if (!c || !g || g->ctx != c) return RO_EINVAL;
    if (g->n == 0 || (!phase && !generation)) return RO_OK;
    return hip_fail(launch_grains_read(launch_of(c), g->tab, g->n, phase, generation));
}

int ro_grains_dispatch(ro_ctx *c, ro_grains *g, const uint32_t *child, int64_t n, uint32_t *out_generation)
{
    if (!c || !g || g->ctx != c || n < 0 || (n > 0 && !child)) return RO_EINVAL;
    if (n == 0) return RO_OK;
    return hip_fail(launch_grains_dispatch(launch_of(c), child, n, g->n, g->tab, out_generation));
}

int ro_grains_retry(ro_ctx *c, ro_grains *g, const uint32_t *child, int64_t n)
{
    if (!c || !g || g->ctx != c || n < 0 || (n > 0 && !child)) return RO_EINVAL;
    if (n == 0) return RO_OK;
    return hip_fail(launch_grains_retry(launch_of(c), child, n, g->n, g->tab));
}

int ro_grains_commit(ro_ctx *c, ro_grains *g, const ro_reports *r, const uint32_t *generation,
                     const int64_t *offsets, int64_t n_parents, uint8_t *state_out, int64_t *counts_dev)
{
    if (!c || !g || g->ctx != c || !r || !offsets || n_parents < 0 || r->n < 0) return RO_EINVAL;
    if (r->n >= ((int64_t)1 << 32)) return RO_EINVAL;                // report index is 32-bit
    if (r->n > 0 && (!r->parent || !r->ordinal || !r->state || !r->off || !generation || !state_out))
        return RO_EINVAL;
    const int64_t need = r->n > 0 ? r->n : 1;
    if (need > g->scratch_cap) {              // grows with the largest call
        const int64_t cap = need > 2 * g->scratch_cap ? need : 2 * g->scratch_cap;
        uint32_t *t = nullptr;
        if (dev_alloc(&t, 4 * cap) != hipSuccess) return RO_EHIP;
        if (g->scratch) {
            (void)hipStreamSynchronize(c->stream);
            (void)hipFree(g->scratch);
        }
        g->scratch = t;
        g->scratch_cap = cap;
    }
    return hip_fail(launch_grains_commit(launch_of(c), r->parent, r->ordinal, r->state, r->off, r->data, generation,
                                         r->n, offsets, n_parents, g->n, g->tab, g->scratch + 2 * g->scratch_cap,
                                         g->scratch + 3 * g->scratch_cap, reinterpret_cast<uint2 *>(g->scratch),
                                         state_out, counts_dev));
}

int ro_stream_create(ro_ctx *c, const int64_t *offsets, int64_t n_parents, int64_t n_children,
                     uint8_t *barrier, ro_stream **out)
{
    if (out) *out = nullptr;
    if (!c || !offsets || !out || n_parents < 0 || n_children < 0 || n_children >= ((int64_t)1 << 32))
        return RO_EINVAL;
    const int64_t P = n_parents, N = n_children;
    int rc = ensure_desc(c, stream_desc_tiles(P, N));
    if (rc) return rc;
    // one allocation, carved into 256-byte aligned arrays
    const size_t sizes[] = {
        (size_t)(N > 0 ? N : 1) * sizeof(Canon),            // canon
        (size_t)((N + 31) / 32 + 1) * sizeof(uint32_t),     // seen
        (size_t)stream_word_count(N) * sizeof(uint32_t),    // words
        (size_t)(P / 64 + 1) * sizeof(uint64_t),            // ready
        (size_t)(P + 1),                                    // emitted
        (size_t)(P + 1) * sizeof(int64_t),                  // ebase
        (size_t)(P + 2) * sizeof(int64_t),                  // evoff
        (size_t)(3 * (P + 1)) * sizeof(int32_t),            // ecnt
        (size_t)(N + 1) * sizeof(int64_t),                  // edst
        (size_t)(N + 1) * sizeof(uint64_t),                 // esrc
        (size_t)(P + 1) * sizeof(uint64_t),                 // gkey
        (size_t)(P + 1),                                    // ebar
        (size_t)(N > 0 ? N : 1) * sizeof(uint32_t),         // cpar
        (size_t)(P + 1) * sizeof(int64_t),                  // mapped
        3 * sizeof(uint32_t),                               // remap
    };
    constexpr int kArrays = (int)(sizeof(sizes) / sizeof(sizes[0]));
    size_t offs[kArrays], total = 0;
    for (int i = 0; i < kArrays; ++i) {
        offs[i] = total;
        total += (sizes[i] + 255) & ~(size_t)255;
    }
    ro_stream *s = (ro_stream *)calloc(1, sizeof(ro_stream));
    if (!s) return RO_EINVAL;
    char *block = nullptr;
    if (hipStreamSynchronize(c->stream) != hipSuccess || dev_block((void **)&block, total) != hipSuccess) {
        free(s);
        return RO_EHIP;
    }
    if (launch_zero_u64(launch_of(c), reinterpret_cast<uint64_t *>(block), (int64_t)(total / 8)) != hipSuccess) {
        (void)hipFree(block);
        free(s);
        return RO_EHIP;
    }
    s->ctx = c;
    s->block = block;
    StreamState &st = s->st;
    st.offsets = offsets;
    st.P = P;
    st.N = N;
    st.canon = (Canon *)(block + offs[0]);
    st.seen = (uint32_t *)(block + offs[1]);
    st.words = (uint32_t *)(block + offs[2]);
    st.ready = (uint64_t *)(block + offs[3]);
    st.emitted = (uint8_t *)(block + offs[4]);
    st.ebase = (int64_t *)(block + offs[5]);
    st.evoff = (int64_t *)(block + offs[6]);
    st.ecnt = (int32_t *)(block + offs[7]);
    st.edst = (int64_t *)(block + offs[8]);
    st.esrc = (uint64_t *)(block + offs[9]);
    st.gkey = (uint64_t *)(block + offs[10]);
    st.ebar = (uint8_t *)(block + offs[11]);
    st.cpar = (uint32_t *)(block + offs[12]);
    st.mapped = (int64_t *)(block + offs[13]);
    st.remap = (uint32_t *)(block + offs[14]);
    st.barrier = barrier;
    st.run_epoch = 1;
    st.gf_epoch = 0;
    if (launch_stream_init(launch_of(c), st) != hipSuccess) {
        (void)hipStreamSynchronize(c->stream);     // a launch that did start still uses the block
        (void)hipFree(block);
        free(s);
        return RO_EHIP;
    }
    *out = s;
    return RO_OK;
}

int ro_stream_batch(ro_ctx *c, ro_stream *s, const uint32_t *queue, const uint8_t *keep, int64_t q_len,
                    int32_t batch_size, uint32_t *out_child, uint32_t *out_parent, uint32_t *out_ordinal,
                    int64_t out_cap, int64_t *n_out_dev, int64_t *n_batches_dev)
{
    if (!c || !s || s->ctx != c || q_len < 0 || batch_size <= 0 || out_cap < 0 || (q_len > 0 && !queue))
        return RO_EINVAL;
    const StreamState &st = s->st;
    uint32_t *const outs[3] = {out_child, out_parent, out_ordinal};
    if (batch_outputs_alias(queue, keep, q_len, st.offsets, st.P, st.barrier, outs, out_cap, nullptr, 0))
        return RO_EINVAL;
    int rc = ensure_desc(c, scan_tiles_for(q_len));
    if (rc) return rc;
    return hip_fail(launch_batch(launch_of(c), queue, keep, q_len, st.offsets, st.P, batch_size, out_child,
                                 out_parent, out_ordinal, out_cap, n_out_dev, n_batches_dev, nullptr, 0, st.barrier,
                                 st.cpar, st.N));
}

int ro_stream_report(ro_ctx *c, ro_stream *s, const ro_reports *r, int64_t *n_rejected_dev)
{
    if (!c || !s || !r || s->ctx != c || r->n < 0) return RO_EINVAL;
    if (r->n > 0 && (!r->parent || !r->ordinal || !r->state || !r->off)) return RO_EINVAL;
    if (s->st.barrier != nullptr && r->n >= ((int64_t)1 << 32)) return RO_EINVAL;
    if (r->n == 0) return RO_OK;
    if (s->st.barrier != nullptr) {
        // a new epoch for this call's first group failures
        if (s->st.gf_epoch == 0xffffffffu) {
            if (launch_zero_u64(launch_of(c), s->st.gkey, s->st.P + 1) != hipSuccess) return RO_EHIP;
            s->st.gf_epoch = 0;
        }
        s->st.gf_epoch += 1;
    }
    return hip_fail(launch_stream_report(launch_of(c), s->st, r->parent, r->ordinal, r->state, r->off, r->data,
                                         r->n, n_rejected_dev));
}

int ro_stream_emit(ro_ctx *c, ro_stream *s, uint32_t *emit_parent, int64_t *emit_off,
                   uint8_t *emit_data, int64_t cap_parents, int64_t cap_bytes,
                   int32_t *n_success, int32_t *n_failed, int32_t *n_skipped,
                   uint8_t *parent_state, int64_t *n_emitted_dev, int64_t *n_bytes_dev)
{
    if (!c || !s || s->ctx != c || !emit_off || cap_parents < 0 || cap_bytes < 0) return RO_EINVAL;
    return hip_fail(launch_stream_emit(launch_of(c), s->st, emit_parent, emit_off, emit_data, cap_parents,
                                       cap_bytes, n_success, n_failed, n_skipped, parent_state, n_emitted_dev,
                                       n_bytes_dev));
}

int ro_stream_reset(ro_ctx *c, ro_stream *s)
{
    if (!c || !s || s->ctx != c) return RO_EINVAL;
    // a new slot epoch, so that the slots of the previous run read as unreported
    if (s->st.run_epoch + 1 > kMaxCanonEpoch) {
        if (launch_clear_tags(launch_of(c), s->st.canon, s->st.N) != hipSuccess) return RO_EHIP;
        s->st.run_epoch = 0;
    }
    s->st.run_epoch += 1;
    return hip_fail(launch_stream_reset(launch_of(c), s->st));
}

int ro_debug_epochs(ro_ctx *c, ro_stream *s, ro_grains *g, int64_t canon_left, int64_t run_left,
                    int64_t gf_left, int64_t fence_left)
{
    if (!c || (s && s->ctx != c) || (g && g->ctx != c)) return RO_EINVAL;
    if (canon_left >= 1 && canon_left < (int64_t)kMaxCanonEpoch) {
        // the next gather runs at epoch max - canon_left + 1
        const uint32_t e = (uint32_t)((int64_t)kMaxCanonEpoch - canon_left + 1);
        if (e > (uint32_t)c->gathers) c->gathers = e;
    }
    if (s) {
        if (run_left >= 1 && run_left < (int64_t)kMaxCanonEpoch &&
            (uint32_t)((int64_t)kMaxCanonEpoch - run_left) > s->st.run_epoch)
            s->st.run_epoch = (uint32_t)((int64_t)kMaxCanonEpoch - run_left);
        if (gf_left >= 1 && gf_left <= 0xffffffffll &&
            (uint32_t)(0xffffffffll - gf_left) > s->st.gf_epoch)
            s->st.gf_epoch = (uint32_t)(0xffffffffll - gf_left);
    }
    (void)fence_left;         // Grains carry no epoch
    return RO_OK;
}

int ro_stream_destroy(ro_stream *s)
{
    if (!s) return RO_EINVAL;
    if (s->ctx) (void)hipStreamSynchronize(s->ctx->stream);
    (void)hipFree(s->block);
    free(s);
    return RO_OK;
}

int ro_rope(ro_ctx *c, const ro_rotary *r, const int32_t *pos, int64_t pos_stride, const ro_rows *x,
            const ro_rows *y, int64_t n, int32_t heads, int32_t D, int32_t dtype, int32_t inverse)
{
    if (!c || n < 0 || heads < 0 || D < 1 || !dtype_ok(dtype) || (inverse != 0 && inverse != 1) ||
        !rotary_ok(r, pos, pos_stride, n, D))
        return RO_EINVAL;
    if (n == 0 || heads == 0) return RO_OK;
    // a workgroup counts the pieces of its tokens' heads in 32 bits
    if (n > INT32_MAX || (int64_t)heads * D > INT32_MAX / 8) return RO_EINVAL;
    if (!rows_ok(x) || !rows_ok(y) || !rows_apart(y, n, heads, D) || rows_clash(x, y, n, heads, D)) return RO_EINVAL;
    return hip_fail(launch_rope(launch_of(c), rotary_of(r, pos, pos_stride), rows_of(x), rows_of(y), n, heads, D, dtype,
                                inverse));
}

int ro_chunk_create(ro_ctx *c, int64_t max_seqs, int64_t max_tokens, int64_t max_pages, ro_chunk **out)
{
    if (out) *out = nullptr;
    if (!c || !out || max_seqs < 0 || max_tokens < 0 || max_pages < 0 || max_seqs >= ((int64_t)1 << 24) ||
        max_tokens >= ((int64_t)1 << 31) || max_pages >= ((int64_t)1 << 31))
        return RO_EINVAL;
    if (max_pages > 0 && max_seqs > ((int64_t)1 << 40) / max_pages) return RO_EINVAL;
    // Work is cut into items for the workgroups that run at once, two per CU;
    // where the rows are few into up to as many again.  Cut tiles are at most
    // twice as many items as that.
    const int64_t few_slots = 4 * (int64_t)c->num_cus, many_slots = 2 * (int64_t)c->num_cus;
    const int64_t few_cap = max_seqs + few_slots + 1;
    const int64_t many_cap = max_tokens * kMaxGroup / kManyRows + max_seqs + many_slots + 1;
    const int64_t count_cap = few_slots + many_slots;
    const int64_t part_cap = 2 * few_slots + 2 * many_slots * (kManyRows / kFewRows);
    const size_t sizes[] = {
        (size_t)(max_seqs > 0 ? max_seqs : 1) * sizeof(ChunkSeq),
        (size_t)(max_seqs * max_pages + 1) * sizeof(uint32_t),
        (size_t)(max_tokens + 1) * sizeof(uint64_t),
        (size_t)(max_tokens + 1) * sizeof(uint32_t),
        sizeof(WorkHead),
        (size_t)few_cap * sizeof(WorkItem),
        (size_t)few_cap * sizeof(WorkItem),
        (size_t)many_cap * sizeof(WorkItem),
        (size_t)count_cap * sizeof(uint32_t),
        (size_t)(max_seqs + 1) * sizeof(int32_t),
        (size_t)(max_seqs + 1) * sizeof(int32_t),
        (size_t)(max_seqs + 1) * sizeof(int64_t),
        (size_t)part_cap * kFewRows * 128 * sizeof(float),
        (size_t)part_cap * kFewRows * sizeof(float2),
    };
    constexpr int kArrays = (int)(sizeof(sizes) / sizeof(sizes[0]));
    size_t offs[kArrays], total = 0;
    for (int i = 0; i < kArrays; ++i) {
        offs[i] = total;
        total += (sizes[i] + 255) & ~(size_t)255;
    }
    ro_chunk *h = (ro_chunk *)calloc(1, sizeof(ro_chunk));
    if (!h) return RO_EINVAL;
    char *b = nullptr;
    if (dev_block((void **)&b, total) != hipSuccess) {
        free(h);
        return RO_EHIP;
    }
    h->ctx = c;
    h->block = b;
    h->max_seqs = max_seqs;
    h->max_tokens = max_tokens;
    h->max_pages = max_pages;
    h->tab.seq = (ChunkSeq *)(b + offs[0]);
    h->tab.table = (uint32_t *)(b + offs[1]);
    h->tab.slot = (uint64_t *)(b + offs[2]);
    h->tab.tok = (uint32_t *)(b + offs[3]);
    h->tab.work = (WorkHead *)(b + offs[4]);
    h->tab.few = (WorkItem *)(b + offs[5]);
    h->tab.few_weigh = (WorkItem *)(b + offs[6]);
    h->tab.many = (WorkItem *)(b + offs[7]);
    h->tab.count = (uint32_t *)(b + offs[8]);
    h->tab.tile_off = (int32_t *)(b + offs[9]);
    h->tab.weigh_off = (int32_t *)(b + offs[10]);
    h->tab.cost_off = (int64_t *)(b + offs[11]);
    h->tab.part_o = (float *)(b + offs[12]);
    h->tab.part_ml = (float2 *)(b + offs[13]);
    h->tab.count_cap = count_cap;
    h->tab.few_cap = few_cap;
    h->tab.many_cap = many_cap;
    h->tab.part_cap = part_cap;
    h->tab.few_slots = (int32_t)few_slots;
    h->tab.many_slots = (int32_t)many_slots;
    *out = h;
    return RO_OK;
}

int ro_chunk_plan(ro_ctx *c, ro_chunk *h, const ro_cache *k, const ro_chunk_args *a)
{
    if (!c || !h || h->ctx != c) return RO_EINVAL;
    h->planned = false;
    if (!a || !cache_ok(k) || a->n_seqs < 0 || a->n_tokens < 0 || a->max_new < 0 || a->table_stride < 0 ||
        a->q_heads < 1 || a->q_heads % k->n_heads != 0 || a->q_heads / k->n_heads > kMaxGroup ||
        (a->causal != 0 && a->causal != 1) || a->window < 0 || a->sinks < 0 || (a->window > 0 && !a->causal))
        return RO_EINVAL;
    if (a->n_seqs > 0 && (!a->q_off || !a->kv_len || (a->table_stride > 0 && !a->table))) return RO_EINVAL;
    if (a->n_seqs == 0 && a->n_tokens > 0) return RO_EINVAL;
    if (a->n_seqs > h->max_seqs || a->n_tokens > h->max_tokens) return RO_ECAP;
    // positions, and (token, head) pairs, are counted in 32 bits
    const int64_t cols = a->table_stride < h->max_pages ? a->table_stride : h->max_pages;
    if (cols * k->page_size > ((int64_t)1 << 30) || a->n_seqs * (cols * k->page_size / kKeys + 1) > INT32_MAX ||
        a->n_tokens * a->q_heads > ((int64_t)1 << 30))
        return RO_EINVAL;
    // a launch has a workgroup for every sequence and key / value head, and fewer than 2^24
    if (a->n_seqs * k->n_heads > ((int64_t)1 << 22)) return RO_EINVAL;
    Chunk &t = h->tab;
    t.cols = cols;
    t.n_seqs = (int32_t)a->n_seqs;
    t.n_tokens = (int32_t)a->n_tokens;
    t.q_heads = a->q_heads;
    t.kv_heads = k->n_heads;
    t.group = a->q_heads / k->n_heads;
    t.head_dim = k->head_dim;
    t.page_shift = __builtin_ctz((unsigned)k->page_size);
    t.causal = a->causal;
    // (a window of all positions there can be is as good as a wider one, and sums with it stay in 32 bits)
    const int64_t most_pos = cols * k->page_size;
    t.window = a->window > most_pos && a->window > 1 ? (int32_t)(most_pos > 1 ? most_pos : 1) : a->window;
    t.sinks = a->sinks;
    t.max_new = (int32_t)(a->max_new < a->n_tokens ? a->max_new : a->n_tokens);
    // Short sequences beside longer ones are narrow tiles if there can be any
    // (every other sequence has at most max_new tokens) and their caches can
    // be long enough to be worth a launch of their own.
    const int64_t shortest = a->n_tokens - (a->n_seqs - 1) * (int64_t)t.max_new;
    const int64_t cached = a->n_seqs * most_pos * k->n_heads * k->head_dim * 4;
    const bool narrow = (int64_t)t.max_new * t.group <= kFewRows || (shortest * t.group <= kFewRows && cached > kNarrowBytes);
    t.few_rows = narrow ? kFewRows : 0;
    // few rows a head, and all rows of a sequence fit LDS beside the keys
    const int64_t most = (int64_t)t.max_new * t.group;
    t.weigh_few = most <= kFewRows && most * t.kv_heads * t.head_dim * 2 <= 65536;
    h->n_pages = k->n_pages;
    h->page_size = k->page_size;
    const PlanArgs p = {a->q_off, a->kv_len, a->table, a->table_stride, k->n_pages, a->max_new};
    const hipError_t e = launch_chunk_plan(launch_of(c), t, p);
    h->planned = e == hipSuccess;
    return hip_fail(e);
}

int ro_chunk_append(ro_ctx *c, ro_chunk *h, const ro_cache *cache, const ro_rotary *r, const int32_t *pos,
                    int64_t pos_stride, const ro_rows *q, const ro_rows *k, const ro_rows *v, const ro_rows *q_out)
{
    if (!chunk_ok(c, h, cache) || (q != nullptr) != (q_out != nullptr)) return RO_EINVAL;
    const Chunk &t = h->tab;
    if (r && !rotary_ok(r, pos, pos_stride, t.n_tokens, t.head_dim)) return RO_EINVAL;
    if (t.n_tokens == 0) return RO_OK;
    if (!rows_ok(k) || !rows_ok(v)) return RO_EINVAL;
    if (q && (!rows_ok(q) || !rows_ok(q_out) || !rows_apart(q_out, t.n_tokens, t.q_heads, t.head_dim) ||
              rows_clash(q, q_out, t.n_tokens, t.q_heads, t.head_dim) ||
              rows_clash(k, q_out, t.n_tokens, t.kv_heads, t.head_dim, t.q_heads) ||
              rows_clash(v, q_out, t.n_tokens, t.kv_heads, t.head_dim, t.q_heads)))
        return RO_EINVAL;
    RotaryArgs ra;
    if (r) ra = rotary_of(r, pos, pos_stride);
    return hip_fail(launch_append(launch_of(c), t, pages_of(cache), r ? &ra : nullptr, rows_of(q), rows_of(k),
                                  rows_of(v), rows_of(q_out), cache->dtype));
}

int ro_chunk_attend(ro_ctx *c, ro_chunk *h, const ro_cache *cache, const ro_rows *q, const ro_rows *out, float *lse,
                    float scale)
{
    if (!chunk_ok(c, h, cache)) return RO_EINVAL;
    const Chunk &t = h->tab;
    if (t.n_tokens == 0) return RO_OK;
    if (!rows_wide(q) || !rows_wide(out) || !rows_apart(out, t.n_tokens, t.q_heads, t.head_dim) ||
        rows_clash(q, out, t.n_tokens, t.q_heads, t.head_dim) || scale - scale != 0.0f)
        return RO_EINVAL;
    return hip_fail(launch_attend(launch_of(c), t, pages_of(cache), rows_of(q), rows_of(out), lse, scale, cache->dtype));
}

int ro_chunk_weigh(ro_ctx *c, ro_chunk *h, const ro_cache *cache, const ro_rows *q, const float *lse,
                   const float *weight_in, float *weight_out, int64_t weight_stride, float scale)
{
    if (!chunk_ok(c, h, cache) || weight_stride < 0) return RO_EINVAL;
    const Chunk &t = h->tab;
    if (t.n_seqs == 0) return RO_OK;
    if (!weight_out || (t.n_tokens > 0 && (!rows_wide(q) || !lse)) || scale - scale != 0.0f)
        return RO_EINVAL;
    const int64_t bytes = t.n_seqs * weight_stride * 4;
    if (weight_in != weight_out && overlap(weight_in, bytes, weight_out, bytes)) return RO_EINVAL;
    return hip_fail(launch_weigh(launch_of(c), t, pages_of(cache), rows_of(q), lse, weight_in, weight_out,
                                 weight_stride, scale, cache->dtype));
}

int ro_chunk_evict(ro_ctx *c, ro_chunk *h, const ro_cache *cache, const float *weight, int64_t weight_stride,
                   const uint32_t *dst_table, int64_t dst_stride, int64_t budget, int64_t first, int64_t last,
                   int32_t *new_len, int32_t *index, float *new_weight)
{
    if (!chunk_ok(c, h, cache) || weight_stride < 0 || dst_stride < 0 || budget < 1 || budget > ((int64_t)1 << 30) ||
        first < 0 || last < 0 || first > budget || last > budget - first)
        return RO_EINVAL;
    const Chunk &t = h->tab;
    if (t.n_seqs == 0) return RO_OK;
    if (!weight || !dst_table || !new_len || !index) return RO_EINVAL;
    const int64_t wb = t.n_seqs * weight_stride * 4, ib = t.n_seqs * budget * 4;
    if (overlap(weight, wb, index, ib) || overlap(weight, wb, new_weight, ib) || overlap(index, ib, new_weight, ib) ||
        overlap(weight, wb, new_len, t.n_seqs * 4) || overlap(index, ib, new_len, t.n_seqs * 4) ||
        overlap(new_weight, ib, new_len, t.n_seqs * 4))
        return RO_EINVAL;
    const EvictArgs a = {weight, weight_stride, dst_table, dst_stride, h->n_pages, (int32_t)budget, (int32_t)first,
                         (int32_t)last, new_len, index, new_weight};
    return hip_fail(launch_evict(launch_of(c), t, pages_of(cache), a));
}

int ro_chunk_destroy(ro_chunk *h)
{
    if (!h) return RO_EINVAL;
    if (h->ctx) (void)hipStreamSynchronize(h->ctx->stream);
    (void)hipFree(h->block);
    free(h);
    return RO_OK;
}

}  // extern "C"
