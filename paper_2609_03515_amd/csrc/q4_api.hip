// C ABI of the paged 4-bit cache: argument validation, workspace layout and launches.  As in api.hip everything is queued
// on the caller's stream; nothing is allocated, synchronised or read back.
#include <float.h>
#include <math.h>

#include "../../include/inertiakv.h"
#include "kernels.h"
#include "kv_common.h"
#include "q4.h"

namespace ikv {
namespace {

static_assert(kFaultCache == (uint32_t)KV_FAULT_CACHE && kFaultNoPages == (uint32_t)KV_FAULT_NO_PAGES &&
                  kFaultSharedPage == (uint32_t)KV_FAULT_SHARED_PAGE,
              "fault bits of the kernels and the ABI");

constexpr size_t kFaultBytes = 256;
// A launch has fewer than 2^32 threads along each extent of its grid, and at most 65535 workgroups along the second and third.
constexpr int kMostHeads = 1 << 16;
constexpr double kMostRowItems = (double)(1 << 28) - 256;  // 16 threads a row of the store and the load, in whole workgroups
constexpr double kMostJoined = (double)(1 << 23) - 1;      // 512 threads a head of the attention's join

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
kv_status hip_status(hipError_t e) { return e == hipSuccess ? KV_OK : KV_ERR_HIP; }
int esize(const kv_q4_shape& s) { return s.dtype == KV_F32 ? 4 : 2; }

kv_status check_shape(const kv_q4_shape* s) {
    if (!s) return KV_ERR_INVALID_ARG;
    if (s->batch < 1 || s->layers < 1 || s->n_q_heads < 1 || s->n_kv_heads < 1 || s->n_pages < 1 || s->max_pages < 1 ||
        s->page_rows < 1)
        return KV_ERR_INVALID_ARG;
    if (s->layers > kMaxLayers || s->batch > 65535) return KV_ERR_UNSUPPORTED;
    if (s->n_q_heads % s->n_kv_heads) return KV_ERR_INVALID_ARG;
    if (s->dtype != KV_F32 && s->dtype != KV_BF16) return KV_ERR_UNSUPPORTED;
    if (s->head_dim != 64 && s->head_dim != 128) return KV_ERR_UNSUPPORTED;
    if (s->n_q_heads / s->n_kv_heads > kMaxGroup || s->n_kv_heads > kMostHeads) return KV_ERR_UNSUPPORTED;
    if (s->page_rows < 16 || s->page_rows > 256 || (s->page_rows & (s->page_rows - 1))) return KV_ERR_UNSUPPORTED;
    // row numbers, items of a row (compaction) and the pages wanted by a batch fit 31 bits, and so does every grid
    const double cap = (double)s->max_pages * s->page_rows;
    if (cap > (double)(1 << 27) || s->batch * cap > 2.0e9) return KV_ERR_UNSUPPORTED;
    if ((double)s->batch * s->layers * s->n_q_heads > 2.0e9 || (double)s->n_pages * s->page_rows > 2.0e9) return KV_ERR_UNSUPPORTED;
    if ((double)s->layers * s->n_pages * s->n_kv_heads * s->page_rows * s->head_dim > 9.0e15) return KV_ERR_UNSUPPORTED;
    return KV_OK;
}

Q4Dims dims_of(const kv_q4_shape& s) {
    Q4Dims d{};
    d.batch = s.batch;
    d.layers = s.layers;
    d.hq = s.n_q_heads;
    d.hkv = s.n_kv_heads;
    d.group = s.n_q_heads / s.n_kv_heads;
    d.d = s.head_dim;
    d.page_rows = s.page_rows;
    d.page_shift = __builtin_ctz((unsigned)s.page_rows);
    d.n_pages = s.n_pages;
    d.max_pages = s.max_pages;
    d.cap = s.max_pages * s.page_rows;
    d.bf16 = s.dtype == KV_BF16;
    d.ks_off = s.page_rows * (s.head_dim / 2);
    d.vc_off = d.ks_off + s.page_rows * (s.head_dim / 32);
    d.vs_off = d.vc_off + d.ks_off;
    d.rec = 2 * d.vc_off;
    return d;
}

kv_status check_cache(const kv_q4_cache* c) {
    if (!c || !c->pool || !c->table || !c->len || !c->refs) return KV_ERR_INVALID_ARG;
    if (!aligned(c->pool, 16) || !aligned(c->table, 4) || !aligned(c->len, 4) || !aligned(c->refs, 4) || !aligned(c->u, 4) ||
        !aligned(c->pos, 4))
        return KV_ERR_UNSUPPORTED;
    return KV_OK;
}

Q4Cache cache_of(const kv_q4_cache& c) { return Q4Cache{c.pool, c.table, c.len, c.refs, c.u, c.pos}; }

kv_status check_ws(void* ws, size_t ws_bytes, size_t need) {
    if (!ws || ws_bytes < need) return KV_ERR_WORKSPACE;
    return aligned(ws, 256) ? KV_OK : KV_ERR_INVALID_ARG;
}

// The page calls' scratch after the fault word.  n_max 0: without the compaction's lists.
size_t page_layout(const Q4Dims& d, int n_max, void* ws, Q4PageScratch* out) {
    size_t off = kFaultBytes;
    auto take = [&](size_t ints) {
        int32_t* p = ws ? reinterpret_cast<int32_t*>(static_cast<char*>(ws) + off) : nullptr;
        off = align256(off + ints * sizeof(int32_t));
        return p;
    };
    Q4PageScratch w{};
    w.need = take(d.batch);
    w.offset = take(d.batch);
    w.source = take(d.batch);
    w.rows = take(d.batch);
    w.moves = take(d.batch);
    w.fresh = take(d.n_pages);
    if (n_max > 0) {
        w.dst = take((size_t)d.batch * n_max);
        w.src = take((size_t)d.batch * n_max);
        w.rank = take((size_t)d.batch * d.max_pages);
        w.replaced = take((size_t)d.batch * d.max_pages);
        const size_t words = d.batch * (((size_t)n_max + 63) / 64);
        w.mask = reinterpret_cast<uint64_t*>(take(2 * words));
        w.prefix = take(words);
        w.old_table = take((size_t)d.batch * d.max_pages);
    }
    if (out) *out = w;
    return off;
}

// The attention's scratch after the fault word: sized for every number of rows up to n_max.
struct AttendLayout {
    Q4AttendPlan plan;
    size_t z_off, stat_off, part_off, opart_off, total;
};
AttendLayout attend_layout(const Q4Dims& d, int n_max, int layer_count, bool scores) {
    AttendLayout L{};
    L.plan = q4_attend_plan(d, layer_count, n_max, scores);
    const size_t slabs = (size_t)layer_count * d.batch * d.hkv, slots = L.plan.most > 1 ? slabs * L.plan.most : 0;
    size_t off = kFaultBytes;
    auto take = [&](size_t bytes) {
        const size_t at = off;
        off = align256(off + bytes);
        return at;
    };
    L.part_off = take(slots * d.group * sizeof(float2));
    L.opart_off = take(slots * d.group * d.d * sizeof(float));
    if (scores) {
        L.stat_off = take(slabs * d.group * sizeof(float2));
        L.z_off = take(slabs * d.group * L.plan.n_stride * sizeof(float));
    }
    L.total = off;
    return L;
}

kv_status check_rows(const kv_q4_shape& s, int layer0, int layer_count, int rows, const void* k, const void* v,
                     const kv_q4_strides* ks, const kv_q4_strides* vs, const int32_t* first, const int32_t* count,
                     bool written) {
    if (layer0 < 0 || layer_count < 1 || layer_count > s.layers - layer0 || rows < 1) return KV_ERR_INVALID_ARG;
    if (rows > s.max_pages * s.page_rows || !k || !v || !ks || !vs) return KV_ERR_INVALID_ARG;
    if ((double)layer_count * s.batch * s.n_kv_heads * rows > kMostRowItems) return KV_ERR_UNSUPPORTED;
    if (!aligned(k, 16) || !aligned(v, 16) || !aligned(first, 4) || !aligned(count, 4)) return KV_ERR_UNSUPPORTED;
    for (const kv_q4_strides* st : {ks, vs})
        for (int64_t x : {st->layer, st->batch, st->head, st->row})
            if (x % (16 / esize(s))) return KV_ERR_UNSUPPORTED;  // 16-byte rows
    for (const kv_q4_strides* st : {ks, vs})
        if (written && ((st->layer == 0 && layer_count > 1) || (st->batch == 0 && s.batch > 1) ||
                        (st->head == 0 && s.n_kv_heads > 1) || (st->row == 0 && rows > 1)))
            return KV_ERR_INVALID_ARG;
    return KV_OK;
}

void set_rows(Q4RowArgs* a, const kv_q4_shape& s, const kv_q4_cache& c, int layer0, int layer_count, int rows,
              const int32_t* first, const int32_t* count, const kv_q4_strides& ks, const kv_q4_strides& vs, void* ws) {
    a->dims = dims_of(s);
    a->cache = cache_of(c);
    a->layer0 = layer0;
    a->layer_count = layer_count;
    a->rows = rows;
    a->first = first;
    a->count = count;
    const int64_t k4[4] = {ks.layer, ks.batch, ks.head, ks.row}, v4[4] = {vs.layer, vs.batch, vs.head, vs.row};
    for (int i = 0; i < 4; ++i) {
        a->ks[i] = k4[i];
        a->vs[i] = v4[i];
    }
    a->faults = static_cast<uint32_t*>(ws);
}

// Checks and arguments that the page calls share.
kv_status page_args(const kv_q4_shape* shape, const kv_q4_cache* cache, int n_max, void* ws, size_t ws_bytes, Q4PageArgs* a) {
    kv_status rc = check_shape(shape);
    if (rc == KV_OK) rc = check_cache(cache);
    if (rc != KV_OK) return rc;
    a->dims = dims_of(*shape);
    a->cache = cache_of(*cache);
    a->n_max = n_max;
    if ((rc = check_ws(ws, ws_bytes, page_layout(a->dims, n_max, nullptr, nullptr))) != KV_OK) return rc;
    page_layout(a->dims, n_max, ws, &a->w);
    a->faults = static_cast<uint32_t*>(ws);
    return KV_OK;
}

}  // namespace
}  // namespace ikv

using namespace ikv;

extern "C" {

kv_status kv_q4_pool_bytes(const kv_q4_shape* shape, size_t* bytes) {
    const kv_status rc = check_shape(shape);
    if (rc != KV_OK) return rc;
    if (!bytes) return KV_ERR_INVALID_ARG;
    *bytes = (size_t)shape->layers * shape->n_pages * shape->n_kv_heads * dims_of(*shape).rec;
    return KV_OK;
}

kv_status kv_q4_workspace_bytes(const kv_q4_shape* shape, int32_t n_max, int32_t layer_count, size_t* bytes) {
    const kv_status rc = check_shape(shape);
    if (rc != KV_OK) return rc;
    const Q4Dims d = dims_of(*shape);
    if (!bytes || n_max < 1 || n_max > d.cap || layer_count < 1 || layer_count > shape->layers) return KV_ERR_INVALID_ARG;
    size_t need = page_layout(d, n_max, nullptr, nullptr);
    for (int l = 1; l <= layer_count; ++l) {  // (calls on fewer layers may cut their slabs into more chunks)
        const size_t t = attend_layout(d, n_max, l, true).total;
        if (t > need) need = t;
    }
    *bytes = need;
    return KV_OK;
}

kv_status kv_q4_reserve(const kv_q4_shape* shape, const kv_q4_cache* cache, const int32_t* add, const int32_t* new_pos,
                        int32_t init, int32_t* granted, void* ws, size_t ws_bytes, void* stream) {
    Q4PageArgs a{};
    const kv_status rc = page_args(shape, cache, 0, ws, ws_bytes, &a);
    if (rc != KV_OK) return rc;
    if (!add || init < KV_INIT_MEAN || init > KV_INIT_ZERO) return KV_ERR_INVALID_ARG;
    if (!aligned(add, 4) || !aligned(new_pos, 4) || !aligned(granted, 4)) return KV_ERR_UNSUPPORTED;
    a.add = add;
    a.new_pos = new_pos;
    a.granted = granted;
    a.init_mode = init == KV_INIT_ZERO ? 0 : init == KV_INIT_MEAN ? 1 : 2;
    return hip_status(launch_q4_reserve(a, static_cast<hipStream_t>(stream)));
}

kv_status kv_q4_store(const kv_q4_shape* shape, const kv_q4_cache* cache, int32_t layer0, int32_t layer_count, int32_t rows,
                      const int32_t* first, const int32_t* count, const void* k, const kv_q4_strides* k_strides, const void* v,
                      const kv_q4_strides* v_strides, void* ws, size_t ws_bytes, void* stream) {
    kv_status rc = check_shape(shape);
    if (rc == KV_OK) rc = check_cache(cache);
    if (rc == KV_OK) rc = check_rows(*shape, layer0, layer_count, rows, k, v, k_strides, v_strides, first, count, false);
    if (rc == KV_OK) rc = check_ws(ws, ws_bytes, kFaultBytes);
    if (rc != KV_OK) return rc;
    Q4RowArgs a{};
    set_rows(&a, *shape, *cache, layer0, layer_count, rows, first, count, *k_strides, *v_strides, ws);
    a.k = k;
    a.v = v;
    return hip_status(launch_q4_store(a, static_cast<hipStream_t>(stream)));
}

kv_status kv_q4_load(const kv_q4_shape* shape, const kv_q4_cache* cache, int32_t layer0, int32_t layer_count, int32_t rows,
                     const int32_t* first, const int32_t* count, void* k, const kv_q4_strides* k_strides, void* v,
                     const kv_q4_strides* v_strides, void* ws, size_t ws_bytes, void* stream) {
    kv_status rc = check_shape(shape);
    if (rc == KV_OK) rc = check_cache(cache);
    if (rc == KV_OK) rc = check_rows(*shape, layer0, layer_count, rows, k, v, k_strides, v_strides, first, count, true);
    if (rc == KV_OK) rc = check_ws(ws, ws_bytes, kFaultBytes);
    if (rc != KV_OK) return rc;
    Q4RowArgs a{};
    set_rows(&a, *shape, *cache, layer0, layer_count, rows, first, count, *k_strides, *v_strides, ws);
    a.k_out = k;
    a.v_out = v;
    return hip_status(launch_q4_load(a, static_cast<hipStream_t>(stream)));
}

kv_status kv_q4_attend(const kv_q4_shape* shape, const kv_q4_cache* cache, int32_t layer0, int32_t layer_count, int32_t n_max,
                       const void* q, const int32_t* cur_pos, float recency_bias, int32_t recency_window, void* o,
                       float* s_out, float alpha, const float* u_prior, float* u_out, void* ws, size_t ws_bytes,
                       void* stream) {
    kv_status rc = check_shape(shape);
    if (rc == KV_OK) rc = check_cache(cache);
    if (rc != KV_OK) return rc;
    const kv_q4_shape& s = *shape;
    const Q4Dims d = dims_of(s);
    if (layer0 < 0 || layer_count < 1 || layer_count > s.layers - layer0 || n_max < 1 || n_max > d.cap) return KV_ERR_INVALID_ARG;
    if (recency_window < 0 || !isfinite(recency_bias) || !q || !o) return KV_ERR_INVALID_ARG;
    const bool biased = recency_window > 0 && recency_bias != 0.0f;
    if (biased && (!cur_pos || !cache->pos)) return KV_ERR_INVALID_ARG;
    if (u_out && (!u_prior || !(alpha >= 0.0f && alpha < 1.0f))) return KV_ERR_INVALID_ARG;
    if (!aligned(q, 16) || !aligned(o, 16) || !aligned(cur_pos, 4) || !aligned(s_out, 4) || !aligned(u_prior, 4) || !aligned(u_out, 4))
        return KV_ERR_UNSUPPORTED;
    const bool scores = s_out || u_out;
    const AttendLayout L = attend_layout(d, n_max, layer_count, scores);
    if ((double)layer_count * L.plan.nchunk > 65535.0) return KV_ERR_UNSUPPORTED;
    if (L.plan.nchunk > 1 && (double)layer_count * s.batch * s.n_q_heads > kMostJoined) return KV_ERR_UNSUPPORTED;
    if ((rc = check_ws(ws, ws_bytes, L.total)) != KV_OK) return rc;
    Q4AttendArgs a{};
    a.dims = d;
    a.cache = cache_of(*cache);
    a.layer0 = layer0;
    a.layer_count = layer_count;
    a.n_max = n_max;
    a.n_stride = L.plan.n_stride;
    a.q = q;
    a.o = o;
    a.cur_pos = cur_pos;
    a.bias = biased ? recency_bias : 0.0f;
    a.window = recency_window;
    constexpr double kLog2e = 1.4426950408889634;
    a.scale2 = (float)(kLog2e / sqrt((double)s.head_dim));
    // (log2(e) times a bias near the type's border is past it; half of that border still hides every logit, and leaves room above
    // the running maximum's start for rows that all have it)
    a.bias2 = (float)fmax(-0.5 * FLT_MAX, fmin(0.5 * FLT_MAX, kLog2e * a.bias));
    a.nchunk = L.plan.nchunk;
    a.chunk_rows = L.plan.chunk_rows;
    a.scored = L.plan.scored;
    a.columns = L.plan.columns;
    char* base = static_cast<char*>(ws);
    a.z = scores ? reinterpret_cast<float*>(base + L.z_off) : nullptr;
    a.stat = scores ? reinterpret_cast<float2*>(base + L.stat_off) : nullptr;
    a.part = reinterpret_cast<float2*>(base + L.part_off);
    a.opart = reinterpret_cast<float*>(base + L.opart_off);
    a.s_out = s_out;
    a.u_prior = u_prior;
    a.u_out = u_out;
    a.alpha = alpha;
    a.faults = reinterpret_cast<uint32_t*>(base);
    return hip_status(launch_q4_attend(a, static_cast<hipStream_t>(stream)));
}

kv_status kv_q4_fork(const kv_q4_shape* shape, const kv_q4_cache* cache, int32_t count, const int32_t* src, const int32_t* dst,
                     void* ws, size_t ws_bytes, void* stream) {
    kv_status rc = check_shape(shape);
    if (rc == KV_OK) rc = check_cache(cache);
    if (rc != KV_OK) return rc;
    if (count < 1 || count > shape->batch || !src || !dst) return KV_ERR_INVALID_ARG;
    if (!aligned(src, 4) || !aligned(dst, 4)) return KV_ERR_UNSUPPORTED;
    if ((rc = check_ws(ws, ws_bytes, kFaultBytes)) != KV_OK) return rc;
    Q4PageArgs a{};
    a.dims = dims_of(*shape);
    a.cache = cache_of(*cache);
    a.faults = static_cast<uint32_t*>(ws);
    a.count = count;
    a.src_slot = src;
    a.dst_slot = dst;
    return hip_status(launch_q4_fork(a, static_cast<hipStream_t>(stream)));
}

kv_status kv_q4_free(const kv_q4_shape* shape, const kv_q4_cache* cache, int32_t count, const int32_t* slots, void* ws,
                     size_t ws_bytes, void* stream) {
    kv_status rc = check_shape(shape);
    if (rc == KV_OK) rc = check_cache(cache);
    if (rc != KV_OK) return rc;
    if (count < 1 || count > shape->batch || !slots) return KV_ERR_INVALID_ARG;
    if (!aligned(slots, 4)) return KV_ERR_UNSUPPORTED;
    if ((rc = check_ws(ws, ws_bytes, kFaultBytes)) != KV_OK) return rc;
    Q4PageArgs a{};
    a.dims = dims_of(*shape);
    a.cache = cache_of(*cache);
    a.faults = static_cast<uint32_t*>(ws);
    a.count = count;
    a.dst_slot = slots;
    return hip_status(launch_q4_free(a, static_cast<hipStream_t>(stream)));
}

kv_status kv_q4_compact(const kv_q4_shape* shape, const kv_q4_cache* cache, int32_t n_max, const uint8_t* keep, void* ws,
                        size_t ws_bytes, void* stream) {
    kv_status rc = check_shape(shape);
    if (rc != KV_OK) return rc;
    if (n_max < 1 || n_max > shape->max_pages * shape->page_rows || !keep) return KV_ERR_INVALID_ARG;
    Q4PageArgs a{};
    if ((rc = page_args(shape, cache, n_max, ws, ws_bytes, &a)) != KV_OK) return rc;
    a.keep = keep;
    return hip_status(launch_q4_compact(a, static_cast<hipStream_t>(stream)));
}

kv_status kv_q4_evict(const kv_q4_shape* shape, const kv_q4_cache* cache, int32_t n_max, const int32_t* budget,
                      uint8_t* keep_out, void* ws, size_t ws_bytes, void* stream) {
    kv_status rc = check_shape(shape);
    if (rc != KV_OK) return rc;
    if (n_max < 1 || n_max > shape->max_pages * shape->page_rows || !budget) return KV_ERR_INVALID_ARG;
    if (!aligned(budget, 4)) return KV_ERR_UNSUPPORTED;
    Q4PageArgs a{};
    if ((rc = page_args(shape, cache, n_max, ws, ws_bytes, &a)) != KV_OK) return rc;
    if (!cache->u || !cache->pos) return KV_ERR_INVALID_ARG;
    a.budget = budget;
    a.keep_out = keep_out;
    return hip_status(launch_q4_compact(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
