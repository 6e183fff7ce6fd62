// The paged 4-bit cache: sizes, addresses and launchers (q4_rows.hip, q4_rotary.hip, q4_attend.hip, q4_queries.hip,
// q4_pages.hip).
//
// A row's elements are held in blocks of 32: 32 codes of 4 bits (OCP microscaling's e2m1: sign, two exponent bits, one
// mantissa bit; the first element in the low half of a byte) and one scale byte E, the power of two 2^(E - 127).  gfx950
// converts pairs of such codes to bf16 with their scale applied in one instruction, exactly (two significant bits).
// The pool is [layers][n_pages][n_kv][record]; a record holds page_rows rows of one KV head: the keys' codes
// [page_rows][d / 2], the keys' scales [page_rows][d / 32], then the values' codes and scales.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace ikv {

constexpr uint32_t kFaultCache = 2u;       // a length, table entry, reference count or index out of its range
constexpr uint32_t kFaultNoPages = 4u;     // too few free pages
constexpr uint32_t kFaultSharedPage = 8u;  // a row to be stored lies in a page that other sequences use too

struct Q4Dims {
    int batch, layers, hq, hkv, group, d, page_rows, page_shift, n_pages, max_pages, cap, bf16;
    // bytes of a record and its parts' offsets
    int ks_off, vc_off, vs_off, rec;
};

struct Q4Cache {
    uint8_t* pool;
    int32_t* table;  // [batch][max_pages]
    int32_t* len;    // [batch]
    int32_t* refs;   // [n_pages]
    float* u;        // [batch][cap]
    int32_t* pos;    // [batch][cap]
};

__host__ __device__ inline size_t q4_record(const Q4Dims& d, int layer, int page, int head) {
    return (((size_t)layer * d.n_pages + page) * d.hkv + head) * d.rec;
}

// Rows written to or read from the cache.  Row r < count[b] (all `rows` without count) of sequence b is cached row
// first[b] + r (without first: the newest rows, first = len - count).
struct Q4RowArgs {
    Q4Dims dims;
    Q4Cache cache;
    int layer0, layer_count, rows;
    const int32_t* first;  // nullable [batch]
    const int32_t* count;  // nullable [batch]
    const void* k;
    const void* v;
    void* k_out;
    void* v_out;
    int64_t ks[4], vs[4];  // strides in elements: layer, sequence, head, row
    uint32_t* faults;
};
hipError_t launch_q4_store(const Q4RowArgs& a, hipStream_t s);
hipError_t launch_q4_load(const Q4RowArgs& a, hipStream_t s);

// The store with keys rotated by their positions, and queries beside them.
struct Q4RotaryArgs {
    Q4RowArgs rows;
    const void* q;             // nullable
    void* q_out;
    int64_t qs[4], os[4];      // strides in elements: layer, sequence, query head, row
    const int32_t* positions;  // [axes][batch][rows]
    int dim, adjacent;         // elements rotated; pairs 2 i, 2 i + 1 instead of i, i + dim / 2
    float scale;
    float inv_freq[64];
    uint8_t axis[64];
};
hipError_t launch_q4_store_rotary(const Q4RotaryArgs& a, hipStream_t s);

// Decode attention over rows [0, len[b]) of every sequence.
struct Q4AttendArgs {
    Q4Dims dims;
    Q4Cache cache;
    int layer0, layer_count, n_max, n_stride;
    const void* q;           // [layer_count][batch][hq][d]
    void* o;
    const int32_t* cur_pos;  // [batch] (bias only)
    float bias;
    int window;
    float scale2;            // log2(e) / sqrt(d)
    float bias2;             // log2(e) * bias
    int nchunk, chunk_rows, scored, columns;  // Q4AttendPlan
    int stat_at, q_at;       // floats of LDS before the waves' statistics, and before an f32 query's parts (set by the launch)
    float* z;                // scores wanted: base-2 logits [slab][group][n_stride], or [slab][n_stride] parts of the scores
    float2* stat;            // scores wanted: [slab][group] (max, 1 / sum of 2^(z - max)), slab = (layer * batch + b) * hkv + head
    float2* part;            // several chunks: [slab][nchunk][group] (max, sum)
    float* opart;            // several chunks: [slab][nchunk][group][d] unnormalised partial outputs
    float* s_out;            // nullable [layer_count][batch][n_max]
    const float* u_prior;    // nullable [batch][cap]
    float* u_out;            // nullable [batch][cap]
    float alpha;
    uint32_t* faults;
};
// How a call on layer_count layers and at most n_max rows is divided: chunks of rows per slab, `most` of them at most (which
// does not fall when n_max grows); or (scored) a slab per workgroup with its logits in LDS.  columns: a head's,
// for the parts of its probabilities.
struct Q4AttendPlan {
    int nchunk, chunk_rows, most, scored, n_stride, columns;
};
Q4AttendPlan q4_attend_plan(const Q4Dims& d, int layer_count, int n_max, bool scores);
hipError_t launch_q4_attend(const Q4AttendArgs& a, hipStream_t s);

// Attention of blocks of queries: the newest rows' queries of a slot in a window (kv_q4_attend_window), or one query of each of
// several slots that share pages (kv_q4_attend_shared).  A block is `vectors` queries; each is `group` columns of a product.
constexpr int kQ4MostVectors = 32;  // queries of a shared block (the bits of a tile's mask; a windowed block has up to 64)
constexpr int kQ4MostColumns = 64;  // columns of a block
constexpr int kQ4Units = 4;  // most workgroups for a CU, where blocks are divided
struct Q4QueryPlan {
    int tiles;    // column tiles of 16 in a block
    int per;      // queries in a column tile
    int vectors;  // queries in a block
    int vector_shift;  // shared: the lowest power of two that is no fewer
    int blocks;   // blocks of a slot (window), or of the batch where its groups fill them (shared)
    int waves;    // of a workgroup
    int marks;    // window with positions: a kernel marks the tiles of which a block sees any row
    int chunks;   // workgroups that divide a block's rows
};
struct Q4QueryArgs {
    Q4Dims dims;
    Q4Cache cache;
    Q4QueryPlan plan;
    int layer0, layer_count, n_max;
    const void* q;
    void* o;
    int64_t qs[4], os[4];    // strides in elements: layer, slot, query head, row
    float scale2;            // log2(e) / sqrt(d)
    int stat_at, q_at;       // floats of LDS before the waves' statistics and the queries (set by the launch)
    float2* part;            // several chunks: [layer][slot][row][query head][chunk] (max, sum)
    float* opart;            // several chunks: likewise, and [d]: unnormalised partial outputs (not written where the sum is 0)
    uint32_t* faults;
    // window
    int rows, window, sinks;
    const int32_t* count;    // nullable [batch]
    uint64_t* visible;       // nullable: [batch][blocks][words] a bit for every 32 rows of which a block sees any
    int words;
    // shared
    const int32_t* group;    // [batch]
    int32_t* heads;          // nullable (at most 64 slots): [batch] whether a block begins with the slot
    int32_t* members;        // likewise: [batch][vectors] the slots of the block that begins with a slot, -1 behind the last
};
Q4QueryPlan q4_window_plan(const Q4Dims& d, int layer_count, int n_max, int rows, int window, int sinks);
Q4QueryPlan q4_shared_plan(const Q4Dims& d, int layer_count, int n_max);
hipError_t launch_q4_window(const Q4QueryArgs& a, hipStream_t s);
hipError_t launch_q4_shared(const Q4QueryArgs& a, hipStream_t s);

// Pages.  Scratch of the calls that allocate pages; the lists are the compaction's.
struct Q4PageScratch {
    int32_t* need;      // [batch] pages wanted
    int32_t* offset;    // [batch] first of them in `fresh`, or -1: not granted
    int32_t* source;    // [batch] reserve: page to be copied, or -1
    int32_t* rows;      // [batch] reserve: rows added; compaction: rows kept (-1: the sequence is left alone)
    int32_t* moves;     // [batch] reserve: rows of `source` in use; compaction: holes
    int32_t* fresh;     // [n_pages] the lowest free pages, ascending
    int32_t* dst;       // [batch][n_max] holes before the new end, ascending, ...
    int32_t* src;       // [batch][n_max] ... and the kept rows behind it that fill them
    int32_t* rank;      // [batch][max_pages] a page's number among those replaced (by the sequence's fresh pages), or -1
    int32_t* replaced;  // [batch][max_pages] the pages replaced
    int32_t* old_table; // [batch][max_pages]
    uint64_t* mask;     // [batch][ceil(n_max / 64)] a bit for every row that stays
    int32_t* prefix;    // [batch][ceil(n_max / 64)] kept rows before each word's
};
struct Q4PageArgs {
    Q4Dims dims;
    Q4Cache cache;
    Q4PageScratch w;
    uint32_t* faults;
    // reserve
    const int32_t* add;      // [batch]
    const int32_t* new_pos;  // nullable [batch]
    int32_t* granted;        // nullable [batch]
    int init_mode;           // 0: zero, 1: mean, 2: min of the cached utilities
    // fork / free
    int count;
    const int32_t* src_slot;
    const int32_t* dst_slot;
    // compaction
    int n_max;
    const uint8_t* keep;     // [batch][cap] (compact)
    const int32_t* budget;   // [batch] (evict)
    uint8_t* keep_out;       // nullable [batch][cap]
};
hipError_t launch_q4_reserve(const Q4PageArgs& a, hipStream_t s);
hipError_t launch_q4_fork(const Q4PageArgs& a, hipStream_t s);
hipError_t launch_q4_free(const Q4PageArgs& a, hipStream_t s);
hipError_t launch_q4_compact(const Q4PageArgs& a, hipStream_t s);  // budget set: evict

}  // namespace ikv
