// Pages of the 4-bit cache: reserving rows (with copy on write), forking, freeing and compacting sequences.
//
// The state is the table, the lengths and one reference count per page; a page is free when its count is 0.  Free pages are
// taken in ascending order, for the sequences in their order, from the counts as they were before the call, so a call's
// result depends on nothing but its inputs.  Counts change by integer atomics (an order does not matter).
//
// A call that allocates runs in launches on the caller's stream: what each sequence needs, the pages for it (one workgroup),
// and the change itself, spread over sequences and layers.  The last one reads what the others wrote in the scratch, never
// the table or the lengths that its own workgroups change.
#include "kv_common.h"
#include "q4.h"

namespace ikv {
namespace {

constexpr int kThreads = 1024;  // workgroups that scan
constexpr int kWaves = kThreads / kWave;
constexpr int kMoveThreads = 256;

// Exclusive prefix sum over the workgroup's threads; *total gets the sum.  Every thread calls it.
__device__ __forceinline__ int block_scan(int x, int* total, int* lds /* kWaves + 1 */) {
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    int inc = x;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const int y = __shfl_up(inc, o, kWave);
        if (lane >= o) inc += y;
    }
    __syncthreads();  // (a call before this one may still read lds)
    if (lane == kWave - 1) lds[wave] = inc;
    __syncthreads();
    if (wave == 0) {
        int w = lane < kWaves ? lds[lane] : 0;
        const int own = w;
#pragma unroll
        for (int o = 1; o < kWaves; o <<= 1) {
            const int y = __shfl_up(w, o, kWave);
            if (lane >= o) w += y;
        }
        if (lane < kWaves) lds[lane] = w - own;
        if (lane == kWaves - 1) lds[kWaves] = w;
    }
    __syncthreads();
    *total = lds[kWaves];
    return lds[wave] + inc - x;
}

__device__ __forceinline__ bool in_pool(const Q4Dims& d, int page) { return (uint32_t)page < (uint32_t)d.n_pages; }
__device__ __forceinline__ int pages_of(const Q4Dims& d, int rows) { return (rows + d.page_rows - 1) >> d.page_shift; }

// The pages for `need`: their places in `fresh` by a prefix sum over the sequences, and `fresh` filled with the lowest free
// pages.  A sequence whose places lie past the last free page is not granted (offset -1).  One workgroup.
__device__ void grant(const Q4PageArgs& a, int* lds) {
    const Q4Dims& d = a.dims;
    int total = 0;
    for (int b0 = 0; b0 < d.batch; b0 += kThreads) {
        const int b = b0 + (int)threadIdx.x;
        int sum;
        const int at = block_scan(b < d.batch ? a.w.need[b] : 0, &sum, lds);
        if (b < d.batch) a.w.offset[b] = total + at;
        total += sum;  // (at most max_pages + 1 a sequence, and batch x rows of a sequence fit 31 bits)
    }
    if (total == 0) return;
    constexpr int kPer = 16;  // counts per thread and step
    int found = 0;
    for (int p0 = 0; p0 < d.n_pages && found < total; p0 += kThreads * kPer) {
        const int p = p0 + (int)threadIdx.x * kPer;
        uint32_t zero = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (p + i < d.n_pages && a.cache.refs[p + i] == 0) zero |= 1u << i;
        int sum;
        int at = found + block_scan(__popc(zero), &sum, lds);
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (zero >> i & 1u) a.w.fresh[at++] = p + i;  // (at most n_pages of them in all)
        found += sum;
    }
    if (found >= total) return;
    bool refused = false;
    for (int b = threadIdx.x; b < d.batch; b += kThreads) {
        const int need = a.w.need[b];
        if (need > 0 && a.w.offset[b] + need > found) {
            a.w.offset[b] = -1;
            refused = true;
        }
    }
    if (refused) atomicOr(a.faults, kFaultNoPages);
}

// ---- reserve ------------------------------------------------------------------------------------------------

__global__ __launch_bounds__(kThreads) void q4_reserve_plan_kernel(Q4PageArgs a) {
    __shared__ int lds[kWaves + 1];
    const Q4Dims& d = a.dims;
    uint32_t fault = 0;
    for (int b = threadIdx.x; b < d.batch; b += kThreads) {
        const int len = a.cache.len[b], add = a.add[b];
        int rows = 0, need = 0, source = -1;
        if (len < 0 || len > d.cap || add < 0 || add > d.cap - len) {
            fault |= kFaultCache;
        } else if (add > 0) {
            rows = add;
            need = pages_of(d, len + add) - pages_of(d, len);
            if (len & (d.page_rows - 1)) {  // the last page is written to: it has to be this sequence's own
                const int page = a.cache.table[(size_t)b * d.max_pages + (len >> d.page_shift)];
                const int refs = in_pool(d, page) ? a.cache.refs[page] : 0;
                if (refs < 1) {
                    fault |= kFaultCache;
                    rows = need = 0;
                } else if (refs > 1) {
                    source = page;
                    ++need;
                }
            }
        }
        a.w.rows[b] = rows;
        a.w.need[b] = need;
        a.w.source[b] = source;
        a.w.moves[b] = len & (d.page_rows - 1);  // rows of the source in use
    }
    if (fault) atomicOr(a.faults, fault);
    __syncthreads();
    grant(a, lds);
}

// `rows` rows of a page's records of one layer, from one page to another, by the whole workgroup.
__device__ __forceinline__ void copy_rows(const Q4Dims& d, uint8_t* pool, int layer, int from, int to, int rows) {
    const int codes = rows * (d.d / 2), scales = rows * (d.d / 32);  // bytes of a part; codes in 16-byte pieces
    const int pieces = codes / 16, halves = scales / 2;
    const int per = 2 * (pieces + halves);
    for (int i = threadIdx.x; i < per * d.hkv; i += blockDim.x) {
        const int g = i / per;
        int j = i % per;
        const uint8_t* s = pool + q4_record(d, layer, from, g);
        uint8_t* t = pool + q4_record(d, layer, to, g);
        if (j < 2 * pieces) {
            const size_t at = (j < pieces ? 0 : d.vc_off) + (size_t)(j % pieces) * 16;
            *reinterpret_cast<u32x4*>(t + at) = *reinterpret_cast<const u32x4*>(s + at);
        } else {
            j -= 2 * pieces;
            const size_t at = (j < halves ? d.ks_off : d.vs_off) + (size_t)(j % halves) * 2;
            *reinterpret_cast<uint16_t*>(t + at) = *reinterpret_cast<const uint16_t*>(s + at);
        }
    }
}

// Workgroup (b, layer): the copy on write of one layer; that of layer 0 also changes the sequence's state.
__global__ __launch_bounds__(kMoveThreads) void q4_reserve_kernel(Q4PageArgs a) {
    const Q4Dims& d = a.dims;
    const int b = blockIdx.x / d.layers, layer = blockIdx.x % d.layers;
    const int offset = a.w.offset[b], need = a.w.need[b], source = a.w.source[b];
    const int rows = offset < 0 ? 0 : a.w.rows[b];
    if (layer == 0 && a.granted && threadIdx.x == 0) a.granted[b] = rows;
    if (rows == 0) return;
    if (layer != 0 && source < 0) return;
    if (source >= 0) {
        copy_rows(d, a.cache.pool, layer, source, a.w.fresh[offset], a.w.moves[b]);
        if (layer != 0) return;
    }
    const int len = a.cache.len[b];
    const int p0 = pages_of(d, len);
    int32_t* table = a.cache.table + (size_t)b * d.max_pages;
    const int again = source >= 0;
    for (int i = threadIdx.x; i < need; i += kMoveThreads) {
        const int page = a.w.fresh[offset + i];
        table[p0 - again + i] = page;
        a.cache.refs[page] = 1;
    }
    if (again && threadIdx.x == 0) atomicSub(&a.cache.refs[source], 1);
    if (a.cache.pos && a.new_pos)
        for (int i = threadIdx.x; i < rows; i += kMoveThreads) a.cache.pos[(size_t)b * d.cap + len + i] = a.new_pos[b] + i;
    if (a.cache.u) {
        float* u = a.cache.u + (size_t)b * d.cap;
        __shared__ double part[kMoveThreads / kWave];
        __shared__ float prior;
        double x = a.init_mode == 2 ? (double)INFINITY : 0.0;
        if (a.init_mode != 0)
            for (int i = threadIdx.x; i < len; i += kMoveThreads) x = a.init_mode == 1 ? x + u[i] : fmin(x, (double)u[i]);
#pragma unroll
        for (int o = kWave / 2; o >= 1; o >>= 1) {
            const double y = __shfl_xor(x, o, kWave);
            x = a.init_mode == 2 ? fmin(x, y) : x + y;
        }
        if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = x;
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int w = 1; w < kMoveThreads / kWave; ++w) x = a.init_mode == 2 ? fmin(x, part[w]) : x + part[w];
            prior = len == 0 || a.init_mode == 0 ? 0.0f : (float)(a.init_mode == 1 ? x / len : x);
        }
        __syncthreads();
        for (int i = threadIdx.x; i < rows; i += kMoveThreads) u[len + i] = prior;
    }
    __syncthreads();
    if (threadIdx.x == 0) a.cache.len[b] = len + rows;
}

// ---- fork, free ---------------------------------------------------------------------------------------------

// Workgroup i: sequence dst[i] becomes a copy of src[i] that shares its pages.  Refused, and reported: a slot out of range, a
// destination that is not empty or is named twice (after the first time), a source that is a destination of the call.
__global__ __launch_bounds__(kThreads) void q4_fork_kernel(Q4PageArgs a) {
    __shared__ int bad;
    const Q4Dims& d = a.dims;
    const int i = blockIdx.x, src = a.src_slot[i], dst = a.dst_slot[i];
    if (threadIdx.x == 0) bad = 0;
    __syncthreads();
    const bool range = (uint32_t)src < (uint32_t)d.batch && (uint32_t)dst < (uint32_t)d.batch;
    int mine = !range;
    for (int j = threadIdx.x; j < a.count; j += kThreads) {
        const int other = a.dst_slot[j];
        mine |= other == src || (j < i && other == dst);
    }
    if (mine) bad = 1;
    __syncthreads();
    if (bad) {  // (before dst's state is read: another workgroup may be writing it)
        if (threadIdx.x == 0) atomicOr(a.faults, kFaultCache);
        return;
    }
    const int len = a.cache.len[src];
    const bool fits = len >= 0 && len <= d.cap && a.cache.len[dst] == 0;
    const int pages = fits ? pages_of(d, len) : 0;
    const int32_t* st = a.cache.table + (size_t)src * d.max_pages;
    mine = !fits;
    for (int j = threadIdx.x; j < pages; j += kThreads) mine |= !in_pool(d, st[j]);
    if (mine) bad = 1;
    __syncthreads();
    if (bad) {
        if (threadIdx.x == 0) atomicOr(a.faults, kFaultCache);
        return;
    }
    int32_t* dt = a.cache.table + (size_t)dst * d.max_pages;
    for (int j = threadIdx.x; j < d.max_pages; j += kThreads) {
        const int page = j < pages ? st[j] : -1;
        dt[j] = page;
        if (j < pages) atomicAdd(&a.cache.refs[page], 1);
    }
    if (a.cache.u)
        for (int j = threadIdx.x; j < len; j += kThreads) a.cache.u[(size_t)dst * d.cap + j] = a.cache.u[(size_t)src * d.cap + j];
    if (a.cache.pos)
        for (int j = threadIdx.x; j < len; j += kThreads) a.cache.pos[(size_t)dst * d.cap + j] = a.cache.pos[(size_t)src * d.cap + j];
    if (threadIdx.x == 0) a.cache.len[dst] = len;
}

// One reference less; a page that has none is reported and left so.
__device__ __forceinline__ uint32_t release(const Q4PageArgs& a, int page) {
    if (!in_pool(a.dims, page)) return kFaultCache;
    if (atomicSub(&a.cache.refs[page], 1) > 0) return 0;
    atomicAdd(&a.cache.refs[page], 1);
    return kFaultCache;
}

// Workgroup i: sequence dst[i] gives its pages back and is empty.  A slot named twice is freed once.
__global__ __launch_bounds__(kMoveThreads) void q4_free_kernel(Q4PageArgs a) {
    const Q4Dims& d = a.dims;
    const int i = blockIdx.x, slot = a.dst_slot[i];
    if ((uint32_t)slot >= (uint32_t)d.batch) {
        if (threadIdx.x == 0) atomicOr(a.faults, kFaultCache);
        return;
    }
    int again = 0;
    for (int j = threadIdx.x; j < i; j += kMoveThreads) again |= a.dst_slot[j] == slot;
    if (__syncthreads_or(again)) return;
    uint32_t fault = 0;
    int32_t* table = a.cache.table + (size_t)slot * d.max_pages;
    for (int j = threadIdx.x; j < d.max_pages; j += kMoveThreads) {
        const int page = table[j];
        if (page == -1) continue;
        fault |= release(a, page);
        table[j] = -1;
    }
    if (fault) atomicOr(a.faults, fault);
    if (threadIdx.x == 0) a.cache.len[slot] = 0;
}

// ---- compaction ---------------------------------------------------------------------------------------------

// Eviction order as one number: larger stays.  Larger utility first, then the lower position.
__device__ __forceinline__ uint64_t rank_key(float u, int pos) { return (uint64_t)float_key(u) << 32 | (uint32_t)~pos; }

// The `budget`-th largest key of n > budget >= 1 rows: radix selection from the highest byte, each pass a histogram of the
// rows that share the bytes chosen so far, until a byte's rows all stay.  Every thread gets it.
__device__ uint64_t nth_key(const float* u, const int32_t* pos, int n, int budget, int* hist /* 256 */, int* lds) {
    __shared__ uint64_t chosen;
    __shared__ int left_s, done_s;
    uint64_t prefix = 0, mask = 0;
    int left = budget;
    for (int shift = 56; shift >= 0; shift -= 8) {
        for (int i = threadIdx.x; i < 256; i += kThreads) hist[i] = 0;
        __syncthreads();
        for (int i0 = 0; i0 < n; i0 += kThreads) {
            const int i = i0 + (int)threadIdx.x;
            bool in = false;
            int digit = 0;
            if (i < n) {
                const uint64_t key = rank_key(u[i], pos[i]);
                in = (key & mask) == prefix;
                digit = (int)(key >> shift) & 255;
            }
            // utilities share their leading bits: lanes with the first lane's digit count together, the rest one by one
            const uint64_t live = __ballot(in);
            if (!live) continue;
            const int first = __shfl(digit, __ffsll((unsigned long long)live) - 1, kWave);
            const uint64_t same = __ballot(in && digit == first);
            if (in && digit != first) atomicAdd(&hist[digit], 1);
            if ((int)(threadIdx.x % kWave) == __ffsll((unsigned long long)same) - 1) atomicAdd(&hist[first], __popcll(same));
        }
        __syncthreads();
        // the byte that holds the left-th row from the top: threads 0 .. 255 hold the digits from 255 down
        const int digit = 255 - (int)threadIdx.x;
        const int c = threadIdx.x < 256 ? hist[digit] : 0;
        int total;
        const int above = block_scan(c, &total, lds);
        if (threadIdx.x < 256 && above < left && above + c >= left) {
            chosen = prefix | (uint64_t)digit << shift;
            left_s = left - above;
            done_s = c == left - above;
        }
        __syncthreads();
        prefix = chosen;
        left = left_s;
        mask |= (uint64_t)255 << shift;
        const bool done = done_s;
        __syncthreads();
        if (done) break;  // every row that shares these bytes stays
    }
    return prefix;
}

// Workgroup b: what sequence b keeps, the rows that are written (holes, and every kept row of a shared page with a hole),
// and the pages wanted.
template <bool kEvict>
__global__ __launch_bounds__(kThreads) void q4_compact_plan_kernel(Q4PageArgs a) {
    __shared__ int lds[kWaves + 1];
    __shared__ int hist[256];
    const Q4Dims& d = a.dims;
    const int b = blockIdx.x, n = a.cache.len[b];
    const int32_t* table = a.cache.table + (size_t)b * d.max_pages;
    int32_t* rank = a.w.rank + (size_t)b * d.max_pages;
    int32_t* old = a.w.old_table + (size_t)b * d.max_pages;
    const size_t rows0 = (size_t)b * a.n_max;
    const int budget = kEvict ? a.budget[b] : 0;
    int bad = n < 0 || n > a.n_max || budget < 0;
    const int pages = bad ? 0 : pages_of(d, n);
    for (int j = threadIdx.x; j < pages; j += kThreads) {
        const int page = table[j];
        bad |= !in_pool(d, page) || a.cache.refs[page] < 1;
        old[j] = page;
        rank[j] = -1;
    }
    bad = __syncthreads_or(bad);
    if (bad) {
        if (threadIdx.x == 0) {
            atomicOr(a.faults, kFaultCache);
            a.w.need[b] = 0;
            a.w.rows[b] = -1;
            a.w.moves[b] = 0;
        }
        return;
    }
    const float* u = a.cache.u + (size_t)b * d.cap;
    const int32_t* pos = a.cache.pos + (size_t)b * d.cap;
    const uint8_t* keep = kEvict ? nullptr : a.keep + (size_t)b * d.cap;
    uint64_t least = 0;  // rows with a key of at least this stay
    if constexpr (kEvict) {
        if (budget > 0 && budget < n) least = nth_key(u, pos, n, budget, hist, lds);
    }
    auto stays = [&](int i) __attribute__((always_inline)) {
        if constexpr (kEvict) return budget > 0 && rank_key(u[i], pos[i]) >= least;
        return keep[i] != 0;
    };
    int mine = 0, kept;
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const bool s = stays(i);
        mine += s;
        if (kEvict && a.keep_out) a.keep_out[(size_t)b * d.cap + i] = s;
    }
    (void)block_scan(mine, &kept, lds);
    // kept rows behind the new end, ascending; pages with a hole that others use too
    int32_t* from = a.w.from + rows0;
    int count = 0;
    for (int i0 = 0; i0 < n; i0 += kThreads) {
        const int i = i0 + (int)threadIdx.x;
        const bool s = i < n && stays(i);
        const bool move = s && i >= kept;
        if (i < kept && !s && a.cache.refs[old[i >> d.page_shift]] > 1) rank[i >> d.page_shift] = 0;
        int sum;
        const int at = block_scan(move, &sum, lds);
        if (move) from[count + at] = i;
        count += sum;
    }
    // the shared ones numbered
    int need = 0;
    const int end = pages_of(d, kept);
    for (int j0 = 0; j0 < end; j0 += kThreads) {
        const int j = j0 + (int)threadIdx.x;
        const bool copy = j < end && rank[j] == 0;
        int sum;
        const int at = block_scan(copy, &sum, lds);
        if (copy) rank[j] = need + at;
        need += sum;
    }
    __syncthreads();
    // the rows written: a hole takes the next of `from`, a kept row of a replaced page itself
    int32_t* dst = a.w.dst + rows0;
    int32_t* src = a.w.src + rows0;
    int moves = 0, holes = 0;
    for (int i0 = 0; i0 < kept; i0 += kThreads) {
        const int i = i0 + (int)threadIdx.x;
        const bool s = i < kept && stays(i);
        const bool hole = i < kept && !s;
        const bool write = hole || (s && rank[i >> d.page_shift] >= 0);
        int sum;
        const int at = block_scan((int)write | (int)hole << 16, &sum, lds);  // (at most 1,024 of each)
        if (write) {
            dst[moves + (at & 0xffff)] = i;
            src[moves + (at & 0xffff)] = hole ? from[holes + (at >> 16)] : i;
        }
        moves += sum & 0xffff;
        holes += sum >> 16;
    }
    if (threadIdx.x == 0) {
        a.w.need[b] = need;
        a.w.rows[b] = kept;
        a.w.moves[b] = moves;
    }
}

__global__ __launch_bounds__(kThreads) void q4_grant_kernel(Q4PageArgs a) {
    __shared__ int lds[kWaves + 1];
    grant(a, lds);
}

// Workgroup (b, layer, KV head): the rows of one slab; the first one of a sequence also changes its state.
__global__ __launch_bounds__(kMoveThreads) void q4_move_kernel(Q4PageArgs a) {
    const Q4Dims& d = a.dims;
    const int slabs = d.layers * d.hkv;
    const int b = blockIdx.x / slabs, slab = blockIdx.x % slabs;
    const int layer = slab / d.hkv, g = slab % d.hkv;
    const int kept = a.w.rows[b], offset = a.w.offset[b];
    if (kept < 0 || offset < 0) return;
    const int moves = a.w.moves[b];
    const int32_t* dst = a.w.dst + (size_t)b * a.n_max;
    const int32_t* src = a.w.src + (size_t)b * a.n_max;
    const int32_t* rank = a.w.rank + (size_t)b * d.max_pages;
    const int32_t* old = a.w.old_table + (size_t)b * d.max_pages;
    auto page_from = [&](int row) __attribute__((always_inline)) { return old[row >> d.page_shift]; };
    auto page_to = [&](int row) __attribute__((always_inline)) {
        const int r = rank[row >> d.page_shift];
        return r < 0 ? old[row >> d.page_shift] : a.w.fresh[offset + r];
    };
    const int pieces = d.d / 32;  // 16-byte pieces of a row's codes
    const int per = 2 * pieces + 2, in = d.page_rows - 1;
    for (int i = threadIdx.x; i < moves * per; i += kMoveThreads) {
        const int m = i / per, j = i % per;
        const int to = dst[m], from = src[m];
        const uint8_t* s = a.cache.pool + q4_record(d, layer, page_from(from), g);
        uint8_t* t = a.cache.pool + q4_record(d, layer, page_to(to), g);
        if (j < 2 * pieces) {
            const int part = j < pieces ? 0 : d.vc_off, at = j % pieces * 16;
            *reinterpret_cast<u32x4*>(t + part + (to & in) * (d.d / 2) + at) =
                *reinterpret_cast<const u32x4*>(s + part + (from & in) * (d.d / 2) + at);
        } else {
            const int part = j == 2 * pieces ? d.ks_off : d.vs_off;
            if (d.d == 128)
                reinterpret_cast<uint32_t*>(t + part)[to & in] = reinterpret_cast<const uint32_t*>(s + part)[from & in];
            else
                reinterpret_cast<uint16_t*>(t + part)[to & in] = reinterpret_cast<const uint16_t*>(s + part)[from & in];
        }
    }
    if (slab != 0) return;
    for (int m = threadIdx.x; m < moves; m += kMoveThreads) {
        const int to = dst[m], from = src[m];
        if (to == from) continue;
        if (a.cache.u) a.cache.u[(size_t)b * d.cap + to] = a.cache.u[(size_t)b * d.cap + from];
        if (a.cache.pos) a.cache.pos[(size_t)b * d.cap + to] = a.cache.pos[(size_t)b * d.cap + from];
    }
    const int end = pages_of(d, kept), had = pages_of(d, a.cache.len[b]);
    int32_t* table = a.cache.table + (size_t)b * d.max_pages;
    uint32_t fault = 0;
    for (int j = threadIdx.x; j < had; j += kMoveThreads) {
        const bool copied = j < end && rank[j] >= 0;
        if (j < end && !copied) continue;
        fault |= release(a, old[j]);
        const int page = copied ? a.w.fresh[offset + rank[j]] : -1;
        table[j] = page;
        if (copied) a.cache.refs[page] = 1;
    }
    if (fault) atomicOr(a.faults, fault);
    __syncthreads();  // (every thread has read the length)
    if (threadIdx.x == 0) a.cache.len[b] = kept;
}

}  // namespace

hipError_t launch_q4_reserve(const Q4PageArgs& a, hipStream_t s) {
    hipLaunchKernelGGL(q4_reserve_plan_kernel, dim3(1), dim3(kThreads), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(q4_reserve_kernel, dim3((uint32_t)a.dims.batch * a.dims.layers), dim3(kMoveThreads), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_q4_fork(const Q4PageArgs& a, hipStream_t s) {
    hipLaunchKernelGGL(q4_fork_kernel, dim3(a.count), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_q4_free(const Q4PageArgs& a, hipStream_t s) {
    hipLaunchKernelGGL(q4_free_kernel, dim3(a.count), dim3(kMoveThreads), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_q4_compact(const Q4PageArgs& a, hipStream_t s) {
    hipLaunchKernelGGL((a.budget ? q4_compact_plan_kernel<true> : q4_compact_plan_kernel<false>), dim3(a.dims.batch),
                       dim3(kThreads), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(q4_grant_kernel, dim3(1), dim3(kThreads), 0, s, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    hipLaunchKernelGGL(q4_move_kernel, dim3((uint32_t)a.dims.batch * a.dims.layers * a.dims.hkv), dim3(kMoveThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace ikv
