// Pages of the 4-bit cache: reserving rows (with copy on write), forking, freeing and compacting sequences.
//
// The state is the table, the lengths and one reference count per page; a page is free when its count is 0.  Free pages are
// taken in ascending order, for the sequences in their order, from the counts as they were before the call, so a call's
// result depends on nothing but its inputs.  Counts change by integer atomics (an order does not matter).
//
// A call that allocates runs in launches on the caller's stream: what each sequence needs, the pages for it (one workgroup),
// and the change itself, spread over sequences and layers.  The last one reads what the others wrote in the scratch, never
// the table or the lengths that its own workgroups change.
#include <type_traits>

#include "kv_common.h"
#include "q4.h"

namespace ikv {
namespace {

constexpr int kThreads = 1024;  // workgroups that scan
constexpr int kWaves = kThreads / kWave;
constexpr int kMoveThreads = 256;

// Exclusive prefix sum over the workgroup's threads; *total gets the sum.  Every thread calls it.
template <int kWaves = kThreads / kWave>
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

// `rows` rows of a record, from one to another, by the whole workgroup.
__device__ __forceinline__ void copy_rows(const Q4Dims& d, const uint8_t* s, uint8_t* t, int rows) {
    const int pieces = rows * (d.d / 2) / 16, halves = rows * (d.d / 32) / 2;  // of a part: 16 bytes of codes, 2 of scales
    for (int i = threadIdx.x; i < 2 * (pieces + halves); i += blockDim.x) {
        if (i < 2 * pieces) {
            const int at = i < pieces ? i * 16 : d.vc_off + (i - pieces) * 16;
            *reinterpret_cast<u32x4*>(t + at) = *reinterpret_cast<const u32x4*>(s + at);
        } else {
            const int j = i - 2 * pieces, at = j < halves ? d.ks_off + j * 2 : d.vs_off + (j - halves) * 2;
            *reinterpret_cast<uint16_t*>(t + at) = *reinterpret_cast<const uint16_t*>(s + at);
        }
    }
}

// Workgroup (KV head, layer, b): the copy on write of one record; the first of a sequence also changes its state.
__global__ __launch_bounds__(kMoveThreads) void q4_reserve_kernel(Q4PageArgs a) {
    const Q4Dims& d = a.dims;
    const int b = blockIdx.z, layer = blockIdx.y, g = blockIdx.x;
    const bool leader = layer == 0 && g == 0;
    const int offset = a.w.offset[b], need = a.w.need[b], source = a.w.source[b];
    const int rows = offset < 0 ? 0 : a.w.rows[b];
    if (leader && a.granted && threadIdx.x == 0) a.granted[b] = rows;
    if (rows == 0) return;
    if (source >= 0)
        copy_rows(d, a.cache.pool + q4_record(d, layer, source, g), a.cache.pool + q4_record(d, layer, a.w.fresh[offset], g),
                  a.w.moves[b]);
    if (!leader) return;
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

// The rows of a thread, `per` consecutive ones, their keys in registers (up to R of them) or read again (R = 0).
template <int R, int kBlock>
struct Rows {
    const float* u;
    const int32_t* pos;
    int n, per, first;
    uint64_t key[R > 0 ? R : 1];
    __device__ __forceinline__ Rows(const float* u_, const int32_t* pos_, int n_)
        : u(u_), pos(pos_), n(n_), per((n_ + kBlock - 1) / kBlock), first((int)threadIdx.x * per) {
        if constexpr (R > 0)
#pragma unroll
            for (int j = 0; j < R; ++j) key[j] = j < per && first + j < n ? rank_key(u[first + j], pos[first + j]) : 0;
    }
    template <typename F>
    __device__ __forceinline__ void each(F f) const {  // f(place, key, exists); every thread makes as many calls
        if constexpr (R > 0) {
#pragma unroll
            for (int j = 0; j < R; ++j)
                if (j < per) f(j, key[j], first + j < n);
        } else {
            for (int j = 0; j < per; ++j) {
                const int i = first + j;
                f(j, i < n ? rank_key(u[i], pos[i]) : 0, i < n);
            }
        }
    }
};

// The smallest key above `last`, over the workgroup.
template <int R, int kBlock>
__device__ uint64_t next_key(const Rows<R, kBlock>& rows, uint64_t last, uint64_t* lds /* waves */) {
    uint64_t best = ~0ull;
    rows.each([&](int, uint64_t key, bool exists) __attribute__((always_inline)) {
        if (exists && key > last && key < best) best = key;
    });
#pragma unroll
    for (int o = kWave / 2; o >= 1; o >>= 1) {
        const uint64_t y = __shfl_xor((unsigned long long)best, o, kWave);
        best = y < best ? y : best;
    }
    __syncthreads();
    if (threadIdx.x % kWave == 0) lds[threadIdx.x / kWave] = best;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kBlock / kWave; ++w) best = lds[w] < best ? lds[w] : best;
    return best;
}

// The `budget`-th largest key of n > budget >= 1 rows: radix selection from the highest byte, each pass a histogram of the
// rows that share the bytes chosen so far, until a byte's rows all stay.  Every thread gets it.
template <int R, int kBlock>
__device__ uint64_t nth_key(const Rows<R, kBlock>& rows, int budget, int* hist /* 256 */, int* lds) {
    __shared__ uint64_t chosen;
    __shared__ int left_s, done_s;
    uint64_t prefix = 0, mask = 0;
    int left = budget;
    for (int shift = 56; shift >= 0; shift -= 8) {
        if (threadIdx.x < 256) hist[threadIdx.x] = 0;
        __syncthreads();
        rows.each([&](int, uint64_t key, bool exists) __attribute__((always_inline)) {
            if (!exists || (key & mask) != prefix) return;
            // utilities share their leading bits: a wave whose rows agree counts once
            const int digit = (int)(key >> shift) & 255;
            const int first = __builtin_amdgcn_readfirstlane(digit);
            const uint64_t live = __ballot(1);
            if (__ballot(digit == first) == live) {
                if ((int)(threadIdx.x % kWave) == __ffsll((unsigned long long)live) - 1) atomicAdd(&hist[first], __popcll(live));
            } else {
                atomicAdd(&hist[digit], 1);
            }
        });
        __syncthreads();
        // the byte that holds the left-th row from the top: threads 0 .. 255 hold the digits from 255 down
        const int digit = 255 - (int)threadIdx.x;
        const int c = threadIdx.x < 256 ? hist[digit] : 0;
        int total;
        const int above = block_scan<kBlock / kWave>(c, &total, lds);
        if (threadIdx.x < 256 && above < left && above + c >= left) {
            chosen = prefix | (uint64_t)digit << shift;
            left_s = left - above;
            done_s = c == left - above;
        }
        __syncthreads();
        prefix = chosen;
        left = left_s;
        mask |= (uint64_t)255 << shift;
        if (done_s) break;  // every row that shares these bytes stays
    }
    return prefix;
}

// Workgroup b: what sequence b keeps, the rows that are written (holes, and every kept row of a shared page with a hole),
// and the pages wanted.  Threads hold consecutive rows, so that one prefix sum of the kept rows, K(i) of them before row i,
// numbers everything: a dropped row i before the new end is hole i - K(i), a kept row behind it the (K(i) - K(end))-th that moves.
constexpr int kFewEvicted = 4;  // so few are found one after the other
template <bool kEvict, int R, int kBlock>
__global__ __launch_bounds__(kBlock) void q4_compact_plan_kernel(Q4PageArgs a) {
    constexpr int kWaves = kBlock / kWave;
    __shared__ int lds[kWaves + 1];
    __shared__ uint64_t lds64[kWaves];
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
    const Rows<kEvict ? R : 0, kBlock> rows(a.cache.u + (size_t)b * d.cap, a.cache.pos + (size_t)b * d.cap, bad ? 0 : n);
    // (rank: -1 for a page of the sequence's own, -2 for a shared one, until the shared ones with a hole are numbered)
    for (int j = threadIdx.x; j < pages; j += kBlock) {
        const int page = table[j];
        const int refs = in_pool(d, page) ? a.cache.refs[page] : 0;
        bad |= refs < 1;
        old[j] = page;
        rank[j] = refs > 1 ? -2 : -1;
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
    // the rows that stay, a bit each (R = 0: asked again)
    const uint8_t* keep = kEvict ? nullptr : a.keep + (size_t)b * d.cap;
    const int per = rows.per, first = rows.first;
    uint64_t least = 0;  // evict: rows with a key of at least this stay
    uint32_t bits = 0;
    int mine = 0;
    if constexpr (kEvict) {
        if (budget > 0 && budget < n) {
            if (n - budget <= kFewEvicted) {
                for (int i = 0; i < n - budget; ++i) least = next_key(rows, i ? least : 0, lds64);
                ++least;
            } else {
                least = nth_key(rows, budget, hist, lds);
            }
        }
        rows.each([&](int j, uint64_t key, bool exists) __attribute__((always_inline)) {
            const bool s = exists && budget > 0 && key >= least;
            mine += s;
            if (R > 0) bits |= (uint32_t)s << j;
            if (a.keep_out && exists) a.keep_out[(size_t)b * d.cap + first + j] = s;
        });
    } else {
        for (int j = 0; j < per && first + j < n; ++j) {
            const bool s = keep[first + j] != 0;
            mine += s;
            if (R > 0) bits |= (uint32_t)s << j;
        }
    }
    auto stays = [&](int i) __attribute__((always_inline)) {
        if constexpr (R > 0) return (bits >> (i - first) & 1u) != 0;
        else if constexpr (kEvict) return budget > 0 && rank_key(rows.u[i], rows.pos[i]) >= least;
        else return keep[i] != 0;
    };
    int kept;
    const int before = block_scan<kWaves>(mine, &kept, lds);
    const int stop = min(n, first + per), stop_in = min(stop, kept);
    // kept rows before the new end; shared pages with a hole there
    int inside = 0, marked = -1;
    for (int i = first; i < stop_in; ++i) {
        const bool s = stays(i);
        inside += s;
        const int j = i >> d.page_shift;
        if (!s && j != marked) {
            marked = j;
            if (rank[j] != -1) rank[j] = 0;
        }
    }
    int in_place;
    (void)block_scan<kWaves>(inside, &in_place, lds);
    // kept rows behind the new end
    int32_t* from = a.w.from + rows0;
    if (stop > kept) {
        int k = before - in_place;
        for (int i = first; i < stop; ++i) {
            const bool s = stays(i);
            if (s && i >= kept) from[k] = i;
            k += s;
        }
    }
    // the shared pages with a hole numbered, the others left as they are
    int need = 0;
    const int end = pages_of(d, kept);
    for (int j0 = 0; j0 < end; j0 += kBlock) {
        const int j = j0 + (int)threadIdx.x;
        const bool copy = j < end && rank[j] == 0;
        int sum;
        const int at = block_scan<kWaves>(copy, &sum, lds);
        if (j < end) rank[j] = copy ? need + at : -1;
        need += sum;
    }
    // the rows written: a hole (-1 - its number, for its one of `from`), a kept row of a replaced page
    int count = 0, moves, page = -1;
    bool replaced = false;
    auto written = [&](int i, bool s) __attribute__((always_inline)) {
        const int j = i >> d.page_shift;
        if (need > 0 && j != page) {
            page = j;
            replaced = rank[j] >= 0;
        }
        return !s || replaced;
    };
    __syncthreads();
    for (int i = first; i < stop_in; ++i) count += written(i, stays(i));
    int at = block_scan<kWaves>(count, &moves, lds);
    int32_t* dst = a.w.dst + rows0;
    int32_t* src = a.w.src + rows0;
    for (int i = first, k = before; i < stop_in; ++i) {
        const bool s = stays(i);
        if (written(i, s)) {
            dst[at] = i;
            src[at++] = s ? i : -1 - (i - k);
        }
        k += s;
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

// Workgroup (part, layer, b): every parts-th kEntries of the sequence's rows, in one layer; the first of a sequence also changes
// its state.  The rows' places are found once for all KV heads; four copies of a thread are in flight together.
constexpr int kEntries = 32;
template <int D>
__global__ __launch_bounds__(kMoveThreads) void q4_move_kernel(Q4PageArgs a) {
    constexpr int kPieces = D / 32, kTogether = 4;  // 16-byte pieces of a row's codes; copies at a time
    typedef typename std::conditional<D == 128, uint32_t, uint16_t>::type scales_t;  // a row's scales
    __shared__ uint32_t place[2][kEntries];         // page * page_rows + row in the page: from, to
    const Q4Dims& d = a.dims;
    const int b = blockIdx.z, layer = blockIdx.y, part = blockIdx.x;
    const int kept = a.w.rows[b], offset = a.w.offset[b];
    if (kept < 0 || offset < 0) return;
    const int moves = a.w.moves[b];
    const int32_t* dst = a.w.dst + (size_t)b * a.n_max;
    const int32_t* src = a.w.src + (size_t)b * a.n_max;
    const int32_t* holes = a.w.from + (size_t)b * a.n_max;
    const int32_t* rank = a.w.rank + (size_t)b * d.max_pages;
    const int32_t* old = a.w.old_table + (size_t)b * d.max_pages;
    auto source = [&](int m) __attribute__((always_inline)) {
        const int r = src[m];
        return r < 0 ? holes[-1 - r] : r;
    };
    const int in = d.page_rows - 1;
    const size_t layer0 = q4_record(d, layer, 0, 0);
    for (int m0 = part * kEntries; m0 < moves; m0 += gridDim.x * kEntries) {
        const int entries = min(kEntries, moves - m0);
        __syncthreads();  // (the places before these are no longer read)
        if ((int)threadIdx.x < 2 * entries) {
            const int which = threadIdx.x & 1, m = threadIdx.x >> 1;
            const int row = which ? dst[m0 + m] : source(m0 + m);
            int page = old[row >> d.page_shift];
            if (which) {
                const int r = rank[row >> d.page_shift];
                if (r >= 0) page = a.w.fresh[offset + r];
            }
            place[which][m] = ((uint32_t)page << d.page_shift) + (row & in);
        }
        __syncthreads();
        auto record = [&](int which, int m, int g, int* row) __attribute__((always_inline)) {
            const uint32_t p = place[which][m];
            *row = p & in;
            return a.cache.pool + layer0 + ((size_t)(p >> d.page_shift) * d.hkv + g) * d.rec;
        };
        const int copies = entries * d.hkv * 2 * kPieces;  // pieces fastest, then entries, then heads
        for (int i0 = threadIdx.x; i0 < copies; i0 += kMoveThreads * kTogether) {
            u32x4 x[kTogether];
            u32x4* to[kTogether];
#pragma unroll
            for (int k = 0; k < kTogether; ++k) {
                const int i = min(i0 + k * kMoveThreads, copies - 1);
                const int j = i % (2 * kPieces), e = i / (2 * kPieces), m = e % entries, g = e / entries;
                const int at = (j < kPieces ? 0 : d.vc_off) + j % kPieces * 16;
                int fr, tr;
                const uint8_t* s = record(0, m, g, &fr);
                uint8_t* t = record(1, m, g, &tr);
                x[k] = *reinterpret_cast<const u32x4*>(s + at + fr * (D / 2));
                to[k] = reinterpret_cast<u32x4*>(t + at + tr * (D / 2));
            }
#pragma unroll
            for (int k = 0; k < kTogether; ++k)
                if (i0 + k * kMoveThreads < copies) *to[k] = x[k];
        }
        for (int i = threadIdx.x; i < entries * d.hkv * 2; i += kMoveThreads) {
            const int at = i & 1 ? d.vs_off : d.ks_off, e = i >> 1, m = e % entries, g = e / entries;
            int fr, tr;
            const uint8_t* s = record(0, m, g, &fr);
            uint8_t* t = record(1, m, g, &tr);
            reinterpret_cast<scales_t*>(t + at)[tr] = reinterpret_cast<const scales_t*>(s + at)[fr];
        }
    }
    if (layer != 0 || part != 0) return;
    for (int m = threadIdx.x; m < moves; m += kMoveThreads) {
        const int to = dst[m], from = source(m);
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
    hipLaunchKernelGGL(q4_reserve_kernel, dim3(a.dims.hkv, a.dims.layers, a.dims.batch), dim3(kMoveThreads), 0, s, a);
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

namespace {
template <bool kEvict>
void launch_plan(const Q4PageArgs& a, hipStream_t s) {
    // threads, and rows of each in registers, by the longest sequence
    const auto launch = [&](auto kern, int threads) { hipLaunchKernelGGL(kern, dim3(a.dims.batch), dim3(threads), 0, s, a); };
    if (a.n_max <= 4 * 256) launch(q4_compact_plan_kernel<kEvict, 4, 256>, 256);
    else if (a.n_max <= 4 * kThreads) launch(q4_compact_plan_kernel<kEvict, 4, kThreads>, kThreads);
    else if (a.n_max <= 32 * kThreads) launch(q4_compact_plan_kernel<kEvict, 32, kThreads>, kThreads);
    else launch(q4_compact_plan_kernel<kEvict, 0, kThreads>, kThreads);
}
}  // namespace

hipError_t launch_q4_compact(const Q4PageArgs& a, hipStream_t s) {
    if (a.budget) launch_plan<true>(a, s);
    else launch_plan<false>(a, s);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(q4_grant_kernel, dim3(1), dim3(kThreads), 0, s, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    // parts of a sequence's rows: eight workgroups per CU in all, no more than there can be entries for
    const int slabs = a.dims.layers * a.dims.batch, most = (a.n_max + kEntries - 1) / kEntries;
    const int want = (8 * 256 + slabs - 1) / slabs, parts = want < most ? want : most;
    const dim3 grid(parts, a.dims.layers, a.dims.batch);
    if (a.dims.d == 128) hipLaunchKernelGGL(q4_move_kernel<128>, grid, dim3(kMoveThreads), 0, s, a);
    else hipLaunchKernelGGL(q4_move_kernel<64>, grid, dim3(kMoveThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace ikv
