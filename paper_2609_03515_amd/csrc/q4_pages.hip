// Pages of the 4-bit cache: reserving rows (with copy on write), forking, freeing and compacting sequences.
//
// The state is the table, the lengths and one reference count per page; a page is free when its count is 0.  Free pages are
// taken in ascending order, for the sequences in their order, from the counts as they were before the call, so a call's
// result depends on nothing but its inputs.  Counts change by integer atomics (an order does not matter).
//
// A call that allocates runs in launches on the caller's stream: what each sequence needs, the pages for it (one workgroup),
// and the change itself, spread over sequences and layers.  The last one reads what the others wrote in the scratch, never
// the table or the lengths that its own workgroups change.
//
// Small calls are launches and chains of dependent loads (2.5 to 8 us a kernel); measured on six samples of prompts of 12,000 to
// 16,384 rows in 8 layers of 8 KV heads: fork 5.4 us, reserve 6.5 + 8.5, eviction to 10%: plan 21.6, pages 5, moves 45 (81 MB
// written by the memory's counter and as much read, in pieces of 64 and 4 bytes: 3.6 TB/s).  The moves took 112 with one workgroup per slab that found every
// row's place for itself, and 48 (one row of each of 256 slabs: 14.7, now 11.3) with the places found between the copies; the plan 45 with a
// prefix sum per 1,024 rows (64 with keys in registers: that unrolls into more code than its instruction fetches are worth), and 28
// with one histogram and with pointers that could be LDS or memory; the fork 10.4 copying 4 bytes a thread.
#include <limits.h>

#include <atomic>
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

__device__ __forceinline__ bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

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
        auto take = [&](float y) __attribute__((always_inline)) { x = a.init_mode == 1 ? x + y : fmin(x, (double)y); };
        if (a.init_mode != 0) {
            const int quads = aligned16(u) ? len / 4 : 0;
#pragma unroll 8
            for (int i = threadIdx.x; i < quads; i += kMoveThreads) {
                const f32x4 y = reinterpret_cast<const f32x4*>(u)[i];
#pragma unroll
                for (int k = 0; k < 4; ++k) take(y[k]);
            }
#pragma unroll 4
            for (int i = quads * 4 + threadIdx.x; i < len; i += kMoveThreads) take(u[i]);
        }
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

// n words (of a slot's utilities or positions) from one place to another, by the whole workgroup: 16 bytes a thread where they are
// aligned (slots are then too), four loads of a thread together.
__device__ __forceinline__ void copy_words(const uint32_t* from, uint32_t* to, int n) {
    constexpr int kTogether = 4;
    const int quads = aligned16(from) && aligned16(to) ? n / 4 : 0;
    for (int j0 = threadIdx.x; j0 < quads; j0 += kThreads * kTogether) {
        u32x4 x[kTogether];
#pragma unroll
        for (int k = 0; k < kTogether; ++k) x[k] = reinterpret_cast<const u32x4*>(from)[min(j0 + k * kThreads, quads - 1)];
#pragma unroll
        for (int k = 0; k < kTogether; ++k)
            if (j0 + k * kThreads < quads) reinterpret_cast<u32x4*>(to)[j0 + k * kThreads] = x[k];
    }
#pragma unroll 4
    for (int j = quads * 4 + threadIdx.x; j < n; j += kThreads) to[j] = from[j];
}

// Workgroup i: sequence dst[i] becomes a copy of src[i] that shares its pages.  Refused, and reported: a slot out of range, a
// destination that is not empty or is named twice (after the first time), a source that is a destination of the call.
__global__ __launch_bounds__(kThreads) void q4_fork_kernel(Q4PageArgs a) {
    __shared__ int bad_call, bad_state;  // (two: a wave may be at the second check while another still reads the first's)
    const Q4Dims& d = a.dims;
    const int i = blockIdx.x, src = a.src_slot[i], dst = a.dst_slot[i];
    if (threadIdx.x == 0) bad_call = bad_state = 0;
    __syncthreads();
    const bool range = (uint32_t)src < (uint32_t)d.batch && (uint32_t)dst < (uint32_t)d.batch;
    int mine = !range;
    for (int j = threadIdx.x; j < a.count; j += kThreads) {
        const int other = a.dst_slot[j];
        mine |= other == src || (j < i && other == dst);
    }
    if (mine) bad_call = 1;
    __syncthreads();
    if (bad_call) {  // (before dst's state is read: another workgroup may be writing it)
        if (threadIdx.x == 0) atomicOr(a.faults, kFaultCache);
        return;
    }
    const int len = a.cache.len[src];
    const bool fits = len >= 0 && len <= d.cap && a.cache.len[dst] == 0;
    const int pages = fits ? pages_of(d, len) : 0;
    const int32_t* st = a.cache.table + (size_t)src * d.max_pages;
    mine = !fits;
    for (int j = threadIdx.x; j < pages; j += kThreads) mine |= !in_pool(d, st[j]);
    if (mine) bad_state = 1;
    __syncthreads();
    if (bad_state) {
        if (threadIdx.x == 0) atomicOr(a.faults, kFaultCache);
        return;
    }
    int32_t* dt = a.cache.table + (size_t)dst * d.max_pages;
    for (int j = threadIdx.x; j < d.max_pages; j += kThreads) {
        const int page = j < pages ? st[j] : -1;
        dt[j] = page;
        if (j < pages) atomicAdd(&a.cache.refs[page], 1);
    }
    const size_t from = (size_t)src * d.cap, to = (size_t)dst * d.cap;
    if (a.cache.u) copy_words(reinterpret_cast<const uint32_t*>(a.cache.u) + from, reinterpret_cast<uint32_t*>(a.cache.u) + to, len);
    if (a.cache.pos) copy_words(reinterpret_cast<const uint32_t*>(a.cache.pos) + from, reinterpret_cast<uint32_t*>(a.cache.pos) + to, len);
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

typedef __attribute__((address_space(3))) uint32_t* lds_words;
typedef __attribute__((address_space(3))) uint64_t* lds_masks;

// Eviction order as one number, larger stays: the utility's key (0 and -0 alike), then (the lower position first) the position
// turned round.  Of rows that agree in both, which a caller that sets no positions may have, the lower row stays.
// The rows of a sequence that a selection looks at (kInLds: their utilities' keys are in LDS).
template <bool kInLds>
struct Ranked {
    const float* u;
    const int32_t* pos;
    lds_words keys;
    int n;
    __device__ __forceinline__ uint32_t key_of(int i) const { return float_key(u[i] + 0.0f); }
    __device__ __forceinline__ uint32_t key(int i) const {
        if constexpr (kInLds) return keys[i];
        else return key_of(i);
    }
    __device__ __forceinline__ uint32_t turned(int i) const { return (uint32_t)pos[i] ^ 0x7fffffffu; }
    __device__ __forceinline__ uint64_t full(int i) const { return (uint64_t)key(i) << 32 | turned(i); }
};
// Where a selection ends: rows with a larger full key stay, and of those with this one the rows before `limit`.
struct Border {
    uint64_t full;
    int limit;
};

// The row that leaves next after those of `last`: the smallest full key, and of equal ones the last row.
template <int kBlock, bool kInLds>
__device__ Border next_border(const Ranked<kInLds>& rows, Border last, uint64_t* lds64, int* lds /* waves */) {
    uint64_t best = ~0ull;
    int row = -1;
#pragma unroll 4
    for (int i = threadIdx.x; i < rows.n; i += kBlock) {
        const uint64_t key = rows.full(i);
        const bool left = key > last.full || (key == last.full && i < last.limit);
        if (left && (key < best || (key == best && i > row))) {
            best = key;
            row = i;
        }
    }
    auto take = [&](uint64_t key, int i) __attribute__((always_inline)) {
        if (key < best || (key == best && i > row)) {
            best = key;
            row = i;
        }
    };
#pragma unroll
    for (int o = kWave / 2; o >= 1; o >>= 1) {
        const uint64_t key = __shfl_xor((unsigned long long)best, o, kWave);
        take(key, __shfl_xor(row, o, kWave));
    }
    __syncthreads();
    if (threadIdx.x % kWave == 0) {
        lds64[threadIdx.x / kWave] = best;
        lds[threadIdx.x / kWave] = row;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kBlock / kWave; ++w) take(lds64[w], lds[w]);
    return {best, row};
}

// The border of the `budget` best of n > budget >= 1 rows, its full key the budget-th largest or a lower one with as many rows
// at least as large: radix selection from the highest byte, each pass a histogram of the rows that share the bytes chosen so
// far, until a byte's rows all stay.  Positions are looked at only where utilities tie across the border, and rows counted only
// where positions do as well.  Every thread gets it.  Utilities share their leading bits, and additions to one LDS word go one
// by one: kHists histograms, by lane.
template <int kBlock>
constexpr int kHistsOf = kBlock / 64;  // (16, or 4 where there are fewer threads to clear and add them)
template <int kBlock, bool kInLds>
__device__ Border nth_border(const Ranked<kInLds>& rows, int budget, int* hist /* 256 * kHists */, int* lds) {
    constexpr int kHists = kHistsOf<kBlock>;
    __shared__ uint32_t digit_s;
    __shared__ int left_s, done_s, limit_s;
    uint32_t high = 0, low = 0, mask = 0;  // of utility and position: the bytes chosen, and which they are
    int left = budget;
    for (int pass = 0; pass < 8; ++pass) {
        const int shift = 24 - pass % 4 * 8;
        if (pass == 4) mask = 0;
        for (int i = threadIdx.x; i < 256 * kHists; i += kBlock) hist[i] = 0;
        __syncthreads();
        auto digit_of = [&](int i, int* digit) __attribute__((always_inline)) {  // and whether the row is still looked at
            uint32_t key = rows.key(i);
            bool in = (key & (pass < 4 ? mask : ~0u)) == high;
            if (pass >= 4 && in) {
                key = rows.turned(i);
                in = (key & mask) == low;
            }
            *digit = (int)(key >> shift) & 255;
            return in;
        };
#pragma unroll 4
        for (int i = threadIdx.x; i < rows.n; i += kBlock) {
            int digit;
            if (digit_of(i, &digit)) atomicAdd(&hist[digit * kHists + threadIdx.x % kHists], 1);
        }
        __syncthreads();
        // the byte that holds the left-th row from the top: threads 0 .. 255 hold the digits from 255 down
        const int digit = 255 - (int)threadIdx.x;
        int c = 0;
        if (threadIdx.x < 256)
#pragma unroll
            for (int k = 0; k < kHists; ++k) c += hist[digit * kHists + k];
        int total;
        const int above = block_scan<kBlock / kWave>(c, &total, lds);
        if (threadIdx.x < 256 && above < left && above + c >= left) {
            digit_s = (uint32_t)digit << shift;
            left_s = left - above;
            done_s = c == left - above;
        }
        __syncthreads();
        if (pass < 4) high |= digit_s;
        else low |= digit_s;
        left = left_s;
        mask |= 255u << shift;
        if (done_s) return {(uint64_t)high << 32 | low, INT_MAX};  // every row that shares these bytes stays
    }
    const uint64_t full = (uint64_t)high << 32 | low;
    for (int i0 = 0, seen = 0; seen < left; i0 += kBlock) {  // (more than `left` rows have this key)
        const int i = i0 + (int)threadIdx.x;
        const bool in = i < rows.n && rows.full(i) == full;
        int sum;
        const int at = seen + block_scan<kBlock / kWave>(in, &sum, lds);
        if (in && at == left - 1) limit_s = i + 1;
        seen += sum;
    }
    __syncthreads();
    return {full, limit_s};
}

// The same of at most kFewRows rows: every row counts those before it.
constexpr int kFewRows = 256;
template <bool kInLds>
__device__ Border border_of_few(const Ranked<kInLds>& rows, int budget, uint64_t* full /* kFewRows */) {
    __shared__ uint32_t key_s;
    __shared__ int last_s, all_s;
    const int i = threadIdx.x;
    const bool in = i < rows.n;
    uint64_t own = 0;
    if (in) full[i] = own = (uint64_t)rows.key(i) << 32;
    __syncthreads();
    int above = 0, alike = 0;
    if (in)
#pragma unroll 8
        for (int j = 0; j < rows.n; ++j) {
            above += full[j] > own;
            alike += full[j] == own;
        }
    if (in && above < budget && above + alike >= budget) {  // (rows of one utility)
        key_s = (uint32_t)(own >> 32);
        all_s = above + alike == budget;
    }
    __syncthreads();
    if (all_s) return {(uint64_t)key_s << 32, INT_MAX};
    if (in) full[i] = own = rows.full(i);
    __syncthreads();
    if (in) {
        int before = 0;
#pragma unroll 8
        for (int j = 0; j < rows.n; ++j) before += full[j] > own || (full[j] == own && j < i);
        if (before == budget - 1) last_s = i;
    }
    __syncthreads();
    return {full[last_s], last_s + 1};
}

// Workgroup b: what sequence b keeps, the rows that move, the shared pages that are replaced, and the pages wanted.
// With K(i) the kept rows before row i, from one mask bit a row and the masks' prefix sums: a dropped row i before the new end
// is hole i - K(i), a kept row behind it the (K(i) - K(end))-th that moves, and a page has a hole when its rows number more than
// K grows over it.
// So few are found one after the other: an eviction of 1, 2, 3, 4 rows of 8 x 3,277 takes 19, 22, 25 and 28 us, by radix passes 32 to
// 34 for any; they meet at 6 there, at 8 for 1,000 rows, and between 1 and 6 for 16,500 and more, as the utilities' bits have it.
constexpr int kFewEvicted = 4;
constexpr int kRowsInLds = 32768;  // masks, prefix sums and keys of so many rows lie in LDS (kInLds), of more in memory
template <bool kEvict, int kBlock, bool kInLds>
__global__ __launch_bounds__(kBlock) void q4_compact_plan_kernel(Q4PageArgs a) {
    constexpr int kWaves = kBlock / kWave;
    __shared__ int lds[kWaves + 1];
    __shared__ uint64_t lds64[kWaves];
    __shared__ int hist[kEvict ? 256 * kHistsOf<kBlock> : 1];
    __shared__ uint64_t few[kEvict ? kFewRows : 1];
    extern __shared__ uint64_t dynamic[];  // masks and their prefix sums, then the keys
    const Q4Dims& d = a.dims;
    const int b = blockIdx.x, n = a.cache.len[b], lane = threadIdx.x % kWave;
    const int32_t* table = a.cache.table + (size_t)b * d.max_pages;
    int32_t* rank = a.w.rank + (size_t)b * d.max_pages;
    int32_t* old = a.w.old_table + (size_t)b * d.max_pages;
    int32_t* replaced = a.w.replaced + (size_t)b * d.max_pages;
    const size_t words = ((size_t)a.n_max + 63) / 64;
    uint64_t* const mask_out = a.w.mask + b * words;
    auto* const mask = [&] {
        if constexpr (kInLds) return (lds_masks)dynamic;
        else return mask_out;
    }();
    auto* const prefix = [&] {
        if constexpr (kInLds) return (lds_words)(dynamic + words);
        else return a.w.prefix + b * words;
    }();
    const int budget = kEvict ? a.budget[b] : 0;
    int bad = n < 0 || n > a.n_max || budget < 0;
    const int pages = bad ? 0 : pages_of(d, n);
    const Ranked<kInLds> rows{a.cache.u + (size_t)b * d.cap, a.cache.pos + (size_t)b * d.cap,
                              (lds_words)(dynamic + words + (words + 1) / 2), bad ? 0 : n};
    const bool select = kEvict && budget > 0 && budget < n;
    if (kInLds && select)
#pragma unroll 4
        for (int i = threadIdx.x; i < rows.n; i += kBlock) rows.keys[i] = rows.key_of(i);
    for (int j = threadIdx.x; j < pages; j += kBlock) {
        const int page = table[j];
        const int refs = in_pool(d, page) ? a.cache.refs[page] : 0;
        bad |= refs < 1;
        old[j] = page;
        rank[j] = refs > 1 ? -2 : -1;  // (-2: shared, until those that are replaced are numbered)
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
    Border least{0, INT_MAX};
    if (select) {
        if (n <= kFewRows) {
            least = border_of_few(rows, budget, few);
        } else if (n - budget <= kFewEvicted) {
            for (int i = 0; i < n - budget; ++i) least = next_border<kBlock, kInLds>(rows, least, lds64, lds);
        } else {
            least = nth_border<kBlock, kInLds>(rows, budget, hist, lds);
        }
    }
    const uint32_t border = (uint32_t)(least.full >> 32), turned = (uint32_t)least.full;
    const bool all_equal = turned == 0 && least.limit == INT_MAX;  // (then no position has to be read)
    // a bit for every row that stays
    const uint8_t* keep = kEvict ? nullptr : a.keep + (size_t)b * d.cap;
    for (int i0 = 0; i0 < n; i0 += kBlock) {
        const int i = i0 + (int)threadIdx.x;
        bool s = false;
        if (i < n) {
            if constexpr (kEvict) {
                const uint32_t key = select ? rows.key(i) : 0;
                s = budget > 0 && key >= border;
                if (s && key == border && !all_equal) {
                    const uint32_t t = rows.turned(i);
                    s = t > turned || (t == turned && i < least.limit);
                }
                if (a.keep_out) a.keep_out[(size_t)b * d.cap + i] = s;
            } else {
                s = keep[i] != 0;
            }
        }
        const uint64_t m = __ballot(s);
        if (lane == 0 && i < n) {
            mask[i >> 6] = m;
            if (kInLds) mask_out[i >> 6] = m;
        }
    }
    __syncthreads();
    int kept = 0;
    for (int w0 = 0; w0 * 64 < n; w0 += kBlock) {
        const int w = w0 + (int)threadIdx.x;
        int sum;
        const int at = block_scan<kWaves>(w * 64 < n ? __popcll(mask[w]) : 0, &sum, lds);
        if (w * 64 < n) prefix[w] = kept + at;
        kept += sum;
    }
    __syncthreads();
    auto before = [&](int i) __attribute__((always_inline)) {  // K(i), i <= n
        return i >= n ? kept : prefix[i >> 6] + __popcll(mask[i >> 6] & ((1ull << (i & 63)) - 1));
    };
    // shared pages with a hole, numbered
    const int end = pages_of(d, kept), in_place = before(kept);
    int need = 0;
    if (in_place < kept)
        for (int j0 = 0; j0 < end; j0 += kBlock) {
            const int j = j0 + (int)threadIdx.x;
            bool copy = false;
            if (j < end) {
                const int from = j << d.page_shift, to = min(kept, from + d.page_rows);
                copy = rank[j] == -2 && before(to) - before(from) < to - from;
            }
            int sum;
            const int at = block_scan<kWaves>(copy, &sum, lds);
            if (j < end) rank[j] = copy ? need + at : -1;
            if (copy) replaced[need + at] = j;
            need += sum;
        }
    else
        for (int j = threadIdx.x; j < end; j += kBlock) rank[j] = -1;
    // holes, and the rows that fill them
    int32_t* dst = a.w.dst + (size_t)b * a.n_max;
    int32_t* src = a.w.src + (size_t)b * a.n_max;
    if (in_place < kept)
#pragma unroll 2
        for (int i = threadIdx.x; i < n; i += kBlock) {
            const uint64_t m = mask[i >> 6];
            const int k = prefix[i >> 6] + __popcll(m & ((1ull << (i & 63)) - 1));
            const bool s = m >> (i & 63) & 1u;
            if (i < kept ? !s : s) (i < kept ? dst : src)[i < kept ? i - k : k - in_place] = i;
        }
    if (threadIdx.x == 0) {
        a.w.need[b] = need;
        a.w.rows[b] = kept;
        a.w.moves[b] = kept - in_place;
    }
}

__global__ __launch_bounds__(kThreads) void q4_grant_kernel(Q4PageArgs a) {
    __shared__ int lds[kWaves + 1];
    grant(a, lds);
}

// What changes in a sequence's state: utilities and positions of the rows that move, table, counts and length.
__device__ void move_state(const Q4PageArgs& a, int b, int kept, int moves, int offset) {
    constexpr int kTogether = 4;
    const Q4Dims& d = a.dims;
    const int32_t* dst = a.w.dst + (size_t)b * a.n_max;
    const int32_t* src = a.w.src + (size_t)b * a.n_max;
    const int32_t* rank = a.w.rank + (size_t)b * d.max_pages;
    const int32_t* old = a.w.old_table + (size_t)b * d.max_pages;
    const int threads = (int)blockDim.x;
    for (int m0 = threadIdx.x; m0 < moves; m0 += threads * kTogether) {
        int to[kTogether];
        float u[kTogether];
        int32_t pos[kTogether];
#pragma unroll
        for (int k = 0; k < kTogether; ++k) {
            const int m = min(m0 + k * threads, moves - 1), from = src[m];
            to[k] = dst[m];
            if (a.cache.u) u[k] = a.cache.u[(size_t)b * d.cap + from];
            if (a.cache.pos) pos[k] = a.cache.pos[(size_t)b * d.cap + from];
        }
#pragma unroll
        for (int k = 0; k < kTogether; ++k) {
            if (m0 + k * threads >= moves) break;
            if (a.cache.u) a.cache.u[(size_t)b * d.cap + to[k]] = u[k];
            if (a.cache.pos) a.cache.pos[(size_t)b * d.cap + to[k]] = pos[k];
        }
    }
    const int end = pages_of(d, kept), had = pages_of(d, a.cache.len[b]);
    int32_t* table = a.cache.table + (size_t)b * d.max_pages;
    uint32_t fault = 0;
    for (int j = threadIdx.x; j < had; j += threads) {
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

// Workgroup (part, layer + 1, b): every parts-th kEntries of the sequence's entries, in one layer; (0, 0, b): the sequence's state.
// Entries are the holes, then the rows of the replaced pages (those that are holes, or behind the end, are none).  Their places,
// chains of loads, are found once for all KV heads by a wave of its own, one round ahead of the others' copies; four copies of a
// thread are in flight together.
constexpr int kEntries = 16, kMoveBlock = kMoveThreads + kWave;
template <int D>
__global__ __launch_bounds__(kMoveBlock) void q4_move_kernel(Q4PageArgs a) {
    constexpr int kPieces = D / 32, kTogether = 4;  // 16-byte pieces of a row's codes; copies at a time
    typedef typename std::conditional<D == 128, uint32_t, uint16_t>::type scales_t;  // a row's scales
    __shared__ uint32_t place_s[2][2][kEntries];    // of every other round: page * page_rows + row in the page: from, to
    __shared__ int entries_s[2];
    const Q4Dims& d = a.dims;
    const int b = blockIdx.z, layer = (int)blockIdx.y - 1, part = blockIdx.x;
    if (layer < 0 && part > 0) return;
    const int kept = a.w.rows[b], offset = a.w.offset[b];
    if (kept < 0 || offset < 0) return;
    const int moves = a.w.moves[b], all = moves + a.w.need[b] * d.page_rows;
    if (layer < 0) {
        move_state(a, b, kept, moves, offset);
        return;
    }
    const int32_t* dst = a.w.dst + (size_t)b * a.n_max;
    const int32_t* src = a.w.src + (size_t)b * a.n_max;
    const int32_t* rank = a.w.rank + (size_t)b * d.max_pages;
    const int32_t* old = a.w.old_table + (size_t)b * d.max_pages;
    const int32_t* replaced = a.w.replaced + (size_t)b * d.max_pages;
    const uint64_t* mask = a.w.mask + b * (((size_t)a.n_max + 63) / 64);
    const int in = d.page_rows - 1;
    const size_t layer0 = q4_record(d, layer, 0, 0);
    auto find = [&](int m0, int buf) __attribute__((always_inline)) {  // by one wave
        const int lane = threadIdx.x % kWave, m = m0 + lane;
        bool is = lane < kEntries && m < all;
        int from = 0, to = 0;
        if (is && m < moves) {
            from = src[m];
            to = dst[m];
        } else if (is) {
            from = to = (replaced[(m - moves) >> d.page_shift] << d.page_shift) + ((m - moves) & in);
            is = to < kept && (mask[to >> 6] >> (to & 63) & 1u);
        }
        const uint64_t live = __ballot(is);
        if (is) {
            const int r = rank[to >> d.page_shift];
            const int page = r >= 0 ? a.w.fresh[offset + r] : old[to >> d.page_shift];
            const int e = __popcll(live & ((1ull << lane) - 1));
            place_s[buf][0][e] = ((uint32_t)old[from >> d.page_shift] << d.page_shift) + (from & in);
            place_s[buf][1][e] = ((uint32_t)page << d.page_shift) + (to & in);
        }
        if (lane == 0) entries_s[buf] = __popcll(live);
    };
    const bool finder = threadIdx.x >= kMoveThreads;
    const int step = gridDim.x * kEntries;
    if (finder) find(part * kEntries, 0);
    int buf = 0;
    for (int m0 = part * kEntries; m0 < all; m0 += step, buf ^= 1) {
        __syncthreads();
        if (finder) {
            if (m0 + step < all) find(m0 + step, buf ^ 1);
            continue;
        }
        const uint32_t(&place)[2][kEntries] = place_s[buf];
        const int entries = entries_s[buf];
        auto record = [&](int which, int m, int g, int* row) __attribute__((always_inline)) {
            const uint32_t p = place[which][m];
            *row = p & in;
            return a.cache.pool + layer0 + ((size_t)(p >> d.page_shift) * d.hkv + g) * d.rec;
        };
        const int copies = entries * d.hkv * 2 * kPieces, scales = entries * d.hkv * 2;  // pieces fastest, then entries, heads
        auto scale_of = [&](int i, uint8_t** to) __attribute__((always_inline)) {
            const int at = i & 1 ? d.vs_off : d.ks_off, e = i >> 1, m = e % entries, g = e / entries;
            int fr, tr;
            const uint8_t* s = record(0, m, g, &fr);
            *to = record(1, m, g, &tr) + at + tr * sizeof(scales_t);
            return reinterpret_cast<const scales_t*>(s + at)[fr];
        };
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
            // the scales beside the first pieces (there are no more of them than pieces)
            const bool scale = i0 < scales;
            uint8_t* scale_to = nullptr;
            const scales_t y = scale ? scale_of(i0, &scale_to) : (scales_t)0;
#pragma unroll
            for (int k = 0; k < kTogether; ++k)
                if (i0 + k * kMoveThreads < copies) *to[k] = x[k];
            if (scale) *reinterpret_cast<scales_t*>(scale_to) = y;
        }
        for (int i = threadIdx.x + kMoveThreads; i < scales; i += kMoveThreads) {
            if ((i - (int)threadIdx.x) % (kMoveThreads * kTogether) == 0) continue;  // (written above)
            uint8_t* to;
            const scales_t y = scale_of(i, &to);
            *reinterpret_cast<scales_t*>(to) = y;
        }
    }
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
template <bool kEvict, int kBlock, bool kInLds>
hipError_t launch_plan(const Q4PageArgs& a, hipStream_t s) {
    auto kern = q4_compact_plan_kernel<kEvict, kBlock, kInLds>;
    const size_t words = ((size_t)a.n_max + 63) / 64;
    size_t lds = kInLds ? (words + (words + 1) / 2) * sizeof(uint64_t) : 0;
    if (kInLds && kEvict) lds += (size_t)a.n_max * sizeof(uint32_t);
    if (lds > 40 * 1024) {  // (beside the 16 KB of the histograms)
        constexpr int kMost = kRowsInLds * 4 + kRowsInLds / 64 * 12;
        static std::atomic<bool> raised[64];
        int dev = 0;
        if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) dev = -1;
        if (dev < 0 || !raised[dev].load(std::memory_order_acquire)) {
            const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, kMost);
            if (e != hipSuccess) return e;
            if (dev >= 0) raised[dev].store(true, std::memory_order_release);
        }
    }
    hipLaunchKernelGGL(kern, dim3(a.dims.batch), dim3(kBlock), lds, s, a);
    return hipGetLastError();
}
template <bool kEvict>
hipError_t launch_plan_by_rows(const Q4PageArgs& a, hipStream_t s) {
    // (short sequences: fewer waves to wait for at every step)
    if (a.n_max <= 1024) return launch_plan<kEvict, 256, true>(a, s);
    return a.n_max <= kRowsInLds ? launch_plan<kEvict, kThreads, true>(a, s) : launch_plan<kEvict, kThreads, false>(a, s);
}
}  // namespace

hipError_t launch_q4_compact(const Q4PageArgs& a, hipStream_t s) {
    hipError_t e = a.budget ? launch_plan_by_rows<true>(a, s) : launch_plan_by_rows<false>(a, s);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(q4_grant_kernel, dim3(1), dim3(kThreads), 0, s, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    // parts of a sequence's rows: four workgroups per CU in all, no more than there can be entries for (two 52 us, three 46.5, four
    // 44.8, six 47.6 in the case above)
    const int slabs = a.dims.layers * a.dims.batch, most = (a.n_max + kEntries - 1) / kEntries;
    const int cus = device_cus() > 0 ? device_cus() : 256;
    const int want = (4 * cus + slabs - 1) / slabs, parts = want < most ? want : most;
    const dim3 grid(parts, a.dims.layers + 1, a.dims.batch);
    if (a.dims.d == 128) hipLaunchKernelGGL(q4_move_kernel<128>, grid, dim3(kMoveBlock), 0, s, a);
    else hipLaunchKernelGGL(q4_move_kernel<64>, grid, dim3(kMoveBlock), 0, s, a);
    return hipGetLastError();
}

}  // namespace ikv
