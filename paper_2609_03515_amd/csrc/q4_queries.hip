// Attention of blocks of queries over the paged 4-bit cache: o = softmax(q . k / sqrt(d)) v over the rows that a query sees.
//
// Window: the queries are those of a slot's newest rows; query at position P sees the rows at positions p <= P that are in the
// window, p > P - window, or among the first, p < sinks.  Shared: one query of each of several slots; where their tables name the
// same page it is read and converted once for all of them.
//
// A block of queries is one or more column tiles, each `per` queries of the group's heads in 16 columns; the tiles of 32 rows, their
// products, probabilities and values are those of the decode attention (q4_attend.hip), with each converted tile used by every
// column tile.  A workgroup takes a block and one KV head; its waves take the block's tiles of rows in turn, each with a running
// maximum, sum and output of its own, joined at the end.  Where there are few blocks their tiles are divided among workgroups, whose
// parts a second kernel joins.
//
// Which tiles: without positions the rows are in order, and the tiles of a window are two runs.  With positions (an eviction leaves
// rows of any position in any place) a kernel before this one marks the tiles of which a block sees any row, a bit each; a wave
// holds a word per lane and finds its k-th tile by their counts.  Shared: a kernel before this one lists, for every slot of a block,
// the pages that no slot before it in the block has, with the queries that each is a page of.
//
// Masked rows get the logit -inf.  A masked row's values may be NaN (a block stored from infinities); 0 times them would spoil the
// column, so tiles that hold such blocks take a side path: the blocks are taken as numbers, and a product of two 0/1 matrices finds
// the outputs whose query sees one.
#include <float.h>
#include <limits.h>

#include <atomic>
#include <type_traits>

#include "kv_common.h"
#include "q4.h"
#include "q4_lane.h"
#include "stream_lane.h"

namespace ikv {
namespace {

constexpr int kAlone = 768;  // blocks of four column tiles from which a wave takes each for itself
constexpr int kKeep = 0;  // rows are read again by other workgroups
constexpr float kNaN = __builtin_nanf("");

typedef int __attribute__((ext_vector_type(4))) i32x4;
typedef const __attribute__((address_space(4))) i32x4* scalar_int4s;

// The kernel's arguments read where they are used, not kept from its beginning on (in spilled scalar registers).
typedef const __attribute__((address_space(4))) Q4QueryArgs* late_args;
__device__ __forceinline__ late_args args_again() {
    late_args p = (late_args)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return p;
}
// A lane's offset, widened where it is used: an address is a scalar base and a 32-bit offset then.
__device__ __forceinline__ uint32_t again(uint32_t x) {
    asm volatile("" : "+v"(x));
    return x;
}
__device__ __forceinline__ float max3(float a, float b, float c) {  // (fmaxf first copies operands that might be signalling NaNs)
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// Two numbers rounded to bf16, to nearest even.
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    typedef float __attribute__((ext_vector_type(2))) f32x2;
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2));
}
__device__ __forceinline__ int wave_max_int(int x) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) x = max(x, __shfl_xor(x, o, kWave));
    return x;
}
__device__ __forceinline__ int lower_bound_of(int at, int window) {  // the window's first position
    return window ? (int)max((int64_t)INT_MIN, (int64_t)at - (window - 1)) : INT_MIN;
}

// A slot's rows and newest rows as a windowed call sees them.
struct Slot {
    int n, count;
    bool bad;
};
__device__ __forceinline__ Slot slot_of(const Q4QueryArgs& a, int b) {
    const int raw = a.cache.len[b];
    Slot s;
    s.n = raw < 0 || raw > a.n_max ? 0 : raw;
    s.count = a.count ? a.count[b] : min(a.rows, s.n);
    s.bad = s.n != raw || s.count < 0 || s.count > a.rows || s.count > s.n;
    if (s.bad) {  // (zeros for all of its queries)
        s.n = 0;
        s.count = a.rows;
    }
    return s;
}

// Tiles that a block sees any row of: one wave to 64 tiles.
constexpr int kMarkWaves = 4;
__global__ __launch_bounds__(kMarkWaves* kWave) void q4_mark_kernel(Q4QueryArgs a) {
    const uint32_t runs = (a.words + kMarkWaves - 1) / kMarkWaves, unit = blockIdx.x / runs;
    const int lane = threadIdx.x % kWave, word = (blockIdx.x - unit * runs) * kMarkWaves + threadIdx.x / kWave;
    const int block = unit % (uint32_t)a.plan.blocks, b = unit / (uint32_t)a.plan.blocks;
    const Slot slot = slot_of(a, b);
    const int v0 = block * a.plan.vectors;
    if (v0 >= slot.count || word >= a.words) return;
    const int32_t* pos = a.cache.pos + (size_t)b * a.dims.cap;
    const int first = slot.n - slot.count + v0;
    int top = INT_MIN, low = INT_MAX;
    for (int i = lane; i < min(a.plan.vectors, slot.count - v0) && first + i < slot.n; i += kWave) {
        top = max(top, pos[first + i]);
        low = min(low, pos[first + i]);
    }
    top = wave_max_int(top);
    low = ~wave_max_int(~low);
    const int from = lower_bound_of(low, a.window);
    uint64_t bits = 0;
    const int row0 = word * 64 * kTile;
    if (row0 < slot.n) {
#pragma unroll 16
        for (int i = 0; i < kTile; ++i) {  // 64 rows: two tiles
            const int row = row0 + i * kWave + lane;
            const int p = pos[min(row, slot.n - 1)];
            const uint64_t any = __ballot(row < slot.n && p <= top && (p >= from || p < a.sinks));
            bits |= (uint64_t)((uint32_t)any != 0) << (2 * i) | (uint64_t)((any >> 32) != 0) << (2 * i + 1);
        }
    }
    if (lane == 0) a.visible[((size_t)b * a.plan.blocks + block) * a.words + word] = bits;
}

// Shared: the block that each slot is in, and the slot's list of pages.  One workgroup per slot.
constexpr int kListThreads = 256;
__global__ __launch_bounds__(kListThreads) void q4_list_kernel(Q4QueryArgs a) {
    __shared__ int members[kQ4MostVectors], lens[kQ4MostVectors], info[2];
    __shared__ int sums[kListThreads / kWave];
    const Q4Dims& d = a.dims;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, b = blockIdx.x, V = a.plan.vectors;
    const int mine = a.group[b];
    // The slots of the group in ascending order are cut into blocks of V; `members` holds the block of slot b.
    if (wave == 0) {
        int seen = 0, rank = -1;  // slots of the group so far, and those before b
        for (int i0 = 0; i0 < d.batch; i0 += kWave) {
            const int i = i0 + lane;
            const bool same = i < d.batch && a.group[i] == mine;
            const uint64_t all = __ballot(same);
            const int r = seen + __popcll(all & ((1ull << lane) - 1));
            seen += __popcll(all);
            if (i0 <= b && b < i0 + kWave) rank = __builtin_amdgcn_readlane(r, b - i0);
            // (before b is found: the last V, which are those that b's block can have)
            if (same && (rank < 0 ? r >= seen - V : r / V == rank / V)) members[r % V] = i;
            if (rank >= 0 && seen >= (rank / V + 1) * V) break;
        }
        if (lane == 0) {
            info[0] = rank % V;
            info[1] = min(V, seen - rank / V * V);
        }
    }
    __syncthreads();
    const int k = info[0], count = info[1];
    if ((int)threadIdx.x < count) {
        const int n = a.cache.len[members[threadIdx.x]];
        lens[threadIdx.x] = n < 0 || n > a.n_max ? 0 : n;
        if ((int)threadIdx.x == k && lens[k] != n) atomicOr(a.faults, kFaultCache);
    }
    if (k == 0 && (int)threadIdx.x < V) a.members[(size_t)b * V + threadIdx.x] = (int)threadIdx.x < count ? members[threadIdx.x] : -1;
    if (threadIdx.x == 0) a.heads[b] = k == 0;
    __syncthreads();
    const int pages = (lens[k] + d.page_rows - 1) >> d.page_shift;
    int done = 0;
    for (int j0 = 0; j0 < pages; j0 += kListThreads) {
        const int j = j0 + (int)threadIdx.x;
        uint32_t mask = 0;
        int page = 0, rows = 0;
        if (j < pages) {
            page = a.cache.table[(size_t)b * d.max_pages + j];
            rows = min(d.page_rows, lens[k] - (j << d.page_shift));
            if ((uint32_t)page >= (uint32_t)d.n_pages) {
                atomicOr(a.faults, kFaultCache);
            } else {
                for (int m = 0; m < count; ++m) {
                    const int left = lens[m] - (j << d.page_shift);
                    if (left > 0 && min(d.page_rows, left) == rows && a.cache.table[(size_t)members[m] * d.max_pages + j] == page) mask |= 1u << m;
                }
            }
        }
        const bool listed = mask && __builtin_ctz(mask) == k;  // (the first slot that has it lists it)
        const uint64_t all = __ballot(listed);
        if (lane == 0) sums[wave] = __popcll(all);
        __syncthreads();
        int at = done + __popcll(all & ((1ull << lane) - 1));
        for (int w = 0; w < kListThreads / kWave; ++w) {
            if (w < wave) at += sums[w];
            done += sums[w];
        }
        if (listed) a.items[(size_t)b * a.list_pages + at] = make_int4(page, rows, (int)mask, 0);
        __syncthreads();
    }
    if (threadIdx.x == 0) a.lists[b] = done;
}

// A tile that is to be loaded: its halves' pages and what is known of them before their rows are.
struct Ref {
    int row;  // window: its first row; shared: the first row in the page
    int page[2], rows[2];
    uint32_t mask[2];
};
struct Half {
    const uint8_t* k;  // the half's first row: keys' codes, ...
    const uint8_t* e;  // ... scales, and the values' of both vc_off bytes on
    int valid;         // rows that take part
    uint32_t mask;     // shared: queries of the block that it is a half of
};
template <int D>
struct KeyTile {
    uint32_t codes[2][D / 32];
    uint32_t scale[2];
    int pos;  // position of row `lane % 32` (window with positions)
};

// Column tiles (CT) of 16; parts of a probability (kP): 3 take all of its 24 bits, 1 rounds it to bf16 (8 bits, to nearest; its
// sum is of the rounded numbers).  kWaves: of a workgroup, which divide a block's tiles and join their outputs; or one.
template <typename T, int D, int CT, int kP, bool kShared, int kWaves>
__global__ __launch_bounds__(kWave* kWaves, CT == 1 ? 4 : 2) void q4_query_kernel(Q4QueryArgs a) {
    constexpr int kThreads = kWave * kWaves;
    constexpr int kKey = D / 32, kOut = D / 16;     // products per half, and for the output
    constexpr int kParts = sizeof(T) == 2 ? 1 : 3;  // bf16 parts of a query
    constexpr int kStride = D + 4;
    constexpr int kJoin = (kWaves + 1) / 2;         // waves whose outputs are joined through LDS at once
    // [wave] values; in their place [joined wave][column][kStride] outputs; then [wave][column] maxima and sums; then the queries
    extern __shared__ float lds[];
    const Q4Dims& d = a.dims;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int group = d.group, per = a.plan.per;

    // unit: KV heads fastest (eight of them fall on the eight XCDs), then the blocks, the last (a window's longest) first
    uint32_t x = blockIdx.x;
    const int g = x % (uint32_t)d.hkv;
    x /= (uint32_t)d.hkv;
    const int nth = x % (uint32_t)a.plan.blocks;
    x /= (uint32_t)a.plan.blocks;
    int b = 0;
    if constexpr (!kShared) {
        b = x % (uint32_t)d.batch;
        x /= (uint32_t)d.batch;
    }
    const int layer = x % (uint32_t)a.layer_count, chunk = x / (uint32_t)a.layer_count;
    const size_t page_bytes = (size_t)d.hkv * d.rec;
    const int step = a.plan.chunks * kWaves, k0 = chunk * kWaves + wave;
    uint32_t fault = 0;

  // Shared: a workgroup takes the nth block, and those `blocks` further on, where small groups make more than there are places for.
  for (int turn = nth;; turn += a.plan.blocks) {
    int lane = threadIdx.x % kWave;
    if constexpr (kShared) asm volatile("" : "+v"(lane));  // (nothing of a lane is worked out before the loop and kept over it)
    const int c = lane % 16, s = lane / 16, part = c / group, head = c - part * group;
    const uint8_t* const pool = a.cache.pool + q4_record(d, a.layer0 + layer, 0, g);
    if constexpr (kShared) {
        // the slot that the block begins with
        b = -1;
        int seen = 0;
        for (int i0 = 0; i0 < d.batch && b < 0; i0 += kWave) {
            const uint64_t is = __ballot(i0 + lane < d.batch && a.heads[min(i0 + lane, d.batch - 1)]);
            const uint64_t it = __ballot((is >> lane & 1) && seen + __popcll(is & ((1ull << lane) - 1)) == turn);
            if (it) b = i0 + __builtin_ctzll(it);
            seen += __popcll(is);
        }
        if (b < 0) break;
    }
    // the block's queries: the lane's in each column tile, its slot and row (-1: none)
    const int32_t* const members = kShared ? a.members + (size_t)b * a.plan.vectors : nullptr;
    const int block = kShared ? 0 : a.plan.blocks - 1 - nth, v0 = block * a.plan.vectors;
    Slot slot{0, 0, false};
    if constexpr (!kShared) {
        slot = slot_of(a, b);
        if (slot.bad && g == 0 && layer == 0 && chunk == 0 && threadIdx.x == 0) atomicOr(a.faults, kFaultCache);
        if (v0 >= slot.count) return;
    }
    auto slot_row = [&](int ct, int vector_in_tile, int& sl, int& row) __attribute__((always_inline)) {
        const int v = ct * per + vector_in_tile;
        sl = b;
        row = 0;
        if constexpr (kShared) {
            sl = members[v];
        } else {
            row = v0 + v;
            if (row >= slot.count) sl = -1;
        }
    };
    __shared__ int places[kShared ? 1 : CT * 16];  // window: the columns' positions (no query: the lowest)
    int top_place = INT_MIN, low_place = INT_MAX;
    if constexpr (!kShared) {
        int top = INT_MIN, low = INT_MAX;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            int sl = -1, row = 0, place = INT_MIN;
            if (part < per) slot_row(ct, part, sl, row);
            if (sl >= 0 && slot.n > 0) {
                const int r = slot.n - slot.count + row;
                place = a.cache.pos ? a.cache.pos[(size_t)b * d.cap + r] : r;
                top = max(top, place);
                low = min(low, place);
            }
            if (wave == 0 && s == 0) places[16 * ct + c] = place;
        }
        top_place = __builtin_amdgcn_readfirstlane(wave_max_int(top));
        low_place = __builtin_amdgcn_readfirstlane(~wave_max_int(~low));
    }

    // queries as bf16 parts in LDS, [part][product][column tile][lane] (in registers one column tile would take 16, and spill as many)
    u32x4* const q_lds = reinterpret_cast<u32x4*>(lds + a.q_at) + lane;
#pragma unroll
    for (int i = 0; i < (CT + kWaves - 1) / kWaves; ++i) {
        const int ct = i * kWaves + wave;
        if (ct >= CT) break;
        int sl = -1, row = 0;
        if (part < per) slot_row(ct, part, sl, row);
        // (no query: any row, not used)
        const T* qp = static_cast<const T*>(a.q) + s * (D / 4);
        if (sl >= 0) qp += layer * a.qs[0] + sl * a.qs[1] + (g * group + head) * a.qs[2] + row * a.qs[3];
        if constexpr (kParts == 1) {
#pragma unroll
            for (int j = 0; j < kKey; ++j) {
                const u32x4 w = reinterpret_cast<const u32x4*>(qp)[j];
                q_lds[(j * CT + ct) * kWave] = sl >= 0 ? w : u32x4{0, 0, 0, 0};
            }
        } else {
#pragma unroll
            for (int j = 0; j < kKey; ++j) {
                float f[8];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const f32x4 w = reinterpret_cast<const f32x4*>(qp)[2 * j + i];
#pragma unroll
                    for (int e = 0; e < 4; ++e) f[4 * i + e] = sl >= 0 ? w[e] : 0.0f;
                }
#pragma unroll
                for (int p = 0; p < 3; ++p) {
                    u32x4 y;
#pragma unroll
                    for (int i = 0; i < 4; ++i) y[i] = high2(__float_as_uint(f[2 * i]), __float_as_uint(f[2 * i + 1]));
                    q_lds[((p * kKey + j) * CT + ct) * kWave] = y;
#pragma unroll
                    for (int i = 0; i < 8; ++i) f[i] -= __uint_as_float(__float_as_uint(f[i]) & 0xffff0000u);
                }
            }
        }
    }

    // The wave's tiles are those of numbers k0, k0 + step, ... of `tiles`.  It looks at 64 of them at a time, one a lane: the pages (or
    // listed pages) of the lane's tile, and a bit for each that takes part.
    int tiles = 0;
    uint32_t all = 0;                              // shared: every query of the block
    int items = 0;                                 // shared: pages that the block's slots list
    __shared__ int list_slot[kShared ? kQ4MostVectors : 1], list_before[kShared ? kQ4MostVectors : 1];  // a member, and pages that those before it list
    const int per_page_shift = kShared ? max(0, d.page_shift - 5) : 0;
    if constexpr (kShared) {
        const int m = lane < a.plan.vectors ? members[lane] : -1;
        int sum = m >= 0 ? a.lists[m] : 0;
        const int mine = sum;
#pragma unroll
        for (int o = 1; o < kQ4MostVectors; o <<= 1) {
            const int up = __shfl_up(sum, o, kWave);
            if (lane >= o) sum += up;
        }
        if (wave == 0 && lane < a.plan.vectors) {
            list_slot[lane] = max(m, 0);
            list_before[lane] = sum - mine;
        }
        items = __builtin_amdgcn_readlane(sum, kQ4MostVectors - 1);
        all = (uint32_t)__ballot(m >= 0);
        tiles = d.page_rows >= kTile ? items << per_page_shift : (items + 1) / 2;
    } else {
        tiles = (slot.n + kTile - 1) / kTile;
    }
    const int top_from = lower_bound_of(top_place, a.window), low_from = lower_bound_of(low_place, a.window);
    const int32_t* const pos = kShared || !a.cache.pos ? nullptr : a.cache.pos + (size_t)b * d.cap;
    int page_of = 0, page_of2 = 0;  // window: pages of the halves; shared: the listed page, its rows in use and its queries (pages of 16
    uint32_t mask_of = 0;           // rows: lanes 32 .. 63 hold the second halves of lanes 0 .. 31's tiles)
    uint64_t left = 0;
    int base = 0;
    const bool pairs = kShared && d.page_rows < kTile;
    const int at_once = pairs ? kWave / 2 : kWave;
    auto look = [&]() __attribute__((always_inline)) {
        int lane = threadIdx.x % kWave;
        asm volatile("" : "+v"(lane));  // (its places are worked out here, not kept over the tiles)
        const late_args late = args_again();
        const int k = k0 + (base + (pairs ? lane % (kWave / 2) : lane)) * step;  // (2^27 rows are 2^22 tiles, and 64 steps fewer than 2^25)
        bool part_of = k < tiles;
        if constexpr (kShared) {
            const int i = pairs ? 2 * k + lane / (kWave / 2) : k >> per_page_shift;
            int before = 0, sl = 0;
            for (int v = 0; v < late->plan.vectors; ++v) {  // the last member that has as many before it: it lists the page
                const int y = list_before[v], z = list_slot[v];
                before = y <= i ? y : before;
                sl = y <= i ? z : sl;
            }
            int4 it = make_int4(0, 0, 0, 0);
            if (part_of && i < items) it = late->items[(size_t)sl * late->list_pages + (i - before)];
            page_of = it.x;
            page_of2 = it.y;
            mask_of = it.z;
            if (pairs) part_of = part_of && lane < kWave / 2;
        } else {
            const int row = k * kTile;
            const int32_t* const table = late->cache.table + (size_t)b * late->dims.max_pages;
            const int last = late->dims.cap - 1;
            page_of = table[min(row, last) >> late->dims.page_shift];
            page_of2 = table[min(row + 16, last) >> late->dims.page_shift];
            if (!pos) {
                part_of = part_of && row <= top_place && (row + kTile > low_from || row < a.sinks);
            } else if (late->visible) {
                part_of = part_of && (late->visible[((size_t)b * late->plan.blocks + block) * late->words + k / 64] >> k % 64 & 1);
            } else {
                // two tiles to a load, eight loads together
                uint64_t bits = 0;
                constexpr int kTogether = 8;
                for (int i0 = 0; i0 < kWave && k0 + (base + i0) * step < tiles; i0 += 2 * kTogether) {
                    int p[kTogether];
#pragma unroll
                    for (int i = 0; i < kTogether; ++i) p[i] = pos[min((k0 + (base + i0 + 2 * i + lane / kTile) * step) * kTile + lane % kTile, last)];
#pragma unroll
                    for (int i = 0; i < kTogether; ++i) {
                        const int r = (k0 + (base + i0 + 2 * i + lane / kTile) * step) * kTile + lane % kTile;
                        const uint64_t any = __ballot(r < slot.n && p[i] <= top_place && (p[i] >= low_from || p[i] < a.sinks));
                        bits |= (uint64_t)((uint32_t)any != 0) << (i0 + 2 * i) | (uint64_t)((any >> 32) != 0) << (i0 + 2 * i + 1);
                    }
                }
                part_of = bits >> lane & 1;
            }
        }
        left = __ballot(part_of);
    };
    // the next tile of them that takes part
    auto fetch = [&](Ref& r) __attribute__((always_inline)) {
        if (!left) return false;
        const int i = __builtin_ctzll(left), k = k0 + (base + i) * step;
        left &= left - 1;
        if constexpr (kShared) {
            r.row = (k & ((1 << per_page_shift) - 1)) * kTile;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int from_lane = pairs && h ? i + kWave / 2 : i;
                r.page[h] = __builtin_amdgcn_readlane(page_of, from_lane);
                r.rows[h] = __builtin_amdgcn_readlane(page_of2, from_lane) - (pairs ? 0 : r.row + 16 * h);
                r.mask[h] = __builtin_amdgcn_readlane(mask_of, from_lane);
            }
        } else {
            r.row = k * kTile;
            r.page[0] = __builtin_amdgcn_readlane(page_of, i);
            r.page[1] = __builtin_amdgcn_readlane(page_of2, i);
        }
        return true;
    };
    auto locate = [&](const Ref& r, Half (&h)[2]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            int page = r.page[i], in;
            if constexpr (kShared) {
                h[i].valid = __builtin_amdgcn_readfirstlane(min(16, max(0, r.rows[i])));
                h[i].mask = h[i].valid ? r.mask[i] : 0;
                in = d.page_rows >= kTile ? r.row + 16 * i : 0;
            } else {
                const int row = r.row + 16 * i;
                h[i].valid = __builtin_amdgcn_readfirstlane(min(16, max(0, slot.n - row)));
                h[i].mask = 0;
                in = row & (d.page_rows - 1);
                if ((uint32_t)page >= (uint32_t)d.n_pages) {
                    if (h[i].valid) fault = kFaultCache;
                    page = h[i].valid = 0;
                }
            }
            const uint8_t* rec = pool + (size_t)(uint32_t)page * page_bytes;
            h[i].k = rec + in * (D / 2);
            h[i].e = rec + d.ks_off + in * (D / 32);
        }
    };
    const int key_row = c % 4 * 4 + c / 4;  // row of a half whose keys the lane holds: result rows 4 s + i are rows 4 i + s
    const uint32_t ko = key_row * (D / 2) + s * (D / 8), eo = D == 128 ? key_row * 4 + s : key_row * 2 + s / 2;
    auto load_keys = [&](KeyTile<D>& t, const Half (&h)[2], int row) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if constexpr (D == 128) {
                const u32x4 w = *reinterpret_cast<const u32x4*>(h[i].k + again(ko));
#pragma unroll
                for (int j = 0; j < 4; ++j) t.codes[i][j] = w[j];
            } else {
                const u32x2 w = *reinterpret_cast<const u32x2*>(h[i].k + again(ko));
                t.codes[i][0] = w[0];
                t.codes[i][1] = w[1];
            }
            t.scale[i] = h[i].e[again(eo)];
        }
        if (pos) t.pos = *reinterpret_cast<const int32_t*>(reinterpret_cast<const char*>(pos) + 4 * again(min(row + lane % kTile, slot.n - 1)));
    };
    uint8_t* const value_lds = reinterpret_cast<uint8_t*>(lds) + wave * kValueBytes<D>;
    const uint8_t* const value_codes = value_lds + s * (D / 2) + c * (D / 32);
    const uint8_t* const value_scales = value_lds + kTile * (D / 2) + s * (D / 32) + (D == 128 ? c / 4 : c / 8);
    auto load_values = [&](const Half (&h)[2]) __attribute__((always_inline)) {
        if constexpr (D == 128) {
            to_lds<16, kKeep>(h[0].k + d.vc_off + again(lane * 16), value_lds);
            to_lds<16, kKeep>(h[1].k + d.vc_off + again(lane * 16), value_lds + 1024);
            to_lds<4, kKeep>((lane & 16 ? h[1].e : h[0].e) + d.vc_off + lane % 16 * 4, value_lds + 2048);
        } else {
            to_lds<16, kKeep>((lane & 32 ? h[1].k : h[0].k) + d.vc_off + lane % 32 * 16, value_lds);
            to_lds<4, kKeep>((lane & 8 ? h[1].e : h[0].e) + d.vc_off + lane % 8 * 4, value_lds + 1024);
        }
    };

    float m[CT], l[CT];
    f32x4 acc[CT][kOut];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        m[ct] = -FLT_MAX;
        l[ct] = 0.0f;
#pragma unroll
        for (int e = 0; e < kOut; ++e) acc[ct][e] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    __syncthreads();

    // Loads run one tile ahead (but for the first of 64).
   for (; k0 + base * step < tiles; base += at_once) {
    look();
    KeyTile<D> keys;
    Half now[2], next[2];
    Ref ref{}, ahead{};
    bool have = fetch(ref), more = false;
    if (have) {
        locate(ref, now);
        load_keys(keys, now, ref.row);
        load_values(now);
        more = fetch(ahead);
    }
    while (have) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the tile's keys, and its values in LDS
        const int row = ref.row;
        const bool whole = now[0].valid + now[1].valid == kTile;
        uint32_t active = ~0u;  // shared: column tiles with a query that the tile is a tile of
        if constexpr (kShared && CT > 1) active = now[0].mask | now[1].mask;
        auto skipped = [&](int ct) __attribute__((always_inline)) {
            return kShared && CT > 1 && !(active >> (ct * per) & ((1u << per) - 1));
        };
        // logits
        f32x4 z[CT][2];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) z[ct][0] = z[ct][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        const float key_scale[2] = {__uint_as_float(keys.scale[0] << 23), __uint_as_float(keys.scale[1] << 23)};
        // (the next product's queries are read while this one's are used: a wave waits for LDS once, not for each)
        u32x4 y[2][kParts * CT];
        auto read_queries = [&](u32x4 (&to)[kParts * CT], int j) __attribute__((always_inline)) {
#pragma unroll
            for (int p = 0; p < kParts; ++p)
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) to[p * CT + ct] = q_lds[((p * kKey + j) * CT + ct) * kWave];
        };
        read_queries(y[0], 0);
#pragma unroll
        for (int j = 0; j < kKey; ++j) {
            if (j + 1 < kKey) read_queries(y[(j + 1) & 1], j + 1);
            const u32x4 k0 = eight(keys.codes[0][j], key_scale[0]), k1 = eight(keys.codes[1][j], key_scale[1]);
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                if (skipped(ct)) continue;
#pragma unroll
                for (int p = kParts - 1; p >= 0; --p) {
                    z[ct][0] = mfma(k0, y[j & 1][p * CT + ct], z[ct][0]);
                    z[ct][1] = mfma(k1, y[j & 1][p * CT + ct], z[ct][1]);
                }
            }
        }
        const int tile_pos = keys.pos;
        // the lane's rows that its column does not see, a bit each: bit j is row 4 (j % 4) + s of half j / 4.  (Without branches: the
        // compiler, ROCm 7.2's, dropped the first element's store from the same conditions joined by ||.)
        auto hidden = [&](uint32_t (&bits)[CT]) __attribute__((always_inline)) {
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) bits[ct] = 0;
            const int s_of = again(s);
            int p[8];
            if constexpr (!kShared) {
                if (pos) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) p[j] = __builtin_amdgcn_ds_bpermute(4 * s_of + 4 * (16 * (j / 4) + 4 * (j % 4)), tile_pos);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) p[j] = row + s_of + 16 * (j / 4) + 4 * (j % 4);
                }
            }
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                int place = 0, from = 0;
                if constexpr (!kShared) {
                    place = places[16 * ct + c];
                    from = a.window ? __builtin_elementwise_sub_sat(place, a.window - 1) : INT_MIN;
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int half = j / 4;
                    uint32_t h = 4 * (j % 4) >= now[half].valid - s_of;
                    if constexpr (kShared) h |= ~(now[half].mask >> (ct * per + part)) & 1u;
                    else h |= (uint32_t)(p[j] > place) | ((uint32_t)(p[j] < from) & (uint32_t)(p[j] >= a.sinks));
                    bits[ct] |= h << j;
                }
            }
        };
        bool plain = whole;  // every column sees every row
        if constexpr (kShared) {
            plain = plain && (now[0].mask & now[1].mask) == all;
        } else {
            const int p = pos ? tile_pos : row + lane % kTile;
            plain = plain && __all(p <= low_place && (p >= top_from || p < a.sinks));
        }
        if (!plain) {
            asm volatile("");
            uint32_t bits[CT];
            hidden(bits);
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int j = 0; j < 8; ++j) z[ct][j / 4][j % 4] = bits[ct] >> j & 1u ? -INFINITY : z[ct][j / 4][j % 4];
        }
        if (more) {
            locate(ahead, next);
            load_keys(keys, next, ahead.row);
        }
        // running maxima, probabilities, their parts
        u32x4 high[CT], mid[kP == 3 ? CT : 1], low[kP == 3 ? CT : 1];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            if (skipped(ct)) continue;
            float top = max3(z[ct][0][0], z[ct][0][1], z[ct][0][2]);
            top = max3(top, z[ct][0][3], z[ct][1][0]);
            top = max3(top, z[ct][1][1], z[ct][1][2]);
            top = max3(top, z[ct][1][3], z[ct][1][3]) * a.scale2;
            if (__any(top > m[ct] + kSlack)) {
                top = rows_allmax(top);
                const float raised = top > m[ct] + kSlack ? top : m[ct];
                const float f = exp2_hw(m[ct] - raised);
                m[ct] = raised;
                l[ct] *= f;
#pragma unroll
                for (int e = 0; e < kOut; ++e) acc[ct][e] *= f;
            }
            float p[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) p[j] = exp2_hw(fmaf(z[ct][j / 4][j % 4], a.scale2, -m[ct]));
            if constexpr (kP == 1) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    high[ct][i] = pack2(p[2 * i], p[2 * i + 1]);
                    l[ct] = Elem<bf16_t>::dot2(high[ct][i], 0x3f803f80u, l[ct]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    l[ct] += p[2 * i] + p[2 * i + 1];
                    const uint32_t w[2] = {__float_as_uint(p[2 * i]), __float_as_uint(p[2 * i + 1])};
                    float y[2], rest[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float upper = __uint_as_float(w[e] & 0xffffff00u);
                        y[e] = upper - __uint_as_float(w[e] & 0xffff0000u);
                        rest[e] = p[2 * i + e] - upper;
                    }
                    high[ct][i] = high2(w[0], w[1]);
                    mid[ct][i] = high2(__float_as_uint(y[0]), __float_as_uint(y[1]));
                    low[ct][i] = high2(__float_as_uint(rest[0]), __float_as_uint(rest[1]));
                }
            }
        }
        // output
        float scale[8];
        uint32_t codes[8];
        bool odd = false;  // a block that is NaN
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int r = 16 * (j / 4) + 4 * (j % 4);  // (and s)
            if constexpr (D == 128) codes[j] = *reinterpret_cast<const uint32_t*>(value_codes + r * (D / 2));
            else codes[j] = *reinterpret_cast<const uint16_t*>(value_codes + r * (D / 2));
            const uint32_t byte = value_scales[r * (D / 32)];
            scale[j] = __uint_as_float(byte << 23);
            odd |= byte == 255u;
        }
        if (!whole) {
            asm volatile("");
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (4 * (j % 4) >= now[j / 4].valid - s) scale[j] = 1.0f;
        }
        if (__any(odd)) {
            asm volatile("");
            u32x4 is;
            uint32_t bits[CT];
            hidden(bits);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                is[i] = (__float_as_uint(scale[2 * i]) == 0x7f800000u ? 0x3f80u : 0u) | (__float_as_uint(scale[2 * i + 1]) == 0x7f800000u ? 0x3f800000u : 0u);
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                u32x4 sees;
#pragma unroll
                for (int i = 0; i < 4; ++i) sees[i] = (bits[ct] >> (2 * i) & 1u ? 0u : 0x3f80u) | (bits[ct] >> (2 * i + 1) & 1u ? 0u : 0x3f800000u);
                const f32x4 n = mfma(is, sees, f32x4{0.0f, 0.0f, 0.0f, 0.0f});
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int e = 0; e < kOut; ++e) acc[ct][e][i] = n[i] > 0.0f ? kNaN : acc[ct][e][i];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (__float_as_uint(scale[j]) == 0x7f800000u) scale[j] = 1.0f;
        }
        if (more) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // this tile's values are out of LDS: the next tile's may come
            load_values(next);
        }
        auto two_columns = [&](auto byte) __attribute__((always_inline)) {
            constexpr int kByte = decltype(byte)::value;
            uint32_t w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = pair<kByte>(codes[j], scale[j]);
            const u32x4 even{low2(w[0], w[1]), low2(w[2], w[3]), low2(w[4], w[5]), low2(w[6], w[7])};
            const u32x4 uneven{high2(w[0], w[1]), high2(w[2], w[3]), high2(w[4], w[5]), high2(w[6], w[7])};
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                if (skipped(ct)) continue;
                f32x4 &e = acc[ct][2 * kByte], &u = acc[ct][2 * kByte + 1];
                if constexpr (kP == 3) {
                    e = mfma(even, low[ct], e);
                    u = mfma(uneven, low[ct], u);
                    e = mfma(even, mid[ct], e);
                    u = mfma(uneven, mid[ct], u);
                }
                e = mfma(even, high[ct], e);
                u = mfma(uneven, high[ct], u);
            }
        };
        two_columns(std::integral_constant<int, 0>());
        two_columns(std::integral_constant<int, 1>());
        if constexpr (D == 128) {
            two_columns(std::integral_constant<int, 2>());
            two_columns(std::integral_constant<int, 3>());
        }
        have = more;
        if (more) {
            now[0] = next[0];
            now[1] = next[1];
            ref = ahead;
            more = fetch(ahead);
        }
    }
   }
    // the waves joined: the upper half into the lower, those through columns of LDS
    constexpr int kColumns = CT * 16;
    float* const stat = lds + a.stat_at;  // [wave][column] maxima, then sums
    __syncthreads();                      // (their values' places are used again)
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) l[ct] = rows_allsum(l[ct]);
    auto mine = [&](int ct) __attribute__((always_inline)) { return lds + ((wave % kJoin) * kColumns + 16 * ct + c) * kStride + s * (D / 4); };
    auto put = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < kOut; e += 4)
                    *reinterpret_cast<f32x4*>(mine(ct) + i * kOut + e) = f32x4{acc[ct][e][i], acc[ct][e + 1][i], acc[ct][e + 2][i], acc[ct][e + 3][i]};
            if (s == 0) {
                stat[wave * kColumns + 16 * ct + c] = m[ct];
                stat[(kWaves + wave) * kColumns + 16 * ct + c] = l[ct];
            }
        }
    };
    // elements e .. e + 3 of column col: the weights' maximum and sum, and the sum over the rows
    const late_args late = args_again();
    auto store = [&](int col, int e, float top, float sum, f32x4 o) __attribute__((always_inline)) {
        const int vt = col % 16 / group, h = col % 16 - vt * group;
        int sl = -1, row = 0;
        if (vt < per) slot_row(col / 16, vt, sl, row);
        if (sl < 0) return;
        if (late->plan.chunks == 1) {
            o *= sum != 0.0f ? 1.0f / sum : 0.0f;
            T* op = static_cast<T*>(late->o) + layer * late->os[0] + sl * late->os[1] + (g * group + h) * late->os[2] + row * late->os[3] + e;
            if constexpr (sizeof(T) == 2) *reinterpret_cast<u32x2*>(op) = u32x2{pack2(o[0], o[1]), pack2(o[2], o[3])};
            else *reinterpret_cast<f32x4*>(op) = o;
        } else {
            // (a part without rows for the query is its sum, 0, alone)
            const size_t at = ((((size_t)layer * late->dims.batch + sl) * late->rows + row) * late->dims.hq + g * group + h) * late->plan.chunks + chunk;
            if (sum != 0.0f) *reinterpret_cast<f32x4*>(late->opart + at * D + e) = o;
            if (e == 0) late->part[at] = make_float2(top, sum);
        }
    };
    if constexpr (kWaves == 1) {
        // (the barrier above: in the place of its values and queries)
        // a column tile at a time through LDS, so that a row's elements are written side by side
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            float* const place_of = lds + c * kStride + s * (D / 4);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < kOut; e += 4)
                    *reinterpret_cast<f32x4*>(place_of + i * kOut + e) = f32x4{acc[ct][e][i], acc[ct][e + 1][i], acc[ct][e + 2][i], acc[ct][e + 3][i]};
            __syncthreads();
            for (int i = lane; i < 16 * (D / 4); i += kWave) {
                const int col = i / (D / 4), e = i % (D / 4) * 4;
                store(16 * ct + col, e, __shfl(m[ct], col, kWave), __shfl(l[ct], col, kWave), *reinterpret_cast<const f32x4*>(lds + col * kStride + e));
            }
            __syncthreads();
        }
    } else {
        if (wave >= kJoin) put();
        __syncthreads();
        if (wave < kJoin) {
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                const float m2 = stat[(wave + kJoin) * kColumns + 16 * ct + c], l2 = stat[(kWaves + wave + kJoin) * kColumns + 16 * ct + c];
                const float top = fmaxf(m[ct], m2), f = exp2_hw(m[ct] - top), f2 = exp2_hw(m2 - top);
                m[ct] = top;
                l[ct] = l[ct] * f + l2 * f2;
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int e = 0; e < kOut; e += 4) {
                        const f32x4 o = *reinterpret_cast<const f32x4*>(mine(ct) + i * kOut + e);
#pragma unroll
                        for (int y = 0; y < 4; ++y) acc[ct][e + y][i] = acc[ct][e + y][i] * f + o[y] * f2;
                    }
            }
        }
        __syncthreads();
        if (wave < kJoin) put();
        __syncthreads();
        for (int i = threadIdx.x; i < kColumns * (D / 4); i += kThreads) {
            const int col = i / (D / 4), e = i % (D / 4) * 4;
            float top = stat[col];
#pragma unroll
            for (int w = 1; w < kJoin; ++w) top = fmaxf(top, stat[w * kColumns + col]);
            float sum = 0.0f;
            f32x4 o{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int w = 0; w < kJoin; ++w) {
                const float f = exp2_hw(stat[w * kColumns + col] - top);
                sum += f * stat[(kWaves + w) * kColumns + col];
                o += *reinterpret_cast<const f32x4*>(lds + (w * kColumns + col) * kStride + e) * f;
            }
            store(col, e, top, sum, o);
        }
    }
    if constexpr (!kShared) break;
    __syncthreads();  // (the next block's values come to the places of these)
  }
    if (fault && threadIdx.x % kWave == 0) atomicOr(a.faults, fault);
}

// The parts of a query head's output joined: 2^split threads to four elements, each of them every 2^split-th part.
constexpr int kPartThreads = 256;
template <typename T, int D, bool kShared>
__global__ __launch_bounds__(kPartThreads) void q4_part_kernel(Q4QueryArgs a, int split, uint32_t heads) {
    constexpr int kQuads = D / 4, kTogether = 4;
    __shared__ f32x4 out[kPartThreads];
    __shared__ float2 stat[kPartThreads];
    const Q4Dims& d = a.dims;
    const int quad = threadIdx.x % kQuads, k = threadIdx.x / kQuads & ((1 << split) - 1);
    const uint32_t i = blockIdx.x * (kPartThreads / kQuads >> split) + threadIdx.x / (kQuads << split);  // a query head
    const int h = i % (uint32_t)d.hq, chunks = a.plan.chunks;
    const uint32_t vector = i / (uint32_t)d.hq;
    const int row = vector % (uint32_t)a.rows, b = vector / (uint32_t)a.rows % (uint32_t)d.batch, layer = vector / (uint32_t)a.rows / (uint32_t)d.batch;
    const bool is = i < heads && (kShared || row < slot_of(a, b).count);
    float top = -FLT_MAX, sum = 0.0f;
    f32x4 o{0.0f, 0.0f, 0.0f, 0.0f};
    if (is) {
        const float2* part = a.part + (size_t)i * chunks;
        const float* from = a.opart + (size_t)i * chunks * D + quad * 4;
        for (int j0 = k; j0 < chunks; j0 += kTogether << split) {
            float2 p[kTogether];
            f32x4 x[kTogether];
#pragma unroll
            for (int j = 0; j < kTogether; ++j) {
                const int at = min(j0 + (j << split), chunks - 1);
                p[j] = part[at];
                if (j0 + (j << split) >= chunks) p[j] = make_float2(-FLT_MAX, 0.0f);
                x[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
                if (p[j].y != 0.0f) x[j] = *reinterpret_cast<const f32x4*>(from + (size_t)at * D);
            }
            float raised = top;
#pragma unroll
            for (int j = 0; j < kTogether; ++j) raised = fmaxf(raised, p[j].x);
            const float f = exp2_hw(top - raised);
            sum *= f;
            o *= f;
            top = raised;
#pragma unroll
            for (int j = 0; j < kTogether; ++j) {
                const float w = exp2_hw(p[j].x - top);
                sum += w * p[j].y;
                o += x[j] * w;
            }
        }
    }
    if (split) {
        out[threadIdx.x] = o;
        stat[threadIdx.x] = make_float2(top, sum);
        __syncthreads();
        if (k == 0) {
            for (int j = 1; j < 1 << split; ++j) {
                const float2 p = stat[threadIdx.x + j * kQuads];
                const float raised = fmaxf(top, p.x), f = exp2_hw(top - raised), w = exp2_hw(p.x - raised);
                sum = sum * f + w * p.y;
                o = o * f + out[threadIdx.x + j * kQuads] * w;
                top = raised;
            }
        }
    }
    if (!is || k != 0) return;
    o *= sum != 0.0f ? 1.0f / sum : 0.0f;
    T* op = static_cast<T*>(a.o) + layer * a.os[0] + b * a.os[1] + h * a.os[2] + row * a.os[3] + quad * 4;
    if constexpr (sizeof(T) == 2) *reinterpret_cast<u32x2*>(op) = u32x2{pack2(o[0], o[1]), pack2(o[2], o[3])};
    else *reinterpret_cast<f32x4*>(op) = o;
}

template <typename T, int D, int CT, int kP, bool kShared, int kWaves>
hipError_t launch_form(Q4QueryArgs a, hipStream_t s) {
    constexpr int kJoined = (kWaves + 1) / 2 * (kWaves > 1 ? CT : 1) * 16 * (D + 4) * (int)sizeof(float), kValues = kWaves * kValueBytes<D>;
    constexpr int kParts = sizeof(T) == 2 ? 1 : 3, kStat = 2 * kWaves * CT * 16;
    static_assert(kJoined % 16 == 0 && kValues % 16 == 0 && kStat % 4 == 0, "queries are read 16 bytes at a time");
    static_assert(CT * 16 <= kQ4MostColumns, "room for the parts of outputs");
    constexpr int kQueries = kParts * (D / 32) * CT * kWave * (int)sizeof(u32x4);
    // (a wave by itself has no statistics, and its outputs come to the place of its queries: eight such workgroups fit a CU)
    a.stat_at = (kJoined > kValues ? kJoined : kValues) / (int)sizeof(float);
    a.q_at = kWaves == 1 ? kValues / (int)sizeof(float) : a.stat_at + kStat;
    static_assert(kWaves > 1 || kJoined <= kValues + kQueries, "outputs in the place of values and queries");
    const size_t lds = (size_t)a.q_at * sizeof(float) + kQueries;
    auto kern = q4_query_kernel<T, D, CT, kP, kShared, kWaves>;
    if (lds > 64 * 1024) {
        static std::atomic<bool> raised[kMaxDevices];
        const hipError_t e = raise_lds_limit(reinterpret_cast<const void*>(kern), raised);
        if (e != hipSuccess) return e;
    }
    const uint32_t slots = kShared ? 1 : a.dims.batch;
    hipLaunchKernelGGL(kern, dim3((uint32_t)a.dims.hkv * a.plan.blocks * slots * a.layer_count * a.plan.chunks), dim3(kWave * kWaves), lds, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.plan.chunks == 1) return e;
    const uint32_t heads = (uint32_t)a.layer_count * a.dims.batch * a.rows * a.dims.hq;
    constexpr int kMostSplit = 31 - __builtin_clz(kPartThreads / (D / 4));
    int split = 0;
    while (split < kMostSplit && (4 << split) < a.plan.chunks) ++split;
    const uint32_t per = kPartThreads / (D / 4) >> split;
    hipLaunchKernelGGL((q4_part_kernel<T, D, kShared>), dim3((heads + per - 1) / per), dim3(kPartThreads), 0, s, a, split, heads);
    return hipGetLastError();
}

constexpr int kQueryWaves = 8;  // of a workgroup that divides a block's tiles
template <typename T, int D, bool kShared>
hipError_t launch_tiles(const Q4QueryArgs& a, hipStream_t s) {
    if constexpr (sizeof(T) == 2) {
        if constexpr (!kShared) {
            if (a.plan.tiles == 4) return launch_form<T, D, 4, 1, kShared, 1>(a, s);
        }
        if (a.plan.tiles == 2) return launch_form<T, D, 2, 1, kShared, kQueryWaves>(a, s);
    }
    return launch_form<T, D, 1, 3, kShared, kQueryWaves>(a, s);
}
template <bool kShared>
hipError_t launch_queries(const Q4QueryArgs& a, hipStream_t s) {
    if (a.dims.bf16) return a.dims.d == 128 ? launch_tiles<bf16_t, 128, kShared>(a, s) : launch_tiles<bf16_t, 64, kShared>(a, s);
    return a.dims.d == 128 ? launch_tiles<float, 128, kShared>(a, s) : launch_tiles<float, 64, kShared>(a, s);
}

int cus_of() { return device_cus() > 0 ? device_cus() : 256; }
// Workgroups of `waves` waves that divide a block's `tiles` tiles: until there are `want` of them, each with a tile for every wave at least.
int chunks_of(int64_t units, int64_t tiles, int waves, int want) {
    const int64_t by_units = (want + units - 1) / units, most = (tiles + waves - 1) / waves;
    return (int)(by_units < most ? by_units : most > 0 ? most : 1);
}

}  // namespace

Q4QueryPlan q4_window_plan(const Q4Dims& d, int layer_count, int n_max, int rows, int window, int sinks) {
    Q4QueryPlan p{};
    p.per = 16 / d.group;
    const int64_t slabs = (int64_t)layer_count * d.batch * d.hkv;
    auto blocks = [&](int tiles) { return (rows + tiles * p.per - 1) / (tiles * p.per); };
    p.tiles = !d.bf16 || rows <= p.per ? 1 : 2;
    if (d.bf16 && slabs * blocks(4) >= kAlone) p.tiles = 4;
    p.vectors = p.tiles * p.per;
    p.blocks = blocks(p.tiles);
    int64_t tiles = (n_max + kTile - 1) / kTile;
    if (window) {  // (rows in order, in a window that ends inside tiles)
        const int64_t seen = ((int64_t)window + sinks + p.vectors) / kTile + 3;
        tiles = tiles < seen ? tiles : seen;
    }
    if (p.tiles == 4) p.chunks = chunks_of(slabs * p.blocks, tiles / 8, 1, kQ4Units * cus_of());
    else p.chunks = chunks_of(slabs * p.blocks, tiles, kQueryWaves, 2 * cus_of());
    return p;
}

Q4QueryPlan q4_shared_plan(const Q4Dims& d, int layer_count, int n_max) {
    Q4QueryPlan p{};
    p.per = 16 / d.group;
    p.tiles = d.bf16 && d.batch > p.per ? 2 : 1;
    p.vectors = p.tiles * p.per;
    p.blocks = (d.batch + p.vectors - 1) / p.vectors;
    p.chunks = chunks_of((int64_t)layer_count * d.hkv * p.blocks, (n_max + kTile - 1) / kTile, kQueryWaves, 2 * cus_of());
    return p;
}

hipError_t launch_q4_window(const Q4QueryArgs& a, hipStream_t s) {
    if (a.visible) {
        hipLaunchKernelGGL(q4_mark_kernel, dim3((uint32_t)((a.words + kMarkWaves - 1) / kMarkWaves) * a.plan.blocks * a.dims.batch),
                           dim3(kMarkWaves * kWave), 0, s, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return launch_queries<false>(a, s);
}

hipError_t launch_q4_shared(const Q4QueryArgs& a, hipStream_t s) {
    hipLaunchKernelGGL(q4_list_kernel, dim3(a.dims.batch), dim3(kListThreads), 0, s, a);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? e : launch_queries<true>(a, s);
}

}  // namespace ikv
