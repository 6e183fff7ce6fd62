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

constexpr int kQueryWaves = 8;
constexpr int kKeep = 0;  // rows are read again by other workgroups
constexpr float kNaN = __builtin_nanf("");

typedef int __attribute__((ext_vector_type(4))) i32x4;
typedef const __attribute__((address_space(4))) i32x4* scalar_int4s;

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

// A set of ascending numbers given by bits (or counts), found by rank.  Lane i of the wave holds the i-th word of a run of 64 and the
// set bits of the words before it in the run; the run moves on as the ranks asked for grow.
struct Ranks {
    const uint64_t* words;
    int total_words, run;  // words in all, the run's first
    uint64_t word;         // the lane's
    int before, base, in_run;

    __device__ __forceinline__ void take() {
        const int i = run + (int)(threadIdx.x % kWave);
        word = i < total_words ? words[i] : 0;
        int sum = __popcll(word);
        const int mine = sum;
#pragma unroll
        for (int o = 1; o < kWave; o <<= 1) {
            const int up = __shfl_up(sum, o, kWave);
            if ((int)(threadIdx.x % kWave) >= o) sum += up;
        }
        before = sum - mine;
        in_run = __builtin_amdgcn_readlane(sum, kWave - 1);
    }
    __device__ __forceinline__ void start(const uint64_t* w, int n) {
        words = w;
        total_words = n;
        run = base = 0;
        take();
    }
    // The number with rank k, or -1 past the last.  Ranks do not fall from call to call.
    __device__ __forceinline__ int at(int k) {
        while (k >= base + in_run) {
            if (run + kWave >= total_words) return -1;
            base += in_run;
            run += kWave;
            take();
        }
        const int r = k - base, lane = __popcll(__ballot(before <= r)) - 1;
        // (lanes without bits have the next one's count: the last of those that are not above r holds it)
        const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)word, lane), hi = __builtin_amdgcn_readlane((int)(uint32_t)(word >> 32), lane);
        int left = r - __builtin_amdgcn_readlane(before, lane);
        uint64_t w = (uint64_t)hi << 32 | lo;
        int bit = 0;
#pragma unroll
        for (int half = 32; half >= 1; half >>= 1) {
            const int low = __popcll(w & ((1ull << half) - 1));
            if (left >= low) {
                left -= low;
                bit += half;
                w >>= half;
            }
        }
        return (run + lane) * 64 + bit;
    }
};

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
    if ((int)threadIdx.x < V) a.members[(size_t)b * V + threadIdx.x] = k == 0 && (int)threadIdx.x < count ? members[threadIdx.x] : -1;
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
// sum is of the rounded numbers).
template <typename T, int D, int CT, int kP, bool kShared>
__global__ __launch_bounds__(kWave* kQueryWaves, CT == 1 ? 4 : 2) void q4_query_kernel(Q4QueryArgs a) {
    constexpr int kThreads = kWave * kQueryWaves;
    constexpr int kKey = D / 32, kOut = D / 16;     // products per half, and for the output
    constexpr int kParts = sizeof(T) == 2 ? 1 : 3;  // bf16 parts of a query
    constexpr int kStride = D + 4;
    constexpr int kJoin = kQueryWaves / 2;          // waves whose outputs are joined through LDS at once
    constexpr bool kQLds = kParts * CT > 1;
    // [wave] values; in their place [joined wave][column][kStride] outputs; then [wave][column] maxima and sums; then the queries
    extern __shared__ float lds[];
    const Q4Dims& d = a.dims;
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int c = lane % 16, s = lane / 16;
    const int group = d.group, per = a.plan.per;

    // unit: KV heads fastest (eight of them fall on the eight XCDs), then the blocks, the last (a window's longest) first
    uint32_t x = blockIdx.x;
    const int g = x % (uint32_t)d.hkv;
    x /= (uint32_t)d.hkv;
    const int block = kShared ? 0 : a.plan.blocks - 1 - x % (uint32_t)a.plan.blocks;
    if constexpr (!kShared) x /= (uint32_t)a.plan.blocks;
    const int b = x % (uint32_t)d.batch;
    x /= (uint32_t)d.batch;
    const int layer = x % (uint32_t)a.layer_count, chunk = x / (uint32_t)a.layer_count;

    // the block's queries: the lane's in each column tile, its slot and row (-1: none)
    const int32_t* const members = kShared ? a.members + (size_t)b * a.plan.vectors : nullptr;
    Slot slot{0, 0, false};
    const int v0 = block * a.plan.vectors;
    if constexpr (kShared) {
        if (((scalar_ints)(uintptr_t)members)[0] < 0) return;
    } else {
        slot = slot_of(a, b);
        if (slot.bad && g == 0 && layer == 0 && chunk == 0 && threadIdx.x == 0) atomicOr(a.faults, kFaultCache);
        if (v0 >= slot.count) return;
    }
    const int part = c / group, head = c - part * group;
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
    int place[CT], from[CT];  // window: the query's position, and its window's first
    bool there[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        int sl = -1, row = 0;
        if (part < per) slot_row(ct, part, sl, row);
        there[ct] = sl >= 0;
        place[ct] = INT_MIN;
        from[ct] = INT_MAX;
        if constexpr (!kShared) {
            if (there[ct] && slot.n > 0) {
                const int r = slot.n - slot.count + row;
                place[ct] = a.cache.pos ? a.cache.pos[(size_t)b * d.cap + r] : r;
                from[ct] = lower_bound_of(place[ct], a.window);
            }
        }
    }

    // queries: bf16 of one column tile in registers, others as bf16 parts in LDS, [part][product][column tile][lane]
    u32x4 q[kQLds ? 1 : kKey];
    u32x4* const q_lds = reinterpret_cast<u32x4*>(lds + a.q_at) + lane;
    for (int ct = kQLds ? wave : 0; ct < CT; ct += kQLds ? kQueryWaves : 1) {
        int sl = -1, row = 0;
        if (part < per) slot_row(ct, part, sl, row);
        const T* qp = static_cast<const T*>(a.q) + layer * a.qs[0] + max(sl, 0) * a.qs[1] + (g * group + head) * a.qs[2] + (sl < 0 ? 0 : row) * a.qs[3] + s * (D / 4);
        if (sl < 0) qp = static_cast<const T*>(a.q) + s * (D / 4);  // (not used: any row)
        if constexpr (kParts == 1) {
#pragma unroll
            for (int j = 0; j < kKey; ++j) {
                const u32x4 w = reinterpret_cast<const u32x4*>(qp)[j], y = sl >= 0 ? w : u32x4{0, 0, 0, 0};
                if constexpr (kQLds) q_lds[(j * CT + ct) * kWave] = y;
                else q[j] = y;
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

    // the tiles: `total` of them, found by rank
    int total = 0, sink_tiles = 0, first_tile = 0, place_top = INT_MIN, place_low = INT_MAX;
    uint32_t all = 0;                          // shared: every query of the block
    int list_before = 0, list_slot = 0, items = 0;  // shared: lane i's member, and the pages that those before it list
    Ranks ranks{};
    const int per_page_shift = kShared ? max(0, d.page_shift - 5) : 0;
    if constexpr (kShared) {
        const int m = lane < a.plan.vectors ? members[lane] : -1;
        list_slot = max(m, 0);
        int sum = m >= 0 ? a.lists[m] : 0;
        const int mine = sum;
#pragma unroll
        for (int o = 1; o < kQ4MostVectors; o <<= 1) {
            const int up = __shfl_up(sum, o, kWave);
            if (lane >= o) sum += up;
        }
        list_before = sum - mine;
        items = __builtin_amdgcn_readlane(sum, kQ4MostVectors - 1);
        if (lane >= a.plan.vectors) list_before = INT_MAX;
        all = (uint32_t)__ballot(m >= 0);
        total = d.page_rows >= kTile ? items << per_page_shift : (items + 1) / 2;
    } else {
        int top = INT_MIN, low = INT_MAX;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
            if (there[ct]) {
                top = max(top, place[ct]);
                low = min(low, place[ct]);
            }
        place_top = __builtin_amdgcn_readfirstlane(wave_max_int(top));
        place_low = __builtin_amdgcn_readfirstlane(~wave_max_int(~low));
        if (slot.n > 0) {
            if (a.cache.pos) {
                ranks.start(a.visible + ((size_t)b * a.plan.blocks + block) * a.words, (slot.n + 64 * kTile - 1) / (64 * kTile));
                total = INT_MAX;
            } else {
                first_tile = max(0, lower_bound_of(place_low, a.window)) / kTile;
                sink_tiles = a.window ? min(a.sinks / kTile + (a.sinks % kTile != 0), first_tile) : 0;
                total = sink_tiles + place_top / kTile - first_tile + 1;
            }
        }
    }
    const int window_from = lower_bound_of(place_top, a.window);
    const int last = d.cap - 1;
    const scalar_ints table = (scalar_ints)(uintptr_t)(a.cache.table + (size_t)b * d.max_pages);
    auto item = [&](int i) __attribute__((always_inline)) {
        const int m = __popcll(__ballot(list_before <= i)) - 1;  // (of members without pages the last one, which has them)
        const int sl = __builtin_amdgcn_readlane(list_slot, m), at = i - __builtin_amdgcn_readlane(list_before, m);
        return ((scalar_int4s)(uintptr_t)a.items)[(size_t)sl * a.list_pages + at];
    };
    auto fetch = [&](int k, Ref& r) __attribute__((always_inline)) {  // whether there is a k-th tile
        if (k >= total) return false;
        if constexpr (kShared) {
            if (d.page_rows >= kTile) {
                const i32x4 it = item(k >> per_page_shift);
                r.row = (k & ((1 << per_page_shift) - 1)) * kTile;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    r.page[h] = it.x;
                    r.rows[h] = it.y - r.row - 16 * h;
                    r.mask[h] = (uint32_t)it.z;
                }
            } else {
                r.row = 0;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const bool is = 2 * k + h < items;
                    const i32x4 it = item(min(2 * k + h, items - 1));
                    r.page[h] = it.x;
                    r.rows[h] = is ? it.y : 0;
                    r.mask[h] = is ? (uint32_t)it.z : 0;
                }
            }
        } else {
            int t = k < sink_tiles ? k : first_tile + k - sink_tiles;
            if (a.cache.pos) t = ranks.at(k);
            if (t < 0) return false;
            r.row = t * kTile;
#pragma unroll
            for (int h = 0; h < 2; ++h) r.page[h] = table[min(r.row + 16 * h, last) >> d.page_shift];
        }
        return true;
    };
    uint32_t fault = 0;
    const uint8_t* const pool = a.cache.pool + q4_record(d, a.layer0 + layer, 0, g);
    const size_t page_bytes = (size_t)d.hkv * d.rec;
    auto locate = [&](const Ref& r, Half (&h)[2]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            int page = r.page[i], in;
            if constexpr (kShared) {
                h[i].valid = min(16, max(0, r.rows[i]));
                h[i].mask = h[i].valid ? r.mask[i] : 0;
                in = d.page_rows >= kTile ? r.row + 16 * i : 0;
            } else {
                const int row = r.row + 16 * i;
                h[i].valid = min(16, max(0, slot.n - row));
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
    const int32_t* const pos = kShared || !a.cache.pos ? nullptr : a.cache.pos + (size_t)b * d.cap;
    auto load_keys = [&](KeyTile<D>& t, const Half (&h)[2], int row) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if constexpr (D == 128) {
                const u32x4 w = *reinterpret_cast<const u32x4*>(h[i].k + ko);
#pragma unroll
                for (int j = 0; j < 4; ++j) t.codes[i][j] = w[j];
            } else {
                const u32x2 w = *reinterpret_cast<const u32x2*>(h[i].k + ko);
                t.codes[i][0] = w[0];
                t.codes[i][1] = w[1];
            }
            t.scale[i] = h[i].e[eo];
        }
        if (pos) t.pos = pos[min(row + lane % kTile, slot.n - 1)];
    };
    uint8_t* const value_lds = reinterpret_cast<uint8_t*>(lds) + wave * kValueBytes<D>;
    const uint8_t* const value_codes = value_lds + s * (D / 2) + c * (D / 32);
    const uint8_t* const value_scales = value_lds + kTile * (D / 2) + s * (D / 32) + (D == 128 ? c / 4 : c / 8);
    auto load_values = [&](const Half (&h)[2]) __attribute__((always_inline)) {
        if constexpr (D == 128) {
            to_lds<16, kKeep>(h[0].k + d.vc_off + lane * 16, value_lds);
            to_lds<16, kKeep>(h[1].k + d.vc_off + lane * 16, value_lds + 1024);
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
    if constexpr (kQLds) __syncthreads();

    // Loads run one tile ahead, page numbers two.
    const int step = a.plan.chunks * kQueryWaves;
    int k = chunk * kQueryWaves + wave;
    KeyTile<D> keys;
    Half now[2], next[2];
    Ref ref{}, ahead{};
    bool have = fetch(k, ref), more = false;
    if (have) {
        locate(ref, now);
        load_keys(keys, now, ref.row);
        load_values(now);
        more = fetch(k + step, ahead);
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
#pragma unroll
        for (int j = 0; j < kKey; ++j) {
            const u32x4 k0 = eight(keys.codes[0][j], key_scale[0]), k1 = eight(keys.codes[1][j], key_scale[1]);
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                if (skipped(ct)) continue;
#pragma unroll
                for (int p = kParts - 1; p >= 0; --p) {
                    u32x4 y;
                    if constexpr (kQLds) y = q_lds[((p * kKey + j) * CT + ct) * kWave];
                    else y = q[j];
                    z[ct][0] = mfma(k0, y, z[ct][0]);
                    z[ct][1] = mfma(k1, y, z[ct][1]);
                }
            }
        }
        const int tile_pos = keys.pos;
        // the lane's rows that its column does not see, a bit each: bit j is row 4 (j % 4) + s of half j / 4.  (Without branches: the
        // compiler, ROCm 7.2's, dropped the first element's store from the same conditions joined by ||.)
        auto hidden = [&](uint32_t (&bits)[CT]) __attribute__((always_inline)) {
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) bits[ct] = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int half = j / 4, in = 4 * (j % 4) + s;
                int p = row + 16 * half + in;
                if constexpr (!kShared)
                    if (pos) p = __shfl(tile_pos, 16 * half + in, kWave);
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) {
                    uint32_t h = in >= now[half].valid;
                    if constexpr (kShared) h |= ~(now[half].mask >> (ct * per + part)) & 1u;
                    else h |= (uint32_t)(p > place[ct]) | ((uint32_t)(p < from[ct]) & (uint32_t)(p >= a.sinks));
                    bits[ct] |= h << j;
                }
            }
        };
        bool plain = whole;  // every column sees every row
        if constexpr (kShared) {
            plain = plain && (now[0].mask & now[1].mask) == all;
        } else {
            const int p = pos ? tile_pos : row + lane % kTile;
            plain = plain && __all(p <= place_low && (p >= window_from || p < a.sinks));
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
            float top = z[ct][0][0];
#pragma unroll
            for (int j = 1; j < 8; ++j) top = fmaxf(top, z[ct][j / 4][j % 4]);
            top *= a.scale2;
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
            k += step;
            more = fetch(k + step, ahead);
        }
    }
    if (fault && lane == 0) atomicOr(a.faults, fault);

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
                stat[(kQueryWaves + wave) * kColumns + 16 * ct + c] = l[ct];
            }
        }
    };
    if (wave >= kJoin) put();
    __syncthreads();
    if (wave < kJoin) {
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            const float m2 = stat[(wave + kJoin) * kColumns + 16 * ct + c], l2 = stat[(kQueryWaves + wave + kJoin) * kColumns + 16 * ct + c];
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
        const int vt = col % 16 / group, h = col % 16 - vt * group;
        int sl = -1, row = 0;
        if (vt < per) slot_row(col / 16, vt, sl, row);
        if (sl < 0) continue;
        float top = stat[col];
#pragma unroll
        for (int w = 1; w < kJoin; ++w) top = fmaxf(top, stat[w * kColumns + col]);
        float sum = 0.0f;
        f32x4 o{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < kJoin; ++w) {
            const float f = exp2_hw(stat[w * kColumns + col] - top);
            sum += f * stat[(kQueryWaves + w) * kColumns + col];
            o += *reinterpret_cast<const f32x4*>(lds + (w * kColumns + col) * kStride + e) * f;
        }
        if (a.plan.chunks == 1) {
            const float inv = sum != 0.0f ? 1.0f / sum : 0.0f;
            T* op = static_cast<T*>(a.o) + layer * a.os[0] + sl * a.os[1] + (g * group + h) * a.os[2] + row * a.os[3] + e;
            o *= inv;
            if constexpr (sizeof(T) == 2) *reinterpret_cast<u32x2*>(op) = u32x2{pack2(o[0], o[1]), pack2(o[2], o[3])};
            else *reinterpret_cast<f32x4*>(op) = o;
        } else {
            // (a part without rows for the query is its sum, 0, alone)
            const size_t at = ((((size_t)layer * d.batch + sl) * a.rows + row) * d.hq + g * group + h) * a.plan.chunks + chunk;
            if (sum != 0.0f) *reinterpret_cast<f32x4*>(a.opart + at * D + e) = o;
            if (e == 0) a.part[at] = make_float2(top, sum);
        }
    }
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

template <typename T, int D, int CT, int kP, bool kShared>
hipError_t launch_form(Q4QueryArgs a, hipStream_t s) {
    constexpr int kJoined = kQueryWaves / 2 * CT * 16 * (D + 4) * (int)sizeof(float), kValues = kQueryWaves * kValueBytes<D>;
    constexpr int kParts = sizeof(T) == 2 ? 1 : 3, kStat = 2 * kQueryWaves * CT * 16;
    static_assert(kJoined % 16 == 0 && kValues % 16 == 0 && kStat % 4 == 0, "queries are read 16 bytes at a time");
    a.stat_at = (kJoined > kValues ? kJoined : kValues) / (int)sizeof(float);
    a.q_at = a.stat_at + kStat;
    const size_t lds = (size_t)a.q_at * sizeof(float) + (kParts * CT > 1 ? (size_t)kParts * (D / 32) * CT * kWave * sizeof(u32x4) : 0);
    auto kern = q4_query_kernel<T, D, CT, kP, kShared>;
    if (lds > 64 * 1024) {
        static std::atomic<bool> raised[kMaxDevices];
        const hipError_t e = raise_lds_limit(reinterpret_cast<const void*>(kern), raised);
        if (e != hipSuccess) return e;
    }
    const uint32_t blocks = kShared ? 1 : a.plan.blocks;
    hipLaunchKernelGGL(kern, dim3((uint32_t)a.dims.hkv * blocks * a.dims.batch * a.layer_count * a.plan.chunks), dim3(kWave * kQueryWaves), lds, s, a);
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

template <typename T, int D, bool kShared>
hipError_t launch_tiles(const Q4QueryArgs& a, hipStream_t s) {
    if constexpr (sizeof(T) == 2)
        if (a.plan.tiles == 2) return launch_form<T, D, 2, 1, kShared>(a, s);
    return launch_form<T, D, 1, 3, kShared>(a, s);
}
template <bool kShared>
hipError_t launch_queries(const Q4QueryArgs& a, hipStream_t s) {
    if (a.dims.bf16) return a.dims.d == 128 ? launch_tiles<bf16_t, 128, kShared>(a, s) : launch_tiles<bf16_t, 64, kShared>(a, s);
    return a.dims.d == 128 ? launch_tiles<float, 128, kShared>(a, s) : launch_tiles<float, 64, kShared>(a, s);
}

// Workgroups that divide a block's `tiles` tiles: until there are two for every CU, each with a tile for every wave at least.
int chunks_of(int64_t units, int tiles) {
    const int cus = device_cus() > 0 ? device_cus() : 256;
    const int64_t want = (2 * cus + units - 1) / units, most = (tiles + kQueryWaves - 1) / kQueryWaves;
    return (int)(want < most ? want : most > 0 ? most : 1);
}

}  // namespace

Q4QueryPlan q4_window_plan(const Q4Dims& d, int layer_count, int n_max, int rows, int window, int sinks) {
    Q4QueryPlan p{};
    p.per = 16 / d.group;
    p.tiles = d.bf16 && rows > p.per ? 2 : 1;
    p.vectors = p.tiles * p.per;
    p.blocks = (rows + p.vectors - 1) / p.vectors;
    int64_t tiles = (n_max + kTile - 1) / kTile;
    if (window) {  // (rows in order, in a window that ends inside tiles)
        const int64_t seen = ((int64_t)window + sinks + p.vectors) / kTile + 3;
        tiles = tiles < seen ? tiles : seen;
    }
    p.chunks = chunks_of((int64_t)layer_count * d.batch * d.hkv * p.blocks, (int)tiles);
    return p;
}

Q4QueryPlan q4_shared_plan(const Q4Dims& d, int layer_count, int n_max) {
    Q4QueryPlan p{};
    p.per = 16 / d.group;
    p.tiles = d.bf16 && d.batch > p.per ? 2 : 1;
    p.vectors = p.tiles * p.per;
    p.blocks = (d.batch + p.vectors - 1) / p.vectors;
    p.chunks = chunks_of((int64_t)layer_count * d.hkv * p.blocks, (n_max + kTile - 1) / kTile);
    return p;
}

hipError_t launch_q4_window(const Q4QueryArgs& a, hipStream_t s) {
    if (a.cache.pos) {
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
