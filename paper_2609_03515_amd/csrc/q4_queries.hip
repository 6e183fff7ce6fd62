// Attention of blocks of queries over the paged 4-bit cache: o = softmax(q . k / sqrt(d)) v over the rows that a query sees.
//
// Window: the queries are those of a slot's newest rows; query at position P sees the rows at positions p <= P that are in the
// window, p > P - window, or among the first, p < sinks.  Shared: one query of each of several slots; where their tables name the
// same page it is read and converted once for all of them.
//
// With z = q . k / sqrt(d) log2(e), a wave keeps for each query m >= max z - kSlack, l = sum 2^(z - m) and acc = sum 2^(z - m) v in
// 32 bits and passes over its rows once; (m, l, acc) of two sets of rows join as m = max(m1, m2), l = l1 2^(m1 - m) + l2 2^(m2 - m).
//
// A block of queries is one to four column tiles, each `per` queries of the group's heads in 16 columns (per = 16 / group); the tiles of
// 32 rows, their products, probabilities and values are those of the decode attention (q4_attend.hip), with each converted tile used
// by every column tile.  A workgroup takes a block and one KV head; its waves take the block's tiles of rows in turn, each with a running
// maximum, sum and output of its own, joined in LDS at the end.  Where there are few blocks their tiles are divided among workgroups,
// whose parts a second kernel joins (4 us).
//
// Which tiles: a wave looks at 64 of its tiles at a time, one a lane, and reads the pages of all of them with one load each.  Without
// positions the rows are in order, and the tiles of a window are found from row numbers.  With positions (an eviction leaves rows of any
// position in any place) the wave reads the positions of its tiles' rows; where it would have many of them a kernel before this one
// marks the tiles of which a block sees any row, a bit each, once for all layers and heads.  Shared: a lane looks at a tile of one slot,
// and at the table entries of the block's other slots there; the first slot with a page has the tile for all that have it.
//
// What bounds it.  One query of each of a few slots, and short windows: latency, the dependent loads len -> table -> records (0.6 to
// 0.8 us each), one tile's 1.1 us, the start of a workgroup, and the join; the 8B layer at its budget takes 13 us and a join of 4, its
// bytes 1.9.  Many shared pages: the bytes of the pages that are read, each once (32 layers of 8 evicted samples: 206 MB, 65 us, 3.2 TB/s
// with each workgroup's start and the join of its eight waves).  A long chunk: vector instructions beside the products (2,048 queries on
// 32,768 rows, 8 KV heads of 4 heads: 1,085 us, 982 TFLOP/s where a product of 8,192 x 8,192 matrices reaches 1,447).  There a tile of 32
// rows takes a wave 374 of them for 64 columns, 64 of which are the products: counters show the SIMDs issuing for 65% of the time and the
// matrix units busy for 40%.  Short ragged chunks (55 us for products of 10) and groups of 7 heads (46 us for bytes of 12): vector
// instructions as well, 62% and 55% of the time, with the matrix units at 14% and 18%; a wave waits for 40% and 35% of its time.
//
// Masked rows get the logit -inf.  A masked row's values may be NaN (a block stored from infinities), or, in rows that were never
// stored, codes of a scale byte of 253 or 254 that exceed the largest bf16 number; 0 times them would spoil the column, so tiles that
// hold such blocks take a side path.  NaN blocks are taken as numbers, and a product of two 0/1 matrices finds the outputs whose query
// sees one; the tile's values are added in quarters, which are bf16 numbers.
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

constexpr int kKeep = 0;  // rows are read again by other workgroups
constexpr float kNaN = __builtin_nanf("");

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
    // (a slot that cannot be has queries, which get zeros, and no rows)
    const int first = slot.n - slot.count + v0, queries = slot.bad ? 0 : min(a.plan.vectors, slot.count - v0);
    int top = INT_MIN, low = INT_MAX;
    for (int i = lane; i < queries; i += kWave) {
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

// Shared, more than 64 slots: the slots of a group in ascending order are cut into blocks of `vectors`; whether a slot begins one,
// and the slots of that.  One wave per slot.
__global__ __launch_bounds__(kWave) void q4_block_kernel(Q4QueryArgs a) {
    __shared__ int members[kQ4MostVectors];
    const Q4Dims& d = a.dims;
    const int lane = threadIdx.x, b = blockIdx.x, V = a.plan.vectors, mine = a.group[b];
    int seen = 0, rank = -1;  // slots of the group so far, and those before b
    for (int i0 = 0; i0 < d.batch; i0 += kWave) {
        const int i = i0 + lane;
        const bool same = i < d.batch && a.group[i] == mine;
        const uint64_t all = __ballot(same);
        const int r = seen + __popcll(all & ((1ull << lane) - 1));
        seen += __popcll(all);
        if (i0 <= b && b < i0 + kWave) {
            rank = __builtin_amdgcn_readlane(r, b - i0);
            if (rank % V) break;
        }
        if (same && rank >= 0 && r >= rank && r < rank + V) members[r - rank] = i;
        if (rank >= 0 && seen >= rank + V) break;
    }
    const bool head = rank % V == 0;
    __syncthreads();
    if (lane == 0) a.heads[b] = head;
    if (head && lane < V) a.members[(size_t)b * V + lane] = lane < seen - rank ? members[lane] : -1;
}

// A tile that is to be loaded: its first row, how many of its rows there are, its halves' pages, and (shared) the queries of the block
// that see it.
struct Ref {
    int row, rows, page[2];
    uint32_t mask;
};
struct Half {
    const uint8_t* k;  // the half's first row: keys' codes, ...
    const uint8_t* e;  // ... scales, and the values' of both vc_off bytes on
    int valid;         // rows that take part
};
template <int D>
struct KeyTile {
    uint32_t codes[2][D / 32];
    uint32_t scale[2];
    int pos;  // position of row `lane % 32` (window with positions)
};

// Column tiles (CT) of 16; parts of a probability (kP): 3 take all of its 24 bits, 1 rounds it to bf16 (8 bits, to nearest; its
// sum is of the rounded numbers, so that a row of equal values comes out exact).  Blocks of bf16 queries with more than one column tile
// round: a weight is off by 2^-8 of itself at most, as a bf16 output is, and its error in an average over many rows is less.  With 3 parts
// those forms spill and wait for the products: a chunk of 2,048 queries on 32,768 rows takes 2.2 times as long, 32 layers of 8 samples 140
// us for 65, two layers of 32 samples of three prompts 76 for 46, one layer of 16 samples 27 for 21, short ragged chunks 81 for 55.  Where
// one column tile is enough nothing waits for the products, and all bits are kept (rounded, the 8B layer would take 1 of its 17 us less).
// (One column tile of 128 elements has a few registers too few for four waves a SIMD: with three, and none spilled, 2,048 slabs of 3,277
// rows take 176 us for 183 seen whole, and 167 for 156 in a masked window.)  kWaves: of a workgroup, which divide a block's tiles and join
// their outputs.
template <typename T, int D, int CT, int kP, bool kShared, int kWaves>
__global__ __launch_bounds__(kWave* kWaves, CT == 1 ? 4 : CT == 2 ? 3 : 2) void q4_query_kernel(Q4QueryArgs a) {
    constexpr int kThreads = kWave * kWaves;
    constexpr int kKey = D / 32, kOut = D / 16;     // products per half, and for the output
    constexpr int kParts = sizeof(T) == 2 ? 1 : 3;  // bf16 parts of a query
    // [wave] values and the queries; in their place the outputs that are joined; then [wave][column] maxima and sums
    extern __shared__ float lds[];
    const Q4Dims& d = a.dims;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int group = d.group, per = a.plan.per;
    // The arguments that only the later batches of tiles and the end need, in LDS: in scalar registers they would be spilled, and a
    // scalar load of an argument in the middle of the kernel takes 1.5 us (arguments lie in host memory).
    constexpr int kArgWords = sizeof(Q4QueryArgs) / 4;
    __shared__ __align__(16) uint32_t arg_words[kArgWords];
    static_assert(sizeof(Q4QueryArgs) % 4 == 0, "copied by words");
    for (int i = threadIdx.x; i < kArgWords; i += kThreads) arg_words[i] = ((const uint32_t*)__builtin_amdgcn_kernarg_segment_ptr())[i];
    const Q4QueryArgs& late = *reinterpret_cast<const Q4QueryArgs*>(arg_words);

    // unit: KV heads fastest (eight of them fall on the eight XCDs); then a window's blocks, the last, its longest, first.  Shared: the
    // blocks slowest, since there may be fewer of them.
    uint32_t x = blockIdx.x;
    auto take = [&](int n) __attribute__((always_inline)) {
        const int i = x % (uint32_t)n;
        x /= (uint32_t)n;
        return i;
    };
    const int g = take(d.hkv);
    int nth = kShared ? 0 : take(a.plan.blocks), b = kShared ? 0 : take(d.batch);
    const int layer = take(a.layer_count), chunk = take(a.plan.chunks);
    if constexpr (kShared) nth = x;
    const size_t page_bytes = (size_t)d.hkv * d.rec;
    const int step = a.plan.chunks * kWaves, k0 = chunk * kWaves + wave;
    uint32_t fault = 0;

  // Shared: a workgroup takes the nth block, and those `blocks` further on, where small groups make more than there are places for.
  for (int turn = nth;; turn += a.plan.blocks) {
    int lane = threadIdx.x % kWave;
    if constexpr (kShared) asm volatile("" : "+v"(lane));  // (nothing of a lane is worked out before the loop and kept over it)
    const int c = lane % 16, s = lane / 16, part = c / group, head = c - part * group;
    const uint8_t* const pool = a.cache.pool + q4_record(d, a.layer0 + layer, 0, g);
    // shared: the block's slots (-1: none) and their rows
    __shared__ int member_of[kShared ? kQ4MostVectors : 1], rows_of[kShared ? kQ4MostVectors : 1];
    if constexpr (kShared) {
        const int V = a.plan.vectors;
        if (wave == 0) {
            int at = lane < V ? lane : -1, it = -1, raw = 0;  // the lane's slot `it`, of `raw` rows, is the block's query `at`
            if (a.heads) {
                int seen = 0;
                b = -1;
                for (int i0 = 0; i0 < d.batch && b < 0; i0 += kWave) {
                    const uint64_t is = __ballot(i0 + lane < d.batch && a.heads[min(i0 + lane, d.batch - 1)]);
                    const uint64_t found = __ballot((is >> lane & 1) && seen + __popcll(is & ((1ull << lane) - 1)) == turn);
                    if (found) b = i0 + __builtin_ctzll(found);
                    seen += __popcll(is);
                }
                if (b >= 0 && lane < V) it = a.members[(size_t)b * V + lane];
                if (it >= 0) raw = a.cache.len[it];
            } else {
                // up to 64 slots, one a lane: as q4_block_kernel.  (Ranks a group at a time, and lengths beside the groups' numbers: the
                // 32 layers of 8 samples take 3 us less so, one layer of 16 1 us.)
                it = min(lane, d.batch - 1);
                const int mine = a.group[it];
                raw = a.cache.len[it];
                const bool is = lane < d.batch;
                int rank = 0;
                for (uint64_t rest = __ballot(is); rest;) {  // a group at a time
                    const uint64_t same = __ballot(is && mine == __builtin_amdgcn_readlane(mine, __builtin_ctzll(rest)));
                    if (same >> lane & 1) rank = __popcll(same & ((1ull << lane) - 1));
                    rest &= ~same;
                }
                const uint64_t heads = __ballot(is && rank % V == 0);
                const uint64_t found = __ballot((heads >> lane & 1) && __popcll(heads & ((1ull << lane) - 1)) == turn);
                if (lane < V) member_of[lane] = -1;
                at = -1;
                if (found) {
                    const int begin = __builtin_ctzll(found), r = rank - __builtin_amdgcn_readlane(rank, begin);
                    if (is && mine == __builtin_amdgcn_readlane(mine, begin) && r >= 0 && r < V) at = r;
                }
            }
            if (at >= 0) {
                const bool bad = raw < 0 || raw > a.n_max;
                member_of[at] = it;
                rows_of[at] = bad ? 0 : raw;
                if (bad && layer == 0 && g == 0 && chunk == 0) atomicOr(a.faults, kFaultCache);
            }
        }
        __syncthreads();
        if (member_of[0] < 0) break;
    }
    // the block's queries: the lane's in each column tile, its slot and row (-1: none)
    const int block = kShared ? 0 : a.plan.blocks - 1 - nth, v0 = block * a.plan.vectors;
    // The wave's tiles are those of numbers k0, k0 + step, ...  It looks at 64 of them at a time, one a lane: the pages of the lane's tile,
    // and a bit for each that takes part.
    // Shared: a lane looks at one tile of one of the block's slots.  Where several name the same pages there, and as many rows, the first
    // of them has the tile for all.  The later slots' tiles are dealt from other waves on, so that those that only they have (behind a
    // prompt, say) do not meet in the waves that have the prompt's last tiles.
    constexpr int kTogether = 8;
    const int at_once = kShared ? kWave >> a.plan.vector_shift : kWave;
    const int32_t* const pos = kShared || !a.cache.pos ? nullptr : a.cache.pos + (size_t)b * d.cap;
    int run = 0;            // shared: tiles of a wave
    uint32_t all = 0;       // shared: every query of the block
    if constexpr (kShared) {
        const int V = a.plan.vectors, sl = lane < V ? member_of[lane] : -1, n = sl >= 0 ? rows_of[min(lane, V - 1)] : 0;
        all = (uint32_t)__ballot(sl >= 0);
        run = ((__builtin_amdgcn_readfirstlane(wave_max_int(n)) + kTile - 1) / kTile + step - 1) / step;
    }
    // (of a lane's tile: the pages of its halves; shared: its first row and rows, and the queries that see it)
    int page_of = 0, page_of2 = 0, row_of = 0, rows_in = 0, held[kTogether];
    uint32_t mask_of = 0;
    uint64_t left = 0, word = 0;
    int base = 0;
    const int how = kShared || !pos ? 0 : a.visible ? 1 : 2;  // window: how tiles are found, by row numbers, marks or positions
    auto load_entries = [&](const Q4QueryArgs& a, int row, int v0, int (&to)[kTogether]) __attribute__((always_inline)) {  // shared: of the block's slots v0 ... at a row
        const int entries = a.dims.max_pages, V = a.plan.vectors, at = min(row, a.dims.cap - 1) >> a.dims.page_shift;
#pragma unroll
        for (int i = 0; i < kTogether; ++i) to[i] = a.cache.table[(size_t)max(member_of[min(v0 + i, V - 1)], 0) * entries + at];
    };
    auto load_look = [&](const Q4QueryArgs& a) __attribute__((always_inline)) {
        int lane = threadIdx.x % kWave;
        asm volatile("" : "+v"(lane));  // (its places are worked out here, not kept over the tiles)
        const int last = a.dims.cap - 1, shift = a.dims.page_shift;
        if constexpr (kShared) {
            const int V = a.plan.vectors, own = lane & ((1 << a.plan.vector_shift) - 1), i = lane >> a.plan.vector_shift;
            const int wave_of = k0 + min(own, V - 1) * max(1, step / V);
            // (a tile behind a full slot has no rows: only the table's index ends at the capacity)
            const int row = ((wave_of < step ? wave_of : wave_of % step) + (base + i) * step) * kTile;
            row_of = row;
            rows_in = own < V && base + i < run && member_of[min(own, V - 1)] >= 0 ? min(kTile, rows_of[min(own, V - 1)] - row) : 0;
            const int32_t* const entry = a.cache.table + (size_t)(own < V ? max(member_of[own], 0) : 0) * a.dims.max_pages;
            page_of = entry[min(row, last) >> shift];
            page_of2 = entry[min(row + 16, last) >> shift];
            load_entries(a, row, 0, held);
        } else {
            const int k = k0 + (base + lane) * step, row = min(k * kTile, last);  // (2^27 rows are 2^22 tiles, and 64 steps fewer than 2^25)
            const int32_t* const entry = a.cache.table + (size_t)b * a.dims.max_pages;
            page_of = entry[row >> shift];
            page_of2 = entry[min(row + 16, last) >> shift];
            if (how == 1) {
                word = a.visible[((size_t)b * a.plan.blocks + block) * a.words + min(k / 64, a.words - 1)];
            } else if (how == 2) {  // two tiles to a load
#pragma unroll
                for (int i = 0; i < kTogether; ++i) held[i] = pos[min((k0 + (base + 2 * i + lane / kTile) * step) * kTile + lane % kTile, last)];
            }
        }
    };
    load_look(a);  // (on their way while the queries are)
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
            sl = member_of[v];
        } else {
            row = v0 + v;
            if (row >= slot.count) sl = -1;
        }
    };
    int place[kShared ? 1 : CT];  // window: the positions of the lane's columns (no query: the lowest)
    if constexpr (!kShared) {
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            int sl = -1, row = 0;
            if (part < per) slot_row(ct, part, sl, row);
            const int r = max(0, slot.n - slot.count + row);
            place[ct] = a.cache.pos ? a.cache.pos[(size_t)b * d.cap + min(r, d.cap - 1)] : r;
            if (sl < 0 || slot.n == 0) place[ct] = INT_MIN;
        }
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
        const int64_t at = layer * a.qs[0] + max(sl, 0) * a.qs[1] + (g * group + (sl < 0 ? 0 : head)) * a.qs[2] + (sl < 0 ? 0 : row) * a.qs[3];
        const T* const qp = static_cast<const T*>(a.q) + at + s * (D / 4);
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

    __shared__ int places[kShared ? 1 : CT * 16];
    int top_place = INT_MIN, low_place = INT_MAX;
    if constexpr (!kShared) {
        int top = INT_MIN, low = INT_MAX;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            const bool is = part < per && v0 + ct * per + part < slot.count;
            if (is) {
                top = max(top, place[ct]);
                low = min(low, place[ct]);
            }
            if (wave == 0 && s == 0) places[16 * ct + c] = place[ct];
        }
        top_place = __builtin_amdgcn_readfirstlane(wave_max_int(top));
        low_place = __builtin_amdgcn_readfirstlane(~wave_max_int(~low));
    }
    const int top_from = lower_bound_of(top_place, a.window), low_from = lower_bound_of(low_place, a.window);
    const int tiles = kShared ? 0 : (slot.n + kTile - 1) / kTile;
    auto look = [&]() __attribute__((always_inline)) {
        int lane = threadIdx.x % kWave;
        asm volatile("" : "+v"(lane));
        bool part_of;
        if constexpr (kShared) {
            const int V = late.plan.vectors, own = lane & ((1 << late.plan.vector_shift) - 1);
            const bool pairs = late.dims.page_rows < kTile;
            // The slots' rows, one a lane (-1: no slot), taken from there: from LDS for each, one layer of 16 samples takes 1 us more.
            const int n = lane < V && member_of[min(lane, V - 1)] >= 0 ? rows_of[min(lane, V - 1)] : -1;
            mask_of = 0;
            for (int v0 = 0; v0 < V; v0 += kTogether) {
                if (v0) load_entries(late, row_of, v0, held);
                int second[kTogether];
                if (pairs) load_entries(late, row_of + 16, v0, second);
#pragma unroll
                for (int i = 0; i < kTogether; ++i) {
                    const int v = min(v0 + i, V - 1), left_of = __builtin_amdgcn_readlane(n, v) - row_of;
                    const bool same = held[i] == page_of && (!pairs || rows_in <= 16 || second[i] == page_of2) && min(kTile, left_of) == rows_in;
                    mask_of |= (uint32_t)same << v;
                }
            }
            part_of = rows_in > 0 && __builtin_ctz(mask_of) == own;
        } else {
            const int k = k0 + (base + lane) * step, row = k * kTile;
            part_of = k < tiles;
            if (how == 0) {
                part_of = part_of && row <= top_place && (row + kTile > low_from || row < a.sinks);
            } else if (how == 1) {
                part_of = part_of && (word >> k % 64 & 1);
            } else {
                uint64_t bits = 0;
                for (int i0 = 0; i0 < kWave && k0 + (base + i0) * step < tiles; i0 += 2 * kTogether) {
                    const int last = late.dims.cap - 1;
#pragma unroll
                    for (int i = 0; i < kTogether; ++i)
                        if (i0) held[i] = pos[min((k0 + (base + i0 + 2 * i + lane / kTile) * step) * kTile + lane % kTile, last)];
#pragma unroll
                    for (int i = 0; i < kTogether; ++i) {
                        const int r = (k0 + (base + i0 + 2 * i + lane / kTile) * step) * kTile + lane % kTile;
                        const uint64_t any = __ballot(r < slot.n && held[i] <= top_place && (held[i] >= low_from || held[i] < a.sinks));
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
        const int i = __builtin_ctzll(left);
        left &= left - 1;
        r.page[0] = __builtin_amdgcn_readlane(page_of, i);
        r.page[1] = __builtin_amdgcn_readlane(page_of2, i);
        if constexpr (kShared) {
            r.row = __builtin_amdgcn_readlane(row_of, i);
            r.rows = __builtin_amdgcn_readlane(rows_in, i);
            r.mask = __builtin_amdgcn_readlane(mask_of, i);
        } else {
            r.row = (k0 + (base + i) * step) * kTile;
            r.rows = slot.n - r.row;
        }
        return true;
    };
    auto locate = [&](const Ref& r, Half (&h)[2]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            int page = r.page[i];
            h[i].valid = __builtin_amdgcn_readfirstlane(min(16, max(0, r.rows - 16 * i)));
            if ((uint32_t)page >= (uint32_t)d.n_pages) {
                if (h[i].valid) fault = kFaultCache;
                page = h[i].valid = 0;
            }
            const int in = (r.row + 16 * i) & (d.page_rows - 1);
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
   if (kShared ? run > 0 : k0 < tiles)
   for (;;) {
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
        if constexpr (kShared && CT > 1) active = ref.mask;
        auto skipped = [&](int ct) __attribute__((always_inline)) {
            return kShared && CT > 1 && !(active >> (ct * per) & ((1u << per) - 1));
        };
        // Two waves meet on a SIMD; one that is past its logits goes first, so that they do not run side by side through the products
        // and then through the exponentials (a chunk of 2,048 queries on 32,768 rows takes 80 us more without).
        if constexpr (CT == 4) __builtin_amdgcn_s_setprio(0);
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
        if constexpr (CT == 4) __builtin_amdgcn_s_setprio(1);
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
                    if constexpr (kShared) h |= ~(ref.mask >> (ct * per + part)) & 1u;
                    else h |= (uint32_t)(p[j] > place) | ((uint32_t)(p[j] < from) & (uint32_t)(p[j] >= a.sinks));
                    bits[ct] |= h << j;
                }
            }
        };
        bool plain = whole;  // every column sees every row
        if constexpr (kShared) {
            plain = plain && ref.mask == all;
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
        // (one branch for all column tiles: a maximum is raised in a few tiles only.  A column tile that is left out has logits 0 here,
        // and its maximum is not looked at again until it takes part.)
        float top[CT];
        bool raise = false;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            top[ct] = max3(z[ct][0][0], z[ct][0][1], z[ct][0][2]);
            top[ct] = max3(top[ct], z[ct][0][3], z[ct][1][0]);
            top[ct] = max3(top[ct], z[ct][1][1], z[ct][1][2]);
            top[ct] = max3(top[ct], z[ct][1][3], z[ct][1][3]) * a.scale2;
            raise |= top[ct] > m[ct] + kSlack && !skipped(ct);
        }
        if (__any(raise)) {
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                if (skipped(ct)) continue;
                const float all_top = rows_allmax(top[ct]);
                const float raised = all_top > m[ct] + kSlack ? all_top : m[ct];
                const float f = exp2_hw(m[ct] - raised);
                m[ct] = raised;
                l[ct] *= f;
#pragma unroll
                for (int e = 0; e < kOut; ++e) acc[ct][e] *= f;
            }
        }
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            if (skipped(ct)) continue;
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
        bool odd = false;  // a block whose numbers are not all bf16 ones
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int r = 16 * (j / 4) + 4 * (j % 4);  // (and s)
            if constexpr (D == 128) codes[j] = *reinterpret_cast<const uint32_t*>(value_codes + r * (D / 2));
            else codes[j] = *reinterpret_cast<const uint16_t*>(value_codes + r * (D / 2));
            const uint32_t byte = value_scales[r * (D / 32)];
            scale[j] = __uint_as_float(byte << 23);
            odd |= byte > 252u;
        }
        if (!whole) {
            asm volatile("");
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (4 * (j % 4) >= now[j / 4].valid - s) scale[j] = 1.0f;
        }
        const bool quarters = __any(odd);
        if (__builtin_expect(quarters, 0)) {  // (out of the way: a chunk of 2,048 queries on 32,768 rows takes 9 us less)
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
            // (rows that were stored have scales of 2^-100 and up, of which a quarter is exact)
#pragma unroll
            for (int j = 0; j < 8; ++j) scale[j] *= 0.25f;
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int e = 0; e < kOut; ++e) acc[ct][e] *= 0.25f;
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
        if (__builtin_expect(quarters, 0)) {
            asm volatile("");
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int e = 0; e < kOut; ++e) acc[ct][e] *= 4.0f;
        }
        have = more;
        if (more) {
            now[0] = next[0];
            now[1] = next[1];
            ref = ahead;
            more = fetch(ahead);
        }
    }
    base += at_once;
    if (kShared ? base >= run : k0 + base * step >= tiles) break;
    load_look(late);
   }
    // The outputs are blocks of 64 lanes' four elements (column c, elements s D / 4 + i kOut + 4 half ...), each joined by one wave: the
    // others' come through LDS, in the place of values and queries, with every wave's maxima and sums.
    constexpr int kColumns = CT * 16, kHalves = kOut / 4, kBlocks = CT * 4 * kHalves;
    float* const stat = lds + a.stat_at;  // [wave][column] maxima, then sums
    f32x4* const parts = reinterpret_cast<f32x4*>(lds) + lane;
    __syncthreads();
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) l[ct] = rows_allsum(l[ct]);
    auto block_of = [&](int q) __attribute__((always_inline)) {
        const int ct = q / (4 * kHalves), i = q / kHalves % 4, e = q % kHalves * 4;
        return f32x4{acc[ct][e][i], acc[ct][e + 1][i], acc[ct][e + 2][i], acc[ct][e + 3][i]};
    };
    if constexpr (kWaves > 1) {
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
            if (s == 0) {
                stat[wave * kColumns + 16 * ct + c] = m[ct];
                stat[(kWaves + wave) * kColumns + 16 * ct + c] = l[ct];
            }
#pragma unroll
        for (int q = 0; q < kBlocks; ++q) {
            const int owner = q % kWaves;
            if (wave != owner) parts[(q * (kWaves - 1) + (wave > owner ? wave - 1 : wave)) * kWave] = block_of(q);
        }
        __syncthreads();
    }
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
        int sl = -1, row = 0;
        if (part < per) slot_row(ct, part, sl, row);
        if (sl < 0) continue;
        float top = m[ct], sum = l[ct], f[kWaves];
        if constexpr (kWaves > 1) {
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                f[w] = stat[w * kColumns + 16 * ct + c];
                top = fmaxf(top, f[w]);
            }
            sum = 0.0f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                f[w] = exp2_hw(f[w] - top);
                sum += f[w] * stat[(kWaves + w) * kColumns + 16 * ct + c];
            }
        }
        const int h = g * group + head, chunks = late.plan.chunks;
        const float inv = sum != 0.0f ? 1.0f / sum : 0.0f;
        T* const op = static_cast<T*>(late.o) + layer * late.os[0] + sl * late.os[1] + h * late.os[2] + row * late.os[3] + s * (D / 4);
        const size_t at = ((((size_t)layer * late.dims.batch + sl) * late.rows + row) * late.dims.hq + h) * chunks + chunk;
        float* const pp = late.opart + at * D + s * (D / 4);
        if (chunks > 1 && wave == 0 && s == 0) late.part[at] = make_float2(top, sum);
#pragma unroll
        for (int x = 0; x < 4 * kHalves; ++x) {
            const int q = ct * 4 * kHalves + x;
            if (wave != q % kWaves) continue;
            f32x4 o = block_of(q);
            if constexpr (kWaves > 1) {
                o *= exp2_hw(m[ct] - top);
#pragma unroll
                for (int w = 0; w < kWaves; ++w)
                    if (w != q % kWaves) o += parts[(q * (kWaves - 1) + (w > q % kWaves ? w - 1 : w)) * kWave] * f[w];
            }
            const int e = x / kHalves * kOut + x % kHalves * 4;
            if (chunks > 1) {
                // (a part without rows for the query is its sum, 0, alone)
                if (sum != 0.0f) *reinterpret_cast<f32x4*>(pp + e) = o;
            } else {
                o *= inv;
                if constexpr (sizeof(T) == 2) *reinterpret_cast<u32x2*>(op + e) = u32x2{pack2(o[0], o[1]), pack2(o[2], o[3])};
                else *reinterpret_cast<f32x4*>(op + e) = o;
            }
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
    {
        // (past the last head, or of a row that is no query: anything that is there)
        const float2* part = a.part + (size_t)min(i, heads - 1) * chunks;
        const float* from = a.opart + (size_t)min(i, heads - 1) * chunks * D + quad * 4;
        for (int j0 = k; j0 < chunks; j0 += kTogether << split) {
            float2 p[kTogether];
            f32x4 x[kTogether];
#pragma unroll
            for (int j = 0; j < kTogether; ++j) {
                const int at = min(j0 + (j << split), chunks - 1);
                p[j] = part[at];
                x[j] = *reinterpret_cast<const f32x4*>(from + (size_t)at * D);
            }
#pragma unroll
            for (int j = 0; j < kTogether; ++j) {  // (a part without rows was not written)
                if (j0 + (j << split) >= chunks) p[j] = make_float2(-FLT_MAX, 0.0f);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[j][e] = p[j].y != 0.0f ? x[j][e] : 0.0f;
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
    constexpr int kParts = sizeof(T) == 2 ? 1 : 3;
    constexpr int kValues = kWaves * kValueBytes<D>, kQueries = kParts * (D / 32) * CT * kWave * (int)sizeof(u32x4);
    constexpr int kJoined = CT * (D / 16) * (kWaves - 1) * kWave * (int)sizeof(f32x4), kStat = kWaves > 1 ? 2 * kWaves * CT * 16 * (int)sizeof(float) : 0;
    static_assert(kJoined % 16 == 0 && kValues % 16 == 0, "queries are read 16 bytes at a time");
    static_assert(CT * 16 <= kQ4MostColumns, "room for the parts of outputs");
    static_assert(!kShared || CT * 16 <= kQ4MostVectors, "a block's slots and their masks (heads of their own: 16 queries a column tile)");
    constexpr int kFirst = kValues + kQueries > kJoined ? kValues + kQueries : kJoined;
    a.q_at = kValues / (int)sizeof(float);
    a.stat_at = kFirst / (int)sizeof(float);
    const size_t lds = kFirst + kStat;
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

template <typename T, int D, bool kShared>
hipError_t launch_tiles(const Q4QueryArgs& a, hipStream_t s) {
    if constexpr (sizeof(T) == 2) {
        if constexpr (!kShared)
            if (a.plan.tiles == 4) return launch_form<T, D, 4, 1, kShared, 2>(a, s);
        if constexpr (kShared)
            if (a.plan.tiles == 2 && a.plan.waves == 8) return launch_form<T, D, 2, 1, kShared, 8>(a, s);
        if (a.plan.tiles == 2) return launch_form<T, D, 2, 1, kShared, 4>(a, s);
    }
    return launch_form<T, D, 1, 3, kShared, 4>(a, s);
}
template <bool kShared>
hipError_t launch_queries(const Q4QueryArgs& a, hipStream_t s) {
    if (a.dims.bf16) return a.dims.d == 128 ? launch_tiles<bf16_t, 128, kShared>(a, s) : launch_tiles<bf16_t, 64, kShared>(a, s);
    return a.dims.d == 128 ? launch_tiles<float, 128, kShared>(a, s) : launch_tiles<float, 64, kShared>(a, s);
}

int cus_of() { return device_cus() > 0 ? device_cus() : 256; }
// Workgroups of `waves` waves that divide a block's `tiles` tiles: no more than `want` in all, and two tiles for a wave at least.
int chunks_of(int64_t units, int64_t tiles, int waves, int want) {
    const int64_t by_units = want / units, most = (tiles + 2 * waves - 1) / (2 * waves), n = by_units < most ? by_units : most;
    return n > 1 ? (int)n : 1;
}

}  // namespace

// Forms; figures of one line were timed side by side.  One column tile: four waves, two workgroups for a CU (the 8B layer at its budget
// 18.0 us; one 20.4, four 18.9; eight waves 19.4).  Two: four waves, as many workgroups as fit a CU, three (128 queries on 32,768 rows
// 105 us, two 114).  Four, each of two waves, as many as a CU holds, where the blocks have 240 tiles of rows for a CU, of all slots'
// queries and as many rows as n_max allows (one slot of 32/8 heads, four column tiles and two: 2,048 queries on 32,768 rows 1,095 us and
// 1,286, 1,024 574 and 689, 256 165 and 186; on 8,192 rows 512 queries 97 and 103, 256 61.4 and 61.7, 128 48 and 37; 2,048 on 2,048 82 and
// 70; 8 prompts of 1,024 132 and 157).
Q4QueryPlan q4_window_plan(const Q4Dims& d, int layer_count, int n_max, int rows, int window, int sinks) {
    Q4QueryPlan p{};
    p.per = 16 / d.group;
    const int64_t slabs = (int64_t)layer_count * d.batch * d.hkv;
    auto blocks = [&](int rows, int tiles) { return (rows + tiles * p.per - 1) / (tiles * p.per); };
    // tiles of n rows that a block sees: with a window (of rows in order) those of it, which ends inside tiles
    auto seen = [&](int n, int vectors) {
        const int64_t all = (n + kTile - 1) / kTile, some = ((int64_t)window + sinks + vectors) / kTile + 3;
        return window && some < all ? some : all;
    };
    const int most = rows < n_max ? rows : n_max;
    const bool long_blocks = (double)slabs * blocks(most, 4) * (double)seen(n_max - most / 2, 4 * p.per) >= 240.0 * cus_of();
    p.tiles = !d.bf16 || rows <= p.per ? 1 : long_blocks ? 4 : 2;
    p.waves = p.tiles == 4 ? 2 : 4;
    p.vectors = p.tiles * p.per;
    p.blocks = blocks(rows, p.tiles);
    const int64_t tiles = seen(n_max, p.vectors);
    p.chunks = chunks_of(slabs * p.blocks, tiles, p.waves, (p.tiles == 1 ? 2 : p.tiles == 2 ? 3 : 4) * cus_of());
    // Where a slot has several blocks, a wave that looks at more than three times 16 tiles finds them by marks: a kernel before it, 6 to 8
    // us, that all layers and heads share.  A single block, a decode step's, looks for itself, by as many waves as its window has tiles
    // for: with positions a narrow window of a long slot has few of them for all its rows (one query on 131,072 rows, 8 KV heads: a
    // window of 8,192 17 us, 1,024 22, 128 60; without positions 15).
    p.marks = p.blocks > 1 && (n_max + kTile - 1) / kTile > 48 * p.chunks * p.waves;
    return p;
}

// Two column tiles: where there are blocks for every CU, a workgroup of eight waves to each, without a join (32 layers of 8 samples
// 65 us, four waves in two and three chunks 8 and 3 more); else four waves, two workgroups for a CU (32 samples of three prompts 46 us,
// three 5 more, one 16 more), since small groups make more blocks than are counted here.
Q4QueryPlan q4_shared_plan(const Q4Dims& d, int layer_count, int n_max) {
    Q4QueryPlan p{};
    p.per = 16 / d.group;
    p.tiles = d.bf16 && d.batch > p.per ? 2 : 1;
    p.vectors = p.tiles * p.per;
    while (1 << p.vector_shift < p.vectors) ++p.vector_shift;
    // (groups that do not fill their blocks make more of them: places for twice as many)
    const int full = (d.batch + p.vectors - 1) / p.vectors;
    p.blocks = 2 * full < d.batch ? 2 * full : d.batch;
    const int64_t units = (int64_t)layer_count * d.hkv * full;
    p.waves = p.tiles == 2 && units >= cus_of() ? 8 : 4;
    p.chunks = p.waves == 8 ? 1 : chunks_of(units, (n_max + kTile - 1) / kTile, p.waves, 2 * cus_of());
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
    if (a.heads) {
        hipLaunchKernelGGL(q4_block_kernel, dim3(a.dims.batch), dim3(kWave), 0, s, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return launch_queries<true>(a, s);
}

}  // namespace ikv
