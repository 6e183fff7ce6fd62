// Decode attention over the paged 4-bit cache, with the eviction score (Eq. 1) and its fold (Eq. 4).
//
// z_h(i) = q_h . k_i / sqrt(d) (+ bias on recent positions), a_h = softmax over the rows i < len, o_h = sum_i a_h(i) v_i;
// s(i) = (1 / H) sum_h a_h(i), u <- alpha u + (1 - alpha) s layer by layer.  Base-2 logits throughout.
//
// A workgroup takes one chunk of rows of one (layer, sequence, KV head) slab for the group's query heads; its waves take
// tiles of 32 rows in turn, each with a running maximum, sum and output of its own, joined at the end of the chunk.  Both
// products run on the matrix cores (16x16x32, bf16 in, 32 bits out); lane 16 s + c of a wave:
//  * keys: row 4 (c % 4) + c / 4 of each half of the tile, elements 32 s ... (d = 64: 16 s ...): 16 (8) consecutive bytes of
//    codes, one scale.  A code with its scale is a bf16 number exactly, and the conversion applies the scale, so the product with a bf16 query is
//    exact up to the order of 32-bit sums.  The query's elements lie in the same order.  f32 queries: three bf16 parts whose
//    sum is the number, a product each.
//  * logits: the result holds rows s, 4 + s, 8 + s, 12 + s of each half for column c.  A column is a head; where three or two times
//    the group fits 16 columns, the heads are there again, for the parts below.
//  * probabilities p = 2^(z - m): as a B operand, the same lane holds the same rows, so nothing moves between lanes.  p is
//    split into three bf16 parts of 8 bits that sum up to all 24 of its bits, a column of its own each or a product of its own
//    (4 layers of 32 x 1 .. 8,192 rows, 7 heads a KV head: 78 us with three products, 75 with two columns and two products, and 72
//    with two parts, which are up to 2^-15 low; in three columns the third costs nothing).
//  * values: loaded to LDS as they lie in memory, without registers; the lane takes the same rows' elements 8 c .. 8 c + 7
//    (d = 64: 4 c ...; the four rows that a read of the wave takes are consecutive, so no two lanes meet in a bank), converted
//    like the keys; pairs of rows of one element are put together by byte permutes of the lane's own registers.
//  * output: column c, elements 32 s .. 32 s + 31 (d = 64: 16 s ...).
// The maximum is raised only when a tile exceeds it by 2^8: p stays below 2^8 and the sums in range, and the rescaling of the
// output is rare.  Rows behind the sequence, and rows of pages that do not exist, get the logit -inf and their values the
// scale 1 (whatever their bytes are), so that they add 0 * a finite number.
//
// What bounds it, measured: all layers of 8 sequences x 3,277 rows x 8 KV heads of 4 (bf16, 913 MB) take 160 us, 5.7 TB/s (a
// large copy reaches 4.9); with the arithmetic left out of a copy of the kernel the same loads take 144, and 164 when they do not
// pass the caches by.  One layer of it (28.5 MB) is a matter of latencies: 13 us and 4 for the join; without the arithmetic 10 and
// 4.  One sequence of 131,072 rows, 143 MB: 27 us + 4.5.
// On the way (all layers): 190 us with the values in registers and cached loads.  Equal shares of all tiles per workgroup, whatever
// sequence they belong to, took 226 (the search for the share, and the state that it needs).
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

constexpr int kMostRows = 8192;       // rows of a chunk, however many slabs there are: a batch may hold one long sequence

// Rows of sequence b that a call attends to: its length, or none of it where that is out of range.
__device__ __forceinline__ int attended(const Q4AttendArgs& a, int b) {
    const int n = a.cache.len[b];
    return n < 0 || n > a.n_max ? 0 : n;
}

// One tile's halves: the places of their rows, and what is loaded of them.
struct Place {
    const uint8_t* k;  // the half's first row: keys' codes, ...
    const uint8_t* e;  // ... scales, and the values' of both vc_off bytes on
    int valid;         // rows that take part
};
template <int D>
struct Keys {
    uint32_t codes[2][D / 32];
    uint32_t scale[2];
    int pos;           // position of row `lane % 32` (with a bias only)
};
// What a wave knows of its slab.
template <int D>
struct Slab {
    const uint8_t* pool;   // the layer's and KV head's first record
    scalar_ints table;
    size_t page_bytes;     // from a page's record to the next page's
    const int32_t* pos;    // null: no bias
    int end, last, n_pages, page_shift, page_rows, ks_off, vc_off;  // (last: the last row that the table has a place for)
    uint32_t ko, eo;  // the lane's offsets from a half's first row
    uint32_t fault;

    __device__ __forceinline__ int page(int row) const { return table[min(row, last) >> page_shift]; }
    __device__ __forceinline__ Place place(int row, int page) {
        Place p;
        p.valid = min(16, max(0, end - row));
        if ((uint32_t)page >= (uint32_t)n_pages) {  // (behind the sequence: anything; its rows are loaded, and take no part)
            if (p.valid) fault = kFaultCache;
            page = p.valid = 0;
        }
        const uint8_t* rec = pool + (size_t)(uint32_t)page * page_bytes;
        const int in = row & (page_rows - 1);
        p.k = rec + in * (D / 2);
        p.e = rec + ks_off + in * (D / 32);
        return p;
    }
    __device__ __forceinline__ void load(Keys<D>& t, const Place (&p)[2], int row0) const {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            if constexpr (D == 128) {
                const u32x4 x = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p[half].k + ko));
#pragma unroll
                for (int j = 0; j < 4; ++j) t.codes[half][j] = x[j];
            } else {
                const u32x2 x = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(p[half].k + ko));
                t.codes[half][0] = x[0];
                t.codes[half][1] = x[1];
            }
            t.scale[half] = p[half].e[eo];
        }
        if (pos) t.pos = pos[min(row0 + (int)(threadIdx.x % kTile), end - 1)];
    }
    __device__ __forceinline__ void load_values(const Place (&p)[2], uint8_t* lds) const {
        const uint32_t lane = threadIdx.x % kWave;
        if constexpr (D == 128) {
            to_lds<16>(p[0].k + vc_off + lane * 16, lds);
            to_lds<16>(p[1].k + vc_off + lane * 16, lds + 1024);
            to_lds<4>((lane & 16 ? p[1].e : p[0].e) + vc_off + lane % 16 * 4, lds + 2048);
        } else {
            to_lds<16>((lane & 32 ? p[1].k : p[0].k) + vc_off + lane % 32 * 16, lds);
            to_lds<4>((lane & 8 ? p[1].e : p[0].e) + vc_off + lane % 8 * 4, lds + 1024);
        }
    }
};

constexpr int kZPad = 16;    // floats between the heads' logits in LDS
constexpr int kQ4Waves = 8;  // (four: one sequence of 131,072 rows 35 us for 34, scored slabs 215 for 190)
// Floats of LDS for the waves' and the heads' statistics: whole 16 bytes, since the logits behind them are accessed so.
__host__ __device__ constexpr int stat_floats(int group) { return (2 * (kQ4Waves + 1) * group + 3) / 4 * 4; }
constexpr bool logits_aligned() {
    for (int group = 1; group <= kMaxGroup; ++group)
        if (stat_floats(group) % 4 || stat_floats(group) < 2 * (kQ4Waves + 1) * group) return false;
    return kZPad % 4 == 0;  // (a head's logits are n_stride + kZPad floats, n_stride a multiple of 64)
}
static_assert(logits_aligned(), "16-byte accesses of the logits in LDS");

// Columns of a head for the parts of its probabilities (CP): as many as fit 16, three, two or one, with one, two and three products.
constexpr int columns_of(int group) { return group <= 5 ? 3 : group <= 8 ? 2 : 1; }
template <typename T, int D, int CP, bool kScored>
__device__ __forceinline__ void attend(const Q4AttendArgs& a) {
    constexpr int kThreads = kWave * kQ4Waves, kStep = kTile * kQ4Waves;
    constexpr int kKey = D / 32, kOut = D / 16;      // products per half, and for the output
    constexpr int kParts = sizeof(T) == 2 ? 1 : 3;   // bf16 parts of a query
    constexpr int kStride = D + 4;
    constexpr int kJoin = 4;                         // waves whose outputs are joined through LDS at once
    // [wave] values; in their place [joined wave][column][kStride] outputs; behind both [wave][head] maxima and sums, then (kScored)
    // the heads' own and the slab's logits [head][rows + kZPad]
    extern __shared__ float lds[];
    const Q4Dims& d = a.dims;
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int c = lane % 16, s = lane / 16;

    // the lane's column: part `part` of head `head` (columns past the last: no head)
    const int group = d.group;
    const int part = c / group, head = c % group;
    const bool column = part < CP;
    const int columns = CP * group;
    // A part is what lies between two cuts of a probability's bits (the highest part's lower bits go with the rounding to bf16).  Two
    // columns: the highest and the middle part in one product, the lowest and nothing in the other.
    const uint32_t cut_low = CP == 3 && part != 1 ? ~0u : 0xffffff00u;
    const uint32_t cut_high = CP == 3 && part == 2 ? 0xffffff00u : CP > 1 && part == 0 ? 0u : 0xffff0000u;
    const uint32_t pick_lowest = CP == 2 && part == 1 ? 0x0c0c0c0cu : 0x07060302u;
    // the lane's places in the wave's LDS: codes of elements D / 16 * c ... of row s, and their scale
    uint8_t* const value_lds = reinterpret_cast<uint8_t*>(lds) + wave * kValueBytes<D>;
    const uint8_t* const value_codes = value_lds + s * (D / 2) + c * (D / 32);
    const uint8_t* const value_scales = value_lds + kTile * (D / 2) + s * (D / 32) + (D == 128 ? c / 4 : c / 8);
    float* const stat = lds + a.stat_at;
    float* const heads = stat + 2 * kQ4Waves * group;  // kScored: [head] maximum, 1 / sum
    float* const zs = stat + stat_floats(group);

    // Grid: KV heads, sequences, then layers and chunks (first chunks first: the later ones, which short sequences lack, spread
    // evenly).  The sequences are turned by one from layer to layer: workgroups a multiple of the CUs apart, which meet on one,
    // would often be of the same sequence (32 sequences of 1 .. 8,192 rows, 16 slabs each: 85 us, turned 78; two prompts of up
    // to 16,400 rows among six short samples: 201 -> 174 with that whole step).
    const int g = blockIdx.x, b = (blockIdx.y + blockIdx.z) % d.batch;
    const int chunk = kScored ? 0 : blockIdx.z / a.layer_count, layer = kScored ? blockIdx.z : blockIdx.z % a.layer_count;
    const int lb = layer * d.batch + b, slab = lb * d.hkv + g;
    const int first = kScored ? 0 : chunk * a.chunk_rows;
    int row = first + wave * kTile;
    const scalar_ints table = (scalar_ints)(uintptr_t)(a.cache.table + (size_t)b * d.max_pages);
    // the first pages of the wave's rows are read beside the length
    const int last = d.cap - 1;
    int page[2], page_now[2];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        page_now[half] = table[min(row + 16 * half, last) >> d.page_shift];
        page[half] = table[min(row + kStep + 16 * half, last) >> d.page_shift];
    }
    const int raw_len = ((scalar_ints)(uintptr_t)a.cache.len)[b];
    const int len = raw_len < 0 || raw_len > a.n_max ? 0 : raw_len;
    if (chunk == 0 && threadIdx.x == 0 && len != raw_len) atomicOr(a.faults, kFaultCache);
    if (first >= len && chunk > 0) return;
    const int end = kScored ? len : min(len, first + a.chunk_rows);

    // the query: bf16 in registers; f32 as three bf16 parts in LDS, [part][product][lane], where all waves read them (48 registers
    // fewer: four waves per SIMD, as bf16)
    u32x4 q[kKey];
    f32x4 qf[sizeof(T) == 2 ? 1 : 2 * kKey];
    {
        const T* qp = static_cast<const T*>(a.q) + ((size_t)lb * d.hq + g * group + head) * D + s * (D / 4);
        if constexpr (kParts == 1) {
#pragma unroll
            for (int j = 0; j < kKey; ++j) {
                const u32x4 x = reinterpret_cast<const u32x4*>(qp)[j];
                q[j] = column ? x : u32x4{0, 0, 0, 0};
            }
        } else if (wave == 0) {
#pragma unroll
            for (int j = 0; j < 2 * kKey; ++j) qf[j] = reinterpret_cast<const f32x4*>(qp)[j];
        }
    }

    const int key_row = c % 4 * 4 + c / 4;  // row of a half whose keys the lane holds: result rows 4 s + i are rows 4 i + s
    Slab<D> sl{a.cache.pool + q4_record(d, a.layer0 + layer, 0, g),
               table,
               (size_t)d.hkv * d.rec,
               a.bias2 != 0.0f ? a.cache.pos + (size_t)b * d.cap : nullptr,
               end, last, d.n_pages, d.page_shift, d.page_rows, d.ks_off, d.vc_off,
               (uint32_t)(key_row * (D / 2) + s * (D / 8)), (uint32_t)(D == 128 ? key_row * 4 + s : key_row * 2 + s / 2), 0};
    const int recent_from = sl.pos ? (int)max((int64_t)INT_MIN, (int64_t)a.cur_pos[b] - (a.window - 1)) : 0;
    float m = -FLT_MAX, l = 0.0f;
    f32x4 acc[kOut];
#pragma unroll
    for (int x = 0; x < kOut; ++x) acc[x] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    // Loads run one tile ahead: a tile's keys are replaced by the next tile's once the logits are taken, its values once the
    // output is; the page numbers run two tiles ahead.
    Keys<D> keys;
    Place now[2], next[2];
    if (row < end) {
#pragma unroll
        for (int half = 0; half < 2; ++half) now[half] = sl.place(row + 16 * half, page_now[half]);
        sl.load(keys, now, row);
        sl.load_values(now, value_lds);
    }
    u32x4* const q_lds = reinterpret_cast<u32x4*>(lds + a.q_at) + lane;
    if constexpr (kParts == 3) {
        if (wave == 0) {
#pragma unroll
            for (int j = 0; j < kKey; ++j) {
                float x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = column ? qf[2 * j + i / 4][i % 4] : 0.0f;
#pragma unroll
                for (int k = 0; k < 3; ++k) {
                    u32x4 y;
#pragma unroll
                    for (int i = 0; i < 4; ++i) y[i] = high2(__float_as_uint(x[2 * i]), __float_as_uint(x[2 * i + 1]));
                    q_lds[(k * kKey + j) * kWave] = y;
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] -= __uint_as_float(__float_as_uint(x[i]) & 0xffff0000u);
                }
            }
        }
        __syncthreads();
    }
    for (; row < end; row += kStep) {
        const bool more = row + kStep < end;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the tile's keys, and its values in LDS
        // logits
        float z[8];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const float scale = __uint_as_float(keys.scale[half] << 23);
            f32x4 r{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int j = 0; j < kKey; ++j) {
                const u32x4 k = eight(keys.codes[half][j], scale);
#pragma unroll
                for (int p = kParts - 1; p >= 0; --p) r = mfma(k, kParts == 1 ? q[j] : q_lds[(p * kKey + j) * kWave], r);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) z[4 * half + i] = r[i] * a.scale2;
        }
        if (sl.pos) {
            const uint32_t recent = (uint32_t)__ballot(keys.pos >= recent_from);  // (lanes 32 .. 63: the same rows again)
            if (recent) {
                const uint32_t mine_recent = recent >> s;
                asm volatile("");  // (a branch: few tiles hold recent rows)
#pragma unroll
                for (int j = 0; j < 8; ++j) z[j] += mine_recent & 1u << (16 * (j / 4) + 4 * (j % 4)) ? a.bias2 : 0.0f;
            }
        }
        if (more) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                next[half] = sl.place(row + kStep + 16 * half, page[half]);
                page[half] = sl.page(row + 2 * kStep + 16 * half);
            }
            sl.load(keys, next, row + kStep);
        }
        const bool whole = now[0].valid + now[1].valid == kTile;  // (uniform)
        if (!whole) {
            asm volatile("");
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (4 * (j % 4) >= now[j / 4].valid - s) z[j] = -INFINITY;
        }
        if ((kScored || a.z) && c < group) {  // (row 4 i + s of a half at 4 s + i)
            float* zp = kScored ? zs + c * (a.n_stride + kZPad) + row + 4 * s
                                : a.z + ((size_t)slab * group + c) * a.n_stride + row + 4 * s;
            *reinterpret_cast<f32x4*>(zp) = f32x4{z[0], z[1], z[2], z[3]};
            *reinterpret_cast<f32x4*>(zp + 16) = f32x4{z[4], z[5], z[6], z[7]};
        }
        // running maximum, probabilities, their parts
        float top = z[0];
#pragma unroll
        for (int j = 1; j < 8; ++j) top = fmaxf(top, z[j]);
        if (__any(top > m + kSlack)) {
            top = rows_allmax(top);
            const float raised = top > m + kSlack ? top : m;
            const float f = exp2_hw(m - raised);
            m = raised;
            l *= f;
#pragma unroll
            for (int x = 0; x < kOut; ++x) acc[x] *= f;
        }
        float p[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            p[j] = exp2_hw(z[j] - m);
            l += p[j];
        }
        u32x4 pp{}, lowest{}, highest{};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t w[2] = {__float_as_uint(p[2 * i]), __float_as_uint(p[2 * i + 1])};
            float x[2], low[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float upper = __uint_as_float(w[k] & cut_low);
                x[k] = upper - __uint_as_float(w[k] & cut_high);
                low[k] = p[2 * i + k] - upper;
            }
            pp[i] = high2(__float_as_uint(x[0]), __float_as_uint(x[1]));
            if constexpr (CP < 3) lowest[i] = __builtin_amdgcn_perm(__float_as_uint(low[1]), __float_as_uint(low[0]), pick_lowest);
            if constexpr (CP == 1) highest[i] = high2(w[0], w[1]);
        }
        // output
        float scale[8];
        uint32_t codes[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int r = 16 * (j / 4) + 4 * (j % 4);  // (and s)
            if constexpr (D == 128) codes[j] = *reinterpret_cast<const uint32_t*>(value_codes + r * (D / 2));
            else codes[j] = *reinterpret_cast<const uint16_t*>(value_codes + r * (D / 2));
            scale[j] = __uint_as_float((uint32_t)value_scales[r * (D / 32)] << 23);
        }
        if (!whole) {
            asm volatile("");
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (4 * (j % 4) >= now[j / 4].valid - s) scale[j] = 1.0f;
        }
        if (more) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // this tile's values are out of LDS: the next tile's may come
            sl.load_values(next, value_lds);
            now[0] = next[0];
            now[1] = next[1];
        }
        auto two_columns = [&](auto byte) __attribute__((always_inline)) {
            constexpr int kByte = decltype(byte)::value;
            uint32_t x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = pair<kByte>(codes[j], scale[j]);
            const u32x4 even{low2(x[0], x[1]), low2(x[2], x[3]), low2(x[4], x[5]), low2(x[6], x[7])};
            const u32x4 odd{high2(x[0], x[1]), high2(x[2], x[3]), high2(x[4], x[5]), high2(x[6], x[7])};
            auto both = [&](u32x4 q) __attribute__((always_inline)) {
                acc[2 * kByte] = mfma(even, q, acc[2 * kByte]);
                acc[2 * kByte + 1] = mfma(odd, q, acc[2 * kByte + 1]);
            };
            if constexpr (CP < 3) both(lowest);
            both(pp);
            if constexpr (CP == 1) both(highest);
        };
        two_columns(std::integral_constant<int, 0>());
        two_columns(std::integral_constant<int, 1>());
        if constexpr (D == 128) {
            two_columns(std::integral_constant<int, 2>());
            two_columns(std::integral_constant<int, 3>());
        }
    }
    if (sl.fault && lane == 0) atomicOr(a.faults, sl.fault);

    // the waves joined: the upper four into the lower, those through columns of LDS, one thread per four elements of a head
    __syncthreads();  // (their values' places are used again)
    l = rows_allsum(l);
    float* const mine = lds + ((wave % kJoin) * columns + c) * kStride + s * (D / 4);
    auto put = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int x = 0; x < kOut; x += 4)
                *reinterpret_cast<f32x4*>(mine + i * kOut + x) = f32x4{acc[x][i], acc[x + 1][i], acc[x + 2][i], acc[x + 3][i]};
        if (s == 0 && part == 0) {
            stat[wave * group + head] = m;
            stat[(kQ4Waves + wave) * group + head] = l;
        }
    };
    if constexpr (kQ4Waves > kJoin) {
        static_assert(kQ4Waves == 2 * kJoin, "one step joins the halves");
        if (wave >= kJoin && column) put();
        __syncthreads();
        if (wave < kJoin && column) {
            const float m2 = stat[(wave + kJoin) * group + head], l2 = stat[(kQ4Waves + wave + kJoin) * group + head];
            const float top = fmaxf(m, m2), f = exp2_hw(m - top), f2 = exp2_hw(m2 - top);
            m = top;
            l = l * f + l2 * f2;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int x = 0; x < kOut; x += 4) {
                    const f32x4 o = *reinterpret_cast<const f32x4*>(mine + i * kOut + x);
#pragma unroll
                    for (int k = 0; k < 4; ++k) acc[x + k][i] = acc[x + k][i] * f + o[k] * f2;
                }
        }
        __syncthreads();
    }
    if (wave < kJoin && column) put();
    __syncthreads();
    const size_t head0 = (size_t)lb * d.hq + g * group;
    const size_t slot = kScored ? 0 : (size_t)slab * a.nchunk + chunk;
    for (int i = threadIdx.x; i < group * (D / 4); i += kThreads) {
        const int h = i / (D / 4), e = i % (D / 4) * 4;
        float top = stat[h];
#pragma unroll
        for (int w = 1; w < kJoin; ++w) top = fmaxf(top, stat[w * group + h]);
        float sum = 0.0f;
        f32x4 o{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < kJoin; ++w) {
            const float f = exp2_hw(stat[w * group + h] - top);
            sum += f * stat[(kQ4Waves + w) * group + h];
            f32x4 x = *reinterpret_cast<const f32x4*>(lds + (w * columns + h) * kStride + e);
#pragma unroll
            for (int k = 1; k < CP; ++k) x += *reinterpret_cast<const f32x4*>(lds + (w * columns + k * group + h) * kStride + e);
            o += x * f;
        }
        const float inv = sum != 0.0f ? 1.0f / sum : 0.0f;
        if (kScored || a.nchunk == 1) {
            T* op = static_cast<T*>(a.o) + (head0 + h) * D + e;
#pragma unroll
            for (int j = 0; j < 4; ++j) Elem<T>::store(op + j, o[j] * inv);
            if (kScored) {
                if (e == 0) {
                    heads[2 * h] = top;
                    heads[2 * h + 1] = inv;
                }
            } else if (e == 0 && a.stat) {
                a.stat[(size_t)slab * group + h] = make_float2(top, inv);
            }
        } else {
            *reinterpret_cast<f32x4*>(a.opart + (slot * group + h) * D + e) = o;
            if (e == 0) a.part[slot * group + h] = make_float2(top, sum);
        }
    }
    if constexpr (kScored) {
        // the slab's part of the scores: sum over the group of 2^(z - m) / sum, four rows per thread
        float* rp = a.z + (size_t)slab * a.n_stride;
        __syncthreads();
        for (int r = threadIdx.x * 4; r < (len + 15) / 16 * 16; r += kThreads * 4) {  // (whole blocks: their rows lie in another order)
            f32x4 x{0.0f, 0.0f, 0.0f, 0.0f};
            for (int h = 0; h < group; ++h) {
                const f32x4 z = *reinterpret_cast<const f32x4*>(zs + h * (a.n_stride + kZPad) + r);
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = fmaf(exp2_hw(z[i] - heads[2 * h]), heads[2 * h + 1], x[i]);
            }
            *reinterpret_cast<f32x4*>(rp + r) = x;
        }
    }
}

template <typename T, int D, int CP, bool kScored>
__global__ __launch_bounds__(kWave* kQ4Waves, 4) void q4_attend_kernel(Q4AttendArgs a) {
    attend<T, D, CP, kScored>(a);
}
template <typename T, int D, bool kScored>
__global__ __launch_bounds__(kWave* kQ4Waves, 4) void q4_attend_pairs_kernel(Q4AttendArgs a) {
    attend<T, D, 2, kScored>(a);
}

// A few chunks: one workgroup per slab joins their outputs and statistics, four elements of a head per thread and all of its
// loads at once (one layer of 64 slabs in 7 chunks, attention and join: 17.5 -> 16.4 us against a workgroup per head).
constexpr int kFewChunks = 8, kFewThreads = 256;
template <typename T, int D>
__global__ __launch_bounds__(kFewThreads) void q4_join_few_kernel(Q4AttendArgs a) {
    const Q4Dims& d = a.dims;
    const int slab = blockIdx.x, g = slab % d.hkv, lb = slab / d.hkv;
    const int chunks = max(1, (attended(a, lb % d.batch) + a.chunk_rows - 1) / a.chunk_rows);
    const size_t slot0 = (size_t)slab * a.nchunk;
    for (int i = threadIdx.x; i < d.group * (D / 4); i += kFewThreads) {
        const int h = i / (D / 4), e = i % (D / 4) * 4;
        float2 p[kFewChunks];
        f32x4 x[kFewChunks];
#pragma unroll
        for (int k = 0; k < kFewChunks; ++k) {
            const size_t at = (slot0 + min(k, chunks - 1)) * d.group + h;
            p[k] = a.part[at];
            if (k < chunks) x[k] = *reinterpret_cast<const f32x4*>(a.opart + at * D + e);
        }
        float top = p[0].x, sum = 0.0f;
#pragma unroll
        for (int k = 1; k < kFewChunks; ++k) top = fmaxf(top, p[k].x);
        f32x4 o{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < kFewChunks; ++k)
            if (k < chunks) {
                const float f = exp2_hw(p[k].x - top);
                sum += f * p[k].y;
                o += x[k] * f;
            }
        const float inv = sum != 0.0f ? 1.0f / sum : 0.0f;
        if (e == 0 && a.stat) a.stat[(size_t)slab * d.group + h] = make_float2(top, inv);
        T* op = static_cast<T*>(a.o) + ((size_t)lb * d.hq + g * d.group + h) * D + e;
#pragma unroll
        for (int j = 0; j < 4; ++j) Elem<T>::store(op + j, o[j] * inv);
    }
}

// More chunks: one workgroup per (slab, head).
constexpr int kJoinThreads = 512;
template <typename T, int D>
__global__ __launch_bounds__(kJoinThreads) void q4_join_kernel(Q4AttendArgs a) {
    constexpr int kQuads = D / 4, kRows = kJoinThreads / kQuads, kJoinWaves = kJoinThreads / kWave, kTogether = 4;
    __shared__ f32x4 red[kRows][kQuads];
    __shared__ float mx[kJoinWaves], sm[kJoinWaves];
    const Q4Dims& d = a.dims;
    const int h = blockIdx.x % d.group, slab = blockIdx.x / d.group, g = slab % d.hkv, lb = slab / d.hkv;
    const int segments = max(1, (attended(a, lb % d.batch) + a.chunk_rows - 1) / a.chunk_rows);
    const size_t slot0 = (size_t)slab * a.nchunk;
    auto part = [&](int i) { return a.part[(slot0 + i) * d.group + h]; };
    float top = -FLT_MAX;
    for (int i = threadIdx.x; i < segments; i += kJoinThreads) top = fmaxf(top, part(i).x);
    top = wave_max(top);
    if (threadIdx.x % kWave == 0) mx[threadIdx.x / kWave] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kJoinWaves; ++w) top = fmaxf(top, mx[w]);
    float sum = 0.0f;
    for (int i = threadIdx.x; i < segments; i += kJoinThreads) {
        const float2 p = part(i);
        sum += exp2_hw(p.x - top) * p.y;
    }
    sum = wave_sum(sum);
    if (threadIdx.x % kWave == 0) sm[threadIdx.x / kWave] = sum;
    const int quad = threadIdx.x % kQuads, r = threadIdx.x / kQuads;
    f32x4 o{0.0f, 0.0f, 0.0f, 0.0f};
    for (int i0 = r; i0 < segments; i0 += kRows * kTogether) {
        f32x4 x[kTogether];
        float f[kTogether];
#pragma unroll
        for (int k = 0; k < kTogether; ++k) {
            const int i = min(i0 + k * kRows, segments - 1);
            x[k] = *reinterpret_cast<const f32x4*>(a.opart + ((slot0 + i) * d.group + h) * D + quad * 4);
            f[k] = part(i).x;
        }
#pragma unroll
        for (int k = 0; k < kTogether; ++k)
            if (i0 + k * kRows < segments) o += x[k] * exp2_hw(f[k] - top);
    }
    red[r][quad] = o;
    __syncthreads();
    sum = 0.0f;
#pragma unroll
    for (int w = 0; w < kJoinWaves; ++w) sum += sm[w];
    const float inv = sum != 0.0f ? 1.0f / sum : 0.0f;
    if (threadIdx.x == 0 && a.stat) a.stat[(size_t)slab * d.group + h] = make_float2(top, inv);
    if (r != 0) return;
#pragma unroll
    for (int i = 1; i < kRows; ++i) o += red[i][quad];
    T* op = static_cast<T*>(a.o) + ((size_t)lb * d.hq + g * d.group + h) * D + quad * 4;
#pragma unroll
    for (int j = 0; j < 4; ++j) Elem<T>::store(op + j, o[j] * inv);
}

// Scores and their fold: 64 rows of a sequence per workgroup, one a lane.  A wave takes the KV heads slice, slice + per, ... of
// one layer, kAhead layers at a time (their loads together; 1 where the waves side by side cover the call's layers); the waves'
// sums of a layer are added in order, and the layers folded in order.  kGroups: the scores' parts were summed over each group by
// the attention.
constexpr int kScoreWaves = 16;
template <bool kGroups, int kAhead>
__global__ __launch_bounds__(kScoreWaves* kWave) void q4_score_kernel(Q4AttendArgs a, int per_shift, int together_shift) {
    __shared__ float part[kAhead][kScoreWaves][kWave];
    const Q4Dims& d = a.dims;
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int waves = blockDim.x / kWave, per = 1 << per_shift, together = 1 << together_shift;  // (layers side by side)
    const int b = blockIdx.y, row = blockIdx.x * kWave + lane;
    const int n = attended(a, b);
    const bool live = row < n;
    const int at = (row & ~15) | (row & 3) << 2 | (row >> 2 & 3);  // place of a row's logits
    const float inv = 1.0f / (float)d.hq;
    const size_t ub = (size_t)b * d.cap + row;
    float u = wave == 0 && live && a.u_out ? a.u_prior[ub] : 0.0f;
    for (int l0 = 0; l0 < a.layer_count; l0 += together * kAhead) {
        float s[kAhead];
#pragma unroll
        for (int q = 0; q < kAhead; ++q) s[q] = 0.0f;
        if ((int)blockIdx.x * kWave < n)
#pragma unroll 4
            for (int g = (wave & (per - 1)); g < d.hkv; g += per) {
                size_t slab[kAhead];
#pragma unroll
                for (int q = 0; q < kAhead; ++q) {
                    const int l = min(l0 + q * together + (wave >> per_shift), a.layer_count - 1);  // (past the last: not used)
                    slab[q] = (size_t)(l * d.batch + b) * d.hkv + g;
                    if constexpr (kGroups) s[q] += a.z[slab[q] * a.n_stride + at];
                }
                if constexpr (!kGroups) {
#pragma unroll 4
                    for (int h = 0; h < d.group; ++h)
#pragma unroll
                        for (int q = 0; q < kAhead; ++q) {
                            const size_t head = slab[q] * d.group + h;
                            const float2 st = a.stat[head];
                            s[q] = fmaf(exp2_hw(a.z[head * a.n_stride + at] - st.x), st.y, s[q]);
                        }
                }
            }
#pragma unroll
        for (int q = 0; q < kAhead; ++q) part[q][wave][lane] = s[q];
        __syncthreads();
        // (wave, layer) pairs: the layer's sum in place of its first slice's
        for (int i = wave; i < together * kAhead; i += waves) {
            const int q = i >> together_shift, w0 = (i & (together - 1)) << per_shift;
            float x = part[q][w0][lane];
            for (int w = 1; w < per; ++w) x += part[q][w0 + w][lane];
            x *= inv;
            part[q][w0][lane] = x;
            const int l = l0 + i;
            if (a.s_out && l < a.layer_count && row < a.n_max) a.s_out[((size_t)l * d.batch + b) * a.n_max + row] = live ? x : 0.0f;
        }
        __syncthreads();
        if (wave == 0 && a.u_out)
#pragma unroll 8
            for (int i = 0; i < together * kAhead && l0 + i < a.layer_count; ++i)
                u = a.alpha * u + (1.0f - a.alpha) * part[i >> together_shift][(i & (together - 1)) << per_shift][lane];
        __syncthreads();
    }
    if (wave == 0 && live && a.u_out) a.u_out[ub] = u;
}

template <typename T, int D, int CP, bool kScored>
hipError_t launch_form(Q4AttendArgs a, hipStream_t s, void (*kern)(Q4AttendArgs)) {
    constexpr int kJoin = 4;
    const int slabs = a.layer_count * a.dims.batch * a.dims.hkv;
    const int joined = kJoin * a.dims.group * CP * (D + 4) * (int)sizeof(float), values = kQ4Waves * kValueBytes<D>;
    a.stat_at = (joined > values ? joined : values) / (int)sizeof(float);
    static_assert(D % 4 == 0 && kValueBytes<D> % 16 == 0, "stat_at is a multiple of 16 bytes");
    size_t lds = (size_t)(a.stat_at + stat_floats(a.dims.group)) * sizeof(float);
    if (kScored) lds += (size_t)a.dims.group * (a.n_stride + kZPad) * sizeof(float);
    if (sizeof(T) == 4) {
        a.q_at = (int)(lds / sizeof(float));
        lds += 3 * (D / 32) * kWave * sizeof(u32x4);
    }
    if (lds > 64 * 1024) {
        static std::atomic<bool> raised[kMaxDevices];
        const hipError_t e = raise_lds_limit(reinterpret_cast<const void*>(kern), raised);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kern, dim3(a.dims.hkv, a.dims.batch, a.layer_count * (kScored ? 1 : a.nchunk)), dim3(kWave * kQ4Waves), lds, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || kScored || a.nchunk == 1) return e;
    if (a.nchunk <= kFewChunks) hipLaunchKernelGGL((q4_join_few_kernel<T, D>), dim3(slabs), dim3(kFewThreads), 0, s, a);
    else hipLaunchKernelGGL((q4_join_kernel<T, D>), dim3(slabs * a.dims.group), dim3(kJoinThreads), 0, s, a);
    return hipGetLastError();
}

template <typename T, int D, bool kScored>
hipError_t launch_columns(const Q4AttendArgs& a, hipStream_t s) {
    if (a.columns == 3) return launch_form<T, D, 3, kScored>(a, s, q4_attend_kernel<T, D, 3, kScored>);
    if (a.columns == 2) return launch_form<T, D, 2, kScored>(a, s, q4_attend_pairs_kernel<T, D, kScored>);
    return launch_form<T, D, 1, kScored>(a, s, q4_attend_kernel<T, D, 1, kScored>);
}
template <typename T, int D>
hipError_t launch_attend(const Q4AttendArgs& a, hipStream_t s) {
    return a.scored ? launch_columns<T, D, true>(a, s) : launch_columns<T, D, false>(a, s);
}

}  // namespace

Q4AttendPlan q4_attend_plan(const Q4Dims& d, int layer_count, int n_max, bool scores) {
    Q4AttendPlan p{};
    const int slabs = layer_count * d.batch * d.hkv;
    const int cus = device_cus() > 0 ? device_cus() : 256;
    p.n_stride = (n_max + 63) / 64 * 64;
    // Chunks: two workgroups per CU in all, as many as it holds.  More cost more than they balance: 512 slabs of 8,192 rows take
    // 102 us in one chunk each, 110 in two, 131 in eight, and 512 of 1 .. 8,192 rows 79, 85 and 94.  But no chunk above 8,192
    // rows: two prompts of up to 16,400 rows among six short samples (512 slabs) 347 -> 312 us with that whole step.
    const int step = kQ4Waves * kTile, want = (2 * cus + slabs - 1) / slabs, by_rows = (n_max + step - 1) / step;
    p.most = want < by_rows ? want : by_rows;
    const int least = (n_max + kMostRows - 1) / kMostRows;
    if (least > p.most) p.most = least;
    // (whole turns of the waves, so there may be fewer: 64 slabs of 4,097 rows in 6 chunks of 768.  One more chunk where a few rows
    // make the turn, 9 of 512 for these, costs more than it balances, and a kernel with a workgroup per head to join them: bf16
    // 18.4 -> 19.6 us, f32 19.1 -> 20.7, 2,049 rows 13.4 -> 17.3; 512 slabs of 8,193 rows 107 -> 109.5)
    const int share = (n_max + p.most - 1) / p.most;
    p.chunk_rows = share > step ? (share + step - 1) / step * step : step;
    p.nchunk = (n_max + p.chunk_rows - 1) / p.chunk_rows;
    // Scored: where a slab's logits fit LDS with two workgroups on a CU, and there is a slab for each: 2,048 slabs of 3,277 rows
    // with scores 188 us, through memory 232.
    const auto fits = [&](int columns) {
        const size_t values = kQ4Waves * (size_t)(d.d == 128 ? kValueBytes<128> : kValueBytes<64>);
        const size_t outputs = 4 * (size_t)d.group * columns * (d.d + 4) * sizeof(float);
        return (values > outputs ? values : outputs) + (stat_floats(d.group) + (size_t)d.group * (p.n_stride + kZPad)) * sizeof(float) +
                   (d.bf16 ? 0 : 3 * (size_t)d.d / 32 * kWave * sizeof(u32x4)) <= kLdsPerCu / 2;
    };
    p.columns = columns_of(d.group);
    p.scored = scores && slabs >= 2 * cus && fits(p.columns);
    // (two columns of outputs take less LDS than three, and a product more: 2,048 slabs of 3,520 rows of 4 heads a KV head 202 us,
    // through memory 240; of 2,900 rows of 5 heads 173 and 224)
    if (scores && slabs >= 2 * cus && p.columns == 3 && !p.scored && fits(2)) {
        p.columns = 2;
        p.scored = 1;
    }
    return p;
}

hipError_t launch_q4_attend(const Q4AttendArgs& a, hipStream_t s) {
    hipError_t e = a.dims.bf16 ? (a.dims.d == 128 ? launch_attend<bf16_t, 128>(a, s) : launch_attend<bf16_t, 64>(a, s))
                                : (a.dims.d == 128 ? launch_attend<float, 128>(a, s) : launch_attend<float, 64>(a, s));
    if (e != hipSuccess || !a.z) return e;
    // Waves: as many as the call's layers have KV heads, up to 16, a power of two of them to a layer: the one that leaves a wave the
    // fewest (layer, KV head) pairs, the lower where they are the same.  (A wave to a layer leaves one sum to add: 32 layers of 8
    // KV heads x 8 sequences x 3,277 rows 17 -> 12 us.)
    int per_shift = 0, least = INT_MAX;
    for (int shift = 0; 1 << shift <= kScoreWaves; ++shift) {
        const int side = kScoreWaves >> shift, pairs = (a.layer_count + side - 1) / side * ((a.dims.hkv + (1 << shift) - 1) >> shift);
        if (pairs < least) {
            least = pairs;
            per_shift = shift;
        }
    }
    int waves_shift = per_shift;
    while ((1 << waves_shift) < a.layer_count << per_shift && (1 << waves_shift) < kScoreWaves) ++waves_shift;
    const int waves = 1 << waves_shift;
    const int blocks = (a.n_max + kWave - 1) / kWave;
    // layers ahead: up to four, the same number in every turn (layers past the last cost as much as others: 6 layers of 21
    // sequences of 491 .. 2,975 rows 32 us in turns of 16 layers, 18 so)
    const int rounds = ((a.layer_count << per_shift) + waves - 1) / waves, turns = (rounds + 3) / 4, ahead = (rounds + turns - 1) / turns;
    auto kern = a.scored ? (ahead == 1   ? q4_score_kernel<true, 1>
                            : ahead == 2 ? q4_score_kernel<true, 2>
                            : ahead == 3 ? q4_score_kernel<true, 3>
                                         : q4_score_kernel<true, 4>)
                         : (ahead == 1   ? q4_score_kernel<false, 1>
                            : ahead == 2 ? q4_score_kernel<false, 2>
                            : ahead == 3 ? q4_score_kernel<false, 3>
                                         : q4_score_kernel<false, 4>);
    hipLaunchKernelGGL(kern, dim3(blocks, a.dims.batch), dim3(waves * kWave), 0, s, a, per_shift,
                       waves_shift - per_shift);
    return hipGetLastError();
}

}  // namespace ikv
