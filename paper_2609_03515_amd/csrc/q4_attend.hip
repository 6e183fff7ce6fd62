// Decode attention over the paged 4-bit cache, with the eviction score (Eq. 1) and its fold (Eq. 4).
//
// z_h(i) = q_h . k_i / sqrt(d) (+ bias on recent positions), a_h = softmax over the rows i < len, o_h = sum_i a_h(i) v_i;
// s(i) = (1 / H) sum_h a_h(i), u <- alpha u + (1 - alpha) s layer by layer.  Base-2 logits throughout.
//
// A workgroup takes one chunk of rows of one (layer, sequence, KV head) slab for the group's query heads; its waves take
// tiles of 32 rows in turn, each with a running maximum, sum and output of its own, joined at the end of the chunk.  Both
// products run on the matrix cores (16x16x32, bf16 in, 32 bits out); lane 16 s + c of a wave:
//  * keys: row c of each half of the tile, elements 32 s ... (d = 64: 16 s ...): 16 consecutive bytes of codes, one scale.
//    A code with its scale is a bf16 number exactly, and the conversion applies the scale, so the product with a bf16 query is
//    exact up to the order of 32-bit sums.  The query's elements lie in the same order.  f32 queries: three bf16 parts whose
//    sum is the number, a product each.
//  * logits: the result holds rows 4 s .. 4 s + 3 of each half for column c.  A column is a head; where two or three times
//    the group fits 16 columns, the heads are there again, for the parts below.
//  * probabilities p = 2^(z - m): as a B operand, the same lane holds the same rows, so nothing moves between lanes.  p is
//    split into bf16 parts, 8 bits each, that sum up to 16 of its bits (bf16 output: an error of 2^-15, the output's own
//    rounding is 2^-8) or to all 24 (f32), a column of its own each or a product of its own.
//  * values: rows 4 s .. 4 s + 3 of each half, elements 8 c .. 8 c + 7 (d = 64: 4 c ...), converted like the keys; pairs of
//    rows of one element are put together by byte permutes of the lane's own registers.
//  * output: column c, elements 32 s .. 32 s + 31 (d = 64: 16 s ...).
// The maximum is raised only when a tile exceeds it by 2^8: p stays below 2^8 and the sums in range, and the rescaling of the
// output is rare.  Rows behind the sequence, and rows of pages that do not exist, get the logit -inf and their values the
// scale 1 (whatever their bytes are), so that they add 0 * a finite number.
#include <float.h>

#include "kv_common.h"
#include "q4.h"

namespace ikv {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kTile = 32;             // rows of a wave's tile: two halves of 16, each in one page
constexpr int kChunkStep = kTile * kWaves;
constexpr int kTargetWgs = 1024;      // workgroups wanted
constexpr float kSlack = 8.0f;

typedef __bf16 __attribute__((ext_vector_type(8))) bf16x8;
typedef uint32_t __attribute__((ext_vector_type(2))) u32x2;
typedef const __attribute__((address_space(4))) int32_t* scalar_ints;  // read by scalar loads: not written by the kernel

// Rows of sequence b that a call attends to: its length, or none of it where that is out of range.
__device__ __forceinline__ int attended(const Q4AttendArgs& a, int b) {
    const int n = a.cache.len[b];
    return n < 0 || n > a.n_max ? 0 : n;
}

__device__ __forceinline__ uint32_t low2(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t high2(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }
__device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
template <int BYTE>
__device__ __forceinline__ uint32_t pair(uint32_t codes, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, BYTE));
}
__device__ __forceinline__ u32x4 eight(uint32_t codes, float scale) {
    return u32x4{pair<0>(codes, scale), pair<1>(codes, scale), pair<2>(codes, scale), pair<3>(codes, scale)};
}
__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// One tile as it is loaded.
template <int D, bool BIAS>
struct Tile {
    static constexpr int kKey = D / 32;   // words of key codes per half
    uint32_t k[2][kKey];
    uint32_t ks[2];
    uint32_t v[8];                        // 8 (d = 64: 4) codes of each of the lane's rows
    uint32_t vs[2][D == 128 ? 4 : 2];     // scales of the lane's rows of a half, a row's bytes together
    int pos[BIAS ? 8 : 1];
    int valid[2];                         // rows of the half that take part (uniform)
};

template <typename T, int D, int CP, int NM, bool BIAS>
struct Lanes {
    const Q4AttendArgs& a;
    int c, s, b, len;
    const uint8_t* pool;   // the layer's and KV head's first record
    scalar_ints table;
    size_t page_bytes;     // from a page's record to the next page's
    uint32_t fault;

    __device__ __forceinline__ void load(Tile<D, BIAS>& t, int row0) {
        const Q4Dims& d = a.dims;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int row = row0 + 16 * half;
            int page = 0, valid = 0;
            if (row < len) {
                page = table[row >> d.page_shift];
                valid = min(16, len - row);
                if ((uint32_t)page >= (uint32_t)d.n_pages) {
                    page = valid = 0;
                    fault = kFaultCache;
                }
            }
            t.valid[half] = valid;
            const int in = row & (d.page_rows - 1);
            const uint8_t* rec = pool + (size_t)page * page_bytes;
            const uint8_t* kr = rec + in * (D / 2);
            const uint8_t* er = rec + d.ks_off + in * (D / 32);
            const uint8_t* vr = rec + d.vc_off + in * (D / 2);
            const uint8_t* fr = rec + d.vs_off + in * (D / 32);
            if constexpr (D == 128) {
                const u32x4 x = *reinterpret_cast<const u32x4*>(kr + (uint32_t)(c * 64 + s * 16));
#pragma unroll
                for (int j = 0; j < 4; ++j) t.k[half][j] = x[j];
                t.ks[half] = er[(uint32_t)(c * 4 + s)];
#pragma unroll
                for (int i = 0; i < 4; ++i) t.v[4 * half + i] = *reinterpret_cast<const uint32_t*>(vr + (uint32_t)((4 * s + i) * 64 + c * 4));
                const u32x4 f = *reinterpret_cast<const u32x4*>(fr + (uint32_t)(s * 16));
#pragma unroll
                for (int i = 0; i < 4; ++i) t.vs[half][i] = f[i];
            } else {
                const u32x2 x = *reinterpret_cast<const u32x2*>(kr + (uint32_t)(c * 32 + s * 8));
                t.k[half][0] = x[0];
                t.k[half][1] = x[1];
                t.ks[half] = er[(uint32_t)(c * 2 + s / 2)];
#pragma unroll
                for (int i = 0; i < 4; ++i) t.v[4 * half + i] = *reinterpret_cast<const uint16_t*>(vr + (uint32_t)((4 * s + i) * 32 + c * 2));
                const u32x2 f = *reinterpret_cast<const u32x2*>(fr + (uint32_t)(s * 8));
                t.vs[half][0] = f[0];
                t.vs[half][1] = f[1];
            }
            if constexpr (BIAS) {
                const int32_t* pr = a.cache.pos + (size_t)b * d.cap + (valid ? row : 0);  // (the first page's rows: in bounds)
#pragma unroll
                for (int i = 0; i < 4; ++i) t.pos[4 * half + i] = pr[4 * s + i];
            }
        }
    }
    // scale byte of the lane's value block in row 4 s + i of a half, at the exponent's place of a float
    __device__ __forceinline__ float value_scale(const Tile<D, BIAS>& t, int half, int i, int turn) const {
        const uint32_t w = D == 128 ? t.vs[half][i] : t.vs[half][i / 2] >> (i % 2 * 16);
        return __uint_as_float(__builtin_amdgcn_alignbit(w, w, turn) & 0x7f800000u);
    }
};

template <typename T, int D, int CP, int NM, bool BIAS>
__global__ __launch_bounds__(kThreads) void q4_attend_kernel(Q4AttendArgs a) {
    constexpr int kKey = D / 32, kOut = D / 16;      // products per half, and for the output
    constexpr int kParts = sizeof(T) == 2 ? 1 : 3;   // bf16 parts of a query
    constexpr int kStride = D + 4;
    extern __shared__ float lds[];                   // [wave][column][kStride], then [wave][column] maxima and sums
    const Q4Dims& d = a.dims;
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int c = lane % 16, s = lane / 16;
    const int slab = blockIdx.x / a.nchunk, chunk = blockIdx.x % a.nchunk;
    const int lb = slab / d.hkv, g = slab % d.hkv, b = lb % d.batch, layer = lb / d.batch;
    const int len_b = a.cache.len[b], len = len_b < 0 || len_b > a.n_max ? 0 : len_b;
    if (len != len_b && chunk == 0 && threadIdx.x == 0) atomicOr(a.faults, kFaultCache);
    const int first = chunk * a.chunk_rows;
    if (first >= len && chunk > 0) return;
    const int end = min(len, first + a.chunk_rows);

    // the lane's column: part `part` of head `head` (columns past the last: no head)
    const int group = d.group;
    const int part = c / group, head = c % group;
    const bool column = part < CP;
    const uint32_t cut1 = part >= 1 ? 0xffff0000u : 0u, cut2 = part >= 2 ? 0xffff0000u : 0u;

    u32x4 q[kParts][kKey];
    {
        const T* qp = static_cast<const T*>(a.q) + ((size_t)lb * d.hq + g * group + head) * D + s * (D / 4);
#pragma unroll
        for (int j = 0; j < kKey; ++j) {
            if constexpr (kParts == 1) {
                const u32x4 x = reinterpret_cast<const u32x4*>(qp)[j];
                q[0][j] = column ? x : u32x4{0, 0, 0, 0};
            } else {
                float x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = column ? static_cast<const float*>(static_cast<const void*>(qp))[8 * j + i] : 0.0f;
#pragma unroll
                for (int k = 0; k < 3; ++k) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) q[k][j][i] = high2(__float_as_uint(x[2 * i]), __float_as_uint(x[2 * i + 1]));
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] -= __uint_as_float(__float_as_uint(x[i]) & 0xffff0000u);
                }
            }
        }
    }

    Lanes<T, D, CP, NM, BIAS> ln{a, c, s, b, end, a.cache.pool + q4_record(d, a.layer0 + layer, 0, g),
                                 (scalar_ints)(uintptr_t)(a.cache.table + (size_t)b * d.max_pages), (size_t)d.hkv * d.rec, 0};
    const int recent_from = BIAS ? a.cur_pos[b] - (a.window - 1) : 0;
    const int turn = (D == 128 ? 8 * (c / 4) : 8 * (c / 8)) + 9 & 31;  // rotation that brings the lane's byte to bit 23
    float m = -FLT_MAX, l = 0.0f;
    f32x4 acc[kOut];
#pragma unroll
    for (int x = 0; x < kOut; ++x) acc[x] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    auto compute = [&](Tile<D, BIAS>& t, int row0) __attribute__((always_inline)) {
        float z[8];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const float scale = __uint_as_float(t.ks[half] << 23);
            f32x4 r{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int j = 0; j < kKey; ++j) {
                const u32x4 k = eight(t.k[half][j], scale);
#pragma unroll
                for (int p = kParts - 1; p >= 0; --p) r = mfma(k, q[p][j], r);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                z[4 * half + i] = r[i] * a.scale2;
                if constexpr (BIAS) z[4 * half + i] += t.pos[4 * half + i] >= recent_from ? a.bias2 : 0.0f;
            }
        }
        const bool whole = t.valid[0] + t.valid[1] == kTile;  // (uniform)
        if (!whole) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (4 * s + j % 4 >= t.valid[j / 4]) z[j] = -INFINITY;
        }
        if (a.z && c < group) {
            float* zp = a.z + ((size_t)slab * group + c) * a.n_stride + row0 + 4 * s;
            *reinterpret_cast<f32x4*>(zp) = f32x4{z[0], z[1], z[2], z[3]};
            *reinterpret_cast<f32x4*>(zp + 16) = f32x4{z[4], z[5], z[6], z[7]};
        }
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
        if constexpr (CP >= 2)
#pragma unroll
            for (int j = 0; j < 8; ++j) p[j] -= __uint_as_float(__float_as_uint(p[j]) & cut1);
        if constexpr (CP >= 3)
#pragma unroll
            for (int j = 0; j < 8; ++j) p[j] -= __uint_as_float(__float_as_uint(p[j]) & cut2);
        u32x4 pp[NM];
#pragma unroll
        for (int k = 0; k < NM; ++k) {
#pragma unroll
            for (int i = 0; i < 4; ++i) pp[k][i] = high2(__float_as_uint(p[2 * i]), __float_as_uint(p[2 * i + 1]));
            if (k + 1 < NM)
#pragma unroll
                for (int j = 0; j < 8; ++j) p[j] -= __uint_as_float(__float_as_uint(p[j]) & 0xffff0000u);
        }
        u32x4 x4[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float scale = ln.value_scale(t, j / 4, j % 4, turn);
            if (!whole && 4 * s + j % 4 >= t.valid[j / 4]) scale = 1.0f;
            if constexpr (D == 128) x4[j] = eight(t.v[j], scale);
            else x4[j] = u32x4{pair<0>(t.v[j], scale), pair<1>(t.v[j], scale), 0, 0};
        }
#pragma unroll
        for (int x = 0; x < kOut; ++x) {
            u32x4 v;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                v[i] = x % 2 ? high2(x4[2 * i][x / 2], x4[2 * i + 1][x / 2]) : low2(x4[2 * i][x / 2], x4[2 * i + 1][x / 2]);
#pragma unroll
            for (int k = NM - 1; k >= 0; --k) acc[x] = mfma(v, pp[k], acc[x]);
        }
    };

    {
        Tile<D, BIAS> t0, t1;
        int row = first + wave * kTile;
        if (row < end) ln.load(t0, row);
        if (row + kChunkStep < end) ln.load(t1, row + kChunkStep);
        while (row < end) {
            compute(t0, row);
            if (row + 2 * kChunkStep < end) ln.load(t0, row + 2 * kChunkStep);
            row += kChunkStep;
            if (row >= end) break;
            compute(t1, row);
            if (row + 2 * kChunkStep < end) ln.load(t1, row + 2 * kChunkStep);
            row += kChunkStep;
        }
    }
    if (ln.fault && lane == 0) atomicOr(a.faults, ln.fault);

    // the waves joined: columns of LDS, then one thread per four elements of a head
    l = rows_allsum(l);
    const int columns = CP * group;
    float* stat = lds + kWaves * columns * kStride;
    if (column) {
        float* out = lds + (wave * columns + c) * kStride + s * (D / 4);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int x = 0; x < kOut; x += 4)
                *reinterpret_cast<f32x4*>(out + i * kOut + x) = f32x4{acc[x][i], acc[x + 1][i], acc[x + 2][i], acc[x + 3][i]};
        if (s == 0 && part == 0) {
            stat[wave * group + head] = m;
            stat[(kWaves + wave) * group + head] = l;
        }
    }
    __syncthreads();
    const size_t head0 = (size_t)lb * d.hq + g * group;
    for (int i = threadIdx.x; i < group * (D / 4); i += kThreads) {
        const int h = i / (D / 4), e = i % (D / 4) * 4;
        float top = stat[h];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) top = fmaxf(top, stat[w * group + h]);
        float sum = 0.0f;
        f32x4 o{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float f = exp2_hw(stat[w * group + h] - top);
            sum += f * stat[(kWaves + w) * group + h];
            f32x4 x = *reinterpret_cast<const f32x4*>(lds + (w * columns + h) * kStride + e);
#pragma unroll
            for (int k = 1; k < CP; ++k) x += *reinterpret_cast<const f32x4*>(lds + (w * columns + k * group + h) * kStride + e);
            o += x * f;
        }
        if (e == 0) a.part[((size_t)slab * a.nchunk + chunk) * group + h] = make_float2(top, sum);
        if (a.nchunk == 1) {
            const float inv = sum != 0.0f ? 1.0f / sum : 0.0f;
            T* op = static_cast<T*>(a.o) + (head0 + h) * D + e;
#pragma unroll
            for (int j = 0; j < 4; ++j) Elem<T>::store(op + j, o[j] * inv);
        } else {
            *reinterpret_cast<f32x4*>(a.opart + (((size_t)slab * a.nchunk + chunk) * group + h) * D + e) = o;
        }
    }
}

// Several chunks: one workgroup per (slab, head) joins their outputs and statistics, and leaves the head's own statistics in
// the place of its first chunk's.
constexpr int kJoinThreads = 256;
template <typename T, int D>
__global__ __launch_bounds__(kJoinThreads) void q4_join_kernel(Q4AttendArgs a) {
    constexpr int kQuads = D / 4, kRows = kJoinThreads / kQuads;
    __shared__ f32x4 red[kRows][kQuads];
    __shared__ float mx[kJoinThreads / kWave], sm[kJoinThreads / kWave];
    const Q4Dims& d = a.dims;
    const int slab = blockIdx.x / d.group, h = blockIdx.x % d.group;
    const int lb = slab / d.hkv, g = slab % d.hkv;
    const int n = attended(a, lb % d.batch);
    const int chunks = max(1, (n + a.chunk_rows - 1) / a.chunk_rows);
    const size_t at = (size_t)slab * a.nchunk * d.group + h;
    float top = -FLT_MAX;
    for (int i = threadIdx.x; i < chunks; i += kJoinThreads) top = fmaxf(top, a.part[at + (size_t)i * d.group].x);
    top = wave_max(top);
    if (threadIdx.x % kWave == 0) mx[threadIdx.x / kWave] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kJoinThreads / kWave; ++w) top = fmaxf(top, mx[w]);
    float sum = 0.0f;
    for (int i = threadIdx.x; i < chunks; i += kJoinThreads) {
        const float2 p = a.part[at + (size_t)i * d.group];
        sum += exp2_hw(p.x - top) * p.y;
    }
    sum = wave_sum(sum);
    if (threadIdx.x % kWave == 0) sm[threadIdx.x / kWave] = sum;
    const int quad = threadIdx.x % kQuads, r = threadIdx.x / kQuads;
    f32x4 o{0.0f, 0.0f, 0.0f, 0.0f};
    for (int i = r; i < chunks; i += kRows) {
        const size_t p = at + (size_t)i * d.group;
        o += *reinterpret_cast<const f32x4*>(a.opart + p * D + quad * 4) * exp2_hw(a.part[p].x - top);
    }
    red[r][quad] = o;
    __syncthreads();
    sum = 0.0f;
#pragma unroll
    for (int w = 0; w < kJoinThreads / kWave; ++w) sum += sm[w];
    if (threadIdx.x == 0) a.part[at] = make_float2(top, sum);
    if (r != 0) return;
#pragma unroll
    for (int i = 1; i < kRows; ++i) o += red[i][quad];
    const float inv = sum != 0.0f ? 1.0f / sum : 0.0f;
    T* op = static_cast<T*>(a.o) + ((size_t)lb * d.hq + g * d.group + h) * D + quad * 4;
#pragma unroll
    for (int j = 0; j < 4; ++j) Elem<T>::store(op + j, o[j] * inv);
}

// Scores of 4 rows a thread of one (layer, sequence), from the logits and the heads' statistics; with one layer in the call
// also its fold.
constexpr int kScoreThreads = 128;
__global__ __launch_bounds__(kScoreThreads) void q4_score_kernel(Q4AttendArgs a, float* s_rows, int s_stride) {
    extern __shared__ float2 stat[];  // [hq]: maximum, 1 / (H sum)
    const Q4Dims& d = a.dims;
    const int blocks = (a.n_max + kScoreThreads * 4 - 1) / (kScoreThreads * 4);
    const int lb = blockIdx.x / blocks, row = (blockIdx.x % blocks * kScoreThreads + threadIdx.x) * 4;
    const int b = lb % d.batch, n = attended(a, b);
    for (int h = threadIdx.x; h < d.hq; h += kScoreThreads) {
        const float2 p = a.part[((size_t)lb * d.hkv + h / d.group) * a.nchunk * d.group + h % d.group];
        stat[h] = make_float2(p.x, p.y != 0.0f ? 1.0f / (p.y * (float)d.hq) : 0.0f);
    }
    __syncthreads();
    if (row >= a.n_max) return;
    f32x4 s{0.0f, 0.0f, 0.0f, 0.0f};
    if (row < n)
        for (int h = 0; h < d.hq; ++h) {
            const f32x4 z = *reinterpret_cast<const f32x4*>(a.z + ((size_t)lb * d.hq + h) * a.n_stride + row);
            const float2 p = stat[h];
#pragma unroll
            for (int i = 0; i < 4; ++i) s[i] = fmaf(exp2_hw(z[i] - p.x), p.y, s[i]);
        }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (row + i >= a.n_max) break;
        const bool live = row + i < n;
        const float x = live ? s[i] : 0.0f;
        if (s_rows) s_rows[(size_t)lb * s_stride + row + i] = x;
        if (a.u_out && a.layer_count == 1 && live) {
            const size_t at = (size_t)b * d.cap + row + i;
            a.u_out[at] = a.alpha * a.u_prior[at] + (1.0f - a.alpha) * x;
        }
    }
}

// The fold of several layers' scores, a row per thread.
constexpr int kFoldThreads = 64;
__global__ __launch_bounds__(kFoldThreads) void q4_fold_kernel(Q4AttendArgs a, const float* s_rows, int s_stride) {
    const Q4Dims& d = a.dims;
    const int blocks = (a.n_max + kFoldThreads - 1) / kFoldThreads;
    const int b = blockIdx.x / blocks, row = blockIdx.x % blocks * kFoldThreads + threadIdx.x;
    if (row >= attended(a, b)) return;
    float u = a.u_prior[(size_t)b * d.cap + row];
#pragma unroll 8
    for (int l = 0; l < a.layer_count; ++l)
        u = a.alpha * u + (1.0f - a.alpha) * s_rows[((size_t)l * d.batch + b) * s_stride + row];
    a.u_out[(size_t)b * d.cap + row] = u;
}

template <typename T, int D, int CP, int NM>
hipError_t launch_attend(const Q4AttendArgs& a, hipStream_t s) {
    const int slabs = a.layer_count * a.dims.batch * a.dims.hkv;
    const size_t lds = (size_t)kWaves * a.dims.group * (CP * (D + 4) + 2) * sizeof(float);
    if (a.bias2 != 0.0f)
        hipLaunchKernelGGL((q4_attend_kernel<T, D, CP, NM, true>), dim3(slabs * a.nchunk), dim3(kThreads), lds, s, a);
    else
        hipLaunchKernelGGL((q4_attend_kernel<T, D, CP, NM, false>), dim3(slabs * a.nchunk), dim3(kThreads), lds, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.nchunk == 1) return e;
    hipLaunchKernelGGL((q4_join_kernel<T, D>), dim3(slabs * a.dims.group), dim3(kJoinThreads), 0, s, a);
    return hipGetLastError();
}

// Columns of the parts of a probability: as many as fit beside each other.
template <int D>
hipError_t launch_by_group(const Q4AttendArgs& a, hipStream_t s) {
    const int group = a.dims.group;
    if (a.dims.bf16) return group <= 8 ? launch_attend<bf16_t, D, 2, 1>(a, s) : launch_attend<bf16_t, D, 1, 2>(a, s);
    return group <= 5 ? launch_attend<float, D, 3, 1>(a, s) : launch_attend<float, D, 1, 3>(a, s);
}

}  // namespace

int q4_attend_chunks(int slabs, int n) {
    const int want = (kTargetWgs + slabs - 1) / slabs, by_rows = (n + kChunkStep - 1) / kChunkStep;
    return want < by_rows ? want : by_rows;
}

void q4_attend_plan(int slabs, int n, int* nchunk, int* chunk_rows) {
    const int chunks = q4_attend_chunks(slabs, n);
    const int rows = (n + chunks - 1) / chunks;
    *chunk_rows = (rows + kChunkStep - 1) / kChunkStep * kChunkStep;
    *nchunk = (n + *chunk_rows - 1) / *chunk_rows;
}

hipError_t launch_q4_attend(const Q4AttendArgs& a, hipStream_t s) {
    hipError_t e = a.dims.d == 128 ? launch_by_group<128>(a, s) : launch_by_group<64>(a, s);
    if (e != hipSuccess || !a.z) return e;
    const int blocks = (a.n_max + kScoreThreads * 4 - 1) / (kScoreThreads * 4);
    float* rows = a.s_out ? a.s_out : a.layer_count > 1 ? a.s_scratch : nullptr;
    const int stride = a.s_out ? a.n_max : a.n_stride;
    hipLaunchKernelGGL(q4_score_kernel, dim3(a.layer_count * a.dims.batch * blocks), dim3(kScoreThreads),
                       a.dims.hq * sizeof(float2), s, a, rows, stride);
    e = hipGetLastError();
    if (e != hipSuccess || !a.u_out || a.layer_count == 1) return e;
    const int folds = (a.n_max + kFoldThreads - 1) / kFoldThreads;
    hipLaunchKernelGGL(q4_fold_kernel, dim3(a.dims.batch * folds), dim3(kFoldThreads), 0, s, a, rows, stride);
    return hipGetLastError();
}

}  // namespace ikv
