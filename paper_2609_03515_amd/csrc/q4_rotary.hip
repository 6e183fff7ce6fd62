// Rotated rows into the paged 4-bit cache.
//
// Pair i of a row's first `dim` elements turns by angle = position[axis(i)] * inv_freq(i): (x, y) -> scale (x cos - y sin,
// x sin + y cos); the other elements pass.  The pairs are elements i and i + dim / 2, or 2 i and 2 i + 1.  Queries are written
// rotated, keys are quantised from their rotated values, values as they are (q4_rows.hip).
//
// Angles, their cosine and sine and the rotation of keys are in 64 bits: a position of 20 bits times a frequency takes 44, and a code
// is then the nearest to the exact rotated element, where 32 bits would choose a neighbour for one element in millions.  They are
// rounded once, to 32 bits with the last bit set where something was cut off (to odd), so that the rounding to a code, of fewer bits
// by far, sees on which side of a border the 64-bit value lies.  Queries, which no border cuts, are turned in 32 bits by cosines
// and sines rounded from 64 (13,000 tokens of 28/4 heads: 69.5 us with everything in 64 bits, of which the conversions were most).
//
// A workgroup takes the rows of 512 / D tokens of one layer, a wave one head of them at a time, a lane 8 elements: the tokens'
// cosines and sines are made once, in LDS, and stay in a lane's registers over the queries' heads.  The partners are loaded beside
// the elements (from the same lines: the second load comes from the cache).
//
// What bounds it: with many rows the memory (one layer of some 13,000 tokens of 28 query and 4 KV heads, three axes: 58 us for 223 MB,
// 3.8 TB/s; queries alone 4.2 TB/s; with nothing written 38 us); with few, one token of 8 slots in 32 layers, latency (7.2 us: the launch
// and a chain of count and length, page, rows).
#include "kv_common.h"
#include "q4.h"
#include "q4_block.h"

namespace ikv {
namespace {

constexpr int kRotaryThreads = 256, kRotaryWaves = kRotaryThreads / kWave;

// x in 32 bits, rounded to odd: exact, or the neighbour whose last bit is set.
__device__ __forceinline__ float to_odd(double x) {
    const float f = (float)x;
    const double back = (double)f;
    uint32_t w = __float_as_uint(f);
    if (back != x && x == x && !(w & 1u)) w += fabs(back) < fabs(x) ? 1u : ~0u;
    return __uint_as_float(w);
}

// A lane's elements as two runs of four: bf16 8 p .. 8 p + 7, f32 4 p .. 4 p + 3 of either half of the row (as read8).
template <typename T, int D>
__device__ __forceinline__ int run_of(int p, int half) {
    return sizeof(T) == 2 ? 8 * p + 4 * half : half * (D / 2) + 4 * p;
}
template <typename T>
__device__ __forceinline__ void read4(const T* at, float (&x)[4]) {
    if constexpr (sizeof(T) == 2) {
        const uint2 w = *reinterpret_cast<const uint2*>(at);
        x[0] = __uint_as_float(w.x << 16);
        x[1] = __uint_as_float(w.x & 0xffff0000u);
        x[2] = __uint_as_float(w.y << 16);
        x[3] = __uint_as_float(w.y & 0xffff0000u);
    } else {
        const f32x4 w = *reinterpret_cast<const f32x4*>(at);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = w[i];
    }
}
// Two numbers rounded to bf16, to nearest even.
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    typedef float __attribute__((ext_vector_type(2))) f32x2;
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2));
}

template <typename T, int D>
__global__ __launch_bounds__(kRotaryThreads) void q4_rotary_kernel(Q4RotaryArgs a) {
    constexpr int kLanes = D / kElems, kTokens = kWave / kLanes;
    __shared__ double2 turn[kTokens][D / 2 + 1];  // (one more: the tokens' rows start in other banks)
    const Q4Dims& d = a.rows.dims;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int p = lane % kLanes, layer = blockIdx.y;
    const int tokens = d.batch * a.rows.rows, pairs = a.dim / 2;

    for (int i = threadIdx.x; i < kTokens * pairs; i += kRotaryThreads) {
        const int t = i / pairs, k = i - t * pairs, token = blockIdx.x * kTokens + t;
        if (token >= tokens) break;
        const int b = token / a.rows.rows, r = token - b * a.rows.rows;
        if (r >= (a.rows.count ? a.rows.count[b] : a.rows.rows)) continue;  // (its positions are not read)
        const int at = a.positions[(size_t)a.axis[k] * tokens + token];
        double s, c;
        sincos((double)at * (double)a.inv_freq[k], &s, &c);
        turn[t][k] = make_double2(c * a.scale, s * a.scale);
    }

    // the lane's token: where its row lies in the cache
    const int token = blockIdx.x * kTokens + lane / kLanes;
    const int b = min(token, tokens - 1) / a.rows.rows, r = min(token, tokens - 1) - b * a.rows.rows;
    const int count = a.rows.count ? a.rows.count[b] : a.rows.rows, len = a.rows.cache.len[b];
    const int64_t row = (a.rows.first ? (int64_t)a.rows.first[b] : (int64_t)len - count) + r;
    const bool wanted = token < tokens && r < count;
    const bool in = row >= 0 && row < len && row < d.cap;
    const int page = a.rows.cache.table[(size_t)b * d.max_pages + (in ? (int)(row >> d.page_shift) : 0)];
    const bool there = in && (uint32_t)page < (uint32_t)d.n_pages;
    const int refs = there ? a.rows.cache.refs[page] : 1;
    const bool stored = wanted && there && refs == 1;
    const int in_page = (int)row & (d.page_rows - 1);
    if (blockIdx.z == 0 && wave == 0 && p == 0) {
        uint32_t fault = 0;
        if (token < tokens && r == 0 && (uint32_t)count > (uint32_t)a.rows.rows) fault |= kFaultCache;
        if (wanted && !there) fault |= kFaultCache;
        if (wanted && refs != 1) fault |= refs > 1 ? kFaultSharedPage : kFaultCache;
        if (fault) atomicOr(a.rows.faults, fault);
    }
    __syncthreads();

    // where the partners of the lane's two runs of four begin (neighbours: the run itself), and what an element and its partner are
    // multiplied with
    int partner[2];
    bool turned[2], low[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int e = run_of<T, D>(p, h);
        turned[h] = e < a.dim;
        low[h] = a.adjacent || e < pairs;
        partner[h] = !turned[h] || a.adjacent ? e : low[h] ? e + pairs : e - pairs;
    }
    auto factors = [&](int h, int i) __attribute__((always_inline)) {
        const int e = run_of<T, D>(p, h), k = a.adjacent ? (e + i) / 2 : low[h] ? e + i : e + i - pairs;
        double2 x = turn[lane / kLanes][turned[h] ? k : 0];
        if (a.adjacent ? i % 2 == 0 : low[h]) x.y = -x.y;
        return x;
    };
    const int first = blockIdx.z * kRotaryWaves + wave, stride = gridDim.z * kRotaryWaves, queries = a.q ? d.hq : 0;
    // the queries' heads, two at a time: their loads together
    if (wanted && first < queries) {
        float c[2][4], s[2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const double2 x = factors(h, i);
                c[h][i] = (float)x.x;
                s[h][i] = (float)x.y;
            }
        const T* const from = static_cast<const T*>(a.q) + layer * a.qs[0] + b * a.qs[1] + r * a.qs[3];
        T* const to = static_cast<T*>(a.q_out) + layer * a.os[0] + b * a.os[1] + r * a.os[3];
        for (int u = first; u < queries; u += 2 * stride) {
            float own[2][2][4], other[2][2][4];
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const T* const row = from + min(u + j * stride, queries - 1) * a.qs[2];
                    read4(row + run_of<T, D>(p, h), own[j][h]);
                    read4(row + partner[h], other[j][h]);
                }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                if (u + j * stride >= queries) break;
                float x[kElems];
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float y = a.adjacent ? own[j][h][i ^ 1] : other[j][h][i];
                        x[4 * h + i] = turned[h] ? fmaf(y, s[h][i], own[j][h][i] * c[h][i]) : own[j][h][i];
                    }
                T* const out = to + (u + j * stride) * a.os[2];
                if constexpr (sizeof(T) == 2) {
                    reinterpret_cast<u32x4*>(out)[p] = u32x4{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])};
                } else {
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        *reinterpret_cast<f32x4*>(out + run_of<T, D>(p, h)) = f32x4{x[4 * h], x[4 * h + 1], x[4 * h + 2], x[4 * h + 3]};
                }
            }
        }
    }
    // the keys' heads and the values'
    if (!stored) return;
    for (int u = first < queries ? first + (queries - first + stride - 1) / stride * stride : first; u < queries + 2 * d.hkv; u += stride) {
        const bool value = u - queries >= d.hkv;
        const int g = value ? u - queries - d.hkv : u - queries;
        float x[kElems];
        if (value) {
            read8<T, D>(static_cast<const T*>(a.rows.v) + layer * a.rows.vs[0] + b * a.rows.vs[1] + g * a.rows.vs[2] + r * a.rows.vs[3], p, x);
        } else {
            const T* const row = static_cast<const T*>(a.rows.k) + layer * a.rows.ks[0] + b * a.rows.ks[1] + g * a.rows.ks[2] + r * a.rows.ks[3];
            float own[2][4], other[2][4];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                read4(row + run_of<T, D>(p, h), own[h]);
                read4(row + partner[h], other[h]);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const double2 f = factors(h, i);
                    const float y = a.adjacent ? own[h][i ^ 1] : other[h][i];
                    x[4 * h + i] = turned[h] ? to_odd((double)own[h][i] * f.x + (double)y * f.y) : own[h][i];
                }
        }
        uint8_t* rec = a.rows.cache.pool + q4_record(d, a.rows.layer0 + layer, page, g);
        uint32_t scales;
        const uint32_t codes = quantise<T, D>(x, p, &scales);
        put_codes<T, D>(rec + (value ? d.vc_off : 0) + in_page * (D / 2), p, codes);
        uint8_t* e = rec + (value ? d.vs_off : d.ks_off);
        if (p == 0) {
            if constexpr (D == 128) reinterpret_cast<uint32_t*>(e)[in_page] = scales;
            else reinterpret_cast<uint16_t*>(e)[in_page] = (uint16_t)scales;
        }
    }
}

template <typename T, int D>
hipError_t launch_rotary(const Q4RotaryArgs& a, hipStream_t s) {
    constexpr int kTokens = kWave / (D / kElems);
    const int blocks = (a.rows.dims.batch * a.rows.rows + kTokens - 1) / kTokens, heads = (a.q ? a.rows.dims.hq : 0) + 2 * a.rows.dims.hkv;
    // The heads of a token block are divided among workgroups (each makes the block's angles again) until there are four for a CU.
    const int cus = device_cus() > 0 ? device_cus() : 256;
    const int most = (heads + kRotaryWaves - 1) / kRotaryWaves, want = (int)((4ll * cus + (int64_t)blocks * a.rows.layer_count - 1) / ((int64_t)blocks * a.rows.layer_count));
    hipLaunchKernelGGL((q4_rotary_kernel<T, D>), dim3(blocks, a.rows.layer_count, want < most ? want : most), dim3(kRotaryThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_q4_store_rotary(const Q4RotaryArgs& a, hipStream_t s) {
    if (a.rows.dims.bf16) return a.rows.dims.d == 128 ? launch_rotary<bf16_t, 128>(a, s) : launch_rotary<bf16_t, 64>(a, s);
    return a.rows.dims.d == 128 ? launch_rotary<float, 128>(a, s) : launch_rotary<float, 64>(a, s);
}

}  // namespace ikv
