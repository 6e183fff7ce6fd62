// Rows into the paged 4-bit cache and back.
//
// Store: each block of 32 elements gets the smallest power of two 2^e with max |x| < 7 * 2^e (6 is the largest code, and
// what lies under 7 is within half of the step from 4 to 6 of it), and its elements x / 2^e rounded to the nearest code,
// ties to the even one, by the hardware's conversion.  e is held to [-100, 125]: below, every product with a code stays a
// normal bf16 number, and what is smaller than 2^-102 becomes zero; above, 6 * 2^125 is still finite.  A block with an
// element that is not finite gets the scale byte 255 and codes 0, which reads back as NaN.
//
// Both directions are bound by memory traffic: a lane takes 8 elements (16 bytes of bf16, 4 bytes of codes), so a row of
// 128 is 16 lanes and a block's maximum needs two steps inside a quad of lanes.
#include "kv_common.h"
#include "q4.h"

namespace ikv {
namespace {

constexpr int kThreads = 256;
constexpr int kElems = 8;       // elements per lane
constexpr int kQ4MinByte = 27;  // e = -100
constexpr int kQ4MaxByte = 252; // e = 125

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_u(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, true);
}

// One row of the cache, for the lanes that hold it: where it lies, or page < 0 (none).
struct RowAt {
    int page, row;
};

// Cached row first + r of sequence b: `wanted` where r < count; a page only where the row exists.
__device__ __forceinline__ RowAt locate(const Q4RowArgs& a, int b, int r, bool* wanted, uint32_t* fault) {
    const Q4Dims& d = a.dims;
    const int count = a.count ? a.count[b] : a.rows;
    *wanted = r < count;
    RowAt at{-1, 0};
    if (!*wanted) return at;
    const int len = a.cache.len[b];
    const int64_t row = (int64_t)(a.first ? a.first[b] : (int64_t)len - count) + r;
    if (row < 0 || row >= len || row >= d.cap) {
        *fault |= kFaultCache;
        return at;
    }
    const int page = a.cache.table[(size_t)b * d.max_pages + (int)(row >> d.page_shift)];
    if ((uint32_t)page >= (uint32_t)d.n_pages) {
        *fault |= kFaultCache;
        return at;
    }
    at.page = page;
    at.row = (int)row & (d.page_rows - 1);
    return at;
}

// Work item `i` of a call: row r of (layer l, sequence b, KV head g), rows fastest.
struct Item {
    int l, b, g, r;
};
__device__ __forceinline__ Item item_of(const Q4RowArgs& a, uint32_t i) {
    const uint32_t slab = i / (uint32_t)a.rows;
    const uint32_t lb = slab / (uint32_t)a.dims.hkv;
    return {(int)(lb / (uint32_t)a.dims.batch), (int)(lb % (uint32_t)a.dims.batch), (int)(slab % (uint32_t)a.dims.hkv),
            (int)(i % (uint32_t)a.rows)};
}
__device__ __forceinline__ size_t source_of(const Item& it, const int64_t (&s)[4]) {
    return (size_t)(it.l * s[0] + it.b * s[1] + it.g * s[2] + it.r * s[3]);
}

template <typename T>
__device__ __forceinline__ void read8(const T* p, float (&x)[kElems]) {
    if constexpr (sizeof(T) == 2) {
        Elem<bf16_t>::unpack(*reinterpret_cast<const u32x4*>(p), x);
    } else {
        const f32x4 lo = reinterpret_cast<const f32x4*>(p)[0], hi = reinterpret_cast<const f32x4*>(p)[1];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = lo[i];
            x[4 + i] = hi[i];
        }
    }
}

// A lane's 8 elements and its quad's block of 32: the codes, and the block's scale byte.
__device__ __forceinline__ uint32_t quantise(const float (&x)[kElems], uint32_t* byte) {
    uint32_t top = 0;  // |x| as integers: order-preserving, NaN above infinity above every number
#pragma unroll
    for (int i = 0; i < kElems; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
    top = max(top, dpp_u<kXor1>(top));
    top = max(top, dpp_u<kXor2>(top));
    // the exponent, one higher from 1.75 * 2^k on: the smallest e with max |x| < 7 * 2^e is then two below it
    const int e = (int)((top + 0x00200000u) >> 23) - 2;
    const bool finite = top < 0x7f800000u;
    const uint32_t E = (uint32_t)min(max(e, kQ4MinByte), kQ4MaxByte);
    const float scale = __uint_as_float(E << 23);
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
    *byte = finite ? E : 255u;
    return finite ? w : 0u;
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void q4_store_kernel(Q4RowArgs a, uint32_t items) {
    constexpr int kLanes = D / kElems;  // lanes per row
    const int p = threadIdx.x % kLanes;
    const uint32_t i = blockIdx.x * (kThreads / kLanes) + threadIdx.x / kLanes;
    if (i >= items) return;  // (whole rows of lanes)
    const Item it = item_of(a, i);
    bool wanted;
    uint32_t fault = 0;
    RowAt at = locate(a, it.b, it.r, &wanted, &fault);
    if (at.page >= 0) {
        const int refs = a.cache.refs[at.page];
        if (refs != 1) {
            fault |= refs > 1 ? kFaultSharedPage : kFaultCache;
            at.page = -1;
        }
    }
    if (fault && p == 0) atomicOr(a.faults, fault);
    if (at.page < 0) return;
    uint8_t* rec = a.cache.pool + q4_record(a.dims, a.layer0 + it.l, at.page, it.g);
    float xk[kElems], xv[kElems];
    read8(static_cast<const T*>(a.k) + source_of(it, a.ks) + p * kElems, xk);
    read8(static_cast<const T*>(a.v) + source_of(it, a.vs) + p * kElems, xv);
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        uint32_t byte;
        const uint32_t codes = quantise(which ? xv : xk, &byte);
        // the row's scale bytes gathered by its lanes, one store for them
        uint32_t word = byte << 8 * (p / 4);
        word |= dpp_u<kMirror8>(word);
        uint8_t* c = rec + (which ? a.dims.vc_off : 0);
        uint8_t* e = rec + (which ? a.dims.vs_off : a.dims.ks_off);
        reinterpret_cast<uint32_t*>(c + at.row * (D / 2))[p] = codes;
        if constexpr (D == 128) {
            word |= dpp_u<kRor8>(word);
            if (p == 0) reinterpret_cast<uint32_t*>(e)[at.row] = word;
        } else {
            if (p == 0) reinterpret_cast<uint16_t*>(e)[at.row] = (uint16_t)word;
        }
    }
}

// 8 codes and their scale as 8 bf16 (exact)
__device__ __forceinline__ u32x4 expand(uint32_t codes, uint32_t byte) {
    const float scale = __uint_as_float(byte << 23);
    u32x4 r;
    r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
    r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
    r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
    r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
    return r;
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void q4_load_kernel(Q4RowArgs a, uint32_t items) {
    constexpr int kLanes = D / kElems;
    const int p = threadIdx.x % kLanes;
    const uint32_t i = blockIdx.x * (kThreads / kLanes) + threadIdx.x / kLanes;
    if (i >= items) return;
    const Item it = item_of(a, i);
    bool wanted;
    uint32_t fault = 0;
    const RowAt at = locate(a, it.b, it.r, &wanted, &fault);
    if (fault && p == 0) atomicOr(a.faults, fault);
    if (!wanted) return;
    uint32_t codes[2] = {0, 0}, byte[2] = {127, 127};  // a row that is not there: zeros
    if (at.page >= 0) {
        const uint8_t* rec = a.cache.pool + q4_record(a.dims, a.layer0 + it.l, at.page, it.g);
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            codes[which] = reinterpret_cast<const uint32_t*>(rec + (which ? a.dims.vc_off : 0) + at.row * (D / 2))[p];
            byte[which] = rec[(which ? a.dims.vs_off : a.dims.ks_off) + at.row * (D / 32) + p / 4];
        }
    }
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        T* out = static_cast<T*>(which ? a.v_out : a.k_out) + source_of(it, which ? a.vs : a.ks) + p * kElems;
        const u32x4 x = expand(codes[which], byte[which]);
        if constexpr (sizeof(T) == 2) {
            *reinterpret_cast<u32x4*>(out) = x;
        } else {
            float f[kElems];
            Elem<bf16_t>::unpack(x, f);
            reinterpret_cast<f32x4*>(out)[0] = f32x4{f[0], f[1], f[2], f[3]};
            reinterpret_cast<f32x4*>(out)[1] = f32x4{f[4], f[5], f[6], f[7]};
        }
    }
}

}  // namespace

hipError_t launch_q4_store(const Q4RowArgs& a, hipStream_t s) {
    const uint32_t items = (uint32_t)a.layer_count * a.dims.batch * a.dims.hkv * a.rows;
    const uint32_t per = kThreads * kElems / a.dims.d;
    const dim3 grid((items + per - 1) / per), block(kThreads);
    if (a.dims.bf16)
        hipLaunchKernelGGL((a.dims.d == 128 ? q4_store_kernel<bf16_t, 128> : q4_store_kernel<bf16_t, 64>), grid, block, 0, s, a, items);
    else
        hipLaunchKernelGGL((a.dims.d == 128 ? q4_store_kernel<float, 128> : q4_store_kernel<float, 64>), grid, block, 0, s, a, items);
    return hipGetLastError();
}

hipError_t launch_q4_load(const Q4RowArgs& a, hipStream_t s) {
    const uint32_t items = (uint32_t)a.layer_count * a.dims.batch * a.dims.hkv * a.rows;
    const uint32_t per = kThreads * kElems / a.dims.d;
    const dim3 grid((items + per - 1) / per), block(kThreads);
    if (a.dims.bf16)
        hipLaunchKernelGGL((a.dims.d == 128 ? q4_load_kernel<bf16_t, 128> : q4_load_kernel<bf16_t, 64>), grid, block, 0, s, a, items);
    else
        hipLaunchKernelGGL((a.dims.d == 128 ? q4_load_kernel<float, 128> : q4_load_kernel<float, 64>), grid, block, 0, s, a, items);
    return hipGetLastError();
}

}  // namespace ikv
