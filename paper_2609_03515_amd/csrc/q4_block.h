// Rows of the paged 4-bit cache: a lane's elements of a dense row, and their codes and scales (q4_rows.hip, q4_rotary.hip).
#pragma once

#include "kv_common.h"
#include "q4.h"

namespace ikv {
namespace {

constexpr int kElems = 8;       // elements per lane
constexpr int kQ4MinByte = 27;  // e = -100
constexpr int kQ4MaxByte = 252; // e = 125

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_u(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, true);
}

// A lane's 8 elements of a row: bf16 elements 8 p .. 8 p + 7, f32 elements 4 p .. 4 p + 3 of either half of the row, so that the
// lanes' 16-byte accesses are consecutive.
template <typename T, int D>
__device__ __forceinline__ void read8(const T* row, int p, float (&x)[kElems]) {
    if constexpr (sizeof(T) == 2) {
        Elem<bf16_t>::unpack(__builtin_nontemporal_load(reinterpret_cast<const u32x4*>(row) + p), x);
    } else {
        const f32x4 lo = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(row) + p);
        const f32x4 hi = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(row) + D / 8 + p);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = lo[i];
            x[4 + i] = hi[i];
        }
    }
}

__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }
// A block's scale byte by its largest |x| as an integer (order-preserving, NaN above infinity above every number): the exponent,
// one higher from 1.75 * 2^k on, less 2 is the smallest e with max |x| < 7 * 2^e.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
    const int e = (int)((top + 0x00200000u) >> 23) - 2;
    return top >= 0x7f800000u ? 255u : (uint32_t)min(max(e, kQ4MinByte), kQ4MaxByte);
}

// The codes of a lane's elements, and its row's scale bytes together (in every lane).
template <typename T, int D>
__device__ __forceinline__ uint32_t quantise(const float (&x)[kElems], int p, uint32_t* scales) {
    uint32_t w = 0;
    if constexpr (sizeof(T) == 2) {  // a block is a quad of lanes
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < kElems; ++i) top = max(top, magnitude(x[i]));
        top = max(top, dpp_u<kXor1>(top));
        top = max(top, dpp_u<kXor2>(top));
        const uint32_t byte = scale_byte(top);
        const float scale = __uint_as_float(byte << 23);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
        if (byte == 255u) w = 0;
        uint32_t s = byte << 8 * (p / 4);
        s |= dpp_u<kMirror8>(s);
        if constexpr (D == 128) s |= dpp_u<kRor8>(s);
        *scales = s;
    } else {  // a block is 8 lanes of one half
        uint32_t top[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            top[h] = max(max(magnitude(x[4 * h]), magnitude(x[4 * h + 1])), max(magnitude(x[4 * h + 2]), magnitude(x[4 * h + 3])));
            top[h] = max(top[h], dpp_u<kXor1>(top[h]));
            top[h] = max(top[h], dpp_u<kXor2>(top[h]));
            top[h] = max(top[h], dpp_u<kMirror8>(top[h]));
        }
        const uint32_t b0 = scale_byte(top[0]), b1 = scale_byte(top[1]);
        const float s0 = __uint_as_float(b0 << 23), s1 = __uint_as_float(b1 << 23);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], s0, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], s0, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], s1, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], s1, 3);
        if (b0 == 255u) w &= 0xffff0000u;
        if (b1 == 255u) w &= 0x0000ffffu;
        if constexpr (D == 128) {
            uint32_t s = (b0 | b1 << 16) << 8 * (p / 8);
            s |= dpp_u<kRor8>(s);
            *scales = s;
        } else {
            *scales = b0 | b1 << 8;
        }
    }
    return w;
}

// A lane's codes in a row of codes, and back.
template <typename T, int D>
__device__ __forceinline__ void put_codes(uint8_t* row, int p, uint32_t w) {
    if constexpr (sizeof(T) == 2) {
        reinterpret_cast<uint32_t*>(row)[p] = w;
    } else {
        reinterpret_cast<uint16_t*>(row)[p] = (uint16_t)w;
        reinterpret_cast<uint16_t*>(row)[D / 8 + p] = (uint16_t)(w >> 16);
    }
}
template <typename T, int D>
__device__ __forceinline__ uint32_t get_codes(const uint8_t* row, int p) {
    if constexpr (sizeof(T) == 2) return reinterpret_cast<const uint32_t*>(row)[p];
    else return reinterpret_cast<const uint16_t*>(row)[p] | (uint32_t)reinterpret_cast<const uint16_t*>(row)[D / 8 + p] << 16;
}

}  // namespace
}  // namespace ikv
