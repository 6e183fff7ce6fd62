// Pieces of the 4-bit cache's attention kernels (q4_attend.hip, q4_queries.hip): tiles of 32 rows, their values in LDS, conversions
// and products.  The lane's elements and rows are described in q4_attend.hip.
#pragma once

#include "kv_common.h"
#include "q4.h"

namespace ikv {
namespace {

constexpr int kTile = 32;             // rows of a wave's tile: two halves of 16, each in one page
constexpr float kSlack = 8.0f;        // what a logit may exceed the running maximum by, in powers of two

typedef __bf16 __attribute__((ext_vector_type(8))) bf16x8;
typedef uint32_t __attribute__((ext_vector_type(2))) u32x2;
typedef const __attribute__((address_space(4))) int32_t* scalar_ints;  // read by scalar loads: not written by the kernel

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

// A tile's values go straight to LDS, [32 rows][D / 2] bytes of codes, then [32 rows][D / 32] scale bytes (a whole load
// instruction's 256 bytes of place, of which the first are used): no registers while they are on their way.
constexpr int kScalePlace = 256;
template <int D>
constexpr int kValueBytes = kTile * (D / 2) + kScalePlace;
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(1))) const void global_void;
constexpr int kNt = 2;  // non-temporal: read once

template <int BYTES, int POLICY = kNt>
__device__ __forceinline__ void to_lds(const uint8_t* from, uint8_t* to) {  // lane i's BYTES to `to` (uniform) + i * BYTES
    static_assert(BYTES == 4 || BYTES == 16, "sizes used here");
    if constexpr (BYTES == 16) __builtin_amdgcn_global_load_lds((global_void*)from, (lds_void*)to, 16, 0, POLICY);
    else __builtin_amdgcn_global_load_lds((global_void*)from, (lds_void*)to, 4, 0, POLICY);
}

}  // namespace
}  // namespace ikv
