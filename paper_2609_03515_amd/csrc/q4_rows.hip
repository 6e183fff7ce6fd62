// Rows into the paged 4-bit cache and back.
//
// Store: each block of 32 elements gets the smallest power of two 2^e with max |x| < 7 * 2^e (6 is the largest code, and
// what lies under 7 is within half of the step from 4 to 6 of it), and its elements x / 2^e rounded to the nearest code,
// ties to the even one, by the hardware's conversion.  e is held to [-100, 125]: below, every product with a code stays a
// normal bf16 number, and what is smaller than 2^-102 becomes zero; above, 6 * 2^125 is still finite.  A block with an
// element that is not finite gets the scale byte 255 and codes 0, which reads back as NaN.
//
// Both directions are bound by memory traffic: a lane takes 8 elements (16 bytes of bf16, 4 bytes of codes), so a row of
// 128 is 16 lanes and a block's maximum needs two or three steps between neighbouring lanes.
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

// A work item: row r of (layer l, sequence b, KV head g), rows fastest, and where it lies in the cache.
struct Item {
    int l, b, g, r;
    bool wanted;     // r < count
    int page, row;   // page < 0: the cache has no such row
};

// Items first, first + step, ... of a thread, located together: their loads in flight at once (items past the last one repeat
// it, and are not wanted).
template <int N>
__device__ __forceinline__ uint32_t locate(const Q4RowArgs& a, uint32_t first, uint32_t step, uint32_t items, Item (&it)[N]) {
    const Q4Dims& d = a.dims;
    uint32_t fault = 0;
    int count[N], len[N], from[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const uint32_t i = min(first + k * step, items - 1);
        const uint32_t slab = i / (uint32_t)a.rows, lb = slab / (uint32_t)d.hkv;
        it[k].r = (int)(i - slab * (uint32_t)a.rows);
        it[k].g = (int)(slab - lb * (uint32_t)d.hkv);
        it[k].l = (int)(lb / (uint32_t)d.batch);
        it[k].b = (int)(lb - (uint32_t)it[k].l * (uint32_t)d.batch);
        count[k] = a.count ? a.count[it[k].b] : a.rows;
        len[k] = a.cache.len[it[k].b];
        from[k] = a.first ? a.first[it[k].b] : 0;
        it[k].wanted = first + k * step < items;
    }
#pragma unroll
    for (int k = 0; k < N; ++k) {
        if (it[k].wanted && it[k].r == 0 && (uint32_t)count[k] > (uint32_t)a.rows) fault |= kFaultCache;
        it[k].wanted = it[k].wanted && it[k].r < count[k];
        const int64_t row = (a.first ? (int64_t)from[k] : (int64_t)len[k] - count[k]) + it[k].r;
        const bool in = row >= 0 && row < len[k] && row < d.cap;
        const int page = a.cache.table[(size_t)it[k].b * d.max_pages + (in ? (int)(row >> d.page_shift) : 0)];
        const bool ok = in && (uint32_t)page < (uint32_t)d.n_pages;
        it[k].page = ok ? page : -1;
        it[k].row = (int)row & (d.page_rows - 1);
        if (it[k].wanted && !ok) fault |= kFaultCache;
    }
    return fault;
}
__device__ __forceinline__ size_t source_of(const Item& it, const int64_t (&s)[4]) {
    return (size_t)(it.l * s[0] + it.b * s[1] + it.g * s[2] + it.r * s[3]);
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

// kItems: rows of keys and of values per lane, their loads together.  Two where that still leaves two workgroups for every CU,
// else one: one layer of 8 sequences of 8 KV heads x 5,000 .. 8,192 rows of bf16, stored and loaded, took 136 us with one, 124
// with two and 131 with four, a decode step's rows of 32 such layers 6.9 us with one and 7.9 with two.  The dense side passes the
// caches by (137 us for the former where nothing does); the pool's side does not, as what is stored is read next (107 us, 5.3
// TB/s of what has to move, a large copy 4.9; the 124 above are with the pool's reads past the caches as well).
template <typename T, int D, int kItems>
__global__ __launch_bounds__(kThreads) void q4_store_kernel(Q4RowArgs a, uint32_t items) {
    constexpr int kLanes = D / kElems, kRows = kThreads / kLanes;  // lanes per row, rows side by side
    const int p = threadIdx.x % kLanes;
    const uint32_t first = blockIdx.x * (kRows * kItems) + threadIdx.x / kLanes;
    if (first >= items) return;  // (whole rows of lanes)
    Item it[kItems];
    uint32_t fault = locate(a, first, kRows, items, it);
    int refs[kItems];
    float x[kItems][2][kElems];
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        refs[k] = it[k].page >= 0 ? a.cache.refs[it[k].page] : 1;
        if (!it[k].wanted) continue;
        read8<T, D>(static_cast<const T*>(a.k) + source_of(it[k], a.ks), p, x[k][0]);
        read8<T, D>(static_cast<const T*>(a.v) + source_of(it[k], a.vs), p, x[k][1]);
    }
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        if (it[k].wanted && refs[k] != 1) fault |= refs[k] > 1 ? kFaultSharedPage : kFaultCache;
        if (!it[k].wanted || it[k].page < 0 || refs[k] != 1) continue;
        uint8_t* rec = a.cache.pool + q4_record(a.dims, a.layer0 + it[k].l, it[k].page, it[k].g);
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            uint32_t scales;
            const uint32_t codes = quantise<T, D>(x[k][which], p, &scales);
            put_codes<T, D>(rec + (which ? a.dims.vc_off : 0) + it[k].row * (D / 2), p, codes);
            uint8_t* e = rec + (which ? a.dims.vs_off : a.dims.ks_off);
            if (p == 0) {
                if constexpr (D == 128) reinterpret_cast<uint32_t*>(e)[it[k].row] = scales;
                else reinterpret_cast<uint16_t*>(e)[it[k].row] = (uint16_t)scales;
            }
        }
    }
    if (fault && p == 0) atomicOr(a.faults, fault);
}

// 8 codes, the first and the last four of which may have different scales, as 8 bf16 (exact)
__device__ __forceinline__ u32x4 expand(uint32_t codes, uint32_t first, uint32_t last) {
    const float s0 = __uint_as_float(first << 23), s1 = __uint_as_float(last << 23);
    u32x4 r;
    r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s0, 0));
    r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s0, 1));
    r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s1, 2));
    r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s1, 3));
    return r;
}

template <typename T, int D, int kItems>
__global__ __launch_bounds__(kThreads) void q4_load_kernel(Q4RowArgs a, uint32_t items) {
    constexpr int kLanes = D / kElems, kRows = kThreads / kLanes;
    const int p = threadIdx.x % kLanes;
    const uint32_t first = blockIdx.x * (kRows * kItems) + threadIdx.x / kLanes;
    if (first >= items) return;
    Item it[kItems];
    const uint32_t fault = locate(a, first, kRows, items, it);
    if (fault && p == 0) atomicOr(a.faults, fault);
    constexpr bool kHalves = sizeof(T) == 4;  // the lane's elements lie in two blocks
    uint32_t codes[kItems][2], byte[kItems][2][2];
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        const uint8_t* rec = a.cache.pool + q4_record(a.dims, a.layer0 + it[k].l, max(it[k].page, 0), it[k].g);
        const int row = it[k].page < 0 ? 0 : it[k].row;
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            const uint8_t* e = rec + (which ? a.dims.vs_off : a.dims.ks_off) + row * (D / 32);
            codes[k][which] = get_codes<T, D>(rec + (which ? a.dims.vc_off : 0) + row * (D / 2), p);
            byte[k][which][0] = e[kHalves ? p / 8 : p / 4];
            byte[k][which][1] = kHalves ? e[D / 64 + p / 8] : byte[k][which][0];
        }
    }
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        if (!it[k].wanted) continue;
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            T* out = static_cast<T*>(which ? a.v_out : a.k_out) + source_of(it[k], which ? a.vs : a.ks);
            // (a row that is not there: zeros)
            const u32x4 x = it[k].page < 0 ? u32x4{0, 0, 0, 0} : expand(codes[k][which], byte[k][which][0], byte[k][which][1]);
            if constexpr (kHalves) {
                float f[kElems];
                Elem<bf16_t>::unpack(x, f);
                __builtin_nontemporal_store(f32x4{f[0], f[1], f[2], f[3]}, reinterpret_cast<f32x4*>(out) + p);
                __builtin_nontemporal_store(f32x4{f[4], f[5], f[6], f[7]}, reinterpret_cast<f32x4*>(out) + D / 8 + p);
            } else {
                __builtin_nontemporal_store(x, reinterpret_cast<u32x4*>(out) + p);
            }
        }
    }
}

template <typename T, int D, int kItems>
hipError_t launch_rows(const Q4RowArgs& a, uint32_t items, hipStream_t s) {
    constexpr uint32_t per = kThreads * kElems / D * kItems;
    const dim3 grid((items + per - 1) / per), block(kThreads);
    if (a.k_out) hipLaunchKernelGGL((q4_load_kernel<T, D, kItems>), grid, block, 0, s, a, items);
    else hipLaunchKernelGGL((q4_store_kernel<T, D, kItems>), grid, block, 0, s, a, items);
    return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_by_rows(const Q4RowArgs& a, hipStream_t s) {
    const uint32_t items = (uint32_t)a.layer_count * a.dims.batch * a.dims.hkv * a.rows;
    const int cus = device_cus() > 0 ? device_cus() : 256;
    return items >= (uint32_t)(2 * cus) * (kThreads * kElems / D * 2) ? launch_rows<T, D, 2>(a, items, s)
                                                                      : launch_rows<T, D, 1>(a, items, s);
}

hipError_t launch(const Q4RowArgs& a, hipStream_t s) {
    if (a.dims.bf16) return a.dims.d == 128 ? launch_by_rows<bf16_t, 128>(a, s) : launch_by_rows<bf16_t, 64>(a, s);
    return a.dims.d == 128 ? launch_by_rows<float, 128>(a, s) : launch_by_rows<float, 64>(a, s);
}

}  // namespace

hipError_t launch_q4_store(const Q4RowArgs& a, hipStream_t s) { return launch(a, s); }
hipError_t launch_q4_load(const Q4RowArgs& a, hipStream_t s) { return launch(a, s); }

}  // namespace ikv
