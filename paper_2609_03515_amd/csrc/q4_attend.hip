// Decode attention over the paged 4-bit cache, with the eviction score (Eq. 1) and its fold (Eq. 4).
//
// z_h(i) = q_h . k_i / sqrt(d) (+ bias on recent positions), a_h = softmax over the rows i < len, o_h = sum_i a_h(i) v_i;
// s(i) = (1 / H) sum_h a_h(i), u <- alpha u + (1 - alpha) s layer by layer.  Base-2 logits throughout.
#include "kv_common.h"
#include "q4.h"

namespace ikv {
namespace {

constexpr int kThreads = 256;

// Rows of sequence b that a call attends to: its length, or none of it where that is out of range.
__device__ __forceinline__ int attended(const Q4AttendArgs& a, int b) {
    const int n = a.cache.len[b];
    return n < 0 || n > a.n_max ? 0 : n;
}

__device__ __forceinline__ float value(uint32_t codes, int i, float scale) {  // element i of 8
    const uint32_t pair = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes >> 8 * (i / 2), scale, 0));
    return __uint_as_float(i % 2 ? pair & 0xffff0000u : pair << 16);
}

template <typename T>
__device__ __forceinline__ float element(const void* p, size_t i) {
    if constexpr (sizeof(T) == 2) return __uint_as_float((uint32_t) static_cast<const uint16_t*>(p)[i] << 16);
    else return static_cast<const float*>(p)[i];
}

// One row per thread.
template <typename T>
__global__ __launch_bounds__(kThreads) void q4_logits_kernel(Q4AttendArgs a) {
    const Q4Dims& d = a.dims;
    const int blocks = (a.n_max + kThreads - 1) / kThreads;
    const int slab = blockIdx.x / blocks, row = blockIdx.x % blocks * kThreads + threadIdx.x;
    const int lb = slab / d.hkv, g = slab % d.hkv, b = lb % d.batch, layer = lb / d.batch;
    const int len = a.cache.len[b];
    if (threadIdx.x == 0 && row == 0 && (len < 0 || len > a.n_max)) atomicOr(a.faults, kFaultCache);
    if (row >= attended(a, b)) return;
    const int page = a.cache.table[(size_t)b * d.max_pages + (row >> d.page_shift)];
    const bool ok = (uint32_t)page < (uint32_t)d.n_pages;
    if (!ok) atomicOr(a.faults, kFaultCache);
    const uint8_t* rec = a.cache.pool + q4_record(d, a.layer0 + layer, ok ? page : 0, g);
    const int in = row & (d.page_rows - 1);
    const bool recent = a.bias != 0.0f && a.cache.pos[(size_t)b * d.cap + row] >= a.cur_pos[b] - (a.window - 1);
    for (int h = 0; h < d.group; ++h) {
        float z = 0.0f;
        const size_t q0 = ((size_t)lb * d.hq + g * d.group + h) * d.d;
        for (int c = 0; c < d.d / 8; ++c) {
            const uint32_t codes = reinterpret_cast<const uint32_t*>(rec + in * (d.d / 2))[c];
            const float scale = __uint_as_float((uint32_t)rec[d.ks_off + in * (d.d / 32) + c / 4] << 23);
            for (int i = 0; i < 8; ++i) z = fmaf(element<T>(a.q, q0 + c * 8 + i), value(codes, i, scale), z);
        }
        z = z * a.scale2 + (recent ? a.bias2 : 0.0f);
        a.z[((size_t)slab * d.group + h) * a.n_stride + row] = ok ? z : -INFINITY;
    }
}

// One (slab, head) per workgroup, one dimension per thread.
template <typename T>
__global__ __launch_bounds__(kThreads) void q4_output_kernel(Q4AttendArgs a) {
    __shared__ float red[kThreads];
    const Q4Dims& d = a.dims;
    const int slab = blockIdx.x / d.group, h = blockIdx.x % d.group;
    const int lb = slab / d.hkv, g = slab % d.hkv, b = lb % d.batch, layer = lb / d.batch;
    const int n = attended(a, b);
    const float* z = a.z + ((size_t)slab * d.group + h) * a.n_stride;
    float m = -INFINITY;
    for (int i = threadIdx.x; i < n; i += kThreads) m = fmaxf(m, z[i]);
    red[threadIdx.x] = m;
    __syncthreads();
    for (int i = 0; i < kThreads; ++i) m = fmaxf(m, red[i]);
    __syncthreads();
    if (m == -INFINITY) m = 0.0f;
    float l = 0.0f;
    for (int i = threadIdx.x; i < n; i += kThreads) l += exp2f(z[i] - m);
    red[threadIdx.x] = l;
    __syncthreads();
    l = 0.0f;
    for (int i = 0; i < kThreads; ++i) l += red[i];
    if (threadIdx.x == 0) a.part[(size_t)slab * d.group + h] = make_float2(m, l);
    const int x = threadIdx.x;
    if (x >= d.d) return;
    float o = 0.0f;
    for (int row = 0; row < n; ++row) {
        const float p = exp2f(z[row] - m);
        const int page = a.cache.table[(size_t)b * d.max_pages + (row >> d.page_shift)];
        if ((uint32_t)page >= (uint32_t)d.n_pages) continue;
        const uint8_t* rec = a.cache.pool + q4_record(d, a.layer0 + layer, page, g);
        const int in = row & (d.page_rows - 1);
        const uint32_t codes = reinterpret_cast<const uint32_t*>(rec + d.vc_off + in * (d.d / 2))[x / 8];
        const float scale = __uint_as_float((uint32_t)rec[d.vs_off + in * (d.d / 32) + x / 32] << 23);
        o = fmaf(p, value(codes, x % 8, scale), o);
    }
    T* out = static_cast<T*>(a.o) + ((size_t)lb * d.hq + g * d.group + h) * d.d + x;
    Elem<T>::store(out, l != 0.0f ? o / l : 0.0f);
}

__global__ __launch_bounds__(kThreads) void q4_score_kernel(Q4AttendArgs a) {
    const Q4Dims& d = a.dims;
    const int blocks = (a.n_max + kThreads - 1) / kThreads;
    const int b = blockIdx.x / blocks, row = blockIdx.x % blocks * kThreads + threadIdx.x;
    if (row >= a.n_max) return;
    const bool live = row < attended(a, b);
    float u = live && a.u_out ? a.u_prior[(size_t)b * d.cap + row] : 0.0f;
    for (int l = 0; l < a.layer_count; ++l) {
        float s = 0.0f;
        if (live)
            for (int h = 0; h < d.hq; ++h) {
                const size_t sh = (size_t)(l * d.batch + b) * d.hq + h;
                const float2 p = a.part[sh];
                s += p.y != 0.0f ? exp2f(a.z[sh * a.n_stride + row] - p.x) / p.y : 0.0f;
            }
        s /= (float)d.hq;
        if (a.s_out) a.s_out[((size_t)l * d.batch + b) * a.n_max + row] = s;
        u = a.alpha * u + (1.0f - a.alpha) * s;
    }
    if (live && a.u_out) a.u_out[(size_t)b * d.cap + row] = u;
}

}  // namespace

void q4_attend_plan(int, int n, int* nchunk, int* chunk_rows) {
    *nchunk = 1;
    *chunk_rows = n;
}

hipError_t launch_q4_attend(const Q4AttendArgs& a, hipStream_t s) {
    const int slabs = a.layer_count * a.dims.batch * a.dims.hkv;
    const int blocks = (a.n_max + kThreads - 1) / kThreads;
    hipLaunchKernelGGL((a.dims.bf16 ? q4_logits_kernel<bf16_t> : q4_logits_kernel<float>), dim3(slabs * blocks), dim3(kThreads), 0, s, a);
    hipLaunchKernelGGL((a.dims.bf16 ? q4_output_kernel<bf16_t> : q4_output_kernel<float>), dim3(slabs * a.dims.group), dim3(kThreads), 0, s, a);
    if (a.s_out || a.u_out) hipLaunchKernelGGL(q4_score_kernel, dim3(a.dims.batch * blocks), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace ikv
