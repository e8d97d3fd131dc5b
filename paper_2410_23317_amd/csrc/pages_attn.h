// What the attention kernels over the pages share: parameters, device-scope access to partial results, the statistics.
#pragma once

#include <float.h>

#include "pages.h"

namespace vlc {

// Running maxima start at the lowest finite number: positions whose logits are all -inf then weigh nothing.
constexpr float kNoMax = -FLT_MAX;

struct PagesAttnParams {
    PagesParams p;
    RowsDev q, k_new, v_new, out;      // k_new.data null: nothing to write
    const float* sm_scale;
    vlc_row_stats stats;
    float* partials;
    int32_t* counters;
    int unit_shift;                    // log2 of the positions of a unit (the few-row kernel)
    int n_units;                       // units, or key splits, that a row of max_len positions has
    int part_floats;                   // floats of a unit's partial result
    int g_inverse;                     // 65536 / g, rounded up: x / g = x g_inverse / 65536 for small x
};

inline PagesAttnParams pages_attn_params(const PagesAttn& c) {
    PagesAttnParams a{};
    const int dtype = c.c.s.dtype;
    a.p = pages_params(c.c);
    a.q = rows_dev(c.q, dtype); a.k_new = rows_dev(c.k_new, dtype); a.v_new = rows_dev(c.v_new, dtype); a.out = rows_dev(c.out, dtype);
    a.sm_scale = c.sm_scale;
    a.stats = c.stats;
    a.partials = (float*)c.workspace;
    a.counters = c.c.dev.counters;
    a.g_inverse = 65536 / a.p.g + 1;
    return a;
}

__device__ __forceinline__ float attn_scale(const PagesAttnParams& a, int l, int d) {
    return a.sm_scale ? a.sm_scale[a.p.layer_begin + l] : rsqrtf((float)d);
}
// Statistics of query row i of query head h; m in the exponent (base 2) domain.
__device__ __forceinline__ void store_stats(const PagesAttnParams& a, int l, int b, int h, int i, float m, float z) {
    const int64_t at = l * a.stats.layer + b * a.stats.request + h * a.stats.head + i;
    a.stats.row_max[at] = z == 0.f ? -INFINITY : m * kLn2;
    a.stats.row_sum[at] = z;
}

// Partial results are written and read with device-scope accesses, which do not stop at an XCD's L2.
__device__ __forceinline__ void store_agent2(float* p, float a, float b) {
    const unsigned long long v = ((unsigned long long)__float_as_uint(b) << 32) | __float_as_uint(a);
    __hip_atomic_store(reinterpret_cast<unsigned long long*>(p), v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// (loads through a buffer resource, with the cache-policy bit that a device-scope atomic load sets: 16 bytes at a time)
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
constexpr int kDeviceScope = 16;
__device__ __forceinline__ __amdgpu_buffer_rsrc_t partials_buffer(const float* base, int bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(base), 0, bytes, 0x00020000);
}
__device__ __forceinline__ f32x4_t buffer_load16_agent(__amdgpu_buffer_rsrc_t b, int off) {
    return __builtin_bit_cast(f32x4_t, (u32x4_t)__builtin_amdgcn_raw_buffer_load_b128(b, off, 0, kDeviceScope));
}
__device__ __forceinline__ float2 buffer_load8_agent(__amdgpu_buffer_rsrc_t b, int off) {
    return __builtin_bit_cast(float2, (u32x2_t)__builtin_amdgcn_raw_buffer_load_b64(b, off, 0, kDeviceScope));
}

// two neighbouring outputs as one store
__device__ __forceinline__ void store_pair(float* p, float a, float b) { *reinterpret_cast<float2*>(p) = make_float2(a, b); }
__device__ __forceinline__ void store_pair(bf16_t* p, float a, float b) {
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
    *reinterpret_cast<bf16x2_t*>(p) = bf16x2_t{(__bf16)a, (__bf16)b};
}

// two bf16 numbers of a word, with those that are no finite numbers replaced by 0
__device__ __forceinline__ uint32_t finite_pair(uint32_t w) {
    const uint32_t lo = (w & 0x7f80u) == 0x7f80u ? 0u : w & 0xffffu;
    const uint32_t hi = (w & 0x7f800000u) == 0x7f800000u ? 0u : w & 0xffff0000u;
    return lo | hi;
}
__device__ __forceinline__ bool is_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

}  // namespace vlc
