// What the two kernels over many query rows (bf16 and fp32 storage) share: the partial results of the key splits.
#pragma once

#include "pages_attn.h"

namespace vlc {

struct PagesRowsParams {
    PagesAttnParams a;                 // a.n_units: key splits
    int row_blocks, groups;            // of a KV head's rows; layers * requests * KV heads
    int steps_per_split;               // key stages (bf16) or tiles (fp32)
    float* part_o;                     // [group][split][rows][D] unnormalised
    float4* part_mz;                   // [group][split][rows] running maximum (base 2), sum that the outputs are divided by, plain sum
};

// Bytes of the partial outputs of n rows, behind which their maxima and sums start.
inline size_t pages_partials_o_bytes(size_t n, int d) { return (n * d * sizeof(float) + 255) / 256 * 256; }

// Merge of the key splits: D / 4 lanes per row, the loads of NB splits in flight together.  A split beyond what the row's block
// saw has left kNoMax and 0.
template <typename T, int D>
__global__ __launch_bounds__(256) void pages_rows_merge_kernel(PagesRowsParams ra) {
    const PagesAttnParams& a = ra.a;
    constexpr int LPR = D / 4, NB = 8;
    const int sub = threadIdx.x % LPR;
    const int group = blockIdx.y, h = group % a.p.Hkv, lb = group / a.p.Hkv, b = lb % a.p.B, l = lb / a.p.B;
    const int r = blockIdx.x * (256 / LPR) + threadIdx.x / LPR, g = a.p.g;
    if (r >= g * chunk_len(a.p, b).c) return;
    const int64_t stride = (int64_t)g * a.p.max_new, p0 = (int64_t)group * a.n_units * stride + r;
    float m = kNoMax, z = 0.f, zs = 0.f;
    f32x4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (int s0 = 0; s0 < a.n_units; s0 += NB) {
        float4 mz[NB];
        f32x4_t f[NB];
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const int64_t at = p0 + min(s0 + j, a.n_units - 1) * stride;
            mz[j] = ra.part_mz[at];
            f[j] = *reinterpret_cast<const f32x4_t*>(ra.part_o + at * D + sub * 4);
        }
        float mn = m;
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            if (s0 + j >= a.n_units) { mz[j] = make_float4(kNoMax, 0.f, 0.f, 0.f); f[j] = f32x4_t{0.f, 0.f, 0.f, 0.f}; }
            mn = fmaxf(mn, mz[j].x);
        }
        const float w0 = exp2_fast(m - mn);
        o *= w0; z *= w0; zs *= w0;
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const float wgt = exp2_fast(mz[j].x - mn);
            o += f[j] * wgt;
            z = fmaf(mz[j].y, wgt, z);
            zs = fmaf(mz[j].z, wgt, zs);
        }
        m = mn;
    }
    const float div = z == 0.f ? 1.f : z;                      // a row without weights: its sums are 0
    T* out = (T*)a.out.at(l, b, h * g + r % g, r / g) + sub * 4;
    store_pair(out, o[0] / div, o[1] / div);
    store_pair(out + 2, o[2] / div, o[3] / div);
    if (sub == 0 && a.stats.row_max) store_stats(a, l, b, h * g + r % g, r / g, m, zs);
}

template <typename T, int D>
inline void launch_pages_rows_merge(const PagesRowsParams& ra, hipStream_t st) {
    constexpr int per = 256 / (D / 4);
    pages_rows_merge_kernel<T, D><<<dim3((ra.a.p.g * ra.a.p.max_new + per - 1) / per, ra.groups), 256, 0, st>>>(ra);
}

}  // namespace vlc
