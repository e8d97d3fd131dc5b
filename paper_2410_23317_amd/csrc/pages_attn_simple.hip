// Attention of a chunk over the pages of its request: the plain version, one wave per query row, any format.
//
// Keys are taken 64 at a time: a lane computes the logit of one key, the wave the running maximum and sum, and then every
// lane its elements of the output from the tile's V rows, which the whole wave reads one after the other.
#include <float.h>

#include "pages.h"

namespace vlc {
namespace {

struct SimpleArgs {
    PagesParams p;
    RowsDev q, out;
    const float* sm_scale;
    vlc_row_stats stats;
};

template <int FMT>
__device__ __forceinline__ float page_elem(const char* base, int64_t at) {
    if constexpr (FMT == kPageBf16) return Elem<bf16_t>::load((const bf16_t*)base + at);
    if constexpr (FMT == kPageF32) return ((const float*)base)[at];
    if constexpr (FMT == kPageInt8) return (float)((const int8_t*)base)[at];
    if constexpr (FMT == kPageFp8) {
        float f[8];
        codes_to_f32<FMT>(make_uint2(((const uint8_t*)base)[at], 0), f);
        return f[0];
    }
}

template <int FMT, int D>
__global__ __launch_bounds__(64) void pages_attn_simple_kernel(SimpleArgs a) {
    typedef PageRow<FMT> R;
    typedef typename R::T T;
    constexpr int EPL = D / 64;
    __shared__ float sQ[D], sP[64];
    __shared__ int64_t sRow[64];
    const int lane = threadIdx.x, i = blockIdx.x, h = blockIdx.y, lb = blockIdx.z, l = lb / a.p.B, b = lb % a.p.B;
    const ChunkLen len = chunk_len(a.p, b);
    if (!len.ok && l == 0 && h == 0 && i == 0 && lane == 0) report_lens(a.p, b);
    if (i >= len.c) return;
    const float scale = a.sm_scale ? a.sm_scale[a.p.layer_begin + l] : rsqrtf((float)D);
    const T* q = (const T*)a.q.at(l, b, h, i);
    for (int e = lane; e < D; e += 64) sQ[e] = Elem<T>::load(q + e);
    __syncthreads();
    const int last = len.n - len.c + i;
    float m = -FLT_MAX, z = 0.f, acc[EPL] = {};
    for (int j0 = 0; j0 <= last; j0 += 64) {
        const int j = j0 + lane;
        const bool seen = j <= last;
        int64_t row = 0;
        float s = -INFINITY, vs = 1.f;
        if (seen) {
            int page = a.p.table[(int64_t)b * a.p.max_pages + (j >> a.p.ps_shift)];
            if ((uint32_t)page >= (uint32_t)a.p.n_pages) {
                set_sticky(a.p.status, VLC_ERR_INVALID_ARG, b, kStickyPage, page);
                page = 0;
            }
            row = page_row0(a.p, a.p.layer_begin + l, page, h / a.p.g) + (j & ((1 << a.p.ps_shift) - 1));
            float dot = 0.f;
            for (int e = 0; e < D; ++e) dot = fmaf(sQ[e], page_elem<FMT>(a.p.k, row * D + e), dot);
            if constexpr (R::kQuantised) { dot *= a.p.k_scale[row]; vs = a.p.v_scale[row]; }
            s = dot * scale;
        }
        sRow[lane] = row;
        const float m_new = fmaxf(m, wave_allreduce_max(s));
        const float w = seen ? exp2_fast((s - m_new) * kLog2e) : 0.f, corr = exp2_fast((m - m_new) * kLog2e);
        z = z * corr + wave_allreduce_sum(w);
        m = m_new;
        sP[lane] = seen ? w * vs : 0.f;
        __syncthreads();
        for (int e = 0; e < EPL; ++e) acc[e] *= corr;
        for (int t = 0; t < 64 && j0 + t <= last; ++t)
            for (int e = 0; e < EPL; ++e) acc[e] = fmaf(sP[t], page_elem<FMT>(a.p.v, sRow[t] * D + lane * EPL + e), acc[e]);
        __syncthreads();
    }
    T* out = (T*)a.out.at(l, b, h, i) + lane * EPL;
    for (int e = 0; e < EPL; ++e) Elem<T>::store(out + e, z == 0.f ? 0.f : acc[e] / z);
    if (a.stats.row_max && lane == 0) {
        const int64_t at = l * a.stats.layer + b * a.stats.request + h * a.stats.head + i;
        a.stats.row_max[at] = z == 0.f ? -INFINITY : m;
        a.stats.row_sum[at] = z;
    }
}

}  // namespace

hipError_t launch_pages_attn_simple(const PagesAttn& c) {
    SimpleArgs a;
    a.p = pages_params(c.c);
    a.q = rows_dev(c.q, c.c.s.dtype);
    a.out = rows_dev(c.out, c.c.s.dtype);
    a.sm_scale = c.sm_scale;
    a.stats = c.stats;
    const dim3 grid(a.p.max_new, a.p.Hq, a.p.n_layers * a.p.B);
    const bool wide = c.c.s.d == 128;
#define LAUNCH(F) (wide ? pages_attn_simple_kernel<F, 128><<<grid, 64, 0, c.c.stream>>>(a) : pages_attn_simple_kernel<F, 64><<<grid, 64, 0, c.c.stream>>>(a))
    switch (page_format(c.c.s)) {
        case kPageBf16: LAUNCH(kPageBf16); break;
        case kPageF32: LAUNCH(kPageF32); break;
        case kPageFp8: LAUNCH(kPageFp8); break;
        case kPageInt8: LAUNCH(kPageInt8); break;
    }
#undef LAUNCH
    return hipGetLastError();
}

}  // namespace vlc
