// Device-side view of the paged prompt cache: lengths, the page table and the rows of a page.
#pragma once

#include "common.h"
#include "internal.h"

namespace vlc {

// How a page holds a row, as a template parameter: the storage type itself, or codes with one fp32 scale per row.
enum PageFormat { kPageBf16, kPageF32, kPageFp8, kPageInt8 };
template <int FMT> struct PageRow;
template <> struct PageRow<kPageBf16> { typedef bf16_t T; static constexpr int kElemBytes = 2; static constexpr bool kQuantised = false; };
template <> struct PageRow<kPageF32> { typedef float T; static constexpr int kElemBytes = 4; static constexpr bool kQuantised = false; };
template <> struct PageRow<kPageFp8> { typedef bf16_t T; static constexpr int kElemBytes = 1; static constexpr bool kQuantised = true; };
template <> struct PageRow<kPageInt8> { typedef bf16_t T; static constexpr int kElemBytes = 1; static constexpr bool kQuantised = true; };

inline PageFormat page_format(const vlc_pages_shape& s) {
    if (s.format == VLC_PAGES_FP8) return kPageFp8;
    if (s.format == VLC_PAGES_INT8) return kPageInt8;
    return s.dtype == VLC_F32 ? kPageF32 : kPageBf16;
}

// Strides of a tensor's rows in bytes.
struct RowsDev {
    char* data;
    int64_t layer, request, head, row;
    __device__ __forceinline__ char* at(int l, int b, int h, int i) const {
        return data + l * layer + b * request + h * head + i * row;
    }
};
inline RowsDev rows_dev(const vlc_rows& r, int dtype) {
    const int64_t es = dtype == VLC_F32 ? 4 : 2;
    return RowsDev{(char*)r.data, r.layer * es, r.request * es, r.head * es, r.row * es};
}

struct PagesParams {
    char* k;
    char* v;
    float* k_scale;
    float* v_scale;
    int32_t* status;
    const int32_t* table;
    const int32_t* lens;
    int B, max_pages, max_new, max_len;
    int Hq, Hkv, g, n_pages, ps_shift;
    int layer_begin, n_layers;
};
inline PagesParams pages_params(const PagesCall& c) {
    PagesParams p;
    p.k = c.dev.k; p.v = c.dev.v; p.k_scale = c.dev.k_scale; p.v_scale = c.dev.v_scale; p.status = c.dev.status;
    p.table = c.chunk.table; p.lens = c.chunk.lens;
    p.B = c.chunk.B; p.max_pages = c.chunk.max_pages; p.max_new = c.chunk.max_new; p.max_len = c.chunk.max_len;
    p.Hq = c.s.Hq; p.Hkv = c.s.Hkv; p.g = c.s.Hq / c.s.Hkv; p.n_pages = c.s.n_pages; p.ps_shift = __builtin_ctz(c.s.page_slots);
    p.layer_begin = c.layer_begin; p.n_layers = c.n_layers;
    return p;
}

// Tokens of request b with the chunk (n) and in it (c); a request whose pair breaks the call's bounds counts as empty.  Reading takes
// no chunk: held_len looks at n alone.
struct ChunkLen {
    int n, c;
    bool ok;
};
__device__ __forceinline__ ChunkLen held_len(const PagesParams& p, int b) {
    ChunkLen r{p.max_len, 0, true};
    if (p.lens) {
        r.n = p.lens[2 * b];
        r.ok = r.n >= 0 && r.n <= p.max_len;
        if (!r.ok) r.n = 0;
    }
    return r;
}
__device__ __forceinline__ ChunkLen chunk_len(const PagesParams& p, int b) {
    ChunkLen r{p.max_len, p.max_new, true};
    if (p.lens) {
        r.n = p.lens[2 * b];
        r.c = p.lens[2 * b + 1];
        r.ok = r.c >= 0 && r.c <= p.max_new && r.n >= r.c && r.n <= p.max_len;
        if (!r.ok) r.n = r.c = 0;
    }
    return r;
}
constexpr int kStickyPage = -1, kStickyLens = -2;
__device__ __forceinline__ void report_lens(const PagesParams& p, int b) {
    set_sticky(p.status, VLC_ERR_INVALID_ARG, b, kStickyLens, p.lens[2 * b]);
}

// First row (of page_slots) of a page's KV head in its layer's order; multiply by the row's bytes, or index the scales.
__device__ __forceinline__ int64_t page_row0(const PagesParams& p, int l, int page, int hkv) {
    return ((((int64_t)l * p.n_pages + page) * p.Hkv) + hkv) << p.ps_shift;
}

// ---- rows of codes -------------------------------------------------------------------------------------
// absmax of a row whose LPR consecutive lanes hold 8 bf16 values each, as the bits of its absolute value: NaN > inf > finite.
template <int LPR>
__device__ __forceinline__ uint32_t row_absmax_bits(const uint4& v) {
    float f[8];
    unpack16(v, f, (const bf16_t*)nullptr);
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(f[e]) & 0x7fffffffu);
#pragma unroll
    for (int o = LPR / 2; o >= 1; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o, kWave));
    return m;
}
// 8 codes and the row's scale; a row with a NaN or an infinity has codes of 0 and a scale of NaN.  (Finite rows of FP8 pages are the
// codes and scales of quantize_row_e4m3, which the compressed cache has and which drops a NaN from the maximum: rows here are read
// back, so such a row has to stay one.)
template <int FMT, int LPR>
__device__ __forceinline__ uint2 quantize_page_row(const uint4& v, float& scale) {
    constexpr float kTop = FMT == kPageFp8 ? 448.0f : 127.0f;
    const uint32_t bits = row_absmax_bits<LPR>(v);
    if (bits >= 0x7f800000u) {
        scale = __uint_as_float(0x7fc00000u);
        return make_uint2(0, 0);
    }
    const float amax = __uint_as_float(bits);
    scale = bits ? amax / kTop : 1.0f;
    float f[8], y[8];
    unpack16(v, f, (const bf16_t*)nullptr);
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = fminf(fmaxf(f[e] / scale, -kTop), kTop);
    if constexpr (FMT == kPageFp8) {
        int lo = 0, hi = 0;
        lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], lo, false);
        lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
        hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], hi, false);
        hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], hi, true);
        return make_uint2((uint32_t)lo, (uint32_t)hi);
    } else {
        uint32_t w[2] = {0, 0};
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e >> 2] |= ((uint32_t)(int)__builtin_rintf(y[e]) & 0xffu) << (8 * (e & 3));
        return make_uint2(w[0], w[1]);
    }
}
// 8 codes as fp32 numbers.
template <int FMT>
__device__ __forceinline__ void codes_to_f32(const uint2& c, float (&f)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t w = e < 4 ? c.x : c.y;
        if constexpr (FMT == kPageInt8) f[e] = (float)(int)(int8_t)(w >> (8 * (e & 3)));
    }
    if constexpr (FMT == kPageFp8) {
        const uint4 b = e4m3x8_to_bf16x8(c);
        unpack16(b, f, (const bf16_t*)nullptr);
    }
}
// 8 codes as bf16 numbers, exactly: E4M3 has 4 significant bits, a signed byte 8.
template <int FMT>
__device__ __forceinline__ uint4 codes_to_bf16(const uint2& c) {
    if constexpr (FMT == kPageFp8) return e4m3x8_to_bf16x8(c);
    float f[8];
    codes_to_f32<FMT>(c, f);
    // the fp32 numbers are integers of at most 8 bits: their upper halves are the bf16 numbers
    auto two = [&](int e) { return __builtin_amdgcn_perm(__float_as_uint(f[e + 1]), __float_as_uint(f[e]), 0x07060302u); };
    return make_uint4(two(0), two(2), two(4), two(6));
}

}  // namespace vlc
