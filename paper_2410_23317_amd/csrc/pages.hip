// Rows into and out of the pages of the prompt cache (gfx950): a chunk's K and V are written, quantised on the way if the
// pages hold codes, and read back as the storage type.
//
// Both kernels move rows: a row of K and the same row of V per group of lanes, 16 bytes of the storage type a lane, so that a
// row's absolute maximum is a reduction inside 8 or 16 lanes and every access is a whole piece of 16 bytes (8 of codes).
// Plain rows are bound by memory: 32768 new tokens of one layer, 268 MB read and written, 52.5 us (fp32: twice the bytes, 102), 5.1 TB/s,
// what a large copy reaches; 2944 tokens of 32 layers read back in 133 us, 5.8 TB/s, from FP8 pages in 100.  A small call is a launch:
// 2000 new tokens of one layer 4.3 us, 2.4 of them the launch's.
// The quantising writer is bound by the vector unit: a full fp32 division for each of a lane's 16 numbers.  32 layers of 10368 tokens into
// FP8 pages take 497 us, in which the SIMDs issue vector instructions all the time (413 a wave; the reader has 152 and takes 342 us, half
// of its cycles): 4.1 TB/s of what is read and written; 64-wide rows into int8 pages 24 us for what the reader moves back in 13.
// Neighbouring groups of lanes take neighbouring rows of the caller's tensor (head_inner).
#include "pages.h"

namespace vlc {
namespace {

__global__ void pages_clear_kernel(int32_t* status, int32_t* counters) {
    const int x = blockIdx.x * blockDim.x + threadIdx.x;
    if (x < 4) status[x] = 0;
    if (x < kMaxPagesRows) counters[x] = 0;
}

struct MoveArgs {
    PagesParams p;
    RowsDev k, v;
    int first, count;          // read: positions [first, first + count)
    int head_inner;            // neighbouring row groups take neighbouring heads (tokens outermost in memory), else neighbouring tokens
};

template <int FMT, int D>
__global__ __launch_bounds__(256) void pages_write_kernel(MoveArgs a) {
    typedef PageRow<FMT> R;
    typedef typename R::T T;
    constexpr int LPR = D * (int)sizeof(T) / 16;               // lanes per row
    const int lb = blockIdx.y, l = lb / a.p.B, b = lb % a.p.B;
    const ChunkLen len = chunk_len(a.p, b);
    const int sub = threadIdx.x % LPR;
    if (!len.ok && l == 0 && blockIdx.x == 0 && threadIdx.x == 0) report_lens(a.p, b);
    const int x = blockIdx.x * (256 / LPR) + threadIdx.x / LPR;
    const int i = a.head_inner ? x / a.p.Hkv : x % a.p.max_new, h = a.head_inner ? x % a.p.Hkv : x / a.p.max_new;
    if (i >= len.c || h >= a.p.Hkv) return;
    const int pos = len.n - len.c + i;
    const int page = a.p.table[(int64_t)b * a.p.max_pages + (pos >> a.p.ps_shift)];
    if ((uint32_t)page >= (uint32_t)a.p.n_pages) {
        if (sub == 0) set_sticky(a.p.status, VLC_ERR_INVALID_ARG, b, kStickyPage, page);
        return;
    }
    const uint4 kx = reinterpret_cast<const uint4*>(a.k.at(l, b, h, i))[sub], vx = reinterpret_cast<const uint4*>(a.v.at(l, b, h, i))[sub];
    const int64_t row = page_row0(a.p, a.p.layer_begin + l, page, h) + (pos & ((1 << a.p.ps_shift) - 1));
    if constexpr (!R::kQuantised) {
        reinterpret_cast<uint4*>(a.p.k)[row * LPR + sub] = kx;
        reinterpret_cast<uint4*>(a.p.v)[row * LPR + sub] = vx;
    } else {
        float ks, vs;
        const uint2 kc = quantize_page_row<FMT, LPR>(kx, ks), vc = quantize_page_row<FMT, LPR>(vx, vs);
        reinterpret_cast<uint2*>(a.p.k)[row * LPR + sub] = kc;
        reinterpret_cast<uint2*>(a.p.v)[row * LPR + sub] = vc;
        if (sub == 0) { a.p.k_scale[row] = ks; a.p.v_scale[row] = vs; }
    }
}

template <int FMT, int D>
__global__ __launch_bounds__(256) void pages_read_kernel(MoveArgs a) {
    typedef PageRow<FMT> R;
    typedef typename R::T T;
    constexpr int LPR = D * (int)sizeof(T) / 16;
    const int lb = blockIdx.y, l = lb / a.p.B, b = lb % a.p.B;
    const ChunkLen len = held_len(a.p, b);
    const int sub = threadIdx.x % LPR;
    if (!len.ok && l == 0 && blockIdx.x == 0 && threadIdx.x == 0) report_lens(a.p, b);
    const int x = blockIdx.x * (256 / LPR) + threadIdx.x / LPR;
    const int i = a.head_inner ? x / a.p.Hkv : x % a.count, h = a.head_inner ? x % a.p.Hkv : x / a.count;
    if (i >= a.count || i >= len.n - a.first || h >= a.p.Hkv) return;
    const int pos = a.first + i;
    int page = a.p.table[(int64_t)b * a.p.max_pages + (pos >> a.p.ps_shift)];
    if ((uint32_t)page >= (uint32_t)a.p.n_pages) {
        if (sub == 0) set_sticky(a.p.status, VLC_ERR_INVALID_ARG, b, kStickyPage, page);
        page = 0;
    }
    const int64_t row = page_row0(a.p, a.p.layer_begin + l, page, h) + (pos & ((1 << a.p.ps_shift) - 1));
    uint4* ko = reinterpret_cast<uint4*>(a.k.at(l, b, h, i)) + sub;
    uint4* vo = reinterpret_cast<uint4*>(a.v.at(l, b, h, i)) + sub;
    if constexpr (!R::kQuantised) {
        *ko = reinterpret_cast<const uint4*>(a.p.k)[row * LPR + sub];
        *vo = reinterpret_cast<const uint4*>(a.p.v)[row * LPR + sub];
    } else {
        const uint2 kc = reinterpret_cast<const uint2*>(a.p.k)[row * LPR + sub], vc = reinterpret_cast<const uint2*>(a.p.v)[row * LPR + sub];
        const float ks = a.p.k_scale[row], vs = a.p.v_scale[row];
        auto values = [](const uint2& c, float s) {
            float f[8];
            codes_to_f32<FMT>(c, f);
            bf16x8_t o;
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = (__bf16)(f[e] * s);
            return __builtin_bit_cast(uint4, o);
        };
        *ko = values(kc, ks);
        *vo = values(vc, vs);
    }
}

template <int FMT, int D>
void launch_move(bool write, const MoveArgs& a, hipStream_t st) {
    constexpr int rows = 256 / (D * (int)sizeof(typename PageRow<FMT>::T) / 16);
    const int64_t n = (int64_t)(write ? a.p.max_new : a.count) * a.p.Hkv;
    const dim3 grid((unsigned)((n + rows - 1) / rows), a.p.n_layers * a.p.B);
    if (write) pages_write_kernel<FMT, D><<<grid, 256, 0, st>>>(a);
    else pages_read_kernel<FMT, D><<<grid, 256, 0, st>>>(a);
}

hipError_t launch_move(bool write, const PagesCall& c, MoveArgs& a, const vlc_rows& k, const vlc_rows& v) {
    a.p = pages_params(c);
    a.k = rows_dev(k, c.s.dtype);
    a.v = rows_dev(v, c.s.dtype);
    a.head_inner = k.head < k.row;
    const bool wide = c.s.d == 128;
    switch (page_format(c.s)) {
        case kPageBf16: wide ? launch_move<kPageBf16, 128>(write, a, c.stream) : launch_move<kPageBf16, 64>(write, a, c.stream); break;
        case kPageF32: wide ? launch_move<kPageF32, 128>(write, a, c.stream) : launch_move<kPageF32, 64>(write, a, c.stream); break;
        case kPageFp8: wide ? launch_move<kPageFp8, 128>(write, a, c.stream) : launch_move<kPageFp8, 64>(write, a, c.stream); break;
        case kPageInt8: wide ? launch_move<kPageInt8, 128>(write, a, c.stream) : launch_move<kPageInt8, 64>(write, a, c.stream); break;
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_pages_clear(const PagesDev& dev, hipStream_t st) {
    pages_clear_kernel<<<kMaxPagesRows / 256, 256, 0, st>>>(dev.status, dev.counters);
    return hipGetLastError();
}

hipError_t launch_pages_write(const PagesCall& c, const vlc_rows& k_new, const vlc_rows& v_new) {
    MoveArgs a{};
    return launch_move(true, c, a, k_new, v_new);
}

hipError_t launch_pages_read(const PagesCall& c, int first, int count, const vlc_rows& k_out, const vlc_rows& v_out) {
    MoveArgs a{};
    a.first = first;
    a.count = count;
    return launch_move(false, c, a, k_out, v_out);
}

}  // namespace vlc
