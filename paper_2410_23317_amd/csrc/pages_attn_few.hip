// Attention of a few new tokens over the pages of their request (gfx950): up to 32 query rows per KV head (the g heads
// of up to 32 / g tokens), which is decoding, and verifying drafted tokens.
//
// Bound by memory: every K and V row is read once and serves all query rows of its KV head.  A (layer, request, KV head) row
// of the cache is cut into units of 2^unit_shift positions, a block of four waves each; the tiles of a unit are dealt
// to the waves, which merge through LDS.  Units of a row leave unnormalised partial results with device-scope stores and
// count themselves; the one that counts last merges them and writes the output (its own stores are acknowledged before it
// counts, so whoever counts last finds all of them in memory).
//
// A tile's operands come from memory in the order the matrix instructions want, without a trip through LDS or across
// lanes.  bf16 (codes are expanded to bf16, exactly, where they are used; K's scale multiplies the finished logit, V's the
// probability before it is rounded to bf16): 32 positions, 8 G + j for lane group G = lane / 16, place j.  Logits
// S^T[position][column] = K Q^T, a column being a query row; a lane fetches the K pieces of the position whose logit comes
// out for its own group, holds 8 logits of one column, and their probabilities are the second product's operand as they
// are; V's operand is a transpose inside the lane (one v_perm_b32 per register) of the rows it fetched.
// fp32 (v_mfma_f32_16x16x4_f32, full fp32 products): 16 positions; a lane's 16 bytes of K hold four contraction indexes of
// its group, its 4 logits are four operands of the second product, and 16 bytes of V four of its output tiles: no permutes.
#include "pages_attn.h"

namespace vlc {
namespace {

constexpr int kWaves = 4, kThreads = kWaves * 64;

// The row of the cache that a block works on.
struct CacheRow {
    const char *k, *v;         // the pool
    const float *ks, *vs;
    int64_t head0;             // (layer * n_pages) * Hkv + kv head
    int Hkv, ps_shift;
    int first_page;            // page index of the unit's first position
    int ids;                   // lane i: page id of page first_page + i
    // first row of the page that holds position t (of a lane's own choosing)
    __device__ __forceinline__ int64_t row_of(int t) const {
        const int id = __shfl(ids, (t >> ps_shift) - first_page, kWave);
        return ((head0 + (int64_t)id * Hkv) << ps_shift) + (t & ((1 << ps_shift) - 1));
    }
};

// What the columns of a block stand for.
template <int NT>
struct Columns {
    int last[NT];              // last position that the lane's column of column tile nt sees
    int len;                   // positions of the request
};

__device__ __forceinline__ float max_over_groups(float v) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float sum_over_groups(float v) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

template <int D, int FMT, int NT>
struct FewTile {                                // bf16 operands
    static constexpr bool Q8 = PageRow<FMT>::kQuantised;
    static constexpr int TK = 32;
    static constexpr int KST = D / 32, KLD = Q8 ? KST / 2 : KST;
    static constexpr int EV = D / 16, VW = Q8 ? EV / 4 : EV / 2;
    static constexpr int RB = D * PageRow<FMT>::kElemBytes;
    static constexpr int NL = 8;                // logits of a lane per column tile
    uint4 qf[NT][KST];
    uint4 kf[2][KLD];
    uint32_t vw[8][VW];
    float ksc[Q8 ? 8 : 1], vsc[Q8 ? 8 : 1];
    f32x4_t acc[NT][EV];                        // acc[.][e][i]: d = EV (4 (lane / 16) + i) + e
    float x[NT][8], m_run[NT], l_run[NT];

    static __device__ __forceinline__ int k_elem(int s, int g) { return Q8 ? 64 * (s >> 1) + 16 * g + 8 * (s & 1) : 32 * s + 8 * g; }
    static __device__ __forceinline__ int acc_d(int e, int i, int lane) { return EV * (4 * (lane >> 4) + i) + e; }

    __device__ __forceinline__ void begin(int nt, const bf16_t* row, int lane) {
#pragma unroll
        for (int s = 0; s < KST; ++s) qf[nt][s] = *reinterpret_cast<const uint4*>(row + k_elem(s, lane >> 4));
        m_run[nt] = kNoMax; l_run[nt] = 0.f;
#pragma unroll
        for (int e = 0; e < EV; ++e) acc[nt][e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    __device__ __forceinline__ void request_k(const CacheRow& r, int t0, int lane) {
        const int at = 8 * ((lane >> 2) & 3) + (lane & 3);      // 8 positions of a group lie in one page
        const char* p = r.k + r.row_of(t0 + at) * RB + (lane >> 4) * 16;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int s = 0; s < KLD; ++s) kf[t][s] = *reinterpret_cast<const uint4*>(p + 4 * t * RB + 64 * s);
        if constexpr (Q8) {
            const float4* sc = reinterpret_cast<const float4*>(r.ks + r.row_of(t0 + 8 * (lane >> 4)));
            const float4 a = sc[0], b = sc[1];
            ksc[0] = a.x; ksc[1] = a.y; ksc[2] = a.z; ksc[3] = a.w; ksc[4] = b.x; ksc[5] = b.y; ksc[6] = b.z; ksc[7] = b.w;
        }
    }
    __device__ __forceinline__ void request_v(const CacheRow& r, int t0, int lane) {
        const int64_t row = r.row_of(t0 + 8 * (lane >> 4));
        const char* p = r.v + row * RB + (lane & 15) * (RB / 16);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if constexpr (VW == 4) {
                const uint4 v = *reinterpret_cast<const uint4*>(p + j * RB);
                vw[j][0] = v.x; vw[j][1] = v.y; vw[j][2] = v.z; vw[j][3] = v.w;
            } else if constexpr (VW == 2) {
                const uint2 v = *reinterpret_cast<const uint2*>(p + j * RB);
                vw[j][0] = v.x; vw[j][1] = v.y;
            } else {
                vw[j][0] = *reinterpret_cast<const uint32_t*>(p + j * RB);
            }
        }
        if constexpr (Q8) {
            const float4* sc = reinterpret_cast<const float4*>(r.vs + row);
            const float4 a = sc[0], b = sc[1];
            vsc[0] = a.x; vsc[1] = a.y; vsc[2] = a.z; vsc[3] = a.w; vsc[4] = b.x; vsc[5] = b.y; vsc[6] = b.z; vsc[7] = b.w;
        }
    }
    template <bool MASKED>
    __device__ __forceinline__ void logits(const Columns<NT>& col, float scale2, int t0, int lane) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            f32x4_t s[NT];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) s[nt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < KST; ++k) {
                uint4 piece;
                if constexpr (Q8) piece = codes_to_bf16<FMT>(k & 1 ? make_uint2(kf[t][k / 2].z, kf[t][k / 2].w) : make_uint2(kf[t][k / 2].x, kf[t][k / 2].y));
                else piece = kf[t][k];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
                    s[nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, piece), __builtin_bit_cast(bf16x8_t, qf[nt][k]), s[nt], 0, 0, 0);
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float v = s[nt][i] * (Q8 ? scale2 * ksc[4 * t + i] : scale2);
                    if (MASKED) v = t0 + 8 * (lane >> 4) + 4 * t + i <= col.last[nt] ? v : -INFINITY;
                    x[nt][4 * t + i] = v;
                }
        }
    }
    // In a tile that some column does not see to its end: V of positions that are not there is 0, and so are numbers of V that
    // are not finite (0 times them is no 0).  Returns whether there were such numbers.
    __device__ __forceinline__ bool clean_v(const Columns<NT>& col, int t0, int lane) {
        bool bad = false;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const bool there = t0 + 8 * (lane >> 4) + j < col.len;
#pragma unroll
            for (int w = 0; w < VW; ++w) {
                if constexpr (Q8) {
                    vw[j][w] = there ? vw[j][w] : 0u;
                } else {
                    const uint32_t f = there ? finite_pair(vw[j][w]) : 0u;
                    bad |= there && f != vw[j][w];
                    vw[j][w] = f;
                }
            }
        }
        return bad;
    }
    template <bool MASKED>
    __device__ __forceinline__ void outputs(const Columns<NT>& col, int t0, int lane) {
        bf16x8_t pb[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float mt = x[nt][0];
#pragma unroll
            for (int j = 1; j < 8; ++j) mt = fmaxf(mt, x[nt][j]);
            const float m_new = fmaxf(m_run[nt], max_over_groups(mt));
            if (__any(m_new > m_run[nt])) {
                const float corr = exp2_fast(m_run[nt] - m_new);
                l_run[nt] *= corr;
#pragma unroll
                for (int e = 0; e < EV; ++e) acc[nt][e] *= corr;
                m_run[nt] = m_new;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float p = exp2_fast(x[nt][j] - m_run[nt]);
                l_run[nt] += p;
                float w = p;
                if constexpr (Q8) {                             // stale slots hold any scale
                    w = p * vsc[j];
                    if (MASKED) w = t0 + 8 * (lane >> 4) + j <= col.last[nt] ? w : 0.f;
                }
                pb[nt][j] = (__bf16)w;
            }
        }
        uint32_t v[8][EV / 2];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if constexpr (!Q8) {
#pragma unroll
                for (int w = 0; w < EV / 2; ++w) v[j][w] = vw[j][w];
            } else {
                const uint4 b = codes_to_bf16<FMT>(make_uint2(vw[j][0], VW == 2 ? vw[j][VW - 1] : 0u));
                v[j][0] = b.x; v[j][1] = b.y;
                if constexpr (VW == 2) { v[j][2] = b.z; v[j][3] = b.w; }
            }
        }
        typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
#pragma unroll
        for (int e = 0; e < EV; ++e) {
            u32x4_t vt;
#pragma unroll
            for (int w = 0; w < 4; ++w) vt[w] = __builtin_amdgcn_perm(v[2 * w + 1][e / 2], v[2 * w][e / 2], e & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
                acc[nt][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, vt), pb[nt], acc[nt][e], 0, 0, 0);
        }
    }
};

template <int D, int NT>
struct FewTile<D, kPageF32, NT> {               // fp32 operands
    static constexpr int TK = 16;
    static constexpr int KP = D / 16, VP = D / 64;      // 16-byte pieces of a lane: of a K row, of a V row
    static constexpr int EV = D / 16;
    static constexpr int RB = D * 4;
    static constexpr int NL = 4;
    f32x4_t qf[NT][KP], kf[KP], vf[4][VP];
    f32x4_t acc[NT][EV];                        // acc[.][4 h + e][i]: d = 64 h + 4 (4 (lane / 16) + i) + e
    float x[NT][4], m_run[NT], l_run[NT];

    static __device__ __forceinline__ int acc_d(int e, int i, int lane) { return 64 * (e >> 2) + 4 * (4 * (lane >> 4) + i) + (e & 3); }
    __device__ __forceinline__ void begin(int nt, const float* row, int lane) {
#pragma unroll
        for (int s = 0; s < KP; ++s) qf[nt][s] = *reinterpret_cast<const f32x4_t*>(row + 16 * s + 4 * (lane >> 4));
        m_run[nt] = kNoMax; l_run[nt] = 0.f;
#pragma unroll
        for (int e = 0; e < EV; ++e) acc[nt][e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    __device__ __forceinline__ void request_k(const CacheRow& r, int t0, int lane) {
        const char* p = r.k + r.row_of(t0 + (lane & 15)) * RB + (lane >> 4) * 16;
#pragma unroll
        for (int s = 0; s < KP; ++s) kf[s] = *reinterpret_cast<const f32x4_t*>(p + 64 * s);
    }
    __device__ __forceinline__ void request_v(const CacheRow& r, int t0, int lane) {
        const char* p = r.v + r.row_of(t0 + 4 * (lane >> 4)) * RB + (lane & 15) * 16;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int h = 0; h < VP; ++h) vf[j][h] = *reinterpret_cast<const f32x4_t*>(p + j * RB + 256 * h);
    }
    template <bool MASKED>
    __device__ __forceinline__ void logits(const Columns<NT>& col, float scale2, int t0, int lane) {
        f32x4_t s[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) s[nt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < KP; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) s[nt] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[k][e], qf[nt][k][e], s[nt], 0, 0, 0);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float v = s[nt][i] * scale2;
                if (MASKED) v = t0 + 4 * (lane >> 4) + i <= col.last[nt] ? v : -INFINITY;
                x[nt][i] = v;
            }
    }
    __device__ __forceinline__ bool clean_v(const Columns<NT>& col, int t0, int lane) {
        bool bad = false;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bool there = t0 + 4 * (lane >> 4) + j < col.len;
#pragma unroll
            for (int h = 0; h < VP; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float f = vf[j][h][e];
                    const bool ok = is_finite(f);
                    bad |= there && !ok;
                    vf[j][h][e] = there && ok ? f : 0.f;
                }
        }
        return bad;
    }
    template <bool MASKED>
    __device__ __forceinline__ void outputs(const Columns<NT>&, int, int) {
        float p[NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float mt = x[nt][0];
#pragma unroll
            for (int j = 1; j < 4; ++j) mt = fmaxf(mt, x[nt][j]);
            const float m_new = fmaxf(m_run[nt], max_over_groups(mt));
            if (__any(m_new > m_run[nt])) {
                const float corr = exp2_fast(m_run[nt] - m_new);
                l_run[nt] *= corr;
#pragma unroll
                for (int e = 0; e < EV; ++e) acc[nt][e] *= corr;
                m_run[nt] = m_new;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) { p[nt][j] = exp2_fast(x[nt][j] - m_run[nt]); l_run[nt] += p[nt][j]; }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < EV; ++e)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) acc[nt][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[j][e >> 2][e & 3], p[nt][j], acc[nt][e], 0, 0, 0);
    }
};

// The unit's new rows into their pages, by the whole block; ids: the page ids as r.ids, -1 for a page that is none.
template <int D, int FMT>
__device__ __forceinline__ void write_new_rows(const PagesAttnParams& a, const CacheRow& r, int l, int b, int h, int from, int to, int first_new, int ids) {
    typedef PageRow<FMT> R;
    typedef typename R::T T;
    constexpr int LPR = D * (int)sizeof(T) / 16;
    const int sub = threadIdx.x % LPR;
    for (int t0 = from; t0 < to; t0 += kThreads / LPR) {        // block-uniform: row_of is a wave's
        const int t = t0 + threadIdx.x / LPR;
        const int64_t row = r.row_of(min(t, to - 1));
        const int id = __shfl(ids, (min(t, to - 1) >> r.ps_shift) - r.first_page, kWave);
        if (t >= to || id < 0) continue;                        // a page that is none is not written to
        const uint4 kx = reinterpret_cast<const uint4*>(a.k_new.at(l, b, h, t - first_new))[sub];
        const uint4 vx = reinterpret_cast<const uint4*>(a.v_new.at(l, b, h, t - first_new))[sub];
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
}

template <int D, int FMT, int NT>
__global__ __launch_bounds__(kThreads, NT == 1 ? 3 : 2) void pages_few_kernel(PagesAttnParams a) {
    typedef typename PageRow<FMT>::T T;
    typedef FewTile<D, FMT, NT> Tile;
    constexpr int TK = Tile::TK, STEP = kWaves * TK, DL = D + 4;
    __shared__ __align__(16) float sMerge[kWaves][16][DL];
    __shared__ int sLast, sNotFinite[kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int rows = a.p.n_layers * a.p.B * a.p.Hkv;
    const int row = blockIdx.x % rows, unit = blockIdx.x / rows;    // the first units of all rows come first
    const int h = row % a.p.Hkv, lb = row / a.p.Hkv, b = lb % a.p.B, l = lb / a.p.B;
    CacheRow r;
    r.k = a.p.k; r.v = a.p.v; r.ks = a.p.k_scale; r.vs = a.p.v_scale;
    r.Hkv = a.p.Hkv; r.ps_shift = a.p.ps_shift;
    r.head0 = (int64_t)(a.p.layer_begin + l) * a.p.n_pages * a.p.Hkv + h;
    r.first_page = (unit << a.unit_shift) >> a.p.ps_shift;
    // the unit's page ids, a lane each (at most 64 pages): requested beside the lengths, which say how many of them count
    int id = 0;
    if (r.first_page + lane < a.p.max_pages) id = a.p.table[(int64_t)b * a.p.max_pages + r.first_page + lane];
    const ChunkLen len = chunk_len(a.p, b);
    if (!len.ok && l == 0 && h == 0 && unit == 0 && tid == 0) report_lens(a.p, b);
    const int begin = unit << a.unit_shift;
    if (len.c == 0 || begin >= len.n) return;
    const int end = min(len.n, begin + (1 << a.unit_shift));
    const int nu = (len.n + (1 << a.unit_shift) - 1) >> a.unit_shift;
    const bool held = r.first_page + lane <= (end - 1) >> a.p.ps_shift;
    const bool bad_id = held && (uint32_t)id >= (uint32_t)a.p.n_pages;
    if (bad_id && wave == 0) set_sticky(a.p.status, VLC_ERR_INVALID_ARG, b, kStickyPage, id);
    r.ids = held && !bad_id ? id : 0;
    const int g = a.p.g, cols = g * len.c, first_new = len.n - len.c;
    if (a.k_new.data && end > first_new) {
        write_new_rows<D, FMT>(a, r, l, b, h, max(begin, first_new), end, first_new, bad_id ? -1 : r.ids);
        __threadfence_block();
        __syncthreads();
    }
    Columns<NT> col;
    col.len = len.n;
    Tile tile;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int c = min(16 * nt + (lane & 15), cols - 1);         // columns beyond the last repeat it; their results are not kept
        col.last[nt] = first_new + c / g;
        tile.begin(nt, (const T*)a.q.at(l, b, h * g + c % g, c / g), lane);
    }
    const float scale2 = attn_scale(a, l, D) * kLog2e;

    bool not_finite = false;                                    // numbers of V were replaced by 0 in a tile
    // Positions behind the last one are read too (slots of the same page, or of page 0 in place of a page that is not there).
    // K of the next tile is requested as soon as the logits are formed, V as soon as the outputs are: the same registers.
    int t0 = begin + wave * TK;
    if (t0 < end) {
        tile.request_k(r, t0, lane);
        tile.request_v(r, t0, lane);
        // Only the last tile of a wave can reach beyond what every column sees: at most 32 new tokens stand at the row's end,
        // and the tiles before a wave's last one end STEP - TK >= 48 positions earlier.
#pragma unroll 1
        for (; t0 + STEP < end; t0 += STEP) {
            tile.template logits<false>(col, scale2, t0, lane);
            tile.request_k(r, t0 + STEP, lane);
            tile.template outputs<false>(col, t0, lane);
            tile.request_v(r, t0 + STEP, lane);
        }
        tile.template logits<true>(col, scale2, t0, lane);
        not_finite = tile.clean_v(col, t0, lane);
        tile.template outputs<true>(col, t0, lane);
    }

    if (__any(not_finite)) {
        if (lane == 0) sNotFinite[wave] = 1;
    } else if (lane == 0) {
        sNotFinite[wave] = 0;
    }
    // What is not finite in V reaches the columns that see it: from memory, a number at a time.  (Codes are finite; a row
    // that was not has a scale of NaN, which the probability takes.)
    auto add_not_finite = [&](int last, int e, float& o0, float& o1) {
        if constexpr (!PageRow<FMT>::kQuantised) {
            for (int t = max(begin, (end - STEP + TK - 1) & -TK); t < min(end, last + 1); ++t) {     // the waves' last tiles
                int page = a.p.table[(int64_t)b * a.p.max_pages + (t >> a.p.ps_shift)];
                if ((uint32_t)page >= (uint32_t)a.p.n_pages) page = 0;
                const T* v = (const T*)a.p.v + (page_row0(a.p, a.p.layer_begin + l, page, h) + (t & ((1 << a.p.ps_shift) - 1))) * D + e;
                const float f0 = Elem<T>::load(v), f1 = Elem<T>::load(v + 1);
                if (!is_finite(f0)) o0 += f0;
                if (!is_finite(f1)) o1 += f1;
            }
        }
    };

    float* part = a.partials + ((int64_t)row * a.n_units + unit) * a.part_floats;
    // ---- merge of the waves, 16 columns at a time: into the output, or into the unit's partial result
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int nc = min(cols - 16 * nt, 16);
        if (nc <= 0) break;
        if (nt) __syncthreads();
        const float z = sum_over_groups(tile.l_run[nt]);
        if ((lane & 15) < nc) {
            float* dst = sMerge[wave][lane & 15];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < Tile::EV; e += 4)
                    *reinterpret_cast<float4*>(dst + Tile::acc_d(e, i, lane)) = make_float4(tile.acc[nt][e][i], tile.acc[nt][e + 1][i], tile.acc[nt][e + 2][i], tile.acc[nt][e + 3][i]);
            if (lane < 16) { dst[D] = tile.m_run[nt]; dst[D + 1] = z; }
        }
        __syncthreads();
        for (int x = tid; x < nc * (D / 2); x += kThreads) {
            const int cc = x / (D / 2), e = x % (D / 2) * 2;
            float m = kNoMax, o0 = 0.f, o1 = 0.f, zz = 0.f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) m = fmaxf(m, sMerge[w][cc][D]);
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const float wgt = exp2_fast(sMerge[w][cc][D] - m);
                o0 = fmaf(sMerge[w][cc][e], wgt, o0);
                o1 = fmaf(sMerge[w][cc][e + 1], wgt, o1);
                zz = fmaf(sMerge[w][cc][D + 1], wgt, zz);
            }
            const int c = 16 * nt + cc;
            if (!PageRow<FMT>::kQuantised && (sNotFinite[0] | sNotFinite[1] | sNotFinite[2] | sNotFinite[3])) add_not_finite(first_new + c / g, e, o0, o1);
            if (nu == 1) {
                T* out = (T*)a.out.at(l, b, h * g + c % g, c / g) + e;
                store_pair(out, zz == 0.f ? 0.f : o0 / zz, zz == 0.f ? 0.f : o1 / zz);
                if (e == 0 && a.stats.row_max) store_stats(a, l, b, h * g + c % g, c / g, m, zz);
            } else {
                store_agent2(part + c * D + e, o0, o1);
                if (e == 0) store_agent2(part + cols * D + 2 * c, m, zz);
            }
        }
    }
    if (nu == 1) return;
    // ---- the unit counts itself once its stores are acknowledged; the last one of the row merges
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0) sLast = __hip_atomic_fetch_add(a.counters + row, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == nu - 1;
    __syncthreads();
    if (!sLast) return;
    if (tid == 0) __hip_atomic_store(a.counters + row, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    // Two neighbouring outputs per thread; if the block has threads for several times all outputs, the units are dealt to
    // them, and the groups of threads merge through LDS.
    const float* parts = a.partials + (int64_t)row * a.n_units * a.part_floats;
    const int pairs = cols * (D / 2);
    const int groups = pairs >= kThreads ? 1 : kThreads / pairs;
    constexpr int NB = 8;                                       // partial results whose loads are in flight together
    float* sPart = &sMerge[0][0][0];                            // [kThreads][4]
    for (int x0 = 0; x0 < pairs; x0 += kThreads) {              // one round unless groups == 1
        const int x = groups == 1 ? x0 + tid : tid % pairs, grp = groups == 1 ? 0 : tid / pairs;
        float m = kNoMax, o0 = 0.f, o1 = 0.f, z = 0.f;
        const int c = x / (D / 2), e = x % (D / 2) * 2;
        if (x < pairs && grp < groups)
#pragma unroll 1
            for (int u0 = grp; u0 < nu; u0 += NB * groups) {
                float2 ml[NB], ov[NB];
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    const int u = min(u0 + j * groups, nu - 1);
                    ml[j] = load_agent2(parts + (int64_t)u * a.part_floats + cols * D + 2 * c);
                    ov[j] = load_agent2(parts + (int64_t)u * a.part_floats + c * D + e);
                    if (u0 + j * groups >= nu) { ml[j] = make_float2(kNoMax, 0.f); ov[j] = make_float2(0.f, 0.f); }
                }
                float mn = m;
#pragma unroll
                for (int j = 0; j < NB; ++j) mn = fmaxf(mn, ml[j].x);
                const float w0 = exp2_fast(m - mn);
                o0 *= w0; o1 *= w0; z *= w0;
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    const float wgt = exp2_fast(ml[j].x - mn);
                    o0 = fmaf(ov[j].x, wgt, o0); o1 = fmaf(ov[j].y, wgt, o1); z = fmaf(ml[j].y, wgt, z);
                }
                m = mn;
            }
        if (groups > 1) {
            __syncthreads();
            *reinterpret_cast<float4*>(sPart + 4 * tid) = make_float4(m, z, o0, o1);
            __syncthreads();
            if (tid < pairs)
                for (int k = 1; k < groups; ++k) {
                    const float4 f = *reinterpret_cast<const float4*>(sPart + 4 * (tid + k * pairs));
                    const float mn = fmaxf(m, f.x), w0 = exp2_fast(m - mn), w1 = exp2_fast(f.x - mn);
                    o0 = o0 * w0 + f.z * w1; o1 = o1 * w0 + f.w * w1; z = z * w0 + f.y * w1;
                    m = mn;
                }
        }
        if (x < pairs && grp == 0) {
            T* out = (T*)a.out.at(l, b, h * g + c % g, c / g) + e;
            store_pair(out, z == 0.f ? 0.f : o0 / z, z == 0.f ? 0.f : o1 / z);
            if (e == 0 && a.stats.row_max) store_stats(a, l, b, h * g + c % g, c / g, m, z);
        }
    }
}

struct FewPlan { int unit_shift, n_units, part_floats; size_t bytes; };

FewPlan plan(const PagesCall& c) {
    FewPlan f;
    const int ps_shift = __builtin_ctz(c.s.page_slots);
    const int64_t rows = (int64_t)c.n_layers * c.chunk.B * c.s.Hkv;
    f.unit_shift = 7;
    while (f.unit_shift < 10 && f.unit_shift < ps_shift + 6 && rows * ((c.chunk.max_len >> f.unit_shift) + 1) > 2048) ++f.unit_shift;
    f.n_units = (c.chunk.max_len + (1 << f.unit_shift) - 1) >> f.unit_shift;
    const int cols = c.s.Hq / c.s.Hkv * c.chunk.max_new;
    f.part_floats = (cols * (c.s.d + 2) + 3) & ~3;
    f.bytes = f.n_units > 1 ? (size_t)rows * f.n_units * f.part_floats * sizeof(float) : 0;
    return f;
}

template <int D, int FMT>
void launch(const PagesAttnParams& a, int cols, hipStream_t st) {
    const unsigned grid = (unsigned)(a.p.n_layers * a.p.B * a.p.Hkv) * a.n_units;
    if (cols <= 16) pages_few_kernel<D, FMT, 1><<<grid, kThreads, 0, st>>>(a);
    else pages_few_kernel<D, FMT, 2><<<grid, kThreads, 0, st>>>(a);
}

}  // namespace

bool pages_few_supported(const PagesCall& c) { return (int64_t)(c.s.Hq / c.s.Hkv) * c.chunk.max_new <= 32; }
size_t pages_few_workspace_bytes(const PagesCall& c) { return plan(c).bytes; }

hipError_t launch_pages_few(const PagesAttn& c) {
    const FewPlan f = plan(c.c);
    PagesAttnParams a = pages_attn_params(c);
    a.unit_shift = f.unit_shift; a.n_units = f.n_units; a.part_floats = f.part_floats;
    const int cols = a.p.g * a.p.max_new;
    const bool wide = c.c.s.d == 128;
    switch (page_format(c.c.s)) {
        case kPageBf16: wide ? launch<128, kPageBf16>(a, cols, c.c.stream) : launch<64, kPageBf16>(a, cols, c.c.stream); break;
        case kPageF32: wide ? launch<128, kPageF32>(a, cols, c.c.stream) : launch<64, kPageF32>(a, cols, c.c.stream); break;
        case kPageFp8: wide ? launch<128, kPageFp8>(a, cols, c.c.stream) : launch<64, kPageFp8>(a, cols, c.c.stream); break;
        case kPageInt8: wide ? launch<128, kPageInt8>(a, cols, c.c.stream) : launch<64, kPageInt8>(a, cols, c.c.stream); break;
    }
    return hipGetLastError();
}

}  // namespace vlc
