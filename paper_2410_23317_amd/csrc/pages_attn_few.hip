// Attention of a few new tokens over the pages of their request (gfx950): up to 64 query rows per KV head (fp32 storage: 32), the g
// heads of up to 64 / g tokens, which is decoding, and verifying drafted tokens.
//
// Bound by memory where there is enough of it: every K and V row is read once and serves all query rows of its KV head (24 FP8
// requests of up to 10369 positions, 287 MB, take 65.6 us on inputs that no cache holds: 4.4 TB/s; 53 to 56 on the same input again,
// which the memory-side cache partly holds; plain rows 114 us, 4.9 TB/s).  A small call is a chain of waits: one token over 2945
// positions (12 MB) takes 10.0 us, over 300 8.4, over 100 6.5.  A (layer, request, KV head) row of the cache is cut into units of 2^unit_shift
// positions, a block of four waves each; the tiles of a unit are dealt to the waves, which merge through LDS.  Units of a row
// leave unnormalised partial results.  Up to 16 query rows they store them with device scope and count themselves; the one
// that counts last merges them and writes the output (its own stores are acknowledged before it counts, so whoever counts last
// finds all of them in memory).  With more rows one block would read the partial results for longer than a second launch takes
// (35 rows, eight int8 requests: 32.2 us, by a second kernel 28.0), which then merges.
// New rows that the call has to write first are kept in LDS as well: the tiles that hold them take them from there instead of
// waiting until the stores can be read back.
//
// A tile's operands come from memory in the order the matrix instructions want, without a trip through LDS or across
// lanes.  bf16 (codes are expanded to bf16, exactly, where they are used; K's scale multiplies the finished logit, V's the
// probability before it is split into two bf16 numbers): 32 positions, 8 G + j for lane group G = lane / 16, place j.  Logits
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

// The new rows of a call that writes them, as the pages hold them: the last tile of a wave takes them from here, so that nothing
// waits until the stores into the pages can be read back.
template <int D, int FMT, int ROWS>
struct NewRows {
    static constexpr int RB = D * PageRow<FMT>::kElemBytes;
    uint4 k[ROWS][RB / 16], v[ROWS][RB / 16];
    float ks[PageRow<FMT>::kQuantised ? ROWS : 1], vs[PageRow<FMT>::kQuantised ? ROWS : 1];
};

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
    // New rows (positions first_new on) in place of what was requested for them.
    template <int ROWS>
    __device__ __forceinline__ void take_new(const NewRows<D, FMT, ROWS>& n, int first_new, int len, int t0, int lane) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int i = t0 + 8 * ((lane >> 2) & 3) + (lane & 3) + 4 * t - first_new;
            if (i >= 0 && i < len - first_new) {
#pragma unroll
                for (int s = 0; s < KLD; ++s) kf[t][s] = *reinterpret_cast<const uint4*>((const char*)n.k[i] + (lane >> 4) * 16 + 64 * s);
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int i = t0 + 8 * (lane >> 4) + j - first_new;
            if (i >= 0 && i < len - first_new) {
                const uint32_t* p = reinterpret_cast<const uint32_t*>((const char*)n.v[i] + (lane & 15) * (RB / 16));
#pragma unroll
                for (int w = 0; w < VW; ++w) vw[j][w] = p[w];
                if constexpr (Q8) { ksc[j] = n.ks[i]; vsc[j] = n.vs[i]; }
            }
        }
    }
    // A logit is rounded before the maximum is taken off: |s| 2^-24 of its weight, less than the output's rounding up to |s| = 2^15.
    // (Taking it off in one fma, as fp32 storage does, makes Q wait for the scale's sign: one token 9.95 -> 10.25 us.)
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
    __device__ __forceinline__ void outputs(const Columns<NT>& col, float, int t0, int lane) {
        bf16x8_t pb[NT], pl[NT];                                // weights as two bf16 numbers: what the first leaves over in the second
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
                if constexpr (Q8) {
                    pb[nt][j] = (__bf16)w;
                    pl[nt][j] = (__bf16)(w - (float)pb[nt][j]);
                } else {            // V may hold infinities: both parts of a weight above 0 are above 0, so that their sum is no NaN
                    const uint32_t first = __float_as_uint(w) & 0xffff0000u;
                    pb[nt][j] = __builtin_bit_cast(__bf16, (uint16_t)(first >> 16));
                    pl[nt][j] = (__bf16)__builtin_amdgcn_fmed3f(w - __uint_as_float(first), w, 0x1p-126f);
                }
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
#pragma unroll
        for (int e = 0; e < EV; ++e) {
            u32x4_t vt;
#pragma unroll
            for (int w = 0; w < 4; ++w) vt[w] = __builtin_amdgcn_perm(v[2 * w + 1][e / 2], v[2 * w][e / 2], e & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                acc[nt][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, vt), pb[nt], acc[nt][e], 0, 0, 0);
                acc[nt][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, vt), pl[nt], acc[nt][e], 0, 0, 0);
            }
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
    template <int ROWS>
    __device__ __forceinline__ void take_new(const NewRows<D, kPageF32, ROWS>& n, int first_new, int len, int t0, int lane) {
        const int i = t0 + (lane & 15) - first_new;
        if (i >= 0 && i < len - first_new) {
#pragma unroll
            for (int s = 0; s < KP; ++s) kf[s] = *reinterpret_cast<const f32x4_t*>((const char*)n.k[i] + (lane >> 4) * 16 + 64 * s);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = t0 + 4 * (lane >> 4) + j - first_new;
            if (i >= 0 && i < len - first_new) {
#pragma unroll
                for (int h = 0; h < VP; ++h) vf[j][h] = *reinterpret_cast<const f32x4_t*>((const char*)n.v[i] + (lane & 15) * 16 + 256 * h);
            }
        }
    }
    // x holds the products Q K^T: the maximum is taken off their logits with one rounding, of the difference (fp32 outputs show
    // the rounding of a large logit).  Q takes the sign of a scale that is not positive, or is 0 for a scale of 0, so that the
    // largest product is the largest logit.
    __device__ __forceinline__ void sign_q(float scale) {
        const float sign = scale < 0.f ? -1.f : scale == 0.f ? 0.f : 1.f;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int s = 0; s < KP; ++s) qf[nt][s] *= sign;
    }
    template <bool MASKED>
    __device__ __forceinline__ void logits(const Columns<NT>& col, float, int t0, int lane) {
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
                float v = s[nt][i];
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
    __device__ __forceinline__ void outputs(const Columns<NT>&, float scale2, int, int) {
        float p[NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float mt = x[nt][0];
#pragma unroll
            for (int j = 1; j < 4; ++j) mt = fmaxf(mt, x[nt][j]);
            const float m_new = fmaxf(m_run[nt], max_over_groups(mt) * scale2);
            if (__any(m_new > m_run[nt])) {
                const float corr = exp2_fast(m_run[nt] - m_new);
                l_run[nt] *= corr;
#pragma unroll
                for (int e = 0; e < EV; ++e) acc[nt][e] *= corr;
                m_run[nt] = m_new;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) { p[nt][j] = exp2_fast(fmaf(x[nt][j], scale2, -m_run[nt])); l_run[nt] += p[nt][j]; }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < EV; ++e)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) acc[nt][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[j][e >> 2][e & 3], p[nt][j], acc[nt][e], 0, 0, 0);
    }
};

// Rows first_new + i, i in [from, to), into LDS and into their pages, by the whole block; ids: the page ids as r.ids, -1 for
// a page that is none and is not written to.
template <int D, int FMT, int ROWS>
__device__ __forceinline__ void write_new_rows(const PagesAttnParams& a, const CacheRow& r, NewRows<D, FMT, ROWS>& n, int l, int b, int h, int from, int to,
                                               int first_new, int ids) {
    typedef PageRow<FMT> R;
    typedef typename R::T T;
    constexpr int LPR = D * (int)sizeof(T) / 16;
    const int sub = threadIdx.x % LPR;
    for (int i0 = from; i0 < to; i0 += kThreads / LPR) {        // block-uniform: row_of is a wave's
        const int i = min(i0 + (int)threadIdx.x / LPR, to - 1), t = first_new + i;
        const int64_t row = r.row_of(t);
        const bool there = __shfl(ids, (t >> r.ps_shift) - r.first_page, kWave) >= 0;
        if (i0 + (int)threadIdx.x / LPR >= to) break;
        const uint4 kx = reinterpret_cast<const uint4*>(a.k_new.at(l, b, h, i))[sub];
        const uint4 vx = reinterpret_cast<const uint4*>(a.v_new.at(l, b, h, i))[sub];
        if constexpr (!R::kQuantised) {
            n.k[i][sub] = kx;
            n.v[i][sub] = vx;
            if (there) {
                reinterpret_cast<uint4*>(a.p.k)[row * LPR + sub] = kx;
                reinterpret_cast<uint4*>(a.p.v)[row * LPR + sub] = vx;
            }
        } else {
            float ks, vs;
            const uint2 kc = quantize_page_row<FMT, LPR>(kx, ks), vc = quantize_page_row<FMT, LPR>(vx, vs);
            reinterpret_cast<uint2*>(n.k[i])[sub] = kc;
            reinterpret_cast<uint2*>(n.v[i])[sub] = vc;
            if (sub == 0) { n.ks[i] = ks; n.vs[i] = vs; }
            if (there) {
                reinterpret_cast<uint2*>(a.p.k)[row * LPR + sub] = kc;
                reinterpret_cast<uint2*>(a.p.v)[row * LPR + sub] = vc;
                if (sub == 0) { a.p.k_scale[row] = ks; a.p.v_scale[row] = vs; }
            }
        }
    }
}

// Outputs e .. e + 3 of column c, and its statistics.
template <typename T>
__device__ __forceinline__ void store_column(const PagesAttnParams& a, int l, int b, int h, int c, int e, const f32x4_t& o, float m, float z) {
    const int head = h * a.p.g + c % a.p.g, i = c / a.p.g;
    T* out = (T*)a.out.at(l, b, head, i) + e;
    const float div = z == 0.f ? 1.f : z;                       // a row without weights: its sums are 0
    store_pair(out, o[0] / div, o[1] / div);
    store_pair(out + 2, o[2] / div, o[3] / div);
    if (e == 0 && a.stats.row_max) store_stats(a, l, b, head, i, m, z);
}

template <int D, int FMT, int NT>
__global__ __launch_bounds__(kThreads, NT == 1 ? 3 : NT == 2 || D == 64 ? 2 : 1) void pages_few_kernel(PagesAttnParams a) {
    constexpr bool ONE_LAUNCH = NT == 1;        // the last unit of a row merges; else a second kernel does
    typedef typename PageRow<FMT>::T T;
    typedef FewTile<D, FMT, NT> Tile;
    constexpr int TK = Tile::TK, STEP = kWaves * TK, DL = D + 4;
    static_assert(16 * NT <= STEP - TK, "the new tokens lie in the waves' last tiles");
    __shared__ __align__(16) float sMerge[kWaves][16][DL];
    __shared__ NewRows<D, FMT, 16 * NT> sNew;
    __shared__ int sLast, sNotFinite[kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    const int h = blockIdx.x, lb = blockIdx.y, unit = blockIdx.z;   // the first units of all rows come first, those that may be empty last
    const int b = lb % a.p.B, l = lb / a.p.B, row = lb * a.p.Hkv + h;
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
    Columns<NT> col;
    col.len = len.n;
    Tile tile;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int c = min(16 * nt + (lane & 15), cols - 1);         // columns beyond the last repeat it; their results are not kept
        const int i = (c * a.g_inverse) >> 16;                      // c / g: c < 64
        col.last[nt] = first_new + i;
        tile.begin(nt, (const T*)a.q.at(l, b, h * g + c - i * g, i), lane);
    }
    float scale = attn_scale(a, l, D);
    if constexpr (FMT == kPageF32) {
        if (!(scale > 0.f)) {
            tile.sign_q(scale);
            scale = scale == 0.f ? 1.f : -scale;
        }
    }
    const float scale2 = scale * kLog2e;

    bool not_finite = false;                                    // numbers of V were replaced by 0 in a tile
    // Positions behind the last one are read too (slots of the same page, or of page 0 in place of a page that is not there).
    // K of the next tile is requested as soon as the logits are formed, V as soon as the outputs are: the same registers.
    int t0 = begin + wave * TK;
    const bool fresh = a.k_new.data && end > first_new;         // block-uniform
    if (t0 < end) {
        tile.request_k(r, t0, lane);
        tile.request_v(r, t0, lane);
    }
    if (fresh) {
        write_new_rows<D, FMT>(a, r, sNew, l, b, h, max(begin - first_new, 0), end - first_new, first_new, bad_id ? -1 : r.ids);
        __syncthreads();
    }
    if (t0 < end) {
        // Only the last tile of a wave can reach beyond what every column sees: the at most 16 NT new tokens stand at the
        // row's end, and the tiles before a wave's last one end STEP - TK = 96 (fp32: 48) positions before the unit does.
#pragma unroll 1
        for (; t0 + STEP < end; t0 += STEP) {
            tile.template logits<false>(col, scale2, t0, lane);
            tile.request_k(r, t0 + STEP, lane);
            tile.template outputs<false>(col, scale2, t0, lane);
            tile.request_v(r, t0 + STEP, lane);
        }
        if (fresh) tile.take_new(sNew, first_new, end, t0, lane);
        tile.template logits<true>(col, scale2, t0, lane);
        if (t0 + TK > first_new + 1) not_finite = tile.clean_v(col, t0, lane);
        tile.template outputs<true>(col, scale2, t0, lane);
    }

    if (__any(not_finite)) {
        if (lane == 0) sNotFinite[wave] = 1;
    } else if (lane == 0) {
        sNotFinite[wave] = 0;
    }
    // What is not finite in V reaches the columns that see it: from memory, a number at a time.  (Codes are finite; a row
    // that was not has a scale of NaN, which the probability takes.)
    auto add_not_finite = [&](int last, int e, f32x4_t& o) {
        if constexpr (!PageRow<FMT>::kQuantised) {
            for (int t = max(begin, (first_new + 1) & -TK); t < min(end, last + 1); ++t) {       // the tiles that were cleaned
                int page = a.p.table[(int64_t)b * a.p.max_pages + (t >> a.p.ps_shift)];
                if ((uint32_t)page >= (uint32_t)a.p.n_pages) page = 0;
                const T* v = (const T*)a.p.v + (page_row0(a.p, a.p.layer_begin + l, page, h) + (t & ((1 << a.p.ps_shift) - 1))) * D + e;
                if (fresh && t >= first_new) v = (const T*)sNew.v[t - first_new] + e;       // its store may still be on its way
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float f = Elem<T>::load(v + i);
                    if (!is_finite(f)) o[i] += f;
                }
            }
        }
    };

    auto store_out = [&](int c, int e, const f32x4_t& o, float m, float z) { store_column<T>(a, l, b, h, c, e, o, m, z); };
    auto any_not_finite = [&]() {
        int any = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) any |= sNotFinite[w];
        return any != 0;
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
        for (int x = tid; x < nc * (D / 4); x += kThreads) {
            const int cc = x / (D / 4), e = x % (D / 4) * 4;
            float m = kNoMax, zz = 0.f;
            f32x4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < kWaves; ++w) m = fmaxf(m, sMerge[w][cc][D]);
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const float wgt = exp2_fast(sMerge[w][cc][D] - m);
                o += *reinterpret_cast<const f32x4_t*>(&sMerge[w][cc][e]) * wgt;
                zz = fmaf(sMerge[w][cc][D + 1], wgt, zz);
            }
            const int c = 16 * nt + cc;
            if (!PageRow<FMT>::kQuantised && any_not_finite()) add_not_finite(first_new + c / g, e, o);
            if (nu == 1) {
                store_out(c, e, o, m, zz);
            } else if constexpr (ONE_LAUNCH) {                      // device-scope stores
                store_agent2(part + c * D + e, o[0], o[1]);
                store_agent2(part + c * D + e + 2, o[2], o[3]);
                if (e == 0) store_agent2(part + cols * D + 2 * c, m, zz);
            } else {
                *reinterpret_cast<f32x4_t*>(part + c * D + e) = o;
                if (e == 0) *reinterpret_cast<float2*>(part + cols * D + 2 * c) = make_float2(m, zz);
            }
        }
    }
    if constexpr (!ONE_LAUNCH) return;
    if (nu == 1) return;
    // ---- the unit counts itself once its stores are acknowledged; the last one of the row merges
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0) sLast = __hip_atomic_fetch_add(a.counters + row, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == nu - 1;
    __syncthreads();
    if (!sLast) return;
    if (tid == 0) __hip_atomic_store(a.counters + row, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    // Four neighbouring outputs per thread and round, the loads of all rounds and of NB units in flight together; if the block
    // has threads for several times all outputs, the units are dealt to them, and the groups of threads merge through LDS.
    constexpr int ROUNDS = (16 * (D / 4) + kThreads - 1) / kThreads, NB = 8;
    const auto parts = partials_buffer(a.partials + (int64_t)row * a.n_units * a.part_floats, nu * a.part_floats * 4);
    const int quads = cols * (D / 4);
    const int groups = quads >= kThreads ? 1 : kThreads / quads;
    const int x0 = groups == 1 ? tid : tid % quads, grp = groups == 1 ? 0 : tid / quads;
    float m[ROUNDS], z[ROUNDS];
    f32x4_t o[ROUNDS];
#pragma unroll
    for (int k = 0; k < ROUNDS; ++k) { m[k] = kNoMax; z[k] = 0.f; o[k] = f32x4_t{0.f, 0.f, 0.f, 0.f}; }
#pragma unroll 1
    for (int u0 = grp; u0 < nu; u0 += NB * groups) {
        float2 ml[ROUNDS][NB];
        f32x4_t ov[ROUNDS][NB];
#pragma unroll
        for (int k = 0; k < ROUNDS; ++k)
            if (k == 0 || k * kThreads < quads) {               // block-uniform
                const int x = min(x0 + k * kThreads, quads - 1), c = x / (D / 4), e = x % (D / 4) * 4;
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    const int at = min(u0 + j * groups, nu - 1) * a.part_floats * 4;
                    ml[k][j] = buffer_load8_agent(parts, at + (cols * D + 2 * c) * 4);
                    ov[k][j] = buffer_load16_agent(parts, at + (c * D + e) * 4);
                }
            }
#pragma unroll
        for (int k = 0; k < ROUNDS; ++k)
            if (k == 0 || k * kThreads < quads) {
                float mn = m[k];
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    if (u0 + j * groups >= nu) { ml[k][j] = make_float2(kNoMax, 0.f); ov[k][j] = f32x4_t{0.f, 0.f, 0.f, 0.f}; }
                    mn = fmaxf(mn, ml[k][j].x);
                }
                const float w0 = exp2_fast(m[k] - mn);
                o[k] *= w0; z[k] *= w0;
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    const float wgt = exp2_fast(ml[k][j].x - mn);
                    o[k] += ov[k][j] * wgt;
                    z[k] = fmaf(ml[k][j].y, wgt, z[k]);
                }
                m[k] = mn;
            }
    }
    if (groups > 1) {
        float* sPart = &sMerge[0][0][0];                        // [kThreads][6]
        float* mine = sPart + 6 * tid;
        mine[0] = m[0]; mine[1] = z[0]; mine[2] = o[0][0]; mine[3] = o[0][1]; mine[4] = o[0][2]; mine[5] = o[0][3];
        __syncthreads();
        if (tid < quads)
            for (int k = 1; k < groups; ++k) {
                const float* f = sPart + 6 * (tid + k * quads);
                const float mn = fmaxf(m[0], f[0]), w0 = exp2_fast(m[0] - mn), w1 = exp2_fast(f[0] - mn);
                o[0] = o[0] * w0 + f32x4_t{f[2], f[3], f[4], f[5]} * w1;
                z[0] = z[0] * w0 + f[1] * w1;
                m[0] = mn;
            }
    }
#pragma unroll
    for (int k = 0; k < ROUNDS; ++k) {
        const int x = x0 + k * kThreads, c = x / (D / 4), e = x % (D / 4) * 4;
        if (grp != 0 || x >= quads) break;
        store_out(c, e, o[k], m[k], z[k]);
    }
}

// Merge of the units of a row, four neighbouring outputs per thread.
template <typename T, int D>
__global__ __launch_bounds__(256) void pages_few_merge_kernel(PagesAttnParams a) {
    const int row = blockIdx.y, h = row % a.p.Hkv, lb = row / a.p.Hkv, b = lb % a.p.B, l = lb / a.p.B;
    const ChunkLen len = chunk_len(a.p, b);
    const int nu = (len.n + (1 << a.unit_shift) - 1) >> a.unit_shift, cols = a.p.g * len.c;
    const int x = blockIdx.x * 256 + threadIdx.x, c = x / (D / 4), e = x % (D / 4) * 4;
    if (nu < 2 || c >= cols) return;
    const float* part = a.partials + (int64_t)row * a.n_units * a.part_floats;
    constexpr int NB = 8;
    float m = kNoMax, z = 0.f;
    f32x4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (int u0 = 0; u0 < nu; u0 += NB) {
        float2 ml[NB];
        f32x4_t ov[NB];
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const float* p = part + (int64_t)min(u0 + j, nu - 1) * a.part_floats;
            ml[j] = *reinterpret_cast<const float2*>(p + cols * D + 2 * c);
            ov[j] = *reinterpret_cast<const f32x4_t*>(p + c * D + e);
        }
        float mn = m;
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            if (u0 + j >= nu) { ml[j] = make_float2(kNoMax, 0.f); ov[j] = f32x4_t{0.f, 0.f, 0.f, 0.f}; }
            mn = fmaxf(mn, ml[j].x);
        }
        const float w0 = exp2_fast(m - mn);
        o *= w0; z *= w0;
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const float wgt = exp2_fast(ml[j].x - mn);
            o += ov[j] * wgt;
            z = fmaf(ml[j].y, wgt, z);
        }
        m = mn;
    }
    store_column<T>(a, l, b, h, c, e, o, m, z);
}

struct FewPlan { int unit_shift, n_units, part_floats; size_t bytes; };

FewPlan plan(const PagesCall& c) {
    FewPlan f;
    const int ps_shift = __builtin_ctz(c.s.page_slots);
    const int64_t rows = (int64_t)c.n_layers * c.chunk.B * c.s.Hkv;
    // Units so long that about 192 blocks cover the call: three quarters of the compute units start at once, and few partial
    // results wait for each other; a request of up to 512 positions is one unit and has none.  Where even 2048 positions make
    // more blocks than that, 1024, which balance requests of different lengths better.  us of one layer, eight KV heads of four
    // query heads, units of 128 / 256 / 512 / 1024 / 2048: one request of 2945 positions 10.1 / 9.1 / 11.0 / 15.4 / 23.3, of 300
    // 8.7 / 8.8 / 8.2, of 1000 9.3 / 10.1 / 12.3 (so 128 up to 64 positions a block), of 10000 19.7 / 15.4 / 13.7 / 16.2 / 24.7, of 32768 48.4 / 33.4 / 27.9 / 25.6 / 25.5;
    // four of 10368 48.6 / 35.3 / 31.9 / 32.7 / 29.0; 24 of up to 10369 (FP8) 99.5 / 67.3 / 53.7 / 54.7 / 57.3.  (The same input again
    // and again; all but the last of plain rows of 128.  The rule counts positions: shorter rows, of codes or of 64 numbers, have the same units.)
    const int64_t per_block = rows * c.chunk.max_len / 192;
    f.unit_shift = per_block > 64 ? 8 : 7;
    while (f.unit_shift < 11 && per_block * 10 > (int64_t)14 << f.unit_shift) ++f.unit_shift;
    if (per_block * 10 > (int64_t)14 << 11) f.unit_shift = 10;
    if (c.chunk.max_len <= 512) f.unit_shift = 9;
    if (f.unit_shift > ps_shift + 6) f.unit_shift = ps_shift + 6;          // a wave holds the page ids of a unit, a lane each
    f.n_units = (c.chunk.max_len + (1 << f.unit_shift) - 1) >> f.unit_shift;
    const int cols = c.s.Hq / c.s.Hkv * c.chunk.max_new;
    f.part_floats = (cols * (c.s.d + 2) + 3) & ~3;
    f.bytes = f.n_units > 1 ? (size_t)rows * f.n_units * f.part_floats * sizeof(float) : 0;
    return f;
}

template <int D, int FMT>
void launch(const PagesAttnParams& a, int cols, hipStream_t st) {
    const int rows = a.p.n_layers * a.p.B * a.p.Hkv;
    const dim3 grid(a.p.Hkv, a.p.n_layers * a.p.B, a.n_units);
    if (cols <= 16) {
        pages_few_kernel<D, FMT, 1><<<grid, kThreads, 0, st>>>(a);
        return;
    }
    if (cols <= 32) pages_few_kernel<D, FMT, 2><<<grid, kThreads, 0, st>>>(a);
    else if constexpr (FMT != kPageF32) {
        if (cols <= 48) pages_few_kernel<D, FMT, 3><<<grid, kThreads, 0, st>>>(a);
        else pages_few_kernel<D, FMT, 4><<<grid, kThreads, 0, st>>>(a);
    }
    if (a.n_units > 1) pages_few_merge_kernel<typename PageRow<FMT>::T, D><<<dim3((cols * (D / 4) + 255) / 256, rows), 256, 0, st>>>(a);
}

}  // namespace

bool pages_few_supported(const PagesCall& c) { return (int64_t)(c.s.Hq / c.s.Hkv) * c.chunk.max_new <= (c.s.dtype == VLC_F32 ? 32 : 64); }
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
