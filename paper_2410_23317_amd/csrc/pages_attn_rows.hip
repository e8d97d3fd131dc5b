// Attention of a chunk over the pages of its request (gfx950, v_mfma_f32_32x32x16_bf16): the chunks of a prompt, more than 64
// query rows per KV head.
//
// A block takes up to 256 query rows of one KV head (rows token after token, the g heads of a token next to each other, so that a
// block needs few masked keys) and walks the keys; a wave owns RB blocks of 32 rows.  As in the window attention, S^T = K Q^T
// per step of 32 keys, so the 16 logits a lane holds belong to ONE query row, the softmax stays in the lane, the
// probabilities are the second operand of O^T += V^T P^T as they are, and V's transpose is the LDS read.
//
// What decides the speed is that matrix and vector instructions always have each other to run beside (a wave's own ones do: a
// matrix instruction occupies its unit for 32 cycles and the issue for 8).  Inside a wave, step j turns its logits into
// probabilities while the products K Q^T of step j + 1 run, then multiplies V while it takes the maxima of the logits of step
// j + 1.  Between waves, every SIMD holds two, which cover each other's waits: eight waves of 32 rows share the keys of a
// block of 128-wide heads, and two blocks of four waves of 64 rows fit a compute unit with 64-wide ones.  2048 tokens of 32
// heads over 32768 keys, us (TFLOP/s): d = 128 one wave per SIMD with 64 rows 1028, two with 32 rows 993 (1073); d = 64 one 811,
// two 588 (905).  A large bf16 matrix product reached 1256 TFLOP/s on that card (1308 on another); neither more lookahead, other wave
// priorities nor none of the lookahead moves the 993 by 1 %.  With 64-wide heads a logit is worth half the products, and the vector unit is
// what is busy: 68 % of the cycles, the matrix unit 44 (d = 128: 50 and 55).  FP8 pages 1144, int8 about 1190 (d = 64: 781 and 799): the
// codes' expansion, two scales, and the sum over rounded weights (see step; 5 % of the time with d = 128, 13 % with 64).  The eight-wave
// instances for codes keep two registers in scratch, 12 bytes a lane, from before the first loop to between the two.
//
// A row's weights are relative to m, which starts as the maximum of its first 32 keys and is raised only when a logit (base 2)
// exceeds it by more than kSlack: the weights are then at most 2^kSlack instead of 1, and the accumulators are rescaled a few times per
// row instead of at every new maximum.  The rescaling stands outside the loop over the steps; inside, the accumulators had two
// definitions and were copied between registers at every step (1372 us instead of 1050).
//
// Keys come in stages of 64 through a ring of four LDS buffers: plain rows go from memory to LDS without registers, requested
// three stages ahead; codes are fetched into registers, expanded to bf16 (exactly) on their way into LDS, and their scales
// multiply the logits and the probabilities.  Probabilities are rounded to bf16 for the product with V, a half step of 2^-8
// each; the sums are fp32, of the probabilities themselves for plain rows and of the rounded ones for codes.  16-byte pieces of a
// row lie at swizzled places, so that neither the reads of K (16 rows, one piece) nor the transposing reads of V (four rows, 64
// bytes) meet on a bank (counted: no conflicts; the writes of expanded codes have some, 3 % of the cycles).
#include "pages_rows.h"
#include "score_tiles.h"

namespace vlc {
namespace {

using tiles::acc_row;

constexpr int kStage = 64;             // keys per stage
constexpr int kRing = 4;
constexpr float kSlack = 10.f;

typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;
typedef __attribute__((address_space(3))) void lds_void_t;
__device__ __forceinline__ uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)(lds_void_t*)p; }

// 64 lanes x 16 bytes from memory to 1024 contiguous bytes of LDS.  The hardware takes LDS's address from m0.
__device__ __forceinline__ void load_to_lds(uint32_t lds, const char* base, uint32_t offset) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(lds), "v"(offset), "s"(base) : "memory");
}

// Place of 16-byte piece p of key row r of a stage, in pieces.
template <int D> __device__ __forceinline__ int k_place(int r, int p) {
    return r * (D / 8) + (D == 128 ? p ^ (r & 15) : p ^ ((r >> 1) & 7));
}
template <int D> __device__ __forceinline__ int v_place(int r, int p) {
    return r * (D / 8) + (D == 128 ? p ^ ((r & 3) << 2) : p ^ (((r >> 1) & 1) << 2));
}

__device__ __forceinline__ float max_across_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// STATS: pages of codes keep the plain sum of the weights too, which only calls that ask for statistics pay (d = 64, two blocks of
// rows a wave, 42 registers in scratch: int8 905 us instead of 799; one block a wave 1000 and more).
template <int D, int FMT, int RB, int W, bool STATS>
__global__ __launch_bounds__(W * 64, 2) void pages_rows_kernel(PagesRowsParams ra) {
    constexpr int kWaves = W, kThreads = W * 64, kRows = 32 * RB * W;
    constexpr bool Q8 = PageRow<FMT>::kQuantised;
    constexpr int KS = D / 16, DT = D / 32, PPR = D / 8;       // k-steps of K Q^T, 32-wide tiles of d, pieces per row
    constexpr int ROWB = D * PageRow<FMT>::kElemBytes;         // bytes of a row in a page
    constexpr int LOADS = 2 * kStage * PPR / kThreads;         // 16-byte pieces of K and V per thread and stage (plain rows)
    constexpr bool ZM = Q8 && (D == 128 || STATS);             // who adds the rounded weights up: the matrix unit, or the vector unit (see step)
    constexpr int kSecond = kStage + 8;                        // where the second parts start: on other banks than the first
    __shared__ __align__(1024) uint4 sK[kRing][kStage * PPR];
    __shared__ __align__(1024) uint4 sV[kRing][kStage * PPR];
    __shared__ __align__(16) float sKs[Q8 ? kRing : 1][kStage], sVs[Q8 ? kRing : 1][kStage], sVi[Q8 ? kRing : 1][ZM ? kStage + 4 : kStage];
    // (scales; sVi: 1 / V's as fp32, or all first and all second parts)
    __shared__ int sBad[2];            // first and last stage in which numbers of V were replaced by 0
    const PagesAttnParams& a = ra.a;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), half = lane >> 5;

    // ---- which rows: the blocks of a KV head on one XCD (the hardware deals consecutive blocks to the 8 XCDs in turn), so that
    // they share its L2, and the row blocks with the most keys first
    const int per_group = ra.row_blocks * a.n_units;
    int group, inner;
    {
        const int id = blockIdx.x, x = id & 7;
        if ((ra.groups & 7) == 0) { group = x + 8 * ((id >> 3) / per_group); inner = (id >> 3) % per_group; }
        else { group = id % ra.groups; inner = id / ra.groups; }
    }
    const int rblk = ra.row_blocks - 1 - inner / a.n_units, split = inner % a.n_units;
    const int h = group % a.p.Hkv, lb = group / a.p.Hkv, b = lb % a.p.B, l = lb / a.p.B;
    const ChunkLen len = chunk_len(a.p, b);
    if (!len.ok && l == 0 && h == 0 && inner == 0 && tid == 0) report_lens(a.p, b);
    const int g = a.p.g, rows = g * len.c, first_new = len.n - len.c;
    const int r0 = rblk * kRows;                          // the block's rows: r0 + 32 RB wave + 32 rb + lane % 32
    if (r0 >= rows) return;
    const int first_last = first_new + r0 / g;                 // last key of the block's first row, and of its last row
    const int last_last = first_new + (min(r0 + kRows, rows) - 1) / g;
    const int st0 = split * ra.steps_per_split, st1 = min(last_last / kStage + 1, st0 + ra.steps_per_split);
    const int st_masked = (first_last + 1) / kStage;           // first stage that some row does not see to its end

    // ---- stages: page ids of 64 pages in a register, a lane each
    const int64_t head0 = (int64_t)(a.p.layer_begin + l) * a.p.n_pages * a.p.Hkv + h;
    const int last_page = (len.n - 1) >> a.p.ps_shift;
    int id_base = INT32_MIN, ids = 0;
    auto need_ids = [&](int key0) {
        const int p0 = key0 >> a.p.ps_shift;
        if (p0 + ((kStage - 1) >> a.p.ps_shift) < id_base + 64 && id_base >= 0) return;
        id_base = p0;
        const int page = p0 + lane;
        int v = page <= last_page ? a.p.table[(int64_t)b * a.p.max_pages + page] : 0;
        if ((uint32_t)v >= (uint32_t)a.p.n_pages) {
            set_sticky(a.p.status, VLC_ERR_INVALID_ARG, b, kStickyPage, v);
            v = 0;
        }
        ids = v;
    };
    if (st0 < st1) need_ids(st0 * kStage);                     // in front of the requests for Q: what K and V wait for
    const float scale = attn_scale(a, l, D), c = tiles::exp_scale(scale);
    bf16x8_t qf[RB][KS];
    int last[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int r = min(r0 + 32 * (RB * wave + rb) + (lane & 31), rows - 1);         // rows beyond the last repeat it
        last[rb] = first_new + r / g;
        const char* q = a.q.at(l, b, h * g + r % g, r / g) + half * 16;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) qf[rb][ks] = *reinterpret_cast<const bf16x8_t*>(q + ks * 32);
    }
    // the products stand for the logits only where the scale is positive: Q takes its sign, and is 0 for a scale of 0
    if (!(scale > 0.f)) {
        const uint32_t flip = scale < 0.f ? 0x80008000u : 0u, keep = scale == 0.f ? 0u : 0xffffffffu;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                uint4 w = __builtin_bit_cast(uint4, qf[rb][ks]);
                w = make_uint4((w.x ^ flip) & keep, (w.y ^ flip) & keep, (w.z ^ flip) & keep, (w.w ^ flip) & keep);
                qf[rb][ks] = __builtin_bit_cast(bf16x8_t, w);
            }
    }
    // what the weights are relative to, their sum, the largest logit, and how far a logit may lie above m (exponent domain)
    float m[RB], z[RB], peak[RB], slack[RB];
    f32x16_t zr[ZM ? RB : 1];          // elements 0 and 1: the sum of the rounded weights over V's scales, in two parts
    f32x16_t o[RB][DT];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        m[rb] = z[rb] = 0.f;
        if constexpr (ZM) zr[rb] = f32x16_t{0};
        peak[rb] = slack[rb] = kNoMax;          // any logit sets the first m
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[rb][dt] = f32x16_t{0};
    }

    // first row (of page_slots) of key's page; keys behind the last one of the request are in its last page, or in page 0
    auto row_of_uniform = [&](int key) {
        const int v = __builtin_amdgcn_readlane(ids, (key >> a.p.ps_shift) - id_base);
        return ((head0 + (int64_t)v * a.p.Hkv) << a.p.ps_shift) + (key & ((1 << a.p.ps_shift) - 1));
    };
    // plain rows: an instruction of a wave moves 64 / PPR rows
    constexpr int RPI = 64 / PPR;
    auto request_plain = [&](int st) {
        const int key0 = st * kStage;
        need_ids(key0);
#pragma unroll
        for (int u = 0; u < LOADS / 2; ++u) {
            const int r = (u * kWaves + wave) * RPI;           // first row of the instruction (wave-uniform); its rows share a page
            const int64_t row = row_of_uniform(key0 + r);
            const int lr = r + lane / PPR, place = lane % PPR; // the lane's row, and the place in it that it fills
            const uint32_t kp = k_place<D>(lr, place) % PPR, vp = v_place<D>(lr, place) % PPR;  // (the swizzle is its own inverse)
            load_to_lds(lds_address(&sK[st & (kRing - 1)][r * PPR]), a.p.k + row * ROWB, (lane / PPR) * ROWB + kp * 16);
            load_to_lds(lds_address(&sV[st & (kRing - 1)][r * PPR]), a.p.v + row * ROWB, (lane / PPR) * ROWB + vp * 16);
        }
    };
    // codes: a thread fetches 16 at a time
    constexpr int CPR = D / 16, CODE_LOADS = kStage * CPR / kThreads > 0 ? kStage * CPR / kThreads : 1;
    struct Codes {
        uint4 k[Q8 ? CODE_LOADS : 1], v[Q8 ? CODE_LOADS : 1];
        float scale;
    } codes;
    auto row_of_lane = [&](int key) {
        const int v = __shfl(ids, (key >> a.p.ps_shift) - id_base, kWave);
        return ((head0 + (int64_t)v * a.p.Hkv) << a.p.ps_shift) + (key & ((1 << a.p.ps_shift) - 1));
    };
    auto request_codes = [&](int st, Codes& c8) {
        const int key0 = st * kStage;
        need_ids(key0);
#pragma unroll
        for (int u = 0; u < CODE_LOADS; ++u) {
            const int x = tid + kThreads * u, r = x / CPR, piece = x % CPR;
            const int64_t row = row_of_lane(key0 + r);
            c8.k[u] = *reinterpret_cast<const uint4*>(a.p.k + row * ROWB + piece * 16);
            c8.v[u] = *reinterpret_cast<const uint4*>(a.p.v + row * ROWB + piece * 16);
        }
        const int64_t row = row_of_lane(key0 + lane);          // waves 0 and 1: the scales
        if (wave < 2) c8.scale = (wave ? a.p.v_scale : a.p.k_scale)[row];
    };
    auto store_codes = [&](int st, const Codes& c8) {
        const int key0 = st * kStage, buf = st & (kRing - 1);
#pragma unroll
        for (int u = 0; u < CODE_LOADS; ++u) {
            const int x = tid + kThreads * u, r = x / CPR, piece = x % CPR;
            const bool there = key0 + r < len.n;               // stale codes may stand for NaN
            const uint4 v = there ? c8.v[u] : make_uint4(0, 0, 0, 0);
            sK[buf][k_place<D>(r, 2 * piece)] = codes_to_bf16<FMT>(make_uint2(c8.k[u].x, c8.k[u].y));
            sK[buf][k_place<D>(r, 2 * piece + 1)] = codes_to_bf16<FMT>(make_uint2(c8.k[u].z, c8.k[u].w));
            sV[buf][v_place<D>(r, 2 * piece)] = codes_to_bf16<FMT>(make_uint2(v.x, v.y));
            sV[buf][v_place<D>(r, 2 * piece + 1)] = codes_to_bf16<FMT>(make_uint2(v.z, v.w));
        }
        // V's scales that are no normal number count as the smallest, so that their reciprocals are numbers (a NaN stays)
        const float vs = c8.scale < 0x1p-126f ? 0x1p-126f : c8.scale;
        if (wave == 0) sKs[buf][lane] = c8.scale * c;
        if (wave == 1) {
            const float inv = vs == vs ? 1.f / vs : 0.f;       // of a NaN: where the key is seen, the weight is NaN already
            sVs[buf][lane] = vs;
            if constexpr (ZM) {
                const __bf16 first = (__bf16)inv;
                __bf16* parts = reinterpret_cast<__bf16*>(sVi[buf]);
                parts[lane] = first;
                parts[kSecond + lane] = (__bf16)(inv - (float)first);
            } else {
                sVi[buf][lane] = inv;
            }
        }
    };

    auto barrier = [&]() {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    // V of a stage that some row does not see to its end: numbers that are not finite become 0 (0 times them is no 0)
    auto clean_v = [&](int st) {
        if constexpr (!Q8) {
            bool bad = false;
#pragma unroll
            for (int u = 0; u < LOADS / 2; ++u) {
                uint4& w = sV[st & (kRing - 1)][tid + kThreads * u];
                const uint4 x = w, f = make_uint4(finite_pair(x.x), finite_pair(x.y), finite_pair(x.z), finite_pair(x.w));
                if (x.x != f.x || x.y != f.y || x.z != f.z || x.w != f.w) { w = f; bad = true; }
            }
            if (bad) { atomicMin(&sBad[0], st); atomicMax(&sBad[1], st); }
            barrier();
        }
    };

    // LDS places of the lane's fragments in step 0 of the ring; step j (32 keys) lies (j mod 2 kRing) kStep bytes behind
    constexpr int kStep = 32 * PPR * 16;
    uint32_t k_at[KS], v_at[DT];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) k_at[ks] = lds_address(&sK[0][k_place<D>(lane & 31, 2 * ks + half)]);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
        // lane (l % 32) owns row 32 dt + l % 32 of V^T, lane half l / 32 keys 16 sp + 4 half + {0..3, 8..11}: the order of the
        // accumulators.  ds_read_b64_tr_b16: lane 4 i + e of 16 names 4 numbers of key i, lane x is given number x of the 4 keys
        const int key = 4 * half + ((lane >> 2) & 3), el = dt * 32 + (lane & 16) + (lane & 3) * 4;
        v_at[dt] = lds_address(&sV[0][v_place<D>(key, el >> 3)]) + (el & 4) * 2;
    }
    auto step_offset = [&](int j) { return (uint32_t)((j & (2 * kRing - 1)) * kStep); };
    typedef const __attribute__((address_space(3))) u32x4_t* LdsPieces;
    bf16x8_t kf[KS];
    auto load_k = [&](int j) {         // fragments of the keys of step j; behind the last one: of whatever the ring holds there
        const uint32_t off = step_offset(j);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) kf[ks] = __builtin_bit_cast(bf16x8_t, *(LdsPieces)(k_at[ks] + off));
    };
    auto products = [&](f32x16_t (&acc)[RB]) {                         // logits of the keys in kf
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) acc[rb] = f32x16_t{0};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) acc[rb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[ks], qf[rb][ks], acc[rb], 0, 0, 0);
    };
    auto scales_of = [&](const float* stage0, int j, float (&f)[16]) { // of the keys whose logits the lane holds
        const float* at = stage0 + (j & (2 * kRing - 1)) * 32 + 4 * half;
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
            const float4 x = *reinterpret_cast<const float4*>(at + 8 * q4);
            f[4 * q4] = x.x; f[4 * q4 + 1] = x.y; f[4 * q4 + 2] = x.z; f[4 * q4 + 3] = x.w;
        }
    };
    // The products become logits in the exponent domain, relative to m (codes: times the key's scale).  Masked: keys that a row
    // does not see.  Returns whether m has to be raised.
    float top[RB];                     // largest of the step
    auto finish_logits = [&](auto masked, int j, f32x16_t (&acc)[RB]) {
        constexpr bool MASKED = decltype(masked)::value;
        float f[16];
        if constexpr (Q8) scales_of(&sKs[0][0], j, f);
        bool raise = false;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                acc[rb][i] = fmaf(acc[rb][i], Q8 ? f[i] : c, -m[rb]);
                if constexpr (MASKED) acc[rb][i] = 32 * j + acc_row(i, lane) <= last[rb] ? acc[rb][i] : -INFINITY;
            }
            float t = acc[rb][0];
#pragma unroll
            for (int i = 1; i < 16; ++i) t = fmaxf(t, acc[rb][i]);
            top[rb] = t;
            peak[rb] = fmaxf(peak[rb], t + m[rb]);
            raise |= t > slack[rb];
        }
        return __any(raise) != 0;
    };
    auto raise_max = [&](f32x16_t (&s)[RB]) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            const float t = max_across_halves(top[rb]);
            const bool first = slack[rb] < 0.f;
            const float by = t > 0.f || (first && t > -INFINITY) ? t : 0.f, corr = first ? 1.f : exp2_fast(-by);
            if (t > -INFINITY) slack[rb] = kSlack;
            m[rb] += by;
            z[rb] *= corr;
            if constexpr (ZM) { zr[rb][0] *= corr; zr[rb][1] *= corr; }
            s[rb] -= by;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) o[rb][dt] *= corr;
        }
    };
    // Step j, whose logits are in s: its probabilities beside the products of step j + 1 (which take their place), its outputs beside the maxima of those.
    auto step = [&](auto masked, auto final, int j, f32x16_t (&s)[RB]) {
        constexpr bool MASKED = decltype(masked)::value, LAST = decltype(final)::value;
        f32x16_t sn[RB];
        if constexpr (!LAST) products(sn);
        bf16x8_t pf[RB][2];
        // Codes: a weight takes V's scale before it is rounded to bf16, and what the outputs are divided by is the sum of the weights
        // as they were rounded, over the scales: where one key has nearly all of a row, as often, its rounding then cancels.  (Plain
        // rows: such a key's weight is near 1, which bf16 has.)  2-norm of the outputs' error in an int8 window, in that of their
        // own rounding to bf16: 1.04 to 1.25 over four random inputs, with the plain sum up to 1.53.  The sum is another product
        // of the weights, with 1 / scale as the sum of two bf16 numbers in the place of V (FP8, 2048 tokens over 32768: 1191 -> 1144 us),
        // but for calls over 64-wide heads without statistics, where its 32 registers do not fit (770 -> 804): there the vector unit adds.
        float f[16] = {}, inv[16] = {};
        if constexpr (Q8) scales_of(&sVs[0][0], j, f);
        if constexpr (Q8 && !ZM) scales_of(&sVi[0][0], j, inv);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            float zs[2] = {0.f, 0.f};
            u32x4_t w4[2];
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                float p[2] = {exp2_fast(s[rb][i]), exp2_fast(s[rb][i + 1])}, to_p[2] = {inv[i], inv[i + 1]};
                if constexpr (!Q8 || STATS) {
                    zs[0] += p[0];
                    zs[1] += p[1];
                }
                if constexpr (Q8) {
                    p[0] *= f[i];
                    p[1] *= f[i + 1];
                    if constexpr (MASKED) {            // any scale stands behind keys that are not seen
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            const bool seen = 32 * j + acc_row(i + x, lane) <= last[rb];
                            p[x] = seen ? p[x] : 0.f;
                            to_p[x] = seen ? to_p[x] : 0.f;
                        }
                    }
                }
                typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
                const uint32_t w = __builtin_bit_cast(uint32_t, bf16x2_t{(__bf16)p[0], (__bf16)p[1]});
                w4[i >> 3][(i >> 1) & 3] = w;
                if constexpr (Q8 && !ZM) {
                    zs[0] = fmaf(bf16_lo(w), to_p[0], zs[0]);
                    zs[1] = fmaf(bf16_hi(w), to_p[1], zs[1]);
                }
            }
            pf[rb][0] = __builtin_bit_cast(bf16x8_t, w4[0]);
            pf[rb][1] = __builtin_bit_cast(bf16x8_t, w4[1]);
            z[rb] += zs[0] + zs[1];
            asm volatile("" : "+v"(z[rb]));    // here, beside the products, not behind the step
        }
        if constexpr (!LAST) load_k(j + 2);
        const uint32_t off = step_offset(j);
#pragma unroll
        for (int sp = 0; sp < 2; ++sp)
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                const lds_s16x4_t* at = (const lds_s16x4_t*)(v_at[dt] + off);          // rows of PPR 16-byte pieces
                const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(at + 16 * sp * PPR * 2));
                const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(at + (16 * sp + 8) * PPR * 2));
                const uint2 x = __builtin_bit_cast(uint2, lo), y = __builtin_bit_cast(uint2, hi);
                const bf16x8_t vf = __builtin_bit_cast(bf16x8_t, make_uint4(x.x, x.y, y.x, y.y));
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) o[rb][dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[rb][sp], o[rb][dt], 0, 0, 0);
            }
        if constexpr (ZM) {
            // rows of the first operand: the first parts of 1 / scale (even ones) and the second parts, in the order of the keys of pf
            const uint16_t* at = reinterpret_cast<const uint16_t*>(sVi[(j >> 1) & (kRing - 1)]) + (lane & 1) * kSecond + (j & 1) * 32 + 4 * half;
#pragma unroll
            for (int sp = 0; sp < 2; ++sp) {
                const uint2 x = *reinterpret_cast<const uint2*>(at + 16 * sp), y = *reinterpret_cast<const uint2*>(at + 16 * sp + 8);
                const bf16x8_t parts = __builtin_bit_cast(bf16x8_t, make_uint4(x.x, x.y, y.x, y.y));
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) zr[rb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(parts, pf[rb][sp], zr[rb], 0, 0, 0);
            }
        }
        if constexpr (LAST) return false;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) asm volatile("" : "+v"(sn[rb]));       // out of the accumulation registers once, not for each use
        const bool raise = finish_logits(masked, j + 1, sn);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) s[rb] = sn[rb];
        return raise;
    };
    auto boundary = [&](int st) {      // makes stage st + 1 visible, requests another
        if constexpr (!Q8) {
            if (st + 2 < st1) asm volatile("s_waitcnt vmcnt(%0)" : : "n"(LOADS) : "memory");
            else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            barrier();
            if (st + 3 < st1) request_plain(st + 3);
        } else {
            if (st + 2 < st1) store_codes(st + 2, codes);
            barrier();
            if (st + 3 < st1) request_codes(st + 3, codes);
        }
    };

    if (tid < 2) sBad[tid] = tid ? -1 : INT32_MAX;
    if (st0 < st1) {
        if constexpr (!Q8) {
            request_plain(st0);
            if (st0 + 1 < st1) request_plain(st0 + 1);
            if (st0 + 2 < st1) request_plain(st0 + 2);
            if (st0 + 2 < st1) asm volatile("s_waitcnt vmcnt(%0)" : : "n"(2 * LOADS) : "memory");
            else if (st0 + 1 < st1) asm volatile("s_waitcnt vmcnt(%0)" : : "n"(LOADS) : "memory");
            else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        } else {
            Codes first, second;
            request_codes(st0, first);
            if (st0 + 1 < st1) request_codes(st0 + 1, second);
            if (st0 + 2 < st1) request_codes(st0 + 2, codes);
            store_codes(st0, first);
            if (st0 + 1 < st1) store_codes(st0 + 1, second);
        }
        barrier();
        if (st0 >= st_masked) clean_v(st0);
        constexpr auto yes = std::true_type{};
        constexpr auto no = std::false_type{};
        f32x16_t s[RB];
        int j = 2 * st0;
        load_k(j);
        products(s);
        load_k(j + 1);
        if (finish_logits(yes, j, s)) raise_max(s);
        // Steps up to jstop.  Raising the maximum stands outside the loop over the steps: inside, the accumulators would have two
        // definitions to choose from, and be copied at every step.
        auto run = [&](auto masked, int jstop) {
#pragma unroll 1
            while (j < jstop) {
                bool raise;
#pragma unroll 1
                do {
                    if (!(j & 1) && (j >> 1) + 1 < st1) {      // a step before the stage's first fragments are read
                        boundary(j >> 1);
                        if constexpr (decltype(masked)::value)
                            if ((j >> 1) + 1 >= st_masked) clean_v((j >> 1) + 1);
                    }
                    raise = step(masked, no, j, s);
                    ++j;
                } while (!raise && j < jstop);
                if (raise) raise_max(s);
            }
        };
        run(no, min(2 * st1, 2 * st_masked) - 2);               // these steps, and what they look ahead to, are seen by all rows
        run(yes, 2 * st1 - 1);
        step(yes, yes, j, s);
    }
    barrier();
    const int64_t prow0 = ((int64_t)group * a.n_units + split) * ((int64_t)g * a.p.max_new);
    // Through LDS, so that memory sees whole rows: a lane holds 4 neighbouring numbers of d at a time, the wave 32 rows of them.
    constexpr int PIECES = D / 4;                              // 16-byte pieces of a row of fp32 numbers
    f32x4_t* sO = reinterpret_cast<f32x4_t*>(wave < W / 2 ? &sK[0][0] : &sV[0][0]) + wave % (W / 2) * (32 * PIECES);
    static_assert(sizeof(sK) >= W / 2 * 32 * PIECES * 16, "the rows of half the waves in each half of the ring");
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int first = r0 + 32 * (RB * wave + rb), r = first + (lane & 31);
        const float top_m = max_across_halves(peak[rb]), to_top = top_m > kNoMax ? exp2_fast(m[rb] - top_m) : 1.f;     // relative to the largest logit from here on
        const float zs = (z[rb] + __shfl_xor(z[rb], 32, kWave)) * to_top;       // the plain sum, if it was kept
        float zt = zs;                                                          // what the outputs are divided by
        if constexpr (ZM) zt = (zr[rb][0] + zr[rb][1]) * to_top;
        const float factor = a.n_units > 1 ? to_top : zt == 0.f ? 0.f : to_top / zt;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
                const f32x4_t x = {o[rb][dt][4 * q4], o[rb][dt][4 * q4 + 1], o[rb][dt][4 * q4 + 2], o[rb][dt][4 * q4 + 3]};
                sO[(lane & 31) * PIECES + ((dt * 8 + 2 * q4 + half) ^ (lane & (PIECES - 1)))] = x * factor;
            }
        if (half == 0 && r < rows) {
            if (a.n_units > 1) ra.part_mz[prow0 + r] = make_float4(top_m, zt, zs, 0.f);
            else if (a.stats.row_max) store_stats(a, l, b, h * g + r % g, r / g, top_m, zs);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // the wave's own writes; no other wave touches its rows
        if (a.n_units > 1) {
#pragma unroll
            for (int i = 0; i < 32 * PIECES / 64; ++i) {
                const int row = (i * 64 + lane) / PIECES, piece = lane % PIECES;
                if (first + row < rows)
                    *reinterpret_cast<f32x4_t*>(ra.part_o + (prow0 + first + row) * D + piece * 4) = sO[row * PIECES + (piece ^ (row & (PIECES - 1)))];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16 * PIECES / 64; ++i) {
                const int row = (i * 64 + lane) / PPR, piece = lane % PPR * 2, rr = first + row;
                const f32x4_t x = sO[row * PIECES + (piece ^ (row & (PIECES - 1)))], y = sO[row * PIECES + ((piece + 1) ^ (row & (PIECES - 1)))];
                const bf16x8_t w = {(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3], (__bf16)y[0], (__bf16)y[1], (__bf16)y[2], (__bf16)y[3]};
                if (rr < rows) *reinterpret_cast<bf16x8_t*>(a.out.at(l, b, h * g + rr % g, rr / g) + piece * 8) = w;
            }
        }
        asm volatile("" ::: "memory");
    }
    // What is not finite in V reaches the rows that see it: added to what was just stored, from memory, a number at a time.
    if (!Q8 && sBad[0] < st1) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        const int t0 = sBad[0] * kStage, t1 = sBad[1] * kStage + kStage - 1;
        for (int x = tid; x < min(kRows, rows - r0) * D; x += kThreads) {
            const int r = r0 + x / D, d = x % D;
            float add = 0.f;
            bool any = false;
            for (int t = t0; t <= min(first_new + r / g, t1); ++t) {
                int page = a.p.table[(int64_t)b * a.p.max_pages + (t >> a.p.ps_shift)];
                if ((uint32_t)page >= (uint32_t)a.p.n_pages) page = 0;
                const float f = Elem<bf16_t>::load((const bf16_t*)a.p.v + (page_row0(a.p, a.p.layer_begin + l, page, h) + (t & ((1 << a.p.ps_shift) - 1))) * D + d);
                if (!is_finite(f)) { add += f; any = true; }
            }
            if (!any) continue;
            if (a.n_units == 1) {
                bf16_t* out = (bf16_t*)a.out.at(l, b, h * g + r % g, r / g) + d;
                *reinterpret_cast<__bf16*>(out) = (__bf16)(Elem<bf16_t>::load(out) + add);
            } else {
                ra.part_o[(prow0 + r) * D + d] += add;
            }
        }
    }
}

struct RowsPlan { int rb, row_blocks, splits, steps_per_split; int64_t groups, rows; size_t o_bytes, bytes; };

RowsPlan plan(const PagesCall& c) {
    RowsPlan p;
    const int g = c.s.Hq / c.s.Hkv;
    p.groups = (int64_t)c.n_layers * c.chunk.B * c.s.Hkv;
    p.rows = (int64_t)g * c.chunk.max_new;
    p.rb = p.rows <= 128 ? 1 : 2;
    p.row_blocks = (int)((p.rows + 128 * p.rb - 1) / (128 * p.rb));
    const int stages = (c.chunk.max_len + kStage - 1) / kStage;
    const int64_t blocks = p.groups * p.row_blocks;
    // A block fills a compute unit (d = 64: half of one); a launch takes as many rounds as it has blocks per 256 (512).  Splitting
    // the keys fills the rounds, at the price of a start and an end per block (8 us; a stage takes 2.1 of 256 rows, 1.4 of 128)
    // and of a second launch through which the partial results go (4 us, and their bytes to memory and back).
    const int resident = c.s.d == 64 ? 512 : 256;
    const double stage_us = (p.rb == 1 ? 1.4 : 2.1) * (c.s.d == 64 ? 1.1 : 1.0);
    int best = 1;
    double least = 1e300;
    for (int ns = 1; ns <= 64 && ns * 2 <= stages + 1 && (ns == 1 || blocks * ns <= 8192); ++ns) {
        const int per = (stages + ns - 1) / ns;
        double us = (double)((blocks * ns + resident - 1) / resident) * (per * stage_us + 8);
        if (ns > 1) us += 4 + (double)p.groups * p.rows * ns * c.s.d * 8 / 5.0e6;
        if (us < least) { least = us; best = ns; }
    }
    p.steps_per_split = (stages + best - 1) / best;
    p.splits = (stages + p.steps_per_split - 1) / p.steps_per_split;
    const size_t n = (size_t)p.groups * p.splits * p.rows;
    p.o_bytes = pages_partials_o_bytes(n, c.s.d);
    p.bytes = p.splits > 1 ? p.o_bytes + n * sizeof(float4) : 0;
    return p;
}

template <int D, int FMT, bool STATS>
void launch_blocks(const PagesRowsParams& ra, int rb, hipStream_t st) {
    const unsigned grid = (unsigned)ra.groups * ra.row_blocks * ra.a.n_units;
    if (rb == 1) pages_rows_kernel<D, FMT, 1, 4, STATS><<<grid, 256, 0, st>>>(ra);
    else if constexpr (D == 128) pages_rows_kernel<D, FMT, 1, 8, STATS><<<grid, 512, 0, st>>>(ra);
    else pages_rows_kernel<D, FMT, 2, 4, STATS><<<grid, 256, 0, st>>>(ra);
}
template <int D, int FMT>
void launch(const PagesRowsParams& ra, int rb, hipStream_t st) {
    if constexpr (PageRow<FMT>::kQuantised) {
        if (ra.a.stats.row_max) launch_blocks<D, FMT, true>(ra, rb, st);
        else launch_blocks<D, FMT, false>(ra, rb, st);
    } else {
        launch_blocks<D, FMT, false>(ra, rb, st);
    }
    if (ra.a.n_units > 1) launch_pages_rows_merge<bf16_t, D>(ra, st);
}

}  // namespace

size_t pages_rows_workspace_bytes(const PagesCall& c) { return plan(c).bytes; }

hipError_t launch_pages_rows(const PagesAttn& c) {
    const RowsPlan p = plan(c.c);
    PagesRowsParams ra;
    ra.a = pages_attn_params(c);
    ra.a.n_units = p.splits;
    ra.row_blocks = p.row_blocks; ra.groups = (int)p.groups; ra.steps_per_split = p.steps_per_split;
    ra.part_o = (float*)c.workspace;
    ra.part_mz = (float4*)((char*)c.workspace + p.o_bytes);
    const bool wide = c.c.s.d == 128;
    switch (page_format(c.c.s)) {
        case kPageBf16: wide ? launch<128, kPageBf16>(ra, p.rb, c.c.stream) : launch<64, kPageBf16>(ra, p.rb, c.c.stream); break;
        case kPageFp8: wide ? launch<128, kPageFp8>(ra, p.rb, c.c.stream) : launch<64, kPageFp8>(ra, p.rb, c.c.stream); break;
        case kPageInt8: wide ? launch<128, kPageInt8>(ra, p.rb, c.c.stream) : launch<64, kPageInt8>(ra, p.rb, c.c.stream); break;
        case kPageF32: break;
    }
    return hipGetLastError();
}

}  // namespace vlc
