// Attention of a chunk over the pages of its request for fp32 storage (gfx950, v_mfma_f32_32x32x2_f32: full fp32 products): more
// than 32 query rows per KV head.
//
// Bound by the matrix cores, which multiply fp32 at a sixteenth of the bf16 rate: 64 cycles an instruction leave room for
// everything else.  A block of four waves takes 128 rows (token after token, a token's heads next to each other), a wave 32 of
// them.  S^T = K Q^T per 32 keys: a lane's 16 logits belong to one query row, and they are the second operand of
// O^T += V^T P^T as they are: instruction i of a tile multiplies keys 8 (i / 4) + 4 half + i % 4, which is the order the
// accumulators have.  K goes through LDS with rows of D + 4 floats, so that the 32 rows of a 16-byte read of a lane half meet
// each bank equally often; V with rows of D floats, read a number per lane, 32 neighbours.
//
// 1024 tokens of 32 heads over 4096 keys: 581 us with d = 128, 300 with 64, 103 and 100 TFLOP/s, where a large fp32 product reaches
// 151.  One LDS buffer, so two barriers a tile.  Few rows pay for 128: 35 rows of 64 (request, KV head) pairs over up to 4099 keys 176 us.
#include "pages_rows.h"
#include "score_tiles.h"

namespace vlc {
namespace {

using tiles::acc_row;

constexpr int kWaves = 4, kThreads = kWaves * 64, kRows = 32 * kWaves, kKeys = 32;

template <int D>
__global__ __launch_bounds__(kThreads, 2) void pages_rows_f32_kernel(PagesRowsParams ra) {
    constexpr int KP = D / 8, DT = D / 32, PPR = D / 4, LOADS = kKeys * PPR / kThreads, PITCH = D + 4;
    __shared__ __align__(16) float sK[kKeys * PITCH], sV[kKeys * D];
    __shared__ int sBad[2];            // first and last tile in which numbers of V were replaced by 0
    const PagesAttnParams& a = ra.a;
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), half = lane >> 5;
    const int group = blockIdx.x % ra.groups, inner = blockIdx.x / ra.groups;
    const int rblk = ra.row_blocks - 1 - inner / a.n_units, split = inner % a.n_units;      // the most keys first
    const int h = group % a.p.Hkv, lb = group / a.p.Hkv, b = lb % a.p.B, l = lb / a.p.B;
    const ChunkLen len = chunk_len(a.p, b);
    if (!len.ok && l == 0 && h == 0 && inner == 0 && tid == 0) report_lens(a.p, b);
    const int g = a.p.g, rows = g * len.c, first_new = len.n - len.c, r0 = rblk * kRows;
    if (r0 >= rows) return;
    const int first_last = first_new + r0 / g, last_last = first_new + (min(r0 + kRows, rows) - 1) / g;
    const int t0 = split * ra.steps_per_split, t1 = min(last_last / kKeys + 1, t0 + ra.steps_per_split);
    const int t_masked = (first_last + 1) / kKeys;             // first tile that some row does not see to its end

    const int r = min(r0 + 32 * wave + (lane & 31), rows - 1), last = first_new + r / g;
    const float scale = attn_scale(a, l, D), c = tiles::exp_scale(scale);
    // the products stand for the logits only where the scale is positive: Q takes its sign, and is 0 for a scale of 0
    const float sign = scale > 0.f ? 1.f : scale < 0.f ? -1.f : 0.f;
    f32x4_t qf[KP];                    // contraction index 8 s + 4 half + e of the lane's row
    const float* q = (const float*)a.q.at(l, b, h * g + r % g, r / g) + 4 * half;
#pragma unroll
    for (int s = 0; s < KP; ++s) qf[s] = *reinterpret_cast<const f32x4_t*>(q + 8 * s) * sign;
    float m = kNoMax, z = 0.f;
    f32x16_t o[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[dt] = f32x16_t{0};

    f32x4_t kr[LOADS], vr[LOADS];
    auto request = [&](int t) {
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
            const int x = tid + kThreads * u, key = min(t * kKeys + x / PPR, len.n - 1);    // keys behind the last one repeat it
            int page = a.p.table[(int64_t)b * a.p.max_pages + (key >> a.p.ps_shift)];
            if ((uint32_t)page >= (uint32_t)a.p.n_pages) {
                set_sticky(a.p.status, VLC_ERR_INVALID_ARG, b, kStickyPage, page);
                page = 0;
            }
            const int64_t at = (page_row0(a.p, a.p.layer_begin + l, page, h) + (key & ((1 << a.p.ps_shift) - 1))) * PPR + x % PPR;
            kr[u] = reinterpret_cast<const f32x4_t*>(a.p.k)[at];
            vr[u] = reinterpret_cast<const f32x4_t*>(a.p.v)[at];
        }
    };
    if (tid < 2) sBad[tid] = tid ? -1 : INT32_MAX;
    if (t0 < t1) request(t0);
#pragma unroll 1
    for (int t = t0; t < t1; ++t) {
        __syncthreads();
        bool bad = false;
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
            const int x = tid + kThreads * u;
            *reinterpret_cast<f32x4_t*>(&sK[x / PPR * PITCH + x % PPR * 4]) = kr[u];
            f32x4_t f = vr[u];
            if (t >= t_masked) {       // numbers of V that are not finite become 0 where a row does not see them (0 times them is no 0)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    bad |= !is_finite(f[e]);
                    f[e] = is_finite(f[e]) ? f[e] : 0.f;
                }
            }
            *reinterpret_cast<f32x4_t*>(&sV[x * 4]) = f;
        }
        if (bad) { atomicMin(&sBad[0], t); atomicMax(&sBad[1], t); }
        __syncthreads();
        if (t + 1 < t1) request(t + 1);
        f32x16_t s = f32x16_t{0};
#pragma unroll
        for (int ks = 0; ks < KP; ++ks) {
            const f32x4_t kf = *reinterpret_cast<const f32x4_t*>(&sK[(lane & 31) * PITCH + 8 * ks + 4 * half]);
#pragma unroll
            for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[e], qf[ks][e], s, 0, 0, 0);
        }
        if (t >= t_masked) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = t * kKeys + acc_row(i, lane) <= last ? s[i] : -INFINITY;
        }
        float top = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
        top = fmaxf(top, __shfl_xor(top, 32, kWave)) * c;
        if (__any(top > m)) {
            const float m_new = fmaxf(m, top), corr = exp2_fast(m - m_new);
            m = m_new;
            z *= corr;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) o[dt] *= corr;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) { s[i] = exp2_fast(fmaf(s[i], c, -m)); z += s[i]; }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float* v = &sV[acc_row(i, lane) * D + (lane & 31)];
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) o[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(v[32 * dt], s[i], o[dt], 0, 0, 0);
        }
    }
    __syncthreads();
    z += __shfl_xor(z, 32, kWave);
    const int64_t prow0 = ((int64_t)group * a.n_units + split) * ((int64_t)g * a.p.max_new);
    if (r0 + 32 * wave + (lane & 31) < rows) {
        const float div = a.n_units == 1 ? z : 1.f;
        float* dst = a.n_units == 1 ? (float*)a.out.at(l, b, h * g + r % g, r / g) : ra.part_o + (prow0 + r) * D;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4)
                *reinterpret_cast<float4*>(dst + dt * 32 + acc_row(4 * q4, lane)) =
                    div == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(o[dt][4 * q4] / div, o[dt][4 * q4 + 1] / div, o[dt][4 * q4 + 2] / div, o[dt][4 * q4 + 3] / div);
        if (half == 0) {
            if (a.n_units > 1) ra.part_mz[prow0 + r] = make_float4(m, z, z, 0.f);
            else if (a.stats.row_max) store_stats(a, l, b, h * g + r % g, r / g, m, z);
        }
    }
    // What is not finite in V reaches the rows that see it: added to what was just stored, from memory, a number at a time.
    if (sBad[0] < t1) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        const int k0 = sBad[0] * kKeys, k1 = sBad[1] * kKeys + kKeys - 1;
        for (int x = tid; x < min(kRows, rows - r0) * D; x += kThreads) {
            const int rr = r0 + x / D, d = x % D;
            float* dst = (a.n_units == 1 ? (float*)a.out.at(l, b, h * g + rr % g, rr / g) : ra.part_o + (prow0 + rr) * D) + d;
            for (int t = k0; t <= min(first_new + rr / g, k1); ++t) {
                int page = a.p.table[(int64_t)b * a.p.max_pages + (t >> a.p.ps_shift)];
                if ((uint32_t)page >= (uint32_t)a.p.n_pages) page = 0;
                const float f = ((const float*)a.p.v)[(page_row0(a.p, a.p.layer_begin + l, page, h) + (t & ((1 << a.p.ps_shift) - 1))) * D + d];
                if (!is_finite(f)) *dst += f;
            }
        }
    }
}

struct Plan { int row_blocks, splits, steps_per_split; int64_t groups, rows; size_t o_bytes, bytes; };

Plan plan(const PagesCall& c) {
    Plan p;
    p.groups = (int64_t)c.n_layers * c.chunk.B * c.s.Hkv;
    p.rows = (int64_t)(c.s.Hq / c.s.Hkv) * c.chunk.max_new;
    p.row_blocks = (int)((p.rows + kRows - 1) / kRows);
    const int tiles = (c.chunk.max_len + kKeys - 1) / kKeys;
    const int64_t blocks = p.groups * p.row_blocks;
    // two blocks a compute unit, two tiles at least for each
    int ns = blocks >= 512 ? 1 : (int)((512 + blocks - 1) / blocks);
    if (ns > (tiles + 1) / 2) ns = (tiles + 1) / 2;
    p.steps_per_split = (tiles + ns - 1) / ns;
    p.splits = (tiles + p.steps_per_split - 1) / p.steps_per_split;
    const size_t n = (size_t)p.groups * p.splits * p.rows;
    p.o_bytes = pages_partials_o_bytes(n, c.s.d);
    p.bytes = p.splits > 1 ? p.o_bytes + n * sizeof(float4) : 0;
    return p;
}

template <int D>
void launch(const PagesRowsParams& ra, hipStream_t st) {
    pages_rows_f32_kernel<D><<<(unsigned)ra.groups * ra.row_blocks * ra.a.n_units, kThreads, 0, st>>>(ra);
    if (ra.a.n_units > 1) launch_pages_rows_merge<float, D>(ra, st);
}

}  // namespace

size_t pages_rows_f32_workspace_bytes(const PagesCall& c) { return plan(c).bytes; }

hipError_t launch_pages_rows_f32(const PagesAttn& c) {
    const Plan p = plan(c.c);
    PagesRowsParams ra;
    ra.a = pages_attn_params(c);
    ra.a.n_units = p.splits;
    ra.row_blocks = p.row_blocks; ra.groups = (int)p.groups; ra.steps_per_split = p.steps_per_split;
    ra.part_o = (float*)c.workspace;
    ra.part_mz = (float4*)((char*)c.workspace + p.o_bytes);
    if (c.c.s.d == 128) launch<128>(ra, c.c.stream);
    else launch<64>(ra, c.c.stream);
    return hipGetLastError();
}

}  // namespace vlc
