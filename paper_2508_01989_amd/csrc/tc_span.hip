// Attention over spans, beside the mixed attention of tc_attention.h and over the same pools in 16 bits: of each row over a window of its sequence's newest tokens and its
// first ones (tc_window_attention), and of sequences that begin with the same cached tokens (tc_shared_attention), whose K and V are then read once for all of them.
//
//   span_attention_kernel  one launch for the whole batch: n_sweeps workgroups sweep K/V tiles for 256 (row, head) pairs of one KV head, or 128 in workgroups of four waves (prefill_item),
//                          the others run decode items, up to 16 (row, head) pairs of one KV head over a range of pages that a wave, or several of a workgroup, stream into registers
//   span_merge_kernel      where the tokens of a row are shared out: its output from the partial results, out = sum_i 2^(m_i - m*) o_i / sum_i 2^(m_i - m*) l_i
//
// What a row attends over is a list of pages (SpanRuns) that begins with those that need no mask, so the main loops of both branches are those of attention over everything.
//
// Sweeps are bound by the matrix cores under the power limit, decodes by the stream from memory.  One MI355X, head_dim 128, bf16 unless stated, calls back to back: 8192 tokens over a window
// of 2048 and 4 sinks, 64/8 heads, 496-533 us and 1.0-1.1 PFLOP/s (1.26 tile by tile: 1.71 us for 256 rows of every unit, from windows of 2048 to 8192; 10 us of a block are not tiles);
// 128 decodes over 2048 and 16, 40/8, half, 152-156 us and 6.5-6.7 TB/s; 2048 tokens and 64 decodes over 1000, 32/8, 68-71 us; 8 decodes over 1024 and 4, 10; 256 decodes behind 8192 shared
// tokens, 32/8, 124 us, 7 of it the combination (0.69 GB read by the counters, where every sequence for itself would read 9); 4 decodes behind 2048, 11.
#include "tc_attention.h"

namespace tc {

namespace {

struct SpanScalars {
    int Hq, Hkv, G;
    int n_sweeps, n_first, n_early;
    int waves_log2;   // log2 of the waves that share a decode item
    int max_cols;     // (row, head) pairs of a decode item at most
    int window, sinks;
    float scale_log2;
    int64_t n_rows;   // rows of partial results
    int32_t *counters;  // arrival counters, or null: partial results are combined by a second launch
    int counter_stride;
};

// Bit t: the row at position p attends over token t of page `page`.
__device__ __forceinline__ uint32_t span_bits(int page, int p, int window, int sinks) {
    const int t0 = page * kBlock;
    const auto below = [](int n) { return (1u << min(max(n, 0), kBlock)) - 1; };
    return below(p - t0 + 1) & (~below(p - window + 1 - t0) | below(sinks - t0));
}

// One wave's sweep over the places [i0, i0 + n_pg) of a span's list of pages (at most 64) for `cols` (row, head) pairs: pair j is packed row qrow + j / G, head kvh * G + j % G.
template <int D, class E, int NS>
__device__ __forceinline__ void span_decode_sweep(const AttnArgs &A, int kvh, int qrow, int cols, const int32_t *__restrict__ pages, const SpanRuns &runs, int i0, int n_pg, int pos,
                                                  int lane, f32x4 (&o)[D / 16], float &m_run, float &l_run) {
    using x8 = typename E::x8;
    constexpr int KS = D / 32;
    const int j = lane & 15, g = lane >> 4, G = A.G;
    const int my_page = pages[runs.page(i0 + min(lane, n_pg - 1))];  // lane i holds the id of page i of the range
    x8 qreg[KS];
    const int jc = min(j, cols - 1);
    const int64_t q_off = ((int64_t)(qrow + jc / G) * A.Hq + kvh * G + jc % G) * D;
#pragma unroll
    for (int kk = 0; kk < KS; kk++) {
        u32x4 w = *reinterpret_cast<const u32x4 *>(A.q + q_off + (4 * kk + g) * 8);
        if (j >= cols) w = u32x4{0u, 0u, 0u, 0u};
        qreg[kk] = __builtin_bit_cast(x8, w);
    }
    const int n_plain = min(max(runs.plain() - i0, 0), n_pg);
    const auto none = [](f32x4 &) {};
    // A ring of NS register stages, as in decode_sweep: pages that need no mask, with a page requested in every turn, then the rest.
    DecodePage<D> st[NS];
#pragma unroll
    for (int u = 0; u < NS - 1; u++)
        if (u < n_pg) decode_fetch<D>(A, kvh, __builtin_amdgcn_readlane(my_page, u), j, g, st[u]);
    int pp = 0;
    for (; pp + 2 * (NS - 1) < n_pg && pp + NS <= n_plain; pp += NS) {
#pragma unroll
        for (int u = 0; u < NS; u++) {
            decode_fetch<D>(A, kvh, __builtin_amdgcn_readlane(my_page, pp + u + NS - 1), j, g, st[(u + NS - 1) % NS]);
            decode_page<D, E>(A, st[u], 0, qreg, o, m_run, l_run, none);
        }
    }
    for (; pp < n_pg; pp += NS) {
#pragma unroll
        for (int u = 0; u < NS; u++) {
            const int cur = pp + u;
            if (cur < n_pg) {
                if (cur + NS - 1 < n_pg) decode_fetch<D>(A, kvh, __builtin_amdgcn_readlane(my_page, cur + NS - 1), j, g, st[(u + NS - 1) % NS]);
                const uint32_t bits = cur < n_plain ? 0xFFFFu : span_bits(runs.page(i0 + cur), pos, A.window, A.sinks);
                decode_page<D, E>(A, st[u], 0, qreg, o, m_run, l_run, [&](f32x4 &s) __attribute__((always_inline)) {
                    if (bits == 0xFFFFu) return;  // (uniform)
                    const uint32_t mine = bits >> (4 * g);
#pragma unroll
                    for (int r = 0; r < 4; r++) s[r] = (mine >> r & 1) ? s[r] : -INFINITY;
                    // V of tokens that are not attended over may be anything: probability 0 times something finite
                    const uint32_t m0 = (mine & 1 ? 0x0000FFFFu : 0u) | (mine & 2 ? 0xFFFF0000u : 0u), m1 = (mine & 4 ? 0x0000FFFFu : 0u) | (mine & 8 ? 0xFFFF0000u : 0u);
#pragma unroll
                    for (int c = 0; c < D / 16; c++) st[u].v[c] = u32x2{st[u].v[c][0] & m0, st[u].v[c][1] & m1};
                });
            }
        }
    }
    l_run += xor_lanes(l_run, 16);
    l_run = half_swap_sum(l_run);
}

// Vectors of four elements v0, v0 + step, .. of the output rows of a merge item, for KV head h: each from its row's partial results, i of them in workspace row
// base + h * kv + i * step + r for row r of the item, for either of two lists.  PEER: other compute units have stored them while this kernel runs.
// (As many requested at a time: 4 / 8 / 16, 33 decodes behind 1008 beside two groups more 17.2 / 16.3 / 16.6 us, 256 behind 8192 124 / 124 / 130, 4 behind 2048 10.1 / 10.2 / 10.8.)
constexpr int kSpanMergeThreads = 256, kSpanMergeBatch = 8;
template <int D, class E, bool PEER>
__device__ __forceinline__ void span_merge_rows(const int32_t *it, int h, const float *ws, uint16_t *out, int64_t n_rows, int Hq, int G, int v0, int v_step) {
    constexpr int VR = D / 4;
    const float *ws_ml = ws + n_rows * D;
    const __amdgpu_buffer_rsrc_t win = peer_window(ws, PEER ? (uint32_t)(n_rows * D * sizeof(float)) : 0u);
    for (int v = v0; v < it[SM_N] * G * VR; v += v_step) {
        const int r = v / VR, d = (v % VR) * 4;
        RowSum acc = {f32x4{0.f, 0.f, 0.f, 0.f}, -1e30f, 0.f};
        const auto add = [&](int64_t base, int n, int64_t step) {
            for (int i0 = 0; i0 < n; i0 += kSpanMergeBatch) {
                f32x4 o[kSpanMergeBatch];
                float2 ml[kSpanMergeBatch];
#pragma unroll
                for (int u = 0; u < kSpanMergeBatch; u++) {
                    if (i0 + u >= n) break;  // (uniform)
                    const int64_t at = base + (i0 + u) * step + r;
                    o[u] = PEER ? load4<true>(win, ws, (uint32_t)((at * D + d) * sizeof(float))) : *reinterpret_cast<const f32x4 *>(ws + at * D + d);
                    ml[u] = load2<PEER>(ws_ml + at * 2);
                }
#pragma unroll
                for (int u = 0; u < kSpanMergeBatch; u++)
                    if (i0 + u < n) acc.add(o[u], ml[u].x, ml[u].y);
            }
        };
        add((int64_t)it[SM_A] + (int64_t)h * it[SM_A_KV], it[SM_NA], it[SM_A_STEP]);
        add((int64_t)it[SM_B] + (int64_t)h * it[SM_B_KV], it[SM_NB], it[SM_B_STEP]);
        const float inv = 1.f / acc.l;
        typename E::x4 w;
#pragma unroll
        for (int e = 0; e < 4; e++) w[e] = (typename E::t)(acc.o[e] * inv);
        *reinterpret_cast<typename E::x4 *>(out + ((int64_t)(it[SM_QROW] + r / G) * Hq + h * G + r % G) * D + d) = w;
    }
}

// Workgroup (x, h, z): share z of merge item x of KV head h.
template <int D, class E>
__global__ void __launch_bounds__(kSpanMergeThreads) span_merge_kernel(const int32_t *__restrict__ merge, const float *__restrict__ ws, uint16_t *__restrict__ out, int64_t n_rows, int Hq, int G) {
    span_merge_rows<D, E, false>(merge + (int64_t)blockIdx.x * kSpanItemInts, blockIdx.y, ws, out, n_rows, Hq, G, blockIdx.z * kSpanMergeThreads + threadIdx.x, gridDim.z * kSpanMergeThreads);
}

// One workgroup's decode items: WAVES >> waves_log2 of them, each run by 1 << waves_log2 waves that share its pages out in contiguous runs and meet in LDS.
template <int D, class E, int NS, int WAVES>
__device__ __forceinline__ void span_decode(const AttnArgs &A, const SpanScalars &sc, const int32_t *__restrict__ items, const int32_t *__restrict__ merge, int unit, float *lds) {
    using x4 = typename E::x4;
    using el = typename E::t;
    constexpr int MT = D / 16, VR = D / 4;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), j = lane & 15, g = lane >> 4;
    const int w2 = sc.waves_log2, team = wave >> w2, n_waves = 1 << w2, part = wave & (n_waves - 1);
    const int32_t *it = items + ((int64_t)unit * (WAVES >> w2) + team) * kSpanItemInts;
    const int kvh = it[SD_KVH], qrow = it[SD_QROW], cols = it[SD_COLS], row = it[SD_ROW], n = it[SD_END] - it[SD_BEGIN], G = A.G;
    const SpanRuns runs = {it[SD_A], it[SD_H], it[SD_F], it[SD_B], it[SD_C], it[SD_E]};
    f32x4 o[MT];
#pragma unroll
    for (int c = 0; c < MT; c++) o[c] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m_run = -1e30f, l_run = 0.f;
    const int p0 = n * part >> w2, p1 = n * (part + 1) >> w2;
    if (p1 > p0)
        span_decode_sweep<D, E, NS>(A, kvh, qrow, cols, A.pages + it[SD_PAGEOFF], runs, it[SD_BEGIN] + p0, p1 - p0, it[SD_POS], lane, o, m_run, l_run);
    const auto out_row = [&](int jj) { return A.out + ((int64_t)(qrow + jj / G) * A.Hq + kvh * G + jj % G) * D; };
    if (w2 == 0) {
        if (n == 0 || j >= cols) return;
        if (row < 0) {
            const float inv = 1.f / l_run;
            uint16_t *dst = out_row(j) + 4 * g;
#pragma unroll
            for (int c = 0; c < MT; c++) {
                x4 w;
#pragma unroll
                for (int e = 0; e < 4; e++) w[e] = (el)(o[c][e] * inv);
                *reinterpret_cast<x4 *>(dst + 16 * c) = w;
            }
        } else {
            float *dst = A.ws_o + ((int64_t)row + j) * D + 4 * g;
#pragma unroll
            for (int c = 0; c < MT; c++) *reinterpret_cast<f32x4 *>(dst + 16 * c) = o[c];
            if (g == 0) *reinterpret_cast<float2 *>(A.ws_ml + ((int64_t)row + j) * 2) = float2{m_run, l_run};
        }
        return;
    }
    const WaveResults<D> res(lds, WAVES, sc.max_cols);
    res.put(wave, lane, o, m_run, l_run);
    __syncthreads();
    if (n == 0) return;
    const int first = wave - part, threads = n_waves * 64;
    for (int v = tid & (threads - 1); v < cols * VR; v += threads) {
        const int jj = v / VR, d = (v % VR) * 4;
        float m = -1e30f;
        for (int i = 0; i < n_waves; i++) m = fmaxf(m, res.get_ml(first + i, jj).x);
        f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
        float l = 0.f;
        for (int i = 0; i < n_waves; i++) {
            const float2 ml = res.get_ml(first + i, jj);
            const float w = fast_exp2(ml.x - m);
            l += w * ml.y;
            acc += res.get(first + i, jj, d) * w;
        }
        if (row < 0) {
            const float inv = 1.f / l;
            x4 w4;
#pragma unroll
            for (int e = 0; e < 4; e++) w4[e] = (el)(acc[e] * inv);
            *reinterpret_cast<x4 *>(out_row(jj) + d) = w4;
        } else if (sc.counters) {
            peer_store4(peer_window(A.ws_o + (int64_t)row * D, (uint32_t)(cols * D * sizeof(float))), (uint32_t)v * 16, acc);
            if (d == 0) peer_store2(A.ws_ml + ((int64_t)row + jj) * 2, m, l);
        } else {
            *reinterpret_cast<f32x4 *>(A.ws_o + ((int64_t)row + jj) * D + d) = acc;
            if (d == 0) *reinterpret_cast<float2 *>(A.ws_ml + ((int64_t)row + jj) * 2) = float2{m, l};
        }
    }
    if (row < 0 || !sc.counters) return;
    // (The whole workgroup runs one item.)  The last workgroup of the sequence and KV head to get here combines all partial results; nobody waits.
    stores_done();
    int32_t *const counter = sc.counters + (it[SD_MERGE] * A.Hkv + kvh) * sc.counter_stride;
    if (!workgroup_arrives_last(counter, it[SD_PARTS], reinterpret_cast<int *>(lds), tid)) return;
    span_merge_rows<D, E, true>(merge + (int64_t)it[SD_MERGE] * kSpanItemInts, kvh, A.ws_o, A.out, sc.n_rows, A.Hq, G, tid, WAVES * 64);
}

template <int D, class E, int WAVES, int PER_CU, int NS, bool SWEEPS>
__global__ void __launch_bounds__(WAVES * 64, PER_CU)
    span_attention_kernel(const uint16_t *__restrict__ k_pool, const uint16_t *__restrict__ v_pool, const uint16_t *__restrict__ q, uint16_t *__restrict__ out,
                          const int32_t *__restrict__ pages, const int32_t *__restrict__ records, const int32_t *__restrict__ items, const int32_t *__restrict__ merge, float *ws, const SpanScalars sc) {
    extern __shared__ __align__(16) char lds[];
    AttnArgs A = {};
    A.k_pool = const_cast<uint16_t *>(k_pool); A.v_pool = const_cast<uint16_t *>(v_pool); A.q = q; A.out = out; A.pages = pages;
    A.ws_o = ws; A.ws_ml = ws + sc.n_rows * D;
    A.Hq = sc.Hq; A.Hkv = sc.Hkv; A.G = sc.G; A.scale_log2 = sc.scale_log2; A.window = sc.window; A.sinks = sc.sinks;
    const int wg = (int)blockIdx.x;
    int unit = wg;
    if constexpr (SWEEPS) {
        // The order of the launch: n_first sweeps and n_early decode units, dealt out evenly in rows of Hkv workgroups, then the other sweeps, then the other units.
        int sweep = -1;
        const int mixed = sc.n_first + sc.n_early;
        if (wg < mixed) {
            const int Hkv = A.Hkv, row = wg / Hkv, rows = mixed / Hkv, sweep_rows = sc.n_first / Hkv;
            const int before = (int)((int64_t)row * sweep_rows / rows);  // rows of sweeps before this one
            if ((int)((int64_t)(row + 1) * sweep_rows / rows) > before) sweep = before * Hkv + wg % Hkv;
            else unit = (row - before) * Hkv + wg % Hkv;
        } else if (wg < sc.n_sweeps + sc.n_early) {
            sweep = wg - sc.n_early;
        } else {
            unit = wg - sc.n_sweeps;
        }
        if (sweep >= 0) {
            for (int r = sweep / A.Hkv;;) {
                const int32_t *rec = records + (int64_t)r * kRecordInts;
                prefill_item<D, E, WAVES, true>(A, rec, sweep % A.Hkv, lds);
                r = rec[SR_NEXT];
                if (r < 0) return;
                __syncthreads();  // the next piece's tile copies reuse the LDS
            }
        }
    }
    span_decode<D, E, NS, WAVES>(A, sc, items, merge, unit, reinterpret_cast<float *>(lds));
}

template <int D, class E>
int launch_span_d(const tc_plan *p, const SpanList &s, const tc_kv_pool *pool, const void *q, void *out, float scale, void *workspace, hipStream_t st) {
    const int32_t *pages = p->dev + p->off_pages, *records = s.dev + s.off_records, *items = s.dev + s.off_items, *merge = s.dev + s.off_merge;
    const SpanScalars sc = {p->Hq, p->Hkv, p->G, s.n_sweeps, s.n_first, s.n_early, s.waves_log2, s.max_cols, s.window, s.sinks, scale * 1.4426950408889634f, s.n_rows,
                            s.fused ? s.dev + s.off_counters : nullptr, s.counter_stride};
    const int grid = s.grid_blocks();
    const auto launch = [&](auto waves, auto per_cu, auto stages, auto sweeps, size_t lds) {
        constexpr int W = decltype(waves)::value, PER_CU = decltype(per_cu)::value, NS = decltype(stages)::value;
        constexpr bool SWEEPS = decltype(sweeps)::value;
        if (SWEEPS) {  // more than 64 KiB of LDS needs an opt-in for each device
            static std::atomic<bool> done[kMaxDevices];
            const bool known = p->device >= 0 && p->device < kMaxDevices;
            if (!known || !done[p->device].load(std::memory_order_acquire)) {
                const hipError_t e = hipFuncSetAttribute((const void *)span_attention_kernel<D, E, W, PER_CU, NS, SWEEPS>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
                if (e != hipSuccess) return (int)e;
                if (known) done[p->device].store(true, std::memory_order_release);
            }
        }
        span_attention_kernel<D, E, W, PER_CU, NS, SWEEPS><<<grid, W * 64, lds, st>>>(
            (const uint16_t *)pool->k_pool, (const uint16_t *)pool->v_pool, (const uint16_t *)q, (uint16_t *)out, pages, records, items, merge, (float *)workspace, sc);
        return (int)hipGetLastError();
    };
    const std::true_type yes;
    const std::false_type no;
    int err;
    if (s.n_sweeps > 0 && s.sweep_waves == kMixedWaves) err = launch(Int<kMixedWaves>(), Int<1>(), Int<kDecodeStages>(), yes, PrefillLds<D, kMixedWaves>::kBytes);
    else if (s.n_sweeps > 0) err = launch(Int<kSmallWaves>(), Int<small_wg_per_cu(D)>(), Int<kDecodeStages>(), yes, PrefillLds<D, kSmallWaves>::kBytes);
    else if (s.wide) err = launch(Int<kDecodeWaves>(), Int<2>(), Int<kWideStages>(), no, decode_lds_bytes(kDecodeWaves, s.max_cols, D));
    else err = launch(Int<kDecodeWaves>(), Int<kDecodeWgPerCu>(), Int<kDecodeStages>(), no, decode_lds_bytes(kDecodeWaves, s.max_cols, D));
    if (err || s.n_merge == 0 || s.fused) return err;
    const unsigned shares = (unsigned)std::max(1, s.merge_rows * p->G * (D / 4) / kSpanMergeThreads);
    span_merge_kernel<D, E><<<dim3((unsigned)s.n_merge, (unsigned)p->Hkv, shares), kSpanMergeThreads, 0, st>>>(merge, (const float *)workspace, (uint16_t *)out, s.n_rows, p->Hq, p->G);
    return (int)hipGetLastError();
}

}  // namespace

int launch_span(const tc_plan *p, const SpanList &s, const tc_kv_pool *pool, const void *q, void *out, float scale, void *workspace, void *stream) {
    hipStream_t st = (hipStream_t)stream;
    if (p->dtype == TC_FP16)
        return p->D == 128 ? launch_span_d<128, Fp16>(p, s, pool, q, out, scale, workspace, st) : launch_span_d<64, Fp16>(p, s, pool, q, out, scale, workspace, st);
    return p->D == 128 ? launch_span_d<128, Bf16>(p, s, pool, q, out, scale, workspace, st) : launch_span_d<64, Bf16>(p, s, pool, q, out, scale, workspace, st);
}

}  // namespace tc
