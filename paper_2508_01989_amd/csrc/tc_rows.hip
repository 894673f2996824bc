// Rows on their way into attention: each head of q and k divided by its root mean square and rotated by its position, in one pass over
// the data, and (the second form) k stored into the paged pool with v beside it.
//
//   y = x * (mean(x^2) + eps)^-1/2 * w,   then (a, b) -> (a cos t - b sin t, b cos t + a sin t)  for each pair, t = position * freq[pair]
//
// Bound by the bytes: every element is read once and written once, 2 bytes each way.
#include "tc_attention.h"

namespace tc {

namespace {

struct RowsBf16 {
    static __device__ __forceinline__ float widen(uint32_t bits) { return __uint_as_float(bits << 16); }
    static __device__ __forceinline__ uint32_t narrow(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
};
struct RowsFp16 {
    static __device__ __forceinline__ float widen(uint32_t bits) { return (float)__builtin_bit_cast(_Float16, (uint16_t)bits); }
    static __device__ __forceinline__ uint32_t narrow(float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); }
};
template <class E>
__device__ __forceinline__ void widen4(u32x2 w, float (&x)[4]) {
#pragma unroll
    for (int e = 0; e < 4; e++) x[e] = E::widen((w[e >> 1] >> (16 * (e & 1))) & 0xFFFF);
}
template <class E>
__device__ __forceinline__ u32x2 narrow4(const float (&x)[4]) {
    return u32x2{E::narrow(x[0]) | E::narrow(x[1]) << 16, E::narrow(x[2]) | E::narrow(x[3]) << 16};
}

// Sum over the lanes of a row, 16 or 8 adjacent lanes, in every one of them.
template <int LANES>
__device__ __forceinline__ float row_sum(float v) {
    const auto add = [&](auto ctrl) {
        v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, 0xF, 0xF, true));
    };
    add(std::integral_constant<int, 0xB1>());   // lane ^ 1
    add(std::integral_constant<int, 0x4E>());   // lane ^ 2
    add(std::integral_constant<int, 0x141>());  // the other four of each eight, mirrored
    if constexpr (LANES == 16) add(std::integral_constant<int, 0x140>());  // the other eight, mirrored
    return v;
}

struct RowsArgs {
    const uint16_t *q, *k, *v, *q_weight, *k_weight;
    const double *freq;
    const int32_t *positions;
    uint16_t *q_out, *k_out;  // k_out: null where k goes into the pool
    uint16_t *k_pool, *v_pool;
    int64_t q_stride, k_stride, v_stride;
    int Hq, Hkv, rotary_dim, adjacent;
    int splits;  // workgroups that share a segment's heads of q and k; the ones behind them store its v
    float eps;
};

constexpr int kRowsThreads = 256;
constexpr int kRowsBatch = 4;  // heads that a thread has under way at once

// The elements of a row lie four and four on its D/8 lanes, so that a lane holds both elements of its pairs and none crosses lanes: where pairs are a
// half of the rotated part apart, lane l holds elements 4 l .. and rotary_dim / 2 + 4 l ..; where they are adjacent, 8 l .. 8 l + 7.  Either way its pairs are 4 l .. 4 l + 3.
// Lanes past the rotated part hold eight adjacent elements of the rest.
template <int D>
struct RowLane {
    int a, b;     // first elements of the lane's two fours
    bool turns;
    __device__ __forceinline__ RowLane(int l, int rotary_dim, int adjacent) {
        const int n = rotary_dim / 8;  // lanes of the rotated part
        turns = l < n;
        if (turns && !adjacent) {
            a = 4 * l;
            b = rotary_dim / 2 + 4 * l;
        } else {
            a = 8 * l;
            b = 8 * l + 4;
        }
    }
};

// Workgroup (x, y): segment x of the batch (up to 16 rows of one sequence, on one page), share y of its heads.  A row of lanes keeps its token, so that a
// thread computes its four angles once, in 64 bits (positions reach 2^31: in 32 bits an angle at 10^6 would be off by 0.06), and takes head after head.
template <int D, class E, bool STORE>
__global__ void __launch_bounds__(kRowsThreads) rows_kernel(const RowsArgs A, const int32_t *__restrict__ segments, const int32_t *__restrict__ seg_pos) {
    constexpr int LANES = D / 8, GROUPS = kRowsThreads / LANES;
    const int32_t *seg = segments + (int64_t)blockIdx.x * kAppendInts;
    const int row0 = seg[0], n_tok = seg[1], tok0 = seg[2];
    const int64_t block = (int64_t)seg[3] * A.Hkv * (kBlock * D);
    const int tid = threadIdx.x;
    if constexpr (STORE) {
        if ((int)blockIdx.y >= A.splits) {  // v: the pool is token-minor
            if (n_tok == 1) {
                const uint16_t *src = A.v + (int64_t)row0 * A.v_stride;
                uint16_t *dst = A.v_pool + block + v_slot(tok0);
                for (int x = tid; x < A.Hkv * D; x += kRowsThreads) dst[(int64_t)x * kBlock] = src[x];
                return;
            }
            // a thread has four slots of one element, which hold adjacent tokens: one store of 8 bytes where all four are new
            for (int x = tid; x < A.Hkv * D * 4; x += kRowsThreads) {
                const int e = x % D, g = x / D % 4, h = x / (4 * D);
                const int t_first = v_slot(4 * g);
                uint16_t val[4];
                int have = 0;
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const int t = t_first + i - tok0;
                    const bool is_new = t >= 0 && t < n_tok;
                    have += is_new;
                    val[i] = is_new ? A.v[(int64_t)(row0 + t) * A.v_stride + h * D + e] : (uint16_t)0;
                }
                uint16_t *dst = A.v_pool + block + (int64_t)(h * D + e) * kBlock + 4 * g;
                if (have == 4) {
                    *reinterpret_cast<u32x2 *>(dst) = u32x2{(uint32_t)val[0] | (uint32_t)val[1] << 16, (uint32_t)val[2] | (uint32_t)val[3] << 16};
                } else {
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        const int t = t_first + i - tok0;
                        if (t >= 0 && t < n_tok) dst[i] = val[i];
                    }
                }
            }
            return;
        }
    }
    const int l = tid % LANES, group = tid / LANES;
    const int per_token = GROUPS / n_tok;  // groups of lanes that share a token's heads
    const int t = group / per_token;
    if (t >= n_tok) return;
    const int row = row0 + t;
    const RowLane<D> lane(l, A.rotary_dim, A.adjacent);
    float c[4], s[4];
#pragma unroll
    for (int e = 0; e < 4; e++) { c[e] = 1.f; s[e] = 0.f; }
    if (lane.turns) {
        const double position = A.positions ? A.positions[row] : seg_pos[blockIdx.x] + t;
#pragma unroll
        for (int e = 0; e < 4; e++) {
            double turns = position * (A.freq[4 * l + e] * 0.15915494309189533576888376337251);  // 1 / (2 pi)
            turns -= __builtin_rint(turns);
            sincospif(2.f * (float)turns, &s[e], &c[e]);
        }
    }
    float wq[8], wk[8];
    const auto weights = [&](const uint16_t *w, float (&x)[8]) {
        float lo[4] = {1.f, 1.f, 1.f, 1.f}, hi[4] = {1.f, 1.f, 1.f, 1.f};
        if (w) {
            widen4<E>(*reinterpret_cast<const u32x2 *>(w + lane.a), lo);
            widen4<E>(*reinterpret_cast<const u32x2 *>(w + lane.b), hi);
        }
#pragma unroll
        for (int e = 0; e < 4; e++) { x[e] = lo[e]; x[4 + e] = hi[e]; }
    };
    weights(A.q_weight, wq);
    weights(A.k_weight, wk);
    const uint16_t *const q = A.q + (int64_t)row * A.q_stride, *const k = A.k + (int64_t)row * A.k_stride;
    uint16_t *const q_out = A.q_out + (int64_t)row * A.Hq * D;
    uint16_t *const k_out = STORE ? A.k_pool + block : A.k_out + (int64_t)row * A.Hkv * D;
    const int heads = A.Hq + A.Hkv, step = per_token * A.splits;
    const int token = tok0 + t;
    for (int h0 = (group - t * per_token) + (int)blockIdx.y * per_token; h0 < heads; h0 += kRowsBatch * step) {
        u32x2 lo[kRowsBatch], hi[kRowsBatch];
#pragma unroll
        for (int u = 0; u < kRowsBatch; u++) {
            const int h = h0 + u * step;
            if (h < heads) {
                const uint16_t *src = h < A.Hq ? q + h * D : k + (h - A.Hq) * D;
                lo[u] = *reinterpret_cast<const u32x2 *>(src + lane.a);
                hi[u] = *reinterpret_cast<const u32x2 *>(src + lane.b);
            }
        }
#pragma unroll
        for (int u = 0; u < kRowsBatch; u++) {
            const int h = h0 + u * step;
            if (h >= heads) break;
            const bool is_q = h < A.Hq;
            float a[4], b[4];
            widen4<E>(lo[u], a);
            widen4<E>(hi[u], b);
            if (is_q ? A.q_weight != nullptr : A.k_weight != nullptr) {
                float sum = 0.f;
#pragma unroll
                for (int e = 0; e < 4; e++) sum = __builtin_fmaf(a[e], a[e], __builtin_fmaf(b[e], b[e], sum));
                sum = row_sum<LANES>(sum);
                float r = 1.f / sqrtf(sum * (1.f / D) + A.eps);
                // Squares past what 32 bits hold, or so small that they lose digits there (bf16 reaches 2^127 and 2^-133): 64 bits, which hold them all.
                if (!(sum < 1e37f) || sum < 1e-30f) {
                    double wide = 0.0;
#pragma unroll
                    for (int e = 0; e < 4; e++) wide += (double)a[e] * a[e] + (double)b[e] * b[e];
#pragma unroll
                    for (int m = 1; m < LANES; m *= 2) wide += __shfl_xor(wide, m, 64);
                    const double rr = 1.0 / sqrt(wide * (1.0 / D) + (double)A.eps);
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        a[e] = (float)(a[e] * rr);
                        b[e] = (float)(b[e] * rr);
                    }
                    r = 1.f;
                }
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    a[e] *= r * (is_q ? wq[e] : wk[e]);
                    b[e] *= r * (is_q ? wq[4 + e] : wk[4 + e]);
                }
            }
            if (A.adjacent) {
#pragma unroll
                for (int e = 0; e < 4; e += 2) {
                    const float x = a[e] * c[e / 2] - a[e + 1] * s[e / 2], y = a[e + 1] * c[e / 2] + a[e] * s[e / 2];
                    const float z = b[e] * c[2 + e / 2] - b[e + 1] * s[2 + e / 2], w = b[e + 1] * c[2 + e / 2] + b[e] * s[2 + e / 2];
                    a[e] = x;
                    a[e + 1] = y;
                    b[e] = z;
                    b[e + 1] = w;
                }
            } else {
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    const float x = a[e] * c[e] - b[e] * s[e], y = b[e] * c[e] + a[e] * s[e];
                    a[e] = x;
                    b[e] = y;
                }
            }
            if (is_q) {
                *reinterpret_cast<u32x2 *>(q_out + h * D + lane.a) = narrow4<E>(a);
                *reinterpret_cast<u32x2 *>(q_out + h * D + lane.b) = narrow4<E>(b);
            } else if (STORE) {  // pool: [D/8][16 tokens][8]
                uint16_t *dst = k_out + (int64_t)(h - A.Hq) * (kBlock * D) + token * 8;
                *reinterpret_cast<u32x2 *>(dst + (lane.a >> 3) * (kBlock * 8) + (lane.a & 7)) = narrow4<E>(a);
                *reinterpret_cast<u32x2 *>(dst + (lane.b >> 3) * (kBlock * 8) + (lane.b & 7)) = narrow4<E>(b);
            } else {
                *reinterpret_cast<u32x2 *>(k_out + (h - A.Hq) * D + lane.a) = narrow4<E>(a);
                *reinterpret_cast<u32x2 *>(k_out + (h - A.Hq) * D + lane.b) = narrow4<E>(b);
            }
        }
    }
}

}  // namespace

int launch_rows(const tc_plan *p, const tc_kv_pool *pool, const tc_qkv_rows *rows, void *q_out, void *k_out, void *stream) {
    if (p->n_append == 0) return 0;
    RowsArgs A;
    A.q = (const uint16_t *)rows->q;
    A.k = (const uint16_t *)rows->k;
    A.v = (const uint16_t *)rows->v;
    A.q_weight = (const uint16_t *)rows->q_weight;
    A.k_weight = (const uint16_t *)rows->k_weight;
    A.freq = rows->freq;
    A.positions = rows->positions;
    A.q_out = (uint16_t *)q_out;
    A.k_out = (uint16_t *)k_out;
    A.k_pool = pool ? (uint16_t *)pool->k_pool : nullptr;
    A.v_pool = pool ? (uint16_t *)pool->v_pool : nullptr;
    A.q_stride = rows->q_stride;
    A.k_stride = rows->k_stride;
    A.v_stride = rows->v_stride;
    A.Hq = p->Hq;
    A.Hkv = p->Hkv;
    A.rotary_dim = rows->rotary_dim;
    A.adjacent = rows->adjacent;
    A.eps = rows->eps;
    A.splits = (int)std::min<int64_t>(4, std::max<int64_t>(1, 2048 / p->n_append));
    const dim3 grid((unsigned)p->n_append, (unsigned)(A.splits + (pool ? 1 : 0)));
    hipStream_t st = (hipStream_t)stream;
    const int32_t *segments = p->dev + p->off_append, *seg_pos = p->dev + p->off_seg_pos;
    const auto launch = [&](auto dim, auto type, auto store) {
        rows_kernel<decltype(dim)::value, decltype(type), decltype(store)::value><<<grid, kRowsThreads, 0, st>>>(A, segments, seg_pos);
    };
    const auto by_store = [&](auto dim, auto type) { pool ? launch(dim, type, std::true_type()) : launch(dim, type, std::false_type()); };
    const auto by_type = [&](auto dim) { p->dtype == TC_FP16 ? by_store(dim, RowsFp16()) : by_store(dim, RowsBf16()); };
    p->D == 128 ? by_type(std::integral_constant<int, 128>()) : by_type(std::integral_constant<int, 64>());
    return (int)hipGetLastError();
}

}  // namespace tc
