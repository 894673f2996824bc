// Rows on their way into attention: each head of q and k divided by its root mean square and rotated by its position, in one pass over
// the data, and (the second form) k stored into the paged pool with v beside it.
//
//   y = x * (mean(x^2) + eps)^-1/2 * w,   then (a, b) -> (a cos t - b sin t, b cos t + a sin t)  for each pair, t = position * freq[pair]
//
// Bound by the bytes: every element is read once and written once, 2 bytes each way; v and k of a single token go into the pages in pieces of 2 and 16 bytes, for each of which memory
// takes 32 (512 decodes, 40/8 heads, write 24 MB by the counters where they have 7.3).  One MI355X, head_dim 128, launches back to back in a graph: 8192 tokens, 64/8, 67-70 us and 4.8-5.0 TB/s
// with the append, 56 us and 5.4 without (a bare copy 5.0); 512 decodes, 40/8, 8.9 and 5.2 us; 8 decodes 4.6 and 3.9, the launch and a chain of three accesses to memory.
#include "tc_attention.h"

namespace tc {

namespace {

template <class E>
__device__ __forceinline__ void widen4(u32x2 w, float (&x)[4]) {
    const typename E::x4 v = __builtin_bit_cast(typename E::x4, w);
#pragma unroll
    for (int e = 0; e < 4; e++) x[e] = (float)v[e];
}
template <class E>
__device__ __forceinline__ u32x2 narrow4(const float (&x)[4]) {
    typename E::x4 v;
#pragma unroll
    for (int e = 0; e < 4; e++) v[e] = (typename E::t)x[e];
    return __builtin_bit_cast(u32x2, v);
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
    int splits;  // workgroups that share a segment
    float eps;
};

constexpr int kRowsThreads = 256;
constexpr int kRowsWorkgroups = 768;
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

// Head `h` of a row, four and four elements: norm, and where the lane has rotated ones (`turns`) rotation by the angles whose cosines and sines are c and s.  (The others are not turned by
// an angle of zero: x - y * 0 would take a NaN or an infinity from one to another, and a zero's sign.)
template <int D, class E>
__device__ __forceinline__ void turn_head(const RowsArgs &A, bool turns, float (&a)[4], float (&b)[4], bool normed, const float (&w)[8], const float (&c)[4], const float (&s)[4]) {
    constexpr int LANES = D / 8;
    if (normed) {
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 4; e++) sum = __builtin_fmaf(a[e], a[e], __builtin_fmaf(b[e], b[e], sum));
        sum = row_sum<LANES>(sum);
        float r = __builtin_amdgcn_rsqf(sum * (1.f / D) + A.eps);  // (to one unit in the last place, of a normal number)
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
        // (The quotient first: it is sqrt(D) at most, while the root times a weight may leave 32 bits where the result does not.)
#pragma unroll
        for (int e = 0; e < 4; e++) {
            a[e] = a[e] * r * w[e];
            b[e] = b[e] * r * w[4 + e];
        }
    }
    const auto turn = [&](float &x, float &y, int pair) {
        const float x0 = x, y0 = y;
        x = turns ? x0 * c[pair] - y0 * s[pair] : x0;
        y = turns ? y0 * c[pair] + x0 * s[pair] : y0;
    };
    if (A.adjacent) {
        turn(a[0], a[1], 0);
        turn(a[2], a[3], 1);
        turn(b[0], b[1], 2);
        turn(b[2], b[3], 3);
    } else {
#pragma unroll
        for (int e = 0; e < 4; e++) turn(a[e], b[e], e);
    }
}

// What a wave stores of a page of the pools at a time: 128 adjacent elements of a token's heads (one head at head_dim 128, two at 64) of up to 16 tokens.  Either pool has them
// in 4 KiB that are adjacent, but in an order in which the lanes that computed them would store 8 bytes here and there, so they are turned round in LDS and stored 1 KiB
// at a time (8192 tokens, 64/8 heads, head_dim 128: q and k alone 55 us, 80 with k and v stored from where they were computed).
// k: piece p (8 elements) of token t at p * 272 + t * 16 bytes; v: element e at e * 32 + e / 8 * 16.  The 16 bytes between keep lanes on different banks.
constexpr int kSlab = 128, kSlabBytes = kSlab / 8 * 272;
struct SlabLane {  // a quarter of a wave has a token: lane l of it, elements and head
    int l, head, group;
};
template <int D>
__device__ __forceinline__ SlabLane slab_lane(int lane) { return {lane % (D / 8), lane % 16 / (D / 8), lane / 16}; }

// Every lane's four chunks of 16 bytes of a slab of k, as they lie in the pool: chunk c is piece c / 16 of token c % 16.
__device__ __forceinline__ void store_slab_k(const char *tile, uint16_t *dst, int n_elements, int n_tok, int tok0, int lane) {
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const int c = i * 64 + lane, p = c / 16, t = c % 16;
        const u32x4 w = *reinterpret_cast<const u32x4 *>(tile + p * 272 + t * 16);
        if (t >= tok0 && t < tok0 + n_tok && p * 8 < n_elements) *reinterpret_cast<u32x4 *>(dst + c * 8) = w;
    }
}
// And of v: chunk c is slots 8 (c % 2) .. of element c / 2.
__device__ __forceinline__ void store_slab_v(const char *tile, uint16_t *dst, int n_elements, int n_tok, int tok0, int lane) {
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const int c = i * 64 + lane, e = c / 2;
        const u32x4 w = *reinterpret_cast<const u32x4 *>(tile + e * 32 + e / 8 * 16 + c % 2 * 16);
        if (e >= n_elements) continue;
        if (n_tok == kBlock) {
            *reinterpret_cast<u32x4 *>(dst + c * 8) = w;
        } else {
#pragma unroll
            for (int x = 0; x < 8; x++) {
                const int t = v_slot(c % 2 * 8 + x);
                if (t >= tok0 && t < tok0 + n_tok) dst[c * 8 + x] = (uint16_t)(w[x / 2] >> (16 * (x & 1)));
            }
        }
    }
}

// Workgroup (x, y): segment x of the batch (up to 16 rows of one sequence, on one page), share y of it.  Its waves take tasks of 4 KiB each and have the next one's data under way while they
// compute: several adjacent heads of one token, or, of more tokens than one, a slab of k or of v (see above).  The angles of the segment are computed once for each
// workgroup, in 64 bits (positions reach 2^31: in 32 bits an angle at 10^6 would be off by 0.06), while the first data is on its way.
// SLABS: there are segments of more tokens than one (a batch of decodes has none, and a kernel of fewer registers).
template <int D, class E, bool STORE, bool SLABS>
__global__ void __launch_bounds__(kRowsThreads) rows_kernel(const RowsArgs A, const int32_t *__restrict__ segments, const int32_t *__restrict__ seg_pos) {
    constexpr int LANES = D / 8, GROUPS = 64 / LANES, WAVES = kRowsThreads / 64, HEADS = GROUPS * kRowsBatch;
    __shared__ __align__(16) float2 turns[kBlock * (D / 2)];  // cosine and sine of each token's angles
    __shared__ __align__(16) char tiles[SLABS ? WAVES * kSlabBytes : 16];
    const int32_t *seg = segments + (int64_t)blockIdx.x * kAppendInts;
    const int row0 = seg[0], n_tok = seg[1], tok0 = seg[2];
    const int64_t block = (int64_t)seg[3] * A.Hkv * (kBlock * D);
    const int tid = threadIdx.x, lane_id = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l = lane_id % LANES, group = lane_id / LANES;
    const RowLane<D> lane(l, A.rotary_dim, A.adjacent);
    const SlabLane sl = slab_lane<D>(lane_id);
    // Tasks: the slabs of k and of v, then `chunks` to a token, those of q and (where there are no slabs) of k.
    const bool in_slabs = SLABS && n_tok > 1;
    const int kv_elements = A.Hkv * D, slabs = in_slabs ? (kv_elements + kSlab - 1) / kSlab : 0;
    const int q_chunks = (A.Hq + HEADS - 1) / HEADS, chunks = q_chunks + (in_slabs ? 0 : (A.Hkv + HEADS - 1) / HEADS);
    const int tasks = 2 * slabs + n_tok * chunks, step = WAVES * A.splits;
    u32x2 lo[kRowsBatch], hi[kRowsBatch];
    const auto fetch = [&](int task) {
        if (task >= tasks) return;
        if (SLABS && task < 2 * slabs) {
            const bool is_k = task < slabs;
            const int x0 = (is_k ? task : task - slabs) * kSlab;
            // k: token 4 u + quarter, so that the quarters have adjacent ones; v: the four tokens of adjacent slots
            const uint16_t *src = is_k ? A.k + (int64_t)row0 * A.k_stride + x0 + sl.head * D : A.v + (int64_t)row0 * A.v_stride + x0 + lane_id % 16 * 8;
            const bool there = x0 + lane_id % 16 * 8 < kv_elements;
#pragma unroll
            for (int u = 0; u < kRowsBatch; u++) {
                const int t = is_k ? 4 * u + sl.group : 4 * sl.group + u - tok0;
                if (t < 0 || t >= n_tok || !there) continue;
                const uint16_t *from = src + (int64_t)t * (is_k ? A.k_stride : A.v_stride);
                lo[u] = *reinterpret_cast<const u32x2 *>(from + (is_k ? lane.a : 0));
                hi[u] = *reinterpret_cast<const u32x2 *>(from + (is_k ? lane.b : 4));
            }
            return;
        }
        const int t = (task - 2 * slabs) / chunks, chunk = task - 2 * slabs - t * chunks;
        const bool is_q = chunk < q_chunks;
        const uint16_t *src = is_q ? A.q + (int64_t)(row0 + t) * A.q_stride : A.k + (int64_t)(row0 + t) * A.k_stride;
        const int heads = is_q ? A.Hq : A.Hkv, h0 = (is_q ? chunk : chunk - q_chunks) * HEADS + group;
#pragma unroll
        for (int u = 0; u < kRowsBatch; u++) {
            const int h = h0 + u * GROUPS;
            if (h < heads) {
                lo[u] = *reinterpret_cast<const u32x2 *>(src + h * D + lane.a);
                hi[u] = *reinterpret_cast<const u32x2 *>(src + h * D + lane.b);
            }
        }
    };
    int task = wave + (int)blockIdx.y * WAVES;
    fetch(task);
    const int pairs = A.rotary_dim / 2;
    for (int x = tid; x < n_tok * pairs; x += kRowsThreads) {
        const int t = x / pairs, i = x - t * pairs;
        const double position = A.positions ? A.positions[row0 + t] : seg_pos[blockIdx.x] + t;
        double angle = position * (A.freq[i] * 0.15915494309189533576888376337251);  // in turns: 1 / (2 pi)
        angle -= __builtin_rint(angle);
        float sine, cosine;
        sincospif(2.f * (float)angle, &sine, &cosine);
        turns[t * (D / 2) + i] = float2{cosine, sine};
    }
    float wq[8], wk[8];
    const auto weights = [&](const uint16_t *weight, float (&w)[8]) {
        float x[4] = {1.f, 1.f, 1.f, 1.f}, y[4] = {1.f, 1.f, 1.f, 1.f};
        if (weight) {
            widen4<E>(*reinterpret_cast<const u32x2 *>(weight + lane.a), x);
            widen4<E>(*reinterpret_cast<const u32x2 *>(weight + lane.b), y);
        }
#pragma unroll
        for (int e = 0; e < 4; e++) { w[e] = x[e]; w[4 + e] = y[e]; }
    };
    weights(A.q_weight, wq);
    weights(A.k_weight, wk);
    if (STORE && !in_slabs) {  // v of a single token: its elements lie 32 bytes apart, a lane to each
        const int first = (int)blockIdx.y * kRowsThreads + tid, v_step = A.splits * kRowsThreads;
        const uint16_t *const src = A.v + (int64_t)row0 * A.v_stride;
        uint16_t *const dst = A.v_pool + block + v_slot(tok0);
        for (int x0 = first; x0 < kv_elements; x0 += 4 * v_step) {
            uint16_t w[4];
#pragma unroll
            for (int i = 0; i < 4; i++)
                if (x0 + i * v_step < kv_elements) w[i] = src[x0 + i * v_step];
#pragma unroll
            for (int i = 0; i < 4; i++)
                if (x0 + i * v_step < kv_elements) dst[(int64_t)(x0 + i * v_step) * kBlock] = w[i];
        }
    }
    __syncthreads();
    const auto angles = [&](int t, float (&c)[4], float (&s)[4]) {
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const float2 x = lane.turns ? turns[t * (D / 2) + 4 * l + e] : float2{1.f, 0.f};
            c[e] = x.x;
            s[e] = x.y;
        }
    };
    for (; task < tasks; task += step) {
        u32x2 lo_now[kRowsBatch], hi_now[kRowsBatch];
#pragma unroll
        for (int u = 0; u < kRowsBatch; u++) {
            lo_now[u] = lo[u];
            hi_now[u] = hi[u];
        }
        fetch(task + step);
        if (SLABS && task < 2 * slabs) {
            char *const tile = tiles + wave * kSlabBytes;
            const bool is_k = task < slabs;
            const int x0 = (is_k ? task : task - slabs) * kSlab;
            if (is_k) {
#pragma unroll
                for (int u = 0; u < kRowsBatch; u++) {
                    const int t = 4 * u + sl.group;
                    if (t >= n_tok) break;
                    float a[4], b[4], c[4], s[4];
                    angles(t, c, s);
                    widen4<E>(lo_now[u], a);
                    widen4<E>(hi_now[u], b);
                    turn_head<D, E>(A, lane.turns, a, b, A.k_weight != nullptr, wk, c, s);
                    char *const to = tile + sl.head * (LANES * 272) + (tok0 + t) * 16;
                    *reinterpret_cast<u32x2 *>(to + (lane.a >> 3) * 272 + (lane.a & 7) * 2) = narrow4<E>(a);
                    *reinterpret_cast<u32x2 *>(to + (lane.b >> 3) * 272 + (lane.b & 7) * 2) = narrow4<E>(b);
                }
            } else {
                const int e0 = lane_id % 16 * 8;
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    const auto word = [&](int u) { return e < 4 ? lo_now[u][e / 2] : hi_now[u][e / 2 - 2]; };
                    const uint32_t pick = e & 1 ? 0x07060302u : 0x05040100u;  // the upper or the lower halves of two words
                    *reinterpret_cast<u32x2 *>(tile + (e0 + e) * 32 + (e0 + e) / 8 * 16 + v_slot(4 * sl.group) * 2) =
                        u32x2{__builtin_amdgcn_perm(word(1), word(0), pick), __builtin_amdgcn_perm(word(3), word(2), pick)};
                }
            }
            __builtin_amdgcn_wave_barrier();
            if (is_k) store_slab_k(tile, A.k_pool + block + (int64_t)x0 * kBlock, kv_elements - x0, n_tok, tok0, lane_id);
            else store_slab_v(tile, A.v_pool + block + (int64_t)x0 * kBlock, kv_elements - x0, n_tok, tok0, lane_id);
            __builtin_amdgcn_wave_barrier();
            continue;
        }
        const int t = (task - 2 * slabs) / chunks, chunk = task - 2 * slabs - t * chunks;
        const bool is_q = chunk < q_chunks;  // (uniform)
        float c[4], s[4];
        angles(t, c, s);
        const auto rows = [&](const float (&w)[8], bool normed, int h0, int heads, uint16_t *dst, int head_stride, int at_a, int at_b) {
#pragma unroll
            for (int u = 0; u < kRowsBatch; u++) {
                const int h = h0 + u * GROUPS;
                if (h >= heads) break;
                float a[4], b[4];
                widen4<E>(lo_now[u], a);
                widen4<E>(hi_now[u], b);
                turn_head<D, E>(A, lane.turns, a, b, normed, w, c, s);
                *reinterpret_cast<u32x2 *>(dst + h * head_stride + at_a) = narrow4<E>(a);
                *reinterpret_cast<u32x2 *>(dst + h * head_stride + at_b) = narrow4<E>(b);
            }
        };
        if (is_q)
            rows(wq, A.q_weight != nullptr, chunk * HEADS + group, A.Hq, A.q_out + (int64_t)(row0 + t) * A.Hq * D, D, lane.a, lane.b);
        else if (STORE)  // a single token, into the pool: [D/8][16 tokens][8]
            rows(wk, A.k_weight != nullptr, (chunk - q_chunks) * HEADS + group, A.Hkv, A.k_pool + block + tok0 * 8, kBlock * D,
                 (lane.a >> 3) * (kBlock * 8) + (lane.a & 7), (lane.b >> 3) * (kBlock * 8) + (lane.b & 7));
        else
            rows(wk, A.k_weight != nullptr, (chunk - q_chunks) * HEADS + group, A.Hkv, A.k_out + (int64_t)(row0 + t) * A.Hkv * D, D, lane.a, lane.b);
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
    // A workgroup a segment where there are enough of them, for the fewer angles (8192 tokens, 512 segments, 68 us; two workgroups each 75, four 73); else as many as have a task
    // for each wave (1234 tokens, 32/32 heads, head_dim 64, 94 segments: one 15.8 us, four 7.7, eight 6.6).  Single tokens: two, whose waves store fewer elements of v each
    // (512 of them, 40/8 heads, head_dim 128, one 9.3 us, two 9.0, three 9.8; 8 of them, 32/8, one 4.8, two 4.6).
    const int chunk = 64 / (p->D / 8) * kRowsBatch, most = (kBlock * ((p->Hq + chunk - 1) / chunk + (p->Hkv + chunk - 1) / chunk) + kRowsThreads / 64 - 1) / (kRowsThreads / 64);
    A.splits = p->n_append_prefill > 0 ? (int)std::min<int64_t>(most, std::max<int64_t>(1, kRowsWorkgroups / p->n_append)) : 2;
    const dim3 grid((unsigned)p->n_append, (unsigned)A.splits);
    hipStream_t st = (hipStream_t)stream;
    const int32_t *segments = p->dev + p->off_append, *seg_pos = p->dev + p->off_seg_pos;
    const auto launch = [&](auto dim, auto type, auto store, auto slabs) {
        rows_kernel<decltype(dim)::value, decltype(type), decltype(store)::value, decltype(slabs)::value><<<grid, kRowsThreads, 0, st>>>(A, segments, seg_pos);
    };
    const std::true_type yes;
    const std::false_type no;
    const auto by_store = [&](auto dim, auto type) { !pool ? launch(dim, type, no, no) : p->n_append_prefill > 0 ? launch(dim, type, yes, yes) : launch(dim, type, yes, no); };
    const auto by_type = [&](auto dim) { p->dtype == TC_FP16 ? by_store(dim, Fp16()) : by_store(dim, Bf16()); };
    p->D == 128 ? by_type(std::integral_constant<int, 128>()) : by_type(std::integral_constant<int, 64>());
    return (int)hipGetLastError();
}

}  // namespace tc
