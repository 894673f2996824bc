// The KV cache in 8 bits (tc_kvq_pool in tc.h): its kernels and their launchers.
//
//   kvq_append_kernel   quantise this iteration's K/V rows into the pages as they are written   (HBM-bound)
//   kvq_read_kernel     the tokens of sequences back in 16 bits                                 (HBM-bound)
//   the attention kernels of tc_attention.h over such a cache
//
// A (block, KV head) tile of K and one of V have a power of two each as their scale: x is held as the E4M3 number nearest to x 2^-e, and
// stands for that number times 2^e, which is exact in the 16-bit type (four significant bits, and the exponents a scale may have keep it in
// range).  So reading back rounds nothing, and attention is that of the 16-bit path over the values the cache stands for.
#include "tc_attention.h"

namespace tc {

// What depends on the 16-bit type: its infinity, and the exponents that a scale may have.  At the highest one the largest bytes would
// stand for more than the type holds (256 2^8 in IEEE half, 256 2^120 in bf16), so the magnitudes end at 240 there.  At the lowest the
// smallest byte stands for the smallest number of IEEE half, of bf16 for the smallest normal one.
template <class E> struct KvqRange;
template <> struct KvqRange<KvE4m3<Bf16>> { static constexpr int kLow = -117, kHigh = 120; static constexpr uint32_t kInf = 0x7F80; };
template <> struct KvqRange<KvE4m3<Fp16>> { static constexpr int kLow = -15, kHigh = 8; static constexpr uint32_t kInf = 0x7C00; };
constexpr float kE4m3Max = 448.f, kE4m3MaxAtHigh = 240.f;

__device__ __forceinline__ uint32_t pack_bytes(float a, float b, float c, float d) {  // to nearest, ties to even
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
// The bytes of a word at another scale.
__device__ __forceinline__ uint32_t rescale_bytes(uint32_t w, float f) {
    const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    return pack_bytes(a[0] * f, a[1] * f, b[0] * f, b[1] * f);
}
// Rows 0..3 of four bytes each, transposed.
__device__ __forceinline__ void transpose4(const uint32_t (&r)[4], uint32_t (&c)[4]) {
    // __builtin_amdgcn_perm(x, y, s): bytes 0-3 of the result's source are y's, 4-7 x's
    const uint32_t lo01 = __builtin_amdgcn_perm(r[1], r[0], 0x05010400), hi01 = __builtin_amdgcn_perm(r[1], r[0], 0x07030602);
    const uint32_t lo23 = __builtin_amdgcn_perm(r[3], r[2], 0x05010400), hi23 = __builtin_amdgcn_perm(r[3], r[2], 0x07030602);
    c[0] = __builtin_amdgcn_perm(lo23, lo01, 0x05040100);
    c[1] = __builtin_amdgcn_perm(lo23, lo01, 0x07060302);
    c[2] = __builtin_amdgcn_perm(hi23, hi01, 0x05040100);
    c[3] = __builtin_amdgcn_perm(hi23, hi01, 0x07060302);
}
// One tensor's exponent for a page, and how its rows are brought to it.
template <class E>
struct Quantiser {
    using R = KvqRange<E>;
    typedef typename E::t el;
    int e;         // exponent of the scale
    float inv;     // 2^-e
    float limit;   // largest magnitude of a byte
    bool special;  // a new value is an infinity or NaN (wave-uniform)
    // Magnitudes of a word's two elements as 16-bit patterns, which are in the order of the numbers; infinities and NaN count as zero.
    static __device__ __forceinline__ uint32_t larger(uint32_t m, uint32_t w, uint32_t &beyond) {
        const uint32_t a = w & 0x7FFF, b = (w >> 16) & 0x7FFF;
        beyond = max(beyond, max(a, b));
        return max(m, max(a >= R::kInf ? 0u : a, b >= R::kInf ? 0u : b));
    }
    static __device__ __forceinline__ float number(uint32_t pattern) { return (float)__builtin_bit_cast(el, (uint16_t)pattern); }
    // `m`, `beyond`: this lane's largest magnitude, without infinities and NaN and with them.  before: the exponent that the page's older rows have, or kLow.
    __device__ __forceinline__ Quantiser(uint32_t m, uint32_t beyond, int before) {
#pragma unroll
        for (int k = 1; k < 64; k *= 2) m = max(m, (uint32_t)__shfl_xor((int)m, k, 64));
        special = __builtin_amdgcn_ballot_w64(beyond >= R::kInf) != 0;
        // the smallest e with m <= 1.75 * 2^8 * 2^e (zero and numbers too small to be normal in 32 bits: below kLow)
        const uint32_t bits = __float_as_uint(number(m));
        const int need = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7FFFFF) > 0x600000 ? 1 : 0);
        e = __builtin_amdgcn_readfirstlane(max(before, min(max(need, R::kLow), R::kHigh)));
        inv = __uint_as_float((uint32_t)(127 - e) << 23);
        limit = e == R::kHigh ? kE4m3MaxAtHigh : kE4m3Max;
    }
    __device__ __forceinline__ float bounded(float x) const { return __builtin_amdgcn_fmed3f(x * inv, -limit, limit); }
    // four elements, in two words, as bytes
    __device__ __forceinline__ uint32_t bytes(uint32_t w0, uint32_t w1) const {
        uint32_t q = pack_bytes(bounded(number(w0 & 0xFFFF)), bounded(number(w0 >> 16)), bounded(number(w1 & 0xFFFF)), bounded(number(w1 >> 16)));
        if (special) {  // E4M3 has no infinity: NaN for either
            if ((w0 & 0x7FFF) >= R::kInf) q = (q & 0xFFFFFF00u) | 0x7F;
            if (((w0 >> 16) & 0x7FFF) >= R::kInf) q = (q & 0xFFFF00FFu) | 0x7F00;
            if ((w1 & 0x7FFF) >= R::kInf) q = (q & 0xFF00FFFFu) | 0x7F0000;
            if (((w1 >> 16) & 0x7FFF) >= R::kInf) q = (q & 0x00FFFFFFu) | 0x7F000000;
        }
        return q;
    }
};

// A wave writes the rows that one sequence adds to one page (1..16 consecutive token indices) for one KV head: it alone writes the tile, so
// it may read, change and write words of which a part is new.  Where the page has older rows, the exponent can only grow, and
// when it does they are brought to it (exact but for the smallest numbers: a power of two moves their exponents).
// K: a lane owns 16 elements of a token, the 16 bytes of a pool piece.  V: a lane owns eight elements of four tokens, which it transposes in
// registers into the words of the token-minor pool.
template <int D, class E>
__global__ void __launch_bounds__(256) kvq_append_kernel(uint8_t *k_pool, uint8_t *v_pool, uint8_t *scales,
                                                         const uint16_t *__restrict__ k_new, const uint16_t *__restrict__ v_new,
                                                         const int32_t *__restrict__ segments, int Hkv) {
    using Q = Quantiser<E>;
    const int lane = threadIdx.x & 63;
    const int h = blockIdx.y * (blockDim.x >> 6) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (h >= Hkv) return;
    const int32_t *seg = segments + (int64_t)blockIdx.x * kAppendInts;
    const int row0 = seg[0], n_tok = seg[1], tok0 = seg[2], tok1 = tok0 + n_tok;
    const int64_t pair = (int64_t)seg[3] * Hkv + h, tile = pair * (kBlock * D);
    const uint16_t *kn = k_new + ((int64_t)(row0 - tok0) * Hkv + h) * D, *vn = v_new + ((int64_t)(row0 - tok0) * Hkv + h) * D;  // of token index 0
    const int64_t row = (int64_t)Hkv * D;
    uint16_t *const exponents = reinterpret_cast<uint16_t *>(scales + 2 * pair);
    const int before = tok0 > 0 ? *exponents : 0;  // K's, V's << 8

    // ---- the new rows
    constexpr int CK = D / 16, TK = 64 / CK, NP = kBlock / TK;  // K: pieces of a token, tokens of a pass, passes
    const int ck = lane % CK, tk = lane / CK;
    u32x4 kw[NP][2];
    uint32_t k_max = 0, k_beyond = 0, v_max = 0, v_beyond = 0;
#pragma unroll
    for (int p = 0; p < NP; p++) {
        const int t = p * TK + tk;
        kw[p][0] = kw[p][1] = u32x4{0u, 0u, 0u, 0u};
        if (t >= tok0 && t < tok1) {
            const u32x4 *src = reinterpret_cast<const u32x4 *>(kn + t * row + ck * 16);
            kw[p][0] = src[0];
            kw[p][1] = src[1];
        }
    }
    constexpr int CV = D / 8;  // V: eight-element pieces of a token
    const int cv = lane % CV, g = lane / CV;
    u32x4 vw[4];
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const int t = 4 * g + i;
        vw[i] = u32x4{0u, 0u, 0u, 0u};
        if (t >= tok0 && t < tok1) vw[i] = *reinterpret_cast<const u32x4 *>(vn + t * row + cv * 8);
    }
#pragma unroll
    for (int p = 0; p < NP; p++)
#pragma unroll
        for (int x = 0; x < 8; x++) k_max = Q::larger(k_max, kw[p][x >> 2][x & 3], k_beyond);
#pragma unroll
    for (int i = 0; i < 4; i++)
#pragma unroll
        for (int x = 0; x < 4; x++) v_max = Q::larger(v_max, vw[i][x], v_beyond);
    const int k_before = tok0 > 0 ? (before & 0xFF) - 127 : KvqRange<E>::kLow, v_before = tok0 > 0 ? (before >> 8) - 127 : KvqRange<E>::kLow;
    const Q qk(k_max, k_beyond, k_before), qv(v_max, v_beyond, v_before);
    // 448 times 2^-126 is far below half of the smallest byte, as is everything under it
    const float k_shrink = __uint_as_float((uint32_t)(127 + max(k_before - qk.e, -126)) << 23);
    const float v_shrink = __uint_as_float((uint32_t)(127 + max(v_before - qv.e, -126)) << 23);
    const bool k_grows = tok0 > 0 && qk.e > k_before, v_grows = tok0 > 0 && qv.e > v_before;

    // ---- K
#pragma unroll
    for (int p = 0; p < NP; p++) {
        const int t = p * TK + tk;
        u32x4 *dst = reinterpret_cast<u32x4 *>(k_pool + tile + (ck * kBlock + t) * 16);
        if (t >= tok0 && t < tok1) {
            u32x4 w;
#pragma unroll
            for (int x = 0; x < 4; x++) w[x] = qk.bytes(kw[p][x >> 1][2 * (x & 1)], kw[p][x >> 1][2 * (x & 1) + 1]);
            *dst = w;
        } else if (k_grows && t < tok0) {
            u32x4 w = *dst;
#pragma unroll
            for (int x = 0; x < 4; x++) w[x] = rescale_bytes(w[x], k_shrink);
            *dst = w;
        }
    }
    // ---- V
    const uint32_t is_new = first_bytes(tok1 - 4 * g) & ~first_bytes(tok0 - 4 * g), is_old = v_grows ? first_bytes(tok0 - 4 * g) : 0;
    if (g < 4 && (is_new | is_old) != 0) {
#pragma unroll
        for (int half = 0; half < 2; half++) {  // elements 4 half .. + 3 of the eight
            uint32_t r[4], c[4];
#pragma unroll
            for (int i = 0; i < 4; i++) r[i] = qv.bytes(vw[i][2 * half], vw[i][2 * half + 1]);
            transpose4(r, c);
#pragma unroll
            for (int i = 0; i < 4; i++) {
                uint32_t *dst = reinterpret_cast<uint32_t *>(v_pool + tile + v8_word<D>(g, cv * 8 + half * 4 + i));
                if (is_new != 0xFFFFFFFFu) {
                    const uint32_t w = *dst;
                    c[i] = (c[i] & is_new) | (is_old ? (rescale_bytes(w, v_shrink) & is_old) : 0) | (w & ~(is_new | is_old));
                }
                *dst = c[i];
            }
        }
    }
    if (lane == 0) *exponents = (uint16_t)((qk.e + 127) | ((qv.e + 127) << 8));
}

// A wave reads one page of one KV head back: the tokens that are real, widened, at the rows they have in k_out / v_out.
template <int D, class E>
__global__ void __launch_bounds__(256) kvq_read_kernel(const uint8_t *__restrict__ k_pool, const uint8_t *__restrict__ v_pool,
                                                       const uint8_t *__restrict__ scales, const int32_t *__restrict__ pages,
                                                       const int32_t *__restrict__ valid, const int32_t *__restrict__ rows, int Hkv,
                                                       uint16_t *__restrict__ k_out, uint16_t *__restrict__ v_out) {
    const int lane = threadIdx.x & 63;
    const int h = blockIdx.y * (blockDim.x >> 6) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (h >= Hkv) return;
    const int64_t pair = (int64_t)pages[blockIdx.x] * Hkv + h, tile = pair * (kBlock * D);
    const int n = valid[blockIdx.x];
    const int64_t at = ((int64_t)((uint32_t)rows[blockIdx.x] - (uint32_t)rows[0]) * Hkv + h) * D, row = (int64_t)Hkv * D;
    const int exponents = *reinterpret_cast<const uint16_t *>(scales + 2 * pair);
    const float ks = scale_of(exponents & 0xFF), vs = scale_of(exponents >> 8);
    constexpr int CK = D / 16, TK = 64 / CK, NP = kBlock / TK;
    const int ck = lane % CK, tk = lane / CK;
    u32x4 kw[NP];
#pragma unroll
    for (int p = 0; p < NP; p++) kw[p] = *reinterpret_cast<const u32x4 *>(k_pool + tile + (ck * kBlock + p * TK + tk) * 16);
    constexpr int CV = D / 8;
    const int cv = lane % CV, g = lane / CV;
    uint32_t vw[8];
#pragma unroll
    for (int i = 0; i < 8; i++) vw[i] = g < 4 ? *reinterpret_cast<const uint32_t *>(v_pool + tile + v8_word<D>(g, cv * 8 + i)) : 0;
#pragma unroll
    for (int p = 0; p < NP; p++) {
        const int t = p * TK + tk;
        if (t < n) {
            u32x4 *dst = reinterpret_cast<u32x4 *>(k_out + at + t * row + ck * 16);
            dst[0] = __builtin_bit_cast(u32x4, E::widen8(kw[p][0], kw[p][1], ks));
            dst[1] = __builtin_bit_cast(u32x4, E::widen8(kw[p][2], kw[p][3], ks));
        }
    }
    const uint32_t lo[4] = {vw[0], vw[1], vw[2], vw[3]}, hi[4] = {vw[4], vw[5], vw[6], vw[7]};
    uint32_t a[4], b[4];
    transpose4(lo, a);
    transpose4(hi, b);
#pragma unroll
    for (int i = 0; i < 4; i++)
        if (4 * g + i < n) *reinterpret_cast<u32x4 *>(v_out + at + (4 * g + i) * row + cv * 8) = __builtin_bit_cast(u32x4, E::widen8(a[i], b[i], vs));
}

// ------------------------------------------------------------------------------------
// Launchers
// ------------------------------------------------------------------------------------
template <int D, class E>
static int append_d(const tc_plan *p, const tc_kvq_pool *pool, const void *k_new, const void *v_new, hipStream_t st) {
    const int waves = std::min(4, p->Hkv);
    const dim3 grid((unsigned)p->n_append, (unsigned)((p->Hkv + waves - 1) / waves));
    kvq_append_kernel<D, E><<<grid, waves * 64, 0, st>>>((uint8_t *)pool->base.k_pool, (uint8_t *)pool->base.v_pool, (uint8_t *)pool->scales,
                                                        (const uint16_t *)k_new, (const uint16_t *)v_new, p->dev + p->off_append, p->Hkv);
    return (int)hipGetLastError();
}

template <int D, class E>
static int read_d(const tc_plan *p, const tc_kvq_pool *pool, int page0, int n_pages, void *k_out, void *v_out, hipStream_t st) {
    const int waves = std::min(4, p->Hkv);
    const dim3 grid((unsigned)n_pages, (unsigned)((p->Hkv + waves - 1) / waves));
    kvq_read_kernel<D, E><<<grid, waves * 64, 0, st>>>((const uint8_t *)pool->base.k_pool, (const uint8_t *)pool->base.v_pool, (const uint8_t *)pool->scales,
                                                      p->dev + p->off_pages + page0, p->dev + p->off_valid + page0, p->dev + p->off_rows + page0, p->Hkv,
                                                      (uint16_t *)k_out, (uint16_t *)v_out);
    return (int)hipGetLastError();
}

// f(head_dim, element type) for the plan's
template <class F>
static int by_shape(const tc_plan *p, const F &f) {
    if (p->dtype == TC_FP16) return p->D == 128 ? f(Int<128>(), KvE4m3<Fp16>()) : f(Int<64>(), KvE4m3<Fp16>());
    return p->D == 128 ? f(Int<128>(), KvE4m3<Bf16>()) : f(Int<64>(), KvE4m3<Bf16>());
}

int launch_kvq_append(const tc_plan *p, const tc_kvq_pool *pool, const void *k_new, const void *v_new, void *stream) {
    if (p->n_append == 0) return 0;
    return by_shape(p, [&](auto d, auto e) { return append_d<decltype(d)::value, decltype(e)>(p, pool, k_new, v_new, (hipStream_t)stream); });
}

int launch_kvq_read(const tc_plan *p, const tc_kvq_pool *pool, int page0, int n_pages, void *k_out, void *v_out, void *stream) {
    if (n_pages == 0) return 0;
    return by_shape(p, [&](auto d, auto e) { return read_d<decltype(d)::value, decltype(e)>(p, pool, page0, n_pages, k_out, v_out, (hipStream_t)stream); });
}

int launch_kvq_attention(const tc_plan *p, const tc_kvq_pool *pool, const void *q, void *out, float scale, void *workspace, void *stream) {
    const AttnArgs A = attention_args(p, &pool->base, pool->scales, q, nullptr, nullptr, out, scale, workspace, kLaunchFused);
    return by_shape(p, [&](auto d, auto e) { return launch_attention_d<decltype(d)::value, decltype(e)>(p, A, kLaunchFused, (hipStream_t)stream); });
}

}  // namespace tc
