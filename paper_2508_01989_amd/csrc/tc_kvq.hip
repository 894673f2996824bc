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

// A wave writes the rows that one sequence adds to one page (1..16 consecutive token indices) for one KV head: it alone writes the tile, so
// it may read, change and write words of which a part is new.  Where the page has older rows, the exponent can only grow, and
// when it does they are brought to it (exact but for the smallest numbers: a power of two moves their exponents).
// K: a lane owns 16 elements of a token, the 16 bytes of a pool piece.  V: a lane owns eight elements of four tokens, which it transposes in
// registers into the words of the token-minor pool.
// CHUNK: the batch has a prefill chunk, whose pages may be new as a whole (a batch of decodes takes 5 % less without what that needs).
// Bound: three bytes of memory traffic per new element, two of them read.  8192 tokens, 8 KV heads, head_dim 128 (50.4 MB) take
// 10.1 us, 5.0 TB/s, what a plain copy of 2 GiB reaches.  Small batches are two accesses to memory one after the other, the segment and then everything else: 8
// tokens 4.0 us, 512 tokens of 512 sequences 5.5 (5.0 back to back; with elements quantised one at a time 8.4).  A wave
// to each (page, KV head) needs no barrier.
template <int D, class E, bool CHUNK>
__global__ void __launch_bounds__(256) kvq_append_kernel(uint8_t *k_pool, uint8_t *v_pool, uint8_t *scales,
                                                         const uint16_t *__restrict__ k_new, const uint16_t *__restrict__ v_new,
                                                         const int32_t *__restrict__ segments, int Hkv) {
    const int lane = threadIdx.x & 63;
    const int h = blockIdx.y * (blockDim.x >> 6) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (h >= Hkv) return;
    const int32_t *seg = segments + (int64_t)blockIdx.x * kAppendInts;
    const int row0 = seg[0], n_tok = seg[1], tok0 = seg[2], tok1 = tok0 + n_tok;
    const int64_t pair = (int64_t)seg[3] * Hkv + h, tile = pair * (kBlock * D);
    const uint16_t *kn = k_new + ((int64_t)(row0 - tok0) * Hkv + h) * D, *vn = v_new + ((int64_t)(row0 - tok0) * Hkv + h) * D;  // of token index 0
    const int64_t row = (int64_t)Hkv * D;
    uint16_t *const exponents = reinterpret_cast<uint16_t *>(scales + 2 * pair);
    const int before = tok0 > 0 ? *exponents : 0;

    // ---- everything that is read, requested at once: the new rows, and the words of V of which a part is new
    constexpr int CK = D / 16, TK = 64 / CK, NP = kBlock / TK;  // K: pieces of a token, tokens of a pass, passes
    const int ck = lane % CK, tk = lane / CK;
    uint32_t kw[NP * 8];
#pragma unroll
    for (int p = 0; p < NP; p++) {
        const int t = p * TK + tk;
        u32x4 a = {0u, 0u, 0u, 0u}, b = a;
        if (t >= tok0 && t < tok1) {
            const u32x4 *src = reinterpret_cast<const u32x4 *>(kn + t * row + ck * 16);
            a = src[0];
            b = src[1];
        }
#pragma unroll
        for (int x = 0; x < 4; x++) {
            kw[8 * p + x] = a[x];
            kw[8 * p + 4 + x] = b[x];
        }
    }
    constexpr int CV = D / 8;  // V: eight-element pieces of a token
    const int cv = lane % CV, g = lane / CV;
    uint32_t vw[16];
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const int t = 4 * g + i;
        u32x4 a = {0u, 0u, 0u, 0u};
        if (t >= tok0 && t < tok1) a = *reinterpret_cast<const u32x4 *>(vn + t * row + cv * 8);
#pragma unroll
        for (int x = 0; x < 4; x++) vw[4 * i + x] = a[x];
    }
    const uint32_t is_new = first_bytes(tok1 - 4 * g) & ~first_bytes(tok0 - 4 * g), is_old = first_bytes(tok0 - 4 * g);
    uint32_t *const words = reinterpret_cast<uint32_t *>(v_pool + tile + v8_word<D>(g & 3, cv * 8));  // the lane's eight are D/8 bytes apart
    const bool in_part = is_new != 0 && is_new != 0xFFFFFFFFu;
    uint32_t was[8] = {};
    if (in_part) {
#pragma unroll
        for (int i = 0; i < 8; i++) was[i] = words[i * (D / 32)];
    }
    Quantiser<E> qk(0, 0, 0), qv(0, 0, 0);
    page_quantisers<E>(kw, vw, before, tok0 > 0, qk, qv);

    // ---- K
#pragma unroll
    for (int p = 0; p < NP; p++) {
        const int t = p * TK + tk;
        u32x4 *dst = reinterpret_cast<u32x4 *>(k_pool + tile + (ck * kBlock + t) * 16);
        if (t >= tok0 && t < tok1) {
            u32x4 w;
#pragma unroll
            for (int x = 0; x < 4; x++) w[x] = qk.bytes(kw[8 * p + 2 * x], kw[8 * p + 2 * x + 1]);
            *dst = w;
        } else if (qk.grows && t < tok0) {
            u32x4 w = *dst;
#pragma unroll
            for (int x = 0; x < 4; x++) w[x] = rescale_bytes(w[x], qk.shrink);
            *dst = w;
        }
    }
    // ---- V.  A page that is all new goes through LDS, so that it is stored in whole pieces (a word at a time the stores of a wave touch a line four times): the eight groups
    // of a tile lie 16 bytes further apart there, without which eight lanes of a store would meet on a bank.  (Two still do, 32 words apart, of the 32 lanes that it takes in at
    // once: half of its LDS cycles are conflicts by the counter, which a kernel at the rate of a copy does not notice.)
    constexpr int kLds = CHUNK ? 8 * (2 * D + 16) : 16;  // of a wave
    const auto lds_at = [](int byte) { return byte + byte / (2 * D) * 16; };
    __shared__ __align__(16) char lds_all[4 * kLds];
    char *const lds = lds_all + (threadIdx.x >> 6) * kLds;
    const bool whole = CHUNK && n_tok == kBlock;
    if (qv.grows && is_old != 0) {
        if (!in_part) {
#pragma unroll
            for (int i = 0; i < 8; i++) was[i] = words[i * (D / 32)];
        }
#pragma unroll
        for (int i = 0; i < 8; i++) was[i] = (rescale_bytes(was[i], qv.shrink) & is_old) | (was[i] & ~is_old);
    }
    if (is_new != 0 || (qv.grows && is_old != 0)) {  // (never for lanes past the fourth group)
#pragma unroll
        for (int half = 0; half < 2; half++) {  // elements 4 half .. + 3 of the eight
            uint32_t r[4], c[4];
#pragma unroll
            for (int i = 0; i < 4; i++) r[i] = qv.bytes(vw[4 * i + 2 * half], vw[4 * i + 2 * half + 1]);
            transpose4(r, c);
#pragma unroll
            for (int i = 0; i < 4; i++) {
                if (whole) *reinterpret_cast<uint32_t *>(lds + lds_at(v8_word<D>(g, cv * 8 + 4 * half + i))) = c[i];
                else words[(4 * half + i) * (D / 32)] = (c[i] & is_new) | (was[4 * half + i] & ~is_new);
            }
        }
    }
    if (whole) {
        __builtin_amdgcn_wave_barrier();  // (the LDS is this wave's own, and its accesses complete in order)
#pragma unroll
        for (int k = 0; k < D / 64; k++) {
            const int at = k * 1024 + lane * 16;
            *reinterpret_cast<u32x4 *>(v_pool + tile + at) = *reinterpret_cast<const u32x4 *>(lds + lds_at(at));
        }
    }
    if (lane == 0) *exponents = (uint16_t)((qk.e + 127) | ((qv.e + 127) << 8));
}

// A wave reads one page of one KV head back: the tokens that are real, widened, at the rows they have in k_out / v_out.  Widening is exact, one instruction for
// two elements.  Bound: three bytes of traffic per element, two of them written; the outputs are streamed past the caches, which nothing reads soon.  16 sequences
// of 34300 tokens in all, 8 KV heads, head_dim 128 (211 MB) 37.5 us, 5.6 TB/s (stores through the caches 47.8); one of 1550 tokens 3.8 us, a chain of three accesses.
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
            __builtin_nontemporal_store(__builtin_bit_cast(u32x4, E::widen8(kw[p][0], kw[p][1], ks)), dst);
            __builtin_nontemporal_store(__builtin_bit_cast(u32x4, E::widen8(kw[p][2], kw[p][3], ks)), dst + 1);
        }
    }
    const uint32_t lo[4] = {vw[0], vw[1], vw[2], vw[3]}, hi[4] = {vw[4], vw[5], vw[6], vw[7]};
    uint32_t a[4], b[4];
    transpose4(lo, a);
    transpose4(hi, b);
#pragma unroll
    for (int i = 0; i < 4; i++)
        if (4 * g + i < n) __builtin_nontemporal_store(__builtin_bit_cast(u32x4, E::widen8(a[i], b[i], vs)), reinterpret_cast<u32x4 *>(v_out + at + (4 * g + i) * row + cv * 8));
}

// ------------------------------------------------------------------------------------
// Launchers
// ------------------------------------------------------------------------------------
template <int D, class E>
static int append_d(const tc_plan *p, const tc_kvq_pool *pool, const void *k_new, const void *v_new, hipStream_t st) {
    const int waves = std::min(4, p->Hkv);
    const dim3 grid((unsigned)p->n_append, (unsigned)((p->Hkv + waves - 1) / waves));
    const auto launch = [&](auto kernel) {
        kernel<<<grid, waves * 64, 0, st>>>((uint8_t *)pool->base.k_pool, (uint8_t *)pool->base.v_pool, (uint8_t *)pool->scales, (const uint16_t *)k_new,
                                            (const uint16_t *)v_new, p->dev + p->off_append, p->Hkv);
        return (int)hipGetLastError();
    };
    return p->n_append_prefill > 0 ? launch(kvq_append_kernel<D, E, true>) : launch(kvq_append_kernel<D, E, false>);
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

int launch_kvq_attention(const tc_plan *p, const tc_kvq_pool *pool, const void *q, const void *k_new, const void *v_new, void *out, float scale, void *workspace,
                         void *stream) {
    const AttnArgs A = attention_args(p, &pool->base, pool->scales, q, k_new, v_new, out, scale, workspace, kLaunchFused);
    return by_shape(p, [&](auto d, auto e) { return launch_attention_d<decltype(d)::value, decltype(e)>(p, A, kLaunchFused, (hipStream_t)stream); });
}

}  // namespace tc

#ifdef TC_WG_TRACE
// Tracing build only: tc_debug_wg_trace for launches over a cache in 8 bits.
extern "C" int tc_debug_kvq_wg_trace(long long *dst, int n) {
    (void)hipDeviceSynchronize();
    return (int)hipMemcpyFromSymbol(dst, HIP_SYMBOL(tc::g_wg_trace), (size_t)n * sizeof(long long));
}
#endif
