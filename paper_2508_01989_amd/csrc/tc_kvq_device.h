// Device code of the KV cache in 8 bits (tc_kvq_pool in tc.h) that its own kernels (tc_kvq.hip) and the attention kernels
// (tc_attention.h) share: bytes to 16-bit elements and back, the scale of a page, places in a tile.
#pragma once
#include <hip/hip_runtime.h>

#include "tc_internal.h"

namespace tc {

typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

// The element types (Bf16, Fp16 of tc_attention.h) over a cache in 8 bits: a byte times the power of two of its block and KV head is exact in
// either type, so bytes are widened on their way to the matrix cores and everything behind that is as for a cache in 16 bits.
// Both directions are one instruction for two elements, the scale included.
template <class Base>
struct KvE4m3 : Base {
    static constexpr bool kKvq = true;
    static __device__ __forceinline__ typename Base::x4 widen4(uint32_t w, float scale) {
        const auto a = Base::template widen2<false>(w, scale), b = Base::template widen2<true>(w, scale);
        return typename Base::x4{a[0], a[1], b[0], b[1]};
    }
    static __device__ __forceinline__ typename Base::x8 widen8(uint32_t lo, uint32_t hi, float scale) {
        const auto a = widen4(lo, scale), b = widen4(hi, scale);
        return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    // the elements of two words over `scale`, to the nearest E4M3 number, ties to the even one
    static __device__ __forceinline__ uint32_t narrow4(uint32_t w0, uint32_t w1, float scale) {
        s16x2 r = s16x2{0, 0};
        r = Base::template narrow2<false>(r, __builtin_bit_cast(typename Base::x2, w0), scale);
        r = Base::template narrow2<true>(r, __builtin_bit_cast(typename Base::x2, w1), scale);
        return __builtin_bit_cast(uint32_t, r);
    }
};

__device__ __forceinline__ float scale_of(int exponent_byte) { return __uint_as_float((uint32_t)exponent_byte << 23); }
// Bytes t of a word that hold tokens below `n` (the four tokens of a word are consecutive): all bits set, the others zero.
__device__ __forceinline__ uint32_t first_bytes(int n) { return n >= 4 ? 0xFFFFFFFFu : n <= 0 ? 0u : (1u << (8 * n)) - 1u; }
// The top bit of every byte of a word that is NaN (all exponent and mantissa bits set).
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) { return ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u; }
// Where the word of V lies that holds tokens 4 g .. 4 g + 3 of element d, in bytes inside a (block, KV head) tile.
template <int D>
__device__ __forceinline__ int v8_word(int g, int d) { return (((d >> 4) & 1) * 64 + g * 16 + (d & 15)) * (D / 8) + (d >> 5) * 4; }

// The bytes of a word at another scale (f = the old over the new one), to nearest, ties to even.
__device__ __forceinline__ uint32_t rescale_bytes(uint32_t w, float f) {
    const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    const int r = __builtin_amdgcn_cvt_pk_fp8_f32(a[0] * f, a[1] * f, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(b[0] * f, b[1] * f, r, true);
}

// What depends on the element type: its infinity, and the exponents that a scale may have.  At the highest one the largest bytes would
// stand for more than the type holds (256 2^8 in IEEE half, 256 2^120 in bf16), so the magnitudes end at 240 there.  At the lowest the
// smallest byte stands for the smallest number of IEEE half, of bf16 for the smallest normal one.
template <class E> struct KvqRange { static constexpr int kLow = -117, kHigh = 120; static constexpr uint32_t kInf = 0x7F80; };  // bf16
struct Fp16;
template <> struct KvqRange<KvE4m3<Fp16>> { static constexpr int kLow = -15, kHigh = 8; static constexpr uint32_t kInf = 0x7C00; };
constexpr float kE4m3Max = 448.f, kE4m3MaxAtHigh = 240.f;

// Magnitudes of 16-bit elements as their patterns without the sign, which are in the order of the numbers: two to a word.
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
template <int N>
__device__ __forceinline__ uint32_t largest(const uint32_t (&w)[N]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < N; i++) m = max2(m, w[i] & 0x7FFF7FFFu);
    return max(m & 0xFFFFu, m >> 16);
}
// The same without infinities and NaN.
template <class E, int N>
__device__ __forceinline__ uint32_t largest_finite(const uint32_t (&w)[N]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < N; i++) {
        const uint32_t a = w[i] & 0x7FFFu, b = (w[i] >> 16) & 0x7FFFu;
        m = max(m, max(a >= KvqRange<E>::kInf ? 0u : a, b >= KvqRange<E>::kInf ? 0u : b));
    }
    return m;
}
// Both halves of a word, each the largest of the wave's 64 lanes.
__device__ __forceinline__ uint32_t wave_max2(uint32_t m) {
    m = max2(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xF, 0xF, true));   // lane ^ 1
    m = max2(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xF, 0xF, true));   // lane ^ 2
    m = max2(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x141, 0xF, 0xF, true));  // the other four of eight
    m = max2(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x140, 0xF, 0xF, true));  // the other eight of sixteen
    const auto r = __builtin_amdgcn_permlane16_swap(m, m, false, false);
    m = max2(r[0], r[1]);
    const auto s = __builtin_amdgcn_permlane32_swap(m, m, false, false);
    return max2(s[0], s[1]);
}

// One tensor's scale for a page, and how its rows are brought to it.
template <class E>
struct Quantiser {
    using R = KvqRange<E>;
    int e;         // exponent of the scale
    float scale;   // 2^e
    float shrink;  // what the page's older rows are multiplied by
    bool grows;    // the page has older rows, at a smaller scale
    bool special;  // a new element is an infinity or NaN, or beyond the last magnitude
    static __device__ __forceinline__ float number(uint32_t pattern) { return (float)__builtin_bit_cast(typename E::t, (uint16_t)pattern); }
    // `finite`: the largest magnitude of the new elements without infinities and NaN, `all`: with them (both the same in all lanes).  before: the
    // exponent that the page's older rows have, or kLow - 1 where it has none.
    __device__ __forceinline__ Quantiser(uint32_t finite, uint32_t all, int before) {
        // the smallest e for which the magnitude is at most 1.75 * 2^8 * 2^e (zero and numbers too small to be normal in 32 bits: below kLow)
        const uint32_t bits = __float_as_uint(number(finite));
        const int need = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7FFFFF) > 0x600000 ? 1 : 0);
        e = __builtin_amdgcn_readfirstlane(max(before, min(max(need, R::kLow), R::kHigh)));
        scale = scale_of(e + 127);
        grows = before >= R::kLow && e > before;
        shrink = scale_of(127 + max(before - e, -126));  // 448 times 2^-126 is far below half of the smallest byte, as is everything under it
        special = __builtin_amdgcn_readfirstlane((int)(all >= R::kInf || e == R::kHigh)) != 0;
    }
    static __device__ __forceinline__ uint32_t one_special(uint32_t pattern, float inv, float limit) {
        if ((pattern & 0x7FFF) >= R::kInf) return 0x7F;  // E4M3 has no infinity: NaN for either
        const float x = __builtin_amdgcn_fmed3f(number(pattern) * inv, -limit, limit);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x, x, 0, false) & 0xFF;
    }
    // four elements, in two words, as bytes
    __device__ __forceinline__ uint32_t bytes(uint32_t w0, uint32_t w1) const {
        if (special) {  // (wave-uniform)
            const float inv = scale_of(127 - e), limit = e == R::kHigh ? kE4m3MaxAtHigh : kE4m3Max;
            return one_special(w0 & 0xFFFF, inv, limit) | one_special(w0 >> 16, inv, limit) << 8 | one_special(w1 & 0xFFFF, inv, limit) << 16 |
                   one_special(w1 >> 16, inv, limit) << 24;
        }
        return E::narrow4(w0, w1, scale);
    }
};
// K's and V's, from the lanes' shares of the new rows; `before`: the page's exponents + 127 (K's, V's << 8), has_older: whether they count.
template <class E, int NK, int NV>
__device__ __forceinline__ void page_quantisers(const uint32_t (&k)[NK], const uint32_t (&v)[NV], int before, bool has_older, Quantiser<E> &qk, Quantiser<E> &qv) {
    using R = KvqRange<E>;
    const uint32_t all = (uint32_t)__builtin_amdgcn_readfirstlane((int)wave_max2(largest(k) | largest(v) << 16));
    uint32_t finite = all;
    if ((all & 0xFFFF) >= R::kInf || (all >> 16) >= R::kInf)
        finite = (uint32_t)__builtin_amdgcn_readfirstlane((int)wave_max2(largest_finite<E>(k) | largest_finite<E>(v) << 16));
    qk = Quantiser<E>(finite & 0xFFFF, all & 0xFFFF, has_older ? (before & 0xFF) - 127 : R::kLow - 1);
    qv = Quantiser<E>(finite >> 16, all >> 16, has_older ? ((before >> 8) & 0xFF) - 127 : R::kLow - 1);
}

}  // namespace tc
