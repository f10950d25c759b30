// Device-side helpers of the attention kernels (gfx950 only).
#pragma once
#include "w4a8_device.hpp"

namespace w4a8 {

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float v2f __attribute__((ext_vector_type(2)));

constexpr float NEG_INF = -__builtin_huge_valf();

__device__ __forceinline__ v4f mfma_16x16x32_bf16(v8bf a, v8bf b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ v16f mfma_32x32x16_bf16(v8bf a, v8bf b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Two float32 -> two bf16 (round to nearest even), `a` in the low half: one instruction.
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    v2bf r;
    r[0] = (__bf16)a;
    r[1] = (__bf16)b;
    return __builtin_bit_cast(uint32_t, r);
}
// The two E4M3 bytes in the low (HIGH: high) half of w as bf16, exactly.
template <bool HIGH> __device__ __forceinline__ uint32_t e4m3_to_bf16(uint32_t w) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, HIGH));
}

// x of this lane against that of the lane 32 (16) away, in both.
__device__ __forceinline__ float max_over_32(float x) {
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
__device__ __forceinline__ float max_over_16(float x) {
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
__device__ __forceinline__ float sum_over_32(float x) {
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}
__device__ __forceinline__ float sum_over_16(float x) {
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}

// A store that does not stay in L2: what a kernel leaves there is written back at its end, which then waits for it.  16 pages of 64 planes, 32
// KB each, copied 17.3 -> 11.6 us, 400 pages 347 -> 318; ten packed prompts of 1024 tokens 118 -> 110.  (Partial results gain nothing by it.)
template <typename T> __device__ __forceinline__ void stream_out(void* p, T x) { __builtin_nontemporal_store(x, static_cast<T*>(p)); }

// Sum of the two bf16 in w, added to c.
__device__ __forceinline__ float add_pair(uint32_t w, float c) {
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(v2bf, w), __builtin_bit_cast(v2bf, 0x3F803F80u), c, false);
}

// A row's weights are 2^(score - m) with m a maximum of earlier scores: it follows a new one only when that is over 2^RISE times as
// large, so that the sums are seldom scaled again.  Weights up to 2^RISE lose nothing in float32 or bf16.
constexpr float RISE = 8.0f;

// 1 / sum of a finished row of decoding.  Maxima are -infinity only where there are no tokens, LOWEST if tokens have scores of -infinity alone: the
// first gives zeros, the second NaN like 0 / 0.  In a join either counts nothing beside other scores.
constexpr float LOWEST = -3.402823466e38f;
__device__ __forceinline__ float inverse_sum(float m, float l) { return m == NEG_INF ? 0.0f : 1.0f / l; }

// h / s rounded to float32 and then to E4M3, as the activation quantization does it, for values h that are bf16: two instructions a quotient.
// high + low is 1 / s up to 2^-45 of it, so h * low + h * high rounds as h / s does, unless h / s lies within 2^-45 of the middle of two
// neighbouring floats.  That changes the byte only if one of the two is a border of E4M3, of five significant bits: then h 2^j = S (K 2^20 +-
// 1) + e with h of 8 bits, S (the scale's) of 24, K = 16 .. 31 and |e| < 32, so S = A 2^20 + f with A = 8 .. 16 and |f| <= 32, and f K = -+A
// modulo 2^20: only K = A = 16 with S = 2^24 - 1, a scale that takes the division.  low has the sign of s and is never zero: zeros keep
// their sign and infinities meet no zero.  Thirteen prompts of 1 .. 1531 tokens, 32 heads: 135 -> 128 us.
struct Bf16Quantizer {
    float s, high, low;
    bool plain;                                                  // wave-uniform
    __device__ __forceinline__ explicit Bf16Quantizer(float scale) : s(scale), plain(plain_divisor(scale) && (~__float_as_uint(scale) & 0x7FFFFF) != 0) {
        high = 1.0f / scale;
        float rest = fmaf(-scale, high, 1.0f);                   // exact
        if (rest < 0.0f) {                                       // 1 / s rounded away from zero: the float before it
            high = __uint_as_float(__float_as_uint(high) - 1);
            rest = fmaf(-scale, high, 1.0f);
        }
        low = fmaxf(rest, 0x1p-60f) * high;
    }
    __device__ __forceinline__ float quotient(float h) const { return fmaf(h, high, h * low); }
    __device__ __forceinline__ uint32_t four(float a, float b, float c, float d) const {
        if (plain) return cvt2(quotient(c), quotient(d), cvt2(quotient(a), quotient(b), 0u, false), true);
        return cvt2(c / s, d / s, cvt2(a / s, b / s, 0u, false), true);
    }
};

// Four bf16 (two in each word) to four E4M3 bytes, those that the activation quantization makes of them.
__device__ __forceinline__ uint32_t quant_bf16(uint32_t lo, uint32_t hi, const Bf16Quantizer& q) {
    return q.four(__uint_as_float(lo << 16), __uint_as_float(lo & 0xFFFF0000u), __uint_as_float(hi << 16), __uint_as_float(hi & 0xFFFF0000u));
}

// Four finished channels of a row, to 8 bytes of bf16 or to 4 E4M3 bytes of those bf16 values.
__device__ __forceinline__ void store_4(uint16_t* p, float a, float b, float c, float d, const Bf16Quantizer&) {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(a, b), pack_bf16(c, d));
}
__device__ __forceinline__ void store_4(uint8_t* p, float a, float b, float c, float d, const Bf16Quantizer& q) {
    *reinterpret_cast<uint32_t*>(p) = quant_bf16(pack_bf16(a, b), pack_bf16(c, d), q);
}

}  // namespace w4a8
