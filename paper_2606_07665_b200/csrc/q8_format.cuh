// The 8-bit cache format on the device: scales, the quantiser, and codes turned into fp16 operands or fp32 values.
//
// A block of consecutive slots (one page, head and side) has a scale s = 2^e and codes of FMT; a code stands for code * s.
// Powers of two make x / s exact, so a code is one rounding of x whatever it is computed with, and codes that are rounded
// again under a larger scale stay within one step of it: a scale that grows at least doubles, the errors of all growths
// add up to less than s.  With quotients of any size (max |x| / 127) every new maximum of a block would round its codes again, without
// that bound.  What the powers cost int8 (normal values, blocks of 16 tokens of 128; rms error relative to the values): 1.05 %
// stored at once and 1.13 % appended one by one, against 0.83 % and 1.04 %.  e4m3 has the same relative steps under any scale.
#pragma once

#include "ac_device.cuh"
#include "q4_format.cuh"

namespace acdev {

constexpr int Q8_INT8 = 0, Q8_E4M3 = 1;
constexpr uint32_t kQ8NaN = 0x7FC00000u;                   // scale of a block that got an infinity or a NaN

template <int FMT>
__host__ __device__ constexpr float q8_largest() { return FMT == Q8_INT8 ? 127.0f : 448.0f; }

// The scale (fp32 bits) for a largest magnitude, given as the bf16 bits of |x|: the least 2^e with |x| <= M 2^e.  M is 127/64
// or 7/4 of a power of two, so adding the rest of the fraction to the bits carries into the exponent just beyond it.
// Magnitudes that need e > 121 (119) keep that one: M 2^e is then the largest bf16 but one or two steps, and clamped codes
// read back finite.
template <int FMT>
__device__ __forceinline__ uint32_t q8_scale_bits(uint32_t amax) {
    if (amax >= 0x7F80u) return kQ8NaN;
    const int e = static_cast<int>((amax + (FMT == Q8_INT8 ? 1u : 31u)) >> 7) - 127 - (FMT == Q8_INT8 ? 6 : 8);
    return static_cast<uint32_t>(max(-100, min(e, FMT == Q8_INT8 ? 121 : 119)) + 127) << 23;
}

// 1 / s: exact for powers of two.  (NaN for the scale NaN.)
__device__ __forceinline__ float q8_inverse(uint32_t scale_bits) { return __frcp_rn(__uint_as_float(scale_bits)); }

// What a block's scale becomes when a writer that needs `need` finds `held`: the larger one, and NaN stays.  (As bits: the
// scales are positive, and NaN has more bits than any of them.)
__device__ __forceinline__ uint32_t q8_join(uint32_t held, uint32_t need) {
    return held >= 0x7F800000u ? kQ8NaN : max(held, need); // a held scale that is no positive number counts as NaN
}

// Four values, already divided by the scale, as codes in the bytes of a word.  For INT8 they are at most 127 in magnitude, but for
// rounding (see q8_clamp).
template <int FMT>
__device__ __forceinline__ uint32_t q8_codes(uint64_t y01, uint64_t y23) {
    float y0, y1, y2, y3;
    if (FMT == Q8_INT8) {
        // adding 1.5 * 2^23 rounds to the nearest even integer, which is then the low byte of the bits
        const uint64_t magic = f32x2(12582912.0f, 12582912.0f);
        f32x2_split(f32x2_add(y01, magic), y0, y1);
        f32x2_split(f32x2_add(y23, magic), y2, y3);
        return __byte_perm(__byte_perm(__float_as_uint(y0), __float_as_uint(y1), 0x0040),
                           __byte_perm(__float_as_uint(y2), __float_as_uint(y3), 0x0040), 0x5410);
    }
    f32x2_split(y01, y0, y1);
    f32x2_split(y23, y2, y3);
    uint16_t lo, hi;                                       // nearest even; beyond 448 the largest code
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(y1), "f"(y0));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(y3), "f"(y2));
    return lo | (static_cast<uint32_t>(hi) << 16);
}

// Codes of two words of two bf16 each, under the scale whose inverse is `inv`.
template <int FMT>
__device__ __forceinline__ uint32_t q8_quantise(uint32_t w0, uint32_t w1, float inv) {
    const uint64_t both = f32x2(inv, inv);
    return q8_codes<FMT>(f32x2_mul(f32x2(__uint_as_float(w0 << 16), __uint_as_float(w0 & 0xFFFF0000u)), both),
                         f32x2_mul(f32x2(__uint_as_float(w1 << 16), __uint_as_float(w1 & 0xFFFF0000u)), both));
}

// Under the largest scale of INT8, 2^121, the largest bf16 is 127.5 s: its values are taken for 127 s.  Two bf16 at a time; every other
// scale holds its values.
template <int FMT>
__device__ __forceinline__ bool q8_needs_clamp(uint32_t scale_bits) { return FMT == Q8_INT8 && scale_bits == (121u + 127u) << 23; }
__device__ __forceinline__ uint32_t q8_clamp(uint32_t w) { return __vminu2(w & 0x7FFF7FFFu, 0x7F7E7F7Eu) | (w & 0x80008000u); }

// The two codes in the low or high half of a word as fp16 operands: exact.
__device__ __forceinline__ uint32_t q8_e4m3x2_to_f16x2(uint16_t two) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(two));
    return r;
}

// Four codes as two fp16 pairs: bytes (0, 1) and (2, 3) of the word.
template <int FMT>
__device__ __forceinline__ void q8_pairs(uint32_t codes, uint32_t& lo, uint32_t& hi) {
    if (FMT == Q8_INT8) {
        // a byte u = code + 128 under the exponent of 1024 is 1024 + u
        const uint32_t u = codes ^ 0x80808080u;
        asm("add.rn.f16x2 %0, %1, %2;" : "=r"(lo) : "r"(__byte_perm(u, 0x64646464u, 0x4140)), "r"(0xE480E480u));
        asm("add.rn.f16x2 %0, %1, %2;" : "=r"(hi) : "r"(__byte_perm(u, 0x64646464u, 0x4342)), "r"(0xE480E480u));
    } else {
        lo = q8_e4m3x2_to_f16x2(static_cast<uint16_t>(codes));
        hi = q8_e4m3x2_to_f16x2(static_cast<uint16_t>(codes >> 16));
    }
}

// The same for bytes (0, 2) and (1, 3).
template <int FMT>
__device__ __forceinline__ void q8_pairs_across(uint32_t codes, uint32_t& even, uint32_t& odd) {
    if (FMT == Q8_INT8) {
        const uint32_t u = codes ^ 0x80808080u;
        asm("add.rn.f16x2 %0, %1, %2;" : "=r"(even) : "r"(__byte_perm(u, 0x64646464u, 0x4240)), "r"(0xE480E480u));
        asm("add.rn.f16x2 %0, %1, %2;" : "=r"(odd) : "r"(__byte_perm(u, 0x64646464u, 0x4341)), "r"(0xE480E480u));
    } else {
        const uint32_t w = __byte_perm(codes, 0u, 0x3120);
        even = q8_e4m3x2_to_f16x2(static_cast<uint16_t>(w));
        odd = q8_e4m3x2_to_f16x2(static_cast<uint16_t>(w >> 16));
    }
}

// Four codes as fp32 values (without the scale).
template <int FMT>
__device__ __forceinline__ void q8_floats(uint32_t codes, float (&x)[4]) {
    if (FMT == Q8_INT8) {
        const uint32_t u = codes ^ 0x80808080u;            // the same under the exponent of 2^23
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = __fsub_rn(__uint_as_float(__byte_perm(u, 0x4B000000u, 0x7440 + i)), 8388736.0f);
    } else {
        uint32_t lo, hi;
        q8_pairs<FMT>(codes, lo, hi);
        asm("{.reg .b16 a, b; mov.b32 {a, b}, %2; cvt.f32.f16 %0, a; cvt.f32.f16 %1, b;}" : "=f"(x[0]), "=f"(x[1]) : "r"(lo));
        asm("{.reg .b16 a, b; mov.b32 {a, b}, %2; cvt.f32.f16 %0, a; cvt.f32.f16 %1, b;}" : "=f"(x[2]), "=f"(x[3]) : "r"(hi));
    }
}

// Codes of the format rounded again after multiplication by `factor` = 2^-k.
template <int FMT>
__device__ __forceinline__ uint32_t q8_again(uint32_t codes, float factor) {
    float x[4];
    q8_floats<FMT>(codes, x);
    const uint64_t both = f32x2(factor, factor);
    return q8_codes<FMT>(f32x2_mul(f32x2(x[0], x[1]), both), f32x2_mul(f32x2(x[2], x[3]), both));
}

// Largest |x| of two bf16 words, half by half; the sign of the result means nothing, and a NaN comes through.
__device__ __forceinline__ uint32_t bf16x2_amax(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// The larger half of such a maximum over the warp, as bits without sign.
__device__ __forceinline__ uint32_t warp_amax(uint32_t m) {
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) m = bf16x2_amax(m, __shfl_xor_sync(0xffffffffu, m, off));
    return max(m & 0x7FFFu, (m >> 16) & 0x7FFFu);
}

}  // namespace acdev
