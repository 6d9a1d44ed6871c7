// The 4-bit cache format on the device: parameters of the pools, the quantiser, and the swizzle under
// which a tile of packed rows sits in shared memory.
#pragma once

#include "ac_device.cuh"

namespace acdev {

// Two bf16 at a time; a NaN in either operand comes through.
__device__ __forceinline__ uint32_t bf16x2_max_nan(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t bf16x2_min_nan(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// min(|a|, |b|) of two bf16 at a time; the sign of the result means nothing.
__device__ __forceinline__ uint32_t bf16x2_min_abs_nan(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("min.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// Two fp32 values in a 64-bit register, operated on by one instruction (each half rounded as on its own).
__device__ __forceinline__ uint64_t f32x2(float lo, float hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void f32x2_split(uint64_t v, float& lo, float& hi) {
    asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ uint64_t f32x2_add(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t f32x2_mul(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t f32x2_fma(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

// What the fast path below cannot decide; out of line, so that it costs the fast path no registers.
__device__ __noinline__ inline uint32_t q4_scale_f64(float lo, float hi) {
    const double range = __dsub_rn(static_cast<double>(hi), static_cast<double>(lo));
    const float s32 = __double2float_rn(__ddiv_rn(range, 15.0));
    return pack_bf16x2(s32, 0.0f) & 0x7FFFu;               // a group of both zeros may give -0: the scale is +0
}
__device__ __noinline__ inline uint32_t q4_code_f64(float x, float lo, float s) {
    const double q = __ddiv_rn(__dsub_rn(static_cast<double>(x), static_cast<double>(lo)), static_cast<double>(s));
    return static_cast<uint32_t>(fminf(static_cast<float>(rint(q)), 15.0f));
}
__device__ __forceinline__ uint32_t q4_code_slow(float x, float lo, float s, float r) {
    const float t = __fsub_rn(x, lo), back = __fsub_rn(t, x);               // TwoSum: what t lost
    const float lost = __fadd_rn(__fsub_rn(x, __fsub_rn(t, back)), __fsub_rn(-lo, back));
    if (!(s >= 0x1p-100f && lost == 0.0f)) return q4_code_f64(x, lo, s);    // (lost is NaN where t overflowed)
    // c is off by one at most; d = t - c s is exact
    const float c = rintf(__fmul_rn(t, r));
    const float d = __fmaf_rn(-c, s, t), half = 0.5f * s;
    uint32_t code = static_cast<uint32_t>(c);
    if (fabsf(d) > half || (fabsf(d) == half && (code & 1u))) code += d > 0.0f ? 1u : 0xffffffffu;
    return code;
}
// Eight codes, side by side, of four words of two bf16 each.
__device__ __noinline__ inline uint32_t q4_codes_slow(uint32_t x0, uint32_t x1, uint32_t x2, uint32_t x3, float lo, float s, float r) {
    if (!(s > 0.0f)) return 0u;
    uint32_t codes = 0u;
#pragma unroll 1
    for (int w = 0; w < 4; ++w) {
        const uint32_t x = w == 0 ? x0 : w == 1 ? x1 : w == 2 ? x2 : x3;
        codes |= (q4_code_slow(__uint_as_float(x << 16), lo, s, r) |
                  (q4_code_slow(__uint_as_float(x & 0xFFFF0000u), lo, s, r) << 4)) << (8 * w);
    }
    return codes;
}

// Quantises W words of two bf16 per lane.  A group is the elements of LANES consecutive, aligned lanes, all of
// which must call this together with `mask` the lanes that execute it.  On return `packed` holds the lane's codes in
// order, eight to a word from the low nibble on, and every lane of the group gets its (s, m) as two bf16, s in the
// low half.
//
// Arithmetic.  Minimum and maximum are exact (kept as the pair (max, -min), one shuffle and one instruction a step;
// NaN comes through, an infinity shows in them).  The format's fp64 quotients are evaluated in fp32 wherever
// that provably rounds alike:
//   scale  s32 = fl(fl(max - min) / 15) is within 2^-22 relative (four of its own ulps) of the quotient, so the bf16
//          next to it is the right one unless the 16 bits cut off lie within 8 of the tie; tiny and overflowing
//          ranges are left to fp64;
//   codes  q = t r + (t - (t r) s) r with t = fl(x - m) and r the approximate reciprocal of s is t / s rounded to fp32 but
//          for 2^-44 (one Newton step on a reciprocal good to 2^-22; the residual is exact).  Where every nonzero |x| of the
//          lane, and m, is at least 2^-12 s, x - m and halves of s are multiples of 2^-20 s: t is exact, a quotient that is
//          not a half is at least 2^-20 from it and q stays on its side, and one that is a half comes out as exactly
//          that; rounding q to an integer is then rounding the quotient.  A lane with a smaller element (one in
//          30 warps of normal values) or a zero decides by d = t - c s instead: beyond s / 2 the neighbour is nearer, at s / 2
//          the even one of the two counts, provided t lost nothing; else, and for tiny or overflowing ranges, fp64.
template <int W, int LANES>
__device__ __forceinline__ uint32_t q4_quantise(const uint32_t (&x)[W], uint32_t (&packed)[(W + 3) / 4], uint32_t mask) {
    uint32_t top = x[0], bottom = x[0], least = x[0];
#pragma unroll
    for (int w = 1; w < W; ++w) {
        top = bf16x2_max_nan(top, x[w]);
        bottom = bf16x2_min_nan(bottom, x[w]);
        least = bf16x2_min_abs_nan(least, x[w]);
    }
    bottom ^= 0x80008000u;
    // (max, -min) of the lane: both halves against each other
    uint32_t both = bf16x2_max_nan(__byte_perm(top, bottom, 0x5410), __byte_perm(top, bottom, 0x7632));
#pragma unroll
    for (int off = 1; off < LANES; off <<= 1) both = bf16x2_max_nan(both, __shfl_xor_sync(mask, both, off));
    const float hi = __uint_as_float(both << 16);
    const float lo = -__uint_as_float(both & 0xFFFF0000u);
#pragma unroll
    for (int w = 0; w < (W + 3) / 4; ++w) packed[w] = 0u;
    if (!(fabsf(hi) < INFINITY && fabsf(lo) < INFINITY)) return 0x7FC00000u;   // s = 0, m = NaN
    const float s32 = __fmul_rn(__fsub_rn(hi, lo), 0x1.111112p-4f);            // 1/15 and one rounding
    const uint32_t u = __float_as_uint(s32);
    uint32_t s16 = (u + 0x7FFFu + ((u >> 16) & 1u)) >> 16;
    if (((u & 0xFFFFu) - 0x7FF8u) <= 16u || !(s32 >= 0x1p-100f && s32 <= 0x1p126f)) s16 = q4_scale_f64(lo, hi);
    const float s = __uint_as_float(s16 << 16);
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(s));
    constexpr float kMagic = 12582912.0f;                  // 1.5 * 2^23: adding it rounds to an integer
    // Codes side by side: the bits of code + kMagic are those of kMagic plus the code, whose multiples come off at the end.
    constexpr uint32_t kEight = 0x11111111u, kBits = 0x4B400000u;
    constexpr uint32_t kMagics = kBits * (W >= 4 ? kEight : kEight & ((1u << (8 * (W % 4))) - 1u));
#pragma unroll
    for (int w = 0; w < W; ++w) {
        const uint64_t t = f32x2_add(f32x2(__uint_as_float(x[w] << 16), __uint_as_float(x[w] & 0xFFFF0000u)), f32x2(-lo, -lo));
        const uint64_t q = f32x2_mul(t, f32x2(r, r));
        const uint64_t near = f32x2_fma(f32x2_fma(q, f32x2(-s, -s), t), f32x2(r, r), q);
        float c0, c1;
        f32x2_split(f32x2_add(near, f32x2(kMagic, kMagic)), c0, c1);
        packed[w / 4] += (__float_as_uint(c0) << (8 * (w % 4))) + (__float_as_uint(c1) << (8 * (w % 4) + 4));
    }
#pragma unroll
    for (int w = 0; w < (W + 3) / 4; ++w) packed[w] -= kMagics;
    const float small = fminf(fabsf(__uint_as_float(least << 16)), fabsf(__uint_as_float(least & 0xFFFF0000u)));
    const bool plain = s >= 0x1p-100f && s32 < INFINITY;
    if (!(plain && fminf(small, lo == 0.0f ? INFINITY : fabsf(lo)) >= s * 0x1p-12f)) {
#pragma unroll
        for (int w = 0; w < W; w += 4) {
            packed[w / 4] = q4_codes_slow(x[w], x[w + 1 < W ? w + 1 : w], x[w + 2 < W ? w + 2 : w], x[w + 3 < W ? w + 3 : w], lo, s, r);
            if (w + 4 > W) packed[w / 4] &= (1u << (8 * (W - w))) - 1u;
        }
    }
    // -0 and +0 compare equal, so the minimum of a group that holds both is either; it is kept as +0
    const uint32_t m16 = lo == 0.0f ? 0u : __float_as_uint(lo) >> 16;
    return s16 | (m16 << 16);
}

// Byte offset of 16-byte chunk `chunk` of row `row` in a tile of packed rows of RB bytes (64 or 32).  The rows
// of a 128-byte line are XORed by a line-dependent unit so that one chunk of eight consecutive rows (what an ldmatrix
// phase reads) falls into eight different 16-byte units.  Rows 8 further are 8 * RB bytes further (same unit), and
// chunk ^ 2 of the same row is the offset ^ 32.
template <int RB>
__device__ __forceinline__ uint32_t q4_tile_offset(int row, int chunk) {
    if (RB == 64) {
        const int line = row >> 1;
        const int f = (line & 1) * 2 + ((line >> 1) & 1) * 5;
        return line * 128 + ((((row & 1) * 4 + chunk) ^ f) << 4);
    }
    const int line = row >> 2;
    return line * 128 + ((((row & 3) * 2 + chunk) ^ ((line & 1) * 3)) << 4);
}

// Eight codes -> eight bf16 values c s + m, each rounded once (a bf16 fma), in order: sm = (s, m).  A nibble under the
// exponent of 128 is 128 + c, exact in bf16.
__device__ __forceinline__ uint4 q4_values(uint32_t codes, uint32_t sm) {
    const uint32_t s2 = __byte_perm(sm, sm, 0x1010), m2 = __byte_perm(sm, sm, 0x3232);
    uint32_t y[4];                                         // elements (i, i + 4)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t c128 = ((codes >> (4 * i)) & 0x000F000Fu) | 0x43004300u;
        uint32_t c;
        asm("add.rn.bf16x2 %0, %1, %2;" : "=r"(c) : "r"(c128), "r"(0xC300C300u));     // - 128
        asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(y[i]) : "r"(c), "r"(s2), "r"(m2));
    }
    return make_uint4(__byte_perm(y[0], y[1], 0x5410), __byte_perm(y[2], y[3], 0x5410),
                      __byte_perm(y[0], y[1], 0x7632), __byte_perm(y[2], y[3], 0x7632));
}

// cp.async of 16 bytes; the second form clears the destination instead where `on` is false.
__device__ __forceinline__ void cp_async_16(uint32_t dst, const void* src, uint64_t policy) {
    asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "l"(policy)
                 : "memory");
}
__device__ __forceinline__ void cp_async_16_or_zero(uint32_t dst, const void* src, bool on, uint64_t policy) {
    asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2, %3;" ::"r"(dst), "l"(src),
                 "r"(on ? 16 : 0), "l"(policy)
                 : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// 8x8 transpose of 16-bit elements across the warp.
__device__ __forceinline__ uint32_t movmatrix_trans(uint32_t x) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}

// D(16x8, fp32) += A(16x16, fp16, row) * B(16x8, fp16, col).
__device__ __forceinline__ void mma_f16_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                              uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// The same with nothing to add to.
__device__ __forceinline__ void mma_f16_16816_zero(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                                   uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%10, %10, %10, %10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
}

__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

__device__ __forceinline__ float ex2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

}  // namespace acdev
