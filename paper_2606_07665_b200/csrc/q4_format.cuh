// The 4-bit cache format on the device: parameters of the pools, the quantiser, and the swizzle under
// which a tile of packed rows sits in shared memory.
#pragma once

#include "ac_device.cuh"

namespace acdev {

// Quantises EPL consecutive elements per lane (bf16 bits).  A group is the elements of LANES consecutive,
// aligned lanes, all of which must call this together with `mask` the lanes that execute it.  On return c[e]
// are the codes, and every lane of the group has the group's (s, m) packed as two bf16 (s in the low half).
//
// Arithmetic, as the format defines it: minimum and maximum are exact; the quotient (max - min) / 15 is an
// fp64 division, rounded to fp32 and then to bf16; the code is rint((x - m) / s) in fp64.  The fp64 division
// is only made where it can matter: t = fl32(x - m) and q = fl32(t / s) are within 2^-22 of the real quotient
// relative (two roundings of 2^-24 each, and the fp64 chain adds 2^-52), q <= 15.1, so |q - quotient| < 4e-6,
// and the fp32 rint decides unless q lies within 1e-4 of a half.
template <int EPL, int LANES>
__device__ __forceinline__ uint32_t q4_quantise(const uint16_t (&x)[EPL], uint32_t (&c)[EPL], uint32_t mask) {
    float f[EPL];
    float lo = INFINITY, hi = -INFINITY;
    uint32_t exponents = 0;                               // all ones in the exponent: infinity or NaN
#pragma unroll
    for (int e = 0; e < EPL; ++e) {
        f[e] = bf16_bits_to_float(x[e]);
        lo = fminf(lo, f[e]);
        hi = fmaxf(hi, f[e]);
        exponents = max(exponents, static_cast<uint32_t>(x[e] & 0x7F80u));
    }
#pragma unroll
    for (int off = 1; off < LANES; off <<= 1) {
        lo = fminf(lo, __shfl_xor_sync(mask, lo, off));
        hi = fmaxf(hi, __shfl_xor_sync(mask, hi, off));
        exponents = max(exponents, __shfl_xor_sync(mask, exponents, off));
    }
    if (exponents == 0x7F80u) {
#pragma unroll
        for (int e = 0; e < EPL; ++e) c[e] = 0u;
        return 0x7FC00000u;                               // s = 0, m = NaN
    }
    const double range = __dsub_rn(static_cast<double>(hi), static_cast<double>(lo));
    const float s32 = __double2float_rn(__ddiv_rn(range, 15.0));
    const uint32_t s16 = pack_bf16x2(s32, 0.0f) & 0x7FFFu;   // a group of both zeros may give -0: the scale is +0
    const float s = __uint_as_float(s16 << 16);
#pragma unroll
    for (int e = 0; e < EPL; ++e) {
        float r = 0.0f;
        if (s > 0.0f) {
            const float q = __fdiv_rn(__fsub_rn(f[e], lo), s);
            r = rintf(q);
            if (!(fabsf(fabsf(q - r) - 0.5f) >= 1e-4f))   // near a half, or x - m beyond fp32
                r = static_cast<float>(rint(__ddiv_rn(__dsub_rn(static_cast<double>(f[e]), static_cast<double>(lo)),
                                                      static_cast<double>(s))));
        }
        c[e] = static_cast<uint32_t>(fminf(r, 15.0f));
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

// cp.async of 16 bytes with zero fill: copies src_bytes (16 or 0) and clears the rest.
__device__ __forceinline__ void cp_async_16(uint32_t dst, const void* src, int src_bytes, uint64_t policy) {
    asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2, %3;" ::"r"(dst), "l"(src),
                 "r"(src_bytes), "l"(policy)
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
