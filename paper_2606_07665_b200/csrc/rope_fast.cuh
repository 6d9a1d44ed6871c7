// Rotation of bf16 pairs in fp32 with the bits of the fp64 evaluation (rope_first_half / rope_second_half).
#pragma once

#include "ac_device.cuh"

namespace acdev {

// x c - y s for x, y of bf16 precision and fp32 c, s, rounded once to bf16.  p = fl(y s) leaves an exact residual
// e = y s - p (one fma), r0 = fl(x c - p) has one rounding of an exact difference, and r = fl(r0 - e).  While |r| is at
// least 2^-20 |p|, e is too small to cancel r0, so r is within ulp(r0)/2 + ulp(r)/2 <= 1.5 ulp(r) of the real value, and
// so is the fp64 evaluation's rounded sum.  Where r is four fp32 ulps clear of every midpoint between bf16 values, all of
// them round to the same bf16.  `open` collects what this does not decide (midpoints 1.4e-4 of all values, deep cancellation,
// tiny and overflowing products, zeros, NaN): such values are evaluated again in fp64.
__device__ __forceinline__ uint32_t rope_turn_f32(float x, float y, float c, float s, bool& open) {
    const float p = __fmul_rn(y, s);
    const float e = __fmaf_rn(y, s, -p);
    const float r = __fsub_rn(__fmaf_rn(x, c, -p), e);
    const uint32_t u = __float_as_uint(r);
    const bool clear = ((u & 0xFFFFu) - 0x7FFCu) > 8u && fabsf(r) >= fmaxf(fabsf(p) * 0x1p-20f, 0x1p-80f) && fabsf(r) <= 0x1p120f;
    open = open || !clear;
    return (u + 0x7FFFu + ((u >> 16) & 1u)) >> 16;
}

// Eight consecutive elements of a vector, as four words of two bf16: out[i] = x[i] c[i] - y[i] s[i], y the partners (or the
// elements themselves, pairwise swapped, for interleaved pairs).  s carries the sign of the half.
__device__ __forceinline__ uint4 rope_turn8(uint4 x, uint4 y, const float (&c)[8], const float (&s)[8]) {
    const uint32_t xw[4] = {x.x, x.y, x.z, x.w}, yw[4] = {y.x, y.y, y.z, y.w};
    uint32_t out[4];
    bool open = false;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const uint32_t lo = rope_turn_f32(__uint_as_float(xw[w] << 16), __uint_as_float(yw[w] << 16), c[2 * w], s[2 * w], open);
        const uint32_t hi = rope_turn_f32(__uint_as_float(xw[w] & 0xFFFF0000u), __uint_as_float(yw[w] & 0xFFFF0000u), c[2 * w + 1], s[2 * w + 1], open);
        out[w] = __byte_perm(lo, hi, 0x5410);
    }
    if (open) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const uint32_t lo = rope_diff_of_products_f64(__uint_as_float(xw[w] << 16), c[2 * w], __uint_as_float(yw[w] << 16), s[2 * w]);
            const uint32_t hi = rope_diff_of_products_f64(__uint_as_float(xw[w] & 0xFFFF0000u), c[2 * w + 1],
                                                          __uint_as_float(yw[w] & 0xFFFF0000u), s[2 * w + 1]);
            out[w] = __byte_perm(lo, hi, 0x5410);
        }
    }
    return make_uint4(out[0], out[1], out[2], out[3]);
}

// One vector held by one warp, element lane * (D/32) + e in x[e]: rotates the first rotary_dim elements as
// rope_variant_vector does without a norm, bit for bit.  `park` is D 16-bit words of shared memory private to the warp.
template <int D>
__device__ __forceinline__ void rope_vector(uint16_t (&x)[D / 32], const float* cos_row, const float* sin_row, int rotary_dim,
                                            int interleaved, uint16_t* park, int lane) {
    constexpr int EPL = D / 32;
    const int half = rotary_dim / 2;
    int partner[EPL];
    float c[EPL], s[EPL];
#pragma unroll
    for (int e = 0; e < EPL; ++e) {
        const int j = lane * EPL + e;
        const bool first = interleaved ? (j & 1) == 0 : j < half;
        const int i = interleaved ? j >> 1 : first ? j : j - half;
        partner[e] = interleaved ? j ^ 1 : first ? j + half : i;
        c[e] = s[e] = 0.0f;
        if (j < rotary_dim) {
            c[e] = cos_row[i];
            s[e] = first ? sin_row[i] : -sin_row[i];
        }
        park[j] = x[e];
    }
    __syncwarp();
#pragma unroll
    for (int e = 0; e < EPL; ++e) {
        if (lane * EPL + e >= rotary_dim) continue;
        const float mine = bf16_bits_to_float(x[e]), other = bf16_bits_to_float(park[partner[e]]);
        bool open = false;
        uint32_t r = rope_turn_f32(mine, other, c[e], s[e], open);
        if (open) r = rope_diff_of_products_f64(mine, c[e], other, s[e]);
        x[e] = static_cast<uint16_t>(r);
    }
    __syncwarp();
}

}  // namespace acdev
