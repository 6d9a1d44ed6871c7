// Rotation of bf16 pairs in fp32 with the bits of the fp64 evaluation (rope_first_half / rope_second_half).
#pragma once

#include "ac_device.cuh"
#include "q4_format.cuh"

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

// Sixteen elements of a vector at a time, with the same result as rope_turn_f32 by half of its instructions.
//
// r = fl(r0 - e) as above.  Its error is at most 1.5 ulp(r), however much cancels: where |r0| < 2^-9 |p|, x c is at least |p| / 2,
// so x c (32 bits) and p are both multiples of 2^-33 |p|, and a difference below 2^-9 |p| of such numbers has at most 24 bits: r0
// is exact, and r has one rounding.  Otherwise |e| < 2^-14 |r0|, and ulp(r0) <= 2 ulp(r).  r (1 + 2^-22) and r (1 - 2^-22) are at
// least two ulps from r on either side; where both round to the same bf16, so does the real value, and the fp64 evaluation.
// That holds in the range where nothing underflows, which is looked up in the results, two at a time, by one
// addition and one maximum (bits below the range wrap to large ones; NaN and infinity are above it).
__device__ __forceinline__ uint64_t f32x2_sub(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("sub.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// The angles of a lane's eight pairs, two to a register.
struct RopeAngles {
    uint64_t c[4], s[4], n[4];                             // cosine, sine, minus sine
    __device__ __forceinline__ void put(int k, const float4& cv, const float4& sv) {
        c[2 * k] = f32x2(cv.x, cv.y), c[2 * k + 1] = f32x2(cv.z, cv.w);
        s[2 * k] = f32x2(sv.x, sv.y), s[2 * k + 1] = f32x2(sv.z, sv.w);
        n[2 * k] = f32x2(-sv.x, -sv.y), n[2 * k + 1] = f32x2(-sv.z, -sv.w);
    }
    __device__ __forceinline__ void set(const float* cos_at, const float* sin_at) {            // from global memory
#pragma unroll
        for (int k = 0; k < 2; ++k)
            put(k, __ldg(reinterpret_cast<const float4*>(cos_at) + k), __ldg(reinterpret_cast<const float4*>(sin_at) + k));
    }
    __device__ __forceinline__ void set_shared(const float* cos_at, const float* sin_at) {
#pragma unroll
        for (int k = 0; k < 2; ++k) put(k, reinterpret_cast<const float4*>(cos_at)[k], reinterpret_cast<const float4*>(sin_at)[k]);
    }
};

// x[0..7]: the words of the lane's 16 elements.  Half-split pairs: words k and k + 4 hold the firsts and the seconds of pairs 2k and
// 2k + 1; interleaved: word j holds pair j.  These are pairs 2k and 2k + 1: out[0], out[1] take the places of their two words; the
// result is zero where all four values are proven, `range` the running maximum of the range test.
template <bool INTERLEAVED>
__device__ __forceinline__ uint32_t rope_turn_two(uint32_t w0, uint32_t w1, uint64_t c, uint64_t s, uint64_t n, uint32_t (&out)[2], uint32_t& range) {
    constexpr uint32_t kLow = (127 - 80) << 7;
    const uint64_t above = f32x2(0x1.000004p0f, 0x1.000004p0f), below = f32x2(0x1.fffff8p-1f, 0x1.fffff8p-1f);
    auto lo = [](uint32_t w) { return __uint_as_float(w << 16); };
    auto hi = [](uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); };
    const uint64_t a = INTERLEAVED ? f32x2(lo(w0), lo(w1)) : f32x2(lo(w0), hi(w0));
    const uint64_t b = INTERLEAVED ? f32x2(hi(w0), hi(w1)) : f32x2(lo(w1), hi(w1));
    const uint64_t p = f32x2_mul(b, n);                    // first: a c - b s
    const uint64_t r = f32x2_sub(f32x2_fma(a, c, p), f32x2_fma(b, s, p));
    const uint64_t p2 = f32x2_mul(a, s);                   // second: b c + a s
    const uint64_t r2 = f32x2_sub(f32x2_fma(b, c, p2), f32x2_fma(a, n, p2));
    float f[2][2], g[2][2];                                // [first, second][pair]: above and below
    f32x2_split(f32x2_mul(r, above), f[0][0], f[0][1]);
    f32x2_split(f32x2_mul(r2, above), f[1][0], f[1][1]);
    f32x2_split(f32x2_mul(r, below), g[0][0], g[0][1]);
    f32x2_split(f32x2_mul(r2, below), g[1][0], g[1][1]);
    uint32_t differ = 0u;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        out[i] = INTERLEAVED ? pack_bf16x2(f[0][i], f[1][i]) : pack_bf16x2(f[i][0], f[i][1]);
        differ |= out[i] ^ (INTERLEAVED ? pack_bf16x2(g[0][i], g[1][i]) : pack_bf16x2(g[i][0], g[i][1]));
        range = __viaddmax_u16x2(out[i] & 0x7FFF7FFFu, (0x10000u - kLow) * 0x10001u, range);
    }
    return differ;
}
__device__ __forceinline__ bool rope_in_range(uint32_t range) {              // 2^-80 to 2^120, as bf16
    constexpr uint32_t kSpan = 200 << 7;
    return __vmaxu2(range, kSpan * 0x10001u) == kSpan * 0x10001u;
}

template <bool INTERLEAVED>
__device__ __forceinline__ void rope_turn16(uint32_t (&x)[8], const RopeAngles& t) {
    uint32_t out[4][2], differ = 0u, range = 0u;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int i0 = INTERLEAVED ? 2 * k : k, i1 = INTERLEAVED ? 2 * k + 1 : k + 4;
        differ |= rope_turn_two<INTERLEAVED>(x[i0], x[i1], t.c[k], t.s[k], t.n[k], out[k], range);
    }
    if (differ != 0u || !rope_in_range(range)) {
        // one warp in sixteen, for a value or two: look for it, and evaluate its pairs in fp64
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t w0 = x[INTERLEAVED ? 2 * k : k], w1 = x[INTERLEAVED ? 2 * k + 1 : k + 4];
            uint32_t again[2], local = 0u;
            if (rope_turn_two<INTERLEAVED>(w0, w1, t.c[k], t.s[k], t.n[k], again, local) == 0u && rope_in_range(local)) continue;
            if (((w0 | w1) & 0x7FFF7FFFu) == 0u) continue; // zeros of the right sign are there already
            float c[2], s[2];
            f32x2_split(t.c[k], c[0], c[1]);
            f32x2_split(t.s[k], s[0], s[1]);
            uint32_t first[2], second[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t aw = INTERLEAVED ? (i ? w1 : w0) << 16 : i ? w0 & 0xFFFF0000u : w0 << 16;
                const uint32_t bw = INTERLEAVED ? (i ? w1 : w0) & 0xFFFF0000u : i ? w1 & 0xFFFF0000u : w1 << 16;
                const float a = __uint_as_float(aw), b = __uint_as_float(bw);
                first[i] = rope_diff_of_products_f64(a, c[i], b, s[i]);
                second[i] = rope_diff_of_products_f64(b, c[i], a, -s[i]);
            }
            out[k][0] = INTERLEAVED ? __byte_perm(first[0], second[0], 0x5410) : __byte_perm(first[0], first[1], 0x5410);
            out[k][1] = INTERLEAVED ? __byte_perm(first[1], second[1], 0x5410) : __byte_perm(second[0], second[1], 0x5410);
        }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        x[INTERLEAVED ? 2 * k : k] = out[k][0];
        x[INTERLEAVED ? 2 * k + 1 : k + 4] = out[k][1];
    }
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
