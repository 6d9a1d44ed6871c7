// Rotary embedding of many tokens per row (prompts), and the tables of cosines and sines for scaled frequencies.
#include <math.h>

#include "ac_internal.h"
#include "rope_fast.cuh"
#include "rope_variant.cuh"

namespace ac {
namespace {

using namespace acdev;

struct RowsParams {
    const uint16_t* q_in;
    uint16_t* q_out;
    const uint16_t* k_in;
    uint16_t* k_out;
    int64_t q_in_token, q_out_token, k_in_token, k_out_token;     // elements from one token to the next
    const int32_t* start_pos;
    const int32_t* row_offsets;
    const float* rope_cos;
    const float* rope_sin;
    const uint16_t* q_norm_w;
    const uint16_t* k_norm_w;
    float norm_eps;
    int max_position, total_tokens, B, Hq, Hkv, rotary_dim, interleaved;
    int chunk, chunks;                                             // heads of one warp, and how many such pieces a token has
    int32_t* status_flag;
};

// Position of a token, or -1 where it has none; the whole warp calls this.  The row is the last one whose offset is <= token:
// each round the 32 lanes look at the ends of 32 equal pieces of what is left.
__device__ __forceinline__ int token_position(const RowsParams& p, int token, int lane) {
    int lo = 0, n = p.B;                                   // the row is in [lo, lo + n)
    while (n > 1) {
        const int piece = (n + 31) / 32;
        const int first = lane * piece;                    // offsets of the pieces' first rows, the first of which is known
        const bool below = lane > 0 && first < n && p.row_offsets[lo + first] <= token;
        const int k = __popc(__ballot_sync(0xffffffffu, below));      // offsets do not decrease: lanes 1 .. k
        lo += k * piece;
        n = min(piece, n - k * piece);
    }
    const int begin = p.row_offsets[lo], end = p.row_offsets[lo + 1];
    const int start = p.start_pos[lo];
    if (token < begin || token >= end || start < 0) return -1;
    const long long pos = static_cast<long long>(start) + (token - begin);
    if (pos >= p.max_position) {
        if (p.status_flag != nullptr && lane == 0) atomicOr(p.status_flag, AC_FLAG_POSITION_OOB);
        return -1;
    }
    return static_cast<int>(pos);
}

// A warp takes `chunk` heads of one token: D/8 lanes per vector, eight elements (16 bytes) each, so that 2 (D = 128) or 4
// vectors are worked on side by side and the token's cosines and sines are loaded once.  A lane's partners in the other
// half are one shuffle away; where pairs are interleaved they are its own elements.
//
// Bound: HBM, 2 bytes in and out per element.  70.3 thousand tokens of 40 heads of 128 (1.44 GB): see the launcher below.
template <int D, bool INTERLEAVED, bool NORM>
__global__ void __launch_bounds__(256) rope_rows_kernel(const RowsParams p) {
    constexpr int LPV = D / 8, VECS = 32 / LPV, U = 4;     // U vectors of a lane in flight
    const int lane = threadIdx.x & 31;
    const long long item = static_cast<long long>(blockIdx.x) * 8 + (threadIdx.x >> 5);
    if (item >= static_cast<long long>(p.total_tokens) * p.chunks) return;
    const int token = static_cast<int>(item / p.chunks);
    const int piece = static_cast<int>(item - static_cast<long long>(token) * p.chunks);
    const int heads = p.Hq + p.Hkv;
    const int h_end = min(heads, (piece + 1) * p.chunk);
    const int at = lane % LPV, h0 = piece * p.chunk + lane / LPV;
    const uint16_t* const q_src = p.q_in + token * p.q_in_token + at * 8;
    const uint16_t* const k_src = p.k_in + token * p.k_in_token + at * 8;

    auto load = [&](uint4 (&x)[U], int h) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int hh = h + u * VECS;
            x[u] = make_uint4(0u, 0u, 0u, 0u);
            if (hh < h_end)
                x[u] = __ldcs(reinterpret_cast<const uint4*>(hh < p.Hq ? q_src + hh * D : k_src + (hh - p.Hq) * D));
        }
    };
    uint4 x[U];
    load(x, h0);                                           // does not wait for the position

    const int pos = token_position(p, token, lane);
    if (pos < 0) return;
    const int half = p.rotary_dim / 2, hl = half / 8;      // lanes of a half
    const bool turned = at * 8 < p.rotary_dim;
    const bool second = !INTERLEAVED && at >= hl;
    const int partner = (lane - at) + (second ? at - hl : at + hl) % LPV;        // of lanes that pass through: anyone
    float c[8], s[8];
    if (turned) {
        const float* cr = p.rope_cos + static_cast<size_t>(pos) * half;
        const float* sr = p.rope_sin + static_cast<size_t>(pos) * half;
        if (INTERLEAVED) {
            const float4 cv = __ldg(reinterpret_cast<const float4*>(cr) + at), sv = __ldg(reinterpret_cast<const float4*>(sr) + at);
            const float cc[4] = {cv.x, cv.y, cv.z, cv.w}, ss[4] = {sv.x, sv.y, sv.z, sv.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                c[2 * i] = c[2 * i + 1] = cc[i];
                s[2 * i] = ss[i];
                s[2 * i + 1] = -ss[i];
            }
        } else {
            const int i0 = (second ? at - hl : at) * 2;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float4 cv = __ldg(reinterpret_cast<const float4*>(cr) + i0 + i), sv = __ldg(reinterpret_cast<const float4*>(sr) + i0 + i);
                const float sign = second ? -1.0f : 1.0f;
                c[4 * i] = cv.x, c[4 * i + 1] = cv.y, c[4 * i + 2] = cv.z, c[4 * i + 3] = cv.w;
                s[4 * i] = sign * sv.x, s[4 * i + 1] = sign * sv.y, s[4 * i + 2] = sign * sv.z, s[4 * i + 3] = sign * sv.w;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) c[i] = s[i] = 0.0f;    // not used
    }

    uint16_t* const q_dst = p.q_out + token * p.q_out_token + at * 8;
    uint16_t* const k_dst = p.k_out + token * p.k_out_token + at * 8;
    for (int h = h0; h < h_end + lane / LPV; h += U * VECS) {      // the same number of rounds for every lane
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int hh = h + u * VECS;
            uint4 v = x[u];
            if (NORM) {
                const bool is_q = hh < p.Hq;
                const uint16_t* w = is_q ? p.q_norm_w : p.k_norm_w;
                const uint32_t raw[4] = {v.x, v.y, v.z, v.w};
                double ss = 0.0;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const double d = static_cast<double>(__uint_as_float((e & 1) ? raw[e >> 1] & 0xFFFF0000u : raw[e >> 1] << 16));
                    ss = __dadd_rn(ss, __dmul_rn(d, d));
                }
#pragma unroll
                for (int off = LPV / 2; off >= 1; off >>= 1) ss = __dadd_rn(ss, __shfl_xor_sync(0xffffffffu, ss, off));
                if (w != nullptr) {
                    const double rr = __ddiv_rn(1.0, __dsqrt_rn(__dadd_rn(__ddiv_rn(ss, static_cast<double>(D)), static_cast<double>(p.norm_eps))));
                    const float rr_hi = static_cast<float>(rr), rr_lo = static_cast<float>(rr - static_cast<double>(rr_hi));
                    const uint4 wv = __ldg(reinterpret_cast<const uint4*>(w) + at);
                    const uint32_t wr[4] = {wv.x, wv.y, wv.z, wv.w};
                    uint32_t y[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        y[e] = rmsnorm_feature(static_cast<uint16_t>(raw[e]), rr, rr_hi, rr_lo, __uint_as_float(wr[e] << 16)) |
                               (static_cast<uint32_t>(rmsnorm_feature(static_cast<uint16_t>(raw[e] >> 16), rr, rr_hi, rr_lo,
                                                                      __uint_as_float(wr[e] & 0xFFFF0000u))) << 16);
                    v = make_uint4(y[0], y[1], y[2], y[3]);
                }
            }
            uint4 other;
            if (INTERLEAVED) {
                other = make_uint4(__byte_perm(v.x, 0u, 0x1032), __byte_perm(v.y, 0u, 0x1032), __byte_perm(v.z, 0u, 0x1032),
                                   __byte_perm(v.w, 0u, 0x1032));
            } else {
                other.x = __shfl_sync(0xffffffffu, v.x, partner);
                other.y = __shfl_sync(0xffffffffu, v.y, partner);
                other.z = __shfl_sync(0xffffffffu, v.z, partner);
                other.w = __shfl_sync(0xffffffffu, v.w, partner);
            }
            if (hh < h_end) {
                if (turned) v = rope_turn8(v, other, c, s);
                __stcs(reinterpret_cast<uint4*>(hh < p.Hq ? q_dst + hh * D : k_dst + (hh - p.Hq) * D), v);
            }
            __syncwarp();
        }
        load(x, h + U * VECS);
    }
}

// The general form, for halves that are no whole number of lanes: a warp per vector, partners through shared memory.
template <int D>
__global__ void __launch_bounds__(256) rope_rows_any_kernel(const RowsParams p) {
    constexpr int EPL = D / 32;
    __shared__ uint16_t s_vec[8][D];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long long item = static_cast<long long>(blockIdx.x) * 8 + warp;
    if (item >= static_cast<long long>(p.total_tokens) * p.chunks) return;
    const int token = static_cast<int>(item / p.chunks);
    const int piece = static_cast<int>(item - static_cast<long long>(token) * p.chunks);
    const int pos = token_position(p, token, lane);
    if (pos < 0) return;
    const int half = p.rotary_dim / 2;
    const int h_end = min(p.Hq + p.Hkv, (piece + 1) * p.chunk);
    for (int h = piece * p.chunk; h < h_end; ++h) {
        const bool is_q = h < p.Hq;
        const uint16_t* src = is_q ? p.q_in + token * p.q_in_token + h * D : p.k_in + token * p.k_in_token + (h - p.Hq) * D;
        uint16_t* dst = is_q ? p.q_out + token * p.q_out_token + h * D : p.k_out + token * p.k_out_token + (h - p.Hq) * D;
        uint16_t x[EPL];
#pragma unroll
        for (int e = 0; e < EPL; ++e) x[e] = src[lane * EPL + e];
        rope_variant_vector<D>(x, is_q ? p.q_norm_w : p.k_norm_w, p.norm_eps, p.rope_cos + static_cast<size_t>(pos) * half,
                               p.rope_sin + static_cast<size_t>(pos) * half, p.rotary_dim, p.interleaved, s_vec[warp], lane);
#pragma unroll
        for (int e = 0; e < EPL; ++e) dst[lane * EPL + e] = x[e];
    }
}

template <int D>
cudaError_t launch_rows(RowsParams p, int sms, cudaStream_t stream) {
    // Pieces of a token: as many as fill the GPU (32 warps per SM) where there are few tokens, of 8 (D = 128) or 16 vectors at least.
    const int heads = p.Hq + p.Hkv;
    constexpr int kLeast = 4 * 32 / (D / 8);
    const long long want = (32ll * sms + p.total_tokens - 1) / p.total_tokens;
    const int most = (heads + kLeast - 1) / kLeast;
    const int chunks = static_cast<int>(want < most ? want : most);
    p.chunk = (heads + chunks - 1) / chunks;
    p.chunk = (p.chunk + kLeast - 1) / kLeast * kLeast;
    p.chunks = (heads + p.chunk - 1) / p.chunk;
    const long long items = static_cast<long long>(p.total_tokens) * p.chunks;
    const long long grid = (items + 7) / 8;
    if (grid > 0x7fffffffll) return cudaErrorInvalidConfiguration;
    const unsigned g = static_cast<unsigned>(grid);
    const bool norm = p.q_norm_w != nullptr || p.k_norm_w != nullptr;
    if (p.rotary_dim % (p.interleaved ? 8 : 16) != 0) rope_rows_any_kernel<D><<<g, 256, 0, stream>>>(p);
    else if (p.interleaved) norm ? rope_rows_kernel<D, true, true><<<g, 256, 0, stream>>>(p) : rope_rows_kernel<D, true, false><<<g, 256, 0, stream>>>(p);
    else norm ? rope_rows_kernel<D, false, true><<<g, 256, 0, stream>>>(p) : rope_rows_kernel<D, false, false><<<g, 256, 0, stream>>>(p);
    return cudaGetLastError();
}

// ---- tables ------------------------------------------------------------------------------------------------
//
// A thread owns one frequency and kRun consecutive positions: cosine and sine of the first position's angle in fp64, then
// one rotation by the frequency's own angle per position (an error of 2^-53 each, 2^-46 after 64 of them: far below the
// fp32 that is written).  Four fp64 operations per pair instead of the hundred of a sine and a cosine.
// Bound: the writes, 4 bytes per entry.
constexpr int kRun = 64;

__global__ void __launch_bounds__(256) rope_tables_kernel(float* __restrict__ cos_out, float* __restrict__ sin_out,
                                                          long long first, int positions, int half, int run, const RopeScaling sc) {
    const long long idx = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x;
    const long long r = idx / half;
    const int i = static_cast<int>(idx - r * half);
    const long long p0 = r * run;
    if (p0 >= positions) return;
    double f = pow(sc.base, -2.0 * i / (2.0 * half));
    if (sc.kind == AC_ROPE_LINEAR) f /= sc.factor;
    if (sc.kind == AC_ROPE_RAMP) {
        const double turns = sc.original * f / 6.283185307179586476925;
        const double keep = fmin(1.0, fmax(0.0, (turns - sc.low) / (sc.high - sc.low)));
        f = keep * f + (1.0 - keep) * f / sc.factor;
    }
    double c, s, cd, sd;
    sincos(static_cast<double>(first + p0) * f, &s, &c);
    sincos(f, &sd, &cd);
    const int n = positions - p0 < run ? static_cast<int>(positions - p0) : run;
    float* co = cos_out + p0 * half + i;
    float* so = sin_out + p0 * half + i;
    for (int j = 0; j < n; ++j) {
        *co = static_cast<float>(sc.magnitude * c);
        *so = static_cast<float>(sc.magnitude * s);
        co += half;
        so += half;
        const double t = c * cd - s * sd;
        s = s * cd + c * sd;
        c = t;
    }
}

}  // namespace

cudaError_t launch_rope_rows(const void* q_in, void* q_out, int64_t q_in_token, int64_t q_out_token, const void* k_in,
                             void* k_out, int64_t k_in_token, int64_t k_out_token, const int32_t* start_pos,
                             const int32_t* row_offsets, int total_tokens, int B, int Hq, int Hkv, int d,
                             const float* rope_cos, const float* rope_sin, int max_position, int32_t* status_flag,
                             const RopeVariant* variant, int sms, cudaStream_t stream) {
    const RopeVariant plain{d, 0, nullptr, nullptr, 0.0f};
    const RopeVariant& r = variant != nullptr ? *variant : plain;
    RowsParams p;
    p.q_in = static_cast<const uint16_t*>(q_in);
    p.q_out = static_cast<uint16_t*>(q_out);
    p.k_in = static_cast<const uint16_t*>(k_in);
    p.k_out = static_cast<uint16_t*>(k_out);
    p.q_in_token = q_in_token;
    p.q_out_token = q_out_token;
    p.k_in_token = k_in_token;
    p.k_out_token = k_out_token;
    p.start_pos = start_pos;
    p.row_offsets = row_offsets;
    p.rope_cos = rope_cos;
    p.rope_sin = rope_sin;
    p.q_norm_w = static_cast<const uint16_t*>(r.q_norm_weight);
    p.k_norm_w = static_cast<const uint16_t*>(r.k_norm_weight);
    p.norm_eps = r.norm_eps;
    p.max_position = max_position;
    p.total_tokens = total_tokens;
    p.B = B;
    p.Hq = Hq;
    p.Hkv = Hkv;
    p.rotary_dim = r.rotary_dim;
    p.interleaved = r.interleaved;
    p.chunk = p.chunks = 0;
    p.status_flag = status_flag;
    return d == 128 ? launch_rows<128>(p, sms, stream) : launch_rows<64>(p, sms, stream);
}

cudaError_t launch_rope_tables(float* rope_cos, float* rope_sin, long long first_position, int positions, int rotary_dim,
                               const RopeScaling& scaling, int sms, cudaStream_t stream) {
    const int half = rotary_dim / 2;
    int run = kRun;                                        // shorter runs where the GPU would not be full
    while (run > 1 && static_cast<long long>((positions + run - 1) / run) * half < 1024ll * sms) run /= 2;
    const long long threads = static_cast<long long>((positions + run - 1) / run) * half;
    const long long grid = (threads + 255) / 256;
    if (grid > 0x7fffffffll) return cudaErrorInvalidConfiguration;
    rope_tables_kernel<<<static_cast<unsigned>(grid), 256, 0, stream>>>(rope_cos, rope_sin, first_position, positions, half, run, scaling);
    return cudaGetLastError();
}

}  // namespace ac
