// Single-token decode attention over the 4-bit paged cache, one CTA per (request, KV head, split).
//
// Mathematics.  A key element is c s + m (code, scale and minimum of its group), so a score is
//     q . k = sum_groups ( s * sum_i c_i q_i  +  m * sum_i q_i ):
// the sums of codes run on the tensor pipe, the scale and the minimum enter once per group, token and head in
// fp32.  For the second product sum_t p_t (c_t s_t + m_t) the scale goes into the weight, p'_t = p_t s_t, and
// sum_t p_t m_t is one fp32 number per group and head.  Neither side ever widens the codes to their values.
//
// Codes as matrix operands.  A nibble isolated at the low end of a 16-bit half is the fp16 subnormal c * 2^-24,
// and at bit 4 it is 16 c * 2^-24: with one AND two of a word's eight codes are a finished operand register,
// exact and without bias.  The 2^24 and the 1/16 of the odd codes are powers of two and are taken back in q (odd
// elements of the fragment are divided by 16) and in the result.  For V a whole byte (c0 + 16 c1) * 2^-24 and its
// high nibble 16 c1 * 2^-24 are the operands instead, and the even element of the result is the difference of the two
// sums: a byte is one permutation away, which saves the shift.  ldmatrix brings both in place: plain for K, transposed
// (as 16-bit halves, four codes of one token) for V.
//
// Tiles.  The codes are the 16-row A operand of mma.m16n8k16 and the query heads its 8 columns (two column
// blocks for groups of 9-16 heads), S^T = K Q^T and O^T = V^T P^T: a KV tile costs half the instructions that it
// costs with the heads as rows.  The accumulator layout of S^T (rows = tokens) is turned into the B operand
// of the second product by an 8x8 transpose between lanes (movmatrix).  The order of the elements inside the
// k dimension is free, so a lane's codes are taken in the order in which they lie in memory.
//
// Weights in fp16: p is relative to a reference that may lag the running maximum by up to 8 (powers of two),
// so that most tiles need no reduction across the warp; p' is kept below 2^15 by a power of two that follows
// the largest V scale seen.  The row's result does not depend on either beyond rounding.
//
// Data movement.  Every warp streams tiles of 32 tokens through its own ring with cp.async (16 bytes a lane,
// zero fill for pages outside the pool); no CTA-wide synchronisation in the main loop.
//
// Bound: HBM in principle, with the arithmetic right behind it.  4 rows of 131072 tokens, 64:8 heads of 128, group 64 (604
// MB): the loads alone take 92 to 97 us, the arithmetic alone 93 (each measured with the other taken out), both
// together 111 us = 5440 GB/s, 0.83 of the measured copy rate of 6546 (a stream that only reads reaches 7400: 0.74);
// back to back for a second or more the board's power limit makes it 135.  64 rows of 128 to 8192 tokens, 32:8 heads
// (285 MB): 58 us = 4900 GB/s.  The instructions per tile are those of unpacking (ALU) and of the per-token scales;
// the fp32 arithmetic is done on pairs of heads (add, mul and fma on f32x2: 120.6 -> 116.0 us at 4 splits).
#include <limits.h>
#include <math.h>

#include "ac_internal.h"
#include "q4_format.cuh"
#include "split_merge.cuh"

namespace ac {
namespace {

using namespace acdev;

constexpr int TILE = 32;                      // tokens per stage
constexpr int GRAN = 16;                      // tokens that are sure to share a page
constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;
constexpr float kLag = 8.0f;                  // how far (in powers of two) the softmax reference may lag
constexpr float kLowest = -3.0e38f;           // reference of a warp that has seen no token

// N consecutive words of shared memory, aligned to their size, in one load.
template <int N>
__device__ __forceinline__ void load_words(uint32_t (&w)[N], const uint8_t* src) {
    if constexpr (N == 1) {
        w[0] = *reinterpret_cast<const uint32_t*>(src);
    } else if constexpr (N == 2) {
        const uint2 v = *reinterpret_cast<const uint2*>(src);
        w[0] = v.x, w[1] = v.y;
    } else {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            const uint4 v = reinterpret_cast<const uint4*>(src)[i];
            w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
        }
    }
}

template <int D, int G, int NW, int STAGES>
struct Q4Smem {
    static constexpr int RB = D / 2;                          // bytes of a token's codes
    static constexpr int PB = 8 * G;                          // bytes of a token's parameters
    static constexpr int K_BYTES = TILE * RB;
    static constexpr int P_BYTES = TILE * PB;
    static constexpr int STAGE_BYTES = 2 * K_BYTES + P_BYTES;  // K codes, V codes, parameters
    static constexpr int RING_BYTES = STAGES * STAGE_BYTES;
    static constexpr int TOTAL = NW * RING_BYTES;
};

struct Q4AttnParams {
    const uint16_t* q;
    Q4View cache;
    const int32_t* block_table;
    const int32_t* context_lens;
    const int32_t* row_order;
    float* partial_o;
    float* partial_lse;
    uint16_t* out;
    uint16_t* out_mirror;                     // always nullptr here (the shared merge knows the field)
    int32_t* arrivals;
    float scale_log2;
    uint32_t gpp;                             // granules per page
    uint32_t gpp_magic;                       // ceil(2^32 / gpp); unused when gpp == 1
    int max_pages_per_seq, new_tokens, num_splits, split_tokens, Hq, Hkv, page_size, num_pages, window, sinks;
};

template <int D, int G, int NT, int NW, int STAGES, int CTAS>
__global__ void __launch_bounds__(NW * 32, CTAS) paged_decode_attn_q4_kernel(const Q4AttnParams p) {
    using L = Q4Smem<D, G, NW, STAGES>;
    constexpr int WARPS = NW, THREADS = NW * 32;
    constexpr int RB = L::RB, PB = L::PB;
    constexpr int CPR = RB / 16;                   // 16-byte chunks per row
    constexpr int NC = D / 32;                     // 16-byte chunks (32 elements) per row
    constexpr int CPG = NC / G;                    // chunks per group

    extern __shared__ __align__(128) uint8_t smem[];

    const int h = blockIdx.x, split = blockIdx.z;
    const int b = p.row_order != nullptr ? p.row_order[blockIdx.y] : static_cast<int>(blockIdx.y);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int g = lane >> 2, t = lane & 3;
    const int HG = p.Hq / p.Hkv;
    const int S = p.num_splits;

    // ---- the row's range: attended tokens laid end to end, in granules of 16 (see the bf16 kernel) ----------
    const int ctx = p.context_lens[b];
    int n_tokens = ctx < 0 ? 0 : ctx + p.new_tokens;
    const long long table_tokens = static_cast<long long>(p.max_pages_per_seq) * p.page_size;
    if (n_tokens > table_tokens) n_tokens = static_cast<int>(table_tokens);
    int tok_lo = 0, window_base = 0, sink_span = 0;
    if (p.window > 0) {
        tok_lo = max(0, n_tokens - p.window);
        if (p.sinks >= tok_lo) {
            tok_lo = 0;
        } else {
            sink_span = (p.sinks + GRAN - 1) / GRAN * GRAN;
            window_base = max(0, tok_lo / GRAN * GRAN - sink_span);
        }
    }
    const int range_tokens = n_tokens - window_base;
    const int tok_begin = split * p.split_tokens;
    // The last split goes on to the row's end: a row that has outgrown the plan is slower, not cut off.
    const int tok_end = split == S - 1 ? range_tokens : min((split + 1) * p.split_tokens, range_tokens);

    auto dependency_sync = [&]() {
        cudaGridDependencySynchronize();
        cudaTriggerProgrammaticLaunchCompletion();
    };
    if (tok_begin >= tok_end) {
        dependency_sync();
        if (split == 0) {                          // a row with no tokens at all: its output is +0
            const size_t o = (static_cast<size_t>(b) * p.Hq + h * HG) * D;
            for (int e = threadIdx.x; e < HG * D; e += THREADS) p.out[o + e] = 0;
        }
        return;
    }

    const int32_t* bt_row = p.block_table + static_cast<size_t>(b) * p.max_pages_per_seq;
    const int n_tiles = (tok_end - tok_begin + TILE - 1) / TILE;
    const int n_my = n_tiles > warp ? (n_tiles - warp + WARPS - 1) / WARPS : 0;
    const uint64_t policy = l2_policy_evict_first();
    auto range0 = [&](int j) { return tok_begin + (warp + j * WARPS) * TILE; };
    // Range positions that are not attended: between the sinks and the window's first token.
    const int hole_lo = tok_lo > 0 ? p.sinks : 0, hole_hi = tok_lo > 0 ? tok_lo - window_base : 0;

    // Where the tiles lie.  The warp looks up the pages of 16 tiles at a time, one granule per lane (lane =
    // tile * 2 + half), and turns them into offsets once; a tile then takes its two by shuffle.  The page ids of the
    // next 16 tiles are loaded ahead.
    auto locate = [&](int j0, int& sub) {          // this lane's granule of the tiles from j0: table index or -1
        const int j = j0 + (lane >> 1);
        const int r = range0(j) + (lane & 1) * GRAN;
        const uint32_t gr = static_cast<uint32_t>(r + (r >= sink_span ? window_base : 0)) / GRAN;
        const uint32_t idx = p.gpp == 1 ? gr : __umulhi(gr, p.gpp_magic);
        sub = static_cast<int>(gr - idx * p.gpp);
        return j < n_my && r < tok_end && idx < static_cast<uint32_t>(p.max_pages_per_seq) ? static_cast<int>(idx) : -1;
    };
    auto load_pages = [&](int j0) {
        int sub;
        const int idx = locate(j0, sub);
        return idx >= 0 ? bt_row[idx] : -1;
    };
    uint32_t gr_off = 0;                           // this lane's granule in the code pools, in units of 16 bytes
    uint32_t gr_param = 0;                         // its index among the parameter granules
    uint32_t gr_ok = 0;                            // bit per lane: the granule has a page (otherwise it reads as zeros)
    auto settle_pages = [&](int j0, int page) {
        int sub;
        locate(j0, sub);
        const bool on = page >= 0 && page < p.num_pages;
        gr_ok = __ballot_sync(0xffffffffu, on);
        gr_off = on ? static_cast<uint32_t>((page * p.cache.stride_page + sub * GRAN * p.cache.stride_token) >> 4) : 0u;
        gr_param = on ? (static_cast<uint32_t>(page) * p.Hkv + h) * p.gpp + sub : 0u;
    };

    // This lane's share of a granule: row lane / CPR (and 8 further at D = 128), chunk lane % CPR.
    constexpr int RPI = 32 / CPR;                  // rows per pass of the warp: 8 or 16
    const int64_t lane_off = static_cast<int64_t>(lane / CPR) * p.cache.stride_token + (lane % CPR) * 16 +
                             static_cast<int64_t>(h) * p.cache.stride_head;
    const uint8_t* const k_lane = p.cache.k_codes + lane_off;
    const uint8_t* const v_lane = p.cache.v_codes + lane_off;
    const int64_t next_rows = static_cast<int64_t>(RPI) * p.cache.stride_token;
    const uint8_t* const k_lane8 = k_lane + next_rows;      // the second pass at D = 128
    const uint8_t* const v_lane8 = v_lane + next_rows;
    const uint32_t ring = smem_addr(smem) + warp * L::RING_BYTES;
    const uint32_t code_dst = ring + q4_tile_offset<RB>(lane / CPR, lane % CPR);
    constexpr int PC = GRAN * PB / 16;             // parameter chunks per granule: 8, 16 or 32
    const uint8_t* const p_lane = reinterpret_cast<const uint8_t*>(p.cache.params) + lane % PC * 16;
    // Each address is one widening multiply-add on a lane's base pointer (the FMA pipe: the integer pipe is the
    // busy one here).
    auto issue = [&](int j, uint32_t stage) {      // stage = byte offset of the stage in the ring
        const int src = 2 * (j & 15);
        const uint32_t ok = (gr_ok >> src) & 3u;
        auto load = [&](auto copy) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const uint64_t off = static_cast<uint64_t>(__shfl_sync(0xffffffffu, gr_off, src + half)) * 16u;
                const bool on = (ok >> half) & 1u;
#pragma unroll
                for (int i = 0; i < GRAN / RPI; ++i) {
                    const uint32_t dst = code_dst + stage + (half * GRAN + i * RPI) * RB;   // whole lines: same swizzle
                    copy(dst, (i ? k_lane8 : k_lane) + off, on);
                    copy(dst + L::K_BYTES, (i ? v_lane8 : v_lane) + off, on);
                }
            }
#pragma unroll
            for (int i = 0; i < (2 * PC + 31) / 32; ++i) {
                const int c = i * 32 + lane;
                const int half = (c / PC) & 1;
                const uint32_t granule = __shfl_sync(0xffffffffu, gr_param, src + half);
                if (2 * PC >= 32 || c < 2 * PC)
                    copy(ring + stage + 2 * L::K_BYTES + c * 16, p_lane + static_cast<uint64_t>(granule) * (GRAN * PB),
                         (ok >> half) & 1u);
            }
        };
        if (ok == 3u) load([&](uint32_t dst, const uint8_t* from, bool) { cp_async_16(dst, from, policy); });
        else load([&](uint32_t dst, const uint8_t* from, bool on) { cp_async_16_or_zero(dst, from, on, policy); });
    };

    // ---- prologue: fill the ring; tiles that hold slot ctx - 1 or later wait for the preceding kernel ---------
    const int dependent_from = (ctx > 0 ? ctx - 1 : 0) - window_base;     // range position, maybe negative
    bool dependency_met = false;
    settle_pages(0, load_pages(0));
    int pages_ahead = load_pages(16);
#pragma unroll
    for (int s = 0; s < STAGES; ++s) {
        if (s < n_my) {
            if (!dependency_met && range0(s) + TILE > dependent_from) {
                dependency_sync();
                dependency_met = true;
            }
            issue(s, s * L::STAGE_BYTES);
        }
        cp_async_commit();
    }
    if (!dependency_met) dependency_sync();                                // q was written by the preceding kernel

    // ---- query fragments (B operand): lane (g, t) holds head g (+ 8), elements in the order of K's codes --------
    uint32_t qb[NT][NC][4];
    float qs[NT][G][2], cs[NT][2];                 // sums of q over a group and score factor, heads 2t and 2t + 1
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int head = g + 8 * nt;
        const bool live = head < HG;
        const uint16_t* src = p.q + (static_cast<size_t>(b) * p.Hq + h * HG + (live ? head : 0)) * D;
        float x[NC][8];
        float mx = 0.0f;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const uint4 raw = *reinterpret_cast<const uint4*>(src + c * 32 + t * 8);
            const uint32_t u[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float f = __uint_as_float((e & 1) ? (u[e >> 1] & 0xFFFF0000u) : (u[e >> 1] << 16));
                x[c][e] = live ? f : 0.0f;
                mx = fmaxf(mx, fabsf(x[c][e]));
            }
        }
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
        // power of two that brings the row's largest element into [2^13, 2^14) (fp16 keeps 11 bits down to 2^-14)
        int k = 13 - (max(1, static_cast<int>(__float_as_uint(mx) >> 23)) - 127);
        k = mx > 0.0f ? min(k, 126) : 0;
        const float up = __uint_as_float(static_cast<uint32_t>(k + 127) << 23);
        const float factor = p.scale_log2 * 16777216.0f * __uint_as_float(static_cast<uint32_t>(127 - k) << 23);
        float sum[G];
#pragma unroll
        for (int gq = 0; gq < G; ++gq) {
            sum[gq] = 0.0f;
#pragma unroll
            for (int w = 0; w < CPG; ++w) {
                const int c = gq * CPG + w;
                float y[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    y[e] = x[c][e] * up;
                    sum[gq] += y[e];
                }
                qb[nt][c][0] = pack_f16x2(y[0], y[4]);
                qb[nt][c][1] = pack_f16x2(y[1] * 0.0625f, y[5] * 0.0625f);
                qb[nt][c][2] = pack_f16x2(y[2], y[6]);
                qb[nt][c][3] = pack_f16x2(y[3] * 0.0625f, y[7] * 0.0625f);
            }
            sum[gq] += __shfl_xor_sync(0xffffffffu, sum[gq], 1);
            sum[gq] += __shfl_xor_sync(0xffffffffu, sum[gq], 2);
            sum[gq] *= 5.9604644775390625e-8f;     // 2^-24, the unit of the code products
            qs[nt][gq][0] = __shfl_sync(0xffffffffu, sum[gq], 8 * t);
            qs[nt][gq][1] = __shfl_sync(0xffffffffu, sum[gq], 8 * t + 4);
        }
        cs[nt][0] = __shfl_sync(0xffffffffu, factor, 8 * t);
        cs[nt][1] = __shfl_sync(0xffffffffu, factor, 8 * t + 4);
    }

    // O^T, heads 2t and 2t + 1 as pairs: [chunk][byte 2g + i of it][.][even element, odd element * 16]
    uint64_t o[NC][2][NT][2];
    float m_run[NT][2];
    uint64_t mo[NT][G];
    uint64_t l_run[NT];
    const uint64_t minus_one = f32x2(-1.0f, -1.0f);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        l_run[nt] = 0ull;
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
            m_run[nt][hh] = kLowest;
#pragma unroll
            for (int gq = 0; gq < G; ++gq) mo[nt][gq] = 0ull;
        }
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int i = 0; i < 2; ++i) o[c][i][nt][0] = o[c][i][nt][1] = 0ull;
    }
    // power of two on V's scales: the largest one seen * vf is in [64, 128); before any, so high that one moves it
    float vf = 1.329227995784916e36f;              // 2^120
    float v_top = 0.0f;

    // ldmatrix addresses, the same for K (word t of a row's chunk lands in lane (row, t)) and, transposed, for V (the
    // 16-bit halves of tokens 2t and 2t + 1 side by side): matrices 0 and 1 are rows 0-7 and 8-15 of one chunk, 2 and
    // 3 of the next.
    const uint32_t mat_off = q4_tile_offset<RB>(((lane >> 3) & 1) * 8 + (lane & 7), lane >> 4);

    // tiles before j_hole may hold masked tokens of the hole, those from j_tail on may lie past the end
    const int j_hole = hole_hi > tok_begin ? ((hole_hi - tok_begin + TILE - 1) / TILE - warp + WARPS - 1) / WARPS : 0;
    const int j_tail = (tok_end - tok_begin) % TILE != 0 ? n_my - 1 : n_my;
    uint32_t stage = 0;
    for (int j = 0; j < n_my; ++j) {
        cp_async_wait<STAGES - 1>();
        __syncwarp();
        const uint32_t kt = ring + stage;
        const uint8_t* pt = smem + warp * L::RING_BYTES + stage + 2 * L::K_BYTES;

        // Which of the tile's tokens count: those before the end, and not between the sinks and the window.
        uint32_t valid = 0xffffffffu;
        if (j >= j_tail || j < j_hole) {
            const int r = range0(j) + lane;
            valid = __ballot_sync(0xffffffffu, r < tok_end && !(r >= hole_lo && r < hole_hi));
        }

        // ---- scores ------------------------------------------------------------------------------------------
        float sc[2][NT][4];
        float top[NT][2];
        uint32_t pr[2][2][2 * G];                  // [sub-block][row g / g + 8]: (s, m) of K's groups, then of V's
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) top[nt][0] = top[nt][1] = -INFINITY;
#pragma unroll
        for (int sb = 0; sb < 2; ++sb) {
            load_words(pr[sb][0], pt + (sb * 16 + g) * PB);
            load_words(pr[sb][1], pt + (sb * 16 + 8 + g) * PB);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) sc[sb][nt][0] = sc[sb][nt][1] = sc[sb][nt][2] = sc[sb][nt][3] = 0.0f;
            uint32_t kw[NC][2];                    // word t of rows g and g + 8, per chunk
#pragma unroll
            for (int c = 0; c < NC; c += 2)        // the next two chunks: one bit of the swizzled unit
                ldmatrix_x4(kw[c][0], kw[c][1], kw[c + 1][0], kw[c + 1][1], kt + sb * 16 * RB + (mat_off ^ (c * 16)));
#pragma unroll
            for (int gq = 0; gq < G; ++gq) {
                float acc[NT][4];
#pragma unroll
                for (int w = 0; w < CPG; ++w) {
                    const int c = gq * CPG + w;
                    const uint32_t x0 = kw[c][0], x1 = kw[c][1], y0 = x0 >> 8, y1 = x1 >> 8;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        if (w == 0)
                            mma_f16_16816_zero(acc[nt], x0 & 0x000F000Fu, x1 & 0x000F000Fu, x0 & 0x00F000F0u,
                                               x1 & 0x00F000F0u, qb[nt][c][0], qb[nt][c][1]);
                        else
                            mma_f16_16816(acc[nt], x0 & 0x000F000Fu, x1 & 0x000F000Fu, x0 & 0x00F000F0u, x1 & 0x00F000F0u,
                                          qb[nt][c][0], qb[nt][c][1]);
                        mma_f16_16816(acc[nt], y0 & 0x000F000Fu, y1 & 0x000F000Fu, y0 & 0x00F000F0u, y1 & 0x00F000F0u,
                                      qb[nt][c][2], qb[nt][c][3]);
                    }
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const uint32_t u = pr[sb][r][gq];
                        const float ks = __uint_as_float(u << 16), km = __uint_as_float(u & 0xFFFF0000u);
                        const uint64_t part = f32x2_fma(f32x2(ks, ks), f32x2(acc[nt][2 * r], acc[nt][2 * r + 1]),
                                                        f32x2(sc[sb][nt][2 * r], sc[sb][nt][2 * r + 1]));
                        f32x2_split(f32x2_fma(f32x2(km, km), f32x2(qs[nt][gq][0], qs[nt][gq][1]), part), sc[sb][nt][2 * r],
                                    sc[sb][nt][2 * r + 1]);
                    }
            }
            if (valid != 0xffffffffu) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (!((valid >> (sb * 16 + (e >> 1) * 8 + g)) & 1u)) sc[sb][nt][e] = -INFINITY;
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int hh = 0; hh < 2; ++hh)
                    top[nt][hh] = fmaxf(top[nt][hh], fmaxf(sc[sb][nt][hh], sc[sb][nt][2 + hh]));
        }

        // ---- V parameters, and whether the references still serve -------------------------------------------------
        if (valid != 0xffffffffu) {                // whatever those slots hold: 0 * NaN must not enter the sums
#pragma unroll
            for (int sb = 0; sb < 2; ++sb)
#pragma unroll
                for (int r = 0; r < 2; ++r)
                    if (!((valid >> (sb * 16 + r * 8 + g)) & 1u)) {
#pragma unroll
                        for (int gq = 0; gq < G; ++gq) pr[sb][r][G + gq] = 0u;
                    }
        }
        // the largest V scale of the tile: each lane looks at one token
        uint32_t own[G];
        load_words(own, pt + lane * PB + 4 * G);
        float v_max = 0.0f;
#pragma unroll
        for (int gq = 0; gq < G; ++gq) v_max = fmaxf(v_max, __uint_as_float(own[gq] << 16));
        if (!((valid >> lane) & 1u)) v_max = 0.0f;
        bool move = v_max * vf >= 128.0f;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int hh = 0; hh < 2; ++hh) {
                top[nt][hh] *= cs[nt][hh];
                move = move || top[nt][hh] > m_run[nt][hh] + kLag;
            }
        if (__any_sync(0xffffffffu, move)) {
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) {
                v_max = fmaxf(v_max, __shfl_xor_sync(0xffffffffu, v_max, off));
                if (off < 4) continue;             // lanes (g, t) of one t hold the same heads
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int hh = 0; hh < 2; ++hh)
                        top[nt][hh] = fmaxf(top[nt][hh], __shfl_xor_sync(0xffffffffu, top[nt][hh], off));
            }
            float vr = 1.0f;
            if (v_max > v_top) {
                v_top = v_max;
                int k = 6 - (static_cast<int>(__float_as_uint(v_top) >> 23) - 127);
                k = max(-126, min(k, 120));
                const float next = __uint_as_float(static_cast<uint32_t>(k + 127) << 23);
                vr = next / vf;
                vf = next;
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float alpha[2];
#pragma unroll
                for (int hh = 0; hh < 2; ++hh) {
                    const float m_new = fmaxf(m_run[nt][hh], top[nt][hh]);
                    alpha[hh] = ex2_approx(m_run[nt][hh] - m_new);
                    m_run[nt][hh] = m_new;
                }
                const uint64_t fade = f32x2(alpha[0], alpha[1]);
                l_run[nt] = f32x2_mul(l_run[nt], fade);
#pragma unroll
                for (int gq = 0; gq < G; ++gq) mo[nt][gq] = f32x2_mul(mo[nt][gq], fade);
                const uint64_t both = f32x2(alpha[0] * vr, alpha[1] * vr);
#pragma unroll
                for (int c = 0; c < NC; ++c)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        o[c][i][nt][0] = f32x2_mul(o[c][i][nt][0], both);
                        o[c][i][nt][1] = f32x2_mul(o[c][i][nt][1], both);
                    }
            }
        }

        // ---- weights ------------------------------------------------------------------------------------------------
        uint32_t pb[2][G][NT][2];                  // B operands: weights times V's scales, tokens 2t, 2t + 1 (+ 8) of head g
#pragma unroll
        for (int sb = 0; sb < 2; ++sb) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const uint64_t factor = f32x2(cs[nt][0], cs[nt][1]), less = f32x2(-m_run[nt][0], -m_run[nt][1]);
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    float a, b;
                    f32x2_split(f32x2_fma(f32x2(sc[sb][nt][2 * r], sc[sb][nt][2 * r + 1]), factor, less), a, b);
                    sc[sb][nt][2 * r] = ex2_approx(a);
                    sc[sb][nt][2 * r + 1] = ex2_approx(b);
                    l_run[nt] = f32x2_add(l_run[nt], f32x2(sc[sb][nt][2 * r], sc[sb][nt][2 * r + 1]));
                }
            }
#pragma unroll
            for (int gq = 0; gq < G; ++gq)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const float f = __uint_as_float(pr[sb][r][G + gq] << 16) * vf;
                        const float vm = __uint_as_float(pr[sb][r][G + gq] & 0xFFFF0000u);
                        const uint64_t pair = f32x2(sc[sb][nt][2 * r], sc[sb][nt][2 * r + 1]);
                        float a, b;
                        f32x2_split(f32x2_mul(pair, f32x2(f, f)), a, b);
                        pb[sb][gq][nt][r] = movmatrix_trans(pack_f16x2(a, b));
                        mo[nt][gq] = f32x2_fma(pair, f32x2(vm, vm), mo[nt][gq]);
                    }
        }

        // ---- O^T += V^T P^T -----------------------------------------------------------------------------------------
        // The tile's own sums come from the tensor pipe, starting at zero; the running ones are added in fp32 proper.  The
        // pipe truncates its accumulator at every step, and with codes that are never negative the error of a long
        // chain is a bias: 2700 tokens of a warp in one chain left 3.6 % of the result of 131072 evenly weighted tokens.
#pragma unroll
        for (int c2 = 0; c2 < NC; c2 += 2) {
            uint32_t vw[2][2][2];                  // [granule][chunk c2, c2 + 1][tokens 0-7, 8-15]
#pragma unroll
            for (int sb = 0; sb < 2; ++sb)
                ldmatrix_x4_trans(vw[sb][0][0], vw[sb][0][1], vw[sb][1][0], vw[sb][1][1],
                                  kt + L::K_BYTES + sb * 16 * RB + (mat_off ^ (c2 * 16)));
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                const int c = c2 + w, gq = c / CPG;
                float sum[2][NT][4];
#pragma unroll
                for (int sb = 0; sb < 2; ++sb) {
                    // halves (four codes) of tokens 2t, 2t + 1 in x and of 2t + 8, 2t + 9 in y; then their upper bytes
                    const uint32_t x = vw[sb][w][0], y = vw[sb][w][1];
                    const uint32_t x1 = __byte_perm(x, 0u, 0x4341), y1 = __byte_perm(y, 0u, 0x4341);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        if (sb == 0) {
                            mma_f16_16816_zero(sum[0][nt], x & 0x00FF00FFu, x & 0x00F000F0u, y & 0x00FF00FFu,
                                               y & 0x00F000F0u, pb[sb][gq][nt][0], pb[sb][gq][nt][1]);
                            mma_f16_16816_zero(sum[1][nt], x1, x1 & 0x00F000F0u, y1, y1 & 0x00F000F0u, pb[sb][gq][nt][0],
                                               pb[sb][gq][nt][1]);
                        } else {
                            mma_f16_16816(sum[0][nt], x & 0x00FF00FFu, x & 0x00F000F0u, y & 0x00FF00FFu, y & 0x00F000F0u,
                                          pb[sb][gq][nt][0], pb[sb][gq][nt][1]);
                            mma_f16_16816(sum[1][nt], x1, x1 & 0x00F000F0u, y1, y1 & 0x00F000F0u, pb[sb][gq][nt][0],
                                          pb[sb][gq][nt][1]);
                        }
                    }
                }
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        const uint64_t byte = f32x2(sum[i][nt][0], sum[i][nt][1]), high = f32x2(sum[i][nt][2], sum[i][nt][3]);
                        o[c][i][nt][0] = f32x2_add(o[c][i][nt][0], f32x2_fma(high, minus_one, byte));
                        o[c][i][nt][1] = f32x2_add(o[c][i][nt][1], high);
                    }
            }
        }

        // ---- refill this stage ------------------------------------------------------------------------------------
        __syncwarp();
        if (j + STAGES < n_my) {
            const int next = j + STAGES;
            if ((next & 15) == 0) {
                settle_pages(next, pages_ahead);
                pages_ahead = load_pages(next + 16);
            }
            issue(next, stage);
        }
        cp_async_commit();
        stage = stage + L::STAGE_BYTES == L::RING_BYTES ? 0u : stage + L::STAGE_BYTES;
    }
    cp_async_wait<0>();
    __syncwarp();

    // ---- combine the warps' results through shared memory (each warp reuses its own ring) --------------------------
    constexpr int WROWS = 8 * NT;
    constexpr int WSTRIDE = D + 8;
    static_assert((WROWS * WSTRIDE + 2 * WROWS) * 4 <= L::RING_BYTES, "merge scratch must fit in a ring");
    float* wo = reinterpret_cast<float*>(smem + warp * L::RING_BYTES);
    float* wm = wo + WROWS * WSTRIDE;
    float* wl = wm + WROWS;
    const float back = 16777216.0f, unscale = 1.0f / vf;       // two factors: their product may leave fp32's range
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
            float l_pair[2];
            f32x2_split(l_run[nt], l_pair[0], l_pair[1]);
            float l = l_pair[hh];
#pragma unroll
            for (int off = 4; off < 32; off <<= 1) l += __shfl_xor_sync(0xffffffffu, l, off);
            const int row = 8 * nt + 2 * t + hh;
            if (g == 0) {
                wm[row] = m_run[nt][hh];
                wl[row] = l;
            }
#pragma unroll
            for (int gq = 0; gq < G; ++gq) {
                float m_pair[2];
                f32x2_split(mo[nt][gq], m_pair[0], m_pair[1]);
                float m = m_pair[hh];
#pragma unroll
                for (int off = 4; off < 32; off <<= 1) m += __shfl_xor_sync(0xffffffffu, m, off);
#pragma unroll
                for (int w = 0; w < CPG; ++w) {
                    const int c = gq * CPG + w;
                    float val[4];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        float even[2], odd[2];
                        f32x2_split(o[c][i][nt][0], even[0], even[1]);
                        f32x2_split(o[c][i][nt][1], odd[0], odd[1]);
                        val[2 * i] = even[hh] * back * unscale + m;
                        val[2 * i + 1] = odd[hh] * (back * 0.0625f) * unscale + m;
                    }
                    *reinterpret_cast<float4*>(wo + row * WSTRIDE + c * 32 + g * 4) = make_float4(val[0], val[1], val[2], val[3]);
                }
            }
        }
    __syncthreads();

    constexpr int C4 = D / 4;
    for (int e = threadIdx.x; e < HG * C4; e += THREADS) {
        const int row = e / C4;
        const int col = (e - row * C4) * 4;
        float mw[WARPS];
        float M = kLowest;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            mw[w] = reinterpret_cast<const float*>(smem + w * L::RING_BYTES)[WROWS * WSTRIDE + row];
            M = fmaxf(M, mw[w]);
        }
        float4 num = make_float4(0.f, 0.f, 0.f, 0.f);
        float den = 0.0f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            const float* base = reinterpret_cast<const float*>(smem + w * L::RING_BYTES);
            const float wgt = exp2f(mw[w] - M);
            const float4 o4 = *reinterpret_cast<const float4*>(base + row * WSTRIDE + col);
            num.x = fmaf(wgt, o4.x, num.x);
            num.y = fmaf(wgt, o4.y, num.y);
            num.z = fmaf(wgt, o4.z, num.z);
            num.w = fmaf(wgt, o4.w, num.w);
            den = fmaf(wgt, base[WROWS * WSTRIDE + WROWS + row], den);
        }
        const float4 val = make_float4(num.x / den, num.y / den, num.z / den, num.w / den);
        const size_t hq = static_cast<size_t>(b) * p.Hq + h * HG + row;
        if (S == 1) {
            *reinterpret_cast<uint2*>(p.out + hq * D + col) =
                make_uint2(pack_bf16x2(val.x, val.y), pack_bf16x2(val.z, val.w));
        } else {
            *reinterpret_cast<float4*>(p.partial_o + (hq * S + split) * D + col) = val;
            if (col == 0) p.partial_lse[hq * S + split] = (M + log2f(den)) * LN2;
        }
    }
    if (S == 1) return;

    // ---- the CTA that arrives last for this (request, KV head) merges the splits (see the bf16 kernel) --------------
    __shared__ int s_is_last;
    const int n_active = min(S, (range_tokens + p.split_tokens - 1) / p.split_tokens);
    __syncthreads();
    if (threadIdx.x == 0) {
        int32_t* counter = p.arrivals + static_cast<size_t>(b) * p.Hkv + h;
        int ticket;
        asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], 1;" : "=r"(ticket) : "l"(counter) : "memory");
        s_is_last = ticket == n_active - 1;
        if (s_is_last) *counter = 0;
    }
    __syncthreads();
    if (!s_is_last) return;
    const size_t hq0 = static_cast<size_t>(b) * p.Hq + h * HG;
    const int items = HG * C4;                     // at most 16 * 32 of them, four per thread
    if (items <= THREADS) merge_splits_from_workspace<D, THREADS, 1, 16>(p, hq0, items, S, n_active);
    else if (items <= 2 * THREADS) merge_splits_from_workspace<D, THREADS, 2, 8>(p, hq0, items, S, n_active);
    else merge_splits_from_workspace<D, THREADS, 4, 4>(p, hq0, items, S, n_active);
}

// Shapes of the CTA, all of 8 or 12 warps per SM (the registers of the arithmetic allow no more):
//   FAT    one CTA per SM, for grids of at most that many (4 rows of 131072 tokens in 4 splits: 116 us against 177 in BASE; 8
//          rows of 512 to 2048 tokens: 7.2 against 8.7);
//   BASE   two CTAs per SM: the second one's stream covers the first one's start and end (the same long rows in 9 splits: 111);
//   SLIM   three CTAs of four warps for grids of more than two waves' worth of short splits, where starts and ends are much
//          of a CTA's life (256 rows of 512 to 2048 tokens: 42.1 against 47.1 us in BASE; 64 rows of up to 8192, unsplit: 83
//          against 58, a long row's CTA is alone at the end).  The border between them, kSlimMaxSplitTokens, lies between these
//          two; it was not swept.
// With more than eight heads per KV head the accumulators double: four or eight warps, 255 registers.
enum class Fit { FAT, BASE, SLIM };
constexpr int kSlimMaxSplitTokens = 2560;

template <int D, int G, int NT, Fit F>
struct Q4Shape {
    static constexpr int NW = NT == 2 ? (F == Fit::FAT ? 8 : 4) : F == Fit::FAT ? 12 : F == Fit::BASE ? 6 : 4;
    static constexpr int STAGES = D == 64 ? 4 : 3;
    static constexpr int CTAS = F == Fit::FAT ? 1 : F == Fit::BASE || NT == 2 ? 2 : 3;
    using Smem = Q4Smem<D, G, NW, STAGES>;
};
#define AC_Q4_KERNEL(D_, G_, NT_, F_)                                                                                \
    paged_decode_attn_q4_kernel<D_, G_, NT_, Q4Shape<D_, G_, NT_, F_>::NW, Q4Shape<D_, G_, NT_, F_>::STAGES,          \
                                Q4Shape<D_, G_, NT_, F_>::CTAS>

template <int D, int G, int NT, Fit F>
cudaError_t launch_q4_shape(const Q4AttnParams& p, int B, cudaStream_t stream) {
    using Shape = Q4Shape<D, G, NT, F>;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(p.Hkv, B, p.num_splits);
    cfg.blockDim = dim3(Shape::NW * 32);
    cfg.dynamicSmemBytes = Shape::Smem::TOTAL;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, AC_Q4_KERNEL(D, G, NT, F), p);
}

template <int D, int G, int NT>
cudaError_t launch_q4(const Q4AttnParams& p, int B, int sms, cudaStream_t stream) {
    const long long ctas = static_cast<long long>(B) * p.Hkv * p.num_splits;
    if (ctas <= sms) return launch_q4_shape<D, G, NT, Fit::FAT>(p, B, stream);
    if (NT == 1 && ctas > 2ll * sms && p.split_tokens <= kSlimMaxSplitTokens) return launch_q4_shape<D, G, NT, Fit::SLIM>(p, B, stream);
    return launch_q4_shape<D, G, NT, Fit::BASE>(p, B, stream);
}

template <int D, int G, int NT, Fit F>
cudaError_t set_q4_shape(int smem_optin) {
    constexpr int bytes = Q4Shape<D, G, NT, F>::Smem::TOTAL;
    if (bytes > smem_optin) return cudaErrorInvalidConfiguration;
    return cudaFuncSetAttribute(AC_Q4_KERNEL(D, G, NT, F), cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
}

template <int D, int G, int NT>
cudaError_t set_q4(int smem_optin) {
    cudaError_t e = set_q4_shape<D, G, NT, Fit::FAT>(smem_optin);
    if (e == cudaSuccess) e = set_q4_shape<D, G, NT, Fit::BASE>(smem_optin);
    if (e == cudaSuccess) e = set_q4_shape<D, G, NT, Fit::SLIM>(smem_optin);
    return e;
}

}  // namespace

cudaError_t q4_attn_set_attributes(int smem_optin) {
    cudaError_t e = set_q4<128, 1, 1>(smem_optin);
    if (e == cudaSuccess) e = set_q4<128, 2, 1>(smem_optin);
    if (e == cudaSuccess) e = set_q4<128, 4, 1>(smem_optin);
    if (e == cudaSuccess) e = set_q4<64, 1, 1>(smem_optin);
    if (e == cudaSuccess) e = set_q4<64, 2, 1>(smem_optin);
    if (e == cudaSuccess) e = set_q4<128, 1, 2>(smem_optin);
    if (e == cudaSuccess) e = set_q4<128, 2, 2>(smem_optin);
    if (e == cudaSuccess) e = set_q4<128, 4, 2>(smem_optin);
    if (e == cudaSuccess) e = set_q4<64, 1, 2>(smem_optin);
    if (e == cudaSuccess) e = set_q4<64, 2, 2>(smem_optin);
    return e;
}

cudaError_t launch_paged_decode_attn_q4(const void* q_rot, const Q4View& cache, const int32_t* block_table,
                                        int max_pages_per_seq, const int32_t* context_lens, int new_tokens,
                                        float scale, int num_splits, int split_tokens, float* partial_o,
                                        float* partial_lse, int32_t* arrivals, void* out, int B, int Hq, int Hkv,
                                        int d, int page_size, int num_pages, int window, int sinks,
                                        const int32_t* row_order, cudaStream_t stream) {
    Q4AttnParams p;
    p.q = static_cast<const uint16_t*>(q_rot);
    p.cache = cache;
    p.block_table = block_table;
    p.context_lens = context_lens;
    p.row_order = row_order;
    p.partial_o = partial_o;
    p.partial_lse = partial_lse;
    p.out = static_cast<uint16_t*>(out);
    p.out_mirror = nullptr;
    p.arrivals = arrivals;
    p.scale_log2 = scale * LOG2E;
    p.gpp = static_cast<uint32_t>(page_size / GRAN);
    p.gpp_magic = p.gpp > 1 ? static_cast<uint32_t>(((1ull << 32) + p.gpp - 1) / p.gpp) : 0u;
    p.max_pages_per_seq = max_pages_per_seq;
    p.new_tokens = new_tokens;
    p.num_splits = num_splits;
    p.split_tokens = split_tokens;
    p.Hq = Hq;
    p.Hkv = Hkv;
    p.page_size = page_size;
    p.num_pages = num_pages;
    p.window = window > 0 ? window : 0;
    p.sinks = window > 0 ? sinks : 0;
    int dev = 0;
    cudaGetDevice(&dev);
    const int sms = device_state(dev).sm_count;
    const int groups = d / cache.group;
    const bool wide = Hq / Hkv > 8;
    if (d == 128) {
        if (groups == 1) return wide ? launch_q4<128, 1, 2>(p, B, sms, stream) : launch_q4<128, 1, 1>(p, B, sms, stream);
        if (groups == 2) return wide ? launch_q4<128, 2, 2>(p, B, sms, stream) : launch_q4<128, 2, 1>(p, B, sms, stream);
        return wide ? launch_q4<128, 4, 2>(p, B, sms, stream) : launch_q4<128, 4, 1>(p, B, sms, stream);
    }
    if (groups == 1) return wide ? launch_q4<64, 1, 2>(p, B, sms, stream) : launch_q4<64, 1, 1>(p, B, sms, stream);
    return wide ? launch_q4<64, 2, 2>(p, B, sms, stream) : launch_q4<64, 2, 1>(p, B, sms, stream);
}

}  // namespace ac
