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
// exact and without bias (five instructions for eight codes).  The 2^24 and the 1/16 of the odd codes are powers
// of two and are taken back in q (odd elements of the fragment are divided by 16) and in the result.
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
// zero fill for pages outside the pool); no CTA-wide synchronisation in the main loop.  Bound: HBM in principle,
// in practice the issue slots of the SM are the close second (about six instructions per cache byte and lane).
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
    static constexpr int TOTAL = NW * RING_BYTES + 128;        // + alignment slack
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
    constexpr int GE = D / G;                      // elements per group
    constexpr int KW = GE / 32;                    // K words (8 codes) per lane, row and group
    constexpr int VE = GE / 8;                     // V elements per lane, token and group: 16, 8 or 4
    constexpr int MT = GE / 16;                    // 16-row tiles of O^T per group

    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (smem_addr(smem_raw) + 127u) & ~127u;
    uint8_t* smem_gen = smem_raw + (smem_base - smem_addr(smem_raw));

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
    const int tok_end = min((split + 1) * p.split_tokens, range_tokens);

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
    const uint32_t ring = smem_base + warp * L::RING_BYTES;
    const int n_tiles = (tok_end - tok_begin + TILE - 1) / TILE;
    const int n_my = n_tiles > warp ? (n_tiles - warp + WARPS - 1) / WARPS : 0;
    const uint64_t policy = l2_policy_evict_first();
    auto range0 = [&](int j) { return tok_begin + (warp + j * WARPS) * TILE; };
    auto token_of = [&](int r) { return r + (r >= sink_span ? window_base : 0); };
    // page-table index and granule inside the page of the granule that starts at token tk
    auto page_index = [&](int tk, int& sub) {
        const uint32_t gr = static_cast<uint32_t>(tk) / GRAN;
        const uint32_t idx = p.gpp == 1 ? gr : __umulhi(gr, p.gpp_magic);
        sub = static_cast<int>(gr - idx * p.gpp);
        return static_cast<int>(idx);
    };
    auto load_page = [&](int j, int half) {        // -1: nothing to read there
        const int r = range0(j) + half * GRAN;
        if (j >= n_my || r >= tok_end) return -1;
        int sub;
        const int idx = page_index(token_of(r), sub);
        return idx < p.max_pages_per_seq ? bt_row[idx] : -1;
    };
    // This lane's share of a granule: row lane / CPR (and 8 further at D = 128), chunk lane % CPR.
    const int64_t lane_off = static_cast<int64_t>(lane / CPR) * p.cache.stride_token + (lane % CPR) * 16 +
                             static_cast<int64_t>(h) * p.cache.stride_head;
    auto issue = [&](int j, int page0, int page1) {
        const uint32_t dst = ring + (j % STAGES) * L::STAGE_BYTES;
        constexpr int RPI = 32 / CPR;              // rows per lane pass: 8 or 16
        const uint8_t* prm[2];
        int ok[2];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int page = half ? page1 : page0;
            const bool on = page >= 0 && page < p.num_pages;
            int sub;
            page_index(token_of(range0(j) + half * GRAN), sub);
            ok[half] = on ? 16 : 0;
            const int64_t pg = on ? page : 0;
            const int slot = on ? sub * GRAN : 0;
            const int64_t off = pg * p.cache.stride_page + slot * p.cache.stride_token + lane_off;
#pragma unroll
            for (int i = 0; i < GRAN / RPI; ++i) {
                const int row = half * GRAN + i * RPI + lane / CPR;
                const uint32_t at = q4_tile_offset<RB>(row, lane % CPR);
                const int64_t o = off + static_cast<int64_t>(i * RPI) * p.cache.stride_token;
                cp_async_16(dst + at, p.cache.k_codes + o, ok[half], policy);
                cp_async_16(dst + L::K_BYTES + at, p.cache.v_codes + o, ok[half], policy);
            }
            prm[half] = reinterpret_cast<const uint8_t*>(p.cache.params) +
                        ((pg * p.Hkv + h) * p.page_size + slot) * PB;
        }
        constexpr int PC = GRAN * PB / 16;         // parameter chunks per granule: 8, 16 or 32
#pragma unroll
        for (int i = 0; i < (2 * PC + 31) / 32; ++i) {
            const int c = i * 32 + lane;
            if (2 * PC >= 32 || c < 2 * PC) {
                const int half = c / PC;
                cp_async_16(dst + 2 * L::K_BYTES + c * 16, (half ? prm[1] : prm[0]) + (c - half * PC) * 16,
                            half ? ok[1] : ok[0], policy);
            }
        }
    };

    // ---- prologue: fill the ring; tiles that hold slot ctx - 1 or later wait for the preceding kernel ---------
    const int dependent_from = (ctx > 0 ? ctx - 1 : 0) - window_base;     // range position, maybe negative
    bool dependency_met = false;
#pragma unroll
    for (int s = 0; s < STAGES; ++s) {
        if (s < n_my) {
            if (!dependency_met && range0(s) + TILE > dependent_from) {
                dependency_sync();
                dependency_met = true;
            }
            issue(s, load_page(s, 0), load_page(s, 1));
        }
        cp_async_commit();
    }
    int next0 = load_page(STAGES, 0), next1 = load_page(STAGES, 1);
    if (!dependency_met) dependency_sync();                                // q was written by the preceding kernel

    // ---- query fragments (B operand): lane (g, t) holds head g (+ 8), elements in the order of K's codes --------
    uint32_t qb[NT][G][KW][4];
    float qs[NT][G][2], cs[NT][2];                 // sums of q over a group and score factor, heads 2t and 2t + 1
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int head = g + 8 * nt;
        const bool live = head < HG;
        const uint16_t* src = p.q + (static_cast<size_t>(b) * p.Hq + h * HG + (live ? head : 0)) * D;
        float x[G][KW][8];
        float mx = 0.0f;
#pragma unroll
        for (int gq = 0; gq < G; ++gq)
#pragma unroll
            for (int w = 0; w < KW; ++w) {
                const uint4 raw = *reinterpret_cast<const uint4*>(src + gq * GE + t * (GE / 4) + w * 8);
                const uint32_t u[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float f = __uint_as_float((e & 1) ? (u[e >> 1] & 0xFFFF0000u) : (u[e >> 1] << 16));
                    x[gq][w][e] = live ? f : 0.0f;
                    mx = fmaxf(mx, fabsf(x[gq][w][e]));
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
            for (int w = 0; w < KW; ++w) {
                float y[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    y[e] = x[gq][w][e] * up;
                    sum[gq] += y[e];
                }
                qb[nt][gq][w][0] = pack_f16x2(y[0], y[4]);
                qb[nt][gq][w][1] = pack_f16x2(y[1] * 0.0625f, y[5] * 0.0625f);
                qb[nt][gq][w][2] = pack_f16x2(y[2], y[6]);
                qb[nt][gq][w][3] = pack_f16x2(y[3] * 0.0625f, y[7] * 0.0625f);
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

    float o[G][MT][NT][4];                         // O^T: rows = elements, columns = heads 2t, 2t + 1
    float mo[NT][G][2], m_run[NT][2], l_run[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
            m_run[nt][hh] = kLowest;
            l_run[nt][hh] = 0.0f;
#pragma unroll
            for (int gq = 0; gq < G; ++gq) {
                mo[nt][gq][hh] = 0.0f;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) o[gq][mt][nt][hh] = o[gq][mt][nt][2 + hh] = 0.0f;
            }
        }
    // power of two on V's scales: the largest one seen * vf is in [64, 128); before any, so high that one moves it
    float vf = 1.329227995784916e36f;              // 2^120
    float v_top = 0.0f;

    // lane parts of the shared-memory addresses
    constexpr int KB = 4 * KW;                     // K bytes per lane, row and group
    uint32_t k_off[G], v_off[G];
#pragma unroll
    for (int gq = 0; gq < G; ++gq) {
        const int kb = gq * (GE / 2) + t * KB;
        k_off[gq] = q4_tile_offset<RB>(g, kb / 16) + kb % 16;
        const int vb = VE == 4 ? gq * (GE / 2) + (g >> 1) * 4 : gq * (GE / 2) + g * (VE / 2);
        v_off[gq] = q4_tile_offset<RB>(2 * t, vb / 16) + vb % 16;
    }
    constexpr uint32_t NEXT_ROW = RB;              // row 2t + 1 sits in the same line: its unit differs in one bit
    constexpr uint32_t ROWS8 = 8 * RB;

    for (int j = 0; j < n_my; ++j) {
        cp_async_wait<STAGES - 1>();
        __syncwarp();
        const uint32_t stage = (j % STAGES) * L::STAGE_BYTES;
        const uint8_t* kt = smem_gen + (ring - smem_base) + stage;
        const uint8_t* vt = kt + L::K_BYTES;
        const uint8_t* pt = vt + L::K_BYTES;

        // Which of the tile's tokens count: those before the end, and not between the sinks and the window.
        const int r0 = range0(j);
        uint32_t valid = 0xffffffffu;
        {
            const int a = token_of(r0), c = token_of(r0 + GRAN);
            const bool hole = (a < tok_lo && a + GRAN > p.sinks) || (c < tok_lo && c + GRAN > p.sinks);
            if (r0 + TILE > tok_end || hole) {
                const int tk = token_of(r0 + (lane & ~15)) + (lane & 15);
                valid = __ballot_sync(0xffffffffu, r0 + lane < tok_end && !(tk >= p.sinks && tk < tok_lo));
            }
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
#pragma unroll
            for (int gq = 0; gq < G; ++gq) {
                float acc[NT][4];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) acc[nt][0] = acc[nt][1] = acc[nt][2] = acc[nt][3] = 0.0f;
                uint32_t w0[KW], w1[KW];
                load_words(w0, kt + sb * 16 * RB + k_off[gq]);
                load_words(w1, kt + sb * 16 * RB + ROWS8 + k_off[gq]);
#pragma unroll
                for (int w = 0; w < KW; ++w) {
                    const uint32_t x0 = w0[w], x1 = w1[w], y0 = x0 >> 8, y1 = x1 >> 8;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        mma_f16_16816(acc[nt], x0 & 0x000F000Fu, x1 & 0x000F000Fu, x0 & 0x00F000F0u, x1 & 0x00F000F0u,
                                      qb[nt][gq][w][0], qb[nt][gq][w][1]);
                        mma_f16_16816(acc[nt], y0 & 0x000F000Fu, y1 & 0x000F000Fu, y0 & 0x00F000F0u, y1 & 0x00F000F0u,
                                      qb[nt][gq][w][2], qb[nt][gq][w][3]);
                    }
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t u = pr[sb][e >> 1][gq];
                        sc[sb][nt][e] = fmaf(__uint_as_float(u & 0xFFFF0000u), qs[nt][gq][e & 1],
                                             fmaf(__uint_as_float(u << 16), acc[nt][e], sc[sb][nt][e]));
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
        float v_max = 0.0f;
#pragma unroll
        for (int sb = 0; sb < 2; ++sb)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int row = sb * 16 + r * 8 + g;
                const bool on = (valid >> row) & 1u;
#pragma unroll
                for (int gq = 0; gq < G; ++gq) {
                    if (!on) pr[sb][r][G + gq] = 0u;   // whatever the slot holds: 0 * NaN must not enter the sums
                    v_max = fmaxf(v_max, __uint_as_float(pr[sb][r][G + gq] << 16));
                }
            }
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
            for (int off = 4; off < 32; off <<= 1) {
                v_max = fmaxf(v_max, __shfl_xor_sync(0xffffffffu, v_max, off));
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
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int hh = 0; hh < 2; ++hh) {
                    const float m_new = fmaxf(m_run[nt][hh], top[nt][hh]);
                    const float alpha = ex2_approx(m_run[nt][hh] - m_new);
                    m_run[nt][hh] = m_new;
                    l_run[nt][hh] *= alpha;
                    const float both = alpha * vr;
#pragma unroll
                    for (int gq = 0; gq < G; ++gq) {
                        mo[nt][gq][hh] *= alpha;
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) {
                            o[gq][mt][nt][hh] *= both;
                            o[gq][mt][nt][2 + hh] *= both;
                        }
                    }
                }
        }

        // ---- weights and O^T += V^T P^T ----------------------------------------------------------------------------
#pragma unroll
        for (int sb = 0; sb < 2; ++sb) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    sc[sb][nt][e] = ex2_approx(fmaf(sc[sb][nt][e], cs[nt][e & 1], -m_run[nt][e & 1]));
                    l_run[nt][e & 1] += sc[sb][nt][e];
                }
#pragma unroll
            for (int gq = 0; gq < G; ++gq) {
                uint32_t pb[NT][2];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const float f = __uint_as_float(pr[sb][r][G + gq] << 16) * vf;
                        const float vm = __uint_as_float(pr[sb][r][G + gq] & 0xFFFF0000u);
                        pb[nt][r] = movmatrix_trans(pack_f16x2(sc[sb][nt][2 * r] * f, sc[sb][nt][2 * r + 1] * f));
                        mo[nt][gq][0] = fmaf(sc[sb][nt][2 * r], vm, mo[nt][gq][0]);
                        mo[nt][gq][1] = fmaf(sc[sb][nt][2 * r + 1], vm, mo[nt][gq][1]);
                    }
                const uint8_t* base = vt + sb * 16 * RB;
                const uint32_t first = v_off[gq], second = v_off[gq] ^ NEXT_ROW;
                constexpr int VW = VE >= 8 ? VE / 8 : 1;
                uint32_t ta[VW], tb[VW], tc[VW], td[VW];
                load_words(ta, base + first);
                load_words(tb, base + second);
                load_words(tc, base + ROWS8 + first);
                load_words(td, base + ROWS8 + second);
#pragma unroll
                for (int w = 0; w < VW; ++w) {
                    // pairs of tokens side by side: 16-bit halves (four codes) of tokens 2t, 2t + 1 and 2t + 8, 2t + 9
#pragma unroll
                    for (int half = 0; half < (VE >= 8 ? 2 : 1); ++half) {
                        const uint32_t sel = VE == 4 ? ((g & 1) ? 0x7632u : 0x5410u) : (half ? 0x7632u : 0x5410u);
                        const uint32_t x = __byte_perm(ta[w], tb[w], sel), y = __byte_perm(tc[w], td[w], sel);
                        const int mt = VE >= 8 ? w * 4 + half * 2 : 0;
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
                            mma_f16_16816(o[gq][mt][nt], x & 0x000F000Fu, x & 0x00F000F0u, y & 0x000F000Fu,
                                          y & 0x00F000F0u, pb[nt][0], pb[nt][1]);
                        const uint32_t x8 = x >> 8, y8 = y >> 8;
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
                            mma_f16_16816(o[gq][mt + 1][nt], x8 & 0x000F000Fu, x8 & 0x00F000F0u, y8 & 0x000F000Fu,
                                          y8 & 0x00F000F0u, pb[nt][0], pb[nt][1]);
                    }
                }
            }
        }

        // ---- refill this stage ------------------------------------------------------------------------------------
        __syncwarp();
        if (j + STAGES < n_my) {
            issue(j + STAGES, next0, next1);
            next0 = load_page(j + STAGES + 1, 0);
            next1 = load_page(j + STAGES + 1, 1);
        }
        cp_async_commit();
    }
    cp_async_wait<0>();
    __syncwarp();

    // ---- combine the warps' results through shared memory (each warp reuses its own ring) --------------------------
    constexpr int WROWS = 8 * NT;
    constexpr int WSTRIDE = D + 8;
    static_assert((WROWS * WSTRIDE + 2 * WROWS) * 4 <= L::RING_BYTES, "merge scratch must fit in a ring");
    float* wo = reinterpret_cast<float*>(smem_gen + warp * L::RING_BYTES);
    float* wm = wo + WROWS * WSTRIDE;
    float* wl = wm + WROWS;
    const float back = 16777216.0f, unscale = 1.0f / vf;       // two factors: their product may leave fp32's range
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
            float l = l_run[nt][hh];
#pragma unroll
            for (int off = 4; off < 32; off <<= 1) l += __shfl_xor_sync(0xffffffffu, l, off);
            const int row = 8 * nt + 2 * t + hh;
            if (g == 0) {
                wm[row] = m_run[nt][hh];
                wl[row] = l;
            }
#pragma unroll
            for (int gq = 0; gq < G; ++gq) {
                float m = mo[nt][gq][hh];
#pragma unroll
                for (int off = 4; off < 32; off <<= 1) m += __shfl_xor_sync(0xffffffffu, m, off);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    const float even = o[gq][mt][nt][hh] * back * unscale + m;
                    const float odd = o[gq][mt][nt][2 + hh] * (back * 0.0625f) * unscale + m;
                    *reinterpret_cast<float2*>(wo + row * WSTRIDE + gq * GE + g * VE + 2 * mt) = make_float2(even, odd);
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
            mw[w] = reinterpret_cast<const float*>(smem_gen + w * L::RING_BYTES)[WROWS * WSTRIDE + row];
            M = fmaxf(M, mw[w]);
        }
        float4 num = make_float4(0.f, 0.f, 0.f, 0.f);
        float den = 0.0f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            const float* base = reinterpret_cast<const float*>(smem_gen + w * L::RING_BYTES);
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
    const int items = HG * C4;                     // at most 16 * 32 of them
    if (items <= THREADS) merge_splits_from_workspace<D, THREADS, 1, 16>(p, hq0, items, S, n_active);
    else if (items <= 2 * THREADS) merge_splits_from_workspace<D, THREADS, 2, 8>(p, hq0, items, S, n_active);
    else merge_splits_from_workspace<D, THREADS, 3, 5>(p, hq0, items, S, n_active);
}

// Shapes of the CTA: warps, ring stages and CTAs per SM by group and head_dim.
template <int D, int G, int NT>
struct Q4Shape {
    static constexpr int NW = NT == 2 || G == 4 ? 6 : 8;
    static constexpr int STAGES = D == 64 ? 4 : 3;
    static constexpr int CTAS = 2;
    using Smem = Q4Smem<D, G, NW, STAGES>;
    static_assert(16 * (D / 4) <= 3 * NW * 32, "the merge's items per thread");
};

template <int D, int G, int NT>
cudaError_t launch_q4(const Q4AttnParams& p, int B, cudaStream_t stream) {
    using Shape = Q4Shape<D, G, NT>;
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
    return cudaLaunchKernelEx(&cfg, paged_decode_attn_q4_kernel<D, G, NT, Shape::NW, Shape::STAGES, Shape::CTAS>, p);
}

template <int D, int G, int NT>
cudaError_t set_q4(int smem_optin) {
    using Shape = Q4Shape<D, G, NT>;
    if (Shape::Smem::TOTAL > smem_optin) return cudaErrorInvalidConfiguration;
    return cudaFuncSetAttribute(paged_decode_attn_q4_kernel<D, G, NT, Shape::NW, Shape::STAGES, Shape::CTAS>,
                                cudaFuncAttributeMaxDynamicSharedMemorySize, Shape::Smem::TOTAL);
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
    const int groups = d / cache.group;
    const bool wide = Hq / Hkv > 8;
    if (d == 128) {
        if (groups == 1) return wide ? launch_q4<128, 1, 2>(p, B, stream) : launch_q4<128, 1, 1>(p, B, stream);
        if (groups == 2) return wide ? launch_q4<128, 2, 2>(p, B, stream) : launch_q4<128, 2, 1>(p, B, stream);
        return wide ? launch_q4<128, 4, 2>(p, B, stream) : launch_q4<128, 4, 1>(p, B, stream);
    }
    if (groups == 1) return wide ? launch_q4<64, 1, 2>(p, B, stream) : launch_q4<64, 1, 1>(p, B, stream);
    return wide ? launch_q4<64, 2, 2>(p, B, stream) : launch_q4<64, 2, 1>(p, B, stream);
}

}  // namespace ac
