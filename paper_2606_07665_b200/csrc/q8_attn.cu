// Single-token decode attention over the 8-bit paged cache, one CTA per (request, KV head, split).
//
// Mathematics.  K and V enter as their codes c, the scale of a block of tokens apart:
//     score_t = sK(t) * (q . cK_t) * scale,      out = sum_t (p_t sV(t)) cV_t / sum_t p_t.
// A granule of 16 tokens lies in one block, so a scale is one fp32 factor per granule, which joins the softmax scale on one
// side and the weights on the other.  Codes are exact as fp16: both products run on the tensor pipe, with q brought into
// fp16's range by a power of two per head (its bf16 digits fit) and fp32 sums.
//
// Tiles.  As in the 4-bit kernel the tokens are the rows of mma.m16n8k16 and the query heads its 8 columns (two column
// blocks for groups of 9-16 heads), S^T = K Q^T and O^T = V^T P^T, with the accumulator of the first turned into the operand
// of the second by an 8x8 transpose between lanes.  ldmatrix brings K's bytes in place four dims of one token to a lane, the k
// dimension of the product in that order; transposed, a 16-bit half of V is two dims of one token, and one permutation of the bytes
// pairs up the tokens.
//
// Weights in fp16: p is relative to a reference that may lag the running maximum by up to 8 (powers of two), so that
// most tiles need no reduction across the warp; p sV is kept below 2^15 by a power of two that follows the largest V scale seen.
// The sums of a tile start at zero and join the running ones in fp32 proper, because the pipe truncates its accumulator
// at every step: a bias where the addends have one sign.
//
// Data movement.  Every warp streams tiles of 32 tokens through its own ring, one box of a tensor map for K and one for V (two
// where pages are no multiple of 32 tokens), no CTA-wide synchronisation in the main loop.
//
// Bound: HBM up to eight heads per KV head: 4 rows of 131072 tokens, 64:8 heads of 128 (1.08 GB): 160 us = 6720 GB/s, 1.04 of the measured
// copy rate; 64 rows of 128 to 8192, 32:8 heads (506 MB): 81 us = 6260 GB/s, int8 84.  Elsewhere the latency of a tile's chain (wait,
// ldmatrix, conversion, dependent products, maximum, exponentials, transpose, products), of which a warp has one open: no unit is near
// its limit.  More heads: 128 rows under a window of 4096, 32:2 heads, int8 (260 MB): 52 us = 5000 GB/s (issue slots 40-47 %, ALU 35,
// tensor pipe 31, 3 warps a scheduler).  Heads of 64: 64 rows of 128 to 8192, 16:4 (127 MB): 27 us = 4640 GB/s (issue slots 32 %, ALU 30,
// tensor pipe 10, 2 warps a scheduler).  Short: 512 tokens of 2 heads 3.9 us, a merge of splits 2 more.
#include <limits.h>
#include <math.h>

#include "ac_internal.h"
#include "q8_format.cuh"
#include "split_merge.cuh"

namespace ac {
namespace {

using namespace acdev;

constexpr int TILE = 32;                      // tokens per stage
constexpr int GRAN = 16;                      // tokens that are sure to share a page and a block
constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;
constexpr float kLag = 8.0f;                  // how far (in powers of two) the softmax reference may lag
constexpr float kLowest = -3.0e38f;           // reference of a warp that has seen no token

template <int D, int NT, int NW, int STAGES>
struct Q8Smem {
    static constexpr int K_BYTES = TILE * D;
    static constexpr int STAGE_BYTES = 2 * K_BYTES;           // K codes, V codes
    static constexpr int RING_BYTES = STAGES * STAGE_BYTES;
    static constexpr int Q_OFFSET = NW * RING_BYTES;          // query fragments, where they do not stay in registers
    static constexpr int Q_BYTES = NT == 2 ? D / 16 * 32 * 16 : 0;
    static constexpr int BAR_OFFSET = Q_OFFSET + Q_BYTES;
    static constexpr int TOTAL = BAR_OFFSET + NW * STAGES * 8 + 1024;      // the swizzle wants rings aligned to 1024
};

struct Q8AttnParams {
    const uint16_t* q;
    const float* scales;
    const int32_t* block_table;
    const int32_t* context_lens;
    const int32_t* row_order;
    float* partial_o;
    float* partial_lse;
    uint16_t* out;
    uint16_t* out_mirror;                     // always nullptr here (the shared merge knows the field)
    int32_t* arrivals;
    int32_t* status_flag;
    int64_t stride_scales;
    float scale_log2;
    uint32_t gpp;                             // granules per page
    uint32_t gpp_magic;                       // ceil(2^32 / gpp); unused when gpp == 1
    int gpb;                                  // granules per block
    int box;                                  // tokens of a tensor-map box: 32 where they are sure to share a page, else 16
    int max_pages_per_seq, new_tokens, num_splits, split_tokens, Hq, Hkv, page_size, num_pages, window, sinks, block;
};

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2,
                                            int c3, uint64_t policy) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        ".L2::cache_hint [%0], [%1, {%3, %4, %5, %6}], [%2], %7;"
        ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "l"(policy)
        : "memory");
}

// Byte offset of 16-byte chunk `chunk` of row `row` in a tile of rows of D bytes, as the tensor map's swizzle places it.
// Rows 8 further are 8 * D bytes further, and chunk ^ 2 of the same row is the offset ^ 32.
template <int D>
__device__ __forceinline__ uint32_t q8_tile_offset(int row, int chunk) {
    return D == 128 ? row * 128 + ((chunk ^ (row & 7)) << 4) : row * 64 + ((chunk ^ ((row >> 1) & 3)) << 4);
}

// 2^-e of 2^e, |e| <= 126.  (A division takes its slow way beside such numbers.)
__device__ __forceinline__ float power_of_two_inverse(float x) { return __uint_as_float((254u << 23) - __float_as_uint(x)); }

template <int D, int FMT, int NT, int NW, int STAGES, int CTAS>
__global__ void __launch_bounds__(NW * 32, CTAS) paged_decode_attn_q8_kernel(
    const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, const Q8AttnParams p) {
    using L = Q8Smem<D, NT, NW, STAGES>;
    constexpr int WARPS = NW, THREADS = NW * 32;
    constexpr int NC = D / 16;                     // 16-byte chunks (16 elements) per row

    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (smem_addr(smem_raw) + 1023u) & ~1023u;
    uint8_t* const smem = smem_raw + (smem_base - smem_addr(smem_raw));

    const int h = blockIdx.x, split = blockIdx.z;
    const int b = p.row_order != nullptr ? p.row_order[blockIdx.y] : static_cast<int>(blockIdx.y);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int g = lane >> 2, t = lane & 3;
    const int HG = p.Hq / p.Hkv;
    const int S = p.num_splits;

    // ---- the row's range: attended tokens laid end to end, in boxes (see the bf16 kernel) ---------------------
    // Without a window the pages of the first tiles do not depend on the row's length: they are asked for beside it.
    const int32_t* bt_row = p.block_table + static_cast<size_t>(b) * p.max_pages_per_seq;
    int page_early = -1;
    if (p.window == 0) {
        const uint32_t gr = (static_cast<uint32_t>(split) * p.split_tokens + (warp + (lane >> 1) * WARPS) * TILE) / GRAN + (lane & 1);
        const uint32_t idx = p.gpp == 1 ? gr : __umulhi(gr, p.gpp_magic);
        if (idx < static_cast<uint32_t>(p.max_pages_per_seq)) page_early = bt_row[idx];
    }
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
            sink_span = (p.sinks + p.box - 1) / p.box * p.box;
            window_base = max(0, tok_lo / p.box * p.box - sink_span);
        }
    }
    const int range_tokens = n_tokens - window_base;
    const int tok_begin = static_cast<int>(min(static_cast<long long>(split) * p.split_tokens, static_cast<long long>(range_tokens)));
    // The last split goes on to the row's end: a row that has outgrown the plan is slower, not cut off.
    const int tok_end = split == S - 1 || range_tokens - tok_begin < p.split_tokens ? range_tokens : tok_begin + p.split_tokens;

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

    const uint32_t ring = smem_base + warp * L::RING_BYTES;
    const uint32_t bars = smem_base + L::BAR_OFFSET + warp * STAGES * 8;
    if (lane == 0) {
        tma_prefetch_descriptor(&k_map);
        tma_prefetch_descriptor(&v_map);
#pragma unroll
        for (int s = 0; s < STAGES; ++s) mbar_init(bars + s * 8, 1);
        mbar_init_fence();
    }
    __syncwarp();

    const int n_tiles = (tok_end - tok_begin + TILE - 1) / TILE;
    const int n_my = n_tiles > warp ? (n_tiles - warp + WARPS - 1) / WARPS : 0;
    const uint64_t policy = l2_policy_evict_first();
    auto range0 = [&](int j) { return tok_begin + (warp + j * WARPS) * TILE; };
    // Range positions that are not attended: between the sinks and the window's first token.
    const int hole_lo = tok_lo > 0 ? p.sinks : 0, hole_hi = tok_lo > 0 ? tok_lo - window_base : 0;

    // Where the tiles lie.  The warp looks up the pages of 16 tiles at a time, one granule per lane (lane = tile * 2 + half);
    // a tile takes its own by shuffle.  The page ids of the next 16 tiles are loaded ahead; the scales, which are needed when a
    // tile has arrived, once the pages are known.
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
    int gr_page = -1, gr_sub = 0;                  // this lane's granule: page (-1: none, it reads as zeros) and place in it
    float gr_k = 0.0f, gr_v = 0.0f;                // its scales; they become the consumed tiles' own when those begin
    auto settle_pages = [&](int j0, int page) {
        locate(j0, gr_sub);
        gr_page = page >= 0 && page < p.num_pages ? page : -1;
    };
    auto load_scales = [&]() {
        gr_k = gr_v = 0.0f;
        if (gr_page >= 0) {
            const float2 s = *reinterpret_cast<const float2*>(p.scales + gr_page * p.stride_scales +
                                                              (h * (p.page_size / p.block) + gr_sub / p.gpb) * 2);
            gr_k = s.x;
            gr_v = s.y;
        }
    };
    // Fetches tile j into its stage.  Page -1 is outside the map: zeros arrive.  With boxes of 16 the tile's second half may
    // lie past the end and stays what it was.
    auto issue = [&](int j, uint32_t stage, uint32_t bar) {
        const int src = 2 * (j & 15);
        const int page0 = __shfl_sync(0xffffffffu, gr_page, src), sub0 = __shfl_sync(0xffffffffu, gr_sub, src);
        const int page1 = __shfl_sync(0xffffffffu, gr_page, src + 1), sub1 = __shfl_sync(0xffffffffu, gr_sub, src + 1);
        if (lane == 0) {
            const uint32_t dst = ring + stage;
            if (p.box == TILE) {
                mbar_arrive_expect_tx(bar, L::STAGE_BYTES);
                tma_load_4d(dst, &k_map, bar, 0, sub0 * GRAN, h, page0, policy);
                tma_load_4d(dst + L::K_BYTES, &v_map, bar, 0, sub0 * GRAN, h, page0, policy);
            } else {
                const bool two = range0(j) + GRAN < tok_end;
                mbar_arrive_expect_tx(bar, two ? L::STAGE_BYTES : L::STAGE_BYTES / 2);
                tma_load_4d(dst, &k_map, bar, 0, sub0 * GRAN, h, page0, policy);
                tma_load_4d(dst + L::K_BYTES, &v_map, bar, 0, sub0 * GRAN, h, page0, policy);
                if (two) {
                    tma_load_4d(dst + GRAN * D, &k_map, bar, 0, sub1 * GRAN, h, page1, policy);
                    tma_load_4d(dst + L::K_BYTES + GRAN * D, &v_map, bar, 0, sub1 * GRAN, h, page1, policy);
                }
            }
        }
    };

    // ---- prologue: fill the ring; tiles that hold the block of slot ctx - 1 or a later one wait for the preceding kernel,
    // which may have rounded that block's codes again; no scale is read before ------------------------------------------
    const int dependent_from = (ctx > 0 ? (ctx - 1) / p.block * p.block : 0) - window_base;     // range position, maybe negative
    bool dependency_met = false;
    int sub_first;
    settle_pages(0, p.window != 0 ? load_pages(0) : locate(0, sub_first) >= 0 ? page_early : -1);
    int pages_ahead = load_pages(16);
#pragma unroll
    for (int s = 0; s < STAGES; ++s) {
        if (s < n_my) {
            if (!dependency_met && range0(s) + TILE > dependent_from) {
                dependency_sync();
                dependency_met = true;
            }
            issue(s, s * L::STAGE_BYTES, bars + s * 8);
        }
    }
    if (!dependency_met) dependency_sync();                                // q was written by the preceding kernel
    load_scales();

    // ---- query fragments (B operand): lane (g, t) holds head g (+ 8), elements in the order of K's bytes ----------
    uint32_t qb[NT][NC][2];
    float cs[NT][2];                               // score factor, heads 2t and 2t + 1
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int head = g + 8 * nt;
        const bool live = head < HG;
        const uint16_t* src = p.q + (static_cast<size_t>(b) * p.Hq + h * HG + (live ? head : 0)) * D;
        float x[NC][4];
        float mx = 0.0f;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const uint2 raw = *reinterpret_cast<const uint2*>(src + c * 16 + t * 4);
            const uint32_t u[2] = {raw.x, raw.y};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
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
        const float factor = p.scale_log2 * __uint_as_float(static_cast<uint32_t>(127 - k) << 23);
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            qb[nt][c][0] = pack_f16x2(x[c][0] * up, x[c][1] * up);
            qb[nt][c][1] = pack_f16x2(x[c][2] * up, x[c][3] * up);
        }
        cs[nt][0] = __shfl_sync(0xffffffffu, factor, 8 * t);
        cs[nt][1] = __shfl_sync(0xffffffffu, factor, 8 * t + 4);
    }

    // With two column blocks the fragments would crowd out the accumulators: they go to shared memory, 16 bytes per chunk and lane
    // (the same for every warp).
    uint8_t* const q_frag = smem + L::Q_OFFSET + lane * 16;
    if constexpr (NT == 2) {
        if (warp == 0) {
#pragma unroll
            for (int c = 0; c < NC; ++c)
                *reinterpret_cast<uint4*>(q_frag + c * 512) = make_uint4(qb[0][c][0], qb[0][c][1], qb[1][c][0], qb[1][c][1]);
        }
        __syncthreads();
    }

    // O^T, heads 2t and 2t + 1 as pairs: [chunk][element 2g + i of it]
    uint64_t o[NC][2][NT];
    float m_run[NT][2];
    uint64_t l_run[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        l_run[nt] = 0ull;
        m_run[nt][0] = m_run[nt][1] = kLowest;
#pragma unroll
        for (int c = 0; c < NC; ++c) o[c][0][nt] = o[c][1][nt] = 0ull;
    }
    // power of two on V's scales: the largest one seen * vf is in [64, 128); before any, so high that one of 2^-119 moves it
    float vf = 8.507059173023462e37f;              // 2^126, whose inverse is a normal number
    float v_top = 0.0f;

    // ldmatrix addresses, the same for K (bytes 4t .. 4t + 3 of a row's chunk land in lane (row, t)) and, transposed, for V:
    // matrices 0 and 1 are rows 0-7 and 8-15 of one chunk, 2 and 3 of the next.
    const uint32_t mat_off = q8_tile_offset<D>(((lane >> 3) & 1) * 8 + (lane & 7), lane >> 4);

    // tiles before j_hole may hold masked tokens of the hole, those from j_tail on may lie past the end
    const int j_hole = hole_hi > tok_begin ? ((hole_hi - tok_begin + TILE - 1) / TILE - warp + WARPS - 1) / WARPS : 0;
    const int j_tail = (tok_end - tok_begin) % TILE != 0 ? n_my - 1 : n_my;
    float k_scale = 0.0f, v_scale = 0.0f;          // scales of this lane's granule among the 16 tiles being consumed
    uint32_t stage = 0, bar = bars, parity = 0;
    bool timed_out = false;
    int j = 0;
    for (; j < n_my; ++j) {
        if ((j & 15) == 0) {
            k_scale = gr_k;
            v_scale = gr_v;
        }
        const int src = 2 * (j & 15);
        float sk[2], sv[2];
#pragma unroll
        for (int sb = 0; sb < 2; ++sb) {
            sk[sb] = __shfl_sync(0xffffffffu, k_scale, src + sb);
            sv[sb] = __shfl_sync(0xffffffffu, v_scale, src + sb);
        }
        if (!__all_sync(0xffffffffu, mbar_wait_bounded(bar, parity))) {
            timed_out = true;
            break;
        }
        const uint32_t kt = ring + stage, vt = kt + L::K_BYTES;

        // Which of the tile's tokens count: those before the end, and not between the sinks and the window.  What the
        // others' slots and scales hold must not enter the sums, not even times zero.
        uint32_t valid = 0xffffffffu;
        if (j >= j_tail || j < j_hole) {
            const int r = range0(j) + lane;
            valid = __ballot_sync(0xffffffffu, r < tok_end && !(r >= hole_lo && r < hole_hi));
            if (!((valid >> lane) & 1u)) {
                uint4* row = reinterpret_cast<uint4*>(smem + (vt - smem_base) + lane * D);
#pragma unroll
                for (int c = 0; c < NC; ++c) row[c] = make_uint4(0u, 0u, 0u, 0u);
            }
            fence_proxy_async_shared();            // before a later copy into these bytes
            __syncwarp();
#pragma unroll
            for (int sb = 0; sb < 2; ++sb)
                if (((valid >> (16 * sb)) & 0xffffu) == 0u) sk[sb] = sv[sb] = 0.0f;
        }

        // ---- scores ------------------------------------------------------------------------------------------
        float sc[2][NT][4];
        float top[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) top[nt][0] = top[nt][1] = -INFINITY;
#pragma unroll
        for (int sb = 0; sb < 2; ++sb) {
            float acc[NT][4];
#pragma unroll
            for (int c = 0; c < NC; c += 2) {
                uint32_t w[4];
                ldmatrix_x4(w[0], w[1], w[2], w[3], kt + sb * GRAN * D + (mat_off ^ (c * 16)));
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    uint32_t a0, a1, a2, a3;
                    q8_pairs<FMT>(w[2 * i], a0, a2);
                    q8_pairs<FMT>(w[2 * i + 1], a1, a3);
                    uint32_t b[NT][2];
                    if constexpr (NT == 2) {
                        const uint4 f = *reinterpret_cast<const uint4*>(q_frag + (c + i) * 512);
                        b[0][0] = f.x, b[0][1] = f.y, b[NT - 1][0] = f.z, b[NT - 1][1] = f.w;
                    } else {
                        b[0][0] = qb[0][c + i][0], b[0][1] = qb[0][c + i][1];
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        if (c + i == 0) mma_f16_16816_zero(acc[nt], a0, a1, a2, a3, b[nt][0], b[nt][1]);
                        else mma_f16_16816(acc[nt], a0, a1, a2, a3, b[nt][0], b[nt][1]);
                    }
                }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const uint64_t factor = f32x2(cs[nt][0] * sk[sb], cs[nt][1] * sk[sb]);
#pragma unroll
                for (int r = 0; r < 2; ++r)
                    f32x2_split(f32x2_mul(f32x2(acc[nt][2 * r], acc[nt][2 * r + 1]), factor), sc[sb][nt][2 * r], sc[sb][nt][2 * r + 1]);
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

        // ---- whether the references still serve ----------------------------------------------------------------
        const float v_max = fmaxf(sv[0], sv[1]);   // the same in every lane
        bool move = v_max * vf >= 128.0f;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int hh = 0; hh < 2; ++hh) move = move || top[nt][hh] > m_run[nt][hh] + kLag;
        if (__any_sync(0xffffffffu, move)) {
#pragma unroll
            for (int off = 4; off < 32; off <<= 1)         // lanes (g, t) of one t hold the same heads
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int hh = 0; hh < 2; ++hh)
                        top[nt][hh] = fmaxf(top[nt][hh], __shfl_xor_sync(0xffffffffu, top[nt][hh], off));
            float vr = 1.0f;
            if (v_max > v_top) {
                v_top = v_max;
                int k = 6 - (static_cast<int>(__float_as_uint(v_top) >> 23) - 127);
                k = max(-126, min(k, 126));
                const float next = __uint_as_float(static_cast<uint32_t>(k + 127) << 23);
                vr = next * power_of_two_inverse(vf);
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
                l_run[nt] = f32x2_mul(l_run[nt], f32x2(alpha[0], alpha[1]));
                const uint64_t both = f32x2(alpha[0] * vr, alpha[1] * vr);
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    o[c][0][nt] = f32x2_mul(o[c][0][nt], both);
                    o[c][1][nt] = f32x2_mul(o[c][1][nt], both);
                }
            }
        }

        // ---- weights -------------------------------------------------------------------------------------------
        uint32_t pb[2][NT][2];                     // B operands: weights times V's scale, tokens 2t, 2t + 1 (+ 8) of head g
#pragma unroll
        for (int sb = 0; sb < 2; ++sb) {
            const float f = sv[sb] * vf;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const uint64_t less = f32x2(-m_run[nt][0], -m_run[nt][1]);
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    float a, b2;
                    f32x2_split(f32x2_add(f32x2(sc[sb][nt][2 * r], sc[sb][nt][2 * r + 1]), less), a, b2);
                    const uint64_t pair = f32x2(ex2_approx(a), ex2_approx(b2));
                    l_run[nt] = f32x2_add(l_run[nt], pair);
                    f32x2_split(f32x2_mul(pair, f32x2(f, f)), a, b2);
                    pb[sb][nt][r] = movmatrix_trans(pack_f16x2(a, b2));
                }
            }
        }

        // ---- O^T += V^T P^T ------------------------------------------------------------------------------------
#pragma unroll
        for (int c2 = 0; c2 < NC; c2 += 2) {
            uint32_t vw[2][2][2];                  // [granule][chunk c2, c2 + 1][tokens 0-7, 8-15]
#pragma unroll
            for (int sb = 0; sb < 2; ++sb)
                ldmatrix_x4_trans(vw[sb][0][0], vw[sb][0][1], vw[sb][1][0], vw[sb][1][1], vt + sb * GRAN * D + (mat_off ^ (c2 * 16)));
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                float sum[NT][4];
#pragma unroll
                for (int sb = 0; sb < 2; ++sb) {
                    uint32_t a0, a1, a2, a3;       // elements 2g and 2g + 1 of tokens 2t, 2t + 1, then of 2t + 8, 2t + 9
                    q8_pairs_across<FMT>(vw[sb][w][0], a0, a1);
                    q8_pairs_across<FMT>(vw[sb][w][1], a2, a3);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        if (sb == 0) mma_f16_16816_zero(sum[nt], a0, a1, a2, a3, pb[sb][nt][0], pb[sb][nt][1]);
                        else mma_f16_16816(sum[nt], a0, a1, a2, a3, pb[sb][nt][0], pb[sb][nt][1]);
                    }
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    o[c2 + w][0][nt] = f32x2_add(o[c2 + w][0][nt], f32x2(sum[nt][0], sum[nt][1]));
                    o[c2 + w][1][nt] = f32x2_add(o[c2 + w][1][nt], f32x2(sum[nt][2], sum[nt][3]));
                }
            }
        }

        // ---- refill this stage ------------------------------------------------------------------------------------
        __syncwarp();
        if (j + STAGES < n_my) {
            const int next = j + STAGES;
            if ((next & 15) == 0) {
                settle_pages(next, pages_ahead);
                load_scales();
                pages_ahead = load_pages(next + 16);
            }
            issue(next, stage, bar);
        }
        stage += L::STAGE_BYTES;
        bar += 8;
        if (stage == L::RING_BYTES) {
            stage = 0;
            bar = bars;
            parity ^= 1u;
        }
    }
    if (timed_out) {
        // Record the failure, then give the copies still in flight a bounded chance to land before this CTA's shared memory is
        // released.
        if (lane == 0 && p.status_flag != nullptr) atomicOr(p.status_flag, AC_FLAG_WAIT_TIMEOUT);
        for (int jj = j; jj < min(n_my, j + STAGES); ++jj) mbar_wait_bounded(bars + (jj % STAGES) * 8, (jj / STAGES) & 1);
    }
    __syncwarp();

    // ---- combine the warps' results through shared memory (each warp reuses its own ring) --------------------------
    constexpr int WROWS = 8 * NT;
    constexpr int WSTRIDE = D + 8;
    static_assert((WROWS * WSTRIDE + 2 * WROWS) * 4 <= L::RING_BYTES, "merge scratch must fit in a ring");
    float* wo = reinterpret_cast<float*>(smem + warp * L::RING_BYTES);
    float* wm = wo + WROWS * WSTRIDE;
    float* wl = wm + WROWS;
    const float unscale = power_of_two_inverse(vf);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        float l[2];
        f32x2_split(l_run[nt], l[0], l[1]);
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
#pragma unroll
            for (int off = 4; off < 32; off <<= 1) l[hh] += __shfl_xor_sync(0xffffffffu, l[hh], off);
            if (g == 0) {
                wm[8 * nt + 2 * t + hh] = m_run[nt][hh];
                wl[8 * nt + 2 * t + hh] = l[hh];
            }
        }
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            float even[2], odd[2];
            f32x2_split(o[c][0][nt], even[0], even[1]);
            f32x2_split(o[c][1][nt], odd[0], odd[1]);
#pragma unroll
            for (int hh = 0; hh < 2; ++hh)
                *reinterpret_cast<float2*>(wo + (8 * nt + 2 * t + hh) * WSTRIDE + c * 16 + 2 * g) = make_float2(even[hh] * unscale, odd[hh] * unscale);
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

// Shapes of the CTA, by the CTAs of the grid, with about 128 KB of loads in flight on an SM, where HBM delivers most (4 rows of
// 131072 tokens, 64:8 heads of 128: 161 us with 8 warps of 2 stages against 173 with 12):
//   FAT    eight warps, one CTA per SM, for grids of at most that many;
//   BASE   four warps, two CTAs per SM: the second one's stream covers the first one's start and end;
//   THREE  three CTAs per SM and
//   SHORT  three warps, four CTAs per SM, for grids of more than two, and more than four, CTAs per SM of short splits, where
//          starts and ends are much of a CTA's life (256 rows of 512 to 2048 tokens, 32:8 heads: BASE 118 us, THREE 111, SHORT
//          109; 128 such rows of 28:4: 30.1, 28.3, 33.8; 64 rows of up to 8192, which are not short: 81, 97 in THREE).
// Groups of 9-16 heads need the arithmetic of more warps: six in BASE (128 rows under a window of 4096, 32:2 heads: 53.6 -> 51.9
// us; heads of 64: 31 -> 23.5), and at most THREE (256 rows, 36:4 heads: 71 -> 68).
enum class Fit { FAT, BASE, THREE, SHORT };
constexpr int kShortSplitTokens = 2560;

constexpr int shape_warps(Fit f, bool wide) { return f == Fit::FAT ? 8 : f == Fit::SHORT ? 3 : f == Fit::BASE && wide ? 6 : 4; }
constexpr int shape_ctas(Fit f) { return f == Fit::FAT ? 1 : f == Fit::BASE ? 2 : f == Fit::THREE ? 3 : 4; }
Fit fit_for(long long ctas, int split_tokens, bool wide, int sms) {
    if (ctas <= sms) return Fit::FAT;
    if (ctas <= 2ll * sms || split_tokens > kShortSplitTokens) return Fit::BASE;
    return ctas > 4ll * sms && !wide ? Fit::SHORT : Fit::THREE;
}

template <int D, int NT, Fit F>
struct Q8Shape {
    static constexpr int NW = shape_warps(F, NT == 2);
    static constexpr int STAGES = D == 64 ? 4 : 2;
    static constexpr int CTAS = shape_ctas(F);
    using Smem = Q8Smem<D, NT, NW, STAGES>;
};
#define AC_Q8_KERNEL(D_, FMT_, NT_, F_)                                                                              \
    paged_decode_attn_q8_kernel<D_, FMT_, NT_, Q8Shape<D_, NT_, F_>::NW, Q8Shape<D_, NT_, F_>::STAGES,                \
                                Q8Shape<D_, NT_, F_>::CTAS>

template <int D, int FMT, int NT, Fit F>
cudaError_t launch_q8_shape(const CUtensorMap& k_map, const CUtensorMap& v_map, const Q8AttnParams& p, int B, cudaStream_t stream) {
    using Shape = Q8Shape<D, NT, F>;
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
    return cudaLaunchKernelEx(&cfg, AC_Q8_KERNEL(D, FMT, NT, F), k_map, v_map, p);
}

template <int D, int FMT, int NT>
cudaError_t launch_q8(const CUtensorMap& k_map, const CUtensorMap& v_map, const Q8AttnParams& p, int B, int sms, cudaStream_t stream) {
    switch (fit_for(static_cast<long long>(B) * p.Hkv * p.num_splits, p.split_tokens, NT == 2, sms)) {
        case Fit::FAT: return launch_q8_shape<D, FMT, NT, Fit::FAT>(k_map, v_map, p, B, stream);
        case Fit::BASE: return launch_q8_shape<D, FMT, NT, Fit::BASE>(k_map, v_map, p, B, stream);
        case Fit::SHORT:
            if constexpr (NT == 1) return launch_q8_shape<D, FMT, NT, Fit::SHORT>(k_map, v_map, p, B, stream);
        default: return launch_q8_shape<D, FMT, NT, Fit::THREE>(k_map, v_map, p, B, stream);
    }
}

template <int D, int FMT, int NT, Fit F>
cudaError_t set_q8_shape(int smem_optin) {
    constexpr int bytes = Q8Shape<D, NT, F>::Smem::TOTAL;
    if (bytes > smem_optin) return cudaErrorInvalidConfiguration;
    return cudaFuncSetAttribute(AC_Q8_KERNEL(D, FMT, NT, F), cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
}

template <int D, int FMT, int NT>
cudaError_t set_q8(int smem_optin) {
    cudaError_t e = set_q8_shape<D, FMT, NT, Fit::FAT>(smem_optin);
    if (e == cudaSuccess) e = set_q8_shape<D, FMT, NT, Fit::BASE>(smem_optin);
    if (e == cudaSuccess) e = set_q8_shape<D, FMT, NT, Fit::THREE>(smem_optin);
    if constexpr (NT == 1) {
        if (e == cudaSuccess) e = set_q8_shape<D, FMT, NT, Fit::SHORT>(smem_optin);
    }
    return e;
}

}  // namespace

cudaError_t q8_attn_set_attributes(int smem_optin) {
    cudaError_t e = set_q8<128, Q8_INT8, 1>(smem_optin);
    if (e == cudaSuccess) e = set_q8<128, Q8_INT8, 2>(smem_optin);
    if (e == cudaSuccess) e = set_q8<128, Q8_E4M3, 1>(smem_optin);
    if (e == cudaSuccess) e = set_q8<128, Q8_E4M3, 2>(smem_optin);
    if (e == cudaSuccess) e = set_q8<64, Q8_INT8, 1>(smem_optin);
    if (e == cudaSuccess) e = set_q8<64, Q8_INT8, 2>(smem_optin);
    if (e == cudaSuccess) e = set_q8<64, Q8_E4M3, 1>(smem_optin);
    if (e == cudaSuccess) e = set_q8<64, Q8_E4M3, 2>(smem_optin);
    return e;
}

void q8_attn_shape(long long ctas, int split_tokens, bool wide, int sms, int* warps, int* per_sm) {
    const Fit f = fit_for(ctas, split_tokens, wide, sms);
    *warps = shape_warps(f, wide);
    *per_sm = shape_ctas(f);
}

int q8_attn_box(int page_size) { return page_size % TILE == 0 ? TILE : GRAN; }

cudaError_t launch_paged_decode_attn_q8(const CUtensorMap& k_map, const CUtensorMap& v_map, const void* q_rot,
                                        const Q8View& cache, const int32_t* block_table, int max_pages_per_seq,
                                        const int32_t* context_lens, int new_tokens, float scale, int num_splits,
                                        int split_tokens, float* partial_o, float* partial_lse, int32_t* arrivals,
                                        void* out, int B, int Hq, int Hkv, int d, int page_size, int num_pages,
                                        int window, int sinks, const int32_t* row_order, int32_t* status_flag,
                                        cudaStream_t stream) {
    Q8AttnParams p;
    p.q = static_cast<const uint16_t*>(q_rot);
    p.scales = cache.scales;
    p.block_table = block_table;
    p.context_lens = context_lens;
    p.row_order = row_order;
    p.partial_o = partial_o;
    p.partial_lse = partial_lse;
    p.out = static_cast<uint16_t*>(out);
    p.out_mirror = nullptr;
    p.arrivals = arrivals;
    p.status_flag = status_flag;
    p.stride_scales = cache.stride_scales;
    p.scale_log2 = scale * LOG2E;
    p.gpp = static_cast<uint32_t>(page_size / GRAN);
    p.gpp_magic = p.gpp > 1 ? static_cast<uint32_t>(((1ull << 32) + p.gpp - 1) / p.gpp) : 0u;
    p.gpb = cache.block / GRAN;
    p.box = q8_attn_box(page_size);
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
    p.block = cache.block;
    int dev = 0;
    cudaGetDevice(&dev);
    const int sms = device_state(dev).sm_count;
    const bool wide = Hq / Hkv > 8;
#define AC_Q8_LAUNCH(D_, FMT_)                                                                                        \
    (wide ? launch_q8<D_, FMT_, 2>(k_map, v_map, p, B, sms, stream) : launch_q8<D_, FMT_, 1>(k_map, v_map, p, B, sms, stream))
    if (d == 128) return cache.format == Q8_INT8 ? AC_Q8_LAUNCH(128, Q8_INT8) : AC_Q8_LAUNCH(128, Q8_E4M3);
    return cache.format == Q8_INT8 ? AC_Q8_LAUNCH(64, Q8_INT8) : AC_Q8_LAUNCH(64, Q8_E4M3);
#undef AC_Q8_LAUNCH
}

}  // namespace ac
