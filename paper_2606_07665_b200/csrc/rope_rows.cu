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
    int chunk, q_chunks, chunks;                                   // heads of a piece of a token; pieces of its q, of q and k
    int32_t* status_flag;
};

// A piece: `chunk` heads of q or of k of one token.
struct Piece {
    const uint16_t* src;
    uint16_t* dst;
    const uint16_t* norm_w;
    int heads;
};
template <int D>
__device__ __forceinline__ Piece find_piece(const RowsParams& p, int token, int piece) {
    const bool is_q = piece < p.q_chunks;
    const int from = (is_q ? piece : piece - p.q_chunks) * p.chunk;
    Piece r;
    r.src = (is_q ? p.q_in + token * p.q_in_token : p.k_in + token * p.k_in_token) + from * D;
    r.dst = (is_q ? p.q_out + token * p.q_out_token : p.k_out + token * p.k_out_token) + from * D;
    r.norm_w = is_q ? p.q_norm_w : p.k_norm_w;
    r.heads = min(p.chunk, (is_q ? p.Hq : p.Hkv) - from);
    return r;
}

// Position of a token of row `row`, or -1 where it has none.
__device__ __forceinline__ int position_in(const RowsParams& p, int row, int token, bool tell) {
    const int begin = p.row_offsets[row], end = p.row_offsets[row + 1], start = p.start_pos[row];
    if (token < begin || token >= end || start < 0) return -1;
    const long long pos = static_cast<long long>(start) + (token - begin);
    if (pos >= p.max_position) {
        if (p.status_flag != nullptr && tell) atomicOr(p.status_flag, AC_FLAG_POSITION_OOB);
        return -1;
    }
    return static_cast<int>(pos);
}

// The row of a token is the last one whose offset is <= token.  Here for one token of the whole warp: each round the 32 lanes
// look at the ends of 32 equal pieces of what is left.
__device__ __forceinline__ int warp_token_position(const RowsParams& p, int token, int lane) {
    int lo = 0, n = p.B;                                   // the row is in [lo, lo + n)
    while (n > 1) {
        const int piece = (n + 31) / 32;
        const int first = lane * piece;                    // offsets of the pieces' first rows, the first of which is known
        const bool below = lane > 0 && first < n && p.row_offsets[lo + first] <= token;
        const int k = __popc(__ballot_sync(0xffffffffu, below));      // offsets do not decrease: lanes 1 .. k
        lo += k * piece;
        n = min(piece, n - k * piece);
    }
    return position_in(p, lo, token, lane == 0);
}
// And for a token of each lane.
__device__ __forceinline__ int lane_token_position(const RowsParams& p, int token) {
    int lo = 0, hi = p.B;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (p.row_offsets[mid] <= token) lo = mid; else hi = mid;
    }
    return position_in(p, lo, token, true);
}

// The sum of squares as rope_variant_vector forms it: D/32 neighbours at a time, these partial sums joined at distances 16, 8, 4, 2, 1.
// a and b are the lane's two runs of eight elements; the runs are brought into order among the D/16 lanes first.
template <int D, bool INTERLEAVED>
__device__ __noinline__ double squares_in_order(uint4 a, uint4 b, int rotary_dim, int lane) {
    constexpr int EPL = D / 32, NP = 8 / EPL, LPV = D / 16;        // elements of a partial sum, partial sums of a run, lanes
    const uint32_t words[2][4] = {{a.x, a.y, a.z, a.w}, {b.x, b.y, b.z, b.w}};
    double part[2][NP], sum[2 * NP];
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            part[r][i] = 0.0;
#pragma unroll
            for (int e = i * EPL; e < (i + 1) * EPL; ++e) {
                const uint32_t w = words[r][e >> 1];
                const double d = static_cast<double>(__uint_as_float((e & 1) ? w & 0xFFFF0000u : w << 16));
                part[r][i] = __fma_rn(d, d, part[r][i]);
            }
        }
    const int at = lane % LPV, turned = rotary_dim / 16;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int run = 2 * at + r;                        // which lane holds it, as its first or second (see LaneElements)
        const bool halves = !INTERLEAVED && run < 2 * turned;
        const int holder = lane - at + (!halves ? at : run < turned ? run : run - turned);
        const bool second = halves ? run >= turned : r == 1;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const double s0 = __shfl_sync(0xffffffffu, part[0][i], holder), s1 = __shfl_sync(0xffffffffu, part[1][i], holder);
            sum[r * NP + i] = second ? s1 : s0;
        }
    }
#pragma unroll
    for (int off = LPV / 2; off >= 1; off >>= 1)
#pragma unroll
        for (int i = 0; i < 2 * NP; ++i) sum[i] = __dadd_rn(sum[i], __shfl_xor_sync(0xffffffffu, sum[i], off));
#pragma unroll
    for (int off = NP; off >= 1; off >>= 1)
#pragma unroll
        for (int i = 0; i < off; ++i) sum[i] = __dadd_rn(sum[i], sum[i + off]);
    return sum[0];
}

// Per-head RMSNorm of a lane's 16 elements (words x), D/16 lanes per vector, with the bits of rope_variant_vector.  The whole warp.
//
// Nearly always the squares add up exactly, in whatever order: elements whose least exponent field is f are multiples of
// q = 2^(f - 134), their squares and sums of them of q^2, and those below 2^53 q^2 are fp64 numbers.  (Zeros do not count; f is taken over
// the warp; the sum is looked at with a bit to spare, since it is rounded where it is not exact.)
//
// Bound: instructions, 50 per element and lane with it, 12 without (issue slots 57 %, ALU 51, 3 warps a scheduler): 70.3 thousand tokens
// of 40 heads of 128 864 us (850 without the look at the exponents), 240 without norms.
template <int D, bool INTERLEAVED>
__device__ __forceinline__ void normalise16(uint32_t (&x)[8], const uint16_t* w0, const uint16_t* w1, float eps, int rotary_dim, int lane) {
    double ss = 0.0;
    uint32_t least = 0xFFFFFFFFu;                          // of the magnitudes minus 1, where zero is the largest
#pragma unroll
    for (int i = 0; i < 8; ++i) least = __viaddmin_u16x2(x[i] & 0x7FFF7FFFu, 0xFFFFFFFFu, least);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const double d = static_cast<double>(__uint_as_float((e & 1) ? x[e >> 1] & 0xFFFF0000u : x[e >> 1] << 16));
        ss = __fma_rn(d, d, ss);                           // d * d is exact
    }
#pragma unroll
    for (int off = D / 32; off >= 1; off >>= 1) ss = __dadd_rn(ss, __shfl_xor_sync(0xffffffffu, ss, off));
    const int f = static_cast<int>((__reduce_min_sync(0xffffffffu, min(least & 0xFFFFu, least >> 16)) + 1u) >> 7);
    const bool exact = (__double2hiint(ss) >> 20) - 1023 + 2 <= 53 + 2 * (f - 134);
    if (!__all_sync(0xffffffffu, exact))
        ss = squares_in_order<D, INTERLEAVED>(make_uint4(x[0], x[1], x[2], x[3]), make_uint4(x[4], x[5], x[6], x[7]), rotary_dim, lane);
    const double rr = __ddiv_rn(1.0, __dsqrt_rn(__dadd_rn(__ddiv_rn(ss, static_cast<double>(D)), static_cast<double>(eps))));
    const float rr_hi = static_cast<float>(rr), rr_lo = static_cast<float>(rr - static_cast<double>(rr_hi));
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const uint4 wv = __ldg(reinterpret_cast<const uint4*>(half ? w1 : w0));
        const uint32_t wr[4] = {wv.x, wv.y, wv.z, wv.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t raw = x[4 * half + e];
            x[4 * half + e] = rmsnorm_feature(static_cast<uint16_t>(raw), rr, rr_hi, rr_lo, __uint_as_float(wr[e] << 16)) |
                              (static_cast<uint32_t>(rmsnorm_feature(static_cast<uint16_t>(raw >> 16), rr, rr_hi, rr_lo,
                                                                     __uint_as_float(wr[e] & 0xFFFF0000u))) << 16);
        }
    }
}

__device__ __forceinline__ void unpack(uint32_t (&x)[8], const uint4& a, const uint4& b) {
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
}

// How the elements of a vector lie in D/16 lanes: a lane holds eight pairs, 16 bytes of either half, or 32 side by side where pairs are
// interleaved (lanes past the rotary part hold 32 as well), so that partners never leave a lane and an angle serves two results.
template <int D, bool INTERLEAVED>
struct LaneElements {
    int at, e0, apart;                                     // lane in the vector; its two runs of eight elements
    bool turned;
    __device__ __forceinline__ LaneElements(int lane, int rotary_dim) {
        at = lane % (D / 16);
        turned = at < rotary_dim / 16;
        e0 = INTERLEAVED || !turned ? 16 * at : 8 * at;
        apart = INTERLEAVED || !turned ? 8 : rotary_dim / 2;
    }
};

// Few tokens: a warp takes a piece, four (D = 128) or eight vectors side by side, straight from and to memory.
template <int D, bool INTERLEAVED, bool NORM>
__global__ void __launch_bounds__(128) rope_rows_kernel(const RowsParams p) {
    constexpr int LPV = D / 16, VECS = 32 / LPV, U = 2;    // U vectors of a lane at a time
    const int lane = threadIdx.x & 31;
    const unsigned item = blockIdx.x * 4 + (threadIdx.x >> 5);
    const int token = static_cast<int>(item / static_cast<unsigned>(p.chunks));
    if (token >= p.total_tokens) return;
    const Piece at = find_piece<D>(p, token, static_cast<int>(item - static_cast<unsigned>(token) * p.chunks));
    const LaneElements<D, INTERLEAVED> le(lane, p.rotary_dim);
    const uint16_t* const src = at.src + le.e0;
    uint16_t* const dst = at.dst + le.e0;

    uint4 x[U][2];
    auto load = [&](int h) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            x[u][0] = x[u][1] = make_uint4(0u, 0u, 0u, 0u);
            if (h + u * VECS < at.heads) {
                x[u][0] = __ldcs(reinterpret_cast<const uint4*>(src + (h + u * VECS) * D));
                x[u][1] = __ldcs(reinterpret_cast<const uint4*>(src + (h + u * VECS) * D + le.apart));
            }
        }
    };
    load(lane / LPV);                                      // does not wait for the position
    const int pos = warp_token_position(p, token, lane);
    if (pos < 0) return;
    RopeAngles angles;
    const size_t angle0 = static_cast<size_t>(pos) * (p.rotary_dim / 2) + (le.turned ? 8 * le.at : 0);
    angles.set(p.rope_cos + angle0, p.rope_sin + angle0);
    for (int h0 = 0; h0 < at.heads; h0 += U * VECS) {
        if (h0 > 0) load(h0 + lane / LPV);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int h = h0 + lane / LPV + u * VECS;
            uint32_t v[8];
            unpack(v, x[u][0], x[u][1]);
            if (NORM && at.norm_w != nullptr) normalise16<D, INTERLEAVED>(v, at.norm_w + le.e0, at.norm_w + le.e0 + le.apart, p.norm_eps, p.rotary_dim, lane);
            if (h < at.heads) {
                if (le.turned) rope_turn16<INTERLEAVED>(v, angles);
                __stcs(reinterpret_cast<uint4*>(dst + h * D), make_uint4(v[0], v[1], v[2], v[3]));
                __stcs(reinterpret_cast<uint4*>(dst + h * D + le.apart), make_uint4(v[4], v[5], v[6], v[7]));
            }
        }
    }
}

// Many tokens: the warps of persistent CTAs share the pieces out evenly.  Each has a ring of stages in shared memory; a stage receives
// a piece and its row of angles by bulk copies, is rotated in place and leaves by a bulk copy, so that the bytes in flight cost no
// registers: while a piece is rotated the next one arrives and the two before it leave.  Where the next 32 pieces lie is looked up at
// a time, one per lane.
//
// Bound: HBM, 2 bytes in and out per element: 70.3 thousand tokens of 40 heads of 128 (1.44 GB) 240 us = 6000 GB/s, 0.93 of the
// copy rate.  (Through registers, as above: 262 at best, 24 warps per SM.)
constexpr int kPieceBytes = 4096, kAngleBytes = 256;       // at most, of a piece and of its cosines or sines
// 70.3 thousand tokens of 40 heads of 128, us, in a burst and in a second of such calls, which the power limit holds back, by (stages,
// stores in flight) of 12 warps: (2, 0) 236 and 238, (3, 1) 238 and 239, (4, 2) 238 and 237, (4, 1) 256 and 235.  Warps that take the
// pieces in turn instead of neighbouring ones, (4, 2): 238 and 242, and 152 instead of 125 with heads of 64.
constexpr int kStreamWarps = 12, kStreamStages = 4;
constexpr int kStores = 2;                                 // stores that may still read their stages while the next piece is fetched
constexpr int kStageBytes = kPieceBytes + 2 * kAngleBytes;
constexpr int kStreamSmem = kStreamWarps * kStreamStages * (kStageBytes + 8) + 128;

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
                 "r"(bytes), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void bulk_load_once(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar, uint64_t policy) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;" ::"r"(dst),
                 "l"(src), "r"(bytes), "r"(bar), "l"(policy)
                 : "memory");
}
__device__ __forceinline__ void bulk_store(void* dst, uint32_t src, uint32_t bytes, uint64_t policy) {
    asm volatile("cp.async.bulk.global.shared::cta.bulk_group.L2::cache_hint [%0], [%1], %2, %3;" ::"l"(dst), "r"(src), "r"(bytes), "l"(policy)
                 : "memory");
}
__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void bulk_wait_read() {         // all but the last N stores have read their stage
    asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(N) : "memory");
}

template <int D, bool INTERLEAVED, bool NORM>
__global__ void __launch_bounds__(kStreamWarps * 32, 1) rope_rows_stream_kernel(const RowsParams p) {
    constexpr int LPV = D / 16, VECS = 32 / LPV, S = kStreamStages;
    extern __shared__ uint8_t smem_raw[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint8_t* const smem = smem_raw + (((smem_addr(smem_raw) + 127u) & ~127u) - smem_addr(smem_raw));
    uint8_t* const ring = smem + warp * S * kStageBytes;
    const uint32_t ring_at = smem_addr(ring);
    const uint32_t bars = smem_addr(smem + kStreamWarps * S * kStageBytes) + warp * S * 8;
    if (lane == 0) {
#pragma unroll
        for (int s = 0; s < S; ++s) mbar_init(bars + s * 8, 1);
        mbar_init_fence();
    }
    __syncwarp();

    const long long items = static_cast<long long>(p.total_tokens) * p.chunks;
    const unsigned warps = gridDim.x * kStreamWarps;
    const long long w = static_cast<long long>(blockIdx.x) * kStreamWarps + warp;
    const long long first = items * w / warps, n_my = items * (w + 1) / warps - first;     // this warp's pieces lie side by side
    const uint32_t angle_bytes = p.rotary_dim * 2;
    const uint64_t policy = l2_policy_evict_first();       // for what is read and written once; the angles serve many pieces
    const LaneElements<D, INTERLEAVED> le(lane, p.rotary_dim);

    // Lane l: piece 32 m + l, where it lies and how many heads it has (0: no position; negative: heads of k), among those being
    // fetched (i_) and among those being rotated (c_).
    const uint16_t* i_src = nullptr;
    uint16_t* i_dst = nullptr;
    uint16_t* c_dst = nullptr;
    int i_heads = 0, i_pos = 0, c_heads = 0;
    auto look_up = [&](long long n0) {
        const long long n = n0 + lane;
        i_heads = 0;
        if (n < n_my) {
            const long long item = first + n;
            const int token = static_cast<int>(item / p.chunks);
            const int piece = static_cast<int>(item - static_cast<long long>(token) * p.chunks);
            i_pos = lane_token_position(p, token);
            if (i_pos >= 0) {
                const Piece what = find_piece<D>(p, token, piece);
                i_src = what.src;
                i_dst = what.dst;
                i_heads = piece < p.q_chunks ? what.heads : -what.heads;
            }
        }
    };
    auto fetch = [&](long long n, int stage) {
        const int from = static_cast<int>(n & 31);
        const unsigned long long src = __shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(i_src), from);
        const int heads = abs(__shfl_sync(0xffffffffu, i_heads, from)), pos = __shfl_sync(0xffffffffu, i_pos, from);
        if (lane == 0) {
            const uint32_t bar = bars + stage * 8, at = ring_at + stage * kStageBytes;
            if (heads > 0) {
                const uint32_t bytes = heads * D * 2;
                mbar_arrive_expect_tx(bar, bytes + 2 * angle_bytes);
                bulk_load_once(at, reinterpret_cast<const void*>(src), bytes, bar, policy);
                const size_t angle0 = static_cast<size_t>(pos) * (p.rotary_dim / 2);
                bulk_load(at + kPieceBytes, p.rope_cos + angle0, angle_bytes, bar);
                bulk_load(at + kPieceBytes + kAngleBytes, p.rope_sin + angle0, angle_bytes, bar);
            } else {
                mbar_arrive(bar);                          // nothing to fetch, nothing to write
            }
        }
    };
    look_up(0);
#pragma unroll
    for (int s = 0; s < S - 1 - kStores; ++s)
        if (s < n_my) fetch(s, s);

    int stage = 0;
    uint32_t parity = 0;
    for (long long n = 0; n < n_my; ++n) {
        if ((n & 31) == 0) c_dst = i_dst, c_heads = i_heads;
        const long long ahead = n + S - 1 - kStores;
        if (ahead < n_my) {
            if ((ahead & 31) == 0) look_up(ahead);
            if (lane == 0) bulk_wait_read<kStores>();
            fetch(ahead, (stage + S - 1 - kStores) % S);
        }
        const int from = static_cast<int>(n & 31);
        const unsigned long long dst = __shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(c_dst), from);
        const int signed_heads = __shfl_sync(0xffffffffu, c_heads, from), heads = abs(signed_heads);
        if (!__all_sync(0xffffffffu, mbar_wait_bounded(bars + stage * 8, parity))) {
            // Record the failure, and give the copies in flight a bounded chance to land before the shared memory is released.
            if (lane == 0 && p.status_flag != nullptr) atomicOr(p.status_flag, AC_FLAG_WAIT_TIMEOUT);
            for (int s = 0; s < S - kStores && n + s < n_my; ++s)
                mbar_wait_bounded(bars + (stage + s) % S * 8, stage + s < S ? parity : parity ^ 1u);
            break;
        }
        if (heads > 0) {
            uint8_t* const at = ring + stage * kStageBytes;
            const uint16_t* const norm_w = signed_heads > 0 ? p.q_norm_w : p.k_norm_w;
            RopeAngles angles;
            const float* cr = reinterpret_cast<const float*>(at + kPieceBytes) + (le.turned ? 8 * le.at : 0);
            angles.set_shared(cr, cr + kAngleBytes / 4);
            uint16_t* const x = reinterpret_cast<uint16_t*>(at) + le.e0;
            for (int h0 = 0; h0 < heads; h0 += VECS) {
                const int h = h0 + lane / LPV;
                const bool on = h < heads;
                uint32_t v[8];
                if (NORM || (on && le.turned)) {
                    uint4* const v0 = reinterpret_cast<uint4*>(x + (on ? h : 0) * D);
                    uint4* const v1 = reinterpret_cast<uint4*>(x + (on ? h : 0) * D + le.apart);
                    unpack(v, *v0, *v1);
                    if (NORM) {
                        if (norm_w != nullptr) normalise16<D, INTERLEAVED>(v, norm_w + le.e0, norm_w + le.e0 + le.apart, p.norm_eps, p.rotary_dim, lane);
                        __syncwarp();                      // lanes without a vector of their own have read another's
                    }
                    if (on) {
                        if (le.turned) rope_turn16<INTERLEAVED>(v, angles);
                        *v0 = make_uint4(v[0], v[1], v[2], v[3]);
                        *v1 = make_uint4(v[4], v[5], v[6], v[7]);
                    }
                }
            }
            fence_proxy_async_shared();
            __syncwarp();
            if (lane == 0) bulk_store(reinterpret_cast<void*>(dst), ring_at + stage * kStageBytes, heads * D * 2, policy);
        }
        if (lane == 0) bulk_commit();                      // a group for every piece, empty where nothing is written
        if (++stage == S) {
            stage = 0;
            parity ^= 1u;
        }
    }
    if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
}

// The general form, for rotary parts that are no whole number of lanes: a warp per vector, partners through shared memory.  Bound: latency,
// a warp has one vector in hand: 70.3 thousand tokens of 40 heads of 128 in 1167 us with a rotary part of 18, 1195 with 34.
template <int D>
__global__ void __launch_bounds__(256) rope_rows_any_kernel(const RowsParams p) {
    constexpr int EPL = D / 32;
    __shared__ uint16_t s_vec[8][D];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const unsigned item = blockIdx.x * 8 + warp;
    const int token = static_cast<int>(item / static_cast<unsigned>(p.chunks));
    if (token >= p.total_tokens) return;
    const int pos = warp_token_position(p, token, lane);
    if (pos < 0) return;
    const Piece at = find_piece<D>(p, token, static_cast<int>(item - static_cast<unsigned>(token) * p.chunks));
    const float* cr = p.rope_cos + static_cast<size_t>(pos) * (p.rotary_dim / 2);
    const float* sr = p.rope_sin + static_cast<size_t>(pos) * (p.rotary_dim / 2);
    for (int h = 0; h < at.heads; ++h) {
        uint16_t x[EPL];
#pragma unroll
        for (int e = 0; e < EPL; ++e) x[e] = at.src[h * D + lane * EPL + e];
        if (at.norm_w != nullptr) rope_variant_vector<D>(x, at.norm_w, p.norm_eps, cr, sr, p.rotary_dim, p.interleaved, s_vec[warp], lane);
        else rope_vector<D>(x, cr, sr, p.rotary_dim, p.interleaved, s_vec[warp], lane);
#pragma unroll
        for (int e = 0; e < EPL; ++e) at.dst[h * D + lane * EPL + e] = x[e];
    }
}

#define AC_ROPE_EACH(DO, D_) DO(D_, false, false) DO(D_, false, true) DO(D_, true, false) DO(D_, true, true)

// From how many bytes of input on the streaming kernel is used: 28 + 4 heads of 128, us, direct and streaming: 200 tokens 3.1 and
// 4.8, 2000 (16 MB) 10.0 and 10.1, 4000 (33 MB) 17.2 and 14.8, 8000 31.2 and 26.0, 16000 59 and 47.
constexpr long long kStreamFromBytes = 24 << 20;

template <int D>
cudaError_t launch_rows(RowsParams p, int sms, cudaStream_t stream) {
    const bool any = p.rotary_dim % 16 != 0;
    const bool norm = p.q_norm_w != nullptr || p.k_norm_w != nullptr;
    const int heads = p.Hq + p.Hkv;
    const bool many = !any && static_cast<long long>(p.total_tokens) * heads * D * 2 >= kStreamFromBytes;
    // Pieces of 4 KB at most; where that leaves warps without one (32 per SM), half or a quarter of it.
    p.chunk = kPieceBytes / (2 * D);
    auto cut = [&]() {
        p.q_chunks = (p.Hq + p.chunk - 1) / p.chunk;
        p.chunks = p.q_chunks + (p.Hkv + p.chunk - 1) / p.chunk;
    };
    cut();
    while (!many && p.chunk > 1024 / (2 * D) && static_cast<long long>(p.total_tokens) * p.chunks < 32ll * sms) {
        p.chunk /= 2;
        cut();
    }
    const long long items = static_cast<long long>(p.total_tokens) * p.chunks;
    if (many) {
        const long long most = (items + kStreamWarps - 1) / kStreamWarps;
        const unsigned grid = static_cast<unsigned>(most < sms ? most : sms);
#define AC_ROPE_STREAM(D_, I_, N_)                                                                                   \
    if ((p.interleaved != 0) == I_ && norm == N_) rope_rows_stream_kernel<D_, I_, N_><<<grid, kStreamWarps * 32, kStreamSmem, stream>>>(p);
        AC_ROPE_EACH(AC_ROPE_STREAM, D)
#undef AC_ROPE_STREAM
        return cudaGetLastError();
    }
    if (items > 0xffffffffll - 8) return cudaErrorInvalidConfiguration;
    if (any) {
        rope_rows_any_kernel<D><<<static_cast<unsigned>((items + 7) / 8), 256, 0, stream>>>(p);
    } else {
        const unsigned grid = static_cast<unsigned>((items + 3) / 4);
#define AC_ROPE_DIRECT(D_, I_, N_)                                                                                   \
    if ((p.interleaved != 0) == I_ && norm == N_) rope_rows_kernel<D_, I_, N_><<<grid, 128, 0, stream>>>(p);
        AC_ROPE_EACH(AC_ROPE_DIRECT, D)
#undef AC_ROPE_DIRECT
    }
    return cudaGetLastError();
}

// ---- tables ------------------------------------------------------------------------------------------------
//
// A thread owns one frequency and `run` consecutive positions: cosine and sine of the first position's angle in fp64, then
// one rotation by the frequency's own angle per position (an error of 2^-52 each, 2^-47 after 32 of them: far below the
// fp32 that is written).  Four fp64 operations per pair instead of the hundred of a sine and a cosine.
// Bound: the writes, 4 bytes per entry: 131072 positions of 64 frequencies (67 MB) 13.4 us, 10.4 at the copy rate (runs of 64: 14.7).
// Few positions: latency (4096 of 32 frequencies 2.6 us in runs of 4, 4.4 without).
constexpr int kRun = 32;

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
    c *= sc.magnitude;
    s *= sc.magnitude;
    const int n = positions - p0 < run ? static_cast<int>(positions - p0) : run;
    float* co = cos_out + p0 * half + i;
    float* so = sin_out + p0 * half + i;
    for (int j = 0; j < n; ++j) {
        *co = static_cast<float>(c);
        *so = static_cast<float>(s);
        co += half;
        so += half;
        const double t = c * cd - s * sd;
        s = s * cd + c * sd;
        c = t;
    }
}

}  // namespace

cudaError_t rope_rows_set_attributes(int smem_optin) {
    if (kStreamSmem > smem_optin) return cudaErrorInvalidConfiguration;
    cudaError_t e = cudaSuccess;
#define AC_ROPE_SET(D_, I_, N_)                                                                                      \
    if (e == cudaSuccess)                                                                                            \
        e = cudaFuncSetAttribute(rope_rows_stream_kernel<D_, I_, N_>, cudaFuncAttributeMaxDynamicSharedMemorySize, kStreamSmem);
    AC_ROPE_EACH(AC_ROPE_SET, 128)
    AC_ROPE_EACH(AC_ROPE_SET, 64)
#undef AC_ROPE_SET
    return e;
}

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
    p.chunk = p.q_chunks = p.chunks = 0;
    p.status_flag = status_flag;
    return d == 128 ? launch_rows<128>(p, sms, stream) : launch_rows<64>(p, sms, stream);
}

cudaError_t launch_rope_tables(float* rope_cos, float* rope_sin, long long first_position, int positions, int rotary_dim,
                               const RopeScaling& scaling, int sms, cudaStream_t stream) {
    const int half = rotary_dim / 2;
    int run = kRun;                                        // shorter runs where the GPU would not be full
    auto runs = [&]() { return (positions - 1ll) / run + 1; };
    while (run > 1 && runs() * half < 128ll * sms) run /= 2;
    const long long threads = runs() * half;
    const long long grid = (threads + 255) / 256;
    if (grid > 0x7fffffffll) return cudaErrorInvalidConfiguration;
    rope_tables_kernel<<<static_cast<unsigned>(grid), 256, 0, stream>>>(rope_cos, rope_sin, first_position, positions, half, run, scaling);
    return cudaGetLastError();
}

}  // namespace ac
