// What writes and reads the 4-bit cache outside attention: RoPE + append of one token per row, and the bulk
// store and load of many tokens per row.
#include "ac_internal.h"
#include "q4_format.cuh"
#include "rope_variant.cuh"

namespace ac {
namespace {

using namespace acdev;

// One warp per head vector of the new token: Hq query heads (rotated into q_out), Hkv keys (rotated, quantised)
// and Hkv values (quantised).  Lane l holds elements l * D/32 ...; a group of 32, 64 or 128 elements is then
// 8, 16 or 32 consecutive lanes (16 or 32 at D = 64).
template <int D, int G>
__global__ void __launch_bounds__(128) rope_kv_append_q4_kernel(
    const uint16_t* q_in, uint16_t* q_out, const uint16_t* __restrict__ k_new, const uint16_t* __restrict__ v_new,
    const Q4View cache, const int32_t* __restrict__ block_table, int max_pages_per_seq,
    const int32_t* __restrict__ context_lens, const float* __restrict__ rope_cos, const float* __restrict__ rope_sin,
    int max_position, int B, int Hq, int Hkv, int page_size, int num_pages, int32_t* status_flag, int rotary_dim,
    int interleaved, const uint16_t* __restrict__ q_norm_w, const uint16_t* __restrict__ k_norm_w, float norm_eps) {
    // As the bf16 append kernel: wait for the preceding kernel, then let the next one in.
    cudaGridDependencySynchronize();
    cudaTriggerProgrammaticLaunchCompletion();
    constexpr int EPL = D / 32;
    __shared__ uint16_t s_vec[4][D];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int heads = Hq + 2 * Hkv;
    const long long vec = static_cast<long long>(blockIdx.x) * 4 + warp;
    if (vec >= static_cast<long long>(B) * heads) return;
    const int b = static_cast<int>(vec / heads);
    const int hh = static_cast<int>(vec % heads);
    const int p = context_lens[b];
    if (p < 0) return;
    const int page_idx = p / page_size;
    if (p >= max_position || page_idx >= max_pages_per_seq) {
        if (status_flag != nullptr && lane == 0) atomicOr(status_flag, AC_FLAG_POSITION_OOB);
        return;
    }
    const bool is_q = hh < Hq;
    const bool is_v = hh >= Hq + Hkv;
    const int h = is_q ? hh : is_v ? hh - Hq - Hkv : hh - Hq;
    int page = 0;
    if (!is_q) {
        page = block_table[static_cast<size_t>(b) * max_pages_per_seq + page_idx];
        if (page < 0 || page >= num_pages) {
            if (status_flag != nullptr && lane == 0) atomicOr(status_flag, AC_FLAG_PAGE_OOB);
            return;
        }
    }
    const uint16_t* src = is_q ? q_in + (static_cast<size_t>(b) * Hq + h) * D
                               : (is_v ? v_new : k_new) + (static_cast<size_t>(b) * Hkv + h) * D;
    uint16_t x[EPL];
#pragma unroll
    for (int e = 0; e < EPL; ++e) x[e] = src[lane * EPL + e];
    if (!is_v)
        rope_variant_vector<D>(x, is_q ? q_norm_w : k_norm_w, norm_eps,
                               rope_cos + static_cast<size_t>(p) * (rotary_dim / 2),
                               rope_sin + static_cast<size_t>(p) * (rotary_dim / 2), rotary_dim, interleaved,
                               s_vec[warp], lane);
    if (is_q) {
        uint16_t* dst = q_out + (static_cast<size_t>(b) * Hq + h) * D;
#pragma unroll
        for (int e = 0; e < EPL; ++e) dst[lane * EPL + e] = x[e];
        return;
    }
    constexpr int LANES = 32 / G;
    uint32_t words[EPL / 2], packed[1];
#pragma unroll
    for (int w = 0; w < EPL / 2; ++w) words[w] = x[2 * w] | (static_cast<uint32_t>(x[2 * w + 1]) << 16);
    const uint32_t sm = q4_quantise<EPL / 2, LANES>(words, packed, 0xffffffffu);
    const int slot = p - page_idx * page_size;
    uint8_t* dst = (is_v ? cache.v_codes : cache.k_codes) + static_cast<int64_t>(page) * cache.stride_page +
                   slot * cache.stride_token + h * cache.stride_head + lane * (EPL / 2);
    if (EPL == 4) *reinterpret_cast<uint16_t*>(dst) = static_cast<uint16_t>(packed[0]);
    else *dst = static_cast<uint8_t>(packed[0]);
    if (lane % LANES == 0) {
        uint32_t* prm = cache.params + ((static_cast<int64_t>(page) * Hkv + h) * page_size + slot) * (2 * G);
        prm[(is_v ? G : 0) + lane / LANES] = sm;
    }
}

// ---- bulk store and load ---------------------------------------------------------------------------------
//
// Every warp takes runs of consecutive tokens in turn and works by itself: its lanes find the slots of one token each (row
// by binary search in row_offsets, position, page), then it goes through the run's (token, head) vectors, K then V, with
// D/16 lanes of 2 x 16 dense bytes (2 x 4 packed ones) per vector and kInHand vectors per lane at a time, so that their
// loads overlap.  (A lane's two pieces lie half a group apart, so that lanes side by side read and write side by side.)
// Bound: HBM, 2 dense and 0.56 packed bytes per element at group 64.  70.3 thousand tokens of 8 heads of 128, K and V: the
// load runs at that bound (65 us, 369 MB), the store at half of it (107 us): its 14 instructions per element, most of
// them the quotient and the extremes, and their latencies at 24 warps per SM.  Runs of 32 vectors against 8, 16 and 64: 169
// against 211, 177 and 174 us for both.  Store CTAs per SM and vectors in hand: (3, 2) 169, (4, 1) 171, (3, 1) 178, (5, 1) 184.
constexpr int kBulkThreads = 256;
constexpr int kRunVectors = 32;                            // vectors of a run, at least, where there are tokens enough
template <bool STORE>
struct Bulk {
    static constexpr int kCtas = STORE ? 3 : 4;            // per SM
    static constexpr int kInHand = STORE ? 2 : 4;          // a packed vector is a quarter of a dense one
};

struct TokenSlot {
    int64_t code;         // byte offset of the token's slot in the code pools; -1: no slot
    int64_t param;        // word offset of head 0's parameters
};

__device__ __forceinline__ TokenSlot find_slot(long long token, const Q4View& cache, int words, const int32_t* block_table,
                                               int max_pages_per_seq, const int32_t* start_pos,
                                               const int32_t* row_offsets, int B, int Hkv, int page_size, int num_pages,
                                               int32_t* status_flag) {
    TokenSlot r{-1, 0};
    if (token >= row_offsets[B]) return r;
    int lo = 0, hi = B;                                    // the last row whose offset is <= token
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (row_offsets[mid] <= token) lo = mid; else hi = mid;
    }
    const int start = start_pos[lo];
    if (start < 0 || token < row_offsets[lo]) return r;    // tokens before row 0 belong to no row: no position below 0
    const long long pos = start + (token - row_offsets[lo]);
    const long long idx = pos / page_size;
    if (idx >= max_pages_per_seq) {
        if (status_flag != nullptr) atomicOr(status_flag, AC_FLAG_POSITION_OOB);
        return r;
    }
    const int page = block_table[static_cast<size_t>(lo) * max_pages_per_seq + idx];
    if (page < 0 || page >= num_pages) {
        if (status_flag != nullptr) atomicOr(status_flag, AC_FLAG_PAGE_OOB);
        return r;
    }
    const int slot = static_cast<int>(pos - idx * page_size);
    r.code = page * cache.stride_page + slot * cache.stride_token;
    r.param = (static_cast<int64_t>(page) * Hkv * page_size + slot) * words;
    return r;
}

template <int D, int G, bool STORE>
__global__ void __launch_bounds__(kBulkThreads, Bulk<STORE>::kCtas) kv_bulk_q4_kernel(
    uint16_t* k, uint16_t* v, const Q4View cache, const int32_t* __restrict__ block_table, int max_pages_per_seq,
    const int32_t* __restrict__ start_pos, const int32_t* __restrict__ row_offsets, int total_tokens, int run, int B,
    int Hkv, int page_size, int num_pages, int32_t* status_flag) {
    constexpr int LPV = D / 16;                            // lanes per vector
    constexpr int VECS = 32 / LPV;                         // vectors per pass of the warp
    constexpr int LANES = LPV / G;                         // lanes per group
    constexpr int kInHand = Bulk<STORE>::kInHand;
    constexpr int WARPS = kBulkThreads / 32;
    __shared__ TokenSlot s_slots[WARPS][32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    TokenSlot* const s_slot = s_slots[warp];

    const int first = lane / LPV;                          // this lane's first vector of the run
    const int group = lane % LPV / LANES, rank = lane % LANES;
    const int piece = group * 2 * LANES + rank;            // its first 16 dense bytes; LANES further the second
    const uint32_t lanes = LPV == 8 ? 0xffu << (lane & 24) : 0xfu << (lane & 28);
    // (token, head) of a lane's vectors is stepped instead of divided, and with it the head's place in a slot
    const int first_t = first / Hkv, first_h = first - first_t * Hkv;
    const int step_t = VECS / Hkv, step_h = VECS - step_t * Hkv;
    const int64_t head_words = static_cast<int64_t>(page_size) * 2 * G;    // parameters of a page and head
    const int64_t code_step = step_h * cache.stride_head, code_wrap = Hkv * cache.stride_head;
    const int64_t param_step = step_h * head_words, param_wrap = Hkv * head_words;

    const unsigned runs = (static_cast<unsigned>(total_tokens) + run - 1) / run;
    for (unsigned r = warp * gridDim.x + blockIdx.x; r < runs; r += gridDim.x * WARPS) {
        const long long t0 = static_cast<long long>(r) * run;
        const int tokens = total_tokens - t0 < run ? static_cast<int>(total_tokens - t0) : run;
        const int vecs = tokens * Hkv;                     // (token, head), head fastest: dense order
        __syncwarp();
        if (lane < tokens)
            s_slot[lane] = find_slot(t0 + lane, cache, 2 * G, block_table, max_pages_per_seq, start_pos, row_offsets, B,
                                     Hkv, page_size, num_pages, status_flag);
        __syncwarp();
        for (int side = 0; side < 2; ++side) {
            uint16_t* dense = (side ? v : k) + (t0 * Hkv + first) * D + piece * 8;
            uint8_t* codes = (side ? cache.v_codes : cache.k_codes) + piece * 4 + first_h * cache.stride_head;
            uint32_t* params = cache.params + side * G + group + first_h * head_words;
            int t = first_t, h = first_h;
            for (int i = first; i < vecs; i += kInHand * VECS, dense += kInHand * VECS * D) {
                bool live[kInHand];
                uint8_t* code_at[kInHand];
                uint32_t* param_at[kInHand];
                uint4 raw[kInHand][2];
                uint32_t word[kInHand][2], sm[kInHand];
#pragma unroll
                for (int u = 0; u < kInHand; ++u) {
                    const bool on = i + u * VECS < vecs;
                    const TokenSlot at = s_slot[on ? t : 0];
                    live[u] = on && at.code >= 0;
                    code_at[u] = codes + at.code;
                    param_at[u] = params + at.param;
                    if (STORE) {
                        if (live[u]) {
                            raw[u][0] = __ldcs(reinterpret_cast<const uint4*>(dense + u * VECS * D));
                            raw[u][1] = __ldcs(reinterpret_cast<const uint4*>(dense + u * VECS * D) + LANES);
                        }
                    } else if (live[u]) {
                        word[u][0] = *reinterpret_cast<const uint32_t*>(code_at[u]);
                        word[u][1] = *reinterpret_cast<const uint32_t*>(code_at[u] + 4 * LANES);
                        sm[u] = *param_at[u];
                    }
                    t += step_t;
                    h += step_h;
                    codes += code_step;
                    params += param_step;
                    if (h >= Hkv) {
                        h -= Hkv;
                        ++t;
                        codes -= code_wrap;
                        params -= param_wrap;
                    }
                }
#pragma unroll
                for (int u = 0; u < kInHand; ++u) {
                    if (STORE) {
                        if (!live[u]) continue;            // uniform over the vector's lanes
                        const uint32_t x[8] = {raw[u][0].x, raw[u][0].y, raw[u][0].z, raw[u][0].w,
                                               raw[u][1].x, raw[u][1].y, raw[u][1].z, raw[u][1].w};
                        uint32_t packed[2];
                        const uint32_t p = q4_quantise<8, LANES>(x, packed, lanes);
                        *reinterpret_cast<uint32_t*>(code_at[u]) = packed[0];
                        *reinterpret_cast<uint32_t*>(code_at[u] + 4 * LANES) = packed[1];
                        if (rank == 0) *param_at[u] = p;
                    } else if (i + u * VECS < vecs) {
                        uint4* to = reinterpret_cast<uint4*>(dense + u * VECS * D);
                        const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
                        __stcs(to, live[u] ? q4_values(word[u][0], sm[u]) : zero);
                        __stcs(to + LANES, live[u] ? q4_values(word[u][1], sm[u]) : zero);
                    }
                }
            }
        }
    }
}

template <int D, int G>
cudaError_t launch_bulk(void* k, void* v, const Q4View& cache, const int32_t* block_table, int max_pages_per_seq,
                        const int32_t* start_pos, const int32_t* row_offsets, int total_tokens, int B, int Hkv,
                        int page_size, int num_pages, int32_t* status_flag, bool store, int sms,
                        cudaStream_t stream) {
    // Ordinary launches: what follows them in the stream may read the cache before its own synchronisation, which
    // is safe only behind kernels that do not signal early.
    const int ctas = (store ? Bulk<true>::kCtas : Bulk<false>::kCtas) * sms;
    // Shorter runs where there would not be one for every warp of the GPU, but no shorter than what a warp has in hand.
    const int in_hand = 32 / (D / 16) * (store ? Bulk<true>::kInHand : Bulk<false>::kInHand);
    int run = kRunVectors > Hkv ? kRunVectors / Hkv : 1;
    while (run > 1 && total_tokens / run < ctas * (kBulkThreads / 32) && run / 2 * Hkv >= in_hand) run /= 2;
    const long long runs = (static_cast<long long>(total_tokens) + run - 1) / run;
    const unsigned grid = static_cast<unsigned>(runs < ctas ? runs : ctas);
    uint16_t* kk = static_cast<uint16_t*>(k);
    uint16_t* vv = static_cast<uint16_t*>(v);
    if (store)
        kv_bulk_q4_kernel<D, G, true><<<grid, kBulkThreads, 0, stream>>>(
            kk, vv, cache, block_table, max_pages_per_seq, start_pos, row_offsets, total_tokens, run, B, Hkv, page_size,
            num_pages, status_flag);
    else
        kv_bulk_q4_kernel<D, G, false><<<grid, kBulkThreads, 0, stream>>>(
            kk, vv, cache, block_table, max_pages_per_seq, start_pos, row_offsets, total_tokens, run, B, Hkv, page_size,
            num_pages, status_flag);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_rope_kv_append_q4(const void* q_in, void* q_out, const void* k_new, const void* v_new,
                                     const Q4View& cache, const int32_t* block_table, int max_pages_per_seq,
                                     const int32_t* context_lens, const float* rope_cos, const float* rope_sin,
                                     int max_position, int B, int Hq, int Hkv, int d, int page_size, int num_pages,
                                     int32_t* status_flag, const RopeVariant* variant, cudaStream_t stream) {
    const RopeVariant plain{d, 0, nullptr, nullptr, 0.0f};
    const RopeVariant& r = variant != nullptr ? *variant : plain;
    const long long vecs = static_cast<long long>(B) * (Hq + 2ll * Hkv);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>((vecs + 3) / 4));
    cfg.blockDim = dim3(128);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
#define AC_Q4_APPEND(D_, G_)                                                                                       \
    cudaLaunchKernelEx(&cfg, rope_kv_append_q4_kernel<D_, G_>, static_cast<const uint16_t*>(q_in),                  \
                       static_cast<uint16_t*>(q_out), static_cast<const uint16_t*>(k_new),                          \
                       static_cast<const uint16_t*>(v_new), cache, block_table, max_pages_per_seq, context_lens,    \
                       rope_cos, rope_sin, max_position, B, Hq, Hkv, page_size, num_pages, status_flag,             \
                       r.rotary_dim, r.interleaved, static_cast<const uint16_t*>(r.q_norm_weight),                  \
                       static_cast<const uint16_t*>(r.k_norm_weight), r.norm_eps)
    const int groups = d / cache.group;
    if (d == 128) return groups == 1 ? AC_Q4_APPEND(128, 1) : groups == 2 ? AC_Q4_APPEND(128, 2) : AC_Q4_APPEND(128, 4);
    return groups == 1 ? AC_Q4_APPEND(64, 1) : AC_Q4_APPEND(64, 2);
#undef AC_Q4_APPEND
}

cudaError_t launch_kv_bulk_q4(void* k, void* v, const Q4View& cache, const int32_t* block_table,
                              int max_pages_per_seq, const int32_t* start_pos, const int32_t* row_offsets,
                              int total_tokens, int B, int Hkv, int d, int page_size, int num_pages,
                              int32_t* status_flag, bool store, int sms, cudaStream_t stream) {
#define AC_Q4_BULK(D_, G_)                                                                                          \
    launch_bulk<D_, G_>(k, v, cache, block_table, max_pages_per_seq, start_pos, row_offsets, total_tokens, B, Hkv,  \
                        page_size, num_pages, status_flag, store, sms, stream)
    const int groups = d / cache.group;
    if (d == 128) return groups == 1 ? AC_Q4_BULK(128, 1) : groups == 2 ? AC_Q4_BULK(128, 2) : AC_Q4_BULK(128, 4);
    return groups == 1 ? AC_Q4_BULK(64, 1) : AC_Q4_BULK(64, 2);
#undef AC_Q4_BULK
}

}  // namespace ac
