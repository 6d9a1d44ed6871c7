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
    uint32_t c[EPL];
    constexpr int LANES = 32 / G;
    const uint32_t sm = q4_quantise<EPL, LANES>(x, c, 0xffffffffu);
    const int slot = p - page_idx * page_size;
    uint8_t* dst = (is_v ? cache.v_codes : cache.k_codes) + static_cast<int64_t>(page) * cache.stride_page +
                   slot * cache.stride_token + h * cache.stride_head + lane * (EPL / 2);
    if (EPL == 4) {
        *reinterpret_cast<uint16_t*>(dst) = static_cast<uint16_t>(c[0] | (c[1] << 4) | (c[EPL - 2] << 8) | (c[EPL - 1] << 12));
    } else {
        *dst = static_cast<uint8_t>(c[0] | (c[1] << 4));
    }
    if (lane % LANES == 0) {
        uint32_t* prm = cache.params + ((static_cast<int64_t>(page) * Hkv + h) * page_size + slot) * (2 * G);
        prm[(is_v ? G : 0) + lane / LANES] = sm;
    }
}

// ---- bulk store and load ---------------------------------------------------------------------------------
//
// A CTA takes kTokens consecutive tokens of the dense side.  One thread per token finds its row (binary search in
// row_offsets), position, page and slot; then the CTA walks (token, side, head) vectors, D/8 lanes of 16 dense
// bytes (4 packed ones) each.  Bound: HBM, 2 dense and 0.56 packed bytes per element at group 64.
constexpr int kTokens = 16;
constexpr int kStoreThreads = 256;

struct TokenSlot {
    int page;             // -1: no slot
    int slot;
};

__device__ __forceinline__ TokenSlot find_slot(long long token, const int32_t* block_table, int max_pages_per_seq,
                                               const int32_t* start_pos, const int32_t* row_offsets, int B,
                                               int page_size, int num_pages, int32_t* status_flag) {
    TokenSlot r{-1, 0};
    if (token >= row_offsets[B]) return r;
    int lo = 0, hi = B;                                    // the last row whose offset is <= token
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (row_offsets[mid] <= token) lo = mid; else hi = mid;
    }
    const int start = start_pos[lo];
    if (start < 0) return r;
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
    r.page = page;
    r.slot = static_cast<int>(pos - idx * page_size);
    return r;
}

template <int D, int G, bool STORE>
__global__ void __launch_bounds__(kStoreThreads) kv_bulk_q4_kernel(
    uint16_t* k, uint16_t* v, const Q4View cache, const int32_t* __restrict__ block_table, int max_pages_per_seq,
    const int32_t* __restrict__ start_pos, const int32_t* __restrict__ row_offsets, int total_tokens, int B, int Hkv,
    int page_size, int num_pages, int32_t* status_flag) {
    constexpr int LPV = D / 8;                             // lanes per vector
    constexpr int VECS = kStoreThreads / LPV;              // vectors in hand at a time
    constexpr int LANES = LPV / G;                         // lanes per group
    __shared__ TokenSlot s_slot[kTokens];
    const long long t0 = static_cast<long long>(blockIdx.x) * kTokens;
    if (threadIdx.x < kTokens) {
        TokenSlot r{-1, 0};
        if (t0 + threadIdx.x < total_tokens)
            r = find_slot(t0 + threadIdx.x, block_table, max_pages_per_seq, start_pos, row_offsets, B, page_size,
                          num_pages, status_flag);
        s_slot[threadIdx.x] = r;
    }
    __syncthreads();
    const int tokens = total_tokens - t0 < kTokens ? static_cast<int>(total_tokens - t0) : kTokens;
    const int sub = threadIdx.x % LPV;
    const int vecs = tokens * 2 * Hkv;                     // (side, token, head), head fastest
    const uint32_t lanes = LPV == 16 ? 0xffffu << (threadIdx.x & 16) : 0xffu << (threadIdx.x & 24);
    for (int i = threadIdx.x / LPV; i < vecs; i += VECS) {
        const int side = i / (tokens * Hkv);
        const int rest = i - side * tokens * Hkv;
        const int t = rest / Hkv;
        const int h = rest - t * Hkv;
        const TokenSlot at = s_slot[t];
        uint16_t* dense = (side ? v : k) + ((t0 + t) * Hkv + h) * D + sub * 8;
        uint8_t* codes = (side ? cache.v_codes : cache.k_codes) + static_cast<int64_t>(at.page) * cache.stride_page +
                         at.slot * cache.stride_token + h * cache.stride_head + sub * 4;
        uint32_t* prm = cache.params + ((static_cast<int64_t>(at.page) * Hkv + h) * page_size + at.slot) * (2 * G) +
                        side * G + sub / LANES;
        if (STORE) {
            if (at.page < 0) continue;                     // uniform over the vector's lanes
            const uint4 raw = *reinterpret_cast<const uint4*>(dense);
            const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
            uint16_t x[8];
            uint32_t c[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = static_cast<uint16_t>(w[e >> 1] >> ((e & 1) * 16));
            const uint32_t sm = q4_quantise<8, LANES>(x, c, lanes);
            uint32_t packed = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) packed |= c[e] << (4 * e);
            *reinterpret_cast<uint32_t*>(codes) = packed;
            if (sub % LANES == 0) *prm = sm;
        } else {
            uint4 o = make_uint4(0u, 0u, 0u, 0u);
            if (at.page >= 0) {
                const uint32_t packed = *reinterpret_cast<const uint32_t*>(codes);
                const uint32_t sm = *prm;
                const float s = __uint_as_float(sm << 16), m = __uint_as_float(sm & 0xFFFF0000u);
                float y[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = fmaf(static_cast<float>((packed >> (4 * e)) & 15u), s, m);
                o = make_uint4(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]),
                               pack_bf16x2(y[6], y[7]));
            }
            *reinterpret_cast<uint4*>(dense) = o;
        }
    }
}

template <int D, int G>
cudaError_t launch_bulk(void* k, void* v, const Q4View& cache, const int32_t* block_table, int max_pages_per_seq,
                        const int32_t* start_pos, const int32_t* row_offsets, int total_tokens, int B, int Hkv,
                        int page_size, int num_pages, int32_t* status_flag, bool store, cudaStream_t stream) {
    // Ordinary launches: what follows them in the stream may read the cache before its own synchronisation, which
    // is safe only behind kernels that do not signal early.
    const unsigned grid = static_cast<unsigned>((static_cast<long long>(total_tokens) + kTokens - 1) / kTokens);
    uint16_t* kk = static_cast<uint16_t*>(k);
    uint16_t* vv = static_cast<uint16_t*>(v);
    if (store)
        kv_bulk_q4_kernel<D, G, true><<<grid, kStoreThreads, 0, stream>>>(
            kk, vv, cache, block_table, max_pages_per_seq, start_pos, row_offsets, total_tokens, B, Hkv, page_size,
            num_pages, status_flag);
    else
        kv_bulk_q4_kernel<D, G, false><<<grid, kStoreThreads, 0, stream>>>(
            kk, vv, cache, block_table, max_pages_per_seq, start_pos, row_offsets, total_tokens, B, Hkv, page_size,
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
                              int32_t* status_flag, bool store, cudaStream_t stream) {
#define AC_Q4_BULK(D_, G_)                                                                                          \
    launch_bulk<D_, G_>(k, v, cache, block_table, max_pages_per_seq, start_pos, row_offsets, total_tokens, B, Hkv,  \
                        page_size, num_pages, status_flag, store, stream)
    const int groups = d / cache.group;
    if (d == 128) return groups == 1 ? AC_Q4_BULK(128, 1) : groups == 2 ? AC_Q4_BULK(128, 2) : AC_Q4_BULK(128, 4);
    return groups == 1 ? AC_Q4_BULK(64, 1) : AC_Q4_BULK(64, 2);
#undef AC_Q4_BULK
}

}  // namespace ac
