// What writes and reads the 8-bit cache outside attention: RoPE + append of one token per row, and the bulk store and load
// of many tokens per row.
#include "ac_internal.h"
#include "q8_format.cuh"
#include "rope_fast.cuh"
#include "rope_variant.cuh"

namespace ac {
namespace {

using namespace acdev;

// Codes of the slots [from, from + n) of one (page, head) rounded again after multiplication by `factor`; the whole warp.
template <int D, int FMT>
__device__ __forceinline__ void requantise(uint8_t* first, int64_t stride_token, int n, float factor, int lane) {
    constexpr int WPT = D / 4, TPP = 32 / WPT, U = 4;      // words per token, tokens side by side, in flight
    uint8_t* at = first + lane / WPT * stride_token + lane % WPT * 4;
    for (int t = lane / WPT; t < n; t += U * TPP, at += U * TPP * stride_token) {
        uint32_t w[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (t + u * TPP < n) w[u] = *reinterpret_cast<const uint32_t*>(at + u * TPP * stride_token);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (t + u * TPP < n) *reinterpret_cast<uint32_t*>(at + u * TPP * stride_token) = q8_again<FMT>(w[u], factor);
    }
}

// The scale of a block for a writer that needs `need` and finds `before` tokens in front of it under the scale `held`: joins the two,
// rounds the held codes again where it grows, stores what has changed and returns it.  `codes` is the writer's first vector.  The
// whole warp, every lane of which has read `held`.
template <int D, int FMT>
__device__ __forceinline__ uint32_t settle_scale(const Q8View& cache, float* cell, uint8_t* codes, int before, uint32_t held, uint32_t need, int lane) {
    uint32_t scale = need;
    __syncwarp();                                          // every lane has read the held scale
    if (before > 0) {
        scale = q8_join(held, need);
        if (scale == held) return scale;
        if (scale != kQ8NaN)
            requantise<D, FMT>(codes - before * cache.stride_token, cache.stride_token, before,
                               __uint_as_float(held) * q8_inverse(scale), lane);
    }
    if (lane == 0) *cell = __uint_as_float(scale);
    return scale;
}

constexpr int kAppendThreads = 128;                        // 256 rows of 36 heads, us: 32 threads 10.0, 64 6.2, 128 5.9, 256 5.7

// One warp per head vector of the new token, as the append kernels of the other formats: Hq query heads (rotated into
// q_out), Hkv keys (rotated, quantised) and Hkv values (quantised).  A growing scale costs the warp the block's codes once
// more; no other warp writes the block.  Bound: latency, length -> page -> scale -> codes; the vector itself is asked
// for at once.  8 rows of 28:4 heads 2.7 us, 256 rows 5.9 (4-bit, whose rotation is fp64: 3.3 and 7.6).
template <int D, int FMT>
__global__ void __launch_bounds__(kAppendThreads) rope_kv_append_q8_kernel(
    const uint16_t* q_in, uint16_t* q_out, const uint16_t* __restrict__ k_new, const uint16_t* __restrict__ v_new,
    const Q8View cache, const int32_t* __restrict__ block_table, int max_pages_per_seq,
    const int32_t* __restrict__ context_lens, const float* __restrict__ rope_cos, const float* __restrict__ rope_sin,
    int max_position, int B, int Hq, int Hkv, int page_size, int num_pages, int32_t* status_flag, int rotary_dim,
    int interleaved, const uint16_t* __restrict__ q_norm_w, const uint16_t* __restrict__ k_norm_w, float norm_eps) {
    // As the other append kernels: wait for the preceding kernel, then let the next one in.
    cudaGridDependencySynchronize();
    cudaTriggerProgrammaticLaunchCompletion();
    constexpr int EPL = D / 32;
    __shared__ uint16_t s_vec[kAppendThreads / 32][D];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int heads = Hq + 2 * Hkv;
    const long long vec = static_cast<long long>(blockIdx.x) * (kAppendThreads / 32) + warp;
    if (vec >= static_cast<long long>(B) * heads) return;
    const int b = static_cast<int>(vec / heads);
    const int hh = static_cast<int>(vec % heads);
    const bool is_q = hh < Hq;
    const bool is_v = hh >= Hq + Hkv;
    const int h = is_q ? hh : is_v ? hh - Hq - Hkv : hh - Hq;
    const uint16_t* src = (is_q ? q_in + (static_cast<size_t>(b) * Hq + h) * D
                                : (is_v ? v_new : k_new) + (static_cast<size_t>(b) * Hkv + h) * D) + lane * EPL;
    uint32_t words[EPL / 2];
    if (EPL == 4) {
        const uint2 w = *reinterpret_cast<const uint2*>(src);
        words[0] = w.x, words[EPL / 2 - 1] = w.y;
    } else {
        words[0] = *reinterpret_cast<const uint32_t*>(src);
    }
    const int p = context_lens[b];
    if (p < 0) return;
    const int page_idx = p / page_size;
    if (p >= max_position || page_idx >= max_pages_per_seq) {
        if (status_flag != nullptr && lane == 0) atomicOr(status_flag, AC_FLAG_POSITION_OOB);
        return;
    }
    int page = 0;
    if (!is_q) {
        page = block_table[static_cast<size_t>(b) * max_pages_per_seq + page_idx];
        if (page < 0 || page >= num_pages) {
            if (status_flag != nullptr && lane == 0) atomicOr(status_flag, AC_FLAG_PAGE_OOB);
            return;
        }
    }
    if (!is_v) {
        uint16_t x[EPL];
#pragma unroll
        for (int e = 0; e < EPL; ++e) x[e] = static_cast<uint16_t>(words[e / 2] >> (16 * (e & 1)));
        const float* cr = rope_cos + static_cast<size_t>(p) * (rotary_dim / 2);
        const float* sr = rope_sin + static_cast<size_t>(p) * (rotary_dim / 2);
        const uint16_t* norm_w = is_q ? q_norm_w : k_norm_w;
        if (norm_w != nullptr) rope_variant_vector<D>(x, norm_w, norm_eps, cr, sr, rotary_dim, interleaved, s_vec[warp], lane);
        else rope_vector<D>(x, cr, sr, rotary_dim, interleaved, s_vec[warp], lane);
#pragma unroll
        for (int w = 0; w < EPL / 2; ++w) words[w] = x[2 * w] | (static_cast<uint32_t>(x[2 * w + 1]) << 16);
    }
    if (is_q) {
        uint16_t* dst = q_out + (static_cast<size_t>(b) * Hq + h) * D + lane * EPL;
        if (EPL == 4) *reinterpret_cast<uint2*>(dst) = make_uint2(words[0], words[EPL / 2 - 1]);
        else *reinterpret_cast<uint32_t*>(dst) = words[0];
        return;
    }
    const int slot = p - page_idx * page_size, before = slot % cache.block;
    uint8_t* codes = (is_v ? cache.v_codes : cache.k_codes) + page * cache.stride_page + slot * cache.stride_token + h * cache.stride_head;
    float* cell = cache.scales + page * cache.stride_scales + (h * (page_size / cache.block) + slot / cache.block) * 2 + is_v;
    const uint32_t held = before > 0 ? __float_as_uint(*cell) : 0u;
    const uint32_t most = warp_amax(EPL == 4 ? bf16x2_amax(words[0], words[EPL / 2 - 1]) : words[0]);
    const uint32_t scale = settle_scale<D, FMT>(cache, cell, codes, before, held, q8_scale_bits<FMT>(most), lane);
    const float inv = q8_inverse(scale);
    if (q8_needs_clamp<FMT>(scale)) {
#pragma unroll
        for (int w = 0; w < EPL / 2; ++w) words[w] = q8_clamp(words[w]);
    }
    const uint32_t packed = q8_quantise<FMT>(words[0], words[EPL / 2 - 1], inv);
    if (EPL == 4) *reinterpret_cast<uint32_t*>(codes + lane * EPL) = packed;
    else *reinterpret_cast<uint16_t*>(codes + lane * EPL) = static_cast<uint16_t>(packed);
}

// ---- bulk store ---------------------------------------------------------------------------------------------
//
// The tokens of one call that fall into one block are a piece; its first token, the first of its row or the first of a
// block, is the piece's leader.  A CTA takes one head of the leaders among `run` consecutive tokens of the dense input (a block's
// worth: one leader, for long rows), K and V.  It has a warp for every 16 slots of a block, so that a piece stays in registers
// between the search for its largest magnitude and the rounding, and is read once.
//
// Bound: HBM, 2 bytes in and 1 out per element.  70.3 thousand tokens of 8 heads of 128, K and V (432 MB), blocks of 16: 69 us = 6260
// GB/s, 0.97 of the copy rate.  By CTAs of one warp (which leave one by one) and of four, 16 warps per SM: 74 and 80 us; 20 warps:
// 69.  Blocks of 64: 77 us (96 with one warp that reads the tokens twice).
constexpr int kHeld = 16;                                  // tokens of a warp

// The row of a token: the last one whose offset is <= token (the whole warp; the search of warp_token_position in rope_rows.cu).
__device__ __forceinline__ int find_row(const int32_t* row_offsets, int B, int token, int lane) {
    int lo = 0, n = B;
    while (n > 1) {
        const int piece = (n + 31) / 32;
        const int first = lane * piece;
        const bool below = lane > 0 && first < n && row_offsets[lo + first] <= token;
        const int k = __popc(__ballot_sync(0xffffffffu, below));
        lo += k * piece;
        n = min(piece, n - k * piece);
    }
    return lo;
}

template <int D, int FMT, bool ONE>
__global__ void __launch_bounds__(ONE ? 32 : 512, ONE ? (D == 64 ? 28 : 20) : 1) kv_store_q8_kernel(
    const uint16_t* __restrict__ k, const uint16_t* __restrict__ v, const Q8View cache, const int32_t* __restrict__ block_table,
    int max_pages_per_seq, const int32_t* __restrict__ start_pos, const int32_t* __restrict__ row_offsets, int total_tokens,
    int run, int B, int Hkv, int page_size, int num_pages, int32_t* status_flag) {
    constexpr int LPV = D / 8, TPP = 32 / LPV;             // lanes per token, tokens side by side
    constexpr int N = kHeld / TPP;                         // passes over a warp's tokens
    __shared__ uint32_t s_most[2][16];
    const int warp = ONE ? 0 : threadIdx.x >> 5, lane = threadIdx.x & 31;
    const unsigned unit = blockIdx.x / static_cast<unsigned>(Hkv);
    const int h = static_cast<int>(blockIdx.x - unit * Hkv);
    const unsigned block = cache.block;
    const long long unit_begin = static_cast<long long>(unit) * run;
    const int until = static_cast<int>(min(static_cast<long long>(total_tokens), unit_begin + run));
    const int t0 = warp * kHeld + lane / LPV, e0 = lane % LPV * 8;     // this lane's first token of a piece, and its elements
    const int64_t token_stride = static_cast<int64_t>(Hkv) * D;

    // (What follows is decided alike by every warp.)
    long long tok = unit_begin;
    while (tok < until) {
        const int row = find_row(row_offsets, B, static_cast<int>(tok), lane);
        const int begin = row_offsets[row];
        const int end = min(row_offsets[row + 1], total_tokens);
        const int start = start_pos[row];
        if (tok < begin) {                                 // tokens before the first row belong to none
            tok = begin;
            continue;
        }
        if (end <= tok) return;                            // behind the last row (or offsets that decrease, a caller's error)
        if (start < 0) {
            tok = end;
            continue;
        }
        const unsigned pos = static_cast<unsigned>(start) + static_cast<unsigned>(tok - begin);      // below 2^32
        const int before = static_cast<int>(pos % block);
        const int n = static_cast<int>(min(static_cast<long long>(block) - before, end - tok));
        if (before != 0 && tok != begin) {                 // led by a token of an earlier unit
            tok += n;
            continue;
        }
        const unsigned idx = pos / static_cast<unsigned>(page_size);
        if (idx >= static_cast<unsigned>(max_pages_per_seq)) {
            if (status_flag != nullptr && threadIdx.x == 0) atomicOr(status_flag, AC_FLAG_POSITION_OOB);
            tok += n;
            continue;
        }
        const int page = block_table[static_cast<size_t>(row) * max_pages_per_seq + idx];
        const uint16_t* src[2] = {k + tok * token_stride + h * D + e0, v + tok * token_stride + h * D + e0};
        uint4 x[2][N];
        uint32_t most[2] = {0u, 0u};
#pragma unroll
        for (int side = 0; side < 2; ++side)
#pragma unroll
            for (int i = 0; i < N; ++i)
                x[side][i] = t0 + i * TPP < n ? __ldg(reinterpret_cast<const uint4*>(src[side] + (t0 + i * TPP) * token_stride))
                                              : make_uint4(0u, 0u, 0u, 0u);
        tok += n;
        if (page < 0 || page >= num_pages) {
            if (status_flag != nullptr && threadIdx.x == 0) atomicOr(status_flag, AC_FLAG_PAGE_OOB);
            continue;
        }
        const int slot = static_cast<int>(pos - idx * page_size);
        const int64_t place = page * cache.stride_page + slot * cache.stride_token + h * cache.stride_head;
        float* cell = cache.scales + page * cache.stride_scales + (h * (page_size / cache.block) + slot / cache.block) * 2;
        float2 held = make_float2(0.0f, 0.0f);
        if (before > 0) held = *reinterpret_cast<const float2*>(cell);
#pragma unroll
        for (int side = 0; side < 2; ++side) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                most[side] = bf16x2_amax(bf16x2_amax(most[side], bf16x2_amax(x[side][i].x, x[side][i].y)), bf16x2_amax(x[side][i].z, x[side][i].w));
            most[side] = warp_amax(most[side]);
        }
        if (!ONE) {
            if (lane == 0) s_most[0][warp] = most[0], s_most[1][warp] = most[1];
            __syncthreads();                               // every warp has read the held scales, too
            for (int w = 0; w < static_cast<int>(blockDim.x) / 32; ++w)
                most[0] = max(most[0], s_most[0][w]), most[1] = max(most[1], s_most[1][w]);
            __syncthreads();                               // before the next piece's
        }
        bool clamp = false;
        float inv[2];
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            const uint32_t need = q8_scale_bits<FMT>(most[side]), was = __float_as_uint(side ? held.y : held.x);
            uint32_t scale = before > 0 ? q8_join(was, need) : need;
            if (warp == 0)
                settle_scale<D, FMT>(cache, cell + side, (side ? cache.v_codes : cache.k_codes) + place, before, was, need, lane);
            inv[side] = q8_inverse(scale);
            clamp = clamp || q8_needs_clamp<FMT>(scale);
        }
        if (FMT == Q8_INT8 && clamp) {                     // (values of the other side are below the bound)
#pragma unroll
            for (int side = 0; side < 2; ++side)
#pragma unroll
                for (int i = 0; i < N; ++i)
                    x[side][i] = make_uint4(q8_clamp(x[side][i].x), q8_clamp(x[side][i].y), q8_clamp(x[side][i].z), q8_clamp(x[side][i].w));
        }
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            uint8_t* dst = (side ? cache.v_codes : cache.k_codes) + place + e0;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int at = t0 + i * TPP;
                const uint4 w = x[side][i];
                if (at < n)
                    *reinterpret_cast<uint2*>(dst + at * cache.stride_token) =
                        make_uint2(q8_quantise<FMT>(w.x, w.y, inv[side]), q8_quantise<FMT>(w.z, w.w, inv[side]));
            }
        }
    }
}

// ---- bulk load ----------------------------------------------------------------------------------------------
//
// A warp takes a run of consecutive tokens: its lanes find the slots of one token each, then it goes through the run's (token,
// head) vectors, K and V together, eight codes (8 bytes in, 16 out) per lane, four vectors of both in hand.
//
// Bound: HBM, 1 byte in and 2 out per element.  70.3 thousand tokens of 8 heads of 128, K and V (432 MB): 74 us = 5840 GB/s, 0.90 of
// the copy rate (32 heads: 0.99).  Persistent warps that take several runs each: 80.  Runs of 32 vectors against 16 and 64: 74,
// 75 and 77; two vectors in hand: 96.
constexpr int kLoadThreads = 64;

struct Q8Slot {
    int64_t code;         // byte offset of the token's slot in the code pools; -1: no slot
    int64_t scale;        // offset of head 0's scale of K
};

__device__ __forceinline__ Q8Slot find_slot(long long token, const Q8View& cache, const int32_t* block_table,
                                            int max_pages_per_seq, const int32_t* start_pos, const int32_t* row_offsets,
                                            int B, int page_size, int num_pages, int32_t* status_flag) {
    Q8Slot r{-1, 0};
    if (token >= row_offsets[B]) return r;
    int lo = 0, hi = B;                                    // the last row whose offset is <= token
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (row_offsets[mid] <= token) lo = mid; else hi = mid;
    }
    const int start = start_pos[lo];
    if (start < 0 || token < row_offsets[lo]) return r;
    const unsigned pos = static_cast<unsigned>(start) + static_cast<unsigned>(token - row_offsets[lo]);      // below 2^32
    const unsigned idx = pos / static_cast<unsigned>(page_size);
    if (idx >= static_cast<unsigned>(max_pages_per_seq)) {
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
    r.scale = page * cache.stride_scales + slot / cache.block * 2;
    return r;
}

template <int FMT>
__device__ __forceinline__ uint4 q8_values(uint2 codes, float s) {
    float a[4], b[4];
    q8_floats<FMT>(codes.x, a);
    q8_floats<FMT>(codes.y, b);
    return make_uint4(pack_bf16x2(a[0] * s, a[1] * s), pack_bf16x2(a[2] * s, a[3] * s), pack_bf16x2(b[0] * s, b[1] * s),
                      pack_bf16x2(b[2] * s, b[3] * s));
}

template <int D, int FMT>
__global__ void __launch_bounds__(kLoadThreads) kv_load_q8_kernel(
    uint16_t* __restrict__ k, uint16_t* __restrict__ v, const Q8View cache, const int32_t* __restrict__ block_table,
    int max_pages_per_seq, const int32_t* __restrict__ start_pos, const int32_t* __restrict__ row_offsets, int total_tokens,
    int run, int B, int Hkv, int page_size, int num_pages, int32_t* status_flag) {
    constexpr int LPV = D / 8, VECS = 32 / LPV, U = 4;
    constexpr int WARPS = kLoadThreads / 32;
    __shared__ Q8Slot s_slots[WARPS][32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    Q8Slot* const s_slot = s_slots[warp];
    const int e0 = lane % LPV * 8;
    const int head_scales = page_size / cache.block * 2;
    const long long first = (static_cast<long long>(blockIdx.x) * WARPS + warp) * run;
    if (first >= total_tokens) return;
    {
        const int tokens = total_tokens - first < run ? static_cast<int>(total_tokens - first) : run;
        const int vecs = tokens * Hkv;
        if (lane < tokens)
            s_slot[lane] = find_slot(first + lane, cache, block_table, max_pages_per_seq, start_pos, row_offsets, B, page_size, num_pages, status_flag);
        __syncwarp();
        for (int i = lane / LPV; i < vecs; i += U * VECS) {
            uint2 codes[2][U];
            float2 s[U];
            bool live[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int vec = i + u * VECS;
                const int t = vec / Hkv, h = vec - t * Hkv;
                live[u] = false;
                if (vec >= vecs) continue;
                const Q8Slot at = s_slot[t];
                live[u] = at.code >= 0;
                if (!live[u]) continue;
                const int64_t place = at.code + h * cache.stride_head + e0;
                codes[0][u] = __ldcs(reinterpret_cast<const uint2*>(cache.k_codes + place));
                codes[1][u] = __ldcs(reinterpret_cast<const uint2*>(cache.v_codes + place));
                s[u] = *reinterpret_cast<const float2*>(cache.scales + at.scale + h * head_scales);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int vec = i + u * VECS;
                if (vec >= vecs) continue;
                const int64_t to = (first * Hkv + vec) * D + e0;
                const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
                __stcs(reinterpret_cast<uint4*>(k + to), live[u] ? q8_values<FMT>(codes[0][u], s[u].x) : zero);
                __stcs(reinterpret_cast<uint4*>(v + to), live[u] ? q8_values<FMT>(codes[1][u], s[u].y) : zero);
            }
        }
    }
}

template <int D, int FMT>
cudaError_t launch_store(const void* k, const void* v, const Q8View& cache, const int32_t* block_table, int max_pages_per_seq,
                         const int32_t* start_pos, const int32_t* row_offsets, int total_tokens, int B, int Hkv, int page_size,
                         int num_pages, int32_t* status_flag, int sms, cudaStream_t stream) {
    // An ordinary launch: what follows it in the stream may read the cache before its own synchronisation, which is safe only
    // behind kernels that do not signal early.
    // Leaders are looked for among `block` tokens, fewer where that leaves warps (32 per SM) without work.
    int run = cache.block;
    while (run > 1 && (total_tokens - 1ll) / run * Hkv < 32ll * sms) run = (run + 1) / 2;
    const long long grid = ((total_tokens - 1ll) / run + 1) * Hkv;
    if (grid > 0x7fffffffll) return cudaErrorInvalidConfiguration;
    const uint16_t* kk = static_cast<const uint16_t*>(k);
    const uint16_t* vv = static_cast<const uint16_t*>(v);
    if (cache.block == kHeld)
        kv_store_q8_kernel<D, FMT, true><<<static_cast<unsigned>(grid), 32, 0, stream>>>(
            kk, vv, cache, block_table, max_pages_per_seq, start_pos, row_offsets, total_tokens, run, B, Hkv, page_size, num_pages, status_flag);
    else
        kv_store_q8_kernel<D, FMT, false><<<static_cast<unsigned>(grid), cache.block / kHeld * 32, 0, stream>>>(
            kk, vv, cache, block_table, max_pages_per_seq, start_pos, row_offsets, total_tokens, run, B, Hkv, page_size, num_pages, status_flag);
    return cudaGetLastError();
}

template <int D, int FMT>
cudaError_t launch_load(void* k, void* v, const Q8View& cache, const int32_t* block_table, int max_pages_per_seq,
                        const int32_t* start_pos, const int32_t* row_offsets, int total_tokens, int B, int Hkv, int page_size,
                        int num_pages, int32_t* status_flag, int sms, cudaStream_t stream) {
    int run = Hkv < 32 ? 32 / Hkv : 1;
    while (run > 1 && total_tokens / run < 32 * sms && run / 2 * Hkv >= 8) run /= 2;
    const long long grid = ((total_tokens - 1ll) / run) / (kLoadThreads / 32) + 1;
    if (grid > 0x7fffffffll) return cudaErrorInvalidConfiguration;
    kv_load_q8_kernel<D, FMT><<<static_cast<unsigned>(grid), kLoadThreads, 0, stream>>>(
        static_cast<uint16_t*>(k), static_cast<uint16_t*>(v), cache, block_table, max_pages_per_seq, start_pos, row_offsets,
        total_tokens, run, B, Hkv, page_size, num_pages, status_flag);
    return cudaGetLastError();
}

}  // namespace

#define AC_Q8_DISPATCH(CALL)                                                                       \
    (d == 128 ? (cache.format == Q8_INT8 ? CALL(128, Q8_INT8) : CALL(128, Q8_E4M3))                \
              : (cache.format == Q8_INT8 ? CALL(64, Q8_INT8) : CALL(64, Q8_E4M3)))

cudaError_t launch_rope_kv_append_q8(const void* q_in, void* q_out, const void* k_new, const void* v_new,
                                     const Q8View& cache, const int32_t* block_table, int max_pages_per_seq,
                                     const int32_t* context_lens, const float* rope_cos, const float* rope_sin,
                                     int max_position, int B, int Hq, int Hkv, int d, int page_size, int num_pages,
                                     int32_t* status_flag, const RopeVariant* variant, cudaStream_t stream) {
    const RopeVariant plain{d, 0, nullptr, nullptr, 0.0f};
    const RopeVariant& r = variant != nullptr ? *variant : plain;
    const long long vecs = static_cast<long long>(B) * (Hq + 2ll * Hkv);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>((vecs + kAppendThreads / 32 - 1) / (kAppendThreads / 32)));
    cfg.blockDim = dim3(kAppendThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
#define AC_Q8_APPEND(D_, F_)                                                                                       \
    cudaLaunchKernelEx(&cfg, rope_kv_append_q8_kernel<D_, F_>, static_cast<const uint16_t*>(q_in),                  \
                       static_cast<uint16_t*>(q_out), static_cast<const uint16_t*>(k_new),                          \
                       static_cast<const uint16_t*>(v_new), cache, block_table, max_pages_per_seq, context_lens,    \
                       rope_cos, rope_sin, max_position, B, Hq, Hkv, page_size, num_pages, status_flag,             \
                       r.rotary_dim, r.interleaved, static_cast<const uint16_t*>(r.q_norm_weight),                  \
                       static_cast<const uint16_t*>(r.k_norm_weight), r.norm_eps)
    return AC_Q8_DISPATCH(AC_Q8_APPEND);
#undef AC_Q8_APPEND
}

cudaError_t launch_kv_bulk_q8(void* k, void* v, const Q8View& cache, const int32_t* block_table, int max_pages_per_seq,
                              const int32_t* start_pos, const int32_t* row_offsets, int total_tokens, int B, int Hkv, int d,
                              int page_size, int num_pages, int32_t* status_flag, bool store, int sms, cudaStream_t stream) {
#define AC_Q8_STORE(D_, F_)                                                                                         \
    launch_store<D_, F_>(k, v, cache, block_table, max_pages_per_seq, start_pos, row_offsets, total_tokens, B, Hkv,  \
                         page_size, num_pages, status_flag, sms, stream)
#define AC_Q8_LOAD(D_, F_)                                                                                          \
    launch_load<D_, F_>(k, v, cache, block_table, max_pages_per_seq, start_pos, row_offsets, total_tokens, B, Hkv,   \
                        page_size, num_pages, status_flag, sms, stream)
    return store ? AC_Q8_DISPATCH(AC_Q8_STORE) : AC_Q8_DISPATCH(AC_Q8_LOAD);
#undef AC_Q8_STORE
#undef AC_Q8_LOAD
}

}  // namespace ac
