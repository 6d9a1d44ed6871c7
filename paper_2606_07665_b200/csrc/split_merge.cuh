// Merge of split-KV partial results inside an attention kernel, shared by the bf16 and the 4-bit kernel.
#pragma once

#include <math.h>

#include "ac_device.cuh"

namespace acdev {

// The merge of the ticket path: the CTA that arrived last combines the splits' partial results of its
// (request, KV head) out of the workspace.  An item is four consecutive output elements of one query
// row; a thread owns ITEMS of them (item = thread + k * THREADS) and walks the splits in groups of GS
// for all its items at once: the ITEMS * GS 16-byte partial loads and their log-sum-exps are issued
// before any is used, so a group costs one L2 round trip whatever the number of items, and groups are
// combined with the same running-maximum rescaling as the main loop.  ITEMS * GS <= 16 keeps the
// loads in registers.  Params is the parameter block of the attention kernel that calls it (partial_o,
// partial_lse, out, out_mirror).
template <int D, int THREADS, int ITEMS, int GS, class Params>
__device__ __forceinline__ void merge_splits_from_workspace(const Params& p, size_t hq0, int items, int S,
                                                            int n_active) {
    constexpr int D4 = D / 4;
    static_assert(ITEMS * GS <= 16, "loads of a group stay in registers");
    const float* lse_g[ITEMS];
    const float4* po[ITEMS];
    bool live[ITEMS];
    float M[ITEMS], den[ITEMS];
    float4 acc[ITEMS];
    size_t out_at[ITEMS];
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
        const int e = threadIdx.x + k * THREADS;
        live[k] = e < items;
        const int row = live[k] ? e / D4 : 0;
        const int c4 = live[k] ? e - row * D4 : 0;
        lse_g[k] = p.partial_lse + (hq0 + row) * S;
        po[k] = reinterpret_cast<const float4*>(p.partial_o + (hq0 + row) * S * D) + c4;
        out_at[k] = (hq0 + row) * D + c4 * 4;
        M[k] = -INFINITY;
        den[k] = 0.0f;
        acc[k] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    for (int s0 = 0; s0 < n_active; s0 += GS) {
        float4 v[ITEMS][GS];
        float l[ITEMS][GS];
#pragma unroll
        for (int k = 0; k < ITEMS; ++k)
#pragma unroll
            for (int u = 0; u < GS; ++u) {
                const bool on = live[k] && s0 + u < n_active;
                l[k][u] = on ? __ldcg(lse_g[k] + s0 + u) : -INFINITY;
                v[k][u] = on ? __ldcg(po[k] + static_cast<size_t>(s0 + u) * D4) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            float gm = M[k];
#pragma unroll
            for (int u = 0; u < GS; ++u) gm = fmaxf(gm, l[k][u]);
            const float rescale = __expf(M[k] - gm);           // 0 on the first group (M = -inf)
            acc[k].x *= rescale;
            acc[k].y *= rescale;
            acc[k].z *= rescale;
            acc[k].w *= rescale;
            den[k] *= rescale;
            M[k] = gm;
#pragma unroll
            for (int u = 0; u < GS; ++u) {
                const float wgt = __expf(l[k][u] - gm);        // 0 for the padding entries
                acc[k].x = fmaf(wgt, v[k][u].x, acc[k].x);
                acc[k].y = fmaf(wgt, v[k][u].y, acc[k].y);
                acc[k].z = fmaf(wgt, v[k][u].z, acc[k].z);
                acc[k].w = fmaf(wgt, v[k][u].w, acc[k].w);
                den[k] += wgt;
            }
        }
    }
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
        if (!live[k]) continue;
        const float inv = 1.0f / den[k];
        const uint2 bits = make_uint2(pack_bf16x2(acc[k].x * inv, acc[k].y * inv),
                                      pack_bf16x2(acc[k].z * inv, acc[k].w * inv));
        *reinterpret_cast<uint2*>(p.out + out_at[k]) = bits;
        if (p.out_mirror != nullptr) *reinterpret_cast<uint2*>(p.out_mirror + out_at[k]) = bits;
    }
}

}  // namespace acdev
