// Page bookkeeping and page copies: reserve, fork, release, trim, compact, copy.
//
// The bookkeeping kernels hand out free pages lowest index first.  For reserve and fork a single CTA walks the reference
// counts in order, 16 pages per thread and step, and turns the free ones into ranks by a scan over the CTA; it stops as
// soon as it has what the call needs.  Compaction needs every live page's rank: CTAs count and rank a chunk of the
// counts each, in two launches.  Bound: latency (a few dependent passes over num_pages * 4 bytes that sit in L2): 8 forks
// with their copies and the release of the children 7.9 us, one page for each of 64 rows 8.0, trim 3.2, the compaction of
// a pool of 512 pages 6.5.  The one CTA's walk grows with what lies in front of the free pages: 36000 live ones make that reserve
// 11.7 us and those forks 13.4.  The copies are bound by HBM, which reads and writes: a warp moves pieces of up to 4 KB, 16
// bytes a lane, eight loads in flight before the first store; a compaction that moves 0.65 GB (1.3 GB read and written) takes
// 222 us = 5870 GB/s, 0.90 of the measured 6546, one of 96 pools (0.79 GB read and written, 300 rows) 127 us.
#include "ac_device.cuh"
#include "ac_internal.h"

namespace ac {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPagesPerThread = 16;
constexpr int kStep = kPlanThreads * kPagesPerThread;
constexpr int kCopyThreads = 256;
constexpr int kPiece = 4096;                  // bytes a warp moves at a time

// Exclusive prefix sum over the THREADS threads of the CTA; *total is the sum.  Every thread calls it.
template <int THREADS = kPlanThreads, class T>
__device__ __forceinline__ T block_scan(T v, T* total) {
    constexpr int WARPS = THREADS / 32;
    static_assert(WARPS <= 32, "one warp scans the warps' sums");
    __shared__ T s_warp[WARPS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    T x = v;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const T y = __shfl_up_sync(0xffffffffu, x, off);
        if (lane >= off) x += y;
    }
    if (lane == 31) s_warp[warp] = x;
    __syncthreads();
    T w = lane < WARPS ? s_warp[lane] : T(0);
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const T y = __shfl_up_sync(0xffffffffu, w, off);
        if (lane >= off) w += y;
    }
    *total = __shfl_sync(0xffffffffu, w, 31);
    const T before = warp > 0 ? __shfl_sync(0xffffffffu, w, warp - 1) : 0;
    __syncthreads();                           // s_warp may be written again
    return before + x - v;
}

// Bit i of the result: page base + i exists and is free.
__device__ __forceinline__ uint32_t free_bits(const int32_t* refs, int base, int num_pages) {
    uint32_t bits = 0;
    if (base + kPagesPerThread <= num_pages) {
        const int4* src = reinterpret_cast<const int4*>(refs + base);
        int4 v[kPagesPerThread / 4];
#pragma unroll
        for (int i = 0; i < kPagesPerThread / 4; ++i) v[i] = src[i];
#pragma unroll
        for (int i = 0; i < kPagesPerThread / 4; ++i)
            bits |= ((v[i].x == 0 ? 1u : 0u) | (v[i].y == 0 ? 2u : 0u) | (v[i].z == 0 ? 4u : 0u) |
                     (v[i].w == 0 ? 8u : 0u)) << (4 * i);
    } else {
        for (int i = 0; i < kPagesPerThread; ++i)
            if (base + i < num_pages && refs[base + i] == 0) bits |= 1u << i;
    }
    return bits;
}

// Writes the `need` lowest free pages to list, in order; returns how many there are (at most need).
__device__ int find_free(const int32_t* refs, int num_pages, int need, int32_t* list) {
    int found = 0;
    for (int at = 0; at < num_pages && found < need; at += kStep) {
        const int base = at + threadIdx.x * kPagesPerThread;
        uint32_t bits = base < num_pages ? free_bits(refs, base, num_pages) : 0u;
        int total;
        int rank = found + block_scan(__popc(bits), &total);
        while (bits != 0 && rank < need) {
            list[rank++] = base + __ffs(bits) - 1;
            bits &= bits - 1;
        }
        found += total;
    }
    __syncthreads();                           // the list is visible to the whole CTA
    return found < need ? found : need;
}

__device__ __forceinline__ void raise(int32_t* status_flag, int bit) {
    if (status_flag != nullptr) atomicOr(status_flag, bit);
}

// Pages that n tokens take.
__device__ __forceinline__ int pages_for(long long n, int page_size) {
    return static_cast<int>((n + page_size - 1) / page_size);
}

// ---- reserve ---------------------------------------------------------------------------------------------

__global__ void __launch_bounds__(kPlanThreads) reserve_kernel(int32_t* block_table, int max_pages_per_seq,
                                                               const int32_t* context_lens, int32_t* refs,
                                                               int new_tokens, int rows, int page_size, int num_pages,
                                                               int32_t* offsets, int32_t* list, int32_t* status_flag) {
    auto pages_of = [&](int r, int& first) {   // pages row r needs, and its first new table index
        const int n = context_lens[r];
        first = 0;
        if (n < 0) return 0;
        first = pages_for(n, page_size);
        const int last = pages_for(static_cast<long long>(n) + new_tokens, page_size);
        return last > max_pages_per_seq ? -1 : last - first;
    };
    long long need = 0;
    for (int at = 0; at < rows; at += kPlanThreads) {
        const int r = at + threadIdx.x;
        int first;
        long long mine = r < rows ? pages_of(r, first) : 0, total;
        if (mine < 0) {
            raise(status_flag, AC_FLAG_POSITION_OOB);
            mine = 0;
        }
        const long long o = need + block_scan(mine, &total);
        if (r < rows) {
            offsets[r] = o > num_pages ? num_pages + 1 : static_cast<int>(o);
        }
        need += total;
    }
    const int want = need > num_pages ? num_pages : static_cast<int>(need);
    const int found = find_free(refs, num_pages, want, list);
    if (need > found && threadIdx.x == 0) raise(status_flag, AC_FLAG_POOL_EXHAUSTED);
    const int lane = threadIdx.x & 31;
    for (int r = threadIdx.x >> 5; r < rows; r += kPlanThreads / 32) {
        int first;
        const int mine = pages_of(r, first);
        const long long off = offsets[r];
        if (mine <= 0 || off + mine > found) continue;
        for (int i = lane; i < mine; i += 32) {
            const int page = list[off + i];
            block_table[static_cast<size_t>(r) * max_pages_per_seq + first + i] = page;
            refs[page] = 1;
        }
    }
}

// ---- page copies -----------------------------------------------------------------------------------------

// The pools as a kernel argument, in two sizes: 3 KB of arguments cost a small launch about half a microsecond.
constexpr int kFewPools = 8;
template <int N>
struct PoolArgs {
    ac_page_pool pool[N];
};

// A warp copies bytes [lo, hi) of a piece (hi - lo <= kPiece, lo a multiple of 16, addresses 16-byte aligned).
__device__ __forceinline__ void copy_piece(char* dst, const char* src, int64_t lo, int64_t hi, int lane) {
    constexpr int N = kPiece / 512;
    const int bytes = static_cast<int>(hi - lo);
    const uint4* s = reinterpret_cast<const uint4*>(src + lo);
    uint4* d = reinterpret_cast<uint4*>(dst + lo);
    const int whole = bytes / 16;
    uint4 v[N];
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i * 32 + lane < whole) v[i] = __ldcs(s + i * 32 + lane);
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i * 32 + lane < whole) __stcs(d + i * 32 + lane, v[i]);
    const int tail = whole * 16 + lane;
    if (tail < bytes) dst[lo + tail] = src[lo + tail];
}

// Jobs (source, destination) with, where lens != nullptr, the length of the sequence whose last page is copied: of that only
// the filled slots.  blockIdx.y is the pool; the warps of its CTAs take (job, segment, piece) units in turn.
__device__ __forceinline__ void run_copies(const ac_page_pool& pool, const int2* jobs, const int32_t* lens, int n,
                                           int page_size, int num_pages, int32_t* status_flag) {
    const int lane = threadIdx.x & 31;
    const bool slots = lens != nullptr && pool.segments != AC_PAGE_WHOLE;
    const int segments = slots ? pool.segments : 1;
    const int64_t seg_bytes = pool.page_bytes / segments;
    const int pieces = static_cast<int>((seg_bytes + kPiece - 1) / kPiece);
    const long long per_job = static_cast<long long>(segments) * pieces;
    const long long units = per_job * n;
    const long long step = static_cast<long long>(gridDim.x) * (kCopyThreads / 32);
    for (long long u = static_cast<long long>(blockIdx.x) * (kCopyThreads / 32) + (threadIdx.x >> 5); u < units;
         u += step) {
        const int job = static_cast<int>(u / per_job);
        const int rest = static_cast<int>(u - job * per_job);
        const int seg = rest / pieces, piece = rest - seg * pieces;
        const int2 j = jobs[job];
        if (j.x < 0 || j.y < 0 || j.x >= num_pages || j.y >= num_pages) {
            if (lens == nullptr && lane == 0) raise(status_flag, AC_FLAG_PAGE_OOB);
            continue;
        }
        if (j.x == j.y) continue;
        const int64_t end = slots ? seg_bytes / page_size * (lens[job] % page_size) : seg_bytes;
        const int64_t lo = static_cast<int64_t>(piece) * kPiece;
        const int64_t hi = min(end, lo + kPiece);
        if (lo >= hi) continue;
        char* base = static_cast<char*>(pool.base) + seg * seg_bytes;
        copy_piece(base + j.y * pool.page_bytes, base + j.x * pool.page_bytes, lo, hi, lane);
    }
}

template <int N>
__global__ void __launch_bounds__(kCopyThreads) copy_pages_kernel(const __grid_constant__ PoolArgs<N> pools,
                                                                  const int2* pairs, int n, int num_pages,
                                                                  int32_t* status_flag) {
    run_copies(pools.pool[blockIdx.y], pairs, nullptr, n, 1, num_pages, status_flag);
}

// ---- fork ------------------------------------------------------------------------------------------------

// Gives every fork that needs a page its page; jobs[i] = (parent's last page, child's page), or (-1, -1) where nothing is
// copied, and lens[i] = the parent's length, or -1 for a fork that does not take place.  What follows goes by this length,
// which was checked against the table here: the parent's own may change meanwhile (a row that is a child of the call too).
__global__ void __launch_bounds__(kPlanThreads) fork_plan_kernel(const int32_t* block_table, int max_pages_per_seq,
                                                                 const int32_t* context_lens, const int32_t* refs,
                                                                 const int2* pairs, int n, int rows, int page_size,
                                                                 int num_pages, int2* jobs, int32_t* lens,
                                                                 int32_t* list, int32_t* status_flag) {
    cudaTriggerProgrammaticLaunchCompletion();             // the next kernel waits for this one before it reads
    int need = 0;
    for (int at = 0; at < n; at += kPlanThreads) {
        const int i = at + threadIdx.x;
        int part = 0, src = -1, state = -1;
        if (i < n) {
            const int2 pc = pairs[i];
            if (pc.x < 0 || pc.x >= rows || pc.y < 0 || pc.y >= rows) {
                raise(status_flag, AC_FLAG_ROW_OOB);
            } else {
                const int len = context_lens[pc.x];
                if (len >= 0 && pages_for(len, page_size) > max_pages_per_seq) {
                    raise(status_flag, AC_FLAG_POSITION_OOB);
                } else if (len >= 0) {
                    part = len % page_size;
                    state = len;
                    if (part > 0) src = block_table[static_cast<size_t>(pc.x) * max_pages_per_seq + len / page_size];
                }
            }
        }
        int total;
        const int rank = need + block_scan(part > 0 ? 1 : 0, &total);
        if (i < n) {
            lens[i] = state;
            jobs[i] = make_int2(src, part > 0 ? rank : -1);      // the rank, until the pages are known
        }
        need += total;
    }
    const int found = find_free(refs, num_pages, min(need, num_pages), list);
    if (need > found && threadIdx.x == 0) raise(status_flag, AC_FLAG_POOL_EXHAUSTED);
    for (int i = threadIdx.x; i < n; i += kPlanThreads) {
        const int2 j = jobs[i];
        if (j.y < 0) continue;                                   // no page needed
        if (j.y >= found) {
            lens[i] = -1;
            jobs[i] = make_int2(-1, -1);
        } else {
            jobs[i].y = list[j.y];
        }
    }
}

// grid.y = 0: the tables, one CTA per fork in turn; grid.y >= 1: the copies in pool grid.y - 1.
template <int N>
__global__ void __launch_bounds__(kCopyThreads) fork_apply_kernel(const __grid_constant__ PoolArgs<N> pools,
                                                                  int32_t* block_table, int max_pages_per_seq,
                                                                  int32_t* context_lens, int32_t* refs,
                                                                  const int2* pairs, const int2* jobs,
                                                                  const int32_t* lens, int n, int rows, int page_size,
                                                                  int num_pages, int32_t* status_flag) {
    cudaGridDependencySynchronize();           // no early signal: what follows may read the tables before its own wait
    if (blockIdx.y > 0) {
        run_copies(pools.pool[blockIdx.y - 1], jobs, lens, n, page_size, num_pages, nullptr);
        return;
    }
    for (int i = blockIdx.x; i < n; i += gridDim.x) {
        const int2 pc = pairs[i];
        if (pc.x < 0 || pc.x >= rows || pc.y < 0 || pc.y >= rows) continue;
        const int len = lens[i];
        if (len < 0) {
            if (threadIdx.x == 0) context_lens[pc.y] = -1;
            continue;
        }
        const int full = len / page_size, part = len - full * page_size;
        const int32_t* from = block_table + static_cast<size_t>(pc.x) * max_pages_per_seq;
        int32_t* to = block_table + static_cast<size_t>(pc.y) * max_pages_per_seq;
        for (int k = threadIdx.x; k < full; k += kCopyThreads) {
            const int page = from[k];
            to[k] = page;
            if (page < 0 || page >= num_pages) raise(status_flag, AC_FLAG_PAGE_OOB);
            else atomicAdd(refs + page, 1);
        }
        if (threadIdx.x == 0) {
            if (part > 0) {
                const int2 j = jobs[i];
                to[full] = j.y;
                refs[j.y] = 1;
                if (j.x < 0 || j.x >= num_pages) raise(status_flag, AC_FLAG_PAGE_OOB);
            }
            context_lens[pc.y] = len;
        }
    }
}

// ---- release ---------------------------------------------------------------------------------------------

__global__ void __launch_bounds__(kCopyThreads) release_kernel(const int32_t* block_table, int max_pages_per_seq,
                                                               int32_t* context_lens, int32_t* refs,
                                                               const int32_t* row_list, int rows, int page_size,
                                                               int num_pages, int32_t* status_flag) {
    __shared__ int s_len;
    const int row = row_list[blockIdx.x];
    if (row < 0 || row >= rows) {
        if (threadIdx.x == 0) raise(status_flag, AC_FLAG_ROW_OOB);
        return;
    }
    if (threadIdx.x == 0) s_len = atomicExch(context_lens + row, -1);    // a row listed twice is dropped once
    __syncthreads();
    const int len = s_len;
    if (len <= 0) return;
    int pages = pages_for(len, page_size);
    if (pages > max_pages_per_seq) {
        if (threadIdx.x == 0) raise(status_flag, AC_FLAG_POSITION_OOB);
        pages = max_pages_per_seq;
    }
    for (int k = threadIdx.x; k < pages; k += kCopyThreads) {
        const int page = block_table[static_cast<size_t>(row) * max_pages_per_seq + k];
        if (page < 0 || page >= num_pages) {
            raise(status_flag, AC_FLAG_PAGE_OOB);
        } else if (atomicSub(refs + page, 1) <= 0) {
            atomicAdd(refs + page, 1);
            raise(status_flag, AC_FLAG_REF_COUNT);
        }
    }
}

// ---- trim ------------------------------------------------------------------------------------------------

// One CTA per row adds the row's pages to counts that were cleared before.
__global__ void __launch_bounds__(kCopyThreads) count_held_kernel(const int32_t* block_table, int max_pages_per_seq,
                                                                  const int32_t* context_lens, int32_t* refs,
                                                                  int page_size, int num_pages, int32_t* status_flag) {
    const int len = context_lens[blockIdx.x];
    if (len <= 0) return;
    int pages = pages_for(len, page_size);
    if (pages > max_pages_per_seq) {
        if (threadIdx.x == 0) raise(status_flag, AC_FLAG_POSITION_OOB);
        pages = max_pages_per_seq;
    }
    for (int k = threadIdx.x; k < pages; k += kCopyThreads) {
        const int page = block_table[static_cast<size_t>(blockIdx.x) * max_pages_per_seq + k];
        if (page < 0 || page >= num_pages) raise(status_flag, AC_FLAG_PAGE_OOB);
        else atomicAdd(refs + page, 1);
    }
}

// ---- compact ---------------------------------------------------------------------------------------------

// Ranks without a scan over the whole pool in one CTA: chunks of kChunk pages are counted, and each chunk's CTA then adds up
// the counts it needs.  (One CTA that walked 40000 pages took 35 us; these two take 6.)
constexpr int kChunkThreads = 256;
constexpr int kChunk = kChunkThreads * kPagesPerThread;

__global__ void __launch_bounds__(kChunkThreads) compact_count_kernel(const int32_t* refs, int num_pages, int32_t* counts) {
    cudaTriggerProgrammaticLaunchCompletion();             // the next kernel waits for this one before it reads
    const int base = blockIdx.x * kChunk + threadIdx.x * kPagesPerThread;
    int live = 0, total;
    if (base < num_pages) live = min(kPagesPerThread, num_pages - base) - __popc(free_bits(refs, base, num_pages));
    block_scan<kChunkThreads>(live, &total);
    if (threadIdx.x == 0) counts[blockIdx.x] = total;
}

// head[0] = moves, head[1] = live pages; moves[k] = (from, to): the k-th live page from id `live` on and the k-th hole
// below; place[p] for p >= live: its k, or -1 where it is free.
__global__ void __launch_bounds__(kChunkThreads) compact_rank_kernel(const int32_t* refs, int num_pages,
                                                                     const int32_t* counts, int32_t* head, int2* moves,
                                                                     int32_t* place, int32_t* live_out) {
    cudaGridDependencySynchronize();
    cudaTriggerProgrammaticLaunchCompletion();             // the next kernel waits for this one before it reads
    const int chunks = gridDim.x, base = blockIdx.x * kChunk + threadIdx.x * kPagesPerThread;
    const uint32_t exist = base >= num_pages ? 0u : num_pages - base >= kPagesPerThread ? 0xffffu : (1u << (num_pages - base)) - 1u;
    const uint32_t open = base < num_pages ? free_bits(refs, base, num_pages) : 0u;
    int mine, live;
    const int inside = block_scan<kChunkThreads>(__popc(exist & ~open), &mine);
    int before = 0;                                        // live pages in the chunks before this one
    if (chunks == 1) {
        live = mine;
    } else {
        int all = 0, ahead = 0;
        for (int c = threadIdx.x; c < chunks; c += kChunkThreads) {
            const int n = counts[c];
            all += n;
            if (c < static_cast<int>(blockIdx.x)) ahead += n;
        }
        block_scan<kChunkThreads>(all, &live);
        block_scan<kChunkThreads>(ahead, &before);
    }
    // live pages below id `live`
    int below_live = 0, part = 0;
    const int edge = live / kChunk;                        // the chunk that holds that border
    for (int c = threadIdx.x; c < edge; c += kChunkThreads) part += chunks == 1 ? mine : counts[c];
    const int edge_base = edge * kChunk + threadIdx.x * kPagesPerThread;
    if (edge_base < live) {
        const int n = min(kPagesPerThread, live - edge_base);
        part += __popc(~free_bits(refs, edge_base, num_pages) & ((1u << n) - 1u));
    }
    block_scan<kChunkThreads>(part, &below_live);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        head[0] = live - below_live;
        head[1] = live;
        if (live_out != nullptr) *live_out = live;
    }
    int rank = before + inside;                            // live pages before this thread's
#pragma unroll
    for (int i = 0; i < kPagesPerThread; ++i) {
        if (!((exist >> i) & 1u)) break;
        const int page = base + i;
        const bool is_free = (open >> i) & 1u;
        if (page < live) {
            if (is_free) moves[page - rank].y = page;
        } else {
            place[page] = is_free ? -1 : rank - below_live;
            if (!is_free) moves[rank - below_live].x = page;
        }
        rank += is_free ? 0 : 1;
    }
}

// grid.y = 0: block table and reference counts; grid.y >= 1: the moves in pool grid.y - 1.
template <int N>
__global__ void __launch_bounds__(kCopyThreads) compact_apply_kernel(const __grid_constant__ PoolArgs<N> pools,
                                                                     const int32_t* block_table, int32_t* table_out,
                                                                     int max_pages_per_seq, const int32_t* context_lens,
                                                                     const int32_t* refs, int32_t* refs_out, int rows,
                                                                     int page_size, int num_pages, const int32_t* head,
                                                                     const int2* moves, const int32_t* place,
                                                                     int32_t* status_flag) {
    cudaGridDependencySynchronize();           // no early signal: what follows may read the tables before its own wait
    const int n = head[0], live = head[1];
    if (blockIdx.y > 0) {
        run_copies(pools.pool[blockIdx.y - 1], moves, nullptr, n, 1, num_pages, nullptr);
        return;
    }
    const int first = blockIdx.x * kCopyThreads + threadIdx.x, step = gridDim.x * kCopyThreads;
    // Counts: each move carries its own two entries; the rest is copied where the output is another buffer.
    for (int k = first; k < n; k += step) {
        const int2 m = moves[k];
        refs_out[m.y] = refs[m.x];
        refs_out[m.x] = 0;
    }
    if (refs_out != refs)
        for (int q = first; q < num_pages; q += step)
            if ((refs[q] != 0) == (q < live)) refs_out[q] = refs[q];
    for (int r = blockIdx.x; r < rows; r += gridDim.x) {
        const int len = context_lens[r];
        const int held = len < 0 ? 0 : min(pages_for(len, page_size), max_pages_per_seq);
        const size_t row = static_cast<size_t>(r) * max_pages_per_seq;
        for (int k = threadIdx.x; k < max_pages_per_seq; k += kCopyThreads) {
            int page = block_table[row + k];
            if (k < held) {
                if (page < 0 || page >= num_pages) {
                    raise(status_flag, AC_FLAG_PAGE_OOB);
                } else if (page >= live) {
                    const int k = place[page];
                    if (k >= 0) page = moves[k].y; else raise(status_flag, AC_FLAG_REF_COUNT);
                }
            }
            table_out[row + k] = page;
        }
    }
}

template <int N>
PoolArgs<N> pool_args(const ac_page_pool* pools, int n_pools) {
    PoolArgs<N> a;
    for (int i = 0; i < N; ++i) a.pool[i] = i < n_pools ? pools[i] : ac_page_pool{nullptr, 0, 1, 0};
    return a;
}

// CTAs per pool: enough warps for every piece of `jobs` pages, at most 8 CTAs per SM over all pools (two waves of the four
// that are resident with 62 or 64 registers a thread).  Fork and compaction raise it to what their tables take.
unsigned copy_grid(const ac_page_pool* pools, int n_pools, long long jobs, int sms) {
    long long most = 1;
    for (int i = 0; i < n_pools; ++i) {
        const int segments = pools[i].segments == AC_PAGE_WHOLE ? 1 : pools[i].segments;
        const long long seg = pools[i].page_bytes / segments;
        const long long units = jobs * segments * ((seg + kPiece - 1) / kPiece);
        const long long ctas = (units + kCopyThreads / 32 - 1) / (kCopyThreads / 32);
        most = ctas > most ? ctas : most;
    }
    const long long cap = (8ll * sms + n_pools - 1) / (n_pools > 0 ? n_pools : 1);
    return static_cast<unsigned>(most < cap ? most : cap);
}

}  // namespace

cudaError_t launch_copy_pages(const ac_page_pool* pools, int n_pools, const int32_t* pairs, int n, int num_pages,
                              int32_t* status_flag, int sms, cudaStream_t stream) {
    const dim3 grid(copy_grid(pools, n_pools, n, sms), n_pools);
    const int2* sd = reinterpret_cast<const int2*>(pairs);
    if (n_pools <= kFewPools)
        copy_pages_kernel<<<grid, kCopyThreads, 0, stream>>>(pool_args<kFewPools>(pools, n_pools), sd, n, num_pages, status_flag);
    else
        copy_pages_kernel<<<grid, kCopyThreads, 0, stream>>>(pool_args<AC_MAX_PAGE_POOLS>(pools, n_pools), sd, n, num_pages,
                                                             status_flag);
    return cudaGetLastError();
}

cudaError_t launch_reserve(int32_t* block_table, int max_pages_per_seq, const int32_t* context_lens, int32_t* refs,
                           int new_tokens, int rows, int page_size, int num_pages, void* workspace,
                           int32_t* status_flag, cudaStream_t stream) {
    int32_t* offsets = static_cast<int32_t*>(workspace);
    reserve_kernel<<<1, kPlanThreads, 0, stream>>>(block_table, max_pages_per_seq, context_lens, refs, new_tokens, rows,
                                                   page_size, num_pages, offsets, offsets + rows, status_flag);
    return cudaGetLastError();
}

cudaError_t launch_fork(const ac_page_pool* pools, int n_pools, int32_t* block_table, int max_pages_per_seq,
                        int32_t* context_lens, int32_t* refs, const int32_t* pairs, int n, int rows, int page_size,
                        int num_pages, void* workspace, int32_t* status_flag, int sms, cudaStream_t stream) {
    int2* jobs = static_cast<int2*>(workspace);
    int32_t* lens = reinterpret_cast<int32_t*>(jobs + n);
    int32_t* list = lens + n;
    const int2* pc = reinterpret_cast<const int2*>(pairs);
    fork_plan_kernel<<<1, kPlanThreads, 0, stream>>>(block_table, max_pages_per_seq, context_lens, refs, pc, n, rows,
                                                     page_size, num_pages, jobs, lens, list, status_flag);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    unsigned x = copy_grid(pools, n_pools, n, sms);
    const unsigned forks = n < 8 * sms ? n : 8 * sms;
    if (x < forks) x = forks;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(x, n_pools + 1);
    cfg.blockDim = dim3(kCopyThreads);
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
#define AC_FORK_APPLY(N_)                                                                                            \
    cudaLaunchKernelEx(&cfg, fork_apply_kernel<N_>, pool_args<N_>(pools, n_pools), block_table, max_pages_per_seq,   \
                       context_lens, refs, pc, static_cast<const int2*>(jobs), static_cast<const int32_t*>(lens), n, \
                       rows, page_size, num_pages, status_flag)
    return n_pools <= kFewPools ? AC_FORK_APPLY(kFewPools) : AC_FORK_APPLY(AC_MAX_PAGE_POOLS);
#undef AC_FORK_APPLY
}

cudaError_t launch_release(const int32_t* block_table, int max_pages_per_seq, int32_t* context_lens, int32_t* refs,
                           const int32_t* row_list, int n, int rows, int page_size, int num_pages,
                           int32_t* status_flag, cudaStream_t stream) {
    release_kernel<<<n, kCopyThreads, 0, stream>>>(block_table, max_pages_per_seq, context_lens, refs, row_list, rows,
                                                   page_size, num_pages, status_flag);
    return cudaGetLastError();
}

cudaError_t launch_trim(const int32_t* block_table, int max_pages_per_seq, const int32_t* context_lens, int32_t* refs,
                        int rows, int page_size, int num_pages, int32_t* status_flag, cudaStream_t stream) {
    const cudaError_t e = cudaMemsetAsync(refs, 0, static_cast<size_t>(num_pages) * sizeof(int32_t), stream);
    if (e != cudaSuccess) return e;
    count_held_kernel<<<rows, kCopyThreads, 0, stream>>>(block_table, max_pages_per_seq, context_lens, refs, page_size,
                                                         num_pages, status_flag);
    return cudaGetLastError();
}

cudaError_t launch_compact(const ac_page_pool* pools, int n_pools, const int32_t* block_table, int32_t* table_out,
                           int max_pages_per_seq, const int32_t* context_lens, const int32_t* refs, int32_t* refs_out,
                           int rows, int page_size, int num_pages, int32_t* live_out, void* workspace,
                           int32_t* status_flag, int sms, cudaStream_t stream) {
    const int chunks = (num_pages + kChunk - 1) / kChunk;
    int32_t* head = static_cast<int32_t*>(workspace);
    int2* moves = reinterpret_cast<int2*>(head + 4);
    int32_t* place = reinterpret_cast<int32_t*>(moves + num_pages / 2 + 1);
    int32_t* counts = place + num_pages;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(chunks);
    cfg.blockDim = dim3(kChunkThreads);
    cfg.stream = stream;
    cudaError_t e;
    if (chunks > 1) {
        compact_count_kernel<<<chunks, kChunkThreads, 0, stream>>>(refs, num_pages, counts);
        if ((e = cudaGetLastError()) != cudaSuccess) return e;
        cfg.attrs = attr;                      // only behind the counting kernel: otherwise after everything before it
        cfg.numAttrs = 1;
    }
    e = cudaLaunchKernelEx(&cfg, compact_rank_kernel, refs, num_pages, static_cast<const int32_t*>(counts), head, moves,
                           place, live_out);
    if (e != cudaSuccess) return e;
    // how many pages move is known on the device only: at most half of them
    unsigned x = copy_grid(pools, n_pools, num_pages / 2 + 1, sms);
    const unsigned table = static_cast<unsigned>(rows < 2 * sms ? rows : 2 * sms);
    if (x < table) x = table;
    cfg.gridDim = dim3(x, n_pools + 1);
    cfg.blockDim = dim3(kCopyThreads);
    cfg.attrs = attr;
    cfg.numAttrs = 1;
#define AC_COMPACT_APPLY(N_)                                                                                         \
    cudaLaunchKernelEx(&cfg, compact_apply_kernel<N_>, pool_args<N_>(pools, n_pools), block_table, table_out,        \
                       max_pages_per_seq, context_lens, refs, refs_out, rows, page_size, num_pages,                  \
                       static_cast<const int32_t*>(head), static_cast<const int2*>(moves),                           \
                       static_cast<const int32_t*>(place), status_flag)
    return n_pools <= kFewPools ? AC_COMPACT_APPLY(kFewPools) : AC_COMPACT_APPLY(AC_MAX_PAGE_POOLS);
#undef AC_COMPACT_APPLY
}

}  // namespace ac
