// Pages of a cache: handing out, forking, freeing, compacting (include/gsa.h).
//
// The reference counts are the only record of what is free: a page is free if its count is 0.  A call that takes pages plans in one
// CTA: the counts become a bitmap in shared memory (one bit a page, at most 128 KB), a scan of its words numbers the free pages, and
// the r-th free page goes to the r-th request, requests in the order of the sequences.  So the outcome depends on nothing but the
// tables, and a call that does not fit is refused before it has changed anything.  Bound: latency of the reads of the counts (65536 of
// them are 256 KB for one SM); a call that takes no page does not read them.  Page copies are a second kernel over the whole GPU, bound
// by HBM (every byte read and written once).  Eight prompts to 32 beams and their release: 13 us, three launches (counts asked
// for together with the lengths changed nothing); 5600 pages of 80 KB of which a fourth move: 6 us of plan, 35 of copies.
#include "gsa_cache.cuh"

namespace gsa {

namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPlanWarps = kPlanThreads / 32;
constexpr int kMaxSeqs = 4096;                   // B <= 4096: four sequences a thread
constexpr int kSeqsPerThread = kMaxSeqs / kPlanThreads;
constexpr int kCopyChunk = 4096;                 // bytes of a page that a warp copies at a time: eight 16-byte loads a lane
// words of the workspace head behind the status word
constexpr int kCopiesWord = 8;                   // pages that the copy kernel moves
constexpr int kLiveWord = 9;                     // compaction: live pages

struct PlanShared {
    int32_t offs[kMaxSeqs + 1];                  // requests in front of each sequence
    uint32_t warp_tot[kPlanWarps];
    uint32_t total, bad, cut;
};

// exclusive prefix over the CTA's threads and the total (two barriers)
__device__ __forceinline__ uint32_t plan_scan(PlanShared& sh, uint32_t v, uint32_t& total) {
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    uint32_t inc = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t u = __shfl_up_sync(0xFFFFFFFFu, inc, o);
        if (lane >= o) inc += u;
    }
    __syncthreads();                             // (warp_tot of the scan before has been read)
    if (lane == 31) sh.warp_tot[wid] = inc;
    __syncthreads();
    const uint32_t tot = sh.warp_tot[lane];
    total = __reduce_add_sync(0xFFFFFFFFu, tot);
    return __reduce_add_sync(0xFFFFFFFFu, lane < wid ? tot : 0u) + inc - v;
}

// Bitmap of the pages whose count is 0 (free) or is not (live), bits behind n_pages clear.
__device__ __forceinline__ void page_bitmap(const CacheView& c, uint32_t* bits, bool live) {
    const int words = (c.n_pages + 31) / 32, lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    for (int w0 = wid * 8; w0 < words; w0 += kPlanWarps * 8) {       // eight loads of a lane in flight
        int32_t r[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int page = (w0 + i) * 32 + lane;
            r[i] = page < c.n_pages ? c.refs[page] : (live ? 0 : 1);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t b = __ballot_sync(0xFFFFFFFFu, live ? r[i] != 0 : r[i] == 0);
            if (lane == 0 && w0 + i < words) bits[w0 + i] = b;
        }
    }
}

// Calls f(rank, page) for every set bit whose rank is below `limit`; ranks count set bits from page 0 on.  Warp w has a run of words.
template <class F>
__device__ __forceinline__ void each_set_page(PlanShared& sh, const uint32_t* bits, int words, uint32_t limit, uint32_t& total, F f) {
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    const int per = (words + kPlanWarps - 1) / kPlanWarps, lo = min(words, wid * per), hi = min(words, lo + per);
    uint32_t mine = 0;
    for (int w = lo + lane; w < hi; w += 32) mine += __popc(bits[w]);
    uint32_t at = __reduce_add_sync(0xFFFFFFFFu, mine);
    {
        // warps in front of this one
        __syncthreads();
        if (lane == 0) sh.warp_tot[wid] = at;
        __syncthreads();
        const uint32_t tot = sh.warp_tot[lane];
        total = __reduce_add_sync(0xFFFFFFFFu, tot);
        at = __reduce_add_sync(0xFFFFFFFFu, lane < wid ? tot : 0u);
    }
    if (total < limit) return;                   // (too few: the caller refuses)
    for (int w0 = lo; w0 < hi && at < limit; w0 += 32) {
        const uint32_t word = w0 + lane < hi ? bits[w0 + lane] : 0u;
        const int in = min(32, hi - w0);
        for (int i = 0; i < in && at < limit; ++i) {
            const uint32_t x = __shfl_sync(0xFFFFFFFFu, word, i);
            const uint32_t rank = at + __popc(x & ((1u << lane) - 1u));
            if (((x >> lane) & 1u) && rank < limit) f(rank, (w0 + i) * 32 + lane);
            at += __popc(x);
        }
    }
}

// the sequence that request r belongs to: offs[b] <= r < offs[b + 1]
__device__ __forceinline__ int seq_of(const PlanShared& sh, int B, uint32_t r) {
    int lo = 0, hi = B - 1;
    while (lo < hi) {
        const int m = (lo + hi + 1) >> 1;
        if ((uint32_t)sh.offs[m] <= r) lo = m; else hi = m - 1;
    }
    return lo;
}

__device__ __forceinline__ void write_head(int32_t* ws, int32_t status, int32_t copies, int32_t live, int32_t mark = 0) {
    for (int i = threadIdx.x; i < kStatusBytes / 4; i += kPlanThreads)
        ws[i] = i == 0 ? status : i == kCopiesWord ? copies : i == kLiveWord ? live : i == kRefusedWord ? mark : 0;
}

__device__ __forceinline__ int pages_of(const CacheView& c, int n) { return (n + c.T - 1) >> c.log_t; }

__global__ void __launch_bounds__(kPlanThreads) gsa_cache_reserve_kernel(const CacheView c, const int32_t* __restrict__ n_new,
                                                                         int32_t* __restrict__ start, int32_t* __restrict__ ws) {
    chain_wait();
    extern __shared__ __align__(16) unsigned char dyn_smem[];
    PlanShared& sh = *reinterpret_cast<PlanShared*>(dyn_smem);
    uint32_t* bits = reinterpret_cast<uint32_t*>(dyn_smem + sizeof(PlanShared));
    const int tid = threadIdx.x;
    const int64_t cap = (int64_t)c.max_pages << c.log_t;
    if (tid == 0) sh.bad = 0u;
    __syncthreads();
    int32_t len[kSeqsPerThread], add[kSeqsPerThread];
    uint32_t need = 0;
#pragma unroll
    for (int i = 0; i < kSeqsPerThread; ++i) {
        const int b = tid * kSeqsPerThread + i;
        len[i] = add[i] = 0;
        if (b < c.B) {
            len[i] = c.lens[b];
            add[i] = n_new[b];
            if (len[i] < 0 || add[i] < 0 || (int64_t)len[i] + add[i] > cap) sh.bad = 1u;
            else need += pages_of(c, len[i] + add[i]) - pages_of(c, len[i]);
        }
    }
    need = min(need, (uint32_t)c.n_pages + 1u);  // (more than there are: refused below; 1024 such sums stay within 32 bits)
    uint32_t total;
    uint32_t at = plan_scan(sh, need, total);
#pragma unroll
    for (int i = 0; i < kSeqsPerThread; ++i) {
        const int b = tid * kSeqsPerThread + i;
        if (b < c.B) {
            sh.offs[b] = (int32_t)at;
            if (!sh.bad) at += pages_of(c, len[i] + add[i]) - pages_of(c, len[i]);
        }
    }
    int32_t status = sh.bad ? kDevBadIndex : kDevOk;
    if (!sh.bad && total) {
        page_bitmap(c, bits, false);
        __syncthreads();
        uint32_t free_pages;
        each_set_page(sh, bits, (c.n_pages + 31) / 32, total, free_pages, [&](uint32_t r, int page) {
            const int b = seq_of(sh, c.B, r);
            const int j = pages_of(c, c.lens[b]) + (int)(r - (uint32_t)sh.offs[b]);
            c.table[(int64_t)b * c.max_pages + j] = page;
            c.refs[page] = 1;
        });
        if (free_pages < total) status = kDevCacheFull;
        __syncthreads();                         // (lens of every sequence has been read)
    }
#pragma unroll
    for (int i = 0; i < kSeqsPerThread; ++i) {
        const int b = tid * kSeqsPerThread + i;
        if (b < c.B) {
            start[b] = status == kDevOk ? len[i] : -1;
            if (status == kDevOk && add[i]) c.lens[b] = len[i] + add[i];
        }
    }
    write_head(ws, status, 0, 0, status == kDevOk ? 0 : kRefusedMark);
}

// Plan of a fork: new pages into the tables, the pages to copy into the list (source, destination).
__global__ void __launch_bounds__(kPlanThreads) gsa_cache_fork_kernel(const CacheView c, const int32_t* __restrict__ src_of,
                                                                      int32_t share, int32_t* __restrict__ ws) {
    chain_wait();
    extern __shared__ __align__(16) unsigned char dyn_smem[];
    PlanShared& sh = *reinterpret_cast<PlanShared*>(dyn_smem);
    uint32_t* bits = reinterpret_cast<uint32_t*>(dyn_smem + sizeof(PlanShared));
    int32_t* list = ws + kStatusBytes / 4;       // n_pages sources, n_pages destinations
    const int tid = threadIdx.x;
    const int64_t cap = (int64_t)c.max_pages << c.log_t;
    if (tid == 0) { sh.bad = 0u; sh.cut = 0u; }
    __syncthreads();
    int32_t len[kSeqsPerThread];                 // of the sequence that b becomes a copy of; -1: b stays
    uint32_t cnt[kSeqsPerThread], need = 0;
#pragma unroll
    for (int i = 0; i < kSeqsPerThread; ++i) {
        const int b = tid * kSeqsPerThread + i;
        len[i] = -1;
        cnt[i] = 0u;
        if (b < c.B) {
            const int src = src_of[b];
            if (src >= 0) {
                if (src >= c.B || src == b || c.lens[b] != 0) sh.bad = 1u;
                else {
                    const int n = c.lens[src];
                    if (src_of[src] >= 0 || n < 0 || n > cap) sh.bad = 1u;
                    else {
                        len[i] = n;
                        cnt[i] = share ? ((n & (c.T - 1)) != 0 ? 1u : 0u) : (uint32_t)pages_of(c, n);
                    }
                }
            }
        }
        need += cnt[i];
    }
    need = min(need, (uint32_t)c.n_pages + 1u);  // (as in the kernel above)
    uint32_t total;
    uint32_t at = plan_scan(sh, need, total);
#pragma unroll
    for (int i = 0; i < kSeqsPerThread; ++i) {
        const int b = tid * kSeqsPerThread + i;
        if (b < c.B) { sh.offs[b] = (int32_t)at; at += cnt[i]; }
    }
    int32_t status = sh.bad ? kDevBadIndex : kDevOk;
    if (!sh.bad && total) {
        page_bitmap(c, bits, false);
        __syncthreads();
        uint32_t free_pages;
        each_set_page(sh, bits, (c.n_pages + 31) / 32, total, free_pages, [&](uint32_t r, int page) {
            const int b = seq_of(sh, c.B, r), src = src_of[b];
            const int first = share ? c.lens[src] >> c.log_t : 0;
            const int j = first + (int)(r - (uint32_t)sh.offs[b]);
            int from = c.table[(int64_t)src * c.max_pages + j];
            if ((uint32_t)from >= (uint32_t)c.n_pages) { sh.cut = 1u; from = page; }      // (a table that names no page: nothing to copy)
            c.table[(int64_t)b * c.max_pages + j] = page;
            c.refs[page] = 1;
            list[r] = from;
            list[c.n_pages + r] = page;
        });
        if (free_pages < total) status = kDevCacheFull;
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < kSeqsPerThread; ++i) {
        const int b = tid * kSeqsPerThread + i;
        if (b < c.B && len[i] >= 0 && status == kDevOk) c.lens[b] = len[i];
    }
    if (status == kDevOk && sh.cut) status = kDevBadIndex;
    // (the second kernel shares pages only if this one went through: its word says how many copies, -1: refused)
    const bool done = status == kDevOk || sh.cut;
    write_head(ws, status, done ? (int32_t)total : -1, 0);
}

// Plan of a compaction: the k-th live page at or behind position n (the number of live pages) takes the place of the k-th free one in
// front of it.  With live(i) = live pages in front of page i, those ranks are i - live(i) and live(i) - live(n).
__global__ void __launch_bounds__(kPlanThreads) gsa_cache_compact_kernel(const CacheView c, int32_t* __restrict__ live_pages,
                                                                         int32_t* __restrict__ ws) {
    chain_wait();
    extern __shared__ __align__(16) unsigned char dyn_smem[];
    PlanShared& sh = *reinterpret_cast<PlanShared*>(dyn_smem);
    uint32_t* bits = reinterpret_cast<uint32_t*>(dyn_smem + sizeof(PlanShared));
    int32_t* src = ws + kStatusBytes / 4;
    int32_t* dst = src + c.n_pages;
    int32_t* remap = dst + c.n_pages;
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    const int words = (c.n_pages + 31) / 32;
    page_bitmap(c, bits, true);
    __syncthreads();
    const int per = (words + kPlanWarps - 1) / kPlanWarps, lo = min(words, wid * per), hi = min(words, lo + per);
    uint32_t mine = 0;
    for (int w = lo + lane; w < hi; w += 32) mine += __popc(bits[w]);
    const uint32_t own = __reduce_add_sync(0xFFFFFFFFu, mine);
    if (lane == 0) sh.warp_tot[wid] = own;
    __syncthreads();
    const uint32_t tot = sh.warp_tot[lane];
    const uint32_t n = __reduce_add_sync(0xFFFFFFFFu, tot);
    uint32_t at = __reduce_add_sync(0xFFFFFFFFu, lane < wid ? tot : 0u);
    // live pages in front of position n
    uint32_t front = 0;
    for (int w = tid; w < (int)(n + 31) / 32; w += kPlanThreads) {
        const uint32_t left = n - (uint32_t)w * 32;
        front += __popc(left >= 32 ? bits[w] : bits[w] & ((1u << left) - 1u));
    }
    uint32_t live_front;
    plan_scan(sh, front, live_front);
    const uint32_t moves = n - live_front;
    for (int w0 = lo; w0 < hi; w0 += 32) {
        const uint32_t word = w0 + lane < hi ? bits[w0 + lane] : 0u;
        const int in = min(32, hi - w0);
        for (int i = 0; i < in; ++i) {
            const uint32_t x = __shfl_sync(0xFFFFFFFFu, word, i);
            const uint32_t page = (uint32_t)(w0 + i) * 32 + lane, before = at + __popc(x & ((1u << lane) - 1u));
            const bool live = (x >> lane) & 1u;
            if (page < (uint32_t)c.n_pages) {
                if (page < n) {
                    if (!live) dst[page - before] = (int32_t)page;
                } else {
                    if (live) src[before - live_front] = (int32_t)page;
                    else remap[page] = -1;
                }
            }
            at += __popc(x);
        }
    }
    __syncthreads();
    for (uint32_t r = tid; r < moves; r += kPlanThreads) {
        const int from = src[r], to = dst[r];
        remap[from] = to;
        c.refs[to] = c.refs[from];
        c.refs[from] = 0;
    }
    if (tid == 0) live_pages[0] = (int32_t)n;
    write_head(ws, kDevOk, (int32_t)moves, (int32_t)n);
}

// ---- what the plans leave to the whole GPU ---------------------------------------------------------------------------------
__device__ __forceinline__ void copy_pages(const CacheView& c, const int32_t* list, int32_t n) {
    const int lane = threadIdx.x & 31;
    const int64_t warps = (int64_t)gridDim.x * (blockDim.x >> 5);
    const int chunks = (int)((c.page_bytes + kCopyChunk - 1) / kCopyChunk);
    for (int64_t i = (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5); i < (int64_t)n * chunks; i += warps) {
        const int32_t r = (int32_t)(i / chunks);
        const int64_t off = (i - (int64_t)r * chunks) * kCopyChunk + lane * 16;
        const unsigned char* s = c.pool + (int64_t)list[r] * c.page_bytes + off;
        unsigned char* d = c.pool + (int64_t)list[c.n_pages + r] * c.page_bytes + off;
        uint4 v[kCopyChunk / 512];
#pragma unroll
        for (int k = 0; k < kCopyChunk / 512; ++k)
            if (off + k * 512 < c.page_bytes) v[k] = *reinterpret_cast<const uint4*>(s + k * 512);
#pragma unroll
        for (int k = 0; k < kCopyChunk / 512; ++k)
            if (off + k * 512 < c.page_bytes) *reinterpret_cast<uint4*>(d + k * 512) = v[k];
    }
}

__global__ void __launch_bounds__(256) gsa_cache_fork_copy_kernel(const CacheView c, const int32_t* __restrict__ src_of, int32_t share,
                                                                  int32_t* __restrict__ ws) {
    chain_wait();
    const int32_t n = ws[kCopiesWord];
    if (n < 0) return;
    if (share) {
        // full pages: one more reference each (integer sums: their order does not matter)
        const int64_t step = (int64_t)gridDim.x * 256;
        for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < (int64_t)c.B * c.max_pages; i += step) {
            const int b = (int)(i / c.max_pages), j = (int)(i - (int64_t)b * c.max_pages), src = src_of[b];
            if (src < 0 || j >= (c.lens[src] >> c.log_t)) continue;
            const int page = c.table[(int64_t)src * c.max_pages + j];
            c.table[i] = page;
            if ((uint32_t)page < (uint32_t)c.n_pages) atomicAdd(c.refs + page, 1);
            else report_bad_index(ws);
        }
    }
    copy_pages(c, ws + kStatusBytes / 4, n);
}

__global__ void __launch_bounds__(256) gsa_cache_compact_copy_kernel(const CacheView c, int32_t* __restrict__ ws) {
    chain_wait();
    const int32_t moves = ws[kCopiesWord], live = ws[kLiveWord];
    if (moves > 0) {
        const int32_t* remap = ws + kStatusBytes / 4 + 2 * (int64_t)c.n_pages;
        const int64_t step = (int64_t)gridDim.x * 256;
        for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < (int64_t)c.B * c.max_pages; i += step) {
            const int page = c.table[i];
            if (page < live || page >= c.n_pages) continue;
            const int to = remap[page];
            if (to >= 0) c.table[i] = to;
            else report_bad_index(ws);           // (a page that a table names and the counts say is free)
        }
    }
    copy_pages(c, ws + kStatusBytes / 4, moves);
}

__global__ void __launch_bounds__(256) gsa_cache_release_kernel(const CacheView c, const int32_t* __restrict__ drop, int32_t* __restrict__ ws) {
    chain_wait();
    bool bad = false;
    for (int b = blockIdx.x; b < c.B; b += gridDim.x) {
        if (!drop[b]) continue;
        const int len = c.lens[b], cap = c.max_pages << c.log_t, n = pages_of(c, min(max(len, 0), cap));
        bad |= len < 0 || len > cap;
        for (int j = threadIdx.x; j < c.max_pages; j += 256) {
            int32_t* at = c.table + (int64_t)b * c.max_pages + j;
            if (j < n) {
                const int page = *at;
                if ((uint32_t)page >= (uint32_t)c.n_pages) bad = true;
                else if (atomicSub(c.refs + page, 1) <= 0) {       // (counts that do not match the tables)
                    atomicAdd(c.refs + page, 1);
                    bad = true;
                }
            }
            *at = -1;
        }
        __syncthreads();                         // (everybody has read the length)
        if (threadIdx.x == 0) c.lens[b] = 0;
    }
    write_flags(ws, bad);
}

size_t plan_smem(const CacheView& c) { return sizeof(PlanShared) + (size_t)(c.n_pages + 31) / 32 * 4; }

template <auto KERN, class... A>
cudaError_t launch_plan(const CacheView& c, cudaStream_t st, A... args) {
    static std::atomic<uint64_t> granted{0};
    const size_t smem = plan_smem(c);
    cudaError_t e = grant_smem(granted, reinterpret_cast<const void*>(KERN), sizeof(PlanShared) + (1 << 20) / 8);
    if (e != cudaSuccess) return e;
    launch_chained(KERN, 1, kPlanThreads, smem, st, args...);
    ++g_launches;
    return cudaGetLastError();
}

}  // namespace

size_t cache_page_list_bytes(const CacheView& c) { return align_up((size_t)c.n_pages * 12, 256); }

cudaError_t launch_cache_reserve(const CacheView& c, const int32_t* n_new, int32_t* start, int32_t* ws, cudaStream_t st) {
    return launch_plan<gsa_cache_reserve_kernel>(c, st, c, n_new, start, ws);
}

cudaError_t launch_cache_fork(const CacheView& c, const int32_t* src_of, bool share, int32_t* ws, cudaStream_t st) {
    cudaError_t e = launch_plan<gsa_cache_fork_kernel>(c, st, c, src_of, share ? 1 : 0, ws);
    if (e != cudaSuccess) return e;
    launch_chained(gsa_cache_fork_copy_kernel, sm_count() * 4, 256, 0, st, c, src_of, share ? 1 : 0, ws);
    ++g_launches;
    return cudaGetLastError();
}

cudaError_t launch_cache_release(const CacheView& c, const int32_t* drop, int32_t* ws, cudaStream_t st) {
    launch_chained(gsa_cache_release_kernel, c.B < kMaxFlags ? c.B : kMaxFlags, 256, 0, st, c, drop, ws);
    ++g_launches;
    return cudaGetLastError();
}

cudaError_t launch_cache_compact(const CacheView& c, int32_t* live_pages, int32_t* ws, cudaStream_t st) {
    cudaError_t e = launch_plan<gsa_cache_compact_kernel>(c, st, c, live_pages, ws);
    if (e != cudaSuccess) return e;
    launch_chained(gsa_cache_compact_copy_kernel, sm_count() * 4, 256, 0, st, c, ws);
    ++g_launches;
    return cudaGetLastError();
}

}  // namespace gsa
