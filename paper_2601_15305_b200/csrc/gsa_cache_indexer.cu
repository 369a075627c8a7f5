// Gated lightning indexer (Eq. 7, Eq. 3) over the k^I in a cache's pages (include/gsa.h), every sequence with a length of its own.
//
// As in gsa_indexer_rows.cu a warp streams keys into the A operand of an MMA against the row's H^I queries.  The rows' keys, cut into
// steps of 32, are dealt to the warps of one wave in equal runs, whatever the lengths (each CTA sums the rows up for itself): lengths
// of 16K to 128K in one batch leave no SM behind.  A warp loads the next step's keys while it computes on the present one, and the pages
// of 32 tiles at a time.
// Bound: the stream of k^I, 2 dI bytes per (row, key); rows of one sequence meet in the L2.  32 rows over 16K to 128K keys of 64: 287 MB in
// and 9 MB out in 53 us, 86 % of a copy's rate.  One row of 32771: 3.7 us, a call's latency.
#include "gsa_cache.cuh"

namespace gsa {

namespace {

constexpr int kWarps = 8;
constexpr int kStepTiles = 2;              // tiles of 16 keys that a warp computes on at a time
constexpr int kStep = kStepTiles * 16;
constexpr int kMaxRows = 2048;             // rows of one launch

__device__ __forceinline__ void ldg32(const void* p, uint4& lo, uint4& hi) {
    asm volatile("ld.global.nc.L1::no_allocate.v8.u32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(lo.x), "=r"(lo.y), "=r"(lo.z), "=r"(lo.w), "=r"(hi.x), "=r"(hi.y), "=r"(hi.z), "=r"(hi.w)
                 : "l"(p));
}

// Lane tig owns the tig-th quarter of every key row (DI/4 consecutive elements); the B operand
// q^I[head = gid] is read with the same split, so both sides agree on which d a k-index means.
template <int DI>
struct KeyTile {
    static constexpr int kElems = DI / 4;              // bf16 per lane and key: 16 (DI 64) or 8 (DI 32)
    uint32_t v[2][kElems / 2];                          // [key gid / gid + 8][packed pairs]
    __device__ __forceinline__ void load(int hf, const unsigned char* kp) {
        if constexpr (kElems == 16) {
            uint4 lo, hi;
            ldg32(kp, lo, hi);
            v[hf][0] = lo.x; v[hf][1] = lo.y; v[hf][2] = lo.z; v[hf][3] = lo.w;
            v[hf][4] = hi.x; v[hf][5] = hi.y; v[hf][6] = hi.z; v[hf][7] = hi.w;
        } else {
            const uint4 x = __ldg(reinterpret_cast<const uint4*>(kp));
            v[hf][0] = x.x; v[hf][1] = x.y; v[hf][2] = x.z; v[hf][3] = x.w;
        }
    }
};

template <int DI, int HI>
struct RowQuery {
    static constexpr int kElems = DI / 4;
    uint32_t qb[kElems / 2];
    float wv[2], bv[2];                                 // heads 2*tig, 2*tig+1 are this lane's columns of S^T
    // row: number of the query row in qI [.., HI, DI] and w [.., HI]
    __device__ __forceinline__ void load(const __nv_bfloat16* qI, const float* w, const float* bI, size_t row, int act, int gid, int tig) {
        const __nv_bfloat16* qp = qI + (row * HI + (gid < HI ? gid : 0)) * DI + tig * kElems;
#pragma unroll
        for (int i = 0; i < kElems / 2; ++i) qb[i] = gid < HI ? *reinterpret_cast<const uint32_t*>(qp + 2 * i) : 0u;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int h = 2 * tig + e;
            wv[e] = h < HI ? w[row * HI + h] : 0.f;
            bv[e] = (bI && h < HI) ? bI[h] * (act == 1 ? 1.0f : -1.4426950408889634f) : 0.f;
        }
    }
    // scores of keys gid and gid + 8 of a tile, in every lane of a key
    __device__ __forceinline__ void score(const KeyTile<DI>& ka, int act, int tig, float (&acc)[2]) const {
        float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < kElems / 4; ++ks)         // one k-step uses 4 of the lane's elements
            mma_bf16_16816(s, ka.v[0][2 * ks], ka.v[1][2 * ks], ka.v[0][2 * ks + 1], ka.v[1][2 * ks + 1], qb[2 * ks], qb[2 * ks + 1]);
        // s[0], s[1]: key gid, heads 2tig, 2tig+1;  s[2], s[3]: key gid + 8
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            float v = 0.f;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                // A NaN stays one (fminf, fmaxf would make it a gate of 2^-80, a closed ReLU: a key that is never chosen, and nothing to
                // show for it).  Columns without a head are 0: a key's infinity times their zeros is none of it.
                const float x = HI == 8 || 2 * tig + e < HI ? s[hf * 2 + e] : 0.f;
                if (act == 1) {                                     // Eq. 3: ReLU
                    v = fmaf(wv[e], max_nan(x + bv[e], 0.f), v);
                } else {
                    float ex, rc;
                    const float arg = min_nan(fmaf(x, -1.4426950408889634f, bv[e]), 80.f);
                    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(ex) : "f"(arg));
                    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(rc) : "f"(1.0f + ex));
                    v = fmaf(wv[e], rc, v);
                }
            }
            v += __shfl_xor_sync(0xFFFFFFFFu, v, 1);
            v += __shfl_xor_sync(0xFFFFFFFFu, v, 2);
            acc[hf] = v;
        }
    }
};

struct CacheIndexArgs {
    CacheView c;
    const __nv_bfloat16* qI;
    const float *w, *bI;
    float* scores;
    int64_t row_stride;
    int32_t* ws;
    int32_t row0, rows, Lq, Lk, act;
};

template <int DI, int HI>
__global__ void __launch_bounds__(kWarps * 32, 2) gsa_cache_indexer_kernel(const CacheIndexArgs a) {
    chain_wait();
    extern __shared__ int32_t cum[];       // [rows + 1] steps in front of each row
    __shared__ int32_t warp_sum[kWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int gid = lane >> 2, tig = lane & 3;
    const CacheView& c = a.c;
    bool bad = false;
    auto keys_of = [&](int32_t row, int32_t& b) -> int32_t {           // visible keys of a row of the launch
        b = (a.row0 + row) / a.Lq;
        return checked_len(c, b, a.Lk, bad) - a.Lq + (a.row0 + row - b * a.Lq) + 1;
    };

    int32_t steps = 0;
    {
        const int per = (a.rows + kWarps * 32 - 1) / (kWarps * 32), r0 = min(a.rows, (int)threadIdx.x * per), r1 = min(a.rows, r0 + per);
        int32_t mine = 0, b;
        for (int r = r0; r < r1; ++r) {
            const int32_t n = (max(keys_of(r, b), 0) + kStep - 1) / kStep;
            cum[r] = n;
            mine += n;
        }
        int32_t inc = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int32_t v = __shfl_up_sync(0xFFFFFFFFu, inc, o);
            if (lane >= o) inc += v;
        }
        if (lane == 31) warp_sum[warp] = inc;
        __syncthreads();
        int32_t at = inc - mine;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            if (w < warp) at += warp_sum[w];
            steps += warp_sum[w];
        }
        for (int r = r0; r < r1; ++r) {
            const int32_t n = cum[r];
            cum[r] = at;
            at += n;
        }
        if (threadIdx.x == 0) cum[a.rows] = steps;
        __syncthreads();
    }
    const int32_t units = gridDim.x * kWarps, unit = warp * gridDim.x + blockIdx.x;
    int32_t g = (int32_t)((int64_t)unit * steps / units);
    const int32_t g_end = (int32_t)((int64_t)(unit + 1) * steps / units);
    int32_t row = 0;                       // the row that holds step g
    for (int32_t rh = a.rows - 1; row < rh;) {
        const int32_t m = (row + rh + 1) >> 1;
        if (cum[m] <= g) row = m; else rh = m - 1;
    }
    using Tile = KeyTile<DI>;
    while (g < g_end) {
        while (cum[row + 1] <= g) ++row;   // (rows that see nothing are passed over)
        int32_t b;
        const int32_t n = keys_of(row, b);
        const int32_t k_end = min(n, (min(cum[row + 1], g_end) - cum[row]) * kStep);
        RowQuery<DI, HI> q;
        q.load(a.qI, a.w, a.bI, (size_t)(a.row0 + row), a.act, gid, tig);
        float* __restrict__ out_row = a.scores + (int64_t)(a.row0 + row) * a.row_stride;
        const unsigned char* const kbase = c.pool + c.keys_off + tig * (Tile::kElems * 2);
        int32_t pages = 0, tile0 = INT32_MIN;          // lane l: page of tile tile0 + l (of the last visible key for a tile behind it)
        auto load = [&](Tile(&ka)[kStepTiles], int32_t k0) {
            if (k0 >= k_end) return;
            const int32_t tile = k0 >> 4;
            if (tile < tile0 || tile + kStepTiles > tile0 + 32) {
                tile0 = tile;
                pages = checked_page(c, b, min((tile0 + lane) * 16, n - 1), bad);
            }
#pragma unroll
            for (int u = 0; u < kStepTiles; ++u) {
                const int32_t page = __shfl_sync(0xFFFFFFFFu, pages, tile + u - tile0);
                const unsigned char* kpage = kbase + (int64_t)page * c.page_bytes;
                // (places behind the row's end: slots of an existing page, whatever they hold; their scores are not stored)
#pragma unroll
                for (int hf = 0; hf < 2; ++hf) ka[u].load(hf, kpage + (uint32_t)((k0 + u * 16 + hf * 8 + gid) & (c.T - 1)) * (DI * 2));
            }
        };
        auto compute = [&](const Tile(&ka)[kStepTiles], int32_t k0) {
#pragma unroll
            for (int u = 0; u < kStepTiles; ++u) {
                float acc[2];
                q.score(ka[u], a.act, tig, acc);
                const int32_t key = k0 + u * 16 + (tig & 1) * 8 + gid;
                if (tig < 2 && key < k_end) out_row[key] = acc[tig & 1];
            }
        };
        Tile even[kStepTiles], odd[kStepTiles];
        int32_t k0 = (g - cum[row]) * kStep;
        load(even, k0);
        while (true) {
            load(odd, k0 + kStep);
            compute(even, k0);
            if ((k0 += kStep) >= k_end) break;
            load(even, k0 + kStep);
            compute(odd, k0);
            if ((k0 += kStep) >= k_end) break;
        }
        g = min(cum[row + 1], g_end);
    }
    write_flags(a.ws, bad, a.row0);
}

template <int DI, int HI>
cudaError_t launch_t(const CacheIndexArgs& a, unsigned ctas, cudaStream_t st) {
    cudaError_t e = launch_chained(gsa_cache_indexer_kernel<DI, HI>, ctas, kWarps * 32, (size_t)(a.rows + 1) * 4, st, a);
    ++g_launches;
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

cudaError_t launch_cache_indexer(const CacheView& c, const gsa_params_t& p, const __nv_bfloat16* qI, const float* w, const float* bI,
                                 float* scores, int64_t row_stride, int32_t* ws, cudaStream_t st) {
    CacheIndexArgs a{};
    a.c = c; a.qI = qI; a.w = w; a.bI = bI; a.scores = scores; a.row_stride = row_stride; a.ws = ws;
    a.Lq = p.Lq; a.Lk = p.Lk; a.act = p.act;
    const int32_t all = p.B * p.Lq;
    for (int32_t r0 = 0; r0 < all; r0 += kMaxRows) {
        a.row0 = r0; a.rows = all - r0 < kMaxRows ? all - r0 : kMaxRows;
        // one wave, or a warp for every step that there can be
        const int64_t most = ((int64_t)a.rows * ((p.Lk + kStep - 1) / kStep) + 3) / 4, wave = (int64_t)sm_count() * 2;
        const unsigned ctas = (unsigned)(most < wave ? most : wave);
        cudaError_t e = cudaErrorInvalidValue;
#define GSA_INDEX_CASE(DI_, HI_) if (p.dI == DI_ && p.HI == HI_) e = launch_t<DI_, HI_>(a, ctas, st)
        GSA_INDEX_CASE(64, 8); GSA_INDEX_CASE(64, 4); GSA_INDEX_CASE(64, 2); GSA_INDEX_CASE(64, 1);
        GSA_INDEX_CASE(32, 8); GSA_INDEX_CASE(32, 4); GSA_INDEX_CASE(32, 2); GSA_INDEX_CASE(32, 1);
#undef GSA_INDEX_CASE
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace gsa
