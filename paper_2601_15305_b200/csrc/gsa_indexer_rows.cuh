// One query row of the gated lightning indexer (Eq. 7, or Eq. 3) against tiles of 16 keys in registers: what the kernels for few rows
// a sequence share (gsa_indexer_rows.cu over contiguous keys, gsa_cache_indexer.cu over the pages of a cache).
#pragma once

#include "gsa_common.cuh"

namespace gsa {

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
    __device__ __forceinline__ void score(const KeyTile<DI>& ka, int act, float (&acc)[2]) const {
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
                if (act == 1) {                                     // Eq. 3: ReLU
                    v = fmaf(wv[e], fmaxf(s[hf * 2 + e] + bv[e], 0.f), v);
                } else {
                    float ex, rc;
                    const float arg = fminf(fmaf(s[hf * 2 + e], -1.4426950408889634f, bv[e]), 80.f);
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

}  // namespace gsa
