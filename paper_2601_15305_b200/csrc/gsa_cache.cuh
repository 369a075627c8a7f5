// The paged 4-bit cache (include/gsa.h) as the kernels see it.
#pragma once

#include "gsa_common.cuh"

namespace gsa {

struct CacheView {
    unsigned char* pool;
    int32_t *table, *lens, *refs;
    int64_t page_bytes;
    int32_t n_pages, T, log_t, max_pages, B;
    int32_t n_kv, d_h, dI;
    int32_t rec;                 // bytes of a token's record: D / 2 K codes, D / 2 V' codes, D / 8 scales, padding (D = n_kv * d_h)
    int32_t keys_off;            // where a page's k^I start: T * rec
};

constexpr int kCacheGroup = 16;  // values that share a scale
// A scale byte n is the top of an fp32 number's bits: exponent field 107 + n / 8 (2^(n / 8 - 20)) and three bits of the mantissa.
constexpr uint32_t kScaleBias = 107u << 3;
constexpr uint32_t kScaleNan = 255u;
// the same in bf16: (byte << 4) + kScaleBiasBf16
constexpr uint32_t kScaleBiasBf16 = kScaleBias << 4;

// tokens of sequence b, at most `cap`; `bad` is raised by a length outside [0, cap]
__device__ __forceinline__ int32_t checked_len(const CacheView& c, int32_t b, int32_t cap, bool& bad) {
    const int32_t n = __ldg(c.lens + b);
    bad |= n < 0 || n > cap;
    return min(max(n, 0), cap);
}
// page of position s (inside the table's row) of sequence b; `bad` is raised, and page 0 taken, by an entry that names none
__device__ __forceinline__ int32_t checked_page(const CacheView& c, int32_t b, int32_t s, bool& bad) {
    const int32_t page = __ldg(c.table + (int64_t)b * c.max_pages + (s >> c.log_t));
    if ((uint32_t)page < (uint32_t)c.n_pages) return page;
    bad = true;
    return 0;
}

// The smaller and the larger of two, NaN if one of them is (fminf and fmaxf give the other).  One instruction either way.
__device__ __forceinline__ float min_nan(float a, float b) {
    float d;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ float max_nan(float a, float b) {
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}

// What the CTAs of a call found wrong.  Each writes a word of its own behind the head, the first one the head, which says how many there are:
// gsa_device_status adds them up.  Nothing has to be cleared ahead of the call, which would be a launch of its own (2 us of the GPU, as
// much of the host).  Called by all threads of every CTA of a one-dimensional grid of at most kMaxFlags; launches of one call
// after its first (`before` != 0) add to the words.
constexpr int kFlagsWord = 10;             // int32 word of the head: number of words behind it (0: the status word is all there is)
constexpr int kMaxFlags = 4096;
// A refused reservation leaves kRefusedMark in this word of the head, next to its status.  The append behind it on the same workspace stores
// nothing, and would otherwise write "nothing wrong" over the only sign of it: it keeps both (`refused`: the status).
constexpr int kRefusedWord = 11;
constexpr int32_t kRefusedMark = 0x52534552;
__device__ __forceinline__ void write_flags(int32_t* ws, bool bad, int32_t before = 0, int32_t refused = kDevOk) {
    const int any = __syncthreads_or(bad);
    if (threadIdx.x == 0) {
        int32_t* mine = ws + kStatusBytes / 4 + blockIdx.x;
        *mine = (any || (before && *mine)) ? kDevBadIndex : kDevOk;
    }
    if (blockIdx.x == 0 && !before)
        for (int i = threadIdx.x; i < kStatusBytes / 4; i += blockDim.x)
            ws[i] = i == 0 ? refused : i == kFlagsWord ? (int32_t)gridDim.x : i == kRefusedWord && refused != kDevOk ? kRefusedMark : 0;
}

// ---- launchers -------------------------------------------------------------------------------------------------------------
size_t cache_page_list_bytes(const CacheView& c);        // scratch of the page calls behind the status head
cudaError_t launch_cache_reserve(const CacheView& c, const int32_t* n_new, int32_t* start, int32_t* ws, cudaStream_t st);
cudaError_t launch_cache_fork(const CacheView& c, const int32_t* src_of, bool share, int32_t* ws, cudaStream_t st);
cudaError_t launch_cache_release(const CacheView& c, const int32_t* drop, int32_t* ws, cudaStream_t st);
cudaError_t launch_cache_compact(const CacheView& c, int32_t* live_pages, int32_t* ws, cudaStream_t st);
cudaError_t launch_cache_append(const CacheView& c, int32_t L_new, const __nv_bfloat16* K, const __nv_bfloat16* V,
                                const __nv_bfloat16* g2, const __nv_bfloat16* kI, const int32_t* n_new, const int32_t* start,
                                int32_t* ws, cudaStream_t st);
cudaError_t launch_cache_read(const CacheView& c, int32_t L, __nv_bfloat16* K, __nv_bfloat16* V, __nv_bfloat16* kI,
                              int32_t* ws, cudaStream_t st);
cudaError_t launch_cache_indexer(const CacheView& c, const gsa_params_t& p, const __nv_bfloat16* qI, const float* w, const float* bI,
                                 float* scores, int64_t row_stride, int32_t* ws, cudaStream_t st);
size_t cache_attn_scratch_bytes(const gsa_params_t& p);
cudaError_t launch_cache_attn(const CacheView& c, const gsa_params_t& p, const __nv_bfloat16* Q, const __nv_bfloat16* g1,
                              const int32_t* idx, const int32_t* kt, __nv_bfloat16* out, int32_t* ws, cudaStream_t st);

}  // namespace gsa
