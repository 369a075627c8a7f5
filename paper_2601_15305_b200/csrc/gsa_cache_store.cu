// Tokens into the pages of a 4-bit cache and back out as contiguous bf16 (include/gsa.h states the format).
//
// One thread per 16 values (one scale) of K and of V' of a token: 32-byte loads, the codes leave as 8 bytes.  Both kernels stream:
// HBM bounds them (append: 6 bytes a value of K and V in, 1.1 out; read: 1.1 in, 4 out).
#include "gsa_cache.cuh"

namespace gsa {

namespace {

constexpr int kStoreThreads = 256;

struct Words8 { uint32_t v[8]; };               // sixteen bf16

__device__ __forceinline__ Words8 load32(const void* p) {
    Words8 w;
    asm volatile("ld.global.nc.L1::no_allocate.v8.u32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(w.v[0]), "=r"(w.v[1]), "=r"(w.v[2]), "=r"(w.v[3]), "=r"(w.v[4]), "=r"(w.v[5]), "=r"(w.v[6]), "=r"(w.v[7])
                 : "l"(p));
    return w;
}
__device__ __forceinline__ void store32(void* p, const Words8& w) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(w.v[0]), "r"(w.v[1]), "r"(w.v[2]), "r"(w.v[3]),
                 "r"(w.v[4]), "r"(w.v[5]), "r"(w.v[6]), "r"(w.v[7])
                 : "memory");
}

// ---- V' = bf16(fp32(V * sigmoid(g2))), the product rounded to fp32 correctly ------------------------------------------------
// The product is formed in fp32 from an exponential with its argument in two parts.  The sigmoid is then within 2 * 10^-7 of the true
// one (over all bf16 logits up to 80 in magnitude), 3.3 units of 2^-24, the product within another unit: at most five units of its
// last place, which kGateUlps doubles.  So only a product that close to the middle between two bf16 numbers -- one in 3100 -- can round
// to another bf16 number than the true one, and is formed again in 64 bits.
constexpr uint32_t kGateUlps = 10;

__device__ __noinline__ float gated_exact(float v, float g) { return (float)((double)v / (1.0 + exp(-(double)g))); }
__device__ __forceinline__ float gated(float v, float g) {
    constexpr float kHi = -1.44269502162933349609375f, kLo = -1.925963033500011e-08f;        // -log2(e) in two parts
    const float a = g * kHi;
    const float lo = fmaf(g, kLo, fmaf(g, kHi, -a));                                           // a + lo = -g log2(e)
    float e, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(a));
    e = fmaf(e, lo * 0.693147180559945f, e);
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + e));
    const float p = v * r;
    const uint32_t off = (__float_as_uint(p) & 0xFFFFu) - (0x8000u - kGateUlps);
    // (logits far out leave the range of the fast exponential, NaN comes out of both; a tiny product may have lost its last bits)
    if (off <= 2u * kGateUlps || !(fabsf(g) <= 80.f) || (fabsf(p) < 1e-30f && v != 0.f)) return gated_exact(v, g);
    return p;
}

__device__ __forceinline__ float lo_f(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// ---- 16 values to codes and a scale ----------------------------------------------------------------------------------------
__device__ __forceinline__ uint2 encode(const Words8& x, uint32_t& byte) {
    auto as2 = [](uint32_t w) { return *reinterpret_cast<const __nv_bfloat162*>(&w); };
    __nv_bfloat162 m = __habs2(as2(x.v[0]));
#pragma unroll
    for (int i = 1; i < 8; ++i) m = __hmax2_nan(m, __habs2(as2(x.v[i])));
    const float2 mf = __bfloat1622float2(m);
    const float amax = fmaxf(mf.x, mf.y);
    if (!(mf.x < INFINITY) || !(mf.y < INFINITY)) {          // an infinity or a NaN
        byte = kScaleNan;
        return make_uint2(0x88888888u, 0x88888888u);
    }
    // max / 7 is exact where it lies between two scales (7 * 17/16 .. of a power of two has at most 8 bits): halves go up as stated
    const int32_t n = (int32_t)((__float_as_uint(__fdiv_rn(amax, 7.0f)) + (1u << 19)) >> 20) - (int32_t)kScaleBias;
    byte = (uint32_t)min(max(n, 0), 254);
    const float s = __uint_as_float((byte + kScaleBias) << 20);
    float inv;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));
    const float limit = 7.0f * s;                            // (matters for the largest scale only: otherwise |x / s| < 7.5)
    // x / s has 8 bits over 4: what is not halfway between two integers is at least 2^-10 away from there, and x * inv is within
    // 2^-19 of x / s.  Adding 768 rounds it to a multiple of 2^-14, which restores the halves; the second sum rounds those to even
    // and leaves u = 8 + code in the last bits.
    auto code = [&](float v) -> uint32_t {
        const float t = fmaf(v, inv, 768.0f);
        return __float_as_uint(t + 12582152.0f) & 15u;
    };
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        w[h] = 0u;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float a = lo_f(x.v[h * 4 + i]), b = hi_f(x.v[h * 4 + i]);
            if (byte == 254u) {
                a = fminf(fmaxf(a, -limit), limit);
                b = fminf(fmaxf(b, -limit), limit);
            }
            w[h] |= code(a) << (8 * i) | code(b) << (8 * i + 4);
        }
    }
    return make_uint2(w[0], w[1]);
}

struct AppendArgs {
    CacheView c;
    const __nv_bfloat16 *K, *V, *g2, *kI;
    const int32_t *n_new, *start;
    int32_t* dev_status;
    int32_t L_new, log_groups;                   // groups of 16 values a token: a power of two
};

template <bool GATE>
__global__ void __launch_bounds__(kStoreThreads) gsa_cache_append_kernel(const AppendArgs a) {
    chain_wait();
    const int b = blockIdx.y, groups = 1 << a.log_groups;
    const int32_t in_seq = (int32_t)(blockIdx.x * kStoreThreads + threadIdx.x);              // (below 2^24 * 64)
    const int i = in_seq >> a.log_groups, g = in_seq & (groups - 1);
    if (i >= a.L_new) return;
    const int64_t token = (int64_t)b * a.L_new + i, item = (token << a.log_groups) + g;
    const int32_t first = a.start[b], n_new = a.n_new[b];
    if (first < 0) return;
    if (n_new > a.L_new && in_seq == 0) report_bad_index(a.dev_status);                      // (tokens that nobody gave)
    if (i >= n_new) return;
    const CacheView& c = a.c;
    const Words8 k = load32(a.K + item * 16);
    Words8 v = load32(a.V + item * 16), gate;
    if constexpr (GATE) gate = load32(a.g2 + item * 16);

    // where the token goes
    const int64_t s = (int64_t)first + i;
    const int32_t cap = c.max_pages << c.log_t;
    bool bad = false;
    if (s >= checked_len(c, b, cap, bad) || bad) { report_bad_index(a.dev_status); return; }
    const int32_t page = c.table[(int64_t)b * c.max_pages + (int32_t)(s >> c.log_t)];
    if ((uint32_t)page >= (uint32_t)c.n_pages || c.refs[page] != 1) { report_bad_index(a.dev_status); return; }
    const int32_t slot = (int32_t)s & (c.T - 1);
    unsigned char* base = c.pool + page * c.page_bytes;
    unsigned char* rec = base + (int64_t)slot * c.rec;
    const int D = c.n_kv * c.d_h;

    if constexpr (GATE) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            v.v[j] = pack_bf16(gated(lo_f(v.v[j]), lo_f(gate.v[j])), gated(hi_f(v.v[j]), hi_f(gate.v[j])));
    }
    uint32_t kb, vb;
    const uint2 kc = encode(k, kb), vc = encode(v, vb);
    *reinterpret_cast<uint2*>(rec + g * 8) = kc;
    *reinterpret_cast<uint2*>(rec + D / 2 + g * 8) = vc;
    const int per_head = c.d_h / kCacheGroup, head = g / per_head, in_head = g - head * per_head;
    unsigned char* sc = rec + D + head * 2 * per_head + in_head;
    sc[0] = (unsigned char)kb;
    sc[per_head] = (unsigned char)vb;
    for (int j = g; j < c.dI / 8; j += groups)
        reinterpret_cast<uint4*>(base + c.keys_off + (int64_t)slot * c.dI * 2)[j] = __ldg(reinterpret_cast<const uint4*>(a.kI + token * c.dI) + j);
}

struct ReadArgs {
    CacheView c;
    __nv_bfloat16 *K, *V, *kI;
    int32_t* dev_status;
    int32_t L, log_groups;
};

// sixteen codes and their scale to bf16: 128 + u by putting the code into the mantissa, then one multiply-add, exact because
// (128 + u) * s - 136 * s has at most seven significant bits and 136 * s at most eight (17 * 15 < 256)
__device__ __forceinline__ Words8 decode(uint2 codes, uint32_t byte) {
    const uint32_t s2 = byte == kScaleNan ? 0x7FFF7FFFu : byte * 0x00100010u + (kScaleBiasBf16 * 0x00010001u);
    const __nv_bfloat162 s = *reinterpret_cast<const __nv_bfloat162*>(&s2), z = __hmul2(s, __float2bfloat162_rn(-136.0f));
    Words8 o;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t w = h ? codes.y : codes.x;
        uint32_t p[4];                           // values (i, i + 4) of this half
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t u = ((w >> (4 * i)) & 0x000F000Fu) | 0x43004300u;
            const __nv_bfloat162 r = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&u), s, z);
            p[i] = *reinterpret_cast<const uint32_t*>(&r);
        }
        o.v[h * 4 + 0] = __byte_perm(p[0], p[1], 0x5410);
        o.v[h * 4 + 1] = __byte_perm(p[2], p[3], 0x5410);
        o.v[h * 4 + 2] = __byte_perm(p[0], p[1], 0x7632);
        o.v[h * 4 + 3] = __byte_perm(p[2], p[3], 0x7632);
    }
    return o;
}

__global__ void __launch_bounds__(kStoreThreads) gsa_cache_read_kernel(const ReadArgs a) {
    chain_wait();
    const CacheView& c = a.c;
    const int b = blockIdx.y, groups = 1 << a.log_groups;
    const int32_t in_seq = (int32_t)(blockIdx.x * kStoreThreads + threadIdx.x);
    const int s = in_seq >> a.log_groups, g = in_seq & (groups - 1);
    if (s >= a.L) return;
    const int64_t token = (int64_t)b * a.L + s, item = (token << a.log_groups) + g;
    bool bad = false;
    const int32_t len = checked_len(c, b, c.max_pages << c.log_t, bad);
    const int32_t page = s < len ? checked_page(c, b, s, bad) : 0, slot = s & (c.T - 1);
    if (bad) report_bad_index(a.dev_status);
    if (s >= len) return;
    const unsigned char* base = c.pool + page * c.page_bytes;
    const unsigned char* rec = base + (int64_t)slot * c.rec;
    const int D = c.n_kv * c.d_h, per_head = c.d_h / kCacheGroup, head = g / per_head;
    const unsigned char* sc = rec + D + head * 2 * per_head + (g - head * per_head);
    uint2 kc, vc;
    uint32_t kb, vb;
    if (a.K) { kc = __ldg(reinterpret_cast<const uint2*>(rec + g * 8)); kb = __ldg(sc); }
    if (a.V) { vc = __ldg(reinterpret_cast<const uint2*>(rec + D / 2 + g * 8)); vb = __ldg(sc + per_head); }
    if (a.K) store32(a.K + item * 16, decode(kc, kb));
    if (a.V) store32(a.V + item * 16, decode(vc, vb));
    if (a.kI)
        for (int j = g; j < c.dI / 8; j += groups)
            reinterpret_cast<uint4*>(a.kI + token * c.dI)[j] = __ldg(reinterpret_cast<const uint4*>(base + c.keys_off + (int64_t)slot * c.dI * 2) + j);
}

}  // namespace

static int log2_of(int v) { int n = 0; while ((1 << n) < v) ++n; return n; }

cudaError_t launch_cache_append(const CacheView& c, int32_t L_new, const __nv_bfloat16* K, const __nv_bfloat16* V,
                                const __nv_bfloat16* g2, const __nv_bfloat16* kI, const int32_t* n_new, const int32_t* start,
                                int32_t* dev_status, cudaStream_t st) {
    AppendArgs a{c, K, V, g2, kI, n_new, start, dev_status, L_new, log2_of(c.n_kv * c.d_h / kCacheGroup)};
    const dim3 grid((unsigned)((((int64_t)L_new << a.log_groups) + kStoreThreads - 1) / kStoreThreads), (unsigned)c.B);
    if (g2) launch_chained(gsa_cache_append_kernel<true>, grid, kStoreThreads, 0, st, a);
    else launch_chained(gsa_cache_append_kernel<false>, grid, kStoreThreads, 0, st, a);
    ++g_launches;
    return cudaGetLastError();
}

cudaError_t launch_cache_read(const CacheView& c, int32_t L, __nv_bfloat16* K, __nv_bfloat16* V, __nv_bfloat16* kI,
                              int32_t* dev_status, cudaStream_t st) {
    ReadArgs a{c, K, V, kI, dev_status, L, log2_of(c.n_kv * c.d_h / kCacheGroup)};
    const dim3 grid((unsigned)((((int64_t)L << a.log_groups) + kStoreThreads - 1) / kStoreThreads), (unsigned)c.B);
    launch_chained(gsa_cache_read_kernel, grid, kStoreThreads, 0, st, a);
    ++g_launches;
    return cudaGetLastError();
}

}  // namespace gsa
