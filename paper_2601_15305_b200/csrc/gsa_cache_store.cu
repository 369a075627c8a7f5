// Tokens into the pages of a 4-bit cache and back out as contiguous bf16 (include/gsa.h states the format).
//
// A warp takes a run of up to 32 tokens: each lane looks up where one of them lies, then the warp goes through their groups of 16 values
// (one scale each), a group of K and of V' a lane: 32-byte loads, the codes leave as 8 bytes.  The next groups are loaded while the
// present ones are worked on.  (With every thread looking up its own token the read kernel had 275 instructions a thread, the
// decoding being 70 of them; with a CTA doing it through shared memory its barriers cost as much.)
// Both kernels stream: HBM bounds them (append: 6 bytes a value of K and V in, 1.1 out; read: 1.1 in, 4 out), next to it, in the append,
// the sigmoids and the rounding.  8192 tokens of 8 KV heads of 128: append 18.4 us (62 MB: 3.4 TB/s; some 590 instructions for a lane's
// 48 values, 59 % of the cycles issue one; five, six or eight CTAs an SM without the loads ahead take 1 to 6 % longer), 12291 read
// back 13 us (67 MB, 5.2 TB/s).
#include "gsa_cache.cuh"

namespace gsa {

namespace {

constexpr int kStoreThreads = 128;
constexpr int kStoreWarps = kStoreThreads / 32;

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

__device__ __forceinline__ float lo_f(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ __nv_bfloat162 as_bf16x2(uint32_t w) { return *reinterpret_cast<const __nv_bfloat162*>(&w); }
// largest magnitude of sixteen bf16 in either half; NaN if one of them is
__device__ __forceinline__ float2 largest(const Words8& x) {
    __nv_bfloat162 m = __habs2(as_bf16x2(x.v[0]));
#pragma unroll
    for (int i = 1; i < 8; ++i) m = __hmax2_nan(m, __habs2(as_bf16x2(x.v[i])));
    return __bfloat1622float2(m);
}

// ---- V' = bf16(fp32(V * sigmoid(g2))), the product rounded to fp32 correctly ------------------------------------------------
// The fast product: -log2(e) in two parts, the first of 16 bits, so that its product with a bf16 logit is exact and the second one's is
// small enough for a linear correction.  Over all bf16 logits up to 40 in magnitude the sigmoid is then within 1.72 * 10^-7 of the true
// one, 2.9 units of 2^-24, the product within one more: less than four units of its last place.  Only a product within kGateUlps units of
// the middle between two bf16 numbers -- one in 4000 at the seven to nine that the test on two at a time makes of it -- can round to another
// bf16 number than the true one, and is formed again in 64 bits.
constexpr uint32_t kGateUlps = 8;
constexpr float kGateRange = 40.f;

__device__ __noinline__ float gated_exact(float v, float g) { return (float)((double)v / (1.0 + exp(-(double)g))); }
__device__ __forceinline__ float gated_fast(float v, float g) {
    constexpr float kHi = -1.44268798828125f;                                      // 16 bits of -log2(e)
    constexpr float kLo = (float)((-1.4426950408889634074 + 1.44268798828125) * 0.69314718055994530942);         // the rest, times ln 2
    float e, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(g * kHi));
    e = fmaf(e, g * kLo, e);
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + e));
    return v * r;
}
// bits 15 and 31: whether the low halves of two products' bits lie within about kGateUlps of 0x8000.  (Two at a time: the sum's carry
// from one half into the other moves that one's limits by one.)
__device__ __forceinline__ uint32_t near_half(float a, float b) {
    static_assert(kGateUlps == 8, "the masks below");
    const uint32_t y = __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x5410) + 0x00080008u;
    const uint32_t z = (y & 0xFFF0FFF0u) ^ 0x80008000u;                            // a zero half: within
    return (z - 0x00010001u) & ~z & 0x80008000u;
}
__device__ __noinline__ uint32_t gated_exact_pair(uint32_t v, uint32_t g) {
    return pack_bf16(gated_exact(lo_f(v), lo_f(g)), gated_exact(hi_f(v), hi_f(g)));
}
__device__ __forceinline__ void gate_values(Words8& v, const Words8& gate) {
    const float2 top = largest(gate);
    uint32_t out[8], doubt = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float a = gated_fast(lo_f(v.v[i]), lo_f(gate.v[i])), b = gated_fast(hi_f(v.v[i]), hi_f(gate.v[i]));
        doubt |= near_half(a, b) >> i;           // (bits 15 - i and 31 - i)
        out[i] = pack_bf16(a, b);
    }
    if (!(top.x <= kGateRange) || !(top.y <= kGateRange)) doubt = 0xFFFFFFFFu;     // (logits far out, or NaN)
    if (doubt) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (doubt & (0x80008000u >> i)) out[i] = gated_exact_pair(v.v[i], gate.v[i]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v.v[i] = out[i];
}

// ---- 16 values to codes and a scale ----------------------------------------------------------------------------------------
__device__ __forceinline__ uint2 encode(Words8 x, uint32_t& byte) {
    const float2 m = largest(x);
    if (!(m.x < INFINITY) || !(m.y < INFINITY)) {            // an infinity or a NaN
        byte = kScaleNan;
        return make_uint2(0x88888888u, 0x88888888u);
    }
    // max / 7 to the nearest scale, halves up.  Seven times the middle between two scales has at most eight bits, so a maximum that is not
    // one of those middles is at least 2^-8 away from it: a factor 1 + 2^-12 puts the middles themselves on the upper side, whatever the
    // product's rounding, and moves nothing else across.
    const int32_t n = (int32_t)((__float_as_uint(fmaxf(m.x, m.y) * (float)(1.000244140625 / 7.0)) + (1u << 19)) >> 20) - (int32_t)kScaleBias;
    byte = (uint32_t)min(max(n, 0), 254);
    const float s = __uint_as_float((byte + kScaleBias) << 20);
    float inv;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));
    if (byte == 254u) {                                      // the largest scale: values may exceed seven times it (25088, exact in bf16)
        const __nv_bfloat162 top = __float2bfloat162_rn(7.0f * s), bottom = __hneg2(top);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const __nv_bfloat162 c = __hmin2(__hmax2(as_bf16x2(x.v[i]), bottom), top);
            x.v[i] = *reinterpret_cast<const uint32_t*>(&c);
        }
    }
    // x / s has 8 bits over 4: what is not halfway between two integers is at least 2^-10 away from there, and x * inv is within
    // 2^-19 of x / s.  Adding 768 rounds it to a multiple of 2^-14, which restores the halves; the second sum rounds those to even
    // and leaves u = 8 + code in the last byte (of 12582912 + u).
    auto code = [&](float v) -> uint32_t { return __float_as_uint(fmaf(v, inv, 768.0f) + 12582152.0f); };
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) b[i] = code(lo_f(x.v[h * 4 + i])) + code(hi_f(x.v[h * 4 + i])) * 16u;        // last byte: both codes
        w[h] = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
    }
    return make_uint2(w[0], w[1]);
}

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

// ---- the kernels -----------------------------------------------------------------------------------------------------------
struct StoreArgs {
    CacheView c;
    __nv_bfloat16 *K, *V, *kI;                   // append reads them, read writes them (any may be null there)
    const __nv_bfloat16* g2;
    const int32_t *n_new, *start;
    int32_t* ws;
    int32_t L, log_groups, rounds;               // rows a sequence; groups of 16 values a token, a power of two; groups of a run: 32 * rounds
    int64_t runs, tokens;                        // tokens: B * L
};

// A token of a run: whether it takes part (its row may then be read), and where its record and its k^I lie, bytes from the pool's start,
// -1 for one that is left out.  In two steps, so that the rows are on their way while the tables are read.
struct Token {
    int b;
    int32_t s;                                   // position in the sequence
    bool wanted;
    int64_t rec, key;
};
template <bool APPEND>
__device__ __forceinline__ Token want_token(const StoreArgs& a, int64_t token, bool& bad) {
    Token t{0, 0, false, -1, 0};
    if (token >= a.tokens) return t;
    t.b = token <= 0xFFFFFFFFll ? (int)((uint32_t)token / (uint32_t)a.L) : (int)(token / a.L);
    t.s = (int)(token - (int64_t)t.b * a.L);
    t.wanted = true;
    if constexpr (APPEND) {
        const int32_t start = __ldg(a.start + t.b), n_new = __ldg(a.n_new + t.b), cap = a.c.max_pages << a.c.log_t;
        t.wanted = start >= 0 && t.s < n_new;
        bad |= start >= 0 && n_new > a.L;        // (tokens that nobody gave)
        if (t.wanted && start >= cap - t.s) {    // (behind the table's end)
            t.wanted = false;
            bad = true;
        }
        t.s += t.wanted ? start : 0;
    }
    return t;
}
template <bool APPEND>
__device__ __forceinline__ void find_token(const StoreArgs& a, Token& t, bool& bad) {
    const CacheView& c = a.c;
    if (!t.wanted) return;
    const int32_t cap = c.max_pages << c.log_t, len = __ldg(c.lens + t.b);
    int32_t page = __ldg(c.table + (int64_t)t.b * c.max_pages + (t.s >> c.log_t));
    bad |= len < 0 || len > cap;
    if (t.s >= len) {
        bad |= APPEND;
        return;
    }
    const bool named = (uint32_t)page < (uint32_t)c.n_pages;
    bad |= !named;
    if constexpr (APPEND) {
        if (!named) return;
        if (__ldg(c.refs + page) != 1) {
            bad = true;
            return;
        }
    } else if (!named) {
        page = 0;
    }
    const int64_t base = (int64_t)page * c.page_bytes;
    const int32_t slot = t.s & (c.T - 1);
    t.rec = base + slot * c.rec;
    t.key = base + c.keys_off + slot * c.dI * 2;
}
// Calls copy(pool offset, row of k^I, 16-byte piece) for the k^I of the tokens whose first group the run has.
template <class F>
__device__ __forceinline__ void each_key_piece(const StoreArgs& a, const Token& mine, int64_t item0, int64_t token0, F copy) {
    const int lane = threadIdx.x & 31, groups = 1 << a.log_groups, log_pieces = a.c.dI == 64 ? 3 : 2;
    const int n = (int)(((item0 + a.rounds * 32 + groups - 1) >> a.log_groups) - ((item0 + groups - 1) >> a.log_groups));
    const int skip = (item0 & (groups - 1)) ? 1 : 0;
    for (int i = lane; i < ((n << log_pieces) + 31) / 32 * 32; i += 32) {
        const int t = skip + (i >> log_pieces);
        const int64_t rec = __shfl_sync(0xFFFFFFFFu, mine.rec, t & 31), key = __shfl_sync(0xFFFFFFFFu, mine.key, t & 31);
        if (i < n << log_pieces && rec >= 0) copy(key, token0 + t, i & ((1 << log_pieces) - 1));
    }
}

// What the first CTA of an append has to keep in the head: the status of a reservation that was refused, if tokens were given that it left
// without a place.  (The mark alone does not tell: the caller may have made places of its own since, or given nothing.)
__device__ __forceinline__ int32_t refused_status(const StoreArgs& a) {
    const int32_t status = a.ws[0];
    bool lost = false;
    for (int b = threadIdx.x; b < a.c.B; b += kStoreThreads) lost |= __ldg(a.start + b) < 0 && __ldg(a.n_new + b) > 0;
    return __syncthreads_or(lost) && (status == kDevCacheFull || status == kDevBadIndex) ? status : kDevOk;
}

template <bool GATE>
__global__ void __launch_bounds__(kStoreThreads, 4) gsa_cache_append_kernel(const StoreArgs a) {
    chain_wait();
    const CacheView& c = a.c;
    const int32_t mark = blockIdx.x == 0 ? a.ws[kRefusedWord] : 0;
    const int lane = threadIdx.x & 31;
    const int D = c.n_kv * c.d_h, log_head = c.d_h == 128 ? 3 : 2, groups = 1 << a.log_groups;       // groups of a head: 8 or 4
    bool bad = false;
    for (int64_t run = (int64_t)blockIdx.x * kStoreWarps + (threadIdx.x >> 5); run < a.runs; run += (int64_t)gridDim.x * kStoreWarps) {
        const int64_t item0 = run * (a.rounds * 32), token0 = item0 >> a.log_groups;
        const int in_token = (int)(item0 & (groups - 1)) + lane;                   // group, counted from the run's first token on
        Token mine = want_token<true>(a, token0 + lane, bad);
        const uint32_t wanted = __ballot_sync(0xFFFFFFFFu, mine.wanted);
        struct { Words8 k, v, g; } in, next;
        auto load = [&](int round, decltype(in)& x) {
            if ((wanted >> ((in_token + round * 32) >> a.log_groups)) & 1u) {
                const int64_t at = (item0 + round * 32 + lane) * 16;
                x.k = load32(a.K + at);
                x.v = load32(a.V + at);
                if constexpr (GATE) x.g = load32(a.g2 + at);
            }
        };
        load(0, in);
        find_token<true>(a, mine, bad);
        for (int round = 0; round < a.rounds; ++round) {
            if (round + 1 < a.rounds) load(round + 1, next);
            const int64_t at = __shfl_sync(0xFFFFFFFFu, mine.rec, (in_token + round * 32) >> a.log_groups);
            if (at >= 0) {
                const int g = (in_token + round * 32) & (groups - 1);
                unsigned char* rec = c.pool + at;
                unsigned char* sc = rec + D + ((g >> log_head) << (log_head + 1)) + (g & ((1 << log_head) - 1));
                uint32_t byte;
                *reinterpret_cast<uint2*>(rec + g * 8) = encode(in.k, byte);
                sc[0] = (unsigned char)byte;
                if constexpr (GATE) gate_values(in.v, in.g);
                *reinterpret_cast<uint2*>(rec + D / 2 + g * 8) = encode(in.v, byte);
                sc[1 << log_head] = (unsigned char)byte;
            }
            in = next;
        }
        each_key_piece(a, mine, item0, token0, [&](int64_t key, int64_t token, int j) {
            reinterpret_cast<uint4*>(c.pool + key)[j] = __ldg(reinterpret_cast<const uint4*>(a.kI + token * c.dI) + j);
        });
    }
    write_flags(a.ws, bad, 0, mark == kRefusedMark ? refused_status(a) : kDevOk);
}

__global__ void __launch_bounds__(kStoreThreads, 8) gsa_cache_read_kernel(const StoreArgs a) {
    chain_wait();
    const CacheView& c = a.c;
    const int lane = threadIdx.x & 31;
    const int D = c.n_kv * c.d_h, log_head = c.d_h == 128 ? 3 : 2, groups = 1 << a.log_groups;
    bool bad = false;
    for (int64_t run = (int64_t)blockIdx.x * kStoreWarps + (threadIdx.x >> 5); run < a.runs; run += (int64_t)gridDim.x * kStoreWarps) {
        const int64_t item0 = run * (a.rounds * 32), token0 = item0 >> a.log_groups;
        const int in_token = (int)(item0 & (groups - 1)) + lane;
        Token mine = want_token<false>(a, token0 + lane, bad);
        find_token<false>(a, mine, bad);
        struct { uint2 k, v; uint32_t kb, vb; bool real; } in, next;
        auto load = [&](int round, decltype(in)& x) {
            const int64_t at = __shfl_sync(0xFFFFFFFFu, mine.rec, (in_token + round * 32) >> a.log_groups);
            x.real = at >= 0;
            if (x.real) {
                const int g = (in_token + round * 32) & (groups - 1);
                const unsigned char* rec = c.pool + at;
                const unsigned char* sc = rec + D + ((g >> log_head) << (log_head + 1)) + (g & ((1 << log_head) - 1));
                x.k = __ldg(reinterpret_cast<const uint2*>(rec + g * 8)); x.kb = __ldg(sc);
                x.v = __ldg(reinterpret_cast<const uint2*>(rec + D / 2 + g * 8)); x.vb = __ldg(sc + (1 << log_head));
            }
        };
        if (a.K || a.V) {
            load(0, in);
            for (int round = 0; round < a.rounds; ++round) {
                if (round + 1 < a.rounds) load(round + 1, next);
                if (in.real) {
                    const int64_t to = (item0 + round * 32 + lane) * 16;
                    if (a.K) store32(a.K + to, decode(in.k, in.kb));
                    if (a.V) store32(a.V + to, decode(in.v, in.vb));
                }
                in = next;
            }
        }
        if (a.kI)
            each_key_piece(a, mine, item0, token0, [&](int64_t key, int64_t token, int j) {
                reinterpret_cast<uint4*>(a.kI + token * c.dI)[j] = __ldg(reinterpret_cast<const uint4*>(c.pool + key) + j);
            });
    }
    write_flags(a.ws, bad);
}

int log2_of(int v) { int n = 0; while ((1 << n) < v) ++n; return n; }

// `warps`: how many an SM holds.  One wave of runs if rounds (at most eight, 31 whole tokens) allow: 8192 tokens in 1.7 waves of four rounds
// took 22.3 us, in one of seven 18.9.
StoreArgs store_args(const CacheView& c, int32_t L, int32_t* ws, int warps, unsigned* ctas) {
    StoreArgs a{};
    a.c = c; a.ws = ws; a.L = L; a.log_groups = log2_of(c.n_kv * c.d_h / kCacheGroup); a.tokens = (int64_t)c.B * L;
    const int64_t items = a.tokens << a.log_groups, wave = (int64_t)sm_count() * warps * 32;
    const int64_t cap = (31 << a.log_groups) / 32 < 8 ? (31 << a.log_groups) / 32 : 8, rounds = (items + wave - 1) / wave;
    a.rounds = (int32_t)(rounds < cap ? rounds : cap);
    a.runs = (items + 32 * a.rounds - 1) / (32 * a.rounds);
    const int64_t want = (a.runs + kStoreWarps - 1) / kStoreWarps;
    *ctas = (unsigned)(want < kMaxFlags ? want : kMaxFlags);
    return a;
}

}  // namespace

cudaError_t launch_cache_append(const CacheView& c, int32_t L_new, const __nv_bfloat16* K, const __nv_bfloat16* V,
                                const __nv_bfloat16* g2, const __nv_bfloat16* kI, const int32_t* n_new, const int32_t* start,
                                int32_t* ws, cudaStream_t st) {
    unsigned ctas;
    StoreArgs a = store_args(c, L_new, ws, 16, &ctas);
    a.K = const_cast<__nv_bfloat16*>(K); a.V = const_cast<__nv_bfloat16*>(V); a.kI = const_cast<__nv_bfloat16*>(kI);
    a.g2 = g2; a.n_new = n_new; a.start = start;
    cudaError_t e = g2 ? launch_chained(gsa_cache_append_kernel<true>, ctas, kStoreThreads, 0, st, a)
                       : launch_chained(gsa_cache_append_kernel<false>, ctas, kStoreThreads, 0, st, a);
    ++g_launches;
    return e != cudaSuccess ? e : cudaGetLastError();
}

cudaError_t launch_cache_read(const CacheView& c, int32_t L, __nv_bfloat16* K, __nv_bfloat16* V, __nv_bfloat16* kI,
                              int32_t* ws, cudaStream_t st) {
    unsigned ctas;
    StoreArgs a = store_args(c, L, ws, 32, &ctas);
    a.K = K; a.V = V; a.kI = kI;
    cudaError_t e = launch_chained(gsa_cache_read_kernel, ctas, kStoreThreads, 0, st, a);
    ++g_launches;
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace gsa
