// Sparse gated attention (Eq. 11, 12, 10) over index sets whose K and V' lie in the pages of a 4-bit cache (include/gsa.h).
//
// A set is walked in tiles of 16 keys; n_kv warps (a unit) take a tile together, one KV head each.  As in gsa_attn.cu keys are the
// M side of an MMA and the group's query heads its N side, and a contraction does not care about the order of its index, so a lane takes
// the codes that lie together in memory:
//   K   lane (gid, tig): the tig-th quarter of the head row of keys gid and gid + 8, eight codes a word; Q is read with the same
//       permutation.                                                               S^T[key, head] = K[key, :] . Q[head, :]
//   V'  lane (gid, tig): the gid-th eighth of keys 2 tig, 2 tig + 1, 2 tig + 8, 2 tig + 9; words of two keys are joined half by half, so
//       that a code position yields the pair (key, key + 1) of one d.                O^T[d, head] += V'^T[d, key] P^T[key, head]
//       At d_h = 128 that eighth is one group of 16 and has one scale.
//   dequantising K  one logical operation puts a code into the mantissa of 128 (bf16), one multiply-add by (s, -136 s) gives code * s,
//       exactly: (128 + u) s - 136 s has at most seven significant bits, 136 s at most eight.
//   dequantising V'  in fp16, whose longer mantissa takes codes at two places of a half word without a shift: (1024 + u) - 1032 or
//       (1024 + 16 u) / 16 - 72, then times s.  Every value of the format is exact in fp16 too (105 * 2^-23 .. 7 * 3584).
// The tile's numerators are rounded to fp16 for the second product.  They are taken against a reference that leaves a row's largest
// between 2^7 and 2^15, so that rounding is at most 2^-11 of a numerator, or 2^-25 where that is less than fp16's normal range goes down
// to: 2^-32 of the row's sum.  (In bf16, 2^-8 of each, the error of the 32 x 128K case against 64 bits is 2.3e-3; with fp16 it is
// 1.7e-3, the output's own rounding.)  Statistics, scores and sums are fp32.
//
// Records come by asynchronous copies into a ring of kStages tiles a warp (2304 bytes each at d_h = 128), so that some 100 KB of an SM
// are in flight; indices are read two tiles ahead of that, pages one.
//
// Work split: the tiles of all rows, one after another, are dealt to the units in equal runs, whatever the sets' sizes (each CTA sums
// up the budgets for itself).  A row that lies within one unit's run is finished there; the others' parts (at most two a unit) go to
// the workspace as softmax state and are merged by a second kernel, in order, so that nothing depends on scheduling.  With more rows than
// kMaxSplitRows a unit takes whole rows in turn instead.
#include "gsa_cache.cuh"

#include <cuda_fp16.h>

namespace gsa {

namespace {

constexpr int kWarps = 8;
constexpr int kTile = 16;                  // keys
constexpr int kStages = 4;                 // tiles of a warp's ring: one being computed on, the others in flight
constexpr int kMinTiles = 2;               // fewest tiles worth a unit of their own
constexpr int kMaxSplitRows = 2048;        // rows whose budgets a CTA sums up (16 KB of its shared memory)
constexpr int kCtasPerSm = 2;
constexpr int kMergeWarps = 8;
constexpr float kRefUnder = 7.0f;          // a new softmax reference lies 2^7 under the score that moved it there,
constexpr float kRefSlack = 15.0f;         // and moves again when a score lies 2^15 above it (fp16 ends at 2^16)

struct CacheAttnArgs {
    CacheView c;
    const __nv_bfloat16 *Q, *g1;
    const int32_t *idx, *kt;
    __nv_bfloat16* out;
    int32_t rows, Lq, Lk, n_h, k_max;
    float scale_log2;
    int32_t units;                         // of the launch; as many as there are tiles for take part
    float* state;                          // [2 * units][n_h][d_h] numerators
    float2* stats;                         // [2 * units][n_h] reference, sum
    int32_t* cum;                          // [rows + 1] tiles in front of each row, written for the merge
    int32_t* flags;                        // [CTAs] whether one met something out of range
    int32_t* status;                       // head of the workspace
};

// units that share `tiles` tiles; unit u has tiles first_tile(u) .. first_tile(u + 1) - 1
__host__ __device__ __forceinline__ int32_t units_for(int64_t tiles, int32_t units) {
    const int64_t most = (tiles + kMinTiles - 1) / kMinTiles;
    return (int32_t)(most < units ? most : units);
}
__device__ __forceinline__ int32_t div_small(int64_t a, int32_t b) {          // a / b, by a 32-bit division where that does
    return a <= 0xFFFFFFFFll ? (int32_t)((uint32_t)a / (uint32_t)b) : (int32_t)(a / b);
}
__device__ __forceinline__ int32_t first_tile(int32_t u, int32_t tiles, int32_t units) { return div_small((int64_t)u * tiles, units); }
__device__ __forceinline__ int32_t unit_of(int32_t tile, int32_t tiles, int32_t units) { return div_small(((int64_t)tile + 1) * units - 1, tiles); }
// A unit keeps its part of a row that starts in front of its run, or with it, in slot 2 u, one that starts inside it in 2 u + 1.

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t transposed(uint32_t a) {
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}
__device__ __forceinline__ void mma_f16_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <int W>
__device__ __forceinline__ void lds_words(uint32_t (&v)[W], uint32_t p) {
    static_assert(W == 1 || W == 2 || W == 4, "4, 8 or 16 bytes");
    if constexpr (W == 4)
        asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(p));
    else if constexpr (W == 2)
        asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v[0]), "=r"(v[1]) : "r"(p));
    else
        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v[0]) : "r"(p));
}
template <int BYTES>
__device__ __forceinline__ uint32_t lds_small(uint32_t p) {
    uint32_t v;
    if constexpr (BYTES == 2) asm volatile("{ .reg .u16 t; ld.shared.u16 t, [%1]; cvt.u32.u16 %0, t; }" : "=r"(v) : "r"(p));
    else asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(p));
    return v;
}
template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t dst, const unsigned char* src) {
    if constexpr (BYTES == 16) cp_async16(dst, src);
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 8;\n" ::"r"(dst), "l"(src));
}
__device__ __forceinline__ uint32_t fma_bf16x2(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t d;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
__device__ __forceinline__ uint32_t fma_f16x2(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t d;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
__device__ __forceinline__ uint32_t add_f16x2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("add.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    uint32_t d;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
// K: codes i and i + 4 of a word as 128 + u
__device__ __forceinline__ uint32_t code_pair(uint32_t w, int i) { return ((w >> (4 * i)) & 0x000F000Fu) | 0x43004300u; }
// a scale byte twice as bf16, and -136 times that
__device__ __forceinline__ uint32_t scale_bf16x2(uint32_t n) { return n == kScaleNan ? 0x7FFF7FFFu : n * 0x00100010u + kScaleBiasBf16 * 0x00010001u; }
__device__ __forceinline__ uint32_t zero_bf16x2(uint32_t s) {
    uint32_t z;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(z) : "r"(s), "r"(0xC308C308u));
    return z;
}
__device__ __forceinline__ float scale_f32(uint32_t n) { return n == kScaleNan ? __uint_as_float(0x7FFFFFFFu) : __uint_as_float((n + kScaleBias) << 20); }
// V': the four codes of a joined half word (two keys) times the keys' scales
__device__ __forceinline__ void values_f16x2(uint32_t (&v)[4], uint32_t m, uint32_t s) {
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
        const uint32_t x = i ? m >> 8 : m;
        v[i] = mul_f16x2(add_f16x2((x & 0x000F000Fu) | 0x64006400u, 0xE408E408u), s);                        // (1024 + u) - 1032
        v[i + 1] = mul_f16x2(fma_f16x2((x & 0x00F000F0u) | 0x64006400u, 0x2C002C00u, 0xD480D480u), s);       // (1024 + 16 u) / 16 - 72
    }
}

// N results of one head, gated and rounded
template <int N>
__device__ __forceinline__ void write_gated(const CacheAttnArgs& a, int64_t at, const float (&o)[N]) {
    const uint4* g = reinterpret_cast<const uint4*>(a.g1 + at);
    uint4* to = reinterpret_cast<uint4*>(a.out + at);
#pragma unroll
    for (int i = 0; i < N / 8; ++i) {
        const uint4 gv = __ldg(g + i);
        const uint32_t gw[4] = {gv.x, gv.y, gv.z, gv.w};
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            w[j] = pack_bf16(o[i * 8 + 2 * j] * fast_sigmoid(__uint_as_float(gw[j] << 16)),
                             o[i * 8 + 2 * j + 1] * fast_sigmoid(__uint_as_float(gw[j] & 0xFFFF0000u)));
        to[i] = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// one stage of a warp's ring: [16 keys][K codes], [16 keys][V' codes, padded: the lanes of a word-wide read then meet all banks],
// [16 keys][scales of K, of V']
template <int DH>
struct Stage {
    static constexpr int kRow = DH / 2, kVRow = DH / 2 + 16, kSRow = DH / 8;
    static constexpr int kV = kTile * kRow, kS = kV + kTile * kVRow, kBytes = kS + kTile * kSRow;
};
__host__ __device__ constexpr size_t row_table_bytes(int rows) { return ((size_t)(2 * rows + 1) * 4 + 15) / 16 * 16; }

template <int DH, int G, bool SPLIT>
__global__ void __launch_bounds__(kWarps * 32, kCtasPerSm) gsa_cache_attn_kernel(const CacheAttnArgs a) {
    chain_wait();
    using St = Stage<DH>;
    constexpr int KW = DH / 32;            // words of K codes a lane has of a key
    constexpr int VW = DH / 64;            // words of V' codes a lane has of a key
    constexpr int KS = DH / 64;            // scale bytes of those K codes
    constexpr int MT = DH / 16;
    constexpr int DL = DH / 8;             // consecutive d of O that a lane holds, for heads 2 tig and 2 tig + 1
    constexpr int CPK = DH / 32, KPI = 32 / CPK;       // 16-byte chunks of a key's codes, keys that one copy of a warp covers
    extern __shared__ __align__(16) unsigned char smem[];  // SPLIT: cum[rows + 1], budget[rows]; the rings
    __shared__ int32_t warp_sum[kWarps];
    __shared__ int32_t cta_bad;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int gid = lane >> 2, tig = lane & 3;
    const CacheView& c = a.c;
    const int n_kv = c.n_kv, subs = kWarps / n_kv;
    const int h = warp & (n_kv - 1);
    const int unit = (warp / n_kv) * gridDim.x + blockIdx.x;
    int32_t* cum = reinterpret_cast<int32_t*>(smem);
    int32_t* budget = cum + a.rows + 1;
    const uint32_t ring = smem_u32(smem) + (SPLIT ? (uint32_t)row_table_bytes(a.rows) : 0u) + warp * (kStages * St::kBytes);
    bool bad = false;
    auto budget_of = [&](int32_t row) -> int32_t {
        const int32_t k = __ldg(a.kt + row);
        bad |= k < 0 || k > a.k_max;
        return clamp_budget(k, a.k_max);
    };
    if (threadIdx.x == 0) cta_bad = 0;

    int32_t tiles = 0, units = gridDim.x * subs;
    if constexpr (SPLIT) {
        // ---- tiles in front of every row ----
        const int per = (a.rows + kWarps * 32 - 1) / (kWarps * 32), r0 = min(a.rows, (int)threadIdx.x * per), r1 = min(a.rows, r0 + per);
        int32_t mine = 0;
        for (int r = r0; r < r1; ++r) {
            const int32_t k = budget_of(r);
            budget[r] = k;
            mine += (k + kTile - 1) / kTile;
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
            tiles += warp_sum[w];
        }
        for (int r = r0; r < r1; ++r) {
            cum[r] = at;
            at += (budget[r] + kTile - 1) / kTile;
        }
        if (threadIdx.x == 0) cum[a.rows] = tiles;
        units = units_for(tiles, units);
    }
    __syncthreads();
    int32_t lo = 0, hi = 0;                // SPLIT: this unit's tiles
    bool works = true;
    if constexpr (SPLIT) {
        works = unit < units;
        if (works) {
            lo = first_tile(unit, tiles, units);
            hi = first_tile(unit + 1, tiles, units);
        }
    }

    // ---- cursors over the unit's tiles: (row, tile of the row, tiles and keys of the row) ----
    struct Cursor { int32_t row, j, n, k; };
    auto open_row = [&](Cursor& q, int32_t row) {          // the first row from `row` on that this unit works on and whose set is not empty
        if constexpr (SPLIT) {
            while (row < a.rows && budget[row] == 0) ++row;
            q.row = row;
            q.k = row < a.rows ? budget[row] : 0;
        } else {
            q.k = 0;
            while (row < a.rows && (q.k = budget_of(row)) == 0) {
                // (an empty set: this unit's warp writes its heads' zeros)
                for (int i = lane; i < G * DH / 8; i += 32)
                    reinterpret_cast<uint4*>(a.out + ((int64_t)row * a.n_h + h * G) * DH)[i] = make_uint4(0u, 0u, 0u, 0u);
                row += units;
            }
            q.row = row;
        }
        q.n = (q.k + kTile - 1) / kTile;
        q.j = 0;
    };
    auto advance = [&](Cursor& q) { if (++q.j >= q.n) open_row(q, q.row + (SPLIT ? 1 : units)); };
    Cursor ahead{};                        // the tile whose indices are read next
    int32_t left = 0;                      // SPLIT: tiles that `ahead` has still to hand out
    if constexpr (SPLIT) {
        if (works) {
            int32_t rl = 0, rh = a.rows - 1;       // the row that holds tile lo (of rows that start there the last: the others are empty)
            while (rl < rh) {
                const int32_t m = (rl + rh + 1) >> 1;
                if (cum[m] <= lo) rl = m; else rh = m - 1;
            }
            ahead.row = rl; ahead.k = budget[rl]; ahead.n = (ahead.k + kTile - 1) / kTile; ahead.j = lo - cum[rl];
            left = hi - lo;
        }
    } else {
        open_row(ahead, unit);
    }
    Cursor cur = ahead;

    // ---- what is in flight: indices (lane & 15), then pages, then records ----
    struct Pos { int32_t raw, n, b, len; };                // n: keys of the tile, 0: no tile
    struct Token { int32_t page, pos, n; };
    int32_t row_b = 0, row_len = 0, row_seen = -1;
    auto next_indices = [&]() -> Pos {
        Pos f{0, 0, 0, 0};
        if (SPLIT ? left <= 0 : ahead.row >= a.rows) return f;
        if (ahead.row != row_seen) {
            row_seen = ahead.row;
            row_b = ahead.row / a.Lq;
            row_len = checked_len(c, row_b, a.Lk, bad);
        }
        f.b = row_b; f.len = row_len;
        f.n = min(kTile, ahead.k - ahead.j * kTile);
        const int j = lane & 15;
        if (j < f.n) f.raw = __ldg(a.idx + (int64_t)ahead.row * a.k_max + ahead.j * kTile + j);
        --left;
        advance(ahead);
        return f;
    };
    auto find_pages = [&](const Pos& f) -> Token {
        Token t{0, 0, f.n};
        if (f.n == 0) return t;
        const int32_t first = __shfl_sync(0xFFFFFFFFu, f.raw, 0);
        t.pos = (lane & 15) < f.n ? f.raw : first;         // places behind the set's end read one of its keys again (P = 0 there)
        if ((uint32_t)t.pos >= (uint32_t)f.len) {
            bad = true;
            t.pos = min(max(t.pos, 0), max(f.len - 1, 0));
        }
        t.page = checked_page(c, f.b, t.pos, bad);
        return t;
    };
    const int D = n_kv * DH;
    const int ckey = lane / CPK, cpiece = lane % CPK;
    const unsigned char* const from_codes = c.pool + h * (DH / 2) + cpiece * 16;
    const unsigned char* const from_scales = c.pool + D + h * (DH / 8);
    const uint32_t to_k = ring + ckey * St::kRow + cpiece * 16, to_v = ring + St::kV + ckey * St::kVRow + cpiece * 16;
    const uint32_t to_s = ring + St::kS + (lane & 15) * St::kSRow;
    int32_t issued = 0;
    auto issue = [&](const Token& t, uint32_t stage) {
        if (t.n) {
            const int64_t at = (int64_t)t.page * c.page_bytes + (int64_t)(t.pos & (c.T - 1)) * c.rec;
            const uint32_t off = stage * St::kBytes;
#pragma unroll
            for (int i = 0; i < kTile / KPI; ++i) {
                const int64_t key_at = __shfl_sync(0xFFFFFFFFu, at, ckey + i * KPI);
                cp_async16(to_k + off + i * KPI * St::kRow, from_codes + key_at);
                cp_async16(to_v + off + i * KPI * St::kVRow, from_codes + key_at + D / 2);
            }
            if (lane < kTile) copy_async<St::kSRow>(to_s + off, from_scales + at);
            ++issued;
        }
        cp_async_commit();                 // (one group a tile, possibly empty)
    };

    Pos ahead_pos;
    Token ahead_token;
    {
        Pos f[kStages];
#pragma unroll
        for (int i = 0; i < kStages; ++i) f[i] = works ? next_indices() : Pos{0, 0, 0, 0};
        Token t[kStages];
#pragma unroll
        for (int i = 0; i < kStages; ++i) t[i] = find_pages(f[i]);
        ahead_pos = works ? next_indices() : Pos{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i + 1 < kStages; ++i) issue(t[i], i);
        ahead_token = t[kStages - 1];
    }

    uint32_t qf[KW][4];
    float o[MT][4], m_run[2], l_run[2];
    bool fresh = true;
    for (int32_t i = 0; i < issued; ++i) {
        if (fresh) {
            fresh = false;
            const bool real = gid < G;
            const __nv_bfloat16* qp = a.Q + ((int64_t)cur.row * a.n_h + h * G + (real ? gid : 0)) * DH + tig * (DH / 4);
#pragma unroll
            for (int w = 0; w < KW; ++w) {
                const uint4 q = real ? __ldg(reinterpret_cast<const uint4*>(qp) + w) : make_uint4(0u, 0u, 0u, 0u);
                qf[w][0] = __byte_perm(q.x, q.z, 0x5410); qf[w][1] = __byte_perm(q.x, q.z, 0x7632);
                qf[w][2] = __byte_perm(q.y, q.w, 0x5410); qf[w][3] = __byte_perm(q.y, q.w, 0x7632);
            }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) o[mt][0] = o[mt][1] = o[mt][2] = o[mt][3] = 0.f;
            m_run[0] = m_run[1] = -INFINITY;
            l_run[0] = l_run[1] = 0.f;
        }
        cp_async_wait<kStages - 2>();      // this tile's records have landed
        __syncwarp();                      // (everybody's, and the stage of the tile before has been read)
        issue(ahead_token, (uint32_t)(i + kStages - 1) % kStages);
        ahead_token = find_pages(ahead_pos);
        ahead_pos = next_indices();
        const uint32_t st = ring + (uint32_t)i % kStages * St::kBytes;

        // ---- S^T = K Q^T ----
        float s[4] = {0.f, 0.f, 0.f, 0.f}, s2[4] = {0.f, 0.f, 0.f, 0.f};
        {
            uint32_t kc[2][KW], ks[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                lds_words<KW>(kc[e], st + (gid + 8 * e) * St::kRow + tig * (KW * 4));
                ks[e] = lds_small<KS>(st + St::kS + (gid + 8 * e) * St::kSRow + tig * KS);
            }
#pragma unroll
            for (int gr = 0; gr < KS; ++gr) {
                const uint32_t sa = scale_bf16x2((ks[0] >> (8 * gr)) & 255u), sb = scale_bf16x2((ks[1] >> (8 * gr)) & 255u);
                const uint32_t za = zero_bf16x2(sa), zb = zero_bf16x2(sb);
#pragma unroll
                for (int w = gr * (KW / KS); w < (gr + 1) * (KW / KS); ++w) {
                    uint32_t pa[4], pb[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        pa[j] = fma_bf16x2(code_pair(kc[0][w], j), sa, za);
                        pb[j] = fma_bf16x2(code_pair(kc[1][w], j), sb, zb);
                    }
                    mma_bf16_16816(s, pa[0], pb[0], pa[1], pb[1], qf[w][0], qf[w][1]);
                    mma_bf16_16816(s2, pa[2], pb[2], pa[3], pb[3], qf[w][2], qf[w][3]);
                }
            }
        }

        // ---- softmax against a reference that few scores move ----
        const int j0 = cur.j * kTile + gid;
        const bool v0 = j0 < cur.k, v1 = j0 + 8 < cur.k;
        float sc[4];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            sc[e] = v0 ? (s[e] + s2[e]) * a.scale_log2 : -INFINITY;
            sc[2 + e] = v1 ? (s[2 + e] + s2[2 + e]) * a.scale_log2 : -INFINITY;
        }
        const bool jump = fmaxf(sc[0], sc[2]) > m_run[0] + kRefSlack || fmaxf(sc[1], sc[3]) > m_run[1] + kRefSlack;
        if (__any_sync(0xFFFFFFFFu, jump)) {
            float alpha[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float mx = fmaxf(sc[e], sc[2 + e]);
                mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 4));
                mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 8));
                mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 16));
                const float m_new = fmaxf(m_run[e], mx - kRefUnder);
                alpha[e] = ex2(m_run[e] - m_new);
                m_run[e] = m_new;
                l_run[e] *= alpha[e];
            }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                o[mt][0] *= alpha[0]; o[mt][1] *= alpha[1]; o[mt][2] *= alpha[0]; o[mt][3] *= alpha[1];
            }
        }
        float p[4];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            p[e] = ex2(sc[e] - m_run[e]);
            p[2 + e] = ex2(sc[2 + e] - m_run[e]);
            l_run[e] += p[e] + p[2 + e];
        }
        const uint32_t pb0 = transposed(pack_f16(p[0], p[1])), pb1 = transposed(pack_f16(p[2], p[3]));

        // ---- O^T += V'^T P^T ----
        {
            uint32_t vc[4][VW];
            float vs[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int key = 2 * tig + (e & 1) + 8 * (e >> 1);
                lds_words<VW>(vc[e], st + St::kV + key * St::kVRow + gid * (VW * 4));
                vs[e] = scale_f32(lds_small<1>(st + St::kS + key * St::kSRow + DH / 16 + (DH == 128 ? gid : gid >> 1)));
            }
            const uint32_t sa = pack_f16(vs[0], vs[1]), sb = pack_f16(vs[2], vs[3]);
#pragma unroll
            for (int w = 0; w < VW; ++w)
#pragma unroll
                for (int hf = 0; hf < 2; ++hf) {
                    uint32_t va[4], vb[4];
                    values_f16x2(va, __byte_perm(vc[0][w], vc[1][w], hf ? 0x7632 : 0x5410), sa);
                    values_f16x2(vb, __byte_perm(vc[2][w], vc[3][w], hf ? 0x7632 : 0x5410), sb);
                    mma_f16_16816(o[w * 4 + hf * 2], va[0], va[1], vb[0], vb[1], pb0, pb1);
                    mma_f16_16816(o[w * 4 + hf * 2 + 1], va[2], va[3], vb[2], vb[3], pb0, pb1);
                }
        }

        // ---- end of the row, or of this unit's part of it ----
        const bool last = i + 1 >= issued;
        if (cur.j + 1 >= cur.n || last) {
            float l[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                l[e] = l_run[e];
                l[e] += __shfl_xor_sync(0xFFFFFFFFu, l[e], 4);
                l[e] += __shfl_xor_sync(0xFFFFFFFFu, l[e], 8);
                l[e] += __shfl_xor_sync(0xFFFFFFFFu, l[e], 16);
            }
            bool whole = true;
            int32_t slot = 0;
            if constexpr (SPLIT) {
                whole = cum[cur.row] >= lo && cum[cur.row + 1] <= hi;
                slot = 2 * unit + (cum[cur.row] > lo ? 1 : 0);
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int head = 2 * tig + e;
                if (head < G) {
                    float v[DL];
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) { v[2 * mt] = o[mt][e]; v[2 * mt + 1] = o[mt][2 + e]; }
                    if (whole) {
                        const float inv = 1.0f / l[e];
#pragma unroll
                        for (int d = 0; d < DL; ++d) v[d] *= inv;
                        write_gated<DL>(a, ((int64_t)cur.row * a.n_h + h * G + head) * DH + gid * DL, v);
                    } else {
                        const int64_t sh = (int64_t)slot * a.n_h + h * G + head;
                        float4* to = reinterpret_cast<float4*>(a.state + sh * DH + gid * DL);
#pragma unroll
                        for (int d = 0; d < DL / 4; ++d) to[d] = make_float4(v[4 * d], v[4 * d + 1], v[4 * d + 2], v[4 * d + 3]);
                        if (gid == 0) a.stats[sh] = make_float2(m_run[e], l[e]);
                    }
                }
            }
            fresh = true;
        }
        if (!last) advance(cur);
    }
    if constexpr (SPLIT) {
        // what the merge needs, and rows with an empty set
        if (blockIdx.x == 0)
            for (int r = threadIdx.x; r <= a.rows; r += kWarps * 32) a.cum[r] = cum[r];
        const int64_t row_vec = (int64_t)a.n_h * DH / 8;
        for (int r = blockIdx.x; r < a.rows; r += gridDim.x)
            if (budget[r] == 0)
                for (int i = threadIdx.x; i < row_vec; i += kWarps * 32) reinterpret_cast<uint4*>(a.out)[r * row_vec + i] = make_uint4(0u, 0u, 0u, 0u);
    }
    if (bad) cta_bad = 1;
    __syncthreads();
    if (threadIdx.x == 0) {
        if constexpr (SPLIT) a.flags[blockIdx.x] = cta_bad;
        else if (cta_bad) report_bad_index(a.status);
    }
}

// Rows whose parts lie in several units' runs: the parts' states in their order, normalised, gated, rounded.  WPI warps share a
// (row, head): all eight of a CTA where a row has many parts, one where it has few.  With by_cut the rows are found by the borders between
// units instead of one by one, and a row is done at the first border inside it.  The last CTA writes the status head.
template <int DH, int WPI>
__global__ void __launch_bounds__(kMergeWarps * 32) gsa_cache_merge_kernel(const CacheAttnArgs a, int32_t by_cut, int32_t items, int32_t ctas) {
    chain_wait();
    constexpr int N = DH / 32;             // d of a lane
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (blockIdx.x == gridDim.x - 1) {
        int bad = 0;
        for (int i = threadIdx.x; i < ctas; i += kMergeWarps * 32) bad |= a.flags[i];
        bad = __syncthreads_or(bad);
        if (threadIdx.x < kStatusBytes / 4) a.status[threadIdx.x] = threadIdx.x == 0 && bad ? kDevBadIndex : kDevOk;
        return;
    }
    __shared__ float part_o[WPI > 1 ? WPI : 1][DH];
    __shared__ float2 part_ml[WPI > 1 ? WPI : 1];
    const int item = blockIdx.x * (kMergeWarps / WPI) + warp / WPI, sub = warp % WPI;
    if (item >= items) return;             // (WPI > 1: one item a CTA, and there are no more CTAs than items)
    const int head = item % a.n_h;
    int32_t row = item / a.n_h;
    const int32_t tiles = a.cum[a.rows], units = units_for(tiles, a.units);
    if (by_cut) {
        const int32_t u = row + 1;
        if (u >= units) return;
        const int32_t x = first_tile(u, tiles, units);
        int32_t rl = 0, rh = a.rows - 1;
        while (rl < rh) {
            const int32_t m = (rl + rh + 1) >> 1;
            if (a.cum[m] <= x) rl = m; else rh = m - 1;
        }
        row = rl;
        if (a.cum[row] == x || first_tile(u - 1, tiles, units) > a.cum[row]) return;
    }
    const int32_t c0 = a.cum[row], c1 = a.cum[row + 1];
    if (c1 <= c0) return;                  // (an empty set: written by the first kernel)
    const int32_t u0 = unit_of(c0, tiles, units), n = unit_of(c1 - 1, tiles, units) - u0 + 1;
    if (n == 1) return;                    // (within one unit)
    const int32_t first_slot = 2 * u0 + (c0 > first_tile(u0, tiles, units) ? 1 : 0);
    float m = -INFINITY, l = 0.f, o[N];
#pragma unroll
    for (int d = 0; d < N; ++d) o[d] = 0.f;
    constexpr int AHEAD = 4;               // parts whose loads are in flight together
    for (int i0 = sub; i0 < n; i0 += WPI * AHEAD) {
        float2 ml[AHEAD];
        float v[AHEAD][N];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int i = i0 + k * WPI;
            ml[k] = make_float2(-INFINITY, 0.f);
#pragma unroll
            for (int d = 0; d < N; ++d) v[k][d] = 0.f;
            if (i < n) {
                const int64_t at = (int64_t)(i == 0 ? first_slot : 2 * (u0 + i)) * a.n_h + head;
                ml[k] = a.stats[at];
                if constexpr (N == 4) {
                    const float4 f = *reinterpret_cast<const float4*>(a.state + at * DH + lane * 4);
                    v[k][0] = f.x; v[k][1] = f.y; v[k][2] = f.z; v[k][3] = f.w;
                } else {
                    const float2 f = *reinterpret_cast<const float2*>(a.state + at * DH + lane * 2);
                    v[k][0] = f.x; v[k][1] = f.y;
                }
            }
        }
        float m_new = m;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) m_new = fmaxf(m_new, ml[k].x);
        const float keep = m == m_new ? 1.0f : ex2(m - m_new);
        l *= keep;
#pragma unroll
        for (int d = 0; d < N; ++d) o[d] *= keep;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (i0 + k * WPI < n) {
                const float w = ex2(ml[k].x - m_new);
                l = fmaf(ml[k].y, w, l);
#pragma unroll
                for (int d = 0; d < N; ++d) o[d] = fmaf(v[k][d], w, o[d]);
            }
        m = m_new;
    }
    if constexpr (WPI > 1) {
#pragma unroll
        for (int d = 0; d < N; ++d) part_o[sub][lane * N + d] = o[d];
        if (lane == 0) part_ml[sub] = make_float2(m, l);
        __syncthreads();
        if (sub != 0) return;
        float m_all = -INFINITY;
#pragma unroll
        for (int w = 0; w < WPI; ++w) m_all = fmaxf(m_all, part_ml[w].x);
        l = 0.f;
#pragma unroll
        for (int d = 0; d < N; ++d) o[d] = 0.f;
#pragma unroll
        for (int w = 0; w < WPI; ++w)
            if (w < n) {                   // (a warp without parts has nothing to add)
                const float f = ex2(part_ml[w].x - m_all);
                l = fmaf(part_ml[w].y, f, l);
#pragma unroll
                for (int d = 0; d < N; ++d) o[d] = fmaf(part_o[w][lane * N + d], f, o[d]);
            }
    }
    const int64_t at = ((int64_t)row * a.n_h + head) * DH + lane * N;
    const uint32_t* g = reinterpret_cast<const uint32_t*>(a.g1 + at);
    const float inv = 1.0f / l;
#pragma unroll
    for (int d = 0; d < N; d += 2) {
        const uint32_t gw = __ldg(g + d / 2);
        reinterpret_cast<uint32_t*>(a.out + at)[d / 2] = pack_bf16(o[d] * inv * fast_sigmoid(__uint_as_float(gw << 16)),
                                                                   o[d + 1] * inv * fast_sigmoid(__uint_as_float(gw & 0xFFFF0000u)));
    }
}

int32_t unit_count(const gsa_params_t& p) { return sm_count() * kCtasPerSm * (kWarps / p.n_kv); }

template <int DH, int G, bool SPLIT>
cudaError_t launch_main(const CacheAttnArgs& a, cudaStream_t st) {
    const int subs = kWarps / a.c.n_kv;
    const size_t smem = (SPLIT ? row_table_bytes(a.rows) : 0) + (size_t)kWarps * kStages * Stage<DH>::kBytes;
    // (set on every call: the attribute belongs to the current device)
    cudaError_t e = cudaFuncSetAttribute(gsa_cache_attn_kernel<DH, G, SPLIT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    e = launch_chained(gsa_cache_attn_kernel<DH, G, SPLIT>, (unsigned)(a.units / subs), kWarps * 32, smem, st, a);
    ++g_launches;
    return e != cudaSuccess ? e : cudaGetLastError();
}

template <int DH, int WPI>
cudaError_t launch_merge(const CacheAttnArgs& a, int32_t by_cut, int32_t items, cudaStream_t st) {
    const unsigned ctas = (unsigned)((items + kMergeWarps / WPI - 1) / (kMergeWarps / WPI)) + 1u;
    cudaError_t e = launch_chained(gsa_cache_merge_kernel<DH, WPI>, ctas, kMergeWarps * 32, 0, st, a, by_cut, items, a.units / (kWarps / a.c.n_kv));
    ++g_launches;
    return e != cudaSuccess ? e : cudaGetLastError();
}

struct Plan { size_t stats, cum, flags, total; };
Plan plan_scratch(const gsa_params_t& p) {
    const size_t slots = 2 * (size_t)unit_count(p), rows = (size_t)p.B * p.Lq;
    Plan w;
    w.stats = align_up(slots * p.n_h * p.d_h * 4, 256);
    w.cum = w.stats + align_up(slots * p.n_h * 8, 256);
    w.flags = w.cum + align_up((rows + 1) * 4, 256);
    w.total = w.flags + align_up((size_t)sm_count() * kCtasPerSm * 4, 256);
    return w;
}

}  // namespace

size_t cache_attn_scratch_bytes(const gsa_params_t& p) {
    return (int64_t)p.B * p.Lq > kMaxSplitRows ? 0 : plan_scratch(p).total;
}

cudaError_t launch_cache_attn(const CacheView& c, const gsa_params_t& p, const __nv_bfloat16* Q, const __nv_bfloat16* g1,
                              const int32_t* idx, const int32_t* kt, __nv_bfloat16* out, int32_t* ws, cudaStream_t st) {
    CacheAttnArgs a{};
    a.c = c; a.Q = Q; a.g1 = g1; a.idx = idx; a.kt = kt; a.out = out;
    a.rows = p.B * p.Lq; a.Lq = p.Lq; a.Lk = p.Lk; a.n_h = p.n_h; a.k_max = p.k_max;
    a.scale_log2 = (p.sm_scale > 0.f ? p.sm_scale : 1.0f / sqrtf((float)p.d_h)) * 1.4426950408889634f;
    a.status = ws;
    const bool split = a.rows <= kMaxSplitRows;
    const int subs = kWarps / p.n_kv;
    a.units = unit_count(p);
    cudaError_t e = cudaSuccess;
    if (split) {
        const Plan w = plan_scratch(p);
        char* s = (char*)ws + kStatusBytes;
        a.state = (float*)s; a.stats = (float2*)(s + w.stats); a.cum = (int32_t*)(s + w.cum); a.flags = (int32_t*)(s + w.flags);
        // no more CTAs than the largest sets would keep busy
        const int64_t most = units_for((int64_t)a.rows * ((p.k_max + kTile - 1) / kTile), a.units);
        a.units = (int32_t)((most + subs - 1) / subs * subs);
    } else {
        e = launch_clear(st, {ws, (size_t)kStatusBytes});  // (with a merge, that writes the head)
    }
    if (e != cudaSuccess) return e;
    e = cudaErrorInvalidValue;
#define GSA_CACHE_CASE(DH_, G_) \
    if (p.d_h == DH_ && p.n_h / p.n_kv == G_) e = split ? launch_main<DH_, G_, true>(a, st) : launch_main<DH_, G_, false>(a, st)
    GSA_CACHE_CASE(128, 1); GSA_CACHE_CASE(128, 2); GSA_CACHE_CASE(128, 4); GSA_CACHE_CASE(128, 8);
    GSA_CACHE_CASE(64, 1); GSA_CACHE_CASE(64, 2); GSA_CACHE_CASE(64, 4); GSA_CACHE_CASE(64, 8);
#undef GSA_CACHE_CASE
    if (e != cudaSuccess || !split) return e;
    const int32_t by_cut = a.rows > a.units - 1 ? 1 : 0;
    const int32_t items = (by_cut ? a.units - 1 : a.rows) * p.n_h;
    const bool many = !by_cut && a.units >= 8 * a.rows;    // parts of a row: eight or more
    if (p.d_h == 128) return many ? launch_merge<128, 8>(a, by_cut, items, st) : launch_merge<128, 1>(a, by_cut, items, st);
    return many ? launch_merge<64, 8>(a, by_cut, items, st) : launch_merge<64, 1>(a, by_cut, items, st);
}

}  // namespace gsa
