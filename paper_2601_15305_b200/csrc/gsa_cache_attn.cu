// Sparse gated attention (Eq. 11, 12, 10) over index sets whose K and V' lie in the pages of a 4-bit cache (include/gsa.h).
//
// A set is walked in tiles of 16 keys; n_kv warps (a unit) take a tile together, one KV head each.  As in gsa_attn.cu keys are the
// M side of an MMA and the group's query heads its N side, and a contraction does not care about the order of its index, so a lane takes
// the codes that lie together in memory.  What a tile costs is taking the codes apart, so as little as possible is done to them:
//   K   lane (gid, tig): the tig-th quarter of the head row of keys gid and gid + 8, eight codes a word; Q is read with the same
//       permutation.  A code u, masked out of its word, IS the fp16 number u * 2^-24 (16 u * 2^-24 in a half word's second place, with
//       Q / 16 against it), and that is the operand: one logical operation for two codes.
//       Scales: in a k-step each of the four lanes of a key has codes of a group of its own.  Up to four query heads leave columns of
//       the MMA free, and those keep the four lanes' groups apart: column (slot, head) of Q^T has Q[head] where lane `slot` supplies
//       the index and 0 elsewhere.  The accumulators are then sums over one group each, Sum u q; their scales (which that lane holds)
//       and the code's offset (-8 Sum q, what the accumulators start from) are applied to them, and the slots are added up by
//       shuffles.                                                                S^T[key, head] = K[key, :] . Q[head, :]
//       (Q as fp16: a power of two of its own brings each head's largest |q| to 2^14 .. 2^15, where every bf16 within 2^-25 of it is exact.)
//       Eight heads fill the columns: there K is dequantised, in bf16, by one multiply-add, (128 + u) s - 136 s, exactly.
//   V'  lane (gid, tig): the gid-th eighth of keys 2 tig, 2 tig + 1, 2 tig + 8, 2 tig + 9; words of two keys are joined half by half, so
//       that a code position yields the pair (key, key + 1) of one d.                O^T[d, head] += V'^T[d, key] P^T[key, head]
//       At d_h = 128 that eighth is one group of 16 and has one scale.  In fp16 (1024 + u) - 1032, or (1024 + 16 u) / 16 - 72, then
//       times s: every value of the format is exact in fp16 too (105 * 2^-23 .. 7 * 3584).
// The tile's numerators are rounded to fp16 for the second product.  They are taken against a reference that leaves a row's largest
// between 2^7 and 2^15, so that rounding is at most 2^-11 of a numerator, or 2^-25 where that is less than fp16's normal range goes down
// to: 2^-32 of the row's sum.  (Scores above 2^24, whose neighbours in fp32 lie 2 and more apart, leave a row's largest at 2^0 to 2^14.  In bf16, 2^-8 of each, the error of the 32 x 128K case against 64 bits is 2.3e-3; with fp16 it is
// 1.7e-3, the output's own rounding.)  Statistics, scores and sums are fp32.
//
// Records come by asynchronous copies into a ring of kStages tiles a warp (2560 bytes each at d_h = 128, V' rows padded), so that some 70 to
// 110 KB of an SM are in flight.  Indices and pages are looked up for blocks of four or eight tiles, each warp of a unit a share of the keys, two blocks
// ahead; the records' addresses pass through shared memory.  The units of an SM are kept abreast, a barrier a block: left alone, the warps
// that the scheduler prefers finish a quarter earlier than the others, which then have the SM half empty.
//
// Work split: the tiles of all rows, one after another, are dealt to the units in equal runs, whatever the sets' sizes (each CTA sums
// up the budgets for itself).  A row that lies within one unit's run is finished there; the others' parts (at most two a unit) go to
// the workspace as softmax state and are merged by a second kernel, in order, so that nothing depends on scheduling.  More rows than
// kMaxSplitRows take several such launches.  Small sets (kOwnTiles) in few rows have a CTA for each row instead, which merges its
// units' parts itself: one launch.
//
// Bound: the issue of instructions, some 500 for a tile and KV head, by four warps a scheduler (the registers allow no more; 57 % of all
// cycles issue one, and most others wait for a fixed latency or the ALU).  32 sequences of 16K to 128K, 16 heads on 8 KV heads of 128: 71 MB of
// records, 30.0 us with the merge (29.4 with one power of two for a KV head's queries instead of one a head; chunk 58.9), 2.4 TB/s; some 6 us pass before the first tile (budgets, indices, pages, records: four loads in a
// row), 18 us in the loop, 6 us from its end to the end of the merge.  257 rows of 1000 of 20011 keys, 32 heads on 8 of 64: 60.6 us.
// (Four query heads at d_h = 128 spill 108 to 244 bytes a thread: 16 sequences of 4K to 32K, 8 KV heads, 26.4 us, with two heads 21.7.)
#include "gsa_cache.cuh"

#include <cuda_fp16.h>

namespace gsa {

namespace {

constexpr int kWarps = 16;                 // one CTA an SM
constexpr int kTile = 16;                  // keys
constexpr int kStages = 4;                 // tiles of a warp's ring: two being computed on, the others in flight (a power of two)
constexpr int kLut = 256;                  // scales by their byte, as fp32
constexpr int kMinTiles = 2;               // fewest tiles worth a unit of their own
constexpr int kMaxSplitRows = 2048;        // rows of one launch, whose budgets a CTA sums up (16 KB of its shared memory)
constexpr int kAddressBlocks = 4;          // blocks of record addresses: being read, next, being written (and a power of two)
constexpr int kOwnTiles = 1, kManyOwnTiles = 4;        // tiles a unit, at most, for rows with a CTA of their own; the same if they occupy half the SMs
constexpr int kMergeWarps = 8;
constexpr float kRefUnder = 7.0f;          // a new softmax reference lies 2^7 under the score that moved it there (2^0 to 2^14 where fp32 cannot tell),
constexpr float kMostNumerator = 32768.0f; // and moves again when a score lies 2^15 above it (fp16 ends at 2^16)

struct CacheAttnArgs {
    CacheView c;
    const __nv_bfloat16 *Q, *g1;
    const int32_t *idx, *kt;
    __nv_bfloat16* out;
    int32_t rows, row0, Lq, Lk, n_h, k_max;            // rows of this launch, the first one's number in the call
    float scale_log2;
    int32_t units;                         // of the launch; as many as there are tiles for take part
    float* state;                          // [2 * units][n_h][d_h] numerators
    float2* stats;                         // [2 * units][n_h] reference, sum
    int4* merges;                          // [merge_items] rows whose parts the merge puts together: row, first slot, parts
    int32_t merge_items, by_cut;           // one for each row, or (by_cut) for each border between units
    int32_t* flags;                        // [CTAs] whether one met something out of range
    int32_t* status;                       // head of the workspace
    int32_t own;                           // a CTA for each row
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
__device__ __forceinline__ uint32_t lds_byte(uint32_t p) {
    uint32_t v;
    asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(p));
    return v;
}
__device__ __forceinline__ uint32_t lds_word(uint32_t p) {
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(p));
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

// fast_sigmoid, but a NaN stays one (there the clamp makes it 2^-126: a row of almost zeros, and nothing to show for it)
__device__ __forceinline__ float gate_of(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + ex2(min_nan(-1.4426950408889634f * x, 126.f))));
    return r;
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
            w[j] = pack_bf16(o[i * 8 + 2 * j] * gate_of(__uint_as_float(gw[j] << 16)),
                             o[i * 8 + 2 * j + 1] * gate_of(__uint_as_float(gw[j] & 0xFFFF0000u)));
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
// tiles of a block of addresses: one or two keys a lane of the unit's warps
constexpr int block_tiles(int NKV) { return NKV >= 4 ? 8 : 4; }
constexpr size_t address_bytes(int NKV) { return (size_t)(kWarps / NKV) * kAddressBlocks * block_tiles(NKV) * kTile * 4; }
template <int DH, int NKV>
constexpr size_t fixed_smem() { return kLut * 4 + address_bytes(NKV) + (size_t)kWarps * kStages * Stage<DH>::kBytes; }

// What the merge has to do: a row whose tiles lie in several units' runs has its first part in the unit that holds its first tile and the
// others in the units behind it.  With by_cut an item is a border between units, and a row's item is the first border inside it.
__device__ __forceinline__ void list_merges(const CacheAttnArgs& a, const int32_t* cum, int32_t tiles, int32_t units) {
    for (int i = threadIdx.x; i < a.merge_items; i += kWarps * 32) {
        int4 m = make_int4(0, 0, 0, 0);
        int32_t row = i;
        bool real = true;
        if (a.by_cut) {
            const int32_t u = i + 1;
            real = u < units;
            if (real) {
                const int32_t x = first_tile(u, tiles, units);
                int32_t rl = 0, rh = a.rows - 1;
                while (rl < rh) {
                    const int32_t mid = (rl + rh + 1) >> 1;
                    if (cum[mid] <= x) rl = mid; else rh = mid - 1;
                }
                row = rl;
                real = cum[row] != x && first_tile(u - 1, tiles, units) <= cum[row];
            }
        }
        if (real && cum[row + 1] > cum[row]) {
            const int32_t u0 = unit_of(cum[row], tiles, units);
            m = make_int4(row, 2 * u0 + (cum[row] > first_tile(u0, tiles, units) ? 1 : 0), unit_of(cum[row + 1] - 1, tiles, units) - u0 + 1, 0);
        }
        a.merges[i] = m;                   // (one part, or none: nothing to do)
    }
}

template <int DH, int G, int NKV>
__global__ void __launch_bounds__(kWarps * 32, 1) gsa_cache_attn_kernel(const CacheAttnArgs a) {
    chain_wait();
    using St = Stage<DH>;
    constexpr int D = NKV * DH;
    constexpr int KW = DH / 32;            // words of K codes a lane has of a key
    constexpr int VW = DH / 64;            // words of V' codes a lane has of a key
    constexpr int KS = DH / 64;            // scales of those K codes
    constexpr int MT = DH / 16;
    constexpr int DL = DH / 8;             // consecutive d of O that a lane holds, for heads 2 tig and 2 tig + 1
    constexpr int CPK = DH / 32, KPI = 32 / CPK;       // 16-byte chunks of a key's codes, keys that one copy of a warp covers
    constexpr int SUBS = kWarps / NKV;
    constexpr int BT = block_tiles(NKV), KPW = BT * kTile / NKV, STEPS = (KPW + 31) / 32;      // keys of a block that a warp looks up
    constexpr bool COLS = G <= 4;          // groups in columns of their own
    constexpr int SETS = G == 4 ? 2 : 1;   // MMAs that the four slots take
    // Scores that a lane ends up with: keys gid and gid + 8 for two heads, 2 tig, + 1 of eight or 2 (tig & 1), + 1 of four; up to two heads
    // (a fourth of the exponentials, half of the shuffles: 32 x 128K 31.2 -> 30.3 us; four heads are 2 % slower with two scores
    // a lane) key gid + 8 (tig >> 1) for head tig & 1, or the one.
    constexpr bool ONE = G <= 2;
    constexpr int NH = ONE ? 1 : 2, NS = ONE ? 1 : 4;      // heads and scores
    constexpr int SPREAD = ONE ? 2 : 4;                    // the lowest bit of the lane numbers that have a head's other keys
    extern __shared__ __align__(16) unsigned char smem[];  // scales, record addresses, rings, cum[rows + 1], budget[rows]
    __shared__ int32_t warp_sum[kWarps];
    __shared__ int32_t cta_bad;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int gid = lane >> 2, tig = lane & 3;
    const CacheView& c = a.c;
    const int h = warp % NKV, sub = warp / NKV;
    const int rows = a.own ? 1 : a.rows, row_base = a.own ? blockIdx.x : 0;
    const int unit = a.own ? sub : sub * gridDim.x + blockIdx.x;
    const uint32_t lut = smem_u32(smem);
    uint32_t* const addresses = reinterpret_cast<uint32_t*>(smem) + kLut + sub * (kAddressBlocks * BT * kTile);       // in units of 16 bytes
    const uint32_t ring = lut + kLut * 4 + (uint32_t)address_bytes(NKV) + warp * (kStages * St::kBytes);
    // the part of a warp: numerators [G][d_h], reference and sum [G]
    auto part_of = [&](int w) { return reinterpret_cast<float*>(smem + kLut * 4 + address_bytes(NKV) + (size_t)w * (kStages * St::kBytes)); };
    float* const own_part = part_of(warp);
    int32_t* const cum = reinterpret_cast<int32_t*>(smem + fixed_smem<DH, NKV>());
    int32_t* const budget = cum + rows + 1;
    bool bad = false;
    if (threadIdx.x == 0) cta_bad = 0;
    if (threadIdx.x < kLut) reinterpret_cast<float*>(smem)[threadIdx.x] = scale_f32(threadIdx.x);
    auto scale_at = [&](uint32_t p) { return __uint_as_float(lds_word(lut + lds_byte(p) * 4)); };      // the scale whose byte is there

    // ---- tiles in front of every row ----
    int32_t tiles = 0;
    {
        const int per = (rows + kWarps * 32 - 1) / (kWarps * 32), r0 = min(rows, (int)threadIdx.x * per), r1 = min(rows, r0 + per);
        int32_t mine = 0;
        for (int r = r0; r < r1; ++r) {
            const int32_t given = __ldg(a.kt + row_base + r), k = clamp_budget(given, a.k_max);
            bad |= given != k;
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
        if (threadIdx.x == 0) cum[rows] = tiles;
        __syncthreads();
    }
    const int32_t units = units_for(tiles, a.own ? SUBS : gridDim.x * SUBS);
    if (!a.own && blockIdx.x == gridDim.x - 1) list_merges(a, cum, tiles, units);
    const int32_t n_most = units ? (tiles + units - 1) / units : 0;        // of any unit
    int32_t lo = 0, n = 0;                 // this unit's tiles: lo .. lo + n - 1
    if (unit < units) {
        lo = first_tile(unit, tiles, units);
        n = first_tile(unit + 1, tiles, units) - lo;
    }
    if (n > 0) {
        int32_t row = 0;                   // the row that holds tile lo (of rows that start there the last: the others are empty)
        for (int32_t rh = rows - 1; row < rh;) {
            const int32_t m = (row + rh + 1) >> 1;
            if (cum[m] <= lo) row = m; else rh = m - 1;
        }

        // the first row's Q is on its way while the tables are read
        constexpr bool kAll = !COLS || G == 4;
        const bool q_mine = kAll || ((gid >> 1) == tig && (gid & 1) < G);          // COLS: this lane's index is this lane's column's slot
        const int q_head = !COLS ? gid : G == 4 ? gid & 3 : gid & 1;
        uint4 q[KW];
        auto load_q = [&](int32_t of_row) {
            const __nv_bfloat16* qp = a.Q + ((int64_t)(row_base + of_row) * a.n_h + h * G + (q_mine ? q_head : 0)) * DH + tig * (DH / 4);
#pragma unroll
            for (int w = 0; w < KW; ++w) q[w] = q_mine ? __ldg(reinterpret_cast<const uint4*>(qp) + w) : make_uint4(0u, 0u, 0u, 0u);
        };
        load_q(row);

        // ---- addresses of the records: a block's indices, then pages ----
        int32_t look_row = row;            // (of this lane's last key)
        struct Look { int32_t raw, seq, len, pos, page; };     // a key: index, sequence and its length; position (-1: none) and page
        auto key_of = [&](int step) { return h * KPW + step * 32 + lane; };          // in the block
        auto load_indices = [&](Look(&k)[STEPS], int block) {
#pragma unroll
            for (int st = 0; st < STEPS; ++st) {
                k[st].seq = -1;
                const int t = block * BT + key_of(st) / kTile;                         // tile of the run
                if ((KPW < 32 && lane >= KPW) || t >= n) continue;
                const int32_t g = lo + t;
                while (cum[look_row + 1] <= g) ++look_row;
                const int j = (g - cum[look_row]) * kTile + (lane & (kTile - 1));
                // places behind the set's end read the tile's first key again (their probabilities are 0)
                k[st].raw = __ldg(a.idx + (int64_t)(row_base + look_row) * a.k_max + (j < budget[look_row] ? j : j & ~(kTile - 1)));
                k[st].seq = (a.row0 + row_base + look_row) / a.Lq;
                k[st].len = __ldg(c.lens + k[st].seq);
            }
        };
        auto load_pages = [&](Look(&k)[STEPS]) {
#pragma unroll
            for (int st = 0; st < STEPS; ++st) {
                k[st].pos = -1;
                if (k[st].seq < 0) continue;
                const int32_t len = min(max(k[st].len, 0), a.Lk);
                bad |= len != k[st].len || (uint32_t)k[st].raw >= (uint32_t)len;
                k[st].pos = min(max(k[st].raw, 0), max(len - 1, 0));
                k[st].page = __ldg(c.table + (int64_t)k[st].seq * c.max_pages + (k[st].pos >> c.log_t));
            }
        };
        auto put_addresses = [&](const Look(&k)[STEPS], int slot) {
#pragma unroll
            for (int st = 0; st < STEPS; ++st)
                if (k[st].pos >= 0) {
                    const bool named = (uint32_t)k[st].page < (uint32_t)c.n_pages;
                    bad |= !named;
                    addresses[slot * (BT * kTile) + key_of(st)] =
                        (uint32_t)(named ? k[st].page : 0) * (uint32_t)(c.page_bytes >> 4) + (uint32_t)(k[st].pos & (c.T - 1)) * (uint32_t)(c.rec >> 4);
                }
        };
        auto unit_sync = [&]() {
            if constexpr (NKV == 1) __syncwarp();
            else asm volatile("bar.sync %0, %1;" ::"r"(1 + sub), "r"(NKV * 32) : "memory");
        };
        const int ckey = lane / CPK, cpiece = lane % CPK;
        const unsigned char* const from_codes = c.pool + h * (DH / 2) + cpiece * 16;
        const unsigned char* const from_scales = c.pool + D + h * (DH / 8);
        const uint32_t to_k = ring + ckey * St::kRow + cpiece * 16, to_v = ring + St::kV + ckey * St::kVRow + cpiece * 16;
        const uint32_t to_s = ring + St::kS + (lane & 15) * St::kSRow;
        // tile t of the run, whose addresses start at `from`, into stage `off`
        auto issue = [&](bool real, const uint32_t* from, uint32_t off) {
            if (real) {
#pragma unroll
                for (int i = 0; i < kTile / KPI; ++i) {
                    const unsigned char* src = from_codes + (uint64_t)from[ckey + i * KPI] * 16u;
                    cp_async16(to_k + off + i * KPI * St::kRow, src);
                    cp_async16(to_v + off + i * KPI * St::kVRow, src + D / 2);
                }
                if (lane < kTile) copy_async<St::kSRow>(to_s + off, from_scales + (uint64_t)from[lane] * 16u);
            }
            cp_async_commit();             // (one group a tile, possibly empty)
        };

        Look look[STEPS];
        {
            Look second[STEPS];
            load_indices(look, 0);
            load_indices(second, 1);
            load_pages(look);
            load_pages(second);
            put_addresses(look, 0);
            put_addresses(second, 1);
        }
        unit_sync();
        auto issue_tile = [&](int32_t t) {
            issue(t < n, addresses + (t & (kAddressBlocks * BT - 1)) * kTile, (uint32_t)(t & (kStages - 1)) * St::kBytes);
        };
#pragma unroll
        for (int t = 0; t + 1 < kStages; ++t) issue_tile(t);

        uint32_t qf[KW][4];                // Q as the B operand
        constexpr bool QPAIR = G == 4 && DH == 64;             // four heads: zeroed for either set ahead of time, where registers allow
        uint32_t qz[QPAIR ? KW : 1][4];
        float q_start[SETS][KS][2];        // COLS: what the accumulators start from, -8 times the group's sum of Q
        constexpr int QS = COLS ? NH : 1;
        float q_scale[QS];                 // of this lane's scores, by head
        float o[MT][4], m_run[NH], l_run[NH];
        int32_t row_first = cum[row], row_end = cum[row + 1], row_k = budget[row];
        auto start_row = [&]() {           // Q into its operand registers, an empty state
            if constexpr (!COLS) {
                q_scale[0] = a.scale_log2;
#pragma unroll
                for (int w = 0; w < KW; ++w) {
                    qf[w][0] = __byte_perm(q[w].x, q[w].z, 0x5410); qf[w][1] = __byte_perm(q[w].x, q[w].z, 0x7632);
                    qf[w][2] = __byte_perm(q[w].y, q[w].w, 0x5410); qf[w][3] = __byte_perm(q[w].y, q[w].w, 0x7632);
                }
            } else {
                // the exponent of this lane's head's largest finite |q|, then of every head's (the lanes whose gid ends in its number)
                uint32_t top = 0;
#pragma unroll
                for (int w = 0; w < KW; ++w) {
                    const uint32_t x[4] = {q[w].x, q[w].y, q[w].z, q[w].w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t lo_e = (x[e] >> 7) & 255u, hi_e = (x[e] >> 23) & 255u;
                        top = max(top, max(lo_e == 255u ? 0u : lo_e, hi_e == 255u ? 0u : hi_e));
                    }
                }
                top = max(top, 20u);
                uint32_t tops[G];
#pragma unroll
                for (int hd = 0; hd < G; ++hd) tops[hd] = __reduce_max_sync(0xFFFFFFFFu, G == 1 || (gid & (G - 1)) == hd ? top : 0u);
                top = tops[0];
#pragma unroll
                for (int hd = 1; hd < G; ++hd) top = (gid & (G - 1)) == hd ? tops[hd] : top;
                const float up = __uint_as_float((127u + 14u + 127u - top) << 23);
#pragma unroll
                for (int e = 0; e < QS; ++e) {                     // over the head's power of two (2^24: what a code's place is worth)
                    uint32_t its = tops[0];
                    if constexpr (G == 2) its = tig & 1 ? tops[1] : tops[0];
                    if constexpr (G == 4) its = tig & 1 ? tops[2 + e] : tops[e];
                    q_scale[e] = a.scale_log2 * 16777216.0f * __uint_as_float((its - 14u) << 23);
                }
                float sum[KS];
#pragma unroll
                for (int gr = 0; gr < KS; ++gr) sum[gr] = 0.f;
#pragma unroll
                for (int w = 0; w < KW; ++w) {
                    float f[8];
                    const uint32_t x[4] = {q[w].x, q[w].y, q[w].z, q[w].w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        f[2 * e] = __uint_as_float(x[e] << 16) * up;
                        f[2 * e + 1] = __uint_as_float(x[e] & 0xFFFF0000u) * up;
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum[w / (KW / KS)] += f[e];
#pragma unroll
                    for (int e = 0; e < 4; ++e) qf[w][e] = (e & 1) ? pack_f16(f[e] * 0.0625f, f[e + 4] * 0.0625f) : pack_f16(f[e], f[e + 4]);
                }
                if constexpr (QPAIR) {
#pragma unroll
                    for (int w = 0; w < KW; ++w)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            qz[w][e] = 2 + (gid >> 2) == tig ? qf[w][e] : 0u;
                            qf[w][e] = (gid >> 2) == tig ? qf[w][e] : 0u;
                        }
                }
                // this lane's columns: slot tig, heads 0 and 1; with four heads slot 2 set + (tig >> 1), heads 2 (tig & 1), + 1
#pragma unroll
                for (int set = 0; set < SETS; ++set)
#pragma unroll
                    for (int gr = 0; gr < KS; ++gr)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const int from_slot = G == 4 ? 2 * set + (tig >> 1) : tig;
                            const int from_gid = G == 4 ? 2 * (tig & 1) + e : 2 * tig + e;
                            q_start[set][gr][e] = -8.0f / 16777216.0f * __shfl_sync(0xFFFFFFFFu, sum[gr], from_gid * 4 + from_slot);
                        }
            }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) o[mt][0] = o[mt][1] = o[mt][2] = o[mt][3] = 0.f;
#pragma unroll
            for (int e = 0; e < NH; ++e) { m_run[e] = -INFINITY; l_run[e] = 0.f; }
        };
        // S^T = K Q^T of the tile in stage `st`, in two steps: the products, and what the scales and slots make of them
        constexpr int ACCS = COLS ? SETS * KS : 2;
        auto multiply = [&](uint32_t st, float(&acc)[ACCS][4]) {
            uint32_t kc[2][KW];
#pragma unroll
            for (int e = 0; e < 2; ++e) lds_words<KW>(kc[e], st + (gid + 8 * e) * St::kRow + tig * (KW * 4));
            if constexpr (COLS) {
#pragma unroll
                for (int set = 0; set < SETS; ++set)
#pragma unroll
                    for (int gr = 0; gr < KS; ++gr)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[set * KS + gr][e] = q_start[set][gr][e & 1];
#pragma unroll
                for (int w = 0; w < KW; ++w) {
                    uint32_t x[2][4];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const uint32_t v = kc[e][w], v8 = v >> 8;
                        x[e][0] = v & 0x000F000Fu; x[e][1] = v & 0x00F000F0u;
                        x[e][2] = v8 & 0x000F000Fu; x[e][3] = v8 & 0x00F000F0u;
                    }
#pragma unroll
                    for (int set = 0; set < SETS; ++set) {
                        // four heads: Q of a set's two slots
                        auto qv = [&](int e) -> uint32_t {
                            if constexpr (QPAIR) return set ? qz[w][e] : qf[w][e];
                            return G != 4 || 2 * set + (gid >> 2) == tig ? qf[w][e] : 0u;
                        };
                        float(&ac)[4] = acc[set * KS + w / (KW / KS)];
                        mma_f16_16816(ac, x[0][0], x[1][0], x[0][1], x[1][1], qv(0), qv(1));
                        mma_f16_16816(ac, x[0][2], x[1][2], x[0][3], x[1][3], qv(2), qv(3));
                    }
                }
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[0][e] = acc[1][e] = 0.f;
#pragma unroll
                for (int gr = 0; gr < KS; ++gr) {
                    const uint32_t sa = scale_bf16x2(lds_byte(st + St::kS + gid * St::kSRow + tig * KS + gr));
                    const uint32_t sb = scale_bf16x2(lds_byte(st + St::kS + (gid + 8) * St::kSRow + tig * KS + gr));
                    const uint32_t za = zero_bf16x2(sa), zb = zero_bf16x2(sb);
#pragma unroll
                    for (int w = gr * (KW / KS); w < (gr + 1) * (KW / KS); ++w) {
                        uint32_t pa[4], pb[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            pa[j] = fma_bf16x2(code_pair(kc[0][w], j), sa, za);
                            pb[j] = fma_bf16x2(code_pair(kc[1][w], j), sb, zb);
                        }
                        mma_bf16_16816(acc[0], pa[0], pb[0], pa[1], pb[1], qf[w][0], qf[w][1]);
                        mma_bf16_16816(acc[1], pa[2], pb[2], pa[3], pb[3], qf[w][2], qf[w][3]);
                    }
                }
            }
        };
        auto scale_up = [&](uint32_t st, const float(&acc)[ACCS][4], float(&s)[NS]) {
            if constexpr (COLS) {
                float t[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int set = 0; set < SETS; ++set) {
                    const int sl = G == 4 ? 2 * set + (tig >> 1) : tig;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
#pragma unroll
                        for (int gr = 0; gr < KS; ++gr) {
                            const float f = scale_at(st + St::kS + (gid + 8 * e) * St::kSRow + sl * KS + gr);
                            t[2 * e] = fmaf(acc[set * KS + gr][2 * e], f, t[2 * e]);
                            if (G > 1) t[2 * e + 1] = fmaf(acc[set * KS + gr][2 * e + 1], f, t[2 * e + 1]);
                        }
                    }
                }
                // sums over the slots' lanes
                if constexpr (ONE) {                       // each keeps a part of them: of one key, then of one head
                    const bool second = tig & 2, odd = tig & 1;
                    float k0 = second ? t[2] : t[0], k1 = second ? t[3] : t[1];
                    k0 += __shfl_xor_sync(0xFFFFFFFFu, second ? t[0] : t[2], 2);
                    if (G == 2) k1 += __shfl_xor_sync(0xFFFFFFFFu, second ? t[1] : t[3], 2);
                    s[0] = (G == 2 && odd ? k1 : k0) + __shfl_xor_sync(0xFFFFFFFFu, G == 2 && !odd ? k1 : k0, 1);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[e] = t[e] + __shfl_xor_sync(0xFFFFFFFFu, t[e], 2);
                }
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) s[e] = acc[0][e] + acc[1][e];
            }
        };
        auto stage_of = [&](int32_t t) { return ring + (uint32_t)(t & (kStages - 1)) * St::kBytes; };
        start_row();
        float acc[ACCS][4], s[NS];
        cp_async_wait<kStages - 2>();
        __syncwarp();
        multiply(ring, acc);
        scale_up(ring, acc, s);
        for (int32_t i = 0; i < n; ++i) {
            // ---- addresses ahead ----
            if ((i & (BT - 1)) == 0) {
                if (i >= BT && i + BT < n_most) {
                    put_addresses(look, ((uint32_t)i / BT + 1) & (kAddressBlocks - 1));
                    __syncthreads();
                }
                if (i + 2 * BT < n) load_indices(look, (int)((uint32_t)i / BT) + 2);
            } else if ((i & (BT - 1)) == BT / 2) {
                if (i - BT / 2 + 2 * BT < n) load_pages(look);
            }
            cp_async_wait<kStages - 3>();  // the next tile's records have landed
            __syncwarp();                  // (everybody's, and the stage of the tile before has been read)
            issue_tile(i + kStages - 1);
            // The next tile's scores are under way while this one's softmax is: four warps a scheduler do not hide one another's latencies.
            // (Behind a row's last tile they are formed again with the next row's Q; behind the last tile of all they are nothing.)
            const uint32_t st = stage_of(i), st_next = stage_of(i + 1);
            multiply(st_next, acc);

            // ---- softmax against a reference that few scores move ----
            const bool row_ends = lo + i + 1 == row_end;
            if (row_ends) {
                const int left = row_k - (lo + i - row_first) * kTile;         // keys of this tile
#pragma unroll
                for (int e = 0; e < NS; ++e)
                    if (gid + 8 * (ONE ? tig >> 1 : e >> 1) >= left) s[e] = -INFINITY;
            }
            float p[NS];
            auto numerators = [&]() -> float {             // and the largest
                float most = 0.f;
#pragma unroll
                for (int e = 0; e < NS; ++e) {
                    // (The score is rounded before the reference is taken off: in one multiply-add the difference from a reference near
                    // 2^28, itself rounded to a multiple of 32, could be anything, and the numerator infinite.)
                    p[e] = ex2(__fadd_rn(__fmul_rn(s[e], q_scale[e & (QS - 1)]), -m_run[e & (NH - 1)]));
                    most = fmaxf(most, p[e]);
                }
                return most;
            };
            if (__any_sync(0xFFFFFFFFu, numerators() > kMostNumerator)) {
                float alpha[NH];
#pragma unroll
                for (int e = 0; e < NH; ++e) {
                    float mx = ONE ? s[e] : fmaxf(s[e], s[e + NS - NH]);
#pragma unroll
                    for (int x = SPREAD; x < 32; x <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, x));
                    const float m_new = fmaxf(m_run[e], __fadd_rn(__fmul_rn(mx, q_scale[e & (QS - 1)]), -kRefUnder));
                    alpha[e] = ex2(m_run[e] - m_new);
                    m_run[e] = m_new;
                    l_run[e] *= alpha[e];
                }
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int e = 0; e < NH; ++e) { o[mt][e] *= alpha[e]; o[mt][2 + e] *= alpha[e]; }
                numerators();
            }
#pragma unroll
            for (int e = 0; e < NS; ++e) l_run[e & (NH - 1)] += p[e];
            // P^T's columns: those of the heads that there are.  With one score a lane the matrix turned over has the heads in columns 0 and 2,
            // and keys 8 to 15 in 4 and 6, which the second operand register has to have in 0 and 2; what the others of O sum up is nothing.
            uint32_t pb0, pb1;
            if constexpr (ONE) {
                pb0 = transposed(pack_f16(p[0], 0.f));
                pb1 = __shfl_xor_sync(0xFFFFFFFFu, pb0, 16);
            } else {
                const bool real = 2 * tig < G;             // (with groups in columns the others have copies)
                pb0 = transposed(real ? pack_f16(p[0], p[NS - 3]) : 0u);
                pb1 = transposed(real ? pack_f16(p[NS - 2], p[NS - 1]) : 0u);
            }

            // ---- O^T += V'^T P^T ----
            {
                uint32_t vc[4][VW];
                float vs[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int key = 2 * tig + (e & 1) + 8 * (e >> 1);
                    lds_words<VW>(vc[e], st + St::kV + key * St::kVRow + gid * (VW * 4));
                    vs[e] = scale_at(st + St::kS + key * St::kSRow + DH / 16 + (DH == 128 ? gid : gid >> 1));
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

            scale_up(st_next, acc, s);

            // ---- end of the row, or of this unit's part of it ----
            if (row_ends || i + 1 == n) {
                int32_t next_row = row;
                if (i + 1 < n) {
                    do ++next_row; while (cum[next_row + 1] <= row_end);           // (rows with an empty set are passed over)
                    load_q(next_row);
                }
                float l[NH];
#pragma unroll
                for (int e = 0; e < NH; ++e) {
                    l[e] = l_run[e];
#pragma unroll
                    for (int x = SPREAD; x < 32; x <<= 1) l[e] += __shfl_xor_sync(0xFFFFFFFFu, l[e], x);
                }
                const bool whole = row_first >= lo && row_end <= lo + n;
                const int32_t part = 2 * unit + (row_first > lo ? 1 : 0);
#pragma unroll
                for (int e = 0; e < NH; ++e) {
                    const int head = NH * tig + e;
                    if (head < G) {
                        float v[DL];
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) { v[2 * mt] = o[mt][e]; v[2 * mt + 1] = o[mt][2 + e]; }
                        if (whole) {
                            const float inv = 1.0f / l[e];
#pragma unroll
                            for (int d = 0; d < DL; ++d) v[d] *= inv;
                            write_gated<DL>(a, ((int64_t)(row_base + row) * a.n_h + h * G + head) * DH + gid * DL, v);
                        } else if (a.own) {
                            // (into the warp's ring, which has done its work)
                            float4* to = reinterpret_cast<float4*>(own_part + head * DH + gid * DL);
#pragma unroll
                            for (int d = 0; d < DL / 4; ++d) to[d] = make_float4(v[4 * d], v[4 * d + 1], v[4 * d + 2], v[4 * d + 3]);
                            if (gid == 0) *reinterpret_cast<float2*>(own_part + G * DH + 2 * head) = make_float2(m_run[e], l[e]);
                        } else {
                            const int64_t sh = (int64_t)part * a.n_h + h * G + head;
                            float4* to = reinterpret_cast<float4*>(a.state + sh * DH + gid * DL);
#pragma unroll
                            for (int d = 0; d < DL / 4; ++d) to[d] = make_float4(v[4 * d], v[4 * d + 1], v[4 * d + 2], v[4 * d + 3]);
                            if (gid == 0) a.stats[sh] = make_float2(m_run[e], l[e]);
                        }
                    }
                }
                if (i + 1 < n) {
                    row = next_row;
                    row_first = row_end; row_end = cum[row + 1]; row_k = budget[row];
                    start_row();
                    multiply(st_next, acc);
                    scale_up(st_next, acc, s);
                }
            }
        }
    }
    if (a.own) {
        __syncthreads();
        if (units > 1) {
            // the row's parts, in order: a warp a head, d_h / 32 of its values a lane
            constexpr int N = DH / 32;
            for (int head = warp; head < NKV * G; head += kWarps) {
                float m = -INFINITY, l = 0.f, o[N];
                for (int u = 0; u < units; ++u) m = fmaxf(m, part_of(u * NKV + head / G)[G * DH + 2 * (head % G)]);
#pragma unroll
                for (int d = 0; d < N; ++d) o[d] = 0.f;
                for (int u = 0; u < units; ++u) {
                    const float* part = part_of(u * NKV + head / G);
                    const float w = ex2(part[G * DH + 2 * (head % G)] - m);
                    l = fmaf(part[G * DH + 2 * (head % G) + 1], w, l);
#pragma unroll
                    for (int d = 0; d < N; ++d) o[d] = fmaf(part[(head % G) * DH + lane * N + d], w, o[d]);
                }
                const int64_t at = ((int64_t)row_base * a.n_h + head) * DH + lane * N;
                const float inv = 1.0f / l;
#pragma unroll
                for (int d = 0; d < N; d += 2) {
                    const uint32_t g = __ldg(reinterpret_cast<const uint32_t*>(a.g1 + at) + d / 2);
                    reinterpret_cast<uint32_t*>(a.out + at)[d / 2] = pack_bf16(o[d] * inv * gate_of(__uint_as_float(g << 16)),
                                                                               o[d + 1] * inv * gate_of(__uint_as_float(g & 0xFFFF0000u)));
                }
            }
        }
    }
    // rows with an empty set
    const int64_t row_vec = (int64_t)a.n_h * DH / 8;
    for (int r = a.own ? 0 : blockIdx.x; r < rows; r += gridDim.x)
        if (budget[r] == 0)
            for (int i = threadIdx.x; i < row_vec; i += kWarps * 32)
                reinterpret_cast<uint4*>(a.out)[(row_base + r) * row_vec + i] = make_uint4(0u, 0u, 0u, 0u);
    if (a.own) {
        write_flags(a.status, bad);
        return;
    }
    if (bad) cta_bad = 1;
    __syncthreads();
    if (threadIdx.x == 0) a.flags[blockIdx.x] = cta_bad;
}

// Rows whose parts lie in several units' runs: the parts' states in their order, normalised, gated, rounded.  WPI warps share a
// (row, head): all eight of a CTA where a row has many parts, one where it has few.  The last CTA writes the status head.
template <int DH, int WPI>
__global__ void __launch_bounds__(kMergeWarps * 32) gsa_cache_merge_kernel(const CacheAttnArgs a, int32_t ctas) {
    chain_wait();
    constexpr int N = DH / 32;             // d of a lane
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (blockIdx.x == gridDim.x - 1) {
        int bad = 0;
        for (int i = threadIdx.x; i < ctas; i += kMergeWarps * 32) bad |= a.flags[i];
        bad = __syncthreads_or(bad);
        if (threadIdx.x < kStatusBytes / 4)                // (a call's later launches add to what its first one found)
            a.status[threadIdx.x] = threadIdx.x == 0 && (bad || (a.row0 && a.status[0])) ? kDevBadIndex : kDevOk;
        return;
    }
    __shared__ float part_o[WPI > 1 ? WPI : 1][DH];
    __shared__ float2 part_ml[WPI > 1 ? WPI : 1];
    const int item = blockIdx.x * (kMergeWarps / WPI) + warp / WPI, sub = warp % WPI;
    if (item >= a.merge_items * a.n_h) return;             // (WPI > 1: one item a CTA, and there are no more CTAs than items)
    const int head = item % a.n_h;
    const int4 todo = a.merges[item / a.n_h];
    const int32_t row = todo.x, first_slot = todo.y, u0 = todo.y >> 1, n = todo.z;
    if (n < 2) return;
    const int64_t at_out = ((int64_t)row * a.n_h + head) * DH + lane * N;
    uint32_t gate[N / 2];
#pragma unroll
    for (int d = 0; d < N / 2; ++d) gate[d] = __ldg(reinterpret_cast<const uint32_t*>(a.g1 + at_out) + d);
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
    const float inv = 1.0f / l;
#pragma unroll
    for (int d = 0; d < N; d += 2)
        reinterpret_cast<uint32_t*>(a.out + at_out)[d / 2] =
            pack_bf16(o[d] * inv * gate_of(__uint_as_float(gate[d / 2] << 16)), o[d + 1] * inv * gate_of(__uint_as_float(gate[d / 2] & 0xFFFF0000u)));
}

int32_t unit_count(const gsa_params_t& p) { return sm_count() * (kWarps / p.n_kv); }

template <int DH, int G, int NKV>
cudaError_t launch_main(const CacheAttnArgs& a, cudaStream_t st) {
    static std::atomic<uint64_t> granted{0};
    constexpr size_t fixed = fixed_smem<DH, NKV>();
    cudaError_t e = grant_smem(granted, reinterpret_cast<const void*>(gsa_cache_attn_kernel<DH, G, NKV>), fixed + row_table_bytes(kMaxSplitRows));
    if (e != cudaSuccess) return e;
    e = launch_chained(gsa_cache_attn_kernel<DH, G, NKV>, (unsigned)(a.own ? a.rows : a.units / (kWarps / NKV)), kWarps * 32, fixed + row_table_bytes(a.own ? 1 : a.rows), st, a);
    ++g_launches;
    return e != cudaSuccess ? e : cudaGetLastError();
}
template <int DH, int G>
cudaError_t launch_heads(const CacheAttnArgs& a, cudaStream_t st) {
    switch (a.c.n_kv) {
        case 1: return launch_main<DH, G, 1>(a, st);
        case 2: return launch_main<DH, G, 2>(a, st);
        case 4: return launch_main<DH, G, 4>(a, st);
        case 8: return launch_main<DH, G, 8>(a, st);
    }
    return cudaErrorInvalidValue;
}
template <int DH>
cudaError_t launch_groups(const CacheAttnArgs& a, cudaStream_t st) {
    switch (a.n_h / a.c.n_kv) {
        case 1: return launch_heads<DH, 1>(a, st);
        case 2: return launch_heads<DH, 2>(a, st);
        case 4: return launch_heads<DH, 4>(a, st);
        case 8: return launch_heads<DH, 8>(a, st);
    }
    return cudaErrorInvalidValue;
}

template <int DH, int WPI>
cudaError_t launch_merge(const CacheAttnArgs& a, cudaStream_t st) {
    const int32_t items = a.merge_items * a.n_h, per = kMergeWarps / WPI;
    cudaError_t e = launch_chained(gsa_cache_merge_kernel<DH, WPI>, (unsigned)((items + per - 1) / per + 1), kMergeWarps * 32, 0, st, a,
                                   a.units / (kWarps / a.c.n_kv));
    ++g_launches;
    return e != cudaSuccess ? e : cudaGetLastError();
}

struct Plan { size_t stats, merges, flags, total; };
Plan plan_scratch(const gsa_params_t& p) {
    const size_t slots = 2 * (size_t)unit_count(p);
    const int64_t rows = (int64_t)p.B * p.Lq, borders = unit_count(p);
    Plan w;
    w.stats = align_up(slots * p.n_h * p.d_h * 4, 256);
    w.merges = w.stats + align_up(slots * p.n_h * 8, 256);
    w.flags = w.merges + align_up((size_t)(rows < borders ? rows : borders) * 16, 256);
    w.total = w.flags + align_up((size_t)sm_count() * 4, 256);
    return w;
}

}  // namespace

size_t cache_attn_scratch_bytes(const gsa_params_t& p) { return plan_scratch(p).total; }

cudaError_t launch_cache_attn(const CacheView& c, const gsa_params_t& p, const __nv_bfloat16* Q, const __nv_bfloat16* g1,
                              const int32_t* idx, const int32_t* kt, __nv_bfloat16* out, int32_t* ws, cudaStream_t st) {
    CacheAttnArgs a{};
    a.c = c; a.Lq = p.Lq; a.Lk = p.Lk; a.n_h = p.n_h; a.k_max = p.k_max;
    a.scale_log2 = (p.sm_scale > 0.f ? p.sm_scale : 1.0f / sqrtf((float)p.d_h)) * 1.4426950408889634f;
    const Plan w = plan_scratch(p);
    char* s = (char*)ws + kStatusBytes;
    a.status = ws; a.state = (float*)s; a.stats = (float2*)(s + w.stats); a.merges = (int4*)(s + w.merges); a.flags = (int32_t*)(s + w.flags);
    const int32_t all = p.B * p.Lq, subs = kWarps / p.n_kv;
    // A CTA for each row, or equal runs and a merge?  A tile takes some 1.5 us where all sixteen warps of an SM have one, the merge 2 to 4.
    // Measured (us in a graph, sets of k keys; own CTA / runs), up to 32 rows: 8 KV heads of 128, k 32 7.0 / 8.8, 64 9.1 / 8.4; two of 128, 128
    // 7.9 / 8.4, 256 10.9 / 8.0; one of 64, 256 6.8 / 7.5, 512 8.3 / 7.2;  128 rows: 8 of 128, 64 9.9 / 11.9; two of 128, 256 11.1 / 16.9.
    if (all <= sm_count() && (p.k_max + kTile - 1) / kTile <= (2 * all >= sm_count() ? kManyOwnTiles : kOwnTiles) * subs) {
        a.own = 1; a.rows = all;
        a.Q = Q; a.g1 = g1; a.out = out; a.idx = idx; a.kt = kt;
        return p.d_h == 128 ? launch_groups<128>(a, st) : launch_groups<64>(a, st);
    }
    for (int32_t r0 = 0; r0 < all; r0 += kMaxSplitRows) {
        const int64_t at = (int64_t)r0 * p.n_h * p.d_h;
        a.row0 = r0; a.rows = all - r0 < kMaxSplitRows ? all - r0 : kMaxSplitRows;
        a.Q = Q + at; a.g1 = g1 + at; a.out = out + at; a.idx = idx + (int64_t)r0 * p.k_max; a.kt = kt + r0;
        // no more CTAs than the largest sets would keep busy, one unit each to begin with
        const int32_t most = units_for((int64_t)a.rows * ((p.k_max + kTile - 1) / kTile), unit_count(p));
        a.units = (most < sm_count() ? most : sm_count()) * subs;
        a.by_cut = a.rows > a.units - 1 ? 1 : 0;
        a.merge_items = a.by_cut ? a.units - 1 : a.rows;
        cudaError_t e = p.d_h == 128 ? launch_groups<128>(a, st) : launch_groups<64>(a, st);
        if (e != cudaSuccess) return e;
        const bool many = !a.by_cut && a.units >= 8 * a.rows;      // parts of a row: eight or more
        if (p.d_h == 128) e = many ? launch_merge<128, 8>(a, st) : launch_merge<128, 1>(a, st);
        else e = many ? launch_merge<64, 8>(a, st) : launch_merge<64, 1>(a, st);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace gsa
