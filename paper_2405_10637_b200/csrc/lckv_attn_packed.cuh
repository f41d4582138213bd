// Decode attention over rows held in 4 bits (lckv_packed.cuh states the layout).
//
//   s_j   = scale * sum_g ( step_jg * sum_{d in g} q_d c_jd  +  low_jg * sum_{d in g} q_d )          c: codes 0 .. 15
//   out_d = sum_j p_j (low_jg + step_jg c_jd) / sum_j p_j
//
// A row of D = 128 is 144 bytes for key and value together, so the bound is the memory only if a code costs less than an
// instruction.  Codes therefore go to the tensor cores (fp16 m16n8k16, fp32 accumulation) as they are: a nibble c in bits 0 .. 3
// of a 16-bit half IS the fp16 subnormal c * 2^-24, one in bits 4 .. 7 c * 2^-20, so a mask is the whole conversion of two codes;
// every second row of the other operand (or of the result) carries the factor 16.  Nothing is rounded on the way in: codes are
// exact, q (bf16) enters scaled by a power of two, exact unless 2^-25 of the head's largest element or less, and steps and
// lows are applied in fp32 to the sums of a group.
//     S^T [tokens x 8] = C_K [tokens x d] . Q^T [d x 8]     tokens are the M dimension, as in lckv_attn_mma.cuh
//     O^T [d x 8]      = C_V^T [d x tokens] . W^T           W = p_j step_jg, one operand per group g
// W is p * step * 2^(14-e) in fp16, 2^e the power of two below the largest step seen so far (a row below 2^-28 of the largest
// weight loses bits, none overflows).
//
// Few query heads leave columns of the tile empty; they are used to share the work on the scores.  With QP = 2, 4 or 8
// columns for the heads of a pair, the tile holds NC = 8 / QP copies of them, and copy k (lanes 2 c4 / QP = k) does
// scaling, exponentials and weights only of every NC-th block of 16 rows.  The transposed weights then stand in the columns
// of their own copy, the columns of the others are zeroed per block, and the copies' outputs are added up at the end of a pair.
//
// EXACT (fp32 outputs).  Codes are all positive and lows all negative, more or less, so what is summed is far larger than the sums:
// scores come out with an error of up to 5e-6 and, where thousands of rows cancel, the tensor cores' truncation shows.  So codes enter as
// c - 8, which is exact too (one more instruction for two codes), with low + 8 step in place of low, W is split into a
// rounded part and the rounding of the rest (a second MMA), 22 bits, and blocks of 16 rows are added in fp32.
//
// bf16 outputs take codes as they are and one W of 11 bits, whose roundings are independent: with the output's own (2^-8 of it at most) the
// rms error over 200 to 32768 rows is 1.52e-3 to 1.82e-3 of the output, where rounding alone makes 1.49e-3 to 1.76e-3.  W in two parts
// would make that 1.49e-3 to 1.76e-3 and 32 x 32 heads of 256 to 4096 rows 66 -> 74 us, 48 x 52 of 4096 245 -> 289, 128 x 4 of 64 19.7 -> 21.1.
// What must not stay is the truncation: it has one sign, so it grows with the rows that a warp sums while what is left of the sums shrinks
// (32768 rows in one warp, eight heads: 3.7e-2 of the output).  So a tile's four blocks are summed by the tensor cores and tiles in fp32
// (48 x 52 heads 238 -> 245 us, the others 0 to 2 %).
//
// Work: a launch is one long sequence of tiles of 64 rows, (sequence, pair, tile), cut into one range per thread block and
// those into one per worker (warp).  A pair that several warps of a block share is joined behind a block barrier; only what
// crosses blocks, at most the first and the last pair of each, takes records, tickets and merging as in lckv_attn_mma.cuh, which
// costs 3 us.  Where whole pairs fill the blocks about as evenly (all rule and no exception with equal lengths),
// blocks are cut between pairs and nothing crosses.  A worker has a ring of whole tiles: keys, values and parameters of
// 64 rows arrive as one bulk copy (the last rows of a sequence as three).
#pragma once
#include "lckv_attn_mma.cuh"
#include "lckv_packed.cuh"

namespace lckv {

#ifndef LCKV_PACKED_WARPS_128
#define LCKV_PACKED_WARPS_128 12
#endif
#ifndef LCKV_PACKED_WARPS_64
#define LCKV_PACKED_WARPS_64 16
#endif
#ifndef LCKV_PACKED_SLOTS
#define LCKV_PACKED_SLOTS 2
#endif
constexpr int kPackedSlots = LCKV_PACKED_SLOTS;   // tiles in a worker's ring
// Workers per thread block, one block per SM.  D = 128: as many rings of two tiles as fit (48 x 52 heads x 4096 rows 238 us; 8 workers with three
// tiles each 285).  D = 64: 16, as many as 128 registers a thread allow (128 x 4 kv heads x 1024 rows 17.0 us, 12 workers 19.5).
__host__ __device__ constexpr int packed_warps(int d) { return d == 128 ? LCKV_PACKED_WARPS_128 : LCKV_PACKED_WARPS_64; }
template <int D>
__host__ __device__ constexpr int packed_smem_bytes() { return packed_warps(D) * kPackedSlots * (packed_tile_bytes<D>() + 8) + 128; }

__device__ __forceinline__ void mma_f16_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// {lo, hi} -> packed f16x2 (round to nearest even), lo in the low half; and back
__device__ __forceinline__ uint32_t cvt_f16x2(float lo, float hi)
{
    uint32_t d;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
__device__ __forceinline__ void f16x2_floats(uint32_t v, float& lo, float& hi)
{
    asm("{\n\t.reg .f16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}" : "=f"(lo), "=f"(hi) : "r"(v));
}

__device__ __forceinline__ uint2 lds64(uint32_t addr)
{
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t lds32(uint32_t addr)
{
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}

// A query head as the B operand of the score MMAs.  EXACT: for codes c - 8.
template <int D, bool EXACT>
struct PackedQuery {
    uint32_t b[D / 16][2];
    float f[2];              // per column of this lane: softmax scale * log2(e) / the scaling of q and codes
    float sum[2][D / 64];    // sum of q over a group * softmax scale * log2(e)
};

// raw[j]: dimensions 32 j + 8 c4 .. + 7 of the query of column g4.
template <int D, bool EXACT>
__device__ __forceinline__ void packed_query(const uint4 (&raw)[D / 32], float scale_log2, int lane, PackedQuery<D, EXACT>& out)
{
    const uint32_t FULL = 0xffffffffu;
    const int c4 = lane & 3;
    float mx = 0.f, sum[D / 64];
#pragma unroll
    for (int g = 0; g < D / 64; ++g) sum[g] = 0.f;
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
        const uint32_t w[4] = {raw[j].x, raw[j].y, raw[j].z, raw[j].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            mx = fmaxf(mx, fmaxf(fabsf(bf16lo(w[i])), fabsf(bf16hi(w[i]))));
            sum[j / 2] += bf16lo(w[i]) + bf16hi(w[i]);
        }
    }
#pragma unroll
    for (int off = 1; off <= 2; off <<= 1) {
        mx = fmaxf(mx, __shfl_xor_sync(FULL, mx, off));
#pragma unroll
        for (int g = 0; g < D / 64; ++g) sum[g] += __shfl_xor_sync(FULL, sum[g], off);
    }
    // largest element to [2^14, 2^15)
    const int up = max(-100, min(100, 14 + 127 - (int)(__float_as_uint(mx) >> 23)));
    const float by = __uint_as_float((uint32_t)(up + 127) << 23), by16 = EXACT ? by : by * 0.0625f;
    const float f = scale_log2 * __uint_as_float((uint32_t)((EXACT ? 0 : 24) - up + 127) << 23);
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
        // nibble i and nibble i + 4 of a word share a register; odd i count 16 times as much (not EXACT)
        const uint32_t w[4] = {raw[j].x, raw[j].y, raw[j].z, raw[j].w};
        out.b[2 * j][0] = cvt_f16x2(bf16lo(w[0]) * by, bf16lo(w[2]) * by);
        out.b[2 * j][1] = cvt_f16x2(bf16hi(w[0]) * by16, bf16hi(w[2]) * by16);
        out.b[2 * j + 1][0] = cvt_f16x2(bf16lo(w[1]) * by, bf16lo(w[3]) * by);
        out.b[2 * j + 1][1] = cvt_f16x2(bf16hi(w[1]) * by16, bf16hi(w[3]) * by16);
    }
    // columns of this lane's accumulators: 2 c4 and 2 c4 + 1
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int src = (2 * c4 + i) * 4;
        out.f[i] = __shfl_sync(FULL, f, src);
#pragma unroll
        for (int g = 0; g < D / 64; ++g) out.sum[i][g] = __shfl_sync(FULL, sum[g], src) * scale_log2;
    }
}

// What a group's codes count from: 0, or EXACT 8.
template <bool EXACT>
__device__ __forceinline__ float packed_low(uint32_t par) { return EXACT ? fmaf(8.f, bf16lo(par), bf16hi(par)) : bf16hi(par); }

// The four fp16 pairs of a word: nibbles (0, 4), (1, 5) x 16, (2, 6), (3, 7) x 16.
__device__ __forceinline__ void nibble_pairs(uint32_t w, uint32_t (&x)[4])
{
    x[0] = w & 0x000f000fu;
    x[1] = w & 0x00f000f0u;
    const uint32_t y = w >> 8;
    x[2] = y & 0x000f000fu;
    x[3] = y & 0x00f000f0u;
}

// ... and as whole numbers c - 8, exact: 1024 + c and 1024 + 16 c are the fp16 numbers with these bits in the mantissa.
__device__ __forceinline__ void nibble_pairs_signed(uint32_t w, uint32_t (&x)[4])
{
    const uint32_t y = w >> 8;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(x[0]) : "r"((w & 0x000f000fu) | 0x64006400u), "r"(0x64086408u));
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(x[1]) : "r"((w & 0x00f000f0u) | 0x64006400u), "r"(0x2c002c00u), "r"(0xd480d480u));
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(x[2]) : "r"((y & 0x000f000fu) | 0x64006400u), "r"(0x64086408u));
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(x[3]) : "r"((y & 0x00f000f0u) | 0x64006400u), "r"(0x2c002c00u), "r"(0xd480d480u));
}

template <bool EXACT>
__device__ __forceinline__ void nibbles(uint32_t w, uint32_t (&x)[4])
{
    if constexpr (EXACT) nibble_pairs_signed(w, x);
    else nibble_pairs(w, x);
}

// Token of row i (0 .. 7) of an MMA tile: pairs are swapped where bit 1 is set, so that the four tokens that a value load of a
// warp touches lie in both halves of the 32 banks.
__device__ __forceinline__ int packed_token(int i) { return i ^ ((i >> 1) & 1); }

struct PackedParams {
    MmaParams m;         // a.K, a.V, a.pre and a.start unused; a.H_q = pairs per sequence
    PackedSlot s;
    int64_t pitch;       // rows of a (sequence, kv head)
    int32_t n_blocks, n_warps;   // thread blocks and warps of each that work
    int32_t pairs_per_block;     // ceil(all pairs / n_blocks)
    uint32_t warps_inverse;      // ceil(2^32 / n_warps)
};

// Position in a launch's tile sequence, in (b, pair, tile) order; pair h = kvh * (pairs per kv head) + sub.
struct PackedCursor {
    int32_t b, kvh, sub;
    uint32_t t, nt;      // tile within the pair; tiles per pair of sequence b
    int32_t nv;          // visible rows of sequence b
};

// (Ordinary loads: the lengths may come from the kernel in front, which this one overlaps.)
__device__ __forceinline__ int32_t packed_visible(const AttnParams& p, int b) { return visible_rows(p.lens[b], p.mode, p.T_cap); }
__device__ __forceinline__ uint32_t packed_tiles(int32_t nv) { return (uint32_t)(nv + kPackedRows - 1) / kPackedRows; }

// Next tile, skipping sequences without tiles.  Safe past the end.
__device__ __forceinline__ void packed_next(PackedCursor& c, const AttnParams& p, int per_kv)
{
    if (++c.t < c.nt) return;
    c.t = 0;
    if (++c.sub < per_kv) return;
    c.sub = 0;
    if (++c.kvh < p.H_kv) return;
    c.kvh = 0;
    do {
        if (++c.b >= p.B) { c.b = p.B; c.nt = 0; c.nv = 0; return; }
        c.nv = packed_visible(p, c.b);
        c.nt = packed_tiles(c.nv);
    } while (c.nt == 0);
}

// n things cut into parts of `each`, the first `more` with one more.
struct PackedShare {
    uint32_t each, more;
    __device__ __forceinline__ PackedShare(uint32_t n, uint32_t parts) : each(n / parts), more(n - n / parts * parts) {}
    __device__ __forceinline__ uint32_t begin(uint32_t w) const { return w * each + min(w, more); }
    __device__ __forceinline__ uint32_t part(uint32_t i) const
    {
        const uint32_t longer = more * (each + 1);
        return i < longer ? i / (each + 1) : more + (i - longer) / each;
    }
};
// The tiles in front of every sequence, per pair of a sequence: before[i] of those in front of sequence i * per (per = 1 up to
// kPackedTable sequences; with more, a stretch of `per` sequences is walked through where it is needed).
constexpr int kPackedTable = 1024;
struct PackedTable {
    uint32_t before[kPackedTable + 1];
    int32_t rows[kPackedTable];   // visible rows (per = 1)
    uint32_t sums[32], longest[32];
};

// The block's threads fill the table; returns the longest sequence's tiles.  Up to 32 sequences every warp fills it by itself (all
// write the same), without waiting for the others.
template <int THREADS>
__device__ __forceinline__ uint32_t packed_table(const AttnParams& p, int per, PackedTable& t)
{
    const uint32_t FULL = 0xffffffffu;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    constexpr int EACH = (kPackedTable + THREADS - 1) / THREADS;     // entries of a thread, side by side
    const int n = (p.B + per - 1) / per;
    if (p.B <= 32) {
        const int32_t nv = lane < p.B ? packed_visible(p, lane) : 0;
        const uint32_t nt = packed_tiles(nv);
        uint32_t incl = nt;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const uint32_t x = __shfl_up_sync(FULL, incl, off);
            if (lane >= off) incl += x;
        }
        t.rows[lane] = nv;
        t.before[lane] = incl - nt;
        if (lane == 31) t.before[32] = incl;
        __syncwarp();
        return __reduce_max_sync(FULL, nt);
    }
    uint32_t mine[EACH], sum = 0, longest = 0;
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
        const int i = (int)threadIdx.x * EACH + e;
        mine[e] = 0;
        if (i < n) {
            for (int b = i * per; b < min(p.B, (i + 1) * per); ++b) {
                const int32_t nv = packed_visible(p, b);
                const uint32_t nt = packed_tiles(nv);
                if (per == 1) t.rows[i] = nv;
                mine[e] += nt;
                longest = max(longest, nt);
            }
        }
        sum += mine[e];
    }
    uint32_t incl = sum;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const uint32_t x = __shfl_up_sync(FULL, incl, off);
        if (lane >= off) incl += x;
    }
    longest = __reduce_max_sync(FULL, longest);
    if (lane == 31) { t.sums[warp] = incl; t.longest[warp] = longest; }
    __syncthreads();
    uint32_t at = incl - sum + __reduce_add_sync(FULL, lane < warp ? t.sums[lane] : 0u);
    longest = __reduce_max_sync(FULL, lane < THREADS / 32 ? t.longest[lane] : 0u);
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
        const int i = (int)threadIdx.x * EACH + e;
        if (i <= n) t.before[i] = at;
        at += mine[e];
    }
    if (threadIdx.x == THREADS - 1 && n == THREADS * EACH) t.before[n] = at;
    __syncthreads();
    return longest;
}

// What a warp does: from the table, by itself.
struct PackedRange {
    uint32_t all;                 // tiles of the launch
    uint32_t begin, end;          // the thread block's
    uint32_t first, count;        // the warp's
    bool whole;                   // blocks are cut between pairs
};
__device__ __forceinline__ PackedRange packed_range(const PackedParams& pp, const PackedTable& t, int per, uint32_t longest, uint32_t block, uint32_t warp,
                                                    int lane, PackedCursor& c)
{
    const AttnParams& p = pp.m.a;
    const uint32_t FULL = 0xffffffffu, H = (uint32_t)p.H_q;
    const int n = (p.B + per - 1) / per;
    PackedRange r;
    r.all = t.before[n] * H;
    // Blocks cut between pairs, if that leaves a warp at most about one tile more than an even cut: a tile is 1 us, records and
    // tickets 3.
    const uint32_t pairs = (uint32_t)p.B * H, blocks = (uint32_t)pp.n_blocks, warps = (uint32_t)pp.n_warps, per_block = (uint32_t)pp.pairs_per_block;
    r.whole = (uint64_t)per_block * longest * blocks <= (uint64_t)r.all + blocks * warps;
    if (r.whole) {
        const auto tiles_before = [&](uint32_t pair) {
            const int b = (int)(pair / H);
            if (b >= p.B) return r.all;
            const int i = b / per;
            uint32_t x = t.before[i];
            for (int k = i * per; k < b; ++k) x += packed_tiles(packed_visible(p, k));
            const uint32_t nt = per == 1 ? t.before[i + 1] - x : packed_tiles(packed_visible(p, b));
            return x * H + (pair - (uint32_t)b * H) * nt;
        };
        r.begin = tiles_before(min(pairs, block * per_block));
        r.end = tiles_before(min(pairs, (block + 1) * per_block));
    } else {
        const PackedShare share(r.all, blocks);
        r.begin = block < blocks ? share.begin(block) : 0u;
        r.end = block < blocks ? share.begin(block + 1) : 0u;
    }
    // n / warps by the inverse, which is too large by less than 16 in 2^32: from 2^28 tiles on the quotient may be one too many
    const uint32_t n_block = r.end - r.begin;
    uint32_t each = warps == 1 ? n_block : __umulhi(n_block, pp.warps_inverse), more = n_block - each * warps;
    if ((int32_t)more < 0) { --each; more += warps; }
    r.first = r.begin + warp * each + min(warp, more);
    r.count = warp < warps ? each + (warp < more ? 1u : 0u) : 0u;
    if (r.count == 0) return r;
    // the last entry whose tiles begin at or in front of x: 32 entries apart, then one by one
    const uint32_t x = r.first / H;
    int i = 32 * (31 - __clz(__ballot_sync(FULL, 32 * lane < n && t.before[min(32 * lane, n)] <= x)));
    i += 31 - __clz(__ballot_sync(FULL, i + lane < n && t.before[min(i + lane, n)] <= x));
    uint32_t base = t.before[i];
    c.b = i;
    if (per == 1) {
        c.nv = t.rows[i];
    } else {
        c.b = i * per;
        for (;;) {
            c.nv = packed_visible(p, c.b);
            const uint32_t nt = packed_tiles(c.nv);
            if (x < base + nt) break;
            base += nt;
            ++c.b;
        }
    }
    c.nt = packed_tiles(c.nv);
    const uint32_t rel = r.first - base * H, h = rel / c.nt;
    c.t = rel - h * c.nt;
    c.kvh = (int)h / pp.m.groups_per_kv;
    c.sub = (int)h - c.kvh * pp.m.groups_per_kv;
    return r;
}

// Part of a pair that a warp leaves to be joined: the pair's first tile, its tiles (0: none), sequence, number, and whether the
// part is in the warp's ring (else in its first record: its ring was still in use).
struct PackedPart { uint32_t begin, nt; int32_t b, h, in_ring; };

template <int D, bool PAGED, int QP, bool EXACT>
__global__ void __launch_bounds__(packed_warps(D) * 32, 1) attn_packed_kernel(const PackedParams pp)
{
    constexpr int R = kPackedRows;
    constexpr int RB = R / 16;                   // 16-row blocks of a tile
    constexpr int J = D / 32;                    // words of a key row per lane
    constexpr int G = D / 64;                    // groups
    constexpr int MT = D / 16;                   // 16-dimension m-tiles of the output MMA
    constexpr int NC = 8 / QP;                   // copies of the pair's heads in a tile's columns
    constexpr int NB = RB / NC;                  // blocks whose scores a lane works on
    constexpr int NS = kPackedSlots;
    constexpr int WARPS = packed_warps(D);
    constexpr int TILE = packed_tile_bytes<D>();
    constexpr int CODES = R * (D / 2);           // bytes of a tile's keys; its values follow, then the parameters
    constexpr int MTL = MT / NC;                 // m-tiles of a finished pair that a lane holds
    constexpr int REC = D * 8 + 16;
    const AttnParams& p = pp.m.a;
    const int HP = pp.m.heads_per_pair, per_kv = pp.m.groups_per_kv, n_q_heads = pp.m.n_q_heads;

    extern __shared__ uint8_t smem_raw[];
    __shared__ PackedPart parts[WARPS][2];
    __shared__ PackedTable table;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int w = blockIdx.x * WARPS + warp;
    const uint32_t FULL = 0xffffffffu;
    const int g4 = lane >> 2, c4 = lane & 3;
    const int copy = 2 * c4 / QP;                // the copy that this lane's columns belong to

    const uint32_t smem0 = (smem_u32(smem_raw) + 127u) & ~127u;
    const uint32_t ring = smem0 + warp * (NS * TILE);
    uint8_t* const ring0 = smem_raw + (smem0 - smem_u32(smem_raw));
    uint8_t* const ring_bytes = ring0 + warp * (NS * TILE);
    static_assert(REC * 4 <= NS * TILE, "a record fits a ring");
    const uint32_t bars = smem0 + WARPS * NS * TILE + warp * (NS * 8);
    if (lane == 0) {
        for (int s = 0; s < NS; ++s) mbar_init(bars + 8 * s, 1);
        fence_mbar_init();
        parts[warp][0].nt = parts[warp][1].nt = 0;
    }
    __syncwarp();

    if (!p.early_kv) pdl_wait_then_release();

    PackedCursor cc = {0, 0, 0, 0u, 0u, 0};
    const int per = (p.B + kPackedTable - 1) / kPackedTable;
    const uint32_t longest = packed_table<WARPS * 32>(p, per, table);
    const PackedRange range = packed_range(pp, table, per, longest, blockIdx.x, (uint32_t)warp, lane, cc);
    const uint32_t n_tiles = range.count;
    PackedCursor ci = cc;

    const int head = min(g4 % QP, HP - 1);       // of the column g4; columns without a head repeat the last one's query
    auto query_of = [&](const PackedCursor& c) {
        return p.q + ((size_t)c.b * n_q_heads + (size_t)(c.kvh * per_kv + c.sub) * HP + head) * D + 8 * c4;
    };
    const uint64_t l2pol = make_l2_policy(p.l2_keep);
    uint32_t issued = 0, islot = 0;
    PageWalker walker;
    auto issue = [&]() {
        int64_t row;
        if constexpr (PAGED) row = max((int64_t)0, walker.row(p, ci.b, ci.kvh, (int)ci.t * R));   // (a row without a page: any row)
        else row = ((int64_t)ci.b * p.H_kv + ci.kvh) * pp.pitch + (int64_t)ci.t * R;
        if (lane == 0) {
            const uint32_t bar = bars + 8 * islot, dst = ring + islot * TILE;
            const uint8_t* src = pp.s.tile<D>(row);
            const int left = ci.nv - (int)ci.t * R;
            if (left >= R) {
                mbar_expect_tx(bar, TILE);
                bulk_g2s_hint(dst, src, TILE, bar, l2pol);
            } else {
                // (an even number of rows: a row's parameters are 8 bytes where D = 64)
                const uint32_t rows = ((uint32_t)left + 1u) & ~1u;
                mbar_expect_tx(bar, rows * (D + D / 8));
                bulk_g2s_hint(dst, src, rows * (D / 2), bar, l2pol);
                bulk_g2s_hint(dst + 2 * CODES, src + 2 * CODES, rows * (8 * G), bar, l2pol);
                bulk_g2s_hint(dst + CODES, src + CODES, rows * (D / 2), bar, l2pol);
            }
        }
        packed_next(ci, p, per_kv);
        ++issued;
        islot = (islot + 1 == NS) ? 0 : islot + 1;
    };
    // The first pair's queries are asked for in front of the tiles (behind those of 12 workers they arrived after 4800 cycles),
    // unless only the tiles may be read yet.
    uint4 q_raw[J];
    auto load_q = [&]() {                        // the query heads of pair cc, NC times
        const uint4* src = reinterpret_cast<const uint4*>(query_of(cc));
#pragma unroll
        for (int j = 0; j < J; ++j) q_raw[j] = src[4 * j];
    };
    if (!p.early_kv && n_tiles) load_q();
    {
        const uint32_t pro = n_tiles < (uint32_t)NS ? n_tiles : (uint32_t)NS;
        while (issued < pro) issue();
    }
    if (p.early_kv) {
        pdl_wait_then_release();
        if (n_tiles) load_q();
    }

    // Sequences that see nothing: zero rows (zero dummy key and value), lse 0.
    for (int b = w; b < p.B; b += gridDim.x * WARPS) {
        if (packed_visible(p, b) == 0) {
            const int n16 = n_q_heads * D * (EXACT ? 4 : 2) / 16;
            uint4* o16 = reinterpret_cast<uint4*>(static_cast<uint8_t*>(p.out) + (size_t)b * n16 * 16);
            for (int i = lane; i < n16; i += 32) o16[i] = make_uint4(0, 0, 0, 0);
            if (p.lse)
                for (int i = lane; i < n_q_heads; i += 32) p.lse[(size_t)b * n_q_heads + i] = 0.f;
        }
    }

    uint32_t cslot = 0, cphase = 0;
    bool ok = true;

    PackedQuery<D, EXACT> q;
    if (n_tiles) packed_query<D, EXACT>(q_raw, p.scale_log2, lane, q);

    // running state of this lane's two columns
    float m_run[2], l_run[2];
    float low_sum[G][2];                         // sum of p * low (EXACT: low + 8 step) over this lane's rows
    float o[MT][4];
    int e_run;                                   // units of o: EXACT 2^(e_run - 14), else 2^(e_run + 10), odd dimensions 2^(e_run + 6)
    auto clear = [&]() {
        m_run[0] = m_run[1] = -INFINITY;
        l_run[0] = l_run[1] = 0.f;
        e_run = -100;
#pragma unroll
        for (int g = 0; g < G; ++g) low_sum[g][0] = low_sum[g][1] = 0.f;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[mt][i] = 0.f;
    };
    clear();
    uint32_t seg_t0 = cc.t;

    bool first_seg = true;
    // A finished part of a pair: the lanes of a row's copies share its dimensions.  r[i] are the values of m-tile copy * MTL + i,
    // [0], [1] of dimension 64 g + 8 g4 + 2 k for the lane's two columns, [2], [3] of the one behind it, with 4 g + k the m-tile.
    float r[MTL][4], l_tot[2], m_fin[2];
    const int q0 = 2 * c4 % QP;                  // the lane's columns: query heads q0 and q0 + 1 of the pair
    const bool holds = q0 < HP, both = q0 + 1 < HP;

    // m-tile copy * MTL + i of r / l_tot -> the output rows of pair (b, h), N of them whose dimensions are neighbours; with the first, lse
    auto write_tiles = [&](auto n_tag, const float (*v)[4], int i, int b, int h) {
        constexpr int N = decltype(n_tag)::value;
        const size_t row0 = (size_t)b * n_q_heads + (size_t)h * HP + q0;
        const int mt = copy * MTL + i;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            if (j == 0 ? !holds : !both) break;
            const float inv = 1.0f / l_tot[j];
            const size_t at = (row0 + j) * D + 64 * (mt / 4) + 8 * g4 + 2 * (mt % 4);
            [[maybe_unused]] uint32_t y[N];
#pragma unroll
            for (int e = 0; e < N; ++e) {
                if constexpr (EXACT) *reinterpret_cast<float2*>(static_cast<float*>(p.out) + at + 2 * e) = make_float2(v[e][j] * inv, v[e][2 + j] * inv);
                else y[e] = cvt_bf16x2(v[e][j] * inv, v[e][2 + j] * inv);
            }
            if constexpr (!EXACT) {
                uint16_t* dst = static_cast<uint16_t*>(p.out) + at;
                if constexpr (N == 4) *reinterpret_cast<uint4*>(dst) = make_uint4(y[0], y[1], y[2], y[3]);
                else if constexpr (N == 2) *reinterpret_cast<uint2*>(dst) = make_uint2(y[0], y[1]);
                else *reinterpret_cast<uint32_t*>(dst) = y[0];
            }
            if (i == 0 && p.lse && g4 == 0 && copy == 0) p.lse[row0 + j] = (m_fin[j] + lg2(l_tot[j])) * 0.6931471805599453f;
        }
    };
    // m-tile i of a record, and its maxima and sums
    auto store_tile = [&](float* rec, int i, const float (&v)[4]) {
        reinterpret_cast<float4*>(rec)[i * 32 + lane] = make_float4(v[0], v[1], v[2], v[3]);
        if (i == 0 && g4 == 0 && copy == 0) {
            *reinterpret_cast<float2*>(rec + MTL * 128 + q0) = make_float2(m_fin[0], m_fin[1]);
            *reinterpret_cast<float2*>(rec + MTL * 128 + 8 + q0) = make_float2(l_tot[0], l_tot[1]);
        }
    };
    // One more record's m-tile, with a running maximum
    auto begin_join = [&](float (&v)[4]) {
        m_fin[0] = m_fin[1] = -INFINITY;
        l_tot[0] = l_tot[1] = 0.f;
        v[0] = v[1] = v[2] = v[3] = 0.f;
    };
    auto join = [&](float (&v)[4], float2 m, float2 l, float4 x) {
        const float M0 = fmaxf(m_fin[0], m.x), M1 = fmaxf(m_fin[1], m.y);
        const float a0 = ex2(m_fin[0] - M0), a1 = ex2(m_fin[1] - M1);      // ex2(-inf) = 0 for the first record
        const float w0 = ex2(m.x - M0), w1 = ex2(m.y - M1);
        m_fin[0] = M0; m_fin[1] = M1;
        l_tot[0] = fmaf(l_tot[0], a0, l.x * w0);
        l_tot[1] = fmaf(l_tot[1], a1, l.y * w1);
        v[0] = fmaf(v[0], a0, x.x * w0);
        v[1] = fmaf(v[1], a1, x.y * w1);
        v[2] = fmaf(v[2], a0, x.z * w0);
        v[3] = fmaf(v[3], a1, x.w * w1);
    };

    for (uint32_t tile = 0; tile < n_tiles; ++tile) {
        const int rows = min(R, cc.nv - (int)cc.t * R);
        const bool pair_end = (cc.t + 1 == cc.nt), last = (tile + 1 == n_tiles);
        if (pair_end && !last) {                 // the next pair's queries come near while this pair's last tile is worked on
            PackedCursor cn = cc;
            packed_next(cn, p, per_kv);
            const uint16_t* next = query_of(cn);
#pragma unroll
            for (int j = 0; j < J; ++j) asm volatile("prefetch.global.L1 [%0];" ::"l"(next + 32 * j));
        }
        // (the whole warp gives up or none: what follows exchanges between its lanes, and a block barrier ends the kernel)
        if (!__all_sync(FULL, mbar_wait_bounded(bars + 8 * cslot, cphase, p.wait_limit))) { ok = false; break; }
        const uint32_t kc = ring + cslot * TILE, vc = kc + CODES, par = kc + 2 * CODES;
        const bool partial = rows < R;

        // ---- scores of this lane's rows in base-2 units; rows past the visible count -inf ----------
        float s[NB][4];
        uint32_t vp[NB][2][G];                   // parameters of the values of this lane's rows
        uint32_t top_step = 0;                   // largest step of a value's group (steps are not negative: bits compare)
        float mt_[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            float own[G][4];
#pragma unroll
            for (int k = 0; k < NC; ++k) {
                const int rb = i * NC + k;
                float acc[G][4];
#pragma unroll
                for (int g = 0; g < G; ++g)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[g][e] = 0.f;
                if (rb * 16 < rows) {
                    const int r0 = rb * 16 + packed_token(g4), r1 = r0 + 8;
                    uint32_t ka[J], kb[J];
                    if constexpr (D == 128) {
                        const uint4 a = lds128(kc + r0 * 64 + c4 * 16), b = lds128(kc + r1 * 64 + c4 * 16);
                        ka[0] = a.x; ka[1] = a.y; ka[2] = a.z; ka[3] = a.w;
                        kb[0] = b.x; kb[1] = b.y; kb[2] = b.z; kb[3] = b.w;
                    } else {
                        const uint2 a = lds64(kc + r0 * 32 + c4 * 8), b = lds64(kc + r1 * 32 + c4 * 8);
                        ka[0] = a.x; ka[1] = a.y;
                        kb[0] = b.x; kb[1] = b.y;
                    }
#pragma unroll
                    for (int j = 0; j < J; ++j) {
                        uint32_t xa[4], xb[4];
                        nibbles<EXACT>(ka[j], xa);
                        nibbles<EXACT>(kb[j], xb);
                        mma_f16_16816(acc[j / 2], xa[0], xb[0], xa[1], xb[1], q.b[2 * j][0], q.b[2 * j][1]);
                        mma_f16_16816(acc[j / 2], xa[2], xb[2], xa[3], xb[3], q.b[2 * j + 1][0], q.b[2 * j + 1][1]);
                    }
                }
#pragma unroll
                for (int g = 0; g < G; ++g)
#pragma unroll
                    for (int e = 0; e < 4; ++e) own[g][e] = k == 0 || copy == k ? acc[g][e] : own[g][e];
            }
            const int r0 = (i * NC + copy) * 16 + packed_token(g4), r1 = r0 + 8;
            uint32_t pa[2 * G], pb[2 * G];
            if constexpr (D == 128) {
                const uint4 x = lds128(par + r0 * 16), y = lds128(par + r1 * 16);
                pa[0] = x.x; pa[1] = x.y; pa[2] = x.z; pa[3] = x.w;
                pb[0] = y.x; pb[1] = y.y; pb[2] = y.z; pb[3] = y.w;
            } else {
                const uint2 x = lds64(par + r0 * 8), y = lds64(par + r1 * 8);
                pa[0] = x.x; pa[1] = x.y;
                pb[0] = y.x; pb[1] = y.y;
            }
            if (partial) {                       // what lies behind the last row was never copied
#pragma unroll
                for (int e = 0; e < 2 * G; ++e) {
                    if (r0 >= rows) pa[e] = 0;
                    if (r1 >= rows) pb[e] = 0;
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t* pr = e < 2 ? pa : pb;
                float t = bf16lo(pr[0]) * own[0][e], u = packed_low<EXACT>(pr[0]) * q.sum[e & 1][0];
                if constexpr (G == 2) {
                    t = fmaf(bf16lo(pr[1]), own[1][e], t);
                    u = fmaf(packed_low<EXACT>(pr[1]), q.sum[e & 1][1], u);
                }
                s[i][e] = fmaf(t, q.f[e & 1], u);
            }
            if (partial) {
                if (r0 >= rows) s[i][0] = s[i][1] = -INFINITY;
                if (r1 >= rows) s[i][2] = s[i][3] = -INFINITY;
            }
#pragma unroll
            for (int g = 0; g < G; ++g) {
                vp[i][0][g] = pa[G + g];
                vp[i][1][g] = pb[G + g];
                top_step = max(top_step, max(pa[G + g] << 16, pb[G + g] << 16));
            }
            mt_[0] = fmaxf(mt_[0], fmaxf(s[i][0], s[i][2]));
            mt_[1] = fmaxf(mt_[1], fmaxf(s[i][1], s[i][3]));
        }
#pragma unroll
        for (int off = QP / 2; off <= 16; off <<= 1) {      // the rows of a column: its copies' lanes and all g4
            mt_[0] = fmaxf(mt_[0], __shfl_xor_sync(FULL, mt_[0], off));
            mt_[1] = fmaxf(mt_[1], __shfl_xor_sync(FULL, mt_[1], off));
        }
        const int e_new = max(e_run, (int)(__reduce_max_sync(FULL, top_step) >> 23) - 127);
        float alpha[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const float m_new = fmaxf(m_run[j], mt_[j]);
            alpha[j] = ex2(m_run[j] - m_new);
            m_run[j] = m_new;
        }
        // (columns of o are those of the transposed weights: this lane's two, whatever the copy)
        float b0 = 1.f, b1 = 1.f;
        if (__any_sync(FULL, alpha[0] != 1.f || alpha[1] != 1.f || e_new != e_run)) {
            const float de = e_new - e_run > 120 ? 0.f : __uint_as_float((uint32_t)(e_run - e_new + 127) << 23);
            b0 = alpha[0] * de;
            b1 = alpha[1] * de;
            if constexpr (EXACT) {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    o[mt][0] *= b0; o[mt][1] *= b1;
                    o[mt][2] *= b0; o[mt][3] *= b1;
                }
            }
#pragma unroll
            for (int g = 0; g < G; ++g) { low_sum[g][0] *= alpha[0]; low_sum[g][1] *= alpha[1]; }
            l_run[0] *= alpha[0];
            l_run[1] *= alpha[1];
            e_run = e_new;
        }
        const float unit = __uint_as_float((uint32_t)(14 - e_run + 127) << 23);     // 2^(14 - e): 2^-113 .. 2^114

        // ---- weights of this lane's rows, transposed: columns of copy k hold block i NC + k -----------
        uint32_t bw[NB][G][2], br[NB][G][2];
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            const float p0 = ex2(s[i][0] - m_run[0]), p1 = ex2(s[i][1] - m_run[1]);
            const float p2 = ex2(s[i][2] - m_run[0]), p3 = ex2(s[i][3] - m_run[1]);
            l_run[0] += p0 + p2;
            l_run[1] += p1 + p3;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const uint32_t pa = vp[i][0][g], pb = vp[i][1][g];
                const float la = packed_low<EXACT>(pa), lb = packed_low<EXACT>(pb);
                low_sum[g][0] = fmaf(p0, la, fmaf(p2, lb, low_sum[g][0]));
                low_sum[g][1] = fmaf(p1, la, fmaf(p3, lb, low_sum[g][1]));
                const float sa = bf16lo(pa) * unit, sb = bf16lo(pb) * unit;
                const float w0 = p0 * sa, w1 = p1 * sa, w2 = p2 * sb, w3 = p3 * sb;
                const uint32_t x = cvt_f16x2(w0, w1), y = cvt_f16x2(w2, w3);
                bw[i][g][0] = movmatrix_trans(x);
                bw[i][g][1] = movmatrix_trans(y);
                if constexpr (EXACT) {
                    float h0, h1, h2, h3;
                    f16x2_floats(x, h0, h1);
                    f16x2_floats(y, h2, h3);
                    br[i][g][0] = movmatrix_trans(cvt_f16x2(w0 - h0, w1 - h1));
                    br[i][g][1] = movmatrix_trans(cvt_f16x2(w2 - h2, w3 - h3));
                }
            }
        }

        // ---- O^T += C_V^T . W^T -------------------------------------------------------------------
        [[maybe_unused]] float sum[EXACT ? 1 : MT][4];       // of this tile (EXACT adds blocks)
        if constexpr (!EXACT) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[mt][i] = 0.f;
        }
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            if (rb * 16 >= rows) continue;
            // tokens of the value loads: rows 2 c4, 2 c4 + 1 of the tile and the two eight further down
            const int t0 = rb * 16 + 2 * c4 + (c4 & 1), t1 = rb * 16 + 2 * c4 + 1 - (c4 & 1);
            uint32_t va[4][G];
            if constexpr (D == 128) {
                const uint2 x0 = lds64(vc + t0 * 64 + g4 * 8), x1 = lds64(vc + t1 * 64 + g4 * 8);
                const uint2 x2 = lds64(vc + (t0 + 8) * 64 + g4 * 8), x3 = lds64(vc + (t1 + 8) * 64 + g4 * 8);
                va[0][0] = x0.x; va[0][1] = x0.y; va[1][0] = x1.x; va[1][1] = x1.y;
                va[2][0] = x2.x; va[2][1] = x2.y; va[3][0] = x3.x; va[3][1] = x3.y;
            } else {
                va[0][0] = lds32(vc + t0 * 32 + g4 * 4);
                va[1][0] = lds32(vc + t1 * 32 + g4 * 4);
                va[2][0] = lds32(vc + (t0 + 8) * 32 + g4 * 4);
                va[3][0] = lds32(vc + (t1 + 8) * 32 + g4 * 4);
            }
            const bool mine = g4 / QP == rb % NC;            // is this lane's column one of the block's copy?
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const uint32_t b0 = mine ? bw[rb / NC][g][0] : 0u, b1 = mine ? bw[rb / NC][g][1] : 0u;
                const uint32_t r0 = EXACT && mine ? br[rb / NC][g][0] : 0u, r1 = EXACT && mine ? br[rb / NC][g][1] : 0u;
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    // nibbles 4 half .. 4 half + 3 of two tokens side by side
                    const uint32_t sel = half ? 0x7632u : 0x5410u;
                    uint32_t xa[4], xb[4];
                    const uint32_t lo = __byte_perm(va[0][g], va[1][g], sel), hi = __byte_perm(va[2][g], va[3][g], sel);
                    nibbles<EXACT>(lo, xa);
                    nibbles<EXACT>(hi, xb);
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int mt = 4 * g + 2 * half + i;
                        if constexpr (EXACT) {
                            // (the tensor cores truncate: a sum of 40 MMAs' results came out 40 * 2^-24 too small)
                            float t[4] = {0.f, 0.f, 0.f, 0.f};
                            mma_f16_16816(t, xa[2 * i], xa[2 * i + 1], xb[2 * i], xb[2 * i + 1], r0, r1);
                            mma_f16_16816(t, xa[2 * i], xa[2 * i + 1], xb[2 * i], xb[2 * i + 1], b0, b1);
#pragma unroll
                            for (int e = 0; e < 4; ++e) o[mt][e] += t[e];
                        } else {
                            mma_f16_16816(sum[mt], xa[2 * i], xa[2 * i + 1], xb[2 * i], xb[2 * i + 1], b0, b1);
                        }
                    }
                }
            }
        }
        if constexpr (!EXACT) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                const uint64_t by = pack_f32x2(b0, b1);
                unpack_f32x2(ffma2(pack_f32x2(o[mt][0], o[mt][1]), by, pack_f32x2(sum[mt][0], sum[mt][1])), o[mt][0], o[mt][1]);
                unpack_f32x2(ffma2(pack_f32x2(o[mt][2], o[mt][3]), by, pack_f32x2(sum[mt][2], sum[mt][3])), o[mt][2], o[mt][3]);
            }
        }
        __syncwarp();
        if (issued < n_tiles) issue();
        cslot = (cslot + 1 == NS) ? 0 : cslot + 1;
        if (cslot == 0) cphase ^= 1;

        // ---- end of this worker's part of the pair? -----------------------------------------
        if (pair_end || last) {
            const int h = cc.kvh * per_kv + cc.sub;
            l_tot[0] = l_run[0]; l_tot[1] = l_run[1];
#pragma unroll
            for (int off = QP / 2; off <= 16; off <<= 1) {
                l_tot[0] += __shfl_xor_sync(FULL, l_tot[0], off);
                l_tot[1] += __shfl_xor_sync(FULL, l_tot[1], off);
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    low_sum[g][0] += __shfl_xor_sync(FULL, low_sum[g][0], off);
                    low_sum[g][1] += __shfl_xor_sync(FULL, low_sum[g][1], off);
                }
            }
            m_fin[0] = m_run[0]; m_fin[1] = m_run[1];
            // the copies' parts, each lane ending up with its share of the dimensions
            if constexpr (NC == 1) {
#pragma unroll
                for (int i = 0; i < MTL; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) r[i][e] = o[i][e];
            } else {
                float half[MT / 2][4];
#pragma unroll
                for (int i = 0; i < MT / 2; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float keep = c4 & 2 ? o[i + MT / 2][e] : o[i][e], give = c4 & 2 ? o[i][e] : o[i + MT / 2][e];
                        half[i][e] = keep + __shfl_xor_sync(FULL, give, 2);
                    }
#pragma unroll
                for (int i = 0; i < MTL; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if constexpr (NC == 2) {
                            r[i][e] = half[i][e];
                        } else {
                            const float keep = c4 & 1 ? half[i + MTL][e] : half[i][e], give = c4 & 1 ? half[i][e] : half[i + MTL][e];
                            r[i][e] = keep + __shfl_xor_sync(FULL, give, 1);
                        }
                    }
            }
            // the units of o, and the lows
            const float pow_e = __uint_as_float((uint32_t)(e_run + 127) << 23);
#pragma unroll
            for (int i = 0; i < MTL; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float low = MTL == 8 ? low_sum[i / 4 % G][e & 1] : G == 2 && copy * MTL >= 4 ? low_sum[G - 1][e & 1] : low_sum[0][e & 1];
                    r[i][e] = fmaf(r[i][e] * (EXACT ? 0x1p-14f : e < 2 ? 0x1p10f : 0x1p6f), pow_e, low);
                }

            if (pair_end && seg_t0 == 0) {
                constexpr int N = MTL < 4 ? MTL : 4;
#pragma unroll
                for (int i = 0; i < MTL; i += N) write_tiles(std::integral_constant<int, N>(), r + i, i, cc.b, h);
            } else {                             // left to be joined
                const int k = first_seg ? 0 : 1;
                float* rec = last ? reinterpret_cast<float*>(ring_bytes) : p.partials + (size_t)(2 * w) * REC;
#pragma unroll
                for (int i = 0; i < MTL; ++i) store_tile(rec, i, r[i]);
                if (lane == 0) parts[warp][k] = {range.first + tile - cc.t, cc.nt, cc.b, h, last ? 1 : 0};
            }
            clear();
        }
        if (!last) {
            packed_next(cc, p, per_kv);
            if (pair_end) {
                load_q();
                packed_query<D, EXACT>(q_raw, p.scale_log2, lane, q);
                seg_t0 = 0;
                first_seg = false;
            }
        }
    }

    if (!ok) {
        if (lane == 0) atomicExch(p.status, kStatusTimeout);
        for (int s = 0; s < NS; ++s) {
            mbar_wait_bounded(bars + 8 * s, 0, 1u << 10);
            mbar_wait_bounded(bars + 8 * s, 1, 1u << 10);
        }
    }

    // ---- pairs that several warps share -------------------------------------------------------------
    // Lane 2 w + k looks at part k of warp w.  Parts of one pair follow one another; (pair, m-tile) items go to the block's warps.
    __syncthreads();
    PackedPart pt = {0, 0, 0, 0, 0};
    if (lane < 2 * WARPS) pt = parts[lane >> 1][lane & 1];
    const uint32_t there = __ballot_sync(FULL, pt.nt != 0);
    if (there == 0) return;
    const uint32_t in_ring = __ballot_sync(FULL, pt.in_ring != 0);
    const uint32_t below = there & ((1u << lane) - 1u);
    const uint32_t before = __shfl_sync(FULL, pt.begin, below ? 31 - __clz(below) : 0);
    const uint32_t heads = __ballot_sync(FULL, pt.nt != 0 && (below == 0 || before != pt.begin));    // first parts of their pairs
    const bool crosses = pt.begin < range.begin || pt.begin + pt.nt > range.end;
    const uint32_t crossing = __ballot_sync(FULL, crosses) & heads;
    const int n_items = __popc(heads) * MTL;
    // what crosses the block's borders becomes one of its two records: 0 for the pair that began before, 1 for one that goes on
    const auto block_record = [&](int block, int k) { return p.partials + (size_t)(2 * (block * WARPS + k) + 1) * REC; };
#pragma unroll 1
    for (int item = warp; item < n_items; item += WARPS) {
        const int i = item % MTL;
        uint32_t left = heads;
        for (int skip = item / MTL; skip > 0; --skip) left &= left - 1;
        const int head_lane = __ffs(left) - 1;
        left &= left - 1;
        uint32_t members = there & ~((1u << head_lane) - 1u) & (left ? (left & -left) - 1u : 0xffffffffu);
        float v[4];
        begin_join(v);
        while (members) {                        // four parts on their way at a time
            float2 m[4], l[4];
            float4 x[4];
            bool is[4];
#pragma unroll
            for (int a = 0; a < 4; ++a) {
                is[a] = members != 0;
                const int e = is[a] ? __ffs(members) - 1 : head_lane;
                members &= members - 1;          // (0 stays 0)
                const float* rec = in_ring >> e & 1 ? reinterpret_cast<const float*>(ring0 + (e >> 1) * (NS * TILE))
                                                    : p.partials + (size_t)(2 * (blockIdx.x * WARPS + (e >> 1))) * REC;
                m[a] = *reinterpret_cast<const float2*>(rec + MTL * 128 + q0);
                l[a] = *reinterpret_cast<const float2*>(rec + MTL * 128 + 8 + q0);
                x[a] = reinterpret_cast<const float4*>(rec)[i * 32 + lane];
            }
#pragma unroll
            for (int a = 0; a < 4; ++a)
                if (is[a]) join(v, m[a], l[a], x[a]);
        }
        const int b = __shfl_sync(FULL, pt.b, head_lane), h = __shfl_sync(FULL, pt.h, head_lane);
        if (crossing >> head_lane & 1) store_tile(block_record((int)blockIdx.x, __shfl_sync(FULL, pt.begin, head_lane) < range.begin ? 0 : 1), i, v);
        else write_tiles(std::integral_constant<int, 1>(), &v, i, b, h);
    }
    if (crossing == 0) return;

    // ---- pairs that several thread blocks share -----------------------------------------------------
    // Few blocks: the one that arrives last merges all.  Many (few pairs, long sequences): chunks of kMmaChunk blocks first, then
    // the chunks' records; a fixed order either way.  Warp k takes the ticket of the k-th of the (at most two) pairs, all warps merge.
    __shared__ struct { int32_t b, h, c_first, first, count, step, kind, merge, all; } join_of[2];
    const int n_cross = __popc(crossing);
    int32_t* at = nullptr;
    int n_parts = 0;
    bool waits = warp < n_cross;
    if (waits) {
        const int head_lane = __ffs(warp == 0 ? crossing : crossing & (crossing - 1)) - 1;
        const uint32_t begin = __shfl_sync(FULL, pt.begin, head_lane), nt = __shfl_sync(FULL, pt.nt, head_lane);
        const PackedShare share(range.all, (uint32_t)pp.n_blocks);
        const int c_first = (int)share.part(begin);
        n_parts = (int)share.part(begin + nt - 1) - c_first + 1;
        const bool two_level = n_parts > kMmaTreeMin;
        const int ck = two_level ? ((int)blockIdx.x - c_first) / kMmaChunk * kMmaChunk : 0;
        at = two_level ? p.counters2 + 2 * (c_first + ck) + (ck == 0 ? 1 : 0) : p.counters + c_first;
        if (lane == head_lane)
            join_of[warp] = {pt.b, pt.h, c_first, c_first + ck, two_level ? min(kMmaChunk, n_parts - ck) : n_parts, 1, 0, 0, two_level ? 0 : 1};
    }
    __syncthreads();                             // (the records' stores are in front of it)
    for (int round = 0; round < 2; ++round) {
        if (waits) {
            if (lane == 0) join_of[warp].merge = atom_add_acq_rel_gpu(at, 1) == join_of[warp].count - 1 ? 1 : 0;
            __syncwarp();
            waits = join_of[warp].merge != 0;    // else someone else arrives later and merges
        }
        if (!__syncthreads_or(waits)) return;
        for (int item = warp; item < n_cross * MTL; item += WARPS) {
            const int i = item % MTL;
            const auto jo = join_of[item / MTL];
            if (!jo.merge) continue;
            // a block's records 0 and 1 are above; 2 and 3 are of a chunk that begins with it; the odd ones are of a pair that began in it
            const auto record = [&](int block) { return block_record(block, jo.kind + (block == jo.c_first ? 1 : 0)); };
            float v[4];
            begin_join(v);
#pragma unroll 1
            for (int r0 = 0; r0 < jo.count; r0 += 8) {       // eight records on their way at a time
                float2 m[8], l[8];
                float4 x[8];
#pragma unroll
                for (int a = 0; a < 8; ++a) {
                    const float* rec = record(jo.first + min(r0 + a, jo.count - 1) * jo.step);
                    m[a] = __ldcg(reinterpret_cast<const float2*>(rec + MTL * 128 + q0));
                    l[a] = __ldcg(reinterpret_cast<const float2*>(rec + MTL * 128 + 8 + q0));
                    x[a] = __ldcg(reinterpret_cast<const float4*>(rec) + i * 32 + lane);
                }
#pragma unroll
                for (int a = 0; a < 8; ++a)
                    if (r0 + a < jo.count) join(v, m[a], l[a], x[a]);
            }
            if (jo.all) write_tiles(std::integral_constant<int, 1>(), &v, i, jo.b, jo.h);
            else store_tile(block_record(jo.first, 2 + (jo.first == jo.c_first ? 1 : 0)), i, v);
        }
        __syncthreads();
        if (waits) {
            if (lane == 0) *at = 0;              // ready for the next launch
            waits = join_of[warp].all == 0;
            __syncwarp();
            if (waits) {                         // from the chunk to the pair
                at = p.counters + join_of[warp].c_first;
                if (lane == 0) {
                    auto& jo = join_of[warp];
                    jo.first = jo.c_first;
                    jo.count = (n_parts + kMmaChunk - 1) / kMmaChunk;
                    jo.step = kMmaChunk;
                    jo.kind = 2;
                    jo.all = 1;
                }
                __syncwarp();
            }
        }
        if (!waits && warp < n_cross && lane == 0) join_of[warp].merge = 0;
    }
}

}  // namespace lckv
