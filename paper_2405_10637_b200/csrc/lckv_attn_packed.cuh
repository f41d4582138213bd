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
// EXACT (fp32 outputs).  Where thousands of rows cancel, two things would show: the rounding of W to 11 bits, and the
// tensor cores' truncation of sums of codes that are all positive.  So W is split into a rounded part and the rounding of
// the rest (a second MMA), and codes enter as c - 8, which is exact too (one more instruction for two codes), with
// low + 8 step in place of low.  A bf16 output's own rounding (2^-9) is 20 times what that would gain.
//
// Work decomposition, merge of split pairs and tickets are those of lckv_attn_mma.cuh.  A worker (warp) has a ring of
// whole tiles: 64 rows of keys, values and parameters arrive as one bulk copy (the last rows of a sequence as three).
#pragma once
#include "lckv_attn_mma.cuh"
#include "lckv_packed.cuh"

namespace lckv {

#ifndef LCKV_PACKED_WARPS
#define LCKV_PACKED_WARPS 12
#endif
#ifndef LCKV_PACKED_SLOTS
#define LCKV_PACKED_SLOTS 2
#endif
constexpr int kPackedWarps = LCKV_PACKED_WARPS;   // workers per CTA, one CTA per SM
constexpr int kPackedSlots = LCKV_PACKED_SLOTS;   // tiles in a worker's ring
template <int D>
__host__ __device__ constexpr int packed_smem_bytes() { return kPackedWarps * kPackedSlots * (packed_tile_bytes<D>() + 8) + 128; }

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

// A query head as the B operand of the score MMAs.
template <int D>
struct PackedQuery {
    uint32_t b[D / 16][2];
    float f[2];              // per column of this lane: softmax scale * log2(e) / the scaling of q and codes
    float sum[2][D / 64];    // sum of q over a group * softmax scale * log2(e)
};

// raw[j]: dimensions 32 j + 8 c4 .. + 7 of the query of column g4.
template <int D>
__device__ __forceinline__ void packed_query(const uint4 (&raw)[D / 32], float scale_log2, int lane, PackedQuery<D>& out)
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
    const float by = __uint_as_float((uint32_t)(up + 127) << 23), by16 = by * 0.0625f;
    const float f = scale_log2 * __uint_as_float((uint32_t)(24 - up + 127) << 23);
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
        // nibble i and nibble i + 4 of a word share a register; odd i count 16 times as much
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

// Token of row i (0 .. 7) of an MMA tile: pairs are swapped where bit 1 is set, so that the four tokens that a value load of a
// warp touches lie in both halves of the 32 banks.
__device__ __forceinline__ int packed_token(int i) { return i ^ ((i >> 1) & 1); }

struct PackedParams {
    MmaParams m;         // a.K, a.V, a.pre and a.start unused; a.H_q = pairs per sequence
    PackedSlot s;
    int64_t pitch;       // rows of a (sequence, kv head)
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

// The launch's tiles are cut into one range per worker; the first `more` ranges are one tile longer.  A warp works out the
// total and where its range begins by itself: the lanes add up the tiles of B / 32 sequences each, and the lane in whose
// part the range begins is looked into with all lanes again, until a lane has one sequence.
struct PackedShare {
    uint32_t each, more;          // tiles of a range; ranges with one more
    __device__ __forceinline__ uint32_t begin(uint32_t w) const { return w * each + min(w, more); }
    __device__ __forceinline__ uint32_t worker(uint32_t tile) const
    {
        const uint32_t longer = more * (each + 1);
        return tile < longer ? tile / (each + 1) : more + (tile - longer) / each;
    }
};
__device__ __forceinline__ uint32_t packed_lane_tiles(const AttnParams& p, int b0, int b1)
{
    uint32_t n = 0;
#pragma unroll 4
    for (int b = b0; b < b1; ++b) n += packed_tiles(packed_visible(p, b));
    return n;
}
__device__ __forceinline__ uint32_t warp_sum_before(uint32_t v, int lane, uint32_t& all)
{
    uint32_t incl = v;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const uint32_t x = __shfl_up_sync(0xffffffffu, incl, off);
        if (lane >= off) incl += x;
    }
    all = __shfl_sync(0xffffffffu, incl, 31);
    return incl - v;
}
// Fills share and, if worker w has tiles, their number and the cursor of the first.
__device__ __forceinline__ uint32_t packed_range(const AttnParams& p, uint32_t w, int per_kv, int lane, PackedShare& share, PackedCursor& c)
{
    const uint32_t FULL = 0xffffffffu, H = (uint32_t)p.H_q;
    int lo = 0, n = p.B, per = (n + 31) / 32;
    int32_t nv = 0;                                  // of the lane's sequence, where it has one
    const auto tiles_of_lane = [&]() {
        const int b0 = lo + min(n, lane * per), b1 = lo + min(n, (lane + 1) * per);
        if (per == 1) {
            nv = b0 < b1 ? packed_visible(p, b0) : 0;
            return packed_tiles(nv);
        }
        return packed_lane_tiles(p, b0, b1);
    };
    uint32_t mine = tiles_of_lane(), all;
    uint32_t before = warp_sum_before(mine, lane, all);
    share.each = all * H / (uint32_t)p.n_workers;
    share.more = all * H - share.each * (uint32_t)p.n_workers;
    const uint32_t first = share.begin(w), count = share.each + (w < share.more ? 1u : 0u);
    if (w >= (uint32_t)p.n_workers || count == 0) return 0;
    const uint32_t x = first / H;                    // tile of the sequences' concatenation in which the range begins
    uint32_t base = 0;
    for (;;) {
        const uint32_t there = __ballot_sync(FULL, base + before <= x && x < base + before + mine);
        const int l = __ffs(there) - 1;
        base += __shfl_sync(FULL, before, l);
        lo += l * per;
        if (per == 1) { c.nv = __shfl_sync(FULL, nv, l); break; }
        n = min(per, n - l * per);
        per = (n + 31) / 32;
        mine = tiles_of_lane();
        before = warp_sum_before(mine, lane, all);
    }
    c.b = lo;
    c.nt = packed_tiles(c.nv);
    const uint32_t rel = first - base * H, h = rel / c.nt;
    c.t = rel - h * c.nt;
    c.kvh = (int)h / per_kv;
    c.sub = (int)h - c.kvh * per_kv;
    return count;
}

// A ticket posted for one of the (at most two) pairs that a worker shares with others.
struct PackedPending { int32_t n, first_odd, b, h, c_first; };

template <int D, bool PAGED, int QP, bool EXACT>
__global__ void __launch_bounds__(kPackedWarps * 32, 1) attn_packed_kernel(const PackedParams pp)
{
    constexpr int R = kPackedRows;
    constexpr int RB = R / 16;                   // 16-row blocks of a tile
    constexpr int J = D / 32;                    // words of a key row per lane
    constexpr int G = D / 64;                    // groups
    constexpr int MT = D / 16;                   // 16-dimension m-tiles of the output MMA
    constexpr int NC = 8 / QP;                   // copies of the pair's heads in a tile's columns
    constexpr int NB = RB / NC;                  // blocks whose scores a lane works on
    constexpr int NS = kPackedSlots;
    constexpr int TILE = packed_tile_bytes<D>();
    constexpr int CODES = R * (D / 2);           // bytes of a tile's keys; its values follow, then the parameters
    constexpr int MTL = MT / NC;                 // m-tiles of a finished pair that a lane holds
    constexpr int REC = D * 8 + 16;
    const AttnParams& p = pp.m.a;
    const int HP = pp.m.heads_per_pair, per_kv = pp.m.groups_per_kv, n_q_heads = pp.m.n_q_heads;

    extern __shared__ uint8_t smem_raw[];
    __shared__ PackedPending pending[kPackedWarps][2];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int w = warp * gridDim.x + blockIdx.x;     // (ranges that are one longer spread over the SMs)
    const uint32_t FULL = 0xffffffffu;
    const int g4 = lane >> 2, c4 = lane & 3;
    const int copy = 2 * c4 / QP;                // the copy that this lane's columns belong to

    const uint32_t smem0 = (smem_u32(smem_raw) + 127u) & ~127u;
    const uint32_t ring = smem0 + warp * (NS * TILE);
    const uint32_t bars = smem0 + kPackedWarps * NS * TILE + warp * (NS * 8);
    if (lane == 0) {
        for (int s = 0; s < NS; ++s) mbar_init(bars + 8 * s, 1);
        fence_mbar_init();
    }
    __syncwarp();

    if (!p.early_kv) pdl_wait_then_release();

    PackedShare share;
    PackedCursor cc = {0, 0, 0, 0u, 0u, 0};
    const uint32_t n_tiles = packed_range(p, (uint32_t)w, per_kv, lane, share, cc);
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
    // The first pair's queries are asked for in front of the tiles, behind which they would wait in line (20 us with 12 workers'
    // tiles in front of them: 4800 cycles), unless only the tiles may be read yet.
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
    for (int b = w < p.n_workers ? w : p.B; b < p.B; b += p.n_workers) {
        if (packed_visible(p, b) == 0) {
            const int n16 = n_q_heads * D * (EXACT ? 4 : 2) / 16;
            uint4* o16 = reinterpret_cast<uint4*>(static_cast<uint8_t*>(p.out) + (size_t)b * n16 * 16);
            for (int i = lane; i < n16; i += 32) o16[i] = make_uint4(0, 0, 0, 0);
            if (p.lse)
                for (int i = lane; i < n_q_heads; i += 32) p.lse[(size_t)b * n_q_heads + i] = 0.f;
        }
    }

    if (n_tiles == 0) return;

    uint32_t cslot = 0, cphase = 0;
    bool ok = true;

    PackedQuery<D> q;
    packed_query<D>(q_raw, p.scale_log2, lane, q);

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

    // Which workers share a pair (of nt tiles from tile `begin` on): worked out when the worker enters a pair that its range
    // cuts, at most its first and its last.
    struct Split { int32_t c_first, n_parts, first_odd; };
    auto split_of = [&](uint32_t begin, uint32_t nt) {
        Split sp;
        sp.c_first = (int32_t)share.worker(begin);
        sp.n_parts = (int32_t)share.worker(begin + nt - 1) - sp.c_first + 1;
        sp.first_odd = begin != share.begin((uint32_t)sp.c_first) ? 1 : 0;   // which record of c_first belongs to this pair
        return sp;
    };
    Split cur = {0, 1, 0};
    const uint32_t first_tile = share.begin((uint32_t)w);
    if (cc.t != 0 || n_tiles < cc.nt) cur = split_of(first_tile - cc.t, cc.nt);
    bool first_seg = true;
    int32_t ticket0 = 0, ticket1 = 0;
    bool armed0 = false, armed1 = false;
    // A finished part of a pair: the lanes of a row's copies share its dimensions.  r[i] are the values of m-tile copy * MTL + i,
    // [0], [1] of dimension 64 g + 8 g4 + 2 k for the lane's two columns, [2], [3] of the one behind it, with 4 g + k the m-tile.
    float r[MTL][4], l_tot[2], m_fin[2];
    const int q0 = 2 * c4 % QP;                  // the lane's columns: query heads q0 and q0 + 1 of the pair
    const bool holds = q0 < HP, both = q0 + 1 < HP;

    // r / l_tot and lse -> the output rows of pair (b, h)
    auto write_rows = [&](int b, int h) {
        const size_t row0 = (size_t)b * n_q_heads + (size_t)h * HP + q0;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            if (j == 0 ? !holds : !both) break;
            const float inv = 1.0f / l_tot[j];
            constexpr int RUN = MTL < 4 ? MTL : 4;           // m-tiles whose dimensions are neighbours
#pragma unroll
            for (int i0 = 0; i0 < MTL; i0 += RUN) {
                const int mt = copy * MTL + i0;
                const size_t at = (row0 + j) * D + 64 * (mt / 4) + 8 * g4 + 2 * (mt % 4);
                float v[2 * RUN];
#pragma unroll
                for (int i = 0; i < RUN; ++i) { v[2 * i] = r[i0 + i][j] * inv; v[2 * i + 1] = r[i0 + i][2 + j] * inv; }
                if constexpr (EXACT) {
                    float* dst = static_cast<float*>(p.out) + at;
#pragma unroll
                    for (int i = 0; i < RUN; ++i) *reinterpret_cast<float2*>(dst + 2 * i) = make_float2(v[2 * i], v[2 * i + 1]);
                } else {
                    uint16_t* dst = static_cast<uint16_t*>(p.out) + at;
                    if constexpr (RUN == 4)
                        *reinterpret_cast<uint4*>(dst) = make_uint4(cvt_bf16x2(v[0], v[1]), cvt_bf16x2(v[2], v[3]), cvt_bf16x2(v[4], v[5]), cvt_bf16x2(v[6], v[7]));
                    else if constexpr (RUN == 2)
                        *reinterpret_cast<uint2*>(dst) = make_uint2(cvt_bf16x2(v[0], v[1]), cvt_bf16x2(v[2], v[3]));
                    else
                        *reinterpret_cast<uint32_t*>(dst) = cvt_bf16x2(v[0], v[1]);
                }
            }
            if (p.lse && g4 == 0 && copy == 0) p.lse[row0 + j] = (m_fin[j] + lg2(l_tot[j])) * 0.6931471805599453f;
        }
    };
    // (r, m_fin, l_tot) -> a partial record
    auto store_record = [&](float* rec) {
        if (!holds) return;
#pragma unroll
        for (int i = 0; i < MTL; ++i) reinterpret_cast<float4*>(rec)[i * 32 + lane] = make_float4(r[i][0], r[i][1], r[i][2], r[i][3]);
        if (g4 == 0 && copy == 0) {
            *reinterpret_cast<float2*>(rec + MTL * 128 + q0) = make_float2(m_fin[0], m_fin[1]);
            *reinterpret_cast<float2*>(rec + MTL * 128 + 8 + q0) = make_float2(l_tot[0], l_tot[1]);
        }
    };
    // Merge of n records in a fixed order, in one pass with running maxima: record i is the one of worker first_w + i * step
    // (its second record if i == 0 and first_slot is set).
    auto merge_records = [&](int n, uint32_t first_w, int step, int first_slot) {
        const float* rec0 = p.partials + (size_t)(2 * first_w) * REC;
        const size_t rstride = (size_t)(2 * step) * REC;
        m_fin[0] = m_fin[1] = -INFINITY;
        l_tot[0] = l_tot[1] = 0.f;
#pragma unroll
        for (int i = 0; i < MTL; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) r[i][e] = 0.f;
        if (!holds) return;
        constexpr int AHEAD = MTL <= 2 ? 8 : MTL == 4 ? 4 : 2;     // records in flight
        for (int i0 = 0; i0 < n; i0 += AHEAD) {
            float2 mm[AHEAD], ll[AHEAD];
            float4 x[AHEAD][MTL];
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) {
                const int i = min(i0 + a, n - 1);
                const float* rec = rec0 + (size_t)i * rstride + (i == 0 ? (size_t)first_slot * REC : 0);
                mm[a] = __ldcg(reinterpret_cast<const float2*>(rec + MTL * 128 + q0));
                ll[a] = __ldcg(reinterpret_cast<const float2*>(rec + MTL * 128 + 8 + q0));
#pragma unroll
                for (int k = 0; k < MTL; ++k) x[a][k] = __ldcg(reinterpret_cast<const float4*>(rec) + k * 32 + lane);
            }
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) {
                if (i0 + a >= n) break;
                const float M0 = fmaxf(m_fin[0], mm[a].x), M1 = fmaxf(m_fin[1], mm[a].y);
                const float a0 = ex2(m_fin[0] - M0), a1 = ex2(m_fin[1] - M1);      // ex2(-inf) = 0 for the first record
                const float w0 = ex2(mm[a].x - M0), w1 = ex2(mm[a].y - M1);
                m_fin[0] = M0; m_fin[1] = M1;
                l_tot[0] = fmaf(l_tot[0], a0, ll[a].x * w0);
                l_tot[1] = fmaf(l_tot[1], a1, ll[a].y * w1);
#pragma unroll
                for (int k = 0; k < MTL; ++k) {
                    r[k][0] = fmaf(r[k][0], a0, x[a][k].x * w0);
                    r[k][1] = fmaf(r[k][1], a1, x[a][k].y * w1);
                    r[k][2] = fmaf(r[k][2], a0, x[a][k].z * w0);
                    r[k][3] = fmaf(r[k][3], a1, x[a][k].w * w1);
                }
            }
        }
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
        if (!mbar_wait_bounded(bars + 8 * cslot, cphase, p.wait_limit)) { ok = false; break; }
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
                        nibble_pairs(ka[j], xa);
                        nibble_pairs(kb[j], xb);
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
                float t = bf16lo(pr[0]) * own[0][e], u = bf16hi(pr[0]) * q.sum[e & 1][0];
                if constexpr (G == 2) {
                    t = fmaf(bf16lo(pr[1]), own[1][e], t);
                    u = fmaf(bf16hi(pr[1]), q.sum[e & 1][1], u);
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
        if (__any_sync(FULL, alpha[0] != 1.f || alpha[1] != 1.f || e_new != e_run)) {
            const float de = e_new - e_run > 120 ? 0.f : __uint_as_float((uint32_t)(e_run - e_new + 127) << 23);
            // (columns of o are those of the transposed weights: this lane's two, whatever the copy)
            const float b0 = alpha[0] * de, b1 = alpha[1] * de;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                o[mt][0] *= b0; o[mt][1] *= b1;
                o[mt][2] *= b0; o[mt][3] *= b1;
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
                const float la = EXACT ? fmaf(8.f, bf16lo(pa), bf16hi(pa)) : bf16hi(pa), lb = EXACT ? fmaf(8.f, bf16lo(pb), bf16hi(pb)) : bf16hi(pb);
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
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    // nibbles 4 half .. 4 half + 3 of two tokens side by side
                    const uint32_t sel = half ? 0x7632u : 0x5410u;
                    uint32_t xa[4], xb[4];
                    const uint32_t lo = __byte_perm(va[0][g], va[1][g], sel), hi = __byte_perm(va[2][g], va[3][g], sel);
                    if constexpr (EXACT) {
                        nibble_pairs_signed(lo, xa);
                        nibble_pairs_signed(hi, xb);
                    } else {
                        nibble_pairs(lo, xa);
                        nibble_pairs(hi, xb);
                    }
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        float (&acc)[4] = o[4 * g + 2 * half + i];
                        mma_f16_16816(acc, xa[2 * i], xa[2 * i + 1], xb[2 * i], xb[2 * i + 1], b0, b1);
                        if constexpr (EXACT)
                            mma_f16_16816(acc, xa[2 * i], xa[2 * i + 1], xb[2 * i], xb[2 * i + 1], mine ? br[rb / NC][g][0] : 0u, mine ? br[rb / NC][g][1] : 0u);
                    }
                }
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

            const bool complete = pair_end && seg_t0 == 0;
            if (complete) {
                write_rows(cc.b, h);
            } else {
                const int c_first = cur.c_first;
                const int first_odd = cur.first_odd, n_parts = cur.n_parts;
                store_record(p.partials + (size_t)(2 * w + (first_seg ? 0 : 1)) * REC);
                // Few parts: the contributor that arrives last merges them all.  Many (few pairs, long sequences): chunks of
                // kMmaChunk consecutive workers first, then the chunks' records; a fixed order either way.  The ticket is
                // posted here and looked at after the last tile; each goes into a variable of its own that nothing reads
                // before.
                int32_t* ticket_at = p.counters + c_first;
                if (n_parts > kMmaTreeMin) {
                    const int ck = (w - c_first) / kMmaChunk * kMmaChunk;
                    ticket_at = p.counters2 + 2 * (c_first + ck) + (ck == 0 ? first_odd : 0);
                }
                if (lane == 0) pending[warp][first_seg ? 0 : 1] = {n_parts, first_odd, cc.b, h, c_first};
                __syncwarp();       // the record's stores (all lanes) are ordered before lane 0's release
                if (first_seg) {
                    if (lane == 0) ticket0 = atom_add_acq_rel_gpu(ticket_at, 1);
                    armed0 = true;
                } else {
                    if (lane == 0) ticket1 = atom_add_acq_rel_gpu(ticket_at, 1);
                    armed1 = true;
                }
            }
            clear();
        }
        if (!last) {
            packed_next(cc, p, per_kv);
            if (pair_end) {
                load_q();
                packed_query<D>(q_raw, p.scale_log2, lane, q);
                seg_t0 = 0;
                first_seg = false;
                if (n_tiles - (tile + 1) < cc.nt) cur = split_of(first_tile + tile + 1, cc.nt);   // the range ends inside this pair
            }
        }
    }

    if (ok) {
        __syncwarp();
#pragma unroll 1
        for (int i = 0; i < 2; ++i) {
            if (!(i == 0 ? armed0 : armed1)) continue;
            const PackedPending pd = pending[warp][i];
            int ticket = __shfl_sync(FULL, i == 0 ? ticket0 : ticket1, 0);
            // a chunk of many parts, or all parts of few
            const bool two_level = pd.n > kMmaTreeMin;
            const int ck = two_level ? (w - pd.c_first) / kMmaChunk * kMmaChunk : 0;
            int n = two_level ? min(kMmaChunk, pd.n - ck) : pd.n, first = pd.c_first + ck, step = 1, slot = ck == 0 ? pd.first_odd : 0;
            int32_t* at = two_level ? p.counters2 + 2 * first + slot : p.counters + first;
#pragma unroll 1
            for (bool whole = !two_level;;) {
                if (ticket != n - 1) break;              // someone else arrives later and merges
                __syncwarp();                            // lane 0's acquire is in front of all lanes' reads of the records
                merge_records(n, (uint32_t)first, step, slot);
                if (lane == 0) *at = 0;                  // ready for the next launch
                if (whole) { write_rows(pd.b, pd.h); break; }
                // the chunk's result becomes the record of the chunk's first worker
                store_record(p.partials + (size_t)(2 * first + slot) * REC);
                __syncwarp();
                at = p.counters + pd.c_first;
                if (lane == 0) ticket = atom_add_acq_rel_gpu(at, 1);
                ticket = __shfl_sync(FULL, ticket, 0);
                n = (pd.n + kMmaChunk - 1) / kMmaChunk; first = pd.c_first; step = kMmaChunk; slot = pd.first_odd;
                whole = true;
            }
        }
    } else {
        if (lane == 0) atomicExch(p.status, kStatusTimeout);
        for (int s = 0; s < NS; ++s) {
            mbar_wait_bounded(bars + 8 * s, 0, 1u << 10);
            mbar_wait_bounded(bars + 8 * s, 1, 1u << 10);
        }
    }
}

}  // namespace lckv
