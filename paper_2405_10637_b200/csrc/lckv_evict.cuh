// The attention weight that cached rows gather, and the eviction of the rows that gathered least.
#pragma once
#include "lckv_attn_packed.cuh"

namespace lckv {

constexpr int kWeightWarps = 4;

struct WeightParams {
    PackedSlot s;             // 4-bit rows, or
    const uint16_t* K;        // bf16 keys
    RowMap map;
    const int32_t* lens;
    const uint16_t* q;        // [batch, H_q, D]
    const float* lse;         // [batch, H_q]
    const float* prev;        // [batch, H_kv, stride] or null
    float* weights;
    int32_t* status;
    int64_t T_cap, stride;
    int32_t H_q, mode;
    int32_t run;              // consecutive tiles of 64 rows per warp
    int32_t runs, heads;      // such runs per (sequence, kv head), and those
    uint32_t wait_limit;
    float scale_log2;
};

//     weights[b, h, j] = prev[b, h, j] + sum over the query heads of kv head h of exp(s_j - lse)      for the visible rows j
//
// A warp takes `run` tiles of 64 rows of one (sequence, kv head); its lanes' place in a tile:
// QP columns of the MMA tile hold query heads (up to eight at a time), and their NC = 8 / QP copies share the exponentials as in
// lckv_attn_packed.cuh: copy k has every NC-th block of 16 rows.  Of the QP / 2 lanes that end up with a row's sum each
// writes another block's.
template <int QP>
struct WeightLane {
    static constexpr int NC = 8 / QP, NB = 4 / NC;
    int g4, c4, copy, q0, mine;
    float l0, l1;             // lse of the lane's two columns, base 2
    bool real0, real1;        // do they hold a query head?
    __device__ __forceinline__ explicit WeightLane(int lane) : g4(lane >> 2), c4(lane & 3), copy(2 * c4 / QP), q0(2 * c4 % QP), mine(q0 / 2) {}
    __device__ __forceinline__ void heads(const float* lse, int first, int group)
    {
        real0 = first + q0 < group;
        real1 = first + q0 + 1 < group;
        l0 = real0 ? lse[first + q0] * 1.4426950408889634f : 0.f;
        l1 = real1 ? lse[first + q0 + 1] * 1.4426950408889634f : 0.f;
    }
    __device__ __forceinline__ int row() const { return (mine * NC + copy) * 16 + g4; }     // the lane writes this row and the eighth behind it
    // scores of block i of the lane's copy -> the sums over all heads, kept by the lane that writes the block
    __device__ __forceinline__ void gather(const float (&s)[4], int i, float& ta, float& tb) const
    {
        float a = (real0 ? ex2(s[0] - l0) : 0.f) + (real1 ? ex2(s[1] - l1) : 0.f);
        float c = (real0 ? ex2(s[2] - l0) : 0.f) + (real1 ? ex2(s[3] - l1) : 0.f);
#pragma unroll
        for (int off = 1; off < QP / 2; off <<= 1) {
            a += __shfl_xor_sync(0xffffffffu, a, off);
            c += __shfl_xor_sync(0xffffffffu, c, off);
        }
        if (i == mine) { ta = a; tb = c; }
    }
};

// bf16 keys go straight from memory into MMA fragments, all of a tile under way before the first is used; a row's four lanes take
// 16 bytes each at a time, and q enters in the order which that gives.  Thread blocks per SM, which registers limit: four over 64 dimensions (128
// registers; the two narrow forms spill 4 and 28 bytes: 128 x 4 kv heads x 1024 rows 15.0 us, with three and no spill 16.9, with five 19.4); over
// 128 dimensions a tile is 128 registers by itself, and two blocks fit without being asked for (32 x 32 heads x 2048 rows 91.5 us; with three, which spill
// 108 bytes, 94.1 and small calls 4.3 -> 6.1, with four 133).
template <int D, int QP>
__global__ void __launch_bounds__(kWeightWarps * 32, D == 64 ? 4 : 1) attention_weights_kernel(const WeightParams p)
{
    constexpr int J = D / 32, NC = 8 / QP, NB = 4 / NC;
    pdl_wait_then_release();
    WeightLane<QP> l((int)threadIdx.x & 31);
    const int64_t unit = (int64_t)blockIdx.x * kWeightWarps + (threadIdx.x >> 5);
    if (unit >= (int64_t)p.heads * p.runs) return;
    const int bh = (int)(unit / p.runs), b = bh / p.map.H_kv, h = bh - b * p.map.H_kv;
    const int nv = visible_rows(p.lens[b], p.mode, p.T_cap);
    const int group = p.H_q / p.map.H_kv;
    const int64_t head0 = (int64_t)b * p.H_q + (int64_t)h * group, step = (int64_t)p.run * 64;
    for (int64_t r0 = (unit - (int64_t)bh * p.runs) * step; r0 < nv; r0 += p.runs * step) {
        const int end = (int)min((int64_t)nv, r0 + step);
        for (int first = 0; first < group; first += QP) {    // the sums of the heads before are read back
            uint4 q[J];
            const uint4* q4 = reinterpret_cast<const uint4*>(p.q + (head0 + min(first + l.g4 % QP, group - 1)) * D) + l.c4;
#pragma unroll
            for (int j = 0; j < J; ++j) q[j] = q4[4 * j];
            l.heads(p.lse + head0, first, group);
            const float* from = first ? p.weights : p.prev;
            for (int base = (int)r0; base < end; base += 64) {
                const int rows = min(64, end - base);
                const int64_t at = max((int64_t)0, p.map.at(b, h, base));
                uint4 ka[4][J], kb[4][J];
                // (rows behind the last one are not read: the last one's keys do in their place)
#pragma unroll
                for (int rb = 0; rb < 4; ++rb) {
                    if (rb * 16 >= rows) break;
                    const uint4* x = reinterpret_cast<const uint4*>(p.K + (at + min(rb * 16 + l.g4, rows - 1)) * D) + l.c4;
                    const uint4* y = reinterpret_cast<const uint4*>(p.K + (at + min(rb * 16 + l.g4 + 8, rows - 1)) * D) + l.c4;
#pragma unroll
                    for (int j = 0; j < J; ++j) { ka[rb][j] = x[4 * j]; kb[rb][j] = y[4 * j]; }
                }
                const int m = l.row();
                const int64_t o = (int64_t)bh * p.stride + base + m;
                float ta = 0.f, tb = 0.f;
                const float before_a = from && m < rows ? from[o] : 0.f, before_b = from && m + 8 < rows ? from[o + 8] : 0.f;
#pragma unroll
                for (int i = 0; i < NB; ++i) {
                    float s[4];
#pragma unroll
                    for (int k = 0; k < NC; ++k) {
                        const int rb = i * NC + k;
                        float acc[4] = {0.f, 0.f, 0.f, 0.f};
                        if (rb * 16 < rows) {
#pragma unroll
                            for (int j = 0; j < J; ++j) {
                                const uint4 x = ka[rb][j], y = kb[rb][j];
                                mma_bf16_16816(acc, x.x, y.x, x.y, y.y, q[j].x, q[j].y);
                                mma_bf16_16816(acc, x.z, y.z, x.w, y.w, q[j].z, q[j].w);
                            }
                        }
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[e] = k == 0 || l.copy == k ? acc[e] * p.scale_log2 : s[e];
                    }
                    l.gather(s, i, ta, tb);
                }
                if (m < rows) p.weights[o] = before_a + ta;
                if (m + 8 < rows) p.weights[o + 8] = before_b + tb;
            }
        }
    }
}

// 4-bit keys: the decode attention's division of the work (one thread block per SM, one range of tiles per warp, whatever the
// lengths; a (sequence, kv head) is a pair) and its rings, here of two tiles' keys and parameters, two bulk copies a tile.  Nothing is to
// be joined.  Codes enter as c - 8 (EXACT there; weights are fp32, and came out 9e-7 off without).  32 x 32 heads of 128 with 256 to
// 4096 rows (190 MB): 49 us, 3.9 TB/s, instructions; with codes as they are 37, 5.1 TB/s (then with 12 warps and three tiles a ring 41, with a
// fixed number of tiles per warp 48 to 60, with tiles in registers and the next one's loads under way 60 to 68).
constexpr int kWeightSlots = 2, kWeightBlockWarps = 16;
template <int D>
__host__ __device__ constexpr int weight_tile_bytes() { return kPackedRows * (D / 2 + D / 8); }
template <int D>
__host__ __device__ constexpr int weight_smem_bytes() { return kWeightBlockWarps * kWeightSlots * (weight_tile_bytes<D>() + 8) + 128; }

template <int D, int QP>
__global__ void __launch_bounds__(kWeightBlockWarps * 32, 1) attention_weights_packed_kernel(const WeightParams p, const PackedParams pp)
{
    constexpr int J = D / 32, G = D / 64, NC = 8 / QP, NB = 4 / NC, NS = kWeightSlots, TILE = weight_tile_bytes<D>(), WARPS = kWeightBlockWarps;
    constexpr int CODES = kPackedRows * (D / 2);
    extern __shared__ uint8_t smem_raw[];
    __shared__ PackedTable table;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t smem0 = (smem_u32(smem_raw) + 127u) & ~127u, ring = smem0 + warp * (NS * TILE), bars = smem0 + WARPS * NS * TILE + warp * (NS * 8);
    if (lane == 0) {
        for (int s = 0; s < NS; ++s) mbar_init(bars + 8 * s, 1);
        fence_mbar_init();
    }
    __syncwarp();
    pdl_wait_then_release();
    PackedCursor cc = {0, 0, 0, 0u, 0u, 0};
    const int per = (pp.m.a.B + kPackedTable - 1) / kPackedTable;
    const uint32_t longest = packed_table<WARPS * 32>(pp.m.a, per, table);
    const uint32_t n_tiles = packed_range(pp, table, per, longest, blockIdx.x, (uint32_t)warp, lane, cc).count;
    if (n_tiles == 0) return;
    WeightLane<QP> l(lane);
    const int group = p.H_q / p.map.H_kv, m = l.row();
    const uint64_t l2pol = make_l2_policy(0.f);
    // the sums so far of this lane's two rows in the tiles that are under way, in turn
    PackedCursor ci = cc;
    float before_a[NS], before_b[NS];
    uint32_t issued = 0;
    const auto row_of = [&](const PackedCursor& c) { return ((int64_t)c.b * p.map.H_kv + c.kvh) * p.stride + (int64_t)c.t * 64 + m; };
    const auto issue = [&](float& a, float& b) {
        const int rows = min(64, ci.nv - (int)ci.t * 64);
        if (lane == 0) {
            const uint32_t slot = issued % NS, bar = bars + 8 * slot, dst = ring + slot * TILE, even = ((uint32_t)rows + 1u) & ~1u;
            const uint8_t* src = p.s.tile<D>(max((int64_t)0, p.map.at(ci.b, ci.kvh, (int)ci.t * 64)));
            mbar_expect_tx(bar, even * (D / 2 + 8 * G));
            bulk_g2s_hint(dst, src, even * (D / 2), bar, l2pol);
            bulk_g2s_hint(dst + CODES, src + 2 * CODES, even * (8 * G), bar, l2pol);
        }
        const float* from = p.prev ? p.prev + row_of(ci) : nullptr;
        a = from && m < rows ? from[0] : 0.f;
        b = from && m + 8 < rows ? from[8] : 0.f;
        packed_next(ci, pp.m.a, 1);
        ++issued;
    };
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        before_a[s] = before_b[s] = 0.f;
        if (issued < n_tiles) issue(before_a[s], before_b[s]);
    }
    PackedQuery<D, true> q;
    const auto load_q = [&](int first) {         // query heads first .. of pair cc
        const int64_t head0 = (int64_t)cc.b * p.H_q + (int64_t)cc.kvh * group;
        uint4 raw[J];
        const uint4* q4 = reinterpret_cast<const uint4*>(p.q + (head0 + min(first + l.g4 % QP, group - 1)) * D) + l.c4;
#pragma unroll
        for (int j = 0; j < J; ++j) raw[j] = q4[4 * j];
        l.heads(p.lse + head0, first, group);
        packed_query<D, true>(raw, p.scale_log2, lane, q);
    };
    load_q(0);
    for (uint32_t tile = 0; tile < n_tiles; ++tile) {
        const int rows = min(64, cc.nv - (int)cc.t * 64);
        const uint32_t slot = tile % NS, kc = ring + slot * TILE, par = kc + CODES;
        if (!__all_sync(0xffffffffu, mbar_wait_bounded(bars + 8 * slot, tile / NS & 1, p.wait_limit))) {      // (all lanes or none)
            if (lane == 0) atomicExch(p.status, kStatusTimeout);
            for (int s = 0; s < NS; ++s) {
                mbar_wait_bounded(bars + 8 * s, 0, 1u << 10);
                mbar_wait_bounded(bars + 8 * s, 1, 1u << 10);
            }
            return;
        }
        float sum_a = 0.f, sum_b = 0.f;
        for (int first = 0; first < group; first += QP) {    // (more than eight query heads: prepared again for every tile)
            if (group > QP) load_q(first);
            float ta = 0.f, tb = 0.f;
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                float own[G][4];
#pragma unroll
                for (int k = 0; k < NC; ++k) {
                    const int rb = i * NC + k, ra = rb * 16 + l.g4;
                    float acc[G][4];
#pragma unroll
                    for (int g = 0; g < G; ++g)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[g][e] = 0.f;
                    if (rb * 16 < rows) {
                        uint32_t ka[J], kb[J];
                        if constexpr (D == 128) {
                            const uint4 x = lds128(kc + ra * 64 + l.c4 * 16), y = lds128(kc + (ra + 8) * 64 + l.c4 * 16);
                            ka[0] = x.x; ka[1] = x.y; ka[2] = x.z; ka[3] = x.w;
                            kb[0] = y.x; kb[1] = y.y; kb[2] = y.z; kb[3] = y.w;
                        } else {
                            const uint2 x = lds64(kc + ra * 32 + l.c4 * 8), y = lds64(kc + (ra + 8) * 32 + l.c4 * 8);
                            ka[0] = x.x; ka[1] = x.y;
                            kb[0] = y.x; kb[1] = y.y;
                        }
#pragma unroll
                        for (int j = 0; j < J; ++j) {
                            uint32_t xa[4], xb[4];
                            nibble_pairs_signed(ka[j], xa);
                            nibble_pairs_signed(kb[j], xb);
                            mma_f16_16816(acc[j / 2], xa[0], xb[0], xa[1], xb[1], q.b[2 * j][0], q.b[2 * j][1]);
                            mma_f16_16816(acc[j / 2], xa[2], xb[2], xa[3], xb[3], q.b[2 * j + 1][0], q.b[2 * j + 1][1]);
                        }
                    }
#pragma unroll
                    for (int g = 0; g < G; ++g)
#pragma unroll
                        for (int e = 0; e < 4; ++e) own[g][e] = k == 0 || l.copy == k ? acc[g][e] : own[g][e];
                }
                // (rows behind the last one: what the slot held before, for weights that nobody writes)
                const int mr = (i * NC + l.copy) * 16 + l.g4;
                uint32_t pa[G], pb[G];
                if constexpr (G == 2) {
                    const uint2 x = lds64(par + mr * 16), y = lds64(par + (mr + 8) * 16);
                    pa[0] = x.x; pa[1] = x.y;
                    pb[0] = y.x; pb[1] = y.y;
                } else {
                    pa[0] = lds32(par + mr * 8);
                    pb[0] = lds32(par + (mr + 8) * 8);
                }
                float s[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t* pr = e < 2 ? pa : pb;
                    float x = bf16lo(pr[0]) * own[0][e], u = packed_low<true>(pr[0]) * q.sum[e & 1][0];
                    if constexpr (G == 2) {
                        x = fmaf(bf16lo(pr[1]), own[1][e], x);
                        u = fmaf(packed_low<true>(pr[1]), q.sum[e & 1][1], u);
                    }
                    s[e] = fmaf(x, q.f[e & 1], u);
                }
                l.gather(s, i, ta, tb);
            }
            sum_a += ta;
            sum_b += tb;
        }
        __syncwarp();
        float then_a = 0.f, then_b = 0.f;
        if (issued < n_tiles) issue(then_a, then_b);
        float* to = p.weights + row_of(cc);
        if (m < rows) to[0] = before_a[0] + sum_a;
        if (m + 8 < rows) to[8] = before_b[0] + sum_b;
#pragma unroll
        for (int s = 0; s + 1 < NS; ++s) { before_a[s] = before_a[s + 1]; before_b[s] = before_b[s + 1]; }
        before_a[NS - 1] = then_a;
        before_b[NS - 1] = then_b;
        const bool pair_end = cc.t + 1 == cc.nt;
        packed_next(cc, pp.m.a, 1);
        if (pair_end && tile + 1 < n_tiles) load_q(0);
    }
}

// ---- eviction -----------------------------------------------------------------------------------------------------------

// Order of weights as whole numbers: larger weight, larger key; -0 as 0; a NaN below all.  And the weight of a key.
__device__ __forceinline__ uint32_t weight_key(float w)
{
    const uint32_t u = __float_as_uint(w + 0.f);
    if ((u & 0x7fffffffu) > 0x7f800000u) return 0u;
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_weight(uint32_t k)
{
    return __uint_as_float(k == 0u ? 0x7fffffffu : (k & 0x80000000u) ? k & 0x7fffffffu : ~k);
}

struct SelectParams {
    const float* weights;     // [batch, H_kv, stride] or null (all equal)
    float* weights_out;       // [batch, H_kv, out_stride] or null; may be `weights`
    int32_t* kept;            // [batch, H_kv, n_keep]
    const int32_t* lens;
    int32_t* lens_out;        // lengths to set (another cache's), or null
    int64_t stride, out_stride, T_cap;
    int32_t H_kv, n_sink, n_recent, n_keep, out_rows;
};

// One thread block per (sequence, kv head); a warp holds the keys of 32 KPT consecutive rows, KPT a thread, in registers
// (KPT = 0, for more rows than the block can hold: keys from memory each time.  KPT = 32 does not fit the 64 registers that 1024 threads leave;
// ptxas spills 540 bytes a thread, and it is still 1.5 to 2.6 times as fast as reading the weights in every round).  The smallest key
// that stays is found two bits at a time: with t the
// bits found so far, count the keys >= t + 1, 2 and 3 units of those bits.  That is at most 16 rounds, fewer when a count
// meets the target (as with distinct weights it soon does).  Then every warp lists its own stretch of rows behind what
// the warps in front of it keep, so rows stay in order and equal weights go by the lowest row.
//
// What bounds it is the chain of rounds, each a block-wide sum, not the 4 bytes per row: thread blocks are as small as the rows
// allow, so that several on an SM cover for each other.
template <int WARPS>
struct SelectShared { int counts[2][3][WARPS], stay[WARPS], middle[WARPS], equal[WARPS]; };

template <int THREADS, int KPT>
__device__ __forceinline__ void evict_select(const SelectParams& p, SelectShared<THREADS / 32>& sh, int n)
{
    constexpr int WARPS = THREADS / 32;
    const uint32_t FULL = 0xffffffffu;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int b = blockIdx.x / p.H_kv;
    const float* w = p.weights ? p.weights + (int64_t)blockIdx.x * p.stride : nullptr;
    float* out = p.weights_out ? p.weights_out + (int64_t)blockIdx.x * p.out_stride : nullptr;
    int32_t* kept = p.kept + (int64_t)blockIdx.x * p.n_keep;
    const int count = min(n, p.n_keep);
    if (p.lens_out && blockIdx.x % p.H_kv == 0 && tid == 0) p.lens_out[b] = count;
    // rows lo .. hi - 1 are this warp's; row lo + 32 i + lane is the thread's i-th
    const int each = KPT ? 32 * KPT : ((n + WARPS - 1) / WARPS + 31) / 32 * 32;
    const int lo = min(n, warp * each), hi = min(n, lo + each);
    const int turns = KPT ? KPT : each / 32;
    uint32_t held[KPT ? KPT : 1] = {};
    const auto weight = [&](int row) { return w ? w[row] : 0.f; };
    const auto key = [&](int i) {
        if constexpr (KPT != 0) return held[i];
        const int row = lo + 32 * i + lane;
        return row < hi ? weight_key(weight(row)) : 0u;
    };
    const int first = n > p.n_keep ? p.n_sink : 0, behind = n > p.n_keep ? n - p.n_recent : 0;   // rows that compete
    if constexpr (KPT != 0) {                // (0 for the others, until the search is over: counted by no round)
#pragma unroll
        for (int i = 0; i < KPT; ++i) {
            const int row = lo + 32 * i + lane;
            held[i] = row >= first && row < min(hi, behind) ? weight_key(weight(row)) : 0u;
        }
    }
    const auto competes = [&](int i) { const int row = lo + 32 * i + lane; return row >= first && row < behind; };
    uint32_t t = 0;
    int target = 0;
    bool met = true;
    if (n > p.n_keep) {
        target = p.n_keep - p.n_sink - p.n_recent;                   // how many of them stay (fewer than compete)
        met = target == 0;
        if (met) t = 0xffffffffu;                                    // (no weight has this key: nothing stays)
        int turn = 0;
        for (int shift = 30; shift >= 0 && !met; shift -= 2) {
            int c[3] = {0, 0, 0};
#pragma unroll
            for (int i = 0; i < (KPT ? KPT : turns); ++i) {
                const uint32_t k = KPT != 0 || competes(i) ? key(i) : 0u;
#pragma unroll
                for (int x = 0; x < 3; ++x) c[x] += k >= t + ((uint32_t)(x + 1) << shift);
            }
#pragma unroll
            for (int x = 0; x < 3; ++x) {
                c[x] = __reduce_add_sync(FULL, c[x]);
                if (lane == 0) sh.counts[turn][x][warp] = c[x];
            }
            __syncthreads();
#pragma unroll
            for (int x = 0; x < 3; ++x) c[x] = __reduce_add_sync(FULL, lane < WARPS ? sh.counts[turn][x][lane] : 0);
            turn ^= 1;
            const int digit = c[2] >= target ? 3 : c[1] >= target ? 2 : c[0] >= target ? 1 : 0;
            t += (uint32_t)digit << shift;
            met = digit > 0 && c[digit > 0 ? digit - 1 : 0] == target;
        }
    }
    if constexpr (KPT != 0) {
#pragma unroll
        for (int i = 0; i < KPT; ++i) {
            const int row = lo + 32 * i + lane;
            if (row < hi && !competes(i)) held[i] = weight_key(weight(row));
        }
    }
    // met: all keys >= t stay; else all keys > t, and of those equal to t the first `ties`.  Rows that do not compete: the first
    // and the last (all, where n <= n_keep).
    const auto kind = [&](int i) {               // 1 stays, 2 equal to t, 0 neither
        const int row = lo + 32 * i + lane;
        if (row >= hi) return 0;
        if (!competes(i)) return 1;
        const uint32_t k = key(i);
        return (met ? k >= t : k > t) ? 1 : !met && k == t ? 2 : 0;
    };
    int n_stay = 0, n_equal = 0, n_middle = 0;
    uint32_t stay_bits = 0, equal_bits = 0;      // bit i: the thread's i-th row (KPT <= 32)
#pragma unroll
    for (int i = 0; i < (KPT ? KPT : turns); ++i) {
        const int c = kind(i);
        n_stay += c == 1;
        n_equal += c == 2;
        n_middle += c == 1 && competes(i);
        if (KPT != 0) {
            stay_bits |= (uint32_t)(c == 1) << i;
            equal_bits |= (uint32_t)(c == 2) << i;
        }
    }
    n_stay = __reduce_add_sync(FULL, n_stay);
    n_equal = __reduce_add_sync(FULL, n_equal);
    n_middle = __reduce_add_sync(FULL, n_middle);
    if (lane == 0) { sh.stay[warp] = n_stay; sh.equal[warp] = n_equal; sh.middle[warp] = n_middle; }
    __syncthreads();                                                 // (behind it the weights in memory are read no more, if KPT)
    const int all_above = __reduce_add_sync(FULL, lane < WARPS ? sh.middle[lane] : 0);
    n_stay = __reduce_add_sync(FULL, lane < warp ? sh.stay[lane] : 0);
    n_equal = __reduce_add_sync(FULL, lane < warp ? sh.equal[lane] : 0);
    const int ties = max(0, target - all_above);
    const uint32_t below = (1u << lane) - 1u;
#pragma unroll
    for (int i = 0; i < (KPT ? KPT : turns); ++i) {
        const int c = KPT != 0 ? 0 : kind(i);
        const bool a = KPT != 0 ? stay_bits >> i & 1 : c == 1, e = KPT != 0 ? equal_bits >> i & 1 : c == 2;
        const uint32_t ab = __ballot_sync(FULL, a), eb = __ballot_sync(FULL, e);
        const int e_rank = n_equal + __popc(eb & below);
        if (a || (e && e_rank < ties)) {
            const int at = n_stay + __popc(ab & below) + min(e_rank, ties);
            kept[at] = lo + 32 * i + lane;
            if (KPT != 0 && out) out[at] = key_weight(key(i));
        }
        n_stay += __popc(ab);
        n_equal += __popc(eb);
    }
    for (int i = count + tid; i < p.n_keep; i += THREADS) kept[i] = -1;
    if (!out) return;
    if constexpr (KPT != 0) {
        for (int i = count + tid; i < p.out_rows; i += THREADS) out[i] = 0.f;
    } else {
        // Rows only move down, so with weights in place a tile is read before it is written, and tiles go upwards.
        __syncthreads();
        for (int i0 = 0; i0 < p.out_rows; i0 += THREADS) {
            const int i = i0 + tid;
            const float x = i < count ? weight(kept[i]) : 0.f;
            __syncthreads();
            if (i < p.out_rows) out[i] = x;
        }
    }
}

template <int THREADS, int KPT>
__global__ void __launch_bounds__(THREADS) evict_select_kernel(const SelectParams p)
{
    __shared__ SelectShared<THREADS / 32> sh;
    pdl_wait_then_release();
    const int n = (int)min((int64_t)max(p.lens[blockIdx.x / p.H_kv], 0), p.T_cap);
    // (the launcher goes by the lengths that the host knows, which a replayed advance leaves behind)
    if (KPT != 0 && n <= THREADS * KPT) evict_select<THREADS, KPT>(p, sh, n);
    else evict_select<THREADS, 0>(p, sh, n);
}

struct MoveParams {
    PackedSlot from, to;      // 4-bit slots
    const uint16_t *K, *V;    // bf16 slots
    uint16_t *K_to, *V_to;
    RowMap map, map_to;
    const int32_t* kept;
    const int32_t* lens;
    int32_t* lens_out;        // set by the block of head 0 (in place), or null
    int32_t* status;          // of the cache written to
    int64_t T_cap;
    int32_t n_keep;
};

constexpr int kStatusNoRow = 2;   // a row had no place (LCKV_ECAPACITY)

// Physical rows of row i of the result of (sequence, kv head) number bh: from and to; negative where there is nothing to do.
struct MoveRow { int64_t from, to; };
__device__ __forceinline__ MoveRow move_row(const MoveParams& p, int bh, int i)
{
    MoveRow r = {-1, -1};
    const int row = i < p.n_keep ? p.kept[(int64_t)bh * p.n_keep + i] : -1;
    if (row < 0) return r;
    const int b = bh / p.map.H_kv, h = bh - b * p.map.H_kv;
    r.from = p.map.at(b, h, row);
    r.to = p.map_to.at(b, h, i);
    if (r.from < 0 || r.to < 0) {
        atomicExch(p.status, kStatusNoRow);
        r.from = -1;
    }
    return r;
}

// A row as units of one size: 9 of 16 bytes (D = 128) or of 8 (D = 64) in 4 bits - four units of keys, four of values, one
// of parameters -, D / 4 of 16 bytes in bf16.
template <int D, bool PACKED>
struct RowUnits {
    static constexpr int kUnits = PACKED ? 9 : D / 4;
    using Unit = typename std::conditional<PACKED && D == 64, uint2, uint4>::type;
    // units from one row to the next, within a tile
    static __device__ __forceinline__ int step(int u) { return PACKED ? (u < 8 ? 4 : 1) : D / 8; }
    static __device__ __forceinline__ const Unit* at(const PackedSlot& s, const uint16_t* K, const uint16_t* V, int64_t row, int u)
    {
        if constexpr (PACKED) {
            if (u < 8) return reinterpret_cast<const Unit*>(s.keys<D>(row) + (u < 4 ? 0 : kPackedRows * (D / 2))) + (u & 3);
            return reinterpret_cast<const Unit*>(s.par<D>(row));
        } else {
            return reinterpret_cast<const Unit*>((u < D / 8 ? K : V) + row * D) + (u < D / 8 ? u : u - D / 8);
        }
    }
};

// From one slot to another of the same kind: blockIdx.x is the (sequence, kv head), blockIdx.y a stretch of its rows; a thread
// has one unit of four neighbouring rows of the result.
constexpr int kMoveRows = 4;
template <int D, bool PACKED>
__global__ void __launch_bounds__(kRowThreads) evict_move_kernel(const MoveParams p)
{
    using U = RowUnits<D, PACKED>;
    pdl_wait_then_release();
    const int b = (int)blockIdx.x / p.map.H_kv, h = (int)blockIdx.x - b * p.map.H_kv;
    const int32_t* kept = p.kept + (int64_t)blockIdx.x * p.n_keep;
    for (int64_t k = (int64_t)blockIdx.y * kRowThreads + threadIdx.x; k < (int64_t)((p.n_keep + kMoveRows - 1) / kMoveRows) * U::kUnits;
         k += (int64_t)gridDim.y * kRowThreads) {
        const uint32_t group = (uint32_t)k / U::kUnits;
        const int u = (int)((uint32_t)k - group * U::kUnits), i = (int)group * kMoveRows;
        int from[kMoveRows];
#pragma unroll
        for (int x = 0; x < kMoveRows; ++x) from[x] = i + x < p.n_keep ? kept[i + x] : -1;
        if (from[0] < 0) continue;
        const int64_t to = p.map_to.at(b, h, i);
        bool lost = to < 0;
        typename U::Unit v[kMoveRows];
#pragma unroll
        for (int x = 0; x < kMoveRows; ++x) {
            if (from[x] < 0 || to < 0) continue;
            const int64_t row = p.map.at(b, h, from[x]);
            if (row < 0) { lost = true; from[x] = -1; continue; }
            v[x] = *U::at(p.from, p.K, p.V, row, u);
        }
        if (to >= 0) {
            auto* dst = const_cast<typename U::Unit*>(U::at(p.to, p.K_to, p.V_to, to, u));
#pragma unroll
            for (int x = 0; x < kMoveRows; ++x)
                if (from[x] >= 0) dst[x * U::step(u)] = v[x];
        }
        if (lost) atomicExch(p.status, kStatusNoRow);
    }
}

// From bf16 rows to 4-bit rows; lanes as in packed_write_kernel, blocks as above, four neighbouring rows a thread.
constexpr int kPackRows = 4;
template <int D>
__global__ void __launch_bounds__(kRowThreads) evict_pack_kernel(const MoveParams p)
{
    pdl_wait_then_release();
    const PackedLane<D> lane((int)threadIdx.x % PackedLane<D>::kLanes);
    constexpr int STEP = rows_per_block<D>() * kPackRows;
    const int b = (int)blockIdx.x / p.map.H_kv, h = (int)blockIdx.x - b * p.map.H_kv;
    const int32_t* kept = p.kept + (int64_t)blockIdx.x * p.n_keep;
    for (int64_t i0 = (int64_t)blockIdx.y * STEP; i0 < p.n_keep; i0 += (int64_t)gridDim.y * STEP) {
        const int i = (int)i0 + (int)threadIdx.x / PackedLane<D>::kLanes * kPackRows;
        int from[kPackRows];
        uint4 x[kPackRows], y[kPackRows];
#pragma unroll
        for (int u = 0; u < kPackRows; ++u) from[u] = i + u < p.n_keep ? kept[i + u] : -1;
        const int64_t to = from[0] >= 0 ? p.map_to.at(b, h, i) : -1;
        bool lost = from[0] >= 0 && to < 0;
#pragma unroll
        for (int u = 0; u < kPackRows; ++u) {
            x[u] = y[u] = make_uint4(0, 0, 0, 0);
            if (from[u] < 0 || to < 0) continue;
            const int64_t row = p.map.at(b, h, from[u]);
            if (row < 0) { lost = true; from[u] = -1; continue; }
            const uint16_t* src = (lane.is_v ? p.V : p.K) + row * D;
            x[u] = *reinterpret_cast<const uint4*>(src + lane.element(0));
            y[u] = *reinterpret_cast<const uint4*>(src + lane.element(1));
        }
        const auto place = lane.at(p.to, max((int64_t)0, to));
#pragma unroll
        for (int u = 0; u < kPackRows; ++u) {
            uint32_t w0, w1, par;
            packed_encode(x[u], y[u], w0, w1, par);
            if (from[u] >= 0 && to >= 0) lane.store(place, u, w0, w1, par);
        }
        if (lost) atomicExch(p.status, kStatusNoRow);
    }
}

// Within one slot: a thread block per (sequence, head) moves tiles upwards; a tile is read whole before it is written, and
// what later tiles read lies behind it (row i of the result was row kept[i] >= i).
template <int D, bool PACKED>
__global__ void __launch_bounds__(1024) evict_in_place_kernel(const MoveParams p)
{
    using U = RowUnits<D, PACKED>;
    constexpr int X = 4;                                   // units per thread and tile
    constexpr int ROWS = X * 1024 / U::kUnits;
    pdl_wait_then_release();
    for (int i0 = 0; i0 < p.n_keep; i0 += ROWS) {
        typename U::Unit v[X];
        int64_t to[X];
#pragma unroll
        for (int x = 0; x < X; ++x) {
            const int k = x * 1024 + threadIdx.x, i = i0 + k / U::kUnits;
            to[x] = -1;
            if (k < ROWS * U::kUnits && i < p.n_keep) {
                const MoveRow r = move_row(p, (int)blockIdx.x, i);
                if (r.from >= 0 && r.from != r.to) {
                    to[x] = r.to;
                    v[x] = *U::at(p.from, p.K, p.V, r.from, k % U::kUnits);
                }
            }
        }
        __syncthreads();
#pragma unroll
        for (int x = 0; x < X; ++x)
            if (to[x] >= 0) *const_cast<typename U::Unit*>(U::at(p.to, p.K_to, p.V_to, to[x], (x * 1024 + (int)threadIdx.x) % U::kUnits)) = v[x];
        __syncthreads();
    }
    if (p.lens_out && blockIdx.x % p.map.H_kv == 0 && threadIdx.x == 0) {
        const int b = blockIdx.x / p.map.H_kv;
        p.lens_out[b] = (int)min(min((int64_t)max(p.lens[b], 0), p.T_cap), (int64_t)p.n_keep);
    }
}

}  // namespace lckv
