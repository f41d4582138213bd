// Products with 4-bit weights: y[m, n] = sum_k x[m, k] * s[n, k/g] * (c[n, k] - z[n, k/g]), for the few rows m
// of a decode step.  c in 0 .. 15, one scale s (bf16) and one zero point z (0 .. 15, or 8 everywhere) per group
// of g = 32, 64 or 128 consecutive k.
//
// Bound by the bytes of the codes: 2 m multiply-adds per half byte, and close behind by the integer instructions that
// turn nibbles into numbers.  The operands are swapped so that 16 output features are the rows of an MMA tile and up to
// 8 rows of x its columns.  A nibble or'ed into the upper mantissa bits of 16.0 is 16 + c (7 or 8 instructions per 8 codes), and
// 16 + z subtracted from it leaves c - z (4 more): in bf16 for x in bf16, in fp16 for x in e4m3, which is converted when it is
// loaded.  All of these are exact, sums are fp32, scales are applied in fp32 once per group.  (Taking x (16 + c) and correcting
// by (16 + z) times a sum of x once per group cancels sums of up to 31 |x|, and needs an MMA with a tile of ones: 4096 x 22016,
// 1 row 12.7 us, 16 rows of e4m3 in groups of 64 20.6, of 32 22.0; this 12.4, 20.2 and 19.7.)
//
// Layout (quant_pack_kernel, once per weight).  The codes are cut into blocks of 32 features x 128 k = 2 KB,
// k fastest; such a block holds [2 halves of 64 k][2 tiles of 16 features][32 lanes][16 bytes], where lane (g, t) of a
// tile (g = lane / 4, t = lane % 4) owns features g and g + 8: its four words are feature g and g + 8 of the half's
// first 32 k, then of the second.  A word holds 8 codes of one feature: k = 4 t .. 4 t + 3 of the two k16 steps of
// its 32 k - what the lane owns of an A fragment, in shared memory, registers or tensor memory alike.  The nibbles are
// placed so that the word, rotated right by 4 i and masked with 0x00780078, has a pair of neighbouring k in the upper
// mantissa bits of two bf16 (i = 0, 2: first step, i = 1, 3: second step); rotated by 3 and 7 and masked with
// 0x0f0f0f0f it has the e4m3 codes of the first and the second step, k in the order 0, 2, 1, 3.
// Behind a block's codes stand its scales, [128 / group][32] bf16, and its zero points, [128 / group][32] bytes, in the
// order g * 4 + tile * 2 + upper half, so that a lane's four are consecutive and one stream brings all that a block
// needs.  The blocks of 4 x 32 features stand together, then come the next 128 k.  k and features are padded to 128 with
// zero scales and codes equal to their zero points.
#pragma once
#include "lckv_project.cuh"

namespace lckv {

constexpr int kQuantFeat = 32;       // features per block of the layout
constexpr int kQuantK = 128;         // k per block of the layout
constexpr int kQuantCodes = kQuantFeat * kQuantK / 2;        // bytes of a block's codes

struct QuantLayout {
    int64_t total;                       // bytes
    int32_t n_blocks, k_blocks;          // n_blocks: a multiple of 4
    int32_t per_block;                   // groups of a block
    int32_t block_bytes, zeros_off;      // zeros_off within a block; 0: none
};
__host__ __device__ inline QuantLayout quant_layout(int64_t n, int64_t k, int group, bool zeros)
{
    QuantLayout y;
    y.n_blocks = (int32_t)((n + 4 * kQuantFeat - 1) / (4 * kQuantFeat)) * 4;
    y.k_blocks = (int32_t)((k + kQuantK - 1) / kQuantK);
    y.per_block = kQuantK / group;
    const int scales = y.per_block * kQuantFeat * 2;
    y.zeros_off = zeros ? kQuantCodes + scales : 0;
    y.block_bytes = kQuantCodes + scales + (zeros ? scales / 2 : 0);
    y.total = (int64_t)y.n_blocks * y.k_blocks * y.block_bytes;
    return y;
}

struct QuantPackParams {
    const uint8_t* codes;    // [n, k / 2], low nibble = even k
    const uint16_t* scales;  // [n, k / group] bf16
    const uint8_t* zeros;    // [n, k / group] or null
    uint8_t* out;
    int32_t n, k, group;
};

// *flag = 1 if one of the n zero points lies above 15.
__global__ void __launch_bounds__(256) quant_zeros_kernel(const uint8_t* zeros, int64_t n, int32_t* flag)
{
    bool bad = false;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (int64_t)gridDim.x * blockDim.x) bad |= zeros[i] > 15;
    if (bad) atomicExch(flag, 1);
}

// A thread block per (32 features, 128 k): one thread per 32-bit word of its codes, then one per scale.
__global__ void __launch_bounds__(256) quant_pack_kernel(const QuantPackParams p)
{
    const QuantLayout y = quant_layout(p.n, p.k, p.group, p.zeros != nullptr);
    const int src_groups = p.k / p.group;
    const int64_t n_all = (int64_t)y.n_blocks * y.k_blocks;
    for (int64_t blk = blockIdx.x; blk < n_all; blk += gridDim.x) {
        const int kb = (int)((blk >> 2) % y.k_blocks), nb = (int)((blk >> 2) / y.k_blocks) * 4 + (int)(blk & 3);
        uint8_t* out = p.out + blk * y.block_bytes;
        for (int i = threadIdx.x; i < kQuantCodes / 4; i += blockDim.x) {
            const int lane = (i >> 2) & 31, tile = (i >> 7) & 1, half = i >> 8;
            const int f = nb * kQuantFeat + tile * 16 + (i & 1) * 8 + (lane >> 2);
            uint32_t w = 0;
            for (int e = 0; e < 8; ++e) {
                const int step = e >> 2, kk = e & 3;
                const int k = kb * kQuantK + half * 64 + ((i >> 1) & 1) * 32 + step * 16 + (lane & 3) * 4 + kk;
                uint32_t c = p.zeros ? 0u : 8u;                                     // padding: equal to its zero point
                if (f < p.n && k < p.k) {
                    const uint8_t two = p.codes[(int64_t)f * (p.k / 2) + k / 2];
                    c = ((k & 1) ? two >> 4 : two) & 15;
                }
                c <<= 3 + 16 * (kk & 1);
                w |= __funnelshift_l(c, c, 4 * ((kk >> 1) * 2 + step));
            }
            reinterpret_cast<uint32_t*>(out)[i] = w;
        }
        for (int i = threadIdx.x; i < y.per_block * kQuantFeat; i += blockDim.x) {
            const int o = i & 31, grp = kb * y.per_block + (i >> 5);                // o = g * 4 + tile * 2 + hi
            const int f = nb * kQuantFeat + ((o >> 1) & 1) * 16 + (o & 1) * 8 + (o >> 2);
            const bool in = f < p.n && grp < src_groups;
            reinterpret_cast<uint16_t*>(out + kQuantCodes)[i] = in ? p.scales[(int64_t)f * src_groups + grp] : (uint16_t)0;
            // a zero point is kept as the low byte of the bf16 number 16 + z (0x4180 + 8 z)
            if (p.zeros) out[y.zeros_off + i] = 0x80 | (in ? p.zeros[(int64_t)f * src_groups + grp] << 3 : 0);
        }
    }
}

struct QuantParams {
    const uint8_t* w;        // the packed blocks
    const void* x;           // bf16 or e4m3 [m, k]
    const float* x_scale;    // e4m3: [m] or [m, x_blocks]
    void* y;
    int64_t x_stride, y_stride;
    int32_t m, n, k, group;
    int32_t n_blocks, k_blocks;
    int32_t x_blocks;        // scales per row of x when there is one per 128 k, else 0
    int32_t y32;
    int32_t k_split;         // thread blocks of a cluster that share the k range
};

// c (+)= a b, m16n8k16 in bf16 or fp16; FIRST starts from zero
template <bool F8, bool FIRST>
__device__ __forceinline__ void quant_mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    if (FIRST) c[0] = c[1] = c[2] = c[3] = 0.f;
    float d0, d1, d2, d3;
    if (F8)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
            : "=f"(d0), "=f"(d1), "=f"(d2), "=f"(d3)
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
            : "=f"(d0), "=f"(d1), "=f"(d2), "=f"(d3)
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
    c[0] = d0; c[1] = d1; c[2] = d2; c[3] = d3;
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void prefetch_l2(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }

// A lane's part of x for one half (64 k) of a block and one tile of 8 rows: 4 k of each k16 step of row g, raw.  (Ordinary loads:
// see lckv_rope.cuh.)
template <bool F8> struct QuantX;
template <> struct QuantX<false> {
    uint2 v[4];
    __device__ __forceinline__ void load(const uint8_t* p)
    {
#pragma unroll
        for (int s = 0; s < 4; ++s) v[s] = *reinterpret_cast<const uint2*>(p + s * 32);
    }
    __device__ __forceinline__ void load_part(const uint8_t* p, bool in, bool in2)
    {
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            v[s] = make_uint2(0, 0);
            if (s < 2 ? in : in2) v[s] = *reinterpret_cast<const uint2*>(p + s * 32);
        }
    }
    // k16 step S of the half
    template <int S> __device__ __forceinline__ void frag(uint32_t& b0, uint32_t& b1) const { b0 = v[S].x; b1 = v[S].y; }
};
template <> struct QuantX<true> {
    uint32_t v[4];
    __device__ __forceinline__ void load(const uint8_t* p)
    {
#pragma unroll
        for (int s = 0; s < 4; ++s) v[s] = *reinterpret_cast<const uint32_t*>(p + s * 16);
    }
    __device__ __forceinline__ void load_part(const uint8_t* p, bool in, bool in2)
    {
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            v[s] = 0;
            if (s < 2 ? in : in2) v[s] = *reinterpret_cast<const uint32_t*>(p + s * 16);
        }
    }
    // k16 step S of the half, in fp16
    template <int S> __device__ __forceinline__ void frag(uint32_t& b0, uint32_t& b1) const
    {
        asm("{\n\t.reg .b16 lo, hi;\n\t"
            "mov.b32 {lo, hi}, %2;\n\t"
            "cvt.rn.f16x2.e4m3x2 %0, lo;\n\t"
            "cvt.rn.f16x2.e4m3x2 %1, hi;\n\t}"
            : "=r"(b0), "=r"(b1) : "r"(v[S]));
    }
};

// (a & mask) | bits in one instruction (left to itself the compiler took two, each with one immediate: 15.9 us where
// this takes 12.8 for a row of 4096 times 22016 features)
__device__ __forceinline__ uint32_t and_or(uint32_t a, uint32_t mask, uint32_t bits)
{
    uint32_t d;
    asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(d) : "r"(a), "r"(mask), "r"(bits));
    return d;
}

__device__ __forceinline__ uint32_t sub_bf16x2(uint32_t a, uint32_t b)
{
    uint32_t d;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t sub_f16x2(uint32_t a, uint32_t b)
{
    uint32_t d;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}

// 32 k of a warp (first or second of a half): FT tiles of 16 features times NT tiles of 8 rows.  zp: 16 + z of features g and
// g + 8 of each tile, as pairs.  FIRST: of a group.
template <bool F8, int FT, int NT, int SECOND, bool FIRST>
__device__ __forceinline__ void quant_32k(float (&grp)[FT][NT][4], const uint32_t (&zp)[FT][2], const uint4 (&c)[FT], const QuantX<F8> (&x)[NT])
{
    constexpr uint32_t MASK = F8 ? 0x03c003c0u : 0x00780078u, SIXTEEN = F8 ? 0x4c004c00u : 0x41804180u;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        uint32_t b[NT][2];
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            if (s == 0) x[j].template frag<SECOND * 2>(b[j][0], b[j][1]);
            else x[j].template frag<SECOND * 2 + 1>(b[j][0], b[j][1]);
        }
#pragma unroll
        for (int i = 0; i < FT; ++i) {
            const uint32_t w0 = SECOND ? c[i].z : c[i].x, w1 = SECOND ? c[i].w : c[i].y;     // features g and g + 8
            uint32_t a[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const uint32_t w = r & 1 ? w1 : w0;
                const uint32_t u = and_or(__funnelshift_r(w, w, (4 * (s + (r & 2)) + (F8 ? 29 : 0)) & 31), MASK, SIXTEEN);
                a[r] = F8 ? sub_f16x2(u, zp[i][r & 1]) : sub_bf16x2(u, zp[i][r & 1]);
            }
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                if (s == 0) quant_mma<F8, FIRST>(grp[i][j], a, b[j][0], b[j][1]);
                else quant_mma<F8, false>(grp[i][j], a, b[j][0], b[j][1]);
            }
        }
    }
}

__host__ __device__ constexpr int quant_warps(int NT) { return NT == 1 ? 8 : 4; }            // per thread block
__host__ __device__ constexpr int quant_slots(int FT) { return FT == 2 ? 4 : 3; }            // blocks in flight per warp
__host__ __device__ constexpr int quant_ctas(int FT, int NT) { return NT == 1 ? (FT == 2 ? 3 : 2) : 3; }   // per SM

// grid: (groups of 16 FT features, tiles of 8 NT rows, k_split), a cluster along z.  The warps of a cluster share the
// k blocks in even runs, each with its own ring of blocks in shared memory, filled by asynchronous copies (a lane copies
// the codes that it will use itself); x comes straight from the L1 and L2 into registers, one block ahead.  A warp
// accumulates 16 FT features x 8 NT rows, and the partial sums are added in a fixed order through shared memory:
// first the warps of a thread block, then the thread blocks of the cluster.  Rows behind the last one repeat it and
// are dropped at the end.
//
// The launch carries the programmatic-serialization attribute: the first blocks of weights, which never are the output
// of the kernel before this one, are requested before its end, x is read after it.
template <bool F8, bool ZEROS, int GROUP, int FT, int NT>
__global__ void __launch_bounds__(quant_warps(NT) * 32, quant_ctas(FT, NT)) quant_mma_kernel(const QuantParams p)
{
    constexpr int COLS = 8 * NT, FEAT = 16 * FT, LD = FEAT + 4, NB = FT / 2, SLOTS = quant_slots(FT), WARPS = quant_warps(NT);
    constexpr int SCALES = kQuantK / GROUP * kQuantFeat * 2, BLOCK = kQuantCodes + SCALES + (ZEROS ? SCALES / 2 : 0);
    extern __shared__ __align__(16) uint8_t quant_smem[];       // [warps][slots][NB blocks]; partial sums afterwards
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const int m0 = blockIdx.y * COLS;
    const int KS = p.k_split, rank = KS > 1 ? (int)cluster_ctarank() : 0;
    const int share = rank * WARPS + warp, shares = KS * WARPS;
    const int kb0 = (int)((uint32_t)(share * p.k_blocks) / (uint32_t)shares), kb1 = (int)((uint32_t)((share + 1) * p.k_blocks) / (uint32_t)shares);
    const uint32_t ring = smem_u32(quant_smem) + warp * (SLOTS * NB * BLOCK);
    // the warp's NB blocks of 32 features, neighbours within their 4
    const int nb0 = blockIdx.x * NB;
    const uint8_t* src0 = p.w + (((int64_t)(nb0 >> 2) * p.k_blocks + kb0) * 4 + (nb0 & 3)) * BLOCK + lane * 16;

    auto fetch = [&](int kb, int slot, const uint8_t* src) {
        if (kb < kb1) {
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const uint32_t dst = ring + (slot * NB + b) * BLOCK + lane * 16;
                const uint8_t* s = src + b * BLOCK;
#pragma unroll
                for (int o = 0; o < kQuantCodes; o += 512) cp_async16(dst + o, s + o);
                if (lane < (BLOCK - kQuantCodes) / 16) cp_async16(dst + kQuantCodes, s + kQuantCodes);
            }
        }
        cp_async_commit();
    };
#pragma unroll
    for (int i = 0; i < SLOTS - 1; ++i) {
        fetch(kb0 + i, i, src0);
        src0 += 4 * BLOCK;
    }
    pdl_wait_then_release();

    constexpr int XB = F8 ? 1 : 2;                               // bytes per element of x
    const uint8_t* px[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int m = m0 + j * 8 + g;
        px[j] = static_cast<const uint8_t*>(p.x) + ((int64_t)(m < p.m ? m : p.m - 1) * p.x_stride + kb0 * kQuantK + t * 4) * XB;
    }
    QuantX<F8> xr[2][NT];
    auto fetch_x = [&](int kb, int h) {                          // at px, which stands at block kb
        const int kh = kb * kQuantK + h * 64;
        if (kh + 64 <= p.k) {
#pragma unroll
            for (int j = 0; j < NT; ++j) xr[h][j].load(px[j] + h * 64 * XB);
        } else {                                                 // the last k, or behind them
#pragma unroll
            for (int j = 0; j < NT; ++j) xr[h][j].load_part(px[j] + h * 64 * XB, kh < p.k, kh + 32 < p.k);
        }
    };
    fetch_x(kb0, 0);
    fetch_x(kb0, 1);

    uint64_t acc[FT][NT][2];                         // pairs of columns, features g and g + 8
    float grp[FT][NT][4];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int i = 0; i < FT; ++i) acc[i][j][0] = acc[i][j][1] = 0;

    // scales of x, one per column 2 t, 2 t + 1 of each tile: of the block (fetched a block ahead) or of the row (at the end)
    float xs[NT][2];
    const float* px_scale[NT][2];
    if (F8) {
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int m = m0 + j * 8 + t * 2 + e;
                px_scale[j][e] = p.x_scale + (int64_t)(m < p.m ? m : p.m - 1) * (p.x_blocks ? p.x_blocks : 1) + (p.x_blocks ? kb0 : 0);
                xs[j][e] = p.x_blocks && kb0 < kb1 ? *px_scale[j][e] : 1.f;
            }
    }

    int slot = 0;
    for (int kb = kb0; kb < kb1; ++kb) {
        fetch(kb + SLOTS - 1, slot == 0 ? SLOTS - 1 : slot - 1, src0);
        src0 += 4 * BLOCK;
        cp_async_wait<SLOTS - 1>();
        __syncwarp();
        const uint32_t blk = ring + slot * (NB * BLOCK);
        slot = slot == SLOTS - 1 ? 0 : slot + 1;
        // The zero points of group gi of the block.
        uint32_t zp[FT][2];
        auto zero_points = [&](int gi) {
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                uint32_t z = 0;
                if (ZEROS) asm volatile("ld.shared.u32 %0, [%1];" : "=r"(z) : "r"(blk + b * BLOCK + kQuantCodes + SCALES + gi * kQuantFeat + g * 4));
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t& to = zp[b * 2 + (i >> 1)][i & 1];
                    if (!ZEROS) to = F8 ? 0x4e004e00u : 0x41c041c0u;                              // 24
                    else if (F8) to = (__byte_perm(z, 0u, 0x4040u + 0x0101u * i) << 3) + 0x48004800u;    // (the stored byte is 0x80 + 8 z)
                    else to = __byte_perm(z, 0x41414141u, 0x4040u + 0x0101u * i);
                }
            }
        };
        // A complete group: its scales; two columns per instruction.  With a scale of x per block the groups of the block are
        // summed first.
        uint64_t blk_sum[FT][NT][2];
        auto fold = [&](int gi) {
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                uint32_t sw[2];
                asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(sw[0]), "=r"(sw[1]) : "r"(blk + b * BLOCK + kQuantCodes + gi * (kQuantFeat * 2) + g * 8));
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int hi = 0; hi < 2; ++hi) {
                        const float f = hi ? bf16hi(sw[i]) : bf16lo(sw[i]);
                        const uint64_t f2 = pack_f32x2(f, f);
#pragma unroll
                        for (int j = 0; j < NT; ++j) {
                            const uint64_t v = pack_f32x2(grp[b * 2 + i][j][hi * 2], grp[b * 2 + i][j][hi * 2 + 1]);
                            if (F8 && GROUP < kQuantK) {
                                blk_sum[b * 2 + i][j][hi] = gi == 0 ? fmul2(f2, v) : ffma2(f2, v, blk_sum[b * 2 + i][j][hi]);
                            } else if (F8) {
                                blk_sum[b * 2 + i][j][hi] = fmul2(f2, v);
                            } else {
                                acc[b * 2 + i][j][hi] = ffma2(f2, v, acc[b * 2 + i][j][hi]);
                            }
                        }
                    }
            }
        };
#pragma unroll
        for (int j = 0; j < NT; ++j) px[j] += kQuantK * XB;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint4 c[FT];
#pragma unroll
            for (int i = 0; i < FT; ++i) c[i] = lds128(blk + (i >> 1) * BLOCK + ((h * 2 + (i & 1)) * 32 + lane) * 16);
            if (h == 0 || GROUP <= 64) zero_points(GROUP == 32 ? h * 2 : GROUP == 64 ? h : 0);
            if (h == 0 || GROUP <= 64) quant_32k<F8, FT, NT, 0, true>(grp, zp, c, xr[h]);
            else quant_32k<F8, FT, NT, 0, false>(grp, zp, c, xr[h]);
            if (GROUP == 32) {
                fold(h * 2);
                zero_points(h * 2 + 1);
            }
            quant_32k<F8, FT, NT, 1, GROUP == 32>(grp, zp, c, xr[h]);
            if (kb + 1 < kb1) fetch_x(kb + 1, h);
            if (h == 1 || GROUP <= 64) fold(GROUP == 32 ? h * 2 + 1 : GROUP == 64 ? h : 0);
        }
        if (F8) {
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const uint64_t x2 = pack_f32x2(xs[j][0], xs[j][1]);
#pragma unroll
                for (int i = 0; i < FT; ++i)
#pragma unroll
                    for (int hi = 0; hi < 2; ++hi) acc[i][j][hi] = ffma2(x2, blk_sum[i][j][hi], acc[i][j][hi]);
                if (p.x_blocks && kb + 1 < kb1) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) xs[j][e] = *++px_scale[j][e];
                }
            }
        }
        __syncwarp();                                // every lane has read the slot before it is filled again
    }

    cp_async_wait<0>();
    __syncthreads();                                 // the rings become the partial sums: [warps][COLS][LD]
    static_assert(SLOTS * NB * BLOCK >= COLS * LD * 4, "the partial sums fit into the rings");
    float* part = reinterpret_cast<float*>(quant_smem);
    float* mine = part + (size_t)warp * COLS * LD;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        float xr_scale[2] = {1.f, 1.f};
        if (F8 && !p.x_blocks) {
#pragma unroll
            for (int e = 0; e < 2; ++e) xr_scale[e] = *px_scale[j][e];
        }
#pragma unroll
        for (int i = 0; i < FT; ++i)
#pragma unroll
            for (int hi = 0; hi < 2; ++hi) {
                float v0, v1;
                unpack_f32x2(acc[i][j][hi], v0, v1);
                float* at = mine + (j * 8 + t * 2) * LD + i * 16 + g + hi * 8;
                at[0] = v0 * xr_scale[0];
                at[LD] = v1 * xr_scale[1];
            }
    }
    __syncthreads();
    // the thread block's sum over its warps, in place in the first warp's part (each thread its own places)
    for (int i = tid; i < COLS * FEAT / 4; i += WARPS * 32) {
        const int c = i / (FEAT / 4), f = (i % (FEAT / 4)) * 4;
        float4 v = *reinterpret_cast<const float4*>(part + c * LD + f);
#pragma unroll
        for (int w = 1; w < WARPS; ++w) {
            const float4 u = *reinterpret_cast<const float4*>(part + ((size_t)w * COLS + c) * LD + f);
            v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
        }
        *reinterpret_cast<float4*>(part + c * LD + f) = v;
    }
    __syncthreads();
    if (KS > 1) cluster_sync_all();
    // each thread block of the cluster finishes a share of the places
    for (int i = rank * (WARPS * 32) + tid; i < COLS * FEAT / 4; i += KS * WARPS * 32) {
        const int c = i / (FEAT / 4), f = (i % (FEAT / 4)) * 4;
        float v[4] = {0.f, 0.f, 0.f, 0.f};
        for (int r = 0; r < KS; ++r) {
            const float4 u = KS > 1 ? ld_cluster_f4(smem_u32(part + c * LD + f), (uint32_t)r)
                                    : *reinterpret_cast<const float4*>(part + c * LD + f);
            v[0] += u.x; v[1] += u.y; v[2] += u.z; v[3] += u.w;
        }
        const int m = m0 + c, n = blockIdx.x * FEAT + f;
        if (m >= p.m) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (n + e >= p.n) break;
            if (p.y32) static_cast<float*>(p.y)[(int64_t)m * p.y_stride + n + e] = v[e];
            else static_cast<uint16_t*>(p.y)[(int64_t)m * p.y_stride + n + e] = (uint16_t)f32_to_bf16_bits(v[e]);
        }
    }
    if (KS > 1) cluster_sync_all();                  // a thread block's shared memory outlives the others' reads
}

}  // namespace lckv
