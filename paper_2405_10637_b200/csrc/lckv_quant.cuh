// Products with 4-bit weights: y[m, n] = sum_k x[m, k] * s[n, k/g] * (c[n, k] - z[n, k/g]), for the few rows m
// of a decode step.  c in 0 .. 15, one scale s (bf16) and one zero point z (0 .. 15, or 8 everywhere) per group
// of g = 32, 64 or 128 consecutive k.
//
// Bound by the bytes of the codes: 2 m multiply-adds per half byte.  The operands are swapped so that 16
// output features are the rows of an m16n8k16 tile and up to 8 rows of x its columns.  c - z is exact in
// bf16 (and in fp16), so the tensor cores see exact weights: a group's sum is accumulated in fp32 and
// multiplied by its scale in fp32 afterwards; nothing is rounded before the output.
//
// Layout (quant_pack_kernel, once per weight).  The codes are cut into blocks of 64 features x 128 k = 4 KB,
// k fastest; such a block holds [2 halves of 64 k][4 tiles of 16 features][32 lanes][16 bytes], where lane
// (g, t) of a tile (g = lane / 4, t = lane % 4) owns features g and g + 8 and, of each 32 k of the half, k = 8 t ..
// 8 t + 7: word s of its 16 bytes is one k16 step's A fragment, words 0 and 1 the first 32 k, 2 and 3 the second.
// Any k order within a group serves a sum, so step s simply takes k = 32 (s / 2) + 8 t + 4 (s % 2) + {0, 1, 2, 3}
// where the fragment wants 2 t, 2 t + 1, 2 t + 8, 2 t + 9; the matching B fragments of two steps are then 16
// consecutive bytes of a row of x.
// The nibbles of a word are ordered so that (word >> 4 i) & 0x000f000f is the pair of fragment register i; or'ed
// onto 0x4300 (bf16 128) a nibble c reads as 128 + c, and subtracting 128 + z is exact.
// Scales and zero points: [block of 64 features][group][64], in the order g * 8 + tile * 2 + upper half, so that a
// lane's eight are consecutive.  k is padded to 128 and features to 64 with zero scales and codes equal to zero.
#pragma once
#include "lckv_project.cuh"

namespace lckv {

constexpr int kQuantFeat = 64;       // features per block of the layout
constexpr int kQuantK = 128;         // k per block of the layout
constexpr int kQuantWarps = 8;

struct QuantLayout {
    int64_t codes_bytes, scales_off, zeros_off, total;   // zeros_off = 0: none
    int32_t n_blocks, k_blocks, groups;                  // groups per feature, padded
};
__host__ __device__ inline QuantLayout quant_layout(int64_t n, int64_t k, int group, bool zeros)
{
    QuantLayout y;
    y.n_blocks = (int32_t)((n + kQuantFeat - 1) / kQuantFeat);
    y.k_blocks = (int32_t)((k + kQuantK - 1) / kQuantK);
    y.groups = y.k_blocks * (kQuantK / group);
    y.codes_bytes = (int64_t)y.n_blocks * y.k_blocks * (kQuantFeat * kQuantK / 2);
    y.scales_off = y.codes_bytes;
    const int64_t s = (int64_t)y.n_blocks * y.groups * kQuantFeat;
    y.zeros_off = zeros ? y.scales_off + 2 * s : 0;
    y.total = y.scales_off + 2 * s + (zeros ? s : 0);
    return y;
}

struct QuantPackParams {
    const uint8_t* codes;    // [n, k / 2], low nibble = even k
    const uint16_t* scales;  // [n, k / group] bf16
    const uint8_t* zeros;    // [n, k / group] or null
    uint8_t* out;
    int32_t n, k, group;
};

// One thread per 32-bit word of the packed codes, then one per scale.
__global__ void __launch_bounds__(256) quant_pack_kernel(const QuantPackParams p)
{
    const QuantLayout y = quant_layout(p.n, p.k, p.group, p.zeros != nullptr);
    const int64_t n_words = y.codes_bytes / 4, n_scales = (int64_t)y.n_blocks * y.groups * kQuantFeat;
    const int src_groups = p.k / p.group;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n_words + n_scales;
         i += (int64_t)gridDim.x * blockDim.x) {
        if (i < n_words) {
            const int s = (int)(i & 3), lane = (int)(i >> 2) & 31, tile = (int)(i >> 7) & 3, half = (int)(i >> 9) & 1;
            const int64_t blk = i >> 10;
            const int kb = (int)(blk % y.k_blocks), nb = (int)(blk / y.k_blocks);
            const int k0 = kb * kQuantK + half * 64 + (s >> 1) * 32 + (lane & 3) * 8 + (s & 1) * 4;   // 4 consecutive k
            uint32_t w = 0;
            for (int hi = 0; hi < 2; ++hi) {
                const int f = nb * kQuantFeat + tile * 16 + hi * 8 + (lane >> 2);
                for (int e = 0; e < 4; ++e) {
                    uint32_t c = p.zeros ? 0u : 8u;                                 // padding: equal to its zero point
                    if (f < p.n && k0 + e < p.k) {
                        const uint8_t two = p.codes[(int64_t)f * (p.k / 2) + (k0 + e) / 2];
                        c = ((e & 1) ? two >> 4 : two) & 15;
                    }
                    // register i = (e / 2) * 2 + hi, element e % 2 of its pair
                    w |= c << (4 * ((e >> 1) * 2 + hi) + 16 * (e & 1));
                }
            }
            reinterpret_cast<uint32_t*>(p.out)[i] = w;
        } else {
            const int64_t j = i - n_words;
            const int o = (int)(j & 63);                                            // g * 8 + tile * 2 + hi
            const int64_t rest = j >> 6;
            const int grp = (int)(rest % y.groups), nb = (int)(rest / y.groups);
            const int f = nb * kQuantFeat + ((o >> 1) & 3) * 16 + (o & 1) * 8 + (o >> 3);
            const bool in = f < p.n && grp < src_groups;
            reinterpret_cast<uint16_t*>(p.out + y.scales_off)[j] = in ? p.scales[(int64_t)f * src_groups + grp] : (uint16_t)0;
            if (p.zeros) p.out[y.zeros_off + j] = in ? (p.zeros[(int64_t)f * src_groups + grp] & 15) : (uint8_t)0;
        }
    }
}

struct QuantParams {
    const uint8_t* codes;
    const uint16_t* scales;
    const uint8_t* zeros;
    const void* x;           // bf16 or e4m3 [m, k]
    const float* x_scale;    // e4m3: [m] or [m, x_blocks]
    void* y;
    int64_t x_stride, y_stride;
    int32_t m, n, k, group, group_shift;
    int32_t n_blocks, k_blocks, groups;
    int32_t x_blocks;        // scales per row of x when there is one per 128 k, else 0
    int32_t y32;
    int32_t k_split;         // blocks of a cluster that share the k range
};

__device__ __forceinline__ uint32_t sub_pair(uint32_t a, uint32_t b, bool f16)
{
    uint32_t d;
    if (f16) asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    else asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
template <bool F16>
__device__ __forceinline__ void quant_mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    if (F16)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Two e4m3 values as a pair of fp16 (exact).
__device__ __forceinline__ uint32_t e4m3_to_f16x2(uint32_t two)
{
    uint32_t d;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(d) : "h"((uint16_t)two));
    return d;
}

// grid: (blocks of 64 features, tiles of 8 NT rows, k_split), a cluster along z.  The warps of a cluster take the
// k blocks in turn; each accumulates 64 features x 8 NT rows, and the partial sums are added in a fixed order
// through shared memory: first the warps of a block, then the blocks of the cluster.
template <bool F8, bool ZEROS, int NT>
__global__ void __launch_bounds__(kQuantWarps * 32) quant_mma_kernel(const QuantParams p)
{
    constexpr int COLS = 8 * NT, LD = kQuantFeat + 4;
    extern __shared__ __align__(16) float part[];       // [warps][COLS][LD]; the block's sum ends up in [0]
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const int nb = blockIdx.x, m0 = blockIdx.y * COLS;
    const int KS = p.k_split, rank = KS > 1 ? (int)cluster_ctarank() : 0;
    pdl_wait_then_release();
    float acc[4][NT][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][j][e] = 0.f;
    constexpr uint32_t magic = F8 ? 0x64006400u : 0x43004300u;
    const int per128 = kQuantK / p.group;

    for (int kb = rank * kQuantWarps + warp; kb < p.k_blocks; kb += KS * kQuantWarps) {
        const uint4* blk = reinterpret_cast<const uint4*>(p.codes + ((int64_t)nb * p.k_blocks + kb) * 4096);
        uint4 c4[2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) c4[h][i] = __ldcs(blk + (h * 4 + i) * 32 + lane);
        float grp[4][NT][4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) grp[i][j][e] = 0.f;
        // scales of x for this block: one per column 2 t, 2 t + 1 of each tile
        float xs[NT][2];
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int m = m0 + j * 8 + t * 2 + e;
                xs[j][e] = 1.f;
                if (F8 && m < p.m) xs[j][e] = p.x_blocks ? __ldg(p.x_scale + (int64_t)m * p.x_blocks + kb) : __ldg(p.x_scale + m);
            }
        uint32_t zp[4][2];                               // 128 + z (or 1024 + z) twice, features g and g + 8 of a tile
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            // B fragments: 8 consecutive k of row g of each tile of x, twice (k is a multiple of 32)
            uint32_t bx[NT][8];
            const int kh = kb * kQuantK + h * 64, k0 = kh + t * 8;
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const int m = m0 + j * 8 + g;
                const bool in = m < p.m && kh < p.k, in2 = m < p.m && kh + 32 < p.k;
                if (F8) {
                    uint2 v = make_uint2(0, 0), u = v;
                    const uint2* px = reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(p.x) + (int64_t)m * p.x_stride + k0);
                    if (in) v = __ldg(px);
                    if (in2) u = __ldg(px + 4);
                    const uint32_t w[4] = {v.x, v.y, u.x, u.y};
#pragma unroll
                    for (int s = 0; s < 4; ++s) {
                        bx[j][2 * s] = e4m3_to_f16x2(w[s] & 0xffffu);
                        bx[j][2 * s + 1] = e4m3_to_f16x2(w[s] >> 16);
                    }
                } else {
                    uint4 v = make_uint4(0, 0, 0, 0), u = v;
                    const uint4* px = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.x) + (int64_t)m * p.x_stride + k0);
                    if (in) v = __ldg(px);
                    if (in2) u = __ldg(px + 4);
                    bx[j][0] = v.x; bx[j][1] = v.y; bx[j][2] = v.z; bx[j][3] = v.w;
                    bx[j][4] = u.x; bx[j][5] = u.y; bx[j][6] = u.z; bx[j][7] = u.w;
                }
            }
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const int step = h * 4 + s;              // k16 step within the block
                if (((step * 16) & (p.group - 1)) == 0 && (ZEROS || step == 0)) {
                    const int gi = kb * per128 + ((step * 16) >> p.group_shift);
                    uint32_t z8[2] = {0x08080808u, 0x08080808u};
                    if (ZEROS) {
                        const uint2 zz = __ldg(reinterpret_cast<const uint2*>(p.zeros + ((int64_t)nb * p.groups + gi) * kQuantFeat + g * 8));
                        z8[0] = zz.x;
                        z8[1] = zz.y;
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const uint32_t z = (z8[i >> 1] >> (16 * (i & 1) + 8 * e)) & 0xffu;
                            zp[i][e] = magic | z | (z << 16);
                        }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t w = s == 0 ? c4[h][i].x : s == 1 ? c4[h][i].y : s == 2 ? c4[h][i].z : c4[h][i].w;
                    uint32_t a[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        a[r] = sub_pair(((w >> (4 * r)) & 0x000f000fu) | magic, zp[i][r & 1], F8);
#pragma unroll
                    for (int j = 0; j < NT; ++j) quant_mma<F8>(grp[i][j], a, bx[j][2 * s], bx[j][2 * s + 1]);
                }
                if ((((step + 1) * 16) & (p.group - 1)) == 0) {
                    // the group is complete: its fp32 sum times its scale (and x's)
                    const int gi = kb * per128 + ((step * 16) >> p.group_shift);
                    const uint4 sv = __ldg(reinterpret_cast<const uint4*>(p.scales + ((int64_t)nb * p.groups + gi) * kQuantFeat + g * 8));
                    const uint32_t sw[4] = {sv.x, sv.y, sv.z, sv.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int j = 0; j < NT; ++j)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                float f = (e & 2) ? bf16hi(sw[i]) : bf16lo(sw[i]);
                                if (F8) f *= xs[j][e & 1];
                                acc[i][j][e] = fmaf(f, grp[i][j][e], acc[i][j][e]);
                                grp[i][j][e] = 0.f;
                            }
                }
            }
        }
    }

    float* mine = part + (size_t)warp * COLS * LD;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                mine[(j * 8 + t * 2 + (e & 1)) * LD + i * 16 + g + (e & 2) * 4] = acc[i][j][e];
    __syncthreads();
    // the block's sum over its warps, in place in the first warp's part (each thread its own places)
    for (int i = tid; i < COLS * kQuantFeat / 4; i += kQuantWarps * 32) {
        const int c = i / (kQuantFeat / 4), f = (i % (kQuantFeat / 4)) * 4;
        float4 v = *reinterpret_cast<const float4*>(part + c * LD + f);
#pragma unroll
        for (int w = 1; w < kQuantWarps; ++w) {
            const float4 u = *reinterpret_cast<const float4*>(part + ((size_t)w * COLS + c) * LD + f);
            v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
        }
        *reinterpret_cast<float4*>(part + c * LD + f) = v;
    }
    __syncthreads();
    if (KS > 1) cluster_sync_all();
    // each block of the cluster finishes a share of the places
    for (int i = rank * (kQuantWarps * 32) + tid; i < COLS * kQuantFeat / 4; i += KS * kQuantWarps * 32) {
        const int c = i / (kQuantFeat / 4), f = (i % (kQuantFeat / 4)) * 4;
        float v[4] = {0.f, 0.f, 0.f, 0.f};
        for (int r = 0; r < KS; ++r) {
            const float4 u = KS > 1 ? ld_cluster_f4(smem_u32(part + c * LD + f), (uint32_t)r)
                                    : *reinterpret_cast<const float4*>(part + c * LD + f);
            v[0] += u.x; v[1] += u.y; v[2] += u.z; v[3] += u.w;
        }
        const int m = m0 + c, n = nb * kQuantFeat + f;
        if (m >= p.m) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (n + e >= p.n) break;
            if (p.y32) static_cast<float*>(p.y)[(int64_t)m * p.y_stride + n + e] = v[e];
            else static_cast<uint16_t*>(p.y)[(int64_t)m * p.y_stride + n + e] = (uint16_t)f32_to_bf16_bits(v[e]);
        }
    }
    if (KS > 1) cluster_sync_all();                      // a block's shared memory outlives the others' reads
}

}  // namespace lckv
