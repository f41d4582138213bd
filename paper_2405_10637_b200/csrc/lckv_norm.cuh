// Root-mean-square norm of rows, with the residual's addition before it and an optional 8-bit output.
//
//   h = x + r;   y = h / sqrt(mean(h^2) + eps) * w      (fp32; the mean over the row's `width` elements)
//   8 bits: scale = max|y| / 448 over a row or over 128 columns, q = e4m3(y / scale), 448 = largest e4m3
//
// h is rounded once to its own type when it is stored; the norm uses the unrounded sum.  Bound by
// memory: each element is read once and written once, so a row's elements stay in registers between the
// pass that sums squares and the one that scales.  A thread holds NV vectors of 8 consecutive elements,
// vector i of the row at i * threads + thread, so that every access is coalesced and 16 consecutive lanes
// hold one 128-column block.
//
// Rows of any other width or alignment (norm_any_kernel) go element by element, staged in shared memory as
// fp32.
#pragma once
#include "lckv_device.cuh"

namespace lckv {

constexpr int kNormMaxWidth = 32768;
constexpr float kE4m3Max = 448.f;

struct NormParams {
    const void* x;
    const void* r;           // residual in, or null
    void* h;                 // residual out, or null
    const void* w;
    void* y;
    float* scale;
    int64_t x_stride;
    int32_t rows, width;
    float eps;
    int32_t x32, r32, w32;   // 1: fp32, 0: bf16
    int32_t out;             // 0 bf16, 1 fp32, 2 e4m3
    int32_t group;           // 8-bit output: 0 = one scale per row, 128 = one per 128 columns
    int32_t n_groups;        // scales per row
};

// max that keeps a NaN of either side
__device__ __forceinline__ float max_nan(float a, float b)
{
    float m;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(b));
    return m;
}
__device__ __forceinline__ uint32_t cvt_e4m3_pair(float lo, float hi)
{
    uint16_t v;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(v) : "f"(hi), "f"(lo));
    return v;
}
// Eight values over their scale, as e4m3.  A block of zeros has scale 0 and stays 0; where the scale is so
// small that its inverse overflows, both sides are multiplied by 2^100 first.
__device__ __forceinline__ uint2 norm_quant8(const float (&f)[8], float s)
{
    float pre = 1.f, inv = 0.f;
    if (s != 0.f) {
        if (s < 0x1p-120f) { pre = 0x1p100f; s *= 0x1p100f; }
        inv = 1.f / s;
    }
    uint2 q;
    q.x = cvt_e4m3_pair(f[0] * pre * inv, f[1] * pre * inv) | (cvt_e4m3_pair(f[2] * pre * inv, f[3] * pre * inv) << 16);
    q.y = cvt_e4m3_pair(f[4] * pre * inv, f[5] * pre * inv) | (cvt_e4m3_pair(f[6] * pre * inv, f[7] * pre * inv) << 16);
    return q;
}
__device__ __forceinline__ uint8_t norm_quant1(float v, float s)
{
    float f[8] = {v, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    return (uint8_t)norm_quant8(f, s).x;
}

// 8 elements at element offset `e`, raw: 16 bytes of bf16 or 32 of fp32.
struct Raw8 { uint4 a, b; };
__device__ __forceinline__ Raw8 norm_load8(const void* base, int is32, int64_t e)
{
    Raw8 r;
    if (is32) {
        const uint4* p = reinterpret_cast<const uint4*>(static_cast<const float*>(base) + e);
        r.a = __ldcs(p);
        r.b = __ldcs(p + 1);
    } else {
        r.a = __ldcs(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(base) + e));
    }
    return r;
}
__device__ __forceinline__ void norm_unpack8(const Raw8& r, int is32, float (&f)[8])
{
    if (is32) {
        f[0] = __uint_as_float(r.a.x); f[1] = __uint_as_float(r.a.y); f[2] = __uint_as_float(r.a.z); f[3] = __uint_as_float(r.a.w);
        f[4] = __uint_as_float(r.b.x); f[5] = __uint_as_float(r.b.y); f[6] = __uint_as_float(r.b.z); f[7] = __uint_as_float(r.b.w);
    } else {
        f[0] = bf16lo(r.a.x); f[1] = bf16hi(r.a.x); f[2] = bf16lo(r.a.y); f[3] = bf16hi(r.a.y);
        f[4] = bf16lo(r.a.z); f[5] = bf16hi(r.a.z); f[6] = bf16lo(r.a.w); f[7] = bf16hi(r.a.w);
    }
}
__device__ __forceinline__ void norm_store8(void* base, int is32, int64_t e, const float (&f)[8])
{
    if (is32) {
        float4* p = reinterpret_cast<float4*>(static_cast<float*>(base) + e);
        p[0] = make_float4(f[0], f[1], f[2], f[3]);
        p[1] = make_float4(f[4], f[5], f[6], f[7]);
    } else {
        *reinterpret_cast<uint4*>(static_cast<uint16_t*>(base) + e) =
            make_uint4(cvt_bf16x2(f[0], f[1]), cvt_bf16x2(f[2], f[3]), cvt_bf16x2(f[4], f[5]), cvt_bf16x2(f[6], f[7]));
    }
}

// Reduction over the threads of a row: a warp, or all warps of the block (blockDim.y == 1 then).
template <bool MAX>
__device__ __forceinline__ float norm_reduce(float v, float* sh)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const float u = __shfl_xor_sync(0xffffffffu, v, o);
        v = MAX ? max_nan(v, u) : v + u;
    }
    if (blockDim.x == 32) return v;
    const int warps = blockDim.x >> 5;
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
    __syncthreads();
    v = (int)(threadIdx.x & 31) < warps ? sh[threadIdx.x & 31] : 0.f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const float u = __shfl_xor_sync(0xffffffffu, v, o);
        v = MAX ? max_nan(v, u) : v + u;
    }
    return v;
}

// 1 / sqrt(mean + eps) of a row whose squares sum to `ss`.  Where fp32 squares overflow, or vanish beside an
// eps that is as small, `again(k)` sums the squares of k h once more with k a power of two that brings them into
// range (the same branch for every thread of a row).
template <typename F>
__device__ __forceinline__ float norm_factor(float ss, const NormParams& p, F again)
{
    const float v = ss / (float)p.width + p.eps;
    if (v >= 0x1p-100f && ss <= 3.402823466e+38f) return rsqrtf(v);
    if (isnan(ss)) return ss;
    const float k = v < 1.f ? 0x1p70f : 0x1p-70f;
    return rsqrtf(again(k) / (float)p.width + p.eps * k * k) * k;
}

template <int NV>
__global__ void __launch_bounds__(1024) norm_vec_kernel(const NormParams p)
{
    __shared__ float sh_sum[32], sh_max[32];
    pdl_wait_then_release();
    const int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    if (row >= p.rows) return;              // (a whole warp: blockDim.y > 1 only with one warp per row)
    const int tx = threadIdx.x, tpr = blockDim.x, n_vec = p.width >> 3;
    Raw8 rx[NV], rr[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int v = i * tpr + tx;
        if (v < n_vec) {
            rx[i] = norm_load8(p.x, p.x32, row * p.x_stride + v * 8);
            if (p.r) rr[i] = norm_load8(p.r, p.r32, row * p.width + v * 8);
        }
    }
    float f[NV][8];
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int v = i * tpr + tx;
        if (v >= n_vec) {
#pragma unroll
            for (int j = 0; j < 8; ++j) f[i][j] = 0.f;
            continue;
        }
        norm_unpack8(rx[i], p.x32, f[i]);
        if (p.r) {
            float g[8];
            norm_unpack8(rr[i], p.r32, g);
#pragma unroll
            for (int j = 0; j < 8; ++j) f[i][j] += g[j];
        }
        if (p.h) norm_store8(p.h, p.r32, row * p.width + v * 8, f[i]);
#pragma unroll
        for (int j = 0; j < 8; ++j) ss = fmaf(f[i][j], f[i][j], ss);
    }
    ss = norm_reduce<false>(ss, sh_sum);
    const float rs = norm_factor(ss, p, [&](float k) {
        float s2 = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) s2 = fmaf(f[i][j] * k, f[i][j] * k, s2);
        if (blockDim.x > 32) __syncthreads();
        return norm_reduce<false>(s2, sh_sum);
    });
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int v = i * tpr + tx;
        float w[8];
        if (v < n_vec) {
            norm_unpack8(norm_load8(p.w, p.w32, v * 8), p.w32, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) f[i][j] = f[i][j] * rs * w[j];
        }
        if (p.out < 2) {
            if (v < n_vec) norm_store8(p.y, p.out, row * p.width + v * 8, f[i]);
            continue;
        }
        float m = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) m = max_nan(m, fabsf(f[i][j]));
        if (p.group) {
            // 16 lanes hold 128 columns
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
            const float s = m / kE4m3Max;
            if (v < n_vec) {
                if ((tx & 15) == 0) p.scale[row * p.n_groups + (v >> 4)] = s;
                *reinterpret_cast<uint2*>(static_cast<uint8_t*>(p.y) + row * p.width + v * 8) = norm_quant8(f[i], s);
            }
        } else {
            top = max_nan(top, m);
        }
    }
    if (p.out == 2 && !p.group) {
        top = norm_reduce<true>(top, sh_max);
        const float s = top / kE4m3Max;
        if (tx == 0) p.scale[row] = s;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = i * tpr + tx;
            if (v >= n_vec) continue;
            *reinterpret_cast<uint2*>(static_cast<uint8_t*>(p.y) + row * p.width + v * 8) = norm_quant8(f[i], s);
        }
    }
}

__device__ __forceinline__ float norm_ld(const void* base, int is32, int64_t e)
{
    return is32 ? static_cast<const float*>(base)[e] : __uint_as_float((uint32_t)static_cast<const uint16_t*>(base)[e] << 16);
}
__device__ __forceinline__ void norm_st(void* base, int is32, int64_t e, float v)
{
    if (is32) static_cast<float*>(base)[e] = v;
    else static_cast<uint16_t*>(base)[e] = (uint16_t)f32_to_bf16_bits(v);
}

// Any width and alignment: one block per row, the row as fp32 in shared memory, element e with thread
// e mod threads.  With a scale per 128 columns a warp takes whole blocks of 128.
__global__ void __launch_bounds__(256) norm_any_kernel(const NormParams p)
{
    extern __shared__ float row_sh[];
    __shared__ float sh_sum[32], sh_max[32];
    pdl_wait_then_release();
    const int64_t row = blockIdx.x;
    const int tx = threadIdx.x, nt = blockDim.x;
    float ss = 0.f;
    for (int e = tx; e < p.width; e += nt) {
        float v = norm_ld(p.x, p.x32, row * p.x_stride + e);
        if (p.r) v += norm_ld(p.r, p.r32, row * p.width + e);
        if (p.h) norm_st(p.h, p.r32, row * p.width + e, v);
        row_sh[e] = v;
        ss = fmaf(v, v, ss);
    }
    ss = norm_reduce<false>(ss, sh_sum);
    const float rs = norm_factor(ss, p, [&](float k) {
        float s2 = 0.f;
        for (int e = tx; e < p.width; e += nt) s2 = fmaf(row_sh[e] * k, row_sh[e] * k, s2);
        __syncthreads();
        return norm_reduce<false>(s2, sh_sum);
    });
    float top = 0.f;
    for (int e = tx; e < p.width; e += nt) {
        const float y = row_sh[e] * rs * norm_ld(p.w, p.w32, e);
        if (p.out < 2) norm_st(p.y, p.out, row * p.width + e, y);
        else row_sh[e] = y;
        top = max_nan(top, fabsf(y));
    }
    if (p.out < 2) return;
    uint8_t* q = static_cast<uint8_t*>(p.y) + row * p.width;
    if (!p.group) {
        top = norm_reduce<true>(top, sh_max);
        const float s = top / kE4m3Max;
        if (tx == 0) p.scale[row] = s;
        for (int e = tx; e < p.width; e += nt) q[e] = norm_quant1(row_sh[e], s);
        return;
    }
    __syncthreads();
    for (int g = tx >> 5; g < p.n_groups; g += nt >> 5) {
        float m = 0.f, y[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int e = g * 128 + j * 32 + (tx & 31);
            y[j] = e < p.width ? row_sh[e] : 0.f;
            m = max_nan(m, fabsf(y[j]));
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
        const float s = m / kE4m3Max;
        if ((tx & 31) == 0) p.scale[row * p.n_groups + g] = s;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int e = g * 128 + j * 32 + (tx & 31);
            if (e < p.width) q[e] = norm_quant1(y[j], s);
        }
    }
}

}  // namespace lckv
