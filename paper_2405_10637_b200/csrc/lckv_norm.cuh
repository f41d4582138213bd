// Root-mean-square norm of rows, with the residual's addition before it and an optional 8-bit output.
//
//   h = x + r;   y = h / sqrt(mean(h^2) + eps) * w      (fp32; the mean over the row's `width` elements)
//   8 bits: scale = max|y| / 448 over a row or over 128 columns, q = e4m3(y / scale), 448 = largest e4m3
//
// h is rounded once to its own type when it is stored; the norm uses the unrounded sum.  Bound by
// memory: each element is read once and written once, so a row's elements stay in registers between the
// pass that sums squares and the one that scales.  A row is held by 8, 16 or 32 lanes, or by the warps of a thread
// block; a thread holds NV vectors of 8 consecutive elements, vector i of the row at i * threads + thread, so that
// every access is coalesced and 16 consecutive lanes hold one 128-column block.
//
// Rows whose width is not a multiple of 8 (EDGES): the vectors lie on the tensor's own 16-byte grid, and only those at
// the two ends of a row, which it shares with its neighbours, go element by element; so do the weights.
//
// Other strides and alignments, and such rows of more than 4096 vectors, go element by element, staged in shared memory as
// fp32 (norm_any_kernel).
#pragma once
#include "lckv_attn_mma.cuh"      // cvt_bf16x2

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
// The weights, which every row reads: through the L1.  (Ordinary loads: see lckv_rope.cuh.)
__device__ __forceinline__ Raw8 norm_weight8(const void* base, int is32, int64_t e)
{
    Raw8 r;
    if (is32) {
        const uint4* p = reinterpret_cast<const uint4*>(static_cast<const float*>(base) + e);
        r.a = p[0];
        r.b = p[1];
    } else {
        r.a = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(base) + e);
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

// Reduction over the threads of a row: blockDim.x lanes of a warp (8, 16 or 32), or all warps of the thread block
// (blockDim.y == 1 then).
template <bool MAX>
__device__ __forceinline__ float norm_reduce(float v, float* sh)
{
    const int lanes = blockDim.x < 32 ? blockDim.x : 32;
    for (int o = lanes >> 1; o > 0; o >>= 1) {
        const float u = __shfl_xor_sync(0xffffffffu, v, o);
        v = MAX ? max_nan(v, u) : v + u;
    }
    if (blockDim.x <= 32) return v;
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
// eps that is as small, `again(k, c)` sums the squares of k h once more with k a power of two that brings them into
// range: the largest h, 2^128, to 2^48, whose squares 32768 times are 2^111; the smallest, 2^-149, to 2^-49.  `again` holds a
// reduction, so all rows of a warp go through it together.
//
// With an eps above 0, at least 2^-149, the factor is at most 2^75 and at least 2^-128, an fp32 number (good to 2^-22 at that end).
// With an eps of 0 it can be 2^149: such calls go to the kernels with SPLIT, where a part of the factor, c, goes into h.
// (Not everywhere: the multiplications by c, never carried out, changed the compiler's registers and cost the ring kernel up to
// a quarter, 512 x 4096 of fp32 6.1 / 7.7 us.)
template <bool SPLIT, typename F>
__device__ __forceinline__ float norm_factor(float ss, const NormParams& p, F again)
{
    const float v = ss / (float)p.width + p.eps;
    const bool fine = (v >= 0x1p-100f && ss <= 3.402823466e+38f) || isnan(ss);
    float rs = isnan(ss) ? ss : rsqrtf(v);
    if (!__all_sync(0xffffffffu, fine)) {
        const bool small = v < 1.f;
        const float k = small ? 0x1p100f : 0x1p-80f, c = !SPLIT || fine ? 1.f : small ? 0x1p100f : 0x1p-4f;
        const float s2 = again(k, c);
        if (!fine) rs = rsqrtf(s2 / (float)p.width + p.eps * k * k) * (k / c);
    }
    return rs;
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

// The types of a call, read from its parameters (one kernel for all, for few rows) or fixed at compile time (one kernel
// each, for many: with the types looked up per vector a row of 4096 took 400 instructions of a warp's 16 elements per
// lane, and the kernel was bound by their issue: 16384 rows 59 us, 43 us with them fixed).
struct NormAnyTypes {
    const NormParams& p;
    __device__ __forceinline__ int x32() const { return p.x32; }
    __device__ __forceinline__ bool res() const { return p.r != nullptr; }
    __device__ __forceinline__ int r32() const { return p.r32; }
    __device__ __forceinline__ int out() const { return p.out; }
    __device__ __forceinline__ int group() const { return p.group; }
};
template <int X32, int RES, int OUT>                 // RES: 0 none, 1 bf16, 2 fp32; OUT: 0 bf16, 1 fp32, 2 e4m3 per row, 3 per 128
struct NormTypes {
    __device__ __forceinline__ NormTypes(const NormParams&) {}
    __device__ __forceinline__ static constexpr int x32() { return X32; }
    __device__ __forceinline__ static constexpr bool res() { return RES != 0; }
    __device__ __forceinline__ static constexpr int r32() { return RES == 2; }
    __device__ __forceinline__ static constexpr int out() { return OUT < 2 ? OUT : 2; }
    __device__ __forceinline__ static constexpr int group() { return OUT == 3 ? 128 : 0; }
};

// A row's place: vector v holds its elements 8 v - off .. 8 v - off + 7.
template <bool EDGES>
struct NormRow {
    int64_t row, x, e;                      // element offsets of vector 0 in x and in the dense tensors
    int off, n_vec, width;
    bool valid;
    __device__ __forceinline__ void set(const NormParams& p, int64_t r)
    {
        row = r;
        width = p.width;
        off = EDGES ? (int)((r * p.width) & 7) : 0;
        x = r * p.x_stride - off;
        e = r * p.width - off;
        check(p);
    }
    __device__ __forceinline__ void check(const NormParams& p)
    {
        valid = row < p.rows;               // (rows behind the last one share a warp with others: no early return)
        n_vec = valid ? (width + off + 7) >> 3 : 0;
    }
    // `step` rows on; xs = step * x_stride, es = step * width
    __device__ __forceinline__ void move(const NormParams& p, int64_t step, int64_t xs, int64_t es)
    {
        row += step;
        if (EDGES) {
            const int o = off;
            off = (o + (int)es) & 7;
            x += xs + o - off;
            e += es + o - off;
        } else {
            x += xs;
            e += es;
        }
        check(p);
    }
    __device__ __forceinline__ bool whole(int v) const { return !EDGES || (v * 8 >= off && v * 8 + 8 <= width + off); }
    __device__ __forceinline__ bool in(int v, int j) const { return v * 8 + j >= off && v * 8 + j < width + off; }
};

template <bool EDGES>
__device__ __forceinline__ void norm_weights(const NormParams& p, const NormRow<EDGES>& w, int v, float (&g)[8])
{
    if (EDGES) {
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] = w.in(v, j) ? norm_ld(p.w, p.w32, v * 8 + j - w.off) : 0.f;
    } else {
        norm_unpack8(norm_weight8(p.w, p.w32, v * 8), p.w32, g);
    }
}

// From h = x + r in f to the outputs of the row; `sh`: 2 x 32 floats; weight(i, g) gives the weights of the thread's i-th vector.
template <int NV, bool EDGES, bool SPLIT, typename Types, typename W>
__device__ __forceinline__ void norm_finish(const NormParams& p, const Types& t, const NormRow<EDGES>& w, float (&f)[NV][8], float* sh, W weight)
{
    const int tx = threadIdx.x, tpr = blockDim.x;
    auto part_store = [&](void* base, int is32, int v, const float (&g)[8]) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (w.in(v, j)) norm_st(base, is32, w.e + v * 8 + j, g[j]);
    };
    uint64_t s2 = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int v = i * tpr + tx;
        if (v < w.n_vec && t.res() && p.h) {
            if (w.whole(v)) norm_store8(p.h, t.r32(), w.e + v * 8, f[i]);
            else part_store(p.h, t.r32(), v, f[i]);
        }
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            const uint64_t h = pack_f32x2(f[i][j], f[i][j + 1]);
            s2 = ffma2(h, h, s2);
        }
    }
    float ss, ss_odd;
    unpack_f32x2(s2, ss, ss_odd);
    ss = norm_reduce<false>(ss + ss_odd, sh);
    const float rs = norm_factor<SPLIT>(ss, p, [&](float k, float c) {
        float s3 = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                s3 = fmaf(f[i][j] * k, f[i][j] * k, s3);
                if constexpr (SPLIT) f[i][j] *= c;
            }
        if (blockDim.x > 32) __syncthreads();
        return norm_reduce<false>(s3, sh);
    });
    const uint64_t rs2 = pack_f32x2(rs, rs);
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int v = i * tpr + tx;
        if (v < w.n_vec) {
            float g[8];
            weight(i, g);
#pragma unroll
            for (int j = 0; j < 8; j += 2)
                unpack_f32x2(fmul2(fmul2(pack_f32x2(f[i][j], f[i][j + 1]), rs2), pack_f32x2(g[j], g[j + 1])), f[i][j], f[i][j + 1]);
        }
        if (t.out() < 2) {
            if (v < w.n_vec) {
                if (w.whole(v)) norm_store8(p.y, t.out(), w.e + v * 8, f[i]);
                else part_store(p.y, t.out(), v, f[i]);
            }
            continue;
        }
        float m = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) m = max_nan(m, fabsf(f[i][j]));
        if (!EDGES && t.group()) {
            // 16 lanes hold 128 columns
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
            const float s = m / kE4m3Max;
            if (v < w.n_vec) {
                if ((tx & 15) == 0) p.scale[w.row * p.n_groups + (v >> 4)] = s;
                *reinterpret_cast<uint2*>(static_cast<uint8_t*>(p.y) + w.e + v * 8) = norm_quant8(f[i], s);
            }
        } else {
            top = max_nan(top, m);
        }
    }
    if (t.out() == 2 && (EDGES || !t.group())) {
        top = norm_reduce<true>(top, sh + 32);
        const float s = top / kE4m3Max;
        if (tx == 0 && w.valid) p.scale[w.row] = s;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = i * tpr + tx;
            if (v >= w.n_vec) continue;
            const uint2 q = norm_quant8(f[i], s);
            uint8_t* y = static_cast<uint8_t*>(p.y) + w.e + v * 8;
            if (w.whole(v)) {
                *reinterpret_cast<uint2*>(y) = q;
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (w.in(v, j)) y[j] = (uint8_t)((j < 4 ? q.x : q.y) >> (8 * (j & 3)));
            }
        }
    }
}

// One row per thread block (or 8, 16 or 32 lanes), straight from global memory: the shortest way for few rows.
template <int NV, int MAX_THREADS, bool EDGES>
__global__ void __launch_bounds__(MAX_THREADS) norm_vec_kernel(const NormParams p)
{
    __shared__ float sh[64];
    pdl_wait_then_release();
    NormRow<EDGES> w;
    w.set(p, (int64_t)blockIdx.x * blockDim.y + threadIdx.y);
    auto part_load = [&](const void* base, int is32, int64_t at, int v) {
        Raw8 r;
        uint32_t u[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            u[j] = 0;
            if (w.in(v, j)) u[j] = is32 ? static_cast<const uint32_t*>(base)[at + j] : static_cast<const uint16_t*>(base)[at + j];
        }
        if (is32) {
            r.a = make_uint4(u[0], u[1], u[2], u[3]);
            r.b = make_uint4(u[4], u[5], u[6], u[7]);
        } else {
            r.a = make_uint4(u[0] | u[1] << 16, u[2] | u[3] << 16, u[4] | u[5] << 16, u[6] | u[7] << 16);
        }
        return r;
    };
    Raw8 rx[NV], rr[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int v = i * blockDim.x + threadIdx.x;
        if (v >= w.n_vec) continue;
        if (w.whole(v)) {
            rx[i] = norm_load8(p.x, p.x32, w.x + v * 8);
            if (p.r) rr[i] = norm_load8(p.r, p.r32, w.e + v * 8);
        } else {
            rx[i] = part_load(p.x, p.x32, w.x + v * 8, v);
            if (p.r) rr[i] = part_load(p.r, p.r32, w.e + v * 8, v);
        }
    }
    float f[NV][8];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int v = i * blockDim.x + threadIdx.x;
#pragma unroll
        for (int j = 0; j < 8; ++j) f[i][j] = 0.f;
        if (v >= w.n_vec) continue;
        norm_unpack8(rx[i], p.x32, f[i]);
        if (p.r) {
            float g[8];
            norm_unpack8(rr[i], p.r32, g);
#pragma unroll
            for (int j = 0; j < 8; ++j) f[i][j] += g[j];
        }
    }
    norm_finish<NV, EDGES, true>(p, NormAnyTypes{p}, w, f, sh, [&](int i, float (&g)[8]) { norm_weights(p, w, i * blockDim.x + threadIdx.x, g); });
}

// The same for many rows: resident thread blocks walk over the rows, and each warp's vectors of the next row are
// on their way into its own places in shared memory while it works on one (asynchronous copies, no barrier but the
// warp's).  The two 16-byte pieces of an fp32 vector are copied so that the warp's lanes read 512 consecutive bytes at
// a time: with a lane's own 32 bytes in two copies each copy moved whole 32-byte sectors for 16 bytes (16384 x 4096 with
// an fp32 residual: 177 us, 140 us).  A deeper ring costs resident thread blocks and was slower (16384 x 4096 plain 43.0 /
// 45.8 us with two / three rows; with an fp32 residual to e4m3 113 / 127 us).
constexpr int kNormRing = 2;
__device__ __forceinline__ void norm_copy16(uint32_t dst, const void* src, int bytes)       // bytes < 16: the rest is 0
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
template <int NV, bool EDGES, typename Types>
__global__ void __launch_bounds__(512) norm_ring_kernel(const NormParams p)
{
    extern __shared__ __align__(16) uint8_t norm_smem[];
    __shared__ float sh[2][64];
    const Types t(p);
    constexpr int XP = Types::x32() ? 2 : 1, PARTS = XP + (Types::res() ? (Types::r32() ? 2 : 1) : 0);   // 16-byte pieces
    pdl_wait_then_release();
    const int tx = threadIdx.x, tpr = blockDim.x;
    const int threads = tpr * blockDim.y;
    const uint32_t slot_bytes = (uint32_t)(NV * PARTS * threads) * 16, smem0 = smem_u32(norm_smem);
    const int64_t step = (int64_t)gridDim.x * blockDim.y, xs = step * p.x_stride, es = step * p.width;
    const int64_t last_e = (int64_t)p.rows * p.width, last_x = (int64_t)(p.rows - 1) * p.x_stride + p.width;
    const bool wide = tpr >= 32;                     // a warp's vectors are neighbours in one row
    const uint32_t lin = threadIdx.y * tpr + tx;
    const int lane = lin & 31;                       // (a warp may hold several rows)
    // vector v = i tpr + tx of the row (of a tensor whose vector 0 is at element `at` and that has `total` elements), into
    // `part` of the slot's i-th vectors
    auto copy = [&](uint32_t dst, const void* base, bool is32, int64_t at, int64_t total, int v, int n_vec) {
        if (!is32) {
            if (v >= n_vec) return;
            const int64_t a = at + v * 8, left = EDGES ? total - a : 8;               // (the last one may reach behind the tensor)
            norm_copy16(dst + lin * 16, static_cast<const uint16_t*>(base) + a, left >= 8 ? 16 : (int)left * 2);
            return;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int c = wide ? h * 32 + lane : 2 * lane + h;                         // 16-byte piece of the warp's 64
            const int u = wide ? v - lane + (c >> 1) : v;
            if (u >= n_vec) continue;
            const int64_t a = at + u * 8 + (c & 1) * 4, left = EDGES ? total - a : 4;
            if (left <= 0) continue;
            norm_copy16(dst + ((lin & ~31u) * 2 + c) * 16, static_cast<const float*>(base) + a, left >= 4 ? 16 : (int)left * 4);
        }
    };
    auto fetch = [&](const NormRow<EDGES>& w, int slot) {
        __syncwarp();                                // the warp has read the slot
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = i * tpr + tx;
            const uint32_t dst = smem0 + slot * slot_bytes + (uint32_t)(i * PARTS * threads) * 16;
            copy(dst, p.x, t.x32(), w.x, last_x, v, w.n_vec);
            if (t.res()) copy(dst + XP * threads * 16, p.r, t.r32(), w.e, last_e, v, w.n_vec);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    auto read = [&](uint32_t src, bool is32, float (&g)[8]) {
        Raw8 r;
        if (is32) {
            r.a = lds128(src + lin * 32);
            r.b = lds128(src + lin * 32 + 16);
        } else {
            r.a = lds128(src + lin * 16);
        }
        norm_unpack8(r, is32, g);
    };
    int64_t base = (int64_t)blockIdx.x * blockDim.y;             // the same for the whole block
    NormRow<EDGES> w, ahead;
    w.set(p, base + threadIdx.y);
    ahead = w;
#pragma unroll
    for (int k = 0; k < kNormRing - 1; ++k) {
        fetch(ahead, k);
        ahead.move(p, step, xs, es);
    }
    // the weights of the thread's vectors stay in registers, where a row's vectors lie alike in every row
    float gw[EDGES ? 1 : NV][8];
    if constexpr (!EDGES) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i * tpr + tx < p.width >> 3) norm_weights(p, w, i * tpr + tx, gw[i]);
    }
    int slot = 0, odd = 0;
    for (; base < p.rows; base += step, odd ^= 1) {
        fetch(ahead, slot == 0 ? kNormRing - 1 : slot - 1);
        ahead.move(p, step, xs, es);
        asm volatile("cp.async.wait_group %0;" ::"n"(kNormRing - 1) : "memory");
        __syncwarp();
        float f[NV][8];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = i * tpr + tx;
#pragma unroll
            for (int j = 0; j < 8; ++j) f[i][j] = 0.f;
            if (v >= w.n_vec) continue;
            const uint32_t src = smem0 + slot * slot_bytes + (uint32_t)(i * PARTS * threads) * 16;
            read(src, t.x32(), f[i]);
            if (t.res()) {
                float g[8];
                read(src + XP * threads * 16, t.r32(), g);
#pragma unroll
                for (int j = 0; j < 8; ++j) f[i][j] += g[j];
            }
            if (EDGES && !w.whole(v)) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (!w.in(v, j)) f[i][j] = 0.f;
            }
        }
        slot = slot == kNormRing - 1 ? 0 : slot + 1;
        // (the other half of sh may still be read by a slower warp)
        norm_finish<NV, EDGES, false>(p, t, w, f, sh[odd], [&](int i, float (&g)[8]) {
            if constexpr (EDGES) norm_weights(p, w, i * tpr + tx, g);
            else {
#pragma unroll
                for (int j = 0; j < 8; ++j) g[j] = gw[i][j];
            }
        });
        w.move(p, step, xs, es);
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
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
    const float rs = norm_factor<true>(ss, p, [&](float k, float c) {
        float s2 = 0.f;
        for (int e = tx; e < p.width; e += nt) {       // (each thread its own elements, as above and below)
            s2 = fmaf(row_sh[e] * k, row_sh[e] * k, s2);
            row_sh[e] *= c;
        }
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
