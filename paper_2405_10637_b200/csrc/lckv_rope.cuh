// Rotary positions: the cos / sin tables, the rotation of a tensor, and the rotation of new queries
// and keys on their way into q_out and into the rows of a cache slot (with the values' copy).
//
//   pair j of a head, position p, angle a = p * theta_j:
//     y0 = x0 cos a - x1 sin a,   y1 = x1 cos a + x0 sin a      (fp32, one rounding to the output type)
//   half layout:        x0 = x[j],  x1 = x[j + rot/2]           (j < rot/2)
//   interleaved layout: x0 = x[2j], x1 = x[2j + 1]
//   dimensions rot .. d-1 of a head are copied.
//
// Three operations on 4 bytes of data: bound by memory for many tokens and by the launch for few.  A
// thread owns one unit of 16 elements of a head - two 16-byte vectors that hold 8 whole pairs, [8u, 8u+8)
// and [rot/2 + 8u, ...) in the half layout, [16u, 16u+16) in the interleaved one - for HP heads of one
// token, so that the 8 cos and 8 sin of the unit are fetched once for HP heads and HP * 32 bytes of
// loads are in flight per thread.  Neighbouring threads hold neighbouring units, then neighbouring
// heads.  Rotary sizes that are not a multiple of 16, and tensors off the 16-byte grid, go pair by pair
// (VEC = false).
#pragma once
#include "lckv_device.cuh"

namespace lckv {

constexpr int kRopeThreads = 256;
constexpr int kRopeMaxPairs = 64;      // rot_dim <= 128 = the largest head
constexpr int kStatusCapacity = 2;     // a row of a replayed append had no place in the cache

struct RopeArgs {
    const float* cos;                  // [positions, half]
    const float* sin;
    int32_t positions, half;           // half = rot_dim / 2
    int32_t interleaved;
    float sgn;                         // +1, or -1 for the transposed rotation
};

struct RopeApplyParams {
    RopeArgs r;
    const int32_t* pos;
    const void* x;
    void* y;
    int64_t x_tok, x_head, y_tok, y_head;   // element strides
    int32_t tokens, heads, d;
};

struct RopeAppendParams {
    RopeArgs r;
    const uint16_t* q;                 // token (b, i) at (b * n_new + i) * q_tok, heads contiguous; null: none
    uint16_t* q_out;                   // contiguous
    const uint16_t* k;                 // null: none
    const uint16_t* v;
    uint16_t* K;                       // the slot
    uint16_t* V;
    const int32_t* lens;
    const int32_t* page_table;
    int32_t* status;
    int64_t q_tok, kv_tok, T_cap;
    int32_t batch, n_new, hq, hkv, d;  // hq = 0 without q, hkv = 0 without k and v
    int32_t n_sink, pt_stride, page_shift;
    int32_t prompt;                    // 0: tokens i < n_new at positions len[b] + i; 1: tokens i < len[b] at i
};

template <typename T> __device__ __forceinline__ float rope_ld(const T* p);
template <> __device__ __forceinline__ float rope_ld(const float* p) { return *p; }
template <> __device__ __forceinline__ float rope_ld(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
__device__ __forceinline__ void rope_st(float* p, float v) { *p = v; }
__device__ __forceinline__ void rope_st(uint16_t* p, float v) { *p = (uint16_t)f32_to_bf16_bits(v); }

// The raw bits of 8 elements, loaded once and stored once (cache-streaming both ways).
template <typename T> struct Vec8;
template <> struct Vec8<uint16_t> {
    uint4 w;
    __device__ __forceinline__ void load(const uint16_t* p) { w = __ldcs(reinterpret_cast<const uint4*>(p)); }
    __device__ __forceinline__ void store(uint16_t* p) const { *reinterpret_cast<uint4*>(p) = w; }
    __device__ __forceinline__ void get(float (&f)[8]) const
    {
        f[0] = bf16lo(w.x); f[1] = bf16hi(w.x); f[2] = bf16lo(w.y); f[3] = bf16hi(w.y);
        f[4] = bf16lo(w.z); f[5] = bf16hi(w.z); f[6] = bf16lo(w.w); f[7] = bf16hi(w.w);
    }
    __device__ __forceinline__ void set(const float (&f)[8])
    {
        w = make_uint4(cvt_bf16x2(f[0], f[1]), cvt_bf16x2(f[2], f[3]), cvt_bf16x2(f[4], f[5]),
                       cvt_bf16x2(f[6], f[7]));
    }
};
template <> struct Vec8<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float* p)
    {
        a = __ldcs(reinterpret_cast<const float4*>(p));
        b = __ldcs(reinterpret_cast<const float4*>(p) + 1);
    }
    __device__ __forceinline__ void store(float* p) const
    {
        *reinterpret_cast<float4*>(p) = a;
        *(reinterpret_cast<float4*>(p) + 1) = b;
    }
    __device__ __forceinline__ void get(float (&f)[8]) const
    {
        f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    }
    __device__ __forceinline__ void set(const float (&f)[8])
    {
        a = make_float4(f[0], f[1], f[2], f[3]);
        b = make_float4(f[4], f[5], f[6], f[7]);
    }
};

// Where unit u of a head lies, whether it is rotated, and its 8 cos and sin at position `pos`.
struct RopeUnit {
    int e0, e1;
    bool turn;
    float c[8], s[8];
    __device__ __forceinline__ void init(const RopeArgs& r, int u)
    {
        turn = u * 8 < r.half;
        if (turn && !r.interleaved) { e0 = u * 8; e1 = r.half + u * 8; }
        else { e0 = u * 16; e1 = u * 16 + 8; }
    }
    __device__ __forceinline__ void fetch(const RopeArgs& r, int u, int pos)
    {
        if (!turn) return;
        pos = pos < 0 ? 0 : (pos < r.positions ? pos : r.positions - 1);
        const float4* pc = reinterpret_cast<const float4*>(r.cos + (int64_t)pos * r.half + u * 8);
        const float4* ps = reinterpret_cast<const float4*>(r.sin + (int64_t)pos * r.half + u * 8);
        const float4 c0 = __ldg(pc), c1 = __ldg(pc + 1), s0 = __ldg(ps), s1 = __ldg(ps + 1);
        c[0] = c0.x; c[1] = c0.y; c[2] = c0.z; c[3] = c0.w; c[4] = c1.x; c[5] = c1.y; c[6] = c1.z; c[7] = c1.w;
        s[0] = s0.x; s[1] = s0.y; s[2] = s0.z; s[3] = s0.w; s[4] = s1.x; s[5] = s1.y; s[6] = s1.z; s[7] = s1.w;
#pragma unroll
        for (int j = 0; j < 8; ++j) s[j] *= r.sgn;
    }
    template <typename T>
    __device__ __forceinline__ void rotate(const RopeArgs& r, Vec8<T>& lo, Vec8<T>& hi) const
    {
        float a[8], b[8], x[8], y[8];
        lo.get(a);
        hi.get(b);
        if (!r.interleaved) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                x[j] = fmaf(-b[j], s[j], a[j] * c[j]);
                y[j] = fmaf(a[j], s[j], b[j] * c[j]);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x[2 * j] = fmaf(-a[2 * j + 1], s[j], a[2 * j] * c[j]);
                x[2 * j + 1] = fmaf(a[2 * j], s[j], a[2 * j + 1] * c[j]);
                y[2 * j] = fmaf(-b[2 * j + 1], s[4 + j], b[2 * j] * c[4 + j]);
                y[2 * j + 1] = fmaf(b[2 * j], s[4 + j], b[2 * j + 1] * c[4 + j]);
            }
        }
        lo.set(x);
        hi.set(y);
    }
};

// One pair (or two copied elements) of a head, for VEC = false.
template <typename T>
__device__ __forceinline__ void rope_pair(const RopeArgs& r, int u, int pos, const T* src, T* dst, bool turn_head)
{
    const bool turn = turn_head && u < r.half;
    const int e0 = turn && !r.interleaved ? u : 2 * u;
    const int e1 = turn && !r.interleaved ? u + r.half : 2 * u + 1;
    if (!turn) {
        const T a = src[e0], b = src[e1];
        dst[e0] = a;
        dst[e1] = b;
        return;
    }
    pos = pos < 0 ? 0 : (pos < r.positions ? pos : r.positions - 1);
    const float c = __ldg(r.cos + (int64_t)pos * r.half + u), s = r.sgn * __ldg(r.sin + (int64_t)pos * r.half + u);
    const float a = rope_ld(src + e0), b = rope_ld(src + e1);
    rope_st(dst + e0, fmaf(-b, s, a * c));
    rope_st(dst + e1, fmaf(a, s, b * c));
}

// The thread's place: token `t`, unit `u`, first head `h0` (further heads at steps of `hg`).  A block
// holds 256 / (units * head groups) tokens, or a 256-thread part (grid.y) of one token.
struct RopePlace { int t, u, h0, hg; bool ok; };
template <bool VEC, int HP>
__device__ __forceinline__ RopePlace rope_place(int tokens, int heads, int d)
{
    RopePlace w;
    const int units = VEC ? d >> 4 : d >> 1;
    w.hg = (heads + HP - 1) / HP;
    const uint32_t per = (uint32_t)(w.hg * units);
    uint32_t r, tl = 0;
    if (per >= (uint32_t)kRopeThreads) {
        r = blockIdx.y * kRopeThreads + threadIdx.x;
        w.t = blockIdx.x;
        w.ok = r < per;
    } else {
        const uint32_t tb = kRopeThreads / per;
        tl = threadIdx.x / per;
        r = threadIdx.x - tl * per;
        const int64_t t = (int64_t)blockIdx.x * tb + tl;
        w.ok = tl < tb && t < tokens;
        w.t = (int)t;
    }
    w.h0 = (int)(r / (uint32_t)units);
    w.u = (int)(r - (uint32_t)w.h0 * units);
    return w;
}

template <typename T, bool VEC, int HP>
__global__ void __launch_bounds__(kRopeThreads) rope_apply_kernel(const RopeApplyParams p)
{
    pdl_wait_then_release();
    const RopePlace w = rope_place<VEC, HP>(p.tokens, p.heads, p.d);
    if (!w.ok) return;
    const T* x = static_cast<const T*>(p.x) + (int64_t)w.t * p.x_tok;
    T* y = static_cast<T*>(p.y) + (int64_t)w.t * p.y_tok;
    const int pos = __ldg(p.pos + w.t);
    if constexpr (!VEC) {
#pragma unroll
        for (int j = 0; j < HP; ++j) {
            const int h = w.h0 + j * w.hg;
            if (h < p.heads) rope_pair(p.r, w.u, pos, x + (int64_t)h * p.x_head, y + (int64_t)h * p.y_head, true);
        }
    } else {
        RopeUnit un;
        un.init(p.r, w.u);
        Vec8<T> lo[HP], hi[HP];
#pragma unroll
        for (int j = 0; j < HP; ++j) {
            const int h = w.h0 + j * w.hg;
            if (h >= p.heads) break;
            lo[j].load(x + (int64_t)h * p.x_head + un.e0);
            hi[j].load(x + (int64_t)h * p.x_head + un.e1);
        }
        un.fetch(p.r, w.u, pos);
#pragma unroll
        for (int j = 0; j < HP; ++j) {
            const int h = w.h0 + j * w.hg;
            if (h >= p.heads) break;
            if (un.turn) un.rotate(p.r, lo[j], hi[j]);
            lo[j].store(y + (int64_t)h * p.y_head + un.e0);
            hi[j].store(y + (int64_t)h * p.y_head + un.e1);
        }
    }
}

// Heads 0 .. hq-1 of a token are its query heads (rotated, to q_out), the next hkv its keys (rotated, to
// the row), the last hkv its values (copied to the row).
template <bool VEC, int HP>
__global__ void __launch_bounds__(kRopeThreads) rope_append_kernel(const RopeAppendParams p)
{
    pdl_wait_then_release();
    const int heads = p.hq + 2 * p.hkv;
    const RopePlace w = rope_place<VEC, HP>(p.batch * p.n_new, heads, p.d);
    if (!w.ok) return;
    const int b = w.t / p.n_new, i = w.t - b * p.n_new;
    const int len = __ldg(p.lens + b);
    if (p.prompt && i >= len) return;
    const int pos = p.prompt ? i : len + i;
    // the row: ring position in a sink + recent-window cache, page look-up in a paged one
    int64_t row = pos;
    if (p.n_sink > 0 && row >= p.T_cap) row = p.n_sink + (row - p.n_sink) % (p.T_cap - p.n_sink);
    bool place = row >= 0 && row < p.T_cap;
    int64_t row0 = 0, head_step = p.T_cap;        // row of head 0, rows between heads
    if (p.page_table) {
        const int id = place ? __ldg(p.page_table + (int64_t)b * p.pt_stride + (row >> p.page_shift)) : -1;
        place = place && id >= 0;
        head_step = (int64_t)1 << p.page_shift;
        row0 = (((int64_t)id * p.hkv) << p.page_shift) + (row & (head_step - 1));
    } else {
        row0 = (int64_t)b * p.hkv * p.T_cap + row;
    }
    // the host refuses calls without room; a graph that replays one finds the lengths on the device
    if (!place && p.hkv > 0 && w.h0 == 0 && w.u == 0) atomicExch(p.status, kStatusCapacity);
    RopeUnit un;
    un.init(p.r, w.u);
    const uint16_t* src[HP];
    uint16_t* dst[HP];
    bool turn[HP];
#pragma unroll
    for (int j = 0; j < HP; ++j) {
        int h = w.h0 + j * w.hg;
        src[j] = nullptr;
        turn[j] = true;
        if (h < p.hq) {
            src[j] = p.q + (int64_t)w.t * p.q_tok + (int64_t)h * p.d;
            dst[j] = p.q_out + ((int64_t)w.t * p.hq + h) * p.d;
        } else if (h < heads && place) {
            h -= p.hq;
            turn[j] = h < p.hkv;
            if (!turn[j]) h -= p.hkv;
            src[j] = (turn[j] ? p.k : p.v) + (int64_t)w.t * p.kv_tok + (int64_t)h * p.d;
            dst[j] = (turn[j] ? p.K : p.V) + (row0 + h * head_step) * p.d;
        }
    }
    if constexpr (!VEC) {
#pragma unroll
        for (int j = 0; j < HP; ++j)
            if (src[j]) rope_pair(p.r, w.u, pos, src[j], dst[j], turn[j]);
    } else {
        Vec8<uint16_t> lo[HP], hi[HP];
#pragma unroll
        for (int j = 0; j < HP; ++j) {
            if (!src[j]) continue;
            lo[j].load(src[j] + un.e0);
            hi[j].load(src[j] + un.e1);
        }
        un.fetch(p.r, w.u, pos);
#pragma unroll
        for (int j = 0; j < HP; ++j) {
            if (!src[j]) continue;
            if (un.turn && turn[j]) un.rotate(p.r, lo[j], hi[j]);
            lo[j].store(dst[j] + un.e0);
            hi[j].store(dst[j] + un.e1);
        }
    }
}

// cos and sin of p * theta_j for p < positions.  `turns` holds theta_j / (2 pi): the angle in turns is
// reduced to [-1/2, 1/2] in fp64 (far positions lose nothing), the functions are then taken in fp32 of
// half turns.  V pairs per thread.
struct RopeTableParams {
    double turns[kRopeMaxPairs];
    float* cos;
    float* sin;
    int64_t n;                         // positions * half
    int32_t half;
    float amplitude;
};

template <int V>
__global__ void __launch_bounds__(kRopeThreads) rope_table_kernel(const __grid_constant__ RopeTableParams p)
{
    pdl_wait_then_release();
    const uint32_t per = (uint32_t)(p.half / V);
    const int64_t i = (int64_t)blockIdx.x * kRopeThreads + threadIdx.x;
    if (i * V >= p.n) return;
    const uint32_t pos = (uint32_t)(i / per), j0 = (uint32_t)(i - (int64_t)pos * per) * V;
    float c[V], s[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        double t = (double)pos * p.turns[j0 + j];
        t -= rint(t);
        sincospif((float)(2.0 * t), &s[j], &c[j]);
        c[j] *= p.amplitude;
        s[j] *= p.amplitude;
    }
    if constexpr (V == 4) {
        *reinterpret_cast<float4*>(p.cos + i * 4) = make_float4(c[0], c[1], c[2], c[3]);
        *reinterpret_cast<float4*>(p.sin + i * 4) = make_float4(s[0], s[1], s[2], s[3]);
    } else {
        p.cos[i] = c[0];
        p.sin[i] = s[0];
    }
}

}  // namespace lckv
