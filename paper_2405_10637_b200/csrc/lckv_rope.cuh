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
// heads (kRopeUnits).  Where the rotated size is not a multiple of 16, a thread takes 8 consecutive elements: an
// interleaved pair lies within them, the other half of a pair in the half layout comes through the warp's corner of
// shared memory, and the thread serves more heads, since its factors are 16 separate loads (kRopeAnySize).
// Tensors off the 16-byte grid go pair by pair (kRopePairs).
//
// A launch may begin before the kernel in front of it has ended, and any operand may come from that one.  So what is read
// after griddepcontrol.wait is read with ordinary loads: __ldg promises that the data do not change while the kernel
// runs, and may be moved in front of the wait.  (The same holds for the norm and the products, whose packed weights alone
// are complete before.)
#pragma once
#include "lckv_attn_mma.cuh"      // cvt_bf16x2

namespace lckv {

constexpr int kRopeThreads = 256;
constexpr int kRopeMostThreads = 384;  // of a block that holds several tokens
enum RopePath { kRopeUnits, kRopeAnySize, kRopePairs };
constexpr int kRopeMaxPairs = 64;      // rot_dim <= 128 = the largest head
constexpr int kStatusCapacity = 2;     // a token of a replayed append had no place in the cache or no position in the tables

struct RopeArgs {
    const float* cos;                  // [positions, half]
    const float* sin;
    int32_t positions, half;           // half = rot_dim / 2
    int32_t interleaved;
    float sgn;                         // +1, or -1 for the transposed rotation
};

struct RopeGrid {
    uint32_t per, inv, tb;
    int32_t hg, units_shift;
};

struct RopeApplyParams {
    RopeArgs r;
    RopeGrid g;
    const int32_t* pos;
    const void* x;
    void* y;
    int64_t x_tok, x_head, y_tok, y_head;   // element strides
    int32_t tokens, heads, d;
    int32_t hp;                        // heads per thread: a multiple of the kernel's HP
};

struct RopeAppendParams {
    RopeArgs r;
    RopeGrid g;
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
    int32_t hp;                        // heads per thread: a multiple of the kernel's HP
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
    __device__ __forceinline__ void zero() { w = make_uint4(0, 0, 0, 0); }
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
    __device__ __forceinline__ void set_until(const float (&f)[8], int n)      // elements 0 .. n-1, n even
    {
        if (n > 0) w.x = cvt_bf16x2(f[0], f[1]);
        if (n > 2) w.y = cvt_bf16x2(f[2], f[3]);
        if (n > 4) w.z = cvt_bf16x2(f[4], f[5]);
        if (n > 6) w.w = cvt_bf16x2(f[6], f[7]);
    }
};
template <> struct Vec8<float> {
    float4 a, b;
    __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
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
    __device__ __forceinline__ void set_until(const float (&f)[8], int n)
    {
        if (n > 0) { a.x = f[0]; a.y = f[1]; }
        if (n > 2) { a.z = f[2]; a.w = f[3]; }
        if (n > 4) { b.x = f[4]; b.y = f[5]; }
        if (n > 6) { b.z = f[6]; b.w = f[7]; }
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
        const float4 c0 = pc[0], c1 = pc[1], s0 = ps[0], s1 = ps[1];
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

// 8 consecutive elements 8 u .. 8 u + 7 of a head, any even rotated size: the factors of each element and of its partner,
// fetched once for all heads of the thread, and where the partner lies.  All 32 lanes of a warp take part; the lanes of
// a head are neighbours.  sh: 256 floats of the warp's own, element i of lane l at [i][l].
struct RopeAny {
    float c[8], s[8];                   // y = x c + partner s
    int from[8];                        // the partner's place in sh (half layout)
    int n;                              // rotated elements among the 8: 0 .. 8, even
    __device__ __forceinline__ void fetch(const RopeArgs& r, int u, int pos)
    {
        const int first = (threadIdx.x & 31) - u, rot = 2 * r.half;
        pos = pos < 0 ? 0 : (pos < r.positions ? pos : r.positions - 1);
        const float* pc = r.cos + (int64_t)pos * r.half;
        const float* ps = r.sin + (int64_t)pos * r.half;
        n = rot - u * 8;
        n = n < 0 ? 0 : n > 8 ? 8 : n;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int e = u * 8 + i;
            const bool low = r.interleaved ? (i & 1) == 0 : e < r.half;
            const int j = r.interleaved ? e >> 1 : low ? e : e - r.half, o = low ? e + r.half : j;
            c[i] = s[i] = 0.f;
            from[i] = 0;
            if (i < n) {
                c[i] = pc[j];
                s[i] = (low ? -r.sgn : r.sgn) * ps[j];
                from[i] = (o & 7) * 32 + first + (o >> 3);
            }
        }
    }
    template <typename T>
    __device__ __forceinline__ void rotate(const RopeArgs& r, Vec8<T>& v, bool turn, float* sh) const
    {
        float x[8], y[8];
        v.get(x);
        if (r.interleaved) {
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = fmaf(x[i ^ 1], s[i], x[i] * c[i]);
        } else {
            const int lane = threadIdx.x & 31;
#pragma unroll
            for (int i = 0; i < 8; ++i) sh[i * 32 + lane] = x[i];
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = fmaf(sh[from[i]], s[i], x[i] * c[i]);
            __syncwarp();
        }
        if (turn) v.set_until(y, n);    // dimensions behind the rotated ones keep their bits
    }
};

// One pair (or two copied elements) of a head, for kRopePairs.
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
    const float c = r.cos[(int64_t)pos * r.half + u], s = r.sgn * r.sin[(int64_t)pos * r.half + u];
    const float a = rope_ld(src + e0), b = rope_ld(src + e1);
    rope_st(dst + e0, fmaf(-b, s, a * c));
    rope_st(dst + e1, fmaf(a, s, b * c));
}

__host__ __device__ constexpr int rope_units(int path, int d) { return path == kRopeUnits ? d / 16 : path == kRopeAnySize ? d / 8 : d / 2; }

// The thread's place: token `t`, unit `u`, first head `h0` (further heads at steps of `hg`).  A block holds `tb` tokens
// of per = units * head groups threads, or a 256-thread part (grid.y) of one token (tb = 0).  The host does the divisions
// (a one-token launch took 0.15 us longer with them here): `inv` = ceil(2^20 / per), with which thread * inv / 2^20 is
// thread / per for all threads below 384.
struct RopePlace { int t, u, h0; bool ok; };
__device__ __forceinline__ RopePlace rope_place(const RopeGrid& g, int tokens)
{
    RopePlace w;
    uint32_t r;
    if (g.tb == 0) {
        r = blockIdx.y * kRopeThreads + threadIdx.x;
        w.t = blockIdx.x;
        w.ok = r < g.per;
    } else {
        const uint32_t tl = (threadIdx.x * g.inv) >> 20;
        r = threadIdx.x - tl * g.per;
        const int64_t t = (int64_t)blockIdx.x * g.tb + tl;
        w.ok = tl < g.tb && t < tokens;
        w.t = (int)t;
    }
    w.h0 = (int)(r >> g.units_shift);
    w.u = (int)(r - ((uint32_t)w.h0 << g.units_shift));
    return w;
}

template <typename T, int PATH, int HP>
__global__ void __launch_bounds__(PATH == kRopeAnySize ? kRopeThreads : kRopeMostThreads) rope_apply_kernel(const RopeApplyParams p)
{
    __shared__ float sh[PATH == kRopeAnySize ? kRopeThreads * 8 : 1];
    pdl_wait_then_release();
    const RopePlace w = rope_place(p.g, p.tokens);
    if (PATH != kRopeAnySize && !w.ok) return;
    const int t = w.ok ? w.t : 0;
    const T* x = static_cast<const T*>(p.x) + (int64_t)t * p.x_tok;
    T* y = static_cast<T*>(p.y) + (int64_t)t * p.y_tok;
    const int pos = p.pos[t];
    if constexpr (PATH == kRopeAnySize) {
        RopeAny any;
        any.fetch(p.r, w.u, pos);
        for (int j0 = 0; j0 < p.hp; j0 += HP) {
            Vec8<T> v[HP];
#pragma unroll
            for (int j = 0; j < HP; ++j) {
                const int h = w.h0 + (j0 + j) * p.g.hg;
                if (w.ok && h < p.heads) v[j].load(x + (int64_t)h * p.x_head + w.u * 8);
                else v[j].zero();
            }
#pragma unroll
            for (int j = 0; j < HP; ++j) {
                const int h = w.h0 + (j0 + j) * p.g.hg;
                const bool in = w.ok && h < p.heads;
                any.rotate(p.r, v[j], in, sh + (threadIdx.x >> 5) * 256);
                if (in) v[j].store(y + (int64_t)h * p.y_head + w.u * 8);
            }
        }
    } else if constexpr (PATH == kRopePairs) {
#pragma unroll
        for (int j = 0; j < HP; ++j) {
            const int h = w.h0 + j * p.g.hg;
            if (h < p.heads) rope_pair(p.r, w.u, pos, x + (int64_t)h * p.x_head, y + (int64_t)h * p.y_head, true);
        }
    } else {
        RopeUnit un;
        un.init(p.r, w.u);
        Vec8<T> lo[HP], hi[HP];
#pragma unroll
        for (int j = 0; j < HP; ++j) {
            const int h = w.h0 + j * p.g.hg;
            if (h >= p.heads) break;
            lo[j].load(x + (int64_t)h * p.x_head + un.e0);
            hi[j].load(x + (int64_t)h * p.x_head + un.e1);
        }
        un.fetch(p.r, w.u, pos);
#pragma unroll
        for (int j = 0; j < HP; ++j) {
            const int h = w.h0 + j * p.g.hg;
            if (h >= p.heads) break;
            if (un.turn) un.rotate(p.r, lo[j], hi[j]);
            lo[j].store(y + (int64_t)h * p.y_head + un.e0);
            hi[j].store(y + (int64_t)h * p.y_head + un.e1);
        }
    }
}

// Heads 0 .. hq-1 of a token are its query heads (rotated, to q_out), the next hkv its keys (rotated, to
// the row), the last hkv its values (copied to the row).
template <int PATH, int HP>
__global__ void __launch_bounds__(PATH == kRopeAnySize ? kRopeThreads : kRopeMostThreads, PATH == kRopeAnySize ? 3 : 1) rope_append_kernel(const RopeAppendParams p)
{
    __shared__ float sh[PATH == kRopeAnySize ? kRopeThreads * 8 : 1];
    pdl_wait_then_release();
    const int heads = p.hq + 2 * p.hkv;
    RopePlace w = rope_place(p.g, p.batch * p.n_new);
    if (PATH != kRopeAnySize && !w.ok) return;
    if (!w.ok) w.t = 0;
    const int b = p.n_new == 1 ? w.t : w.t / p.n_new, i = w.t - b * p.n_new;
    const int len = p.lens[b];
    if (p.prompt && i >= len) {
        if (PATH != kRopeAnySize) return;
        w.ok = false;
    }
    const int pos = p.prompt ? i : (int)((uint32_t)len + (uint32_t)i);
    // the row: ring position in a sink + recent-window cache, page look-up in a paged one
    int64_t row = pos;
    if (p.n_sink > 0 && row >= p.T_cap) row = p.n_sink + (row - p.n_sink) % (p.T_cap - p.n_sink);
    bool place = row >= 0 && row < p.T_cap;
    int64_t row0 = 0, head_step = p.T_cap;        // row of head 0, rows between heads
    if (p.page_table) {
        const int id = place ? p.page_table[(int64_t)b * p.pt_stride + (row >> p.page_shift)] : -1;
        place = place && id >= 0;
        head_step = (int64_t)1 << p.page_shift;
        row0 = (((int64_t)id * p.hkv) << p.page_shift) + (row & (head_step - 1));
    } else {
        row0 = (int64_t)b * p.hkv * p.T_cap + row;
    }
    // The host refuses calls without a position in the tables or without a row; a graph that replays one finds the lengths on
    // the device.  A token without a position is left out whole, one without a row loses its key and value.  (Looked at here:
    // in front of the row the test took 4 registers more, one thread block less fitted on an SM, and 8 prompts of up to 4096
    // tokens of 96 heads of 128 took 292 us for 208.)
    const bool known = (uint32_t)pos < (uint32_t)p.r.positions;
    if (!(known && (place || p.hkv == 0)) && w.ok && w.h0 == 0 && w.u == 0) atomicExch(p.status, kStatusCapacity);
    if (!known) {
        if (PATH != kRopeAnySize) return;
        w.ok = false;
    }
    // where head h of the token is read and written, and whether it is rotated; false: nowhere
    auto where = [&](int h, const uint16_t*& src, uint16_t*& dst, bool& turn) {
        turn = true;
        if (!w.ok || h >= heads) return false;
        if (h < p.hq) {
            src = p.q + (int64_t)w.t * p.q_tok + (int64_t)h * p.d;
            dst = p.q_out + ((int64_t)w.t * p.hq + h) * p.d;
            return true;
        }
        if (!place) return false;
        h -= p.hq;
        turn = h < p.hkv;
        if (!turn) h -= p.hkv;
        src = (turn ? p.k : p.v) + (int64_t)w.t * p.kv_tok + (int64_t)h * p.d;
        dst = (turn ? p.K : p.V) + (row0 + h * head_step) * p.d;
        return true;
    };
    const uint16_t* src[HP];
    uint16_t* dst[HP];
    bool turn[HP], in[HP];
    if constexpr (PATH == kRopePairs) {
#pragma unroll
        for (int j = 0; j < HP; ++j)
            if (where(w.h0 + j * p.g.hg, src[j], dst[j], turn[j])) rope_pair(p.r, w.u, pos, src[j], dst[j], turn[j]);
    } else if constexpr (PATH == kRopeAnySize) {
        RopeAny any;
        any.fetch(p.r, w.u, pos);
        for (int j0 = 0; j0 < p.hp; j0 += HP) {
            Vec8<uint16_t> v[HP];
#pragma unroll
            for (int j = 0; j < HP; ++j) {
                in[j] = where(w.h0 + (j0 + j) * p.g.hg, src[j], dst[j], turn[j]);
                if (in[j]) v[j].load(src[j] + w.u * 8);
                else v[j].zero();
            }
#pragma unroll
            for (int j = 0; j < HP; ++j) {
                any.rotate(p.r, v[j], in[j] && turn[j], sh + (threadIdx.x >> 5) * 256);
                if (in[j]) v[j].store(dst[j] + w.u * 8);
            }
        }
    } else {
        RopeUnit un;
        un.init(p.r, w.u);
        Vec8<uint16_t> lo[HP], hi[HP];
#pragma unroll
        for (int j = 0; j < HP; ++j)
            if (!where(w.h0 + j * p.g.hg, src[j], dst[j], turn[j])) src[j] = nullptr;
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

// The lengths after an append of several tokens (of one: advance_kernel).
__global__ void advance_by_kernel(int32_t* __restrict__ lens, int B, int by)
{
    const int b = blockIdx.x * blockDim.x + threadIdx.x;
    if (b < B) lens[b] += by;
}

// cos and sin of p * theta_j for p < positions.  `turns` holds theta_j / (2 pi) modulo 1 in units of 2^-64: the angle of
// position p is p * turns modulo 2^64, exact in integers, so far positions lose nothing.  Its upper 32 bits are split into a
// quarter turn and a rest of at most an eighth, for which the Taylor series of sin (to x^9) and cos (to x^10) are off by
// less than 2e-9.  The rest is rounded to fp32 and the series are summed in fp32, so that sine and cosine are off by at most 1e-7
// where fp32's own rounding is 3e-8, and the amplitude is an fp32 number (6e-8): with fp64 and one rounding the kernel took 2.5
// times as long (below), and the rotations that read the tables round to bf16's 4e-3 or fp32's 6e-8 of their result.  V neighbouring
// pairs and P positions per thread.
//
// 67 MB of tables for 131072 positions of 64 pairs: 10.4 us of stores.  Reducing the angle in fp64 and calling the
// library's sincospif took 34.6 us (fp64 rounding and conversions run at a sixteenth of the rate).
struct RopeTableParams {
    uint64_t turns[kRopeMaxPairs];
    float* cos;
    float* sin;
    int64_t n;                         // positions * half
    int64_t step;                      // items between a thread's positions: a multiple of half / V
    int32_t half;
    float amplitude;
};

__device__ __forceinline__ void rope_sincos(uint32_t turn, float& s, float& c)
{
    const uint32_t q = (turn + 0x20000000u) >> 30;
    const float x = (float)(int32_t)(turn - (q << 30)) * 1.4629180792671596e-9f;        // 2 pi / 2^32
    const float x2 = x * x;
    float ps = fmaf(x2, 2.7557319e-6f, -1.9841270e-4f);                                 // 1/9!, -1/7!
    ps = fmaf(ps, x2, 8.3333333e-3f);
    ps = fmaf(ps, x2, -1.6666667e-1f);
    ps = fmaf(ps * x2, x, x);
    float pc = fmaf(x2, -2.7557319e-7f, 2.4801587e-5f);                                 // -1/10!, 1/8!
    pc = fmaf(pc, x2, -1.3888889e-3f);
    pc = fmaf(pc, x2, 4.1666667e-2f);
    pc = fmaf(pc, x2, -0.5f);
    pc = fmaf(pc, x2, 1.0f);
    s = q & 1 ? pc : ps;
    c = q & 1 ? ps : pc;
    s = __uint_as_float(__float_as_uint(s) ^ ((q & 2) << 30));
    c = __uint_as_float(__float_as_uint(c) ^ (((q + 1) & 2) << 30));
}

template <int V, int P>
__global__ void __launch_bounds__(kRopeThreads) rope_table_kernel(const __grid_constant__ RopeTableParams p)
{
    pdl_wait_then_release();
    const uint32_t per = (uint32_t)(p.half / V);
    int64_t i = (int64_t)blockIdx.x * kRopeThreads + threadIdx.x;
    if (i >= p.step) return;
    uint32_t pos = (uint32_t)(i / per);
    const uint32_t j0 = (uint32_t)(i - (int64_t)pos * per) * V, stride = (uint32_t)(p.step / per);
    uint32_t hi[V], lo[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        hi[j] = (uint32_t)(p.turns[j0 + j] >> 32);
        lo[j] = (uint32_t)p.turns[j0 + j];
    }
#pragma unroll
    for (int k = 0; k < P; ++k, i += p.step, pos += stride) {
        if (i * V >= p.n) return;
        float c[V], s[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            rope_sincos(pos * hi[j] + __umulhi(pos, lo[j]), s[j], c[j]);
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
}

}  // namespace lckv
