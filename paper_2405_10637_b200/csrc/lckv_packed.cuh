// Rows held in 4 bits: how they are laid out, written and read back.
//
// A group is 64 neighbouring dimensions of one key or one value.  With low and high its smallest and largest element,
//     step = bf16((high/16 - low/16) * fp32(16/15)),  0 where below 2^-120
//     code = rint((x/16 - low/16) * 1/(step/16)) in 0 .. 15,   the element stands for low + step * code
// (fp32; the sixteenths keep a group that spans bf16's whole range from overflowing).  A group with an infinity or a NaN
// stands for NaN: low is NaN, step 0 (steps are always finite and not negative).
//
// Three arrays per slot, indexed by the physical row:
//   kc, vc [rows][D/2] bytes   codes.  A 32-bit word holds eight neighbouring dimensions, dimension 8 w + i in bits 4 i.
//                              A key's words lie in the order in which the four lanes that share a row of an MMA tile
//                              take them (word 4 j + c at c * D/32 + j); a value's so that the words of the two groups
//                              alternate (D = 128: word w at 2 (w mod 8) + w / 8).
//   par    [rows][2 D/64]      per group step (low half) and low (high half), bf16: the key's groups, then the value's.
// Row pitch of a (sequence, head) is the capacity rounded up to 64 rows, so that every tile starts on 16 bytes and none
// leaves the slot; pages hold a multiple of 64 rows anyway.
#pragma once
#include "lckv_small_kernels.cuh"

namespace lckv {

constexpr float kPackedRatio = 1.0666667222976685f;   // fp32(16 / 15)
constexpr float kPackedMinStep = 7.523163845262640e-37f;   // 2^-120

struct PackedSlot {
    uint8_t* kc;
    uint8_t* vc;
    uint32_t* par;
};

// Physical row of row r of (sequence, kv head): slots of `pitch` rows per (sequence, head), or pages.
struct RowMap {
    const int32_t* page_table;    // null: not paged
    int64_t pitch;
    int32_t H_kv, pt_stride, page_shift;
    __device__ __forceinline__ int64_t at(int b, int h, int r) const      // negative: no page
    {
        if (page_table) {
            const int64_t id = page_table[(int64_t)b * pt_stride + (r >> page_shift)];
            return id < 0 ? -1 : ((id * H_kv + h) << page_shift) + (r & ((1 << page_shift) - 1));
        }
        return ((int64_t)b * H_kv + h) * pitch + r;
    }
};

__device__ __forceinline__ uint32_t max2_nan(uint32_t a, uint32_t b)
{
    uint32_t d;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t min2_nan(uint32_t a, uint32_t b)
{
    uint32_t d;
    asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}

// Position of word w (dimensions 8 w .. 8 w + 7) in a row's codes.
template <int D>
__device__ __forceinline__ int packed_k_word(int w) { return (w & 3) * (D / 32) + (w >> 2); }
template <int D>
__device__ __forceinline__ int packed_v_word(int w) { return D == 128 ? 2 * (w & 7) + (w >> 3) : w; }

// Eight lanes (a multiple of eight and the seven behind it) hold a group, eight elements each: their codes and the group's
// parameters (the same in all eight).
__device__ __forceinline__ void packed_encode(uint4 x, uint32_t& word, uint32_t& par)
{
    uint32_t mx = max2_nan(max2_nan(x.x, x.y), max2_nan(x.z, x.w));
    uint32_t mn = min2_nan(min2_nan(x.x, x.y), min2_nan(x.z, x.w));
    mx = max2_nan(mx, (mx >> 16) | (mx << 16));
    mn = min2_nan(mn, (mn >> 16) | (mn << 16));
    // largest in the low half, smallest in the high half: one exchange serves both
#pragma unroll
    for (int off = 1; off <= 4; off <<= 1) {
        const uint32_t o = __shfl_xor_sync(0xffffffffu, (mx & 0xffffu) | (mn & 0xffff0000u), off);
        mx = max2_nan(mx, o);
        mn = min2_nan(mn, o);
    }
    const float high = bf16lo(mx), low = bf16hi(mn);
    const float low16 = low * 0.0625f;
    uint32_t step_bits = f32_to_bf16_bits(__fmul_rn(__fmaf_rn(high, 0.0625f, -low16), kPackedRatio));
    float step = __uint_as_float(step_bits << 16);
    if (step < kPackedMinStep) { step = 0.f; step_bits = 0; }
    const bool finite = fabsf(high) < INFINITY && fabsf(low) < INFINITY;    // (false for a NaN)
    const float inv = step > 0.f && finite ? __frcp_rn(step * 0.0625f) : 0.f;
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    word = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float v = (i & 1) ? bf16hi(w[i >> 1]) : bf16lo(w[i >> 1]);
        const float t = fminf(__fmul_rn(__fmaf_rn(v, 0.0625f, -low16), inv), 15.f);
        // adding 1.5 * 2^23 rounds to a whole number, ties to even, and leaves it in the low bits
        word |= (__float_as_uint(__fadd_rn(t, 12582912.f)) & 15u) << (4 * i);
    }
    par = step_bits | (mn & 0xffff0000u);
    if (!finite) { word = 0; par = 0x7fc00000u; }
}

// Element i of a word: low + step * code.
__device__ __forceinline__ float packed_value(uint32_t word, int i, float step, float low)
{
    return __fmaf_rn(step, (float)((word >> (4 * i)) & 15u), low);
}

struct PackedWriteParams {
    PackedSlot s;
    RowMap map;
    const uint16_t* k;        // [batch, n, H_kv, D] (append: n = 1)
    const uint16_t* v;
    const int32_t* lens;
    int64_t T_cap;
    int32_t batch, n, n_sink;
    int32_t prompt;           // 1: token i < len goes to row i; 0: one token, to row len (ring position with n_sink)
};

// A token's key and value of one head take D/8 lanes each, side by side: one warp holds one such row of D = 128 or two of
// D = 64, and a row's parameters leave in one store of neighbouring words.
template <int D>
__global__ void __launch_bounds__(256) packed_write_kernel(const PackedWriteParams p)
{
    constexpr int LANES = D / 4;                 // lanes of a row: D/8 for the key, D/8 for the value
    pdl_wait_then_release();
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t item = i / LANES;
    const int l = (int)(i % LANES);
    const int64_t n_items = (int64_t)p.batch * p.n * p.map.H_kv;
    const bool there = item < n_items;
    const int64_t it = there ? item : n_items - 1;
    const int h = (int)(it % p.map.H_kv);
    const int64_t tok = it / p.map.H_kv;
    const int b = (int)(tok / p.n);
    const int is_v = l >= D / 8, w = l % (D / 8);
    int64_t row;
    bool ok = there;
    if (p.prompt) {
        row = tok % p.n;
        ok = ok && row < p.lens[b] && row < p.T_cap;
    } else {
        row = p.lens[b];
        if (p.n_sink > 0 && row >= p.T_cap) row = p.n_sink + (row - p.n_sink) % (p.T_cap - p.n_sink);
        ok = ok && row >= 0 && row < p.T_cap;
    }
    const int64_t at = ok ? p.map.at(b, h, (int)row) : -1;
    ok = at >= 0;
    uint4 x = make_uint4(0, 0, 0, 0);
    if (ok) x = *reinterpret_cast<const uint4*>((is_v ? p.v : p.k) + it * D + w * 8);
    uint32_t word, par;
    packed_encode(x, word, par);                 // (all lanes: it exchanges between them)
    if (!ok) return;
    uint32_t* codes = reinterpret_cast<uint32_t*>(is_v ? p.s.vc : p.s.kc) + at * (D / 8);
    codes[is_v ? packed_v_word<D>(w) : packed_k_word<D>(w)] = word;
    if ((w & 7) == 0) p.s.par[at * (D / 32) + is_v * (D / 64) + (w >> 3)] = par;
}

struct RowReadParams {
    PackedSlot s;             // 4-bit rows, or
    const uint16_t* K;        // bf16 rows (null: 4-bit)
    const uint16_t* V;
    RowMap map;
    const int32_t* lens;
    void* k;                  // [batch, n, H_kv, D] bf16 or fp32
    void* v;
    int64_t T_cap;
    int32_t batch, n, f32;
};

// Rows 0 .. len-1 of a slot as tokens; the same lanes per row as packed_write_kernel.
template <int D>
__global__ void __launch_bounds__(256) row_read_kernel(const RowReadParams p)
{
    constexpr int LANES = D / 4;
    pdl_wait_then_release();
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t item = i / LANES;
    if (item >= (int64_t)p.batch * p.n * p.map.H_kv) return;
    const int l = (int)(i % LANES), is_v = l >= D / 8, w = l % (D / 8);
    const int h = (int)(item % p.map.H_kv);
    const int64_t tok = item / p.map.H_kv;
    const int b = (int)(tok / p.n), row = (int)(tok % p.n);
    if (row >= p.lens[b] || row >= p.T_cap) return;
    const int64_t at = p.map.at(b, h, row);
    if (at < 0) return;
    const int64_t dst = item * D + w * 8;
    float y[8];
    if (p.K) {
        const uint4 x = *reinterpret_cast<const uint4*>((is_v ? p.V : p.K) + at * D + w * 8);
        if (!p.f32) {
            *reinterpret_cast<uint4*>(static_cast<uint16_t*>(is_v ? p.v : p.k) + dst) = x;
            return;
        }
        const uint32_t u[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = (e & 1) ? bf16hi(u[e >> 1]) : bf16lo(u[e >> 1]);
    } else {
        const uint32_t word = reinterpret_cast<const uint32_t*>(is_v ? p.s.vc : p.s.kc)[at * (D / 8) + (is_v ? packed_v_word<D>(w) : packed_k_word<D>(w))];
        const uint32_t par = p.s.par[at * (D / 32) + is_v * (D / 64) + (w >> 3)];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = packed_value(word, e, bf16lo(par), bf16hi(par));
    }
    if (p.f32) {
        float4* o = reinterpret_cast<float4*>(static_cast<float*>(is_v ? p.v : p.k) + dst);
        o[0] = make_float4(y[0], y[1], y[2], y[3]);
        o[1] = make_float4(y[4], y[5], y[6], y[7]);
    } else {
        *reinterpret_cast<uint4*>(static_cast<uint16_t*>(is_v ? p.v : p.k) + dst) =
            make_uint4(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7]));
    }
}

}  // namespace lckv
