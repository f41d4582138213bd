// Rows held in 4 bits: how they are laid out, written and read back.
//
// A group is 64 neighbouring dimensions of one key or one value.  With low and high its smallest and largest element,
//     step = bf16((high/16 - low/16) * fp32(16/15)),  0 where below 2^-120
//     code = rint((x/16 - low/16) * 1/(step/16)) in 0 .. 15,   the element stands for low + step * code
// (fp32; the sixteenths keep a group that spans bf16's whole range from overflowing).  A group with an infinity or a NaN
// stands for NaN: low is NaN, step 0 (steps are always finite and not negative).
//
// A slot is a sequence of tiles of 64 physical rows, 72 D bytes each, which one bulk copy brings:
//     keys   [64][D/2] bytes      codes.  A 32-bit word holds eight neighbouring dimensions, dimension 8 w + i in bits 4 i.
//                                 A key's words lie in the order in which the four lanes that share a row of an MMA tile
//                                 take them: word 4 j + c at c * D/32 + j.
//     values [64][D/2] bytes      ..., so that the words of the two groups alternate: word w at 2 (w mod 8) + w / 8 (D = 128)
//     parameters [64][2 D/64]     per group step (low half) and low (high half), bf16: the key's groups, then the value's
// Row pitch of a (sequence, head) is the capacity rounded up to 64 rows; pages hold a multiple of 64 rows anyway.
#pragma once
#include "lckv_attn_mma.cuh"

namespace lckv {

constexpr float kPackedRatio = 1.0666667222976685f;   // fp32(16 / 15)
constexpr float kPackedMinStep = 7.523163845262640e-37f;   // 2^-120

constexpr int kPackedRows = 64;                   // rows of a tile
template <int D>
__host__ __device__ constexpr int packed_tile_bytes() { return kPackedRows * (D + D / 8); }

struct PackedSlot {
    uint8_t* base;
    template <int D>
    __device__ __forceinline__ uint8_t* tile(int64_t row) const { return base + (row >> 6) * packed_tile_bytes<D>(); }
    template <int D>
    __device__ __forceinline__ uint8_t* keys(int64_t row) const { return tile<D>(row) + (row & 63) * (D / 2); }
    template <int D>
    __device__ __forceinline__ uint8_t* values(int64_t row) const { return keys<D>(row) + kPackedRows * (D / 2); }
    template <int D>
    __device__ __forceinline__ uint32_t* par(int64_t row) const { return reinterpret_cast<uint32_t*>(tile<D>(row) + kPackedRows * D + (row & 63) * (D / 8)); }
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

// Where a lane stands in a row: D/16 lanes for the key, then as many for the value; four lanes share a group, and lane c of a
// group has its words c and c + 4 (16 elements), which lie side by side among a key's codes.
template <int D>
struct PackedLane {
    static constexpr int kLanes = D / 8;          // of a row
    int is_v, c, g;
    __device__ __forceinline__ explicit PackedLane(int l) : is_v(l >= D / 16), c(l & 3), g(D == 128 ? (l >> 2) & 1 : 0) {}
    __device__ __forceinline__ int word(int i) const { return 8 * g + c + 4 * i; }
    __device__ __forceinline__ int element(int i) const { return 8 * word(i); }
    // the lane's place in physical row `row`; the rows behind it in the same tile lie D/2 and D/8 bytes on
    struct Place { uint32_t *codes, *par; };
    __device__ __forceinline__ Place at(const PackedSlot& s, int64_t row) const
    {
        Place p;
        p.codes = is_v ? reinterpret_cast<uint32_t*>(s.values<D>(row)) + packed_v_word<D>(word(0)) : reinterpret_cast<uint32_t*>(s.keys<D>(row)) + packed_k_word<D>(word(0));
        p.par = s.par<D>(row) + is_v * (D / 64) + g;
        return p;
    }
    static constexpr int kValueStep = D == 128 ? 8 : 4;      // words from a value's word c to its word c + 4
    __device__ __forceinline__ void store(Place p, int row, uint32_t w0, uint32_t w1, uint32_t par) const
    {
        uint32_t* codes = p.codes + row * (D / 8);
        if (is_v) {
            codes[0] = w0;
            codes[kValueStep] = w1;
        } else {
            *reinterpret_cast<uint2*>(codes) = make_uint2(w0, w1);
        }
        if (c == 0) p.par[row * (D / 32)] = par;
    }
    __device__ __forceinline__ void load(Place p, int row, uint32_t& w0, uint32_t& w1, uint32_t& par) const
    {
        const uint32_t* codes = p.codes + row * (D / 8);
        if (is_v) {
            w0 = codes[0];
            w1 = codes[kValueStep];
        } else {
            const uint2 w = *reinterpret_cast<const uint2*>(codes);
            w0 = w.x;
            w1 = w.y;
        }
        par = p.par[row * (D / 32)];
    }
};

// Eight elements as a word of codes.  Adding 1.5 * 2^23 rounds to a whole number, ties to even, and leaves it in the low bits;
// the sum of those numbers' bit patterns times 16^i is the word plus a constant.  (A quotient is below 15.5 without a limit: the
// step is off by 2^-8 at most.)  Two elements an instruction; not so the last addition, which would be fused with the product in
// front of it although both say where they round.
__device__ __forceinline__ uint32_t packed_codes(uint4 x, float low16, float inv)
{
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    const uint64_t sixteenth = pack_f32x2(0.0625f, 0.0625f), minus_low = pack_f32x2(-low16, -low16), by = pack_f32x2(inv, inv);
    uint32_t word = 0u - 0x4b400000u * 0x11111111u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float lo, hi;
        unpack_f32x2(fmul2(ffma2(pack_f32x2(bf16lo(w[i]), bf16hi(w[i])), sixteenth, minus_low), by), lo, hi);
        word += __float_as_uint(__fadd_rn(lo, 12582912.f)) * (1u << (8 * i)) + __float_as_uint(__fadd_rn(hi, 12582912.f)) * (16u << (8 * i));
    }
    return word;
}

// Four lanes (a multiple of four and the three behind it) hold a group, 16 elements each: their codes and the group's
// parameters (the same in all four).
__device__ __forceinline__ void packed_encode(uint4 x, uint4 y, uint32_t& w0, uint32_t& w1, uint32_t& par)
{
    uint32_t mx = max2_nan(max2_nan(max2_nan(x.x, x.y), max2_nan(x.z, x.w)), max2_nan(max2_nan(y.x, y.y), max2_nan(y.z, y.w)));
    uint32_t mn = min2_nan(min2_nan(min2_nan(x.x, x.y), min2_nan(x.z, x.w)), min2_nan(min2_nan(y.x, y.y), min2_nan(y.z, y.w)));
    mx = max2_nan(mx, __byte_perm(mx, 0, 0x1032));
    mn = min2_nan(mn, __byte_perm(mn, 0, 0x1032));
    // largest in the low half, smallest in the high half: one exchange serves both
#pragma unroll
    for (int off = 1; off <= 2; off <<= 1) {
        const uint32_t o = __shfl_xor_sync(0xffffffffu, __byte_perm(mx, mn, 0x7610), off);
        mx = max2_nan(mx, o);
        mn = min2_nan(mn, o);
    }
    const float high = bf16lo(mx), low = bf16hi(mn);
    const float low16 = low * 0.0625f;
    uint32_t step_bits = cvt_bf16x2(__fmul_rn(__fmaf_rn(high, 0.0625f, -low16), kPackedRatio), 0.f);
    float step = __uint_as_float(step_bits << 16);
    if (step < kPackedMinStep) { step = 0.f; step_bits = 0; }
    const bool finite = fabsf(high) < INFINITY && fabsf(low) < INFINITY;    // (false for a NaN)
    const float inv = step > 0.f && finite ? __frcp_rn(step * 0.0625f) : 0.f;
    w0 = packed_codes(x, low16, inv);
    w1 = packed_codes(y, low16, inv);
    par = step_bits | (mn & 0xffff0000u);
    if (!finite) { w0 = w1 = 0; par = 0x7fc00000u; }
}

// What a word's elements stand for.  2^23 + c are fp32 numbers with c in their low bits.
__device__ __forceinline__ void packed_values(uint32_t word, uint32_t par, float (&y)[8])
{
    const uint64_t step = pack_f32x2(bf16lo(par), bf16lo(par)), low = pack_f32x2(bf16hi(par), bf16hi(par));
    const uint64_t minus = pack_f32x2(-8388608.f, -8388608.f);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w = word >> (8 * i);
        uint64_t c = pack_f32x2(__uint_as_float((w & 15u) | 0x4b000000u), __uint_as_float((w >> 4 & 15u) | 0x4b000000u));
        asm("add.rn.f32x2 %0, %1, %2;" : "=l"(c) : "l"(c), "l"(minus));
        unpack_f32x2(ffma2(step, c, low), y[2 * i], y[2 * i + 1]);
    }
}

struct PackedWriteParams {
    PackedSlot s;
    RowMap map;
    const uint16_t* k;        // [batch, n, H_kv, D] (append: n = 1)
    const uint16_t* v;
    const int32_t* lens;
    int64_t T_cap;
    int32_t batch, n, n_sink; // appended: to row len, or its place in the ring behind n_sink rows; prompts: token i < len to row i
};

// Thread blocks over rows: 256 threads, and U rows a thread whose loads are all under way before the first is used (blocks of one
// row a thread spend their time waiting for the length, then for the row: prompts of 8 x 4096 tokens of 32 heads of
// 128 took 164 us to write and 132 us to read with one, 115 and 88 with four).  Four neighbouring rows lie in one tile.
constexpr int kRowThreads = 256;
template <int D>
__host__ __device__ constexpr int rows_per_block() { return kRowThreads / PackedLane<D>::kLanes; }

// The new token of every sequence: a thread block's rows are (sequence, head)s.
template <int D>
__global__ void __launch_bounds__(kRowThreads) packed_append_kernel(const PackedWriteParams p)
{
    pdl_wait_then_release();
    const PackedLane<D> lane((int)threadIdx.x % PackedLane<D>::kLanes);
    const uint32_t H = (uint32_t)p.map.H_kv, item = blockIdx.x * rows_per_block<D>() + threadIdx.x / PackedLane<D>::kLanes;
    const uint32_t b = item / H, h = item - b * H;
    const bool in = b < (uint32_t)p.batch;
    uint4 x = make_uint4(0, 0, 0, 0), y = x;
    int64_t row = -1;
    if (in) {
        const uint16_t* src = (lane.is_v ? p.v : p.k) + (int64_t)item * D;
        x = *reinterpret_cast<const uint4*>(src + lane.element(0));
        y = *reinterpret_cast<const uint4*>(src + lane.element(1));
        row = p.lens[b];
        if (p.n_sink > 0 && row >= p.T_cap) row = p.n_sink + (row - p.n_sink) % (p.T_cap - p.n_sink);
    }
    const int64_t at = row >= 0 && row < p.T_cap ? p.map.at((int)b, (int)h, (int)row) : -1;
    uint32_t w0, w1, par;
    packed_encode(x, y, w0, w1, par);            // (all lanes: it exchanges between them)
    if (at >= 0) lane.store(lane.at(p.s, at), 0, w0, w1, par);
}

// Prompts: blockIdx.y (and on in steps of the grid) is the sequence, blockIdx.x a stretch of its (U tokens, head) items.
template <int D, int U>
__global__ void __launch_bounds__(kRowThreads) packed_write_kernel(const PackedWriteParams p)
{
    pdl_wait_then_release();
    const PackedLane<D> lane((int)threadIdx.x % PackedLane<D>::kLanes);
    const uint32_t H = (uint32_t)p.map.H_kv, item = blockIdx.x * rows_per_block<D>() + threadIdx.x / PackedLane<D>::kLanes;
    const uint32_t group = item / H, h = item - group * H;
    const int tok = (int)group * U;
    const int64_t step = (int64_t)H * D;
    for (int b = blockIdx.y; b < p.batch; b += gridDim.y) {
        const int n = (int)min((int64_t)min(p.n, p.lens[b]), p.T_cap);
        if ((int64_t)(blockIdx.x * rows_per_block<D>() / H) * U >= n) continue;      // (the whole block)
        const int64_t at = tok < n ? p.map.at(b, (int)h, tok) : -1;
        const uint16_t* src = (lane.is_v ? p.v : p.k) + (((int64_t)b * p.n + tok) * H + h) * D;
        uint4 x[U], y[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            x[u] = y[u] = make_uint4(0, 0, 0, 0);
            if (tok + u < n) {
                x[u] = *reinterpret_cast<const uint4*>(src + u * step + lane.element(0));
                y[u] = *reinterpret_cast<const uint4*>(src + u * step + lane.element(1));
            }
        }
        const auto to = lane.at(p.s, max((int64_t)0, at));
#pragma unroll
        for (int u = 0; u < U; ++u) {
            uint32_t w0, w1, par;
            packed_encode(x[u], y[u], w0, w1, par);        // (all lanes: it exchanges between them)
            if (at >= 0 && tok + u < n) lane.store(to, u, w0, w1, par);
        }
    }
}

struct RowReadParams {
    PackedSlot s;             // 4-bit rows, or
    const uint16_t* K;        // bf16 rows
    const uint16_t* V;
    RowMap map;
    const int32_t* lens;
    void* k;                  // [batch, n, H_kv, D] bf16 or fp32
    void* v;
    int64_t T_cap;
    int32_t batch, n;
};

// Rows 0 .. len-1 of a slot as tokens; lanes and blocks as in packed_write_kernel.
template <int D, bool PACKED, bool F32, int U>
__global__ void __launch_bounds__(kRowThreads) row_read_kernel(const RowReadParams p)
{
    pdl_wait_then_release();
    const PackedLane<D> lane((int)threadIdx.x % PackedLane<D>::kLanes);
    const uint32_t H = (uint32_t)p.map.H_kv, item = blockIdx.x * rows_per_block<D>() + threadIdx.x / PackedLane<D>::kLanes;
    const uint32_t group = item / H, h = item - group * H;
    const int tok = (int)group * U;
    const int64_t step = (int64_t)H * D;
    for (int b = blockIdx.y; b < p.batch; b += gridDim.y) {
        const int n = (int)min((int64_t)min(p.n, p.lens[b]), p.T_cap);
        if (tok >= n) continue;
        const int64_t at = p.map.at(b, (int)h, tok);
        if (at < 0) continue;
        uint32_t w[U][2], par[U];
        uint4 x[U][2];
        const auto from = lane.at(p.s, at);
        const uint16_t* row = (lane.is_v ? p.V : p.K) + at * D;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (tok + u >= n) break;
            if constexpr (PACKED) lane.load(from, u, w[u][0], w[u][1], par[u]);
            else
#pragma unroll
                for (int i = 0; i < 2; ++i) x[u][i] = *reinterpret_cast<const uint4*>(row + u * D + lane.element(i));
        }
        const int64_t dst0 = (((int64_t)b * p.n + tok) * H + h) * D;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (tok + u >= n) break;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int64_t dst = dst0 + u * step + lane.element(i);
                if constexpr (!PACKED && !F32) {
                    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(lane.is_v ? p.v : p.k) + dst) = x[u][i];
                } else {
                    float y[8];
                    if constexpr (PACKED) {
                        packed_values(w[u][i], par[u], y);
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const uint32_t pair = (&x[u][i].x)[e >> 1];
                            y[e] = (e & 1) ? bf16hi(pair) : bf16lo(pair);
                        }
                    }
                    if constexpr (F32) {
                        float4* o = reinterpret_cast<float4*>(static_cast<float*>(lane.is_v ? p.v : p.k) + dst);
                        o[0] = make_float4(y[0], y[1], y[2], y[3]);
                        o[1] = make_float4(y[4], y[5], y[6], y[7]);
                    } else {
                        *reinterpret_cast<uint4*>(static_cast<uint16_t*>(lane.is_v ? p.v : p.k) + dst) =
                            make_uint4(cvt_bf16x2(y[0], y[1]), cvt_bf16x2(y[2], y[3]), cvt_bf16x2(y[4], y[5]), cvt_bf16x2(y[6], y[7]));
                    }
                }
            }
        }
    }
}

}  // namespace lckv
