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
    int64_t T_cap, stride;
    int32_t H_q, mode;
    float scale_log2;
};

// weights[b, h, j] = prev[b, h, j] + sum over the query heads of kv head h of exp(s_j - lse), for the visible rows j.
// One thread block per (sequence, kv head) and 256 rows, a warp per 64.  The keys go straight from memory into MMA
// fragments: the four lanes of a row take 16 bytes each, which fixes the order of the dimensions, and q follows it.
template <int D, bool PACKED>
__global__ void __launch_bounds__(kWeightWarps * 32) attention_weights_kernel(const WeightParams p)
{
    constexpr int J = D / 32, G = D / 64;
    pdl_wait_then_release();
    const uint32_t FULL = 0xffffffffu;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g4 = lane >> 2, c4 = lane & 3;
    const int b = blockIdx.x / p.map.H_kv, h = blockIdx.x % p.map.H_kv;
    const int nv = visible_rows(p.lens[b], p.mode, p.T_cap);
    const int group = p.H_q / p.map.H_kv;
    const int64_t head0 = (int64_t)b * p.H_q + (int64_t)h * group;
    const int64_t w0 = ((int64_t)b * p.map.H_kv + h) * p.stride;
    for (int64_t r64 = ((int64_t)blockIdx.y * kWeightWarps + warp) * 64; r64 < nv; r64 += (int64_t)gridDim.y * kWeightWarps * 64) {
        const int base = (int)r64, rows = min(64, nv - base);
        const int64_t at = p.map.at(b, h, base);
        float sum[4][2];
#pragma unroll
        for (int rb = 0; rb < 4; ++rb) sum[rb][0] = sum[rb][1] = 0.f;
        for (int first = 0; first < group; first += 8) {     // eight query heads at a time
            uint4 raw[J];
            const bool real = first + g4 < group;
            const uint4* q4 = reinterpret_cast<const uint4*>(p.q + (head0 + first + (real ? g4 : 0)) * D) + c4;
#pragma unroll
            for (int j = 0; j < J; ++j) raw[j] = q4[4 * j];
            const bool real0 = first + 2 * c4 < group, real1 = first + 2 * c4 + 1 < group;
            const float l0 = real0 ? p.lse[head0 + first + 2 * c4] * 1.4426950408889634f : 0.f;
            const float l1 = real1 ? p.lse[head0 + first + 2 * c4 + 1] * 1.4426950408889634f : 0.f;
            PackedQuery<D> q;
            if constexpr (PACKED) packed_query<D>(raw, p.scale_log2, lane, q);
#pragma unroll
            for (int rb = 0; rb < 4; ++rb) {
                if (rb * 16 >= rows) continue;
                const int r0 = rb * 16 + g4, r1 = r0 + 8;
                // (rows behind the last one are not read: any row's keys do in their place)
                const int64_t a0 = at < 0 ? 0 : at + min(r0, rows - 1), a1 = at < 0 ? 0 : at + min(r1, rows - 1);
                float s[4];
                if constexpr (PACKED) {
                    uint32_t ka[J], kb[J];
                    if constexpr (D == 128) {
                        const uint4 x = *reinterpret_cast<const uint4*>(p.s.kc + a0 * 64 + c4 * 16), y = *reinterpret_cast<const uint4*>(p.s.kc + a1 * 64 + c4 * 16);
                        ka[0] = x.x; ka[1] = x.y; ka[2] = x.z; ka[3] = x.w;
                        kb[0] = y.x; kb[1] = y.y; kb[2] = y.z; kb[3] = y.w;
                    } else {
                        const uint2 x = *reinterpret_cast<const uint2*>(p.s.kc + a0 * 32 + c4 * 8), y = *reinterpret_cast<const uint2*>(p.s.kc + a1 * 32 + c4 * 8);
                        ka[0] = x.x; ka[1] = x.y;
                        kb[0] = y.x; kb[1] = y.y;
                    }
                    uint32_t pa[G], pb[G];
#pragma unroll
                    for (int g = 0; g < G; ++g) {
                        pa[g] = p.s.par[a0 * (2 * G) + g];
                        pb[g] = p.s.par[a1 * (2 * G) + g];
                    }
                    float acc[G][4];
#pragma unroll
                    for (int g = 0; g < G; ++g)
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[g][i] = 0.f;
#pragma unroll
                    for (int j = 0; j < J; ++j) {
                        uint32_t xa[4], xb[4];
                        nibble_pairs(ka[j], xa);
                        nibble_pairs(kb[j], xb);
                        mma_f16_16816(acc[j / 2], xa[0], xb[0], xa[1], xb[1], q.b[2 * j][0], q.b[2 * j][1]);
                        mma_f16_16816(acc[j / 2], xa[2], xb[2], xa[3], xb[3], q.b[2 * j + 1][0], q.b[2 * j + 1][1]);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t* pr = i < 2 ? pa : pb;
                        float t = bf16lo(pr[0]) * acc[0][i], u = bf16hi(pr[0]) * q.sum[i & 1][0];
                        if constexpr (G == 2) {
                            t = fmaf(bf16lo(pr[1]), acc[1][i], t);
                            u = fmaf(bf16hi(pr[1]), q.sum[i & 1][1], u);
                        }
                        s[i] = fmaf(t, q.f[i & 1], u);
                    }
                } else {
                    float acc[4] = {0.f, 0.f, 0.f, 0.f};
                    const uint4* x = reinterpret_cast<const uint4*>(p.K + a0 * D) + c4;
                    const uint4* y = reinterpret_cast<const uint4*>(p.K + a1 * D) + c4;
                    uint4 ka[J], kb[J];
#pragma unroll
                    for (int j = 0; j < J; ++j) { ka[j] = x[4 * j]; kb[j] = y[4 * j]; }
#pragma unroll
                    for (int j = 0; j < J; ++j) {
                        mma_bf16_16816(acc, ka[j].x, kb[j].x, ka[j].y, kb[j].y, raw[j].x, raw[j].y);
                        mma_bf16_16816(acc, ka[j].z, kb[j].z, ka[j].w, kb[j].w, raw[j].z, raw[j].w);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[i] = acc[i] * p.scale_log2;
                }
                sum[rb][0] += (real0 ? ex2(s[0] - l0) : 0.f) + (real1 ? ex2(s[1] - l1) : 0.f);
                sum[rb][1] += (real0 ? ex2(s[2] - l0) : 0.f) + (real1 ? ex2(s[3] - l1) : 0.f);
            }
        }
#pragma unroll
        for (int rb = 0; rb < 4; ++rb) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float t = sum[rb][i];
                t += __shfl_xor_sync(FULL, t, 1);
                t += __shfl_xor_sync(FULL, t, 2);
                const int r = rb * 16 + 8 * i + g4;
                if (c4 == i && r < rows) {
                    const int64_t o = w0 + base + r;
                    p.weights[o] = p.prev ? p.prev[o] + t : t;
                }
            }
        }
    }
}

// ---- eviction -----------------------------------------------------------------------------------------------------------

constexpr int kSelectThreads = 1024;
constexpr int kSelectMostKeys = 48 * 1024;   // keys that a thread block keeps in shared memory

// Order of weights as whole numbers: larger weight, larger key; -0 as 0; a NaN below all.
__device__ __forceinline__ uint32_t weight_key(float w)
{
    const uint32_t u = __float_as_uint(w + 0.f);
    if ((u & 0x7fffffffu) > 0x7f800000u) return 0u;
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

struct SelectParams {
    const float* weights;     // [batch, H_kv, stride] or null (all equal)
    float* weights_out;       // [batch, H_kv, out_stride] or null; may be `weights`
    int32_t* kept;            // [batch, H_kv, n_keep]
    const int32_t* lens;
    int32_t* lens_out;        // lengths to set (another cache's), or null
    int64_t stride, out_stride, T_cap;
    int32_t H_kv, n_sink, n_recent, n_keep, out_rows, keys;
};

// One thread block per (sequence, kv head).  The smallest key that stays is found bit by bit: with t the bits found so
// far, count the keys >= t | bit.  That is at most 32 counts, fewer when a count meets the target (as with distinct
// weights it soon does).  Then every warp lists its own stretch of rows behind what the warps in front of it keep, so rows
// stay in order and equal weights go by the lowest row.
__global__ void __launch_bounds__(kSelectThreads) evict_select_kernel(const SelectParams p)
{
    extern __shared__ uint32_t keys[];
    __shared__ int counts[2][32], above[32], equal[32];
    pdl_wait_then_release();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int b = blockIdx.x / p.H_kv;
    const int len = p.lens[b];
    const int n = (int)min((int64_t)max(len, 0), p.T_cap);
    const float* w = p.weights ? p.weights + (int64_t)blockIdx.x * p.stride : nullptr;
    int32_t* kept = p.kept + (int64_t)blockIdx.x * p.n_keep;
    const int count = min(n, p.n_keep);
    if (p.lens_out && blockIdx.x % p.H_kv == 0 && tid == 0) p.lens_out[b] = count;
    if (n <= p.n_keep) {
        for (int i = tid; i < p.n_keep; i += kSelectThreads) kept[i] = i < n ? i : -1;
    } else {
        const int first = p.n_sink, m = n - p.n_recent - first;      // rows that compete
        const int target = p.n_keep - p.n_sink - p.n_recent;         // and how many of them stay (< m)
        const bool held = m <= p.keys;
        const auto key = [&](int i) { return held ? keys[i] : w ? weight_key(w[first + i]) : 0x80000000u; };
        if (held) {
            for (int i = tid; i < m; i += kSelectThreads) keys[i] = w ? weight_key(w[first + i]) : 0x80000000u;
            __syncthreads();
        }
        uint32_t t = 0;
        int turn = 0;
        const auto count_from = [&](uint32_t from) {
            int c = 0;
            for (int i = tid; i < m; i += kSelectThreads) c += key(i) >= from;
            c = __reduce_add_sync(0xffffffffu, c);
            if (lane == 0) counts[turn][warp] = c;
            __syncthreads();
            c = __reduce_add_sync(0xffffffffu, counts[turn][lane]);
            turn ^= 1;
            return c;
        };
        bool met = target == 0;
        if (met) t = 0xffffffffu;                                    // (no weight has this key: nothing stays)
        for (int bit = 31; bit >= 0 && !met; --bit) {
            const int c = count_from(t | (1u << bit));
            if (c >= target) t |= 1u << bit;
            met = c == target;
        }
        // met: all keys >= t stay; else all keys > t, and of those equal to t the first `ties`
        const int each = ((m + 31) / 32 + 31) / 32 * 32;             // rows per warp
        const int lo = min(m, warp * each), hi = min(m, lo + each);
        int n_above = 0, n_equal = 0;
        for (int i = lo + lane; i - lane < hi; i += 32) {
            const uint32_t k = i < hi ? key(i) : 0u;
            n_above += __popc(__ballot_sync(0xffffffffu, i < hi && (met ? k >= t : k > t)));
            n_equal += __popc(__ballot_sync(0xffffffffu, i < hi && !met && k == t));
        }
        if (lane == 0) { above[warp] = n_above; equal[warp] = n_equal; }
        __syncthreads();
        const int all_above = __reduce_add_sync(0xffffffffu, above[lane]);
        n_above = __reduce_add_sync(0xffffffffu, lane < warp ? above[lane] : 0);
        n_equal = __reduce_add_sync(0xffffffffu, lane < warp ? equal[lane] : 0);
        const int ties = target - all_above;
        const uint32_t below = (1u << lane) - 1u;
        for (int i = lo + lane; i - lane < hi; i += 32) {
            const uint32_t k = i < hi ? key(i) : 0u;
            const bool a = i < hi && (met ? k >= t : k > t), e = i < hi && !met && k == t;
            const uint32_t ab = __ballot_sync(0xffffffffu, a), eb = __ballot_sync(0xffffffffu, e);
            const int e_rank = n_equal + __popc(eb & below);
            const int at = first + n_above + __popc(ab & below) + min(e_rank, ties);
            if (a || (e && e_rank < ties)) kept[at] = first + i;
            n_above += __popc(ab);
            n_equal += __popc(eb);
        }
        for (int i = tid; i < p.n_sink; i += kSelectThreads) kept[i] = i;
        for (int i = tid; i < p.n_recent; i += kSelectThreads) kept[p.n_keep - p.n_recent + i] = n - p.n_recent + i;
    }
    if (!p.weights_out) return;
    // Rows only move down, so with weights in place a tile is read before it is written, and tiles go upwards.
    __syncthreads();
    float* out = p.weights_out + (int64_t)blockIdx.x * p.out_stride;
    for (int i0 = 0; i0 < p.out_rows; i0 += kSelectThreads) {
        const int i = i0 + tid;
        float x = 0.f;
        if (i < count && w) x = w[kept[i]];
        __syncthreads();
        if (i < p.out_rows) out[i] = x;
    }
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
    int32_t batch, n_keep;
};

constexpr int kStatusNoRow = 2;   // a row had no place (LCKV_ECAPACITY)

// Physical rows of item (b, h, i): from and to; negative where there is nothing to do.
struct MoveRow { int64_t from, to; };
__device__ __forceinline__ MoveRow move_row(const MoveParams& p, int64_t item)
{
    MoveRow r = {-1, -1};
    const int row = p.kept[item];
    if (row < 0) return r;
    const int i = (int)(item % p.n_keep);
    const int64_t bh = item / p.n_keep;
    const int h = (int)(bh % p.map.H_kv), b = (int)(bh / p.map.H_kv);
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
    static __device__ __forceinline__ const Unit* at(const PackedSlot& s, const uint16_t* K, const uint16_t* V, int64_t row, int u)
    {
        if constexpr (PACKED) {
            if (u < 4) return reinterpret_cast<const Unit*>(s.kc + row * (D / 2)) + u;
            if (u < 8) return reinterpret_cast<const Unit*>(s.vc + row * (D / 2)) + (u - 4);
            return reinterpret_cast<const Unit*>(s.par + row * (D / 32));
        } else {
            return reinterpret_cast<const Unit*>((u < D / 8 ? K : V) + row * D) + (u < D / 8 ? u : u - D / 8);
        }
    }
};

// From one slot to another of the same kind.
template <int D, bool PACKED>
__global__ void __launch_bounds__(256) evict_move_kernel(const MoveParams p, int64_t items)
{
    using U = RowUnits<D, PACKED>;
    pdl_wait_then_release();
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t item = i / U::kUnits;
    if (item >= items) return;
    const int u = (int)(i % U::kUnits);
    const MoveRow r = move_row(p, item);
    if (r.from < 0) return;
    const auto v = *U::at(p.from, p.K, p.V, r.from, u);
    *const_cast<typename U::Unit*>(U::at(p.to, p.K_to, p.V_to, r.to, u)) = v;
}

// From bf16 rows to 4-bit rows; lanes as in packed_write_kernel.
template <int D>
__global__ void __launch_bounds__(256) evict_pack_kernel(const MoveParams p, int64_t items)
{
    constexpr int LANES = D / 4;
    pdl_wait_then_release();
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t item = i / LANES;
    const int l = (int)(i % LANES), is_v = l >= D / 8, w = l % (D / 8);
    MoveRow r = {-1, -1};
    if (item < items) r = move_row(p, item);
    uint4 x = make_uint4(0, 0, 0, 0);
    if (r.from >= 0) x = *reinterpret_cast<const uint4*>((is_v ? p.V : p.K) + r.from * D + w * 8);
    uint32_t word, par;
    packed_encode(x, word, par);
    if (r.from < 0) return;
    uint32_t* codes = reinterpret_cast<uint32_t*>(is_v ? p.to.vc : p.to.kc) + r.to * (D / 8);
    codes[is_v ? packed_v_word<D>(w) : packed_k_word<D>(w)] = word;
    if ((w & 7) == 0) p.to.par[r.to * (D / 32) + is_v * (D / 64) + (w >> 3)] = par;
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
    const int64_t item0 = (int64_t)blockIdx.x * p.n_keep;
    for (int i0 = 0; i0 < p.n_keep; i0 += ROWS) {
        typename U::Unit v[X];
        int64_t to[X];
#pragma unroll
        for (int x = 0; x < X; ++x) {
            const int k = x * 1024 + threadIdx.x, i = i0 + k / U::kUnits;
            to[x] = -1;
            if (k < ROWS * U::kUnits && i < p.n_keep) {
                const MoveRow r = move_row(p, item0 + i);
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
