// Products with 4-bit weights on the 5th-generation tensor cores, for batches beyond a few rows.
//
// Same mathematics and the same packed weights as lckv_quant.cuh: D[128 features x NB rows] = C . x^T, NB <= 128, with the
// exact c - z as the A operand in tensor memory and x as the B operand in shared memory.  A group's D is a fresh
// accumulator; it is read back, multiplied by its scale in fp32 and added to the result in registers, so that no scale is
// rounded into a weight and the sums over groups are plain fp32.
//
//   warps 0, 2    producers: one bulk copy of packed weights per 128 k; TMA boxes of x (128-byte swizzle)
//   warp 1        one thread issues tcgen05.mma: A from tensor memory, B from shared memory
//   fold warps    tensor memory -> registers (thread = feature, 32 columns a warp), times scale, into fp32 sums; the
//                 epilogue.  4 warps for up to 32 rows, 16 beyond.  They fetch the scales from the L2 two blocks ahead
//   nibble warps  nibbles -> A: sets of 4 warps take the k blocks in turn, each with an A buffer of its own, so that
//                 the chain copy -> nibbles -> tensor memory -> MMA of one block is hidden behind the other sets.  A
//                 warp owns 32 features = its quadrant of the tensor memory, and the words that a lane owns in the
//                 packed layout are exactly what it stores with tcgen05.st.16x256b (bf16) or 16x128b (e4m3)
//
// A role that runs through a step alone is the step's time: what a role waits for and computes per step is kept short
// (rings kept by addition, uniform descriptors, one wait for the fold warps).
//
//   x in bf16: kind::f16, A = (16 + c) - (16 + z) in bf16, one subtraction per pair on the otherwise idle FMA pipe.
//   x in e4m3: kind::f8f6f4, A = c / 512 in e4m3, and a second product with A' = -z / 512, the same for all k of a
//              group, accumulated into the same D.
//
// Bound by the integer instructions of the nibbles for few rows (7 or 6 per 8 codes: 224 cycles per SM and 128 x 128 block)
// and by the MMAs for many (512 cycles at NB = 128).  Few features: d_model is shared by a cluster whose partial results meet
// in distributed shared memory, as in lckv_project.cuh, in a fixed order.  Every wait is bounded; one that runs out sets
// the status word, if the caller gave one, and the tile's results become NaN.  Any role may give up alone; the roles that
// started copies and MMAs then wait for their end before the thread block's memory serves the result.
#pragma once
#include "lckv_quant.cuh"

namespace lckv {

// Polls of a wait.  A constant: with the limit read from the parameters the roles took 3 to 5 % longer (512 rows of bf16 60.3 / 63.5 us).
constexpr uint32_t kQ5WaitLimit = 1u << 16;
constexpr int kQ5MaxStages = 12;

__host__ __device__ constexpr int q5_fold_warps(int NBMAX) { return NBMAX / 8; }     // 32 columns each, by 4 quadrants
// Sets of nibble warps, and A buffers.  In e4m3, with half of the nibbles' instructions, two sets suffice, which leaves the
// fold warps 72 registers a thread (512 rows, 4096 x 12288: 92.9 / 89.6 us with three / two).  Groups of 128 need no more; groups
// of 64 and 32 still spill a few (stack frames of 8 and 24 to 32 bytes).
__host__ __device__ constexpr int q5_sets(int NBMAX, bool f8) { return NBMAX > 32 ? (f8 ? 2 : 3) : 4; }
__host__ __device__ constexpr int q5_threads(int NBMAX, bool f8) { return (4 + q5_fold_warps(NBMAX) + 4 * q5_sets(NBMAX, f8)) * 32; }
__host__ __device__ constexpr int q5_block(int group, bool zeros)      // bytes of 32 features x 128 k
{
    return kQuantCodes + kQuantK / group * kQuantFeat * (zeros ? 3 : 2);
}
__host__ __device__ inline int q5_stage_bytes(int NB, bool f8, int block) { return NB * (f8 ? 128 : 256) + 4 * block; }
constexpr int kQ5OutLd = 128 + 4;       // fp32 column of the result, padded
constexpr int kQ5XScales = 4096;        // x scales of two k blocks for every fold warp
__host__ __device__ inline int q5_pipe_bytes(int NB, bool f8, int block, int stages)      // the result is staged in it
{
    const int pipe = stages * q5_stage_bytes(NB, f8, block), out = NB * kQ5OutLd * 4;
    return pipe > out ? pipe : out;
}
__host__ __device__ inline int q5_smem_bytes(int NB, bool f8, int block, int stages)
{
    return q5_pipe_bytes(NB, f8, block, stages) + (f8 ? kQ5XScales : 0) + 512 + 1024;
}

struct Quant5Params {
    const uint8_t* w;
    const float* x_scale;
    void* y;
    int32_t* status;         // or null
    int64_t y_stride;
    int32_t m, n, k;
    int32_t n_blocks, k_blocks;
    int32_t x_blocks;
    int32_t y32, y_vec;      // y_vec: 4 features of y can be stored at once
    int32_t k_split, NB, stages;
    int32_t w_limit, x_limit;            // blocks of 128 k that a thread block requests; fewer than there are only in tests
};

// D[tmem] (+)= A[tmem] * B[smem], fp32 accumulate (ACC = 0: from zero); bf16 and e4m3 inputs.
template <int ACC>
__device__ __forceinline__ void tc5_mma_ts_f16(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "n"(ACC)
        : "memory");
}
template <int ACC>
__device__ __forceinline__ void tc5_mma_ts_f8(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "n"(ACC)
        : "memory");
}
// 1 in one lane of a converged warp, 0 in the others.
__device__ __forceinline__ uint32_t elect_one()
{
    uint32_t p;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "elect.sync _|p, 0xffffffff;\n\t"
        "selp.b32 %0, 1, 0, p;\n\t}"
        : "=r"(p));
    return p;
}
__host__ __device__ constexpr uint32_t tc5_idesc_f8(int M, int N)      // e4m3 x e4m3 -> fp32, both K-major
{
    return (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
// 16 rows x 8 columns of 32 bits per 4 registers: lane (g, t) holds columns 2 t, 2 t + 1 of rows g and g + 8.
__device__ __forceinline__ void tmem_st_16x256_x4(uint32_t taddr, const uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.st.sync.aligned.16x256b.x4.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
          "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
// 16 rows x 4 columns of 32 bits per 2 registers: lane (g, t) holds column t of rows g and g + 8.
__device__ __forceinline__ void tmem_st_16x128_x4(uint32_t taddr, const uint32_t (&r)[8])
{
    asm volatile("tcgen05.st.sync.aligned.16x128b.x4.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// 16 consecutive 32-bit columns of this thread's tensor-memory lane, not waited for.
__device__ __forceinline__ void tmem_ld16_nowait(uint32_t taddr, float* r)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]),
                   "=f"(r[9]), "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15])
                 : "r"(taddr)
                 : "memory");
}
__device__ __forceinline__ float lds_f32(uint32_t addr)
{
    float v;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}
// Place in a ring of n slots and the parity of its round.  A role that waits for a slot to be filled waits for `phase`, one
// that waits for it to be free for phase ^ 1 (true at once in the first round).  Kept by addition: a division by the
// number of slots per step and role was half of a step's time.
struct RingPos {
    int s;
    uint32_t phase;
    __device__ __forceinline__ void next(int n, int by = 1)
    {
        s += by;
        if (s >= n) { s -= n; phase ^= 1; }
    }
};

template <bool F8, bool ZEROS, int GROUP, int NBMAX>
__global__ void __launch_bounds__(q5_threads(NBMAX, F8), 1)
quant_tc5_kernel(const Quant5Params p, const __grid_constant__ CUtensorMap tmX)
{
    constexpr int BLOCK = q5_block(GROUP, ZEROS), SCALES = kQuantK / GROUP * kQuantFeat * 2, GPS = kQuantK / GROUP;
    constexpr int FOLD = q5_fold_warps(NBMAX), FOLD0 = 4, DEQ0 = FOLD0 + FOLD, SETS = q5_sets(NBMAX, F8), NBC = 32;
    constexpr int A_COLS = F8 ? 32 + (ZEROS ? GPS * 8 : 0) : 64, CONST_COLS = F8 && !ZEROS ? 8 : 0;
    constexpr int TM_NEED = SETS * A_COLS + CONST_COLS + 2 * NBMAX;
    constexpr uint32_t TM_COLS = TM_NEED <= 32 ? 32 : TM_NEED <= 64 ? 64 : TM_NEED <= 128 ? 128 : TM_NEED <= 256 ? 256 : 512;
    static_assert(TM_NEED <= 512, "tensor memory");
    static_assert(16 * kQ5MaxStages + 16 * SETS + 56 <= 512, "barriers");
    constexpr uint32_t A_CONST = SETS * A_COLS, D0 = A_CONST + CONST_COLS;
    constexpr int ROW = F8 ? 128 : 256;              // bytes of x per row and k block
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem0 = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const int NB = p.NB, NS = p.stages;
    const int x_bytes = NB * ROW;
    const uint32_t sX = smem0, sW = sX + NS * x_bytes;                                // x tiles, weights
    const uint32_t sXS = smem0 + (uint32_t)q5_pipe_bytes(NB, F8, BLOCK, NS);          // x scales
    const uint32_t bars = sXS + (F8 ? kQ5XScales : 0);
    const uint32_t bFull = bars, bEmpty = bars + 8 * kQ5MaxStages, bAFull = bars + 16 * kQ5MaxStages, bAEmpty = bAFull + 8 * SETS,
                   bDFull = bAFull + 16 * SETS, bDEmpty = bDFull + 16, bDrain = bDFull + 32, sTaddr = bDFull + 40, sBad = sTaddr + 4,
                   sIssued = sTaddr + 8;             // stages that the two producers have requested
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    const int m0 = blockIdx.y * NB, nb0 = blockIdx.x * 4;
    const int KS = p.k_split;
    const uint32_t rank = KS > 1 ? cluster_ctarank() : 0u;
    const int k_lo = (int)rank * p.k_blocks / KS, k_hi = ((int)rank + 1) * p.k_blocks / KS, n_k = k_hi - k_lo;

    if (tid == 0) {
        for (int s = 0; s < NS; ++s) { mbar_init(bFull + 8 * s, 2); mbar_init(bEmpty + 8 * s, 5); }
        for (int s = 0; s < SETS; ++s) { mbar_init(bAFull + 8 * s, 4); mbar_init(bAEmpty + 8 * s, 1); }
        for (int s = 0; s < 2; ++s) {
            mbar_init(bDFull + 8 * s, 1);
            mbar_init(bDEmpty + 8 * s, FOLD);
        }
        mbar_init(bDrain, 1);
        asm volatile("st.shared.u32 [%0], %1;" ::"r"(sBad), "r"(0) : "memory");
        fence_mbar_init();
    }
    if (warp == 1) tmem_alloc(sTaddr, TM_COLS);
    tc5_fence_before();
    __syncthreads();
    tc5_fence_after();
    uint32_t tm;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tm) : "r"(sTaddr));
    if (CONST_COLS) {
        if (warp >= DEQ0 && warp < DEQ0 + 4) {           // A' = -8 / 512 for all k, thread = feature
            asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%1,%1,%1,%1,%1,%1,%1};"
                         ::"r"(tm + A_CONST + ((uint32_t)((warp & 3) * 32) << 16)), "r"(0x88888888u) : "memory");
            tmem_st_wait();
        }
        tc5_fence_before();
        __syncthreads();
        tc5_fence_after();
    }

    float* out = reinterpret_cast<float*>(smem_raw + (smem0 - smem_u32(smem_raw)));
    // The end of every role: all MMAs and copies of the block are done, and a wait that ran out is known to all.
    int mma_lane = 0;                                // which lane of warp 1 issues MMAs
    auto finish = [&](bool ok) -> uint32_t {
        if (!ok) {
            asm volatile("st.shared.u32 [%0], %1;" ::"r"(sBad), "r"(1) : "memory");
            if (p.status) atomicExch(p.status, kStatusTimeout);
        }
        tc5_fence_before();
        __syncthreads();
        tc5_fence_after();
        uint32_t bad;
        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(bad) : "r"(sBad) : "memory");
        if (bad) {
            // Without a wait that ran out the fold warps have seen every MMA end, and so every copy land.  Here copies and MMAs may
            // still be under way.  The producers may have stopped at different stages, at most NS apart: the one behind arrives
            // for what it has not requested, so that the barriers of the last NS stages count the bytes that are under way.
            if (warp == 0 || warp == 2) {
                int mine, other;
                asm volatile("ld.shared.u32 %0, [%1];" : "=r"(mine) : "r"(sIssued + 2u * warp) : "memory");
                asm volatile("ld.shared.u32 %0, [%1];" : "=r"(other) : "r"(sIssued + 4u - 2u * warp) : "memory");
                if (lane == 0)
                    for (int k = mine; k < other; ++k) mbar_arrive(bFull + 8 * (k % NS));
                const int end = mine > other ? mine : other;
                for (int k = end > NS ? end - NS : 0; k < end; ++k) (void)mbar_wait_bounded(bFull + 8 * (k % NS), (k / NS) & 1, kQ5WaitLimit);
            } else if (warp == 1) {
                if (lane == mma_lane) tc5_commit(bDrain);
                __syncwarp();
                (void)mbar_wait_bounded(bDrain, 0, kQ5WaitLimit);
            }
            __syncthreads();
        }
        return bad;
    };

    bool ok = true;
    if (warp != 0) pdl_wait();                       // the bounded waits below count no other kernel's time
    if (warp == 0 || warp == 2) {
        // ------------------------------------------------------------------ producers: weights (0), x (2)
        // (weights never come from the kernel before this one: the first stages are requested before its end)
        const bool is_w = warp == 0;
        const uint32_t leader = elect_one();
        const uint8_t* src = p.w + ((int64_t)blockIdx.x * p.k_blocks + k_lo) * (4 * BLOCK);
        RingPos r = {0, 0};
        const int limit = is_w ? p.w_limit : p.x_limit, n_mine = n_k < limit ? n_k : limit;
        int issued = 0;
        for (; issued < n_mine; ++issued, r.next(NS)) {
            if (is_w && issued == NS) pdl_wait();    // (from here on it waits for work that waits for x)
            ok = mbar_wait_bounded(bEmpty + 8 * r.s, r.phase ^ 1, kQ5WaitLimit);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            if (leader) {
                mbar_expect_tx(bFull + 8 * r.s, is_w ? (uint32_t)(4 * BLOCK) : (uint32_t)x_bytes);
                if (is_w) {
                    bulk_g2s(sW + r.s * 4 * BLOCK, src + (int64_t)issued * (4 * BLOCK), 4 * BLOCK, bFull + 8 * r.s);
                } else {
                    const int x = (k_lo + issued) * kQuantK;
                    tma_load_2d(sX + r.s * x_bytes, &tmX, x, m0, bFull + 8 * r.s);
                    if (!F8) tma_load_2d(sX + r.s * x_bytes + NB * 128, &tmX, x + 64, m0, bFull + 8 * r.s);
                }
            }
            __syncwarp();
        }
        if (leader) asm volatile("st.shared.u32 [%0], %1;" ::"r"(sIssued + 2u * warp), "r"(issued) : "memory");
        __syncwarp();
        pdl_release();
        finish(ok);
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer
        // The whole warp runs the loop, so that addresses and descriptors stay in uniform registers; one elected lane
        // issues.  (With a loop of one lane alone an MMA took 90 cycles to issue, whatever its size.)
        const uint32_t leader = elect_one();
        const uint32_t idesc = F8 ? tc5_idesc_f8(128, NB) : tc5_idesc(128, NB, 0);
        const uint64_t desc0 = tc5_desc(sX, 16, 1024);
        const uint32_t tmu = __shfl_sync(0xffffffffu, tm, 0);
        RingPos r = {0, 0}, ra = {0, 0}, rd = {0, 0};
        for (int k = 0; k < n_k; ++k, r.next(NS), ra.next(SETS)) {
            // (the nibble warps that filled A have seen the stage's copies land, x among them)
            ok = mbar_wait_bounded(bAFull + 8 * ra.s, ra.phase, kQ5WaitLimit);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            tc5_fence_after();
            const uint32_t a0 = tmu + ra.s * A_COLS;
            const uint64_t xd = desc0 + (uint32_t)(r.s * x_bytes >> 4), xd2 = xd + (uint32_t)(NB * 128 >> 4);
#pragma unroll
            for (int gl = 0; gl < GPS; ++gl, rd.next(2)) {
                ok = mbar_wait_bounded(bDEmpty + 8 * rd.s, rd.phase ^ 1, kQ5WaitLimit);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc5_fence_after();
                const uint32_t d = tmu + D0 + rd.s * NBMAX;
                if (leader) {
                    if constexpr (F8) {
#pragma unroll
                        for (int i = 0; i < GROUP / 32; ++i) {
                            const int k32 = gl * (GROUP / 32) + i;
                            if (i == 0) tc5_mma_ts_f8<0>(d, a0 + k32 * 8, xd + k32 * 2, idesc);
                            else tc5_mma_ts_f8<1>(d, a0 + k32 * 8, xd + k32 * 2, idesc);
                            tc5_mma_ts_f8<1>(d, ZEROS ? a0 + 32 + gl * 8 : tmu + A_CONST, xd + k32 * 2, idesc);
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < GROUP / 16; ++i) {
                            const int k16 = gl * (GROUP / 16) + i;
                            if (i == 0) tc5_mma_ts_f16<0>(d, a0 + k16 * 8, (k16 < 4 ? xd : xd2) + (k16 & 3) * 2, idesc);
                            else tc5_mma_ts_f16<1>(d, a0 + k16 * 8, (k16 < 4 ? xd : xd2) + (k16 & 3) * 2, idesc);
                        }
                    }
                    tc5_commit(bDFull + 8 * rd.s);
                    if (gl == GPS - 1) {
                        tc5_commit(bAEmpty + 8 * ra.s);
                        tc5_commit(bEmpty + 8 * r.s);
                    }
                }
                __syncwarp();
            }
            if (!ok) break;
        }
        mma_lane = __ffs(__ballot_sync(0xffffffffu, leader)) - 1;
        finish(ok);
    } else if (warp < FOLD0) {
        finish(true);
    } else if (warp < DEQ0) {
        // ------------------------------------------------------------------ fold
        const int q4 = warp & 3, c0 = ((warp - FOLD0) >> 2) * NBC;
        const uint32_t dl = tm + D0 + ((uint32_t)(q4 * 32) << 16) + c0;
        uint64_t acc[NBC / 2];                       // pairs of columns
#pragma unroll
        for (int c = 0; c < NBC / 2; ++c) acc[c] = 0;
        // This feature's scale of the next two steps' groups, straight from the packed weights.
        const int so = (lane & 7) * 4 + (lane >> 4) * 2 + ((lane >> 3) & 1);         // its place among 32
        const uint16_t* ps = reinterpret_cast<const uint16_t*>(p.w + (((int64_t)blockIdx.x * p.k_blocks + k_lo) * 4 + q4) * BLOCK + kQuantCodes) + so;
        uint16_t sc[2][GPS];
        auto fetch_groups = [&](int k, uint16_t (&to)[GPS]) {
#pragma unroll
            for (int gl = 0; gl < GPS; ++gl) to[gl] = k < n_k ? __ldg(ps + (int64_t)k * (2 * BLOCK) + gl * kQuantFeat) : (uint16_t)0;
        };
        fetch_groups(0, sc[0]);
        fetch_groups(1, sc[1]);
        // one scale of x per row and k block: lane c fetches column c two blocks ahead, and the warp reads them back from its
        // own corner of shared memory
        float xn[2];
        auto fetch_scales = [&](int k, float& to) {
            const int m = m0 + c0 + lane;
            to = k < n_k && c0 + lane < NB && m < p.m ? p.x_scale[(int64_t)m * p.x_blocks + k_lo + k] : 0.f;
        };
        if (F8 && p.x_blocks) {
            fetch_scales(0, xn[0]);
            fetch_scales(1, xn[1]);
        }
        // D is free once its last columns are in registers, before they are added (512 rows of bf16: 62.9 / 60.6 us; up to 32
        // rows, and in e4m3, where it costs registers, no gain)
        constexpr bool EARLY = NBMAX > 32 && !F8;
        RingPos rd = {0, 0};
        // (`blocks` is a constant of each of its two copies: asked in the inner loop it cost 512 rows in e4m3 88.5 us for 72.1)
        auto step = [&](const bool blocks, int k, uint16_t (&scale)[GPS], float& xk) {
            const uint32_t xs0 = sXS + (uint32_t)(((warp - FOLD0) * 2 + (k & 1)) * NBC) * 4;
            if (blocks) {
                asm volatile("st.shared.f32 [%0], %1;" ::"r"(xs0 + lane * 4), "f"(xk) : "memory");
                __syncwarp();
                fetch_scales(k + 2, xk);
            }
#pragma unroll
            for (int gl = 0; gl < GPS; ++gl, rd.next(2)) {
                float f = __uint_as_float((uint32_t)scale[gl] << 16);
                if (F8) f *= 512.f;
                const uint64_t f2 = pack_f32x2(f, f);
                ok = mbar_wait_bounded(bDFull + 8 * rd.s, rd.phase, kQ5WaitLimit);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) return;
                tc5_fence_after();
                const uint32_t d = dl + rd.s * NBMAX;
                auto free_d = [&] {
                    tc5_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bDEmpty + 8 * rd.s);
                };
#pragma unroll
                for (int c = 0; c < NBC; c += 16) {
                    float v[16];
                    if (c0 + c >= NB) {
                        if (EARLY && c + 16 == NBC) free_d();
                        continue;
                    }
                    tmem_ld16_nowait(d + c, v);
                    tmem_ld_wait();
                    if (EARLY && c + 16 == NBC) free_d();
#pragma unroll
                    for (int j = 0; j < 16; j += 4) {
                        uint64_t fa = f2, fb = f2;
                        if (blocks) {
                            const uint4 x4 = lds128(xs0 + (c + j) * 4);
                            fa = fmul2(f2, pack_f32x2(__uint_as_float(x4.x), __uint_as_float(x4.y)));
                            fb = fmul2(f2, pack_f32x2(__uint_as_float(x4.z), __uint_as_float(x4.w)));
                        }
                        acc[(c + j) / 2] = ffma2(fa, pack_f32x2(v[j], v[j + 1]), acc[(c + j) / 2]);
                        acc[(c + j) / 2 + 1] = ffma2(fb, pack_f32x2(v[j + 2], v[j + 3]), acc[(c + j) / 2 + 1]);
                    }
                }
                if (!EARLY) free_d();
            }
            fetch_groups(k + 2, scale);
        };
        auto steps = [&](const bool blocks) {
            for (int k = 0; k < n_k && ok; k += 2) {
                step(blocks, k, sc[0], xn[0]);
                if (k + 1 < n_k && ok) step(blocks, k + 1, sc[1], xn[1]);
            }
        };
        if (F8 && p.x_blocks) steps(true);
        else steps(false);
        const uint32_t bad = finish(ok);
        // the block's stages become its result, [column][feature] in fp32
#pragma unroll
        for (int c = 0; c < NBC; c += 2) {
            if (c0 + c >= NB) break;
            float v0, v1;
            unpack_f32x2(acc[c / 2], v0, v1);
            if (bad) v0 = v1 = __uint_as_float(0x7fffffffu);
            out[(c0 + c) * kQ5OutLd + q4 * 32 + lane] = v0;
            out[(c0 + c + 1) * kQ5OutLd + q4 * 32 + lane] = v1;
        }
    } else {
        // ------------------------------------------------------------------ nibbles -> A
        const int q4 = warp & 3, set = (warp - DEQ0) >> 2;
        RingPos r = {set, 0};                        // (the ring has at least as many slots as there are sets)
        uint32_t free_phase = 1;
        for (int k = set; k < n_k && ok; k += SETS, r.next(NS, SETS), free_phase ^= 1) {
            const int s = r.s;
            ok = mbar_wait_bounded(bFull + 8 * s, r.phase, kQ5WaitLimit) &&
                 mbar_wait_bounded(bAEmpty + 8 * set, free_phase, kQ5WaitLimit);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            tc5_fence_after();
            const uint32_t blk = sW + (s * 4 + q4) * BLOCK;
            const uint32_t a0 = tm + set * A_COLS + ((uint32_t)(q4 * 32) << 16);
#pragma unroll
            for (int tile = 0; tile < 2; ++tile) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint4 c = lds128(blk + ((h * 2 + tile) * 32 + lane) * 16);
                    const uint32_t w[4] = {c.x, c.y, c.z, c.w};              // (k32, upper half of the features)
                    if constexpr (F8) {
                        uint32_t r[8];
#pragma unroll
                        for (int j = 0; j < 2; ++j)
#pragma unroll
                            for (int st = 0; st < 2; ++st)
#pragma unroll
                                for (int hi = 0; hi < 2; ++hi)
                                    r[j * 4 + st * 2 + hi] =
                                        __byte_perm(__funnelshift_r(w[j * 2 + hi], w[j * 2 + hi], 3 + 4 * st) & 0x0f0f0f0fu, 0, 0x3120);
                        tmem_st_16x128_x4(a0 + ((uint32_t)(tile * 16) << 16) + h * 16, r);
                    } else {
                        uint32_t r[16];
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            uint32_t zp[2] = {0x41c041c0u, 0x41c041c0u};     // 16 + 8
                            if (ZEROS) {
                                const int gl = (h * 64 + j * 32) / GROUP;
                                uint32_t z;
                                asm volatile("ld.shared.u32 %0, [%1];" : "=r"(z) : "r"(blk + kQuantCodes + SCALES + gl * kQuantFeat + (lane >> 2) * 4) : "memory");
                                zp[0] = __byte_perm(z, 0x41414141u, tile ? 0x4242u : 0x4040u);
                                zp[1] = __byte_perm(z, 0x41414141u, tile ? 0x4343u : 0x4141u);
                            }
#pragma unroll
                            for (int st = 0; st < 2; ++st)
#pragma unroll
                                for (int hi = 0; hi < 2; ++hi)
#pragma unroll
                                    for (int pr = 0; pr < 2; ++pr) {
                                        const uint32_t u = w[j * 2 + hi];
                                        r[(j * 2 + st) * 4 + hi * 2 + pr] =
                                            sub_bf16x2(and_or(__funnelshift_r(u, u, 4 * (pr * 2 + st)), 0x00780078u, 0x41804180u), zp[hi]);
                                    }
                        }
                        tmem_st_16x256_x4(a0 + ((uint32_t)(tile * 16) << 16) + h * 32, r);
                    }
                }
            }
            if constexpr (F8 && ZEROS) {
                // A' of each group: -z / 512, one value per feature (thread = feature here)
#pragma unroll
                for (int gl = 0; gl < GPS; ++gl) {
                    uint32_t z;
                    const int so = (lane & 7) * 4 + (lane >> 4) * 2 + ((lane >> 3) & 1);
                    asm volatile("ld.shared.u8 %0, [%1];" : "=r"(z) : "r"(blk + kQuantCodes + SCALES + gl * kQuantFeat + so) : "memory");
                    z = ((z >> 3) & 15u) | 0x80u;
                    z *= 0x01010101u;
                    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%1,%1,%1,%1,%1,%1,%1};" ::"r"(a0 + 32 + gl * 8), "r"(z) : "memory");
                }
            }
            tmem_st_wait();
            tc5_fence_before();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(bEmpty + 8 * s);         // the codes have been read
                mbar_arrive(bAFull + 8 * set);
            }
        }
        finish(ok);
    }
    if (warp == 1) tmem_dealloc(tm, TM_COLS);
    pdl_wait();                                      // y may still be read by the kernel before this one
    __syncthreads();
    if (KS > 1) cluster_sync_all();
    const int n_places = NB * 32;                    // 4 features each
    for (int i = (int)rank * (int)blockDim.x + tid; i < n_places; i += KS * (int)blockDim.x) {
        const int c = i >> 5, f = (i & 31) * 4, m = m0 + c, n = nb0 * kQuantFeat + f;
        if (m >= p.m || n >= p.n) continue;
        float v[4] = {0.f, 0.f, 0.f, 0.f};
        for (int r = 0; r < KS; ++r) {
            const float4 u = KS > 1 ? ld_cluster_f4(smem_u32(out + c * kQ5OutLd + f), (uint32_t)r)
                                    : *reinterpret_cast<const float4*>(out + c * kQ5OutLd + f);
            v[0] += u.x; v[1] += u.y; v[2] += u.z; v[3] += u.w;
        }
        if (F8 && !p.x_blocks) {
            const float xs = p.x_scale[m];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] *= xs;
        }
        const int64_t at = (int64_t)m * p.y_stride + n;
        if (p.y32) {
            float* y = static_cast<float*>(p.y) + at;
            if (p.y_vec && n + 3 < p.n) *reinterpret_cast<float4*>(y) = make_float4(v[0], v[1], v[2], v[3]);
            else
                for (int e = 0; e < 4 && n + e < p.n; ++e) y[e] = v[e];
        } else {
            uint16_t* y = static_cast<uint16_t*>(p.y) + at;
            if (p.y_vec && n + 3 < p.n) *reinterpret_cast<uint2*>(y) = make_uint2(cvt_bf16x2(v[0], v[1]), cvt_bf16x2(v[2], v[3]));
            else
                for (int e = 0; e < 4 && n + e < p.n; ++e) y[e] = (uint16_t)f32_to_bf16_bits(v[e]);
        }
    }
    if (KS > 1) cluster_sync_all();                  // a block's shared memory outlives the others' reads
}

}  // namespace lckv
