// C entry points of the operators around the attention: rotary positions, the rotated append, the residual
// norm, products with 4-bit weights.  Included at the end of lckv_api.cu (they share its cache object and helpers).
#pragma once

namespace {

// Do [a, a + na) and [b, b + nb) share a byte?
bool ranges_meet(const void* a, int64_t na, const void* b, int64_t nb)
{
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return x < y + (uintptr_t)nb && y < x + (uintptr_t)na;
}

bool aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

template <typename... KArgs, typename... Args>
cudaError_t launch_pdl_dims(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, Args... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

int rope_args(const lckv_rope_t* r, int head_dim, lckv::RopeArgs* out)
{
    if (!r || r->struct_size != sizeof(lckv_rope_t) || !r->cos || !r->sin) return LCKV_EINVAL;
    if (r->rot_dim < 2 || (r->rot_dim & 1) || r->rot_dim > head_dim) return LCKV_EINVAL;
    if (r->positions < 1 || (r->interleaved != 0 && r->interleaved != 1)) return LCKV_EINVAL;
    if (!aligned(r->cos, 4) || !aligned(r->sin, 4)) return LCKV_EINVAL;
    out->cos = r->cos;
    out->sin = r->sin;
    out->positions = r->positions;
    out->half = r->rot_dim / 2;
    out->interleaved = r->interleaved;
    out->sgn = 1.f;
    return LCKV_OK;
}

bool rope_tables_meet(const lckv_rope_t* r, const void* out, int64_t bytes)
{
    const int64_t n = (int64_t)r->positions * (r->rot_dim / 2) * 4;
    return ranges_meet(out, bytes, r->cos, n) || ranges_meet(out, bytes, r->sin, n);
}

bool rope_tables_vector(const lckv_rope_t* r) { return r->rot_dim % 16 == 0 && aligned(r->cos, 16) && aligned(r->sin, 16); }

// Heads per thread: four when there are enough units to fill the GPU's threads one and a half times (one fetch of the
// unit's cos and sin serves four heads and four pairs of loads are in flight: 32768 tokens of 8 heads of 64 13.2 us, with
// one 15.1 us), one when there are few (64 x 8 tokens of 96 heads 6.1 us, with four 6.5 us).
bool rope_many(int64_t units, int sms) { return units * 2 >= (int64_t)sms * 2048 * 3; }

// Where a thread fetches its factors one by one: as many heads as leave half of the GPU's threads busy, in fours.
int rope_heads(int path, int hp, int64_t tokens, int heads, int d, int sms)
{
    if (path != lckv::kRopeAnySize || hp == 1) return hp;
    const int64_t fit = tokens * heads * (d / 8) / ((int64_t)sms * 1024);
    return (int)std::max<int64_t>(4, std::min<int64_t>(fit, heads) / 4 * 4);
}

// A token takes `per` threads.  Blocks of 256, or of up to 384 where 256 would leave a fifth of them idle and there are many
// tokens: 96 heads of 128, four a thread, make 192 (32768 tokens 248 us, with one token in 256 threads 259; 16384 tokens of
// 32768 places 136, 145: a block whose tokens lie behind their prompts costs a nanosecond).
dim3 rope_grid(int64_t tokens, int heads, int d, int path, int hp, lckv::RopeGrid* g, dim3* block)
{
    const int units = lckv::rope_units(path, d);             // a power of two, as d is
    g->hg = (heads + hp - 1) / hp;
    g->units_shift = 0;
    while ((1 << g->units_shift) < units) ++g->units_shift;
    g->per = (uint32_t)(g->hg * units);
    g->inv = ((1u << 20) + g->per - 1) / g->per;
    g->tb = 0;
    *block = dim3(lckv::kRopeThreads);
    if (g->per >= (uint32_t)lckv::kRopeThreads)
        return dim3((unsigned)tokens, (g->per + lckv::kRopeThreads - 1) / lckv::kRopeThreads);
    g->tb = lckv::kRopeThreads / g->per;
    const uint32_t more = lckv::kRopeMostThreads / g->per;
    if (path != lckv::kRopeAnySize && tokens >= (1 << 14) && g->tb * g->per * 5 < (uint32_t)lckv::kRopeThreads * 4 && more > g->tb) {
        g->tb = more;
        *block = dim3((more * g->per + 31) / 32 * 32);
    }
    return dim3((unsigned)((tokens + g->tb - 1) / g->tb));
}

template <typename T>
void (*rope_apply_variant(int path, int hp))(lckv::RopeApplyParams)
{
    if (path == lckv::kRopePairs) return lckv::rope_apply_kernel<T, lckv::kRopePairs, 1>;
    if (path == lckv::kRopeUnits) return hp == 4 ? lckv::rope_apply_kernel<T, lckv::kRopeUnits, 4> : lckv::rope_apply_kernel<T, lckv::kRopeUnits, 1>;
    return hp == 4 ? lckv::rope_apply_kernel<T, lckv::kRopeAnySize, 4> : lckv::rope_apply_kernel<T, lckv::kRopeAnySize, 1>;
}

bool capturing(cudaStream_t st, int* rc)
{
    cudaStreamCaptureStatus cs = cudaStreamCaptureStatusNone;
    *rc = cuda_ok(cudaStreamIsCapturing(st, &cs)) ? LCKV_OK : LCKV_ECUDA;
    return cs != cudaStreamCaptureStatusNone;
}

// Does every sequence own pages for its next `extra` rows, on the device too?
bool pages_ready(const lckv_cache* c, int batch, int extra)
{
    if (!c->cfg.page_rows) return true;
    if (c->pt_dirty) return false;
    for (int b = 0; b < batch; ++b)
        if (((int64_t)c->n_pages_of[b] << c->page_shift) < (int64_t)c->h_lens[b] + extra) return false;
    return true;
}

int rope_into_cache(lckv_cache* c, int slot, const lckv_rope_t* rope, const void* q, int64_t q_stride, void* q_out,
                    const void* k, const void* v, int64_t kv_stride, int n, int batch, int advance_len, bool prompt,
                    cudaStream_t st)
{
    if (!c || batch < 1 || batch > c->cfg.max_batch || n < 1) return LCKV_EINVAL;
    if (slot < 0 || slot >= c->plan.n_slots) return LCKV_EINVAL;
    if (k && c->cfg.kv_bits == 4) return LCKV_EINVAL;       // (rotate, then lckv_append_kv)
    if ((q == nullptr) != (q_out == nullptr) || (k == nullptr) != (v == nullptr) || (!q && !k)) return LCKV_EINVAL;
    if (advance_len && !k) return LCKV_EINVAL;
    const int d = c->cfg.head_dim, hq = q ? c->cfg.n_q_heads : 0, hkv = k ? c->cfg.n_kv_heads : 0;
    lckv::RopeAppendParams p;
    if (int rc = rope_args(rope, d, &p.r)) return rc;
    const int64_t tokens = (int64_t)batch * n;
    if (tokens >= (1ll << 31)) return LCKV_EINVAL;
    if (q_stride == 0) q_stride = (int64_t)hq * d;
    if (kv_stride == 0) kv_stride = (int64_t)hkv * d;
    if (q && q_stride < (int64_t)hq * d) return LCKV_EINVAL;
    if (k && kv_stride < (int64_t)hkv * d) return LCKV_EINVAL;
    if (!aligned(q, 2) || !aligned(q_out, 2) || !aligned(k, 2) || !aligned(v, 2)) return LCKV_EINVAL;
    if (q) {
        // q_out may be q itself (contiguous), else it lies apart from everything that is read
        const int64_t out_bytes = tokens * hq * d * 2, q_bytes = ((tokens - 1) * q_stride + (int64_t)hq * d) * 2;
        const int64_t kv_bytes = k ? ((tokens - 1) * kv_stride + (int64_t)hkv * d) * 2 : 0;
        if (!(q_out == q && q_stride == (int64_t)hq * d) && ranges_meet(q_out, out_bytes, q, q_bytes)) return LCKV_EINVAL;
        if (rope_tables_meet(rope, q_out, out_bytes)) return LCKV_EINVAL;
        if (k && (ranges_meet(q_out, out_bytes, k, kv_bytes) || ranges_meet(q_out, out_bytes, v, kv_bytes)))
            return LCKV_EINVAL;
    }
    int64_t longest = 0;
    for (int b = 0; b < batch; ++b) longest = std::max<int64_t>(longest, c->h_lens[b]);
    if (prompt) {
        if (int rc = prefill_check(c, n, batch, false)) return rc;
        if (longest > rope->positions) return LCKV_EINVAL;
    } else {
        if (longest + n > rope->positions) return LCKV_EINVAL;
        if (c->cfg.stream_sink > 0) {
            // no two tokens of one call may share a row of the ring
            if (k && n > c->cfg.max_seq - c->cfg.stream_sink) return LCKV_EINVAL;
        } else if (k && longest + n > c->cfg.max_seq) {      // (a query alone needs a position, not a row)
            return LCKV_ECAPACITY;
        }
    }
    int rc = LCKV_OK;
    const int extra = prompt || !k ? 0 : n;
    if (capturing(st, &rc) && (advance_len || (k && !pages_ready(c, batch, extra)))) return LCKV_EINVAL;
    if (rc) return rc;
    int sms = c->sm_count;
    if (k) {
        if (int rc2 = ensure_pages(c, batch, extra)) return rc2;
        if (int rc2 = sync_page_table(c, st)) return rc2;
    }
    p.q = static_cast<const uint16_t*>(q);
    p.q_out = static_cast<uint16_t*>(q_out);
    p.k = static_cast<const uint16_t*>(k);
    p.v = static_cast<const uint16_t*>(v);
    p.K = slot_k(c, slot);
    p.V = slot_v(c, slot);
    p.lens = c->d_lens;
    p.page_table = c->d_pt;
    p.status = c->d_status;
    p.q_tok = q_stride;
    p.kv_tok = kv_stride;
    p.T_cap = c->cfg.max_seq;
    p.batch = batch;
    p.n_new = n;
    p.hq = hq;
    p.hkv = hkv;
    p.d = d;
    p.n_sink = c->cfg.stream_sink;
    p.pt_stride = c->pt_stride;
    p.page_shift = c->page_shift;
    p.prompt = prompt ? 1 : 0;
    const bool vec = aligned(q, 16) && aligned(q_out, 16) && aligned(k, 16) && aligned(v, 16) && q_stride % 8 == 0 && kv_stride % 8 == 0;
    const int path = !vec ? lckv::kRopePairs : rope_tables_vector(rope) ? lckv::kRopeUnits : lckv::kRopeAnySize;
    const int heads = hq + 2 * hkv;
    const int hp = vec && rope_many(tokens * heads * (d / 16), sms) ? 4 : 1;
    p.hp = rope_heads(path, hp, tokens, heads, d, sms);
    dim3 block;
    const dim3 grid = rope_grid(tokens, heads, d, path, p.hp, &p.g, &block);
    const auto kernel = path == lckv::kRopePairs   ? lckv::rope_append_kernel<lckv::kRopePairs, 1>
                        : path == lckv::kRopeUnits ? (hp == 4 ? lckv::rope_append_kernel<lckv::kRopeUnits, 4> : lckv::rope_append_kernel<lckv::kRopeUnits, 1>)
                                                   : (hp == 4 ? lckv::rope_append_kernel<lckv::kRopeAnySize, 4> : lckv::rope_append_kernel<lckv::kRopeAnySize, 1>);
    const cudaError_t e = launch_pdl_dims(kernel, grid, block, 0, st, p);
    if (!cuda_ok(e)) return LCKV_ECUDA;
    if (advance_len) {
        if (int rc2 = launch_advance(c, batch, st, n)) return rc2;
        mirror_advance(c, batch, n);
    }
    return LCKV_OK;
}

// Tokens and heads at their strides: does no element lie in two places of the tensor?
bool rope_layout_ok(int64_t tok, int64_t head, int64_t tokens, int64_t heads, int64_t d)
{
    if (tok < 0 || head < 0) return false;
    if (heads > 1 && head < d) return false;
    if (tokens > 1 && tok < d) return false;
    if (tokens == 1 || heads == 1) return true;
    return tok >= (heads - 1) * head + d || head >= (tokens - 1) * tok + d;
}

}  // namespace

namespace {

// Threads of a row of n_vec vectors at nv vectors each: 8, 16 or 32 lanes of a warp, or whole warps.  With a scale per 128
// columns at least the 16 lanes that hold one such block.
int norm_threads(int n_vec, int nv, bool blocks)
{
    const int t = (n_vec + nv - 1) / nv;
    return t <= 8 && !blocks ? 8 : t <= 16 ? 16 : (t + 31) / 32 * 32;
}

struct NormShape { int tpr, rpb, smem, sms; };

template <int NV, bool EDGES, int X32, int RES, int OUT>
cudaError_t norm_ring_launch(const lckv::NormParams& p, const NormShape& g, cudaStream_t st)
{
    const auto kernel = lckv::norm_ring_kernel<NV, EDGES, lckv::NormTypes<X32, RES, OUT>>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 224 * 1024);
    if (e != cudaSuccess) return e;
    int per_sm = 0;
    e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, g.tpr * g.rpb, g.smem);
    if (e != cudaSuccess) return e;
    const int64_t blocks = std::min<int64_t>((int64_t)g.sms * std::max(1, per_sm), ((int64_t)p.rows + g.rpb - 1) / g.rpb);
    return launch_pdl_dims(kernel, dim3((unsigned)blocks), dim3(g.tpr, g.rpb), g.smem, st, p);
}
template <int NV, bool EDGES, int X32, int RES>
cudaError_t norm_ring_out(const lckv::NormParams& p, const NormShape& g, cudaStream_t st)
{
    if constexpr (!EDGES)
        if (p.out == 2 && p.group) return norm_ring_launch<NV, EDGES, X32, RES, 3>(p, g, st);
    return p.out == 0   ? norm_ring_launch<NV, EDGES, X32, RES, 0>(p, g, st)
           : p.out == 1 ? norm_ring_launch<NV, EDGES, X32, RES, 1>(p, g, st)
                        : norm_ring_launch<NV, EDGES, X32, RES, 2>(p, g, st);
}
template <int NV, bool EDGES>
cudaError_t norm_ring(const lckv::NormParams& p, const NormShape& g, cudaStream_t st)
{
    if (p.x32)
        return !p.r ? norm_ring_out<NV, EDGES, 1, 0>(p, g, st) : !p.r32 ? norm_ring_out<NV, EDGES, 1, 1>(p, g, st) : norm_ring_out<NV, EDGES, 1, 2>(p, g, st);
    return !p.r ? norm_ring_out<NV, EDGES, 0, 0>(p, g, st) : !p.r32 ? norm_ring_out<NV, EDGES, 0, 1>(p, g, st) : norm_ring_out<NV, EDGES, 0, 2>(p, g, st);
}

// Vectors that a thread of the largest kernel holds: eight, of a row of up to 512 x 8.  A row of 32762 or more elements that shares its
// first and last vector with its neighbours can touch 4097.
constexpr int kNormMostVectors = 8;
bool norm_row_fits(int n_vec) { return n_vec <= 512 * kNormMostVectors; }

// Few rows (up to one per SM): one vector per thread, the shortest chain.  More: the ring, two vectors per thread
// (a thread block of 256 threads serves a row of 4096), four where a row has more than 1024 vectors.  Not the ring
// where fp32 tensors make the bytes and not the instructions the bound and rows are short: 2^26 elements, ring / one row
// per thread block, us, with 512, 2048, 4096, 8192 columns: bf16 50 / 61, 45 / 65, 43 / 70, 45 / 77; bf16 + bf16 95 / 103,
// 98 / 104, 96 / 110, 96 / 116; bf16 + fp32 149 / 121, 150 / 125, 150 / 129, 150 / 133; fp32 to bf16 69 / 67, 68 / 71, 65 / 74,
// 61 / 80; bf16 + fp32 to e4m3 144 / 120, 138 / 126, 122 / 131, 135 / 138.  Few more rows than SMs, 150, 300, 512, 1024,
// 2048 of 4096: bf16 + bf16 2.5 / 2.8, 3.3 / 3.3, 3.6 / 3.6, 5.7 / 6.6, 9.6 / 13.9; to e4m3 by row 3.0 / 3.3, 4.2 / 4.1, 4.5 / 4.4, 7.6 / 7.5,
// 12.8 / 15.6; bf16 + fp32 to e4m3 3.4 / 3.9, 4.7 / 5.5, 5.6 / 5.9, 9.3 / 10.4, 15.5 / 19.4; of 6656: bf16 + bf16 3.1 / 3.3, 4.2 / 5.4, 5.3 / 6.7,
// 9.5 / 13.3, 16.4 / 26.1; to e4m3 by row 4.0 / 3.8, 5.5 / 6.2, 7.0 / 7.6, 12.9 / 15.6, 21.4 / 28.0.  Nor the ring with an eps of 0 (norm_factor).
cudaError_t norm_launch(const lckv::NormParams& p, int n_vec, bool edges, int sms, cudaStream_t st)
{
    const bool fp32 = p.x32 || (p.r && p.r32);
    const bool many = p.rows > sms;
    if (many && p.eps > 0.f && (!fp32 || edges || n_vec > 512 + 256 || (p.out == 2 && n_vec >= 512))) {
        const int nv = n_vec > 1024 ? 4 : 2;
        NormShape g;
        g.tpr = norm_threads(n_vec, nv, p.group != 0);
        g.rpb = g.tpr <= 32 ? 128 / g.tpr : 1;
        const int parts = (p.x32 ? 2 : 1) + (p.r ? (p.r32 ? 2 : 1) : 0);
        const int64_t smem = (int64_t)lckv::kNormRing * nv * parts * g.tpr * g.rpb * 16;
        g.smem = (int)smem;
        g.sms = sms;
        if (g.tpr <= 512 && smem <= 222 * 1024) {
            if (nv == 2) return edges ? norm_ring<2, true>(p, g, st) : norm_ring<2, false>(p, g, st);
            if (!edges) return norm_ring<4, false>(p, g, st);
        }
    }
    int nv = many && n_vec >= 64 ? 2 : 1;
    while ((n_vec + nv - 1) / nv > (nv == 1 ? 1024 : 512)) nv *= 2;
    if (nv > kNormMostVectors) return cudaErrorInvalidValue;         // (the caller sends no such row here)
    const int tpr = norm_threads(n_vec, nv, p.group != 0), rpb = tpr <= 32 ? 128 / tpr : 1;
    const auto kernel = !edges ? (nv == 1   ? lckv::norm_vec_kernel<1, 1024, false>
                                  : nv == 2 ? lckv::norm_vec_kernel<2, 512, false> : nv == 4 ? lckv::norm_vec_kernel<4, 512, false> : lckv::norm_vec_kernel<8, 512, false>)
                               : (nv == 1   ? lckv::norm_vec_kernel<1, 1024, true>
                                  : nv == 2 ? lckv::norm_vec_kernel<2, 512, true> : nv == 4 ? lckv::norm_vec_kernel<4, 512, true> : lckv::norm_vec_kernel<8, 512, true>);
    return launch_pdl_dims(kernel, dim3((unsigned)((p.rows + rpb - 1) / rpb)), dim3(tpr, rpb), 0, st, p);
}

}  // namespace

extern "C" {

int lckv_rope_tables(float* cos, float* sin, int32_t positions, int32_t rot_dim, const lckv_rope_scaling_t* s, void* stream)
{
    if (!cos || !sin || !s || s->struct_size != sizeof(lckv_rope_scaling_t)) return LCKV_EINVAL;
    if (positions < 1 || rot_dim < 2 || (rot_dim & 1) || rot_dim > 2 * lckv::kRopeMaxPairs) return LCKV_EINVAL;
    if (!aligned(cos, 4) || !aligned(sin, 4)) return LCKV_EINVAL;
    const int half = rot_dim / 2;
    const int64_t n = (int64_t)positions * half;
    if (ranges_meet(cos, n * 4, sin, n * 4)) return LCKV_EINVAL;
    if (s->kind < 0 || s->kind > 3) return LCKV_EINVAL;
    if (!(s->base > 1.0) || !std::isfinite(s->base)) return LCKV_EINVAL;
    const double amplitude = s->amplitude == 0.0 ? 1.0 : s->amplitude;
    if (!std::isfinite((float)amplitude)) return LCKV_EINVAL;
    if (s->kind != 0 && (!(s->factor > 0.0) || !std::isfinite(s->factor))) return LCKV_EINVAL;
    if (s->kind == 3 && (!(s->original > 0.0) || !std::isfinite(s->original) || !(s->low >= 0.0) || !(s->high > s->low) ||
                         !std::isfinite(s->high)))
        return LCKV_EINVAL;
    const double two_pi = 6.283185307179586476925286766559;
    lckv::RopeTableParams p;
    const double base = s->kind == 2 && rot_dim > 2 ? s->base * std::pow(s->factor, (double)rot_dim / (rot_dim - 2.0)) : s->base;
    if (!std::isfinite(base)) return LCKV_EINVAL;              // (an infinite base would make every frequency but the first 0)
    for (int i = 0; i < half; ++i) {
        double theta = std::pow(base, -2.0 * i / rot_dim);
        if (s->kind == 1) theta /= s->factor;
        if (s->kind == 3) {
            double keep = (s->original * theta / two_pi - s->low) / (s->high - s->low);
            keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
            theta *= keep + (1.0 - keep) / s->factor;
        }
        double turns = theta / two_pi;
        if (!std::isfinite(turns)) return LCKV_EINVAL;       // a factor so small that base or frequency leave fp64
        turns -= std::floor(turns);
        p.turns[i] = (uint64_t)std::ldexp(turns, 64);        // (turns < 1: at most 2^64 - 2^11)
    }
    p.cos = cos;
    p.sin = sin;
    p.n = n;
    p.half = half;
    p.amplitude = (float)amplitude;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool vec = half % 4 == 0 && aligned(cos, 16) && aligned(sin, 16);
    // four positions per thread where that leaves enough threads (one fetch of the frequencies serves them all)
    const int v = vec ? 4 : 1, many = positions >= 4096 ? 4 : 1;
    p.step = ((int64_t)positions + many - 1) / many * (half / v);
    const dim3 grid((unsigned)((p.step + lckv::kRopeThreads - 1) / lckv::kRopeThreads)), block(lckv::kRopeThreads);
    const cudaError_t e = vec ? (many == 4 ? launch_pdl_dims(lckv::rope_table_kernel<4, 4>, grid, block, 0, st, p)
                                           : launch_pdl_dims(lckv::rope_table_kernel<4, 1>, grid, block, 0, st, p))
                              : (many == 4 ? launch_pdl_dims(lckv::rope_table_kernel<1, 4>, grid, block, 0, st, p)
                                           : launch_pdl_dims(lckv::rope_table_kernel<1, 1>, grid, block, 0, st, p));
    return cuda_ok(e) ? LCKV_OK : LCKV_ECUDA;
}

int lckv_rope_apply(const lckv_rope_t* rope, const int32_t* positions, const void* x, int64_t x_token_stride,
                    int64_t x_head_stride, void* y, int64_t y_token_stride, int64_t y_head_stride, int32_t n_tokens,
                    int32_t n_heads, int32_t head_dim, int32_t dtype, int32_t transpose, void* stream)
{
    if (!positions || !x || !y || n_tokens < 1 || n_heads < 1 || n_heads > 65536) return LCKV_EINVAL;
    if (head_dim != 64 && head_dim != 128) return LCKV_EINVAL;
    if ((dtype != 0 && dtype != 1) || (transpose != 0 && transpose != 1)) return LCKV_EINVAL;
    lckv::RopeApplyParams p;
    if (int rc = rope_args(rope, head_dim, &p.r)) return rc;
    const int size = dtype ? 4 : 2;
    if (!aligned(x, size) || !aligned(y, size) || !aligned(positions, 4)) return LCKV_EINVAL;
    if (x_token_stride < 0 || x_head_stride < 0) return LCKV_EINVAL;      // (0: one token or head, read many times)
    if (!rope_layout_ok(y_token_stride, y_head_stride, n_tokens, n_heads, head_dim)) return LCKV_EINVAL;
    const int64_t last = (int64_t)n_tokens - 1, top = (int64_t)n_heads - 1;
    const int64_t x_span = last * x_token_stride + top * x_head_stride + head_dim;
    const int64_t y_span = last * y_token_stride + top * y_head_stride + head_dim;
    if (ranges_meet(x, x_span * size, y, y_span * size)) {
        // one buffer: in place, or other heads of the same tokens
        const bool same = (x_token_stride == y_token_stride || last == 0) && (x_head_stride == y_head_stride || top == 0);
        const int64_t apart = std::abs((int64_t)((intptr_t)y - (intptr_t)x)) / size, row = top * y_head_stride + head_dim;
        if (!same || !(apart == 0 || (apart >= row && apart + row <= y_token_stride))) return LCKV_EINVAL;
    }
    if (rope_tables_meet(rope, y, y_span * size) || ranges_meet(y, y_span * size, positions, (int64_t)n_tokens * 4)) return LCKV_EINVAL;
    p.r.sgn = transpose ? -1.f : 1.f;
    p.pos = positions;
    p.x = x;
    p.y = y;
    p.x_tok = x_token_stride;
    p.x_head = x_head_stride;
    p.y_tok = y_token_stride;
    p.y_head = y_head_stride;
    p.tokens = n_tokens;
    p.heads = n_heads;
    p.d = head_dim;
    int sms = 0;
    if (int rc = device_sm_count(&sms)) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int64_t grain = 16 / size;
    const bool vec = aligned(x, 16) && aligned(y, 16) && x_token_stride % grain == 0 && x_head_stride % grain == 0 &&
                     y_token_stride % grain == 0 && y_head_stride % grain == 0;
    const int path = !vec ? lckv::kRopePairs : rope_tables_vector(rope) ? lckv::kRopeUnits : lckv::kRopeAnySize;
    const int hp = vec && rope_many((int64_t)n_tokens * n_heads * (head_dim / 16), sms) ? 4 : 1;
    p.hp = rope_heads(path, hp, n_tokens, n_heads, head_dim, sms);
    dim3 block;
    const dim3 grid = rope_grid(n_tokens, n_heads, head_dim, path, p.hp, &p.g, &block);
    const cudaError_t e = launch_pdl_dims(dtype ? rope_apply_variant<float>(path, hp) : rope_apply_variant<uint16_t>(path, hp), grid, block, 0, st, p);
    return cuda_ok(e) ? LCKV_OK : LCKV_ECUDA;
}

int lckv_rope_append_kv(lckv_cache_t* c, int32_t slot, const lckv_rope_t* rope, const void* q, int64_t q_stride, void* q_out,
                        const void* k_new, const void* v_new, int64_t kv_stride, int32_t n_new, int32_t batch,
                        int32_t advance_len, void* stream)
{
    return rope_into_cache(c, slot, rope, q, q_stride, q_out, k_new, v_new, kv_stride, n_new, batch, advance_len, false,
                           static_cast<cudaStream_t>(stream));
}

int lckv_rope_prefill_write_kv(lckv_cache_t* c, int32_t slot, const lckv_rope_t* rope, const void* q, int64_t q_stride,
                               void* q_out, const void* k, const void* v, int64_t kv_stride, int32_t n_max, int32_t batch,
                               void* stream)
{
    return rope_into_cache(c, slot, rope, q, q_stride, q_out, k, v, kv_stride, n_max, batch, 0, true,
                           static_cast<cudaStream_t>(stream));
}

int lckv_rms_norm(const void* x, int64_t x_stride, int32_t x_dtype, const void* residual, void* residual_out,
                  int32_t residual_dtype, const void* weight, int32_t weight_dtype, void* y, int32_t y_kind, float* y_scale,
                  int32_t scale_group, int32_t rows, int32_t width, float eps, void* stream)
{
    if (!x || !weight || !y || rows < 1 || width < 1 || width > lckv::kNormMaxWidth) return LCKV_EINVAL;
    if ((x_dtype | residual_dtype | weight_dtype) & ~1) return LCKV_EINVAL;
    if (y_kind < 0 || y_kind > 2 || (y_kind == 2) != (y_scale != nullptr)) return LCKV_EINVAL;
    if (scale_group != 0 && !(scale_group == 128 && y_kind == 2)) return LCKV_EINVAL;
    if (residual_out && !residual) return LCKV_EINVAL;
    if (!(eps >= 0.f) || !std::isfinite(eps)) return LCKV_EINVAL;
    if (x_stride == 0) x_stride = width;
    if (x_stride < width) return LCKV_EINVAL;
    const int xs = x_dtype ? 4 : 2, rs = residual_dtype ? 4 : 2, ws = weight_dtype ? 4 : 2;
    const int ys = y_kind == 1 ? 4 : y_kind == 0 ? 2 : 1;
    if (!aligned(x, xs) || !aligned(residual, rs) || !aligned(residual_out, rs) || !aligned(weight, ws) || !aligned(y, ys) ||
        !aligned(y_scale, 4))
        return LCKV_EINVAL;
    const int n_groups = scale_group ? (width + 127) / 128 : 1;
    {
        // an output may take the place of an input of the same type and layout; else it lies apart
        const int64_t n = (int64_t)rows * width, x_bytes = ((int64_t)(rows - 1) * x_stride + width) * xs;
        struct Range { const void* p; int64_t bytes; int size; bool dense; };
        const Range in[3] = {{x, x_bytes, xs, x_stride == width}, {residual, residual ? n * rs : 0, rs, true}, {weight, (int64_t)width * ws, 0, false}};
        const Range out[3] = {{residual_out, residual_out ? n * rs : 0, rs, true}, {y, n * ys, ys, true},
                              {y_scale, y_scale ? (int64_t)rows * n_groups * 4 : 0, 0, false}};
        for (int o = 0; o < 3; ++o) {
            if (!out[o].bytes) continue;
            for (int i = 0; i < 3; ++i)
                if (in[i].bytes && ranges_meet(out[o].p, out[o].bytes, in[i].p, in[i].bytes) &&
                    !(out[o].p == in[i].p && out[o].size == in[i].size && out[o].dense && in[i].dense))
                    return LCKV_EINVAL;
            for (int j = 0; j < o; ++j)
                if (out[j].bytes && ranges_meet(out[o].p, out[o].bytes, out[j].p, out[j].bytes)) return LCKV_EINVAL;
        }
    }
    lckv::NormParams p;
    p.x = x;
    p.r = residual;
    p.h = residual_out;
    p.w = weight;
    p.y = y;
    p.scale = y_scale;
    p.x_stride = x_stride;
    p.rows = rows;
    p.width = width;
    p.eps = eps;
    p.x32 = x_dtype;
    p.r32 = residual_dtype;
    p.w32 = weight_dtype;
    p.out = y_kind;
    p.group = scale_group;
    p.n_groups = n_groups;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool grid16 = aligned(x, 16) && aligned(residual, 16) && aligned(residual_out, 16) && aligned(y, y_kind == 2 ? 8 : 16);
    const bool even = grid16 && width % 8 == 0 && x_stride % 8 == 0 && aligned(weight, 16);
    const int n_vec = (width + (even ? 7 : 14)) / 8;
    const bool edges = grid16 && !even && x_stride == width && !scale_group && norm_row_fits(n_vec);
    cudaError_t e;
    if (even || edges) {
        int sms = 0;
        if (int rc = device_sm_count(&sms)) return rc;
        e = norm_launch(p, n_vec, edges, sms, st);
    } else {
        const size_t smem = (size_t)width * 4;
        if (smem > 47 * 1024 &&      // (beside the static arrays)
            !cuda_ok(cudaFuncSetAttribute(lckv::norm_any_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, lckv::kNormMaxWidth * 4)))
            return LCKV_ECUDA;
        e = launch_pdl_dims(lckv::norm_any_kernel, dim3((unsigned)rows), dim3(256), smem, st, p);
    }
    return cuda_ok(e) ? LCKV_OK : LCKV_ECUDA;
}

}  // extern "C"

namespace {

std::atomic<int32_t> quant_w_limit{INT32_MAX}, quant_x_limit{INT32_MAX};        // lckv_quant_set_copy_limits

bool quant_shape_ok(int32_t n, int32_t k, int32_t group)
{
    return n >= 1 && k >= 1 && n <= (1 << 24) && k <= (1 << 24) && (group == 32 || group == 64 || group == 128) && k % group == 0;
}

// How a launch of thread blocks that each take `feat` features would share n_blocks x k_blocks blocks of weights: the
// cluster size with the shortest time, counted as rounds over the SMs times (one thread block's weights + what it takes to
// start, join and store, about as long as `fixed` blocks of weights).
struct QuantSplit { int ks; int64_t cost; };
QuantSplit quant_split(int64_t tiles, int k_blocks, int blocks_per_k, int fixed, int min_k, int64_t slots, int sms)
{
    QuantSplit best = {1, INT64_MAX};
    for (int ks = 1; ks <= 8; ++ks) {
        if (ks > 1 && (ks * min_k > k_blocks || (slots && tiles * ks > slots))) break;
        const int64_t cost = ((tiles * ks + sms - 1) / sms) * ((int64_t)((k_blocks + ks - 1) / ks) * blocks_per_k + fixed);
        if (cost < best.cost) best = {ks, cost};
    }
    return best;
}

template <bool F8, bool ZEROS, int GROUP, int FT, int NT>
cudaError_t launch_quant_mma(lckv::QuantParams& p, int ks, cudaStream_t st)
{
    constexpr int scales = lckv::kQuantK / GROUP * lckv::kQuantFeat * 2;
    constexpr int block = lckv::kQuantCodes + scales + (ZEROS ? scales / 2 : 0);
    constexpr int smem = lckv::quant_warps(NT) * lckv::quant_slots(FT) * (FT / 2) * block;
    const cudaError_t e = cudaFuncSetAttribute(lckv::quant_mma_kernel<F8, ZEROS, GROUP, FT, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    p.k_split = ks;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((p.n + 16 * FT - 1) / (16 * FT), (p.m + 8 * NT - 1) / (8 * NT), ks);
    cfg.blockDim = dim3(lckv::quant_warps(NT) * 32);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = 1;
    at[0].val.clusterDim.y = 1;
    at[0].val.clusterDim.z = ks;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, lckv::quant_mma_kernel<F8, ZEROS, GROUP, FT, NT>, p);
}

// Tensor map of x as boxes of 128 bytes x box_rows rows, 128-byte swizzle, zeros outside.
int quant_x_map(CUtensorMap* tm, const lckv::QuantParams& p, bool f8, int box_rows)
{
    if (!f8) return make_tensor_map_pitch(tm, const_cast<void*>(p.x), (uint64_t)p.m, (uint64_t)p.k, (uint64_t)p.x_stride * 2, box_rows);
    return make_tensor_map_typed(tm, CU_TENSOR_MAP_DATA_TYPE_UINT8, 128, const_cast<void*>(p.x), (uint64_t)p.m, (uint64_t)p.k,
                                 (uint64_t)p.x_stride, box_rows);
}

template <bool F8, bool ZEROS, int GROUP, int NBMAX>
int launch_quant_tc5(const lckv::QuantParams& q, int sms, int32_t* status, cudaStream_t st)
{
    lckv::Quant5Params p;
    p.w = q.w;
    p.x_scale = q.x_scale;
    p.y = q.y;
    p.status = status;
    p.y_stride = q.y_stride;
    p.m = q.m;
    p.n = q.n;
    p.k = q.k;
    p.n_blocks = q.n_blocks;
    p.k_blocks = q.k_blocks;
    p.x_blocks = q.x_blocks;
    p.y32 = q.y32;
    p.y_vec = q.y_stride % 4 == 0 && aligned(q.y, q.y32 ? 16 : 8);
    // equal tiles of rows when the batch needs several
    const int m_tiles = (q.m + NBMAX - 1) / NBMAX;
    p.NB = ((q.m + m_tiles - 1) / m_tiles + 15) / 16 * 16;
    const int block = lckv::q5_block(GROUP, ZEROS);
    p.stages = (220 * 1024 - (F8 ? lckv::kQ5XScales : 0)) / lckv::q5_stage_bytes(p.NB, F8, block);
    p.stages = std::min(p.stages, lckv::kQ5MaxStages);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((p.n_blocks + 3) / 4, m_tiles);
    const int64_t tiles = (int64_t)cfg.gridDim.x * m_tiles;
    const int ks = quant_split(tiles, p.k_blocks, 1, 10, 4, 0, sms).ks;        // one thread block per SM
    p.k_split = ks;
    p.w_limit = quant_w_limit.load(std::memory_order_relaxed);
    p.x_limit = quant_x_limit.load(std::memory_order_relaxed);
    CUtensorMap tm;
    if (int rc = quant_x_map(&tm, q, F8, p.NB)) return rc;
    const int smem = lckv::q5_smem_bytes(p.NB, F8, block, p.stages);
    auto kernel = lckv::quant_tc5_kernel<F8, ZEROS, GROUP, NBMAX>;
    if (!cuda_ok(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024))) return LCKV_ECUDA;
    cfg.gridDim.z = ks;
    cfg.blockDim = dim3(lckv::q5_threads(NBMAX, F8));
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = 1;
    at[0].val.clusterDim.y = 1;
    at[0].val.clusterDim.z = ks;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    return cuda_ok(cudaLaunchKernelEx(&cfg, kernel, p, tm)) ? LCKV_OK : LCKV_ECUDA;
}

// Up to 16 rows: mma.sync kernel, 8 rows a tile; a warp takes 32 or 64 features, whichever the count above says shares out
// better (measured at 1 row, k = 4096: 4096 features 4.4 / 4.8 us, 12288 7.5 / 8.6 us, 22016 12.4 / 13.4 us; the count takes 32 in the
// last two and 64 in the first, which was the faster one, 5.5 / 4.6, while a tile of ones corrected for zero points), 64 for two
// tiles of rows, where x costs as much to fetch as the weights (16 rows, 22016 features: 22.3 / 16.6 us).  Beyond, the tcgen05 kernel
// (mma.sync / tcgen05, 4096 features: 16 rows 6.8 / 7.9 us, 32 rows 10.2 / 8.6; 22016 features: 16 rows 16.3 / 29.2, 32 rows 27.0 / 30.6).
template <bool F8, bool ZEROS, int GROUP>
int launch_quant_rows(lckv::QuantParams& p, int sms, int32_t* status, cudaStream_t st)
{
    if (p.m > 16)
        return p.m <= 32 ? launch_quant_tc5<F8, ZEROS, GROUP, 32>(p, sms, status, st)
                         : launch_quant_tc5<F8, ZEROS, GROUP, 128>(p, sms, status, st);
    const int64_t tiles2 = (p.n + 31) / 32, tiles4 = (p.n + 63) / 64;
    cudaError_t e;
    if (p.m > 8) {
        const QuantSplit s = quant_split(tiles4, p.k_blocks, 4, 8, lckv::quant_warps(2), (int64_t)lckv::quant_ctas(4, 2) * sms, sms);
        e = launch_quant_mma<F8, ZEROS, GROUP, 4, 2>(p, s.ks, st);
    } else {
        const QuantSplit s2 = quant_split(tiles2, p.k_blocks, 2, 8, lckv::quant_warps(1), (int64_t)lckv::quant_ctas(2, 1) * sms, sms);
        const QuantSplit s4 = quant_split(tiles4, p.k_blocks, 4, 8, lckv::quant_warps(1), (int64_t)lckv::quant_ctas(4, 1) * sms, sms);
        e = s4.cost <= s2.cost ? launch_quant_mma<F8, ZEROS, GROUP, 4, 1>(p, s4.ks, st)
                               : launch_quant_mma<F8, ZEROS, GROUP, 2, 1>(p, s2.ks, st);
    }
    return cuda_ok(e) ? LCKV_OK : LCKV_ECUDA;
}

template <bool F8, bool ZEROS>
int launch_quant_group(lckv::QuantParams& p, int sms, int32_t* status, cudaStream_t st)
{
    return p.group == 32   ? launch_quant_rows<F8, ZEROS, 32>(p, sms, status, st)
           : p.group == 64 ? launch_quant_rows<F8, ZEROS, 64>(p, sms, status, st)
                           : launch_quant_rows<F8, ZEROS, 128>(p, sms, status, st);
}

}  // namespace

extern "C" {

size_t lckv_quant_bytes(int32_t n, int32_t k, int32_t group, int32_t has_zeros)
{
    if (!quant_shape_ok(n, k, group) || (has_zeros != 0 && has_zeros != 1)) return 0;
    return (size_t)lckv::quant_layout(n, k, group, has_zeros != 0).total;
}

int lckv_quant_pack(const void* codes, const void* scales, const void* zeros, int32_t n, int32_t k, int32_t group, void* packed,
                    size_t packed_bytes, void* stream)
{
    if (!codes || !scales || !packed || !quant_shape_ok(n, k, group)) return LCKV_EINVAL;
    if (!aligned(scales, 2)) return LCKV_EINVAL;
    const lckv::QuantLayout y = lckv::quant_layout(n, k, group, zeros != nullptr);
    if (!aligned(packed, 256) || packed_bytes < (size_t)y.total) return LCKV_ENOMEM;
    const int64_t src = (int64_t)n * (k / group);
    if (ranges_meet(packed, y.total, codes, (int64_t)n * (k / 2)) || ranges_meet(packed, y.total, scales, src * 2) ||
        (zeros && ranges_meet(packed, y.total, zeros, src)))
        return LCKV_EINVAL;
    lckv::QuantPackParams p;
    p.codes = static_cast<const uint8_t*>(codes);
    p.scales = static_cast<const uint16_t*>(scales);
    p.zeros = static_cast<const uint8_t*>(zeros);
    p.out = static_cast<uint8_t*>(packed);
    p.n = n;
    p.k = k;
    p.group = group;
    int sms = 0;
    if (int rc = device_sm_count(&sms)) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    int rc = LCKV_OK;
    if (capturing(st, &rc)) return LCKV_EINVAL;
    if (rc) return rc;
    if (zeros) {
        // a zero point above 15 has no place in the layout; the packed weight's first word serves as the flag until it is written
        int32_t* flag = reinterpret_cast<int32_t*>(packed);
        int32_t bad = 0;
        if (!cuda_ok(cudaMemsetAsync(flag, 0, 4, st))) return LCKV_ECUDA;
        lckv::quant_zeros_kernel<<<sms, 256, 0, st>>>(p.zeros, src, flag);
        if (!cuda_ok(cudaGetLastError())) return LCKV_ECUDA;
        if (!cuda_ok(cudaMemcpyAsync(&bad, flag, 4, cudaMemcpyDeviceToHost, st)) || !cuda_ok(cudaStreamSynchronize(st))) return LCKV_ECUDA;
        if (bad) return LCKV_EINVAL;
    }
    lckv::quant_pack_kernel<<<sms * 8, 256, 0, st>>>(p);
    if (!cuda_ok(cudaGetLastError())) return LCKV_ECUDA;
    // lckv_quant_linear requests weights before the kernel in front of it has ended: they are complete from here on
    return cuda_ok(cudaStreamSynchronize(st)) ? LCKV_OK : LCKV_ECUDA;
}

int lckv_quant_linear(const void* packed, int32_t n, int32_t k, int32_t group, int32_t has_zeros, const void* x, int64_t x_stride,
                      int32_t x_kind, const float* x_scale, int32_t x_scale_group, void* y, int64_t y_stride, int32_t y_dtype,
                      int32_t rows, int32_t* dev_status, void* stream)
{
    if (!packed || !x || !y || !quant_shape_ok(n, k, group) || (has_zeros != 0 && has_zeros != 1)) return LCKV_EINVAL;
    if (rows < 1 || rows > (1 << 19)) return LCKV_EINVAL;
    if (x_kind < 0 || x_kind > 1 || y_dtype < 0 || y_dtype > 1) return LCKV_EINVAL;
    if ((x_kind == 1) != (x_scale != nullptr)) return LCKV_EINVAL;
    if (x_scale_group != 0 && !(x_kind == 1 && x_scale_group == 128)) return LCKV_EINVAL;
    if (x_stride == 0) x_stride = k;
    if (y_stride == 0) y_stride = n;
    if (x_stride < k || y_stride < n) return LCKV_EINVAL;
    const int xs = x_kind ? 1 : 2, ys = y_dtype ? 4 : 2;
    if (!aligned(packed, 256) || !aligned(x, 16) || (x_stride * xs) % 16 || !aligned(y, ys) || !aligned(x_scale, 4) || !aligned(dev_status, 4)) return LCKV_EINVAL;
    const lckv::QuantLayout lay = lckv::quant_layout(n, k, group, has_zeros != 0);
    const int64_t y_bytes = ((int64_t)(rows - 1) * y_stride + n) * ys;
    const int64_t n_scales = (int64_t)rows * (x_scale_group ? (k + 127) / 128 : 1);
    if (ranges_meet(y, y_bytes, x, ((int64_t)(rows - 1) * x_stride + k) * xs) || ranges_meet(y, y_bytes, packed, lay.total) ||
        (x_scale && ranges_meet(y, y_bytes, x_scale, n_scales * 4)) || (dev_status && ranges_meet(y, y_bytes, dev_status, 4)))
        return LCKV_EINVAL;
    lckv::QuantParams p;
    p.w = static_cast<const uint8_t*>(packed);
    p.x = x;
    p.x_scale = x_scale;
    p.y = y;
    p.x_stride = x_stride;
    p.y_stride = y_stride;
    p.m = rows;
    p.n = n;
    p.k = k;
    p.group = group;
    p.n_blocks = lay.n_blocks;
    p.k_blocks = lay.k_blocks;
    p.x_blocks = x_scale_group ? (k + 127) / 128 : 0;
    p.y32 = y_dtype;
    int sms = 0;
    if (int rc = device_sm_count(&sms)) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return x_kind ? (has_zeros ? launch_quant_group<true, true>(p, sms, dev_status, st) : launch_quant_group<true, false>(p, sms, dev_status, st))
                  : (has_zeros ? launch_quant_group<false, true>(p, sms, dev_status, st) : launch_quant_group<false, false>(p, sms, dev_status, st));
}

int lckv_quant_set_copy_limits(int32_t weights, int32_t x)
{
    if (weights < -1 || x < -1) return LCKV_EINVAL;
    quant_w_limit.store(weights < 0 ? INT32_MAX : weights, std::memory_order_relaxed);
    quant_x_limit.store(x < 0 ? INT32_MAX : x, std::memory_order_relaxed);
    return LCKV_OK;
}

}  // extern "C"
