// C entry points of compact caches: reading rows back, gathered attention weights, eviction.  Included at the end of
// lckv_api.cu (they share its cache object and helpers).
#pragma once

namespace {

// Rows that an eviction leaves sequence b with.
struct RowsKept {
    const lckv_cache* src;
    int n_keep;
    int operator()(int b) const { return std::min(src->h_lens[b], n_keep); }
};

// Does every sequence b < batch own pages for its first rows(b) rows, on the device too?
bool pages_cover(const lckv_cache* c, const RowsKept& rows, int batch)
{
    if (!c->cfg.page_rows) return true;
    if (c->pt_dirty) return false;
    for (int b = 0; b < batch; ++b)
        if (((int64_t)c->n_pages_of[b] << c->page_shift) < rows(b)) return false;
    return true;
}

// Pages for the first rows(b) rows of every sequence; on exhaustion nothing changes.
int cover_pages(lckv_cache* c, const RowsKept& rows, int batch)
{
    if (!c->cfg.page_rows) return LCKV_OK;
    size_t need = 0;
    for (int b = 0; b < batch; ++b)
        need += (size_t)std::max(0, ((rows(b) + c->cfg.page_rows - 1) >> c->page_shift) - c->n_pages_of[b]);
    if (need > c->free_pages.size()) return LCKV_ECAPACITY;
    for (int b = 0; b < batch; ++b)
        while (((int64_t)c->n_pages_of[b] << c->page_shift) < rows(b)) {
            c->h_pt[(size_t)b * c->pt_stride + c->n_pages_of[b]++] = c->free_pages.back();
            c->free_pages.pop_back();
            c->pt_dirty = true;
        }
    return LCKV_OK;
}

// Pages behind the first rows(b) rows go back to the pool (which held them all once, so it does not grow).
void release_pages(lckv_cache* c, const RowsKept& rows, int batch)
{
    if (!c->cfg.page_rows) return;
    for (int b = 0; b < batch; ++b)
        while (c->n_pages_of[b] > 0 && ((int64_t)(c->n_pages_of[b] - 1) << c->page_shift) >= rows(b)) {
            int32_t& e = c->h_pt[(size_t)b * c->pt_stride + --c->n_pages_of[b]];
            c->free_pages.push_back(e);
            e = -1;
            c->pt_dirty = true;
        }
}

template <int D, bool PACKED>
void (*read_variant(int dtype, bool four))(lckv::RowReadParams)
{
    if (four) return dtype ? lckv::row_read_kernel<D, PACKED, true, 4> : lckv::row_read_kernel<D, PACKED, false, 4>;
    return dtype ? lckv::row_read_kernel<D, PACKED, true, 1> : lckv::row_read_kernel<D, PACKED, false, 1>;
}

// Thread blocks for `units` pieces of every (sequence, kv head), `per` a block.
dim3 move_grid(int64_t heads, int64_t units, int64_t per) { return dim3((unsigned)heads, (unsigned)std::min<int64_t>(65535, (units + per - 1) / per)); }

template <int D, bool PACKED>
cudaError_t launch_move(const lckv::MoveParams& p, bool in_place, int64_t heads, cudaStream_t st)
{
    if (in_place) return launch_pdl_dims(lckv::evict_in_place_kernel<D, PACKED>, dim3((unsigned)heads), dim3(1024), 0, st, p);
    const int64_t units = (int64_t)((p.n_keep + lckv::kMoveRows - 1) / lckv::kMoveRows) * lckv::RowUnits<D, PACKED>::kUnits;
    const dim3 grid = move_grid(heads, units, lckv::kRowThreads);
    return launch_pdl_dims(lckv::evict_move_kernel<D, PACKED>, grid, dim3(lckv::kRowThreads), 0, st, p);
}

// The smallest thread block that holds the rows in registers.  148 heads, us, and with the next larger block: 1024 rows 6.1, 14.5; 4096 rows 14.7,
// 21.0; 8192 rows 25.5, 26.7; 16384 rows 29.9, 53.8 (the same order for 1 to 1184 heads).  A block that holds them, and one that reads
// the weights again in every round: 1500 rows 11.6, 14.4; 8192 rows 25.5, 44; 16384 rows 29.9, 78; 32768 rows 58, 152.
cudaError_t launch_select(const lckv::SelectParams& s, int64_t most, int64_t heads, cudaStream_t st)
{
    const dim3 grid((unsigned)heads);
    if (most <= 1024) return launch_pdl_dims(lckv::evict_select_kernel<128, 8>, grid, dim3(128), 0, st, s);
    if (most <= 4096) return launch_pdl_dims(lckv::evict_select_kernel<256, 16>, grid, dim3(256), 0, st, s);
    if (most <= 8192) return launch_pdl_dims(lckv::evict_select_kernel<512, 16>, grid, dim3(512), 0, st, s);
    if (most <= 16384) return launch_pdl_dims(lckv::evict_select_kernel<1024, 16>, grid, dim3(1024), 0, st, s);
    if (most <= 32768) return launch_pdl_dims(lckv::evict_select_kernel<1024, 32>, grid, dim3(1024), 0, st, s);
    return launch_pdl_dims(lckv::evict_select_kernel<1024, 0>, grid, dim3(1024), 0, st, s);
}

template <int D>
cudaError_t launch_weights(const lckv::WeightParams& p, const lckv::PackedParams* pp, int group, int64_t blocks, cudaStream_t st)
{
    if (!pp) {
        const auto kernel = group <= 2 ? lckv::attention_weights_kernel<D, 2> : group <= 4 ? lckv::attention_weights_kernel<D, 4> : lckv::attention_weights_kernel<D, 8>;
        return launch_pdl_dims(kernel, dim3((unsigned)blocks), dim3(32 * lckv::kWeightWarps), 0, st, p);
    }
    const auto kernel = group <= 2   ? lckv::attention_weights_packed_kernel<D, 2>
                        : group <= 4 ? lckv::attention_weights_packed_kernel<D, 4>
                                     : lckv::attention_weights_packed_kernel<D, 8>;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, lckv::weight_smem_bytes<D>());
    if (e != cudaSuccess) return e;
    return launch_pdl_dims(kernel, dim3((unsigned)blocks), dim3(32 * lckv::kWeightBlockWarps), lckv::weight_smem_bytes<D>(), st, p, *pp);
}

}  // namespace

extern "C" {

int lckv_cache_read_kv(lckv_cache_t* c, int32_t slot, void* k, void* v, int32_t dtype, int32_t n_max, int32_t batch, void* stream)
{
    if (!c || !k || !v || slot < 0 || slot >= c->plan.n_slots || (dtype != 0 && dtype != 1)) return LCKV_EINVAL;
    if (!aligned(k, 16) || !aligned(v, 16)) return LCKV_EINVAL;
    if (int rc = prefill_check(c, n_max, batch, false)) return rc;
    const int d = c->cfg.head_dim;
    const int64_t bytes = (int64_t)batch * n_max * c->cfg.n_kv_heads * d * (dtype ? 4 : 2);
    dim3 grid;
    const bool four = four_tokens(c, n_max, batch);
    if (ranges_meet(k, bytes, v, bytes) || ranges_meet(k, bytes, c->base, (int64_t)c->lay.total_bytes) ||
        ranges_meet(v, bytes, c->base, (int64_t)c->lay.total_bytes) || !row_grid(c, n_max, four ? 4 : 1, batch, &grid))
        return LCKV_EINVAL;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    int rc = LCKV_OK;
    const bool capture = capturing(st, &rc);
    if (rc) return rc;
    if (capture && !pages_ready(c, 0, 0)) return LCKV_EINVAL;      // (the rows' pages are there; is the table?)
    if (int rc2 = sync_page_table(c, st)) return rc2;
    lckv::RowReadParams p;
    p.s = packed_slot(c, slot);
    p.K = slot_k(c, slot);
    p.V = slot_v(c, slot);
    p.map = row_map(c);
    p.lens = c->d_lens;
    p.k = k;
    p.v = v;
    p.T_cap = c->cfg.max_seq;
    p.batch = batch;
    p.n = n_max;
    const bool packed = c->cfg.kv_bits == 4;
    const auto kernel = d == 128 ? (packed ? read_variant<128, true>(dtype, four) : read_variant<128, false>(dtype, four))
                                 : (packed ? read_variant<64, true>(dtype, four) : read_variant<64, false>(dtype, four));
    const cudaError_t e = launch_pdl_dims(kernel, grid, dim3(lckv::kRowThreads), 0, st, p);
    return cuda_ok(e) ? LCKV_OK : LCKV_ECUDA;
}

int lckv_attention_weights(lckv_cache_t* c, int32_t slot, int32_t mode, const void* q, const float* lse, const float* previous, float* weights,
                           int64_t stride, int32_t batch, void* stream)
{
    if (!c || !q || !lse || !weights || batch < 1 || batch > c->cfg.max_batch) return LCKV_EINVAL;
    if (slot < 0 || slot >= c->plan.n_slots) return LCKV_EINVAL;
    if (mode != LCKV_MODE_CONDENSED && mode != LCKV_MODE_STANDARD) return LCKV_EINVAL;
    if (stride == 0) stride = c->cfg.max_seq;
    if (stride < c->cfg.max_seq || !aligned(q, 16) || !aligned(lse, 4) || !aligned(previous, 4) || !aligned(weights, 4)) return LCKV_EINVAL;
    const int64_t rows = (int64_t)batch * c->cfg.n_kv_heads, heads = (int64_t)batch * c->cfg.n_q_heads;
    if (rows > INT32_MAX) return LCKV_EINVAL;
    const int64_t bytes = ((rows - 1) * stride + c->cfg.max_seq) * 4;
    if ((previous && previous != weights && ranges_meet(weights, bytes, previous, bytes)) || ranges_meet(weights, bytes, q, heads * c->cfg.head_dim * 2) ||
        ranges_meet(weights, bytes, lse, heads * 4) || ranges_meet(weights, bytes, c->base, (int64_t)c->lay.total_bytes))
        return LCKV_EINVAL;
    if (max_len(c, batch) + mode > c->cfg.max_seq) return LCKV_ECAPACITY;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    int rc = LCKV_OK;
    const bool capture = capturing(st, &rc);
    if (rc) return rc;
    if (capture && !pages_ready(c, batch, mode)) return LCKV_EINVAL;
    if (int rc2 = ensure_pages(c, batch, mode)) return rc2;
    if (int rc2 = sync_page_table(c, st)) return rc2;
    lckv::WeightParams p;
    p.s = packed_slot(c, slot);
    p.K = slot_k(c, slot);
    p.map = row_map(c);
    p.lens = c->d_lens;
    p.q = static_cast<const uint16_t*>(q);
    p.lse = lse;
    p.prev = previous;
    p.weights = weights;
    p.T_cap = c->cfg.max_seq;
    p.stride = stride;
    p.H_q = c->cfg.n_q_heads;
    p.mode = mode;
    p.scale_log2 = c->scale_log2;
    p.status = c->d_status;
    p.wait_limit = c->wait_limit;
    const bool wide = c->cfg.head_dim == 128;
    const int group = c->cfg.n_q_heads / c->cfg.n_kv_heads;
    if (c->cfg.kv_bits == 4) {
        lckv::PackedParams pp = {};
        pp.m.a.lens = c->d_lens;
        pp.m.a.T_cap = c->cfg.max_seq;
        pp.m.a.B = batch;
        pp.m.a.H_q = pp.m.a.H_kv = c->cfg.n_kv_heads;
        pp.m.a.mode = mode;
        pp.m.groups_per_kv = 1;
        packed_shares(pp, c->sm_count, c->sm_count * lckv::kWeightBlockWarps, lckv::kWeightBlockWarps);
        const cudaError_t e = wide ? launch_weights<128>(p, &pp, group, c->sm_count, st) : launch_weights<64>(p, &pp, group, c->sm_count, st);
        return cuda_ok(e) ? LCKV_OK : LCKV_ECUDA;
    }
    // Warps for the longest sequence that the host knows (one whose sequence turns out longer in a replay goes on behind the last run), of two
    // tiles of 64 rows where an SM has 64 or more: the second tile's keys are asked for while the first's are used, and the query is loaded once (64
    // tiles an SM of 16 kv heads of 128 32.5 us, with one a warp 34.1; 221 tiles 91.3, 98.5, with four 98.2).  With few, fewer warps are what
    // counts (7 tiles an SM 5.6 us, with one 4.2); from 24 to 60 both take the same within 5 %.
    int64_t longest = 1;
    for (int b = 0; b < batch; ++b) longest = std::max<int64_t>(longest, std::min(c->h_lens[b], c->cfg.max_seq - mode) + mode);
    const int64_t tiles = (longest + 63) / 64;
    p.run = tiles * rows >= 64 * (int64_t)c->sm_count ? 2 : 1;
    p.runs = (int)((tiles + p.run - 1) / p.run);
    p.heads = (int)rows;
    const int64_t blocks = ((int64_t)p.runs * rows + lckv::kWeightWarps - 1) / lckv::kWeightWarps;
    if (blocks > INT32_MAX) return LCKV_EINVAL;
    const cudaError_t e = wide ? launch_weights<128>(p, nullptr, group, blocks, st) : launch_weights<64>(p, nullptr, group, blocks, st);
    return cuda_ok(e) ? LCKV_OK : LCKV_ECUDA;
}

int lckv_evict_kv(lckv_cache_t* dst, int32_t dst_slot, const lckv_cache_t* src, int32_t src_slot, const float* weights, int64_t weights_stride,
                  float* weights_out, int64_t out_stride, int32_t* kept, int32_t n_sink, int32_t n_recent, int32_t n_keep, int32_t batch,
                  int32_t set_len, void* stream)
{
    if (!dst || !src || !kept || batch < 1 || batch > dst->cfg.max_batch || batch > src->cfg.max_batch) return LCKV_EINVAL;
    if (dst_slot < 0 || dst_slot >= dst->plan.n_slots || src_slot < 0 || src_slot >= src->plan.n_slots) return LCKV_EINVAL;
    const bool in_place = dst == src;
    if (in_place && dst_slot != src_slot) return LCKV_EINVAL;
    const int d = src->cfg.head_dim, hkv = src->cfg.n_kv_heads;
    if (dst->cfg.head_dim != d || dst->cfg.n_kv_heads != hkv || dst->cfg.stream_sink > 0 || src->cfg.stream_sink > 0) return LCKV_EINVAL;
    if (src->cfg.kv_bits == 4 && dst->cfg.kv_bits != 4) return LCKV_EINVAL;
    if (n_keep < 1 || n_keep > dst->cfg.max_seq || n_sink < 0 || n_recent < 0 || (int64_t)n_sink + n_recent > n_keep) return LCKV_EINVAL;
    if (weights_stride == 0) weights_stride = src->cfg.max_seq;
    if (out_stride == 0) out_stride = dst->cfg.max_seq;
    if (weights_stride < src->cfg.max_seq || out_stride < dst->cfg.max_seq) return LCKV_EINVAL;
    if (!aligned(weights, 4) || !aligned(weights_out, 4) || !aligned(kept, 4)) return LCKV_EINVAL;
    const int64_t rows = (int64_t)batch * hkv, items = rows * n_keep;
    if (rows > INT32_MAX || (int64_t)n_keep * (d / 4) > INT32_MAX) return LCKV_EINVAL;    // (units of a head are counted in 32 bits)
    const int64_t w_bytes = ((rows - 1) * weights_stride + src->cfg.max_seq) * 4, o_bytes = ((rows - 1) * out_stride + dst->cfg.max_seq) * 4;
    const bool same = weights_out && weights_out == weights && out_stride == weights_stride;
    if (weights && weights_out && !same && ranges_meet(weights, w_bytes, weights_out, o_bytes)) return LCKV_EINVAL;
    if ((weights && ranges_meet(kept, items * 4, weights, w_bytes)) || (weights_out && ranges_meet(kept, items * 4, weights_out, o_bytes))) return LCKV_EINVAL;
    for (const lckv_cache* c : {(const lckv_cache*)dst, src}) {
        const int64_t total = (int64_t)c->lay.total_bytes;
        if (ranges_meet(kept, items * 4, c->base, total) || (weights_out && ranges_meet(weights_out, o_bytes, c->base, total))) return LCKV_EINVAL;
    }
    const RowsKept rows_kept = {src, n_keep};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    int rc = LCKV_OK;
    const bool capture = capturing(st, &rc);
    if (rc) return rc;
    if (src->pt_dirty && !in_place) return LCKV_EINVAL;     // (no call has brought the source's pages to the device yet)
    if (capture && (set_len || !pages_cover(dst, rows_kept, batch))) return LCKV_EINVAL;
    if (int rc2 = cover_pages(dst, rows_kept, batch)) return rc2;
    if (int rc2 = sync_page_table(dst, st)) return rc2;

    lckv::SelectParams s;
    s.weights = weights;
    s.weights_out = weights_out;
    s.kept = kept;
    s.lens = src->d_lens;
    s.lens_out = set_len && !in_place ? dst->d_lens : nullptr;
    s.stride = weights_stride;
    s.out_stride = out_stride;
    s.T_cap = src->cfg.max_seq;
    s.H_kv = hkv;
    s.n_sink = n_sink;
    s.n_recent = n_recent;
    s.n_keep = n_keep;
    s.out_rows = dst->cfg.max_seq;
    // A replay may find any length up to the capacity; an eager call's are known.
    int64_t most = 1;
    for (int b = 0; b < batch; ++b) most = std::max<int64_t>(most, src->h_lens[b]);
    if (capture) most = src->cfg.max_seq;
    if (!cuda_ok(launch_select(s, most, rows, st))) return LCKV_ECUDA;

    lckv::MoveParams p;
    p.from = packed_slot(src, src_slot);
    p.to = packed_slot(dst, dst_slot);
    p.K = slot_k(src, src_slot);
    p.V = slot_v(src, src_slot);
    p.K_to = slot_k(dst, dst_slot);
    p.V_to = slot_v(dst, dst_slot);
    p.map = row_map(src);
    p.map_to = row_map(dst);
    p.kept = kept;
    p.lens = src->d_lens;
    p.lens_out = set_len && in_place ? dst->d_lens : nullptr;
    p.status = dst->d_status;
    p.T_cap = src->cfg.max_seq;
    p.n_keep = n_keep;
    cudaError_t e;
    if (src->cfg.kv_bits == 4) {
        e = d == 128 ? launch_move<128, true>(p, in_place, rows, st) : launch_move<64, true>(p, in_place, rows, st);
    } else if (dst->cfg.kv_bits == 4) {
        e = d == 128 ? launch_pdl_dims(lckv::evict_pack_kernel<128>, move_grid(rows, n_keep, lckv::rows_per_block<128>() * lckv::kPackRows), dim3(lckv::kRowThreads), 0, st, p)
                     : launch_pdl_dims(lckv::evict_pack_kernel<64>, move_grid(rows, n_keep, lckv::rows_per_block<64>() * lckv::kPackRows), dim3(lckv::kRowThreads), 0, st, p);
    } else {
        e = d == 128 ? launch_move<128, false>(p, in_place, rows, st) : launch_move<64, false>(p, in_place, rows, st);
    }
    if (!cuda_ok(e)) return LCKV_ECUDA;
    if (set_len) {
        for (int b = 0; b < batch; ++b) dst->h_lens[b] = rows_kept(b);
        release_pages(dst, rows_kept, batch);
        return sync_page_table(dst, st);    // (not capturing; behind the moves, which go by the table as it was)
    }
    return LCKV_OK;
}

}  // extern "C"
