// C-ABI host side of the paged cache: argument validation and launches of pec_qk_norm_rope, pec_paged_append and
// pec_attn_paged.  Part of pec_attn.hip.
#pragma once

namespace {

// Elements between tokens, from an argument that may be 0 for packed; negative: not one.
int64_t token_stride(int64_t stride, int heads) {
    const int64_t packed = (int64_t)heads * kHeadDim;
    if (stride == 0) return packed;
    return stride >= packed && stride % 8 == 0 && stride <= ((int64_t)1 << 25) ? stride : -1;
}

int check_cache(const pec_shape_t* s, const pec_paged_cache_t* c, PagedKv* out) {
    if (!c || !c->k || !c->v || c->n_pages <= 0 || c->page_size <= 0 || c->reserved != 0) return PEC_ERR_INVALID_ARGUMENT;
    if (c->page_size < 8 || (c->page_size & (c->page_size - 1)) != 0 || c->n_pages > 0x7fffffff) return PEC_ERR_UNSUPPORTED;
    if (misaligned(c->k) || misaligned(c->v) || ((c->page_stride | c->row_stride | c->head_stride) & 7)) return PEC_ERR_MISALIGNED;
    const int64_t most = (int64_t)1 << 30;      // elements inside a page, 2^31 bytes
    if (c->row_stride < kHeadDim || c->row_stride > most || (s->n_kv_heads > 1 && (c->head_stride < kHeadDim || c->head_stride > most)) ||
        c->page_stride < 0 || c->page_stride > ((int64_t)1 << 45) || (c->n_pages > 1 && c->page_stride < kHeadDim))
        return PEC_ERR_INVALID_ARGUMENT;
    const int64_t head_stride = s->n_kv_heads > 1 ? c->head_stride : 0;
    if ((c->page_size - 1) * c->row_stride + (s->n_kv_heads - 1) * head_stride + kHeadDim > most) return PEC_ERR_UNSUPPORTED;
    out->k = static_cast<unsigned char*>(c->k);
    out->v = static_cast<unsigned char*>(c->v);
    out->page_b = c->page_stride * 2;
    out->row_b = (uint32_t)(c->row_stride * 2);
    out->head_b = (uint32_t)(head_stride * 2);
    out->last_page = (uint32_t)(c->n_pages - 1);
    out->log_page = 0;
    while ((1 << out->log_page) < c->page_size) ++out->log_page;
    return PEC_OK;
}

int check_batch(const pec_paged_batch_t* b, int page_size, PagedBatch* out) {
    if (!b || b->batch < 0 || b->total_q < 0 || b->table_len < 0 || b->max_len_q < 0 || b->max_len_k < 0) return PEC_ERR_INVALID_ARGUMENT;
    if (b->total_q > kMaxRows) return PEC_ERR_UNSUPPORTED;
    if (b->batch > 0 && b->total_q > 0) {
        if (!b->cu_seqlens_q || !b->seqlens_k || (b->table_len > 0 && !b->block_table)) return PEC_ERR_INVALID_ARGUMENT;
        if ((reinterpret_cast<uintptr_t>(b->cu_seqlens_q) | reinterpret_cast<uintptr_t>(b->seqlens_k) |
             reinterpret_cast<uintptr_t>(b->block_table)) & 3u)
            return PEC_ERR_MISALIGNED;
    }
    out->cu_q = b->cu_seqlens_q;
    out->len_k = b->seqlens_k;
    out->table = b->block_table;
    out->batch = b->batch;
    out->table_len = b->table_len;
    out->total_q = (int32_t)b->total_q;
    out->max_keys = (int32_t)std::min<int64_t>((int64_t)b->table_len * page_size, kMaxRows);
    return PEC_OK;
}

// Workspace of pec_attn_paged.  Partial results (O and LSE of so many rows) of paged_step_kernel's spans, two slots each, or of
// fwd_il_kernel's items, 256 rows each -- the two run one after the other; the steps ahead of every sequence; the work list.
struct PagedLayout {
    int log_heads, bm, units;            // of a work list's items
    int64_t capacity, slots;
    size_t off_lse, off_prefix, off_work, off_counters, off_splits, bytes;
};
constexpr int64_t kPagedSlabs = 1024;    // items' partial results: four for every compute unit
PagedLayout paged_layout(int cu, const pec_shape_t* shape, int32_t batch, int64_t total_q) {
    auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
    PagedLayout l;
    l.log_heads = most_log_heads_per_item(shape->n_q_heads, shape->n_kv_heads);
    l.bm = kBM >> l.log_heads;
    l.units = shape->n_q_heads >> l.log_heads;
    const bool list = total_q * (shape->n_q_heads / shape->n_kv_heads) > kPagedFewRows;
    l.slots = list ? kPagedSlabs / l.units : 0;
    l.capacity = list ? total_q / l.bm + batch + l.slots : 0;
    const size_t rows = std::max((size_t)cu * kPagedWaves1 * 2 * 32, (size_t)l.slots * l.units * kBM);
    l.off_lse = rows * kHeadDim * sizeof(float);
    l.off_prefix = up(l.off_lse + rows * sizeof(float));
    l.off_work = up(l.off_prefix + ((size_t)batch + 2) * sizeof(int32_t));
    l.off_counters = up(l.off_work + (size_t)l.capacity * sizeof(WorkItem));
    l.off_splits = l.off_counters + 256;
    l.bytes = up(l.off_splits + (size_t)(l.slots / 2 + 1) * sizeof(PagedSplit));
    return l;
}

int check_norm_rope(const pec_norm_rope_t* n, NormRopeParams* p) {
    if (!n) return PEC_OK;      // nothing is done to the rows
    if (!(n->eps >= 0.f) || n->n_positions < 0 || n->rotary_dim < 0 || n->reserved != 0) return PEC_ERR_INVALID_ARGUMENT;
    if (n->rotary_dim % 16 != 0 || n->rotary_dim > kHeadDim || n->n_positions > kMaxRows) return PEC_ERR_UNSUPPORTED;
    if (n->rotary_dim > 0 && (!n->cos_sin || n->n_positions == 0)) return PEC_ERR_INVALID_ARGUMENT;
    if (((reinterpret_cast<uintptr_t>(n->q_weight) | reinterpret_cast<uintptr_t>(n->k_weight)) & 3u) || misaligned(n->cos_sin))
        return PEC_ERR_MISALIGNED;
    p->q_weight = n->q_weight;
    p->k_weight = n->k_weight;
    p->table = n->cos_sin;
    p->n_positions = (int32_t)n->n_positions;
    p->rotary = n->rotary_dim;
    p->interleaved = n->interleaved != 0;
    p->eps = n->eps;
    return PEC_OK;
}

template <bool NORM, bool APPEND>
void launch_norm_rope(const NormRopeParams& p, dim3 grid, hipStream_t st) {
    const dim3 threads(kNormRopeThreads);
    if (p.rotary == 0)
        hipLaunchKernelGGL((norm_rope_kernel<NORM, kPairsNone, APPEND>), grid, threads, 0, st, p);
    else if (p.interleaved)
        hipLaunchKernelGGL((norm_rope_kernel<NORM, kPairsNext, APPEND>), grid, threads, 0, st, p);
    else if (p.rotary == kHeadDim)
        hipLaunchKernelGGL((norm_rope_kernel<NORM, kPairsFar, APPEND>), grid, threads, 0, st, p);
    else
        hipLaunchKernelGGL((norm_rope_kernel<NORM, kPairsHalf, APPEND>), grid, threads, 0, st, p);
}

int launch_norm_rope(NormRopeParams& p, bool append, hipStream_t st) {
    p.parts = norm_rope_parts(compute_units(), p.tokens, (p.n_q_heads + 3) / 4 + (append ? 2 : 1) * ((p.n_kv_heads + 3) / 4));
    const int64_t waves = (int64_t)p.tokens * p.parts;
    const int64_t blocks = (waves + kNormRopeThreads / 64 - 1) / (kNormRopeThreads / 64);
    const dim3 grid((unsigned)std::min<int64_t>(blocks, kNormRopeRow), (unsigned)((blocks + kNormRopeRow - 1) / kNormRopeRow));
    const bool norm = p.q_weight || p.k_weight;
    if (append && norm) launch_norm_rope<true, true>(p, grid, st);
    else if (append) launch_norm_rope<false, true>(p, grid, st);
    else if (norm) launch_norm_rope<true, false>(p, grid, st);
    else launch_norm_rope<false, false>(p, grid, st);
    return hipGetLastError() == hipSuccess ? PEC_OK : PEC_ERR_HIP;
}

}  // namespace

extern "C" {

int pec_qk_norm_rope(const pec_shape_t* shape, const pec_norm_rope_t* norm_rope, const void* q, int64_t q_stride, const void* k,
                     int64_t k_stride, const int32_t* positions, int64_t pos0, int64_t tokens, void* q_out, void* k_out,
                     void* stream) {
    if (int rc = check_shape(shape, nullptr)) return rc;
    if (shape->flags != 0) return PEC_ERR_UNSUPPORTED;
    NormRopeParams p{};
    if (!norm_rope || tokens < 0 || pos0 < 0) return PEC_ERR_INVALID_ARGUMENT;
    if (int rc = check_norm_rope(norm_rope, &p)) return rc;
    if (tokens > kMaxRows) return PEC_ERR_UNSUPPORTED;
    if (tokens == 0) return PEC_OK;
    if ((!q && !k) || (q && !q_out) || (k && !k_out)) return PEC_ERR_INVALID_ARGUMENT;
    if (!positions && p.rotary > 0 && pos0 > p.n_positions - tokens) return PEC_ERR_INVALID_ARGUMENT;
    p.q_stride = token_stride(q_stride, shape->n_q_heads);
    p.k_stride = token_stride(k_stride, shape->n_kv_heads);
    if ((q && p.q_stride < 0) || (k && p.k_stride < 0)) return PEC_ERR_INVALID_ARGUMENT;
    if (misaligned(q) || misaligned(k) || misaligned(q_out) || misaligned(k_out) || (reinterpret_cast<uintptr_t>(positions) & 3u))
        return PEC_ERR_MISALIGNED;
    p.q = static_cast<const __bf16*>(q);
    p.k = static_cast<const __bf16*>(k);
    p.q_out = static_cast<__bf16*>(q_out);
    p.k_out = static_cast<__bf16*>(k_out);
    p.positions = positions;
    p.pos0 = pos0;
    p.tokens = (int32_t)tokens;
    p.n_q_heads = q ? shape->n_q_heads : 0;
    p.n_kv_heads = k ? shape->n_kv_heads : 0;
    return launch_norm_rope(p, false, static_cast<hipStream_t>(stream));
}

int pec_paged_append(const pec_shape_t* shape, const pec_norm_rope_t* norm_rope, const pec_paged_cache_t* cache,
                     const pec_paged_batch_t* batch, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                     const void* v, int64_t v_stride, void* q_out, void* stream) {
    if (int rc = check_shape(shape, nullptr)) return rc;
    if (shape->flags != 0) return PEC_ERR_UNSUPPORTED;
    NormRopeParams p{};
    if (int rc = check_cache(shape, cache, &p.cache)) return rc;
    if (int rc = check_batch(batch, cache->page_size, &p.batch)) return rc;
    if (int rc = check_norm_rope(norm_rope, &p)) return rc;
    if (batch->batch == 0 || batch->total_q == 0) return PEC_OK;
    if (!k || !v || (q && !q_out)) return PEC_ERR_INVALID_ARGUMENT;
    p.q_stride = token_stride(q_stride, shape->n_q_heads);
    p.k_stride = token_stride(k_stride, shape->n_kv_heads);
    p.v_stride = token_stride(v_stride, shape->n_kv_heads);
    if ((q && p.q_stride < 0) || p.k_stride < 0 || p.v_stride < 0) return PEC_ERR_INVALID_ARGUMENT;
    if (misaligned(q) || misaligned(k) || misaligned(v) || misaligned(q_out)) return PEC_ERR_MISALIGNED;
    p.q = static_cast<const __bf16*>(q);
    p.k = static_cast<const __bf16*>(k);
    p.v = static_cast<const __bf16*>(v);
    p.q_out = static_cast<__bf16*>(q_out);
    p.tokens = (int32_t)batch->total_q;
    p.n_q_heads = q ? shape->n_q_heads : 0;
    p.n_kv_heads = shape->n_kv_heads;
    return launch_norm_rope(p, true, static_cast<hipStream_t>(stream));
}

size_t pec_paged_workspace_bytes(const pec_shape_t* shape, int32_t batch, int64_t total_q) {
    if (!shape || shape->n_q_heads <= 0 || shape->n_kv_heads <= 0 || batch < 0 || total_q < 0) return 0;
    if (shape->n_q_heads % shape->n_kv_heads != 0) return 0;
    return paged_layout(compute_units(), shape, batch, total_q).bytes;
}

int pec_attn_paged(const pec_shape_t* shape, const pec_paged_cache_t* cache, const pec_paged_batch_t* batch, const void* q,
                   int64_t q_stride, int causal, void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    float scale;
    if (int rc = check_shape(shape, &scale)) return rc;
    if (shape->flags & ~(uint32_t)PEC_FLAG_SIMPLE_KERNEL) return PEC_ERR_UNSUPPORTED;
    PagedAttnParams p{};
    if (int rc = check_cache(shape, cache, &p.cache)) return rc;
    if (int rc = check_batch(batch, cache->page_size, &p.batch)) return rc;
    if (batch->batch == 0 || batch->total_q == 0) return PEC_OK;
    if (!q || !out || !lse) return PEC_ERR_INVALID_ARGUMENT;
    p.q_stride = token_stride(q_stride, shape->n_q_heads);
    if (p.q_stride < 0) return PEC_ERR_INVALID_ARGUMENT;
    if (misaligned(q) || misaligned(out) || misaligned(workspace) || (reinterpret_cast<uintptr_t>(lse) & 3u)) return PEC_ERR_MISALIGNED;
    const bool simple = (shape->flags & PEC_FLAG_SIMPLE_KERNEL) != 0;
    if (!simple && (!workspace || workspace_bytes < pec_paged_workspace_bytes(shape, batch->batch, batch->total_q))) return PEC_ERR_WORKSPACE;
    p.q = static_cast<const __bf16*>(q);
    p.out = out;
    p.lse = lse;
    p.n_q_heads = shape->n_q_heads;
    p.n_kv_heads = shape->n_kv_heads;
    p.group = shape->n_q_heads / shape->n_kv_heads;
    p.causal = causal != 0;
    p.out_f32 = shape->out_dtype == PEC_F32;
    p.scale = scale;
    p.scale_log2 = scale * kLog2e;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (simple) {
        const int64_t rows = batch->total_q * shape->n_q_heads;
        hipLaunchKernelGGL(paged_simple_kernel, dim3((unsigned)std::min<int64_t>(rows, 1 << 20)), dim3(64), 0, st, p);
        return hipGetLastError() == hipSuccess ? PEC_OK : PEC_ERR_HIP;
    }
    if (batch->batch > kPagedChunks * 64) return PEC_ERR_UNSUPPORTED;
    const int cu = std::max(8, compute_units() & ~7), g = p.group;
    if (batch->total_q * g > 0x7fffffff - 64) return PEC_ERR_UNSUPPORTED;      // rows of a KV head
    const int64_t len_q = batch->max_len_q > 0 ? std::min(batch->max_len_q, batch->total_q) : batch->total_q;
    const PagedLayout l = paged_layout(compute_units(), shape, batch->batch, batch->total_q);
    char* const ws = static_cast<char*>(workspace);
    const int64_t len_k = batch->max_len_k > 0 ? std::min<int64_t>(batch->max_len_k, p.batch.max_keys) : p.batch.max_keys;
    const PagedCut cut = paged_cut(cu, p.n_q_heads, p.n_kv_heads, batch->batch, batch->total_q, len_q, len_k);

    if (cut.units) {
        PagedStepParams s{};
        s.a = p;
        s.cut = StepCut{fast_div(g), 5, p.causal, 0x7fffffff};
        const int64_t groups = (batch->total_q * g / 32 + batch->batch) * p.n_kv_heads;
        if (groups > 0x7fffff00) return PEC_ERR_UNSUPPORTED;
        const dim3 grid((unsigned)std::min<int64_t>((groups + 7) / 8 * 8, kUnitsRow), (unsigned)((groups + kUnitsRow - 1) / kUnitsRow));
        if (cut.unit_waves == 4)
            hipLaunchKernelGGL((paged_step_kernel<1, 4, 1, true>), grid, dim3(4 * 64), 0, st, s);
        else
            hipLaunchKernelGGL((paged_step_kernel<1, kPagedWaves1, 1, true>), grid, dim3(kPagedWaves1 * 64), 0, st, s);
        return hipGetLastError() == hipSuccess ? PEC_OK : PEC_ERR_HIP;
    }
    if (cut.steps) {
        PagedStepParams s{};
        s.a = p;
        s.part_out = reinterpret_cast<float*>(ws);
        s.part_lse = reinterpret_cast<float*>(ws + l.off_lse);
        s.prefix = reinterpret_cast<int32_t*>(ws + l.off_prefix);
        s.cut = StepCut{fast_div(g), cut.nt == 1 ? 5 : 6, p.causal, cut.list ? cut.few_rows : 0x7fffffff};
        const int waves = cu * (cut.nt == 1 ? kPagedWaves1 : kPagedWaves2);
        if (p.n_kv_heads > waves) return PEC_ERR_UNSUPPORTED;      // a wavefront for every KV head
        s.n_spans = fast_div(waves / p.n_kv_heads);
        s.kv_heads = fast_div(p.n_kv_heads);
        s.unit_rows = (int32_t)std::min<int64_t>(32 * cut.nt, len_q * g);
        // every tile step has a number
        const int64_t per_seq = (std::min<int64_t>(cut.list ? cut.few_rows : len_q * g, len_q * g) + 32 * cut.nt - 1) / (32 * cut.nt);
        const int64_t row_tiles = cut.list ? batch->batch * per_seq : batch->total_q * g / (32 * cut.nt) + batch->batch;
        if ((double)row_tiles * (p.batch.max_keys / kStepTile + 1) > 2147483647.0) return PEC_ERR_UNSUPPORTED;
        if (cut.nt == 1)
            hipLaunchKernelGGL((paged_step_kernel<1, kPagedWaves1, 1, false>), dim3(cu), dim3(kPagedWaves1 * 64), 0, st, s);
        else
            hipLaunchKernelGGL((paged_step_kernel<2, kPagedWaves2, 2, false>), dim3(cu), dim3(kPagedWaves2 * 64), 0, st, s);
        if (hipGetLastError() != hipSuccess) return PEC_ERR_HIP;
        // (beside a list most of these sequences are decode steps; the tokens of others are merged one after the other)
        const int tokens = cut.list ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>(len_q, 256));
        const int64_t rows = (int64_t)batch->batch * tokens, waves_wanted = (int64_t)cu * 8;
        const unsigned heads = (unsigned)shape->n_q_heads;
        // pieces of the longest unit, as far as the hints tell: a step each at most, and four times a sequence's share of the spans
        const int64_t pieces = std::min({len_k / kStepTile, (int64_t)s.n_spans.d, 4 * (int64_t)s.n_spans.d / batch->batch});
        if (rows * heads >= waves_wanted)
            hipLaunchKernelGGL(paged_merge_kernel<1>, dim3((unsigned)std::min<int64_t>((rows + 3) / 4, 1 << 16), heads), dim3(256), 0, st, s,
                               tokens);
        else if (pieces < 128 || rows * heads > 512)
            hipLaunchKernelGGL(paged_merge_kernel<4>, dim3((unsigned)rows, heads), dim3(256), 0, st, s, tokens);
        else
            hipLaunchKernelGGL(paged_merge_kernel<16>, dim3((unsigned)rows, heads), dim3(1024), 0, st, s, tokens);
        if (hipGetLastError() != hipSuccess) return PEC_ERR_HIP;
    }
    if (!cut.list) return PEC_OK;
    if (l.capacity * l.units > 0x7fffffff) return PEC_ERR_UNSUPPORTED;
    PagedListParams w{};
    w.batch = p.batch;
    w.bm = l.bm;
    w.log_bm = 8 - l.log_heads;
    w.group = g;
    w.units = l.units;
    w.causal = p.causal;
    w.few_rows = cut.steps ? cut.few_rows : 0;
    w.capacity = (int32_t)l.capacity;
    w.slot_capacity = (int32_t)l.slots;
    w.cu = cu;
    w.work = reinterpret_cast<WorkItem*>(ws + l.off_work);
    w.counters = reinterpret_cast<int32_t*>(ws + l.off_counters);
    w.splits = reinterpret_cast<PagedSplit*>(ws + l.off_splits);
    hipLaunchKernelGGL(paged_list_kernel, dim3(1), dim3(1024), 0, st, w);
    if (hipGetLastError() != hipSuccess) return PEC_ERR_HIP;
    FwdParams f{};
    f.q = p.q;
    f.k = reinterpret_cast<const __bf16*>(p.cache.k);
    f.v = reinterpret_cast<const __bf16*>(p.cache.v);
    f.out = out;
    f.lse = lse;
    f.lse_stride = batch->total_q;
    f.causal = p.causal;
    f.n_q_heads = p.n_q_heads;
    f.n_kv_heads = p.n_kv_heads;
    f.group = g;
    f.log_heads = l.log_heads;
    f.n_items = (int32_t)l.capacity;
    f.out_f32 = p.out_f32;
    f.scale_log2 = p.scale_log2;
    f.work = w.work;
    f.n_work = w.counters;
    f.sched = w.counters + 8;
    f.q_row_stride = p.q_stride;
    f.part_out = reinterpret_cast<float*>(ws);
    f.part_lse = reinterpret_cast<float*>(ws + l.off_lse);
    f.table = p.batch.table_len > 0 ? p.batch.table : p.batch.cu_q;      // (a word to look at where there is no page: no key is in it)
    f.table_len = p.batch.table_len;
    f.page_b = p.cache.page_b;
    f.row_b = p.cache.row_b;
    f.head_b = p.cache.head_b;
    f.last_page = p.cache.last_page;
    f.log_page = p.cache.log_page;
    const int64_t groups = std::min<int64_t>(cu, (l.capacity * l.units + 7) / 8 * 8);
    hipLaunchKernelGGL(fwd_il_kernel<kFwdPaged>, dim3((unsigned)groups), dim3(512), 0, st, f);
    if (hipGetLastError() != hipSuccess) return PEC_ERR_HIP;
    if (l.slots > 1) {
        hipLaunchKernelGGL(paged_ranges_merge_kernel, dim3((unsigned)std::min<int64_t>(l.slots / 2 * l.units * 32, 4 * cu)), dim3(256), 0, st, w,
                           f.part_out, f.part_lse, l.log_heads, p.n_q_heads, p.out_f32, out, lse);
        if (hipGetLastError() != hipSuccess) return PEC_ERR_HIP;
    }
    return PEC_OK;
}

}  // extern "C"
