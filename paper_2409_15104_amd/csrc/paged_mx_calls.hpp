// C-ABI host side of the paged cache in 4 bits: argument validation and launches of pec_paged_append_mx, pec_paged_read_mx and
// pec_attn_paged_mx.  Part of pec_attn.hip.
#pragma once

namespace {

int check_cache_mx(const pec_shape_t* s, const pec_paged_cache_mx_t* c, PagedMx* out) {
    if (!c || !c->k || !c->v || !c->k_scale || !c->v_scale || c->n_pages <= 0 || c->page_size <= 0 || c->reserved != 0)
        return PEC_ERR_INVALID_ARGUMENT;
    if (c->page_size < 8 || (c->page_size & (c->page_size - 1)) != 0 || c->n_pages > 0x7fffffff) return PEC_ERR_UNSUPPORTED;
    if (misaligned(c->k) || misaligned(c->v) || misaligned(c->k_scale) || misaligned(c->v_scale) ||
        ((c->page_stride | c->row_stride | c->head_stride) & 15) || ((c->scale_page_stride | c->scale_head_stride) & 7))
        return PEC_ERR_MISALIGNED;
    const int64_t most = (int64_t)1 << 31, most_page = (int64_t)1 << 46, scales = (int64_t)c->page_size * kMxGroups;      // bytes
    const bool heads = s->n_kv_heads > 1, pages = c->n_pages > 1;
    if (c->row_stride < kMxRowBytes || c->row_stride > most || (heads && (c->head_stride < kMxRowBytes || c->head_stride > most)) ||
        (heads && (c->scale_head_stride < scales || c->scale_head_stride > most)) || c->page_stride < 0 || c->page_stride > most_page ||
        c->scale_page_stride < 0 || c->scale_page_stride > most_page || (pages && (c->page_stride < kMxRowBytes || c->scale_page_stride < scales)))
        return PEC_ERR_INVALID_ARGUMENT;
    const int64_t head_stride = heads ? c->head_stride : 0, scale_head_stride = heads ? c->scale_head_stride : 0;
    if ((c->page_size - 1) * c->row_stride + (s->n_kv_heads - 1) * head_stride + kMxRowBytes > most - 16 ||
        (s->n_kv_heads - 1) * scale_head_stride + scales > most - 16)
        return PEC_ERR_UNSUPPORTED;
    out->k = static_cast<unsigned char*>(c->k);
    out->v = static_cast<unsigned char*>(c->v);
    out->ks = static_cast<unsigned char*>(c->k_scale);
    out->vs = static_cast<unsigned char*>(c->v_scale);
    out->page_b = c->page_stride;
    out->scale_page_b = c->scale_page_stride;
    out->row_b = (uint32_t)c->row_stride;
    out->head_b = (uint32_t)head_stride;
    out->scale_head_b = (uint32_t)scale_head_stride;
    out->last_page = (uint32_t)(c->n_pages - 1);
    out->log_page = 0;
    while ((1 << out->log_page) < c->page_size) ++out->log_page;
    return PEC_OK;
}

// Whether neighbouring heads' rows of a token are neighbours in memory: 64 bytes each, half a cache line.
bool mx_by_token(const PagedMx& mx) { return mx.head_b < mx.row_b; }
constexpr int kMxStepRows = kMxMostUnitRows;      // of a slot of a partial result, at most
// Spans of all KV heads: one for every wavefront of eight to a compute unit at most, and one for every head at least.
int mx_most_spans(int cu, int n_kv_heads) { return std::max((cu & ~7) * 8, (n_kv_heads + 63) / 64 * 64); }
// Workspace of pec_attn_paged_mx: pec_attn_paged's, then the area (paged_mx_area_kernel.hpp) of so many pages.
struct MxLayout {
    PagedLayout paged;
    size_t off_area, off_used, off_owner, off_table, off_k, off_v, bytes;
};
MxLayout mx_layout(const pec_shape_t* shape, int32_t batch, int64_t total_q, int64_t pages) {
    auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
    MxLayout l;
    l.paged = paged_layout(compute_units(), shape, batch, total_q, (size_t)mx_most_spans(std::max(8, compute_units()), shape->n_kv_heads) * 2 * kMxStepRows);
    l.off_area = up(l.paged.bytes);
    l.off_used = up(l.off_area + (size_t)batch * sizeof(int32_t));
    l.off_owner = l.off_used + 256;
    l.off_table = l.off_owner + (size_t)pages * sizeof(int32_t);
    l.off_k = up(l.off_table + (size_t)(pages + 1) * sizeof(int32_t));
    l.off_v = l.off_k + (size_t)pages * shape->n_kv_heads * kMxAreaHeadBytes;
    l.bytes = l.off_v + (size_t)pages * shape->n_kv_heads * kMxAreaHeadBytes;
    return l;
}
// Pages that a workspace of so many bytes, at least those of no page, has room for.
int64_t mx_area_pages(const pec_shape_t* shape, int32_t batch, int64_t total_q, size_t bytes) {
    const size_t none = mx_layout(shape, batch, total_q, 0).bytes, page = 2 * (size_t)shape->n_kv_heads * kMxAreaHeadBytes + 2 * sizeof(int32_t);
    int64_t pages = (int64_t)std::min<size_t>((bytes - none + 256) / page, 0x7fffffff);
    while (pages > 0 && mx_layout(shape, batch, total_q, pages).bytes > bytes) --pages;      // (what is rounded up: once or not at all)
    return pages;
}

// The sequences of the launch straight from their codes: units, or spans and their merge.
int mx_steps(const PagedAttnParams& p, const PagedMx& mx, const PagedLayout& l, int cu, const MxPlan& plan, int64_t len_q, int64_t len_k, char* ws,
             hipStream_t st) {
    using std::integral_constant;
    const int64_t batch = p.batch.batch, total_q = p.batch.total_q;
    const int g = p.group, nt = plan.nt;
    // units of a KV head at most: of all packed rows, or of sequences that this launch is for
    int64_t row_tiles = total_q * g / (16 * nt) + batch;
    if (p.batch.most_q != 0) row_tiles = std::min(row_tiles, batch * (((int64_t)p.batch.most_q * g + 16 * nt - 1) / (16 * nt)));
    const bool small = mx.log_page < 4;
    PagedMxStepParams s{};
    s.a = p;
    s.cut = MxCut{fast_div(g), fast_div(16 * nt), p.causal};
    dim3 grid;
    // WAVES, HEADS: wavefronts to a span or unit, KV heads side by side in a workgroup (paged_mx_step_kernel)
    auto launch = [&](auto tiles, auto waves, auto heads, auto units, auto pages_of_eight) {
        constexpr int WAVES = decltype(waves)::value, HEADS = decltype(heads)::value;
        hipLaunchKernelGGL((paged_mx_step_kernel<decltype(tiles)::value, WAVES, HEADS, decltype(units)::value, decltype(pages_of_eight)::value>),
                           grid, dim3((unsigned)(HEADS * WAVES) * 64), 0, st, s, mx);
    };
    const integral_constant<int, 1> one{};
    const integral_constant<int, 2> two{};
    const integral_constant<int, 3> three{};
    const integral_constant<int, 4> four{};
    const integral_constant<int, 8> eight{};
    const std::true_type yes{};
    const std::false_type no{};
    if (plan.units && !small) {
        // two heads to a workgroup where they share cache lines (64 sequences of 510: 17.6 us with one, 11.7 with two)
        const int heads = nt == 1 && plan.waves == 4 && mx_by_token(mx) && p.n_kv_heads % 2 == 0 ? 2 : 1;
        s.kv_heads = fast_div(p.n_kv_heads / heads);
        const int64_t groups = row_tiles * s.kv_heads.d;
        if (groups > 0x7fffff00) return PEC_ERR_UNSUPPORTED;
        grid = dim3((unsigned)std::min<int64_t>((groups + 7) / 8 * 8, kUnitsRow), (unsigned)((groups + kUnitsRow - 1) / kUnitsRow));
        if (nt == 3) launch(three, four, one, yes, no);
        else if (nt == 2) launch(two, four, one, yes, no);
        else if (plan.waves == 8) launch(one, eight, one, yes, no);
        else if (heads == 2) launch(one, four, two, yes, no);
        else launch(one, four, one, yes, no);
        return hipGetLastError() == hipSuccess ? PEC_OK : PEC_ERR_HIP;
    }
    s.part_out = reinterpret_cast<float*>(ws);
    s.part_lse = reinterpret_cast<float*>(ws + l.off_lse);
    s.prefix = reinterpret_cast<int32_t*>(ws + l.off_prefix);
    // Single row tiles, by token: eight heads side by side, a wavefront for each one's span, so that whole token rows are read by one compute
    // unit at one time (4 x 110,000 tokens, 64 / 8 heads: 106 us, with the heads apart 118 ... 124); else four wavefronts to a
    // span and two workgroups to a compute unit (the same by heads: 85).
    const bool side_by_side = nt == 1 && !small && mx_by_token(mx) && p.n_kv_heads % 8 == 0;
    const int heads = side_by_side ? 8 : 1, lines = p.n_kv_heads / heads;
    const int groups = std::max(side_by_side ? cu : 2 * cu, (p.n_kv_heads + 63) / 64 * 64 / heads);
    s.n_spans = fast_div(groups / lines);
    s.kv_heads = fast_div(lines);
    s.unit_rows = (int32_t)std::min<int64_t>(16 * nt, len_q * g);
    if ((double)row_tiles * (p.batch.max_keys / kStepTile + 1) > 2147483647.0) return PEC_ERR_UNSUPPORTED;      // every tile step has a number
    grid = dim3((unsigned)groups);
    if (side_by_side) launch(one, one, eight, no, no);
    else if (small && nt == 1) launch(one, four, one, no, yes);
    else if (small && nt == 2) launch(two, four, one, no, yes);
    else if (small) launch(three, four, one, no, yes);
    else if (nt == 1) launch(one, four, one, no, no);
    else if (nt == 2) launch(two, four, one, no, no);
    else launch(three, four, one, no, no);
    if (hipGetLastError() != hipSuccess) return PEC_ERR_HIP;
    launch_paged_merge(s, cu, (int)std::max<int64_t>(1, std::min<int64_t>(len_q, 256)), len_k, st);
    return hipGetLastError() == hipSuccess ? PEC_OK : PEC_ERR_HIP;
}

}  // namespace

extern "C" {

int pec_paged_append_mx(const pec_shape_t* shape, const pec_norm_rope_t* norm_rope, const pec_paged_cache_mx_t* cache,
                        const pec_paged_batch_t* batch, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                        const void* v, int64_t v_stride, void* q_out, void* stream) {
    if (int rc = check_shape(shape, nullptr)) return rc;
    if (shape->flags != 0) return PEC_ERR_UNSUPPORTED;
    NormRopeParams p{};
    PagedMx c;
    if (int rc = check_cache_mx(shape, cache, &c)) return rc;
    p.cache.k = c.k;
    p.cache.v = c.v;
    p.cache.page_b = c.page_b;
    p.cache.row_b = c.row_b;
    p.cache.head_b = c.head_b;
    p.cache.last_page = c.last_page;
    p.cache.log_page = c.log_page;
    p.k_scale = c.ks;
    p.v_scale = c.vs;
    p.scale_page_b = c.scale_page_b;
    p.scale_head_b = c.scale_head_b;
    return append_call(p, kToMxPages, cache->page_size, shape, norm_rope, batch, q, q_stride, k, k_stride, v, v_stride, q_out, stream);
}

int pec_paged_read_mx(const pec_shape_t* shape, const pec_paged_cache_mx_t* cache, const pec_paged_batch_t* batch, void* k_out,
                      void* v_out, void* stream) {
    if (int rc = check_shape(shape, nullptr)) return rc;
    if (shape->flags != 0) return PEC_ERR_UNSUPPORTED;
    PagedMxReadParams p{};
    if (int rc = check_cache_mx(shape, cache, &p.cache)) return rc;
    if (int rc = check_batch(batch, cache->page_size, &p.batch)) return rc;
    if (batch->batch == 0 || batch->total_q == 0) return PEC_OK;
    if (!k_out || !v_out) return PEC_ERR_INVALID_ARGUMENT;
    if (misaligned(k_out) || misaligned(v_out)) return PEC_ERR_MISALIGNED;
    p.k_out = static_cast<__bf16*>(k_out);
    p.v_out = static_cast<__bf16*>(v_out);
    p.n_kv_heads = shape->n_kv_heads;
    const int64_t groups = (batch->total_q + 3) / 4;
    p.parts = norm_rope_parts(compute_units(), groups, 2 * (int64_t)p.n_kv_heads);
    const int64_t blocks = (groups * p.parts + 3) / 4;
    const dim3 grid((unsigned)std::min<int64_t>(blocks, kMxReadRow), (unsigned)((blocks + kMxReadRow - 1) / kMxReadRow));
    hipLaunchKernelGGL(paged_mx_read_kernel, grid, dim3(256), 0, static_cast<hipStream_t>(stream), p);
    return hipGetLastError() == hipSuccess ? PEC_OK : PEC_ERR_HIP;
}

size_t pec_paged_mx_workspace_bytes(const pec_shape_t* shape, int32_t batch, int64_t total_q, int64_t total_k) {
    if (!shape || shape->n_q_heads <= 0 || shape->n_kv_heads <= 0 || batch < 0 || total_q < 0 || total_k < 0) return 0;
    if (shape->n_q_heads % shape->n_kv_heads != 0) return 0;
    const int64_t pages = total_k > 0 ? std::min<int64_t>(total_k / kMxAreaPage + batch, 0x7fffffff) : 0;      // (a sequence's last page is in part its own)
    return mx_layout(shape, batch, total_q, pages).bytes;
}

int pec_attn_paged_mx(const pec_shape_t* shape, const pec_paged_cache_mx_t* cache, const pec_paged_batch_t* batch, const void* q,
                      int64_t q_stride, int causal, void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    float scale;
    if (int rc = check_shape(shape, &scale)) return rc;
    if (shape->flags & ~(uint32_t)PEC_FLAG_SIMPLE_KERNEL) return PEC_ERR_UNSUPPORTED;
    PagedAttnParams p{};
    PagedMx mx;
    if (int rc = check_cache_mx(shape, cache, &mx)) return rc;
    if (int rc = check_batch(batch, cache->page_size, &p.batch)) return rc;
    if (batch->batch == 0 || batch->total_q == 0) return PEC_OK;
    if (!q || !out || !lse) return PEC_ERR_INVALID_ARGUMENT;
    p.q_stride = token_stride(q_stride, shape->n_q_heads);
    if (p.q_stride < 0) return PEC_ERR_INVALID_ARGUMENT;
    if (misaligned(q) || misaligned(out) || misaligned(workspace) || (reinterpret_cast<uintptr_t>(lse) & 3u)) return PEC_ERR_MISALIGNED;
    const bool simple = (shape->flags & PEC_FLAG_SIMPLE_KERNEL) != 0;
    if (!simple && (!workspace || workspace_bytes < pec_paged_mx_workspace_bytes(shape, batch->batch, batch->total_q, 0))) return PEC_ERR_WORKSPACE;
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
        hipLaunchKernelGGL(paged_mx_simple_kernel, dim3((unsigned)std::min<int64_t>(rows, 1 << 20)), dim3(64), 0, st, p, mx);
        return hipGetLastError() == hipSuccess ? PEC_OK : PEC_ERR_HIP;
    }
    if (batch->batch > kPagedChunks * 64) return PEC_ERR_UNSUPPORTED;
    const int cu = std::max(8, compute_units() & ~7), g = p.group;
    if (batch->total_q * g > 0x7fffffff - 64) return PEC_ERR_UNSUPPORTED;      // rows of a KV head
    const int64_t len_q = batch->max_len_q > 0 ? std::min(batch->max_len_q, batch->total_q) : batch->total_q;
    const PagedLayout l = mx_layout(shape, batch->batch, batch->total_q, 0).paged;
    char* const ws = static_cast<char*>(workspace);
    const int64_t len_k = batch->max_len_k > 0 ? std::min<int64_t>(batch->max_len_k, p.batch.max_keys) : p.batch.max_keys;
    const bool may_list = l.capacity > 0 && l.capacity * l.units <= 0x7fffffff;      // (launch_paged_list's limit)
    const int64_t pages = may_list ? mx_area_pages(shape, batch->batch, batch->total_q, workspace_bytes) : 0;
    const MxCall call = mx_call(cu, p.n_q_heads, p.n_kv_heads, batch->batch, batch->total_q, batch->max_len_q, len_k, pages);
    int64_t most = batch->batch;      // sequences that the area may be for
    if (call.apart) {
        p.batch.least_q = 0;
        p.batch.most_q = call.few_q;
        if (int rc = mx_steps(p, mx, l, cu, call.few, call.few_q, len_k, ws, st)) return rc;
        p.batch.least_q = call.few_q + 1;
        p.batch.most_q = 0x7fffffff;
        most = std::min(most, batch->total_q / (call.few_q + 1));
    }
    // What finds no room in the area, if that can be, is left to the steps.
    const bool room = most * (((int64_t)p.batch.max_keys + kMxAreaPage - 1) / kMxAreaPage) <= pages;
    MxAreaParams a{};
    if (call.many.list) {
        const MxLayout m = mx_layout(shape, batch->batch, batch->total_q, pages);
        a.cache = mx;
        a.batch = p.batch;
        a.capacity = (int32_t)pages;
        a.n_kv_heads = p.n_kv_heads;
        a.area = reinterpret_cast<int32_t*>(ws + m.off_area);
        a.owner = reinterpret_cast<int32_t*>(ws + m.off_owner);
        a.table = reinterpret_cast<int32_t*>(ws + m.off_table);
        a.used = reinterpret_cast<int32_t*>(ws + m.off_used);
        a.k = reinterpret_cast<unsigned char*>(ws + m.off_k);
        a.v = reinterpret_cast<unsigned char*>(ws + m.off_v);
        hipLaunchKernelGGL(paged_mx_area_kernel, dim3(1), dim3(1024), 0, st, a);
        if (hipGetLastError() != hipSuccess) return PEC_ERR_HIP;
        p.batch.area = a.area;
    }
    if (!call.many.list || !room) {
        MxPlan plan = call.many;
        if (call.apart && plan.list) plan.units = true;      // (few sequences or none: 25 with a chunk among them 5 us, as spans and their merge 40)
        p.batch.area_side = 0;
        if (int rc = mx_steps(p, mx, l, cu, plan, len_q, len_k, ws, st)) return rc;
    }
    if (!call.many.list) return PEC_OK;
    const int64_t fill = std::min<int64_t>(pages * p.n_kv_heads, (int64_t)cu * 16);
    hipLaunchKernelGGL(paged_mx_fill_kernel, dim3((unsigned)fill), dim3(256), 0, st, a);
    if (hipGetLastError() != hipSuccess) return PEC_ERR_HIP;
    p.batch.area_side = 1;
    p.batch.table = a.table;
    p.batch.table_len = 1;
    p.cache.k = a.k;
    p.cache.v = a.v;
    p.cache.page_b = (int64_t)p.n_kv_heads * kMxAreaHeadBytes;
    p.cache.row_b = kRowBytes;
    p.cache.head_b = kMxAreaHeadBytes;
    p.cache.last_page = (uint32_t)(pages - 1);
    p.cache.log_page = 6;
    static_assert(kMxAreaPage == 64, "log_page");
    return launch_paged_list(p, l, cu, 0, ws, st);
}

}  // extern "C"
