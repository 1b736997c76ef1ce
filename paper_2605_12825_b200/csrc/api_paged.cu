// C-ABI entry points of the paged-cache calls and of the token sampler: argument validation and dispatch.
#include <cmath>
#include <cstdlib>
#include <cstring>
#include "paged.cuh"

namespace orthrus {
namespace {

bool aligned(const void *p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
bool page_size_ok(int32_t n) { return n >= 1 && n <= 1024 && (n & (n - 1)) == 0; }

orthrus_status_t check_workspace(const void *workspace, size_t bytes)      // of the calls that may do without one
{
    return workspace && (bytes < (size_t)kHeaderBytes || !aligned(workspace, 16)) ? ORTHRUS_ERR_WORKSPACE : ORTHRUS_OK;
}

// what the host can see of a layer; `attend`: for the attention calls
orthrus_status_t check_paged(const orthrus_paged_layer_t *L, bool attend)
{
    if (!L) return ORTHRUS_ERR_INVALID_ARG;
    if (L->batch < 1 || L->n_q_heads < 1 || L->n_kv_heads < 1 || L->block < 1 || L->max_pages < 1 || L->n_pages < 1 ||
        L->n_q_heads % L->n_kv_heads != 0 || L->max_len_hint < 0 || !(L->softmax_scale >= 0.f) || std::isinf(L->softmax_scale))
        return ORTHRUS_ERR_INVALID_ARG;
    if (L->flags & ~(uint32_t)(ORTHRUS_LAYER_CACHE_QUIESCENT | ORTHRUS_LAYER_NO_EARLY_LAUNCH)) return ORTHRUS_ERR_INVALID_ARG;
    if (L->dtype != ORTHRUS_BF16 && L->dtype != ORTHRUS_FP32) return ORTHRUS_ERR_UNSUPPORTED;
    if (L->head_dim != 32 && L->head_dim != 64 && L->head_dim != 128 && L->head_dim != 256) return ORTHRUS_ERR_UNSUPPORTED;
    if (!page_size_ok(L->page_size) || L->block > (attend ? 64 : 1 << 20) || L->n_q_heads > 65535) return ORTHRUS_ERR_UNSUPPORTED;
    // (a position and what a kernel adds to it to look ahead fit 31 bits)
    if ((long long)L->max_pages * L->page_size > 0x7fff0000LL || L->n_pages > 0x7fffffffLL) return ORTHRUS_ERR_UNSUPPORTED;
    if (attend && (L->batch > 16384 || (long long)L->batch * L->n_kv_heads > (1 << 24))) return ORTHRUS_ERR_UNSUPPORTED;
    if ((long long)L->batch * L->block > 0x7fffffffLL) return ORTHRUS_ERR_UNSUPPORTED;
    return ORTHRUS_OK;
}

orthrus_status_t check_pages(const orthrus_paged_layer_t *L)
{
    if (!L->k_pages || !L->v_pages || !aligned(L->k_pages, 16) || !aligned(L->v_pages, 16)) return ORTHRUS_ERR_INVALID_ARG;
    return ORTHRUS_OK;
}

// the tensor-core kernel, unless a path of the plain arithmetic is asked for (orthrus_set_path)
bool use_tc(const orthrus_paged_layer_t &L) { return paged_tc_shape(L) && !simt_forced(); }

orthrus_status_t attend(const orthrus_paged_layer_t *L, int causal, const void *q, void *out, void *ws, size_t ws_bytes, void *stream)
{
    orthrus_status_t st = check_paged(L, true);
    if (st == ORTHRUS_OK) st = check_pages(L);
    if (st != ORTHRUS_OK) return st;
    if (!q || !out || !ws || !L->block_table || !L->cache_len || !aligned(q, 16) || !aligned(out, 16) || !aligned(ws, 16) ||
        !aligned(L->block_table, 4) || !aligned(L->cache_len, 4) || !aligned(L->n_new, 4))
        return ORTHRUS_ERR_INVALID_ARG;
    const bool tc = use_tc(*L);
    if (!tc && !paged_simt_shape(*L)) return ORTHRUS_ERR_UNSUPPORTED;
    // (the larger of the two kernels', so that a workspace of the size that callers are told serves either)
    if (ws_bytes < orthrus_paged_attend_workspace_bytes(L)) return ORTHRUS_ERR_WORKSPACE;
    PagedParams p;
    p.q = q; p.k_pages = L->k_pages; p.v_pages = L->v_pages; p.table = L->block_table; p.cache_len = L->cache_len;
    p.n_new = L->n_new; p.out = out; p.status = static_cast<int32_t *>(ws);
    p.B = L->batch; p.K = L->block; p.Hq = L->n_q_heads; p.Hkv = L->n_kv_heads; p.G = p.Hq / p.Hkv; p.d = L->head_dim;
    p.page_shift = __builtin_ctz((unsigned)L->page_size); p.max_pages = L->max_pages; p.n_pages = L->n_pages;
    p.max_pos = L->max_pages * L->page_size;
    p.causal = causal;
    p.scale_log2 = (L->softmax_scale > 0.f ? L->softmax_scale : 1.f / sqrtf((float)p.d)) * 1.4426950408889634f;
    p.early = !(L->flags & ORTHRUS_LAYER_NO_EARLY_LAUNCH);
    p.quiescent = (L->flags & ORTHRUS_LAYER_CACHE_QUIESCENT) != 0;
    cudaStream_t cs = static_cast<cudaStream_t>(stream);
    set_last_path(tc ? "tcgen05" : "simt");
    const cudaError_t e = tc ? launch_paged_attend_tc(p, *L, static_cast<unsigned char *>(ws) + kHeaderBytes, cs)
                             : launch_paged_attend_simt(p, *L, static_cast<unsigned char *>(ws) + kHeaderBytes, cs);
    return e == cudaSuccess ? ORTHRUS_OK : ORTHRUS_ERR_CUDA;
}

}  // namespace
}  // namespace orthrus

using namespace orthrus;

extern "C" {

orthrus_status_t orthrus_page_tables(int32_t batch, int32_t page_size, int32_t n_pages, int32_t max_pages, int32_t max_new,
        const int32_t *cache_len, const int32_t *n_new, const int32_t *held_in, int32_t *held_out, int32_t *block_table,
        int32_t *free_list, const int32_t *n_free_in, int32_t *n_free_out, int32_t *granted, int64_t *slot_map,
        void *workspace, size_t workspace_bytes, void *stream)
{
    if (batch < 1 || n_pages < 1 || max_pages < 1 || max_new < 1) return ORTHRUS_ERR_INVALID_ARG;
    if (batch > 8192 || !page_size_ok(page_size) || max_new > (1 << 24)) return ORTHRUS_ERR_UNSUPPORTED;
    if ((long long)max_pages * page_size > 0x7fff0000LL) return ORTHRUS_ERR_UNSUPPORTED;
    const void *const all[] = {cache_len, n_new, held_in, held_out, block_table, free_list, n_free_in, n_free_out, granted};
    for (const void *x : all)
        if (!x || !aligned(x, 4)) return ORTHRUS_ERR_INVALID_ARG;
    if (!slot_map || !aligned(slot_map, 8)) return ORTHRUS_ERR_INVALID_ARG;
    const orthrus_status_t st = check_workspace(workspace, workspace_bytes);
    if (st != ORTHRUS_OK) return st;
    PageTablesParams p;
    p.B = batch; p.page_shift = __builtin_ctz((unsigned)page_size); p.n_pages = n_pages; p.max_pages = max_pages; p.max_new = max_new;
    p.cache_len = cache_len; p.n_new = n_new; p.held_in = held_in; p.held_out = held_out; p.table = block_table;
    p.free_list = free_list; p.n_free_in = n_free_in; p.n_free_out = n_free_out; p.granted = granted; p.slot_map = slot_map;
    p.status = static_cast<int32_t *>(workspace);
    return launch_page_tables(p, static_cast<cudaStream_t>(stream)) == cudaSuccess ? ORTHRUS_OK : ORTHRUS_ERR_CUDA;
}

orthrus_status_t orthrus_paged_kv_write(const orthrus_paged_layer_t *layer, const int64_t *slot_map, const void *k_blk,
        const void *v_blk, void *workspace, size_t workspace_bytes, void *stream)
{
    orthrus_status_t st = check_paged(layer, false);
    if (st == ORTHRUS_OK) st = check_pages(layer);
    if (st != ORTHRUS_OK) return st;
    if (!slot_map || !k_blk || !v_blk || !aligned(slot_map, 8) || !aligned(k_blk, 16) || !aligned(v_blk, 16)) return ORTHRUS_ERR_INVALID_ARG;
    if ((st = check_workspace(workspace, workspace_bytes)) != ORTHRUS_OK) return st;
    return launch_paged_kv_write(*layer, slot_map, nullptr, k_blk, v_blk, 1.0, nullptr, static_cast<int32_t *>(workspace),
                                 static_cast<cudaStream_t>(stream)) == cudaSuccess ? ORTHRUS_OK : ORTHRUS_ERR_CUDA;
}

orthrus_status_t orthrus_rope_paged_kv_write(const orthrus_paged_layer_t *layer, const int64_t *slot_map, const void *q,
        const void *k_blk, const void *v_blk, float rope_theta, void *q_out, void *workspace, size_t workspace_bytes,
        void *stream)
{
    orthrus_status_t st = check_paged(layer, false);
    if (st == ORTHRUS_OK) st = check_pages(layer);
    if (st != ORTHRUS_OK) return st;
    if (!slot_map || !q || !k_blk || !v_blk || !q_out || !layer->cache_len || !aligned(slot_map, 8) || !aligned(q, 16) ||
        !aligned(k_blk, 16) || !aligned(v_blk, 16) || !aligned(q_out, 16) || !aligned(layer->cache_len, 4) ||
        !(rope_theta > 0.f) || std::isinf(rope_theta))
        return ORTHRUS_ERR_INVALID_ARG;
    if ((st = check_workspace(workspace, workspace_bytes)) != ORTHRUS_OK) return st;
    return launch_paged_kv_write(*layer, slot_map, q, k_blk, v_blk, (double)rope_theta, q_out, static_cast<int32_t *>(workspace),
                                 static_cast<cudaStream_t>(stream)) == cudaSuccess ? ORTHRUS_OK : ORTHRUS_ERR_CUDA;
}

orthrus_status_t orthrus_paged_commit_len(const orthrus_paged_layer_t *layer, const int32_t *n_commit, void *workspace,
        size_t workspace_bytes, void *stream)
{
    orthrus_status_t st = check_paged(layer, false);
    if (st != ORTHRUS_OK) return st;
    if (!n_commit || !layer->cache_len || !aligned(n_commit, 4) || !aligned(layer->cache_len, 4)) return ORTHRUS_ERR_INVALID_ARG;
    if ((st = check_workspace(workspace, workspace_bytes)) != ORTHRUS_OK) return st;
    // the length update of the contiguous cache, whose capacity is what the table can name
    orthrus_layer_t L = {};
    L.batch = layer->batch; L.block = layer->block; L.flags = layer->flags; L.cache_len = layer->cache_len;
    L.capacity = (int64_t)layer->max_pages * layer->page_size;
    return launch_commit_len(L, n_commit, static_cast<int32_t *>(workspace), static_cast<cudaStream_t>(stream)) == cudaSuccess
               ? ORTHRUS_OK : ORTHRUS_ERR_CUDA;
}

size_t orthrus_paged_attend_workspace_bytes(const orthrus_paged_layer_t *layer)
{
    if (check_paged(layer, true) != ORTHRUS_OK) return 0;
    const size_t tc = paged_tc_shape(*layer) ? paged_tc_workspace_bytes(*layer) : 0, simt = paged_simt_workspace_bytes(*layer);
    return kHeaderBytes + (tc > simt ? tc : simt);
}

orthrus_status_t orthrus_paged_ar_attend(const orthrus_paged_layer_t *layer, const void *q, void *out, void *workspace,
        size_t workspace_bytes, void *stream)
{
    return attend(layer, 1, q, out, workspace, workspace_bytes, stream);
}

orthrus_status_t orthrus_paged_diffusion_attend(const orthrus_paged_layer_t *layer, const void *q, void *out, void *workspace,
        size_t workspace_bytes, void *stream)
{
    return attend(layer, 0, q, out, workspace, workspace_bytes, stream);
}

orthrus_status_t orthrus_sample_tokens(const void *logits, int32_t dtype, int32_t rows, int32_t vocab, int64_t row_stride,
        const float *temperature, const int32_t *top_k, const float *top_p, const float *min_p, const float *u,
        int32_t *token, float *logprob, void *stream)
{
    if (rows < 1 || vocab < 1 || row_stride < vocab) return ORTHRUS_ERR_INVALID_ARG;
    if (dtype != ORTHRUS_BF16 && dtype != ORTHRUS_FP32) return ORTHRUS_ERR_UNSUPPORTED;
    if (rows > (1 << 20) || vocab > (1 << 24) || row_stride > (1LL << 40)) return ORTHRUS_ERR_UNSUPPORTED;
    if (!logits || !temperature || !u || !token || !aligned(logits, dtype == ORTHRUS_FP32 ? 4 : 2)) return ORTHRUS_ERR_INVALID_ARG;
    const void *const all[] = {temperature, top_k, top_p, min_p, u, token, logprob};
    for (const void *x : all)
        if (!aligned(x, 4)) return ORTHRUS_ERR_INVALID_ARG;
    return launch_sample_tokens(logits, dtype, rows, vocab, row_stride, temperature, top_k, top_p, min_p, u, token, logprob,
                                static_cast<cudaStream_t>(stream)) == cudaSuccess ? ORTHRUS_OK : ORTHRUS_ERR_CUDA;
}

}  // extern "C"
