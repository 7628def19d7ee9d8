// C-ABI entry points: context, argument validation, dispatch to the kernel launchers.
#include <math.h>
#include <stdlib.h>

#include <new>

#include "hs_common.cuh"
#include "hs_layout.h"
#include "hs_ptx.cuh"

extern "C" const char* hs_status_string(hs_status s) {
    switch (s) {
        case HS_OK: return "ok";
        case HS_ERR_INVALID_ARG: return "invalid argument";
        case HS_ERR_SHAPE: return "unsupported shape";
        case HS_ERR_UNSUPPORTED: return "unsupported";
        case HS_ERR_WORKSPACE: return "workspace too small";
        case HS_ERR_CUDA: return "CUDA error";
        case HS_ERR_TIMEOUT: return "device-side wait expired";
        case HS_ERR_BAD_TREE: return "malformed tree";
        case HS_ERR_BAD_PAGE: return "page table entry or cache length outside the pool";
        case HS_ERR_STATIC_LIMIT: return "batch exceeds the built-in scratch of the allocation-free entry point";
    }
    return "unknown status";
}

extern "C" size_t hs_workspace_bytes(int32_t max_batch, int32_t max_rows, int32_t vocab, int32_t hq, int32_t hkv) {
    if (max_batch < 1 || max_rows < 1 || vocab < 1 || hq < 1 || hkv < 1) return 0;
    size_t chunks = hs_row_chunks(vocab, HS_F32);
    // entropy pass: two partials per warp, sixteen warps per SM (room for 152 SMs; with less the shares get longer)
    size_t quant = (size_t)2 * 152 * 16 * HS_ROW_PARTIAL_BYTES + 512;
    // acceptance: three per-row result arrays (256-byte aligned each) + chunk partials of target and draft rows
    size_t accept = 3 * hs_align_up((size_t)max_rows * 8, 256) +
                    (size_t)2 * (max_rows * chunks > 152 * 16 ? max_rows * chunks : 152 * 16) * HS_ACC_PARTIAL_BYTES +
                    (size_t)(max_batch < 256 ? max_batch : 256) * 2048 + 512;      // shared bonus draws
    // (the attention merges its KV splits on chip: no workspace)
    size_t scratch = quant > accept ? quant : accept;
    return HS_COUNTER_BYTES + hs_align_up(scratch, 256) + 256;
}

extern "C" hs_status hs_create(hs_ctx** out, int32_t device, size_t workspace_bytes) {
    if (!out) return HS_ERR_INVALID_ARG;
    *out = nullptr;
    if (workspace_bytes < HS_COUNTER_BYTES + 256) return HS_ERR_WORKSPACE;
    int ndev = 0;
    HS_CUDA_OK(cudaGetDeviceCount(&ndev));
    if (device < 0 || device >= ndev) return HS_ERR_INVALID_ARG;
    HS_CUDA_OK(cudaSetDevice(device));
    int sm_count = 0, major = 0;
    HS_CUDA_OK(cudaDeviceGetAttribute(&sm_count, cudaDevAttrMultiProcessorCount, device));
    HS_CUDA_OK(cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, device));
    if (major != 10) return HS_ERR_UNSUPPORTED;                   // built for sm_100a only
    hs_ctx* c = new (std::nothrow) hs_ctx();
    if (!c) return HS_ERR_INVALID_ARG;
    c->device = device;
    c->sm_count = sm_count;
    void* p = nullptr;
    if (cudaMalloc(&p, workspace_bytes) != cudaSuccess) { delete c; return HS_ERR_CUDA; }
    c->ws = (char*)p;
    c->ws_bytes = workspace_bytes;
    c->counters = (int*)p;
    c->n_counters = HS_COUNTER_BYTES / sizeof(int);
    c->scratch = c->ws + HS_COUNTER_BYTES;
    c->scratch_bytes = workspace_bytes - HS_COUNTER_BYTES;
    if (cudaMemset(p, 0, HS_COUNTER_BYTES) != cudaSuccess) { cudaFree(p); delete c; return HS_ERR_CUDA; }
    cudaDriverEntryPointQueryResult qres;
    void* fn = nullptr;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &qres) != cudaSuccess ||
        qres != cudaDriverEntryPointSuccess || !fn) {
        cudaFree(p); delete c; return HS_ERR_CUDA;
    }
    c->encode_tiled = fn;
    const char* no_pdl = getenv("HS_DISABLE_PDL");
    c->pdl = !(no_pdl && no_pdl[0] == '1');
    c->prefetch = 0;
    c->row_pass = HS_ROW_PASS_AUTO;
    c->attn_ready = false;
    c->walk_ready = false;
    c->quant_ready = false;
    c->warps_ready = false;
    c->cart_ready = false;
    c->paged_ready = false;
    c->cart_ctas = 0;
    c->stream_part = c->part_sms = nullptr;
    if (cudaDeviceSynchronize() != cudaSuccess) { cudaFree(p); delete c; return HS_ERR_CUDA; }
    *out = c;
    return HS_OK;
}

extern "C" hs_status hs_destroy(hs_ctx* ctx) {
    if (!ctx) return HS_ERR_INVALID_ARG;
    cudaSetDevice(ctx->device);
    cudaFree(ctx->ws);
    delete ctx;
    return HS_OK;
}

// One thread waits on a barrier that nothing ever completes; the bounded wait gives up after limit_ns and
// records HS_ERR_TIMEOUT in the context's error word.
__global__ void wait_selftest_kernel(int* err, unsigned long long limit_ns) {
    __shared__ unsigned long long s_bar;
    const unsigned int bar = smem_u32(&s_bar);
    mbar_init(bar, 1);
    mbar_init_fence();
    mbar_wait_limit(bar, 0u, err, limit_ns);
}

hs_status hs_launch_wait_selftest(hs_ctx* ctx, uint64_t limit_ns, cudaStream_t stream) {
    wait_selftest_kernel<<<1, 1, 0, stream>>>(ctx->counters + HS_CNT_ERROR, (unsigned long long)limit_ns);
    return cudaGetLastError() == cudaSuccess ? HS_OK : HS_ERR_CUDA;
}

extern "C" hs_status hs_set_prefetch(hs_ctx* ctx, int32_t flags) {
    if (!ctx || (flags & ~(HS_PREFETCH_LOGITS | HS_PREFETCH_KV))) return HS_ERR_INVALID_ARG;
    ctx->prefetch = flags;
    return HS_OK;
}

extern "C" hs_status hs_set_row_pass(hs_ctx* ctx, int32_t variant) {
    if (!ctx || variant < HS_ROW_PASS_AUTO || variant > HS_ROW_PASS_STREAM) return HS_ERR_INVALID_ARG;
    ctx->row_pass = variant;
    return HS_OK;
}

extern "C" hs_status hs_selftest_wait_timeout(hs_ctx* ctx, uint64_t limit_ns, hs_stream stream) {
    if (!ctx || !hs_on_device(ctx)) return HS_ERR_INVALID_ARG;
    if (limit_ns < 1000ull) limit_ns = 1000ull;
    if (limit_ns > 10000000ull) limit_ns = 10000000ull;
    return hs_launch_wait_selftest(ctx, limit_ns, (cudaStream_t)stream);
}

extern "C" hs_status hs_device_error(hs_ctx* ctx, int32_t* host_out) {
    if (!ctx || !host_out) return HS_ERR_INVALID_ARG;
    HS_CUDA_OK(cudaSetDevice(ctx->device));
    HS_CUDA_OK(cudaDeviceSynchronize());
    int v = 0;
    HS_CUDA_OK(cudaMemcpy(&v, ctx->counters + HS_CNT_ERROR, sizeof(int), cudaMemcpyDeviceToHost));
    if (v != 0) HS_CUDA_OK(cudaMemset(ctx->counters + HS_CNT_ERROR, 0, sizeof(int)));
    *host_out = v;
    return HS_OK;
}

static bool tree_ok(const hs_tree_batch* t) {
    return t && t->batch >= 1 && t->batch <= HS_MAX_BATCH && t->n_nodes_total >= t->batch &&
           t->n_nodes_total <= HS_MAX_ROWS && t->node_off && t->parent && t->token;
}
static bool policy_ok(const hs_policy* p) {
    if (!p || p->top_k < 1 || p->top_k > HS_MAX_TOPK || p->d_base < 0 || p->n_default < 1) return false;
    for (int i = 0; i + 1 < 7; ++i)
        if (!(p->thresholds[i] <= p->thresholds[i + 1])) return false;
    for (int i = 0; i < 3; ++i)
        if (p->gamma_pct[i] < 0) return false;
    return p->phi_mode >= 0 && p->phi_mode <= 1 && p->pstar_mode >= 0 && p->pstar_mode <= 1 &&
           p->entropy_mode >= 0 && p->entropy_mode <= 1;
}
static bool logits_ok(const void* p, hs_dtype dtype, int64_t row_stride, int32_t vocab) {
    if (!p || ((uintptr_t)p & 15)) return false;
    if (dtype != HS_F32 && dtype != HS_BF16) return false;
    int vec = dtype == HS_BF16 ? 8 : 4;
    return vocab >= 1 && row_stride >= vocab && row_stride % vec == 0;
}

extern "C" hs_status hs_entropy_quantify(hs_ctx* ctx, const hs_tree_batch* tree, const void* draft_logits,
                                         hs_dtype dtype, int64_t row_stride, int32_t vocab,
                                         const hs_policy* policy, const hs_quant_out* out, hs_stream stream) {
    if (!ctx || !out || !hs_on_device(ctx)) return HS_ERR_INVALID_ARG;
    if (!tree_ok(tree) || !policy_ok(policy) || !logits_ok(draft_logits, dtype, row_stride, vocab))
        return HS_ERR_INVALID_ARG;
    if (!out->row_max || !out->row_lse || !out->h_full || !out->i_topk || !out->i_trunc || !out->topk_val ||
        !out->topk_idx || !out->logc || !out->score || !out->phi || !out->depth || !out->pstar_node ||
        !out->phi_star || !out->status)
        return HS_ERR_INVALID_ARG;
    return hs_launch_quantify(ctx, tree, draft_logits, dtype, row_stride, vocab, policy, out, (cudaStream_t)stream);
}

static bool pruned_out_ok(const hs_pruned_tree* out) {
    return out && out->bin && out->d_prime && out->n_prime && out->n_keep && out->keep_off && out->keep_idx &&
           out->new_parent && out->new_depth && out->keep_rank && out->anc_mask && out->status;
}

extern "C" hs_status hs_entropy_quantify_prune(hs_ctx* ctx, const hs_tree_batch* tree, const void* draft_logits,
                                               hs_dtype dtype, int64_t row_stride, int32_t vocab,
                                               const hs_policy* policy, const hs_quant_out* quant,
                                               const hs_pruned_tree* pruned, hs_stream stream) {
    if (!ctx || !quant || !hs_on_device(ctx)) return HS_ERR_INVALID_ARG;
    if (!tree_ok(tree) || !policy_ok(policy) || !logits_ok(draft_logits, dtype, row_stride, vocab))
        return HS_ERR_INVALID_ARG;
    if (!quant->row_max || !quant->row_lse || !quant->h_full || !quant->i_topk || !quant->i_trunc || !quant->topk_val ||
        !quant->topk_idx || !quant->logc || !quant->score || !quant->phi || !quant->depth || !quant->pstar_node ||
        !quant->phi_star || !quant->status || !pruned_out_ok(pruned))
        return HS_ERR_INVALID_ARG;
    hs_status st = hs_launch_quantify(ctx, tree, draft_logits, dtype, row_stride, vocab, policy, quant,
                                      (cudaStream_t)stream, false);
    if (st != HS_OK) return st;
    return hs_launch_tree_prune(ctx, tree, draft_logits, dtype, row_stride, vocab, policy, quant, pruned,
                                (cudaStream_t)stream);
}

extern "C" hs_status hs_stratify_prune(hs_ctx* ctx, const hs_tree_batch* tree, const hs_quant_out* quant,
                                       const hs_policy* policy, const hs_pruned_tree* out, hs_stream stream) {
    if (!ctx || !quant || !out || !hs_on_device(ctx)) return HS_ERR_INVALID_ARG;
    if (!tree_ok(tree) || !policy_ok(policy)) return HS_ERR_INVALID_ARG;
    if (!quant->score || !quant->phi_star || !quant->depth || !quant->status) return HS_ERR_INVALID_ARG;
    if (!out->bin || !out->d_prime || !out->n_prime || !out->n_keep || !out->keep_off || !out->keep_idx ||
        !out->new_parent || !out->new_depth || !out->keep_rank || !out->anc_mask || !out->status)
        return HS_ERR_INVALID_ARG;
    return hs_launch_stratify_prune(ctx, tree, quant, policy, out, (cudaStream_t)stream);
}

extern "C" hs_status hs_stratify_prune_budget(hs_ctx* ctx, const hs_tree_batch* tree, const hs_quant_out* quant,
                                              const hs_policy* policy, const int32_t* slo_class, int32_t budget,
                                              const hs_pruned_tree* out, hs_stream stream) {
    if (!ctx || !quant || !out || !slo_class || budget < 0 || !hs_on_device(ctx)) return HS_ERR_INVALID_ARG;
    if (!tree_ok(tree) || !policy_ok(policy)) return HS_ERR_INVALID_ARG;
    if (!quant->score || !quant->phi_star || !quant->depth || !quant->status) return HS_ERR_INVALID_ARG;
    if (!out->bin || !out->d_prime || !out->n_prime || !out->n_keep || !out->keep_off || !out->keep_idx ||
        !out->new_parent || !out->new_depth || !out->keep_rank || !out->anc_mask || !out->status)
        return HS_ERR_INVALID_ARG;
    return hs_launch_stratify_prune_budget(ctx, tree, quant, policy, slo_class, budget, out, (cudaStream_t)stream);
}

static bool pruned_ok(const hs_pruned_tree* p) {
    return p && p->n_keep && p->keep_off && p->keep_idx && p->new_parent && p->new_depth && p->keep_rank &&
           p->anc_mask && p->status;
}

extern "C" hs_status hs_tree_verify_attention(hs_ctx* ctx, const hs_pruned_tree* pruned, const hs_attn_desc* d,
                                              const void* q, const void* k_tree, const void* v_tree,
                                              const void* k_cache, const void* v_cache, void* out,
                                              float* lse_out, hs_stream stream) {
    if (!ctx || !d || !pruned_ok(pruned) || !q || !k_tree || !v_tree || !out || !hs_on_device(ctx))
        return HS_ERR_INVALID_ARG;
    if (d->batch < 1 || d->batch > HS_MAX_BATCH || d->max_rows < 1 || d->max_rows > HS_MAX_ROWS ||
        d->max_nodes < 1 || d->max_nodes > HS_MAX_NODES || d->kv_total < 0 || d->max_kv_len < 0 ||
        d->max_kv_len > d->kv_total || !d->kv_off)
        return HS_ERR_INVALID_ARG;
    if (d->kv_total > 0 && (!k_cache || !v_cache)) return HS_ERR_INVALID_ARG;
    if (d->layout != HS_ROWS_COMPACT && d->layout != HS_ROWS_ORIGINAL) return HS_ERR_INVALID_ARG;
    if (d->layout == HS_ROWS_ORIGINAL && !d->node_off) return HS_ERR_INVALID_ARG;
    if (d->head_dim != HS_HEAD_DIM || d->hq < 1 || d->hkv < 1 || d->hq % d->hkv != 0 || d->hq / d->hkv > 16)
        return HS_ERR_SHAPE;
    if (d->kv_total > 0 && (d->kv_token_stride % 8 != 0 || d->kv_head_stride % 8 != 0 ||
                            d->kv_token_stride < HS_HEAD_DIM || d->kv_head_stride < HS_HEAD_DIM))
        return HS_ERR_SHAPE;
    if (((uintptr_t)q | (uintptr_t)k_tree | (uintptr_t)v_tree | (uintptr_t)k_cache | (uintptr_t)v_cache |
         (uintptr_t)out) & 15)
        return HS_ERR_INVALID_ARG;
    return hs_launch_attention(ctx, pruned, d, q, k_tree, v_tree, k_cache, v_cache, out, lse_out,
                               (cudaStream_t)stream);
}

extern "C" hs_status hs_accept_path(hs_ctx* ctx, const hs_tree_batch* tree, const hs_pruned_tree* pruned,
                                    const void* target_logits, int32_t target_layout, const void* draft_logits,
                                    hs_dtype dtype, int64_t row_stride, int32_t vocab, const int32_t* mode,
                                    const float* temperature, uint64_t seed, uint64_t offset,
                                    const float* uniforms, const hs_accept_out* out, hs_stream stream) {
    if (!ctx || !out || !mode || !temperature || !hs_on_device(ctx) || (offset >> 63)) return HS_ERR_INVALID_ARG;
    if (!tree_ok(tree) || !pruned_ok(pruned) || !logits_ok(target_logits, dtype, row_stride, vocab))
        return HS_ERR_INVALID_ARG;
    if (draft_logits && ((uintptr_t)draft_logits & 15)) return HS_ERR_INVALID_ARG;
    if (target_layout != HS_ROWS_COMPACT && target_layout != HS_ROWS_ORIGINAL) return HS_ERR_INVALID_ARG;
    if (!out->accept_len || !out->path_nodes || !out->path_compact || !out->path_tokens || !out->bonus_token ||
        !out->terminal_rank || !out->status || out->path_cap < 2)
        return HS_ERR_INVALID_ARG;
    return hs_launch_accept(ctx, tree, pruned, target_logits, target_layout, draft_logits, dtype, row_stride,
                            vocab, mode, temperature, seed, offset, uniforms, out, (cudaStream_t)stream);
}

extern "C" hs_status hs_philox_uniforms(hs_ctx* ctx, uint64_t seed, uint64_t offset, const int32_t* b,
                                        const int32_t* node, const int32_t* stream_id, int32_t count,
                                        float* out, hs_stream stream) {
    if (!ctx || !b || !node || !stream_id || !out || count < 0 || !hs_on_device(ctx) || (offset >> 63))
        return HS_ERR_INVALID_ARG;
    if (count == 0) return HS_OK;
    return hs_launch_philox(seed, offset, b, node, stream_id, count, out, (cudaStream_t)stream);
}

// for the Python binding's native module
extern "C" int hs_context_device(const hs_ctx* ctx) { return ctx->device; }

// ---- the paged cache ---------------------------------------------------------------------------------------------------
static hs_status cache_check(const hs_kv_cache* c) {
    if (!c || !c->k || !c->v || !c->k_scale || !c->v_scale || !c->page_table || !c->kv_len) return HS_ERR_INVALID_ARG;
    if (((uintptr_t)c->k | (uintptr_t)c->v | (uintptr_t)c->k_scale | (uintptr_t)c->v_scale) & 15) return HS_ERR_INVALID_ARG;
    if (c->batch < 1 || c->batch > HS_MAX_BATCH || c->n_pages < 1 || c->max_pages < 1) return HS_ERR_INVALID_ARG;
    if (c->head_dim != HS_HEAD_DIM || c->hkv < 1 || c->hkv > 1024 || c->page_size < 16 || c->page_size > 1024 ||
        (c->page_size & (c->page_size - 1)) || (int64_t)c->max_pages * c->page_size >= (1 << 30))
        return HS_ERR_SHAPE;
    return HS_OK;
}
// strides of rows of `heads` heads of `dim` values that are loaded as 16-byte vectors
static bool strides_ok(int64_t token_stride, int64_t head_stride, int32_t heads, int32_t dim, hs_dtype dtype) {
    const int vec = dtype == HS_BF16 ? 8 : 4;
    return token_stride % vec == 0 && head_stride % vec == 0 && token_stride >= dim && (heads == 1 || head_stride >= dim);
}
static bool dtype_ok(hs_dtype dtype) { return dtype == HS_F32 || dtype == HS_BF16; }

extern "C" hs_status hs_kv_append(hs_ctx* ctx, const hs_kv_cache* cache, const void* k, const void* v, hs_dtype dtype,
                                  int64_t token_stride, int64_t head_stride, const int32_t* row_off, int32_t n_rows,
                                  int32_t* len_out, hs_stream stream) {
    if (!ctx || !hs_on_device(ctx)) return HS_ERR_INVALID_ARG;
    if (hs_status st = cache_check(cache)) return st;
    if (n_rows < 0 || !row_off || !dtype_ok(dtype) || len_out == cache->kv_len) return HS_ERR_INVALID_ARG;
    if (n_rows > 0 && (!k || !v || (((uintptr_t)k | (uintptr_t)v) & 15))) return HS_ERR_INVALID_ARG;
    if (n_rows > 0 && !strides_ok(token_stride, head_stride, cache->hkv, HS_HEAD_DIM, dtype)) return HS_ERR_SHAPE;
    return hs_launch_kv_append(ctx, cache, k, v, dtype, token_stride, head_stride, row_off, n_rows, len_out, (cudaStream_t)stream);
}

extern "C" hs_status hs_kv_append_path(hs_ctx* ctx, const hs_kv_cache* cache, const hs_pruned_tree* pruned,
                                       const hs_accept_out* accept, int32_t layout, const int32_t* node_off,
                                       const void* k_tree, const void* v_tree, int32_t max_rows, int32_t* len_out,
                                       hs_stream stream) {
    if (!ctx || !hs_on_device(ctx)) return HS_ERR_INVALID_ARG;
    if (hs_status st = cache_check(cache)) return st;
    if (!pruned || !accept || !pruned->status || !pruned->n_keep || !pruned->keep_off || !accept->status || !accept->accept_len || !accept->path_nodes ||
        !accept->path_compact || accept->path_cap < 1 || !k_tree || !v_tree || max_rows < 1 || max_rows > HS_MAX_ROWS ||
        len_out == cache->kv_len)
        return HS_ERR_INVALID_ARG;
    if (layout != HS_ROWS_COMPACT && layout != HS_ROWS_ORIGINAL) return HS_ERR_INVALID_ARG;
    if (layout == HS_ROWS_ORIGINAL && !node_off) return HS_ERR_INVALID_ARG;
    if (((uintptr_t)k_tree | (uintptr_t)v_tree) & 15) return HS_ERR_INVALID_ARG;
    return hs_launch_kv_append_path(ctx, cache, pruned, accept, layout, node_off, k_tree, v_tree, max_rows, len_out,
                                    (cudaStream_t)stream);
}

extern "C" hs_status hs_kv_read(hs_ctx* ctx, const hs_kv_cache* cache, const int32_t* row_off, const int32_t* first,
                                int32_t n_rows, void* k_out, void* v_out, hs_dtype dtype, int64_t token_stride,
                                int64_t head_stride, hs_stream stream) {
    if (!ctx || !hs_on_device(ctx)) return HS_ERR_INVALID_ARG;
    if (hs_status st = cache_check(cache)) return st;
    if (n_rows < 0 || !row_off || !dtype_ok(dtype)) return HS_ERR_INVALID_ARG;
    if (n_rows == 0) return HS_OK;
    if (!k_out || !v_out || (((uintptr_t)k_out | (uintptr_t)v_out) & 15)) return HS_ERR_INVALID_ARG;
    if (!strides_ok(token_stride, head_stride, cache->hkv, HS_HEAD_DIM, dtype)) return HS_ERR_SHAPE;
    return hs_launch_kv_read(ctx, cache, row_off, first, n_rows, k_out, v_out, dtype, token_stride, head_stride, (cudaStream_t)stream);
}

extern "C" hs_status hs_tree_verify_attention_paged(hs_ctx* ctx, const hs_pruned_tree* pruned, const hs_kv_cache* cache,
                                                    const hs_paged_attn_desc* d, const void* q, const void* k_tree,
                                                    const void* v_tree, void* out, float* lse_out, hs_stream stream) {
    if (!ctx || !d || !pruned || !pruned->n_keep || !pruned->keep_off || !pruned->keep_idx || !pruned->anc_mask || !pruned->status || !q || !k_tree ||
        !v_tree || !out || !hs_on_device(ctx))
        return HS_ERR_INVALID_ARG;
    if (hs_status st = cache_check(cache)) return st;
    if (d->max_rows < 1 || d->max_rows > HS_MAX_ROWS || d->max_nodes < 1 || d->max_nodes > HS_MAX_NODES || d->max_kv_len < 0)
        return HS_ERR_INVALID_ARG;
    if (d->layout != HS_ROWS_COMPACT && d->layout != HS_ROWS_ORIGINAL) return HS_ERR_INVALID_ARG;
    if (d->layout == HS_ROWS_ORIGINAL && !d->node_off) return HS_ERR_INVALID_ARG;
    // (the kernel takes the maximum of unscaled scores)
    if (!(d->sm_scale > 0.f) || !(d->sm_scale <= 3.0e38f)) return HS_ERR_INVALID_ARG;
    if (d->hq < 1 || d->hq % cache->hkv != 0 || d->hq / cache->hkv > 16 || (int64_t)cache->batch * cache->hkv > 65535) return HS_ERR_SHAPE;
    if ((int64_t)cache->n_pages * cache->hkv * cache->page_size > 0x7fffffffll) return HS_ERR_SHAPE;      // rows of the tensor map
    if ((int64_t)d->max_rows * d->hq > 0x7fffffffll) return HS_ERR_SHAPE;
    if (((uintptr_t)q | (uintptr_t)k_tree | (uintptr_t)v_tree | (uintptr_t)out) & 15) return HS_ERR_INVALID_ARG;
    return hs_launch_attention_paged(ctx, pruned, cache, d, q, k_tree, v_tree, out, lse_out, (cudaStream_t)stream);
}

// ---- rotary positions --------------------------------------------------------------------------------------------------
extern "C" hs_status hs_rope_init(hs_rope* rope, const hs_rope_config* c) {
    if (!rope || !c) return HS_ERR_INVALID_ARG;
    if (c->head_dim < 16 || c->head_dim > 2 * HS_MAX_ROPE_PAIRS || c->head_dim % 16 || c->rotary_dim < 16 || c->rotary_dim > c->head_dim ||
        c->rotary_dim % 16)
        return HS_ERR_SHAPE;
    if (c->interleaved < 0 || c->interleaved > 1 || c->scaling < HS_ROPE_PLAIN || c->scaling > HS_ROPE_TABLE) return HS_ERR_INVALID_ARG;
    const double two_pi = 6.283185307179586476925286766559, n = c->rotary_dim;
    const bool scaled = c->scaling != HS_ROPE_PLAIN && c->scaling != HS_ROPE_TABLE;
    if (c->scaling == HS_ROPE_TABLE ? !c->inv_freq : !(c->base > 1.0 && isfinite(c->base))) return HS_ERR_INVALID_ARG;
    if (scaled && !(c->factor > 0.0 && isfinite(c->factor))) return HS_ERR_INVALID_ARG;
    if (c->scaling == HS_ROPE_LLAMA &&
        !(c->original_len > 0.0 && c->low_freq_factor > 0.0 && c->high_freq_factor > c->low_freq_factor && isfinite(c->high_freq_factor) && isfinite(c->original_len)))
        return HS_ERR_INVALID_ARG;
    if (c->scaling == HS_ROPE_YARN &&
        !(c->original_len > 0.0 && isfinite(c->original_len) && c->beta_slow > 0.0 && c->beta_fast >= c->beta_slow && isfinite(c->beta_fast) &&
          c->attn_factor >= 0.0 && isfinite(c->attn_factor)))
        return HS_ERR_INVALID_ARG;
    hs_rope r = {};
    r.head_dim = c->head_dim;
    r.rotary_dim = c->rotary_dim;
    r.interleaved = c->interleaved;
    r.scale = 1.f;
    double base = c->base, lo = 0.0, hi = 0.0;
    if (c->scaling == HS_ROPE_NTK) base *= pow(c->factor, n / (n - 2.0));
    if (c->scaling == HS_ROPE_YARN) {
        auto pair_of = [&](double turns) { return n * log(c->original_len / (turns * two_pi)) / (2.0 * log(base)); };
        lo = fmax(floor(pair_of(c->beta_fast)), 0.0);
        hi = fmin(ceil(pair_of(c->beta_slow)), n - 1.0);
        r.scale = (float)(c->attn_factor > 0.0 ? c->attn_factor : c->factor > 1.0 ? 0.1 * log(c->factor) + 1.0 : 1.0);
    }
    for (int i = 0; i < c->rotary_dim / 2; ++i) {
        double f = c->scaling == HS_ROPE_TABLE ? c->inv_freq[i] : pow(base, -2.0 * i / n);
        if (c->scaling == HS_ROPE_LINEAR) f /= c->factor;
        if (c->scaling == HS_ROPE_LLAMA) {
            const double turns = c->original_len * f / two_pi;         // over the original length
            const double s = (turns - c->low_freq_factor) / (c->high_freq_factor - c->low_freq_factor);
            if (turns < c->low_freq_factor) f /= c->factor;
            else if (turns <= c->high_freq_factor) f = (1.0 - s) * f / c->factor + s * f;
        }
        if (c->scaling == HS_ROPE_YARN) {
            const double ramp = fmin(fmax((i - lo) / fmax(hi - lo, 0.001), 0.0), 1.0);
            f = f / c->factor * ramp + f * (1.0 - ramp);
        }
        if (!(f >= 0.0) || !isfinite(f)) return HS_ERR_INVALID_ARG;
        // whole turns fall away; 2^64 times what is left, in long double (64 bits of mantissa)
        long double turn = (long double)f / 6.283185307179586476925286766559005768L;
        turn -= floorl(turn);
        const long double units = turn * 18446744073709551616.0L;
        r.turns[i] = units >= 18446744073709551615.0L ? 0ull : (uint64_t)(units + 0.5L);
    }
    *rope = r;
    return HS_OK;
}

static hs_status rope_check(const hs_rope* r) {
    if (!r) return HS_ERR_INVALID_ARG;
    if (r->head_dim < 16 || r->head_dim > 2 * HS_MAX_ROPE_PAIRS || r->head_dim % 16 || r->rotary_dim < 16 || r->rotary_dim > r->head_dim ||
        r->rotary_dim % 16 || r->interleaved < 0 || r->interleaved > 1)
        return HS_ERR_INVALID_ARG;
    return HS_OK;
}
static hs_status heads_check(const hs_heads* x, int32_t dim, hs_dtype dtype) {
    if (!x || !x->in || !x->out || (((uintptr_t)x->in | (uintptr_t)x->out) & 15)) return HS_ERR_INVALID_ARG;
    if (x->heads < 1 || x->heads > 1024) return HS_ERR_SHAPE;
    if (!strides_ok(x->in_token_stride, x->in_head_stride, x->heads, dim, dtype) ||
        !strides_ok(x->out_token_stride, x->out_head_stride, x->heads, dim, dtype))
        return HS_ERR_SHAPE;
    // in place means the same place: with other strides a row would be read after another was written over it
    if (x->in == x->out && (x->in_token_stride != x->out_token_stride || (x->heads > 1 && x->in_head_stride != x->out_head_stride)))
        return HS_ERR_INVALID_ARG;
    return HS_OK;
}

extern "C" hs_status hs_rotary(hs_ctx* ctx, const hs_rope* rope, const int32_t* pos, int32_t n_rows, const hs_heads* q,
                               const hs_heads* k, hs_dtype dtype, hs_stream stream) {
    if (!ctx || !hs_on_device(ctx) || n_rows < 0 || (n_rows > 0 && !pos) || !dtype_ok(dtype)) return HS_ERR_INVALID_ARG;
    if (hs_status st = rope_check(rope)) return st;
    if (n_rows == 0) return HS_OK;
    if (hs_status st = heads_check(q, rope->head_dim, dtype)) return st;
    if (k) if (hs_status st = heads_check(k, rope->head_dim, dtype)) return st;
    return hs_launch_rotary(ctx, rope, pos, n_rows, q, k, dtype, (cudaStream_t)stream);
}

extern "C" hs_status hs_rotary_tree(hs_ctx* ctx, const hs_rope* rope, const hs_pruned_tree* pruned, const int32_t* kv_len,
                                    int32_t batch, int32_t max_nodes, int32_t max_rows, int32_t layout,
                                    const int32_t* node_off, const hs_heads* q, const hs_heads* k, hs_dtype dtype,
                                    hs_stream stream) {
    if (!ctx || !hs_on_device(ctx) || !pruned || !pruned->n_keep || !pruned->keep_off || !pruned->keep_idx || !pruned->new_depth ||
        !pruned->status || !kv_len || !dtype_ok(dtype))
        return HS_ERR_INVALID_ARG;
    if (batch < 1 || batch > HS_MAX_BATCH || max_nodes < 1 || max_nodes > HS_MAX_NODES || max_rows < 1 || max_rows > HS_MAX_ROWS)
        return HS_ERR_INVALID_ARG;
    if (layout != HS_ROWS_COMPACT && layout != HS_ROWS_ORIGINAL) return HS_ERR_INVALID_ARG;
    if (layout == HS_ROWS_ORIGINAL && !node_off) return HS_ERR_INVALID_ARG;
    if (hs_status st = rope_check(rope)) return st;
    if (hs_status st = heads_check(q, rope->head_dim, dtype)) return st;
    if (k) if (hs_status st = heads_check(k, rope->head_dim, dtype)) return st;
    return hs_launch_rotary_tree(ctx, rope, pruned, kv_len, batch, max_nodes, max_rows, layout, node_off, q, k, dtype,
                                 (cudaStream_t)stream);
}
