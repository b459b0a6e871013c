// C-ABI entry points of the 8-bit cache: store / load, append, recall and attention.
#include "pi_api_guard.cuh"
#include "pi_kv8.cuh"

extern "C" int64_t pi_kv8_block_bytes(pi_ctx* ctx) {
    if (!ctx) return PI_ERR_INVALID_ARG;
    return kv8_block_bytes(ctx->cfg.n_kv_heads, ctx->cfg.block_tokens);
}

extern "C" int pi_kv8_store(pi_ctx* ctx, int64_t n_tokens, const void* k_dev, int64_t k_token_stride, int64_t k_head_stride,
                            int64_t k_outer_stride, const void* v_dev, int64_t v_token_stride, int64_t v_head_stride,
                            int64_t v_outer_stride, int64_t inner_tokens, const int64_t* slot_map_dev, void* store, int64_t n_blocks,
                            void* stream) {
    if (!ctx || n_tokens < 0 || n_tokens > INT32_MAX || inner_tokens < 0 || inner_tokens > INT32_MAX || n_blocks < 1 || n_blocks > INT32_MAX)
        return PI_ERR_INVALID_ARG;
    const int64_t ks[3] = {k_token_stride, k_head_stride, k_outer_stride}, vs[3] = {v_token_stride, v_head_stride, v_outer_stride};
    for (int i = 0; i < 3; ++i) {
        if (ks[i] < 0 || vs[i] < 0) return PI_ERR_INVALID_ARG;
        if (ks[i] % 8 || vs[i] % 8) return PI_ERR_BAD_ALIGN;
    }
    if (n_tokens == 0) return PI_OK;
    if (!k_dev || !v_dev || !store) return PI_ERR_INVALID_ARG;
    if (!slot_map_dev && n_tokens > n_blocks * ctx->cfg.block_tokens) return PI_ERR_INVALID_ARG;
    if (!pi_aligned16(k_dev) || !pi_aligned16(v_dev) || !pi_aligned16(store)) return PI_ERR_BAD_ALIGN;
    DeviceGuard guard(ctx->device);
    if (!guard.ok()) return PI_ERR_CUDA;
    void* dst = nullptr;
    const int rc = device_view(store, &dst);
    if (rc != PI_OK) return rc;
    return pi_launch_kv8_store(ctx, n_tokens, k_dev, ks, v_dev, vs, static_cast<int>(inner_tokens), slot_map_dev, dst, n_blocks,
                               static_cast<cudaStream_t>(stream));
}

extern "C" int pi_kv8_load(pi_ctx* ctx, int64_t n_out, const void* store, int64_t n_blocks, const int32_t* blocks_dev, void* kv_dev, void* stream) {
    if (!ctx || n_out < 0 || n_blocks < 1 || n_blocks > INT32_MAX) return PI_ERR_INVALID_ARG;
    // one warp 16 rows of K or of V, four to a CTA
    if (n_out > INT32_MAX / (static_cast<int64_t>(ctx->cfg.n_kv_heads) * (ctx->cfg.block_tokens / 16))) return PI_ERR_UNSUPPORTED_DIM;
    if (n_out == 0) return PI_OK;
    if (!store || !kv_dev || (!blocks_dev && n_out > n_blocks)) return PI_ERR_INVALID_ARG;
    if (!pi_aligned16(store) || !pi_aligned16(kv_dev)) return PI_ERR_BAD_ALIGN;
    DeviceGuard guard(ctx->device);
    if (!guard.ok()) return PI_ERR_CUDA;
    void* src = nullptr;
    const int rc = device_view(store, &src);
    if (rc != PI_OK) return rc;
    return pi_launch_kv8_load(ctx, n_out, src, n_blocks, blocks_dev, kv_dev, static_cast<cudaStream_t>(stream));
}

extern "C" int pi_append_kv8(pi_ctx* ctx, int layer, int batch, uint32_t step, const uint32_t* step_dev, const void* k_new_dev,
                             const void* v_new_dev, const int32_t* ctx_len_dev, void* host_kv8_pinned, int64_t host_seq_stride_bytes,
                             const int32_t* page_table_dev, int64_t page_table_seq_stride, int32_t n_pages, void* pool8_dev,
                             int32_t* block_table_dev, int32_t* slot_block_dev, uint32_t* slot_stamp_dev, void* digest_dev, void* stream) {
    if (!valid(ctx, layer, batch)) return PI_ERR_INVALID_ARG;
    if (ctx->cfg.n_local_blocks < 1) return PI_ERR_INVALID_ARG;     // as pi_append_kv: the block being filled must stay resident
    if (!k_new_dev || !v_new_dev || !ctx_len_dev || !host_kv8_pinned || !pool8_dev || !block_table_dev || !slot_block_dev ||
        !slot_stamp_dev || !digest_dev || (!step_dev && step == 0) || host_seq_stride_bytes < 0)
        return PI_ERR_INVALID_ARG;
    if (page_table_dev && (page_table_seq_stride < 1 || n_pages < 1)) return PI_ERR_INVALID_ARG;
    if (!pi_aligned16(k_new_dev) || !pi_aligned16(v_new_dev) || !pi_aligned16(host_kv8_pinned) || !pi_aligned16(pool8_dev) ||
        !pi_aligned16(digest_dev) || host_seq_stride_bytes % 16)
        return PI_ERR_BAD_ALIGN;
    DeviceGuard guard(ctx->device);
    if (!guard.ok()) return PI_ERR_CUDA;
    void* dst = nullptr;
    const int rc = device_view(host_kv8_pinned, &dst);
    if (rc != PI_OK) return rc;
    return pi_launch_append_kv8(ctx, ctx->solo_head[layer], batch, step, step_dev, k_new_dev, v_new_dev, ctx_len_dev, dst,
                                page_table_dev ? 0 : host_seq_stride_bytes, pool8_dev, block_table_dev, slot_block_dev, slot_stamp_dev,
                                digest_dev, page_table_dev, page_table_seq_stride, n_pages, static_cast<cudaStream_t>(stream));
}

extern "C" int pi_recall_kv8(pi_ctx* ctx, int layer, int batch, const void* host_kv8_pinned, int64_t host_seq_stride_bytes,
                             const int32_t* page_table_dev, int64_t page_table_seq_stride, int32_t n_pages, void* pool8_dev,
                             const pi_extent* recall_list_dev, int32_t list_capacity, const int32_t* recall_count_dev, void* stream) {
    if (!valid(ctx, layer, batch)) return PI_ERR_INVALID_ARG;
    if (!host_kv8_pinned || !pool8_dev || !recall_list_dev || !recall_count_dev || list_capacity < 1) return PI_ERR_INVALID_ARG;
    if (page_table_dev && (page_table_seq_stride < 1 || n_pages < 1)) return PI_ERR_INVALID_ARG;
    if (host_seq_stride_bytes < 0 || host_seq_stride_bytes % 16 || !pi_aligned16(host_kv8_pinned) || !pi_aligned16(pool8_dev) ||
        !pi_aligned16(recall_list_dev))
        return PI_ERR_BAD_ALIGN;
    DeviceGuard guard(ctx->device);
    if (!guard.ok()) return PI_ERR_CUDA;
    void* src = nullptr;
    const int rc = device_view(host_kv8_pinned, &src);
    if (rc != PI_OK) return rc;
    const int64_t bytes = kv8_block_bytes(ctx->cfg.n_kv_heads, ctx->cfg.block_tokens);
    return pi_launch_recall(ctx, batch, 1, src, page_table_dev ? 0 : host_seq_stride_bytes, pool8_dev, ctx->cfg.pool_slots * bytes,
                            recall_list_dev, list_capacity, recall_count_dev, bytes, bytes, 0, page_table_dev, page_table_seq_stride,
                            n_pages, bytes, static_cast<cudaStream_t>(stream));
}

extern "C" int pi_sparse_decode_attn_kv8(pi_ctx* ctx, int layer, int batch, const void* q_dev, const void* pool8_dev,
                                         const int32_t* sel_slots_dev, const int32_t* sel_blocks_dev, const int32_t* sel_count_dev,
                                         const int32_t* ctx_len_dev, void* out_dev, float* lse_dev, void* stream) {
    if (!valid(ctx, layer, batch)) return PI_ERR_INVALID_ARG;
    if (!q_dev || !pool8_dev || !sel_slots_dev || !sel_blocks_dev || !sel_count_dev || !ctx_len_dev || !out_dev) return PI_ERR_INVALID_ARG;
    if (!pi_aligned16(q_dev) || !pi_aligned16(pool8_dev) || !pi_aligned16(out_dev)) return PI_ERR_BAD_ALIGN;
    DeviceGuard guard(ctx->device);
    if (!guard.ok()) return PI_ERR_CUDA;
    return pi_launch_attn_kv8(ctx, batch, q_dev, pool8_dev, sel_slots_dev, sel_blocks_dev, sel_count_dev, ctx_len_dev, out_dev, lse_dev,
                              static_cast<cudaStream_t>(stream));
}
