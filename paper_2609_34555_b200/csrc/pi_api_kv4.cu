// C-ABI entry points around the 4-bit cache: page assignment, norm + rotation, 4-bit store / load, append, recall and
// attention.  They make the context's device current for the launch, whichever device the caller had.
#include <cmath>

#include "pi_kv4.cuh"

namespace {

class DeviceGuard {
public:
    explicit DeviceGuard(int device) {
        if (cudaGetDevice(&before_) != cudaSuccess) { (void)cudaGetLastError(); ok_ = false; return; }
        if (before_ != device) {
            if (cudaSetDevice(device) != cudaSuccess) { (void)cudaGetLastError(); ok_ = false; return; }
            changed_ = true;
        }
    }
    ~DeviceGuard() { if (changed_) (void)cudaSetDevice(before_); }
    DeviceGuard(const DeviceGuard&) = delete;
    DeviceGuard& operator=(const DeviceGuard&) = delete;
    bool ok() const { return ok_; }
private:
    int before_ = 0;
    bool changed_ = false, ok_ = true;
};

bool valid(const pi_ctx* ctx, int layer, int batch) {
    return ctx && layer >= 0 && layer < ctx->cfg.n_layers && batch >= 1 && batch <= ctx->cfg.max_batch;
}

// The device's address of a store in device memory or in pinned host memory.
int device_view(const void* p, void** out) {
    cudaPointerAttributes attr;
    if (cudaPointerGetAttributes(&attr, p) != cudaSuccess) { (void)cudaGetLastError(); return PI_ERR_NOT_PINNED; }
    *out = const_cast<void*>(p);
    if (attr.type == cudaMemoryTypeHost) {
        if (!attr.devicePointer) return PI_ERR_NOT_PINNED;
        *out = attr.devicePointer;
    } else if (attr.type != cudaMemoryTypeDevice && attr.type != cudaMemoryTypeManaged) {
        return PI_ERR_NOT_PINNED;
    }
    return PI_OK;
}

}  // namespace

extern "C" int64_t pi_kv4_block_bytes(pi_ctx* ctx) {
    if (!ctx) return PI_ERR_INVALID_ARG;
    return kv4_block_bytes(ctx->cfg.n_kv_heads, ctx->cfg.block_tokens);
}

extern "C" int pi_assign_pages(pi_ctx* ctx, int batch, const int32_t* old_len_dev, const int32_t* new_len_dev, int32_t* page_table_dev,
                               int64_t page_table_seq_stride, int32_t* free_pages_dev, int32_t n_pages, int64_t* free_state_dev,
                               int32_t* token_start_dev, int64_t n_tokens, int64_t* slot_map_dev, int32_t* positions_dev, void* stream) {
    if (!valid(ctx, 0, batch)) return PI_ERR_INVALID_ARG;
    if (!old_len_dev || !new_len_dev || !page_table_dev || !free_pages_dev || !free_state_dev) return PI_ERR_INVALID_ARG;
    if (page_table_seq_stride < 1 || n_pages < 1 || n_tokens < 0 || n_tokens > (1 << 30)) return PI_ERR_INVALID_ARG;
    if ((slot_map_dev && !pi_aligned16(slot_map_dev)) || (positions_dev && !pi_aligned16(positions_dev)) ||
        (reinterpret_cast<uintptr_t>(free_state_dev) & 7u))
        return PI_ERR_BAD_ALIGN;
    DeviceGuard guard(ctx->device);
    if (!guard.ok()) return PI_ERR_CUDA;
    return pi_launch_assign_pages(ctx, batch, old_len_dev, new_len_dev, page_table_dev, page_table_seq_stride, n_pages, free_pages_dev,
                                  free_state_dev, token_start_dev, n_tokens, slot_map_dev, positions_dev, static_cast<cudaStream_t>(stream));
}

extern "C" int pi_qk_norm_rope(pi_ctx* ctx, int64_t n_tokens, int dtype, const void* q_dev, int64_t q_token_stride, const void* k_dev,
                               int64_t k_token_stride, const int32_t* positions_dev, const float* q_weight_dev, const float* k_weight_dev,
                               float eps, const float* inv_freq_dev, int rot_dim, int interleaved, void* q_out_dev, void* k_out_dev,
                               void* stream) {
    if (!ctx || n_tokens < 0 || n_tokens > INT32_MAX) return PI_ERR_INVALID_ARG;
    if (dtype != PI_DTYPE_BF16 && dtype != PI_DTYPE_FP16 && dtype != PI_DTYPE_FP32) return PI_ERR_INVALID_ARG;
    if (rot_dim < 0 || rot_dim > PI_HEAD_DIM || rot_dim % 2) return PI_ERR_UNSUPPORTED_DIM;
    if (interleaved != 0 && interleaved != 1) return PI_ERR_INVALID_ARG;
    if ((rot_dim > 0 && !inv_freq_dev) || (q_weight_dev == nullptr) != (k_weight_dev == nullptr) || !(eps >= 0.f) || !std::isfinite(eps))
        return PI_ERR_INVALID_ARG;
    if (n_tokens == 0) return PI_OK;
    if (!q_dev || !k_dev || !positions_dev || !q_out_dev || !k_out_dev) return PI_ERR_INVALID_ARG;
    if (q_token_stride < static_cast<int64_t>(ctx->cfg.n_q_heads) * PI_HEAD_DIM || k_token_stride < static_cast<int64_t>(ctx->cfg.n_kv_heads) * PI_HEAD_DIM)
        return PI_ERR_INVALID_ARG;
    const int64_t unit = dtype == PI_DTYPE_FP32 ? 4 : 8;           // elements in 16 bytes
    if (q_token_stride % unit || k_token_stride % unit || !pi_aligned16(q_dev) || !pi_aligned16(k_dev) || !pi_aligned16(q_out_dev) ||
        !pi_aligned16(k_out_dev) || (q_weight_dev && (!pi_aligned16(q_weight_dev) || !pi_aligned16(k_weight_dev))))
        return PI_ERR_BAD_ALIGN;
    DeviceGuard guard(ctx->device);
    if (!guard.ok()) return PI_ERR_CUDA;
    return pi_launch_qk_norm_rope(ctx, static_cast<int>(n_tokens), dtype, q_dev, q_token_stride, k_dev, k_token_stride, positions_dev,
                                  q_weight_dev, k_weight_dev, eps, inv_freq_dev, rot_dim, interleaved, q_out_dev, k_out_dev,
                                  static_cast<cudaStream_t>(stream));
}

extern "C" int pi_kv4_store(pi_ctx* ctx, int64_t n_tokens, const void* k_dev, int64_t k_token_stride, int64_t k_head_stride,
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
    return pi_launch_kv4_store(ctx, n_tokens, k_dev, ks, v_dev, vs, static_cast<int>(inner_tokens), slot_map_dev, dst, n_blocks,
                               static_cast<cudaStream_t>(stream));
}

extern "C" int pi_kv4_load(pi_ctx* ctx, int64_t n_out, const void* store, int64_t n_blocks, const int32_t* blocks_dev, void* kv_dev, void* stream) {
    if (!ctx || n_out < 0 || n_blocks < 1 || n_blocks > INT32_MAX) return PI_ERR_INVALID_ARG;
    // one warp a tile, eight to a CTA
    if (n_out > INT32_MAX / (static_cast<int64_t>(ctx->cfg.n_kv_heads) * (ctx->cfg.block_tokens / 16))) return PI_ERR_UNSUPPORTED_DIM;
    if (n_out == 0) return PI_OK;
    if (!store || !kv_dev || (!blocks_dev && n_out > n_blocks)) return PI_ERR_INVALID_ARG;
    if (!pi_aligned16(store) || !pi_aligned16(kv_dev)) return PI_ERR_BAD_ALIGN;
    DeviceGuard guard(ctx->device);
    if (!guard.ok()) return PI_ERR_CUDA;
    void* src = nullptr;
    const int rc = device_view(store, &src);
    if (rc != PI_OK) return rc;
    return pi_launch_kv4_load(ctx, n_out, src, n_blocks, blocks_dev, kv_dev, static_cast<cudaStream_t>(stream));
}

extern "C" int pi_append_kv4(pi_ctx* ctx, int layer, int batch, uint32_t step, const uint32_t* step_dev, const void* k_new_dev,
                             const void* v_new_dev, const int32_t* ctx_len_dev, void* host_kv4_pinned, int64_t host_seq_stride_bytes,
                             const int32_t* page_table_dev, int64_t page_table_seq_stride, int32_t n_pages, void* pool4_dev,
                             int32_t* block_table_dev, int32_t* slot_block_dev, uint32_t* slot_stamp_dev, void* digest_dev, void* stream) {
    if (!valid(ctx, layer, batch)) return PI_ERR_INVALID_ARG;
    if (ctx->cfg.n_local_blocks < 1) return PI_ERR_INVALID_ARG;     // as pi_append_kv: the block being filled must stay resident
    if (!k_new_dev || !v_new_dev || !ctx_len_dev || !host_kv4_pinned || !pool4_dev || !block_table_dev || !slot_block_dev ||
        !slot_stamp_dev || !digest_dev || (!step_dev && step == 0) || host_seq_stride_bytes < 0)
        return PI_ERR_INVALID_ARG;
    if (page_table_dev && (page_table_seq_stride < 1 || n_pages < 1)) return PI_ERR_INVALID_ARG;
    if (!pi_aligned16(k_new_dev) || !pi_aligned16(v_new_dev) || !pi_aligned16(host_kv4_pinned) || !pi_aligned16(pool4_dev) ||
        !pi_aligned16(digest_dev) || host_seq_stride_bytes % 16)
        return PI_ERR_BAD_ALIGN;
    DeviceGuard guard(ctx->device);
    if (!guard.ok()) return PI_ERR_CUDA;
    void* dst = nullptr;
    const int rc = device_view(host_kv4_pinned, &dst);
    if (rc != PI_OK) return rc;
    return pi_launch_append(ctx, ctx->solo_head[layer], batch, step, k_new_dev, v_new_dev, ctx_len_dev, dst,
                            page_table_dev ? 0 : host_seq_stride_bytes, pool4_dev, block_table_dev, slot_block_dev, slot_stamp_dev,
                            digest_dev, page_table_dev, page_table_seq_stride, n_pages, step_dev, 1, static_cast<cudaStream_t>(stream));
}

extern "C" int pi_recall_kv4(pi_ctx* ctx, int layer, int batch, const void* host_kv4_pinned, int64_t host_seq_stride_bytes,
                             const int32_t* page_table_dev, int64_t page_table_seq_stride, int32_t n_pages, void* pool4_dev,
                             const pi_extent* recall_list_dev, int32_t list_capacity, const int32_t* recall_count_dev, void* stream) {
    if (!valid(ctx, layer, batch)) return PI_ERR_INVALID_ARG;
    if (!host_kv4_pinned || !pool4_dev || !recall_list_dev || !recall_count_dev || list_capacity < 1) return PI_ERR_INVALID_ARG;
    if (page_table_dev && (page_table_seq_stride < 1 || n_pages < 1)) return PI_ERR_INVALID_ARG;
    if (host_seq_stride_bytes < 0 || host_seq_stride_bytes % 16 || !pi_aligned16(host_kv4_pinned) || !pi_aligned16(pool4_dev) ||
        !pi_aligned16(recall_list_dev))
        return PI_ERR_BAD_ALIGN;
    DeviceGuard guard(ctx->device);
    if (!guard.ok()) return PI_ERR_CUDA;
    void* src = nullptr;
    const int rc = device_view(host_kv4_pinned, &src);
    if (rc != PI_OK) return rc;
    const int64_t bytes = kv4_block_bytes(ctx->cfg.n_kv_heads, ctx->cfg.block_tokens);
    return pi_launch_recall(ctx, batch, 1, src, page_table_dev ? 0 : host_seq_stride_bytes, pool4_dev, ctx->cfg.pool_slots * bytes,
                            recall_list_dev, list_capacity, recall_count_dev, bytes, bytes, 0, page_table_dev, page_table_seq_stride,
                            n_pages, bytes, static_cast<cudaStream_t>(stream));
}

extern "C" int pi_sparse_decode_attn_kv4(pi_ctx* ctx, int layer, int batch, const void* q_dev, const void* pool4_dev,
                                         const int32_t* sel_slots_dev, const int32_t* sel_blocks_dev, const int32_t* sel_count_dev,
                                         const int32_t* ctx_len_dev, void* out_dev, float* lse_dev, void* stream) {
    if (!valid(ctx, layer, batch)) return PI_ERR_INVALID_ARG;
    if (!q_dev || !pool4_dev || !sel_slots_dev || !sel_blocks_dev || !sel_count_dev || !ctx_len_dev || !out_dev) return PI_ERR_INVALID_ARG;
    if (!pi_aligned16(q_dev) || !pi_aligned16(pool4_dev) || !pi_aligned16(out_dev)) return PI_ERR_BAD_ALIGN;
    DeviceGuard guard(ctx->device);
    if (!guard.ok()) return PI_ERR_CUDA;
    return pi_launch_attn_kv4(ctx, batch, q_dev, pool4_dev, sel_slots_dev, sel_blocks_dev, sel_count_dev, ctx_len_dev, out_dev, lse_dev,
                              static_cast<cudaStream_t>(stream));
}
