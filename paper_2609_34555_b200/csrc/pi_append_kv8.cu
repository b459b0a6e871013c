// Append of the decode step's new token to a cache in 8 bits (the kernel: pi_append_core.cuh).
#include "pi_append_core.cuh"

int pi_launch_append_kv8(pi_ctx* c, int h_star, int batch, uint32_t step, const uint32_t* step_dev, const void* k_new, const void* v_new,
                         const int32_t* ctx_len, void* host_kv, int64_t host_stride, void* pool, int32_t* table, int32_t* slot_block,
                         uint32_t* slot_stamp, void* digest, const int32_t* page_table, int64_t page_stride, int32_t n_pages, cudaStream_t stream) {
    AppendParams p;
    append_params(p, c, h_star, step, step_dev, k_new, v_new, ctx_len, host_kv, host_stride, pool, table, slot_block, slot_stamp, digest,
                  page_table, page_stride, n_pages, kv8_block_bytes(c->cfg.n_kv_heads, c->cfg.block_tokens));
    PI_CUDA_TRY(pi_launch_pdl(append_kernel<8>, dim3(batch), dim3(APPEND_THREADS), 0, stream, p));
    PI_CUDA_TRY(cudaGetLastError());
    return PI_OK;
}
