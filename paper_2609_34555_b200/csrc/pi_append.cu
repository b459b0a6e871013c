// Append of the decode step's new token: K/V rows into the pool slot of the current block
// and, through the mapped pinned pointer, into the host store; running min / max of the
// retrieval head's digest; a pool slot for a block that has just been opened.  One CTA per
// sequence; a few KB per sequence, latency-bound.
#include "pi_append_core.cuh"

int pi_launch_append(pi_ctx* c, int h_star, int batch, uint32_t step, const void* k_new, const void* v_new,
                     const int32_t* ctx_len, void* host_kv, int64_t host_stride, void* pool, int32_t* table,
                     int32_t* slot_block, uint32_t* slot_stamp, void* digest, const int32_t* page_table,
                     int64_t page_stride, int32_t n_pages, const uint32_t* step_dev, int kv4, cudaStream_t stream) {
    AppendParams p;
    const int64_t block_bytes = kv4 ? kv4_block_bytes(c->cfg.n_kv_heads, c->cfg.block_tokens)
                                    : static_cast<int64_t>(c->cfg.n_kv_heads) * 2 * c->cfg.block_tokens * PI_HEAD_DIM * 2;
    append_params(p, c, h_star, step, step_dev, k_new, v_new, ctx_len, host_kv, host_stride, pool, table, slot_block, slot_stamp, digest,
                  page_table, page_stride, n_pages, block_bytes);
    PI_CUDA_TRY(pi_launch_pdl(kv4 ? append_kernel<4> : append_kernel<16>, dim3(batch), dim3(APPEND_THREADS), 0, stream, p));
    PI_CUDA_TRY(cudaGetLastError());
    return PI_OK;
}
