// C-ABI entry point of the attention over packed prompts.
#include "pi_api_guard.cuh"

extern "C" int pi_prompt_attn(pi_ctx* ctx, int n_seqs, int dtype, int64_t n_q, const void* q_dev, int64_t q_token_stride, int64_t q_head_stride,
                              int64_t n_k, const void* k_dev, int64_t k_token_stride, int64_t k_head_stride, const void* v_dev,
                              int64_t v_token_stride, int64_t v_head_stride, const int32_t* q_start_dev, const int32_t* k_start_dev, void* out_dev,
                              float* lse_dev, void* stream) {
    if (!valid(ctx, 0, n_seqs)) return PI_ERR_INVALID_ARG;
    if (dtype != PI_DTYPE_BF16 && dtype != PI_DTYPE_FP16) return PI_ERR_INVALID_ARG;
    // (tile coordinates run past the last token by less than a tile, and stay in 32 bits)
    constexpr int64_t most = INT32_MAX - 256, widest = (int64_t(1) << 39) / (2 * 16);
    if (n_q < 0 || n_q > most || n_k < 0 || n_k > most) return PI_ERR_INVALID_ARG;
    if (n_q == 0) return PI_OK;
    if (!q_dev || !q_start_dev || !out_dev || (n_k > 0 && (!k_dev || !v_dev))) return PI_ERR_INVALID_ARG;
    const int64_t strides[6] = {q_token_stride, q_head_stride, k_token_stride, k_head_stride, v_token_stride, v_head_stride};
    for (int i = 0; i < (n_k ? 6 : 2); ++i) {
        if (strides[i] < 8 || strides[i] > widest) return PI_ERR_INVALID_ARG;
        if (strides[i] % 8) return PI_ERR_BAD_ALIGN;
    }
    if (!pi_aligned16(q_dev) || !pi_aligned16(out_dev) || (n_k > 0 && (!pi_aligned16(k_dev) || !pi_aligned16(v_dev)))) return PI_ERR_BAD_ALIGN;
    DeviceGuard guard(ctx->device);
    if (!guard.ok()) return PI_ERR_CUDA;
    return pi_launch_prompt_attn(ctx, n_seqs, dtype, static_cast<int>(n_q), static_cast<int>(n_k), q_dev, q_token_stride, q_head_stride, k_dev,
                                 n_k ? k_token_stride : PI_HEAD_DIM, n_k ? k_head_stride : PI_HEAD_DIM, v_dev, n_k ? v_token_stride : PI_HEAD_DIM,
                                 n_k ? v_head_stride : PI_HEAD_DIM, q_start_dev, k_start_dev ? k_start_dev : q_start_dev, out_dev, lse_dev,
                                 static_cast<cudaStream_t>(stream));
}
