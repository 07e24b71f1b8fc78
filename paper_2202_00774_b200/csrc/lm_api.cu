// extern "C" entry points of the operators around a language model's linear layers: argument validation and dispatch.
#include "sdgp_internal.cuh"

namespace {

bool aligned(const void* p, size_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

bool valid_dtype(sdgp_dtype d) { return d == SDGP_BF16 || d == SDGP_FP16 || d == SDGP_FP32; }

sdgp_status status_of(cudaError_t e) { return e == cudaSuccess ? SDGP_OK : SDGP_ERR_CUDA; }

// The compressed pruned copy that a gradient pass writes beside (or instead of) dL/dO [rows, K].
sdgp_status check_compressed(const void* values, const void* meta, int64_t K, int n, int m, int scheme, sdgp_dtype dtype) {
  if (!values && !meta) return SDGP_OK;
  if (scheme < 0 || scheme > 2 || m < 1 || m > 32 || n < 1 || n > m) return SDGP_ERR_INVALID_ARG;
  if (m != 4 && m != 8 && m != 16 && m != 32) return SDGP_ERR_UNSUPPORTED;
  if (K % m != 0) return SDGP_ERR_INVALID_ARG;
  if (n > 2 || dtype == SDGP_FP32) return SDGP_ERR_UNSUPPORTED;
  if (K % 16 != 0 || !aligned(values, 16) || !aligned(meta, 16)) return SDGP_ERR_ALIGNMENT;
  return SDGP_OK;
}

}  // namespace

extern "C" {

sdgp_status sdgp_token_logprob(const void* logits, const int64_t* targets, int64_t rows, int64_t K, int64_t classes, sdgp_dtype dtype,
                               int top, float* logprob, float* entropy, float* lse, float* top_logprob, int64_t* top_token,
                               void* stream) {
  if (!valid_dtype(dtype) || rows < 0 || classes < 1 || classes > K || top < 0 || top > classes) return SDGP_ERR_INVALID_ARG;
  if (top > 32 || K > 0x7FFFFFFF || rows > 0x7FFFFFFF) return SDGP_ERR_UNSUPPORTED;
  if (rows == 0) return SDGP_OK;
  if (!logits || !targets || !logprob) return SDGP_ERR_INVALID_ARG;
  if (!aligned(logits, 16) || !aligned(targets, 8) || !aligned(logprob, 4) || !aligned(entropy, 4) || !aligned(lse, 4) ||
      !aligned(top_logprob, 4) || !aligned(top_token, 8))
    return SDGP_ERR_ALIGNMENT;
  if (!top_logprob && !top_token) top = 0;
  return status_of(sdgp::launch_token_logprob(logits, targets, rows, K, classes, (int)dtype, top, logprob, entropy, lse, top_logprob,
                                              top_token, (cudaStream_t)stream));
}

sdgp_status sdgp_token_logprob_backward(const void* logits, const int64_t* targets, const float* lse, const float* entropy,
                                        const float* d_logprob, const float* d_entropy, int64_t rows, int64_t K, int64_t classes, int n,
                                        int m, sdgp_scheme scheme, uint64_t seed, sdgp_dtype dtype, void* grad, void* values, void* meta,
                                        void* stream) {
  if (!valid_dtype(dtype) || rows < 0 || classes < 1 || classes > K) return SDGP_ERR_INVALID_ARG;
  if (K > 0x7FFFFFFF || rows > 0x7FFFFFFF) return SDGP_ERR_UNSUPPORTED;
  const sdgp_status st = check_compressed(values, meta, K, n, m, (int)scheme, dtype);
  if (st != SDGP_OK) return st;
  if (rows == 0 || (!grad && !values && !meta)) return SDGP_OK;
  if (!logits || !targets || !lse || (d_entropy && !entropy)) return SDGP_ERR_INVALID_ARG;
  if (!aligned(logits, 16) || !aligned(grad, 16) || !aligned(targets, 8) || !aligned(lse, 4) || !aligned(entropy, 4) ||
      !aligned(d_logprob, 4) || !aligned(d_entropy, 4))
    return SDGP_ERR_ALIGNMENT;
  if ((rows * K) / 4096 >= 0x7FFFFFFF) return SDGP_ERR_UNSUPPORTED;
  return status_of(sdgp::launch_token_logprob_backward(logits, targets, lse, entropy, d_logprob, d_entropy, rows, K, classes, n, m,
                                                       (int)scheme, seed, (int)dtype, grad, values, meta, (cudaStream_t)stream));
}

static sdgp_status check_norm(int64_t rows, int64_t C, int64_t groups, sdgp_dtype dtype) {
  if (!valid_dtype(dtype) || rows < 0 || C < 1 || groups < 0) return SDGP_ERR_INVALID_ARG;
  if (groups == 0 ? rows != 0 : rows % groups != 0) return SDGP_ERR_INVALID_ARG;  // (no rows may have a gate each)
  if (rows > (int64_t)1 << 28 || C > (int64_t)1 << 24) return SDGP_ERR_UNSUPPORTED;
  return SDGP_OK;
}

sdgp_status sdgp_residual_norm(const void* branch, const void* residual, const void* post_weight, const void* gate, const void* pre_weight,
                               int64_t rows, int64_t C, int64_t groups, float alpha, float eps, sdgp_dtype dtype, void* out, void* y,
                               float* post_rstd, float* pre_rstd, void* stream) {
  const sdgp_status st = check_norm(rows, C, groups, dtype);
  if (st != SDGP_OK || rows == 0) return st;
  if (!branch || !residual || !out || (pre_weight && !y) || (!pre_weight && y)) return SDGP_ERR_INVALID_ARG;
  for (const void* p : {branch, residual, post_weight, gate, pre_weight, (const void*)out, (const void*)y})
    if (!aligned(p, 16)) return SDGP_ERR_ALIGNMENT;
  if (!aligned(post_rstd, 4) || !aligned(pre_rstd, 4)) return SDGP_ERR_ALIGNMENT;
  return status_of(sdgp::launch_residual_norm(branch, residual, post_weight, gate, pre_weight, rows, C, gate ? groups : 1, alpha, eps,
                                              (int)dtype, out, y, post_rstd, pre_rstd, (cudaStream_t)stream));
}

size_t sdgp_workspace_size_residual_norm_backward(int64_t rows, int64_t C, int64_t groups) {
  if (check_norm(rows, C, groups, SDGP_BF16) != SDGP_OK || rows == 0) return 0;
  return (sdgp::residual_norm_backward_floats(rows, C, groups) * sizeof(float) + 255) / 256 * 256;
}

sdgp_status sdgp_residual_norm_backward(const void* branch, const void* out, const void* d_out, const void* d_y, const void* post_weight,
                                        const void* gate, const void* pre_weight, const float* post_rstd, const float* pre_rstd,
                                        int64_t rows, int64_t C, int64_t groups, float alpha, int n, int m, sdgp_scheme scheme,
                                        uint64_t seed, sdgp_dtype dtype, void* d_residual, void* d_branch, float* d_gate,
                                        float* d_post_weight, float* d_pre_weight, void* values, void* meta, void* workspace,
                                        size_t workspace_bytes, void* stream) {
  sdgp_status st = check_norm(rows, C, groups, dtype);
  if (st == SDGP_OK) st = check_compressed(values, meta, C, n, m, (int)scheme, dtype);
  if (st != SDGP_OK) return st;
  if ((d_gate && !gate) || (d_post_weight && !post_weight) || (d_pre_weight && !pre_weight)) return SDGP_ERR_INVALID_ARG;
  for (const float* p : {post_rstd, pre_rstd, (const float*)d_gate, (const float*)d_post_weight, (const float*)d_pre_weight})
    if (!aligned(p, 4)) return SDGP_ERR_ALIGNMENT;
  if (rows == 0) {  // sums over no rows
    cudaError_t e = cudaSuccess;
    for (float* p : {d_gate, d_post_weight, d_pre_weight})
      if (p && e == cudaSuccess) e = cudaMemsetAsync(p, 0, (size_t)C * (p == d_gate ? (size_t)groups : 1) * sizeof(float), (cudaStream_t)stream);
    return status_of(e);
  }
  if (!branch || (!d_out && !d_y) || (post_weight && !post_rstd)) return SDGP_ERR_INVALID_ARG;
  if (d_y ? !out || !pre_weight || !pre_rstd : d_pre_weight != nullptr) return SDGP_ERR_INVALID_ARG;
  for (const void* p : {branch, out, d_out, d_y, post_weight, gate, pre_weight, (const void*)d_residual, (const void*)d_branch})
    if (!aligned(p, 16)) return SDGP_ERR_ALIGNMENT;
  if (!workspace || !aligned(workspace, 256) || workspace_bytes < sdgp_workspace_size_residual_norm_backward(rows, C, groups))
    return SDGP_ERR_WORKSPACE;
  return status_of(sdgp::launch_residual_norm_backward(branch, out, d_out, d_y, post_weight, gate, pre_weight, post_rstd, pre_rstd, rows, C,
                                                       groups, alpha, n, m, (int)scheme, seed, (int)dtype, d_residual, d_branch, d_gate,
                                                       d_post_weight, d_pre_weight, values, meta, (float*)workspace,
                                                       (cudaStream_t)stream));
}

sdgp_status sdgp_fp8_quantize(const void* x, int64_t rows, int64_t K, int block_rows, sdgp_dtype dtype, void* q, float* scale, void* stream) {
  if (!valid_dtype(dtype) || rows < 0 || K < 0) return SDGP_ERR_INVALID_ARG;
  if ((block_rows != 1 && block_rows != 128) || rows > 0x7FFFFFFF || K > 0x7FFFFFFF) return SDGP_ERR_UNSUPPORTED;
  if (rows == 0 || K == 0) return SDGP_OK;
  if (!x || !q || !scale) return SDGP_ERR_INVALID_ARG;
  if (K % 16 != 0 || !aligned(x, 16) || !aligned(q, 16) || !aligned(scale, 4)) return SDGP_ERR_ALIGNMENT;
  // (the grid: a CTA takes 64 blocks of rows, or one square)
  const int64_t blocks = (K + 127) / 128;
  if ((block_rows == 128 ? (rows + 127) / 128 * blocks : rows * blocks / 64) >= 0x7FFFFFFF) return SDGP_ERR_UNSUPPORTED;
  return status_of(sdgp::launch_fp8_quantize(x, rows, K, block_rows, (int)dtype, q, scale, (cudaStream_t)stream));
}

sdgp_status sdgp_fp8_linear(const void* xq, const float* x_scale, const void* wq, const float* w_scale, void* y, int64_t rows,
                            int64_t features, int64_t K, sdgp_dtype dtype, void* stream) {
  if (!valid_dtype(dtype) || rows < 0 || features < 0 || K < 1) return SDGP_ERR_INVALID_ARG;
  if (rows > 0x7FFFFF00 || features > 0x7FFFFF00 || K > 0x7FFFFF00) return SDGP_ERR_UNSUPPORTED;
  if (rows == 0 || features == 0) return SDGP_OK;
  if (!xq || !x_scale || !wq || !w_scale || !y) return SDGP_ERR_INVALID_ARG;
  if (K % 16 != 0 || !aligned(xq, 16) || !aligned(wq, 16) || !aligned(y, 16) || !aligned(x_scale, 4) || !aligned(w_scale, 4))
    return SDGP_ERR_ALIGNMENT;
  return sdgp::launch_fp8_linear(xq, x_scale, wq, w_scale, y, rows, features, K, (int)dtype, (cudaStream_t)stream);
}

}  // extern "C"
