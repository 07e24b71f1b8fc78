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

}  // extern "C"
