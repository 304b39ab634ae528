// vocab_api.cu -- argument checks of the C entry points over vocabulary logits
// (include/slimwise_moe.h), which hold no state and need no workspace.
#include <cmath>

#include "vocab.cuh"

using namespace slimwise;

namespace {

bool on(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// The checks that the three share.  0 rows are a no-op for the caller to see.
int check_rows(const void *logits, int32_t dtype, int32_t rows, int32_t vocab, int64_t stride) {
  if (dtype != SLIMWISE_DTYPE_BF16 && dtype != SLIMWISE_DTYPE_FP32)
    return SLIMWISE_ERR_UNSUPPORTED_SHAPE;
  if (rows < 0 || rows > (1 << 20)) return SLIMWISE_ERR_INVALID_ARG;
  if (vocab < 1 || vocab > kVocabMax) return SLIMWISE_ERR_UNSUPPORTED_SHAPE;
  if (stride < vocab || stride > ((int64_t)1 << 40)) return SLIMWISE_ERR_INVALID_ARG;
  if (rows == 0) return SLIMWISE_OK;
  if (!logits) return SLIMWISE_ERR_INVALID_ARG;
  return on(logits, dtype == SLIMWISE_DTYPE_BF16 ? 2 : 4) ? SLIMWISE_OK
                                                          : SLIMWISE_ERR_UNSUPPORTED_SHAPE;
}

bool good_temperature(float t) { return t >= 1e-6f && t <= 1e6f; }

int status(cudaError_t e) { return e == cudaSuccess ? SLIMWISE_OK : SLIMWISE_ERR_CUDA; }

}  // namespace

extern "C" {

int slimwise_top_logits(const void *logits, int32_t dtype, int32_t rows, int32_t vocab,
                        int64_t row_stride, int32_t k, float temperature, int32_t *ids,
                        float *logp, float *log_rest, void *stream) {
  int rc = check_rows(logits, dtype, rows, vocab, row_stride);
  if (rc) return rc;
  if (k < 1 || k > kTopMax || k > vocab || !good_temperature(temperature))
    return SLIMWISE_ERR_INVALID_ARG;
  if (rows == 0) return SLIMWISE_OK;
  if (!ids || !logp || !log_rest) return SLIMWISE_ERR_INVALID_ARG;
  if (!on(ids, 4) || !on(logp, 4) || !on(log_rest, 4)) return SLIMWISE_ERR_UNSUPPORTED_SHAPE;
  return status(launch_top_logits(logits, dtype, rows, vocab, row_stride, k, temperature, ids,
                                  logp, log_rest, static_cast<cudaStream_t>(stream)));
}

int slimwise_distill_loss(const void *logits, int32_t dtype, int32_t rows, int32_t vocab,
                          int64_t row_stride, const int32_t *labels, const int32_t *top_ids,
                          const float *top_logp, const float *log_rest, int32_t k, float alpha,
                          float temperature, const float *row_weight, float *row_loss,
                          float *loss, void *grad, int64_t grad_stride, void *stream) {
  int rc = check_rows(logits, dtype, rows, vocab, row_stride);
  if (rc) return rc;
  if (k < 1 || k > kTopMax || k > vocab || !good_temperature(temperature) ||
      !(alpha >= 0.0f && alpha <= 1.0f))
    return SLIMWISE_ERR_INVALID_ARG;
  if (grad && (grad_stride < vocab || grad_stride > ((int64_t)1 << 40)))
    return SLIMWISE_ERR_INVALID_ARG;
  if (rows == 0) return SLIMWISE_OK;
  if (!labels || !top_ids || !top_logp || !log_rest || !row_loss) return SLIMWISE_ERR_INVALID_ARG;
  const int size = dtype == SLIMWISE_DTYPE_BF16 ? 2 : 4;
  if (!on(labels, 4) || !on(top_ids, 4) || !on(top_logp, 4) || !on(log_rest, 4) ||
      !on(row_weight, 4) || !on(row_loss, 4) || !on(loss, 4) || !on(grad, (uintptr_t)size))
    return SLIMWISE_ERR_UNSUPPORTED_SHAPE;
  if (grad && !(grad == logits && grad_stride == row_stride)) {
    // in place means every row in place; any other overlap would be read after it was written
    const uintptr_t a = reinterpret_cast<uintptr_t>(logits), b = reinterpret_cast<uintptr_t>(grad);
    const uintptr_t an = (uintptr_t)size * ((uintptr_t)(rows - 1) * row_stride + vocab);
    const uintptr_t bn = (uintptr_t)size * ((uintptr_t)(rows - 1) * grad_stride + vocab);
    // (rows of one buffer beside each other do not overlap: the same stride, columns apart)
    const int64_t step = size * row_stride, row = size * (int64_t)vocab;
    const int64_t apart = ((int64_t)(b - a) % step + step) % step;
    const bool beside = grad_stride == row_stride && apart >= row && apart + row <= step;
    if (a < b + bn && b < a + an && !beside) return SLIMWISE_ERR_INVALID_ARG;
  }
  return status(launch_distill_loss(logits, dtype, rows, vocab, row_stride, labels, top_ids,
                                    top_logp, log_rest, k, alpha, temperature, row_weight,
                                    row_loss, loss, grad, grad_stride,
                                    static_cast<cudaStream_t>(stream)));
}

int slimwise_sample(const void *logits, int32_t dtype, int32_t rows, int32_t vocab,
                    int64_t row_stride, const float *temperature, const int32_t *top_k,
                    const float *top_p, const float *min_p, const float *uniform,
                    int32_t *tokens, float *logprob, void *stream) {
  int rc = check_rows(logits, dtype, rows, vocab, row_stride);
  if (rc) return rc;
  if (rows == 0) return SLIMWISE_OK;
  if (!uniform || !tokens || !logprob) return SLIMWISE_ERR_INVALID_ARG;
  if (!on(temperature, 4) || !on(top_k, 4) || !on(top_p, 4) || !on(min_p, 4) ||
      !on(uniform, 4) || !on(tokens, 4) || !on(logprob, 4))
    return SLIMWISE_ERR_UNSUPPORTED_SHAPE;
  return status(launch_sample(logits, dtype, rows, vocab, row_stride, temperature, top_k, top_p,
                              min_p, uniform, tokens, logprob,
                              static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
