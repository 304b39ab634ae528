// train_api.cu -- argument checks of the C entry points around the layer
// (include/slimwise_moe.h): embedding, norm and the head's cross entropy.
#include <cmath>

#include "train.cuh"
#include "vocab.cuh"

using namespace slimwise;

namespace {

bool on(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
int size_of(int32_t dtype) { return dtype == SLIMWISE_DTYPE_BF16 ? 2 : 4; }
bool known(int32_t dtype) { return dtype == SLIMWISE_DTYPE_BF16 || dtype == SLIMWISE_DTYPE_FP32; }

// Rows of `width` elements, `stride` apart.
struct Rows {
  const void *base;
  int32_t dtype;
  int64_t rows, width, stride;
  int64_t bytes() const { return size_of(dtype) * (rows ? (rows - 1) * stride + width : 0); }
};

bool good_stride(int64_t stride, int64_t width) { return stride >= width && stride <= ((int64_t)1 << 40); }

// Whether two of them share memory.  Rows of the same stride that lie between each
// other's do not.
bool overlap(const Rows &x, const Rows &y) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(x.base), b = reinterpret_cast<uintptr_t>(y.base);
  if (!x.base || !y.base || a >= b + y.bytes() || b >= a + x.bytes()) return false;
  const int64_t step = x.stride * size_of(x.dtype);
  if (step != y.stride * size_of(y.dtype)) return true;
  const int64_t apart = ((int64_t)(b - a) % step + step) % step;
  return !(apart >= x.width * size_of(x.dtype) && apart + y.width * size_of(y.dtype) <= step);
}

Rows vec(const void *p, int64_t n) { return {p, SLIMWISE_DTYPE_FP32, 1, n, n}; }

// The checks that the norm's two entry points share; 0 rows are for the caller to see.
int check_norm(int32_t dtype, int32_t rows, int32_t hidden) {
  if (!known(dtype)) return SLIMWISE_ERR_UNSUPPORTED_SHAPE;
  if (rows < 0 || rows > (1 << 20)) return SLIMWISE_ERR_INVALID_ARG;
  if (hidden < 1 || hidden > kRowMax) return SLIMWISE_ERR_UNSUPPORTED_SHAPE;
  return SLIMWISE_OK;
}

int check_table(int32_t rows, int32_t hidden, int32_t vocab) {
  if (rows < 0 || rows > (1 << 20)) return SLIMWISE_ERR_INVALID_ARG;
  if (hidden < 1 || hidden > kRowMax || vocab < 1 || vocab > kEmbedVocabMax)
    return SLIMWISE_ERR_UNSUPPORTED_SHAPE;
  return SLIMWISE_OK;
}

int check_head(int32_t rows, int32_t hidden, int32_t vocab) {
  if (rows < 0 || rows > (1 << 20)) return SLIMWISE_ERR_INVALID_ARG;
  if (hidden < 8 || hidden > kRowMax || hidden % 8 != 0 || vocab < 1 || vocab > kVocabMax)
    return SLIMWISE_ERR_UNSUPPORTED_SHAPE;
  return SLIMWISE_OK;
}

int status(cudaError_t e) { return e == cudaSuccess ? SLIMWISE_OK : SLIMWISE_ERR_CUDA; }

}  // namespace

extern "C" {

int slimwise_embed(const void *table, int32_t dtype, int32_t vocab, int32_t hidden,
                   int64_t row_stride, const int32_t *ids, int32_t rows, float scale, void *out,
                   int64_t out_stride, void *stream) {
  const int rc = check_table(rows, hidden, vocab);
  if (rc) return rc;
  if (!known(dtype)) return SLIMWISE_ERR_UNSUPPORTED_SHAPE;
  if (!good_stride(row_stride, hidden) || !good_stride(out_stride, hidden) || !std::isfinite(scale))
    return SLIMWISE_ERR_INVALID_ARG;
  if (rows == 0) return SLIMWISE_OK;
  if (!table || !ids || !out) return SLIMWISE_ERR_INVALID_ARG;
  if (!on(table, size_of(dtype)) || !on(out, size_of(dtype)) || !on(ids, 4))
    return SLIMWISE_ERR_UNSUPPORTED_SHAPE;
  const Rows o = {out, dtype, rows, hidden, out_stride};
  if (overlap(o, {table, dtype, vocab, hidden, row_stride}) || overlap(o, vec(ids, rows)))
    return SLIMWISE_ERR_INVALID_ARG;
  return status(launch_embed(table, dtype, vocab, hidden, row_stride, ids, rows, scale, out,
                             out_stride, static_cast<cudaStream_t>(stream)));
}

int slimwise_embed_grad_workspace_size(int32_t rows, int32_t hidden, size_t *bytes) {
  const int rc = check_table(rows, hidden, 1);
  if (rc) return rc;
  if (!bytes) return SLIMWISE_ERR_INVALID_ARG;
  *bytes = embed_grad_workspace(rows, hidden);
  return SLIMWISE_OK;
}

int slimwise_embed_grad(const void *grad, int32_t dtype, int32_t rows, int32_t hidden,
                        int64_t row_stride, const int32_t *ids, float scale, void *out,
                        int32_t out_dtype, int32_t vocab, int64_t out_stride, int32_t accumulate,
                        void *stream, void *workspace, size_t workspace_bytes) {
  const int rc = check_table(rows, hidden, vocab);
  if (rc) return rc;
  if (!known(dtype) || !known(out_dtype)) return SLIMWISE_ERR_UNSUPPORTED_SHAPE;
  if (!good_stride(row_stride, hidden) || !good_stride(out_stride, hidden) || !std::isfinite(scale))
    return SLIMWISE_ERR_INVALID_ARG;
  if (rows == 0 && accumulate) return SLIMWISE_OK;
  if (!out || !workspace || (rows > 0 && (!grad || !ids))) return SLIMWISE_ERR_INVALID_ARG;
  if (!on(out, size_of(out_dtype)) || !on(grad, size_of(dtype)) || !on(ids, 4) || !on(workspace, 256))
    return SLIMWISE_ERR_UNSUPPORTED_SHAPE;
  const size_t need = embed_grad_workspace(rows, hidden);
  if (workspace_bytes < need) return SLIMWISE_ERR_WORKSPACE;
  const Rows o = {out, out_dtype, vocab, hidden, out_stride}, g = {grad, dtype, rows, hidden, row_stride};
  const Rows w = vec(workspace, (int64_t)(need / 4)), i = vec(ids, rows);
  if (overlap(o, g) || overlap(o, i) || overlap(w, o) || overlap(w, g) || overlap(w, i))
    return SLIMWISE_ERR_INVALID_ARG;
  return status(launch_embed_grad(grad, dtype, rows, hidden, row_stride, ids, scale, out, out_dtype,
                                  vocab, out_stride, accumulate != 0, workspace,
                                  static_cast<cudaStream_t>(stream)));
}

int slimwise_norm(const void *x, int32_t dtype, int32_t rows, int32_t hidden, int64_t row_stride,
                  const float *weight, const float *bias, int32_t layer, float eps, void *y,
                  int64_t y_stride, float *mean, float *rstd, void *stream) {
  const int rc = check_norm(dtype, rows, hidden);
  if (rc) return rc;
  if (!good_stride(row_stride, hidden) || !good_stride(y_stride, hidden) ||
      !(eps >= 0.0f && eps <= 1e30f))
    return SLIMWISE_ERR_INVALID_ARG;
  if (rows == 0) return SLIMWISE_OK;
  if (!x || !weight || !y || !rstd || (layer != 0) != (mean != nullptr)) return SLIMWISE_ERR_INVALID_ARG;
  if (!on(x, size_of(dtype)) || !on(y, size_of(dtype)) || !on(weight, 4) || !on(bias, 4) ||
      !on(mean, 4) || !on(rstd, 4))
    return SLIMWISE_ERR_UNSUPPORTED_SHAPE;
  const Rows in = {x, dtype, rows, hidden, row_stride}, o = {y, dtype, rows, hidden, y_stride};
  const Rows w = vec(weight, hidden), b = vec(bias, hidden), m = vec(mean, rows), r = vec(rstd, rows);
  if (overlap(o, in) || overlap(o, w) || overlap(o, b) || overlap(o, m) || overlap(o, r) ||
      overlap(m, in) || overlap(r, in) || overlap(m, r) || overlap(m, w) || overlap(r, w) ||
      overlap(m, b) || overlap(r, b))
    return SLIMWISE_ERR_INVALID_ARG;
  return status(launch_norm(x, dtype, rows, hidden, row_stride, weight, bias, layer != 0, eps, y,
                            y_stride, mean, rstd, static_cast<cudaStream_t>(stream)));
}

int slimwise_norm_grad_workspace_size(int32_t rows, int32_t hidden, size_t *bytes) {
  const int rc = check_norm(SLIMWISE_DTYPE_FP32, rows, hidden);
  if (rc) return rc;
  if (!bytes) return SLIMWISE_ERR_INVALID_ARG;
  *bytes = norm_grad_workspace(rows, hidden);
  return SLIMWISE_OK;
}

int slimwise_norm_grad(const void *dy, int64_t dy_stride, const void *x, int32_t dtype, int32_t rows,
                       int32_t hidden, int64_t row_stride, const float *weight, const float *mean,
                       const float *rstd, void *dx, int64_t dx_stride, float *dweight, float *dbias,
                       void *stream, void *workspace, size_t workspace_bytes) {
  const int rc = check_norm(dtype, rows, hidden);
  if (rc) return rc;
  if (!good_stride(dy_stride, hidden) || !good_stride(row_stride, hidden) || !good_stride(dx_stride, hidden))
    return SLIMWISE_ERR_INVALID_ARG;
  if (rows == 0) return SLIMWISE_OK;
  // (the bias has a gradient in layer norm alone)
  if (!dy || !x || !weight || !rstd || !dx || !dweight || !workspace || (dbias && !mean))
    return SLIMWISE_ERR_INVALID_ARG;
  const int size = size_of(dtype);
  if (!on(dy, size) || !on(x, size) || !on(dx, size) || !on(weight, 4) || !on(mean, 4) || !on(rstd, 4) ||
      !on(dweight, 4) || !on(dbias, 4) || !on(workspace, 4))
    return SLIMWISE_ERR_UNSUPPORTED_SHAPE;
  const size_t need = norm_grad_workspace(rows, hidden);
  if (workspace_bytes < need) return SLIMWISE_ERR_WORKSPACE;
  const Rows in[] = {{dy, dtype, rows, hidden, dy_stride}, {x, dtype, rows, hidden, row_stride},
                     vec(weight, hidden), vec(mean, rows), vec(rstd, rows)};
  const Rows to[] = {{dx, dtype, rows, hidden, dx_stride}, vec(dweight, hidden), vec(dbias, hidden),
                     vec(workspace, (int64_t)(need / 4))};
  for (int i = 0; i < 4; ++i) {
    for (const Rows &r : in)
      if (overlap(to[i], r)) return SLIMWISE_ERR_INVALID_ARG;
    for (int j = 0; j < i; ++j)
      if (overlap(to[i], to[j])) return SLIMWISE_ERR_INVALID_ARG;
  }
  return status(launch_norm_grad(dy, dy_stride, x, dtype, rows, hidden, row_stride, weight, mean, rstd,
                                 dx, dx_stride, dweight, dbias, workspace,
                                 static_cast<cudaStream_t>(stream)));
}

int slimwise_linear_loss_workspace_size(int32_t rows, int32_t hidden, int32_t vocab,
                                        int32_t grad_hidden, int32_t grad_weight, size_t *bytes) {
  const int rc = check_head(rows, hidden, vocab);
  if (rc) return rc;
  if (!bytes) return SLIMWISE_ERR_INVALID_ARG;
  *bytes = rows ? linear_loss_workspace(rows, hidden, vocab, grad_hidden != 0, grad_weight != 0) : 0;
  return SLIMWISE_OK;
}

int slimwise_linear_loss(const void *hidden, int64_t hidden_stride, const void *weight,
                         int64_t weight_stride, int32_t rows, int32_t width, int32_t vocab,
                         const int32_t *labels, const float *row_weight, float *row_loss, float *loss,
                         void *grad_hidden, int64_t grad_hidden_stride, void *grad_weight,
                         int32_t grad_weight_dtype, int64_t grad_weight_stride, void *stream,
                         void *workspace, size_t workspace_bytes) {
  const int rc = check_head(rows, width, vocab);
  if (rc) return rc;
  if (!good_stride(hidden_stride, width) || !good_stride(weight_stride, width) ||
      (grad_hidden && !good_stride(grad_hidden_stride, width)) ||
      (grad_weight && !good_stride(grad_weight_stride, width)))
    return SLIMWISE_ERR_INVALID_ARG;
  if (grad_weight && !known(grad_weight_dtype)) return SLIMWISE_ERR_UNSUPPORTED_SHAPE;
  if (rows == 0) return SLIMWISE_OK;
  if (!hidden || !weight || !labels || !row_loss || !workspace) return SLIMWISE_ERR_INVALID_ARG;
  // TMA copies and 16-byte accesses: rows start on 16-byte boundaries
  const int gw = grad_weight ? 16 / size_of(grad_weight_dtype) : 1;
  if (hidden_stride % 8 || weight_stride % 8 || (grad_hidden && grad_hidden_stride % 8) ||
      (grad_weight && grad_weight_stride % gw) || !on(hidden, 16) || !on(weight, 16) ||
      !on(grad_hidden, 16) || !on(grad_weight, 16) || !on(labels, 4) || !on(row_weight, 4) ||
      !on(row_loss, 4) || !on(loss, 4) || !on(workspace, 256))
    return SLIMWISE_ERR_UNSUPPORTED_SHAPE;
  const size_t need = linear_loss_workspace(rows, width, vocab, grad_hidden != nullptr, grad_weight != nullptr);
  if (workspace_bytes < need) return SLIMWISE_ERR_WORKSPACE;
  const int32_t bf16 = SLIMWISE_DTYPE_BF16;
  const Rows in[] = {{hidden, bf16, rows, width, hidden_stride}, {weight, bf16, vocab, width, weight_stride},
                     vec(labels, rows), vec(row_weight, rows)};
  const Rows to[] = {{grad_hidden, bf16, rows, width, grad_hidden_stride},
                     {grad_weight, grad_weight_dtype, vocab, width, grad_weight_stride},
                     vec(row_loss, rows), vec(loss, 1), vec(workspace, (int64_t)(need / 4))};
  for (int i = 0; i < 5; ++i) {
    for (const Rows &r : in)
      if (overlap(to[i], r)) return SLIMWISE_ERR_INVALID_ARG;
    for (int j = 0; j < i; ++j)
      if (overlap(to[i], to[j])) return SLIMWISE_ERR_INVALID_ARG;
  }
  const LinearLossArgs a = {hidden, hidden_stride, weight, weight_stride, rows, width, vocab, labels,
                            row_weight, row_loss, loss, grad_hidden, grad_hidden_stride, grad_weight,
                            grad_weight_dtype, grad_weight_stride};
  return status(launch_linear_loss(a, workspace, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
