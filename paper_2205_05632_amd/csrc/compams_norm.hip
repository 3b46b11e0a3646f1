// The C ABI of the layer norm and of the join of a transformer block: checks of arguments.
#include <math.h>

#include <initializer_list>

#include "compams_norm.h"

namespace compams {
namespace {

bool any_gradient(const compams_norm& a) { return a.dgamma || a.dbeta || a.dbias; }

bool norm_valid(const compams_norm* a, bool join) {
  return a && rows_valid(a->n, a->rows, a->cols) && float_type(a->type) &&
         (a->stream_type == a->type || a->stream_type == COMPAMS_F32) && a->eps >= 0.0f && isfinite(a->eps) &&
         (!join || drop_valid(a->drop));
}

// A matrix: 0 if it is in order (or not there), else the status.
int check_matrix(const void* p, int64_t ld, const compams_norm& a, int32_t type) {
  if (!p) return COMPAMS_OK;
  if (!stride_valid(ld, a.cols)) return COMPAMS_INVALID_ARG;
  return aligned_to(p, type_size(type)) ? COMPAMS_OK : COMPAMS_BAD_ALIGNMENT;
}
int check_vectors(const compams_norm& a, bool join) {
  const float* const all[] = {a.gamma, a.beta, a.bias, a.mean, a.rstd};
  for (const float* p : all)
    if (!aligned_to(p, 4)) return COMPAMS_BAD_ALIGNMENT;
  return join && !aligned_to(a.drop.step, 8) ? COMPAMS_BAD_ALIGNMENT : COMPAMS_OK;
}
int first_bad(std::initializer_list<int> all) {
  for (int s : all)
    if (s != COMPAMS_OK) return s;
  return COMPAMS_OK;
}

NormArgs make_args(const compams_norm& a, bool join) {
  NormArgs k = {};
  k.n = static_cast<uint32_t>(a.n);
  k.rows = static_cast<uint32_t>(a.rows);
  k.cols = static_cast<uint32_t>(a.cols);
  k.count.n = static_cast<float>(k.cols);
  k.count.inverse = 1.0f / k.count.n;
  k.total = k.n * k.rows;
  k.eps = a.eps;
  k.join = join;
  if (join) k.drop = make_drop(a.drop);
  k.gamma = a.gamma; k.beta = a.beta; k.bias = join ? a.bias : nullptr;
  k.x = a.x; k.residual = a.residual; k.h = a.h; k.y = a.y; k.mean = a.mean; k.rstd = a.rstd;
  k.ld_x = a.ld_x; k.ld_residual = a.ld_residual; k.ld_h = a.ld_h; k.ld_y = a.ld_y;
  k.dy = a.dy; k.dh = join ? a.dh : nullptr; k.dx = join ? a.dx : nullptr; k.dresidual = a.dresidual;
  k.ld_dy = a.ld_dy; k.ld_dh = a.ld_dh; k.ld_dx = a.ld_dx; k.ld_dresidual = a.ld_dresidual;
  k.grad[0] = a.dgamma; k.grad[1] = a.dbeta; k.grad[2] = join ? a.dbias : nullptr;
  k.ld_grad[0] = a.ld_dgamma; k.ld_grad[1] = a.ld_dbeta; k.ld_grad[2] = a.ld_dbias;
  k.accumulate = a.accumulate != 0;
  return k;
}

int forward(const compams_norm* a, bool join, hipStream_t stream) {
  if (!norm_valid(a, join)) return COMPAMS_INVALID_ARG;
  if (a->rows == 0) return COMPAMS_OK;
  if (!a->y || (join ? !a->x : !a->h)) return COMPAMS_INVALID_ARG;
  if (!join && (a->x || a->residual || a->bias)) return COMPAMS_INVALID_ARG;
  const int bad = first_bad({check_matrix(a->x, a->ld_x, *a, a->type), check_matrix(a->h, a->ld_h, *a, a->stream_type),
                             check_matrix(a->residual, a->ld_residual, *a, a->stream_type),
                             check_matrix(a->y, a->ld_y, *a, a->type), check_vectors(*a, join)});
  if (bad != COMPAMS_OK) return bad;
  const hipError_t err = norm_forward(make_args(*a, join), a->type, a->stream_type, stream);
  return err == hipSuccess ? COMPAMS_OK : COMPAMS_HIP_ERROR;
}

int backward(const compams_norm* a, bool join, hipStream_t stream) {
  if (!norm_valid(a, join) || (a->accumulate != 0 && a->accumulate != 1)) return COMPAMS_INVALID_ARG;
  if (!join && (a->dx || a->dh || a->dbias)) return COMPAMS_INVALID_ARG;
  if (!any_gradient(*a) && !a->dresidual && !a->dx) return COMPAMS_INVALID_ARG;
  NormArgs k = make_args(*a, join);
  for (uint32_t i = 0; i < kGradients; ++i) {
    if (!k.grad[i]) continue;
    if (a->n > 1 && (k.ld_grad[i] < a->cols || k.ld_grad[i] >= (static_cast<int64_t>(1) << 40))) return COMPAMS_INVALID_ARG;
    if (!aligned_to(k.grad[i], 4)) return COMPAMS_BAD_ALIGNMENT;
  }
  if (a->rows > 0) {
    if (!a->dy || !a->h || !a->mean || !a->rstd) return COMPAMS_INVALID_ARG;
    const int bad = first_bad({check_matrix(a->dy, a->ld_dy, *a, a->type), check_matrix(a->h, a->ld_h, *a, a->stream_type),
                               check_matrix(k.dh, a->ld_dh, *a, a->stream_type), check_matrix(k.dx, a->ld_dx, *a, a->type),
                               check_matrix(a->dresidual, a->ld_dresidual, *a, a->stream_type), check_vectors(*a, join)});
    if (bad != COMPAMS_OK) return bad;
  }
  const Cut cut = norm_cut(k.n, k.rows, k.cols, join, any_gradient(*a));
  if (cut.sums_bytes + cut.partial_bytes > 0) {
    if (!a->workspace) return COMPAMS_INVALID_ARG;
    if (!aligned_to(a->workspace, 256)) return COMPAMS_BAD_ALIGNMENT;
    if (a->workspace_bytes < cut.sums_bytes + cut.partial_bytes) return COMPAMS_WORKSPACE_TOO_SMALL;
  }
  k.sums = static_cast<float2*>(a->workspace);
  k.partial = reinterpret_cast<float*>(static_cast<char*>(a->workspace) + cut.sums_bytes);
  k.parts = cut.parts;
  k.part_rows = cut.part_rows;
  const hipError_t err = norm_backward(k, a->type, a->stream_type, stream);
  return err == hipSuccess ? COMPAMS_OK : COMPAMS_HIP_ERROR;
}

}  // namespace
}  // namespace compams

extern "C" {

size_t compams_norm_workspace_size(const compams_norm* a) {
  if (!compams::norm_valid(a, false)) return 0;
  // (for either of the two calls)
  size_t most = 0;
  for (const bool join : {false, true}) {
    const compams::Cut c = compams::norm_cut(static_cast<uint32_t>(a->n), static_cast<uint32_t>(a->rows),
                                             static_cast<uint32_t>(a->cols), join, compams::any_gradient(*a));
    if (c.sums_bytes + c.partial_bytes > most) most = c.sums_bytes + c.partial_bytes;
  }
  return most;
}
int compams_layer_norm_forward(const compams_norm* a, void* hip_stream) {
  return compams::forward(a, false, static_cast<hipStream_t>(hip_stream));
}
int compams_layer_norm_backward(const compams_norm* a, void* hip_stream) {
  return compams::backward(a, false, static_cast<hipStream_t>(hip_stream));
}
int compams_dropout_add_norm_forward(const compams_norm* a, void* hip_stream) {
  return compams::forward(a, true, static_cast<hipStream_t>(hip_stream));
}
int compams_dropout_add_norm_backward(const compams_norm* a, void* hip_stream) {
  return compams::backward(a, true, static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
