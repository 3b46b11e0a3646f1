// Layer norm and the join of a transformer block (bias, dropout, residual add, layer norm), forward and backward, with the
// gradients of the weights per worker.
#include <math.h>

#include <initializer_list>

#include "compams_rows.h"

namespace compams {
namespace {

constexpr uint32_t kGradients = 3;  // dgamma, dbeta, dbias

struct NormArgs {
  uint32_t n, rows, cols;  // workers, rows of each, columns
  uint32_t total;          // n * rows
  float eps;
  bool join;
  Drop drop;
  const float *gamma, *beta, *bias;
  const void *x, *residual, *dy, *dh;
  void *h, *y, *dx, *dresidual;
  int64_t ld_x, ld_residual, ld_h, ld_y, ld_dy, ld_dh, ld_dx, ld_dresidual;
  float *mean, *rstd;
  float* grad[kGradients];
  int64_t ld_grad[kGradients];
  bool accumulate;
  float2* sums;       // per row: sum(u) / C and sum(u z) / C, on the route of wide rows
  float* partial;     // [worker][part][which gradient][column]
  uint32_t parts;     // parts that a worker's rows are summed in
  uint32_t part_rows; // rows of a part
};

template <typename T>
__device__ __forceinline__ const T* row_of(const void* base, int64_t ld, uint32_t r) {
  return static_cast<const T*>(base) + static_cast<int64_t>(r) * ld;
}
template <typename T>
__device__ __forceinline__ T* row_of(void* base, int64_t ld, uint32_t r) {
  return static_cast<T*>(base) + static_cast<int64_t>(r) * ld;
}

// A weight's group, or the value that stands for one that is not there.
__device__ __forceinline__ void load_weight(float (&v)[kGroup], const float* w, uint32_t c, uint32_t cols, float absent) {
  if (w) {
    load_group(v, w, c, cols);
  } else {
#pragma unroll
    for (uint32_t j = 0; j < kGroup; ++j) v[j] = absent;
  }
}

// h of a group before it is rounded: the input of a layer norm, or residual + dropout(x + bias).
template <typename T, typename H>
__device__ __forceinline__ void form_h(float (&v)[kGroup], const NormArgs& a, uint64_t offset, uint32_t r, uint32_t c) {
  if (!a.join) {
    load_group(v, row_of<H>(static_cast<const void*>(a.h), a.ld_h, r), c, a.cols);
    return;
  }
  float w[kGroup];
  load_group(v, row_of<T>(a.x, a.ld_x, r), c, a.cols);
  load_weight(w, a.bias, c, a.cols, 0.0f);
#pragma unroll
  for (uint32_t j = 0; j < kGroup; ++j) v[j] += w[j];
  drop_group(v, a.drop, offset, r, c);
  if (a.residual) {
    load_group(w, row_of<H>(a.residual, a.ld_residual, r), c, a.cols);
#pragma unroll
    for (uint32_t j = 0; j < kGroup; ++j) v[j] = w[j] + v[j];
  }
}

// ---- Rows of any width: a workgroup goes over its row once for every sum ---------------------------------------
constexpr uint32_t kWideThreads = 1024;

template <typename T, typename H>
__global__ __launch_bounds__(kWideThreads) void k_norm_forward_wide(NormArgs a) {
  __shared__ float slots[2][1][16];
  const uint64_t offset = a.join ? drop_offset(a.drop) : 0u;
  const float count = static_cast<float>(a.cols);
  for (uint32_t r = blockIdx.x; r < a.total; r += gridDim.x) {
    float s[1] = {0.0f};
    for (uint32_t c = threadIdx.x * kGroup; c < a.cols; c += kWideThreads * kGroup) {
      float v[kGroup];
      form_h<T, H>(v, a, offset, r, c);
      for (uint32_t j = 0; j < kGroup; ++j) s[0] += c + j < a.cols ? v[j] : 0.0f;
    }
    sum_block(s, slots[0], kWideThreads / 64);
    const float mean = s[0] / count;
    s[0] = 0.0f;
    for (uint32_t c = threadIdx.x * kGroup; c < a.cols; c += kWideThreads * kGroup) {
      float v[kGroup];
      form_h<T, H>(v, a, offset, r, c);
      for (uint32_t j = 0; j < kGroup; ++j) {
        const float d = v[j] - mean;
        s[0] += c + j < a.cols ? d * d : 0.0f;
      }
    }
    sum_block(s, slots[1], kWideThreads / 64);
    const float rstd = 1.0f / sqrtf(s[0] / count + a.eps);
    for (uint32_t c = threadIdx.x * kGroup; c < a.cols; c += kWideThreads * kGroup) {
      float v[kGroup], g[kGroup], b[kGroup];
      form_h<T, H>(v, a, offset, r, c);
      if (a.join && a.h) store_group(row_of<H>(a.h, a.ld_h, r), c, a.cols, v);
      load_weight(g, a.gamma, c, a.cols, 1.0f);
      load_weight(b, a.beta, c, a.cols, 0.0f);
      for (uint32_t j = 0; j < kGroup; ++j) v[j] = (v[j] - mean) * rstd * g[j] + b[j];
      store_group(row_of<T>(a.y, a.ld_y, r), c, a.cols, v);
    }
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[r] = mean;
      if (a.rstd) a.rstd[r] = rstd;
    }
  }
}

// z of a group from h as it was stored.
template <typename H>
__device__ __forceinline__ void load_z(float (&z)[kGroup], const NormArgs& a, uint32_t r, uint32_t c, float mean, float rstd) {
  load_group(z, row_of<H>(static_cast<const void*>(a.h), a.ld_h, r), c, a.cols);
#pragma unroll
  for (uint32_t j = 0; j < kGroup; ++j) z[j] = (z[j] - mean) * rstd;
}

template <typename T, typename H>
__global__ __launch_bounds__(kWideThreads) void k_norm_sums_wide(NormArgs a) {
  __shared__ float slots[2][2][16];
  uint32_t turn = 0;
  const float count = static_cast<float>(a.cols);
  for (uint32_t r = blockIdx.x; r < a.total; r += gridDim.x, turn ^= 1) {
    const float mean = a.mean[r], rstd = a.rstd[r];
    float s[2] = {0.0f, 0.0f};
    for (uint32_t c = threadIdx.x * kGroup; c < a.cols; c += kWideThreads * kGroup) {
      float u[kGroup], z[kGroup], g[kGroup];
      load_group(u, row_of<T>(a.dy, a.ld_dy, r), c, a.cols);
      load_weight(g, a.gamma, c, a.cols, 1.0f);
      load_z<H>(z, a, r, c, mean, rstd);
      for (uint32_t j = 0; j < kGroup; ++j) {
        u[j] *= g[j];
        s[0] += c + j < a.cols ? u[j] : 0.0f;
        s[1] += c + j < a.cols ? u[j] * z[j] : 0.0f;
      }
    }
    sum_block(s, slots[turn], kWideThreads / 64);
    if (threadIdx.x == 0) a.sums[r] = make_float2(s[0] / count, s[1] / count);
  }
}

// The gradient of h in a group, from the two sums of its row: dy and z are left in u and z.
template <typename T, typename H>
__device__ __forceinline__ void form_d(float (&d)[kGroup], float (&u)[kGroup], float (&z)[kGroup], const NormArgs& a,
                                       uint32_t r, uint32_t c) {
  const float mean = a.mean[r], rstd = a.rstd[r];
  const float2 s = a.sums[r];
  float g[kGroup];
  load_group(u, row_of<T>(a.dy, a.ld_dy, r), c, a.cols);
  load_weight(g, a.gamma, c, a.cols, 1.0f);
  load_z<H>(z, a, r, c, mean, rstd);
#pragma unroll
  for (uint32_t j = 0; j < kGroup; ++j) d[j] = (u[j] * g[j] - s.x - z[j] * s.y) * rstd;
  if (a.dh) {
    load_group(g, row_of<H>(a.dh, a.ld_dh, r), c, a.cols);
#pragma unroll
    for (uint32_t j = 0; j < kGroup; ++j) d[j] += g[j];
  }
}

// The weights' gradients: 256 columns by one part of a worker's rows to a workgroup, eight of them at a time.
constexpr uint32_t kTileGroups = 32, kTileRows = 8;

// One column's sum over a part, to where it belongs: the partial sums, or where a worker has one part, the gradient.
__device__ __forceinline__ void emit_gradient(const NormArgs& a, uint32_t worker, uint32_t part, uint32_t which, uint32_t c,
                                              float sum) {
  if (a.parts > 1) {
    a.partial[((static_cast<size_t>(worker) * a.parts + part) * kGradients + which) * a.cols + c] = sum;
  } else {
    float* const p = a.grad[which] + static_cast<int64_t>(worker) * a.ld_grad[which] + c;
    *p = a.accumulate ? *p + sum : sum;
  }
}

template <typename T, typename H>
__global__ __launch_bounds__(kTileGroups * kTileRows) void k_norm_columns_wide(NormArgs a) {
  __shared__ float tile[kTileRows][kTileGroups * kGroup];
  const uint32_t c = (blockIdx.x * kTileGroups + threadIdx.x % kTileGroups) * kGroup, lane_row = threadIdx.x / kTileGroups;
  const uint64_t offset = a.join ? drop_offset(a.drop) : 0u;
  const uint32_t w = blockIdx.z;
  for (uint32_t part = blockIdx.y; part < a.parts; part += gridDim.y) {
    float sum[kGradients][kGroup] = {};
    const uint32_t first = part * a.part_rows, left = a.rows - first;
    const uint32_t rows = left < a.part_rows ? left : a.part_rows;
    if (c < a.cols) {
      for (uint32_t i = lane_row; i < rows; i += kTileRows) {
        const uint32_t r = w * a.rows + first + i;
        float d[kGroup], u[kGroup], z[kGroup];
        form_d<T, H>(d, u, z, a, r, c);
        if (a.grad[2]) drop_group(d, a.drop, offset, r, c);
#pragma unroll
        for (uint32_t j = 0; j < kGroup; ++j) {
          sum[0][j] += u[j] * z[j];
          sum[1][j] += u[j];
          sum[2][j] += d[j];
        }
      }
    }
    for (uint32_t k = 0; k < kGradients; ++k) {
      if (!a.grad[k]) continue;
      __syncthreads();
#pragma unroll
      for (uint32_t j = 0; j < kGroup; ++j) tile[lane_row][threadIdx.x % kTileGroups * kGroup + j] = sum[k][j];
      __syncthreads();
      const uint32_t col = blockIdx.x * kTileGroups * kGroup + threadIdx.x;
      if (col < a.cols) {
        float s = 0.0f;
        for (uint32_t i = 0; i < kTileRows; ++i) s += tile[i][threadIdx.x];
        emit_gradient(a, w, part, k, col, s);
      }
    }
  }
}

// The parts' sums added up in their order: 64 columns to a workgroup, a quarter of the parts to each wavefront.
__global__ __launch_bounds__(256) void k_norm_join_parts(NormArgs a) {
  __shared__ float tile[4][64];
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, which = blockIdx.y;
  if (!a.grad[which]) return;
  const uint32_t tiles = (a.cols + 63) / 64;
  for (uint32_t t = blockIdx.x; t < tiles; t += gridDim.x) {
    const uint32_t c = t * 64 + lane, w = blockIdx.z;
    float s = 0.0f;
    if (c < a.cols) {
      const float* p = a.partial + (static_cast<size_t>(w) * a.parts * kGradients + which) * a.cols + c;
      const size_t step = static_cast<size_t>(kGradients) * a.cols;
      const uint32_t share = (a.parts + 3) / 4, from = wave * share, to = from + share < a.parts ? from + share : a.parts;
      for (uint32_t i = from; i < to; ++i) s += p[i * step];
    }
    __syncthreads();
    tile[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && c < a.cols) {
      s = (tile[0][lane] + tile[1][lane]) + (tile[2][lane] + tile[3][lane]);
      float* const out = a.grad[which] + static_cast<int64_t>(w) * a.ld_grad[which] + c;
      *out = a.accumulate ? *out + s : s;
    }
  }
}

template <typename T, typename H>
__global__ __launch_bounds__(kWideThreads) void k_norm_backward_wide(NormArgs a) {
  const uint64_t offset = a.join ? drop_offset(a.drop) : 0u;
  for (uint32_t r = blockIdx.x; r < a.total; r += gridDim.x) {
    for (uint32_t c = threadIdx.x * kGroup; c < a.cols; c += kWideThreads * kGroup) {
      float d[kGroup], u[kGroup], z[kGroup];
      form_d<T, H>(d, u, z, a, r, c);
      if (a.dresidual) store_group(row_of<H>(a.dresidual, a.ld_dresidual, r), c, a.cols, d);
      if (a.dx) {
        drop_group(d, a.drop, offset, r, c);
        store_group(row_of<T>(a.dx, a.ld_dx, r), c, a.cols, d);
      }
    }
  }
}

// No row at all: the gradients are sums over nothing.
__global__ __launch_bounds__(256) void k_norm_no_rows(NormArgs a) {
  const uint32_t which = blockIdx.y;
  if (!a.grad[which]) return;
  for (uint32_t c = blockIdx.x * 256 + threadIdx.x; c < a.cols; c += gridDim.x * 256)
    a.grad[which][static_cast<int64_t>(blockIdx.z) * a.ld_grad[which] + c] = 0.0f;
}

// ---- Host ------------------------------------------------------------------------------------------------------
template <typename F>
hipError_t by_types(int32_t type, int32_t stream_type, F f) {
  if (type == COMPAMS_F32) return f(float(), float());
  if (type == COMPAMS_F16) return stream_type == COMPAMS_F32 ? f(half_t(), float()) : f(half_t(), half_t());
  return stream_type == COMPAMS_F32 ? f(bfloat_t(), float()) : f(bfloat_t(), bfloat_t());
}

constexpr uint32_t kMostBlocks = 1u << 21;  // of 1024 threads: a dimension has room for 2^32 threads in all
inline uint32_t blocks_for(uint64_t wanted) { return wanted < kMostBlocks ? static_cast<uint32_t>(wanted) : kMostBlocks; }
inline uint32_t at_most(uint32_t v, uint32_t most) { return v < most ? v : most; }

bool any_gradient(const compams_norm& a) { return a.dgamma || a.dbeta || a.dbias; }

// How a backward call is cut up, and what of the workspace it takes.
struct Cut {
  uint32_t parts, part_rows;
  size_t sums_bytes, partial_bytes;
};
inline size_t up256(size_t v) { return (v + 255) / 256 * 256; }
Cut cut_of(const compams_norm& a) {
  Cut c = {};
  if (a.rows == 0) return c;
  c.part_rows = 64;
  c.parts = static_cast<uint32_t>((a.rows + c.part_rows - 1) / c.part_rows);
  c.sums_bytes = up256(static_cast<size_t>(a.n) * a.rows * sizeof(float2));
  if (any_gradient(a) && c.parts > 1)
    c.partial_bytes = up256(static_cast<size_t>(a.n) * c.parts * kGradients * a.cols * sizeof(float));
  return c;
}

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

int norm_forward(const compams_norm* a, bool join, hipStream_t stream) {
  if (!norm_valid(a, join)) return COMPAMS_INVALID_ARG;
  if (a->rows == 0) return COMPAMS_OK;
  if (!a->y || (join ? !a->x : !a->h)) return COMPAMS_INVALID_ARG;
  if (!join && (a->x || a->residual || a->bias)) return COMPAMS_INVALID_ARG;
  const int bad = first_bad({check_matrix(a->x, a->ld_x, *a, a->type), check_matrix(a->h, a->ld_h, *a, a->stream_type),
                             check_matrix(a->residual, a->ld_residual, *a, a->stream_type),
                             check_matrix(a->y, a->ld_y, *a, a->type), check_vectors(*a, join)});
  if (bad != COMPAMS_OK) return bad;
  const NormArgs k = make_args(*a, join);
  const hipError_t err = by_types(a->type, a->stream_type, [&](auto t, auto h) {
    using T = decltype(t);
    using H = decltype(h);
    hipLaunchKernelGGL((k_norm_forward_wide<T, H>), dim3(blocks_for(k.total)), dim3(kWideThreads), 0, stream, k);
    return hipGetLastError();
  });
  return err == hipSuccess ? COMPAMS_OK : COMPAMS_HIP_ERROR;
}

int norm_backward(const compams_norm* a, bool join, hipStream_t stream) {
  if (!norm_valid(a, join) || (a->accumulate != 0 && a->accumulate != 1)) return COMPAMS_INVALID_ARG;
  if (!join && (a->dx || a->dh || a->dbias)) return COMPAMS_INVALID_ARG;
  if (!any_gradient(*a) && !a->dresidual && !a->dx) return COMPAMS_INVALID_ARG;
  NormArgs k = make_args(*a, join);
  for (uint32_t i = 0; i < kGradients; ++i) {
    if (!k.grad[i]) continue;
    if (a->n > 1 && (k.ld_grad[i] < a->cols || k.ld_grad[i] >= (static_cast<int64_t>(1) << 40))) return COMPAMS_INVALID_ARG;
    if (!aligned_to(k.grad[i], 4)) return COMPAMS_BAD_ALIGNMENT;
  }
  const dim3 grid_columns(at_most((k.cols + 63) / 64, 4096), kGradients, k.n);
  if (a->rows == 0) {
    if (k.accumulate || !any_gradient(*a)) return COMPAMS_OK;
    hipLaunchKernelGGL(k_norm_no_rows, dim3(at_most((k.cols + 255) / 256, 4096), kGradients, k.n), dim3(256),
                       0, stream, k);
    return hipGetLastError() == hipSuccess ? COMPAMS_OK : COMPAMS_HIP_ERROR;
  }
  if (!a->dy || !a->h || !a->mean || !a->rstd) return COMPAMS_INVALID_ARG;
  const int bad = first_bad({check_matrix(a->dy, a->ld_dy, *a, a->type), check_matrix(a->h, a->ld_h, *a, a->stream_type),
                             check_matrix(k.dh, a->ld_dh, *a, a->stream_type), check_matrix(k.dx, a->ld_dx, *a, a->type),
                             check_matrix(a->dresidual, a->ld_dresidual, *a, a->stream_type), check_vectors(*a, join)});
  if (bad != COMPAMS_OK) return bad;
  const Cut cut = cut_of(*a);
  if (cut.sums_bytes + cut.partial_bytes > 0) {
    if (!a->workspace) return COMPAMS_INVALID_ARG;
    if (!aligned_to(a->workspace, 256)) return COMPAMS_BAD_ALIGNMENT;
    if (a->workspace_bytes < cut.sums_bytes + cut.partial_bytes) return COMPAMS_WORKSPACE_TOO_SMALL;
  }
  k.sums = static_cast<float2*>(a->workspace);
  k.partial = reinterpret_cast<float*>(static_cast<char*>(a->workspace) + cut.sums_bytes);
  k.parts = cut.parts;
  k.part_rows = cut.part_rows;
  const hipError_t err = by_types(a->type, a->stream_type, [&](auto t, auto h) {
    using T = decltype(t);
    using H = decltype(h);
    hipLaunchKernelGGL((k_norm_sums_wide<T, H>), dim3(blocks_for(k.total)), dim3(kWideThreads), 0, stream, k);
    if (any_gradient(*a)) {
      constexpr uint32_t kTileCols = kTileGroups * kGroup;
      hipLaunchKernelGGL((k_norm_columns_wide<T, H>),
                         dim3((k.cols + kTileCols - 1) / kTileCols, at_most(k.parts, 32768), k.n),
                         dim3(kTileGroups * kTileRows), 0, stream, k);
      if (k.parts > 1) hipLaunchKernelGGL(k_norm_join_parts, grid_columns, dim3(256), 0, stream, k);
    }
    // (the outputs last: they may be the inputs' own buffers)
    if (k.dx || k.dresidual)
      hipLaunchKernelGGL((k_norm_backward_wide<T, H>), dim3(blocks_for(k.total)), dim3(kWideThreads), 0, stream, k);
    return hipGetLastError();
  });
  return err == hipSuccess ? COMPAMS_OK : COMPAMS_HIP_ERROR;
}

}  // namespace
}  // namespace compams

extern "C" {

size_t compams_norm_workspace_size(const compams_norm* a) {
  if (!compams::norm_valid(a, false)) return 0;
  const compams::Cut c = compams::cut_of(*a);
  return c.sums_bytes + c.partial_bytes;
}
int compams_layer_norm_forward(const compams_norm* a, void* hip_stream) {
  return compams::norm_forward(a, false, static_cast<hipStream_t>(hip_stream));
}
int compams_layer_norm_backward(const compams_norm* a, void* hip_stream) {
  return compams::norm_backward(a, false, static_cast<hipStream_t>(hip_stream));
}
int compams_dropout_add_norm_forward(const compams_norm* a, void* hip_stream) {
  return compams::norm_forward(a, true, static_cast<hipStream_t>(hip_stream));
}
int compams_dropout_add_norm_backward(const compams_norm* a, void* hip_stream) {
  return compams::norm_backward(a, true, static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
