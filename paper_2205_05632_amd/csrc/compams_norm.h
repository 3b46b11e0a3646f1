// What the kernels of the layer norm and of the join share.
#pragma once

#include <math.h>

#include "compams_rows.h"

namespace compams {

constexpr uint32_t kGradients = 3;  // dgamma, dbeta, dbias

// A number and its inverse, to the nearest.
struct Count {
  float n, inverse;
};

struct NormArgs {
  uint32_t n, rows, cols;  // workers, rows of each, columns
  uint32_t total;          // n * rows
  float eps;
  bool join;
  Count count;             // of columns
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

// The same in two steps (see load_early).
template <Width WIDTH = kAnyWidth>
__device__ __forceinline__ Group<float>::type load_weight_early(const float* w, uint32_t c, uint32_t cols, float absent) {
  if (WIDTH == kFullGroups || WIDTH == kWholeGroups || w) return load_early<WIDTH>(w, c, cols);
  Group<float>::type raw;
#pragma unroll
  for (uint32_t j = 0; j < kGroup; ++j) raw[j] = absent;
  return raw;
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

// A row's statistics from its sums, each step rounded once, so that they are the same whatever team holds the row: the quotient
// and the inverse root by the hardware's approximations, put right by what is left over (with the compiler's quotients and
// roots 8 x 3117 x 1601 float16 takes 47.6 us for 45.3: they need registers that a wavefront goes for).
__device__ __forceinline__ float mean_of(float sum, Count count) {
  const float q = sum * count.inverse;
  return fabsf(q) < INFINITY ? fmaf(fmaf(-q, count.n, sum), count.inverse, q) : q;
}
__device__ __forceinline__ float rstd_of(float squares, Count count, float eps) {
  const float v = mean_of(squares, count) + eps, x = rsqrtf(v);
  if (!(v > 0.0f && v < INFINITY)) return x;
  const float t = v * x;
  return fmaf(0.5f * x, fmaf(-fmaf(v, x, -t), x, fmaf(-t, x, 1.0f)), x);
}

// How a row's team of lanes is made up.
enum TeamKind {
  kInWave = 0,  // 8, 16, 32 or 64 lanes of a wavefront; a workgroup of 256 threads has several teams
  kBlock = 1,   // a whole workgroup
  kPair = 2     // an odd number of half wavefronts, two such teams to a workgroup
};
constexpr uint32_t kTeamThreads = 256;  // of a workgroup of kInWave
struct Team {
  TeamKind kind;
  uint32_t lanes, each;  // lanes of a team; groups that a lane takes (0: rows are not held in registers)
};
inline uint32_t team_threads(const Team& t) {
  return t.kind == kInWave ? kTeamThreads : t.kind == kBlock ? t.lanes : 2 * t.lanes;
}
// This lane's team within the workgroup, its place there, and the teams of a workgroup.
template <TeamKind KIND>
__device__ __forceinline__ uint32_t team_of_lane(uint32_t lanes) {
  return KIND == kInWave ? threadIdx.x / lanes : KIND == kBlock ? 0u : threadIdx.x >= lanes ? 1u : 0u;
}
template <TeamKind KIND>
__device__ __forceinline__ uint32_t lane_of_team(uint32_t lanes, uint32_t team) {
  return KIND == kInWave ? threadIdx.x & (lanes - 1) : KIND == kBlock ? threadIdx.x : threadIdx.x - team * lanes;
}
template <TeamKind KIND>
__device__ __forceinline__ uint32_t teams_together(uint32_t lanes) {
  return KIND == kInWave ? kTeamThreads / lanes : KIND == kBlock ? 1u : 2u;
}
// Sums over the lanes of a team.
template <TeamKind KIND, int N>
__device__ __forceinline__ void sum_over_team(float (&v)[N], float (*slots)[kSlots], uint32_t lanes, uint32_t team) {
  if constexpr (KIND == kInWave) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = sum_lanes(v[i], lanes);
  } else if constexpr (KIND == kBlock) {
    sum_team<false>(v, slots, 0, lanes / 64);
  } else {
    sum_team<true>(v, slots, team * (lanes / 32), lanes / 32);
  }
}

// ---- Host ------------------------------------------------------------------------------------------------------
template <typename F>
inline hipError_t by_types(int32_t type, int32_t stream_type, F f) {
  if (type == COMPAMS_F32) return f(float(), float());
  if (type == COMPAMS_F16) return stream_type == COMPAMS_F32 ? f(half_t(), float()) : f(half_t(), half_t());
  return stream_type == COMPAMS_F32 ? f(bfloat_t(), float()) : f(bfloat_t(), bfloat_t());
}

constexpr uint32_t kMostBlocks = 1u << 21;  // of 1024 threads: a dimension has room for 2^32 threads in all
inline uint32_t blocks_for(uint64_t wanted) { return wanted < kMostBlocks ? static_cast<uint32_t>(wanted) : kMostBlocks; }
inline uint32_t at_most(uint32_t v, uint32_t most) { return v < most ? v : most; }

// How a backward call is cut up, and what of the workspace it takes.
struct Cut {
  uint32_t parts, part_rows;
  size_t sums_bytes, partial_bytes;
};
Cut norm_cut(uint32_t n, uint32_t rows, uint32_t cols, bool join, bool gradients);

hipError_t norm_forward(const NormArgs& a, int32_t type, int32_t stream_type, hipStream_t stream);
hipError_t norm_backward(const NormArgs& a, int32_t type, int32_t stream_type, hipStream_t stream);

}  // namespace compams
