// Layer norm and the join of a transformer block, backward, with the gradients of the weights per worker.
#include <math.h>

#include "compams_norm.h"

namespace compams {
namespace {

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

// ---- Rows that a team of lanes holds in registers ---------------------------------------------------------------
// As in the forward pass; a lane keeps to its columns: it adds up the weights' gradients of the rows that its team takes.  A
// workgroup takes one part of a worker's rows and leaves one sum per column.  The parts take the rows in turn, so that the
// workgroups that run together go through memory together (8 x 8192 x 768, join: 161 us, with a stretch of rows each 171).
// 8 x 8192 x 768 with an fp32 stream: 156 us and 11 for the sums of the parts, 4.8 TB/s; a kernel that only reads and writes
// the same arrays takes 141.  The next row's loads ahead of this one's arithmetic, or two rows of a team at once, changed
// nothing: the rows of the other workgroups of a compute unit do as much.

// Values summed over the teams of a wavefront: over the lanes that are multiples of `lanes` apart.
template <uint32_t NG>
__device__ __forceinline__ void sum_teams(float (&v)[NG][kGroup], uint32_t lanes) {
  if (lanes == 64) return;
  if (lanes <= 8) {
#pragma unroll
    for (uint32_t k = 0; k < NG; ++k)
#pragma unroll
      for (uint32_t j = 0; j < kGroup; ++j) v[k][j] += dpp<0x128>(v[k][j]);  // a row's lanes turned by 8
  }
  if (lanes <= 16) {
#pragma unroll
    for (uint32_t k = 0; k < NG; ++k)
#pragma unroll
      for (uint32_t j = 0; j < kGroup; ++j) {
        const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v[k][j]), __float_as_uint(v[k][j]), false, false);
        v[k][j] = __uint_as_float(s[0]) + __uint_as_float(s[1]);
      }
  }
#pragma unroll
  for (uint32_t k = 0; k < NG; ++k)
#pragma unroll
    for (uint32_t j = 0; j < kGroup; ++j) {
      const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[k][j]), __float_as_uint(v[k][j]), false, false);
      v[k][j] = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    }
}

template <typename T, typename H, uint32_t NG, TeamKind KIND, bool JOIN, Width WIDTH>
__global__ __launch_bounds__(KIND == kInWave ? kTeamThreads : NG == 2 && JOIN ? 768 : 1024) void k_norm_backward(NormArgs a,
                                                                                                          uint32_t lanes) {
  constexpr bool FULL = WIDTH == kFullGroups || WIDTH == kWholeGroups;  // nothing is left out of the call
  constexpr uint32_t kOf = JOIN ? 3 : 2;
  __shared__ float slots[2][2][kSlots];
  extern __shared__ float tile[];  // a row of columns for each wavefront (kInWave), or one (kPair)
  const uint32_t team = team_of_lane<KIND>(lanes), lane = lane_of_team<KIND>(lanes, team);
  const uint32_t together = teams_together<KIND>(lanes);
  const uint64_t offset = JOIN ? drop_offset(a.drop) : 0u;
  typename Group<float>::type g[NG];
#pragma unroll
  for (uint32_t k = 0; k < NG; ++k) {
    const uint32_t c = (k * lanes + lane) * kGroup;
    g[k] = load_weight_early<WIDTH>(a.gamma, c, a.cols, 1.0f);
    settle_if<WIDTH, float>(g[k], c, a.cols);
  }
  uint32_t turn = 0;
  for (uint32_t job = blockIdx.x; job < a.n * a.parts; job += gridDim.x) {
    const uint32_t w = job / a.parts, part = job % a.parts;
    float sum[kOf][NG][kGroup] = {};
    for (uint32_t i = part * together; i < a.rows; i += a.parts * together, turn ^= 1) {
      // (a team without a row of its own goes over the last one again: the teams of a pair meet at barriers)
      const bool spare = KIND != kBlock && i + team >= a.rows;
      if (KIND == kInWave && spare) break;
      const uint32_t r = w * a.rows + (spare ? a.rows - 1 : i + team);
      typename Group<T>::type raw_y[NG];
      typename Group<H>::type raw_h[NG], raw_g[NG];
#pragma unroll
      for (uint32_t k = 0; k < NG; ++k) {
        const uint32_t c = (k * lanes + lane) * kGroup;
        raw_y[k] = load_early<WIDTH>(row_of<T>(a.dy, a.ld_dy, r), c, a.cols);
        raw_h[k] = load_early<WIDTH>(row_of<H>(static_cast<const void*>(a.h), a.ld_h, r), c, a.cols);
        if (JOIN && (FULL || a.dh)) raw_g[k] = load_early<WIDTH>(row_of<H>(a.dh, a.ld_dh, r), c, a.cols);
      }
      const float mean = a.mean[r], rstd = a.rstd[r];
      // Beyond the row's last column h and u are read as 0, and z is the mean's size: nothing in a product with u while that
      // is a number.  Where it is none, the entries that these statistics belong to are the mean, and their z is 0.  (Telling
      // those columns apart takes a join of 8 x 4096 x 773 a sixth longer; lanes without a group are left out below.)
      constexpr bool kEnd = WIDTH == kAnyWidth || WIDTH == kOneGroup;
      const float rstd_of_sums = !kEnd || fabsf(mean * rstd) < INFINITY ? rstd : 0.0f;
      float s[2] = {0.0f, 0.0f};
#pragma unroll
      for (uint32_t k = 0; k < NG; ++k) {
        const uint32_t c = (k * lanes + lane) * kGroup;
        float z[kGroup], u[kGroup];
        settle_if<WIDTH, T>(raw_y[k], c, a.cols);
        settle_if<WIDTH, H>(raw_h[k], c, a.cols);
        unpack(u, raw_y[k]);
        unpack(z, raw_h[k]);
        const float before = s[1];
#pragma unroll
        for (uint32_t j = 0; j < kGroup; ++j) {
          // (columns beyond the last: dy and, read from gamma's end, the weight are 0)
          u[j] *= g[k][j];
          s[0] += u[j];
          s[1] = fmaf(u[j], (z[j] - mean) * rstd_of_sums, s[1]);
        }
        if (WIDTH == kWholeGroups && c >= a.cols) s[1] = before;
      }
      sum_over_team<KIND>(s, slots[turn], lanes, team);
      if (KIND == kPair && spare) continue;
      const float s0 = mean_of(s[0], a.count), s1 = mean_of(s[1], a.count);
#pragma unroll
      for (uint32_t k = 0; k < NG; ++k) {
        const uint32_t c = (k * lanes + lane) * kGroup;
        float z[kGroup], u[kGroup];
        unpack(u, raw_y[k]);
        unpack(z, raw_h[k]);
#pragma unroll
        for (uint32_t j = 0; j < kGroup; ++j) {
          z[j] = (z[j] - mean) * rstd;
          sum[0][k][j] = fmaf(u[j], z[j], sum[0][k][j]);
          sum[1][k][j] += u[j];
          u[j] = (fmaf(u[j], g[k][j], -s0) - z[j] * s1) * rstd;
        }
        if constexpr (JOIN) {
          if (FULL || a.dh) {
            settle_if<WIDTH, H>(raw_g[k], c, a.cols);
            unpack(z, raw_g[k]);
#pragma unroll
            for (uint32_t j = 0; j < kGroup; ++j) u[j] += z[j];
          }
        }
        if (FULL || a.dresidual) store_group<H, WIDTH>(row_of<H>(a.dresidual, a.ld_dresidual, r), c, a.cols, u);
        if constexpr (JOIN) {
          if (FULL || a.dx || a.grad[2]) {
            drop_group(u, a.drop, offset, r, c);
            if (FULL || a.dx) store_group<T, WIDTH>(row_of<T>(a.dx, a.ld_dx, r), c, a.cols, u);
#pragma unroll
            for (uint32_t j = 0; j < kGroup; ++j) sum[2][k][j] += u[j];
          }
        }
      }
    }
#pragma unroll
    for (uint32_t which = 0; which < kOf; ++which) {
      if (!FULL && !a.grad[which]) continue;
      if constexpr (KIND == kInWave) {
        const uint32_t across = NG * lanes * kGroup;
        sum_teams(sum[which], lanes);
        __syncthreads();
        if ((threadIdx.x & 63u) < lanes) {
#pragma unroll
          for (uint32_t k = 0; k < NG; ++k)
            __builtin_memcpy(&tile[(threadIdx.x >> 6) * across + (k * lanes + lane) * kGroup], sum[which][k],
                             sizeof(sum[which][k]));
        }
        __syncthreads();
        for (uint32_t c = threadIdx.x; c < a.cols; c += kTeamThreads)
          emit_gradient(a, w, part, which, c, (tile[c] + tile[across + c]) + (tile[2 * across + c] + tile[3 * across + c]));
      } else {
        if constexpr (KIND == kPair) {  // the second team's sums to the first
          __syncthreads();
          if (team == 1) __builtin_memcpy(&tile[lane * kGroup], sum[which][0], sizeof(sum[which][0]));
          __syncthreads();
          if (team == 1) continue;
#pragma unroll
          for (uint32_t j = 0; j < kGroup; ++j) sum[which][0][j] += tile[lane * kGroup + j];
        }
        if (a.parts > 1) {
          float* const row = a.partial + ((static_cast<size_t>(w) * a.parts + part) * kGradients + which) * a.cols;
#pragma unroll
          for (uint32_t k = 0; k < NG; ++k) store_group<float, WIDTH>(row, (k * lanes + lane) * kGroup, a.cols, sum[which][k]);
        } else {
#pragma unroll
          for (uint32_t k = 0; k < NG; ++k)
#pragma unroll
            for (uint32_t j = 0; j < kGroup; ++j) {
              const uint32_t c = (k * lanes + lane) * kGroup + j;
              if (WIDTH == kFullGroups || c < a.cols) emit_gradient(a, w, part, which, c, sum[which][k][j]);
            }
        }
      }
    }
  }
}

// ---- Rows of any width: a pass for the rows' sums, one for the columns' and one for the outputs --------------------
constexpr uint32_t kWideThreads = 1024;

// z of a group from h as it was stored.
template <typename H>
__device__ __forceinline__ void load_z(float (&z)[kGroup], const NormArgs& a, uint32_t r, uint32_t c, float mean, float rstd) {
  load_group(z, row_of<H>(static_cast<const void*>(a.h), a.ld_h, r), c, a.cols);
#pragma unroll
  for (uint32_t j = 0; j < kGroup; ++j) z[j] = (z[j] - mean) * rstd;
}

template <typename T, typename H>
__global__ __launch_bounds__(kWideThreads) void k_norm_sums_wide(NormArgs a) {
  __shared__ float slots[2][2][kSlots];
  uint32_t turn = 0;
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
    if (threadIdx.x == 0) a.sums[r] = make_float2(mean_of(s[0], a.count), mean_of(s[1], a.count));
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

// ---- What both take ------------------------------------------------------------------------------------------------
// The parts' sums added up in their order: 64 columns to a workgroup, a sixteenth of the parts to each wavefront.  (Where there
// are fewer than sixteen, as many wavefronts; 8 x 24 x 9062, three parts: 35.8 us a call, with sixteen 43.4.)
constexpr uint32_t kJoinThreads = 1024, kJoinWaves = kJoinThreads / 64;
__global__ __launch_bounds__(kJoinThreads) void k_norm_join_parts(NormArgs a) {
  __shared__ float tile[kJoinWaves][64];
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, waves = blockDim.x / 64, which = blockIdx.y, w = blockIdx.z;
  if (!a.grad[which]) return;
  const uint32_t tiles = (a.cols + 63) / 64;
  for (uint32_t t = blockIdx.x; t < tiles; t += gridDim.x) {
    const uint32_t c = t * 64 + lane;
    float s = 0.0f;
    if (c < a.cols) {
      const float* const p = a.partial + (static_cast<size_t>(w) * a.parts * kGradients + which) * a.cols + c;
      const size_t step = static_cast<size_t>(kGradients) * a.cols;
      const uint32_t share = (a.parts + waves - 1) / waves, from = wave * share;
      const uint32_t to = from + share < a.parts ? from + share : a.parts;
#pragma unroll 8
      for (uint32_t i = from; i < to; ++i) s += p[i * step];
    }
    __syncthreads();
    tile[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && c < a.cols) {
      s = 0.0f;
      for (uint32_t i = 0; i < waves; ++i) s += tile[i][lane];
      float* const out = a.grad[which] + static_cast<int64_t>(w) * a.ld_grad[which] + c;
      *out = a.accumulate ? *out + s : s;
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

// The team that a row of `groups` groups is given; us, norm / join, bfloat16 and a stream in fp32:
//   8 x 2048 x  640: pair of 96 27.3 / 43.4, 32 x 3 30.0 / 47.5       8 x 8192 x 768: join, 32 x 3 (229 registers) 158, pair 161
//   8 x 3117 x 1280, float16: pair of 160 51.5 / 100, 192 53.4 / 81.6; x 1600: pair of 224 66.1 / 108, 256 63.7 / 103
//   8 x 2048 x 1024: 64 x 2 41.2 / 60.6, 128 41.1 / 60.5, in parts of 32 rows 42.3 / 62.7 and 49.6 / 62.5
//   8 x 6167 x  512: 64 58.5 / 88.1, all float16 40.2 / 60.8; 32 x 2 55.9 / 84.7 and 38.8 / 57.9
Team backward_team(uint32_t rows, uint32_t groups, bool join) {
  if (groups > 48 && groups <= 64) return {kInWave, 32, 2};
  if (groups <= 48) {
    uint32_t lanes = 8;
    while (lanes < groups) lanes *= 2;
    return {kInWave, lanes, 1};
  }
  const uint32_t halves = (groups + 31) / 32;
  // (a join's four wavefronts to a SIMD seldom hold three workgroups of five: a row of three wavefronts instead of two of five,
  // but where a worker has few rows: 8 x 400 x 1280 pair 18.5, 192 22.1; 3 x 401 x 1601 17.4 and 21.2; 8 x 1000 x 1280 41.9
  // and 33.3)
  if (halves == 3 || ((!join || rows <= 512) && (halves == 5 || halves == 7))) return {kPair, halves * 32, 1};
  if (groups <= 128) return {kInWave, 64, 2};
  // (two groups a lane take a join 168 registers: twelve wavefronts at most)
  const uint32_t each = groups <= 1024 ? 1 : groups <= (join ? 1536 : 2048) ? 2 : 0;
  return {kBlock, each ? (groups + 64 * each - 1) / (64 * each) * 64 : 0, each};
}

template <typename T, typename H, bool JOIN>
void launch_team(const Team& t, const NormArgs& k, hipStream_t stream) {
  const dim3 grid(blocks_for(static_cast<uint64_t>(k.n) * k.parts)), block(team_threads(t));
  const size_t lines = t.kind == kInWave ? kTeamThreads / 64 : t.kind == kPair ? 1 : 0;
  const size_t lds = lines * t.each * t.lanes * kGroup * sizeof(float);
  const bool all = k.gamma && k.dresidual && k.grad[0] && k.grad[1] && (!JOIN || (k.dh && k.dx && k.grad[2]));
  const bool full = all && k.cols == t.lanes * t.each * kGroup, whole = all && k.cols % kGroup == 0;
#define COMPAMS_BACKWARD_OF(NG, KIND, WIDTH) \
  hipLaunchKernelGGL((k_norm_backward<T, H, NG, KIND, JOIN, WIDTH>), grid, block, lds, stream, k, t.lanes)
#define COMPAMS_BACKWARD(NG, KIND)                         \
  do {                                                     \
    if (full) COMPAMS_BACKWARD_OF(NG, KIND, kFullGroups);  \
    else if (whole) COMPAMS_BACKWARD_OF(NG, KIND, kWholeGroups); \
    else COMPAMS_BACKWARD_OF(NG, KIND, kAnyWidth);         \
  } while (0)
  if (t.kind == kInWave) {
    if (k.cols < kGroup) COMPAMS_BACKWARD_OF(1, kInWave, kOneGroup);
    else if (t.each == 1) COMPAMS_BACKWARD(1, kInWave);
    else COMPAMS_BACKWARD(2, kInWave);
  } else if (t.kind == kPair) {
    COMPAMS_BACKWARD(1, kPair);
  } else {
    if (t.each == 1) COMPAMS_BACKWARD(1, kBlock);
    else COMPAMS_BACKWARD(2, kBlock);
  }
#undef COMPAMS_BACKWARD
#undef COMPAMS_BACKWARD_OF
}

Team team_of(uint32_t rows, uint32_t cols, bool join) { return backward_team(rows, (cols + kGroup - 1) / kGroup, join); }

inline size_t up256(size_t v) { return (v + 255) / 256 * 256; }

}  // namespace

// Parts are a function of a worker's rows and columns alone, so that its sums do not depend on the other workers.  Small
// ones fill the device with few workers, large ones leave fewer sums to be joined with many; us by rows of a part, 768
// columns, norm / join:
//   1 x 1024:  8 15.0 / 16.3,  16 14.9 / 16.5,  32 17.4 / 23.9      8 x 1024: 8 17.3, 16 17.8, 32 21.7 (norm)
//   1 x 8192: 16 18.4 / 27.2,  32 21.7 / 33.8,  64 33.2 / 53.0      8 x 8192: 16 168, 32 166, 64 161 (join)
// (5 x 211 x 1111, norm: 4 15.4, 8 15.4; 3 x 401 x 1601, join: 4 17.9, 8 17.4, 16 22.9; 8 x 256 x 12000, join: 8 109, 16 122;
// 8 x 2048 x 4096, join: 8 234, 16 227, 32 232.)  Short rows are cheap and their teams many: two turns for each (join, 8 x 6167
// x 173, 8 teams: 8 41.7, 16 32.7; 8 x 13028 x 68, 16 teams: 16 41.9, 32 31.4; 1 x 6167 x 256: 8 16.9, 16 17.0).  A few rows
// of a workgroup each take a compute unit 2 to 4 us apiece (join, 8 x 24 x 9062: 4 27.4, 8 35.9; 5 x 61 x 7431: 4 28.2, 8 34.6;
// 8 x 128 x 6000: 4 30.1, 8 31.6; beyond that the sums weigh more: 8 x 256 x 12000 4 91.8, 8 82.6).
Cut norm_cut(uint32_t n, uint32_t rows, uint32_t cols, bool join, bool gradients) {
  Cut c = {};
  if (rows == 0) return c;
  const Team team = team_of(rows, cols, join);
  const uint32_t together = team.each ? team_threads(team) / team.lanes : 1;
  c.part_rows = team.each && team.kind == kBlock && rows <= 128 ? 4 : 8;
  while (c.part_rows < 64 && c.part_rows * 2 <= rows / 512) c.part_rows *= 2;
  if (team.kind == kInWave && team.lanes < 64 && c.part_rows < 2 * together) c.part_rows = 2 * together;
  if (rows <= 4 * together) c.part_rows = rows;  // a few turns, and no launch to join (8 x 16 x 1000 15.8 -> 11.1 us)
  c.parts = (rows + c.part_rows - 1) / c.part_rows;
  if (team.each == 0) c.sums_bytes = up256(static_cast<size_t>(n) * rows * sizeof(float2));
  if (gradients && c.parts > 1)
    c.partial_bytes = up256(static_cast<size_t>(n) * c.parts * kGradients * cols * sizeof(float));
  return c;
}

hipError_t norm_backward(const NormArgs& k, int32_t type, int32_t stream_type, hipStream_t stream) {
  const bool gradients = k.grad[0] || k.grad[1] || k.grad[2];
  if (k.rows == 0) {
    if (k.accumulate || !gradients) return hipSuccess;
    hipLaunchKernelGGL(k_norm_no_rows, dim3(at_most((k.cols + 255) / 256, 4096), kGradients, k.n), dim3(256), 0, stream, k);
    return hipGetLastError();
  }
  const Team team = team_of(k.rows, k.cols, k.join);
  return by_types(type, stream_type, [&](auto t, auto h) {
    using T = decltype(t);
    using H = decltype(h);
    if (team.each == 0) {
      hipLaunchKernelGGL((k_norm_sums_wide<T, H>), dim3(blocks_for(k.total)), dim3(kWideThreads), 0, stream, k);
      constexpr uint32_t kTileCols = kTileGroups * kGroup;
      if (gradients)
        hipLaunchKernelGGL((k_norm_columns_wide<T, H>), dim3((k.cols + kTileCols - 1) / kTileCols, at_most(k.parts, 32768), k.n),
                           dim3(kTileGroups * kTileRows), 0, stream, k);
      // (the outputs last: they may be the inputs' own buffers)
      if (k.dx || k.dresidual)
        hipLaunchKernelGGL((k_norm_backward_wide<T, H>), dim3(blocks_for(k.total)), dim3(kWideThreads), 0, stream, k);
    } else if (k.join) {
      launch_team<T, H, true>(team, k, stream);
    } else {
      launch_team<T, H, false>(team, k, stream);
    }
    if (gradients && k.parts > 1)
      hipLaunchKernelGGL(k_norm_join_parts, dim3(at_most((k.cols + 63) / 64, 4096), kGradients, k.n),
                         dim3(64 * at_most(k.parts, kJoinWaves)), 0, stream, k);
    return hipGetLastError();
  });
}

}  // namespace compams
