// Layer norm and the join of a transformer block, forward.
#include <math.h>

#include "compams_norm.h"

namespace compams {
namespace {

// ---- Rows that a team of lanes holds in registers ---------------------------------------------------------------
// Its lanes take the row's groups of eight columns in turn, NG of them each; the row is read once, and mean and variance are
// two sums over what the registers hold.  65536 x 768 from fp32 to bfloat16: 53 us, 5.7 TB/s; the join with an fp32 stream:
// 114 us, 5.3 TB/s; kernels that only read and write the same arrays take 52 and 108.
// kFullGroups: the team has no lane to spare and everything that a call may leave out is there - the usual widths and the
// usual calls, without a test of any of it for every group (a join of rows of 768: 177 vector instructions a group for 494).
// kWholeGroups: the same calls of a multiple of eight columns, where only lanes without a group are told apart (8 x 6167 x 576,
// join with an fp32 stream: 68.2 us, with the masks of any width 89.7).
template <typename T, typename H, uint32_t NG, TeamKind KIND, bool JOIN, Width WIDTH>
__global__ __launch_bounds__(KIND == kInWave ? kTeamThreads : 1024) void k_norm_forward(NormArgs a, uint32_t lanes) {
  constexpr bool FULL = WIDTH == kFullGroups || WIDTH == kWholeGroups;  // nothing is left out of the call
  __shared__ float slots[2][1][kSlots];
  const uint32_t team = team_of_lane<KIND>(lanes), lane = lane_of_team<KIND>(lanes, team);
  const uint32_t together = teams_together<KIND>(lanes);
  const uint64_t offset = JOIN ? drop_offset(a.drop) : 0u;
  for (uint32_t first = blockIdx.x * together; first < a.total; first += gridDim.x * together) {
    // (a team without a row of its own goes over the last one again: the teams of a pair meet at barriers)
    const bool spare = KIND != kBlock && first + team >= a.total;
    if (KIND == kInWave && spare) break;
    const uint32_t r = spare ? a.total - 1 : first + team;
    typename Group<float>::type g[NG], b[NG];
    float v[NG][kGroup];
    if constexpr (JOIN) {
      typename Group<T>::type x[NG];
      typename Group<H>::type res[NG];
      typename Group<float>::type bias[NG];
#pragma unroll
      for (uint32_t k = 0; k < NG; ++k) x[k] = load_early<WIDTH>(row_of<T>(a.x, a.ld_x, r), (k * lanes + lane) * kGroup, a.cols);
      if (FULL || a.residual) {
#pragma unroll
        for (uint32_t k = 0; k < NG; ++k)
          res[k] = load_early<WIDTH>(row_of<H>(a.residual, a.ld_residual, r), (k * lanes + lane) * kGroup, a.cols);
      }
#pragma unroll
      for (uint32_t k = 0; k < NG; ++k) bias[k] = load_weight_early<WIDTH>(a.bias, (k * lanes + lane) * kGroup, a.cols, 0.0f);
#pragma unroll
      for (uint32_t k = 0; k < NG; ++k) {
        g[k] = load_weight_early<WIDTH>(a.gamma, (k * lanes + lane) * kGroup, a.cols, 1.0f);
        b[k] = load_weight_early<WIDTH>(a.beta, (k * lanes + lane) * kGroup, a.cols, 0.0f);
      }
#pragma unroll
      for (uint32_t k = 0; k < NG; ++k) {
        const uint32_t c = (k * lanes + lane) * kGroup;
        settle_if<WIDTH, T>(x[k], c, a.cols);
        settle_if<WIDTH, float>(bias[k], c, a.cols);
        unpack(v[k], x[k]);
#pragma unroll
        for (uint32_t j = 0; j < kGroup; ++j) v[k][j] += bias[k][j];
        drop_group(v[k], a.drop, offset, r, c);
        if (FULL || a.residual) {
          float w[kGroup];
          settle_if<WIDTH, H>(res[k], c, a.cols);
          unpack(w, res[k]);
#pragma unroll
          for (uint32_t j = 0; j < kGroup; ++j) v[k][j] = w[j] + v[k][j];
        }
      }
    } else {
      typename Group<H>::type x[NG];
#pragma unroll
      for (uint32_t k = 0; k < NG; ++k)
        x[k] = load_early<WIDTH>(row_of<H>(static_cast<const void*>(a.h), a.ld_h, r), (k * lanes + lane) * kGroup, a.cols);
#pragma unroll
      for (uint32_t k = 0; k < NG; ++k) {
        g[k] = load_weight_early<WIDTH>(a.gamma, (k * lanes + lane) * kGroup, a.cols, 1.0f);
        b[k] = load_weight_early<WIDTH>(a.beta, (k * lanes + lane) * kGroup, a.cols, 0.0f);
      }
#pragma unroll
      for (uint32_t k = 0; k < NG; ++k) {
        settle_if<WIDTH, H>(x[k], (k * lanes + lane) * kGroup, a.cols);
        unpack(v[k], x[k]);
      }
    }
    // (columns beyond the last hold 0)
    float s[1] = {0.0f};
#pragma unroll
    for (uint32_t k = 0; k < NG; ++k)
#pragma unroll
      for (uint32_t j = 0; j < kGroup; ++j) s[0] += v[k][j];
    sum_over_team<KIND>(s, slots[0], lanes, team);
    const float mean = mean_of(s[0], a.count);
    s[0] = 0.0f;
#pragma unroll
    for (uint32_t k = 0; k < NG; ++k) {
      const uint32_t c = (k * lanes + lane) * kGroup;
      if (WIDTH == kFullGroups || c + kGroup <= a.cols) {
#pragma unroll
        for (uint32_t j = 0; j < kGroup; ++j) s[0] = fmaf(v[k][j] - mean, v[k][j] - mean, s[0]);
      } else if constexpr (WIDTH != kWholeGroups) {
        uint32_t left = a.cols - c;  // (wraps around where no column is left: negative below)
        forget(left);
#pragma unroll
        for (uint32_t j = 0; j < kGroup; ++j) {
          const float d = static_cast<int32_t>(j) < static_cast<int32_t>(left) ? v[k][j] - mean : 0.0f;
          s[0] = fmaf(d, d, s[0]);
        }
      }
    }
    sum_over_team<KIND>(s, slots[1], lanes, team);
    if (KIND == kPair && spare) continue;
    const float rstd = rstd_of(s[0], a.count, a.eps);
#pragma unroll
    for (uint32_t k = 0; k < NG; ++k) {
      const uint32_t c = (k * lanes + lane) * kGroup;
      if (JOIN && (FULL || a.h)) store_group<H, WIDTH>(row_of<H>(a.h, a.ld_h, r), c, a.cols, v[k]);
      if constexpr (WIDTH != kWholeGroups) {  // (lanes without a group store none)
        settle_if<WIDTH, float>(g[k], c, a.cols);
        settle_if<WIDTH, float>(b[k], c, a.cols);
      }
#pragma unroll
      for (uint32_t j = 0; j < kGroup; ++j) v[k][j] = fmaf((v[k][j] - mean) * rstd, g[k][j], b[k][j]);
      store_group<T, WIDTH>(row_of<T>(a.y, a.ld_y, r), c, a.cols, v[k]);
    }
    if (lane == 0) {
      if (FULL || a.mean) a.mean[r] = mean;
      if (FULL || a.rstd) a.rstd[r] = rstd;
    }
  }
}

// ---- Rows of any width: a workgroup goes over its row once for every sum ---------------------------------------
constexpr uint32_t kWideThreads = 1024;

template <typename T, typename H>
__global__ __launch_bounds__(kWideThreads) void k_norm_forward_wide(NormArgs a) {
  __shared__ float slots[2][1][kSlots];
  const uint64_t offset = a.join ? drop_offset(a.drop) : 0u;
  for (uint32_t r = blockIdx.x; r < a.total; r += gridDim.x) {
    float s[1] = {0.0f};
    for (uint32_t c = threadIdx.x * kGroup; c < a.cols; c += kWideThreads * kGroup) {
      float v[kGroup];
      form_h<T, H>(v, a, offset, r, c);
      for (uint32_t j = 0; j < kGroup; ++j) s[0] += c + j < a.cols ? v[j] : 0.0f;
    }
    sum_block(s, slots[0], kWideThreads / 64);
    const float mean = mean_of(s[0], a.count);
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
    const float rstd = rstd_of(s[0], a.count, a.eps);
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

// The team that a row of `groups` groups is given.  No lane to spare counts most; then few lanes, so that a wavefront's rows
// share what a row costs besides its columns; then few registers.  What is taken and another, us, norm / join, everything
// there, all float16 | from bfloat16 and a stream in fp32:
// 8 x 4096 rows (65536 of 768, 8 x 3117 of 1600 and 1601)
//    768: 32 x 3 38.1 / 72.4 | 52.3 / 110, pair of 96 38.0 / 74.6 | 52.4 / 115, 128 43.5 / 79.6 | 53.9 / 125
//   1000: 64 x 2 26.9 / 53.1 | 36.2 / 80.5, 128 27.3 / 55.6 | 36.7 / 82.6
//   1280: pair of 160 36.2 / 66.7 | 45.5 / 100, 64 x 3 39.7 / 70.0 | 47.5 / 103, 192 35.4 / 70.5 | 46.9 / 105
//   1600: pair of 224 36.2 / 67.5 | 46.3 / 96.6, 256 34.9 / 70.1 | 46.2 / 102
//   1601: pair of 224 44.0 / 92.3 | 48.8 / 109, 256 45.3 / 84.5 | 47.9 / 106 (a join takes 256)
//   2048: 256 56.0 / 108 | 74.8 / 159, 128 x 2 56.8 / 112 | 76.9 / 157, 64 x 4 (a join) 113 | 145
// 8 x 6167 rows (13028 of 68, 2048 of 2304 and 2900, 1000 of 6144 and 7168)
//     68: 8 x 2 11.5 / 20.0 | 11.9 / 21.3, 16 13.6 / 22.3 | 14.0 / 23.3
//    200: 16 x 2 9.3 / 15.2 | 11.0 / 27.3, 32 9.3 / 14.4 | 10.9 / 25.6
//    300: 16 x 3 15.1 / 33.8 | 17.9 / 50.3, 64 22.7 / 41.8 | 24.0 / 45.1 (a join takes 64)
//    384: 16 x 3 13.3 / 30.7 | 21.1 / 43.6, 64 15.5 / 30.5 | 21.8 / 45.8
//    512: 32 x 2 20.5 / 38.0 | 27.8 / 56.3, 64 21.0 / 38.5 | 27.6 / 58.5
//   2304: 192 x 2 38.1 / 69.5 | 47.0 / 95.3, 320 38.8 / 68.3 | 46.7 / 97.0
//   2900: 192 x 2 47.6 / 82.2 | 58.8 / 120, 384 52.4 / 95.0 | 60.3 / 121
//   6144: 384 x 2 51.5 / 102 | 61.6 / 126, 768 58.8 / 79.9 | 64.4 / 118 (a join takes 768)
//   7168: 512 x 2 62.3 / 113 | 70.5 / 139, 896 72.3 / 104 | 80.3 / 158 (a join takes 896)
// Beyond 16384 columns four groups a lane, norm, whole groups: 8 x 300 x 20000 65.5 | 81.7, the route of wide rows 73.3 | 87.5,
// x 30008 90.2 | 115 and 109 | 134 (six or seven registers do not fit).  With the masks of a row's end many more do not (600 x
// 10484 as 384 x 4 121, as 704 x 2 66.9), nor with a join (8 x 200 x 32768 258 | 322, the route of wide rows 178 | 227).
// `whole`: rows of whole groups and nothing left out of the call.  Anything else has the masks, whatever the width (without
// beta 8 x 300 x 30008 float16 four groups a lane 124, the route of wide rows 87; a join without bias 8 x 3117 x 1600 pair 56,
// 256 46).
Team forward_team(uint32_t cols, bool join, bool whole) {
  const uint32_t groups = (cols + kGroup - 1) / kGroup;
  if (groups <= 64) {
    if (groups <= 8) return {kInWave, 8, 1};
    if (groups <= 16) return {kInWave, 8, 2};
    if (groups <= 32) return {kInWave, 16, 2};
    if (groups <= 48) return groups <= 40 && join ? Team{kInWave, 64, 1} : Team{kInWave, 16, 3};
    return {kInWave, 32, 2};
  }
  if (groups <= 96) return {kInWave, 32, 3};
  if (groups <= 128) return {kInWave, 64, 2};
  const uint32_t halves = (groups + 31) / 32;
  if (halves == 5 || (halves == 7 && (!join || whole))) return {kPair, halves * 32, 1};
  if (halves == 8 && join) return {kInWave, 64, 4};
  if (groups > 256 && groups <= 384) return {kBlock, 192, 2};
  if (!join && groups > 640 && groups <= 2048) return {kBlock, (groups + 255) / 256 * 128, 2};
  if (groups > 2048 && groups <= 4096 && whole && !join) return {kBlock, (groups + 255) / 256 * 64, 4};
  const uint32_t each = groups <= 1024 ? 1 : groups <= 2048 ? 2 : 0;
  return {kBlock, each ? (groups + 64 * each - 1) / (64 * each) * 64 : 0, each};
}

bool whole_groups(const NormArgs& k) {
  return k.cols % kGroup == 0 && k.gamma && k.beta && k.mean && k.rstd && (!k.join || (k.bias && k.residual && k.h));
}

template <typename T, typename H, bool JOIN>
void launch_team(const Team& t, const NormArgs& k, hipStream_t stream) {
  const uint32_t threads = team_threads(t), together = threads / t.lanes;
  const dim3 grid(blocks_for((static_cast<uint64_t>(k.total) + together - 1) / together));
  const dim3 block(threads);
  const bool whole = whole_groups(k), full = whole && k.cols == t.lanes * t.each * kGroup;
#define COMPAMS_FORWARD_OF(NG, KIND, WIDTH) \
  hipLaunchKernelGGL((k_norm_forward<T, H, NG, KIND, JOIN, WIDTH>), grid, block, 0, stream, k, t.lanes)
#define COMPAMS_FORWARD(NG, KIND)                           \
  do {                                                      \
    if (full) COMPAMS_FORWARD_OF(NG, KIND, kFullGroups);    \
    else if (whole) COMPAMS_FORWARD_OF(NG, KIND, kWholeGroups); \
    else COMPAMS_FORWARD_OF(NG, KIND, kAnyWidth);           \
  } while (0)
  if (t.kind == kInWave) {
    switch (t.each) {
      case 1:
        if (k.cols < kGroup) COMPAMS_FORWARD_OF(1, kInWave, kOneGroup);
        else COMPAMS_FORWARD(1, kInWave);
        break;
      case 2: COMPAMS_FORWARD(2, kInWave); break;
      case 3: COMPAMS_FORWARD(3, kInWave); break;
      default:
        if constexpr (JOIN) COMPAMS_FORWARD(4, kInWave);
        break;
    }
  } else if (t.kind == kPair) {
    COMPAMS_FORWARD(1, kPair);
  } else {
    switch (t.each) {
      case 1: COMPAMS_FORWARD(1, kBlock); break;
      case 2: COMPAMS_FORWARD(2, kBlock); break;
      default:  // (of whole groups alone)
        if constexpr (!JOIN) {
          if (full) COMPAMS_FORWARD_OF(4, kBlock, kFullGroups);
          else COMPAMS_FORWARD_OF(4, kBlock, kWholeGroups);
        }
        break;
    }
  }
#undef COMPAMS_FORWARD
#undef COMPAMS_FORWARD_OF
}

}  // namespace

hipError_t norm_forward(const NormArgs& k, int32_t type, int32_t stream_type, hipStream_t stream) {
  const Team team = forward_team(k.cols, k.join, whole_groups(k));
  return by_types(type, stream_type, [&](auto t, auto h) {
    using T = decltype(t);
    using H = decltype(h);
    if (team.each == 0)
      hipLaunchKernelGGL((k_norm_forward_wide<T, H>), dim3(blocks_for(k.total)), dim3(kWideThreads), 0, stream, k);
    else if (k.join) launch_team<T, H, true>(team, k, stream);
    else launch_team<T, H, false>(team, k, stream);
    return hipGetLastError();
  });
}

}  // namespace compams
