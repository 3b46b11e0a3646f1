// Dropout from a counter-based generator, alone or added to a residual stream.
#include "compams_rows.h"

namespace compams {
namespace {

struct DropoutArgs {
  uint32_t total, cols;
  uint32_t across;  // workgroups side by side in a row
  uint32_t wide;    // lanes side by side in a workgroup: a power of two
  const void *x, *residual;
  void* y;
  int64_t ld_x, ld_residual, ld_y;
  Drop drop;
};
constexpr uint32_t kThreads = 256;

// Bound by memory, with the generator close behind: 20 products of 32 x 32 bits for eight columns (one row a lane, its place
// formed for itself, 82 % of the vector unit's time).  49152 x 1024 bfloat16: 36.7 us, 5.5 TB/s; without arithmetic 35.5.
constexpr uint32_t kRows = 4;  // rows that a lane takes, its columns in each

// FULL: a multiple of eight columns, a lane has a whole group or none (8 x 1127 x 1816 added to an fp32 stream 39.0 us, 1812
// 47.3).  SAME: a wavefront's lanes are all in one row, whose number is a scalar then, and with it two of the generator's
// twenty products.
template <typename X, typename Y, bool FULL, bool SAME, bool ADD>
__global__ __launch_bounds__(kThreads) void k_dropout(DropoutArgs a) {
  const uint32_t tall = kThreads / a.wide;
  const uint32_t c = (blockIdx.x % a.across * a.wide + (threadIdx.x & (a.wide - 1))) * kGroup;
  if (c >= a.cols) return;
  uint32_t down = threadIdx.x / a.wide;
  if constexpr (SAME) down = __builtin_amdgcn_readfirstlane(down);
  const uint64_t offset = drop_offset(a.drop);
  const uint32_t step = gridDim.x / a.across * tall * kRows;
  for (uint64_t first = blockIdx.x / a.across * tall * kRows + down; first < a.total; first += step) {
    typename Group<X>::type x[kRows];
    typename Group<Y>::type res[kRows];
#pragma unroll
    for (uint32_t q = 0; q < kRows; ++q) {
      // (a row beyond the last: the last one again, not stored below)
      const uint64_t in = first + q * tall, r = in < a.total ? in : a.total - 1;
      const X* const from = static_cast<const X*>(a.x) + static_cast<int64_t>(r) * a.ld_x;
      x[q] = FULL ? load_early<kFullGroups>(from, c, a.cols) : load_raw(from, c, a.cols);
      if constexpr (ADD) {
        const Y* const add = static_cast<const Y*>(a.residual) + static_cast<int64_t>(r) * a.ld_residual;
        res[q] = FULL ? load_early<kFullGroups>(add, c, a.cols) : load_raw(add, c, a.cols);
      }
    }
#pragma unroll
    for (uint32_t q = 0; q < kRows; ++q) {
      const uint64_t r = first + q * tall;
      if (r >= a.total) break;
      float v[kGroup];
      unpack(v, x[q]);
      drop_group(v, a.drop, offset, static_cast<uint32_t>(r), c);
      if constexpr (ADD) {
        float w[kGroup];
        unpack(w, res[q]);
#pragma unroll
        for (uint32_t j = 0; j < kGroup; ++j) v[j] = w[j] + v[j];
      }
      store_group<Y, FULL ? kFullGroups : kAnyWidth>(static_cast<Y*>(a.y) + static_cast<int64_t>(r) * a.ld_y, c, a.cols, v);
    }
  }
}

template <typename X, typename Y, bool ADD>
void launch_by_width(const DropoutArgs& a, uint32_t blocks, hipStream_t stream) {
  const bool full = a.cols % kGroup == 0;
  if (full && a.wide >= 64) hipLaunchKernelGGL((k_dropout<X, Y, true, true, ADD>), dim3(blocks), dim3(kThreads), 0, stream, a);
  else if (full) hipLaunchKernelGGL((k_dropout<X, Y, true, false, ADD>), dim3(blocks), dim3(kThreads), 0, stream, a);
  else hipLaunchKernelGGL((k_dropout<X, Y, false, false, ADD>), dim3(blocks), dim3(kThreads), 0, stream, a);
}
template <typename X, typename Y>
hipError_t launch_dropout(const DropoutArgs& a, uint32_t blocks, hipStream_t stream) {
  if (a.residual) launch_by_width<X, Y, true>(a, blocks, stream);
  else launch_by_width<X, Y, false>(a, blocks, stream);
  return hipGetLastError();
}

}  // namespace
}  // namespace compams

extern "C" int compams_dropout(int32_t n, int64_t rows, int64_t cols, int32_t x_type, int32_t y_type, const void* x,
                               int64_t ld_x, const void* residual, int64_t ld_residual, void* y, int64_t ld_y,
                               const compams_drop* drop, void* hip_stream) {
  using namespace compams;
  if (!rows_valid(n, rows, cols) || !float_type(x_type) || !float_type(y_type) || !drop || !drop_valid(*drop))
    return COMPAMS_INVALID_ARG;
  if (x_type != y_type && x_type != COMPAMS_F32 && y_type != COMPAMS_F32) return COMPAMS_INVALID_ARG;
  if (rows == 0) return COMPAMS_OK;
  if (!x || !y || !stride_valid(ld_x, cols) || !stride_valid(ld_y, cols) || (residual && !stride_valid(ld_residual, cols)))
    return COMPAMS_INVALID_ARG;
  if (!aligned_to(x, type_size(x_type)) || !aligned_to(y, type_size(y_type)) || !aligned_to(residual, type_size(y_type)) ||
      !aligned_to(drop->step, 8))
    return COMPAMS_BAD_ALIGNMENT;
  DropoutArgs a = {};
  a.total = static_cast<uint32_t>(n * rows);
  a.cols = static_cast<uint32_t>(cols);
  a.x = x; a.residual = residual; a.y = y;
  a.ld_x = ld_x; a.ld_residual = ld_residual; a.ld_y = ld_y;
  a.drop = make_drop(*drop);
  const uint32_t groups = (a.cols + kGroup - 1) / kGroup;
  // As many lanes side by side as divide a row into whole parts, if that is half a wavefront or more; else one part, or
  // parts of a workgroup, with lanes to spare.
  a.wide = kThreads;
  while (a.wide > 1 && groups % a.wide != 0) a.wide /= 2;
  if (a.wide < 32) {
    a.wide = 1;
    while (a.wide < groups && a.wide < kThreads) a.wide *= 2;
  }
  a.across = (groups + a.wide - 1) / a.wide;
  const uint32_t tall = kThreads / a.wide;
  // (a dimension has room for 2^32 threads: rows beyond are taken in further turns)
  const uint64_t down = (static_cast<uint64_t>(a.total) + tall * kRows - 1) / (tall * kRows), most = (1u << 23) / a.across;
  const uint32_t blocks = static_cast<uint32_t>(down < most ? down : most > 0 ? most : 1) * a.across;
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  hipError_t err;
  if (x_type == COMPAMS_F32)
    err = y_type == COMPAMS_F32   ? launch_dropout<float, float>(a, blocks, stream)
          : y_type == COMPAMS_F16 ? launch_dropout<float, half_t>(a, blocks, stream)
                                  : launch_dropout<float, bfloat_t>(a, blocks, stream);
  else if (x_type == COMPAMS_F16)
    err = y_type == COMPAMS_F32 ? launch_dropout<half_t, float>(a, blocks, stream)
                                : launch_dropout<half_t, half_t>(a, blocks, stream);
  else
    err = y_type == COMPAMS_F32 ? launch_dropout<bfloat_t, float>(a, blocks, stream)
                                : launch_dropout<bfloat_t, bfloat_t>(a, blocks, stream);
  return err == hipSuccess ? COMPAMS_OK : COMPAMS_HIP_ERROR;
}
