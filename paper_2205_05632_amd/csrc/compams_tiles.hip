// What the product kernels share besides their tiles: operands copied to where they can be read in whole pieces.
#include "compams_tiles.h"

namespace compams {
namespace {

// One lane to a piece of 16 bytes; bound by memory.  (Rows that start on 16 bytes and have whole pieces are not copied.)
template <typename T>
__global__ __launch_bounds__(256) void k_pack(Packing p) {
  constexpr uint32_t kEach = 16 / sizeof(T);
  typedef typename Fragment<T>::type Piece;
  const Packing::Job& j = p.job[blockIdx.y];
  for (uint64_t i = blockIdx.x * 256u + threadIdx.x; i < j.pieces; i += gridDim.x * 256u) {
    const uint64_t row = i / j.per_row;
    const uint32_t c = static_cast<uint32_t>(i - row * j.per_row) * kEach;
    const T* const from = static_cast<const T*>(j.from) + static_cast<int64_t>(row) * j.ld + c;
    Piece v;
    if (c + kEach <= j.cols) {
      __builtin_memcpy(&v, from, sizeof(v));  // (wherever it starts)
    } else {
#pragma unroll
      for (uint32_t k = 0; k < kEach; ++k) v[k] = c + k < j.cols ? from[k] : static_cast<T>(0.0f);
    }
    static_cast<Piece*>(j.to)[i] = v;
  }
}

}  // namespace

void run_packing(const Packing& p, size_t size, hipStream_t stream) {
  if (p.count == 0) return;
  uint64_t most = 1;
  for (uint32_t i = 0; i < p.count; ++i) most = p.job[i].pieces > most ? p.job[i].pieces : most;
  const uint64_t blocks = (most + 255) / 256;
  const dim3 grid(static_cast<uint32_t>(blocks < 16384 ? blocks : 16384), p.count);
  if (size == 4) hipLaunchKernelGGL(k_pack<float>, grid, dim3(256), 0, stream, p);
  else hipLaunchKernelGGL(k_pack<half_t>, grid, dim3(256), 0, stream, p);  // (bits)
}

}  // namespace compams
