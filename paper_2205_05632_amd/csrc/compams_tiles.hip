// What the product kernels share besides their tiles: operands copied to where they can be read in whole pieces.
#include "compams_tiles.h"

namespace compams {
namespace {

// A workgroup takes whole rows, a lane a piece of 16 bytes of each of AT_ONCE at a time, as many lanes side by side as a row
// has pieces.  (Rows that start on 16 bytes and have whole pieces are not copied.)
template <typename T>
__device__ __forceinline__ typename Fragment<T>::type piece_of(const T* from, uint32_t c, uint32_t cols) {
  constexpr uint32_t kEach = 16 / sizeof(T);
  typename Fragment<T>::type v = {};
  if (c + kEach <= cols) {
    __builtin_memcpy(&v, from + c, sizeof(v));  // (wherever it starts)
  } else {
#pragma unroll
    for (uint32_t k = 0; k < kEach; ++k)
      if (c + k < cols) v[k] = from[c + k];
  }
  return v;
}
template <typename T, uint32_t AT_ONCE>
__global__ __launch_bounds__(256) void k_pack(Packing p) {
  typedef typename Fragment<T>::type Piece;
  const Packing::Job& j = p.job[blockIdx.y];
  const uint32_t side = j.per_row < 256 ? 256 / j.per_row : 1;  // rows side by side
  const uint32_t in = j.per_row < 256 ? threadIdx.x / j.per_row : 0;
  if (in >= side) return;
  const int64_t step = static_cast<int64_t>(gridDim.x) * side * AT_ONCE;
  for (int64_t first = static_cast<int64_t>(blockIdx.x) * side * AT_ONCE + in; first < j.rows; first += step)
    for (uint32_t c = threadIdx.x - in * j.per_row; c < j.per_row; c += 256) {
      Piece v[AT_ONCE];
#pragma unroll
      for (uint32_t q = 0; q < AT_ONCE; ++q) {
        const int64_t r = first + q * side;
        v[q] = piece_of(static_cast<const T*>(j.from) + (r < j.rows ? r : j.rows - 1) * j.ld, c * (16 / sizeof(T)), j.cols);
      }
#pragma unroll
      for (uint32_t q = 0; q < AT_ONCE; ++q) {
        const int64_t r = first + q * side;
        if (r < j.rows) static_cast<Piece*>(j.to)[r * j.per_row + c] = v[q];
      }
    }
}

}  // namespace

void run_packing(const Packing& p, size_t size, hipStream_t stream) {
  if (p.count == 0) return;
  const auto blocks = [&](uint32_t at_once) {
    uint64_t most = 1;
    for (uint32_t i = 0; i < p.count; ++i) {
      const Packing::Job& j = p.job[i];
      const uint64_t each = static_cast<uint64_t>(j.per_row < 256 ? 256 / j.per_row : 1) * at_once;
      const uint64_t of_job = (static_cast<uint64_t>(j.rows) + each - 1) / each;
      most = of_job > most ? of_job : most;
    }
    return static_cast<uint32_t>(most < 16384 ? most : 16384);
  };
  // (10007 x 777 float16 9.4 us with four, 1111 x 777 7.7)
  const bool many = blocks(4) >= 1024;
  const dim3 grid(blocks(many ? 4 : 1), p.count);
#define COMPAMS_PACK(T, AT_ONCE) hipLaunchKernelGGL((k_pack<T, AT_ONCE>), grid, dim3(256), 0, stream, p)
  if (size == 4 && many) COMPAMS_PACK(float, 4);
  else if (size == 4) COMPAMS_PACK(float, 1);
  else if (many) COMPAMS_PACK(half_t, 4);  // (bits)
  else COMPAMS_PACK(half_t, 1);
#undef COMPAMS_PACK
}

}  // namespace compams
