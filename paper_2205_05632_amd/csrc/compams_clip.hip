// The norm of every worker's gradient over all its tensors, and the gradient cut to a largest norm.
#include "compams_rows.h"

namespace compams {
namespace {

constexpr uint32_t kThreads = 256;
constexpr uint32_t kTurns = 4;                               // groups of eight entries to a lane
constexpr uint32_t kChunk = kThreads * kGroup * kTurns;      // entries of a tensor's row to a workgroup

// The tensors of a launch: they travel with the kernel's arguments.
constexpr uint32_t kMostTensors = 64;
struct Tensor {
  const void* from;
  void* to;
  int64_t ld_from, ld_to;
  int64_t count;
  uint32_t first;           // number of its first chunk in the launch
  uint16_t from_type, to_type;
};
struct ClipArgs {
  uint32_t n, tensors, chunks;    // of the launch; chunks: of a worker
  uint32_t before, all;           // chunks of a worker in the launches before, and in all
  double* partial;                // [worker][chunk]
  float *norms, *factors;         // of the workspace
  float *norms_out, *factors_out;
  float max_norm, scale;
  Tensor tensor[kMostTensors];
};

// The tensor that chunk number c is of.
__device__ __forceinline__ uint32_t tensor_of(const ClipArgs& a, uint32_t c) {
  uint32_t at = 0;
#pragma unroll
  for (uint32_t step = kMostTensors / 2; step > 0; step /= 2)
    if (at + step < a.tensors && a.tensor[at + step].first <= c) at += step;
  return at;
}

__device__ __forceinline__ double sum_wave(double v) {
#pragma unroll
  for (int d = 32; d > 0; d /= 2) v += __shfl_xor(v, d);
  return v;
}
// Over a workgroup of `waves` wavefronts, in the first lane.
__device__ __forceinline__ double sum_doubles(double v, double* slots, uint32_t waves) {
  v = sum_wave(v);
  if (threadIdx.x % 64 == 0) slots[threadIdx.x / 64] = v;
  __syncthreads();
  double s = slots[0];
  for (uint32_t k = 1; k < waves; ++k) s += slots[k];
  return s;
}

// What is beyond the row's last entry is 0.
template <typename T>
__device__ __forceinline__ void load_eight(float (&v)[kGroup], const T* row, int64_t c, int64_t count) {
  if (c + kGroup <= count) {
    typename Group<T>::type raw;
    __builtin_memcpy(&raw, row + c, sizeof(raw));
    unpack(v, raw);
  } else {
#pragma unroll
    for (uint32_t j = 0; j < kGroup; ++j) v[j] = c + j < count ? to_float(row[c + j]) : 0.0f;
  }
}
template <typename T>
__device__ __forceinline__ void store_eight(T* row, int64_t c, int64_t count, const float (&v)[kGroup]) {
  if (c + kGroup <= count) {
    typename Group<T>::type raw;
#pragma unroll
    for (uint32_t j = 0; j < kGroup; ++j) raw[j] = static_cast<T>(v[j]);
    __builtin_memcpy(row + c, &raw, sizeof(raw));
  } else {
#pragma unroll
    for (uint32_t j = 0; j < kGroup; ++j)
      if (c + j < count) row[c + j] = static_cast<T>(v[j]);
  }
}

template <typename T>
__device__ __forceinline__ double squares(const Tensor& t, uint32_t w, uint32_t chunk) {
  const T* const row = static_cast<const T*>(t.from) + static_cast<int64_t>(w) * t.ld_from;
  const int64_t first = static_cast<int64_t>(chunk) * kChunk + threadIdx.x * kGroup;
  float v[kTurns][kGroup];
#pragma unroll
  for (uint32_t k = 0; k < kTurns; ++k) load_eight(v[k], row, first + k * kThreads * kGroup, t.count);
  double s = 0.0;
#pragma unroll
  for (uint32_t k = 0; k < kTurns; ++k)
#pragma unroll
    for (uint32_t j = 0; j < kGroup; ++j) s = fma(static_cast<double>(v[k][j]), static_cast<double>(v[k][j]), s);
  return s;
}

// Bound by memory.  A square of an fp32 number is exact in fp64 up to its last five bits, and no sum of them leaves its range.
__global__ __launch_bounds__(kThreads) void k_clip_norm(ClipArgs a) {
  __shared__ double slots[kThreads / 64];
  const uint32_t w = blockIdx.y, i = tensor_of(a, blockIdx.x);
  const Tensor& t = a.tensor[i];
  const uint32_t chunk = blockIdx.x - t.first;
  double s = t.from_type == COMPAMS_F32   ? squares<float>(t, w, chunk)
             : t.from_type == COMPAMS_F16 ? squares<half_t>(t, w, chunk)
                                          : squares<bfloat_t>(t, w, chunk);
  s = sum_doubles(s, slots, kThreads / 64);
  if (threadIdx.x == 0) a.partial[static_cast<uint64_t>(w) * a.all + a.before + blockIdx.x] = s;
}

__global__ __launch_bounds__(kThreads) void k_clip_factor(ClipArgs a) {
  __shared__ double slots[kThreads / 64];
  const uint32_t w = blockIdx.x;
  double s = 0.0;
  for (uint32_t c = threadIdx.x; c < a.all; c += kThreads) s += a.partial[static_cast<uint64_t>(w) * a.all + c];
  s = sum_doubles(s, slots, kThreads / 64);
  if (threadIdx.x != 0) return;
  const double norm = sqrt(s) * a.scale;
  const float factor = !(s < INFINITY) ? 0.0f : norm > a.max_norm ? static_cast<float>(a.scale * (a.max_norm / norm)) : a.scale;
  a.factors[w] = factor;
  if (a.norms_out) a.norms_out[w] = static_cast<float>(norm);
  if (a.factors_out) a.factors_out[w] = factor;
  // (a factor of 0 tells the next kernel to write zeros whatever is there; one that underflows does the same)
}

template <typename F, typename T>
__device__ __forceinline__ void scaled(const Tensor& t, uint32_t w, uint32_t chunk, float factor) {
  const F* const row = static_cast<const F*>(t.from) + static_cast<int64_t>(w) * t.ld_from;
  T* const to = static_cast<T*>(t.to) + static_cast<int64_t>(w) * t.ld_to;
  const int64_t first = static_cast<int64_t>(chunk) * kChunk + threadIdx.x * kGroup;
  float v[kTurns][kGroup];
#pragma unroll
  for (uint32_t k = 0; k < kTurns; ++k) load_eight(v[k], row, first + k * kThreads * kGroup, t.count);
#pragma unroll
  for (uint32_t k = 0; k < kTurns; ++k) {
#pragma unroll
    for (uint32_t j = 0; j < kGroup; ++j) v[k][j] = factor == 0.0f ? 0.0f : v[k][j] * factor;
    store_eight(to, first + k * kThreads * kGroup, t.count, v[k]);
  }
}

// A chunk that is multiplied by one where it stands is left alone.
__global__ __launch_bounds__(kThreads) void k_clip_scale(ClipArgs a) {
  const uint32_t w = blockIdx.y, i = tensor_of(a, blockIdx.x);
  const Tensor& t = a.tensor[i];
  const uint32_t chunk = blockIdx.x - t.first;
  const float factor = a.factors[w];
  if (!t.to || (factor == 1.0f && t.to == t.from && t.ld_to == t.ld_from)) return;
  if (t.from_type == COMPAMS_F32) scaled<float, float>(t, w, chunk, factor);
  else if (t.from_type == COMPAMS_F16 && t.to_type == COMPAMS_F16) scaled<half_t, half_t>(t, w, chunk, factor);
  else if (t.from_type == COMPAMS_F16) scaled<half_t, float>(t, w, chunk, factor);
  else if (t.to_type == COMPAMS_BF16) scaled<bfloat_t, bfloat_t>(t, w, chunk, factor);
  else scaled<bfloat_t, float>(t, w, chunk, factor);
}

// ---- Checks --------------------------------------------------------------------------------------------------
inline uint64_t chunks_of(const compams_clip_tensor& t) { return (static_cast<uint64_t>(t.count) + kChunk - 1) / kChunk; }
int check(const compams_clip* a) {
  if (!a || a->n < 1 || a->n > 65535 || a->tensors < 0 || (a->tensors > 0 && !a->tensor) || !(a->max_norm >= 0.0f) ||
      !(a->scale > 0.0f) || a->scale == INFINITY)
    return COMPAMS_INVALID_ARG;
  uint64_t chunks = 0;
  for (int32_t i = 0; i < a->tensors; ++i) {
    const compams_clip_tensor& t = a->tensor[i];
    constexpr int64_t kMost = static_cast<int64_t>(1) << 40;
    if (t.count < 0 || t.count >= kMost || !float_type(t.from_type)) return COMPAMS_INVALID_ARG;
    if (t.count == 0) continue;
    if (!t.from || (a->n > 1 && (t.ld_from < t.count || t.ld_from >= kMost))) return COMPAMS_INVALID_ARG;
    if (!aligned_to(t.from, type_size(t.from_type))) return COMPAMS_BAD_ALIGNMENT;
    if (t.to) {
      if (!float_type(t.to_type) || (t.to_type != t.from_type && t.to_type != COMPAMS_F32) ||
          (a->n > 1 && (t.ld_to < t.count || t.ld_to >= kMost)) || (t.to == t.from && t.to_type != t.from_type))
        return COMPAMS_INVALID_ARG;
      if (!aligned_to(t.to, type_size(t.to_type))) return COMPAMS_BAD_ALIGNMENT;
    }
    chunks += chunks_of(t);
  }
  // (a launch's workgroups of one worker: 2^24 in a dimension of 2^32 threads)
  return chunks < (1u << 24) - 1 ? COMPAMS_OK : COMPAMS_INVALID_ARG;
}
inline size_t up256(size_t v) { return (v + 255) / 256 * 256; }
uint64_t all_chunks(const compams_clip& a) {
  uint64_t c = 0;
  for (int32_t i = 0; i < a.tensors; ++i) c += chunks_of(a.tensor[i]);
  return c;
}
size_t factors_bytes(const compams_clip& a) { return up256(static_cast<size_t>(a.n) * sizeof(float)); }
size_t bytes_of(const compams_clip& a) { return factors_bytes(a) + up256(static_cast<size_t>(a.n) * all_chunks(a) * sizeof(double)); }

// launch(k) for every kMostTensors tensors.
template <typename Launch>
void by_launch(const compams_clip& a, ClipArgs& k, Launch launch) {
  k.before = 0;
  for (int32_t i = 0; i < a.tensors;) {
    k.tensors = k.chunks = 0;
    for (; i < a.tensors && k.tensors < kMostTensors; ++i) {
      const compams_clip_tensor& t = a.tensor[i];
      if (t.count == 0) continue;
      k.tensor[k.tensors++] = {t.from, t.to, t.ld_from, t.ld_to, t.count, k.chunks, static_cast<uint16_t>(t.from_type), static_cast<uint16_t>(t.to_type)};
      k.chunks += static_cast<uint32_t>(chunks_of(t));
    }
    if (k.chunks) launch(k);
    k.before += k.chunks;
  }
}

}  // namespace
}  // namespace compams

extern "C" {

size_t compams_clip_workspace_size(const compams_clip* a) {
  return compams::check(a) == COMPAMS_OK ? compams::bytes_of(*a) : 0;
}

int compams_clip_gradients(const compams_clip* a, void* hip_stream) {
  using namespace compams;
  const int checked = check(a);
  if (checked != COMPAMS_OK) return checked;
  if (!aligned_to(a->norms, 4) || !aligned_to(a->factors, 4)) return COMPAMS_BAD_ALIGNMENT;
  if (!a->workspace) return COMPAMS_INVALID_ARG;
  if (!aligned_to(a->workspace, 256)) return COMPAMS_BAD_ALIGNMENT;
  if (a->workspace_bytes < bytes_of(*a)) return COMPAMS_WORKSPACE_TOO_SMALL;
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  ClipArgs k = {};
  k.n = static_cast<uint32_t>(a->n);
  k.all = static_cast<uint32_t>(all_chunks(*a));
  k.factors = static_cast<float*>(a->workspace);
  k.partial = reinterpret_cast<double*>(static_cast<char*>(a->workspace) + factors_bytes(*a));
  k.norms_out = a->norms;
  k.factors_out = a->factors;
  k.max_norm = a->max_norm;
  k.scale = a->scale;
  by_launch(*a, k, [&](const ClipArgs& l) { hipLaunchKernelGGL(k_clip_norm, dim3(l.chunks, l.n), dim3(kThreads), 0, stream, l); });
  hipLaunchKernelGGL(k_clip_factor, dim3(k.n), dim3(kThreads), 0, stream, k);
  by_launch(*a, k, [&](const ClipArgs& l) { hipLaunchKernelGGL(k_clip_scale, dim3(l.chunks, l.n), dim3(kThreads), 0, stream, l); });
  return hipGetLastError() == hipSuccess ? COMPAMS_OK : COMPAMS_HIP_ERROR;
}

}  // extern "C"
