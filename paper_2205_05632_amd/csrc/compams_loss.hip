// Softmax cross-entropy with its gradient, every worker's loss the mean over its tokens.
#include <math.h>

#include "compams_rows.h"

namespace compams {
namespace {

struct LossArgs {
  uint32_t n, rows, vocab, total;
  const void* logits;
  void* dlogits;
  int64_t ld_logits, ld_dlogits;
  const void* targets;
  bool wide_targets;  // 64 bits
  int64_t ignore;
  float grad_scale;
  float *mean_loss, *losses;
  uint32_t* counts;  // per worker: rows that are learnt from
};

__device__ __forceinline__ int64_t target_of(const LossArgs& a, uint32_t r) {
  return a.wide_targets ? static_cast<const int64_t*>(a.targets)[r]
                        : static_cast<int64_t>(static_cast<const int32_t*>(a.targets)[r]);
}

constexpr uint32_t kLossThreads = 1024, kLossWaves = kLossThreads / 64;

struct Max {
  // (a NaN on either side is passed over here; it comes back through the sum)
  __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};

__global__ __launch_bounds__(kLossThreads) void k_loss_count(LossArgs a) {
  __shared__ float slots[1][16];
  for (uint32_t w = blockIdx.x; w < a.n; w += gridDim.x) {
    uint32_t mine = 0;
    for (uint32_t i = threadIdx.x; i < a.rows; i += kLossThreads) mine += target_of(a, w * a.rows + i) != a.ignore;
    // two halves, each exact in fp32 (a worker has fewer than 2^31 rows, a lane at most 2^21 of them)
    __syncthreads();
    float s[1] = {static_cast<float>(mine & 0xfffu)};
    sum_block(s, slots, kLossWaves);
    __syncthreads();
    float t[1] = {static_cast<float>(mine >> 12)};
    sum_block(t, slots, kLossWaves);
    if (threadIdx.x == 0) a.counts[w] = static_cast<uint32_t>(s[0]) + (static_cast<uint32_t>(t[0]) << 12);
  }
}

// Rows of any width: a workgroup goes over its row twice, once for the running maximum and sum, once for the gradient.
template <typename T>
__global__ __launch_bounds__(kLossThreads) void k_loss_wide(LossArgs a) {
  __shared__ float slots[2][kLossWaves];
  for (uint32_t r = blockIdx.x; r < a.total; r += gridDim.x) {
    const int64_t target = target_of(a, r);
    const T* const row = static_cast<const T*>(a.logits) + static_cast<int64_t>(r) * a.ld_logits;
    T* const out = a.dlogits ? static_cast<T*>(a.dlogits) + static_cast<int64_t>(r) * a.ld_dlogits : nullptr;
    if (target == a.ignore) {
      if (a.losses && threadIdx.x == 0) a.losses[r] = 0.0f;
      const float zero[kGroup] = {};
      if (out)
        for (uint32_t c = threadIdx.x * kGroup; c < a.vocab; c += kLossThreads * kGroup) store_group(out, c, a.vocab, zero);
      continue;
    }
    const bool inside = target >= 0 && target < static_cast<int64_t>(a.vocab);
    const float of_target = inside ? to_float(row[target]) : __builtin_nanf("");
    float top = -INFINITY, sum = 0.0f;
    for (uint32_t c = threadIdx.x * kGroup; c < a.vocab; c += kLossThreads * kGroup) {
      float v[kGroup];
      load_group(v, row, c, a.vocab);
      float m = top;
#pragma unroll
      for (uint32_t j = 0; j < kGroup; ++j) m = c + j < a.vocab ? fmaxf(m, v[j]) : m;
      // (no finite entry so far: a lane's sum stays 0, or becomes NaN with one)
      sum = top == -INFINITY ? sum : sum * expf(top - m);
      top = m;
#pragma unroll
      for (uint32_t j = 0; j < kGroup; ++j)
        if (c + j < a.vocab) sum += v[j] == -INFINITY ? 0.0f : expf(v[j] - top);
    }
    const float wave_top = over_lanes(top, 64, Max());
    __syncthreads();  // the slots may still be read for the row before
    if ((threadIdx.x & 63u) == 0) slots[0][threadIdx.x >> 6] = wave_top;
    __syncthreads();
    float all_top = slots[0][0];
    for (uint32_t w = 1; w < kLossWaves; ++w) all_top = fmaxf(all_top, slots[0][w]);
    sum = sum_lanes(top == -INFINITY ? sum : sum * expf(top - all_top), 64);
    if ((threadIdx.x & 63u) == 0) slots[1][threadIdx.x >> 6] = sum;
    __syncthreads();
    float all_sum = 0.0f;
    for (uint32_t w = 0; w < kLossWaves; ++w) all_sum += slots[1][w];
    // a row without any finite entry, or with a target that is none, has no softmax and no loss
    const float log_sum = logf(all_sum) + all_top;
    const bool none = !inside || all_top == -INFINITY;
    if (a.losses && threadIdx.x == 0) a.losses[r] = none ? __builtin_nanf("") : log_sum - of_target;
    if (!out) continue;
    const float count = static_cast<float>(a.counts[r / a.rows]);
    const float factor = none ? __builtin_nanf("") : a.grad_scale / count;
    const float share = factor / all_sum;
    for (uint32_t c = threadIdx.x * kGroup; c < a.vocab; c += kLossThreads * kGroup) {
      float v[kGroup];
      load_group(v, row, c, a.vocab);
#pragma unroll
      for (uint32_t j = 0; j < kGroup; ++j)
        v[j] = expf(v[j] - all_top) * share - (static_cast<int64_t>(c + j) == target ? factor : 0.0f);
      store_group(out, c, a.vocab, v);
    }
  }
}

// A worker's losses added up and divided.
__global__ __launch_bounds__(kLossThreads) void k_loss_mean(LossArgs a) {
  __shared__ float slots[2][1][16];
  uint32_t turn = 0;
  for (uint32_t w = blockIdx.x; w < a.n; w += gridDim.x, turn ^= 1) {
    float s[1] = {0.0f};
    for (uint32_t i = threadIdx.x; i < a.rows; i += kLossThreads) s[0] += a.losses[static_cast<size_t>(w) * a.rows + i];
    sum_block(s, slots[turn], kLossWaves);
    if (threadIdx.x == 0) a.mean_loss[w] = a.counts[w] ? s[0] / static_cast<float>(a.counts[w]) : 0.0f;
  }
}

bool loss_valid(const compams_loss* a) {
  return a && rows_valid(a->n, a->rows, a->vocab) && float_type(a->type) &&
         (a->target_type == COMPAMS_I32 || a->target_type == COMPAMS_I64);
}
inline size_t up256(size_t v) { return (v + 255) / 256 * 256; }
inline size_t counts_bytes(const compams_loss& a) { return up256(static_cast<size_t>(a.n) * sizeof(uint32_t)); }
inline size_t losses_bytes(const compams_loss& a) {
  return a.losses || !a.mean_loss ? 0 : up256(static_cast<size_t>(a.n) * a.rows * sizeof(float));
}

}  // namespace
}  // namespace compams

extern "C" {

size_t compams_loss_workspace_size(const compams_loss* a) {
  return compams::loss_valid(a) ? compams::counts_bytes(*a) + compams::losses_bytes(*a) : 0;
}

int compams_cross_entropy(const compams_loss* a, void* hip_stream) {
  using namespace compams;
  if (!loss_valid(a) || (!a->mean_loss && !a->losses && !a->dlogits)) return COMPAMS_INVALID_ARG;
  if (!aligned_to(a->mean_loss, 4) || !aligned_to(a->losses, 4)) return COMPAMS_BAD_ALIGNMENT;
  if (a->rows > 0) {
    if (!a->logits || !a->targets || !stride_valid(a->ld_logits, a->vocab) ||
        (a->dlogits && !stride_valid(a->ld_dlogits, a->vocab)))
      return COMPAMS_INVALID_ARG;
    if (!aligned_to(a->logits, type_size(a->type)) || !aligned_to(a->dlogits, type_size(a->type)) ||
        !aligned_to(a->targets, type_size(a->target_type)))
      return COMPAMS_BAD_ALIGNMENT;
  }
  if (!a->workspace) return COMPAMS_INVALID_ARG;
  if (!aligned_to(a->workspace, 256)) return COMPAMS_BAD_ALIGNMENT;
  if (a->workspace_bytes < counts_bytes(*a) + losses_bytes(*a)) return COMPAMS_WORKSPACE_TOO_SMALL;
  LossArgs k = {};
  k.n = static_cast<uint32_t>(a->n);
  k.rows = static_cast<uint32_t>(a->rows);
  k.vocab = static_cast<uint32_t>(a->vocab);
  k.total = k.n * k.rows;
  k.logits = a->logits; k.dlogits = a->dlogits;
  k.ld_logits = a->ld_logits; k.ld_dlogits = a->ld_dlogits;
  k.targets = a->targets;
  k.wide_targets = a->target_type == COMPAMS_I64;
  k.ignore = a->ignore_index;
  k.grad_scale = a->grad_scale;
  k.mean_loss = a->mean_loss;
  k.counts = static_cast<uint32_t*>(a->workspace);
  k.losses = a->losses ? a->losses
             : a->mean_loss ? reinterpret_cast<float*>(static_cast<char*>(a->workspace) + counts_bytes(*a)) : nullptr;
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  hipLaunchKernelGGL(k_loss_count, dim3(k.n), dim3(kLossThreads), 0, stream, k);
  if (k.total) {
    const dim3 grid(k.total < (1u << 21) ? k.total : (1u << 21));
    if (a->type == COMPAMS_F32) hipLaunchKernelGGL(k_loss_wide<float>, grid, dim3(kLossThreads), 0, stream, k);
    else if (a->type == COMPAMS_F16) hipLaunchKernelGGL(k_loss_wide<half_t>, grid, dim3(kLossThreads), 0, stream, k);
    else hipLaunchKernelGGL(k_loss_wide<bfloat_t>, grid, dim3(kLossThreads), 0, stream, k);
  }
  if (k.mean_loss) hipLaunchKernelGGL(k_loss_mean, dim3(k.n), dim3(kLossThreads), 0, stream, k);
  return hipGetLastError() == hipSuccess ? COMPAMS_OK : COMPAMS_HIP_ERROR;
}

}  // extern "C"
