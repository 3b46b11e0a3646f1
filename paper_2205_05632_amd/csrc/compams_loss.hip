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
  float lift;  // of the gradient's exponentials, see exp_below
  float *mean_loss, *losses;
  uint32_t* counts;  // per worker: rows that are learnt from; NULL where whoever asks counts them
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

// The rows of a worker that are learnt from, counted by the `lanes` lanes of a team (or of a wavefront of one), `AT_ONCE`
// loads under way in each.
template <uint32_t AT_ONCE, typename I>
__device__ __forceinline__ uint32_t count_targets(const I* targets, uint32_t rows, int64_t ignore, uint32_t lane,
                                                  uint32_t lanes) {
  uint32_t mine = 0;
  for (uint32_t first = lane; first < rows; first += lanes * AT_ONCE) {
    I t[AT_ONCE];
#pragma unroll
    for (uint32_t k = 0; k < AT_ONCE; ++k) {  // (beyond the last row: that one, left out below)
      const uint32_t i = first + k * lanes;
      t[k] = targets[i < rows ? i : rows - 1];
    }
#pragma unroll
    for (uint32_t k = 0; k < AT_ONCE; ++k) mine += first + k * lanes < rows && t[k] != ignore;
  }
  return mine;
}
template <uint32_t AT_ONCE>
__device__ __forceinline__ uint32_t count_rows(const LossArgs& a, uint32_t w, uint32_t lane, uint32_t lanes) {
  const size_t from = static_cast<size_t>(w) * a.rows;
  return a.wide_targets ? count_targets<AT_ONCE>(static_cast<const int64_t*>(a.targets) + from, a.rows, a.ignore, lane, lanes)
                        : count_targets<AT_ONCE>(static_cast<const int32_t*>(a.targets) + from, a.rows, a.ignore, lane, lanes);
}

__global__ __launch_bounds__(kLossThreads) void k_loss_count(LossArgs a) {
  __shared__ float slots[1][kSlots];
  for (uint32_t w = blockIdx.x; w < a.n; w += gridDim.x) {
    const uint32_t mine = count_rows<8>(a, w, threadIdx.x, kLossThreads);
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

// exp(v - top) = 2^((v - top) log2(e)) for v <= top.  (The difference first: with log2(e) top taken off in one multiply-add
// instead, 2 % faster at 8192 x 50257, tops from 1e9 on leave more of their rounding than an exponent holds.)
//
// Rows of 32 bits: the exponent as a whole number and a part in -1/2 .. 1/2, which is formed with the rounding of the product
// and of log2(e) put right, so that the result is off by three units of 2^-24 at any distance.  (Rounded once, an exponent of
// -60 is off by up to 2^-19: 22 such units of the result.)  Distances beyond 200 are taken as that: whatever they are, 0 is left.
// Rows of 16 bits: the product rounded once, three instructions for ten.  With the difference's rounding an entry is off by
// 2.3 (top - v) units of 2^-24, at a distance of 87, the largest that leaves a normal number, by 2^-16 of itself, where its
// gradient is rounded to 2^-9 or 2^-12; of their sum it is the mean distance by weight, log(vocab) at most.  Results below
// 2^-126 are 0.
//
// lift: the result is 2^lift times as large, so that no entry is lost that the gradient's scale makes a normal number again
// (grad_scale < 2^lift; for 16 bits two more units for each power of two, the largest entry stays exact).
constexpr float kLog2E = 1.44269504088896340736f;
constexpr float kShift = 0x1.8p23f;  // what is added to it is rounded to a whole number, which is in the low bits then
constexpr float kLog2ERest = static_cast<float>(1.44269504088896340736 - static_cast<double>(kLog2E));
template <typename T>
__device__ __forceinline__ float exp_below(float v, float top, float lift = 0.0f) {
  if constexpr (sizeof(T) < 4) {
    return __builtin_amdgcn_exp2f(fmaf(v - top, kLog2E, lift));
  } else {
    const float away = __builtin_elementwise_maximum(v - top, -200.0f);  // (a NaN stays one)
    const float shifted = fmaf(away, kLog2E, kShift + lift), whole = shifted - (kShift + lift);
    const float part = fmaf(away, kLog2ERest, fmaf(away, kLog2E, -whole));
    return __builtin_amdgcn_ldexpf(__builtin_amdgcn_exp2f(part), static_cast<int16_t>(__float_as_uint(shifted)));
  }
}

// (With float16 no number that a gradient can hold comes from an exponential below 2^-126.)
template <typename T>
__device__ __forceinline__ float lift_of(const LossArgs& a) {
  return __is_same(T, half_t) ? 0.0f : a.lift;
}

// ---- Rows that a team of lanes holds in registers ---------------------------------------------------------------
// A team is 16 to 64 lanes of a wavefront or a whole workgroup.  The row is read once and kept as it came, in
// groups of 16 bytes; its maximum, the sum of its exponentials and its gradient are three passes over registers.  (The
// exponentials of 16-bit rows are formed twice: kept in fp32 they would take two times the row's registers again, and what
// hides one row's reads and reductions is the other rows that fit a compute unit.  Those of fp32 rows take their logits'
// place.)  8192 x 50257 bfloat16: 312 us, of which reading, the barriers and writing alone take 298; 5.3 TB/s.
//
// The groups start at the row's first multiple of 16 bytes: rows of an odd vocabulary, one after another, start anywhere,
// and accesses across cache lines cost a sixth of the time.  What is left at the row's two ends, up to seven columns
// each, goes one by one to the first sixteen lanes.
template <typename T>
struct Logits {
  static constexpr uint32_t kEach = 16 / sizeof(T);
  typedef T type __attribute__((ext_vector_type(16 / sizeof(T))));
};

// A group is forgotten before every pass, so that it is unpacked again instead of kept in fp32 beside (with 16 groups of
// bfloat16 that spilled 178 registers).
template <typename V>
__device__ __forceinline__ void forget_group(V& raw) {
  typedef uint32_t Words __attribute__((ext_vector_type(4)));
  Words w;
  __builtin_memcpy(&w, &raw, 16);
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i) {
    uint32_t v = w[i];
    forget(v);
    w[i] = v;
  }
  __builtin_memcpy(&raw, &w, 16);
}

constexpr uint32_t kTeamThreads = 256, kRowThreads = 512;
constexpr uint64_t kStreamBytes = 32u << 20;

enum RowKind {
  kWaveRows = 0,   // a team of 16 to 64 lanes to a row, 256 threads to a workgroup
  kBlockRow = 1,   // a workgroup to a row
  kWorkerRows = 2  // a wavefront to a row, a workgroup to all rows of a worker, whose mean it forms as well
};

// (20 groups of fp32 are kept to the registers that leave room for a second row: 8 x 500 x 33000 202 us for 224, 207 with
// exponentials rounded as those of 16-bit rows are.)
template <typename T, uint32_t NG, RowKind KIND, bool STREAM>
__global__ __launch_bounds__(KIND == kWaveRows ? kTeamThreads : KIND == kBlockRow ? kRowThreads : kLossThreads,
                             NG == 20 && sizeof(T) == 4 ? 4 : 1)
void k_loss(LossArgs a, uint32_t lanes) {
  constexpr uint32_t kEach = Logits<T>::kEach;
  constexpr bool kKept = sizeof(T) == 4;
  const float lift = lift_of<T>(a);
  typedef typename Logits<T>::type V;
  __shared__ float tops[2][kLossWaves];
  __shared__ float slots[2][2][kSlots];
  constexpr bool WAVE = KIND != kBlockRow;
  const uint32_t lane = WAVE ? threadIdx.x & (lanes - 1) : threadIdx.x, team = WAVE ? threadIdx.x / lanes : 0u;
  const uint32_t together = KIND == kWaveRows ? kTeamThreads / lanes : KIND == kBlockRow ? 1u : kLossWaves, waves = lanes / 64;
  uint32_t turn = 0;
  float of_worker[2] = {0.0f, 0.0f};  // kWorkerRows: losses, and rows that are learnt from
  if constexpr (KIND == kWorkerRows) {
    float c[1] = {static_cast<float>(count_rows<1>(a, blockIdx.x, threadIdx.x, kLossThreads))};
    sum_block(c, slots[0], kLossWaves);
    of_worker[1] = c[0];
  }
  const uint32_t from = (KIND == kWorkerRows ? blockIdx.x * a.rows : blockIdx.x * together) + team;
  const uint32_t to = KIND == kWorkerRows ? blockIdx.x * a.rows + a.rows : a.total;
  for (uint32_t r = from; r < to; r += KIND == kWorkerRows ? together : gridDim.x * together) {
    const T* const logits = static_cast<const T*>(a.logits) + static_cast<int64_t>(r) * a.ld_logits;
    T* const out = a.dlogits ? static_cast<T*>(a.dlogits) + static_cast<int64_t>(r) * a.ld_dlogits : nullptr;
    const int64_t target = target_of(a, r);
    if (target == a.ignore) {  // nothing is read, whatever stands there
      if (a.losses && lane == 0) a.losses[r] = 0.0f;
      if (out)
        for (uint32_t c = lane * kGroup; c < a.vocab; c += lanes * kGroup) {
          const float zero[kGroup] = {};
          store_group(out, c, a.vocab, zero);
        }
      continue;
    }
    uint32_t head = static_cast<uint32_t>(-reinterpret_cast<uintptr_t>(logits) % 16 / sizeof(T));
    head = head < a.vocab ? head : a.vocab;
    const uint32_t groups = (a.vocab - head) / kEach, tail = head + groups * kEach;
    const char* const inner = reinterpret_cast<const char*>(logits + head);
    V raw[NG] = {};
    if (groups) {
#pragma unroll
      for (uint32_t k = 0; k < NG; ++k) {  // (lanes beyond the last group read that one, and leave it out below)
        const uint32_t g = k * lanes + lane;
        raw[k] = *reinterpret_cast<const V*>(inner + (g < groups ? g : groups - 1) * 16u);
      }
    }
    const uint32_t end = lane < 8 ? (lane < head ? lane : a.vocab) : lane < 16 ? tail + (lane - 8) : a.vocab;
    const float at_end = end < a.vocab ? to_float(logits[end]) : -INFINITY;
    const uint32_t w = r / a.rows;
    // (2^12 of them at most: exact in fp32; a.counts is there where there may be more)
    const float count = a.counts || KIND == kWorkerRows ? 0.0f : static_cast<float>(count_rows<4>(a, w, lane, lanes));
    const bool inside = target >= 0 && target < static_cast<int64_t>(a.vocab);
    float of_target = inside ? to_float(logits[target]) : 0.0f;
    float top = at_end;
    if (groups) {
#pragma unroll
      for (uint32_t k = 0; k < NG; ++k) {
#pragma unroll
        for (uint32_t j = 0; j < kEach; ++j) top = fmaxf(top, to_float(raw[k][j]));
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    top = over_lanes(top, WAVE ? lanes : 64u, Max());
    if (!WAVE && waves > 1) {
      if ((threadIdx.x & 63u) == 0) tops[turn][threadIdx.x >> 6] = top;
      __syncthreads();
      for (uint32_t i = 0; i < waves; ++i) top = fmaxf(top, tops[turn][i]);
    }
    uint32_t again = lane;
    const float in_sum = kKept ? lift : 0.0f;  // (kept for the gradient)
    forget(again);
    float s[2] = {exp_below<T>(at_end, top, in_sum), count};
#pragma unroll
    for (uint32_t k = 0; k < NG; ++k) {
      forget_group(raw[k]);
      float e[kEach];
#pragma unroll
      for (uint32_t j = 0; j < kEach; ++j) e[j] = exp_below<T>(to_float(raw[k][j]), top, in_sum);
      if constexpr (kKept) __builtin_memcpy(&raw[k], e, sizeof(raw[k]));
#pragma unroll
      for (uint32_t n = kEach / 2; n > 0; n /= 2)
#pragma unroll
        for (uint32_t j = 0; j < n; ++j) e[j] += e[j + n];
      s[0] += k * lanes + again < groups ? e[0] : 0.0f;
      __builtin_amdgcn_sched_barrier(0);
    }
    // The target's logit is here before the last barrier: behind it another wavefront may write the gradient over it.
    asm volatile("" : "+v"(of_target));
    if constexpr (WAVE) {
      s[0] = sum_lanes(s[0], lanes);
      s[1] = sum_lanes(s[1], lanes);
    } else {
      sum_block(s, slots[turn], waves);
    }
    turn ^= 1;
    if constexpr (kKept) s[0] = __builtin_amdgcn_ldexpf(s[0], -static_cast<int>(lift));
    const bool none = !inside || top == -INFINITY;
    // (the large numbers first: their difference is what the loss is made of, a sum of them would round it away)
    const float loss = none ? __builtin_nanf("") : (top - of_target) + logf(s[0]);
    of_worker[0] += loss;
    if (a.losses && lane == 0) a.losses[r] = loss;
    if (!out) continue;
    if (a.counts) s[1] = static_cast<float>(a.counts[w]);
    if (KIND == kWorkerRows) s[1] = of_worker[1];
    // a row without a softmax or a loss has no gradient
    const float factor = none ? __builtin_nanf("") : a.grad_scale / s[1];
    const float share = __builtin_amdgcn_ldexpf(factor / s[0], -static_cast<int>(lift));
    const bool aligned = reinterpret_cast<uintptr_t>(out) % 16 == reinterpret_cast<uintptr_t>(logits) % 16;
    const uint32_t hot = inside ? static_cast<uint32_t>(target) : a.vocab;
    char* const inner_out = reinterpret_cast<char*>(out + head);
    forget(again);
#pragma unroll
    for (uint32_t k = 0; k < NG; ++k) {
      const uint32_t g = k * lanes + again;
      forget_group(raw[k]);
      float v[kEach];
#pragma unroll
      for (uint32_t j = 0; j < kEach; ++j) {
        const float l = to_float(raw[k][j]);
        v[j] = (kKept ? l : exp_below<T>(l, top, lift)) * share;
      }
      const uint32_t at = hot - head - g * kEach;
      if (at < kEach) {
#pragma unroll
        for (uint32_t j = 0; j < kEach; ++j) v[j] -= at == j ? factor : 0.0f;
      }
      V o;
#pragma unroll
      for (uint32_t j = 0; j < kEach; ++j) o[j] = static_cast<T>(v[j]);
      if (g < groups) {
        if (!aligned) __builtin_memcpy(inner_out + g * 16u, &o, 16);
        else if (STREAM) __builtin_nontemporal_store(o, reinterpret_cast<V*>(inner_out + g * 16u));
        else *reinterpret_cast<V*>(inner_out + g * 16u) = o;
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    if (end < a.vocab) out[end] = static_cast<T>(exp_below<T>(at_end, top, lift) * share - (end == hot ? factor : 0.0f));
  }
  if constexpr (KIND == kWorkerRows) {
    // (the same in all lanes of a wavefront: one of them counts)
    if (lane == 0) slots[1][0][team] = of_worker[0];
    __syncthreads();
    if (threadIdx.x == 0 && a.mean_loss) {
      float sum = 0.0f;
      for (uint32_t i = 0; i < kLossWaves; ++i) sum += slots[1][0][i];
      a.mean_loss[blockIdx.x] = of_worker[1] > 0.0f ? sum / of_worker[1] : 0.0f;
    }
  }
}

// ---- Rows of any width: a workgroup goes over its row twice, once for a running maximum and sum, once for the gradient.
constexpr uint32_t kAhead = 4;  // groups that a lane requests at once

// One more value to a lane's maximum and sum.  What the sum counts from moves up rarely after the first few.
template <typename T>
struct Running {
  float top = -INFINITY, sum = 0.0f;
  __device__ __forceinline__ void raise(float m) {
    if (!(m > top)) return;
    sum = top == -INFINITY ? sum : sum * exp_below<T>(top, m);  // (without a finite entry so far it is 0 or NaN)
    top = m;
  }
  __device__ __forceinline__ void add(float v) { sum += top == -INFINITY ? (v != v ? v : 0.0f) : exp_below<T>(v, top); }
};

template <typename T, bool STREAM>
__global__ __launch_bounds__(kLossThreads) void k_loss_wide(LossArgs a) {
  constexpr uint32_t kEach = Logits<T>::kEach;
  typedef typename Logits<T>::type V;
  __shared__ float tops[kLossWaves], sums[kLossWaves];
  const float lift = lift_of<T>(a);
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
    const float of_target = inside ? to_float(row[target]) : 0.0f;
    // groups from the row's first multiple of 16 bytes, and its two ends, as above
    uint32_t head = static_cast<uint32_t>(-reinterpret_cast<uintptr_t>(row) % 16 / sizeof(T));
    head = head < a.vocab ? head : a.vocab;
    const uint32_t groups = (a.vocab - head) / kEach, tail = head + groups * kEach, lane = threadIdx.x;
    const uint32_t end = lane < 8 ? (lane < head ? lane : a.vocab) : lane < 16 ? tail + (lane - 8) : a.vocab;
    const float at_end = end < a.vocab ? to_float(row[end]) : -INFINITY;
    const V* const inner = reinterpret_cast<const V*>(row + head);
    Running<T> run;
    if (end < a.vocab) {
      run.raise(at_end);
      run.add(at_end);
    }
    for (uint32_t first = lane; first < groups; first += kLossThreads * kAhead) {
      V raw[kAhead];
#pragma unroll
      for (uint32_t k = 0; k < kAhead; ++k) {  // (beyond the last group: that one, left out below)
        const uint32_t g = first + k * kLossThreads;
        raw[k] = inner[g < groups ? g : groups - 1];
      }
      float m = -INFINITY;
#pragma unroll
      for (uint32_t k = 0; k < kAhead; ++k)
#pragma unroll
        for (uint32_t j = 0; j < kEach; ++j) m = fmaxf(m, to_float(raw[k][j]));
      run.raise(m);
#pragma unroll
      for (uint32_t k = 0; k < kAhead; ++k) {
        if (first + k * kLossThreads >= groups) break;
#pragma unroll
        for (uint32_t j = 0; j < kEach; ++j) run.add(to_float(raw[k][j]));
      }
    }
    const float wave_top = over_lanes(run.top, 64, Max());
    __syncthreads();  // the slots may still be read for the row before
    if (lane % 64 == 0) tops[lane / 64] = wave_top;
    __syncthreads();
    float top = tops[0];
    for (uint32_t w = 1; w < kLossWaves; ++w) top = fmaxf(top, tops[w]);
    const float mine = sum_lanes(run.top == -INFINITY ? run.sum : run.sum * exp_below<T>(run.top, top), 64);
    if (lane % 64 == 0) sums[lane / 64] = mine;
    __syncthreads();
    float sum = 0.0f;
    for (uint32_t w = 0; w < kLossWaves; ++w) sum += sums[w];
    const bool none = !inside || top == -INFINITY;
    if (a.losses && lane == 0) a.losses[r] = none ? __builtin_nanf("") : (top - of_target) + logf(sum);
    if (!out) continue;
    const float factor = none ? __builtin_nanf("") : a.grad_scale / static_cast<float>(a.counts[r / a.rows]);
    const float share = __builtin_amdgcn_ldexpf(factor / sum, -static_cast<int>(lift));
    const bool aligned = reinterpret_cast<uintptr_t>(out) % 16 == reinterpret_cast<uintptr_t>(row) % 16;
    const uint32_t hot = inside ? static_cast<uint32_t>(target) : a.vocab;
    char* const inner_out = reinterpret_cast<char*>(out + head);
    for (uint32_t first = lane; first < groups; first += kLossThreads * kAhead) {
      V raw[kAhead];
#pragma unroll
      for (uint32_t k = 0; k < kAhead; ++k) {
        const uint32_t g = first + k * kLossThreads;
        raw[k] = inner[g < groups ? g : groups - 1];
      }
#pragma unroll
      for (uint32_t k = 0; k < kAhead; ++k) {
        const uint32_t g = first + k * kLossThreads, at = hot - head - g * kEach;
        if (g >= groups) break;
        V o;
#pragma unroll
        for (uint32_t j = 0; j < kEach; ++j)
          o[j] = static_cast<T>(exp_below<T>(to_float(raw[k][j]), top, lift) * share - (at == j ? factor : 0.0f));
        char* const p = inner_out + static_cast<size_t>(g) * 16;
        if (!aligned) __builtin_memcpy(p, &o, 16);
        else if (STREAM) __builtin_nontemporal_store(o, reinterpret_cast<V*>(p));
        else *reinterpret_cast<V*>(p) = o;
      }
    }
    if (end < a.vocab) out[end] = static_cast<T>(exp_below<T>(at_end, top, lift) * share - (end == hot ? factor : 0.0f));
  }
}

// A worker's losses added up and divided by their count.
__global__ __launch_bounds__(kLossThreads) void k_loss_mean(LossArgs a) {
  __shared__ float slots[2][2][kSlots];
  uint32_t turn = 0;
  for (uint32_t w = blockIdx.x; w < a.n; w += gridDim.x, turn ^= 1) {
    float s[2] = {0.0f, a.counts ? 0.0f : static_cast<float>(count_rows<8>(a, w, threadIdx.x, kLossThreads))};
    const float* const losses = a.losses + static_cast<size_t>(w) * a.rows;
    for (uint32_t first = threadIdx.x; first < a.rows; first += kLossThreads * 8) {
      float l[8];
#pragma unroll
      for (uint32_t k = 0; k < 8; ++k) {  // (eight loads under way in each lane)
        const uint32_t i = first + k * kLossThreads;
        l[k] = losses[i < a.rows ? i : a.rows - 1];
      }
#pragma unroll
      for (uint32_t k = 0; k < 8; ++k) s[0] += first + k * kLossThreads < a.rows ? l[k] : 0.0f;
    }
    sum_block(s, slots[turn], kLossWaves);
    if (a.counts) s[1] = static_cast<float>(a.counts[w]);
    if (threadIdx.x == 0) a.mean_loss[w] = s[1] > 0.0f ? s[0] / s[1] : 0.0f;
  }
}

// The team and the number of groups per lane that a row of `groups` groups is given (0 groups per lane: none).  A workgroup
// of at most 512 threads leaves room for two rows and more on a compute unit, so that one row's reads are under way while
// another's exponentials are formed: 8192 rows of bfloat16, us by threads x groups:
//   vocabulary  4096: 256 x 2 32.5, 128 x 4 30.3, 64 x 8 31.9      8192: 256 x 4 56.8, 128 x 8 58.3, 64 x 16 58.8
//              16384: 1024 x 2 152, 512 x 4 97, 256 x 8 101, 128 x 16 110      32000: 512 x 8 182, 256 x 16 193
//              50257: 832 x 8 400, 448 x 16 312, 256 x 32 311, 320 x 20 467 (waves that do not go evenly into four)
// 8 x 6284 rows of 2268 float16: 64 x 5 91.0, 128 x 3 111, 192 x 2 135; 8 x 3000 rows of 5000 bfloat16: 128 x 5 89.8, 192 x 4
// 93.9; of 10000: 256 x 5 170, 320 x 4 191
// and 2048 rows of  40000: 448 x 12 66.9, 320 x 16 77.6; 1078 rows of 67875: 448 x 20 89, 320 x 32 114; of 80387: 512 x 20 96,
// 320 x 32 120; of 98000: 512 x 24 113, 384 x 32 130; of 33000 fp32: 448 x 20 68.9, 320 x 32 78.4.
struct Team {
  RowKind kind;
  uint32_t lanes, each;
};
Team loss_team(uint32_t rows, uint32_t groups) {
  // A few short rows of each worker: the launch that would form the means costs more than going over them one after another
  // (8 x 32 x 1000 fp32: 10.5 us a call, with a launch more 12.5; on the device 8.2 and 4.0 + 2.8 and a gap).  However many
  // workers there are, so that a worker's losses are the same bits beside any others (300 x 32 x 1000 fp32 16.6 and 16.9, 1000 x
  // 4 x 40 11.1 and 13.1, 3000 x 32 x 256 bfloat16 47.5 and 35.2).
  if (rows <= 2 * kLossWaves && groups <= 256) return {kWorkerRows, 64, groups <= 64 ? 1u : groups <= 128 ? 2u : 4u};
  // Short rows: few lanes with up to four groups, so that what a row costs besides its columns (its reductions, logarithm and
  // quotients) is shared by the rows of a wavefront.  (16 x 9882 rows of float16, us on the device and the two small launches:
  // 133 columns 32 x 1 52.3, 16 x 2 43.6, 16 x 4 55.4; 260 columns 64 x 1 92.5, 32 x 2 75.3, 16 x 4 63.0, 16 x 8 90.0;
  // 512 columns 64 x 1 99.7, 32 x 2 85.3, 16 x 4 73.3; 8 x 9882 x 1000: 64 x 2 81.8, 32 x 4 73.7, 16 x 8 86.0.)
  if (groups <= 256) {
    uint32_t lanes = 16;  // (as many as the two ends may have columns)
    while (lanes * 4 < groups) lanes *= 2;
    return {kWaveRows, lanes, groups <= lanes ? 1 : (groups + lanes - 1) / lanes};
  }
  if (groups <= 384) return {kWaveRows, 64, (groups + 63) / 64};
  if (groups > 512 && groups <= 640) return {kBlockRow, 128, 5};
  if (groups > 1024 && groups <= 1280) return {kBlockRow, 256, 5};
  uint32_t each = 0;
  for (const uint32_t k : {4u, 8u, 12u, 16u, 20u, 24u, 32u})
    if (each == 0 && groups <= k * kRowThreads) each = k;
  return {kBlockRow, each ? (groups + 64 * each - 1) / (64 * each) * 64 : 0, each};
}

// STREAM: the gradient is written past the memory-side cache.  (A template parameter: between two stores that differ in
// nothing else the compiler drops the hint.)
template <typename T, bool STREAM>
void launch_loss(const Team& t, const LossArgs& k, hipStream_t stream) {
  constexpr uint64_t kMost = 1u << 21;  // workgroups: a dimension has room for 2^32 threads in all
  const uint64_t together = t.kind == kWaveRows ? kTeamThreads / t.lanes : 1;
  const uint64_t wanted = t.kind == kWorkerRows ? k.n : (k.total + together - 1) / together;
  const dim3 grid(static_cast<uint32_t>(wanted < kMost ? wanted : kMost));
  const dim3 block(t.kind == kWaveRows ? kTeamThreads : t.kind == kWorkerRows ? kLossThreads : t.lanes);
#define COMPAMS_LOSS(NG, KIND) hipLaunchKernelGGL((k_loss<T, NG, KIND, STREAM>), grid, block, 0, stream, k, t.lanes)
  if (t.kind == kWorkerRows) {
    if (t.each == 1) COMPAMS_LOSS(1, kWorkerRows);
    else if (t.each == 2) COMPAMS_LOSS(2, kWorkerRows);
    else COMPAMS_LOSS(4, kWorkerRows);
  } else if (t.kind == kWaveRows) {
    if (t.each == 1) COMPAMS_LOSS(1, kWaveRows);
    else if (t.each == 2) COMPAMS_LOSS(2, kWaveRows);
    else if (t.each == 3) COMPAMS_LOSS(3, kWaveRows);
    else if (t.each == 4) COMPAMS_LOSS(4, kWaveRows);
    else if (t.each == 5) COMPAMS_LOSS(5, kWaveRows);
    else COMPAMS_LOSS(6, kWaveRows);
  } else {
    switch (t.each) {
      case 0: hipLaunchKernelGGL((k_loss_wide<T, STREAM>), grid, dim3(kLossThreads), 0, stream, k); break;
      case 4: COMPAMS_LOSS(4, kBlockRow); break;
      case 5: COMPAMS_LOSS(5, kBlockRow); break;
      case 8: COMPAMS_LOSS(8, kBlockRow); break;
      case 12: COMPAMS_LOSS(12, kBlockRow); break;
      case 16: COMPAMS_LOSS(16, kBlockRow); break;
      case 20: COMPAMS_LOSS(20, kBlockRow); break;
      case 24: COMPAMS_LOSS(24, kBlockRow); break;
      default: COMPAMS_LOSS(32, kBlockRow); break;
    }
  }
#undef COMPAMS_LOSS
}

// Whether every row's team counts its worker's targets by itself: where they are few for a row, or few beside its logits, and
// few in all, for a launch that counts them costs 2 to 3 us and then reads each only once (us a call with it / without, targets
// of 64 bits; float16 and bfloat16: 8 x 105 x 83 16.5 / 14.2, 16 x 512 x 1000 16.7 / 15.5, 16 x 1024 x 1000 22.3 / 25.3,
// 1 x 2000 x 50257 80.3 / 78.6, 4 x 1500 x 20000 93.2 / 95.2, 1 x 4000 x 50257 158 / 168, 1 x 8000 x 50257 297 / 323; fp32:
// 8 x 1024 x 8192 94.7 / 91.8, 8 x 1024 x 32000 350 / 344, 1 x 4000 x 50257 348 / 363).  (They are counted in fp32, exactly.)
bool counts_inside(const LossArgs& k, const Team& t) {
  if (t.kind == kWorkerRows) return true;  // (the workgroup that has all of a worker's rows)
  const uint64_t in_all = static_cast<uint64_t>(k.total) * k.rows;
  return t.each != 0 && ((k.rows <= 512 && in_all <= 1u << 22) || (k.rows <= k.vocab / 4 && in_all <= 1u << 23));
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
  // |factor| <= |grad_scale| < 2^lift.  (At most 96: the sum of an fp32 row is formed so too, with 2^31 entries.)
  const float size = fabsf(k.grad_scale);
  k.lift = size > 1.0f ? fminf(static_cast<float>(ilogbf(fminf(size, 0x1p96f)) + 1), 96.0f) : 0.0f;
  k.mean_loss = a->mean_loss;
  k.losses = a->losses ? a->losses
             : a->mean_loss ? reinterpret_cast<float*>(static_cast<char*>(a->workspace) + counts_bytes(*a)) : nullptr;
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const uint32_t each = 16 / static_cast<uint32_t>(type_size(a->type));
  const Team team = loss_team(k.rows, (k.vocab + each - 1) / each);
  if (!counts_inside(k, team)) {
    k.counts = static_cast<uint32_t*>(a->workspace);
    hipLaunchKernelGGL(k_loss_count, dim3(k.n), dim3(kLossThreads), 0, stream, k);
  }
  if (k.total) {
    // What does not stay in the memory-side cache until it is read again need not pass through it (8192 rows of bfloat16,
    // streamed / not: vocabulary 4096 29.5 / 35.8 us, 16384 98.3 / 102, 32000 182 / 189, 50257 312 / 317).
    const bool stream_out = static_cast<uint64_t>(k.total) * k.vocab * type_size(a->type) > kStreamBytes;
    const auto launch = [&](auto t) {
      if (stream_out) launch_loss<decltype(t), true>(team, k, stream);
      else launch_loss<decltype(t), false>(team, k, stream);
    };
    if (a->type == COMPAMS_F32) launch(float());
    else if (a->type == COMPAMS_F16) launch(half_t());
    else launch(bfloat_t());
  }
  if (k.mean_loss && (team.kind != kWorkerRows || k.total == 0))
    hipLaunchKernelGGL(k_loss_mean, dim3(k.n), dim3(kLossThreads), 0, stream, k);
  return hipGetLastError() == hipSuccess ? COMPAMS_OK : COMPAMS_HIP_ERROR;
}

}  // extern "C"
