// A gated feed-forward block up to its product, m = act(x Wg' + bg) * (x Wu' + bu), and the gradients of its two projections.
#include "compams_tiles.h"

#include <utility>

namespace compams {
namespace {

// ---- Activations ---------------------------------------------------------------------------------------------
// The processor's 2^x and 1 / x, a unit each; after the product with log2 e, rounded once, e^z is off by 1.2 |z| units.
__device__ __forceinline__ float exp_fast(float z) { return __expf(z); }
__device__ __forceinline__ float logistic(float a) { return __builtin_amdgcn_rcpf(1.0f + exp_fast(-a)); }

// The normal distribution's integral up to a, with e = exp(-a^2 / 2), which the density needs too: for z = |a| / sqrt 2,
// erfc(z) = e p(t) / (1 + 2 z) with a polynomial in t = (z - 2) / (z + 2) (the form of Shepherd and Laframboise, "Chebyshev
// approximation of (1 + 2 x) exp(x^2) erfc x", 1981; the coefficients by interpolation at the Chebyshev points of 0 <= z <= 10.2, as
// fp32 off by 3.6e-8 at most, 3.1e-8 of the value).  Negative a keep their digits.  (8290 x 576 float16 backward: 51 us with the
// library's erfcf.)
__device__ __forceinline__ float normal_cdf(float a, float e) {
  const float z = fminf(fabsf(a) * 0.70710678118654752f, 16.0f), up = z + 2.0f, one = fmaf(2.0f, z, 1.0f);
  const float r = __builtin_amdgcn_rcpf(up * one), t = (z - 2.0f) * (r * one);
  float p = -0.00042251546983607113f;
  p = fmaf(p, t, -0.0012606343952938914f);
  p = fmaf(p, t, 0.0013287677429616451f);
  p = fmaf(p, t, 0.008661998435854912f);
  p = fmaf(p, t, -0.008062068372964859f);
  p = fmaf(p, t, -0.05421387776732445f);
  p = fmaf(p, t, 0.16405519843101501f);
  p = fmaf(p, t, -0.16603043675422668f);
  p = fmaf(p, t, -0.09276396036148071f);
  p = fmaf(p, t, 1.2769783735275269f);
  const float tail = 0.5f * e * (p * (r * up));
  return a > 0.0f ? 1.0f - tail : tail;
}

// act(a), and its derivative where SLOPE, for results of 16 bits.
template <int ACT, bool SLOPE>
__device__ __forceinline__ float activate_fast(float a, float& slope) {
  if constexpr (ACT == COMPAMS_RELU) {
    if constexpr (SLOPE) slope = a > 0.0f ? 1.0f : a != a ? a : 0.0f;
    return a > 0.0f || a != a ? a : 0.0f;
  } else if constexpr (ACT == COMPAMS_SIGMOID) {
    const float q = logistic(a);
    if constexpr (SLOPE) slope = q * logistic(-a);  // (1 - q would lose its digits for large a)
    return q;
  } else if constexpr (ACT == COMPAMS_SILU) {
    const float q = logistic(a), v = a < -88.0f ? -0.0f : a * q;  // (beyond it q is 0)
    if constexpr (SLOPE) slope = a > 88.0f ? q : q + v * logistic(-a);  // (infinity times 0 beyond it)
    return v;
  } else if constexpr (ACT == COMPAMS_GELU) {
    const float e = exp_fast(-0.5f * a * a), cdf = normal_cdf(a, e);
    if constexpr (SLOPE) slope = a * a > 400.0f ? cdf : cdf + a * e * 0.3989422804014327f;
    return a < -14.0f ? -0.0f : a * cdf;
  } else {
    // (1 + tanh u) / 2 = logistic(2 u)
    const float a2 = a * a, u2 = 1.5957691216057308f * a * (1.0f + 0.044715f * a2);
    const float q = logistic(u2);
    if constexpr (SLOPE) {
      const float inner = 1.5957691216057308f * (1.0f + 3.0f * 0.044715f * a2);
      slope = a2 > 400.0f ? q : q + a * q * logistic(-u2) * inner;
    }
    return a < -14.0f ? -0.0f : a * q;
  }
}

// The same for fp32 results, which keep their digits at any a (rounded once, an exponential's argument z costs it |z| units): one
// exponential E = e^-|z|, of which logistic(z) and logistic(-z) are 1 / (1 + E) and E / (1 + E), and what the roundings of z leave
// over.  (2048 x 8192 backward, bound by memory: gelu 73.5 us, tanh's 75.2, silu 70.8; with a unit for every one of z 72.9, 70.6,
// 71.6.  8192 x 768 x 2048 forward: 2 to 3 % more.)
struct Both {
  float of, of_minus;  // logistic(z), logistic(-z)
};
__device__ __forceinline__ Both logistics(float z, float rest = 0.0f) {
  const float e = fabsf(z) > 87.33f ? 0.0f : exp_kept(-fabsf(z));  // (below 2^-126 it counts as 0)
  const float more = fmaf(e, z > 0.0f ? -rest : rest, e), y = 1.0f + more;
  const float r = __builtin_amdgcn_rcpf(y), big = fmaf(fmaf(-y, r, 1.0f), r, r), small = more * big;
  return z > 0.0f ? Both{big, small} : Both{small, big};
}
template <int ACT, bool SLOPE>
__device__ __forceinline__ float activate_kept(float a, float& slope) {
  if constexpr (ACT == COMPAMS_RELU) {
    return activate_fast<ACT, SLOPE>(a, slope);
  } else if constexpr (ACT == COMPAMS_SIGMOID) {
    const Both q = logistics(a);
    if constexpr (SLOPE) slope = q.of * q.of_minus;
    return q.of;
  } else if constexpr (ACT == COMPAMS_SILU) {
    const Both q = logistics(a);
    const float v = a < -200.0f ? -0.0f : a * q.of;  // (infinity times 0 beyond these)
    if constexpr (SLOPE) slope = a > 200.0f ? q.of : fmaf(v, q.of_minus, q.of);
    return v;
  } else {
    const float at = __builtin_elementwise_minimum(__builtin_elementwise_maximum(a, -20.0f), 20.0f);  // (a NaN stays one)
    const float a2 = at * at, rest2 = fmaf(at, at, -a2);  // their sum is the square
    float q, density;                                     // slope: q + a density
    if constexpr (ACT == COMPAMS_GELU) {
      float e = exp_kept(-0.5f * a2);
      e = fmaf(e, -0.5f * rest2, e);
      q = normal_cdf(at, e);
      density = e * 0.3989422804014327f;
    } else {
      // u2 = c (1 + k a^2) a, each product with what its rounding left over
      constexpr double kC = 1.5957691216057307118, kK = 0.044715;
      constexpr float c = static_cast<float>(kC), c_rest = static_cast<float>(kC - static_cast<double>(c));
      constexpr float k = static_cast<float>(kK), k_rest = static_cast<float>(kK - static_cast<double>(k));
      const float in = fmaf(k, a2, 1.0f), in_rest = fmaf(k, a2, 1.0f - in) + fmaf(k, rest2, k_rest * a2);
      const float ca = c * at, ca_rest = fmaf(c, at, -ca) + c_rest * at;
      const float u2 = ca * in, u2_rest = fmaf(ca, in, -u2) + fmaf(ca, in_rest, ca_rest * in);
      const Both both = logistics(u2, u2_rest);
      q = both.of;
      density = both.of * both.of_minus * c * fmaf(3.0f * k, a2, 1.0f);
    }
    if constexpr (SLOPE) slope = fmaf(at, density, q);
    return a < -14.0f ? -0.0f : a * q;
  }
}
template <int ACT, bool SLOPE, typename T>
__device__ __forceinline__ float activate(float a, float& slope) {
  if constexpr (sizeof(T) == 4) return activate_kept<ACT, SLOPE>(a, slope);
  else return activate_fast<ACT, SLOPE>(a, slope);
}

// ---- Forward -------------------------------------------------------------------------------------------------
struct ForwardArgs {
  Read x, gate_weight, up_weight;
  const float *gate_bias, *up_bias;
  void *m, *gate, *up;
  int64_t ld_m, ld_gate, ld_up;
  uint32_t total, cols, hidden, tall, wide;
};

// A tile of 256 x 256 is 256 rows of x and 128 columns of each projection, which take turns of sixteen: what belongs together
// is in one lane's registers.  Bound by the matrix cores and, with K = 768, by the tile's three outputs.
template <typename TL, int ACT>
__global__ __launch_bounds__(TL::kThreads) void k_gated_forward(ForwardArgs a) {
  using T = typename TL::T;
  COMPAMS_TILE_LDS(TL, lds);
  const uint32_t tiles = a.tall * a.wide, id = tile_id();
  if (id >= tiles) return;
  uint32_t down, across;
  tile_at(by_die(id, tiles), a.tall, a.wide, down, across);
  const uint32_t m0 = down * TL::kM, h0 = across * (TL::kN / 2);
  TL t;
  t.clear();
  t.run([&](uint32_t, Side& x, Side& g, Side& u) {
    x = side<T, kAlong>(a.x.p, a.x.ld, a.total, m0, a.cols);
    g = side<T, kAlong>(a.gate_weight.p, a.gate_weight.ld, a.hidden, h0, a.cols);
    u = side<T, kAlong>(a.up_weight.p, a.up_weight.ld, a.hidden, h0, a.cols);
  }, 1, a.cols, lds);
  // The biases, then the product in the place of the first projection's sums.
  const uint32_t h1 = h0 + TL::first_n() / 2;
#pragma unroll
  for (uint32_t j = 0; j < TL::FN; j += 2) {
    const uint32_t h = h1 + TL::lane_n() + j * 8;
    f32x4 bg = {}, bu = {};
#pragma unroll
    for (uint32_t q = 0; q < 4; ++q) {
      if (a.gate_bias && h + q < a.hidden) bg[q] = a.gate_bias[h + q];
      if (a.up_bias && h + q < a.hidden) bu[q] = a.up_bias[h + q];
    }
#pragma unroll
    for (uint32_t i = 0; i < TL::FM; ++i) {
      t.sum[i][j] += bg;
      t.sum[i][j + 1] += bu;
    }
  }
  constexpr uint32_t kPieces = TL::FN * 2;
  __syncthreads();  // (others may still read what they multiply)
  const auto store = [&](void* to, int64_t ld, auto of) {
    t.template rows_of<kPieces>(lds.a[0], of, [&](uint32_t m, uint32_t c, const f32x4& v) {
      const uint32_t r = m0 + m, h = h1 + c;
      if (r < a.total) store4(static_cast<T*>(to) + static_cast<int64_t>(r) * ld + h, v, static_cast<int64_t>(a.hidden) - h);
    });
  };
  if (a.gate) store(a.gate, a.ld_gate, [&](uint32_t i, uint32_t j) { return t.sum[i][2 * j]; });
  if (a.up) store(a.up, a.ld_up, [&](uint32_t i, uint32_t j) { return t.sum[i][2 * j + 1]; });
  store(a.m, a.ld_m, [&](uint32_t i, uint32_t j) {
    f32x4 m;
    float none;
#pragma unroll
    for (uint32_t q = 0; q < 4; ++q) m[q] = activate<ACT, false, T>(t.sum[i][2 * j][q], none) * t.sum[i][2 * j + 1][q];
    return m;
  });
}

template <typename T, uint32_t WM, uint32_t WN, uint32_t FM, uint32_t FN>
void launch_forward(ForwardArgs& a, int act, hipStream_t stream) {
  using TL = Tiles<T, kAlong, kAlong, WM, WN, FM, FN, true>;
  a.tall = static_cast<uint32_t>(tiles_of(a.total, TL::kM));
  a.wide = static_cast<uint32_t>(tiles_of(a.hidden, TL::kN / 2));
  const dim3 grid = tile_grid(static_cast<uint64_t>(a.tall) * a.wide), block(TL::kThreads);
  switch (act) {
    case COMPAMS_SILU: hipLaunchKernelGGL((k_gated_forward<TL, COMPAMS_SILU>), grid, block, 0, stream, a); break;
    case COMPAMS_GELU: hipLaunchKernelGGL((k_gated_forward<TL, COMPAMS_GELU>), grid, block, 0, stream, a); break;
    case COMPAMS_GELU_TANH: hipLaunchKernelGGL((k_gated_forward<TL, COMPAMS_GELU_TANH>), grid, block, 0, stream, a); break;
    case COMPAMS_RELU: hipLaunchKernelGGL((k_gated_forward<TL, COMPAMS_RELU>), grid, block, 0, stream, a); break;
    default: hipLaunchKernelGGL((k_gated_forward<TL, COMPAMS_SIGMOID>), grid, block, 0, stream, a); break;
  }
}
// Few rows: the weights are read once and there is little to do with them.  A workgroup takes sixteen columns of both
// projections, its wavefronts 128 bytes of k in turn, straight from memory into registers (no row has to be aligned), and
// their sums are joined in LDS.  A lane's two pieces of 16 bytes lie side by side, so that a read's neighbours fill whole
// lines: k may be taken in any order that is the same for both operands.  Bound by memory (16 x 4096 x 8192 bfloat16, 134 MB:
// 64 x 64 tiles 50 us).
template <typename T>
__device__ __forceinline__ typename Fragment<T>::type load_piece(const char* row, uint32_t at, uint32_t cols) {
  constexpr uint32_t kEach = 16 / sizeof(T);
  typename Fragment<T>::type v = {};
  if (at + kEach <= cols) {
    __builtin_memcpy(&v, row + at * sizeof(T), sizeof(v));
  } else {
#pragma unroll
    for (uint32_t j = 0; j < kEach; ++j)
      if (at + j < cols) v[j] = reinterpret_cast<const T*>(row)[at + j];
  }
  return v;
}
// Up to 32 rows, and up to 64 where every workgroup has a compute unit of its own.  (us, this and tiles: 32 rows of bfloat16,
// 4096 x 4096 17.1 and 29.5, 2048 x 8192 17.2 and 17.1; 64 rows 26.6 and 29.6, 27.2 and 17.2, 768 x 2048 9.1 and 8.0, 4096 x 1024
// 25.6 and 19.3; fp32 64 rows 50 and 84, 79 and 44, 15.3 and 18.4, 48 and 83.)
inline bool few_rows(int64_t total, int64_t hidden) { return total <= 32 || (total <= 64 && hidden <= 16 * 256); }

template <typename T, int ACT, uint32_t FM, uint32_t WAVES>
__global__ __launch_bounds__(WAVES * 64) void k_gated_few(ForwardArgs a) {
  constexpr uint32_t kEach = 16 / sizeof(T), kDeep = 8 * kEach;  // k of a step
  constexpr uint32_t kAhead = 2;                                 // steps whose loads are under way at once
  __shared__ f32x4 joined[WAVES][2 * FM][64];
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63u, l = lane & 15u, g = lane >> 4;
  const uint32_t h0 = blockIdx.x * 16, h = min(h0 + l, a.hidden - 1);
  const char* const of_gate = static_cast<const char*>(a.gate_weight.p) + h * a.gate_weight.ld;
  const char* const of_up = static_cast<const char*>(a.up_weight.p) + h * a.up_weight.ld;
  const char* of_x[FM];
#pragma unroll
  for (uint32_t i = 0; i < FM; ++i) of_x[i] = static_cast<const char*>(a.x.p) + min(i * 16 + l, a.total - 1) * a.x.ld;
  f32x4 sum[2 * FM];
#pragma unroll
  for (uint32_t i = 0; i < 2 * FM; ++i) sum[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  typedef typename Fragment<T>::type Piece;
  const auto take = [&](uint32_t s, Piece (&gate)[2], Piece (&up)[2], Piece (&x)[FM][2], bool whole) {
#pragma unroll
    for (uint32_t q = 0; q < 2; ++q) {
      const uint32_t at = s * kDeep + (2 * g + q) * kEach, cols = whole ? ~0u : a.cols;
      gate[q] = load_piece<T>(of_gate, at, cols);
      up[q] = load_piece<T>(of_up, at, cols);
#pragma unroll
      for (uint32_t i = 0; i < FM; ++i) x[i][q] = load_piece<T>(of_x[i], at, cols);
    }
  };
  const auto add = [&](const Piece (&gate)[2], const Piece (&up)[2], const Piece (&x)[FM][2]) {
#pragma unroll
    for (uint32_t q = 0; q < 2; ++q)
#pragma unroll
      for (uint32_t i = 0; i < FM; ++i) {
        multiply(sum[2 * i], x[i][q], gate[q]);
        multiply(sum[2 * i + 1], x[i][q], up[q]);
      }
  };
  const uint32_t full = a.cols / kDeep;
  uint32_t s = wave;
  for (; s + (kAhead - 1) * WAVES < full; s += kAhead * WAVES) {
    Piece gate[kAhead][2], up[kAhead][2], x[kAhead][FM][2];
#pragma unroll
    for (uint32_t u = 0; u < kAhead; ++u) take(s + u * WAVES, gate[u], up[u], x[u], true);
    __builtin_amdgcn_sched_barrier(0);  // (all on their way before the first is waited for)
#pragma unroll
    for (uint32_t u = 0; u < kAhead; ++u) add(gate[u], up[u], x[u]);
  }
  for (; s <= full; s += WAVES) {  // (the last step may be a part of one, or nothing)
    Piece gate[2], up[2], x[FM][2];
    take(s, gate, up, x, false);
    add(gate, up, x);
  }
#pragma unroll
  for (uint32_t i = 0; i < 2 * FM; ++i) joined[wave][i][lane] = sum[i];
  __syncthreads();
  for (uint32_t e = threadIdx.x; e < FM * 256; e += WAVES * 64) {
    // entry (m, c) of a tile is number c % 4 of lane m + 16 (c / 4)
    const uint32_t i = e / 256, m = e / 16 % 16, c = e % 16, r = i * 16 + m, to = h0 + c;
    if (r >= a.total || to >= a.hidden) continue;
    float ga = a.gate_bias ? a.gate_bias[to] : 0.0f, ub = a.up_bias ? a.up_bias[to] : 0.0f;
    float sg = 0.0f, su = 0.0f;
#pragma unroll
    for (uint32_t k = 0; k < WAVES; ++k) {
      sg += joined[k][2 * i][m + 16 * (c / 4)][c % 4];
      su += joined[k][2 * i + 1][m + 16 * (c / 4)][c % 4];
    }
    ga += sg;
    ub += su;
    float none;
    if (a.gate) static_cast<T*>(a.gate)[r * a.ld_gate + to] = static_cast<T>(ga);
    if (a.up) static_cast<T*>(a.up)[r * a.ld_up + to] = static_cast<T>(ub);
    static_cast<T*>(a.m)[r * a.ld_m + to] = static_cast<T>(activate<ACT, false, T>(ga, none) * ub);
  }
}

template <typename T, int ACT>
void launch_few(const ForwardArgs& a, hipStream_t stream) {
  const dim3 grid((a.hidden + 15) / 16);
  // (eight wavefronts where each has two steps or more)
  const bool many = a.cols * sizeof(T) >= 16 * 128;
  if (a.total <= 16 && many) hipLaunchKernelGGL((k_gated_few<T, ACT, 1, 8>), grid, dim3(512), 0, stream, a);
  else if (a.total <= 16) hipLaunchKernelGGL((k_gated_few<T, ACT, 1, 4>), grid, dim3(256), 0, stream, a);
  else if (a.total > 32) hipLaunchKernelGGL((k_gated_few<T, ACT, 4, 4>), grid, dim3(256), 0, stream, a);
  else if (many) hipLaunchKernelGGL((k_gated_few<T, ACT, 2, 8>), grid, dim3(512), 0, stream, a);
  else hipLaunchKernelGGL((k_gated_few<T, ACT, 2, 4>), grid, dim3(256), 0, stream, a);
}

template <typename T>
void launch_few(const ForwardArgs& a, int act, hipStream_t stream) {
  switch (act) {
    case COMPAMS_SILU: launch_few<T, COMPAMS_SILU>(a, stream); break;
    case COMPAMS_GELU: launch_few<T, COMPAMS_GELU>(a, stream); break;
    case COMPAMS_GELU_TANH: launch_few<T, COMPAMS_GELU_TANH>(a, stream); break;
    case COMPAMS_RELU: launch_few<T, COMPAMS_RELU>(a, stream); break;
    default: launch_few<T, COMPAMS_SIGMOID>(a, stream); break;
  }
}
template <typename T>
void launch_forward(ForwardArgs& a, int act, hipStream_t stream) {
  if (few_rows(a.total, a.hidden)) return launch_few<T>(a, act, stream);
  switch (tile_size({{a.total, 2 * static_cast<uint64_t>(a.hidden), 1, a.cols}}, sizeof(T) == 4)) {
    case kTile256:
      if constexpr (sizeof(T) == 2) launch_forward<T, 4, 2, 4, 8>(a, act, stream);
      break;  // (64 columns of a projection to a wavefront)
    case kTile128: launch_forward<T, 2, 2, 4, 4>(a, act, stream); break;
    default: launch_forward<T, 2, 2, 2, 2>(a, act, stream); break;
  }
}

// ---- Backward ------------------------------------------------------------------------------------------------
struct BackwardArgs {
  const void *dm, *gate, *up;
  void *dgate, *dup;
  int64_t ld_dm, ld_gate, ld_up, ld_dgate, ld_dup;
  float* bias[2];       // of worker 0, or null
  int64_t ld_bias[2];
  float* partial;       // [worker][part][2][hidden], where there is more than one part
  uint32_t n, rows, hidden;
  uint32_t across, wide, parts, part_rows;
  uint32_t accumulate;
};
constexpr uint32_t kThreads = 256;
constexpr uint32_t kTogether = 4;  // rows of a lane

// A workgroup takes a part of a worker's rows and wide * 8 columns of them, a lane eight columns of every (256 / wide)-th row.
// Bound by memory: three matrices read, two written.
template <typename T, int ACT, bool BIAS>
__global__ __launch_bounds__(kThreads) void k_gated_backward(BackwardArgs a) {
  __shared__ float sums[BIAS ? 2 * kThreads * kGroup : 1];
  const uint32_t tall = kThreads / a.wide, id = tile_id();
  const uint32_t strip = id % a.across, piece = id / a.across;
  if (piece >= a.n * a.parts) return;
  const uint32_t w = piece / a.parts, part = piece - w * a.parts;
  const uint32_t lane = threadIdx.x & (a.wide - 1), down = threadIdx.x / a.wide;
  const uint32_t c = (strip * a.wide + lane) * kGroup;
  const uint32_t first = part * a.part_rows, last = min(first + a.part_rows, a.rows);
  float sg[kGroup] = {}, su[kGroup] = {};
  if (c < a.hidden) {
    // (kTogether rows' loads under way at once: outputs may lie over inputs, so the compiler keeps the order of accesses)
    for (uint32_t in = first + down; in < last; in += tall * kTogether) {
      typename Group<T>::type dm_raw[kTogether], g_raw[kTogether], u_raw[kTogether];
#pragma unroll
      for (uint32_t q = 0; q < kTogether; ++q) {
        const int64_t r = static_cast<int64_t>(w) * a.rows + min(in + q * tall, last - 1);
        dm_raw[q] = load_raw(static_cast<const T*>(a.dm) + r * a.ld_dm, c, a.hidden);
        g_raw[q] = load_raw(static_cast<const T*>(a.gate) + r * a.ld_gate, c, a.hidden);
        u_raw[q] = load_raw(static_cast<const T*>(a.up) + r * a.ld_up, c, a.hidden);
      }
#pragma unroll
      for (uint32_t q = 0; q < kTogether; ++q) {
        if (in + q * tall >= last) break;
        const int64_t r = static_cast<int64_t>(w) * a.rows + in + q * tall;
        float dm[kGroup], g[kGroup], u[kGroup], dg[kGroup], du[kGroup];
        unpack(dm, dm_raw[q]);
        unpack(g, g_raw[q]);
        unpack(u, u_raw[q]);
#pragma unroll
        for (uint32_t j = 0; j < kGroup; ++j) {
          float slope;
          const float v = activate<ACT, true, T>(g[j], slope);
          dg[j] = dm[j] * u[j] * slope;
          du[j] = dm[j] * v;
          if constexpr (BIAS) {
            sg[j] += dg[j];
            su[j] += du[j];
          }
        }
        store_group<T>(static_cast<T*>(a.dgate) + r * a.ld_dgate, c, a.hidden, dg);
        store_group<T>(static_cast<T*>(a.dup) + r * a.ld_dup, c, a.hidden, du);
      }
    }
  }
  if constexpr (BIAS) {
#pragma unroll
    for (uint32_t j = 0; j < kGroup; ++j) {
      sums[j * kThreads + threadIdx.x] = sg[j];
      sums[(kGroup + j) * kThreads + threadIdx.x] = su[j];
    }
    __syncthreads();
    // sixteen sums for each of `wide` groups
    for (uint32_t i = threadIdx.x; i < 2 * kGroup * a.wide; i += kThreads) {
      const uint32_t which = i / (kGroup * a.wide), of = i % (kGroup * a.wide), j = of % kGroup, l = of / kGroup;
      const uint32_t column = (strip * a.wide + l) * kGroup + j;
      float s = 0.0f;
      for (uint32_t k = 0; k < tall; ++k) s += sums[(which * kGroup + j) * kThreads + k * a.wide + l];
      if (column >= a.hidden) continue;
      if (a.parts > 1) {
        a.partial[((static_cast<uint64_t>(w) * a.parts + part) * 2 + which) * a.hidden + column] = s;
      } else if (a.bias[which]) {
        float* const to = a.bias[which] + static_cast<int64_t>(w) * a.ld_bias[which] + column;
        *to = a.accumulate ? *to + s : s;
      }
    }
  }
}

// The parts' sums of 32 columns, 32 lanes to a column.
constexpr uint32_t kBiasTurns = 32;
__global__ __launch_bounds__(32 * kBiasTurns) void k_gated_bias(BackwardArgs a) {
  __shared__ float sums[kBiasTurns][33];
  const uint32_t l = threadIdx.x % 32, turn = threadIdx.x / 32;
  const uint32_t column = blockIdx.x * 32 + l, which = blockIdx.z;
  if (!a.bias[which]) return;
  for (uint32_t w = blockIdx.y; w < a.n; w += gridDim.y) {
    float s = 0.0f;
    if (column < a.hidden)
#pragma unroll 4
      for (uint32_t p = turn; p < a.parts; p += kBiasTurns)
        s += a.partial[((static_cast<uint64_t>(w) * a.parts + p) * 2 + which) * a.hidden + column];
    sums[turn][l] = s;
    __syncthreads();
    if (turn == 0 && column < a.hidden) {
      float all = 0.0f;
#pragma unroll
      for (uint32_t k = 0; k < kBiasTurns; ++k) all += sums[k][l];
      float* const to = a.bias[which] + static_cast<int64_t>(w) * a.ld_bias[which] + column;
      *to = a.accumulate ? *to + all : all;
    }
    __syncthreads();
  }
}

template <typename T, int ACT>
void launch_backward(const BackwardArgs& a, uint64_t blocks, hipStream_t stream) {
  if (a.bias[0] || a.bias[1]) hipLaunchKernelGGL((k_gated_backward<T, ACT, true>), tile_grid(blocks), dim3(kThreads), 0, stream, a);
  else hipLaunchKernelGGL((k_gated_backward<T, ACT, false>), tile_grid(blocks), dim3(kThreads), 0, stream, a);
}
template <typename T>
void launch_backward(const BackwardArgs& a, int act, uint64_t blocks, hipStream_t stream) {
  switch (act) {
    case COMPAMS_SILU: launch_backward<T, COMPAMS_SILU>(a, blocks, stream); break;
    case COMPAMS_GELU: launch_backward<T, COMPAMS_GELU>(a, blocks, stream); break;
    case COMPAMS_GELU_TANH: launch_backward<T, COMPAMS_GELU_TANH>(a, blocks, stream); break;
    case COMPAMS_RELU: launch_backward<T, COMPAMS_RELU>(a, blocks, stream); break;
    default: launch_backward<T, COMPAMS_SIGMOID>(a, blocks, stream); break;
  }
}

// ---- Checks --------------------------------------------------------------------------------------------------
bool gated_valid(const compams_gated* a) {
  return a && rows_valid(a->n, a->rows, a->hidden) && a->hidden <= kMostEntries && float_type(a->type) &&
         a->activation >= COMPAMS_SILU && a->activation <= COMPAMS_SIGMOID;
}
bool forward_valid(const compams_gated* a) {
  return gated_valid(a) && a->cols >= 1 && a->cols <= kMostEntries && tiles_fit(a->n * a->rows, 2 * a->hidden, 1);
}

struct Operands {
  Matrix x, gate, up;
};
Operands operands(const compams_gated& a) {
  const size_t size = type_size(a.type);
  return {{a.x, a.ld_x, a.n * a.rows, a.cols, size},
          {a.gate_weight, a.ld_gate_weight, a.hidden, a.cols, size},
          {a.up_weight, a.ld_up_weight, a.hidden, a.cols, size}};
}
size_t forward_bytes(const compams_gated& a) {
  if (few_rows(a.n * a.rows, a.hidden)) return 0;
  const Operands o = operands(a);
  return o.x.packed_bytes() + o.gate.packed_bytes() + o.up.packed_bytes();
}

// How a worker's rows are cut: the lanes side by side in a workgroup and the rows of a part.
struct BackwardCut {
  uint32_t wide, across, parts, part_rows;
};
BackwardCut backward_cut(const compams_gated& a) {
  BackwardCut c;
  const uint64_t groups = (static_cast<uint64_t>(a.hidden) + kGroup - 1) / kGroup;
  // (several rows of a workgroup are added up in it, so that fewer parts are written)
  c.wide = lanes_across(groups);
  c.across = static_cast<uint32_t>((groups + c.wide - 1) / c.wide);
  const uint64_t tall = kThreads / c.wide;
  uint64_t rows = tall * 8;  // of a part
  // (so that the workgroups can be numbered)
  const uint64_t most = (1u << 30) / c.across / static_cast<uint64_t>(a.n) + 1;
  if ((static_cast<uint64_t>(a.rows) + rows - 1) / rows > most) rows = (static_cast<uint64_t>(a.rows) + most - 1) / most;
  c.part_rows = static_cast<uint32_t>(rows);
  c.parts = static_cast<uint32_t>((static_cast<uint64_t>(a.rows) + rows - 1) / rows);
  if (c.parts == 0) c.parts = 1;
  return c;
}
size_t backward_bytes(const compams_gated& a) {
  const BackwardCut c = backward_cut(a);
  if (c.parts == 1 || (!a.dgate_bias && !a.dup_bias)) return 0;
  return (static_cast<size_t>(a.n) * c.parts * 2 * a.hidden * sizeof(float) + 255) / 256 * 256;
}
}  // namespace
}  // namespace compams

extern "C" {

size_t compams_gated_forward_workspace_size(const compams_gated* a) {
  return compams::forward_valid(a) ? compams::forward_bytes(*a) : 0;
}
size_t compams_gated_backward_workspace_size(const compams_gated* a) {
  return compams::gated_valid(a) ? compams::backward_bytes(*a) : 0;
}

int compams_gated_forward(const compams_gated* a, void* hip_stream) {
  using namespace compams;
  if (!forward_valid(a)) return COMPAMS_INVALID_ARG;
  if (a->rows == 0) return COMPAMS_OK;
  const size_t size = type_size(a->type);
  if (!a->x || !a->gate_weight || !a->up_weight || !a->m || !stride_valid(a->ld_x, a->cols) ||
      !stride_valid(a->ld_gate_weight, a->cols) || !stride_valid(a->ld_up_weight, a->cols) || !stride_valid(a->ld_m, a->hidden) ||
      (a->gate && !stride_valid(a->ld_gate, a->hidden)) || (a->up && !stride_valid(a->ld_up, a->hidden)))
    return COMPAMS_INVALID_ARG;
  if (!aligned_to(a->x, size) || !aligned_to(a->gate_weight, size) || !aligned_to(a->up_weight, size) || !aligned_to(a->m, size) ||
      !aligned_to(a->gate, size) || !aligned_to(a->up, size) || !aligned_to(a->gate_bias, 4) || !aligned_to(a->up_bias, 4))
    return COMPAMS_BAD_ALIGNMENT;
  if (a->m == a->gate || a->m == a->up || (a->gate && a->gate == a->up)) return COMPAMS_INVALID_ARG;
  const int status = workspace_status(a->workspace, a->workspace_bytes, forward_bytes(*a));
  if (status != COMPAMS_OK) return status;
  // (other workgroups still read the inputs)
  const int64_t total = a->n * a->rows;
  const Area out[] = {area(a->m, total, a->hidden, a->ld_m, size), area(a->gate, total, a->hidden, a->ld_gate, size),
                      area(a->up, total, a->hidden, a->ld_up, size)};
  if (meet(out[0], out[1]) || meet(out[0], out[2]) || meet(out[1], out[2])) return COMPAMS_INVALID_ARG;
  for (const Area& in : {area(a->x, total, a->cols, a->ld_x, size), area(a->gate_weight, a->hidden, a->cols, a->ld_gate_weight, size),
                         area(a->up_weight, a->hidden, a->cols, a->ld_up_weight, size), area(a->gate_bias, 1, a->hidden, 0, 4),
                         area(a->up_bias, 1, a->hidden, 0, 4)})
    if (meet(out[0], in) || meet(out[1], in) || meet(out[2], in)) return COMPAMS_INVALID_ARG;
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  ForwardArgs k = {};
  const Operands o = operands(*a);
  const auto as_is = [&](const Matrix& m) { return Read{m.p, m.ld * static_cast<int64_t>(size)}; };
  if (few_rows(a->n * a->rows, a->hidden)) {
    k.x = as_is(o.x);
    k.gate_weight = as_is(o.gate);
    k.up_weight = as_is(o.up);
  } else {
    Packing packing;
    char* room = static_cast<char*>(a->workspace);
    k.x = packing.add(o.x, room);
    k.gate_weight = packing.add(o.gate, room);
    k.up_weight = packing.add(o.up, room);
    run_packing(packing, size, stream);
  }
  k.gate_bias = a->gate_bias; k.up_bias = a->up_bias;
  k.m = a->m; k.gate = a->gate; k.up = a->up;
  k.ld_m = a->ld_m; k.ld_gate = a->ld_gate; k.ld_up = a->ld_up;
  k.total = static_cast<uint32_t>(a->n * a->rows);
  k.cols = static_cast<uint32_t>(a->cols);
  k.hidden = static_cast<uint32_t>(a->hidden);
  if (a->type == COMPAMS_F32) launch_forward<float>(k, a->activation, stream);
  else if (a->type == COMPAMS_F16) launch_forward<half_t>(k, a->activation, stream);
  else launch_forward<bfloat_t>(k, a->activation, stream);
  return hipGetLastError() == hipSuccess ? COMPAMS_OK : COMPAMS_HIP_ERROR;
}

int compams_gated_backward(const compams_gated* a, void* hip_stream) {
  using namespace compams;
  if (!gated_valid(a) || (a->accumulate != 0 && a->accumulate != 1)) return COMPAMS_INVALID_ARG;
  const size_t size = type_size(a->type);
  for (const auto& [p, ld] : {std::pair<float*, int64_t>{a->dgate_bias, a->ld_dgate_bias}, {a->dup_bias, a->ld_dup_bias}}) {
    if (!p) continue;
    if (a->n > 1 && (ld < a->hidden || ld >= (static_cast<int64_t>(1) << 40))) return COMPAMS_INVALID_ARG;
    if (!aligned_to(p, 4)) return COMPAMS_BAD_ALIGNMENT;
  }
  if (a->dgate_bias && a->dgate_bias == a->dup_bias) return COMPAMS_INVALID_ARG;
  if (a->rows > 0) {
    if (!a->dm || !a->gate || !a->up || !a->dgate || !a->dup || !stride_valid(a->ld_dm, a->hidden) ||
        !stride_valid(a->ld_gate, a->hidden) || !stride_valid(a->ld_up, a->hidden) || !stride_valid(a->ld_dgate, a->hidden) ||
        !stride_valid(a->ld_dup, a->hidden))
      return COMPAMS_INVALID_ARG;
    if (!aligned_to(a->dm, size) || !aligned_to(a->gate, size) || !aligned_to(a->up, size) || !aligned_to(a->dgate, size) ||
        !aligned_to(a->dup, size))
      return COMPAMS_BAD_ALIGNMENT;
    if (a->dgate == a->dup) return COMPAMS_INVALID_ARG;
  } else if (!a->dgate_bias && !a->dup_bias) {
    return COMPAMS_OK;
  }
  const int status = workspace_status(a->workspace, a->workspace_bytes, backward_bytes(*a));
  if (status != COMPAMS_OK) return status;
  // (what is written over an input in other places than it is read from would be read by other workgroups)
  const int64_t total = a->n * a->rows;
  const Area out[] = {area(a->dgate, total, a->hidden, a->ld_dgate, size), area(a->dup, total, a->hidden, a->ld_dup, size)};
  const Area bias[] = {area(a->dgate_bias, a->n, a->hidden, a->ld_dgate_bias, 4), area(a->dup_bias, a->n, a->hidden, a->ld_dup_bias, 4)};
  if (meet(out[0], out[1]) || meet(bias[0], bias[1])) return COMPAMS_INVALID_ARG;
  for (const Area& in : {area(a->dm, total, a->hidden, a->ld_dm, size), area(a->gate, total, a->hidden, a->ld_gate, size),
                         area(a->up, total, a->hidden, a->ld_up, size)})
    for (int i = 0; i < 2; ++i)
      if ((meet(out[i], in) && !same(out[i], in)) || meet(bias[i], in) || meet(bias[i], out[0]) || meet(bias[i], out[1]))
        return COMPAMS_INVALID_ARG;
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const BackwardCut cut = backward_cut(*a);
  BackwardArgs k = {};
  k.dm = a->dm; k.gate = a->gate; k.up = a->up; k.dgate = a->dgate; k.dup = a->dup;
  k.ld_dm = a->ld_dm; k.ld_gate = a->ld_gate; k.ld_up = a->ld_up; k.ld_dgate = a->ld_dgate; k.ld_dup = a->ld_dup;
  k.bias[0] = a->dgate_bias; k.bias[1] = a->dup_bias;
  k.ld_bias[0] = a->ld_dgate_bias; k.ld_bias[1] = a->ld_dup_bias;
  k.partial = static_cast<float*>(a->workspace);
  k.n = static_cast<uint32_t>(a->n);
  k.rows = static_cast<uint32_t>(a->rows);
  k.hidden = static_cast<uint32_t>(a->hidden);
  k.wide = cut.wide; k.across = cut.across; k.parts = cut.parts; k.part_rows = cut.part_rows;
  k.accumulate = static_cast<uint32_t>(a->accumulate);
  const uint64_t blocks = static_cast<uint64_t>(k.across) * k.n * k.parts;
  if (a->type == COMPAMS_F32) launch_backward<float>(k, a->activation, blocks, stream);
  else if (a->type == COMPAMS_F16) launch_backward<half_t>(k, a->activation, blocks, stream);
  else launch_backward<bfloat_t>(k, a->activation, blocks, stream);
  if (cut.parts > 1 && (k.bias[0] || k.bias[1]))
    hipLaunchKernelGGL(k_gated_bias, dim3((k.hidden + 31) / 32, k.n < 16384 ? k.n : 16384, 2), dim3(32 * kBiasTurns), 0, stream, k);
  return hipGetLastError() == hipSuccess ? COMPAMS_OK : COMPAMS_HIP_ERROR;
}

}  // extern "C"
