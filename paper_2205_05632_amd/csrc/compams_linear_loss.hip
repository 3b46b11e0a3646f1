// Softmax cross-entropy of an output layer, with logits l = weight x that are never stored, and its gradients.
//
// The vocabulary is gone over twice.  First every tile of the logits leaves a maximum and a sum of exponentials for each of
// its rows, from which a row's loss and its softmax's denominator follow.  Then, piece by piece of the vocabulary, the logits
// are formed again, turned into d = softmax - [target], and multiplied by the piece's weights (dx, whose fp32 sums wait in the
// workspace from piece to piece) and by x (dweight, of which a piece holds whole rows).  Four products of the logits' size
// instead of three, two more for the digits of d where the operands have 16 bits, and no matrix of rows x vocabulary.
//
// d times 2^14 is held in float16 where the operands have 16 bits, in two parts: the second is the rounded rest of the first,
// so that both together are off by 2^-23 of an entry or 2^-39 of the largest possible one.  Both products take both parts. (With
// the first alone dx would be formed from eleven bits of every probability: 8192 x 50257 x 768 bfloat16 in 3.5 instead of 4.1 ms,
// but float16 up to 1.5 times as far from 64 bits, and few digits right where a column's terms cancel.  In bfloat16 three parts
// would be needed, and half as many products again.) bfloat16 operands of these products are therefore turned into float16, each
// column times the power of two that brings its largest entry just below 2^15, and the results' columns are scaled back: what
// 2^-39 of the largest entry of its own column does not reach is lost, as it is next to it in an fp32 sum.
#include "compams_tiles.h"

namespace compams {
namespace {

constexpr uint32_t kThreads = 256;

// What d and the operands of its products are held in, in how many parts, and how often d.
template <typename T>
struct HeldAs { typedef half_t type; };
template <>
struct HeldAs<float> { typedef float type; };
template <typename T>
using Held = typename HeldAs<T>::type;
template <typename T>
constexpr uint32_t kParts = sizeof(T) == 4 ? 1 : 2;
template <typename T>
constexpr float kHeld = sizeof(T) == 4 ? 1.0f : 16384.0f;
template <typename T>
constexpr bool kScaled = __is_same(T, bfloat_t);  // columns are scaled

// What the gradient needs of a row: d_c = e^(l_c - top) over - [c = target].
struct RowStat {
  float top, over;  // over: 1 / sum of e^(l - top); 0 for an ignored row, NaN for one without a softmax or a loss
  int32_t target;   // -1 for such rows
  uint32_t none;
};

struct Piece {
  uint32_t first, width;  // its first entry and how many
  char* d;                // [part][row][entry]
};

struct LossArgs {
  Read x, weight;     // x: as the caller has it (ignored rows too)
  Read x_held;        // x with zeros in ignored rows, and the weight, as the second pass's products read them
  Read weight_held;
  uint32_t* tops;     // bits of the largest entry of every column: of each worker's x, then of the weight
  const void* targets;
  int64_t ignore;
  uint32_t wide_targets;
  uint32_t n, rows, total, cols, vocab;
  uint32_t tall, wide;       // tiles of the launch
  uint32_t tall_weight;      // of dweight, beside those of dx
  uint32_t wide_next;        // of the next piece's d
  float2* partial;           // [span of columns][row]: maximum, sum
  float* of_target;          // the target's logit of every row
  RowStat* stat;
  float* factor;             // grad_scale / count of every worker
  float grad_scale;
  float *mean_loss, *losses;
  // a piece of the vocabulary that is multiplied, and the one after it, whose d is made meanwhile
  Piece now, next;
  int64_t ld_d;              // bytes from row to row of d
  int64_t part_bytes;
  float* dx_sum;             // fp32 sums of dx, of every split
  uint32_t splits;           // parts of a piece's columns whose sums of dx are formed apart
  void* dx;
  int64_t ld_dx;
  float* dweight;
  int64_t ld_dweight, stride_dweight;
  uint32_t accumulate, begin, end;  // begin, end: the first and the last piece
};

__device__ __forceinline__ int64_t target_of(const LossArgs& a, uint32_t r) {
  return a.wide_targets ? static_cast<const int64_t*>(a.targets)[r] : static_cast<const int32_t*>(a.targets)[r];
}

// The power of two that a column is multiplied by, from the bits of its largest entry.
__device__ __forceinline__ int shift_of(uint32_t top) {
  const int exponent = static_cast<int>(top >> 7) - 127;  // (bfloat16: eight bits of exponent over seven)
  return exponent == 128 ? 0 : min(14 - exponent, 126);   // (infinities and NaNs stay what they are)
}

// A workgroup's share of a matrix that is gone over by columns: `wide` lanes side by side with eight columns each, for `each`
// rows of the matrix a lane.  Matrices are the workers' x, and the weight as number n.
struct ColumnsArgs {
  const void *x, *weight;
  int64_t ld_x, ld_weight;        // entries
  uint32_t wide, across, each, parts_x, parts_weight;
};
struct Share {
  uint32_t matrix, first, last, column, step;  // rows first, first + step, ... before `last`
};
__device__ __forceinline__ bool share_of(const LossArgs& a, const ColumnsArgs& c, Share& s) {
  const uint32_t strip = tile_id() % c.across, tall = kThreads / c.wide;
  uint32_t part = tile_id() / c.across;
  const uint32_t of_x = c.parts_x * a.n;
  s.matrix = part < of_x ? part / c.parts_x : a.n;
  part = part < of_x ? part - s.matrix * c.parts_x : part - of_x;
  const uint32_t rows = s.matrix < a.n ? a.rows : a.vocab;
  s.step = tall;
  s.last = static_cast<uint32_t>(min(static_cast<uint64_t>(rows), static_cast<uint64_t>(part + 1) * tall * c.each));
  s.first = part * tall * c.each + threadIdx.x / c.wide;
  s.column = (strip * c.wide + threadIdx.x % c.wide) * kGroup;
  return s.column < a.cols && part < (s.matrix < a.n ? c.parts_x : c.parts_weight);
}

// The largest entry of every column.  (Whichever comes first: a maximum.)
__global__ __launch_bounds__(kThreads) void k_linear_loss_tops(LossArgs a, ColumnsArgs c) {
  __shared__ uint32_t joined[kThreads][kGroup + 1];
  Share s;
  const bool mine = share_of(a, c, s);
  uint32_t top[kGroup] = {};
  if (mine) {
    const bool of_x = s.matrix < a.n;
    const uint32_t row0 = of_x ? s.matrix * a.rows : 0;
    const bfloat_t* const p = static_cast<const bfloat_t*>(of_x ? c.x : c.weight);
    const int64_t ld = of_x ? c.ld_x : c.ld_weight;
#pragma unroll 4
    for (uint32_t r = s.first; r < s.last; r += s.step) {
      if (of_x && target_of(a, row0 + r) == a.ignore) continue;
      const typename Group<bfloat_t>::type raw = load_raw(p + static_cast<int64_t>(row0 + r) * ld, s.column, a.cols);
#pragma unroll
      for (uint32_t j = 0; j < kGroup; ++j) {
        uint16_t bits;
        __builtin_memcpy(&bits, reinterpret_cast<const char*>(&raw) + 2 * j, 2);
        top[j] = max(top[j], static_cast<uint32_t>(bits & 0x7fffu));
      }
    }
  }
#pragma unroll
  for (uint32_t j = 0; j < kGroup; ++j) joined[threadIdx.x][j] = top[j];
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < c.wide * kGroup; i += kThreads) {
    uint32_t most = 0;
    for (uint32_t k = i / kGroup; k < kThreads; k += c.wide) most = max(most, joined[k][i % kGroup]);
    const uint32_t column = tile_id() % c.across * c.wide * kGroup + i;
    if (column < a.cols && most) atomicMax(a.tops + static_cast<uint64_t>(s.matrix) * a.cols + column, most);
  }
}

// x with zeros in the rows that nothing is learnt from - whatever they hold, they add nothing to a weight's gradient (a NaN
// there would, times the zero that d is) - and, of bfloat16, both matrices in float16 with their columns scaled.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_linear_loss_hold(LossArgs a, ColumnsArgs c) {
  typedef typename Group<Held<T>>::type Out;
  Share s;
  if (!share_of(a, c, s)) return;
  const bool of_x = s.matrix < a.n;
  const uint32_t row0 = of_x ? s.matrix * a.rows : 0;
  const T* const p = static_cast<const T*>(of_x ? c.x : c.weight);
  const int64_t ld = of_x ? c.ld_x : c.ld_weight;
  char* const to = static_cast<char*>(const_cast<void*>(of_x ? a.x_held.p : a.weight_held.p));
  const int64_t ld_to = of_x ? a.x_held.ld : a.weight_held.ld;
  int shift[kGroup] = {};
  if constexpr (kScaled<T>) {
#pragma unroll
    for (uint32_t j = 0; j < kGroup; ++j)
      shift[j] = s.column + j < a.cols ? shift_of(a.tops[static_cast<uint64_t>(s.matrix) * a.cols + s.column + j]) : 0;
  }
#pragma unroll 4
  for (uint32_t r = s.first; r < s.last; r += s.step) {
    Out out = {};
    if (!of_x || target_of(a, row0 + r) != a.ignore) {
      const typename Group<T>::type raw = load_raw(p + static_cast<int64_t>(row0 + r) * ld, s.column, a.cols);
#pragma unroll
      for (uint32_t j = 0; j < kGroup; ++j) {
        if constexpr (kScaled<T>) out[j] = static_cast<half_t>(ldexpf(to_float(raw[j]), shift[j]));
        else out[j] = raw[j];
      }
    }
    char* const at = to + static_cast<int64_t>(row0 + r) * ld_to + s.column * sizeof(Held<T>);
    if (sizeof(Held<T>) == 2 || s.column + kGroup <= a.cols + 3) {
      __builtin_memcpy(__builtin_assume_aligned(at, 16), &out, sizeof(out));
    } else {  // (fp32: a row is padded to four entries)
      __builtin_memcpy(__builtin_assume_aligned(at, 16), &out, sizeof(out) / 2);
    }
  }
}

template <typename TL>
__device__ __forceinline__ void logits(TL& t, const LossArgs& a, uint32_t m0, uint32_t v0, const TileLds& lds) {
  using T = typename TL::T;
  t.clear();
  t.run([&](uint32_t, Side& x, Side& w, Side&) {
    x = side<T, kAlong>(a.x.p, a.x.ld, a.total, m0, a.cols);
    w = side<T, kAlong>(a.weight.p, a.weight.ld, a.vocab, v0, a.cols);
  }, 1, a.cols, lds);
}

// op over the four lanes (l, l + 16, l + 32, l + 48) that share a row of a tile.
template <typename Op>
__device__ __forceinline__ float over_row(float v, Op op) {
  const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = op(__uint_as_float(s[0]), __uint_as_float(s[1]));
  const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return op(__uint_as_float(q[0]), __uint_as_float(q[1]));
}
struct Max {
  __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
// e^z for z <= 0.  fp32 keeps its digits at any distance z; of 16-bit operands the product with log2(e) is rounded once, which puts
// an entry off by 1.2 |z| units of 2^-24 (their sum by the mean distance by weight, log(vocab) at most), while the parts of d hold it
// to 2^-39 of the largest.
template <typename T>
__device__ __forceinline__ float exp_of(float z) {
  if constexpr (sizeof(T) == 4) return exp_kept(z);
  else return __builtin_amdgcn_exp2f(z * 1.44269504088896341f);
}
// What a row's logits are compared with: their maximum, or 0 where that is minus infinity (e^(l - top) is 0 then, and not a
// NaN).
__device__ __forceinline__ float base_of(float top) { return top == -INFINITY ? 0.0f : top; }

// First pass.  A wavefront has 64 columns of its rows in every size of tile, so that a row's sums are added up in the same
// order beside however many others.
constexpr uint32_t kSpan = 64;
template <typename TL>
__global__ __launch_bounds__(TL::kThreads) void k_linear_loss_stats(LossArgs a) {
  static_assert(TL::FN * 16 == kSpan, "a wavefront's columns");
  COMPAMS_TILE_LDS(TL, lds);
  const uint32_t tiles = a.tall * a.wide, id = tile_id();
  if (id >= tiles) return;
  uint32_t down, across;
  tile_at(by_die(id, tiles), a.tall, a.wide, down, across);
  const uint32_t m0 = down * TL::kM, n0 = across * TL::kN;
  // (the targets before the products: after them, each of a lane's rows would wait for its own)
  const uint32_t r0 = m0 + TL::first_m() + TL::lane_m();
  int32_t target[TL::FM];
#pragma unroll
  for (uint32_t i = 0; i < TL::FM; ++i) {
    const int64_t of_row = target_of(a, min(r0 + i * 16, a.total - 1));
    target[i] = of_row >= 0 && of_row < a.vocab ? static_cast<int32_t>(of_row) : -1;
  }
  TL t;
  logits(t, a, m0, n0, lds);
  const uint32_t span = n0 + TL::first_n(), n1 = span + TL::lane_n();
  if (span >= a.vocab) return;
  if (span + kSpan > a.vocab) {  // (the same for the wavefront)
#pragma unroll
    for (uint32_t i = 0; i < TL::FM; ++i)
#pragma unroll
      for (uint32_t j = 0; j < TL::FN; ++j)
#pragma unroll
        for (uint32_t q = 0; q < 4; ++q)
          if (n1 + j * 16 + q >= a.vocab) t.sum[i][j][q] = -INFINITY;
  }
  // (rows beside one another and sums in fours: what one waits for is filled with the others)
  float top[TL::FM], sum[TL::FM];
#pragma unroll
  for (uint32_t i = 0; i < TL::FM; ++i) {
    f32x4 most = t.sum[i][0];
#pragma unroll
    for (uint32_t j = 1; j < TL::FN; ++j)
#pragma unroll
      for (uint32_t q = 0; q < 4; ++q) most[q] = fmaxf(most[q], t.sum[i][j][q]);
    top[i] = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3]));
  }
#pragma unroll
  for (uint32_t i = 0; i < TL::FM; ++i) top[i] = over_row(top[i], Max());
#pragma unroll
  for (uint32_t i = 0; i < TL::FM; ++i) {
    const float base = base_of(top[i]);
    f32x4 s;
#pragma unroll
    for (uint32_t j = 0; j < TL::FN; ++j)
#pragma unroll
      for (uint32_t q = 0; q < 4; ++q) {
        const float e = exp_of<typename TL::T>(t.sum[i][j][q] - base);
        s[q] = j == 0 ? e : s[q] + e;
      }
    sum[i] = (s[0] + s[1]) + (s[2] + s[3]);
  }
#pragma unroll
  for (uint32_t i = 0; i < TL::FM; ++i) sum[i] = over_row(sum[i], Add());
#pragma unroll
  for (uint32_t i = 0; i < TL::FM; ++i) {
    const uint32_t r = r0 + i * 16, at = static_cast<uint32_t>(target[i]) - n1;
    if (r >= a.total) continue;
    if (threadIdx.x % 64 < 16) a.partial[static_cast<uint64_t>(span / kSpan) * a.total + r] = make_float2(top[i], sum[i]);
    if (at < kSpan) {
#pragma unroll
      for (uint32_t j = 0; j < TL::FN; ++j)
#pragma unroll
        for (uint32_t q = 0; q < 4; ++q)
          if (at == j * 16 + q) a.of_target[r] = t.sum[i][j][q];
    }
  }
}

// A row's loss and softmax from its spans' maxima and sums: sixteen rows to a workgroup, 64 lanes to a row.
constexpr uint32_t kJoinLanes = 64;
__global__ __launch_bounds__(16 * kJoinLanes) void k_linear_loss_join(LossArgs a) {
  __shared__ float2 part[kJoinLanes][17];
  const uint32_t l = threadIdx.x % 16, turn = threadIdx.x / 16, spans = (a.vocab - 1) / kSpan + 1;
  if (a.tops)  // (cleared for the kernels that follow)
    for (uint64_t i = blockIdx.x * blockDim.x + threadIdx.x; i < static_cast<uint64_t>(a.n + 1) * a.cols;
         i += static_cast<uint64_t>(gridDim.x) * blockDim.x)
      a.tops[i] = 0;
  for (uint64_t first = blockIdx.x * 16u; first < a.total; first += static_cast<uint64_t>(gridDim.x) * 16) {
    const uint64_t r = first + l;
    float top = -INFINITY, s = 0.0f;
    if (r < a.total)
#pragma unroll 4
      for (uint32_t k = turn; k < spans; k += kJoinLanes) {
        const float2 one = a.partial[static_cast<uint64_t>(k) * a.total + r];
        const float more = fmaxf(top, one.x), base = base_of(more);
        s = s * exp_kept(top - base) + one.y * exp_kept(one.x - base);
        top = more;
      }
    // (the lanes of a row in a tree, every half in the other's place)
    for (uint32_t half = kJoinLanes / 2; half >= 16; half /= 2) {
      part[turn][l] = make_float2(top, s);
      __syncthreads();
      if (turn < half) {
        const float2 one = part[turn + half][l];
        const float more = fmaxf(top, one.x), base = base_of(more);
        s = s * exp_kept(top - base) + one.y * exp_kept(one.x - base);
        top = more;
      }
      __syncthreads();
    }
    if (turn < 16) part[turn][l] = make_float2(top, s);
    __syncthreads();
    if (turn == 0 && r < a.total) {
      float most = part[0][l].x;
#pragma unroll
      for (uint32_t k = 1; k < 16; ++k) most = fmaxf(most, part[k][l].x);
      float sum = 0.0f;  // (a row without a finite logit: e^(NaN))
#pragma unroll
      for (uint32_t k = 0; k < 16; ++k) sum += part[k][l].y * exp_kept(part[k][l].x - most);
      const int64_t t = target_of(a, static_cast<uint32_t>(r));
      const bool learnt = t != a.ignore, inside = t >= 0 && t < a.vocab;
      const float loss = inside ? (most - a.of_target[r]) + logf(sum) : NAN;
      // (a target of probability 0 has an infinite loss, and a gradient; a sum that is no number has neither)
      float over = 1.0f / sum;
      if (!inside || !(most < INFINITY)) over = NAN;
      if (a.losses) a.losses[r] = learnt ? (over == over ? loss : NAN) : 0.0f;
      a.stat[r] = {most, learnt ? over : 0.0f, learnt && inside ? static_cast<int32_t>(t) : -1, 0u};
    }
    __syncthreads();
  }
}

// A worker's mean loss, and the factor of its gradients.
__global__ __launch_bounds__(1024) void k_linear_loss_mean(LossArgs a) {
  __shared__ float slots[2][2][kSlots];
  uint32_t turn = 0;
  for (uint32_t w = blockIdx.x; w < a.n; w += gridDim.x, turn ^= 1u) {
    float s[2] = {0.0f, 0.0f};
    uint32_t count = 0;
    for (uint32_t in = threadIdx.x; in < a.rows; in += 1024) {
      const uint32_t r = w * a.rows + in;
      if (target_of(a, r) == a.ignore) continue;
      ++count;
      s[0] += a.losses[r];
    }
    s[1] = static_cast<float>(count);  // (fp32 counts exactly up to 2^24 rows of a worker)
    sum_block(s, slots[turn], 16);
    if (threadIdx.x == 0) {
      if (a.mean_loss) a.mean_loss[w] = s[1] > 0.0f ? s[0] / s[1] : 0.0f;
      if (a.factor) a.factor[w] = s[1] > 0.0f ? a.grad_scale / s[1] : 0.0f;
    }
  }
}

// Second pass, a tile of the next piece's d.  Entries behind the vocabulary's last are written too, as 0: they are read as a
// part of the last 16 bytes.
template <typename TL>
__device__ __forceinline__ void gradient_tile(const LossArgs& a, uint32_t id, const TileLds& lds) {
  using T = typename TL::T;
  const Piece p = a.next;
  uint32_t down, across;
  tile_at(by_die(id, a.tall * a.wide_next), a.tall, a.wide_next, down, across);
  const uint32_t m0 = down * TL::kM, n0 = across * TL::kN;
  TL t;
  logits(t, a, m0, p.first + n0, lds);
  const uint32_t n1 = n0 + TL::first_n() + TL::lane_n();
  const bool last = n0 + TL::kN > p.width;
#pragma unroll
  for (uint32_t i = 0; i < TL::FM; ++i) {
    const uint32_t r = m0 + TL::first_m() + TL::lane_m() + i * 16;
    const RowStat s = a.stat[min(r, a.total - 1)];
    const float over = s.over * kHeld<T>;
    const uint32_t at = static_cast<uint32_t>(s.target) - p.first - n1;
#pragma unroll
    for (uint32_t j = 0; j < TL::FN; ++j)
#pragma unroll
      for (uint32_t q = 0; q < 4; ++q) {
        // (the minimum: an ignored row's logits may be anything, and none is above its row's maximum in any other)
        float d = exp_of<T>(fminf(t.sum[i][j][q] - s.top, 0.0f)) * over;
        d -= at == j * 16 + q ? kHeld<T> : 0.0f;
        t.sum[i][j][q] = last && n1 + j * 16 + q >= p.width ? 0.0f : d;
      }
  }
  t.rows(lds.a[0], [&](uint32_t m, uint32_t n, const f32x4& v) {
    if (m0 + m >= a.total || n0 + n >= p.width + 16 / sizeof(T)) return;
    typedef Held<T> H4 __attribute__((ext_vector_type(4)));
    char* const to = p.d + static_cast<int64_t>(m0 + m) * a.ld_d + (n0 + n) * sizeof(Held<T>);
    H4 part;
#pragma unroll
    for (uint32_t q = 0; q < 4; ++q) part[q] = static_cast<Held<T>>(v[q]);
    *reinterpret_cast<H4*>(to) = part;
    if constexpr (kParts<T> == 2) {
      H4 rest;
#pragma unroll
      for (uint32_t q = 0; q < 4; ++q) rest[q] = static_cast<Held<T>>(v[q] - to_float(part[q]));
      *reinterpret_cast<H4*>(to + a.part_bytes) = rest;
    }
  });
}

// 2^-shift of four columns.
template <typename T>
__device__ __forceinline__ f32x4 scales(const LossArgs& a, uint32_t matrix, uint32_t n) {
  f32x4 v = {1.0f, 1.0f, 1.0f, 1.0f};
  if constexpr (kScaled<T>) {
#pragma unroll
    for (uint32_t q = 0; q < 4; ++q)
      if (a.tops && n + q < a.cols) v[q] = ldexpf(1.0f, -shift_of(a.tops[static_cast<uint64_t>(matrix) * a.cols + n + q]));
  }
  return v;
}

template <typename T>
__device__ __forceinline__ void store_dx(const LossArgs& a, uint32_t r, uint32_t n, f32x4 v, const f32x4& of_column) {
  const bool learnt = a.stat[r].over != 0.0f;
  const float f = a.factor[r / a.rows] / kHeld<T>;
#pragma unroll
  for (uint32_t q = 0; q < 4; ++q) v[q] = learnt ? v[q] * of_column[q] * f : 0.0f;
  store4(static_cast<T*>(a.dx) + static_cast<int64_t>(r) * a.ld_dx + n, v, static_cast<int64_t>(a.cols) - n);
}

// A tile of dx: k is the piece's columns, once for each part of d, the lesser first.  The sums go on from those of the pieces
// before.
template <typename TL, typename T>
__device__ __forceinline__ void input_tile(const LossArgs& a, uint32_t id, const TileLds& lds) {
  const uint32_t each = a.tall * a.wide, mine = by_die(id, each * a.splits), split = mine / each;
  uint32_t down, across;
  tile_at(mine - split * each, a.tall, a.wide, down, across);
  const uint32_t m0 = down * TL::kM, n0 = across * TL::kN, padded = (a.cols + 3) / 4 * 4;
  const uint32_t share = ((a.now.width + a.splits - 1) / a.splits + 63) / 64 * 64;
  const uint32_t k0 = min(split * share, a.now.width), width = min(share, a.now.width - k0);
  const auto sums = [&](uint32_t r, uint32_t n) {
    return reinterpret_cast<f32x4*>(a.dx_sum + (static_cast<uint64_t>(split) * a.total + r) * padded + n);
  };
  TL t;
  t.clear();
  if (!a.begin)
    t.each([&](uint32_t m, uint32_t n, f32x4& v) {
      if (m0 + m < a.total && n0 + n < a.cols) v = *sums(m0 + m, n0 + n);
    });
  t.template run<false>([&](uint32_t i, Side& d, Side& w, Side&) {
    const char* const part = a.now.d + (kParts<T> - 1 - i) * a.part_bytes;
    d = side<typename TL::T, kAlong>(part + k0 * sizeof(typename TL::T), a.ld_d, a.total, m0, width);
    const char* const rows = static_cast<const char*>(a.weight_held.p) + static_cast<int64_t>(a.now.first + k0) * a.weight_held.ld;
    w = side<typename TL::T, kAcross>(rows, a.weight_held.ld, a.cols, n0, width);
  }, kParts<T>, width, lds);
  const bool end = a.end && a.splits == 1;
  const f32x4 of_column = end ? scales<T>(a, a.n, n0 + TL::row_n()) : f32x4{};
  t.rows(lds.a[0], [&](uint32_t m, uint32_t n, f32x4 v) {
    const uint32_t r = m0 + m;
    if (r >= a.total || n0 + n >= a.cols) return;
    if (end) store_dx<T>(a, r, n0 + n, v, of_column);
    else *sums(r, n0 + n) = v;
  });
}

// A tile of dweight's rows of this piece, of one worker: k is the worker's rows, once for each part of d, the lesser first.
template <typename TL, typename T>
__device__ __forceinline__ void weight_tile(const LossArgs& a, uint32_t id, const TileLds& lds) {
  const uint32_t each = a.tall_weight * a.wide, mine = by_die(id, each * a.n), w = mine / each;
  uint32_t down, across;
  tile_at(mine - w * each, a.tall_weight, a.wide, down, across);
  const uint32_t m0 = down * TL::kM, n0 = across * TL::kN;
  TL t;
  t.clear();
  const int64_t row = static_cast<int64_t>(w) * a.rows;
  t.run([&](uint32_t i, Side& d, Side& x, Side&) {
    const char* const part = a.now.d + (kParts<T> - 1 - i) * a.part_bytes;
    const uint32_t columns = static_cast<uint32_t>(a.ld_d / sizeof(typename TL::T));
    d = side<typename TL::T, kAcross>(part + row * a.ld_d, a.ld_d, columns, m0, a.rows);
    x = side<typename TL::T, kAcross>(static_cast<const char*>(a.x_held.p) + row * a.x_held.ld, a.x_held.ld, a.cols, n0, a.rows);
  }, kParts<T>, a.rows, lds);  // (what d has behind `width` meets no sum that is stored)
  const f32x4 f = scales<T>(a, w, n0 + TL::row_n());
  const float factor = a.factor[w] / kHeld<T>;
  float* const to = a.dweight + w * a.stride_dweight + static_cast<int64_t>(a.now.first) * a.ld_dweight;
  t.rows(lds.a[0], [&](uint32_t m, uint32_t n, const f32x4& v) {
    if (m0 + m < a.now.width)
      add4(to + static_cast<int64_t>(m0 + m) * a.ld_dweight + n0 + n, v * f * factor, static_cast<int64_t>(a.cols) - n0 - n,
           a.accumulate);
  });
}

// A piece's products, and the d of the piece after it, in one launch: dx has few tiles of many steps (the piece's columns are
// its k), dweight many of few, d's tiles store more than they multiply, and together they fill the card.  (8192 x 50257 x 768
// bfloat16, in one launch each 96 tiles of dx and 384 of dweight left a third of it idle; d apart 165 us, the products 375 for
// 8448 columns.) dx's tiles come first, the shortest last.
template <typename D, typename X, typename W, typename T>
__global__ __launch_bounds__(X::kThreads, X::STEP == 64 && sizeof(T) == 2 ? 3 : 2) void k_linear_loss_piece(LossArgs a) {
  static_assert(X::kBytesA == W::kBytesA && X::kBytesB == W::kBytesB && X::kThreads == W::kThreads, "one kind of tile");
  static_assert(X::kBytesA == D::kBytesA && X::kBytesB == D::kBytesB && X::kThreads == D::kThreads, "one kind of tile");
  COMPAMS_TILE_LDS(X, lds);
  const bool any = a.now.width != 0;
  const uint32_t of_dx = any && a.dx ? a.tall * a.wide * a.splits : 0;
  const uint32_t of_weight = any && a.dweight ? a.tall_weight * a.wide * a.n : 0;
  const uint32_t of_d = a.next.width ? a.tall * a.wide_next : 0;
  uint32_t id = tile_id();
  if (id < of_dx) return input_tile<X, T>(a, id, lds);
  id -= of_dx;
  if (id < of_weight) return weight_tile<W, T>(a, id, lds);
  id -= of_weight;
  if (id < of_d) gradient_tile<D>(a, id, lds);
}

// dx from the sums of its splits, four entries to a lane.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_linear_loss_input(LossArgs a) {
  const uint32_t per_row = (a.cols + 3) / 4;
  const uint64_t all = static_cast<uint64_t>(a.total) * per_row;
  for (uint64_t i = blockIdx.x * kThreads + threadIdx.x; i < all; i += static_cast<uint64_t>(gridDim.x) * kThreads) {
    const uint32_t r = static_cast<uint32_t>(i / per_row), n = static_cast<uint32_t>(i - static_cast<uint64_t>(r) * per_row) * 4;
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
    for (uint32_t s = 0; s < a.splits; ++s) v += reinterpret_cast<const f32x4*>(a.dx_sum)[s * all + i];
    store_dx<T>(a, r, n, v, scales<T>(a, a.n, n));
  }
}

// ---- Launches ------------------------------------------------------------------------------------------------
template <typename T, uint32_t WM, uint32_t WN, uint32_t FM, uint32_t FN>
void launch_stats(LossArgs& a, hipStream_t stream) {
  using TL = Tiles<T, kAlong, kAlong, WM, WN, FM, FN>;
  a.tall = static_cast<uint32_t>(tiles_of(a.total, TL::kM));
  a.wide = static_cast<uint32_t>(tiles_of(a.vocab, TL::kN));
  hipLaunchKernelGGL(k_linear_loss_stats<TL>, tile_grid(static_cast<uint64_t>(a.tall) * a.wide), dim3(TL::kThreads), 0, stream, a);
}
template <typename T>
void launch_stats(LossArgs& a, hipStream_t stream) {
  switch (tile_size({{a.total, a.vocab, 1, a.cols}}, sizeof(T) == 4)) {
    case kTile256:
      if constexpr (sizeof(T) == 2) launch_stats<T, 2, 4, 8, 4>(a, stream);
      break;
    case kTile128: launch_stats<T, 2, 2, 4, 4>(a, stream); break;
    default: launch_stats<T, 4, 1, 1, 4>(a, stream); break;
  }
}
template <typename T, uint32_t WM, uint32_t WN, uint32_t FM, uint32_t FN, uint32_t STEP = 128>
void launch_piece(LossArgs& a, hipStream_t stream) {
  using D = Tiles<T, kAlong, kAlong, WM, WN, FM, FN, false, STEP>;
  using X = Tiles<Held<T>, kAlong, kAcross, WM, WN, FM, FN, false, STEP>;
  using W = Tiles<Held<T>, kAcross, kAcross, WM, WN, FM, FN, false, STEP>;
  a.tall = static_cast<uint32_t>(tiles_of(a.total, X::kM));
  a.tall_weight = static_cast<uint32_t>(tiles_of(a.now.width, X::kM));
  a.wide = static_cast<uint32_t>(tiles_of(a.cols, X::kN));
  a.wide_next = static_cast<uint32_t>(tiles_of(a.next.width, X::kN));
  uint64_t tiles = static_cast<uint64_t>(a.tall) * a.wide_next;
  if (a.now.width)
    tiles += static_cast<uint64_t>(a.wide) * ((a.dx ? static_cast<uint64_t>(a.tall) * a.splits : 0) +
                                              (a.dweight ? static_cast<uint64_t>(a.tall_weight) * a.n : 0));
  if (tiles) hipLaunchKernelGGL((k_linear_loss_piece<D, X, W, T>), tile_grid(tiles), dim3(X::kThreads), 0, stream, a);
}
template <typename T>
void launch_piece(LossArgs& a, TileSize size, hipStream_t stream) {
  switch (size) {
    case kTile256:
      if constexpr (sizeof(T) == 2) launch_piece<T, 2, 2, 8, 4, 64>(a, stream);
      break;
    case kTile128: launch_piece<T, 2, 2, 4, 4>(a, stream); break;
    default: launch_piece<T, 2, 2, 2, 2>(a, stream); break;
  }
}

// ---- The workspace -------------------------------------------------------------------------------------------
bool linear_loss_valid(const compams_linear_loss* a) {
  return a && rows_valid(a->n, a->rows, a->cols) && a->cols <= kMostEntries && a->vocab >= 1 &&
         a->vocab < (static_cast<int64_t>(1) << 31) && float_type(a->type) &&
         (a->target_type == COMPAMS_I32 || a->target_type == COMPAMS_I64) && (a->accumulate == 0 || a->accumulate == 1) &&
         tiles_fit(a->n * a->rows, a->vocab, 1) && tiles_fit(a->n * a->rows, a->cols, 16) && tiles_fit(a->vocab, a->cols, a->n);
}
struct Room {
  size_t x = 0, weight = 0, x_held = 0, weight_held = 0, tops = 0, partial = 0, of_target = 0, stat = 0, losses = 0, factor = 0;
  size_t d = 0, dx_sum = 0;
  uint32_t piece = 0, pieces = 0, splits = 1;
  size_t all() const {
    return x + weight + x_held + weight_held + tops + partial + of_target + stat + losses + factor + (pieces > 1 ? 2 : 1) * d + dx_sum;
  }
};
inline size_t up256(size_t v) { return (v + 255) / 256 * 256; }
inline uint32_t parts_of(int32_t type) { return type == COMPAMS_F32 ? kParts<float> : kParts<half_t>; }

// A piece's d: wide enough for the products that read it to fill the card, and for dx's sums, which are read and written with
// every piece, to be little beside it.
constexpr size_t kPieceBytes = 96u << 20;  // (two of them)
constexpr uint32_t kLeastPiece = 1024;

struct Operands {
  Matrix x, weight;
};
Operands operands(const compams_linear_loss& a) {
  const size_t size = type_size(a.type);
  return {{a.x, a.ld_x, a.n * a.rows, a.cols, size}, {a.weight, a.ld_weight, a.vocab, a.cols, size}};
}
Room room_of(const compams_linear_loss& a) {
  Room r;
  const size_t total = static_cast<size_t>(a.n) * a.rows, size = type_size(a.type);
  const bool gradient = a.dx || a.dweight;
  r.factor = up256(static_cast<size_t>(a.n) * sizeof(float));
  if (total == 0) return r;
  const Operands o = operands(a);
  r.x = o.x.packed_bytes();
  r.weight = o.weight.packed_bytes();
  r.partial = up256(tiles_of(a.vocab, kSpan) * total * sizeof(float2));
  r.of_target = up256(total * sizeof(float));
  r.stat = up256(total * sizeof(RowStat));
  r.losses = a.losses ? 0 : up256(total * sizeof(float));
  if (!gradient) return r;
  if (a.dweight) r.x_held = up256(total * o.x.packed_row_bytes());
  if (a.type == COMPAMS_BF16) {
    if (a.dx) r.weight_held = up256(static_cast<size_t>(a.vocab) * o.weight.packed_row_bytes());
    r.tops = up256((static_cast<size_t>(a.n) + 1) * a.cols * sizeof(uint32_t));
  }
  const size_t column = total * size * parts_of(a.type);
  uint64_t piece = kPieceBytes / column / 256 * 256;
  if (piece < kLeastPiece) piece = kLeastPiece;
  r.pieces = static_cast<uint32_t>(tiles_of(a.vocab, piece));
  r.piece = static_cast<uint32_t>((tiles_of(a.vocab, r.pieces) + 255) / 256 * 256);
  r.pieces = static_cast<uint32_t>(tiles_of(a.vocab, r.piece));
  r.d = up256(column * r.piece);  // (of one)
  if (a.dx) r.splits = splits_of(total, a.cols, a.vocab < r.piece ? a.vocab : r.piece, size == 4);
  if (a.dx && (r.pieces > 1 || r.splits > 1)) r.dx_sum = up256(r.splits * total * ((a.cols + 3) / 4 * 4) * sizeof(float));
  return r;
}

// The kernels that go over x and the weight by columns.
template <typename T>
void run_hold(const LossArgs& k, const compams_linear_loss& a, hipStream_t stream) {
  // (fewer rows a lane where that leaves compute units idle, 2048 x 256 fp32 9.7 us with sixteen; but every workgroup's maxima are
  // joined in memory, so not too few of those)
  const auto launch = [&](uint32_t least, auto go) {
    ColumnsArgs c = {a.x, a.weight, a.ld_x, a.ld_weight, 1, 1, 16, 0, 0};
    const uint32_t groups = (k.cols + kGroup - 1) / kGroup;
    c.wide = lanes_across(groups);
    c.across = (groups + c.wide - 1) / c.wide;
    const uint64_t tall = kThreads / c.wide, rows = (k.x_held.p ? k.total : 0) + (kScaled<T> && a.dx ? k.vocab : 0);
    while (c.each > least && rows * c.across < 512 * tall * c.each) c.each /= 2;
    const uint64_t each = tall * c.each;
    if (k.x_held.p) c.parts_x = static_cast<uint32_t>(tiles_of(k.rows, static_cast<uint32_t>(each)));
    if (kScaled<T> && a.dx) c.parts_weight = static_cast<uint32_t>(tiles_of(k.vocab, static_cast<uint32_t>(each)));
    const uint64_t blocks = (static_cast<uint64_t>(c.parts_x) * k.n + c.parts_weight) * c.across;
    if (blocks) go(tile_grid(blocks), c);
  };
  if constexpr (kScaled<T>)
    launch(8, [&](dim3 grid, const ColumnsArgs& c) { hipLaunchKernelGGL(k_linear_loss_tops, grid, dim3(kThreads), 0, stream, k, c); });
  launch(2, [&](dim3 grid, const ColumnsArgs& c) { hipLaunchKernelGGL(k_linear_loss_hold<T>, grid, dim3(kThreads), 0, stream, k, c); });
}

template <typename T>
void run_linear_loss(LossArgs& k, const compams_linear_loss& a, const Room& room, hipStream_t stream) {
  const bool gradient = a.dx || a.dweight;
  if (k.total) {
    launch_stats<T>(k, stream);
    const uint32_t blocks = (k.total + 15) / 16;
    hipLaunchKernelGGL(k_linear_loss_join, dim3(blocks < 65536 ? blocks : 65536), dim3(16 * kJoinLanes), 0, stream, k);
  }
  if (a.mean_loss || gradient) hipLaunchKernelGGL(k_linear_loss_mean, dim3(k.n), dim3(1024), 0, stream, k);
  if (!gradient) return;
  if (!k.total) {
    if (a.dweight && !a.accumulate) {  // the sums of no rows
      k.now.width = k.vocab;
      k.tops = nullptr;
      launch_piece<T>(k, kTile64, stream);
    }
    return;
  }
  run_hold<T>(k, a, stream);
  const auto piece = [&](uint32_t p) {
    if (p >= room.pieces) return Piece{0, 0, nullptr};
    const uint32_t first = p * room.piece, left = k.vocab - first;
    return Piece{first, left < room.piece ? left : room.piece, k.now.d + (p & 1u ? room.d : 0)};
  };
  char* const d = k.now.d;
  const auto size = [&] {
    return tile_size({{a.dx ? k.total : 0, k.cols, k.splits, static_cast<uint64_t>(k.now.width) * kParts<T> / k.splits},
                      {a.dweight ? k.now.width : 0, k.cols, k.n, static_cast<uint64_t>(k.rows) * kParts<T>},
                      {k.total, k.next.width, 1, k.cols}}, sizeof(T) == 4);
  };
  k.next = piece(0);
  k.now = {0, 0, d};
  launch_piece<T>(k, size(), stream);
  for (uint32_t p = 0; p < room.pieces; ++p) {
    k.now.d = d;
    const Piece now = piece(p), next = piece(p + 1);
    k.now = now;
    k.next = next;
    k.begin = p == 0;
    k.end = p + 1 == room.pieces;
    launch_piece<T>(k, size(), stream);
  }
  if (a.dx && k.splits > 1) {
    const uint64_t blocks = (static_cast<uint64_t>(k.total) * ((k.cols + 3) / 4) + kThreads - 1) / kThreads;
    const dim3 grid(static_cast<uint32_t>(blocks < 16384 ? blocks : 16384));
    hipLaunchKernelGGL(k_linear_loss_input<T>, grid, dim3(kThreads), 0, stream, k);
  }
}

}  // namespace
}  // namespace compams

extern "C" {

size_t compams_linear_loss_workspace_size(const compams_linear_loss* a) {
  return compams::linear_loss_valid(a) ? compams::room_of(*a).all() : 0;
}

int compams_linear_cross_entropy(const compams_linear_loss* a, void* hip_stream) {
  using namespace compams;
  if (!linear_loss_valid(a) || (!a->mean_loss && !a->losses && !a->dx && !a->dweight)) return COMPAMS_INVALID_ARG;
  if (!aligned_to(a->mean_loss, 4) || !aligned_to(a->losses, 4) || !aligned_to(a->dweight, 4)) return COMPAMS_BAD_ALIGNMENT;
  if (a->dweight && !gradient_valid(a->n, a->vocab, a->cols, a->ld_dweight, a->stride_dweight)) return COMPAMS_INVALID_ARG;
  const size_t size = type_size(a->type);
  if (a->rows > 0) {
    if (!a->x || !a->weight || !a->targets || !stride_valid(a->ld_x, a->cols) || !stride_valid(a->ld_weight, a->cols) ||
        (a->dx && !stride_valid(a->ld_dx, a->cols)))
      return COMPAMS_INVALID_ARG;
    if (!aligned_to(a->x, size) || !aligned_to(a->weight, size) || !aligned_to(a->dx, size) ||
        !aligned_to(a->targets, type_size(a->target_type)))
      return COMPAMS_BAD_ALIGNMENT;
  }
  const Room room = room_of(*a);
  const int status = workspace_status(a->workspace, a->workspace_bytes, room.all());
  if (status != COMPAMS_OK) return status;
  // (what is written while it is still read, here or by a later launch; x is read for the last time before the launch that writes dx)
  const int64_t total = a->n * a->rows;
  const Area in[] = {area(a->x, total, a->cols, a->ld_x, size), area(a->weight, a->vocab, a->cols, a->ld_weight, size),
                     area(a->targets, 1, total, 0, type_size(a->target_type))};
  const Area out[] = {area(a->dx, total, a->cols, a->ld_dx, size),
                      Gradients{a->dweight, a->n, a->vocab, a->cols, a->ld_dweight, a->stride_dweight}.extents(),
                      area(a->losses, 1, total, 0, 4), area(a->mean_loss, 1, a->n, 0, 4)};
  for (int i = 0; i < 4; ++i) {
    for (int j = 0; j < i; ++j)
      if (meet(out[i], out[j])) return COMPAMS_INVALID_ARG;
    for (int j = i == 0 ? 1 : 0; j < 3; ++j)
      if (total && meet(out[i], in[j])) return COMPAMS_INVALID_ARG;
  }
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  LossArgs k = {};
  char* at = static_cast<char*>(a->workspace);
  if (a->rows > 0) {
    const Operands o = operands(*a);
    Packing packing;
    k.x = packing.add(o.x, at);
    k.weight = packing.add(o.weight, at);
    run_packing(packing, size, stream);
    if (room.x_held) k.x_held = {at, o.x.packed_row_bytes()};
    k.weight_held = room.weight_held ? Read{at + room.x_held, o.weight.packed_row_bytes()} : k.weight;
  }
  const auto take = [&](size_t bytes) {
    char* const p = at;
    at += bytes;
    return p;
  };
  take(room.x_held);
  take(room.weight_held);
  k.tops = room.tops ? reinterpret_cast<uint32_t*>(take(room.tops)) : nullptr;
  k.partial = reinterpret_cast<float2*>(take(room.partial));
  k.of_target = reinterpret_cast<float*>(take(room.of_target));
  k.stat = reinterpret_cast<RowStat*>(take(room.stat));
  float* const losses = reinterpret_cast<float*>(take(room.losses));
  k.losses = a->losses ? a->losses : losses;
  k.factor = reinterpret_cast<float*>(take(room.factor));
  k.now.d = take((room.pieces > 1 ? 2 : 1) * room.d);
  k.dx_sum = reinterpret_cast<float*>(take(room.dx_sum));
  k.splits = room.splits;
  k.targets = a->targets;
  k.ignore = a->ignore_index;
  k.wide_targets = a->target_type == COMPAMS_I64;
  k.n = static_cast<uint32_t>(a->n);
  k.rows = static_cast<uint32_t>(a->rows);
  k.total = k.n * k.rows;
  k.cols = static_cast<uint32_t>(a->cols);
  k.vocab = static_cast<uint32_t>(a->vocab);
  k.grad_scale = a->grad_scale;
  k.mean_loss = a->mean_loss;
  k.ld_d = static_cast<int64_t>(room.piece) * size;
  k.part_bytes = k.ld_d * k.total;
  k.dx = a->dx; k.ld_dx = a->ld_dx;
  k.dweight = a->dweight; k.ld_dweight = a->ld_dweight; k.stride_dweight = a->stride_dweight;
  k.accumulate = static_cast<uint32_t>(a->accumulate);
  if (a->type == COMPAMS_F32) run_linear_loss<float>(k, *a, room, stream);
  else if (a->type == COMPAMS_F16) run_linear_loss<half_t>(k, *a, room, stream);
  else run_linear_loss<bfloat_t>(k, *a, room, stream);
  return hipGetLastError() == hipSuccess ? COMPAMS_OK : COMPAMS_HIP_ERROR;
}

}  // extern "C"
