// Softmax cross-entropy of an output layer, with logits l = weight x that are never stored, and its gradients.
//
// The vocabulary is gone over twice.  First every tile of the logits leaves a maximum and a sum of exponentials for each of its
// rows, from which a row's loss and its softmax's denominator follow.  Then, piece by piece of the vocabulary, the logits are formed
// again, turned into d = softmax - [target], and multiplied by the piece's weights (dx, whose fp32 sums wait in the workspace
// from piece to piece) and by x (dweight, of which a piece holds whole rows).  Five products of the logits' size instead of three, more
// for the digits of d, and no matrix of rows x vocabulary.
//
// d is held in T, in PARTS: d = first + second (+ third), each the rounded rest of those before, for dweight is fp32 and needs
// fp32's digits of it: fp32 one part, fp16 two (d times 2^14: the second is off by 2^-39 of the largest d), bfloat16 three (2^-25 of
// each d).  dx, of type T, takes the first part alone: one more rounding of half a step.
#include "compams_tiles.h"

namespace compams {
namespace {

constexpr uint32_t kThreads = 256;

template <typename T>
constexpr uint32_t kParts = sizeof(T) == 4 ? 1 : __is_same(T, half_t) ? 2 : 3;
// d as it is held is this often d.
template <typename T>
constexpr float kHeld = __is_same(T, half_t) ? 16384.0f : 1.0f;

// What the gradient needs of a row: d_c = e^(l_c - top) over - [c = target].
struct RowStat {
  float top, over;  // over: 1 / sum of e^(l - top); 0 for an ignored row, NaN for one without a softmax or a loss
};

struct LossArgs {
  Read x, weight;     // x: as the caller has it (ignored rows too)
  Read x_learnt;      // x with zeros in ignored rows
  const void* targets;
  int64_t ignore;
  uint32_t wide_targets;
  uint32_t n, rows, total, cols, vocab;
  uint32_t tall, wide;       // tiles of the launch
  float2* partial;           // [span of columns][row]: maximum, sum
  float* of_target;          // the target's logit of every row
  RowStat* stat;
  float* factor;             // grad_scale / count of every worker
  float grad_scale;
  float *mean_loss, *losses;
  // a piece of the vocabulary
  uint32_t first, width;     // its first entry and how many
  void* d;                   // [part][row][piece]
  int64_t ld_d;              // bytes
  int64_t part_bytes;
  float* dx_sum;             // fp32 sums of dx
  void* dx;
  int64_t ld_dx;
  float* dweight;
  int64_t ld_dweight, stride_dweight;
  uint32_t aligned;          // 1: four of dx at once, 2: of dweight
  uint32_t accumulate, begin, end;  // begin, end: the first and the last piece
};

__device__ __forceinline__ int64_t target_of(const LossArgs& a, uint32_t r) {
  return a.wide_targets ? static_cast<const int64_t*>(a.targets)[r] : static_cast<const int32_t*>(a.targets)[r];
}

// x with zeros in the rows that nothing is learnt from: whatever they hold, they add nothing to a weight's gradient.  (A NaN there
// would, times the zero that d is.)
template <typename T>
__global__ __launch_bounds__(kThreads) void k_linear_loss_rows(LossArgs a, const T* x, int64_t ld_x) {
  constexpr uint32_t kEach = 16 / sizeof(T);
  typedef typename Fragment<T>::type Piece;
  const uint32_t per_row = (a.cols + kEach - 1) / kEach;
  const uint64_t pieces = static_cast<uint64_t>(a.total) * per_row;
  for (uint64_t i = blockIdx.x * kThreads + threadIdx.x; i < pieces; i += static_cast<uint64_t>(gridDim.x) * kThreads) {
    const uint32_t row = static_cast<uint32_t>(i / per_row), c = static_cast<uint32_t>(i - static_cast<uint64_t>(row) * per_row) * kEach;
    Piece v = {};
    if (target_of(a, row) != a.ignore) {
      const T* const from = x + static_cast<int64_t>(row) * ld_x + c;
      if (c + kEach <= a.cols) {
        __builtin_memcpy(&v, from, sizeof(v));
      } else {
#pragma unroll
        for (uint32_t k = 0; k < kEach; ++k)
          if (c + k < a.cols) v[k] = from[k];
      }
    }
    static_cast<Piece*>(const_cast<void*>(a.x_learnt.p))[i] = v;
  }
}

template <typename TL>
__device__ __forceinline__ bool logits(TL& t, const LossArgs& a, uint32_t& m0, uint32_t& n0, lds_char* a0, lds_char* b0, lds_char* a1, lds_char* b1) {
  using T = typename TL::T;
  const uint32_t tiles = a.tall * a.wide, id = tile_id();
  if (id >= tiles) return false;
  uint32_t down, across;
  tile_at(by_die(id, tiles), a.tall, a.wide, down, across);
  m0 = down * TL::kM;
  n0 = across * TL::kN;
  t.clear();
  t.run([&](uint32_t, Side& x, Side& w, Side&) {
    x = side<T, kAlong>(a.x.p, a.x.ld, a.total, m0, a.cols);
    w = side<T, kAlong>(a.weight.p, a.weight.ld, a.vocab, a.first + n0, a.cols);
  }, 1, a.cols, a0, b0, a1, b1);
  return true;
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
// e^(l - top), and 0 where nothing has come yet that is more than minus infinity (a NaN stays one, an infinity gives one).
__device__ __forceinline__ float base_of(float top) { return top == -INFINITY ? 0.0f : top; }

// First pass.  A wavefront has 64 columns of its rows in every size of tile, so that a row's sums are added up in the same order
// beside however many others.
constexpr uint32_t kSpan = 64;
template <typename TL>
__global__ __launch_bounds__(TL::kThreads) void k_linear_loss_stats(LossArgs a) {
  static_assert(TL::FN * 16 == kSpan, "a wavefront's columns");
  COMPAMS_TILE_LDS(TL);
  TL t;
  uint32_t m0, n0;
  if (!logits(t, a, m0, n0, COMPAMS_TILE_LDS_ARGS)) return;
  const uint32_t span = n0 + TL::first_n(), n1 = span + TL::lane_n();
  if (span >= a.vocab) return;
#pragma unroll
  for (uint32_t i = 0; i < TL::FM; ++i) {
    const uint32_t r = m0 + TL::first_m() + TL::lane_m() + i * 16;
    float top = -INFINITY;
#pragma unroll
    for (uint32_t j = 0; j < TL::FN; ++j)
#pragma unroll
      for (uint32_t q = 0; q < 4; ++q) {
        if (n1 + j * 16 + q >= a.vocab) t.sum[i][j][q] = -INFINITY;
        top = fmaxf(top, t.sum[i][j][q]);
      }
    top = over_row(top, Max());
    const float base = base_of(top);
    float s = 0.0f;
#pragma unroll
    for (uint32_t j = 0; j < TL::FN; ++j)
#pragma unroll
      for (uint32_t q = 0; q < 4; ++q) s += __expf(t.sum[i][j][q] - base);
    s = over_row(s, Add());
    if (r >= a.total) continue;
    if (threadIdx.x % 64 < 16) a.partial[static_cast<uint64_t>(span / kSpan) * a.total + r] = make_float2(top, s);
    const int64_t at = target_of(a, r) - n1;
    if (at >= 0 && at < kSpan) {
#pragma unroll
      for (uint32_t j = 0; j < TL::FN; ++j)
#pragma unroll
        for (uint32_t q = 0; q < 4; ++q)
          if (at == j * 16 + q && n1 + at < a.vocab) a.of_target[r] = t.sum[i][j][q];
    }
  }
}

// A row's loss and softmax from its spans' maxima and sums: sixteen rows to a workgroup, sixteen lanes to a row.
__global__ __launch_bounds__(kThreads) void k_linear_loss_join(LossArgs a) {
  __shared__ float2 part[16][17];
  const uint32_t l = threadIdx.x % 16, turn = threadIdx.x / 16, spans = (a.vocab - 1) / kSpan + 1;
  for (uint64_t first = blockIdx.x * 16u; first < a.total; first += static_cast<uint64_t>(gridDim.x) * 16) {
    const uint64_t r = first + l;
    float top = -INFINITY, s = 0.0f;
    if (r < a.total)
      for (uint32_t k = turn; k < spans; k += 16) {
        const float2 one = a.partial[static_cast<uint64_t>(k) * a.total + r];
        const float more = fmaxf(top, one.x), base = base_of(more);
        s = s * __expf(top - base) + one.y * __expf(one.x - base);
        top = more;
      }
    part[turn][l] = make_float2(top, s);
    __syncthreads();
    if (turn == 0 && r < a.total) {
      float most = part[0][l].x;
#pragma unroll
      for (uint32_t k = 1; k < 16; ++k) most = fmaxf(most, part[k][l].x);
      float sum = 0.0f;  // (a row without a finite logit: e^(NaN))
#pragma unroll
      for (uint32_t k = 0; k < 16; ++k) sum += part[k][l].y * (part[k][l].x == most && most != -INFINITY ? 1.0f : __expf(part[k][l].x - most));
      const int64_t t = target_of(a, static_cast<uint32_t>(r));
      const bool learnt = t != a.ignore, inside = t >= 0 && t < a.vocab;
      const float loss = inside ? (most - a.of_target[r]) + logf(sum) : NAN;
      // (a target of probability 0 has an infinite loss, and a gradient; a sum that is no number has neither)
      float over = 1.0f / sum;
      if (!inside || !(most < INFINITY)) over = NAN;
      if (a.losses) a.losses[r] = learnt ? (over == over ? loss : NAN) : 0.0f;
      a.stat[r] = {most, learnt ? over : 0.0f};
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

// Second pass, a piece's d.  Entries behind the vocabulary's last are written too, as 0: they are read as a part of the last 16 bytes.
template <typename TL>
__global__ __launch_bounds__(TL::kThreads) void k_linear_loss_gradient(LossArgs a) {
  using T = typename TL::T;
  COMPAMS_TILE_LDS(TL);
  TL t;
  uint32_t m0, n0;
  if (!logits(t, a, m0, n0, COMPAMS_TILE_LDS_ARGS)) return;
  const uint32_t n1 = n0 + TL::first_n() + TL::lane_n();
#pragma unroll
  for (uint32_t i = 0; i < TL::FM; ++i) {
    const uint32_t r = m0 + TL::first_m() + TL::lane_m() + i * 16;
    if (r >= a.total) continue;
    const RowStat s = a.stat[r];
    const int64_t at = target_of(a, r) - a.first;
    char* const to = static_cast<char*>(a.d) + static_cast<int64_t>(r) * a.ld_d;
#pragma unroll
    for (uint32_t j = 0; j < TL::FN; ++j) {
      const uint32_t n = n1 + j * 16;
      if (n >= a.width + 16 / sizeof(T)) continue;
      f32x4 d;
#pragma unroll
      for (uint32_t q = 0; q < 4; ++q) {
        d[q] = __expf(t.sum[i][j][q] - s.top) * s.over;
        if (at == n + q) d[q] -= 1.0f;
        d[q] = s.over == 0.0f || n + q >= a.width ? 0.0f : d[q] * kHeld<T>;
      }
      typedef T T4 __attribute__((ext_vector_type(4)));
#pragma unroll
      for (uint32_t p = 0; p < kParts<T>; ++p) {
        T4 part;
#pragma unroll
        for (uint32_t q = 0; q < 4; ++q) {
          part[q] = static_cast<T>(d[q]);
          d[q] -= to_float(part[q]);
        }
        *reinterpret_cast<T4*>(to + p * a.part_bytes + n * sizeof(T)) = part;
      }
    }
  }
}

// dx of all rows.  The sums go on from those of the pieces before, so that they do not depend on where pieces end.
template <typename TL>
__global__ __launch_bounds__(TL::kThreads) void k_linear_loss_input(LossArgs a) {
  using T = typename TL::T;
  COMPAMS_TILE_LDS(TL);
  const uint32_t tiles = a.tall * a.wide, id = tile_id();
  if (id >= tiles) return;
  uint32_t down, across;
  tile_at(by_die(id, tiles), a.tall, a.wide, down, across);
  const uint32_t m0 = down * TL::kM, n0 = across * TL::kN;
  const uint32_t padded = (a.cols + 3) / 4 * 4;
  const auto sums = [&](uint32_t r, uint32_t n) { return reinterpret_cast<f32x4*>(a.dx_sum + static_cast<uint64_t>(r) * padded + n); };
  TL t;
  t.clear();
  if (!a.begin)
    t.each([&](uint32_t m, uint32_t n, f32x4& v) {
      if (m0 + m < a.total && n0 + n < a.cols) v = *sums(m0 + m, n0 + n);
    });
  t.run([&](uint32_t, Side& d, Side& w, Side&) {
    d = side<T, kAlong>(a.d, a.ld_d, a.total, m0, a.width);
    w = side<T, kAcross>(static_cast<const char*>(a.weight.p) + static_cast<int64_t>(a.first) * a.weight.ld, a.weight.ld, a.cols, n0, a.width);
  }, 1, a.width, COMPAMS_TILE_LDS_ARGS);
  t.rows((lds_char*)lds_a0, [&](uint32_t m, uint32_t n, f32x4 v) {
    const uint32_t r = m0 + m;
    if (r >= a.total || n0 + n >= a.cols) return;
    if (!a.end) {
      *sums(r, n0 + n) = v;
      return;
    }
    const bool learnt = a.stat[r].over != 0.0f;
    const float f = a.factor[r / a.rows] / kHeld<T>;
#pragma unroll
    for (uint32_t q = 0; q < 4; ++q) v[q] = learnt ? v[q] * f : 0.0f;
    store4(static_cast<T*>(a.dx) + static_cast<int64_t>(r) * a.ld_dx + n0 + n, v, static_cast<int64_t>(a.cols) - n0 - n, a.aligned & 1u);
  });
}

// dweight's rows of this piece, for every worker: k is the worker's rows, once for each part of d, the least first.
template <typename TL>
__global__ __launch_bounds__(TL::kThreads) void k_linear_loss_weight(LossArgs a) {
  using T = typename TL::T;
  COMPAMS_TILE_LDS(TL);
  const uint32_t each = a.tall * a.wide, tiles = each * a.n, id = tile_id();
  if (id >= tiles) return;
  const uint32_t mine = by_die(id, tiles), w = mine / each;
  uint32_t down, across;
  tile_at(mine - w * each, a.tall, a.wide, down, across);
  const uint32_t m0 = down * TL::kM, n0 = across * TL::kN;
  TL t;
  t.clear();
  const int64_t row = static_cast<int64_t>(w) * a.rows;
  t.run([&](uint32_t i, Side& d, Side& x, Side&) {
    const char* const part = static_cast<const char*>(a.d) + (kParts<T> - 1 - i) * a.part_bytes;
    d = side<T, kAcross>(part + row * a.ld_d, a.ld_d, a.width, m0, a.rows);  // (entries behind `width` meet no stored sum)
    x = side<T, kAcross>(static_cast<const char*>(a.x_learnt.p) + row * a.x_learnt.ld, a.x_learnt.ld, a.cols, n0, a.rows);
  }, kParts<T>, a.rows, COMPAMS_TILE_LDS_ARGS);
  const float f = a.factor[w] / kHeld<T>;
  float* const to = a.dweight + w * a.stride_dweight + static_cast<int64_t>(a.first) * a.ld_dweight;
  t.rows((lds_char*)lds_a0, [&](uint32_t m, uint32_t n, const f32x4& v) {
    if (m0 + m < a.width)
      add4(to + static_cast<int64_t>(m0 + m) * a.ld_dweight + n0 + n, v * f, static_cast<int64_t>(a.cols) - n0 - n, a.aligned >> 1 & 1u,
           a.accumulate);
  });
}

// ---- Launches ------------------------------------------------------------------------------------------------
enum Pass { kStats, kGradient, kInput, kWeight };

template <Pass PASS, typename T, uint32_t WM, uint32_t WN, uint32_t FM, uint32_t FN>
void launch_pass(LossArgs& a, hipStream_t stream) {
  constexpr Form A = PASS == kWeight ? kAcross : kAlong, B = PASS == kInput || PASS == kWeight ? kAcross : kAlong;
  using TL = Tiles<T, A, B, WM, WN, FM, FN>;
  a.tall = static_cast<uint32_t>(tiles_of(PASS == kWeight ? a.width : a.total, TL::kM));
  a.wide = static_cast<uint32_t>(tiles_of(PASS == kStats ? a.vocab : PASS == kGradient ? a.width : a.cols, TL::kN));
  const dim3 grid = tile_grid(static_cast<uint64_t>(a.tall) * a.wide * (PASS == kWeight ? a.n : 1)), block(TL::kThreads);
  if constexpr (PASS == kStats) hipLaunchKernelGGL(k_linear_loss_stats<TL>, grid, block, 0, stream, a);
  else if constexpr (PASS == kGradient) hipLaunchKernelGGL(k_linear_loss_gradient<TL>, grid, block, 0, stream, a);
  else if constexpr (PASS == kInput) hipLaunchKernelGGL(k_linear_loss_input<TL>, grid, block, 0, stream, a);
  else hipLaunchKernelGGL(k_linear_loss_weight<TL>, grid, block, 0, stream, a);
}
template <Pass PASS>
TileSize pass_size(const LossArgs& a) {
  if (PASS == kStats) return tile_size(a.total, a.vocab, 1);
  if (PASS == kGradient) return tile_size(a.total, a.width, 1);
  if (PASS == kInput) return tile_size(a.total, a.cols, 1);
  return tile_size(a.width, a.cols, a.n);
}
template <Pass PASS, typename T>
void launch_pass(LossArgs& a, hipStream_t stream) {
  switch (pass_size<PASS>(a)) {
    case kTile256: launch_pass<PASS, T, 2, 4, 8, 4>(a, stream); break;
    case kTile128: launch_pass<PASS, T, 2, 2, 4, 4>(a, stream); break;
    default:
      if constexpr (PASS == kStats) launch_pass<PASS, T, 4, 1, 1, 4>(a, stream);
      else launch_pass<PASS, T, 2, 2, 2, 2>(a, stream);
      break;
  }
}

// ---- The workspace -------------------------------------------------------------------------------------------
bool linear_loss_valid(const compams_linear_loss* a) {
  return a && rows_valid(a->n, a->rows, a->cols) && a->cols <= kMostEntries && a->vocab >= 1 &&
         a->vocab < (static_cast<int64_t>(1) << 31) && float_type(a->type) &&
         (a->target_type == COMPAMS_I32 || a->target_type == COMPAMS_I64) && (a->accumulate == 0 || a->accumulate == 1) &&
         tiles_fit(a->n * a->rows, a->vocab, 1) && tiles_fit(a->n * a->rows, a->cols, 1) && tiles_fit(a->vocab, a->cols, a->n);
}
struct Room {
  size_t x = 0, weight = 0, x_learnt = 0, partial = 0, of_target = 0, stat = 0, losses = 0, factor = 0, d = 0, dx_sum = 0;
  uint32_t piece = 0, pieces = 0;
  size_t all() const { return x + weight + x_learnt + partial + of_target + stat + losses + factor + d + dx_sum; }
};
inline size_t up256(size_t v) { return (v + 255) / 256 * 256; }
inline uint32_t parts_of(int32_t type) { return type == COMPAMS_F32 ? kParts<float> : type == COMPAMS_F16 ? kParts<half_t> : kParts<bfloat_t>; }

// A piece's d is to stay in the memory-side cache between the products that make and read it, and to be wide enough for them to
// fill the card.
constexpr size_t kPieceBytes = 192u << 20;
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
  if (a.dweight) r.x_learnt = up256(total * o.x.packed_row_bytes());
  const size_t column = total * size * parts_of(a.type);
  uint64_t piece = kPieceBytes / column / 256 * 256;
  if (piece < kLeastPiece) piece = kLeastPiece;
  r.pieces = static_cast<uint32_t>(tiles_of(a.vocab, piece));
  r.piece = static_cast<uint32_t>((tiles_of(a.vocab, r.pieces) + 255) / 256 * 256);
  r.pieces = static_cast<uint32_t>(tiles_of(a.vocab, r.piece));
  r.d = up256(column * r.piece);
  if (a.dx && r.pieces > 1) r.dx_sum = up256(total * ((a.cols + 3) / 4 * 4) * sizeof(float));
  return r;
}

template <typename T>
void run_linear_loss(LossArgs& k, const compams_linear_loss& a, const Room& room, hipStream_t stream) {
  const bool gradient = a.dx || a.dweight;
  if (k.total) {
    if (k.x_learnt.p) {
      const uint64_t pieces = static_cast<uint64_t>(k.total) * (k.x_learnt.ld / 16), blocks = (pieces + kThreads - 1) / kThreads;
      hipLaunchKernelGGL(k_linear_loss_rows<T>, dim3(static_cast<uint32_t>(blocks < 16384 ? blocks : 16384)), dim3(kThreads), 0, stream, k,
                         static_cast<const T*>(a.x), a.ld_x);
    }
    launch_pass<kStats, T>(k, stream);
    const uint32_t blocks = (k.total + 15) / 16;
    hipLaunchKernelGGL(k_linear_loss_join, dim3(blocks < 65536 ? blocks : 65536), dim3(kThreads), 0, stream, k);
  }
  if (a.mean_loss || gradient) hipLaunchKernelGGL(k_linear_loss_mean, dim3(k.n), dim3(1024), 0, stream, k);
  if (!gradient) return;
  if (!k.total) {
    if (a.dweight && !a.accumulate) {  // the sums of no rows
      k.width = k.vocab;
      launch_pass<kWeight, T>(k, stream);
    }
    return;
  }
  for (uint32_t p = 0; p < room.pieces; ++p) {
    k.first = p * room.piece;
    k.width = k.vocab - k.first < room.piece ? k.vocab - k.first : room.piece;
    k.begin = p == 0;
    k.end = p + 1 == room.pieces;
    launch_pass<kGradient, T>(k, stream);
    if (a.dx) launch_pass<kInput, T>(k, stream);
    if (a.dweight) launch_pass<kWeight, T>(k, stream);
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
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  LossArgs k = {};
  char* at = static_cast<char*>(a->workspace);
  if (a->rows > 0) {
    const Operands o = operands(*a);
    Packing packing;
    k.x = packing.add(o.x, at);
    k.weight = packing.add(o.weight, at);
    run_packing(packing, size, stream);
    if (room.x_learnt) k.x_learnt = {at, o.x.packed_row_bytes()};
  }
  const auto take = [&](size_t bytes) {
    char* const p = at;
    at += bytes;
    return p;
  };
  take(room.x_learnt);
  k.partial = reinterpret_cast<float2*>(take(room.partial));
  k.of_target = reinterpret_cast<float*>(take(room.of_target));
  k.stat = reinterpret_cast<RowStat*>(take(room.stat));
  float* const losses = reinterpret_cast<float*>(take(room.losses));
  k.losses = a->losses ? a->losses : losses;
  k.factor = reinterpret_cast<float*>(take(room.factor));
  k.d = take(room.d);
  k.dx_sum = reinterpret_cast<float*>(take(room.dx_sum));
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
  k.aligned = (aligned_to(a->dx, 4 * size) && a->ld_dx % 4 == 0) |
              (aligned_to(a->dweight, 16) && a->ld_dweight % 4 == 0 && a->stride_dweight % 4 == 0) << 1;
  k.accumulate = static_cast<uint32_t>(a->accumulate);
  if (a->type == COMPAMS_F32) run_linear_loss<float>(k, *a, room, stream);
  else if (a->type == COMPAMS_F16) run_linear_loss<half_t>(k, *a, room, stream);
  else run_linear_loss<bfloat_t>(k, *a, room, stream);
  return hipGetLastError() == hipSuccess ? COMPAMS_OK : COMPAMS_HIP_ERROR;
}

}  // extern "C"
