// The gradients behind one or two projections that read the same x: of x, and of the weights for every worker.
#include "compams_tiles.h"

namespace compams {
namespace {

struct ProjectionArgs {
  Read d[2], weight[2], x;
  void* dx;
  int64_t ld_dx;
  float* dweight[2];
  int64_t ld[2], stride[2];
  uint32_t n, rows, total, cols, hidden;
  uint32_t count;         // projections
  uint32_t weights;       // of their weights' gradients, how many are asked for
  uint32_t of[2];         // which
  uint32_t accumulate;
  uint32_t splits;        // parts of the projections' outputs whose sums of dx are formed apart,
  float* sums;            // and these: [split][row][cols]
  uint32_t tall, wide;    // tiles of dx
  uint32_t tall_weight;   // of a weight's gradient, beside those
};

// dx = dgate Wg + dup Wu: k goes through the one projection's outputs and then the other's, so that dx is rounded once.  The
// weights' rows go across k: they are read as they lie and transposed on the way out of LDS.
template <typename TL>
__device__ __forceinline__ void input_tile(const ProjectionArgs& a, uint32_t id, const TileLds& lds) {
  using T = typename TL::T;
  const uint32_t each = a.tall * a.wide, mine = by_die(id, each * a.splits), split = mine / each;
  uint32_t down, across;
  tile_at(mine - split * each, a.tall, a.wide, down, across);
  const uint32_t m0 = down * TL::kM, n0 = across * TL::kN;
  const uint32_t share = ((a.hidden + a.splits - 1) / a.splits + 63) / 64 * 64;
  const uint32_t k0 = min(split * share, a.hidden), k = min(share, a.hidden - k0);
  TL t;
  t.clear();
  t.run([&](uint32_t i, Side& d, Side& w, Side&) {
    d = side<T, kAlong>(static_cast<const char*>(a.d[i].p) + k0 * sizeof(T), a.d[i].ld, a.total, m0, k);
    w = side<T, kAcross>(static_cast<const char*>(a.weight[i].p) + static_cast<int64_t>(k0) * a.weight[i].ld, a.weight[i].ld,
                         a.cols, n0, k);
  }, a.count, k, lds);
  t.rows(lds.a[0], [&](uint32_t m, uint32_t n, const f32x4& v) {
    const uint32_t r = m0 + m;
    const int64_t left = static_cast<int64_t>(a.cols) - n0 - n;
    if (r >= a.total) return;
    if (a.splits == 1) store4(static_cast<T*>(a.dx) + static_cast<int64_t>(r) * a.ld_dx + n0 + n, v, left);
    else store4(a.sums + (static_cast<int64_t>(split) * a.total + r) * a.cols + n0 + n, v, left);
  });
}

// dx from the sums of its splits.
template <typename T>
__global__ __launch_bounds__(256) void k_projection_input(ProjectionArgs a) {
  const uint64_t all = static_cast<uint64_t>(a.total) * a.cols;
  for (uint64_t i = blockIdx.x * 256u + threadIdx.x; i < all; i += static_cast<uint64_t>(gridDim.x) * 256) {
    float v = 0.0f;
    for (uint32_t s = 0; s < a.splits; ++s) v += a.sums[s * all + i];
    const uint64_t r = i / a.cols;
    static_cast<T*>(a.dx)[static_cast<int64_t>(r) * a.ld_dx + static_cast<int64_t>(i - r * a.cols)] = static_cast<T>(v);
  }
}

// dW of worker i = d_i' x_i: a worker's rows are k, so both operands go across it. fp32 sums go straight to where the step
// reads them.
template <typename TL>
__device__ __forceinline__ void weight_tile(const ProjectionArgs& a, uint32_t id, const TileLds& lds) {
  using T = typename TL::T;
  const uint32_t each = a.tall_weight * a.wide, mine = by_die(id, each * a.weights * a.n), matrix = mine / each;
  const uint32_t which = a.of[matrix % a.weights], w = matrix / a.weights;
  uint32_t down, across;
  tile_at(mine - matrix * each, a.tall_weight, a.wide, down, across);
  const uint32_t m0 = down * TL::kM, n0 = across * TL::kN;
  TL t;
  t.clear();
  t.run([&](uint32_t, Side& d, Side& x, Side&) {
    const int64_t first = static_cast<int64_t>(w) * a.rows;
    d = side<T, kAcross>(static_cast<const char*>(a.d[which].p) + first * a.d[which].ld, a.d[which].ld, a.hidden, m0, a.rows);
    x = side<T, kAcross>(static_cast<const char*>(a.x.p) + first * a.x.ld, a.x.ld, a.cols, n0, a.rows);
  }, 1, a.rows, lds);
  float* const to = a.dweight[which] + w * a.stride[which];
  t.rows(lds.a[0], [&](uint32_t m, uint32_t n, const f32x4& v) {
    if (m0 + m < a.hidden)
      add4(to + static_cast<int64_t>(m0 + m) * a.ld[which] + n0 + n, v, static_cast<int64_t>(a.cols) - n0 - n, a.accumulate);
  });
}

// All of it in one launch: dx has few tiles with many terms to a sum, the weights' gradients many with few, and together they
// fill the card (8 x 1024 x 768 x 2048 bfloat16: 64.5 + 66.7 us apart). dx's tiles come first.
template <typename X, typename W>
__global__ __launch_bounds__(X::kThreads, 2) void k_projections(ProjectionArgs a) {
  static_assert(X::kBytesA == W::kBytesA && X::kBytesB == W::kBytesB && X::kThreads == W::kThreads, "one kind of tile");
  COMPAMS_TILE_LDS(X, lds);
  const uint32_t of_dx = a.dx ? a.tall * a.wide * a.splits : 0, of_weights = a.tall_weight * a.wide * a.weights * a.n;
  const uint32_t id = tile_id();
  if (id < of_dx) input_tile<X>(a, id, lds);
  else if (id < of_dx + of_weights) weight_tile<W>(a, id - of_dx, lds);
}

template <typename T, uint32_t WM, uint32_t WN, uint32_t FM, uint32_t FN, uint32_t STEP = 128>
void launch(ProjectionArgs& a, hipStream_t stream) {
  using X = Tiles<T, kAlong, kAcross, WM, WN, FM, FN, false, STEP>;
  using W = Tiles<T, kAcross, kAcross, WM, WN, FM, FN, false, STEP>;
  a.tall = static_cast<uint32_t>(tiles_of(a.total, X::kM));
  a.tall_weight = static_cast<uint32_t>(tiles_of(a.hidden, X::kM));
  a.wide = static_cast<uint32_t>(tiles_of(a.cols, X::kN));
  const uint64_t tiles = static_cast<uint64_t>(a.wide) * ((a.dx ? static_cast<uint64_t>(a.tall) * a.splits : 0) +
                                                          static_cast<uint64_t>(a.tall_weight) * a.weights * a.n);
  if (tiles) hipLaunchKernelGGL((k_projections<X, W>), tile_grid(tiles), dim3(X::kThreads), 0, stream, a);
}
template <typename T>
void launch(ProjectionArgs& a, hipStream_t stream) {
  switch (tile_size({{a.dx ? a.total : 0, a.cols, a.splits, static_cast<uint64_t>(a.hidden) * a.count / a.splits},
                     {a.weights ? a.hidden : 0, a.cols, static_cast<uint64_t>(a.weights) * a.n, a.rows}}, sizeof(T) == 4)) {
    case kTile256:
      if constexpr (sizeof(T) == 2) launch<T, 2, 2, 8, 4, 64>(a, stream);
      break;
    case kTile128: launch<T, 2, 2, 4, 4>(a, stream); break;
    default: launch<T, 2, 2, 2, 2>(a, stream); break;
  }
  if (a.dx && a.splits > 1) {
    const uint64_t blocks = (static_cast<uint64_t>(a.total) * a.cols + 255) / 256;
    hipLaunchKernelGGL(k_projection_input<T>, dim3(static_cast<uint32_t>(blocks < 16384 ? blocks : 16384)), dim3(256), 0, stream,
                       a);
  }
}

// ---- Checks --------------------------------------------------------------------------------------------------
bool projections_valid(const compams_projections* a) {
  return a && rows_valid(a->n, a->rows, a->hidden) && a->hidden <= kMostEntries && a->cols >= 1 && a->cols <= kMostEntries &&
         float_type(a->type) && (a->dup || (!a->up_weight && !a->dup_weight) || a->rows == 0) &&
         (a->accumulate == 0 || a->accumulate == 1) && tiles_fit(a->n * a->rows, a->cols, 16) &&
         tiles_fit(a->hidden, a->cols, 2 * a->n);
}
struct Operands {
  Matrix d[2], x, weight[2];
};
Operands operands(const compams_projections& a) {
  const size_t size = type_size(a.type);
  const int64_t total = a.n * a.rows;
  return {{{a.dgate, a.ld_dgate, total, a.hidden, size}, {a.dup, a.ld_dup, total, a.hidden, size}},
          {a.x, a.ld_x, total, a.cols, size},
          {{a.gate_weight, a.ld_gate_weight, a.hidden, a.cols, size}, {a.up_weight, a.ld_up_weight, a.hidden, a.cols, size}}};
}
uint32_t dx_splits(const compams_projections& a) {
  return splits_of(static_cast<uint64_t>(a.n) * a.rows, a.cols, static_cast<uint64_t>(a.hidden) * (a.dup ? 2 : 1),
                   a.type == COMPAMS_F32);
}
size_t sums_bytes(const compams_projections& a) {
  const size_t splits = dx_splits(a);
  return a.dx && splits > 1 ? (splits * a.n * a.rows * a.cols * sizeof(float) + 255) / 256 * 256 : 0;
}
size_t projections_bytes(const compams_projections& a) {
  if (a.rows == 0) return 0;
  const Operands o = operands(a);
  size_t bytes = 0;
  for (int i = 0; i < 2; ++i) {
    if (o.d[i].p) bytes += o.d[i].packed_bytes();
    if (a.dx && o.weight[i].p) bytes += o.weight[i].packed_bytes();
  }
  return bytes + (o.x.p && (a.dgate_weight || a.dup_weight) ? o.x.packed_bytes() : 0) + sums_bytes(a);
}

}  // namespace
}  // namespace compams

extern "C" {

size_t compams_projections_workspace_size(const compams_projections* a) {
  return compams::projections_valid(a) ? compams::projections_bytes(*a) : 0;
}

int compams_projections_backward(const compams_projections* a, void* hip_stream) {
  using namespace compams;
  if (!projections_valid(a) || (!a->dx && !a->dgate_weight && !a->dup_weight)) return COMPAMS_INVALID_ARG;
  const size_t size = type_size(a->type);
  float* const dweight[2] = {a->dgate_weight, a->dup_weight};
  const int64_t ld[2] = {a->ld_dgate_weight, a->ld_dup_weight}, stride[2] = {a->stride_dgate_weight, a->stride_dup_weight};
  for (int i = 0; i < 2; ++i) {
    if (!dweight[i]) continue;
    if (!gradient_valid(a->n, a->hidden, a->cols, ld[i], stride[i])) return COMPAMS_INVALID_ARG;
    if (!aligned_to(dweight[i], 4)) return COMPAMS_BAD_ALIGNMENT;
  }
  if (dweight[0] && dweight[0] == dweight[1]) return COMPAMS_INVALID_ARG;
  const Operands o = operands(*a);
  if (a->rows > 0) {
    const bool weights = dweight[0] || dweight[1];
    for (int i = 0; i < 2; ++i) {
      if (i == 1 && !a->dup) break;
      if (!o.d[i].p || !stride_valid(o.d[i].ld, a->hidden)) return COMPAMS_INVALID_ARG;
      if (a->dx && (!o.weight[i].p || !stride_valid(o.weight[i].ld, a->cols))) return COMPAMS_INVALID_ARG;
      if (!aligned_to(o.d[i].p, size) || (a->dx && !aligned_to(o.weight[i].p, size))) return COMPAMS_BAD_ALIGNMENT;
    }
    if ((weights && (!a->x || !stride_valid(a->ld_x, a->cols))) || (a->dx && !stride_valid(a->ld_dx, a->cols)))
      return COMPAMS_INVALID_ARG;
    if ((weights && !aligned_to(a->x, size)) || !aligned_to(a->dx, size)) return COMPAMS_BAD_ALIGNMENT;
  }
  const int status = workspace_status(a->workspace, a->workspace_bytes, projections_bytes(*a));
  if (status != COMPAMS_OK) return status;
  // (other workgroups still read the inputs)
  const Gradients of_weight[] = {{dweight[0], a->n, a->hidden, a->cols, ld[0], stride[0]},
                                 {dweight[1], a->n, a->hidden, a->cols, ld[1], stride[1]}};
  if (meet(of_weight[0], of_weight[1])) return COMPAMS_INVALID_ARG;
  const auto as_area = [&](const Matrix& m) { return area(m.p, m.rows, m.cols, m.ld, m.size); };
  const Area dx = area(a->dx, a->n * a->rows, a->cols, a->ld_dx, size), none = {};
  const Area extents[] = {of_weight[0].extents(), of_weight[1].extents()};
  const bool weights = dweight[0] || dweight[1];
  if (meet(extents[0], dx) || meet(extents[1], dx)) return COMPAMS_INVALID_ARG;
  for (const Area& in : {as_area(o.d[0]), as_area(o.d[1]), weights ? as_area(o.x) : none, a->dx ? as_area(o.weight[0]) : none,
                         a->dx ? as_area(o.weight[1]) : none})
    if (meet(dx, in) || meet(extents[0], in) || meet(extents[1], in)) return COMPAMS_INVALID_ARG;
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  ProjectionArgs k = {};
  if (a->rows > 0) {
    // (two launches at most: a launch has room for four matrices)
    Packing one, two;
    char* room = static_cast<char*>(a->workspace);
    for (int i = 0; i < 2; ++i) {
      if (o.d[i].p) k.d[i] = one.add(o.d[i], room);
      if (a->dx && o.weight[i].p) k.weight[i] = one.add(o.weight[i], room);
    }
    if (o.x.p && (dweight[0] || dweight[1])) k.x = two.add(o.x, room);
    run_packing(one, size, stream);
    run_packing(two, size, stream);
    k.dx = a->dx;
    k.sums = reinterpret_cast<float*>(room);
  }
  k.ld_dx = a->ld_dx;
  k.splits = dx_splits(*a);
  k.count = a->dup ? 2 : 1;
  k.n = static_cast<uint32_t>(a->n);
  k.rows = static_cast<uint32_t>(a->rows);
  k.total = k.n * k.rows;
  k.cols = static_cast<uint32_t>(a->cols);
  k.hidden = static_cast<uint32_t>(a->hidden);
  k.accumulate = static_cast<uint32_t>(a->accumulate);
  for (int i = 0; i < 2; ++i) {
    k.dweight[i] = dweight[i];
    k.ld[i] = ld[i];
    k.stride[i] = stride[i];
    if (dweight[i]) k.of[k.weights++] = static_cast<uint32_t>(i);
  }
  if (a->type == COMPAMS_F32) launch<float>(k, stream);
  else if (a->type == COMPAMS_F16) launch<half_t>(k, stream);
  else launch<bfloat_t>(k, stream);
  return hipGetLastError() == hipSuccess ? COMPAMS_OK : COMPAMS_HIP_ERROR;
}

}  // extern "C"
