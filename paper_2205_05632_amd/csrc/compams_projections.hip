// The gradients behind one or two projections that read the same x: of x, and of the weights for every worker.
#include "compams_tiles.h"

namespace compams {
namespace {

struct InputArgs {  // dx = dgate Wg + dup Wu
  Read d[2], weight[2];
  void* dx;
  int64_t ld_dx;
  uint32_t count, total, cols, hidden, tall, wide;
};

// k goes through the one projection's outputs and then the other's, so that dx is rounded once.  The weights' rows go across k:
// they are read as they lie and transposed on the way out of LDS.
template <typename TL>
__global__ __launch_bounds__(TL::kThreads) void k_projection_input(InputArgs a) {
  using T = typename TL::T;
  COMPAMS_TILE_LDS(TL, lds);
  const uint32_t tiles = a.tall * a.wide, id = tile_id();
  if (id >= tiles) return;
  uint32_t down, across;
  tile_at(by_die(id, tiles), a.tall, a.wide, down, across);
  const uint32_t m0 = down * TL::kM, n0 = across * TL::kN;
  TL t;
  t.clear();
  t.run([&](uint32_t i, Side& d, Side& w, Side&) {
    d = side<T, kAlong>(a.d[i].p, a.d[i].ld, a.total, m0, a.hidden);
    w = side<T, kAcross>(a.weight[i].p, a.weight[i].ld, a.cols, n0, a.hidden);
  }, a.count, a.hidden, lds);
  t.rows(lds.a[0], [&](uint32_t m, uint32_t n, const f32x4& v) {
    if (m0 + m < a.total)
      store4(static_cast<T*>(a.dx) + static_cast<int64_t>(m0 + m) * a.ld_dx + n0 + n, v, static_cast<int64_t>(a.cols) - n0 - n);
  });
}

struct WeightArgs {  // dW of worker i = d_i' x_i
  Read d[2], x;
  float* dweight[2];
  int64_t ld[2], stride[2];
  uint32_t n, rows, cols, hidden, tall, wide, count, accumulate;
};

// A worker's rows are k, so both operands go across it.  fp32 sums go straight to where the step reads them.
template <typename TL>
__global__ __launch_bounds__(TL::kThreads) void k_projection_weight(WeightArgs a) {
  using T = typename TL::T;
  COMPAMS_TILE_LDS(TL, lds);
  const uint32_t each = a.tall * a.wide, tiles = each * a.count * a.n, id = tile_id();
  if (id >= tiles) return;
  const uint32_t mine = by_die(id, tiles), which = mine / each % a.count, w = mine / each / a.count;
  uint32_t down, across;
  tile_at(mine % each, a.tall, a.wide, down, across);
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
    if (m0 + m >= a.hidden) return;
    add4(to + static_cast<int64_t>(m0 + m) * a.ld[which] + n0 + n, v, static_cast<int64_t>(a.cols) - n0 - n, a.accumulate);
  });
}

template <typename T, uint32_t WM, uint32_t WN, uint32_t FM, uint32_t FN>
void launch_input(InputArgs& a, hipStream_t stream) {
  using TL = Tiles<T, kAlong, kAcross, WM, WN, FM, FN>;
  a.tall = static_cast<uint32_t>(tiles_of(a.total, TL::kM));
  a.wide = static_cast<uint32_t>(tiles_of(a.cols, TL::kN));
  hipLaunchKernelGGL(k_projection_input<TL>, tile_grid(static_cast<uint64_t>(a.tall) * a.wide), dim3(TL::kThreads), 0, stream, a);
}
template <typename T, uint32_t WM, uint32_t WN, uint32_t FM, uint32_t FN>
void launch_weight(WeightArgs& a, hipStream_t stream) {
  using TL = Tiles<T, kAcross, kAcross, WM, WN, FM, FN>;
  a.tall = static_cast<uint32_t>(tiles_of(a.hidden, TL::kM));
  a.wide = static_cast<uint32_t>(tiles_of(a.cols, TL::kN));
  hipLaunchKernelGGL(k_projection_weight<TL>, tile_grid(static_cast<uint64_t>(a.tall) * a.wide * a.count * a.n), dim3(TL::kThreads), 0,
                     stream, a);
}
template <typename T>
void launch_both(InputArgs& in, WeightArgs& of, hipStream_t stream) {
  if (in.dx && in.total) {
    switch (tile_size(in.total, in.cols, 1)) {
      case kTile256: launch_input<T, 2, 4, 8, 4>(in, stream); break;
      case kTile128: launch_input<T, 2, 2, 4, 4>(in, stream); break;
      default: launch_input<T, 2, 2, 2, 2>(in, stream); break;
    }
  }
  if (of.count) {
    switch (tile_size(of.hidden, of.cols, static_cast<uint64_t>(of.count) * of.n)) {
      case kTile256: launch_weight<T, 2, 4, 8, 4>(of, stream); break;
      case kTile128: launch_weight<T, 2, 2, 4, 4>(of, stream); break;
      default: launch_weight<T, 2, 2, 2, 2>(of, stream); break;
    }
  }
}

// ---- Checks --------------------------------------------------------------------------------------------------
bool projections_valid(const compams_projections* a) {
  return a && rows_valid(a->n, a->rows, a->hidden) && a->hidden <= kMostEntries && a->cols >= 1 && a->cols <= kMostEntries &&
         float_type(a->type) && (a->dup || (!a->up_weight && !a->dup_weight) || a->rows == 0) &&
         (a->accumulate == 0 || a->accumulate == 1) && tiles_fit(a->n * a->rows, a->cols, 1) && tiles_fit(a->hidden, a->cols, 2 * a->n);
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
size_t projections_bytes(const compams_projections& a) {
  if (a.rows == 0) return 0;
  const Operands o = operands(a);
  size_t bytes = 0;
  for (int i = 0; i < 2; ++i) {
    if (o.d[i].p) bytes += o.d[i].packed_bytes();
    if (a.dx && o.weight[i].p) bytes += o.weight[i].packed_bytes();
  }
  return bytes + (o.x.p && (a.dgate_weight || a.dup_weight) ? o.x.packed_bytes() : 0);
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
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  InputArgs in = {};
  WeightArgs of = {};
  if (a->rows > 0) {
    // (two launches at most: a launch has room for four matrices)
    Packing one, two;
    char* room = static_cast<char*>(a->workspace);
    for (int i = 0; i < 2; ++i) {
      if (o.d[i].p) in.d[i] = one.add(o.d[i], room);
      if (a->dx && o.weight[i].p) in.weight[i] = one.add(o.weight[i], room);
    }
    if (o.x.p && (dweight[0] || dweight[1])) of.x = two.add(o.x, room);
    run_packing(one, size, stream);
    run_packing(two, size, stream);
  }
  in.dx = a->dx;
  in.ld_dx = a->ld_dx;
  in.count = a->dup ? 2 : 1;
  in.total = static_cast<uint32_t>(a->n * a->rows);
  in.cols = of.cols = static_cast<uint32_t>(a->cols);
  in.hidden = of.hidden = static_cast<uint32_t>(a->hidden);
  of.n = static_cast<uint32_t>(a->n);
  of.rows = static_cast<uint32_t>(a->rows);
  of.accumulate = static_cast<uint32_t>(a->accumulate);
  for (int i = 0; i < 2; ++i) {
    if (!dweight[i]) continue;
    of.d[of.count] = in.d[i];
    of.dweight[of.count] = dweight[i];
    of.ld[of.count] = ld[i];
    of.stride[of.count] = stride[i];
    ++of.count;
  }
  if (a->type == COMPAMS_F32) launch_both<float>(in, of, stream);
  else if (a->type == COMPAMS_F16) launch_both<half_t>(in, of, stream);
  else launch_both<bfloat_t>(in, of, stream);
  return hipGetLastError() == hipSuccess ? COMPAMS_OK : COMPAMS_HIP_ERROR;
}

}  // extern "C"
