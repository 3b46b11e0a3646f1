// The norm of every worker's gradient over all its tensors, and the gradient cut to a largest norm.
#include <algorithm>
#include <cstdlib>

#include "compams_tiles.h"

namespace compams {
namespace {

constexpr uint32_t kThreads = 256;
constexpr uint32_t kChunk = 4096;  // entries of a tensor's row to a workgroup
// A lane takes 16 bytes of the tensor at a time, neighbouring lanes neighbouring bytes.
template <typename F>
constexpr uint32_t kPiece = 16 / sizeof(F);
template <typename F>
constexpr uint32_t kTurns = kChunk / (kThreads * kPiece<F>);
template <typename T, uint32_t N>
struct Few {
  typedef T type __attribute__((ext_vector_type(N)));
  typedef type loose __attribute__((aligned(sizeof(T))));  // where rows start anywhere
};

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
  uint32_t n;
  uint32_t tensors, chunks;       // of the launch; chunks: of a worker
  uint32_t each, parts;           // chunks to a part, and parts of a worker in the launch
  uint32_t before, all;           // parts of a worker in the launches before, and in all
  double* partial;                // [worker][part]: sums of squares
  float *norms, *factors;         // the caller's, or null
  float* known;                   // factors, in the workspace
  float max_norm, scale;
  Tensor tensor[kMostTensors];
};
// Parts of a worker, and one more for each launch of kMostTensors tensors at most, whose last part may be a small one.  Every
// workgroup that scales a chunk adds them up for itself, some four to a lane.
constexpr uint32_t kMostParts = 1024;

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

// STREAM: past the caches.  (A template parameter: between two accesses that differ in nothing else the compiler drops the
// hint.) What is beyond the row's last entry is 0.
template <bool STREAM, typename F>
__device__ __forceinline__ void load_chunk(float (&v)[kTurns<F>][kPiece<F>], const F* row, int64_t first, int64_t count) {
  typedef Few<F, kPiece<F>> Load;
  const int64_t c = first + threadIdx.x * kPiece<F>;
  if (first + kChunk <= count) {  // (the same for the workgroup: all loads under way at once)
    typename Load::type raw[kTurns<F>];
#pragma unroll
    for (uint32_t k = 0; k < kTurns<F>; ++k) {
      const typename Load::loose* const at = reinterpret_cast<const typename Load::loose*>(row + c + k * kThreads * kPiece<F>);
      if constexpr (STREAM) raw[k] = __builtin_nontemporal_load(at);
      else raw[k] = *at;
    }
#pragma unroll
    for (uint32_t k = 0; k < kTurns<F>; ++k)
#pragma unroll
      for (uint32_t j = 0; j < kPiece<F>; ++j) v[k][j] = to_float(raw[k][j]);
  } else {
#pragma unroll
    for (uint32_t k = 0; k < kTurns<F>; ++k) {
      const int64_t at = c + k * kThreads * kPiece<F>;
      typename Load::type raw = {};
      if (at + kPiece<F> <= count) {
        raw = *reinterpret_cast<const typename Load::loose*>(row + at);
      } else {
#pragma unroll
        for (uint32_t j = 0; j < kPiece<F>; ++j)
          if (at + j < count) raw[j] = row[at + j];
      }
#pragma unroll
      for (uint32_t j = 0; j < kPiece<F>; ++j) v[k][j] = to_float(raw[j]);
    }
  }
}
template <bool STREAM, typename F, typename T>
__device__ __forceinline__ void store_chunk(T* row, int64_t first, int64_t count, const float (&v)[kTurns<F>][kPiece<F>]) {
  typedef Few<T, kPiece<F>> Store;
  const int64_t c = first + threadIdx.x * kPiece<F>;
  const bool whole = first + kChunk <= count;
#pragma unroll
  for (uint32_t k = 0; k < kTurns<F>; ++k) {
    const int64_t at = c + k * kThreads * kPiece<F>;
    if (whole || at + kPiece<F> <= count) {
      typename Store::type raw;
#pragma unroll
      for (uint32_t j = 0; j < kPiece<F>; ++j) raw[j] = static_cast<T>(v[k][j]);
      typename Store::loose* const to = reinterpret_cast<typename Store::loose*>(row + at);
      if constexpr (STREAM) __builtin_nontemporal_store(raw, to);
      else *to = raw;
    } else {
#pragma unroll
      for (uint32_t j = 0; j < kPiece<F>; ++j)
        if (at + j < count) row[at + j] = static_cast<T>(v[k][j]);
    }
  }
}

template <bool STREAM, typename F>
__device__ __forceinline__ double squares(const Tensor& t, uint32_t w, uint32_t chunk) {
  float v[kTurns<F>][kPiece<F>];
  const F* const row = static_cast<const F*>(t.from) + static_cast<int64_t>(w) * t.ld_from;
  load_chunk<STREAM>(v, row, static_cast<int64_t>(chunk) * kChunk, t.count);
  double s = 0.0;
#pragma unroll
  for (uint32_t k = 0; k < kTurns<F>; ++k)
#pragma unroll
    for (uint32_t j = 0; j < kPiece<F>; ++j) s = fma(static_cast<double>(v[k][j]), static_cast<double>(v[k][j]), s);
  return s;
}

// Sums of squares of a worker's parts.  Bound by memory (712 MB fp32 read and nothing else: 120 us, past the caches 108).  A
// square of an fp32 number is exact in fp64 up to its last five bits, and no sum of them leaves its range.
template <bool STREAM>
__global__ __launch_bounds__(kThreads) void k_clip_norm(ClipArgs a) {
  __shared__ double slots[kThreads / 64];
  const uint32_t w = blockIdx.y, last = min((blockIdx.x + 1) * a.each, a.chunks);
  double s = 0.0;
  for (uint32_t c = blockIdx.x * a.each; c < last; ++c) {
    const Tensor& t = a.tensor[tensor_of(a, c)];
    s += t.from_type == COMPAMS_F32   ? squares<STREAM, float>(t, w, c - t.first)
         : t.from_type == COMPAMS_F16 ? squares<STREAM, half_t>(t, w, c - t.first)
                                      : squares<STREAM, bfloat_t>(t, w, c - t.first);
  }
  s = sum_doubles(s, slots, kThreads / 64);
  if (threadIdx.x == 0) a.partial[static_cast<uint64_t>(w) * a.all + a.before + blockIdx.x] = s;
}

// A worker's factor, from its parts, added up in the same order by everybody.  It is 0 where zeros are to be written whatever
// is there.
__device__ __forceinline__ float factor_of(const ClipArgs& a, uint32_t w, double* slots, bool tell) {
  double s = 0.0;
  for (uint32_t i = threadIdx.x; i < a.all; i += kThreads) s += a.partial[static_cast<uint64_t>(w) * a.all + i];
  s = sum_doubles(s, slots, kThreads / 64);
  const double norm = sqrt(s) * a.scale;
  const float factor = !(s < INFINITY) ? 0.0f : norm > a.max_norm ? static_cast<float>(a.scale * (a.max_norm / norm)) : a.scale;
  if (tell && threadIdx.x == 0) {
    if (a.norms) a.norms[w] = static_cast<float>(norm);
    if (a.factors) a.factors[w] = factor;
  }
  return factor;
}

// The factors of many chunks, once for all of them, or of a call that writes nothing else.
__global__ __launch_bounds__(kThreads) void k_clip_factor(ClipArgs a) {
  __shared__ double slots[kThreads / 64];
  const float factor = factor_of(a, blockIdx.x, slots, true);
  if (threadIdx.x == 0) a.known[blockIdx.x] = factor;
}

// Entries of a row in front of the first one on 32 bytes: a chunk's pieces start there, the entries before are the first
// chunk's besides.  (Not where squares are added up: their order would be the address's.)
template <typename T>
__device__ __forceinline__ uint32_t before_whole(const T* row, int64_t count) {
  const uint32_t n = (32u - static_cast<uint32_t>(reinterpret_cast<uintptr_t>(row) & 31u)) % 32u / sizeof(T);
  return n < count ? n : static_cast<uint32_t>(count);
}
template <bool STREAM, typename F, typename T>
__device__ __forceinline__ void scaled(const ClipArgs& a, const Tensor& t, uint32_t w, uint32_t chunk, double* slots, bool tell) {
  const F* const row = static_cast<const F*>(t.from) + static_cast<int64_t>(w) * t.ld_from;
  T* const to = static_cast<T*>(t.to) + static_cast<int64_t>(w) * t.ld_to;
  const uint32_t head = before_whole(to, t.count);
  const int64_t first = static_cast<int64_t>(chunk) * kChunk;
  const bool mine = chunk == 0 && threadIdx.x < head;
  float v[kTurns<F>][kPiece<F>], one = 0.0f;
  load_chunk<STREAM>(v, row + head, first, t.count - head);
  if (mine) one = to_float(row[threadIdx.x]);
  const float factor = STREAM ? a.known[w] : factor_of(a, w, slots, tell);  // (while the entries are on their way)
  if (factor == 1.0f && t.to == t.from && t.ld_to == t.ld_from) return;
#pragma unroll
  for (uint32_t k = 0; k < kTurns<F>; ++k)
#pragma unroll
    for (uint32_t j = 0; j < kPiece<F>; ++j) v[k][j] = factor == 0.0f ? 0.0f : v[k][j] * factor;
  store_chunk<STREAM, F>(to + head, first, t.count - head, v);
  if (mine) to[threadIdx.x] = static_cast<T>(factor == 0.0f ? 0.0f : one * factor);
}

// From the last chunk to the first: what was read last for the norms is what the caches still have.  A chunk that is
// multiplied by one where it stands is left alone.  Bound by memory: 16 x 11.2 million fp32 read and written take 238 us in
// this shape (16 bytes a lane, four times, past the caches), 260 to 275 in others.
template <bool STREAM>
__global__ __launch_bounds__(kThreads) void k_clip_scale(ClipArgs a) {
  __shared__ double slots[kThreads / 64];
  const uint32_t w = a.n - 1 - blockIdx.y, c = a.chunks - 1 - blockIdx.x;
  const Tensor& t = a.tensor[tensor_of(a, c)];
  const uint32_t chunk = c - t.first;
  const bool tell = c == 0 && a.before == 0;
  if (!t.to) {
    if (!STREAM && tell) factor_of(a, w, slots, true);
  } else if (t.from_type == COMPAMS_F32) {
    scaled<STREAM, float, float>(a, t, w, chunk, slots, tell);
  } else if (t.from_type == COMPAMS_F16) {
    if (t.to_type == COMPAMS_F16) scaled<STREAM, half_t, half_t>(a, t, w, chunk, slots, tell);
    else scaled<STREAM, half_t, float>(a, t, w, chunk, slots, tell);
  } else {
    if (t.to_type == COMPAMS_BF16) scaled<STREAM, bfloat_t, bfloat_t>(a, t, w, chunk, slots, tell);
    else scaled<STREAM, bfloat_t, float>(a, t, w, chunk, slots, tell);
  }
}

// Norms of no entries.
__global__ __launch_bounds__(kThreads) void k_clip_none(ClipArgs a) {
  const uint32_t w = blockIdx.x * kThreads + threadIdx.x;
  if (w >= a.n) return;
  if (a.norms) a.norms[w] = 0.0f;
  if (a.factors) a.factors[w] = a.scale;
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
          (a->n > 1 && (t.ld_to < t.count || t.ld_to >= kMost)) || (t.to == t.from && (t.to_type != t.from_type || (a->n > 1 && t.ld_to != t.ld_from))))
        return COMPAMS_INVALID_ARG;
      if (!aligned_to(t.to, type_size(t.to_type))) return COMPAMS_BAD_ALIGNMENT;
    }
    chunks += chunks_of(t);
  }
  // (a launch's workgroups of one worker: 2^24 in a dimension of 2^32 threads)
  return chunks < (1u << 24) - 1 ? COMPAMS_OK : COMPAMS_INVALID_ARG;
}
// Whether what is written lies over nothing that is read elsewhere: no worker's rows of a tensor over another worker's, which
// would be scaled before they are read, and of the first worker no tensor's rows over another's: a tensor that is listed twice
// would be scaled twice, or once.  (Rows that are only read may be the same.)
bool apart(const compams_clip& a) {
  for (int32_t i = 0; i < a.tensors; ++i) {
    const compams_clip_tensor& t = a.tensor[i];
    if (t.to != t.from && meet(area(t.from, a.n, t.count, t.ld_from, type_size(t.from_type)),
                               area(t.to, a.n, t.count, t.ld_to, type_size(t.to_type))))
      return false;
  }
  struct Row {
    const char *begin, *end;
    bool written;
  };
  if (a.tensors == 0) return true;
  Row* const rows = static_cast<Row*>(std::malloc(2 * sizeof(Row) * static_cast<size_t>(a.tensors)));
  if (!rows) return false;
  size_t count = 0;
  const auto add = [&](const void* p, int64_t entries, int32_t type, bool written) {
    const char* const at = static_cast<const char*>(p);
    rows[count++] = {at, at + entries * static_cast<int64_t>(type_size(type)), written};
  };
  for (int32_t i = 0; i < a.tensors; ++i) {
    const compams_clip_tensor& t = a.tensor[i];
    if (t.count == 0) continue;
    if (t.to != t.from) add(t.from, t.count, t.from_type, false);
    if (t.to) add(t.to, t.count, t.to_type, true);
  }
  std::sort(rows, rows + count, [](const Row& x, const Row& y) { return x.begin < y.begin; });
  const char *any = nullptr, *written = nullptr;  // how far the rows so far go
  bool good = true;
  for (size_t i = 0; i < count; ++i) {
    const Row& r = rows[i];
    if (r.begin < (r.written ? any : written)) good = false;
    any = r.end > any ? r.end : any;
    if (r.written && r.end > written) written = r.end;
  }
  std::free(rows);
  return good;
}
inline size_t up256(size_t v) { return (v + 255) / 256 * 256; }

// How a worker's chunks are cut into parts, the same beside however many other workers.
struct Cut {
  uint64_t chunks = 0, bytes = 0;  // of a worker, in all
  uint32_t each = 1, parts = 0;
};
Cut cut_of(const compams_clip& a) {
  Cut c;
  for (int32_t i = 0; i < a.tensors; ++i) {
    c.chunks += chunks_of(a.tensor[i]);
    c.bytes += static_cast<uint64_t>(a.tensor[i].count) * type_size(a.tensor[i].from_type);
  }
  c.each = static_cast<uint32_t>((c.chunks + kMostParts - 1) / kMostParts);
  if (c.each == 0) c.each = 1;
  uint32_t in = 0;
  uint64_t chunks = 0;  // of a launch
  for (int32_t i = 0; i <= a.tensors; ++i) {
    if (i == a.tensors || in == kMostTensors) {
      c.parts += static_cast<uint32_t>((chunks + c.each - 1) / c.each);
      in = 0;
      chunks = 0;
    }
    if (i < a.tensors && a.tensor[i].count) {
      ++in;
      chunks += chunks_of(a.tensor[i]);
    }
  }
  return c;
}
size_t known_bytes(const compams_clip& a) { return up256(static_cast<size_t>(a.n) * sizeof(float)); }
size_t bytes_of(const compams_clip& a) {
  return known_bytes(a) + up256(static_cast<size_t>(a.n) * cut_of(a).parts * sizeof(double));
}

// launch(k) for every kMostTensors tensors.
template <typename Launch>
void by_launch(const compams_clip& a, ClipArgs& k, Launch launch) {
  k.before = 0;
  for (int32_t i = 0; i < a.tensors;) {
    k.tensors = k.chunks = 0;
    for (; i < a.tensors && k.tensors < kMostTensors; ++i) {
      const compams_clip_tensor& t = a.tensor[i];
      if (t.count == 0) continue;
      k.tensor[k.tensors++] = {t.from, t.to, t.ld_from, t.ld_to, t.count, k.chunks, static_cast<uint16_t>(t.from_type),
                               static_cast<uint16_t>(t.to_type)};
      k.chunks += static_cast<uint32_t>(chunks_of(t));
    }
    k.parts = (k.chunks + k.each - 1) / k.each;
    if (k.chunks) launch(k);
    k.before += k.parts;
  }
}

// Gradients that no cache holds until they are read again.  (us by size, through the caches and past them: into other rows
// 128 MB 66 and 68, 160 84 and 84, 192 104 and 99, 224 126 and 115; in place 128 65 and 70, 192 91 and 101, 256 122 and 133, 384
// 206 and 195.)
constexpr uint64_t kStreamBytes = 192u << 20;

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
  if (!apart(*a)) return COMPAMS_INVALID_ARG;
  const int status = workspace_status(a->workspace, a->workspace_bytes, bytes_of(*a));
  if (status != COMPAMS_OK) return status;
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const Cut cut = cut_of(*a);
  ClipArgs k = {};
  const uint32_t n = static_cast<uint32_t>(a->n);
  k.n = n;
  k.all = cut.parts;
  k.each = cut.each;
  k.known = static_cast<float*>(a->workspace);
  k.partial = reinterpret_cast<double*>(static_cast<char*>(a->workspace) + known_bytes(*a));
  k.norms = a->norms;
  k.factors = a->factors;
  k.max_norm = a->max_norm;
  k.scale = a->scale;
  if (cut.chunks == 0) {
    hipLaunchKernelGGL(k_clip_none, dim3((n + kThreads - 1) / kThreads), dim3(kThreads), 0, stream, k);
  } else {
    bool written = false;
    for (int32_t i = 0; i < a->tensors; ++i) written = written || (a->tensor[i].to && a->tensor[i].count);
    const bool past = cut.bytes * n > kStreamBytes;
    by_launch(*a, k, [&](const ClipArgs& l) {
      if (past) hipLaunchKernelGGL(k_clip_norm<true>, dim3(l.parts, n), dim3(kThreads), 0, stream, l);
      else hipLaunchKernelGGL(k_clip_norm<false>, dim3(l.parts, n), dim3(kThreads), 0, stream, l);
    });
    if (past || !written) hipLaunchKernelGGL(k_clip_factor, dim3(n), dim3(kThreads), 0, stream, k);
    if (written) by_launch(*a, k, [&](const ClipArgs& l) {
      if (past) hipLaunchKernelGGL(k_clip_scale<true>, dim3(l.chunks, n), dim3(kThreads), 0, stream, l);
      else hipLaunchKernelGGL(k_clip_scale<false>, dim3(l.chunks, n), dim3(kThreads), 0, stream, l);
    });
  }
  return hipGetLastError() == hipSuccess ? COMPAMS_OK : COMPAMS_HIP_ERROR;
}

}  // extern "C"
