// Device-side helpers of the operators on activations: element types, a lane's eight columns, sums over the lanes that
// share a row, and the generator of the dropout masks.  (wave64 only)
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/compams.h"

namespace compams {

// ---- Element types -------------------------------------------------------------------------------------------
typedef _Float16 half_t;
typedef __bf16 bfloat_t;

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(half_t v) { return static_cast<float>(v); }
__device__ __forceinline__ float to_float(bfloat_t v) { return static_cast<float>(v); }

// e^z to three units of 2^-24 at any z: the exponent of 2 as a whole number and a part in -1/2 .. 1/2, which is formed with the
// rounding of the product and of log2(e) put right.  (Rounded once, an exponent of 60 is off by up to 2^-19: 22 such units of the
// result.)  Beyond 200 in size z counts as that: whatever it is, 0 or infinity is left.  A NaN stays one.
__device__ __forceinline__ float exp_kept(float z) {
  constexpr double kExact = 1.44269504088896340736;
  constexpr float kLog2E = static_cast<float>(kExact), kRest = static_cast<float>(kExact - static_cast<double>(kLog2E));
  constexpr float kShift = 0x1.8p23f;  // what is added to it is rounded to a whole number, which is in the low bits then
  const float at = __builtin_elementwise_minimum(__builtin_elementwise_maximum(z, -200.0f), 200.0f);
  const float shifted = fmaf(at, kLog2E, kShift), whole = shifted - kShift;
  const float part = fmaf(at, kRest, fmaf(at, kLog2E, -whole));
  return __builtin_amdgcn_ldexpf(__builtin_amdgcn_exp2f(part), static_cast<int16_t>(__float_as_uint(shifted)));
}

// A lane works on groups of eight neighbouring columns: 16 bytes of the narrow types, and one counter of the generator.
constexpr uint32_t kGroup = 8;

template <typename T>
struct Group {
  typedef T type __attribute__((ext_vector_type(8)));
};

// Makes the compiler forget what it knows of a value: what follows from it is formed where it is used.
__device__ __forceinline__ void forget(uint32_t& v) { asm volatile("" : "+v"(v)); }

// A group's words moved down by S elements, where bit S of `by` is set.
template <uint32_t S, typename T, typename Words>
__device__ __forceinline__ void move_down(Words& w, uint32_t by) {
  constexpr uint32_t kPerWord = 4 / sizeof(T), kWords = kGroup / kPerWord, kStep = S / kPerWord;
  Words moved = {};
#pragma unroll
  for (uint32_t i = 0; i < kWords; ++i) {
    if constexpr (S >= kPerWord) {
      if (i + kStep < kWords) moved[i] = w[i + kStep];
    } else {  // half a word
      moved[i] = (w[i] >> 16) | (i + 1 < kWords ? w[i + 1 < kWords ? i + 1 : i] << 16 : 0u);
    }
  }
#pragma unroll
  for (uint32_t i = 0; i < kWords; ++i) w[i] = by & S ? moved[i] : w[i];
}

// What a kernel knows of its rows' width.
enum Width {
  kAnyWidth = 0,   // at least eight columns
  kFullGroups = 1, // no lane has a group that reaches beyond the last column
  kOneGroup = 2,   // fewer than eight columns: no wide load fits, and one lane has all of them
  kWholeGroups = 3 // a multiple of eight columns: lanes have a group of the row or, beyond its last, none
};

// Columns c .. c + 7 of a row of `cols` >= 8 columns, in two steps.  The load is one wide one whatever c is, of the row's
// last eight columns where the group would reach beyond them; rows may start at any multiple of the element's size
// (unaligned accesses are the processor's).  settle() then moves such a group into its place, with 0 beyond the last
// column: apart from the load, so that all of a row's loads are under way before the first one is waited for.  (With the
// groups at a row's end read one by one and at once, a row of 1601 columns took a workgroup 2.3 us in the backward pass.)
template <Width WIDTH = kAnyWidth, typename T>
__device__ __forceinline__ typename Group<T>::type load_early(const T* row, uint32_t c, uint32_t cols) {
  typename Group<T>::type raw;
  if constexpr (WIDTH == kOneGroup) {
#pragma unroll
    for (uint32_t j = 0; j < kGroup; ++j) raw[j] = c + j < cols ? row[c + j] : static_cast<T>(0.0f);
  } else {
    __builtin_memcpy(&raw, row + (WIDTH == kFullGroups || c < cols - kGroup ? c : cols - kGroup), sizeof(raw));
  }
  return raw;
}
template <typename T>
__device__ __forceinline__ void settle(typename Group<T>::type& raw, uint32_t c, uint32_t cols) {
  if (c + kGroup <= cols) return;
  uint32_t by = c + kGroup - cols;
  forget(by);  // (its comparisons, the same for every row, would be kept in, and spilled from, scalar registers)
  typedef uint32_t Words __attribute__((ext_vector_type(kGroup * sizeof(T) / 4)));
  Words w;
  __builtin_memcpy(&w, &raw, sizeof(w));
  move_down<4, T>(w, by);
  move_down<2, T>(w, by);
  move_down<1, T>(w, by);
#pragma unroll
  for (uint32_t i = 0; i < kGroup * sizeof(T) / 4; ++i) w[i] = by < kGroup ? w[i] : 0u;
  __builtin_memcpy(&raw, &w, sizeof(w));
}
template <Width WIDTH, typename T>
__device__ __forceinline__ void settle_if(typename Group<T>::type& raw, uint32_t c, uint32_t cols) {
  if constexpr (WIDTH == kAnyWidth) settle<T>(raw, c, cols);
  if constexpr (WIDTH == kWholeGroups) {
    typedef uint32_t Words __attribute__((ext_vector_type(kGroup * sizeof(T) / 4)));
    Words w;
    __builtin_memcpy(&w, &raw, sizeof(w));
#pragma unroll
    for (uint32_t i = 0; i < kGroup * sizeof(T) / 4; ++i) w[i] = c < cols ? w[i] : 0u;
    __builtin_memcpy(&raw, &w, sizeof(w));
  }
}
// The same in one, for rows of any width.
template <typename T>
__device__ __forceinline__ typename Group<T>::type load_raw(const T* row, uint32_t c, uint32_t cols) {
  typename Group<T>::type raw;
  if (cols >= kGroup) {
    raw = load_early(row, c, cols);
    settle<T>(raw, c, cols);
  } else {
    raw = load_early<kOneGroup>(row, c, cols);
  }
  return raw;
}
template <typename V>
__device__ __forceinline__ void unpack(float (&v)[kGroup], const V& raw) {
#pragma unroll
  for (uint32_t j = 0; j < kGroup; ++j) v[j] = to_float(raw[j]);
}
template <typename T>
__device__ __forceinline__ void load_group(float (&v)[kGroup], const T* row, uint32_t c, uint32_t cols) {
  unpack(v, load_raw(row, c, cols));
}

// Each value rounded to T once, to the nearest.
template <typename T, Width WIDTH = kAnyWidth>
__device__ __forceinline__ void store_group(T* row, uint32_t c, uint32_t cols, const float (&v)[kGroup]) {
  if (WIDTH == kFullGroups || (WIDTH == kWholeGroups ? c < cols : c + kGroup <= cols)) {
    typename Group<T>::type raw;
#pragma unroll
    for (uint32_t j = 0; j < kGroup; ++j) raw[j] = static_cast<T>(v[j]);
    __builtin_memcpy(row + c, &raw, sizeof(raw));
  } else if (WIDTH != kWholeGroups && c < cols) {  // as four, two and one
    uint32_t left = cols - c;
    forget(left);
    typedef uint32_t Words __attribute__((ext_vector_type(kGroup * sizeof(T) / 4)));
    typename Group<T>::type raw;
#pragma unroll
    for (uint32_t j = 0; j < kGroup; ++j) raw[j] = static_cast<T>(v[j]);
    Words w;
    __builtin_memcpy(&w, &raw, sizeof(raw));
    if (left & 4u) __builtin_memcpy(row + c, &w, 4 * sizeof(T));
    move_down<4, T>(w, left);
    if (left & 2u) __builtin_memcpy(row + c + (left & 4u), &w, 2 * sizeof(T));
    move_down<2, T>(w, left);
    if (left & 1u) __builtin_memcpy(row + c + (left & 6u), &w, sizeof(T));
  }
}

// ---- The generator -------------------------------------------------------------------------------------------
// Philox-4x32 with ten rounds (Salmon, Moraes, Dror, Shaw 2011): w -> (hi(M1 w2) ^ w1 ^ k0, lo(M1 w2), hi(M0 w0) ^ w3 ^ k1,
// lo(M0 w0)), the key stepping by the golden ratio and by sqrt(3) - 1.
__device__ __forceinline__ uint32_t xor3(uint32_t a, uint32_t b, uint32_t c) {
  return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96);
}
__device__ __forceinline__ void philox(uint32_t (&w)[4], uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int turn = 0; turn < 10; ++turn) {
    const uint64_t a = static_cast<uint64_t>(w[0]) * 0xD2511F53u, b = static_cast<uint64_t>(w[2]) * 0xCD9E8D57u;
    w[0] = xor3(static_cast<uint32_t>(b >> 32), w[1], k0);
    w[2] = xor3(static_cast<uint32_t>(a >> 32), w[3], k1);
    w[1] = static_cast<uint32_t>(b);
    w[3] = static_cast<uint32_t>(a);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
}

// What a kernel needs of a compams_drop.  threshold 0 (p < 2^-17) keeps everything and makes no numbers.
struct Drop {
  uint32_t threshold;  // 0 .. 65536
  float scale;
  uint64_t seed, offset;
  const uint64_t* step;
};
inline Drop make_drop(const compams_drop& d) {
  const uint32_t t = static_cast<uint32_t>(d.p * 65536.0 + 0.5);
  return {t, t >= 65536u ? 0.0f : static_cast<float>(65536.0 / (65536.0 - t)), d.seed, d.offset, d.step};
}
inline bool drop_valid(const compams_drop& d) { return d.p >= 0.0 && d.p <= 1.0; }  // (false for a NaN)

// The offset as the kernel sees it.
__device__ __forceinline__ uint64_t drop_offset(const Drop& d) { return d.offset + (d.step ? *d.step : 0u); }

// Dropout of the group of columns c .. c + 7 (c a multiple of 8) of row r.  A dropped entry becomes 0 by selection: its
// value may be anything.
__device__ __forceinline__ void drop_group(float (&v)[kGroup], const Drop& d, uint64_t offset, uint32_t r, uint32_t c) {
  if (d.threshold == 0) return;
  uint32_t w[4] = {c / kGroup, r, static_cast<uint32_t>(offset), static_cast<uint32_t>(offset >> 32)};
  philox(w, static_cast<uint32_t>(d.seed), static_cast<uint32_t>(d.seed >> 32));
#pragma unroll
  for (uint32_t j = 0; j < kGroup; ++j) {
    const uint32_t u = j % 2 ? w[j / 2] >> 16 : w[j / 2] & 0xffffu;
    v[j] = u >= d.threshold ? v[j] * d.scale : 0.0f;
  }
}

// ---- Sums ----------------------------------------------------------------------------------------------------
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __uint_as_float(static_cast<uint32_t>(
      __builtin_amdgcn_update_dpp(0, static_cast<int>(__float_as_uint(v)), CTRL, 0xF, 0xF, true)));
}

// op over each aligned group of `lanes` lanes (8, 16, 32 or 64), the same bits in all of them: data-parallel-primitive
// moves inside a row of 16 lanes, then the two instructions that swap halves between rows.
template <typename Op>
__device__ __forceinline__ float over_lanes(float v, uint32_t lanes, Op op) {
  v = op(v, dpp<0xB1>(v));    // lane ^ 1
  v = op(v, dpp<0x4E>(v));    // lane ^ 2
  v = op(v, dpp<0x141>(v));   // the mirror of each half row
  if (lanes > 8) v = op(v, dpp<0x140>(v));  // the mirror of each row
  if (lanes > 16) {
    const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = op(__uint_as_float(s[0]), __uint_as_float(s[1]));
  }
  if (lanes > 32) {
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = op(__uint_as_float(s[0]), __uint_as_float(s[1]));
  }
  return v;
}
struct Add {
  __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};
__device__ __forceinline__ float sum_lanes(float v, uint32_t lanes) { return over_lanes(v, lanes, Add()); }

// Sums of N numbers over a team of several wavefronts, or of an odd number of half wavefronts (HALVES), the same bits in
// every lane of it: `parts` wavefronts or halves, 16 at most, the team's first being number `first` of the workgroup.  Every
// lane takes one part's sum and they are added across lanes: one read instead of `parts` that wait for each other.  `slots`
// is used again by the next call, so calls that follow each other take two of them in turn: then one barrier is enough (a
// wavefront can be one call ahead of the slowest reader, not two).
constexpr uint32_t kSlots = 32;
template <bool HALVES, int N>
__device__ __forceinline__ void sum_team(float (&v)[N], float (*slots)[kSlots], uint32_t first, uint32_t parts) {
  constexpr uint32_t kLanes = HALVES ? 32 : 64;
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = sum_lanes(v[i], kLanes);
  if (!HALVES && parts == 1) return;
  if (threadIdx.x % kLanes == 0) {
#pragma unroll
    for (int i = 0; i < N; ++i) slots[i][threadIdx.x / kLanes] = v[i];
  }
  __syncthreads();
  const uint32_t mine = threadIdx.x & 15u;
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = sum_lanes(mine < parts ? slots[i][first + mine] : 0.0f, 16);
}
// Over the whole workgroup.
template <int N>
__device__ __forceinline__ void sum_block(float (&v)[N], float (*slots)[kSlots], uint32_t waves) {
  sum_team<false>(v, slots, 0, waves);
}

// ---- Argument checks that the entry points share ---------------------------------------------------------------
inline size_t type_size(int32_t t) { return t == COMPAMS_F32 || t == COMPAMS_I32 ? 4 : t == COMPAMS_I64 ? 8 : 2; }
inline bool float_type(int32_t t) { return t == COMPAMS_F32 || t == COMPAMS_F16 || t == COMPAMS_BF16; }
inline bool aligned_to(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
inline bool rows_valid(int32_t n, int64_t rows, int64_t cols) {
  return n >= 1 && n <= 65535 && rows >= 0 && rows < (static_cast<int64_t>(1) << 31) && cols >= 1 &&
         cols < (static_cast<int64_t>(1) << 31) && static_cast<int64_t>(n) * rows < (static_cast<int64_t>(1) << 31);
}
// A matrix that is there: its stride covers a row, and no offset into it leaves 62 bits.
inline bool stride_valid(int64_t ld, int64_t cols) { return ld >= cols && ld < (static_cast<int64_t>(1) << 31) + 4096; }

}  // namespace compams
