// Products of matrices on the matrix cores, one tile of the result to a workgroup: D(m, n) = sum over k of A(m, k) B(n, k),
// with fp32 sums.  The kernels that use it differ in what they do with the tile.  (wave64 only)
//
// A step takes 128 bytes of k, 64 entries of the 16-bit types, 32 of fp32 (or half as many).  Both operands' tiles of a step
// go from memory into LDS without passing through registers, 16 bytes a lane, while the step before is multiplied (two
// buffers, one barrier a step).  Reads beyond a matrix give zeros (the buffer descriptors' own bounds), and what rows along k
// have behind their last entry in the same 16 bytes is overwritten with zeros in LDS, so no length has to be a multiple of
// anything; rows have to start on 16 bytes.
#pragma once

#include <initializer_list>

#include "compams_areas.h"
#include "compams_rows.h"

namespace compams {

// How an operand lies in memory: its rows go along k (entries of a row follow one another in k), or across it (a row has
// one k, and all m or n).
enum Form { kAlong, kAcross };


typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char lds_char;

// A lane's 16 bytes of an operand, as one instruction (four of fp32) takes them: row or column l % 16 of sixteen, and of k
// eight entries from 8 (l / 16) on (fp32: four from 4 (l / 16) on, one to an instruction).
template <typename T>
struct Fragment {
  typedef T type __attribute__((ext_vector_type(16 / sizeof(T))));
};

// d(n, m) += sum of b(n, k) a(m, k).  The rows of the instruction are n: a lane gets m = l % 16 and the four neighbouring
// n from 4 (l / 16) on, which lie next to one another in a row of the result.
__device__ __forceinline__ void multiply(f32x4& d, Fragment<half_t>::type a, Fragment<half_t>::type b) {
  d = __builtin_amdgcn_mfma_f32_16x16x32_f16(b, a, d, 0, 0, 0);
}
__device__ __forceinline__ void multiply(f32x4& d, Fragment<bfloat_t>::type a, Fragment<bfloat_t>::type b) {
  d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, a, d, 0, 0, 0);
}
__device__ __forceinline__ void multiply(f32x4& d, Fragment<float>::type a, Fragment<float>::type b) {
#pragma unroll
  for (int i = 0; i < 4; ++i) d = __builtin_amdgcn_mfma_f32_16x16x4f32(b[i], a[i], d, 0, 0, 0);
}

// Places in LDS.  An operand's tile has EXTENT rows (or columns) of m or n.
//
// kAlong: EXTENT rows of STEP bytes.  The 16 bytes c of row r are kept at place c ^ (r % 8) of the row: the sixteen rows that a
// fragment is read from then begin in eight different places of the 128 bytes that LDS gives at once.
//
// kAcross: a row of EXTENT entries for every k of the step. 16-bit types are read with the transposing read: sixteen lanes
// read four k of sixteen columns (32 bytes a row), and get four k of one column each.  The pairs of 16 bytes are moved by k so
// that the rows of a read do not meet. fp32 is read entry by entry, 64 bytes a row.
template <typename T, uint32_t EXTENT>
__device__ __forceinline__ uint32_t moved(uint32_t k) {
  if constexpr (sizeof(T) == 2) return 2 * ((k & 3u) | (EXTENT >= 128 ? (k >> 1) & 4u : 0u));
  else return (k >> 2 & 3u) * 4;
}

template <typename T, Form F, uint32_t EXTENT, uint32_t STEP>
struct Place {
  static constexpr uint32_t kRowBytes = F == kAlong ? STEP : EXTENT * sizeof(T);
  static constexpr uint32_t kPerRow = kRowBytes / 16;  // 16-byte pieces
  static constexpr uint32_t kBytes = EXTENT * STEP;

  // kAlong: what a piece's number is changed by in row `row`.
  __device__ static __forceinline__ uint32_t turned(uint32_t row) { return STEP == 128 ? row & 7u : row >> 1 & 3u; }

  // kAlong: zeros behind the first `keep` of the step's entries, as far as those 16 bytes go (a multiple: nothing).
  __device__ static __forceinline__ void cut(lds_char* tile, uint32_t keep, uint32_t threads) {
    constexpr uint32_t kEach = 16 / sizeof(T);
    for (uint32_t row = threadIdx.x; row < EXTENT; row += threads) {
      typedef __attribute__((address_space(3))) typename Fragment<T>::type Kept;
      Kept* const at = reinterpret_cast<Kept*>(tile + row * kRowBytes + (keep / kEach ^ turned(row)) * 16);
      typename Fragment<T>::type v = *at;
#pragma unroll
      for (uint32_t j = 1; j < kEach; ++j) v[j] = j < keep % kEach ? v[j] : T(0);
      *at = v;
    }
  }

  // The row and the piece of it that is kept at 16-byte place p.
  __device__ static __forceinline__ void of(uint32_t p, uint32_t& row, uint32_t& piece) {
    row = p / kPerRow;
    piece = p % kPerRow ^ (F == kAlong ? turned(row) : moved<T, EXTENT>(row));
  }

  // The fragment of rows (columns) first .. first + 15 and the sub-th 64 bytes of the step's k.
  __device__ static __forceinline__ typename Fragment<T>::type read(const lds_char* tile, uint32_t first, uint32_t sub) {
    const uint32_t lane = threadIdx.x & 63u, l = lane & 15u, g = lane >> 4;
    typename Fragment<T>::type v;
    if constexpr (F == kAlong) {
      const uint32_t row = first + l, piece = (sub * 4 + g) ^ turned(row);
      v = *reinterpret_cast<const __attribute__((address_space(3))) typename Fragment<T>::type*>(tile + row * kRowBytes +
                                                                                                 piece * 16);
    } else if constexpr (sizeof(T) == 2) {
      const uint32_t k = sub * 32 + g * 8 + (l >> 2);
      const uint32_t piece = first / 8 + (l >> 1 & 1u), in = (l & 1u) * 8;
      s16x4 part[2];
#pragma unroll
      for (uint32_t h = 0; h < 2; ++h)  // (k and k + 4 are moved alike)
        part[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(
            tile + (k + 4 * h) * kRowBytes + (piece ^ moved<T, EXTENT>(k)) * 16 + in));
      __builtin_memcpy(&v, part, sizeof(v));
    } else {
      const uint32_t column = first + l;
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i) {
        const uint32_t k = sub * 16 + g * 4 + i;
        v[i] = *reinterpret_cast<const __attribute__((address_space(3))) float*>(
            tile + k * kRowBytes + (column / 4 ^ moved<T, EXTENT>(k)) * 16 + column % 4 * 4);
      }
    }
    return v;
  }
};

// An operand, from the tile's first row or column on: its bytes' bounds go with it.
struct Side {
  const char* p;
  uint32_t ld;      // bytes from row to row
  uint32_t extent;  // kAlong: rows from the tile's first on; kAcross: bytes of a row from the tile's first column on
  uint32_t k;       // entries of k
};
template <typename T, Form F>
__device__ __forceinline__ Side side(const void* p, int64_t ld, uint32_t total, uint32_t first, uint32_t k) {
  const char* const at = static_cast<const char*>(p);
  if (F == kAlong) return {at + static_cast<int64_t>(first) * ld, static_cast<uint32_t>(ld), total - first, k};
  return {at + static_cast<int64_t>(first) * sizeof(T), static_cast<uint32_t>(ld),
          (total - first) * static_cast<uint32_t>(sizeof(T)), k};
}

template <typename T, Form F, uint32_t EXTENT, uint32_t WAVES, uint32_t STEP>
struct Loader {
  using At = Place<T, F, EXTENT, STEP>;
  static constexpr uint32_t kRows = 1024 / STEP;  // kAlong: rows of an instruction
  static constexpr uint32_t kLoads = At::kBytes / (WAVES * 1024);
  static_assert(kLoads * WAVES * 1024 == At::kBytes, "a tile is loaded in whole instructions of every wave");
  uint32_t row[kLoads], piece[kLoads];

  __device__ __forceinline__ void init(uint32_t wave) {
    const uint32_t lane = threadIdx.x & 63u;
#pragma unroll
    for (uint32_t i = 0; i < kLoads; ++i) At::of((i * WAVES + wave) * 64 + lane, row[i], piece[i]);
  }
  // TWO: the tile's rows are those of two operands in turns of sixteen.
  template <bool TWO>
  __device__ __forceinline__ void load(const Side& one, const Side& two, uint32_t k0, lds_char* tile, uint32_t wave) const {
    const __amdgpu_buffer_rsrc_t of_one = bounds(one, k0, TWO);
    const __amdgpu_buffer_rsrc_t of_two = TWO ? bounds(two, k0, TWO) : of_one;
    const uint32_t left = (one.k - k0) * static_cast<uint32_t>(sizeof(T));
#pragma unroll
    for (uint32_t i = 0; i < kLoads; ++i) {
      uint32_t r = row[i], ld = one.ld;
      bool second = false;
      if constexpr (TWO) {
        second = ((i * WAVES + wave) * kRows / 16) & 1u;  // (the same for the wave: an instruction has eight or sixteen rows)
        r = r / 32 * 16 + r % 16;
        ld = second ? two.ld : one.ld;
      }
      uint32_t at = r * ld + piece[i] * 16;
      if constexpr (F == kAlong) at = piece[i] * 16 < left ? at : 0x80000000u;  // (the entries behind a row's end are another's)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          second ? of_two : of_one, (__attribute__((address_space(3))) void*)(tile + (i * WAVES + wave) * 1024), 16, at, 0, 0, 0);
    }
  }
  // Up to the end of the last row's last word: an entry of 16 bits that ends it in the middle of one would be cut off with it.
  __device__ static __forceinline__ uint32_t whole(uint32_t bytes) { return (bytes + 3) / 4 * 4; }
  __device__ static __forceinline__ __amdgpu_buffer_rsrc_t bounds(const Side& s, uint32_t k0, bool two) {
    const char* p;
    uint32_t bytes;
    if constexpr (F == kAlong) {
      const uint32_t rows = min(s.extent, two ? EXTENT / 2 : EXTENT);
      p = s.p + k0 * sizeof(T);
      bytes = (rows - 1) * s.ld + whole((s.k - k0) * static_cast<uint32_t>(sizeof(T)));
    } else {
      const uint32_t rows = min(s.k - k0, STEP / static_cast<uint32_t>(sizeof(T)));
      p = s.p + static_cast<int64_t>(k0) * s.ld;
      bytes = (rows - 1) * s.ld + whole(s.extent);
    }
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(p), 0, static_cast<int>(bytes), 0x00020000);
  }
};

// The two buffers of a workgroup's tiles.
struct TileLds {
  lds_char *a[2], *b[2];
};

// A workgroup of WM x WN wavefronts, each with FM x FN tiles of 16 x 16.
template <typename T_, Form FA_, Form FB_, uint32_t WM_, uint32_t WN_, uint32_t FM_, uint32_t FN_, bool TWO_ = false,
          uint32_t STEP_ = 128>
struct Tiles {
  static constexpr uint32_t STEP = STEP_, kStep = STEP_ / sizeof(T_);  // of k, in bytes and in entries
  using T = T_;
  static constexpr Form FA = FA_, FB = FB_;
  static constexpr uint32_t WM = WM_, WN = WN_, FM = FM_, FN = FN_;
  static constexpr bool kTwo = TWO_;  // B is two matrices, in turns of sixteen columns of the result
  static constexpr uint32_t kWaves = WM * WN, kThreads = kWaves * 64, kM = WM * FM * 16, kN = WN * FN * 16;
  using PlaceA = Place<T, FA, kM, STEP>;
  using PlaceB = Place<T, FB, kN, STEP>;
  static constexpr uint32_t kBytesA = PlaceA::kBytes, kBytesB = PlaceB::kBytes;
  // fp32 sums are formed in two levels, 64 terms and then these: they are off by the roundings of so many, not of all of them
  // (dweight of 16000 random rows by 0.4e-6 of itself, in a row 2.3e-6).  It costs 2 to 4 % (8192 x 768 x 2048 gated forward 401 ->
  // 414 us, projections' gradients 789 -> 804; 128 terms at a time, as a branch in the loop, take half as many registers again:
  // 462), and tiles of 256, which are no faster in fp32.  Of 16-bit operands the sums stay in a row: most are rounded to 16 bits.
  static constexpr bool kLevels = sizeof(T_) == 4;
  f32x4 sum[FM][FN], whole[kLevels ? FM : 1][kLevels ? FN : 1];

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (uint32_t i = 0; i < FM; ++i)
#pragma unroll
      for (uint32_t j = 0; j < FN; ++j) sum[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  __device__ static __forceinline__ uint32_t wave() { return __builtin_amdgcn_readfirstlane(threadIdx.x / 64); }
  // The first row and column, in the tile, of a wavefront's part, and of a lane's entries in a tile of 16 x 16.
  __device__ static __forceinline__ uint32_t first_m() { return wave() / WN * (FM * 16); }
  __device__ static __forceinline__ uint32_t first_n() { return wave() % WN * (FN * 16); }
  __device__ static __forceinline__ uint32_t lane_m() { return threadIdx.x & 15u; }
  __device__ static __forceinline__ uint32_t lane_n() { return (threadIdx.x >> 4 & 3u) * 4; }

  // The sums of some steps join those before.  (first: what is there is what the steps' are to join)
  __device__ __forceinline__ void join(bool first = false) {
    if constexpr (kLevels) {
#pragma unroll
      for (uint32_t i = 0; i < FM; ++i)
#pragma unroll
        for (uint32_t j = 0; j < FN; ++j) {
          whole[i][j] = first ? sum[i][j] : whole[i][j] + sum[i][j];
          sum[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
    }
  }
  __device__ __forceinline__ void joined() {
    if constexpr (kLevels) {
#pragma unroll
      for (uint32_t i = 0; i < FM; ++i)
#pragma unroll
        for (uint32_t j = 0; j < FN; ++j) sum[i][j] += whole[i][j];
    }
  }

  __device__ __forceinline__ void step(const lds_char* a, const lds_char* b) {
    const uint32_t m = first_m(), n = first_n();
#pragma unroll
    for (uint32_t sub = 0; sub < STEP / 64; ++sub) {
      typename Fragment<T>::type fa[FM], fb[FN];
#pragma unroll
      for (uint32_t j = 0; j < FN; ++j) fb[j] = PlaceB::read(b, n + j * 16, sub);
#pragma unroll
      for (uint32_t i = 0; i < FM; ++i) fa[i] = PlaceA::read(a, m + i * 16, sub);
#pragma unroll
      for (uint32_t i = 0; i < FM; ++i)
#pragma unroll
        for (uint32_t j = 0; j < FN; ++j) multiply(sum[i][j], fa[i], fb[j]);
      __builtin_amdgcn_sched_barrier(0);  // (else the fragments of both halves are read at once, and registers spilled)
    }
  }

  // sum += the products of `count` pairs of operands, all with the same k.  pair(i, a, b, b2) gives the i-th; one or two. CUT: rows
  // along k may have something other than zeros behind their last entry.
  template <bool CUT = true, typename Pair>
  __device__ __forceinline__ void run(Pair pair, uint32_t count, uint32_t k, const TileLds& lds) {
    const uint32_t w = wave();
    Loader<T, FA, kM, kWaves, STEP> la;
    Loader<T, FB, kN, kWaves, STEP> lb;
    la.init(w);
    lb.init(w);
    const uint32_t steps = (k + kStep - 1) / kStep * count;
    if (steps == 0) return;
    uint32_t at = 0, k0 = 0;
    Side a, b, b2;
    pair(0u, a, b, b2);
    const auto load = [&](lds_char* ta, lds_char* tb) {
      la.template load<false>(a, a, k0, ta, w);
      lb.template load<kTwo>(b, b2, k0, tb, w);
      k0 += kStep;
      if (k0 >= k) {
        k0 = 0;
        if (++at < count) pair(at, a, b, b2);
      }
    };
    join(true);
    load(lds.a[0], lds.b[0]);
    if constexpr (CUT && (FA == kAlong || FB == kAlong)) {
      // The last step of a pair whose rows end within 16 bytes: what follows there may be anything, a NaN too.
      const auto cut = [&](lds_char* ta, lds_char* tb) {
        if (k % (16 / sizeof(T)) == 0) return;
        if constexpr (FA == kAlong) PlaceA::cut(ta, k % kStep, kThreads);
        if constexpr (FB == kAlong) PlaceB::cut(tb, k % kStep, kThreads);
        __syncthreads();
      };
      const auto first_ends = [&](uint32_t s) { return count == 2 && 2 * s == steps; };
      // (the last step stands apart, in one place for both buffers: registers are spilled with its cut in the loop, 8192 x
      // 50257 x 768 first pass 628 -> 725 us, and far more with a copy of the step for each buffer)
      uint32_t s = 1;
      for (; s + 1 < steps; s += 2) {
        arrived();
        load(lds.a[1], lds.b[1]);
        if (first_ends(s)) cut(lds.a[0], lds.b[0]);
        step(lds.a[0], lds.b[0]);
        arrived();
        load(lds.a[0], lds.b[0]);
        if (first_ends(s + 1)) cut(lds.a[1], lds.b[1]);
        step(lds.a[1], lds.b[1]);
        join();
      }
      arrived();
      lds_char *ta = lds.a[0], *tb = lds.b[0];
      if (s < steps) {
        load(lds.a[1], lds.b[1]);
        if (first_ends(s)) cut(ta, tb);
        step(ta, tb);
        arrived();
        ta = lds.a[1];
        tb = lds.b[1];
      }
      cut(ta, tb);
      step(ta, tb);
    } else {
      for (uint32_t s = 2; s <= steps; s += 2) {
        arrived();
        load(lds.a[1], lds.b[1]);
        step(lds.a[0], lds.b[0]);
        arrived();
        if (s < steps) load(lds.a[0], lds.b[0]);
        step(lds.a[1], lds.b[1]);
        join();
      }
      if (steps & 1u) {
        arrived();
        step(lds.a[0], lds.b[0]);
      }
    }
    joined();
  }
  // What this wavefront loaded is in LDS, and so is everybody's; everybody is done with the step before.
  __device__ static __forceinline__ void arrived() {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  }
  // visit(row, column, four neighbouring entries) of the tile, as the matrix cores leave them: 64 bytes of each of sixteen
  // rows at a time.
  template <typename Visit>
  __device__ __forceinline__ void each(Visit visit) {
    const uint32_t m = first_m() + lane_m(), n = first_n() + lane_n();
#pragma unroll
    for (uint32_t i = 0; i < FM; ++i)
#pragma unroll
      for (uint32_t j = 0; j < FN; ++j) visit(m + i * 16, n + j * 16, sum[i][j]);
  }

  // The same by way of LDS, a row's entries in neighbouring lanes, for what is stored: a wavefront's part of a row goes to
  // memory at once (8192 x 8192 fp32 stored and nothing else: 54 us, in pieces of 64 bytes 69).  Each wavefront has room for
  // sixteen of its rows in `lds`; piece c of row r is at place c ^ r. of(i, j): what is to be stored of the i, j-th tile of 16
  // x 16, PIECES / 4 of them side by side.
  template <uint32_t PIECES, typename Of, typename Visit>
  __device__ __forceinline__ void rows_of(lds_char* lds, Of of, Visit visit) {
    static_assert(16 * PIECES * 16 * kWaves <= kBytesA, "sixteen rows of every wavefront");
    const uint32_t lane = threadIdx.x & 63u, m = lane_m();
    lds_char* const mine = lds + wave() * (16 * PIECES * 16);
    const uint32_t c = lane % PIECES;
    const auto at = [](lds_char* from, uint32_t row, uint32_t piece) {
      return reinterpret_cast<__attribute__((address_space(3))) f32x4*>(from + (row * PIECES + (piece ^ (row & (PIECES - 1)))) * 16);
    };
#pragma unroll
    for (uint32_t i = 0; i < FM; ++i) {
      settled();
#pragma unroll
      for (uint32_t j = 0; j < PIECES / 4; ++j)
        *at(mine, m, j * 4 + lane / 16) = of(i, j);
      settled();
#pragma unroll
      for (uint32_t q = 0; q < 16 * PIECES / 64; ++q) {
        const uint32_t r = q * (64 / PIECES) + lane / PIECES;
        const f32x4 v = *at(mine, r, c);
        visit(first_m() + i * 16 + r, c * 4, v);
      }
    }
  }
  template <typename Visit>
  __device__ __forceinline__ void rows(lds_char* lds, Visit visit) {
    __syncthreads();  // (others may still read what they multiply)
    const uint32_t n = first_n();
    rows_of<FN * 4>(lds, [&](uint32_t i, uint32_t j) { return sum[i][j]; },
                    [&](uint32_t r, uint32_t c, const f32x4& v) { visit(r, n + c, v); });
  }
  // The first of a lane's columns there, which are the same in every row.
  __device__ static __forceinline__ uint32_t row_n() { return first_n() + (threadIdx.x & 63u) % (FN * 4) * 4; }
  // A wavefront's accesses of LDS before this come before those after it.
  __device__ static __forceinline__ void settled() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
};

// (Four arrays of their own: the compiler then knows that what is read is not what is being loaded.)
#define COMPAMS_TILE_LDS(TILES, NAME)                                                                                         \
  __shared__ __attribute__((aligned(1024))) char lds_a0[TILES::kBytesA], lds_b0[TILES::kBytesB], lds_a1[TILES::kBytesA],       \
      lds_b1[TILES::kBytesB];                                                                                                \
  const compams::TileLds NAME = {{(compams::lds_char*)lds_a0, (compams::lds_char*)lds_a1},                                     \
                                 {(compams::lds_char*)lds_b0, (compams::lds_char*)lds_b1}}

// Workgroups go to the eight dies in turn, each with a cache of its own: a die gets workgroups that follow one another.
__device__ __forceinline__ uint32_t by_die(uint32_t id, uint32_t total) {
  const uint32_t die = id % 8, in = id / 8, each = total / 8, more = total % 8;
  return die * each + min(die, more) + in;
}

// Four neighbouring entries of a row, each rounded to T once; `left` entries of the row from the first on are there.  (Rows
// may start at any multiple of an entry's size: unaligned accesses are the processor's.)
template <typename T>
__device__ __forceinline__ void store4(T* p, const f32x4& v, int64_t left) {
  typedef T T4 __attribute__((ext_vector_type(4)));
  T4 t;
#pragma unroll
  for (int i = 0; i < 4; ++i) t[i] = static_cast<T>(v[i]);
  if (left >= 4) {
    __builtin_memcpy(p, &t, sizeof(t));
  } else {
#pragma unroll
    for (int i = 0; i < 3; ++i)
      if (i < left) p[i] = t[i];
  }
}
// The same of a weight's gradient: written, or added to what is there.
__device__ __forceinline__ void add4(float* p, f32x4 v, int64_t left, bool accumulate) {
  if (accumulate) {
    f32x4 before = {};
    if (left >= 4) {
      __builtin_memcpy(&before, p, sizeof(before));
    } else {
#pragma unroll
      for (int i = 0; i < 3; ++i)
        if (i < left) before[i] = p[i];
    }
    v += before;
  }
  store4(p, v, left);
}

// ---- Host side -----------------------------------------------------------------------------------------------

// Longest row of a product's operand, in entries: offsets within a tile of 256 rows are 31 bits.
constexpr int64_t kMostEntries = 1 << 20;
constexpr int64_t kMostRowBytes = 1 << 23;

// A matrix as a caller has it, and as the product kernels read it: rows that start on 16 bytes.  What is not like that is
// copied into the workspace first, with zeros behind the rows (`packed`).
struct Matrix {
  const void* p;
  int64_t ld;  // entries
  int64_t rows, cols;
  size_t size;  // bytes of an entry
  bool as_is() const {
    return aligned_to(p, 16) && (rows <= 1 || (ld * size % 16 == 0 && ld * static_cast<int64_t>(size) <= kMostRowBytes));
  }
  int64_t packed_row_bytes() const { return (cols * static_cast<int64_t>(size) + 15) / 16 * 16; }
  size_t packed_bytes() const { return as_is() ? 0 : (static_cast<size_t>(rows) * packed_row_bytes() + 255) / 256 * 256; }
};
struct Read {  // what a kernel gets
  const void* p;
  int64_t ld;  // bytes
};
constexpr uint32_t kMostPacked = 4;
struct Packing {
  uint32_t count = 0;
  struct Job {
    const void* from;
    void* to;
    int64_t ld;  // entries
    int64_t rows;
    uint32_t per_row, cols;  // pieces of 16 bytes, entries
  } job[kMostPacked];
  // How the kernels are to read `m`; moves `workspace` on by what it takes of it.
  Read add(const Matrix& m, char*& workspace) {
    if (m.as_is()) return {m.p, m.rows <= 1 ? m.packed_row_bytes() : m.ld * static_cast<int64_t>(m.size)};
    const Read r = {workspace, m.packed_row_bytes()};
    const uint32_t per_row = static_cast<uint32_t>(m.packed_row_bytes() / 16);
    job[count++] = {m.p, workspace, m.ld, m.rows, per_row, static_cast<uint32_t>(m.cols)};
    workspace += m.packed_bytes();
    return r;
  }
};
// Enqueues the copies (one launch, or none).
void run_packing(const Packing& p, size_t size, hipStream_t stream);

// Tiles as workgroups: a dimension has room for 2^32 threads.
constexpr uint32_t kGridX = 1u << 21;
inline dim3 tile_grid(uint64_t tiles) {
  return dim3(static_cast<uint32_t>(tiles < kGridX ? tiles : kGridX), static_cast<uint32_t>((tiles + kGridX - 1) / kGridX));
}
__device__ __forceinline__ uint32_t tile_id() { return blockIdx.y * kGridX + blockIdx.x; }

// Tile number `id` of a result of tall x wide tiles: strips of eight tiles down, within them column after column, so that the
// workgroups of a die share rows of both operands in its cache.
__device__ __forceinline__ void tile_at(uint32_t id, uint32_t tall, uint32_t wide, uint32_t& down, uint32_t& across) {
  const uint32_t strip = id / (8 * wide), in = id - strip * 8 * wide, height = min(8u, tall - strip * 8);
  down = strip * 8 + in % height;
  across = in / height;
}

// Which size of tile the results of a launch are made with, each of them `many` matrices of rows x cols with `k` terms in a
// sum.  The larger a tile, the higher its rate; but the compute units' shares of few large tiles are uneven, and a tile alone
// on a compute unit has nothing beside it while it loads.  Rates of a full card, and of one tile to a compute unit, relative
// to the first (8192 x 8192 x 768 bfloat16, TFLOP/s: 256 x 256 1340, 128 x 128 1130, 64 x 64 770; alone, 1024 x 1024 x 2048
// and the like: 1100, 800, 375. fp32, where the matrix cores bound every size, 128 x 128 133, 64 x 64 130, alone 100).  Launches of
// more than one kind of result take 256 x 128 in steps of 64 bytes for the largest, of which two and three workgroups share a
// compute unit: one stores while another multiplies (8 x 1024 x 768 x 2048 projections' gradients 115 us, with 128 x 128 123).
enum TileSize { kTile256, kTile128, kTile64 };
struct Work {
  uint64_t rows, cols, many, k;
};
inline TileSize tile_size(std::initializer_list<Work> all, bool wide_type) {
  const auto cost = [&](uint64_t edge, uint64_t across, double full, double alone, double apiece) {
    double sum = 0.0, longest = 0.0;
    uint64_t tiles = 0;
    for (const Work& w : all) {
      const uint64_t count = (w.rows + edge - 1) / edge * ((w.cols + across - 1) / across) * w.many;
      if (count == 0 || w.k == 0) continue;
      const double one = static_cast<double>(edge * across) * static_cast<double>(w.k) + apiece;
      tiles += count;
      sum += static_cast<double>(count) * one;
      longest = one > longest ? one : longest;
    }
    // whole tiles to a compute unit
    const double share = tiles ? sum / static_cast<double>(tiles) * static_cast<double>((tiles + 255) / 256) : 0.0;
    return (share / full > longest / alone) ? share / full : longest / alone;
  };
  // (the last: what a tile takes besides its products, some 2 us to load the first step and to store, as far as the others on
  // its compute unit do not hide it: 180 x 3818 x 29084 bfloat16, sums of 90 terms in 54000 tiles of 64 x 64, 564 us)
  const double large = all.size() > 1 ? cost(256, 128, 0.97, 0.6, 2.6e6) : cost(256, 256, 1.0, 0.97, 6e6);
  const double middle = wide_type ? cost(128, 128, 1.0, 0.9, 0.4e6) : cost(128, 128, 0.84, 0.6, 2.6e6);
  const double small = wide_type ? cost(64, 64, 0.97, 0.75, 0.15e6) : cost(64, 64, 0.57, 0.28, 1e6);
  if (!wide_type && large <= middle && large <= small) return kTile256;  // (fp32's two levels of sums fill the registers before)
  return middle <= small ? kTile128 : kTile64;
}
// Into how many parts the k of a result is cut whose tiles are too few for the card, each part with 1024 terms and more (fp32,
// whose products take longer: 512): their sums are joined afterwards.  (us of dx behind two projections, rows x cols x hidden; fp32
// with 256, 512 and 1024 terms at least: 2048 x 256 x 768 27, 28, 38; 64 x 256 x 1024 14, 18, 29; 512 x 512 x 2048 37, 30, 31;
// 300 x 768 x 2304 40, 37, 35.  bfloat16 with 512 and 1024: 13.1 and 11.5, 12.6 and 13.0, 15.3 and 13.5, 16.4 and 14.3.)
inline uint32_t splits_of(uint64_t rows, uint64_t cols, uint64_t k, bool wide_type) {
  const uint64_t tiles = (rows + 63) / 64 * ((cols + 63) / 64), most = k / (wide_type ? 512 : 1024);
  uint64_t splits = tiles ? 1024 / tiles : 1;
  if (splits > most) splits = most;
  return static_cast<uint32_t>(splits > 16 ? 16 : splits > 1 ? splits : 1);
}
inline uint64_t tiles_of(uint64_t count, uint32_t edge) { return (count + edge - 1) / edge; }

// Lanes side by side of a workgroup that goes down the columns of a matrix of `groups` groups of eight: up to a wavefront's width, and
// as many as leave few of them without a column (72 groups, 8290 rows of float16: 64 lanes 33.0 us, 8 lanes 25.8).
inline uint32_t lanes_across(uint64_t groups) {
  uint32_t best = 64;
  uint64_t least = ~0ull;
  for (uint32_t wide = 64; wide >= 8; wide /= 2) {
    const uint64_t lanes = (groups + wide - 1) / wide * wide;
    if (lanes + lanes / 16 < least) {
      least = lanes;
      best = wide;
    }
  }
  while (best > 1 && best / 2 >= groups) best /= 2;
  return best;
}
// A weight's gradients, a matrix for each of n workers.
inline bool gradient_valid(int32_t n, int64_t rows, int64_t cols, int64_t ld, int64_t stride) {
  constexpr int64_t kMost = static_cast<int64_t>(1) << 40;
  return (rows <= 1 || (ld >= cols && ld < kMost)) && (n <= 1 || (stride >= 0 && stride < kMost && stride >= cols));
}
// Whether the tiles of a result can be numbered, `many` results of 64 x 64 tiles.
inline bool tiles_fit(int64_t rows, int64_t cols, int64_t many) {
  return static_cast<double>((rows + 63) / 64) * static_cast<double>((cols + 63) / 64) * static_cast<double>(many) < 2147483648.0;
}
inline int workspace_status(const void* p, size_t bytes, size_t need) {
  if (need == 0) return COMPAMS_OK;
  if (!p) return COMPAMS_INVALID_ARG;
  if (!aligned_to(p, 256)) return COMPAMS_BAD_ALIGNMENT;
  return bytes < need ? COMPAMS_WORKSPACE_TOO_SMALL : COMPAMS_OK;
}

}  // namespace compams
