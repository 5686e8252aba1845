// Shared pieces of the kernels around a recurrence (convolution, norms, selective scan): rows of
// fp32 values from 16-bit or 32-bit storage, stretches of packed sequences, sums over partial
// results, host checks.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "deltalog.h"
#include "dl_internal.h"
#include "dl_scan.hpp"

namespace dl {

// ------------------------------------------------------------------ rows
// V consecutive values as they are stored: 2 to 32 bytes, aligned to 16 at most.  Kept as whole words, so
// that a row loaded ahead is not waited for until its values are asked for.
template <int V, typename T>
struct alignas(V * sizeof(T) < 16 ? V * sizeof(T) : 16) Raw {
  uint32_t w[V * sizeof(T) / 4];
  __device__ __forceinline__ float get(int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    else return __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16);
  }
  __device__ __forceinline__ void set(const float (&x)[V]) {
    typedef __attribute__((ext_vector_type(2))) float f32x2;
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
#pragma unroll
    for (int i = 0; i < int(V * sizeof(T) / 4); ++i) {
      if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(x[i]);
      else w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x[2 * i], x[2 * i + 1]}), bf16x2));
    }
  }
};
template <>
struct Raw<1, uint16_t> {
  uint16_t w;
  __device__ __forceinline__ float get(int) const { return widen(w); }
  __device__ __forceinline__ void set(const float (&x)[1]) { narrow(&w, x[0]); }
};
template <int V, typename T>
__device__ __forceinline__ Raw<V, T> load_raw(const T* p) {
  return *reinterpret_cast<const Raw<V, T>*>(p);
}
template <int V, typename T>
__device__ __forceinline__ void widen_row(const Raw<V, T>& r, float (&x)[V]) {
#pragma unroll
  for (int i = 0; i < V; ++i) x[i] = r.get(i);
}
template <int V, typename T>
__device__ __forceinline__ void load_row(const T* p, float (&x)[V]) {
  widen_row(load_raw<V>(p), x);
}
template <int V, typename T>
__device__ __forceinline__ void store_row(T* p, const float (&x)[V]) {
  Raw<V, T> r;
  r.set(x);
  *reinterpret_cast<Raw<V, T>*>(p) = r;
}

// ------------------------------------------------------------------ lanes
template <int CTRL>
__device__ __forceinline__ float from_lane(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
// The sum over aligned groups of N lanes, in all of them: neighbours in a quad, then mirror images
// among 8 and among 16 lanes.  Every lane of a group takes part.
template <int N>
__device__ __forceinline__ float lanes_sum(float x) {
  static_assert(N == 4 || N == 8 || N == 16, "within rows of 16 lanes");
  x += from_lane<0xB1>(x);                    // quad_perm [1,0,3,2]
  x += from_lane<0x4E>(x);                    // quad_perm [2,3,0,1]
  if constexpr (N >= 8) x += from_lane<0x141>(x);   // row_half_mirror
  if constexpr (N >= 16) x += from_lane<0x140>(x);  // row_mirror
  return x;
}
// Two sums over lane pairs, one for each half of the lanes: a(l) + a(l ^ 32) in lanes 0-31 and
// b(l) + b(l ^ 32) in lanes 32-63; a(l) + a(l ^ 16) in even rows of 16 lanes and b's in odd ones;
// a(l) + a(l ^ 8) in the first eight lanes of a row and b's in the last.
__device__ __forceinline__ float halves_sum32(float a, float b) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float halves_sum16(float a, float b) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float halves_sum8(float a, float b) {
  const bool last = threadIdx.x & 8;
  return (last ? b : a) + from_lane<0x128>(last ? a : b);   // row_ror:8
}

constexpr float LOG2E = 1.4426950408889634f;

// What t = x log2 e, as it is rounded, leaves of x: x - t ln 2, to 0.05 2^-24 |x|.  Where that is not a number or
// large (x beyond all exponents) some number up to 1, which finds a factor of 0.
__device__ __forceinline__ float left_of(float x, float t) {
  return __builtin_amdgcn_fmed3f(fmaf(t, -0.69314718f, x), -1.0f, 1.0f);
}

// 1 / (1 + e^-x): 0 and 1 at the infinities.  The exponential's argument is rounded: alone, that is 1.2 2^-24 |x| of
// e^-x, less than a bf16 output's rounding by far, so TO = uint16_t leaves it there (four instructions).  TO =
// float: the derivative s (1 - s) times what the rounding left, and the result is good to (6 + |x| / 16) 2^-24.
template <typename TO>
__device__ __forceinline__ float sigmoid(float x) {
  const float t = x * -LOG2E, s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(t));
  if constexpr (sizeof(TO) == 2) return s;
  return fmaf(-fmaf(-s, s, s), left_of(-x, t), s);
}

// ------------------------------------------------------------------ stretches of sequences
// Sequences are cut into stretches of `len` tokens.  Stretch j of sequence i, whose first token is
// row c_i, has the number c_i / len + i + j: c_{i+1} / len - c_i / len + 1 is at least the number of
// stretches of sequence i and at least 1, so numbers differ, and tokens / len + n are enough.  An
// empty sequence has one stretch without tokens (its state passes through).  Numbers that no
// stretch has are idle.
struct Stretch {
  int seq, slot;
  int first, count;   // token rows
  int seq_first, seq_len;
  bool idle;
  __device__ bool begins() const { return first == seq_first; }
  __device__ bool ends() const { return first + count == seq_first + seq_len; }
};
__host__ __device__ inline int64_t stretches(int64_t n, int64_t tokens, int len) {
  return tokens / len + n;
}

// By all lanes of a wave, for a number that is the same in all of them.  Up to 63 sequences are looked at
// at once, in one trip to memory; more 64 at a time.  Whatever the tables hold, what comes back lies
// within N rows and B slots.
__device__ __forceinline__ Stretch find_stretch(const int32_t* cu, const int32_t* seq_slot, int n,
                                                int N, int B, int len, int f) {
  const int lane = threadIdx.x & 63;
  auto row = [&](int i) { return min(max(cu[i], 0), N); };
  int seq, begin, end, slot;
  if (n < 64) {
    const int c = row(min(lane, n)), at = seq_slot[min(lane, n - 1)];
    const int hits = __popcll(__ballot(lane < n && c / len + lane <= f));
    seq = __builtin_amdgcn_readfirstlane(max(hits - 1, 0));
    begin = __builtin_amdgcn_readlane(c, seq);
    end = __builtin_amdgcn_readlane(c, seq + 1);
    slot = __builtin_amdgcn_readlane(at, seq);
  } else {
    int lo = 0, size = n;
    while (size > 1) {
      const int step = (size + 63) >> 6, i = lo + lane * step;
      const bool at_or_before = lane * step < size && row(i) / len + i <= f;
      const int hits = __popcll(__ballot(at_or_before));
      const int skip = hits > 0 ? (hits - 1) * step : 0;
      lo += skip;
      size = min(step, size - skip);
    }
    seq = lo;
    begin = row(lo);
    end = row(lo + 1);
    slot = seq_slot[lo];
  }
  Stretch s;
  s.seq = __builtin_amdgcn_readfirstlane(seq);
  s.slot = __builtin_amdgcn_readfirstlane(slot);
  s.seq_first = __builtin_amdgcn_readfirstlane(begin);
  s.seq_len = max(__builtin_amdgcn_readfirstlane(end) - s.seq_first, 0);
  // The division is the vector unit's: its result is told to be the same in all lanes, or all that follows
  // from it is taken for a lane's own.
  const int before = __builtin_amdgcn_readfirstlane(s.seq_first / len);
  const int64_t off = int64_t(f - (before + s.seq)) * len;
  s.idle = off < 0 || off > s.seq_len || (off > 0 && off == s.seq_len) || s.slot < 0 || s.slot >= B;
  s.first = s.idle ? 0 : s.seq_first + int(off);
  s.count = s.idle ? 0 : min(len, s.seq_len - int(off));
  return s;
}

// ------------------------------------------------------------------ sums of partial results
// Sums over the rows of part (stride floats apart), whose columns are up to three outputs side by side;
// an output that is null is left out.
struct ColumnSums {
  const float* part;
  int64_t rows, stride;
  float* out[3];
  int64_t width[3];
};
hipError_t launch_column_sums(const ColumnSums& p, hipStream_t s);

// ------------------------------------------------------------------ host
inline bool aligned_to(const void* p, uintptr_t a) {
  return (reinterpret_cast<uintptr_t>(p) % a) == 0;
}
// Up to DL_MAX_STRIDE: offsets of 16 rows fit 32 bits.
inline bool good_stride(int64_t stride, int64_t width) {
  return stride >= width && stride % 8 == 0 && stride <= DL_MAX_STRIDE;
}
inline size_t round256(size_t x) { return (x + 255) & ~size_t(255); }
inline bool grid_fits(int64_t blocks, int threads) {
  return blocks <= 0x7fffffff && blocks * threads <= int64_t(0xffffffff);
}

template <typename K, typename P>
hipError_t start_rows(K* kernel, int64_t grid, int block, const P& p, hipStream_t s) {
  P q = p;
  void* args[] = {&q};
  return hipLaunchKernel(reinterpret_cast<const void*>(kernel), dim3(unsigned(grid)), dim3(block),
                         args, 0, s);
}

inline int check_row_tables(const dl_tables* t) {
  if (!t || !t->cu_tokens || !t->seq_slot) return DL_E_NULL;
  if (!aligned_to(t->cu_tokens, 4) || !aligned_to(t->seq_slot, 4)) return DL_E_ALIGN;
  return DL_OK;
}

}  // namespace dl

#define DL_TRY(x)                 \
  do {                            \
    const int rc_ = (x);          \
    if (rc_ != DL_OK) return rc_; \
  } while (0)
