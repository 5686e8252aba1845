// Shared pieces of the sequence kernels (prefill and its backward pass): fp32 values on the
// matrix cores, the workspace's layout, chunk bookkeeping.
//
// The recurrence of Eq. 3 over a chunk of T = 32 tokens, with l_i the log-decay summed from
// the chunk's start through token i (per key, or the same for all keys; 0 without decay), S
// the state before the chunk, and (x)_i a row of a token matrix:
//
//   Kh_i = k_i e^{l_i}     Qh_i = q_i e^{l_i}     Kb_i = k_i e^{l_T - l_i}
//   G_ij = sum_r k_ir k_jr e^{l_ir - l_jr}  (i > j)
//   P_ij = sum_r q_ir k_jr e^{l_ir - l_jr}  (i >= j)
//   U = V                                        (pair (k, v))
//   U = beta E,  (I + G beta) E = V - Kh S       (delta rule: E = N (V - Kh S))
//   O = Qh S + P U           S <- e^{l_T} S + Kb^T U
//
// RWKV6 reads the state before its token: q_i takes l_{i-1}, and P_ii = sum_r q u k.
// Every exponent that is taken is of a sum of log-decays over a stretch of tokens, so with
// log-decays <= 0 nothing overflows.  log-decays below -104 (e^-104 is 0 in fp32) count as
// -104: a gate of exactly 0 (log -inf) forgets exactly, with no inf - inf.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "deltalog.h"
#include "dl_internal.h"

namespace dl {

constexpr int CT = DL_CHUNK;   // tokens of a chunk

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

// Eight terms of an fp32 operand of fp32 MFMAs, terms 0 to 3 in hi and 4 to 7 in lo.
struct Full {
  f32x4 hi, lo;
};
// Eight terms of an fp32 factor of bf16 keys, queries or output gradients, which are exact in bf16: three
// bf16 numbers each, every one the nearest to what those before it leave.  That is all 24 bits, so the
// products are exact.  Three bf16 MFMAs of 32 terms take 48 cycles, eight fp32 ones 256.  (Two numbers are
// off by up to 2^-17: states then came out 5e-6 from 64 bits instead of 1e-7.)
struct Three {
  bf16x8 a, b, c;
};
// The first two of them, good to 2^-17: for outputs in bf16, which are good to 2^-8.  Of a product of two
// such operands b b is left out, 2^-16 at the most.
struct Pair {
  bf16x8 a, b;
};

__device__ __forceinline__ Full full8(const float* x) {
  return Full{{x[0], x[1], x[2], x[3]}, {x[4], x[5], x[6], x[7]}};
}
// 44 VALU instructions: three conversions a pair, two of them widened again, the differences.
__device__ __forceinline__ Three three8(const float* x) {
  typedef __attribute__((ext_vector_type(2))) float f32x2;
  typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
  u32x4 a, b, c;
  auto narrowed = [](f32x2 v) { return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2)); };
  auto left = [](f32x2 v, uint32_t n) {
    return f32x2{v[0] - __uint_as_float(n << 16), v[1] - __uint_as_float(n & 0xffff0000u)};
  };
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    f32x2 v = {x[2 * e], x[2 * e + 1]};
    a[e] = narrowed(v);
    v = left(v, a[e]);
    b[e] = narrowed(v);
    c[e] = narrowed(left(v, b[e]));
  }
  return Three{__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), __builtin_bit_cast(bf16x8, c)};
}
template <typename OP>
__device__ __forceinline__ OP operand8(const float* x) {
  if constexpr (std::is_same_v<OP, Full>) {
    return full8(x);
  } else {
    const Three t = three8(x);
    if constexpr (std::is_same_v<OP, Pair>) return Pair{t.a, t.b};
    else return t;
  }
}

// acc += a b over 32 terms.  Lane l holds of the 16x16 result rows 4(l/16)+r, column l%16;
// of a row l%16, of b column l%16, and of both the same eight terms: which eight is free as
// long as a and b agree.  With the terms chosen as a lane's own rows of two 16x16 results side
// by side, those results are an operand of the next product without any exchange between lanes.
// Terms that are tokens: 16(e/4)+4(l/16)+e%4, results' rows being tokens in their order ("state
// order").  Terms that are keys: 8(l/16)+e, in their order, with row 4g+r of result f standing
// for key state_key(f, g, r).
__device__ __forceinline__ f32x4 mma(bf16x8 a, bf16x8 b, f32x4 acc) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, acc, 0, 0, 0);
}
// Four terms, one of each lane of a row or column.
__device__ __forceinline__ f32x4 mma(float a, float b, f32x4 acc) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, acc, 0, 0, 0);
}
// acc + low += a b: two sums, so that fewer instructions wait for the one before.
__device__ __forceinline__ void mma(bf16x8 a, const Three& b, f32x4& acc, f32x4& low) {
  low = mma(a, b.c, low);
  acc = mma(a, b.a, acc);
  low = mma(a, b.b, low);
}
__device__ __forceinline__ void mma(const Full& a, const Full& b, f32x4& acc, f32x4& low) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    acc = mma(a.hi[e], b.hi[e], acc);
    low = mma(a.lo[e], b.lo[e], low);
  }
}
// For outputs: without b's last part where they are bf16.
__device__ __forceinline__ void mma_out(bf16x8 a, const Three& b, f32x4& acc, f32x4& low) {
  acc = mma(a, b.a, acc);
  low = mma(a, b.b, low);
}
__device__ __forceinline__ void mma_out(const Pair& a, const Pair& b, f32x4& acc, f32x4& low) {
  low = mma(a.b, b.a, low);
  acc = mma(a.a, b.a, acc);
  low = mma(a.a, b.b, low);
}
__device__ __forceinline__ void mma_out(const Full& a, const Full& b, f32x4& acc, f32x4& low) {
  mma(a, b, acc, low);
}
__device__ __forceinline__ f32x4 mma(bf16x8 a, const Three& b, f32x4 acc) {
  acc = mma(a, b.c, acc);
  acc = mma(a, b.b, acc);
  return mma(a, b.a, acc);
}
__device__ __forceinline__ f32x4 mma(const Full& a, const Full& b, f32x4 acc) {
#pragma unroll
  for (int e = 0; e < 4; ++e) acc = mma(a.hi[e], b.hi[e], acc);
#pragma unroll
  for (int e = 0; e < 4; ++e) acc = mma(a.lo[e], b.lo[e], acc);
  return acc;
}
__host__ __device__ constexpr int state_key(int f, int g, int r) {
  return 32 * (f >> 1) + 8 * g + 4 * (f & 1) + r;
}
__device__ __forceinline__ int state_term(int lane, int e) {
  return 16 * (e >> 2) + 4 * (lane >> 4) + (e & 3);
}

// What a wave's lanes have written to LDS, its other lanes may read: a wave's LDS accesses happen in
// order, so this only keeps the compiler from moving them across.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(uint16_t x) { return __uint_as_float(uint32_t(x) << 16); }
__device__ __forceinline__ void narrow(float* p, float x) { *p = x; }
__device__ __forceinline__ void narrow(uint16_t* p, float x) {
  const __bf16 b = (__bf16)x;             // nearest even
  *p = __builtin_bit_cast(uint16_t, b);
}

// A state or state gradient of either dtype.
__device__ __forceinline__ float load_state(const void* S, bool bf16, int64_t i) {
  return bf16 ? widen(static_cast<const uint16_t*>(S)[i]) : static_cast<const float*>(S)[i];
}
__device__ __forceinline__ void store_state(void* S, bool bf16, int64_t i, float x) {
  if (bf16) narrow(static_cast<uint16_t*>(S) + i, x);
  else static_cast<float*>(S)[i] = x;
}

// ------------------------------------------------------------------ operands in LDS
// A token x key plane: 32 rows of 16-byte pieces (8 bf16; or four fp32, of eight keys the others in the
// same piece of the second half), piece x of row r at piece_at(r, x).  The exchange of pieces within a
// row lets 16 rows of one piece (an operand over keys) and four pieces of four rows (one over tokens)
// each lie in different banks.  NP: pieces in a row.
template <int NP>
__host__ __device__ constexpr int piece_swap(int r) {
  return NP >= 16  ? ((r & 3) << 2) | ((r >> 2) & 3)
         : NP == 8 ? ((r & 2) << 1) | ((r >> 2) & 3)
         : NP == 4 ? (r >> 1) & 2
                   : 0;
}
template <int NP>
__host__ __device__ constexpr int piece_at(int r, int x) {
  return r * NP + (x ^ piece_swap<NP>(r));
}

typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(4))) short s16x4;

__device__ __forceinline__ bf16x8 join(bf16x4 a, bf16x4 b) {
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}
// Four rows of one column: of each 16 lanes, lane i gives the address of four columns of row
// i/4, the (i%4)-th such four, and receives column i of the four rows.
__device__ __forceinline__ bf16x4 read_column(const unsigned char* lds) {
  typedef __attribute__((address_space(3))) s16x4 lds_t;
  return __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t*)lds));
}

// Operands from a plane, exact in bf16 (bf16x8), Full or Pair, its second half `half` bytes on.
// Tokens 16 tt + l%16, terms: keys 32 s + 8 (l/16) + e.
template <typename OP, int NP>
__device__ __forceinline__ OP rows_operand(const unsigned char* plane, int half, int tt, int s, int lane) {
  const unsigned char* at = plane + 16 * piece_at<NP>(16 * tt + (lane & 15), 4 * s + (lane >> 4));
  if constexpr (std::is_same_v<OP, bf16x8>)
    return *reinterpret_cast<const bf16x8*>(at);
  else if constexpr (std::is_same_v<OP, Pair>)
    return Pair{*reinterpret_cast<const bf16x8*>(at), *reinterpret_cast<const bf16x8*>(at + half)};
  else
    return Full{*reinterpret_cast<const f32x4*>(at), *reinterpret_cast<const f32x4*>(at + half)};
}
// Keys state_key(f, ., .) in the place of l%16, terms: the chunk's tokens (state order).
template <typename OP, int NP>
__device__ __forceinline__ OP cols_operand(const unsigned char* plane, int half, int f, int lane) {
  const int i = lane & 15, g = lane >> 4;
  if constexpr (std::is_same_v<OP, bf16x8>) {
    const int r = 4 * g + (i >> 2), x = 4 * (f >> 1) + (i & 3);
    const unsigned char* at = plane + 8 * (f & 1);
    return join(read_column(at + 16 * piece_at<NP>(r, x)), read_column(at + 16 * piece_at<NP>(r + 16, x)));
  } else {
    // Key i is in piece i / 4 of these 32 keys' eight, half f & 1.  Rows 4 g + e and 16 + 4 g + e; their
    // exchange of pieces is g's with e's, so one address serves all e.
    static_assert(NP >= 8 && piece_swap<NP>(4 + 1) == (piece_swap<NP>(4) ^ piece_swap<NP>(1)), "see above");
    const unsigned char* at = plane + half * (f & 1) + 16 * (4 * g * NP + ((i >> 2) ^ g)) + 4 * (i & 3);
    Full o;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int to = 16 * (e * NP + ((4 * (f >> 1)) ^ piece_swap<NP>(e)));
      o.hi[e] = *reinterpret_cast<const float*>(at + to);
      o.lo[e] = *reinterpret_cast<const float*>(at + to + 256 * NP);
    }
    return o;
  }
}

// ------------------------------------------------------------------ workspace
// One block per (chunk, head), chunk-major:
//   planes  Kh, Qh, Kb: token x key, two halves, as they lie in LDS.  Not there ("raw") for
//           bf16 keys and queries with one log-decay per head or none: the keys and queries
//           themselves are the planes, exact in bf16, and e^{l_i} (f) and e^{l_T-l_i} (g)
//           scale token rows of fp32 products instead.
//   squares N (beta N where no backward pass asks for E), P and (backward) P^T, M^T: token x token,
//           two halves, in fragment order: a half of the eight terms (state order) that a lane feeds
//           a product is 16 consecutive bytes.
// The first half lies before the second.  The order makes what one pass reads of a block two runs
// of bytes (a pass without outputs takes neither P nor Qh).
struct WsLayout {
  int dk, dv;
  bool raw, bwd;
  static constexpr int SQ = CT * CT * 2;                                 // one square, one half
  __host__ __device__ int plane() const { return CT * dk * 2; }          // one plane, one half
  __host__ __device__ int p() const { return 0; }
  __host__ __device__ int n() const { return 2 * SQ; }
  __host__ __device__ int kh() const { return 4 * SQ; }
  __host__ __device__ int qh() const { return kh() + (raw ? 0 : 2 * plane()); }
  __host__ __device__ int kb() const { return qh() + (raw ? 0 : 2 * plane()); }
  __host__ __device__ int dec() const { return kb() + (raw ? 0 : 2 * plane()); }  // fp32 [dk] e^{l_T} (not raw)
  __host__ __device__ int beta() const { return dec() + dk * 4; }        // fp32 [CT]
  __host__ __device__ int f() const { return beta() + CT * 4; }          // fp32 [CT] (raw)
  __host__ __device__ int g() const { return f() + CT * 4; }             // fp32 [CT] (raw)
  __host__ __device__ int pt() const { return g() + CT * 4; }
  __host__ __device__ int mt() const { return pt() + 2 * SQ; }
  __host__ __device__ int s0() const { return mt() + 2 * SQ; }           // fp32 S, [dv/16][dk][16]
  __host__ __device__ int ds() const { return s0() + dk * dv * 4; }      // fp32 D, [dv/16][dk][16]
  __host__ __device__ int e() const { return ds() + dk * dv * 4; }       // fp32 [CT][dv]
  __host__ __device__ int z() const { return e() + CT * dv * 4; }        // fp32 Z, [dv/16][CT][16]
  __host__ __device__ int du() const { return z() + CT * dv * 4; }       // fp32 [dk]
  __host__ __device__ int64_t block() const { return bwd ? du() + dk * 4 : pt(); }
};

// Everything the sequence kernels need, passed by value (all pointers are device pointers).
struct SeqParams {
  const void* S_in;      // [B,H,dk,dv] or null (zero states)
  void* S_out;           // [B,H,dk,dv] (backward: gradient of S_in, or null)
  const void* dS_out;    // [B,H,dk,dv] or null (backward: gradient of the final states)
  const void* q;         // [N,H,dk]
  const void* k;         // [N,H,dk]
  const void* v;         // [N,H,dv]
  const void* d_o;       // [N,H,dv] (backward)
  const float* beta;     // [N,H]
  const float* lam;      // [N,H,dl]
  const float* u;        // [H,dk]
  void* o;               // [N,H,dv]
  void *dq, *dk_, *dv_;  // gradients
  float *dbeta, *dlam, *du;
  const int32_t *cu_tokens, *cu_chunks, *chunks, *seq_slot, *order;
  unsigned char* ws;
  float* seg;            // segment states (seg_len > 0)
  int32_t n, N, B, H, dv, max_chunks;
  int32_t seg_len, segs;      // chunks of a segment (0: sequences are walked whole), segments
  bool delta, state_bf16, bwd, raw;
};

// Waves of a workgroup that walks chunks, 16 value columns each.  While there are few waves for
// the 256 CUs, workgroups of two spread them (a wave alone on its SIMD is at its fastest), as
// long as all run at once: with raw operands LDS and registers hold four of them on a CU for 64 keys
// and two for 128; with planes from the workspace two or three for 64 (taken as four: the last ones
// start when the first are done) and one for 128.  Then four waves, then whole heads, which share
// their operands.
inline int walk_waves(int64_t heads, int dk, int dv, bool raw) {
  const int64_t waves = heads * (dv / 16);
  const int64_t two = dk == 64 ? 2048 : raw ? 1024 : 512;   // what workgroups of two keep running
  return waves <= two ? 2 : waves <= 1024 ? 4 : dv / 16;
}

// Long sequences on few heads: the walk is one chain per sequence and head, and most of the chip
// has nothing to do.  The state after a segment of chunks is M S + L, S the state before it; so
// all segments but the last are walked at once for L (from a zero state) and, with the delta
// rule, for M (from the identity, without values: dk more columns), the states between segments
// follow by one product each, and then all segments are walked at once for the outputs.  Without
// the delta rule M is the decay.  That is about 2.3 times the work (1.5 without the delta rule) in
// as many parallel parts as there is room for, and worth it up to 320 waves (then there are three
// parts at least) and from 48 chunks a sequence on average.  Workgroups of four waves.
// Measured, one bf16 sequence, whole call with its tables, whole -> in segments, us: GDN 128 x 128, 8
// heads of 8192 tokens 556 -> 143, 32 of 3200 237 -> 157, 32 of 1536 123 -> 95, 64 of 2048 (512 waves)
// 165 -> 163; KDA, the same, 1055 -> 252, 462 -> 338, 232 -> 169, 347 -> 330; RWKV6 64 x 64, 40 heads of
// 4096 239 -> 131; fp32 GDN 1231 -> 269, 542 -> 363, 263 -> 179.  32 GDN heads of 8192: whole 582; in
// four segments 360, of which 171 for L and M, 14 for the states, 163 for the outputs; in three 379, in
// five 360.
struct SegPlan {
  int len, segs;          // chunks of a segment (0: none), room for segments
};
inline SegPlan seg_plan(int64_t n, int64_t tokens, int64_t H, int dv, bool delta) {
  const int64_t waves = n * H * (dv / 16);
  if (n == 0 || waves > 320) return {0, 0};
  const int64_t avg = tokens / DL_CHUNK / n;
  if (avg < 48) return {0, 0};
  int64_t parts = (delta ? 1024 : 2048) / waves;
  if (parts > 16) parts = 16;
  int64_t len = (avg + parts - 1) / parts;
  if (len < 16) len = 16;
  return {int(len), int((tokens / DL_CHUNK + n) / len + n)};
}
// Floats of one (sequence, segment, head): L (later the segment's first state) and M.
__host__ __device__ inline int64_t seg_floats(int dk, int dv, bool delta) {
  return int64_t(dk) * (dv + (delta ? dk : 0));
}

struct ChunkRow {
  int seq, first, count, slot;
};
// The chunk's row of the tables, or a count of 0 where there is nothing to do: no such
// chunk, or a slot or token range that does not fit the buffers of this call.
__device__ __forceinline__ ChunkRow chunk_row(const SeqParams& p, int c) {
  const int32_t* t = p.chunks + 4 * int64_t(c);
  ChunkRow r{t[0], t[1], t[2], t[3]};
  const bool ok = r.seq >= 0 && r.seq < p.n && r.slot >= 0 && r.slot < p.B && r.first >= 0 &&
                  r.count > 0 && r.count <= CT && r.first <= p.N - r.count;
  if (!ok) r.count = 0;
  return r;
}

}  // namespace dl
