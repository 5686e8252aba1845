// The serial passes over a sequence's chunks: forward (states and outputs) and backward
// (state gradients and value gradients).
//
// A workgroup of NW waves walks the chunks of one (sequence, head); each wave owns NT tiles of
// 16 value columns and keeps its dk x 16 NT piece of the state (or of the state's gradient) in
// registers as MFMA results.  Columns never meet, so the waves share nothing but the chunk's
// operands, which go through LDS: each chunk's are loaded into registers while the chunk before
// is computed, and written to LDS between two barriers.  Inside a chunk every product's result
// is the next product's operand as it stands (state order), without a trip through LDS.
#pragma once

#include "dl_scan.hpp"

namespace dl {

// A triangular square's three 16 x 16 blocks that are not zero, (0, 0), (1, 0) and (1, 1) of a LOWER
// one, (0, 0), (0, 1) and (1, 1) of an upper one, as operands over the tokens of their columns.
struct Square {
  f32x4 m[3];
};
template <bool LOWER>
__device__ __forceinline__ Square square_at(const unsigned char* lds, int lane) {
  auto block = [&](int i, int j) {
    return *reinterpret_cast<const f32x4*>(lds + 16 * (64 * i + lane) + j * WsLayout::SQ);
  };
  return Square{{block(0, 0), LOWER ? block(1, 0) : block(0, 1), block(1, 1)}};
}
// r += m b over the chunk's tokens.
template <bool LOWER>
__device__ __forceinline__ void square_mma(const Square& m, const Full& b, f32x4& r0, f32x4& r1) {
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    r0 = mma(m.m[0][e], b.hi[e], r0);
    x = mma(m.m[1][e], LOWER ? b.hi[e] : b.lo[e], x);
    r1 = mma(m.m[2][e], b.lo[e], r1);
  }
  (LOWER ? r1 : r0) += x;
}

// Result tiles [2][NT] (tokens 16 tt + 4 g + r) as operands over the chunk's tokens.
template <typename OP, int NT>
__device__ __forceinline__ OP tokens_operand(const f32x4 (&x)[2][NT], int t) {
  float a[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) a[e] = x[e >> 2][t][e & 3];
  return operand8<OP>(a);
}
template <typename OP, int NKT, int NT>
__device__ __forceinline__ OP state_operand(const f32x4 (&S)[NKT][NT], int s, int t) {
  float a[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) a[e] = S[2 * s + (e >> 2)][t][e & 3];
  return operand8<OP>(a);
}

enum PassId { PASS_OUT = 0, PASS_SAVE = 1, PASS_BACK = 2, PASS_SEG = 3 };

// One chunk's operands on their way from memory to LDS.
template <int DK, int NT, int NW, bool RAW, bool DELTA, int PASS, typename TIN>
struct Stage {
  using Op = std::conditional_t<RAW, bf16x8, Full>;    // an operand from a plane,
  using By = std::conditional_t<RAW, Three, Full>;     // and what it is multiplied with;
  // the same for outputs
  using OutOp = std::conditional_t<RAW, bf16x8, std::conditional_t<sizeof(TIN) == 2, Pair, Full>>;
  using OutBy = std::conditional_t<RAW, Three, std::conditional_t<sizeof(TIN) == 2, Pair, Full>>;
  static constexpr int T = 64 * NW, VC = 16 * NT * NW, NP = DK / 8;
  static constexpr int HALF = CT * DK * 2;                     // bytes of half a plane
  static constexpr int PL = RAW ? 0 : HALF, SQ = WsLayout::SQ, SQ2 = 2 * SQ;
  static constexpr int FAC = 4 * DK + 12 * CT;
  static constexpr bool BACK = PASS == PASS_BACK, OUT = PASS == PASS_OUT;
  static constexpr bool WITH_Q = BACK || OUT;
  // Raw planes' operands are read ahead of the products before theirs; fp32 ones, whose products take
  // five times as long, one by one: registers would not do for all.
  static constexpr bool AHEAD = RAW;
  // LDS offsets, of the workspace block: first P, N, Kh (what of them the pass needs), then Qh,
  // Kb, the factors, and backward P^T, M^T.
  static constexpr int A_P = 0;
  static constexpr int A_N = OUT ? SQ2 : 0;
  static constexpr int A_KH = A_N + (!BACK && DELTA ? SQ2 : 0);
  static constexpr int HEAD = A_KH + (DELTA ? 2 * PL : 0);
  static constexpr int A_QH = HEAD;
  static constexpr int A_KB = A_QH + (WITH_Q ? 2 * PL : 0);
  static constexpr int A_DEC = A_KB + 2 * PL;
  static constexpr int A_BETA = A_DEC + 4 * DK, A_F = A_BETA + 4 * CT, A_G = A_F + 4 * CT;
  static constexpr int A_PT = A_DEC + FAC;
  static constexpr int A_MT = A_PT + (BACK ? SQ2 : 0);
  static constexpr int LINEAR = A_MT + (BACK && DELTA ? SQ2 : 0);
  static constexpr int A_K = LINEAR, A_Q = A_K + (RAW ? HALF : 0);
  static constexpr int A_V = A_Q + (RAW && WITH_Q ? HALF : 0);
  static constexpr int VNP = VC * int(sizeof(TIN)) / 16;       // pieces of a value row
  static constexpr int VROW = sizeof(TIN) == 2 ? VC * 2 : VC * 4 + 16;
  static constexpr int BYTES = A_V + CT * VROW;

  static constexpr int NLIN = (LINEAR / 16 + T - 1) / T;
  // Rounds of a plane's pieces and of the values'.  Eight waves have twice as many threads as a plane
  // of 64 keys has pieces: those past the last load it once more and store nothing.
  static constexpr int KQ = CT * NP;
  static constexpr int NKQ = RAW ? (KQ + T - 1) / T : 0;
  static constexpr int NV = CT * VNP / T;
  static_assert(!RAW || NKQ * T >= KQ, "every key piece has a thread");
  static_assert(CT * VNP % T == 0, "whole rounds of value pieces");
  u32x4 lin[NLIN], kk[NKQ ? NKQ : 1], qq[NKQ ? NKQ : 1], vv[NV];

  // Everything but the thread's own 32-bit offsets is the same for all lanes.  vals: row 0,
  // this workgroup's first column, of this head's value rows (stride H dv).
  __device__ __forceinline__ void load(const SeqParams& p, const unsigned char* blk, int first,
                                       int count, int h, const TIN* vals, int tid) {
    const WsLayout w{DK, p.dv, RAW, p.bwd};
    const uint32_t from = BACK ? w.kh() : OUT ? w.p() : w.n();
    const uint32_t gap = (WITH_Q ? w.qh() : w.kb()) - HEAD;
#pragma unroll
    for (int i = 0; i < NLIN; ++i) {
      uint32_t x = 16 * (i * T + tid);
      if ((i + 1) * 16 * T > LINEAR) x = min(x, uint32_t(LINEAR - 16));
      if (i * 16 * T >= HEAD) x += gap;
      else if ((i + 1) * 16 * T <= HEAD) x += from;
      else x += x >= uint32_t(HEAD) ? gap : from;
      lin[i] = *reinterpret_cast<const u32x4*>(blk + x);
    }
    if constexpr (RAW) {
      const uint32_t stride = uint32_t(p.H) * DK * 2, last = uint32_t(count - 1) * stride;
      const int64_t at = (int64_t(first) * p.H + h) * DK * 2;
      const unsigned char* kb = static_cast<const unsigned char*>(p.k) + at;
      const unsigned char* qb = static_cast<const unsigned char*>(p.q) + at;
#pragma unroll
      for (int i = 0; i < NKQ; ++i) {
        int x = i * T + tid;
        if ((i + 1) * T > KQ) x = min(x, KQ - 1);
        const int r = x / NP, pc = (x % NP) ^ piece_swap<NP>(r);
        const uint32_t o = min(r * stride, last) + 16 * pc;
        kk[i] = *reinterpret_cast<const u32x4*>(kb + o);
        if constexpr (WITH_Q) qq[i] = *reinterpret_cast<const u32x4*>(qb + o);
      }
    }
    const uint32_t stride = uint32_t(p.H) * uint32_t(p.dv) * sizeof(TIN);
    const uint32_t last = uint32_t(count - 1) * stride;
    const unsigned char* vb = reinterpret_cast<const unsigned char*>(vals + int64_t(first) * p.H * p.dv);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int x = i * T + tid, r = x / VNP;
      vv[i] = *reinterpret_cast<const u32x4*>(vb + (min(r * stride, last) + 16 * (x % VNP)));
    }
  }
  // Rows past the chunk's end become zero here: a test in load() would wait for the data.
  __device__ __forceinline__ void store(unsigned char* lds, int count, int tid) {
    if (count < CT) {
      const u32x4 zero = {0, 0, 0, 0};
      if constexpr (RAW)
#pragma unroll
        for (int i = 0; i < NKQ; ++i)
          if ((i * T + tid) / NP >= count) kk[i] = qq[i] = zero;
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if ((i * T + tid) / VNP >= count) vv[i] = zero;
    }
#pragma unroll
    for (int i = 0; i < NLIN; ++i) {
      const int x = 16 * (i * T + tid);
      if ((i + 1) * 16 * T <= LINEAR || x < LINEAR) *reinterpret_cast<u32x4*>(lds + x) = lin[i];
    }
    if constexpr (RAW) {
#pragma unroll
      for (int i = 0; i < NKQ; ++i) {
        const int x = i * T + tid;
        if ((i + 1) * T > KQ && x >= KQ) continue;
        *reinterpret_cast<u32x4*>(lds + A_K + 16 * x) = kk[i];
        if constexpr (WITH_Q) *reinterpret_cast<u32x4*>(lds + A_Q + 16 * x) = qq[i];
      }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int x = i * T + tid;
      *reinterpret_cast<u32x4*>(lds + value_piece(x / VNP, x % VNP)) = vv[i];
    }
  }
  static __device__ __forceinline__ int value_piece(int r, int x) {
    return A_V + (sizeof(TIN) == 2 ? 16 * piece_at<VNP>(r, x) : r * VROW + 16 * x);
  }
  // A wave's result tiles over its own value columns, which it has read, and from there to
  // memory in 16-byte pieces: out points to row 0, the wave's first column.  Rows from count on
  // write the last row once more: with a store that some lanes or chunks skip, the wait for
  // the next chunk's loads would have to be one for every store as well.
  static __device__ __forceinline__ void results(unsigned char* lds, const f32x4 (&x)[2][NT], int ct0,
                                                 TIN* out, int64_t stride, int count, int lane) {
    const int c16 = lane & 15, g = lane >> 4;
    constexpr int PER = 16 / int(sizeof(TIN));
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int col = 16 * (ct0 + t) + c16;
          narrow(reinterpret_cast<TIN*>(lds + value_piece(16 * tt + 4 * g + r, col / PER)) + col % PER,
                 x[tt][t][r]);
        }
    wave_sync();
    constexpr int WP = 16 * NT / PER;                        // pieces of a row
#pragma unroll
    for (int i = 0; i < CT * WP / 64; ++i) {
      const int y = i * 64 + lane, r = min(y / WP, count - 1), pc = y % WP;
      const u32x4 z = *reinterpret_cast<const u32x4*>(lds + value_piece(r, 16 * ct0 / PER + pc));
      *reinterpret_cast<u32x4*>(out + r * stride + PER * pc) = z;
    }
  }
  // Value rows as result tiles: tokens 16 tt + 4 g + r, column 16 ct + l%16.
  static __device__ __forceinline__ f32x4 values(const unsigned char* lds, int tt, int ct, int lane) {
    f32x4 x;
    if constexpr (sizeof(TIN) == 2) {
      const int i = lane & 15, r = 16 * tt + 4 * (lane >> 4) + (i >> 2);
      const bf16x4 a =
          read_column(lds + A_V + 8 * (i & 1) + 16 * piece_at<VNP>(r, 2 * ct + ((i >> 1) & 1)));
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = (float)a[e];
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        x[e] = *reinterpret_cast<const float*>(lds + A_V + (16 * tt + 4 * (lane >> 4) + e) * VROW +
                                               4 * (16 * ct + (lane & 15)));
    }
    return x;
  }
  static __device__ __forceinline__ f32x4 factor(const unsigned char* lds, int at, int tt, int lane) {
    return *reinterpret_cast<const f32x4*>(lds + at + 4 * (16 * tt + 4 * (lane >> 4)));
  }
  // Operands from the planes; raw ones have no second half.
  template <typename OP = Op>
  static __device__ __forceinline__ OP rows(const unsigned char* lds, int raw_at, int at, int tt, int s,
                                            int lane) {
    return rows_operand<OP, NP>(lds + (RAW ? raw_at : at), RAW ? 0 : HALF, tt, s, lane);
  }
  static __device__ __forceinline__ Op cols(const unsigned char* lds, int raw_at, int at, int f, int lane) {
    return cols_operand<Op, NP>(lds + (RAW ? raw_at : at), RAW ? 0 : HALF, f, lane);
  }
  // e^{l_T} for keys state_key(f, g, r)
  static __device__ __forceinline__ f32x4 decay(const unsigned char* lds, int f, int lane) {
    if constexpr (RAW) {
      const float d = *reinterpret_cast<const float*>(lds + A_F + 4 * (CT - 1));
      return f32x4{d, d, d, d};
    } else {
      return *reinterpret_cast<const f32x4*>(lds + A_DEC + 4 * state_key(f, lane >> 4, 0));
    }
  }
};

// Where a workgroup stands: (sequence, segment, head, first value column) and its chunks.
struct Walk {
  int seq, h, slot, v0, j, c0, c1, first, end;
  bool last;               // the sequence ends here
  int64_t seg_at;          // floats into the segment states
  __device__ __forceinline__ int row(int c) const { return first + CT * (c - c0); }
  __device__ __forceinline__ int count(int c) const { return min(CT, end - row(c)); }
};
// Segments stand one after the other, sequence by sequence: those of sequence s from here on, room
// for cu_chunks[s + 1] - cu_chunks[s] chunks, and for one segment at least.
__device__ __forceinline__ int seg_base(const SeqParams& p, int s) {
  return max(p.cu_chunks[s], 0) / p.seg_len + s;
}
// cols: the columns walked, dv or (segments of a delta rule) dv + dk.  segments: p.seg_len counts,
// else sequences are walked whole.
template <int VC>
__device__ __forceinline__ bool start_walk(const SeqParams& p, int b, int cols, bool segments,
                                           int64_t seg_size, Walk& k) {
  const int nvt = cols / VC;
  k.v0 = VC * (b % nvt);
  k.h = (b / nvt) % p.H;
  const int i = b / nvt / p.H;
  k.j = 0;
  if (segments) {                              // the last sequence that starts at i or before
    int lo = 0, hi = p.n - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (seg_base(p, mid) <= i) lo = mid;
      else hi = mid - 1;
    }
    k.seq = lo;
    k.j = i - seg_base(p, lo);
    if (k.j < 0) return false;
  } else {
    k.seq = p.order[i];                        // longest first: none starts when the rest is done
  }
  if (k.seq < 0 || k.seq >= p.n) return false;
  k.slot = p.seq_slot[k.seq];
  if (k.slot < 0 || k.slot >= p.B) return false;
  k.c0 = max(p.cu_chunks[k.seq], 0);
  k.c1 = min(p.cu_chunks[k.seq + 1], p.max_chunks);
  k.first = max(p.cu_tokens[k.seq], 0);
  k.end = min(p.cu_tokens[k.seq + 1], p.N);
  k.c1 = min(k.c1, k.c0 + (max(k.end - k.first, 0) + CT - 1) / CT);
  k.last = true;
  k.seg_at = 0;
  if (segments) {
    const int from = k.c0 + k.j * p.seg_len;   // seg_base: at most cu_chunks[seq] + i * seg_len
    if (k.j > 0 && from >= k.c1) return false;
    k.first += CT * (from - k.c0);
    k.c0 = from;
    k.last = k.c1 - from <= p.seg_len;
    if (!k.last) k.c1 = from + p.seg_len;
    k.seg_at = (int64_t(i) * p.H + k.h) * seg_size;
  }
  return true;
}

template <int NKT, int NT>
__device__ __forceinline__ void read_state(f32x4 (&S)[NKT][NT], const void* base, const SeqParams& p,
                                           int64_t at, int lane) {
#pragma unroll
  for (int f = 0; f < NKT; ++f)
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int t = 0; t < NT; ++t)
        S[f][t][r] = base ? load_state(base, p.state_bf16,
                                       at + int64_t(state_key(f, lane >> 4, r)) * p.dv + 16 * t)
                          : 0.f;
}
template <int NKT, int NT>
__device__ __forceinline__ void read_floats(f32x4 (&S)[NKT][NT], const float* base, int dv, int v,
                                            int lane) {
#pragma unroll
  for (int f = 0; f < NKT; ++f)
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int t = 0; t < NT; ++t)
        S[f][t][r] = base[int64_t(state_key(f, lane >> 4, r)) * dv + v + 16 * t];
}
template <int NKT, int NT>
__device__ __forceinline__ void write_state(const f32x4 (&S)[NKT][NT], void* base, bool bf16, int dv,
                                            int64_t at, int lane) {
#pragma unroll
  for (int f = 0; f < NKT; ++f)
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int t = 0; t < NT; ++t)
        store_state(base, bf16, at + int64_t(state_key(f, lane >> 4, r)) * dv + 16 * t, S[f][t][r]);
}

// Results into the workspace, [column tile][row][16]; rows: KEYS (of a state), or tokens.  They are
// read once, by a later kernel, and there are more of them than caches hold: stored past the
// caches, what follows finds its operands there (a GDN training step of 2 x 2048 tokens, 32 heads
// of 128 x 128: 613 -> 577 us, of which the gradients 199 -> 176, when its products were shorter).
template <bool KEYS, int NR, int NT>
__device__ __forceinline__ void save_tiles(const f32x4 (&x)[NR][NT], unsigned char* base, int tile,
                                           int lane) {
  float* at = reinterpret_cast<float*>(base) + tile * NR * 256;
  const uint32_t o = (KEYS ? 128 : 64) * (lane >> 4) + (lane & 15);
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int f = 0; f < NR; ++f)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        __builtin_nontemporal_store(
            float(x[f][t][r]), at + o + t * NR * 256 + 16 * (KEYS ? state_key(f, 0, r) : 16 * f + r));
}

// PASS_OUT writes outputs and final states; PASS_SAVE the states before each chunk and E, for
// the backward pass.
//
// Two LDS buffers: while chunk c is computed from one, chunk c + 1 goes from registers to the
// other and c + 2 from memory to registers, and at its end the wave reads what chunk c + 1
// starts with.  What the state needs comes first, outputs follow.
template <int DK, int NT, int NW, bool RAW, bool DELTA, int PASS, typename TIN>
__device__ __forceinline__ void walk_forward(
    const SeqParams& p, int group,
    unsigned char (&lds)[2][Stage<DK, NT, NW, RAW, DELTA, PASS, TIN>::BYTES]) {
  using St = Stage<DK, NT, NW, RAW, DELTA, PASS, TIN>;
  using Op = typename St::Op;
  using By = typename St::By;
  constexpr int NKT = DK / 16, NKS = DK / 32;
  constexpr bool OUT = PASS == PASS_OUT;
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, c16 = lane & 15;
  Walk k;
  constexpr bool SEG = PASS == PASS_SEG;
  const int cols = p.dv + (SEG && DELTA ? DK : 0);
  const bool segments = SEG || (OUT && p.seg_len);
  if (!start_walk<St::VC>(p, group, cols, segments, seg_floats(DK, p.dv, DELTA), k)) return;
  const bool unit = SEG && DELTA && k.v0 >= p.dv;              // columns of M
  if (SEG && (k.last || (unit && k.j == 0))) return;           // nobody asks for these
  const WsLayout w{DK, p.dv, RAW, p.bwd};
  const int ct0 = wave * NT, v = k.v0 + 16 * ct0 + c16;        // this lane's first column
  const int64_t state_at = (int64_t(k.slot) * p.H + k.h) * DK * p.dv + v;
  const int64_t row_stride = int64_t(p.H) * p.dv;
  const TIN* vals = static_cast<const TIN*>(p.v) + int64_t(k.h) * p.dv + (unit ? 0 : k.v0);
  St st;
  auto block = [&](int c) { return p.ws + (int64_t(c) * p.H + k.h) * w.block(); };
  auto fetch = [&](int c) {
    c = min(c, k.c1 - 1);
    st.load(p, block(c), k.row(c), k.count(c), k.h, vals, tid);
  };

  f32x4 U[2][NT], S[NKT][NT], ff[2];
  Op ak[2][NKS];
  Square an;
  auto ahead = [&](const unsigned char* l) {
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        U[tt][t] = St::values(l, tt, ct0 + t, lane);
        if (SEG && DELTA && unit) U[tt][t] = zero;             // no values
      }
      if constexpr (RAW) ff[tt] = St::factor(l, St::A_F, tt, lane);
      if constexpr (DELTA) {
#pragma unroll
        for (int s = 0; s < NKS; ++s)
          if constexpr (St::AHEAD) ak[tt][s] = St::rows(l, St::A_K, St::A_KH, tt, s, lane);
      }
    }
    if constexpr (DELTA) an = square_at<true>(l + St::A_N, lane);
  };
  auto chunk = [&](int c, unsigned char* cur, unsigned char* nxt) __attribute__((always_inline)) {
    __syncthreads();
    st.store(nxt, k.count(min(c + 1, k.c1 - 1)), tid);
    fetch(c + 2);
    if constexpr (PASS == PASS_SAVE) save_tiles<true>(S, block(c) + w.s0(), k.v0 / 16 + ct0, lane);

    // Kh S, R = V - Kh S, E = N R (but for PASS_SAVE N holds beta N, and U comes at once)
    using OutBy = typename St::OutBy;
    By sb[NKS][NT];
    OutBy so[NKS][NT];
    f32x4 X[2][NT], XL[2][NT];
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
      for (int t = 0; t < NT; ++t) X[tt][t] = XL[tt][t] = zero;
#pragma unroll
    for (int s = 0; s < NKS; ++s)
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        if constexpr (DELTA) {
          sb[s][t] = state_operand<By, NKT, NT>(S, s, t);
#pragma unroll
          for (int tt = 0; tt < 2; ++tt) {
            if constexpr (!St::AHEAD) ak[tt][s] = St::rows(cur, St::A_K, St::A_KH, tt, s, lane);
            mma(ak[tt][s], sb[s][t], X[tt][t], XL[tt][t]);
          }
        }
        if constexpr (OUT) {
          if constexpr (DELTA && std::is_same_v<By, OutBy>) so[s][t] = sb[s][t];
          else so[s][t] = state_operand<OutBy, NKT, NT>(S, s, t);
        }
      }
    Op ac[NKT];
    f32x4 gf[2], be[2];
#pragma unroll
    for (int f = 0; f < NKT; ++f)
      if constexpr (St::AHEAD) ac[f] = St::cols(cur, St::A_K, St::A_KB, f, lane);
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      if constexpr (RAW) gf[tt] = St::factor(cur, St::A_G, tt, lane);
      if constexpr (DELTA && PASS == PASS_SAVE) be[tt] = St::factor(cur, St::A_BETA, tt, lane);
    }
    if constexpr (DELTA) {
      Full rb[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
          X[tt][t] += XL[tt][t];
          U[tt][t] -= RAW ? X[tt][t] * ff[tt] : X[tt][t];
        }
        rb[t] = tokens_operand<Full, NT>(U, t);
        U[0][t] = U[1][t] = zero;
        square_mma<true>(an, rb[t], U[0][t], U[1][t]);
      }
    }
    if constexpr (PASS == PASS_SAVE) {
      save_tiles<false>(U, block(c) + w.e(), k.v0 / 16 + ct0, lane);
      if constexpr (DELTA) {
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
          for (int t = 0; t < NT; ++t) U[tt][t] *= be[tt];
      }
    }
    Full ub[NT];
    By gb[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      if constexpr (OUT || !RAW) ub[t] = tokens_operand<Full, NT>(U, t);
      if constexpr (RAW) {
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) U[tt][t] *= gf[tt];
        gb[t] = tokens_operand<By, NT>(U, t);
      } else {
        gb[t] = ub[t];
      }
    }
    // S <- e^{l_T} S + Kb^T U
#pragma unroll
    for (int f = 0; f < NKT; ++f) {
      const f32x4 d = St::decay(cur, f, lane);
      if constexpr (!St::AHEAD) ac[f] = St::cols(cur, St::A_K, St::A_KB, f, lane);
#pragma unroll
      for (int t = 0; t < NT; ++t) S[f][t] = mma(ac[f], gb[t], S[f][t] * d);
    }
    __syncthreads();
    if constexpr (OUT) {
      f32x4 O[2][NT], OL[2][NT], fo[2];
      const Square ap = square_at<true>(cur + St::A_P, lane);
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        fo[tt] = ff[tt];
#pragma unroll
        for (int t = 0; t < NT; ++t) O[tt][t] = OL[tt][t] = zero;
      }
#pragma unroll
      for (int s = 0; s < NKS; ++s)
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
          const auto aq = St::template rows<typename St::OutOp>(cur, St::A_Q, St::A_QH, tt, s, lane);
#pragma unroll
          for (int t = 0; t < NT; ++t) mma_out(aq, so[s][t], O[tt][t], OL[tt][t]);
        }
      ahead(nxt);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
          O[tt][t] += OL[tt][t];
          if constexpr (RAW) O[tt][t] *= fo[tt];
        }
        square_mma<true>(ap, ub[t], O[0][t], O[1][t]);
      }
      St::results(cur, O, ct0,
                  static_cast<TIN*>(p.o) + int64_t(k.row(c)) * row_stride + int64_t(k.h) * p.dv +
                      k.v0 + 16 * ct0,
                  row_stride, k.count(c), lane);
    } else {
      ahead(nxt);
    }
  };

  if (k.c0 < k.c1) fetch(k.c0);
  float* seg = p.seg + k.seg_at;               // L, then the segment's first state: [dk][dv]; M
  if (PASS == PASS_SAVE || (SEG ? k.j == 0 : k.j == 0 && k.last))
    read_state(S, p.S_in, p, state_at, lane);
  else if constexpr (OUT) read_floats(S, seg, p.dv, v, lane);
  else if constexpr (SEG)
#pragma unroll
    for (int f = 0; f < NKT; ++f)
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int t = 0; t < NT; ++t)
          S[f][t][r] = unit && state_key(f, lane >> 4, r) == v + 16 * t - p.dv ? 1.f : 0.f;
  if (k.c0 < k.c1) {
    st.store(lds[0], k.count(k.c0), tid);
    fetch(k.c0 + 1);
    __syncthreads();
    ahead(lds[0]);
    // Two chunks a round while both buffers are within an LDS instruction's offset (64 KiB):
    // their addresses are then the same registers.
    if constexpr (OUT && sizeof(lds) <= 65536) {
      for (int c = k.c0;;) {
        chunk(c, lds[0], lds[1]);
        if (++c == k.c1) break;
        chunk(c, lds[1], lds[0]);
        if (++c == k.c1) break;
      }
    } else {
#pragma unroll 1
      for (int c = k.c0; c < k.c1; ++c) chunk(c, lds[(c - k.c0) & 1], lds[(c - k.c0 + 1) & 1]);
    }
  }
  if constexpr (OUT) {
    if (k.last) write_state(S, p.S_out, p.state_bf16, p.dv, state_at, lane);
  }
  if constexpr (SEG) {
    if (unit) write_state(S, seg + DK * p.dv, false, DK, v - p.dv, lane);
    else write_state(S, seg, false, p.dv, v, lane);
  }
}

// Backward over the chunks, last to first, with D the gradient of the state after a chunk:
//   dU = P^T dO + Kb D      Z = M^T dU,  Y = beta Z   (no delta rule: Y = dU)
//   dV = Y                  D <- e^{l_T} D + Qh^T dO - Kh^T Y
// LDS as in the forward pass.
template <int DK, int NT, int NW, bool RAW, bool DELTA, typename TIN>
__device__ __forceinline__ void walk_backward(
    const SeqParams& p, int group,
    unsigned char (&lds)[2][Stage<DK, NT, NW, RAW, DELTA, PASS_BACK, TIN>::BYTES]) {
  using St = Stage<DK, NT, NW, RAW, DELTA, PASS_BACK, TIN>;
  using Op = typename St::Op;
  using By = typename St::By;
  constexpr int NKT = DK / 16, NKS = DK / 32;
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, c16 = lane & 15;
  Walk k;
  if (!start_walk<St::VC>(p, group, p.dv, false, 0, k)) return;
  const WsLayout w{DK, p.dv, RAW, true};
  const int ct0 = wave * NT, v = k.v0 + 16 * ct0 + c16;
  const int64_t state_at = (int64_t(k.slot) * p.H + k.h) * DK * p.dv + v;
  const int64_t row_stride = int64_t(p.H) * p.dv;
  const TIN* vals = static_cast<const TIN*>(p.d_o) + int64_t(k.h) * p.dv + k.v0;
  St st;
  auto block = [&](int c) { return p.ws + (int64_t(c) * p.H + k.h) * w.block(); };
  auto fetch = [&](int c) {
    c = max(c, k.c0);
    st.load(p, block(c), k.row(c), k.count(c), k.h, vals, tid);
  };

  f32x4 G[2][NT], D[NKT][NT];
  Op ar[2][NKS];
  auto ahead = [&](const unsigned char* l) {
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
#pragma unroll
      for (int t = 0; t < NT; ++t) G[tt][t] = St::values(l, tt, ct0 + t, lane);    // dO
#pragma unroll
      for (int s = 0; s < NKS; ++s)
        if constexpr (St::AHEAD) ar[tt][s] = St::rows(l, St::A_K, St::A_KB, tt, s, lane);
    }
  };
  auto chunk = [&](int c, unsigned char* cur, unsigned char* nxt) __attribute__((always_inline)) {
    __syncthreads();
    st.store(nxt, k.count(max(c - 1, k.c0)), tid);
    fetch(c - 2);
    save_tiles<true>(D, block(c) + w.ds(), k.v0 / 16 + ct0, lane);

    f32x4 Y[2][NT], gf[2], ff[2], be[2];
    Op ac[NKT];
    const Square apt = square_at<false>(cur + St::A_PT, lane);
    Square amt;
    if constexpr (DELTA) amt = square_at<false>(cur + St::A_MT, lane);
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      if constexpr (RAW) {
        gf[tt] = St::factor(cur, St::A_G, tt, lane);
        ff[tt] = St::factor(cur, St::A_F, tt, lane);
      }
      if constexpr (DELTA) {
        be[tt] = St::factor(cur, St::A_BETA, tt, lane);
      }
    }
    // dU
    f32x4 YL[2][NT];
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
      for (int t = 0; t < NT; ++t) Y[tt][t] = YL[tt][t] = zero;
#pragma unroll
    for (int s = 0; s < NKS; ++s)
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const By sb = state_operand<By, NKT, NT>(D, s, t);
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
          if constexpr (!St::AHEAD) ar[tt][s] = St::rows(cur, St::A_K, St::A_KB, tt, s, lane);
          mma(ar[tt][s], sb, Y[tt][t], YL[tt][t]);
        }
      }
#pragma unroll
    for (int f = 0; f < NKT; ++f)
      if constexpr (St::AHEAD) ac[f] = St::cols(cur, St::A_Q, St::A_QH, f, lane);
    By gb[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const Full o = tokens_operand<Full, NT>(G, t);
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        Y[tt][t] += YL[tt][t];
        if constexpr (RAW) Y[tt][t] *= gf[tt];
      }
      square_mma<false>(apt, o, Y[0][t], Y[1][t]);
      if constexpr (RAW) {
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) G[tt][t] *= ff[tt];
      }
      gb[t] = tokens_operand<By, NT>(G, t);
    }
    // the outputs' share of D needs nothing of Y
#pragma unroll
    for (int f = 0; f < NKT; ++f) {
      const f32x4 d = St::decay(cur, f, lane);
      if constexpr (!St::AHEAD) ac[f] = St::cols(cur, St::A_Q, St::A_QH, f, lane);
#pragma unroll
      for (int t = 0; t < NT; ++t) D[f][t] = mma(ac[f], gb[t], D[f][t] * d);
    }
    if constexpr (DELTA) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const Full rb = tokens_operand<Full, NT>(Y, t);
        Y[0][t] = Y[1][t] = zero;
        square_mma<false>(amt, rb, Y[0][t], Y[1][t]);
      }
    }
    save_tiles<false>(Y, block(c) + w.z(), k.v0 / 16 + ct0, lane);
    if constexpr (DELTA) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        f32x4 m[2][1];
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
          Y[tt][t] *= be[tt];
          m[tt][0] = RAW ? -Y[tt][t] * ff[tt] : -Y[tt][t];
        }
        const By yb = tokens_operand<By, 1>(m, 0);
#pragma unroll
        for (int f = 0; f < NKT; ++f)
          D[f][t] = mma(St::cols(cur, St::A_K, St::A_KH, f, lane), yb, D[f][t]);
      }
    }
    __syncthreads();
    ahead(nxt);
    St::results(cur, Y, ct0,
                static_cast<TIN*>(p.dv_) + int64_t(k.row(c)) * row_stride + int64_t(k.h) * p.dv +
                    k.v0 + 16 * ct0,
                row_stride, k.count(c), lane);
  };

  if (k.c0 < k.c1) fetch(k.c1 - 1);
  read_state(D, p.dS_out, p, state_at, lane);
  if (k.c0 < k.c1) {
    st.store(lds[0], k.count(k.c1 - 1), tid);
    fetch(k.c1 - 2);
    __syncthreads();
    ahead(lds[0]);
    if constexpr (sizeof(lds) <= 65536) {
      for (int c = k.c1 - 1;;) {
        chunk(c, lds[0], lds[1]);
        if (--c < k.c0) break;
        chunk(c, lds[1], lds[0]);
        if (--c < k.c0) break;
      }
    } else {
#pragma unroll 1
      for (int c = k.c1 - 1; c >= k.c0; --c)
        chunk(c, lds[(k.c1 - 1 - c) & 1], lds[(k.c1 - c) & 1]);
    }
  }
  if (p.S_out) write_state(D, p.S_out, p.state_bf16, p.dv, state_at, lane);
}

// Workgroups go round the chip's eight XCDs, each with an L2 of its own.  The `share` workgroups of
// one head read the same operands, chunk by chunk at about the same time, so they are placed on
// one XCD: of `groups` workgroups, of which every ROUND-th lands on the same one, which one this is.
// Four workgroups a head (64 heads of 2048 tokens, 128 x 128): 142 MB fetched instead of 489.
template <int ROUND>
__device__ __forceinline__ int xcd_place(int b, int groups, int share) {
  const int block = ROUND * share;
  if (b >= groups / block * block) return b;
  const int in = b % block;
  return b - in + in % ROUND * share + in / ROUND;
}

// One wave to a SIMD (64 heads of 2048 tokens, 128 x 128, GDN, bf16): 152 us, 2.4 a chunk; the wave
// issues in 50% of its cycles (vector instructions 33%), the matrix cores are busy in 34%, and it waits
// for its own results in the rest: it is one chain.  Two (256 heads of 4096): 487 us, vector 50% and
// matrix 48% of a SIMD's cycles, 1.4 GB moved, 2.9 TB/s.  With planes (KDA, 384 ragged heads, 12345
// tokens) 410 us, matrix 66%: fp32 products.
template <int DK, int NT, int NW, bool RAW, bool DELTA, int PASS, typename TIN>
__global__ __launch_bounds__(64 * NW) void forward_kernel(SeqParams p) {
  __shared__ __attribute__((aligned(16))) unsigned char
      lds[2][Stage<DK, NT, NW, RAW, DELTA, PASS, TIN>::BYTES];
  const int share = (p.dv + (PASS == PASS_SEG && DELTA ? DK : 0)) / (16 * NT * NW);
  walk_forward<DK, NT, NW, RAW, DELTA, PASS, TIN>(p, xcd_place<8>(blockIdx.x, gridDim.x, share), lds);
}

// The states between a sequence's segments, one after the other, a workgroup for 16 columns and a
// wave for 16 keys of them: S_1 = L_0 (segment 0 started from the initial state), S_j+1 = M_j S_j +
// L_j; S_j takes L_j's place, and the initial state that of L_0: where S_out is S_in, the last
// segment writes it while the first one may not have started.  Without the delta rule M_j is the
// decay over the segment.  A step is a chain of one load, one product and one exchange of S through
// LDS; M_j and L_j do not depend on S and are fetched a step ahead.
template <int DK, bool RAW, bool DELTA>
__global__ __launch_bounds__(4 * DK) void join_kernel(SeqParams p) {
  constexpr int NKS = DK / 32, PITCH = 18;     // 8 rows further: 16 banks further
  __shared__ float sh[2][DK * PITCH];
  const int lane = threadIdx.x & 63, f = threadIdx.x >> 6, c16 = lane & 15, g = lane >> 4;
  const int nvt = p.dv / 16, b = blockIdx.x, v = 16 * (b % nvt) + c16, h = b / nvt % p.H;
  const int seq = b / nvt / p.H, slot = p.seq_slot[seq];
  if (slot < 0 || slot >= p.B) return;
  const int c0 = max(p.cu_chunks[seq], 0), c1 = min(p.cu_chunks[seq + 1], p.max_chunks);
  const int parts = (c1 - c0 + p.seg_len - 1) / p.seg_len, base = seg_base(p, seq);
  if (parts <= 1) return;
  const int64_t size = seg_floats(DK, p.dv, DELTA);
  auto at = [&](int j) { return p.seg + (int64_t(base + j) * p.H + h) * size; };
  auto column = [&](int j) {                   // this lane's keys of L_j or S_j
    const float* x = at(j) + int64_t(state_key(f, g, 0)) * p.dv + v;
    return f32x4{x[0], x[p.dv], x[2 * p.dv], x[3 * p.dv]};
  };
  auto place = [&](int j, f32x4 S) {
    float* x = at(j) + int64_t(state_key(f, g, 0)) * p.dv + v;
#pragma unroll
    for (int r = 0; r < 4; ++r) x[r * p.dv] = S[r];
  };

  f32x4 S = column(0), L = column(1), first = {0.f, 0.f, 0.f, 0.f};
  if (p.S_in) {
    const int64_t x = ((int64_t(slot) * p.H + h) * DK + state_key(f, g, 0)) * p.dv + v;
#pragma unroll
    for (int r = 0; r < 4; ++r) first[r] = load_state(p.S_in, p.state_bf16, x + r * p.dv);
  }
  place(0, first);
  if constexpr (DELTA) {
    auto rows = [&](int j, f32x4 (&m)[2 * NKS]) {
      const float* M = at(j) + DK * p.dv + state_key(f, c16 >> 2, c16 & 3) * DK + 8 * g;
#pragma unroll
      for (int s = 0; s < 2 * NKS; ++s)
        m[s] = *reinterpret_cast<const f32x4*>(M + 32 * (s >> 1) + 4 * (s & 1));
    };
    f32x4 m[2 * NKS];
    rows(1, m);
    for (int j = 1; j + 1 < parts; ++j) {
      float* x = sh[j & 1];
#pragma unroll
      for (int r = 0; r < 4; ++r) x[(state_key(f, g, 0) + r) * PITCH + c16] = S[r];
      place(j, S);
      Full am[NKS];
#pragma unroll
      for (int s = 0; s < NKS; ++s) {
        float a[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) a[e] = m[2 * s + (e >> 2)][e & 3];
        am[s] = full8(a);
      }
      S = L;
      const int next = min(j + 1, parts - 2);  // the last one's M is never made
      L = column(next);
      rows(next, m);
      __syncthreads();
#pragma unroll
      for (int s = 0; s < NKS; ++s) {
        float a[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) a[e] = x[(32 * s + 8 * g + e) * PITCH + c16];
        S = mma(am[s], full8(a), S);
      }
    }
  } else {
    const WsLayout w{DK, p.dv, RAW, false};
    for (int j = 1; j + 1 < parts; ++j) {
      f32x4 d = {1.f, 1.f, 1.f, 1.f};
#pragma unroll 8
      for (int c = c0 + j * p.seg_len; c < c0 + (j + 1) * p.seg_len; ++c) {
        const unsigned char* blk = p.ws + (int64_t(c) * p.H + h) * w.block();
        if constexpr (RAW) d *= *reinterpret_cast<const float*>(blk + w.f() + 4 * (CT - 1));
        else d *= *reinterpret_cast<const f32x4*>(blk + w.dec() + 4 * state_key(f, g, 0));
      }
      place(j, S);
      S = d * S + L;
      L = column(min(j + 1, parts - 2));
    }
  }
  place(parts - 1, S);
}

// The backward pass's two walks in one launch: neither needs the other, and each alone leaves
// most of the chip waiting while sequences and heads are few (64 heads of 2048 tokens, 128 x 128: of
// kernels that took 139 + 186 us one after the other, 260 in one launch; these take 279: 235 MB read
// and 723 MB written, of which the states before and the state gradients after every chunk are 537).
// Even workgroups go backward, odd ones forward.
template <int DK, int NT, int NW, bool RAW, bool DELTA, typename TIN>
__global__ __launch_bounds__(64 * NW) void both_kernel(SeqParams p) {
  using Save = Stage<DK, NT, NW, RAW, DELTA, PASS_SAVE, TIN>;
  using Back = Stage<DK, NT, NW, RAW, DELTA, PASS_BACK, TIN>;
  constexpr int BYTES = 2 * (Save::BYTES > Back::BYTES ? Save::BYTES : Back::BYTES);
  __shared__ __attribute__((aligned(16))) unsigned char lds[BYTES];
  const int group = xcd_place<4>(blockIdx.x >> 1, gridDim.x >> 1, p.dv / (16 * NT * NW));
  if (blockIdx.x & 1)
    walk_forward<DK, NT, NW, RAW, DELTA, PASS_SAVE, TIN>(
        p, group, *reinterpret_cast<unsigned char(*)[2][Save::BYTES]>(&lds));
  else
    walk_backward<DK, NT, NW, RAW, DELTA, TIN>(
        p, group, *reinterpret_cast<unsigned char(*)[2][Back::BYTES]>(&lds));
}

}  // namespace dl
