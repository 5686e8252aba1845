// Per-chunk operands of the sequence kernels: everything of a chunk that does not depend on
// the state, so that the serial pass over chunks is matrix products alone.
#pragma once

#include "dl_scan.hpp"

namespace dl {

// One log-decay per head (or none) | per key | per key, read before the token (RWKV6).
constexpr int SL = CT + 4;             // row of a token x token matrix in LDS (16-byte rows)

enum DecayClass { DC_SCALAR = 0, DC_KEY = 1, DC_BONUS = 2 };

constexpr float LOG2E = 1.44269504088896341f;
constexpr float LOG_FLOOR = -104.f;   // e^-104 rounds to 0 in fp32
// The log-decay that counts, in powers of two.  Not fmaxf, which would make a NaN the floor.
__device__ __forceinline__ float log2_decay(float x) { return (x < LOG_FLOOR ? LOG_FLOOR : x) * LOG2E; }
// A diagonal 16 x 16 block of G and P factors through e^{l_i - m} e^{m - l_j} with m the
// log-decay at its middle; both factors stay below 2^WIDE unless the block decays by more.
constexpr float WIDE = 80.f;

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ void load8(const float* p, float* x) {
  const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
  for (int e = 0; e < 4; ++e) { x[e] = a[e]; x[4 + e] = b[e]; }
}
__device__ __forceinline__ void load8(const uint16_t* p, float* x) {
  const u32x4 a = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[2 * e] = __uint_as_float(a[e] << 16);
    x[2 * e + 1] = __uint_as_float(a[e] & 0xffff0000u);
  }
}

// A chunk's inputs in LDS, rows past its end as zero (log-decays: as no decay).  l holds
// cumulative log-decays in powers of two (l log2 e).
template <int DC, int DK, typename TIN>
struct ChunkIn {
  static constexpr int LD = DK + 16 / int(sizeof(TIN)), LL = DC == DC_SCALAR ? 4 : DK + 4;
  __attribute__((aligned(16))) TIN k[CT][LD], q[CT][LD];
  __attribute__((aligned(16))) float l[CT][LL];      // scalar: l[t][0]
  float beta[CT];
  int wide;

  __device__ __forceinline__ float at(int t, int r) const { return l[t][DC == DC_SCALAR ? 0 : r]; }
  // what q_i takes: l_i, or l_{i-1} for RWKV6
  __device__ __forceinline__ float at_q(int t, int r) const {
    if constexpr (DC == DC_BONUS) return t ? l[t - 1][r] : 0.f;
    else return at(t, r);
  }
  __device__ __forceinline__ void at8(int t, int r, float* x) const {
    if constexpr (DC == DC_SCALAR) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = l[t][0];
    } else {
      load8(&l[t][r], x);
    }
  }
  __device__ __forceinline__ void at_q8(int t, int r, float* x) const {
    if constexpr (DC == DC_BONUS) {
      load8(&l[t ? t - 1 : 0][r], x);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = t ? x[e] : 0.f;
    } else {
      at8(t, r, x);
    }
  }

  template <int NT, bool DELTA>
  __device__ void load(const SeqParams& p, const ChunkRow& row, int h, int tid) {
    constexpr int PER = 16 / int(sizeof(TIN)), NPC = DK / PER, NI = CT * NPC / NT;
    static_assert(CT * NPC % NT == 0 && CT * DK / 4 % NT == 0, "whole rounds");
    u32x4 kk[NI], qq[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int x = i * NT + tid, t = x / NPC;
      const int64_t a = (int64_t(row.first + min(t, row.count - 1)) * p.H + h) * DK + PER * (x % NPC);
      kk[i] = *reinterpret_cast<const u32x4*>(static_cast<const TIN*>(p.k) + a);
      qq[i] = *reinterpret_cast<const u32x4*>(static_cast<const TIN*>(p.q) + a);
    }
    f32x4 lam[DC == DC_SCALAR ? 1 : CT * DK / 4 / NT];
    float one = 0.f;
    if constexpr (DC == DC_SCALAR) {
      if (tid < row.count && p.lam) one = p.lam[int64_t(row.first + tid) * p.H + h];
    } else {
      constexpr int LP = DK / 4;
#pragma unroll
      for (int i = 0; i < CT * LP / NT; ++i) {
        const int x = i * NT + tid, t = x / LP;
        // lam is 4-byte aligned only
        typedef __attribute__((ext_vector_type(4), aligned(4))) float f32x4_any;
        lam[i] = *reinterpret_cast<const f32x4_any*>(
            p.lam + (int64_t(row.first + min(t, row.count - 1)) * p.H + h) * DK + 4 * (x % LP));
      }
    }
    float b = 0.f;
    if (tid < CT) {
      if (DELTA && tid < row.count) b = p.beta[int64_t(row.first + tid) * p.H + h];
      beta[tid] = b;
    }
    if (tid == 0) wide = 0;
    const u32x4 zero = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int x = i * NT + tid, t = x / NPC;
      *reinterpret_cast<u32x4*>(&k[t][PER * (x % NPC)]) = t < row.count ? kk[i] : zero;
      *reinterpret_cast<u32x4*>(&q[t][PER * (x % NPC)]) = t < row.count ? qq[i] : zero;
    }
    if constexpr (DC == DC_SCALAR) {
      if (tid < 64) {
        float x = tid < row.count ? log2_decay(one) : 0.f;
#pragma unroll
        for (int d = 1; d < CT; d *= 2) {
          const float y = __shfl_up(x, d);
          if (tid >= d) x += y;
        }
        if (tid < CT) l[tid][0] = x;
      }
    } else {
      constexpr int LP = DK / 4;
#pragma unroll
      for (int i = 0; i < CT * LP / NT; ++i) {
        const int x = i * NT + tid, t = x / LP;
        f32x4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = t < row.count ? log2_decay(lam[i][e]) : 0.f;
        *reinterpret_cast<f32x4*>(&l[t][4 * (x % LP)]) = y;
      }
      __syncthreads();
      if (tid < DK) {
        float x[CT];
#pragma unroll
        for (int t = 0; t < CT; ++t) x[t] = l[t][tid];
#pragma unroll
        for (int t = 1; t < CT; ++t) {
          x[t] += x[t - 1];
          l[t][tid] = x[t];
        }
        if (x[CT / 2 - 1] < -WIDE || x[CT - 1] - x[CT / 2 - 1] < -WIDE) wide = 1;
      }
    }
    __syncthreads();
  }
};

// G (strictly lower) and P (lower; RWKV6: strictly, and its bonus on the diagonal), by three
// of the workgroup's waves; by all of them, pair by pair, where a block decays too far.  On
// fp32 MFMA: the operands are used once, so splitting them (44 instructions for eight values)
// would cost more than the matrix cores' slower fp32 rate, which nothing else here waits for.
template <int DC, int DK, bool DELTA, typename TIN>
__device__ void pair_products(const ChunkIn<DC, DK, TIN>& in, float (*G)[SL], float (*P)[SL],
                              float* diag, const SeqParams& p, int h, int tid) {
  const int lane = tid & 63, wave = tid >> 6, c16 = lane & 15, g = lane >> 4;
  if constexpr (DC == DC_BONUS) {
    // eight lanes per token
    const int t = tid >> 3;
    float s = 0.f;
    for (int r = 8 * (tid & 7); r < DK; r += 64) {
      float a[8], b[8];
      load8(&in.q[t][r], a);
      load8(&in.k[t][r], b);
#pragma unroll
      for (int e = 0; e < 8; ++e) s += a[e] * p.u[int64_t(h) * DK + r + e] * b[e];
    }
    s += __shfl_xor(s, 1);
    s += __shfl_xor(s, 2);
    s += __shfl_xor(s, 4);
    if ((tid & 7) == 0) diag[t] = s;
    __syncthreads();
  }
  const bool wide = DC != DC_SCALAR && in.wide != 0;
  if (wave == 3) {
    for (int i = lane; i < 16 * 16; i += 64) G[i / 16][16 + i % 16] = P[i / 16][16 + i % 16] = 0.f;
  } else if (!(wide && wave < 2)) {
    const int bi = wave == 0 ? 0 : 1, bj = wave == 1 ? 1 : 0;   // (0,0), (1,1), (1,0)
    const int ref = wave == 0 ? 7 : wave == 1 ? 23 : 15;
    const int i = 16 * bi + c16, j = 16 * bj + c16;
    f32x4 ag[2], ap[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) ag[x] = ap[x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < DK / 32; ++s) {
      const int r = 32 * s + 8 * g;
      float ak[8], aq[8], b[8];
      load8(&in.k[i][r], ak);
      load8(&in.q[i][r], aq);
      load8(&in.k[j][r], b);
      if constexpr (DC != DC_SCALAR) {
        float m[8], li[8], lq[8], lj[8];
        in.at8(ref, r, m);
        in.at8(i, r, li);
        in.at8(j, r, lj);
        if (DC == DC_BONUS) in.at_q8(i, r, lq);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if (DC == DC_BONUS) {
            aq[e] *= exp2_of(lq[e] - m[e]);
          } else {
            const float f = exp2_of(li[e] - m[e]);
            aq[e] *= f;
            ak[e] *= f;
          }
          b[e] *= exp2_of(m[e] - lj[e]);
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if constexpr (DELTA)
          ag[e & 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(ak[e], b[e], ag[e & 1], 0, 0, 0);
        ap[e & 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(aq[e], b[e], ap[e & 1], 0, 0, 0);
      }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int ri = 16 * bi + 4 * g + r;
      float x = ap[0][r] + ap[1][r], y = ag[0][r] + ag[1][r];
      if constexpr (DC == DC_SCALAR) {
        const float f = exp2_of(in.l[ri][0] - in.l[j][0]);
        x *= f;
        y *= f;
      }
      if constexpr (DC == DC_BONUS) P[ri][j] = ri > j ? x : ri == j ? diag[ri] : 0.f;
      else P[ri][j] = ri >= j ? x : 0.f;
      G[ri][j] = ri > j ? y : 0.f;
    }
  }
  if (wide) {
    for (int x = tid; x < 2 * 256; x += 256) {
      const int b = x >> 8, i = 16 * b + ((x >> 4) & 15), j = 16 * b + (x & 15);
      float sg = 0.f, sp = 0.f;
      if (i >= j) {
#pragma unroll 1
        for (int r = 0; r < DK; ++r) {
          const float kj = widen(in.k[j][r]), lj = in.at(j, r);
          sg += widen(in.k[i][r]) * kj * exp2_of(in.at(i, r) - lj);
          if (DC == DC_KEY || i > j)
            sp += widen(in.q[i][r]) * kj * exp2_of(in.at_q(i, r) - lj);
        }
      }
      G[i][j] = i > j ? sg : 0.f;
      P[i][j] = (DC == DC_BONUS && i == j) ? diag[i] : sp;
    }
  }
  __syncthreads();
}

// N = (I + G beta)^-1 over G, and (BWD) M = (I + beta G)^-1, by one wave.  The two diagonal
// 16 x 16 blocks of each by forward substitution, a column per lane in registers; then the
// lower left block, N21 = -N22 (G21 beta) N11 and M21 = -M22 (beta G21) M11, by fp32 MFMA:
// 120 multiplications a lane instead of 496.
template <bool BWD>
__device__ __forceinline__ void solve(float (*G)[SL], float (*M)[SL], const float* beta, int lane) {
  const int c16 = lane & 15, g = lane >> 4, o = lane & 16;
  const bool second = BWD && lane >= 32;
  float x[16], y[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int m = 0; m < i; m += 4) {
      const f32x4 row = *reinterpret_cast<const f32x4*>(&G[o + i][o + m]);   // 0 from column i on
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (m + e < i) s[e] += row[e] * y[m + e];
    }
    const float b = beta[o + i], t = (s[0] + s[1]) + (s[2] + s[3]), d = i == c16 ? 1.f : 0.f;
    x[i] = d - (second ? b * t : t);
    y[i] = second ? x[i] : b * x[i];
  }
  float (*out)[SL] = second ? M : G;
  if (BWD || lane < 32) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      out[o + i][o + c16] = x[i];
      if (second && !o) M[i][16 + c16] = 0.f;
    }
  }
  wave_sync();
  f32x4 tn = {0.f, 0.f, 0.f, 0.f}, tm = tn;
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    const float a = G[16 + c16][4 * s + g];
    tn = __builtin_amdgcn_mfma_f32_16x16x4f32(a * beta[4 * s + g], G[4 * s + g][c16], tn, 0, 0, 0);
    if (BWD) tm = __builtin_amdgcn_mfma_f32_16x16x4f32(a * beta[16 + c16], M[4 * s + g][c16], tm, 0, 0, 0);
  }
  f32x4 rn = {0.f, 0.f, 0.f, 0.f}, rm = rn;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    rn = __builtin_amdgcn_mfma_f32_16x16x4f32(G[16 + c16][16 + 4 * g + r], tn[r], rn, 0, 0, 0);
    if (BWD) rm = __builtin_amdgcn_mfma_f32_16x16x4f32(M[16 + c16][16 + 4 * g + r], tm[r], rm, 0, 0, 0);
  }
  wave_sync();
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    G[16 + 4 * g + r][c16] = -rn[r];
    if (BWD) M[16 + 4 * g + r][c16] = -rm[r];
  }
}

// Eight values as the two halves of an operand.
__device__ __forceinline__ void put(unsigned char* base, int half, int unit, const float* x) {
  const Full s = full8(x);
  *reinterpret_cast<f32x4*>(base + 16 * unit) = s.hi;
  *reinterpret_cast<f32x4*>(base + half + 16 * unit) = s.lo;
}
__device__ __forceinline__ void put_pair(unsigned char* base, int half, int unit, const float* x) {
  const Pair s = operand8<Pair>(x);
  *reinterpret_cast<bf16x8*>(base + 16 * unit) = s.a;
  *reinterpret_cast<bf16x8*>(base + half + 16 * unit) = s.b;
}

// The squares from LDS matrices, by NTH threads.
template <int NTH, bool DELTA, bool BWD>
__device__ __forceinline__ void put_squares(unsigned char* blk, const WsLayout& w,
                                            const float (*P)[SL], const float (*N)[SL],
                                            const float (*M)[SL], const float* beta, int tid) {
#pragma unroll
  for (int x = tid; x < CT * CT / 8; x += NTH) {
    const int lane = x & 63, i = 16 * (x >> 6) + (lane & 15), t0 = 4 * (lane >> 4);
    float a[8];
    auto row = [&](const float (*m)[SL], float f) {
      const f32x4 u = *reinterpret_cast<const f32x4*>(&m[i][t0]);
      const f32x4 v = *reinterpret_cast<const f32x4*>(&m[i][16 + t0]);
#pragma unroll
      for (int e = 0; e < 4; ++e) { a[e] = f * u[e]; a[4 + e] = f * v[e]; }
    };
    if constexpr (!BWD) {
      row(P, 1.f);
      put(blk + w.p(), WsLayout::SQ, x, a);
    }
    if constexpr (DELTA) {
      row(N, BWD ? 1.f : beta[i]);
      put(blk + w.n(), WsLayout::SQ, x, a);
    }
    if constexpr (BWD) {
#pragma unroll
      for (int e = 0; e < 8; ++e) a[e] = P[state_term(lane, e)][i];
      put(blk + w.pt(), WsLayout::SQ, x, a);
      if constexpr (DELTA) {
#pragma unroll
        for (int e = 0; e < 8; ++e) a[e] = M[state_term(lane, e)][i];
        put(blk + w.mt(), WsLayout::SQ, x, a);
      }
    }
  }
}

// BWD: for the backward pass.
// Bound by memory: 12345 tokens, 32 heads of 128 keys (KDA, bf16) 184 us for 417 MB read and
// 724 MB written (the planes), 6.2 TB/s, where a large copy reaches 5.55.
template <int DC, int DK, bool DELTA, bool BWD, typename TIN>
__global__ __launch_bounds__(256) void prep_kernel(SeqParams p) {
  __shared__ ChunkIn<DC, DK, TIN> in;
  __shared__ __attribute__((aligned(16))) float G[CT][SL], P[CT][SL], M[BWD ? CT : 1][SL];
  __shared__ float diag[CT];
  const int tid = threadIdx.x;
  const int h = blockIdx.x % p.H, c = blockIdx.x / p.H;
  const ChunkRow row = chunk_row(p, c);
  if (row.count == 0) return;
  const WsLayout w{DK, p.dv, false, BWD};
  unsigned char* blk = p.ws + (int64_t(c) * p.H + h) * w.block();

  in.template load<256, DELTA>(p, row, h, tid);
  pair_products<DC, DK, DELTA, TIN>(in, G, P, diag, p, h, tid);
  // One wave solves while the others go on to the planes.
  if (DELTA && tid < 64) solve<BWD>(G, M, in.beta, tid);

  float* dec = reinterpret_cast<float*>(blk + w.dec());
  float* beta = reinterpret_cast<float*>(blk + w.beta());
  if (tid < DK) dec[tid] = exp2_of(in.at(CT - 1, tid));
  if (tid < CT) beta[tid] = in.beta[tid];
  constexpr int NP = DK / 8;
  for (int x = tid; x < CT * NP; x += 256) {
    const int t = x / NP, r = 8 * (x % NP), at = piece_at<NP>(t, x % NP);
    float k[8], q[8], l[8], lq[8], lT[8], f[8];
    load8(&in.k[t][r], k);
    load8(&in.q[t][r], q);
    in.at8(t, r, l);
    in.at8(CT - 1, r, lT);
    if (DC == DC_BONUS) in.at_q8(t, r, lq);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      f[e] = exp2_of(l[e]);
      q[e] *= DC == DC_BONUS ? exp2_of(lq[e]) : f[e];
      lT[e] = k[e] * exp2_of(lT[e] - l[e]);
      k[e] *= f[e];
    }
    if constexpr (DELTA) put(blk + w.kh(), w.plane(), at, k);
    if constexpr (!BWD && sizeof(TIN) == 2) put_pair(blk + w.qh(), w.plane(), at, q);
    else put(blk + w.qh(), w.plane(), at, q);
    put(blk + w.kb(), w.plane(), at, lT);
  }
  __syncthreads();
  put_squares<256, DELTA, BWD>(blk, w, P, G, M, in.beta, tid);
}

// The same for bf16 keys and queries with one log-decay per head or none, one wave per
// (chunk, head): the operands of k k^T and q k^T come straight from memory, exact in bf16, and
// only the squares and the row factors are written.  Bound by memory: 32768 tokens, 32 heads of
// 128 keys (GDN) 150 us for 613 MB read and 281 MB written, 6 TB/s.
template <int DK, bool DELTA, bool BWD>
__global__ __launch_bounds__(64) void raw_prep_kernel(SeqParams p) {
  constexpr int NKS = DK / 32;
  __shared__ __attribute__((aligned(16))) float G[CT][SL], P[CT][SL], M[BWD ? CT : 1][SL], betas[CT];
  const int lane = threadIdx.x, c16 = lane & 15, g = lane >> 4;
  const int h = blockIdx.x % p.H, c = blockIdx.x / p.H;
  const ChunkRow row = chunk_row(p, c);
  if (row.count == 0) return;
  const WsLayout w{DK, p.dv, true, BWD};
  unsigned char* blk = p.ws + (int64_t(c) * p.H + h) * w.block();

  bf16x8 kf[2][NKS], qf[2][NKS];
#pragma unroll
  for (int tt = 0; tt < 2; ++tt) {
    const int t = 16 * tt + c16;
    const int64_t at = (int64_t(row.first + min(t, row.count - 1)) * p.H + h) * DK + 8 * g;
#pragma unroll
    for (int s = 0; s < NKS; ++s) {
      kf[tt][s] = *reinterpret_cast<const bf16x8*>(static_cast<const uint16_t*>(p.k) + at + 32 * s);
      qf[tt][s] = *reinterpret_cast<const bf16x8*>(static_cast<const uint16_t*>(p.q) + at + 32 * s);
    }
    if (t >= row.count) {
      const u32x4 zero = {0, 0, 0, 0};
#pragma unroll
      for (int s = 0; s < NKS; ++s) kf[tt][s] = qf[tt][s] = __builtin_bit_cast(bf16x8, zero);
    }
  }
  const bool live = lane < row.count;
  const int64_t tok = int64_t(row.first + (live ? lane : 0)) * p.H + h;
  float l = live && p.lam ? log2_decay(p.lam[tok]) : 0.f;
  const float beta = DELTA && live ? p.beta[tok] : 0.f;
#pragma unroll
  for (int d = 1; d < CT; d *= 2) {
    const float y = __shfl_up(l, d);
    if (lane >= d) l += y;
  }
  const float lT = __shfl(l, CT - 1);
  if (lane < CT) {
    float* fac = reinterpret_cast<float*>(blk + w.beta());
    fac[lane] = betas[lane] = beta;
    fac[CT + lane] = exp2_of(l);
    fac[2 * CT + lane] = exp2_of(lT - l);
  }
#pragma unroll
  for (int b = 0; b < 3; ++b) {                 // (0,0), (1,1), (1,0)
    const int bi = b == 0 ? 0 : 1, bj = b == 1 ? 1 : 0;
    f32x4 ag = {0.f, 0.f, 0.f, 0.f}, ap = ag;
#pragma unroll
    for (int s = 0; s < NKS; ++s) {
      if constexpr (DELTA) ag = mma(kf[bi][s], kf[bj][s], ag);
      ap = mma(qf[bi][s], kf[bj][s], ap);
    }
    const int j = 16 * bj + c16;
    const float lj = __shfl(l, j);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int i = 16 * bi + 4 * g + r;
      const float x = exp2_of(__shfl(l, i) - lj);
      P[i][j] = i >= j ? ap[r] * x : 0.f;
      G[i][j] = i > j ? ag[r] * x : 0.f;
    }
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) G[4 * g + r][16 + c16] = P[4 * g + r][16 + c16] = 0.f;
  __syncthreads();
  if constexpr (DELTA) solve<BWD>(G, M, betas, lane);
  __syncthreads();
  put_squares<64, DELTA, BWD>(blk, w, P, G, M, betas, lane);
}

}  // namespace dl
