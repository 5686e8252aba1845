// Per-chunk operands of the sequence kernels: everything of a chunk that does not depend on
// the state, so that the serial pass over chunks is matrix products alone.
#pragma once

#include "dl_scan.hpp"

namespace dl {

enum DecayClass { DC_SCALAR = 0, DC_KEY = 1, DC_BONUS = 2 };  // one per head (or none) | per key | per key, RWKV6

constexpr float LOG_FLOOR = -104.f;   // e^-104 rounds to 0 in fp32
// A diagonal 16 x 16 block of G and P factors through e^{l_i - m} e^{m - l_j} with m the
// log-decay at its middle; both factors stay below e^60 unless the block decays by more.
constexpr float WIDE = 60.f;

// LDS of one (chunk, head): inputs widened to fp32, cumulative log-decays, G and P.
template <int DK>
struct PrepShared {
  float k[CT][DK + 4], q[CT][DK + 4];
  float l[CT][DK + 4];              // l_i (per key)
  float lq[CT][DK + 4];             // what q_i takes: l_i, or l_{i-1} for RWKV6 (per key)
  float sl[CT];                     // l_i (one per head)
  float beta[CT];
  float G[CT][CT + 1], P[CT][CT + 1], Nm[CT][CT + 1], Mm[CT][CT + 1];
  float diag[CT];
  int wide;
};

template <int DC, int DK, typename TIN>
__device__ void load_chunk(PrepShared<DK>& sh, const SeqParams& p, const ChunkRow& row, int h,
                           int tid, int nt) {
  const TIN* k = static_cast<const TIN*>(p.k);
  const TIN* q = static_cast<const TIN*>(p.q);
  for (int i = tid; i < CT * DK; i += nt) {
    const int t = i / DK, r = i % DK;
    const bool live = t < row.count;
    const int64_t at = (int64_t(row.first + (live ? t : 0)) * p.H + h) * DK + r;
    const float kv = widen(k[at]), qv = widen(q[at]);
    sh.k[t][r] = live ? kv : 0.f;
    sh.q[t][r] = live ? qv : 0.f;
  }
  if (tid < CT) {
    const bool live = tid < row.count && p.delta;
    sh.beta[tid] = live ? p.beta[int64_t(row.first + tid) * p.H + h] : 0.f;
  }
  if (tid == 0) sh.wide = 0;
  if constexpr (DC == DC_SCALAR) {
    if (tid < 64) {
      float x = 0.f;
      if (tid < row.count && p.lam)
        x = fmaxf(p.lam[int64_t(row.first + tid) * p.H + h], LOG_FLOOR);
#pragma unroll
      for (int d = 1; d < CT; d *= 2) {
        const float y = __shfl_up(x, d);
        if (tid >= d) x += y;
      }
      if (tid < CT) sh.sl[tid] = x;
    }
  } else {
    __syncthreads();               // wide is cleared
    for (int r = tid; r < DK; r += nt) {
      const float* lam = p.lam + (int64_t(row.first) * p.H + h) * DK + r;
      float acc = 0.f, half = 0.f;
#pragma unroll 8
      for (int t = 0; t < CT; ++t) {
        if (t == CT / 2) half = acc;
        sh.lq[t][r] = acc;
        if (t < row.count) acc += fmaxf(lam[int64_t(t) * p.H * DK], LOG_FLOOR);
        if (DC == DC_KEY) sh.lq[t][r] = acc;
        sh.l[t][r] = acc;
      }
      if (-half > WIDE || half - acc > WIDE) atomicOr(&sh.wide, 1);
    }
  }
  __syncthreads();
}

// G (strictly lower) and P (lower; RWKV6 strictly, plus its bonus diagonal) into LDS.
template <int DC, int DK>
__device__ void pair_products(PrepShared<DK>& sh, const SeqParams& p, int h, int tid, int nt) {
  const int lane = tid & 63, wave = tid >> 6, nw = nt >> 6;
  const int c16 = lane & 15, g = lane >> 4;
  const bool wide = DC != DC_SCALAR && sh.wide != 0;
  // Upper blocks are zero; the products below write the three lower ones.
  for (int i = tid; i < 16 * 16; i += nt) sh.G[i / 16][16 + i % 16] = sh.P[i / 16][16 + i % 16] = 0.f;
  if constexpr (DC == DC_BONUS) {
    for (int t = wave; t < CT; t += nw) {
      float s = 0.f;
      for (int r = lane; r < DK; r += 64) s += sh.q[t][r] * p.u[int64_t(h) * DK + r] * sh.k[t][r];
#pragma unroll
      for (int d = 1; d < 64; d *= 2) s += __shfl_xor(s, d);
      if (lane == 0) sh.diag[t] = s;
    }
    __syncthreads();
  }
  for (int task = wave; task < 6; task += nw) {
    const bool isP = task & 1;
    const int blk = task >> 1;              // (0,0), (1,1), (1,0)
    const int bi = blk == 0 ? 0 : 1, bj = blk == 1 ? 1 : 0;
    if (wide && blk != 2) continue;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    const int i = 16 * bi + c16, j = 16 * bj + c16;
    const int ref = blk == 0 ? 7 : blk == 1 ? 23 : 15;
    for (int s = 0; s < DK / 32; ++s) {
      float a[8], b[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int r = 32 * s + 8 * g + e;
        a[e] = isP ? sh.q[i][r] : sh.k[i][r];
        b[e] = sh.k[j][r];
        if constexpr (DC != DC_SCALAR) {
          const float m = sh.l[ref][r];
          a[e] *= __expf((isP ? sh.lq[i][r] : sh.l[i][r]) - m);
          b[e] *= __expf(m - sh.l[j][r]);
        }
      }
      acc = mma3(split8(a), split8(b), acc);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int ri = 16 * bi + 4 * g + r, cj = j;
      float x = acc[r];
      if constexpr (DC == DC_SCALAR) x *= __expf(fminf(sh.sl[ri] - sh.sl[cj], 0.f));
      if (isP) {
        if constexpr (DC == DC_BONUS) x = ri > cj ? x : ri == cj ? sh.diag[ri] : 0.f;
        else x = ri >= cj ? x : 0.f;
        sh.P[ri][cj] = x;
      } else {
        sh.G[ri][cj] = ri > cj ? x : 0.f;
      }
    }
  }
  if (wide) {                               // pair by pair, the exponent of the difference
    for (int x = tid; x < 2 * 256; x += nt) {
      const int b = x >> 8, i = 16 * b + ((x >> 4) & 15), j = 16 * b + (x & 15);
      float sg = 0.f, sp = 0.f;
      if (i >= j) {
        for (int r = 0; r < DK; ++r) {
          const float kj = sh.k[j][r];
          sg += sh.k[i][r] * kj * __expf(sh.l[i][r] - sh.l[j][r]);
          if (DC == DC_KEY || i > j) sp += sh.q[i][r] * kj * __expf(fminf(sh.lq[i][r] - sh.l[j][r], 0.f));
        }
      }
      sh.G[i][j] = i > j ? sg : 0.f;
      sh.P[i][j] = (DC == DC_BONUS && i == j) ? sh.diag[i] : sp;
    }
  }
  __syncthreads();
}

// N = (I + G beta)^-1 in lanes 0-31, M = (I + beta G)^-1 in lanes 32-63 of one wave, a
// column per lane by forward substitution.
template <int DK>
__device__ void solve(PrepShared<DK>& sh, int lane) {
  const int j = lane & 31;
  const bool second = lane >= 32;
  float y[CT];
#pragma unroll
  for (int i = 0; i < CT; ++i) {
    float s = 0.f;
#pragma unroll
    for (int m = 0; m < i; ++m) s += sh.G[i][m] * y[m];
    const float b = sh.beta[i], d = i == j ? 1.f : 0.f;
    const float x = d - (second ? b * s : s);
    y[i] = second ? x : b * x;
    if (second) sh.Mm[i][j] = x;
    else sh.Nm[i][j] = x;
  }
}

template <int DC, int DK>
__device__ __forceinline__ float prep_l(const PrepShared<DK>& sh, int t, int r) {
  if constexpr (DC == DC_SCALAR) return sh.sl[t];
  else return sh.l[t][r];
}
template <int DC, int DK>
__device__ __forceinline__ float prep_lq(const PrepShared<DK>& sh, int t, int r) {
  if constexpr (DC == DC_SCALAR) return sh.sl[t];
  else return sh.lq[t][r];
}

__device__ __forceinline__ void put(unsigned char* base, int half, int unit, const float* x) {
  const Split s = split8(x);
  *reinterpret_cast<bf16x8*>(base + 16 * unit) = s.hi;
  *reinterpret_cast<bf16x8*>(base + half + 16 * unit) = s.lo;
}

// The squares from LDS matrices, by NTH threads.
template <int NTH, int LD>
__device__ __forceinline__ void put_squares(unsigned char* blk, const WsLayout& w, const SeqParams& p,
                                            const float (*P)[LD], const float (*Nm)[LD],
                                            const float (*Mm)[LD], int tid) {
  for (int x = tid; x < CT * CT / 8; x += NTH) {
    const int lane = x & 63, i = 16 * (x >> 6) + (lane & 15);
    float a[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) a[e] = P[i][state_term(lane, e)];
    put(blk + w.p(), WsLayout::SQ, x, a);
    if (p.delta) {
#pragma unroll
      for (int e = 0; e < 8; ++e) a[e] = Nm[i][state_term(lane, e)];
      put(blk + w.n(), WsLayout::SQ, x, a);
    }
    if (p.bwd) {
#pragma unroll
      for (int e = 0; e < 8; ++e) a[e] = P[state_term(lane, e)][i];
      put(blk + w.pt(), WsLayout::SQ, x, a);
      if (p.delta) {
#pragma unroll
        for (int e = 0; e < 8; ++e) a[e] = Mm[state_term(lane, e)][i];
        put(blk + w.mt(), WsLayout::SQ, x, a);
      }
    }
  }
}

template <int DC, int DK, typename TIN>
__global__ __launch_bounds__(256) void prep_kernel(SeqParams p) {
  __shared__ PrepShared<DK> sh;
  const int tid = threadIdx.x, nt = 256;
  const int h = blockIdx.x % p.H, c = blockIdx.x / p.H;
  const ChunkRow row = chunk_row(p, c);
  if (row.count == 0) return;
  const WsLayout w{DK, p.dv, false, p.bwd};
  unsigned char* blk = p.ws + (int64_t(c) * p.H + h) * w.block();

  load_chunk<DC, DK, TIN>(sh, p, row, h, tid, nt);
  pair_products<DC, DK>(sh, p, h, tid, nt);
  if (p.delta) {
    if (tid < 64) solve(sh, tid);
    __syncthreads();
  }
  float* dec = reinterpret_cast<float*>(blk + w.dec());
  float* beta = reinterpret_cast<float*>(blk + w.beta());
  for (int r = tid; r < DK; r += nt) dec[r] = __expf(prep_l<DC>(sh, CT - 1, r));
  if (tid < CT) beta[tid] = sh.beta[tid];

  constexpr int NP = DK / 8;
  for (int x = tid; x < CT * NP; x += nt) {
    const int t = x / NP, k0 = 8 * (x % NP), at = piece_at<NP>(t, x % NP);
    float a[8], b[8], d[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int r = k0 + e;
      const float l = prep_l<DC>(sh, t, r);
      a[e] = sh.k[t][r] * __expf(l);
      b[e] = sh.q[t][r] * __expf(prep_lq<DC>(sh, t, r));
      d[e] = sh.k[t][r] * __expf(prep_l<DC>(sh, CT - 1, r) - l);
    }
    if (p.delta) put(blk + w.kh(), w.plane(), at, a);
    put(blk + w.qh(), w.plane(), at, b);
    put(blk + w.kb(), w.plane(), at, d);
  }
  put_squares<256>(blk, w, p, sh.P, sh.Nm, sh.Mm, tid);
}

// The same for bf16 keys and queries with one log-decay per head or none, one wave per
// (chunk, head): the operands of k k^T and q k^T come straight from memory, exact in bf16, and
// only the squares and the row factors are written.
template <int DK>
__global__ __launch_bounds__(64) void raw_prep_kernel(SeqParams p) {
  constexpr int NKS = DK / 32;
  __shared__ float G[CT][CT + 1], P[CT][CT + 1], Mm[CT][CT + 1];
  const int lane = threadIdx.x, c16 = lane & 15, g = lane >> 4;
  const int h = blockIdx.x % p.H, c = blockIdx.x / p.H;
  const ChunkRow row = chunk_row(p, c);
  if (row.count == 0) return;
  const WsLayout w{DK, p.dv, true, p.bwd};
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
  float l = live && p.lam ? fmaxf(p.lam[tok], LOG_FLOOR) : 0.f;
  const float beta = live && p.delta ? p.beta[tok] : 0.f;
#pragma unroll
  for (int d = 1; d < CT; d *= 2) {
    const float y = __shfl_up(l, d);
    if (lane >= d) l += y;
  }
  const float lT = __shfl(l, CT - 1);
  if (lane < CT) {
    float* fac = reinterpret_cast<float*>(blk + w.beta());
    fac[lane] = beta;
    fac[CT + lane] = __expf(l);
    fac[2 * CT + lane] = __expf(lT - l);
  }
#pragma unroll
  for (int b = 0; b < 3; ++b) {                 // (0,0), (1,1), (1,0)
    const int bi = b == 0 ? 0 : 1, bj = b == 1 ? 1 : 0;
    f32x4 ag = {0.f, 0.f, 0.f, 0.f}, ap = ag;
#pragma unroll
    for (int s = 0; s < NKS; ++s) {
      if (p.delta) ag = mma(kf[bi][s], kf[bj][s], ag);
      ap = mma(qf[bi][s], kf[bj][s], ap);
    }
    const int j = 16 * bj + c16;
    const float lj = __shfl(l, j);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int i = 16 * bi + 4 * g + r;
      const float x = __expf(fminf(__shfl(l, i) - lj, 0.f));
      P[i][j] = i >= j ? ap[r] * x : 0.f;
      G[i][j] = i > j ? ag[r] * x : 0.f;
    }
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) G[4 * g + r][16 + c16] = P[4 * g + r][16 + c16] = 0.f;
  __syncthreads();
  if (p.delta) {
    // as solve(): row i of G is used at step i alone, and N's row i replaces it
    const int j = lane & 31;
    const bool second = lane >= 32;
    float y[CT];
#pragma unroll
    for (int i = 0; i < CT; ++i) {
      float s = 0.f;
#pragma unroll
      for (int m = 0; m < i; ++m) s += G[i][m] * y[m];
      const float b = __shfl(beta, i), d = i == j ? 1.f : 0.f;
      const float x = d - (second ? b * s : s);
      y[i] = second ? x : b * x;
      __syncthreads();
      if (second) Mm[i][j] = x;
      else G[i][j] = x;
    }
    __syncthreads();
  }
  put_squares<64>(blk, w, p, P, G, Mm, lane);
}

}  // namespace dl
