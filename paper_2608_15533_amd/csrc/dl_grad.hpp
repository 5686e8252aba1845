// Gradients of queries, keys, log-decays and betas, one workgroup per (chunk, head), from what
// the two serial passes left: the state S before the chunk, the gradient D of the state after
// it, E and Z (U = beta E, Y = beta Z; U = E and Y = Z without the delta rule).
//
//   dQh = dO S^T   dKh = -Y S^T   dKb = U D^T     (token x key)
//   dP = dO U^T (i >= j)   dG = -Y U^T (i > j)    (token x token)
//   dq_i = e^{l_i} dQh_i + sum_{j<=i} dP_ij e^{l_i-l_j} k_j
//   dk_i = dk'_i + dk''_i:
//     dk'_i  = e^{l_i} dKh_i + sum_{j<i} dG_ij e^{l_i-l_j} k_j            (reads the state)
//     dk''_j = e^{l_T-l_j} dKb_j + sum_{i>=j} (dP_ij q_i + dG_ij k_i) e^{l_i-l_j}  (writes it)
//   dbeta_i = E_i . Z_i
//   dl_i = q_i dq_i + k_i dk'_i - k_i dk''_i,   dlam_t = sum_{s>=t} dl_s + sum_v (S' D)
// with S' the state after the chunk: sum_v S' D = e^{l_T} sum_v S D + sum_j Kb_j dKb_j.
// RWKV6: q_i dq_i counts towards l_{i-1}, and its bonus pair (dP_ii) goes to q, k and u alone.
//
// Each wave owns 16 keys and all tokens, as MFMA results: a lane has one key and the eight tokens
// 16 tt + 4 g + r, which are also the terms (state order) that it feeds a product over tokens, so
// keys, queries and decay factors are fetched once for both uses.  dO, E and Z go once through
// planes in LDS, from which every wave reads its operands; S and D, which no two waves share, go
// from memory to registers.
//
// Bound by the saved states and, half of the time, by the fp32 products with them: 2 x 2048 tokens,
// 32 heads of 128 x 128 (GDN, bf16) 219 us for 780 MB read and 76 MB written, 3.9 TB/s, the matrix
// cores busy in 41% of the cycles.
#pragma once

#include "dl_prep.hpp"

namespace dl {

// One key's eight tokens of a lane, in state order.
template <int LD>
__device__ __forceinline__ void lane_tokens(const uint16_t (*m)[LD], int f, int lane, float* x) {
  const int i = lane & 15, r = 4 * (lane >> 4) + (i >> 2);
  const bf16x4 a = read_column(reinterpret_cast<const unsigned char*>(&m[r][16 * f + 4 * (i & 3)]));
  const bf16x4 b = read_column(reinterpret_cast<const unsigned char*>(&m[r + 16][16 * f + 4 * (i & 3)]));
#pragma unroll
  for (int e = 0; e < 4; ++e) { x[e] = (float)a[e]; x[4 + e] = (float)b[e]; }
}
template <int LD>
__device__ __forceinline__ void lane_tokens(const float (*m)[LD], int f, int lane, float* x) {
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = m[state_term(lane, e)][16 * f + (lane & 15)];
}

// acc += m b (TR: m^T b) for the result tile of tokens 16 tt.., m lower triangular token x token,
// b a lane's eight tokens of its key.  On fp32 MFMA: what a pair gives to q_i dq_i it takes from
// k_j dk''_j, and dlam's suffix sums keep the difference, so both must see the same product (with
// operands in two bf16 halves dlam of RWKV6 came out 3e-5 off instead of 1e-6).
template <bool TR>
__device__ __forceinline__ f32x4 pair_mma(const float (*m)[SL], int tt, const float* b, f32x4 acc,
                                          int lane) {
  const int i = 16 * tt + (lane & 15), t0 = 4 * (lane >> 4);
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    if (TR ? half < tt : half > tt) continue;     // blocks that are zero
    f32x4 a;
    if constexpr (TR) {
#pragma unroll
      for (int e = 0; e < 4; ++e) a[e] = m[16 * half + t0 + e][i];
    } else {
      a = *reinterpret_cast<const f32x4*>(&m[i][16 * half + t0]);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
      acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[4 * half + e], acc, 0, 0, 0);
  }
  return acc;
}

template <int DC, int DK, int DV, typename TIN>
struct GradShared {
  static constexpr bool LO = sizeof(TIN) == 4;           // dO has a second half
  static constexpr int NP = DV / 8, HALF = CT * DV * 2;
  static constexpr int A_E = 0, A_Z = 2 * HALF, A_DO = 4 * HALF;
  ChunkIn<DC, DK, TIN> in;
  union {
    __attribute__((aligned(16))) unsigned char planes[(LO ? 6 : 5) * HALF];
    struct {
      __attribute__((aligned(16))) float dP[CT][SL], dG[CT][SL];
    };
  };
  float tok_sum[DK / 16][CT + 1];
};

// The planes' rows: dO (rows past the chunk's end as 0), E and Z, and dbeta on the way.
template <int DC, int DK, int DV, int NTH, bool DELTA, typename TIN>
__device__ __forceinline__ void load_planes(GradShared<DC, DK, DV, TIN>& sh, const SeqParams& p,
                                            const ChunkRow& row, int h, const float* E,
                                            const float* Z, int tid) {
  using Sh = GradShared<DC, DK, DV, TIN>;
  constexpr int NP = Sh::NP;
#pragma unroll
  for (int x = tid; x < CT * NP; x += NTH) {
    const int t = x / NP, pc = x % NP, at = piece_at<NP>(t, pc);
    const int from = ((pc >> 1) * CT + t) * 16 + 8 * (pc & 1);      // [value tile][token][16]
    float e[8], z[8];
    load8(E + from, e);
    if constexpr (DELTA) load8(Z + from, z);
    const TIN* d = static_cast<const TIN*>(p.d_o) +
                   (int64_t(row.first + min(t, row.count - 1)) * p.H + h) * DV + 8 * pc;
    const bool live = t < row.count;
    if constexpr (Sh::LO) {
      float o[8];
      load8(d, o);
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i] = live ? o[i] : 0.f;
      put(sh.planes + Sh::A_DO, Sh::HALF, at, o);
    } else {
      const u32x4 zero = {0, 0, 0, 0}, o = *reinterpret_cast<const u32x4*>(d);
      *reinterpret_cast<u32x4*>(sh.planes + Sh::A_DO + 16 * at) = live ? o : zero;
    }
    put(sh.planes + Sh::A_E, Sh::HALF, at, e);
    if constexpr (DELTA) {
      put(sh.planes + Sh::A_Z, Sh::HALF, at, z);
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) s += e[i] * z[i];
#pragma unroll
      for (int i = 1; i < NP; i *= 2) s += __shfl_xor(s, i);
      if (pc == 0 && live) p.dbeta[int64_t(row.first + t) * p.H + h] = s;
    }
  }
}

// Waves to a SIMD: two workgroups on a CU for 128 keys (128 registers), where that spills none.
template <int DC, int DK, typename TIN>
constexpr int grad_waves() {
  return DK == 64 ? 3 : DC == DC_BONUS || sizeof(TIN) == 4 ? 2 : 4;
}

template <int DC, int DK, int DV, bool DELTA, typename TIN>
__global__ __launch_bounds__(4 * DK, (grad_waves<DC, DK, TIN>())) void grad_kernel(SeqParams p) {
  using Sh = GradShared<DC, DK, DV, TIN>;
  constexpr int NTH = 4 * DK, NW = DK / 16, HALF = Sh::HALF, NP = Sh::NP;
  constexpr bool LO = Sh::LO;
  using Out = std::conditional_t<LO, Full, bf16x8>;      // dO's rows, and what they are multiplied with
  using By = std::conditional_t<LO, Full, Three>;
  __shared__ Sh sh;
  ChunkIn<DC, DK, TIN>& in = sh.in;
  auto& dP = sh.dP;
  auto& dG = sh.dG;
  auto& tok_sum = sh.tok_sum;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int c16 = lane & 15, g = lane >> 4;
  const int h = blockIdx.x % p.H, c = blockIdx.x / p.H;
  const WsLayout w{DK, DV, p.raw, true};
  unsigned char* blk = p.ws + (int64_t(c) * p.H + h) * w.block();
  float* du = reinterpret_cast<float*>(blk + w.du());
  const ChunkRow row = chunk_row(p, c);
  if (row.count == 0) {
    if (DC == DC_BONUS && tid < DK) du[tid] = 0.f;
    return;
  }
  const float* S = reinterpret_cast<const float*>(blk + w.s0());
  const float* D = reinterpret_cast<const float*>(blk + w.ds());

  // S and D of this lane's key, ahead of everything that is waited for
  const int mine = (((g >> 1) * DK) + 16 * wave + c16) * 16 + 8 * (g & 1);
  float xs[DV / 32][8], xd[DV / 32][8];
#pragma unroll
  for (int s = 0; s < DV / 32; ++s) {
    load8(S + mine + 2 * s * DK * 16, xs[s]);
    load8(D + mine + 2 * s * DK * 16, xd[s]);
  }
  load_planes<DC, DK, DV, NTH, DELTA, TIN>(sh, p, row, h, reinterpret_cast<const float*>(blk + w.e()),
                                    reinterpret_cast<const float*>(blk + w.z()), tid);
  in.template load<NTH, DELTA>(p, row, h, tid);   // and every thread past this point

  auto operand = [&](int at, int tt, int s) {
    return rows_operand<Full, NP>(sh.planes + at, HALF, tt, s, lane);
  };
  // Products over the value columns: token x key ...
  f32x4 aq[2], ar[2], ac[2];
  float dot = 0.f;
#pragma unroll
  for (int tt = 0; tt < 2; ++tt) aq[tt] = ar[tt] = ac[tt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int s = 0; s < DV / 32; ++s) {
#pragma unroll
    for (int e = 0; e < 8; ++e) dot += xs[s][e] * xd[s][e];
    const Full bs = full8(xs[s]), bd = full8(xd[s]);
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      if constexpr (DELTA) ar[tt] = mma(operand(Sh::A_Z, tt, s), bs, ar[tt]);
      ac[tt] = mma(operand(Sh::A_E, tt, s), bd, ac[tt]);
    }
    const By bo = operand8<By>(xs[s]);
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
      aq[tt] = mma(rows_operand<Out, NP>(sh.planes + Sh::A_DO, HALF, tt, s, lane), bo, aq[tt]);
  }
  // ... and token x token: block (0,0), (1,1) or (1,0) of dP and dG by one wave each.
  f32x4 ap = {0.f, 0.f, 0.f, 0.f}, ag = ap;
  const int bi = wave == 0 ? 0 : 1, bj = wave == 1 ? 1 : 0;
  if (wave < 3) {
#pragma unroll
    for (int s = 0; s < DV / 32; ++s) {
      const Full b = operand(Sh::A_E, bj, s);
      if constexpr (LO) {
        ap = mma(operand(Sh::A_DO, bi, s), b, ap);
      } else {
        const bf16x8 o = rows_operand<bf16x8, NP>(sh.planes + Sh::A_DO, 0, bi, s, lane);
        float a[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) a[e] = (float)o[e];
        ap = mma(full8(a), b, ap);
      }
      if constexpr (DELTA) ag = mma(operand(Sh::A_Z, bi, s), b, ag);
    }
  }
  __syncthreads();                                // the squares take the planes' place
  if (wave < 3) {
    const int j = 16 * bj + c16;
    const float bj_ = DELTA ? in.beta[j] : 1.f;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int ri = 16 * bi + 4 * g + r;
      float f = bj_;
      if (DC == DC_SCALAR) f *= exp2_of(in.l[ri][0] - in.l[j][0]);
      if constexpr (DC == DC_BONUS) {
        if (ri == j) tok_sum[0][j] = ap[r];      // the bonus pair, apart from the others
        dP[ri][j] = ri > j ? ap[r] * f : 0.f;
      } else {
        dP[ri][j] = ri >= j ? ap[r] * f : 0.f;
      }
      dG[ri][j] = ri > j ? -ag[r] * f * in.beta[ri] : 0.f;
    }
  } else if (wave == 3) {
    for (int x = lane; x < 256; x += 64) dP[x >> 4][16 + (x & 15)] = dG[x >> 4][16 + (x & 15)] = 0.f;
  }
  __syncthreads();

  f32x4 be[2];
#pragma unroll
  for (int tt = 0; tt < 2; ++tt)
    be[tt] = DELTA ? *reinterpret_cast<const f32x4*>(&in.beta[16 * tt + 4 * g])
                     : f32x4{1.f, 1.f, 1.f, 1.f};
  float ck[8], cq[8];                          // scalar log-decay: sums over this wave's keys
#pragma unroll
  for (int e = 0; e < 8; ++e) ck[e] = cq[e] = 0.f;
  float bnd_all = 0.f;

  const int key = 16 * wave + c16;
  float k[8], q[8], l[8], lq[8];
  lane_tokens(in.k, wave, lane, k);
  lane_tokens(in.q, wave, lane, q);
  const float lT = in.at(CT - 1, key);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    l[e] = in.at(state_term(lane, e), key);
    lq[e] = DC == DC_BONUS ? in.at_q(state_term(lane, e), key) : l[e];
  }
  float share = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int tt = e >> 2, r = e & 3;
    const float fl = exp2_of(l[e]), fr = exp2_of(lT - l[e]) * be[tt][r];
    aq[tt][r] *= DC == DC_BONUS ? exp2_of(lq[e]) : fl;
    ar[tt][r] *= -fl * be[tt][r];
    ac[tt][r] *= fr;
    share += k[e] * ac[tt][r];
  }
  float bnd = dot * exp2_of(lT) + share;
  bnd += __shfl_xor(bnd, 16);
  bnd += __shfl_xor(bnd, 32);

  // pairs inside the chunk
  if constexpr (DC == DC_SCALAR) {
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      aq[tt] = pair_mma<false>(dP, tt, k, aq[tt], lane);
      ac[tt] = pair_mma<true>(dP, tt, q, ac[tt], lane);
      if constexpr (DELTA) {
        ar[tt] = pair_mma<false>(dG, tt, k, ar[tt], lane);
        ac[tt] = pair_mma<true>(dG, tt, k, ac[tt], lane);
      }
    }
  } else if (!in.wide) {
    // Rows of the first half against m = l_7, of the second against m = l_23: e^{l_i - m}
    // outside the product, e^{m - l_j} inside.  The first half's rows use no token of the
    // second (0 there: its factor could overflow); the second half's factors of earlier
    // tokens are at most 1.  For dk'' the two change places.
    const float m0 = in.at(7, key), m1 = in.at(23, key);
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    float s0[8], s1[8];
    f32x4 pq[2], pr[2], pc[2];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      s0[e] = e < 4 ? k[e] * exp2_of(m0 - l[e]) : 0.f;
      s1[e] = k[e] * exp2_of(m1 - l[e]);
    }
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      pq[tt] = pair_mma<false>(dP, tt, tt ? s1 : s0, zero, lane);
      if constexpr (DELTA) pr[tt] = pair_mma<false>(dG, tt, tt ? s1 : s0, zero, lane);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int tt = e >> 2, r = e & 3;
      const float m = tt ? m1 : m0;
      const float out = exp2_of(l[e] - m);
      aq[tt][r] += pq[tt][r] * (DC == DC_BONUS ? exp2_of(lq[e] - m) : out);
      if constexpr (DELTA) ar[tt][r] += pr[tt][r] * out;
      s0[e] = q[e] * exp2_of(lq[e] - m0);
      s1[e] = e < 4 ? 0.f : q[e] * exp2_of(lq[e] - m1);
    }
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) pc[tt] = pair_mma<true>(dP, tt, tt ? s1 : s0, zero, lane);
    if constexpr (DELTA) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        s0[e] = k[e] * exp2_of(l[e] - m0);
        s1[e] = e < 4 ? 0.f : k[e] * exp2_of(l[e] - m1);
      }
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) pc[tt] = pair_mma<true>(dG, tt, tt ? s1 : s0, pc[tt], lane);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
      ac[e >> 2][e & 3] += pc[e >> 2][e & 3] * exp2_of((e < 4 ? m0 : m1) - l[e]);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int tt = e >> 2, r = e & 3, i = state_term(lane, e);
      float sq = 0.f, sr = 0.f, sc = 0.f;
#pragma unroll 1
      for (int j = 0; j < CT; ++j) {
        const float kj = widen(in.k[j][key]), qj = widen(in.q[j][key]);
        const float lj = in.at(j, key), lqj = in.at_q(j, key);
        if (j < i || (j == i && DC == DC_KEY)) {
          sq += dP[i][j] * kj * exp2_of(lq[e] - lj);
          sr += dG[i][j] * kj * exp2_of(l[e] - lj);
        }
        if (j > i || (j == i && DC == DC_KEY))
          sc += dP[j][i] * qj * exp2_of(lqj - l[e]) + dG[j][i] * kj * exp2_of(lj - l[e]);
      }
      aq[tt][r] += sq;
      ar[tt][r] += sr;
      ac[tt][r] += sc;
    }
  }

  // log-decays
  if constexpr (DC == DC_SCALAR) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      ck[e] += q[e] * aq[e >> 2][e & 3] + k[e] * (ar[e >> 2][e & 3] - ac[e >> 2][e & 3]);
    bnd_all += bnd;
    // Every product is read here, ahead of the branches around the stores below: behind a taken
    // branch the compiler has let other instructions overwrite the addend of an MFMA that was
    // still running.  So the sums may not move past them.
#pragma unroll
    for (int e = 0; e < 8; ++e) asm volatile("" : "+v"(ck[e]));
  } else {
    // suffix sums over tokens: over r in the lane, over g across lanes, then the halves
    float sum[2], after[2];
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      float s = 0.f;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        ck[4 * tt + r] = k[4 * tt + r] * (ar[tt][r] - ac[tt][r]);
        cq[4 * tt + r] = q[4 * tt + r] * aq[tt][r];
        s += ck[4 * tt + r] + cq[4 * tt + r];
      }
      float y = __shfl_down(s, 16);
      float t = s + (g < 3 ? y : 0.f);
      y = __shfl_down(t, 32);
      t += g < 2 ? y : 0.f;
      sum[tt] = __shfl(t, c16);
      y = __shfl_down(t, 16);
      after[tt] = g < 3 ? y : 0.f;
    }
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      float acc = bnd + (tt ? 0.f : sum[1]) + after[tt];
#pragma unroll
      for (int r = 3; r >= 0; --r) {
        const int t = 16 * tt + 4 * g + r;
        acc += ck[4 * tt + r];
        if (DC == DC_KEY) acc += cq[4 * tt + r];
        if (t < row.count) p.dlam[(int64_t(row.first + t) * p.H + h) * DK + key] = acc;
        if (DC == DC_BONUS) acc += cq[4 * tt + r];
      }
    }
  }

  // queries and keys
  TIN* dqp = static_cast<TIN*>(p.dq) + (int64_t(row.first) * p.H + h) * DK + key;
  TIN* dkp = static_cast<TIN*>(p.dk_) + (int64_t(row.first) * p.H + h) * DK + key;
  const float u = DC == DC_BONUS ? p.u[int64_t(h) * DK + key] : 0.f;
  float dus = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int tt = e >> 2, r = e & 3, t = 16 * tt + 4 * g + r;
    float xq = aq[tt][r], xk = ar[tt][r] + ac[tt][r];
    if constexpr (DC == DC_BONUS) {
      const float own_pair = tok_sum[0][t];
      xq += own_pair * u * k[e];
      xk += own_pair * u * q[e];
      dus += own_pair * q[e] * k[e];
    }
    if (t < row.count) {
      narrow(dqp + int64_t(t) * p.H * DK, xq);
      narrow(dkp + int64_t(t) * p.H * DK, xk);
    }
  }
  if constexpr (DC == DC_BONUS) {
    dus += __shfl_xor(dus, 16);
    dus += __shfl_xor(dus, 32);
    if (g == 0) du[key] = dus;
  }

  if constexpr (DC == DC_SCALAR) {
    // without a log-decay too: only the store is left out (what follows the products directly
    // is the same for every call)
#pragma unroll
    for (int d = 1; d < 16; d *= 2) {
      bnd_all += __shfl_xor(bnd_all, d);
#pragma unroll
      for (int e = 0; e < 8; ++e) ck[e] += __shfl_xor(ck[e], d);
    }
    if (c16 == 0) {
#pragma unroll
      for (int e = 0; e < 8; ++e) tok_sum[wave][state_term(lane, e)] = ck[e];
      if (g == 0) tok_sum[wave][CT] = bnd_all;
    }
    __syncthreads();
    if (tid < 64) {
      float s = 0.f;
      if (tid <= CT)
#pragma unroll
        for (int x = 0; x < NW; ++x) s += tok_sum[x][tid];
#pragma unroll
      for (int d = 1; d <= CT; d *= 2) {           // suffix sums over lanes 0..CT
        const float y = __shfl_down(s, d);
        if (tid + d <= CT) s += y;
      }
      if (p.dlam && tid < row.count) p.dlam[int64_t(row.first + tid) * p.H + h] = s;
    }
  }
}

// du [H,dk]: the chunks' shares added in a fixed order, one workgroup per head.  5 us for 134
// chunks of 40 heads, of which a launch is most.
template <int DK>
__global__ __launch_bounds__(1024) void bonus_grad_kernel(SeqParams p) {
  constexpr int PARTS = 1024 / DK;
  __shared__ float sum[PARTS][DK];
  const int h = blockIdx.x, r = threadIdx.x % DK, part = threadIdx.x / DK;
  const WsLayout w{DK, p.dv, p.raw, true};
  const int last = min(p.cu_chunks[p.n], p.max_chunks);
  float s = 0.f;
  for (int c = part; c < last; c += PARTS)
    s += reinterpret_cast<const float*>(p.ws + (int64_t(c) * p.H + h) * w.block() + w.du())[r];
  sum[part][r] = s;
  __syncthreads();
  if (part == 0) {
    for (int i = 1; i < PARTS; ++i) s += sum[i][r];
    p.du[int64_t(h) * DK + r] = s;
  }
}

}  // namespace dl
