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
// Each wave owns dk/64 tiles of 16 keys and all tokens, as MFMA results: a lane has one key
// and the eight tokens 16 tt + 4 g + r, which are also the terms (state order) that it feeds a
// product over tokens, so keys, queries and decay factors are fetched once for both uses.
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

// A token x token matrix (or its transpose) as an operand over tokens.
template <bool TR>
__device__ __forceinline__ Split square_operand(const float (*m)[SL], int tt, int lane) {
  float a[8];
  const int i = 16 * tt + (lane & 15);
#pragma unroll
  for (int e = 0; e < 8; ++e) a[e] = TR ? m[state_term(lane, e)][i] : m[i][state_term(lane, e)];
  return split8(a);
}

// A token row's eight values as an operand over values; bf16 ones are exact (lo unused).
__device__ __forceinline__ Split value_operand(const uint16_t* at, bool live) {
  Split s;
  u32x4 x = *reinterpret_cast<const u32x4*>(at);
  const u32x4 zero = {0, 0, 0, 0};
  if (!live) x = zero;
  s.hi = __builtin_bit_cast(bf16x8, x);
  return s;
}
__device__ __forceinline__ Split value_operand(const float* at, bool live) {
  float x[8];
  load8(at, x);
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = live ? x[e] : 0.f;
  return split8(x);
}

template <int DC, int DK, int DV, typename TIN>
__global__ __launch_bounds__(256) void grad_kernel(SeqParams p) {
  constexpr int KT = DK / 64;                  // key tiles of a wave
  constexpr bool LO = sizeof(TIN) == 4;        // dO has a second half
  __shared__ ChunkIn<DC, DK, TIN> in;
  __shared__ __attribute__((aligned(16))) float dP[CT][SL], dG[CT][SL];
  __shared__ float tok_sum[4][CT + 1];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int c16 = lane & 15, g = lane >> 4;
  const int h = blockIdx.x % p.H, c = blockIdx.x / p.H;
  const WsLayout w{DK, p.dv, p.raw, true};
  unsigned char* blk = p.ws + (int64_t(c) * p.H + h) * w.block();
  float* du = reinterpret_cast<float*>(blk + w.du());
  const ChunkRow row = chunk_row(p, c);
  if (row.count == 0) {
    if (DC == DC_BONUS && tid < DK) du[tid] = 0.f;
    return;
  }
  const float* S = reinterpret_cast<const float*>(blk + w.s0());
  const float* D = reinterpret_cast<const float*>(blk + w.ds());
  const float* E = reinterpret_cast<const float*>(blk + w.e());
  const float* Z = reinterpret_cast<const float*>(blk + w.z());
  const TIN* dop = static_cast<const TIN*>(p.d_o) + (int64_t(row.first) * p.H + h) * p.dv;
  const int64_t do_row = int64_t(p.H) * p.dv;

  in.template load<256>(p, row, h, tid);

  // Row x, values v..v+7 of what the serial passes saved ([value tile][row][16]).
  auto saved = [](const float* m, int rows, int x, int v, float* out) {
    load8(m + ((v >> 4) * rows + x) * 16 + (v & 15), out);
  };

  // Products over the value columns: token x key ...
  f32x4 aq[KT][2], ar[KT][2], ac[KT][2];
  float dot[KT];
#pragma unroll
  for (int x = 0; x < KT; ++x) {
    dot[x] = 0.f;
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) aq[x][tt] = ar[x][tt] = ac[x][tt] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
#pragma unroll
  for (int s = 0; s < DV / 32; ++s) {
    const int v = 32 * s + 8 * g;
    Split od[2], oz[2], oe[2];
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      const int t = 16 * tt + c16;
      float x[8];
      od[tt] = value_operand(dop + min(t, row.count - 1) * do_row + v, t < row.count);
      if (p.delta) {
        saved(Z, CT, t, v, x);
        oz[tt] = split8(x);
      }
      saved(E, CT, t, v, x);
      oe[tt] = split8(x);
    }
#pragma unroll
    for (int x = 0; x < KT; ++x) {
      const int key = 16 * (wave * KT + x) + c16;
      float xs[8], xd[8];
      saved(S, DK, key, v, xs);
      saved(D, DK, key, v, xd);
#pragma unroll
      for (int e = 0; e < 8; ++e) dot[x] += xs[e] * xd[e];
      const Split bs = split8(xs), bd = split8(xd);
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        aq[x][tt] = mma(od[tt].hi, bs.lo, aq[x][tt]);
        if constexpr (LO) aq[x][tt] = mma(od[tt].lo, bs.hi, aq[x][tt]);
        aq[x][tt] = mma(od[tt].hi, bs.hi, aq[x][tt]);
        if (p.delta) ar[x][tt] = mma3(oz[tt], bs, ar[x][tt]);
        ac[x][tt] = mma3(oe[tt], bd, ac[x][tt]);
      }
    }
  }
  // ... and token x token: a block of dP and dG per wave; the last wave has dbeta.
  if (wave < 3) {
    const int bi = wave == 0 ? 0 : 1, bj = wave == 1 ? 1 : 0;   // (0,0), (1,1), (1,0)
    const int i = 16 * bi + c16, j = 16 * bj + c16;
    f32x4 ap = {0.f, 0.f, 0.f, 0.f}, ag = ap;
#pragma unroll
    for (int s = 0; s < DV / 32; ++s) {
      const int v = 32 * s + 8 * g;
      float x[8];
      saved(E, CT, j, v, x);
      const Split b = split8(x);
      const Split a = value_operand(dop + min(i, row.count - 1) * do_row + v, i < row.count);
      ap = mma(a.hi, b.lo, ap);
      if constexpr (LO) ap = mma(a.lo, b.hi, ap);
      ap = mma(a.hi, b.hi, ap);
      if (p.delta) {
        saved(Z, CT, i, v, x);
        ag = mma3(split8(x), b, ag);
      }
    }
    const float bj_ = p.delta ? in.beta[j] : 1.f;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int ri = 16 * bi + 4 * g + r;
      float f = bj_;
      if (DC == DC_SCALAR) f *= exp2_of(fminf(in.l[ri][0] - in.l[j][0], 0.f));
      if constexpr (DC == DC_BONUS) {
        if (ri == j) tok_sum[0][j] = ap[r];      // the bonus pair, apart from the others
        dP[ri][j] = ri > j ? ap[r] * f : 0.f;
      } else {
        dP[ri][j] = ri >= j ? ap[r] * f : 0.f;
      }
      dG[ri][j] = ri > j ? -ag[r] * f * in.beta[ri] : 0.f;
    }
  } else {
    for (int x = lane; x < 256; x += 64) dP[x >> 4][16 + (x & 15)] = dG[x >> 4][16 + (x & 15)] = 0.f;
    if (p.delta) {
      const int t = lane >> 1;                 // two lanes a token
      f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int v = 8 * (lane & 1); v < DV; v += 16) {
        const int at = ((v >> 4) * CT + t) * 16 + (v & 15);
#pragma unroll
        for (int y = 0; y < 8; y += 4)
          sum += *reinterpret_cast<const f32x4*>(E + at + y) * *reinterpret_cast<const f32x4*>(Z + at + y);
      }
      float s = (sum[0] + sum[1]) + (sum[2] + sum[3]);
      s += __shfl_xor(s, 1);
      if (!(lane & 1) && t < row.count) p.dbeta[int64_t(row.first + t) * p.H + h] = s;
    }
  }
  __syncthreads();

  f32x4 be[2];
#pragma unroll
  for (int tt = 0; tt < 2; ++tt)
    be[tt] = p.delta ? *reinterpret_cast<const f32x4*>(&in.beta[16 * tt + 4 * g])
                     : f32x4{1.f, 1.f, 1.f, 1.f};
  float ck[8], cq[8];                          // scalar log-decay: sums over this wave's keys
#pragma unroll
  for (int e = 0; e < 8; ++e) ck[e] = cq[e] = 0.f;
  float bnd_all = 0.f;

#pragma unroll
  for (int x = 0; x < KT; ++x) {
    const int f = wave * KT + x, key = 16 * f + c16;
    float k[8], q[8], l[8], lq[8];
    lane_tokens(in.k, f, lane, k);
    lane_tokens(in.q, f, lane, q);
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
      aq[x][tt][r] *= DC == DC_BONUS ? exp2_of(lq[e]) : fl;
      ar[x][tt][r] *= -fl * be[tt][r];
      ac[x][tt][r] *= fr;
      share += k[e] * ac[x][tt][r];
    }
    float bnd = dot[x] * exp2_of(lT) + share;
    bnd += __shfl_xor(bnd, 16);
    bnd += __shfl_xor(bnd, 32);

    // pairs inside the chunk
    if constexpr (DC == DC_SCALAR) {
      const Split bk = split8(k), bq = split8(q);
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        const Split a = square_operand<false>(dP, tt, lane), at = square_operand<true>(dP, tt, lane);
        aq[x][tt] = mma3(a, bk, aq[x][tt]);
        ac[x][tt] = mma3(at, bq, ac[x][tt]);
        if (p.delta) {
          const Split b = square_operand<false>(dG, tt, lane), bt = square_operand<true>(dG, tt, lane);
          ar[x][tt] = mma3(b, bk, ar[x][tt]);
          ac[x][tt] = mma3(bt, bk, ac[x][tt]);
        }
      }
    } else if (!in.wide) {
      // Rows of the first half against m = l_7, of the second against m = l_23: e^{l_i - m}
      // outside the product, e^{m - l_j} inside.  The first half's rows use no token of the
      // second (0 there: its factor could overflow); the second half's factors of earlier
      // tokens are at most 1.  For dk'' the two change places.
      const float m0 = in.at(7, key), m1 = in.at(23, key);
      float kin0[8], kin1[8], s0[8], s1[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        kin0[e] = e < 4 ? k[e] * exp2_of(m0 - l[e]) : 0.f;
        kin1[e] = k[e] * exp2_of(m1 - l[e]);
      }
      const Split bk0 = split8(kin0), bk1 = split8(kin1);
      f32x4 zero = {0.f, 0.f, 0.f, 0.f};
      f32x4 pq[2], pr[2], pc[2];
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        const Split a = square_operand<false>(dP, tt, lane);
        const Split ax = square_operand<false>(dG, tt, lane);
        pq[tt] = mma3(a, tt ? bk1 : bk0, zero);
        pr[tt] = p.delta ? mma3(ax, tt ? bk1 : bk0, zero) : zero;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        s0[e] = q[e] * exp2_of(lq[e] - m0);
        s1[e] = e < 4 ? 0.f : q[e] * exp2_of(lq[e] - m1);
      }
      const Split bq0 = split8(s0), bq1 = split8(s1);
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
        pc[tt] = mma3(square_operand<true>(dP, tt, lane), tt ? bq1 : bq0, zero);
      if (p.delta) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          s0[e] = k[e] * exp2_of(l[e] - m0);
          s1[e] = e < 4 ? 0.f : k[e] * exp2_of(l[e] - m1);
        }
        const Split c0 = split8(s0), c1 = split8(s1);
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
          pc[tt] = mma3(square_operand<true>(dG, tt, lane), tt ? c1 : c0, pc[tt]);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int tt = e >> 2, r = e & 3;
        const float m = tt ? m1 : m0;
        const float out = exp2_of(l[e] - m);
        aq[x][tt][r] += pq[tt][r] * (DC == DC_BONUS ? exp2_of(lq[e] - m) : out);
        ar[x][tt][r] += pr[tt][r] * out;
        ac[x][tt][r] += pc[tt][r] * exp2_of(m - l[e]);
      }
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
            sq += dP[i][j] * kj * exp2_of(fminf(lq[e] - lj, 0.f));
            sr += dG[i][j] * kj * exp2_of(l[e] - lj);
          }
          if (j > i || (j == i && DC == DC_KEY))
            sc += dP[j][i] * qj * exp2_of(fminf(lqj - l[e], 0.f)) + dG[j][i] * kj * exp2_of(lj - l[e]);
        }
        aq[x][tt][r] += sq;
        ar[x][tt][r] += sr;
        ac[x][tt][r] += sc;
      }
    }

    // log-decays
    if constexpr (DC == DC_SCALAR) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        ck[e] += q[e] * aq[x][e >> 2][e & 3] + k[e] * (ar[x][e >> 2][e & 3] - ac[x][e >> 2][e & 3]);
      bnd_all += bnd;
    } else {
      // suffix sums over tokens: over r in the lane, over g across lanes, then the halves
      float sum[2], after[2];
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        float s = 0.f;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          ck[4 * tt + r] = k[4 * tt + r] * (ar[x][tt][r] - ac[x][tt][r]);
          cq[4 * tt + r] = q[4 * tt + r] * aq[x][tt][r];
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
      float xq = aq[x][tt][r], xk = ar[x][tt][r] + ac[x][tt][r];
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
  }

  if constexpr (DC == DC_SCALAR) {
    if (p.dlam) {
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
        if (tid <= CT) s = tok_sum[0][tid] + tok_sum[1][tid] + tok_sum[2][tid] + tok_sum[3][tid];
#pragma unroll
        for (int d = 1; d <= CT; d *= 2) {         // suffix sums over lanes 0..CT
          const float y = __shfl_down(s, d);
          if (tid + d <= CT) s += y;
        }
        if (tid < row.count) p.dlam[int64_t(row.first + tid) * p.H + h] = s;
      }
    }
  }
}

// du [H,dk]: the chunks' shares added in a fixed order, one workgroup per head.
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
