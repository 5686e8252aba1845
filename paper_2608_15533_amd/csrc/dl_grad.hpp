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
#pragma once

#include "dl_prep.hpp"

namespace dl {

template <int DK>
struct GradShared {
  PrepShared<DK> in;
  float dq[CT][DK + 1], dkr[CT][DK + 1], dkc[CT][DK + 1];
  float dP[CT][CT + 1], dG[CT][CT + 1];
  float bnd[DK];
  float tok_sum[CT];
};

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

template <int DC, int DK, typename TIN>
__global__ __launch_bounds__(256) void grad_kernel(SeqParams p) {
  __shared__ GradShared<DK> sh;
  PrepShared<DK>& in = sh.in;
  const int tid = threadIdx.x, nt = 256, lane = tid & 63, wave = tid >> 6;
  const int c16 = lane & 15, g = lane >> 4;
  const int h = blockIdx.x % p.H, c = blockIdx.x / p.H;
  const WsLayout w{DK, p.dv, p.raw, true};
  unsigned char* blk = p.ws + (int64_t(c) * p.H + h) * w.block();
  float* du = reinterpret_cast<float*>(blk + w.du());
  const ChunkRow row = chunk_row(p, c);
  if (row.count == 0) {
    if (DC == DC_BONUS)
      for (int r = tid; r < DK; r += nt) du[r] = 0.f;
    return;
  }
  const float* S = reinterpret_cast<const float*>(blk + w.s0());
  const float* D = reinterpret_cast<const float*>(blk + w.ds());
  const float* E = reinterpret_cast<const float*>(blk + w.e());
  const float* Z = reinterpret_cast<const float*>(blk + w.z());
  const TIN* dop = static_cast<const TIN*>(p.d_o) + (int64_t(row.first) * p.H + h) * p.dv;

  load_chunk<DC, DK, TIN>(in, p, row, h, tid, nt);

  auto do_row = [&](int t, int v, float* x) {
    load8(dop + int64_t(min(t, row.count - 1)) * p.H * p.dv + v, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = t < row.count ? x[e] : 0.f;
  };
  auto scaled = [&](const float* m, int t, int v, float f, float* x) {
    load8(m + t * p.dv + v, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= f;
  };

  // token x key products over the value columns
  for (int kt = wave; kt < DK / 16; kt += 4) {
    const int key = 16 * kt + c16;
    f32x4 aq[2], ar[2], ac[2];
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) aq[tt] = ar[tt] = ac[tt] = f32x4{0.f, 0.f, 0.f, 0.f};
    float dot = 0.f;
    for (int s = 0; s < p.dv / 32; ++s) {
      const int v = 32 * s + 8 * g;
      float xs[8], xd[8], x[8];
      load8(S + key * p.dv + v, xs);
      load8(D + key * p.dv + v, xd);
#pragma unroll
      for (int e = 0; e < 8; ++e) dot += xs[e] * xd[e];
      const Split bs = split8(xs), bd = split8(xd);
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        const int t = 16 * tt + c16;
        const float be = p.delta ? in.beta[t] : 1.f;
        do_row(t, v, x);
        aq[tt] = mma3(split8(x), bs, aq[tt]);
        if (p.delta) {
          scaled(Z, t, v, -be, x);
          ar[tt] = mma3(split8(x), bs, ar[tt]);
        }
        scaled(E, t, v, be, x);
        ac[tt] = mma3(split8(x), bd, ac[tt]);
      }
    }
    float share = 0.f;                       // sum_j Kb_j dKb_j
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int t = 16 * tt + 4 * g + r;
        const float l = prep_l<DC>(in, t, key);
        const float dkb = ac[tt][r] * __expf(prep_l<DC>(in, CT - 1, key) - l);
        share += in.k[t][key] * dkb;
        sh.dq[t][key] = aq[tt][r] * __expf(prep_lq<DC>(in, t, key));
        sh.dkr[t][key] = ar[tt][r] * __expf(l);
        sh.dkc[t][key] = dkb;
      }
    dot = dot * __expf(prep_l<DC>(in, CT - 1, key)) + share;
    dot += __shfl_xor(dot, 16);
    dot += __shfl_xor(dot, 32);
    if (g == 0) sh.bnd[key] = dot;
  }
  // token x token products
  for (int task = wave; task < 8; task += 4) {
    const bool isP = task & 1;
    const int bi = task >> 2, bj = (task >> 1) & 1;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    if (bi >= bj && (isP || p.delta)) {
      for (int s = 0; s < p.dv / 32; ++s) {
        const int v = 32 * s + 8 * g, i = 16 * bi + c16, j = 16 * bj + c16;
        float a[8], b[8];
        if (isP) do_row(i, v, a);
        else scaled(Z, i, v, -in.beta[i], a);
        scaled(E, j, v, p.delta ? in.beta[j] : 1.f, b);
        acc = mma3(split8(a), split8(b), acc);
      }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int i = 16 * bi + 4 * g + r, j = 16 * bj + c16;
      if (isP) sh.dP[i][j] = i >= j ? acc[r] : 0.f;
      else sh.dG[i][j] = i > j ? acc[r] : 0.f;
    }
  }
  // dbeta
  if (p.delta) {
    const int t = tid >> 3, part = tid & 7;      // eight lanes per token
    float s = 0.f;
    for (int v = part; v < p.dv; v += 8) s += E[t * p.dv + v] * Z[t * p.dv + v];
    s += __shfl_xor(s, 1);
    s += __shfl_xor(s, 2);
    s += __shfl_xor(s, 4);
    if (part == 0 && t < row.count) p.dbeta[int64_t(row.first + t) * p.H + h] = s;
  }
  __syncthreads();

  // pairs inside the chunk, a key per thread and the tokens split over the rest
  constexpr int PER = 256 / DK;
  const int r = tid % DK, part = tid / DK;
  for (int i = part; i < CT; i += PER) {
    float aq = 0.f, ar = 0.f, ac = 0.f;
    const float li = prep_l<DC>(in, i, r), lqi = prep_lq<DC>(in, i, r);
    for (int j = 0; j < i; ++j) {
      const float lj = prep_l<DC>(in, j, r), kj = in.k[j][r];
      aq += sh.dP[i][j] * kj * __expf(fminf(lqi - lj, 0.f));
      ar += sh.dG[i][j] * kj * __expf(li - lj);
    }
    if (DC != DC_BONUS) aq += sh.dP[i][i] * in.k[i][r];
    for (int m = i + 1; m < CT; ++m) {
      const float lm = prep_l<DC>(in, m, r), lqm = prep_lq<DC>(in, m, r);
      ac += sh.dP[m][i] * in.q[m][r] * __expf(fminf(lqm - li, 0.f)) +
            sh.dG[m][i] * in.k[m][r] * __expf(lm - li);
    }
    if (DC != DC_BONUS) ac += sh.dP[i][i] * in.q[i][r];
    sh.dq[i][r] += aq;
    sh.dkr[i][r] += ar;
    sh.dkc[i][r] += ac;
  }
  __syncthreads();

  // log-decays: suffix sums over the chunk's tokens
  if constexpr (DC == DC_SCALAR) {
    if (p.dlam) {
      const int t = tid >> 3, sub = tid & 7;       // eight lanes per token
      float s = 0.f, bs = 0.f;
      for (int x = sub; x < DK; x += 8) {
        s += in.q[t][x] * sh.dq[t][x] + in.k[t][x] * (sh.dkr[t][x] - sh.dkc[t][x]);
        bs += sh.bnd[x];
      }
#pragma unroll
      for (int d = 1; d < 8; d *= 2) {
        s += __shfl_xor(s, d);
        bs += __shfl_xor(bs, d);
      }
      if (sub == 0) sh.tok_sum[t] = s;
      __syncthreads();
      if (sub == 0 && t < row.count) {
        float acc = bs;
        for (int m = CT - 1; m >= t; --m) acc += sh.tok_sum[m];
        p.dlam[int64_t(row.first + t) * p.H + h] = acc;
      }
    }
  } else if (tid < DK) {
    float acc = sh.bnd[tid];
    for (int t = CT - 1; t >= 0; --t) {
      const float fromq = in.q[t][tid] * sh.dq[t][tid];
      acc += in.k[t][tid] * (sh.dkr[t][tid] - sh.dkc[t][tid]);
      if (DC == DC_KEY) acc += fromq;
      if (t < row.count) p.dlam[(int64_t(row.first + t) * p.H + h) * DK + tid] = acc;
      if (DC == DC_BONUS) acc += fromq;
    }
  }

  // queries and keys
  TIN* dqp = static_cast<TIN*>(p.dq) + (int64_t(row.first) * p.H + h) * DK;
  TIN* dkp = static_cast<TIN*>(p.dk_) + (int64_t(row.first) * p.H + h) * DK;
  const float ur = DC == DC_BONUS ? p.u[int64_t(h) * DK + r] : 0.f;
  for (int t = part; t < row.count; t += PER) {
    float xq = sh.dq[t][r], xk = sh.dkr[t][r] + sh.dkc[t][r];
    if (DC == DC_BONUS) {
      xq += sh.dP[t][t] * ur * in.k[t][r];
      xk += sh.dP[t][t] * ur * in.q[t][r];
    }
    narrow(dqp + int64_t(t) * p.H * DK + r, xq);
    narrow(dkp + int64_t(t) * p.H * DK + r, xk);
  }
  if (DC == DC_BONUS && tid < DK) {
    float s = 0.f;
    for (int t = 0; t < CT; ++t) s += sh.dP[t][t] * in.q[t][tid] * in.k[t][tid];
    du[tid] = s;
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
