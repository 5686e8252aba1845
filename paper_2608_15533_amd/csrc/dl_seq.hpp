// The serial passes over a sequence's chunks: forward (states and outputs) and backward
// (state gradients and value gradients).  One wave owns VT = 16 NT value columns of one
// (sequence, head) and keeps its dk x VT piece of the state (or of its gradient) in registers
// as MFMA results; columns do not meet, so waves never wait for each other.
//
// Column j of tile t of a wave is v0 + NT * (j) + t: a lane's NT values are adjacent in memory.
#pragma once

#include "dl_scan.hpp"

namespace dl {

template <int NT, typename T>
__device__ __forceinline__ void load_cols(const T* p, float* x) {
#pragma unroll
  for (int t = 0; t < NT; ++t) x[t] = widen(p[t]);
}

// Result tiles [2][NT] (tokens 16 tt + 4 g + r) as operands over the chunk's tokens.
template <int NT>
__device__ __forceinline__ Split tokens_operand(const f32x4 (&x)[2][NT], int t) {
  float a[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) a[e] = x[e >> 2][t][e & 3];
  return split8(a);
}
template <int NKT, int NT>
__device__ __forceinline__ Split state_operand(const f32x4 (&S)[NKT][NT], int s, int t) {
  float a[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) a[e] = S[2 * s + (e >> 2)][t][e & 3];
  return split8(a);
}

__device__ __forceinline__ Split plane_at(const unsigned char* base, int plane, int unit) {
  return load_split(reinterpret_cast<const uint16_t*>(base + 16 * unit),
                    reinterpret_cast<const uint16_t*>(base + plane + 16 * unit));
}

template <int DK, int NT, bool DELTA, typename TIN>
__global__ __launch_bounds__(64) void forward_kernel(SeqParams p) {
  constexpr int NKT = DK / 16, NKS = DK / 32;
  const int lane = threadIdx.x, c16 = lane & 15, g = lane >> 4;
  const int nvt = p.dv / (16 * NT);
  const int b = blockIdx.x, vt = b % nvt, h = (b / nvt) % p.H, seq = b / nvt / p.H;
  const int slot = p.seq_slot[seq];
  if (slot < 0 || slot >= p.B) return;
  const int v = 16 * NT * vt + NT * c16;
  const WsLayout w{DK, p.dv, p.bwd};
  const int64_t state_at = (int64_t(slot) * p.H + h) * DK * p.dv + v;

  f32x4 S[NKT][NT];
#pragma unroll
  for (int f = 0; f < NKT; ++f)
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int t = 0; t < NT; ++t)
        S[f][t][r] = p.S_in ? load_state(p.S_in, p.state_bf16,
                                         state_at + int64_t(16 * f + 4 * g + r) * p.dv + t)
                            : 0.f;

  const int c0 = max(p.cu_chunks[seq], 0), c1 = min(p.cu_chunks[seq + 1], p.max_chunks);
  for (int c = c0; c < c1; ++c) {
    const ChunkRow row = chunk_row(p, c);
    if (row.count == 0) continue;
    unsigned char* blk = p.ws + (int64_t(c) * p.H + h) * w.block();
    const TIN* vp = static_cast<const TIN*>(p.v) + (int64_t(row.first) * p.H + h) * p.dv + v;
    f32x4 U[2][NT], O[2][NT];
    // V, rows past the chunk's end as 0
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int tok = 16 * tt + 4 * g + r;
        float x[NT];
        load_cols<NT>(vp + int64_t(min(tok, row.count - 1)) * p.H * p.dv, x);
#pragma unroll
        for (int t = 0; t < NT; ++t) U[tt][t][r] = tok < row.count ? x[t] : 0.f;
      }
    if (p.bwd) {
      float* s0 = reinterpret_cast<float*>(blk + w.s0()) + v;
#pragma unroll
      for (int f = 0; f < NKT; ++f)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int t = 0; t < NT; ++t) s0[(16 * f + 4 * g + r) * p.dv + t] = S[f][t][r];
    }
    // Kh S and Qh S
    f32x4 X[2][NT];
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
      for (int t = 0; t < NT; ++t) O[tt][t] = X[tt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < NKS; ++s) {
      Split sb[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) sb[t] = state_operand<NKT, NT>(S, s, t);
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        const int unit = (tt * NKS + s) * 64 + lane;
        if constexpr (DELTA) {
          const Split a = plane_at(blk + w.kh(), w.plane(), unit);
#pragma unroll
          for (int t = 0; t < NT; ++t) X[tt][t] = mma3(a, sb[t], X[tt][t]);
        }
        const Split a = plane_at(blk + w.qh(), w.plane(), unit);
#pragma unroll
        for (int t = 0; t < NT; ++t) O[tt][t] = mma3(a, sb[t], O[tt][t]);
      }
    }
    if constexpr (DELTA) {
      Split rb[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) U[tt][t] -= X[tt][t];
        rb[t] = tokens_operand<NT>(U, t);
      }
      const float* beta = reinterpret_cast<const float*>(blk + w.beta());
      float* eo = reinterpret_cast<float*>(blk + w.e()) + v;
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        const Split a = plane_at(blk + w.n(), w.sq(), tt * 64 + lane);
#pragma unroll
        for (int t = 0; t < NT; ++t) U[tt][t] = mma3(a, rb[t], f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int tok = 16 * tt + 4 * g + r;
          const float be = beta[tok];
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            if (p.bwd) eo[tok * p.dv + t] = U[tt][t][r];
            U[tt][t][r] *= be;
          }
        }
      }
    } else if (p.bwd) {
      float* eo = reinterpret_cast<float*>(blk + w.e()) + v;
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int t = 0; t < NT; ++t) eo[(16 * tt + 4 * g + r) * p.dv + t] = U[tt][t][r];
    }
    Split ub[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) ub[t] = tokens_operand<NT>(U, t);
    // S <- e^{l_T} S + Kb^T U
    const float* dec = reinterpret_cast<const float*>(blk + w.dec());
#pragma unroll
    for (int f = 0; f < NKT; ++f) {
      const f32x4 d = *reinterpret_cast<const f32x4*>(dec + 16 * f + 4 * g);
      const Split a = plane_at(blk + w.kbt(), w.plane(), f * 64 + lane);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int r = 0; r < 4; ++r) S[f][t][r] *= d[r];
        S[f][t] = mma3(a, ub[t], S[f][t]);
      }
    }
    if (p.o) {
      TIN* op = static_cast<TIN*>(p.o) + (int64_t(row.first) * p.H + h) * p.dv + v;
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        const Split a = plane_at(blk + w.p(), w.sq(), tt * 64 + lane);
#pragma unroll
        for (int t = 0; t < NT; ++t) O[tt][t] = mma3(a, ub[t], O[tt][t]);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int tok = 16 * tt + 4 * g + r;
          if (tok < row.count)
#pragma unroll
            for (int t = 0; t < NT; ++t) narrow(op + int64_t(tok) * p.H * p.dv + t, O[tt][t][r]);
        }
      }
    }
  }
  if (p.S_out) {
#pragma unroll
    for (int f = 0; f < NKT; ++f)
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int t = 0; t < NT; ++t)
          store_state(p.S_out, p.state_bf16, state_at + int64_t(16 * f + 4 * g + r) * p.dv + t,
                      S[f][t][r]);
  }
}

// Backward over the chunks, last to first, with D the gradient of the state after a chunk:
//   dU = P^T dO + Kb D      Z = M^T dU,  Y = beta Z   (no delta rule: Y = dU)
//   dV = Y                  D <- e^{l_T} D + Qh^T dO - Kh^T Y
template <int DK, int NT, bool DELTA, typename TIN>
__global__ __launch_bounds__(64) void backward_kernel(SeqParams p) {
  constexpr int NKT = DK / 16, NKS = DK / 32;
  const int lane = threadIdx.x, c16 = lane & 15, g = lane >> 4;
  const int nvt = p.dv / (16 * NT);
  const int b = blockIdx.x, vt = b % nvt, h = (b / nvt) % p.H, seq = b / nvt / p.H;
  const int slot = p.seq_slot[seq];
  if (slot < 0 || slot >= p.B) return;
  const int v = 16 * NT * vt + NT * c16;
  const WsLayout w{DK, p.dv, true};
  const int64_t state_at = (int64_t(slot) * p.H + h) * DK * p.dv + v;

  f32x4 D[NKT][NT];
#pragma unroll
  for (int f = 0; f < NKT; ++f)
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int t = 0; t < NT; ++t)
        D[f][t][r] = p.dS_out ? load_state(p.dS_out, p.state_bf16,
                                           state_at + int64_t(16 * f + 4 * g + r) * p.dv + t)
                              : 0.f;

  const int c0 = max(p.cu_chunks[seq], 0), c1 = min(p.cu_chunks[seq + 1], p.max_chunks);
  for (int c = c1 - 1; c >= c0; --c) {
    const ChunkRow row = chunk_row(p, c);
    if (row.count == 0) continue;
    unsigned char* blk = p.ws + (int64_t(c) * p.H + h) * w.block();
    const int64_t at = (int64_t(row.first) * p.H + h) * p.dv + v;
    const TIN* dop = static_cast<const TIN*>(p.d_o) + at;
    f32x4 G[2][NT];                        // dO
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int tok = 16 * tt + 4 * g + r;
        float x[NT];
        load_cols<NT>(dop + int64_t(min(tok, row.count - 1)) * p.H * p.dv, x);
#pragma unroll
        for (int t = 0; t < NT; ++t) G[tt][t][r] = tok < row.count ? x[t] : 0.f;
      }
    float* ds = reinterpret_cast<float*>(blk + w.ds()) + v;
#pragma unroll
    for (int f = 0; f < NKT; ++f)
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int t = 0; t < NT; ++t) ds[(16 * f + 4 * g + r) * p.dv + t] = D[f][t][r];

    Split gb[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) gb[t] = tokens_operand<NT>(G, t);
    f32x4 Y[2][NT];
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      const Split a = plane_at(blk + w.pt(), w.sq(), tt * 64 + lane);
#pragma unroll
      for (int t = 0; t < NT; ++t) Y[tt][t] = mma3(a, gb[t], f32x4{0.f, 0.f, 0.f, 0.f});
    }
#pragma unroll
    for (int s = 0; s < NKS; ++s) {
      Split sb[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) sb[t] = state_operand<NKT, NT>(D, s, t);
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        const Split a = plane_at(blk + w.kb(), w.plane(), (tt * NKS + s) * 64 + lane);
#pragma unroll
        for (int t = 0; t < NT; ++t) Y[tt][t] = mma3(a, sb[t], Y[tt][t]);
      }
    }
    if constexpr (DELTA) {
      Split rb[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) rb[t] = tokens_operand<NT>(Y, t);
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        const Split a = plane_at(blk + w.mt(), w.sq(), tt * 64 + lane);
#pragma unroll
        for (int t = 0; t < NT; ++t) Y[tt][t] = mma3(a, rb[t], f32x4{0.f, 0.f, 0.f, 0.f});
      }
    }
    const float* beta = reinterpret_cast<const float*>(blk + w.beta());
    float* zo = reinterpret_cast<float*>(blk + w.z()) + v;
    TIN* dvp = static_cast<TIN*>(p.dv_) + at;
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int tok = 16 * tt + 4 * g + r;
        const float be = DELTA ? beta[tok] : 1.f;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          zo[tok * p.dv + t] = Y[tt][t][r];
          Y[tt][t][r] *= be;
          if (tok < row.count) narrow(dvp + int64_t(tok) * p.H * p.dv + t, Y[tt][t][r]);
        }
      }
    Split yb[NT];
    if constexpr (DELTA) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) Y[tt][t] = -Y[tt][t];
        yb[t] = tokens_operand<NT>(Y, t);
      }
    }
    const float* dec = reinterpret_cast<const float*>(blk + w.dec());
#pragma unroll
    for (int f = 0; f < NKT; ++f) {
      const f32x4 d = *reinterpret_cast<const f32x4*>(dec + 16 * f + 4 * g);
      const Split a = plane_at(blk + w.qht(), w.plane(), f * 64 + lane);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int r = 0; r < 4; ++r) D[f][t][r] *= d[r];
        D[f][t] = mma3(a, gb[t], D[f][t]);
      }
      if constexpr (DELTA) {
        const Split ak = plane_at(blk + w.kht(), w.plane(), f * 64 + lane);
#pragma unroll
        for (int t = 0; t < NT; ++t) D[f][t] = mma3(ak, yb[t], D[f][t]);
      }
    }
  }
  if (p.S_out) {
#pragma unroll
    for (int f = 0; f < NKT; ++f)
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int t = 0; t < NT; ++t)
          store_state(p.S_out, p.state_bf16, state_at + int64_t(16 * f + 4 * g + r) * p.dv + t,
                      D[f][t][r]);
  }
}

}  // namespace dl
