// Selective state space scan: formulas and pieces that its kernels share.
//
// A channel has S states.  With raw_t = dt_t + bias, d_t = softplus(raw_t), u_t = d_t x_t:
//   h_t = a_t . h_{t-1} + u_t B_t,  a_t = e^{d_t A},   y_t = <C_t, h_t> + skip x_t,   out_t = y_t silu(z_t).
// Over a stretch of tokens h = (e^{A sum d}) . h_before + E, E what the stretch leaves from zero states:
// so all stretches of all sequences run at once for E, the states between them follow one by one
// ("join"), and all run at once again for the outputs.
// Backward, with w_t = d out_t silu(z_t) the gradient of y_t, G_t that of h_t:
//   G_t = w_t C_t + a_{t+1} . G_{t+1};  with m_t = a_t . h_{t-1}:
//   dB_t = sum over channels of G_t u_t,   dC_t = sum over channels of w_t h_t,
//   dx_t = d_t <G_t, B_t> + skip w_t,      draw_t = sigmoid(raw_t) (<G_t, A m_t> + x_t <G_t, B_t>),
//   dA = sum_t d_t G_t . m_t,  dskip = sum_t w_t x_t,  dbias = sum_t draw_t,  dz_t = dout_t y_t silu'(z_t).
// The gradient before a stretch is e^{A sum d} . G_after + F, F = sum_t (a_first .. a_t) . C_t w_t.
//
// Work is split by channel over a wave's lanes and by state over a workgroup's waves, four states
// each: B_t and C_t are the same for all lanes and come through scalar registers, sums over states
// are in a lane but for the last step, and what a token needs of its channel (d, u) is formed once
// and passed through LDS.  Bound by vector instructions: an exponential, two products and two
// sums for every (token, channel, state).
#pragma once

#include "dl_rows.hpp"

namespace dl {

struct SsmParams {
  const void *x, *dt, *z, *Bm, *Cm;
  int64_t x_stride, dt_stride, z_stride, b_stride, c_stride;
  const float *A, *skip, *bias;
  const float* h_in;            // [B,D,S] or null
  float* h_out;                 // [B,D,S] (backward: gradient of h_in, or null)
  void* y;
  const void* dy;               // backward
  const float* dh_out;          // [B,D,S] or null
  void *dx, *ddt, *dz;
  void *dB, *dC;
  const int32_t *cu, *seq_slot, *slots;
  float *E, *F, *sums;          // [stretches][S/4][D][4] twice, [stretches][D]; null: sequences whole
  float *tiles, *tile_sums;     // backward: what a stretch has left before every tile but the first,
                                // [stretches][inner][S/4][D][4], and the sums of d there, [stretches][inner][D]
  float *part;                  // backward: [stretches][D*S + 2 D] partial sums of dA, dskip, dbias
  float *rows;                  // backward: [blocks][N][2 S] partial sums of dB, dC
  int32_t n, N, B, D, S, len, blocks, inner;   // blocks: of 64 channels; inner: tiles of a stretch less one
};

__device__ __forceinline__ float decay(float d, float a2) { return __builtin_amdgcn_exp2f(d * a2); }

// log(1 + e^x) = max(x, 0) + log(1 + e), e = e^-|x|; log(1 + e) = 2 artanh(q), q = e / (2 + e) <= 1/3, with
// artanh(q) / q - 1 as a cubic in q^2, fitted for the smallest largest error (5e-9).  No step loses a small e,
// as 1 + e would, and e is made good for the rounding of its exponential's argument, so steps that barely move are
// good to (9 + |x| / 16) 2^-24 (without: 1.2 |x| 2^-24 more; three of the 14 instructions, 2% of a prompt of 8192 x 4096
// channels, 1% of a step).  Two more are slow ones; the library's two functions take 100.
__device__ __forceinline__ float softplus(float x) {
  const float t = fabsf(x) * -LOG2E, e0 = __builtin_amdgcn_exp2f(t);
  const float e = fmaf(e0, left_of(-fabsf(x), t), e0);
  const float q = e * __builtin_amdgcn_rcpf(2.0f + e), s = q * q;
  float r = fmaf(0.14012256f, s, 0.13999565f);
  r = fmaf(r, s, 0.2001085f);
  r = fmaf(r, s, 0.33333206f);
  r = fmaf(r * s, q, q);
  return fmaf(2.0f, r, fmaxf(x, 0.0f));
}

// Four consecutive values of a row that is the same for all lanes, through scalar registers.
template <typename T>
struct Four;
template <>
struct Four<float> {
  f32x4 v;
  __device__ __forceinline__ void load(const float* p) {
    typedef const __attribute__((address_space(4))) f32x4 scalar_t;
    v = *(scalar_t*)(uintptr_t)p;
  }
  __device__ __forceinline__ float at(int i) const { return v[i]; }
  __device__ __forceinline__ void settle() { asm volatile("" : "+s"(v)); }
};
template <>
struct Four<uint16_t> {
  typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
  u32x2 v;
  __device__ __forceinline__ void load(const uint16_t* p) {
    typedef const __attribute__((address_space(4))) u32x2 scalar_t;
    v = *(scalar_t*)(uintptr_t)p;
  }
  __device__ __forceinline__ float at(int i) const {
    return __uint_as_float(i & 1 ? v[i >> 1] & 0xffff0000u : v[i >> 1] << 16);
  }
  __device__ __forceinline__ void settle() { asm volatile("" : "+s"(v)); }
};
// B and C of TB tokens, a wave's four states each.  Scalar loads return in any order, so the first use
// of one waits for all: they are asked for before a tile's steps are formed and settled behind that.
template <int TB, bool WITH_C, typename T>
struct TileRows {
  Four<T> B[TB], C[WITH_C ? TB : 1];
  // Rows past the count-th are that row again.
  __device__ __forceinline__ void load(const T* b, int64_t b_stride, const T* c, int64_t c_stride, int count = TB) {
#pragma unroll
    for (int t = 0; t < TB; ++t) {
      B[t].load(b);
      b += t + 1 < count ? b_stride : 0;
      if constexpr (WITH_C) {
        C[t].load(c);
        c += t + 1 < count ? c_stride : 0;
      }
    }
  }
  __device__ __forceinline__ void settle() {
#pragma unroll
    for (int t = 0; t < TB; ++t) {
      B[t].settle();
      if constexpr (WITH_C) C[t].settle();
    }
  }
};

// A thread's values of a tile's rows, tile by tile: the tile's address is the same for all threads (scalar
// registers), the thread's offset in it 32 bits.
template <int EV, typename T>
struct Cursor {
  char* at;
  int64_t tile;          // bytes from a tile to the next
  uint32_t off;
  __device__ __forceinline__ Cursor(const void* base, int64_t stride, int64_t row, int c0, int te, int ce,
                                    int tokens)
      : at(const_cast<char*>(static_cast<const char*>(base)) + (row * stride + c0) * int64_t(sizeof(T))),
        tile(tokens * stride * int64_t(sizeof(T))),
        off(uint32_t(te) * uint32_t(stride) * uint32_t(sizeof(T)) + uint32_t(ce) * uint32_t(sizeof(T))) {}
  __device__ __forceinline__ Raw<EV, T> load() const {
    return *reinterpret_cast<const Raw<EV, T>*>(at + off);
  }
  __device__ __forceinline__ void store(const float (&x)[EV]) const {
    store_row<EV>(reinterpret_cast<T*>(at + off), x);
  }
  __device__ __forceinline__ void move(int tiles) { at += tiles * tile; }
};

__device__ __forceinline__ int wave_index() {
  return __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
}

}  // namespace dl
