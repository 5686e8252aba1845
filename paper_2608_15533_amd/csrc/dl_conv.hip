// Short causal convolution of every channel: entry points and kernels.
//
// With W taps, K = W - 1, and e the sequence's state rows followed by its inputs:
//   a_t = bias + sum_j w_j e_{t+j},  y_t = act(a_t),  state after L tokens: e_L .. e_{L+K-1}.
// Gradients, with g_t = dy_t act'(a_t) (0 outside the sequence):
//   de_r = sum_j w_j g_{r-j} (+ ds_out row r - L where there is one),  dw_j = sum_t g_t e_{t+j},
//   dbias = sum_t g_t.
// Bound by memory: every input is read once and every output written once, but for the K rows that
// neighbouring stretches of a sequence share.
#include "dl_rows.hpp"

namespace dl {
namespace {

struct ConvParams {
  const void* x;
  const float *w, *bias;
  const void* s_in;          // [B,K,D] or null
  void* s_out;               // [B,K,D] (backward: gradient of s_in, or null)
  void* y;                   // (backward: dx)
  const void *dy, *ds_out;   // backward
  float* part;               // backward: [stretches][D W + D] partial sums of dw and dbias
  const int32_t *cu, *seq_slot, *slots;
  int64_t stride;
  int32_t n, N, B, D, len, blocks;   // blocks: workgroups across the channels
};

// silu(a) and its derivative from s = sigmoid(a).
template <typename T>
__device__ __forceinline__ float silu(float a) {
  return a * sigmoid<T>(a);
}
template <typename T>
__device__ __forceinline__ float silu_slope(float a) {
  const float s = sigmoid<T>(a);
  return s * (1.0f + a * (1.0f - s));
}

template <int W, int V>
struct Taps {
  float w[W][V], bias[V];
  __device__ __forceinline__ void load(const ConvParams& p, int c) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
#pragma unroll
      for (int j = 0; j < W; ++j) w[j][i] = p.w[(c + i) * W + j];
      bias[i] = p.bias ? p.bias[c + i] : 0.0f;
    }
  }
  // a_t from the rows before the newest (oldest first) and the newest.
  __device__ __forceinline__ void apply(const float (&past)[W - 1][V], const float (&x)[V],
                                        float (&a)[V]) const {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      float s = bias[i];
#pragma unroll
      for (int j = 0; j + 1 < W; ++j) s = fmaf(w[j][i], past[j][i], s);
      a[i] = fmaf(w[W - 1][i], x[i], s);
    }
  }
};

template <int R, int V>
__device__ __forceinline__ void push(float (&past)[R][V], const float (&x)[V]) {
#pragma unroll
  for (int i = 0; i < V; ++i) {
#pragma unroll
    for (int j = 0; j + 1 < R; ++j) past[j][i] = past[j + 1][i];
    past[R - 1][i] = x[i];
  }
}

// A wave: one stretch, 64 V channels.  The first stretch of a sequence also writes its final
// state: the lane that reads a state's channels is the one that writes them (s_out may be s_in).
template <int W, bool SILU, typename T>
__global__ __launch_bounds__(64) void conv_kernel(ConvParams p) {
  constexpr int V = 4, K = W - 1, U = 8;
  const int c = (int(blockIdx.x % p.blocks) * 64 + int(threadIdx.x)) * V;
  const Stretch s = find_stretch(p.cu, p.seq_slot, p.n, p.N, p.B, p.len, blockIdx.x / p.blocks);
  if (s.idle || c >= p.D) return;
  const T* x = static_cast<const T*>(p.x) + int64_t(s.first) * p.stride + c;
  T* y = static_cast<T*>(p.y) + int64_t(s.first) * p.D + c;
  const int64_t state = int64_t(s.slot) * K * p.D + c;

  float past[K][V];
  if (s.begins()) {
    Raw<V, T> in[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (p.s_in) in[k] = load_raw<V>(static_cast<const T*>(p.s_in) + state + int64_t(k) * p.D);
      else in[k] = Raw<V, T>{};
      widen_row(in[k], past[k]);
    }
    // Row L + k of (state, inputs).
    Raw<V, T> out[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int r = s.seq_len + k - K;
      if (r >= 0) {
        out[k] = load_raw<V>(x + int64_t(r) * p.stride);
      } else {
#pragma unroll
        for (int q = 0; q < K; ++q)
          if (r + K == q) out[k] = in[q];
      }
    }
#pragma unroll
    for (int k = 0; k < K; ++k)
      *reinterpret_cast<Raw<V, T>*>(static_cast<T*>(p.s_out) + state + int64_t(k) * p.D) = out[k];
  } else {
#pragma unroll
    for (int k = 0; k < K; ++k) load_row<V>(x + int64_t(k - K) * p.stride, past[k]);
  }
  if (s.count == 0) return;
  Taps<W, V> taps;
  taps.load(p, c);
  // U rows under way while the U before them are worked on; past the end the last row again.
  Raw<V, T> next[U];
  auto fetch = [&](int t) {
#pragma unroll
    for (int i = 0; i < U; ++i) next[i] = load_raw<V>(x + int64_t(min(t + i, s.count - 1)) * p.stride);
  };
  fetch(0);
  for (int t = 0; t < s.count; t += U) {
    Raw<V, T> in[U];
#pragma unroll
    for (int i = 0; i < U; ++i) in[i] = next[i];
    if (t + U < s.count) fetch(t + U);
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (t + i >= s.count) break;
      float row[V], a[V];
      widen_row(in[i], row);
      taps.apply(past, row, a);
      push(past, row);
      if (SILU) {
#pragma unroll
        for (int e = 0; e < V; ++e) a[e] = silu<T>(a[e]);
      }
      store_row<V>(y + int64_t(t + i) * p.D, a);
    }
  }
}

template <int W, bool SILU, typename T>
__global__ __launch_bounds__(64) void conv_step_kernel(ConvParams p) {
  constexpr int V = 16 / sizeof(T), K = W - 1;
  const int c = (int(blockIdx.x % p.blocks) * 64 + int(threadIdx.x)) * V;
  const int i = blockIdx.x / p.blocks;
  const int slot = p.slots ? p.slots[i] : i;
  if (c >= p.D || slot < 0 || slot >= p.B) return;
  const Raw<V, T> in = load_raw<V>(static_cast<const T*>(p.x) + int64_t(i) * p.stride + c);
  const int64_t state = int64_t(slot) * K * p.D + c;
  Raw<V, T> old[K];
#pragma unroll
  for (int k = 0; k < K; ++k) old[k] = load_raw<V>(static_cast<const T*>(p.s_in) + state + int64_t(k) * p.D);
  Taps<W, V> taps;
  taps.load(p, c);
  float past[K][V], row[V], a[V];
#pragma unroll
  for (int k = 0; k < K; ++k) widen_row(old[k], past[k]);
  widen_row(in, row);
  taps.apply(past, row, a);
  if (SILU) {
#pragma unroll
    for (int e = 0; e < V; ++e) a[e] = silu<T>(a[e]);
  }
  store_row<V>(static_cast<T*>(p.y) + int64_t(i) * p.D + c, a);
#pragma unroll
  for (int k = 0; k < K; ++k)
    *reinterpret_cast<Raw<V, T>*>(static_cast<T*>(p.s_out) + state + int64_t(k) * p.D) =
        k + 1 < K ? old[k + 1 < K ? k + 1 : k] : in;
}

// A wave: one stretch, 64 V channels.  Token t is read at step t and row t - K of de is done with it.
// The K tokens behind the stretch are read too, for their g alone.
template <int W, bool SILU, typename T>
__global__ __launch_bounds__(64) void conv_backward_kernel(ConvParams p) {
  constexpr int V = 4, K = W - 1, U = 4;
  const int c = (int(blockIdx.x % p.blocks) * 64 + int(threadIdx.x)) * V;
  const int f = blockIdx.x / p.blocks;
  const Stretch s = find_stretch(p.cu, p.seq_slot, p.n, p.N, p.B, p.len, f);
  if (c >= p.D) return;
  float dw[W][V] = {}, db[V] = {};
  if (!s.idle) {
    const T* x = static_cast<const T*>(p.x) + int64_t(s.first) * p.stride + c;
    const T* dy = static_cast<const T*>(p.dy) + int64_t(s.first) * p.D + c;
    T* dx = static_cast<T*>(p.y) + int64_t(s.first) * p.D + c;
    const int64_t state = int64_t(s.slot) * K * p.D + c;
    const bool begins = s.begins();
    const int left = s.seq_first + s.seq_len - s.first;          // tokens from here to the end
    Taps<W, V> taps;
    taps.load(p, c);
    float past[K][V], g[K][V] = {};
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (!begins) load_row<V>(x + int64_t(k - K) * p.stride, past[k]);
      else if (p.s_in) load_row<V>(static_cast<const T*>(p.s_in) + state + int64_t(k) * p.D, past[k]);
      else
#pragma unroll
        for (int e = 0; e < V; ++e) past[k][e] = 0.0f;
    }
    // Rows of de that are this stretch's: its tokens, and the state's rows where it begins.
    const int steps = s.count + K;
    Raw<V, T> next[U], above[U];
    auto fetch = [&](int t) {
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int r = min(t + i, left - 1);
        next[i] = load_raw<V>(x + int64_t(r) * p.stride);
        above[i] = load_raw<V>(dy + int64_t(r) * p.D);
      }
    };
    if (left > 0) fetch(0);                                      // else an empty sequence
    for (int t = 0; t < steps; t += U) {
      Raw<V, T> in[U], up[U];
#pragma unroll
      for (int i = 0; i < U; ++i) {
        in[i] = next[i];
        up[i] = above[i];
      }
      if (left > 0 && t + U < steps) fetch(t + U);
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int u = t + i;
        if (u >= steps) break;
        float now[V] = {};                                       // g of this token
        if (u < left) {
          float row[V], a[V];
          widen_row(in[i], row);
          widen_row(up[i], now);
          if (SILU) {
            taps.apply(past, row, a);
#pragma unroll
            for (int e = 0; e < V; ++e) now[e] *= silu_slope<T>(a[e]);
          }
          if (u < s.count) {
#pragma unroll
            for (int e = 0; e < V; ++e) {
#pragma unroll
              for (int j = 0; j < K; ++j) dw[j][e] = fmaf(now[e], past[j][e], dw[j][e]);
              dw[K][e] = fmaf(now[e], row[e], dw[K][e]);
              db[e] += now[e];
            }
          }
          push(past, row);
        }
        const int r = u - K;                                     // the row of de that is done
        if (r >= 0 || begins) {
          float d[V];
#pragma unroll
          for (int e = 0; e < V; ++e) {
            d[e] = taps.w[0][e] * now[e];
#pragma unroll
            for (int j = 1; j < W; ++j) d[e] = fmaf(taps.w[j][e], g[K - j][e], d[e]);
          }
          const int k = r - left + K;                            // the final state's row it is, if any
          if (k >= 0 && p.ds_out) {
            float more[V];
            load_row<V>(static_cast<const T*>(p.ds_out) + state + int64_t(k) * p.D, more);
#pragma unroll
            for (int e = 0; e < V; ++e) d[e] += more[e];
          }
          if (r >= 0) store_row<V>(dx + int64_t(r) * p.D, d);
          else if (p.s_out) store_row<V>(static_cast<T*>(p.s_out) + state + int64_t(r + K) * p.D, d);
        }
        push(g, now);
      }
    }
  }
  float* part = p.part + int64_t(f) * p.D * (W + 1);
#pragma unroll
  for (int e = 0; e < V; ++e) {
#pragma unroll
    for (int j = 0; j < W; ++j) part[int64_t(c + e) * W + j] = dw[j][e];
    part[int64_t(p.D) * W + c + e] = db[e];
  }
}

enum Pass { STEP, FORWARD, BACKWARD };
template <int W, bool SILU, typename T>
hipError_t launch_pass(Pass pass, const ConvParams& q, int64_t rows, hipStream_t s) {
  ConvParams p = q;
  const int v = pass == STEP ? int(16 / sizeof(T)) : 4;
  p.blocks = (p.D + 64 * v - 1) / (64 * v);
  if (pass == STEP) return start_rows(&conv_step_kernel<W, SILU, T>, rows * p.blocks, 64, p, s);
  if (pass == FORWARD) return start_rows(&conv_kernel<W, SILU, T>, rows * p.blocks, 64, p, s);
  return start_rows(&conv_backward_kernel<W, SILU, T>, rows * p.blocks, 64, p, s);
}
template <bool SILU, typename T>
hipError_t launch_width(Pass pass, const dl_conv_desc* d, const ConvParams& p, int64_t rows, hipStream_t s) {
  switch (d->width) {
    case 2: return launch_pass<2, SILU, T>(pass, p, rows, s);
    case 3: return launch_pass<3, SILU, T>(pass, p, rows, s);
    default: return launch_pass<4, SILU, T>(pass, p, rows, s);
  }
}
hipError_t launch(Pass pass, const dl_conv_desc* d, const ConvParams& p, int64_t rows, hipStream_t s) {
  const bool silu = d->activation == DL_ACT_SILU;
  if (d->in_dtype == DL_BF16)
    return silu ? launch_width<true, uint16_t>(pass, d, p, rows, s)
                : launch_width<false, uint16_t>(pass, d, p, rows, s);
  return silu ? launch_width<true, float>(pass, d, p, rows, s)
              : launch_width<false, float>(pass, d, p, rows, s);
}

// Tokens of a stretch: as long as enough waves are left (each reads W - 1 rows of its neighbours, backward twice,
// and writes a row of partial sums).  4096 tokens of 12288 channels forward and backward: 126 us with half as
// many waves, 120 with these, 128 with stretches of 32 for both; 12345 tokens of 4096 channels 49 and 47.
int stretch_len(const dl_conv_desc* d, int32_t n, int32_t tokens, bool backward) {
  const int64_t blocks = (int64_t(d->channels) + 255) / 256, waves = backward ? 2048 : 4096;
  int len = 16;
  while (len < 256 && stretches(n, tokens, 2 * len) * blocks >= waves) len *= 2;
  return len;
}

int check_desc(const dl_conv_desc* d) {
  if (!d) return DL_E_NULL;
  if (d->abi_version != DL_ABI_VERSION) return DL_E_VERSION;
  if (d->width < 2 || d->width > 4) return DL_E_UNSUPPORTED;
  if (d->activation != DL_ACT_NONE && d->activation != DL_ACT_SILU) return DL_E_UNSUPPORTED;
  if (d->channels < 8 || d->channels % 8 != 0 || d->channels > (1 << 24)) return DL_E_SHAPE;
  if (d->num_slots < 1) return DL_E_SHAPE;
  if (d->in_dtype != DL_F32 && d->in_dtype != DL_BF16) return DL_E_DTYPE;
  return DL_OK;
}

// One workgroup per (stretch or row, 256 channels) at most.
int check_grid(const dl_conv_desc* d, int64_t rows) {
  const int64_t blocks = (int64_t(d->channels) + 255) / 256;
  return grid_fits(rows * blocks, 64) ? DL_OK : DL_E_SHAPE;
}

int check_counts(const dl_conv_desc* d, int32_t n, int32_t tokens, bool backward) {
  if (n < 0 || tokens < 0 || n > d->num_slots) return DL_E_SHAPE;
  return check_grid(d, stretches(n, tokens, stretch_len(d, n, tokens, backward)));
}

int check_rows(const dl_conv_desc* d, const dl_conv_rows* r, bool any) {
  if (!r || !r->w || (any && !r->x)) return DL_E_NULL;
  if (!aligned_to(r->x, 16) || !aligned_to(r->w, 4) || !aligned_to(r->bias, 4)) return DL_E_ALIGN;
  if (any && !good_stride(r->x_stride, d->channels)) return DL_E_SHAPE;
  return DL_OK;
}

ConvParams params(const dl_conv_desc* d, const void* s_in, void* s_out, const dl_conv_rows* r, void* y,
                  int32_t n, int32_t tokens, bool backward = false) {
  ConvParams p{};
  p.x = r->x;
  p.w = r->w;
  p.bias = r->bias;
  p.s_in = s_in;
  p.s_out = s_out;
  p.y = y;
  p.stride = r->x_stride;
  p.n = n;
  p.N = tokens;
  p.B = d->num_slots;
  p.D = d->channels;
  p.len = stretch_len(d, n, tokens, backward);
  return p;
}

}  // namespace
}  // namespace dl

using namespace dl;

extern "C" {

int dl_conv_step(const dl_conv_desc* desc, const void* s_in, void* s_out, const dl_conv_rows* rows,
                 void* y, const int32_t* slots, int32_t n, hipStream_t stream) {
  DL_TRY(check_desc(desc));
  if (n < 0 || n > desc->num_slots) return DL_E_SHAPE;
  DL_TRY(check_grid(desc, n));
  if (n == 0) return DL_OK;               // nothing to do, whatever the pointers are
  if (!slots && n != desc->num_slots) return DL_E_SHAPE;
  DL_TRY(check_rows(desc, rows, true));
  if (!s_in || !s_out || !y) return DL_E_NULL;
  if (!aligned_to(s_in, 16) || !aligned_to(s_out, 16) || !aligned_to(y, 16) || !aligned_to(slots, 4))
    return DL_E_ALIGN;
  ConvParams p = params(desc, s_in, s_out, rows, y, n, n);
  p.slots = slots;
  return launch(STEP, desc, p, n, stream) == hipSuccess ? DL_OK : DL_E_HIP;
}

int dl_conv_prefill(const dl_conv_desc* desc, const void* s_in, void* s_out, const dl_conv_rows* rows,
                    void* y, const dl_tables* tables, int32_t n, int32_t tokens, hipStream_t stream) {
  DL_TRY(check_desc(desc));
  DL_TRY(check_counts(desc, n, tokens, false));
  if (n == 0) return DL_OK;               // nothing to do, whatever the pointers are
  DL_TRY(check_rows(desc, rows, tokens > 0));
  DL_TRY(check_row_tables(tables));
  if (!s_out || (tokens > 0 && !y)) return DL_E_NULL;
  if (!aligned_to(s_in, 16) || !aligned_to(s_out, 16) || !aligned_to(y, 16)) return DL_E_ALIGN;
  ConvParams p = params(desc, s_in, s_out, rows, y, n, tokens);
  p.cu = tables->cu_tokens;
  p.seq_slot = tables->seq_slot;
  const hipError_t e = launch(FORWARD, desc, p, stretches(n, tokens, p.len), stream);
  return e == hipSuccess ? DL_OK : DL_E_HIP;
}

int dl_conv_workspace_bytes(const dl_conv_desc* desc, int32_t n, int32_t tokens, size_t* bytes) {
  DL_TRY(check_desc(desc));
  DL_TRY(check_counts(desc, n, tokens, true));
  if (!bytes) return DL_E_NULL;
  const size_t rows = size_t(stretches(n, tokens, stretch_len(desc, n, tokens, true)));
  *bytes = n == 0 ? 0 : rows * size_t(desc->channels) * size_t(desc->width + 1) * sizeof(float);
  return DL_OK;
}

int dl_conv_backward(const dl_conv_desc* desc, const void* s_in, const dl_conv_rows* rows, const void* dy,
                     const void* ds_out, const dl_conv_grads* g, const dl_tables* tables, int32_t n,
                     int32_t tokens, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  DL_TRY(check_desc(desc));
  DL_TRY(check_counts(desc, n, tokens, true));
  if (n == 0) return DL_OK;               // nothing to do, whatever the pointers are
  DL_TRY(check_rows(desc, rows, tokens > 0));
  DL_TRY(check_row_tables(tables));
  if (!g || !g->dw || (rows->bias && !g->dbias) || (tokens > 0 && (!dy || !g->dx))) return DL_E_NULL;
  if (!aligned_to(s_in, 16) || !aligned_to(dy, 16) || !aligned_to(ds_out, 16) || !aligned_to(g->dx, 16) ||
      !aligned_to(g->ds, 16) || !aligned_to(g->dw, 4) || !aligned_to(g->dbias, 4))
    return DL_E_ALIGN;
  size_t need = 0;
  DL_TRY(dl_conv_workspace_bytes(desc, n, tokens, &need));
  if (!workspace) return DL_E_NULL;
  if (!aligned_to(workspace, 256)) return DL_E_ALIGN;
  if (workspace_bytes < need) return DL_E_SHAPE;
  ConvParams p = params(desc, s_in, g->ds, rows, g->dx, n, tokens, true);
  p.cu = tables->cu_tokens;
  p.seq_slot = tables->seq_slot;
  p.dy = dy;
  p.ds_out = ds_out;
  const int64_t parts = stretches(n, tokens, p.len), D = p.D, W = desc->width;
  p.part = static_cast<float*>(workspace);
  hipError_t e = launch(BACKWARD, desc, p, parts, stream);
  if (e == hipSuccess)
    e = launch_column_sums({p.part, parts, D * (W + 1), {g->dw, p.bias ? g->dbias : nullptr, nullptr}, {D * W, D, 0}},
                           stream);
  return e == hipSuccess ? DL_OK : DL_E_HIP;
}

}  // extern "C"
