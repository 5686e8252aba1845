// Norms of queries and keys for each head, with the rotation by position: entry points and kernels.
//
// For a head x of a token at position p, with r = (c sum x^2 + eps)^(-1/2), c = 1 (L2) or 1 / d (root
// mean square), r = 1 without a norm:  n = scale r (w . x);  of the first rot places those of a pair
// (a, b) become (a cos - b sin, a sin + b cos) with the angle p freq_i.  Every head is written rep times.
// Gradients, g the sum over the rep copies turned back and scaled:  dw = sum g r x,
// dx = r (w . g) - x c r^3 <w . g, x>.
// Bound by memory: every head is read once and written rep times.
#include <float.h>

#include "dl_rows.hpp"

namespace dl {
namespace {

struct QkParams {
  const void *q, *k;
  void *qo, *ko;               // outputs (backward: dq, dk)
  const void *dqo, *dko;       // backward
  const int32_t *pos, *used;
  const float *freq, *wq, *wk;
  float* part;                 // backward: [workgroups, 2, d] partial sums, or null
  int64_t q_stride, k_stride;
  float share, eps, q_scale;   // share: c above
  int32_t N, H, rep, rot, per; // per: tokens of a workgroup
};

constexpr int NT = 256;        // threads of a workgroup
constexpr int V = 8;           // values of a head that a lane holds, in two fours
constexpr int U = 2;           // heads of queries and of keys that a lane has under way

// cos and sin of position x frequency, the product in 64 bits: an angle of a million radians keeps
// all of its fraction of a turn.
__device__ __forceinline__ float2 turn_of(int pos, float freq) {
  const double turns = double(pos) * double(freq) * 0.15915494309189533577;
  const float part = float(turns - rint(turns));
  float2 cs;
  sincospif(2.0f * part, &cs.y, &cs.x);
  return cs;
}

// A lane's places in a head: eight in a row, but with halves that turn both places of four pairs, so
// that no lane needs another's.
enum Turn { NONE = DL_TURN_NONE, HALVES = DL_TURN_HALVES, PAIRS = DL_TURN_PAIRS };
template <int T>
struct Places {
  int lo, hi;                  // first places of the two fours
  bool turned;
  __device__ __forceinline__ Places(int li, int rot) {
    turned = T != NONE && li * V < rot;
    lo = T == HALVES && turned ? li * 4 : li * V;
    hi = T == HALVES && turned ? rot / 2 + li * 4 : li * V + 4;
  }
  template <typename E>
  __device__ __forceinline__ void load(const E* row, Raw<4, E> (&r)[2]) const {
    r[0] = load_raw<4>(row + lo);
    r[1] = load_raw<4>(row + hi);
  }
  template <typename E>
  __device__ __forceinline__ void store(E* row, const float (&x)[V]) const {
    const float a[4] = {x[0], x[1], x[2], x[3]}, b[4] = {x[4], x[5], x[6], x[7]};
    store_row<4>(row + lo, a);
    store_row<4>(row + hi, b);
  }
  __device__ __forceinline__ int at(int i) const { return i < 4 ? lo + i : hi + i - 4; }
};
template <typename E>
__device__ __forceinline__ void widen_fours(const Raw<4, E> (&r)[2], float (&x)[V]) {
#pragma unroll
  for (int i = 0; i < V; ++i) x[i] = r[i >> 2].get(i & 3);
}

// The angles of a lane's four pairs.
template <int T>
struct Angles {
  float c[4], s[4];
  __device__ __forceinline__ Angles(const float2* lds, int li, bool turned) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 cs = T != NONE && turned ? lds[4 * li + i] : make_float2(1.0f, 0.0f);
      c[i] = cs.x;
      s[i] = cs.y;
    }
  }
  // Turned by the angles, or back.
  __device__ __forceinline__ void apply(float (&x)[V], bool back) const {
    if (T == NONE) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int u = T == HALVES ? i : 2 * i, v = T == HALVES ? i + 4 : 2 * i + 1;
      const float sn = back ? -s[i] : s[i], a = x[u], b = x[v];
      x[u] = fmaf(a, c[i], -b * sn);
      x[v] = fmaf(a, sn, b * c[i]);
    }
  }
};

// The angles of `count` tokens, a thread for each: 256 are one turn of the workgroup.
template <int T>
__device__ __forceinline__ void fill_angles(const QkParams& p, int64_t first, int count, float2* lds) {
  if (T == NONE) return;
  const int half = p.rot / 2;
  for (int i = threadIdx.x; i < count * half; i += NT) lds[i] = turn_of(p.pos[first + i / half], p.freq[i % half]);
  __syncthreads();
}

constexpr int MOST = 8;        // tokens of a workgroup

// A workgroup: `per` tokens, one after the other; D / 8 lanes a head.
template <int D, int T, bool NORM, typename E>
__global__ __launch_bounds__(NT) void qk_kernel(QkParams p) {
  constexpr int LPH = D / V, HEADS = NT / LPH;
  __shared__ float2 lds[T == NONE ? 1 : MOST * D / 2];
  const int li = threadIdx.x % LPH, group = threadIdx.x / LPH;
  const int rows = p.used ? min(max(*p.used, 0), p.N) : p.N;
  const int64_t first = int64_t(blockIdx.x) * p.per;
  const int count = int(min(int64_t(p.per), rows - first));
  if (count <= 0) return;
  const Places<T> place(li, p.rot);
  float w[2][V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    w[0][i] = (p.wq ? p.wq[place.at(i)] : 1.0f) * p.q_scale;
    w[1][i] = p.wk ? p.wk[place.at(i)] : 1.0f;
  }
  fill_angles<T>(p, first, count, lds);
  for (int j = 0; j < count; ++j) {
    const int64_t token = first + j;
    const Angles<T> turn(lds + j * (p.rot / 2), li, place.turned);
    const E* in[2] = {static_cast<const E*>(p.q) + token * p.q_stride, static_cast<const E*>(p.k) + token * p.k_stride};
    E* out[2] = {static_cast<E*>(p.qo) + token * p.H * p.rep * D, static_cast<E*>(p.ko) + token * p.H * p.rep * D};
    for (int h0 = group; h0 < p.H; h0 += HEADS * U) {
      Raw<4, E> raw[2][U][2];
#pragma unroll
      for (int kind = 0; kind < 2; ++kind)
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (h0 + u * HEADS < p.H) place.load(in[kind] + (h0 + u * HEADS) * D, raw[kind][u]);
#pragma unroll
      for (int kind = 0; kind < 2; ++kind)
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int h = h0 + u * HEADS;
          if (h >= p.H) break;
          float x[V];
          widen_fours(raw[kind][u], x);
          float r = 1.0f;
          if (NORM) {
            float ss = 0.0f;
#pragma unroll
            for (int i = 0; i < V; ++i) ss = fmaf(x[i], x[i], ss);
            r = __builtin_amdgcn_rsqf(fmaf(lanes_sum<LPH>(ss), p.share, p.eps));
          }
#pragma unroll
          for (int i = 0; i < V; ++i) x[i] *= r * w[kind][i];
          turn.apply(x, false);
          for (int c = 0; c < p.rep; ++c) place.store(out[kind] + (int64_t(h) * p.rep + c) * D, x);
        }
    }
  }
}

template <int D, int T, bool NORM, typename E>
__global__ __launch_bounds__(NT) void qk_backward_kernel(QkParams p) {
  constexpr int LPH = D / V, HEADS = NT / LPH;
  __shared__ float2 lds[T == NONE ? 1 : MOST * D / 2];
  __shared__ float sums[HEADS][D];
  const int li = threadIdx.x % LPH, group = threadIdx.x / LPH;
  const int rows = p.used ? min(max(*p.used, 0), p.N) : p.N;
  const int64_t first = int64_t(blockIdx.x) * p.per;
  const int count = int(max(min(int64_t(p.per), rows - first), int64_t(0)));
  const Places<T> place(li, p.rot);
  float w[2][V], dw[2][V] = {};
#pragma unroll
  for (int i = 0; i < V; ++i) {
    w[0][i] = p.wq ? p.wq[place.at(i)] : 1.0f;
    w[1][i] = p.wk ? p.wk[place.at(i)] : 1.0f;
  }
  fill_angles<T>(p, first, count, lds);
  for (int j = 0; j < count; ++j) {
    const int64_t token = first + j;
    const Angles<T> turn(lds + j * (p.rot / 2), li, place.turned);
    const E* in[2] = {static_cast<const E*>(p.q) + token * p.q_stride, static_cast<const E*>(p.k) + token * p.k_stride};
    const E* up[2] = {static_cast<const E*>(p.dqo) + token * p.H * p.rep * D,
                      static_cast<const E*>(p.dko) + token * p.H * p.rep * D};
    E* out[2] = {static_cast<E*>(p.qo) + token * p.H * D, static_cast<E*>(p.ko) + token * p.H * D};
    for (int h = group; h < p.H; h += HEADS) {
      Raw<4, E> raw[2][2], own[2][2];
#pragma unroll
      for (int kind = 0; kind < 2; ++kind) {
        place.load(in[kind] + h * D, raw[kind]);
        place.load(up[kind] + int64_t(h) * p.rep * D, own[kind]);
      }
#pragma unroll
      for (int kind = 0; kind < 2; ++kind) {
        float x[V], g[V];
        widen_fours(raw[kind], x);
        widen_fours(own[kind], g);
        for (int c = 1; c < p.rep; ++c) {
          Raw<4, E> next[2];
          float more[V];
          place.load(up[kind] + (int64_t(h) * p.rep + c) * D, next);
          widen_fours(next, more);
#pragma unroll
          for (int i = 0; i < V; ++i) g[i] += more[i];
        }
        turn.apply(g, true);
        float ss = 0.0f, along = 0.0f;
#pragma unroll
        for (int i = 0; i < V; ++i) ss = fmaf(x[i], x[i], ss);
        const float r = NORM ? __builtin_amdgcn_rsqf(fmaf(lanes_sum<LPH>(ss), p.share, p.eps)) : 1.0f;
        const float scale = (kind ? 1.0f : p.q_scale) * r;
#pragma unroll
        for (int i = 0; i < V; ++i) {
          g[i] *= scale;
          dw[kind][i] = fmaf(g[i], x[i], dw[kind][i]);
          g[i] *= w[kind][i];
          along = fmaf(g[i], x[i], along);
        }
        if (NORM) {
          const float back = lanes_sum<LPH>(along) * r * r * p.share;
#pragma unroll
          for (int i = 0; i < V; ++i) g[i] = fmaf(-back, x[i], g[i]);
        }
        place.store(out[kind] + int64_t(h) * D, g);
      }
    }
  }
  if (!p.part) return;
#pragma unroll
  for (int kind = 0; kind < 2; ++kind) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < V; ++i) sums[group][place.at(i)] = dw[kind][i];
    __syncthreads();
    if (threadIdx.x < D) {
      float s = 0.0f;
#pragma unroll
      for (int i = 0; i < HEADS; ++i) s += sums[i][threadIdx.x];
      p.part[(int64_t(blockIdx.x) * 2 + kind) * D + threadIdx.x] = s;
    }
  }
}

template <int D, int T, bool NORM, typename E>
hipError_t launch_type(const QkParams& p, bool backward, int64_t grid, hipStream_t s) {
  return backward ? start_rows(&qk_backward_kernel<D, T, NORM, E>, grid, NT, p, s)
                  : start_rows(&qk_kernel<D, T, NORM, E>, grid, NT, p, s);
}
template <int D, int T>
hipError_t launch_turn(const dl_qk_desc* d, const QkParams& p, bool backward, int64_t grid, hipStream_t s) {
  const bool norm = d->norm != DL_NORM_NONE;
  if (d->in_dtype == DL_BF16)
    return norm ? launch_type<D, T, true, uint16_t>(p, backward, grid, s)
                : launch_type<D, T, false, uint16_t>(p, backward, grid, s);
  return norm ? launch_type<D, T, true, float>(p, backward, grid, s)
              : launch_type<D, T, false, float>(p, backward, grid, s);
}
template <int D>
hipError_t launch_dim(const dl_qk_desc* d, const QkParams& p, bool backward, int64_t grid, hipStream_t s) {
  switch (d->turn) {
    case DL_TURN_HALVES: return launch_turn<D, HALVES>(d, p, backward, grid, s);
    case DL_TURN_PAIRS: return launch_turn<D, PAIRS>(d, p, backward, grid, s);
    default: return launch_turn<D, NONE>(d, p, backward, grid, s);
  }
}

// Tokens of a workgroup: they share its angles' arithmetic (12345 rows of 32 heads: 132 us with a token a
// workgroup, 79 with four), and backward the partial sums.
int tokens_per(int32_t n, bool backward) { return std::max(1, std::min(backward ? MOST : 4, n / 512)); }

int check_desc(const dl_qk_desc* d) {
  if (!d) return DL_E_NULL;
  if (d->abi_version != DL_ABI_VERSION) return DL_E_VERSION;
  if (d->head_dim != 64 && d->head_dim != 128) return DL_E_UNSUPPORTED;
  if (d->norm < DL_NORM_NONE || d->norm > DL_NORM_RMS) return DL_E_UNSUPPORTED;
  if (d->turn < DL_TURN_NONE || d->turn > DL_TURN_PAIRS) return DL_E_UNSUPPORTED;
  if (d->heads < 1 || d->rep < 1 || int64_t(d->heads) * d->rep > DL_MAX_HEADS) return DL_E_SHAPE;
  if (d->turn == DL_TURN_NONE ? d->rot != 0 : d->rot < 16 || d->rot > d->head_dim || d->rot % 16 != 0)
    return DL_E_SHAPE;
  // Without an eps above 0 a head of zeros has no norm, and the reciprocal root takes one below the normal numbers
  // for 0; what is not a number is neither.
  if (d->norm != DL_NORM_NONE && !(d->eps >= FLT_MIN)) return DL_E_UNSUPPORTED;
  if (d->in_dtype != DL_F32 && d->in_dtype != DL_BF16) return DL_E_DTYPE;
  return DL_OK;
}

int check_rows(const dl_qk_desc* d, const dl_qk_rows* r) {
  if (!r || !r->q || !r->k) return DL_E_NULL;
  if (d->turn != DL_TURN_NONE && (!r->pos || !r->freq)) return DL_E_NULL;
  if ((r->wq == nullptr) != (r->wk == nullptr)) return DL_E_NULL;
  if (!aligned_to(r->q, 16) || !aligned_to(r->k, 16) || !aligned_to(r->pos, 4) || !aligned_to(r->freq, 4) ||
      !aligned_to(r->wq, 4) || !aligned_to(r->wk, 4) || !aligned_to(r->used, 4))
    return DL_E_ALIGN;
  const int64_t width = int64_t(d->heads) * d->head_dim;
  if (!good_stride(r->q_stride, width) || !good_stride(r->k_stride, width)) return DL_E_SHAPE;
  return DL_OK;
}

QkParams params(const dl_qk_desc* d, const dl_qk_rows* r, void* qo, void* ko, int32_t n, bool backward) {
  QkParams p{};
  p.q = r->q;
  p.k = r->k;
  p.qo = qo;
  p.ko = ko;
  p.pos = r->pos;
  p.used = r->used;
  p.freq = r->freq;
  p.wq = r->wq;
  p.wk = r->wk;
  p.q_stride = r->q_stride;
  p.k_stride = r->k_stride;
  p.share = d->norm == DL_NORM_RMS ? 1.0f / float(d->head_dim) : 1.0f;
  p.eps = d->eps;
  p.q_scale = d->q_scale;
  p.N = n;
  p.H = d->heads;
  p.rep = d->rep;
  p.rot = d->rot;
  p.per = tokens_per(n, backward);
  return p;
}

hipError_t launch(const dl_qk_desc* d, const QkParams& p, bool backward, hipStream_t s) {
  const int64_t grid = (int64_t(p.N) + p.per - 1) / p.per;
  return d->head_dim == 128 ? launch_dim<128>(d, p, backward, grid, s)
                            : launch_dim<64>(d, p, backward, grid, s);
}

int check_count(int32_t n) { return n < 0 || !grid_fits(n, NT) ? DL_E_SHAPE : DL_OK; }

}  // namespace
}  // namespace dl

using namespace dl;

extern "C" {

int dl_qk_norm(const dl_qk_desc* desc, const dl_qk_rows* rows, void* q_out, void* k_out, int32_t n,
               hipStream_t stream) {
  DL_TRY(check_desc(desc));
  DL_TRY(check_count(n));
  if (n == 0) return DL_OK;               // nothing to do, whatever the pointers are
  DL_TRY(check_rows(desc, rows));
  if (!q_out || !k_out) return DL_E_NULL;
  if (!aligned_to(q_out, 16) || !aligned_to(k_out, 16)) return DL_E_ALIGN;
  return launch(desc, params(desc, rows, q_out, k_out, n, false), false, stream) == hipSuccess ? DL_OK : DL_E_HIP;
}

int dl_qk_workspace_bytes(const dl_qk_desc* desc, int32_t n, size_t* bytes) {
  DL_TRY(check_desc(desc));
  DL_TRY(check_count(n));
  if (!bytes) return DL_E_NULL;
  const int64_t per = tokens_per(n, true);
  *bytes = size_t((n + per - 1) / per) * 2 * size_t(desc->head_dim) * sizeof(float);
  return DL_OK;
}

int dl_qk_norm_backward(const dl_qk_desc* desc, const dl_qk_rows* rows, const void* dq_out, const void* dk_out,
                        const dl_qk_grads* g, int32_t n, void* workspace, size_t workspace_bytes,
                        hipStream_t stream) {
  DL_TRY(check_desc(desc));
  DL_TRY(check_count(n));
  if (n == 0) return DL_OK;               // nothing to do, whatever the pointers are
  DL_TRY(check_rows(desc, rows));
  if (!dq_out || !dk_out || !g || !g->dq || !g->dk) return DL_E_NULL;
  if (!aligned_to(dq_out, 16) || !aligned_to(dk_out, 16) || !aligned_to(g->dq, 16) || !aligned_to(g->dk, 16) ||
      !aligned_to(g->dwq, 4) || !aligned_to(g->dwk, 4))
    return DL_E_ALIGN;
  QkParams p = params(desc, rows, g->dq, g->dk, n, true);
  p.dqo = dq_out;
  p.dko = dk_out;
  if (p.wq) {
    if (!g->dwq || !g->dwk) return DL_E_NULL;
    size_t need = 0;
    DL_TRY(dl_qk_workspace_bytes(desc, n, &need));
    if (!workspace) return DL_E_NULL;
    if (!aligned_to(workspace, 256)) return DL_E_ALIGN;
    if (workspace_bytes < need) return DL_E_SHAPE;
    p.part = static_cast<float*>(workspace);
  }
  hipError_t e = launch(desc, p, true, stream);
  const int64_t parts = (int64_t(n) + p.per - 1) / p.per, d = desc->head_dim;
  if (e == hipSuccess && p.part)
    e = launch_column_sums({p.part, parts, 2 * d, {g->dwq, g->dwk, nullptr}, {d, d, 0}}, stream);
  return e == hipSuccess ? DL_OK : DL_E_HIP;
}

}  // extern "C"
