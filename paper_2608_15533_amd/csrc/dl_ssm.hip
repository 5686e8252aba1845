// Selective state space scan: entry points, forward pass, single tokens.
#include "dl_ssm.hpp"
#include "dl_ssm_bwd.hpp"

namespace dl {
namespace {

// Tokens whose steps lie in LDS at a time, and whose B (and C) a wave holds in 32 scalar registers: 64
// do not fit beside the pointers (8192 x 4096 outputs: 229 us instead of 199).  With 64 states a workgroup is 16 waves, and
// two of them on a compute unit need the registers of eight waves to a SIMD: at most four tokens then, half as many in
// bf16 and as many as ever in fp32.  With that limit and LDS twice (AHEAD below) 8192 x 1024, both passes, took 227 us
// instead of 265, fp32 279 instead of 364.  With 32 and 16 states the limit costs more than it gives (236 -> 239, 250 -> 283).
template <int S, bool OUT, typename T>
constexpr int tile_tokens = OUT && S > 32 ? 4 : (OUT ? 16 : 32) / int(sizeof(T));

// A workgroup: one stretch, 64 channels; wave w has states 4 w .. 4 w + 3.  OUT: outputs and final
// states; else E and the sum of d, of stretches that others follow.  AHEAD: LDS is there twice, and the next tile's
// steps are formed before the barrier that ends a tile: one barrier instead of two (with 32 states 250 us, not 237).
template <int S, bool OUT, typename T>
__global__ __launch_bounds__(S * 16, S > 32 ? 8 : 1) void ssm_kernel(SsmParams p) {
  constexpr int TILE = tile_tokens<S, OUT, T>, NW = S / 4, NT = 64 * NW;
  constexpr int EV = TILE * 64 >= NT ? TILE * 64 / NT : 1, CG = 64 / EV;
  constexpr bool AHEAD = OUT && S > 32;
  constexpr int NB = AHEAD ? 2 : 1;
  __shared__ __attribute__((aligned(16))) float step[NB][TILE][64], input[NB][TILE][64];
  __shared__ __attribute__((aligned(16))) float partial[NB][OUT ? NW : 1][OUT ? TILE : 1][64];
  const int f = blockIdx.x / p.blocks, c0 = int(blockIdx.x % p.blocks) * 64;
  const Stretch s = find_stretch(p.cu, p.seq_slot, p.n, p.N, p.B, p.len, f);
  if (s.idle || (!OUT && s.ends())) return;
  const int lane = threadIdx.x & 63, w = wave_index(), c = c0 + lane;
  const bool live = c < p.D;
  // This thread's part of a tile: a token, EV channels.
  const int te = threadIdx.x / CG, ce = (threadIdx.x % CG) * EV;
  const bool le = c0 + ce < p.D && te < TILE;        // D is a multiple of 8: all EV or none
  const int64_t at = int64_t(f) * p.D * S + (int64_t(w) * p.D + c) * 4;   // of E

  float a2[4], h[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    a2[i] = live ? p.A[int64_t(c) * S + 4 * w + i] * LOG2E : 0.0f;
    h[i] = 0.0f;
  }
  const int64_t state = (int64_t(s.slot) * p.D + c) * S + 4 * w;
  if (OUT && live && (p.E || p.h_in)) {
    const f32x4 v = *reinterpret_cast<const f32x4*>(p.E ? p.E + at : p.h_in + state);
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = v[i];
  }
  float bias[EV], skip[EV], total[EV];
#pragma unroll
  for (int e = 0; e < EV; ++e) {
    bias[e] = p.bias && le ? p.bias[c0 + ce + e] : 0.0f;
    skip[e] = OUT && p.skip && le ? p.skip[c0 + ce + e] : 0.0f;
    total[e] = 0.0f;
  }
  typedef Cursor<EV, T> At;
  At xs(p.x, p.x_stride, s.first, c0, te, ce, TILE), ds(p.dt, p.dt_stride, s.first, c0, te, ce, TILE);
  At zs(p.z, p.z_stride, s.first, c0, te, ce, TILE), ys(p.y, p.D, s.first, c0, te, ce, TILE);
  const T* bp = static_cast<const T*>(p.Bm) + int64_t(s.first) * p.b_stride + 4 * w;
  const T* cp = static_cast<const T*>(p.Cm) + int64_t(s.first) * p.c_stride + 4 * w;
  Raw<EV, T> rx{}, rd{}, rz{};
  auto fetch = [&](int j) {
    if (le && j * TILE + te < s.count) {
      rx = xs.load();
      rd = ds.load();
      if (OUT && p.z) rz = zs.load();
    }
    xs.move(1);
    ds.move(1);
    zs.move(1);
  };
  TileRows<TILE, OUT, T> rows;
  Raw<EV, T> kx{}, kz{};                   // this thread's rows of the tile before
  auto prepare = [&](int j, int buf) {
    const int count = min(TILE, s.count - j * TILE);
    const bool mine = le && te < count;
    if (count == TILE) rows.load(bp, p.b_stride, cp, p.c_stride);
    if (te < TILE) {
#pragma unroll
      for (int e = 0; e < EV; ++e) {
        const float d = mine ? softplus(rd.get(e) + bias[e]) : 0.0f;
        step[buf][te][ce + e] = d;
        input[buf][te][ce + e] = mine ? d * rx.get(e) : 0.0f;
        total[e] += d;
      }
    }
  };
  auto keep = [&](int j) {
    kx = rx;
    kz = rz;
    fetch(j + 1);
  };
  if (s.count > 0) fetch(0);
  if (AHEAD && s.count > 0) {
    prepare(0, 0);
    keep(0);
    if (s.count >= TILE) rows.settle();
    __syncthreads();
  }
  for (int j = 0, buf = 0; j * TILE < s.count; ++j) {
    const int count = min(TILE, s.count - j * TILE);
    const bool mine = le && te < count;
    if (!AHEAD) {
      prepare(j, 0);
      keep(j);
      if (count == TILE) rows.settle();
      __syncthreads();
    }
    auto token = [&](int t, const Four<T>& B, const Four<T>& C) {
      const float d = step[buf][t][lane], u = input[buf][t][lane];
      float y = 0.0f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        h[i] = fmaf(decay(d, a2[i]), h[i], u * B.at(i));
        if (OUT) y = i ? fmaf(C.at(i), h[i], y) : C.at(0) * h[0];
      }
      if (OUT) partial[buf][w][t][lane] = y;
    };
    if (count == TILE) {
#pragma unroll
      for (int t = 0; t < TILE; ++t) token(t, rows.B[t], rows.C[OUT ? t : 0]);
    } else {
      for (int t = 0; t < count; ++t) {
        Four<T> B, C;
        B.load(bp + t * p.b_stride);
        C.load(cp + t * p.c_stride);
        token(t, B, C);
      }
    }
    bp += TILE * p.b_stride;
    cp += TILE * p.c_stride;
    const bool more = (j + 1) * TILE < s.count;
    if (AHEAD && more) {
      prepare(j + 1, buf ^ 1);
      if (s.count - (j + 1) * TILE >= TILE) rows.settle();
    }
    __syncthreads();
    if (OUT && mine) {
      float y[EV];
#pragma unroll
      for (int e = 0; e < EV; ++e) {
        y[e] = 0.0f;
#pragma unroll
        for (int i = 0; i < NW; ++i) y[e] += partial[buf][i][te][ce + e];
        const float z = kz.get(e);
        y[e] = fmaf(skip[e], kx.get(e), y[e]);
        if (p.z) y[e] *= z * sigmoid<T>(z);
      }
      ys.store(y);
    }
    ys.move(1);
    if (AHEAD) {
      keep(j + 1);
      buf ^= 1;
    }
  }
  if (OUT) {
    if (s.ends() && live) *reinterpret_cast<f32x4*>(p.h_out + state) = f32x4{h[0], h[1], h[2], h[3]};
    return;
  }
  if (live) *reinterpret_cast<f32x4*>(p.E + at) = f32x4{h[0], h[1], h[2], h[3]};
  // The sum of d over the stretch: each thread's own tokens, then the tile's tokens in order.
  if (te < TILE) {
#pragma unroll
    for (int e = 0; e < EV; ++e) step[0][te][ce + e] = total[e];
  }
  __syncthreads();
  if (w == 0 && live) {
    float sum = 0.0f;
#pragma unroll
    for (int t = 0; t < TILE; ++t) sum += step[0][t][lane];
    p.sums[int64_t(f) * p.D + c] = sum;
  }
}

// States before every stretch, in place of what each leaves from zero; a thread for one state of one
// sequence.  BWD: likewise from the end, gradients behind every stretch.
template <bool BWD>
__global__ __launch_bounds__(256) void ssm_join_kernel(SsmParams p) {
  const int64_t per = int64_t(p.D) * p.S, groups = (per + 255) / 256;
  const int seq = int(blockIdx.x / groups);
  const int64_t i = int64_t(blockIdx.x % groups) * 256 + threadIdx.x;
  const int first = min(max(p.cu[seq], 0), p.N), end = min(max(p.cu[seq + 1], first), p.N);
  const int slot = p.seq_slot[seq], base = first / p.len + seq;
  const int parts = max(1, (end - first + p.len - 1) / p.len);
  if (i >= per || slot < 0 || slot >= p.B) return;
  const int c = int((i >> 2) % p.D), k = int(i / (4 * int64_t(p.D))) * 4 + int(i & 3);
  const float a2 = p.A[int64_t(c) * p.S + k] * LOG2E;
  const int64_t state = (int64_t(slot) * p.D + c) * p.S + k;
  float* E = p.E + i;
  float h = p.h_in ? p.h_in[state] : 0.0f;
  constexpr int U = 16;          // loads in flight: they do not wait for the states
  for (int j = 0; j < parts; j += U) {
    float e[U], d[U];
#pragma unroll
    for (int q = 0; q < U; ++q) {
      const int64_t r = base + min(j + q, parts - 1);
      const bool there = j + q + 1 < parts;          // the last stretch leaves nothing here
      e[q] = there ? E[r * per] : 0.0f;
      d[q] = there ? p.sums[r * p.D + c] : 0.0f;
    }
#pragma unroll
    for (int q = 0; q < U; ++q) {
      if (j + q >= parts) break;
      E[(base + j + q) * per] = h;
      h = fmaf(decay(d[q], a2), h, e[q]);
    }
  }
  if (!BWD) return;
  float* F = p.F + i;
  float g = p.dh_out ? p.dh_out[state] : 0.0f;
  for (int j = parts - 1; j >= 0; j -= U) {
    float e[U], d[U];
#pragma unroll
    for (int q = 0; q < U; ++q) {
      const int64_t r = base + max(j - q, 0);
      const bool there = j - q > 0;                  // nothing is asked of the first
      e[q] = there ? F[r * per] : 0.0f;
      d[q] = there ? p.sums[r * p.D + c] : 0.0f;
    }
#pragma unroll
    for (int q = 0; q < U; ++q) {
      if (j - q < 0) break;
      F[(base + j - q) * per] = g;
      g = fmaf(decay(d[q], a2), g, e[q]);
    }
  }
}

// One token a slot: four states a lane, S / 4 lanes a channel.
template <int S, typename T>
__global__ __launch_bounds__(256) void ssm_step_kernel(SsmParams p) {
  constexpr int L = S / 4, CH = 256 / L;
  const int i = blockIdx.x / p.blocks, c = int(blockIdx.x % p.blocks) * CH + int(threadIdx.x) / L;
  const int k = (threadIdx.x % L) * 4;
  const int slot = p.slots ? p.slots[i] : i;
  if (c >= p.D || slot < 0 || slot >= p.B) return;
  const int64_t state = (int64_t(slot) * p.D + c) * S + k;
  const f32x4 old = *reinterpret_cast<const f32x4*>(p.h_in + state);
  float B[4], C[4];
  load_row<4>(static_cast<const T*>(p.Bm) + i * p.b_stride + k, B);
  load_row<4>(static_cast<const T*>(p.Cm) + i * p.c_stride + k, C);
  const float x = widen(static_cast<const T*>(p.x)[i * p.x_stride + c]);
  const float raw = widen(static_cast<const T*>(p.dt)[i * p.dt_stride + c]) + (p.bias ? p.bias[c] : 0.0f);
  const float d = softplus(raw), u = d * x;
  f32x4 h;
  float y = 0.0f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    h[e] = fmaf(decay(d, p.A[int64_t(c) * S + k + e] * LOG2E), old[e], u * B[e]);
    y = fmaf(C[e], h[e], y);
  }
  *reinterpret_cast<f32x4*>(p.h_out + state) = h;
  y = lanes_sum<L>(y);
  if (k) return;
  if (p.skip) y = fmaf(p.skip[c], x, y);
  if (p.z) {
    const float z = widen(static_cast<const T*>(p.z)[i * p.z_stride + c]);
    y *= z * sigmoid<T>(z);
  }
  narrow(static_cast<T*>(p.y) + int64_t(i) * p.D + c, y);
}

template <int S, typename T>
hipError_t launch_prefill(const SsmParams& p, hipStream_t s) {
  const int64_t grid = stretches(p.n, p.N, p.len) * p.blocks;
  if (p.E) {
    hipError_t e = start_rows(&ssm_kernel<S, false, T>, grid, S * 16, p, s);
    const int64_t groups = (int64_t(p.D) * S + 255) / 256;
    if (e == hipSuccess) e = start_rows(&ssm_join_kernel<false>, groups * p.n, 256, p, s);
    if (e != hipSuccess) return e;
  }
  return start_rows(&ssm_kernel<S, true, T>, grid, S * 16, p, s);
}

template <int S, typename T>
hipError_t launch_backward(const SsmParams& p, hipStream_t s) {
  hipError_t e = launch_ssm_ends(S, sizeof(T) == 2, p, s);
  if (p.E) {
    const int64_t groups = (int64_t(p.D) * S + 255) / 256;
    if (e == hipSuccess) e = start_rows(&ssm_join_kernel<true>, groups * p.n, 256, p, s);
  }
  if (e == hipSuccess) e = launch_ssm_grad(S, sizeof(T) == 2, p, s);
  return e;
}

template <int S, typename T>
hipError_t launch_step(const SsmParams& q, hipStream_t s) {
  SsmParams p = q;
  p.blocks = (p.D + 1024 / S - 1) / (1024 / S);
  return start_rows(&ssm_step_kernel<S, T>, int64_t(p.n) * p.blocks, 256, p, s);
}

enum Pass { STEP, FORWARD, BACKWARD };
template <int S, typename T>
hipError_t launch_pass(Pass pass, const SsmParams& p, hipStream_t s) {
  return pass == STEP ? launch_step<S, T>(p, s) : pass == FORWARD ? launch_prefill<S, T>(p, s)
                                                                 : launch_backward<S, T>(p, s);
}
template <typename T>
hipError_t launch_states(Pass pass, const SsmParams& p, hipStream_t s) {
  switch (p.S) {
    case 16: return launch_pass<16, T>(pass, p, s);
    case 32: return launch_pass<32, T>(pass, p, s);
    default: return launch_pass<64, T>(pass, p, s);
  }
}
hipError_t launch(Pass pass, const dl_ssm_desc* d, const SsmParams& p, hipStream_t s) {
  return d->in_dtype == DL_BF16 ? launch_states<uint16_t>(pass, p, s) : launch_states<float>(pass, p, s);
}

int blocks_of(const dl_ssm_desc* d) { return (d->channels + 63) / 64; }

// Tokens of a stretch: as long as the call's tokens leave enough waves to fill the chip and to even out ragged ends,
// however many sequences they are.  Forward with 2048, 4096, 8192, 16384 and 32768 waves: 8192 tokens of one sequence, 4096
// channels x 16 states, 394, 283, 254, 247, 254 us; 1024 x 64 588, 260, 224, 227, 250; 12 ragged ones, 6000 tokens of 2048 x 32,
// 298, 209, 193, 193, 214; 8 of 1024 tokens, 4096 x 16, 337, 250, 240, 229, 240.  Not so where the sequences are waves
// enough by themselves and a longer stretch leaves nothing to walk twice: 32 of 512 tokens 316, 317, 329, 393, 422; the
// rule does not look at them.  Backward longer ones leave fewer states to join and rows of partial sums: 4096 tokens
// in two sequences, 4096 x 16, 2048 x 32 and 1024 x 64, whole step, with 32, 64, 128 and 256 tokens 513, 483, 479, 513;
// 526, 490, 478, 492; 558, 511, 484, 539 us.  16 where 32 tokens leave fewer than 2048 waves: 777 tokens of 200 channels
// 47 us, 58 with 32, 64 of 4096 channels forward 14 us instead of 18; where 32 leave 4000, 500 tokens of 1024 x 64 would
// take 35 instead of 29.  Up to 32 tokens stay whole, forward in one kernel: 9 us, 14 in two parts.
int stretch_len(const dl_ssm_desc* d, int32_t tokens, bool backward) {
  const int64_t waves = int64_t(blocks_of(d)) * (d->states / 4), least = backward ? 8192 : 16384;
  int64_t len = tokens > 32 ? 16 : 32;
  while (len < (backward ? 256 : tokens) && tokens / (2 * len) * waves >= (len < 32 ? 2048 : least)) len *= 2;
  return int(backward ? len : std::min<int64_t>(len, std::max(tokens, 1)));
}
// One stretch a sequence: nothing to join.
bool whole(int32_t tokens, int len) { return tokens <= len; }

int check_desc(const dl_ssm_desc* d) {
  if (!d) return DL_E_NULL;
  if (d->abi_version != DL_ABI_VERSION) return DL_E_VERSION;
  if (d->states != 16 && d->states != 32 && d->states != 64) return DL_E_UNSUPPORTED;
  if (d->channels < 8 || d->channels % 8 != 0 || d->channels > (1 << 20)) return DL_E_SHAPE;
  if (d->num_slots < 1) return DL_E_SHAPE;
  if (d->in_dtype != DL_F32 && d->in_dtype != DL_BF16) return DL_E_DTYPE;
  return DL_OK;
}

int check_counts(const dl_ssm_desc* d, int32_t n, int32_t tokens, bool backward) {
  if (n < 0 || tokens < 0 || n > d->num_slots) return DL_E_SHAPE;
  const int64_t rows = stretches(n, tokens, stretch_len(d, tokens, backward));
  if (!grid_fits(rows * blocks_of(d), d->states * 16)) return DL_E_SHAPE;
  const int64_t groups = (int64_t(d->channels) * d->states + 255) / 256;
  if (!grid_fits(groups * n, 256)) return DL_E_SHAPE;
  const int64_t pieces = int64_t(stretch_len(d, tokens, true)) * 2 * d->states / 256;   // of dB's and dC's sums
  return !backward || grid_fits(rows * pieces, 256) ? DL_OK : DL_E_SHAPE;
}

int check_rows(const dl_ssm_desc* d, const dl_ssm_rows* r, bool any) {
  if (!r || !r->A || (any && (!r->x || !r->dt || !r->B || !r->C))) return DL_E_NULL;
  for (const void* v : {r->x, r->dt, r->z, r->B, r->C})
    if (!aligned_to(v, 16)) return DL_E_ALIGN;
  if (!aligned_to(r->A, 4) || !aligned_to(r->skip, 4) || !aligned_to(r->dt_bias, 4)) return DL_E_ALIGN;
  if (!any) return DL_OK;
  if (!good_stride(r->x_stride, d->channels) || !good_stride(r->dt_stride, d->channels) ||
      (r->z && !good_stride(r->z_stride, d->channels)) || !good_stride(r->b_stride, d->states) ||
      !good_stride(r->c_stride, d->states))
    return DL_E_SHAPE;
  return DL_OK;
}

SsmParams params(const dl_ssm_desc* d, const float* h_in, float* h_out, const dl_ssm_rows* r, int32_t n,
                 int32_t tokens) {
  SsmParams p{};
  p.x = r->x;
  p.dt = r->dt;
  p.z = r->z;
  p.Bm = r->B;
  p.Cm = r->C;
  p.x_stride = r->x_stride;
  p.dt_stride = r->dt_stride;
  p.z_stride = r->z_stride;
  p.b_stride = r->b_stride;
  p.c_stride = r->c_stride;
  p.A = r->A;
  p.skip = r->skip;
  p.bias = r->dt_bias;
  p.h_in = h_in;
  p.h_out = h_out;
  p.n = n;
  p.N = tokens;
  p.B = d->num_slots;
  p.D = d->channels;
  p.S = d->states;
  p.blocks = blocks_of(d);
  return p;
}

// Workspace, 256-byte aligned parts: E, sums (sequences in several stretches); backward F, then the
// tiles' starts and the partial sums.
struct Layout {
  size_t E = 0, F = 0, sums = 0, tiles = 0, tile_sums = 0, part = 0, rows = 0, all = 0;
};
Layout layout(const dl_ssm_desc* d, int32_t n, int32_t tokens, bool backward) {
  const int len = stretch_len(d, tokens, backward);
  const size_t parts = size_t(stretches(n, tokens, len)), D = size_t(d->channels), S = size_t(d->states);
  Layout l;
  auto take = [&](size_t floats) {
    const size_t at = l.all;
    l.all += round256(floats * sizeof(float));
    return at;
  };
  if (!whole(tokens, len)) {
    l.E = take(parts * D * S);
    l.sums = take(parts * D);
    if (backward) l.F = take(parts * D * S);
  }
  if (backward) {
    const size_t inner = parts * size_t(len / ssm_grad_tile(d->states) - 1);
    l.tiles = take(inner * D * S);
    l.tile_sums = take(inner * D);
    l.part = take(parts * D * (S + 2));
    l.rows = take(size_t(blocks_of(d)) * size_t(tokens) * 2 * S);
  }
  return l;
}

void set_workspace(SsmParams& p, const dl_ssm_desc* d, const Layout& l, void* ws, bool backward) {
  char* at = static_cast<char*>(ws);
  p.len = stretch_len(d, p.N, backward);
  p.inner = p.len / ssm_grad_tile(d->states) - 1;
  if (!whole(p.N, p.len)) {
    p.E = reinterpret_cast<float*>(at + l.E);
    p.sums = reinterpret_cast<float*>(at + l.sums);
    p.F = reinterpret_cast<float*>(at + l.F);
  }
  p.tiles = reinterpret_cast<float*>(at + l.tiles);
  p.tile_sums = reinterpret_cast<float*>(at + l.tile_sums);
  p.part = reinterpret_cast<float*>(at + l.part);
  p.rows = reinterpret_cast<float*>(at + l.rows);
}

int check_workspace(const Layout& l, const void* ws, size_t bytes) {
  if (l.all == 0) return DL_OK;
  if (!ws) return DL_E_NULL;
  if (!aligned_to(ws, 256)) return DL_E_ALIGN;
  return bytes < l.all ? DL_E_SHAPE : DL_OK;
}

}  // namespace
}  // namespace dl

using namespace dl;

extern "C" {

int dl_ssm_step(const dl_ssm_desc* desc, const float* h_in, float* h_out, const dl_ssm_rows* rows, void* y,
                const int32_t* slots, int32_t n, hipStream_t stream) {
  DL_TRY(check_desc(desc));
  if (n < 0 || n > desc->num_slots) return DL_E_SHAPE;
  if (!grid_fits(int64_t(n) * ((int64_t(desc->channels) * desc->states + 1023) / 1024), 256)) return DL_E_SHAPE;
  if (n == 0) return DL_OK;               // nothing to do, whatever the pointers are
  if (!slots && n != desc->num_slots) return DL_E_SHAPE;
  DL_TRY(check_rows(desc, rows, true));
  if (!h_in || !h_out || !y) return DL_E_NULL;
  if (!aligned_to(h_in, 16) || !aligned_to(h_out, 16) || !aligned_to(y, 16) || !aligned_to(slots, 4))
    return DL_E_ALIGN;
  SsmParams p = params(desc, h_in, h_out, rows, n, n);
  p.y = y;
  p.slots = slots;
  return launch(STEP, desc, p, stream) == hipSuccess ? DL_OK : DL_E_HIP;
}

int dl_ssm_workspace_bytes(const dl_ssm_desc* desc, int32_t n, int32_t tokens, int32_t backward,
                           size_t* bytes) {
  DL_TRY(check_desc(desc));
  DL_TRY(check_counts(desc, n, tokens, backward != 0));
  DL_TRY(check_counts(desc, n, tokens, false));
  if (!bytes) return DL_E_NULL;
  *bytes = 0;
  if (n == 0) return DL_OK;
  *bytes = layout(desc, n, tokens, false).all;
  if (backward) *bytes = std::max(*bytes, layout(desc, n, tokens, true).all);
  return DL_OK;
}

int dl_ssm_prefill(const dl_ssm_desc* desc, const float* h_in, float* h_out, const dl_ssm_rows* rows, void* y,
                   const dl_tables* tables, int32_t n, int32_t tokens, void* workspace,
                   size_t workspace_bytes, hipStream_t stream) {
  DL_TRY(check_desc(desc));
  DL_TRY(check_counts(desc, n, tokens, false));
  if (n == 0) return DL_OK;               // nothing to do, whatever the pointers are
  DL_TRY(check_rows(desc, rows, tokens > 0));
  DL_TRY(check_row_tables(tables));
  const Layout l = layout(desc, n, tokens, false);
  DL_TRY(check_workspace(l, workspace, workspace_bytes));
  if (!h_out || (tokens > 0 && !y)) return DL_E_NULL;
  if (!aligned_to(h_in, 16) || !aligned_to(h_out, 16) || !aligned_to(y, 16)) return DL_E_ALIGN;
  SsmParams p = params(desc, h_in, h_out, rows, n, tokens);
  p.y = y;
  p.cu = tables->cu_tokens;
  p.seq_slot = tables->seq_slot;
  set_workspace(p, desc, l, workspace, false);
  return launch(FORWARD, desc, p, stream) == hipSuccess ? DL_OK : DL_E_HIP;
}

int dl_ssm_backward(const dl_ssm_desc* desc, const float* h_in, const dl_ssm_rows* rows, const void* dy,
                    const float* dh_out, const dl_ssm_grads* g, const dl_tables* tables, int32_t n,
                    int32_t tokens, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  DL_TRY(check_desc(desc));
  DL_TRY(check_counts(desc, n, tokens, true));
  if (n == 0) return DL_OK;               // nothing to do, whatever the pointers are
  DL_TRY(check_rows(desc, rows, tokens > 0));
  DL_TRY(check_row_tables(tables));
  if (!g || !g->dA || (rows->skip && !g->dskip) || (rows->dt_bias && !g->dbias)) return DL_E_NULL;
  if (tokens > 0 && (!dy || !g->dx || !g->ddt || !g->dB || !g->dC || (rows->z && !g->dz))) return DL_E_NULL;
  for (const void* v : {static_cast<const void*>(h_in), dy, static_cast<const void*>(dh_out),
                        static_cast<const void*>(g->dx), static_cast<const void*>(g->ddt),
                        static_cast<const void*>(g->dz), static_cast<const void*>(g->dB),
                        static_cast<const void*>(g->dC), static_cast<const void*>(g->ds)})
    if (!aligned_to(v, 16)) return DL_E_ALIGN;
  if (!aligned_to(g->dA, 4) || !aligned_to(g->dskip, 4) || !aligned_to(g->dbias, 4)) return DL_E_ALIGN;
  const Layout l = layout(desc, n, tokens, true);
  DL_TRY(check_workspace(l, workspace, workspace_bytes));
  SsmParams p = params(desc, h_in, g->ds, rows, n, tokens);
  p.cu = tables->cu_tokens;
  p.seq_slot = tables->seq_slot;
  p.dy = dy;
  p.dh_out = dh_out;
  p.dx = g->dx;
  p.ddt = g->ddt;
  p.dz = g->dz;
  p.dB = g->dB;
  p.dC = g->dC;
  set_workspace(p, desc, l, workspace, true);
  hipError_t e = launch(BACKWARD, desc, p, stream);
  const int64_t parts = stretches(n, tokens, p.len), D = p.D, S = p.S, row = D * (S + 2);
  if (e == hipSuccess)
    e = launch_column_sums({p.part, parts, row, {g->dA, p.skip ? g->dskip : nullptr, p.bias ? g->dbias : nullptr},
                            {D * S, D, D}}, stream);
  return e == hipSuccess ? DL_OK : DL_E_HIP;
}

}  // extern "C"
