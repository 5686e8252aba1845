// Selective state space scan: the backward pass's kernels.
#include "dl_ssm_bwd.hpp"

namespace dl {
namespace {

// A thread's part of a tile: one token, EV channels.
template <int S, typename T>
struct Part {
  static constexpr int TB = ssm_grad_tile(S), NT = S * 16, EV = TB * 64 >= NT ? TB * 64 / NT : 1, CG = 64 / EV;
  int te, ce, c;
  bool live;                     // D is a multiple of 8: all EV channels or none
  float bias[EV];
  __device__ __forceinline__ Part(const SsmParams& p, int c0) {
    te = threadIdx.x / CG;
    ce = (threadIdx.x % CG) * EV;
    c = c0 + ce;
    live = c < p.D && te < TB;
#pragma unroll
    for (int e = 0; e < EV; ++e) bias[e] = p.bias && live ? p.bias[c + e] : 0.0f;
  }
  __device__ __forceinline__ Cursor<EV, T> rows(const void* base, int64_t stride, int first) const {
    return Cursor<EV, T>(base, stride, first, c - ce, te, ce, TB);
  }
};

// E, F and the sum of d of a stretch, 64 channels; wave w has states 4 w .. 4 w + 3.  On the way, before
// every tile but the first, what the stretch has left so far and the sum of d: the gradients start there.  Registers
// for eight waves to a SIMD let two workgroups of 16 waves share a compute unit (a step of 1024 x 64 channels x
// states 502 -> 483 us).
template <int S, typename T>
__global__ __launch_bounds__(S * 16, S > 16 ? 8 : 1) void ssm_ends_kernel(SsmParams p) {
  typedef Part<S, T> P;
  constexpr int TB = P::TB, EV = P::EV;
  constexpr bool AHEAD = S > 16;
  constexpr int NB = AHEAD ? 2 : 1;
  __shared__ __attribute__((aligned(16))) float step[NB][TB][64], input[NB][TB][64], grad[NB][TB][64];
  const int f = blockIdx.x / p.blocks, c0 = int(blockIdx.x % p.blocks) * 64;
  const Stretch s = find_stretch(p.cu, p.seq_slot, p.n, p.N, p.B, p.len, f);
  if (s.idle) return;
  const int lane = threadIdx.x & 63, w = wave_index(), c = c0 + lane;
  const P part(p, c0);
  float a2[4], h[4] = {}, g[4] = {}, decays[4], sum = 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    a2[i] = c < p.D ? p.A[int64_t(c) * S + 4 * w + i] * LOG2E : 0.0f;
    decays[i] = 1.0f;
  }
  const T* bp = static_cast<const T*>(p.Bm) + int64_t(s.first) * p.b_stride + 4 * w;
  const T* cp = static_cast<const T*>(p.Cm) + int64_t(s.first) * p.c_stride + 4 * w;
  Cursor<EV, T> xs = part.rows(p.x, p.x_stride, s.first), ds = part.rows(p.dt, p.dt_stride, s.first);
  Cursor<EV, T> os = part.rows(p.dy, p.D, s.first), zs = part.rows(p.z, p.z_stride, s.first);
  Raw<EV, T> rx{}, rd{}, ro{}, rz{};
  auto fetch = [&](int j) {
    if (part.live && j * TB + part.te < s.count) {
      rx = xs.load();
      rd = ds.load();
      ro = os.load();
      if (p.z) rz = zs.load();
    }
    xs.move(1);
    ds.move(1);
    os.move(1);
    zs.move(1);
  };
  TileRows<TB, true, T> rows;
  auto prepare = [&](int j, int buf) {
    const int count = min(TB, s.count - j * TB);
    const bool mine = part.live && part.te < count;
    if (count == TB) rows.load(bp, p.b_stride, cp, p.c_stride);
    if (part.te < TB) {
#pragma unroll
      for (int e = 0; e < EV; ++e) {
        const float d = mine ? softplus(rd.get(e) + part.bias[e]) : 0.0f, z = rz.get(e);
        step[buf][part.te][part.ce + e] = d;
        input[buf][part.te][part.ce + e] = mine ? d * rx.get(e) : 0.0f;
        grad[buf][part.te][part.ce + e] = mine ? ro.get(e) * (p.z ? z * sigmoid<T>(z) : 1.0f) : 0.0f;
      }
    }
    fetch(j + 1);
    if (count == TB) rows.settle();
  };
  if (s.count > 0) fetch(0);
  if (AHEAD && s.count > 0) {
    prepare(0, 0);
    __syncthreads();
  }
  for (int j = 0, buf = 0; j * TB < s.count; ++j) {
    const int count = min(TB, s.count - j * TB);
    if (!AHEAD) {
      prepare(j, 0);
      __syncthreads();
    }
    if (j > 0 && c < p.D) {
      const int64_t tile = int64_t(f) * p.inner + j - 1;
      *reinterpret_cast<f32x4*>(p.tiles + tile * p.D * S + (int64_t(w) * p.D + c) * 4) = f32x4{h[0], h[1], h[2], h[3]};
      if (w == 0) p.tile_sums[tile * p.D + c] = sum;
    }
    auto token = [&](int t, const Four<T>& B, const Four<T>& C) {
      const float d = step[buf][t][lane], u = input[buf][t][lane], up = grad[buf][t][lane];
      sum += d;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float a = decay(d, a2[i]);
        h[i] = fmaf(a, h[i], u * B.at(i));
        decays[i] *= a;
        g[i] = fmaf(decays[i], up * C.at(i), g[i]);
      }
    };
    if (count == TB) {
#pragma unroll
      for (int t = 0; t < TB; ++t) token(t, rows.B[t], rows.C[t]);
    } else {
      for (int t = 0; t < count; ++t) {
        Four<T> B, C;
        B.load(bp + t * p.b_stride);
        C.load(cp + t * p.c_stride);
        token(t, B, C);
      }
    }
    bp += TB * p.b_stride;
    cp += TB * p.c_stride;
    if (AHEAD) {
      if ((j + 1) * TB < s.count) prepare(j + 1, buf ^ 1);
      buf ^= 1;
    }
    __syncthreads();
  }
  if (p.E && c < p.D) {
    const int64_t at = int64_t(f) * p.D * S + (int64_t(w) * p.D + c) * 4;
    *reinterpret_cast<f32x4*>(p.E + at) = f32x4{h[0], h[1], h[2], h[3]};
    *reinterpret_cast<f32x4*>(p.F + at) = f32x4{g[0], g[1], g[2], g[3]};
    if (w == 0) p.sums[int64_t(f) * p.D + c] = sum;
  }
}

// Sums over the 64 lanes of eight values; lane l is left with number sum_number(l).
__device__ __forceinline__ float eight_sums(const float (&v)[8]) {
  float s[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) s[i] = halves_sum32(v[i], v[i + 4]);
  return lanes_sum<8>(halves_sum8(halves_sum16(s[0], s[1]), halves_sum16(s[2], s[3])));
}
__device__ __forceinline__ int sum_number(int l) {
  return 4 * (l >> 5) + 2 * ((l >> 3) & 1) + ((l >> 4) & 1);
}

// Every gradient of a stretch's tokens, 64 channels; wave w has states 4 w .. 4 w + 3.  Tiles from the last
// to the first: a tile starts from what the stretch had left there and its decayed first state; its decays a_t
// and m_t = a_t . h_{t-1} are held in registers, then come its tokens backwards.
// With 32 or 64 states LDS is there twice, and the next tile's steps are formed before the barrier that ends a tile's
// walk: one barrier a tile, and its last part runs beside other waves' next walk (4096 tokens of 2048 x 32 and 1024
// x 64 channels x states, whole step: 511 -> 493 and 576 -> 540 us; ssm_ends_kernel likewise, 485 and 530).  With 16 a
// compute unit has three workgroups for that, and it would cost one of them.
template <int S, typename T>
__global__ __launch_bounds__(S * 16, S == 16 ? 3 : 4) void ssm_grad_kernel(SsmParams p) {
  typedef Part<S, T> P;
  constexpr int TB = P::TB, EV = P::EV, NW = S / 4;
  constexpr bool AHEAD = S > 16;
  constexpr int NB = AHEAD ? 2 : 1;
  __shared__ __attribute__((aligned(16))) float step[NB][TB][64], input[NB][TB][64], grad[NB][TB][64];
  __shared__ __attribute__((aligned(16))) float sum_gb[NB][NW][TB][64], sum_gm[NB][NW][TB][64], sum_ch[NB][NW][TB][64];
  const int f = blockIdx.x / p.blocks, block = int(blockIdx.x % p.blocks), c0 = block * 64;
  const Stretch s = find_stretch(p.cu, p.seq_slot, p.n, p.N, p.B, p.len, f);
  const int lane = threadIdx.x & 63, w = wave_index(), c = c0 + lane;
  const bool live = c < p.D;
  const P part(p, c0);
  float dA[4] = {}, dskip[EV] = {}, dbias[EV] = {};
  if (!s.idle) {
    float a2[4], g[4] = {}, skip[EV];
#pragma unroll
    for (int i = 0; i < 4; ++i) a2[i] = live ? p.A[int64_t(c) * S + 4 * w + i] * LOG2E : 0.0f;
#pragma unroll
    for (int e = 0; e < EV; ++e) skip[e] = p.skip && part.live ? p.skip[part.c + e] : 0.0f;
    const int64_t state = (int64_t(s.slot) * p.D + c) * S + 4 * w;
    const int64_t quad = (int64_t(w) * p.D + c) * 4, at = int64_t(f) * p.D * S + quad;
    const float* hp = p.E ? p.E + at : p.h_in ? p.h_in + state : nullptr;
    const float* gp = p.E ? p.F + at : p.dh_out ? p.dh_out + state : nullptr;
    f32x4 first{};
    if (live && hp) first = *reinterpret_cast<const f32x4*>(hp);
    if (live && gp) {
      const f32x4 v = *reinterpret_cast<const f32x4*>(gp);
#pragma unroll
      for (int i = 0; i < 4; ++i) g[i] = v[i];
    }
    const T* bp = static_cast<const T*>(p.Bm) + int64_t(s.first) * p.b_stride + 4 * w;
    const T* cp = static_cast<const T*>(p.Cm) + int64_t(s.first) * p.c_stride + 4 * w;
    const int tiles = (s.count + TB - 1) / TB, last = s.first + max(tiles - 1, 0) * TB;
    Cursor<EV, T> xs = part.rows(p.x, p.x_stride, last), ds = part.rows(p.dt, p.dt_stride, last);
    Cursor<EV, T> os = part.rows(p.dy, p.D, last), zs = part.rows(p.z, p.z_stride, last);
    Cursor<EV, T> dxs = part.rows(p.dx, p.D, last), dds = part.rows(p.ddt, p.D, last);
    Cursor<EV, T> dzs = part.rows(p.dz, p.D, last);
    // Rows as they are stored and the tile's start, a tile ahead.
    Raw<EV, T> rx{}, rd{}, ro{}, rz{};
    f32x4 left{};
    float since = 0.0f;
    auto fetch = [&](int j) {
      if (part.live && j * TB + part.te < s.count) {
        rx = xs.load();
        rd = ds.load();
        ro = os.load();
        if (p.z) rz = zs.load();
      }
      xs.move(-1);
      ds.move(-1);
      os.move(-1);
      zs.move(-1);
      if (j > 0 && live) {
        const int64_t tile = int64_t(f) * p.inner + j - 1;
        left = *reinterpret_cast<const f32x4*>(p.tiles + tile * p.D * S + quad);
        since = p.tile_sums[tile * p.D + c];
      }
    };
    // A tile's steps, rows and start; its raw rows are kept for its own gradients.
    TileRows<TB, true, T> rows;
    float h[4];
    auto prepare = [&](int j, int buf) {
      const int t0 = j * TB, count = min(TB, s.count - t0);
      const bool mine = part.live && part.te < count;
      rows.load(bp + int64_t(t0) * p.b_stride, p.b_stride, cp + int64_t(t0) * p.c_stride, p.c_stride, count);
#pragma unroll
      for (int i = 0; i < 4; ++i) h[i] = j > 0 ? fmaf(decay(since, a2[i]), first[i], left[i]) : first[i];
      if (part.te < TB) {
#pragma unroll
        for (int e = 0; e < EV; ++e) {
          const float d = mine ? softplus(rd.get(e) + part.bias[e]) : 0.0f, z = rz.get(e);
          step[buf][part.te][part.ce + e] = d;
          input[buf][part.te][part.ce + e] = mine ? d * rx.get(e) : 0.0f;
          grad[buf][part.te][part.ce + e] = mine ? ro.get(e) * (p.z ? z * sigmoid<T>(z) : 1.0f) : 0.0f;
        }
      }
    };
    Raw<EV, T> kx{}, kd{}, ko{}, kz{};
    auto keep = [&] {
      kx = rx;
      kd = rd;
      ko = ro;
      kz = rz;
    };
    if (tiles > 0) fetch(tiles - 1);
    if (AHEAD && tiles > 0) {
      prepare(tiles - 1, 0);
      keep();
      if (tiles > 1) fetch(tiles - 2);
      rows.settle();
      __syncthreads();
    }
    for (int j = tiles - 1, buf = 0; j >= 0; --j) {
      const int t0 = j * TB, count = min(TB, s.count - t0);
      const bool mine = part.live && part.te < count;
      if (!AHEAD) {
        prepare(j, 0);
        keep();
        if (j > 0) fetch(j - 1);
        rows.settle();
        __syncthreads();
      }
      auto walk = [&](auto whole) {
        constexpr bool ALL = decltype(whole)::value;
        float a[TB][4], m[TB][4];
#pragma unroll
        for (int t = 0; t < TB; ++t) {
          if (!ALL && t >= count) break;
          const float dd = step[buf][t][lane], u = input[buf][t][lane];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            a[t][i] = decay(dd, a2[i]);
            m[t][i] = a[t][i] * h[i];
            h[i] = fmaf(u, rows.B[t].at(i), m[t][i]);
          }
        }
        float kept = 0.0f;
        int place = lane & 7;
        asm volatile("" : "+v"(place));          // compared where it is used: eight masks kept spill registers
#pragma unroll
        for (int t = TB - 1; t >= 0; --t) {
          if (ALL || t < count) {
            const float dd = step[buf][t][lane], u = input[buf][t][lane], v = grad[buf][t][lane];
            float gb = 0.0f, gm = 0.0f, ch = 0.0f, over[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float b = rows.B[t].at(i), cc = rows.C[t].at(i);
              g[i] = fmaf(v, cc, g[i]);
              const float ht = fmaf(u, b, m[t][i]), x0 = g[i] * m[t][i];
              gb = fmaf(g[i], b, gb);
              gm = fmaf(x0, a2[i], gm);
              ch = fmaf(cc, ht, ch);
              dA[i] = fmaf(x0, dd, dA[i]);
              over[i] = g[i] * u;
              over[4 + i] = ht * v;
              g[i] *= a[t][i];
            }
            sum_gb[buf][w][t][lane] = gb;
            sum_gm[buf][w][t][lane] = gm;
            if (p.z) sum_ch[buf][w][t][lane] = ch;
            const float one = eight_sums(over);
            if (place == (t & 7)) kept = one;
          }
          if ((t & 7) == 0) {
            const int tt = t + place, k = sum_number(lane);   // numbers 0-3: B's states, 4-7: C's
            if (tt < count)
              p.rows[(int64_t(block) * p.N + s.first + t0 + tt) * (2 * S) + (k >> 2) * S + 4 * w + (k & 3)] = kept;
          }
        }
      };
      if (count == TB) walk(std::true_type{});
      else walk(std::false_type{});
      if (AHEAD && j > 0) {
        prepare(j - 1, buf ^ 1);
        rows.settle();
      }
      __syncthreads();
      if (mine) {
        float dx[EV], ddt[EV], dz[EV];
#pragma unroll
        for (int e = 0; e < EV; ++e) {
          float gb = 0.0f, gm = 0.0f, ch = 0.0f;
          __builtin_amdgcn_sched_barrier(0);     // not all partial sums at once: registers
#pragma unroll 4
          for (int i = 0; i < NW; ++i) {
            gb += sum_gb[buf][i][part.te][part.ce + e];
            gm += sum_gm[buf][i][part.te][part.ce + e];
            if (p.z) ch += sum_ch[buf][i][part.te][part.ce + e];
          }
          const float x = kx.get(e), z = kz.get(e), sz = sigmoid<T>(z);
          const float up = grad[buf][part.te][part.ce + e];
          dx[e] = fmaf(step[buf][part.te][part.ce + e], gb, skip[e] * up);
          ddt[e] = sigmoid<T>(kd.get(e) + part.bias[e]) * fmaf(x, gb, gm * 0.69314718f);   // A = a2 / log2 e
          dskip[e] = fmaf(up, x, dskip[e]);
          dbias[e] += ddt[e];
          dz[e] = ko.get(e) * fmaf(skip[e], x, ch) * sz * (1.0f + z * (1.0f - sz));
        }
        dxs.store(dx);
        dds.store(ddt);
        if (p.z) dzs.store(dz);
      }
      dxs.move(-1);
      dds.move(-1);
      dzs.move(-1);
      // What a thread reads of step and grad here, it alone writes in a later tile.
      if (AHEAD) {
        keep();
        if (j > 1) fetch(j - 2);
        buf ^= 1;
      }
    }
    if (s.begins() && p.h_out && live)
      *reinterpret_cast<f32x4*>(p.h_out + state) = f32x4{g[0], g[1], g[2], g[3]};
  }
  // Partial sums over the stretch; an idle one adds zeros.
  float* sums = p.part + int64_t(f) * p.D * (S + 2);
  if (live) {
#pragma unroll
    for (int i = 0; i < 4; ++i) sums[int64_t(c) * S + 4 * w + i] = dA[i];
  }
  __syncthreads();
  if (part.te < TB) {
#pragma unroll
    for (int e = 0; e < EV; ++e) {
      step[0][part.te][part.ce + e] = dskip[e];
      input[0][part.te][part.ce + e] = dbias[e];
    }
  }
  __syncthreads();
  if (w == 0 && live) {
    float a = 0.0f, b = 0.0f;
#pragma unroll
    for (int t = 0; t < TB; ++t) {
      a += step[0][t][lane];
      b += input[0][t][lane];
    }
    sums[int64_t(p.D) * S + c] = a;
    sums[int64_t(p.D) * (S + 1) + c] = b;
  }
}

// dB and dC: the sums over blocks of channels, in their order, eight loads at a time.  A workgroup for 256
// of a stretch's sums.
template <int S, typename T>
__global__ __launch_bounds__(256) void ssm_rows_kernel(SsmParams p) {
  constexpr int U = 8;
  const int pieces = p.len * 2 * S / 256;
  const Stretch s = find_stretch(p.cu, p.seq_slot, p.n, p.N, p.B, p.len, blockIdx.x / pieces);
  const int i = int(blockIdx.x % pieces) * 256 + int(threadIdx.x);
  if (s.idle || i >= s.count * 2 * S) return;
  const int64_t row = int64_t(s.first) + i / (2 * S), apart = int64_t(p.N) * (2 * S);
  const int k = i % (2 * S);
  const float* at = p.rows + row * (2 * S) + k;
  float sum = 0.0f;
  for (int b = 0; b < p.blocks; b += U) {
    float v[U];
#pragma unroll
    for (int j = 0; j < U; ++j) v[j] = b + j < p.blocks ? at[(b + j) * apart] : 0.0f;
#pragma unroll
    for (int j = 0; j < U; ++j) sum += v[j];
  }
  narrow(static_cast<T*>(k < S ? p.dB : p.dC) + row * S + k % S, sum);
}

template <int S, typename T>
hipError_t launch_grad(const SsmParams& p, hipStream_t s) {
  const int64_t parts = stretches(p.n, p.N, p.len);
  hipError_t e = start_rows(&ssm_grad_kernel<S, T>, parts * p.blocks, S * 16, p, s);
  if (e == hipSuccess)
    e = start_rows(&ssm_rows_kernel<S, T>, parts * (p.len * 2 * S / 256), 256, p, s);
  return e;
}
template <int S, typename T>
hipError_t launch_ends(const SsmParams& p, hipStream_t s) {
  return start_rows(&ssm_ends_kernel<S, T>, stretches(p.n, p.N, p.len) * p.blocks, S * 16, p, s);
}

}  // namespace

hipError_t launch_ssm_ends(int states, bool bf16, const SsmParams& p, hipStream_t s) {
  switch (states) {
    case 16: return bf16 ? launch_ends<16, uint16_t>(p, s) : launch_ends<16, float>(p, s);
    case 32: return bf16 ? launch_ends<32, uint16_t>(p, s) : launch_ends<32, float>(p, s);
    default: return bf16 ? launch_ends<64, uint16_t>(p, s) : launch_ends<64, float>(p, s);
  }
}
hipError_t launch_ssm_grad(int states, bool bf16, const SsmParams& p, hipStream_t s) {
  switch (states) {
    case 16: return bf16 ? launch_grad<16, uint16_t>(p, s) : launch_grad<16, float>(p, s);
    case 32: return bf16 ? launch_grad<32, uint16_t>(p, s) : launch_grad<32, float>(p, s);
    default: return bf16 ? launch_grad<64, uint16_t>(p, s) : launch_grad<64, float>(p, s);
  }
}

}  // namespace dl
