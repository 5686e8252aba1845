// Chunk tables and slot maps of a ragged batch, from request lengths in device memory.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "deltalog.h"
#include "dl_internal.h"

namespace dl {
namespace {

struct TableParams {
  const int32_t* lens;
  const int32_t* slots;   // or null: sequence i has slot i
  dl_tables t;
  int32_t* err;           // or null
  int32_t n, tokens, num_slots, max_chunks;
};

constexpr int SCAN_NT = 1024;
constexpr int ORDERED = 1024;    // sequences that are put in order
constexpr int FEW = 4096;        // sequences that one launch handles

// More than FEW sequences: running token and chunk counts, one workgroup.  A length below 0 counts as 0, and a
// sequence that would run past the token rows ends with them.
__global__ __launch_bounds__(SCAN_NT) void table_scan_kernel(TableParams p) {
  __shared__ int64_t part_t[SCAN_NT / 64];
  __shared__ int part_c[SCAN_NT / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int64_t base_t = 0;
  int base_c = 0, bad = 0;
  for (int i0 = 0; i0 < p.n; i0 += SCAN_NT) {
    const int i = i0 + tid;
    int32_t len = i < p.n ? p.lens[i] : 0;
    if (len < 0) { len = 0; bad |= 4; }
    int64_t x = len;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int64_t y = __shfl_up(x, d);
      if (lane >= d) x += y;
    }
    if (lane == 63) part_t[wave] = x;
    __syncthreads();
    int64_t before = base_t, all = base_t;
    for (int k = 0; k < SCAN_NT / 64; ++k) {
      if (k < wave) before += part_t[k];
      all += part_t[k];
    }
    const int64_t end64 = before + x, begin64 = end64 - len;
    if (end64 > p.tokens && i < p.n) bad |= 4;
    const int begin = int(begin64 < p.tokens ? begin64 : p.tokens);
    const int end = int(end64 < p.tokens ? end64 : p.tokens);
    int cx = (end - begin + DL_CHUNK - 1) / DL_CHUNK;
    const int mine = cx;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int y = __shfl_up(cx, d);
      if (lane >= d) cx += y;
    }
    if (lane == 63) part_c[wave] = cx;
    __syncthreads();
    int cbefore = base_c, call = base_c;
    for (int k = 0; k < SCAN_NT / 64; ++k) {
      if (k < wave) cbefore += part_c[k];
      call += part_c[k];
    }
    if (i < p.n) {
      p.t.cu_tokens[i] = begin;
      p.t.cu_chunks[i] = cbefore + cx - mine;
      int slot = p.slots ? p.slots[i] : i;
      if (slot < 0 || slot >= p.num_slots) { slot = -1; bad |= 1; }
      p.t.seq_slot[i] = slot;
      if (i == p.n - 1) {
        p.t.cu_tokens[p.n] = end;
        p.t.cu_chunks[p.n] = cbefore + cx;
      }
    }
    base_t = all;
    base_c = call;
    if (i < p.n) p.t.order[i] = i;
    __syncthreads();
  }
  if (bad && p.err) atomicOr(p.err, bad);
}

// The last i in [0, n) with cu[i] <= x (cu[0] = 0 <= x): of several that start at x the last,
// which is the one that is not empty.
__device__ __forceinline__ int owner(const int32_t* cu, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (cu[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

__device__ __forceinline__ int4 chunk_of(int c, const int32_t* cu_t, const int32_t* cu_c,
                                         const int32_t* slot, int n) {
  if (c >= cu_c[n]) return make_int4(-1, 0, 0, -1);
  const int s = owner(cu_c, n, c), first = cu_t[s] + DL_CHUNK * (c - cu_c[s]);
  return make_int4(s, first, min(DL_CHUNK, cu_t[s + 1] - first), slot[s]);
}

__global__ __launch_bounds__(256) void table_fill_kernel(TableParams p) {
  const int64_t x = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (x < p.max_chunks)
    reinterpret_cast<int4*>(p.t.chunks)[x] =
        chunk_of(int(x), p.t.cu_tokens, p.t.cu_chunks, p.t.seq_slot, p.n);
  const int64_t r = x - p.max_chunks;
  if (r >= 0 && r < p.tokens)
    p.t.row_slot[r] = r < p.t.cu_tokens[p.n] ? p.t.seq_slot[owner(p.t.cu_tokens, p.n, int(r))] : -1;
}

// Up to 4 NT sequences in one launch: every workgroup adds the lengths up for itself in LDS (four
// sequences a thread) and fills four chunk or token rows a thread from there; the first also
// writes what there is one of.  Measured against two launches, of which the second waits for the
// first and searches in memory: 5 sequences 9 us -> 6, 2000 sequences with a million rows 15 -> 9.
template <int NT>
__global__ __launch_bounds__(NT) void table_few_kernel(TableParams p) {
  constexpr int MOST = 4 * NT;
  constexpr bool ORDER = MOST <= ORDERED;
  __shared__ __attribute__((aligned(16))) int32_t cu_t[MOST + 1], cu_c[MOST + 1], slot[MOST];
  __shared__ __attribute__((aligned(16))) int32_t count[ORDER ? MOST : 4];
  __shared__ int64_t part_t[NT / 64];
  __shared__ int part_c[NT / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int bad = 0;
  int32_t len[4];
  int64_t sum = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int i = 4 * tid + j;
    len[j] = i < p.n ? p.lens[i] : 0;
    int s = i < p.n ? (p.slots ? p.slots[i] : i) : 0;
    if (len[j] < 0) { len[j] = 0; bad |= 4; }
    if (s < 0 || s >= p.num_slots) { s = -1; bad |= 1; }
    slot[i] = s;
    sum += len[j];
  }
  int64_t x = sum;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int64_t y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  if (lane == 63) part_t[wave] = x;
  __syncthreads();
  int64_t at = x - sum;
  for (int k = 0; k < wave; ++k) at += part_t[k];
  int chunks = 0, many[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int i = 4 * tid + j;
    const int begin = int(at < p.tokens ? at : p.tokens);
    at += len[j];
    const int end = int(at < p.tokens ? at : p.tokens);
    if (at > p.tokens && i < p.n) bad |= 4;
    many[j] = (end - begin + DL_CHUNK - 1) / DL_CHUNK;
    cu_t[i] = begin;
    if (i == MOST - 1) cu_t[MOST] = end;
    if constexpr (ORDER) count[i] = i < p.n ? many[j] : -1;
    chunks += many[j];
  }
  int c = chunks;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int y = __shfl_up(c, d);
    if (lane >= d) c += y;
  }
  if (lane == 63) part_c[wave] = c;
  __syncthreads();
  c -= chunks;
  for (int k = 0; k < wave; ++k) c += part_c[k];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    cu_c[4 * tid + j] = c;
    c += many[j];
  }
  if (tid == NT - 1) cu_c[MOST] = c;
  __syncthreads();

  if (blockIdx.x == 0) {
    for (int i = tid; i <= p.n; i += NT) {
      p.t.cu_tokens[i] = cu_t[i];
      p.t.cu_chunks[i] = cu_c[i];
    }
    for (int i = tid; i < p.n; i += NT) {
      p.t.seq_slot[i] = slot[i];
      if constexpr (ORDER) {
        // place of a sequence: how many are longer, or as long and before it
        const int mine = count[i];
        int place = 0;
        for (int j = 0; j < p.n; j += 4) {
          const int4 o = *reinterpret_cast<const int4*>(&count[j]);     // past n: -1
          place += (o.x > mine || (o.x == mine && j < i)) + (o.y > mine || (o.y == mine && j + 1 < i)) +
                   (o.z > mine || (o.z == mine && j + 2 < i)) + (o.w > mine || (o.w == mine && j + 3 < i));
        }
        p.t.order[place] = i;
      } else {
        p.t.order[i] = i;
      }
    }
    if (bad && p.err) atomicOr(p.err, bad);
  }
  // four rows in a row a thread: one search, then on from there
  const int64_t group = int64_t(blockIdx.x) * NT + tid, chunk_groups = (int64_t(p.max_chunks) + 3) / 4;
  if (group < chunk_groups) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t y = 4 * group + j;
      if (y < p.max_chunks) reinterpret_cast<int4*>(p.t.chunks)[y] = chunk_of(int(y), cu_t, cu_c, slot, p.n);
    }
  } else if (const int64_t r0 = 4 * (group - chunk_groups); r0 < p.tokens) {
    const int end = cu_t[p.n];
    int s = r0 < end ? owner(cu_t, p.n, int(r0)) : 0;
    int32_t x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t r = r0 + j;
      if (r < end)
        while (r >= cu_t[s + 1]) ++s;
      x[j] = r < end ? slot[s] : -1;
    }
    typedef __attribute__((ext_vector_type(4), aligned(4))) int32_t i32x4_any;
    if (r0 + 4 <= p.tokens) {
      *reinterpret_cast<i32x4_any*>(p.t.row_slot + r0) = i32x4_any{x[0], x[1], x[2], x[3]};
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (r0 + j < p.tokens) p.t.row_slot[r0 + j] = x[j];
    }
  }
}

}  // namespace

hipError_t launch_tables(const int32_t* lens, const int32_t* slots, int32_t n, int32_t tokens,
                         int32_t num_slots, const dl_tables& t, int32_t* err, int32_t max_chunks,
                         hipStream_t s) {
  TableParams p{lens, slots, t, err, n, tokens, num_slots, max_chunks};
  void* args[] = {&p};
  const int64_t places = int64_t(max_chunks) + tokens;
  const int64_t groups = (int64_t(max_chunks) + 3) / 4 + (int64_t(tokens) + 3) / 4;
  if (n <= ORDERED)
    return hipLaunchKernel(reinterpret_cast<const void*>(&table_few_kernel<ORDERED / 4>),
                           dim3(unsigned((groups + ORDERED / 4 - 1) / (ORDERED / 4))),
                           dim3(ORDERED / 4), args, 0, s);
  if (n <= FEW)
    return hipLaunchKernel(reinterpret_cast<const void*>(&table_few_kernel<FEW / 4>),
                           dim3(unsigned((groups + FEW / 4 - 1) / (FEW / 4))), dim3(FEW / 4), args, 0, s);
  const hipError_t e = hipLaunchKernel(reinterpret_cast<const void*>(&table_scan_kernel), dim3(1),
                                       dim3(SCAN_NT), args, 0, s);
  if (e != hipSuccess) return e;
  return hipLaunchKernel(reinterpret_cast<const void*>(&table_fill_kernel),
                         dim3(unsigned((places + 255) / 256)), dim3(256), args, 0, s);
}

}  // namespace dl
