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

// Running token and chunk counts, one workgroup.  A length below 0 counts as 0, and a
// sequence that would run past the token rows ends with them.
__global__ __launch_bounds__(SCAN_NT) void table_scan_kernel(TableParams p) {
  __shared__ int64_t part_t[SCAN_NT / 64];
  __shared__ int part_c[SCAN_NT / 64];
  __shared__ __attribute__((aligned(16))) int count[SCAN_NT];
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
    if (p.n > SCAN_NT && i < p.n) p.t.order[i] = i;
    count[tid] = i < p.n ? mine : -1;
    __syncthreads();
  }
  if (p.n <= SCAN_NT && tid < p.n) {
    // place of a sequence: how many are longer, or as long and before it
    const int mine = count[tid];
    int place = 0;
    for (int j = 0; j < p.n; j += 4) {
      const int4 c = *reinterpret_cast<const int4*>(&count[j]);     // past n: -1
      place += (c.x > mine || (c.x == mine && j < tid)) + (c.y > mine || (c.y == mine && j + 1 < tid)) +
               (c.z > mine || (c.z == mine && j + 2 < tid)) + (c.w > mine || (c.w == mine && j + 3 < tid));
    }
    p.t.order[place] = tid;
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

__global__ __launch_bounds__(256) void table_fill_kernel(TableParams p) {
  const int64_t x = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (x < p.max_chunks) {
    const int c = int(x);
    int4 row = make_int4(-1, 0, 0, -1);
    if (c < p.t.cu_chunks[p.n]) {
      const int s = owner(p.t.cu_chunks, p.n, c);
      const int first = p.t.cu_tokens[s] + DL_CHUNK * (c - p.t.cu_chunks[s]);
      row = make_int4(s, first, min(DL_CHUNK, p.t.cu_tokens[s + 1] - first), p.t.seq_slot[s]);
    }
    reinterpret_cast<int4*>(p.t.chunks)[c] = row;
  }
  const int64_t r = x - p.max_chunks;
  if (r >= 0 && r < p.tokens)
    p.t.row_slot[r] = r < p.t.cu_tokens[p.n] ? p.t.seq_slot[owner(p.t.cu_tokens, p.n, int(r))] : -1;
}

}  // namespace

hipError_t launch_tables(const int32_t* lens, const int32_t* slots, int32_t n, int32_t tokens,
                         int32_t num_slots, const dl_tables& t, int32_t* err, int32_t max_chunks,
                         hipStream_t s) {
  TableParams p{lens, slots, t, err, n, tokens, num_slots, max_chunks};
  void* args[] = {&p};
  const hipError_t e = hipLaunchKernel(reinterpret_cast<const void*>(&table_scan_kernel), dim3(1),
                                       dim3(SCAN_NT), args, 0, s);
  if (e != hipSuccess) return e;
  const int64_t places = int64_t(max_chunks) + tokens;
  return hipLaunchKernel(reinterpret_cast<const void*>(&table_fill_kernel),
                         dim3(unsigned((places + 255) / 256)), dim3(256), args, 0, s);
}

}  // namespace dl
