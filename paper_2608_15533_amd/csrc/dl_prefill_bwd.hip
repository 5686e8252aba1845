// Whole sequences: the backward pass's launches.
#include "dl_grad.hpp"
#include "dl_seq.hpp"

namespace dl {
namespace {

template <typename K>
hipError_t start(K* kernel, int64_t grid, int block, const SeqParams& p, hipStream_t s) {
  SeqParams q = p;
  void* args[] = {&q};
  return hipLaunchKernel(reinterpret_cast<const void*>(kernel), dim3(unsigned(grid)), dim3(block),
                         args, 0, s);
}

template <int DC, int DK, bool DELTA, typename TIN>
hipError_t launch_grad(const SeqParams& p, hipStream_t s) {
  const int64_t grid = int64_t(p.max_chunks) * p.H;
  return p.dv == 128 ? start(&grad_kernel<DC, DK, 128, DELTA, TIN>, grid, 4 * DK, p, s)
                     : start(&grad_kernel<DC, DK, 64, DELTA, TIN>, grid, 4 * DK, p, s);
}

template <int DK, bool RAW, bool DELTA, typename TIN>
hipError_t launch_walks(const SeqParams& p, hipStream_t s) {
  const int64_t heads = int64_t(p.n) * p.H;
  const int waves = walk_waves(2 * heads, DK, p.dv, RAW);
  const int64_t grid = 2 * heads * (p.dv / 16 / waves);
  switch (waves) {
    case 2: return start(&both_kernel<DK, 1, 2, RAW, DELTA, TIN>, grid, 128, p, s);
    case 4: return start(&both_kernel<DK, 1, 4, RAW, DELTA, TIN>, grid, 256, p, s);
    default: return start(&both_kernel<DK, 1, 8, RAW, DELTA, TIN>, grid, 512, p, s);
  }
}

template <int DK, typename TIN>
hipError_t launch_backward_shape(int op, const SeqParams& p, hipStream_t s) {
  hipError_t e = hipErrorInvalidValue;
  if constexpr (sizeof(TIN) == 2)
    if (p.raw) e = p.delta ? launch_walks<DK, true, true, TIN>(p, s) : launch_walks<DK, true, false, TIN>(p, s);
  if (!p.raw) e = p.delta ? launch_walks<DK, false, true, TIN>(p, s) : launch_walks<DK, false, false, TIN>(p, s);
  if (e != hipSuccess) return e;
  switch (op) {
    case DL_OP_GDN: return launch_grad<DC_SCALAR, DK, true, TIN>(p, s);
    case DL_OP_KDA: return launch_grad<DC_KEY, DK, true, TIN>(p, s);
    case DL_OP_GLA: return launch_grad<DC_KEY, DK, false, TIN>(p, s);
    case DL_OP_RWKV6:
      e = launch_grad<DC_BONUS, DK, false, TIN>(p, s);
      return e != hipSuccess ? e : start(&bonus_grad_kernel<DK>, p.H, 1024, p, s);
  }
  return launch_grad<DC_SCALAR, DK, false, TIN>(p, s);   // RetNet, linear attention
}

}  // namespace

hipError_t launch_backward(const dl_desc* d, const SeqParams& p, hipStream_t s) {
  if (d->in_dtype == DL_BF16)
    return d->dk == 128 ? launch_backward_shape<128, uint16_t>(d->op, p, s)
                        : launch_backward_shape<64, uint16_t>(d->op, p, s);
  return d->dk == 128 ? launch_backward_shape<128, float>(d->op, p, s)
                      : launch_backward_shape<64, float>(d->op, p, s);
}

}  // namespace dl
