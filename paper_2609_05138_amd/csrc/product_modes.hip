// Host side of the products with epilogues of their own.
#include "product_modes.h"

namespace som {
namespace {

__global__ void __launch_bounds__(256) k_join_extra(const ExtraArgs a) {
  join_extra(a, static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x);
}

}  // namespace

hipError_t launch_mode(int mode, int shape, const ProductArgs& a, hipStream_t stream) {
  return a.elem == kF16 ? launch_modes_f16(mode, shape, a, stream) : launch_modes_bf16(mode, shape, a, stream);
}

hipError_t launch_extra(ExtraArgs a, float* partial, hipStream_t stream) {
  a.dma = rows_on_16(a);
  const RuledPlan p = plan_extra(a.I, a.J, a.K, a.elem, a.p_kc, a.q_kc, a.dma, a.symmetric);
  set_launch(a, p, partial, p.upper);
  if (p.upper) return launch_mirror_f16(p.shape, a, stream);
  const hipError_t e = launch_mode(kExtra, p.shape, a, stream);
  if (e != hipSuccess || p.splits == 1) return e;
  hipLaunchKernelGGL(k_join_extra, dim3(static_cast<uint32_t>((join_threads(a) + 255) / 256)), dim3(256), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_parts(ExtraArgs& a, float* partial, hipStream_t stream) {
  a.dma = rows_on_16(a);
  const RuledPlan p = plan_extra(a.I, a.J, a.K, a.elem, a.p_kc, a.q_kc, a.dma);
  set_launch(a, p, partial);
  return launch_mode(kExtra, p.shape, a, stream);
}

}  // namespace som
