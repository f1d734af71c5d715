// The distillation kernels (distill.cuh) of bf16 logits.
#include "distill.cuh"

namespace adapm {

void launch_distill_bf16(const DistillArgs& a, int sms, cudaStream_t stream) {
  launch_distill_type<ADAPM_BF16>(a, sms, stream);
}

}  // namespace adapm
