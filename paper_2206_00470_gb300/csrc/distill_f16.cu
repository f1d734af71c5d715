// The distillation kernels (distill.cuh) of fp16 logits.
#include "distill.cuh"

namespace adapm {

void launch_distill_f16(const DistillArgs& a, int sms, cudaStream_t stream) {
  launch_distill_type<ADAPM_F16>(a, sms, stream);
}

}  // namespace adapm
