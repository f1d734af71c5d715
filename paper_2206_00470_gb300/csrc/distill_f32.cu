// The distillation kernels (distill.cuh) of fp32 logits.
#include "distill.cuh"

namespace adapm {

void launch_distill_f32(const DistillArgs& a, int sms, cudaStream_t stream) {
  launch_distill_type<ADAPM_F32>(a, sms, stream);
}

}  // namespace adapm
