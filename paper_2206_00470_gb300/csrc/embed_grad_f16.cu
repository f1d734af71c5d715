// embed_grad for gradients of type __half (embed_grad.cuh).
#include "embed_grad.cuh"

namespace adapm {

GradPlan grad_plan_f16(const GradArgs& a, int sms) { return grad_plan_typed<__half>(a, sms); }
void launch_embed_grad_f16(const GradArgs& a, const GradPlan& p, cudaStream_t stream) {
  launch_grad_typed<__half>(a, p, stream);
}

}  // namespace adapm
