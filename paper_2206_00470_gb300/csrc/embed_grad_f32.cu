// embed_grad for gradients of type float (embed_grad.cuh).
#include "embed_grad.cuh"

namespace adapm {

GradPlan grad_plan_f32(const GradArgs& a, int sms) { return grad_plan_typed<float>(a, sms); }
void launch_embed_grad_f32(const GradArgs& a, const GradPlan& p, cudaStream_t stream) {
  launch_grad_typed<float>(a, p, stream);
}

}  // namespace adapm
