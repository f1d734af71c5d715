// embed_grad for gradients of type __nv_bfloat16 (embed_grad.cuh).
#include "embed_grad.cuh"

namespace adapm {

GradPlan grad_plan_bf16(const GradArgs& a, int sms) { return grad_plan_typed<__nv_bfloat16>(a, sms); }
void launch_embed_grad_bf16(const GradArgs& a, const GradPlan& p, cudaStream_t stream) {
  launch_grad_typed<__nv_bfloat16>(a, p, stream);
}

}  // namespace adapm
