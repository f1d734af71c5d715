// embed_grad: by the gradient's type (embed_grad.cuh), each in a translation
// unit of its own.
#include "adapm.h"
#include "embed.cuh"

namespace adapm {

GradPlan grad_plan_f32(const GradArgs& a, int sms);
GradPlan grad_plan_f16(const GradArgs& a, int sms);
GradPlan grad_plan_bf16(const GradArgs& a, int sms);
void launch_embed_grad_f32(const GradArgs& a, const GradPlan& p, cudaStream_t stream);
void launch_embed_grad_f16(const GradArgs& a, const GradPlan& p, cudaStream_t stream);
void launch_embed_grad_bf16(const GradArgs& a, const GradPlan& p, cudaStream_t stream);

GradPlan grad_plan(const GradArgs& a, int sms) {
  if (a.grad.type == ADAPM_F32) return grad_plan_f32(a, sms);
  return a.grad.type == ADAPM_F16 ? grad_plan_f16(a, sms) : grad_plan_bf16(a, sms);
}

void launch_embed_grad(const GradArgs& a, const GradPlan& p, cudaStream_t stream) {
  if (a.grad.type == ADAPM_F32) launch_embed_grad_f32(a, p, stream);
  else if (a.grad.type == ADAPM_F16) launch_embed_grad_f16(a, p, stream);
  else launch_embed_grad_bf16(a, p, stream);
}

}  // namespace adapm
