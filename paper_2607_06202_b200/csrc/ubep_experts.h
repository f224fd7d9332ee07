// Host-visible launchers of the kernels in ubep_experts.cu and ubep_route.cu; arguments as the C ABI's, already checked.
#pragma once

#include <cuda_runtime.h>

#include "../../include/ubep.h"

namespace ubep {

cudaError_t launch_expert_gated(const ubep_expert_rows_t& r, const void* x, const float* x_scale, const void* w, int H, int I, int act,
                                void* h, void* pre, void* scratch, cudaStream_t st, int* launches);
cudaError_t launch_expert_gated_backward(const ubep_expert_rows_t& r, const void* x, const float* x_scale, const void* w, const void* pre,
                                         const void* grad_h, int H, int I, int act, void* grad_pre, void* grad_x, void* grad_w,
                                         void* scratch, cudaStream_t st, int* launches);
cudaError_t launch_expert_linear(const ubep_expert_rows_t& r, const void* x, const void* w, const void* bias, const float* row_scale,
                                 const void* residual, int K, int N, int act, void* y, void* pre, cudaStream_t st, int* launches);
cudaError_t launch_expert_linear_backward(const ubep_expert_rows_t& r, const void* x, const void* w, const void* pre,
                                          const float* row_scale, const void* grad_y, int K, int N, int act, void* grad_pre,
                                          void* grad_x, void* grad_w, void* grad_bias, float* grad_scale, float* scratch,
                                          cudaStream_t st, int* launches);
cudaError_t launch_route(const void* logits, int type, int T, int E, int k, int renormalize, int32_t* topk_idx, float* topk_w,
                         cudaStream_t st);
cudaError_t launch_route_backward(const void* logits, int type, const int32_t* topk_idx, const float* grad_w, int T, int E, int k,
                                  int renormalize, void* grad_logits, cudaStream_t st);

}  // namespace ubep
