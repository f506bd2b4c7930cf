// The operators around and beside the local attention: what the C ABI layer (operators_api.cu) launches.
#pragma once
#include "sparse_common.cuh"

namespace slide_attn {

// Group norm over [B][P][C].  group_norm_workspace: of the forward (maps = 1) or the backward (2); false where the shape is not supported.
bool group_norm_workspace(long long B, long long P, int C, int groups, slide_attn_dtype dtype, int maps, size_t* bytes);
cudaError_t launch_group_norm_forward(const void* x, const float* gamma, const float* beta, long long B, long long P, int C, int groups, float eps,
                                      slide_attn_activation act, slide_attn_dtype dtype, void* y, float* mean, float* rstd, void* workspace,
                                      cudaStream_t stream);
cudaError_t launch_group_norm_backward(const void* x, const float* gamma, const float* beta, const float* mean, const float* rstd, const void* dy,
                                       long long B, long long P, int C, int groups, slide_attn_activation act, slide_attn_dtype dtype, void* dx,
                                       float* dgamma, float* dbeta, void* workspace, cudaStream_t stream);

bool dropout_supports(long long images, long long per_image, bool whole_images);
cudaError_t launch_dropout(const void* x, const void* residual, void* y, long long images, long long per_image, double p, bool whole_images,
                           const unsigned long long* rng, slide_attn_dtype dtype, int num_sms, cudaStream_t stream);

// pooled: 2 B heads blocks head_dim doubles; the backward's workspace: see Prepared in sparse_bwd_kernel.cu.
cudaError_t launch_select(sparse::Geometry g, long long B, int head_dim, slide_attn_dtype dtype, const void* q, const void* k, double* pooled,
                          int* idx, int num_sms, cudaStream_t stream);
cudaError_t launch_sparse_forward(sparse::Geometry g, long long B, int head_dim, slide_attn_dtype dtype, const void* q, const void* k,
                                  const void* v, const int* idx, void* out, float* lse, int num_sms, cudaStream_t stream);
cudaError_t launch_sparse_backward(sparse::Geometry g, long long B, int head_dim, slide_attn_dtype dtype, const sparse::BackwardMaps& m,
                                   void* workspace, int num_sms, cudaStream_t stream);

}  // namespace slide_attn
