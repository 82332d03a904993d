// What the two paths of the vocabulary's cross entropy share: vocabloss.cu and, for a few tokens, vocabloss_few.cu.
#pragma once
#include "packed.cuh"

namespace chela {

// Factor of a sum of 2^(z - before) whose maximum becomes `now`.  Nothing yet (-infinity twice) stays as it is, and so does a
// sum that NaN logits left there: the maximum passes over them, the sum does not.
__device__ __forceinline__ float rescale(float before, float now) { return before == now ? 1.f : ex2(before - now); }

// 0 where the sizes are not for this path: more than a few tokens, or rows too wide for it
size_t vocabloss_few_workspace_bytes(int T, int V, int D, chela_dtype_t in_dtype, bool grad);
chela_status_t launch_vocabloss_few_fwd(const chela_vocabloss_args_t &a, float *loss, float *lse, void *workspace, cudaStream_t stream);
chela_status_t launch_vocabloss_few_bwd(const chela_vocabloss_args_t &a, const float *lse, const float *d_loss, const float *d_lse, void *d_h, const void *d_w_in, void *d_w,
                                        chela_dtype_t grad_dtype, void *workspace, cudaStream_t stream);

}  // namespace chela
