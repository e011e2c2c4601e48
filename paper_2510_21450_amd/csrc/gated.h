// Host entry points of the gated linear recurrence (gated_kernels.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>

namespace pararnn {

size_t gated_workspace_bytes(int dtype, int B, int L, int H, int G);
size_t gated_checkpoint_bytes(int dtype, int B, int L, int H, int G);
int gated_forward(int dtype, const void *u, const float *h0, const int *lengths, int B, int L, int H, int G, void *h,
                  float *h_last, float *checkpoints, void *workspace, size_t workspace_bytes, unsigned int spin_limit, hipStream_t st);
int gated_backward(int dtype, const void *u, const float *checkpoints, const int *lengths, const void *dL_dh,
                   const float *dL_dlast, int B, int L, int H, int G, void *dL_du, float *dL_dh0, void *workspace,
                   size_t workspace_bytes, unsigned int spin_limit, hipStream_t st);

}  // namespace pararnn
