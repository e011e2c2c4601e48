// Host entry points of the input projection with 4-bit weights and of the gated layer's single step (q4_kernels.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>

namespace pararnn {

size_t q4_packed_bytes(int H, int G, int n_heads);
size_t q4_scale_bytes(int H, int G, int n_heads, int group);
int q4_quantize(const float *Wx, int H, int G, int n_heads, int group, void *packed, void *scales, hipStream_t st);
int q4_pack(const signed char *codes, const void *code_scales, int H, int G, int n_heads, int group, void *packed, void *scales,
            hipStream_t st);
int q4_dequantize(const void *packed, const void *scales, int H, int G, int n_heads, int group, float *Wx, hipStream_t st);
int q4_set_products(int mode);
int q4_products();
int q4_exact_rows(int H, int G, int n_heads);
size_t q4_workspace_bytes(int dtype, int B, int L, int H, int G, int n_heads, int group);
int q4_project(int dtype, const void *x, const void *packed, const void *scales, const float *bias, int B, int L, int H, int G,
               int n_heads, int group, void *u, void *workspace, size_t workspace_bytes, hipStream_t st);
int q4_step(int dtype, const void *x, const void *packed, const void *scales, const float *bias, const float *h, int B, int H, int G,
            int n_heads, int group, void *y, float *h_next, hipStream_t st);

}  // namespace pararnn
