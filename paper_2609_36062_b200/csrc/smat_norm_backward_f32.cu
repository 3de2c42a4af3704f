// Gradients of the norm, fp32 rows.
#include "smat_norm_backward.cuh"

cudaError_t smat_launch_norm_backward_f32(NormArgs& a, int vec, float* dw, float* ds, cudaStream_t st) {
  return vec == 4 ? moded<float, 4>(a, dw, ds, st) : moded<float, 1>(a, dw, ds, st);
}
