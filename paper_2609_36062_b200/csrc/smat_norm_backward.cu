// Gradients of the norm, bf16 rows (a translation unit for each type: they are what the library's build waits for).
#include "smat_norm_backward.cuh"

// CTAs of a backward pass over many rows, all groups together: as many as run at once (for either layout of the row), one at least
// for each group.
int smat_norm_partials(int groups, int width) {
  int most = groups;
  for (const bool roomy : {false, true}) {
    const int lanes = norm_shape(width, roomy).lanes, all = NORM_SMS * norm_ctas_an_sm(512, lanes <= 32 ? 256 : lanes);
    if (all > most) most = all;
  }
  return most;
}

cudaError_t smat_launch_norm_backward(NormArgs& a, int bf16, int vec, float* dw, float* ds, cudaStream_t st) {
  if (!bf16) return smat_launch_norm_backward_f32(a, vec, dw, ds, st);
  return vec == 8 ? moded<__nv_bfloat16, 8>(a, dw, ds, st)
                  : vec == 2 ? moded<__nv_bfloat16, 2>(a, dw, ds, st) : moded<__nv_bfloat16, 1>(a, dw, ds, st);
}
