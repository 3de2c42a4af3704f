// Gated linear recurrence of every channel: what its kernels share.
#pragma once
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include "smat_launch.cuh"
#include "smat_rows.cuh"

constexpr int REC_THREADS = 256, REC_WARPS = REC_THREADS / 32, REC_MAX_CLUSTER = 8;
constexpr int64_t REC_CTAS = 148 * 2;     // as many as run at once

struct RecArgs {
  const void *x, *log_a, *h;      // forward: x; backward: dh and the h that was kept
  void *out, *dlog_a;             // forward: h; backward: dx
  RowStride xs, as, hs, os, das;
  const float *begin;             // the state that enters the first token in the order of the recurrence (h0, dhT), or null
  const float *h0;                // backward: the state before token 0, or null
  float* end;                     // the state behind the last (hT, dh0), or null
  int64_t T;
  int channels;
};

// a * state + x, a closed gate forgetting the state whatever it is.
__device__ __forceinline__ float rec_step(float a, float state, float x) { return a == 0.f ? x : fmaf(a, state, x); }

// Whether a sum of numbers times zero has met one that is not finite.  Only then does a closed gate need looking at (0 * state is
// no zero): the loops over tokens run without it, and once more with it where what they come to is not finite.
__device__ __forceinline__ bool rec_not_finite(float zeros) { return zeros != 0.f; }

// CTAs of a cluster, which take tiles in turn: as many as fill the GPU, and no more than there are tiles.
inline unsigned rec_ranks(int64_t columns, int64_t batch, int64_t tiles) {
  unsigned ranks = 1;
  while (2 * ranks <= REC_MAX_CLUSTER && 2 * ranks <= tiles && columns * batch * 2 * ranks <= REC_CTAS) ranks *= 2;
  return ranks;
}

// The kernel whose tiles move by TMA (smat_recurrence_tma.cu), where every operand's rows are whole multiples of 16 bytes apart.
// bf16: of x, gates.
bool smat_recurrence_tma_supported(const RecArgs& a, int batch, int x_bf16, int gate_bf16, bool back);
cudaError_t smat_launch_recurrence_tma(const RecArgs& a, int batch, int x_bf16, int gate_bf16, bool back, cudaStream_t st);
