// Gated linear recurrence of every channel: what its kernels share.
#pragma once
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include "smat_launch.cuh"
#include "smat_room.h"
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

// The factor of a piece of tokens is the product of its gates, and zero only where one of them is closed: a product of open gates that
// fp32 has no number for (nine of exp(-12)) is held at the smallest one, so that a state that is not finite stays so.  For a finite
// state this is the error that products below 2^-126 have anyway, 2^-149 of it.  (A product with a gate that is NaN needs no care: what
// that gate leaves is NaN by itself, until a closed one.)
constexpr float REC_LEAST = 0x1p-149f;
__device__ __forceinline__ float rec_factor(float product, float least_gate) { return fmaxf(product, fminf(least_gate, REC_LEAST)); }
// ... of two pieces in a row.
__device__ __forceinline__ float rec_joined(float later, float earlier) { return rec_factor(later * earlier, fminf(later, earlier)); }

// Whether a sum of numbers times zero has met one that is not finite.  Only then does a closed gate need looking at (0 * state is
// no zero): the loops over tokens run without it, and once more with it where what they come to is not finite.
__device__ __forceinline__ bool rec_not_finite(float zeros) { return zeros != 0.f; }

// How many clusters of `ranks` CTAs of this kernel run at once on the current device; -1: not known.  (Which SMs a cluster may use is
// up to the device: of 296 places of CTAs, clusters of 8, 4 and 2 had 264, 280 and 296.)
template <typename... KArgs>
int rec_clusters(void (*kernel)(KArgs...), size_t smem, unsigned ranks) {
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = ranks;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(ranks);
  cfg.blockDim = dim3(REC_THREADS);
  cfg.dynamicSmemBytes = smem;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  int n = 0;
  if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) == cudaSuccess) return n;
  cudaGetLastError();
  return -1;
}

// What one kernel's rec_clusters come to.
using RecRoom = SmatRoom<REC_MAX_CLUSTER>;

// CTAs of a cluster, which take tiles in turn: as many as all run at once, and no more than there are tiles; one where the device does
// not tell.  A second wave costs as much as the first (16 K tokens of 2112 bf16 channels 42 us, with one cluster of eight too many,
// 2176 channels, 67).
template <typename... KArgs>
unsigned rec_ranks(RecRoom& room, void (*kernel)(KArgs...), size_t smem, int64_t columns, int64_t batch, int64_t tiles) {
  int device = -1;
  if (cudaGetDevice(&device) != cudaSuccess) cudaGetLastError();
  unsigned ranks = REC_MAX_CLUSTER;
  while (ranks > 1 && (ranks > tiles || columns * batch * ranks > REC_CTAS ||
                       columns * batch > room(device, ranks, [&] { return rec_clusters(kernel, smem, ranks); })))
    --ranks;
  return ranks;
}

// The kernel whose tiles move by TMA (smat_recurrence_tma.cu), where every operand's rows are whole multiples of 16 bytes, and as far apart.
// bf16: of x, gates.
bool smat_recurrence_tma_supported(const RecArgs& a, int batch, int x_bf16, int gate_bf16, bool back);
cudaError_t smat_launch_recurrence_tma(const RecArgs& a, int batch, int x_bf16, int gate_bf16, bool back, cudaStream_t st);
