// What the norm's two directions share: arguments, the layout of a row over lanes, sums over a row, the gate's function.
//
// A row of `width` columns belongs to `lanes` lanes (part of a warp: a power of two, or whole warps), each with E columns of it in
// registers, VEC at a time: columns (n * lanes + lane) * VEC for n < E / VEC.  Rows of a head are held by part of a warp or a warp and meet by shuffles; rows of a
// model by a CTA.  A CTA's rows all belong to one group, so that its weights stay in registers while it walks over the rows;
// the next rows are on their way while one is summed.  Groups are the fastest part of the CTA's number: the CTAs that run together
// cover the same tokens of all groups, whichever of the two layouts ([b, h, T, d] or [b, T, h, d]) a tensor has.
#pragma once
#include <cuda_runtime.h>

#include "smat_launch.cuh"
#include "smat_rows.cuh"

constexpr int NORM_MAX_WIDTH = 16384;
constexpr int NORM_SMS = 148;

// An operand, and by how much a thread's element of it moves from one tile of a CTA to the next: `step`, and `wrap` more where the
// next tile belongs to the next sequence.
struct NormOperand {
  void* data;
  RowStride at;
  int64_t step, wrap;
};
struct NormArgs {
  NormOperand x, residual, gate, dy, dh_in, y, h, dh, dx, dgate;
  const float *weight, *scale;
  int64_t weight_group;
  float *dw, *ds;             // partial rows [groups][CTAs of a group][width], or null
  uint32_t batch, T;          // (1, batch * T) where every operand has its sequences one behind the other
  uint32_t tiles;             // of a sequence: as many tokens as a CTA has rows
  uint32_t groups, ctas;      // CTAs of a group
  uint32_t step_batch, step_tile;   // ctas = step_batch * tiles + step_tile
  int width, lanes;
  float eps, inv_width;
  int sigmoid;
};

// A CTA's place in its walk over the tiles: sequence b, tile i of it.
struct NormWalk {
  uint32_t b, i, slots, slot;
  bool wrapped;
  __device__ __forceinline__ NormWalk(const NormArgs& a)
      : slots(blockDim.x / a.lanes), slot(threadIdx.x / a.lanes), wrapped(false) {
    const uint32_t tile = blockIdx.x / a.groups;
    b = tile / a.tiles;
    i = tile - b * a.tiles;
  }
  __device__ __forceinline__ void next(const NormArgs& a) {
    b += a.step_batch;
    i += a.step_tile;
    wrapped = i >= a.tiles;
    if (wrapped) {
      i -= a.tiles;
      ++b;
    }
  }
  __device__ __forceinline__ bool more(const NormArgs& a) const { return b < a.batch; }
  __device__ __forceinline__ bool in(const NormArgs& a) const { return b < a.batch && i * slots + slot < a.T; }
  template <typename T>
  __device__ __forceinline__ T* seat(const NormOperand& o, uint32_t g, int col) const {
    return static_cast<T*>(o.data) + b * o.at.batch + g * o.at.head + (i * slots + slot) * o.at.token + col;
  }
};
template <typename T>
__device__ __forceinline__ void norm_move(T*& p, const NormOperand& o, bool wrapped) {
  p += o.step;
  if (wrapped) p += o.wrap;
}

// What a kernel is compiled for: rows alone, with the residual stream (forward) or the branch's scale (backward), behind a block with
// one of the gates, or anything, decided by the operands that are given.
// A kernel that asks at run time issues twice the instructions of one that does not, and it is instructions that bound the gated
// norms of heads.
enum NormMode { NORM_ROWS, NORM_STREAM, NORM_SILU, NORM_SIGMOID, NORM_ANY };

// Pairs of columns: one instruction for both (FFMA2 and its like).
__device__ __forceinline__ float2 norm_both(float v) { return make_float2(v, v); }
template <int VEC, int E, typename V>
__device__ __forceinline__ float2 norm_pair(const V (&v)[E / VEC], int j) {
  return make_float2(v[2 * j / VEC].get(2 * j % VEC), v[(2 * j + 1) / VEC].get((2 * j + 1) % VEC));
}

template <typename T>
__device__ __forceinline__ float2 norm_sigmoid(float2 z) {
  if constexpr (sizeof(T) == 4) {
    return make_float2(1.f / (1.f + expf(-z.x)), 1.f / (1.f + expf(-z.y)));
  } else {      // rounded to bf16 soon: powers and reciprocals within 2^-22, results below 2^-126 zero
    float2 e = __fmul2_rn(z, norm_both(-1.4426950408889634f)), r;
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(e.x));
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(e.y));
    e = __fadd2_rn(e, norm_both(1.f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.x) : "f"(e.x));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.y) : "f"(e.y));
    return r;
  }
}

// Rows on their way, for operands that move in 16-byte pieces: DEPTH rows of N operands, each thread's pieces in places of its own of
// shared memory, filled by asynchronous copies.  Nobody else reads them, so that no barrier is needed; with the next row in
// registers instead (24 KB an SM on the way) the gated norms of heads took 157 us for 122 us of bytes.
template <int N, int DEPTH>
struct NormRing {
  uint32_t base, stride, slot = 0;
  __device__ __forceinline__ NormRing(void* shared)
      : base((uint32_t)__cvta_generic_to_shared(shared) + threadIdx.x * 16u), stride(blockDim.x * 16u) {}
  __device__ __forceinline__ void fetch(int k, const void* from, bool in) const {      // zeros where it is not in
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(base + (slot * N + k) * stride), "l"(from), "r"(in ? 16 : 0)
                 : "memory");
  }
  __device__ __forceinline__ void fetched() { asm volatile("cp.async.commit_group;" ::: "memory"); }
  __device__ __forceinline__ void wait() const { asm volatile("cp.async.wait_group %0;" ::"n"(DEPTH - 1) : "memory"); }
  __device__ __forceinline__ void landed() const { asm volatile("cp.async.wait_all;" ::: "memory"); }
  template <typename V>
  __device__ __forceinline__ void read(int k, V& v) const {
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v.w[0]), "=r"(v.w[1]), "=r"(v.w[2]), "=r"(v.w[3]) : "r"(base + (slot * N + k) * stride) : "memory");
  }
  __device__ __forceinline__ void next() { slot = slot + 1 == DEPTH ? 0 : slot + 1; }
};
// Whether a row of `operands` pieces a thread has room in shared memory (fp32 rows of more than 8192 columns do not).
__host__ __device__ constexpr bool norm_rings(int operands, int threads) { return operands * threads * 16 <= 160 * 1024; }
// Rows on their way for a thread that has room for so many pieces of 16 bytes (the forward pass 8: with four CTAs an SM, and so that
// small calls take no more shared memory than every kernel may, asking for more costs a call of the runtime; the backward pass 16).
__host__ __device__ constexpr int norm_depth(int operands, int pieces, int threads) {
  const int depth = (threads > 512 ? 8 : pieces) / operands;
  return depth > 5 ? 5 : depth < 1 ? 1 : depth;
}

// Sums over the lanes of a row, the same in each of them: inside a warp by shuffles, then one word of shared memory a warp and
// shuffles again.  `turn` alternates between the two halves of the exchange buffer, so that one barrier a sum is enough.
template <int N>
__device__ __forceinline__ void norm_row_sum(float (&v)[N], int lanes, int turn, float (*part)[32][N]) {
  for (int o = min(lanes, 32) / 2; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
  if (lanes <= 32) return;
  const int warps = lanes / 32, lane = threadIdx.x & 31;
  if (lane == 0)
#pragma unroll
    for (int i = 0; i < N; ++i) part[turn & 1][threadIdx.x >> 5][i] = v[i];
  __syncthreads();
  const int all = warps > 16 ? 32 : warps > 8 ? 16 : warps > 4 ? 8 : warps > 2 ? 4 : 2, other = lane & (all - 1);
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = other < warps ? part[turn & 1][other][i] : 0.f;
  for (int o = all / 2; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
}

// Columns a lane holds, the CTA's threads at most and the lanes, by the width: a power of two up to a warp, then whole warps.  Sixteen
// columns where a kernel has registers for them (`roomy`) and the row is longer than a head's, else eight: what a thread does once
// a row is most of what it issues (norm gradients of 512 columns: 114 us with eight and a barrier a row).  The gradients
// with a scale or a gate have registers for eight (sixteen spilled 800 bytes).
struct NormShape {
  int columns, threads, lanes;
};
inline NormShape norm_shape(int width, bool roomy) {
  const int columns = width > 8 * 1024 || (roomy && width > 256) ? 16 : 8;
  int lanes = 1;
  while (lanes < 32 && lanes * columns < width) lanes *= 2;
  if (lanes * columns < width) lanes = (width + columns * 32 - 1) / (columns * 32) * 32;
  return {columns, lanes <= 256 ? 256 : lanes <= 512 ? 512 : lanes <= 768 && columns == 8 ? 768 : 1024, lanes};
}

// The walk of at most `ctas` CTAs a group over tiles of `slots` tokens.
inline void norm_walk(NormArgs* a, uint32_t slots, uint32_t ctas) {
  a->tiles = (a->T + slots - 1) / slots;
  const uint32_t all = a->tiles * a->batch;
  a->ctas = ctas < 1 ? 1 : ctas > all ? all : ctas;
  a->step_batch = a->ctas / a->tiles;
  a->step_tile = a->ctas % a->tiles;
  for (NormOperand* o : {&a->x, &a->residual, &a->gate, &a->dy, &a->dh_in, &a->y, &a->h, &a->dh, &a->dx, &a->dgate}) {
    o->step = a->step_batch * o->at.batch + (int64_t)a->step_tile * slots * o->at.token;
    o->wrap = o->at.batch - (int64_t)a->tiles * slots * o->at.token;
  }
}

inline int norm_ctas_an_sm(int resident, uint32_t threads) { return threads >= (uint32_t)resident ? 1 : resident / (int)threads; }

// A launch with a ring of `operands` pieces a row (none: 0) for each of its threads.  CTAs walk over the rows, so that each SM has to
// get as many of them: they ask for so much shared memory that no more fit.  (Where a fourth one fitted beside three, SMs that
// drained early took four of the next launch and left others with two: the gated norm of heads took 167 us for 132.)
template <typename Kernel>
cudaError_t norm_launch(Kernel kernel, int operands, int pieces, size_t least, int most_threads, int an_sm, dim3 grid, uint32_t threads, cudaStream_t st, const NormArgs& a) {
  size_t bytes = operands && norm_rings(operands, most_threads) ? (size_t)norm_depth(operands, pieces, most_threads) * operands * threads * 16 : 0;
  if (bytes < least) bytes = least;
  const size_t no_more = (size_t)228 * 1024 / (an_sm + 1) - 1024 + 256;      // (1 KB a CTA is the system's)
  if (bytes < no_more && an_sm > 2) bytes = no_more;
  if (bytes + 512 > 48 * 1024) {      // (with the exchange that a kernel has besides)
    const cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (err != cudaSuccess) return err;
  }
  return smat_launch_pdl(kernel, grid, threads, bytes, st, a);
}

// Launchers of the two directions.  vec: elements that the rows of all operands can be moved by (16 bytes of them, 2 bf16, or 1).
int smat_norm_partials(int groups, int width);      // rows of partial sums, for any call of this width
cudaError_t smat_launch_norm_forward(NormArgs& a, int bf16, int vec, cudaStream_t st);
cudaError_t smat_launch_norm_backward(NormArgs& a, int bf16, int vec, float* dw, float* ds, cudaStream_t st);
cudaError_t smat_launch_norm_backward_f32(NormArgs& a, int vec, float* dw, float* ds, cudaStream_t st);
