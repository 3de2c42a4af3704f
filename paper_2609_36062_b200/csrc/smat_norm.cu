// Root-mean-square norm of rows, before a block or behind it:
//     h = residual + scale x,   r = 1 / sqrt(mean(h²) + eps),   y = h r w act(gate),
// and its gradients: with u = dy act(gate) and n = h r,
//     dn = u w,   dh = r (dn - n mean(dn n)) + dh_in,   dx = scale dh,   dgate = dy n w act'(gate),
//     dw = Σ_rows u n,   dscale = Σ_rows x dh.
// mean(dn n) = r mean(dn h): both sums that a row needs are over what it reads, so it is read once.
//
// Streams over rows with one sum (forward) or two (backward) in the way.  A row belongs to the lanes of part of a warp, of a warp
// or of a CTA: as few as hold it in registers with at most VPT pieces of 16 bytes a lane, so that short rows (a head) meet by
// shuffles alone.  The CTAs of the backward pass walk over the rows with the sums of dw and dscale in registers, one
// column set a thread, and leave one partial row each; a second kernel adds these in a fixed order.
#include <cuda_runtime.h>

#include "smat_launch.cuh"
#include "smat_rows.cuh"

namespace {

constexpr int NORM_THREADS = 256;          // of a CTA that holds several rows
constexpr int NORM_MAX_WIDTH = 16384;
constexpr int NORM_PARTIALS = 148 * 8;     // CTAs of a backward pass at most, all groups together (plus one a group)

struct NormArgs {
  const void *x, *residual, *gate, *dy, *dh_in;
  void *y, *h, *dh, *dx, *dgate;
  RowStride xs, rs, gs, dys, dhis, ys, hs, dhs, dxs, dgs;
  const float *weight, *scale;
  int64_t weight_group;
  float *dw, *ds;             // partial rows [groups][CTAs of a group][width], or null
  uint32_t rows, T;           // batch * T, T
  int width, lanes;           // lanes of a row: a power of two
  float eps, inv_width;
  int sigmoid;
};

template <typename T>
__device__ __forceinline__ float exp_of(float v) { return sizeof(T) == 4 ? expf(v) : __expf(v); }

// act(z), and with SLOPE its derivative.
template <typename T>
__device__ __forceinline__ float gate_of(float z, int sigmoid) {
  const float d = 1.f + exp_of<T>(-z), top = sigmoid ? 1.f : z;
  return sizeof(T) == 4 ? top / d : __fdividef(top, d);
}
template <typename T>
__device__ __forceinline__ void gate_of(float z, int sigmoid, float* act, float* slope) {
  const float d = 1.f + exp_of<T>(-z), s = sizeof(T) == 4 ? 1.f / d : __fdividef(1.f, d);
  *act = sigmoid ? s : z * s;
  *slope = sigmoid ? s * (1.f - s) : s * fmaf(z, 1.f - s, 1.f);
}

// Sums over the lanes of a row, the same in each of them.  `turn` alternates between the two halves of the exchange buffer, so
// that one barrier a sum is enough.
template <int N>
__device__ __forceinline__ void row_sum(float (&v)[N], int lanes, int turn) {
  for (int o = min(lanes, 32) / 2; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
  if (lanes <= 32) return;
  __shared__ float part[2][N][32];
  const int warp = threadIdx.x >> 5;
  if ((threadIdx.x & 31) == 0)
#pragma unroll
    for (int i = 0; i < N; ++i) part[turn & 1][i][warp] = v[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    v[i] = 0.f;
    for (int w = 0; w < lanes / 32; ++w) v[i] += part[turn & 1][i][w];
  }
}

__device__ __forceinline__ int64_t at(const RowStride& s, uint32_t b, uint32_t g, uint32_t t) {
  return b * s.batch + g * s.head + t * s.token;
}

template <typename T, int VEC, int VPT>
__global__ void __launch_bounds__(1024) norm_forward_kernel(const NormArgs a) {
  pdl_trigger();
  const uint32_t slot = threadIdx.x / a.lanes, row = blockIdx.x * (blockDim.x / a.lanes) + slot, g = blockIdx.y;
  const int lane = threadIdx.x % a.lanes;
  const bool valid = row < a.rows;
  const uint32_t b = valid ? row / a.T : 0u, t = valid ? row - b * a.T : 0u;
  pdl_wait();
  RowVec<T, VEC> x[VPT], r[VPT], z[VPT];
#pragma unroll
  for (int n = 0; n < VPT; ++n) {
    const int col = (n * a.lanes + lane) * VEC;
    x[n].clear();
    if (a.residual) r[n].clear();
    if (!valid || col >= a.width) continue;
    x[n].load(static_cast<const T*>(a.x) + at(a.xs, b, g, t) + col);
    if (a.residual) r[n].load(static_cast<const T*>(a.residual) + at(a.rs, b, g, t) + col);
    if (a.gate) z[n].load(static_cast<const T*>(a.gate) + at(a.gs, b, g, t) + col);
  }
  float h[VPT][VEC], sum[1] = {0.f};
#pragma unroll
  for (int n = 0; n < VPT; ++n) {
    const int col = (n * a.lanes + lane) * VEC;
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      float v = x[n].get(i);
      if (a.scale && col < a.width) v *= a.scale[col + i];
      if (a.residual) v += r[n].get(i);
      h[n][i] = v;
      sum[0] = fmaf(v, v, sum[0]);
    }
  }
  row_sum(sum, a.lanes, 0);
  const float rs = rsqrtf(fmaf(sum[0], a.inv_width, a.eps));
#pragma unroll
  for (int n = 0; n < VPT; ++n) {
    const int col = (n * a.lanes + lane) * VEC;
    if (!valid || col >= a.width) continue;
    RowVec<T, VEC> out;
    if (a.h) {
      out.set(h[n]);
      out.store(static_cast<T*>(a.h) + at(a.hs, b, g, t) + col);
    }
    float y[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      y[i] = h[n][i] * rs * a.weight[g * a.weight_group + col + i];
      if (a.gate) y[i] *= gate_of<T>(z[n].get(i), a.sigmoid);
    }
    out.set(y);
    out.store(static_cast<T*>(a.y) + at(a.ys, b, g, t) + col);
  }
}

template <typename T, int VEC, int VPT>
__global__ void __launch_bounds__(1024) norm_backward_kernel(const NormArgs a) {
  pdl_trigger();
  const uint32_t slots = blockDim.x / a.lanes, slot = threadIdx.x / a.lanes, g = blockIdx.y;
  const int lane = threadIdx.x % a.lanes;
  pdl_wait();
  float dw[VPT][VEC], ds[VPT][VEC];
#pragma unroll
  for (int n = 0; n < VPT; ++n)
#pragma unroll
    for (int i = 0; i < VEC; ++i) dw[n][i] = ds[n][i] = 0.f;
  int turn = 0;
  for (uint32_t first = blockIdx.x * slots; first < a.rows; first += gridDim.x * slots, ++turn) {
    const uint32_t row = first + slot;
    const bool valid = row < a.rows;
    const uint32_t b = valid ? row / a.T : 0u, t = valid ? row - b * a.T : 0u;
    RowVec<T, VEC> dy[VPT], h[VPT], z[VPT], x[VPT], in[VPT];
#pragma unroll
    for (int n = 0; n < VPT; ++n) {
      const int col = (n * a.lanes + lane) * VEC;
      dy[n].clear();
      h[n].clear();
      z[n].clear();
      x[n].clear();
      in[n].clear();
      if (!valid || col >= a.width) continue;
      dy[n].load(static_cast<const T*>(a.dy) + at(a.dys, b, g, t) + col);
      h[n].load(static_cast<const T*>(a.h) + at(a.hs, b, g, t) + col);
      if (a.gate) z[n].load(static_cast<const T*>(a.gate) + at(a.gs, b, g, t) + col);
      if (a.dh_in) in[n].load(static_cast<const T*>(a.dh_in) + at(a.dhis, b, g, t) + col);
      if (a.ds) x[n].load(static_cast<const T*>(a.x) + at(a.xs, b, g, t) + col);
    }
    float sum[2] = {0.f, 0.f};
#pragma unroll
    for (int n = 0; n < VPT; ++n) {
      const int col = (n * a.lanes + lane) * VEC;
      if (col >= a.width) continue;
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const float v = h[n].get(i);
        float u = dy[n].get(i);
        if (a.gate) u *= gate_of<T>(z[n].get(i), a.sigmoid);
        sum[0] = fmaf(v, v, sum[0]);
        sum[1] = fmaf(u * a.weight[g * a.weight_group + col + i], v, sum[1]);
      }
    }
    row_sum(sum, a.lanes, turn);
    const float rs = rsqrtf(fmaf(sum[0], a.inv_width, a.eps));
    const float mean = sum[1] * rs * a.inv_width;      // mean(dn n)
#pragma unroll
    for (int n = 0; n < VPT; ++n) {
      const int col = (n * a.lanes + lane) * VEC;
      if (!valid || col >= a.width) continue;
      float dh[VEC], dg[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const float norm = h[n].get(i) * rs, w = a.weight[g * a.weight_group + col + i];
        float u = dy[n].get(i);
        if (a.gate) {
          float act, slope;
          gate_of<T>(z[n].get(i), a.sigmoid, &act, &slope);
          dg[i] = u * norm * w * slope;
          u *= act;
        }
        dw[n][i] = fmaf(u, norm, dw[n][i]);
        dh[i] = rs * fmaf(-norm, mean, u * w);
        if (a.dh_in) dh[i] += in[n].get(i);
        if (a.ds) ds[n][i] = fmaf(x[n].get(i), dh[i], ds[n][i]);
      }
      RowVec<T, VEC> out;
      out.set(dh);
      out.store(static_cast<T*>(a.dh) + at(a.dhs, b, g, t) + col);
      if (a.gate) {
        out.set(dg);
        out.store(static_cast<T*>(a.dgate) + at(a.dgs, b, g, t) + col);
      }
      if (a.dx) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) dh[i] *= a.scale[col + i];
        out.set(dh);
        out.store(static_cast<T*>(a.dx) + at(a.dxs, b, g, t) + col);
      }
    }
  }
  // this CTA's partial rows: the slots of a column in order
  __shared__ float sums[NORM_THREADS * VEC * VPT];
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    float* part = which ? a.ds : a.dw;
    if (!part) continue;
    part += ((int64_t)g * gridDim.x + blockIdx.x) * a.width;
    if (slots == 1) {
#pragma unroll
      for (int n = 0; n < VPT; ++n) {
        const int col = (n * a.lanes + lane) * VEC;
        if (col >= a.width) continue;
#pragma unroll
        for (int i = 0; i < VEC; ++i) part[col + i] = which ? ds[n][i] : dw[n][i];
      }
      continue;
    }
    const int padded = a.lanes * VPT * VEC;
    __syncthreads();
#pragma unroll
    for (int n = 0; n < VPT; ++n)
#pragma unroll
      for (int i = 0; i < VEC; ++i) sums[slot * padded + (n * a.lanes + lane) * VEC + i] = which ? ds[n][i] : dw[n][i];
    __syncthreads();
    for (int col = threadIdx.x; col < a.width; col += blockDim.x) {
      float v = 0.f;
      for (uint32_t k = 0; k < slots; ++k) v += sums[k * padded + col];
      part[col] = v;
    }
  }
}

// Sums of the partial rows: blockIdx.y = 0 dw (group by group where it has a row for each), 1 dscale.
constexpr int SUM_COLS = 32, SUM_WARPS = 32;
__global__ void __launch_bounds__(SUM_COLS* SUM_WARPS) norm_sum_kernel(const float* dw_parts, const float* ds_parts, float* dw, float* ds,
                                                                       int parts, int groups, int width, int grouped) {
  __shared__ float sums[SUM_WARPS][SUM_COLS];
  pdl_trigger();
  pdl_wait();
  const bool scale = blockIdx.y == 1;
  const float* from = scale ? ds_parts : dw_parts;
  float* to = scale ? ds : dw;
  const int g = blockIdx.z;
  if (!to || (g > 0 && (scale || !grouped))) return;
  int64_t rows = parts;
  if (!scale && grouped) {
    from += (int64_t)g * parts * width;
    to += (int64_t)g * width;
  } else {
    rows *= groups;
  }
  const int col = blockIdx.x * SUM_COLS + (threadIdx.x & 31), warp = threadIdx.x >> 5;
  float v = 0.f;
  if (col < width)
    for (int64_t r = warp; r < rows; r += SUM_WARPS) v += from[r * width + col];
  sums[warp][threadIdx.x & 31] = v;
  __syncthreads();
  if (warp == 0 && col < width) {
    v = 0.f;
#pragma unroll
    for (int w = 0; w < SUM_WARPS; ++w) v += sums[w][threadIdx.x & 31];
    to[col] = v;
  }
}

int pow2_at_least(int n) {
  int p = 1;
  while (p < n) p *= 2;
  return p;
}

// CTAs along the rows of a backward pass.
uint32_t backward_ctas(const NormArgs& a, int slots, int groups) {
  const uint32_t want = (uint32_t)(NORM_PARTIALS / groups > 0 ? NORM_PARTIALS / groups : 1);
  const uint32_t most = (uint32_t)(((uint64_t)a.rows + slots - 1) / slots);
  return most < want ? most : want;
}

template <typename T, int VEC, int VPT>
cudaError_t launch_forward(NormArgs& a, int groups, cudaStream_t st) {
  const int pieces = (a.width + VEC - 1) / VEC;
  a.lanes = pow2_at_least((pieces + VPT - 1) / VPT);
  const int threads = a.lanes <= 32 ? NORM_THREADS : a.lanes, slots = threads / a.lanes;
  const dim3 grid((unsigned)(((uint64_t)a.rows + slots - 1) / slots), (unsigned)groups);
  return smat_launch_pdl(norm_forward_kernel<T, VEC, VPT>, grid, threads, 0, st, a);
}

template <typename T, int VEC, int VPT>
cudaError_t launch_backward(NormArgs& a, int groups, float* dw, float* ds, cudaStream_t st) {
  const int pieces = (a.width + VEC - 1) / VEC;
  a.lanes = pow2_at_least((pieces + VPT - 1) / VPT);
  const int threads = a.lanes <= 32 ? NORM_THREADS : a.lanes, slots = threads / a.lanes;
  const uint32_t ctas = backward_ctas(a, slots, groups);
  cudaError_t err = smat_launch_pdl(norm_backward_kernel<T, VEC, VPT>, dim3(ctas, (unsigned)groups), threads, 0, st, a);
  if (err != cudaSuccess || (!dw && !ds)) return err;
  const int grouped = a.weight_group ? 1 : 0;
  const dim3 grid((unsigned)((a.width + SUM_COLS - 1) / SUM_COLS), ds ? 2u : 1u, (unsigned)(grouped ? groups : 1));
  return smat_launch_pdl(norm_sum_kernel, grid, SUM_COLS * SUM_WARPS, 0, st, static_cast<const float*>(a.dw),
                         static_cast<const float*>(a.ds), dw, ds, (int)ctas, groups, a.width, grouped);
}

// Pieces a lane holds: the fewest that keep a row within a CTA, and in the forward pass up to four where that keeps it within a warp.
template <typename T, int VEC>
cudaError_t forward(NormArgs& a, int groups, cudaStream_t st) {
  const int pieces = (a.width + VEC - 1) / VEC;
  if constexpr (VEC == 1) {
    return pieces <= 4096 ? launch_forward<T, 1, 4>(a, groups, st) : launch_forward<T, 1, 16>(a, groups, st);
  } else {
    if (pieces <= 32) return launch_forward<T, VEC, 1>(a, groups, st);
    return pieces <= 1024 ? launch_forward<T, VEC, 2>(a, groups, st) : launch_forward<T, VEC, 4>(a, groups, st);
  }
}
template <typename T, int VEC>
cudaError_t backward(NormArgs& a, int groups, float* dw, float* ds, cudaStream_t st) {
  const int pieces = (a.width + VEC - 1) / VEC;
  if constexpr (VEC == 1) {
    return pieces <= 4096 ? launch_backward<T, 1, 4>(a, groups, dw, ds, st) : launch_backward<T, 1, 16>(a, groups, dw, ds, st);
  } else {
    return pieces <= 512 ? launch_backward<T, VEC, 1>(a, groups, dw, ds, st) : launch_backward<T, VEC, 4>(a, groups, dw, ds, st);
  }
}

smat_status check_problem(const smat_norm_problem* p) {
  if (!p || !p->weight) return SMAT_ERR_NULL;
  if (p->dtype != SMAT_F32 && p->dtype != SMAT_BF16) return SMAT_ERR_DTYPE;
  if (p->activation != SMAT_ACT_SILU && p->activation != SMAT_ACT_SIGMOID) return SMAT_ERR_UNSUPPORTED;
  if (p->batch < 1 || p->T < 1 || p->groups < 1 || p->groups > 65535 || p->width < 1 || p->width > NORM_MAX_WIDTH)
    return SMAT_ERR_SHAPE;
  if (p->T > INT32_MAX || p->T * p->batch > INT32_MAX) return SMAT_ERR_SHAPE;
  if (p->weight_group != 0 && p->weight_group != p->width) return SMAT_ERR_SHAPE;
  if (!(p->eps >= 0.f)) return SMAT_ERR_SHAPE;
  if ((reinterpret_cast<uintptr_t>(p->weight) | reinterpret_cast<uintptr_t>(p->scale)) & 3) return SMAT_ERR_ALIGN;
  return SMAT_OK;
}

struct Operand {
  const smat_rows* rows;
  bool output;
};
template <int N>
smat_status check_rows(const smat_norm_problem* p, const Operand (&ops)[N], bool* wide) {
  *wide = p->width % (p->dtype == SMAT_BF16 ? 8 : 4) == 0;
  for (const Operand& o : ops) {
    if (!o.rows) continue;
    if (!o.rows->data) return SMAT_ERR_NULL;
    if (!rows_ok(o.rows, p->batch, p->groups, p->T, p->width, o.output)) return SMAT_ERR_SHAPE;
  }
  for (const Operand& o : ops) {
    if (rows_misaligned(o.rows, p->dtype)) return SMAT_ERR_ALIGN;
    *wide = *wide && rows_in_16(o.rows, p->dtype, p->batch, p->groups, p->T);
  }
  return SMAT_OK;
}

NormArgs arguments(const smat_norm_problem* p) {
  NormArgs a{};
  a.weight = p->weight;
  a.weight_group = p->weight_group;
  a.scale = p->scale;
  a.rows = (uint32_t)(p->T * p->batch);
  a.T = (uint32_t)p->T;
  a.width = p->width;
  a.eps = p->eps;
  a.inv_width = 1.f / (float)p->width;
  a.sigmoid = p->activation == SMAT_ACT_SIGMOID;
  return a;
}
const void* in(const smat_rows* r) { return r ? r->data : nullptr; }
void* out(const smat_rows* r) { return r ? r->data : nullptr; }

}  // namespace

extern "C" {

smat_status smat_norm_forward(const smat_norm_problem* p, const smat_rows* x, const smat_rows* residual, const smat_rows* gate,
                              const smat_rows* y, const smat_rows* h, void* cuda_stream) {
  if (!x || !y) return SMAT_ERR_NULL;
  smat_status s = check_problem(p);
  if (s != SMAT_OK) return s;
  bool wide;
  s = check_rows(p, {{x, false}, {residual, false}, {gate, false}, {y, true}, {h, true}}, &wide);
  if (s != SMAT_OK) return s;
  if (!rows_device_ok()) return SMAT_ERR_ARCH;
  NormArgs a = arguments(p);
  a.x = x->data; a.xs = row_stride(x);
  a.residual = in(residual); a.rs = row_stride(residual);
  a.gate = in(gate); a.gs = row_stride(gate);
  a.y = y->data; a.ys = row_stride(y);
  a.h = out(h); a.hs = row_stride(h);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const cudaError_t err = p->dtype == SMAT_BF16
                              ? (wide ? forward<__nv_bfloat16, 8>(a, p->groups, st) : forward<__nv_bfloat16, 1>(a, p->groups, st))
                              : (wide ? forward<float, 4>(a, p->groups, st) : forward<float, 1>(a, p->groups, st));
  return err == cudaSuccess ? SMAT_OK : SMAT_ERR_LAUNCH;
}

size_t smat_norm_workspace_bytes(const smat_norm_problem* p) {
  if (check_problem(p) != SMAT_OK) return 0;
  const size_t ctas = NORM_PARTIALS > p->groups ? NORM_PARTIALS : p->groups;
  return ctas * (size_t)p->width * sizeof(float) * (p->scale ? 2 : 1);
}

smat_status smat_norm_backward(const smat_norm_problem* p, const smat_rows* dy, const smat_rows* h, const smat_rows* gate,
                               const smat_rows* x, const smat_rows* dh_in, const smat_rows* dh, const smat_rows* dx,
                               const smat_rows* dgate, float* dweight, float* dscale, void* workspace, size_t workspace_bytes,
                               void* cuda_stream) {
  if (!dy || !h || !dh) return SMAT_ERR_NULL;
  smat_status s = check_problem(p);
  if (s != SMAT_OK) return s;
  // a gate's gradient comes with the gate, that of the scale with the rows that it multiplies
  if ((gate != nullptr) != (dgate != nullptr) || (dscale && !x)) return SMAT_ERR_NULL;
  if ((dx || dscale) && !p->scale) return SMAT_ERR_NULL;
  bool wide;
  s = check_rows(p, {{dy, false}, {h, false}, {gate, false}, {dscale ? x : nullptr, false}, {dh_in, false}, {dh, true}, {dx, true}, {dgate, true}}, &wide);
  if (s != SMAT_OK) return s;
  if ((reinterpret_cast<uintptr_t>(dweight) | reinterpret_cast<uintptr_t>(dscale)) & 3) return SMAT_ERR_ALIGN;
  if (dweight || dscale) {
    if (!workspace) return SMAT_ERR_NULL;
    if (workspace_bytes < smat_norm_workspace_bytes(p)) return SMAT_ERR_WORKSPACE;
    if (reinterpret_cast<uintptr_t>(workspace) & 255) return SMAT_ERR_ALIGN;
  }
  if (!rows_device_ok()) return SMAT_ERR_ARCH;
  NormArgs a = arguments(p);
  a.dy = dy->data; a.dys = row_stride(dy);
  a.h = out(h); a.hs = row_stride(h);
  a.gate = in(gate); a.gs = row_stride(gate);
  if (dscale) { a.x = x->data; a.xs = row_stride(x); }
  a.dh_in = in(dh_in); a.dhis = row_stride(dh_in);
  a.dh = dh->data; a.dhs = row_stride(dh);
  a.dx = out(dx); a.dxs = row_stride(dx);
  a.dgate = out(dgate); a.dgs = row_stride(dgate);
  const size_t ctas = NORM_PARTIALS > p->groups ? NORM_PARTIALS : p->groups;
  if (dweight) a.dw = static_cast<float*>(workspace);
  if (dscale) a.ds = static_cast<float*>(workspace) + ctas * p->width;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const int g = p->groups;
  const cudaError_t err = p->dtype == SMAT_BF16 ? (wide ? backward<__nv_bfloat16, 8>(a, g, dweight, dscale, st)
                                                        : backward<__nv_bfloat16, 1>(a, g, dweight, dscale, st))
                                                : (wide ? backward<float, 4>(a, g, dweight, dscale, st)
                                                        : backward<float, 1>(a, g, dweight, dscale, st));
  return err == cudaSuccess ? SMAT_OK : SMAT_ERR_LAUNCH;
}

}  // extern "C"
