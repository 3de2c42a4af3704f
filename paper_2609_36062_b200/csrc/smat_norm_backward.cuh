// Gradients of the root-mean-square norm: with r = 1 / sqrt(mean(h²) + eps), n = h r and u = dy act(gate),
//     dn = u w,   dh = r (dn - n mean(dn n)) + dh_in,   dx = scale dh,   dgate = dy n w act'(gate),
//     dw = Σ_rows u n,   dscale = Σ_rows x dh.
// mean(dn n) = r mean(dn h): both sums that a row needs are over what it reads, so it is read once (see smat_norm.cuh for the
// layout).  A CTA keeps the sums of dw and dscale over its rows in registers, one column set a thread, and leaves one partial
// row of each; a second kernel adds these in a fixed order.
#pragma once
#include "smat_norm.cuh"

namespace {

// Operands a kernel reads: dy, h, dh_in, and the branch's rows or the gate or both.
__host__ __device__ constexpr int norm_operands(int mode) { return mode == NORM_ROWS ? 3 : mode == NORM_ANY ? 5 : 4; }

template <typename T, int VEC, int E, int THREADS, int MODE>
__global__ void __launch_bounds__(THREADS, THREADS == 256 ? 2 : 1) norm_backward_kernel(const NormArgs a) {
  constexpr int VPT = E / VEC;
  constexpr bool ANY = MODE == NORM_ANY, SCALE = ANY || MODE == NORM_STREAM, GATE = ANY || MODE == NORM_SILU || MODE == NORM_SIGMOID;
  __shared__ __align__(8) float exchange[2][32][2];
  const bool scaled = MODE == NORM_STREAM || (ANY && a.ds), branch = SCALE && a.dx.data, more = a.dh_in.data != nullptr;
  const bool gated = MODE == NORM_SILU || MODE == NORM_SIGMOID || (ANY && a.gate.data);
  const bool sigmoid = MODE == NORM_SIGMOID || (ANY && a.sigmoid);
  const uint32_t g = blockIdx.x % a.groups;
  const int lane = threadIdx.x % a.lanes, column = lane * VEC, apart = a.lanes * VEC;
  NormWalk at(a);
  const uint32_t slots = at.slots, slot = at.slot;
  pdl_wait();
  constexpr int N = norm_operands(MODE) * VPT, DEPTH = norm_depth(N, 16, THREADS);
  constexpr bool RING = VEC * sizeof(T) == 16 && norm_rings(N, THREADS);
  constexpr int X = 3 * VPT, Z = (ANY ? 4 : 3) * VPT;      // places of the branch's rows and of the gate
  extern __shared__ uint4 rows_shared[];
  NormRing<N, DEPTH> ring(rows_shared);
  struct Row {
    RowVec<T, VEC> dy[VPT], h[VPT], z[GATE ? VPT : 1], x[SCALE ? VPT : 1], in[VPT];
  } next;
  const T *dyp = at.seat<T>(a.dy, g, column), *hp = at.seat<T>(a.h, g, column), *zp = at.seat<T>(a.gate, g, column);
  const T *xp = at.seat<T>(a.x, g, column), *ip = at.seat<T>(a.dh_in, g, column);
  T *dhp = at.seat<T>(a.dh, g, column), *dxp = at.seat<T>(a.dx, g, column), *dgp = at.seat<T>(a.dgate, g, column);
  // asks for the rows of the walk's place, and moves on
  const auto load = [&]() {
    const bool in = at.in(a);
#pragma unroll
    for (int n = 0; n < VPT; ++n) {
      const bool mine = in && column + n * apart < a.width;
      if constexpr (RING) {
        ring.fetch(n, dyp + n * apart, mine);
        ring.fetch(VPT + n, hp + n * apart, mine);
        if (more) ring.fetch(2 * VPT + n, ip + n * apart, mine);
        if constexpr (SCALE) if (scaled) ring.fetch(X + n, xp + n * apart, mine);
        if constexpr (GATE) if (gated) ring.fetch(Z + n, zp + n * apart, mine);
      } else {
        next.dy[n].clear();
        next.h[n].clear();
        if constexpr (GATE) next.z[n].clear();
        if constexpr (SCALE) next.x[n].clear();
        next.in[n].clear();
        if (!mine) continue;
        next.dy[n].load(dyp + n * apart);
        next.h[n].load(hp + n * apart);
        if constexpr (GATE) if (gated) next.z[n].load(zp + n * apart);
        if constexpr (SCALE) if (scaled) next.x[n].load(xp + n * apart);
        if (more) next.in[n].load(ip + n * apart);
      }
    }
    if constexpr (RING) {
      ring.fetched();
      ring.next();
    }
    at.next(a);
    norm_move(dyp, a.dy, at.wrapped);
    norm_move(hp, a.h, at.wrapped);
    if (gated) norm_move(zp, a.gate, at.wrapped);
    if (scaled) norm_move(xp, a.x, at.wrapped);
    if (more) norm_move(ip, a.dh_in, at.wrapped);
  };
  NormWalk to(a);      // the rows that are worked on
  if constexpr (RING) {
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) load();
  } else {
    load();
  }
  float2 w[E / 2], dw[E / 2], ds[SCALE ? E / 2 : 1], factor[SCALE ? E / 2 : 1];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int col = column + e / VEC * apart + e % VEC;
    const float v = col < a.width ? a.weight[g * a.weight_group + col] : 0.f;
    if (e % 2) w[e / 2].y = v;
    else w[e / 2].x = v;
    dw[e / 2] = norm_both(0.f);
    if constexpr (SCALE) {
      ds[e / 2] = norm_both(0.f);
      const float f = branch && col < a.width ? a.scale[col] : 0.f;
      if (e % 2) factor[e / 2].y = f;
      else factor[e / 2].x = f;
    }
  }
  for (int turn = 0;; ++turn) {
    Row in;
    const bool here = to.in(a);
    if constexpr (RING) {
      ring.wait();
#pragma unroll
      for (int n = 0; n < VPT; ++n) {
        ring.read(n, in.dy[n]);
        ring.read(VPT + n, in.h[n]);
        if (more) ring.read(2 * VPT + n, in.in[n]);
        if constexpr (SCALE) if (scaled) ring.read(X + n, in.x[n]);
        if constexpr (GATE) if (gated) ring.read(Z + n, in.z[n]);
      }
    } else {
      in = next;
      load();
    }
    // u = dy act, and what dgate is but for n: dy w act'
    float2 u[E / 2], slope[GATE ? E / 2 : 1], squares = norm_both(0.f), products = norm_both(0.f);
#pragma unroll
    for (int j = 0; j < E / 2; ++j) {
      const float2 v = norm_pair<VEC, E>(in.h, j);
      u[j] = norm_pair<VEC, E>(in.dy, j);
      if constexpr (GATE) {
        if (gated) {
          const float2 z = norm_pair<VEC, E>(in.z, j), e = norm_sigmoid<T>(z), act = sigmoid ? e : __fmul2_rn(z, e);
          const float2 rest = __ffma2_rn(e, norm_both(-1.f), norm_both(1.f));
          slope[j] = __fmul2_rn(sigmoid ? __fmul2_rn(e, rest) : __ffma2_rn(act, rest, e), __fmul2_rn(u[j], w[j]));
          u[j] = __fmul2_rn(u[j], act);
        }
      }
      squares = __ffma2_rn(v, v, squares);
      products = __ffma2_rn(__fmul2_rn(u[j], w[j]), v, products);
    }
    if constexpr (RING) load();      // (into the places that have just been read)
    float sum[2] = {squares.x + squares.y, products.x + products.y};
    norm_row_sum(sum, a.lanes, turn, exchange);
    const float r = here ? rsqrtf(fmaf(sum[0], a.inv_width, a.eps)) : 0.f;      // (a slot without a row adds nothing, at eps = 0 either)
    const float2 rs = norm_both(r), mean = norm_both(-r * (sum[1] * r * a.inv_width));      // -r mean(dn n)
    float2 dh[E / 2];
#pragma unroll
    for (int j = 0; j < E / 2; ++j) {
      const float2 n = __fmul2_rn(norm_pair<VEC, E>(in.h, j), rs);
      if constexpr (GATE) slope[j] = __fmul2_rn(slope[j], n);
      dw[j] = __ffma2_rn(u[j], n, dw[j]);
      dh[j] = __ffma2_rn(__fmul2_rn(u[j], w[j]), rs, __fmul2_rn(n, mean));
      if (more) dh[j] = __fadd2_rn(dh[j], norm_pair<VEC, E>(in.in, j));
      if constexpr (SCALE) if (scaled) ds[j] = __ffma2_rn(norm_pair<VEC, E>(in.x, j), dh[j], ds[j]);
    }
#pragma unroll
    for (int n = 0; n < VPT; ++n) {
      if (!here || column + n * apart >= a.width) continue;
      const auto at_pair = [&](const float2* v, int i) { return (n * VEC + i) % 2 ? v[(n * VEC + i) / 2].y : v[(n * VEC + i) / 2].x; };
      float v[VEC];
      RowVec<T, VEC> out;
#pragma unroll
      for (int i = 0; i < VEC; ++i) v[i] = at_pair(dh, i);
      out.set(v);
      out.store(dhp + n * apart);
      if constexpr (GATE) {
        if (gated) {
#pragma unroll
          for (int i = 0; i < VEC; ++i) v[i] = at_pair(slope, i);
          out.set(v);
          out.store(dgp + n * apart);
        }
      }
      if constexpr (SCALE) {
        if (branch) {
#pragma unroll
          for (int i = 0; i < VEC; ++i) v[i] = at_pair(dh, i) * at_pair(factor, i);
          out.set(v);
          out.store(dxp + n * apart);
        }
      }
    }
    to.next(a);
    if (!to.more(a)) break;
    norm_move(dhp, a.dh, to.wrapped);
    if (branch) norm_move(dxp, a.dx, to.wrapped);
    if (gated) norm_move(dgp, a.dgate, to.wrapped);
  }
  pdl_trigger();      // not before: CTAs of the next launch would take places that these are laid out for
  if constexpr (RING) ring.landed();
  // this CTA's partial rows: the slots of a column in order
  float* sums = reinterpret_cast<float*>(rows_shared);      // (in the place of the rows, which have been read)
#pragma unroll
  for (int which = 0; which < (SCALE ? 2 : 1); ++which) {
    float* part = which ? a.ds : a.dw;
    if (!part) continue;
    const float2* sum = which ? ds : dw;
    const auto sum_of = [&](int e) { return e % 2 ? sum[e / 2].y : sum[e / 2].x; };
    part += ((int64_t)g * a.ctas + blockIdx.x / a.groups) * a.width;
    if (slots == 1) {
#pragma unroll
      for (int n = 0; n < VPT; ++n) {
        const int col = (n * a.lanes + lane) * VEC;
        if (col >= a.width) continue;
#pragma unroll
        for (int i = 0; i < VEC; ++i) part[col + i] = sum_of(n * VEC + i);
      }
      continue;
    }
    if constexpr (THREADS == 256) {
      const int padded = a.lanes * E;
      __syncthreads();
#pragma unroll
      for (int n = 0; n < VPT; ++n)
#pragma unroll
        for (int i = 0; i < VEC; ++i) sums[slot * padded + (n * a.lanes + lane) * VEC + i] = sum_of(n * VEC + i);
      __syncthreads();
      for (int col = threadIdx.x; col < a.width; col += blockDim.x) {
        float v = 0.f;
        for (uint32_t k = 0; k < slots; ++k) v += sums[k * padded + col];
        part[col] = v;
      }
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
  if (col < width) {
    // (eight rows on their way at a time: a chain of single loads took longer than the rows of 512 columns had)
    constexpr int AHEAD = 8;
    for (int64_t r = warp; r < rows; r += SUM_WARPS * AHEAD) {
      float part[AHEAD];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) part[i] = r + i * SUM_WARPS < rows ? from[(r + i * SUM_WARPS) * width + col] : 0.f;
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) v += part[i];
    }
  }
  sums[warp][threadIdx.x & 31] = v;
  __syncthreads();
  if (warp == 0 && col < width) {
    v = 0.f;
#pragma unroll
    for (int w = 0; w < SUM_WARPS; ++w) v += sums[w][threadIdx.x & 31];
    to[col] = v;
  }
}

template <typename T, int VEC, int E, int THREADS, int MODE>
cudaError_t launch(NormArgs& a, const NormShape& s, float* dw, float* ds, cudaStream_t st) {
  a.lanes = s.lanes;
  const uint32_t threads = s.lanes <= 32 ? 256 : s.lanes, slots = threads / s.lanes;
  norm_walk(&a, slots, (uint32_t)(NORM_SMS * norm_ctas_an_sm(512, threads)) / a.groups);
  cudaError_t err = norm_launch(norm_backward_kernel<T, VEC, E, THREADS, MODE>, VEC * sizeof(T) == 16 ? norm_operands(MODE) * E / VEC : 0, 16, slots > 1 ? 256 * E * sizeof(float) : 0,
                                THREADS, norm_ctas_an_sm(512, threads), dim3(a.ctas * a.groups), threads, st, a);
  if (err != cudaSuccess || (!dw && !ds)) return err;
  const int grouped = a.weight_group ? 1 : 0;
  const dim3 grid((unsigned)((a.width + SUM_COLS - 1) / SUM_COLS), ds ? 2u : 1u, grouped ? a.groups : 1u);
  return smat_launch_pdl(norm_sum_kernel, grid, SUM_COLS * SUM_WARPS, 0, st, static_cast<const float*>(a.dw),
                         static_cast<const float*>(a.ds), dw, ds, (int)a.ctas, (int)a.groups, a.width, grouped);
}

template <typename T, int VEC, int MODE>
cudaError_t shaped(NormArgs& a, float* dw, float* ds, cudaStream_t st) {
  constexpr bool WHOLE = VEC * sizeof(T) == 16, ROOMY = WHOLE && MODE == NORM_ROWS;
  const NormShape s = norm_shape(a.width, ROOMY);
  constexpr int WIDE = WHOLE ? MODE : NORM_ANY;      // (rows of single elements or pairs: one kernel for all long ones)
  if (s.columns == 16) {
    if constexpr (ROOMY) {
      if (s.threads == 256) return launch<T, VEC, 16, 256, MODE>(a, s, dw, ds, st);
      if (s.threads == 512) return launch<T, VEC, 16, 512, MODE>(a, s, dw, ds, st);
    }
    return launch<T, VEC, 16, 1024, WIDE>(a, s, dw, ds, st);
  }
  if (s.threads == 256) return launch<T, VEC, 8, 256, MODE>(a, s, dw, ds, st);
  if constexpr (!ROOMY) {
    if (s.threads == 512) return launch<T, VEC, 8, 512, MODE>(a, s, dw, ds, st);
    return s.threads == 768 ? launch<T, VEC, 8, 768, WIDE>(a, s, dw, ds, st) : launch<T, VEC, 8, 1024, WIDE>(a, s, dw, ds, st);
  }
  return cudaErrorInvalidValue;
}

template <typename T, int VEC>
cudaError_t moded(NormArgs& a, float* dw, float* ds, cudaStream_t st) {
  if (!a.gate.data) return ds ? shaped<T, VEC, NORM_STREAM>(a, dw, ds, st) : a.dx.data ? shaped<T, VEC, NORM_ANY>(a, dw, ds, st) : shaped<T, VEC, NORM_ROWS>(a, dw, ds, st);
  if (!ds && !a.dx.data) return a.sigmoid ? shaped<T, VEC, NORM_SIGMOID>(a, dw, ds, st) : shaped<T, VEC, NORM_SILU>(a, dw, ds, st);
  return shaped<T, VEC, NORM_ANY>(a, dw, ds, st);
}

}  // namespace
