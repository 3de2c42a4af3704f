// Root-mean-square norm of rows, before a block or behind it:
//     h = residual + scale x,   r = 1 / sqrt(mean(h²) + eps),   y = h r w act(gate).
// A stream over rows with one sum in the way; see smat_norm.cuh for the layout.
#include "smat_norm.cuh"

namespace {

// Threads an SM holds: what the registers allow.
__host__ __device__ constexpr int norm_resident(int mode, int columns) { return mode == NORM_ANY || columns > 8 ? 768 : 1024; }
// Operands a kernel reads: the rows, the residual, the gate.
__host__ __device__ constexpr int norm_operands(int mode) { return mode == NORM_ROWS ? 1 : mode == NORM_ANY ? 3 : 2; }

template <typename T, int VEC, int E, int THREADS, int MODE>
__global__ void __launch_bounds__(THREADS, norm_resident(MODE, E) >= THREADS ? norm_resident(MODE, E) / THREADS : 1) norm_forward_kernel(const NormArgs a) {
  constexpr int VPT = E / VEC;
  constexpr bool ANY = MODE == NORM_ANY;
  __shared__ float exchange[2][32][1];
  const bool residual = MODE == NORM_STREAM || (ANY && a.residual.data), keeps = (ANY || MODE == NORM_STREAM) && a.h.data;
  const bool scaled = MODE == NORM_STREAM || ANY;
  const bool gated = MODE == NORM_SILU || MODE == NORM_SIGMOID || (ANY && a.gate.data);
  const bool sigmoid = MODE == NORM_SIGMOID || (ANY && a.sigmoid);
  const uint32_t g = blockIdx.x % a.groups;
  const int lane = threadIdx.x % a.lanes, column = lane * VEC, apart = a.lanes * VEC;
  NormWalk at(a);
  pdl_wait();
  constexpr int N = norm_operands(MODE) * VPT, DEPTH = norm_depth(N, 8, THREADS);
  constexpr bool RING = VEC * sizeof(T) == 16 && norm_rings(N, THREADS);
  extern __shared__ uint4 rows_shared[];
  NormRing<N, DEPTH> ring(rows_shared);
  RowVec<T, VEC> x[VPT], r[VPT], z[VPT];
  const T *xp = at.seat<T>(a.x, g, column), *rp = at.seat<T>(a.residual, g, column), *zp = at.seat<T>(a.gate, g, column);
  T *yp = at.seat<T>(a.y, g, column), *hp = at.seat<T>(a.h, g, column);
  // asks for the rows of the walk's place, and moves on
  const auto load = [&]() {
    const bool in = at.in(a);
#pragma unroll
    for (int n = 0; n < VPT; ++n) {
      const bool mine = in && column + n * apart < a.width;
      if constexpr (RING) {
        ring.fetch(n, xp + n * apart, mine);
        if (residual) ring.fetch(VPT + n, rp + n * apart, mine);
        if (gated) ring.fetch((ANY ? 2 : 1) * VPT + n, zp + n * apart, mine);
      } else {
        x[n].clear();
        if (residual) r[n].clear();
        if (gated) z[n].clear();
        if (!mine) continue;
        x[n].load(xp + n * apart);
        if (residual) r[n].load(rp + n * apart);
        if (gated) z[n].load(zp + n * apart);
      }
    }
    if constexpr (RING) {
      ring.fetched();
      ring.next();
    }
    at.next(a);
    norm_move(xp, a.x, at.wrapped);
    if (residual) norm_move(rp, a.residual, at.wrapped);
    if (gated) norm_move(zp, a.gate, at.wrapped);
  };
  NormWalk to(a);      // the rows that are worked on
  if constexpr (RING) {
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) load();
  } else {
    load();
  }
  float2 w[E / 2], s[E / 2];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int col = column + e / VEC * apart + e % VEC;
    const float wv = col < a.width ? a.weight[g * a.weight_group + col] : 0.f, sv = scaled && a.scale && col < a.width ? a.scale[col] : 1.f;
    if (e % 2) { w[e / 2].y = wv; s[e / 2].y = sv; }
    else { w[e / 2].x = wv; s[e / 2].x = sv; }
  }
  // (all slots of a CTA go through the same tiles, so that they meet at its barriers)
  for (int turn = 0;; ++turn) {
    float2 h[E / 2], y[E / 2], squares = norm_both(0.f);
    if constexpr (RING) {
      ring.wait();
#pragma unroll
      for (int n = 0; n < VPT; ++n) {
        ring.read(n, x[n]);
        if (residual) ring.read(VPT + n, r[n]);
        if (gated) ring.read((ANY ? 2 : 1) * VPT + n, z[n]);
      }
    }
#pragma unroll
    for (int j = 0; j < E / 2; ++j) {
      h[j] = norm_pair<VEC, E>(x, j);
      if (residual) h[j] = __ffma2_rn(h[j], s[j], norm_pair<VEC, E>(r, j));
      else if (scaled) h[j] = __fmul2_rn(h[j], s[j]);
      squares = __ffma2_rn(h[j], h[j], squares);
      y[j] = __fmul2_rn(h[j], w[j]);
      if (gated) {
        const float2 q = norm_pair<VEC, E>(z, j);
        y[j] = __fmul2_rn(y[j], norm_sigmoid<T>(q));
        if (!sigmoid) y[j] = __fmul2_rn(y[j], q);
      }
    }
    const bool here = to.in(a);
    load();
    float sum[1] = {squares.x + squares.y};
    norm_row_sum(sum, a.lanes, turn, exchange);
    const float2 rs = norm_both(rsqrtf(fmaf(sum[0], a.inv_width, a.eps)));
#pragma unroll
    for (int n = 0; n < VPT; ++n) {
      if (!here || column + n * apart >= a.width) continue;
      float v[VEC];
      RowVec<T, VEC> out;
      if (keeps) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = (n * VEC + i) % 2 ? h[(n * VEC + i) / 2].y : h[(n * VEC + i) / 2].x;
        out.set(v);
        out.store(hp + n * apart);
      }
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const float2 q = __fmul2_rn(y[(n * VEC + i) / 2], rs);
        v[i] = (n * VEC + i) % 2 ? q.y : q.x;
      }
      out.set(v);
      out.store(yp + n * apart);
    }
    to.next(a);
    if (!to.more(a)) break;
    norm_move(yp, a.y, to.wrapped);
    if (keeps) norm_move(hp, a.h, to.wrapped);
  }
  pdl_trigger();      // not before: CTAs of the next launch would take places that these are laid out for
  if constexpr (RING) ring.landed();
}

template <typename T, int VEC, int E, int THREADS, int MODE>
cudaError_t launch(NormArgs& a, const NormShape& s, cudaStream_t st) {
  a.lanes = s.lanes;
  const uint32_t threads = s.lanes <= 32 ? 256 : s.lanes, slots = threads / s.lanes;
  // as many CTAs as run at once, a group's share of them each, but none without a row
  norm_walk(&a, slots, (uint32_t)(NORM_SMS * norm_ctas_an_sm(norm_resident(MODE, E), threads)) / a.groups);
  return norm_launch(norm_forward_kernel<T, VEC, E, THREADS, MODE>, VEC * sizeof(T) == 16 ? norm_operands(MODE) * E / VEC : 0, 8, 0, THREADS,
                     norm_ctas_an_sm(norm_resident(MODE, E), threads),
                     dim3(a.ctas * a.groups), threads, st, a);
}

template <typename T, int VEC, int MODE>
cudaError_t shaped(NormArgs& a, cudaStream_t st) {
  constexpr bool WHOLE = VEC * sizeof(T) == 16, ROOMY = WHOLE && (MODE == NORM_ROWS || MODE == NORM_STREAM);
  const NormShape s = norm_shape(a.width, ROOMY);
  constexpr int WIDE = WHOLE ? MODE : NORM_ANY;      // (rows of single elements or pairs: one kernel for all long ones)
  if (s.columns == 16) {
    if constexpr (ROOMY) {
      if (s.threads == 256) return launch<T, VEC, 16, 256, MODE>(a, s, st);
      if (s.threads == 512) return launch<T, VEC, 16, 512, MODE>(a, s, st);
    }
    return launch<T, VEC, 16, 1024, WIDE>(a, s, st);
  }
  if (s.threads == 256) return launch<T, VEC, 8, 256, MODE>(a, s, st);
  if constexpr (!ROOMY) {
    if (s.threads == 512) return launch<T, VEC, 8, 512, MODE>(a, s, st);
    return s.threads == 768 ? launch<T, VEC, 8, 768, WIDE>(a, s, st) : launch<T, VEC, 8, 1024, WIDE>(a, s, st);
  }
  return cudaErrorInvalidValue;
}

template <typename T, int VEC>
cudaError_t moded(NormArgs& a, cudaStream_t st) {
  if (!a.gate.data && a.residual.data) return shaped<T, VEC, NORM_STREAM>(a, st);
  if (!a.residual.data && !a.scale && !a.h.data) {
    if (!a.gate.data) return shaped<T, VEC, NORM_ROWS>(a, st);
    return a.sigmoid ? shaped<T, VEC, NORM_SIGMOID>(a, st) : shaped<T, VEC, NORM_SILU>(a, st);
  }
  return shaped<T, VEC, NORM_ANY>(a, st);
}

}  // namespace

// vec: elements that every operand's rows can be moved by.
cudaError_t smat_launch_norm_forward(NormArgs& a, int bf16, int vec, cudaStream_t st) {
  if (bf16) return vec == 8 ? moded<__nv_bfloat16, 8>(a, st) : vec == 2 ? moded<__nv_bfloat16, 2>(a, st) : moded<__nv_bfloat16, 1>(a, st);
  return vec == 4 ? moded<float, 4>(a, st) : moded<float, 1>(a, st);
}

namespace {

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

// Elements that the rows of all operands can be moved by: pieces of 16 bytes, pairs of bf16, or one at a time.
struct Operand {
  const smat_rows* rows;
  bool output;
};
template <int N>
smat_status check_rows(const smat_norm_problem* p, const Operand (&ops)[N], int* pieces) {
  const int vec = p->dtype == SMAT_BF16 ? 8 : 4;
  bool wide = p->width % vec == 0, pairs = p->dtype == SMAT_BF16 && p->width % 2 == 0;
  for (const Operand& o : ops) {
    if (!o.rows) continue;
    if (!o.rows->data) return SMAT_ERR_NULL;
    if (!rows_ok(o.rows, p->batch, p->groups, p->T, p->width, o.output)) return SMAT_ERR_SHAPE;
  }
  for (const Operand& o : ops) {
    if (rows_misaligned(o.rows, p->dtype)) return SMAT_ERR_ALIGN;
    wide = wide && rows_at_multiples(o.rows, p->dtype, p->batch, p->groups, p->T, 16);
    pairs = pairs && rows_at_multiples(o.rows, p->dtype, p->batch, p->groups, p->T, 4);
  }
  *pieces = wide ? vec : pairs ? 2 : 1;
  return SMAT_OK;
}

NormArgs arguments(const smat_norm_problem* p) {
  NormArgs a{};
  a.weight = p->weight;
  a.weight_group = p->weight_group;
  a.scale = p->scale;
  a.batch = (uint32_t)p->batch;
  a.T = (uint32_t)p->T;
  a.width = p->width;
  a.eps = p->eps;
  a.inv_width = 1.f / (float)p->width;
  a.groups = (uint32_t)p->groups;
  a.sigmoid = p->activation == SMAT_ACT_SIGMOID;
  return a;
}
// One sequence of all tokens where every operand has them one behind the other (an absent operand's strides are zero).
void norm_join(NormArgs* a) {
  NormOperand* all[] = {&a->x, &a->residual, &a->gate, &a->dy, &a->dh_in, &a->y, &a->h, &a->dh, &a->dx, &a->dgate};
  if (a->T > 1 && a->batch > 1)
    for (const NormOperand* o : all)
      if (o->at.batch != (int64_t)a->T * o->at.token) return;
  if (a->T == 1)
    for (NormOperand* o : all) o->at.token = o->at.batch;
  a->T *= a->batch;
  a->batch = 1;
}
NormOperand operand(const smat_rows* r) { return r ? NormOperand{r->data, row_stride(r), 0, 0} : NormOperand{}; }

}  // namespace

extern "C" {

smat_status smat_norm_forward(const smat_norm_problem* p, const smat_rows* x, const smat_rows* residual, const smat_rows* gate,
                              const smat_rows* y, const smat_rows* h, void* cuda_stream) {
  if (!x || !y) return SMAT_ERR_NULL;
  smat_status s = check_problem(p);
  if (s != SMAT_OK) return s;
  int vec;
  s = check_rows(p, {{x, false}, {residual, false}, {gate, false}, {y, true}, {h, true}}, &vec);
  if (s != SMAT_OK) return s;
  if (!rows_device_ok()) return SMAT_ERR_ARCH;
  NormArgs a = arguments(p);
  a.x = operand(x);
  a.residual = operand(residual);
  a.gate = operand(gate);
  a.y = operand(y);
  a.h = operand(h);
  norm_join(&a);
  const cudaError_t err = smat_launch_norm_forward(a, p->dtype == SMAT_BF16, vec, static_cast<cudaStream_t>(cuda_stream));
  return err == cudaSuccess ? SMAT_OK : SMAT_ERR_LAUNCH;
}

size_t smat_norm_workspace_bytes(const smat_norm_problem* p) {
  if (check_problem(p) != SMAT_OK) return 0;
  return (size_t)smat_norm_partials(p->groups, p->width) * (size_t)p->width * sizeof(float) * (p->scale ? 2 : 1);
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
  int vec;
  s = check_rows(p, {{dy, false}, {h, false}, {gate, false}, {dscale ? x : nullptr, false}, {dh_in, false}, {dh, true}, {dx, true}, {dgate, true}}, &vec);
  if (s != SMAT_OK) return s;
  if ((reinterpret_cast<uintptr_t>(dweight) | reinterpret_cast<uintptr_t>(dscale)) & 3) return SMAT_ERR_ALIGN;
  if (dweight || dscale) {
    if (!workspace) return SMAT_ERR_NULL;
    if (workspace_bytes < smat_norm_workspace_bytes(p)) return SMAT_ERR_WORKSPACE;
    if (reinterpret_cast<uintptr_t>(workspace) & 255) return SMAT_ERR_ALIGN;
  }
  if (!rows_device_ok()) return SMAT_ERR_ARCH;
  NormArgs a = arguments(p);
  a.dy = operand(dy);
  a.h = operand(h);
  a.gate = operand(gate);
  if (dscale) a.x = operand(x);
  a.dh_in = operand(dh_in);
  a.dh = operand(dh);
  a.dx = operand(dx);
  a.dgate = operand(dgate);
  const size_t ctas = (size_t)smat_norm_partials(p->groups, p->width);
  if (dweight) a.dw = static_cast<float*>(workspace);
  if (dscale) a.ds = static_cast<float*>(workspace) + ctas * p->width;
  norm_join(&a);
  const cudaError_t err = smat_launch_norm_backward(a, p->dtype == SMAT_BF16, vec, dweight, dscale, static_cast<cudaStream_t>(cuda_stream));
  return err == cudaSuccess ? SMAT_OK : SMAT_ERR_LAUNCH;
}

}  // extern "C"
