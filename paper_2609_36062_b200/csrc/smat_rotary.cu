// Rotary positions: y = scale * R(θ) x on the first `rotated` columns of every row of Q and K, R a plane rotation of each pair by
// θ = position * frequency; the adjoint turns back by the same angle.
//
// The pass is a stream: every row is read once and written once, and the work between is two products and two sums a pair.
// A thread keeps one piece of the columns of one token (VEC pairs: two 16-byte words) and walks over the heads of Q and K
// with it, so that the angles of a token are formed once and not once a head: position * frequency in fp64 (in fp32 a position
// of 10^6 leaves an angle that is off by 0.06), reduced to a fraction of a turn there, then fp32 sincospi of a number below 1.
#include <cuda_runtime.h>

#include "smat_launch.cuh"
#include "smat_rows.cuh"

namespace {

constexpr int ROT_THREADS = 256, ROT_UNROLL = 4;
constexpr uint32_t ROT_CTAS = 148 * 4 * 6;   // six times as many as run at once (fp32 gradients of 4 x 5056: 57 us, with one time 61)

struct RotaryArgs {
  const void* x[2];
  void* y[2];
  RowStride xs[2], ys[2];
  int heads[2];
  uint32_t rows, T;           // batch * T, T
  int units, turned;          // pieces of a row: all, and those that hold pairs
  int d, rotated, span;       // span: heads that a CTA takes
  int copy[2];                // the columns behind the pairs have to be copied (the output is not the input)
  float scale, sign;
  const double* frequencies;
  const int64_t* positions;
  int64_t positions_batch, first;
};

// A piece: VEC pairs, as the elements [lo, lo + VEC) and [hi, hi + VEC); behind the pairs the next 2 VEC elements.
template <typename T, int VEC, bool INTER>
__global__ void __launch_bounds__(ROT_THREADS) rotary_kernel(const RotaryArgs a) {
  pdl_trigger();
  const uint32_t slots = ROT_THREADS / a.units;
  const uint32_t slot = threadIdx.x / a.units;
  const int unit = threadIdx.x - slot * a.units;
  const uint32_t row = blockIdx.x * slots + slot;
  pdl_wait();
  if (slot >= slots || row >= a.rows) return;
  const uint32_t b = row / a.T, t = row - b * a.T;
  const bool turns = unit < a.turned;
  bool both = true;   // the last piece behind the pairs may be half a piece
  int lo, hi;
  if (!turns) {
    lo = a.rotated + (unit - a.turned) * 2 * VEC;
    hi = lo + VEC;
    both = hi + VEC <= a.d;
  } else if (INTER) {
    lo = unit * 2 * VEC;
    hi = lo + VEC;
  } else {
    lo = unit * VEC;
    hi = lo + a.rotated / 2;
  }
  float c[VEC], s[VEC];
  if (turns) {
    const int64_t at = a.positions ? a.positions[(int64_t)b * a.positions_batch + t] : a.first + t;
    const double p = (double)at * 0.15915494309189533577;   // 1 / 2 pi
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      const double turn = p * a.frequencies[unit * VEC + i];
      sincospif((float)(2.0 * (turn - rint(turn))), &s[i], &c[i]);
      c[i] *= a.scale;
      s[i] *= a.scale * a.sign;
    }
  }
  const int total = a.heads[0] + a.heads[1];
  int h0 = blockIdx.y * a.span;
  const int h1 = min(h0 + a.span, total);
  for (; h0 < h1; h0 += ROT_UNROLL) {
    RowVec<T, VEC> u[ROT_UNROLL], v[ROT_UNROLL];
#pragma unroll
    for (int n = 0; n < ROT_UNROLL; ++n) {
      if (h0 + n >= h1) break;
      const int k = h0 + n >= a.heads[0], h = h0 + n - (k ? a.heads[0] : 0);
      const T* x = static_cast<const T*>(a.x[k]) + b * a.xs[k].batch + h * a.xs[k].head + t * a.xs[k].token;
      u[n].load(x + lo);
      if (both) v[n].load(x + hi);
    }
#pragma unroll
    for (int n = 0; n < ROT_UNROLL; ++n) {
      if (h0 + n >= h1) break;
      const int k = h0 + n >= a.heads[0], h = h0 + n - (k ? a.heads[0] : 0);
      T* y = static_cast<T*>(a.y[k]) + b * a.ys[k].batch + h * a.ys[k].head + t * a.ys[k].token;
      if (turns) {
        float f[2 * VEC], g[2 * VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) { f[i] = u[n].get(i); f[VEC + i] = v[n].get(i); }
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          const int one = INTER ? 2 * i : i, two = INTER ? 2 * i + 1 : VEC + i;
          g[one] = f[one] * c[i] - f[two] * s[i];
          g[two] = f[two] * c[i] + f[one] * s[i];
        }
        u[n].set(g);
        v[n].set(g + VEC);
      } else if (!a.copy[k]) {
        continue;
      }
      u[n].store(y + lo);
      if (both) v[n].store(y + hi);
    }
  }
}

template <typename T, int VEC>
cudaError_t launch(RotaryArgs& a, int interleaved, cudaStream_t st) {
  a.turned = a.rotated / 2 / VEC;
  a.units = a.turned + (a.d - a.rotated + 2 * VEC - 1) / (2 * VEC);
  const uint32_t slots = ROT_THREADS / a.units, blocks = (uint32_t)(((uint64_t)a.rows + slots - 1) / slots);
  const int total = a.heads[0] + a.heads[1];
  // heads of a token stay with one CTA, which forms their angles once, as long as the CTAs fill the GPU
  int parts = (int)((ROT_CTAS + blocks - 1) / blocks);
  if (parts > total) parts = total;
  a.span = (total + parts - 1) / parts;
  const dim3 grid(blocks, (unsigned)((total + a.span - 1) / a.span));
  return interleaved ? smat_launch_pdl(rotary_kernel<T, VEC, true>, grid, ROT_THREADS, 0, st, a)
                     : smat_launch_pdl(rotary_kernel<T, VEC, false>, grid, ROT_THREADS, 0, st, a);
}

}  // namespace

extern "C" smat_status smat_rotary(const smat_rotary_problem* p, const smat_rows* q, const smat_rows* k, const smat_rows* q_out,
                                   const smat_rows* k_out, void* cuda_stream) {
  if (!p || !q || !q_out || !q->data || !q_out->data || !p->frequencies) return SMAT_ERR_NULL;
  if ((k != nullptr) != (k_out != nullptr) || (k && (!k->data || !k_out->data))) return SMAT_ERR_NULL;
  if (p->dtype != SMAT_F32 && p->dtype != SMAT_BF16) return SMAT_ERR_DTYPE;
  if (p->batch < 1 || p->q_heads < 1 || p->T < 1 || (k && p->k_heads < 1) || p->q_heads > 32767 || (k && p->k_heads > 32767))
    return SMAT_ERR_SHAPE;
  if (p->T > INT32_MAX || p->T * p->batch > INT32_MAX) return SMAT_ERR_SHAPE;
  if (p->d < 1 || p->d > 512 || p->rotated < 2 || p->rotated > p->d || p->rotated % 2) return SMAT_ERR_SHAPE;
  const int kh = k ? p->k_heads : 0;
  if (!rows_ok(q, p->batch, p->q_heads, p->T, p->d, false) || !rows_ok(q_out, p->batch, p->q_heads, p->T, p->d, true) ||
      !rows_ok(k, p->batch, kh, p->T, p->d, false) || !rows_ok(k_out, p->batch, kh, p->T, p->d, true))
    return SMAT_ERR_SHAPE;
  if (p->positions && (p->positions_batch < 0 || p->positions_batch > ((int64_t)1 << 40))) return SMAT_ERR_SHAPE;
  if (rows_misaligned(q, p->dtype) || rows_misaligned(k, p->dtype) || rows_misaligned(q_out, p->dtype) ||
      rows_misaligned(k_out, p->dtype) || (reinterpret_cast<uintptr_t>(p->frequencies) & 7) ||
      (reinterpret_cast<uintptr_t>(p->positions) & 7))
    return SMAT_ERR_ALIGN;
  if (!rows_device_ok()) return SMAT_ERR_ARCH;
  RotaryArgs a{};
  const smat_rows *in[2] = {q, k}, *out[2] = {q_out, k_out};
  for (int i = 0; i < 2; ++i) {
    if (!in[i]) continue;
    a.x[i] = in[i]->data;
    a.y[i] = out[i]->data;
    a.xs[i] = row_stride(in[i]);
    a.ys[i] = row_stride(out[i]);
    a.copy[i] = in[i]->data != out[i]->data;
  }
  a.heads[0] = p->q_heads;
  a.heads[1] = kh;
  a.rows = (uint32_t)(p->T * p->batch);
  a.T = (uint32_t)p->T;
  a.d = p->d;
  a.rotated = p->rotated;
  a.scale = p->scale;
  a.sign = p->adjoint ? -1.f : 1.f;
  a.frequencies = p->frequencies;
  a.positions = p->positions;
  a.positions_batch = p->positions_batch;
  a.first = p->first;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  // pieces of 16 bytes, pairs of elements, or one at a time (90 of 128 columns turned: 120 us where 96 take 47)
  const auto moves = [&](int vec) {
    const unsigned bytes = (unsigned)(vec * dtype_bytes(p->dtype));
    return p->d % vec == 0 && p->rotated % (2 * vec) == 0 && rows_at_multiples(q, p->dtype, p->batch, p->q_heads, p->T, bytes) &&
           rows_at_multiples(k, p->dtype, p->batch, kh, p->T, bytes) && rows_at_multiples(q_out, p->dtype, p->batch, p->q_heads, p->T, bytes) &&
           rows_at_multiples(k_out, p->dtype, p->batch, kh, p->T, bytes);
  };
  const int il = p->interleaved;
  cudaError_t err;
  if (p->dtype == SMAT_BF16)
    err = moves(8) ? launch<__nv_bfloat16, 8>(a, il, st) : moves(2) ? launch<__nv_bfloat16, 2>(a, il, st) : launch<__nv_bfloat16, 1>(a, il, st);
  else
    err = moves(4) ? launch<float, 4>(a, il, st) : moves(2) ? launch<float, 2>(a, il, st) : launch<float, 1>(a, il, st);
  return err == cudaSuccess ? SMAT_OK : SMAT_ERR_LAUNCH;
}
