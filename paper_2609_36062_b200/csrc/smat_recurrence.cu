// Gated linear recurrence of every channel, h_t = a_t h_{t-1} + x_t with a_t = exp(log_a_t), and its gradients
//     c_t = a_t (dh_t + c_{t+1}),   dx_t = dh_t + c_{t+1},   dlog_a_t = c_t h_{t-1},
// the same kind of recurrence from the last token to the first.  Below, s counts tokens in the order of the recurrence.
//
// Tokens s in a row map the state that enters them to the one that leaves them, state -> A state + H, and two such maps in a row
// are one again: (A, H) then (A', H') is (A' A, A' H + H').  So a long sequence is cut into pieces whose maps are formed side by
// side, joined in order, and applied: a CTA takes 64 channels (a line of 128 bytes of bf16) and walks over the tokens a tile at a time; in the
// tile a thread has VEC channels of STEPS tokens in registers, forms their map, the maps meet by shuffles (a warp) and shared
// memory (the CTA), and the thread goes over its tokens again from the state that enters them.  Every input is read once,
// and the next tile's loads are in flight meanwhile.  Where there are too few channels and sequences to fill the GPU, the CTAs of
// a cluster take tiles in turn and hand their tile's map to one another through distributed shared memory: one cluster barrier a
// round, no flags in global memory, and sums in an order that is the same from run to run.
//
// Bound by HBM.  A closed gate (a = 0) drops what came before it, also where that is not finite.
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include "smat_launch.cuh"
#include "smat_rows.cuh"

namespace {

namespace cg = cooperative_groups;

constexpr int REC_THREADS = 256, REC_WARPS = REC_THREADS / 32, REC_MAX_CLUSTER = 8;

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
__device__ __forceinline__ float step(float a, float state, float x) { return a == 0.f ? x : fmaf(a, state, x); }

// What a thread holds of a tile: VEC channels of STEPS tokens.
template <typename TX, typename TA, int VEC, int STEPS, bool BACK>
struct Share {
  RowVec<TX, VEC> x[STEPS];
  RowVec<TA, VEC> a[STEPS];
  RowVec<TX, VEC> h[BACK ? STEPS : 1];

  // Tokens s .. s + STEPS - 1; those from T on are left as they are (their number is `count`).
  __device__ __forceinline__ void load(const RecArgs& p, const TX* xp, const TA* ap, const TX* hp, int64_t s, int count) {
#pragma unroll
    for (int l = 0; l < STEPS; ++l) {
      if (l >= count) break;
      const int64_t t = BACK ? p.T - 1 - (s + l) : s + l;
      x[l].load(xp + t * p.xs.token);
      a[l].load(ap + t * p.as.token);
      if (BACK && t > 0) h[l].load(hp + (t - 1) * p.hs.token);
    }
  }
};

// The tokens of a share from `state` on: outputs stored, `state` becomes the one behind them.
template <typename TX, typename TA, int VEC, int STEPS, bool BACK>
__device__ __forceinline__ void apply(const RecArgs& p, const Share<TX, TA, VEC, STEPS, BACK>& in, const float (&gate)[STEPS][VEC],
                                      float (&state)[VEC], TX* op, TA* dap, const float* h0, int64_t s, int count) {
#pragma unroll
  for (int l = 0; l < STEPS; ++l) {
    if (l >= count) break;
    const int64_t t = BACK ? p.T - 1 - (s + l) : s + l;
    float v[VEC];
    if (BACK) {
      float d[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        v[i] = in.x[l].get(i) + state[i];                                  // dx
        state[i] = gate[l][i] == 0.f ? 0.f : gate[l][i] * v[i];            // c
        const float before = t > 0 ? in.h[l].get(i) : h0 ? h0[i] : 0.f;
        d[i] = gate[l][i] == 0.f ? 0.f : state[i] * before;
      }
      RowVec<TA, VEC> da;
      da.set(d);
      da.store(dap + t * p.das.token);
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) v[i] = state[i] = step(gate[l][i], state[i], in.x[l].get(i));
    }
    RowVec<TX, VEC> o;
    o.set(v);
    o.store(op + t * p.os.token);
  }
}

// Short sequences: a thread takes VEC channels of a sequence from the first token to the last.
template <typename TX, typename TA, int VEC, bool BACK>
__global__ void __launch_bounds__(REC_THREADS) recurrence_short_kernel(const RecArgs p, uint32_t pieces) {
  constexpr int STEPS = 2;
  pdl_trigger();
  const uint32_t n = blockIdx.x * REC_THREADS + threadIdx.x, b = blockIdx.y;
  pdl_wait();
  if (n >= pieces) return;
  const int c = (int)n * VEC;
  const TX* xp = static_cast<const TX*>(p.x) + b * p.xs.batch + c;
  const TA* ap = static_cast<const TA*>(p.log_a) + b * p.as.batch + c;
  const TX* hp = BACK ? static_cast<const TX*>(p.h) + b * p.hs.batch + c : nullptr;
  TX* op = static_cast<TX*>(p.out) + b * p.os.batch + c;
  TA* dap = BACK ? static_cast<TA*>(p.dlog_a) + b * p.das.batch + c : nullptr;
  const int64_t row = (int64_t)b * p.channels + c;
  float state[VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) state[i] = p.begin ? p.begin[row + i] : 0.f;
  for (int64_t s = 0; s < p.T; s += STEPS) {
    const int count = (int)(p.T - s < STEPS ? p.T - s : STEPS);
    Share<TX, TA, VEC, STEPS, BACK> in;
    in.load(p, xp, ap, hp, s, count);
    float gate[STEPS][VEC];
#pragma unroll
    for (int l = 0; l < STEPS; ++l) {
      if (l >= count) break;
#pragma unroll
      for (int i = 0; i < VEC; ++i) gate[l][i] = expf(in.a[l].get(i));
    }
    apply<TX, TA, VEC, STEPS, BACK>(p, in, gate, state, op, dap, p.h0 ? p.h0 + row : nullptr, s, count);
  }
  if (p.end) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) p.end[row + i] = state[i];
  }
}

// LANES lanes hold the channels of a token; a tile is REC_THREADS / LANES * STEPS tokens.
template <typename TX, typename TA, int VEC, int LANES, int STEPS, bool BACK>
__global__ void __launch_bounds__(REC_THREADS, 2) recurrence_kernel(const RecArgs p) {
  constexpr int COLS = LANES * VEC, TILE = REC_THREADS / LANES * STEPS;
  static_assert(COLS <= REC_THREADS, "a thread joins the warps' maps of one channel");
  __shared__ float2 warp_map[REC_WARPS][COLS];                  // (A, H) of a warp's tokens
  __shared__ float entering[REC_WARPS][COLS];                   // the state that enters a warp's tokens
  __shared__ float2 tile_map[2][REC_MAX_CLUSTER][COLS];         // (A, H) of the cluster's tiles, this round's and the last one's
  const cg::cluster_group cluster = cg::this_cluster();
  const int ranks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int column = lane % LANES, part = tid / LANES;          // this thread's channels, and its place in the tile
  const uint32_t b = blockIdx.z;
  const int c0 = blockIdx.y * COLS, c = c0 + column * VEC;
  const bool valid = c < p.channels;
  pdl_trigger();
  if (ranks > 1) cluster.sync();      // all of the cluster run before one writes to another's shared memory
  pdl_wait();
  const TX* xp = static_cast<const TX*>(p.x) + b * p.xs.batch + c;
  const TA* ap = static_cast<const TA*>(p.log_a) + b * p.as.batch + c;
  const TX* hp = BACK ? static_cast<const TX*>(p.h) + b * p.hs.batch + c : nullptr;
  TX* op = static_cast<TX*>(p.out) + b * p.os.batch + c;
  TA* dap = BACK ? static_cast<TA*>(p.dlog_a) + b * p.das.batch + c : nullptr;
  const float* h0 = p.h0 ? p.h0 + (int64_t)b * p.channels + c : nullptr;
  const int64_t row = (int64_t)b * p.channels + c0 + tid;       // of the channel whose maps this thread joins
  const bool joins = tid < COLS && c0 + tid < p.channels;
  float carry = joins && p.begin ? p.begin[row] : 0.f;

  const int64_t round = (int64_t)ranks * TILE;
  int64_t s = (int64_t)rank * TILE + part * STEPS;
  auto count_at = [&](int64_t at) { return !valid || at >= p.T ? 0 : (int)(p.T - at < STEPS ? p.T - at : STEPS); };
  Share<TX, TA, VEC, STEPS, BACK> next;
  next.load(p, xp, ap, hp, s, count_at(s));
  int turn = 0;
  for (int64_t first = 0; first < p.T; first += round, s += round, turn ^= 1) {
    const Share<TX, TA, VEC, STEPS, BACK> in = next;
    const int count = count_at(s);
    next.load(p, xp, ap, hp, s + round, count_at(s + round));
    // the map of this thread's tokens
    float gate[STEPS][VEC], A[VEC], H[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) { A[i] = 1.f; H[i] = 0.f; }
#pragma unroll
    for (int l = 0; l < STEPS; ++l) {
      if (l >= count) break;
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const float a = expf(in.a[l].get(i)), x = in.x[l].get(i);
        gate[l][i] = a;
        A[i] *= a;
        H[i] = BACK ? (a == 0.f ? 0.f : a * (H[i] + x)) : step(a, H[i], x);
      }
    }
    // ... of the warp's tokens up to and with this thread's
#pragma unroll
    for (int o = LANES; o < 32; o *= 2) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const float before_A = __shfl_up_sync(0xffffffffu, A[i], o), before_H = __shfl_up_sync(0xffffffffu, H[i], o);
        if (lane >= o) {
          H[i] = step(A[i], before_H, H[i]);
          A[i] = A[i] == 0.f ? 0.f : A[i] * before_A;
        }
      }
    }
    if (lane >= 32 - LANES)
#pragma unroll
      for (int i = 0; i < VEC; ++i) warp_map[warp][column * VEC + i] = make_float2(A[i], H[i]);
    // ... and up to this thread's, without it
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      const float a = __shfl_up_sync(0xffffffffu, A[i], LANES), h = __shfl_up_sync(0xffffffffu, H[i], LANES);
      A[i] = lane >= LANES ? a : 1.f;
      H[i] = lane >= LANES ? h : 0.f;
    }
    __syncthreads();
    if (ranks > 1) {
      if (tid < COLS) {
        float2 m = warp_map[0][tid];
#pragma unroll
        for (int w = 1; w < REC_WARPS; ++w) {
          const float2 n = warp_map[w][tid];
          m = make_float2(n.x == 0.f ? 0.f : n.x * m.x, step(n.x, m.y, n.y));
        }
        for (int r = 0; r < ranks; ++r) *cluster.map_shared_rank(&tile_map[turn][rank][tid], r) = m;
      }
      cluster.sync();
    }
    if (tid < COLS) {
      float state = carry, behind = carry;
      if (ranks > 1) {
        for (int r = 0; r < ranks; ++r) {
          if (r == rank) state = behind;
          const float2 m = tile_map[turn][r][tid];
          behind = step(m.x, behind, m.y);
        }
      }
#pragma unroll
      for (int w = 0; w < REC_WARPS; ++w) {
        entering[w][tid] = state;
        const float2 m = warp_map[w][tid];
        state = step(m.x, state, m.y);
      }
      carry = ranks > 1 ? behind : state;
    }
    __syncthreads();
    float state[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) state[i] = step(A[i], entering[warp][column * VEC + i], H[i]);
    apply<TX, TA, VEC, STEPS, BACK>(p, in, gate, state, op, dap, h0, s, count);
  }
  if (p.end && rank == 0 && joins) p.end[row] = carry;
}

constexpr int64_t REC_SHORT = 8;          // tokens up to which a thread takes a sequence by itself
constexpr int64_t REC_CTAS = 148 * 2;     // as many as run at once

template <typename TX, typename TA, int VEC, int LANES, int STEPS, bool BACK>
cudaError_t launch(const RecArgs& a, int batch, cudaStream_t st) {
  if (a.T <= REC_SHORT) {
    const uint32_t pieces = (uint32_t)((a.channels + VEC - 1) / VEC);
    return smat_launch_pdl(recurrence_short_kernel<TX, TA, VEC, BACK>, dim3((pieces + REC_THREADS - 1) / REC_THREADS, (unsigned)batch),
                           REC_THREADS, 0, st, a, pieces);
  }
  constexpr int COLS = LANES * VEC, TILE = REC_THREADS / LANES * STEPS;
  const int64_t columns = (a.channels + COLS - 1) / COLS, tiles = (a.T + TILE - 1) / TILE;
  // tiles in turn over the CTAs of a cluster until they fill the GPU
  unsigned ranks = 1;
  while (ranks < REC_MAX_CLUSTER && 2 * ranks <= tiles && columns * batch * ranks < REC_CTAS) ranks *= 2;
  return smat_launch_pdl_cluster(recurrence_kernel<TX, TA, VEC, LANES, STEPS, BACK>, dim3(ranks, (unsigned)columns, (unsigned)batch),
                                 REC_THREADS, 0, ranks, st, a);
}

template <bool BACK>
cudaError_t dispatch(const RecArgs& a, const smat_recurrence_problem* p, bool wide, cudaStream_t st) {
  if (p->dtype == SMAT_F32)
    return wide ? launch<float, float, 4, 16, 4, BACK>(a, p->batch, st) : launch<float, float, 1, 32, 4, BACK>(a, p->batch, st);
  if (p->gate_dtype == SMAT_BF16)
    return wide ? launch<__nv_bfloat16, __nv_bfloat16, 8, 8, 4, BACK>(a, p->batch, st)
                : launch<__nv_bfloat16, __nv_bfloat16, 1, 32, 4, BACK>(a, p->batch, st);
  return wide ? launch<__nv_bfloat16, float, 4, 16, 4, BACK>(a, p->batch, st)
              : launch<__nv_bfloat16, float, 1, 32, 4, BACK>(a, p->batch, st);
}

struct Operand {
  const smat_rows* rows;
  smat_dtype dtype;
  bool output;
};
// wide: 16-byte pieces of the widest operand everywhere.
template <int N>
smat_status check(const smat_recurrence_problem* p, const Operand (&ops)[N], const float* const (&states)[3], bool* wide) {
  if (!p) return SMAT_ERR_NULL;
  for (const Operand& o : ops)
    if (!o.rows || !o.rows->data) return SMAT_ERR_NULL;
  if ((p->dtype != SMAT_F32 && p->dtype != SMAT_BF16) || (p->gate_dtype != p->dtype && p->gate_dtype != SMAT_F32))
    return SMAT_ERR_DTYPE;
  if (p->batch < 1 || p->batch > 65535 || p->T < 1 || p->T > ((int64_t)1 << 40) || p->channels < 1 || p->channels > (1 << 20))
    return SMAT_ERR_SHAPE;
  *wide = p->channels % (p->gate_dtype == SMAT_BF16 ? 8 : 4) == 0;
  for (const Operand& o : ops)
    if (!rows_ok(o.rows, p->batch, 1, p->T, p->channels, o.output)) return SMAT_ERR_SHAPE;
  for (const Operand& o : ops) {
    if (rows_misaligned(o.rows, o.dtype)) return SMAT_ERR_ALIGN;
    *wide = *wide && rows_in_16(o.rows, o.dtype, p->batch, 1, p->T);
  }
  for (const float* s : states)
    if (reinterpret_cast<uintptr_t>(s) & 3) return SMAT_ERR_ALIGN;
  return rows_device_ok() ? SMAT_OK : SMAT_ERR_ARCH;
}

}  // namespace

extern "C" {

smat_status smat_recurrence_forward(const smat_recurrence_problem* p, const smat_rows* x, const smat_rows* log_a, const float* h0,
                                    const smat_rows* h, float* hT, void* cuda_stream) {
  if (!p) return SMAT_ERR_NULL;
  bool wide;
  const smat_status s = check(p, {{x, p->dtype, false}, {log_a, p->gate_dtype, false}, {h, p->dtype, true}}, {h0, hT, nullptr}, &wide);
  if (s != SMAT_OK) return s;
  RecArgs a{};
  a.x = x->data; a.xs = row_stride(x);
  a.log_a = log_a->data; a.as = row_stride(log_a);
  a.out = h->data; a.os = row_stride(h);
  a.begin = h0;
  a.end = hT;
  a.T = p->T;
  a.channels = p->channels;
  return dispatch<false>(a, p, wide, static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? SMAT_OK : SMAT_ERR_LAUNCH;
}

smat_status smat_recurrence_backward(const smat_recurrence_problem* p, const smat_rows* log_a, const smat_rows* h, const smat_rows* dh,
                                     const float* h0, const float* dhT, const smat_rows* dx, const smat_rows* dlog_a, float* dh0,
                                     void* cuda_stream) {
  if (!p) return SMAT_ERR_NULL;
  bool wide;
  const smat_status s = check(p, {{log_a, p->gate_dtype, false}, {h, p->dtype, false}, {dh, p->dtype, false}, {dx, p->dtype, true},
                                  {dlog_a, p->gate_dtype, true}}, {h0, dhT, dh0}, &wide);
  if (s != SMAT_OK) return s;
  RecArgs a{};
  a.x = dh->data; a.xs = row_stride(dh);
  a.log_a = log_a->data; a.as = row_stride(log_a);
  a.h = h->data; a.hs = row_stride(h);
  a.out = dx->data; a.os = row_stride(dx);
  a.dlog_a = dlog_a->data; a.das = row_stride(dlog_a);
  a.begin = dhT;
  a.h0 = h0;
  a.end = dh0;
  a.T = p->T;
  a.channels = p->channels;
  return dispatch<true>(a, p, wide, static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? SMAT_OK : SMAT_ERR_LAUNCH;
}

}  // extern "C"
