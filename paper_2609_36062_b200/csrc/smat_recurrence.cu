// Gated linear recurrence of every channel, h_t = a_t h_{t-1} + x_t with a_t = exp(log_a_t), and its gradients
//     c_t = a_t (dh_t + c_{t+1}),   dx_t = dh_t + c_{t+1},   dlog_a_t = c_t h_{t-1},
// the same kind of recurrence from the last token to the first.  Below, s counts tokens in the order of the recurrence.
//
// Tokens s in a row map the state that enters them to the one that leaves them, state -> A state + H, and two such maps in a row
// are one again: (A, H) then (A', H') is (A' A, A' H + H') (A' A as rec_joined has it).  So a long sequence is cut into pieces whose maps are formed side by
// side, joined in order, and applied: a CTA takes 64 channels (a line of 128 bytes of bf16) and walks over the tokens a tile at a time; in the
// tile a thread has VEC channels of STEPS tokens in registers, forms their map, the maps meet by shuffles (a warp) and shared
// memory (the CTA), and the thread goes over its tokens again from the state that enters them.  Every input is read once,
// and the next tile's loads are in flight meanwhile.  Where there are too few channels and sequences to fill the GPU, the CTAs of
// a cluster take tiles in turn and hand their tile's map to one another through distributed shared memory: one cluster barrier a
// round, no flags in global memory, and sums in an order that is the same from run to run.  Where sequences are many and short, a
// thread takes its channels of a whole sequence instead (rec_sequential).
//
// Bound by HBM.  A closed gate (a = 0) drops what came before it, also where that is not finite.
#include <type_traits>

#include "smat_recurrence.cuh"

namespace {

namespace cg = cooperative_groups;

// Where an operand's tokens of one tile lie: the same address for all threads of a CTA, and a thread's distance from it.  So the
// address arithmetic of a token is left to the uniform datapath (64-bit products of token and stride in every thread were
// a fifth of all instructions).  s counts tokens in the order of the recurrence, t = s or T - 1 - s.
template <typename T, typename OFF>
struct Place {
  const T* base;      // of the last thread's tokens (backward) or the first's: the lowest address
  int64_t token;      // elements from one s to the next
  OFF off;
  __device__ __forceinline__ T* at(int l) const { return const_cast<T*>(base + l * token + off); }
};

// What a thread holds of a tile: VEC channels of STEPS tokens.
template <typename TX, typename TA, int VEC, int STEPS, bool BACK>
struct Share {
  RowVec<TX, VEC> x[STEPS];
  RowVec<TA, VEC> a[STEPS];
  RowVec<TX, VEC> h[BACK ? STEPS : 1];

  // `count` tokens, and behind them tokens that leave the state as it is.  The last of `left` tokens up to the end of the
  // sequence is token 0 of a backward pass, which has none before it.
  template <typename OFF>
  __device__ __forceinline__ void load(const Place<TX, OFF>& xp, const Place<TA, OFF>& ap, const Place<TX, OFF>& hp, int count, int64_t left) {
    if (count == STEPS && (!BACK || left > STEPS)) {
#pragma unroll
      for (int l = 0; l < STEPS; ++l) {
        x[l].load(xp.at(l));
        a[l].load(ap.at(l));
        if (BACK) h[l].load(hp.at(l));
      }
      return;
    }
#pragma unroll
    for (int l = 0; l < STEPS; ++l) {
      x[l].clear();
      a[l].clear();
      if (BACK) h[l].clear();
      if (l >= count) continue;
      x[l].load(xp.at(l));
      a[l].load(ap.at(l));
      if (BACK && l + 1 < left) h[l].load(hp.at(l));
    }
  }
};

// One channel of a share's token l, from the state before it.  Backward the output v_t = x_t + c_{t+1} is carried instead of the state
// c_t = a_t v_t, so that a token is one fused product and sum either way, and the values behind a closed gate are the same, bit for
// bit, whatever came before it.
template <bool CLOSED, bool BACK, int VEC, int STEPS>
__device__ __forceinline__ void advance(const float (&gate)[STEPS][VEC], int l, int i, float x, float& v, float& state) {
  const float a = gate[l][i];
  if (BACK) {
    const float before = l ? gate[l ? l - 1 : 0][i] : 1.f;
    if (l == 0) v = x + state;
    else v = CLOSED ? rec_step(before, v, x) : fmaf(before, v, x);
    state = CLOSED && a == 0.f ? 0.f : a * v;
  } else {
    v = state = CLOSED ? rec_step(a, state, x) : fmaf(a, state, x);
  }
}

// The map (A, H) of a share's tokens.
template <bool CLOSED, typename TX, typename TA, int VEC, int STEPS, bool BACK>
__device__ __forceinline__ void map_of(const Share<TX, TA, VEC, STEPS, BACK>& in, const float (&gate)[STEPS][VEC], float (&A)[VEC],
                                       float (&H)[VEC]) {
  float v[VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) { A[i] = 1.f; H[i] = v[i] = 0.f; }
#pragma unroll
  for (int l = 0; l < STEPS; ++l) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      A[i] *= gate[l][i];
      advance<CLOSED, BACK>(gate, l, i, in.x[l].get(i), v[i], H[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < VEC; ++i) {
    if (A[i] > 0.f) continue;
    float least = gate[0][i];
#pragma unroll
    for (int l = 1; l < STEPS; ++l) least = fminf(least, gate[l][i]);
    A[i] = rec_factor(A[i], least);
  }
}

// The tokens of a share from `state` on: outputs stored, `state` becomes the one behind them.  Returns zero if all of it is finite.
// h0: of this thread's channels, or null; only token 0 of a backward pass, the last of `left`, looks at it.
template <bool CLOSED, typename TX, typename TA, int VEC, int STEPS, bool BACK, typename OFF>
__device__ __forceinline__ float apply(const Share<TX, TA, VEC, STEPS, BACK>& in, const float (&gate)[STEPS][VEC], float (&state)[VEC],
                                       const Place<TX, OFF>& op, const Place<TA, OFF>& dap, const float* h0, int count, int64_t left) {
  float zeros = 0.f, v[VEC], d[VEC];
  const bool last = BACK && left <= STEPS;
#pragma unroll
  for (int i = 0; i < VEC; ++i) v[i] = 0.f;
#pragma unroll
  for (int l = 0; l < STEPS; ++l) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      advance<CLOSED, BACK>(gate, l, i, in.x[l].get(i), v[i], state[i]);
      if (BACK) {
        float before = in.h[BACK ? l : 0].get(i);
        if (last && l + 1 == left && h0) before = h0[i];
        d[i] = CLOSED && gate[l][i] == 0.f ? 0.f : state[i] * before;
        zeros = fmaf(d[i], 0.f, zeros);
      }
    }
    if (l < count) {
      RowVec<TX, VEC> o;
      o.set(v);
      o.store(op.at(l));
      if constexpr (BACK) {
        RowVec<TA, VEC> da;
        da.set(d);
        da.store(dap.at(l));
      }
    }
  }
#pragma unroll
  for (int i = 0; i < VEC; ++i) zeros = fmaf(state[i], 0.f, zeros);
  return zeros;
}

template <typename TX, typename TA, int VEC, int STEPS, bool BACK, typename OFF>
__device__ __forceinline__ void apply(const Share<TX, TA, VEC, STEPS, BACK>& in, const float (&gate)[STEPS][VEC], float (&state)[VEC],
                                      const Place<TX, OFF>& op, const Place<TA, OFF>& dap, const float* h0, int count, int64_t left) {
  float entered[VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) entered[i] = state[i];
  if (!rec_not_finite(apply<false>(in, gate, state, op, dap, h0, count, left))) return;
#pragma unroll
  for (int i = 0; i < VEC; ++i) state[i] = entered[i];
  apply<true>(in, gate, state, op, dap, h0, count, left);
}

// exp of the log-gates.  From -4 up, 2^(x log2 e) with one rounding of the exponent: it is off by 2^-22 there, and the power by 2^-22
// of itself; below, where the rounded exponent would cost more, expf.
template <typename TX, typename TA, int VEC, int STEPS, bool BACK>
__device__ __forceinline__ void gates_of(const Share<TX, TA, VEC, STEPS, BACK>& in, float (&gate)[STEPS][VEC]) {
  float least = 0.f;
#pragma unroll
  for (int l = 0; l < STEPS; ++l)
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      const float x = in.a[l].get(i);
      least = fminf(least, x);
      asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(gate[l][i]) : "f"(x * 1.4426950408889634f));
    }
  if (least >= -4.f) return;
#pragma unroll
  for (int l = 0; l < STEPS; ++l)
#pragma unroll
    for (int i = 0; i < VEC; ++i) gate[l][i] = expf(in.a[l].get(i));
}

// Sequences that are short for their number: a thread takes VEC channels of a sequence from the first token to the last, STEPS of them
// while the next STEPS are on their way.  No maps, nothing to join.
constexpr int SEQ_THREADS = 128;
template <typename TX, typename TA, int VEC, int STEPS, bool BACK>
__global__ void __launch_bounds__(SEQ_THREADS) recurrence_sequential_kernel(const RecArgs p, uint32_t pieces) {
  pdl_trigger();
  const uint32_t n = blockIdx.x * SEQ_THREADS + threadIdx.x, b = blockIdx.y;
  pdl_wait();
  if (n >= pieces) return;
  const int c = (int)n * VEC;
  const int64_t row = (int64_t)b * p.channels + c;
  const auto place = [&](auto* data, const RowStride& at, int before) {
    using P = Place<std::remove_const_t<std::remove_pointer_t<decltype(data)>>, uint64_t>;
    return P{data + b * at.batch + (BACK ? p.T - 1 - before : 0) * at.token + c, BACK ? -at.token : at.token, 0};
  };
  auto xp = place(static_cast<const TX*>(p.x), p.xs, 0), hp = place(static_cast<const TX*>(p.h), p.hs, 1);
  auto ap = place(static_cast<const TA*>(p.log_a), p.as, 0);
  auto op = place(static_cast<const TX*>(p.out), p.os, 0);
  auto dap = place(static_cast<const TA*>(p.dlog_a), p.das, 0);
  const auto move = [](auto& at) { at.base += STEPS * at.token; };
  const auto count_at = [&](int64_t left) { return left < 0 ? 0 : (int)(left < STEPS ? left : STEPS); };
  float state[VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) state[i] = p.begin ? p.begin[row + i] : 0.f;
  Share<TX, TA, VEC, STEPS, BACK> next;
  next.load(xp, ap, hp, count_at(p.T), p.T);
  for (int64_t left = p.T; left > 0; left -= STEPS) {
    const Share<TX, TA, VEC, STEPS, BACK> in = next;
    move(xp);
    move(ap);
    if (BACK) move(hp);
    if (left > STEPS) next.load(xp, ap, hp, count_at(left - STEPS), left - STEPS);
    float gate[STEPS][VEC];
    gates_of(in, gate);
    apply(in, gate, state, op, dap, p.h0 ? p.h0 + row : nullptr, count_at(left), left);
    move(op);
    if (BACK) move(dap);
  }
  if (p.end) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) p.end[row + i] = state[i];
  }
}

// LANES lanes hold the channels of a token; a tile is REC_THREADS / LANES * STEPS tokens.
template <typename TX, typename TA, int VEC, int LANES, int STEPS, bool BACK, typename OFF>
__global__ void __launch_bounds__(REC_THREADS, 2) recurrence_kernel(const RecArgs p) {
  constexpr int COLS = LANES * VEC, TILE = REC_THREADS / LANES * STEPS;
  static_assert(COLS <= REC_THREADS && (LANES == 16 || LANES == 32), "a thread joins the warps' maps of one channel; halves of a warp");
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
  if (ranks > 1) cluster.sync();      // all of the cluster run before one writes to another's shared memory
  pdl_wait();
  const float* h0 = p.h0 && valid ? p.h0 + (int64_t)b * p.channels + c : nullptr;
  const int64_t row = (int64_t)b * p.channels + c0 + tid;       // of the channel whose maps this thread joins
  const bool joins = tid < COLS && c0 + tid < p.channels;
  float carry = joins && p.begin ? p.begin[row] : 0.f;

  const int64_t round = (int64_t)ranks * TILE;
  const int64_t begin = (int64_t)rank * TILE;
  // an operand's place at this CTA's tile of round 0, `before` tokens before its own
  const auto place = [&](auto* data, const RowStride& at, int before) {
    using P = Place<std::remove_const_t<std::remove_pointer_t<decltype(data)>>, OFF>;
    const int64_t t = BACK ? p.T - 1 - begin - before - (TILE - STEPS) : begin;
    return P{data + b * at.batch + t * at.token + c0, BACK ? -at.token : at.token,
             (OFF)((OFF)(BACK ? TILE - STEPS - part * STEPS : part * STEPS) * (OFF)at.token + (OFF)(column * VEC))};
  };
  auto xp = place(static_cast<const TX*>(p.x), p.xs, 0), hp = place(static_cast<const TX*>(p.h), p.hs, 1);
  auto ap = place(static_cast<const TA*>(p.log_a), p.as, 0);
  auto op = place(static_cast<const TX*>(p.out), p.os, 0);
  auto dap = place(static_cast<const TA*>(p.dlog_a), p.das, 0);
  const auto move = [&](auto& at) { at.base += round * at.token; };
  const auto count_at = [&](int64_t at) { return !valid || at >= p.T ? 0 : (int)(p.T - at < STEPS ? p.T - at : STEPS); };
  int64_t s = begin + part * STEPS;
  Share<TX, TA, VEC, STEPS, BACK> next;
  next.load(xp, ap, hp, count_at(s), p.T - s);
  int turn = 0;
  for (int64_t first = 0; first < p.T; first += round, s += round, turn ^= 1) {
    const Share<TX, TA, VEC, STEPS, BACK> in = next;
    const int count = count_at(s);
    move(xp);
    move(ap);
    if (BACK) move(hp);
    next.load(xp, ap, hp, count_at(s + round), p.T - s - round);
    // the map of this thread's tokens
    float gate[STEPS][VEC], A[VEC], H[VEC], zeros = 0.f;
    gates_of(in, gate);
    map_of<false>(in, gate, A, H);
#pragma unroll
    for (int i = 0; i < VEC; ++i) zeros = fmaf(H[i], 0.f, zeros);
    if (rec_not_finite(zeros)) map_of<true>(in, gate, A, H);
    // ... of the tokens before them in the warp (with 16 lanes a token: the other half's), and of all of the warp's
    float before_A[VEC], before_H[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      before_A[i] = 1.f;
      before_H[i] = 0.f;
      if (LANES == 16) {
        const float a = __shfl_up_sync(0xffffffffu, A[i], 16), h = __shfl_up_sync(0xffffffffu, H[i], 16);
        if (lane >= 16) {
          before_A[i] = a;
          before_H[i] = h;
          H[i] = rec_step(A[i], h, H[i]);
          A[i] = rec_joined(A[i], a);
        }
      }
    }
    if (lane >= 32 - LANES)
#pragma unroll
      for (int i = 0; i < VEC; ++i) warp_map[warp][column * VEC + i] = make_float2(A[i], H[i]);
    __syncthreads();
    if (ranks > 1) {
      if (tid < COLS) {
        float2 m = warp_map[0][tid];
#pragma unroll
        for (int w = 1; w < REC_WARPS; ++w) {
          const float2 n = warp_map[w][tid];
          m = make_float2(rec_joined(n.x, m.x), rec_step(n.x, m.y, n.y));
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
          behind = rec_step(m.x, behind, m.y);
        }
      }
#pragma unroll
      for (int w = 0; w < REC_WARPS; ++w) {
        entering[w][tid] = state;
        const float2 m = warp_map[w][tid];
        state = rec_step(m.x, state, m.y);
      }
      carry = ranks > 1 ? behind : state;
    }
    __syncthreads();
    float state[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) state[i] = rec_step(before_A[i], entering[warp][column * VEC + i], before_H[i]);
    apply(in, gate, state, op, dap, h0, count, p.T - s);
    move(op);
    if (BACK) move(dap);
  }
  pdl_trigger();      // not before: CTAs of the next launch would take places that these are laid out for
  if (p.end && rank == 0 && joins) p.end[row] = carry;
}

constexpr int64_t REC_NEAR = (int64_t)1 << 24;   // elements between two of a tile's 128 tokens, where 32 bits hold a tile

// Whether a thread takes a sequence by itself.  Its time grows with T by itself, that of tiles with the waves of CTAs (a CTA takes 64
// channels of a sequence, REC_CTAS run at once).  2048 channels of bf16, tiles against threads, in us, forward and backward:
//   1 sequence   (1 wave)     8 tokens  2.5, 3.1  1.7, 2.2      64 tokens  2.6, 2.7  5.2, 8.8
//   32           (4 waves)   32 tokens  8.6, 9.2  4.5, 6.9     128 tokens   13, 18    14, 33
//   512         (56 waves)   64 tokens  151, 207   66, 115     256 tokens  325, 448  256, 456
bool rec_sequential(const RecArgs& a, int batch, bool back) {
  const int64_t columns = (a.channels + 63) / 64, waves = (columns * batch + REC_CTAS - 1) / REC_CTAS;
  const int64_t most = (back ? 8 : 16) * waves, cap = back ? 128 : 256;
  return a.T <= (most < cap ? most : cap);
}

template <typename TX, typename TA, int VEC, int LANES, int STEPS, bool BACK, typename OFF>
cudaError_t launch(const RecArgs& a, int batch, cudaStream_t st) {
  constexpr int COLS = LANES * VEC, TILE = REC_THREADS / LANES * STEPS;
  const int64_t columns = (a.channels + COLS - 1) / COLS, tiles = (a.T + TILE - 1) / TILE;
  const auto kernel = recurrence_kernel<TX, TA, VEC, LANES, STEPS, BACK, OFF>;
  static RecRoom room;
  const unsigned ranks = rec_ranks(room, kernel, 0, columns, batch, tiles);
  return smat_launch_pdl_cluster(kernel, dim3(ranks, (unsigned)columns, (unsigned)batch), REC_THREADS, 0, ranks, st, a);
}

template <typename TX, typename TA, int VEC, bool BACK>
cudaError_t launch_sequential(const RecArgs& a, int batch, cudaStream_t st) {
  constexpr int STEPS = BACK || sizeof(TX) + sizeof(TA) > 4 ? 4 : 8;      // as many as registers hold twice
  const uint32_t pieces = (uint32_t)((a.channels + VEC - 1) / VEC);
  const dim3 grid((pieces + SEQ_THREADS - 1) / SEQ_THREADS, (unsigned)batch);
  // Few tokens: with fewer registers more threads run at once (512 sequences of 4 tokens 4.5 us, with STEPS 8.2).
  if (a.T <= 4) return smat_launch_pdl(recurrence_sequential_kernel<TX, TA, VEC, 2, BACK>, grid, SEQ_THREADS, 0, st, a, pieces);
  return smat_launch_pdl(recurrence_sequential_kernel<TX, TA, VEC, STEPS, BACK>, grid, SEQ_THREADS, 0, st, a, pieces);
}

template <bool BACK>
cudaError_t dispatch(const RecArgs& a, const smat_recurrence_problem* p, bool wide, cudaStream_t st) {
  const int x_bf16 = p->dtype == SMAT_BF16, gate_bf16 = p->gate_dtype == SMAT_BF16;
  using bf16 = __nv_bfloat16;
  if (rec_sequential(a, p->batch, BACK)) {
    if (p->dtype == SMAT_F32)
      return wide ? launch_sequential<float, float, 4, BACK>(a, p->batch, st) : launch_sequential<float, float, 1, BACK>(a, p->batch, st);
    if (gate_bf16) return wide ? launch_sequential<bf16, bf16, 4, BACK>(a, p->batch, st) : launch_sequential<bf16, bf16, 1, BACK>(a, p->batch, st);
    return wide ? launch_sequential<bf16, float, 4, BACK>(a, p->batch, st) : launch_sequential<bf16, float, 1, BACK>(a, p->batch, st);
  }
  if (smat_recurrence_tma_supported(a, p->batch, x_bf16, gate_bf16, BACK))
    return smat_launch_recurrence_tma(a, p->batch, x_bf16, gate_bf16, BACK, st);
  constexpr int S = BACK ? 4 : 8;
  if (p->dtype == SMAT_F32)
    return wide ? launch<float, float, 4, 16, 4, BACK, uint32_t>(a, p->batch, st) : launch<float, float, 1, 32, S, BACK, uint64_t>(a, p->batch, st);
  if (gate_bf16)
    return wide ? launch<bf16, bf16, 4, 16, S, BACK, uint32_t>(a, p->batch, st) : launch<bf16, bf16, 1, 32, S, BACK, uint64_t>(a, p->batch, st);
  return wide ? launch<bf16, float, 4, 16, 4, BACK, uint32_t>(a, p->batch, st) : launch<bf16, float, 1, 32, S, BACK, uint64_t>(a, p->batch, st);
}

struct Operand {
  const smat_rows* rows;
  smat_dtype dtype;
  bool output;
};
// wide: four channels at a time everywhere (8 bytes of bf16, 16 of fp32), and the tokens of a tile within 2^31 elements.
template <int N>
smat_status check(const smat_recurrence_problem* p, const Operand (&ops)[N], const float* const (&states)[3], bool* wide) {
  if (!p) return SMAT_ERR_NULL;
  for (const Operand& o : ops)
    if (!o.rows || !o.rows->data) return SMAT_ERR_NULL;
  if ((p->dtype != SMAT_F32 && p->dtype != SMAT_BF16) || (p->gate_dtype != p->dtype && p->gate_dtype != SMAT_F32))
    return SMAT_ERR_DTYPE;
  if (p->batch < 1 || p->batch > 65535 || p->T < 1 || p->T > ((int64_t)1 << 40) || p->channels < 1 || p->channels > (1 << 20))
    return SMAT_ERR_SHAPE;
  *wide = p->channels % 4 == 0;
  for (const Operand& o : ops)
    if (!rows_ok(o.rows, p->batch, 1, p->T, p->channels, o.output)) return SMAT_ERR_SHAPE;
  for (const Operand& o : ops) {
    if (rows_misaligned(o.rows, o.dtype)) return SMAT_ERR_ALIGN;
    *wide = *wide && rows_at_multiples(o.rows, o.dtype, p->batch, 1, p->T, 4 * dtype_bytes(o.dtype)) && o.rows->token <= REC_NEAR;
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
