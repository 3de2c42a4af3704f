// The recurrence of long sequences whose tiles move by TMA (see smat_recurrence.cu for how tiles, warps and threads are joined).
//
// A tile is COLS channels of GROUPS * STEPS tokens of every operand, in one stage of a ring in shared memory; outputs take the place of
// the inputs there and leave by TMA too.  A group of COLS / 2 threads has STEPS tokens of it, a thread two channels of these: it forms
// their map, and goes over them again from the state that enters them.  So loads and stores cost a thread one instruction of a fixed offset a
// token, where their addresses had taken a third of all it issued, and the next tiles are on their way without registers.
// Tokens behind the end, and channels beyond the last, are read as zeros: x = 0 and log_a = 0 leave the state as it is.  A
// backward pass goes over the same tiles from the last to the first, and reads h one token before dh.
//
// The CTAs of a cluster exchange the maps of their tiles by stores into one another's shared memory that complete on the reader's
// mbarrier (a cluster barrier a round, which waits for all of a CTA's writes, was the longest stall).  They are formed a round
// ahead, so that a round hides their way.  What sends the map of round n + 1 comes after a barrier behind all reads of those of
// round n - 1, which lay in the same buffer, and after the maps of round n have come from all others: two buffers are enough.
//
// Bound by what a round issues and waits for: 64 K tokens of 2048 bf16 channels (256 CTAs, eight to a cluster) take 155 to 160 us, by
// the GPU, where their bytes take 122 (0.76 to 0.79 of the measured copy rate), gradients of 4 x 8 K with fp32 gates 168 of 143 (0.85);
// without TMA, maps a round ahead and pairs of channels the first took 233 us.
#include <type_traits>

#include "smat_recurrence.cuh"
#include "smat_tc.cuh"

namespace {

namespace cg = cooperative_groups;

constexpr int VEC = 2;
constexpr int PORTER = REC_THREADS - 32;      // the thread that issues copies
constexpr long long WAIT_LIMIT = 4000000000LL;   // SM clock cycles before a wait gives up

template <typename TX, typename TA, int COLS, int STEPS, bool BACK>
struct Tile {
  static constexpr int GROUPS = REC_THREADS * VEC / COLS, TOKENS = GROUPS * STEPS;
  static constexpr uint32_t X = TOKENS * COLS * sizeof(TX), A = TOKENS * COLS * sizeof(TA);
  static constexpr uint32_t BYTES = X + A + (BACK ? X : 0);
  static constexpr uint32_t A_AT = X, H_AT = X + A;
};

// Waits are given up after about two seconds.  `lost` keeps a thread's later waits short, and what follows is NaN: a tile that has not
// come has the map of NaN, and states whose maps have not come are NaN.  A CTA in which a thread has given up (`gave_up`, read behind the round's
// barrier) asks for no more tiles and sends no more maps, for a barrier whose phase is open cannot be armed again and the others may
// still read the buffer that the next maps go to; so the others give up too.  At the end the cluster meets: no CTA leaves while
// another may still send to its shared memory.
__device__ __forceinline__ void wait(uint64_t* bar, uint32_t parity, bool& lost) {
  if (tc::mbar_try_wait(bar, parity)) return;
  const long long start = clock64();
  while (!lost && !tc::mbar_try_wait(bar, parity)) lost = clock64() - start > WAIT_LIMIT;
}
// The same for what other CTAs of the cluster have sent.
__device__ __forceinline__ bool try_wait_sent(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n.reg .pred p;\n"
      "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n"
      "selp.u32 %0, 1, 0, p;\n}\n"
      : "=r"(ok) : "r"(tc::smem_u32(bar)), "r"(parity) : "memory");
  return ok != 0;
}
__device__ __forceinline__ void wait_sent(uint64_t* bar, uint32_t parity, bool& lost) {
  if (try_wait_sent(bar, parity)) return;
  const long long start = clock64();
  while (!lost && !try_wait_sent(bar, parity)) lost = clock64() - start > WAIT_LIMIT;
}

// An address of this CTA's shared memory in that of another of the cluster.
__device__ __forceinline__ uint32_t in_rank(const void* p, int rank) {
  uint32_t a;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(tc::smem_u32(p)), "r"(rank));
  return a;
}
__device__ __forceinline__ void send(uint32_t to, uint32_t bar, float2 v) {
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%2, %3}, [%1];" ::"r"(to), "r"(bar), "f"(v.x), "f"(v.y)
               : "memory");
}

__device__ __forceinline__ void store_tile(const CUtensorMap* map, const void* from, int x, int y, int z) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];"
               ::"l"(map), "r"(tc::smem_u32(from)), "r"(x), "r"(y), "r"(z) : "memory");
}

// Two channels of a token in shared memory.
template <typename T>
__device__ __forceinline__ RowVec<T, VEC> load_piece(const char* p) {
  RowVec<T, VEC> v;
  if constexpr (sizeof(T) == 2) {
    v.w[0] = *reinterpret_cast<const uint32_t*>(p);
  } else {
    const uint2 w = *reinterpret_cast<const uint2*>(p);
    v.w[0] = w.x; v.w[1] = w.y;
  }
  return v;
}
template <typename T>
__device__ __forceinline__ void store_piece(float2 f, char* p) {
  RowVec<T, VEC> v;
  const float flat[2] = {f.x, f.y};
  v.set(flat);
  v.store(reinterpret_cast<T*>(p));
}
template <typename T>
__device__ __forceinline__ float2 pair(const RowVec<T, VEC>& v) { return make_float2(v.get(0), v.get(1)); }
__device__ __forceinline__ float2 closed_step(float2 a, float2 s, float2 x) {
  return make_float2(rec_step(a.x, s.x, x.x), rec_step(a.y, s.y, x.y));
}
__device__ __forceinline__ float2 unless_closed(float2 a, float2 v) { return make_float2(a.x == 0.f ? 0.f : v.x, a.y == 0.f ? 0.f : v.y); }

// exp of the log-gates.  From -4 up, 2^(x log2 e) with one rounding of the exponent, which is off by 2^-22 there, and the power by 2^-22
// of itself; below, where the rounded exponent would cost more, expf.
template <typename T, int STEPS>
__device__ __forceinline__ void open_gates(const RowVec<T, VEC> (&a)[STEPS], float2 (&gate)[STEPS]) {
  bool near;
  if constexpr (sizeof(T) == 2) {
    __nv_bfloat162 least = __floats2bfloat162_rn(0.f, 0.f);
#pragma unroll
    for (int l = 0; l < STEPS; ++l) least = __hmin2(least, *reinterpret_cast<const __nv_bfloat162*>(&a[l].w[0]));
    near = fminf(__low2float(least), __high2float(least)) >= -4.f;
  } else {
    float least = 0.f;
#pragma unroll
    for (int l = 0; l < STEPS; ++l) least = fminf(least, fminf(a[l].get(0), a[l].get(1)));
    near = least >= -4.f;
  }
  if (near) {
#pragma unroll
    for (int l = 0; l < STEPS; ++l) {
      gate[l] = __fmul2_rn(pair(a[l]), make_float2(1.4426950408889634f, 1.4426950408889634f));
      asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(gate[l].x));
      asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(gate[l].y));
    }
  } else {
#pragma unroll
    for (int l = 0; l < STEPS; ++l) gate[l] = make_float2(expf(a[l].get(0)), expf(a[l].get(1)));
  }
}

struct Maps {
  CUtensorMap x, log_a, h, out, dlog_a;
};

template <typename TX, typename TA, int COLS, int STEPS, int STAGES, bool BACK>
__global__ void __launch_bounds__(REC_THREADS, 2) recurrence_tma_kernel(const __grid_constant__ Maps maps, const float* begin, const float* h0,
                                                                        float* end, int T, int channels) {
  using Shape = Tile<TX, TA, COLS, STEPS, BACK>;
  static_assert(STAGES >= 4, "a round's tile is asked for two rounds before its map is formed, one round ahead");
  static_assert(COLS <= REC_THREADS / 4 && 32 * VEC % COLS == 0, "one thread joins the states of a channel, one of another warp sends its map");
  constexpr int GROUPS = Shape::GROUPS;
  extern __shared__ __align__(128) char stages[];
  __shared__ __align__(16) float2 group_map[2][GROUPS][COLS];       // (A, H) of a group's tokens, of this round and of the next
  __shared__ __align__(16) float entering[2][GROUPS][COLS];         // the state that enters a group's tokens
  __shared__ __align__(8) float2 tile_map[2][REC_MAX_CLUSTER][COLS];
  __shared__ uint64_t full[STAGES], maps_in[2];
  __shared__ volatile int gave_up;
  const cg::cluster_group cluster = cg::this_cluster();
  const int ranks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int tid = threadIdx.x, lane = tid % (COLS / VEC), group = tid / (COLS / VEC);
  const int channel = tid % COLS;      // whose states or maps this thread joins
  const bool joins = tid < COLS, sends = tid >= REC_THREADS / 2 && tid < REC_THREADS / 2 + COLS;
  const int b = blockIdx.z, c0 = blockIdx.y * COLS;
  if (tid == 0) {
    for (int i = 0; i < STAGES; ++i) tc::mbar_init(&full[i], 1);
    tc::mbar_init(&maps_in[0], 1);
    tc::mbar_init(&maps_in[1], 1);
    tc::fence_barrier_init();
    gave_up = 0;
  }
  if (ranks > 1) cluster.sync();      // all of the cluster run, with their barriers ready, before one sends to another
  else __syncthreads();
  pdl_wait();
  const int tiles = (T + Shape::TOKENS - 1) / Shape::TOKENS, rounds = (tiles + ranks - 1) / ranks;
  // this CTA's tile of a round is number round * ranks + rank in the order of the recurrence; the last round may have none for it
  const int own_rounds = (tiles - rank + ranks - 1) / ranks;
  const auto token_of = [&](int round) { return (BACK ? tiles - 1 - (round * ranks + rank) : round * ranks + rank) * Shape::TOKENS; };
  int asked = 0;      // of the thread that issues copies: tiles so far
  const auto fetch = [&](int round) {
    if (round >= own_rounds) return;
    asked = round + 1;
    char* to = stages + (round % STAGES) * Shape::BYTES;
    uint64_t* bar = &full[round % STAGES];
    const int t = token_of(round);
    tc::mbar_expect_tx(bar, Shape::BYTES);
    tc::tma_load_3d(to, &maps.x, c0, t, b, bar);
    tc::tma_load_3d(to + Shape::A_AT, &maps.log_a, c0, t, b, bar);
    if (BACK) tc::tma_load_3d(to + Shape::H_AT, &maps.h, c0, t - 1, b, bar);
  };
  const auto put = [&](int round) {      // the outputs of a round, once all threads have written them
    if (round < own_rounds) {
      const char* from = stages + (round % STAGES) * Shape::BYTES;
      store_tile(&maps.out, from, c0, token_of(round), b);
      if (BACK) store_tile(&maps.dlog_a, from + Shape::A_AT, c0, token_of(round), b);
    }
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
  };
  if (tid == PORTER)
    for (int r = 0; r < STAGES; ++r) fetch(r);

  const bool mine = c0 + channel < channels;
  const int64_t row = (int64_t)b * channels + c0;
  float carry = joins && mine && begin ? begin[row + channel] : 0.f;
  bool lost = false;
  // this thread's first token (in the order of the recurrence) in a tile, and from one to the next
  const int place = (BACK ? Shape::TOKENS - 1 - group * STEPS : group * STEPS) * COLS + lane * VEC;
  constexpr int WAY = BACK ? -COLS : COLS;

  // A thread's tokens of a round: gates and rows from the time that their map is formed until they are gone over again.
  struct Tokens {
    float2 gate[STEPS];
    RowVec<TX, VEC> x[STEPS];
  };
  // The states behind a thread's tokens, from `state` on: put(l, what leaves as the output, the state behind the token) for each.
  // Backward the output v_t = x_t + c_{t+1} is carried instead of the state c_t = a_t v_t, so that a token is one fused product and sum
  // either way, and the values behind a closed gate are the same, bit for bit, whatever came before it.
  const auto states = [](const Tokens& k, auto closed, float2 state, auto put) {
    constexpr bool CLOSED = decltype(closed)::value;
    [[maybe_unused]] float2 v = state;
#pragma unroll
    for (int l = 0; l < STEPS; ++l) {
      const float2 x = pair(k.x[l]);
      if constexpr (BACK) {
        if (l == 0) v = __fadd2_rn(x, state);
        else v = CLOSED ? closed_step(k.gate[l - 1], v, x) : __ffma2_rn(k.gate[l - 1], v, x);
        state = __fmul2_rn(k.gate[l], v);
        if (CLOSED) state = unless_closed(k.gate[l], state);
        put(l, v, state);
      } else {
        state = CLOSED ? closed_step(k.gate[l], state, x) : __ffma2_rn(k.gate[l], state, x);
        put(l, state, state);
      }
    }
    return state;
  };
  const auto form = [&](int round, int stage, uint32_t phase, Tokens& k) {
    float2 A = make_float2(1.f, 1.f), H = make_float2(0.f, 0.f);
    if (round < own_rounds) {
      wait(&full[stage], phase, lost);
      const char* xs = stages + stage * Shape::BYTES + place * sizeof(TX);
      const char* as = stages + stage * Shape::BYTES + Shape::A_AT + place * sizeof(TA);
      RowVec<TA, VEC> a[STEPS];
#pragma unroll
      for (int l = 0; l < STEPS; ++l) {
        a[l] = load_piece<TA>(as + l * WAY * (int)sizeof(TA));
        k.x[l] = load_piece<TX>(xs + l * WAY * (int)sizeof(TX));
      }
      open_gates(a, k.gate);
#pragma unroll
      for (int l = 0; l < STEPS; ++l) A = __fmul2_rn(A, k.gate[l]);
      if (!(A.x > 0.f && A.y > 0.f)) {
        float2 least = k.gate[0];
#pragma unroll
        for (int l = 1; l < STEPS; ++l) least = make_float2(fminf(least.x, k.gate[l].x), fminf(least.y, k.gate[l].y));
        A = make_float2(rec_factor(A.x, least.x), rec_factor(A.y, least.y));
      }
      const auto nothing = [](int, float2, float2) {};
      H = states(k, std::false_type(), make_float2(0.f, 0.f), nothing);
      if (rec_not_finite(fmaf(H.x, 0.f, H.y * 0.f))) H = states(k, std::true_type(), make_float2(0.f, 0.f), nothing);
      if (lost) {
        gave_up = 1;
        H = make_float2(NAN, NAN);
      }
    }
    *reinterpret_cast<float4*>(&group_map[round & 1][group][lane * VEC]) = make_float4(A.x, H.x, A.y, H.y);
  };
  // This CTA's map of a round to all ranks.  (It is what all threads issue together that counts: with the maps and states of a channel
  // joined by two threads each, or by four in all warps alike, 64 K tokens took 171 and 188 us.)
  const auto publish = [&](int round) {
    if (!sends || ranks == 1) return;
    const int turn = round & 1, stop = gave_up;
    float2 m = group_map[turn][0][channel];
#pragma unroll
    for (int w = 1; w < GROUPS; ++w) {
      const float2 n = group_map[turn][w][channel];
      m = make_float2(rec_joined(n.x, m.x), rec_step(n.x, m.y, n.y));
    }
    if (stop) return;
    if (channel == 0) tc::mbar_expect_tx(&maps_in[turn], ranks * COLS * sizeof(float2));
    for (int r = 0; r < ranks; ++r) send(in_rank(&tile_map[turn][rank][channel], r), in_rank(&maps_in[turn], r), m);
  };
  // The states that enter the warps' tokens; the maps of a round have been on their way for a round.
  const auto enter = [&](int round) {
    if (!joins) return;
    const int turn = round & 1;
    float state = carry;
    if (ranks > 1) {
      wait_sent(&maps_in[turn], (round >> 1) & 1, lost);
      float behind = carry;
#pragma unroll
      for (int r = 0; r < REC_MAX_CLUSTER; ++r) {
        if (r >= ranks) break;
        if (r == rank) state = behind;
        const float2 m = tile_map[turn][r][channel];
        behind = rec_step(m.x, behind, m.y);
      }
      carry = behind;
      if (lost) {
        gave_up = 1;
        state = carry = NAN;
      }
    }
    // (eight maps at a time ahead of the stores, which the compiler does not move them across)
#pragma unroll
    for (int w = 0; w < GROUPS; w += 8) {
      float2 m[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) m[i] = group_map[turn][w + i][channel];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        entering[turn][w + i][channel] = state;
        state = rec_step(m[i].x, state, m[i].y);
      }
    }
    if (ranks == 1) carry = state;
  };
  // A round's tokens again, from the state that enters them.
  const auto apply = [&](int round, char* stage, const Tokens& k) {
    if (round >= own_rounds) return;
    char* xs = stage + place * sizeof(TX);
    char* as = stage + Shape::A_AT + place * sizeof(TA);
    const char* hs = stage + Shape::H_AT + place * sizeof(TX);
    const float2 from = *reinterpret_cast<const float2*>(&entering[round & 1][group][lane * VEC]);
    const bool first = BACK && token_of(round) == 0 && group == GROUPS - 1;      // token 0 is this thread's last
    const auto go = [&](auto closed) {
      [[maybe_unused]] constexpr bool CLOSED = decltype(closed)::value;
      const float2 none = make_float2(0.f, 0.f);
      float2 zeros = none;
      const float2 behind = states(k, closed, from, [&](int l, float2 out, float2 state) {
        store_piece<TX>(out, xs + l * WAY * (int)sizeof(TX));
        if constexpr (BACK) {
          float2 before = pair(load_piece<TX>(hs + l * WAY * (int)sizeof(TX)));
          if (l == STEPS - 1 && first && h0) {
            const int c = lane * VEC;
            before = make_float2(c0 + c < channels ? h0[row + c] : 0.f, c0 + c + 1 < channels ? h0[row + c + 1] : 0.f);
          }
          float2 d = __fmul2_rn(state, before);
          if (CLOSED) d = unless_closed(k.gate[l], d);
          else zeros = __ffma2_rn(d, none, zeros);
          store_piece<TA>(d, as + l * WAY * (int)sizeof(TA));
        }
      });
      zeros = __ffma2_rn(behind, none, zeros);
      return zeros.x + zeros.y;
    };
    if (rec_not_finite(go(std::false_type()))) go(std::true_type());
    tc::fence_proxy_async();      // seen by the copy that takes the tile away
  };
  // the stage of the round whose tokens are gone over, and the parity in which the next one's tile comes
  int at = 0;
  uint32_t phase = 0;
  const auto step = [&](int round, const Tokens& now, Tokens& next) {
    char* stage = stages + at * Shape::BYTES;
    at = at + 1 == STAGES ? 0 : at + 1;
    phase ^= at == 0;
    // (forward, and with maps of more ranks to come, the states wait until the next maps are formed: 64 K tokens on eight ranks 179 to
    // 172 us, gradients of 32 K 172 to 136; gradients of one or two ranks take 167 us this way and 179 the other)
    const bool states_first = BACK && ranks <= 2;
    if (states_first) enter(round);
    if (round + 1 < rounds) form(round + 1, at, phase, next);
    if (!states_first) enter(round);
    __syncthreads();
    if (tid == PORTER && round > 0) {
      put(round - 1);
      if (round > 1) {
        asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");      // the outputs of round - 2 have been taken away
        if (!gave_up) fetch(round - 2 + STAGES);
      }
    }
    if (round + 1 < rounds) publish(round + 1);
    apply(round, stage, now);
  };

  Tokens even, odd;
  form(0, 0, 0, even);
  __syncthreads();
  publish(0);
  for (int round = 0; round < rounds; round += 2) {
    step(round, even, odd);
    if (round + 1 < rounds) step(round + 1, odd, even);
  }
  // (the barrier before the trigger: behind it CTAs of the next launch take places as those of a cluster leave one by one, and 64 K tokens
  // of 512 channels took 57 us for 50)
  if (ranks > 1) asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");
  __syncthreads();
  if (tid == PORTER) {
    put(rounds - 1);
    asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  }
  if (end && rank == 0 && mine && tid < COLS) end[row + tid] = carry;
  if (ranks > 1) asm volatile("barrier.cluster.wait;" ::: "memory");
  pdl_trigger();      // not before: CTAs of the next launch would take places that these are laid out for
  if (tid == PORTER && gave_up) {
    // tiles that were waited for in vain land before the CTA leaves, or not within the limit; so do maps that the others sent before
    // they came here (a microsecond)
    for (int r = asked > STAGES ? asked - STAGES : 0; r < asked; ++r) {
      bool late = false;
      wait(&full[r % STAGES], (r / STAGES) & 1, late);
    }
    for (const long long start = clock64(); clock64() - start < 1000000;) {}
  }
}

template <typename TX, typename TA, int COLS, int STEPS, int STAGES, bool BACK>
cudaError_t launch(const RecArgs& a, int batch, cudaStream_t st) {
  using Shape = Tile<TX, TA, COLS, STEPS, BACK>;
  Maps maps{};
  const auto make = [&](CUtensorMap* m, const void* data, const RowStride& s, int bytes) {
    return smat_make_map_rows(m, data, bytes, (uint64_t)a.channels, (uint64_t)a.T, (uint64_t)batch, (uint64_t)s.token * bytes,
                              (uint64_t)(batch > 1 ? s.batch : s.token) * bytes, COLS, Shape::TOKENS);
  };
  if (!make(&maps.x, a.x, a.xs, sizeof(TX)) || !make(&maps.log_a, a.log_a, a.as, sizeof(TA)) || !make(&maps.out, a.out, a.os, sizeof(TX)))
    return cudaErrorInvalidValue;
  if (BACK && (!make(&maps.h, a.h, a.hs, sizeof(TX)) || !make(&maps.dlog_a, a.dlog_a, a.das, sizeof(TA)))) return cudaErrorInvalidValue;
  const auto kernel = recurrence_tma_kernel<TX, TA, COLS, STEPS, STAGES, BACK>;
  constexpr size_t bytes = (size_t)STAGES * Shape::BYTES;
  const cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  if (err != cudaSuccess) return err;
  const int64_t columns = (a.channels + COLS - 1) / COLS, tiles = (a.T + Shape::TOKENS - 1) / Shape::TOKENS;
  static RecRoom room;
  const unsigned ranks = rec_ranks(room, kernel, bytes, columns, batch, tiles);
  return smat_launch_pdl_cluster(kernel, dim3(ranks, (unsigned)columns, (unsigned)batch), REC_THREADS, bytes, ranks, st, maps, a.begin, a.h0, a.end,
                                 (int)a.T, a.channels);
}

template <typename TX, typename TA, int STEPS, int STAGES, bool BACK>
cudaError_t narrow(const RecArgs& a, int batch, int cols, cudaStream_t st) {
  static_assert(STEPS % 2 == 1, "the groups of a warp read different banks");
  return cols == 32 ? launch<TX, TA, 32, STEPS, STAGES, BACK>(a, batch, st) : launch<TX, TA, 16, STEPS, STAGES, BACK>(a, batch, st);
}

// Channels of a tile.  A long sequence of few channels leaves SMs idle with 64 (a line of bf16): with 32 or 16, whose rows are half and a
// quarter of a line, a CTA has two and four times as many tokens a tile, and more CTAs run.  16 K tokens of bf16, forward and backward,
// in us, with 64, 32, 16:   512 channels  29, 42   23, 32   16, 23        704 channels  29, 45   24, 34   20, 28
//                          1024 channels  37, 54   25, 34   27, 37       1728 channels  41, 61   35, 50   45, 79
//                          2048 channels  43, 66   42, 61   46, 79,
// and 512 tokens of 512 channels 3.0, 3.9   2.9, 3.3   3.3, 3.5.  (fp32: 704 channels 59, 80   43, 55   33, 45; 2048  78, 117   74, 115
// 81, 118.)
int rec_cols(const RecArgs& a, int batch) {
  const int64_t columns = (a.channels + 63) / 64 * batch;
  return a.T < 2048 || columns > 28 ? 64 : columns > 11 ? 32 : 16;
}

}  // namespace

bool smat_recurrence_tma_supported(const RecArgs& a, int batch, int x_bf16, int gate_bf16, bool back) {
  if (a.T > (1 << 30)) return false;      // coordinates of tokens
  const auto fits = [&](const void* data, const RowStride& s, int bytes) {
    uint64_t bits = reinterpret_cast<uintptr_t>(data) | (uint64_t)(s.token * bytes);
    if (batch > 1) bits |= (uint64_t)(s.batch * bytes);
    const int64_t most = (int64_t)1 << 36;
    return (bits & 15) == 0 && s.token >= a.channels && s.token < most && (batch == 1 || (s.batch > 0 && s.batch < most));
  };
  const int x = x_bf16 ? 2 : 4, g = gate_bf16 ? 2 : 4;
  // A store ends at a multiple of 16 bytes, not at the row's last element: rows of 13 bf16 channels, 16 apart, had zeros written behind each.
  if (a.channels * x % 16 != 0 || (back && a.channels * g % 16 != 0)) return false;
  return fits(a.x, a.xs, x) && fits(a.log_a, a.as, g) && fits(a.out, a.os, x) && (!back || (fits(a.h, a.hs, x) && fits(a.dlog_a, a.das, g)));
}

// Tokens of a thread and stages: as many as two CTAs an SM have room for, and five stages or more (with four a tile comes late: gradients
// of 64 K tokens with fp32 gates 341 us with <4, 5>, 461 with <5, 4>).  In between, more tokens a round pay where eight CTAs hand the
// states on (32 K of fp32: <4, 5> 158 us, <3, 7> 168; gradients <2, 7> 264, <3, 5> 220), more stages where one or two do (4 x 8 K: 149 and
// 138).  (One CTA an SM with tiles three times as long issues half the instructions a token, but eight warps do not hide their
// latency: 64 K tokens 260 us.)
cudaError_t smat_launch_recurrence_tma(const RecArgs& a, int batch, int x_bf16, int gate_bf16, bool back, cudaStream_t st) {
  using bf16 = __nv_bfloat16;
  const int cols = rec_cols(a, batch);
  if (cols < 64) {
    if (!x_bf16) return back ? narrow<float, float, 3, 5, true>(a, batch, cols, st) : narrow<float, float, 3, 7, false>(a, batch, cols, st);
    if (gate_bf16) return back ? narrow<bf16, bf16, 5, 6, true>(a, batch, cols, st) : narrow<bf16, bf16, 7, 6, false>(a, batch, cols, st);
    return back ? narrow<bf16, float, 3, 7, true>(a, batch, cols, st) : narrow<bf16, float, 5, 6, false>(a, batch, cols, st);
  }
  if (!x_bf16) {
    if (back) return launch<float, float, 64, 3, 5, true>(a, batch, st);
    const int64_t columns = (a.channels + 63) / 64;
    return columns * batch * 4 > REC_CTAS ? launch<float, float, 64, 3, 7, false>(a, batch, st) : launch<float, float, 64, 4, 5, false>(a, batch, st);
  }
  if (gate_bf16) return back ? launch<bf16, bf16, 64, 6, 5, true>(a, batch, st) : launch<bf16, bf16, 64, 9, 5, false>(a, batch, st);
  return back ? launch<bf16, float, 64, 4, 5, true>(a, batch, st) : launch<bf16, float, 64, 6, 5, false>(a, batch, st);
}
