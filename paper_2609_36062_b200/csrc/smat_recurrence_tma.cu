// The recurrence of long sequences whose tiles move by TMA (see smat_recurrence.cu for how tiles, warps and threads are joined).
//
// A tile is 64 channels of 16 * STEPS tokens of every operand, in one stage of a ring in shared memory; outputs take the place of
// the inputs there and leave by TMA too.  A thread has four channels of STEPS tokens: it forms their map, and goes over
// them again from the state that enters them.  So loads and stores cost a thread one instruction of a fixed offset a token,
// where their addresses had taken a third of all it issued, and the next tiles are on their way without registers.  Tokens behind
// the end, and channels beyond the last, are read as zeros: x = 0 and log_a = 0 leave the state as it is.  A backward pass goes
// over the same tiles from the last to the first, and reads h one token before dh.
//
// The CTAs of a cluster exchange the maps of their tiles by stores into one another's shared memory that complete on the reader's
// mbarrier.  (A cluster barrier a round, which waits for all of a CTA's writes, was the longest stall.)  A rank that sends the map
// of round n + 1 has read those of round n, so two buffers are enough.
#include "smat_recurrence.cuh"
#include <type_traits>

#include "smat_tc.cuh"

namespace {

namespace cg = cooperative_groups;

constexpr int COLS = 64, VEC = 4, LANES = COLS / VEC, PARTS = REC_THREADS / LANES;
constexpr int PORTER = REC_THREADS - 32;      // the thread that issues copies: not of the warps that join maps
constexpr long long WAIT_LIMIT = 4000000000LL;   // SM clock cycles before a wait gives up

template <typename TX, typename TA, int STEPS, bool BACK>
struct Tile {
  static constexpr int TOKENS = PARTS * STEPS;
  static constexpr uint32_t X = TOKENS * COLS * sizeof(TX), A = TOKENS * COLS * sizeof(TA);
  static constexpr uint32_t BYTES = X + A + (BACK ? X : 0);
  static constexpr uint32_t A_AT = X, H_AT = X + A;
};

// Gives up after about two seconds.  What follows from a tile that has not come is NaN; `lost` keeps later waits short.
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

__device__ __forceinline__ void send(void* to, int rank, uint64_t* bar, float2 v) {
  asm volatile(
      "{\n.reg .b32 a, b;\n"
      "mapa.shared::cluster.u32 a, %0, %2;\n"
      "mapa.shared::cluster.u32 b, %1, %2;\n"
      "st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [a], {%3, %4}, [b];\n}\n"
      ::"r"(tc::smem_u32(to)), "r"(tc::smem_u32(bar)), "r"(rank), "f"(v.x), "f"(v.y) : "memory");
}

__device__ __forceinline__ void store_tile(const CUtensorMap* map, const void* from, int x, int y, int z) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];"
               ::"l"(map), "r"(tc::smem_u32(from)), "r"(x), "r"(y), "r"(z) : "memory");
}

template <typename T>
__device__ __forceinline__ void load_piece(RowVec<T, VEC>& v, const char* p) {
  if constexpr (sizeof(T) == 2) {
    const uint2 w = *reinterpret_cast<const uint2*>(p);
    v.w[0] = w.x; v.w[1] = w.y;
  } else {
    const uint4 w = *reinterpret_cast<const uint4*>(p);
    v.w[0] = w.x; v.w[1] = w.y; v.w[2] = w.z; v.w[3] = w.w;
  }
}
template <typename T>
__device__ __forceinline__ void store_piece(const float2 (&f)[2], char* p) {
  RowVec<T, VEC> v;
  const float flat[4] = {f[0].x, f[0].y, f[1].x, f[1].y};
  v.set(flat);
  v.store(reinterpret_cast<T*>(p));
}
template <typename T>
__device__ __forceinline__ float2 pair(const RowVec<T, VEC>& v, int j) { return make_float2(v.get(2 * j), v.get(2 * j + 1)); }
__device__ __forceinline__ float2 closed_step(float2 a, float2 s, float2 x) {
  return make_float2(rec_step(a.x, s.x, x.x), rec_step(a.y, s.y, x.y));
}
__device__ __forceinline__ float2 unless_closed(float2 a, float2 v) { return make_float2(a.x == 0.f ? 0.f : v.x, a.y == 0.f ? 0.f : v.y); }

struct Maps {
  CUtensorMap x, log_a, h, out, dlog_a;
};

template <typename TX, typename TA, int STEPS, int STAGES, bool BACK>
__global__ void __launch_bounds__(REC_THREADS, 2) recurrence_tma_kernel(const __grid_constant__ Maps maps, const float* begin, const float* h0,
                                                                        float* end, int64_t T, int channels) {
  using Shape = Tile<TX, TA, STEPS, BACK>;
  static_assert(STAGES >= 3, "a round's tile is asked for in an earlier round");
  extern __shared__ __align__(128) char stages[];
  __shared__ __align__(16) float2 warp_map[REC_WARPS][COLS];                  // (A, H) of a warp's tokens
  __shared__ __align__(16) float entering[REC_WARPS][COLS];                   // the state that enters a warp's tokens
  __shared__ __align__(8) float2 tile_map[2][REC_MAX_CLUSTER][COLS];
  __shared__ uint64_t full[STAGES], maps_in[2];
  const cg::cluster_group cluster = cg::this_cluster();
  const int ranks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, column = lane % LANES, part = tid / LANES;
  const int b = blockIdx.z, c0 = blockIdx.y * COLS;
  if (tid == 0) {
    for (int i = 0; i < STAGES; ++i) tc::mbar_init(&full[i], 1);
    tc::mbar_init(&maps_in[0], 1);
    tc::mbar_init(&maps_in[1], 1);
    tc::fence_barrier_init();
  }
  pdl_trigger();
  if (ranks > 1) cluster.sync();      // all of the cluster run, with their barriers ready, before one sends to another
  else __syncthreads();
  pdl_wait();
  const int64_t tiles = (T + Shape::TOKENS - 1) / Shape::TOKENS;
  const int rounds = (int)((tiles + ranks - 1) / ranks);
  // this CTA's tile of a round, by its place in the order of the recurrence; none from `tiles` on
  const auto turn_of = [&](int round) { return (int64_t)round * ranks + rank; };
  const auto token_of = [&](int round) { return (int)((BACK ? tiles - 1 - turn_of(round) : turn_of(round)) * Shape::TOKENS); };
  const auto fetch = [&](int round) {
    if (round >= rounds || turn_of(round) >= tiles) return;
    char* to = stages + (round % STAGES) * Shape::BYTES;
    uint64_t* bar = &full[round % STAGES];
    const int t = token_of(round);
    tc::mbar_expect_tx(bar, Shape::BYTES);
    tc::tma_load_3d(to, &maps.x, c0, t, b, bar);
    tc::tma_load_3d(to + Shape::A_AT, &maps.log_a, c0, t, b, bar);
    if (BACK) tc::tma_load_3d(to + Shape::H_AT, &maps.h, c0, t - 1, b, bar);
  };
  const auto put = [&](int round) {      // the outputs of a round, once all threads have written them
    if (turn_of(round) < tiles) {
      const char* from = stages + (round % STAGES) * Shape::BYTES;
      store_tile(&maps.out, from, c0, token_of(round), b);
      if (BACK) store_tile(&maps.dlog_a, from + Shape::A_AT, c0, token_of(round), b);
    }
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
  };
  if (tid == PORTER)
    for (int r = 0; r < STAGES; ++r) fetch(r);

  const bool joins = tid < COLS, mine = joins && c0 + tid < channels;
  const int64_t row = (int64_t)b * channels + c0;
  float carry = mine && begin ? begin[row + tid] : 0.f;
  bool lost = false;
  // offset of this thread's first token (in the order of the recurrence) in a tile, and from one to the next
  const int place = BACK ? Shape::TOKENS - 1 - part * STEPS : part * STEPS;
  constexpr int WAY = BACK ? -COLS : COLS;
  for (int round = 0; round < rounds; ++round) {
    const bool here = turn_of(round) < tiles;
    char* stage = stages + (round % STAGES) * Shape::BYTES;
    char* xs = stage + (place * COLS + column * VEC) * sizeof(TX);
    char* as = stage + Shape::A_AT + (place * COLS + column * VEC) * sizeof(TA);
    const char* hs = stage + Shape::H_AT + (place * COLS + column * VEC) * sizeof(TX);
    RowVec<TX, VEC> x[STEPS];
    float2 gate[STEPS][2], A[2], H[2];
    A[0] = A[1] = make_float2(1.f, 1.f);
    H[0] = H[1] = make_float2(0.f, 0.f);
    if (here) {
      wait(&full[round % STAGES], (round / STAGES) & 1, lost);
      float least = 0.f;
      RowVec<TA, VEC> a[STEPS];
#pragma unroll
      for (int l = 0; l < STEPS; ++l) {
        load_piece(x[l], xs + l * WAY * (int)sizeof(TX));
        load_piece(a[l], as + l * WAY * (int)sizeof(TA));
      }
      // exp: from -4 up, 2^(x log2 e) with one rounding of the exponent, which is off by 2^-22 there, and the power by 2^-22 of
      // itself; below, where the rounded exponent would cost more, expf
#pragma unroll
      for (int l = 0; l < STEPS; ++l)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float2 v = pair(a[l], j);
          least = fminf(least, fminf(v.x, v.y));
          gate[l][j] = __fmul2_rn(v, make_float2(1.4426950408889634f, 1.4426950408889634f));
          asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(gate[l][j].x));
          asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(gate[l][j].y));
        }
      if (!(least >= -4.f)) {
#pragma unroll
        for (int l = 0; l < STEPS; ++l)
#pragma unroll
          for (int j = 0; j < 2; ++j) gate[l][j] = make_float2(expf(a[l].get(2 * j)), expf(a[l].get(2 * j + 1)));
      }
      // the map of this thread's tokens
#pragma unroll
      for (int l = 0; l < STEPS; ++l)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          A[j] = __fmul2_rn(A[j], gate[l][j]);
          H[j] = BACK ? __fmul2_rn(gate[l][j], __fadd2_rn(H[j], pair(x[l], j))) : __ffma2_rn(gate[l][j], H[j], pair(x[l], j));
        }
      const float zeros = fmaf(H[0].x, 0.f, fmaf(H[0].y, 0.f, fmaf(H[1].x, 0.f, H[1].y * 0.f)));
      if (rec_not_finite(zeros)) {
        H[0] = H[1] = make_float2(0.f, 0.f);
#pragma unroll
        for (int l = 0; l < STEPS; ++l)
#pragma unroll
          for (int j = 0; j < 2; ++j)
            H[j] = BACK ? unless_closed(gate[l][j], __fmul2_rn(gate[l][j], __fadd2_rn(H[j], pair(x[l], j))))
                        : closed_step(gate[l][j], H[j], pair(x[l], j));
      }
      if (lost) H[0] = H[1] = make_float2(NAN, NAN);
    }
    // ... of the other half's tokens before them, and of all of the warp's
    float2 before_A[2], before_H[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const float2 a = make_float2(__shfl_up_sync(0xffffffffu, A[j].x, 16), __shfl_up_sync(0xffffffffu, A[j].y, 16));
      const float2 h = make_float2(__shfl_up_sync(0xffffffffu, H[j].x, 16), __shfl_up_sync(0xffffffffu, H[j].y, 16));
      before_A[j] = lane < 16 ? make_float2(1.f, 1.f) : a;
      before_H[j] = lane < 16 ? make_float2(0.f, 0.f) : h;
      if (lane >= 16) {
        H[j] = closed_step(A[j], h, H[j]);
        A[j] = __fmul2_rn(A[j], a);
        *reinterpret_cast<float4*>(&warp_map[warp][column * VEC + 2 * j]) = make_float4(A[j].x, H[j].x, A[j].y, H[j].y);
      }
    }
    __syncthreads();
    if (tid == PORTER && round > 0) {
      put(round - 1);
      if (round > 1) {
        asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");      // the outputs of round - 2 have been taken away
        fetch(round - 2 + STAGES);
      }
    }
    if (joins) {
      const int turn = round & 1;
      if (ranks > 1) {
        float2 m = warp_map[0][tid];
#pragma unroll
        for (int w = 1; w < REC_WARPS; ++w) {
          const float2 n = warp_map[w][tid];
          m = make_float2(n.x * m.x, rec_step(n.x, m.y, n.y));
        }
        if (tid == 0) tc::mbar_expect_tx(&maps_in[turn], ranks * COLS * sizeof(float2));
        for (int r = 0; r < ranks; ++r) send(&tile_map[turn][rank][tid], r, &maps_in[turn], m);
        wait_sent(&maps_in[turn], (round >> 1) & 1, lost);
        if (lost) carry = NAN;
      }
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
    if (!here) continue;
    // the tokens again, from the state that enters them
    const float4 e = *reinterpret_cast<const float4*>(&entering[warp][column * VEC]);
    float2 state[2] = {closed_step(before_A[0], make_float2(e.x, e.y), before_H[0]), closed_step(before_A[1], make_float2(e.z, e.w), before_H[1])};
    const bool first = BACK && token_of(round) == 0 && part == PARTS - 1;      // token 0 is this thread's last
    const auto go = [&](auto closed) {
      constexpr bool CLOSED = decltype(closed)::value;
      float2 s[2] = {state[0], state[1]}, zeros = make_float2(0.f, 0.f);
      const float2 none = make_float2(0.f, 0.f);
#pragma unroll
      for (int l = 0; l < STEPS; ++l) {
        float2 v[2], d[2];
        RowVec<TX, VEC> h;
        if (BACK) load_piece(h, hs + l * WAY * (int)sizeof(TX));
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float2 a = gate[l][j];
          if (BACK) {
            v[j] = __fadd2_rn(pair(x[l], j), s[j]);                      // dx
            s[j] = __fmul2_rn(a, v[j]);                                  // c
            if (CLOSED) s[j] = unless_closed(a, s[j]);
            float2 before = pair(h, j);
            if (l == STEPS - 1 && first && h0) {
              const int c = column * VEC + 2 * j;
              before = make_float2(c0 + c < channels ? h0[row + c] : 0.f, c0 + c + 1 < channels ? h0[row + c + 1] : 0.f);
            }
            d[j] = __fmul2_rn(s[j], before);
            if (CLOSED) d[j] = unless_closed(a, d[j]);
            else zeros = __ffma2_rn(d[j], none, zeros);
          } else {
            v[j] = s[j] = CLOSED ? closed_step(a, s[j], pair(x[l], j)) : __ffma2_rn(a, s[j], pair(x[l], j));
          }
        }
        store_piece<TX>(v, xs + l * WAY * (int)sizeof(TX));
        if constexpr (BACK) store_piece<TA>(d, as + l * WAY * (int)sizeof(TA));
      }
      zeros = __ffma2_rn(s[0], none, __ffma2_rn(s[1], none, zeros));
      return zeros.x + zeros.y;
    };
    if (rec_not_finite(go(std::false_type()))) go(std::true_type());
    tc::fence_proxy_async();      // seen by the copy that takes the tile away
  }
  __syncthreads();
  if (tid == PORTER) {
    put(rounds - 1);
    asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    // copies that were waited for in vain land before the CTA leaves, or not within the limit
    for (int r = rounds > STAGES ? rounds - STAGES : 0; lost && r < rounds; ++r) {
      bool late = false;
      if (turn_of(r) < tiles) wait(&full[r % STAGES], (r / STAGES) & 1, late);
    }
  }
  if (end && rank == 0 && mine) end[row + tid] = carry;
}

template <typename TX, typename TA, int STEPS, int STAGES, bool BACK>
cudaError_t launch(const RecArgs& a, int batch, cudaStream_t st) {
  using Shape = Tile<TX, TA, STEPS, BACK>;
  Maps maps{};
  const auto make = [&](CUtensorMap* m, const void* data, const RowStride& s, int bytes) {
    return smat_make_map_rows(m, data, bytes, (uint64_t)a.channels, (uint64_t)a.T, (uint64_t)batch, (uint64_t)s.token * bytes,
                              (uint64_t)(batch > 1 ? s.batch : s.token) * bytes, COLS, Shape::TOKENS);
  };
  if (!make(&maps.x, a.x, a.xs, sizeof(TX)) || !make(&maps.log_a, a.log_a, a.as, sizeof(TA)) || !make(&maps.out, a.out, a.os, sizeof(TX)))
    return cudaErrorInvalidValue;
  if (BACK && (!make(&maps.h, a.h, a.hs, sizeof(TX)) || !make(&maps.dlog_a, a.dlog_a, a.das, sizeof(TA)))) return cudaErrorInvalidValue;
  const auto kernel = recurrence_tma_kernel<TX, TA, STEPS, STAGES, BACK>;
  constexpr size_t bytes = (size_t)STAGES * Shape::BYTES;
  const cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  if (err != cudaSuccess) return err;
  const int64_t columns = (a.channels + COLS - 1) / COLS, tiles = (a.T + Shape::TOKENS - 1) / Shape::TOKENS;
  const unsigned ranks = rec_ranks(columns, batch, tiles);
  return smat_launch_pdl_cluster(kernel, dim3(ranks, (unsigned)columns, (unsigned)batch), REC_THREADS, bytes, ranks, st, maps, a.begin, a.h0, a.end,
                                 a.T, a.channels);
}

}  // namespace

bool smat_recurrence_tma_supported(const RecArgs& a, int batch, int x_bf16, int gate_bf16, bool back) {
  if (a.T > (1 << 30)) return false;      // coordinates of tokens
  const auto fits = [&](const void* data, const RowStride& s, int bytes) {
    uint64_t bits = reinterpret_cast<uintptr_t>(data) | (uint64_t)(s.token * bytes);
    if (batch > 1) bits |= (uint64_t)(s.batch * bytes);
    const int64_t most = (int64_t)1 << 36;
    return (bits & 15) == 0 && s.token > 0 && s.token < most && (batch == 1 || (s.batch > 0 && s.batch < most));
  };
  const int x = x_bf16 ? 2 : 4, g = gate_bf16 ? 2 : 4;
  return fits(a.x, a.xs, x) && fits(a.log_a, a.as, g) && fits(a.out, a.os, x) && (!back || (fits(a.h, a.hs, x) && fits(a.dlog_a, a.das, g)));
}

// Stages and tokens of a tile: two CTAs an SM, with two tiles or more on their way.
cudaError_t smat_launch_recurrence_tma(const RecArgs& a, int batch, int x_bf16, int gate_bf16, bool back, cudaStream_t st) {
  using bf16 = __nv_bfloat16;
  if (!x_bf16) return back ? launch<float, float, 2, 4, true>(a, batch, st) : launch<float, float, 4, 3, false>(a, batch, st);
  if (gate_bf16) return back ? launch<bf16, bf16, 4, 4, true>(a, batch, st) : launch<bf16, bf16, 8, 3, false>(a, batch, st);
  return back ? launch<bf16, float, 4, 3, true>(a, batch, st) : launch<bf16, float, 4, 4, false>(a, batch, st);
}
