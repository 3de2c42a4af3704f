// Type table of the decode cache in 8 bits, and back.  A row of p entries gets the largest m of eight significant bits (a bf16 number)
// with m max|row| <= 127: code = entry * m rounded to the nearest whole number (even between two), value = code * (1 / m).  With eight
// bits in m both products are exact in twice the entry's bits, so that m and the codes are the same in any arithmetic; a quotient 127 / max
// that is rounded before it is cut to eight bits is not (next to such a number it takes the step of 2^-7 to the other side: 8 rows in a
// million of fp32, every code of the row another).  The cut costs less than 2^-7 of the range.  A code's value is off by at most half
// a unit, max|row| / 254 (1 + 2^-7).
//
// Streams: a row is held by the lanes that read it in 16-byte pieces (p = 128 of bf16: 16 lanes, 8 codes each), its largest entry
// found by shuffles.  PACK_ROWS rows are in flight a thread.  Packing is bound by HBM only with few instructions an entry: with a
// conversion and shifts for every code (16 an entry) the table of 16 heads of 1463 states took 210 us, 175 by bytes.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "smat_internal.h"
#include "smat_launch.cuh"
#include "smat_rows.cuh"

namespace {

constexpr int PACK_THREADS = 256, PACK_ROWS = 4;

// The CTAs behind those of the rows copy what follows the table (running states, gates).
__device__ __forceinline__ void copy_tail(const uint4* from, uint4* to, int64_t words, int64_t block) {
  const int64_t i = block * PACK_THREADS + threadIdx.x;
  if (i < words) to[i] = from[i];
}

template <typename TU, int P>
__global__ void __launch_bounds__(PACK_THREADS) pack_kernel(const TU* table, int8_t* codes, float* units, int64_t rows,
                                                            int64_t row_blocks, const uint4* tail_from, uint4* tail_to, int64_t tail) {
  constexpr int VEC = 16 / (int)sizeof(TU), LANES = P / VEC, SLOTS = PACK_THREADS / LANES;
  pdl_trigger();
  pdl_wait();
  if ((int64_t)blockIdx.x >= row_blocks) {
    copy_tail(tail_from, tail_to, tail, blockIdx.x - row_blocks);
    return;
  }
  const int lane = threadIdx.x % LANES;
  const int64_t first = (int64_t)blockIdx.x * (SLOTS * PACK_ROWS) + threadIdx.x / LANES;
  RowVec<TU, VEC> in[PACK_ROWS];
#pragma unroll
  for (int n = 0; n < PACK_ROWS; ++n) {
    const int64_t row = first + n * SLOTS;
    in[n].clear();
    if (row < rows) in[n].load(table + row * P + lane * VEC);
  }
#pragma unroll
  for (int n = 0; n < PACK_ROWS; ++n) {
    const int64_t row = first + n * SLOTS;
    // bits of the largest |entry|: in the order of the numbers, with inf and NaN above all of them
    uint32_t top = 0u;
    if constexpr (sizeof(TU) == 2) {
#pragma unroll
      for (int i = 0; i < VEC / 2; ++i) top = __vmaxu2(top, in[n].w[i] & 0x7fff7fffu);
      top = max(top & 0xffff0000u, top << 16);
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) top = max(top, in[n].w[i] & 0x7fffffffu);
    }
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    const bool finite = top < 0x7f800000u;
    float m = 0.f;
    if (top != 0u && finite) {
      const float most = __uint_as_float(top);
      uint32_t bits = __float_as_uint(fminf(__fdiv_rn(127.f, most), 0x1p126f)) & 0xffff0000u;
      if (fmaf(__uint_as_float(bits), most, -127.f) > 0.f) bits -= 0x10000u;      // rounded up to it: one step of the eighth bit less
      m = __uint_as_float(bits);
    }
    // entry * m + 1.5 * 2^23: the product is exact inside the fused operation, and the sum's one rounding is that to a whole number
    uint32_t word[VEC / 4];
    const float2 mm = make_float2(m, m), whole = make_float2(12582912.f, 12582912.f);
#pragma unroll
    for (int i = 0; i < VEC; i += 4) {
      const float2 c0 = __ffma2_rn(make_float2(in[n].get(i), in[n].get(i + 1)), mm, whole);
      const float2 c1 = __ffma2_rn(make_float2(in[n].get(i + 2), in[n].get(i + 3)), mm, whole);
      const uint32_t lo = __byte_perm(__float_as_uint(c0.x), __float_as_uint(c0.y), 0x0040);
      const uint32_t hi = __byte_perm(__float_as_uint(c1.x), __float_as_uint(c1.y), 0x0040);
      word[i / 4] = finite ? __byte_perm(lo, hi, 0x5410) : 0u;
    }
    if (row >= rows) continue;
    uint32_t* to = reinterpret_cast<uint32_t*>(codes + row * P + lane * VEC);
    if constexpr (VEC == 8) *reinterpret_cast<uint2*>(to) = make_uint2(word[0], word[1]);
    else *to = word[0];
    if (lane == 0) units[row] = !finite ? __uint_as_float(0x7fc00000u) : m > 0.f ? __frcp_rn(m) : 0.f;
  }
}

template <typename TU, int P>
__global__ void __launch_bounds__(PACK_THREADS) unpack_kernel(const int8_t* codes, const float* units, TU* table, int64_t rows,
                                                              int64_t row_blocks, const uint4* tail_from, uint4* tail_to, int64_t tail) {
  constexpr int VEC = 16 / (int)sizeof(TU), LANES = P / VEC, SLOTS = PACK_THREADS / LANES;
  pdl_trigger();
  pdl_wait();
  if ((int64_t)blockIdx.x >= row_blocks) {
    copy_tail(tail_from, tail_to, tail, blockIdx.x - row_blocks);
    return;
  }
  const int lane = threadIdx.x % LANES;
  const int64_t first = (int64_t)blockIdx.x * (SLOTS * PACK_ROWS) + threadIdx.x / LANES;
  RowVec<float, VEC / 4> in[PACK_ROWS];      // VEC codes
  float unit[PACK_ROWS];
#pragma unroll
  for (int n = 0; n < PACK_ROWS; ++n) {
    const int64_t row = first + n * SLOTS;
    if (row >= rows) break;
    in[n].load(reinterpret_cast<const float*>(codes + row * P + lane * VEC));
    unit[n] = units[row];
  }
#pragma unroll
  for (int n = 0; n < PACK_ROWS; ++n) {
    const int64_t row = first + n * SLOTS;
    if (row >= rows) break;
    float v[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) v[i] = (float)(int8_t)(in[n].w[i / 4] >> (8 * (i % 4))) * unit[n];
    if (unit[n] > 0x1p120f) {      // half a unit above an entry at the end of the type's range: its largest number
      const float most = sizeof(TU) == 2 ? 0x1.fep127f : 0x1.fffffep127f;
#pragma unroll
      for (int i = 0; i < VEC; ++i) v[i] = fminf(fmaxf(v[i], -most), most);
    }
    RowVec<TU, VEC> out;
    out.set(v);
    out.store(table + row * P + lane * VEC);
  }
}

struct Blocks {
  int64_t rows, all, words;
};
template <typename TU, int P>
Blocks blocks(int64_t rows, size_t tail) {
  constexpr int PER = PACK_THREADS / (P / (16 / (int)sizeof(TU))) * PACK_ROWS;
  Blocks b;
  b.rows = (rows + PER - 1) / PER;
  b.words = (int64_t)(tail / 16);
  b.all = b.rows + (b.words + PACK_THREADS - 1) / PACK_THREADS;
  return b;
}

template <typename TU, int P>
cudaError_t pack(const void* table, void* codes, float* units, int64_t rows, const void* from, void* to, size_t tail, cudaStream_t st) {
  const Blocks b = blocks<TU, P>(rows, tail);
  if (b.all > INT32_MAX) return cudaErrorInvalidValue;
  return smat_launch_pdl(pack_kernel<TU, P>, dim3((unsigned)b.all), PACK_THREADS, 0, st, static_cast<const TU*>(table),
                         static_cast<int8_t*>(codes), units, rows, b.rows, static_cast<const uint4*>(from), static_cast<uint4*>(to), b.words);
}
template <typename TU, int P>
cudaError_t unpack(const void* codes, const float* units, void* table, int64_t rows, const void* from, void* to, size_t tail, cudaStream_t st) {
  const Blocks b = blocks<TU, P>(rows, tail);
  if (b.all > INT32_MAX) return cudaErrorInvalidValue;
  return smat_launch_pdl(unpack_kernel<TU, P>, dim3((unsigned)b.all), PACK_THREADS, 0, st, static_cast<const int8_t*>(codes), units,
                         static_cast<TU*>(table), rows, b.rows, static_cast<const uint4*>(from), static_cast<uint4*>(to), b.words);
}

}  // namespace

cudaError_t smat_launch_pack(const void* table, int table_bf16, void* codes, float* units, int64_t rows, int p, const void* tail_from,
                             void* tail_to, size_t tail, cudaStream_t st) {
  if ((p != 64 && p != 128) || tail % 16) return cudaErrorInvalidValue;
  if (table_bf16)
    return p == 64 ? pack<__nv_bfloat16, 64>(table, codes, units, rows, tail_from, tail_to, tail, st)
                   : pack<__nv_bfloat16, 128>(table, codes, units, rows, tail_from, tail_to, tail, st);
  return p == 64 ? pack<float, 64>(table, codes, units, rows, tail_from, tail_to, tail, st)
                 : pack<float, 128>(table, codes, units, rows, tail_from, tail_to, tail, st);
}

cudaError_t smat_launch_unpack(const void* codes, const float* units, void* table, int table_bf16, int64_t rows, int p,
                               const void* tail_from, void* tail_to, size_t tail, cudaStream_t st) {
  if ((p != 64 && p != 128) || tail % 16) return cudaErrorInvalidValue;
  if (table_bf16)
    return p == 64 ? unpack<__nv_bfloat16, 64>(codes, units, table, rows, tail_from, tail_to, tail, st)
                   : unpack<__nv_bfloat16, 128>(codes, units, table, rows, tail_from, tail_to, tail, st);
  return p == 64 ? unpack<float, 64>(codes, units, table, rows, tail_from, tail_to, tail, st)
                 : unpack<float, 128>(codes, units, table, rows, tail_from, tail_to, tail, st);
}
