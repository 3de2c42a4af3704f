// Rows of contiguous features at any stride: loads and stores of VEC elements of a row as floats, and the host-side checks
// of the operators that take such rows (rotary positions, norms, the recurrence).
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/smat.h"
#include "smat_internal.h"

// VEC elements as they lie in memory.  They are read once, past the L1 cache.
template <typename T, int VEC>
struct RowVec {
  static constexpr int BYTES = VEC * (int)sizeof(T), WORDS = BYTES < 4 ? 1 : BYTES / 4;
  uint32_t w[WORDS];

  __device__ __forceinline__ void load(const T* p) {
    if constexpr (BYTES == 2) {
      uint16_t v;
      asm volatile("ld.global.L1::no_allocate.u16 %0, [%1];" : "=h"(v) : "l"(p) : "memory");
      w[0] = v;
    } else if constexpr (BYTES == 4) {
      asm volatile("ld.global.L1::no_allocate.u32 %0, [%1];" : "=r"(w[0]) : "l"(p) : "memory");
    } else if constexpr (BYTES == 8) {
      asm volatile("ld.global.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(p) : "memory");
    } else {
#pragma unroll
      for (int i = 0; i < BYTES / 16; ++i)
        asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(w[4 * i]), "=r"(w[4 * i + 1]), "=r"(w[4 * i + 2]), "=r"(w[4 * i + 3])
                     : "l"(reinterpret_cast<const char*>(p) + 16 * i) : "memory");
    }
  }
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (BYTES == 2) {
      *reinterpret_cast<uint16_t*>(p) = (uint16_t)w[0];
    } else if constexpr (BYTES == 4) {
      *reinterpret_cast<uint32_t*>(p) = w[0];
    } else if constexpr (BYTES == 8) {
      *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    } else {
#pragma unroll
      for (int i = 0; i < BYTES / 16; ++i)
        reinterpret_cast<uint4*>(p)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) w[i] = 0u;
  }
  __device__ __forceinline__ float get(int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    else return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
  }
  // Rounded once, to the nearest value of the element type.
  __device__ __forceinline__ void set(const float* v) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) w[i] = __float_as_uint(v[i]);
    } else if constexpr (VEC == 1) {
      w[0] = __bfloat16_as_ushort(__float2bfloat16_rn(v[0]));
    } else {
#pragma unroll
      for (int i = 0; i < VEC / 2; ++i) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&b);
      }
    }
  }
};

// Strides of an operand on the device.
struct RowStride {
  int64_t batch, head, token;
};
inline RowStride row_stride(const smat_rows* r) { return r ? RowStride{r->batch, r->head, r->token} : RowStride{0, 0, 0}; }

inline int dtype_bytes(smat_dtype t) { return t == SMAT_BF16 ? 2 : 4; }

// Whether every row of r begins at a multiple of `bytes` (strides of dimensions of one entry do not matter).
inline bool rows_at_multiples(const smat_rows* r, smat_dtype t, int64_t batch, int64_t heads, int64_t tokens, unsigned bytes) {
  if (!r) return true;
  const int64_t e = dtype_bytes(t);
  uint64_t bits = reinterpret_cast<uintptr_t>(r->data);
  if (batch > 1) bits |= (uint64_t)(r->batch * e);
  if (heads > 1) bits |= (uint64_t)(r->head * e);
  if (tokens > 1) bits |= (uint64_t)(r->token * e);
  return (bits & (bytes - 1)) == 0;
}

inline bool rows_misaligned(const smat_rows* r, smat_dtype t) {
  return r && (reinterpret_cast<uintptr_t>(r->data) & (uintptr_t)(dtype_bytes(t) - 1)) != 0;
}

// Strides that address 64-bit elements without overflow and, for an output, rows that do not overlap one another: sorted by
// stride, each dimension steps over all of the smaller ones.
inline bool rows_ok(const smat_rows* r, int64_t batch, int64_t heads, int64_t tokens, int64_t width, bool output) {
  if (!r) return true;
  int64_t size[3] = {batch, heads, tokens}, step[3] = {r->batch, r->head, r->token};
  for (int i = 0; i < 3; ++i) {
    if (size[i] == 1) step[i] = 0;
    if (step[i] < 0 || (step[i] > 0 && (size[i] - 1) > (((int64_t)1 << 58) / step[i]))) return false;
  }
  if (!output) return true;
  for (int i = 0; i < 3; ++i)
    for (int j = i + 1; j < 3; ++j)
      if (step[j] < step[i]) {
        const int64_t a = step[i], b = size[i];
        step[i] = step[j]; size[i] = size[j];
        step[j] = a; size[j] = b;
      }
  int64_t extent = width;
  for (int i = 0; i < 3; ++i) {
    if (size[i] == 1) continue;
    if (step[i] < extent) return false;
    extent += step[i] * (size[i] - 1);
  }
  return true;
}

// Every kernel of the library is sm_100a code: a call that would launch on another device reports it instead.
inline bool rows_device_ok() {
  const bool ok = smat_tc_available();
  if (!ok) cudaGetLastError();
  return ok;
}
