// What the operators around the linear maps share: 16-bit types, the paged cache, and which sequence a token row belongs to.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math_constants.h>
#include <stdint.h>

#include <type_traits>

#include "common.cuh"

namespace ls {

constexpr int OP_BAD_PAGE = 1;  // bits of the flag an operator leaves: a table entry outside the cache, or a position beyond the table
constexpr int OP_BAD_ROWS = 2;  // row counts that do not ascend within [0, T], or a negative length
constexpr int OP_TIMEOUT = 4;   // a bounded wait ran out

// Keys and values of one layer, [page][head][slot][d] behind strides (in elements)
struct PagedKv {
  void *k, *v;
  long long page_stride, head_stride, slot_stride;
  int n_pages, page_shift, n_kv, d;
};

template <typename T>
__device__ __forceinline__ float to_f32(T v);
template <>
__device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <>
__device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }

// two values rounded to nearest, one 32-bit word (the low half is a's)
template <typename T>
__device__ __forceinline__ unsigned pack2(float a, float b);
template <>
__device__ __forceinline__ unsigned pack2<__nv_bfloat16>(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const unsigned*>(&v);
}
template <>
__device__ __forceinline__ unsigned pack2<__half>(float a, float b) {
  const __half2 v = __floats2half2_rn(a, b);
  return *reinterpret_cast<const unsigned*>(&v);
}

// Blackwell's packed fp32 arithmetic: two values a register pair
__device__ __forceinline__ unsigned long long two(float a, float b) {
  unsigned long long r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void split(unsigned long long x, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x)); }
__device__ __forceinline__ unsigned long long fma2(unsigned long long a, unsigned long long b, unsigned long long c) {
  unsigned long long r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ unsigned long long add2(unsigned long long a, unsigned long long b) {
  unsigned long long r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ unsigned long long mul2(unsigned long long a, unsigned long long b) {
  unsigned long long r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// The sequence that token row `row` belongs to: the last b < B with cu[b] <= row (-1: none).  A whole warp asks; every round probes 32
// places, so the dependent loads are two up to 1024 sequences.  Whatever cu holds, the answer lies in [-1, B).
__device__ __forceinline__ int seq_of_row(const int* cu, int B, int row, int lane) {
  int lo = 0, n = B;  // candidates cu[lo .. lo + n)
  while (n > 0) {
    const int step = (n + 31) / 32, at = lo + lane * step;
    const bool le = lane * step < n && __ldg(cu + at) <= row;
    const int c = __popc(__ballot_sync(0xffffffffu, le));  // (ascending: the probes that hold come first)
    if (c == 0) return lo - 1;
    const int first = lo + (c - 1) * step;  // holds; the next probe does not
    n = min(step, lo + n - first) - 1, lo = first + 1;
  }
  return lo - 1;
}

}  // namespace ls
