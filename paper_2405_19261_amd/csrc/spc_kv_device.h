// spc_kv_device.h -- what the kernels of the paged key/value cache share: rows of
// a chunk and the pages of a sequence, and sixteen bytes of keys or values.
#pragma once

#include <math.h>

#include <type_traits>

#include "spc_internal.h"

namespace spc {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4a2 __attribute__((aligned(2)));
typedef u32x4 u32x4a4 __attribute__((aligned(4)));
typedef u32x2 u32x2a2 __attribute__((aligned(2)));

constexpr float kNegInf = -__builtin_huge_valf();
constexpr float kF8Max = 448.0f;  // the largest e4m3 value

// Rows of sequence b: [first, first + n).
struct Chunk {
  int64_t first;
  int32_t n;
};
__device__ __forceinline__ Chunk chunk_of(const KvParams& P, int b) {
  if (!P.start) return Chunk{(int64_t)b * P.n, P.n};
  const int64_t lo = min(max((int64_t)P.start[b], (int64_t)0), P.rows);
  const int64_t hi = min(max((int64_t)P.start[b + 1], lo), P.rows);
  return Chunk{lo, (int32_t)(hi - lo)};
}
// The sequence of row r, or -1 (rows before the first and behind the last one).
__device__ __forceinline__ int sequence_of(const KvParams& P, int64_t r) {
  if (!P.start) return (int)(r / P.n);
  int lo = 0, hi = P.B;  // the first b with start[b + 1] > r
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (P.start[mid + 1] > r) hi = mid;
    else lo = mid + 1;
  }
  return lo < P.B && r >= P.start[lo] ? lo : -1;
}
// The page of position t of sequence b, or -1: past the table, or no page.
__device__ __forceinline__ int page_of(const KvParams& P, int b, int64_t t) {
  if (t < 0 || t >= (int64_t)P.width * P.S) return -1;
  const int p = P.table[(int64_t)b * P.width + (int)t / P.S];
  return p >= 0 && p < P.pages ? p : -1;
}

// Sixteen bytes of the cache: eight bfloat16 or sixteen e4m3 values.
__device__ __forceinline__ u32x4 load16(const void* p, int64_t bytes) {
  return *reinterpret_cast<const u32x4*>(static_cast<const char*>(p) + bytes);
}
// The step-th eight values of them as bfloat16 (exact for e4m3).
template <bool F8>
__device__ __forceinline__ bf16x8 widen(const u32x4& w, int step) {
  if constexpr (F8) {
    const uint32_t lo = w[2 * step], hi = w[2 * step + 1];
    const u32x4 y{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false)),
                  __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true)),
                  __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false)),
                  __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true))};
    return __builtin_bit_cast(bf16x8, y);
  } else {
    return __builtin_bit_cast(bf16x8, w);
  }
}
// The first n values, zeros behind them (n may be negative).
template <bool F8>
__device__ __forceinline__ void first_of(u32x4& w, int n) {
  constexpr int kPer = F8 ? 4 : 2, kBits = 32 / kPer;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int m = min(max(n - j * kPer, 0), kPer) * kBits;
    w[j] &= m == 32 ? 0xffffffffu : (1u << m) - 1u;
  }
}

// The values from the n-th on, zeros before them (n may be negative).
template <bool F8>
__device__ __forceinline__ void without_first(u32x4& w, int n) {
  constexpr int kPer = F8 ? 4 : 2, kBits = 32 / kPer;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int m = min(max(n - j * kPer, 0), kPer) * kBits;
    w[j] &= m == 32 ? 0u : ~((1u << m) - 1u);
  }
}

}  // namespace
}  // namespace spc
