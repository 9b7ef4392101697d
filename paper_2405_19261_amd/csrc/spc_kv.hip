// spc_kv.hip -- gfx950 kernels of the paged key/value cache: writing new
// tokens (in bfloat16 or quantised to e4m3), reading tokens back, and the
// attention of a chunk of new tokens over the cache.
//
// A page holds S consecutive tokens of one sequence, keys as [H][S][D] and
// values as [H][D][S]: transposed, because the attention's second product
// takes V^T as the left operand of a matrix instruction, whose lanes then load
// eight consecutive tokens of one dimension with one instruction, as they load
// eight dimensions of one key.  Chunks of few rows take their operands straight
// from memory (k_kv_attend), chunks of many through LDS (k_kv_attend_rows).
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

template <int SRC>
__device__ __forceinline__ float source(const void* p, int64_t i) {
  if constexpr (SRC == SPC_BF16)
    return __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(p)[i] << 16);
  else return reinterpret_cast<const float*>(p)[i];
}

// e4m3 of x / scale, both halves of a pair; out-of-range values saturate.
__device__ __forceinline__ uint8_t to_f8(float x) {
  x = fminf(fmaxf(x, -kF8Max), kF8Max);
  return (uint8_t)(__builtin_amdgcn_cvt_pk_fp8_f32(x, x, 0, false) & 0xff);
}

// A wavefront per (row, head).  8 bits: the scale is the largest magnitude
// over 448, not below the smallest normal float, and values divide by it with
// one correctly rounded division, so that the codes are those of the formula.
template <int SRC, bool F8>
__global__ void __launch_bounds__(256) k_kv_write(KvParams P) {
  const int lane = threadIdx.x & 63;
  const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int h = blockIdx.y;
  if (r >= P.rows) return;
  const int b = sequence_of(P, r);
  if (b < 0) return;
  const Chunk c = chunk_of(P, b);
  const int64_t t = (int64_t)P.len[b] - c.n + (r - c.first);
  const int page = page_of(P, b, t);
  if (page < 0) return;
  const int slot = (int)(t % P.S);
  const int64_t head = (int64_t)page * P.H + h;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const int64_t at = r * (which ? P.v_stride : P.k_stride) + (int64_t)h * P.D;
    float x[4], amax = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int d = i * 64 + lane;
      x[i] = d < P.D ? source<SRC>(which ? P.v_new : P.k_new, at + d) : 0.0f;
      amax = fmaxf(amax, fabsf(x[i]));
    }
    float scale = 1.0f;
    if constexpr (F8) {
#pragma unroll
      for (int d = 32; d; d >>= 1) amax = fmaxf(amax, __shfl_xor(amax, d));
      scale = fmaxf(amax / kF8Max, 1.17549435e-38f);
      if (lane == 0) (which ? P.v_scale : P.k_scale)[head * P.S + slot] = scale;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int d = i * 64 + lane;
      if (d >= P.D) continue;
      const int64_t to = which ? (head * P.D + d) * P.S + slot : (head * P.S + slot) * P.D + d;
      if constexpr (F8) static_cast<uint8_t*>(which ? P.v : P.k)[to] = to_f8(x[i] / scale);
      else static_cast<__bf16*>(which ? P.v : P.k)[to] = (__bf16)x[i];
    }
  }
}

// Sixteen bytes of the cache: eight bfloat16 or sixteen e4m3 values.
__device__ __forceinline__ u32x4 load16(const void* p, int64_t bytes) {
  return *reinterpret_cast<const u32x4*>(static_cast<const char*>(p) + bytes);
}
// Chunks of many rows: a workgroup takes 64 rows of a head, a wavefront a row at
// a time, and turns the values around in LDS, so that eight tokens of a dimension
// are one store (16 bytes, or 8 of 8 bits) where the page has them all; one by
// one they are 64 stores of 2 bytes to as many lines (4500 float32 rows of 8
// heads of 128 into bfloat16: 37 us so, 20 us with the tiles, 12 at the rate of
// a copy).
template <int SRC, bool F8, int D>
__global__ void __launch_bounds__(256) k_kv_write_tile(KvParams P) {
  constexpr int E = D / 64, kRow = 66;  // an odd number of words between dimensions
  typedef typename std::conditional<F8, uint8_t, uint16_t>::type T;
  __shared__ T turned[D * kRow];
  __shared__ int32_t pages[64], slots[64], whole[9];
  const int lane = threadIdx.x & 63, h = blockIdx.y;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int64_t r0 = (int64_t)blockIdx.x * 64;
  const int n = (int)min(P.rows - r0, (int64_t)64);
  if (wave == 0) {
    int page = -1, slot = 0;
    const int b = lane < n ? sequence_of(P, r0 + lane) : -1;
    if (b >= 0) {
      const Chunk c = chunk_of(P, b);
      const int64_t t = (int64_t)P.len[b] - c.n + (r0 + lane - c.first);
      page = page_of(P, b, t);
      slot = page < 0 ? 0 : (int)(t % P.S);
    }
    pages[lane] = page;
    slots[lane] = slot;
  }
  __syncthreads();
  const uint64_t live = __ballot(pages[lane] >= 0);  // the rows that are written
  if (!live) return;
  const int some = __builtin_ctzll(live);
  // kAtOnce rows of a wavefront at a time: their loads are under way together
  constexpr int kAtOnce = 4;
  for (int i0 = wave * kAtOnce; i0 < n; i0 += 4 * kAtOnce) {
    float x[kAtOnce][2][E];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int i = min(i0 + k, n - 1);
      const int64_t r = r0 + (live >> i & 1 ? i : some);  // (no other row is read)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        x[k][0][e] = source<SRC>(P.k_new, r * P.k_stride + (int64_t)h * D + e * 64 + lane);
        x[k][1][e] = source<SRC>(P.v_new, r * P.v_stride + (int64_t)h * D + e * 64 + lane);
      }
    }
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int i = i0 + k, page = i < n ? pages[i] : -1;
      if (page < 0) continue;  // (a wavefront's)
      const int64_t line = ((int64_t)page * P.H + h) * P.S + slots[i];
#pragma unroll
      for (int which = 0; which < 2; ++which) {
        float scale = 1.0f;
        if constexpr (F8) {
          float amax = 0.0f;
#pragma unroll
          for (int e = 0; e < E; ++e) amax = fmaxf(amax, fabsf(x[k][which][e]));
#pragma unroll
          for (int d = 32; d; d >>= 1) amax = fmaxf(amax, __shfl_xor(amax, d));
          scale = fmaxf(amax / kF8Max, 1.17549435e-38f);
          if (lane == 0) (which ? P.v_scale : P.k_scale)[line] = scale;
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
          T y;
          if constexpr (F8) y = to_f8(x[k][which][e] / scale);
          else y = __builtin_bit_cast(uint16_t, (__bf16)x[k][which][e]);
          if (which) turned[(e * 64 + lane) * kRow + i] = y;
          else static_cast<T*>(P.k)[line * D + e * 64 + lane] = y;
        }
      }
    }
  }
  __syncthreads();
  // values: 9 groups of eight slots cover 64 rows; a group that starts at a slot
  // which is a multiple of eight and lies in one page is one store a dimension
  const int lead = slots[0] & 7;
  if (threadIdx.x < 9) {
    const int i0 = (int)threadIdx.x * 8 - lead;
    bool one = i0 >= 0 && i0 + 8 <= n && pages[i0] >= 0 && (slots[i0] & 7) == 0;
    if (one)
      for (int e = 1; e < 8; ++e)
        one &= pages[i0 + e] == pages[i0] && slots[i0 + e] == slots[i0] + e;
    whole[threadIdx.x] = one;
  }
  __syncthreads();
  for (int k = (int)threadIdx.x; k < D * 9; k += 256) {
    const int g = k % 9, d = k / 9, i0 = g * 8 - lead;
    const T* src = turned + d * kRow;
    T* dst = static_cast<T*>(P.v);
    const bool one = whole[g];
    if (one) {
      T* to = dst + (((int64_t)pages[i0] * P.H + h) * D + d) * P.S + slots[i0];
      uint32_t w[F8 ? 2 : 4];
#pragma unroll
      for (int e = 0; e < (F8 ? 2 : 4); ++e) {
        if constexpr (F8)
          w[e] = (uint32_t)src[i0 + 4 * e] | (uint32_t)src[i0 + 4 * e + 1] << 8 |
                 (uint32_t)src[i0 + 4 * e + 2] << 16 | (uint32_t)src[i0 + 4 * e + 3] << 24;
        else w[e] = (uint32_t)src[i0 + 2 * e] | (uint32_t)src[i0 + 2 * e + 1] << 16;
      }
      if constexpr (F8) *reinterpret_cast<u32x2*>(to) = u32x2{w[0], w[1]};
      else *reinterpret_cast<u32x4*>(to) = u32x4{w[0], w[1], w[2], w[3]};
    } else {
      for (int e = 0; e < 8; ++e) {
        const int i = i0 + e;
        if (i < 0 || i >= n || pages[i] < 0) continue;
        dst[(((int64_t)pages[i] * P.H + h) * D + d) * P.S + slots[i]] = src[i];
      }
    }
  }
}

// The values of sixteen bytes of the cache.
template <bool F8>
__device__ __forceinline__ void values_of(const u32x4& w, float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (F8) {
      x[4 * i] = __builtin_amdgcn_cvt_f32_fp8(w[i], 0);
      x[4 * i + 1] = __builtin_amdgcn_cvt_f32_fp8(w[i], 1);
      x[4 * i + 2] = __builtin_amdgcn_cvt_f32_fp8(w[i], 2);
      x[4 * i + 3] = __builtin_amdgcn_cvt_f32_fp8(w[i], 3);
    } else {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
}
__device__ __forceinline__ uint32_t two_bf16(float a, float b) {
  return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)a) |
         (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)b) << 16;
}

// 64 positions of a head by a workgroup, in groups of 16 (a group lies in one
// page).  Keys go from 16-byte loads to 16-byte stores; values are turned around
// in LDS, in 32 bits.  Bound by the bytes: 134M values of e4m3 to bfloat16 take
// 96 us (4.2 TB/s); one wavefront a position, whose loads of a value's
// dimensions lie a page row apart, took 244.
template <int DST, bool F8, int D>
__global__ void __launch_bounds__(256) k_kv_read(KvParams P) {
  constexpr int EB = F8 ? 1 : 2, N = 16 / EB;       // values of a load
  constexpr int OB = DST == SPC_BF16 ? 2 : 4, kRow = D + 1;
  __shared__ float turned[64 * kRow];
  __shared__ int32_t pages[4], slots[4];
  const int h = blockIdx.y, b = blockIdx.z;
  const int64_t t0 = (int64_t)blockIdx.x * 64;
  const int64_t end = min((int64_t)P.L, (int64_t)P.len[b]);
  if (t0 >= end) return;
  if (threadIdx.x < 4) {
    const int64_t t = t0 + 16 * threadIdx.x;
    pages[threadIdx.x] = t < end ? page_of(P, b, t) : -1;
    slots[threadIdx.x] = (int)(t % P.S);
  }
  __syncthreads();
  const int64_t out0 = ((int64_t)b * P.L + t0) * P.H + h;  // row of position t0 + i: out0 + i H
  const auto store = [&](void* p, int i, int d, const float* x, int n) {
    char* to = static_cast<char*>(p) + ((out0 + (int64_t)i * P.H) * D + d) * OB;
#pragma unroll
    for (int k = 0; k < n * OB / 16; ++k) {
      u32x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (DST == SPC_BF16) w[e] = two_bf16(x[8 * k + 2 * e], x[8 * k + 2 * e + 1]);
        else w[e] = __float_as_uint(x[4 * k + e]);
      }
      *reinterpret_cast<u32x4*>(to + 16 * k) = w;
    }
  };
  // keys: load k of position i
  for (int k = (int)threadIdx.x; k < 64 * (D / N); k += 256) {
    const int d = k % (D / N) * N, i = k / (D / N), page = pages[i >> 4];
    if (page < 0 || t0 + i >= end) continue;
    const int64_t line = ((int64_t)page * P.H + h) * P.S + slots[i >> 4] + (i & 15);
    float x[N];
    values_of<F8>(load16(P.k, (line * D + d) * EB), x);
    if constexpr (F8) {
      const float scale = P.k_scale[line];
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] *= scale;
    }
    store(P.k_out, i, d, x, N);
  }
  // values: load of N positions of dimension d
  for (int k = (int)threadIdx.x; k < D * (64 / N); k += 256) {
    const int i = k % (64 / N) * N, d = k / (64 / N), page = pages[i >> 4];
    if (page < 0) continue;
    const int64_t head = (int64_t)page * P.H + h;
    const int slot = slots[i >> 4] + (i & 15);
    float x[N];
    values_of<F8>(load16(P.v, ((head * D + d) * P.S + slot) * EB), x);
    if constexpr (F8) {
#pragma unroll
      for (int e = 0; e < N; e += 4) {
        const f32x4 scale = *reinterpret_cast<const f32x4*>(P.v_scale + head * P.S + slot + e);
#pragma unroll
        for (int c = 0; c < 4; ++c) x[e + c] *= scale[c];
      }
    }
#pragma unroll
    for (int e = 0; e < N; ++e) turned[(i + e) * kRow + d] = x[e];
  }
  __syncthreads();
  for (int k = (int)threadIdx.x; k < 64 * (D / 8); k += 256) {
    const int d = k % (D / 8) * 8, i = k / (D / 8);
    if (pages[i >> 4] < 0 || t0 + i >= end) continue;
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = turned[i * kRow + d + e];
    store(P.v_out, i, d, x, 8);
  }
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

// ------------------------------------------------------------------ attention
// The rows of a key/value head are the pairs (new token i, query head g of the
// head's group), i first; a workgroup takes 16 MT of them and a share of the
// keys, its four wavefronts every fourth tile of T keys.  Scores are taken
// transposed, S^T = K Q^T, sixteen keys at a time, so chosen that lane 16 j + c
// holds row c's scores of T/4 consecutive keys, which is what the second product
// O^T = V^T P^T wants as right operand: neither P nor the running statistics of
// a row move between lanes but for the row's own reductions over j, and these
// only when its maximum grows.  Keys and values are read once per workgroup,
// straight to registers, sixteen bytes a lane: with 8-bit values a lane's bytes
// are two steps of the products, so there T = 64, else 32.  Which dimension
// stands where in Q K^T does not matter so long as Q is loaded alike.
// Statistics and O are held in 32 bits.  P (with 8-bit values times their scale)
// is rounded to bfloat16, by at most 2^-8, because the matrix unit takes both
// operands in one type; its sum is of the values before that.  (The error of
// answers to random values: 2.0e-3 to 2.3e-3, with P in 32 bits 1.7e-3, which is
// their own rounding to bfloat16.)  Bound by the bytes of the cache for few rows
// (32 sequences over 4096 tokens, 8 heads of 128, one row: bfloat16 101 us, 5.3
// TB/s, e4m3 52; 8 rows of 4 heads each, bfloat16, 114), by the vector
// instructions of the softmax and of widening 8 bits for more.
constexpr int kAttendWaves = 4;
// A share of the keys has at least as many: a tile for each wavefront, or in
// k_kv_attend_rows, whose wavefronts take every tile together, 512.  (One token
// over 1500 bfloat16 tokens of 8 heads: 13.9 us in shares of 512, 6.9 in shares
// of 128, and the join 4.4.)

constexpr int share_keys(int tile_rows, bool f8) { return tile_rows > 64 ? 512 : f8 ? 256 : 128; }

// The first position that a row at position t sees (under 0: from 0).  A row
// before position 0 sees nothing: it is taken as at 0, where no window of 32 bits
// passes them.
__device__ __forceinline__ int32_t first_seen(const KvParams& P, int32_t t) {
  return P.window > 0 ? max(t, 0) - P.window + 1 : 0;
}

// The keys that rows of a chunk's tokens i0 .. i1 see: tiles of T from `begin`
// (a multiple of T), cut into shares of `per` tiles.
struct Span {
  int32_t begin, tiles, shares, per;
};
template <int T, int MIN>
__device__ __forceinline__ Span span_of(const KvParams& P, int32_t len, int n, int i0, int i1,
                                        int splits) {
  const int32_t end = min(min(len, P.width * P.S), len - n + i1 + 1);
  Span s;
  s.begin = max(first_seen(P, len - n + i0), 0) & ~(T - 1);
  s.tiles = end > s.begin ? (end - s.begin + T - 1) / T : 0;
  s.shares = max(1, min(splits, s.tiles / (MIN / T)));
  s.per = (s.tiles + s.shares - 1) / s.shares;
  return s;
}

// Wavefronts a SIMD that registers are kept free for: two where they then do not
// spill.
constexpr int attend_waves(int D, bool f8, int mt) {
  return D <= 128 && mt * D <= (f8 ? 128 : 256) ? 2 : 1;
}

template <int D, bool F8, int MT>
__global__ void __launch_bounds__(64 * kAttendWaves, attend_waves(D, F8, MT))
    k_kv_attend(KvParams P) {
  constexpr int EB = F8 ? 1 : 2, T = F8 ? 64 : 32;
  constexpr int kQuarters = T / 16, kG = T / 4;  // score tiles; a lane's keys
  constexpr int kL = D * EB / 64;                // 16-byte loads of a key row by four lanes
  constexpr int kSteps = 2 / EB;                 // matrix steps in 16 bytes
  constexpr int kC = D / 32, kM = D / 16;
  constexpr int kPad = 4;
  __shared__ float o_lds[kAttendWaves][16][D + kPad];
  __shared__ float m_lds[kAttendWaves][16], l_lds[kAttendWaves][16];
  // Workgroups are dealt to the 8 dies in turn: those of one sequence and head
  // (and share of its keys) go to one die, whose cache then holds their keys, the
  // row tiles that see most keys first.
  const uint32_t tiles_x = (uint32_t)(((int64_t)P.n * (P.heads / P.H) + 16 * MT - 1) / (16 * MT));
  const uint32_t group = blockIdx.x / 8 / tiles_x * 8 + blockIdx.x % 8;
  const uint32_t tile_x = tiles_x - 1 - blockIdx.x / 8 % tiles_x;
  if (group >= (uint32_t)(P.H * P.B * P.splits)) return;
  const int h = (int)(group % P.H), z = (int)(group / P.H), share = z % P.splits, b = z / P.splits;
  const int lane = threadIdx.x & 63, c16 = lane & 15, j = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const Chunk ch = chunk_of(P, b);
  const int G = P.heads / P.H;
  const int64_t rows = (int64_t)min(ch.n, P.n) * G, r0 = (int64_t)tile_x * (16 * MT);
  if (r0 >= rows) return;
  const int32_t len = max(P.len[b], 0), there = min(len, P.width * P.S);
  const int i0 = (int)(r0 / G), i1 = (int)((min(r0 + 16 * MT, rows) - 1) / G);
  const Span span = span_of<T, share_keys(16 * MT, F8)>(P, len, ch.n, i0, i1, P.splits);
  if (share >= span.shares) return;
  const int tile0 = share * span.per, tile1 = min(span.tiles, tile0 + span.per);
  const int32_t pos0 = len - ch.n;

  bf16x8 q[MT][kC];
  int32_t last[MT], first[MT];  // the keys a row sees
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int64_t r = min(r0 + 16 * mt + c16, rows - 1);
    const int i = (int)(r / G), g = (int)(r % G);
    const int64_t q_at = (ch.first + i) * P.q_stride + (int64_t)(h * G + g) * D;
#pragma unroll
    for (int c = 0; c < kC; ++c) {
      const int d = c / kSteps * (32 * kSteps) + j * (8 * kSteps) + c % kSteps * 8;
      q[mt][c] = __builtin_bit_cast(
          bf16x8, u32x4(*reinterpret_cast<const u32x4a2*>(static_cast<const uint16_t*>(P.q) + q_at + d)));
    }
    last[mt] = pos0 + i;
    first[mt] = first_seen(P, last[mt]);
  }
  // a tile within these is seen whole by every row
  const int32_t all_from = first_seen(P, pos0 + i1);
  const int32_t all_to = min(pos0 + i0 + 1, there);

  f32x4 o[MT][kM] = {};
  float m[MT], l[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    m[mt] = kNegInf;
    l[mt] = 0.0f;
  }
  const int32_t* table = P.table + (int64_t)b * P.width;
  // the page index of a position in the table, and the page there (or -1)
  const auto index_of = [&](uint32_t t) {
    return P.s16_magic ? __umulhi(t >> 4, P.s16_magic) : t >> 4;
  };
  const auto page_at = [&](int32_t t) {
    const int p = table[index_of((uint32_t)min(t, there - 1))];
    return t < there && (uint32_t)p < (uint32_t)P.pages ? p : -1;
  };
  // where this lane reads of a tile at t0: a row of K, and its own keys of V
  const int key = kG * (c16 >> 2);
  struct Where {
    int64_t k, v;  // bytes
    int64_t scale;
    int ps, any;
  };
  const auto where = [&](int32_t t0, int pk, int ps) {
    const uint32_t tk = (uint32_t)(t0 + key), ts = (uint32_t)(t0 + kG * j);
    const int slot_k = (int)(tk - index_of(tk) * (uint32_t)P.S) + (c16 & 3);
    const int slot = (int)(ts - index_of(ts) * (uint32_t)P.S);
    const int64_t hk = (int64_t)max(pk, 0) * P.H + h, hs = (int64_t)max(ps, 0) * P.H + h;
    Where w;
    w.k = ((hk * P.S + slot_k) * D) * EB + 16 * j;
    w.v = ((hs * D + c16) * P.S + slot) * EB;
    w.scale = hs * P.S + slot;
    w.ps = ps;
    w.any = __any((pk | ps) < 0);
    return w;
  };
  u32x4 kf[kQuarters][kL];
  const auto load_k = [&](const Where& w) {
#pragma unroll
    for (int qd = 0; qd < kQuarters; ++qd)
#pragma unroll
      for (int c = 0; c < kL; ++c) kf[qd][c] = load16(P.k, w.k + 4 * qd * D * EB + 64 * c);
  };
  int tile = tile0 + wave;
  Where now{};
  if (tile < tile1) {
    const int32_t t0 = span.begin + T * tile;
    now = where(t0, page_at(t0 + key), page_at(t0 + kG * j));
    load_k(now);
  }
  for (; tile < tile1; tile += kAttendWaves) {
    const int32_t t0 = span.begin + T * tile, ts = t0 + kG * j;
    // the next tile's pages
    const int32_t tn = t0 + T * kAttendWaves;
    const bool more = tile + kAttendWaves < tile1;
    int pk = -1, ps = -1;
    if (more) {
      pk = page_at(tn + key);
      ps = page_at(tn + kG * j);
    }
    u32x4 vf[kM];
#pragma unroll
    for (int d = 0; d < kM; ++d) vf[d] = load16(P.v, now.v + (int64_t)(16 * d) * P.S * EB);
    f32x4 ks[kQuarters], vs[kQuarters];
    if constexpr (F8) {
#pragma unroll
      for (int qd = 0; qd < kQuarters; ++qd) {
        ks[qd] = *reinterpret_cast<const f32x4*>(P.k_scale + now.scale + 4 * qd);
        vs[qd] = *reinterpret_cast<const f32x4*>(P.v_scale + now.scale + 4 * qd);
      }
    }
    f32x4 s[MT][kQuarters];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int qd = 0; qd < kQuarters; ++qd) s[mt][qd] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int c = 0; c < kC; ++c)
#pragma unroll
      for (int qd = 0; qd < kQuarters; ++qd) {
        const bf16x8 k8 = widen<F8>(kf[qd][c / kSteps], c % kSteps);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
          s[mt][qd] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k8, q[mt][c], s[mt][qd], 0, 0, 0);
      }
    if constexpr (F8) {
#pragma unroll
      for (int qd = 0; qd < kQuarters; ++qd) ks[qd] *= P.scale;
    }
    const bool whole = t0 >= all_from && t0 + T <= all_to && !now.any;
    const bool page = now.ps >= 0;
    if (more) {
      now = where(tn, pk, ps);
      load_k(now);
    }
    bf16x8 p[MT][kSteps];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      float x[kG];
#pragma unroll
      for (int e = 0; e < kG; ++e) {
        if constexpr (F8) x[e] = s[mt][e >> 2][e & 3] * ks[e >> 2][e & 3];
        else x[e] = s[mt][e >> 2][e & 3] * P.scale;
      }
      if (!whole) {  // uniform
        const int32_t hi = page ? min(there - 1, last[mt]) : -1;
#pragma unroll
        for (int e = 0; e < kG; ++e)
          x[e] = ((ts + e <= hi) & (ts + e >= first[mt])) ? x[e] : kNegInf;
      }
      float mx = x[0];
#pragma unroll
      for (int e = 1; e < kG; ++e) mx = fmaxf(mx, x[e]);
      if (__any(mx > m[mt])) {  // some row's maximum grows
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float m_new = fmaxf(m[mt], mx);
        const float fade = m_new == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(m[mt] - m_new);
        m[mt] = m_new;
        l[mt] *= fade;
#pragma unroll
        for (int d = 0; d < kM; ++d) o[mt][d] *= fade;
      }
      const float base = m[mt] == kNegInf ? 0.0f : m[mt];  // (nothing seen yet)
#pragma unroll
      for (int e = 0; e < kG; ++e) {
        float w = __builtin_amdgcn_exp2f(x[e] - base);
        l[mt] += w;
        if constexpr (F8) {
          w *= vs[e >> 2][e & 3];
          if (!whole) w = x[e] == kNegInf ? 0.0f : w;  // (an unseen key's scale may be junk)
        }
        p[mt][e >> 3][e & 7] = (__bf16)w;
      }
    }
    if (!whole) {  // what lies behind the last key may be anything, NaN too
      const int live = page ? there - ts : 0;
#pragma unroll
      for (int d = 0; d < kM; ++d) first_of<F8>(vf[d], live);
    }
#pragma unroll
    for (int d = 0; d < kM; ++d)
#pragma unroll
      for (int step = 0; step < kSteps; ++step) {
        const bf16x8 v8 = widen<F8>(vf[d], step);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
          o[mt][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v8, p[mt][step], o[mt][d], 0, 0, 0);
      }
  }

  // join the wavefronts, 16 rows at a time; a share that is all of its keys ends
  // here, others leave O, the maximum and the sum to k_kv_join
  const bool alone = span.shares == 1;
  float* part = P.part + ((((int64_t)z * P.H + h) * tiles_x + tile_x) * (16 * MT)) *
                             (int64_t)(D + 2);
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    l[mt] += __shfl_xor(l[mt], 16);
    l[mt] += __shfl_xor(l[mt], 32);
    if (mt) __syncthreads();
    if (j == 0) {
      m_lds[wave][c16] = m[mt];
      l_lds[wave][c16] = l[mt];
    }
    __syncthreads();
    float top = m_lds[0][c16];
#pragma unroll
    for (int w = 1; w < kAttendWaves; ++w) top = fmaxf(top, m_lds[w][c16]);
    const float fade = m[mt] == kNegInf ? 0.0f : __builtin_amdgcn_exp2f(m[mt] - top);
#pragma unroll
    for (int d = 0; d < kM; ++d)
      *reinterpret_cast<f32x4*>(&o_lds[wave][c16][16 * d + 4 * j]) = o[mt][d] * fade;
    __syncthreads();
    for (int k = (int)threadIdx.x; k < 16 * (D / 4); k += 64 * kAttendWaves) {
      const int row = k / (D / 4), d = k % (D / 4) * 4;
      const int64_t r = r0 + 16 * mt + row;
      if (r >= rows) continue;
      float t = m_lds[0][row];
#pragma unroll
      for (int w = 1; w < kAttendWaves; ++w) t = fmaxf(t, m_lds[w][row]);
      float sum = 0.0f;
      f32x4 y{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int w = 0; w < kAttendWaves; ++w) {
        if (m_lds[w][row] != kNegInf)
          sum += l_lds[w][row] * __builtin_amdgcn_exp2f(m_lds[w][row] - t);
        y += *reinterpret_cast<const f32x4*>(&o_lds[w][row][d]);
      }
      if (alone) {
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        const int i = (int)(r / G), g = (int)(r % G);
        bf16x4 z;
#pragma unroll
        for (int e = 0; e < 4; ++e) z[e] = (__bf16)(y[e] * inv);
        *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(P.out) + (ch.first + i) * P.out_stride +
                                  (int64_t)(h * G + g) * D + d) = __builtin_bit_cast(u32x2, z);
      } else {
        float* to = part + (int64_t)(16 * mt + row) * (D + 2);
#pragma unroll
        for (int e = 0; e < 4; ++e) to[2 + d + e] = y[e];
        if (d == 0) {
          to[0] = t;
          to[1] = sum;
        }
      }
    }
  }
}

// Keys in a tile of k_kv_attend_rows.
constexpr int rows_tile(int D, bool f8) { return f8 || D <= 128 ? 64 : 32; }

// The same for chunks of many rows: a workgroup takes 128, each wavefront 32 of
// its own over all of the share's keys, so that a tile of keys and values is
// read once for 128 rows. Tiles pass through LDS, in the order the lanes of the
// products want them (a wavefront's read is 1 KiB in a row, without conflicts),
// double-buffered: the next tile's are written behind the products of this one
// and the loads of the one after it are then under way.  What bounds it is the
// LDS, whose reads of a tile take as long as the products of 32 rows with it,
// and the softmax's vector instructions: 4 chunks of 1024 rows over 4096 tokens,
// 32/8 heads of 128, take 383 to 406 us in bfloat16 (593 to 629 TFLOP/s; by 406,
// 515 us with 32 keys a tile, 653 with 64 rows a workgroup and its wavefronts apart
// over the keys) and 437 in e4m3.
template <int D, bool F8>
__global__ void __launch_bounds__(64 * kAttendWaves, D <= 128 ? 2 : 1) k_kv_attend_rows(KvParams P) {
  constexpr int MT = 2, kRows = 16 * MT * kAttendWaves;
  constexpr int EB = F8 ? 1 : 2, T = rows_tile(D, F8);
  constexpr int kQuarters = T / 16, kG = T / 4;
  constexpr int kL = D * EB / 64, kSteps = 2 / EB, kC = D / 32, kM = D / 16;
  constexpr int kVL = T * EB / 64;                   // 16-byte loads of a lane's keys of V
  constexpr int kFrags = kQuarters * kL + kM * kVL;  // of 1 KiB: K's, then V's
  constexpr int kMine = kFrags / kAttendWaves;       // that a wavefront brings
  static_assert(kQuarters * kL % kAttendWaves == 0 && kM * kVL % kAttendWaves == 0, "whole shares");
  __shared__ u32x4 frags[2][kFrags][64];
  __shared__ float scales[2][2][F8 ? T : 1];         // of keys, of values
  const uint32_t tiles_x = (uint32_t)(((int64_t)P.n * (P.heads / P.H) + kRows - 1) / kRows);
  const uint32_t group = blockIdx.x / 8 / tiles_x * 8 + blockIdx.x % 8;
  const uint32_t tile_x = tiles_x - 1 - blockIdx.x / 8 % tiles_x;
  if (group >= (uint32_t)(P.H * P.B * P.splits)) return;
  const int h = (int)(group % P.H), z = (int)(group / P.H), share = z % P.splits, b = z / P.splits;
  const int lane = threadIdx.x & 63, c16 = lane & 15, j = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const Chunk ch = chunk_of(P, b);
  const int G = P.heads / P.H;
  const int64_t rows = (int64_t)min(ch.n, P.n) * G, r0 = (int64_t)tile_x * kRows;
  if (r0 >= rows) return;
  const int32_t len = max(P.len[b], 0), there = min(len, P.width * P.S), pos0 = len - ch.n;
  const Span span =
      span_of<T, share_keys(kRows, F8)>(P, len, ch.n, (int)(r0 / G),
                                        (int)((min(r0 + kRows, rows) - 1) / G), P.splits);
  if (share >= span.shares) return;
  const int tile0 = share * span.per, tile1 = min(span.tiles, tile0 + span.per);

  // this wavefront's rows (the last row again behind the end)
  const int64_t w0 = r0 + 16 * MT * wave;
  bf16x8 q[MT][kC];
  int32_t last[MT], first[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int64_t r = min(w0 + 16 * mt + c16, rows - 1);
    const int i = (int)(r / G), g = (int)(r % G);
    const int64_t q_at = (ch.first + i) * P.q_stride + (int64_t)(h * G + g) * D;
#pragma unroll
    for (int c = 0; c < kC; ++c) {
      const int d = c / kSteps * (32 * kSteps) + j * (8 * kSteps) + c % kSteps * 8;
      q[mt][c] = __builtin_bit_cast(
          bf16x8, u32x4(*reinterpret_cast<const u32x4a2*>(static_cast<const uint16_t*>(P.q) + q_at + d)));
    }
    last[mt] = pos0 + i;
    first[mt] = first_seen(P, last[mt]);
  }
  const int i0 = (int)(min(w0, rows - 1) / G), i1 = (int)((min(w0 + 16 * MT, rows) - 1) / G);
  const int32_t all_from = first_seen(P, pos0 + i1);
  const int32_t all_to = min(pos0 + i0 + 1, there);

  f32x4 o[MT][kM] = {};
  float m[MT] = {kNegInf, kNegInf}, l[MT] = {0.0f, 0.0f};
  const int32_t* table = P.table + (int64_t)b * P.width;
  const auto index_of = [&](uint32_t t) {
    return P.s16_magic ? __umulhi(t >> 4, P.s16_magic) : t >> 4;
  };
  const auto page_at = [&](int32_t t) {
    const int p = table[index_of((uint32_t)min(t, there - 1))];
    return t < there && (uint32_t)p < (uint32_t)P.pages ? p : -1;
  };
  const int key = kG * (c16 >> 2);
  // the fragments this wavefront brings of a tile at t0, and a lane's scale
  u32x4 mine[kMine];
  float my_scale = 0.0f;
  int page_next = -1, page_now = -1;  // the page of this lane's own keys
  const auto bring = [&](int32_t t0) {
    const int pk = page_at(t0 + key), ps = page_at(t0 + kG * j);
    const uint32_t tk = (uint32_t)(t0 + key), ts = (uint32_t)(t0 + kG * j);
    const int slot_k = (int)(tk - index_of(tk) * (uint32_t)P.S) + (c16 & 3);
    const int slot = (int)(ts - index_of(ts) * (uint32_t)P.S);
    const int64_t hk = (int64_t)max(pk, 0) * P.H + h, hs = (int64_t)max(ps, 0) * P.H + h;
    const int64_t at_k = (hk * P.S + slot_k) * D * EB + 16 * j;
    const int64_t at_v = ((hs * D + c16) * P.S + slot) * EB;
    page_next = ps;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const int f = wave + i * kAttendWaves;
      if (i < kQuarters * kL / kAttendWaves)
        mine[i] = load16(P.k, at_k + (f / kL) * 4 * D * EB + f % kL * 64);
      else
        mine[i] = load16(P.v, at_v + (int64_t)(16 * ((f - kQuarters * kL) / kVL)) * P.S * EB +
                                  (f - kQuarters * kL) % kVL * 16);
    }
    if constexpr (F8) {
      if (threadIdx.x < 2 * T) {  // a thread a key and kind
        const uint32_t t = (uint32_t)t0 + threadIdx.x % T;
        const int p = page_at((int32_t)t);
        const int64_t at = ((int64_t)max(p, 0) * P.H + h) * P.S + (t - index_of(t) * (uint32_t)P.S);
        my_scale = p < 0 ? 0.0f : threadIdx.x < T ? P.k_scale[at] * P.scale : P.v_scale[at];
      }
    }
  };
  const auto put = [&](int buf) {
#pragma unroll
    for (int i = 0; i < kMine; ++i) frags[buf][wave + i * kAttendWaves][lane] = mine[i];
    if constexpr (F8)
      if (threadIdx.x < 2 * T) scales[buf][threadIdx.x / T][threadIdx.x % T] = my_scale;
  };
  if (tile0 < tile1) {
    bring(span.begin + T * tile0);
    put(0);
    page_now = page_next;
    if (tile0 + 1 < tile1) bring(span.begin + T * (tile0 + 1));
  }
  __syncthreads();
  for (int tile = tile0; tile < tile1; ++tile) {
    const int buf = (tile - tile0) & 1;
    const int32_t t0 = span.begin + T * tile, ts = t0 + kG * j;
    f32x4 s[MT][kQuarters];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int qd = 0; qd < kQuarters; ++qd) s[mt][qd] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int qd = 0; qd < kQuarters; ++qd)
#pragma unroll
      for (int c = 0; c < kC; ++c) {
        const bf16x8 k8 = widen<F8>(frags[buf][qd * kL + c / kSteps][lane], c % kSteps);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
          s[mt][qd] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k8, q[mt][c], s[mt][qd], 0, 0, 0);
      }
    const bool whole = t0 >= all_from && t0 + T <= all_to && !__any(page_now < 0);
    bf16x8 p[MT][kG / 8];
    float x[MT][kG], mx[MT];
    bool grows = false;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
      for (int e = 0; e < kG; ++e) {
        if constexpr (F8) x[mt][e] = s[mt][e >> 2][e & 3] * scales[buf][0][kG * j + e];
        else x[mt][e] = s[mt][e >> 2][e & 3] * P.scale;
      }
      if (!whole) {  // uniform
        const int32_t hi = page_now >= 0 ? min(there - 1, last[mt]) : -1;
#pragma unroll
        for (int e = 0; e < kG; ++e)
          x[mt][e] = ((ts + e <= hi) & (ts + e >= first[mt])) ? x[mt][e] : kNegInf;
      }
      mx[mt] = x[mt][0];
#pragma unroll
      for (int e = 1; e < kG; ++e) mx[mt] = fmaxf(mx[mt], x[mt][e]);
      grows |= mx[mt] > m[mt];
    }
    if (__any(grows)) {  // some row's maximum grows
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        mx[mt] = fmaxf(mx[mt], __shfl_xor(mx[mt], 16));
        mx[mt] = fmaxf(mx[mt], __shfl_xor(mx[mt], 32));
        const float m_new = fmaxf(m[mt], mx[mt]);
        const float fade = m_new == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(m[mt] - m_new);
        m[mt] = m_new;
        l[mt] *= fade;
#pragma unroll
        for (int d = 0; d < kM; ++d) o[mt][d] *= fade;
      }
    }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const float base = m[mt] == kNegInf ? 0.0f : m[mt];  // (nothing seen yet)
#pragma unroll
      for (int e = 0; e < kG; ++e) {
        float w = __builtin_amdgcn_exp2f(x[mt][e] - base);
        l[mt] += w;
        if constexpr (F8) {
          w *= scales[buf][1][kG * j + e];
          if (!whole) w = x[mt][e] == kNegInf ? 0.0f : w;  // (an unseen key's scale may be junk)
        }
        p[mt][e >> 3][e & 7] = (__bf16)w;
      }
    }
    const int live = page_now >= 0 ? there - ts : 0;
#pragma unroll
    for (int d = 0; d < kM; ++d)
#pragma unroll
      for (int part = 0; part < kVL; ++part) {
        u32x4 v = frags[buf][kQuarters * kL + d * kVL + part][lane];
        // what lies behind the last key may be anything, NaN too
        if (!whole) first_of<F8>(v, live - part * 8);
#pragma unroll
        for (int step = 0; step < kSteps; ++step) {
          const bf16x8 v8 = widen<F8>(v, step);
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
            o[mt][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v8, p[mt][part * kSteps + step],
                                                               o[mt][d], 0, 0, 0);
        }
      }
    // (the buffer written here was last read before the last barrier)
    if (tile + 1 < tile1) {
      put(buf ^ 1);
      page_now = page_next;
      if (tile + 2 < tile1) bring(t0 + 2 * T);
    }
    __syncthreads();
  }

  const bool alone = span.shares == 1;
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    l[mt] += __shfl_xor(l[mt], 16);
    l[mt] += __shfl_xor(l[mt], 32);
    const int64_t r = w0 + 16 * mt + c16;
    if (r >= rows) continue;
    if (alone) {
      const float inv = l[mt] == 0.0f ? 0.0f : 1.0f / l[mt];
      const int i = (int)(r / G), g = (int)(r % G);
      uint16_t* out = static_cast<uint16_t*>(P.out) + (ch.first + i) * P.out_stride +
                      (int64_t)(h * G + g) * D + 4 * j;
#pragma unroll
      for (int d = 0; d < kM; ++d) {
        bf16x4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = (__bf16)(o[mt][d][e] * inv);
        *reinterpret_cast<u32x2*>(out + 16 * d) = __builtin_bit_cast(u32x2, y);
      }
    } else {
      float* to = P.part + ((((int64_t)z * P.H + h) * tiles_x + tile_x) * kRows + (r - r0)) *
                               (int64_t)(D + 2);
#pragma unroll
      for (int d = 0; d < kM; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e) to[2 + 16 * d + 4 * j + e] = o[mt][d][e];
      if (j == 0) {
        to[0] = m[mt];
        to[1] = l[mt];
      }
    }
  }
}

// The shares of a row joined, in their order: a wavefront a row.
template <int D, int T, int MIN>
__global__ void __launch_bounds__(256) k_kv_join(KvParams P, int tile_rows) {
  const int b = blockIdx.z, h = blockIdx.y, lane = threadIdx.x & 63;
  const Chunk ch = chunk_of(P, b);
  const int G = P.heads / P.H;
  const int64_t rows = (int64_t)min(ch.n, P.n) * G;
  const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (r >= rows) return;
  const int64_t x = r / tile_rows, tiles_x = ((int64_t)P.n * G + tile_rows - 1) / tile_rows;
  const int64_t r0 = x * tile_rows;
  const Span span = span_of<T, MIN>(P, max(P.len[b], 0), ch.n, (int)(r0 / G),
                                    (int)((min(r0 + tile_rows, rows) - 1) / G), P.splits);
  if (span.shares == 1) return;
  const auto part = [&](int s) {
    return P.part + (((((int64_t)b * P.splits + s) * P.H + h) * tiles_x + x) * tile_rows + (r - r0)) *
                        (int64_t)(D + 2);
  };
  // the shares' maxima and sums, a lane a share (two: at most kKvShares)
  static_assert(kKvShares == 128, "two a lane");
  const float m0 = lane < span.shares ? part(lane)[0] : kNegInf;
  const float m1 = lane + 64 < span.shares ? part(lane + 64)[0] : kNegInf;
  float sum = lane < span.shares ? part(lane)[1] : 0.0f;
  float sum1 = lane + 64 < span.shares ? part(lane + 64)[1] : 0.0f;
  float top = fmaxf(m0, m1);
#pragma unroll
  for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  const float f0 = m0 == kNegInf ? 0.0f : __builtin_amdgcn_exp2f(m0 - top);
  const float f1 = m1 == kNegInf ? 0.0f : __builtin_amdgcn_exp2f(m1 - top);
  sum = sum * f0 + sum1 * f1;
#pragma unroll
  for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
  constexpr int E = D / 64;
  float y[E] = {};
  for (int s0 = 0; s0 < span.shares; s0 += 8) {  // eight shares' values under way together
    float v[8][E];
#pragma unroll
    for (int k = 0; k < 8; ++k)
#pragma unroll
      for (int e = 0; e < E; ++e) v[k][e] = part(min(s0 + k, span.shares - 1))[2 + lane * E + e];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int s = s0 + k;
      const float fade = s < span.shares ? __shfl(s < 64 ? f0 : f1, s & 63) : 0.0f;
#pragma unroll
      for (int e = 0; e < E; ++e) y[e] += v[k][e] * fade;
    }
  }
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  const int i = (int)(r / G), g = (int)(r % G);
  __bf16* out = static_cast<__bf16*>(P.out) + (ch.first + i) * P.out_stride + (int64_t)(h * G + g) * D;
#pragma unroll
  for (int e = 0; e < E; ++e) out[lane * E + e] = (__bf16)(y[e] * inv);
}

}  // namespace

namespace {
template <int SRC, bool F8>
void write(const KvParams& P, hipStream_t stream) {
  // Rows by tiles where sequences bring many.  us by row / by tile, 8 heads of 128:
  // into bfloat16, 32 sequences of 16 rows 8.8 / 9.3, of 24 9.2 / 9.2, of 32 11.0 /
  // 9.2, 4 of 512 17.9 / 9.6; into e4m3, 32 of 32 11.7 / 17.4, of 64 17.4 / 18.7, of
  // 128 28.4 / 22.1, 8 of 1000 51 / 30.
  if (P.rows >= (F8 ? 128 : 32) * (int64_t)P.B) {
    const dim3 grid((uint32_t)((P.rows + 63) / 64), P.H), block(256);
    if (P.D == 64) k_kv_write_tile<SRC, F8, 64><<<grid, block, 0, stream>>>(P);
    else if (P.D == 128) k_kv_write_tile<SRC, F8, 128><<<grid, block, 0, stream>>>(P);
    else k_kv_write_tile<SRC, F8, 256><<<grid, block, 0, stream>>>(P);
  } else {
    k_kv_write<SRC, F8><<<dim3((uint32_t)((P.rows + 3) / 4), P.H), 256, 0, stream>>>(P);
  }
}
template <int DST, bool F8>
void read(const KvParams& P, hipStream_t stream) {
  const dim3 grid((uint32_t)((P.L + 63) / 64), P.H, P.B), block(256);
  if (P.D == 64) k_kv_read<DST, F8, 64><<<grid, block, 0, stream>>>(P);
  else if (P.D == 128) k_kv_read<DST, F8, 128><<<grid, block, 0, stream>>>(P);
  else k_kv_read<DST, F8, 256><<<grid, block, 0, stream>>>(P);
}
}  // namespace

hipError_t launch_kv_write(const KvParams& P, int dtype, hipStream_t stream) {
  if (dtype == SPC_BF16) P.f8 ? write<SPC_BF16, true>(P, stream) : write<SPC_BF16, false>(P, stream);
  else P.f8 ? write<SPC_F32, true>(P, stream) : write<SPC_F32, false>(P, stream);
  return hipGetLastError();
}

hipError_t launch_kv_read(const KvParams& P, int dtype, hipStream_t stream) {
  if (dtype == SPC_BF16) P.f8 ? read<SPC_BF16, true>(P, stream) : read<SPC_BF16, false>(P, stream);
  else P.f8 ? read<SPC_F32, true>(P, stream) : read<SPC_F32, false>(P, stream);
  return hipGetLastError();
}

namespace {
template <int D, bool F8>
void attend(const KvParams& P, hipStream_t stream) {
  const int64_t rows = (int64_t)P.n * (P.heads / P.H);
  const int64_t groups = ((int64_t)P.H * P.B * P.splits + 7) / 8 * 8;
  const dim3 grid((uint32_t)((rows + P.tile_rows - 1) / P.tile_rows * groups));
  const dim3 block(64 * kAttendWaves);
  if (P.tile_rows == 16) k_kv_attend<D, F8, 1><<<grid, block, 0, stream>>>(P);
  else if (P.tile_rows == 128) k_kv_attend_rows<D, F8><<<grid, block, 0, stream>>>(P);
  else if constexpr (!F8 || D == 64) k_kv_attend<D, F8, 2><<<grid, block, 0, stream>>>(P);
  if (P.splits > 1) {
    const dim3 join((uint32_t)((rows + 3) / 4), P.H, P.B);
    if (P.tile_rows == 128)
      k_kv_join<D, rows_tile(D, F8), share_keys(128, F8)><<<join, 256, 0, stream>>>(P, 128);
    else
      k_kv_join<D, F8 ? 64 : 32, share_keys(64, F8)><<<join, 256, 0, stream>>>(P, P.tile_rows);
  }
}
}  // namespace

int kv_share_keys(int tile_rows, bool f8) { return share_keys(tile_rows, f8); }

hipError_t launch_kv_attend(const KvParams& P, hipStream_t stream) {
  if (P.D == 64) P.f8 ? attend<64, true>(P, stream) : attend<64, false>(P, stream);
  else if (P.D == 128) P.f8 ? attend<128, true>(P, stream) : attend<128, false>(P, stream);
  else P.f8 ? attend<256, true>(P, stream) : attend<256, false>(P, stream);
  return hipGetLastError();
}

}  // namespace spc
