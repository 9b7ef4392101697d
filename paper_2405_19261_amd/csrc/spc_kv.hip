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
#include "spc_kv_attend.h"

namespace spc {
namespace {

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

int kv_share_keys(int tile_rows, bool f8, bool shared) {
  return share_keys(tile_rows, f8, shared ? kShared : kOwn);
}

hipError_t launch_kv_attend(const KvParams& P, hipStream_t stream) {
  if (P.D == 64) P.f8 ? attend<64, true, kOwn>(P, stream) : attend<64, false, kOwn>(P, stream);
  else if (P.D == 128) P.f8 ? attend<128, true, kOwn>(P, stream) : attend<128, false, kOwn>(P, stream);
  else P.f8 ? attend<256, true, kOwn>(P, stream) : attend<256, false, kOwn>(P, stream);
  return hipGetLastError();
}

}  // namespace spc
