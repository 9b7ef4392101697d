// spc_kv.hip -- gfx950 kernels of the paged key/value cache: writing new
// tokens (in bfloat16 or quantised to e4m3), reading tokens back, and the
// attention of a chunk of new tokens over the cache.
//
// A page holds S consecutive tokens of one sequence, keys as [H][S][D] and
// values as [H][D][S]: transposed, because the attention's second product
// takes V^T as the left operand of a matrix instruction, whose lanes then load
// eight consecutive tokens of one dimension with one instruction, as they load
// eight dimensions of one key.  No operand passes through LDS.
#include <math.h>

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
  const int p = P.table[(int64_t)b * P.width + t / P.S];
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

template <bool F8>
__device__ __forceinline__ float cached(const void* p, int64_t i) {
  if constexpr (F8)
    return __builtin_amdgcn_cvt_f32_fp8((uint32_t)static_cast<const uint8_t*>(p)[i], 0);
  else return __uint_as_float((uint32_t)static_cast<const uint16_t*>(p)[i] << 16);
}
template <int DST>
__device__ __forceinline__ void dense(void* p, int64_t i, float x) {
  if constexpr (DST == SPC_BF16) static_cast<__bf16*>(p)[i] = (__bf16)x;
  else static_cast<float*>(p)[i] = x;
}

// A wavefront per (position, head).
template <int DST, bool F8>
__global__ void __launch_bounds__(256) k_kv_read(KvParams P) {
  const int lane = threadIdx.x & 63;
  const int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int h = blockIdx.y, b = blockIdx.z;
  if (t >= P.L) return;
  const int64_t w = ((int64_t)b * P.L + t) * P.H + h;
  const int page = t < P.len[b] ? page_of(P, b, t) : -1;
  if (page < 0) return;
  const int slot = (int)(t % P.S);
  const int64_t head = (int64_t)page * P.H + h;
  const float ks = F8 ? P.k_scale[head * P.S + slot] : 1.0f;
  const float vs = F8 ? P.v_scale[head * P.S + slot] : 1.0f;
  for (int d = lane; d < P.D; d += 64) {
    dense<DST>(P.k_out, w * P.D + d, cached<F8>(P.k, (head * P.S + slot) * P.D + d) * ks);
    dense<DST>(P.v_out, w * P.D + d, cached<F8>(P.v, (head * P.D + d) * P.S + slot) * vs);
  }
}

// Eight consecutive cached values as bfloat16 (exact for e4m3).
template <bool F8>
struct Frag {
  uint32_t w[F8 ? 2 : 4];
};
template <bool F8>
__device__ __forceinline__ Frag<F8> load_frag(const void* p, int64_t i) {
  Frag<F8> f;
  if constexpr (F8) {
    const u32x2 x = *reinterpret_cast<const u32x2*>(static_cast<const uint8_t*>(p) + i);
    f.w[0] = x.x; f.w[1] = x.y;
  } else {
    const u32x4 x = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(p) + i);
    f.w[0] = x.x; f.w[1] = x.y; f.w[2] = x.z; f.w[3] = x.w;
  }
  return f;
}
__device__ __forceinline__ bf16x8 widen(const Frag<false>& f) {
  const u32x4 x{f.w[0], f.w[1], f.w[2], f.w[3]};
  return __builtin_bit_cast(bf16x8, x);
}
__device__ __forceinline__ bf16x8 widen(const Frag<true>& f) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f.w[0], 1.0f, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f.w[0], 1.0f, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f.w[1], 1.0f, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f.w[1], 1.0f, true);
  return bf16x8{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}
// The first `n` of eight values, zeros behind them (n may be negative).
template <bool F8>
__device__ __forceinline__ void first_of(Frag<F8>& f, int n) {
  constexpr int kPer = F8 ? 4 : 2, kBits = 32 / kPer;
#pragma unroll
  for (int j = 0; j < 8 / kPer; ++j) {
    const int m = n - j * kPer;
    f.w[j] = m >= kPer ? f.w[j] : m <= 0 ? 0u : f.w[j] & ((1u << (m * kBits)) - 1u);
  }
}

// Attention of 16 rows by one wavefront.  The rows of a key/value head are the
// pairs (new token i, query head g of the head's group), i first.  Scores are
// taken transposed, S^T = K Q^T, in tiles of 32 keys: lane 16 j + c then holds
// row c's scores of keys 8 j .. 8 j + 7, which is what the second product
// O^T = V^T P^T wants of it as right operand: neither P nor the running
// maximum and sum of a row ever moves between lanes but for the row's own
// reductions over j.  Statistics and O are held in 32 bits; P is rounded to
// bfloat16 (by at most 2^-8) for the matrix unit, its sum is of the values before that.
template <int D, bool F8>
__global__ void __launch_bounds__(64) k_kv_attend(KvParams P) {
  constexpr int kC = D / 32, kM = D / 16;
  const int b = blockIdx.z, h = blockIdx.y;
  const int lane = threadIdx.x, c16 = lane & 15, j = lane >> 4;
  const Chunk ch = chunk_of(P, b);
  const int G = P.heads / P.H;
  const int64_t rows = (int64_t)min(ch.n, P.n) * G, r0 = (int64_t)blockIdx.x * 16;
  if (r0 >= rows) return;
  const int64_t r = min(r0 + c16, rows - 1);
  const bool live = r0 + c16 < rows;
  const int i = (int)(r / G), g = (int)(r % G);
  const int64_t q_at = (ch.first + i) * P.q_stride + (int64_t)(h * G + g) * D;
  bf16x8 q[kC];
#pragma unroll
  for (int c = 0; c < kC; ++c)
    q[c] = __builtin_bit_cast(bf16x8, u32x4(*reinterpret_cast<const u32x4a2*>(
                                          static_cast<const uint16_t*>(P.q) + q_at + 32 * c + 8 * j)));
  const int64_t len = P.len[b];
  const int64_t there = min(len, (int64_t)P.width * P.S);  // tokens the table holds
  const int64_t last = len - ch.n + i;                     // the row's own position
  const int64_t first = P.window > 0 ? last - P.window + 1 : 0;
  // keys of the tile's first and last row bound the loop
  const int64_t i_end = (min(r0 + 16, rows) - 1) / G;
  const int64_t end = min(there, len - ch.n + i_end + 1);
  const int64_t begin = P.window > 0 ? max(len - ch.n + r0 / G - P.window + 1, (int64_t)0) : 0;
  f32x4 o[kM] = {};
  float m = kNegInf, l = 0.0f;
  for (int64_t t0 = begin & ~(int64_t)31; t0 < end; t0 += 32) {
    // the pages of this lane's key (as a row of K) and of its eight keys
    const int64_t tk = t0 + 8 * (c16 >> 2) + (c16 & 3), ts = t0 + 8 * j;
    const int pk = tk < there ? page_of(P, b, tk) : -1;
    const int ps = ts < there ? page_of(P, b, ts) : -1;
    const int64_t hk = ((int64_t)max(pk, 0) * P.H + h) * P.S * D + (pk < 0 ? 0 : tk % P.S) * D;
    const int64_t hs = (int64_t)max(ps, 0) * P.H + h;
    f32x4 s[2] = {};
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int c = 0; c < kC; ++c)
        s[half] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            widen(load_frag<F8>(P.k, hk + (pk < 0 ? 0 : 4 * half) * D + 32 * c + 8 * j)), q[c],
            s[half], 0, 0, 0);
    float x[8], vs[8];
    const int slot = (int)(ts % P.S);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float k_scale = P.scale;
      vs[e] = 1.0f;
      if constexpr (F8) {
        k_scale *= P.k_scale[hs * P.S + slot + e];
        vs[e] = P.v_scale[hs * P.S + slot + e];
      }
      const int64_t t = ts + e;
      const bool seen = ps >= 0 && t < there && t <= last && t >= first;
      x[e] = seen ? s[e >> 2][e & 3] * k_scale : kNegInf;
      if (!seen) vs[e] = 0.0f;
    }
    float mx = x[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) mx = fmaxf(mx, x[e]);
    mx = fmaxf(mx, __shfl_xor(mx, 16));
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    const float m_new = fmaxf(m, mx);
    const float base = m_new == kNegInf ? 0.0f : m_new;  // (nothing seen yet)
    const float fade = __builtin_amdgcn_exp2f(m - base);
    m = m_new;
    l *= fade;
    bf16x8 p;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float w = __builtin_amdgcn_exp2f(x[e] - base);
      l += w;
      p[e] = (__bf16)(w * vs[e]);
    }
    const int live_keys = ps < 0 ? 0 : (int)min(there - ts, (int64_t)8);
#pragma unroll
    for (int mt = 0; mt < kM; ++mt) {
      Frag<F8> v = load_frag<F8>(P.v, (hs * D + 16 * mt + c16) * P.S + slot);
      first_of<F8>(v, live_keys);  // what lies behind may be anything, NaN too
      o[mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(v), p, o[mt] * fade, 0, 0, 0);
    }
  }
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  if (!live) return;
  const float inv = l > 0.0f ? 1.0f / l : 0.0f;
  uint16_t* out = static_cast<uint16_t*>(P.out) + (ch.first + i) * P.out_stride + (int64_t)(h * G + g) * D;
#pragma unroll
  for (int mt = 0; mt < kM; ++mt) {
    bf16x4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = (__bf16)(o[mt][e] * inv);
    *reinterpret_cast<u32x2a2*>(out + 16 * mt + 4 * j) = __builtin_bit_cast(u32x2, y);
  }
}

}  // namespace

hipError_t launch_kv_write(const KvParams& P, int dtype, hipStream_t stream) {
  const dim3 grid((uint32_t)((P.rows + 3) / 4), P.H), block(256);
  if (dtype == SPC_BF16) {
    if (P.f8) k_kv_write<SPC_BF16, true><<<grid, block, 0, stream>>>(P);
    else k_kv_write<SPC_BF16, false><<<grid, block, 0, stream>>>(P);
  } else {
    if (P.f8) k_kv_write<SPC_F32, true><<<grid, block, 0, stream>>>(P);
    else k_kv_write<SPC_F32, false><<<grid, block, 0, stream>>>(P);
  }
  return hipGetLastError();
}

hipError_t launch_kv_read(const KvParams& P, int dtype, hipStream_t stream) {
  const dim3 grid((uint32_t)((P.L + 3) / 4), P.H, P.B), block(256);
  if (dtype == SPC_BF16) {
    if (P.f8) k_kv_read<SPC_BF16, true><<<grid, block, 0, stream>>>(P);
    else k_kv_read<SPC_BF16, false><<<grid, block, 0, stream>>>(P);
  } else {
    if (P.f8) k_kv_read<SPC_F32, true><<<grid, block, 0, stream>>>(P);
    else k_kv_read<SPC_F32, false><<<grid, block, 0, stream>>>(P);
  }
  return hipGetLastError();
}

namespace {
template <int D>
void attend(const KvParams& P, hipStream_t stream) {
  const int G = P.heads / P.H;
  const dim3 grid((uint32_t)(((int64_t)P.n * G + 15) / 16), P.H, P.B), block(64);
  if (P.f8) k_kv_attend<D, true><<<grid, block, 0, stream>>>(P);
  else k_kv_attend<D, false><<<grid, block, 0, stream>>>(P);
}
}  // namespace

hipError_t launch_kv_attend(const KvParams& P, hipStream_t stream) {
  if (P.D == 64) attend<64>(P, stream);
  else if (P.D == 128) attend<128>(P, stream);
  else attend<256>(P, stream);
  return hipGetLastError();
}

}  // namespace spc
