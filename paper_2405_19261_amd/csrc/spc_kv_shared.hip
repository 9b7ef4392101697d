// spc_kv_shared.hip -- gfx950 kernels of the attentions whose rows share keys: to
// an encoder's states, and of a batch behind one prefix.
//
// Cross attention is the cache's attention with one limit for all rows and a byte a
// key that may mask it: bits a lane, taken once a tile; a masked key's score is minus
// infinity and its value zero, whatever the page holds.  Bound by the bytes of the
// cache where rows are few (up to 6 rows of 32 sequences to 544 tokens on average, 16
// heads of 64: 19 us, 3.8 TB/s), in 8 bits by widening them (8 rows of 16 sequences to 4096
// masked tokens, 32/8 heads of 128: 39 us, 3.6 TB/s), and by the matrix unit and the
// softmax together where rows are many (even chunks of 1024 rows 717 to 862 TFLOP/s).
//
// Behind a prefix, softmax statistics join: (m, l, o) of the prefix's keys and of a
// sequence's own give m = max, l = sum l_i 2^(m_i - m), o = sum o_i 2^(m_i - m) / l.
// So the prefix is one sequence whose rows are those of all, and is read once.
#include "spc_kv_attend.h"

namespace spc {
namespace {

// The shares of a row of a batch behind a prefix: the prefix's (taken for the
// rows of all sequences together), then those of its own tokens, joined in
// that order by a wavefront.  own.splits = 0: no sequence has tokens of its own.
// (10 us for 8 rows of 32 sequences of 32 heads of 128, ten shares each: 4.3 TB/s.)
template <int D>
__global__ void __launch_bounds__(256) k_shared_join(KvParams own, KvParams pre, int own_T,
                                                     int own_least, int pre_T, int pre_least) {
  const int b = blockIdx.z, h = blockIdx.y, lane = threadIdx.x & 63;
  const Chunk ch = chunk_of(own, b);
  const int G = own.heads / own.H;
  const int64_t rows = (int64_t)min(ch.n, own.n) * G;
  const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (r >= rows) return;
  const int shares_pre = span_of<kShared>(pre, pre_T, pre_least, 0, 0, 0, 0, pre.splits).shares;
  int shares_own = 0;
  const int64_t x = r / own.tile_rows, r0 = x * own.tile_rows;
  if (own.splits)
    shares_own = span_of<kBehind>(own, own_T, own_least, max(own.len[b], 0), ch.n, token_of(own, G, r0),
                               token_of(own, G, min(r0 + own.tile_rows, rows) - 1), own.splits)
                     .shares;
  const int shares = shares_pre + shares_own;
  // shares lie `step` floats apart, from the row's first one
  const int64_t tiles_own = ((int64_t)own.n * G + own.tile_rows - 1) / own.tile_rows;
  const int64_t tiles_pre = (pre.rows * G + pre.tile_rows - 1) / pre.tile_rows;
  const int64_t row_pre = ch.first * G + r;
  const float* of_pre = pre.part + (h * tiles_pre * pre.tile_rows + row_pre) * (D + 2);
  const int64_t step_pre = (int64_t)own.H * tiles_pre * pre.tile_rows * (D + 2);
  const float* of_own =
      own.part + (((int64_t)b * own.splits * own.H + h) * tiles_own * own.tile_rows + r) * (D + 2);
  const int64_t step_own = (int64_t)own.H * tiles_own * own.tile_rows * (D + 2);
  const auto part = [&](int s) {
    return s < shares_pre ? of_pre + s * step_pre : of_own + (s - shares_pre) * step_own;
  };
  // sixteen shares' values under way together, the first of them with the statistics
  constexpr int E = D / 64, kAtOnce = 16;
  float v[kAtOnce][E];
  const auto load = [&](int s0) {
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k)
      if (s0 + k < shares)  // uniform
#pragma unroll
        for (int e = 0; e < E; ++e) v[k][e] = part(s0 + k)[2 + lane * E + e];
  };
  // the shares' maxima and sums, four a lane
  static_assert(kKvShares == 128, "both together at most four a lane");
  float f[4], l[4], sum = 0.0f, top = kNegInf;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const bool there = lane + 64 * k < shares;
    f[k] = there ? part(lane + 64 * k)[0] : kNegInf;
    l[k] = there ? part(lane + 64 * k)[1] : 0.0f;
  }
  load(0);
#pragma unroll
  for (int k = 0; k < 4; ++k) top = fmaxf(top, f[k]);
#pragma unroll
  for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    f[k] = f[k] == kNegInf ? 0.0f : __builtin_amdgcn_exp2f(f[k] - top);
    sum += l[k] * f[k];
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
  float y[E] = {};
  for (int s0 = 0; s0 < shares; s0 += kAtOnce) {
    if (s0) load(s0);
    const float of_lane = s0 < 64 ? f[0] : s0 < 128 ? f[1] : s0 < 192 ? f[2] : f[3];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      if (s0 + k >= shares) break;  // uniform
      const float fade = __shfl(of_lane, (s0 + k) & 63);
#pragma unroll
      for (int e = 0; e < E; ++e) y[e] += v[k][e] * fade;
    }
  }
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  const int i = token_of(own, G, r), g = (int)(r - (int64_t)i * G);
  __bf16* out =
      static_cast<__bf16*>(own.out) + (ch.first + i) * own.out_stride + (int64_t)(h * G + g) * D;
#pragma unroll
  for (int e = 0; e < E; ++e) out[lane * E + e] = (__bf16)(y[e] * inv);
}

// Both attentions in one launch, the prefix's workgroups first: apart, the card
// drains between them, and neither fills it (32 sequences of one token behind 8192,
// 260 of their own on average, 32/8 heads of 128, bfloat16: 25 and 15 us apart, 22
// together, at 3.1 TB/s: the few tiles of each workgroup do not cover its start; 64
// rows of 4 sequences behind 4000 with 1000 of their own, 16/4 heads of 256, 140 a
// call apart, 120 together; 256 rows of 4 behind 2048, up to 2048 of their own, 32/8
// heads of 128, 118 and 99).
template <int D, bool F8, int PRE, int OWN>
__global__ void __launch_bounds__(64 * kAttendWaves, D <= 128 ? 2 : 1)
    k_shared_both(KvParams own, KvParams pre, uint32_t pre_blocks) {
  static_assert(OWN <= 2 || PRE > 2, "many rows of a sequence are many of all");
  constexpr size_t kRows = PRE > 2 ? sizeof(RowsLds<D, F8>) : 0;
  constexpr size_t kBytes = kRows > sizeof(AttendLds<D>) ? kRows : sizeof(AttendLds<D>);
  __shared__ __align__(16) char lds[kBytes];
  if (blockIdx.x < pre_blocks) {
    if constexpr (PRE > 2)
      attend_many<D, F8, kShared>(pre, blockIdx.x, *reinterpret_cast<RowsLds<D, F8>*>(lds));
    else
      attend_few<D, F8, PRE, kShared>(pre, blockIdx.x, *reinterpret_cast<AttendLds<D>*>(lds));
  } else if constexpr (OWN > 2) {
    attend_many<D, F8, kBehind>(own, blockIdx.x - pre_blocks,
                                *reinterpret_cast<RowsLds<D, F8>*>(lds));
  } else {
    attend_few<D, F8, OWN, kBehind>(own, blockIdx.x - pre_blocks,
                                    *reinterpret_cast<AttendLds<D>*>(lds));
  }
}

// Rows of a workgroup in sixteens: 1 or 8 of the prefix, 1, 2 or 8 of the others.
template <int D, bool F8, int PRE, int OWN>
void both(const KvParams& own, const KvParams& pre, hipStream_t stream) {
  const uint32_t pre_blocks = attend_blocks<kShared>(pre);
  const uint32_t own_blocks = own.splits ? attend_blocks<kBehind>(own) : 0;
  k_shared_both<D, F8, PRE, OWN>
      <<<pre_blocks + own_blocks, 64 * kAttendWaves, 0, stream>>>(own, pre, pre_blocks);
}

template <int D, bool F8>
void shared(const KvParams& own, const KvParams& pre, hipStream_t stream) {
  if (own.tile_rows == 128) {
    both<D, F8, 8, 8>(own, pre, stream);
  } else if (pre.tile_rows == 128) {
    if (own.tile_rows == 16) both<D, F8, 8, 1>(own, pre, stream);
    else if constexpr (!F8 || D == 64) both<D, F8, 8, 2>(own, pre, stream);
  } else if (own.tile_rows == 16) {
    both<D, F8, 1, 1>(own, pre, stream);
  } else if constexpr (!F8 || D == 64) {
    both<D, F8, 1, 2>(own, pre, stream);
  }
  const int64_t rows = (int64_t)own.n * (own.heads / own.H);
  k_shared_join<D><<<dim3((uint32_t)((rows + 3) / 4), own.H, own.B), 256, 0, stream>>>(
      own, pre, tile_keys(D, F8, own.tile_rows), share_keys(own.tile_rows, F8, kBehind),
      tile_keys(D, F8, pre.tile_rows), share_keys(pre.tile_rows, F8, kShared));
}

}  // namespace

hipError_t launch_kv_attend_shared(const KvParams& own, const KvParams& pre, hipStream_t stream) {
  if (own.D == 64) own.f8 ? shared<64, true>(own, pre, stream) : shared<64, false>(own, pre, stream);
  else if (own.D == 128)
    own.f8 ? shared<128, true>(own, pre, stream) : shared<128, false>(own, pre, stream);
  else own.f8 ? shared<256, true>(own, pre, stream) : shared<256, false>(own, pre, stream);
  return hipGetLastError();
}

hipError_t launch_cross_attend(const KvParams& P, hipStream_t stream) {
  if (P.D == 64) P.f8 ? attend<64, true, kCross>(P, stream) : attend<64, false, kCross>(P, stream);
  else if (P.D == 128)
    P.f8 ? attend<128, true, kCross>(P, stream) : attend<128, false, kCross>(P, stream);
  else P.f8 ? attend<256, true, kCross>(P, stream) : attend<256, false, kCross>(P, stream);
  return hipGetLastError();
}

}  // namespace spc
