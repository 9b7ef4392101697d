// spc_kv_attend.h -- the attention kernels over the paged key/value cache.
#pragma once

#include "spc_kv_device.h"

namespace spc {
namespace {

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


// The first position that a row at position t sees (under 0: from 0).  A row
// before position 0 sees nothing: it is taken as at 0, where no window of 32 bits
// passes them.
__device__ __forceinline__ int32_t first_seen(const KvParams& P, int32_t t) {
  return P.window > 0 ? max(t, 0) - P.window + 1 : 0;
}

// What rows attend to:
//   kOwn     the tokens of their sequence up to themselves
//   kBehind  those of them from P.from on
//   kCross   all tokens of their sequence whose mask byte is not 0
//   kShared  the first P.shared tokens (of P.table's only row) up to themselves;
//            the rows of all sequences are taken as those of one
enum AttendMode { kOwn, kBehind, kCross, kShared };

// A share of the keys has at least as many: a tile for each wavefront, or in
// k_kv_attend_rows, whose wavefronts take every tile together, 512 (of a shared
// prefix, which few workgroups take, behind it, where the shares are joined anyhow,
// and of an encoder's states, whose number the launch bounds instead, 256).  (One token
// over 1500 bfloat16 tokens of 8 heads: 13.9 us in shares of 512, 6.9 in shares of 128,
// and the join 4.4.  Behind a prefix, by 512 / 256: 40 rows of 8 sequences with up to
// 1000 tokens of their own, 32/8 heads of 128 in e4m3, 87 / 67; 64 rows of 4 with 1000,
// 16/4 heads of 256 in bfloat16, 120 / 103; where there are enough workgroups, 600 rows
// of 2 with 548, 16/4 heads of 128, 68 / 72.)
constexpr int share_keys(int tile_rows, bool f8, int mode = kOwn) {
  return tile_rows > 64 ? (mode != kOwn ? 256 : 512) : f8 ? 256 : 128;
}

// The tokens whose rows a launch is sized for, a sequence.
template <int MODE>
__device__ __forceinline__ int32_t tokens_of(const KvParams& P) {
  return MODE == kShared ? (int32_t)P.rows : P.n;
}
template <int MODE>
__device__ __forceinline__ Chunk rows_of(const KvParams& P, int b) {
  return MODE == kShared ? Chunk{0, (int32_t)P.rows} : chunk_of(P, b);
}
// Positions from here on are in no page (or, of kCross, past the mask).
template <int MODE>
__device__ __forceinline__ int32_t tokens_there(const KvParams& P, int32_t len) {
  const int32_t held = P.width * P.S;
  if (MODE == kShared) return min(P.shared, held);
  if (MODE == kCross && P.mask) return min(min(len, held), P.mask_width);
  return min(len, held);
}
// The new token of row r of a key/value head, G rows a token.
__device__ __forceinline__ int token_of(const KvParams& P, int G, int64_t r) {
  const uint32_t x = (uint32_t)r;  // (under 2^31: a launch has fewer than 2^24 tiles of rows)
  if (P.g_magic) return (int)__umulhi(x, P.g_magic);
  return (int)(G == 1 ? x : x / (uint32_t)G);
}
// The positions that row i of ch sees.
struct Limits {
  int32_t first, last;
};
template <int MODE>
__device__ __forceinline__ Limits limits_of(const KvParams& P, const Chunk& ch, int32_t len,
                                            int32_t there, int i) {
  if constexpr (MODE == kCross) return Limits{0, there - 1};
  if constexpr (MODE == kShared) {
    const int b = sequence_of(P, i);
    if (b < 0) return Limits{0, -1};
    const Chunk c = chunk_of(P, b);
    const int32_t t = max(P.len[b], 0) - c.n + (int32_t)(i - c.first);
    return Limits{first_seen(P, t), min(t, there - 1)};
  }
  const int32_t t = len - ch.n + i;
  return Limits{MODE == kBehind ? max(first_seen(P, t), P.from) : first_seen(P, t), t};
}

// The keys that rows of a chunk's tokens i0 .. i1 see: tiles of T from `begin`
// (a multiple of T), cut into shares of `per` tiles of at least `least` keys.  (Of
// kShared all: its shares are the same for every row.)
struct Span {
  int32_t begin, tiles, shares, per;
};
template <int MODE>
__device__ __forceinline__ Span span_of(const KvParams& P, int T, int least, int32_t len, int n,
                                        int i0, int i1, int splits) {
  const int32_t there = tokens_there<MODE>(P, len);
  const int32_t end = MODE <= kBehind ? min(there, len - n + i1 + 1) : there;
  Span s;
  s.begin = MODE <= kBehind
                ? max(first_seen(P, len - n + i0), MODE == kBehind ? P.from : 0) & ~(T - 1)
                : 0;
  s.tiles = end > s.begin ? (end - s.begin + T - 1) / T : 0;
  s.shares = max(1, min(splits, s.tiles / (least / T)));
  s.per = (s.tiles + s.shares - 1) / s.shares;
  return s;
}

// N bytes of a mask, those from the n-th on as zeros.
template <int N>
struct MaskBytes {
  uint32_t w[N / 4];
};
template <int N>
__device__ __forceinline__ MaskBytes<N> mask_bytes(const uint8_t* p, int n) {
  typedef uint32_t any_u32 __attribute__((aligned(1)));
  MaskBytes<N> m;
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    if (n >= 4 * i + 4) m.w[i] = *reinterpret_cast<const any_u32*>(p + 4 * i);
    else {
      m.w[i] = 0;
#pragma unroll
      for (int e = 0; e < 3; ++e)
        if (n > 4 * i + e) m.w[i] |= (uint32_t)p[4 * i + e] << (8 * e);
    }
  }
  return m;
}
// A bit a byte: whether it is not 0.
template <int N>
__device__ __forceinline__ uint32_t mask_bits(const MaskBytes<N>& m) {
  uint32_t bits = 0;
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    const uint32_t y = (((m.w[i] & 0x7f7f7f7fu) + 0x7f7f7f7fu) | m.w[i]) & 0x80808080u;
    // bits 7, 15, 23 and 31 to the lowest of the top byte, in their order
    bits |= ((y >> 7) * 0x01020408u >> 24 & 15u) << (4 * i);
  }
  return bits;
}
// Word j of sixteen bytes' values: ones where the value's bit is set.
template <bool F8>
__device__ __forceinline__ uint32_t word_mask(uint32_t bits, int j) {
  if constexpr (F8) return ((bits >> (4 * j) & 15u) * 0x00204081u & 0x01010101u) * 0xffu;
  const uint32_t b = bits >> (2 * j) & 3u;
  return (b & 1u) * 0xffffu | (b >> 1) * 0xffff0000u;
}

// Wavefronts a SIMD that registers are kept free for: two where they then do not
// spill.
constexpr int attend_waves(int D, bool f8, int mt) {
  return D <= 128 && mt * D <= (f8 ? 128 : 256) ? 2 : 1;
}

// Positions that some, and that all of a wavefront's rows see: from <= t < to.
struct Seen {
  int32_t from, to, all_from, all_to;
};
template <int MT>
__device__ __forceinline__ Seen seen_by(const int32_t (&first)[MT], const int32_t (&last)[MT]) {
  Seen s{0x7fffffff, 0, 0, 0x7fffffff};
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    s.from = min(s.from, max(first[mt], 0));
    s.to = max(s.to, last[mt] + 1);
    s.all_from = max(s.all_from, first[mt]);
    s.all_to = min(s.all_to, last[mt] + 1);
  }
#pragma unroll
  for (int d = 8; d; d >>= 1) {  // (lanes 16 j + c hold row c)
    s.from = min(s.from, __shfl_xor(s.from, d));
    s.to = max(s.to, __shfl_xor(s.to, d));
    s.all_from = max(s.all_from, __shfl_xor(s.all_from, d));
    s.all_to = min(s.all_to, __shfl_xor(s.all_to, d));
  }
  s.from = __builtin_amdgcn_readfirstlane(s.from);
  s.to = __builtin_amdgcn_readfirstlane(s.to);
  s.all_from = __builtin_amdgcn_readfirstlane(s.all_from);
  s.all_to = __builtin_amdgcn_readfirstlane(s.all_to);
  return s;
}

template <int D>
struct AttendLds {
  float o[kAttendWaves][16][D + 4];
  float m[kAttendWaves][16], l[kAttendWaves][16];
};

template <int D, bool F8, int MT, int MODE>
__device__ __forceinline__ void attend_few(const KvParams& P, uint32_t block, AttendLds<D>& lds) {
  constexpr int EB = F8 ? 1 : 2, T = F8 ? 64 : 32;
  constexpr int kQuarters = T / 16, kG = T / 4;  // score tiles; a lane's keys
  constexpr int kL = D * EB / 64;                // 16-byte loads of a key row by four lanes
  constexpr int kSteps = 2 / EB;                 // matrix steps in 16 bytes
  constexpr int kC = D / 32, kM = D / 16;
  auto& o_lds = lds.o;
  auto& m_lds = lds.m;
  auto& l_lds = lds.l;
  // Workgroups are dealt to the 8 dies in turn: those of one sequence and head
  // (and share of its keys) go to one die, whose cache then holds their keys, the
  // row tiles that see most keys first.
  const uint32_t tiles_x =
      (uint32_t)(((int64_t)tokens_of<MODE>(P) * (P.heads / P.H) + 16 * MT - 1) / (16 * MT));
  const uint32_t group = block / 8 / tiles_x * 8 + block % 8;
  const uint32_t tile_x = tiles_x - 1 - block / 8 % tiles_x;
  if (group >= (uint32_t)(P.H * (MODE == kShared ? 1 : P.B) * P.splits)) return;
  const int h = (int)(group % P.H), z = (int)(group / P.H), share = z % P.splits, b = z / P.splits;
  const int lane = threadIdx.x & 63, c16 = lane & 15, j = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const Chunk ch = rows_of<MODE>(P, b);
  const int G = P.heads / P.H;
  const int64_t rows = (int64_t)min(ch.n, tokens_of<MODE>(P)) * G, r0 = (int64_t)tile_x * (16 * MT);
  if (r0 >= rows) return;
  const int32_t len = MODE == kShared ? 0 : max(P.len[b], 0), there = tokens_there<MODE>(P, len);
  const int i0 = token_of(P, G, r0), i1 = token_of(P, G, min(r0 + 16 * MT, rows) - 1);
  const Span span =
      span_of<MODE>(P, T, share_keys(16 * MT, F8, MODE), len, ch.n, i0, i1, P.splits);
  if (share >= span.shares) return;
  int tile0 = share * span.per, tile1 = min(span.tiles, tile0 + span.per);

  bf16x8 q[MT][kC];
  int32_t last[MT], first[MT];  // the keys a row sees
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int64_t r = min(r0 + 16 * mt + c16, rows - 1);
    const int i = token_of(P, G, r), g = (int)(r - (int64_t)i * G);
    const int64_t q_at = (ch.first + i) * P.q_stride + (int64_t)(h * G + g) * D;
#pragma unroll
    for (int c = 0; c < kC; ++c) {
      const int d = c / kSteps * (32 * kSteps) + j * (8 * kSteps) + c % kSteps * 8;
      q[mt][c] = __builtin_bit_cast(
          bf16x8, u32x4(*reinterpret_cast<const u32x4a2*>(static_cast<const uint16_t*>(P.q) + q_at + d)));
    }
    const Limits seen = limits_of<MODE>(P, ch, len, there, i);
    last[mt] = seen.last;
    first[mt] = seen.first;
  }
  // a tile within these is seen whole by every row
  int32_t all_from, all_to;
  if constexpr (MODE == kShared) {
    const Seen seen = seen_by<MT>(first, last);
    all_from = seen.all_from;
    all_to = seen.all_to;
    tile0 = max(tile0, seen.from / T);  // (no other is seen by any)
    tile1 = min(tile1, (seen.to + T - 1) / T);
  } else {
    all_from = limits_of<MODE>(P, ch, len, there, i1).first;
    all_to = min(limits_of<MODE>(P, ch, len, there, i0).last + 1, there);
  }

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
    MaskBytes<kG> mask;
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
    if constexpr (MODE == kCross)
      if (P.mask)
        w.mask = mask_bytes<kG>(P.mask + b * P.mask_stride + (int32_t)ts, there - (int32_t)ts);
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
    bool whole = t0 >= all_from && t0 + T <= all_to && !now.any;
    const bool page = now.ps >= 0;
    uint32_t see = 0xffffffffu;  // of kCross: this lane's keys that are seen
    if constexpr (MODE == kCross) {
      const int live = page ? there - ts : 0;
      see = live <= 0 ? 0u : live >= kG ? (1u << kG) - 1u : (1u << live) - 1u;
      if (P.mask) see &= mask_bits(now.mask);
      whole = !__any(see != (1u << kG) - 1u);
    }
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
        for (int e = 0; e < kG; ++e) {
          if constexpr (MODE == kCross) x[e] = see >> e & 1u ? x[e] : kNegInf;
          else x[e] = ((ts + e <= hi) & (ts + e >= first[mt])) ? x[e] : kNegInf;
        }
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
    if (!whole) {  // what lies outside the keys (or is masked) may be anything, NaN too
      const int live = page ? there - ts : 0;
#pragma unroll
      for (int d = 0; d < kM; ++d) {
        if constexpr (MODE == kCross) {
#pragma unroll
          for (int i = 0; i < 4; ++i) vf[d][i] &= word_mask<F8>(see, i);
        } else {
          first_of<F8>(vf[d], live);
          if (MODE == kBehind && P.from > ts) without_first<F8>(vf[d], P.from - ts);
        }
      }
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
  const bool alone = MODE != kShared && MODE != kBehind && span.shares == 1;
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
        const int i = token_of(P, G, r), g = (int)(r - (int64_t)i * G);
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

template <int D, bool F8, int MT, int MODE>
__global__ void __launch_bounds__(64 * kAttendWaves, attend_waves(D, F8, MT))
    k_kv_attend(KvParams P) {
  __shared__ AttendLds<D> lds;
  attend_few<D, F8, MT, MODE>(P, blockIdx.x, lds);
}

// Where a tile of keys lies: its four lane groups' kG consecutive keys, each in one
// page.  All of it is the same for a wavefront, so pages are read and offsets are
// computed by the scalar unit, a tile ahead of the loads that need them, and a lane
// selects its group's.
template <int D, int EB, int kG>
struct TilePages {
  int32_t p[4];
  int64_t head[4];  // where the group's page holds the head, in bytes
  int32_t slot[4];  // of the group's first key
  uint32_t valid;   // a bit a group

  __device__ __forceinline__ static uint32_t index_of(const KvParams& P, uint32_t t) {
    return P.s16_magic ? __umulhi(t >> 4, P.s16_magic) : t >> 4;
  }
  __device__ __forceinline__ void fetch(const KvParams& P, const int32_t* table, int32_t there,
                                        int32_t t0) {
    typedef const __attribute__((address_space(4))) int32_t* Constant;
    const Constant of = (Constant)table;
#pragma unroll
    for (int g = 0; g < 4; ++g) p[g] = of[index_of(P, (uint32_t)min(t0 + kG * g, there - 1))];
  }
  // Waits for the pages here rather than at a read of LDS.
  __device__ __forceinline__ void arrive() {
#pragma unroll
    for (int g = 0; g < 4; ++g) asm volatile("" : "+s"(p[g]));
  }
  __device__ __forceinline__ void place(const KvParams& P, int h, int32_t there, int32_t t0) {
    valid = 0;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const uint32_t t = (uint32_t)(t0 + kG * g);
      const bool ok = (int32_t)t < there && (uint32_t)p[g] < (uint32_t)P.pages;
      valid |= (uint32_t)ok << g;
      slot[g] = (int32_t)(t - index_of(P, t) * (uint32_t)P.S);
      // (a cache has fewer than 2^32 pages of a head: one is 1 KiB at least)
      head[g] = (int64_t)((uint64_t)((ok ? (uint32_t)p[g] : 0u) * (uint32_t)P.H + (uint32_t)h) *
                          (uint32_t)(P.S * D * EB));
    }
  }
  template <class X>
  __device__ __forceinline__ static X select(X a, X b, X c, X d, int g) {
    const X lo = g & 1 ? b : a, hi = g & 1 ? d : c;
    return g & 2 ? hi : lo;
  }
  __device__ __forceinline__ int64_t head_of(int g) const {
    return select(head[0], head[1], head[2], head[3], g);
  }
  __device__ __forceinline__ int32_t slot_of(int g) const {
    return select(slot[0], slot[1], slot[2], slot[3], g);
  }
};

// Keys in a tile of k_kv_attend_rows.
constexpr int rows_tile(int D, bool f8) { return f8 || D <= 128 ? 64 : 32; }

// The same for chunks of many rows: a workgroup takes 128, each wavefront 32 of
// its own over all of the share's keys, so that a tile of keys and values is
// read once for 128 rows. Tiles pass through LDS, in bfloat16 (8 bits are widened
// once, as they are written) and in the order the lanes of the products want them (a
// wavefront's read is 1 KiB in a row, without conflicts), double-buffered: the next
// tile's are written behind the products of this one and the loads of the one after
// it are then under way.  A fragment is read four products' operands ahead.  What
// bounds it is that two wavefronts a SIMD do not keep the matrix unit under the
// softmax's vector instructions (about 300 a tile, 1300 of its cycles, where the
// products are 1024) and the LDS, whose reads of a tile take as long as the products
// with it: 4 chunks of 1024 rows over 4096 tokens, 32/8 heads of 128, take 323 us in
// bfloat16 (745 TFLOP/s) and 363 in e4m3; without the reads ahead and with values
// masked as they were read, 383 and 437 (by 406, 515 us with 32 keys a tile, 653 with
// 64 rows a workgroup and its wavefronts apart over the keys).  64 rows a wavefront,
// with the next tile's scores taken under this one's powers, 521 against 379 us where
// keys are shared: the accumulators do not stay in one register file.
template <int D, bool F8>
struct RowsLds {
  // 1 KiB fragments of keys, then of values, of two tiles, in bfloat16; scales of keys,
  // of values
  u32x4 frags[2][rows_tile(D, F8) * D * 4 / 1024][64];
  float scales[2][2][F8 ? rows_tile(D, F8) : 1];
  int32_t seen_from[kAttendWaves], seen_to[kAttendWaves];
};

template <int D, bool F8, int MODE>
__device__ __forceinline__ void attend_many(const KvParams& P, uint32_t block, RowsLds<D, F8>& lds) {
  constexpr int MT = 2, kRows = 16 * MT * kAttendWaves;
  constexpr int EB = F8 ? 1 : 2, T = rows_tile(D, F8);
  constexpr int kQuarters = T / 16, kG = T / 4;
  constexpr int kL = D * EB / 64, kSteps = 2 / EB, kC = D / 32, kM = D / 16;
  constexpr int kVL = T * EB / 64;                   // 16-byte loads of a lane's keys of V
  constexpr int kLoads = kQuarters * kL + kM * kVL;  // of 1 KiB: K's, then V's
  constexpr int kMine = kLoads / kAttendWaves;       // that a wavefront brings
  constexpr int kKeyFrags = kQuarters * kC, kFrags = kKeyFrags + kM * (T / 32);
  constexpr int kAhead = 4;                          // reads of LDS under way
  // The reference of a row's powers follows its maximum when that is more than
  // kSlack above (powers up to 2^8 are as exact): O is then multiplied rarely.  A
  // bfloat16 cache's scores are scaled within the power's argument, a negative scale
  // is taken as a positive one of negated queries.  (kOwn keeps the sums it always had.)
  constexpr float kSlack = MODE == kOwn ? 0.0f : 8.0f;
  constexpr bool kFused = MODE != kOwn && !F8;
  const uint32_t sign = kFused && P.scale < 0.0f ? 0x80008000u : 0u;
  const float scale = fmaxf(fabsf(P.scale), 1e-37f);  // (not 0, for minus infinity times it)
  static_assert(kQuarters * kL % kAttendWaves == 0 && kM * kVL % kAttendWaves == 0, "whole shares");
  static_assert(sizeof(lds.frags) == 2 * kFrags * 1024, "two tiles");
  auto& frags = lds.frags;
  auto& scales = lds.scales;
  const uint32_t tiles_x =
      (uint32_t)(((int64_t)tokens_of<MODE>(P) * (P.heads / P.H) + kRows - 1) / kRows);
  const uint32_t group = block / 8 / tiles_x * 8 + block % 8;
  const uint32_t tile_x = tiles_x - 1 - block / 8 % tiles_x;
  if (group >= (uint32_t)(P.H * (MODE == kShared ? 1 : P.B) * P.splits)) return;
  const int h = (int)(group % P.H), z = (int)(group / P.H), share = z % P.splits, b = z / P.splits;
  const int lane = threadIdx.x & 63, c16 = lane & 15, j = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const Chunk ch = rows_of<MODE>(P, b);
  const int G = P.heads / P.H;
  const int64_t rows = (int64_t)min(ch.n, tokens_of<MODE>(P)) * G, r0 = (int64_t)tile_x * kRows;
  if (r0 >= rows) return;
  const int32_t len = MODE == kShared ? 0 : max(P.len[b], 0), there = tokens_there<MODE>(P, len);
  const Span span =
      span_of<MODE>(P, T, share_keys(kRows, F8, MODE), len, ch.n, token_of(P, G, r0),
                    token_of(P, G, min(r0 + kRows, rows) - 1), P.splits);
  if (share >= span.shares) return;
  int tile0 = share * span.per, tile1 = min(span.tiles, tile0 + span.per);

  // this wavefront's rows (the last row again behind the end)
  const int64_t w0 = r0 + 16 * MT * wave;
  bf16x8 q[MT][kC];
  int32_t last[MT], first[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int64_t r = min(w0 + 16 * mt + c16, rows - 1);
    const int i = token_of(P, G, r), g = (int)(r - (int64_t)i * G);
    const int64_t q_at = (ch.first + i) * P.q_stride + (int64_t)(h * G + g) * D;
#pragma unroll
    for (int c = 0; c < kC; ++c) {
      const int d = c / kSteps * (32 * kSteps) + j * (8 * kSteps) + c % kSteps * 8;
      u32x4 w = *reinterpret_cast<const u32x4a2*>(static_cast<const uint16_t*>(P.q) + q_at + d);
      w ^= sign;
      q[mt][c] = __builtin_bit_cast(bf16x8, w);
    }
    const Limits seen = limits_of<MODE>(P, ch, len, there, i);
    last[mt] = seen.last;
    first[mt] = seen.first;
  }
  int32_t all_from, all_to;
  if constexpr (MODE == kShared) {
    auto& seen_from = lds.seen_from;
    auto& seen_to = lds.seen_to;
    const Seen seen = seen_by<MT>(first, last);
    all_from = seen.all_from;
    all_to = seen.all_to;
    if (lane == 0) {
      seen_from[wave] = seen.from;
      seen_to[wave] = seen.to;
    }
    __syncthreads();
    int32_t from = seen_from[0], to = seen_to[0];
#pragma unroll
    for (int w = 1; w < kAttendWaves; ++w) {
      from = min(from, seen_from[w]);
      to = max(to, seen_to[w]);
    }
    tile0 = max(tile0, __builtin_amdgcn_readfirstlane(from) / T);  // (no other is seen by any)
    tile1 = min(tile1, (__builtin_amdgcn_readfirstlane(to) + T - 1) / T);
  } else {
    const int i0 = token_of(P, G, min(w0, rows - 1));
    const int i1 = token_of(P, G, min(w0 + 16 * MT, rows) - 1);
    all_from = limits_of<MODE>(P, ch, len, there, i1).first;
    all_to = min(limits_of<MODE>(P, ch, len, there, i0).last + 1, there);
  }

  f32x4 o[MT][kM] = {};
  float m[MT] = {kNegInf, kNegInf}, l[MT] = {0.0f, 0.0f};
  const int32_t* table = P.table + (int64_t)b * P.width;
  // the fragments this wavefront brings of a tile at t0, and a lane's scale
  u32x4 mine[kMine];
  float my_scale = 0.0f;
  TilePages<D, EB, kG> pages;
  uint32_t valid_next = 0, valid_now = 0;  // groups of keys that are in a page
  int32_t ts_next = 0;                     // the first of this lane's own keys
  MaskBytes<kG> mask_next{};
  uint32_t see = 0;                        // of this tile: this lane's keys that are there
  const int lane_k = (c16 & 3) * D * EB + 16 * j + wave / kL * 4 * D * EB + wave % kL * 64;
  const int lane_v = (c16 + wave / kVL * 16) * P.S * EB + wave % kVL * 16;
  const int step_v = kAttendWaves / kVL * 16 * P.S * EB;
  const auto bring = [&](int32_t t0) {
    pages.place(P, h, there, t0);
    valid_next = pages.valid;
    ts_next = t0 + kG * j;
    if constexpr (MODE == kCross)
      if (P.mask) mask_next = mask_bytes<kG>(P.mask + b * P.mask_stride + ts_next, there - ts_next);
    const int gk = c16 >> 2;
    const char* k = static_cast<const char*>(P.k) + pages.head_of(gk) +
                    (pages.slot_of(gk) * (D * EB) + lane_k);
    const char* v = static_cast<const char*>(P.v) + pages.head_of(j) + (pages.slot_of(j) * EB + lane_v);
    constexpr int kKeys = kQuarters * kL / kAttendWaves;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {  // fragments wave, wave + 4, ...
      if (i < kKeys)
        mine[i] = load16(k, kAttendWaves * i / kL * 4 * D * EB + kAttendWaves * i % kL * 64);
      else mine[i] = load16(v, (int64_t)((i - kKeys) * step_v));
    }
    if constexpr (F8) {
      if (threadIdx.x < 2 * T) {  // a thread a key and kind
        const bool ok = t0 + lane < there && (pages.valid >> j & 1u);
        const int64_t at = pages.head_of(j) / D + pages.slot_of(j) + c16;
        my_scale = !ok ? 0.0f : threadIdx.x < T ? P.k_scale[at] * P.scale : P.v_scale[at];
      }
    }
  };
  const auto put = [&](int buf) {
    // values outside the keys (or masked) may be anything, NaN too: zeros instead
    constexpr uint32_t kAll = (1u << kG) - 1u;
    const int live = valid_next >> j & 1u ? there - ts_next : 0;
    see = live <= 0 ? 0u : live >= kG ? kAll : (1u << live) - 1u;
    if (MODE == kBehind && P.from > ts_next) see &= kAll << min(P.from - ts_next, kG);
    if constexpr (MODE == kCross)
      if (P.mask) see &= mask_bits(mask_next);
    if (__any(see != kAll)) {
#pragma unroll
      for (int i = kQuarters * kL / kAttendWaves; i < kMine; ++i) {
        const int part = (wave + i * kAttendWaves - kQuarters * kL) % kVL;
#pragma unroll
        for (int w = 0; w < 4; ++w) mine[i][w] &= word_mask<F8>(see >> (8 * part), w);
      }
    }
#pragma unroll
    for (int i = 0; i < kMine; ++i)
#pragma unroll
      for (int step = 0; step < kSteps; ++step)
        frags[buf][(wave + i * kAttendWaves) * kSteps + step][lane] =
            __builtin_bit_cast(u32x4, widen<F8>(mine[i], step));
    if constexpr (F8)
      if (threadIdx.x < 2 * T) scales[buf][threadIdx.x / T][threadIdx.x % T] = my_scale;
  };
  if (tile0 < tile1) {
    pages.fetch(P, table, there, span.begin + T * tile0);
    bring(span.begin + T * tile0);
    if (tile0 + 1 < tile1) pages.fetch(P, table, there, span.begin + T * (tile0 + 1));
    put(0);
    valid_now = valid_next;
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
    __builtin_amdgcn_s_setprio(1);
    {
      u32x4 ring[kAhead];
#pragma unroll
      for (int f = 0; f < kAhead; ++f) ring[f] = frags[buf][f][lane];
#pragma unroll
      for (int f = 0; f < kKeyFrags; ++f) {
        const bf16x8 k8 = __builtin_bit_cast(bf16x8, ring[f % kAhead]);
        if (f + kAhead < kKeyFrags) ring[f % kAhead] = frags[buf][f + kAhead][lane];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
          s[mt][f / kC] =
              __builtin_amdgcn_mfma_f32_16x16x32_bf16(k8, q[mt][f % kC], s[mt][f / kC], 0, 0, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x100, kAhead, 0);
#pragma unroll
      for (int f = 0; f < kKeyFrags; ++f) {
        __builtin_amdgcn_sched_group_barrier(0x8, MT, 0);
        if (f + kAhead < kKeyFrags) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
    }
    __builtin_amdgcn_s_setprio(0);
    if (tile + 2 < tile1) pages.fetch(P, table, there, t0 + 2 * T);
    const bool whole = MODE == kCross ? !__any(see != (1u << kG) - 1u)
                                      : t0 >= all_from && t0 + T <= all_to && valid_now == 15u;
    bf16x8 p[MT][kG / 8];
    float x[MT][kG], mx[MT];
    bool grows = false;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int e = 0; e < kG; ++e) {
        x[mt][e] = s[mt][e >> 2][e & 3];
        if constexpr (F8) x[mt][e] *= scales[buf][0][kG * j + e];
        else if constexpr (!kFused) x[mt][e] *= P.scale;
      }
    if (!whole) {  // uniform
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        const int32_t hi = valid_now >> j & 1u ? min(there - 1, last[mt]) : -1;
#pragma unroll
        for (int e = 0; e < kG; ++e) {
          if constexpr (MODE == kCross) x[mt][e] = see >> e & 1u ? x[mt][e] : kNegInf;
          else x[mt][e] = ((ts + e <= hi) & (ts + e >= first[mt])) ? x[mt][e] : kNegInf;
        }
      }
    }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      mx[mt] = x[mt][0];
#pragma unroll
      for (int e = 1; e < kG; ++e) mx[mt] = fmaxf(mx[mt], x[mt][e]);
      if constexpr (kFused) mx[mt] *= scale;
      grows |= mx[mt] > m[mt] + kSlack;
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
        float w = __builtin_amdgcn_exp2f(kFused ? fmaf(x[mt][e], scale, -base) : x[mt][e] - base);
        l[mt] += w;
        if constexpr (F8) {
          w *= scales[buf][1][kG * j + e];
          if (!whole) w = x[mt][e] == kNegInf ? 0.0f : w;  // (an unseen key's scale may be junk)
        }
        p[mt][e >> 3][e & 7] = (__bf16)w;
      }
    }
    if (tile + 2 < tile1) pages.arrive();
    __builtin_amdgcn_s_setprio(1);
    // (V's fragments: those of the next products are under way)
    constexpr int kValues = kM * (T / 32);
    u32x4 ring[kAhead];
#pragma unroll
    for (int f = 0; f < kAhead; ++f) ring[f] = frags[buf][kKeyFrags + f][lane];
#pragma unroll
    for (int f = 0; f < kValues; ++f) {
      const int d = f / (T / 32), part = f % (T / 32);
      const bf16x8 v8 = __builtin_bit_cast(bf16x8, ring[f % kAhead]);
      if (f + kAhead < kValues) ring[f % kAhead] = frags[buf][kKeyFrags + f + kAhead][lane];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
        o[mt][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v8, p[mt][part], o[mt][d], 0, 0, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x100, kAhead, 0);
#pragma unroll
    for (int f = 0; f < kValues; ++f) {
      __builtin_amdgcn_sched_group_barrier(0x8, MT, 0);
      if (f + kAhead < kValues) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_s_setprio(0);
    // (the buffer written here was last read before the last barrier)
    if (tile + 1 < tile1) {
      put(buf ^ 1);
      valid_now = valid_next;
      if (tile + 2 < tile1) bring(t0 + 2 * T);
    }
    __syncthreads();
  }

  const bool alone = MODE != kShared && MODE != kBehind && span.shares == 1;
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    l[mt] += __shfl_xor(l[mt], 16);
    l[mt] += __shfl_xor(l[mt], 32);
    const int64_t r = w0 + 16 * mt + c16;
    if (r >= rows) continue;
    if (alone) {
      const float inv = l[mt] == 0.0f ? 0.0f : 1.0f / l[mt];
      const int i = token_of(P, G, r), g = (int)(r - (int64_t)i * G);
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

template <int D, bool F8, int MODE>
__global__ void __launch_bounds__(64 * kAttendWaves, D <= 128 ? 2 : 1) k_kv_attend_rows(KvParams P) {
  __shared__ RowsLds<D, F8> lds;
  attend_many<D, F8, MODE>(P, blockIdx.x, lds);
}

// The shares of a row joined, in their order: a wavefront a row.
template <int D, int MODE>
__global__ void __launch_bounds__(256) k_kv_join(KvParams P, int tile_rows, int T, int least) {
  const int b = blockIdx.z, h = blockIdx.y, lane = threadIdx.x & 63;
  const Chunk ch = chunk_of(P, b);
  const int G = P.heads / P.H;
  const int64_t rows = (int64_t)min(ch.n, P.n) * G;
  const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (r >= rows) return;
  const int64_t x = r / tile_rows, tiles_x = ((int64_t)P.n * G + tile_rows - 1) / tile_rows;
  const int64_t r0 = x * tile_rows;
  const Span span = span_of<MODE>(P, T, least, max(P.len[b], 0), ch.n, token_of(P, G, r0),
                                  token_of(P, G, min(r0 + tile_rows, rows) - 1), P.splits);
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
  const int i = token_of(P, G, r), g = (int)(r - (int64_t)i * G);
  __bf16* out = static_cast<__bf16*>(P.out) + (ch.first + i) * P.out_stride + (int64_t)(h * G + g) * D;
#pragma unroll
  for (int e = 0; e < E; ++e) out[lane * E + e] = (__bf16)(y[e] * inv);
}

// Keys in a tile of the kernel that takes tile_rows rows.
constexpr int tile_keys(int D, bool f8, int tile_rows) {
  return tile_rows > 64 ? rows_tile(D, f8) : f8 ? 64 : 32;
}

// Workgroups of a launch: a multiple of the 8 dies.
template <int MODE>
uint32_t attend_blocks(const KvParams& P) {
  const int64_t rows = (int64_t)(MODE == kShared ? P.rows : P.n) * (P.heads / P.H);
  const int64_t groups = ((int64_t)P.H * (MODE == kShared ? 1 : P.B) * P.splits + 7) / 8 * 8;
  return (uint32_t)((rows + P.tile_rows - 1) / P.tile_rows * groups);
}

template <int D, bool F8, int MODE>
void attend_shares(const KvParams& P, hipStream_t stream) {
  const dim3 grid(attend_blocks<MODE>(P));
  const dim3 block(64 * kAttendWaves);
  if (P.tile_rows == 128) k_kv_attend_rows<D, F8, MODE><<<grid, block, 0, stream>>>(P);
  else if (P.tile_rows == 16) k_kv_attend<D, F8, 1, MODE><<<grid, block, 0, stream>>>(P);
  else if constexpr (!F8 || D == 64) k_kv_attend<D, F8, 2, MODE><<<grid, block, 0, stream>>>(P);
}

template <int D, bool F8, int MODE>
void attend(const KvParams& P, hipStream_t stream) {
  attend_shares<D, F8, MODE>(P, stream);
  if (P.splits > 1) {
    const int64_t rows = (int64_t)P.n * (P.heads / P.H);
    const dim3 join((uint32_t)((rows + 3) / 4), P.H, P.B);
    k_kv_join<D, MODE><<<join, 256, 0, stream>>>(P, P.tile_rows, tile_keys(D, F8, P.tile_rows),
                                                 share_keys(P.tile_rows, F8, MODE));
  }
}

}  // namespace
}  // namespace spc
