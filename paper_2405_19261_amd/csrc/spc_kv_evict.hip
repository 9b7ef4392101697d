// spc_kv_evict.hip -- gfx950 kernels that keep a paged cache bounded: the attention
// weight that cached tokens get from new ones, and the tokens of the largest
// weights into other pages.
#include <algorithm>

#include "spc_kv_attend.h"

namespace spc {
namespace {

// ------------------------------------------------------------------ weights
// A[t] += sum over the rows (new token, query head) of a key/value head of
// softmax_t(scale q.k_t), in two steps: every row's largest score and its sum of
// 2^(score - largest), over shares of the keys, then the sums over rows.  Where
// rows are few, the first step leaves the scores in the workspace (4 bytes a row
// and key, against 2 D of the key) and the second reads these (k_weigh_rows,
// k_weigh_sum); where they are many, it takes the products again with a tile of
// keys in registers (k_weigh_tile, k_weigh_keys), and scores are never stored.
// Each weight is one workgroup's, its rows always added in one order: no atomics.
// Few rows are bound by the bytes of the keys (one token of 32 sequences over 4096, 8
// heads of 128 in bfloat16: 48 us, 5.6 TB/s, and 7 for the second step), many by the
// vector instructions of two softmaxes (34 to 43 % of the cycles) and uneven lengths,
// with the start of workgroups that have few tiles (up to 32 tokens of 4 sequences over
// up to 16384 in e4m3: 29 and 30 us at 1.5 wavefronts a SIMD, where the products are 5
// and the bytes 9; 600 tokens of 2 over 2048: 22, 27 and 5).

// The first step: as k_kv_attend, without values.
template <int D, bool F8, int MT>
__global__ void __launch_bounds__(64 * kAttendWaves, D <= 128 && MT * (F8 ? 2 : 1) < 4 ? 4 : 2)
    k_weigh_rows(KvParams P) {
  constexpr int EB = F8 ? 1 : 2, T = F8 ? 64 : 32;
  constexpr int kQuarters = T / 16, kG = T / 4;
  constexpr int kL = D * EB / 64, kSteps = 2 / EB, kC = D / 32;
  __shared__ float m_lds[kAttendWaves][16 * MT], l_lds[kAttendWaves][16 * MT];
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
  const int32_t len = max(P.len[b], 0), there = tokens_there<kOwn>(P, len);
  const int i0 = token_of(P, G, r0), i1 = token_of(P, G, min(r0 + 16 * MT, rows) - 1);
  const Span span = span_of<kOwn>(P, T, share_keys(16 * MT, F8), len, ch.n, i0, i1, P.splits);
  if (share >= span.shares) return;
  const int tile0 = share * span.per, tile1 = min(span.tiles, tile0 + span.per);

  bf16x8 q[MT][kC];
  int32_t last[MT], first[MT];
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
    const Limits seen = limits_of<kOwn>(P, ch, len, there, i);
    last[mt] = seen.last;
    first[mt] = seen.first;
  }
  const int32_t all_from = limits_of<kOwn>(P, ch, len, there, i1).first;
  const int32_t all_to = min(limits_of<kOwn>(P, ch, len, there, i0).last + 1, there);

  float m[MT], l[MT];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    m[mt] = kNegInf;
    l[mt] = 0.0f;
  }
  const int32_t* table = P.table + (int64_t)b * P.width;
  const auto index_of = [&](uint32_t t) {
    return P.s16_magic ? __umulhi(t >> 4, P.s16_magic) : t >> 4;
  };
  const auto page_at = [&](int32_t t) {
    const int p = table[index_of((uint32_t)min(t, there - 1))];
    return t < there && (uint32_t)p < (uint32_t)P.pages ? p : -1;
  };
  const int key = kG * (c16 >> 2);
  u32x4 kf[kQuarters][kL];
  f32x4 ks[kQuarters];
  int any = 0, own_page = -1;  // some lane's page is none; the page of this lane's own keys
  const auto load = [&](int32_t t0, int pk, int ps) {
    const uint32_t tk = (uint32_t)(t0 + key), ts = (uint32_t)(t0 + kG * j);
    const int slot_k = (int)(tk - index_of(tk) * (uint32_t)P.S) + (c16 & 3);
    const int64_t at = (((int64_t)max(pk, 0) * P.H + h) * P.S + slot_k) * D * EB + 16 * j;
#pragma unroll
    for (int qd = 0; qd < kQuarters; ++qd)
#pragma unroll
      for (int c = 0; c < kL; ++c) kf[qd][c] = load16(P.k, at + 4 * qd * D * EB + 64 * c);
    if constexpr (F8) {
      const int slot = (int)(ts - index_of(ts) * (uint32_t)P.S);
      const int64_t line = ((int64_t)max(ps, 0) * P.H + h) * P.S + slot;
#pragma unroll
      for (int qd = 0; qd < kQuarters; ++qd)
        ks[qd] = *reinterpret_cast<const f32x4*>(P.k_scale + line + 4 * qd);
    }
    any = __any((pk | ps) < 0);
    own_page = ps;
  };
  const int64_t held = (int64_t)P.width * P.S;
  int tile = tile0 + wave;
  if (tile < tile1) {
    const int32_t t0 = span.begin + T * tile;
    load(t0, page_at(t0 + key), page_at(t0 + kG * j));
  }
  for (; tile < tile1; tile += kAttendWaves) {
    const int32_t t0 = span.begin + T * tile, ts = t0 + kG * j;
    const int32_t tn = t0 + T * kAttendWaves;
    const bool more = tile + kAttendWaves < tile1;
    int pk = -1, ps = -1;
    if (more) {
      pk = page_at(tn + key);
      ps = page_at(tn + kG * j);
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
    const bool whole = t0 >= all_from && t0 + T <= all_to && !any;
    const bool page = own_page >= 0;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int qd = 0; qd < kQuarters; ++qd) {
        s[mt][qd] *= P.scale;
        if constexpr (F8) s[mt][qd] *= ks[qd];
      }
    if (more) load(tn, pk, ps);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      float x[kG];
#pragma unroll
      for (int e = 0; e < kG; ++e) x[e] = s[mt][e >> 2][e & 3];
      if (!whole) {  // uniform
        const int32_t hi = page ? min(there - 1, last[mt]) : -1;
#pragma unroll
        for (int e = 0; e < kG; ++e)
          x[e] = ((ts + e <= hi) & (ts + e >= first[mt])) ? x[e] : kNegInf;
      }
      const int64_t r = r0 + 16 * mt + c16;
      if (r < rows && ts < held) {  // (a tile may reach past the table's last slot)
        float* to = P.scores + ((b * (int64_t)P.H + h) * P.n * G + r) * held + ts;
#pragma unroll
        for (int e = 0; e < kG; e += 4)
          *reinterpret_cast<f32x4*>(to + e) = f32x4{x[e], x[e + 1], x[e + 2], x[e + 3]};
      }
      float mx = x[0];
#pragma unroll
      for (int e = 1; e < kG; ++e) mx = fmaxf(mx, x[e]);
      if (__any(mx > m[mt])) {  // some lane's maximum grows (each lane keeps its own)
        const float m_new = fmaxf(m[mt], mx);
        l[mt] *= m_new == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(m[mt] - m_new);
        m[mt] = m_new;
      }
      const float base = m[mt] == kNegInf ? 0.0f : m[mt];
#pragma unroll
      for (int e = 0; e < kG; ++e) l[mt] += __builtin_amdgcn_exp2f(x[e] - base);
    }
  }
  // join the lanes and wavefronts of a row
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    float top = fmaxf(m[mt], __shfl_xor(m[mt], 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    float sum = m[mt] == kNegInf ? l[mt] : l[mt] * __builtin_amdgcn_exp2f(m[mt] - top);
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if (j == 0) {
      m_lds[wave][16 * mt + c16] = top;
      l_lds[wave][16 * mt + c16] = sum;
    }
  }
  __syncthreads();
  if (threadIdx.x < 16 * MT) {
    float top = m_lds[0][threadIdx.x], sum = 0.0f;
#pragma unroll
    for (int w = 1; w < kAttendWaves; ++w) top = fmaxf(top, m_lds[w][threadIdx.x]);
#pragma unroll
    for (int w = 0; w < kAttendWaves; ++w) {
      const float mw = m_lds[w][threadIdx.x], lw = l_lds[w][threadIdx.x];
      sum += mw == kNegInf ? lw : lw * __builtin_amdgcn_exp2f(mw - top);
    }
    float* to = P.part + 2 * ((((int64_t)z * P.H + h) * tiles_x + tile_x) * (16 * MT) + threadIdx.x);
    to[0] = top;
    to[1] = sum;
  }
}

// The first step of many rows: 128 of them a workgroup, 32 a wavefront, over every
// tile of 64 keys of the share.  The keys pass through LDS in the order of the
// products' lanes, double-buffered, 8-bit ones widened once as they are written.
// Every lane keeps a maximum and a sum of its own keys until the end.
template <int D, bool F8>
__global__ void __launch_bounds__(64 * kAttendWaves, D > 128 ? 2 : F8 && D == 128 ? 3 : 4) k_weigh_tile(KvParams P) {
  constexpr int MT = 2, kRows = 16 * MT * kAttendWaves, T = 64;
  constexpr int EB = F8 ? 1 : 2, kQuarters = T / 16, kG = T / 4;
  constexpr int kL = D * EB / 64, kSteps = 2 / EB, kC = D / 32;
  constexpr int kMine = kQuarters * kL / kAttendWaves;  // 16-byte loads of a lane
  __shared__ u32x4 frags[2][kQuarters * kC][64];
  __shared__ float scales[2][F8 ? T : 1];
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
  const int32_t len = max(P.len[b], 0), there = tokens_there<kOwn>(P, len);
  const Span span = span_of<kOwn>(P, T, kWeighShare, len, ch.n, token_of(P, G, r0),
                                  token_of(P, G, min(r0 + kRows, rows) - 1), P.splits);
  if (share >= span.shares) return;
  const int tile0 = share * span.per, tile1 = min(span.tiles, tile0 + span.per);
  // this wavefront's rows (the last row again behind the end); a negative scale is
  // taken as a positive one of negated queries, so that maxima need no scaling
  const int64_t w0 = r0 + 16 * MT * wave;
  const uint32_t sign = P.scale < 0.0f ? 0x80008000u : 0u;
  const float scale = fmaxf(fabsf(P.scale), 1e-37f);  // (not 0, for minus infinity times it)
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
    const Limits seen = limits_of<kOwn>(P, ch, len, there, i);
    last[mt] = seen.last;
    first[mt] = seen.first;
  }
  const int i0 = token_of(P, G, min(w0, rows - 1));
  const int i1 = token_of(P, G, min(w0 + 16 * MT, rows) - 1);
  const int32_t all_from = limits_of<kOwn>(P, ch, len, there, i1).first;
  const int32_t all_to = min(limits_of<kOwn>(P, ch, len, there, i0).last + 1, there);

  float m[MT] = {kNegInf, kNegInf}, l[MT] = {0.0f, 0.0f};
  const int32_t* table = P.table + (int64_t)b * P.width;
  u32x4 mine[kMine];
  float my_scale = 0.0f;
  TilePages<D, EB, kG> pages;
  uint32_t valid_next = 0, valid_now = 0;  // groups of keys that are in a page
  const int lane_k = (c16 & 3) * D * EB + 16 * j + wave / kL * 4 * D * EB + wave % kL * 64;
  const auto bring = [&](int32_t t0) {
    pages.place(P, h, there, t0);
    valid_next = pages.valid;
    const int gk = c16 >> 2;
    const char* k = static_cast<const char*>(P.k) + pages.head_of(gk) +
                    (pages.slot_of(gk) * (D * EB) + lane_k);
#pragma unroll
    for (int i = 0; i < kMine; ++i)  // fragments wave, wave + 4, ...
      mine[i] = load16(k, kAttendWaves * i / kL * 4 * D * EB + kAttendWaves * i % kL * 64);
    if constexpr (F8) {
      if (wave == 0) {
        const bool ok = t0 + lane < there && (pages.valid >> j & 1u);
        my_scale = ok ? P.k_scale[pages.head_of(j) / D + pages.slot_of(j) + c16] : 0.0f;
      }
    }
  };
  const auto put = [&](int buf) {
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const int f = wave + i * kAttendWaves;
#pragma unroll
      for (int step = 0; step < kSteps; ++step)
        frags[buf][f * kSteps + step][lane] = __builtin_bit_cast(u32x4, widen<F8>(mine[i], step));
    }
    if constexpr (F8)
      if (wave == 0) scales[buf][lane] = my_scale;
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
    {
      constexpr int kAhead = 4, kKeys = kQuarters * kC;
      u32x4 ring[kAhead];
#pragma unroll
      for (int f = 0; f < kAhead; ++f) ring[f] = frags[buf][f][lane];
#pragma unroll
      for (int f = 0; f < kKeys; ++f) {
        const bf16x8 k8 = __builtin_bit_cast(bf16x8, ring[f % kAhead]);
        if (f + kAhead < kKeys) ring[f % kAhead] = frags[buf][f + kAhead][lane];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
          s[mt][f / kC] =
              __builtin_amdgcn_mfma_f32_16x16x32_bf16(k8, q[mt][f % kC], s[mt][f / kC], 0, 0, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x100, kAhead, 0);
#pragma unroll
      for (int f = 0; f < kKeys; ++f) {
        __builtin_amdgcn_sched_group_barrier(0x8, MT, 0);
        if (f + kAhead < kKeys) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
    }
    if (tile + 2 < tile1) pages.fetch(P, table, there, t0 + 2 * T);
    const bool whole = t0 >= all_from && t0 + T <= all_to && valid_now == 15u;
    float x[MT][kG], mx[MT];
    bool grows = false;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int e = 0; e < kG; ++e) {
        x[mt][e] = s[mt][e >> 2][e & 3];
        if constexpr (F8) x[mt][e] *= scales[buf][kG * j + e];
      }
    if (!whole) {  // uniform
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        const int32_t hi = valid_now >> j & 1u ? min(there - 1, last[mt]) : -1;
        const int lo_e = first[mt] - ts, hi_e = hi - ts;  // this lane's keys that the row sees
#pragma unroll
        for (int e = 0; e < kG; ++e) x[mt][e] = (e <= hi_e && e >= lo_e) ? x[mt][e] : kNegInf;
      }
    }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      mx[mt] = x[mt][0];
#pragma unroll
      for (int e = 1; e < kG; ++e) mx[mt] = fmaxf(mx[mt], x[mt][e]);
      mx[mt] *= scale;
      grows |= mx[mt] > m[mt] + 8.0f;  // (powers up to 2^8 are as exact)
    }
    if (__any(grows)) {  // some lane's maximum grows
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        const float m_new = fmaxf(m[mt], mx[mt]);
        l[mt] *= m[mt] == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(m[mt] - m_new);
        m[mt] = m_new;
      }
    }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const float base = m[mt] == kNegInf ? 0.0f : m[mt];
#pragma unroll
      for (int e = 0; e < kG; ++e) l[mt] += __builtin_amdgcn_exp2f(fmaf(x[mt][e], scale, -base));
    }
    // (the buffer written here was last read before the last barrier)
    if (tile + 1 < tile1) {
      put(buf ^ 1);
      valid_now = valid_next;
      if (tile + 2 < tile1) bring(t0 + 2 * T);
    }
    __syncthreads();
  }
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    float top = fmaxf(m[mt], __shfl_xor(m[mt], 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    float sum = m[mt] == kNegInf ? 0.0f : l[mt] * __builtin_amdgcn_exp2f(m[mt] - top);
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    const int64_t r = w0 + 16 * mt + c16;
    if (r < rows && j == 0) {
      float* to = P.part + 2 * ((((int64_t)z * P.H + h) * tiles_x + tile_x) * kRows + (r - r0));
      to[0] = top;
      to[1] = sum;
    }
  }
}

// A row's largest score and one over its sum, from its shares.
struct RowStat {
  float m, inv;
};
__device__ __forceinline__ RowStat row_stat(const KvParams& P, int T, int least, int b, int h,
                                            const Chunk& ch, int64_t rows, int64_t r) {
  const int G = P.heads / P.H;
  const int64_t x = r / P.tile_rows, r0 = x * P.tile_rows;
  const int64_t tiles_x = ((int64_t)P.n * G + P.tile_rows - 1) / P.tile_rows;
  const Span span =
      span_of<kOwn>(P, T, least, max(P.len[b], 0), ch.n, token_of(P, G, r0),
                    token_of(P, G, min(r0 + P.tile_rows, rows) - 1), P.splits);
  const float* part = P.part + 2 * ((((int64_t)b * P.splits * P.H + h) * tiles_x) * P.tile_rows + r);
  const int64_t step = 2 * (int64_t)P.H * tiles_x * P.tile_rows;
  float top = kNegInf, sum = 0.0f;
  for (int s0 = 0; s0 < span.shares; s0 += 8) {  // eight shares under way together
    float m[8], l[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int64_t at = min(s0 + k, span.shares - 1) * step;
      m[k] = part[at];
      l[k] = part[at + 1];
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (s0 + k >= span.shares) break;
      const float m_new = fmaxf(top, m[k]);
      if (m_new == kNegInf) sum += l[k];  // (nothing seen: 0, or NaN)
      else sum = sum * (top == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(top - m_new)) +
                 l[k] * (m[k] == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(m[k] - m_new));
      top = m_new;
    }
  }
  return RowStat{top == kNegInf ? 0.0f : top, sum == 0.0f ? 0.0f : 1.0f / sum};
}

// The weight position t had: new tokens begin at zero.
__device__ __forceinline__ float weight_before(const KvParams& P, int b, int h, int64_t t,
                                               int64_t pos0) {
  return P.weights && t < pos0 ? P.weights[((int64_t)b * P.H + h) * P.weights_stride + t] : 0.0f;
}

// The second step of few rows: 1024 positions a workgroup, four rows of a thread's
// four positions under way together, the first of them before the statistics.
__global__ void __launch_bounds__(256) k_weigh_sum(KvParams P, int T, int least) {
  __shared__ float m_lds[kWeighRows], inv_lds[kWeighRows];
  const int h = blockIdx.y, b = blockIdx.z;
  const Chunk ch = chunk_of(P, b);
  const int32_t len = max(P.len[b], 0), there = tokens_there<kOwn>(P, len);
  const int32_t end = min(there, P.L), t0 = (int32_t)blockIdx.x * 1024;
  if (t0 >= end) return;
  const int G = P.heads / P.H, n = min(ch.n, P.n);
  const int rows = n * G;
  const int64_t pos0 = (int64_t)len - ch.n, held = (int64_t)P.width * P.S;
  const float* scores = P.scores + (b * (int64_t)P.H + h) * P.n * G * held + t0 + threadIdx.x;
  const auto at = [&](int k) { return t0 + 256 * k + (int)threadIdx.x; };
  float s[4][4], sum[4] = {};
  const auto load = [&](int r0) {
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (r0 + r < rows && at(k) < end) s[r][k] = scores[(r0 + r) * held + 256 * k];
  };
  load(0);
  float before[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) before[k] = at(k) < end ? weight_before(P, b, h, at(k), pos0) : 0.0f;
  if ((int)threadIdx.x < rows) {
    const RowStat x = row_stat(P, T, least, b, h, ch, rows, threadIdx.x);
    m_lds[threadIdx.x] = x.m;
    inv_lds[threadIdx.x] = x.inv;
  }
  __syncthreads();
  for (int r0 = 0; r0 < rows; r0 += 4) {
    if (r0) load(r0);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      if (r0 + r >= rows) break;
      const Limits seen = limits_of<kOwn>(P, ch, len, there, (r0 + r) / G);
      const float m = m_lds[r0 + r], inv = inv_lds[r0 + r];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (at(k) >= seen.first && at(k) <= min(seen.last, end - 1))
          sum[k] += __builtin_amdgcn_exp2f(s[r][k] - m) * inv;
    }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (at(k) < end)
      P.out_weights[((int64_t)b * P.H + h) * P.weights_stride + at(k)] = before[k] + sum[k];
}

// The second step of many rows: each of four wavefronts holds 64 keys, all take the
// same rows, 64 at a time through LDS, whose statistics the workgroup has put there
// (kWeighStats rows at a time).  Where all rows are at most two such pieces, which
// then stay in LDS, a workgroup goes on to further keys.  Rows that see some of the
// keys are cut into P.parts, whose sums k_weigh_add adds, where there are too few
// keys to fill the card.
template <int D, bool F8>
__global__ void __launch_bounds__(64 * kAttendWaves, D <= 128 ? 2 : 1) k_weigh_keys(KvParams P) {
  constexpr int EB = F8 ? 1 : 2, T = 64, kQuarters = 4, kG = 16, kBlock = 64;
  constexpr int kL = D * EB / 64, kSteps = 2 / EB, kC = D / 32, kTiles = kBlock / 16;
  static_assert(kTiles == kAttendWaves, "a wavefront brings 16 rows");
  __shared__ u32x4 rows_lds[2][kTiles][kC][64];
  __shared__ float stats[2 * kWeighStats];
  const int h = blockIdx.y, z = blockIdx.z, b = z / P.parts, part = z % P.parts;
  const int lane = threadIdx.x & 63, c16 = lane & 15, j = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const Chunk ch = chunk_of(P, b);
  const int32_t len = max(P.len[b], 0), there = tokens_there<kOwn>(P, len);
  const int32_t end = min(there, P.L);
  constexpr int kKeys = T * kAttendWaves;  // of a workgroup at a time
  int32_t wg0 = (int32_t)blockIdx.x * kKeys;
  if (wg0 >= end) return;
  const int G = P.heads / P.H;
  const int64_t rows = (int64_t)min(ch.n, P.n) * G, pos0 = (int64_t)len - ch.n;
  const int32_t* table = P.table + (int64_t)b * P.width;
  const int64_t row = (int64_t)b * P.H + h;
  const bool stay = rows <= 2 * kBlock;  // all rows are in LDS
  TilePages<D, EB, kG> pages;
  uint32_t valid = 0;
  u32x4 raw[kQuarters][kL];
  f32x4 ks[F8 ? kQuarters : 1];
  const auto bring_keys = [&](int32_t t0) {
    pages.place(P, h, there, t0);
    valid = pages.valid;
    const int gk = c16 >> 2;
    const char* k = static_cast<const char*>(P.k) + pages.head_of(gk) +
                    ((pages.slot_of(gk) + (c16 & 3)) * (D * EB) + 16 * j);
#pragma unroll
    for (int qd = 0; qd < kQuarters; ++qd)
#pragma unroll
      for (int c = 0; c < kL; ++c) raw[qd][c] = load16(k, 4 * qd * D * EB + 64 * c);
    if constexpr (F8) {
      const float* scale = P.k_scale + (pages.head_of(j) / D + pages.slot_of(j));
#pragma unroll
      for (int qd = 0; qd < kQuarters; ++qd) ks[qd] = *reinterpret_cast<const f32x4*>(scale + 4 * qd);
    }
  };
  const auto row_at = [&](int64_t position) { return (position - pos0) * G; };
  u32x4 mine[kC];
  const auto bring = [&](int block) {
    const int64_t r = min((int64_t)block * kBlock + 16 * wave + c16, rows - 1);
    const int i = token_of(P, G, r), g = (int)(r - (int64_t)i * G);
    const int64_t q_at = (ch.first + i) * P.q_stride + (int64_t)(h * G + g) * D;
#pragma unroll
    for (int c = 0; c < kC; ++c) {
      const int d = c / kSteps * (32 * kSteps) + j * (8 * kSteps) + c % kSteps * 8;
      mine[c] = *reinterpret_cast<const u32x4a2*>(static_cast<const uint16_t*>(P.q) + q_at + d);
    }
  };
  const auto put = [&](int buf) {
#pragma unroll
    for (int c = 0; c < kC; ++c) rows_lds[buf][wave][c][lane] = mine[c];
  };
  constexpr int kChunk = kWeighStats / kBlock;
  const auto statistics = [&](int64_t s0, int64_t s1) {
    for (int64_t r = s0 + threadIdx.x; r < min(s1, rows); r += 64 * kAttendWaves) {
      const RowStat x = row_stat(P, T, kWeighShare, b, h, ch, rows, r);
      stats[2 * (r - s0)] = x.m;
      stats[2 * (r - s0) + 1] = x.inv;
    }
  };
  // (the next keys' loads are under way with the products where registers allow)
  constexpr bool kEarly = D * EB <= 128;
  const int32_t hop = (int32_t)gridDim.x * kKeys;
  pages.fetch(P, table, there, wg0 + T * wave);
  bring_keys(wg0 + T * wave);
  if (wg0 + hop < end) pages.fetch(P, table, there, wg0 + hop + T * wave);
  if (stay) {
    for (int block = 0; block * kBlock < rows; ++block) {
      bring(block);
      put(block);
    }
    statistics(0, 2 * kBlock);
    __syncthreads();
  }
  for (; wg0 < end; wg0 += hop) {
    const int32_t t0 = wg0 + T * wave, ts = t0 + kG * j, next = wg0 + hop;
    const int32_t t = ts + c16;  // this lane's key in the end
    const float before = P.parts == 1 && t < end ? weight_before(P, b, h, t, pos0) : 0.0f;
    // rows that see some of the workgroup's keys, and those that see all of the wavefront's
    int64_t r_end = rows, r_all_end = rows;
    if (P.window > 0) {
      r_end = min(rows, row_at((int64_t)wg0 + kKeys - 1 + P.window));
      r_all_end = min(rows, row_at((int64_t)t0 + P.window));
    }
    const int64_t r_all = row_at((int64_t)t0 + T - 1);
    const int block0 = (int)(max(row_at(wg0), (int64_t)0) / kBlock);
    const int blocks = max((int)((max(r_end, (int64_t)0) + kBlock - 1) / kBlock) - block0, 0);
    const int per = (blocks + P.parts - 1) / P.parts;
    const int first = block0 + min(part * per, blocks), last = block0 + min((part + 1) * per, blocks);
    const int live = valid >> j & 1u ? min(there - ts, kG) : 0;
    const bool all_live = !__any(live < kG);
    bf16x8 k8[kQuarters][kC];
    float factor[F8 ? kG : 1];
#pragma unroll
    for (int qd = 0; qd < kQuarters; ++qd)
#pragma unroll
      for (int c = 0; c < kC; ++c) k8[qd][c] = widen<F8>(raw[qd][c / kSteps], c % kSteps);
    if constexpr (F8) {
#pragma unroll
      for (int e = 0; e < kG; ++e) factor[e] = ks[e >> 2][e & 3] * P.scale;
    }
    const auto bring_next = [&] {
      if (next >= end) return;
      bring_keys(next + T * wave);
      if (next + hop < end) pages.fetch(P, table, there, next + hop + T * wave);
    };
    if constexpr (kEarly) bring_next();
    float acc[kG] = {};
    // a tile of 16 rows from r0, of which buf holds tile; stats begin at row s0
    const auto take = [&](auto all, int64_t r0, int buf, int tile, int64_t s0) {
      bf16x8 q[kC];
#pragma unroll
      for (int c = 0; c < kC; ++c) q[c] = __builtin_bit_cast(bf16x8, rows_lds[buf][tile][c][lane]);
      const int64_t r = min(r0 + c16, rows - 1);
      const float m = stats[2 * (r - s0)], inv = stats[2 * (r - s0) + 1];
      f32x4 s[kQuarters];
#pragma unroll
      for (int qd = 0; qd < kQuarters; ++qd) s[qd] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int c = 0; c < kC; ++c)
#pragma unroll
        for (int qd = 0; qd < kQuarters; ++qd)
          s[qd] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k8[qd][c], q[c], s[qd], 0, 0, 0);
      if constexpr (decltype(all)::value) {
#pragma unroll
        for (int e = 0; e < kG; ++e)
          acc[e] = fmaf(__builtin_amdgcn_exp2f(
                            fmaf(s[e >> 2][e & 3], F8 ? factor[F8 ? e : 0] : P.scale, -m)),
                        inv, acc[e]);
      } else {
        const Limits seen = limits_of<kOwn>(P, ch, len, there, token_of(P, G, r));
        // this lane's keys that the row sees: lo <= e < hi
        const int lo = max(seen.first - ts, 0);
        const int hi = r0 + c16 < rows ? min(live, seen.last + 1 - ts) : 0;
#pragma unroll
        for (int e = 0; e < kG; ++e) {
          const float w = __builtin_amdgcn_exp2f(fmaf(s[e >> 2][e & 3],
                                                      F8 ? factor[F8 ? e : 0] : P.scale, -m)) * inv;
          acc[e] += (e >= lo && e < hi) ? w : 0.0f;
        }
      }
    };
    const auto take_block = [&](int block, int buf, int64_t s0) {
      const int64_t r0 = (int64_t)block * kBlock;
      if (all_live && r0 >= r_all && r0 + kBlock <= r_all_end) {  // uniform
#pragma unroll
        for (int tile = 0; tile < kTiles; ++tile) take(std::true_type(), r0 + 16 * tile, buf, tile, s0);
      } else {
#pragma unroll 1
        for (int tile = 0; tile < kTiles; ++tile)
          if (r0 + 16 * tile < rows) take(std::false_type(), r0 + 16 * tile, buf, tile, s0);
      }
    };
    if (stay) {
      for (int block = first; block < last; ++block) take_block(block, block, 0);
    } else {
      if (first < last) bring(first);
      for (int chunk = first; chunk < last; chunk += kChunk) {
        const int chunk_end = min(chunk + kChunk, last);
        const int64_t s0 = (int64_t)chunk * kBlock;
        // (the last reads of the chunk before are behind its last barrier)
        statistics(s0, (int64_t)chunk_end * kBlock);
        if (chunk == first) {
          put(0);
          if (first + 1 < last) bring(first + 1);
        }
        __syncthreads();
        for (int block = chunk; block < chunk_end; ++block) {
          const int buf = (block - first) & 1;
          take_block(block, buf, s0);
          // (the buffer written here was last read before the last barrier)
          if (block + 1 < last) {
            put(buf ^ 1);
            if (block + 2 < last) bring(block + 2);
          }
          __syncthreads();
        }
      }
    }
    if constexpr (!kEarly) bring_next();
    // over the 16 lanes that hold rows of the same keys: a lane keeps half of the sums
    // and gives the other half, until it has those of its own key
#pragma unroll
    for (int d = 8; d; d >>= 1)
#pragma unroll
      for (int e = 0; e < d; ++e) {
        const float keep = c16 & d ? acc[e + d] : acc[e], give = c16 & d ? acc[e] : acc[e + d];
        acc[e] = keep + __shfl_xor(give, d);
      }
    if (t < end) {
      if (P.parts > 1)
        P.sums[((int64_t)part * P.B * P.H + row) * min((int64_t)P.width * P.S, (int64_t)P.L) + t] =
            acc[0];
      else P.out_weights[row * P.weights_stride + t] = before + acc[0];
    }
  }
}

// The sums of k_weigh_keys' parts of the rows, in their order.
__global__ void __launch_bounds__(256) k_weigh_add(KvParams P) {
  const int h = blockIdx.y, b = blockIdx.z;
  const Chunk ch = chunk_of(P, b);
  const int32_t len = max(P.len[b], 0), end = min(tokens_there<kOwn>(P, len), P.L);
  const int32_t t = (int32_t)(blockIdx.x * 256 + threadIdx.x);
  if (t >= end) return;
  const int64_t row = (int64_t)b * P.H + h, n = min((int64_t)P.width * P.S, (int64_t)P.L);
  float sum = 0.0f;
  for (int part = 0; part < P.parts; ++part)
    sum += P.sums[((int64_t)part * P.B * P.H + row) * n + t];
  P.out_weights[row * P.weights_stride + t] =
      weight_before(P, b, h, t, (int64_t)len - ch.n) + sum;
}

template <int D, bool F8>
void weigh(const KvParams& P, hipStream_t stream) {
  const int64_t rows = (int64_t)P.n * (P.heads / P.H), held = (int64_t)P.width * P.S;
  const int64_t groups = ((int64_t)P.H * P.B * P.splits + 7) / 8 * 8;
  const dim3 grid((uint32_t)((rows + P.tile_rows - 1) / P.tile_rows * groups));
  const int64_t end = held < P.L ? held : P.L;  // positions that get a weight
  if (P.scores) {
    if (P.tile_rows == 16) k_weigh_rows<D, F8, 1><<<grid, 64 * kAttendWaves, 0, stream>>>(P);
    else k_weigh_rows<D, F8, 2><<<grid, 64 * kAttendWaves, 0, stream>>>(P);
    k_weigh_sum<<<dim3((uint32_t)((end + 1023) / 1024), P.H, P.B), 256, 0, stream>>>(
        P, F8 ? 64 : 32, share_keys(P.tile_rows, F8));
    return;
  }
  k_weigh_tile<D, F8><<<grid, 64 * kAttendWaves, 0, stream>>>(P);
  // (where rows stay in LDS, two workgroups a compute unit take all keys in turn)
  int64_t key_groups = (end + 255) / 256;
  if (rows <= 128) key_groups = std::min<int64_t>(key_groups, (511 + P.B * P.H) / (P.B * P.H));
  k_weigh_keys<D, F8><<<dim3((uint32_t)key_groups, P.H, P.B * P.parts), 64 * kAttendWaves, 0,
                        stream>>>(P);
  if (P.parts > 1)
    k_weigh_add<<<dim3((uint32_t)((end + 255) / 256), P.H, P.B), 256, 0, stream>>>(P);
}

// ------------------------------------------------------------------ eviction
// Which tokens of a sequence and head stay: one workgroup finds the weight of the
// last one kept by counting, 8 bits of it a pass, the highest first, among those
// that agree in the bits before, until all or few of them are left, which it ranks;
// then it writes the positions of what is above that weight, and of the first ones
// equal to it, in their order.  Weights are compared as 32-bit words of their order:
// 0 for a position that is in no page (never kept), 1 for a NaN, the largest for
// tokens that stay whatever they weigh.  A lane takes four positions in a row (of one
// page), KEYS in all, in registers; of rows longer than THREADS times KEYS they are
// taken again from memory every pass.  Bound by its chain of barriers, in long rows by
// what one compute unit's LDS counts: 1200 positions 7.5 us, 8192 11, 28385 27 (11,
// 17 and 36 with a position a lane, all passes to the last, a kept token's weight
// loaded where it is written).
__device__ __forceinline__ uint32_t order_of(uint32_t u) {
  if ((u & 0x7fffffffu) > 0x7f800000u) return 1u;
  if (u == 0x80000000u) u = 0u;  // (-0 as 0)
  return u >> 31 ? ~u : u | 0x80000000u;
}
// t / S of positions under 2^30.
__device__ __forceinline__ uint32_t page_index(const KvParams& C, uint32_t t) {
  return C.s16_magic ? __umulhi(t >> 4, C.s16_magic) : t >> 4;
}
// Sums over the lanes up to each: inside rows of 16, then of the rows before.
template <int N>
__device__ __forceinline__ uint32_t lanes_up(uint32_t v) {  // row_shr: 0 where there is none
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x110 + N, 0xf, 0xf, false);
}
__device__ __forceinline__ uint32_t lane_of(uint32_t v, int lane) {
  return (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
}
__device__ __forceinline__ uint32_t sums_upto(uint32_t v) {
  v += lanes_up<1>(v);
  v += lanes_up<2>(v);
  v += lanes_up<4>(v);
  v += lanes_up<8>(v);
  const uint32_t a = lane_of(v, 15), b = a + lane_of(v, 31), c = b + lane_of(v, 47);
  const int row = (threadIdx.x & 63) >> 4;
  return v + (row == 0 ? 0u : row == 1 ? a : row == 2 ? b : c);
}
// Lanes below this one in the mask, and n.
__device__ __forceinline__ uint32_t count_below(uint64_t mask, uint32_t n) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, n));
}

template <int THREADS, int KEYS>
__global__ void __launch_bounds__(THREADS) k_evict_select(EvictParams P) {
  // copies of a count: lanes that add to one bin do not wait for each other, and a
  // bin's copies lie in different banks
  constexpr int kCopies = 16, kCopy = 257, kWaves = THREADS / 64;
  constexpr int kRuns = KEYS / 4, kCounts = kRuns * kWaves, kFew = 64;
  __shared__ uint32_t bins[kCopies * kCopy];
  __shared__ __align__(16) uint32_t total[256];
  __shared__ uint32_t counts[kCounts], few[kFew], few_count;
  const int h = blockIdx.x, b = blockIdx.y, tid = (int)threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const KvParams& C = P.cache;
  const int32_t whole_len = max(C.len[b], 0);
  const int32_t len = (int32_t)min((int64_t)whole_len, (int64_t)C.width * C.S);
  const int32_t weighed = min(len, P.length);  // positions that have a weight
  const float* weights = P.weights + ((int64_t)b * C.H + h) * P.weights_stride;
  const int32_t* table = C.table + (int64_t)b * C.width;
  const int32_t recent = max(whole_len - P.recent, 0);  // tokens from here on stay
  uint32_t key[KEYS];
  const auto fill = [&](int32_t base) {  // (len > 0)
    u32x4 w[kRuns];
    int32_t page[kRuns];
    const auto at = [&](int i) { return base + 4 * (i * THREADS + tid); };
    if (weighed >= 4) {  // uniform; at the end, the last four
#pragma unroll
      for (int i = 0; i < kRuns; ++i)
        w[i] = *reinterpret_cast<const u32x4a4*>(weights + min(at(i), weighed - 4));
    } else {
#pragma unroll
      for (int i = 0; i < kRuns; ++i) w[i] = u32x4{0u, 0u, 0u, 0u};
      if (at(0) == 0)
#pragma unroll
        for (int k = 0; k < 3; ++k)
          if (k < weighed) w[0][k] = __float_as_uint(weights[k]);
    }
#pragma unroll
    for (int i = 0; i < kRuns; ++i) page[i] = table[page_index(C, (uint32_t)min(at(i), len - 1))];
#pragma unroll
    for (int i = 0; i < kRuns; ++i) {
      const int32_t t = at(i), past = weighed >= 4 ? min(max(t - (weighed - 4), 0), 4) : 0;
      u32x4 x = w[i];
      if (past & 1) x = u32x4{x[1], x[2], x[3], 0u};
      if (past & 2) x = u32x4{x[2], x[3], 0u, 0u};
      if (past & 4) x = u32x4{0u, 0u, 0u, 0u};
      const bool there = (uint32_t)page[i] < (uint32_t)C.pages;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t o = t + k < P.first || t + k >= recent ? 0xffffffffu : order_of(x[k]);
        key[4 * i + k] = there && t + k < len ? o : 0u;
      }
    }
  };
  constexpr int32_t kStep = THREADS * KEYS;
  const bool held = len <= kStep;
#pragma unroll
  for (int i = 0; i < KEYS; ++i) key[i] = 0u;
  for (int i = tid; i < kCopies * kCopy; i += THREADS) bins[i] = 0u;
  if (tid == 0) few_count = 0u;
  if (held && len) fill(0);
  __syncthreads();
  // the kept-th largest key, and how many of that value are kept (all: what is above 0)
  uint32_t border = 0u, need = 0u, kept = 0u;
  for (int shift = 24;; shift -= 8) {
    for (int32_t base = 0; base < len; base += kStep) {
      if (!held) fill(base);
#pragma unroll
      for (int i = 0; i < KEYS; ++i)
        if (key[i] && (shift == 24 || key[i] >> (shift + 8) == border))
          atomicAdd(&bins[(lane & (kCopies - 1)) * kCopy + (key[i] >> shift & 255u)], 1u);
    }
    __syncthreads();
    if (tid < 256) {  // (and the counts are zero again)
      uint32_t n = 0;
#pragma unroll
      for (int c = 0; c < kCopies; ++c) {
        n += bins[c * kCopy + tid];
        bins[c * kCopy + tid] = 0u;
      }
      total[255 - tid] = n;
    }
    __syncthreads();
    // every wavefront for itself: bins from the largest down, four a lane
    const u32x4 n = *reinterpret_cast<const u32x4*>(&total[4 * lane]);
    const uint32_t sum = n[0] + n[1] + n[2] + n[3], upto = sums_upto(sum);
    if (shift == 24) {
      const uint32_t there = lane_of(upto, 63);
      kept = min((uint32_t)P.keep, there);
      if (kept == there) break;
      need = kept;
    }
    uint32_t before = upto - sum, digit = 0u, ahead = 0u, left = 0u;
    bool found = false;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (before < need && before + n[k] >= need) {
        found = true;
        digit = (uint32_t)(255 - 4 * lane - k);
        ahead = before;
        left = n[k];
      }
      before += n[k];
    }
    const int at = __ffsll((unsigned long long)__ballot(found)) - 1;
    border = border << 8 | lane_of(digit, at);
    need -= lane_of(ahead, at);
    left = lane_of(left, at);  // that begin with these bits, of which `need` stay
    if (shift == 0) break;
    if (left == need) {
      border = max(border << shift, 1u) - 1u;
      need = 0u;
      break;
    }
    if (left <= kFew) {
      for (int32_t base = 0; base < len; base += kStep) {
        if (!held) fill(base);
#pragma unroll
        for (int i = 0; i < KEYS; ++i)
          if (key[i] && key[i] >> shift == border) {
            const uint32_t at_few = atomicAdd(&few_count, 1u);
            if (at_few < kFew) few[at_few] = key[i];
          }
      }
      __syncthreads();
      const uint32_t x = lane < (int)left ? few[lane] : 0u;
      uint32_t larger = 0u, same = 0u;
      for (int j = 0; j < (int)left; ++j) {
        const uint32_t y = lane_of(x, j);
        larger += y > x;
        same += y == x;
      }
      const int last = __ffsll((unsigned long long)__ballot(lane < (int)left && larger < need &&
                                                           larger + same >= need)) - 1;
      border = lane_of(x, last);
      need -= lane_of(larger, last);
      break;
    }
  }
  // positions in their order
  uint32_t above = 0, equal = 0;  // before the present ones
  int32_t* index = P.out_index + ((int64_t)b * C.H + h) * P.keep;
  float* out_w = P.out_weights ? P.out_weights + ((int64_t)b * C.H + h) * P.out_stride : nullptr;
  for (int32_t base = 0; base < len; base += kStep) {
    if (!held) fill(base);
    // what is above (the lower half of a word) and equal, by runs of the wavefronts
    uint32_t mine = 0u;
#pragma unroll
    for (int i = 0; i < kRuns; ++i) {
      uint32_t n = 0u;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t x = key[4 * i + k];
        n += (uint32_t)__popcll(__ballot(x > border)) +
             ((uint32_t)__popcll(__ballot(x && x == border)) << 16);
      }
      mine = lane == i ? n : mine;
    }
    if (lane < kRuns) counts[lane * kWaves + wave] = mine;
    __syncthreads();
    // (the masks are taken again: hundreds of them spill from the scalar registers)
#pragma unroll
    for (int i = 0; i < KEYS; ++i) asm("" : "+v"(key[i]));
    static_assert(THREADS * KEYS < 65536, "two counts a word");
    constexpr int kEach = (kCounts + 63) / 64;
    static_assert(kEach == 1 || (kEach == 2 && kWaves % 2 == 0), "by the wavefront's parity");
    uint32_t part[kEach], sum = 0u;
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const int at = lane * kEach + k;
      part[k] = at < kCounts ? counts[at] : 0u;
      sum += part[k];
    }
    const uint32_t upto = sums_upto(sum);
    const uint32_t of_mine = upto - sum + (kEach == 2 && (wave & 1) ? part[0] : 0u);
#pragma unroll
    for (int i = 0; i < kRuns; ++i) {
      const uint32_t pre = lane_of(of_mine, (i * kWaves + wave) / kEach);
      uint32_t ra = above + (pre & 0xffffu), re = equal + (pre >> 16);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t x = key[4 * i + k];
        ra = count_below(__ballot(x > border), ra);
        re = count_below(__ballot(x && x == border), re);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t x = key[4 * i + k];
        const bool a = x > border, e = x && x == border;
        if (a || (e && re < need)) {
          const uint32_t at = ra + min(re, need);
          const int32_t t = base + 4 * (i * THREADS + tid) + k;
          index[at] = t;
          if (out_w) {
            float w = __uint_as_float(x >> 31 ? x ^ 0x80000000u : ~x);
            if (x == 1u || x == 0xffffffffu) w = t < P.length ? weights[t] : 0.0f;
            out_w[at] = w;
          }
        }
        ra += a;
        re += e;
      }
    }
    const uint32_t all = lane_of(upto, 63);
    above += all & 0xffffu;
    equal += all >> 16;
    if (base + kStep < len) __syncthreads();
  }
  for (int64_t i = (int64_t)kept + tid; i < P.keep; i += THREADS) index[i] = -1;
  if (h == 0 && tid == 0) P.out_len[b] = (int32_t)kept;
}

// The kept tokens of a head to their new places, 64 a workgroup.  Keys go as rows.
// Values are gathered in LDS from the sixteen-byte pieces (N tokens of a dimension)
// that hold a kept token, each loaded once, as many dimensions at a time as fit, and
// stored as whole pieces.  Bound by the bytes, of values those of every piece with a
// kept token: half of 8 sequences of up to 8192, 8 heads of 128 in bfloat16, 44 us
// (62 with loads and stores of one value a lane).
template <int D, bool F8>
__global__ void __launch_bounds__(256) k_evict_move(EvictParams P) {
  constexpr int EB = F8 ? 1 : 2, kLoads = D * EB / 16, N = 16 / EB, kPieces = 64 / N;
  constexpr int kHeld = 2048;  // pieces of a dimension that LDS holds
  typedef typename std::conditional<F8, uint8_t, uint16_t>::type E;
  __shared__ u32x4 held[kHeld];
  __shared__ int64_t from_key[64], to_key[64];  // lines of the key pages; to: -1, none
  __shared__ int64_t piece_at[64];              // of values: bytes, dimension 0
  __shared__ int64_t to_value[kPieces];         // of a whole piece, -1: element by element
  __shared__ uint16_t place[64];                // a token's piece and place in it
  __shared__ int32_t pieces;
  const int h = blockIdx.y, b = blockIdx.z, tid = (int)threadIdx.x;
  const KvParams& C = P.cache;
  const int kept = P.out_len[b];
  const int64_t j0 = (int64_t)blockIdx.x * 64;
  if (j0 >= kept) return;
  const int n = (int)min((int64_t)64, kept - j0);
  if (tid < 64) {
    const int i = min(tid, n - 1);
    const int32_t t = max(P.out_index[((int64_t)b * C.H + h) * P.keep + j0 + i], 0);
    const int32_t j = (int32_t)j0 + i;
    const uint32_t ij = page_index(C, (uint32_t)j), it = page_index(C, (uint32_t)t);
    const int p = P.out_table[(int64_t)b * P.out_width + ij];
    const int from = C.table[(int64_t)b * C.width + it];
    const int sf = t - (int)it * C.S, st = j - (int)ij * C.S;
    const bool ok = tid < n && (uint32_t)p < (uint32_t)C.pages && (uint32_t)from < (uint32_t)C.pages &&
                    !(p == from && sf == st);  // (in place: not moved)
    const int64_t hf = (int64_t)(ok ? from : 0) * C.H + h, ht = (int64_t)(ok ? p : 0) * C.H + h;
    from_key[tid] = hf * C.S + sf;
    to_key[tid] = ok ? ht * C.S + st : -1;
    // the pieces, numbered where they begin (tokens ascend)
    const int id = ok ? t / N : -1;
    const int id_before = __shfl_up(id, 1);
    const bool first = ok && (tid == 0 || id_before != id);
    const uint64_t firsts = __ballot(first);
    const int piece = (int)__popcll(firsts & (((uint64_t)2 << tid) - 1)) - 1;
    if (first) piece_at[piece] = (hf * D * C.S + (sf & ~(N - 1))) * EB;
    place[tid] = (uint16_t)(max(piece, 0) * N + (sf & (N - 1)));
    const uint64_t all = __ballot(ok);
    if (tid % N == 0) {
      const uint64_t mask = ((uint64_t)1 << N) - 1;
      to_value[tid / N] = (all >> tid & mask) == mask ? (ht * D * C.S + st) * EB : -1;
    }
    if (tid == 0) pieces = (int)__popcll(firsts);
  }
  __syncthreads();
  const int count = pieces;
  if (count == 0) return;  // (all in place)
  // dimensions at a time: a power of two, so that the pieces fit
  int dims = D;
  while (dims * count > kHeld) dims >>= 1;
  const int shift = 31 - __clz(dims);
  const int64_t stride = (int64_t)C.S * EB;  // between dimensions
  for (int d0 = 0; d0 < D; d0 += dims) {
    constexpr int kAtOnce = kHeld / 256;
    u32x4 v[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int i = k * 256 + tid;
      if (i < count << shift)
        v[k] = load16(C.v, piece_at[i >> shift] + (d0 + (i & (dims - 1))) * stride);
    }
    if (d0 == 0) {  // keys, under the first loads
      for (int k = tid; k < 64 * kLoads; k += 256) {
        const int i = k / kLoads, d = k % kLoads * 16;
        if (to_key[i] < 0) continue;
        *reinterpret_cast<u32x4*>(static_cast<char*>(C.k) + to_key[i] * (D * EB) + d) =
            load16(C.k, from_key[i] * (D * EB) + d);
      }
      if constexpr (F8) {
        if (tid < 128 && to_key[tid & 63] >= 0) {
          float* scale = tid < 64 ? C.k_scale : C.v_scale;
          scale[to_key[tid & 63]] = scale[from_key[tid & 63]];
        }
      }
    }
    if (d0) __syncthreads();
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int i = k * 256 + tid;
      if (i < count << shift) held[i] = v[k];
    }
    __syncthreads();
    const E* lds = reinterpret_cast<const E*>(held);
    for (int k = tid; k < kPieces << shift; k += 256) {
      const int d = k & (dims - 1), q = k >> shift;
      E x[N];
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const int at = place[q * N + e];
        x[e] = lds[(((at / N) << shift) + d) * N + at % N];
      }
      const int64_t to = to_value[q];
      if (to >= 0) {
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if constexpr (F8)
            w[i] = (uint32_t)x[4 * i] | (uint32_t)x[4 * i + 1] << 8 | (uint32_t)x[4 * i + 2] << 16 |
                   (uint32_t)x[4 * i + 3] << 24;
          else w[i] = (uint32_t)x[2 * i] | (uint32_t)x[2 * i + 1] << 16;
        }
        *reinterpret_cast<u32x4*>(static_cast<char*>(C.v) + to + (d0 + d) * stride) = w;
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const int64_t line = to_key[q * N + e];
          if (line < 0) continue;
          const int64_t page_head = line / C.S;
          static_cast<E*>(C.v)[(page_head * D + d0 + d) * C.S + (line - page_head * C.S)] = x[e];
        }
      }
    }
  }
}

template <int D, bool F8>
void move(const EvictParams& P, hipStream_t stream) {
  k_evict_move<D, F8><<<dim3((uint32_t)((P.keep + 63) / 64), P.cache.H, P.cache.B), 256, 0, stream>>>(P);
}

}  // namespace

hipError_t launch_kv_weigh(const KvParams& P, hipStream_t stream) {
  if (P.D == 64) P.f8 ? weigh<64, true>(P, stream) : weigh<64, false>(P, stream);
  else if (P.D == 128) P.f8 ? weigh<128, true>(P, stream) : weigh<128, false>(P, stream);
  else P.f8 ? weigh<256, true>(P, stream) : weigh<256, false>(P, stream);
  return hipGetLastError();
}

hipError_t launch_kv_evict(const EvictParams& P, hipStream_t stream) {
  const KvParams& C = P.cache;
  const int64_t tokens = (int64_t)C.width * C.S;
  const dim3 heads(C.H, C.B);
  // As many threads as hold the positions, and no more registers.  (us a call by 256 /
  // 1024 threads, 32 sequences of 1500, 16 heads 36 / 42, of 64 of 2000, 32 heads 60 /
  // 108; by 16 / 32 positions, 12000 20 / 27.)
  if (tokens <= 2048) k_evict_select<256, 8><<<heads, 256, 0, stream>>>(P);
  else if (tokens <= 8192) k_evict_select<1024, 8><<<heads, 1024, 0, stream>>>(P);
  else if (tokens <= 16384) k_evict_select<1024, 16><<<heads, 1024, 0, stream>>>(P);
  else k_evict_select<1024, 32><<<heads, 1024, 0, stream>>>(P);
  if (C.D == 64) C.f8 ? move<64, true>(P, stream) : move<64, false>(P, stream);
  else if (C.D == 128) C.f8 ? move<128, true>(P, stream) : move<128, false>(P, stream);
  else C.f8 ? move<256, true>(P, stream) : move<256, false>(P, stream);
  return hipGetLastError();
}

}  // namespace spc
