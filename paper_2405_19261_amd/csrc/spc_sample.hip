// spc_sample.hip -- gfx950 kernels of the truncated distributions: a token
// drawn from, or logits cut to, softmax(z / T) under top-k, top-p and min-p.
//
// All three filters keep a prefix of the row's descending order (ties: lowest
// index first), so together they keep a prefix too, and its end is one pair
// (key, index): an entry is kept exactly when its logit's key is above the
// cut's, or equal to it with an index no higher than the cut's.  No row is
// sorted; the cut is found by counting:
//
//   bins     Entries are counted into bins of 1/16 octave of probability:
//            with t = 16 z log2(e) / T, bin floor(t).  A bin holds its
//            entries' count and mass.  The mass of an entry relative to its
//            bin's lower edge is 2^(f/16), f = t - floor(t), kept as the
//            fixed-point integer of 2^(f/16) - 1 in [0, 0.0443), so that a
//            bin's mass does not depend on the order its entries came in.
//            Bins kBins - 1 and further below the row's maximum (64 octaves)
//            are one bin without mass (a share of the row under V 2^-64).
//   the cut  Scans over the bins find the bin in which the count reaches k,
//            or the mass reaches p times the mass of the first k; inside that
//            bin the keys are narrowed by further counts (1024 ranges a pass)
//            to one value, and equal values by index.
//   the draw Kept entries weigh 2^((t - t_max)/16) in fixed point: sums are
//            exact, so the inverse CDF in vocabulary order is a function of
//            the inputs alone.
//
// All arithmetic on probabilities is in 64 bits (t, the weights and the sums):
// a sampled token and the kept set are discrete, and 32-bit sums over 256 000
// entries move a border of the CDF by more than an entry's mass.
#include <math.h>

#include <algorithm>

#include "spc_internal.h"

// t = z c is rounded before its floor is taken from it, everywhere alike: a
// product fused into the difference could leave a fraction under 0.
#pragma clang fp contract(off)

namespace spc {
namespace {

constexpr int kNT = 1024;  // threads of a workgroup
constexpr int kNW = kNT / 64;
constexpr int kBins = 1024;
constexpr double kBinsPerNat = 23.083120654223414518;  // 16 log2(e)
constexpr double kLn2by16 = 0.043321698784996581839;   // ln(2) / 16
constexpr int kNoIndex = 0x7fffffff;

typedef uint32_t w4 __attribute__((ext_vector_type(4)));
typedef w4 w4a4 __attribute__((aligned(4)));
typedef w4 w4a2 __attribute__((aligned(2)));

template <int DT>
struct Elem {
  static constexpr int EB = DT == 1 ? 2 : 4;
  static constexpr int VW = 16 / EB;  // entries of a lane load
};

// The logit as the order and the masses see it: NaN as -inf, +inf as the
// largest finite value, -0 as +0.
__device__ __forceinline__ float clean(float z) {
  return (z == z ? fminf(z, 3.40282347e38f) : -__builtin_huge_valf()) + 0.0f;
}
// A monotone map of floats to unsigned integers.
__device__ __forceinline__ uint32_t key_of(float z) {
  const uint32_t u = __float_as_uint(z);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float of_key(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}
constexpr uint32_t kKeyLowest = 0x00800000u;  // key of the lowest finite float

// 2^(f/16) - 1 for f in [0, 1): the series of e^x - 1 (x < 0.0434; the next
// term is under 4e-16).
__device__ __forceinline__ double frac_mass(double f) {
  const double x = f * kLn2by16;
  double r = 1.0 / 5040;
  r = fma(r, x, 1.0 / 720);
  r = fma(r, x, 1.0 / 120);
  r = fma(r, x, 1.0 / 24);
  r = fma(r, x, 1.0 / 6);
  r = fma(r, x, 0.5);
  r = fma(r, x, 1.0);
  return r * x;
}
// rint(x 2^s) of 0 <= x 2^s < 2^51 as an integer.
__device__ __forceinline__ uint64_t fixed_point(double x, double scale) {
  const double m = fma(x, scale, 4503599627370496.0);  // + 2^52
  return (uint64_t)__double_as_longlong(m) & 0xfffffffffffffull;
}

template <class T>
__device__ __forceinline__ T wave_incl_scan(T v, int lane) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const T o = __shfl_up(v, d);
    if (lane >= d) v += o;
  }
  return v;
}

// What a row's settings ask for.
struct Ask {
  double c;       // 16 log2(e) / T
  double logm;    // T ln(min_p) (-inf: off)
  int32_t k;      // 0: off
  float p;        // 1: off
  bool greedy, valid;
};

__device__ __forceinline__ Ask ask_of(const TruncParams& P, int64_t seq) {
  const float T = P.temp_ps ? P.temp_ps[seq] : P.temp;
  const float m = P.min_p_ps ? P.min_p_ps[seq] : P.min_p;
  Ask a;
  a.k = P.top_k_ps ? P.top_k_ps[seq] : P.top_k;
  a.p = P.top_p_ps ? P.top_p_ps[seq] : P.top_p;
  a.valid = T >= 0.0f && T < __builtin_huge_valf() && a.k >= 0 && a.p > 0.0f && a.p <= 1.0f &&
            m >= 0.0f && m <= 1.0f;
  a.greedy = T == 0.0f;
  a.c = a.greedy ? 1.0 : kBinsPerNat / (double)T;
  a.logm = m > 0.0f ? (double)T * log((double)m) : -(double)__builtin_huge_valf();
  return a;
}

// The kept entries of a row: key above `key`, or equal with index <= `idx`.
struct Cut {
  uint32_t key;
  int32_t idx;
};
__device__ __forceinline__ bool kept(const Cut& c, uint32_t key, int64_t idx) {
  return key > c.key || (key == c.key && idx <= c.idx);
}
// The more restrictive of two cuts.
__device__ __forceinline__ Cut tighter(const Cut& a, const Cut& b) {
  if (a.key != b.key) return a.key > b.key ? a : b;
  return Cut{a.key, min(a.idx, b.idx)};
}

// Row entries read from memory at every pass.  Thread t's lane load i covers
// entries (i kNT + t) VW ..; sub-chunk i kNW + wave is a wavefront's lane load.
template <int DT>
struct ScanRow {
  const char* row;
  int32_t V;
  static constexpr int VW = Elem<DT>::VW;
  __device__ __forceinline__ int loads() const { return (int)(((int64_t)V + kNT * VW - 1) / (kNT * VW)); }
  // f(entry, logit, the entry's bits) over the thread's entries of lane loads [i0, i1)
  template <class F>
  __device__ __forceinline__ void each(int i0, int i1, F&& f) const {
    for (int i = i0; i < i1; ++i) {
      const int64_t e0 = ((int64_t)i * kNT + threadIdx.x) * VW;
      uint32_t w[4];
      int n = 0;
      if (e0 < V) n = load(e0, w);
#pragma unroll
      for (int e = 0; e < VW; ++e)
        if (e < n) f(e0 + e, value(w, e), bits(w, e));
    }
  }
  // the lane load at entry e0 < V; the number of its entries
  __device__ __forceinline__ int load(int64_t e0, uint32_t (&w)[4]) const {
    const int n = (int)min((int64_t)VW, (int64_t)V - e0);
    const char* a = row + e0 * Elem<DT>::EB;
    if (n == VW) {
      w4 v;
      if constexpr (DT == 1) v = *reinterpret_cast<const w4a2*>(a);
      else v = *reinterpret_cast<const w4a4*>(a);
      w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (DT == 1) {
          const uint16_t* s = reinterpret_cast<const uint16_t*>(a);
          w[j] = (2 * j < n ? (uint32_t)s[2 * j] : 0xff80u) |
                 ((2 * j + 1 < n ? (uint32_t)s[2 * j + 1] : 0xff80u) << 16);
        } else {
          w[j] = j < n ? reinterpret_cast<const uint32_t*>(a)[j] : 0xff800000u;
        }
      }
    }
    return n;
  }
  static __device__ __forceinline__ uint32_t bits(const uint32_t (&w)[4], int e) {
    if constexpr (DT == 1) return (e & 1) ? w[e >> 1] >> 16 : w[e >> 1] & 0xffffu;
    else return w[e];
  }
  static __device__ __forceinline__ float value(const uint32_t (&w)[4], int e) {
    if constexpr (DT == 1)
      return clean(__uint_as_float((e & 1) ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16));
    else return clean(__uint_as_float(w[e]));
  }
};

struct Shared {
  uint64_t mass[kBins];
  uint32_t cnt[kBins];
  uint64_t wave64[kNW];
  double waved[kNW];
  uint32_t wave32[kNW];
  uint32_t red[2];
  // first_reaching's answer
  int32_t found, last;
  uint32_t above_cnt, in_cnt;
  double above_mass, in_mass;
  // the draw's
  uint64_t before;
  int32_t token;
  uint32_t token_key;
};

// Fixed-point scales for rows of V entries: a bin's mass (V terms under
// 0.0444) and the draw's weights (V terms of at most 1) stay under 2^63.
__device__ __forceinline__ int log2_ceil(int32_t V) { return 32 - __builtin_clz((uint32_t)(V - 1) | 1u); }
__device__ __forceinline__ int mass_bits(int32_t V) { return min(51, 67 - log2_ceil(V)); }
__device__ __forceinline__ int draw_bits(int32_t V) { return min(50, 62 - log2_ceil(V)); }

// A wavefront's maximum or minimum over the block, of unsigned values.
template <bool MAX>
__device__ __forceinline__ uint32_t block_extreme(Shared& S, uint32_t x) {
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    const uint32_t o = __shfl_xor(x, d);
    x = MAX ? max(x, o) : min(x, o);
  }
  if ((threadIdx.x & 63) == 0) S.wave32[threadIdx.x >> 6] = x;
  __syncthreads();
  x = S.wave32[0];
#pragma unroll
  for (int i = 1; i < kNW; ++i) x = MAX ? max(x, S.wave32[i]) : min(x, S.wave32[i]);
  __syncthreads();
  return x;
}

// Counts c and masses m, one of each per thread, in thread order: the first
// thread at which the inclusive sum reaches what is wanted (want_c entries, or
// with by_mass a mass of want_m), else the last thread with c != 0; -1 if there
// is none.  S holds the sums before that thread and its own.
__device__ __forceinline__ int first_reaching(Shared& S, uint32_t c, double m, bool by_mass,
                                              uint32_t want_c, double want_m) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t ci = wave_incl_scan(c, lane);
  double mi = wave_incl_scan(m, lane);
  if (lane == 63) {
    S.wave32[wave] = ci;
    S.waved[wave] = mi;
  }
  if (threadIdx.x == 0) {
    S.found = kNoIndex;
    S.last = -1;
  }
  __syncthreads();
  uint32_t bc = 0;
  double bm = 0;
  for (int i = 0; i < wave; ++i) {
    bc += S.wave32[i];
    bm += S.waved[i];
  }
  double me = __shfl_up(mi, 1);
  if (lane == 0) me = 0;
  const bool here = c != 0 && (by_mass ? bm + mi >= want_m : bc + ci >= want_c);
  if (here) atomicMin(&S.found, (int)threadIdx.x);
  if (c != 0) atomicMax(&S.last, (int)threadIdx.x);
  __syncthreads();
  const int at = S.found == kNoIndex ? S.last : S.found;
  if ((int)threadIdx.x == at) {
    S.above_cnt = bc + ci - c;
    S.above_mass = bm + me;
    S.in_cnt = c;
    S.in_mass = m;
  }
  __syncthreads();
  return at;
}

// Where a sum over entries in the order of x (ascending) reaches what is
// wanted: the value of x, the sums before it and those of the entries at it.
struct Reached {
  uint32_t x, above_cnt, in_cnt;
  double above_mass, in_mass;
};

// take(key, entry, x): whether an entry takes part, and its x in [lo, hi].
// Masses are 2^(f/16) per entry.  1024 ranges of x a pass, at most four passes.
template <class Row, class Take>
__device__ Reached narrow(Shared& S, const Row& row, double c, int mb, uint32_t lo, uint32_t hi,
                          bool by_mass, uint32_t want_c, double want_m, Take&& take) {
  Reached r{0, 0, 0, 0.0, 0.0};
  const double scale = exp2((double)mb), unscale = exp2((double)-mb);
  for (;;) {
    const uint32_t span = hi - lo;
    const int shift = max(0, 22 - (span ? __builtin_clz(span) : 32));
    S.cnt[threadIdx.x] = 0;
    S.mass[threadIdx.x] = 0;
    __syncthreads();
    row.each(0, row.loads(), [&](int64_t e, float z, uint32_t) {
      const uint32_t key = key_of(z);
      uint32_t x;
      if (!take(key, e, x) || x < lo || x > hi) return;
      const double t = (double)z * c;
      atomicAdd(&S.cnt[(x - lo) >> shift], 1u);
      atomicAdd((unsigned long long*)&S.mass[(x - lo) >> shift],
                (unsigned long long)fixed_point(frac_mass(t - floor(t)), scale));
    });
    __syncthreads();
    const uint32_t n = S.cnt[threadIdx.x];
    const double m = (double)n + (double)S.mass[threadIdx.x] * unscale;
    const int at = first_reaching(S, n, m, by_mass, want_c - r.above_cnt, want_m - r.above_mass);
    if (at < 0) return r;  // (nothing takes part: no caller asks that)
    r.above_cnt += S.above_cnt;
    r.above_mass += S.above_mass;
    r.in_cnt = S.in_cnt;
    r.in_mass = S.in_mass;
    lo += (uint32_t)at << shift;
    hi = min(hi, lo + ((1u << shift) - 1u));
    __syncthreads();
    if (shift == 0) {
      r.x = lo;
      return r;
    }
  }
}

// The cut of `want_c` entries (or the fewest whose mass reaches want_m) of the
// bin `bin` below the row's maximum, and the mass they have (relative to the
// bin's lower edge).
template <class Row>
__device__ Cut cut_in_bin(Shared& S, const Row& row, double c, double top, int bin, int mb,
                          bool by_mass, uint32_t want_c, double want_m, double& mass) {
  // the bin's keys: a range, as the bins are monotone in the key
  uint32_t lo = 0xffffffffu, hi = 0;
  row.each(0, row.loads(), [&](int64_t, float z, uint32_t) {
    const uint32_t key = key_of(z);
    if (key < kKeyLowest) return;
    const double d = top - floor((double)z * c);
    if (d >= (double)bin && (bin == kBins - 1 || d < (double)(bin + 1))) {
      lo = min(lo, key);
      hi = max(hi, key);
    }
  });
  lo = block_extreme<false>(S, lo);
  hi = block_extreme<true>(S, hi);
  const Reached v = narrow(S, row, c, mb, ~hi, ~lo, by_mass, want_c, want_m,
                           [&](uint32_t key, int64_t, uint32_t& x) {
                             x = ~key;
                             return key >= kKeyLowest;
                           });
  const uint32_t key = ~v.x;
  // of the entries at that key, the first `need` by index
  const double each = v.in_mass / (double)v.in_cnt;
  uint32_t need;
  if (by_mass) {
    const double n = ceil((want_m - v.above_mass) / each);
    need = n < 1.0 ? 1u : n > (double)v.in_cnt ? v.in_cnt : (uint32_t)n;
  } else {
    need = min(want_c - v.above_cnt, v.in_cnt);
  }
  mass = v.above_mass + each * (double)need;
  if (need == v.in_cnt) return Cut{key, kNoIndex};
  const Reached i = narrow(S, row, c, mb, 0u, (uint32_t)(row.V - 1), false, need, 0.0,
                           [&](uint32_t k, int64_t e, uint32_t& x) {
                             x = (uint32_t)e;
                             return k == key;
                           });
  return Cut{key, (int32_t)i.x};
}

// The cut of a row whose largest logit is `zmax` (finite).
template <class Row>
__device__ Cut cut_of(Shared& S, const Row& row, const Ask& a, float zmax) {
  Cut cut{kKeyLowest, kNoIndex};
  // min-p: the lowest float not below max z + T ln(min_p)
  const double zmin = (double)zmax + a.logm;
  if (zmin > (double)of_key(kKeyLowest)) {
    uint32_t k = key_of((float)zmin + 0.0f);
    if ((double)of_key(k) < zmin) ++k;
    cut.key = max(cut.key, k);
  }
  const bool by_k = a.k > 0 && a.k < row.V, by_p = a.p < 1.0f;
  if (!by_k && !by_p) return cut;
  const double top = floor((double)zmax * a.c);
  const int mb = mass_bits(row.V);
  const double scale = exp2((double)mb);
  S.cnt[threadIdx.x] = 0;
  S.mass[threadIdx.x] = 0;
  __syncthreads();
  row.each(0, row.loads(), [&](int64_t, float z, uint32_t) {
    if (!(z > -__builtin_huge_valf())) return;
    const double t = (double)z * a.c, b = floor(t);
    const int bin = (int)fmin(top - b, (double)(kBins - 1));
    atomicAdd(&S.cnt[bin], 1u);
    if (bin < kBins - 1)
      atomicAdd((unsigned long long*)&S.mass[bin],
                (unsigned long long)fixed_point(frac_mass(t - b), scale));
  });
  __syncthreads();
  const uint32_t n = S.cnt[threadIdx.x];
  const double edge = exp2(-(double)threadIdx.x * 0.0625);
  const double m = threadIdx.x == kBins - 1
                       ? 0.0
                       : ((double)n + (double)S.mass[threadIdx.x] * exp2((double)-mb)) * edge;
  // the mass of the first k entries (of all of them)
  double whole = 0.0;
  if (by_k) {
    const int kbin = first_reaching(S, n, m, false, (uint32_t)a.k, 0.0);
    const uint32_t above = S.above_cnt, in = S.in_cnt;
    const double k_above = S.above_mass, in_mass = S.in_mass;
    __syncthreads();
    if ((uint32_t)a.k > above + in) {  // the row has fewer
      whole = k_above + in_mass;
    } else {
      double part;
      cut = tighter(cut, cut_in_bin(S, row, a.c, top, kbin, mb, false, (uint32_t)a.k - above, 0.0,
                                    part));
      whole = k_above + (kbin == kBins - 1 ? 0.0 : part * exp2(-(double)kbin * 0.0625));
    }
  }
  if (!by_p) return cut;
  if (!by_k) {
    (void)first_reaching(S, n, m, false, 0xffffffffu, 0.0);  // (the last filled bin)
    whole = S.above_mass + S.in_mass;
    __syncthreads();
  }
  const double want = (double)a.p * whole;
  const int pbin = first_reaching(S, n, m, true, 0u, want);
  const double above = S.above_mass;
  __syncthreads();
  double part;
  return tighter(cut, cut_in_bin(S, row, a.c, top, pbin, mb, true, 0u,
                                 (want - above) * exp2((double)pbin * 0.0625), part));
}

// Weight of an entry in the draw.
__device__ __forceinline__ uint64_t weight(float z, double c, double zmax, double scale) {
  return fixed_point(exp2(((double)z - zmax) * c * 0.0625), scale);
}

// The kept token at which the cumulative weight in vocabulary order exceeds
// u times the total; `total` is set to the total.  S.token and its key.
template <class Row>
__device__ void draw(Shared& S, const Row& row, const Cut& cut, double c, float zmax, float u,
                     double& total) {
  constexpr int VW = Row::VW;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const double zm = (double)zmax;
  const double scale = exp2((double)draw_bits(row.V));
  int64_t lo = 0, n = ((int64_t)row.V + 64 * VW - 1) / (64 * VW);  // sub-chunks
  uint64_t thr = 0;
  bool first = true;
  for (;;) {
    const int64_t G = (n + kBins - 1) / kBins;  // sub-chunks to a sum
    S.mass[threadIdx.x] = 0;
    __syncthreads();
    for (int i = (int)(lo / kNW); i <= (int)((lo + n - 1) / kNW); ++i) {
      const int64_t sub = (int64_t)i * kNW + wave;
      uint64_t s = 0;
      if (sub >= lo && sub < lo + n)
        row.each(i, i + 1, [&](int64_t e, float z, uint32_t) {
          if (kept(cut, key_of(z), e)) s += weight(z, c, zm, scale);
        });
      if (__any(s != 0)) {
#pragma unroll
        for (int d = 32; d; d >>= 1) s += __shfl_xor((unsigned long long)s, d);
        if (lane == 0) atomicAdd((unsigned long long*)&S.mass[(sub - lo) / G], (unsigned long long)s);
      }
    }
    __syncthreads();
    const uint64_t own = S.mass[threadIdx.x];
    uint64_t in = wave_incl_scan((unsigned long long)own, lane);
    if (lane == 63) S.wave64[wave] = in;
    if (threadIdx.x == 0) S.found = kNoIndex;
    __syncthreads();
    uint64_t base = 0, sum = 0;
#pragma unroll
    for (int i = 0; i < kNW; ++i) {
      if (i < wave) base += S.wave64[i];
      sum += S.wave64[i];
    }
    in += base;
    if (first) {
      const double x = fmin((double)u * (double)sum, (double)sum);
      thr = x > 0.0 ? min((uint64_t)x, sum - 1) : 0;
      total = (double)sum / scale;
      first = false;
    }
    if (in > thr && in - own <= thr) {  // one thread
      S.found = (int)threadIdx.x;
      S.before = in - own;
    }
    __syncthreads();
    const int g = S.found;
    thr -= S.before;
    lo += (int64_t)g * G;
    n = min(G, n - (int64_t)g * G);
    __syncthreads();
    if (G == 1) break;
  }
  if (wave == 0) {
    const int64_t e0 = (lo * 64 + lane) * VW;
    uint32_t w[4];
    const int ne = e0 < row.V ? row.load(e0, w) : 0;
    uint64_t s = 0;
#pragma unroll
    for (int e = 0; e < VW; ++e) {
      if (e >= ne) continue;
      const float z = Row::value(w, e);
      if (kept(cut, key_of(z), e0 + e)) s += weight(z, c, zm, scale);
    }
    const uint64_t in = wave_incl_scan((unsigned long long)s, lane);
    if (in > thr && in - s <= thr) {
      uint64_t at = in - s;
      bool done = false;
#pragma unroll
      for (int e = 0; e < VW; ++e) {
        if (e >= ne || done) continue;
        const float z = Row::value(w, e);
        if (!kept(cut, key_of(z), e0 + e)) continue;
        at += weight(z, c, zm, scale);
        if (at > thr) {
          S.token = (int)(e0 + e);
          S.token_key = key_of(z);
          done = true;
        }
      }
    }
  }
  __syncthreads();
}

// A workgroup per row, which it reads from memory at every pass.
template <int DT>
__global__ void __launch_bounds__(kNT) k_sample(TruncParams P) {
  __shared__ Shared S;
  const int64_t r = blockIdx.x;
  const ScanRow<DT> row{static_cast<const char*>(P.z) + r * P.ld * Elem<DT>::EB, P.V};
  const Ask a = ask_of(P, r);
  float zmax = -__builtin_huge_valf();
  row.each(0, row.loads(), [&](int64_t, float z, uint32_t) { zmax = fmaxf(zmax, z); });
  const uint32_t kmax = block_extreme<true>(S, key_of(zmax));
  zmax = of_key(kmax);
  if (!a.valid || kmax < kKeyLowest) {
    if (threadIdx.x == 0) {
      P.out_token[r] = -1;
      if (P.out_kept) P.out_kept[r] = 0;
      if (P.out_logprob) P.out_logprob[r] = -__builtin_huge_valf();
    }
    return;
  }
  if (a.greedy) {
    uint32_t first = 0xffffffffu;
    row.each(0, row.loads(), [&](int64_t e, float z, uint32_t) {
      if (key_of(z) == kmax) first = min(first, (uint32_t)e);
    });
    first = block_extreme<false>(S, first);
    if (threadIdx.x == 0) {
      P.out_token[r] = (int32_t)first;
      if (P.out_kept) P.out_kept[r] = 1;
      if (P.out_logprob) P.out_logprob[r] = 0.0f;
    }
    return;
  }
  const Cut cut = cut_of(S, row, a, zmax);
  if (P.out_kept) {
    if (threadIdx.x == 0) S.red[0] = 0;
    __syncthreads();
    uint32_t n = 0;
    row.each(0, row.loads(), [&](int64_t e, float z, uint32_t) { n += kept(cut, key_of(z), e); });
#pragma unroll
    for (int d = 32; d; d >>= 1) n += __shfl_xor(n, d);
    if ((threadIdx.x & 63) == 0) atomicAdd(&S.red[0], n);
    __syncthreads();
  }
  double total;
  draw(S, row, cut, a.c, zmax, P.uniforms[r], total);
  if (threadIdx.x == 0) {
    P.out_token[r] = S.token;
    if (P.out_kept) P.out_kept[r] = (int32_t)S.red[0];
    if (P.out_logprob)
      P.out_logprob[r] = (float)(((double)of_key(S.token_key) - (double)zmax) * a.c * kLn2by16 -
                                 log(total));
  }
}

// The row's entries outside `cut` as -inf, the others as they are (all of
// them with `whole`, none with `none`).
template <class Row, int DT>
__device__ void write_cut(const Row& row, char* out, const Cut& cut, bool whole, bool none) {
  constexpr int VW = Row::VW;
  for (int i = 0; i < row.loads(); ++i) {
    const int64_t e0 = ((int64_t)i * kNT + threadIdx.x) * VW;
    if (e0 >= row.V) continue;
    uint32_t w[4], o[4];
    const int n = row.load(e0, w);
#pragma unroll
    for (int e = 0; e < VW; ++e) {
      const bool k = !none && (whole || kept(cut, key_of(Row::value(w, e)), e0 + e));
      if constexpr (DT == 1) {
        const uint32_t b = k ? Row::bits(w, e) : 0xff80u;
        o[e >> 1] = (e & 1) ? o[e >> 1] | (b << 16) : b;
      } else {
        o[e] = k ? w[e] : 0xff800000u;
      }
    }
    char* a = out + e0 * Elem<DT>::EB;
    if (n == VW) {
      const w4 v{o[0], o[1], o[2], o[3]};
      if constexpr (DT == 1) *reinterpret_cast<w4a2*>(a) = v;
      else *reinterpret_cast<w4a4*>(a) = v;
    } else {
#pragma unroll
      for (int e = 0; e < VW; ++e)
        if (e < n) {
          if constexpr (DT == 1) reinterpret_cast<uint16_t*>(a)[e] = (uint16_t)Row::bits(o, e);
          else reinterpret_cast<uint32_t*>(a)[e] = o[e];
        }
    }
  }
}

template <int DT>
__global__ void __launch_bounds__(kNT) k_truncate(TruncParams P) {
  __shared__ Shared S;
  const int64_t r = blockIdx.x;
  const ScanRow<DT> row{static_cast<const char*>(P.z) + r * P.ld * Elem<DT>::EB, P.V};
  char* out = static_cast<char*>(P.out) + r * P.out_ld * Elem<DT>::EB;
  const Ask a = ask_of(P, r / P.rows_per_seq);
  float zmax = -__builtin_huge_valf();
  row.each(0, row.loads(), [&](int64_t, float z, uint32_t) { zmax = fmaxf(zmax, z); });
  const uint32_t kmax = block_extreme<true>(S, key_of(zmax));
  const bool none = !a.valid || kmax < kKeyLowest, whole = a.greedy;
  Cut cut{kKeyLowest, kNoIndex};
  if (!none && !whole) cut = cut_of(S, row, a, of_key(kmax));
  __syncthreads();
  write_cut<ScanRow<DT>, DT>(row, out, cut, whole, none);
}

}  // namespace

// (P.R at most kMaxRows)
hipError_t launch_truncated(const TruncParams& P, int dtype, hipStream_t stream) {
  const dim3 grid((uint32_t)P.R), block(kNT);
  if (P.out) {
    if (dtype == SPC_BF16) k_truncate<1><<<grid, block, 0, stream>>>(P);
    else k_truncate<0><<<grid, block, 0, stream>>>(P);
  } else {
    if (dtype == SPC_BF16) k_sample<1><<<grid, block, 0, stream>>>(P);
    else k_sample<0><<<grid, block, 0, stream>>>(P);
  }
  return hipGetLastError();
}

}  // namespace spc
