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
//            or the mass reaches p times the mass of the first k.  The entries
//            of these bins are taken out; up to kRanked of them are ranked
//            against each other, more are narrowed by counts of ranges of keys
//            (1024 a pass) to one value, and equal values by index.
//   the draw Kept entries weigh 2^((t - t_max)/16) in fixed point: sums are
//            exact, so the inverse CDF in vocabulary order is a function of
//            the inputs alone.  A uniform of less than a unit of them (0) is
//            decided among the entries that weigh nothing, by their masses.
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
constexpr int kBins = kTruncBins;
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

__device__ __forceinline__ double pow2(int e) {  // -1022 <= e <= 1023
  return __longlong_as_double((long long)(1023 + e) << 52);
}
// 2^(f/16) - 1 for f in [0, 1), the series of e^x - 1 at x = f ln(2)/16 < 0.0434.
// In bins, which hold it in units of 2^-37 or less: to the sixth power, the rest
// under 6e-14.  In weights: to the seventh, the rest under 4e-16.
constexpr double kF1 = kLn2by16, kF2 = kF1 * kLn2by16 / 2, kF3 = kF2 * kLn2by16 / 3,
                 kF4 = kF3 * kLn2by16 / 4, kF5 = kF4 * kLn2by16 / 5, kF6 = kF5 * kLn2by16 / 6,
                 kF7 = kF6 * kLn2by16 / 7;
__device__ __forceinline__ double frac_mass(double f) {
  double r = fma(kF7, f, kF6);
  r = fma(r, f, kF5);
  r = fma(r, f, kF4);
  r = fma(r, f, kF3);
  r = fma(r, f, kF2);
  r = fma(r, f, kF1);
  return r * f;
}
// rint(x 2^s) of 0 <= x 2^s < 2^51 as an integer.
constexpr double kTwo52 = 4503599627370496.0;
__device__ __forceinline__ uint64_t fixed_point(double x, double scale) {
  const double m = fma(x, scale, kTwo52);
  return (uint64_t)__double_as_longlong(m) & 0xfffffffffffffull;
}
// The units of 2^-BITS in 2^(f/16) - 1, above the bits of 2^52.
template <int BITS>
__device__ __forceinline__ uint64_t frac_units(double f) {
  constexpr double s = (double)(1ull << BITS);
  double r = fma(kF6 * s, f, kF5 * s);
  r = fma(r, f, kF4 * s);
  r = fma(r, f, kF3 * s);
  r = fma(r, f, kF2 * s);
  r = fma(r, f, kF1 * s);
  return (uint64_t)__double_as_longlong(fma(r, f, kTwo52));
}
constexpr uint64_t kTwo52Bits = 0x4330000000000000ull;

__device__ __forceinline__ int wave_id() {
  return __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
}

// Inclusive sums over a wavefront (DPP row shifts and broadcasts; 64-bit
// values as two halves).
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ uint64_t dpp(uint64_t x) {
  return (uint64_t)dpp<CTRL, ROWS>((uint32_t)x) |
         (uint64_t)dpp<CTRL, ROWS>((uint32_t)(x >> 32)) << 32;
}
template <int CTRL, int ROWS>
__device__ __forceinline__ double dpp(double x) {
  return __longlong_as_double((long long)dpp<CTRL, ROWS>((uint64_t)__double_as_longlong(x)));
}
template <class T>
__device__ __forceinline__ T wave_incl_scan(T v) {
  v += dpp<0x111, 0xf>(v);  // row_shr
  v += dpp<0x112, 0xf>(v);
  v += dpp<0x114, 0xf>(v);
  v += dpp<0x118, 0xf>(v);
  v += dpp<0x142, 0xa>(v);  // row_bcast 15, 31
  v += dpp<0x143, 0xc>(v);
  return v;
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {  // in lane 63
  v = max(v, dpp<0x111, 0xf>(v));
  v = max(v, dpp<0x112, 0xf>(v));
  v = max(v, dpp<0x114, 0xf>(v));
  v = max(v, dpp<0x118, 0xf>(v));
  v = max(v, dpp<0x142, 0xa>(v));
  v = max(v, dpp<0x143, 0xc>(v));
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

// The kept entries of a row: logit above z, or equal with index <= idx.  Logits
// are compared as they are stored: a NaN is never kept, and +inf is not above
// a cut at the largest finite value.
constexpr float kLowest = -3.40282347e38f;  // the lowest finite float
struct Cut {
  float z;
  int32_t idx;
};
__device__ __forceinline__ bool kept(const Cut& c, float z, int64_t idx) {
  const float above = c.z == -kLowest ? __builtin_huge_valf() : c.z;  // uniform
  return z > above || (z >= c.z && idx <= c.idx);
}
// The more restrictive of two cuts.
__device__ __forceinline__ Cut tighter(const Cut& a, const Cut& b) {
  if (a.z != b.z) return a.z > b.z ? a : b;
  return Cut{a.z, min(a.idx, b.idx)};
}


// ------------------------------------------------------------------ rows
template <int DT>
struct RowOf {
  static constexpr int VW = Elem<DT>::VW;
  static __device__ __forceinline__ uint32_t bits(const uint32_t (&w)[4], int e) {
    if constexpr (DT == 1) return (e & 1) ? w[e >> 1] >> 16 : w[e >> 1] & 0xffffu;
    else return w[e];
  }
  static __device__ __forceinline__ float of_bits(uint32_t b) {
    return clean(__uint_as_float(DT == 1 ? b << 16 : b));
  }
  static __device__ __forceinline__ float raw(const uint32_t (&w)[4], int e) {
    if constexpr (DT == 1)
      return __uint_as_float((e & 1) ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
    else return __uint_as_float(w[e]);
  }
  static __device__ __forceinline__ float value(const uint32_t (&w)[4], int e) {
    return clean(raw(w, e));
  }
};
// The lane load at entry e0 < V of a row in memory, -inf behind its end; the
// number of its entries.
template <int DT>
__device__ __forceinline__ int load_lane(const char* row, int64_t e0, int32_t V,
                                         uint32_t (&w)[4]) {
  constexpr int VW = Elem<DT>::VW;
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

// A row read from memory at every pass: thread t's lane load i covers entries
// (i kNT + t) VW ...
template <int DT>
struct ScanRow : RowOf<DT> {
  using RowOf<DT>::VW;
  const char* row;
  int32_t V;
  __device__ __forceinline__ ScanRow(const char* r, int32_t v) : row(r), V(v) {}
  __device__ __forceinline__ int loads() const {
    return (int)(((int64_t)V + kNT * VW - 1) / (kNT * VW));
  }
  __device__ __forceinline__ int load(int64_t e0, uint32_t (&w)[4]) const {
    return load_lane<DT>(row, e0, V, w);
  }
  __device__ __forceinline__ float at(int64_t e) const {
    return RowOf<DT>::of_bits(DT == 1 ? reinterpret_cast<const uint16_t*>(row)[e]
                                      : reinterpret_cast<const uint32_t*>(row)[e]);
  }
  // f(entry, logit as stored, its bits) over the thread's entries
  template <class F>
  __device__ __forceinline__ void each(F&& f) const {
    for (int i = 0; i < loads(); ++i) {
      const int64_t e0 = ((int64_t)i * kNT + threadIdx.x) * VW;
      if (e0 >= V) continue;
      uint32_t w[4];
      const int n = load(e0, w);
#pragma unroll
      for (int e = 0; e < VW; ++e)
        if (e < n) f(e0 + e, RowOf<DT>::raw(w, e), RowOf<DT>::bits(w, e));
    }
  }
};

// A row (or a slice of one) of at most kTruncHeld entries held in LDS, in order; what
// lies behind its end is -inf, which no pass counts.  Thread t's entries are
// the E from t E on, its lane loads taken from another place on by each thread
// so that a wavefront's reads spread over the banks.
template <int DT, int U>
struct HeldRow : RowOf<DT> {
  using RowOf<DT>::VW;
  static constexpr int E = U * VW;
  const w4* lds;
  int32_t V;
  __device__ __forceinline__ HeldRow(const w4* l, int32_t v) : lds(l), V(v) {}
  __device__ __forceinline__ int loads() const { return (V + kNT * VW - 1) / (kNT * VW); }
  __device__ __forceinline__ int load(int64_t e0, uint32_t (&w)[4]) const {
    const w4 v = lds[e0 / VW];
    w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    return (int)min((int64_t)VW, (int64_t)V - e0);
  }
  __device__ __forceinline__ float at(int64_t e) const {
    return RowOf<DT>::of_bits(DT == 1 ? reinterpret_cast<const uint16_t*>(lds)[e]
                                      : reinterpret_cast<const uint32_t*>(lds)[e]);
  }
  template <class F>
  __device__ __forceinline__ void each(F&& f) const {
    if ((int)threadIdx.x * E >= V) return;
    for (int j = 0; j < U; ++j) {
      const int e0 = (int)threadIdx.x * E + ((j + (int)threadIdx.x) & (U - 1)) * VW;
      uint32_t w[4];
      load(e0, w);
#pragma unroll
      for (int e = 0; e < VW; ++e) f(e0 + e, RowOf<DT>::raw(w, e), RowOf<DT>::bits(w, e));
    }
  }
};

// Entries of a row taken out of it.
struct Item {
  uint32_t bits;
  int32_t idx;
};
template <int DT>
struct ItemRow : RowOf<DT> {
  const Item* item;
  int32_t V, n;  // of a row of V entries
  __device__ __forceinline__ ItemRow(const Item* i, int32_t v, int32_t m) : item(i), V(v), n(m) {}
  template <class F>
  __device__ __forceinline__ void each(F&& f) const {
    for (int j = (int)threadIdx.x; j < n; j += kNT) {
      const Item x = item[j];
      f(x.idx, RowOf<DT>::of_bits(x.bits), x.bits);
    }
  }
};

// ------------------------------------------------------------------ the cut
constexpr int kItems = 1024;   // entries of the bins in question held in LDS
constexpr int kRanked = 256;   // as many are ranked against each other

struct Found {
  int32_t state, at;  // 2: reached, 1: the last entry, 0: no entry
  uint32_t above_cnt, in_cnt;
  double above_mass, in_mass;
};

struct Shared {
  uint64_t mass[kBins];
  uint32_t cnt[kBins];
  double edge[kBins];          // 2^(-i/16)
  Item items[kItems];
  double waved[kNW];
  uint64_t wave64[kNW];
  uint32_t wave32[kNW];
  uint32_t n_items;
  Found found[2][kNW];
  Cut cut;                     // resolve_ranked's answer
  // the draw's
  int32_t sum_at;
  uint64_t before;
};

__device__ __forceinline__ int log2_ceil(int32_t V) {
  return 32 - __builtin_clz((uint32_t)(V - 1) | 1u);
}
// Fixed-point scales: sums of V terms of at most 2^(1/16) stay under 2^63,
// and a term under 2^51.
__device__ __forceinline__ int sum_bits(int32_t V) { return min(50, 61 - log2_ceil(V)); }
// Bin masses are sums of units of 2^-37; of at most kTruncHeld entries they take
// 48 bits (kTruncHeld terms under 0.0444 2^37) under 16 of count.
constexpr int kPackBits = 37;

__device__ __forceinline__ uint32_t block_max(uint32_t* wave32, uint32_t x) {
  x = wave_max(x);
  if ((threadIdx.x & 63) == 63) wave32[threadIdx.x >> 6] = x;
  __syncthreads();
  x = wave_max(wave32[threadIdx.x & 15]);
  x = (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
  __syncthreads();
  return x;
}
template <bool MAX>
__device__ __forceinline__ uint32_t block_extreme(Shared& S, uint32_t x) {
  x = block_max(S.wave32, MAX ? x : ~x);
  return MAX ? x : ~x;
}

// A lane's value, in every lane (`lane` is uniform).
template <class T>
__device__ __forceinline__ T lane_value(T v, int lane) {
  if constexpr (sizeof(T) == 4) {
    return (T)__builtin_amdgcn_readlane((int)v, lane);
  } else {
    const uint64_t x = __builtin_bit_cast(uint64_t, v);
    const uint64_t y = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, lane) |
                       (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(x >> 32), lane)
                           << 32;
    return __builtin_bit_cast(T, y);
  }
}
template <class T>
__device__ __forceinline__ T row_incl_scan(T v) {  // over 16 lanes
  v += dpp<0x111, 0xf>(v);
  v += dpp<0x112, 0xf>(v);
  v += dpp<0x114, 0xf>(v);
  v += dpp<0x118, 0xf>(v);
  return v;
}

// Counts c and masses m, one of each per thread, summed in thread order.  Every
// wavefront scans the wavefronts' 16 sums in its first lanes.
struct Sums {
  uint32_t c, upto_c;
  double m, upto_m, before_m;  // inclusive, exclusive
};
__device__ __forceinline__ Sums sums_of(Shared& S, uint32_t c, double m) {
  const int lane = threadIdx.x & 63, wave = wave_id();
  const uint32_t ci = wave_incl_scan(c);
  const double mi = wave_incl_scan(m);
  if (lane == 63) {
    S.wave32[wave] = ci;
    S.waved[wave] = mi;
  }
  __syncthreads();
  const uint32_t wc = row_incl_scan(S.wave32[lane & 15]);
  const double wm = row_incl_scan(S.waved[lane & 15]);
  const uint32_t bc = wave ? lane_value(wc, wave - 1) : 0u;
  const double bm = wave ? lane_value(wm, wave - 1) : 0.0;
  double me = dpp<0x138, 0xf>(mi);  // wave_shr: the lane before
  if (lane == 0) me = 0;
  __syncthreads();
  return Sums{c, bc + ci, m, bm + mi, bm + me};
}

// The first thread whose sum up to it reaches want_c entries (by_mass: a mass
// of want_m), or the last thread with an entry; -1 if there is none.  And the
// sums before that thread, and its own.  `slot` differs from the last call's.
struct Reached {
  int at;
  uint32_t above_cnt, in_cnt;
  double above_mass, in_mass;
};
__device__ __forceinline__ Reached reach(Shared& S, int slot, const Sums& x, bool by_mass,
                                         uint32_t want_c, double want_m) {
  const int lane = threadIdx.x & 63, wave = wave_id();
  const bool some = x.c != 0;
  const uint64_t any = __ballot(some && (by_mass ? x.upto_m >= want_m : x.upto_c >= want_c));
  const uint64_t all = __ballot(some);
  const int mine = any ? __builtin_ctzll(any) : all ? 63 - __builtin_clzll(all) : 0;
  if (lane == mine)
    S.found[slot][wave] = Found{any ? 2 : all ? 1 : 0, (int)threadIdx.x, x.upto_c - x.c, x.c,
                                x.before_m, x.m};
  __syncthreads();
  const int state = S.found[slot][lane & 15].state;
  const uint32_t yes = (uint32_t)__ballot(state == 2) & 0xffffu;
  const uint32_t may = (uint32_t)__ballot(state == 1) & 0xffffu;
  if (!(yes | may)) return Reached{-1, 0, 0, 0.0, 0.0};
  const Found f = S.found[slot][yes ? __builtin_ctz(yes) : 31 - __builtin_clz(may)];
  return Reached{f.at, f.above_cnt, f.in_cnt, f.above_mass, f.in_mass};
}

// The bin of t below a row's top bin.
__device__ __forceinline__ int bin_of(double top, double t) {
  return (int)fmin(top - floor(t), (double)(kBins - 1));
}

// The mass of an entry relative to its bin's lower edge, rounded as the bins
// hold it: sums over entries and over bins then agree where no rounding need
// part them (a row of equal logits, say, and its half).
constexpr double kUnit = 1.0 / (double)(1ull << kPackBits);
__device__ __forceinline__ double entry_mass(double f) {
  return 1.0 + (double)(frac_units<kPackBits>(f) - kTwo52Bits) * kUnit;
}

// The bin of an entry (as it is stored), which is neither -inf nor NaN, and the
// units of its mass above 2^52's bits.  (The last bin's mass is not used.)
__device__ __forceinline__ uint32_t bin_and_units(float z, double c, double top, uint64_t& m) {
  const double t = (double)fminf(z, -kLowest) * c, b = floor(t);
  m = frac_units<kPackBits>(t - b);
  return min((uint32_t)(int)(top - b), (uint32_t)(kBins - 1));
}
constexpr uint64_t kOnePacked = (1ull << 48) - kTwo52Bits;

// Entries of a bfloat16 row take few values: those of magnitudes 2^-6 to 2^6 are
// counted by value, and each value met enters its bin once, as often as it was
// met.  A count is a few integer operations and one 32-bit add in LDS, where
// the mass of an entry is about 20 operations in 64 bits (65.5M entries: k_slice_bins
// 80 us entry by entry).  Others go to their bins one by one.
constexpr uint32_t kMagFirst = 0x3c80, kMags = 12 * 128, kValues = 2 * kMags;
// Adds an entry to the bins of at most kTruncHeld entries.
__device__ __forceinline__ void add_packed(uint64_t* mass, float z, double c, double top) {
  if (!(z > -__builtin_huge_valf())) return;
  uint64_t m;
  const uint32_t bin = bin_and_units(z, c, top, m);
  atomicAdd((unsigned long long*)&mass[bin], (unsigned long long)(m + kOnePacked));
}
// To the bins of any number: counts apart.
__device__ __forceinline__ void add_unpacked(Shared& S, float z, double c, double top) {
  if (!(z > -__builtin_huge_valf())) return;
  uint64_t m;
  const uint32_t bin = bin_and_units(z, c, top, m);
  atomicAdd(&S.cnt[bin], 1u);
  atomicAdd((unsigned long long*)&S.mass[bin], (unsigned long long)(m - kTwo52Bits));
}

__device__ __forceinline__ void add_value(uint64_t* mass, uint32_t* values, uint32_t h, double c,
                                          double top) {
  const uint32_t m = (h & 0x7fffu) - kMagFirst;
  if (m < kMags) {
    atomicAdd(&values[m + (h >> 15) * kMags], 1u);
  } else {
    add_packed(mass, __uint_as_float(h << 16), c, top);
  }
}
// The counted values into their bins (between barriers).
__device__ __forceinline__ void add_values(uint64_t* mass, const uint32_t* values, double c,
                                           double top) {
  for (uint32_t i = threadIdx.x; i < kValues; i += kNT) {
    const uint64_t n = values[i];
    if (!n) continue;
    const uint32_t h = i < kMags ? i + kMagFirst : (i - kMags + kMagFirst) | 0x8000u;
    uint64_t m;
    const uint32_t bin = bin_and_units(__uint_as_float(h << 16), c, top, m);
    atomicAdd((unsigned long long*)&mass[bin], (unsigned long long)((m + kOnePacked) * n));
  }
}

// What a row's bins say about its cut.  Bins are counted down from the top.
struct Plan {
  int32_t kbin;      // the bin top-k ends in, or -1
  uint32_t k_need;   // entries it keeps of that bin
  double k_above;    // mass of the bins above it, or (kbin = -1) of all
  int32_t plo, phi;  // the bins top-p may end in, or -1 (not before plo, if k ends inside its bin)
  double p_above;    // mass of the bins above plo
  uint32_t items;    // entries in those bins
};

// n entries of mass m (relative to the top bin's lower edge): thread i's bin i.
// key_bin: the bin of min-p's cut (kBins: none).
__device__ __forceinline__ Plan make_plan(Shared& S, const Ask& a, int32_t V, uint32_t n,
                                          double m, int key_bin) {
  Plan p{-1, 0, 0.0, -1, -1, 0.0, 0};
  const bool by_p = a.p < 1.0f;
  const Sums x = sums_of(S, n, m);
  // (no count is reached without top-k: the last filled bin, whose sums are the row's)
  const Reached k = reach(S, 0, x, false, a.k > 0 && a.k < V ? (uint32_t)a.k : 0xffffffffu, 0.0);
  const bool by_k = a.k > 0 && a.k < V && (uint32_t)a.k <= k.above_cnt + k.in_cnt;
  double lo, hi;  // bounds of the mass of the first k
  if (by_k) {
    p.kbin = k.at;
    p.k_need = (uint32_t)a.k - k.above_cnt;
    p.k_above = lo = k.above_mass;
    hi = k.above_mass + k.in_mass;
    p.items = k.in_cnt;
  } else {
    p.k_above = lo = hi = k.above_mass + k.in_mass;
  }
  if (by_p) {
    // (sums over bins and sums over entries differ in rounding: far less than 2^-30)
    const Reached l = reach(S, 1, x, true, 0u, (double)a.p * lo * (1.0 - 0x1p-30));
    const Reached h = reach(S, 0, x, true, 0u, (double)a.p * hi * (1.0 + 0x1p-30));
    p.plo = l.at;
    p.phi = h.at;
    p.p_above = l.above_mass;
    p.items = h.above_cnt + h.in_cnt - l.above_cnt + (p.phi < p.kbin ? p.items : 0u);
  }
  // min-p's cut lies above them: they do not matter
  if (by_p ? key_bin < p.plo : by_k && key_bin < p.kbin) {
    p.kbin = p.plo = p.phi = -1;
    p.items = 0;
  }
  return p;
}

// The lowest float whose t is at least `edge` (t is monotone in the logit).
__device__ __forceinline__ float lowest_at(double edge, double c) {
  const double g = fmin(fmax(edge / c, (double)kLowest), -(double)kLowest);
  uint32_t k = key_of((float)g + 0.0f);
  while (k > kKeyLowest && floor((double)of_key(k - 1) * c) >= edge) --k;
  while (k < ~kKeyLowest && floor((double)of_key(k) * c) < edge) ++k;
  return of_key(k);
}
// The logits of bins first .. last: lo <= z, not z >= hi (NaN: no bound; +inf too
// is under it).
struct Range {
  float lo, hi;
};
// The logits of the bins in question: two ranges.
struct Question {
  Range k, p;
};
// (the four edges in four lanes)
__device__ __forceinline__ Question question_of(const Plan& p, double top, double c) {
  const int lane = threadIdx.x & 63;
  const bool of_k = lane < 2, low = !(lane & 1);
  const int first = of_k ? p.kbin : p.plo, last = of_k ? p.kbin : p.phi;
  float z;
  if (first < 0) z = low ? __builtin_nanf("") : 0.0f;  // (no logit is >= NaN)
  else if (low && last >= kBins - 1) z = kLowest;
  else if (!low && first == 0) z = __builtin_nanf("");
  else z = lowest_at(low ? top - last : top - first + 1.0, c);
  const auto lane_z = [z](int i) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(z), i));
  };
  return Question{{lane_z(0), lane_z(1)}, {lane_z(2), lane_z(3)}};
}
__device__ __forceinline__ bool asked(const Question& q, float z) {
  return (z >= q.k.lo && !(z >= q.k.hi)) || (z >= q.p.lo && !(z >= q.p.hi));
}

// Where a sum over entries in ascending x reaches what is wanted: the value of
// x, the sums before it and those of the entries at it.
// take(key, entry, x): whether an entry takes part, and its x in [lo, hi].
// Masses are relative to the edge of bin `first` (no entry lies above it).  1024
// ranges of x a pass, at most four passes.
struct Narrowed {
  uint32_t x, above_cnt, in_cnt;
  double above_mass, in_mass;
};
template <class Row, class Take>
__device__ __noinline__ Narrowed narrow(Shared& S, const Row& row, double c, double top,
                                        int first, uint32_t lo, uint32_t hi, bool masses, bool by_mass,
                                        uint32_t want_c, double want_m, Take take) {
  Narrowed r{0, 0, 0, 0.0, 0.0};
  int slot = 0;
  const int sb = sum_bits(row.V);
  const double scale = pow2(sb), unscale = pow2(-sb);
  for (;;) {
    const uint32_t span = hi - lo;
    const int shift = max(0, 22 - (span ? __builtin_clz(span) : 32));
    S.cnt[threadIdx.x] = 0;
    S.mass[threadIdx.x] = 0;
    __syncthreads();
    row.each([&](int64_t e, float raw, uint32_t) {
      const float z = clean(raw);
      const uint32_t key = key_of(z);
      uint32_t x;
      if (!take(key, e, x) || x < lo || x > hi) return;
      atomicAdd(&S.cnt[(x - lo) >> shift], 1u);
      if (masses) {
        const double t = (double)z * c, b = floor(t);
        const int bin = (int)fmin(top - b, (double)(kBins - 1));
        atomicAdd((unsigned long long*)&S.mass[(x - lo) >> shift],
                  (unsigned long long)fixed_point(entry_mass(t - b) * S.edge[bin - first],
                                                  scale));
      }
    });
    __syncthreads();
    const uint32_t n = S.cnt[threadIdx.x];
    const Reached f = reach(S, slot ^= 1, sums_of(S, n, (double)S.mass[threadIdx.x] * unscale),
                            by_mass, want_c - r.above_cnt, want_m - r.above_mass);
    if (f.at < 0) return r;  // (nothing takes part: no caller asks that)
    r.above_cnt += f.above_cnt;
    r.above_mass += f.above_mass;
    r.in_cnt = f.in_cnt;
    r.in_mass = f.in_mass;
    lo += (uint32_t)f.at << shift;
    hi = min(hi, lo + ((1u << shift) - 1u));
    if (shift == 0) {
      r.x = lo;
      return r;
    }
  }
}

// The cut that keeps want_c entries (or the fewest whose mass reaches want_m,
// relative to the edge of `first`) of bins first .. last, and their mass.
template <class Row>
__device__ __noinline__ Cut cut_in_bins(Shared& S, const Row& row, double c, double top,
                                        int first, int last, bool by_mass, uint32_t want_c, double want_m,
                                        double& mass) {
  // the keys there are in the bins
  const Range in = question_of(Plan{-1, 0, 0.0, first, last, 0.0, 0}, top, c).p;
  uint32_t lo = 0xffffffffu, hi = 0;
  row.each([&](int64_t, float z, uint32_t) {
    if (z >= in.lo && !(z >= in.hi)) {
      const uint32_t key = key_of(clean(z));
      lo = min(lo, key);
      hi = max(hi, key);
    }
  });
  lo = block_extreme<false>(S, lo);
  hi = block_extreme<true>(S, hi);
  const Narrowed v = narrow(S, row, c, top, first, ~hi, ~lo, true, by_mass, want_c, want_m,
                            [](uint32_t key, int64_t, uint32_t& x) {
                              x = ~key;
                              return true;
                            });
  const uint32_t key = ~v.x;
  // of the entries at that key, the first `need` by index
  const double each = v.in_mass / (double)v.in_cnt;
  uint32_t need;
  if (by_mass) {
    const double n = ceil((want_m - v.above_mass) / each);
    need = n >= (double)v.in_cnt ? v.in_cnt : n > 1.0 ? (uint32_t)n : 1u;
  } else {
    need = min(want_c - v.above_cnt, v.in_cnt);
  }
  mass = v.above_mass + each * (double)need;
  if (need == v.in_cnt) return Cut{of_key(key), kNoIndex};
  const Narrowed i = narrow(S, row, c, top, first, 0u, (uint32_t)(row.V - 1), false, false, need, 0.0,
                            [key](uint32_t k, int64_t e, uint32_t& x) {
                              x = (uint32_t)e;
                              return k == key;
                            });
  return Cut{of_key(key), (int32_t)i.x};
}

// The mass that top-p asks for of bins plo and on, `whole` being that of the first
// k.  Sums of up to V terms are rounded at 2^-53 here and there: what comes within
// 2^-48 of the whole has reached it, so that entries of one mass are cut where
// their number says (p = 1/2 of 262 142 equal ones: 131 071).  p has 24 bits: up to
// 2^24 such entries p n is an integer or further from one than 2^-48 p n.
__device__ __forceinline__ double wanted(const Ask& a, const Plan& p, double whole) {
  return (double)a.p * whole * (1.0 - 0x1p-48) - p.p_above;
}

// The cut by top-k and top-p, from the entries of the bins in question (or all
// entries of the row).
template <class Row>
__device__ __forceinline__ Cut resolve(Shared& S, const Row& row, const Ask& a, double top,
                                       const Plan& p) {
  Cut cut{kLowest, kNoIndex};
  double whole = p.k_above;
  if (p.kbin >= 0) {
    double part;
    cut = cut_in_bins(S, row, a.c, top, p.kbin, p.kbin, false, p.k_need, 0.0, part);
    if (p.kbin < kBins - 1) whole += part * S.edge[p.kbin];
  }
  if (p.plo >= 0) {
    double part;
    const double want = wanted(a, p, whole) / S.edge[p.plo];
    cut = tighter(cut, cut_in_bins(S, row, a.c, top, p.plo, p.phi, true, 0u, want, part));
  }
  return cut;
}

// The same for at most kRanked entries in LDS: each entry's place in the order
// is counted against all others, by the whole workgroup; the sums over the
// places are the first wavefront's, four places a lane.
template <int DT>
__device__ __forceinline__ Cut resolve_ranked(Shared& S, const Ask& a, double top, const Plan& p,
                                              int n) {
  using Row = RowOf<DT>;
  static_assert(kRanked == 256 && kNT == 4 * kRanked, "four threads an entry, four entries a lane");
  uint32_t* place = S.cnt;            // (no bin is in use)
  uint32_t* order = S.cnt + kRanked;
  const int j = (int)threadIdx.x & (kRanked - 1);
  if (threadIdx.x < kRanked) place[j] = 0;
  __syncthreads();
  if (j < n) {
    const Item x = S.items[j];
    const float z = Row::of_bits(x.bits);
    uint32_t c = 0;
    for (int i = (int)threadIdx.x / kRanked; i < n; i += kNT / kRanked) {
      const Item y = S.items[i];
      const float zy = Row::of_bits(y.bits);
      c += zy > z || (zy == z && y.idx < x.idx);
    }
    if (c) atomicAdd(&place[j], c);
  }
  __syncthreads();
  if ((int)threadIdx.x < n) order[place[j]] = (uint32_t)j;
  __syncthreads();
  if (threadIdx.x < 64) {
    const int lane = (int)threadIdx.x;
    int bin[4];
    double mass[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      bin[e] = -2;
      mass[e] = 0.0;
      if (4 * lane + e < n) {
        const double t = (double)Row::of_bits(S.items[order[4 * lane + e]].bits) * a.c;
        bin[e] = bin_of(top, t);
        mass[e] = entry_mass(t - floor(t));
      }
    }
    // the place in bins first .. last that reaches what is wanted (else their last)
    const auto reach_place = [&](int first, int last, bool by_mass, double want) {
      double sum = 0.0, own[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool in = bin[e] >= first && bin[e] <= last;
        own[e] = !in ? 0.0 : by_mass ? mass[e] * S.edge[bin[e] - first] : 1.0;
        sum += own[e];
      }
      const double in = wave_incl_scan(sum);
      double before = dpp<0x138, 0xf>(in);  // wave_shr: the lane before
      if (lane == 0) before = 0.0;
      const uint64_t yes = __ballot(sum > 0.0 && in >= want), some = __ballot(sum > 0.0);
      const int at = yes ? __builtin_ctzll(yes) : 63 - __builtin_clzll(some | 1);
      int e_at = -1;
      double s = before;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (own[e] > 0.0 && (e_at < 0 || s < want)) {
          e_at = e;
          s += own[e];
        }
      }
      return 4 * at + __builtin_amdgcn_readlane(e_at, at);
    };
    Cut cut{kLowest, kNoIndex};
    double whole = p.k_above;
    const auto cut_at = [&](int at) {
      const Item x = S.items[order[max(at, 0)]];
      return Cut{Row::of_bits(x.bits), x.idx};
    };
    if (p.kbin >= 0) {
      const int at = reach_place(p.kbin, p.kbin, false, (double)p.k_need);
      cut = cut_at(at);
      if (p.kbin < kBins - 1) {  // the mass of the bin's entries up to there
        double m = 0.0;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (bin[e] == p.kbin && 4 * lane + e <= at) m += mass[e];
        m = lane_value(wave_incl_scan(m), 63);
        whole += m * S.edge[p.kbin];
      }
    }
    if (p.plo >= 0)
      cut = tighter(cut, cut_at(reach_place(p.plo, p.phi, true,
                                            wanted(a, p, whole) / S.edge[p.plo])));
    if (lane == 0) S.cut = cut;
  }
  __syncthreads();
  return S.cut;
}

// min-p's cut: the lowest float not below max z + T ln(min_p).
__device__ __forceinline__ Cut min_p_cut(const Ask& a, float zmax) {
  Cut cut{kLowest, kNoIndex};
  const double zmin = (double)zmax + a.logm;
  if (zmin > (double)kLowest) {
    uint32_t k = key_of((float)zmin + 0.0f);
    if ((double)of_key(k) < zmin) ++k;
    cut.z = of_key(k);
  }
  return cut;
}
__device__ __forceinline__ int cut_bin(const Ask& a, const Cut& c, double top) {
  return c.z > kLowest ? bin_of(top, (double)c.z * a.c) : kBins;
}

// 2^-(i/16): a product of at most four roots of 2 and a power (within 2^-50).
__device__ __forceinline__ void fill_edges(Shared& S) {
  const int i = (int)threadIdx.x;
  double x = pow2(-(i >> 4));
  x *= i & 8 ? 0.70710678118654752440 : 1.0;
  x *= i & 4 ? 0.84089641525371454303 : 1.0;
  x *= i & 2 ? 0.91700404320467123174 : 1.0;
  x *= i & 1 ? 0.95760328069857364694 : 1.0;
  S.edge[i] = x;
}

// The cut of a row in one workgroup; zmax its largest logit (finite), `whole` the
// row in memory.  PACK: at most kTruncHeld entries.
template <bool PACK, int DT, class Row>
__device__ __forceinline__ Cut cut_of(Shared& S, uint32_t* values, const Row& row,
                                      const ScanRow<DT>& whole, const Ask& a, float zmax,
                                      double top) {
  const Cut floor_cut = min_p_cut(a, zmax);
  if (!(a.k > 0 && a.k < row.V) && a.p >= 1.0f) return floor_cut;
  S.cnt[threadIdx.x] = 0;
  S.mass[threadIdx.x] = 0;
  if (threadIdx.x == 0) S.n_items = 0;
  if constexpr (PACK && DT == 1)
    for (uint32_t i = threadIdx.x; i < kValues; i += kNT) values[i] = 0;
  __syncthreads();
  if constexpr (PACK && DT == 1) {
    row.each([&](int64_t, float, uint32_t h) { add_value(S.mass, values, h, a.c, top); });
    __syncthreads();
    add_values(S.mass, values, a.c, top);
  } else if constexpr (PACK) {
    row.each([&](int64_t, float z, uint32_t) { add_packed(S.mass, z, a.c, top); });
  } else {
    row.each([&](int64_t, float z, uint32_t) { add_unpacked(S, z, a.c, top); });
  }
  __syncthreads();
  uint64_t m = S.mass[threadIdx.x];
  const uint32_t n = PACK ? (uint32_t)(m >> 48) : S.cnt[threadIdx.x];
  if (PACK) m &= (1ull << 48) - 1;
  const double mass = threadIdx.x == kBins - 1
                          ? 0.0
                          : ((double)n + (double)m * kUnit) * S.edge[threadIdx.x];
  const Plan p = make_plan(S, a, row.V, n, mass, cut_bin(a, floor_cut, top));
  if (p.kbin < 0 && p.plo < 0) return floor_cut;
  if (p.items > (uint32_t)kItems) return tighter(floor_cut, resolve(S, whole, a, top, p));
  const Question q = question_of(p, top, a.c);
  row.each([&](int64_t e, float z, uint32_t bits) {
    if (asked(q, z)) {
      const uint32_t at = atomicAdd(&S.n_items, 1u);
      if (at < (uint32_t)kItems) S.items[at] = Item{bits, (int32_t)e};
    }
  });
  __syncthreads();
  if (p.items <= (uint32_t)kRanked)
    return tighter(floor_cut, resolve_ranked<DT>(S, a, top, p, (int)p.items));
  return tighter(floor_cut,
                 resolve(S, ItemRow<DT>(S.items, row.V, (int)p.items), a, top, p));
}

// ------------------------------------------------------------------ the draw
// Weight of an entry: 2^((t - top)/16), 64 octaves below the top none.
__device__ __forceinline__ uint64_t weight(const Shared& S, float z, double c, double top,
                                           double scale) {
  const double t = (double)z * c, b = floor(t);
  const int bin = (int)fmin(top - b, (double)(kBins - 1));
  return bin < kBins - 1 ? fixed_point((1.0 + frac_mass(t - b)) * S.edge[bin], scale) : 0;
}

// Weights `own`, one per thread in vocabulary order: the thread at which their
// sum exceeds thr (first: thr is set to u times the total); thr becomes what is
// left of it there.  Returns the total.
__device__ __forceinline__ uint64_t find_sum(Shared& S, uint64_t own, bool first, float u,
                                             uint64_t& thr, int& at) {
  const int lane = threadIdx.x & 63, wave = wave_id();
  uint64_t in = wave_incl_scan(own);
  if (lane == 63) S.wave64[wave] = in;
  __syncthreads();
  const uint64_t ws = row_incl_scan(S.wave64[lane & 15]);
  const uint64_t sum = lane_value(ws, 15);
  in += wave ? lane_value(ws, wave - 1) : 0;
  if (first) {
    // floor(u sum), exactly (u is a float32, 2^56 u an integer but for u under
    // 2^-32): a uniform that falls on the border between two tokens is decided
    // as the definition says, in a row of equal weights too
    const uint64_t x = u > 0.0f ? (uint64_t)(fmin((double)u, 1.0) * 0x1p56) : 0;
    const uint64_t at_u = (uint64_t)__umul64hi(sum, x) << 8 | (sum * x) >> 56;
    thr = at_u < sum ? at_u : sum - 1;
  }
  if (in > thr && in - own <= thr) {  // one thread
    S.sum_at = (int)threadIdx.x;
    S.before = in - own;
  }
  __syncthreads();
  at = S.sum_at;
  thr -= S.before;
  return sum;
}

// The kept token at weight thr of entries [lo, lo + n) of a row, which have that
// much: each thread sums a share of them, until a share is one entry.
template <class Row>
__device__ __forceinline__ int64_t draw_among(Shared& S, const Row& row, const Cut& cut, double c,
                                              double top, double scale, int64_t lo, int64_t n,
                                              uint64_t thr) {
  for (;;) {
    const int64_t q = (n + kNT - 1) / kNT;
    const int64_t e0 = (int64_t)threadIdx.x * q, e1 = min(e0 + q, n);
    uint64_t s = 0;
    for (int64_t e = lo + e0; e < lo + e1; ++e) {
      const float z = row.at(e);
      if (kept(cut, z, e)) s += weight(S, z, c, top, scale);
    }
    int at;
    (void)find_sum(S, s, false, 0.0f, thr, at);
    lo += (int64_t)at * q;
    n = min(q, n - (int64_t)at * q);
    __syncthreads();
    if (q == 1) return lo;
  }
}

// A uniform of less than one unit of the weights (0, as a rule) falls on `token`
// among the weights, the first that does not round to nothing.  The entries
// before it have masses all the same: the first of them whose cumulative mass
// exceeds x units (u times the total), in 64-bit floats, or `token`.  (A mass is
// relative to the largest: one that is 0 there, past 2^-1074, is none.)
template <int DT>
__device__ __noinline__ int64_t draw_below_a_unit(Shared& S, const ScanRow<DT>& row, const Cut& cut,
                                                  double c, double top, double scale, float zmax,
                                                  int64_t token, double x) {
  const double t_max = (double)zmax * c, most = exp2((t_max - top) * 0.0625) * scale;
  int64_t lo = 0, n = token;
  for (int slot = 1; n > 0; slot ^= 1) {
    const int64_t q = (n + kNT - 1) / kNT, e0 = (int64_t)threadIdx.x * q;
    uint32_t some = 0;
    double m = 0.0;
    for (int64_t e = lo + e0; e < lo + min(e0 + q, n); ++e) {
      const float z = row.at(e);
      const double w = kept(cut, z, e) ? exp2(((double)z * c - t_max) * 0.0625) * most : 0.0;
      some += w > 0.0;
      m += w;
    }
    const double past = __longlong_as_double(__double_as_longlong(x) + 1);  // the next float
    const Reached f = reach(S, slot, sums_of(S, some, m), true, 0u, past);
    if (f.at < 0 || (lo == 0 && n == token && !(f.above_mass + f.in_mass > x))) return token;
    lo += (int64_t)f.at * q;
    n = min(q, n - (int64_t)f.at * q);
    x = fmax(x - f.above_mass, 0.0);
    if (q == 1) return lo;
  }
  return token;
}
template <int DT>
__device__ __forceinline__ int64_t draw_past_units(Shared& S, const ScanRow<DT>& row, const Cut& cut,
                                                   double c, double top, double scale, float zmax,
                                                   int64_t token, float u, uint64_t sum) {
  const double x = u > 0.0f ? (double)u * (double)sum : 0.0;
  return x < 1.0 ? draw_below_a_unit(S, row, cut, c, top, scale, zmax, token, x) : token;
}

// Entries kept, over the block.
__device__ __forceinline__ uint32_t block_sum(Shared& S, uint32_t k) {
  k = wave_incl_scan(k);
  if ((threadIdx.x & 63) == 63) S.wave32[threadIdx.x >> 6] = k;
  __syncthreads();
  k = lane_value(row_incl_scan(S.wave32[threadIdx.x & 15]), 15);
  __syncthreads();
  return k;
}

__device__ __forceinline__ void no_token(const TruncParams& P, int64_t r) {
  if (threadIdx.x == 0) {
    P.out_token[r] = -1;
    if (P.out_kept) P.out_kept[r] = 0;
    if (P.out_logprob) P.out_logprob[r] = -__builtin_huge_valf();
  }
}
__device__ __forceinline__ void greedy_token(const TruncParams& P, int64_t r, uint32_t token) {
  if (threadIdx.x == 0) {
    P.out_token[r] = (int32_t)token;
    if (P.out_kept) P.out_kept[r] = 1;
    if (P.out_logprob) P.out_logprob[r] = 0.0f;
  }
}
__device__ __forceinline__ void drawn_token(const TruncParams& P, int64_t r, int64_t token,
                                            float z, const Ask& a, double top, double total,
                                            uint32_t n_kept) {
  if (threadIdx.x == 0) {
    P.out_token[r] = (int32_t)token;
    if (P.out_kept) P.out_kept[r] = (int32_t)n_kept;
    if (P.out_logprob)
      P.out_logprob[r] = (float)(((double)z * a.c - top) * kLn2by16 - log(total));
  }
}

// The weight of a thread's kept entries of a held row, and their number.  The
// weights are taken one of each thread at a time: few of a thread's entries are
// kept as a rule, and some of every wavefront's.
template <int DT, int U>
__device__ __forceinline__ uint64_t held_weight(const Shared& S, const HeldRow<DT, U>& row,
                                                int64_t first, const Cut& cut, const Ask& a,
                                                double top, double scale, uint32_t& n) {
  constexpr int VW = Elem<DT>::VW, E = HeldRow<DT, U>::E;
  static_assert(E <= 32, "a bit for each of a thread's entries");
  uint32_t mask = 0;
  if ((int)threadIdx.x * E < row.V)
    for (int j = 0; j < U; ++j) {
      const int at = ((j + (int)threadIdx.x) & (U - 1)) * VW, e0 = (int)threadIdx.x * E + at;
      uint32_t w[4], bits = 0;
      row.load(e0, w);
#pragma unroll
      for (int e = 0; e < VW; ++e)
        bits |= (kept(cut, RowOf<DT>::raw(w, e), first + e0 + e) ? 1u : 0u) << e;
      mask |= bits << at;
    }
  n = __popc(mask);
  uint64_t s = 0;
  while (mask) {
    const int e = __builtin_ctz(mask);
    mask &= mask - 1;
    s += weight(S, row.at((int)threadIdx.x * E + e), a.c, top, scale);
  }
  return s;
}

// The draw of a row in one workgroup: held, or read from memory.
template <int DT, int U>
__device__ __forceinline__ void draw(Shared& S, const TruncParams& P, int64_t r,
                                     const HeldRow<DT, U>& row, const ScanRow<DT>& mem,
                                     const Cut& cut, const Ask& a, double top, float zmax) {
  constexpr int E = HeldRow<DT, U>::E;
  const double scale = pow2(sum_bits(row.V));
  uint32_t n;
  const uint64_t s = held_weight(S, row, 0, cut, a, top, scale, n);
  const uint32_t n_kept = P.out_kept ? block_sum(S, n) : 0;
  uint64_t thr = 0;
  int at;
  const uint64_t sum = find_sum(S, s, true, P.uniforms[r], thr, at);
  __syncthreads();
  int64_t token = draw_among(S, row, cut, a.c, top, scale, (int64_t)at * E,
                             min(E, row.V - at * E), thr);
  token = draw_past_units(S, mem, cut, a.c, top, scale, zmax, token, P.uniforms[r], sum);
  drawn_token(P, r, token, row.at(token), a, top, (double)sum / scale, n_kept);
}
template <int DT>
__device__ __forceinline__ void draw(Shared& S, const TruncParams& P, int64_t r,
                                     const ScanRow<DT>& row, const ScanRow<DT>&, const Cut& cut,
                                     const Ask& a, double top, float zmax) {
  const double scale = pow2(sum_bits(row.V));
  const int64_t q = ((int64_t)row.V + kNT - 1) / kNT, e0 = (int64_t)threadIdx.x * q;
  uint32_t n = 0;
  uint64_t s = 0;
  for (int64_t e = e0; e < min(e0 + q, (int64_t)row.V); ++e) {
    const float z = row.at(e);
    if (kept(cut, z, e)) {
      s += weight(S, z, a.c, top, scale);
      ++n;
    }
  }
  const uint32_t n_kept = P.out_kept ? block_sum(S, n) : 0;
  uint64_t thr = 0;
  int at;
  const uint64_t sum = find_sum(S, s, true, P.uniforms[r], thr, at);
  __syncthreads();
  int64_t token = draw_among(S, row, cut, a.c, top, scale, (int64_t)at * q,
                             min(q, row.V - (int64_t)at * q), thr);
  token = draw_past_units(S, row, cut, a.c, top, scale, zmax, token, P.uniforms[r], sum);
  drawn_token(P, r, token, row.at(token), a, top, (double)sum / scale, n_kept);
}

// The row's entries outside `cut` as -inf, the others as they are (all of
// them with `whole`, none with `none`).
template <int DT, class Row>
__device__ __forceinline__ void write_lane(const Row& row, char* out, int64_t e0,
                                           const uint32_t (&w)[4], int n, const Cut& cut,
                                           bool whole, bool none) {
  constexpr int VW = Elem<DT>::VW;
  uint32_t o[4];
#pragma unroll
  for (int e = 0; e < VW; ++e) {
    const bool k = !none && (whole || kept(cut, Row::raw(w, e), e0 + e));
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
template <int DT, class Row>
__device__ __forceinline__ void write_cut(const Row& row, char* out, const Cut& cut, bool whole,
                                          bool none) {
  constexpr int VW = Elem<DT>::VW;
  for (int i = 0; i < row.loads(); ++i) {
    const int64_t e0 = ((int64_t)i * kNT + threadIdx.x) * VW;
    if (e0 >= row.V) continue;
    uint32_t w[4];
    const int n = row.load(e0, w);
    write_lane<DT>(row, out, e0, w, n, cut, whole, none);
  }
}

// One row by one workgroup.
template <bool PACK, int DT, bool CUT, class Row>
__device__ __forceinline__ void one_row(Shared& S, uint32_t* values, const TruncParams& P, int64_t r,
                                        const Row& row, const ScanRow<DT>& mem, float zmax) {
  const Ask a = ask_of(P, r / P.rows_per_seq);
  fill_edges(S);
  const uint32_t kmax = block_extreme<true>(S, key_of(clean(zmax)));
  zmax = of_key(kmax);
  const bool none = !a.valid || kmax < kKeyLowest;
  const double top = floor((double)zmax * a.c);
  if constexpr (CUT) {
    Cut cut{kLowest, kNoIndex};
    if (!none && !a.greedy) cut = cut_of<PACK, DT>(S, values, row, mem, a, zmax, top);
    __syncthreads();
    write_cut<DT>(row, static_cast<char*>(P.out) + r * P.out_ld * Elem<DT>::EB, cut,
                  a.valid && a.greedy, none);
  } else if (none) {
    no_token(P, r);
  } else if (a.greedy) {
    uint32_t first = 0xffffffffu;
    row.each([&](int64_t e, float z, uint32_t) {
      if (z >= zmax) first = min(first, (uint32_t)e);
    });
    greedy_token(P, r, block_extreme<false>(S, first));
  } else {
    const Cut cut = cut_of<PACK, DT>(S, values, row, mem, a, zmax, top);
    draw(S, P, r, row, mem, cut, a, top, zmax);
  }
}

// A workgroup per row, which it holds in LDS: U lane loads a thread.  One row of
// 1000 entries takes 11.4 us, nearly all of it a chain of some 20 barriers; one of
// 32 128 float32 entries 29 us, of which 1.6 are the loads, 6 the bins, 5 finding the
// entries in question and 6 the weights and the draw.
template <int DT, int U, bool CUT>
__global__ void __launch_bounds__(kNT) k_trunc_held(TruncParams P) {
  constexpr int VW = Elem<DT>::VW;
  __shared__ Shared S;
  __shared__ w4 held[U * kNT];
  __shared__ uint32_t values[DT == 1 ? kValues : 1];
  const int64_t r = blockIdx.x;
  const char* src = static_cast<const char*>(P.z) + r * P.ld * Elem<DT>::EB;
  constexpr uint32_t kPad = DT == 1 ? 0xff80ff80u : 0xff800000u;
  float zmax = -__builtin_huge_valf();
  uint32_t w[U][4];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int e0 = (i * kNT + (int)threadIdx.x) * VW;
#pragma unroll
    for (int j = 0; j < 4; ++j) w[i][j] = kPad;
    if (e0 < P.V) load_lane<DT>(src, e0, P.V, w[i]);
  }
#pragma unroll
  for (int i = 0; i < U; ++i) {
#pragma unroll
    for (int e = 0; e < VW; ++e) zmax = fmaxf(zmax, RowOf<DT>::raw(w[i], e));
    held[i * kNT + threadIdx.x] = w4{w[i][0], w[i][1], w[i][2], w[i][3]};
  }
  one_row<true, DT, CUT>(S, values, P, r, HeldRow<DT, U>(held, P.V), ScanRow<DT>(src, P.V), zmax);
}

// ------------------------------------------------------------------ long rows
// Rows of more than kTruncHeld entries are cut into slices, a workgroup to each, in
// four launches: the slices' bins; the row's plan from them; the slices again,
// for what is kept for sure and the entries in question; and the row's end.
// What bounds them: 32 rows of 256 000 bfloat16 entries, 9.6 + 11 + 18 + 19 us,
// are mostly the chains of barriers of the plan and the end, one workgroup a row;
// of 256 rows to be cut (45 + 12 + 64 + 15 us) the first reads 131 MB at 2.9
// TB/s, bound by the counting, and the third reads and writes them at 4.1 TB/s.
// Slices of four lane loads a thread: with two the 256 rows take 57 + 17 + 71 +
// 15 us, with one 84 + 27 + 84 + 15 (a slice writes 8 KiB of bins, and its
// workgroup's start and end stay the same).
constexpr int kSliceLoads = 4;

// Bins of a slice, relative to the slice's own maximum: bins lie on one grid
// for the whole row, so that a row's bins are sums of its slices'.
template <int DT, int U>
__global__ void __launch_bounds__(kNT) k_slice_bins(TruncParams P) {
  constexpr int VW = Elem<DT>::VW;
  constexpr int64_t N = (int64_t)kNT * U * VW;
  __shared__ uint64_t bins[kBins];
  __shared__ uint32_t values[DT == 1 ? kValues : 1], wave32[kNW];
  const int s = blockIdx.x;
  const int64_t r = blockIdx.y;
  const char* src = static_cast<const char*>(P.z) + r * P.ld * Elem<DT>::EB;
  constexpr uint32_t kPad = DT == 1 ? 0xff80ff80u : 0xff800000u;
  uint32_t w[U][4];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int64_t e0 = s * N + (i * kNT + (int)threadIdx.x) * VW;
#pragma unroll
    for (int j = 0; j < 4; ++j) w[i][j] = kPad;
    if (e0 < P.V) load_lane<DT>(src, e0, P.V, w[i]);
  }
  bins[threadIdx.x] = 0;
  if constexpr (DT == 1)
    for (uint32_t i = threadIdx.x; i < kValues; i += kNT) values[i] = 0;
  float zmax = -__builtin_huge_valf();
#pragma unroll
  for (int i = 0; i < U; ++i)
#pragma unroll
    for (int e = 0; e < VW; ++e) zmax = fmaxf(zmax, RowOf<DT>::raw(w[i], e));
  const uint32_t kmax = block_max(wave32, key_of(clean(zmax)));
  zmax = of_key(kmax);
  if (threadIdx.x == 0) P.slice_max[r * P.slices + s] = zmax;
  const Ask a = ask_of(P, r / P.rows_per_seq);
  if (!a.valid || a.greedy || kmax < kKeyLowest || (!(a.k > 0 && a.k < P.V) && a.p >= 1.0f)) return;
  const double top = floor((double)zmax * a.c);
#pragma unroll
  for (int i = 0; i < U; ++i)
#pragma unroll
    for (int e = 0; e < VW; ++e) {
      if constexpr (DT == 1) add_value(bins, values, RowOf<DT>::bits(w[i], e), a.c, top);
      else add_packed(bins, RowOf<DT>::raw(w[i], e), a.c, top);
    }
  __syncthreads();
  if constexpr (DT == 1) {
    add_values(bins, values, a.c, top);
    __syncthreads();
  }
  P.slice_bins[(r * P.slices + s) * kBins + threadIdx.x] = bins[threadIdx.x];
}

enum RowMode : int32_t { kRowNone, kRowGreedy, kRowCut, kRowScan };
struct RowPlan {
  int32_t mode;
  float zmax, floor_z, sure_z;  // min-p's cut; entries not below sure_z are kept
  double top;
  Plan plan;
  Question q;
  uint32_t n_items, first;      // entries put into the list; the argmax (greedy rows)
};

__global__ void __launch_bounds__(kNT) k_slice_plan(TruncParams P) {
  __shared__ Shared S;
  const int64_t r = blockIdx.x;
  const float* maxima = P.slice_max + r * P.slices;
  float zmax = -__builtin_huge_valf();
  for (int s = (int)threadIdx.x; s < P.slices; s += kNT) zmax = fmaxf(zmax, maxima[s]);
  fill_edges(S);
  const uint32_t kmax = block_extreme<true>(S, key_of(zmax));
  zmax = of_key(kmax);
  const Ask a = ask_of(P, r / P.rows_per_seq);
  RowPlan R{};
  R.mode = !a.valid || kmax < kKeyLowest ? kRowNone : a.greedy ? kRowGreedy : kRowCut;
  R.zmax = zmax;
  R.first = 0xffffffffu;
  R.plan.kbin = R.plan.plo = -1;
  if (R.mode == kRowCut) {
    R.top = floor((double)zmax * a.c);
    const Cut floor_cut = min_p_cut(a, zmax);
    R.sure_z = R.floor_z = floor_cut.z;
    if ((a.k > 0 && a.k < P.V) || a.p < 1.0f) {
      const uint64_t* bins = P.slice_bins + r * P.slices * kBins;
      const int i = (int)threadIdx.x;
      uint32_t n = 0, rest = 0;
      uint64_t m = 0;
      // kNT slices' shifts at a time (in S.cnt), then their bins
      for (int s0 = 0; s0 < P.slices; s0 += kNT) {
        const int ns = min(P.slices - s0, kNT);
        __syncthreads();
        if (i < ns) {
          const float zs = maxima[s0 + i];  // (a slice of nothing: nowhere)
          S.cnt[i] = zs < kLowest ? (uint32_t)kBins
                                  : min((uint32_t)(int)(R.top - floor((double)zs * a.c)),
                                        (uint32_t)(kBins - 1));
        }
        __syncthreads();
#pragma unroll 8
        for (int s = 0; s < ns; ++s) {
          const int shift = (int)S.cnt[s];
          const uint64_t* b = bins + (int64_t)(s0 + s) * kBins;
          const uint64_t x = b[max(i - shift, 0)], y = b[i];
          if (i >= shift && i < kBins - 1) {
            n += (uint32_t)(x >> 48);
            m += x & ((1ull << 48) - 1);
          }
          // the row's last bin takes all that the shift moves there
          if (shift < kBins && i + shift >= kBins - 1) rest += (uint32_t)(y >> 48);
        }
      }
      rest = block_sum(S, rest);
      if (i == kBins - 1) n = rest;
      const double mass = i == kBins - 1 ? 0.0 : ((double)n + (double)m * kUnit) * S.edge[i];
      R.plan = make_plan(S, a, P.V, n, mass, cut_bin(a, floor_cut, R.top));
      R.q = question_of(R.plan, R.top, a.c);
      if (R.plan.items > (uint32_t)P.items_max) R.mode = kRowScan;
      if (R.plan.plo >= 0 || R.plan.kbin >= 0) {
        const float hi = R.plan.plo >= 0 ? R.q.p.hi : R.q.k.hi;
        R.sure_z = hi == hi ? fmaxf(R.floor_z, hi) : __builtin_huge_valf();  // (inf: none)
      }
    }
  }
  if (threadIdx.x == 0) reinterpret_cast<RowPlan*>(P.row_plan)[r] = R;
}

template <int DT, int U, bool CUT>
__global__ void __launch_bounds__(kNT) k_slice_keep(TruncParams P) {
  constexpr int VW = Elem<DT>::VW;
  constexpr int64_t N = (int64_t)kNT * U * VW;
  __shared__ Shared S;
  __shared__ w4 held[U * kNT];
  const int s = blockIdx.x;
  const int64_t r = blockIdx.y;
  RowPlan* plan = reinterpret_cast<RowPlan*>(P.row_plan) + r;
  const int mode = plan->mode;
  if (mode == kRowScan || (!CUT && mode == kRowNone)) return;
  const char* src = static_cast<const char*>(P.z) + r * P.ld * Elem<DT>::EB;
  constexpr uint32_t kPad = DT == 1 ? 0xff80ff80u : 0xff800000u;
  const Ask a = ask_of(P, r / P.rows_per_seq);
  if (!CUT) fill_edges(S);
  const float sure_z = plan->sure_z;
  const Cut sure{sure_z, sure_z <= -kLowest ? kNoIndex : -1};
  const Question q = plan->q;
  const bool ask = plan->plan.kbin >= 0 || plan->plan.plo >= 0;
  char* out = CUT ? static_cast<char*>(P.out) + r * P.out_ld * Elem<DT>::EB : nullptr;
  const ScanRow<DT> row(src, P.V);
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int64_t e0 = s * N + (i * kNT + (int)threadIdx.x) * VW;
    uint32_t w[4] = {kPad, kPad, kPad, kPad};
    if (e0 < P.V) {
      const int n = load_lane<DT>(src, e0, P.V, w);
      if (CUT) write_lane<DT>(row, out, e0, w, n, sure, mode == kRowGreedy, mode == kRowNone);
    }
    held[i * kNT + threadIdx.x] = w4{w[0], w[1], w[2], w[3]};
  }
  __syncthreads();
  const int left = (int)min(N, P.V - s * N);
  const HeldRow<DT, U> mine(held, left);
  if (mode == kRowCut && ask) {
    // the entries in question, to the row's list
    Item* list = reinterpret_cast<Item*>(P.items) + r * P.items_max;
    mine.each([&](int64_t e, float z, uint32_t bits) {
      if (asked(q, z)) {
        const uint32_t at = atomicAdd(&plan->n_items, 1u);
        if (at < (uint32_t)P.items_max) list[at] = Item{bits, (int32_t)(s * N + e)};
      }
    });
  }
  if constexpr (!CUT) {
    if (mode == kRowGreedy) {
      mine.each([&](int64_t e, float z, uint32_t) {
        if (z >= plan->zmax) atomicMin(&plan->first, (uint32_t)(s * N + e));
      });
      return;
    }
    uint32_t n;
    uint64_t x = held_weight(S, mine, s * N, sure, a, plan->top, pow2(sum_bits(P.V)), n);
    x = wave_incl_scan(x);
    if ((threadIdx.x & 63) == 63)
      P.sub_weight[(r * P.slices + s) * kNW + (threadIdx.x >> 6)] = x;
    n = block_sum(S, n);
    if (threadIdx.x == 0) P.slice_kept[r * P.slices + s] = n;
  }
}

template <int DT, bool CUT>
__global__ void __launch_bounds__(kNT) k_slice_end(TruncParams P, int sub) {
  __shared__ Shared S;
  const int64_t r = blockIdx.x;
  const RowPlan R = reinterpret_cast<const RowPlan*>(P.row_plan)[r];
  const ScanRow<DT> row(static_cast<const char*>(P.z) + r * P.ld * Elem<DT>::EB, P.V);
  if (R.mode == kRowScan) {
    one_row<false, DT, CUT>(S, nullptr, P, r, row, row, R.zmax);
    return;
  }
  if (R.mode == kRowNone) {
    if (!CUT) no_token(P, r);
    return;
  }
  if (R.mode == kRowGreedy) {
    if (!CUT) greedy_token(P, r, R.first);
    return;
  }
  const Ask a = ask_of(P, r / P.rows_per_seq);
  const bool ask = R.plan.kbin >= 0 || R.plan.plo >= 0;
  if (CUT && !ask) return;
  fill_edges(S);
  const Item* list = reinterpret_cast<const Item*>(P.items) + r * P.items_max;
  const int n_items = ask ? (int)R.plan.items : 0;
  Cut cut{R.floor_z, kNoIndex};
  if (ask) {
    if (n_items <= kItems) {
      if ((int)threadIdx.x < n_items) S.items[threadIdx.x] = list[threadIdx.x];
      __syncthreads();
      cut = tighter(cut, n_items <= kRanked
                             ? resolve_ranked<DT>(S, a, R.top, R.plan, n_items)
                             : resolve(S, ItemRow<DT>(S.items, P.V, n_items), a, R.top, R.plan));
    } else {
      __syncthreads();
      cut = tighter(cut, resolve(S, ItemRow<DT>(list, P.V, n_items), a, R.top, R.plan));
    }
  }
  if constexpr (CUT) {
    char* out = static_cast<char*>(P.out) + r * P.out_ld * Elem<DT>::EB;
    for (int i = (int)threadIdx.x; i < n_items; i += kNT) {
      const Item x = list[i];
      if (!kept(cut, RowOf<DT>::of_bits(x.bits), x.idx)) continue;
      if constexpr (DT == 1) reinterpret_cast<uint16_t*>(out)[x.idx] = (uint16_t)x.bits;
      else reinterpret_cast<uint32_t*>(out)[x.idx] = x.bits;
    }
  } else {
    // weights by groups of G sub-chunks of `sub` entries
    const double scale = pow2(sum_bits(P.V));
    const int64_t subs = ((int64_t)P.V + sub - 1) / sub, G = (subs + kNT - 1) / kNT;
    const uint64_t* weights = P.sub_weight + r * P.slices * kNW;
    uint64_t own = 0;
    for (int64_t g = threadIdx.x * G; g < min((threadIdx.x + 1) * G, subs); ++g) own += weights[g];
    uint32_t n = 0;
    for (int i = (int)threadIdx.x; i < P.slices; i += kNT) n += P.slice_kept[r * P.slices + i];
    __syncthreads();
    S.mass[threadIdx.x] = own;
    __syncthreads();
    for (int i = (int)threadIdx.x; i < n_items; i += kNT) {
      const Item x = list[i];
      const float z = RowOf<DT>::of_bits(x.bits);
      if (!kept(cut, z, x.idx)) continue;
      ++n;
      atomicAdd((unsigned long long*)&S.mass[x.idx / (sub * G)],
                (unsigned long long)weight(S, z, a.c, R.top, scale));
    }
    n = block_sum(S, n);
    uint64_t thr = 0;
    int at;
    const uint64_t sum = find_sum(S, S.mass[threadIdx.x], true, P.uniforms[r], thr, at);
    __syncthreads();
    const int64_t lo = (int64_t)at * G * sub;
    int64_t token = draw_among(S, row, cut, a.c, R.top, scale, lo, min(G * sub, P.V - lo), thr);
    token = draw_past_units(S, row, cut, a.c, R.top, scale, R.zmax, token, P.uniforms[r], sum);
    drawn_token(P, r, token, row.at(token), a, R.top, (double)sum / scale, n);
  }
}

template <int DT, int U, bool CUT>
void launch_slices(const TruncParams& P, hipStream_t stream) {
  const dim3 grid((uint32_t)P.slices, (uint32_t)P.R), rows((uint32_t)P.R), block(kNT);
  k_slice_bins<DT, U><<<grid, block, 0, stream>>>(P);
  k_slice_plan<<<rows, block, 0, stream>>>(P);
  k_slice_keep<DT, U, CUT><<<grid, block, 0, stream>>>(P);
  k_slice_end<DT, CUT><<<rows, block, 0, stream>>>(P, 64 * U * Elem<DT>::VW);
}

template <int DT, bool CUT>
void launch_rows(const TruncParams& P, hipStream_t stream) {
  constexpr int N = kNT * Elem<DT>::VW;  // entries of a lane load of a workgroup
  const dim3 grid((uint32_t)P.R), block(kNT);
  if (P.slices) {
    launch_slices<DT, kSliceLoads, CUT>(P, stream);
  } else if (P.V <= N) k_trunc_held<DT, 1, CUT><<<grid, block, 0, stream>>>(P);
  else if (P.V <= 2 * N) k_trunc_held<DT, 2, CUT><<<grid, block, 0, stream>>>(P);
  else if (P.V <= 4 * N) k_trunc_held<DT, 4, CUT><<<grid, block, 0, stream>>>(P);
  else if constexpr (DT == 0) k_trunc_held<DT, 8, CUT><<<grid, block, 0, stream>>>(P);
}

}  // namespace

int trunc_slice_elems(int dtype) { return kNT * kSliceLoads * (dtype == SPC_BF16 ? 8 : 4); }
size_t trunc_plan_bytes() { return sizeof(RowPlan); }
size_t trunc_item_bytes() { return sizeof(Item); }

// (P.R at most kMaxRows)
hipError_t launch_truncated(const TruncParams& P, int dtype, hipStream_t stream) {
  if (dtype == SPC_BF16) {
    if (P.out) launch_rows<1, true>(P, stream);
    else launch_rows<1, false>(P, stream);
  } else {
    if (P.out) launch_rows<0, true>(P, stream);
    else launch_rows<0, false>(P, stream);
  }
  return hipGetLastError();
}

}  // namespace spc
