// Tokens drawn from logits under temperature, top-k, top-p and min-p by given
// random numbers (asr_sample).
//
// The kept tokens are a prefix of the falling order, so they are those up to a cut: a
// logit and, among the tokens that have it, the last that is kept.  Nothing is sorted.
// A block of 1024 threads takes a row, each wave a sixteenth of it, which comes from L2
// again at each pass.  After the largest logit M (and each thread's):
//
// float32 logits, bf16 ones with a small top-k or up to 16384 tokens:
//   1. a bin that the cut cannot lie behind: bins are the leading bits of M - l (256 to an
//      octave), filled with counts for top-k (up to 768 wanted tokens: of the threads'
//      largest alone) or, for top-p, with the float32 weights of the threads' largest and
//      of every fourth or eighth other token.  The latter is a guess that 2. checks;
//   2. the tokens up to that bin, in the order of tokens, into lists of the waves in LDS,
//      and the weights of all; the cuts are found by finer bins of the lists, the draws
//      by the lists' sums.
//   Where a wave's list would be longer than 512 tokens, counts or weights of the whole
//   row are filled into bins for each cut in turn, only the cut's own bin is listed, and
//   draws go by sums over segments of 4 loads of a wave.
// more bf16 logits, with top-k above 768 or top-p: tokens are counted by value, in LDS; counts times
//   weights give the sums and the cuts, one pass over the tokens the segments' sums, each
//   value's weight looked up.
//
// Weights are whole numbers, so sums do not depend on an order: 2^(i / 512) from a table
// times a polynomial, in 64 bits.  Bound by instructions (a weight takes 22, 13 of them on
// doubles: some 0.2 ns a token of a row) and by the fetch of code that runs once, some 0.1 us
// for 64 bytes, hence loops where they cost nothing.  A row of 51865 under top-p
// takes 24 to 39 us by what it keeps (max 4, guess 5, list and weights 16, cut 4 on the way; 62
// where the lists cannot hold it), 128 rows under all filters 32, 256 bf16 rows of 131071 with 5
// draws 75 (max 12, counts 14, their weights and cuts 18, segments 17, draws 7); sorting each row
// took 302, 1453, 3805.
#include <algorithm>

#include "asr_device.h"

namespace asr {
namespace {

constexpr int SM_NT = 1024, SM_NW = SM_NT / 64;
constexpr int SM_BINS = 8192, SM_FINE = 2048, SM_TAB = 512;
constexpr int SM_LIST = 512, SM_NARROW = 256;      // of a wave: all tokens up to a bin, those of one bin
constexpr int SM_U = 4;                            // loads under way, and in a segment
constexpr int SM_FEW = 768;                        // wanted tokens that the threads' largest may bound
constexpr int SM_VALUES = 16384;                   // bf16 tokens above which values are counted
constexpr int SM_MEMBERS = 64;

#define SM_INLINE __attribute__((always_inline))

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef uint16_t u16x8u __attribute__((ext_vector_type(8), aligned(2)));

// A lane's tokens of one load: 16 bytes.
template <typename T>
constexpr int kPer = 16 / sizeof(T);

// A wave's part of a row: `steps` times 64 lanes' loads from token `first` on.
template <typename T>
struct RowOf {
  static constexpr int E = kPer<T>;
  const T* p;
  int V, steps, first;

  __device__ __forceinline__ uint4 fetch(int base) const {
    if (base + E <= V) {
      if constexpr (sizeof(T) == 4)
        return __builtin_bit_cast(uint4, *(const f32x4u*)(p + base));
      else
        return __builtin_bit_cast(uint4, *(const u16x8u*)(p + base));
    }
    uint4 u;                                               // -inf past the end
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 4; ++i) ((float*)&u)[i] = base + i < V ? p[base + i] : -INFINITY;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) ((uint16_t*)&u)[i] = base + i < V ? p[base + i] : (uint16_t)0xff80u;
    }
    return u;
  }
  static __device__ __forceinline__ void floats(const uint4& u, float* x) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 4) {
        x[i] = __uint_as_float(w[i]);
      } else {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      }
    }
  }
  __device__ __forceinline__ int base(int step) const { return first + (step * 64 + (int)(threadIdx.x & 63)) * E; }
  // f(first token, 16 bytes) over the wave's part; after(segment) behind each SM_U steps.
  // U loads at once; 1: one ahead, in the least code, where f is long.
  template <int U, class F, class G>
  __device__ SM_INLINE void raw(F&& f, G&& after) const {
    const int seg = (int)(threadIdx.x >> 6) * ((steps + SM_U - 1) / SM_U);
    if constexpr (U == 1) {
      uint4 next = fetch(base(0));
#pragma unroll 1
      for (int i = 0; i < steps; ++i) {
        const uint4 u = next;
        next = fetch(base(i + 1));
        f(base(i), u);
        if (i % SM_U == SM_U - 1 || i == steps - 1) after(seg + i / SM_U);
      }
    } else {
      static_assert(U == SM_U, "");
#pragma unroll 1
      for (int i = 0; i < steps; i += SM_U) {
        uint4 u[SM_U];
#pragma unroll
        for (int j = 0; j < SM_U; ++j) u[j] = fetch(base(i + j));
#pragma unroll
        for (int j = 0; j < SM_U; ++j)
          if (i + j < steps) f(base(i + j), u[j]);
        after(seg + i / SM_U);
      }
    }
  }
  // f(first token, x)
  template <int U, class F, class G>
  __device__ SM_INLINE void each(F&& f, G&& after) const {
    raw<U>(
        [&](int base, const uint4& u) SM_INLINE {
          float x[E];
          floats(u, x);
          f(base, x);
        },
        after);
  }
  template <int U, class F>
  __device__ SM_INLINE void each(F&& f) const {
    each<U>(f, [](int) SM_INLINE {});
  }
  __device__ __forceinline__ int segments() const { return SM_NW * ((steps + SM_U - 1) / SM_U); }
  // the first token of a segment's step for this lane; steps of the segment
  __device__ __forceinline__ int segment_steps(int seg) const {
    return min(steps - seg % ((steps + SM_U - 1) / SM_U) * SM_U, SM_U);
  }
  __device__ __forceinline__ int segment_base(int seg, int step) const {
    const int per = (steps + SM_U - 1) / SM_U;
    return ((seg / per * steps + seg % per * SM_U + step) * 64 + (int)(threadIdx.x & 63)) * E;
  }
};

// e^{(l - M) / T} in whole units of 2^-unit.
struct Weights {
  const double* tab;       // 2^(unit + i / 512)
  int unit;
  double top, c;           // 512 log2(e) / T
  double least;            // place of 2^-60 units: what weighs less counts as that, nothing in every sum
  __device__ __forceinline__ double place(float l) const { return ((double)l - top) * c; }
  __device__ __forceinline__ double weight(float l) const { return power(fmax(place(l), least)); }   // (0 times -inf, too)
  // 2^(unit + y / 512)
  __device__ __forceinline__ double power(double y) const {
    constexpr double kMagic = 6755399441055744.0;          // 1.5 * 2^52: the nearest whole number is in the low bits
    const double t = y + kMagic;
    const int k = __double2loint(t);
    const double r = y - (t - kMagic);
    constexpr double a1 = 6.93147180559945286e-01 / 512, a2 = a1 * a1 / 2, a3 = a1 * a1 * a1 / 6;   // (the next term: 9e-15)
    const double e = tab[k & (SM_TAB - 1)];
    const double v = fma(fma(fma(a3, r, a2), r, a1), r * e, e);
    // times 2^(k / 512), in the exponent
    return __hiloint2double(__double2hiint(v) + (int)((uint32_t)(k & ~(SM_TAB - 1)) << 11), __double2loint(v));
  }
  // log2(x), x > 0: the float instruction's, and what its power leaves of x
  __device__ __forceinline__ double log2_of(double x) const {
    int exponent;
    const double f = 2.0 * frexp(x, &exponent);
    const double near = (double)__builtin_amdgcn_logf((float)f);
    const double rest = fma(f, ldexp(power(near * -(double)SM_TAB), -unit), -1.0);      // (below 2^-22: the cube is nothing)
    return exponent - 1 + near + fma(-0.5 * rest, rest, rest) * 1.4426950408889634074;
  }
  // 2^52 leaves the whole number in the low bits
  static __device__ __forceinline__ uint64_t rounded(double weight) {
    return (uint64_t)__double_as_longlong(weight + 4503599627370496.0) & 0xfffffffffffffull;
  }
  __device__ __forceinline__ uint64_t whole(float l) const { return rounded(weight(l)); }
};

// Kept: logits above `l`, and of those at it tokens up to `last`.
struct Cut {
  float l;
  int last;
  __device__ __forceinline__ bool keeps(float x, int token) const { return x > l || (x == l && token <= last); }
};
// Rises as logits fall; zeros of either sign are one logit.
__device__ __forceinline__ uint32_t falling(float l) { return ~ordered_u32(l + 0.f); }
__device__ __forceinline__ float of_falling(uint32_t k) { return from_ordered_u32(~k); }

// Bins of M - l: 0 below 2^-12, 256 to each octave, the last from 2^20 on.
constexpr int SM_SHIFT = 15, SM_BIN0 = (127 - 12) << (23 - SM_SHIFT);
static_assert(SM_BINS == 32 << (23 - SM_SHIFT), "32 octaves");
__device__ __forceinline__ uint32_t depth(float top, float l) { return __float_as_uint(top - l); }
__device__ __forceinline__ int bin_of(uint32_t depth) { return min(max((int)(depth >> SM_SHIFT) - SM_BIN0, 0), SM_BINS - 1); }
__device__ __forceinline__ uint32_t bin_begin(int b) { return b <= 0 ? 0u : (uint32_t)(b + SM_BIN0) << SM_SHIFT; }
__device__ __forceinline__ uint32_t bin_end(int b) { return b >= SM_BINS - 1 ? 0xffffffffu : (uint32_t)(b + 1 + SM_BIN0) << SM_SHIFT; }

struct Lds {
  double tab[SM_TAB];
  union {
    uint64_t bins[SM_BINS];
    struct {
      float logit[SM_NW][SM_LIST];
      int32_t token[SM_NW][SM_LIST];
    } list;
  };
  union {
    uint32_t counts[SM_BINS];
    struct {
      uint64_t fine[SM_FINE];
      uint32_t fine_n[SM_FINE];
    };
    uint64_t seg[SM_NT];
  };
  struct {
    float logit[SM_NW][SM_NARROW];
    int32_t token[SM_NW][SM_NARROW];
  } narrow;
  uint64_t sums[2][SM_NW];
  uint64_t found_before, found_in, found_other;
  uint32_t found, members, members2;
  float tops[SM_NW], lows[SM_NW];
  float member_logit[SM_MEMBERS];
  int32_t member_token[SM_MEMBERS];
  int32_t first, bad, token;
};
static_assert(kRulesMaxVocab <= SM_NT * SM_U * 64 * 4, "a segment a thread");

// bf16 logits by their values: SV_N values from the row's largest down (where that is below 4,
// 17279 or more of them negative ones: to -256, which is not one of them), the last for all behind.
constexpr int SV_N = 33 * SM_NT, SV_IDS = 2048;
struct ValuesLds {
  double tab[SM_TAB];
  uint32_t hist[SV_N];                     // tokens of a value, then where its weight is, in bytes
  union {
    uint64_t weight[SV_IDS + 1];           // the last: 0
    struct {
      uint64_t mass[SV_N / 64];
      uint32_t n[SV_N / 64];
    } part;                                // of 64 values
  };
  uint64_t seg[SM_NT / 2];
  uint32_t ties[SM_NT / 2];                // at the cut's value before a segment
  uint64_t sums[2][SM_NW];
  uint64_t found_before, found_other;
  uint32_t found, ids;
};
static_assert(sizeof(ValuesLds) <= 163840, "the LDS of a CU");
typedef int16_t i16x2 __attribute__((ext_vector_type(2)));
// Of two bf16, numbers that rise as they fall, the zeros' equal; and back.
__device__ __forceinline__ i16x2 falling2(uint32_t u) {
  const i16x2 x = __builtin_bit_cast(i16x2, u), negative = x >> 15;
  return (x ^ ~negative) + (negative | (int16_t)-32768);
}
__device__ __forceinline__ uint32_t falling16(uint32_t b) { return b & 0x8000u ? b - 1 : 0x7fffu - b; }
__device__ __forceinline__ float of_falling16(uint32_t k) { return __uint_as_float((k & 0x8000u ? k + 1 : 0x7fffu - k) << 16); }

// Inclusive sum over the lanes before (data-parallel moves: rows of 16, then their ends).
__device__ __forceinline__ uint64_t wave_scan(uint64_t v) {
#define SM_STEP(ctrl, rows)                                                                          \
  do {                                                                                               \
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, ctrl, rows, 0xf, false);          \
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), ctrl, rows, 0xf, false);  \
    v += (uint64_t)hi << 32 | lo;                                                                    \
  } while (0)
  SM_STEP(0x111, 0xf);                     // row_shr 1, 2, 4, 8
  SM_STEP(0x112, 0xf);
  SM_STEP(0x114, 0xf);
  SM_STEP(0x118, 0xf);
  SM_STEP(0x142, 0xa);                     // row_bcast 15 to rows 1 and 3, 31 to rows 2 and 3
  SM_STEP(0x143, 0xc);
#undef SM_STEP
  return v;
}
// The same of doubles.
__device__ __forceinline__ double wave_sum64(double v) {
#define SM_STEP(ctrl, rows)                                                                          \
  v += __hiloint2double(__builtin_amdgcn_update_dpp(0, __double2hiint(v), ctrl, rows, 0xf, false),   \
                        __builtin_amdgcn_update_dpp(0, __double2loint(v), ctrl, rows, 0xf, false))
  SM_STEP(0x111, 0xf);
  SM_STEP(0x112, 0xf);
  SM_STEP(0x114, 0xf);
  SM_STEP(0x118, 0xf);
  SM_STEP(0x142, 0xa);
  SM_STEP(0x143, 0xc);
#undef SM_STEP
  return v;
}
__device__ __forceinline__ uint64_t lane_value(uint64_t v, int lane) {
  return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), lane) << 32 |
         (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane);
}
// Exclusive sums over the threads; the sum over all in *total.  (Code that runs once is
// bound by its fetch, some 0.1 us for 64 bytes: the waves' sums are joined by a scan too.)
template <class S>
__device__ __forceinline__ uint64_t block_scan(uint64_t v, S& s, uint64_t* total, int which = 0) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint64_t x = wave_scan(v);
  if (which == 0) __syncthreads();
  if (lane == 63) s.sums[which][wave] = x;
  __syncthreads();
  const uint64_t upto = wave_scan(s.sums[which][lane & (SM_NW - 1)]);       // (lanes 0 to 15: of the waves)
  *total = lane_value(upto, SM_NW - 1);
  return (wave ? lane_value(upto, wave - 1) : 0) + x - v;
}
template <class S>
__device__ __forceinline__ void block_scan2(uint64_t a, uint64_t b, S& s, uint64_t* before_a, uint64_t* va, uint64_t* before_b,
                                            uint64_t* vb) {
  *before_a = block_scan(a, s, va);
  *before_b = block_scan(b, s, vb, 1);
}
// The sum of a over the threads, always in the same order; *before and *total of b as above.
template <class S>
__device__ __forceinline__ double block_sum_scan(double a, uint64_t b, S& s, uint64_t* before, uint64_t* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const double x = wave_sum64(a);
  __syncthreads();
  if (lane == 63) s.sums[1][wave] = (uint64_t)__double_as_longlong(x);
  *before = block_scan(b, s, total);       // (its barriers stand for both)
  return __longlong_as_double((long long)lane_value((uint64_t)__double_as_longlong(wave_sum64(__longlong_as_double((long long)s.sums[1][lane & (SM_NW - 1)]))), SM_NW - 1));
}
__device__ __forceinline__ uint64_t block_add(uint64_t v, Lds& s) {
  uint64_t all;
  block_scan(v, s, &all);
  return all;
}

template <int BYTES>
__device__ __forceinline__ void clear(void* p) {
  static_assert(BYTES % (16 * SM_NT) == 0, "");
#pragma unroll
  for (int i = 0; i < BYTES / (16 * SM_NT); ++i) ((uint4*)p)[i * SM_NT + threadIdx.x] = uint4{0, 0, 0, 0};
}
// The bin at which the running sum reaches goal(sum of all), into found, found_before and
// found_in; the sum of all.  The bins are complete behind this function's first barrier.
template <int N, class X, class G>
__device__ __forceinline__ uint64_t find_bin(const X* bins, Lds& s, G&& goal_of) {
  constexpr int P = N / SM_NT;
  const int b = threadIdx.x * P;
  uint64_t x[P], sum = 0, total;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < P; ++i) sum += x[i] = bins[b + i];
  uint64_t before = block_scan(sum, s, &total);
  const uint64_t goal = goal_of(total);
  if (before < goal && goal <= before + sum) {
#pragma unroll
    for (int i = 0; i < P; ++i) {
      if (before < goal && goal <= before + x[i]) s.found = b + i, s.found_before = before, s.found_in = x[i];
      before += x[i];
    }
  }
  __syncthreads();
  return total;
}

// A wave's list, in the order of tokens.
struct List {
  const float* logit;
  const int32_t* token;
  int n;
};

// The last token, in falling order, of those listed and kept by `in` up to which their count or
// their weights reach `goal` (at least 1, at most the whole).
__device__ SM_INLINE Cut cut_list(const List& e, Cut in, bool by_count, uint64_t goal, const Weights& w, Lds& s) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float hi = -INFINITY, lo = INFINITY;
  for (int i = lane; i < e.n; i += 64) {
    const float x = e.logit[i];
    if (in.keeps(x, e.token[i])) hi = fmaxf(hi, x), lo = fminf(lo, x);
  }
  hi = wave_max_lanes(hi);
  lo = -wave_max_lanes(-lo);
  __syncthreads();
  clear<sizeof(s.fine)>(s.fine);
  if (lane == 0) s.tops[wave] = hi, s.lows[wave] = lo;
  if (threadIdx.x == 0) s.members = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < SM_NW; ++i) hi = fmaxf(hi, s.tops[i]), lo = fminf(lo, s.lows[i]);
  uint64_t rest = goal;
  float l = hi;                            // (often all have one logit)
  if (hi != lo) {
    // bins of one width over their range: most often the cut's holds a few tokens
    const float range = hi - lo, by = range > 1e-30f && range < 1e30f ? (SM_FINE - 1) / range : 0.f;
    auto bin = [&](float x) SM_INLINE { return min((int)((hi - x) * by), SM_FINE - 1); };
    for (int i = lane; i < e.n; i += 64) {
      const float x = e.logit[i];
      if (in.keeps(x, e.token[i])) atomicAdd((unsigned long long*)&s.fine[bin(x)], by_count ? 1ull : (unsigned long long)w.whole(x));
    }
    find_bin<SM_FINE>(s.fine, s, [&](uint64_t) SM_INLINE { return goal; });
    const int found = s.found;
    rest -= s.found_before;
    for (int i = lane; i < e.n; i += 64) {
      const float x = e.logit[i];
      if (in.keeps(x, e.token[i]) && bin(x) == found) {
        const uint32_t at = atomicAdd(&s.members, 1u);
        if (at < SM_MEMBERS) s.member_logit[at] = x, s.member_token[at] = e.token[i];
      }
    }
    __syncthreads();
    const int m = s.members;
    if (m <= SM_MEMBERS) {                   // (every wave for itself)
      const float x = lane < m ? s.member_logit[lane] : -INFINITY;
      const int token = lane < m ? s.member_token[lane] : INT32_MAX;
      const uint64_t y = lane >= m ? 0 : by_count ? 1 : w.whole(x);
      uint64_t before = 0;
      for (int j = 0; j < m; ++j) {
        const float o = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), j));
        const int t = __builtin_amdgcn_readlane(token, j);
        before += o > x || (o == x && t < token) ? lane_value(y, j) : 0;
      }
      const int at = __ffsll((unsigned long long)__ballot(before < rest && rest <= before + y)) - 1;
      return {__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), at)), __builtin_amdgcn_readlane(token, at)};
    }
    // many in one bin: by the digits of their logits
    uint32_t prefix = 0;
  #pragma unroll 1
    for (int level = 0; level < 3; ++level) {
      const int shift = level == 0 ? 21 : level == 1 ? 10 : 0, bits = level == 2 ? 10 : 11;
      __syncthreads();
      clear<sizeof(s.fine)>(s.fine);
      __syncthreads();
      for (int i = lane; i < e.n; i += 64) {
        const float x = e.logit[i];
        const uint32_t k = falling(x);
        if (in.keeps(x, e.token[i]) && bin(x) == found && (level == 0 || !((k ^ prefix) >> (shift + bits))))
          atomicAdd((unsigned long long*)&s.fine[k >> shift & ((1 << bits) - 1)], by_count ? 1ull : (unsigned long long)w.whole(x));
      }
      find_bin<SM_FINE>(s.fine, s, [&](uint64_t) SM_INLINE { return rest; });
      prefix |= s.found << shift;
      rest -= s.found_before;
    }
    l = of_falling(prefix);
  }
  // the first of those at the cut's logit
  const uint64_t each = by_count ? 1 : max(w.whole(l), (uint64_t)1), ties = (rest + each - 1) / each;
  const int per = (e.n + 63) / 64, begin = min(lane * per, e.n), end = min(begin + per, e.n);
  uint64_t n = 0, t;
  for (int i = begin; i < end; ++i) n += e.logit[i] == l && in.keeps(l, e.token[i]);
  uint64_t at = block_scan(n, s, &t);
  for (int i = begin; i < end; ++i)
    if (e.logit[i] == l && in.keeps(l, e.token[i]) && ++at == ties) s.token = e.token[i];
  __syncthreads();
  return {l, s.token};
}

template <typename T>
__global__ __launch_bounds__(SM_NT) void k_sample(SampleLaunch a, int unit) {
  extern __shared__ __attribute__((aligned(16))) char sample_lds[];
  Lds& s = *(Lds*)sample_lds;
  constexpr int E = kPer<T>;
  const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  RowOf<T> r;
  r.p = (const T*)a.logits + row * a.ld;
  r.V = a.vocab;
  r.steps = (a.vocab + SM_NT * E - 1) / (SM_NT * E);
  r.first = wave * r.steps * 64 * E;
  const int set = a.set ? a.set[row] : row;
  const bool has = set >= 0 && set < a.sets;
  const float temperature = has && a.temperature ? a.temperature[set] : 1.f;
  const bool greedy = !(temperature > 0.f);
  int32_t top_k = has && a.top_k ? a.top_k[set] : 0;
  const float top_p = has && a.top_p ? a.top_p[set] : 1.f, min_p = has && a.min_p ? a.min_p[set] : 0.f;

  const float uniform = lane < a.draws ? a.u[(int64_t)row * a.draws + lane] : 0.f;

  // the largest logit
  if (tid < SM_TAB) s.tab[tid] = ldexp(exp2((double)tid / SM_TAB), unit);
  if (tid == 0) s.bad = 0, s.first = INT32_MAX;
  clear<sizeof(s.bins)>(s.bins);
  clear<sizeof(s.counts)>(s.counts);
  float mine = -INFINITY;
  bool nan = false;
  r.template each<SM_U>([&](int, const float* x) SM_INLINE {
#pragma unroll
    for (int i = 0; i < E; i += 2) {
      mine = fmaxf(mine, fmaxf(x[i], x[i + 1]));
      nan |= __builtin_isunordered(x[i], x[i + 1]);
    }
  });
  float top = wave_max_lanes(mine);
  if (lane == 0) s.tops[wave] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < SM_NW; ++i) top = fmaxf(top, s.tops[i]);
  top += 0.f;                              // (not -0, from which 0 would be -0 away)
  if (nan || top == INFINITY) s.bad = 1;
  __syncthreads();
  int32_t* token_out = a.token + (int64_t)row * a.draws;
  float* logprob_out = a.logprob ? a.logprob + (int64_t)row * a.draws : nullptr;
  if (s.bad || top == -INFINITY) {
    if (tid < a.draws) {
      token_out[tid] = -1;
      if (logprob_out) logprob_out[tid] = s.bad ? NAN : -INFINITY;
    }
    if (tid == 0 && a.kept) a.kept[row] = 0;
    return;
  }
  constexpr double kScale = 512.0 * 1.4426950408889634074;
  const Weights w = {s.tab, unit, (double)top, kScale / (greedy ? 1.0 : (double)temperature), -512.0 * (unit + 60)};
  double all = 0.0;                        // of all weights, not rounded, once `have_all`
  auto answer = [&](int d, int token, float l) SM_INLINE {
    token_out[d] = token;
    if (logprob_out) logprob_out[d] = (float)((w.place(l) * (1.0 / SM_TAB) - w.log2_of(ldexp(all, -unit))) * 0.69314718055994530942);
  };
  auto goal_of = [&](int d, uint64_t mass) SM_INLINE {
    const float u = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(uniform), d));
    return min((uint64_t)((u > 0.f ? fmin((double)u, 1.0 - 0x1p-24) : 0.0) * (double)mass), mass - 1);
  };

  if (greedy) {
    int at = INT32_MAX;
    double whole_row = 0.0;
    r.template each<1>([&](int base, const float* x) SM_INLINE {
#pragma unroll
      for (int i = E - 1; i >= 0; --i) {
        if (x[i] == top) at = min(at, base + i);
      }
      if (logprob_out) {
#pragma unroll
        for (int i = 0; i < E; ++i) whole_row += w.weight(x[i]);
      }
    });
    if (at < INT32_MAX) atomicMin(&s.first, at);
    uint64_t t0, t1;
    all = block_sum_scan(whole_row, 0, s, &t0, &t1);
    if (tid < a.draws) answer(tid, s.first, top);
    if (tid == 0 && a.kept) a.kept[row] = 1;
    return;
  }
  if (min_p > 1.f) top_k = 1;              // (the first is kept all the same)
  bool k_on = top_k > 0 && top_k < a.vocab;
  const bool p_on = top_p < 1.f;
  auto p_goal = [&](uint64_t mass) SM_INLINE {       // the least whole sum that is not below top_p of the mass
    const double part = (double)top_p * (double)mass;
    return part > 0.0 ? max((uint64_t)ceil(part), (uint64_t)1) : (uint64_t)1;
  };
  auto k_goal = [&](uint64_t) SM_INLINE { return (uint64_t)top_k; };
  Cut cut = {-INFINITY, -1};
  // min-p as a cut: the least logit whose weight is at least min_p
  Cut least = cut;
  if (min_p > 0.f && min_p <= 1.f) {
    const double bound = SM_TAB * w.log2_of((double)min_p);
    auto passes = [&](uint32_t k) SM_INLINE { return w.place(of_falling(k)) >= bound; };
    const uint32_t first = falling(top), end = falling(-INFINITY);
    const uint32_t near = falling((float)fmax(fmin(w.top + bound / w.c, w.top), -3e38));
    uint32_t in = near - first < 16 ? first : near - 16, out = end - near < 16 ? end : near + 16;   // (keys, falling logits)
    if (!passes(in)) in = first;
    if (passes(out)) out = end;
    while (out - in > 1) {
      const uint32_t mid = in + (out - in) / 2;
      if (passes(mid)) in = mid; else out = mid;
    }
    least = {of_falling(in), INT32_MAX};
  }
  auto tighter = [&](Cut x) SM_INLINE { return least.l > x.l ? least : x; };

  // ---- bf16: all that the cut takes is how many tokens have each value
  if constexpr (E == 8) {
    ValuesLds& v = *(ValuesLds*)sample_lds;
    const uint32_t first_key = falling16(__float_as_uint(top) >> 16);
    const i16x2 from = {(int16_t)first_key, (int16_t)first_key};
    const uint32_t none = falling16(0xff80u) - first_key;           // -inf
    // (false: tokens behind the values that are counted matter)
    auto by_values = [&]() SM_INLINE {
      __syncthreads();
      for (int i = tid; i < SV_N / 4; i += SM_NT) ((uint4*)v.hist)[i] = uint4{0, 0, 0, 0};
      if (tid == 0) v.ids = 0;
      __syncthreads();
      auto at2 = [&](uint32_t u) SM_INLINE { return __builtin_bit_cast(uint32_t, falling2(u) - from); };
      r.template raw<SM_U>(
          [&](int, const uint4& u) SM_INLINE {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t k = at2(((const uint32_t*)&u)[i]);
              atomicAdd(&v.hist[min(k & 0xffffu, (uint32_t)SV_N - 1)], 1u);
              atomicAdd(&v.hist[min(k >> 16, (uint32_t)SV_N - 1)], 1u);
            }
          },
          [](int) SM_INLINE {});
      __syncthreads();
      auto count_of = [&](uint32_t b) SM_INLINE { return b == SV_N - 1 || b == none ? 0u : v.hist[b]; };
      auto weight_of = [&](uint32_t b) SM_INLINE { return w.whole(of_falling16(first_key + b)); };
      double row_sum = 0.0;
      // (three at a time, as most hold nothing)
      constexpr int W = 3;
      static_assert(SV_N % (W * SM_NT) == 0, "");
#pragma unroll 1
      for (int i = 0; i < SV_N / SM_NT; i += W) {
        uint32_t c[W], any = 0;
#pragma unroll
        for (int j = 0; j < W; ++j) any |= c[j] = count_of((i + j) * SM_NT + tid);
        const bool some = __any(any != 0);
#pragma unroll 1
        for (int j = i; j < i + W; ++j) {
          uint64_t n = 0, mass = 0;
          if (some) {
            const double y = w.weight(of_falling16(first_key + j * SM_NT + tid));
            n = wave_scan(c[0]);
            mass = wave_scan(c[0] * w.rounded(y));
            row_sum += c[0] ? c[0] * y : 0.0;
          }
          if (lane == 63) v.part.n[j * SM_NW + wave] = (uint32_t)n, v.part.mass[j * SM_NW + wave] = mass;
#pragma unroll
          for (int m = 0; m < W - 1; ++m) c[m] = c[m + 1];
        }
      }
      __syncthreads();
      const bool has_part = tid < SV_N / 64;
      const uint64_t n = has_part ? v.part.n[tid] : 0, mass = has_part ? v.part.mass[tid] : 0;
      uint64_t n_before, n_all, mass_before, mass_all;
      block_scan2(n, mass, v, &n_before, &n_all, &mass_before, &mass_all);
      if (v.hist[SV_N - 1] && (w.place(of_falling16(first_key + SV_N - 1)) >= w.least || (k_on && n_all < (uint64_t)top_k))) return false;
      uint64_t t0, t1;
      all = block_sum_scan(row_sum, 0, v, &t0, &t1);
      uint32_t end = 0, ties = 0;          // kept: values before `end`, and of that one the first `ties` tokens
      uint64_t each = 0, kept_mass = mass_all;
      auto locate = [&](bool by_count, uint64_t goal) SM_INLINE {
        const uint64_t own = by_count ? n : mass, before = by_count ? n_before : mass_before;
        if (before < goal && goal <= before + own) v.found = tid, v.found_before = before, v.found_other = mass_before;
        __syncthreads();
        const uint32_t b = v.found * 64 + lane, c = count_of(b);
        const uint64_t y = weight_of(b), z = by_count ? c : c * y, upto = v.found_before + wave_scan(z);
        const uint64_t weights = v.found_other + wave_scan(c * y) - c * y;
        const int at = __ffsll((unsigned long long)__ballot(upto - z < goal && goal <= upto)) - 1;
        const uint64_t rest = goal - lane_value(upto - z, at);
        const uint32_t there = __builtin_amdgcn_readlane(c, at);
        each = lane_value(y, at);
        end = __builtin_amdgcn_readlane(b, at);
        ties = (uint32_t)(by_count ? rest : (rest + each - 1) / each);
        kept_mass = lane_value(weights, at) + ties * each;
        if (ties == there) ++end, ties = 0;
        __syncthreads();
      };
      const bool k_cuts = k_on && n_all >= (uint64_t)top_k;
#pragma unroll 1
      for (int by = 0; by < 2; ++by)
        if (by == 0 ? k_cuts : p_on) locate(by == 0, by == 0 ? (uint64_t)top_k : p_goal(kept_mass));
      if (!k_cuts && !p_on) end = min(none, (uint32_t)SV_N - 1);   // all
      if (least.l > -INFINITY) {
        const uint32_t u = __float_as_uint(least.l), behind = falling16((u >> 31 ? u : u + 0xffffu) >> 16) - first_key + 1;
        if (behind <= end) end = behind, ties = 0;
      }
      // the kept values' weights, and for every value the place of its weight: the others' is 0
      uint64_t kept_n = 0;
      kept_mass = 0;
      const int kept_steps = ((int)end + SM_NT - 1) / SM_NT;
#pragma unroll 1
      for (int i = 0; i < kept_steps; ++i) {
        const uint32_t b = i * SM_NT + tid, c = b < end ? count_of(b) : 0;
        uint32_t place = SV_IDS;
        if (c) {
          const uint64_t y = weight_of(b);
          place = atomicAdd(&v.ids, 1u);
          if (place < SV_IDS) v.weight[place] = y;
          kept_n += c;
          kept_mass += c * y;
        }
        v.hist[b] = place * 8;
      }
      for (int i = kept_steps * (SM_NT / 4) + tid; i < SV_N / 4; i += SM_NT)
        ((uint4*)v.hist)[i] = uint4{SV_IDS * 8, SV_IDS * 8, SV_IDS * 8, SV_IDS * 8};
      if (tid == 0) v.weight[SV_IDS] = 0;
      uint64_t kept_all, mass_kept;
      block_scan2(kept_n, kept_mass, v, &t0, &kept_all, &t1, &mass_kept);
      mass_kept += ties * each;
      if (tid == 0 && a.kept) a.kept[row] = (int32_t)kept_all + ties;
      // segments' sums
      const bool table = v.ids <= SV_IDS;
      uint64_t part = 0;
      uint32_t equal = 0;
      r.template raw<SM_U>(
          [&](int, const uint4& u) SM_INLINE {
            uint32_t k[E];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t both = at2(((const uint32_t*)&u)[i]);
              k[2 * i] = both & 0xffffu, k[2 * i + 1] = both >> 16;
            }
            if (ties) {
#pragma unroll
              for (int i = 0; i < E; ++i) equal += k[i] == end;
            }
            if (table) {
#pragma unroll
              for (int i = 0; i < E; ++i) k[i] = v.hist[min(k[i], (uint32_t)SV_N - 1)];
#pragma unroll
              for (int i = 0; i < E; ++i) part += *(const uint64_t*)((const char*)v.weight + k[i]);
            } else {
#pragma unroll 1
              for (int i = 0; i < E; ++i) {
                part += k[0] < end ? weight_of(k[0]) : 0;
#pragma unroll
                for (int j = 0; j < E - 1; ++j) k[j] = k[j + 1];
              }
            }
          },
          [&](int seg) SM_INLINE {
            if (__any(part != 0)) part = lane_value(wave_scan(part), 63);
            uint32_t e = 0;
            if (ties && __any(equal)) e = (uint32_t)lane_value(wave_scan(equal), 63);
            if (lane == 0) v.seg[seg] = part, v.ties[seg] = e;
            part = 0, equal = 0;
          });
      __syncthreads();
      const int segments = r.segments();
      const uint64_t own_ties = tid < segments ? v.ties[tid] : 0;
      const uint64_t ties_before = block_scan(own_ties, v, &t0);
      uint64_t own = tid < segments ? v.seg[tid] : 0;
      if (ties_before < ties) own += min(ties - ties_before, own_ties) * each;
      const uint64_t upto = block_scan(own, v, &t0) + own;
      if (tid < segments) v.seg[tid] = upto, v.ties[tid] = (uint32_t)ties_before;
      __syncthreads();
      for (int d = wave; d < a.draws; d += SM_NW) {
        const uint64_t goal = goal_of(d, mass_kept);
        int lo = 0, hi = segments - 1;                             // the first segment whose sum is above goal
        while (lo < hi) {
          const int mid = (lo + hi) / 2;
          if (v.seg[mid] > goal) hi = mid; else lo = mid + 1;
        }
        uint64_t c = lo ? v.seg[lo - 1] : 0;
        uint32_t tied = v.ties[lo];
        const int steps = r.segment_steps(lo);
        uint4 ahead[SM_U];
#pragma unroll
        for (int j = 0; j < SM_U; ++j) ahead[j] = r.fetch(j < steps ? r.segment_base(lo, j) : a.vocab);
#pragma unroll 1
        for (int j = 0; j < steps; ++j) {
          const uint4 u = ahead[0];
#pragma unroll
          for (int m = 0; m < SM_U - 1; ++m) ahead[m] = ahead[m + 1];
          uint64_t z[E], of_lane = 0;
          uint32_t k[E], equal_lane = 0;
          const int base = r.segment_base(lo, j);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t both = at2(((const uint32_t*)&u)[i]);
            k[2 * i] = both & 0xffffu, k[2 * i + 1] = both >> 16;
          }
#pragma unroll
          for (int i = 0; i < E; ++i) equal_lane += k[i] == end;
          const uint32_t scanned_ties = (uint32_t)wave_scan(equal_lane);
          uint32_t nth = tied + scanned_ties - equal_lane;
          tied += __builtin_amdgcn_readlane(scanned_ties, 63);
#pragma unroll
          for (int i = 0; i < E; ++i) {
            z[i] = table ? *(const uint64_t*)((const char*)v.weight + v.hist[min(k[i], (uint32_t)SV_N - 1)]) : k[i] < end ? weight_of(k[i]) : 0;
            if (k[i] == end && nth++ < ties) z[i] = each;
            of_lane += z[i];
          }
          const uint64_t scanned = wave_scan(of_lane);
          uint64_t at = c + scanned - of_lane;
          int chosen = -1;
          uint32_t chosen_key = 0;
#pragma unroll
          for (int i = 0; i < E; ++i) {
            if (at <= goal && goal < at + z[i]) chosen = i, chosen_key = k[i];
            at += z[i];
          }
          c += lane_value(scanned, 63);
          if (chosen >= 0) answer(d, base + chosen, of_falling16(first_key + chosen_key));
        }
      }
      return true;
    };
    // Values take the same time whatever is kept, lists as much as there is before the cut.
    // Lists / values, us, 128 rows of logits with a deviation of 3, of 1.5 and of 0.5:
    //    12001  top-k 2000  23 / 36, 28 / 36, 33 / 31   top-p 0.5  34 / 33, 22 / 36, 42 / 31   0.9  36 / 33, 40 / 37, 33 / 32
    //    24000  top-k 2000  27 / 31, 30 / 34, 37 / 30   top-p 0.5  41 / 32, 28 / 35, 41 / 30   0.9  47 / 32, 39 / 35, 41 / 30
    //    51866  top-k 1000  41 / 43, 40 / 47, 49 / 42   top-p 0.5  31 / 44, 45 / 48, 67 / 43   0.9  40 / 44, 64 / 48, 69 / 43
    //   131071  top-k 1000  78 / 70, 75 / 73, 89 / 69   top-p 0.5  68 / 70, 139 / 75, 141 / 71 0.9  89 / 71, 135 / 75, 146 / 71
    // (the last 256 rows), and top-k 50 and 768 of 51866 28 / 43 and 37 / 43.  Over top-k 769 to
    // half of the tokens, top-p 0.3 to 0.99 and both, lists take 0.63 to 1.02 of the values' time at
    // 8200 tokens (by deviation), 0.81 to 1.18 at 12001, 0.82 to 1.34 at 16000 (1.01 on the whole),
    // 0.99 to 1.45 at 51866.
    if (a.vocab > SM_VALUES && (k_on ? top_k > SM_FEW : p_on)) {
      if (by_values()) return;
      __syncthreads();
      all = 0.0;
      clear<sizeof(s.bins)>(s.bins);
      clear<sizeof(s.counts)>(s.counts);
      __syncthreads();
    }
  }

  // ---- a bin that the cut is not behind: `last`; tokens before it
  int last = -1;
  uint64_t before = 0;
  bool counted = false, have_all = false;
  auto count_bins = [&]() SM_INLINE {                // the bin of top-k's cut; false where there are no more tokens than that
    r.template each<SM_U>([&](int, const float* x) SM_INLINE {
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (x[i] > -INFINITY) atomicAdd(&s.counts[bin_of(depth(top, x[i]))], 1u);
    });
    counted = true;
    if (find_bin<SM_BINS>(s.counts, s, k_goal) <= (uint64_t)top_k) return false;
    last = s.found, before = s.found_before;
    return true;
  };
  bool few = true;                         // the tokens up to it may fit the lists
  if (r.steps * 64 * E <= SM_LIST) {
    last = SM_BINS - 1;
  } else if (k_on) {
    if (top_k <= SM_FEW) {
      if (mine > -INFINITY) atomicAdd(&s.counts[bin_of(depth(top, mine))], 1u);
      if (find_bin<SM_BINS>(s.counts, s, k_goal) >= (uint64_t)top_k) {
        last = s.found;
      } else {
        clear<sizeof(s.counts)>(s.counts);
        __syncthreads();
      }
    }
    if (last < 0) {
      k_on = count_bins();
      few = k_on && before + s.found_in <= SM_NW * SM_LIST * 3 / 4;
    }
  }
  if (last < 0 && p_on) {
    // counts above 43 bits of weights, in units of 2^-22
    constexpr uint64_t kOne = 1ull << 43;
    const float c = (float)fmin(w.c / 512.0, 3e38);
    auto note = [&](float x, int times) SM_INLINE {
      const uint32_t n = (uint32_t)(__builtin_amdgcn_exp2f((x - top) * c) * 0x1p22f + 0.5f);
      if (n) atomicAdd((unsigned long long*)&s.bins[bin_of(depth(top, x))], (unsigned long long)((kOne + n) * times));
    };
    if (mine > -INFINITY) note(mine, 1);
    r.template each<1>([&](int, const float* x) SM_INLINE {
      if (x[0] != mine && x[0] > -INFINITY) note(x[0], E);
    });
    __syncthreads();
    constexpr int P = SM_BINS / SM_NT;
    uint64_t x[P], weights = 0, n = 0, w_before, n_before, w_all, n_all;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      x[i] = s.bins[tid * P + i];
      weights += x[i] & (kOne - 1);
      n += x[i] >> 43;
    }
    if (tid == 0) s.found = SM_BINS - 1, s.found_other = ~0ull;
    block_scan2(weights, n, s, &w_before, &w_all, &n_before, &n_all);
    const uint64_t goal = (uint64_t)((double)w_all * fmax(0.2 + 0.8 * (double)top_p, 0.2));
    if (w_before < goal && goal <= w_before + weights) {
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const uint64_t y = x[i] & (kOne - 1);
        n_before += x[i] >> 43;
        if (w_before < goal && goal <= w_before + y) s.found = tid * P + i, s.found_other = n_before;
        w_before += y;
      }
    }
    __syncthreads();
    last = s.found;
    few = s.found_other <= SM_NW * SM_LIST * 3 / 4;
  } else if (last < 0 && least.l > -INFINITY) {
    last = bin_of(depth(top, least.l));
  }

  // The tokens of bins `from` to `to` that `cut` keeps into the waves' lists of `room`; whether
  // they fit.
  List e;
  uint64_t listed_all;
  float listed_low;
  auto list_bins = [&](int from, int to, float* logit, int32_t* token, int room, bool sum_all) SM_INLINE {
    const uint32_t lo = bin_begin(from), width = bin_end(to) - lo;
    int n = 0;
    double sum = 0.0;                      // (a lane's, in the order of its tokens: always the same)
    float low = INFINITY;
    __syncthreads();
    r.template each<1>([&](int base, const float* x) SM_INLINE {
      uint64_t is[E], any = 0;
#pragma unroll
      for (int i = 0; i < E; ++i) {
        is[i] = __ballot(depth(top, x[i]) - lo < width);
        any |= is[i];
      }
      if (sum_all) {
#pragma unroll
        for (int i = 0; i < E; ++i) sum += w.weight(x[i]);
      }
      if (any) {
        uint32_t at = n;
#pragma unroll
        for (int i = 0; i < E; ++i)
          if (is[i]) {
            is[i] &= __ballot(cut.keeps(x[i], base + i));
            at = __builtin_amdgcn_mbcnt_hi((uint32_t)(is[i] >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)is[i], at));
            n += __popcll(is[i]);
          }
#pragma unroll
        for (int i = 0; i < E; ++i)
          if (is[i]) {
            const bool in = is[i] >> lane & 1;
            low = in ? fminf(low, x[i]) : low;
            if (in && at < (uint32_t)room) logit[at] = x[i], token[at] = base + i;
            at += in;
          }
      }
    });
    e = {logit, token, n};
    low = -wave_max_lanes(-low);
    if (lane == 0) s.lows[wave] = low;
    if (tid == 0) s.members = s.members2 = 0;
    clear<sizeof(s.fine)>(s.fine);
    ((uint2*)s.fine_n)[tid] = uint2{0, 0};
    uint64_t t0, over;
    const double sum_of = block_sum_scan(sum, lane == 0 ? (n > room ? 1ull << 32 : 0) + (uint64_t)n : 0, s, &t0, &over);
    if (sum_all) all = sum_of, have_all = true;
    listed_all = over & 0xffffffffu;
    listed_low = -wave_max_lanes(-s.lows[lane & (SM_NW - 1)]);
    return over >> 32 == 0;
  };

  if (last >= 0 && few && list_bins(0, last, s.list.logit[wave], s.list.token[wave], SM_LIST, logprob_out || (p_on && !k_on))) {
    const int per = (e.n + 63) / 64, begin = min(lane * per, e.n), end = min(begin + per, e.n);
    bool fine = true;
    const bool k_cuts = k_on && listed_all > (uint64_t)top_k;
    if (k_cuts || p_on) {
      // both cuts from the same bins, of one width: most often a cut's holds a few tokens
      const float range = top - listed_low, scale = range > 1e-30f && range < 1e30f ? (SM_FINE - 1) / range : 0.f;
      auto bin = [&](float x) SM_INLINE { return min((int)((top - x) * scale), SM_FINE - 1); };
      for (int i = lane; i < e.n; i += 64) {
        const int b = bin(e.logit[i]);
        atomicAdd((unsigned long long*)&s.fine[b], (unsigned long long)w.whole(e.logit[i]));
        atomicAdd(&s.fine_n[b], 1u);
      }
      __syncthreads();
      const ulonglong2 y = ((const ulonglong2*)s.fine)[tid];
      const uint2 c = ((const uint2*)s.fine_n)[tid];
      uint64_t y_before, mass, c_before, t0;
      block_scan2(y.x + y.y, c.x + c.y, s, &y_before, &mass, &c_before, &t0);
#pragma unroll 1
      for (int by = k_cuts ? 0 : 1; by < (p_on ? 2 : 1); ++by) {
        uint64_t goal = top_k;
        if (by == 1) {
          goal = p_goal(k_on ? mass : (uint64_t)all);
          fine = goal <= mass;             // the guess was far enough
          if (!fine) break;
        }
        const uint64_t before = by ? y_before : c_before, one = by ? y.x : c.x, two = by ? y.y : c.y;
        if (before < goal && goal <= before + one + two) {
          const bool second = before + one < goal;
          s.found = 2 * tid + second, s.found_before = second ? before + one : before, s.found_other = second ? y_before + y.x : y_before;
        }
        __syncthreads();
        const int found = s.found;
        const uint64_t rest = goal - s.found_before, lighter = s.found_other;
        uint32_t* members = by ? &s.members2 : &s.members;
        for (int i = lane; i < e.n; i += 64) {
          const float x = e.logit[i];
          if (bin(x) == found && cut.keeps(x, e.token[i])) {
            const uint32_t at = atomicAdd(members, 1u);
            if (at < SM_MEMBERS) s.member_logit[at] = x, s.member_token[at] = e.token[i];
          }
        }
        __syncthreads();
        const int m = *members;
        if (m > SM_MEMBERS) {
          cut = cut_list(e, cut, by == 0, goal, w, s);
          if (by == 0 && p_on) {
            mass = 0;
            for (int i = begin; i < end; ++i) mass += cut.keeps(e.logit[i], e.token[i]) ? w.whole(e.logit[i]) : 0;
            mass = block_add(mass, s);
          }
          continue;
        }
        // (every wave for itself)
        const float x = lane < m ? s.member_logit[lane] : -INFINITY;
        const int token = lane < m ? s.member_token[lane] : INT32_MAX;
        const uint64_t own = lane < m ? w.whole(x) : 0;
        uint64_t heavier = 0, rank = 0;
        for (int j = 0; j < m; ++j) {
          const float o = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), j));
          const int t = __builtin_amdgcn_readlane(token, j);
          const bool first = o > x || (o == x && t < token);
          heavier += first ? lane_value(own, j) : 0;
          rank += first;
        }
        const bool last_kept = lane < m && (by ? heavier < rest && rest <= heavier + own : rank + 1 == rest);
        const int at = __ffsll((unsigned long long)__ballot(last_kept)) - 1;
        cut = {__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), at)), __builtin_amdgcn_readlane(token, at)};
        if (by == 0) mass = lighter + lane_value(heavier + own, at);
      }
    }
    if (fine) {
      cut = tighter(cut);
      uint64_t sum = 0, n = 0, mass, from, n_before, n_all;
      for (int i = begin; i < end; ++i)
        if (cut.keeps(e.logit[i], e.token[i])) sum += w.whole(e.logit[i]), ++n;
      block_scan2(sum, n, s, &from, &mass, &n_before, &n_all);
      if (tid == 0 && a.kept) a.kept[row] = (int32_t)n_all;
      for (int d = 0; d < a.draws; ++d) {
        const uint64_t goal = goal_of(d, mass);
        if (goal < from || goal >= from + sum) continue;
        uint64_t c = from;
        for (int i = begin; i < end; ++i) {
          const float l = e.logit[i];
          const uint64_t y = cut.keeps(l, e.token[i]) ? w.whole(l) : 0;
          if (c <= goal && goal < c + y) answer(d, e.token[i], l);
          c += y;
        }
      }
      return;
    }
  }

  // ---- many tokens: each cut's bin, then its list
  // (a bin too full for the lists: digits over the row)
  auto cut_row = [&](bool by_count, uint64_t rest) SM_INLINE {
    const Cut in = cut;
    const uint32_t lo = bin_begin(last), width = bin_end(last) - lo;
    uint32_t prefix = 0;
#pragma unroll 1
    for (int level = 0; level < 3; ++level) {
      const int shift = level == 0 ? 21 : level == 1 ? 10 : 0, bits = level == 2 ? 10 : 11;
      __syncthreads();
      clear<sizeof(s.fine)>(s.fine);
      __syncthreads();
      r.template each<1>([&](int base, const float* x) SM_INLINE {
#pragma unroll
        for (int i = 0; i < E; ++i) {
          const uint32_t k = falling(x[i]);
          if (depth(top, x[i]) - lo < width && in.keeps(x[i], base + i) && (level == 0 || !((k ^ prefix) >> (shift + bits))))
            atomicAdd((unsigned long long*)&s.fine[k >> shift & ((1 << bits) - 1)], by_count ? 1ull : (unsigned long long)w.whole(x[i]));
        }
      });
      find_bin<SM_FINE>(s.fine, s, [&](uint64_t) SM_INLINE { return rest; });
      prefix |= s.found << shift;
      rest -= s.found_before;
    }
    const float l = of_falling(prefix);
    const uint64_t each = by_count ? 1 : max(w.whole(l), (uint64_t)1), ties = (rest + each - 1) / each;
    // the last of the kept ones at the cut's logit: its segment, then its step
    __syncthreads();
    uint64_t n = 0, t;
    r.template each<1>(
        [&](int base, const float* x) SM_INLINE {
#pragma unroll
          for (int i = 0; i < E; ++i) n += __popcll(__ballot(x[i] == l && in.keeps(l, base + i)));
        },
        [&](int seg) SM_INLINE {
          if (lane == 0) s.seg[seg] = n;
          n = 0;
        });
    __syncthreads();
    const uint64_t own = tid < r.segments() ? s.seg[tid] : 0, at = block_scan(own, s, &t);
    if (at < ties && ties <= at + own) s.found = tid, s.found_before = at;
    __syncthreads();
    if (wave == 0) {
      uint64_t c = s.found_before;
      const int steps = r.segment_steps(s.found);
      for (int j = 0; j < steps; ++j) {
        float x[E];
        const int base = r.segment_base(s.found, j);
        r.floats(r.fetch(base), x);
        uint32_t mine_at = 0, of_step = 0;
#pragma unroll
        for (int i = 0; i < E; ++i) {
          const uint64_t is = __ballot(x[i] == l && in.keeps(l, base + i));
          mine_at = __builtin_amdgcn_mbcnt_hi((uint32_t)(is >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)is, mine_at));
          of_step += __popcll(is);
        }
#pragma unroll
        for (int i = 0; i < E; ++i)
          if (x[i] == l && in.keeps(l, base + i) && c + ++mine_at == ties) s.token = base + i;
        c += of_step;
      }
    }
    __syncthreads();
    return Cut{l, s.token};
  };
  // weights of what `cut` keeps of bins `from` to `to` into the bins; those of all
  auto weigh = [&](int from, int to, bool sum_all) SM_INLINE {
    const uint32_t lo = bin_begin(from), width = bin_end(to) - lo;
    double sum = 0.0;
    r.template each<1>([&](int base, const float* x) SM_INLINE {
      bool in[E], some = sum_all;
#pragma unroll
      for (int i = 0; i < E; ++i) some |= in[i] = depth(top, x[i]) - lo < width && cut.keeps(x[i], base + i);
      if (!__any(some)) return;
      uint64_t y[E];
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const double z = w.weight(x[i]);
        sum += z;
        y[i] = w.rounded(z);
      }
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (in[i] && y[i]) atomicAdd((unsigned long long*)&s.bins[bin_of(depth(top, x[i]))], (unsigned long long)y[i]);
    });
    uint64_t t0, t1;
    if (sum_all) all = block_sum_scan(sum, 0, s, &t0, &t1), have_all = true;
  };
  if (k_on || p_on) {
    __syncthreads();
    clear<sizeof(s.bins)>(s.bins);
    if (k_on && !counted) {
      clear<sizeof(s.counts)>(s.counts);
      __syncthreads();
      k_on = count_bins();
    }
    __syncthreads();
  }
  const int k_bin = k_on ? last : SM_BINS - 1;
#pragma unroll 1
  for (int by = 0; by < 2; ++by) {
    uint64_t goal = top_k;
    if (!(by == 0 ? k_on : p_on)) continue;
    if (by == 1) {
      weigh(0, k_bin, !have_all && (logprob_out || !k_on));
      find_bin<SM_BINS>(s.bins, s, [&](uint64_t mass) SM_INLINE { return goal = p_goal(mass); });
      last = s.found, before = s.found_before;
    }
    goal -= before;
    const bool fits = list_bins(last, last, s.narrow.logit[wave], s.narrow.token[wave], SM_NARROW, false);
    cut = fits ? cut_list(e, cut, by == 0, goal, w, s) : cut_row(by == 0, goal);
  }
  cut = tighter(cut);
  double sum = 0.0;
  uint64_t n = 0, part = 0;
  const bool sum_all = logprob_out && !have_all;
  __syncthreads();
  r.template each<1>(
      [&](int base, const float* x) SM_INLINE {
        bool in[E], some = sum_all;
#pragma unroll
        for (int i = 0; i < E; ++i) some |= in[i] = cut.keeps(x[i], base + i);
        if (!__any(some)) return;
#pragma unroll
        for (int i = 0; i < E; ++i) {
          const double z = w.weight(x[i]);
          n += in[i];
          sum += z;
          part += in[i] ? w.rounded(z) : 0;
        }
      },
      [&](int seg) SM_INLINE {
        if (__any(part != 0)) part = lane_value(wave_scan(part), 63);
        if (lane == 0) s.seg[seg] = part;
        part = 0;
      });
  uint64_t t0, n_all, mass;
  const double sum_of = block_sum_scan(sum, n, s, &t0, &n_all);
  if (sum_all) all = sum_of;
  if (tid == 0 && a.kept) a.kept[row] = (int32_t)n_all;
  const int segments = r.segments();
  const uint64_t own = tid < segments ? s.seg[tid] : 0, upto = block_scan(own, s, &mass) + own;
  if (tid < segments) s.seg[tid] = upto;
  __syncthreads();
  for (int d = wave; d < a.draws; d += SM_NW) {
    const uint64_t goal = goal_of(d, mass);
    int lo = 0, hi = segments - 1;                             // the first segment whose sum is above goal
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (s.seg[mid] > goal) hi = mid; else lo = mid + 1;
    }
    uint64_t c = lo ? s.seg[lo - 1] : 0;
    const int steps = r.segment_steps(lo);
    uint4 ahead[SM_U];
#pragma unroll
    for (int j = 0; j < SM_U; ++j) ahead[j] = r.fetch(j < steps ? r.segment_base(lo, j) : a.vocab);
#pragma unroll 1
    for (int j = 0; j < steps; ++j) {
      const uint4 u = ahead[0];
#pragma unroll
      for (int m = 0; m < SM_U - 1; ++m) ahead[m] = ahead[m + 1];
      float x[E];
      uint64_t z[E], of_lane = 0;
      const int base = r.segment_base(lo, j);
      r.floats(u, x);
#pragma unroll
      for (int i = 0; i < E; ++i) of_lane += z[i] = cut.keeps(x[i], base + i) ? w.whole(x[i]) : 0;
      const uint64_t scanned = wave_scan(of_lane);
      uint64_t at = c + scanned - of_lane;
#pragma unroll
      for (int i = 0; i < E; ++i) {
        if (at <= goal && goal < at + z[i]) answer(d, base + i, x[i]);
        at += z[i];
      }
      c += lane_value(scanned, 63);
    }
  }
}

template <typename T>
constexpr int kLds = sizeof(T) == 2 ? (int)std::max(sizeof(Lds), sizeof(ValuesLds)) : (int)sizeof(Lds);
template <typename T>
hipError_t launch(const SampleLaunch& a, int unit, hipStream_t s) {
  const hipError_t e = hipFuncSetAttribute((const void*)k_sample<T>, hipFuncAttributeMaxDynamicSharedMemorySize, kLds<T>);
  if (e != hipSuccess) return e;
  k_sample<T><<<dim3((unsigned)a.rows), SM_NT, kLds<T>, s>>>(a, unit);
  return hipSuccess;
}

}  // namespace

hipError_t sample(const SampleLaunch& a, bool bf16, hipStream_t s) {
  int log2 = 0;
  while ((1 << log2) < a.vocab) ++log2;
  const int unit = log2 < 12 ? 50 : 62 - log2;
  return bf16 ? launch<bf16_t>(a, unit, s) : launch<float>(a, unit, s);
}

}  // namespace asr
