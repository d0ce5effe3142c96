// Tokens drawn from logits under temperature, top-k, top-p and min-p by given
// random numbers (asr_sample).
//
// The kept tokens are a prefix of the falling order, so they are those above a cut:
// a logit and, among the tokens that have it, how many of the first.  Nothing is
// sorted.  A block of 1024 threads takes a row, which stays in its XCD's L2 between
// passes:
//   1. the largest logit M, and each thread's;
//   2. a bin that the cut cannot lie behind: bins are the leading bits of M - l (32 to an
//      octave), filled with counts for top-k (few wanted tokens: from the threads'
//      largest alone) or with weights for top-p;
//   3. the tokens up to that bin, in the order of tokens, into a list in LDS: the
//      cuts by the digits of the list's logits, the draws by its sums.
// Where the list would be longer than 4096 the cuts are found by digits over the row
// again, and draws by sums of 64 lanes' tokens.
//
// Weights are whole numbers, so sums do not depend on an order: 2^(i / 512) from a table
// times a polynomial, in 64 bits.
#include "asr_device.h"

namespace asr {
namespace {

constexpr int SM_NT = 1024, SM_NW = SM_NT / 64;
constexpr int SM_BINS = 8192, SM_LIST = 4096, SM_TAB = 512;
constexpr int SM_FEW = 768;              // wanted tokens that the threads' largest may bound

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef uint16_t u16x8u __attribute__((ext_vector_type(8), aligned(2)));

// A lane's tokens of one step: 16 bytes.
template <typename T>
constexpr int kPer = 16 / sizeof(T);

template <typename T>
struct RowOf {
  static constexpr int E = kPer<T>;
  const T* p;
  int V;
  // tokens base .. base + E - 1; -inf past the end
  __device__ __forceinline__ void load(int base, float* x) const {
    if (base + E <= V) {
      if constexpr (sizeof(T) == 4) {
        const f32x4u a = *(const f32x4u*)(p + base);
#pragma unroll
        for (int i = 0; i < E; ++i) x[i] = a[i] + 0.f;      // (zeros of either sign are one logit)
      } else {
        const u16x8u a = *(const u16x8u*)(p + base);
#pragma unroll
        for (int i = 0; i < E; ++i) x[i] = bf2f(a[i]) + 0.f;
      }
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i) x[i] = base + i < V ? St<T>::ld(p, base + i) + 0.f : -INFINITY;
    }
  }
  // f(segment, first token, x) over the row; a segment is 64 lanes' tokens of a step
  template <class F>
  __device__ __forceinline__ void each(F&& f) const {
    constexpr int U = sizeof(T) == 4 ? 4 : 2, STEP = SM_NT * E;
    const int wave = threadIdx.x >> 6;
    for (int b0 = 0; b0 < V; b0 += U * STEP) {
      float x[U][E];
#pragma unroll
      for (int u = 0; u < U; ++u) load(b0 + u * STEP + (int)threadIdx.x * E, x[u]);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (b0 + u * STEP < V) f((b0 / STEP + u) * SM_NW + wave, b0 + u * STEP + (int)threadIdx.x * E, x[u]);
    }
  }
};

// e^{(l - M) / T} and its whole number of units of 2^-unit.
struct Weights {
  const double* tab;       // 2^(i / 512)
  double top, c;           // 512 log2(e) / T
  int unit;
  __device__ __forceinline__ double scaled(float l, int by) const {
    const double y = ((double)l - top) * c;
    if (!(y > -512.0 * 1080)) return 0.0;                  // (nothing in 64 bits; -inf; 0 times -inf)
    constexpr double kMagic = 6755399441055744.0;          // 1.5 * 2^52: the nearest whole number is in the low bits
    const double t = y + kMagic;
    const int k = __double2loint(t);
    const double r = y - (t - kMagic);
    constexpr double a1 = 6.93147180559945286e-01 / 512, a2 = a1 * a1 / 2, a3 = a1 * a1 * a1 / 6;   // (the next term: 9e-15)
    const double e = fma(fma(fma(a3, r, a2), r, a1), r, 1.0);
    return ldexp(tab[k & (SM_TAB - 1)] * e, (k >> 9) + by);
  }
  __device__ __forceinline__ double value(float l) const { return scaled(l, 0); }
  __device__ __forceinline__ uint64_t whole(float l) const {
    return (uint64_t)__double_as_longlong(scaled(l, unit) + 4503599627370496.0) & 0xfffffffffffffull;   // + 2^52
  }
};

// Tokens whose falling key is below `key`, and of those at it the first `ties`.
struct Cut {
  uint32_t key, ties;
};
__device__ __forceinline__ uint32_t falling(float l) { return ~ordered_u32(l); }
__device__ __forceinline__ float of_falling(uint32_t k) { return from_ordered_u32(~k); }

struct Lds {
  double tab[SM_TAB];
  union {
    uint64_t bins[SM_BINS];
    struct {
      float logit[SM_LIST];
      int32_t token[SM_LIST];
      uint64_t digits[256];
    } list;
  };
  uint64_t seg[kRulesMaxVocab / 256];
  uint64_t sums[SM_NW];
  uint64_t found_before, found_in;
  uint32_t found;
  float tops[SM_NW];
  int32_t first, bad;
};

__device__ __forceinline__ uint64_t wave_add(uint64_t v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor((unsigned long long)v, o, 64);
  return v;
}
__device__ __forceinline__ uint64_t wave_scan(uint64_t v) {    // inclusive
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint64_t y = __shfl_up((unsigned long long)v, o, 64);
    if (lane >= o) v += y;
  }
  return v;
}
// Exclusive sum over the threads; the sum of all in *total.
__device__ uint64_t block_scan(uint64_t v, Lds& s, uint64_t* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint64_t x = wave_scan(v);
  __syncthreads();
  if (lane == 63) s.sums[wave] = x;
  __syncthreads();
  uint64_t before = 0, all = 0;
#pragma unroll
  for (int i = 0; i < SM_NW; ++i) {
    const uint64_t y = s.sums[i];
    before += i < wave ? y : 0;
    all += y;
  }
  *total = all;
  return before + x - v;
}
__device__ uint64_t block_add(uint64_t v, Lds& s) {
  const uint64_t x = wave_add(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s.sums[threadIdx.x >> 6] = x;
  __syncthreads();
  uint64_t all = 0;
#pragma unroll
  for (int i = 0; i < SM_NW; ++i) all += s.sums[i];
  return all;
}

template <int N>
__device__ __forceinline__ void clear_bins(uint64_t* bins) {
  for (int i = threadIdx.x; i < N; i += SM_NT) bins[i] = 0;
  __syncthreads();
}
// The bin at which the running sum reaches `goal`, what is before it and in it; false
// where all bins sum to less.
template <int N>
__device__ bool find_bin(const uint64_t* bins, uint64_t goal, Lds& s, uint64_t* total) {
  constexpr int P = (N + SM_NT - 1) / SM_NT;
  const int b = threadIdx.x * P;
  uint64_t x[P], sum = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < P; ++i) {
    x[i] = b + i < N ? bins[b + i] : 0;
    sum += x[i];
  }
  uint64_t before = block_scan(sum, s, total);
  if (before < goal && goal <= before + sum) {
#pragma unroll
    for (int i = 0; i < P; ++i) {
      if (before < goal && goal <= before + x[i]) s.found = b + i, s.found_before = before, s.found_in = x[i];
      before += x[i];
    }
  }
  __syncthreads();
  return goal <= *total;
}

// Leading bits of M - l, rising as logits fall.
__device__ __forceinline__ int bin_of(float top, float l) { return (int)(__float_as_uint(top - l) >> 18); }

template <typename T>
__global__ __launch_bounds__(SM_NT) void k_sample(SampleLaunch a, int unit) {
  extern __shared__ __attribute__((aligned(16))) char sample_lds[];
  Lds& s = *(Lds*)sample_lds;
  constexpr int E = kPer<T>;
  const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const RowOf<T> x_of = {(const T*)a.logits + row * a.ld, a.vocab};
  const int set = a.set ? a.set[row] : row;
  const bool has = set >= 0 && set < a.sets;
  const float temperature = has && a.temperature ? a.temperature[set] : 1.f;
  const bool greedy = !(temperature > 0.f);
  const int32_t top_k = has && a.top_k ? a.top_k[set] : 0;
  const float top_p = has && a.top_p ? a.top_p[set] : 1.f, min_p_given = has && a.min_p ? a.min_p[set] : 0.f;

  // the largest logit
  float mine = -INFINITY;
  bool nan = false;
  x_of.each([&](int, int, const float* x) {
#pragma unroll
    for (int i = 0; i < E; ++i) {
      mine = fmaxf(mine, x[i]);
      nan |= x[i] != x[i];
    }
  });
  for (int i = tid; i < SM_TAB; i += SM_NT) s.tab[i] = exp2((double)i / SM_TAB);
  if (tid == 0) s.bad = 0, s.first = a.vocab;
  float top = wave_max_lanes(mine);
  if (lane == 0) s.tops[wave] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < SM_NW; ++i) top = fmaxf(top, s.tops[i]);
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
  const Weights w = {s.tab, (double)top, 512.0 * 1.4426950408889634074 / (greedy ? 1.0 : (double)temperature), unit};
  const double inv_unit = ldexp(1.0, -unit);
  uint64_t all = 0;                        // of all weights
  auto answer = [&](int d, int token, float l) {
    token_out[d] = token;
    if (logprob_out)
      logprob_out[d] = (float)(((double)l - w.top) * (w.c / (512.0 * 1.4426950408889634074)) - log((double)all * inv_unit));
  };

  if (greedy) {
    int at = a.vocab;
    x_of.each([&](int, int base, const float* x) {
#pragma unroll
      for (int i = E - 1; i >= 0; --i) {
        all += w.whole(x[i]);
        if (x[i] == top) at = min(at, base + i);
      }
    });
    if (at < a.vocab) atomicMin(&s.first, at);
    all = block_add(all, s);
    if (tid < a.draws) answer(tid, s.first, top);
    if (tid == 0 && a.kept) a.kept[row] = 1;
    return;
  }
  const double min_p = min_p_given > 0.f ? (double)min_p_given : 0.0;
  bool k_on = top_k > 0 && top_k < a.vocab;
  const bool p_on = top_p < 1.f;
  auto p_goal = [&](uint64_t mass) {       // the least whole sum that is not below top_p of the mass
    const double part = (double)top_p * (double)mass;
    return part > 0.0 ? max((uint64_t)ceil(part), (uint64_t)1) : (uint64_t)1;
  };

  // a bin that the cut is not behind
  int last = -1;
  uint64_t before = 0, total;
  bool have_all = false, exact_bin = false;
  if (k_on && top_k <= SM_FEW) {
    clear_bins<SM_BINS>(s.bins);
    if (mine > -INFINITY) atomicAdd((unsigned long long*)&s.bins[bin_of(top, mine)], 1ull);
    if (find_bin<SM_BINS>(s.bins, top_k, s, &total)) last = s.found;
  }
  auto count_bins = [&] {
    __syncthreads();
    clear_bins<SM_BINS>(s.bins);
    x_of.each([&](int, int, const float* x) {
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (x[i] > -INFINITY) atomicAdd((unsigned long long*)&s.bins[bin_of(top, x[i])], 1ull);
    });
    if (find_bin<SM_BINS>(s.bins, top_k, s, &total) && (uint64_t)top_k < total) {
      last = s.found, before = s.found_before, exact_bin = true;
    } else {
      k_on = false, last = -1;
    }
  };
  if (k_on && last < 0) count_bins();
  if (!k_on && p_on) {
    // what weighs less than (1 - p) / V cannot be where the sum passes p of it: those
    // tokens sum to less than 1 - p of the largest weight alone
    const uint64_t least = (uint64_t)((1.0 - (double)top_p) / a.vocab * ldexp(1.0, unit));
    __syncthreads();
    clear_bins<SM_BINS>(s.bins);
    uint64_t rest = 0;
    x_of.each([&](int, int, const float* x) {
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const uint64_t y = w.whole(x[i]);
        if (y > least)
          atomicAdd((unsigned long long*)&s.bins[bin_of(top, x[i])], (unsigned long long)y);
        else
          rest += y;
      }
    });
    all = block_add(rest, s);
    find_bin<SM_BINS>(s.bins, 0, s, &total);
    all += total;
    have_all = true;
    find_bin<SM_BINS>(s.bins, min(p_goal(all), total), s, &total);
    last = s.found, before = s.found_before, exact_bin = true;
  }

  const int segments = (a.vocab + 64 * E - 1) / (64 * E), rounded = (segments + SM_NW - 1) / SM_NW * SM_NW;
  uint64_t listed = SM_LIST + 1;
  if (last >= 0) {
    uint64_t sum = 0;
    __syncthreads();
    x_of.each([&](int seg, int, const float* x) {
      int n = 0;
#pragma unroll
      for (int i = 0; i < E; ++i) {
        n += __popcll(__ballot(bin_of(top, x[i]) <= last && x[i] > -INFINITY));
        if (!have_all) sum += w.whole(x[i]);
      }
      if (lane == 0) s.seg[seg] = n;
    });
    if (!have_all) all = block_add(sum, s), have_all = true;
    __syncthreads();
    uint64_t n[4], mine4 = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      n[i] = 4 * tid + i < rounded ? s.seg[4 * tid + i] : 0;
      mine4 += n[i];
    }
    uint64_t at = block_scan(mine4, s, &listed);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (4 * tid + i < rounded) s.seg[4 * tid + i] = at;
      at += n[i];
    }
    __syncthreads();
  }

  if (listed <= SM_LIST) {
    const int count = (int)listed;
    x_of.each([&](int seg, int base, const float* x) {
      bool in[E];
      int at = (int)s.seg[seg];
      uint64_t any = 0;
#pragma unroll
      for (int i = 0; i < E; ++i) {
        in[i] = bin_of(top, x[i]) <= last && x[i] > -INFINITY;
        const uint64_t is = __ballot(in[i]);
        at += __popcll(is & ((1ull << lane) - 1));
        any |= is;
      }
      if (any) {
#pragma unroll
        for (int i = 0; i < E; ++i)
          if (in[i]) {
            s.list.logit[at] = x[i];
            s.list.token[at] = base + i;
            ++at;
          }
      }
    });
    __syncthreads();
    constexpr int L = SM_LIST / SM_NT;
    float x[L];
    uint32_t key[L];
    uint64_t y[L];
    const uint32_t best = falling(top);
    uint32_t widest = 0;
#pragma unroll
    for (int i = 0; i < L; ++i) {
      const int at = L * tid + i;
      const bool in = at < count;
      x[i] = in ? s.list.logit[at] : -INFINITY;
      y[i] = in ? w.whole(x[i]) : 0;
      key[i] = in ? falling(x[i]) - best : 0xffffffffu;
      if (in) widest = max(widest, key[i]);
    }
    widest = wave_max_u32(widest);
    if (lane == 0) s.tops[wave] = __uint_as_float(widest);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < SM_NW; ++i) widest = max(widest, __float_as_uint(s.tops[i]));
    const int digits = widest ? (39 - __clz(widest)) / 8 : 1;

    bool kept[L];
#pragma unroll
    for (int i = 0; i < L; ++i) kept[i] = L * tid + i < count;
    // keeps what is before the cut at `goal` of counts or weights of what is kept now
    auto cut_list = [&](bool by_count, uint64_t goal) {
      uint32_t prefix = 0;
      uint64_t sum = 0;
      for (int d = digits - 1; d >= 0; --d) {
        for (int i = tid; i < 256; i += SM_NT) s.list.digits[i] = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < L; ++i)
          if (kept[i] && (d == 3 || key[i] >> (8 * d + 8) == prefix >> (8 * d + 8)))
            atomicAdd((unsigned long long*)&s.list.digits[key[i] >> (8 * d) & 255], by_count ? 1ull : (unsigned long long)y[i]);
        uint64_t t;
        find_bin<256>(s.list.digits, goal - sum, s, &t);
        prefix |= s.found << (8 * d);
        sum += s.found_before;
        __syncthreads();
      }
      // the first of those at the cut's logit
      const uint64_t each = by_count ? 1 : max(w.whole(of_falling(prefix + best)), (uint64_t)1);
      const uint64_t ties = (goal - sum + each - 1) / each;
      uint64_t at = 0, t;
#pragma unroll
      for (int i = 0; i < L; ++i) at += kept[i] && key[i] == prefix;
      at = block_scan(at, s, &t);
#pragma unroll
      for (int i = 0; i < L; ++i) {
        if (kept[i] && key[i] == prefix) {
          kept[i] = at < ties;
          ++at;
        } else {
          kept[i] = kept[i] && key[i] < prefix;
        }
      }
    };
    if (k_on) cut_list(true, top_k);
    if (p_on) {
      uint64_t mass = all;
      if (k_on) {
        mass = 0;
#pragma unroll
        for (int i = 0; i < L; ++i) mass += kept[i] ? y[i] : 0;
        mass = block_add(mass, s);
      }
      cut_list(false, p_goal(mass));
    }
    if (min_p > 0.0) {
#pragma unroll
      for (int i = 0; i < L; ++i)
        if (kept[i] && key[i] == 0) atomicMin(&s.first, L * tid + i);
      __syncthreads();
#pragma unroll
      for (int i = 0; i < L; ++i) kept[i] = kept[i] && (L * tid + i == s.first || w.value(x[i]) >= min_p);
    }
    uint64_t sum = 0, mass, n = 0;
#pragma unroll
    for (int i = 0; i < L; ++i) {
      if (!kept[i]) y[i] = 0;
      sum += y[i];
      n += kept[i];
    }
    n = block_add(n, s);
    if (tid == 0 && a.kept) a.kept[row] = (int32_t)n;
    const uint64_t from = block_scan(sum, s, &mass);
    for (int d = 0; d < a.draws; ++d) {
      const float u = a.u[(int64_t)row * a.draws + d];
      const uint64_t goal = min((uint64_t)((u > 0.f ? fmin((double)u, 1.0 - 0x1p-24) : 0.0) * (double)mass), mass - 1);
      if (from <= goal && goal < from + sum) {
        uint64_t c = from;
#pragma unroll
        for (int i = 0; i < L; ++i) {
          if (c <= goal && goal < c + y[i]) answer(d, s.list.token[L * tid + i], x[i]);
          c += y[i];
        }
      }
    }
    return;
  }

  // ---- many tokens: cuts by digits over the row
  Cut cut = {falling(-INFINITY), 0};
  bool tied = false;                       // only some of the tokens at the cut's logit
  // the cut at which the counts or weights of what `cut` leaves, before + those of
  // bin `last`, reach goal
  auto cut_row = [&](bool by_count, uint64_t goal) {
    const Cut in = cut;
    uint32_t prefix = 0;
    uint64_t sum = before, here = 0;
#pragma unroll 1
    for (int level = 0; level < 3; ++level) {
      const int shift = level == 0 ? 21 : level == 1 ? 10 : 0, bits = level == 2 ? 10 : 11;
      __syncthreads();
      clear_bins<2048>(s.bins);
      x_of.each([&](int, int, const float* x) {
#pragma unroll
        for (int i = 0; i < E; ++i) {
          const uint32_t k = falling(x[i]);
          if (bin_of(top, x[i]) != last || !(x[i] > -INFINITY) || (level > 0 && (k ^ prefix) >> (shift + bits))) continue;
          if (by_count)
            atomicAdd((unsigned long long*)&s.bins[k >> shift & ((1 << bits) - 1)], 1ull);
          else if (k < in.key)
            atomicAdd((unsigned long long*)&s.bins[k >> shift & ((1 << bits) - 1)], (unsigned long long)w.whole(x[i]));
        }
      });
      __syncthreads();
      const float l = of_falling(in.key);
      if (!by_count && in.ties && tid == 0 && bin_of(top, l) == last && !(level > 0 && (in.key ^ prefix) >> (shift + bits)))
        s.bins[in.key >> shift & ((1 << bits) - 1)] += in.ties * w.whole(l);
      uint64_t t;
      find_bin<2048>(s.bins, goal - sum, s, &t);
      prefix |= s.found << shift;
      sum += s.found_before;
      here = s.found_in;
    }
    const uint64_t each = by_count ? 1 : max(w.whole(of_falling(prefix)), (uint64_t)1);
    const uint64_t ties = (goal - sum + each - 1) / each;
    tied = ties * each < here || (prefix == in.key && tied);
    cut = {prefix, (uint32_t)ties};
  };
  if (k_on) {
    if (!exact_bin) count_bins();
    if (k_on) cut_row(true, top_k);
  }
  if (p_on) {
    if (k_on) {
      // weights of what top-k leaves
      __syncthreads();
      clear_bins<SM_BINS>(s.bins);
      x_of.each([&](int, int, const float* x) {
#pragma unroll
        for (int i = 0; i < E; ++i)
          if (falling(x[i]) < cut.key) atomicAdd((unsigned long long*)&s.bins[bin_of(top, x[i])], (unsigned long long)w.whole(x[i]));
      });
      __syncthreads();
      const float l = of_falling(cut.key);
      if (tid == 0) s.bins[bin_of(top, l)] += cut.ties * w.whole(l);
      find_bin<SM_BINS>(s.bins, 0, s, &total);
      find_bin<SM_BINS>(s.bins, p_goal(total), s, &total);
      last = s.found, before = s.found_before;
      cut_row(false, p_goal(total));
    } else {
      cut_row(false, min(p_goal(all), total));
    }
  }
  // the last token at the cut's logit that is kept
  int last_tie = cut.ties ? a.vocab : -1;
  if (tied) {
    __syncthreads();
    x_of.each([&](int seg, int, const float* x) {
      int n = 0;
#pragma unroll
      for (int i = 0; i < E; ++i) n += __popcll(__ballot(falling(x[i]) == cut.key));
      if (lane == 0) s.seg[seg] = n;
    });
    __syncthreads();
    uint64_t n[4], mine4 = 0, t;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      n[i] = 4 * tid + i < rounded ? s.seg[4 * tid + i] : 0;
      mine4 += n[i];
    }
    uint64_t at = block_scan(mine4, s, &t);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (at < cut.ties && cut.ties <= at + n[i]) s.found = 4 * tid + i, s.found_before = at;
      at += n[i];
    }
    __syncthreads();
    if (wave == 0) {
      float x[E];
      const int base = (int)s.found * 64 * E + lane * E;
      x_of.load(base, x);
      uint32_t c = (uint32_t)s.found_before;
#pragma unroll
      for (int i = 0; i < E; ++i) c += __popcll(__ballot(falling(x[i]) == cut.key) & ((1ull << lane) - 1));
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (falling(x[i]) == cut.key && ++c == cut.ties) s.first = base + i;
    }
    __syncthreads();
    last_tie = s.first;
    __syncthreads();
    if (tid == 0) s.first = a.vocab;
  }
  if (min_p > 0.0) {
    int at = a.vocab;
    __syncthreads();
    x_of.each([&](int, int base, const float* x) {
#pragma unroll
      for (int i = E - 1; i >= 0; --i)
        if (x[i] == top) at = min(at, base + i);
    });
    if (at < a.vocab) atomicMin(&s.first, at);
    __syncthreads();
  }
  const int first_best = s.first;
  const bool bare = !k_on && !p_on;
  auto keeps = [&](float l, int token) {
    if (!(l > -INFINITY)) return false;
    const uint32_t k = falling(l);
    if (!bare && (k > cut.key || (k == cut.key && token > last_tie))) return false;
    return !(min_p > 0.0) || token == first_best || w.value(l) >= min_p;
  };
  uint64_t sum = 0, n = 0;
  __syncthreads();
  x_of.each([&](int seg, int base, const float* x) {
    uint64_t part = 0;
    bool some = false;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const bool in = keeps(x[i], base + i);
      some |= in;
      n += in;
      const uint64_t y = !have_all || in ? w.whole(x[i]) : 0;
      sum += y;
      part += in ? y : 0;
    }
    part = __any(some) ? wave_add(part) : 0;
    if (lane == 0) s.seg[seg] = part;
  });
  if (!have_all) all = block_add(sum, s);
  n = block_add(n, s);
  if (tid == 0 && a.kept) a.kept[row] = (int32_t)n;
  __syncthreads();
  uint64_t y[4], mine4 = 0, mass;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y[i] = 4 * tid + i < rounded ? s.seg[4 * tid + i] : 0;
    mine4 += y[i];
  }
  uint64_t at = block_scan(mine4, s, &mass);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    at += y[i];
    if (4 * tid + i < rounded) s.seg[4 * tid + i] = at;        // up to and with it
  }
  __syncthreads();
  for (int d = wave; d < a.draws; d += SM_NW) {
    const float u = a.u[(int64_t)row * a.draws + d];
    const uint64_t goal = min((uint64_t)((u > 0.f ? fmin((double)u, 1.0 - 0x1p-24) : 0.0) * (double)mass), mass - 1);
    int lo = 0, hi = rounded - 1;                              // the first segment whose sum is above goal
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (s.seg[mid] > goal) hi = mid; else lo = mid + 1;
    }
    float x[E];
    uint64_t z[E], own = 0;
    const int base = lo * 64 * E + lane * E;
    x_of.load(base, x);
#pragma unroll
    for (int i = 0; i < E; ++i) {
      z[i] = keeps(x[i], base + i) ? w.whole(x[i]) : 0;
      own += z[i];
    }
    uint64_t c = (lo ? s.seg[lo - 1] : 0) + wave_scan(own) - own;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      if (c <= goal && goal < c + z[i]) answer(d, base + i, x[i]);
      c += z[i];
    }
  }
}

}  // namespace

hipError_t sample(const SampleLaunch& a, bool bf16, hipStream_t s) {
  int log2 = 0;
  while ((1 << log2) < a.vocab) ++log2;
  const int unit = log2 < 12 ? 50 : 62 - log2;
  const void* k = bf16 ? (const void*)k_sample<bf16_t> : (const void*)k_sample<float>;
  const hipError_t e = hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, sizeof(Lds));
  if (e != hipSuccess) return e;
  if (bf16)
    k_sample<bf16_t><<<dim3((unsigned)a.rows), SM_NT, sizeof(Lds), s>>>(a, unit);
  else
    k_sample<float><<<dim3((unsigned)a.rows), SM_NT, sizeof(Lds), s>>>(a, unit);
  return hipSuccess;
}

}  // namespace asr
