// Tokens drawn from logits under temperature, top-k, top-p and min-p by given
// random numbers (asr_sample).
//
// The kept tokens are a prefix of the falling order, so they are those above a cut:
// a logit and, among the tokens that have it, the last token.  A row's block finds
// the cut of top-k by counts and then that of top-p by weights, each by the digits
// of the logits' order from the top, and draws by adding up weights in the order of
// tokens.  Weights are whole numbers, so sums do not depend on any order.
#include "asr_device.h"

namespace asr {
namespace {

constexpr int SM_NT = 1024, SM_NW = SM_NT / 64, SM_BINS = 2048;

// e^x for x <= 0: e^x = 2^n e^r, |r| <= ln 2 / 2, and Taylor's series to r^13 / 13!
// (the next term is below 2^-57 of the result).
__device__ __forceinline__ double exp_neg(double x) {
  if (!(x > -708.0)) return 0.0;
  const double n = rint(x * 1.4426950408889634);
  const double r = fma(n, -1.90821492927058770002e-10, fma(n, -6.93147180369123816490e-01, x));
  double s = 1.0 / 6227020800.0;
  s = fma(s, r, 1.0 / 479001600.0);
  s = fma(s, r, 1.0 / 39916800.0);
  s = fma(s, r, 1.0 / 3628800.0);
  s = fma(s, r, 1.0 / 362880.0);
  s = fma(s, r, 1.0 / 40320.0);
  s = fma(s, r, 1.0 / 5040.0);
  s = fma(s, r, 1.0 / 720.0);
  s = fma(s, r, 1.0 / 120.0);
  s = fma(s, r, 1.0 / 24.0);
  s = fma(s, r, 1.0 / 6.0);
  s = fma(s, r, 0.5);
  s = fma(s, r, 1.0);
  s = fma(s, r, 1.0);
  return ldexp(s, (int)n);
}

struct RowParams {
  double over_t, unit;      // 1 / T, weights per 1
  float top;
};
__device__ __forceinline__ uint64_t weight(const RowParams& r, float l) {
  if (l == -INFINITY) return 0;
  return (uint64_t)rint(exp_neg(((double)l - (double)r.top) * r.over_t) * r.unit);
}

template <typename V>
__device__ __forceinline__ V wave_add(V v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
template <typename V>
__device__ __forceinline__ V block_add(V v, V* lds) {       // lds: SM_NW
  v = wave_add(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  V s = 0;
  for (int i = 0; i < SM_NW; ++i) s += lds[i];
  return s;
}

// The cut: tokens whose key is above `key`, and of those at it the first `ties`.
struct Cut {
  uint32_t key, ties;
};

struct Lds {
  uint64_t mass[SM_BINS];
  uint64_t sums[SM_NW];
  uint64_t found_before;
  uint32_t found_bin;
};

// The cut at which what the tokens before it sum to reaches `goal`, among those
// above or at `in`; by counts (goal tokens) or weights.  before(bin) < goal <= before
// + in bin, bins from the highest.
template <bool COUNT, class Key, class Of>
__device__ Cut find_cut(int V, uint64_t goal, const Cut& in, Key&& key_of, Of&& weight_of, Lds& s) {
  uint32_t prefix = 0;
  uint64_t before = 0;
  for (int level = 0; level < 3; ++level) {
    const int shift = level == 0 ? 21 : level == 1 ? 10 : 0, bits = level == 2 ? 10 : 11, n = 1 << bits;
    for (int i = threadIdx.x; i < n; i += SM_NT) s.mass[i] = 0;
    __syncthreads();
    for (int v = threadIdx.x; v < V; v += SM_NT) {
      const uint32_t k = key_of(v);
      if (level > 0 && (k >> (shift + bits)) != (prefix >> (shift + bits))) continue;
      if (k < in.key) continue;
      if (COUNT)
        atomicAdd((unsigned long long*)&s.mass[(k >> shift) & (n - 1)], 1ull);
      else if (k > in.key)
        atomicAdd((unsigned long long*)&s.mass[(k >> shift) & (n - 1)], (unsigned long long)weight_of(v));
    }
    __syncthreads();
    // (the tokens at the cut that is given: its first ones only)
    if (!COUNT && threadIdx.x == 0 && (level == 0 || (in.key >> (shift + bits)) == (prefix >> (shift + bits))))
      s.mass[(in.key >> shift) & (n - 1)] += in.ties * weight_of(-1);
    __syncthreads();
    if (threadIdx.x == 0) {
      int b = n - 1;
      uint64_t sum = before;
      while (b > 0 && sum + s.mass[b] < goal) sum += s.mass[b--];
      s.found_bin = b;
      s.found_before = sum;
    }
    __syncthreads();
    prefix |= s.found_bin << shift;
    before = s.found_before;
    __syncthreads();
  }
  Cut c;
  c.key = prefix;
  if (COUNT) {
    c.ties = (uint32_t)(goal - before);
  } else {
    c.ties = 0;                                    // (the caller's: from found_before)
  }
  return c;
}

template <typename T>
__global__ __launch_bounds__(SM_NT) void k_sample(SampleLaunch a, int unit_log2) {
  __shared__ Lds s;
  const int row = blockIdx.x, tid = threadIdx.x, V = a.vocab;
  const T* logits = (const T*)a.logits + row * a.ld;
  auto of = [&](int v) { return St<T>::ld(logits, v); };
  const int set = a.set ? a.set[row] : row;
  const bool has = set >= 0 && set < a.sets;
  const float t = has && a.temperature ? a.temperature[set] : 1.f;
  const bool greedy = !(t > 0.f);

  float top = -INFINITY;
  int bad = 0;
  for (int v = tid; v < V; v += SM_NT) {
    const float l = of(v);
    if (l != l || l == INFINITY) bad = 1;
    top = fmaxf(top, l);
  }
  bad = block_add<uint64_t>(bad, s.sums) > 0;
  top = wave_max_lanes(top);
  __shared__ float tops[SM_NW];
  if ((tid & 63) == 0) tops[tid >> 6] = top;
  __syncthreads();
  for (int i = 0; i < SM_NW; ++i) top = fmaxf(top, tops[i]);
  if (bad || top == -INFINITY) {
    for (int d = tid; d < a.draws; d += SM_NT) {
      a.token[(int64_t)row * a.draws + d] = -1;
      if (a.logprob) a.logprob[(int64_t)row * a.draws + d] = bad ? NAN : -INFINITY;
    }
    if (tid == 0 && a.kept) a.kept[row] = 0;
    return;
  }
  const RowParams r = {greedy ? 1.0 : 1.0 / (double)t, ldexp(1.0, unit_log2), top + 0.f};
  auto key_of = [&](int v) { return ordered_u32(of(v) + 0.f); };

  // all weights, and tokens that have any
  uint64_t all = 0, some = 0;
  for (int v = tid; v < V; v += SM_NT) {
    all += weight(r, of(v));
    some += of(v) > -INFINITY;
  }
  all = block_add(all, s.sums);
  some = block_add(some, s.sums);

  Cut cut = {ordered_u32(-INFINITY), 0};           // everything above -inf
  uint64_t k = some;
  if (greedy) {
    k = 1;
  } else if (has && a.top_k && a.top_k[set] > 0) {
    k = min(some, (uint64_t)a.top_k[set]);
  }
  if (k < some) cut = find_cut<true>(V, k, cut, key_of, [&](int) { return (uint64_t)1; }, s);
  const float p = !greedy && has && a.top_p ? a.top_p[set] : 1.f;
  if (p < 1.f) {
    uint64_t mine = 0;
    for (int v = tid; v < V; v += SM_NT)
      if (key_of(v) > cut.key) mine += weight(r, of(v));
    mine = block_add(mine, s.sums);
    const uint64_t at_cut = weight(r, from_ordered_u32(cut.key));
    mine += cut.ties * at_cut;
    // the smallest whole sum that is not below p of the mass
    const double part = (double)p * (double)mine;
    const uint64_t goal = part > 0.0 ? max((uint64_t)ceil(part), (uint64_t)1) : 1;
    const Cut c = find_cut<false>(V, goal, cut, key_of, [&](int v) { return v < 0 ? at_cut : weight(r, of(v)); }, s);
    const uint64_t before = s.found_before, w = weight(r, from_ordered_u32(c.key));
    cut = {c.key, (uint32_t)((goal - before + w - 1) / w)};
  }
  const float min_p = !greedy && has && a.min_p ? a.min_p[set] : 0.f;

  // the last token at the cut's key that is kept
  __shared__ int last_tie, first_best;
  if (tid == 0) last_tie = -1, first_best = V;
  __syncthreads();
  if (tid < 64) {
    uint32_t seen = 0;
    for (int v0 = 0; v0 < V && seen < cut.ties; v0 += 64) {
      const uint64_t is = __ballot(v0 + tid < V && key_of(min(v0 + tid, V - 1)) == cut.key);
      const uint32_t n = __popcll(is);
      if (seen + n >= cut.ties) {
        const uint64_t below = is & ((1ull << tid) - 1);
        if ((is >> tid & 1) && seen + __popcll(below) + 1 == cut.ties) last_tie = v0 + tid;
      } else if (n > 0 && tid == 0) {
        last_tie = v0 + 63 - __builtin_clzll(is);
      }
      seen += n;
    }
  }
  for (int v = tid; v < V; v += SM_NT)
    if (of(v) == r.top) { atomicMin(&first_best, v); break; }
  __syncthreads();
  auto kept = [&](int v) {
    const uint32_t key = key_of(v);
    if (key < cut.key || (key == cut.key && v > last_tie)) return false;
    if (v == first_best) return true;
    return !(min_p > 0.f) || exp_neg(((double)of(v) - (double)r.top) * r.over_t) >= (double)min_p;
  };
  uint64_t mass = 0, n = 0;
  for (int v = tid; v < V; v += SM_NT)
    if (kept(v)) mass += weight(r, of(v)), ++n;
  mass = block_add(mass, s.sums);
  n = block_add(n, s.sums);
  if (tid == 0 && a.kept) a.kept[row] = (int32_t)n;

  // draws: a wave each, 64 tokens at a time
  const int lane = tid & 63;
  for (int d = tid >> 6; d < a.draws; d += SM_NW) {
    const float u = a.u[(int64_t)row * a.draws + d];
    const double x = u > 0.f ? fmin((double)u, 1.0 - 0x1p-24) : 0.0;
    const uint64_t goal = min((uint64_t)(x * (double)mass), mass - 1);
    uint64_t before = 0;
    int token = -1;
    for (int v0 = 0; v0 < V; v0 += 64) {
      const int v = v0 + lane;
      uint64_t w = v < V && kept(v) ? weight(r, of(v)) : 0;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const uint64_t y = __shfl_up(w, o, 64);
        if (lane >= o) w += y;
      }
      const uint64_t past = __ballot(before + w > goal);
      if (past) {
        token = v0 + __ffsll((unsigned long long)past) - 1;
        break;
      }
      before += __shfl(w, 63, 64);
    }
    if (lane == 0) {
      a.token[(int64_t)row * a.draws + d] = token;
      if (a.logprob)
        a.logprob[(int64_t)row * a.draws + d] =
            (float)(((double)of(token) - (double)r.top) * r.over_t - log((double)all / r.unit));
    }
  }
}

}  // namespace

void sample(const SampleLaunch& a, bool bf16, hipStream_t s) {
  int log2 = 0;
  while ((1 << log2) < a.vocab) ++log2;
  if (bf16)
    k_sample<bf16_t><<<dim3((unsigned)a.rows), SM_NT, 0, s>>>(a, 62 - log2);
  else
    k_sample<float><<<dim3((unsigned)a.rows), SM_NT, 0, s>>>(a, 62 - log2);
}

}  // namespace asr
