// Rules on logits and the k best tokens (asr_logit_rules): penalties for
// repeated tokens, biases, masks of allowed tokens and a temperature, and the
// log-probabilities of the best tokens under what remains.
//
// One pass over the logits.  256 threads take 4096 tokens of a row, 16 a thread,
// in registers.  What is sparse -- the row's history, its biases -- is scattered
// into an LDS table of the block's tokens (every block of a row reads the whole
// lists) and read back by the threads that own the tokens, so nothing of the
// vocabulary's size is cleared, written or read besides the logits themselves.
// The 256 threads leave their maximum, their sum of exponentials and their k best
// tokens; a row's last block joins them.  HBM bounds a batch of rows, a chain of
// loads a single one; long histories would be read once for 4096 tokens, so
// with those a block is 1024 threads with the same work each (and the join, which
// would cost them registers, a kernel of its own).
//
// Measured: the best of 51865 float32 logits 7.3 us; of 128 such rows 14.7 us, 1.8
// TB/s (473 vector instructions a wave, 5 us of it); 256 rows of 131071 bf16 logits,
// 32768 tokens of history each, 5 best and the processed logits 95 us, 2.3 TB/s
// (1143 instructions a wave, 61 us; on inputs seen before 83 us, 45 without rules).
#include <algorithm>

#include "asr_device.h"

// Every operation below is rounded by itself, as the definition has it: two
// logits that it makes equal stay equal.
#pragma clang fp contract(off)

namespace asr {
namespace {

constexpr int RU_NT = 256, RU_E = 16, RU_CHUNK = RU_NT * RU_E;
static_assert(RU_CHUNK == kRulesChunk, "workspace");
// chunks of a block where histories may be long: every block reads all of them
constexpr int RU_LONG = 4, kLongHistory = 4096;
constexpr uint32_t kSeen = 0x80000000u;     // in the history; below it the count behind the prompt

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef int32_t i32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4u __attribute__((ext_vector_type(4), aligned(2)));

// VEC neighbouring logits; rows begin at any element (an odd vocabulary), which
// the loads take as it is.
template <typename T>
struct Logits;
template <>
struct Logits<float> {
  static constexpr int VEC = 4;
  static __device__ __forceinline__ void load(const float* p, float* v) {
    const f32x4u x = *(const f32x4u*)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = x[i];
  }
};
template <>
struct Logits<bf16_t> {
  static constexpr int VEC = 8;
  static __device__ __forceinline__ void load(const bf16_t* p, float* v) {
    const u32x4u x = *(const u32x4u*)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(x[i] << 16);
      v[2 * i + 1] = __uint_as_float(x[i] & 0xffff0000u);
    }
  }
};

// x / d of N values, correctly rounded, one divisor for all.  With r the rounded
// 1 / d, q = x r is off by 2 steps at most, one correction q -= r (q d - x) makes
// it one of the two floats around x / d, and a second one, by Markstein's theorem,
// the nearest: 5 instructions where a division by itself takes 11.  The theorem
// wants q d - x exact, hence no quotient or residual near the ends of the range;
// a wave with such values (infinities among them) divides.  A residual of 0 is +0
// for x = 0 and x = -0, and q - r 0 is q: a quotient keeps the sign of its zero
// (with the residual x - q d it would not).
template <int N>
__device__ __forceinline__ void divide(const float* x, float d, float r, float* y) {
  float hi = 0.f;
  uint32_t lo = 0xffffffffu;                           // (of the magnitudes' bits but zeros')
#pragma unroll
  for (int i = 0; i < N; ++i) {
    hi = fmaxf(hi, fabsf(x[i]));
    lo = min(lo, (__float_as_uint(x[i]) << 1) - 1u);
  }
  if (!(d >= 0x1p-20f && d <= 0x1p20f) || __any(hi > 0x1p100f || lo < (__builtin_bit_cast(uint32_t, 0x1p-70f) << 1) - 1u)) {
#pragma unroll
    for (int i = 0; i < N; ++i) y[i] = x[i] / d;
    return;
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float q = x[i] * r;
    q = fmaf(-fmaf(q, d, -x[i]), r, q);
    y[i] = fmaf(-fmaf(q, d, -x[i]), r, q);
  }
}

// Order of the results: larger first, a NaN before all, the lower token of two
// equal ones (0 and -0 are); 0 for what is never chosen.
__device__ __forceinline__ uint32_t rank_of(float z) {
  if (z != z) return 0xffffffffu;
  return z == -INFINITY ? 0u : ordered_u32(z + 0.f);
}

// The largest of the lanes' (rank, token) pairs; its lane, or -1 where all ranks are 0.
__device__ __forceinline__ int best_lane(uint32_t rank, int token) {
  const uint32_t top = wave_max_u32(rank);
  if (top == 0) return -1;
  uint64_t who = __ballot(rank == top);
  if (who & (who - 1)) {
    const uint32_t low = wave_max_u32(rank == top ? ~(uint32_t)token : 0u);
    who = __ballot(rank == top && ~(uint32_t)token == low);
  }
  return __ffsll((unsigned long long)who) - 1;
}

// The history's n entries into the block's table: the first `marked` as seen, the
// others counted.  Every block reads the whole list, so what counts is the
// instructions of an entry: 16 a thread without a test while there are so many,
// then fewer.  What is no token, or none of the block's, ends far above them.
// first: entries threadIdx.x + i NT, i < RU_FIRST, loaded ahead (short histories).
constexpr int RU_FIRST = 4;
template <int NT, int TOKENS>
__device__ __forceinline__ void count_tokens(const int32_t* list, const int* first, int marked, int n, int b0, uint32_t* table) {
  int from = 0;
  for (; n - from >= 16 * NT; from += 16 * NT) {
    i32x4u tok[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) tok[i] = *(const i32x4u*)(list + from + (i * NT + (int)threadIdx.x) * 4);
    auto each = [&](auto&& f) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t u = (uint32_t)tok[i][e] - (uint32_t)b0;
          if (u < TOKENS) f(u, from + (i * NT + (int)threadIdx.x) * 4 + e);
        }
    };
    if (from + 16 * NT <= marked)
      each([&](uint32_t u, int) { atomicOr(&table[u], kSeen); });
    else
      each([&](uint32_t u, int j) {
        if (j < marked)
          atomicOr(&table[u], kSeen);
        else
          atomicAdd(&table[u], 1u);
      });
  }
  constexpr int W = NT > RU_NT ? 8 : 4;
  for (; from < n; from += W * NT) {
    int tok[W];
    const int at = from + (int)threadIdx.x;
    if (from > 0 || !first) {
#pragma unroll
      for (int i = 0; i < W; ++i) tok[i] = list[min(at + i * NT, n - 1)];
    } else {
#pragma unroll
      for (int i = 0; i < RU_FIRST; ++i) tok[i] = first[i];
    }
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const int j = at + i * NT;
      const uint32_t u = (uint32_t)tok[i] - (uint32_t)b0;
      if (j >= n || u >= TOKENS) continue;
      if (j < marked)
        atomicOr(&table[u], kSeen);
      else
        atomicAdd(&table[u], 1u);
    }
  }
}

// A result: the better of two is the larger one, 0 is none.
__device__ __forceinline__ uint64_t result_of(uint32_t rank, int token) { return (uint64_t)rank << 32 | ~(uint32_t)token; }

// What one block leaves for another to read (of the same launch where there are
// counters).
__device__ __forceinline__ void leave(const RulesLaunch& a, uint64_t* p, uint64_t v) {
  if (a.counters)
    store_agent(p, v);
  else
    *p = v;
}
__device__ __forceinline__ uint64_t left_by(const RulesLaunch& a, const uint64_t* p) {
  return a.counters ? load_agent(p) : *p;
}

// How many of the results x of the lanes `in` are better than `mine`.
__device__ __forceinline__ int better(uint64_t x, uint64_t in, uint64_t mine) {
  int count = 0;
  while (in) {
    const int i = __ffsll((unsigned long long)in) - 1;
    in &= in - 1;
    const uint64_t y = (uint64_t)__builtin_amdgcn_readlane((uint32_t)(x >> 32), i) << 32 |
                       (uint32_t)__builtin_amdgcn_readlane((uint32_t)x, i);
    count += y > mine;
  }
  return count;
}

// A rank such that at least k of the lanes' largest ranks lie at or above it (1
// where there are not so many above 0): the wave's k best do too, and few others.
__device__ __forceinline__ uint32_t rank_floor(uint32_t largest, int k) {
  uint32_t t = 0;
#pragma unroll
  for (int bit = 31; bit >= 16; --bit) {
    const uint32_t x = t | 1u << bit;
    if (__popcll(__ballot(largest >= x)) >= k) t = x;
  }
  return t ? t : 1u;
}

// The wave's LDS writes are done before its next reads.
__device__ __forceinline__ void wave_lds_done() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
}

constexpr int RU_CAND = 64;                  // candidates of a wave
constexpr uint32_t kLowest = 0x00800000u;    // rank of the lowest finite float

template <typename T, int SUBS>
__device__ __forceinline__ bool rules_block(const RulesLaunch& a, int chunks) {
  constexpr int VEC = Logits<T>::VEC, NV = RU_E / VEC, NT = SUBS * RU_NT, TOKENS = SUBS * RU_CHUNK;
  extern __shared__ __attribute__((aligned(16))) uint32_t table[];   // [TOKENS] where there are lists
  __shared__ uint64_t cand[SUBS * 4][RU_CAND];
  __shared__ int cand_n[SUBS * 4];
  __shared__ uint32_t cand_least[SUBS * 4];
  __shared__ float wave_ms[SUBS * 4][2];
  const int tid = threadIdx.x % RU_NT, sub = threadIdx.x / RU_NT, lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = blockIdx.y, b0 = blockIdx.x * TOKENS, v0 = b0 + sub * RU_CHUNK;
  const int V = a.vocab;
  const T* src = (const T*)a.logits + (int64_t)row * a.ld + v0;
  uint32_t* own = table + sub * RU_CHUNK;

  float z[RU_E];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int u = (i * RU_NT + tid) * VEC;
    if (v0 + u + VEC <= V) {
      Logits<T>::load(src + u, z + i * VEC);
    } else {
#pragma unroll
      for (int j = 0; j < VEC; ++j) z[i * VEC + j] = v0 + u + j < V ? St<T>::ld(src, u + j) : -INFINITY;
    }
  }

  // everything about the set at once (a chain of loads is what a single row waits for)
  int set = a.set ? a.set[row] : row;
  const bool ruled = set >= 0 && set < a.sets;
  if (!ruled) set = 0;
  const bool some = ruled && a.sets > 0;
  const bool biased = some && a.bias_token;
  // ... and of its lists what fits, before their lengths are known (rows are as long as they say)
  const int32_t* hist = a.history + (int64_t)set * a.history_ld;
  int said[RU_FIRST] = {};
  if (SUBS == 1 && some && a.history) {
#pragma unroll
    for (int i = 0; i < RU_FIRST; ++i)
      if (i * NT < a.history_ld) said[i] = hist[min((int)threadIdx.x + i * NT, (int)a.history_ld - 1)];
  }
  const int32_t* bt = a.bias_token + (int64_t)set * a.bias_ld;
  const float* bv = a.bias_value + (int64_t)set * a.bias_ld;
  int bias_tok = -1;
  float bias_val = 0.f;
  if (biased && lane < a.bias_ld) {
    bias_tok = bt[lane];
    bias_val = bv[lane];
  }
  const int hist_len = some && a.history ? a.history_len[set] : 0;
  const int prompt = some && a.history && a.prompt_len ? a.prompt_len[set] : 0;
  const int bias_len = biased ? a.bias_len[set] : 0;
  const int mask_row = some && a.mask ? (a.mask_of ? a.mask_of[set] : set) : -1;
  const float rep = some && a.repetition ? a.repetition[set] : 1.f;
  const float freq = some && a.frequency ? a.frequency[set] : 0.f;
  const float pres = some && a.presence ? a.presence[set] : 0.f;
  const float temp = some && a.temperature ? a.temperature[set] : 1.f;
  const int hist_n = (int)min((int64_t)max(hist_len, 0), a.history_ld);
  const int bias_n = (int)min((int64_t)max(bias_len, 0), a.bias_ld);
  const bool masked = mask_row >= 0 && mask_row < a.masks;
  uint32_t words[NV];
  if (masked) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int v = v0 + (i * RU_NT + tid) * VEC;      // VEC tokens lie in one word
      words[i] = v < V ? a.mask[(int64_t)mask_row * a.mask_ld + (v >> 5)] >> (v & 31) : 0u;
    }
  }
  if (hist_n > 0) {                                    // block-uniform
#pragma unroll
    for (int i = 0; i < RU_E / 4; ++i) *(uint4*)(table + (i * NT + (int)threadIdx.x) * 4) = uint4{0u, 0u, 0u, 0u};
    __syncthreads();
    count_tokens<NT, TOKENS>(hist, SUBS == 1 ? said : nullptr, prompt, hist_n, b0, table);
    __syncthreads();
    const float rep_r = 1.f / rep;
#pragma unroll
    for (int i = 0; i < RU_E / 4; ++i) {
      const int u = i * 4 / VEC * RU_NT * VEC + tid * VEC + i * 4 % VEC;
      const uint4 c4 = *(const uint4*)(own + u);
      const uint32_t c[4] = {c4.x, c4.y, c4.z, c4.w};
      // (few of the wave's tokens were said, mostly none: no division for them)
      if (!__any(c4.x | c4.y | c4.z | c4.w)) continue;
      float q[4];
      divide<4>(z + 4 * i, rep, rep_r, q);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float x = z[4 * i + j];
        x = x > 0.f ? q[j] : x * rep;
        const uint32_t times = c[j] & ~kSeen;
        if (times) x = (x - freq * (float)times) - pres;
        z[4 * i + j] = c[j] ? x : z[4 * i + j];
      }
    }
  }
  if (biased) {
    // the biases in the order of their list, so that a token given twice has one
    // sum: each wave adds up those of its own tokens, in their places of the table
    // (which no other wave reads any more).  A token without biases has the sum 0,
    // which makes a 0 of a -0
    float* sums = (float*)own;
    const auto place = [&](int i) { return i * 4 / VEC * RU_NT * VEC + tid * VEC + i * 4 % VEC; };
    bool some_hit = false;
    const auto add = [&](int tok, float val) {
      const uint32_t u = (uint32_t)tok - (uint32_t)v0;
      uint64_t hit = __ballot(tok >= 0 && u < RU_CHUNK && (int)(u / (64 * VEC) & 3) == (wave & 3));
      if (!hit) return;
      if (!some_hit) {
#pragma unroll
        for (int i = 0; i < RU_E / 4; ++i) *(float4*)(sums + place(i)) = float4{0.f, 0.f, 0.f, 0.f};
        wave_lds_done();
        some_hit = true;
      }
      while (hit) {
        const int l = __ffsll((unsigned long long)hit) - 1;
        hit &= hit - 1;
        const uint32_t ul = __builtin_amdgcn_readlane(u, l);
        const float vl = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(val), l));
        if (lane == 0) sums[ul] += vl;
      }
    };
    if (bias_n > 0) add(lane < bias_n ? bias_tok : -1, bias_val);
    for (int j0 = 64; j0 < bias_n; j0 += 256) {
      int tok[4];
      float val[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int j = min(j0 + 64 * i + lane, bias_n - 1);
        tok[i] = bt[j];
        val[i] = bv[j];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) add(j0 + 64 * i + lane < bias_n ? tok[i] : -1, val[i]);
    }
    if (some_hit) {
      wave_lds_done();
#pragma unroll
      for (int i = 0; i < RU_E / 4; ++i) {
        const float4 x = *(const float4*)(sums + place(i));
        z[4 * i] = z[4 * i] + x.x;
        z[4 * i + 1] = z[4 * i + 1] + x.y;
        z[4 * i + 2] = z[4 * i + 2] + x.z;
        z[4 * i + 3] = z[4 * i + 3] + x.w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < RU_E; ++i) z[i] = z[i] + 0.f;
    }
  }
  if (temp > 0.f && temp != 1.f) divide<RU_E>(z, temp, 1.f / temp, z);
  if (masked) {
    // (after the division, which infinities would slow down)
    const float none = temp > 0.f ? -INFINITY / temp : -INFINITY;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < VEC; ++j)
        if (!(words[i] >> j & 1)) z[i * VEC + j] = none;
  }
  if (a.out) {
    float* dst = a.out + (int64_t)row * a.out_ld + v0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int u = (i * RU_NT + tid) * VEC;
      if (v0 + u + VEC <= V) {
#pragma unroll
        for (int j = 0; j < VEC; j += 4) {
          const f32x4u x = {z[i * VEC + j], z[i * VEC + j + 1], z[i * VEC + j + 2], z[i * VEC + j + 3]};
          *(f32x4u*)(dst + u + j) = x;
        }
      } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j)
          if (v0 + u + j < V) dst[u + j] = z[i * VEC + j];
      }
    }
  }
  if (a.k == 0) return false;
  // past the vocabulary: -inf, whatever the rules made of it
  if (v0 + RU_CHUNK > V) {
#pragma unroll
    for (int i = 0; i < RU_E; ++i)
      if (v0 + ((i / VEC) * RU_NT + tid) * VEC + i % VEC >= V) z[i] = -INFINITY;
  }

  float largest = z[0];
#pragma unroll
  for (int i = 1; i < RU_E; ++i) largest = fmaxf(largest, z[i]);
  const float mx = wave_max_lanes(largest);
  const float ref = mx == -INFINITY ? 0.f : mx;
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < RU_E; ++i) sum += __builtin_amdgcn_exp2f((z[i] - ref) * 1.4426950408889634f);
  sum = wave_sum_lanes(sum);
  if (lane == 0) {
    wave_ms[wave][0] = mx;
    wave_ms[wave][1] = sum;
  }

  // the wave's candidates, its k best among them: what is not below the floor
  const auto token_of = [&](int i) { return v0 + ((i / VEC) * RU_NT + tid) * VEC + i % VEC; };
  int n = RU_CAND + 1;
  uint32_t least_rank = 0;
  if (sum == sum) {                                    // (a NaN or +inf would not compare: the other way)
    least_rank = max(a.k == 1 ? rank_of(mx) : rank_floor(rank_of(largest), a.k), kLowest);
    const float least = from_ordered_u32(least_rank);
    n = 0;
#pragma unroll
    for (int i = 0; i < RU_E; ++i) {
      const uint64_t in = __ballot(z[i] >= least);
      if (!in) continue;
      const int at = n + __builtin_amdgcn_mbcnt_hi((uint32_t)(in >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)in, 0));
      if (z[i] >= least && at < RU_CAND) cand[wave][at] = result_of(rank_of(z[i]), token_of(i));
      n += __popcll(in);
    }
  }
  if (n > RU_CAND) {
    least_rank = 0;
    // many equal ones: k rounds, each lane offering the best that it has not yet given
    uint32_t given = 0;
    for (n = 0; n < a.k; ++n) {
      uint32_t r = 0;
      int tok = 0;
#pragma unroll
      for (int i = 0; i < RU_E; ++i) {
        const uint32_t x = given >> i & 1 ? 0u : rank_of(z[i]);
        if (x > r) {
          r = x;
          tok = i;
        }
      }
      const int l = best_lane(r, token_of(tok));
      if (l < 0) break;
      if (lane == l) {
        cand[wave][n] = result_of(r, token_of(tok));
        given |= 1u << tok;
      }
    }
  }
  if (lane == 0) {
    cand_n[wave] = n;
    cand_least[wave] = least_rank;
  }
  __syncthreads();
  if (v0 >= V) return true;
  // the 256 threads': a candidate's place is the number of better ones, and none
  // below the highest floor of their waves has a place below k
  const int chunk = blockIdx.x * SUBS + sub, w0 = wave & ~3;
  uint64_t* keys = (uint64_t*)(a.ws + (int64_t)a.rows * chunks * 2) + ((int64_t)row * chunks + chunk) * a.k;
  int m[4], have = 0;
  uint32_t least = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    have += m[w] = __builtin_amdgcn_readfirstlane(cand_n[w0 + w]);
    least = max(least, (uint32_t)__builtin_amdgcn_readfirstlane(cand_least[w0 + w]));
  }
  const auto above = [&](uint64_t x) { return __ballot(x && (uint32_t)(x >> 32) >= least); };
  if (have <= 64) {                                    // one wave, a candidate a lane
    if (wave == w0) {
      const int w = (lane >= m[0]) + (lane >= m[0] + m[1]) + (lane >= m[0] + m[1] + m[2]);
      const int at = lane - (w > 0 ? m[0] : 0) - (w > 1 ? m[1] : 0) - (w > 2 ? m[2] : 0);
      const uint64_t mine = lane < have ? cand[w0 + w][at] : 0;
      const int place = better(mine, above(mine), mine);
      if (lane < have && place < a.k) leave(a, keys + place, mine);
    }
  } else {
    const uint64_t mine = lane < n ? cand[wave][lane] : 0;
    int place = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const uint64_t x = lane < m[w] ? cand[w0 + w][lane] : 0;
      place += better(x, above(x), mine);
    }
    if (lane < n && place < a.k) leave(a, keys + place, mine);
  }
  if (wave == w0) {
    if (lane >= have && lane < a.k) leave(a, keys + lane, 0);
    if (lane == 0) {
      float M = wave_ms[w0][0], S = 0.f;
#pragma unroll
      for (int w = 1; w < 4; ++w) M = fmaxf(M, wave_ms[w0 + w][0]);
#pragma unroll
      for (int w = 0; w < 4; ++w)
        S += wave_ms[w0 + w][0] == M
                 ? wave_ms[w0 + w][1]
                 : wave_ms[w0 + w][1] * __builtin_amdgcn_exp2f((wave_ms[w0 + w][0] - M) * 1.4426950408889634f);
      leave(a, (uint64_t*)a.ws + (int64_t)row * chunks + chunk, (uint64_t)__float_as_uint(S) << 32 | __float_as_uint(M));
    }
  }
  return true;
}

// A row's blocks joined, one wave a row, in the same way: a floor under the k
// best, the few above it, the place of each.
// rules_lds: the lists, then RU_CAND candidates (one wave: its LDS accesses keep
// their order).
__device__ __forceinline__ void join_row(const RulesLaunch& a, int chunks, int row, int lane, uint64_t* rules_lds) {
  constexpr int LISTS = kRulesMaxVocab / RU_CHUNK / 64;
  const int n = chunks * a.k;
  const uint64_t* keys = (const uint64_t*)(a.ws + (int64_t)a.rows * chunks * 2) + (int64_t)row * n;
  const uint64_t* ms = (const uint64_t*)a.ws + (int64_t)row * chunks;
  float m[LISTS], s[LISTS], M = -INFINITY;
#pragma unroll
  for (int i = 0; i < LISTS; ++i) {
    const int c = lane + 64 * i;
    m[i] = -INFINITY;
    s[i] = 0.f;
    if (c < chunks) {
      const uint64_t x = left_by(a, ms + c);
      m[i] = __uint_as_float((uint32_t)x);
      s[i] = __uint_as_float((uint32_t)(x >> 32));
    }
    M = fmaxf(M, m[i]);
  }
  uint32_t largest = 0;
  for (int i0 = 0; i0 < n; i0 += 4 * 64) {
    uint64_t x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = i0 + 64 * i + lane < n ? left_by(a, keys + i0 + 64 * i + lane) : 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      largest = max(largest, (uint32_t)(x[i] >> 32));
      if (i0 + 64 * i + lane < n) rules_lds[i0 + 64 * i + lane] = x[i];
    }
  }
  M = wave_max_lanes(M);
  float S = 0.f;
#pragma unroll
  for (int i = 0; i < LISTS; ++i)
    S += m[i] == M ? s[i] : s[i] * __builtin_amdgcn_exp2f((m[i] - M) * 1.4426950408889634f);
  // logprob = (z - M) - log sum_v e^{z - M}: with M in it (z minus M + log sum) the
  // result would be off by half a step of M, all there is of a near-certain token's
  const float log_sum = logf(wave_sum_lanes(S));
  wave_lds_done();
  auto put = [&](int place, uint64_t x) {
    const uint32_t r = (uint32_t)(x >> 32);
    const float z = r == 0xffffffffu ? NAN : from_ordered_u32(r);
    a.token[(int64_t)row * a.k + place] = x ? (int)~(uint32_t)x : -1;
    a.logprob[(int64_t)row * a.k + place] = x ? (z - M) - log_sum : -INFINITY;
  };
  uint64_t* cand = rules_lds + n;
  const uint32_t least = rank_floor(largest, a.k);
  int have = 0;
  for (int i0 = 0; i0 < n; i0 += 64) {
    const uint64_t x = i0 + lane < n ? rules_lds[i0 + lane] : 0;
    const uint64_t in = __ballot((uint32_t)(x >> 32) >= least);
    const int at = have + __builtin_amdgcn_mbcnt_hi((uint32_t)(in >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)in, 0));
    if ((uint32_t)(x >> 32) >= least && at < RU_CAND) cand[at] = x;
    have += __popcll(in);
  }
  wave_lds_done();
  if (have <= RU_CAND) {
    const uint64_t mine = lane < have ? cand[lane] : 0;
    const int place = better(mine, __ballot(lane < have), mine);
    if (lane < have && place < a.k) put(place, mine);
    if (lane >= have && lane < a.k) put(lane, 0);
    return;
  }
  // many equal ones: lane l goes down the sorted lists of blocks l, l + 64, ...
  int at[LISTS];
#pragma unroll
  for (int i = 0; i < LISTS; ++i) at[i] = 0;
  for (int i = 0; i < a.k; ++i) {
    uint64_t x = 0;
    int from = 0;
#pragma unroll
    for (int j = 0; j < LISTS; ++j) {
      const int c = lane + 64 * j;
      if (c >= chunks || at[j] >= a.k) continue;
      const uint64_t y = rules_lds[c * a.k + at[j]];
      if (y > x) {
        x = y;
        from = j;
      }
    }
    const int l = best_lane((uint32_t)(x >> 32), (int)~(uint32_t)x);
    if (l < 0) {
      if (lane == 0) put(i, 0);
    } else if (lane == l) {
      put(i, x);
#pragma unroll
      for (int j = 0; j < LISTS; ++j) at[j] += j == from;
    }
  }
}

// (JOINED by itself: it takes registers that a full GPU would miss)
template <typename T, bool JOINED>
__global__ __launch_bounds__(RU_NT) void k_rules(RulesLaunch a, int chunks) {
  const bool some = rules_block<T, 1>(a, chunks);
  if constexpr (JOINED) {
    extern __shared__ __attribute__((aligned(16))) uint32_t table[];
    const int row = blockIdx.y;
    if (some && arrive_last(a.counters + row, gridDim.x) && threadIdx.x < 64)
      join_row(a, chunks, row, threadIdx.x, (uint64_t*)table);
  }
}
// (two of these blocks fit a CU only with at most 64 vector and 80 scalar
// registers a wave: 256 rows of 131071, 32768 tokens of history 151 -> 110 us)
template <typename T>
__global__ __launch_bounds__(RU_LONG * RU_NT) __attribute__((amdgpu_waves_per_eu(8), amdgpu_num_sgpr(80)))
void k_rules_long(RulesLaunch a, int chunks) {
  rules_block<T, RU_LONG>(a, chunks);
}

__global__ __launch_bounds__(64) void k_rules_join(RulesLaunch a, int chunks) {
  extern __shared__ uint64_t rules_lds[];
  join_row(a, chunks, blockIdx.x, threadIdx.x, rules_lds);
}

template <typename T>
void rules(const RulesLaunch& a, hipStream_t s) {
  const int chunks = (a.vocab + RU_CHUNK - 1) / RU_CHUNK;
  const bool lists = a.history || a.bias_token;
  const size_t join_lds = a.k > 0 ? ((size_t)chunks * a.k + RU_CAND) * sizeof(uint64_t) : 0;
  if (a.history_ld >= kLongHistory) {
    static_assert(RU_LONG * RU_CHUNK * 4 <= 65536, "dynamic LDS without asking");
    k_rules_long<T><<<dim3((chunks + RU_LONG - 1) / RU_LONG, a.rows), RU_LONG * RU_NT,
                      lists ? RU_LONG * RU_CHUNK * 4 : 0, s>>>(a, chunks);
    if (a.k > 0) k_rules_join<<<a.rows, 64, join_lds, s>>>(a, chunks);
  } else {
    const size_t lds = lists ? RU_CHUNK * 4 : 0;
    if (a.counters)
      k_rules<T, true><<<dim3(chunks, a.rows), RU_NT, std::max(lds, join_lds), s>>>(a, chunks);
    else
      k_rules<T, false><<<dim3(chunks, a.rows), RU_NT, lds, s>>>(a, chunks);
    if (a.k > 0 && !a.counters) k_rules_join<<<a.rows, 64, join_lds, s>>>(a, chunks);
  }
}

__global__ __launch_bounds__(64) void k_note_rows(SlotRuleArrays a, const int32_t* slots, const int32_t* tokens,
                                                  const int32_t* pos, const int32_t* scalars, int D) {
  const int i = blockIdx.x * 64 + threadIdx.x;
  if (i >= D) return;
  const int slot = slots[i], p = pos[i];
  a.history[(int64_t)slot * kTextCtx + p] = tokens[i];
  a.history_len[slot] = p + 1;
  a.prompt_len[slot] = scalars[i];
  a.mask_of[slot] = scalars[D + i];
  a.bias_len[slot] = scalars[2 * D + i];
  a.repetition[slot] = __int_as_float(scalars[3 * D + i]);
  a.frequency[slot] = __int_as_float(scalars[4 * D + i]);
  a.presence[slot] = __int_as_float(scalars[5 * D + i]);
  a.temperature[slot] = __int_as_float(scalars[6 * D + i]);
}

}  // namespace

void note_rows(const SlotRuleArrays& a, const int32_t* slots, const int32_t* tokens, const int32_t* pos,
               const int32_t* scalars, int D, hipStream_t s) {
  if (D > 0) k_note_rows<<<(D + 63) / 64, 64, 0, s>>>(a, slots, tokens, pos, scalars, D);
}

size_t rules_ws_bytes(int rows, int vocab, int k) {
  const size_t chunks = (vocab + RU_CHUNK - 1) / RU_CHUNK;
  return k > 0 ? (size_t)rows * chunks * (1 + k) * 8 : 0;
}

void logit_rules(const RulesLaunch& a, bool bf16, hipStream_t s) {
  if (a.rows <= 0) return;
  if (bf16)
    rules<bf16_t>(a, s);
  else
    rules<float>(a, s);
}

}  // namespace asr
