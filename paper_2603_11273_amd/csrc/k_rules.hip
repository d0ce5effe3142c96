// Rules on logits and the k best tokens (asr_logit_rules): penalties for
// repeated tokens, biases, masks of allowed tokens and a temperature, and the
// log-probabilities of the best tokens under what remains.
//
// One pass over the logits.  A block takes 4096 tokens of a row, 16 a thread, in
// registers.  What is sparse -- the row's history, its biases -- is scattered into
// an LDS table of the block's tokens (every block of a row reads the whole
// lists, a few KB) and read back by the threads that own the tokens, so nothing
// of the vocabulary's size is cleared, written or read besides the logits
// themselves.  The block leaves its maximum, its sum of exponentials and its k
// best tokens; a second, short kernel joins a row's blocks.  HBM bounds a batch
// of rows, two launches a single one.
#include "asr_device.h"

// Every operation below is rounded by itself, as the definition has it: two
// logits that it makes equal stay equal.
#pragma clang fp contract(off)

namespace asr {
namespace {

constexpr int RU_NT = 256, RU_E = 16, RU_CHUNK = RU_NT * RU_E;
static_assert(RU_CHUNK == kRulesChunk, "workspace");
constexpr uint32_t kSeen = 0x80000000u;     // in the history; below it the count behind the prompt

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
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

template <typename T>
__global__ __launch_bounds__(RU_NT) void k_rules(RulesLaunch a) {
  constexpr int VEC = Logits<T>::VEC, NV = RU_E / VEC;
  __shared__ __attribute__((aligned(16))) uint32_t count[RU_CHUNK];
  __shared__ __attribute__((aligned(16))) float bias[RU_CHUNK];
  __shared__ uint2 best[4][kRulesMaxK];
  __shared__ float wave_ms[4][2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int chunk = blockIdx.x, row = blockIdx.y, v0 = chunk * RU_CHUNK;
  const int V = a.vocab;
  const T* src = (const T*)a.logits + (int64_t)row * a.ld + v0;

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

  int set = a.set ? a.set[row] : row;
  const bool ruled = set >= 0 && set < a.sets;
  if (!ruled) set = 0;
  const int hist_n = ruled && a.history ? (int)min((int64_t)max(a.history_len[set], 0), a.history_ld) : 0;
  const int bias_n = ruled && a.bias_token ? (int)min((int64_t)max(a.bias_len[set], 0), a.bias_ld) : 0;
  const int mask_row = ruled && a.mask ? (a.mask_of ? a.mask_of[set] : set) : -1;
  if (hist_n > 0 || bias_n > 0) {                      // block-uniform
#pragma unroll
    for (int i = 0; i < RU_E / 4; ++i) {
      *(uint4*)(count + (i * RU_NT + tid) * 4) = uint4{0u, 0u, 0u, 0u};
      *(float4*)(bias + (i * RU_NT + tid) * 4) = float4{0.f, 0.f, 0.f, 0.f};
    }
    __syncthreads();
    const int32_t* hist = a.history + (int64_t)set * a.history_ld;
    const int prompt = a.prompt_len ? a.prompt_len[set] : 0;
    for (int j0 = tid; j0 < hist_n; j0 += 8 * RU_NT) {
      int tok[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) tok[i] = j0 + i * RU_NT < hist_n ? hist[j0 + i * RU_NT] : -1;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t u = (uint32_t)tok[i] - (uint32_t)v0;
        if (tok[i] < 0 || u >= RU_CHUNK) continue;
        if (j0 + i * RU_NT < prompt)
          atomicOr(&count[u], kSeen);
        else
          atomicAdd(&count[u], 1u);
      }
    }
    // the biases in the order of their list, so that a token given twice has
    // one sum: a wave takes the tokens that are its number modulo 4, one after
    // the other
    const int32_t* bt = a.bias_token + (int64_t)set * a.bias_ld;
    const float* bv = a.bias_value + (int64_t)set * a.bias_ld;
    for (int j0 = 0; j0 < bias_n; j0 += 64) {
      const bool in = j0 + lane < bias_n;
      const int tok = in ? bt[j0 + lane] : -1;
      const float val = in ? bv[j0 + lane] : 0.f;
      const uint32_t u = (uint32_t)tok - (uint32_t)v0;
      uint64_t hit = __ballot(tok >= 0 && u < RU_CHUNK && (tok & 3) == wave);
      while (hit) {
        const int l = __ffsll((unsigned long long)hit) - 1;
        hit &= hit - 1;
        const uint32_t ul = __builtin_amdgcn_readlane(u, l);
        const float vl = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(val), l));
        if (lane == 0) bias[ul] += vl;
      }
    }
    __syncthreads();
    const float rep = a.repetition ? a.repetition[set] : 1.f;
    const float freq = a.frequency ? a.frequency[set] : 0.f;
    const float pres = a.presence ? a.presence[set] : 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const int u = (i * RU_NT + tid) * VEC + j;
        const uint32_t c = count[u];
        float x = z[i * VEC + j];
        if (c) {
          x = x > 0.f ? x / rep : x * rep;
          const uint32_t times = c & ~kSeen;
          if (times) x = (x - freq * (float)times) - pres;
        }
        if (bias_n > 0) x = x + bias[u];
        z[i * VEC + j] = x;
      }
    }
  }
  if (mask_row >= 0 && mask_row < a.masks) {
    const uint32_t* words = a.mask + (int64_t)mask_row * a.mask_ld;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int v = v0 + (i * RU_NT + tid) * VEC;      // VEC tokens lie in one word
      const uint32_t w = v < V ? words[v >> 5] >> (v & 31) : 0u;
#pragma unroll
      for (int j = 0; j < VEC; ++j)
        if (!(w >> j & 1)) z[i * VEC + j] = -INFINITY;
    }
  }
  if (ruled && a.temperature) {
    const float t = a.temperature[set];
    if (t > 0.f && t != 1.f) {
#pragma unroll
      for (int i = 0; i < RU_E; ++i) z[i] = z[i] / t;
    }
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
  if (a.k == 0) return;
  // past the vocabulary: -inf, whatever the rules made of it
  if (v0 + RU_CHUNK > V) {
#pragma unroll
    for (int i = 0; i < RU_E; ++i)
      if (v0 + ((i / VEC) * RU_NT + tid) * VEC + i % VEC >= V) z[i] = -INFINITY;
  }

  float mx = z[0];
#pragma unroll
  for (int i = 1; i < RU_E; ++i) mx = fmaxf(mx, z[i]);
  mx = wave_max_lanes(mx);
  const float ref = mx == -INFINITY ? 0.f : mx;
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < RU_E; ++i) sum += __builtin_amdgcn_exp2f((z[i] - ref) * 1.4426950408889634f);
  sum = wave_sum_lanes(sum);
  if (lane == 0) {
    wave_ms[wave][0] = mx;
    wave_ms[wave][1] = sum;
  }

  // the wave's k best: each lane offers the best that it has not yet given
  uint32_t given = 0;
  uint32_t rank = 0;
  int token = 0;
  auto offer = [&]() {
    rank = 0;
    token = 0;
#pragma unroll
    for (int i = 0; i < RU_E; ++i) {
      const uint32_t r = given >> i & 1 ? 0u : rank_of(z[i]);
      if (r > rank) {
        rank = r;
        token = i;
      }
    }
    token = v0 + ((token / VEC) * RU_NT + tid) * VEC + token % VEC;
  };
  offer();
  for (int i = 0; i < a.k; ++i) {
    const int l = best_lane(rank, token);
    if (l < 0) {
      if (lane == 0) best[wave][i] = uint2{0u, 0u};
      continue;
    }
    if (lane == l) {
      best[wave][i] = uint2{rank, (uint32_t)token};
      const int u = token - v0;
      given |= 1u << (u / (RU_NT * VEC) * VEC + u % VEC);
      offer();
    }
  }
  __syncthreads();
  if (wave != 0) return;
  // the block's: a token's place is the number of better ones
  uint2* keys = (uint2*)(a.ws + (int64_t)a.rows * gridDim.x * 2) + ((int64_t)row * gridDim.x + chunk) * a.k;
  const int n = 4 * a.k;
  uint2 mine = {0u, 0u};
  if (lane < n) mine = best[lane / a.k][lane % a.k];
  int place = 0, have = 0;
  for (int i = 0; i < n; ++i) {
    const uint32_t r = __builtin_amdgcn_readlane(mine.x, i), t = __builtin_amdgcn_readlane(mine.y, i);
    place += r > mine.x || (r == mine.x && t < mine.y);
    have += r != 0;
  }
  if (mine.x != 0 && place < a.k) keys[place] = mine;
  if (lane >= have && lane < a.k) keys[lane] = uint2{0u, 0u};
  if (lane == 0) {
    float M = wave_ms[0][0], S = 0.f;
#pragma unroll
    for (int w = 1; w < 4; ++w) M = fmaxf(M, wave_ms[w][0]);
#pragma unroll
    for (int w = 0; w < 4; ++w)
      S += wave_ms[w][0] == M ? wave_ms[w][1]
                              : wave_ms[w][1] * __builtin_amdgcn_exp2f((wave_ms[w][0] - M) * 1.4426950408889634f);
    *((float2*)a.ws + (int64_t)row * gridDim.x + chunk) = float2{M, S};
  }
}

// A row's blocks joined, one wave a row: lane l goes down the sorted lists of
// blocks l, l + 64, ...
__global__ __launch_bounds__(64) void k_rules_join(RulesLaunch a, int chunks) {
  constexpr int LISTS = kRulesMaxVocab / RU_CHUNK / 64;
  extern __shared__ uint2 rules_lds[];
  const int row = blockIdx.x, lane = threadIdx.x, n = chunks * a.k;
  const uint2* keys = (const uint2*)(a.ws + (int64_t)a.rows * chunks * 2) + (int64_t)row * n;
  const float2* ms = (const float2*)a.ws + (int64_t)row * chunks;
  float m[LISTS], s[LISTS], M = -INFINITY;
#pragma unroll
  for (int i = 0; i < LISTS; ++i) {
    const int c = lane + 64 * i;
    const float2 x = c < chunks ? ms[c] : float2{-INFINITY, 0.f};
    m[i] = x.x;
    s[i] = x.y;
    M = fmaxf(M, x.x);
  }
  for (int i = lane; i < n; i += 64) rules_lds[i] = keys[i];
  M = wave_max_lanes(M);
  float S = 0.f;
#pragma unroll
  for (int i = 0; i < LISTS; ++i)
    S += m[i] == M ? s[i] : s[i] * __builtin_amdgcn_exp2f((m[i] - M) * 1.4426950408889634f);
  const float log_sum = logf(wave_sum_lanes(S));
  __syncthreads();
  int at[LISTS];
#pragma unroll
  for (int i = 0; i < LISTS; ++i) at[i] = 0;
  uint32_t rank = 0;
  int token = 0, from = 0;
  auto offer = [&]() {
    rank = 0;
#pragma unroll
    for (int i = 0; i < LISTS; ++i) {
      const int c = lane + 64 * i;
      if (c >= chunks || at[i] >= a.k) continue;
      const uint2 x = rules_lds[c * a.k + at[i]];
      if (x.x > rank) {                                // (equal: the lower chunk has the lower tokens)
        rank = x.x;
        token = (int)x.y;
        from = i;
      }
    }
  };
  offer();
  for (int i = 0; i < a.k; ++i) {
    const int l = best_lane(rank, token);
    if (l < 0) {
      if (lane == 0) {
        a.token[(int64_t)row * a.k + i] = -1;
        a.logprob[(int64_t)row * a.k + i] = -INFINITY;
      }
    } else if (lane == l) {
      const float z = rank == 0xffffffffu ? NAN : from_ordered_u32(rank);
      a.token[(int64_t)row * a.k + i] = token;
      a.logprob[(int64_t)row * a.k + i] = (z - M) - log_sum;
#pragma unroll
      for (int j = 0; j < LISTS; ++j) at[j] += j == from;
      offer();
    }
  }
}

}  // namespace

size_t rules_ws_bytes(int rows, int vocab, int k) {
  const size_t chunks = (vocab + RU_CHUNK - 1) / RU_CHUNK;
  return k > 0 ? (size_t)rows * chunks * (1 + k) * 8 : 0;
}

void logit_rules(const RulesLaunch& a, bool bf16, hipStream_t s) {
  if (a.rows <= 0) return;
  const int chunks = (a.vocab + RU_CHUNK - 1) / RU_CHUNK;
  if (bf16)
    k_rules<bf16_t><<<dim3(chunks, a.rows), RU_NT, 0, s>>>(a);
  else
    k_rules<float><<<dim3(chunks, a.rows), RU_NT, 0, s>>>(a);
  if (a.k > 0) k_rules_join<<<a.rows, 64, (size_t)chunks * a.k * sizeof(uint2), s>>>(a, chunks);
}

}  // namespace asr
