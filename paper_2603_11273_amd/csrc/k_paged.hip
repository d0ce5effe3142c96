// Attention of new tokens over the pages of their sequence (asr_attend_pages).
//
// The codes are the traffic: 128 bytes a key and head for 4 * 64 operations a
// query.  A block takes a part of the keys of one (sequence, cache head) and up
// to 32 of the sequence's queries; its four waves take the part's blocks of 64 keys
// in turn, each with a running maximum, sum and weighted values of its own, joined
// through LDS at the end; the parts of a row are joined from (max, sum, values)
// records by the last of its blocks or a second kernel, or not at all where there is one
// part.
//
// Codes go from memory to the matrix instructions without LDS.  With lane = 16 g + m,
// four score tiles S^T = K Q^T of 16 keys are loaded so that they leave lane (m, g) with
// query m's scores of keys 16 g .. 16 g + 15 of the 64; the second product O^T = V^T
// P^T takes exactly those from that lane, and of V^T, which lies [dim][position] in the
// pool, 16 bytes of one dim: no permutes.  Row m of product t is dim 4 m + t,
// which leaves the lane with 16 consecutive dims of its query.  An instruction turns
// two codes into bf16, exactly; the block's scales multiply scores and probabilities.
#include "asr_device.h"

namespace asr {
namespace {

constexpr int PA_NW = 4;                 // waves of a block
constexpr int PA_OLD = 68;               // floats a query's row takes in LDS: 16 lanes, 64 banks
constexpr float kRaise = 8.f;            // the reference follows the maximum from 2^8 on

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint4 load_once(const uint8_t* p) {
  return __builtin_bit_cast(uint4, __builtin_nontemporal_load((const u32x4*)p));
}

struct PagedArgs {
  PagedLaunch c;
  int per, tiles;
  uint32_t units;
};

// Eight codes as bf16.
__device__ __forceinline__ bf16x8 values8(uint32_t a, uint32_t b) {
  const uint4 u = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, true)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, true))};
  return __builtin_bit_cast(bf16x8, u);
}

// Floats as sums of bf16 for the matrix instructions: a pair where the result is
// bf16 (one bf16 alone would move a score of 20 by 0.04, the pair by 2e-4), three,
// which is all of them, where it is float32.  A pair is off by up to 2^-17 of the number
// where its first is rounded (queries), 2^-16 where it is cut (weights): against products in
// float32 one result of 150 to 200 comes out a bf16 step apart, as far from 64 bits as the other.
template <typename T>
constexpr int kTerms = sizeof(T) == 2 ? 2 : 3;
template <int N>
struct Terms {
  bf16x8 x[N];
  // rounded terms of y
  __device__ __forceinline__ void round(const float* y) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float r = y[i];
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const __bf16 h = (__bf16)r;
        x[n][i] = h;
        r -= (float)h;
      }
    }
  }
  // the first terms cut off, not rounded: a byte permute for two
  __device__ __forceinline__ void cut(const float* y) {
    uint4 u[N];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float a = y[2 * i], b = y[2 * i + 1];
#pragma unroll
      for (int n = 0; n < N - 1; ++n) {
        ((uint32_t*)&u[n])[i] = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302);
        a -= __uint_as_float(__float_as_uint(a) & 0xffff0000u);
        b -= __uint_as_float(__float_as_uint(b) & 0xffff0000u);
      }
      ((uint32_t*)&u[N - 1])[i] = pack2_bf16(a, b);
    }
#pragma unroll
    for (int n = 0; n < N; ++n) x[n] = __builtin_bit_cast(bf16x8, u[n]);
  }
  __device__ __forceinline__ f32x4 product(bf16x8 a, f32x4 c) const {
#pragma unroll
    for (int n = N - 1; n >= 0; --n) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, x[n], c, 0, 0, 0);
    return c;
  }
};

// Reduction over the four lanes that share lane % 16.
__device__ __forceinline__ float lanes16_max(float v) {
  const uint32_t u = __float_as_uint(v);
  const auto p16 = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  v = fmaxf(__uint_as_float(p16[0]), __uint_as_float(p16[1]));
  const uint32_t w = __float_as_uint(v);
  const auto p32 = __builtin_amdgcn_permlane32_swap(w, w, false, false);
  return fmaxf(__uint_as_float(p32[0]), __uint_as_float(p32[1]));
}
__device__ __forceinline__ float lanes16_sum(float v) {
  const uint32_t u = __float_as_uint(v);
  const auto p16 = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  v = __uint_as_float(p16[0]) + __uint_as_float(p16[1]);
  const uint32_t w = __float_as_uint(v);
  const auto p32 = __builtin_amdgcn_permlane32_swap(w, w, false, false);
  return __uint_as_float(p32[0]) + __uint_as_float(p32[1]);
}

// Rows of a sequence: [start, start + count).  A start behind the rows (a padded list's, up
// to 2^31 - 1) has none: count stays in [0, max_rows], so that its product with the queries
// of a row holds in 32 bits.
__device__ __forceinline__ void rows_of(const PagedLaunch& c, int seq, int* start, int* count) {
  const int s = c.row_start ? c.row_start[seq] : seq, e = c.row_start ? c.row_start[seq + 1] : seq + 1;
  *start = s;
  *count = s < 0 || s >= c.rows ? 0 : min(min(max(e, s), c.rows) - s, c.max_rows);
}

// (max, sum) of part `part` of a row and head; a sum of 0 says that the part has no
// key (and no values).
__device__ __forceinline__ float2* record(const PagedLaunch& c, int row, int h, int part) {
  return (float2*)(c.rec + (int64_t)c.rows * c.n_head * c.parts * kHeadDim) + ((int64_t)row * c.n_head + h) * c.parts + part;
}

// The bytes of 16 keys from `key` on that lie in [lo, hi).
__device__ __forceinline__ void keep_keys(uint4* v, int key, int lo, int hi) {
  uint32_t* w = (uint32_t*)v;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t mask = 0;
#pragma unroll
    for (int b = 0; b < 4; ++b)
      if (key + 4 * i + b >= lo && key + 4 * i + b < hi) mask |= 0xffu << (8 * b);
    w[i] &= mask;
  }
}
// 0x80 in every byte that is a NaN code.
__device__ __forceinline__ uint32_t nan_codes(uint32_t c) { return ((c & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

// out of a row and head from its parts' records, a wave's work, lane = dim: a chain of
// loads, so all it needs is loaded at once, PA_JOIN records at a time; which of them hold
// anything they say themselves.  HERE: records of the same launch.
constexpr int PA_JOIN = 16;
template <typename T, bool HERE>
struct Join {
  const float* val;
  const float2* ml;
  int parts, lane;
  float v[PA_JOIN];
  float2 rec;
  __device__ __forceinline__ Join(const PagedLaunch& c, int row, int h)
      : val(c.rec + ((int64_t)row * c.n_head + h) * c.parts * kHeadDim + (threadIdx.x & 63)), ml(record(c, row, h, 0)),
        parts(c.parts), lane(threadIdx.x & 63) {
    load(0);
  }
  __device__ __forceinline__ void load(int p0) {
    rec = float2{-INFINITY, 0.f};
    if (lane < PA_JOIN && p0 + lane < parts)
      rec = HERE ? __builtin_bit_cast(float2, load_agent((const uint64_t*)&ml[p0 + lane])) : ml[p0 + lane];
#pragma unroll
    for (int p = 0; p < PA_JOIN; ++p) {
      const float* x = val + (int64_t)(p0 + p) * kHeadDim;
      v[p] = p0 + p >= parts ? 0.f : HERE ? load_agent(x) : *x;
    }
  }
  __device__ __forceinline__ void store(const PagedLaunch& c, int row, int h) {
    float M = -INFINITY, L = 0.f, acc = 0.f;
    for (int p0 = 0; p0 < parts; p0 += PA_JOIN) {
      if (p0 > 0) load(p0);
      const bool there = !(rec.y == 0.f);
      const uint64_t some = __ballot(there);
      if (!some) continue;
      const float top = fmaxf(M, wave_max_lanes(there ? rec.x : -INFINITY));
      const float keep = M == top ? 1.f : __builtin_amdgcn_exp2f(M - top);
      const float fac = !there ? 0.f : rec.x == top ? 1.f : __builtin_amdgcn_exp2f(rec.x - top);
      M = top;
      L = L * keep + wave_sum_lanes(there ? fac * rec.y : 0.f);
      acc *= keep;
#pragma unroll
      for (int j = 0; j < PA_JOIN; ++j)
        if (some >> j & 1) acc += __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(fac), j)) * v[j];
    }
    St<T>::st((T*)c.out, row * c.out_ld + h * kHeadDim + lane, L == 0.f ? 0.f : acc / L);
  }
};

template <typename T, int QT>
__global__ __launch_bounds__(PA_NW * 64) __attribute__((amdgpu_waves_per_eu(QT == 1 ? 3 : 2)))
void k_attend_pages(PagedArgs a) {
  extern __shared__ __attribute__((aligned(16))) float paged_lds[];
  constexpr int N = kTerms<T>;
  uint32_t u = blockIdx.x;
  const int ctile = (int)((u >> 3) % a.tiles), col0 = ctile * 16 * QT;
  u = (u >> 3) / a.tiles * 8 + (u & 7);
  if (u >= a.units) return;
  const int head = (int)(u % a.c.c.kv_heads);
  u /= a.c.c.kv_heads;
  const int seq = (int)(u % a.c.c.sequences), part = (int)(u / a.c.c.sequences);
  int start, count;
  rows_of(a.c, seq, &start, &count);
  if (col0 >= count * a.per) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int m = lane & 15, g = lane >> 4;
  int k0 = part * a.c.part;
  int bound = (int)min((int64_t)k0 + a.c.part, (int64_t)a.c.max_keys);
  if (a.c.even) {
    // equal parts of what the tile's queries see
    int lo = INT32_MAX, hi = 0;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const int j = (col0 + 16 * t + m) / a.per;
      if (j >= count) continue;
      const int f = max(a.c.first[start + j], 0), e = min(a.c.length[start + j], a.c.max_keys);
      if (f < e) lo = min(lo, f), hi = max(hi, e);
    }
    lo = (int)~wave_max_u32(~(uint32_t)lo) & -kPageBlock;
    hi = (int)wave_max_u32((uint32_t)hi);
    const int n = max(((hi - lo + a.c.parts - 1) / a.c.parts + kPageBlock - 1) / kPageBlock, PA_NW) * kPageBlock;
    k0 = hi > lo ? (int)min((int64_t)lo + (int64_t)part * n, (int64_t)hi & -kPageBlock) : 0;
    bound = hi > lo ? (int)min((int64_t)lo + (int64_t)(part + 1) * n, (int64_t)hi) : 0;
    if (hi > lo && (int64_t)lo + (int64_t)part * n >= hi) bound = k0;       // (nothing left for it)
    k0 = __builtin_amdgcn_readfirstlane(k0);
    bound = __builtin_amdgcn_readfirstlane(bound);
  }

  // the wave's blocks of keys: lane i knows the i-th's page
  const int per = a.c.c.page / kPageBlock;
  const int mine = k0 / kPageBlock + wave + PA_NW * lane;
  int page = -1;
  if (mine * kPageBlock < bound) page = a.c.c.table[(int64_t)seq * a.c.c.table_ld + mine / per];

  // the keys that each column sees, and those that some column does
  int first[QT], end[QT], row[QT];
  int lo = INT32_MAX, hi = 0, all_lo = 0, all_hi = INT32_MAX;
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int j = (col0 + 16 * t + m) / a.per;
    row[t] = j < count ? start + j : -1;
    first[t] = 0, end[t] = INT32_MAX;
    if (row[t] >= 0) {
      first[t] = a.c.first ? max(a.c.first[row[t]], 0) : 0;
      end[t] = max(min(a.c.length[row[t]], bound), 0);
      if (first[t] < end[t]) lo = min(lo, first[t]), hi = max(hi, end[t]);
      all_lo = max(all_lo, first[t]);
      all_hi = min(all_hi, end[t]);
    }
  }
  lo = (int)~wave_max_u32(~(uint32_t)lo);
  hi = (int)wave_max_u32((uint32_t)hi);
  all_lo = (int)wave_max_u32((uint32_t)all_lo);
  all_hi = (int)~wave_max_u32(~(uint32_t)all_hi);

  const bool there = page >= 0 && page < a.c.c.pages && mine * kPageBlock < hi && (mine + 1) * kPageBlock > lo;
  uint64_t todo = __ballot(there);
  const int inner = mine % per;
  float k_scale = 0.f, v_scale = 0.f;
  if (there) {
    const float* s = a.c.c.scales + page * a.c.c.scale_stride + (int64_t)head * per + inner;
    k_scale = s[0];
    v_scale = s[(int64_t)a.c.c.kv_heads * per];
  }
  const uint32_t k_off = (16 * (m >> 2) + (m & 3)) * kHeadDim + 16 * g, v_off = 4 * m * kPageBlock + 16 * g;
  const int64_t v_at = (int64_t)a.c.c.kv_heads * per * (kPageBlock * kHeadDim);
  uint4 k[4], v[4];
  const uint8_t* block;
  auto find = [&](int i) {
    const int p = __builtin_amdgcn_readlane(page, i), in = __builtin_amdgcn_readlane(inner, i);
    block = a.c.c.codes + p * a.c.c.page_stride + ((int64_t)head * per + in) * (kPageBlock * kHeadDim);
  };
  auto load_keys = [&] {
#pragma unroll
    for (int j = 0; j < 4; ++j) k[j] = load_once(block + k_off + j * 4 * kHeadDim);
  };
  auto load_values = [&] {
#pragma unroll
    for (int t = 0; t < 4; ++t) v[t] = load_once(block + v_at + v_off + t * kPageBlock);
  };
  int at = -1;                             // the block at hand, of the wave's
  auto advance = [&] {
    at = todo ? __ffsll((unsigned long long)todo) - 1 : -1;
    todo &= todo - 1;
    if (at >= 0) find(at);
  };
  advance();
  if (at >= 0) {
    load_keys();
    load_values();
  }

  Terms<N> q[QT][2];
#pragma unroll
  for (int t = 0; t < QT; ++t)
#pragma unroll
    for (int d = 0; d < 2; ++d) {
      float y[8] = {};
      if (row[t] >= 0) {
        const int h = head * a.per + (col0 + 16 * t + m) % a.per;
        const float* p = a.c.q + row[t] * a.c.q_ld + h * kHeadDim + 16 * g + 8 * d;
        const float4 x = *(const float4*)p, z = *(const float4*)(p + 4);
        const float w[8] = {x.x, x.y, x.z, x.w, z.x, z.y, z.z, z.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = w[i] * a.c.qmul;
      }
      q[t][d].round(y);
    }
  f32x4 o[QT][4];
  float mx[QT], l[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    mx[t] = -INFINITY;
    l[t] = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[t][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // The next block's keys are under way as soon as this one's have given their
  // scores, its values as soon as this one's are bf16.
  while (at >= 0) {
    const int key0 = k0 + (wave + PA_NW * at) * kPageBlock, key = key0 + 16 * g;
    const float ks = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(k_scale), at));
    float vs = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v_scale), at));
    const bool mixed = key0 < all_lo || key0 + kPageBlock > all_hi;   // some column does not see some key
    advance();
    float s[QT][16];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bf16x8 ka = values8(k[j].x, k[j].y), kb = values8(k[j].z, k[j].w);
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        f32x4 c = {0.f, 0.f, 0.f, 0.f};
        c = q[t][0].product(ka, c);
        c = q[t][1].product(kb, c);
#pragma unroll
        for (int r = 0; r < 4; ++r) s[t][4 * j + r] = c[r] * ks;
      }
    }
    if (at >= 0) load_keys();
    bool nans = false;
    if (mixed) {
#pragma unroll
      for (int t = 0; t < 4; ++t) keep_keys(&v[t], key, lo, hi);
      // a NaN among the values is for the columns that see it: kept apart
      uint32_t bad = 0;
#pragma unroll
      for (int t = 0; t < 4; ++t) bad |= nan_codes(v[t].x) | nan_codes(v[t].y) | nan_codes(v[t].z) | nan_codes(v[t].w);
      nans = __any(bad != 0);
      // (and so is a scale's, which 0 times it would spread)
      if (!(fabsf(vs) < INFINITY)) {
        vs = 1.f;
#pragma unroll
        for (int t = 0; t < QT; ++t)
          if (max(first[t], key0) < min(end[t], key0 + kPageBlock)) {
#pragma unroll
            for (int i = 0; i < 4; ++i) o[t][i] = f32x4{NAN, NAN, NAN, NAN};
          }
      }
    }
    if (nans) {
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        uint32_t* w = (uint32_t*)&v[t];
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          uint4 is;
          uint32_t* x = (uint32_t*)&is;
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint32_t b = nan_codes(w[2 * hf + i]);
            x[2 * i] = (b & 0x80u ? 0x3f80u : 0u) | (b & 0x8000u ? 0x3f800000u : 0u);
            x[2 * i + 1] = (b & 0x800000u ? 0x3f80u : 0u) | (b & 0x80000000u ? 0x3f800000u : 0u);
            w[2 * hf + i] &= ~((b >> 7) * 0xffu);
          }
#pragma unroll
          for (int c = 0; c < QT; ++c) {
            bf16x8 sees;
#pragma unroll
            for (int i = 0; i < 8; ++i)
              sees[i] = (__bf16)(key + 8 * hf + i >= first[c] && key + 8 * hf + i < end[c] ? 1.f : 0.f);
            const f32x4 n = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, is), sees, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (n[r] > 0.f) o[c][t][r] = NAN;
          }
        }
      }
    }
    bf16x8 f[4][2];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      f[t][0] = values8(v[t].x, v[t].y);
      f[t][1] = values8(v[t].z, v[t].w);
    }
    if (at >= 0) load_values();
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      if (mixed) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (key + i < first[t] || key + i >= end[t]) s[t][i] = -INFINITY;
      }
      float top = s[t][0];
#pragma unroll
      for (int i = 1; i < 16; ++i) top = fmaxf(top, s[t][i]);
      // the reference of the exponents is a query's own matter: another query of
      // the tile that raises its own leaves this one's factor at exactly 1
      if (__any(top > mx[t] + kRaise)) {
        top = lanes16_max(top);
        const float ref = top > mx[t] + kRaise ? top : mx[t];
        const float fac = ref == mx[t] ? 1.f : __builtin_amdgcn_exp2f(mx[t] - ref);
        mx[t] = ref;
        l[t] *= fac;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[t][i] *= fac;
      }
      const float ref = mx[t] == -INFINITY ? 0.f : mx[t];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[t][i] = __builtin_amdgcn_exp2f(s[t][i] - ref);
        l[t] += s[t][i];
        s[t][i] *= vs;
      }
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        Terms<N> p;
        p.cut(s[t] + 8 * hf);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[t][i] = p.product(f[i][hf], o[t][i]);
      }
    }
  }

  // the waves' states to LDS: values [wave][query][PA_OLD], max and sum behind
  float* w = paged_lds + wave * (QT * 16 * PA_OLD);
  float* ml = paged_lds + PA_NW * (QT * 16 * PA_OLD);
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const float sum = lanes16_sum(l[t]);
    float* x = w + (16 * t + m) * PA_OLD + 16 * g;
#pragma unroll
    for (int i = 0; i < 4; ++i) *(float4*)(x + 4 * i) = float4{o[t][0][i], o[t][1][i], o[t][2][i], o[t][3][i]};
    if (g == 0) {
      ml[(wave * QT * 16 + 16 * t + m) * 2] = mx[t];
      ml[(wave * QT * 16 + 16 * t + m) * 2 + 1] = sum;
    }
  }
  __syncthreads();
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int qi = 16 * t + (tid >> 4), d4 = (tid & 15) * 4, col = col0 + qi, j = col / a.per;
    if (j >= count) continue;
    const int r = start + j, h = head * a.per + col - j * a.per;
    float M = -INFINITY, L = 0.f;
    float4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < PA_NW; ++i) M = fmaxf(M, ml[(i * QT * 16 + qi) * 2]);
#pragma unroll
    for (int i = 0; i < PA_NW; ++i) {
      const float mw = ml[(i * QT * 16 + qi) * 2], lw = ml[(i * QT * 16 + qi) * 2 + 1];
      const float fac = mw == M ? 1.f : __builtin_amdgcn_exp2f(mw - M);
      const float4 y = *(const float4*)(paged_lds + (i * QT * 16 + qi) * PA_OLD + d4);
      L += fac * lw;
      x.x += fac * y.x;
      x.y += fac * y.y;
      x.z += fac * y.z;
      x.w += fac * y.w;
    }
    if (a.c.parts == 1) {
      // (divided as the join does it: the same bits however many parts there may be)
      St<T>::st4((T*)a.c.out, r * a.c.out_ld + h * kHeadDim + d4,
                 L == 0.f ? float4{0.f, 0.f, 0.f, 0.f} : float4{x.x / L, x.y / L, x.z / L, x.w / L});
    } else {
      float* v = a.c.rec + (((int64_t)r * a.c.n_head + h) * a.c.parts + part) * kHeadDim + d4;
      float2* ml = record(a.c, r, h, part);
      if (QT == 1 && a.c.counters) {
        if (L != 0.f) {
          store_agent((uint64_t*)v, __builtin_bit_cast(uint64_t, float2{x.x, x.y}));
          store_agent((uint64_t*)v + 1, __builtin_bit_cast(uint64_t, float2{x.z, x.w}));
        }
        if (d4 == 0) store_agent((uint64_t*)ml, __builtin_bit_cast(uint64_t, float2{M, L}));
      } else {
        if (L != 0.f) *(float4*)v = x;
        if (d4 == 0) *ml = float2{M, L};
      }
    }
  }
  if (QT == 1 && a.c.counters && arrive_last(a.c.counters + ((int64_t)seq * a.c.c.kv_heads + head) * a.tiles + ctile, a.c.parts)) {
    const int cols = min(count * a.per - col0, 16 * QT);
    for (int col = wave; col < cols; col += PA_NW) {
      const int j = (col0 + col) / a.per, r = start + j, h = head * a.per + col0 + col - j * a.per;
      Join<T, true>(a.c, r, h).store(a.c, r, h);
    }
  }
}

template <typename T>
__global__ __launch_bounds__(256) void k_join_pages(PagedArgs a) {
  const uint32_t w = blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (w >= (uint32_t)a.c.rows * a.c.n_head) return;
  const int row = (int)(w / a.c.n_head), h = (int)(w % a.c.n_head);
  Join<T, false> join(a.c, row, h);
  if (a.c.row_start) {
    // the row's sequence is the last one that starts at or before it
    int start = -1, end = 0;
    for (int s0 = 0; s0 < a.c.c.sequences; s0 += 64) {
      const int x = a.c.row_start[min(s0 + lane, a.c.c.sequences)];
      const int n = __popcll(__ballot(s0 + lane < a.c.c.sequences && x <= row));
      if (n == 0) break;
      start = __builtin_amdgcn_readlane(x, n - 1);
      end = n < 64 ? __builtin_amdgcn_readlane(x, n) : a.c.row_start[s0 + 64];
    }
    if (start < 0 || row >= end || row - start >= a.c.max_rows) return;
  } else if (row >= a.c.c.sequences) {
    return;
  }
  join.store(a.c, row, h);
}

template <typename T, int QT>
void launch(const PagedArgs& a, int64_t blocks, hipStream_t s) {
  constexpr int lds = PA_NW * QT * 16 * (PA_OLD + 2) * 4;
  static_assert(lds <= 65536, "without an attribute");
  k_attend_pages<T, QT><<<dim3((unsigned)blocks), PA_NW * 64, lds, s>>>(a);
}

template <typename T>
void attend(const PagedLaunch& c, hipStream_t s) {
  PagedArgs a{};
  a.c = c;
  a.per = c.n_head / c.c.kv_heads;
  const int cols = c.max_rows * a.per, qt = paged_query_tiles(cols);
  a.tiles = (cols + 16 * qt - 1) / (16 * qt);
  a.units = (uint32_t)((int64_t)c.c.sequences * c.parts * c.c.kv_heads);
  const int64_t blocks = ((int64_t)a.units + 7) / 8 * 8 * a.tiles;        // (below 2^24: the caller)
  qt == 1 ? launch<T, 1>(a, blocks, s) : launch<T, 2>(a, blocks, s);
  if (c.parts != 1 && !c.counters) k_join_pages<T><<<dim3((unsigned)(((int64_t)c.rows * c.n_head + 3) / 4)), 256, 0, s>>>(a);
}

}  // namespace

int paged_query_tiles(int cols) { return cols <= 16 ? 1 : 2; }

void attend_pages(const PagedLaunch& c, bool bf16, hipStream_t s) { bf16 ? attend<bf16_t>(c, s) : attend<float>(c, s); }

}  // namespace asr
