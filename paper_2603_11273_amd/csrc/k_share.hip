// Decode attention of rows that share keys (asr_attend_shared): the rows of a
// group -- hypotheses of one clip -- attend over keys that all of them share
// and, behind those, over keys of their own.
//
// The keys are the traffic: a group's shared keys are read once for all of its
// queries, 256 bytes (bf16) a key and head for 4 * 64 operations a query, so up
// to some hundred queries a group HBM is the bound.  A block takes a part of
// the keys of one (group, cache head) and up to 64 of the group's queries; its
// four waves take the part's 32-key (fp32: 16-key) tiles in turn, each with a
// running maximum, sum and weighted values of its own, joined through LDS at the
// end; the parts of a row are joined from (max, sum, values) records by a second
// kernel, or not at all where there is one part.
//
// Keys and values go from memory to the matrix instructions without LDS.  With
// lane = 16 g + m, the scores S^T = K Q^T of a 16-key tile leave lane (m, g)
// with query m's scores of tile rows 4 g .. 4 g + 3.  bf16: tile rows are loaded
// so that two tiles leave the lane keys 8 g .. 8 g + 7 of 32; the second product
// O^T = V^T P^T takes exactly those eight keys from lane (m, g), so the
// probabilities stay where they are.  Its other operand is V^T with rows = dims:
// lane (m, g) loads dims 4 m .. 4 m + 3 of keys 8 g + j (eight 8-byte loads, 128
// bytes a key over the 16 lanes) and picks one dim's eight keys with four byte
// permutes; row m of product t then is dim 4 m + t, which leaves the lane with 16
// consecutive dims of its query.  fp32: one 16-key tile, four dims a load, no
// permutes.
//
// Measured (bf16, 20 heads): 8 groups of 16 rows on 65536 keys 425 us, 6.7 TB/s; 24
// groups of 5 on 1500 and up to 224 own 48 us, 5.3 TB/s; 5 rows on 1540 8.5 us, two
// launches' latency.
#include "asr_device.h"

namespace asr {
namespace {

constexpr int SH_NW = 4;                 // waves of a block
constexpr int SH_OLD = 68;               // floats a query's row takes in LDS: 16 lanes, 64 banks
constexpr float kRaise = 8.f;            // the reference follows the maximum from 2^8 on

// Loads of keys and values pass the caches as data that is read once: 8 x 16
// rows on 65536 shared keys 515 -> 486 us, 24 x 5 on 1500 54 -> 49.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
template <typename V>
__device__ __forceinline__ V load16(const char* p) {
  return __builtin_bit_cast(V, __builtin_nontemporal_load((const u32x4*)p));
}
__device__ __forceinline__ uint2 load8(const char* p) {
  return __builtin_bit_cast(uint2, __builtin_nontemporal_load((const u32x2*)p));
}

struct ShareArgs {
  ShareLaunch c;
  int per, tiles, own_tiles;
  uint32_t prefix_units, prefix_blocks;
};

// The keys of one tile in a lane's registers, and the two products with them.
template <typename T>
struct KeyTile;

template <>
struct KeyTile<bf16_t> {
  static constexpr int KEYS = 32, NS = 8;     // keys of a tile, scores of a lane
  uint4 k[2][2];
  uint2 v[8];
  // q: dims 8 g + i and 32 + 8 g + i of the lane's query as hi + lo: its bf16
  // rounding alone would move a score of 20 by 0.04, the pair by 2e-4
  struct Query {
    bf16x8 hi[2], lo[2];
    __device__ __forceinline__ void set(const float* p, int g, float mul) {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const float4 a = *(const float4*)(p + 32 * s + 8 * g), b = *(const float4*)(p + 32 * s + 8 * g + 4);
        const float x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float y = x[i] * mul;
          const __bf16 h = (__bf16)y;
          hi[s][i] = h;
          lo[s][i] = (__bf16)(y - (float)h);
        }
      }
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int i = 0; i < 8; ++i) hi[s][i] = lo[s][i] = (__bf16)0.f;
    }
  };
  // keys of the lane's scores: first + i
  static __device__ __forceinline__ int first_key(int g) { return 8 * g; }
  // tile at kb, vb, of which n keys are left (past the end: the last key again, masked later)
  __device__ __forceinline__ void load_keys(const char* kb, uint32_t pos_bytes, int n, int m, int g) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t off = (uint32_t)min((m >> 2) * 8 + (m & 3) + 4 * h, n - 1) * pos_bytes + 16 * g;
      k[h][0] = load16<uint4>(kb + off);
      k[h][1] = load16<uint4>(kb + off + 64);
    }
  }
  __device__ __forceinline__ void load_values(const char* vb, uint32_t pos_bytes, int n, int m, int g) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      v[j] = load8(vb + (uint32_t)min(8 * g + j, n - 1) * pos_bytes + 8 * m);
  }
  __device__ __forceinline__ void drop_values(int key0, int n) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (key0 + j >= n) v[j] = uint2{0u, 0u};
  }
  __device__ __forceinline__ void scores(const Query& q, float* s) const {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      f32x4 a = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int d = 0; d < 2; ++d) {
        const bf16x8 kk = __builtin_bit_cast(bf16x8, k[h][d]);
        a = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kk, q.lo[d], a, 0, 0, 0);
        a = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kk, q.hi[d], a, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) s[4 * h + i] = a[i];
    }
  }
  // V^T fragments (once for all queries of the tile)
  __device__ __forceinline__ void fragments(bf16x8* f) const {
    uint4 u[4];
    uint32_t* w = (uint32_t*)u;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      w[p] = __builtin_amdgcn_perm(v[2 * p + 1].x, v[2 * p].x, 0x05040100);
      w[4 + p] = __builtin_amdgcn_perm(v[2 * p + 1].x, v[2 * p].x, 0x07060302);
      w[8 + p] = __builtin_amdgcn_perm(v[2 * p + 1].y, v[2 * p].y, 0x05040100);
      w[12 + p] = __builtin_amdgcn_perm(v[2 * p + 1].y, v[2 * p].y, 0x07060302);
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) f[t] = __builtin_bit_cast(bf16x8, u[t]);
  }
  using Frag = bf16x8;
  // o += V^T p, the probabilities as bf16 pairs hi + lo (hi cut off, not
  // rounded: one byte permute for two): a single rounding to bf16 would add as
  // much error again as the rounding of the result.  hi is cut from the float
  // below, so lo is never 0 where p is not: an infinite value stays infinite
  static __device__ __forceinline__ void accumulate(const Frag* f, const float* p, f32x4* o) {
    uint4 hi, lo;
    uint32_t *hw = (uint32_t*)&hi, *lw = (uint32_t*)&lo;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t a = __builtin_elementwise_sub_sat(__float_as_uint(p[2 * i]), 1u);
      const uint32_t b = __builtin_elementwise_sub_sat(__float_as_uint(p[2 * i + 1]), 1u);
      hw[i] = __builtin_amdgcn_perm(b, a, 0x07060302);
      lw[i] = pack2_bf16(p[2 * i] - __uint_as_float(a & 0xffff0000u),
                         p[2 * i + 1] - __uint_as_float(b & 0xffff0000u));
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[t], __builtin_bit_cast(bf16x8, lo), o[t], 0, 0, 0);
      o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[t], __builtin_bit_cast(bf16x8, hi), o[t], 0, 0, 0);
    }
  }
};

template <>
struct KeyTile<float> {
  static constexpr int KEYS = 16, NS = 4;
  float4 k[4], v[4];
  struct Query {
    float x[16];
    __device__ __forceinline__ void set(const float* p, int g, float mul) {
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const float4 a = *(const float4*)(p + 16 * s + 4 * g);
        x[4 * s] = a.x * mul;
        x[4 * s + 1] = a.y * mul;
        x[4 * s + 2] = a.z * mul;
        x[4 * s + 3] = a.w * mul;
      }
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = 0.f;
    }
  };
  static __device__ __forceinline__ int first_key(int g) { return 4 * g; }
  __device__ __forceinline__ void load_keys(const char* kb, uint32_t pos_bytes, int n, int m, int g) {
    // (four lanes read 64 bytes of a key at once; the query's dims lie alike)
    const uint32_t off = (uint32_t)min(m, n - 1) * pos_bytes + 16 * g;
#pragma unroll
    for (int s = 0; s < 4; ++s) k[s] = load16<float4>(kb + off + 64 * s);
  }
  __device__ __forceinline__ void load_values(const char* vb, uint32_t pos_bytes, int n, int m, int g) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      v[j] = load16<float4>(vb + (uint32_t)min(4 * g + j, n - 1) * pos_bytes + 16 * m);
  }
  __device__ __forceinline__ void drop_values(int key0, int n) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (key0 + j >= n) v[j] = float4{0.f, 0.f, 0.f, 0.f};
  }
  __device__ __forceinline__ void scores(const Query& q, float* s) const {
    // two chains: a matrix instruction waits for the one before it in its chain
    f32x4 a = {0.f, 0.f, 0.f, 0.f}, b = a;
    const float* kk = (const float*)k;
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      a = __builtin_amdgcn_mfma_f32_16x16x4f32(kk[i], q.x[i], a, 0, 0, 0);
      b = __builtin_amdgcn_mfma_f32_16x16x4f32(kk[i + 1], q.x[i + 1], b, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = a[i] + b[i];
  }
  struct Frag {
    float4 v;
  };
  __device__ __forceinline__ void fragments(Frag* f) const {
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j].v = v[j];
  }
  static __device__ __forceinline__ void accumulate(const Frag* f, const float* p, f32x4* o) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      o[0] = __builtin_amdgcn_mfma_f32_16x16x4f32(f[j].v.x, p[j], o[0], 0, 0, 0);
      o[1] = __builtin_amdgcn_mfma_f32_16x16x4f32(f[j].v.y, p[j], o[1], 0, 0, 0);
      o[2] = __builtin_amdgcn_mfma_f32_16x16x4f32(f[j].v.z, p[j], o[2], 0, 0, 0);
      o[3] = __builtin_amdgcn_mfma_f32_16x16x4f32(f[j].v.w, p[j], o[3], 0, 0, 0);
    }
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

// The keys [first, first + n) of an entry (a group or a row) of a cache; a slot
// outside the cache has none, a range past its end stops there.
struct Range {
  int slot, first, n;
};
__device__ __forceinline__ Range key_range(const ShareKeys& c, int entry) {
  Range r;
  r.slot = c.slot ? c.slot[entry] : entry;
  r.first = c.first ? max(c.first[entry], 0) : 0;
  const int n = c.len ? c.len[entry] : c.most;
  r.n = max(min(min(n, c.most), c.positions - r.first), 0);
  if (r.slot < 0 || r.slot >= c.slots) r.slot = 0, r.n = 0;
  return r;
}

// (max, sum) of part `part` of the row at `place` and head h; a sum of kNoKeys
// says that the part has none (and no values).
constexpr float kNoKeys = -1.f;
__device__ __forceinline__ float2* record(const ShareLaunch& c, int place, int h, int part) {
  const int parts = c.np + c.no;
  return (float2*)(c.rec + (int64_t)c.rows * c.n_head * parts * kHeadDim) + ((int64_t)place * c.n_head + h) * parts + part;
}

// Keys [k0, k1) of `r` for the queries [col0, col0 + 16 QT) of `count` rows from
// place `start`; leaves their records as part `part`, or the result where a row
// has only this part.
template <typename T, int QT>
__device__ __forceinline__ void attend_part(const ShareArgs& a, const ShareKeys& c, const Range& r, int k0, int k1, int head,
                                            int start, int count, int col0, int part, float* lds) {
  using Tile = KeyTile<T>;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int m = lane & 15, g = lane >> 4;
  const int n = k1 - k0;
  const int64_t at = (int64_t)r.slot * c.slot_stride + (int64_t)head * c.head_stride + (int64_t)(r.first + k0) * c.pos_stride;
  const char *kb = (const char*)((const T*)c.k + at), *vb = (const char*)((const T*)c.v + at);
  const uint32_t pos_bytes = (uint32_t)c.pos_stride * sizeof(T);
  constexpr int STEP = SH_NW * Tile::KEYS;
  const int64_t step_bytes = (int64_t)STEP * pos_bytes;
  kb += (int64_t)(wave * Tile::KEYS) * pos_bytes;
  vb += (int64_t)(wave * Tile::KEYS) * pos_bytes;
  Tile tile;
  if (wave * Tile::KEYS < n) {
    tile.load_keys(kb, pos_bytes, n - wave * Tile::KEYS, m, g);
    tile.load_values(vb, pos_bytes, n - wave * Tile::KEYS, m, g);
  }

  typename Tile::Query q[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int col = col0 + 16 * t + m, j = col / a.per;
    int row = -1;
    if (j < count) row = a.c.row_of ? a.c.row_of[start + j] : start + j;
    if (row >= 0 && row < a.c.rows)
      q[t].set(a.c.q + (int64_t)row * a.c.q_ld + (head * a.per + col - j * a.per) * kHeadDim, g, a.c.qmul);
    else
      q[t].clear();
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

  // The next tile's keys are under way as soon as this one's have given their
  // scores, its values as soon as this one's are fragments: one set of registers
  // each, hence more waves, and the loads never stop.
  for (int t0 = wave * Tile::KEYS; t0 < n; t0 += STEP) {
    const int key0 = t0 + Tile::first_key(g);
    const bool tail = t0 + Tile::KEYS > n, more = t0 + STEP < n;   // wave-uniform
    float s[QT][Tile::NS];
#pragma unroll
    for (int t = 0; t < QT; ++t) tile.scores(q[t], s[t]);
    kb += step_bytes;
    vb += step_bytes;
    if (more) tile.load_keys(kb, pos_bytes, n - t0 - STEP, m, g);
    if (tail) tile.drop_values(key0, n);
    typename Tile::Frag f[4];
    tile.fragments(f);
    if (more) tile.load_values(vb, pos_bytes, n - t0 - STEP, m, g);
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      if (tail) {
#pragma unroll
        for (int i = 0; i < Tile::NS; ++i)
          if (key0 + i >= n) s[t][i] = -INFINITY;
      }
      float top = s[t][0];
#pragma unroll
      for (int i = 1; i < Tile::NS; ++i) top = fmaxf(top, s[t][i]);
      // the reference of the exponents is a query's own matter: another query
      // of the tile that raises its own leaves this one's factor at exactly 1
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
      float p[Tile::NS];
#pragma unroll
      for (int i = 0; i < Tile::NS; ++i) {
        p[i] = __builtin_amdgcn_exp2f(s[t][i] - ref);
        l[t] += p[i];
      }
      Tile::accumulate(f, p, o[t]);
    }
  }

  // the waves' states to LDS: values [wave][query][SH_OLD], max and sum behind
  float* lo = lds + wave * (QT * 16 * SH_OLD);
  float* ml = lds + SH_NW * (QT * 16 * SH_OLD);
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const float sum = lanes16_sum(l[t]);
    float* w = lo + (16 * t + m) * SH_OLD + 16 * g;
#pragma unroll
    for (int i = 0; i < 4; ++i) *(float4*)(w + 4 * i) = float4{o[t][0][i], o[t][1][i], o[t][2][i], o[t][3][i]};
    if (g == 0) {
      ml[(wave * QT * 16 + 16 * t + m) * 2] = mx[t];
      ml[(wave * QT * 16 + 16 * t + m) * 2 + 1] = sum;
    }
  }
  __syncthreads();
  const int parts = a.c.np + a.c.no;
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int qi = 16 * t + (tid >> 4), d4 = (tid & 15) * 4;
    const int col = col0 + qi, j = col / a.per, h = head * a.per + col - j * a.per;
    if (j >= count) continue;
    const int row = a.c.row_of ? a.c.row_of[start + j] : start + j;
    if (row < 0 || row >= a.c.rows) continue;
    float M = -INFINITY, L = 0.f;
    float4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < SH_NW; ++w) M = fmaxf(M, ml[(w * QT * 16 + qi) * 2]);
#pragma unroll
    for (int w = 0; w < SH_NW; ++w) {
      const float mw = ml[(w * QT * 16 + qi) * 2], lw = ml[(w * QT * 16 + qi) * 2 + 1];
      const float fac = mw == M ? 1.f : __builtin_amdgcn_exp2f(mw - M);
      const float4 x = *(const float4*)(lds + (w * QT * 16 + qi) * SH_OLD + d4);
      L += fac * lw;
      v.x += fac * x.x;
      v.y += fac * x.y;
      v.z += fac * x.z;
      v.w += fac * x.w;
    }
    if (parts == 1) {
      const float inv = n > 0 ? 1.f / L : 0.f;         // no keys: zeros
      St<T>::st4((T*)a.c.out, (int64_t)row * a.c.out_ld + h * kHeadDim + d4,
                 float4{v.x * inv, v.y * inv, v.z * inv, v.w * inv});
    } else {
      const int64_t rh = (int64_t)(start + j) * a.c.n_head + h;
      *(float4*)(a.c.rec + (rh * parts + part) * kHeadDim + d4) = v;
      if (d4 == 0) *record(a.c, start + j, h, part) = float2{M, L};
    }
  }
}

// Blocks: the parts of the shared keys, then those of the rows' own.  Blocks go
// to the XCDs in turn, so the query tiles of one part lie 8 blocks apart: they
// read the same keys through one L2.
template <typename T, int QT>
__global__ __launch_bounds__(SH_NW * 64) __attribute__((amdgpu_waves_per_eu(QT == 1 ? 4 : QT == 2 ? 3 : 2)))
void k_attend_shared(ShareArgs a) {
  extern __shared__ __attribute__((aligned(16))) float share_lds[];
  uint32_t u = blockIdx.x;
  if (u < a.prefix_blocks) {
    const int tile = (int)((u >> 3) % a.tiles);
    u = (u >> 3) / a.tiles * 8 + (u & 7);
    if (u >= a.prefix_units) return;
    const int head = (int)(u % a.c.n_kv);
    u /= a.c.n_kv;
    const int part = (int)(u % a.c.np), grp = (int)(u / a.c.np);
    // (all of the block's numbers in one go: memory answers late once it is busy)
    const Range r = key_range(a.c.prefix, grp);
    const int start = a.c.group_start[grp], end = a.c.group_start[grp + 1];
    const int count = min(min(end, a.c.rows) - start, a.c.max_group);
    if (start < 0 || tile * 16 * QT >= count * a.per) return;
    const int k0 = part * a.c.prefix_part, k1 = min(k0 + a.c.prefix_part, r.n);
    if (k0 >= k1 && a.c.np + a.c.no > 1) {
      const int col = tile * 16 * QT + (int)threadIdx.x, j = col / a.per;
      if (threadIdx.x < 16 * QT && j < count)
        *record(a.c, start + j, head * a.per + col - j * a.per, part) = float2{-INFINITY, kNoKeys};
      return;
    }
    attend_part<T, QT>(a, a.c.prefix, r, min(k0, k1), k1, head, start, count, tile * 16 * QT, part, share_lds);
  } else {
    u -= a.prefix_blocks;
    const int head = (int)(u % a.c.n_kv);
    u /= a.c.n_kv;
    const int tile = (int)(u % a.own_tiles);
    u /= a.own_tiles;
    const int part = (int)(u % a.c.no), i = (int)(u / a.c.no);
    const int row = a.c.row_of ? a.c.row_of[i] : i, first = a.c.group_start[0], end = a.c.group_start[a.c.groups];
    if (i < first || i >= end || row < 0 || row >= a.c.rows) return;
    const Range r = key_range(a.c.own, row);
    const int k0 = part * a.c.own_part, k1 = min(k0 + a.c.own_part, r.n);
    if (k0 >= k1 && a.c.np + a.c.no > 1) {
      const int col = tile * 16 + (int)threadIdx.x;
      if (threadIdx.x < 16 && col < a.per)
        *record(a.c, i, head * a.per + col, a.c.np + part) = float2{-INFINITY, kNoKeys};
      return;
    }
    attend_part<T, 1>(a, a.c.own, r, min(k0, k1), k1, head, i, 1, tile * 16, a.c.np + part, share_lds);
  }
}

// out of a row and head from its parts' records; one wave each, lane = dim.  A
// row's group is the last one that starts at or before its place.  The kernel is
// a chain of loads, so all it needs is loaded at once, SH_JOIN records at a time;
// which of them there are they say themselves.
constexpr int SH_JOIN = 16;
template <typename T>
__global__ __launch_bounds__(256) void k_attend_join(ShareArgs a) {
  const uint32_t w = blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (w >= (uint32_t)a.c.rows * a.c.n_head) return;
  const int i = (int)(w / a.c.n_head), h = (int)(w % a.c.n_head);
  const int parts = a.c.np + a.c.no;
  const float* val = a.c.rec + (int64_t)w * parts * kHeadDim + lane;
  const float2* ml = record(a.c, i, h, 0);
  float v[SH_JOIN];
  float2 rec;
  auto load = [&](int p0) {
    rec = lane < SH_JOIN && p0 + lane < parts ? ml[p0 + lane] : float2{-INFINITY, kNoKeys};
#pragma unroll
    for (int p = 0; p < SH_JOIN; ++p) v[p] = p0 + p < parts ? val[(int64_t)(p0 + p) * kHeadDim] : 0.f;
  };
  load(0);
  const int row = a.c.row_of ? a.c.row_of[i] : i, end = a.c.group_start[a.c.groups];
  int start = -1;
  for (int g0 = 0; g0 < a.c.groups; g0 += 64) {
    const int x = a.c.group_start[min(g0 + lane, a.c.groups - 1)];
    const int n = __popcll(__ballot(g0 + lane < a.c.groups && x <= i));
    if (n == 0) break;
    start = __builtin_amdgcn_readlane(x, n - 1);
  }
  if (start < 0 || i >= end || i - start >= a.c.max_group) return;
  if (row < 0 || row >= a.c.rows) return;
  float M = -INFINITY, L = 0.f, acc = 0.f;
  bool any = false;
  for (int p0 = 0; p0 < parts; p0 += SH_JOIN) {
    if (p0 > 0) load(p0);
    const bool there = rec.y != kNoKeys;               // (a sum is 0 or more, or NaN)
    const uint64_t some = __ballot(there);
    if (!some) continue;
    any = true;
    const float top = fmaxf(M, wave_max_lanes(rec.x));
    const float keep = M == top ? 1.f : __builtin_amdgcn_exp2f(M - top);
    const float fac = !there ? 0.f : rec.x == top ? 1.f : __builtin_amdgcn_exp2f(rec.x - top);
    M = top;
    L = L * keep + wave_sum_lanes(there ? fac * rec.y : 0.f);
    acc *= keep;
#pragma unroll
    for (int j = 0; j < SH_JOIN; ++j)
      if (some >> j & 1) acc += __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(fac), j)) * v[j];
  }
  St<T>::st((T*)a.c.out, (int64_t)row * a.c.out_ld + h * kHeadDim + lane, any ? acc / L : 0.f);
}

template <typename T, int QT>
hipError_t launch(const ShareArgs& a, int64_t blocks, hipStream_t s) {
  constexpr int lds = SH_NW * QT * 16 * (SH_OLD + 2) * 4;
  if (lds > 65536) {
    const hipError_t e = hipFuncSetAttribute((const void*)k_attend_shared<T, QT>,
                                             hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (e != hipSuccess) return e;
  }
  k_attend_shared<T, QT><<<dim3((unsigned)blocks), SH_NW * 64, lds, s>>>(a);
  return hipSuccess;
}

template <typename T>
hipError_t attend(const ShareLaunch& c, hipStream_t s) {
  ShareArgs a{};
  a.c = c;
  a.per = c.n_head / c.n_kv;
  const int cols = c.max_group * a.per;
  const int qt = share_query_tiles(cols);
  a.tiles = (cols + 16 * qt - 1) / (16 * qt);
  a.own_tiles = (a.per + 15) / 16;
  a.prefix_units = (uint32_t)((int64_t)c.groups * c.np * c.n_kv);
  a.prefix_blocks = (a.prefix_units + 7) / 8 * 8 * a.tiles;
  const int64_t blocks = a.prefix_blocks + (int64_t)c.rows * c.no * a.own_tiles * c.n_kv;   // (below 2^31: the caller)
  if (blocks > 0) {
    const hipError_t e = qt == 1 ? launch<T, 1>(a, blocks, s) : qt == 2 ? launch<T, 2>(a, blocks, s) : launch<T, 4>(a, blocks, s);
    if (e != hipSuccess) return e;
  }
  if (c.np + c.no != 1)
    k_attend_join<T><<<dim3((unsigned)(((int64_t)c.rows * c.n_head + 3) / 4)), 256, 0, s>>>(a);
  return hipSuccess;
}

}  // namespace

int share_query_tiles(int cols) { return cols <= 16 ? 1 : cols <= 32 ? 2 : 4; }

hipError_t attend_shared(const ShareLaunch& c, bool bf16, hipStream_t s) {
  return bf16 ? attend<bf16_t>(c, s) : attend<float>(c, s);
}

// One wave per (row, head): lane = dim.
template <typename T>
__global__ __launch_bounds__(64) void k_append_kv(const float* __restrict__ qkv, T* cache, int64_t slot_stride,
                                                  int64_t layer_off, const int32_t* __restrict__ slots,
                                                  const int32_t* __restrict__ pos, int n_head) {
  const int h = blockIdx.x, row = blockIdx.y, lane = threadIdx.x, d = n_head * kHeadDim;
  T* k = cache + (int64_t)slots[row] * slot_stride + layer_off + ((int64_t)h * kTextCtx + pos[row]) * kHeadDim;
  const float* src = qkv + (int64_t)row * 3 * d + h * kHeadDim + lane;
  St<T>::st(k, lane, src[d]);
  St<T>::st(k + (int64_t)n_head * kTextCtx * kHeadDim, lane, src[2 * d]);
}
template <typename T>
void decode_append_kv(const float* qkv, T* cache, int64_t slot_stride, int64_t layer_off, const int32_t* slots,
                      const int32_t* pos, int D, int n_head, hipStream_t s) {
  if (D > 0) k_append_kv<T><<<dim3(n_head, D), 64, 0, s>>>(qkv, cache, slot_stride, layer_off, slots, pos, n_head);
}
template void decode_append_kv<float>(const float*, float*, int64_t, int64_t, const int32_t*, const int32_t*, int, int,
                                      hipStream_t);
template void decode_append_kv<bf16_t>(const float*, bf16_t*, int64_t, int64_t, const int32_t*, const int32_t*, int, int,
                                       hipStream_t);

// One block per (layer, key or value, head): 16 bytes a thread.
__global__ __launch_bounds__(256) void k_copy_runs(const uint4* __restrict__ src, uint4* __restrict__ dst, int ld, int first, int n) {
  const int64_t at = (int64_t)blockIdx.x * ld + first;
  for (int i = threadIdx.x; i < n; i += 256) dst[at + i] = src[at + i];
}
template <typename T>
void copy_self_kv(const T* src, T* dst, int blocks, int p0, int p1, hipStream_t s) {
  constexpr int U = kHeadDim * sizeof(T) / 16;         // 16-byte units of a position
  if (p1 > p0)
    k_copy_runs<<<blocks, 256, 0, s>>>((const uint4*)src, (uint4*)dst, kTextCtx * U, p0 * U, (p1 - p0) * U);
}
template void copy_self_kv<float>(const float*, float*, int, int, int, hipStream_t);
template void copy_self_kv<bf16_t>(const bf16_t*, bf16_t*, int, int, int, hipStream_t);

}  // namespace asr
