// A cache in pages of e4m3 codes: new keys and values into it (asr_write_pages)
// and the page tables of a next step (asr_next_tables).
#include <algorithm>

#include "asr_device.h"

namespace asr {
namespace {

// ---------------------------------------------------------------------------
// Writing
// ---------------------------------------------------------------------------
constexpr int kLeastScale = 127 - 120, kMostScale = 127 + 120;   // exponent fields

// Exponent field of the smallest power of two, in range, of which 448 are >= top
// (the bits of a finite magnitude): 448 = 1.75 * 2^8, so a significand above 1.75
// carries into the next power.
__device__ __forceinline__ int need_exp(uint32_t top) {
  return min(max((int)((top + 0x1fffffu) >> 23) - 8, kLeastScale), kMostScale);
}
// Exponent field of a block's scale, rounded up to a power of two in range.
__device__ __forceinline__ int held_exp(float s) {
  const uint32_t u = __float_as_uint(s);
  return s > 0.f ? min(max((int)((u + 0x7fffffu) >> 23), kLeastScale), kMostScale) : kLeastScale;
}
__device__ __forceinline__ float exp_scale(int e) { return __uint_as_float((uint32_t)e << 23); }

__device__ __forceinline__ uint32_t magnitude(float x) {      // 0 for what is not finite
  const uint32_t u = __float_as_uint(x) & 0x7fffffffu;
  return u < 0x7f800000u ? u : 0u;
}
// Two values in e4m3, already over the scale (nearest even by the instruction)
__device__ __forceinline__ uint32_t code2(float a, float b) {
  const float x = fminf(fmaxf(a, -448.f), 448.f), y = fminf(fmaxf(b, -448.f), 448.f);
  uint32_t c = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x, y, 0, false) & 0xffffu;
  if (magnitude(a) != (__float_as_uint(a) & 0x7fffffffu)) c = (c & 0xff00u) | 0x7fu;
  if (magnitude(b) != (__float_as_uint(b) & 0x7fffffffu)) c = (c & 0x00ffu) | 0x7f00u;
  return c;
}
__device__ __forceinline__ uint32_t code4(const float* x) { return code2(x[0], x[1]) | code2(x[2], x[3]) << 16; }
typedef float f32x2v __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t rescale4(uint32_t c, float by) {
  const f32x2v a = __builtin_amdgcn_cvt_pk_f32_fp8(c, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(c, true);
  const float x[4] = {a.x * by, a.y * by, b.x * by, b.y * by};
  return code4(x);
}

// Four values that are finite and, over the scale, at most 448.
__device__ __forceinline__ uint32_t code4_plain(const float* x, float inv) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * inv, x[1] * inv, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2] * inv, x[3] * inv, lo, true);
}

// Bytes [lo, hi) of the 16 at a dword-aligned place.
__device__ __forceinline__ void store_some(uint8_t* p, const uint32_t* w, int lo, int hi) {
  if (lo <= 0 && hi >= 16) {
    *(uint4*)p = uint4{w[0], w[1], w[2], w[3]};
    return;
  }
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (i >= lo && i < hi) p[i] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
}

// 16 values; the address is a multiple of 16 bytes.
__device__ __forceinline__ void load16(const float* p, float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float4 v = ((const float4*)p)[i];
    x[4 * i] = v.x, x[4 * i + 1] = v.y, x[4 * i + 2] = v.z, x[4 * i + 3] = v.w;
  }
}
__device__ __forceinline__ void load16(const bf16_t* p, float* x) {
  const uint4 v[2] = {((const uint4*)p)[0], ((const uint4*)p)[1]};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t u = ((const uint32_t*)v)[i];
    x[2 * i] = __uint_as_float(u << 16), x[2 * i + 1] = __uint_as_float(u & 0xffff0000u);
  }
}

// What a block of positions gets: tokens start + i to positions length + i, i < count.
struct NewTokens {
  int start, count;
  uint32_t length, stop;                   // positions from length to stop, at most 2^30
};
__device__ __forceinline__ NewTokens new_tokens(const PageWriteLaunch& a, int seq) {
  const int length = a.length[seq];
  int start = a.token_start ? a.token_start[seq] : seq, end = a.token_start ? a.token_start[seq + 1] : seq + 1;
  start = max(start, 0);
  end = min(min(end, a.tokens), start > INT32_MAX - a.max_new ? INT32_MAX : start + a.max_new);
  end = max(end, start);                   // (an end far below the start: their distance passes 32 bits)
  const uint32_t most = a.c.columns * a.c.page;
  return {start, length < 0 ? 0 : end - start, (uint32_t)length, min((uint32_t)length + (uint32_t)(end - start), most)};
}
// Codes and scale of a head's block of positions in a page; keys or values.
struct BlockPlace {
  uint8_t* codes;
  float* scale;
};
__device__ __forceinline__ BlockPlace block_place(const Pages& c, int page, uint32_t p0, int head, int which) {
  const int per = c.page / kPageBlock;
  const int64_t at = (int64_t)(which * c.kv_heads + head) * per + p0 % (uint32_t)c.page / kPageBlock;
  return {c.codes + page * c.page_stride + at * (kPageBlock * kHeadDim), c.scales + page * c.scale_stride + at};
}
// A block's scale with new values up to `top` behind `old` positions: the factor that
// earlier codes take where it grew.
struct NewScale {
  int e;
  bool grew;
  float by;
};
__device__ __forceinline__ NewScale new_scale(uint32_t top, int old, const float* scale) {
  NewScale n = {need_exp(top), false, 1.f};
  if (old > 0) {
    const float s = *scale;
    n.e = max(n.e, held_exp(s));
    n.grew = s != exp_scale(n.e);
    n.by = (s > 0.f ? s : exp_scale(kLeastScale)) / exp_scale(n.e);
  }
  return n;
}

// One block of 256 threads per (sequence, touched block of positions, head, keys or
// values); thread = (position, 16 dims).  Values lie [dim][position] and are turned in LDS.
// Bound by memory: 36000 bf16 tokens of 20 heads, 276 MB, in 58 us where no cache holds them
// (4.8 TB/s), in 49 where the last level holds some (the same call again).  A thread of 4
// positions x 4 dims turns its codes in registers, but its loads of 8 bytes cost more than
// that saves (71 us).  What is not finite is looked for once a block: without any, codes
// need neither bounds nor a test.
constexpr int PW_PITCH = 68;               // bytes of a dim in LDS: the four groups of dims write to banks of their own
template <typename T>
__global__ __launch_bounds__(256) void k_write_pages(PageWriteLaunch a, int touched) {
  __shared__ uint32_t tops[2][4];
  __shared__ __attribute__((aligned(16))) uint8_t turn[64 * PW_PITCH];
  const int tid = threadIdx.x;
  uint32_t u = blockIdx.x;
  const int which = u & 1;
  u >>= 1;
  const int head = (int)(u % a.c.kv_heads);
  u /= a.c.kv_heads;
  const int nth = (int)(u % touched), seq = (int)(u / touched);
  const NewTokens t = new_tokens(a, seq);
  if (t.count <= 0) return;
  const uint32_t p0 = (t.length / kPageBlock + nth) * kPageBlock;
  if (t.length >= t.stop || p0 >= t.stop) return;
  const int old = max((int)(t.length - p0), 0), last = (int)min(t.stop - p0, (uint32_t)kPageBlock);
  const int page = a.c.table[(int64_t)seq * a.c.table_ld + p0 / (uint32_t)a.c.page];
  if (page < 0 || page >= a.c.pages) return;
  const BlockPlace b = block_place(a.c, page, p0, head, which);

  float x[16];
  uint32_t top = 0;
  const int pos = tid >> 2, d0 = (tid & 3) * 16;
  const T* src = (const T*)(which ? a.v : a.k) + (t.start + ((int64_t)p0 - t.length) + pos) * a.ld + head * kHeadDim + d0;
  const bool fresh = pos >= old && pos < last;
  if (fresh) load16(src, x);
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    if (!fresh) x[i] = 0.f;
    top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
  }
  top = wave_max_u32(top);
  if ((tid & 63) == 0) tops[0][tid >> 6] = top;
  __syncthreads();
  top = max(max(tops[0][0], tops[0][1]), max(tops[0][2], tops[0][3]));
  const bool finite = top < 0x7f800000u;
  if (!finite) {                           // of those that are
    top = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) top = max(top, magnitude(x[i]));
    top = wave_max_u32(top);
    if ((tid & 63) == 0) tops[1][tid >> 6] = top;
    __syncthreads();
    top = max(max(tops[1][0], tops[1][1]), max(tops[1][2], tops[1][3]));
  }
  const NewScale n = new_scale(top, old, b.scale);
  const float inv = exp_scale(254 - n.e);
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (finite) {
      w[i] = code4_plain(x + 4 * i, inv);
    } else {
      const float y[4] = {x[4 * i] * inv, x[4 * i + 1] * inv, x[4 * i + 2] * inv, x[4 * i + 3] * inv};
      w[i] = code4(y);
    }
  }
  if (which == 0) {
    uint8_t* p = b.codes + pos * kHeadDim + d0;
    if (fresh) {
      *(uint4*)p = uint4{w[0], w[1], w[2], w[3]};
    } else if (n.grew && pos < old) {
      const uint4 c = *(const uint4*)p;
      *(uint4*)p = uint4{rescale4(c.x, n.by), rescale4(c.y, n.by), rescale4(c.z, n.by), rescale4(c.w, n.by)};
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) turn[(d0 + i) * PW_PITCH + pos] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
    __syncthreads();
    const int dim = tid >> 2, t0 = (tid & 3) * 16, from = n.grew ? 0 : old;
    uint8_t* p = b.codes + dim * kPageBlock + t0;
    if (t0 + 16 > from && t0 < last) {
      uint32_t c[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) c[i] = *(const uint32_t*)(turn + dim * PW_PITCH + t0 + 4 * i);
      if (n.grew && t0 < old) {
        const uint4 o = *(const uint4*)p;
        const uint32_t r[4] = {rescale4(o.x, n.by), rescale4(o.y, n.by), rescale4(o.z, n.by), rescale4(o.w, n.by)};
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (t0 + i < old) c[i >> 2] = (c[i >> 2] & ~(0xffu << (8 * (i & 3)))) | (r[i >> 2] & (0xffu << (8 * (i & 3))));
      }
      store_some(p, c, from - t0, last - t0);
    }
  }
  __syncthreads();                         // (every thread has read the scale)
  if (tid == 0) *b.scale = exp_scale(n.e);
}

// A token a sequence: one wave per (sequence, head, keys or values), lane = dim: 16
// times fewer waves than the blocks above, so that all of them run at once (128
// sequences of 20 heads: 14.3 -> 8.9 us).
template <typename T>
__global__ __launch_bounds__(256) void k_write_step(PageWriteLaunch a) {
  const int lane = threadIdx.x & 63;
  uint32_t u = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int which = u & 1;
  u >>= 1;
  const int head = (int)(u % a.c.kv_heads), seq = (int)(u / a.c.kv_heads);
  if (seq >= a.c.sequences) return;
  const NewTokens t = new_tokens(a, seq);
  if (t.count <= 0 || t.length >= t.stop) return;
  const float x = St<T>::ld((const T*)(which ? a.v : a.k) + t.start * a.ld + head * kHeadDim, lane);
  const int page = a.c.table[(int64_t)seq * a.c.table_ld + t.length / (uint32_t)a.c.page];
  if (page < 0 || page >= a.c.pages) return;
  const int old = (int)(t.length % kPageBlock);
  const BlockPlace b = block_place(a.c, page, t.length - old, head, which);
  const NewScale n = new_scale(wave_max_u32(magnitude(x)), old, b.scale);
  const uint32_t code = code2(x * exp_scale(254 - n.e), 0.f) & 0xffu;
  if (n.grew) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      // 16 dims of a position, or 16 positions of a dim
      const int row = i * 16 + (lane >> 2), col = (lane & 3) * 16;
      uint8_t* p = b.codes + row * 64 + col;
      if ((which ? col : row) >= old) continue;
      const uint4 c = *(const uint4*)p;
      uint32_t r[4] = {rescale4(c.x, n.by), rescale4(c.y, n.by), rescale4(c.z, n.by), rescale4(c.w, n.by)};
      if (which) store_some(p, r, 0, old - col); else *(uint4*)p = uint4{r[0], r[1], r[2], r[3]};
    }
  }
  b.codes[which ? lane * kPageBlock + old : old * kHeadDim + lane] = (uint8_t)code;
  // (the wave has read the scale: the factors above come from it)
  if (lane == 0) *b.scale = exp_scale(n.e);
}

// ---------------------------------------------------------------------------
// Page tables
// ---------------------------------------------------------------------------
// One block finds the new tables, many copy the pages.  The first is a chain of steps
// between barriers, so everything that fits stays in LDS: the pages' two bits (kept by
// some sequence, kept as a full page by some), what is known of each sequence, the old
// table, the free pages that are given out.  Free pages are counted by the bits, a
// word's 32 at once.  Who keeps a partly filled page is settled in a word per page of
// the workspace, which only the sequences' last pages touch.
constexpr int32_t kNobody = 0x7fffffff;
constexpr int TB_NT = 1024, TB_WORDS = 8192, TB_SPOTS = 4096, TB_SEQS = 1024, TB_ENTRIES = 8192;
// Bytes of a page that a block copies at a time, 16 a thread (16384 in four loads each,
// which leave fewer blocks: 120 beams' last pages, 13 MB read and written, 16 us instead of 4).
constexpr int TB_CHUNK = 4096;

struct SeqArrays {             // of each sequence
  int32_t *parent, *length;    // it goes on from (or -1), positions it keeps
  int32_t *full, *kept, *want; // pages: full ones, all kept, wanted
  int32_t *first_ask, *from;   // asks before its own; the page that it gets a copy of, or -1
  int32_t *gap;                // the first entry without a page
};
__host__ __device__ inline SeqArrays seq_arrays(int32_t* p, int n) {
  return {p, p + n, p + 2 * (int64_t)n, p + 3 * (int64_t)n, p + 4 * (int64_t)n, p + 5 * (int64_t)n, p + 6 * (int64_t)n, p + 7 * (int64_t)n};
}
struct TablesWork {            // words of the workspace
  int32_t* counts;             // pages to copy
  int32_t* pairs;              // [pages + sequences][2] from, to
  int32_t* owner;              // [pages] of a last page: s + 1
  int32_t* to;                 // [pages] where a page moves
  int32_t* spots;              // [pages] free pages, in order
  uint32_t *used, *full;       // a bit per page
  SeqArrays seq;
  int32_t* old_table;          // [sequences][columns]
};
__host__ __device__ inline TablesWork tables_work(int32_t* ws, int sequences, int columns, int pages) {
  TablesWork w;
  const int words = (pages + 31) / 32;
  w.counts = ws;
  w.pairs = w.counts + 16;
  w.owner = w.pairs + 2 * ((int64_t)pages + sequences);
  w.to = w.owner + pages;
  w.spots = w.to + pages;
  w.used = (uint32_t*)w.spots + pages;
  w.full = w.used + words;
  int32_t* p = (int32_t*)w.full + words;
  w.seq = seq_arrays(p, sequences);
  w.old_table = p + 8 * (int64_t)sequences;
  return w;
}

struct TablesLds {
  uint32_t used[TB_WORDS], full[TB_WORDS];
  int32_t spots[TB_SPOTS], seq[8 * TB_SEQS], table[TB_ENTRIES];
  int sums[16];
  int copies;
};

// Exclusive sum over the block's 1024 threads; *total gets the sum of all.
__device__ __forceinline__ int block_scan(int v, int* sums, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int x = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 63) sums[wave] = x;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    if (i < wave) before += sums[i];
    all += sums[i];
  }
  *total = all;
  return before + x - v;
}

// IN: the bits and what is known of the sequences fit in LDS.
template <bool IN>
__global__ __launch_bounds__(TB_NT) void k_next_tables(TablesLaunch a, bool in_place) {
  extern __shared__ __attribute__((aligned(16))) char tables_lds[];
  TablesLds& l = *(TablesLds*)tables_lds;
  const TablesWork w = tables_work(a.ws, a.sequences, a.columns, a.pages);
  const int tid = threadIdx.x, n = a.sequences, words = (a.pages + 31) / 32;
  const SeqArrays q = IN ? seq_arrays(l.seq, TB_SEQS) : w.seq;
  uint32_t *used = IN ? l.used : w.used, *full = IN ? l.full : w.full;
  const auto clear_word = [&](uint32_t* p) {
    if constexpr (IN) *p = 0; else store_agent(p, 0u);
  };
  const auto word_of = [&](const uint32_t* p) -> uint32_t {
    if constexpr (IN) return *p; else return load_agent(p);
  };
  const auto is_page = [&](int p) { return p >= 0 && p < a.pages; };

  // the old table, where its entries are read twice from near or would be overwritten
  const int entries = n * a.columns;       // (at most 2^26)
  const bool near = entries <= TB_ENTRIES;
  const int32_t* table = a.table;
  int64_t ld = a.table_ld;
  if (near || in_place) {
    int32_t* copy = near ? l.table : w.old_table;
    for (int i = tid; i < entries; i += TB_NT) copy[i] = a.table[i / a.columns * a.table_ld + i % a.columns];
    table = copy, ld = a.columns;
  }
  for (int i = tid; i < words; i += TB_NT) clear_word(&used[i]), clear_word(&full[i]);
  const int most = a.columns * a.page;
  for (int s = tid; s < n; s += TB_NT) {
    const int parent = a.parent ? a.parent[s] : s, want = a.want ? min(max(a.want[s], 0), most) : 0;
    const bool goes_on = parent >= 0 && parent < n;
    const int length = goes_on ? min(max(a.length[parent], 0), most) : 0;
    const int whole = length / a.page, kept = whole + (whole * a.page < length);
    q.parent[s] = goes_on ? parent : -1;
    q.length[s] = length;
    q.full[s] = whole;
    q.kept[s] = kept;
    q.want[s] = max(kept, (want + a.page - 1) / a.page);
    q.gap[s] = a.columns;
    if (whole < kept) {
      const int p = a.table[parent * a.table_ld + whole];
      if (is_page(p)) store_agent(&w.owner[p], kNobody);
    }
  }
  if (tid == 0) l.copies = 0;
  // (the atomics of other waves come behind these stores in the L2)
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();

  // what is kept, by whom
  for (int i = tid; i < entries; i += TB_NT) {
    const int s = i / a.columns, j = i - s * a.columns;
    if (j >= q.kept[s]) continue;
    const int p = table[q.parent[s] * ld + j];
    if (!is_page(p)) continue;
    atomicOr(&used[p >> 5], 1u << (p & 31));
    if (j < q.full[s])
      atomicOr(&full[p >> 5], 1u << (p & 31));
    else
      atomicMin(&w.owner[p], s + 1);
  }
  __syncthreads();
  // asks of each sequence
  int asked = 0;
  for (int s0 = 0; s0 < n; s0 += TB_NT) {
    const int s = s0 + tid;
    int mine = 0;
    if (s < n) {
      int from = -1;
      if (q.full[s] < q.kept[s]) {
        const int p = table[q.parent[s] * ld + q.full[s]];
        if (is_page(p) && ((word_of(&full[p >> 5]) >> (p & 31) & 1) || load_agent(&w.owner[p]) != s + 1)) from = p;
      }
      q.from[s] = from;
      mine = (from >= 0) + q.want[s] - q.kept[s];
    }
    int total;
    const int before = block_scan(mine, l.sums, &total);
    if (s < n) q.first_ask[s] = asked + before;
    asked += total;
  }
  // free pages: a thread's words lie together
  const int per = (words + TB_NT - 1) / TB_NT, first = min(tid * per, words), end = min(first + per, words);
  const auto pages_of = [&](int i) { return i * 32 + 32 <= a.pages ? 0xffffffffu : (1u << (a.pages & 31)) - 1; };
  int free = 0, free_before = 0, mine = 0;
  for (int i = first; i < end; ++i) mine += __popc(~word_of(&used[i]) & pages_of(i));
  free_before = block_scan(mine, l.sums, &free);
  const int granted = min(asked, free), in_use = a.pages - free + granted;
  const auto behind = [&](int i) {         // the bits of pages from in_use on
    return i * 32 >= in_use ? 0xffffffffu : i * 32 + 32 <= in_use ? 0u : 0xffffffffu << (in_use & 31);
  };
  int moves = 0, moves_before = 0;
  if (a.compact) {
    mine = 0;
    for (int i = first; i < end; ++i) mine += __popc(word_of(&used[i]) & behind(i));
    moves_before = block_scan(mine, l.sums, &moves);
  }
  // the first of them, as many as are given out
  const int need = moves + granted;
  int32_t* spots = need <= TB_SPOTS ? l.spots : w.spots;
  for (int i = first; i < end && free_before < need; ++i)
    for (uint32_t bits = ~word_of(&used[i]) & pages_of(i); bits && free_before < need; bits &= bits - 1)
      spots[free_before++] = i * 32 + __ffs(bits) - 1;
  __syncthreads();
  if (moves) {
    for (int i = first; i < end; ++i)
      for (uint32_t bits = word_of(&used[i]) & behind(i); bits; bits &= bits - 1) {
        const int p = i * 32 + __ffs(bits) - 1, to = spots[moves_before];
        w.to[p] = to;
        *(int2*)&w.pairs[2 * moves_before++] = int2{p, to};
      }
    __syncthreads();
  }
  // tables
  for (int i = tid; i < entries; i += TB_NT) {
    const int s = i / a.columns, j = i - s * a.columns, kept = q.kept[s], from = q.from[s];
    const bool copied = from >= 0 && j == q.full[s];
    int p = -1;
    if (j < kept && !copied) {
      p = table[q.parent[s] * ld + j];
      p = !is_page(p) ? -1 : moves && p >= in_use ? w.to[p] : p;
    } else if (j < q.want[s]) {
      const int ask = q.first_ask[s] + (copied ? 0 : (from >= 0) + j - kept);
      p = ask < granted ? spots[moves + ask] : -1;
      if (copied && p >= 0) *(int2*)&w.pairs[2 * (moves + atomicAdd(&l.copies, 1))] = int2{from, p};
    }
    a.new_table[s * a.new_ld + j] = p;
    if (p < 0) atomicMin(&q.gap[s], j);
  }
  __syncthreads();
  for (int s = tid; s < n; s += TB_NT) {
    a.new_length[s] = q.length[s];
    if (a.room) {
      if constexpr (IN) a.room[s] = q.gap[s] * a.page; else a.room[s] = load_agent(&q.gap[s]) * a.page;
    }
  }
  if (tid == 0) {
    w.counts[0] = moves + l.copies;
    if (a.info) a.info[0] = in_use, a.info[1] = asked - granted, a.info[2] = l.copies, a.info[3] = moves;
  }
}

template <typename V>
__device__ __forceinline__ void copy_bytes(const char* from, char* to, int64_t begin, int64_t end) {
  for (int64_t i = begin + threadIdx.x * sizeof(V); i < end; i += 256 * sizeof(V)) *(V*)(to + i) = *(const V*)(from + i);
}
// Chunks of pages, over all that are to be copied.  None of them is copied from and to.
template <typename V>
__global__ __launch_bounds__(256) void k_copy_pages(TablesLaunch a, uint32_t chunks) {
  const TablesWork w = tables_work(a.ws, a.sequences, a.columns, a.pages);
  const uint32_t units = (uint32_t)w.counts[0] * chunks;      // (of memory that is there, so below 2^32)
  for (uint32_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int2 pair = *(const int2*)&w.pairs[2 * (u / chunks)];
    const int64_t begin = (int64_t)(u % chunks) * TB_CHUNK;
    copy_bytes<V>((const char*)a.codes + pair.x * a.code_stride, (char*)a.codes + pair.y * a.code_stride, begin,
                  min(begin + TB_CHUNK, a.code_bytes));
    if (begin == 0)
      copy_bytes<uint32_t>((const char*)a.scales + pair.x * a.scale_stride, (char*)a.scales + pair.y * a.scale_stride, 0, a.scale_bytes);
  }
}

}  // namespace

void write_pages(const PageWriteLaunch& a, bool bf16, hipStream_t s) {
  if (a.max_new == 1) {
    const unsigned blocks = (unsigned)(((int64_t)a.c.sequences * a.c.kv_heads * 2 + 3) / 4);
    if (bf16)
      k_write_step<bf16_t><<<dim3(blocks), 256, 0, s>>>(a);
    else
      k_write_step<float><<<dim3(blocks), 256, 0, s>>>(a);
    return;
  }
  const int touched = (int)(((int64_t)a.max_new + 2 * kPageBlock - 2) / kPageBlock);
  const unsigned blocks = (unsigned)((int64_t)a.c.sequences * touched * a.c.kv_heads * 2);
  if (bf16)
    k_write_pages<bf16_t><<<dim3(blocks), 256, 0, s>>>(a, touched);
  else
    k_write_pages<float><<<dim3(blocks), 256, 0, s>>>(a, touched);
}

int64_t tables_ws_words(int sequences, int columns, int pages) {
  return 16 + 5 * (int64_t)pages + 2 * (int64_t)((pages + 31) / 32) + 10 * (int64_t)sequences + (int64_t)sequences * columns;
}

hipError_t next_tables(const TablesLaunch& a, hipStream_t s) {
  const bool in_place = (const int32_t*)a.new_table == a.table, in = a.pages <= 32 * TB_WORDS && a.sequences <= TB_SEQS;
  const auto kernel = in ? k_next_tables<true> : k_next_tables<false>;
  const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, sizeof(TablesLds));
  if (e != hipSuccess) return e;
  kernel<<<1, TB_NT, sizeof(TablesLds), s>>>(a, in_place);
  if (!a.codes && !a.scales) return hipSuccess;
  const int chunks = (int)std::max<int64_t>(1, (a.code_bytes + TB_CHUNK - 1) / TB_CHUNK);
  const int64_t most = ((int64_t)a.sequences + (a.compact ? a.pages : 0)) * chunks;
  if (most == 0) return hipSuccess;
  const unsigned blocks = (unsigned)std::min<int64_t>(most, 8192);
  const bool wide = !(((uintptr_t)a.codes | (uint64_t)a.code_stride | (uint64_t)a.code_bytes) & 15);
  if (wide)
    k_copy_pages<uint4><<<dim3(blocks), 256, 0, s>>>(a, chunks);
  else
    k_copy_pages<uint32_t><<<dim3(blocks), 256, 0, s>>>(a, chunks);
  return hipSuccess;
}

}  // namespace asr
