// A cache in pages of e4m3 codes: new keys and values into it (asr_write_pages)
// and the page tables of a next step (asr_next_tables).
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

// One block of 256 threads per (sequence, touched block of positions, head, keys or
// values); thread = (position, 16 dims).
template <typename T>
__global__ __launch_bounds__(256) void k_write_pages(PageWriteLaunch a, int touched) {
  __shared__ uint32_t tops[4];
  __shared__ __attribute__((aligned(16))) uint8_t turn[64 * 80];
  const int tid = threadIdx.x;
  uint32_t u = blockIdx.x;
  const int which = u & 1;
  u >>= 1;
  const int head = (int)(u % a.c.kv_heads);
  u /= a.c.kv_heads;
  const int nth = (int)(u % touched), seq = (int)(u / touched);
  const int length = a.length[seq];
  int start = a.token_start ? a.token_start[seq] : seq, end = a.token_start ? a.token_start[seq + 1] : seq + 1;
  start = max(start, 0);
  end = min(min(end, a.tokens), start > INT32_MAX - a.max_new ? INT32_MAX : start + a.max_new);
  if (length < 0 || end <= start) return;
  const int64_t block = (int64_t)length / kPageBlock + nth, p0 = block * kPageBlock;
  const int64_t stop = min((int64_t)length + (end - start), (int64_t)a.c.columns * a.c.page);
  if (p0 >= stop) return;
  const int old = (int)max((int64_t)length - p0, (int64_t)0), last = (int)min(stop - p0, (int64_t)kPageBlock);
  const int page = a.c.table[(int64_t)seq * a.c.table_ld + p0 / a.c.page];
  if (page < 0 || page >= a.c.pages) return;
  const int per = a.c.page / kPageBlock;
  const int64_t at = ((int64_t)which * a.c.kv_heads + head) * per + (p0 % a.c.page) / kPageBlock;
  uint8_t* codes = a.c.codes + page * a.c.page_stride + at * (kPageBlock * kHeadDim);
  float* scale = a.c.scales + page * a.c.scale_stride + at;

  const int pos = tid >> 2, d0 = (tid & 3) * 16;
  const bool fresh = pos >= old && pos < last;
  float x[16];
  uint32_t top = 0;
  if (fresh) {
    const T* src = (const T*)(which ? a.v : a.k) + (start + (p0 + pos - length)) * a.ld + head * kHeadDim + d0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      x[i] = St<T>::ld(src, i);
      top = max(top, magnitude(x[i]));
    }
  }
  top = wave_max_u32(top);
  if ((tid & 63) == 0) tops[tid >> 6] = top;
  __syncthreads();
  top = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
  int e = need_exp(top);
  float by = 1.f;
  bool grew = false;
  if (old > 0) {
    const float s = *scale;
    e = max(e, held_exp(s));
    grew = s != exp_scale(e);
    by = (s > 0.f ? s : exp_scale(kLeastScale)) / exp_scale(e);
  }
  const float inv = exp_scale(254 - e);
  uint32_t w[4] = {0, 0, 0, 0};
  if (fresh) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float y[4] = {x[4 * i] * inv, x[4 * i + 1] * inv, x[4 * i + 2] * inv, x[4 * i + 3] * inv};
      w[i] = code4(y);
    }
  }
  if (which == 0) {
    uint8_t* p = codes + pos * kHeadDim + d0;
    if (fresh) {
      *(uint4*)p = uint4{w[0], w[1], w[2], w[3]};
    } else if (grew && pos < old) {
      const uint4 c = *(const uint4*)p;
      *(uint4*)p = uint4{rescale4(c.x, by), rescale4(c.y, by), rescale4(c.z, by), rescale4(c.w, by)};
    }
  } else {
    // values lie [dim][position]: thread = (dim, 16 positions)
    if (fresh)
      for (int i = 0; i < 16; ++i) turn[(d0 + i) * 80 + pos] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
    __syncthreads();
    const int dim = tid >> 2, t0 = (tid & 3) * 16;
    uint8_t* p = codes + dim * kPageBlock + t0;
    const int from = grew ? 0 : old;
    if (t0 + 16 <= from || t0 >= last) goto done;
    {
      uint32_t c[4];
      for (int i = 0; i < 4; ++i) c[i] = *(const uint32_t*)(turn + dim * 80 + t0 + 4 * i);
      if (grew && t0 < old) {
        const uint4 o = *(const uint4*)p;
        const uint32_t r[4] = {rescale4(o.x, by), rescale4(o.y, by), rescale4(o.z, by), rescale4(o.w, by)};
        for (int i = 0; i < 16; ++i)
          if (t0 + i < old) c[i >> 2] = (c[i >> 2] & ~(0xffu << (8 * (i & 3)))) | (r[i >> 2] & (0xffu << (8 * (i & 3))));
      }
      store_some(p, c, from - t0, last - t0);
    }
  }
done:
  __syncthreads();
  if (tid == 0) *scale = exp_scale(e);
}

// ---------------------------------------------------------------------------
// Page tables
// ---------------------------------------------------------------------------
constexpr int32_t kNobody = 0x7fffffff;

struct TablesWork {          // words of the workspace
  int32_t* owner;            // [pages] 0: read by some, s + 1: written by s
  int32_t* to;               // [pages] where a page moves, itself otherwise
  int32_t* spots;            // [pages] free pages, in order
  int32_t* first_ask;        // [sequences + 1] asks before a sequence's
  int32_t* copy_from;        // [sequences] page that a sequence has a copy of, or -1
  int32_t* copy_to;
  int32_t* counts;           // moves
  int32_t* old_table;        // [sequences][columns], [sequences]
  int32_t* old_length;
};
__host__ __device__ inline TablesWork tables_work(int32_t* ws, int sequences, int columns, int pages) {
  TablesWork w;
  w.owner = ws;
  w.to = w.owner + pages;
  w.spots = w.to + pages;
  w.first_ask = w.spots + pages;
  w.copy_from = w.first_ask + sequences + 1;
  w.copy_to = w.copy_from + sequences;
  w.counts = w.copy_to + sequences;
  w.old_length = w.counts + 16;
  w.old_table = w.old_length + sequences;
  return w;
}

struct NextSeq {
  int parent, length, full, kept, want;      // pages: full ones, all kept, wanted
};
__device__ __forceinline__ NextSeq next_seq(const TablesLaunch& a, const int32_t* lengths, int s) {
  NextSeq n;
  n.parent = a.parent ? a.parent[s] : s;
  const int most = a.columns * a.page;
  n.length = n.parent >= 0 && n.parent < a.sequences ? min(max(lengths[n.parent], 0), most) : 0;
  n.full = n.length / a.page;
  n.kept = (n.length + a.page - 1) / a.page;
  const int want = a.want ? min(max(a.want[s], 0), most) : 0;
  n.want = max(n.kept, (want + a.page - 1) / a.page);
  return n;
}

// Exclusive sum over the block's 1024 threads; *total gets the sum of all.
__device__ __forceinline__ int block_scan(int v, int* total) {
  __shared__ int sums[16];
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
  for (int i = 0; i < 16; ++i) {
    if (i < wave) before += sums[i];
    all += sums[i];
  }
  *total = all;
  return before + x - v;
}

// One block: claims, asks, free pages, tables.
__global__ __launch_bounds__(1024) void k_next_tables(TablesLaunch a, bool in_place) {
  const TablesWork w = tables_work(a.ws, a.sequences, a.columns, a.pages);
  const int tid = threadIdx.x;
  const int32_t *table = a.table, *lengths = a.length;
  int64_t ld = a.table_ld;
  if (in_place) {
    for (int64_t i = tid; i < (int64_t)a.sequences * a.columns; i += 1024) w.old_table[i] = a.table[i / a.columns * a.table_ld + i % a.columns];
    for (int i = tid; i < a.sequences; i += 1024) w.old_length[i] = a.length[i];
    table = w.old_table, lengths = w.old_length, ld = a.columns;
  }
  for (int i = tid; i < a.pages; i += 1024) store_agent(&w.owner[i], kNobody);
  __threadfence_block();
  __syncthreads();
  const int wave = tid >> 6, lane = tid & 63;
  for (int s = wave; s < a.sequences; s += 16) {
    const NextSeq n = next_seq(a, lengths, s);
    for (int j = lane; j < n.kept; j += 64) {
      const int p = table[n.parent * ld + j];
      if (p >= 0 && p < a.pages) atomicMin(&w.owner[p], j < n.full ? 0 : s + 1);
    }
  }
  __syncthreads();
  // asks of each sequence
  int asked = 0;
  for (int s0 = 0; s0 < a.sequences; s0 += 1024) {
    const int s = s0 + tid;
    int mine = 0;
    if (s < a.sequences) {
      const NextSeq n = next_seq(a, lengths, s);
      int from = -1;
      if (n.full < n.kept) {
        const int p = table[n.parent * ld + n.full];
        if (p >= 0 && p < a.pages && load_agent(&w.owner[p]) != s + 1) from = p;
      }
      w.copy_from[s] = from;
      w.copy_to[s] = -1;
      mine = (from >= 0) + n.want - n.kept;
    }
    int total;
    const int before = block_scan(mine, &total);
    if (s < a.sequences) w.first_ask[s] = asked + before;
    asked += total;
  }
  // free pages in order
  int free = 0;
  for (int p0 = 0; p0 < a.pages; p0 += 1024) {
    const int p = p0 + tid;
    const int is = p < a.pages && load_agent(&w.owner[p]) == kNobody;
    int total;
    const int before = block_scan(is, &total);
    if (is) w.spots[free + before] = p;
    if (p < a.pages) w.to[p] = p;
    free += total;
  }
  __syncthreads();
  const int granted = min(asked, free), in_use = a.pages - free + granted;
  int moves = 0;
  if (a.compact) {
    for (int p0 = 0; p0 < a.pages; p0 += 1024) {
      const int p = p0 + tid;
      const int is = p < a.pages && p >= in_use && load_agent(&w.owner[p]) != kNobody;
      int total;
      const int before = block_scan(is, &total);
      if (is) w.to[p] = w.spots[moves + before];
      moves += total;
    }
    __syncthreads();
  }
  // tables
  int copies = 0;
  for (int s = wave; s < a.sequences; s += 16) {
    const NextSeq n = next_seq(a, lengths, s);
    const int from = w.copy_from[s], ask0 = w.first_ask[s];
    int32_t* row = a.new_table + s * a.new_ld;
    int gap = a.columns;
    for (int j0 = 0; j0 < a.columns; j0 += 64) {
      const int j = j0 + lane;
      int p = -1;
      if (j < n.kept && !(j == n.full && from >= 0)) {
        p = table[n.parent * ld + j];
        p = p >= 0 && p < a.pages ? w.to[p] : -1;
      } else if (j < n.want) {
        const int ask = ask0 + (j < n.kept ? 0 : (from >= 0) + j - n.kept);
        p = ask < granted ? w.spots[moves + ask] : -1;
        if (j < n.kept) {
          w.copy_to[s] = p;
          copies += p >= 0;
        }
      }
      if (j < a.columns) row[j] = p;
      const uint64_t holes = __ballot(p < 0);
      if (gap == a.columns && holes) gap = min(a.columns, j0 + __ffsll((unsigned long long)holes) - 1);
    }
    if (lane == 0) {
      a.new_length[s] = n.length;
      if (a.room) a.room[s] = gap * a.page;
    }
  }
  int total;
  block_scan(copies, &total);
  if (tid == 0) {
    w.counts[0] = moves;
    if (a.info) a.info[0] = in_use, a.info[1] = asked - granted, a.info[2] = total, a.info[3] = moves;
  }
}

// One block per sequence's copy, then per page that may move.
__global__ __launch_bounds__(256) void k_copy_pages(TablesLaunch a) {
  const TablesWork w = tables_work(a.ws, a.sequences, a.columns, a.pages);
  int src, dst;
  if (blockIdx.x < (uint32_t)a.sequences) {
    src = w.copy_from[blockIdx.x], dst = w.copy_to[blockIdx.x];
    if (dst < 0) return;
  } else {
    src = blockIdx.x - a.sequences;
    dst = w.to[src];
    if (dst == src) return;
  }
  const uint32_t* c = (const uint32_t*)((const char*)a.codes + src * a.code_stride);
  uint32_t* d = (uint32_t*)((char*)a.codes + dst * a.code_stride);
  for (int64_t i = threadIdx.x; i < a.code_bytes / 4; i += 256) d[i] = c[i];
  c = (const uint32_t*)((const char*)a.scales + src * a.scale_stride);
  d = (uint32_t*)((char*)a.scales + dst * a.scale_stride);
  for (int64_t i = threadIdx.x; i < a.scale_bytes / 4; i += 256) d[i] = c[i];
}

}  // namespace

void write_pages(const PageWriteLaunch& a, bool bf16, hipStream_t s) {
  const int touched = (int)(((int64_t)a.max_new + 2 * kPageBlock - 2) / kPageBlock);
  const unsigned blocks = (unsigned)((int64_t)a.c.sequences * touched * a.c.kv_heads * 2);
  if (bf16)
    k_write_pages<bf16_t><<<dim3(blocks), 256, 0, s>>>(a, touched);
  else
    k_write_pages<float><<<dim3(blocks), 256, 0, s>>>(a, touched);
}

int64_t tables_ws_words(int sequences, int columns, int pages) {
  return 3 * (int64_t)pages + 4 * (int64_t)sequences + 17 + (int64_t)sequences * columns;
}

void next_tables(const TablesLaunch& a, hipStream_t s) {
  k_next_tables<<<1, 1024, 0, s>>>(a, (const int32_t*)a.new_table == a.table);
  if (a.codes || a.scales) k_copy_pages<<<dim3((unsigned)(a.sequences + (a.compact ? a.pages : 0))), 256, 0, s>>>(a);
}

}  // namespace asr
