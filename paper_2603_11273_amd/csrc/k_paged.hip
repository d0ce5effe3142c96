// Attention of new tokens over the pages of their sequence (asr_attend_pages).
#include "asr_device.h"

namespace asr {
namespace {

typedef float f32x2v __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void values4(uint32_t c, float* x) {
  const f32x2v a = __builtin_amdgcn_cvt_pk_f32_fp8(c, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(c, true);
  x[0] = a.x, x[1] = a.y, x[2] = b.x, x[3] = b.y;
}

// One wave per (row, query head) over blocks of 64 keys: lane = key for the scores,
// lane = dim for the values.
template <typename T>
__global__ __launch_bounds__(64) void k_attend_pages(PagedLaunch a) {
  __shared__ float q[kHeadDim], p[kPageBlock];
  const int lane = threadIdx.x, h = (int)(blockIdx.x % a.n_head), row = (int)(blockIdx.x / a.n_head);
  int seq = -1;
  if (a.row_start) {
    int lo = 0, hi = a.c.sequences;          // the last sequence that starts at or before the row
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (a.row_start[mid] <= row) lo = mid + 1; else hi = mid;
    }
    seq = lo - 1;
    if (seq < 0 || row >= a.row_start[seq + 1] || row - a.row_start[seq] >= a.max_rows || a.row_start[seq] < 0) return;
  } else {
    seq = row;
    if (seq >= a.c.sequences) return;
  }
  const int head = h / (a.n_head / a.c.kv_heads), per = a.c.page / kPageBlock;
  const int first = a.first ? max(a.first[row], 0) : 0;
  const int n = (int)min((int64_t)min(a.length[row], a.max_keys), (int64_t)a.c.columns * a.c.page);
  q[lane] = a.q[row * a.q_ld + h * kHeadDim + lane] * a.qmul;
  float M = -INFINITY, L = 0.f, acc = 0.f;
  bool any = false;
  for (int b = first / kPageBlock; b * kPageBlock < n; ++b) {
    const int page = a.c.table[(int64_t)seq * a.c.table_ld + b / per];
    if (page < 0 || page >= a.c.pages) continue;
    const int64_t at = (int64_t)head * per + b % per, vat = at + (int64_t)a.c.kv_heads * per;
    const uint8_t* codes = a.c.codes + page * a.c.page_stride;
    const float* scales = a.c.scales + page * a.c.scale_stride;
    const int key = b * kPageBlock + lane;
    const bool sees = key >= first && key < n;
    if (!__any(sees)) continue;
    any = true;
    __syncthreads();
    float s = 0.f;
    const uint4* k = (const uint4*)(codes + (at * kPageBlock + lane) * kHeadDim);
    for (int i = 0; i < 4; ++i) {
      const uint4 c = k[i];
      const uint32_t w[4] = {c.x, c.y, c.z, c.w};
      for (int j = 0; j < 4; ++j) {
        float x[4];
        values4(w[j], x);
        for (int d = 0; d < 4; ++d) s = fmaf(x[d], q[16 * i + 4 * j + d], s);
      }
    }
    s = sees ? s * scales[at] : -INFINITY;
    const bool bad = __any(sees && s != s);
    const float top = fmaxf(M, wave_max(s));
    const float ref = top == -INFINITY ? 0.f : top;
    const float keep = M == top ? 1.f : exp2f(M - ref);
    M = top;
    const float e = sees ? exp2f(s - ref) : 0.f;
    L = bad ? NAN : L * keep + wave_sum(e);
    p[lane] = e;
    __syncthreads();
    const uint4* v = (const uint4*)(codes + (vat * kPageBlock + lane) * kPageBlock);
    float sum = 0.f;
    for (int i = 0; i < 4; ++i) {
      const uint4 c = v[i];
      const uint32_t w[4] = {c.x, c.y, c.z, c.w};
      for (int j = 0; j < 4; ++j) {
        float x[4];
        values4(w[j], x);
        for (int d = 0; d < 4; ++d) {
          const int at_key = b * kPageBlock + 16 * i + 4 * j + d;
          if (at_key >= first && at_key < n) sum = fmaf(x[d], p[16 * i + 4 * j + d], sum);
        }
      }
    }
    acc = acc * keep + sum * scales[vat];
  }
  St<T>::st((T*)a.out, row * a.out_ld + h * kHeadDim + lane, any ? acc / L : 0.f);
}

}  // namespace

hipError_t attend_pages(const PagedLaunch& a, bool bf16, hipStream_t s) {
  const unsigned blocks = (unsigned)((int64_t)a.rows * a.n_head);
  if (bf16)
    k_attend_pages<bf16_t><<<dim3(blocks), 64, 0, s>>>(a);
  else
    k_attend_pages<float><<<dim3(blocks), 64, 0, s>>>(a);
  return hipSuccess;
}

}  // namespace asr
