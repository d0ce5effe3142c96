// Entry points of the stateless operators: argument checks, the split of the work,
// and the launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <exception>
#include <string>

#include "asr_kernels.h"
#include "errors.h"

using namespace asr;

namespace {

bool aligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

template <class F>
asr_status guarded(F&& f) {
  try {
    return f();
  } catch (const std::exception&) {
    return ASR_EDEVICE;   // (only a message can fail to be made)
  }
}

asr_status launched(hipError_t e) {
  if (e == hipSuccess) e = hipGetLastError();
  return e == hipSuccess ? ASR_OK : fail(ASR_EDEVICE, std::string("kernel launch: ") + hipGetErrorString(e));
}

// ---------------------------------------------------------------------------
// Attention over shared keys
// ---------------------------------------------------------------------------
asr_status check_keys(const asr_keys& c, int32_t most, int es, const char* name) {
  const std::string n(name);
  if (most == 0) return ASR_OK;
  if (!c.k || !c.v) return fail(ASR_EINVAL, n + ": NULL keys or values");
  if (!aligned(c.k, 16) || !aligned(c.v, 16)) return fail(ASR_EINVAL, n + ": keys and values must be 16-byte aligned");
  if (c.slots <= 0 || c.positions <= 0) return fail(ASR_EINVAL, n + ": slots and positions must be positive");
  if (most > c.positions) return fail(ASR_EINVAL, n + ": more keys than positions");
  const int64_t unit = 16 / es;
  if (c.slot_stride < 0 || c.head_stride < 0 || c.slot_stride % unit || c.head_stride % unit || c.pos_stride % unit)
    return fail(ASR_EINVAL, n + ": strides must be multiples of 16 bytes");
  // (a tile of 32 keys is addressed with 32 bits)
  if (c.pos_stride < kHeadDim || c.pos_stride * es > 262144)
    return fail(ASR_EINVAL, n + ": pos_stride out of [64 elements, 262144 bytes]");
  return ASR_OK;
}

int cu_count() {
  static const int n = [] {
    int dev = 0, v = 0;
    if (hipGetDevice(&dev) != hipSuccess ||
        hipDeviceGetAttribute(&v, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || v <= 0) {
      (void)hipGetLastError();
      v = 256;                                         // (sizes asked for without a GPU)
    }
    return v;
  }();
  return n;
}

ShareKeys keys_of(const asr_keys& c, int32_t most) {
  return {c.k, c.v, c.slot_stride, c.head_stride, c.pos_stride, c.slot, c.first, c.len, c.slots, c.positions, most};
}

int parts_of(int keys, int part) { return (int)(((int64_t)keys + part - 1) / part); }

// Keys per part, `keys` at most for each of `units` (a group's queries and a cache
// head, or a row and one).  One block per CU reads nearly as fast as several, so
// with P parts a unit the work takes ceil(units P / CUs) turns of keys / P keys
// and what a part costs besides (its first loads, its records), `fixed` keys'
// worth; only the largest P of 1, 2, .. turns come into question.  Measured
// (bf16, 20 heads, us): 8 groups of 16 rows on 65536 keys in parts of 2048 /
// 4096 / 8192 / 16384 487 / 446 / 426 / 455, the rule's 8192; 64 rows on 30011
// in 1024 / 1536 / 2560 / 4096 64 / 59 / 52 / 60, the rule's 2560; 24 x 5 on 1500
// in 512 / 768 / 1536 51 / 50 / 49, the rule's one part.  Lengths that may differ
// need more parts, as the longest unit would be last: 16 groups on 515 to 8191
// keys in 768 / 1408 / 2048 41 / 43 / 48, hence three turns at least.
int part_keys(int64_t units, int64_t keys, bool ragged, int fixed, int step) {
  if (keys <= step) return step;
  const int64_t cus = cu_count();
  int64_t best = step, best_cost = INT64_MAX;
  for (int64_t turns = ragged ? 3 : 1; turns <= 8; ++turns) {
    const int64_t p = std::max<int64_t>(1, cus * turns / units);
    const int64_t n = ((keys + p - 1) / p + step - 1) / step * step;
    const int64_t cost = (units * ((keys + n - 1) / n) + cus - 1) / cus * (n + fixed);
    if (cost < best_cost) best = n, best_cost = cost;
  }
  return (int)best;
}

// The shared keys of groups of different lengths, `part` the part of the rule above.
// While the parts are few (up to four blocks a CU) all start at once and whole CUs
// get long ones or short ones.  So parts of n, as many as pay: lengths all over [0,
// keys] cost units keys / 2 keys, units keys / n / 2 times `fixed`, both shared by
// the CUs, the last part (n) and the join of keys / n records, `record` keys' worth
// each, least at n = sqrt(keys (units fixed / 2 CUs + record)).  96 sets of groups
// of at random 1 to 65536 keys: 6.1 % less time on average, 12 x 8 units on up to
// 7383 keys 55 -> 43 us, 19 x 12 on 9309 86 -> 60.  With more parts than that the
// CUs even out by themselves, and groups that turn out alike would only pay for
// theirs (8 x 20 units on 65536 keys 425 -> 466).
int part_keys_ragged(int64_t units, int64_t keys, int part, int fixed, int record, int step) {
  const int64_t cus = cu_count();
  if (keys <= part || units * ((keys + part - 1) / part) > 4 * cus) return part;
  const double least = std::sqrt((double)keys * ((double)units * fixed / (2.0 * cus) + record));
  const int64_t n = std::max<int64_t>(1, std::llround(least / step)) * step, parts = (keys + n - 1) / n;
  return (int)((keys + parts - 1) / parts + step - 1) / step * step;
}

asr_status plan_attention(const asr_attention* a, ShareLaunch* s, size_t* bytes) {
  if (!a) return fail(ASR_EINVAL, "NULL argument");
  if (a->dtype != ASR_F32 && a->dtype != ASR_BF16) return fail(ASR_EINVAL, "dtype");
  const int es = a->dtype == ASR_BF16 ? 2 : 4;
  if (a->n_head <= 0 || a->n_kv_head <= 0 || a->n_head % a->n_kv_head || a->n_head > 65536)
    return fail(ASR_EINVAL, "n_kv_head must divide n_head (at most 65536)");
  if (a->rows < 0 || a->groups < 0 || a->max_prefix < 0 || a->max_own < 0) return fail(ASR_EINVAL, "negative size");
  if (a->rows > 0 && (a->max_group < 1 || a->max_group > a->rows)) return fail(ASR_EINVAL, "max_group out of [1, rows]");
  if (a->part_keys != 0 && (a->part_keys < 128 || a->part_keys > 8192 || a->part_keys % 128))
    return fail(ASR_EINVAL, "part_keys must be 0 or a multiple of 128, at most 8192");
  if (!std::isfinite(a->scale)) return fail(ASR_EINVAL, "scale");
  asr_status st = check_keys(a->prefix, a->max_prefix, es, "prefix");
  if (st != ASR_OK) return st;
  st = check_keys(a->own, a->max_own, es, "own");
  if (st != ASR_OK) return st;
  s->q = a->q;
  s->q_ld = a->q_ld;
  s->out = a->out;
  s->out_ld = a->out_ld;
  s->qmul = a->scale * 1.4426950408889634f;
  s->group_start = a->group_start;
  s->row_of = a->row_of;
  s->rows = a->rows;
  s->groups = a->groups;
  s->max_group = a->max_group;
  s->n_head = a->n_head;
  s->n_kv = a->n_kv_head;
  s->prefix = keys_of(a->prefix, a->max_prefix);
  s->own = keys_of(a->own, a->max_own);
  const int64_t per = a->n_head / a->n_kv_head, cols = a->max_group * per;
  if (cols > INT32_MAX) return fail(ASR_EINVAL, "too many queries in a group");
  if (a->max_prefix > (1 << 30) || a->max_own > (1 << 30)) return fail(ASR_EINVAL, "more than 2^30 keys");
  const int64_t tile = 16 * share_query_tiles((int)cols), tiles = (cols + tile - 1) / tile, own_tiles = (per + 15) / 16;
  const int64_t units = (int64_t)a->groups * a->n_kv_head * tiles, own_units = (int64_t)a->rows * a->n_kv_head * own_tiles;
  if (a->part_keys) {
    s->prefix_part = s->own_part = a->part_keys;
  } else {
    // (float32: half as many keys in the same bytes, a tile of each wave in half as many)
    const int step = 256 / es;
    const auto fixed = [&](int64_t queries) { return (int)(200 + 10 * std::min<int64_t>(queries, 64)) * 2 / es; };
    const bool ragged = a->groups > 1 && a->prefix.len;
    s->prefix_part = part_keys(std::max<int64_t>(units, 1), a->max_prefix, ragged, fixed(cols), step);
    // (a record in the join: 10 bf16 keys, 5 of float32)
    if (ragged) s->prefix_part = part_keys_ragged(units, a->max_prefix, s->prefix_part, fixed(cols), 20 / es, step);
    s->own_part = part_keys(std::max<int64_t>(own_units, 1), a->max_own, a->rows > 1 && a->own.len, fixed(per), step);
  }
  s->np = parts_of(a->max_prefix, s->prefix_part);
  s->no = parts_of(a->max_own, s->own_part);
  const double blocks = ((double)units * s->np + 8.0 * tiles) + (double)own_units * s->no;
  // (a launch has fewer than 2^32 threads: 256 a block, 64 a row and head)
  if (blocks >= 16777216.0 || (double)a->rows * a->n_head >= 67108864.0) return fail(ASR_EINVAL, "too much work for one call");
  const int64_t parts = s->np + s->no;
  *bytes = parts > 1 ? kCounters * 4 + (size_t)a->rows * a->n_head * parts * (kHeadDim + 2) * 4 : 0;
  return ASR_OK;
}

// ---------------------------------------------------------------------------
// Rules on logits
// ---------------------------------------------------------------------------
asr_status plan_rules(const asr_rules* r, RulesLaunch* s, size_t* bytes) {
  if (!r) return fail(ASR_EINVAL, "NULL argument");
  if (r->dtype != ASR_F32 && r->dtype != ASR_BF16) return fail(ASR_EINVAL, "dtype");
  if (r->rows < 0 || r->rows > 65535) return fail(ASR_EINVAL, "rows out of [0, 65535]");
  if (r->vocab < 1 || r->vocab > kRulesMaxVocab) return fail(ASR_EINVAL, "vocab out of [1, 1048576]");
  if (r->k < 0 || r->k > kRulesMaxK) return fail(ASR_EINVAL, "k out of [0, 16]");
  if (r->sets < 0 || r->masks < 0) return fail(ASR_EINVAL, "negative size");
  // (the kernels step past a list's end with 32 bits)
  constexpr int64_t kMostEntries = 1 << 30;
  if (r->history && (r->history_ld < 0 || r->history_ld > kMostEntries || !r->history_len))
    return fail(ASR_EINVAL, "history needs history_len and a row length of at most 2^30");
  if (r->bias_token && (r->bias_ld < 0 || r->bias_ld > kMostEntries || !r->bias_value || !r->bias_len))
    return fail(ASR_EINVAL, "bias_token needs bias_value, bias_len and a row length of at most 2^30");
  if (r->mask && r->mask_ld < (r->vocab + 31) / 32) return fail(ASR_EINVAL, "mask_ld shorter than the vocabulary");
  *s = {r->logits, r->ld, r->rows, r->vocab, r->sets, r->set, r->history, r->history_ld, r->history_len, r->prompt_len,
        r->repetition, r->frequency, r->presence, r->bias_token, r->bias_value, r->bias_ld, r->bias_len, r->mask,
        r->mask_ld, r->masks, r->mask_of, r->temperature, r->out, r->out_ld, r->k, r->token, r->logprob, nullptr, nullptr};
  *bytes = r->k > 0 ? kCounters * 4 + rules_ws_bytes(r->rows, r->vocab, r->k) : 0;
  return ASR_OK;
}

asr_status check_ws(const void* ws, size_t have, size_t need) {
  if (need == 0) return ASR_OK;
  if (have < need) return fail(ASR_ENOMEM, "ws of " + std::to_string(have) + " bytes, " + std::to_string(need) + " needed");
  if (!ws || !aligned(ws, 256)) return fail(ASR_EINVAL, "ws must be 256-byte aligned");
  return ASR_OK;
}

// ---------------------------------------------------------------------------
// Pages of 8 bits
// ---------------------------------------------------------------------------
asr_status check_pages(const asr_pages& c, Pages* p) {
  if (c.kv_heads <= 0 || c.kv_heads > 65536) return fail(ASR_EINVAL, "kv_heads out of [1, 65536]");
  if (c.page < kPageBlock || c.page > 4096 || c.page % kPageBlock) return fail(ASR_EINVAL, "page must be a multiple of 64, at most 4096");
  if (c.pages < 1 || c.sequences < 0 || c.columns < 1) return fail(ASR_EINVAL, "pages and columns must be positive, sequences not negative");
  if ((int64_t)c.columns * c.page > (1 << 30)) return fail(ASR_EINVAL, "more than 2^30 positions in a sequence");
  const int64_t blocks = 2 * (int64_t)c.kv_heads * (c.page / kPageBlock);
  if (c.page_stride < blocks * kPageBlock * kHeadDim || c.page_stride % 16 || c.scale_stride < blocks)
    return fail(ASR_EINVAL, "page_stride must be a multiple of 16 bytes, and the strides at least a page's size");
  if (c.table_ld < c.columns) return fail(ASR_EINVAL, "table_ld below columns");
  if (!c.codes || !aligned(c.codes, 16) || !c.scales || !aligned(c.scales, 4)) return fail(ASR_EINVAL, "codes must be 16-byte aligned, scales 4-byte, neither NULL");
  if (!c.table) return fail(ASR_EINVAL, "NULL table");
  *p = {c.codes, c.scales, c.page_stride, c.scale_stride, c.table, c.table_ld, c.kv_heads, c.page, c.pages, c.sequences, c.columns};
  return ASR_OK;
}

// A part is a block of 64 keys for each of four waves at least; a lane knows the page
// of each of its wave's blocks.
constexpr int kPartStep = 4 * kPageBlock, kMostPart = 64 * kPartStep;

// Keys per part, `keys` at most for each of `units` (a sequence's queries and a cache
// head).  With P parts of n keys the call takes the turns of equal units, of n and what a
// part costs besides (`fixed` keys' worth) each; units of all lengths up to `keys` take
// their average share, the last parts, which end alone, and the parts' costs; a second
// kernel joins more than one part.  Whether lengths differ is not known here, so P is
// least for the sum of both.  Measured (us, bf16, by parts of 2048 / 4096 / 8192 keys):
// 64 x 8 units of 515 to 8191 keys 60 / 61 / 67, all of 8191 92 / 86 / 84; 16 x 8 of 65536
// 171 / 168 / 166; 24 x 8 of 6000 39 / 35 / 35; the rule's: 61, 86, 168, 35.
int paged_part(int64_t units, int64_t keys, bool ragged, int fixed) {
  const int64_t cus = cu_count(), least = std::max<int64_t>(1, (keys + kMostPart - 1) / kMostPart);
  const int64_t most = std::max(least, std::min<int64_t>((keys + kPartStep - 1) / kPartStep, 8 * cus / units));
  int64_t best = kPartStep;
  double best_cost = HUGE_VAL;
  for (int64_t p = least; p <= most; ++p) {
    const int64_t n = std::max<int64_t>(1, ((keys + p - 1) / p + kPartStep - 1) / kPartStep) * kPartStep;
    const int64_t blocks = units * ((keys + n - 1) / n);
    double cost = (double)((blocks + cus - 1) / cus) * (double)(n + fixed) + (blocks > units ? 600 : 0);
    if (ragged)
      cost += (double)units * keys / (2.0 * cus) + 0.75 * n + fixed * std::max(1.0, blocks / (2.0 * cus)) + (blocks > units ? 600 : 0);
    if (cost < best_cost) best = n, best_cost = cost;
  }
  return (int)best;
}

asr_status plan_paged(const asr_paged_attention* a, PagedLaunch* s, size_t* bytes) {
  if (!a) return fail(ASR_EINVAL, "NULL argument");
  if (a->dtype != ASR_F32 && a->dtype != ASR_BF16) return fail(ASR_EINVAL, "dtype");
  const asr_status st = check_pages(a->cache, &s->c);
  if (st != ASR_OK) return st;
  if (a->n_head <= 0 || a->n_head % a->cache.kv_heads || a->n_head > 65536)
    return fail(ASR_EINVAL, "kv_heads must divide n_head (at most 65536)");
  if (a->rows < 0 || a->max_keys < 0) return fail(ASR_EINVAL, "negative size");
  if (a->rows > 0 && (a->max_rows < 1 || a->max_rows > a->rows)) return fail(ASR_EINVAL, "max_rows out of [1, rows]");
  if (!a->row_start && a->rows > a->cache.sequences) return fail(ASR_EINVAL, "more rows than sequences, and no row_start");
  if (a->part_keys != 0 && (a->part_keys < 256 || a->part_keys > 16384 || a->part_keys % 256))
    return fail(ASR_EINVAL, "part_keys must be 0 or a multiple of 256, at most 16384");
  // (scores are powers of 2 in the kernel: the scale is taken times log2(e), a float too)
  const float qmul = a->scale * 1.4426950408889634f;
  if (!std::isfinite(qmul)) return fail(ASR_EINVAL, "scale must be finite, below 2.3e38 in magnitude");
  const int64_t most = std::min<int64_t>(a->max_keys, (int64_t)a->cache.columns * a->cache.page);
  const int64_t per = a->n_head / a->cache.kv_heads, cols = (a->row_start ? a->max_rows : 1) * per;
  if (cols > INT32_MAX) return fail(ASR_EINVAL, "too many queries in a sequence");
  const int64_t tile = 16 * paged_query_tiles((int)cols), tiles = (cols + tile - 1) / tile;
  const int64_t units = (int64_t)a->cache.sequences * a->cache.kv_heads * tiles;
  if (a->part_keys) {
    s->part = a->part_keys;
  } else {
    s->part = paged_part(std::max<int64_t>(units, 1), most, a->cache.sequences > 1, 400 + 20 * (int)std::min<int64_t>(cols, 64));
  }
  s->parts = std::max(parts_of((int)most, s->part), 1);
  const double blocks = ((double)units * s->parts + 8.0 * tiles);
  // (a launch has fewer than 2^32 threads: 256 a block, 64 a row and head)
  if (blocks >= 16777216.0 || (double)a->rows * a->n_head >= 67108864.0) return fail(ASR_EINVAL, "too much work for one call");
  s->q = a->q;
  s->q_ld = a->q_ld;
  s->out = a->out;
  s->out_ld = a->out_ld;
  s->qmul = qmul;
  s->row_start = a->row_start;
  s->first = a->first;
  s->length = a->length;
  s->n_head = a->n_head;
  s->rows = a->rows;
  s->max_rows = a->row_start ? a->max_rows : 1;
  s->max_keys = (int32_t)most;
  s->blocks = (int64_t)units * s->parts;
  // (windows: positions would leave most parts nothing; 7 chunks of up to 33 rows on up to
  // 4001 keys, windows of 1000: 19.8 -> 15.9 us)
  s->even = a->first && !a->part_keys && s->parts > 1;
  *bytes = s->parts > 1 ? kCounters * 4 + (size_t)a->rows * a->n_head * s->parts * (kHeadDim + 2) * 4 : 0;
  return ASR_OK;
}

asr_status plan_tables(const asr_page_tables* t, TablesLaunch* s, size_t* bytes) {
  if (!t) return fail(ASR_EINVAL, "NULL argument");
  if (t->sequences < 0 || t->columns < 1 || t->page < 1 || t->pages < 1) return fail(ASR_EINVAL, "sizes must be positive");
  if (t->pages > (1 << 22) || (int64_t)t->sequences * t->columns > (1 << 26) || (int64_t)t->columns * t->page > (1 << 30))
    return fail(ASR_EINVAL, "more than 2^22 pages, 2^26 table entries or 2^30 positions in a sequence");
  if (t->table_ld < t->columns || t->new_ld < t->columns) return fail(ASR_EINVAL, "table_ld or new_ld below columns");
  if (t->codes && (t->code_bytes < 0 || t->code_bytes % 4 || t->code_stride < t->code_bytes || t->code_stride % 4 || !aligned(t->codes, 4)))
    return fail(ASR_EINVAL, "codes: sizes and addresses must be multiples of 4 bytes, the stride at least the size");
  if (t->scales && (t->scale_bytes < 0 || t->scale_bytes % 4 || t->scale_stride < t->scale_bytes || t->scale_stride % 4 || !aligned(t->scales, 4)))
    return fail(ASR_EINVAL, "scales: sizes and addresses must be multiples of 4 bytes, the stride at least the size");
  *s = {t->sequences, t->columns, t->page, t->pages, t->compact != 0, t->table, t->table_ld, t->length, t->parent, t->want,
        t->new_table, t->new_ld, t->new_length, t->room, t->info, t->codes, t->code_stride, t->codes ? t->code_bytes : 0,
        t->scales, t->scale_stride, t->scales ? t->scale_bytes : 0, nullptr};
  *bytes = 4 * (kCounters + (size_t)tables_ws_words(t->sequences, t->columns, t->pages));
  return ASR_OK;
}

bool overlap(const void* a, int64_t a_bytes, const void* b, int64_t b_bytes) {
  return (uintptr_t)a < (uintptr_t)b + (uint64_t)b_bytes && (uintptr_t)b < (uintptr_t)a + (uint64_t)a_bytes;
}

// ---------------------------------------------------------------------------
// Sampling
// ---------------------------------------------------------------------------
asr_status plan_sample(const asr_sampling* a, SampleLaunch* s, size_t* bytes) {
  if (!a) return fail(ASR_EINVAL, "NULL argument");
  if (a->dtype != ASR_F32 && a->dtype != ASR_BF16) return fail(ASR_EINVAL, "dtype");
  if (a->rows < 0 || a->rows > 65535) return fail(ASR_EINVAL, "rows out of [0, 65535]");
  if (a->vocab < 1 || a->vocab > kRulesMaxVocab) return fail(ASR_EINVAL, "vocab out of [1, 1048576]");
  if (a->draws < 1 || a->draws > kSampleMaxDraws) return fail(ASR_EINVAL, "draws out of [1, 64]");
  if (a->sets < 0) return fail(ASR_EINVAL, "negative size");
  *s = {a->logits, a->ld, a->rows, a->vocab, a->sets, a->draws, a->u, a->set, a->temperature, a->top_k, a->top_p, a->min_p,
        a->token, a->logprob, a->kept};
  *bytes = 0;
  return ASR_OK;
}

}  // namespace

extern "C" {

asr_status asr_attend_shared_size(const asr_attention* a, size_t* bytes) {
  return guarded([&]() -> asr_status {
    if (!bytes) return fail(ASR_EINVAL, "NULL argument");
    ShareLaunch s{};
    return plan_attention(a, &s, bytes);
  });
}

asr_status asr_attend_shared(const asr_attention* a, void* ws, size_t ws_bytes, void* stream) {
  return guarded([&]() -> asr_status {
    ShareLaunch s{};
    size_t need = 0;
    asr_status st = plan_attention(a, &s, &need);
    if (st != ASR_OK) return st;
    if (a->rows == 0 || a->groups == 0) return ASR_OK;
    if (!a->q || !a->out || !a->group_start) return fail(ASR_EINVAL, "NULL q, out or group_start");
    const int64_t width = (int64_t)a->n_head * kHeadDim;
    if (a->q_ld < width || a->out_ld < width || a->q_ld % 4 || a->out_ld % 4)
      return fail(ASR_EINVAL, "q_ld and out_ld must be multiples of 4, at least n_head * 64");
    if (!aligned(a->q, 16) || !aligned(a->out, 16)) return fail(ASR_EINVAL, "q and out must be 16-byte aligned");
    st = check_ws(ws, ws_bytes, need);
    if (st != ASR_OK) return st;
    s.rec = need ? (float*)ws + kCounters : nullptr;
    return launched(attend_shared(s, a->dtype == ASR_BF16, (hipStream_t)stream));
  });
}

asr_status asr_logit_rules_size(const asr_rules* r, size_t* bytes) {
  return guarded([&]() -> asr_status {
    if (!bytes) return fail(ASR_EINVAL, "NULL argument");
    RulesLaunch s{};
    return plan_rules(r, &s, bytes);
  });
}

asr_status asr_logit_rules(const asr_rules* r, void* ws, size_t ws_bytes, void* stream) {
  return guarded([&]() -> asr_status {
    RulesLaunch s{};
    size_t need = 0;
    asr_status st = plan_rules(r, &s, &need);
    if (st != ASR_OK) return st;
    if (r->rows == 0) return ASR_OK;
    if (!r->logits || r->ld < r->vocab) return fail(ASR_EINVAL, "logits: NULL, or ld below the vocabulary");
    if (!aligned(r->logits, r->dtype == ASR_BF16 ? 2 : 4)) return fail(ASR_EINVAL, "logits must be aligned to their type");
    if (r->out && (r->out_ld < r->vocab || !aligned(r->out, 4))) return fail(ASR_EINVAL, "out: out_ld below the vocabulary, or unaligned");
    if (r->out && (const void*)r->out == r->logits && (r->dtype != ASR_F32 || r->out_ld != r->ld))
      return fail(ASR_EINVAL, "out may be the logits only in float32 with out_ld = ld");
    if (r->k > 0 && (!r->token || !r->logprob)) return fail(ASR_EINVAL, "k > 0 needs token and logprob");
    if (!r->out && r->k == 0) return fail(ASR_EINVAL, "nothing asked for: neither out nor k");
    st = check_ws(ws, ws_bytes, need);
    if (st != ASR_OK) return st;
    s.ws = (float*)ws + kCounters;
    // up to a block a CU the row's last block joins the others' results, above that
    // a second kernel does (us, 10 best of 51866 tokens: 5 rows 11.2 / 11.7, 64 rows
    // 14.5 / 14.3, 128 rows 23.6 / 19.7; one launch also spares the host 4 us)
    const int64_t blocks = (int64_t)r->rows * ((r->vocab + kRulesChunk - 1) / kRulesChunk);
    s.counters = r->k > 0 && blocks <= cu_count() ? (uint32_t*)ws : nullptr;
    logit_rules(s, r->dtype == ASR_BF16, (hipStream_t)stream);
    return launched(hipSuccess);
  });
}

asr_status asr_write_pages(const asr_page_write* w, void* stream) {
  return guarded([&]() -> asr_status {
    if (!w) return fail(ASR_EINVAL, "NULL argument");
    if (w->dtype != ASR_F32 && w->dtype != ASR_BF16) return fail(ASR_EINVAL, "dtype");
    PageWriteLaunch s{};
    const asr_status st = check_pages(w->cache, &s.c);
    if (st != ASR_OK) return st;
    if (w->tokens < 0 || w->max_new < 0) return fail(ASR_EINVAL, "negative size");
    if (!w->token_start && w->tokens < w->cache.sequences) return fail(ASR_EINVAL, "fewer tokens than sequences, and no token_start");
    if (w->cache.sequences == 0 || w->tokens == 0 || w->max_new == 0) return ASR_OK;
    if (!w->k || !w->v || !w->length) return fail(ASR_EINVAL, "NULL k, v or length");
    const int64_t unit = w->dtype == ASR_BF16 ? 8 : 4;
    if (!aligned(w->k, 16) || !aligned(w->v, 16) || w->ld < (int64_t)w->cache.kv_heads * kHeadDim || w->ld % unit)
      return fail(ASR_EINVAL, "k and v must be 16-byte aligned, ld a multiple of 16 bytes and at least kv_heads * 64");
    s.k = w->k;
    s.v = w->v;
    s.ld = w->ld;
    s.token_start = w->token_start;
    s.length = w->length;
    s.tokens = w->tokens;
    s.max_new = w->token_start ? std::min(w->max_new, w->tokens) : 1;
    // (a launch has fewer than 2^32 threads)
    if ((double)w->cache.sequences * w->cache.kv_heads * 2 * ((double)s.max_new / kPageBlock + 2) >= 16777216.0)
      return fail(ASR_EINVAL, "too much work for one call");
    write_pages(s, w->dtype == ASR_BF16, (hipStream_t)stream);
    return launched(hipSuccess);
  });
}

asr_status asr_attend_pages_size(const asr_paged_attention* a, size_t* bytes) {
  return guarded([&]() -> asr_status {
    if (!bytes) return fail(ASR_EINVAL, "NULL argument");
    PagedLaunch s{};
    return plan_paged(a, &s, bytes);
  });
}

asr_status asr_attend_pages(const asr_paged_attention* a, void* ws, size_t ws_bytes, void* stream) {
  return guarded([&]() -> asr_status {
    PagedLaunch s{};
    size_t need = 0;
    asr_status st = plan_paged(a, &s, &need);
    if (st != ASR_OK) return st;
    if (a->rows == 0 || a->cache.sequences == 0) return ASR_OK;
    if (!a->q || !a->out || !a->length) return fail(ASR_EINVAL, "NULL q, out or length");
    const int64_t width = (int64_t)a->n_head * kHeadDim;
    if (a->q_ld < width || a->out_ld < width || a->q_ld % 4 || a->out_ld % 4)
      return fail(ASR_EINVAL, "q_ld and out_ld must be multiples of 4, at least n_head * 64");
    if (!aligned(a->q, 16) || !aligned(a->out, 16)) return fail(ASR_EINVAL, "q and out must be 16-byte aligned");
    st = check_ws(ws, ws_bytes, need);
    if (st != ASR_OK) return st;
    s.rec = need ? (float*)ws + kCounters : nullptr;
    // With up to three blocks a CU and two queries a wave, the last block of a row's parts
    // joins them; above that a second kernel does (us, last block / kernel: a row on 1500
    // keys, 6 heads 7.8 / 9.7, 4 rows of 32 heads on 4000 10 / 12, 24 rows on 6000 36 / 37;
    // 64 on 8191 100 / 95; 2 x 3 rows on 8000, 12 queries a cache head 13.6 / 12.2).
    const int64_t queries = (int64_t)s.max_rows * (s.n_head / s.c.kv_heads);
    s.counters = need && s.blocks <= 3 * cu_count() && queries <= 8 ? (uint32_t*)ws : nullptr;
    attend_pages(s, a->dtype == ASR_BF16, (hipStream_t)stream);
    return launched(hipSuccess);
  });
}

asr_status asr_next_tables_size(const asr_page_tables* t, size_t* bytes) {
  return guarded([&]() -> asr_status {
    if (!bytes) return fail(ASR_EINVAL, "NULL argument");
    TablesLaunch s{};
    return plan_tables(t, &s, bytes);
  });
}

asr_status asr_next_tables(const asr_page_tables* t, void* ws, size_t ws_bytes, void* stream) {
  return guarded([&]() -> asr_status {
    TablesLaunch s{};
    size_t need = 0;
    asr_status st = plan_tables(t, &s, &need);
    if (st != ASR_OK) return st;
    if (t->sequences > 0) {
      if (!t->table || !t->length || !t->new_table || !t->new_length) return fail(ASR_EINVAL, "NULL table or length");
      const bool same = (const void*)t->table == t->new_table, same_length = (const void*)t->length == t->new_length;
      if (same != same_length || (same && t->table_ld != t->new_ld))
        return fail(ASR_EINVAL, "in place are both the table and the lengths, with one stride");
      const int64_t n = t->sequences;
      if (!same && (overlap(t->table, ((n - 1) * t->table_ld + t->columns) * 4, t->new_table, ((n - 1) * t->new_ld + t->columns) * 4) ||
                    overlap(t->length, n * 4, t->new_length, n * 4)))
        return fail(ASR_EINVAL, "the new table or lengths overlap the old ones");
    }
    st = check_ws(ws, ws_bytes, need);
    if (st != ASR_OK) return st;
    s.ws = (int32_t*)ws + kCounters;
    return launched(next_tables(s, (hipStream_t)stream));
  });
}

asr_status asr_sample_size(const asr_sampling* a, size_t* bytes) {
  return guarded([&]() -> asr_status {
    if (!bytes) return fail(ASR_EINVAL, "NULL argument");
    SampleLaunch s{};
    return plan_sample(a, &s, bytes);
  });
}

asr_status asr_sample(const asr_sampling* a, void* ws, size_t ws_bytes, void* stream) {
  return guarded([&]() -> asr_status {
    SampleLaunch s{};
    size_t need = 0;
    asr_status st = plan_sample(a, &s, &need);
    if (st != ASR_OK) return st;
    if (a->rows == 0) return ASR_OK;
    if (!a->logits || a->ld < a->vocab) return fail(ASR_EINVAL, "logits: NULL, or ld below the vocabulary");
    if (!aligned(a->logits, a->dtype == ASR_BF16 ? 2 : 4)) return fail(ASR_EINVAL, "logits must be aligned to their type");
    if (!a->u || !a->token) return fail(ASR_EINVAL, "NULL u or token");
    st = check_ws(ws, ws_bytes, need);
    if (st != ASR_OK) return st;
    return launched(sample(s, a->dtype == ASR_BF16, (hipStream_t)stream));
  });
}

}  // extern "C"
