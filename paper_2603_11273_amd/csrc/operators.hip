// Entry points of the stateless decode operators: argument checks, the split of
// the work, and the launches.
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

}  // extern "C"
