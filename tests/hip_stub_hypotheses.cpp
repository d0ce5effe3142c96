// Hypotheses, rules and their decode steps on the CPU: the program defines the HIP calls of the
// library itself ("device" memory is host memory, kernels do nothing, copies happen at once), says
// what the kernels left for the copies back, and checks what the library makes of it.  One scenario
// per name on the command line.
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <functional>
#include <string>
#include <vector>

#include "asr.h"

namespace {
// called before each copy to the host with what it copies and its number since the last wait
std::function<void(void* src, size_t n, int number)> results;
int copies = 0;
int graphs = 0;          // that are kept
int replays = 0;
constexpr int kToHost = 2;
}  // namespace

extern "C" {
int hipGetDeviceCount(int* n) { *n = 1; return 0; }
int hipSetDevice(int) { return 0; }
int hipGetDevice(int* d) { *d = 0; return 0; }
int hipDeviceGetAttribute(int* v, int, int) { *v = 256; return 0; }
int hipOccupancyMaxActiveBlocksPerMultiprocessor(int* n, const void*, int, size_t) { *n = 1; return 0; }
int hipFuncSetAttribute(const void*, int, int) { return 0; }
int hipLaunchKernel(const void*, unsigned long long, unsigned long long, void**, size_t, void*) { return 0; }
int hipGetLastError() { return 0; }
const char* hipGetErrorString(int) { return "made to fail"; }
int hipMemcpyAsync(void* dst, const void* src, size_t n, int kind, void*) {
  if (kind == kToHost && results) results(const_cast<void*>(src), n, copies++);
  memcpy(dst, src, n);
  return 0;
}
int hipStreamSynchronize(void*) { copies = 0; return 0; }
int hipDeviceSynchronize() { return 0; }
int hipStreamCreateWithFlags(void** s, unsigned) { *s = malloc(1); return 0; }
int hipStreamDestroy(void* s) { free(s); return 0; }
int hipEventCreateWithFlags(void** e, unsigned) { *e = malloc(1); return 0; }
int hipEventDestroy(void* e) { free(e); return 0; }
int hipEventRecord(void*, void*) { return 0; }
int hipStreamWaitEvent(void*, void*, unsigned) { return 0; }
int hipStreamBeginCapture(void*, int) { return 0; }
int hipStreamEndCapture(void*, void** g) { *g = malloc(1); return 0; }
int hipGraphDestroy(void* g) { free(g); return 0; }
int hipGraphInstantiate(void** ex, void*, void*, char*, size_t) { *ex = malloc(1); ++graphs; return 0; }
int hipGraphExecDestroy(void* ex) { free(ex); --graphs; return 0; }
int hipGraphLaunch(void*, void*) { ++replays; return 0; }
}

#define OK(x)                                                                       \
  do {                                                                              \
    if ((x) != ASR_OK) return printf("%s: %s\n", #x, asr_last_error()), 1;          \
  } while (0)
#define CHECK(x)                                                                    \
  do {                                                                              \
    if (!(x)) return printf("line %d: %s (last error: %s)\n", __LINE__, #x, asr_last_error()), 1; \
  } while (0)

namespace {

struct Context {
  asr_ctx* c = nullptr;
  void *block = nullptr, *hyp = nullptr;
  ~Context() {
    if (c) asr_destroy(c);
    free(block);
    free(hyp);
  }
  int make(int n_enc, int slots, int vocab, int max_bias, int n_masks) {
    asr_model_cfg cfg{80, 64, n_enc, 1, 1, 64, vocab, ASR_F32, slots, 1, slots, 16};
    OK(asr_create(&cfg, 0, &c));
    size_t bytes = 0;
    OK(asr_workspace_size(c, &bytes));
    block = aligned_alloc(256, bytes);
    memset(block, 0, bytes);
    OK(asr_bind(c, block, bytes, nullptr));
    int32_t n = 0;
    OK(asr_n_params(c, &n));
    std::vector<std::vector<float>> data(n);
    std::vector<const float*> tensors(n);
    for (int i = 0; i < n; ++i) {
      int64_t numel = 0;
      OK(asr_param_numel(c, i, &numel));
      data[i].resize(numel);
      tensors[i] = data[i].data();
    }
    OK(asr_load_weights(c, tensors.data(), n, 0));
    OK(asr_hypotheses_size(c, max_bias, n_masks, &bytes));
    hyp = aligned_alloc(256, bytes);
    memset(hyp, 0, bytes);
    OK(asr_bind_hypotheses(c, max_bias, n_masks, hyp, bytes));
    return 0;
  }
};

// Three requests on two slots under default rules: a row whose rules allow no token and a row
// with a NaN end their own requests, and everything else goes on.
int serve() {
  Context x;
  if (x.make(1, 2, 40, 0, 1)) return 1;
  asr_slot_rules rules{1.f, 0.f, 0.f, 1.f, 0, 0, 0, nullptr, nullptr};
  OK(asr_set_slot_rules(x.c, -1, &rules));
  asr_serve_cfg cfg{};
  cfg.cross_tokens = 1500;
  cfg.max_admit = 1;
  cfg.tok_num = 27;
  cfg.tok_den = 10;
  cfg.start_token = 1;
  OK(asr_serve_config(x.c, &cfg));
  std::vector<float> pcm(64000, 0.f);
  for (int64_t id = 0; id < 3; ++id) OK(asr_submit(x.c, id, pcm.data(), (int64_t)pcm.size(), 16000, 0, 0, 0, 0));
  int64_t preempted[2], admitted[2], decoded[2], finished[2];
  int32_t slot[2], token[2];
  asr_serve_out out{2, 0, preempted, 0, admitted, slot, 0, decoded, token, 0, finished, 0};
  int now = 0, dead = -1;
  bool nan = false;
  results = [&](void* src, size_t n, int number) {
    for (size_t i = 0; i < n / 4; ++i) {
      if (number == 0)
        ((int32_t*)src)[i] = (int)i == dead && !nan ? -1 : 7 + now;
      else
        ((float*)src)[i] = (int)i == dead && nan ? NAN : -0.5f;
    }
  };
  auto step = [&] { return asr_serve_step(x.c, now++, &out); };
  for (int i = 0; i < 3; ++i) OK(step());
  CHECK(out.n_decoded == 2 && decoded[0] == 0 && decoded[1] == 1 && out.n_finished == 0);
  dead = 0;                                            // request 0, with three tokens by now
  OK(step());
  CHECK(out.n_decoded == 2 && token[0] == -1 && token[1] == 7 + now);
  CHECK(out.n_finished == 1 && finished[0] == 0);
  int32_t got[448], n = 0;
  OK(asr_serve_tokens(x.c, 0, got, 448, &n));
  CHECK(n == 3 && got[0] >= 7 && got[1] >= 7 && got[2] >= 7);
  dead = -1;
  OK(step());                                          // request 2 takes its slot
  CHECK(out.n_admitted == 1 && admitted[0] == 2 && out.n_decoded == 2 && out.n_finished == 0);
  dead = 1;                                            // (rows in the order of admission)
  nan = true;
  CHECK(step() == ASR_EDEVICE && strstr(asr_last_error(), "request 2"));
  CHECK(out.n_decoded == 2 && token[1] == -1 && out.n_finished == 1 && finished[0] == 2);
  OK(asr_serve_tokens(x.c, 2, got, 448, &n));
  CHECK(n == 1);
  dead = -1;
  for (int i = 0; i < 40 && !(out.n_finished == 1 && finished[0] == 1); ++i) OK(step());
  OK(asr_serve_tokens(x.c, 1, got, 448, &n));
  CHECK(n == 11);                                      // 4 s at 2.7 tokens a second
  for (int i = 0; i < n; ++i) CHECK(got[i] >= 7);
  printf("serve: ok\n");
  return 0;
}

// A row without rules in a step with one that has some: infinite logits, all of them -infinite
// and NaN ones give what they give without the other row.
int beside() {
  Context x;
  if (x.make(0, 3, 40, 0, 1)) return 1;
  int32_t slots[3] = {0, 1, 2}, left[3] = {40, 40, 40}, tokens[3] = {1, 2, 3}, argmax[3], done[3], best[6];
  int64_t ids[3] = {-1, -1, -1};
  float logprob[6];
  std::vector<float> E(1500 * 64);
  for (int i = 0; i < 3; ++i) OK(asr_debug_set_encoder_out(x.c, slots + i, ids + i, left + i, 1, E.data(), 0));
  asr_slot_rules rules{1.5f, 0.f, 0.f, 1.f, 0, -1, 0, nullptr, nullptr};
  OK(asr_set_slot_rules(x.c, 1, &rules));
  asr_step_in in{0, nullptr, 3, slots, tokens, nullptr};
  asr_step_out out{nullptr, argmax, done};
  int32_t token[3] = {5, 6, -1}, own[3] = {9, 30, 0};
  float lp[3] = {NAN, -0.5f, -INFINITY};
  int asked = 0;
  results = [&](void* src, size_t n, int) {
    const void* from[3] = {token, lp, own};
    if (asked < 3 && n == 12) memcpy(src, from[asked], n);
    ++asked;
  };
  auto step = [&] { return asked = 0, asr_step(x.c, &in, &out); };
  OK(step());
  CHECK(asked == 3 && argmax[0] == 9 && argmax[1] == 6 && argmax[2] == 0);
  own[2] = -1 - 17;                                    // a NaN at 17
  CHECK(step() == ASR_EDEVICE && strstr(asr_last_error(), "NaN"));
  CHECK(argmax[0] == 9 && argmax[1] == 6 && argmax[2] == 17);
  token[2] = 8;
  lp[0] = lp[2] = -1.f;
  OK(step());
  CHECK(asked == 2 && argmax[0] == 5 && argmax[1] == 6 && argmax[2] == 8);
  lp[1] = NAN;                                         // of the row with rules
  CHECK(step() == ASR_EDEVICE && asked == 2);
  lp[1] = -1.f;
  lp[0] = NAN;                                         // asked for candidates, a row's are what they are
  results = [&](void* src, size_t n, int number) {
    for (size_t i = 0; i < n / 4; ++i)
      if (number == 0)
        ((int32_t*)src)[i] = 5 + (int)i;
      else
        ((float*)src)[i] = i == 0 ? NAN : -1.f;
  };
  CHECK(asr_step_topk(x.c, &in, &out, 2, best, logprob) == ASR_EDEVICE);
  CHECK(argmax[0] == 5 && argmax[2] == 9 && best[5] == 10);
  printf("beside: ok\n");
  return 0;
}

// Steps of 256 shapes with rules, of 16 without, and a change of the shapes in use: the graphs
// kept are bounded, every shape without rules keeps its own, and new shapes come to theirs.
int shapes() {
  Context x;
  if (x.make(0, 16, 40, 0, 1)) return 1;
  const int most = 128;
  int32_t slots[16], tokens[16] = {}, argmax[16], done[16], best[256], left = 448;
  int64_t id = -1;
  float logprob[256];
  std::vector<float> E(1500 * 64);
  for (int i = 0; i < 16; ++i) slots[i] = i;
  auto renew = [&](int i) { return asr_debug_set_encoder_out(x.c, slots + i, &id, &left, 1, E.data(), 0); };
  int steps = 0;
  auto step = [&](int rows, int k) -> asr_status {
    if (steps++ % 440 == 0)                            // positions end at 448
      for (int i = 0; i < 16; ++i)
        if (asr_status st = renew(i)) return st;
    asr_step_in in{0, nullptr, rows, slots, tokens, nullptr};
    asr_step_out out{nullptr, argmax, done};
    return k ? asr_step_topk(x.c, &in, &out, k, best, logprob) : asr_step(x.c, &in, &out);
  };
  for (int round = 0; round < 3; ++round)
    for (int rows = 1; rows <= 16; ++rows)
      for (int k = 1; k <= 16; ++k) {
        OK(step(rows, k));
        CHECK(graphs <= most);
      }
  CHECK(graphs == most && replays == 2 * most);        // the first to come keep theirs
  for (int round = 0; round < 3; ++round)
    for (int rows = 1; rows <= 16; ++rows) OK(step(rows, 0));
  CHECK(graphs == most + 16);
  int before = replays;
  OK(step(16, 16));
  CHECK(replays == before);                            // no room yet
  for (int i = 0; i < 600; ++i) OK(step(1 + i % 16, 0));
  before = replays;
  for (int i = 0; i < 3; ++i) OK(step(16, 16));
  CHECK(replays == before + 3 && graphs == most + 16);
  for (int i = 0; i < 16; ++i) OK(renew(i));
  steps = 1;
  for (int round = 0; round < 3; ++round)              // families: forks one after the other
    for (int rows = 2; rows <= 8; ++rows) {
      for (int i = 1; i < rows; ++i) {
        OK(asr_release_slot(x.c, i));
        OK(asr_fork_slot(x.c, 0, i));
      }
      for (int k = 0; k <= 16; ++k) OK(step(rows, k));
      for (int i = 1; i < rows; ++i) OK(asr_release_slot(x.c, i));
      for (int i = 1; i < rows; ++i) OK(renew(i));
      CHECK(graphs <= most + 16);
    }
  before = replays;
  for (int rows = 1; rows <= 16; ++rows) OK(step(rows, 0));
  CHECK(replays == before + 16);
  printf("shapes: ok\n");
  return 0;
}

// Biases that would leave a row no probabilities are refused when they are given.
int biases() {
  Context x;
  if (x.make(0, 2, 40, 3, 0)) return 1;
  int32_t slot = 0, left = 9, token[3] = {1, 2, 1};
  int64_t id = -1;
  std::vector<float> E(1500 * 64);
  OK(asr_debug_set_encoder_out(x.c, &slot, &id, &left, 1, E.data(), 0));
  float value[3] = {-INFINITY, 3.4e38f, -3.4e38f};
  asr_slot_rules rules{1.f, 0.f, 0.f, 1.f, 0, -1, 3, token, value};
  for (int to = -1; to <= 0; ++to) {
    OK(asr_set_slot_rules(x.c, to, &rules));
    for (float bad : {INFINITY, NAN, -NAN}) {
      value[1] = bad;
      CHECK(asr_set_slot_rules(x.c, to, &rules) == ASR_EINVAL);
      value[1] = 0.f;
    }
    token[2] = 40;
    CHECK(asr_set_slot_rules(x.c, to, &rules) == ASR_EINVAL);
    token[2] = 1;
  }
  printf("biases: ok\n");
  return 0;
}

}  // namespace

int main(int argc, char** argv) {
  for (int i = 1; i < argc; ++i) {
    const std::string name = argv[i];
    results = nullptr;
    copies = 0;
    const int bad = name == "serve"    ? serve()
                    : name == "beside" ? beside()
                    : name == "shapes" ? shapes()
                    : name == "biases" ? biases()
                                       : (printf("no scenario %s\n", argv[i]), 1);
    if (bad) return bad;
  }
  return 0;
}
