// The entry points' host side without a device: this program stands in for the HIP
// runtime that libpolyglot.so calls.  Device memory is host memory, nothing that is
// launched runs, and every call is written down.  argv[1] names what is looked at;
// exit status 0: as it should be, 1: not (the reason on stdout).
#include <hip/hip_runtime_api.h>
#include <sys/mman.h>

#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <set>
#include <string>
#include <vector>

#include "polyglot.h"

namespace {

struct LaunchRecord {
  dim3 grid, block;
  hipStream_t stream;
  polyglot_logits_args logits;  // where the kernel's arguments begin with them
  uint64_t* head;
};
std::vector<LaunchRecord> launches;
bool record_logits = false;
std::map<void*, size_t> blocks;
size_t to_device = 0;        // bytes of the largest copy from the host
long events = 0;             // created and not destroyed
std::vector<std::string> order;  // records, waits and synchronisations
std::set<hipStream_t> capturing, gone;

hipError_t launched(dim3 grid, dim3 block, void** args, hipStream_t s) {
  LaunchRecord r{grid, block, s, {}, nullptr};
  if (record_logits) std::memcpy(&r.logits, args[0], sizeof(r.logits));
  launches.push_back(r);
  return hipSuccess;
}

std::string name(hipStream_t s) { return std::to_string(reinterpret_cast<uintptr_t>(s)); }

int checks = 0;
#define CHECK(c)                                          \
  do {                                                    \
    ++checks;                                             \
    if (!(c)) {                                           \
      std::printf("line %d: not (%s)\n", __LINE__, #c);   \
      std::exit(1);                                       \
    }                                                     \
  } while (0)

}  // namespace

extern "C" {
void** __hipRegisterFatBinary(const void*) { static void* p; return &p; }
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void*, char*, const char*, unsigned, void*, void*, dim3*,
                           dim3*, int*) {}
void __hipRegisterVar(void**, void*, char*, char*, int, size_t, int, int) {}
hipError_t __hipPopCallConfiguration(dim3*, dim3*, size_t*, hipStream_t*) { return hipSuccess; }
hipError_t hipGetSymbolAddress(void** p, const void*) {
  static char room[1 << 16];
  *p = room;
  return hipSuccess;
}
hipError_t hipMalloc(void** p, size_t n) {
  *p = mmap(nullptr, n, PROT_READ | PROT_WRITE, MAP_PRIVATE | MAP_ANONYMOUS | MAP_NORESERVE, -1, 0);
  if (*p == MAP_FAILED) return hipErrorOutOfMemory;
  blocks[*p] = n;
  return hipSuccess;
}
hipError_t hipFree(void* p) {
  if (!blocks.count(p)) return hipErrorInvalidValue;
  munmap(p, blocks[p]);
  blocks.erase(p);
  return hipSuccess;
}
hipError_t hipMemset(void* p, int v, size_t n) {
  if (v || n <= 1 << 20) std::memset(p, v, n);  // (what is mapped anew is zero)
  return hipSuccess;
}
hipError_t hipMemsetAsync(void* p, int v, size_t n, hipStream_t) { return hipMemset(p, v, n); }
hipError_t hipMemset2DAsync(void* p, size_t pitch, int v, size_t w, size_t h, hipStream_t) {
  for (size_t i = 0; i < h; ++i) std::memset(static_cast<char*>(p) + i * pitch, v, w);
  return hipSuccess;
}
hipError_t hipMemcpy(void* d, const void* s, size_t n, hipMemcpyKind k) {
  if (k == hipMemcpyHostToDevice && n > to_device) to_device = n;
  std::memcpy(d, s, n);
  return hipSuccess;
}
hipError_t hipMemcpyAsync(void* d, const void* s, size_t n, hipMemcpyKind k, hipStream_t) {
  return hipMemcpy(d, s, n, k);
}
hipError_t hipLaunchKernel(const void*, dim3 g, dim3 b, void** a, size_t, hipStream_t s) {
  return launched(g, b, a, s);
}
hipError_t hipExtLaunchKernel(const void*, dim3 g, dim3 b, void** a, size_t, hipStream_t s,
                              hipEvent_t, hipEvent_t, int) {
  return launched(g, b, a, s);
}
hipError_t hipEventCreate(hipEvent_t* e) {
  *e = reinterpret_cast<hipEvent_t>(std::malloc(1));
  ++events;
  return hipSuccess;
}
hipError_t hipEventCreateWithFlags(hipEvent_t* e, unsigned) { return hipEventCreate(e); }
hipError_t hipEventDestroy(hipEvent_t e) {
  std::free(e);
  --events;
  return hipSuccess;
}
hipError_t hipEventElapsedTime(float* ms, hipEvent_t, hipEvent_t) {
  *ms = 0.5f;
  return hipSuccess;
}
hipError_t hipEventRecord(hipEvent_t, hipStream_t s) {
  if (gone.count(s)) return hipErrorContextIsDestroyed;
  order.push_back("record " + name(s));
  return hipSuccess;
}
hipError_t hipStreamWaitEvent(hipStream_t s, hipEvent_t, unsigned) {
  order.push_back("wait " + name(s));
  return hipSuccess;
}
hipError_t hipStreamSynchronize(hipStream_t) { return hipSuccess; }
hipError_t hipDeviceSynchronize() {
  order.push_back("all");
  return hipSuccess;
}
hipError_t hipStreamIsCapturing(hipStream_t s, hipStreamCaptureStatus* c) {
  if (gone.count(s)) return hipErrorContextIsDestroyed;
  *c = capturing.count(s) ? hipStreamCaptureStatusActive : hipStreamCaptureStatusNone;
  return hipSuccess;
}
hipError_t hipStreamCreateWithFlags(hipStream_t* s, unsigned) {
  *s = reinterpret_cast<hipStream_t>(std::malloc(1));
  return hipSuccess;
}
hipError_t hipStreamDestroy(hipStream_t s) {
  std::free(s);
  return hipSuccess;
}
hipError_t hipStreamBeginCapture(hipStream_t, hipStreamCaptureMode) { return hipSuccess; }
hipError_t hipStreamEndCapture(hipStream_t, hipGraph_t*) { return hipSuccess; }
hipError_t hipGraphInstantiate(hipGraphExec_t*, hipGraph_t, hipGraphNode_t*, char*, size_t) {
  return hipSuccess;
}
hipError_t hipGraphLaunch(hipGraphExec_t, hipStream_t) { return hipSuccess; }
hipError_t hipGraphDestroy(hipGraph_t) { return hipSuccess; }
hipError_t hipGraphExecDestroy(hipGraphExec_t) { return hipSuccess; }
hipError_t hipGetDevice(int* d) {
  *d = 0;
  return hipSuccess;
}
hipError_t hipGetLastError() { return hipSuccess; }
const char* hipGetErrorString(hipError_t) { return "error"; }
}

namespace {

polyglot_ctx* context() {
  polyglot_config cfg{};
  cfg.V = 1000;
  cfg.d = 16;
  cfg.win = 5;
  cfg.H = 8;
  cfg.max_batch = 1;
  polyglot_ctx* ctx = nullptr;
  CHECK(polyglot_init(&cfg, nullptr, &ctx) == POLYGLOT_OK);
  launches.clear();
  order.clear();
  return ctx;
}

float* room() {  // an address; nothing reads or writes it
  static float p[64];
  return p;
}

// Scores of many rows: every launch has fewer than 2^32 threads, and together they
// take each row once, with its own part of everything that goes by row.
void many_rows() {
  polyglot_ctx* ctx = context();
  const int rows = (1 << 24) + 5, V = 3;
  CHECK(polyglot_reserve_logits(ctx, rows, V) == POLYGLOT_OK);
  char* const base = reinterpret_cast<char*>(room());
  polyglot_logits_args a{};
  a.logits = base;
  a.out = base + 4;
  a.history = reinterpret_cast<int32_t*>(base + 8);
  a.lengths = reinterpret_cast<int32_t*>(base + 12);
  a.prompt = reinterpret_cast<int32_t*>(base + 16);
  a.repetition = reinterpret_cast<float*>(base + 20);
  a.presence = reinterpret_cast<float*>(base + 24);
  a.frequency = reinterpret_cast<float*>(base + 28);
  a.bias = reinterpret_cast<float*>(base + 32);
  a.mask = reinterpret_cast<uint32_t*>(base + 36);
  a.token = reinterpret_cast<int32_t*>(base + 40);
  a.lse = reinterpret_cast<float*>(base + 44);
  a.rows = rows;
  a.V = V;
  a.dtype = POLYGLOT_BF16;
  a.history_cap = 2;
  a.ld_logits = 5;
  a.ld_out = 4;
  a.ld_history = 3;
  a.ld_mask = 2;
  record_logits = true;
  for (int form = 0; form < 3; ++form) {  // own masks and biases; one of each; masks by number
    a.masks = form == 1 ? 1 : rows;
    a.ld_bias = form == 1 ? 0 : 7;
    a.mask_rows = form == 2 ? reinterpret_cast<int32_t*>(base + 48) : nullptr;
    if (form == 2) a.masks = 4;
    launches.clear();
    CHECK(polyglot_logits(ctx, &a) == POLYGLOT_OK);
    int64_t r = 0;
    for (const LaunchRecord& l : launches) {
      CHECK((uint64_t)l.grid.x * l.grid.y * l.grid.z * l.block.x < (uint64_t)1 << 32);
      const polyglot_logits_args& b = l.logits;
      CHECK((int64_t)l.grid.x == b.rows);  // one part to a row of three words
      const auto at = [&](const void* p, const void* first, int64_t bytes) {
        return static_cast<const char*>(p) - static_cast<const char*>(first) == r * bytes;
      };
      CHECK(at(b.logits, a.logits, 2 * a.ld_logits));
      CHECK(at(b.out, a.out, 2 * a.ld_out));
      CHECK(at(b.history, a.history, 4 * a.ld_history));
      CHECK(at(b.lengths, a.lengths, 4) && at(b.prompt, a.prompt, 4));
      CHECK(at(b.repetition, a.repetition, 4) && at(b.presence, a.presence, 4));
      CHECK(at(b.frequency, a.frequency, 4));
      CHECK(at(b.bias, a.bias, 4 * a.ld_bias));
      CHECK(at(b.mask, a.mask, form == 0 ? 4 * a.ld_mask : 0));
      CHECK(form == 2 ? at(b.mask_rows, a.mask_rows, 4) : !b.mask_rows);
      CHECK(b.masks == (form == 0 ? b.rows : a.masks));
      CHECK(at(b.token, a.token, 4) && at(b.lse, a.lse, 4));
      r += b.rows;
    }
    CHECK(r == rows);
  }
  a.token = nullptr;  // what is not there stays away
  a.lse = nullptr;
  a.history = nullptr;
  a.lengths = a.prompt = nullptr;
  a.repetition = a.presence = a.frequency = a.bias = nullptr;
  a.mask = nullptr;
  a.mask_rows = nullptr;
  launches.clear();
  CHECK(polyglot_logits(ctx, &a) == POLYGLOT_OK);
  for (const LaunchRecord& l : launches) {
    const polyglot_logits_args& b = l.logits;
    CHECK(!b.token && !b.lse && !b.history && !b.lengths && !b.prompt && !b.repetition);
    CHECK(!b.presence && !b.frequency && !b.bias && !b.mask && !b.mask_rows);
  }
}

// What is enqueued after a change of the stream waits for what was enqueued before it:
// the calls of a context share its workspace.
void streams() {
  polyglot_ctx* ctx = context();
  const auto stream = [](uintptr_t k) { return reinterpret_cast<hipStream_t>(k); };
  const auto change = [&](uintptr_t k) { return polyglot_set_stream(ctx, stream(k)); };
  const auto said = [&](std::vector<std::string> want) {
    const bool same = order == want;
    order.clear();
    return same;
  };
  const long before = events;
  CHECK(change(16) == POLYGLOT_OK && said({"record 0", "wait 16"}));
  CHECK(change(16) == POLYGLOT_OK && said({}));
  CHECK(change(32) == POLYGLOT_OK && said({"record 16", "wait 32"}));
  CHECK(change(0) == POLYGLOT_OK && said({"record 32", "wait 0"}));
  CHECK(change(16) == POLYGLOT_OK && said({"record 0", "wait 16"}));
  CHECK(events <= before + 1);
  // into a graph that is being captured and out of it: its nodes cannot wait for what
  // is outside, nor what is outside for them
  capturing = {stream(48)};
  CHECK(change(48) == POLYGLOT_OK && said({}));
  CHECK(change(16) == POLYGLOT_OK && said({}));
  CHECK(change(48) == POLYGLOT_OK && said({}));
  capturing.clear();  // what ran before the capture is waited for also after it
  CHECK(change(32) == POLYGLOT_OK && said({"record 16", "wait 32"}));
  CHECK(change(16) == POLYGLOT_OK && said({"record 32", "wait 16"}));
  // a stream that is gone: what it held is waited for with everything else
  gone = {stream(16)};
  CHECK(change(32) == POLYGLOT_OK && said({"all"}));
  // the calls go where the last change says
  polyglot_dropout_args a{};
  a.x = a.y = room();
  a.rows = a.d = 1;
  a.ld_x = a.ld_y = 1;
  CHECK(polyglot_dropout(ctx, &a) == POLYGLOT_OK && launches.back().stream == stream(32));
  CHECK(polyglot_set_stream(nullptr, nullptr) == POLYGLOT_ENULL);
  CHECK(polyglot_destroy(ctx) == POLYGLOT_OK && events == 0);
}

// A program that asks for the times of one kind of kernels alone keeps no more event
// pairs than it makes between two questions; the other kind's times are kept.
void times() {
  polyglot_ctx* ctx = context();
  CHECK(polyglot_set_timing(ctx, 1) == POLYGLOT_OK);
  polyglot_dropout_args a{};
  a.x = a.y = room();
  a.rows = a.d = 1;
  a.ld_x = a.ld_y = 1;
  double ms[POLYGLOT_NKERNELS + POLYGLOT_NOPKERNELS];
  int32_t n[POLYGLOT_NKERNELS + POLYGLOT_NOPKERNELS];
  long after_one = 0;
  for (int i = 0; i < 100; ++i) {
    for (int k = 0; k < 3; ++k) CHECK(polyglot_dropout(ctx, &a) == POLYGLOT_OK);
    CHECK(polyglot_kernel_times(ctx, ms, n) == POLYGLOT_OK);
    for (int k = 0; k < POLYGLOT_NKERNELS; ++k) CHECK(n[k] == 0 && ms[k] == 0);
    if (i == 0) after_one = events;
  }
  CHECK(events == after_one);
  CHECK(polyglot_operator_times(ctx, ms, n) == POLYGLOT_OK);
  CHECK(n[POLYGLOT_OPK_DROPOUT] == 300 && ms[POLYGLOT_OPK_DROPOUT] == 150.0);
  CHECK(n[POLYGLOT_OPK_LOGITS] == 0);
  CHECK(polyglot_operator_times(ctx, ms, n) == POLYGLOT_OK && n[POLYGLOT_OPK_DROPOUT] == 0);
  // the other way round
  for (int i = 0; i < 100; ++i) {
    CHECK(polyglot_score(ctx, room(), room(), room(), room(), room(),
                         reinterpret_cast<int32_t*>(room()), 1, room()) == POLYGLOT_OK);
    CHECK(polyglot_operator_times(ctx, ms, n) == POLYGLOT_OK);
    for (int k = 0; k < POLYGLOT_NOPKERNELS; ++k) CHECK(n[k] == 0);
    if (i == 0) after_one = events;
  }
  CHECK(events == after_one);
  CHECK(polyglot_kernel_times(ctx, ms, n) == POLYGLOT_OK);
  int all = 0;
  for (int k = 0; k < POLYGLOT_NKERNELS; ++k) all += n[k];
  CHECK(all >= 100 && all % 100 == 0);
  CHECK(polyglot_destroy(ctx) == POLYGLOT_OK && events == 0);
}

// Reserving makes the counters on the device: nothing of their size on the host.  Every
// line starts with tag 1 and nothing counted, all else is zero.
void reserve() {
  polyglot_ctx* ctx = context();
  const auto newest = [] {  // the largest block
    std::pair<void*, size_t> b{nullptr, 0};
    for (const auto& k : blocks)
      if (k.second > b.second) b = k;
    return b;
  };
  const auto whole = [&](size_t lines, size_t all) {
    const auto b = newest();
    const uint64_t* w = static_cast<const uint64_t*>(b.first);
    CHECK(b.second >= 8 * all);
    for (size_t i = 0; i < b.second / 8; ++i)
      if (w[i] != (i % 16 == 0 && i < 16 * lines ? (uint64_t)1 << 32 : 0)) return false;
    return true;
  };
  to_device = 0;
  const int rows = 1 << 20;
  CHECK(polyglot_reserve_logits(ctx, rows, 3000) == POLYGLOT_OK);
  CHECK(whole(rows, (size_t)rows * (16 + 3 * 3)));
  CHECK(polyglot_reserve_logits(ctx, 0, 0) == POLYGLOT_OK);
  CHECK(polyglot_reserve_recurrence(ctx, 1000, 1 << 16) == POLYGLOT_OK);
  const size_t tiles = 2 * (1 << 16) / 32 + 1;  // the narrowest, doubled for a group's idle lanes
  CHECK(whole(tiles, tiles * 16));
  CHECK(polyglot_reserve_recurrence(ctx, 0, 0) == POLYGLOT_OK);
  CHECK(to_device <= 4096);
  CHECK(polyglot_destroy(ctx) == POLYGLOT_OK && blocks.empty());
}

}  // namespace

int main(int argc, char** argv) {
  const std::map<std::string, void (*)()> all = {{"many_rows", many_rows}, {"streams", streams}, {"times", times},
                                                        {"reserve", reserve}};
  const auto it = argc > 1 ? all.find(argv[1]) : all.end();
  if (it == all.end()) return 2;
  it->second();
  std::printf("%d checks\n", checks);
  return 0;
}
