// The library's context and what every entry point does with it: error
// returns, workspace allocation, per-kernel event timing.
#pragma once
#include "polyglot.h"

#include <hip/hip_ext.h>
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>
#include <string>
#include <utility>
#include <vector>

#include "launch.h"
#include "operators.h"

namespace pg {

struct GraphKey {
  const void* p[7];
  const void* losses;
  int S, B;
  float lr;
  hipStream_t stream;
  bool operator==(const GraphKey& o) const {
    return std::memcmp(p, o.p, sizeof(p)) == 0 && losses == o.losses && S == o.S && B == o.B &&
           std::memcmp(&lr, &o.lr, sizeof(float)) == 0 && stream == o.stream;
  }
};

// What the polyglot_reserve_* calls allocated.
struct OpWorkspace {
  int64_t rec_tokens = 0;
  int rec_D = 0;
  ScanSpace rec;
  int log_rows = 0, log_V = 0;
  uint64_t *log_head = nullptr, *log_words = nullptr;  // one block: counters, words
};

// A kernel's event pairs that are counted and not yet asked for.
struct KernelTime {
  double ms = 0.0;
  int32_t launches = 0;
};

}  // namespace pg

struct polyglot_ctx {
  polyglot_config cfg{};
  hipStream_t stream = nullptr;
  // a step's sort depends only on its ids: it runs on a second stream,
  // forked from `stream` and joined back before the table update.  In a
  // multi-step call the sort of step s+1 (sort set (s+1)&1) runs while step s
  // computes.
  hipStream_t side = nullptr;
  hipEvent_t ev_fork = nullptr, ev_sorted[2] = {nullptr, nullptr},
             ev_done[2] = {nullptr, nullptr};
  hipStream_t eager = nullptr;   // the stream whose calls run as they are made (not a capture's)
  hipEvent_t ev_swap = nullptr;  // where it was left for another
  int device = 0;
  int Hp = 0, NT = 0, K = 0, c = 0, cpw = 0;
  bool large = false;  // hidden layer above 64 units: the three-contraction path
  int max_entries = 0, max_tiles = 0, max_parts = 0, max_chunks = 0;
  int seg_stride = 0, part_stride = 0;
  pg::Workspace ws{};
  std::vector<void*> allocs;
  std::string err;
  bool have_sorted = false;
  int last_N = 0, last_passes = 0, last_set = 0;
  bool set_dirty = false;  // an assignment marked its rows and failed to take the marks back
  hipGraphExec_t gexec = nullptr;
  pg::GraphKey gkey{};
  bool gvalid = false;
  pg::OpWorkspace op{};
  // per-kernel timing
  bool timing = false;
  bool capturing = false;
  std::vector<hipEvent_t> ev_pool;
  std::vector<std::pair<int, std::pair<hipEvent_t, hipEvent_t>>> ev_marks;
  pg::KernelTime times[POLYGLOT_NKERNELS + POLYGLOT_NOPKERNELS];  // by kernel id
};

namespace pg {

inline int fail(polyglot_ctx* ctx, int code, const std::string& msg) {
  if (ctx) ctx->err = msg;
  return code;
}

inline int hip_fail(polyglot_ctx* ctx, hipError_t e, const char* what) {
  return fail(ctx, POLYGLOT_EHIP, std::string(what) + ": " + hipGetErrorString(e));
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

template <class T>
hipError_t alloc(polyglot_ctx* ctx, T** p, size_t count) {
  void* q = nullptr;
  hipError_t e = hipMalloc(&q, std::max<size_t>(count, 1) * sizeof(T));
  if (e == hipSuccess) {
    ctx->allocs.push_back(q);
    *p = static_cast<T*>(q);
  }
  return e;
}

inline hipEvent_t take_event(polyglot_ctx* ctx) {
  if (!ctx->ev_pool.empty()) {
    hipEvent_t ev = ctx->ev_pool.back();
    ctx->ev_pool.pop_back();
    return ev;
  }
  hipEvent_t ev = nullptr;
  if (hipEventCreate(&ev) != hipSuccess) return nullptr;
  return ev;
}

// Takes all event pairs into the kernels' totals, then moves those of the kernel ids
// [first, first + n) out to ms and launches; the others' stay for their own question.
inline int collect_times(polyglot_ctx* ctx, int first, int n, double* ms, int32_t* launches,
                         const char* what) {
  hipError_t e = hipStreamSynchronize(ctx->stream);
  if (e == hipSuccess) e = hipStreamSynchronize(ctx->side);
  if (e != hipSuccess) return hip_fail(ctx, e, what);
  for (auto& m : ctx->ev_marks) {
    float t = 0.f;
    if (hipEventElapsedTime(&t, m.second.first, m.second.second) == hipSuccess) {
      ctx->times[m.first].ms += t;
      ctx->times[m.first].launches += 1;
    }
    ctx->ev_pool.push_back(m.second.first);
    ctx->ev_pool.push_back(m.second.second);
  }
  ctx->ev_marks.clear();
  for (int k = 0; k < n; ++k) {
    KernelTime& t = ctx->times[first + k];
    ms[k] = t.ms;
    launches[k] = t.launches;
    t = KernelTime{};
  }
  return POLYGLOT_OK;
}

// Launch parameters for kernel id `kid` on stream `st`.  When timing is on
// (and no graph is being captured) every launch made with it gets its own
// start/stop event pair, bound to the kernel's dispatch.
struct Timed {
  polyglot_ctx* ctx;
  int kid;
  Launch L;
  Timed(polyglot_ctx* c, int k, hipStream_t st) : ctx(c), kid(k) {
    L.s = st;
    if (ctx->timing && !ctx->capturing) {
      L.owner = this;
      L.take = &Timed::take;
    }
  }
  Timed(polyglot_ctx* c, int k) : Timed(c, k, c->stream) {}
  Timed(const Timed&) = delete;
  Timed& operator=(const Timed&) = delete;
  static bool take(void* owner, hipEvent_t* start, hipEvent_t* stop) {
    Timed* t = static_cast<Timed*>(owner);
    hipEvent_t a = take_event(t->ctx), b = take_event(t->ctx);
    if (!a || !b) {
      if (a) t->ctx->ev_pool.push_back(a);
      if (b) t->ctx->ev_pool.push_back(b);
      return false;
    }
    t->ctx->ev_marks.push_back({t->kid, {a, b}});
    *start = a;
    *stop = b;
    return true;
  }
};

}  // namespace pg
