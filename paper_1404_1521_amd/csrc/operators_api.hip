// Entry points of the sequence operators (include/polyglot.h): argument
// checks, workspace, launches.
#include "polyglot.h"

#include <cmath>

#include "entry.h"

using namespace pg;

namespace {

// Most parts of a row of V scores.
int64_t logits_parts(int V) { return (V + (int64_t)kLogitsMinTile - 1) / kLogitsMinTile; }

constexpr int kLogitsMaxV = 1 << 30;  // places in a row fit an int

// A zeroed block of `lines` words of counters, each line's first with tag 1, and
// `words` more behind them (their tag 0: nothing has written them).  All of it is made on
// the device: the counters of many rows are gigabytes.
hipError_t heads(polyglot_ctx* ctx, uint64_t** head, size_t lines, size_t words) {
  const size_t n = lines + words + 1;
  uint64_t* p = nullptr;
  hipError_t e = hipMalloc(reinterpret_cast<void**>(&p), n * sizeof(uint64_t));
  if (e != hipSuccess) return e;
  e = hipMemsetAsync(p, 0, n * sizeof(uint64_t), ctx->stream);
  if (e == hipSuccess && lines > 0)  // the lowest byte of each line's tag
    e = hipMemset2DAsync(reinterpret_cast<char*>(p) + 4, kHeadLine * sizeof(uint64_t), 1, 1,
                         lines / kHeadLine, ctx->stream);
  if (e == hipSuccess) e = hipStreamSynchronize(ctx->stream);
  if (e == hipSuccess) *head = p;
  else (void)hipFree(p);
  return e;
}

}  // namespace

extern "C" {

int polyglot_dropout(polyglot_ctx* ctx, const polyglot_dropout_args* args) {
  if (!ctx || !args) return POLYGLOT_ENULL;
  return entry([&] {
    const polyglot_dropout_args& a = *args;
    if (a.rows < 0) return fail(ctx, POLYGLOT_EBATCH, "dropout: rows must not be negative");
    if (a.d < 1 || !format_ok(a.dtype) || !(a.p >= 0.f && a.p <= 1.f))
      return fail(ctx, POLYGLOT_EINVAL, "dropout: bad width, storage format or p");
    if (a.ids && ((a.id_bytes != 4 && a.id_bytes != 8) || a.table_rows < 1))
      return fail(ctx, POLYGLOT_EINVAL, "dropout: bad id size or table");
    if (a.rows == 0) return POLYGLOT_OK;
    if (!a.x || !a.y) return fail(ctx, POLYGLOT_ENULL, "dropout: NULL pointer");
    if (!rows_ok(a.ld_x, a.ids ? a.table_rows : a.rows, a.d) || !rows_ok(a.ld_y, a.rows, a.d) ||
        (a.add && !rows_ok(a.ld_add, a.rows, a.d)))
      return fail(ctx, POLYGLOT_EINVAL, "dropout: rows closer than their width, or too many");
    if ((a.y == a.x && (a.ids || a.ld_y != a.ld_x)) || (a.y == a.add && a.ld_y != a.ld_add))
      return fail(ctx, POLYGLOT_EINVAL, "dropout: y overlaps an input with other rows");
    const size_t es = size_of(a.dtype);
    if (!aligned(a.x, es) || !aligned(a.add, es) || !aligned(a.y, es) ||
        (a.ids && !aligned(a.ids, a.id_bytes)) || !aligned(a.site_dev, 4))
      return fail(ctx, POLYGLOT_EINVAL, "dropout: misaligned pointer");
    DropoutCall c{};
    c.a = a;
    c.flag = ctx->ws.flag;
    c.threshold = (uint32_t)(a.p * 65536.0 + 0.5);
    c.groups = (int)((a.d + 7LL) / 8);
    c.groups_inv = (uint32_t)(((1ull << 32) + c.groups - 1) / c.groups);
    if (c.threshold < 65536u) c.scale = (float)(65536.0 / (65536u - c.threshold));
    Timed tm(ctx, kOpKernels + POLYGLOT_OPK_DROPOUT);
    const hipError_t e = launch_dropout(c, tm.L);
    return e == hipSuccess ? POLYGLOT_OK : hip_fail(ctx, e, "dropout launch");
  });
}

}  // extern "C"

namespace {

// The checks that the recurrence and its gradient share; `what` names the call.
template <class A>
int check_recurrence(polyglot_ctx* ctx, const A& a, const std::string& what) {
  if (a.tokens < 0 || a.tokens > INT32_MAX || a.nseq < 1)
    return fail(ctx, POLYGLOT_EBATCH, what + ": bad token or sequence count");
  if (a.D < 1 || a.group < 1 || a.group > 256 || a.D % a.group != 0)
    return fail(ctx, POLYGLOT_EINVAL, what + ": D must be whole groups of at most 256 channels");
  if (!format_ok(a.dtype))
    return fail(ctx, POLYGLOT_EINVAL, what + ": bad storage format");
  if (a.form != POLYGLOT_GATE_RAW && a.form != POLYGLOT_GATE_SIGMOID)
    return fail(ctx, POLYGLOT_EINVAL, what + ": bad form of the gate");
  if (a.offsets ? a.offset_bytes != 4 && a.offset_bytes != 8 : a.tokens % a.nseq != 0)
    return fail(ctx, POLYGLOT_EINVAL, what + ": offsets of 4 or 8 bytes, or sequences of one length");
  if (a.offsets && !aligned(a.offsets, a.offset_bytes))
    return fail(ctx, POLYGLOT_EINVAL, what + ": misaligned offsets");
  // one token per sequence needs no scan; other calls use the reserved workspace
  if ((a.offsets || a.tokens != a.nseq) &&
      (!ctx->op.rec.head || a.tokens > ctx->op.rec_tokens || a.D > ctx->op.rec_D))
    return fail(ctx, POLYGLOT_EBATCH, what + ": above the reserved tokens or channels");
  return POLYGLOT_OK;
}

template <class A>
RecCall recurrence_call(polyglot_ctx* ctx, const A& a) {
  RecCall c{};
  c.gate = a.gate;
  c.x = a.x;
  c.h0 = a.h0;
  c.offsets = a.offsets;
  c.flag = ctx->ws.flag;
  c.ld_gate = a.ld_gate;
  c.ld_x = a.ld_x;
  c.tokens = (int)a.tokens;
  c.nseq = a.nseq;
  c.D = a.D;
  c.group = a.group;
  c.offset_bytes = a.offset_bytes;
  return c;
}

}  // namespace

extern "C" {

int polyglot_recurrence(polyglot_ctx* ctx, const polyglot_recurrence_args* args) {
  if (!ctx || !args) return POLYGLOT_ENULL;
  return entry([&] {
    const polyglot_recurrence_args& a = *args;
    int rc = check_recurrence(ctx, a, "recurrence");
    if (rc) return rc;
    rc = check_rows(ctx, a.tokens, size_of(a.dtype),
                    {{a.gate, a.ld_gate, a.D / a.group}, {a.x, a.ld_x, a.D}, {a.h, a.ld_h, a.D}},
                    "recurrence");
    if (rc) return rc;
    if (!aligned(a.h0, 4) || !aligned(a.last, 4))
      return fail(ctx, POLYGLOT_EINVAL, "recurrence: misaligned state");
    if (a.tokens > 0 && ((a.h == a.x && a.ld_h != a.ld_x) || a.h == a.gate))
      return fail(ctx, POLYGLOT_EINVAL, "recurrence: h overlaps an input with other rows");
    RecCall c = recurrence_call(ctx, a);
    c.init = a.h0;
    c.out = a.h;
    c.ld_out = a.ld_h;
    c.fin = a.last;
    c.down = a.reverse != 0;
    Timed tm(ctx, kOpKernels + POLYGLOT_OPK_RECURRENCE);
    const hipError_t e = launch_recurrence(c, a.dtype, a.form, false, ctx->op.rec, tm.L);
    return e == hipSuccess ? POLYGLOT_OK : hip_fail(ctx, e, "recurrence launch");
  });
}

int polyglot_recurrence_grad(polyglot_ctx* ctx, const polyglot_recurrence_grad_args* args) {
  if (!ctx || !args) return POLYGLOT_ENULL;
  return entry([&] {
    const polyglot_recurrence_grad_args& a = *args;
    int rc = check_recurrence(ctx, a, "recurrence_grad");
    if (rc) return rc;
    const int gates = a.D / a.group;
    const bool raw = a.form == POLYGLOT_GATE_RAW;
    rc = check_rows(ctx, a.tokens, size_of(a.dtype),
                    {{a.gate, a.ld_gate, gates}, {a.h, a.ld_h, a.D}, {a.dh, a.ld_dh, a.D},
                     {a.dgate, a.ld_dgate, gates}, {a.dx, a.ld_dx, a.D},
                     raw ? Rows{a.dx, a.ld_dx, a.D} : Rows{a.x, a.ld_x, a.D}},
                    "recurrence_grad");
    if (rc) return rc;
    if (!aligned(a.h0, 4) || !aligned(a.dlast, 4) || !aligned(a.dh0, 4))
      return fail(ctx, POLYGLOT_EINVAL, "recurrence_grad: misaligned state");
    if (a.tokens > 0 &&
        (a.dx == a.h || a.dx == a.gate || (a.dx == a.dh && a.ld_dx != a.ld_dh) ||
         (a.dx == a.x && a.ld_dx != a.ld_x) || a.dgate == a.gate || a.dgate == a.x ||
         a.dgate == a.h || a.dgate == a.dh || a.dgate == a.dx))
      return fail(ctx, POLYGLOT_EINVAL, "recurrence_grad: an output overlaps another tensor");
    RecCall c = recurrence_call(ctx, a);
    c.h = a.h;
    c.dh = a.dh;
    c.ld_h = a.ld_h;
    c.ld_dh = a.ld_dh;
    c.init = a.dlast;
    c.out = a.dx;
    c.ld_out = a.ld_dx;
    c.dgate = a.dgate;
    c.ld_dgate = a.ld_dgate;
    c.fin = a.dh0;
    c.down = a.reverse == 0;
    Timed tm(ctx, kOpKernels + POLYGLOT_OPK_RECURRENCE_GRAD);
    const hipError_t e = launch_recurrence(c, a.dtype, a.form, true, ctx->op.rec, tm.L);
    return e == hipSuccess ? POLYGLOT_OK : hip_fail(ctx, e, "recurrence_grad launch");
  });
}

int polyglot_reserve_recurrence(polyglot_ctx* ctx, int64_t max_tokens, int32_t max_D) {
  if (!ctx) return POLYGLOT_ENULL;
  return entry([&] {
    if (max_tokens < 0 || max_tokens > INT32_MAX || max_D < 0)
      return fail(ctx, POLYGLOT_EINVAL, "reserve_recurrence: bad token count or width");
    OpWorkspace& op = ctx->op;
    hipError_t e = hipStreamSynchronize(ctx->stream);
    if (e != hipSuccess) return hip_fail(ctx, e, "reserve_recurrence: sync");
    if (op.rec.head) e = hipFree(op.rec.head);
    op.rec = ScanSpace{};
    op.rec_tokens = op.rec_D = 0;
    ScanSpace sp = scan_space(max_tokens, max_D);
    if (e == hipSuccess)
      e = heads(ctx, &sp.head, (size_t)sp.counters * kHeadLine, sp.flags + sp.words);
    if (e != hipSuccess) return hip_fail(ctx, e, "reserve_recurrence");
    op.rec = sp;
    op.rec_tokens = max_tokens;
    op.rec_D = max_D;
    return POLYGLOT_OK;
  });
}

int polyglot_logits(polyglot_ctx* ctx, const polyglot_logits_args* args) {
  if (!ctx || !args) return POLYGLOT_ENULL;
  return entry([&] {
    const polyglot_logits_args& a = *args;
    if (a.rows < 0) return fail(ctx, POLYGLOT_EBATCH, "logits: rows must not be negative");
    if (a.V < 1 || a.V > kLogitsMaxV || !format_ok(a.dtype) || a.history_cap < 0)
      return fail(ctx, POLYGLOT_EINVAL, "logits: bad vocabulary, storage format or history_cap");
    if (a.rows == 0) return POLYGLOT_OK;
    if (!a.logits) return fail(ctx, POLYGLOT_ENULL, "logits: NULL scores");
    if (!a.out && !a.token && !a.lse) return fail(ctx, POLYGLOT_ENULL, "logits: no output");
    if (!rows_ok(a.ld_logits, a.rows, a.V) || (a.out && !rows_ok(a.ld_out, a.rows, a.V)) ||
        (a.history && !rows_ok(a.ld_history, a.rows, a.history_cap)) ||
        (a.bias && a.ld_bias != 0 && !rows_ok(a.ld_bias, a.rows, a.V)))
      return fail(ctx, POLYGLOT_EINVAL, "logits: rows closer than their width, or too many");
    if (a.mask && (a.masks < 1 || !rows_ok(a.ld_mask, a.masks, (a.V + 31LL) / 32) ||
                   (!a.mask_rows && a.masks != 1 && a.masks != a.rows)))
      return fail(ctx, POLYGLOT_EINVAL, "logits: one mask, one per row, or mask_rows");
    if (a.out == a.logits && a.ld_out != a.ld_logits)
      return fail(ctx, POLYGLOT_EINVAL, "logits: out overlaps logits with other rows");
    const size_t es = size_of(a.dtype);
    if (!aligned(a.logits, es) || !aligned(a.out, es))
      return fail(ctx, POLYGLOT_EINVAL, "logits: misaligned scores");
    const void* words[] = {a.history, a.lengths, a.prompt, a.repetition, a.presence, a.frequency,
                           a.bias, a.mask, a.mask_rows, a.token, a.lse};
    for (const void* p : words)
      if (!aligned(p, 4)) return fail(ctx, POLYGLOT_EINVAL, "logits: misaligned pointer");
    OpWorkspace& op = ctx->op;
    if ((a.token || a.lse) && (!op.log_head || a.rows > op.log_rows || a.V > op.log_V))
      return fail(ctx, POLYGLOT_EBATCH, "logits: above the reserved rows or vocabulary");
    LogitsCall c{};
    c.a = a;
    c.flag = ctx->ws.flag;
    if (a.token || a.lse) {
      c.head = op.log_head;
      c.stride = logits_parts(op.log_V);
      c.words = op.log_words;
    }
    Timed tm(ctx, kOpKernels + POLYGLOT_OPK_LOGITS);
    const hipError_t e = launch_logits(c, tm.L);
    return e == hipSuccess ? POLYGLOT_OK : hip_fail(ctx, e, "logits launch");
  });
}

int polyglot_reserve_logits(polyglot_ctx* ctx, int32_t max_rows, int32_t max_V) {
  if (!ctx) return POLYGLOT_ENULL;
  return entry([&] {
    if (max_rows < 0 || max_V < 0)
      return fail(ctx, POLYGLOT_EINVAL, "reserve_logits: bad rows or vocabulary");
    OpWorkspace& op = ctx->op;
    hipError_t e = hipStreamSynchronize(ctx->stream);
    if (e != hipSuccess) return hip_fail(ctx, e, "reserve_logits: sync");
    if (op.log_head) e = hipFree(op.log_head);
    op.log_head = op.log_words = nullptr;
    op.log_rows = op.log_V = 0;
    const size_t lines = (size_t)max_rows * kHeadLine;
    e = e == hipSuccess ? heads(ctx, &op.log_head, lines, 3 * (size_t)max_rows * logits_parts(max_V))
                        : e;
    if (e != hipSuccess) return hip_fail(ctx, e, "reserve_logits");
    op.log_words = op.log_head + lines;
    op.log_rows = max_rows;
    op.log_V = max_V;
    return POLYGLOT_OK;
  });
}

int polyglot_operator_times(polyglot_ctx* ctx, double* ms, int32_t* launches) {
  if (!ctx || !ms || !launches) return POLYGLOT_ENULL;
  return entry([&] {
    return collect_times(ctx, kOpKernels, POLYGLOT_NOPKERNELS, ms, launches,
                         "operator_times: sync");
  });
}

}  // extern "C"
