// Entry points of the convolution, the selective scan, the beams' selection and the
// reordering (include/polyglot.h): argument checks, workspace, launches.
#include "polyglot.h"

#include "entry.h"

using namespace pg;

namespace {

constexpr int64_t kMaxTokens = 1 << 30;
constexpr int kMaxChannels = 1 << 20, kMaxStates = 64;
constexpr int64_t kMaxRowDistance = (1 << 25) - 1;  // a tile's offsets fit 32 bits
constexpr int64_t kMaxBeamParts = 1 << 23;  // workgroups of the selection

int64_t beam_parts(int64_t V) { return (V + kBeamMinPart - 1) / kBeamMinPart; }

// No output may be an input, or an output twice.
bool apart(std::initializer_list<const void*> outs, std::initializer_list<const void*> ins) {
  for (auto a = outs.begin(); a != outs.end(); ++a) {
    if (!*a) continue;
    for (const void* b : ins)
      if (*a == b) return false;
    for (auto b = a + 1; b != outs.end(); ++b)
      if (*a == *b) return false;
  }
  return true;
}

bool all_aligned(std::initializer_list<const void*> all, size_t to) {
  for (const void* p : all)
    if (!aligned(p, to)) return false;
  return true;
}

// What the packed calls share.
template <class A>
int check_packed(polyglot_ctx* ctx, const A& a, const std::string& what) {
  if (a.tokens < 0 || a.tokens > kMaxTokens || a.nseq < 1 || a.nseq > kMaxTokens)
    return fail(ctx, POLYGLOT_EBATCH, what + ": bad token or sequence count");
  if (a.D < 1 || a.D > kMaxChannels || !format_ok(a.dtype))
    return fail(ctx, POLYGLOT_EINVAL, what + ": bad width or storage format");
  if (a.offsets ? a.offset_bytes != 4 && a.offset_bytes != 8 : a.tokens % a.nseq != 0)
    return fail(ctx, POLYGLOT_EINVAL, what + ": offsets of 4 or 8 bytes, or sequences of one length");
  if (a.offsets && !aligned(a.offsets, a.offset_bytes))
    return fail(ctx, POLYGLOT_EINVAL, what + ": misaligned offsets");
  return POLYGLOT_OK;
}

template <class A>
Packed packed(polyglot_ctx* ctx, const A& a) {
  return Packed{a.offsets, ctx->ws.flag, a.offset_bytes, (int)a.tokens, a.nseq};
}

template <class A>
bool single(const A& a) {
  return !a.offsets && a.tokens == a.nseq;
}

template <class A>
int check_convolution(polyglot_ctx* ctx, const A& a, const std::string& what) {
  const int rc = check_packed(ctx, a, what);
  if (rc) return rc;
  if (a.taps < 1 || a.taps > kConvMaxK) return fail(ctx, POLYGLOT_EINVAL, what + ": 1 to 4 taps");
  if (!a.weight) return fail(ctx, POLYGLOT_ENULL, what + ": NULL weight");
  if (!all_aligned({a.weight, a.bias}, 4) || !aligned(a.state, size_of(a.dtype)))
    return fail(ctx, POLYGLOT_EINVAL, what + ": misaligned weight, bias or state");
  return POLYGLOT_OK;
}

template <class A>
int check_selective(polyglot_ctx* ctx, const A& a, const std::string& what) {
  const int rc = check_packed(ctx, a, what);
  if (rc) return rc;
  if (a.states < 1 || a.states > kMaxStates || a.groups < 1 || a.D % a.groups != 0)
    return fail(ctx, POLYGLOT_EINVAL, what + ": 1 to 64 states, groups that divide D");
  if (!a.A) return fail(ctx, POLYGLOT_ENULL, what + ": NULL A");
  if (!all_aligned({a.A, a.skip, a.delta_bias, a.h0}, 4) || !aligned(a.marks, 16))
    return fail(ctx, POLYGLOT_EINVAL, what + ": misaligned pointer");
  return POLYGLOT_OK;
}

// Only the gradient's room goes by the tokens (dB and dC of the workgroups).
template <class A>
int check_selective_room(polyglot_ctx* ctx, const A& a, bool grad, const std::string& what) {
  const OpWorkspace& op = ctx->op;
  if (!op.sel || a.D > op.sel_D || a.states > op.sel_states)
    return fail(ctx, POLYGLOT_EBATCH, what + ": above the reserved channels or states");
  if (grad && a.tokens > op.sel_tokens)
    return fail(ctx, POLYGLOT_EBATCH, what + ": above the reserved tokens");
  return POLYGLOT_OK;
}

template <class A>
SelCall selective_call(polyglot_ctx* ctx, const A& a) {
  SelCall c{};
  c.x = a.x;
  c.delta = a.delta;
  c.B = a.B;
  c.C = a.C;
  c.z = a.z;
  c.A = a.A;
  c.skip = a.skip;
  c.bias = a.delta_bias;
  c.h0 = a.h0;
  c.ld_x = a.ld_x;
  c.ld_delta = a.ld_delta;
  c.ld_B = a.ld_B;
  c.ld_C = a.ld_C;
  c.ld_z = a.ld_z;
  c.seqs = packed(ctx, a);
  c.D = a.D;
  c.N = a.states;
  c.groups = a.groups;
  c.softplus = a.softplus != 0;
  return c;
}

}  // namespace

extern "C" {

int polyglot_convolution(polyglot_ctx* ctx, const polyglot_convolution_args* args) {
  if (!ctx || !args) return POLYGLOT_ENULL;
  return entry([&] {
    const polyglot_convolution_args& a = *args;
    int rc = check_convolution(ctx, a, "convolution");
    if (rc) return rc;
    const size_t es = size_of(a.dtype);
    rc = check_rows(ctx, a.tokens, es, {{a.x, a.ld_x, a.D}, {a.y, a.ld_y, a.D}}, "convolution");
    if (rc) return rc;
    if (!aligned(a.last, es)) return fail(ctx, POLYGLOT_EINVAL, "convolution: misaligned state");
    if (!apart({a.y, a.last}, {a.x, a.weight, a.bias, single(a) && a.last == a.state ? nullptr : a.state}))
      return fail(ctx, POLYGLOT_EINVAL, "convolution: an output overlaps another tensor");
    ConvCall c{};
    c.x = a.x;
    c.state = a.state;
    c.weight = a.weight;
    c.bias = a.bias;
    c.y = a.y;
    c.last = a.last;
    c.ld_x = a.ld_x;
    c.ld_y = a.ld_y;
    c.seqs = packed(ctx, a);
    c.D = a.D;
    c.silu = a.silu != 0;
    Timed tm(ctx, kOpKernels + POLYGLOT_OPK_CONVOLUTION);
    const hipError_t e = single(a) ? launch_convolution_step(c, a.taps, a.dtype, tm.L)
                                   : launch_convolution(c, a.taps, a.dtype, tm.L);
    return e == hipSuccess ? POLYGLOT_OK : hip_fail(ctx, e, "convolution launch");
  });
}

int polyglot_convolution_grad(polyglot_ctx* ctx, const polyglot_convolution_grad_args* args) {
  if (!ctx || !args) return POLYGLOT_ENULL;
  return entry([&] {
    const polyglot_convolution_grad_args& a = *args;
    int rc = check_convolution(ctx, a, "convolution_grad");
    if (rc) return rc;
    const size_t es = size_of(a.dtype);
    rc = check_rows(ctx, a.tokens, es, {{a.x, a.ld_x, a.D}, {a.dy, a.ld_dy, a.D}, {a.dx, a.ld_dx, a.D}},
                    "convolution_grad");
    if (rc) return rc;
    if (!a.dweight) return fail(ctx, POLYGLOT_ENULL, "convolution_grad: NULL dweight");
    if (!all_aligned({a.dweight, a.dbias}, 4) || !all_aligned({a.dlast, a.dstate}, es))
      return fail(ctx, POLYGLOT_EINVAL, "convolution_grad: misaligned pointer");
    if (!apart({a.dx, a.dweight, a.dbias, a.dstate}, {a.x, a.weight, a.bias, a.state, a.dy, a.dlast}))
      return fail(ctx, POLYGLOT_EINVAL, "convolution_grad: an output overlaps another tensor");
    if (!ctx->op.sel || a.D > ctx->op.sel_D)
      return fail(ctx, POLYGLOT_EBATCH, "convolution_grad: above the reserved channels");
    ConvCall c{};
    c.x = a.x;
    c.state = a.state;
    c.weight = a.weight;
    c.bias = a.bias;
    c.dy = a.dy;
    c.dlast = a.dlast;
    c.dx = a.dx;
    c.dweight = a.dweight;
    c.dbias = a.dbias;
    c.dstate = a.dstate;
    c.ld_x = a.ld_x;
    c.ld_dy = a.ld_dy;
    c.ld_dx = a.ld_dx;
    c.seqs = packed(ctx, a);
    c.D = a.D;
    c.silu = a.silu != 0;
    c.part = ctx->op.conv_part;
    Timed tm(ctx, kOpKernels + POLYGLOT_OPK_CONVOLUTION_GRAD);
    const hipError_t e = launch_convolution_grad(c, a.taps, a.dtype, tm.L);
    return e == hipSuccess ? POLYGLOT_OK : hip_fail(ctx, e, "convolution_grad launch");
  });
}

int polyglot_selective(polyglot_ctx* ctx, const polyglot_selective_args* args) {
  if (!ctx || !args) return POLYGLOT_ENULL;
  return entry([&] {
    const polyglot_selective_args& a = *args;
    int rc = check_selective(ctx, a, "selective");
    if (rc) return rc;
    const bool step = single(a) && !a.marks;
    const int GN = a.groups * a.states;
    rc = check_rows(ctx, a.tokens, size_of(a.dtype),
                    {{a.x, a.ld_x, a.D}, {a.delta, a.ld_delta, a.D}, {a.B, a.ld_B, GN}, {a.C, a.ld_C, GN},
                     {a.y, a.ld_y, a.D}, a.z ? Rows{a.z, a.ld_z, a.D} : Rows{a.x, a.ld_x, a.D}},
                    "selective", kMaxRowDistance);
    if (rc) return rc;
    if (!aligned(a.last, 4)) return fail(ctx, POLYGLOT_EINVAL, "selective: misaligned state");
    if (!apart({a.y, a.last, a.marks}, {a.x, a.delta, a.B, a.C, a.z, a.A, a.skip, a.delta_bias,
                                        step && a.last == a.h0 ? nullptr : a.h0}))
      return fail(ctx, POLYGLOT_EINVAL, "selective: an output overlaps another tensor");
    SelCall c = selective_call(ctx, a);
    c.y = a.y;
    c.ld_y = a.ld_y;
    c.last = a.last;
    c.marks = a.marks;
    hipError_t e;
    if (step) {
      Timed tm(ctx, kOpKernels + POLYGLOT_OPK_SELECTIVE);
      e = launch_selective_step(c, a.dtype, tm.L);
    } else {
      rc = check_selective_room(ctx, a, false, "selective");
      if (rc) return rc;
      Timed tm(ctx, kOpKernels + POLYGLOT_OPK_SELECTIVE);
      e = launch_selective(c, a.dtype, ctx->op.sel_space, tm.L);
    }
    return e == hipSuccess ? POLYGLOT_OK : hip_fail(ctx, e, "selective launch");
  });
}

int polyglot_selective_grad(polyglot_ctx* ctx, const polyglot_selective_grad_args* args) {
  if (!ctx || !args) return POLYGLOT_ENULL;
  return entry([&] {
    const polyglot_selective_grad_args& a = *args;
    int rc = check_selective(ctx, a, "selective_grad");
    if (rc) return rc;
    const int GN = a.groups * a.states;
    const Rows x{a.x, a.ld_x, a.D};
    rc = check_rows(ctx, a.tokens, size_of(a.dtype),
                    {x, {a.delta, a.ld_delta, a.D}, {a.B, a.ld_B, GN}, {a.C, a.ld_C, GN}, {a.dy, a.ld_dy, a.D},
                     a.z ? Rows{a.z, a.ld_z, a.D} : x, {a.dx, a.ld_dx, a.D}, {a.ddelta, a.ld_ddelta, a.D},
                     {a.dB, a.ld_dB, GN}, {a.dC, a.ld_dC, GN}, a.z ? Rows{a.dz, a.ld_dz, a.D} : x},
                    "selective_grad", kMaxRowDistance);
    if (rc) return rc;
    if (!a.dA || (a.tokens > 0 && !a.marks))
      return fail(ctx, POLYGLOT_ENULL, "selective_grad: NULL dA or marks");
    if (!all_aligned({a.dlast, a.dA, a.dskip, a.ddelta_bias, a.dh0}, 4))
      return fail(ctx, POLYGLOT_EINVAL, "selective_grad: misaligned pointer");
    if (!apart({a.dx, a.ddelta, a.dB, a.dC, a.z ? a.dz : nullptr, a.dA, a.dskip, a.ddelta_bias, a.dh0},
               {a.x, a.delta, a.B, a.C, a.z, a.dy, a.A, a.skip, a.delta_bias, a.h0, a.dlast, a.marks}))
      return fail(ctx, POLYGLOT_EINVAL, "selective_grad: an output overlaps another tensor");
    rc = check_selective_room(ctx, a, true, "selective_grad");
    if (rc) return rc;
    SelCall c = selective_call(ctx, a);
    c.dy = a.dy;
    c.ld_dy = a.ld_dy;
    c.dlast = a.dlast;
    c.marks = const_cast<float*>(a.marks);
    c.dx = a.dx;
    c.ddelta = a.ddelta;
    c.dB = a.dB;
    c.dC = a.dC;
    c.dz = a.dz;
    c.dA = a.dA;
    c.dskip = a.dskip;
    c.dbias = a.ddelta_bias;
    c.dh0 = a.dh0;
    c.ld_dx = a.ld_dx;
    c.ld_ddelta = a.ld_ddelta;
    c.ld_dB = a.ld_dB;
    c.ld_dC = a.ld_dC;
    c.ld_dz = a.ld_dz;
    Timed tm(ctx, kOpKernels + POLYGLOT_OPK_SELECTIVE_GRAD);
    const hipError_t e = launch_selective_grad(c, a.dtype, ctx->op.sel_space, tm.L);
    return e == hipSuccess ? POLYGLOT_OK : hip_fail(ctx, e, "selective_grad launch");
  });
}

int polyglot_reserve_selective(polyglot_ctx* ctx, int64_t max_tokens, int32_t max_D, int32_t max_states) {
  if (!ctx) return POLYGLOT_ENULL;
  return entry([&] {
    if (max_tokens < 0 || max_tokens > kMaxTokens || max_D < 0 || max_D > kMaxChannels || max_states < 0 ||
        max_states > kMaxStates)
      return fail(ctx, POLYGLOT_EINVAL, "reserve_selective: bad token count, width or states");
    OpWorkspace& op = ctx->op;
    hipError_t e = hipStreamSynchronize(ctx->stream);
    if (e != hipSuccess) return hip_fail(ctx, e, "reserve_selective: sync");
    if (op.sel) e = hipFree(op.sel);
    op.sel = nullptr;
    op.sel_tokens = 0;
    op.sel_D = op.sel_states = 0;
    const SelRoom r = selective_room(max_tokens, max_D, max_states);
    const size_t conv = convolution_room(max_D);
    // every part starts at a multiple of 64 words
    const auto up = [](size_t n) { return (n + 63) / 64 * 64; };
    const size_t scan = up(r.states) + up(r.sums) + up(r.info) + up(r.states) + up(r.part_s) + up(r.part_bc);
    float* p = nullptr;
    if (e == hipSuccess) e = hipMalloc(reinterpret_cast<void**>(&p), (scan + up(conv)) * sizeof(float));
    if (e != hipSuccess) return hip_fail(ctx, e, "reserve_selective");
    op.sel = p;
    SelSpace& s = op.sel_space;
    const auto take = [&](size_t n) {
      float* q = p;
      p += up(n);
      return q;
    };
    s.states = take(r.states);
    s.sums = take(r.sums);
    s.info = reinterpret_cast<uint32_t*>(take(r.info));
    s.part_a = take(r.states);
    s.part_s = take(r.part_s);
    s.part_bc = take(r.part_bc);
    op.conv_part = take(conv);
    op.sel_tokens = max_tokens;
    op.sel_D = max_D;
    op.sel_states = max_states;
    return POLYGLOT_OK;
  });
}

int polyglot_beam(polyglot_ctx* ctx, const polyglot_beam_args* args) {
  if (!ctx || !args) return POLYGLOT_ENULL;
  return entry([&] {
    const polyglot_beam_args& a = *args;
    if (a.groups < 0 || a.beams < 1 || (int64_t)a.groups * a.beams > INT32_MAX)
      return fail(ctx, POLYGLOT_EBATCH, "beam: bad group or beam count");
    if (a.V < 1 || a.V > (1 << 30) || (int64_t)a.beams * a.V >= (int64_t)1 << 32 || !format_ok(a.dtype))
      return fail(ctx, POLYGLOT_EINVAL, "beam: bad vocabulary or storage format, or too many words of a group");
    if (a.picks < 1 || a.picks > kBeamPicks) return fail(ctx, POLYGLOT_EINVAL, "beam: 1 to 64 picks");
    if (a.groups == 0) return POLYGLOT_OK;
    const int rows = a.groups * a.beams;
    const int rc = check_rows(ctx, rows, size_of(a.dtype), {{a.scores, a.ld_scores, a.V}}, "beam");
    if (rc) return rc;
    if (!a.total || !a.parent || !a.token || !a.out) return fail(ctx, POLYGLOT_ENULL, "beam: NULL pointer");
    if (!all_aligned({a.total, a.lse, a.finished, a.parent, a.token, a.out}, 4))
      return fail(ctx, POLYGLOT_EINVAL, "beam: misaligned pointer");
    if (a.finished && (a.end < 0 || a.end >= a.V))
      return fail(ctx, POLYGLOT_EINVAL, "beam: the end is no word");
    // total may be out: the second launch alone writes, and reads neither
    if (!apart({a.parent, a.token, a.out},
               {a.scores, a.lse, a.finished, a.out == a.total ? nullptr : a.total}))
      return fail(ctx, POLYGLOT_EINVAL, "beam: an output overlaps another tensor");
    const OpWorkspace& op = ctx->op;
    if (!op.beam_keys || rows > op.beam_rows || a.V > op.beam_V || a.picks > op.beam_picks)
      return fail(ctx, POLYGLOT_EBATCH, "beam: above the reserved rows, vocabulary or picks");
    BeamCall c{};
    c.scores = a.scores;
    c.total = a.total;
    c.lse = a.lse;
    c.finished = a.finished;
    c.parent = a.parent;
    c.token = a.token;
    c.out = a.out;
    c.keys = op.beam_keys;
    c.ld = a.ld_scores;
    c.groups = a.groups;
    c.beams = a.beams;
    c.V = a.V;
    c.picks = a.picks;
    c.end = a.end;
    Timed tm(ctx, kOpKernels + POLYGLOT_OPK_BEAM);
    const hipError_t e = launch_beam(c, a.dtype, tm.L);
    return e == hipSuccess ? POLYGLOT_OK : hip_fail(ctx, e, "beam launch");
  });
}

int polyglot_reserve_beam(polyglot_ctx* ctx, int32_t max_rows, int32_t max_V, int32_t max_picks) {
  if (!ctx) return POLYGLOT_ENULL;
  return entry([&] {
    if (max_rows < 0 || max_V < 0 || max_V > (1 << 30) || max_picks < 0 || max_picks > kBeamPicks ||
        max_rows * beam_parts(max_V) > kMaxBeamParts)
      return fail(ctx, POLYGLOT_EINVAL, "reserve_beam: bad rows, vocabulary or picks");
    OpWorkspace& op = ctx->op;
    hipError_t e = hipStreamSynchronize(ctx->stream);
    if (e != hipSuccess) return hip_fail(ctx, e, "reserve_beam: sync");
    if (op.beam_keys) e = hipFree(op.beam_keys);
    op.beam_keys = nullptr;
    op.beam_rows = op.beam_V = op.beam_picks = 0;
    uint64_t* p = nullptr;
    const size_t n = (size_t)max_rows * beam_parts(max_V) * max_picks + 1;
    if (e == hipSuccess) e = hipMalloc(reinterpret_cast<void**>(&p), n * sizeof(uint64_t));
    if (e != hipSuccess) return hip_fail(ctx, e, "reserve_beam");
    op.beam_keys = p;
    op.beam_rows = max_rows;
    op.beam_V = max_V;
    op.beam_picks = max_picks;
    return POLYGLOT_OK;
  });
}

int polyglot_reorder(polyglot_ctx* ctx, const polyglot_row_copy* items, int32_t count, const int32_t* ids,
                     int32_t rows) {
  if (!ctx) return POLYGLOT_ENULL;
  return entry([&] {
    if (count < 0 || rows < 0) return fail(ctx, POLYGLOT_EBATCH, "reorder: bad count");
    if (count == 0 || rows == 0) return POLYGLOT_OK;
    if (!items || !ids) return fail(ctx, POLYGLOT_ENULL, "reorder: NULL pointer");
    if (!aligned(ids, 4)) return fail(ctx, POLYGLOT_EINVAL, "reorder: misaligned ids");
    for (int i = 0; i < count; ++i) {
      const polyglot_row_copy& m = items[i];
      if (m.row_bytes < 0 || m.in_rows < 1 || !rows_ok(m.ld_in, m.in_rows, m.row_bytes) ||
          !rows_ok(m.ld_out, rows, m.row_bytes))
        return fail(ctx, POLYGLOT_EINVAL, "reorder: rows closer than their length, or too many");
      if (m.row_bytes > 0 && (!m.in || !m.out)) return fail(ctx, POLYGLOT_ENULL, "reorder: NULL pointer");
      for (int j = 0; j < count && m.row_bytes > 0; ++j)
        if (m.out == items[j].in || (i != j && m.out == items[j].out))
          return fail(ctx, POLYGLOT_EINVAL, "reorder: an output overlaps another tensor");
    }
    Timed tm(ctx, kOpKernels + POLYGLOT_OPK_REORDER);
    for (int from = 0; from < count; from += kReorderItems) {
      ReorderCall c{};
      c.ids = ids;
      c.flag = ctx->ws.flag;
      c.rows = rows;
      for (int i = from; i < std::min(count, from + kReorderItems); ++i) {
        const polyglot_row_copy& m = items[i];
        if (m.row_bytes == 0) continue;
        RowCopy r{};
        r.in = static_cast<const char*>(m.in);
        r.out = static_cast<char*>(m.out);
        r.row_bytes = m.row_bytes;
        r.ld_in = m.ld_in;
        r.ld_out = m.ld_out;
        r.in_rows = m.in_rows;
        r.pieces = (m.row_bytes + kReorderPiece - 1) / kReorderPiece;
        const uint64_t all = reinterpret_cast<uintptr_t>(m.in) | reinterpret_cast<uintptr_t>(m.out) |
                             (uint64_t)m.row_bytes | (uint64_t)(m.in_rows > 1 ? m.ld_in : 0) |
                             (uint64_t)(rows > 1 ? m.ld_out : 0);
        r.unit = all % 16 == 0 ? 16 : all % 4 == 0 ? 4 : all % 2 == 0 ? 2 : 1;
        c.item[c.count] = r;
        c.first[c.count + 1] = c.first[c.count] + r.pieces * rows;
        ++c.count;
      }
      const hipError_t e = launch_reorder(c, tm.L);
      if (e != hipSuccess) return hip_fail(ctx, e, "reorder launch");
    }
    return POLYGLOT_OK;
  });
}

}  // extern "C"
