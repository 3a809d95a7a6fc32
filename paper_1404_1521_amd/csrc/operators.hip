// Launches of the dropout and the scores.
#include "operators.h"

#include <algorithm>

#include "dropout_dev.h"
#include "logits_dev.h"

namespace pg {

namespace {

// A launch has fewer than 2^32 threads: larger tensors take several, of whole rows.
template <class T>
hipError_t dropout_of(const DropoutCall& call, const Launch& L) {
  auto k = call.a.ids ? (call.a.add ? k_dropout<T, true, true> : k_dropout<T, false, true>)
                      : (call.a.add ? k_dropout<T, true, false> : k_dropout<T, false, false>);
  const int64_t most = std::max<int64_t>(1, ((int64_t)1 << 31) / call.groups);
  for (int64_t row = 0; row < call.a.rows; row += most) {
    DropoutCall c = call;
    c.a.rows = std::min(most, call.a.rows - row);
    c.a.first_row += row;
    if (c.a.ids)
      c.a.ids = static_cast<const char*>(c.a.ids) + row * c.a.id_bytes;
    else
      c.a.x = static_cast<const T*>(c.a.x) + row * c.a.ld_x;
    if (c.a.add) c.a.add = static_cast<const T*>(c.a.add) + row * c.a.ld_add;
    c.a.y = static_cast<T*>(c.a.y) + row * c.a.ld_y;
    const int64_t grid = (c.a.rows * c.groups + kBlock - 1) / kBlock;
    const hipError_t e = pg_launch(k, dim3((uint32_t)grid), dim3(kBlock), 0, L, c);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// p, if it is there, `by` elements on.
template <class P>
void advance(P*& p, int64_t by) {
  if (p) p += by;
}

// The rows [row, row + rows) of a call.
template <class T>
LogitsCall logits_rows(LogitsCall c, int64_t row, int rows) {
  polyglot_logits_args& a = c.a;
  a.logits = static_cast<const T*>(a.logits) + row * a.ld_logits;
  if (a.out) a.out = static_cast<T*>(a.out) + row * a.ld_out;
  advance(a.history, row * a.ld_history);
  for (const int32_t** p : {&a.lengths, &a.prompt, &a.mask_rows}) advance(*p, row);
  for (const float** p : {&a.repetition, &a.presence, &a.frequency}) advance(*p, row);
  advance(a.bias, row * a.ld_bias);
  if (!a.mask_rows && a.masks > 1) {  // a mask for each row
    advance(a.mask, row * a.ld_mask);
    a.masks = rows;
  }
  advance(a.token, row);
  advance(a.lse, row);
  advance(c.head, row * kHeadLine);
  advance(c.words, row * c.stride * 3);
  a.rows = rows;
  return c;
}

// E words to a thread.  A launch has fewer than 2^32 threads: more rows take several.
template <class T>
hipError_t logits_of(const LogitsCall& call, int E, const Launch& L) {
  const bool many = call.a.history && call.a.history_cap > 32767;
  auto k = E == 32   ? (many ? k_logits<T, 32, true> : k_logits<T, 32, false>)
           : E == 16 ? (many ? k_logits<T, 16, true> : k_logits<T, 16, false>)
           : E == 8  ? (many ? k_logits<T, 8, true> : k_logits<T, 8, false>)
                     : (many ? k_logits<T, 4, true> : k_logits<T, 4, false>);
  const int most = (int)(((int64_t)1 << 32) / kBlock - 1) / call.tiles;  // V <= 2^30: at least 16
  for (int64_t row = 0; row < call.a.rows; row += most) {
    const LogitsCall c =
        logits_rows<T>(call, row, (int)std::min<int64_t>(most, call.a.rows - row));
    const hipError_t e = pg_launch(k, dim3(c.a.rows * c.tiles), dim3(kBlock), 0, L, c);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_dropout(const DropoutCall& c, const Launch& L) {
  return by_format(c.a.dtype, [&](auto v) { return dropout_of<decltype(v)>(c, L); });
}

hipError_t launch_logits(LogitsCall c, const Launch& L) {
  // Long parts read the history and the row's rules fewer times; short ones spread a few
  // rows over the chip.  The longest that give every CU two workgroups: 256 rows of
  // 1,000,000 in parts of 2,048 words 456 us, 4,096 328, 8,192 266, 16,384 (fewer
  // workgroups to a CU) 276; 48 rows of 32,003 in parts of 1,024 9.8, 2,048 9.2, 4,096
  // 10.2.
  int E = 32;
  while (E > 4 && (int64_t)c.a.rows * ceil_div(c.a.V, E * kBlock) < 2 * kCus) E /= 2;
  c.tiles = ceil_div(c.a.V, E * kBlock);
  return by_format(c.a.dtype, [&](auto v) { return logits_of<decltype(v)>(c, E, L); });
}

}  // namespace pg
