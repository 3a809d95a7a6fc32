// Argument blocks and launches of the sequence operators (dropout, gated
// linear recurrence, scores).
#pragma once
#include "polyglot.h"

#include "common.h"
#include "formats.h"
#include "launch.h"

namespace pg {

// Words that many workgroups count in lie this many 64-bit words apart: 128 bytes,
// a cache line.  Atomics on one line take turns, at 10 to 17 ns each.
constexpr int64_t kHeadLine = 16;

struct DropoutCall {
  polyglot_dropout_args a;
  uint32_t* flag;
  uint32_t threshold;  // an element is dropped where its 16 bits are below
  float scale;         // 65536 / (65536 - threshold); 0 where everything is dropped
  int groups;          // of eight columns, in a row
  uint32_t groups_inv; // ceil(2^32 / groups)
};

// The recurrence and its gradient are one scan, s = c s + b, in one of the two
// directions: over the state h with c = a and b = x or (1 - a) x, or, against
// the reading direction, over mu with c = a and b = a dh.
struct RecCall {
  const void* gate;
  const void* x;
  const void* h;       // gradient only
  const void* dh;      // gradient only
  const float* h0;     // the state before a sequence's first token (gradient: h_{t-1} there)
  const float* init;   // the scan's state before the first token that it meets: h0, or dlast
  const void* offsets;
  void* out;           // h, or dx
  void* dgate;         // gradient only
  float* fin;          // the scan's state after a sequence: last, or dh0
  uint32_t* flag;
  int64_t ld_gate, ld_x, ld_h, ld_dh, ld_out, ld_dgate;
  int tokens, nseq, D, group, offset_bytes;
  int down;            // 1: the scan goes from a sequence's last token to its first
};

// How a scan is cut (ScanLds has the rest).
struct ScanPlan {
  int lanes_log2;        // lanes of a row of threads: four channels each
  int tiles, chunks;     // of the channels and of the tokens; a workgroup for each pair
  int lanes_per_group, groups_per_tile;  // shared gates
  int counters;
  uint64_t* head;        // [counters >= tiles][kHeadLine] tag << 32 | next chunk; null: no chunk waits
  int group_log2;        // chunks of a group
  uint64_t* flags;       // [tiles][chunks + groups]
  uint64_t* words;       // [tiles] of [chunks][2][4][lanes], [groups][3][4][lanes]
};

// What a context keeps for its scans: the counters (tag 1 at first), then the flags
// and words (zeros at first).
struct ScanSpace {
  uint64_t* head = nullptr;
  int counters = 0;
  size_t flags = 0, words = 0;
};

struct LogitsCall {
  polyglot_logits_args a;
  uint32_t* flag;
  int tiles;             // parts of a row, a workgroup each
  uint64_t* head;        // [rows][kHeadLine] tag << 32 | parts done; null: neither token nor lse
  uint64_t* words;       // [rows][stride][3] of a part: largest score, its word, sum of exponentials
  int64_t stride;        // parts that a row has room for
};

// Calls f with a value of the storage type `dtype` (POLYGLOT_F32, _BF16, _F16).
template <class F>
hipError_t by_format(int dtype, F f) {
  if (dtype == POLYGLOT_F32) return f(float{});
  if (dtype == POLYGLOT_BF16) return f(BF16{});
  return f(F16{});
}

hipError_t launch_dropout(const DropoutCall& c, const Launch& L);
// `space` matters only to calls of other than one token per sequence.
hipError_t launch_recurrence(const RecCall& c, int dtype, int form, bool grad,
                             const ScanSpace& space, const Launch& L);
// The room that scans of up to `tokens` tokens and D channels need (head stays null).
ScanSpace scan_space(int64_t tokens, int D);
hipError_t launch_logits(LogitsCall c, const Launch& L);
constexpr int kLogitsMinTile = 1024;  // words of the shortest part

}  // namespace pg
