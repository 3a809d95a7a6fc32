// Argument blocks and launches of the sequence operators (dropout, gated
// linear recurrence, scores).
#pragma once
#include "polyglot.h"

#include "common.h"
#include "launch.h"

namespace pg {

struct DropoutCall {
  polyglot_dropout_args a;
  uint32_t* flag;
  uint32_t threshold;  // an element is dropped where its 16 bits are below
  float scale;         // 65536 / (65536 - threshold); 0 where everything is dropped
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

struct LogitsCall {
  polyglot_logits_args a;
  uint32_t* flag;
};

hipError_t launch_dropout(const DropoutCall& c, const Launch& L);
hipError_t launch_recurrence(const RecCall& c, int dtype, int form, bool grad, const Launch& L);
hipError_t launch_logits(const LogitsCall& c, const Launch& L);

}  // namespace pg
