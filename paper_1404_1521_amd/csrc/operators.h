// Argument blocks and launches of the sequence operators (dropout, gated
// linear recurrence, scores; convolution, selective scan, beams, reordering).
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

// Of sequences of T tokens each, one behind the other: the first that starts at lo or later.
// (No sum of the two: a sequence may have 2^30 tokens, and lo lie past them.)
__host__ __device__ inline int first_equal(int lo, int T) { return T ? lo / T + (lo % T != 0) : 0; }

// Packed sequences of a call.
struct Packed {
  const void* offsets;  // [nseq + 1] of offset_bytes each, or null: tokens / nseq tokens each
  uint32_t* flag;
  int offset_bytes, tokens, nseq;
};

// Pieces dealt out to parts in their order, to the first `more` of them each + 1, to the others `each`.
struct Shares {
  int each, more;
  Shares() = default;
  Shares(int64_t pieces, int64_t parts) : each((int)(pieces / parts)), more((int)(pieces % parts)) {}
  // The first piece of a part, a piece being `size` tokens; `tokens` where there is none.
  __host__ __device__ int first(int64_t part, int size, int tokens) const {
    const int64_t at = (part * each + (part < more ? part : more)) * size;
    return (int)(at < tokens ? at : tokens);
  }
};

// The selective scan and its gradient (the gradient's in the second half).
struct SelCall {
  const void *x, *delta, *B, *C, *z;
  const float *A, *skip, *bias, *h0;
  void* y;
  float *last, *marks;
  const void* dy;
  const float* dlast;
  void *dx, *ddelta, *dB, *dC, *dz;
  float *dA, *dskip, *dbias, *dh0;
  int64_t ld_x, ld_delta, ld_B, ld_C, ld_z, ld_y, ld_dy, ld_dx, ld_ddelta, ld_dB, ld_dC, ld_dz;
  Packed seqs;
  int D, N, groups, softplus;
};

constexpr int kSelectiveTile = 16;  // POLYGLOT_SELECTIVE_MARK
// What a range passes on: nothing (a sequence ends or starts at its end), the state of a
// sequence that starts in it, or its own carry too.
constexpr uint32_t kSelNone = 0, kSelClosed = 1, kSelOpen = 2;
constexpr int kSelGroup = 16;  // ranges
constexpr int kSelNear = 32;   // ranges that are taken in one by one where there are groups

// A kernel's lanes to a channel (four states each), its waves and its channels.
__host__ __device__ constexpr int sel_lanes(int N) { return N <= 8 ? 2 : N <= 16 ? 4 : N <= 32 ? 8 : 16; }
__host__ __device__ constexpr int sel_waves(int lanes) { return lanes == 2 ? 2 : 4; }
__host__ __device__ constexpr int sel_channels(int lanes) { return sel_waves(lanes) * 2 * kWave / lanes; }

// How a selective scan is cut: a workgroup for each range of tokens and block of channels.
struct SelPlan {
  Shares share;            // tiles of a range
  int ranges;
  int blocks, all_blocks;  // of a head's channels, of all
  int NM;                  // places of a mark's row
  float* states;           // [ranges][D][places] what a range passes on
  float* sums;             // [ranges][D] the sum of its steps
  uint32_t* info;          // [ranges]
  int groups;              // of kSelGroup ranges, or 0: states, sums and info of each of them
  float* group_states;     //   lie behind those of the ranges
  float* group_sums;
  uint32_t* group_info;
  float* part_a;           // [ranges][D][places] dA
  float* part_s;           // [ranges][2][D] dskip and the bias's gradient
  float* part_bc;          // [blocks][tokens][groups][2][N] dB and dC
};
struct SelRoom {  // values of each
  size_t states, sums, info, part_s, part_bc;
};
struct SelSpace {
  float *states, *sums, *part_a, *part_s, *part_bc;
  uint32_t* info;
};

// The short causal convolution and its gradient.
struct ConvCall {
  const void *x, *state;
  const float *weight, *bias;
  void *y, *last;
  const void *dy, *dlast;
  void *dx, *dstate;
  float *dweight, *dbias;
  int64_t ld_x, ld_y, ld_dy, ld_dx;
  Packed seqs;
  int D, silu;
  int lanes_log2, blocks;  // lanes of a row of threads; rows of blocks
  int chunk, groups;       // tokens of a row of threads; workgroups for a row of blocks
  float* part;             // [groups][K + 1][D] sums of the weights' and the bias's gradients
};
constexpr int kConvMaxK = 4;
constexpr int kConvStep = 8;           // tokens that a row of threads reads ahead
// Where the tokens give as many.  Half or twice as many are alike: 65,536 x 2,048 bfloat16 in
// 123 to 128 us with each.
constexpr int kConvWorkgroups = 1024;
// Waves to a SIMD of the gradient, whose workgroups are to run all at once.
constexpr int conv_grad_waves(size_t size) { return size == 4 ? 2 : 3; }

struct BeamCall {
  const void* scores;
  const float *total, *lse;
  const int32_t* finished;
  int32_t *parent, *token;
  float* out;
  uint64_t* keys;  // [rows][parts][picks]
  int64_t ld;
  int groups, beams, V, picks, end;
  int parts;  // of a row
};
constexpr int kBeamPicks = 64;   // most
constexpr int kBeamMinPart = 1024;  // words of the shortest part

constexpr int kReorderItems = 32;            // tensors of a launch
constexpr int kReorderPiece = 16 * 4 * kBlock;  // bytes of a workgroup's copy
struct RowCopy {
  const char* in;
  char* out;
  int64_t row_bytes, ld_in, ld_out, pieces;
  int in_rows, unit;  // bytes that every address and length is a multiple of
};
struct ReorderCall {
  RowCopy item[kReorderItems];
  int64_t first[kReorderItems + 1];  // piece of each tensor; all pieces behind the last
  const int32_t* ids;
  uint32_t* flag;
  int rows, count;
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

hipError_t launch_selective(const SelCall& c, int dtype, SelSpace space, const Launch& L);
hipError_t launch_selective_grad(const SelCall& c, int dtype, SelSpace space, const Launch& L);
hipError_t launch_selective_step(const SelCall& c, int dtype, const Launch& L);
// The room that selective scans of up to `tokens` tokens, D channels and N states need.
SelRoom selective_room(int64_t tokens, int D, int N);

hipError_t launch_convolution(ConvCall c, int K, int dtype, const Launch& L);
hipError_t launch_convolution_step(ConvCall c, int K, int dtype, const Launch& L);
hipError_t launch_convolution_grad(ConvCall c, int K, int dtype, const Launch& L);
// Floats of ConvCall::part for gradients of up to D channels.
size_t convolution_room(int D);
hipError_t launch_beam(BeamCall c, int dtype, const Launch& L);
hipError_t launch_reorder(const ReorderCall& c, const Launch& L);

}  // namespace pg
