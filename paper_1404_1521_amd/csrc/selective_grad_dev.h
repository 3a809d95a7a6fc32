// The gradient of the selective scan.  With v' the gradient of v and mu what comes back
// from the token after (dlast after a sequence's last one):
//   lambda = v' C + mu,  mu <- a lambda,  q = a lambda h_{t-1}
//   dC = sum_c v' h, dB = sum_c lambda D x, dA = sum_t D q
//   d(D) = sum_n q A + x e,  dx = D e + skip v',  e = sum_n lambda B
//
// The ranges are those of the forward pass, taken from their ends.  A tile starts from the
// mark that the forward pass left, the states before its first token, goes through its 16
// tokens in two halves, each once forward, with decays and states kept in registers, and
// once back.  The sums over the states go over LN lanes by DPP moves; those over the
// channels over the other lanes, two values at a time by half-wave and row swaps, then over
// the waves in LDS and over the workgroups in a last launch, always in the same order.
//
// What bounds it are vector instructions, as in the forward pass: a state and token take 48
// cycles on the way back, 20 for the states again and 10 for those of a first half that are
// needed to reach the second, and about 15 for the sums over lanes.  At 32,768 x 2,048
// bfloat16 with 16 states and a gate: 252 us for what comes back, 1,037 for the tiles (462 M
// vector instructions, 0.84 of the cycles by the counters), and 22 for the sums; its bytes are
// 234.  Halves of eight tokens, because the states of eight are 64 registers and those of 16,
// 128, beside what the way back needs.
#pragma once
#include "selective_dev.h"

namespace pg {

// Eight values of each lane summed over the 64 / LN lanes of the same states: lane l keeps
// value 4 (l / 32) + 2 (l / 16 % 2) + {0, 1}.
template <int LN>
__device__ __forceinline__ void sum_channels(const float (&v)[8], float (&out)[2]) {
  float u[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[i]), __float_as_uint(v[i + 4]),
                                                    false, false);
    u[i] = __uint_as_float(s[0]) + __uint_as_float(s[1]);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(u[i]), __float_as_uint(u[i + 2]),
                                                    false, false);
    out[i] = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    if constexpr (LN <= 8) out[i] += lane_moved<0x128>(out[i]);  // row_ror:8
    if constexpr (LN <= 4) out[i] += lane_moved<0x124>(out[i]);  // row_ror:4
    if constexpr (LN <= 2) out[i] += lane_moved<0x122>(out[i]);  // row_ror:2
    here(out[i]);
  }
}

// A tile of the gradient's inputs on its way to a thread.
template <class T, int LN>
struct GradTile {
  using S = SelShape<LN>;
  QuadTile<T, S> raw, gy, xv, zv;
  StateTile<T, LN> states;
  // Without X, of what the first launch reads: neither x nor B.
  template <bool X>
  __device__ __forceinline__ void load(const SelCall& c, const SelPlace<LN>& w, int t0, int count) {
    const T* none = nullptr;
    const bool whole = whole_tile<S>(w, count);
    raw.load(c.delta, c.ld_delta, RowSpot::of(none, c.ld_delta, w.k0, w.q0), t0, count, whole, w);
    gy.load(c.dy, c.ld_dy, RowSpot::of(none, c.ld_dy, w.k0, w.q0), t0, count, whole, w);
    if (X) xv.load(c.x, c.ld_x, RowSpot::of(none, c.ld_x, w.k0, w.q0), t0, count, whole, w);
    if (c.z) zv.load(c.z, c.ld_z, RowSpot::of(none, c.ld_z, w.k0, w.q0), t0, count, whole, w);
    states.load(X ? c.B : nullptr, c.ld_B, c.C, c.ld_C, t0, count, w.head, c.N);
  }
  // The tile's steps, D x and v' to LDS.  Tokens past the tile's and channels past the
  // workgroup's: zeros, which change nothing.  KEEP: the softplus' slopes and the gate's
  // sigmoid, too.
  template <bool X, bool KEEP = false>
  __device__ __forceinline__ void put(const SelCall& c, const SelPlace<LN>& w, int count, float* step,
                                      float* dx, float* dv, float* slope = nullptr, float* gate = nullptr) const {
    float bias[4], d[S::EACH][4];
    load_four(c.bias, w.q0, w.qn, bias);
    tile_steps<T, LN, KEEP>(raw, bias, c.softplus, w, count, whole_tile<S>(w, count), d, slope);
    const bool gated = c.z != nullptr;
#pragma unroll
    for (int e = 0; e < S::EACH; ++e) {
      const int at = quad_place<S>(e);
      if (at < 0) continue;
      f4 u, v;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (X) u[j] = d[e][j] * xv.q[e].get(j);
        v[j] = gy.q[e].get(j);
      }
      if (gated) {
        f4 sg;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          sg[j] = sigmoid(zv.q[e].get(j));
          v[j] *= zv.q[e].get(j) * sg[j];
        }
        if (KEEP) st4(gate + at, sg);
      }
      st4(step + at, f4{d[e][0], d[e][1], d[e][2], d[e][3]});
      if (X) st4(dx + at, u);
      st4(dv + at, v);
    }
  }
};

// What comes back through each range that a sequence runs into, from that sequence's end in
// it or from nothing.
template <class T, int LN>
__global__ __launch_bounds__(SelShape<LN>::THREADS) void k_selective_grad_ends(SelArgs) {
  using S = SelShape<LN>;
  __shared__ SelLds<LN> s;
  const SelArgsPtr args = sel_args();
  const SelArgs& first = again(args);
  const int t = threadIdx.x;
  const int range = blockIdx.x / first.p.all_blocks, block = blockIdx.x % first.p.all_blocks;
  const SelPlace<LN> w(first.c, first.p, block);
  const int lo = first.p.share.first(range, kSelTile, first.c.seqs.tokens);
  const int hi = first.p.share.first(range + 1, kSelTile, first.c.seqs.tokens);
  const RangeEnd end = range_start(first.c.seqs, lo, hi);
  const int to = end.at, seq = end.seq;
  if (t == 0 && block == 0) first.p.info[range] = end.kind;
  if (end.kind == kSelNone) return;

  int tile = (to - 1 - lo) / kSelTile;
  GradTile<T, LN> in;
  in.template load<false>(first.c, w, lo + tile * kSelTile, min(kSelTile, to - lo - tile * kSelTile));
  float A[2][4], mu[2][4], sum[2] = {0.f, 0.f};
  load_rates(first.c, w, A);
#pragma unroll
  for (int r = 0; r < 2; ++r)
    load_states(seq >= 0 ? state_row(first.c.dlast, seq, first.c) : nullptr, w, r, first.c.N, mu[r]);
  for (; tile >= 0; --tile) {
    const int t0 = lo + tile * kSelTile;
    const SelCall& c = again(args).c;
    __syncthreads();
    in.template put<false>(c, w, min(kSelTile, to - t0), s.step, nullptr, s.dx);
    in.states.put(s.B, s.C);
    if (tile > 0) in.template load<false>(c, w, t0 - kSelTile, kSelTile);
    __syncthreads();
#pragma unroll 4
    for (int k = kSelTile - 1; k >= 0; --k) {
      const float2 d = *reinterpret_cast<const float2*>(s.step + k * S::CB + w.lane_c);
      const float2 g = *reinterpret_cast<const float2*>(s.dx + k * S::CB + w.lane_c);
      const f4 C = ld4(s.C + k * S::NP + 4 * w.nl);
      const float dd[2] = {d.x, d.y}, gg[2] = {g.x, g.y};
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        sum[r] += dd[r];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          mu[r][j] = exp2_fast(dd[r] * A[r][j]) * __fmaf_rn(gg[r], C[j], mu[r][j]);
      }
    }
  }
  const SelArgs& last = again(args);
  pass_on(last.c, last.p, range, w, mu, sum);
}

// LDS of the gradient: what comes in and goes out of each token and channel (D x makes
// room for e, v' for v), the tile's B and C, the waves' sums for dB and dC.
template <int LN>
struct alignas(16) SelGradLds {
  using S = SelShape<LN>;
  SelLds<LN> in;
  float dv[kSelTile * S::CB], dstep[kSelTile * S::CB];
  float part[S::W][kSelTile][2][S::NP];
  // The softplus' slopes and the gate's sigmoid, kept by the thread that reads them: 20
  // operations less for a token and channel, 32,768 x 2,048 of 16 states 1,350 -> 1,312 us,
  // 16,384 x 1,024 of 32 states 663 -> 652; but of 64, where a token and channel weigh little,
  // 1,315 -> 1,354, and with up to 8 states a CU has no room for all of its workgroups.
  static constexpr bool KEEP = LN == 4 || LN == 8;
  float slope[KEEP ? kSelTile * S::CB : 1], gate[KEEP ? kSelTile * S::CB : 1];
  int list[S::THREADS + 1];
};

// Two waves to a SIMD: 250 registers hold the half tile's states, decays computed twice.  Loads
// of the next tile kept through a tile do not fit beside them (all three launches 6% longer,
// with registers spilled).
template <class T, int LN>
__global__ __launch_bounds__(SelShape<LN>::THREADS, 2) void k_selective_grad(SelArgs) {
  using S = SelShape<LN>;
  constexpr int H = kSelTile / 2;
  __shared__ SelGradLds<LN> g;
  SelLds<LN>& s = g.in;
  const SelArgsPtr args = sel_args();
  const SelArgs& first = again(args);
  const int t = threadIdx.x, lane = t & (kWave - 1), wave = t / kWave;
  const int range = blockIdx.x / first.p.all_blocks, block = blockIdx.x % first.p.all_blocks;
  const SelPlace<LN> w(first.c, first.p, block);
  const int lo = first.p.share.first(range, kSelTile, first.c.seqs.tokens);
  const int hi = first.p.share.first(range + 1, kSelTile, first.c.seqs.tokens);

  check_places(first.c.seqs, range, first.p.ranges, S::THREADS, first.c.dh0 != nullptr, g.list, [&](int i) {
    const SelCall& c = again(args).c;
    for (int r = 0; r < 2; ++r) {
      float v[4];
      load_states(state_row(c.dlast, i, c), w, r, c.N, v);
      store_states(state_row(c.dh0, i, c), w, r, c.N, v);
    }
  });

  float A[2][4], dA[2][4], mu[2][4];
  load_rates(first.c, w, A);
#pragma unroll
  for (int r = 0; r < 2; ++r)
#pragma unroll
    for (int j = 0; j < 4; ++j) dA[r][j] = mu[r][j] = 0.f;
  float dskip[4] = {0.f, 0.f, 0.f, 0.f}, dbias[4] = {0.f, 0.f, 0.f, 0.f};
  const bool gated = first.c.z != nullptr;
  const int tiles = lo < hi ? ceil_div(hi - lo, kSelTile) : 0;
  DownCursor cursor{};
  if (tiles > 0) {
    const SelArgs& a = again(args);
    const int next = first_place(a.c.seqs, hi);
    if (t < kWave) cursor.read(a.c.seqs, first_place(a.c.seqs, hi + 1));
    // unless a sequence ends here
    if (hi < a.c.seqs.tokens && !(next <= a.c.seqs.nseq && place_of(a.c.seqs, next) == hi))
      carry_into<LN>(a.c, a.p, range, -1, w, A, mu);
  }

  for (int tile = tiles - 1; tile >= 0; --tile) {
    const int t0 = lo + tile * kSelTile, count = min(kSelTile, hi - t0);
    {
      const SelCall& c = again(args).c;
      GradTile<T, LN> in;
      in.template load<true>(c, w, t0, count);
      in.template put<true, SelGradLds<LN>::KEEP>(c, w, count, s.step, s.dx, g.dv, g.slope, g.gate);
      in.states.put(s.B, s.C);
      if (t < kWave) mark_tile(c.seqs, t0, t0 + count, cursor, s.marks);
    }
    __syncthreads();
    const uint32_t starts = __builtin_amdgcn_readfirstlane(s.marks.starts);
    const uint32_t stops = __builtin_amdgcn_readfirstlane(s.marks.stops);
    // the states before the first half, and before the second one
    float first_h[2][4], h[2][4];
    {
      const SelArgs& a = again(args);
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        f4 m = kZero4;
        if (w.has(r) && 4 * w.nl < a.c.N)
          m = ld4(a.c.marks + ((int64_t)(t0 / kSelTile) * a.c.D + w.c0 + w.lane_c + r) * a.p.NM + 4 * w.nl);
#pragma unroll
        for (int j = 0; j < 4; ++j) first_h[r][j] = h[r][j] = m[j];
      }
    }
    const auto halves = [&](auto is_plain) {
      constexpr bool PLAIN = decltype(is_plain)::value;  // no sequence starts or stops here
      // The states of the sequence that starts or stops at token k, of one of the tensors.
      const auto states_at = [&](const int* places, int k, const float* SelCall::* of, float (&v)[2][4]) {
        const SelCall& c = again(args).c;
        const float* row = state_row(c.*of, __builtin_amdgcn_readfirstlane(places[k]), c);
#pragma unroll
        for (int r = 0; r < 2; ++r) load_states(row, w, r, c.N, v[r]);
      };
      // What a token brings, on its way from LDS while the token before is worked on.
      struct Token {
        float2 d, u, dv;
        f4 B, C;
      };
      const auto fetch = [&](int k, bool back) {
        Token o;
        o.d = *reinterpret_cast<const float2*>(s.step + k * S::CB + w.lane_c);
        o.u = *reinterpret_cast<const float2*>(s.dx + k * S::CB + w.lane_c);
        o.B = ld4(s.B + k * S::NP + 4 * w.nl);
        if (back) {
          o.dv = *reinterpret_cast<const float2*>(g.dv + k * S::CB + w.lane_c);
          o.C = ld4(s.C + k * S::NP + 4 * w.nl);
        }
        return o;
      };
      const auto forward = [&](int k, const Token& o) {
        if (!PLAIN && (starts >> k & 1)) states_at(s.marks.start, k, &SelCall::h0, h);
        const float dd[2] = {o.d.x, o.d.y}, uu[2] = {o.u.x, o.u.y};
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            h[r][j] = __fmaf_rn(exp2_fast(dd[r] * A[r][j]), h[r][j], uu[r] * o.B[j]);
      };
      const bool second = count > H;
      if (second) {
        Token now = fetch(0, false);
#pragma unroll 2
        for (int k = 0; k < H; ++k) {
          const Token next = fetch(k + 1, false);
          forward(k, now);
          __builtin_amdgcn_sched_barrier(0);
          now = next;
        }
      }
      for (int half = second; half >= 0; --half) {
        const int base = half * H;
        float before[2][4], hs[H][2][4];
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
          for (int j = 0; j < 4; ++j) before[r][j] = h[r][j] = half ? h[r][j] : first_h[r][j];
        Token now = fetch(base, false);
#pragma unroll
        for (int i = 0; i < H; ++i) {
          const Token next = fetch(base + min(i + 1, H - 1), i == H - 1);
          forward(base + i, now);
#pragma unroll
          for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int j = 0; j < 4; ++j) hs[i][r][j] = h[r][j];
          __builtin_amdgcn_sched_barrier(0);
          now = next;
        }
#pragma unroll
        for (int i = H - 1; i >= 0; --i) {
          const int k = base + i;
          const Token next = fetch(base + max(i - 1, 0), true);
          if (!PLAIN && (stops >> k & 1)) states_at(s.marks.stop, k, &SelCall::dlast, mu);
          const bool starts_here = !PLAIN && (starts >> k & 1);
          float hp[2][4];
#pragma unroll
          for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int j = 0; j < 4; ++j) hp[r][j] = i ? hs[i ? i - 1 : 0][r][j] : before[r][j];
          if (starts_here) states_at(s.marks.start, k, &SelCall::h0, hp);
          // (here: the decays are computed again, not kept from the way forward)
          here(now.d.x), here(now.d.y);
          const float dd[2] = {now.d.x, now.d.y}, uu[2] = {now.u.x, now.u.y};
          const float vv[2] = {now.dv.x, now.dv.y};
          const f4 B = now.B, C = now.C;
          float both[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};  // dB, dC
          float e[2], ds[2], v[2];
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            e[r] = ds[r] = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float lam = __fmaf_rn(vv[r], C[j], mu[r][j]);
              both[j] = __fmaf_rn(lam, uu[r], both[j]);
              both[4 + j] = __fmaf_rn(vv[r], hs[i][r][j], both[4 + j]);
              e[r] = __fmaf_rn(lam, B[j], e[r]);
              mu[r][j] = lam * exp2_fast(dd[r] * A[r][j]);
              const float q = mu[r][j] * hp[r][j];
              ds[r] = __fmaf_rn(q, A[r][j], ds[r]);
              dA[r][j] = __fmaf_rn(q, dd[r], dA[r][j]);
              here(dA[r][j]);
            }
            e[r] = sum_states<LN>(e[r]);
            ds[r] = sum_states<LN>(ds[r]);
          }
          if (gated) {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              v[r] = 0.f;
#pragma unroll
              for (int j = 0; j < 4; ++j) v[r] = __fmaf_rn(C[j], hs[i][r][j], v[r]);
              v[r] = sum_states<LN>(v[r]);
            }
            if (w.nl == 0)
              *reinterpret_cast<float2*>(g.dv + k * S::CB + w.lane_c) = float2{v[0], v[1]};
          }
          if (w.nl == 0) {
            *reinterpret_cast<float2*>(s.dx + k * S::CB + w.lane_c) = float2{e[0], e[1]};
            *reinterpret_cast<float2*>(g.dstep + k * S::CB + w.lane_c) = float2{ds[0], ds[1]};
          }
          float pair[2];
          sum_channels<LN>(both, pair);
          if (lane % 16 < LN)
            *reinterpret_cast<float2*>(&g.part[wave][k][lane / 32][4 * w.nl + 2 * (lane / 16 % 2)]) =
                float2{pair[0], pair[1]};
          if (starts_here) {
            const SelCall& c = again(args).c;
            float* row = state_row(c.dh0, __builtin_amdgcn_readfirstlane(s.marks.start[k]), c);
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              store_states(row, w, r, c.N, mu[r]);
#pragma unroll
              for (int j = 0; j < 4; ++j) mu[r][j] = 0.f;
            }
          }
          __builtin_amdgcn_sched_barrier(0);
          now = next;
        }
      }
    };
    if ((starts | stops) == 0) halves(std::true_type{});
    else halves(std::false_type{});
    __syncthreads();

    const SelArgs& a = again(args);
    const SelCall& c = a.c;
    const bool whole = whole_tile<S>(w, count), skips = c.skip != nullptr;
    const bool soft = c.softplus;
    constexpr bool KEEP = SelGradLds<LN>::KEEP;
    const T* none = nullptr;
    QuadTile<T, S> raw, gy, xv, zv;
    gy.load(c.dy, c.ld_dy, RowSpot::of(none, c.ld_dy, w.k0, w.q0), t0, count, whole, w);
    xv.load(c.x, c.ld_x, RowSpot::of(none, c.ld_x, w.k0, w.q0), t0, count, whole, w);
    if (gated) zv.load(c.z, c.ld_z, RowSpot::of(none, c.ld_z, w.k0, w.q0), t0, count, whole, w);
    if (soft && !KEEP) raw.load(c.delta, c.ld_delta, RowSpot::of(none, c.ld_delta, w.k0, w.q0), t0, count, whole, w);
    float bias[4], skip[4];
    load_four(c.bias, w.q0, w.qn, bias);
    load_four(c.skip, w.q0, w.qn, skip);
#pragma unroll
    for (int el = 0; el < S::EACH; ++el) {
      const int at = quad_place<S>(el);
      if (at < 0 || (!whole && (w.k0 + el * S::STEP >= count || w.qn == 0))) continue;
      const f4 e = ld4(s.dx + at), st = ld4(s.step + at), ds = ld4(g.dstep + at);
      const int64_t row = t0 + el * S::STEP;
      const auto put = [&](void* base, int64_t ld, const float (&v)[4]) {
        T* to = static_cast<T*>(base);
        put_quad(RowSpot::of(to, ld, w.k0, w.q0).at(to, ld, row), v, w.qn);
      };
      float gv[4], out[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) gv[j] = gy.q[el].get(j);
      if (gated) {
        const f4 sv = ld4(g.dv + at);
        f4 kept;
        if (KEEP) kept = ld4(g.gate + at);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float zj = zv.q[el].get(j), sg = KEEP ? kept[j] : sigmoid(zj);
          const float v = __fmaf_rn(skip[j], skips ? xv.q[el].get(j) : 0.f, sv[j]);
          out[j] = gv[j] * v * (sg * __fmaf_rn(zj, 1.f - sg, 1.f));
          gv[j] *= zj * sg;
        }
        put(c.dz, c.ld_dz, out);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) out[j] = st[j] * e[j];
      if (skips) {
#pragma unroll
        for (int j = 0; j < 4; ++j) out[j] = __fmaf_rn(skip[j], gv[j], out[j]);
      }
      put(c.dx, c.ld_dx, out);
#pragma unroll
      for (int j = 0; j < 4; ++j) dskip[j] = __fmaf_rn(gv[j], xv.q[el].get(j), dskip[j]);
#pragma unroll
      for (int j = 0; j < 4; ++j) out[j] = __fmaf_rn(xv.q[el].get(j), e[j], kLn2 * ds[j]);
      if (soft) {
        f4 kept;
        if (KEEP) kept = ld4(g.slope + at);
#pragma unroll
        for (int j = 0; j < 4; ++j) out[j] *= KEEP ? kept[j] : sigmoid(raw.q[el].get(j) + bias[j]);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) dbias[j] += out[j];
      put(c.ddelta, c.ld_ddelta, out);
    }
    for (int i = t; i < count * 2 * S::NP; i += S::THREADS) {
      const int k = i / (2 * S::NP), which = i / S::NP % 2, n = i % S::NP;
      if (n >= c.N) continue;
      float v = g.part[0][k][which][n];
#pragma unroll
      for (int j = 1; j < S::W; ++j) v += g.part[j][k][which][n];
      const int64_t row = t0 + (int64_t)k;
      if (a.p.blocks == 1) {
        T* to = which ? static_cast<T*>(c.dC) + row * c.ld_dC : static_cast<T*>(c.dB) + row * c.ld_dB;
        to[(int64_t)w.head * c.N + n] = Elem<T>::put(settled(v));
      } else {
        const int64_t place = (((int64_t)(block % a.p.blocks) * c.seqs.tokens + row) * c.groups + w.head) * 2;
        a.p.part_bc[(place + which) * c.N + n] = v;
      }
    }
  }

  const SelArgs& a = again(args);
#pragma unroll
  for (int r = 0; r < 2; ++r)
    if (w.has(r))
      st4(a.p.part_a + ((int64_t)range * a.c.D + w.c0 + w.lane_c + r) * S::NP + 4 * w.nl,
          f4{dA[r][0], dA[r][1], dA[r][2], dA[r][3]});
  // the threads of a quad of channels, in order
  __syncthreads();
  constexpr int kBusy = kSelTile * S::QUADS < S::THREADS ? kSelTile * S::QUADS : S::THREADS;
  if (t < kBusy) {
    st4(s.step + t * 4, f4{dskip[0], dskip[1], dskip[2], dskip[3]});
    st4(s.dx + t * 4, f4{dbias[0], dbias[1], dbias[2], dbias[3]});
  }
  __syncthreads();
  for (int i = t; i < w.nc; i += S::THREADS) {
    float u = 0.f, v = 0.f;
    for (int j = 0; j < kBusy / S::QUADS; ++j) {
      u += s.step[j * S::CB + i];
      v += s.dx[j * S::CB + i];
    }
    a.p.part_s[((int64_t)range * 2) * a.c.D + w.c0 + i] = u;
    a.p.part_s[((int64_t)range * 2 + 1) * a.c.D + w.c0 + i] = v;
  }
}

// The sums over the ranges (dA, dskip, the bias's) and over the workgroups of a head's
// channels (dB, dC).
template <class T>
__global__ __launch_bounds__(kBlock) void k_selective_sums(SelCall c, SelPlan p, int NP, int param_blocks) {
  const int t = threadIdx.x;
  if ((int)blockIdx.x < param_blocks) {
    const int64_t o = (int64_t)blockIdx.x * kSumOutputs + t % kSumOutputs, n_a = (int64_t)c.D * c.N;
    const float* from = nullptr;
    int64_t ld = 0;
    float* to = nullptr;
    if (o < n_a) {
      from = p.part_a + o / c.N * NP + o % c.N;
      ld = (int64_t)c.D * NP;
      to = c.dA + o;
    } else if (o < n_a + 2 * (int64_t)c.D) {
      const int64_t i = o - n_a;
      from = p.part_s + i;
      ld = 2 * (int64_t)c.D;
      if (i < c.D) to = c.dskip ? c.dskip + i : nullptr;
      else to = c.dbias ? c.dbias + i - c.D : nullptr;
    }
    const float v = sum_parts(from, ld, p.ranges, to != nullptr);
    if (t < kSumOutputs && to) *to = v;
    return;
  }
  const int64_t width = (int64_t)c.groups * 2 * c.N, all = width * c.seqs.tokens;
  for (int64_t i = ((int64_t)blockIdx.x - param_blocks) * kBlock + t; i < all;
       i += (int64_t)(gridDim.x - param_blocks) * kBlock) {
    float v = 0.f;
#pragma unroll 8
    for (int b = 0; b < p.blocks; ++b) v += p.part_bc[b * all + i];
    const int64_t row = i / width;
    const int rest = (int)(i % width), head = rest / (2 * c.N), which = rest / c.N % 2, n = rest % c.N;
    T* to = which ? static_cast<T*>(c.dC) + row * c.ld_dC : static_cast<T*>(c.dB) + row * c.ld_dB;
    to[(int64_t)head * c.N + n] = Elem<T>::put(settled(v));
  }
}

}  // namespace pg
