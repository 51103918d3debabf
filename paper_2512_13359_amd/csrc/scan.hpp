// The gated linear recurrence over a rollout's steps: what its forward and backward kernels
// share (layout of the columns, masks, the composition of step ranges) and their launch shapes.
//
// A column is one (sequence, channel); a range of its steps maps the state before it to the state
// after it by s' = P s + S.  Ranges compose associatively, so a workgroup's W waves take U steps
// each of the same 64 V columns, exchange (P, S) through LDS and redo their steps from the true
// state with the inputs still in registers: every element is read once.  Where the columns are too few
// to fill the chip the steps are split over K workgroups as well, whose (P, S) a first launch
// leaves in the caller's workspace.
//
// P = 0 stands for a cut (an episode's end) and nothing else: what was before a cut must not reach
// what is after it, be it NaN or infinite.  A product that underflows keeps the smallest denormal.  P is kept finite: a
// cut stays one beside any gates, and a state of zero gives S, in which gates that are not finite show as NaN.
#pragma once

#include "auv_internal.hpp"
#include "layers.hpp"

namespace auv {

struct SeqTensor {
  char* p;
  int64_t so, si, st;   // strides of the outer, inner and time axes, elements
};
struct SeqState {
  float* p;
  int64_t sn, sc;
};

struct ScanArgs {
  SeqTensor gate, x, h, dout, dgate, dx;
  SeqState h0, last;     // backward: last is the gradient of the last state, dh0 the result
  SeqState dh0;
  const float* done;     // [T][n] or null
  const int32_t* lens;   // [n] or null
  float* agg;            // [K][tiles][V][2][64]
  float* before;         // the same of the forward pass, for a gradient that forms the states again
  float* marks;          // the state before each round, [K][rounds][tiles][V][64]; null: in LDS
  int T, n, c;
  int Li, Lo;            // columns as [Lo][Li]; Li is the axis of unit stride
  int nvec;              // vectors per row of Li
  int chunk;             // steps per workgroup, a multiple of W U (of U in the first launch)
  int K, tiles;
  bool grouped;   // neighbouring tiles on one XCD
  bool shared;    // plain stores
};

__device__ __forceinline__ float smallest() { return __uint_as_float(1u); }

// NaN and infinities as the largest numbers
__device__ __forceinline__ float finite(float P) { return fminf(fmaxf(P, -3.402823466e38f), 3.402823466e38f); }

// P2 P1 where zero stands for a cut only
__device__ __forceinline__ float chain(float P2, float P1) {
  const float p = finite(P2 * P1);
  return p == 0.0f && P2 != 0.0f && P1 != 0.0f ? smallest() : p;
}
__device__ __forceinline__ float after(float P, float S, float s) { return P == 0.0f ? S : __builtin_fmaf(P, s, S); }

// A workgroup's tile of columns and chunk of steps.  Where rows do not start at a cache line, neighbouring tiles go to one
// XCD (workgroups are dealt out to the eight in turn), so that the parts of a line that two tiles share meet in one L2:
// 4095 x 23 fp32 columns x 500 steps, forward and backward 382 -> 358 us.  Aligned rows share none (16384 x 64 bf16 columns x
// 64 steps, forward 75 us, grouped 73), and chunks of steps run faster dealt out (2 x 256 x 32768, forward and backward 111, grouped 120).
struct Place {
  int tile, chunk;
  __device__ __forceinline__ explicit Place(const ScanArgs& a) {
    uint32_t q = blockIdx.x;
    if (a.grouped) {
      const uint32_t all = gridDim.x, x = q & 7u;
      q = x * (all >> 3) + min(x, all & 7u) + (q >> 3);
    }
    chunk = (int)(q / (uint32_t)a.tiles);
    tile = (int)(q - (uint32_t)chunk * a.tiles);
  }
};

// One lane's V columns.  NI: the inner axis is the sequence (one environment per column);
// else it is the channel, rows of several sequences in one where they lie end to end.
template <int V, bool NI> struct Columns {
  bool active;
  int o, ib, shift;    // row, first column loaded, columns of it that belong to the neighbour
  int na, kb;          // NI false: sequence of column ib; columns k >= kb belong to the next one

  __device__ __forceinline__ Columns(const ScanArgs& a, int tile, int lane) {
    const int64_t id = (int64_t)tile * 64 + lane, all = (int64_t)a.Lo * a.nvec;
    active = id < all;
    const int64_t q = active ? id : all - 1;
    o = (int)(q / a.nvec);
    const int i0 = (int)(q - (int64_t)o * a.nvec) * V;
    ib = min(i0, a.Li - V);
    shift = i0 - ib;
    if (NI) {
      na = ib;
      kb = V;
    } else {
      na = o + ib / a.c;
      kb = a.c - ib % a.c;
    }
  }
  __device__ __forceinline__ int seq(int k) const { return NI ? ib + k : na + (k >= kb); }
  __device__ __forceinline__ int64_t state_at(const ScanArgs& a, const SeqState& s, int k) const {
    const int ch = NI ? o : ib % a.c + k - (k >= kb ? a.c : 0);
    return seq(k) * s.sn + ch * s.sc;
  }
  __device__ __forceinline__ int64_t at(const SeqTensor& t) const { return o * t.so + ib * t.si; }
  template <class T> __device__ __forceinline__ T* base(const SeqTensor& t) const {
    return reinterpret_cast<T*>(t.p) + at(t);
  }

  // Bits of the columns whose episode ended at a step, of those whose sequence is over by it.
  // Flags and lengths are loaded apart from their use (Flags below).
  static constexpr int NF = NI ? V : (V > 1 ? 2 : 1);
  struct Flags { float f[NF]; };
  __device__ __forceinline__ Flags load_done(const ScanArgs& a, int t) const {
    Flags r;
    const float* p = a.done + (int64_t)t * a.n;
    if constexpr (NI) {
#pragma unroll
      for (int k = 0; k < V; ++k) r.f[k] = p[ib + k];
    } else {
      r.f[0] = p[na];
      if constexpr (V > 1) r.f[1] = p[min(na + 1, a.n - 1)];
    }
    return r;
  }
  __device__ __forceinline__ uint32_t bits(const bool* b) const {
    if constexpr (NI) {
      uint32_t m = 0;
#pragma unroll
      for (int k = 0; k < V; ++k) m |= (uint32_t)b[k] << k;
      return m;
    } else if constexpr (V == 1) {
      return b[0];
    } else {
      const uint32_t lo = kb >= V ? (1u << V) - 1u : (1u << kb) - 1u;
      return (b[0] ? lo : 0u) | (b[1] ? ((1u << V) - 1u) & ~lo : 0u);
    }
  }
  __device__ __forceinline__ uint32_t ended(const Flags& d) const {
    bool b[NF];
#pragma unroll
    for (int k = 0; k < NF; ++k) b[k] = d.f[k] != 0.0f;
    return bits(b);
  }
  struct Lens { int v[NF], soonest; };   // soonest: no column of the wave is over before it
  __device__ __forceinline__ Lens load_lens(const ScanArgs& a) const {
    Lens r;
    r.soonest = a.T;
#pragma unroll
    for (int k = 0; k < NF; ++k) {
      r.v[k] = a.lens ? a.lens[NI ? ib + k : min(na + k, a.n - 1)] : a.T;
      r.soonest = min(r.soonest, r.v[k]);
    }
    if (a.lens)
      for (int d = 1; d < 64; d <<= 1) r.soonest = min(r.soonest, __shfl_xor(r.soonest, d));
    r.soonest = __builtin_amdgcn_readfirstlane(r.soonest);
    return r;
  }
  __device__ __forceinline__ uint32_t over(const Lens& l, int t) const {
    if (t < l.soonest) return 0;
    bool b[NF];
#pragma unroll
    for (int k = 0; k < NF; ++k) b[k] = t >= l.v[k];
    return bits(b);
  }
};

// (P, S) of V columns in LDS or in the workspace: [V][2][64], a lane's values 64 floats apart; with the S of both
// directions [V][3][64], of which I = 1 or 2 is run
template <int V, int N = 2> __device__ __forceinline__ void put_range(float* p, int lane, const float* P, const float* S,
                                                                      const float* S2 = nullptr) {
#pragma unroll
  for (int k = 0; k < V; ++k) {
    p[(N * k) * 64 + lane] = P[k];
    p[(N * k + 1) * 64 + lane] = S[k];
    if constexpr (N == 3) p[(N * k + 2) * 64 + lane] = S2[k];
  }
}
template <int V, int N = 2, int I = 1> __device__ __forceinline__ void run_range(const float* p, int lane, float* s) {
#pragma unroll
  for (int k = 0; k < V; ++k) s[k] = after(p[(N * k) * 64 + lane], p[(N * k + I) * 64 + lane], s[k]);
}
template <int V> __device__ __forceinline__ void join_range(const float* p, int lane, float* P, float* S) {
#pragma unroll
  for (int k = 0; k < V; ++k) {
    const float p2 = p[(2 * k) * 64 + lane], s2 = p[(2 * k + 1) * 64 + lane];
    S[k] = after(p2, s2, S[k]);
    P[k] = chain(p2, P[k]);
  }
}
// The P of a wave's own steps: finite, zero where a cut lies in them, never by underflow
template <int V> __device__ __forceinline__ void mark_cut(float* P, uint32_t cut) {
#pragma unroll
  for (int k = 0; k < V; ++k) P[k] = cut >> k & 1u ? 0.0f : (P[k] == 0.0f ? smallest() : finite(P[k]));
}

// Steps per wave and round, and the most waves of a workgroup (256 registers a lane)
template <int V> constexpr int scan_steps() { return V >= 4 ? 4 : 8; }
template <int V> constexpr int scan_grad_steps() { return V >= 2 ? 4 : 8; }
constexpr int SCAN_WAVES = 8;

// Flags are rare: the selects for a step are jumped over where no lane of the wave has one.
__device__ __forceinline__ bool any_lane(uint32_t bits) { return __ballot(bits != 0u) != 0ull; }

// f and the input's share of U steps from t0 on; steps from tend on hold the state
template <class T, int V, int U, bool SIG, bool MASK, bool NI>
struct ForwardSteps {
  Vec<T, V> z[U], x[U];
  typename Columns<V, NI>::Flags d[MASK ? U : 1];

  __device__ __forceinline__ void load(const ScanArgs& a, const Columns<V, NI>& col, const T* gate, const T* in, int t0,
                                       int tend) {
    const T *pz = gate + t0 * a.gate.st, *px = in + t0 * a.x.st;
#pragma unroll
    for (int u = 0; u < U; ++u, pz += a.gate.st, px += a.x.st) {
      if (t0 + u < tend) {
        z[u].load(pz);
        x[u].load(px);
        if constexpr (MASK)
          if (a.done) d[u] = col.load_done(a, t0 + u);
      }
    }
  }
  __device__ __forceinline__ void masks(const ScanArgs& a, const Columns<V, NI>& col,
                                        const typename Columns<V, NI>::Lens& len, int u, int t, uint32_t& done,
                                        uint32_t& hold) const {
    hold = col.over(len, t);
    done = a.done ? col.ended(d[u]) & ~hold : 0u;
  }
  // f and the input's share of one step
  __device__ __forceinline__ void step(int u, uint32_t hold, float* f, float* in) const {
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const float zz = z[u].get(k), xx = x[u].get(k);
      if constexpr (SIG) {
        float g;
        sigmoid2<T>(zz, f[k], g);
        in[k] = g * xx;
      } else {
        f[k] = zz;
        in[k] = xx;
      }
    }
    if (MASK && any_lane(hold)) {
#pragma unroll
      for (int k = 0; k < V; ++k)
        if (hold >> k & 1u) f[k] = 1.0f, in[k] = 0.0f;
    }
  }
};

// One more step of a range's (P, S)
template <bool MASK, int V>
__device__ __forceinline__ void append(float* P, float* S, const float* f, const float* in, uint32_t done) {
#pragma unroll
  for (int k = 0; k < V; ++k) {
    P[k] *= f[k];
    S[k] = __builtin_fmaf(f[k], S[k], in[k]);
  }
  if (MASK && any_lane(done)) {
#pragma unroll
    for (int k = 0; k < V; ++k)
      if (done >> k & 1u) P[k] = 1.0f, S[k] = 0.0f;
  }
}

// launches implemented in scan.hip (shape and argument checks) and scan_backward.hip
struct ScanShape {
  int V, W, K, steps;   // steps: per wave and round
  bool ni;
};
int launch_scan_ranges(const char* fn, const ScanArgs& a, const ScanShape& sh, bool bf16, bool sig, hipStream_t s);   // forward, to a.agg
int launch_scan_forward(const ScanArgs& a, const ScanShape& sh, bool bf16, bool sig, hipStream_t s);
int launch_scan_backward(const ScanArgs& a, const ScanShape& sh, bool bf16, bool sig, hipStream_t s);

// The instance of kernel family KERN for a shape: KERN<T, V, SIG, MASK, NI>
#define AUV_SCAN_AXIS(KERN, T, V, SIG, MASK) \
  (sh.ni ? (const void*)KERN<T, V, SIG, MASK, true> : (const void*)KERN<T, V, SIG, MASK, false>)
#define AUV_SCAN_PICK(KERN, T, V, SIG) (mask ? AUV_SCAN_AXIS(KERN, T, V, SIG, true) : AUV_SCAN_AXIS(KERN, T, V, SIG, false))
#define AUV_SCAN_KIND(KERN, T, V) (sig ? AUV_SCAN_PICK(KERN, T, V, true) : AUV_SCAN_PICK(KERN, T, V, false))
#define AUV_SCAN_KERNEL(KERN)                        \
  (bf16 ? (sh.V == 4   ? AUV_SCAN_KIND(KERN, __bf16, 4) \
           : sh.V == 2 ? AUV_SCAN_KIND(KERN, __bf16, 2) \
                       : AUV_SCAN_KIND(KERN, __bf16, 1)) \
        : (sh.V == 4   ? AUV_SCAN_KIND(KERN, float, 4)  \
           : sh.V == 2 ? AUV_SCAN_KIND(KERN, float, 2)  \
                       : AUV_SCAN_KIND(KERN, float, 1)))

}  // namespace auv
