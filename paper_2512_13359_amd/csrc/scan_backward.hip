// Gated linear recurrence, gradient (scan.hip: the forward pass, shapes and argument checks).
// With G_t the gradient that reaches the state after step t (G_{T-1} = dlast):
//   g_t = dh_t + (1 - done_t) G_t,  G_{t-1} = f_t g_t,  dh0 = G_{-1}
//   sigmoid: dx = (1 - f) g, dgate = f (1 - f) (s_{t-1} - x) g;  decay: dx = g, dgate = s_{t-1} g
//   held steps: dx = dgate = 0, G_{t-1} = dh_t + G_t.
// The same ranges as forward, run from the last step to the first: G before a range is P G + S of
// the G after it.
#include "scan.hpp"

namespace auv {

template <class T, int V, int U, bool SIG, bool MASK, bool NI>
struct BackwardSteps {
  Vec<T, V> z[U], dh[U];
  typename Columns<V, NI>::Flags d[MASK ? U : 1];

  __device__ __forceinline__ void load(const ScanArgs& a, const Columns<V, NI>& col, const T* gate, const T* dout, int t0,
                                       int tend) {
    const T *pz = gate + t0 * a.gate.st, *pd = dout + t0 * a.dout.st;
#pragma unroll
    for (int u = 0; u < U; ++u, pz += a.gate.st, pd += a.dout.st) {
      dh[u].w = 0;
      if (t0 + u < tend) {
        z[u].load(pz);
        if (a.dout.p) dh[u].load(pd);
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
  // f and the weight 1 - f of the input
  __device__ __forceinline__ void gates(int u, uint32_t hold, float* f, float* in) const {
#pragma unroll
    for (int k = 0; k < V; ++k) {
      if constexpr (SIG) {
        sigmoid2<T>(z[u].get(k), f[k], in[k]);
      } else {
        f[k] = z[u].get(k);
        in[k] = 1.0f;
      }
    }
    if (MASK && any_lane(hold)) {
#pragma unroll
      for (int k = 0; k < V; ++k)
        if (hold >> k & 1u) f[k] = 1.0f, in[k] = 0.0f;
    }
  }
  // one step earlier in a range's (P, S)
  __device__ __forceinline__ void prepend(int u, const float* f, uint32_t done, float* P, float* S) const {
    if (MASK && any_lane(done)) {
#pragma unroll
      for (int k = 0; k < V; ++k)
        if (done >> k & 1u) P[k] = 1.0f, S[k] = 0.0f;
    }
#pragma unroll
    for (int k = 0; k < V; ++k) {
      P[k] *= f[k];
      S[k] = f[k] * (dh[u].get(k) + S[k]);
    }
  }
};

// (P, S) of every chunk of steps but the first
template <class T, int V, bool SIG, bool MASK, bool NI>
__global__ __launch_bounds__(64 * SCAN_WAVES) void k_scan_grad_ranges(ScanArgs a) {
  constexpr int U = scan_grad_steps<V>();
  extern __shared__ float lds[];   // [W][V][2][64]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), W = blockDim.x >> 6;
  const Place at(a);
  const Columns<V, NI> col(a, at.tile, lane);
  const T* gate = col.template base<T>(a.gate);
  const T* dout = a.dout.p ? col.template base<T>(a.dout) : nullptr;
  typename Columns<V, NI>::Lens len{};
  if constexpr (MASK) len = col.load_lens(a);
  const int chunk = at.chunk + 1;
  const int part = a.chunk / W, tb = chunk * a.chunk + wave * part, te = min(a.T, tb + part);
  float P[V], S[V];
#pragma unroll
  for (int k = 0; k < V; ++k) P[k] = 1.0f, S[k] = 0.0f;
  uint32_t cut = 0;
  for (int t0 = tb + part - U; t0 >= tb; t0 -= U) {
    BackwardSteps<T, V, U, SIG, MASK, NI> st;
    st.load(a, col, gate, dout, t0, te);
#pragma unroll
    for (int u = U - 1; u >= 0; --u) {
      if (t0 + u < te) {
        uint32_t done = 0, hold = 0;
        if constexpr (MASK) st.masks(a, col, len, u, t0 + u, done, hold);
        float f[V], in[V];
        st.gates(u, hold, f, in);
        st.prepend(u, f, done, P, S);
        cut |= done;
      }
    }
  }
  mark_cut<V>(P, cut);
  put_range<V>(lds + wave * 128 * V, lane, P, S);
  __syncthreads();
  if (wave != W - 1) return;
  for (int w = W - 2; w >= 0; --w) join_range<V>(lds + w * 128 * V, lane, P, S);
  put_range<V>(a.agg + ((int64_t)chunk * a.tiles + at.tile) * 128 * V, lane, P, S);
}

// Whether the backward pass forms the states again from gate and input instead of reading them from h: a state in 16 bits would
// leave dgate = f (1 - f) (s - x) g little of a state that follows its input (2 % wrong for x = 1 + 0.01 noise, where
// rounding dgate itself is 0.17 %).
template <class T> constexpr bool forms_states() { return sizeof(T) == 2; }

// The same with what the results need besides: the input, and the output of the step before or the state before the round
template <class T, int V, int U, bool SIG, bool MASK, bool NI>
struct BackwardRound : BackwardSteps<T, V, U, SIG, MASK, NI> {
  static constexpr bool FORM = forms_states<T>();
  Vec<T, V> x[U], hb[FORM ? 1 : U];
  float mark[FORM ? V : 1];
  typename Columns<V, NI>::Flags db;   // done of the step before the first

  __device__ __forceinline__ void load(const ScanArgs& a, const Columns<V, NI>& col, const T* gate, const T* dout,
                                       const T* in, const T* h, int t0, int tend) {
    BackwardSteps<T, V, U, SIG, MASK, NI>::load(a, col, gate, dout, t0, tend);
    const T *px = in + t0 * a.x.st, *ph = h + (t0 - 1) * a.h.st;
#pragma unroll
    for (int u = 0; u < U; ++u, px += a.x.st, ph += a.h.st) {
      if constexpr (FORM) x[u].w = 0;
      if (t0 + u < tend) {
        if constexpr (SIG || FORM) x[u].load(px);
        if constexpr (!FORM)
          if (t0 + u > 0) hb[u].load(ph);
      }
    }
    if constexpr (MASK && !FORM)
      if (a.done && t0 > 0 && t0 < tend) db = col.load_done(a, t0 - 1);
  }
  // the input's share of a step
  __device__ __forceinline__ void shares(int u, uint32_t hold, const float* w, float* v) const {
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = SIG ? w[k] * x[u].get(k) : x[u].get(k);
    if (MASK && any_lane(hold)) {
#pragma unroll
      for (int k = 0; k < V; ++k)
        if (hold >> k & 1u) v[k] = 0.0f;
    }
  }
};

// The state before every round of a workgroup's steps, in LDS ([round][V][64], steps below AUV_SCAN_SPLIT_STEPS) or in the workspace.
template <int V> struct Marks {
  float *global, *local;
  int64_t stride;
  int lane;

  __device__ __forceinline__ Marks(const ScanArgs& a, const Place& at, int span, float* lds, int lane)
      : global(nullptr), local(lds), stride((int64_t)a.tiles * 64 * V), lane(lane) {
    if (a.marks) global = a.marks + ((int64_t)at.chunk * (a.chunk / span) * a.tiles + at.tile) * 64 * V;
  }
  __device__ __forceinline__ void put(int round, const float* s) const {
    float* p = global ? global + round * stride : nullptr;
#pragma unroll
    for (int k = 0; k < V; ++k) {
      if (global) p[k * 64 + lane] = s[k];
      else local[(round * V + k) * 64 + lane] = s[k];
    }
  }
  __device__ __forceinline__ void get(int round, float* s) const {
    const float* p = global ? global + round * stride : nullptr;
#pragma unroll
    for (int k = 0; k < V; ++k) s[k] = global ? p[k * 64 + lane] : local[(round * V + k) * 64 + lane];
  }
};

// The gradients, rounds and waves from the last step to the first.  bf16: a walk from the first step to the last before it
// leaves the state before each round, and a round forms its states from there.  Bound by HBM, gate, input, output (bf16: gate and
// input a second time, a quarter of a tensor out and in) and its gradient in, two gradients out: 4096 x 64 bf16 columns x 512 steps
// in 432 us (4.7 TB/s; with the states read from h 338), 4095 x 23 fp32 x 500 with ends and lengths in 222 (4.3).
template <class T, int V, bool SIG, bool MASK, bool NI>
__global__ __launch_bounds__(64 * SCAN_WAVES) void k_scan_backward(ScanArgs a) {
  constexpr int U = scan_grad_steps<V>();
  constexpr bool FORM = forms_states<T>();
  constexpr int N = FORM ? 3 : 2;   // P and the S of the gradient, or of both directions
  extern __shared__ float lds[];    // [2][W][V][N][64], by round parity; then the marks
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), W = blockDim.x >> 6;
  const Place at(a);
  const Columns<V, NI> col(a, at.tile, lane);
  const T *gate = col.template base<T>(a.gate), *in = col.template base<T>(a.x), *hp = FORM ? nullptr : col.template base<T>(a.h);
  const T* dout = a.dout.p ? col.template base<T>(a.dout) : nullptr;
  T *dgate = col.template base<T>(a.dgate), *dx = col.template base<T>(a.dx);
  typename Columns<V, NI>::Lens len{};
  if constexpr (MASK) len = col.load_lens(a);
  const int tb = at.chunk * a.chunk, te = min(a.T, tb + a.chunk);
  const int span = W * U, rounds = (te - tb - 1) / span + 1;
  const Marks<V> marks(a, at, span, lds + 2 * W * 64 * V * N, lane);

  if constexpr (FORM) {
    float s[V];
#pragma unroll
    for (int k = 0; k < V; ++k) s[k] = a.h0.p ? a.h0.p[col.state_at(a, a.h0, k)] : 0.0f;
    if (at.chunk) {   // the chunks before this one, a part per wave
      float P[V], S[V];
#pragma unroll
      for (int k = 0; k < V; ++k) P[k] = 1.0f, S[k] = 0.0f;
      const int j1 = (int)((int64_t)(wave + 1) * at.chunk / W);
      for (int j = (int)((int64_t)wave * at.chunk / W); j < j1; ++j)
        join_range<V>(a.before + ((int64_t)j * a.tiles + at.tile) * 128 * V, lane, P, S);
      put_range<V>(lds + wave * 128 * V, lane, P, S);
      __syncthreads();
      for (int w = 0; w < W; ++w) run_range<V>(lds + w * 128 * V, lane, s);
      __syncthreads();
    }
    ForwardSteps<T, V, U, SIG, MASK, NI> next;
    if (rounds > 1) next.load(a, col, gate, in, tb + wave * U, te);
    int parity = 0;
    for (int r = 0;; ++r, parity ^= 1) {
      if (wave == 0) marks.put(r, s);
      if (r == rounds - 1) break;   // steps of a round before the last are all below te
      const int t0 = tb + r * span + wave * U;
      const ForwardSteps<T, V, U, SIG, MASK, NI> st = next;
      if (r + 2 < rounds) next.load(a, col, gate, in, t0 + span, te);
      float P[V], S[V];
      uint32_t cut = 0;
#pragma unroll
      for (int k = 0; k < V; ++k) P[k] = 1.0f, S[k] = W > 1 ? 0.0f : s[k];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        uint32_t done = 0, hold = 0;
        if constexpr (MASK) st.masks(a, col, len, u, t0 + u, done, hold);
        float f[V], v[V];
        st.step(u, hold, f, v);
        append<MASK, V>(P, S, f, v, done);
        cut |= done;
      }
      if (W > 1) {
        mark_cut<V>(P, cut);
        float* x = lds + parity * W * 128 * V;
        put_range<V>(x + wave * 128 * V, lane, P, S);
        __syncthreads();
        for (int w = 0; w < W; ++w) run_range<V>(x + w * 128 * V, lane, s);
      } else {
#pragma unroll
        for (int k = 0; k < V; ++k) s[k] = S[k];
      }
    }
    __syncthreads();   // the marks are there, the waves' ranges read
  }

  float G[V];
#pragma unroll
  for (int k = 0; k < V; ++k) G[k] = a.last.p ? a.last.p[col.state_at(a, a.last, k)] : 0.0f;
  const int later = a.K - 1 - at.chunk;
  if (later) {   // the chunks after this one, a part per wave
    float P[V], S[V];
#pragma unroll
    for (int k = 0; k < V; ++k) P[k] = 1.0f, S[k] = 0.0f;
    const int j0 = (int)((int64_t)wave * later / W), j1 = (int)((int64_t)(wave + 1) * later / W);
    for (int j = j0; j < j1; ++j)   // from the last chunk down
      join_range<V>(a.agg + ((int64_t)(a.K - 1 - j) * a.tiles + at.tile) * 128 * V, lane, P, S);
    float* x = lds + W * 64 * V * N;
    put_range<V>(x + wave * 128 * V, lane, P, S);
    __syncthreads();
    for (int w = 0; w < W; ++w) run_range<V>(x + w * 128 * V, lane, G);
  }

  // the next round's loads are in flight while a round is computed
  BackwardRound<T, V, U, SIG, MASK, NI> next;
  auto load = [&](int r) {
    next.load(a, col, gate, dout, in, hp, tb + r * span + wave * U, te);
    if constexpr (FORM) marks.get(r, next.mark);
  };
  load(rounds - 1);
  int parity = 0;
  for (int r = rounds - 1; r >= 0; --r, parity ^= 1) {
    const int t0 = tb + r * span + wave * U;
    const BackwardRound<T, V, U, SIG, MASK, NI> st = next;
    if (r > 0) load(r - 1);
    float f[U][V], w1[U][V];
    uint32_t done[U], hold[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      done[u] = hold[u] = 0;
      if (t0 + u < te) {
        if constexpr (MASK) st.masks(a, col, len, u, t0 + u, done[u], hold[u]);
        st.gates(u, hold[u], f[u], w1[u]);
      } else {
#pragma unroll
        for (int k = 0; k < V; ++k) f[u][k] = 1.0f, w1[u][k] = 0.0f;
      }
    }
    float before[V];   // G before the round's first step
    float s[V];        // the state before the wave's first step
    if constexpr (FORM) {
#pragma unroll
      for (int k = 0; k < V; ++k) s[k] = st.mark[k];
    }
    if (W > 1) {
      float P[V], S[V], S2[V];
      uint32_t cut = 0;
      if constexpr (FORM) {
#pragma unroll
        for (int k = 0; k < V; ++k) P[k] = 1.0f, S2[k] = 0.0f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          float v[V];
          st.shares(u, hold[u], w1[u], v);
          append<MASK, V>(P, S2, f[u], v, done[u]);
        }
      }
#pragma unroll
      for (int k = 0; k < V; ++k) P[k] = 1.0f, S[k] = 0.0f;
#pragma unroll
      for (int u = U - 1; u >= 0; --u) {
        st.prepend(u, f[u], done[u], P, S);
        cut |= done[u];
      }
      mark_cut<V>(P, cut);
      float* x = lds + parity * W * 64 * V * N;
      put_range<V, N>(x + wave * 64 * V * N, lane, P, S, S2);
      __syncthreads();
      if constexpr (FORM)
        for (int w = 0; w < wave; ++w) run_range<V, N, 2>(x + w * 64 * V * N, lane, s);
      for (int w = W - 1; w > wave; --w) run_range<V, N>(x + w * 64 * V * N, lane, G);
#pragma unroll
      for (int k = 0; k < V; ++k) before[k] = G[k];
      for (int w = wave; w >= 0; --w) run_range<V, N>(x + w * 64 * V * N, lane, before);
    }
    float sp[U][V];   // the state before each step
    if constexpr (FORM) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float v[V];
        st.shares(u, hold[u], w1[u], v);
#pragma unroll
        for (int k = 0; k < V; ++k) {
          sp[u][k] = s[k];
          s[k] = __builtin_fmaf(f[u][k], s[k], v[k]);
        }
        if (MASK && any_lane(done[u])) {
#pragma unroll
          for (int k = 0; k < V; ++k)
            if (done[u] >> k & 1u) s[k] = 0.0f;
        }
      }
    }
#pragma unroll
    for (int u = U - 1; u >= 0; --u) {
      if (t0 + u < te) {
        const int t = t0 + u;
        float gz[V], gx[V];
        uint32_t fresh = 0;   // columns whose state before this step is a new episode's zero
        if constexpr (!FORM) {
          if (t > 0) {
#pragma unroll
            for (int k = 0; k < V; ++k) sp[u][k] = st.hb[u].get(k);
          } else {
#pragma unroll
            for (int k = 0; k < V; ++k) sp[u][k] = a.h0.p ? a.h0.p[col.state_at(a, a.h0, k)] : 0.0f;
          }
          if constexpr (MASK) fresh = u ? done[u > 0 ? u - 1 : 0] : (a.done && t > 0 ? col.ended(st.db) : 0u);
        }
        if constexpr (MASK) {
          if (any_lane(fresh | done[u])) {
#pragma unroll
            for (int k = 0; k < V; ++k) {
              if (!FORM && (fresh >> k & 1u)) sp[u][k] = 0.0f;
              if (done[u] >> k & 1u) G[k] = 0.0f;
            }
          }
        }
#pragma unroll
        for (int k = 0; k < V; ++k) {
          const float g = st.dh[u].get(k) + G[k];
          if constexpr (SIG) {
            gx[k] = w1[u][k] * g;
            gz[k] = f[u][k] * (sp[u][k] - st.x[u].get(k)) * gx[k];
          } else {
            gx[k] = g;
            gz[k] = sp[u][k] * g;
          }
          G[k] = f[u][k] * g;
        }
        if (MASK && any_lane(hold[u])) {
#pragma unroll
          for (int k = 0; k < V; ++k)
            if (hold[u] >> k & 1u) gx[k] = gz[k] = 0.0f;
        }
        if (col.active) {
          store_own<T, V>(dgate + t * a.dgate.st, gz, col.shift, a.shared);
          store_own<T, V>(dx + t * a.dx.st, gx, col.shift, a.shared);
        }
      }
    }
    if (W > 1) {
#pragma unroll
      for (int k = 0; k < V; ++k) G[k] = before[k];
    }
  }
  if (a.dh0.p && at.chunk == 0 && wave == 0 && col.active) {
#pragma unroll
    for (int k = 0; k < V; ++k)
      if (k >= col.shift) a.dh0.p[col.state_at(a, a.dh0, k)] = G[k];
  }
}

int launch_scan_backward(const ScanArgs& a, const ScanShape& sh, bool bf16, bool sig, hipStream_t s) {
  const char* fn = "auv_scan_backward";
  const bool mask = a.done || a.lens;
  ScanArgs arg = a;
  void* args[1] = {&arg};
  const size_t tile = sizeof(float) * 64 * sh.V;
  if (sh.K > 1) {
    if (bf16) {
      ScanArgs fwd = a;
      fwd.agg = a.before;
      if (int rc = launch_scan_ranges(fn, fwd, sh, bf16, sig, s)) return rc;
    }
    if (int rc = launch_kernel(fn, AUV_SCAN_KERNEL(k_scan_grad_ranges), dim3(a.tiles * (sh.K - 1)), dim3(64 * sh.W), args,
                               2 * sh.W * tile, s))
      return rc;
  }
  const size_t marks = bf16 && !a.marks ? (size_t)((a.T - 1) / (sh.W * sh.steps) + 1) : 0;   // in LDS
  return launch_kernel(fn, AUV_SCAN_KERNEL(k_scan_backward), dim3(a.tiles * sh.K), dim3(64 * sh.W), args,
                       (2 * sh.W * (bf16 ? 3 : 2) + marks) * tile, s);
}

}  // namespace auv
