// Gated linear recurrence, forward (kernels and C interface; scan_backward.hip: its gradient).
//   sigmoid: f = sigma(gate), h_t = f s_{t-1} + (1 - f) x_t     decay: f = gate, h_t = f s_{t-1} + x_t
//   s_t = 0 where the episode ended at step t, else h_t; steps from a sequence's length on hold
//   the state (h_t = s_t = s_{t-1}; their gate, input and done are not looked at).
#include <algorithm>
#include <cmath>

#include "scan.hpp"

namespace auv {

// (P, S) of every chunk of steps but the last: each wave runs a contiguous part of its chunk, the
// first wave joins the parts.  Reads gate and input once: 2 x 256 bf16 columns x 32768 steps in 14 us (4.8 TB/s).
template <class T, int V, bool SIG, bool MASK, bool NI>
__global__ __launch_bounds__(64 * SCAN_WAVES) void k_scan_ranges(ScanArgs a) {
  constexpr int U = scan_steps<V>();
  extern __shared__ float lds[];   // [W][V][2][64]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), W = blockDim.x >> 6;
  const Place at(a);
  const Columns<V, NI> col(a, at.tile, lane);
  const T *gate = col.template base<T>(a.gate), *in = col.template base<T>(a.x);
  typename Columns<V, NI>::Lens len{};
  if constexpr (MASK) len = col.load_lens(a);
  const int part = a.chunk / W, tb = at.chunk * a.chunk + wave * part, te = min(a.T, tb + part);
  float P[V], S[V];
#pragma unroll
  for (int k = 0; k < V; ++k) P[k] = 1.0f, S[k] = 0.0f;
  uint32_t cut = 0;
  for (int t0 = tb; t0 < te; t0 += U) {
    ForwardSteps<T, V, U, SIG, MASK, NI> st;
    st.load(a, col, gate, in, t0, te);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (t0 + u < te) {
        uint32_t done = 0, hold = 0;
        if constexpr (MASK) st.masks(a, col, len, u, t0 + u, done, hold);
        float f[V], v[V];
        st.step(u, hold, f, v);
        append<MASK, V>(P, S, f, v, done);
        cut |= done;
      }
    }
  }
  mark_cut<V>(P, cut);
  put_range<V>(lds + wave * 128 * V, lane, P, S);
  __syncthreads();
  if (wave) return;
  for (int w = 1; w < W; ++w) join_range<V>(lds + w * 128 * V, lane, P, S);
  put_range<V>(a.agg + ((int64_t)at.chunk * a.tiles + at.tile) * 128 * V, lane, P, S);
}

// The states: the waves' ranges joined round by round, each wave's steps redone from the true state with gate and input still
// in registers.  Bound by HBM, three tensors once: 16384 x 64 bf16 columns x 64 steps in 73 us (5.5 TB/s), 4096 x 64 x 512
// in 175 (4.6), 4095 x 23 fp32 x 500 with the sequence fastest, ends and lengths in 141 (4.0; aligned rows without them 106); below some
// thousand columns by a round's chain (load, ranges through LDS, steps: about 1.5 us for 32 or 64 steps).
template <class T, int V, bool SIG, bool MASK, bool NI>
__global__ __launch_bounds__(64 * SCAN_WAVES) void k_scan_forward(ScanArgs a) {
  constexpr int U = scan_steps<V>();
  extern __shared__ float lds[];   // [2][W][V][2][64], by round parity
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), W = blockDim.x >> 6;
  const Place at(a);
  const Columns<V, NI> col(a, at.tile, lane);
  const T *gate = col.template base<T>(a.gate), *in = col.template base<T>(a.x);
  T* out = col.template base<T>(a.h);
  typename Columns<V, NI>::Lens len{};
  if constexpr (MASK) len = col.load_lens(a);
  const int tb = at.chunk * a.chunk, te = min(a.T, tb + a.chunk);

  float s[V];
#pragma unroll
  for (int k = 0; k < V; ++k) s[k] = a.h0.p ? a.h0.p[col.state_at(a, a.h0, k)] : 0.0f;
  if (at.chunk) {   // the chunks before this one, a part per wave
    float P[V], S[V];
#pragma unroll
    for (int k = 0; k < V; ++k) P[k] = 1.0f, S[k] = 0.0f;
    const int j1 = (int)((int64_t)(wave + 1) * at.chunk / W);
    for (int j = (int)((int64_t)wave * at.chunk / W); j < j1; ++j)
      join_range<V>(a.agg + ((int64_t)j * a.tiles + at.tile) * 128 * V, lane, P, S);
    put_range<V>(lds + (W + wave) * 128 * V, lane, P, S);
    __syncthreads();
    for (int w = 0; w < W; ++w) run_range<V>(lds + (W + w) * 128 * V, lane, s);
  }

  // the next round's loads are in flight while a round is computed
  ForwardSteps<T, V, U, SIG, MASK, NI> next;
  next.load(a, col, gate, in, tb + wave * U, te);
  int parity = 0;
  for (int r0 = tb; r0 < te; r0 += W * U, parity ^= 1) {
    const int t0 = r0 + wave * U;
    const ForwardSteps<T, V, U, SIG, MASK, NI> st = next;
    next.load(a, col, gate, in, t0 + W * U, te);
    float f[U][V], v[U][V];
    uint32_t done[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      done[u] = 0;
      if (t0 + u < te) {
        uint32_t hold = 0;
        if constexpr (MASK) st.masks(a, col, len, u, t0 + u, done[u], hold);
        st.step(u, hold, f[u], v[u]);
      } else {
#pragma unroll
        for (int k = 0; k < V; ++k) f[u][k] = 1.0f, v[u][k] = 0.0f;
      }
    }
    float end[V];   // the state after the round
    if (W > 1) {
      float P[V], S[V];
      uint32_t cut = 0;
#pragma unroll
      for (int k = 0; k < V; ++k) P[k] = 1.0f, S[k] = 0.0f;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        append<MASK, V>(P, S, f[u], v[u], done[u]);
        cut |= done[u];
      }
      mark_cut<V>(P, cut);
      float* x = lds + parity * W * 128 * V;
      put_range<V>(x + wave * 128 * V, lane, P, S);
      __syncthreads();
      for (int w = 0; w < wave; ++w) run_range<V>(x + w * 128 * V, lane, s);
#pragma unroll
      for (int k = 0; k < V; ++k) end[k] = s[k];
      for (int w = wave; w < W; ++w) run_range<V>(x + w * 128 * V, lane, end);
    }
    T* po = out + t0 * a.h.st;
#pragma unroll
    for (int u = 0; u < U; ++u, po += a.h.st) {
      if (t0 + u < te) {
        float h[V];
#pragma unroll
        for (int k = 0; k < V; ++k) s[k] = h[k] = __builtin_fmaf(f[u][k], s[k], v[u][k]);
        if (MASK && any_lane(done[u])) {
#pragma unroll
          for (int k = 0; k < V; ++k)
            if (done[u] >> k & 1u) s[k] = 0.0f;
        }
        if (col.active) store_own<T, V>(po, h, col.shift, a.shared);
      }
    }
    if (W > 1) {
#pragma unroll
      for (int k = 0; k < V; ++k) s[k] = end[k];
    }
  }
  if (a.last.p && at.chunk == a.K - 1 && wave == 0 && col.active) {
#pragma unroll
    for (int k = 0; k < V; ++k)
      if (k >= col.shift) a.last.p[col.state_at(a, a.last, k)] = s[k];
  }
}

int launch_scan_ranges(const char* fn, const ScanArgs& a, const ScanShape& sh, bool bf16, bool sig, hipStream_t s) {
  const bool mask = a.done || a.lens;
  ScanArgs arg = a;
  void* args[1] = {&arg};
  return launch_kernel(fn, AUV_SCAN_KERNEL(k_scan_ranges), dim3(a.tiles * (sh.K - 1)), dim3(64 * sh.W), args,
                       sh.W * sizeof(float) * 128 * sh.V, s);
}

int launch_scan_forward(const ScanArgs& a, const ScanShape& sh, bool bf16, bool sig, hipStream_t s) {
  const bool mask = a.done || a.lens;
  ScanArgs arg = a;
  void* args[1] = {&arg};
  const size_t range = sizeof(float) * 128 * sh.V;
  if (sh.K > 1)
    if (int rc = launch_scan_ranges("auv_scan_forward", a, sh, bf16, sig, s)) return rc;
  return launch_kernel("auv_scan_forward", AUV_SCAN_KERNEL(k_scan_forward), dim3(a.tiles * sh.K), dim3(64 * sh.W), args,
                       2 * sh.W * range, s);
}

// ----------------------------------------------------------------------- shapes -------

// Whether the strides are none below zero and no axis spans 2^44 elements or more.
static bool spans(const int64_t* stride, const int64_t* size, int n) {
  for (int k = 0; k < n; ++k)
    if (stride[k] < 0 || (size[k] > 1 && stride[k] > ((int64_t)1 << 44) / (size[k] - 1))) return false;
  return true;
}

// Whether no two elements of an output share memory: each axis steps over all of the ones inside it.
static bool disjoint(const int64_t* stride, const int64_t* size, int n) {
  int order[3] = {0, 1, 2};
  std::sort(order, order + n, [&](int i, int j) { return stride[i] < stride[j]; });
  int64_t span = 1;
  for (int q = 0; q < n; ++q) {
    const int i = order[q];
    if (size[i] == 1) continue;
    if (stride[i] < span) return false;
    span = stride[i] * (size[i] - 1) + span;
  }
  return true;
}

static int check_state(const char* fn, const char* name, const auv_seq_state& s, const auv_scan* d, bool output) {
  if (!s.p) return AUV_OK;
  if (reinterpret_cast<uintptr_t>(s.p) & 3u) return set_error(AUV_EINVAL, "%s: '%s' is not 4-byte aligned", fn, name);
  const int64_t st[2] = {s.sn, s.sc}, size[2] = {d->n, d->c};
  if (!spans(st, size, 2)) return set_error(AUV_EINVAL, "%s: '%s' has a negative stride or spans 2^44 elements or more", fn, name);
  if (output && !disjoint(st, size, 2)) return set_error(AUV_EINVAL, "%s: elements of '%s' share memory", fn, name);
  return AUV_OK;
}

static int check_seq(const char* fn, const char* name, const auv_seq& s, const auv_scan* d, bool output) {
  if (!s.p) return set_error(AUV_EINVAL, "%s: '%s' is NULL", fn, name);
  if (reinterpret_cast<uintptr_t>(s.p) & (d->type == AUV_BF16 ? 1u : 3u))
    return set_error(AUV_EINVAL, "%s: '%s' is not aligned to its elements", fn, name);
  const int64_t st[3] = {s.st, s.sn, s.sc}, size[3] = {d->T, d->n, d->c};
  if (!spans(st, size, 3)) return set_error(AUV_EINVAL, "%s: '%s' has a negative stride or spans 2^44 elements or more", fn, name);
  if (output && !disjoint(st, size, 3)) return set_error(AUV_EINVAL, "%s: elements of '%s' share memory", fn, name);
  return AUV_OK;
}

static int check_scan(const char* fn, const auv_scan* d) {
  if (!d) return set_error(AUV_EINVAL, "%s: NULL argument", fn);
  if (d->T < 1 || d->n < 1 || d->c < 1) return set_error(AUV_EINVAL, "%s: T, n and c must be >= 1", fn);
  if ((int64_t)d->n * d->c > ((int64_t)1 << 30)) return set_error(AUV_EINVAL, "%s: n c exceeds 2^30", fn);
  if (d->T > (1 << 30)) return set_error(AUV_EINVAL, "%s: T exceeds 2^30", fn);
  if (d->type != AUV_FP32 && d->type != AUV_BF16) return set_error(AUV_EINVAL, "%s: unknown type %d", fn, d->type);
  if (d->kind != AUV_SCAN_SIGMOID && d->kind != AUV_SCAN_DECAY) return set_error(AUV_EINVAL, "%s: unknown kind %d", fn, d->kind);
  if ((reinterpret_cast<uintptr_t>(d->done) | reinterpret_cast<uintptr_t>(d->lens)) & 3u)
    return set_error(AUV_EINVAL, "%s: 'done' or 'lens' is not 4-byte aligned", fn);
  return AUV_OK;
}

static SeqTensor inner_first(const auv_seq& s, bool ni) {
  return {static_cast<char*>(s.p), ni ? s.sc : s.sn, ni ? s.sn : s.sc, s.st};
}

// Columns, vectors, waves per workgroup and chunks for the tensors of one pass.
static void scan_shape(const auv_scan* d, const auv_seq* const* seqs, int count, bool grad, ScanArgs& a, ScanShape& sh) {
  const int n = d->n, c = d->c;
  bool unit_c = true, unit_n = true, rows = true;
  for (int k = 0; k < count; ++k) {
    unit_c &= c == 1 || seqs[k]->sc == 1;
    unit_n &= n == 1 || seqs[k]->sn == 1;
    rows &= n == 1 || seqs[k]->sn == c;
  }
  // the axis that is contiguous in every tensor; with none, the shorter stride, element by element
  sh.ni = (unit_c && unit_n) ? c == 1 : (unit_c || unit_n) ? unit_n : d->x.sn < d->x.sc;
  const bool unit = unit_c || unit_n, flat = !sh.ni && unit_c && rows;
  a.Li = sh.ni ? n : (flat ? n * c : c);
  a.Lo = sh.ni ? c : (flat ? 1 : n);
  const int cus = compute_units();
  auto tiles_of = [&](int V) { return (int)(((int64_t)a.Lo * ((a.Li + V - 1) / V) + 63) / 64); };
  // A vector that straddles sequences straddles two at most.
  auto fits = [&](int V) { return unit && a.Li >= V && (sh.ni || c >= V || a.Li == c); };
  // Wide vectors where they leave four waves per CU: bf16, 4096 x 64 columns x 512 steps, both directions: V = 4 in 595
  // us, V = 2 640, V = 1 997.  Else two columns per lane: they make the fewest lane accesses that still fill the chip
  // (37037 bf16 columns x 700: V = 4 in 199, V = 2 153, V = 1 146); but
  // one where only that gives a workgroup per CU without splitting the steps and an access is 4 bytes all the same
  // (fp32, 16384 columns x 1024: V = 1 in 142, V = 2 split in four 167).
  sh.V = fits(4) && tiles_of(4) >= 4 * cus ? 4 : fits(2) && tiles_of(1) > 1 ? 2 : 1;
  if (sh.V == 2 && d->type == AUV_FP32 && tiles_of(2) < cus && tiles_of(1) >= cus) sh.V = 1;
  a.nvec = (a.Li + sh.V - 1) / sh.V;
  a.tiles = tiles_of(sh.V);
  const int U = sh.steps = sh.V >= (grad ? 2 : 4) ? 4 : 8;   // scan_steps, scan_grad_steps
  // Waves per workgroup until there are eight per CU (4095 x 23 fp32 columns x 500 steps, 736 tiles, forward and backward: one wave
  // 160 and 355 us, two 145 and 260, four 142 and 243; where there are eight anyway one wave is best, 16384 x 64 bf16 columns x 64 steps
  // forward: 74, two waves 87); four per CU do for accesses of 16 bytes (4096 x 64 fp32 columns x 128: one wave 73 and 149, two 79 and 157).
  // A bf16 gradient leaves the state before each round: rounds of 8 steps at least (a quarter of a tensor in the workspace, or
  // 16 KB of LDS; backward of 16384 x 64 columns x 64 steps: 4 steps 215 us, 8 187, 16 194; 4096 x 64 x 512: 8 411, 16 495).
  sh.W = 1;
  const bool marks = grad && d->type == AUV_BF16;
  const int enough = sh.V == 4 && d->type == AUV_FP32 ? 4 : 8;
  while (sh.W < SCAN_WAVES && sh.W * U < d->T && ((int64_t)a.tiles * sh.W < enough * cus || (marks && sh.W * U < 8))) sh.W *= 2;
  const int span = sh.W * U, rounds = (d->T - 1) / span + 1;
  // Steps split over workgroups where there is less than one per CU, up to two per CU: reads gate and input (or dout) once more.
  // bf16, forward and backward: 2048 columns x 4096 steps whole 147 and 470 us, split in 16 23 and 55, in 32 21 and 44, in 64 26 and 51;
  // 16384 columns x 1024 steps whole 41 and 122, in four 33 and 70, in eight 37 and 73; 32768 columns (256 tiles) whole 43 and 123, in
  // two 51 and 114.
  sh.K = 1;
  const bool in_place = d->last.p && d->last.p == d->h0.p;   // its chunks would read what the last one writes
  if (sh.W == SCAN_WAVES && rounds >= 4 && d->T >= AUV_SCAN_SPLIT_STEPS && a.tiles < cus && !in_place)
    sh.K = std::min((2 * cus - 1) / a.tiles + 1, rounds);
  a.chunk = ((rounds - 1) / sh.K + 1) * span;
  sh.K = (d->T - 1) / a.chunk + 1;
  a.K = sh.K;
  a.grouped = sh.K == 1 && d->x.st * (d->type == AUV_BF16 ? 2 : 4) % 128 != 0;
  // Stores pass by the caches (16384 x 64 bf16 columns x 64 steps: 81 us without the hint, 72 with it), but for fp32 rows that share
  // lines (4095 x 23 columns x 500 steps, forward and backward 359 us plain, 375 with it; bf16, 37037 columns x 700 steps: 158 plain, 159).
  a.shared = a.grouped && d->type == AUV_FP32;
  a.T = d->T;
  a.n = n;
  a.c = c;
  a.done = d->done;
  a.lens = d->lens;
}

static void forward_args(const auv_scan* d, ScanArgs& a, ScanShape& sh) {
  const auv_seq* seqs[3] = {&d->gate, &d->x, &d->h};
  scan_shape(d, seqs, 3, false, a, sh);
  a.gate = inner_first(d->gate, sh.ni);
  a.x = inner_first(d->x, sh.ni);
  a.h = inner_first(d->h, sh.ni);
}

static void backward_args(const auv_scan* d, const auv_scan_grad* g, ScanArgs& a, ScanShape& sh) {
  const auv_seq* seqs[6] = {&d->gate, &d->h, &g->dgate, &g->dx, &d->x, &g->dout};
  int count = 5;
  if (g->dout.p) seqs[count++] = &g->dout;
  scan_shape(d, seqs, count, true, a, sh);
  a.gate = inner_first(d->gate, sh.ni);
  a.x = inner_first(d->x, sh.ni);
  a.h = inner_first(d->h, sh.ni);
  a.dout = inner_first(g->dout, sh.ni);
  a.dgate = inner_first(g->dgate, sh.ni);
  a.dx = inner_first(g->dx, sh.ni);
}

// A call's workspace: the ranges of split steps, a bf16 gradient's in both directions, and its states before the rounds.
static int64_t place_work(const auv_scan* d, const auv_scan_grad* g, ScanArgs& a, const ScanShape& sh, void* work) {
  const bool form = g && d->type == AUV_BF16;
  const int64_t range = sh.K > 1 ? (int64_t)sh.K * a.tiles * 128 * sh.V : 0;   // floats
  const int64_t marks = form && d->T >= AUV_SCAN_SPLIT_STEPS ? (int64_t)sh.K * (a.chunk / (sh.W * sh.steps)) * a.tiles * 64 * sh.V : 0;
  a.agg = static_cast<float*>(work);
  a.before = work && form ? a.agg + range : nullptr;
  a.marks = work && marks ? a.agg + 2 * range : nullptr;
  return (range * (form ? 2 : 1) + marks) * (int64_t)sizeof(float);
}

}  // namespace auv

// ------------------------------------------------------------------ C interface ----
using namespace auv;

extern "C" {

int64_t auv_scan_work_bytes(const auv_scan* d, const auv_scan_grad* g) {
  if (check_scan("auv_scan_work_bytes", d)) return -1;
  ScanArgs a{};
  ScanShape sh{};
  if (g) backward_args(d, g, a, sh);
  else forward_args(d, a, sh);
  return place_work(d, g, a, sh, nullptr);
}

int auv_scan_forward(const auv_scan* d, void* work, void* stream) {
  const char* fn = "auv_scan_forward";
  if (int rc = check_scan(fn, d)) return rc;
  if (int rc = check_seq(fn, "gate", d->gate, d, false)) return rc;
  if (int rc = check_seq(fn, "x", d->x, d, false)) return rc;
  if (int rc = check_seq(fn, "h", d->h, d, true)) return rc;
  if (int rc = check_state(fn, "h0", d->h0, d, false)) return rc;
  if (int rc = check_state(fn, "last", d->last, d, true)) return rc;
  if (int rc = check_apart(fn, {{"h", d->h.p}, {"last", d->last.p}},
                           {{"gate", d->gate.p}, {"x", d->x.p}, {"done", d->done}, {"lens", d->lens}}))
    return rc;
  if (int rc = check_apart(fn, {{"h", d->h.p}}, {{"h0", d->h0.p}})) return rc;   // 'last' may be 'h0'
  if (d->last.p && d->last.p == d->h0.p && (d->last.sn != d->h0.sn || d->last.sc != d->h0.sc))
    return set_error(AUV_EINVAL, "%s: 'last' is the memory of 'h0' with other strides", fn);
  ScanArgs a{};
  ScanShape sh{};
  forward_args(d, a, sh);
  if (place_work(d, nullptr, a, sh, work) && (!work || !aligned16(work)))
    return set_error(AUV_EINVAL, "%s: 'work' is NULL or not 16-byte aligned", fn);
  a.h0 = {d->h0.p, d->h0.sn, d->h0.sc};
  a.last = {d->last.p, d->last.sn, d->last.sc};
  return launch_scan_forward(a, sh, d->type == AUV_BF16, d->kind == AUV_SCAN_SIGMOID, (hipStream_t)stream);
}

int auv_scan_backward(const auv_scan* d, const auv_scan_grad* g, void* work, void* stream) {
  const char* fn = "auv_scan_backward";
  if (int rc = check_scan(fn, d)) return rc;
  if (!g) return set_error(AUV_EINVAL, "%s: NULL argument", fn);
  if (int rc = check_seq(fn, "gate", d->gate, d, false)) return rc;
  if (int rc = check_seq(fn, "x", d->x, d, false)) return rc;
  if (int rc = check_seq(fn, "h", d->h, d, false)) return rc;
  if (g->dout.p)
    if (int rc = check_seq(fn, "dout", g->dout, d, false)) return rc;
  if (int rc = check_seq(fn, "dgate", g->dgate, d, true)) return rc;
  if (int rc = check_seq(fn, "dx", g->dx, d, true)) return rc;
  if (int rc = check_state(fn, "h0", d->h0, d, false)) return rc;
  if (int rc = check_state(fn, "dlast", g->dlast, d, false)) return rc;
  if (int rc = check_state(fn, "dh0", g->dh0, d, true)) return rc;
  if (int rc = check_apart(fn, {{"dgate", g->dgate.p}, {"dx", g->dx.p}, {"dh0", g->dh0.p}},
                           {{"gate", d->gate.p}, {"x", d->x.p}, {"h", d->h.p}, {"dout", g->dout.p}, {"done", d->done}, {"lens", d->lens},
                            {"h0", d->h0.p}, {"dlast", g->dlast.p}}))
    return rc;
  ScanArgs a{};
  ScanShape sh{};
  backward_args(d, g, a, sh);
  if (place_work(d, g, a, sh, work) && (!work || !aligned16(work)))
    return set_error(AUV_EINVAL, "%s: 'work' is NULL or not 16-byte aligned", fn);
  a.h0 = {d->h0.p, d->h0.sn, d->h0.sc};
  a.last = {g->dlast.p, g->dlast.sn, g->dlast.sc};
  a.dh0 = {g->dh0.p, g->dh0.sn, g->dh0.sc};
  return launch_scan_backward(a, sh, d->type == AUV_BF16, d->kind == AUV_SCAN_SIGMOID, (hipStream_t)stream);
}

}  // extern "C"
