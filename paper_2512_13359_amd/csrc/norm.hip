// Group norm with an activation, channels last, and its gradient; dropout (kernels and C interface).
//   xhat = (x - mean) rstd over the S positions and C / G channels of a group, u = w xhat + b, y = act(u)
//   du = dy act'(u), dw = sum du xhat, db = sum du, d = du w,
//   dx = rstd (d - mean(d) - xhat mean(d xhat)); with dropout both x and dx pass the mask.
#include <algorithm>
#include <cmath>
#include <numeric>

#include "dropout.hpp"
#include "layers.hpp"

namespace auv {

struct NormArgs {
  char *x, *y, *dout, *dx;
  int64_t x_sn, x_ss, y_sn, y_ss, dout_sn, dout_ss, dx_sn, dx_ss;
  const float *w, *b;
  float *mean, *rstd;
  float* part;    // per-block partial results (general form: [n chunks][C] or [n chunks][2][C])
  float* coef;    // backward, general form: [n][G][2] means of d and d xhat
  float *dw, *db;
  float eps;
  int act, n, S, C, G, Cg;
  int m, lanes;   // rows form: elements of a group, lanes per group
  int chunks, per;   // general form: chunks of S positions each
  int tile;          // general form: vectors per workgroup
  int part_rows;     // rows of C partial sums
  DropArgs drop;
};

// Sum over a team of 1 to 64 lanes (a power of two), every lane gets it: moves within rows of 16
// lanes, then lane swaps.
__device__ __forceinline__ float team_sum(float v, int lanes) {
  if (lanes > 1) v += dpp_move<DPP_QUAD_SWAP1>(v);
  if (lanes > 2) v += dpp_move<DPP_QUAD_SWAP2>(v);
  if (lanes > 4) v += dpp_move<DPP_ROW_HALF_MIRROR>(v);   // the other quad of eight lanes, equal in its four
  if (lanes > 8) v += dpp_move<DPP_ROW_MIRROR>(v);
  if (lanes > 16) {
    float u = v;
    asm("s_nop 1\n\tv_permlane16_swap_b32 %0, %1" : "+v"(v), "+v"(u));
    v += u;
  }
  if (lanes > 32) {
    float u = v;
    asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(v), "+v"(u));
    v += u;
  }
  return v;
}

// -------------------------------------------------------------------- rows form -------
// A group of up to 1024 contiguous numbers (S = 1, or one group over dense positions) held in the
// registers of 1 to 64 lanes: read once, statistics by lane swaps, written once.  A team of lanes
// keeps its channels over all of its rows, and with them weights and the sums of their gradients.
template <class T, int V, int NV> struct RowTeam {
  int lane, team, at[NV], shift[NV];

  __device__ __forceinline__ explicit RowTeam(const NormArgs& a) {
    lane = threadIdx.x & (a.lanes - 1);
    team = threadIdx.x / a.lanes;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int e0 = (j * a.lanes + lane) * V;
      at[j] = min(e0, a.m - V);
      shift[j] = min(e0 - at[j], V);
    }
  }
  __device__ __forceinline__ int channel(const NormArgs& a, int g, int j, int k) const {
    return a.S == 1 ? g * a.m + at[j] + k : (at[j] + k) % a.C;
  }
  // of a row's vector j: bit k, whether its element is kept
  __device__ __forceinline__ uint32_t keep(const NormArgs& a, int64_t sample, int g, int j) const {
    if (a.S == 1) return keep_from<V>(a.drop, (uint32_t)sample, g * a.m + at[j]);
    uint32_t bits = 0;
    int pos = at[j] / a.C, c = at[j] % a.C;
    for (int k = 0; k < V;) {
      const int run = min(V - k, a.C - c);
      bits |= (keep_from<V>(a.drop, (uint32_t)(sample * a.S + pos), c) & ((1u << run) - 1u)) << k;
      k += run;
      ++pos;
      c = 0;
    }
    return bits;
  }
};

template <class T, int V, int NV, bool DROP>
__global__ __launch_bounds__(256) void k_norm_rows(NormArgs a) {
  const RowTeam<T, V, NV> tm(a);
  const int per = 256 / a.lanes;
  const int64_t rows = (int64_t)a.n * a.G, stride = (int64_t)gridDim.x * per;   // a multiple of G
  int64_t r = (int64_t)blockIdx.x * per + tm.team;
  const int g = a.G == 1 ? 0 : (int)(r % a.G);
  int64_t sample = a.G == 1 ? r : r / a.G;
  const int64_t samples = a.G == 1 ? stride : stride / a.G;
  float w[NV][V], b[NV][V];
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const int c = tm.channel(a, g, j, k);
      w[j][k] = a.w ? a.w[c] : 1.0f;
      b[j][k] = a.b ? a.b[c] : 0.0f;
    }
  const float inv = 1.0f / (float)a.m;
  const T* x = reinterpret_cast<const T*>(a.x) + sample * a.x_sn + g * a.m;
  T* y = reinterpret_cast<T*>(a.y) + sample * a.y_sn + g * a.m;
  Vec<T, V> next[NV];
  if (r < rows) {
#pragma unroll
    for (int j = 0; j < NV; ++j) next[j].load(x + tm.at[j]);
  }
  for (; r < rows; r += stride, sample += samples, y += samples * a.y_sn) {
    Vec<T, V> q[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) q[j] = next[j];
    x += samples * a.x_sn;
    if (r + stride < rows) {
#pragma unroll
      for (int j = 0; j < NV; ++j) next[j].load(x + tm.at[j]);
    }
    float v[NV][V], sum = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      uint32_t keep = 0;
      if constexpr (DROP) keep = tm.keep(a, sample, g, j);
#pragma unroll
      for (int k = 0; k < V; ++k) {
        v[j][k] = q[j].get(k);
        if constexpr (DROP) v[j][k] = keep >> k & 1u ? v[j][k] * a.drop.scale : 0.0f;
        if (k >= tm.shift[j]) sum += v[j][k];
      }
    }
    const float mean = team_sum(sum, a.lanes) * inv;
    float ss = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int k = 0; k < V; ++k) {
        v[j][k] -= mean;
        if (k >= tm.shift[j]) ss = __builtin_fmaf(v[j][k], v[j][k], ss);
      }
    const float rstd = rsqrt_of(__builtin_fmaf(team_sum(ss, a.lanes), inv, a.eps));
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int k = 0; k < V; ++k) v[j][k] = __builtin_fmaf(v[j][k] * rstd, w[j][k], b[j][k]);
    act_all<T, NV * V>(a.act, &v[0][0]);
#pragma unroll
    for (int j = 0; j < NV; ++j) store_own<T, V>(y + tm.at[j], v[j], tm.shift[j], false);
    if (tm.lane == 0) {
      a.mean[r] = mean;
      a.rstd[r] = rstd;
    }
  }
}

template <class T, int V, int NV, bool DROP>
__global__ __launch_bounds__(256) void k_norm_rows_grad(NormArgs a) {
  const RowTeam<T, V, NV> tm(a);
  const int per = 256 / a.lanes;
  const int64_t rows = (int64_t)a.n * a.G, stride = (int64_t)gridDim.x * per;   // a multiple of G
  int64_t r = (int64_t)blockIdx.x * per + tm.team;
  const int g = a.G == 1 ? 0 : (int)(r % a.G);
  int64_t sample = a.G == 1 ? r : r / a.G;
  const int64_t samples = a.G == 1 ? stride : stride / a.G, first = sample;
  float w[NV][V], b[NV][V], dw[NV][V], db[NV][V];
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const int c = tm.channel(a, g, j, k);
      w[j][k] = a.w ? a.w[c] : 1.0f;
      b[j][k] = a.b ? a.b[c] : 0.0f;
      dw[j][k] = db[j][k] = 0.0f;
    }
  const float inv = 1.0f / (float)a.m;
  const T* x = reinterpret_cast<const T*>(a.x) + sample * a.x_sn + g * a.m;
  const T* dy = reinterpret_cast<const T*>(a.dout) + sample * a.dout_sn + g * a.m;
  T* dx = reinterpret_cast<T*>(a.dx) + sample * a.dx_sn + g * a.m;
  Vec<T, V> next_x[NV], next_e[NV];
  float next_mean = 0.0f, next_rstd = 0.0f;
  auto load = [&](int64_t row) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      next_x[j].load(x + tm.at[j]);
      next_e[j].load(dy + tm.at[j]);
    }
    next_mean = a.mean[row];
    next_rstd = a.rstd[row];
  };
  if (r < rows) load(r);
  for (; r < rows; r += stride, sample += samples, dx += samples * a.dx_sn) {
    Vec<T, V> q[NV], e[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) q[j] = next_x[j], e[j] = next_e[j];
    const float mean = next_mean, rstd = next_rstd;
    x += samples * a.x_sn;
    dy += samples * a.dout_sn;
    if (r + stride < rows) load(r + stride);
    float xh[NV][V], d[NV][V], s1 = 0.0f, s2 = 0.0f;
    uint32_t keep[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      keep[j] = 0;
      if constexpr (DROP) keep[j] = tm.keep(a, sample, g, j);
#pragma unroll
      for (int k = 0; k < V; ++k) {
        float v = q[j].get(k);
        if constexpr (DROP) v = keep[j] >> k & 1u ? v * a.drop.scale : 0.0f;
        xh[j][k] = (v - mean) * rstd;
        d[j][k] = __builtin_fmaf(xh[j][k], w[j][k], b[j][k]);
      }
    }
    slope_all<T, NV * V>(a.act, &d[0][0]);
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int k = 0; k < V; ++k) {
        float du = e[j].get(k) * d[j][k];
        if (k < tm.shift[j]) du = 0.0f;
        dw[j][k] = __builtin_fmaf(du, xh[j][k], dw[j][k]);
        db[j][k] += du;
        d[j][k] = du * w[j][k];
        s1 += d[j][k];
        s2 = __builtin_fmaf(d[j][k], xh[j][k], s2);
      }
    s1 = team_sum(s1, a.lanes) * inv;
    s2 = team_sum(s2, a.lanes) * inv;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float o[V];
#pragma unroll
      for (int k = 0; k < V; ++k) {
        o[k] = rstd * (d[j][k] - s1 - xh[j][k] * s2);
        if constexpr (DROP) o[k] = keep[j] >> k & 1u ? o[k] * a.drop.scale : 0.0f;
      }
      store_own<T, V>(dx + tm.at[j], o, tm.shift[j], false);
    }
  }
  if (!a.part) return;
  // [part row][2][channels]: a team's own sums where there are several groups (team t holds group
  // t mod G), else the workgroup's
  if (a.G > 1) {
    float* p = a.part + first * 2 * a.C + g * a.m;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int k = 0; k < V; ++k)
        if (k >= tm.shift[j]) {
          p[tm.at[j] + k] = dw[j][k];
          p[a.C + tm.at[j] + k] = db[j][k];
        }
    return;
  }
  extern __shared__ float red[];   // [waves][2][m]
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int k = 0; k < V; ++k)
      for (int s = a.lanes; s < 64; s <<= 1) {
        dw[j][k] += __shfl_xor(dw[j][k], s);
        db[j][k] += __shfl_xor(db[j][k], s);
      }
  const int wave = threadIdx.x >> 6;
  if ((int)(threadIdx.x & 63) < a.lanes) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int k = 0; k < V; ++k)
        if (k >= tm.shift[j]) {
          red[(2 * wave) * a.m + tm.at[j] + k] = dw[j][k];
          red[(2 * wave + 1) * a.m + tm.at[j] + k] = db[j][k];
        }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * a.m; i += 256) {
    float s = 0.0f;
    for (int q = 0; q < 4; ++q) s += red[2 * q * a.m + i];
    a.part[(int64_t)blockIdx.x * 2 * a.m + i] = s;
  }
}

// ----------------------------------------------------------------- general form -------
// Any S and groups: a thread keeps V channels and walks over positions; statistics per channel and
// chunk of positions, joined per group by a second launch, applied by a third.
template <class T, int V> struct Walker {
  bool on;
  int i, chunk, c, shift, row, step, s0, s1;   // sample, chunk, channel, positions [s0, s1) from s0 + row on by `step`
  int base, local;                             // the tile's first channel; channels of the tile

  __device__ __forceinline__ explicit Walker(const NormArgs& a) {
    i = blockIdx.x / a.chunks;
    chunk = blockIdx.x - i * a.chunks;
    step = 256 / a.tile;
    row = threadIdx.x / a.tile;
    const int64_t c0 = ((int64_t)blockIdx.y * a.tile + threadIdx.x % a.tile) * V;
    on = row < step && c0 < a.C;
    c = (int)min(c0, (int64_t)(a.C - V));
    shift = (int)min(c0 - c, (int64_t)V);
    base = blockIdx.y * a.tile * V;
    local = min(a.tile * V, a.C - base);
    s0 = chunk * a.per;
    s1 = min(a.S, s0 + a.per);
  }
  __device__ __forceinline__ const T* in(const char* p, int64_t sn) const {
    return reinterpret_cast<const T*>(p) + i * sn + c;
  }
  __device__ __forceinline__ void dropped(const NormArgs& a, int s, float* v) const {
    const uint32_t keep = keep_from<V>(a.drop, (uint32_t)((int64_t)i * a.S + s), c);
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = keep >> k & 1u ? v[k] * a.drop.scale : 0.0f;
  }
};

// Joins (na, ma, Ma) with (nb, mb, Mb): counts, means and sums of squares about the mean (Chan, Golub
// and LeVeque 1979).
__device__ __forceinline__ void join_moments(float& na, float& ma, float& Ma, float nb, float mb, float Mb) {
  const float n = na + nb;
  if (n > 0.0f) {
    const float f = nb / n, d = mb - ma;
    ma = __builtin_fmaf(d, f, ma);
    Ma += __builtin_fmaf(d * d, na * f, Mb);
    na = n;
  }
}

template <class T, int V, bool DROP>
__global__ __launch_bounds__(256) void k_norm_stats(NormArgs a) {
  extern __shared__ float red[];   // [2][step][tile V]
  const Walker<T, V> wk(a);
  const int width = a.tile * V;
  if (wk.on) {
    // sums about the thread's first value: a member of the set, so the subtraction below loses at
    // most the set's size in ulps
    const T* x = wk.in(a.x, a.x_sn);
    float first[V], s1[V], s2[V];
#pragma unroll
    for (int k = 0; k < V; ++k) first[k] = s1[k] = s2[k] = 0.0f;
    int count = 0;
    for (int s = wk.s0 + wk.row; s < wk.s1; s += wk.step) {
      Vec<T, V> q;
      q.load(x + s * a.x_ss);
      float v[V];
#pragma unroll
      for (int k = 0; k < V; ++k) v[k] = q.get(k);
      if constexpr (DROP) wk.dropped(a, s, v);
#pragma unroll
      for (int k = 0; k < V; ++k) {
        if (count == 0) first[k] = v[k];
        const float d = v[k] - first[k];
        s1[k] += d;
        s2[k] = __builtin_fmaf(d, d, s2[k]);
      }
      ++count;
    }
    const float inv = count ? 1.0f / (float)count : 0.0f;
    float* p = red + wk.row * width + wk.c - wk.base;
#pragma unroll
    for (int k = 0; k < V; ++k)
      if (k >= wk.shift) {
        p[k] = __builtin_fmaf(s1[k], inv, first[k]);
        p[wk.step * width + k] = fmaxf(__builtin_fmaf(-s1[k] * inv, s1[k], s2[k]), 0.0f);
      }
  }
  __syncthreads();
  float2* out = reinterpret_cast<float2*>(a.part) + (int64_t)blockIdx.x * a.C + wk.base;
  for (int q = threadIdx.x; q < wk.local; q += 256) {
    float n = 0.0f, mean = 0.0f, M = 0.0f;
    for (int r = 0; r < wk.step; ++r) {
      const int count = (wk.s1 - wk.s0 - r + wk.step - 1) / wk.step;
      if (count > 0) join_moments(n, mean, M, (float)count, red[r * width + q], red[(wk.step + r) * width + q]);
    }
    out[q] = make_float2(mean, M);
  }
}

// mean and rstd of one group from its channels' chunks
__global__ __launch_bounds__(256) void k_norm_stats_join(NormArgs a) {
  __shared__ float sh[3][4];
  const int i = blockIdx.x / a.G, g = blockIdx.x - i * a.G;
  const float2* p = reinterpret_cast<const float2*>(a.part) + (int64_t)i * a.chunks * a.C + g * a.Cg;
  float n = 0.0f, mean = 0.0f, M = 0.0f;
  for (int64_t e = threadIdx.x; e < (int64_t)a.chunks * a.Cg; e += blockDim.x) {
    const int chunk = (int)(e / a.Cg), c = (int)(e - (int64_t)chunk * a.Cg);
    const float2 v = p[(int64_t)chunk * a.C + c];
    join_moments(n, mean, M, (float)(min(a.S, (chunk + 1) * a.per) - chunk * a.per), v.x, v.y);
  }
  for (int d = 1; d < 64; d <<= 1) {
    const float nb = __shfl_xor(n, d), mb = __shfl_xor(mean, d), Mb = __shfl_xor(M, d);
    join_moments(n, mean, M, nb, mb, Mb);
  }
  const int wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) {
    sh[0][wave] = n;
    sh[1][wave] = mean;
    sh[2][wave] = M;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < (int)blockDim.x / 64; ++w) join_moments(n, mean, M, sh[0][w], sh[1][w], sh[2][w]);
    a.mean[blockIdx.x] = mean;
    a.rstd[blockIdx.x] = rsqrt_of(M / n + a.eps);
  }
}

// a thread's channels: mean and rstd of their groups, weight and bias
template <int V> struct ChannelValues {
  float mean[V], rstd[V], w[V], b[V];
  __device__ __forceinline__ ChannelValues(const NormArgs& a, int i, int c) {
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const int64_t g = (int64_t)i * a.G + (c + k) / a.Cg;
      mean[k] = a.mean[g];
      rstd[k] = a.rstd[g];
      w[k] = a.w ? a.w[c + k] : 1.0f;
      b[k] = a.b ? a.b[c + k] : 0.0f;
    }
  }
};

template <class T, int V, bool DROP>
__global__ __launch_bounds__(256) void k_norm_apply(NormArgs a) {
  const Walker<T, V> wk(a);
  if (!wk.on) return;
  const T* x = wk.in(a.x, a.x_sn);
  T* y = const_cast<T*>(wk.in(a.y, a.y_sn));
  const ChannelValues<V> ch(a, wk.i, wk.c);
  for (int s = wk.s0 + wk.row; s < wk.s1; s += wk.step) {
    Vec<T, V> q;
    q.load(x + s * a.x_ss);
    float v[V];
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = q.get(k);
    if constexpr (DROP) wk.dropped(a, s, v);
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = __builtin_fmaf((v[k] - ch.mean[k]) * ch.rstd[k], ch.w[k], ch.b[k]);
    act_all<T, V>(a.act, v);
    store_own<T, V>(y + s * a.y_ss, v, wk.shift, false);
  }
}

template <class T, int V, bool DROP>
__global__ __launch_bounds__(256) void k_norm_grad_sums(NormArgs a) {
  extern __shared__ float red[];   // [2][step][tile V]
  const Walker<T, V> wk(a);
  const int width = a.tile * V;
  if (wk.on) {
    const T *x = wk.in(a.x, a.x_sn), *dy = wk.in(a.dout, a.dout_sn);
    const ChannelValues<V> ch(a, wk.i, wk.c);
    float dw[V], db[V];
#pragma unroll
    for (int k = 0; k < V; ++k) dw[k] = db[k] = 0.0f;
    for (int s = wk.s0 + wk.row; s < wk.s1; s += wk.step) {
      Vec<T, V> q, e;
      q.load(x + s * a.x_ss);
      e.load(dy + s * a.dout_ss);
      float v[V], u[V];
#pragma unroll
      for (int k = 0; k < V; ++k) v[k] = q.get(k);
      if constexpr (DROP) wk.dropped(a, s, v);
#pragma unroll
      for (int k = 0; k < V; ++k) {
        v[k] = (v[k] - ch.mean[k]) * ch.rstd[k];
        u[k] = __builtin_fmaf(v[k], ch.w[k], ch.b[k]);
      }
      slope_all<T, V>(a.act, u);
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const float du = e.get(k) * u[k];
        dw[k] = __builtin_fmaf(du, v[k], dw[k]);
        db[k] += du;
      }
    }
    float* p = red + wk.row * width + wk.c - wk.base;
#pragma unroll
    for (int k = 0; k < V; ++k)
      if (k >= wk.shift) {
        p[k] = dw[k];
        p[wk.step * width + k] = db[k];
      }
  }
  __syncthreads();
  float* out = a.part + (int64_t)blockIdx.x * 2 * a.C + wk.base;
  for (int q = threadIdx.x; q < wk.local; q += 256) {
    float dw = 0.0f, db = 0.0f;
    for (int r = 0; r < wk.step; ++r) {
      dw += red[r * width + q];
      db += red[(wk.step + r) * width + q];
    }
    out[q] = dw;
    out[a.C + q] = db;
  }
}

// means of d = du w and of d xhat over one group
__global__ __launch_bounds__(256) void k_norm_grad_join(NormArgs a) {
  __shared__ float sh[2][4];
  const int i = blockIdx.x / a.G, g = blockIdx.x - i * a.G;
  const float* p = a.part + (int64_t)i * a.chunks * 2 * a.C + g * a.Cg;
  float s1 = 0.0f, s2 = 0.0f;
  for (int64_t e = threadIdx.x; e < (int64_t)a.chunks * a.Cg; e += blockDim.x) {
    const int chunk = (int)(e / a.Cg), c = (int)(e - (int64_t)chunk * a.Cg);
    const float w = a.w ? a.w[g * a.Cg + c] : 1.0f;
    s2 = __builtin_fmaf(w, p[(int64_t)chunk * 2 * a.C + c], s2);
    s1 = __builtin_fmaf(w, p[((int64_t)chunk * 2 + 1) * a.C + c], s1);
  }
  s1 = team_sum(s1, 64);
  s2 = team_sum(s2, 64);
  const int wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) {
    sh[0][wave] = s1;
    sh[1][wave] = s2;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < (int)blockDim.x / 64; ++w) {
      s1 += sh[0][w];
      s2 += sh[1][w];
    }
    const float m = (float)a.S * (float)a.Cg;
    a.coef[2 * (int64_t)blockIdx.x] = s1 / m;
    a.coef[2 * (int64_t)blockIdx.x + 1] = s2 / m;
  }
}

template <class T, int V, bool DROP>
__global__ __launch_bounds__(256) void k_norm_grad_apply(NormArgs a) {
  const Walker<T, V> wk(a);
  if (!wk.on) return;
  const T *x = wk.in(a.x, a.x_sn), *dy = wk.in(a.dout, a.dout_sn);
  T* dx = const_cast<T*>(wk.in(a.dx, a.dx_sn));
  const ChannelValues<V> ch(a, wk.i, wk.c);
  float m1[V], m2[V];
#pragma unroll
  for (int k = 0; k < V; ++k) {
    const float* p = a.coef + 2 * ((int64_t)wk.i * a.G + (wk.c + k) / a.Cg);
    m1[k] = p[0];
    m2[k] = p[1];
  }
  for (int s = wk.s0 + wk.row; s < wk.s1; s += wk.step) {
    Vec<T, V> q, e;
    q.load(x + s * a.x_ss);
    e.load(dy + s * a.dout_ss);
    float v[V], u[V];
    uint32_t keep = 0;
    if constexpr (DROP) keep = keep_from<V>(a.drop, (uint32_t)((int64_t)wk.i * a.S + s), wk.c);
#pragma unroll
    for (int k = 0; k < V; ++k) {
      float xv = q.get(k);
      if constexpr (DROP) xv = keep >> k & 1u ? xv * a.drop.scale : 0.0f;
      v[k] = (xv - ch.mean[k]) * ch.rstd[k];
      u[k] = __builtin_fmaf(v[k], ch.w[k], ch.b[k]);
    }
    slope_all<T, V>(a.act, u);
#pragma unroll
    for (int k = 0; k < V; ++k) {
      v[k] = ch.rstd[k] * (e.get(k) * u[k] * ch.w[k] - m1[k] - v[k] * m2[k]);
      if constexpr (DROP) v[k] = keep >> k & 1u ? v[k] * a.drop.scale : 0.0f;
    }
    store_own<T, V>(dx + s * a.dx_ss, v, wk.shift, false);
  }
}

// dweight and dbias: the fixed-order sum of the partial rows [part_rows][2][S][C] (row r of S C: q = r / S, at q 2 S + r - q S = q S + r; S = 1 but in the rows
// form of one group over several positions); 16 channels x 64 row lanes per workgroup.
__global__ __launch_bounds__(1024) void k_norm_param_sum(NormArgs a, int S) {
  __shared__ float sh[64][17];
  const int col = threadIdx.x & 15, lane = threadIdx.x >> 4, c = blockIdx.x * 16 + col;
  float* out = blockIdx.y ? a.db : a.dw;
  if (!out) return;
  float s = 0.0f;
  if (c < a.C) {
    const float* p = a.part + blockIdx.y * (int64_t)S * a.C + c;
    const int64_t rows = (int64_t)a.part_rows * S;
#pragma unroll 8
    for (int64_t r = lane; r < rows; r += 64) {
      const int64_t q = S == 1 ? r : r / S;
      s += p[(q * S + r) * a.C];
    }
  }
  sh[lane][col] = s;
  __syncthreads();
  for (int d = 32; d; d >>= 1) {
    if (lane < d) sh[lane][col] += sh[lane + d][col];
    __syncthreads();
  }
  if (lane == 0 && c < a.C) out[c] = sh[0][col];
}

// ---------------------------------------------------------------------- dropout -------
struct DropoutArgs {
  const char *x, *add;
  char* y;
  int64_t x_sn, x_ss, add_sn, add_ss, y_sn, y_ss;
  int S, C, blocks;     // blocks of eight channels per row
  int64_t first, count; // blocks of the launch
  DropArgs drop;
};

// One Philox block's eight elements per thread.
template <class T>
__global__ __launch_bounds__(256) void k_dropout(DropoutArgs a) {
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (id >= a.count) return;
  const int64_t row = (a.first + id) / a.blocks;
  const int b = (int)((a.first + id) - row * a.blocks), c = 8 * b;
  const int64_t i = a.S == 1 ? row : row / a.S, s = row - i * a.S;
  const T* x = reinterpret_cast<const T*>(a.x) + i * a.x_sn + s * a.x_ss + c;
  const T* add = a.add ? reinterpret_cast<const T*>(a.add) + i * a.add_sn + s * a.add_ss + c : nullptr;
  T* y = reinterpret_cast<T*>(a.y) + i * a.y_sn + s * a.y_ss + c;
  constexpr int V = 16 / sizeof(T), NV = 8 / V;
  const int own = min(8, a.C - c);
  float v[8], z[8];
  if (own == 8) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      Vec<T, V> q;
      q.load(x + j * V);
#pragma unroll
      for (int k = 0; k < V; ++k) v[j * V + k] = q.get(k);
      if (add) {
        q.load(add + j * V);
#pragma unroll
        for (int k = 0; k < V; ++k) z[j * V + k] = q.get(k);
      }
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      v[k] = k < own ? (float)x[k] : 0.0f;
      z[k] = k < own && add ? (float)add[k] : 0.0f;
    }
  }
  const uint32_t keep = a.drop.drop ? keep_bits(a.drop, (uint32_t)row, b) : 255u;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    v[k] = keep >> k & 1u ? v[k] * a.drop.scale : 0.0f;
    if (add) v[k] += z[k];
  }
  if (own == 8) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      Vec<T, V> q;
      q.set(v + j * V);
      q.stream(y + j * V);
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < own) y[k] = to_elem<T>(v[k]);
  }
}

// -------------------------------------------------------------------- host side -------

static DropArgs drop_args(const auv_drop* d) {
  DropArgs D{};
  D.scale = 1.0f;
  if (d) {
    D.key0 = (uint32_t)d->seed;
    D.key1 = (uint32_t)(d->seed >> 32);
    D.step = d->step;
    D.tag = 3u | d->site << 8;
    D.row0 = d->row0;
    D.drop = d->drop;
    D.scale = 65536.0f / (float)(65536u - d->drop);
  }
  return D;
}

static int check_drop(const char* fn, const auv_drop* d, int64_t rows) {
  if (d->site >= (1u << 24)) return set_error(AUV_EINVAL, "%s: dropout site must be below 2^24", fn);
  if (d->drop >= 65536u) return set_error(AUV_EINVAL, "%s: dropout probability must be below 65536 / 65536", fn);
  if (rows + d->row0 > ((int64_t)1 << 32)) return set_error(AUV_EINVAL, "%s: row0 + n s exceeds 2^32", fn);
  return AUV_OK;
}

static int check_rows(const char* fn, const char* name, const auv_rows& r, int type, int n, int s, int c, bool output) {
  if (!r.p) return set_error(AUV_EINVAL, "%s: '%s' is NULL", fn, name);
  if (reinterpret_cast<uintptr_t>(r.p) & (type == AUV_BF16 ? 1u : 3u))
    return set_error(AUV_EINVAL, "%s: '%s' is not aligned to its elements", fn, name);
  const int64_t most = (int64_t)1 << 44;
  if (r.sn < 0 || r.ss < 0 || r.sn > most / n || r.ss > most / s)
    return set_error(AUV_EINVAL, "%s: '%s' has a negative stride or spans 2^44 elements or more", fn, name);
  if (output) {   // rows apart, and samples apart from rows (or the other way round)
    const int64_t row = c, inner = std::min(n > 1 ? r.sn : most, s > 1 ? r.ss : most);
    const bool by_s = s > 1 && (n == 1 || r.ss <= r.sn);
    const int64_t span = by_s ? r.ss * (s - 1) + row : (n > 1 ? r.sn * (n - 1) + row : row);
    const int64_t outer = by_s ? (n > 1 ? r.sn : most) : (s > 1 ? r.ss : most);
    if (inner < row || outer < span) return set_error(AUV_EINVAL, "%s: elements of '%s' share memory", fn, name);
  }
  return AUV_OK;
}

struct NormPlan {
  bool rows;         // rows form
  int V, NV, lanes, m, blocks;
  int tile, tiles, chunks, per;
  int64_t part_rows, width;   // partial rows of [2][width] floats (backward)
};

// General form: chunks of at least four passes of a workgroup, four workgroups per CU where S allows.
static int plan_general(const char* fn, const auv_norm* d, NormPlan& p) {
  // a workgroup per sample and group, whose threads a launch counts in 32 bits
  if ((int64_t)d->n * d->groups >= (1 << 24)) return set_error(AUV_EINVAL, "%s: n groups must be below 2^24", fn);
  const int full = d->type == AUV_BF16 ? 8 : 4;
  p.rows = false;
  p.V = d->c >= full ? full : 1;
  const int vecs = (d->c - 1) / p.V + 1;
  p.tile = std::min(vecs, 256);
  p.tiles = (vecs - 1) / p.tile + 1;
  const int step = 256 / p.tile;
  const int64_t want = ((int64_t)4 * compute_units() - 1) / ((int64_t)d->n * p.tiles) + 1;
  p.chunks = (int)std::max<int64_t>(1, std::min<int64_t>(want, (d->s - 1) / (4 * step) + 1));
  p.per = (d->s - 1) / p.chunks + 1;
  p.chunks = (d->s - 1) / p.per + 1;
  p.part_rows = (int64_t)d->n * p.chunks;
  p.width = d->c;
  return AUV_OK;
}

static bool plan_rows(const auv_norm* d, bool dense, bool backward, NormPlan& p) {
  const int full = d->type == AUV_BF16 ? 8 : 4;
  const int64_t m = (int64_t)d->s * (d->c / d->groups);
  if (m > 1024 || !(d->s == 1 || (d->groups == 1 && dense))) return false;
  p.rows = true;
  p.m = (int)m;
  p.V = p.m >= full ? full : 1;
  const int vecs = (p.m - 1) / p.V + 1;
  p.lanes = 1;
  while (p.lanes < 64 && p.lanes < vecs) p.lanes *= 2;
  p.NV = 1;
  while (p.NV * p.lanes < vecs) p.NV *= 2;
  const int per = 256 / p.lanes, unit = d->groups / std::gcd(d->groups, per);   // teams: a multiple of the groups
  const int64_t rows = (int64_t)d->n * d->groups;
  const int64_t most = (int64_t)compute_units() * (backward ? 4 : 8);
  if (unit > most) return false;
  const int64_t want = std::min((rows - 1) / per + 1, most);
  p.blocks = (int)(want < unit ? unit : want / unit * unit);
  p.part_rows = d->groups == 1 ? p.blocks : (int64_t)p.blocks * per / d->groups;
  p.width = d->groups == 1 ? p.m : d->c;
  return true;
}

static int64_t plan_bytes(const auv_norm* d, const NormPlan& p, bool backward) {
  if (p.rows) return backward ? p.part_rows * 2 * p.width * (int64_t)sizeof(float) : 0;
  const int64_t part = (p.part_rows * 2 * d->c * (int64_t)sizeof(float) + 15) / 16 * 16;
  return part + (backward ? 2 * (int64_t)sizeof(float) * d->n * d->groups : 0);
}

static int check_norm(const char* fn, const auv_norm* d) {
  if (!d) return set_error(AUV_EINVAL, "%s: NULL argument", fn);
  if (d->n < 1 || d->s < 1 || d->c < 1 || d->groups < 1) return set_error(AUV_EINVAL, "%s: n, s, c and groups must be >= 1", fn);
  if (d->c % d->groups) return set_error(AUV_EINVAL, "%s: %d groups do not divide %d channels", fn, d->groups, d->c);
  if (d->c > (1 << 20) || (int64_t)d->n * d->s > 0x7FFFFFFF || (int64_t)d->n * d->s * d->c > ((int64_t)1 << 40) ||
      (int64_t)d->n * d->groups > 0x7FFFFFFF)
    return set_error(AUV_EINVAL, "%s: sizes too large", fn);
  if (d->type != AUV_FP32 && d->type != AUV_BF16) return set_error(AUV_EINVAL, "%s: unknown type %d", fn, d->type);
  if (d->act < AUV_ACTIVATION_NONE || d->act > AUV_ACTIVATION_TANH)
    return set_error(AUV_EINVAL, "%s: unknown activation %d", fn, d->act);
  if (!(d->eps >= 0.0f) || !std::isfinite(d->eps)) return set_error(AUV_EINVAL, "%s: eps must be finite and >= 0", fn);
  const void* p[4] = {d->weight, d->bias, d->mean, d->rstd};
  for (const void* q : p)
    if (reinterpret_cast<uintptr_t>(q) & 3u) return set_error(AUV_EINVAL, "%s: a parameter or statistic is not 4-byte aligned", fn);
  if (d->drop)
    if (int rc = check_drop(fn, d->drop, (int64_t)d->n * d->s)) return rc;
  return AUV_OK;
}

static int64_t norm_bytes(const char* fn, const auv_norm* d, bool backward) {
  NormPlan p{};
  int64_t most = 0;
  const bool rows = plan_rows(d, true, backward, p);
  if (rows) most = plan_bytes(d, p, backward);
  if (!plan_rows(d, false, backward, p)) {
    if (plan_general(fn, d, p)) return rows ? most : -1;
    most = std::max(most, plan_bytes(d, p, backward));
  }
  return most;
}

static NormArgs norm_args(const auv_norm* d, const NormPlan& p) {
  NormArgs a{};
  a.x = static_cast<char*>(d->x.p);
  a.x_sn = d->x.sn;
  a.x_ss = d->x.ss;
  a.w = d->weight;
  a.b = d->bias;
  a.mean = d->mean;
  a.rstd = d->rstd;
  a.eps = d->eps;
  a.act = d->act;
  a.n = d->n;
  a.S = d->s;
  a.C = d->c;
  a.G = d->groups;
  a.Cg = d->c / d->groups;
  a.m = p.m;
  a.lanes = p.lanes;
  a.chunks = p.chunks;
  a.per = p.per;
  a.tile = p.tile;
  a.part_rows = (int)p.part_rows;
  a.drop = drop_args(d->drop);
  return a;
}

#define AUV_ROWS_KERNEL(KERN, D)                                                                             \
  (bf16 ? (p.V == 8 ? (p.NV == 1 ? (const void*)KERN<__bf16, 8, 1, D> : (const void*)KERN<__bf16, 8, 2, D>) \
                    : (const void*)KERN<__bf16, 1, 1, D>)                                                    \
        : (p.V == 4 ? (p.NV == 1   ? (const void*)KERN<float, 4, 1, D>                                       \
                       : p.NV == 2 ? (const void*)KERN<float, 4, 2, D>                                       \
                                   : (const void*)KERN<float, 4, 4, D>)                                      \
                    : (const void*)KERN<float, 1, 1, D>))
#define AUV_GENERAL_KERNEL(KERN, D)                                                              \
  (bf16 ? (p.V == 8 ? (const void*)KERN<__bf16, 8, D> : (const void*)KERN<__bf16, 1, D>)         \
        : (p.V == 4 ? (const void*)KERN<float, 4, D> : (const void*)KERN<float, 1, D>))
#define AUV_DROPPED(PICK, KERN) (drop ? PICK(KERN, true) : PICK(KERN, false))

}  // namespace auv

// ------------------------------------------------------------------ C interface ----
using namespace auv;

extern "C" {

int auv_dropout(const auv_drop* drop, int32_t type, int32_t n, int32_t s, int32_t c, const auv_rows* x,
                const auv_rows* add, const auv_rows* y, void* stream) {
  const char* fn = "auv_dropout";
  if (!drop || !x || !y) return set_error(AUV_EINVAL, "%s: NULL argument", fn);
  if (n < 1 || s < 1 || c < 1) return set_error(AUV_EINVAL, "%s: n, s and c must be >= 1", fn);
  if (c > (1 << 30)) return set_error(AUV_EINVAL, "%s: c exceeds 2^30", fn);
  if (type != AUV_FP32 && type != AUV_BF16) return set_error(AUV_EINVAL, "%s: unknown type %d", fn, type);
  if (int rc = check_drop(fn, drop, (int64_t)n * s)) return rc;
  if (int rc = check_rows(fn, "x", *x, type, n, s, c, false)) return rc;
  if (int rc = check_rows(fn, "y", *y, type, n, s, c, true)) return rc;
  const bool with = add && add->p;
  if (with)
    if (int rc = check_rows(fn, "add", *add, type, n, s, c, false)) return rc;
  auto other = [&](const auv_rows* r) { return r->p == y->p && ((n > 1 && r->sn != y->sn) || (s > 1 && r->ss != y->ss)); };
  if (other(x) || (with && other(add))) return set_error(AUV_EINVAL, "%s: 'y' is an input's memory with other strides", fn);
  DropoutArgs a{};
  a.x = static_cast<const char*>(x->p);
  a.x_sn = x->sn;
  a.x_ss = x->ss;
  if (with) {
    a.add = static_cast<const char*>(add->p);
    a.add_sn = add->sn;
    a.add_ss = add->ss;
  }
  a.y = static_cast<char*>(y->p);
  a.y_sn = y->sn;
  a.y_ss = y->ss;
  a.S = s;
  a.C = c;
  a.blocks = (c - 1) / 8 + 1;
  a.drop = drop_args(drop);
  const int64_t all = (int64_t)n * s * a.blocks, most = (int64_t)1 << 31;   // threads of a launch fit 32 bits
  for (a.first = 0; a.first < all; a.first += most) {
    a.count = std::min(all - a.first, most);
    void* args[1] = {&a};
    const void* k = type == AUV_BF16 ? (const void*)k_dropout<__bf16> : (const void*)k_dropout<float>;
    if (int rc = launch_kernel(fn, k, dim3((unsigned)((a.count - 1) / 256 + 1)), dim3(256), args, 0, (hipStream_t)stream))
      return rc;
  }
  return AUV_OK;
}

int64_t auv_norm_work_bytes(const auv_norm* d, int32_t backward) {
  if (check_norm("auv_norm_work_bytes", d)) return -1;
  return norm_bytes("auv_norm_work_bytes", d, backward != 0);
}

int auv_norm_forward(const auv_norm* d, const auv_rows* y, void* work, void* stream) {
  const char* fn = "auv_norm_forward";
  if (int rc = check_norm(fn, d)) return rc;
  if (!y || !d->mean || !d->rstd) return set_error(AUV_EINVAL, "%s: NULL argument", fn);
  if (int rc = check_rows(fn, "x", d->x, d->type, d->n, d->s, d->c, false)) return rc;
  if (int rc = check_rows(fn, "y", *y, d->type, d->n, d->s, d->c, true)) return rc;
  if (y->p == d->x.p) return set_error(AUV_EINVAL, "%s: 'y' is the memory of 'x'", fn);
  const bool bf16 = d->type == AUV_BF16, drop = d->drop && d->drop->drop;
  NormPlan p{};
  if (!plan_rows(d, d->x.ss == d->c && y->ss == d->c, false, p))
    if (int rc = plan_general(fn, d, p)) return rc;
  if (!p.rows && (!work || !aligned16(work)))
    return set_error(AUV_EINVAL, "%s: 'work' is NULL or not 16-byte aligned", fn);
  NormArgs a = norm_args(d, p);
  a.y = static_cast<char*>(y->p);
  a.y_sn = y->sn;
  a.y_ss = y->ss;
  a.part = static_cast<float*>(work);
  void* args[1] = {&a};
  hipStream_t s = (hipStream_t)stream;
  if (p.rows) return launch_kernel(fn, AUV_DROPPED(AUV_ROWS_KERNEL, k_norm_rows), dim3(p.blocks), dim3(256), args, 0, s);
  const dim3 grid((unsigned)p.part_rows, p.tiles);
  const size_t lds = 2 * sizeof(float) * (256 / p.tile) * p.tile * p.V;
  if (int rc = launch_kernel(fn, AUV_DROPPED(AUV_GENERAL_KERNEL, k_norm_stats), grid, dim3(256), args, lds, s)) return rc;
  const dim3 join((int64_t)p.chunks * a.Cg > 256 ? 256 : 64);
  if (int rc = launch_kernel(fn, (const void*)k_norm_stats_join, dim3(d->n * d->groups), join, args, 0, s)) return rc;
  return launch_kernel(fn, AUV_DROPPED(AUV_GENERAL_KERNEL, k_norm_apply), grid, dim3(256), args, 0, s);
}

int auv_norm_backward(const auv_norm* d, const auv_norm_grad* g, void* work, void* stream) {
  const char* fn = "auv_norm_backward";
  if (int rc = check_norm(fn, d)) return rc;
  if (!g || !d->mean || !d->rstd) return set_error(AUV_EINVAL, "%s: NULL argument", fn);
  if (int rc = check_rows(fn, "x", d->x, d->type, d->n, d->s, d->c, false)) return rc;
  if (int rc = check_rows(fn, "dout", g->dout, d->type, d->n, d->s, d->c, false)) return rc;
  if (int rc = check_rows(fn, "dx", g->dx, d->type, d->n, d->s, d->c, true)) return rc;
  if (g->dx.p == d->x.p || g->dx.p == g->dout.p) return set_error(AUV_EINVAL, "%s: 'dx' is an input's memory", fn);
  if ((reinterpret_cast<uintptr_t>(g->dweight) | reinterpret_cast<uintptr_t>(g->dbias)) & 3u)
    return set_error(AUV_EINVAL, "%s: 'dweight' or 'dbias' is not 4-byte aligned", fn);
  if (g->dweight && g->dweight == g->dbias) return set_error(AUV_EINVAL, "%s: 'dweight' and 'dbias' are the same memory", fn);
  if (!work || !aligned16(work)) return set_error(AUV_EINVAL, "%s: 'work' is NULL or not 16-byte aligned", fn);
  const bool bf16 = d->type == AUV_BF16, drop = d->drop && d->drop->drop, params = g->dweight || g->dbias;
  NormPlan p{};
  if (!plan_rows(d, d->x.ss == d->c && g->dout.ss == d->c && g->dx.ss == d->c, true, p))
    if (int rc = plan_general(fn, d, p)) return rc;
  NormArgs a = norm_args(d, p);
  a.dout = static_cast<char*>(g->dout.p);
  a.dout_sn = g->dout.sn;
  a.dout_ss = g->dout.ss;
  a.dx = static_cast<char*>(g->dx.p);
  a.dx_sn = g->dx.sn;
  a.dx_ss = g->dx.ss;
  a.dw = g->dweight;
  a.db = g->dbias;
  a.part = p.rows && !params ? nullptr : static_cast<float*>(work);
  int S = 1;   // positions within a partial row
  void* args[1] = {&a};
  hipStream_t s = (hipStream_t)stream;
  if (p.rows) {
    const size_t lds = d->groups == 1 && params ? 4 * 2 * sizeof(float) * p.m : 0;
    if (int rc = launch_kernel(fn, AUV_DROPPED(AUV_ROWS_KERNEL, k_norm_rows_grad), dim3(p.blocks), dim3(256), args, lds, s))
      return rc;
    if (d->groups == 1) S = d->s;
  } else {
    const dim3 grid((unsigned)p.part_rows, p.tiles);
    const size_t lds = 2 * sizeof(float) * (256 / p.tile) * p.tile * p.V;
    a.coef = a.part + (p.part_rows * 2 * d->c + 3) / 4 * 4;
    if (int rc = launch_kernel(fn, AUV_DROPPED(AUV_GENERAL_KERNEL, k_norm_grad_sums), grid, dim3(256), args, lds, s)) return rc;
    const dim3 join((int64_t)p.chunks * a.Cg > 256 ? 256 : 64);
    if (int rc = launch_kernel(fn, (const void*)k_norm_grad_join, dim3(d->n * d->groups), join, args, 0, s)) return rc;
    if (int rc = launch_kernel(fn, AUV_DROPPED(AUV_GENERAL_KERNEL, k_norm_grad_apply), grid, dim3(256), args, 0, s)) return rc;
  }
  if (!params) return AUV_OK;
  void* sum_args[2] = {&a, &S};
  return launch_kernel(fn, (const void*)k_norm_param_sum, dim3((d->c - 1) / 16 + 1, 2), dim3(1024), sum_args, 0, s);
}

}  // extern "C"
