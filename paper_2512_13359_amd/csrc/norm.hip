// Group norm with an activation, channels last, and its gradient (block and chunk forms, C interface;
// norm_rows.hip: the rows form).
//   xhat = (x - mean) rstd over the S positions and C / G channels of a group, u = w xhat + b, y = act(u)
//   du = dy act'(u), dw = sum du xhat, db = sum du, d = du w,
//   dx = rstd (d - mean(d) - xhat mean(d xhat)); with dropout both x and dx pass the mask.
#include <algorithm>
#include <cmath>
#include <numeric>

#include "norm.hpp"

namespace auv {

__device__ __forceinline__ int lanes_for(int n) {   // the least power of two that is n at least, 64 at most
  return n >= 64 ? 64 : n <= 1 ? 1 : 1 << (32 - __clz(n - 1));
}

// du for V elements: x's value after dropout in, xhat out
template <class T, int V>
__device__ __forceinline__ void grad_of(int act, const float* w, const float* b, const Vec<T, V>& e, const float* xh, float* du) {
#pragma unroll
  for (int k = 0; k < V; ++k) du[k] = __builtin_fmaf(xh[k], w[k], b[k]);
  slope_all<T, V>(act, du);
#pragma unroll
  for (int k = 0; k < V; ++k) du[k] *= e.get(k);
}

// ------------------------------------------------------------------- block form -------
// A workgroup holds `pack` samples at a time in registers, R vectors per thread: a thread keeps V channels and takes
// every step-th position of its sample.  Sums go from threads to columns (channels of a sample) to groups through LDS.
// Read and written once; bound by the chain of a pass (load, two sums of three barriers each, store) where samples are small:
// 30000 x 8 x 32 bf16 in 8 groups, forward 19 us (1.6 TB/s) and backward 34; 20000 x 2000 fp32 82 (3.9) and 119 (4.0).
template <class T, int V, int R> struct BlockTeam {
  bool on;
  int c, shift, p, row, q;   // channel, sample of the pass, first position, row of LDS

  __device__ __forceinline__ explicit BlockTeam(const NormArgs& a) {
    const int cv = threadIdx.x % a.tile;
    q = threadIdx.x / a.tile;
    on = q < a.pack * a.step;
    p = q / a.step;
    row = q - p * a.step;
    c = min(cv * V, a.C - V);
    shift = cv * V - c;
  }
};

// Sums over the positions of each sample's columns, a value per thread and channel in, columns [pack][C] in LDS out; a column is
// a channel, or (merged) a vector of channels of one group, [pack][C / V].  rows [pack step][columns of a sample] and
// parts [threads] are LDS scratch.
template <int V, class Team>
__device__ __forceinline__ void column_sums(const NormArgs& a, const Team& tm, const float* v, bool merged, float* rows, float* parts,
                                            float* cols) {
  const int C = merged ? a.tile : a.C, width = a.pack * C, threads = blockDim.x;
  float* own = (a.step == 1 ? cols : rows) + tm.q * C;
  if (tm.on) {
    if (merged) {
      float s = 0.0f;
#pragma unroll
      for (int k = 0; k < V; ++k) s += v[k];
      own[tm.c / V] = s;
    } else {
#pragma unroll
      for (int k = 0; k < V; ++k)
        if (k >= tm.shift) own[tm.c + k] = v[k];
    }
  }
  __syncthreads();
  if (a.step == 1) return;
  const int segs = min(a.step, threads / width);   // threads per column
  if (segs > 1) {
    const int t = threadIdx.x, seg = t / width, i = t - seg * width;
    if (seg < segs) {
      const int p = i / C;
      const float* from = rows + (p * a.step) * C + (i - p * C);
      float s = 0.0f;
      for (int r = seg; r < a.step; r += segs) s += from[r * C];
      parts[t] = s;
    }
    __syncthreads();
    for (int t2 = threadIdx.x; t2 < width; t2 += threads) {
      float s = 0.0f;
      for (int g = 0; g < segs; ++g) s += parts[g * width + t2];
      cols[t2] = s;
    }
  } else {
    for (int i = threadIdx.x; i < width; i += threads) {
      const int p = i / C;
      const float* from = rows + (p * a.step) * C + (i - p * C);
      float s = 0.0f;
      for (int r = 0; r < a.step; ++r) s += from[r * C];
      cols[i] = s;
    }
  }
  __syncthreads();
}

// Per group of each sample: done(sample of the pass, group, sum of the group's columns) by one lane; a barrier after it.
template <int V, class Done>
__device__ __forceinline__ void group_sums(const NormArgs& a, const float* cols, bool merged, Done done) {
  const int Cg = merged ? a.Cg / V : a.Cg, lanes = lanes_for(Cg), all = a.pack * a.G;
  for (int t = threadIdx.x; t / lanes < all; t += blockDim.x) {
    const int i = t / lanes, l = t & (lanes - 1);   // group i of the pass: Cg columns from i Cg on
    float s = 0.0f;
    for (int c = l; c < Cg; c += lanes) s += cols[i * Cg + c];
    s = team_sum(s, lanes);
    if (l == 0) done(i, s);
  }
  __syncthreads();
}

template <class T, int V, int R, bool DROP>
__global__ __launch_bounds__(512) void k_norm_block(NormArgs a) {
  if constexpr (DROP) a.drop.count();
  extern __shared__ float lds[];
  const BlockTeam<T, V, R> tm(a);
  const int width = a.pack * a.C, all = a.pack * a.G;
  const bool merged = a.Cg % V == 0;   // a thread's channels are of one group
  float *mean = lds, *rstd = mean + all, *cols = rstd + all, *parts = cols + width, *rows = parts + blockDim.x;
  float w[V], b[V];
  int g[V];
#pragma unroll
  for (int k = 0; k < V; ++k) {
    w[k] = a.w ? a.w[tm.c + k] : 1.0f;
    b[k] = a.b ? a.b[tm.c + k] : 0.0f;
    g[k] = tm.p * a.G + (tm.c + k) / a.Cg;
  }
  const float inv = 1.0f / ((float)a.S * (float)a.Cg);
  for (int64_t first = (int64_t)blockIdx.x * a.pack; first < a.n; first += (int64_t)gridDim.x * a.pack) {
    const int64_t i = first + tm.p;
    const bool live = tm.on && i < a.n;
    const T* x = reinterpret_cast<const T*>(a.x) + i * a.x_sn + tm.c;
    Vec<T, V> q[R];
    Draws<V> keep[R];
    float sum[V];
#pragma unroll
    for (int k = 0; k < V; ++k) sum[k] = 0.0f;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int s = tm.row + r * a.step;
      if (live && s < a.S) q[r].load(x + s * a.x_ss);
    }
    auto value = [&](int r, int k) {
      const float v = q[r].get(k);
      if constexpr (DROP) return keep[r].kept(a.drop, k) ? v * a.drop.scale : 0.0f;
      else return v;
    };
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int s = tm.row + r * a.step;
      if (live && s < a.S) {
        if constexpr (DROP) keep[r].draw(a.drop, (uint32_t)(i * a.S + s), tm.c);
#pragma unroll
        for (int k = 0; k < V; ++k) sum[k] += value(r, k);
      }
    }
    column_sums<V>(a, tm, sum, merged, rows, parts, cols);
    group_sums<V>(a, cols, merged, [&](int j, float s) { mean[j] = s * inv; });
    float m[V];
#pragma unroll
    for (int k = 0; k < V; ++k) {
      m[k] = tm.on ? mean[g[k]] : 0.0f;
      sum[k] = 0.0f;
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (live && tm.row + r * a.step < a.S) {
#pragma unroll
        for (int k = 0; k < V; ++k) {
          const float d = value(r, k) - m[k];
          sum[k] = __builtin_fmaf(d, d, sum[k]);
        }
      }
    column_sums<V>(a, tm, sum, merged, rows, parts, cols);
    group_sums<V>(a, cols, merged, [&](int j, float s) {
      const float f = rsqrt_of(__builtin_fmaf(s, inv, a.eps));
      rstd[j] = f;
      if (first * a.G + j < (int64_t)a.n * a.G) {
        a.mean[first * a.G + j] = mean[j];
        a.rstd[first * a.G + j] = f;
      }
    });
    if (live) {
      T* y = reinterpret_cast<T*>(a.y) + i * a.y_sn + tm.c;
      float f[V];
#pragma unroll
      for (int k = 0; k < V; ++k) f[k] = rstd[g[k]];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int s = tm.row + r * a.step;
        if (s < a.S) {
          float u[V];
#pragma unroll
          for (int k = 0; k < V; ++k) u[k] = __builtin_fmaf((value(r, k) - m[k]) * f[k], w[k], b[k]);
          act_all<T, V>(a.act, u);
          store_own<T, V>(y + s * a.y_ss, u, tm.shift, false);
        }
      }
    }
  }
}

// Merged: the V channels of a thread are of one group, whose values are held once.
template <class T, int V, int R, bool DROP, bool MERGED>
__global__ __launch_bounds__(512) void k_norm_block_grad(NormArgs a) {
  if constexpr (DROP) a.drop.count();
  extern __shared__ float lds[];
  constexpr int VG = MERGED ? 1 : V;   // groups of a thread
  const BlockTeam<T, V, R> tm(a);
  const int width = a.pack * a.C, all = a.pack * a.G;
  float *m1 = lds, *m2 = m1 + all, *cols = m2 + all, *parts = cols + width, *rows = parts + blockDim.x;
  float w[V], b[V], dw[V], db[V];
  int g[VG];
#pragma unroll
  for (int k = 0; k < V; ++k) {
    w[k] = a.w ? a.w[tm.c + k] : 1.0f;
    b[k] = a.b ? a.b[tm.c + k] : 0.0f;
    dw[k] = db[k] = 0.0f;
  }
#pragma unroll
  for (int k = 0; k < VG; ++k) g[k] = tm.p * a.G + (tm.c + k) / a.Cg;
  const float inv = 1.0f / ((float)a.S * (float)a.Cg);
  for (int64_t first = (int64_t)blockIdx.x * a.pack; first < a.n; first += (int64_t)gridDim.x * a.pack) {
    const int64_t i = first + tm.p;
    const bool live = tm.on && i < a.n;
    const T* x = reinterpret_cast<const T*>(a.x) + i * a.x_sn + tm.c;
    const T* dy = reinterpret_cast<const T*>(a.dout) + i * a.dout_sn + tm.c;
    Vec<T, V> q[R], e[R];
    Draws<V> keep[R];
    float mean[VG], rstd[VG], s1[V], s2[V];
#pragma unroll
    for (int k = 0; k < V; ++k) s1[k] = s2[k] = 0.0f;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int s = tm.row + r * a.step;
      if (live && s < a.S) {
        q[r].load(x + s * a.x_ss);
        e[r].load(dy + s * a.dout_ss);
      }
    }
#pragma unroll
    for (int k = 0; k < VG; ++k) {
      mean[k] = live ? a.mean[first * a.G + g[k]] : 0.0f;
      rstd[k] = live ? a.rstd[first * a.G + g[k]] : 0.0f;
    }
    // xhat and du; computed again for the result where there are several vectors to hold
    auto both = [&](int r, float* xh, float* du) {
#pragma unroll
      for (int k = 0; k < V; ++k) {
        float v = q[r].get(k);
        if constexpr (DROP) v = keep[r].kept(a.drop, k) ? v : 0.0f;
        xh[k] = __builtin_fmaf(v, a.drop.scale, -mean[MERGED ? 0 : k]) * rstd[MERGED ? 0 : k];
      }
      grad_of<T, V>(a.act, w, b, e[r], xh, du);
    };
    float xh[V], du[V];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int s = tm.row + r * a.step;
      if (live && s < a.S) {
        if constexpr (DROP) keep[r].draw(a.drop, (uint32_t)(i * a.S + s), tm.c);
        both(r, xh, du);
#pragma unroll
        for (int k = 0; k < V; ++k) {
          s1[k] += du[k];
          s2[k] = __builtin_fmaf(du[k], xh[k], s2[k]);
        }
      }
    }
#pragma unroll
    for (int k = 0; k < V; ++k) {
      db[k] += s1[k];
      dw[k] += s2[k];
      s1[k] *= w[k];
      s2[k] *= w[k];
    }
    column_sums<V>(a, tm, s1, MERGED, rows, parts, cols);
    group_sums<V>(a, cols, MERGED, [&](int j, float s) { m1[j] = s * inv; });
    column_sums<V>(a, tm, s2, MERGED, rows, parts, cols);
    group_sums<V>(a, cols, MERGED, [&](int j, float s) { m2[j] = s * inv; });
    if (live) {
      T* dx = reinterpret_cast<T*>(a.dx) + i * a.dx_sn + tm.c;
      float c1[VG], c2[VG];
#pragma unroll
      for (int k = 0; k < VG; ++k) {
        c1[k] = m1[g[k]];
        c2[k] = m2[g[k]];
      }
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int s = tm.row + r * a.step;
        if (s < a.S) {
          if constexpr (R > 1) both(r, xh, du);
#pragma unroll
          for (int k = 0; k < V; ++k) {
            const int kg = MERGED ? 0 : k;
            du[k] = rstd[kg] * a.drop.scale * (du[k] * w[k] - c1[kg] - xh[k] * c2[kg]);
            if constexpr (DROP) du[k] = keep[r].kept(a.drop, k) ? du[k] : 0.0f;
          }
          store_own<T, V>(dx + s * a.dx_ss, du, tm.shift, false);
        }
      }
    }
  }
  if (!a.part) return;
  // the workgroup's sums, [2][C]: over its samples as well
  for (int plane = 0; plane < 2; ++plane) {
    column_sums<V>(a, tm, plane ? db : dw, false, rows, parts, cols);
    for (int c = threadIdx.x; c < a.C; c += blockDim.x) {
      double s = 0.0;
      for (int p = 0; p < a.pack; ++p) s += (double)cols[p * a.C + c];
      a.part[((int64_t)blockIdx.x * 2 + plane) * a.C + c] = (float)s;
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------ chunk form -------
// A workgroup walks over a chunk of a sample's positions and a tile of its channels, a thread keeping V channels.  The
// first launch leaves every chunk's and tile's share of the statistics of the tile's groups, [n][chunk][tile][held]; the second
// joins a group's shares in its first instructions.  Bound by HBM and the second read: 32 x 4096 x 256 bf16 in 32 groups with SiLU, 15 us for the
// statistics (4.5 TB/s) and 26 for the rest (5.2); backward 70.  Samples of one position are far from it: 20000 rows of 4104 bf16
// channels 554 us forward (0.6 TB/s) and 1110 backward (0.4).
template <class T, int V> struct Walker {
  bool on;
  int i, chunk, c, shift, row, step, s0, s1;   // sample, chunk, channel, positions [s0, s1) from s0 + row on by `step`
  int base, local, g0, g1;                     // the tile's first channel, its channels, its first and last group

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
    g0 = base / a.Cg;
    g1 = (base + local - 1) / a.Cg;
    s0 = chunk * a.per;
    s1 = min(a.S, s0 + a.per);
  }
  __device__ __forceinline__ const T* in(const char* p, int64_t sn) const {
    return reinterpret_cast<const T*>(p) + i * sn + c;
  }
  // channels [lo, hi) of the tile, counted from its base, that belong to group g
  __device__ __forceinline__ void channels_of(const NormArgs& a, int g, int& lo, int& hi) const {
    lo = max(g * a.Cg - base, 0);
    hi = min((g + 1) * a.Cg - base, local);
  }
  __device__ __forceinline__ float2* share(const NormArgs& a) const {   // of this chunk and tile, from group g0 on
    return reinterpret_cast<float2*>(a.groups) + (((int64_t)i * a.chunks + chunk) * a.tiles + blockIdx.y) * a.held;
  }
  // f(lane, lanes, share of group g by chunk and tile, its positions and channels) for all of them, dealt out to `lanes` lanes
  template <class F> __device__ __forceinline__ void shares_of(const NormArgs& a, int g, int lane, int lanes, F f) const {
    const int wide = a.tile * V, t0 = g * a.Cg / wide, t1 = (g * a.Cg + a.Cg - 1) / wide, nt = t1 - t0 + 1;
    const float2* p = reinterpret_cast<const float2*>(a.groups) + ((int64_t)i * a.chunks * a.tiles + t0) * a.held;
    const int first = g - t0 * wide / a.Cg;   // its place in the tile it starts in; it is the first of the others
    for (int k = lane; k < a.chunks * nt; k += lanes) {
      const int ch = k / nt, t = k - ch * nt, c0 = (t0 + t) * wide;
      const int count = min((g + 1) * a.Cg, c0 + wide) - max(g * a.Cg, c0);
      f(p[((int64_t)ch * a.tiles + t) * a.held + (t ? 0 : first)], min(a.S, (ch + 1) * a.per) - ch * a.per, count);
    }
  }
  // whether this workgroup writes group g's statistics
  __device__ __forceinline__ bool writes(const NormArgs& a, int g) const { return chunk == 0 && g * a.Cg >= base; }
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

__device__ __forceinline__ void join_lanes(float& n, float& m, float& M, int lanes) {
  for (int d = 1; d < lanes; d <<= 1) {
    const float nb = __shfl_xor(n, d), mb = __shfl_xor(m, d), Mb = __shfl_xor(M, d);
    join_moments(n, m, M, nb, mb, Mb);
  }
}

// U positions at a time: their loads are in flight together.  The second launch walks the chunk back (BACK): what the
// first one read last is still in its XCD's L2, where the same workgroup of the same grid runs.
template <class T, int V, int U, bool BACK, class F>
__device__ __forceinline__ void walk(const Walker<T, V>& wk, const T* x, int64_t stride, F f) {
  const int mine = wk.s1 - wk.s0 > wk.row ? (wk.s1 - wk.s0 - wk.row - 1) / wk.step + 1 : 0;   // positions of the thread
  for (int n = 0; n < mine; n += U) {
    Vec<T, V> q[U];
    int s[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      s[u] = wk.s0 + wk.row + (BACK ? mine - 1 - n - u : n + u) * wk.step;
      if (n + u < mine) q[u].load(x + s[u] * stride);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (n + u < mine) f(s[u], q[u]);
  }
}
template <class T, int V, int U, bool BACK, class F>
__device__ __forceinline__ void walk(const Walker<T, V>& wk, const T* x, int64_t stride, const T* dy, int64_t dstride, F f) {
  const int mine = wk.s1 - wk.s0 > wk.row ? (wk.s1 - wk.s0 - wk.row - 1) / wk.step + 1 : 0;
  for (int n = 0; n < mine; n += U) {
    Vec<T, V> q[U], e[U];
    int s[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      s[u] = wk.s0 + wk.row + (BACK ? mine - 1 - n - u : n + u) * wk.step;
      if (n + u < mine) {
        q[u].load(x + s[u] * stride);
        e[u].load(dy + s[u] * dstride);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (n + u < mine) f(s[u], q[u], e[u]);
  }
}

template <class T, int V, bool DROP>
__global__ __launch_bounds__(256) void k_norm_stats(NormArgs a) {
  if constexpr (DROP) a.drop.count();
  extern __shared__ float red[];   // means and squares about them, [2][step][tile V]
  const Walker<T, V> wk(a);
  const int width = a.tile * V;
  float *means = red, *squares = red + wk.step * width;
  if (wk.on) {
    // sums about the thread's first value: a member of the set, so the subtraction below loses at
    // most the set's size in ulps
    float first[V], s1[V], s2[V];
#pragma unroll
    for (int k = 0; k < V; ++k) first[k] = s1[k] = s2[k] = 0.0f;
    int count = 0;
    walk<T, V, 4, false>(wk, wk.in(a.x, a.x_sn), a.x_ss, [&](int s, const Vec<T, V>& q) {
      float v[V];
#pragma unroll
      for (int k = 0; k < V; ++k) v[k] = q.get(k);
      if constexpr (DROP) {
        Draws<V> keep;
        keep.draw(a.drop, (uint32_t)((int64_t)wk.i * a.S + s), wk.c);
#pragma unroll
        for (int k = 0; k < V; ++k) v[k] = keep.kept(a.drop, k) ? v[k] * a.drop.scale : 0.0f;
      }
#pragma unroll
      for (int k = 0; k < V; ++k) {
        if (count == 0) first[k] = v[k];
        const float d = v[k] - first[k];
        s1[k] += d;
        s2[k] = __builtin_fmaf(d, d, s2[k]);
      }
      ++count;
    });
    const float inv = count ? 1.0f / (float)count : 0.0f;
    const int at = wk.row * width + wk.c - wk.base;
#pragma unroll
    for (int k = 0; k < V; ++k)
      if (k >= wk.shift) {
        means[at + k] = __builtin_fmaf(s1[k], inv, first[k]);
        squares[at + k] = fmaxf(__builtin_fmaf(-s1[k] * inv, s1[k], s2[k]), 0.0f);
      }
  }
  __syncthreads();
  // a group's mean, then its squares about it, over the tile's rows and channels of the group
  const int groups = wk.g1 - wk.g0 + 1, whole = (wk.s1 - wk.s0) / wk.step, rest = (wk.s1 - wk.s0) % wk.step;
  const int lanes = lanes_for(min(min(a.Cg, wk.local) * wk.step, groups >= 256 ? 1 : 256 / groups));
  for (int t = threadIdx.x; t / lanes < groups; t += 256) {
    const int g = wk.g0 + t / lanes, l = t & (lanes - 1);
    int lo, hi;
    wk.channels_of(a, g, lo, hi);
    const int wide = hi - lo, all = wide * wk.step;
    float s = 0.0f, M = 0.0f;
    for (int e = l; e < all; e += lanes) {
      const int r = e / wide, q = lo + e - r * wide;
      s = __builtin_fmaf((float)(whole + (r < rest)), means[r * width + q], s);
    }
    const float mean = team_sum(s, lanes) / ((float)(wk.s1 - wk.s0) * (float)wide);
    for (int e = l; e < all; e += lanes) {
      const int r = e / wide, q = lo + e - r * wide;
      const float d = means[r * width + q] - mean;
      M += __builtin_fmaf((float)(whole + (r < rest)) * d, d, squares[r * width + q]);
    }
    M = team_sum(M, lanes);
    if (l == 0) wk.share(a)[g - wk.g0] = make_float2(mean, M);
  }
}

// a thread's channels: weight and bias, and a value per group from LDS (indexed from the tile's first group)
template <int V> struct ChannelValues {
  float w[V], b[V];
  int g[V];
  __device__ __forceinline__ ChannelValues(const NormArgs& a, int c, int g0) {
#pragma unroll
    for (int k = 0; k < V; ++k) {
      g[k] = (c + k) / a.Cg - g0;
      w[k] = a.w ? a.w[c + k] : 1.0f;
      b[k] = a.b ? a.b[c + k] : 0.0f;
    }
  }
};

template <class T, int V, bool DROP>
__global__ __launch_bounds__(256) void k_norm_apply(NormArgs a) {
  if constexpr (DROP) a.drop.count();
  extern __shared__ float lds[];   // mean and rstd of the tile's groups
  const Walker<T, V> wk(a);
  const int groups = wk.g1 - wk.g0 + 1;
  float *gm = lds, *gr = lds + groups;
  const int lanes = lanes_for(min(a.chunks, 256 / min(groups, 256)));
  for (int t = threadIdx.x; wk.g0 + t / lanes <= wk.g1; t += 256) {
    const int g = wk.g0 + t / lanes, l = t & (lanes - 1);
    float n = 0.0f, mean = 0.0f, M = 0.0f;
    wk.shares_of(a, g, l, lanes, [&](float2 v, int positions, int channels) {
      join_moments(n, mean, M, (float)positions * (float)channels, v.x, v.y);
    });
    join_lanes(n, mean, M, lanes);
    if (l == 0) {
      const float rstd = rsqrt_of(M / n + a.eps);
      gm[g - wk.g0] = mean;
      gr[g - wk.g0] = rstd;
      if (wk.writes(a, g)) {
        a.mean[(int64_t)wk.i * a.G + g] = mean;
        a.rstd[(int64_t)wk.i * a.G + g] = rstd;
      }
    }
  }
  __syncthreads();
  if (!wk.on) return;
  T* y = const_cast<T*>(wk.in(a.y, a.y_sn));
  const ChannelValues<V> ch(a, wk.c, wk.g0);
  float mean[V], rstd[V];
#pragma unroll
  for (int k = 0; k < V; ++k) {   // a neighbour's channels before the tile's are not stored
    mean[k] = gm[max(ch.g[k], 0)];
    rstd[k] = gr[max(ch.g[k], 0)];
  }
  walk<T, V, 4, true>(wk, wk.in(a.x, a.x_sn), a.x_ss, [&](int s, const Vec<T, V>& q) {
    float v[V];
    Draws<V> keep;
    if constexpr (DROP) keep.draw(a.drop, (uint32_t)((int64_t)wk.i * a.S + s), wk.c);
#pragma unroll
    for (int k = 0; k < V; ++k) {
      v[k] = q.get(k);
      if constexpr (DROP) v[k] = keep.kept(a.drop, k) ? v[k] * a.drop.scale : 0.0f;
      v[k] = __builtin_fmaf((v[k] - mean[k]) * rstd[k], ch.w[k], ch.b[k]);
    }
    act_all<T, V>(a.act, v);
    store_own<T, V>(y + s * a.y_ss, v, wk.shift, false);
  });
}

// MANY: a workgroup takes every `slots`-th sample and keeps the sums of the parameters' gradients over them in registers, so that
// 65536 rows of 8192 bf16 channels leave 192 partial rows (13 MB), not one each.
template <class T, int V, bool DROP, bool MANY>
__global__ __launch_bounds__(256) void k_norm_grad_sums(NormArgs a) {
  if constexpr (DROP) a.drop.count();
  extern __shared__ float red[];   // [2][step][tile V], then sums in their first rows
  Walker<T, V> wk(a);
  const int width = a.tile * V;
  float *dws = red, *dbs = red + wk.step * width;
  float* out = a.part ? a.part + (int64_t)blockIdx.x * 2 * a.C + wk.base : nullptr;
  float all_w[V], all_b[V];
#pragma unroll
  for (int k = 0; k < V; ++k) all_w[k] = all_b[k] = 0.0f;
  auto put = [&](const float* dw, const float* db) {
    const int at = wk.row * width + wk.c - wk.base;
#pragma unroll
    for (int k = 0; k < V; ++k)
      if (k >= wk.shift) {
        dws[at + k] = dw[k];
        dbs[at + k] = db[k];
      }
  };
  // the rows' sums, f(channel of the tile, dw, db) for each by one lane
  auto sum_rows = [&](auto f) {
    const int per = lanes_for(min(wk.step, wk.local >= 256 ? 1 : 256 / wk.local));   // lanes per channel
    for (int t = threadIdx.x; t / per < wk.local; t += 256) {
      const int q = t / per, l = t & (per - 1);
      float dw = 0.0f, db = 0.0f;
      for (int r = l; r < wk.step; r += per) {
        dw += dws[r * width + q];
        db += dbs[r * width + q];
      }
      dw = team_sum(dw, per);
      db = team_sum(db, per);
      if (l == 0) f(q, dw, db);
    }
  };
  for (;;) {
    if (wk.on) {
      const ChannelValues<V> ch(a, wk.c, 0);
      float mean[V], rstd[V], dw[V], db[V];
#pragma unroll
      for (int k = 0; k < V; ++k) {
        mean[k] = a.mean[(int64_t)wk.i * a.G + ch.g[k]];
        rstd[k] = a.rstd[(int64_t)wk.i * a.G + ch.g[k]];
        dw[k] = db[k] = 0.0f;
      }
      walk<T, V, 2, false>(wk, wk.in(a.x, a.x_sn), a.x_ss, wk.in(a.dout, a.dout_sn), a.dout_ss, [&](int s, const Vec<T, V>& q, const Vec<T, V>& e) {
        float xh[V], du[V];
        Draws<V> keep;
        if constexpr (DROP) keep.draw(a.drop, (uint32_t)((int64_t)wk.i * a.S + s), wk.c);
#pragma unroll
        for (int k = 0; k < V; ++k) {
          float v = q.get(k);
          if constexpr (DROP) v = keep.kept(a.drop, k) ? v : 0.0f;
          xh[k] = __builtin_fmaf(v, a.drop.scale, -mean[k]) * rstd[k];
        }
        grad_of<T, V>(a.act, ch.w, ch.b, e, xh, du);
#pragma unroll
        for (int k = 0; k < V; ++k) {
          dw[k] = __builtin_fmaf(du[k], xh[k], dw[k]);
          db[k] += du[k];
        }
      });
      put(dw, db);
      if constexpr (MANY) {
#pragma unroll
        for (int k = 0; k < V; ++k) {
          all_w[k] += dw[k];
          all_b[k] += db[k];
        }
      }
    }
    __syncthreads();
    sum_rows([&](int q, float dw, float db) {   // row 0 of a channel is its team's own
      if (!MANY && out) {
        out[q] = dw;
        out[a.C + q] = db;
      }
      const float w = a.w ? a.w[wk.base + q] : 1.0f;
      dws[q] = dw * w;
      dbs[q] = db * w;
    });
    __syncthreads();
    const int lanes = lanes_for(min(a.Cg, wk.local));
    for (int t = threadIdx.x; wk.g0 + t / lanes <= wk.g1; t += 256) {
      const int g = wk.g0 + t / lanes, l = t & (lanes - 1);
      int lo, hi;
      wk.channels_of(a, g, lo, hi);
      float s1 = 0.0f, s2 = 0.0f;
      for (int q = lo + l; q < hi; q += lanes) {
        s1 += dbs[q];
        s2 += dws[q];
      }
      s1 = team_sum(s1, lanes);
      s2 = team_sum(s2, lanes);
      if (l == 0) wk.share(a)[g - wk.g0] = make_float2(s1, s2);
    }
    if constexpr (!MANY) return;
    wk.i += gridDim.x / a.chunks;
    if (wk.i >= a.n) break;
    __syncthreads();
  }
  if (!out) return;
  __syncthreads();
  if (wk.on) put(all_w, all_b);
  __syncthreads();
  sum_rows([&](int q, float dw, float db) {
    out[q] = dw;
    out[a.C + q] = db;
  });
}

template <class T, int V, bool DROP>
__global__ __launch_bounds__(256) void k_norm_grad_apply(NormArgs a) {
  if constexpr (DROP) a.drop.count();
  extern __shared__ float lds[];   // means of d and of d xhat of the tile's groups
  const Walker<T, V> wk(a);
  const int groups = wk.g1 - wk.g0 + 1;
  float *g1 = lds, *g2 = lds + groups;
  const float inv = 1.0f / ((float)a.S * (float)a.Cg);
  const int lanes = lanes_for(min(a.chunks, 256 / min(groups, 256)));
  for (int t = threadIdx.x; wk.g0 + t / lanes <= wk.g1; t += 256) {
    const int g = wk.g0 + t / lanes, l = t & (lanes - 1);
    float s1 = 0.0f, s2 = 0.0f;
    wk.shares_of(a, g, l, lanes, [&](float2 v, int, int) {
      s1 += v.x;
      s2 += v.y;
    });
    s1 = team_sum(s1, lanes);
    s2 = team_sum(s2, lanes);
    if (l == 0) {
      g1[g - wk.g0] = s1 * inv;
      g2[g - wk.g0] = s2 * inv;
    }
  }
  __syncthreads();
  if (!wk.on) return;
  T* dx = const_cast<T*>(wk.in(a.dx, a.dx_sn));
  const ChannelValues<V> ch(a, wk.c, wk.g0);
  float mean[V], rstd[V], m1[V], m2[V];
#pragma unroll
  for (int k = 0; k < V; ++k) {   // a neighbour's channels before the tile's are not stored
    const int64_t g = (int64_t)wk.i * a.G + wk.g0 + ch.g[k];
    mean[k] = a.mean[g];
    rstd[k] = a.rstd[g];
    m1[k] = g1[max(ch.g[k], 0)];
    m2[k] = g2[max(ch.g[k], 0)];
  }
  walk<T, V, 2, true>(wk, wk.in(a.x, a.x_sn), a.x_ss, wk.in(a.dout, a.dout_sn), a.dout_ss, [&](int s, const Vec<T, V>& q, const Vec<T, V>& e) {
    float xh[V], du[V];
    Draws<V> keep;
    if constexpr (DROP) keep.draw(a.drop, (uint32_t)((int64_t)wk.i * a.S + s), wk.c);
#pragma unroll
    for (int k = 0; k < V; ++k) {
      float v = q.get(k);
      if constexpr (DROP) v = keep.kept(a.drop, k) ? v : 0.0f;
      xh[k] = __builtin_fmaf(v, a.drop.scale, -mean[k]) * rstd[k];
    }
    grad_of<T, V>(a.act, ch.w, ch.b, e, xh, du);
#pragma unroll
    for (int k = 0; k < V; ++k) {
      du[k] = rstd[k] * a.drop.scale * (du[k] * ch.w[k] - m1[k] - xh[k] * m2[k]);
      if constexpr (DROP) du[k] = keep.kept(a.drop, k) ? du[k] : 0.0f;
    }
    store_own<T, V>(dx + s * a.dx_ss, du, wk.shift, false);
  });
}

// dweight and dbias: the fixed-order sum of the partial rows [part_rows][2][C], in 64 bits (a chain of additions in 32 would
// cost the sums of many rows a digit); 16 channels x 64 row lanes per workgroup.
__global__ __launch_bounds__(1024) void k_norm_param_sum(NormArgs a) {
  __shared__ double sh[64][17];
  const int col = threadIdx.x & 15, lane = threadIdx.x >> 4, c = blockIdx.x * 16 + col;
  float* out = blockIdx.y ? a.db : a.dw;
  if (!out) return;
  double s = 0.0;
  if (c < a.C) {
    const float* p = a.part + (int64_t)blockIdx.y * a.C + c;
#pragma unroll 8
    for (int r = lane; r < a.part_rows; r += 64) s += (double)p[(int64_t)r * 2 * a.C];
  }
  sh[lane][col] = s;
  __syncthreads();
  for (int d = 32; d; d >>= 1) {
    if (lane < d) sh[lane][col] += sh[lane + d][col];
    __syncthreads();
  }
  if (lane == 0 && c < a.C) out[c] = (float)sh[0][col];
}

// -------------------------------------------------------------------- host side -------

// Workgroups per CU, each for many rows: 262144 x 256 bf16 with SiLU (and dropout), forward 8 per CU 58 us (62), 2 65 (81), 32 77
// (79); backward 3 per CU 89 (91), 2 87 (97), 8 91 (95).
static bool plan_rows(const auv_norm* d, bool dense, bool backward, NormPlan& p) {
  const int full = d->type == AUV_BF16 ? 8 : 4;
  const int64_t m = (int64_t)d->s * (d->c / d->groups);
  if (m > 1024 || !(d->s == 1 || (d->groups == 1 && dense))) return false;
  p.form = NORM_ROWS;
  p.m = (int)m;
  p.V = p.m >= full ? full : 1;
  const int vecs = (p.m - 1) / p.V + 1;
  p.lanes = 1;
  while (p.lanes < 64 && p.lanes < vecs) p.lanes *= 2;
  p.R = 1;
  while (p.R * p.lanes < vecs) p.R *= 2;
  const int per = 256 / p.lanes, unit = d->groups / std::gcd(d->groups, per);   // teams: a multiple of the groups
  const int64_t rows = (int64_t)d->n * d->groups;
  const int64_t most = (int64_t)compute_units() * (backward ? 3 : 8);   // workgroups, see below
  if (unit > most) return false;
  const int64_t want = std::min((rows - 1) / per + 1, most);
  p.blocks = (int)(want < unit ? unit : want / unit * unit);
  p.part_rows = d->groups <= per ? p.blocks : (int64_t)p.blocks * per / d->groups;
  return true;
}

// Up to four vectors per thread of at most 256, or 512; several samples per workgroup where one leaves threads idle.
static bool plan_block(const auv_norm* d, NormPlan& p) {
  const int full = d->type == AUV_BF16 ? 8 : 4;
  p.form = NORM_BLOCK;
  p.V = d->c >= full ? full : 1;
  const int64_t vecs = (d->c - 1) / p.V + 1, all = vecs * d->s;
  if (vecs > 512 || all > 4 * 512) return false;
  p.tile = (int)vecs;
  p.tiles = 1;
  p.pack = (int)std::min<int64_t>(d->n, std::max<int64_t>(1, 256 / all));
  bool fits = false;
  for (int most = 256; most <= 512 && !fits; most *= 2)
    for (p.R = 1; p.R <= 4; p.R *= 2)
      if ((fits = p.tile * ((d->s - 1) / p.R + 1) <= most)) break;
  if (!fits) return false;
  p.step = (d->s - 1) / p.R + 1;
  p.threads = (p.pack * p.step * p.tile + 63) / 64 * 64;
  // 24 waves per CU at most (262144 x 8 x 3 bf16 in 3 groups, forward: 43 us, 32 waves 55, 16 58); launch_block takes as many
  // of them as are resident
  p.blocks = (int)std::min<int64_t>((d->n - 1) / p.pack + 1, (int64_t)compute_units() * (1536 / p.threads));
  p.part_rows = p.blocks;
  return true;
}

#define AUV_NORM_TYPES(KERN, ...)                                                                               \
  (bf16 ? (p.V == 8 ? (const void*)KERN<__bf16, 8, __VA_ARGS__> : (const void*)KERN<__bf16, 1, __VA_ARGS__>) \
        : (p.V == 4 ? (const void*)KERN<float, 4, __VA_ARGS__> : (const void*)KERN<float, 1, __VA_ARGS__>))
#define AUV_SUMS_KERNEL(MANY) (drop ? AUV_NORM_TYPES(k_norm_grad_sums, true, MANY) : AUV_NORM_TYPES(k_norm_grad_sums, false, MANY))
#define AUV_CHUNK_KERNEL(KERN) (drop ? AUV_NORM_TYPES(KERN, true) : AUV_NORM_TYPES(KERN, false))
#define AUV_BLOCK_GRAD(R, D) (merged ? AUV_NORM_TYPES(k_norm_block_grad, R, D, true) : AUV_NORM_TYPES(k_norm_block_grad, R, D, false))
#define AUV_BLOCK_GRAD_DROP(R) (drop ? AUV_BLOCK_GRAD(R, true) : AUV_BLOCK_GRAD(R, false))
#define AUV_BLOCK_DROP(KERN, R) (drop ? AUV_NORM_TYPES(KERN, R, true) : AUV_NORM_TYPES(KERN, R, false))
#define AUV_BLOCK_KERNEL(KERN) \
  (p.R == 1 ? AUV_BLOCK_DROP(KERN, 1) : p.R == 2 ? AUV_BLOCK_DROP(KERN, 2) : AUV_BLOCK_DROP(KERN, 4))

static size_t block_lds(const auv_norm* d, const NormPlan& p) {   // see the kernels: groups, columns, parts, rows
  const size_t cols = (size_t)p.pack * d->c;
  return sizeof(float) * (2 * (size_t)p.pack * d->groups + cols + p.threads + (p.step > 1 ? cols * p.step : 0));
}

// The block form's launch, by workgroups that are all resident: each keeps weights and sums over its samples, and one more
// round of a few would last as long as all others (11803 x 8 x 160 fp32 in 32 groups, tanh and dropout, backward: 12 waves per CU,
// which the registers hold, 79 us, 16 109, 8 97).
static int launch_block(const char* fn, const auv_norm* d, NormPlan& p, NormArgs& a, bool grad, hipStream_t s) {
  const bool bf16 = d->type == AUV_BF16, drop = d->drop && d->drop->drop, merged = a.Cg % p.V == 0;
  const void* k = !grad ? AUV_BLOCK_KERNEL(k_norm_block)
                  : p.R == 1 ? AUV_BLOCK_GRAD_DROP(1) : p.R == 2 ? AUV_BLOCK_GRAD_DROP(2) : AUV_BLOCK_GRAD_DROP(4);
  const size_t lds = block_lds(d, p);
  if (p.blocks > compute_units()) {
    int resident = 0;
    if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&resident, k, p.threads, lds) != hipSuccess || resident < 1) {
      (void)hipGetLastError();
      resident = 1;
    }
    p.blocks = std::min(p.blocks, compute_units() * resident);
    p.part_rows = a.part_rows = p.blocks;
  }
  void* args[1] = {&a};
  return launch_kernel(fn, k, dim3(p.blocks), dim3(p.threads), args, lds, s);
}

// Chunks of at least four passes of a workgroup, two workgroups per CU where the positions allow (4 x 8192 x 512 bf16 in 32
// groups, forward and backward: two per CU 31 and 50 us, four 39 and 61, one pass per chunk more still).
static int plan_chunks(const char* fn, const auv_norm* d, NormPlan& p) {
  // a workgroup per sample at least, whose threads a launch counts in 32 bits
  if (d->n >= (1 << 24)) return set_error(AUV_EINVAL, "%s: n must be below 2^24 for samples of this size", fn);
  const int full = d->type == AUV_BF16 ? 8 : 4;
  p.form = NORM_CHUNKS;
  p.V = d->c >= full ? full : 1;
  const int vecs = (d->c - 1) / p.V + 1;
  p.tile = std::min(vecs, 256);
  p.tiles = (vecs - 1) / p.tile + 1;
  const int step = 256 / p.tile;
  const int64_t want = ((int64_t)2 * compute_units() - 1) / ((int64_t)d->n * p.tiles) + 1;
  p.chunks = (int)std::max<int64_t>(1, std::min<int64_t>(want, (d->s - 1) / (4 * step) + 1));
  p.per = (d->s - 1) / p.chunks + 1;
  p.chunks = (d->s - 1) / p.per + 1;
  // Partial sums of the parameters' gradients: one row per chunk where that is little beside it (32 positions: an eighth of the
  // tensor at most), else as many as workgroups are resident (three per CU), each over several samples.
  const int64_t resident = std::max<int64_t>(1, (int64_t)3 * compute_units() / ((int64_t)p.tiles * p.chunks));
  p.part_rows = p.chunks * (p.per >= 32 ? (int64_t)d->n : std::min<int64_t>(d->n, resident));
  return AUV_OK;
}

static int plan(const char* fn, const auv_norm* d, bool dense, bool backward, NormPlan& p) {
  p = NormPlan{};
  if (plan_rows(d, dense, backward, p) || plan_block(d, p)) return AUV_OK;
  return plan_chunks(fn, d, p);
}

// groups that a tile of channels can hold a part of
static int tile_groups(const auv_norm* d, const NormPlan& p) {
  const int wide = std::min(p.tile * p.V, d->c), cg = d->c / d->groups;
  return std::min(d->groups, (wide - 1) / cg + 2);
}

static int64_t part_floats(const NormPlan& p, int64_t c, bool backward) {
  return backward ? (p.part_rows * 2 * c + 3) / 4 * 4 : 0;
}

static int64_t plan_bytes(const auv_norm* d, const NormPlan& p, bool backward) {
  const int64_t shares = p.form == NORM_CHUNKS ? (int64_t)d->n * p.chunks * p.tiles * tile_groups(d, p) * 2 : 0;
  return (part_floats(p, d->c, backward) + shares) * (int64_t)sizeof(float);
}

static int check_norm(const char* fn, const auv_norm* d) {
  if (!d) return set_error(AUV_EINVAL, "%s: NULL argument", fn);
  if (d->n < 1 || d->s < 1 || d->c < 1 || d->groups < 1) return set_error(AUV_EINVAL, "%s: n, s, c and groups must be >= 1", fn);
  if (d->c % d->groups) return set_error(AUV_EINVAL, "%s: %d groups do not divide %d channels", fn, d->groups, d->c);
  if (d->c > (1 << 20) || (int64_t)d->n * d->s > 0x7FFF0000 || (int64_t)d->n * d->s * d->c > ((int64_t)1 << 40) ||
      (int64_t)d->n * d->groups > 0x7FFF0000)
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

// What either kind of strides needs (dense ones may take the rows form).
static int64_t norm_bytes(const char* fn, const auv_norm* d, bool backward) {
  NormPlan p{};
  if (plan(fn, d, true, backward, p)) return -1;
  const int64_t dense = plan_bytes(d, p, backward);
  if (plan(fn, d, false, backward, p)) return -1;
  return std::max(dense, plan_bytes(d, p, backward));
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
  a.tile = p.tile;
  a.tiles = p.tiles;
  a.step = p.step;
  a.pack = p.pack;
  a.chunks = p.chunks;
  a.per = p.per;
  a.held = p.form == NORM_CHUNKS ? tile_groups(d, p) : 0;
  a.part_rows = (int)p.part_rows;
  a.drop = drop_args(d->drop);
  return a;
}

}  // namespace auv

// ------------------------------------------------------------------ C interface ----
using namespace auv;

extern "C" {

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
  if (int rc = check_apart(fn, {{"y", y->p}, {"mean", d->mean}, {"rstd", d->rstd}}, {{"x", d->x.p}, {"weight", d->weight}, {"bias", d->bias}}))
    return rc;
  const bool bf16 = d->type == AUV_BF16, drop = d->drop && d->drop->drop;
  NormPlan p{};
  if (int rc = plan(fn, d, d->x.ss == d->c && y->ss == d->c, false, p)) return rc;
  if (p.form == NORM_CHUNKS && (!work || !aligned16(work)))
    return set_error(AUV_EINVAL, "%s: 'work' is NULL or not 16-byte aligned", fn);
  NormArgs a = norm_args(d, p);
  a.y = static_cast<char*>(y->p);
  a.y_sn = y->sn;
  a.y_ss = y->ss;
  a.groups = static_cast<float*>(work);
  void* args[1] = {&a};
  hipStream_t s = (hipStream_t)stream;
  if (p.form == NORM_ROWS) return launch_norm_rows(fn, a, p, bf16, false, 0, s);
  if (p.form == NORM_BLOCK) return launch_block(fn, d, p, a, false, s);
  const dim3 grid((unsigned)(d->n * p.chunks), p.tiles);
  const size_t lds = 2 * sizeof(float) * (256 / p.tile) * p.tile * p.V;
  if (int rc = launch_kernel(fn, AUV_CHUNK_KERNEL(k_norm_stats), grid, dim3(256), args, lds, s)) return rc;
  return launch_kernel(fn, AUV_CHUNK_KERNEL(k_norm_apply), grid, dim3(256), args, 2 * sizeof(float) * a.held, s);
}

int auv_norm_backward(const auv_norm* d, const auv_norm_grad* g, void* work, void* stream) {
  const char* fn = "auv_norm_backward";
  if (int rc = check_norm(fn, d)) return rc;
  if (!g || !d->mean || !d->rstd) return set_error(AUV_EINVAL, "%s: NULL argument", fn);
  if (int rc = check_rows(fn, "x", d->x, d->type, d->n, d->s, d->c, false)) return rc;
  if (int rc = check_rows(fn, "dout", g->dout, d->type, d->n, d->s, d->c, false)) return rc;
  if (int rc = check_rows(fn, "dx", g->dx, d->type, d->n, d->s, d->c, true)) return rc;
  if ((reinterpret_cast<uintptr_t>(g->dweight) | reinterpret_cast<uintptr_t>(g->dbias)) & 3u)
    return set_error(AUV_EINVAL, "%s: 'dweight' or 'dbias' is not 4-byte aligned", fn);
  if (int rc = check_apart(fn, {{"dx", g->dx.p}, {"dweight", g->dweight}, {"dbias", g->dbias}},
                           {{"x", d->x.p}, {"dout", g->dout.p}, {"weight", d->weight}, {"bias", d->bias}, {"mean", d->mean}, {"rstd", d->rstd}}))
    return rc;
  if (!work || !aligned16(work)) return set_error(AUV_EINVAL, "%s: 'work' is NULL or not 16-byte aligned", fn);
  const bool bf16 = d->type == AUV_BF16, drop = d->drop && d->drop->drop, params = g->dweight || g->dbias;
  NormPlan p{};
  if (int rc = plan(fn, d, d->x.ss == d->c && g->dout.ss == d->c && g->dx.ss == d->c, true, p)) return rc;
  NormArgs a = norm_args(d, p);
  a.dout = static_cast<char*>(g->dout.p);
  a.dout_sn = g->dout.sn;
  a.dout_ss = g->dout.ss;
  a.dx = static_cast<char*>(g->dx.p);
  a.dx_sn = g->dx.sn;
  a.dx_ss = g->dx.ss;
  a.dw = g->dweight;
  a.db = g->dbias;
  a.part = params ? static_cast<float*>(work) : nullptr;
  void* args[1] = {&a};
  hipStream_t s = (hipStream_t)stream;
  if (p.form == NORM_ROWS) {
    const int teams = 256 / p.lanes;
    const size_t lds = d->groups <= teams && params ? (size_t)teams * 2 * p.m * sizeof(float) : 0;
    if (int rc = launch_norm_rows(fn, a, p, bf16, true, lds, s)) return rc;
  } else if (p.form == NORM_BLOCK) {
    if (int rc = launch_block(fn, d, p, a, true, s)) return rc;
  } else {
    const dim3 sums((unsigned)p.part_rows, p.tiles), grid((unsigned)(d->n * p.chunks), p.tiles);
    const size_t lds = 2 * sizeof(float) * (256 / p.tile) * p.tile * p.V;
    a.groups = static_cast<float*>(work) + part_floats(p, d->c, true);
    const void* k = sums.x < grid.x ? AUV_SUMS_KERNEL(true) : AUV_SUMS_KERNEL(false);
    if (int rc = launch_kernel(fn, k, sums, dim3(256), args, lds, s)) return rc;
    if (int rc = launch_kernel(fn, AUV_CHUNK_KERNEL(k_norm_grad_apply), grid, dim3(256), args, 2 * sizeof(float) * a.held, s))
      return rc;
  }
  if (!params) return AUV_OK;
  return launch_kernel(fn, (const void*)k_norm_param_sum, dim3((d->c - 1) / 16 + 1, 2), dim3(1024), args, 0, s);
}

}  // extern "C"
