// Group norm, rows form (kernels).
#include "norm.hpp"

namespace auv {

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
  // the draws of a row's vector j
  __device__ __forceinline__ void draw(const NormArgs& a, int64_t sample, int g, int j, Draws<V>& keep) const {
    if (a.S == 1) {
      keep.draw(a.drop, (uint32_t)sample, g * a.m + at[j]);
      return;
    }
    int pos = at[j] / a.C, c = at[j] % a.C;
    if (a.C % V == 0) {
      keep.draw(a.drop, (uint32_t)(sample * a.S + pos), c);
      return;
    }
    uint32_t bits = 0;   // the vector may go over several positions
    for (int k = 0; k < V;) {
      const int run = min(V - k, min(a.C - c, 8 - (c & 7)));
      bits |= (drop_bits(a.drop, (uint32_t)(sample * a.S + pos), c >> 3) >> (c & 7) & ((1u << run) - 1u)) << k;
      k += run;
      c += run;
      if (c == a.C) ++pos, c = 0;
    }
    keep.set(bits);
  }
};

// Bound by HBM, x in and y out: 262144 x 256 bf16 with SiLU and dropout in 70 us (3.8 TB/s) between backward passes, in 62 alone
// (without dropout 58, 4.7 TB/s): Philox's 18 quarter-rate products per eight elements fill the VALU beside it.
template <class T, int V, int NV, bool DROP, bool FULL>
__global__ __launch_bounds__(256) void k_norm_rows(NormArgs a) {
  if constexpr (DROP) a.drop.count();
  constexpr bool full = FULL;   // every lane's vectors are whole and its own
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
      // kept values enter unscaled: mean and deviations are scaled instead
      Draws<V> keep;
      if constexpr (DROP) tm.draw(a, sample, g, j, keep);
#pragma unroll
      for (int k = 0; k < V; ++k) {
        v[j][k] = q[j].get(k);
        if constexpr (DROP) v[j][k] = keep.kept(a.drop, k) ? v[j][k] : 0.0f;
      }
    }
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int k = 0; k < V; ++k) sum += full || k >= tm.shift[j] ? v[j][k] : 0.0f;
    const float mean = team_sum(sum, a.lanes) * inv;
    float ss = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int k = 0; k < V; ++k) {
        v[j][k] -= mean;
        const float d = full || k >= tm.shift[j] ? v[j][k] : 0.0f;
        ss = __builtin_fmaf(d, d, ss);
      }
    const float rstd = rsqrt_of(__builtin_fmaf(team_sum(ss, a.lanes), inv * a.drop.scale * a.drop.scale, a.eps));
    const float f = rstd * a.drop.scale;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int k = 0; k < V; ++k) v[j][k] = __builtin_fmaf(v[j][k] * f, w[j][k], b[j][k]);
    act_all<T, NV * V>(a.act, &v[0][0]);
#pragma unroll
    for (int j = 0; j < NV; ++j) store_own<T, V>(y + tm.at[j], v[j], full ? 0 : tm.shift[j], false);
    if (tm.lane == 0) {
      a.mean[r] = mean * a.drop.scale;
      a.rstd[r] = rstd;
    }
  }
}

// Bound by HBM, x and dy in and dx out: the same in 86 us (4.7 TB/s); alone with the parameters' sum 91 (without dropout 89).
template <class T, int V, int NV, bool DROP, bool FULL>
__global__ __launch_bounds__(256) void k_norm_rows_grad(NormArgs a) {
  if constexpr (DROP) a.drop.count();
  constexpr bool full = FULL;   // every lane's vectors are whole and its own
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
    Draws<V> keep[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if constexpr (DROP) tm.draw(a, sample, g, j, keep[j]);
#pragma unroll
      for (int k = 0; k < V; ++k) {
        float v = q[j].get(k);
        if constexpr (DROP) v = keep[j].kept(a.drop, k) ? v : 0.0f;
        xh[j][k] = __builtin_fmaf(v, a.drop.scale, -mean) * rstd;
        d[j][k] = __builtin_fmaf(xh[j][k], w[j][k], b[j][k]);
      }
    }
    slope_all<T, NV * V>(a.act, &d[0][0]);
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int k = 0; k < V; ++k) {
        float du = e[j].get(k) * d[j][k];
        if (!full && k < tm.shift[j]) du = 0.0f;
        dw[j][k] = __builtin_fmaf(du, xh[j][k], dw[j][k]);
        db[j][k] += du;
        d[j][k] = du * w[j][k];
        s1 += d[j][k];
        s2 = __builtin_fmaf(d[j][k], xh[j][k], s2);
      }
    team_sums(s1, s2, a.lanes);
    s1 *= inv;
    s2 *= inv;
    const float f = rstd * a.drop.scale;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float o[V];
#pragma unroll
      for (int k = 0; k < V; ++k) {
        o[k] = f * (d[j][k] - s1 - xh[j][k] * s2);
        if constexpr (DROP) o[k] = keep[j].kept(a.drop, k) ? o[k] : 0.0f;
      }
      store_own<T, V>(dx + tm.at[j], o, full ? 0 : tm.shift[j], false);
    }
  }
  if (!a.part) return;
  // [part row][2][C].  More groups than teams: a team's own sums, team t those of group t mod G; else the workgroup's,
  // summed over its teams of a group (and over positions) through LDS.
  if (a.G > per) {
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
  extern __shared__ float red[];   // [teams][2][m]
  float* own = red + tm.team * 2 * a.m;
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int k = 0; k < V; ++k)
      if (k >= tm.shift[j]) {
        own[tm.at[j] + k] = dw[j][k];
        own[a.m + tm.at[j] + k] = db[j][k];
      }
  __syncthreads();
  const int g0 = (int)((int64_t)blockIdx.x * per % a.G);   // the first team's group
  for (int i = threadIdx.x; i < 2 * a.C; i += 256) {
    const int plane = i >= a.C, c = i - plane * a.C;
    const int group = a.S == 1 ? c / a.m : 0, at = plane * a.m + (a.S == 1 ? c - group * a.m : c);
    double s = 0.0;
    for (int t = (group - g0 + a.G) % a.G; t < per; t += a.G)
      for (int pos = 0; pos < a.S; ++pos) s += (double)red[t * 2 * a.m + at + pos * a.C];
    a.part[(int64_t)blockIdx.x * 2 * a.C + i] = (float)s;
  }
}

#define AUV_ROWS_FULL(KERN, T, V, NV, D) (full ? (const void*)KERN<T, V, NV, D, true> : (const void*)KERN<T, V, NV, D, false>)
#define AUV_ROWS_KERNEL(KERN, D)                                                                    \
  (bf16 ? (p.V == 8 ? (p.R == 1 ? AUV_ROWS_FULL(KERN, __bf16, 8, 1, D) : AUV_ROWS_FULL(KERN, __bf16, 8, 2, D)) \
                    : (const void*)KERN<__bf16, 1, 1, D, false>)                                    \
        : (p.V == 4 ? (p.R == 1   ? AUV_ROWS_FULL(KERN, float, 4, 1, D)                             \
                       : p.R == 2 ? AUV_ROWS_FULL(KERN, float, 4, 2, D)                             \
                                  : AUV_ROWS_FULL(KERN, float, 4, 4, D))                            \
                    : (const void*)KERN<float, 1, 1, D, false>))

int launch_norm_rows(const char* fn, const NormArgs& a, const NormPlan& p, bool bf16, bool grad, size_t lds, hipStream_t s) {
  const bool drop = a.drop.drop, full = a.m == p.R * a.lanes * p.V;
  NormArgs arg = a;
  void* args[1] = {&arg};
  const void* k = grad ? (drop ? AUV_ROWS_KERNEL(k_norm_rows_grad, true) : AUV_ROWS_KERNEL(k_norm_rows_grad, false))
                       : (drop ? AUV_ROWS_KERNEL(k_norm_rows, true) : AUV_ROWS_KERNEL(k_norm_rows, false));
  return launch_kernel(fn, k, dim3(p.blocks), dim3(256), args, lds, s);
}

}  // namespace auv
