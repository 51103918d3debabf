// Dropout from the counter-based generator (kernel and C interface): y = x or 0 by the element's draw, scaled,
// plus another tensor where given.
#include <algorithm>

#include "dropout.hpp"
#include "layers.hpp"

namespace auv {

struct DropoutArgs {
  const char *x, *add;
  char* y;
  int64_t x_sn, x_ss, add_sn, add_ss, y_sn, y_ss;
  int S, C, blocks;     // blocks of eight channels per row
  uint32_t first;       // first row of the launch
  int64_t count;        // blocks of the launch
  DropArgs drop;
};

// One Philox block's eight elements per thread.  Bound by HBM: 524288 x 256 bf16 into a residual in 134 us (6.0 TB/s; among
// other kernels 142), 100003 x 257 fp32 out of wider rows in 39 (5.2; 36).
// In place (y = x or add): a thread reads its own elements only, before it writes them.
template <class T>
__global__ __launch_bounds__(256) void k_dropout(DropoutArgs a) {
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (id >= a.count) return;
  // a launch covers whole rows and fewer than 2^32 blocks
  const uint32_t up = (uint32_t)id / (uint32_t)a.blocks;
  const int b = (int)((uint32_t)id - up * (uint32_t)a.blocks), c = 8 * b;
  const uint32_t row = a.first + up;
  const int64_t i = a.S == 1 ? row : row / (uint32_t)a.S, s = row - i * a.S;
  const T* x = reinterpret_cast<const T*>(a.x) + i * a.x_sn + s * a.x_ss + c;
  const T* add = a.add ? reinterpret_cast<const T*>(a.add) + i * a.add_sn + s * a.add_ss + c : nullptr;
  T* y = reinterpret_cast<T*>(a.y) + i * a.y_sn + s * a.y_ss + c;
  constexpr int V = 16 / sizeof(T), NV = 8 / V;
  const int own = min(8, a.C - c);
  float v[8], z[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) v[k] = z[k] = 0.0f;
  if (own == 8) {
    Vec<T, V> q[NV], e[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) q[j].load(x + j * V);
    if (add) {
#pragma unroll
      for (int j = 0; j < NV; ++j) e[j].load(add + j * V);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      v[k] = q[k / V].get(k % V);
      if (add) z[k] = e[k / V].get(k % V);
    }
  } else {
    // every load from the row's end on is of its last element: loads without a branch, all in flight at once
    const int last = own - 1;
    Vec<T, 1> q[8], e[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) q[k].load(x + min(k, last));
    if (add) {
#pragma unroll
      for (int k = 0; k < 8; ++k) e[k].load(add + min(k, last));
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      v[k] = q[k].get(0);
      if (add) z[k] = e[k].get(0);
    }
  }
  if (a.drop.drop) {
    a.drop.count();
    Draws<8> keep;
    keep.draw(a.drop, row, c);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = keep.kept(a.drop, k) ? v[k] * a.drop.scale : 0.0f;
  }
  if (add) {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] += z[k];
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

DropArgs drop_args(const auv_drop* d) {
  DropArgs D{};
  D.scale = 1.0f;
  if (d) {
    D.key0 = (uint32_t)d->seed;
    D.key1 = (uint32_t)(d->seed >> 32);
    D.step = d->step;
    D.tag = 3u | d->site << 8;
    D.row0 = d->row0;
    D.drop = d->drop;
    D.counter = d->counter;
    D.scale = 65536.0f / (float)(65536u - d->drop);
  }
  return D;
}

int check_drop(const char* fn, const auv_drop* d, int64_t rows) {
  if (d->site >= (1u << 24)) return set_error(AUV_EINVAL, "%s: dropout site must be below 2^24", fn);
  if (d->drop >= 65536u) return set_error(AUV_EINVAL, "%s: dropout probability must be below 65536 / 65536", fn);
  if (reinterpret_cast<uintptr_t>(d->counter) & 3u) return set_error(AUV_EINVAL, "%s: dropout's counter is not 4-byte aligned", fn);
  if (rows + d->row0 > ((int64_t)1 << 32)) return set_error(AUV_EINVAL, "%s: row0 + n s exceeds 2^32", fn);
  return AUV_OK;
}

int check_rows(const char* fn, const char* name, const auv_rows& r, int type, int n, int s, int c, bool output) {
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
  const int64_t rows = (int64_t)n * s, most = std::max<int64_t>(1, ((int64_t)1 << 31) / a.blocks);   // rows of a launch
  for (int64_t first = 0; first < rows; first += most) {
    a.first = (uint32_t)first;
    a.count = std::min(rows - first, most) * a.blocks;
    void* args[1] = {&a};
    const void* k = type == AUV_BF16 ? (const void*)k_dropout<__bf16> : (const void*)k_dropout<float>;
    if (int rc = launch_kernel(fn, k, dim3((unsigned)((a.count - 1) / 256 + 1)), dim3(256), args, 0, (hipStream_t)stream))
      return rc;
  }
  return AUV_OK;
}

}  // extern "C"
