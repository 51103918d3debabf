// Building blocks of the network layers outside the fused MLPs (gated recurrence, group norm,
// dropout): element types, vector accesses of any alignment, gates and activations.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <initializer_list>

#include "auv_internal.hpp"

namespace auv {

// A call's tensors by name; none of the outputs may start where an input or another output does.
struct Named {
  const char* name;
  const void* p;   // may be null
};
inline int check_apart(const char* fn, std::initializer_list<Named> outputs, std::initializer_list<Named> inputs) {
  for (const Named* o = outputs.begin(); o != outputs.end(); ++o) {
    if (!o->p) continue;
    for (const Named& i : inputs)
      if (i.p == o->p) return set_error(AUV_EINVAL, "%s: '%s' is the memory of '%s', an input", fn, o->name, i.name);
    for (const Named* q = outputs.begin(); q != o; ++q)
      if (q->p == o->p) return set_error(AUV_EINVAL, "%s: '%s' and '%s' are the same memory", fn, q->name, o->name);
  }
  return AUV_OK;
}

// A kernel by its address; `fn` is the entry point named in the error.
inline int launch_kernel(const char* fn, const void* kernel, dim3 grid, dim3 block, void** args, size_t lds, hipStream_t s) {
  const hipError_t e = hipLaunchKernel(kernel, grid, block, args, lds, s);
  if (e != hipSuccess) {
    (void)hipGetLastError();
    return set_error(AUV_ELAUNCH, "%s: launch failed: %s", fn, hipGetErrorString(e));
  }
  return AUV_OK;
}

// ------------------------------------------------------------------ vector accesses --
// V elements of a row as one access of up to 16 bytes.  Rows start at any multiple of the
// element size (halves of a projection, odd channel counts), so the type claims no more: gfx950
// loads and stores global memory at any byte address.
template <int BYTES> struct WordOf;
template <> struct WordOf<2> { typedef uint16_t type __attribute__((may_alias)); };
template <> struct WordOf<4> { typedef uint32_t type __attribute__((aligned(2), may_alias)); };
template <> struct WordOf<8> { typedef uint32_t type __attribute__((ext_vector_type(2), aligned(2), may_alias)); };
template <> struct WordOf<16> { typedef uint32_t type __attribute__((ext_vector_type(4), aligned(2), may_alias)); };

template <class T, int V> struct Vec {
  typename WordOf<V * (int)sizeof(T)>::type w;

  __device__ __forceinline__ void load(const T* p) { w = *reinterpret_cast<const decltype(w)*>(p); }
  __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<decltype(w)*>(p) = w; }
  // past the caches' use: what a launch writes once and does not read
  __device__ __forceinline__ void stream(T* p) const { __builtin_nontemporal_store(w, reinterpret_cast<decltype(w)*>(p)); }
  __device__ __forceinline__ float get(int k) const {
    if constexpr (sizeof(T) == 4 && V == 1) return __uint_as_float(w);
    else if constexpr (sizeof(T) == 4) return __uint_as_float(w[k]);
    else if constexpr (V == 1) return __uint_as_float((uint32_t)w << 16);
    else {
      uint32_t d;
      if constexpr (V == 2) d = w;
      else d = w[k >> 1];
      return __uint_as_float(k & 1 ? d & 0xFFFF0000u : d << 16);
    }
  }
  // rounds to the element type, nearest even (the one rounding of a stored value)
  __device__ __forceinline__ void set(const float* v) {
    if constexpr (sizeof(T) == 4 && V == 1) w = __float_as_uint(v[0]);
    else if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int k = 0; k < V; ++k) w[k] = __float_as_uint(v[k]);
    } else if constexpr (V == 1) w = bits(v[0]);
    else if constexpr (V == 2) w = pair(v[0], v[1]);
    else {
#pragma unroll
      for (int k = 0; k < V / 2; ++k) w[k] = pair(v[2 * k], v[2 * k + 1]);
    }
  }
  __device__ __forceinline__ static uint16_t bits(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
  __device__ __forceinline__ static uint32_t pair(float a, float b) {
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, b2{(__bf16)a, (__bf16)b});
  }
};

template <class T> __device__ __forceinline__ T to_elem(float v) {
  if constexpr (sizeof(T) == 4) return v;
  else return (__bf16)v;
}

// Stores the elements k >= shift of a vector whose first ones belong to its neighbour: rows of a
// length that V does not divide end in a vector moved back to end with the row.
// `shared`: rows share cache lines, whose parts are to meet in L2.
template <class T, int V> __device__ __forceinline__ void store_own(T* p, const float* v, int shift, bool shared) {
  if (shift == 0) {
    Vec<T, V> r;
    r.set(v);
    if (shared) {   // kept apart from the other branch, or the two stores would be joined into one without the hint
      asm volatile("");
      r.store(p);
      asm volatile("");
    } else {
      r.stream(p);
    }
  } else {
#pragma unroll
    for (int k = 1; k < V; ++k)
      if (k >= shift) p[k] = to_elem<T>(v[k]);
  }
}

// ------------------------------------------------------------------------ functions --
// e^v.  fp32 tensors keep the product's low part (the instruction's own error is one ulp; the
// rounded product alone would give |v| / 2 ulp); bf16 tensors do without.
template <class T> __device__ __forceinline__ float exp_of(float v) {
  const float L = 1.44269504088896340736f;
  const float p = v * L;
  const float e = __builtin_amdgcn_exp2f(p);
  if constexpr (sizeof(T) == 4) {
    const float lo = __builtin_fmaf(v, L, -p) + v * 1.92596299e-8f;
    return fabsf(v) < 80.0f ? __builtin_fmaf(e, lo * 0.693147180559945f, e) : e;
  }
  return e;
}

// f = sigma(z) and g = 1 - f = sigma(-z), neither by a difference: f = 1 / (1 + e^-z), g = e^-z f.
template <class T> __device__ __forceinline__ void sigmoid2(float z, float& f, float& g) {
  const float e = exp_of<T>(-z);
  const float d = 1.0f + e;
  float r = __builtin_amdgcn_rcpf(d);
  if constexpr (sizeof(T) == 4) r = d < 1e30f ? __builtin_fmaf(__builtin_fmaf(-d, r, 1.0f), r, r) : r;
  f = r;
  g = e > 1e30f ? 1.0f : e * r;
}

// tanh(u): (1 - e) / (1 + e) with e = e^-2|u|, whose difference loses nothing from 0.3 on; below it
// the series in u^2 (Taylor), its first term left out 2e-9 relative there.
template <class T> __device__ __forceinline__ float tanh_of(float u) {
  const float e = exp_of<T>(-2.0f * fabsf(u)), d = 1.0f + e;
  float r = __builtin_amdgcn_rcpf(d);
  r = __builtin_fmaf(__builtin_fmaf(-d, r, 1.0f), r, r);
  const float big = copysignf((1.0f - e) * r, u), q = u * u;
  float p = __builtin_fmaf(q, -8.8632355e-3f, 2.1869489e-2f);
  p = __builtin_fmaf(q, p, -5.3968254e-2f);
  p = __builtin_fmaf(q, p, 0.13333334f);
  p = __builtin_fmaf(q, p, -0.33333334f);
  return fabsf(u) < 0.3f ? __builtin_fmaf(u * q, p, u) : big;
}

constexpr int ACT_NONE = 0, ACT_RELU = 1, ACT_SILU = 2, ACT_TANH = 3;

template <class T> __device__ __forceinline__ float act_of(int act, float u) {
  if (act == ACT_RELU) return u < 0.0f ? 0.0f : u;   // NaN stays
  if (act == ACT_SILU) {
    float f, g;
    sigmoid2<T>(u, f, g);
    return u * f;
  }
  if (act == ACT_TANH) return tanh_of<T>(u);
  return u;
}

template <class T> __device__ __forceinline__ float act_slope(int act, float u) {
  if (act == ACT_RELU) return u > 0.0f ? 1.0f : 0.0f;
  if (act == ACT_SILU) {
    float f, g;
    sigmoid2<T>(u, f, g);
    return __builtin_fmaf(u * g, f, f);
  }
  if (act == ACT_TANH) {   // 4 e / (1 + e)^2 with e = e^-2|u|: no difference 1 - tanh^2
    const float e = exp_of<T>(-2.0f * fabsf(u)), d = 1.0f + e;
    float r = __builtin_amdgcn_rcpf(d);
    r = __builtin_fmaf(__builtin_fmaf(-d, r, 1.0f), r, r);
    return 4.0f * e * r * r;
  }
  return 1.0f;
}

// u <- act(u), u <- act'(u) for M values: one choice for all
template <class T, int M> __device__ __forceinline__ void act_all(int act, float* u) {
  auto each = [&](int which) {
#pragma unroll
    for (int k = 0; k < M; ++k) u[k] = act_of<T>(which, u[k]);
  };
  if (act == ACT_RELU) each(ACT_RELU);
  else if (act == ACT_SILU) each(ACT_SILU);
  else if (act == ACT_TANH) each(ACT_TANH);
}
template <class T, int M> __device__ __forceinline__ void slope_all(int act, float* u) {
  auto each = [&](int which) {
#pragma unroll
    for (int k = 0; k < M; ++k) u[k] = act_slope<T>(which, u[k]);
  };
  if (act == ACT_RELU) each(ACT_RELU);
  else if (act == ACT_SILU) each(ACT_SILU);
  else if (act == ACT_TANH) each(ACT_TANH);
  else each(ACT_NONE);
}

// 1 / sqrt(v): the instruction (one ulp) and a Newton step, far from the ends of the range
__device__ __forceinline__ float rsqrt_of(float v) {
  if (!(v > 1e-30f && v < 1e30f)) return 1.0f / sqrtf(v);
  const float r = __builtin_amdgcn_rsqf(v);
  return __builtin_fmaf(r * 0.5f, __builtin_fmaf(-v * r, r, 1.0f), r);
}

}  // namespace auv
