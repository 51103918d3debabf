// Dropout's draws (tag 3 of the counter-based generator): 16 bits per element, eight elements of a
// row per Philox block.
#pragma once

#include "auv_internal.hpp"

namespace auv {

struct DropArgs {
  uint32_t key0, key1, step, tag, row0;
  uint32_t drop;   // dropped below this; 0: keep all (and draw nothing)
  float scale;     // 65536 / (65536 - drop)
  const uint32_t* counter;

  // first thing in a kernel that draws
  __device__ __forceinline__ void count() {
    if (counter) step += *counter;
  }
};

// host side (dropout.hip): arguments of a launch; d may be null
DropArgs drop_args(const auv_drop* d);
int check_drop(const char* fn, const auv_drop* d, int64_t rows);
int check_rows(const char* fn, const char* name, const auv_rows& r, int type, int n, int s, int c, bool output);

// The block of elements 8 b to 8 b + 7 of a row: ten rounds on 64-bit products (one instruction for both
// halves of a product).
__device__ __forceinline__ U4 drop_block(const DropArgs& D, uint32_t row, uint32_t b) {
  uint32_t c0 = D.row0 + row, c1 = D.step, c2 = D.tag, c3 = b, k0 = D.key0, k1 = D.key1;
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t p0 = (uint64_t)0xD2511F53u * c0, p1 = (uint64_t)0xCD9E8D57u * c2;
    c0 = (uint32_t)(p1 >> 32) ^ c1 ^ k0;
    c1 = (uint32_t)p1;
    c2 = (uint32_t)(p0 >> 32) ^ c3 ^ k1;
    c3 = (uint32_t)p0;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return U4{c0, c1, c2, c3};
}

// Bit j: whether element 8 b + j of the row is kept.
__device__ __forceinline__ uint32_t drop_bits(const DropArgs& D, uint32_t row, uint32_t b) {
  const U4 q = drop_block(D, row, b);
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    m |= ((w[j] & 0xFFFFu) >= D.drop ? 1u : 0u) << (2 * j);
    m |= ((w[j] >> 16) >= D.drop ? 1u : 0u) << (2 * j + 1);
  }
  return m;
}

// The draws of V elements of a row as halves of V / 2 words, compared where they are used.
template <int V> struct Draws {
  uint32_t w[(V + 1) / 2];
  __device__ __forceinline__ bool kept(const DropArgs& D, int k) const {
    return (k & 1 ? w[k >> 1] >> 16 : w[k >> 1] & 0xFFFFu) >= D.drop;
  }
  // from bits: a half above or below every threshold
  __device__ __forceinline__ void set(uint32_t bits) {
#pragma unroll
    for (int i = 0; i < (V + 1) / 2; ++i) w[i] = (bits >> 2 * i & 1u ? 0xFFFFu : 0u) | (bits >> 2 * i & 2u ? 0xFFFF0000u : 0u);
  }
  // elements from channel c of a row on; they lie in two blocks at most
  __device__ __forceinline__ void draw(const DropArgs& D, uint32_t row, uint32_t c) {
    const uint32_t j = c & 7u;
    if (j % V == 0) {
      const U4 q = drop_block(D, row, c >> 3);
      if constexpr (V == 8) {
        w[0] = q.x, w[1] = q.y, w[2] = q.z, w[3] = q.w;
      } else if constexpr (V == 4) {
        w[0] = j ? q.z : q.x;
        w[1] = j ? q.w : q.y;
      } else {
        const uint32_t lo = j & 2u ? q.y : q.x, hi = j & 2u ? q.w : q.z, u = j & 4u ? hi : lo;
        w[0] = j & 1u ? u >> 16 : u;
      }
    } else {
      // kept from sharing the block above, which would then become bits first in either case
      asm volatile("" : "+v"(row));
      uint32_t m = drop_bits(D, row, c >> 3) >> j;
      if (j + V > 8) m |= drop_bits(D, row, (c >> 3) + 1) << (8 - j);
      set(m);
    }
  }
};

}  // namespace auv
