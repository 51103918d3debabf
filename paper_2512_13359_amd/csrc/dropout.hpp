// Dropout's draws (tag 3 of the counter-based generator): 16 bits per element, eight elements of a
// row per Philox block.
#pragma once

#include "auv_internal.hpp"

namespace auv {

struct DropArgs {
  uint32_t key0, key1, step, tag, row0;
  uint32_t drop;   // dropped below this; 0: keep all (and draw nothing)
  float scale;     // 65536 / (65536 - drop)
};

// Bit j: whether element 8 b + j of the row is kept.
__device__ __forceinline__ uint32_t keep_bits(const DropArgs& D, uint32_t row, uint32_t b) {
  // ten rounds on 64-bit products (one instruction for both halves)
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
  const uint32_t w[4] = {c0, c1, c2, c3};
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    m |= ((w[j] & 0xFFFFu) >= D.drop ? 1u : 0u) << (2 * j);
    m |= ((w[j] >> 16) >= D.drop ? 1u : 0u) << (2 * j + 1);
  }
  return m;
}

// The same for V elements from channel c of a row on; they lie in two blocks at most.
template <int V> __device__ __forceinline__ uint32_t keep_from(const DropArgs& D, uint32_t row, uint32_t c) {
  uint32_t m = keep_bits(D, row, c >> 3) >> (c & 7);
  if (V > 1 && (c & 7) + V > 8) m |= keep_bits(D, row, (c >> 3) + 1) << (8 - (c & 7));
  return m;
}

}  // namespace auv
