// Group norm: what its three forms share.
//   rows    a group is up to 1024 contiguous numbers (one position, or one group over dense positions): in
//           the registers of 1 to 64 lanes (norm_rows.hip)
//   block   a sample is up to a few thousand vectors: in the registers of a workgroup (norm.hip)
//   chunks  larger samples: statistics by one launch, applied by the next, which reads the sample again (norm.hip)
#pragma once

#include "dropout.hpp"
#include "layers.hpp"

namespace auv {

struct NormArgs {
  char *x, *y, *dout, *dx;
  int64_t x_sn, x_ss, y_sn, y_ss, dout_sn, dout_ss, dx_sn, dx_ss;
  const float *w, *b;
  float *mean, *rstd;
  float* part;    // backward: rows of partial sums of dw and db, [2][C] each; null where neither is wanted
  float* groups;  // chunk form: [n][chunk][tile][held][2] moments (forward) or sums of d and d xhat (backward)
  float *dw, *db;
  float eps;
  int act, n, S, C, G, Cg;
  int m, lanes;      // rows form: elements of a group, lanes per group
  int tile, tiles;   // vectors of a row per workgroup, workgroups across it
  int step, pack;    // block form: positions per pass, samples per pass
  int chunks, per;   // chunk form: chunks of `per` positions
  int held;          // chunk form: groups that a tile can hold a part of
  int part_rows;
  DropArgs drop;
};

// Form and launch shape of a call.
enum NormForm { NORM_ROWS, NORM_BLOCK, NORM_CHUNKS };
struct NormPlan {
  NormForm form;
  int V, R, blocks, threads;   // vector; vectors per lane (rows) or thread (block); workgroups of the launch and their size
  int m, lanes, tile, tiles, step, pack, chunks, per;
  int64_t part_rows;           // backward: partial rows of [2][C] floats
};

constexpr int DPP_ROW_MIRROR = 0x140, DPP_ROW_HALF_MIRROR = 0x141;   // lane i of 16 from 15 - i, of 8 from 7 - i

// Sum over a team of LANES lanes (a power of two), every lane gets it: moves within rows of 16 lanes, then lane swaps.
template <int LANES> __device__ __forceinline__ float lanes_sum(float v) {
  if constexpr (LANES > 1) v += dpp_move<DPP_QUAD_SWAP1>(v);
  if constexpr (LANES > 2) v += dpp_move<DPP_QUAD_SWAP2>(v);
  if constexpr (LANES > 4) v += dpp_move<DPP_ROW_HALF_MIRROR>(v);   // the other quad of eight lanes, equal in its four
  if constexpr (LANES > 8) v += dpp_move<DPP_ROW_MIRROR>(v);
  if constexpr (LANES > 16) {
    float u = v;
    asm("s_nop 1\n\tv_permlane16_swap_b32 %0, %1" : "+v"(v), "+v"(u));
    v += u;
  }
  if constexpr (LANES > 32) {
    float u = v;
    asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(v), "+v"(u));
    v += u;
  }
  return v;
}
// the same for a number of lanes that the launch knows
__device__ __forceinline__ float team_sum(float v, int lanes) {
  if (lanes == 64) return lanes_sum<64>(v);
  if (lanes == 32) return lanes_sum<32>(v);
  if (lanes == 16) return lanes_sum<16>(v);
  if (lanes == 8) return lanes_sum<8>(v);
  if (lanes == 4) return lanes_sum<4>(v);
  return lanes == 2 ? lanes_sum<2>(v) : v;
}
// two sums at once
__device__ __forceinline__ void team_sums(float& v, float& u, int lanes) {
  if (lanes == 64) v = lanes_sum<64>(v), u = lanes_sum<64>(u);
  else if (lanes == 32) v = lanes_sum<32>(v), u = lanes_sum<32>(u);
  else v = team_sum(v, lanes), u = team_sum(u, lanes);
}

int launch_norm_rows(const char* fn, const NormArgs& a, const NormPlan& p, bool bf16, bool grad, size_t lds, hipStream_t s);

}  // namespace auv
