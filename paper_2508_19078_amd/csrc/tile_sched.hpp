// Row tiles of a grouped product: the block's own prefix of tiles per slot, the
// tile's slot and rows, and the tiles that the block walks.
#pragma once

#include "ffn_common.hpp"

namespace fm {
namespace {

constexpr int MAX_S = 1023;   // slots of a layer (512 routed + 511 shared)

// Block prefix of row tiles: pre[s] = tiles of the slots before s, s in [0, S].
__device__ __forceinline__ void tile_sched(int* pre, int* wsum, const RowArgs& ra, int tile_rows) {
  const int tid = threadIdx.x, lane = lane_id(), wave = tid >> 6;
  int carry = 0;
  for (int b = 0; b < ra.S; b += 256) {
    const int s = b + tid;
    int n = 0;
    if (s < ra.S) {
      const int rows = s < ra.S_r ? ra.offsets[s + 1] - ra.offsets[s] : ra.Tn;
      n = (rows + tile_rows - 1) / tile_rows;
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(n, o);
      if (lane >= o) n += v;
    }
    if (lane == 63) wsum[wave] = n;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const int v = wsum[w];
      if (w < wave) n += v;
    }
    if (s < ra.S) pre[s + 1] = carry + n;
    carry += wsum[0] + wsum[1] + wsum[2] + wsum[3];
    __syncthreads();
  }
  if (tid == 0) pre[0] = 0;
  __syncthreads();
}

// The slot of row tile m: the number of slots whose tiles all lie before it.
__device__ __forceinline__ int tile_slot(const int* pre, int S, int m) {
  int c = 0;
  for (int b = 0; b < S; b += 64) {
    const int s = b + lane_id();
    c += __builtin_popcountll(__ballot(s < S && pre[s + 1] <= m));
  }
  return __builtin_amdgcn_readfirstlane(c);
}

// One row tile: its slot's rows from the tile's first on, and its column tile.
struct RowTile {
  SlotRows sr;
  int s, m0, n;
  int rows;     // rows of the slot from m0 on
  size_t ob;    // first row in the per-row buffers
};
__device__ __forceinline__ RowTile row_tile_at(const int* pre, const RowArgs& ra, int t, int NT, int RA) {
  RowTile r;
  r.s = tile_slot(pre, ra.S, t / NT);
  const int mb = __builtin_amdgcn_readfirstlane(pre[r.s]);
  const int mt = __builtin_amdgcn_readfirstlane(pre[r.s + 1]) - mb;
  int m;
  band_order(t - mb * NT, mt, NT, 8, m, r.n);
  r.sr = slot_rows(r.s, ra.offsets, ra.S_r, ra.Tn, ra.k);
  r.m0 = m * RA;
  r.rows = r.sr.nrows - r.m0;
  r.ob = (size_t)(r.sr.orow0 + r.m0);
  return r;
}

// This block's tiles of a row product: [lo, hi) by step, the XCD's own range.
struct Span {
  int lo, hi, step;
};
__device__ __forceinline__ Span row_span(const int* pre, const RowArgs& ra, int NT) {
  const long long total = (long long)pre[ra.S] * NT;
  const int x = blockIdx.x % N_XCD;
  return Span{__builtin_amdgcn_readfirstlane((int)(total * x / N_XCD)) + (int)(blockIdx.x / N_XCD),
              __builtin_amdgcn_readfirstlane((int)(total * (x + 1) / N_XCD)), (int)(gridDim.x / N_XCD)};
}

}  // namespace
}  // namespace fm
