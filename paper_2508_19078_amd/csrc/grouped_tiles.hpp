// How a grouped product on low-bit rows walks its tiles: the row tiles before each
// slot, a block's share of the tiles, a tile's slot and rows, and the grid.
#pragma once

#include "ffn_common.hpp"

namespace fm {
namespace {

// Row tiles before each slot, tiles[s] for s in [0, S]: one block of 256 threads,
// thread i the slots 4 i to 4 i + 3 (S <= 1023).
__device__ __forceinline__ void count_tiles(const RowArgs& ra, int tile_rows, int32_t* tiles) {
  __shared__ int wave_sum[4];
  const int s0 = threadIdx.x * 4, lane = lane_id(), wave = threadIdx.x >> 6;
  int n[4], own = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int s = s0 + i;
    const int rows = s < ra.S_r ? ra.offsets[s + 1] - ra.offsets[s] : s < ra.S ? ra.Tn : 0;
    n[i] = (rows + tile_rows - 1) / tile_rows;
    own += n[i];
  }
  int before = own;   // inclusive over the wave's lanes
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int v = __shfl_up(before, o);
    if (lane >= o) before += v;
  }
  if (lane == 63) wave_sum[wave] = before;
  __syncthreads();
  before -= own;
  for (int w = 0; w < wave; ++w) before += wave_sum[w];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (s0 + i <= ra.S) tiles[s0 + i] = before;
    before += n[i];
  }
}

// A block's tiles of a grouped product with NT column tiles: XCD x (blocks go to
// the XCDs in turn) walks its eighth of them, slot by slot, so that the row tiles
// of a slot, which share its weights, meet in one L2.
struct TileWalk {
  int at, end, step;
};
__device__ __forceinline__ TileWalk tile_walk(const RowArgs& ra, int NT) {
  const long long all = (long long)ld_scalar(ra.mbase + ra.S) * NT;
  const int x = blockIdx.x % N_XCD;
  return TileWalk{(int)(all * x / N_XCD) + (int)(blockIdx.x / N_XCD), (int)(all * (x + 1) / N_XCD),
                (int)(gridDim.x / N_XCD)};
}

struct TileRows {
  SlotRows sr;
  int s, m0, n;   // slot, first row in it, column tile
  int rows;       // rows of the slot from m0 on
  size_t ob;      // m0's row in the per-row buffers
};
__device__ __forceinline__ TileRows tile_rows_at(const RowArgs& ra, int t, int NT, int tile_rows) {
  const int m = t / NT;
  int s = 0;   // the slots that end at or before row tile m
  for (int b = 0; b < ra.S; b += 64) {
    const int i = b + lane_id();
    s += __builtin_popcountll(__ballot(i < ra.S && gptr(ra.mbase)[min(i, ra.S - 1) + 1] <= m));
  }
  TileRows r;
  r.s = __builtin_amdgcn_readfirstlane(s);
  const int first = ld_scalar(ra.mbase + r.s), count = ld_scalar(ra.mbase + r.s + 1) - first;
  int mt;
  band_order(t - first * NT, count, NT, 8, mt, r.n);
  r.sr = slot_rows(r.s, ra.offsets, ra.S_r, ra.Tn, ra.k);
  r.m0 = mt * tile_rows;
  r.rows = r.sr.nrows - r.m0;
  r.ob = (size_t)(r.sr.orow0 + r.m0);
  return r;
}

// The i-th slot with rows (s = -1: there is none), and its rows.
__device__ __forceinline__ int active_slot(const RowArgs& ra, int i, SlotRows& sr) {
  int before = 0;
  for (int b = 0; b < ra.S; b += 64) {
    const int s = b + lane_id(), sc = max(min(s, ra.S_r - 1), 0);
    int lo = 0, hi = 0;
    if (ra.S_r > 0) lo = gptr(ra.offsets)[sc], hi = gptr(ra.offsets)[sc + 1];
    unsigned long long m = __ballot(s < ra.S && (s >= ra.S_r || hi > lo));
    const int n = __builtin_popcountll(m);
    if (i < before + n) {
      for (int drop = i - before; drop > 0; --drop) m &= m - 1;
      const int at = __builtin_amdgcn_readfirstlane(__builtin_ctzll(m)), sl = b + at;
      sr.shared = sl >= ra.S_r;
      const int first = __builtin_amdgcn_readlane(lo, at);
      sr.nrows = sr.shared ? ra.Tn : __builtin_amdgcn_readlane(hi, at) - first;
      sr.xrow0 = sr.shared ? 0 : first;
      sr.orow0 = sr.shared ? (long)ra.Tn * ra.k + (long)(sl - ra.S_r) * ra.Tn : first;
      return sl;
    }
    before += n;
  }
  return -1;
}

// BPC blocks per compute unit, a multiple of the XCDs, at most one per tile.
template <class C> dim3 tile_grid(const RowArgs& ra, int NT) {
  const long long R = (long long)ra.Tn * ra.k;
  const long long tiles = (R / C::RA + (R < ra.S_r ? R : ra.S_r) +
                           (long long)(ra.S - ra.S_r) * ((ra.Tn + C::RA - 1) / C::RA)) * NT;
  const long long most = (long long)(device_cus() + N_XCD - 1) / N_XCD * N_XCD * C::BPC;
  const long long g = (tiles + N_XCD - 1) / N_XCD * N_XCD;
  return dim3((unsigned)(g < most ? g : most));
}

}  // namespace
}  // namespace fm
