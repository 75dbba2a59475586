// The router's balance loss, the gradient of the router's logits, and the
// products of the router's backward for a dense gradient (the formulas stand in
// the header at moe_balance_loss, moe_balance_loss_bwd and moe_router_bwd).
//
// Softmax over the experts.  A token belongs to G lanes of a wave (8, 16, 32 or
// 64, the least that hold one expert each; 64 lanes of NE experts each above 64),
// so its maximum and sum are butterflies within the group, and a lane keeps the
// sums over tokens of its own experts.
//
// Sums over the tokens of a sequence.  A block takes BAL_C tokens, walks the
// sequences that cross them and leaves, for each, its sums of p, counts and
// number of tokens at slot block + sequence: going through a block's sequences
// and on to the next block's, either index grows, so no two pairs share a slot.
// A block per sequence then adds its slots in a fixed order.  No float atomics.
//
// Measured at 8192 tokens, 64 experts, top-6, 4 sequences: 8.7 us for the blocks, 6.8
// for the sequences, 8.4 for the logits' gradient (2 and 4 MB: all three are a launch
// and chains of dependent loads and exchanges).  The first pass with its tokens one
// after another, without LDS, took 25 us.
#include <algorithm>
#include <type_traits>

#include "common.hpp"
#include "gemm_bf16.hpp"

namespace fm {
namespace {

constexpr int BAL_C = 32;        // tokens per block of the first pass
constexpr int BAL_MAX_B = 4096;  // sequences
constexpr int BAL_MAX_T = 1 << 30;   // tokens: a block's first token and its end are 32-bit
constexpr int BAL_GRID = 1 << 23;    // blocks per launch: with 2^32 threads or more, some do not run

template <int G> __device__ __forceinline__ float group_sum(float v) {
#pragma unroll
  for (int o = G / 2; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// The logits of U rows for this lane's experts sub + 64 i (row u at rows[u]; -inf
// past E), then p in their place; all 0 for a row of nothing but -inf.  The rows'
// steps are interleaved, so that one row's loads and exchanges cover another's.
template <int G, int NE, int U>
__device__ __forceinline__ void rows_softmax(const float* const (&rows)[U], int sub, int E, float (&p)[U][NE]) {
  float m[U], s[U];
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int i = 0; i < NE; ++i) p[u][i] = sub + 64 * i < E ? gptr(rows[u])[sub + 64 * i] : -INFINITY;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    m[u] = p[u][0];
#pragma unroll
    for (int i = 1; i < NE; ++i) m[u] = fmaxf(m[u], p[u][i]);   // drops a NaN; exp(NaN - m) brings it back
  }
#pragma unroll
  for (int o = G / 2; o > 0; o >>= 1)
#pragma unroll
    for (int u = 0; u < U; ++u) m[u] = fmaxf(m[u], __shfl_xor(m[u], o));
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const float base = m[u] == -INFINITY ? 0.f : m[u];
    s[u] = 0.f;
#pragma unroll
    for (int i = 0; i < NE; ++i) {
      p[u][i] = expf(p[u][i] - base);
      s[u] += p[u][i];
    }
  }
#pragma unroll
  for (int o = G / 2; o > 0; o >>= 1)
#pragma unroll
    for (int u = 0; u < U; ++u) s[u] += __shfl_xor(s[u], o);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const float r = s[u] == 0.f ? 0.f : 1.0f / s[u];
#pragma unroll
    for (int i = 0; i < NE; ++i) p[u][i] *= r;
  }
}

__device__ __forceinline__ int seg_at(const int32_t* seg, int b, int Tn) {
  return min(max(seg[b], 0), Tn);
}

// Scratch of the loss: per slot (blocks + B) sums of p and counts [E] and the
// number of tokens; per block its tokens; per sequence its share of the loss.
struct BalWs {
  double* lpart;
  float* psum;
  int32_t* pcnt;
  int32_t* pn;
  int32_t* blockn;
  int32_t* done;
};
inline int bal_blocks(int T) { return T > 0 ? cdiv(T, BAL_C) : 1; }
inline size_t bal_bytes(int T, int E, int B) {
  const size_t nb = bal_blocks(T), slots = nb + B;
  return 8 * (size_t)B + slots * E * 8 + slots * 4 + nb * 4 + 16;
}
inline BalWs bal_at(void* ws, int T, int E, int B) {
  const size_t nb = bal_blocks(T), slots = nb + B;
  BalWs w;
  w.lpart = (double*)ws;
  w.psum = (float*)(w.lpart + B);
  w.pcnt = (int32_t*)(w.psum + slots * E);
  w.pn = w.pcnt + slots * E;
  w.blockn = w.pn + slots;
  w.done = w.blockn + nb;
  return w;
}

struct BalArgs {
  const float* logits;
  const int32_t* idx;
  const int32_t* seg;
  const uint8_t* keep;
  int Tn, E, k, B;
};

template <int G, int NE> __global__ __launch_bounds__(256) void k_balance_rows(BalArgs a, BalWs w, int block0) {
  constexpr int NG = 256 / G;              // groups per block
  constexpr int U = BAL_C > NG ? (BAL_C / NG < 4 ? BAL_C / NG : 4) : 1;   // tokens of a group in flight
  __shared__ float sp[BAL_C][G * NE];      // p of the block's tokens, 0 where not kept
  __shared__ int scnt[G * NE], skept[BAL_C];
  extern __shared__ int segs[];            // B + 1 when there are sequences
  const int sub = threadIdx.x % G, grp = threadIdx.x / G, block = block0 + (int)blockIdx.x;
  const int t0 = min(block * BAL_C, a.Tn), nt = min(BAL_C, a.Tn - t0);
  if (block == 0 && threadIdx.x == 0) *w.done = 0;
  if (a.seg)
    for (int i = threadIdx.x; i <= a.B; i += 256) segs[i] = seg_at(a.seg, i, a.Tn);
  // this thread's choices: every 256th of the block's
  constexpr int MC = BAL_C * 16 / 256;
  int ce[MC], ct[MC];
#pragma unroll
  for (int c = 0; c < MC; ++c) {
    const int i = threadIdx.x + 256 * c;
    ct[c] = i / a.k;
    ce[c] = ct[c] < nt ? a.idx[(size_t)t0 * a.k + i] : -1;
    if (ct[c] < nt && a.keep && !a.keep[t0 + ct[c]]) ce[c] = -1;
  }
  if (threadIdx.x < BAL_C) skept[threadIdx.x] = (int)threadIdx.x < nt && (!a.keep || a.keep[t0 + threadIdx.x]);
#pragma unroll
  for (int r0 = 0; r0 < BAL_C; r0 += U * NG) {
    const float* rows[U];
    float p[U][NE];
    if (r0 + grp >= nt) break;   // whole groups
#pragma unroll
    for (int u = 0; u < U; ++u) rows[u] = a.logits + (size_t)(t0 + min(r0 + grp + u * NG, nt - 1)) * a.E;
    rows_softmax<G, NE, U>(rows, sub, a.E, p);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = r0 + grp + u * NG;
      if (r >= nt) break;
      const bool kept = !a.keep || a.keep[t0 + r];
#pragma unroll
      for (int i = 0; i < NE; ++i) sp[r][sub + G * i] = kept ? p[u][i] : 0.f;
    }
  }
  __syncthreads();
  int b = 0, total = 0;
  if (a.seg) {   // the first sequence that ends behind t0
    int hi = a.B;
    while (b < hi) {
      const int mid = (b + hi) >> 1;
      if (segs[mid + 1] <= t0) b = mid + 1;
      else hi = mid;
    }
  }
  for (; b < a.B; ++b) {
    const int s0 = a.seg ? max(segs[b] - t0, 0) : 0, s1 = a.seg ? min(segs[b + 1] - t0, nt) : nt;
    if (s0 >= nt) break;
    if (s1 <= s0) continue;
    for (int e = threadIdx.x; e < G * NE; e += 256) scnt[e] = 0;
    __syncthreads();
    // integer counts: their order does not matter
#pragma unroll
    for (int c = 0; c < MC; ++c)
      if (ct[c] >= s0 && ct[c] < s1 && (unsigned)ce[c] < (unsigned)a.E) atomicAdd(&scnt[ce[c]], 1);
    const size_t slot = (size_t)block + b;
    float s = 0.f;
    if ((int)threadIdx.x < a.E)
      for (int r = s0; r < s1; ++r) s += sp[r][threadIdx.x];
    int n = 0;
    for (int r = s0; r < s1; ++r) n += skept[r];
    __syncthreads();
    if ((int)threadIdx.x < a.E) {
      w.psum[slot * a.E + threadIdx.x] = s;
      w.pcnt[slot * a.E + threadIdx.x] = scnt[threadIdx.x];
    }
    if (threadIdx.x == 0) w.pn[slot] = n;
    total += n;
    __syncthreads();   // scnt is read
  }
  if (threadIdx.x == 0) w.blockn[block] = total;
}

// One block per sequence: EP = E rounded up to a power of two, 1024 / EP groups of
// threads that each take every (1024 / EP)-th slot.
__global__ __launch_bounds__(1024) void k_balance_final(BalArgs a, BalWs w, int nb, int EP, float coef,
                                                        int32_t* __restrict__ counts, float* __restrict__ dprob,
                                                        float* __restrict__ loss) {
  __shared__ double red[1024];
  __shared__ int redi[1024];
  __shared__ int wn[16], wb[16];
  __shared__ double wl[16];
  __shared__ int last;
  const int b = blockIdx.x, e = threadIdx.x & (EP - 1), g = threadIdx.x / EP, ng = 1024 / EP;
  const int lane = lane_id(), wave = threadIdx.x >> 6;
  const int s0 = a.seg ? seg_at(a.seg, b, a.Tn) : 0, s1 = a.seg ? seg_at(a.seg, b + 1, a.Tn) : a.Tn;
  const int i0 = s0 / BAL_C, i1 = s1 > s0 ? (s1 - 1) / BAL_C + 1 : i0;
  int n = 0, own = 0, c = 0;   // tokens of all sequences, of this one; choices of e
  for (int i = threadIdx.x; i < nb; i += 1024) n += w.blockn[i];
  for (int i = i0 + (int)threadIdx.x; i < i1; i += 1024) own += w.pn[i + b];
  double s = 0.0;
  if (e < a.E) {
#pragma unroll 4
    for (int i = i0 + g; i < i1; i += ng) {
      s += (double)w.psum[(size_t)(i + b) * a.E + e];
      c += w.pcnt[(size_t)(i + b) * a.E + e];
    }
  }
  // lanes with the same expert, then (below) the waves
  for (int o = EP; o < 64; o <<= 1) {
    s += __shfl_xor(s, o);
    c += __shfl_xor(c, o);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    n += __shfl_xor(n, o);
    own += __shfl_xor(own, o);
  }
  if (lane == 0) wn[wave] = n, wb[wave] = own;
  red[threadIdx.x] = s;
  redi[threadIdx.x] = c;
  __syncthreads();
  double part = 0.0;
  if (threadIdx.x < (unsigned)a.E) {
    const int step = EP < 64 ? 64 : EP;
    for (int h = threadIdx.x + step; h < 1024; h += step) s += red[h], c += redi[h];
    n = own = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) n += wn[i], own += wb[i];
    const double dp = own > 0 ? (double)coef * a.E * c / ((double)a.k * n * own) : 0.0;
    counts[(size_t)b * a.E + e] = c;
    dprob[(size_t)b * a.E + e] = (float)dp;
    part = dp * s;
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) part += __shfl_xor(part, o);
  if (lane == 0) wl[wave] = part;   // E <= 256: 0 from wave 4 on
  __syncthreads();
  if (threadIdx.x == 0) {
    part = wl[0] + wl[1] + wl[2] + wl[3];
    if (gridDim.x == 1) *loss = (float)part;
    __hip_atomic_store(w.lpart + b, part, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    // the block that finishes last adds the sequences' shares, in their order
    last = gridDim.x > 1 && __hip_atomic_fetch_add(w.done, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == (int)gridDim.x - 1;
  }
  if (gridDim.x == 1) return;
  __syncthreads();
  if (!last) return;
  part = 0.0;
  for (int i = threadIdx.x; i < (int)gridDim.x; i += 1024)
    part += __hip_atomic_load(w.lpart + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) part += __shfl_xor(part, o);
  __syncthreads();   // wl is read
  if (lane == 0) wl[wave] = part;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < 16; ++i) part += wl[i];
    *loss = (float)part;
  }
}

struct DlogitArgs {
  const float *logits, *dprob, *dloss;
  const int32_t* seg;
  const uint8_t* keep;
  const float* gate;
  const int32_t* idx;
  const float* dgate;
  int Tn, E, k, B;
  float* out;
};

// One group of lanes per token, U tokens of a group at once.  The k <= E <= G
// choices of a token lie in the group's first lanes and are dealt from there (E >
// 64: k <= 16 of 64 lanes).
template <int G, int NE> constexpr int dlogit_rows() { return G == 64 ? 2 : 1; }
template <int G, int NE> __global__ __launch_bounds__(256) void k_balance_dlogits(DlogitArgs a, int block0) {
  constexpr int NG = 256 / G, U = dlogit_rows<G, NE>();
  extern __shared__ int segs[];   // B + 1 when there are sequences
  const int sub = threadIdx.x % G, grp = threadIdx.x / G;
  if (a.seg) {
    for (int i = threadIdx.x; i <= a.B; i += 256) segs[i] = seg_at(a.seg, i, a.Tn);
    __syncthreads();
  }
  const float up = a.dloss ? *a.dloss : 1.f;
  long t[U];
  const float* rows[U];
  bool in[U];
  int b[U];
  float d[U][NE], w[U][NE];
  int ei[U];
  float gv[U], dv[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    t[u] = (((long)block0 + blockIdx.x) * U + u) * NG + grp;
    const long tc = min(t[u], (long)a.Tn - 1);
    rows[u] = a.logits + (size_t)tc * a.E;
    in[u] = !a.keep || a.keep[tc];
    b[u] = 0;
    if (a.seg) {   // the sequence with segs[b] <= t < segs[b + 1]
      int lo = 0, hi = a.B;
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (segs[mid + 1] <= tc) lo = mid + 1;
        else hi = mid;
      }
      in[u] = in[u] && lo < a.B && segs[lo] <= tc;
      b[u] = min(lo, a.B - 1);
    }
#pragma unroll
    for (int i = 0; i < NE; ++i) w[u][i] = sub + 64 * i < a.E ? a.dprob[(size_t)b[u] * a.E + sub + 64 * i] : 0.f;
    const bool chosen = a.gate && sub < a.k;
    const size_t r = (size_t)tc * a.k + sub;
    ei[u] = chosen ? a.idx[r] : -1;
    gv[u] = chosen ? a.gate[r] : 0.f;
    dv[u] = chosen ? a.dgate[r] : 0.f;
  }
  rows_softmax<G, NE, U>(rows, sub, a.E, d);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float q = 0.f;
#pragma unroll
    for (int i = 0; i < NE; ++i) q = fmaf(d[u][i], w[u][i], q);
    q = group_sum<G>(q);
#pragma unroll
    for (int i = 0; i < NE; ++i) d[u][i] = in[u] ? up * d[u][i] * (w[u][i] - q) : 0.f;
    if (a.gate) {
      dv[u] = gv[u] * (dv[u] - group_sum<G>(gv[u] * dv[u]));
      for (int j = 0; j < a.k; ++j) {
        const int e = __shfl(ei[u], j, G);
        const float v = __shfl(dv[u], j, G);
#pragma unroll
        for (int i = 0; i < NE; ++i) d[u][i] += e == sub + 64 * i ? v : 0.f;
      }
    }
    if (t[u] < a.Tn) {
#pragma unroll
      for (int i = 0; i < NE; ++i)
        if (sub + 64 * i < a.E) a.out[(size_t)t[u] * a.E + sub + 64 * i] = d[u][i];
    }
  }
}

// fn(integral_constant G, integral_constant NE)
template <int G_, int NE_> struct ExpertLanes {
  static constexpr int G = G_, NE = NE_;
};
template <typename Fn> void with_expert_lanes(int E, Fn fn) {
  if (E <= 8) fn(ExpertLanes<8, 1>{});
  else if (E <= 16) fn(ExpertLanes<16, 1>{});
  else if (E <= 32) fn(ExpertLanes<32, 1>{});
  else if (E <= 64) fn(ExpertLanes<64, 1>{});
  else if (E <= 128) fn(ExpertLanes<64, 2>{});
  else fn(ExpertLanes<64, 4>{});
}

// ------------------------------------------------- products of the backward --
// A block owns some columns and a part of the token range; bf16 blocks walk it in
// slabs of 64 tokens, of which they form dX and add to their part of dWr at once: the
// slab's dlogits are read and taken apart once for both.
//
// bf16.  dlogits are fp32, the other operand is bf16: an fp32 value is the sum of
// three bf16 (high, middle, low: 8 bits each), whose products with a bf16 are exact
// in fp32, so dWr and dX are three MFMAs each with fp32 accuracy
// (v_mfma_f32_32x32x16_bf16, 16 times the rate of the fp32 MFMA).  An infinity or NaN of X
// meets the first part alone: a later one may be 0 where the sum is not, and 0 times it is
// no number.  One of Wr is left to the stores, which add its products with the whole
// dlogits: a second set of products beside the first took the registers of the sums.
// The three planes lie in LDS as [64 tokens][32 experts], X as [64 tokens][32 columns]
// per wave: dWr sums over tokens and reads both transposed (ds_read_b64_tr_b16), dX
// sums over experts and reads the planes along their rows (16-byte chunks of a row
// swizzled by (row / 4) % 4, so that 16 rows read at one chunk cover the 64 banks
// once).  Wr's fragments stay in registers.  8192 tokens, d = 2048, 64 experts: 32.9 us
// with the sums of dWr's parts in 5.2 us more (72 MB for both outputs: 14 us at the rate
// of a copy); calls for dX alone 20, for dWr and dbias alone 28, for all 36.  A block has 4
// slabs, each a chain of loads, conversion, exchange through LDS, products and stores (the
// matrix cores are busy for 14 % of it).  32 parts of the token range measured best at this
// width (with 128 columns per block, and sums in 32 bits, 33 + 12.5 us, 16 parts 36.7 + 7.4,
// 64 parts 34.1 + 20.6: a part of dWr is 512 KB, written and read); narrower layers were not
// measured and leave compute units idle.  128 < E: 166 us at 256 experts, with 372 bytes per lane in
// scratch.  On fp32 MFMAs, dX and dWr by separate blocks, 64 experts took 124 + 18 us.
//
// fp32.  v_mfma_f32_32x32x2_f32: an operand lane holds one value, row lane % 32 at k
// = lane / 32, a coalesced read of the row-major inputs whichever of them runs along k.
// The same size: calls for dX alone 71 us, for dWr and dbias alone 44, for all 105.  dX's
// lanes read their own token's dlogits one by one.
//
// Both: rows m of dX's first operand are dealt to columns tile_column(m).

constexpr int RB_SLAB = 64;     // tokens
constexpr int RB_SPLITS = 32;   // most parts of the token range
constexpr int RB_PAD = 320;     // floats between them

typedef double f64x4_t __attribute__((ext_vector_type(4)));

struct RouterBwd {
  const float* dl;
  const void *X, *Wr;
  int Tn, d, E;
  void* dX;
  int acc_dx;
  float* part;           // [splits][E][d], stride apart, or NULL
  double* partb;         // [splits][E], or NULL
  long stride;
  int span;              // tokens per split, a multiple of RB_SLAB
};

// The old dX of a lane's 16 columns plus the sums, or these alone, to dX (fp32).
__device__ __forceinline__ void put_dx(float* o, int cols, bool add, const f32x16_t& acc) {
#pragma unroll
  for (int i = 0; i < 16; i += 4) {
    if (i >= cols) continue;
    f32x4_t r = {acc[i], acc[i + 1], acc[i + 2], acc[i + 3]};
    if (add) r += load4(o + i);
    store4(o + i, r);
  }
}

// a + b + c = v exactly (to a multiple of 2^-133, where bf16 ends), each the upper half of
// an fp32 and so a bf16 (8 bits of v each, one sign).  Cut off, not rounded: a finite v has finite parts, and an infinity is a.
__device__ __forceinline__ void split3(f32x4_t v, u32x2_t (&p)[3]) {
  uint32_t r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = __float_as_uint(v[i]);
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    p[k] = u32x2_t{r[0] >> 16 | (r[1] & 0xFFFF0000u), r[2] >> 16 | (r[3] & 0xFFFF0000u)};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float f = __uint_as_float(r[i]);
      r[i] = fabsf(f) == INFINITY ? 0u : __float_as_uint(f - __uint_as_float(r[i] & 0xFFFF0000u));
    }
  }
}

// The halves of x that are infinities or NaN as bits 15 and 31 of the result.
__device__ __forceinline__ uint32_t none_bits(uint32_t x) { return ((x & 0x7F807F80u) + 0x00800080u) & 0x80008000u; }
__device__ __forceinline__ bool has_none(const bf16x8_t& x) {
  const u32x4_t v = __builtin_bit_cast(u32x4_t, x);
  return (none_bits(v[0]) | none_bits(v[1]) | none_bits(v[2]) | none_bits(v[3])) != 0;
}
// x with `in` in their places, but with their signs.
__device__ __forceinline__ bf16x8_t without_none(const bf16x8_t& x, uint32_t in) {
  u32x4_t v = __builtin_bit_cast(u32x4_t, x);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t at = (none_bits(v[i]) >> 15) * 0xFFFFu;
    v[i] = (v[i] & (~at | 0x80008000u)) | (at & in);
  }
  return __builtin_bit_cast(bf16x8_t, v);
}

// NT = expert tiles of 32.  8 waves: wave w takes columns 32 CB (w % 4) + [0, 32 CB)
// and tokens 32 (w / 4) + [0, 32) of each slab; the two halves of dWr meet in LDS at
// the end.  CB = 2 where the sums fit the registers: a plane's fragment then serves
// two MFMAs.
template <int NT> struct RouterTile {
  static constexpr int CB = NT <= 2 ? 2 : 1, COLS = 128 * CB;
  static constexpr int X_BYTES = CB * 32 * 64;         // a wave's part of a slab, [CB][32 tokens][32 columns]
  static constexpr int BLK = RB_SLAB * 64;             // a plane's [64 tokens][32 experts]
  static constexpr int OUT = 32 * CB * 32 * 4;         // a wave's dX tile, fp32
  static constexpr int LDS = 2 * 8 * X_BYTES + 3 * NT * BLK + 8 * OUT;
  static_assert(LDS <= 160 * 1024 && 4 * NT * CB * 4096 <= LDS, "slab, and half of the sums");
};
template <int NT> __global__ __launch_bounds__(512, 2) void k_router_bf16(RouterBwd a) {
  typedef RouterTile<NT> C;
  constexpr int CB = C::CB, BLK = C::BLK;
  __shared__ __align__(16) char lds_[C::LDS];
  FM_LDS char* const xs = (FM_LDS char*)lds_;
  FM_LDS char* const pl = xs + 2 * 8 * C::X_BYTES;
  FM_LDS char* const out = pl + 3 * NT * BLK + wave_id() * C::OUT;
  const int lane = lane_id(), wave = wave_id(), m = lane & 31, h = lane >> 5, th = wave >> 2;
  const int ct = (a.d + C::COLS - 1) / C::COLS, split = blockIdx.x / ct;
  const int c0 = (blockIdx.x % ct) * C::COLS + (wave & 3) * 32 * CB;
  const int t0 = split * a.span, t1 = min(t0 + a.span, a.Tn);
  const bool on = c0 < a.d, dw = a.part && on, dx = a.dX && on;
  const bool bias = a.partb && blockIdx.x % ct == 0;
  const bf16* const X = (const bf16*)a.X;

  // X: this wave's columns and tokens, 16 tokens of a column block per instruction;
  // columns past d repeat the last
  auto load_x = [&](int t, int buf) {
    if (!dw) return;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) {
        const int r = min(t + 32 * th + 16 * u + (lane >> 2), t1 - 1);
        const int c = min(c0 + 32 * cb + 8 * (lane & 3), a.d - 8);
        dma16(X + (size_t)r * a.d + c, xs + (buf * 8 + wave) * C::X_BYTES + cb * 2048 + u * 1024);
      }
  };
  // dlogits: thread q of the slab's quads, 4 experts of token q / (8 NT)
  constexpr int QT = 8 * NT, QN = RB_SLAB * QT / 512;
  const int quad = threadIdx.x % QT, e0 = 4 * quad;
  f32x4_t dl[QN];
  f64x4_t bsum = {0., 0., 0., 0.};   // the bias's gradient: in 64 bits, like a plain sum over the tokens
  auto load_dl = [&](int t) {
#pragma unroll
    for (int i = 0; i < QN; ++i) {
      const int r = t + threadIdx.x / QT + i * (512 / QT);
      const FM_GLOBAL float* const p = gptr(a.dl) + (size_t)min(r, t1 - 1) * a.E;
      if (a.E % 4 == 0) {   // whole quads, 16-byte aligned
        dl[i] = *(const FM_GLOBAL f32x4_t*)(p + min(e0, a.E - 4));
        if (r >= t1 || e0 >= a.E) dl[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        continue;
      }
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const float v = p[min(e0 + x, a.E - 1)];
        dl[i][x] = r < t1 && e0 + x < a.E ? v : 0.f;
      }
    }
  };
  load_x(t0, 0);
  load_dl(t0);
  // Wr: lane m's columns, experts 16 s + 8 h + [0, 8)
  bf16x8_t wf[CB][2 * NT];
  bool wr_none = false;   // an infinity or NaN among the wave's: it takes part as 1 or -1 and is added at the end
  if (dx) {
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
      const FM_GLOBAL uint16_t* const Wr = (const FM_GLOBAL uint16_t*)a.Wr + min(c0 + 32 * cb + tile_column(m), a.d - 1);
#pragma unroll
      for (int s = 0; s < 2 * NT; ++s) {
        uint32_t v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int e = 16 * s + 8 * h + i;
          v[i] = Wr[(size_t)min(e, a.E - 1) * a.d];
          if (e >= a.E) v[i] = 0;
        }
        wf[cb][s] = __builtin_bit_cast(bf16x8_t, u32x4_t{v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16});
        wr_none |= has_none(wf[cb][s]);
        wf[cb][s] = without_none(wf[cb][s], 0x3F803F80u);
      }
    }
    wr_none = __ballot(wr_none) != 0;
  }
  f32x16_t acc[NT][CB];
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[j][cb][i] = 0.f;
  B16Frag<false, 32, 1> fr;
  fr.init(0);
  // as fr, for the swizzled planes: rows 8 (lane / 32) + [0, 4) and + [4, 8) of a step
  const uint32_t f0 = fr.off[0] ^ (uint32_t)(2 * h) << 4, f1 = f0 ^ 16;
  auto read_pl = [&](const FM_LDS char* blk, int ks) {
    const FM_LDS char* const p = blk + ks * 1024;
    const u32x2_t w0 = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((FM_LDS i16x4_t*)(p + f0)));
    const u32x2_t w1 = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((FM_LDS i16x4_t*)(p + 256 + f1)));
    return __builtin_bit_cast(bf16x8_t, u32x4_t{w0[0], w0[1], w1[0], w1[1]});
  };

  int buf = 0;
  for (int t = t0; t < t1; t += RB_SLAB, buf ^= 1) {
    wait_vmcnt<0>();
    if (dw && t + RB_SLAB > t1) {   // rows behind the last token: 0, not 0 times what stands there
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int cb = 0; cb < CB; ++cb)
          if (t + 32 * th + 16 * u + (lane >> 2) >= t1)
            *(FM_LDS u32x4_t*)(xs + (buf * 8 + wave) * C::X_BYTES + cb * 2048 + u * 1024 + lane * 16) = u32x4_t{0, 0, 0, 0};
    }
    __syncthreads();   // the planes of the last slab are read
#pragma unroll
    for (int i = 0; i < QN; ++i) {
      u32x2_t p[3];
      split3(dl[i], p);
      const int r = threadIdx.x / QT + i * (512 / QT);
#pragma unroll
      for (int k = 0; k < 3; ++k)
        *(FM_LDS u32x2_t*)(pl + (k * NT + (quad >> 3)) * BLK + r * 64 + ((((quad & 7) >> 1) ^ ((r >> 2) & 3)) << 4) + (quad & 1) * 8) = p[k];
      if (bias) bsum += __builtin_convertvector(dl[i], f64x4_t);
    }
    __syncthreads();
    if (t + RB_SLAB < t1) {
      load_x(t + RB_SLAB, buf ^ 1);
      load_dl(t + RB_SLAB);
    }
    // dX first: its stores are on their way while dWr multiplies
    if (dx) {
      f32x16_t o[CB];
#pragma unroll
      for (int cb = 0; cb < CB; ++cb)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[cb][i] = 0.f;
#pragma unroll
      for (int s = 0; s < 2 * NT; ++s)
#pragma unroll
        for (int k = 0; k < 3; ++k) {
          const FM_LDS char* const p = pl + (k * NT + (s >> 1)) * BLK + (32 * th + m) * 64 +
                                       (((2 * (s & 1) + h) ^ ((m >> 2) & 3)) << 4);
          const bf16x8_t v = __builtin_bit_cast(bf16x8_t, *(const FM_LDS u32x4_t*)p);
#pragma unroll
          for (int cb = 0; cb < CB; ++cb) o[cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wf[cb][s], v, o[cb], 0, 0, 0);
        }
      // out through LDS, whole lines of a row at once: [32 tokens][32 CB fp32], chunks
      // of 16 bytes swizzled by the row
      constexpr int CH = 8 * CB, PIECES = 4 * CB;   // chunks of a row, 16-byte pieces of it in bf16
#pragma unroll
      for (int cb = 0; cb < CB; ++cb)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *(FM_LDS f32x4_t*)(out + m * (CH * 16) + (((8 * cb + 4 * h + q) ^ (m & (CH - 1))) << 4)) =
              f32x4_t{o[cb][4 * q], o[cb][4 * q + 1], o[cb][4 * q + 2], o[cb][4 * q + 3]};
      wave_lds_fence();
#pragma unroll
      for (int u = 0; u < PIECES / 2; ++u) {
        const int q = (64 / PIECES) * u + lane / PIECES, pc = lane % PIECES;
        const int r = t + 32 * th + q, c = c0 + 8 * pc;
        float v[8];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const f32x4_t w = *(const FM_LDS f32x4_t*)(out + q * (CH * 16) + (((2 * pc + x) ^ (q & (CH - 1))) << 4));
#pragma unroll
          for (int e = 0; e < 4; ++e) v[4 * x + e] = w[e];
        }
        if (r >= t1 || c >= a.d) continue;
        if (wr_none) {   // rare: what Wr's infinities and NaN add
          for (int e = 0; e < a.E; ++e) {
            const float g = gptr(a.dl)[(size_t)r * a.E + e];
            float w[8];
            unpack16(ld16((const bf16*)a.Wr + (size_t)e * a.d + c), w, (bf16*)nullptr);
#pragma unroll
            for (int x = 0; x < 8; ++x)
              if (!(fabsf(w[x]) < INFINITY)) v[x] = fmaf(g, w[x], v[x]);
          }
        }
        bf16* const at = (bf16*)a.dX + (size_t)r * a.d + c;
        if (a.acc_dx) {
          float old[8];
          unpack16(ld16(at), old, (bf16*)nullptr);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] += old[e];
        }
        st16(at, pack16(v, (bf16*)nullptr));
      }
      wave_lds_fence();   // the next slab's dX takes the place
    }
    if (dw) {
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        bf16x8_t x[CB];
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) x[cb] = fr.read(xs + (buf * 8 + wave) * C::X_BYTES + cb * 2048, 0, ks);
        bool none = false;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) none |= has_none(x[cb]);
        none = __ballot(none) != 0;
#pragma unroll
        for (int k = 0; k < 3; ++k) {
          if (k == 1 && none) {
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) x[cb] = without_none(x[cb], 0u);
          }
#pragma unroll
          for (int j = 0; j < NT; ++j) {
            const bf16x8_t v = read_pl(pl + (k * NT + j) * BLK, 2 * th + ks);
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) acc[j][cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, x[cb], acc[j][cb], 0, 0, 0);
          }
        }
      }
    }
  }
  if (a.part) {   // the tokens' halves add up through LDS: [wave % 4][tile][quad][lane]
    __syncthreads();
    auto at = [&](int j, int cb, int q) {
      return (FM_LDS f32x4_t*)(xs + ((((wave & 3) * NT + j) * CB + cb) * 4 + q) * 1024 + lane * 16);
    };
    if (th == 1) {
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int cb = 0; cb < CB; ++cb)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            *at(j, cb, q) = f32x4_t{acc[j][cb][4 * q], acc[j][cb][4 * q + 1], acc[j][cb][4 * q + 2], acc[j][cb][4 * q + 3]};
    }
    __syncthreads();
    if (th == 0 && dw) {
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int cb = 0; cb < CB; ++cb)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const f32x4_t v = *at(j, cb, q);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int e = 32 * j + 8 * q + 4 * h + i, c = c0 + 32 * cb + m;
              if (e < a.E && c < a.d) gptr(a.part)[(size_t)split * a.stride + (size_t)e * a.d + c] = acc[j][cb][4 * q + i] + v[i];
            }
          }
    }
  }
  if (bias) {   // the block's threads with the same experts, in order
    __syncthreads();
    FM_LDS f64x4_t* const b4 = (FM_LDS f64x4_t*)xs;
    b4[threadIdx.x] = bsum;
    __syncthreads();
    if (threadIdx.x < QT) {
      for (int g = 1; g < 512 / QT; ++g) bsum += b4[threadIdx.x + g * QT];
#pragma unroll
      for (int x = 0; x < 4; ++x)
        if (e0 + x < a.E) gptr(a.partb)[(size_t)split * a.E + e0 + x] = bsum[x];
    }
  }
}

template <int NT> __global__ __launch_bounds__(256) void k_router_f32(RouterBwd a) {
  const int lane = lane_id(), wave = wave_id(), m = lane & 31, h = lane >> 5;
  const int ct = (a.d + 127) / 128, split = blockIdx.x / ct;
  const int c0 = (blockIdx.x % ct) * 128 + wave * 32;
  if (c0 >= a.d) return;
  const int t0 = split * a.span, t1 = min(t0 + a.span, a.Tn);
  const FM_GLOBAL float* const dl = gptr(a.dl);
  if (a.part || a.partb) {
    const int c = min(c0 + tile_column(m), a.d - 1);
    const bool bias = a.partb && c0 == 0;
    const FM_GLOBAL float* const X = (const FM_GLOBAL float*)a.X;
    f32x16_t acc[NT];
    double bs[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      bs[j] = 0.;
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[j][i] = 0.f;
    }
    constexpr int U = NT <= 2 ? 8 : 4;   // steps (2 tokens each) whose loads are in flight together
    for (int t = t0; t < t1; t += 2 * U) {
      float x[U], v[U][NT];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int r = t + 2 * u + h, rc = min(r, t1 - 1);
        x[u] = a.X ? X[(size_t)rc * a.d + c] : 0.f;
        if (r >= t1) x[u] = 0.f;
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          v[u][j] = dl[(size_t)rc * a.E + min(32 * j + m, a.E - 1)];
          if (r >= t1 || 32 * j + m >= a.E) v[u][j] = 0.f;
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          if (bias) bs[j] += v[u][j];
          acc[j] = __builtin_amdgcn_mfma_f32_32x32x2f32(x[u], v[u][j], acc[j], 0, 0, 0);
        }
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int e = 32 * j + m;
      if (e >= a.E) continue;
      if (bias) {
        const double s = bs[j] + __shfl_xor(bs[j], 32);
        if (h == 0) gptr(a.partb)[(size_t)split * a.E + e] = s;
      }
      if (a.part) {
        float* o = a.part + (size_t)split * a.stride + (size_t)e * a.d + c0 + 16 * h;
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          if (c0 + 16 * h + i < a.d) store4(o + i, f32x4_t{acc[j][i], acc[j][i + 1], acc[j][i + 2], acc[j][i + 3]});
      }
    }
  }
  if (!a.dX) return;
  // this wave's 32 columns of Wr: half h holds experts 32 j + 16 h + [0, 16)
  const int c = min(c0 + tile_column(m), a.d - 1);
  const FM_GLOBAL float* const Wr = (const FM_GLOBAL float*)a.Wr;
  float w[NT][16];
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int e = 32 * j + 16 * h + i;
      w[j][i] = e < a.E ? Wr[(size_t)min(e, a.E - 1) * a.d + c] : 0.f;
    }
  for (int t = t0; t < t1; t += 32) {
    const int r = min(t + m, t1 - 1);
    f32x16_t acc;
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = 0.f;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      float v[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int e = 32 * j + 16 * h + i;
        v[i] = e < a.E ? dl[(size_t)r * a.E + min(e, a.E - 1)] : 0.f;
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(w[j][i], v[i], acc, 0, 0, 0);
    }
    if (t + m < t1) put_dx((float*)a.dX + (size_t)r * a.d + c0 + 16 * h, a.d - c0 - 16 * h, a.acc_dx, acc);
  }
}

// dWr and dbias from their parts: a block takes 64 quads of columns, its 4 groups of
// threads every fourth part, and the groups' sums are added in order.  In 64 bits: up to
// 32 parts of many tokens each, which may nearly cancel.
__global__ __launch_bounds__(256) void k_router_dw(const float* __restrict__ part, const double* __restrict__ partb,
                                                   int splits, long stride, long n, int E, int accumulate,
                                                   float* __restrict__ dWr,
                                                   float* __restrict__ dbias) {
  __shared__ f64x4_t red[4][64];
  const int q = threadIdx.x & 63, g = threadIdx.x >> 6;
  const long i = ((long)blockIdx.x * 64 + q) * 4;
  if (dWr) {
    f64x4_t v = {0., 0., 0., 0.};
    if (i < n) {
#pragma unroll 8
      for (int p = g; p < splits; p += 4) v += __builtin_convertvector(load4(part + (size_t)p * stride + i), f64x4_t);
    }
    red[g][q] = v;
    __syncthreads();
    if (g == 0 && i < n) {
      v = red[0][q] + red[1][q] + red[2][q] + red[3][q];
      if (accumulate) v += __builtin_convertvector(load4(dWr + i), f64x4_t);
      store4(dWr + i, __builtin_convertvector(v, f32x4_t));
    }
  }
  if (dbias && blockIdx.x == 0 && threadIdx.x < (unsigned)E) {
    double v = accumulate ? dbias[threadIdx.x] : 0.;
#pragma unroll 8
    for (int p = 0; p < splits; ++p) v += partb[(size_t)p * E + threadIdx.x];
    dbias[threadIdx.x] = (float)v;
  }
}

// Columns of a block.
inline int router_cols(int E, bool is_bf16) { return is_bf16 && E <= 64 ? 256 : 128; }
// Parts of the token range, at most: blocks of 8 waves for every compute unit (bf16;
// fp32: two of 4 waves).  Grows with T, so a workspace for T serves fewer tokens too.
inline int router_most_parts(int T, int d, int E, bool is_bf16) {
  const int s = cdiv(is_bf16 ? 256 : 512, cdiv(d, router_cols(E, is_bf16)));
  const int most = s < RB_SPLITS ? s : RB_SPLITS, slabs = cdiv(T, RB_SLAB);
  return slabs < most ? slabs : most;
}
// The parts: whole slabs in each, at least one.  A part without a slab would leave its
// block with X still requested into the LDS that the sums pass through at its end.
struct RouterParts {
  int n, span;   // parts, tokens of each (the last may hold fewer)
};
inline RouterParts router_parts(int T, int d, int E, bool is_bf16) {
  if (T == 0) return {0, 0};
  const int slabs = cdiv(T, RB_SLAB), each = cdiv(slabs, router_most_parts(T, d, E, is_bf16));
  return {cdiv(slabs, each), each * RB_SLAB};
}
// Floats between two parts: not a power of two, which would put the same place of all
// parts on one memory channel.
inline long router_stride(int d, int E) { return (long)E * d + RB_PAD; }

void launch_router_bwd(const RouterBwd& a, bool is_bf16, int splits, hipStream_t st) {
  const dim3 g(splits * cdiv(a.d, router_cols(a.E, is_bf16)));
  auto run = [&](auto nt) {
    constexpr int NT = decltype(nt)::value;
    if (is_bf16) hipLaunchKernelGGL((k_router_bf16<NT>), g, dim3(512), 0, st, a);
    else hipLaunchKernelGGL((k_router_f32<NT>), g, dim3(256), 0, st, a);
  };
  if (a.E <= 32) run(std::integral_constant<int, 1>{});
  else if (a.E <= 64) run(std::integral_constant<int, 2>{});
  else if (a.E <= 128) run(std::integral_constant<int, 4>{});
  else run(std::integral_constant<int, 8>{});
}

int check_balance_shape(int T, int E, int B, const void* seg) {
  if (T < 0 || E <= 0 || B <= 0) return fail(MOE_ERR_ARG, "T=%d E=%d B=%d", T, E, B);
  if (E > 256) return fail(MOE_ERR_UNSUPPORTED, "E=%d > 256", E);
  if (T > BAL_MAX_T) return fail(MOE_ERR_UNSUPPORTED, "T=%d > 2^30", T);
  if (B > BAL_MAX_B) return fail(MOE_ERR_UNSUPPORTED, "B=%d > %d", B, BAL_MAX_B);
  if (!seg && B != 1) return fail(MOE_ERR_ARG, "B=%d without seg", B);
  return MOE_OK;
}

}  // namespace
}  // namespace fm

using namespace fm;

extern "C" size_t moe_balance_loss_workspace_size(int T, int E, int B) {
  if (T < 0 || E <= 0 || B <= 0) return 0;
  return bal_bytes(T, E, B);
}

extern "C" int moe_balance_loss(const float* logits, const int32_t* idx, const int32_t* seg, const uint8_t* keep,
                                int T, int E, int k, int B, float coef, int32_t* counts, float* dprob, float* loss,
                                void* ws, size_t ws_bytes, void* stream) {
  clear_error();
  FM_TRY(check_balance_shape(T, E, B, seg));
  if (k <= 0) return fail(MOE_ERR_ARG, "k=%d", k);
  if (k > 16 || k > E) return fail(MOE_ERR_UNSUPPORTED, "k=%d must be <= min(E, 16)", k);
  if (!(coef > -3e38f && coef < 3e38f)) return fail(MOE_ERR_ARG, "coef=%g must be finite", (double)coef);
  if (T > 0) { FM_TRY(need(logits, "logits")); FM_TRY(need(idx, "idx")); }
  FM_TRY(need(counts, "counts")); FM_TRY(need(dprob, "dprob")); FM_TRY(need(loss, "loss")); FM_TRY(need(ws, "ws"));
  FM_TRY(need_aligned(logits, "logits")); FM_TRY(need_aligned(idx, "idx")); FM_TRY(need_aligned(seg, "seg"));
  FM_TRY(need_aligned(keep, "keep")); FM_TRY(need_aligned(counts, "counts")); FM_TRY(need_aligned(dprob, "dprob"));
  FM_TRY(need_aligned(loss, "loss")); FM_TRY(need_aligned(ws, "ws"));
  if (ws_bytes < bal_bytes(T, E, B))
    return fail(MOE_ERR_WORKSPACE, "workspace %zu < %zu bytes", ws_bytes, bal_bytes(T, E, B));
  hipStream_t st = as_stream(stream);
  const BalArgs a{logits, idx, seg, keep, T, E, k, B};
  const BalWs w = bal_at(ws, T, E, B);
  const int nb = bal_blocks(T);
  with_expert_lanes(E, [&](auto l) {
    typedef decltype(l) L;
    for (int b0 = 0; b0 < nb; b0 += BAL_GRID)
      hipLaunchKernelGGL((k_balance_rows<L::G, L::NE>), dim3(std::min(nb - b0, BAL_GRID)), dim3(256),
                         seg ? (B + 1) * sizeof(int) : 0, st, a, w, b0);
  });
  FM_TRY(check_launch("moe_balance_loss"));
  int EP = 1;
  while (EP < E) EP *= 2;
  hipLaunchKernelGGL(k_balance_final, dim3(B), dim3(1024), 0, st, a, w, nb, EP, coef, counts, dprob, loss);
  return check_launch("moe_balance_loss");
}

extern "C" int moe_balance_loss_bwd(const float* logits, const float* dprob, const float* dloss, const int32_t* seg,
                                    const uint8_t* keep, const float* gate, const int32_t* idx, const float* dgate,
                                    int T, int E, int k, int B, float* dlogits, void* stream) {
  clear_error();
  FM_TRY(check_balance_shape(T, E, B, seg));
  if (T > 0 && ((gate != nullptr) != (idx != nullptr) || (gate != nullptr) != (dgate != nullptr)))
    return fail(MOE_ERR_ARG, "gate, idx and dgate must be given together or not at all");
  if (gate && k <= 0) return fail(MOE_ERR_ARG, "k=%d", k);
  if (gate && (k > 16 || k > E)) return fail(MOE_ERR_UNSUPPORTED, "k=%d must be <= min(E, 16)", k);
  if (T == 0) return MOE_OK;
  FM_TRY(need(logits, "logits")); FM_TRY(need(dprob, "dprob")); FM_TRY(need(dlogits, "dlogits"));
  FM_TRY(need_aligned(logits, "logits")); FM_TRY(need_aligned(dprob, "dprob")); FM_TRY(need_aligned(dloss, "dloss"));
  FM_TRY(need_aligned(seg, "seg")); FM_TRY(need_aligned(keep, "keep")); FM_TRY(need_aligned(gate, "gate"));
  FM_TRY(need_aligned(idx, "idx")); FM_TRY(need_aligned(dgate, "dgate")); FM_TRY(need_aligned(dlogits, "dlogits"));
  const DlogitArgs a{logits, dprob, dloss, seg, keep, gate, idx, dgate, T, E, k, B, dlogits};
  with_expert_lanes(E, [&](auto l) {
    typedef decltype(l) L;
    const int nb = cdiv(T, dlogit_rows<L::G, L::NE>() * (256 / L::G));
    for (int b0 = 0; b0 < nb; b0 += BAL_GRID)
      hipLaunchKernelGGL((k_balance_dlogits<L::G, L::NE>), dim3(std::min(nb - b0, BAL_GRID)), dim3(256),
                         seg ? (B + 1) * sizeof(int) : 0, as_stream(stream), a, b0);
  });
  return check_launch("moe_balance_loss_bwd");
}

extern "C" size_t moe_router_bwd_workspace_size(int T, int d, int E) {
  if (T < 0 || d <= 0 || E <= 0) return 0;
  const int a = router_most_parts(T, d, E, true), b = router_most_parts(T, d, E, false);   // for either type
  return (size_t)(a > b ? a : b) * (router_stride(d, E) * sizeof(float) + E * sizeof(double));
}

extern "C" int moe_router_bwd(const float* dlogits, const void* X, const void* Wr, int dtype, int T, int d, int E,
                              void* dX, int accumulate_dx, float* dWr, float* dbias, int accumulate_dw, void* ws,
                              size_t ws_bytes, void* stream) {
  clear_error();
  FM_TRY(need_dtype_float(dtype, "dtype"));
  if (T < 0 || d <= 0 || E <= 0) return fail(MOE_ERR_ARG, "T=%d d=%d E=%d", T, d, E);
  if (E > 256) return fail(MOE_ERR_UNSUPPORTED, "E=%d > 256", E);
  if (T > BAL_MAX_T) return fail(MOE_ERR_UNSUPPORTED, "T=%d > 2^30", T);
  if (d % 8) return fail(MOE_ERR_UNSUPPORTED, "d=%d not a multiple of 8", d);
  // the sum of dWr's parts has a thread for each of its elements
  if ((long)E * d > 1L << 30) return fail(MOE_ERR_UNSUPPORTED, "E=%d d=%d: more than 2^30 weights", E, d);
  if (T > 0) {
    FM_TRY(need(dlogits, "dlogits"));
    if (dX) FM_TRY(need(Wr, "Wr"));
    if (dWr) FM_TRY(need(X, "X"));
    if (dX && dX == X) return fail(MOE_ERR_ARG, "dX must not alias X");
  }
  FM_TRY(need_aligned(dlogits, "dlogits")); FM_TRY(need_aligned(X, "X")); FM_TRY(need_aligned(Wr, "Wr"));
  FM_TRY(need_aligned(dX, "dX")); FM_TRY(need_aligned(dWr, "dWr")); FM_TRY(need_aligned(dbias, "dbias"));
  FM_TRY(need_aligned(ws, "ws"));
  const bool dw = dWr || dbias;
  if (dw && T > 0) {
    FM_TRY(need(ws, "ws"));
    if (ws_bytes < moe_router_bwd_workspace_size(T, d, E))
      return fail(MOE_ERR_WORKSPACE, "workspace %zu < %zu bytes", ws_bytes, moe_router_bwd_workspace_size(T, d, E));
  }
  if (T == 0 && (!dw || accumulate_dw)) return MOE_OK;
  hipStream_t st = as_stream(stream);
  const bool is_bf16 = dtype == MOE_BF16;
  const auto [splits, span] = router_parts(T, d, E, is_bf16);
  RouterBwd a{};
  a.dl = dlogits; a.X = dWr ? X : nullptr; a.Wr = Wr;
  a.Tn = T; a.d = d; a.E = E;
  a.dX = dX; a.acc_dx = accumulate_dx;
  a.part = dWr ? (float*)ws : nullptr;
  a.stride = router_stride(d, E);
  a.partb = dbias ? (double*)((float*)ws + (size_t)splits * a.stride) : nullptr;   // E d and the padding are even
  if (T > 0) {
    a.span = span;
    launch_router_bwd(a, is_bf16, splits, st);
    FM_TRY(check_launch("moe_router_bwd"));
  }
  if (dw) {
    const long n = (long)E * d;
    hipLaunchKernelGGL(k_router_dw, dim3(dWr ? cdiv(n, 256) : 1), dim3(256), 0, st, a.part, a.partb, splits, a.stride,
                       n, E, accumulate_dw, dWr, dbias);
    FM_TRY(check_launch("moe_router_bwd"));
  }
  return MOE_OK;
}
