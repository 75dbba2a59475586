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
#include "common.hpp"
#include "gemm_bf16.hpp"

namespace fm {
namespace {

constexpr int BAL_C = 64;        // tokens per block of the first pass
constexpr int BAL_MAX_B = 4096;  // sequences

template <int G> __device__ __forceinline__ float group_max(float v) {
#pragma unroll
  for (int o = G / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}
template <int G> __device__ __forceinline__ float group_sum(float v) {
#pragma unroll
  for (int o = G / 2; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// p of a row for this lane's experts sub + 64 i; all 0 for a row of nothing but
// -inf.  (fmaxf drops a NaN; exp(NaN - m) brings it back.)
template <int G, int NE>
__device__ __forceinline__ void row_softmax(const float* row, int sub, int E, float* p) {
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < NE; ++i) {
    p[i] = sub + 64 * i < E ? row[sub + 64 * i] : -INFINITY;
    m = fmaxf(m, p[i]);
  }
  m = group_max<G>(m);
  const float base = m == -INFINITY ? 0.f : m;
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < NE; ++i) {
    p[i] = expf(p[i] - base);
    s += p[i];
  }
  s = group_sum<G>(s);
  const float r = s == 0.f ? 0.f : 1.0f / s;
#pragma unroll
  for (int i = 0; i < NE; ++i) p[i] *= r;
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

template <int G, int NE> __global__ __launch_bounds__(256) void k_balance_rows(BalArgs a, BalWs w) {
  constexpr int NG = 256 / G;   // groups per block
  __shared__ float ssum[NG][G * NE + 1];
  __shared__ int scnt[NG][G * NE + 1];
  __shared__ int sn[NG];
  const int sub = threadIdx.x % G, grp = threadIdx.x / G;
  const int t0 = min(blockIdx.x * BAL_C, a.Tn), t1 = min(t0 + BAL_C, a.Tn);
  if (blockIdx.x == 0 && threadIdx.x == 0) *w.done = 0;
  int b = 0;
  if (a.seg) {   // the first sequence that ends behind t0
    int hi = a.B;
    while (b < hi) {
      const int mid = (b + hi) >> 1;
      if (seg_at(a.seg, mid + 1, a.Tn) <= t0) b = mid + 1;
      else hi = mid;
    }
  }
  int total = 0;
  for (; b < a.B; ++b) {
    const int s0 = a.seg ? max(seg_at(a.seg, b, a.Tn), t0) : t0;
    const int s1 = a.seg ? min(seg_at(a.seg, b + 1, a.Tn), t1) : t1;
    if (s0 >= t1) break;
    if (s1 <= s0) continue;
    float acc[NE];
    int cnt[NE], n = 0;
#pragma unroll
    for (int i = 0; i < NE; ++i) acc[i] = 0.f, cnt[i] = 0;
    for (int t = s0 + grp; t < s1; t += NG) {
      if (a.keep && !a.keep[t]) continue;
      float p[NE];
      row_softmax<G, NE>(a.logits + (size_t)t * a.E, sub, a.E, p);
      ++n;
#pragma unroll
      for (int i = 0; i < NE; ++i) acc[i] += p[i];
      for (int j = 0; j < a.k; ++j) {
        const int e = a.idx[(size_t)t * a.k + j];
#pragma unroll
        for (int i = 0; i < NE; ++i) cnt[i] += e == sub + 64 * i;
      }
    }
    __syncthreads();   // the last sequence's sums are read
#pragma unroll
    for (int i = 0; i < NE; ++i) ssum[grp][sub + G * i] = acc[i], scnt[grp][sub + G * i] = cnt[i];
    if (sub == 0) sn[grp] = n;
    __syncthreads();
    const size_t slot = (size_t)blockIdx.x + b;
    for (int e = threadIdx.x; e < a.E; e += 256) {
      float s = 0.f;
      int c = 0;
      for (int g = 0; g < NG; ++g) s += ssum[g][e], c += scnt[g][e];
      w.psum[slot * a.E + e] = s;
      w.pcnt[slot * a.E + e] = c;
    }
    n = 0;
    for (int g = 0; g < NG; ++g) n += sn[g];
    if (threadIdx.x == 0) w.pn[slot] = n;
    total += n;
  }
  if (threadIdx.x == 0) w.blockn[blockIdx.x] = total;
}

// Sum over the block's 1024 threads in a fixed order, in every thread.
template <typename V> __device__ __forceinline__ V block_sum(V v, V* red) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  __syncthreads();
  if (lane_id() == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[0];
  for (int i = 1; i < 16; ++i) v += red[i];
  return v;
}

// One block per sequence: EP = E rounded up to a power of two, 1024 / EP groups of
// threads that each take every (1024 / EP)-th slot.
__global__ __launch_bounds__(1024) void k_balance_final(BalArgs a, BalWs w, int nb, int EP, float coef,
                                                        int32_t* __restrict__ counts, float* __restrict__ dprob,
                                                        float* __restrict__ loss) {
  __shared__ double red[1024];
  __shared__ int redi[1024];
  __shared__ int last;
  const int b = blockIdx.x, e = threadIdx.x & (EP - 1), g = threadIdx.x / EP, ng = 1024 / EP;
  const int s0 = a.seg ? seg_at(a.seg, b, a.Tn) : 0, s1 = a.seg ? seg_at(a.seg, b + 1, a.Tn) : a.Tn;
  const int i0 = s0 / BAL_C, i1 = s1 > s0 ? (s1 - 1) / BAL_C + 1 : i0;
  int n = 0, nbv = 0;
  for (int i = threadIdx.x; i < nb; i += 1024) n += w.blockn[i];
  for (int i = i0 + (int)threadIdx.x; i < i1; i += 1024) nbv += w.pn[i + b];
  n = block_sum(n, redi);
  nbv = block_sum(nbv, redi);
  double s = 0.0;
  int c = 0;
  if (e < a.E)
    for (int i = i0 + g; i < i1; i += ng) {
      s += (double)w.psum[(size_t)(i + b) * a.E + e];
      c += w.pcnt[(size_t)(i + b) * a.E + e];
    }
  __syncthreads();
  red[threadIdx.x] = s;
  redi[threadIdx.x] = c;
  __syncthreads();
  double part = 0.0;
  if (threadIdx.x < (unsigned)a.E) {
    for (int h = 1; h < ng; ++h) s += red[h * EP + e], c += redi[h * EP + e];
    const double dp = nbv > 0 ? (double)coef * a.E * c / ((double)a.k * n * nbv) : 0.0;
    counts[(size_t)b * a.E + e] = c;
    dprob[(size_t)b * a.E + e] = (float)dp;
    part = dp * s;
  }
  __syncthreads();
  part = block_sum(part, red);
  // the block that finishes last adds the sequences' shares, in their order
  if (threadIdx.x == 0) {
    __hip_atomic_store(w.lpart + b, part, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    last = __hip_atomic_fetch_add(w.done, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == (int)gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
  part = 0.0;
  for (int i = threadIdx.x; i < (int)gridDim.x; i += 1024)
    part += __hip_atomic_load(w.lpart + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  part = block_sum(part, red);
  if (threadIdx.x == 0) *loss = (float)part;
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

// One group of lanes per token, BAL_D tokens per group.
constexpr int BAL_D = 4;
template <int G, int NE> __global__ __launch_bounds__(256) void k_balance_dlogits(DlogitArgs a) {
  constexpr int NG = 256 / G;
  extern __shared__ int segs[];   // B + 1 when there are sequences
  const int sub = threadIdx.x % G, grp = threadIdx.x / G;
  if (a.seg) {
    for (int i = threadIdx.x; i <= a.B; i += 256) segs[i] = seg_at(a.seg, i, a.Tn);
    __syncthreads();
  }
  const float up = a.dloss ? *a.dloss : 1.f;
  for (int u = 0; u < BAL_D; ++u) {
    const long t = ((long)blockIdx.x * BAL_D + u) * NG + grp;
    if (t >= a.Tn) return;
    bool in = !a.keep || a.keep[t];
    int b = 0;
    if (a.seg) {   // the sequence with segs[b] <= t < segs[b + 1]
      int lo = 0, hi = a.B;
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (segs[mid + 1] <= t) lo = mid + 1;
        else hi = mid;
      }
      b = lo;
      in = in && b < a.B && segs[b] <= t;
    }
    float d[NE];
#pragma unroll
    for (int i = 0; i < NE; ++i) d[i] = 0.f;
    if (in) {
      float p[NE], w[NE], q = 0.f;
      row_softmax<G, NE>(a.logits + (size_t)t * a.E, sub, a.E, p);
#pragma unroll
      for (int i = 0; i < NE; ++i) {
        w[i] = sub + 64 * i < a.E ? a.dprob[(size_t)b * a.E + sub + 64 * i] : 0.f;
        q = fmaf(p[i], w[i], q);
      }
      q = group_sum<G>(q);
#pragma unroll
      for (int i = 0; i < NE; ++i) d[i] = up * p[i] * (w[i] - q);
    }
    if (a.gate) {
      const size_t r = (size_t)t * a.k;
      float inner = 0.f;
      for (int j = 0; j < a.k; ++j) inner = fmaf(a.gate[r + j], a.dgate[r + j], inner);
      for (int j = 0; j < a.k; ++j) {
        const int e = a.idx[r + j];
        const float v = a.gate[r + j] * (a.dgate[r + j] - inner);
#pragma unroll
        for (int i = 0; i < NE; ++i) d[i] += e == sub + 64 * i ? v : 0.f;
      }
    }
#pragma unroll
    for (int i = 0; i < NE; ++i)
      if (sub + 64 * i < a.E) a.out[(size_t)t * a.E + sub + 64 * i] = d[i];
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
// Both products on v_mfma_f32_32x32x2_f32 (operands exact in fp32).  An operand
// lane holds one value, row lane % 32 at k = lane / 32, which is a coalesced read
// of the row-major inputs whichever of them runs along k.  Output rows m of a tile
// (the first operand's) are dealt to columns so that a lane's 16 sums are 16
// consecutive columns: column(m) = 16 ((m / 4) % 2) + 4 (m / 8) + m % 4.
__device__ __forceinline__ int tile_column(int m) { return 16 * ((m >> 2) & 1) + 4 * (m >> 3) + (m & 3); }

constexpr int RB_SPLITS = 32;   // most parts of the token range in dWr

struct RouterBwd {
  const float* dl;
  const void *X, *Wr;
  int Tn, d, E;
  void* dX;
  int acc_dx;
  float *part, *partb;   // [splits][E][d], [splits][E], or NULL
  int splits, span;      // tokens per split
  int n_dw;              // blocks of the weight gradient, before those of dX
  int xt;                // token tiles per block of dX
};

// NT = expert tiles of 32.
template <typename T, int NT> __global__ __launch_bounds__(256) void k_router_bwd(RouterBwd a) {
  const int lane = lane_id(), wave = wave_id(), m = lane & 31, h = lane >> 5;
  const int ct = (a.d + 127) / 128;   // blocks of 4 column tiles
  if ((int)blockIdx.x < a.n_dw) {
    const int split = blockIdx.x / ct, c0 = (blockIdx.x % ct) * 128 + wave * 32;
    const int t0 = split * a.span, t1 = min(t0 + a.span, a.Tn);
    const int c = min(c0 + tile_column(m), a.d - 1);
    const bool bias = a.partb && c0 == 0, on = c0 < a.d;
    if (!on) return;
    f32x16_t acc[NT];
    float bs[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      bs[j] = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[j][i] = 0.f;
    }
    const T* X = (const T*)a.X;
    for (int t = t0; t < t1; t += 2) {
      const int tt = t + h;
      const bool in = tt < t1;
      const float x = in && X ? to_float(X[(size_t)tt * a.d + c]) : 0.f;
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const int e = 32 * j + m;
        const float v = in && e < a.E ? a.dl[(size_t)tt * a.E + e] : 0.f;
        bs[j] += v;
        acc[j] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, v, acc[j], 0, 0, 0);
      }
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int e = 32 * j + m;
      if (e >= a.E) continue;
      if (bias) {
        const float s = bs[j] + __shfl_xor(bs[j], 32);
        if (h == 0) a.partb[(size_t)split * a.E + e] = s;
      }
      if (a.part) {
        float* o = a.part + ((size_t)split * a.E + e) * a.d + c0 + 16 * h;
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          if (c0 + 16 * h + i < a.d)
            st16(o + i, u32x4_t{__float_as_uint(acc[j][i]), __float_as_uint(acc[j][i + 1]),
                                __float_as_uint(acc[j][i + 2]), __float_as_uint(acc[j][i + 3])});
      }
    }
    return;
  }
  const int blk = blockIdx.x - a.n_dw;
  const int c0 = (blk % ct) * 128 + wave * 32, c = min(c0 + tile_column(m), a.d - 1);
  if (c0 >= a.d) return;
  // this wave's 32 columns of Wr: half h holds experts 32 j + 16 h + [0, 16)
  const T* Wr = (const T*)a.Wr;
  float w[NT][16];
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int e = 32 * j + 16 * h + i;
      w[j][i] = e < a.E ? to_float(Wr[(size_t)e * a.d + c]) : 0.f;
    }
  T* dX = (T*)a.dX;
  constexpr int V = 16 / sizeof(T);
  for (int u = 0; u < a.xt; ++u) {
    const long t0 = ((long)(blk / ct) * a.xt + u) * 32;
    if (t0 >= a.Tn) break;
    const long t = t0 + m < a.Tn ? t0 + m : a.Tn - 1;
    f32x16_t acc;
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = 0.f;
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int e = 32 * j + 16 * h + i;
        const float v = e < a.E ? a.dl[(size_t)t * a.E + e] : 0.f;
        acc = __builtin_amdgcn_mfma_f32_32x32x2f32(w[j][i], v, acc, 0, 0, 0);
      }
    if (t0 + m >= a.Tn) continue;
    T* o = dX + (size_t)t * a.d + c0 + 16 * h;
#pragma unroll
    for (int i = 0; i < 16; i += V) {
      if (c0 + 16 * h + i >= a.d) continue;
      float r[V];
#pragma unroll
      for (int x = 0; x < V; ++x) r[x] = acc[i + x];
      if (a.acc_dx) {
        float old[V];
        unpack16(ld16(o + i), old, (T*)nullptr);
#pragma unroll
        for (int x = 0; x < V; ++x) r[x] += old[x];
      }
      st16(o + i, pack16(r, (T*)nullptr));
    }
  }
}

// dWr and dbias from their parts, in split order; 4 columns per thread.
__global__ __launch_bounds__(256) void k_router_dw(const float* __restrict__ part, const float* __restrict__ partb,
                                                   int splits, long n, int E, int accumulate, float* __restrict__ dWr,
                                                   float* __restrict__ dbias) {
  const long i = ((long)blockIdx.x * 256 + threadIdx.x) * 4;
  if (dWr && i < n) {
    f32x4_t s = {0.f, 0.f, 0.f, 0.f};
    if (accumulate) s = load4(dWr + i);
    f32x4_t v = {0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < splits; ++p) v += load4(part + (size_t)p * n + i);
    store4(dWr + i, s + v);
  }
  if (dbias && blockIdx.x == 0 && threadIdx.x < (unsigned)E) {
    float v = 0.f;
    for (int p = 0; p < splits; ++p) v += partb[(size_t)p * E + threadIdx.x];
    dbias[threadIdx.x] = accumulate ? dbias[threadIdx.x] + v : v;
  }
}

// Parts of the token range for dWr: enough blocks for the card, 64 tokens at
// least in each.
inline int router_splits(int T, int d) {
  const int ct = cdiv(d, 128);
  int s = cdiv(512, ct);
  if (s > RB_SPLITS) s = RB_SPLITS;
  const int most = cdiv(T, 64);
  return s < most ? s : most;
}

template <typename T> void launch_router_bwd(RouterBwd a, int blocks, hipStream_t st) {
  const dim3 g(blocks), b(256);
  if (a.E <= 32) hipLaunchKernelGGL((k_router_bwd<T, 1>), g, b, 0, st, a);
  else if (a.E <= 64) hipLaunchKernelGGL((k_router_bwd<T, 2>), g, b, 0, st, a);
  else if (a.E <= 128) hipLaunchKernelGGL((k_router_bwd<T, 4>), g, b, 0, st, a);
  else hipLaunchKernelGGL((k_router_bwd<T, 8>), g, b, 0, st, a);
}

int check_balance_shape(int T, int E, int B, const void* seg) {
  if (T < 0 || E <= 0 || B <= 0) return fail(MOE_ERR_ARG, "T=%d E=%d B=%d", T, E, B);
  if (E > 256) return fail(MOE_ERR_UNSUPPORTED, "E=%d > 256", E);
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
    hipLaunchKernelGGL((k_balance_rows<L::G, L::NE>), dim3(nb), dim3(256), 0, st, a, w);
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
    hipLaunchKernelGGL((k_balance_dlogits<L::G, L::NE>), dim3(cdiv(T, BAL_D * (256 / L::G))), dim3(256),
                       seg ? (B + 1) * sizeof(int) : 0, as_stream(stream), a);
  });
  return check_launch("moe_balance_loss_bwd");
}

extern "C" size_t moe_router_bwd_workspace_size(int T, int d, int E) {
  if (T < 0 || d <= 0 || E <= 0) return 0;
  return (size_t)router_splits(T, d) * E * ((size_t)d + 1) * sizeof(float);
}

extern "C" int moe_router_bwd(const float* dlogits, const void* X, const void* Wr, int dtype, int T, int d, int E,
                              void* dX, int accumulate_dx, float* dWr, float* dbias, int accumulate_dw, void* ws,
                              size_t ws_bytes, void* stream) {
  clear_error();
  FM_TRY(need_dtype_float(dtype, "dtype"));
  if (T < 0 || d <= 0 || E <= 0) return fail(MOE_ERR_ARG, "T=%d d=%d E=%d", T, d, E);
  if (E > 256) return fail(MOE_ERR_UNSUPPORTED, "E=%d > 256", E);
  if (d % 8) return fail(MOE_ERR_UNSUPPORTED, "d=%d not a multiple of 8", d);
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
  const int ct = cdiv(d, 128), splits = T > 0 && dw ? router_splits(T, d) : 0;
  RouterBwd a{};
  a.dl = dlogits; a.X = dWr ? X : nullptr; a.Wr = Wr;
  a.Tn = T; a.d = d; a.E = E;
  a.dX = dX; a.acc_dx = accumulate_dx;
  a.part = dWr ? (float*)ws : nullptr;
  a.partb = dbias ? (float*)ws + (size_t)splits * E * d : nullptr;
  a.splits = splits;
  a.span = splits ? cdiv(cdiv(T, splits), 2) * 2 : 0;
  a.n_dw = splits * ct;
  const int tiles = cdiv(T, 32);
  a.xt = cdiv(tiles, cdiv(1024, ct));
  const long blocks = a.n_dw + (dX && T > 0 ? (long)ct * cdiv(tiles, a.xt) : 0);
  if (blocks > 0) {
    if (dtype == MOE_BF16) launch_router_bwd<bf16>(a, (int)blocks, st);
    else launch_router_bwd<float>(a, (int)blocks, st);
    FM_TRY(check_launch("moe_router_bwd"));
  }
  if (dw) {
    const long n = (long)E * d;
    hipLaunchKernelGGL(k_router_dw, dim3(dWr ? cdiv(n, 1024) : 1), dim3(256), 0, st, a.part, a.partb, splits, n, E,
                       accumulate_dw, dWr, dbias);
    FM_TRY(check_launch("moe_router_bwd"));
  }
  return MOE_OK;
}
