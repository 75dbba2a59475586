// Routing from the router's logits by scores (the formulas stand in the header at
// moe_route_scored): softmax or sigmoid scores, a bias on the selection, expert groups,
// top-k, and the gradient of the logits.
//
// 16 lanes per token, four tokens per wave: lane q holds experts 64 c + 4 q to + 3 for
// chunks c, as they lie in memory.  A selection round is a maximum over the lane's keys
// and four row rotations over the lanes; rank j ends in lane j.
//
// The selection is that of keys in fp64, but fp64 is seldom needed.  Without sel_bias
// the logits themselves order the experts, exactly.  With it, keys in fp32 decide where
// neighbours in rank order (the first one left out among them), and the worst group kept
// and the best one not, lie further apart than twice the keys' error; a wave with a token
// where they do not selects again from keys in fp64.
#include "common.hpp"
#include "ffn_common.hpp"

namespace fm {
namespace {

constexpr int GT_TOK = 16;   // tokens per block of four waves
constexpr int GT_MAXK = 16, GT_MAXG = 32;
constexpr int NOBODY = 0x7FFFFFFF;

struct Gating {
  int E, k, n_group, topk_group, group_top, size;   // size: experts of a group
  bool sigmoid, renorm;
  float scale;
};

// x of lane (q + N) % 16 of the row.
template <int N> __device__ __forceinline__ float ror(float x) { return dpp_f<0x120 + N>(x); }
template <int N> __device__ __forceinline__ int ror(int x) {
  return __builtin_amdgcn_update_dpp(0, x, 0x120 + N, 0xF, 0xF, false);
}
template <int N> __device__ __forceinline__ double ror(double x) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  return __builtin_bit_cast(double, (uint64_t)(uint32_t)ror<N>((int)(b >> 32)) << 32 | (uint32_t)ror<N>((int)(uint32_t)b));
}
// f over the 16 lanes of a row, in every one of them.
template <typename K, typename F> __device__ __forceinline__ K row_fold(K x, F f) {
  x = f(x, ror<8>(x));
  x = f(x, ror<4>(x));
  x = f(x, ror<2>(x));
  return f(x, ror<1>(x));
}
template <typename K> __device__ __forceinline__ K larger(K a, K b) { return a > b ? a : b; }
template <typename K> __device__ __forceinline__ K row_max(K x) { return row_fold(x, [](K a, K b) { return larger(a, b); }); }
template <typename K> __device__ __forceinline__ K row_sum(K x) { return row_fold(x, [](K a, K b) { return a + b; }); }

template <typename K> __device__ __forceinline__ K minus_inf() { return -(K)__builtin_inff(); }
template <typename K> __device__ __forceinline__ bool before(K va, int ia, K vb, int ib) { return va > vb || (va == vb && ia < ib); }
template <typename K> __device__ __forceinline__ K number(K x) { return x == x ? x : minus_inf<K>(); }

__device__ __forceinline__ float e_to(float x) { return expf(x); }
__device__ __forceinline__ double e_to(double x) { return exp(x); }

// 1 / (1 + exp(-z)) without an overflow; times exp(-m) where z < 0 (m <= 0).
template <typename K> __device__ __forceinline__ K logistic(K z, K m = 0) {
  if (z >= 0) return 1 / (1 + e_to(-z));
  return z == minus_inf<K>() ? (K)0 : e_to(z - m) / (1 + e_to(z));
}
// exp(z - m) with m the largest of the z: infinities share 1, -inf alone is nothing.
template <typename K> __device__ __forceinline__ K softmax_part(K z, K m) {
  const K inf = -minus_inf<K>();
  return m == inf ? (K)(z == inf) : z == -inf ? (K)0 : e_to(z - m);
}

// Scores of this lane's experts (0 for places behind E, whose z is -inf).
template <typename K, int N> __device__ __forceinline__ void scores(const Gating& g, const float (&z)[N], K (&s)[N]) {
  if (g.sigmoid) {
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = logistic<K>((K)z[i]);
    return;
  }
  float m = z[0];
#pragma unroll
  for (int i = 1; i < N; ++i) m = larger(m, z[i]);
  m = row_max(m);
  K sum = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) sum += s[i] = softmax_part<K>((K)z[i], (K)m);
  sum = row_sum(sum);
#pragma unroll
  for (int i = 0; i < N; ++i) s[i] = sum > 0 ? s[i] / sum : (K)0;
}

// What a selection leaves in lane j of a row: the choice of rank j.
struct Choice {
  int e;
  bool sure;   // false: fp32 keys did not decide
};

// Selection for a row's token.  key: the experts' keys; of: what the groups rank by;
// gap: neighbours in rank order must differ by more to be sure (0: keys are exact).
template <typename K, int N>
__device__ __forceinline__ Choice select(const Gating& g, const K (&key)[N], const K (&of)[N], K gap, K group_gap, K* row) {
  const int lane = lane_id(), q = lane & 15;
  bool sure = true;
  uint32_t left = 0;   // this lane's experts that may still be chosen
  uint32_t kept = ~0u;
  if (g.n_group > 1) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int e = 64 * (i / 4) + 4 * q + i % 4;
      if (e < g.E) row[e] = of[i];
    }
    wave_lds_fence();
    // lane q ranks groups q and q + 16, reading their experts from different places
    K r[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int grp = q + 16 * h;
      K a = minus_inf<K>(), b = minus_inf<K>();
      if (grp < g.n_group) {
        int at = q % g.size;
        for (int i = 0; i < g.size; ++i) {
          const K v = row[grp * g.size + at];
          b = larger(b, v < a ? v : a);
          a = larger(a, v);
          if (++at == g.size) at = 0;
        }
      }
      r[h] = g.group_top == 2 ? number(a + b) : a;
    }
    wave_lds_fence();
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (q + 16 * h < g.n_group) row[q + 16 * h] = r[h];
    wave_lds_fence();
    K worst = -minus_inf<K>(), best = minus_inf<K>();   // of the groups kept, of the others
    uint32_t bits = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int grp = q + 16 * h;
      int ahead = 0;
      for (int o = 0; o < g.n_group; ++o) ahead += before(row[o], o, r[h], grp);
      const bool in = grp < g.n_group && ahead < g.topk_group;
      if (in) {
        bits |= 1u << grp;
        worst = r[h] < worst ? r[h] : worst;
      } else if (grp < g.n_group) {
        best = larger(best, r[h]);
      }
    }
    kept = (uint32_t)row_fold((int)bits, [](int a, int b) { return a | b; });
    worst = -row_max(-worst);
    best = row_max(best);
    if (group_gap > 0 && g.topk_group < g.n_group && !(worst - best > group_gap)) sure = false;
    wave_lds_fence();
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int e = 64 * (i / 4) + 4 * q + i % 4;
    if (e < g.E && (g.n_group == 1 || (kept >> (e / g.size) & 1))) left |= 1u << i;
  }
  int mine = 0;
  K last = 0;
  const int rounds = gap > 0 ? g.k + 1 : g.k;   // one more shows how far the first left out is
  for (int j = 0; j < rounds; ++j) {
    K v = minus_inf<K>();
    int e = NOBODY;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int ei = 64 * (i / 4) + 4 * q + i % 4;
      if ((left >> i & 1) && before(key[i], ei, v, e)) v = key[i], e = ei;
    }
    auto step = [&](K v2, int e2) {
      if (before(v2, e2, v, e)) v = v2, e = e2;
    };
    step(ror<8>(v), ror<8>(e));
    step(ror<4>(v), ror<4>(e));
    step(ror<2>(v), ror<2>(e));
    step(ror<1>(v), ror<1>(e));
    if (e != NOBODY) {
      if (j > 0 && gap > 0 && !(last - v > gap)) sure = false;
      if (q == (e >> 2 & 15)) left &= ~(1u << (4 * (e >> 6) + (e & 3)));
    }
    last = v;
    if (q == j) mine = e;
  }
  return Choice{mine, sure};
}

// N / 4 chunks of 64 experts.  32768 tokens of 256 experts in 8 groups: see DESIGN.
template <int N>
__global__ __launch_bounds__(256) void k_route_scored(Gating g, const float* __restrict__ logits,
                                                      const float* __restrict__ sel_bias, const uint8_t* __restrict__ keep,
                                                      int T, int32_t* __restrict__ idx, float* __restrict__ gate,
                                                      int32_t* __restrict__ counts) {
  __shared__ double rows[GT_TOK][16 * N];
  __shared__ int hist[16 * N];
  const int lane = lane_id(), q = lane & 15, tok = threadIdx.x >> 4;
  if (counts) {
    for (int e = threadIdx.x; e < g.E; e += 256) hist[e] = 0;
    __syncthreads();
  }
  for (int t0 = blockIdx.x * GT_TOK; t0 < T; t0 += gridDim.x * GT_TOK) {
    const int t = t0 + tok, tc = min(t, T - 1);   // rows behind the last token repeat it
    const float* const zr = logits + (size_t)tc * g.E;
    float z[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int e = 64 * (i / 4) + 4 * q + i % 4;
      z[i] = e < g.E ? number(gptr(zr)[e]) + 0.f : minus_inf<float>();
    }
    Choice c;
    if (sel_bias) {
      float s[N], key[N];
      scores<float>(g, z, s);
      float top = 0.f;   // the largest finite key's magnitude
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int e = 64 * (i / 4) + 4 * q + i % 4;
        key[i] = e < g.E ? number(s[i] + gptr(sel_bias)[e]) : minus_inf<float>();
        const float a = fabsf(key[i]);
        if (a < __builtin_inff()) top = larger(top, a);
      }
      // steps of 2^-24 of a score (below 1): exponential and quotient 5, the softmax's sum 20
      // more, so keys differ by 2^-21 or 2^-18.4 from the exact ones' difference at most, and
      // by half a step of the larger each
      const float gap = (g.sigmoid ? 0x1p-20f : 0x1p-18f) + 0x1p-22f * row_max(top);
      c = select(g, key, key, gap, g.group_top == 2 ? 4 * gap : gap, (float*)rows[tok]);
      if (__any(!c.sure)) {
        double sd[N], kd[N];
        scores<double>(g, z, sd);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const int e = 64 * (i / 4) + 4 * q + i % 4;
          kd[i] = e < g.E ? number(sd[i] + (double)gptr(sel_bias)[e]) : minus_inf<double>();
        }
        c = select(g, kd, kd, 0.0, 0.0, rows[tok]);
      }
    } else if (g.n_group > 1 && g.group_top == 2) {
      float s[N];
      scores<float>(g, z, s);
      c = select(g, z, s, 0.f, g.sigmoid ? 0x1p-18f : 0x1p-16f, (float*)rows[tok]);   // sums of two
      if (__any(!c.sure)) {
        double sd[N], zd[N];
        scores<double>(g, z, sd);
#pragma unroll
        for (int i = 0; i < N; ++i) zd[i] = z[i];
        c = select(g, zd, sd, 0.0, 0.0, rows[tok]);
      }
    } else {
      c = select(g, z, z, 0.f, 0.f, (float*)rows[tok]);
    }
    // gates: lane j the choice of rank j
    const bool mine = q < g.k;
    const float zj = mine ? number(gptr(zr)[c.e]) : minus_inf<float>();
    float w, S = 1.f;
    if (g.renorm) {
      const float m = row_max(zj);
      w = g.sigmoid ? logistic(zj, fminf(m, 0.f)) : softmax_part(zj, m);
      if (!mine) w = 0.f;
      S = row_sum(w);
    } else if (g.sigmoid) {
      w = logistic(zj);
    } else {
      float m = z[0], sum = 0.f;
#pragma unroll
      for (int i = 1; i < N; ++i) m = larger(m, z[i]);
      m = row_max(m);
#pragma unroll
      for (int i = 0; i < N; ++i) sum += softmax_part(z[i], m);
      w = softmax_part(zj, m);
      S = row_sum(sum);
    }
    if (mine && t < T) {
      idx[(size_t)t * g.k + q] = c.e;
      gate[(size_t)t * g.k + q] = S > 0.f ? g.scale * (w / S) : 0.f;
      if (counts && (!keep || keep[t])) atomicAdd(&hist[c.e], 1);
    }
  }
  if (counts) {
    __syncthreads();
    for (int e = threadIdx.x; e < g.E; e += 256)
      if (hist[e]) atomicAdd(&counts[e], hist[e]);
  }
}

// The logits' gradient: lane j forms the share of choice j, the shares meet in an LDS row,
// which goes out 16 bytes per lane.
template <int N>
__global__ __launch_bounds__(256) void k_route_scored_bwd(Gating g, const float* logits, const int32_t* __restrict__ idx,
                                                          const float* __restrict__ dgate, int T, float* dlogits,
                                                          int accumulate) {
  __shared__ __align__(16) float rows[GT_TOK][16 * N];
  const int lane = lane_id(), q = lane & 15, tok = threadIdx.x >> 4;
  const int t = blockIdx.x * GT_TOK + tok, tc = min(t, T - 1);
  const float* const zr = logits + (size_t)tc * g.E;
  const bool dense = !g.sigmoid && !g.renorm;
  int e = q < g.k ? gptr(idx)[(size_t)tc * g.k + q] : -1;
  const bool mine = e >= 0 && e < g.E;
  const float zj = mine ? number(gptr(zr)[e]) : minus_inf<float>();
  const float dg = mine ? g.scale * gptr(dgate)[(size_t)tc * g.k + q] : 0.f;
  float z[N], m = minus_inf<float>(), sum = 0.f;
  if (dense) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int ei = 64 * (i / 4) + 4 * q + i % 4;
      z[i] = ei < g.E ? number(gptr(zr)[ei]) : minus_inf<float>();
      m = larger(m, z[i]);
    }
    m = row_max(m);
#pragma unroll
    for (int i = 0; i < N; ++i) sum += z[i] = softmax_part(z[i], m);
    sum = row_sum(sum);
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] = sum > 0.f ? z[i] / sum : 0.f;
  }
  float val, inner = 0.f;
  if (g.renorm) {
    const float mj = row_max(zj);
    float w = g.sigmoid ? logistic(zj, fminf(mj, 0.f)) : softmax_part(zj, mj);
    if (!mine) w = 0.f;
    const float S = row_sum(w);
    const float share = S > 0.f ? w / S : 0.f;
    // the derivative of ln s by the logit is 1 - s, or for the softmax 1 (the shares' sum is 1)
    val = share * (dg - row_sum(share * dg)) * (g.sigmoid ? logistic(-zj) : 1.f);
  } else if (g.sigmoid) {
    val = logistic(zj) * logistic(-zj) * dg;
  } else {
    const float s = sum > 0.f ? softmax_part(zj, m) / sum : 0.f;
    inner = row_sum(mine ? s * dg : 0.f);
    val = dg;
  }
  if (!mine) val = 0.f, e = -1;
  // an expert named twice: the first of its lanes takes both shares
  bool first = mine;
  float total = 0.f;
  for (int j = 0; j < g.k; ++j) {
    const int ej = __shfl(e, (lane & 48) + j);
    const float vj = __shfl(val, (lane & 48) + j);
    if (ej == e) {
      total += vj;
      if (j < q) first = false;
    }
  }
  float* const row = rows[tok];
  float* const out = dlogits + (size_t)tc * g.E;
  if (accumulate && !dense) {
    if (first && t < T) gptr(out)[e] += total;
    return;
  }
#pragma unroll
  for (int c = 0; c < N / 4; ++c) *(u32x4_t*)(row + 64 * c + 4 * q) = u32x4_t{0, 0, 0, 0};
  wave_lds_fence();
  if (first) row[e] = total;
  wave_lds_fence();
  if (t >= T) return;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int ei = 64 * (i / 4) + 4 * q + i % 4;
    if (ei >= g.E) continue;
    float v = row[ei];
    if (dense) v = z[i] * (v - inner);
    gptr(out)[ei] = accumulate ? gptr(out)[ei] + v : v;
  }
}

__global__ __launch_bounds__(256) void k_bias_update(const int32_t* __restrict__ counts, int E, float rate,
                                                     float* __restrict__ sel_bias) {
  __shared__ int64_t part[4];
  const int e = threadIdx.x;
  const int64_t n = e < E ? counts[e] : 0;
  int64_t all = n;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) all += __shfl_xor((long long)all, o);
  if (lane_id() == 0) part[e >> 6] = all;
  __syncthreads();
  all = part[0] + part[1] + part[2] + part[3];
  if (e < E) sel_bias[e] += all > n * E ? rate : all < n * E ? -rate : 0.f;
}

int check_gating(const moe_gating* g, int T) {
  if (!g) return fail(MOE_ERR_ARG, "gating must not be NULL");
  if (T < 0 || g->E <= 0 || g->k <= 0) return fail(MOE_ERR_ARG, "T=%d E=%d k=%d", T, g->E, g->k);
  if (T > 1 << 30) return fail(MOE_ERR_UNSUPPORTED, "T=%d > 2^30", T);
  if (g->E > 256) return fail(MOE_ERR_UNSUPPORTED, "E=%d > 256", g->E);
  if (g->k > GT_MAXK || g->k > g->E) return fail(MOE_ERR_UNSUPPORTED, "k=%d must be <= min(E, 16)", g->k);
  if (g->score != MOE_SCORE_SOFTMAX && g->score != MOE_SCORE_SIGMOID)
    return fail(MOE_ERR_UNSUPPORTED, "score=%d: expected MOE_SCORE_SOFTMAX or MOE_SCORE_SIGMOID", g->score);
  if (g->n_group <= 0 || g->E % g->n_group) return fail(MOE_ERR_ARG, "n_group=%d must divide E=%d", g->n_group, g->E);
  if (g->n_group > GT_MAXG) return fail(MOE_ERR_UNSUPPORTED, "n_group=%d > 32", g->n_group);
  const int size = g->E / g->n_group;
  if (g->topk_group <= 0 || g->topk_group > g->n_group)
    return fail(MOE_ERR_ARG, "topk_group=%d outside 1 to n_group=%d", g->topk_group, g->n_group);
  if (g->k > g->topk_group * size)
    return fail(MOE_ERR_ARG, "k=%d choices from %d groups of %d experts", g->k, g->topk_group, size);
  if (g->group_top != 1 && g->group_top != 2) return fail(MOE_ERR_UNSUPPORTED, "group_top=%d: expected 1 or 2", g->group_top);
  if (g->n_group > 1 && g->group_top > size) return fail(MOE_ERR_ARG, "group_top=%d of groups of %d", g->group_top, size);
  if (!(__builtin_fabsf(g->scale) < __builtin_inff())) return fail(MOE_ERR_ARG, "scale=%g", g->scale);
  return MOE_OK;
}

Gating device_gating(const moe_gating* g) {
  // groups that all stay change nothing
  const int n = g->topk_group == g->n_group ? 1 : g->n_group;
  return Gating{g->E, g->k, n, n == 1 ? 1 : g->topk_group, g->group_top, g->E / n, g->score == MOE_SCORE_SIGMOID,
                g->renorm != 0, g->scale};
}

}  // namespace
}  // namespace fm

using namespace fm;

extern "C" int moe_route_scored(const moe_gating* g, const float* logits, const float* sel_bias, const uint8_t* keep, int T,
                                int32_t* idx, float* gate, int32_t* counts, void* stream) {
  clear_error();
  FM_TRY(check_gating(g, T));
  if (T == 0) return MOE_OK;
  FM_TRY(need(logits, "logits")); FM_TRY(need(idx, "idx")); FM_TRY(need(gate, "gate"));
  FM_TRY(need_aligned(logits, "logits")); FM_TRY(need_aligned(sel_bias, "sel_bias")); FM_TRY(need_aligned(keep, "keep"));
  FM_TRY(need_aligned(idx, "idx")); FM_TRY(need_aligned(gate, "gate")); FM_TRY(need_aligned(counts, "counts"));
  const Gating dg = device_gating(g);
  // with counts every block adds its own histogram: fewer blocks, each several times
  const int blocks = cdiv(T, GT_TOK), most = counts ? 4 * device_cus() : 1 << 20;
  const dim3 grid(blocks < most ? blocks : most);
#define FM_GT(N)                                                                                              \
  hipLaunchKernelGGL(k_route_scored<N>, grid, dim3(256), 0, as_stream(stream), dg, logits, sel_bias, keep, T, idx, gate, \
                     counts)
  if (g->E <= 64) FM_GT(4);
  else if (g->E <= 128) FM_GT(8);
  else FM_GT(16);
#undef FM_GT
  return check_launch("moe_route_scored");
}

extern "C" int moe_route_scored_bwd(const moe_gating* g, const float* logits, const int32_t* idx, const float* dgate, int T,
                                    float* dlogits, int accumulate, void* stream) {
  clear_error();
  FM_TRY(check_gating(g, T));
  if (T == 0) return MOE_OK;
  FM_TRY(need(logits, "logits")); FM_TRY(need(idx, "idx")); FM_TRY(need(dgate, "dgate")); FM_TRY(need(dlogits, "dlogits"));
  FM_TRY(need_aligned(logits, "logits")); FM_TRY(need_aligned(idx, "idx")); FM_TRY(need_aligned(dgate, "dgate"));
  FM_TRY(need_aligned(dlogits, "dlogits"));
  if (accumulate && dlogits == logits) return fail(MOE_ERR_ARG, "dlogits must not alias logits when accumulating");
  const Gating dg = device_gating(g);
  // launches of less than 2^32 threads
  const int step = 1 << 27;
  for (int t = 0; t < T; t += step) {
    const int n = T - t < step ? T - t : step;
    const dim3 grid(cdiv(n, GT_TOK));
    const size_t r = (size_t)t;
#define FM_GT(N)                                                                                                   \
  hipLaunchKernelGGL(k_route_scored_bwd<N>, grid, dim3(256), 0, as_stream(stream), dg, logits + r * g->E, idx + r * g->k, \
                     dgate + r * g->k, n, dlogits + r * g->E, accumulate != 0)
    if (g->E <= 64) FM_GT(4);
    else if (g->E <= 128) FM_GT(8);
    else FM_GT(16);
#undef FM_GT
  }
  return check_launch("moe_route_scored_bwd");
}

extern "C" int moe_route_bias_update(const int32_t* counts, int E, float rate, float* sel_bias, void* stream) {
  clear_error();
  if (E <= 0) return fail(MOE_ERR_ARG, "E=%d", E);
  if (E > 256) return fail(MOE_ERR_UNSUPPORTED, "E=%d > 256", E);
  if (!(__builtin_fabsf(rate) < __builtin_inff())) return fail(MOE_ERR_ARG, "rate=%g", rate);
  FM_TRY(need(counts, "counts")); FM_TRY(need(sel_bias, "sel_bias"));
  FM_TRY(need_aligned(counts, "counts")); FM_TRY(need_aligned(sel_bias, "sel_bias"));
  hipLaunchKernelGGL(k_bias_update, dim3(1), dim3(256), 0, as_stream(stream), counts, E, rate, sel_bias);
  return check_launch("moe_route_bias_update");
}
