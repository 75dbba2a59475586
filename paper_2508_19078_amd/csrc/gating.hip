// Routing from the router's logits by scores (the formulas stand in the header at
// moe_route_scored): softmax or sigmoid scores, a bias on the selection, expert groups,
// top-k, and the gradient of the logits.
//
// 16 lanes per token, four tokens per wave: lane q holds experts 64 c + 4 q to + 3 for
// chunks c, as they lie in memory.
//
// The selection is that of keys in fp64 (or of the logits, exactly), but it is made on 32
// bits: a key's distance from the bottom of a window below the largest, in 24 bits, then
// 255 - expert, so that one unsigned maximum finds a round's winner and its index, and the
// next round's is the largest of the differences to it that wrap.  The map to 24 bits does
// not decrease (it is held to them at both ends), so where neighbours in rank order (the first one left out among them)
// differ by more than the fp32 keys' error, and the worst group kept and the best one not
// do, the selection is the exact one.  Elsewhere fp64 decides, on as few keys as it takes (a
// kernel of 32768 tokens always meets some such, and waits for its slowest wave): the
// largest keys of groups that are near the border; the 16 first in rank order, a lane each,
// if the last of them is clearly behind the k-th; all keys where that does not hold or the
// largest is no number.
#include "common.hpp"
#include "ffn_common.hpp"

namespace fm {
namespace {

constexpr int GT_TOK = 16;   // tokens per block of four waves
constexpr int GT_MAXK = 16, GT_MAXG = 32;
constexpr int NOBODY = 0x7FFFFFFF;

struct Gating {
  int E, k, n_group, topk_group, group_top;
  int size;    // experts of a group
  int lanes;   // lanes of a chunk that hold a group of 4, 8, .. 64 experts, or 0
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

__device__ __forceinline__ uint32_t larger3(uint32_t a, uint32_t b, uint32_t c) { return max(max(a, b), c); }
__device__ __forceinline__ uint32_t row_max_u(uint32_t x) {
  x = max(x, (uint32_t)ror<8>((int)x));
  x = max(x, (uint32_t)ror<4>((int)x));
  x = max(x, (uint32_t)ror<2>((int)x));
  return max(x, (uint32_t)ror<1>((int)x));
}

// Expert of place i of lane q.
__device__ __forceinline__ int expert_at(int i, int q) { return 64 * (i / 4) + 4 * q + i % 4; }

// The rows' logits, NaN as -inf, -inf behind E.
template <int N> __device__ __forceinline__ void load_logits(const float* zr, int E, int q, float (&z)[N]) {
  const float none = minus_inf<float>();
  if ((E & 3) == 0) {   // rows of whole 16-byte chunks
#pragma unroll
    for (int c = 0; c < N / 4; ++c) {
      u32x4_t v = {0, 0, 0, 0};
      const int e = expert_at(4 * c, q);
      if (e < E) v = ld16(zr + e);
#pragma unroll
      for (int b = 0; b < 4; ++b) z[4 * c + b] = e < E ? __builtin_fmaxf(__uint_as_float(v[b]), none) : none;
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int e = expert_at(i, q);
      z[i] = e < E ? __builtin_fmaxf(gptr(zr)[e], none) : none;
    }
  }
}

// Scores with the hardware's exponential and reciprocal, for deciding a selection and a
// softmax's denominator.  Steps of 2^-24 of a score (below 1): sigmoid 4 (the exponent's
// rounding weighs |z| s (1 - s) < 1/4, exponential and reciprocal 2 each), softmax 3 and
// its sum's 20, common to a row.  total: a softmax's sum; m its largest logit.
template <int N> __device__ __forceinline__ void fast_scores(const Gating& g, const float (&z)[N], float (&s)[N], float& m, float& total) {
  constexpr float L2E = 1.4426950408889634f;
  if (g.sigmoid) {
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-L2E * z[i]));
    return;
  }
  m = z[0];
#pragma unroll
  for (int i = 1; i < N; ++i) m = larger(m, z[i]);
  m = row_max(m);
  float sum = 0.f;
  if (__any(!(fabsf(m) < __builtin_inff()))) {
#pragma unroll
    for (int i = 0; i < N; ++i) sum += s[i] = softmax_part(z[i], m);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) sum += s[i] = __builtin_amdgcn_exp2f((z[i] - m) * L2E);
  }
  total = row_sum(sum);
  const float inv = total > 0.f ? 1.f / total : 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) s[i] *= inv;
}

// The two largest of two lanes' (h, l), h >= l, by a DPP control.
template <int CTRL> __device__ __forceinline__ void merge_two(float& h, float& l) {
  const float h2 = dpp_f<CTRL>(h), l2 = dpp_f<CTRL>(l);
  l = larger(larger(fminf(h, h2), l), l2);
  h = larger(h, h2);
}

// Between what a group's rank r in fp32, of its largest key h and its second l (if two
// count), lies in fp64.  A key is off by its score's error err and half a step of its own, which a
// bias can make far larger than the largest key's; the sum by half a step.  Steps count
// twice here, which covers the roundings of the bounds.  A rank that fp32 cannot hold is
// beyond all that it can; infinite keys are exact.
__device__ __forceinline__ void rank_bounds(float h, float l, float r, bool two, float err, float& lo, float& hi) {
  const float inf = __builtin_inff();
  const float e = two ? 2 * err + 0x1p-23f * (fabsf(h) + fabsf(l) + fabsf(r)) : err + 0x1p-23f * fabsf(h);
  const bool fits = fabsf(r) < inf, over = two && l > -inf;
  lo = fits ? r - e : over && r > 0 ? 0x1.fp127f : r;
  hi = fits ? r + e : over && r < 0 ? -0x1.fp127f : r;
}

// Which of this lane's chunks lie in a group that stays (bits), from the groups' keys.
// Groups of 4, 8, .. 64 experts are lanes of one chunk; of others the ranks are read from
// LDS key by key and bits has one per expert.  near: where a group kept and one not may
// have changed places by the error err of their keys' scores (0: keys are exact, ties as
// defined), the experts that decide between such groups, which are those not clearly below
// what their group ranks by.
template <int N>
__device__ __forceinline__ uint32_t groups_kept(const Gating& g, const float (&of)[N], float err, float* row, uint32_t& near) {
  const int q = lane_id() & 15;
  const float none = minus_inf<float>();
  const bool two = g.group_top == 2;
  float worst = -none, best = none;   // the least that a kept group's rank may be, the most that another's may
  uint32_t left = 0;
  if (g.lanes > 0) {
    float r[N / 4], last[N / 4], lo[N / 4], hi[N / 4];   // ranks, the least key in them, their bounds
    const int mine = q / g.lanes, per = 16 / g.lanes;
#pragma unroll
    for (int c = 0; c < N / 4; ++c) {
      const float a = of[4 * c], b = of[4 * c + 1], x = of[4 * c + 2], y = of[4 * c + 3];
      const float h1 = larger(a, b), l1 = fminf(a, b), h2 = larger(x, y), l2 = fminf(x, y);
      float h = larger(h1, h2), l = larger(larger(fminf(h1, h2), l1), l2);
      if (g.lanes > 1) merge_two<0xB1>(h, l);     // quad_perm [1, 0, 3, 2]
      if (g.lanes > 2) merge_two<0x4E>(h, l);     // quad_perm [2, 3, 0, 1]
      if (g.lanes > 4) merge_two<0x141>(h, l);    // row_half_mirror
      if (g.lanes > 8) merge_two<0x140>(h, l);    // row_mirror
      r[c] = two ? __builtin_fmaxf(h + l, none) : h;
      last[c] = two ? l : h;
      rank_bounds(h, l, r[c], two, err, lo[c], hi[c]);
      const int grp = c * per + mine;
      if (q % g.lanes == 0 && grp < g.n_group) row[grp] = r[c];
    }
    wave_lds_fence();
    int ahead[N / 4];
#pragma unroll
    for (int c = 0; c < N / 4; ++c) ahead[c] = 0;
    for (int o = 0; o < g.n_group; ++o) {
      const float v = row[o];
#pragma unroll
      for (int c = 0; c < N / 4; ++c) ahead[c] += v > r[c] || (v == r[c] && o < c * per + mine);
    }
#pragma unroll
    for (int c = 0; c < N / 4; ++c) {
      if (c * per + mine >= g.n_group) continue;
      if (ahead[c] < g.topk_group) {
        left |= 15u << (4 * c);
        worst = fminf(worst, lo[c]);
      } else {
        best = larger(best, hi[c]);
      }
    }
    worst = -row_max(-worst);
    best = row_max(best);
    if (err > 0.f && !(worst > best))
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int c = i / 4;
        const bool open = left >> i & 1 ? lo[c] <= best : hi[c] >= worst;
        if (open && !(of[i] < last[c] - (2 * err + 0x1p-22f * fabsf(last[c])))) near |= 1u << i;
      }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (expert_at(i, q) < g.E) row[expert_at(i, q)] = of[i];
    wave_lds_fence();
    // lane q ranks groups q and q + 16
    float r[2], lo[2], hi[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float a = none, b = none;
      if (q + 16 * h < g.n_group)
        for (int i = 0; i < g.size; ++i) {
          const float v = row[(q + 16 * h) * g.size + i];
          b = larger(b, fminf(v, a));
          a = larger(a, v);
        }
      r[h] = two ? __builtin_fmaxf(a + b, none) : a;
      rank_bounds(a, b, r[h], two, err, lo[h], hi[h]);
    }
    wave_lds_fence();
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (q + 16 * h < g.n_group) row[q + 16 * h] = r[h];
    wave_lds_fence();
    uint32_t in = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int grp = q + 16 * h;
      int ahead = 0;
      for (int o = 0; o < g.n_group; ++o) ahead += before(row[o], o, r[h], grp);
      if (grp >= g.n_group) continue;
      if (ahead < g.topk_group) {
        in |= 1u << grp;
        worst = fminf(worst, lo[h]);
      } else {
        best = larger(best, hi[h]);
      }
    }
    in = (uint32_t)row_fold((int)in, [](int a, int b) { return a | b; });
#pragma unroll
    for (int i = 0; i < N; ++i) left |= (in >> (min(expert_at(i, q), g.E - 1) / g.size) & 1u) << i;
    worst = -row_max(-worst);
    best = row_max(best);
    if (err > 0.f && !(worst > best)) near = ~0u;
  }
  wave_lds_fence();
  return left;
}

// A row of keys in LDS: 16 N of experts, then 32 for the groups' ranks.
template <int N> constexpr int key_row = 16 * N + GT_MAXG;

// Scores of a row in fp64 (loops that are not unrolled: this code is there in case).
struct ExactScores {
  const float* zr;
  bool sigmoid;
  double m, sum;
  __device__ __forceinline__ ExactScores(const Gating& g, const float* zr_, int places) : zr(zr_), sigmoid(g.sigmoid) {
    m = minus_inf<double>(), sum = 0;
    if (sigmoid) return;
    const int q = lane_id() & 15;
#pragma nounroll
    for (int i = 0; i < places; ++i)
      if (expert_at(i, q) < g.E) m = larger(m, logit(expert_at(i, q)));
    m = row_max(m);
#pragma nounroll
    for (int i = 0; i < places; ++i)
      if (expert_at(i, q) < g.E) sum += softmax_part(logit(expert_at(i, q)), m);
    sum = row_sum(sum);
  }
  __device__ __forceinline__ double logit(int e) const { return number(gptr(zr)[e]); }
  __device__ __forceinline__ double of(int e) const {
    return sigmoid ? logistic<double>(logit(e)) : sum > 0 ? softmax_part(logit(e), m) / sum : 0.0;
  }
};

// The groups that stay (bits), by ranks of the keys in a row of LDS.
__device__ __forceinline__ uint32_t groups_exact(const Gating& g, const double* row, double* ranks) {
  const int q = lane_id() & 15;
  double r[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    double a = minus_inf<double>(), b = a;
    if (q + 16 * h < g.n_group)
#pragma unroll 4
      for (int i = 0; i < g.size; ++i) {
        const double v = row[(q + 16 * h) * g.size + i];
        b = larger(b, v < a ? v : a);
        a = larger(a, v);
      }
    r[h] = g.group_top == 2 ? number(a + b) : a;
    if (q + 16 * h < g.n_group) ranks[q + 16 * h] = r[h];
  }
  wave_lds_fence();
  uint32_t kept = 0;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    int ahead = 0;
#pragma unroll 4
    for (int o = 0; o < g.n_group; ++o) ahead += before(ranks[o], o, r[h], q + 16 * h);
    if (q + 16 * h < g.n_group && ahead < g.topk_group) kept |= 1u << (q + 16 * h);
  }
  wave_lds_fence();
  return (uint32_t)row_fold((int)kept, [](int a, int b) { return a | b; });
}

// This lane's experts in the groups of `kept`.
__device__ __forceinline__ uint32_t in_groups(const Gating& g, uint32_t kept, int places) {
  const int q = lane_id() & 15;
  uint32_t left = 0;
#pragma nounroll
  for (int i = 0; i < places; ++i) {
    const int e = expert_at(i, q);
    if (e < g.E && (g.n_group == 1 || (kept >> (e / g.size) & 1))) left |= 1u << i;
  }
  return left;
}

// groups_kept's bits, one per expert, with fp64 keys of the experts in near.
template <bool BIAS, int N>
__device__ __forceinline__ uint32_t near_groups(const Gating& g, const float (&of)[N], const float* zr, const float* sel_bias,
                                                uint32_t near, double* row) {
  const int q = lane_id() & 15;
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (expert_at(i, q) < g.E) row[expert_at(i, q)] = of[i];
  const ExactScores s(g, zr, N);
#pragma nounroll
  for (int i = 0; i < N; ++i) {
    const int e = expert_at(i, q);
    const bool mine = (near >> i & 1) && e < g.E;
    if (!__any(mine)) continue;
    if (mine) row[e] = BIAS ? number(s.of(e) + (double)gptr(sel_bias)[e]) : s.of(e);
  }
  wave_lds_fence();
  return in_groups(g, groups_exact(g, row, row + 16 * N), N);
}

// The selection from keys in fp64 (BIAS) or the logits, group ranks in fp64, of a wave's
// four tokens.  Returns the choice of rank q.
template <bool BIAS, int N>
__device__ __forceinline__ int select_exact(const Gating& g, const float* zr, const float* sel_bias, double* row) {
  const int q = lane_id() & 15;
  const bool ranks = g.n_group > 1 && g.group_top == 2;
  auto put = [&](auto key) {
#pragma nounroll
    for (int i = 0; i < N; ++i)
      if (expert_at(i, q) < g.E) row[expert_at(i, q)] = key(expert_at(i, q));
    wave_lds_fence();
  };
  const ExactScores s(g, zr, BIAS || ranks ? N : 0);
  uint32_t kept = ~0u;
  if (BIAS) put([&](int e) { return number(s.of(e) + (double)gptr(sel_bias)[e]); });
  else if (ranks) put([&](int e) { return s.of(e); });
  else put([&](int e) { return s.logit(e); });
  if (g.n_group > 1) kept = groups_exact(g, row, row + 16 * N);
  if (!BIAS && ranks) put([&](int e) { return s.logit(e); });
  uint32_t left = in_groups(g, kept, N);
  int mine = 0;
#pragma nounroll
  for (int j = 0; j < g.k; ++j) {
    double v = minus_inf<double>();
    int e = NOBODY;
#pragma unroll 2
    for (int i = 0; i < N; ++i) {
      const int ei = expert_at(i, q);
      const double vi = row[min(ei, g.E - 1)];
      if ((left >> i & 1) && before(vi, ei, v, e)) v = vi, e = ei;
    }
    auto step = [&](double v2, int e2) {
      if (before(v2, e2, v, e)) v = v2, e = e2;
    };
    step(ror<8>(v), ror<8>(e));
    step(ror<4>(v), ror<4>(e));
    step(ror<2>(v), ror<2>(e));
    step(ror<1>(v), ror<1>(e));
    if (q == (e >> 2 & 15)) left &= ~(1u << (4 * (e >> 6) + (e & 3)));
    if (q == j) mine = e;
  }
  wave_lds_fence();
  return mine;
}

// The first n <= 16 experts in rank order, lane q's the q-th, put in order by keys in fp64
// (BIAS) or the logits.  Returns the choice of rank q.
template <bool BIAS, int N>
__device__ __forceinline__ int order_exact(const Gating& g, const float* zr, const float* sel_bias, int e, int n, double* row) {
  const int q = lane_id() & 15;
  const bool on = q < n;
  e = on ? e : 0;
  const ExactScores s(g, zr, BIAS ? N : 0);
  const double key = BIAS ? number(s.of(e) + (double)gptr(sel_bias)[e]) : s.logit(e);
  int* const who = (int*)(row + 16);
  row[q] = key;
  who[q] = e;
  wave_lds_fence();
  int ahead = 0;
  for (int o = 0; o < n; ++o) ahead += before(row[o], who[o], key, e);
  wave_lds_fence();
  if (on) who[ahead] = e;
  wave_lds_fence();
  e = who[q];
  wave_lds_fence();
  return e;
}

// N / 4 chunks of 64 experts.  WAVES: 4, or with counts, which each block adds to memory from
// a histogram of its own, as many as the registers allow (additions to one address come
// some 17 ns apart, whatever block they are of: 512 blocks cost 8.6 us).
//
// Bound by the rounds' vector instructions, and by latency at few tokens: 1 token 3.3 us; 1000
// of 60 experts, top-5, 5.6; 8192 of 64, top-6 in groups, 5.8 without counts and 10.1 with; 32768
// of 256, top-8 from 4 of 8 groups, 35 and 38.6 (34 MB: 6.6 us of bytes).  Selecting on fp64 keys
// throughout, that last pass and its gradient took 136 us in place of 50.
template <int N, bool BIAS, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void k_route_scored(Gating g, const float* __restrict__ logits,
                                                      const float* __restrict__ sel_bias, const uint8_t* __restrict__ keep,
                                                      int T, int32_t* __restrict__ idx, float* __restrict__ gate,
                                                      int32_t* __restrict__ counts) {
  constexpr int TOK = 4 * WAVES;
  __shared__ double rows[TOK][key_row<N>];
  __shared__ int hist[16 * N];
  const int lane = lane_id(), q = lane & 15, tok = threadIdx.x >> 4;
  if (counts) {
    for (int e = threadIdx.x; e < g.E; e += 64 * WAVES) hist[e] = 0;
    __syncthreads();
  }
  float bias[N];
  if (BIAS) {
#pragma unroll
    for (int i = 0; i < N; ++i) bias[i] = gptr(sel_bias)[min(expert_at(i, q), g.E - 1)];
  }
  for (int t0 = blockIdx.x * TOK; t0 < T; t0 += gridDim.x * TOK) {
    const int t = t0 + tok, tc = min(t, T - 1);   // rows behind the last token repeat it
    const float* const zr = logits + (size_t)tc * g.E;
    float z[N], s[N], m = 0.f, total = 0.f;
    load_logits<N>(zr, g.E, q, z);
    bool sure = true;
    const bool two = g.n_group > 1 && g.group_top == 2;
    if (BIAS || two || (!g.sigmoid && !g.renorm)) fast_scores<N>(g, z, s, m, total);
    // a score's error, and that of the difference of two keys: half a step of each besides
    const float err = g.sigmoid ? 0x1p-22f : 0x1p-19f;
    float gap = 2 * err;
    float top = minus_inf<float>();
    uint32_t left = ~0u;
    // keys, into s with a bias
    if (BIAS) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        s[i] = __builtin_fmaxf(s[i] + bias[i], minus_inf<float>());
        if (expert_at(i, q) >= g.E) s[i] = minus_inf<float>();
        top = larger(top, s[i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) top = larger(top, z[i]);
    }
    top = row_max(top);
    constexpr float WINDOW = BIAS ? 2.f : 32.f;
    if (BIAS) gap += 0x1p-23f * (fabsf(top) + WINDOW);
    if (g.n_group > 1) {
      uint32_t near = 0;
      if (BIAS || two) left = groups_kept<N>(g, s, 1.0625f * err, (float*)rows[tok], near);
      else left = groups_kept<N>(g, z, 0.f, (float*)rows[tok], near);
      if (__any(near != 0)) left = near_groups<BIAS, N>(g, s, zr, sel_bias, near, rows[tok]);
    }
    if (!(fabsf(top) < __builtin_inff())) sure = false;
    // packed keys: 1 + the distance from the window's bottom, then 255 - expert; 0: cannot be
    // chosen.  (The bottom may be rounded down, by more than the window far from zero: the
    // distance is held to 24 bits, and keys that meet at the end of them are not apart.)
    constexpr float UNITS = 0xFFFFFE.0p0f / WINDOW;
    const float bottom = top - WINDOW;
    uint32_t pk[N];
    const uint32_t base = 256 + 255 - 4 * q;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float d = __builtin_amdgcn_fmed3f(((BIAS ? s[i] : z[i]) - bottom) * UNITS, 0.f, 0xFFFFFE.0p0f);
      const uint32_t v = ((uint32_t)d << 8) + (base - expert_at(i, 0));
      pk[i] = expert_at(i, q) < g.E && (left >> i & 1) ? v : 0u;
    }
    uint32_t win = 0;
#pragma unroll
    for (int i = 0; i < N; i += 2) win = larger3(win, pk[i], pk[i + 1]);
    win = row_max_u(win);
    // (two keys, two units of rounding and one of the cut; with more than the window nothing is apart)
    const uint32_t need = BIAS ? (uint32_t)fminf(gap * UNITS, 0x1p25f) + 4u : 1u;
    const int places = g.topk_group * g.size, rounds = min(g.k + 1, places);
    int mine = 0;
    uint32_t kth = 0;
    bool apart = true;   // neighbours in rank order
    auto following = [&] {
      uint32_t next = 0;
#pragma unroll
      for (int i = 0; i < N; i += 2) next = larger3(next, pk[i] - win, pk[i + 1] - win);   // those below win wrap
      return row_max_u(next) + win;
    };
    for (int j = 0;; ++j) {
      if (q == j) mine = 255 - (int)(win & 255u);
      if (j == g.k - 1) kth = win >> 8;
      if (j + 1 >= rounds) break;
      const uint32_t next = following();
      if ((win >> 8) - (next >> 8) < need) apart = false;
      win = next;
    }
    if (__any(!sure)) {
      mine = select_exact<BIAS, N>(g, zr, sel_bias, rows[tok]);
    } else if (__any(!apart)) {
      const int more = min(16, places);
      for (int j = rounds; j < more; ++j) {
        win = following();
        if (q == j) mine = 255 - (int)(win & 255u);
      }
      if (__any(places > 16 && kth - (win >> 8) < need)) mine = select_exact<BIAS, N>(g, zr, sel_bias, rows[tok]);
      else mine = order_exact<BIAS, N>(g, zr, sel_bias, mine, more, rows[tok]);
    }
    // gates: lane j the choice of rank j
    const bool on = q < g.k;
    const float zj = on ? number(gptr(zr)[mine]) : minus_inf<float>();
    float w, S = 1.f;
    if (g.renorm) {
      const float mj = row_max(zj);
      w = g.sigmoid ? logistic(zj, fminf(mj, 0.f)) : softmax_part(zj, mj);
      if (!on) w = 0.f;
      S = row_sum(w);
    } else if (g.sigmoid) {
      w = logistic(zj);
    } else {
      w = softmax_part(zj, m);
      S = total;
    }
    if (on && t < T) {
      idx[(size_t)t * g.k + q] = mine;
      gate[(size_t)t * g.k + q] = S > 0.f ? g.scale * (w / S) : 0.f;
      if (counts && (!keep || keep[t])) atomicAdd(&hist[mine], 1);
    }
  }
  if (counts) {
    __syncthreads();
    for (int e = threadIdx.x; e < g.E; e += 64 * WAVES)
      if (hist[e]) atomicAdd(&counts[e], hist[e]);
  }
}

// The logits' gradient: lane j forms the share of choice j, the shares meet in an LDS row,
// which goes out 16 bytes per lane.  Bound by the bytes of dlogits: 32768 x 256 in 11.2
// us (36 MB, 3.2 TB/s), 8192 x 64 in 4.0.
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
    load_logits<N>(zr, g.E, q, z);
#pragma unroll
    for (int i = 0; i < N; ++i) m = larger(m, z[i]);
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
  for (int c = 0; c < N / 4; ++c) {
    const int e0 = expert_at(4 * c, q);
    if (e0 >= g.E) continue;
    u32x4_t v = *(const u32x4_t*)(row + e0);
    if (dense)
#pragma unroll
      for (int b = 0; b < 4; ++b) v[b] = __float_as_uint(z[4 * c + b] * (__uint_as_float(v[b]) - inner));
    if ((g.E & 3) == 0) {
      if (accumulate) {
        const u32x4_t old = ld16(out + e0);
#pragma unroll
        for (int b = 0; b < 4; ++b) v[b] = __float_as_uint(__uint_as_float(old[b]) + __uint_as_float(v[b]));
      }
      st16(out + e0, v);
    } else {
#pragma unroll
      for (int b = 0; b < 4; ++b)
        if (e0 + b < g.E) gptr(out)[e0 + b] = accumulate ? gptr(out)[e0 + b] + __uint_as_float(v[b]) : __uint_as_float(v[b]);
    }
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
  const int size = g->E / n, lanes = size >= 4 && size <= 64 && (size & (size - 1)) == 0 ? size / 4 : 0;
  return Gating{g->E, g->k, n, n == 1 ? 1 : g->topk_group, g->group_top, size, lanes, g->score == MOE_SCORE_SIGMOID,
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
  // (16 waves of 128 registers hold up to 128 experts, 8 waves 256)
  const bool wide = counts && T > 2048;
  const int waves = !wide ? 4 : g->E <= 128 ? 16 : 8;
  const int blocks = cdiv(T, 4 * waves), most = wide ? device_cus() : 1 << 20;
  const dim3 grid(blocks < most ? blocks : most);
#define FM_GT(N, BIAS, WAVES)                                                                                            \
  hipLaunchKernelGGL((k_route_scored<N, BIAS, WAVES>), grid, dim3(64 * WAVES), 0, as_stream(stream), dg, logits, sel_bias, \
                     keep, T, idx, gate, counts)
#define FM_GT_B(N, WIDE)                                             \
  if (wide) { if (sel_bias) FM_GT(N, true, WIDE); else FM_GT(N, false, WIDE); } \
  else { if (sel_bias) FM_GT(N, true, 4); else FM_GT(N, false, 4); }
  if (g->E <= 64) { FM_GT_B(4, 16) }
  else if (g->E <= 128) { FM_GT_B(8, 16) }
  else { FM_GT_B(16, 8) }
#undef FM_GT_B
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
