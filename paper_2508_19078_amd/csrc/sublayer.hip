// The norms around a block, forward and backward, in one pass over the rows:
// post-norm, gate and residual scale of the block's output into the stream, the
// stream's pre-norm, and the gradients of both (the formulas stand in the
// header at moe_sublayer_norm).
//
// Both directions are bound by memory: a row is read once, kept in registers
// over its reductions and written once.  A row belongs to TPR threads of a block
// (16 or 64 lanes of a wave, or the whole block), NCB chunks of 16 bytes each,
// chunk i of thread r at column (r + i TPR) V; a block of NT threads walks groups
// of NT / TPR rows, and the gains of a thread's columns stay in its registers over
// all of them.  The backward keeps its sums for the gains' gradients there too, in 64 bits
// (in 32, the 64 rows of a block at 32768 tokens cost three times the error of one
// rounding; the time grew by 1-2 %, by 5 % at d = 256), and leaves them, one row of partial sums per
// block, to a second launch that adds them in a fixed order (no float atomics).
//
// Measured at 8192 rows of 2048 bf16, post-norm and gate: forward 24.0 us (134 MB, 5.6
// TB/s), backward 39.2 us (201 MB, 5.1 TB/s) and 4.6 us for the second launch; 1023
// rows of 1000 fp32, pre-norm: 7.5 us and 4.2.  A single row of 4096 takes 4.6 us: a
// launch, one load's latency and two reductions.  (The second launch with 8 groups of
// threads per block, each adding 64 partial sums one after another, took 9.6 us.)
#include "common.hpp"

namespace fm {
namespace {

constexpr int SL_MAX_D = 8192;
constexpr int SL_MAX_BLOCKS = 512;   // blocks of the backward, and rows of its partial sums

// Sum of v over the TPR threads of a row; every thread gets the same bits.  red:
// two arrays of one float per wave, taken in turn by consecutive sums (turn): a
// wave that writes an array has passed the barrier of the sum in between, before
// which every wave had read it.
template <int TPR, int NW> __device__ __forceinline__ float row_sum(float v, float (*red_)[NW], int& turn) {
#pragma unroll
  for (int o = (TPR < 64 ? TPR : 64) / 2; o > 0; o >>= 1) v += __shfl_xor(v, o);
  if constexpr (TPR > 64) {
    float* const red = red_[turn];
    turn ^= 1;
    if (lane_id() == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < TPR / 64; ++w) v += red[w];
  }
  return v;
}

__device__ __forceinline__ float rstd_of(float ss, int d, float eps) {
  const float ms = ss / (float)d + eps;
  return ms > 0.f ? 1.0f / sqrtf(ms) : ms == 0.f ? 0.f : ms;   // NaN stays NaN
}

// The fp32 gains of V columns from c (1 where there are none).
template <int V> __device__ __forceinline__ void gains(const float* w, int c, bool on, float* out) {
#pragma unroll
  for (int i = 0; i < V; i += 4) {
    const u32x4_t raw = w && on ? ld16(w + c + i) : u32x4_t{0x3F800000u, 0x3F800000u, 0x3F800000u, 0x3F800000u};
    unpack16(raw, out + i, (float*)nullptr);
  }
}

struct NormFwd {
  const void *X, *Y;
  const float *gate, *w_post, *w_pre;
  int Tn, d, post;
  float alpha, eps;
  void *S, *N;
  float *rstd_y, *rstd_s;
};

template <typename T, int TPR, int NCB, int NT>
__global__ __launch_bounds__(NT) void k_sublayer(NormFwd a) {
  constexpr int V = 16 / sizeof(T), RPB = NT / TPR;
  __shared__ float red[2][NT / 64];
  int turn = 0;
  const int sub = threadIdx.x % TPR, rb = threadIdx.x / TPR;
  const T *X = (const T*)a.X, *Y = (const T*)a.Y;
  T *S = (T*)a.S, *N = (T*)a.N;
  const u32x4_t zero = {0, 0, 0, 0};
  float wq[NCB][V], wn[NCB][V];
#pragma unroll
  for (int i = 0; i < NCB; ++i) {
    const int c = (sub + i * TPR) * V;
    gains<V>(a.w_post, c, c < a.d, wq[i]);
    gains<V>(a.w_pre, c, c < a.d, wn[i]);
  }
  for (long g = blockIdx.x; g * RPB < a.Tn; g += gridDim.x) {
    const long row = g * RPB + rb;
    const bool live = row < a.Tn;
    const size_t base = (size_t)(live ? row : 0) * a.d;
    u32x4_t xv[NCB], yv[NCB];
#pragma unroll
    for (int i = 0; i < NCB; ++i) {
      const int c = (sub + i * TPR) * V;
      const bool on = live && c < a.d;
      xv[i] = on ? ld16(X + base + c) : zero;
      yv[i] = on && Y ? ld16(Y + base + c) : zero;
    }
    float gt = a.gate && live ? a.gate[row] : 1.f;
    if (a.post) {
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < NCB; ++i) {
        float y[V];
        unpack16(yv[i], y, (T*)nullptr);
#pragma unroll
        for (int e = 0; e < V; ++e) ss = fmaf(y[e], y[e], ss);
      }
      const float ry = rstd_of(row_sum<TPR, NT / 64>(ss, red, turn), a.d, a.eps);
      if (a.rstd_y && live && sub == 0) a.rstd_y[row] = ry;
      gt *= ry;
    }
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < NCB; ++i) {
      float x[V], y[V];
      unpack16(xv[i], x, (T*)nullptr);
      unpack16(yv[i], y, (T*)nullptr);
#pragma unroll
      for (int e = 0; e < V; ++e) x[e] = Y ? fmaf(gt, y[e] * wq[i][e], a.alpha * x[e]) : a.alpha * x[e];
      xv[i] = pack16(x, (T*)nullptr);
      unpack16(xv[i], x, (T*)nullptr);
#pragma unroll
      for (int e = 0; e < V; ++e) ss = fmaf(x[e], x[e], ss);
    }
    float rs = 0.f;
    if (N) {
      rs = rstd_of(row_sum<TPR, NT / 64>(ss, red, turn), a.d, a.eps);
      if (a.rstd_s && live && sub == 0) a.rstd_s[row] = rs;
    }
#pragma unroll
    for (int i = 0; i < NCB; ++i) {
      const int c = (sub + i * TPR) * V;
      if (!live || c >= a.d) continue;
      if (S) st16(S + base + c, xv[i]);
      if (N) {
        float x[V];
        unpack16(xv[i], x, (T*)nullptr);
#pragma unroll
        for (int e = 0; e < V; ++e) x[e] = x[e] * rs * wn[i][e];
        st16(N + base + c, pack16(x, (T*)nullptr));
      }
    }
  }
}

struct NormBwd {
  const void *dS, *dN, *S, *Y;
  const float *gate, *w_post, *w_pre, *rstd_y, *rstd_s;
  int Tn, d, post;
  float alpha;
  void *dX, *dY;
  float* dgate;
  float* part;   // [blocks][2][d]: sums of dw_post, then of dw_pre
  int want_post, want_pre;
};

template <typename T, int TPR, int NCB, int NT>
__global__ __launch_bounds__(NT) void k_sublayer_bwd(NormBwd a) {
  constexpr int V = 16 / sizeof(T), RPB = NT / TPR;
  __shared__ float red[2][NT / 64];
  int turn = 0;
  const int sub = threadIdx.x % TPR, rb = threadIdx.x / TPR;
  const T *dS = (const T*)a.dS, *dN = (const T*)a.dN, *S = (const T*)a.S, *Y = (const T*)a.Y;
  T *dX = (T*)a.dX, *dY = (T*)a.dY;
  const u32x4_t zero = {0, 0, 0, 0};
  float wq[NCB][V], wn[NCB][V];
  double gq[NCB][V], gn[NCB][V];
#pragma unroll
  for (int i = 0; i < NCB; ++i) {
    const int c = (sub + i * TPR) * V;
    gains<V>(a.w_post, c, c < a.d, wq[i]);
    gains<V>(a.w_pre, c, c < a.d, wn[i]);
#pragma unroll
    for (int e = 0; e < V; ++e) gq[i][e] = gn[i][e] = 0.;
  }
  const float id = 1.0f / (float)a.d;
  for (long g = blockIdx.x; g * RPB < a.Tn; g += gridDim.x) {
    const long row = g * RPB + rb;
    const bool live = row < a.Tn;
    const size_t base = (size_t)(live ? row : 0) * a.d;
    u32x4_t sv[NCB], yv[NCB], hv[NCB], nv[NCB];
#pragma unroll
    for (int i = 0; i < NCB; ++i) {
      const int c = (sub + i * TPR) * V;
      const bool on = live && c < a.d;
      sv[i] = on && dN ? ld16(S + base + c) : zero;
      nv[i] = on && dN ? ld16(dN + base + c) : zero;
      hv[i] = on && dS ? ld16(dS + base + c) : zero;
      yv[i] = on && Y ? ld16(Y + base + c) : zero;
    }
    const float rs = dN && live ? a.rstd_s[row] : 0.f;
    const float ry = a.post ? (live ? a.rstd_y[row] : 0.f) : 1.f;
    const float gt = a.gate && live ? a.gate[row] : 1.f;
    float D[NCB][V];
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < NCB; ++i) {
      float s[V], n[V];
      unpack16(sv[i], s, (T*)nullptr);
      unpack16(nv[i], n, (T*)nullptr);
      unpack16(hv[i], D[i], (T*)nullptr);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float xh = s[e] * rs;
        gn[i][e] += n[e] * xh;
        m = fmaf(n[e] * wn[i][e], xh, m);
      }
    }
    if (dN) {
      m = row_sum<TPR, NT / 64>(m, red, turn) * id;
#pragma unroll
      for (int i = 0; i < NCB; ++i) {
        float s[V], n[V];
        unpack16(sv[i], s, (T*)nullptr);
        unpack16(nv[i], n, (T*)nullptr);
#pragma unroll
        for (int e = 0; e < V; ++e) D[i][e] = fmaf(rs, fmaf(-s[e] * rs, m, n[e] * wn[i][e]), D[i][e]);
      }
    }
    if (dX) {
#pragma unroll
      for (int i = 0; i < NCB; ++i) {
        const int c = (sub + i * TPR) * V;
        float x[V];
#pragma unroll
        for (int e = 0; e < V; ++e) x[e] = a.alpha * D[i][e];
        if (live && c < a.d) st16(dX + base + c, pack16(x, (T*)nullptr));
      }
    }
    if (!Y) continue;
    // sum_i D u w_post: the gate's gradient, and gate times it the sum of dv u
    float q = 0.f;
#pragma unroll
    for (int i = 0; i < NCB; ++i) {
      float y[V];
      unpack16(yv[i], y, (T*)nullptr);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float Du = D[i][e] * (y[e] * ry);
        gq[i][e] += gt * Du;
        q = fmaf(Du, wq[i][e], q);
      }
    }
    if (a.dgate || a.post) q = row_sum<TPR, NT / 64>(q, red, turn);
    if (a.dgate && live && sub == 0) a.dgate[row] = q;
    if (dY) {
      const float mu = a.post ? gt * q * id : 0.f;
#pragma unroll
      for (int i = 0; i < NCB; ++i) {
        const int c = (sub + i * TPR) * V;
        float y[V];
        unpack16(yv[i], y, (T*)nullptr);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float dv = gt * D[i][e] * wq[i][e];
          y[e] = a.post ? ry * fmaf(-(y[e] * ry), mu, dv) : dv;
        }
        if (live && c < a.d) st16(dY + base + c, pack16(y, (T*)nullptr));
      }
    }
  }
  if (!a.part) return;
  // the rows of a block that share columns add up through LDS, group 0 first
  constexpr int WIDE = RPB > 1 ? TPR * NCB * V : 1;
  __shared__ double acc[WIDE];
  float* const part = a.part + (size_t)blockIdx.x * 2 * a.d;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    if (!(which ? a.want_pre : a.want_post)) continue;
    if constexpr (RPB > 1) {
      for (int r = 0; r < RPB; ++r) {
        __syncthreads();
        if (rb == r) {
#pragma unroll
          for (int i = 0; i < NCB; ++i)
#pragma unroll
            for (int e = 0; e < V; ++e) {
              double& v = which ? gn[i][e] : gq[i][e];
              double& at = acc[(sub + i * TPR) * V + e];
              v = at = r ? at + v : v;
            }
        }
      }
    }
    if (rb == RPB - 1) {
#pragma unroll
      for (int i = 0; i < NCB; ++i) {
        const int c = (sub + i * TPR) * V;
        if (c >= a.d) continue;
#pragma unroll
        for (int e = 0; e < V; e += 4) {
          float v[4];
#pragma unroll
          for (int x = 0; x < 4; ++x) v[x] = (float)(which ? gn[i][e + x] : gq[i][e + x]);
          st16(part + which * (size_t)a.d + c + e, pack16(v, (float*)nullptr));
        }
      }
    }
  }
}

// out[c] = (accumulate ? out[c] : 0) + the partial sums of column c: 32 columns per
// block (8 quads), its 128 groups of threads every 128th block's sums, which are then
// added pairwise.  In 64 bits: up to 512 sums of many rows each, which may nearly cancel.
__global__ __launch_bounds__(1024) void k_sublayer_dw(const float* __restrict__ part, int blocks, int d,
                                                      int accumulate, float* __restrict__ dw_post,
                                                      float* __restrict__ dw_pre) {
  typedef float f4 __attribute__((ext_vector_type(4)));
  typedef double d4 __attribute__((ext_vector_type(4)));
  __shared__ d4 red[128][8];
  const int which = blockIdx.y, q = threadIdx.x & 7, grp = threadIdx.x >> 3, c = blockIdx.x * 32 + 4 * q;
  float* const out = which ? dw_pre : dw_post;
  if (!out) return;
  d4 s = {0., 0., 0., 0.};
  if (c < d) {
#pragma unroll 4
    for (int b = grp; b < blocks; b += 128)
      s += __builtin_convertvector(*(const FM_GLOBAL f4*)(part + ((size_t)b * 2 + which) * d + c), d4);
  }
  red[grp][q] = s;
#pragma unroll
  for (int h = 64; h > 0; h >>= 1) {
    __syncthreads();
    if (grp < h) red[grp][q] = s += red[grp + h][q];
  }
  if (grp == 0 && c < d) {
    if (accumulate) s += __builtin_convertvector(*(const FM_GLOBAL f4*)(out + c), d4);
    *(FM_GLOBAL f4*)(out + c) = __builtin_convertvector(s, f4);
  }
}

// The threads per row for n chunks: 16 or 64 lanes where a lane then holds at
// most 2 chunks, else a block of 256 (up to 2 chunks each) or 1024.
template <int TPR_, int NCB_, int NT_> struct RowShape {
  static constexpr int TPR = TPR_, NCB = NCB_, NT = NT_;
};
template <typename T, typename Fn> void with_row_shape(int d, Fn fn) {
  const int n = d / (16 / (int)sizeof(T));
  if (n <= 16) fn(RowShape<16, 1, 256>{});
  else if (n <= 64) fn(RowShape<64, 1, 256>{});
  else if (n <= 128) fn(RowShape<64, 2, 256>{});
  else if (n <= 256) fn(RowShape<256, 1, 256>{});
  else if (n <= 512) fn(RowShape<256, 2, 256>{});
  else if (n <= 1024) fn(RowShape<1024, 1, 1024>{});
  else if constexpr (sizeof(T) == 4) fn(RowShape<1024, 2, 1024>{});   // d > 4096
}

template <typename T> void launch_fwd(const NormFwd& a, hipStream_t st) {
  with_row_shape<T>(a.d, [&](auto shape) {
    typedef decltype(shape) R;
    const int groups = cdiv(a.Tn, R::NT / R::TPR);
    const int most = device_cus() * (2048 / R::NT);
    hipLaunchKernelGGL((k_sublayer<T, R::TPR, R::NCB, R::NT>), dim3(groups < most ? groups : most), dim3(R::NT), 0, st, a);
  });
}

template <typename T> int launch_bwd(const NormBwd& a, hipStream_t st) {
  int blocks = 0;
  with_row_shape<T>(a.d, [&](auto shape) {
    typedef decltype(shape) R;
    const int groups = cdiv(a.Tn, R::NT / R::TPR);
    const int most = R::NT == 1024 ? SL_MAX_BLOCKS / 2 : SL_MAX_BLOCKS;
    blocks = groups < most ? groups : most;
    if (blocks > 0)
      hipLaunchKernelGGL((k_sublayer_bwd<T, R::TPR, R::NCB, R::NT>), dim3(blocks), dim3(R::NT), 0, st, a);
  });
  return blocks;
}

int check_norm_shape(int T, int d, int dtype) {
  FM_TRY(need_dtype_float(dtype, "dtype"));
  if (T < 0 || d <= 0) return fail(MOE_ERR_ARG, "T=%d d=%d", T, d);
  if (d % 8 || d > SL_MAX_D) return fail(MOE_ERR_UNSUPPORTED, "d=%d must be a multiple of 8 up to %d", d, SL_MAX_D);
  return MOE_OK;
}
int need_finite(float v, const char* name) {
  if (!(v > -3e38f && v < 3e38f)) return fail(MOE_ERR_ARG, "%s=%g must be finite", name, (double)v);
  return MOE_OK;
}

}  // namespace
}  // namespace fm

using namespace fm;

extern "C" int moe_sublayer_norm(const void* X, const void* Y, const float* gate, const float* w_post,
                                 const float* w_pre, int T, int d, int dtype, float alpha, int post_norm, float eps,
                                 void* S, void* N, float* rstd_y, float* rstd_s, void* stream) {
  clear_error();
  FM_TRY(check_norm_shape(T, d, dtype));
  FM_TRY(need_finite(alpha, "alpha"));
  if (!(eps >= 0.f && eps < 1e30f)) return fail(MOE_ERR_ARG, "eps=%g must be finite and >= 0", (double)eps);
  if (!Y && (T > 0) && (gate || w_post || rstd_y || post_norm))
    return fail(MOE_ERR_ARG, "without Y, gate, w_post and rstd_y must be NULL and post_norm 0");
  if (!post_norm && rstd_y) return fail(MOE_ERR_ARG, "rstd_y without post_norm");
  if (T == 0) return MOE_OK;
  FM_TRY(need(X, "X"));
  if (!S && !N) return fail(MOE_ERR_ARG, "S and N must not both be NULL");
  if (!N && rstd_s) return fail(MOE_ERR_ARG, "rstd_s without N");
  if (S && S == N) return fail(MOE_ERR_ARG, "S and N must not alias each other");
  FM_TRY(need_aligned(X, "X")); FM_TRY(need_aligned(Y, "Y")); FM_TRY(need_aligned(gate, "gate"));
  FM_TRY(need_aligned(w_post, "w_post")); FM_TRY(need_aligned(w_pre, "w_pre")); FM_TRY(need_aligned(S, "S"));
  FM_TRY(need_aligned(N, "N")); FM_TRY(need_aligned(rstd_y, "rstd_y")); FM_TRY(need_aligned(rstd_s, "rstd_s"));
  const NormFwd a{X, Y, gate, w_post, w_pre, T, d, post_norm ? 1 : 0, alpha, eps, S, N, rstd_y, rstd_s};
  if (dtype == MOE_BF16) launch_fwd<bf16>(a, as_stream(stream));
  else launch_fwd<float>(a, as_stream(stream));
  return check_launch("moe_sublayer_norm");
}

extern "C" size_t moe_sublayer_norm_bwd_workspace_size(int T, int d) {
  if (T < 0 || d <= 0) return 0;
  return (size_t)(T < SL_MAX_BLOCKS ? T : SL_MAX_BLOCKS) * 2 * d * sizeof(float);
}

extern "C" int moe_sublayer_norm_bwd(const void* dS, const void* dN, const void* S, const void* Y, const float* gate,
                                     const float* w_post, const float* w_pre, const float* rstd_y,
                                     const float* rstd_s, int T, int d, int dtype, float alpha, int post_norm,
                                     void* dX, void* dY, float* dgate, float* dw_post, float* dw_pre,
                                     int accumulate_dw, void* ws, size_t ws_bytes, void* stream) {
  clear_error();
  FM_TRY(check_norm_shape(T, d, dtype));
  FM_TRY(need_finite(alpha, "alpha"));
  if (T > 0) {
    if (!dS && !dN) return fail(MOE_ERR_ARG, "dS and dN must not both be NULL");
    if (dN) { FM_TRY(need(S, "S")); FM_TRY(need(rstd_s, "rstd_s")); }
    if (!Y && (gate || w_post || post_norm || dY || dgate || dw_post))
      return fail(MOE_ERR_ARG, "without Y, gate, w_post, dY, dgate and dw_post must be NULL and post_norm 0");
    if (post_norm) FM_TRY(need(rstd_y, "rstd_y"));
    if (dX && dX == dY) return fail(MOE_ERR_ARG, "dX and dY must not alias each other");
  }
  FM_TRY(need_aligned(dS, "dS")); FM_TRY(need_aligned(dN, "dN")); FM_TRY(need_aligned(S, "S"));
  FM_TRY(need_aligned(Y, "Y")); FM_TRY(need_aligned(gate, "gate")); FM_TRY(need_aligned(w_post, "w_post"));
  FM_TRY(need_aligned(w_pre, "w_pre")); FM_TRY(need_aligned(rstd_y, "rstd_y")); FM_TRY(need_aligned(rstd_s, "rstd_s"));
  FM_TRY(need_aligned(dX, "dX")); FM_TRY(need_aligned(dY, "dY")); FM_TRY(need_aligned(dgate, "dgate"));
  FM_TRY(need_aligned(dw_post, "dw_post")); FM_TRY(need_aligned(dw_pre, "dw_pre")); FM_TRY(need_aligned(ws, "ws"));
  const bool dw = dw_post || dw_pre;
  if (dw && T > 0) {
    FM_TRY(need(ws, "ws"));
    if (ws_bytes < moe_sublayer_norm_bwd_workspace_size(T, d))
      return fail(MOE_ERR_WORKSPACE, "workspace %zu < %zu bytes", ws_bytes, moe_sublayer_norm_bwd_workspace_size(T, d));
  }
  if (T == 0 && (!dw || accumulate_dw)) return MOE_OK;
  hipStream_t st = as_stream(stream);
  int blocks = 0;
  if (T > 0) {
    const NormBwd a{dS, dN, S, Y, gate, w_post, w_pre, rstd_y, rstd_s, T, d, post_norm ? 1 : 0, alpha, dX, dY, dgate,
                    dw ? (float*)ws : nullptr, dw_post != nullptr, dw_pre != nullptr};
    blocks = dtype == MOE_BF16 ? launch_bwd<bf16>(a, st) : launch_bwd<float>(a, st);
    FM_TRY(check_launch("moe_sublayer_norm_bwd"));
  }
  if (dw) {
    hipLaunchKernelGGL(k_sublayer_dw, dim3(cdiv(d, 32), 2), dim3(1024), 0, st, (const float*)ws, blocks, d, accumulate_dw,
                       dw_post, dw_pre);
    FM_TRY(check_launch("moe_sublayer_norm_bwd"));
  }
  return MOE_OK;
}
