// The global norm of a step's gradients and their clipped copies (the formulas stand in
// the header at moe_grad_norm and moe_grad_clip).
//
// All tensors of a set together are one run of elements, which is cut into equal ranges,
// one per wave: a wave finds the tensor its range begins in (64 starts per probe) and
// walks on from there, so that neither many small tensors nor a few large ones leave
// waves idle.  A segment of a tensor is read 16 bytes per lane from its first aligned
// element on; what is before and behind goes element by element.  Both passes are bound
// by HBM.  Squares are taken and summed in fp64 (no overflow of large gradients, no loss
// of small ones; two vector instructions per element, less than the loads take).
//
// 571 million fp32 elements in 198 tensors: squares in 411 us (5.6 TB/s), clipped copies in
// 890 (5.1 TB/s of reads and writes).  786 KB in 24: 3.3 us, 1.8 to 4.8 for the sum of the
// blocks' parts, 3.3: launches.
#include "common.hpp"

namespace fm {
namespace {

constexpr int GN_BLOCKS = 1024;   // most blocks: 16 waves per compute unit
constexpr int GN_BATCH = 4;       // 16-byte loads a lane has in flight

struct TensorSet {
  void* const* data;
  const int64_t* start;
  int n;
  int64_t total;
};

// The last tensor that begins at or before element x (0 if there is none).
__device__ __forceinline__ int tensor_at(const TensorSet& g, int64_t x) {
  int a = 0, b = g.n;
  while (b - a > 1) {
    const int step = (b - a + 63) / 64, i = a + lane_id() * step;
    const int below = __builtin_popcountll(__ballot(i < b && gptr(g.start)[min(i, b - 1)] <= x));
    a += max(below - 1, 0) * step;
    b = min(b, a + step);
  }
  return __builtin_amdgcn_readfirstlane(a);
}

// Calls f(i, first element within tensor i, elements) for the parts of tensors in
// [x, end), frozen tensors left out.
template <typename F> __device__ __forceinline__ void walk(const TensorSet& g, int64_t x, int64_t end, F f) {
  if (x >= end) return;
  for (int i = tensor_at(g, x); i < g.n && x < end; ++i) {
    const int64_t s0 = ld_scalar(g.start + i), s1 = ld_scalar(g.start + i + 1), e = s1 < end ? s1 : end;
    if (e <= x) continue;
    if (ld_scalar(g.data + i)) f(i, x - s0, e - x);
    x = e;
  }
}

// 16 bytes aligned to an element only.
template <typename T> struct unaligned16;
template <> struct unaligned16<float> { typedef u32x4_t type __attribute__((aligned(4))); };
template <> struct unaligned16<bf16> { typedef u32x4_t type __attribute__((aligned(2))); };

// Elements before the first 16-byte boundary of p, at most n.
template <typename T> __device__ __forceinline__ int head_of(const T* p, int64_t n) {
  const int h = (int)((16 - ((uintptr_t)p & 15)) & 15) / (int)sizeof(T);
  return h < n ? h : (int)n;
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) v += __shfl_xor(v, o);
  return v;
}

// The sum over a block's threads, in thread 0.
template <int WAVES> __device__ __forceinline__ double block_sum(double v) {
  __shared__ double part[WAVES];
  v = wave_sum(v);
  if (lane_id() == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = 0;
  if (threadIdx.x == 0)
#pragma unroll
    for (int w = 0; w < WAVES; ++w) s += part[w];
  return s;
}

__device__ __forceinline__ void put_norm(double s, int accumulate, double* sumsq, float* norm) {
  if (accumulate) s += *sumsq;
  *sumsq = s;
  if (norm) *norm = (float)sqrt(s);
}

// Sums of squares of the waves' ranges of `per` elements, one per block.
template <typename T>
__global__ __launch_bounds__(256) void k_grad_sumsq(TensorSet g, int64_t per, double* __restrict__ part) {
  constexpr int V = 16 / sizeof(T);
  const int lane = lane_id();
  const int64_t w = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t x0 = w * per, x1 = x0 + per < g.total ? x0 + per : g.total;
  double acc[V];
#pragma unroll
  for (int i = 0; i < V; ++i) acc[i] = 0;
  walk(g, x0, x1, [&](int i, int64_t at, int64_t n) {
    const T* p = (const T*)ld_scalar(g.data + i) + at;
    const int head = head_of(p, n);
    if (lane < head) {
      const double v = to_float(p[lane]);
      acc[0] = fma(v, v, acc[0]);
    }
    p += head;
    n -= head;
    const int64_t nv = n / V;
    auto add = [&](const u32x4_t& raw) {
      float v[V];
      unpack16(raw, v, (T*)nullptr);
#pragma unroll
      for (int e = 0; e < V; ++e) acc[e] = fma((double)v[e], (double)v[e], acc[e]);
    };
    int64_t c = lane;
    for (; c + 64 * (GN_BATCH - 1) < nv; c += 64 * GN_BATCH) {
      u32x4_t raw[GN_BATCH];
#pragma unroll
      for (int u = 0; u < GN_BATCH; ++u) raw[u] = ld16(p + (c + 64 * u) * V);
#pragma unroll
      for (int u = 0; u < GN_BATCH; ++u) add(raw[u]);
    }
    for (; c < nv; c += 64) add(ld16(p + c * V));
    if (lane < (int)(n - nv * V)) {
      const double v = to_float(p[nv * V + lane]);
      acc[0] = fma(v, v, acc[0]);
    }
  });
  double s = 0;
#pragma unroll
  for (int i = 0; i < V; ++i) s += acc[i];
  s = block_sum<4>(s);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

__global__ __launch_bounds__(1024) void k_grad_norm(const double* __restrict__ part, int blocks, int accumulate,
                                                    double* __restrict__ sumsq, float* __restrict__ norm) {
  const double s = block_sum<16>((int)threadIdx.x < blocks ? part[threadIdx.x] : 0.0);
  if (threadIdx.x == 0) put_norm(s, accumulate, sumsq, norm);
}

// Of bf16 the rounding is to nearest even also where the product is no number (a NaN
// stays one).
__device__ __forceinline__ float scaled(float v, float c, float*) { return v * c; }
__device__ __forceinline__ bf16 scaled(bf16 v, float c, bf16*) { return bf16{(uint16_t)pk_bf16(to_float(v) * c, 0.f)}; }

template <typename T>
__global__ __launch_bounds__(256) void k_grad_clip(TensorSet g, int64_t per, const double* __restrict__ sumsq, float max_norm,
                                                   float eps, void* const* out) {
  constexpr int V = 16 / sizeof(T);
  const double den = sqrt(ld_scalar(sumsq)) + (double)eps;
  const double q = (double)max_norm / den;
  const float coef = den == 0 || q > 1 ? 1.f : (float)q;   // a NaN stays
  if (!out && coef == 1.f) return;
  const int lane = lane_id();
  const int64_t w = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t x0 = w * per, x1 = x0 + per < g.total ? x0 + per : g.total;
  walk(g, x0, x1, [&](int i, int64_t at, int64_t n) {
    const T* p = (const T*)ld_scalar(g.data + i) + at;
    T* o = out ? (T*)ld_scalar(out + i) : (T*)ld_scalar(g.data + i);
    if (!o) return;
    o += at;
    const int head = head_of(p, n);
    if (lane < head) o[lane] = scaled(p[lane], coef, (T*)nullptr);
    p += head;
    o += head;
    n -= head;
    const int64_t nv = n / V;
    auto put = [&](int64_t c, const u32x4_t& raw) {
      float v[V];
      unpack16(raw, v, (T*)nullptr);
#pragma unroll
      for (int e = 0; e < V; ++e) v[e] *= coef;
      *(FM_GLOBAL typename unaligned16<T>::type*)(o + c * V) = pack16(v, (T*)nullptr);
    };
    int64_t c = lane;
    for (; c + 64 * (GN_BATCH - 1) < nv; c += 64 * GN_BATCH) {
      u32x4_t raw[GN_BATCH];
#pragma unroll
      for (int u = 0; u < GN_BATCH; ++u) raw[u] = ld16(p + (c + 64 * u) * V);
#pragma unroll
      for (int u = 0; u < GN_BATCH; ++u) put(c + 64 * u, raw[u]);
    }
    for (; c < nv; c += 64) put(c, ld16(p + c * V));
    if (lane < (int)(n - nv * V)) o[nv * V + lane] = scaled(p[nv * V + lane], coef, (T*)nullptr);
  });
}

// Blocks for a set, and the elements of a wave's range: whole batches, at least one.
int set_blocks(const moe_tensor_set* g, int64_t* per) {
  const int64_t batch = 64 * GN_BATCH * (16 / esize(g->dtype));
  int64_t blocks = (g->total + 4 * batch - 1) / (4 * batch);
  blocks = blocks < 1 ? 1 : blocks < GN_BLOCKS ? blocks : GN_BLOCKS;
  const int64_t each = (g->total + 4 * blocks - 1) / (4 * blocks);
  *per = (each + batch - 1) / batch * batch;
  return (int)blocks;
}

int check_set(const moe_tensor_set* g, const char* name) {
  if (!g) return fail(MOE_ERR_ARG, "%s must not be NULL", name);
  if (g->n <= 0 || g->total < 0) return fail(MOE_ERR_ARG, "%s: n=%d total=%lld", name, g->n, g->total);
  if (g->n > 1 << 20 || g->total > 1LL << 48)
    return fail(MOE_ERR_UNSUPPORTED, "%s: n=%d above 2^20 or total=%lld above 2^48", name, g->n, g->total);
  FM_TRY(need_dtype_float(g->dtype, "dtype"));
  FM_TRY(need((const void*)g->data, "data")); FM_TRY(need(g->start, "start"));
  FM_TRY(need_aligned((const void*)g->data, "data")); FM_TRY(need_aligned(g->start, "start"));
  return MOE_OK;
}

TensorSet device_set(const moe_tensor_set* g) { return TensorSet{g->data, g->start, g->n, g->total}; }

}  // namespace
}  // namespace fm

using namespace fm;

extern "C" size_t moe_grad_norm_workspace_size(void) { return GN_BLOCKS * sizeof(double); }

extern "C" int moe_grad_norm(const moe_tensor_set* g, int accumulate, double* sumsq, float* norm, void* ws,
                             size_t ws_bytes, void* stream) {
  clear_error();
  FM_TRY(check_set(g, "g"));
  FM_TRY(need(sumsq, "sumsq")); FM_TRY(need(ws, "ws"));
  FM_TRY(need_aligned(sumsq, "sumsq")); FM_TRY(need_aligned(norm, "norm")); FM_TRY(need_aligned(ws, "ws"));
  const size_t bytes = moe_grad_norm_workspace_size();
  if (ws_bytes < bytes) return fail(MOE_ERR_WORKSPACE, "workspace %zu < %zu bytes", ws_bytes, bytes);
  hipStream_t st = as_stream(stream);
  int64_t per;
  const int blocks = set_blocks(g, &per);
  double* const part = (double*)ws;
  if (g->dtype == MOE_BF16)
    hipLaunchKernelGGL(k_grad_sumsq<bf16>, dim3(blocks), dim3(256), 0, st, device_set(g), per, part);
  else
    hipLaunchKernelGGL(k_grad_sumsq<float>, dim3(blocks), dim3(256), 0, st, device_set(g), per, part);
  hipLaunchKernelGGL(k_grad_norm, dim3(1), dim3(1024), 0, st, part, blocks, accumulate != 0, sumsq, norm);
  return check_launch("moe_grad_norm");
}

extern "C" int moe_grad_clip(const moe_tensor_set* g, const double* sumsq, float max_norm, float eps,
                             const moe_tensor_set* out, void* stream) {
  clear_error();
  FM_TRY(check_set(g, "g"));
  FM_TRY(need(sumsq, "sumsq")); FM_TRY(need_aligned(sumsq, "sumsq"));
  if (!(max_norm >= 0.f) || __builtin_isinf(max_norm)) return fail(MOE_ERR_ARG, "max_norm=%g", max_norm);
  if (!(eps >= 0.f) || __builtin_isinf(eps)) return fail(MOE_ERR_ARG, "eps=%g", eps);
  if (out) {
    FM_TRY(check_set(out, "out"));
    if (out->n != g->n || out->dtype != g->dtype || out->total != g->total)
      return fail(MOE_ERR_ARG, "out: n=%d dtype=%d total=%lld, g has %d, %d, %lld", out->n, out->dtype, out->total, g->n,
                  g->dtype, g->total);
  }
  hipStream_t st = as_stream(stream);
  int64_t per;
  const int blocks = set_blocks(g, &per);
  void* const* o = out ? out->data : nullptr;
  if (g->dtype == MOE_BF16)
    hipLaunchKernelGGL(k_grad_clip<bf16>, dim3(blocks), dim3(256), 0, st, device_set(g), per, sumsq, max_norm, eps, o);
  else
    hipLaunchKernelGGL(k_grad_clip<float>, dim3(blocks), dim3(256), 0, st, device_set(g), per, sumsq, max_norm, eps, o);
  return check_launch("moe_grad_clip");
}
