// Microscaled 4-bit rows (MXFP4) and the grouped SwiGLU forward on them (the
// formulas stand in the header at moe_quantize_mxfp4 and
// moe_grouped_swiglu_fwd_mx4).
//
// The products run on v_mfma_scale_f32_32x32x64_f8f6f4 with both operands e2m1:
// a lane holds 32 consecutive k of one row (16 bytes) and the scale byte of
// exactly that block, lane l row l % 32 and k block l / 32, so packed rows are
// MFMA fragments as they lie in memory.
//
// * Slabs of 256 k go global -> LDS with global_load_lds_dwordx4, whole 128-byte lines
//   of 8 rows per instruction, into two buffers; the scales of 512 k of a row (16
//   bytes) follow through registers.  The number of requests to L2 counts, not their
//   bytes alone: with half lines and a scale dword per row and 128 k (128 x 256 tiles, a
//   ring of three, two blocks per compute unit) the same products took 2.03 and 1.15 ms
//   at 262144 rows, d = 4096, I = 1024.  Now 1.44 and 0.96 (3.1 and 2.3 PFLOP/s; the
//   instruction alone, on registers, reaches 7.2): the matrix cores are busy for 37 and
//   29 % of the cycles, L2's channels take a read in 28 and 16 % of them, HBM moves 2.6
//   and 3.2 TB/s.  None of them is full: what is left is latency, one slab in flight per
//   block and the ends of the tiles (44 us each in gate-up).  With the next tile's setup
//   and first slab before the epilogue it ran 3-8 % slower.
// * Weights are the first operand, so a lane's 16 sums of a 32 x 32 tile belong to
//   one activation row; weight rows are dealt to the operand's rows so that they
//   are 16 consecutive columns (tile_column).  Two lanes then hold a whole
//   32-block of H: its maximum is 15 comparisons and one exchange, and H is
//   quantised in registers.
// * X and H in the workspace have rows of whole 256-blocks, zero behind the row's
//   end, so weight chunks past K (clamped reads) meet zero codes.
#include <type_traits>

#include "debug.hpp"
#include "ffn_common.hpp"
#include "ffn_tile.hpp"
#include "gemm_bf16.hpp"
#include "grouped_tiles.hpp"

namespace fm {
namespace {

typedef int i32x8_t __attribute__((ext_vector_type(8)));

__host__ __device__ constexpr int up32(int n) { return (n + 31) / 32 * 32; }
__host__ __device__ constexpr int up128(int n) { return (n + 127) / 128 * 128; }
// 128-blocks of an activation row in the workspace: an even number.
__host__ __device__ constexpr int act_blocks(int n) { return (n + 255) / 256 * 2; }

// Block scale of a largest magnitude, given as the bits of its absolute value:
// floor(log2) - 2, biased by 127; 255 for infinities and NaN.
__device__ __forceinline__ uint32_t mx_byte(uint32_t top) {
  const uint32_t e = top >> 23;
  return e == 255 ? 255u : e < 2 ? 0u : e - 2;
}
// 2^(127 - byte), by which an element is multiplied (exactly, but for results far
// below the smallest code).
__device__ __forceinline__ float mx_inv(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

// Eight values times s as codes, the first in the lowest bits.
__device__ __forceinline__ uint32_t mx_codes8(const float* v, float s) {
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0] * s, v[1] * s, 1.0f, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2] * s, v[3] * s, 1.0f, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4] * s, v[5] * s, 1.0f, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6] * s, v[7] * s, 1.0f, 3);
  return c;
}

__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// 8 columns from c of a row (0 past cols).
template <typename T> __device__ __forceinline__ void load8(const T* row, int c, int cols, float (&v)[8]) {
  if (c < cols) {
    unpack16(ld16(row + c), v, (T*)nullptr);
    if constexpr (sizeof(T) == 4) unpack16(ld16(row + c + 4), v + 4, (T*)nullptr);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.f;
  }
}

// 128 columns of a row in 16 lanes, 8 each (q: lane within them): this lane's codes, and
// the four blocks' scale bytes in every lane.
__device__ __forceinline__ uint32_t quantize128(const float (&v)[8], int q, uint32_t& scales) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, abs_bits(v[i]));
  top = max(top, (uint32_t)__shfl_xor((int)top, 1));
  top = max(top, (uint32_t)__shfl_xor((int)top, 2));
  const uint32_t byte = mx_byte(top);
  uint32_t s = byte << (8 * (q >> 2));
  s |= (uint32_t)__shfl_xor((int)s, 4);
  s |= (uint32_t)__shfl_xor((int)s, 8);
  scales = s;
  return byte == 255 ? 0u : mx_codes8(v, mx_inv(byte));
}

// x of another lane of the quad.
template <int CTRL> __device__ __forceinline__ uint32_t quad_u(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, false);
}

// quantize128 of bf16 as they lie in memory: magnitudes compare as 16-bit integers, and
// the conversion takes pairs and the scale itself (a power of two that is no subnormal).
__device__ __forceinline__ uint32_t quantize128(const u32x4_t& x, int q, uint32_t& scales) {
  typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));
  auto mag = [&](int i) { return __builtin_bit_cast(u16x2_t, x[i] & 0x7FFF7FFFu); };
  const u16x2_t m = __builtin_elementwise_max(__builtin_elementwise_max(mag(0), mag(1)), __builtin_elementwise_max(mag(2), mag(3)));
  uint32_t top = max((uint32_t)m[0], (uint32_t)m[1]) << 16;
  top = max(top, quad_u<0xB1>(top));   // quad_perm [1, 0, 3, 2]
  top = max(top, quad_u<0x4E>(top));   // quad_perm [2, 3, 0, 1]
  const uint32_t byte = mx_byte(top);
  uint32_t s = byte << (8 * (q >> 2));
  s |= (uint32_t)__shfl_xor((int)s, 4);
  s |= (uint32_t)__shfl_xor((int)s, 8);
  scales = s;
  if (byte == 255) return 0u;
  if (byte == 0) {
    float v[8];
    unpack16(x, v, (bf16*)nullptr);
    return mx_codes8(v, mx_inv(0));
  }
  const float f = __uint_as_float(byte << 23);
  auto pair = [&](int i) {
    const uint32_t w = x[i];   // (a bit cast of the vector's element itself takes element 0)
    return __builtin_bit_cast(bf16x2_t, w);
  };
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, pair(0), f, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, pair(1), f, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, pair(2), f, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, pair(3), f, 3);
}

// Columns [128 blk, 128 blk + 128) of a row to memory; codes up to column code_cols.
template <typename T>
__device__ __forceinline__ void quantize_row(const T* row, int cols, int blk, int q, int code_cols, uint8_t* codes,
                                             uint8_t* scale) {
  const int c = blk * 128 + q * 8;
  uint32_t s, code;
  if constexpr (sizeof(T) == 2) {
    u32x4_t x = {0, 0, 0, 0};
    if (c < cols) x = ld16(row + c);
    code = quantize128(x, q, s);
  } else {
    float v[8];
    load8(row, c, cols, v);
    code = quantize128(v, q, s);
  }
  if (c < code_cols) *(FM_GLOBAL uint32_t*)(codes + c / 2) = code;
  if (q == 0) *(FM_GLOBAL uint32_t*)(scale + blk * 4) = s;
}

// 90112 rows of 2048 bf16: 100 us, 4.7 TB/s of the 467 MB read and written.
template <typename T>
__global__ __launch_bounds__(256) void k_quantize_mx(const T* __restrict__ W, uint32_t items, int cols, int nb,
                                                     uint8_t* __restrict__ codes, uint8_t* __restrict__ scale) {
  const uint32_t item = blockIdx.x * 16 + threadIdx.x / 16;
  if (item >= items) return;
  const uint32_t r = item / nb;
  quantize_row(W + (size_t)r * cols, cols, (int)(item - r * nb), threadIdx.x % 16, up32(cols),
              codes + (size_t)r * (up32(cols) / 2), scale + (size_t)r * nb * 4);
}

// The value of the low 4 bits, an e2m1 code: 0, 0.5 and then exponent and mantissa
// shifted into an fp32.
__device__ __forceinline__ float mx_value(uint32_t c) {
  const uint32_t m = c & 7u;
  const uint32_t bits = m < 2 ? m * 0x3F000000u : ((m >> 1) + 126u) << 23 | (m & 1u) << 22;
  return __uint_as_float(bits | (c & 8u) << 28);
}

// 90112 rows of 2048 bf16: 83 us, 5.6 TB/s.  (Code by code through mx_value 117 us.)
template <typename T>
__global__ __launch_bounds__(256) void k_dequant_mx(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scale,
                                                    uint32_t items, int cols, int n8, T* __restrict__ out) {
  const uint32_t item = blockIdx.x * 256 + threadIdx.x;
  if (item >= items) return;
  const uint32_t r = item / n8, c = (item - r * n8) * 8;
  const uint32_t code = *(const FM_GLOBAL uint32_t*)(codes + (size_t)r * (up32(cols) / 2) + c / 2);
  const uint32_t byte = scale[(size_t)r * (up128(cols) / 32) + c / 32];
  T* o = out + (size_t)r * cols + c;
  if (byte == 255 || byte == 0) {   // NaN, or a scale that is a subnormal
    const float s = __uint_as_float(byte ? 0x7FC00000u : 0x00400000u);
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = mx_value(code >> (4 * i)) * s;
    st16(o, pack16(v, (T*)nullptr));
    if constexpr (sizeof(T) == 4) st16(o + 4, pack16(v + 4, (T*)nullptr));
    return;
  }
  const float s = __uint_as_float(byte << 23);
  if constexpr (sizeof(T) == 2) {
    auto pair = [](bf16x2_t v) { return __builtin_bit_cast(uint32_t, v); };
    st16(o, u32x4_t{pair(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, s, 0)), pair(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, s, 1)),
                    pair(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, s, 2)), pair(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, s, 3))});
  } else {
    auto put = [&](int i, f32x2_t a, f32x2_t b) {
      st16(o + i, u32x4_t{__float_as_uint(a[0]), __float_as_uint(a[1]), __float_as_uint(b[0]), __float_as_uint(b[1])});
    };
    put(0, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, s, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, s, 1));
    put(4, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, s, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, s, 3));
  }
}

// ------------------------------------------------------- grouped products ----

struct MxPtrs {
  const uint8_t* const* qg;
  const uint8_t* const* qu;
  const uint8_t* const* qd;
  const uint8_t* const* sg;
  const uint8_t* const* su;
  const uint8_t* const* sd;
};

constexpr int MX_FEW = 8;   // most tokens of a call that takes the kernels for few

// Workspace: row-tile prefix, X and H as packed rows of whole 256-blocks.
struct MxWs {
  int32_t* mbase;
  uint8_t *xq, *xs, *hq, *hs;
  float* hf;   // H of a call of few tokens, [rows][I]
};
inline size_t round256(size_t b) { return (b + 255) / 256 * 256; }
inline MxWs mx_ws_at(void* ws, const moe_layer_mx4* L, int T, int k, size_t* bytes) {
  const size_t S = L->S_routed + L->S_shared, R = (size_t)T * (k + L->S_shared);
  const size_t nd = act_blocks(L->d), nI = act_blocks(L->I);
  MxWs w;
  char* p = (char*)ws;
  auto take = [&](size_t b) {
    char* at = p;
    p += round256(b);
    return at;
  };
  w.mbase = (int32_t*)take((S + 1) * 4);
  w.xq = (uint8_t*)take((size_t)T * nd * 64);
  w.xs = (uint8_t*)take((size_t)T * nd * 4);
  w.hq = (uint8_t*)take(R * nI * 64);
  w.hs = (uint8_t*)take(R * nI * 4);
  w.hf = (float*)take((size_t)(T < MX_FEW ? T : MX_FEW) * (k + L->S_shared) * L->I * 4);
  *bytes = (size_t)(p - (char*)ws);
  return w;
}

// X's tokens as packed rows; the last block builds the row-tile prefix instead.
__global__ __launch_bounds__(256) void k_mx_prep(const bf16* __restrict__ X, RowArgs ra, int tile_rows, int nb,
                                                 uint8_t* __restrict__ xq, uint8_t* __restrict__ xs,
                                                 int32_t* __restrict__ mbase) {
  if (blockIdx.x == gridDim.x - 1) {
    count_tiles(ra, tile_rows, mbase);
    return;
  }
  const uint32_t item = blockIdx.x * 16 + threadIdx.x / 16;   // below 2^26: T up128(d) <= 2^32
  if (item >= (uint32_t)ra.Tn * nb) return;
  const uint32_t r = item / nb;
  quantize_row(X + (size_t)r * ra.d, ra.d, (int)(item - r * nb), threadIdx.x % 16, nb * 128, xq + (size_t)r * nb * 64,
              xs + (size_t)r * nb * 4);
}

// RA activation rows x RB weight rows by 2 x WN waves; BPC blocks per compute unit.
template <int RA_, int RB_, int WN_, int BPC_> struct MxCfg {
  static constexpr int RA = RA_, RB = RB_, WN = WN_, NW = 2 * WN, BPC = BPC_;
  static constexpr int TM = RA / 2, TN = RB / WN, MI = TM / 32, NJ = TN / 32;
  static constexpr int A_BYTES = RA * 128, SLAB = A_BYTES + RB * 128;   // 256 k
  static constexpr int A_INS = RA / 8 / NW, B_INS = RB / 8 / NW;        // 8 rows each, per wave
  static constexpr int SCALES = (RA + RB) * 16;                         // 512 k
  static constexpr int LDS = 2 * (SLAB + SCALES);
  static_assert(RA % (8 * NW) == 0 && RA % 64 == 0 && RB % (8 * NW) == 0 && NJ == 2 && RA + RB <= 64 * NW, "tile");
  static_assert(BPC * LDS <= 160 * 1024, "LDS");
};

// Chunk swizzles of a 128-byte slab row: 16 consecutive lanes' rows at one logical
// chunk on 16 distinct 4-bank groups; lanes read activation rows in order, weight
// rows in the order of tile_column.
__device__ __forceinline__ int mx_swz_a(int r) { return (r >> 1) & 7; }
__device__ __forceinline__ int mx_swz_b(int r) { return ((r >> 1) & 3) | ((r >> 2) & 4); }

// One operand pair of a tile, rows relative to it.  w2: the second of two matrices
// whose 32-row blocks alternate (gate, up).
struct MxTile {
  const uint8_t *x, *xs;        // activations' codes and scales
  const int32_t* tok;           // row -> activation row (gathered), or NULL
  int rows, Tn;                 // activation rows of the tile's slot from the tile on
  const uint8_t *w, *w2, *s, *s2;
  int wrows;                    // weight rows (per matrix) from the tile on
  int kx, kw;                   // 128-blocks of an activation row (even); 32-blocks of a weight row
};

// acc += X W^T.  LDS: two slabs, then two groups of scales [RA + RB rows][16 bytes].
// The barrier at the top of slab kt says that it has landed and that every wave has
// read slab kt - 1, whose buffer then takes slab kt + 1.  Scales of group g (slabs 2 g
// and 2 g + 1) are requested at slab 2 g - 2 and put into LDS at slab 2 g - 1.
template <class C, bool PAIR>
__device__ __forceinline__ void mx_gemm(const MxTile& t, FM_LDS char* lds, f32x16_t (&acc)[C::MI][C::NJ]) {
  const int lane = lane_id(), wave = wave_id();
  const int nk = t.kx / 2;   // slabs
  const uint32_t ldx = t.kx * 64, ldw = t.kw * 16;
  const int sx = t.kx, sw = (t.kw + 3) / 4;   // dwords of scale rows
  FM_LDS char* const sc = lds + 2 * C::SLAB;
  uint32_t oa[C::A_INS], ob[C::B_INS];
  auto xrow = [&](int r) {
    r = min(r, t.rows - 1);
    return (uint32_t)(t.tok ? min(max(gptr(t.tok)[r], 0), t.Tn - 1) : r);
  };
  auto wrow = [&](int r) { return (uint32_t)min(PAIR ? 32 * (r >> 6) + (r & 31) : r, t.wrows - 1); };
#pragma unroll
  for (int u = 0; u < C::A_INS; ++u) {
    const int r = 8 * (wave * C::A_INS + u) + (lane >> 3);
    oa[u] = xrow(r) * ldx + 16 * ((lane & 7) ^ mx_swz_a(r));
  }
#pragma unroll
  for (int u = 0; u < C::B_INS; ++u) {
    const int r = 8 * (wave * C::B_INS + u) + (lane >> 3);
    ob[u] = wrow(r) * ldw + 16 * ((lane & 7) ^ mx_swz_b(r));
  }
  // behind a row's end, weights repeat their row's last chunk (it meets zeros)
  auto issue = [&](int slab) {
    FM_LDS char* const l = lds + (slab & 1) * C::SLAB;
#pragma unroll
    for (int u = 0; u < C::A_INS; ++u)
      dma16s(t.x + (size_t)slab * 128, oa[u], l + (wave * C::A_INS + u) * 1024);
#pragma unroll
    for (int u = 0; u < C::B_INS; ++u) {
      const int ins = wave * C::B_INS + u;
      const uint8_t* const w = (PAIR && ((ins >> 2) & 1) ? t.w2 : t.w) + (size_t)slab * 128;
      uint32_t o = ob[u];
      if (8 * slab + 8 > t.kw) {
        const int k = (lane & 7) ^ mx_swz_b(8 * ins + (lane >> 3));
        o += 16 * (min(k, t.kw - 1 - 8 * slab) - k);
      }
      dma16s(w, o, l + C::A_BYTES + ins * 1024);
    }
  };
  // this lane's scale row (waves past the rows repeat the last)
  const int sr = min(64 * wave + lane, C::RA + C::RB - 1), br = sr - C::RA;
  const bool wside = 64 * wave >= C::RA;
  const uint8_t* const sp = wside ? (PAIR && ((br >> 5) & 1) ? t.s2 : t.s) + (size_t)wrow(br) * sw * 4
                                  : t.xs + (size_t)xrow(sr) * sx * 4;
  const int slen = wside ? sw : sx;
  typedef u32x4_t u32x4_a4 __attribute__((aligned(4)));
  // dwords [4 g, 4 g + 4) of a row of n, the last group moved back to end with the row
  auto group_at = [](int g, int n) { return max(min(4 * g, n - 4), 0); };
  auto load_scales = [&](int g) {
    u32x4_t v;
    if (slen >= 4) return (u32x4_t)*(const FM_GLOBAL u32x4_a4*)(sp + 4 * group_at(g, slen));
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = *(const FM_GLOBAL uint32_t*)(sp + 4 * min(i, slen - 1));
    return v;
  };
  auto put_scales = [&](int g, const u32x4_t& v) {
    if (64 * wave < C::RA + C::RB) *(FM_LDS u32x4_t*)(sc + (g & 1) * C::SCALES + sr * 16) = v;
  };
  const int row0 = (wave & 1) * C::TM, col0 = (wave >> 1) * C::TN;
  const int m = lane & 31, h = lane >> 5;
  uint32_t fa[C::MI], fb[C::NJ];
#pragma unroll
  for (int i = 0; i < C::MI; ++i) {
    const int r = row0 + 32 * i + m;
    fa[i] = r * 128 + ((h ^ mx_swz_a(r)) << 4);
  }
#pragma unroll
  for (int j = 0; j < C::NJ; ++j) {
    const int r = col0 + 32 * j + tile_column(m);
    fb[j] = C::A_BYTES + r * 128 + ((h ^ mx_swz_b(r)) << 4);
  }
  const uint32_t ga = (row0 + m) * 16, gb = (C::RA + col0 + tile_column(m)) * 16;
#pragma unroll
  for (int i = 0; i < C::MI; ++i)
#pragma unroll
    for (int j = 0; j < C::NJ; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

  issue(0);
  put_scales(0, load_scales(0));
  u32x4_t next;
#pragma nounroll
  for (int kt = 0; kt < nk; ++kt) {
    wait_vmcnt<0>();
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (kt + 1 < nk) issue(kt + 1);
    if (!(kt & 1)) {
      if (kt + 2 < nk) next = load_scales(kt / 2 + 1);
    } else if (kt + 1 < nk) {
      put_scales(kt / 2 + 1, next);
    }
    const FM_LDS char* const l = lds + (kt & 1) * C::SLAB;
    const FM_LDS char* const s = sc + ((kt >> 1) & 1) * C::SCALES;
    const FM_LDS char* const s_x = s + 4 * (2 * kt - group_at(kt >> 1, sx));
    const FM_LDS char* const s_w = s + 4 * (2 * kt - group_at(kt >> 1, sw));
    const bool half = 2 * kt + 1 == sw;   // the slab's second 128 k lie past the weights: scale 0 there
    u32x4_t xa[2][C::MI], xb[2][C::NJ];
    int sa[2][C::MI], sb[2][C::NJ];
    auto read = [&](int st) {
      int flip = st << 5;
      asm volatile("" : "+s"(flip));   // not hoisted: the 24 addresses would take the registers of the sums
#pragma unroll
      for (int i = 0; i < C::MI; ++i) xa[st & 1][i] = *(const FM_LDS u32x4_t*)(l + (fa[i] ^ flip));
#pragma unroll
      for (int j = 0; j < C::NJ; ++j) xb[st & 1][j] = *(const FM_LDS u32x4_t*)(l + (fb[j] ^ flip));
    };
    auto scales = [&](int q) {   // of 128 k: blocks h and h + 2 in bytes 0 and 2
#pragma unroll
      for (int i = 0; i < C::MI; ++i) sa[q][i] = *(const FM_LDS int*)(s_x + ga + 512 * i + 4 * q) >> (8 * h);
#pragma unroll
      for (int j = 0; j < C::NJ; ++j) {
        sb[q][j] = *(const FM_LDS int*)(s_w + gb + 512 * j + (half ? 0 : 4 * q)) >> (8 * h);
        if (q == 1 && half) sb[q][j] = 0;
      }
    };
    auto wide = [](const u32x4_t& v) { return i32x8_t{(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0}; };
    auto multiply = [&](auto st_) {
      constexpr int st = decltype(st_)::value, by = 2 * (st & 1);
#pragma unroll
      for (int j = 0; j < C::NJ; ++j)
#pragma unroll
        for (int i = 0; i < C::MI; ++i)
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide(xb[st & 1][j]), wide(xa[st & 1][i]), acc[i][j], 4,
                                                                      4, by, sb[st >> 1][j], by, sa[st >> 1][i]);
    };
    // a step's fragments are read while the one before it multiplies, and not earlier
    // (two sets of registers)
    scales(0);
    read(0);
    sched_fence();
    read(1);
    multiply(std::integral_constant<int, 0>{});
    sched_fence();
    scales(1);
    read(2);
    multiply(std::integral_constant<int, 1>{});
    sched_fence();
    read(3);
    multiply(std::integral_constant<int, 2>{});
    sched_fence();
    multiply(std::integral_constant<int, 3>{});
  }
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

struct MxArgs {
  MxPtrs W;
  MxWs w;
  const int32_t* perm_token;
  RowArgs ra;
  bf16* O;
};

// H = MX(silu(MX(X) Qg^T) (MX(X) Qu^T)) of one tile, RB / 2 columns.
template <class C> __device__ __forceinline__ void mx_gate_up_tile(const MxArgs& a, FM_LDS char* lds, const TileRows& r) {
  const RowArgs& ra = a.ra;
  const int I = ra.I, nI = act_blocks(I), kd = act_blocks(ra.d), n0 = r.n * (C::RB / 2);
  const size_t lw = up32(ra.d) / 2, ls = up128(ra.d) / 32;
  MxTile t;
  t.x = a.w.xq + (r.sr.shared ? (size_t)r.m0 * kd * 64 : 0);
  t.xs = a.w.xs + (r.sr.shared ? (size_t)r.m0 * kd * 4 : 0);
  t.tok = r.sr.shared ? nullptr : a.perm_token + r.sr.xrow0 + r.m0;
  t.rows = r.rows;
  t.Tn = ra.Tn;
  t.w = ld_scalar(a.W.qg + r.s) + n0 * lw;
  t.w2 = ld_scalar(a.W.qu + r.s) + n0 * lw;
  t.s = ld_scalar(a.W.sg + r.s) + n0 * ls;
  t.s2 = ld_scalar(a.W.su + r.s) + n0 * ls;
  t.wrows = I - n0;
  t.kx = kd;
  t.kw = up32(ra.d) / 32;
  f32x16_t acc[C::MI][C::NJ];
  mx_gemm<C, true>(t, lds, acc);
  const int lane = lane_id_here(), wave = wave_id(), h = lane >> 5;
  const int col = n0 + (wave >> 1) * 32;   // of this wave's 32-block
#pragma unroll
  for (int i = 0; i < C::MI; ++i) {
    const int row = (wave & 1) * C::TM + 32 * i + (lane & 31);
    float v[16];
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float g = acc[i][0][e];
      v[e] = col + 16 * h + e < I ? g * sigm_fast(g) * acc[i][1][e] : 0.f;
      top = max(top, abs_bits(v[e]));
    }
    top = max(top, (uint32_t)__shfl_xor((int)top, 32));
    const uint32_t byte = mx_byte(top);
    const float inv = mx_inv(byte);
    u32x2_t code = {mx_codes8(v, inv), mx_codes8(v + 8, inv)};
    if (byte == 255) code = u32x2_t{0u, 0u};
    if (row < r.rows) {
      *(FM_GLOBAL u32x2_t*)(a.w.hq + (r.ob + row) * nI * 64 + col / 2 + 8 * h) = code;
      if (h == 0) *(FM_GLOBAL uint8_t*)(a.w.hs + (r.ob + row) * nI * 4 + col / 32) = (uint8_t)byte;
      // the row's padding, behind the last tile
      if (n0 + C::RB / 2 >= I)
        for (int c = col + C::RB / 2; c < nI * 128; c += C::RB / 2) {
          *(FM_GLOBAL u32x2_t*)(a.w.hq + (r.ob + row) * nI * 64 + c / 2 + 8 * h) = u32x2_t{0u, 0u};
          if (h == 0) *(FM_GLOBAL uint8_t*)(a.w.hs + (r.ob + row) * nI * 4 + c / 32) = 0;
        }
    }
  }
}

// O = MX(H) Qd^T of one tile, RB columns.  A wave's 32 rows x 64 columns go out through
// LDS, so that a store covers whole lines of 8 rows (from the registers it touched 32
// rows, 16 bytes of each).  stage: 4 KB per wave that the next tile's first slab and
// scales leave alone, whichever its height.
template <class C>
__device__ __forceinline__ void mx_down_tile(const MxArgs& a, FM_LDS char* lds, FM_LDS char* stage, const TileRows& r) {
  const RowArgs& ra = a.ra;
  const int d = ra.d, nI = act_blocks(ra.I), n0 = r.n * C::RB;
  MxTile t;
  t.x = a.w.hq + r.ob * nI * 64;
  t.xs = a.w.hs + r.ob * nI * 4;
  t.tok = nullptr;
  t.rows = r.rows;
  t.Tn = ra.Tn;
  t.w = ld_scalar(a.W.qd + r.s) + (size_t)n0 * (up32(ra.I) / 2);
  t.s = ld_scalar(a.W.sd + r.s) + (size_t)n0 * (up128(ra.I) / 32);
  t.w2 = t.s2 = nullptr;
  t.wrows = d - n0;
  t.kx = nI;
  t.kw = up32(ra.I) / 32;
  f32x16_t acc[C::MI][C::NJ];
  mx_gemm<C, false>(t, lds, acc);
  const int lane = lane_id_here(), wave = wave_id(), h = lane >> 5;
  FM_LDS char* const mine = stage + wave * 4096;   // [32 rows][8 chunks of 16 bytes], chunks swizzled by the row
  const int m = lane & 31, col = n0 + (wave >> 1) * C::TN + 8 * (lane & 7);
#pragma unroll
  for (int i = 0; i < C::MI; ++i) {
#pragma unroll
    for (int j = 0; j < C::NJ; ++j)
#pragma unroll
      for (int e = 0; e < 16; e += 8) {
        float v[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) v[x] = acc[i][j][e + x];
        *(FM_LDS u32x4_t*)(mine + m * 128 + (((4 * j + 2 * h + e / 8) ^ (m & 7)) << 4)) = pack16(v, (bf16*)nullptr);
      }
    wave_lds_fence();
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int q = 8 * u + (lane >> 3), row = (wave & 1) * C::TM + 32 * i + q;
      const u32x4_t v = *(const FM_LDS u32x4_t*)(mine + q * 128 + (((lane & 7) ^ (q & 7)) << 4));
      if (row < r.rows && col < d) st16(a.O + (r.ob + row) * d + col, v);
    }
    wave_lds_fence();
  }
}

template <class C, class BIG, bool DOWN>
__device__ __forceinline__ void mx_tile(const MxArgs& a, FM_LDS char* lds, const TileRows& r) {
  // the first 4 KB per wave behind the larger tile's first slab: inside the second slab
  // of either height, which the next tile requests only behind its first barrier
  static_assert(BIG::SLAB + BIG::NW * 4096 <= 2 * C::SLAB, "stage");
  if constexpr (DOWN) mx_down_tile<C>(a, lds, lds + BIG::SLAB, r);
  else mx_gate_up_tile<C>(a, lds, r);
}

// C: the tile; HALF: its half-height form for tiles with at most half the rows left.
template <class C, class HALF, bool DOWN> __global__ __launch_bounds__(64 * C::NW, C::BPC * C::NW / 4) void k_mx_tiles(MxArgs a) {
  __shared__ __align__(16) char lds_[C::LDS];
  FM_LDS char* const lds = (FM_LDS char*)lds_;
  constexpr int COLS = DOWN ? C::RB : C::RB / 2;
  const int NT = ((DOWN ? a.ra.d : a.ra.I) + COLS - 1) / COLS;
  const TileWalk walk = tile_walk(a.ra, NT);
  for (int tt = walk.at; tt < walk.end; tt += walk.step) {
    const TileRows r = tile_rows_at(a.ra, tt, NT, C::RA);
    if (r.rows <= HALF::RA) mx_tile<HALF, C, DOWN>(a, lds, r);
    else mx_tile<C, C, DOWN>(a, lds, r);
  }
}

typedef MxCfg<256, 256, 4, 1> M256;
typedef MxCfg<128, 256, 4, 1> M128;
typedef MxCfg<128, 128, 2, 2> Q128;
typedef MxCfg<64, 128, 2, 2> Q64;

// --------------------------------------------------------- a few tokens ----
// Calls of a few tokens are bound by latency and by the weights' bytes, which have to be
// spread over all compute units: a block takes 8 columns of H (8 gate and 8 up rows, one
// fragment of v_mfma_scale_f32_16x16x128_f8f6f4: lane l row l % 16, k block l / 16), or
// 32 of O, of one slot, and its NW waves split k into consecutive parts whose sums meet
// in LDS.  No ring: a wave requests BS steps of weights straight into registers, and the
// block quantises its activation rows into LDS while they are on their way (a launch
// before, for the activations alone, costs some 3 us; a lane that quantised the 32
// activations of its own row and k block repeated it for 16 rows, mostly empty ones, and
// was bound by vector instructions).  H goes through the workspace in fp32 and is
// quantised the same way.  Rows come 16 at a time.  Blocks exist for the slots that may
// hold rows only: the i-th of them is found by a ballot over the offsets.

// Rows of nb 128-blocks in LDS: codes, then scales; padded so that 16 rows' chunks at
// one place lie on different banks.
struct MxFewRows {
  FM_LDS char* codes;
  FM_LDS char* scale;
  int ld, lds;
};
__host__ __device__ constexpr int mx_few_row_bytes(int nb) { return nb * 64 + 16 + nb * 4 + 4; }
__device__ __forceinline__ MxFewRows mx_few_rows(FM_LDS char* at, int nb, int rows) {
  return MxFewRows{at, at + rows * (nb * 64 + 16), nb * 64 + 16, nb * 4 + 4};
}

// The block's n rows (row(r): pointer) of cols columns, quantised into LDS.
template <int THREADS, typename Row>
__device__ __forceinline__ void mx_few_stage(const MxFewRows& l, int n, int nb, int cols, Row row) {
  for (int item = threadIdx.x / 16; item < n * nb; item += THREADS / 16) {
    const int r = item / nb, blk = item - r * nb, q = threadIdx.x % 16;
    float v[8];
    load8(row(r), blk * 128 + q * 8, cols, v);
    uint32_t s;
    const uint32_t code = quantize128(v, q, s);
    *(FM_LDS uint32_t*)(l.codes + r * l.ld + blk * 64 + q * 4) = code;
    if (q == 0) *(FM_LDS uint32_t*)(l.scale + r * l.lds + blk * 4) = s;
  }
}

// Sums over this wave's steps [k0, k1) of 128 k: NF fragments of 16 weight rows (codes
// at w[f], scales at s[f], both of this lane's row) by the 16 activation rows that
// stage() puts into LDS (n of them are there).
template <int NF, int BS, typename Stage>
__device__ __forceinline__ void mx_few_sums(const uint8_t* const (&w)[NF], const uint8_t* const (&s)[NF], int kw,
                                            const MxFewRows& l, int n, int k0, int k1, Stage stage,
                                            f32x4_t (&acc)[NF]) {
  const int kb = lane_id() >> 4, r = min(lane_id() & 15, n - 1);
  u32x4_t wc[BS][NF];
  uint32_t ws[BS][NF];
  auto load = [&](int k) {
#pragma unroll
    for (int u = 0; u < BS; ++u) {
      if (k + u >= k1) break;
#pragma unroll
      for (int f = 0; f < NF; ++f) {
        wc[u][f] = ld16(w[f] + 16 * min(4 * (k + u) + kb, kw - 1));   // a chunk behind the row meets zero activations
        ws[u][f] = *(const FM_GLOBAL uint32_t*)(s[f] + 4 * (k + u));
      }
    }
  };
  auto wide = [](const u32x4_t& v) { return i32x8_t{(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0}; };
  load(k0);
  stage();
  __syncthreads();
  for (int k = k0; k < k1; k += BS) {
    if (k > k0) load(k);
#pragma unroll
    for (int u = 0; u < BS; ++u) {
      if (k + u >= k1) break;
      const u32x4_t xc = *(const FM_LDS u32x4_t*)(l.codes + r * l.ld + (4 * (k + u) + kb) * 16);
      const int xb = *(const FM_LDS uint8_t*)(l.scale + r * l.lds + 4 * (k + u) + kb);
#pragma unroll
      for (int f = 0; f < NF; ++f)
        acc[f] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wide(wc[u][f]), wide(xc), acc[f], 4, 4, 0,
                                                                  (int)(ws[u][f] >> (8 * kb)), 0, xb);
    }
  }
}

// The waves' sums through LDS: [wave][f][lane] quads; element (row, weight row n) of
// fragment f is in quad lane 16 (n / 4) + row, component n % 4.
template <int NF, int NW>
__device__ __forceinline__ float mx_few_sum(const FM_LDS f32x4_t* red, int f, int row, int n) {
  const FM_LDS float* const p = (const FM_LDS float*)(red + f * 64 + 16 * (n >> 2) + row) + (n & 3);
  float v = 0.f;
#pragma unroll
  for (int w = 0; w < NW; ++w) v += p[w * NF * 256];
  return v;
}

// This wave's part of n steps.
template <int NW> __device__ __forceinline__ void mx_few_part(int n, int& k0, int& k1) {
  const int per = (n + NW - 1) / NW, w = wave_id();
  k0 = min(w * per, n);
  k1 = min(k0 + per, n);
}

extern __shared__ __align__(16) char mx_few_lds[];

// One token of the first layer below (4 of 16 slots): 8.7 us, and k_mx_few_down 4.0; the
// weights' 18 MB are 3.5 us.  A copy of this kernel without the weights' loads took 5.2
// us, without the quantisation 7.2, with neither 3.5: latency of a launch and of the
// chain offsets - row - codes - weights.  With 32 columns of H per block 13.9.
template <int NW, int BS>
__global__ __launch_bounds__(64 * NW) void k_mx_few_gate_up(MxArgs a, const bf16* __restrict__ X, int NT, int max_rows) {
  FM_LDS f32x4_t* const red = (FM_LDS f32x4_t*)mx_few_lds;
  const RowArgs& ra = a.ra;
  SlotRows sr;
  const int sl = active_slot(ra, blockIdx.x / NT, sr);
  if (sl < 0) return;
  const int n0 = (blockIdx.x % NT) * 8, I = ra.I, kd = up128(ra.d) / 128;
  const int lane = lane_id(), r16 = lane & 15;
  const MxFewRows l = mx_few_rows((FM_LDS char*)mx_few_lds + NW * 1024, kd, max_rows);
  // weight rows: 8 of gate, 8 of up (I % 8 == 0)
  const size_t wr = n0 + (r16 & 7);
  const uint8_t* const w[1] = {(r16 < 8 ? ld_scalar(a.W.qg + sl) : ld_scalar(a.W.qu + sl)) + wr * (up32(ra.d) / 2)};
  const uint8_t* const s[1] = {(r16 < 8 ? ld_scalar(a.W.sg + sl) : ld_scalar(a.W.su + sl)) + wr * kd * 4};
  int k0, k1;
  mx_few_part<NW>(kd, k0, k1);
  for (int m0 = 0; m0 < sr.nrows; m0 += max_rows) {
    const int n = min(max_rows, sr.nrows - m0);
    f32x4_t acc[1] = {{0.f, 0.f, 0.f, 0.f}};
    mx_few_sums<1, BS>(w, s, up32(ra.d) / 32, l, n, k0, k1, [&] {
      mx_few_stage<64 * NW>(l, n, kd, ra.d, [&](int r) {
        const size_t tok = sr.shared ? m0 + r : min(max(gptr(a.perm_token)[sr.xrow0 + m0 + r], 0), ra.Tn - 1);
        return X + tok * ra.d;
      });
    }, acc);
    red[wave_id() * 64 + lane] = acc[0];
    __syncthreads();
    for (int i = threadIdx.x; i < 8 * n; i += 64 * NW) {
      const int row = i >> 3, c = i & 7;
      const float g = mx_few_sum<1, NW>(red, 0, row, c), u = mx_few_sum<1, NW>(red, 0, row, 8 + c);
      gptr(a.w.hf)[(size_t)(sr.orow0 + m0 + row) * I + n0 + c] = g * sigm_fast(g) * u;
    }
    __syncthreads();   // red and the rows are read
  }
}

template <int NW, int BS>
__global__ __launch_bounds__(64 * NW) void k_mx_few_down(MxArgs a, int NT, int max_rows) {
  FM_LDS f32x4_t* const red = (FM_LDS f32x4_t*)mx_few_lds;
  const RowArgs& ra = a.ra;
  SlotRows sr;
  const int sl = active_slot(ra, blockIdx.x / NT, sr);
  if (sl < 0) return;
  const int n0 = (blockIdx.x % NT) * 32, d = ra.d, nI = up128(ra.I) / 128;
  const int lane = lane_id(), r16 = lane & 15;
  const MxFewRows l = mx_few_rows((FM_LDS char*)mx_few_lds + NW * 2048, nI, max_rows);
  const uint8_t *w[2], *s[2];
#pragma unroll
  for (int f = 0; f < 2; ++f) {
    const size_t r = min(n0 + 16 * f + r16, d - 1);
    w[f] = ld_scalar(a.W.qd + sl) + r * (up32(ra.I) / 2);
    s[f] = ld_scalar(a.W.sd + sl) + r * nI * 4;
  }
  int k0, k1;
  mx_few_part<NW>(nI, k0, k1);
  for (int m0 = 0; m0 < sr.nrows; m0 += max_rows) {
    const int n = min(max_rows, sr.nrows - m0);
    const size_t row0 = (size_t)(sr.orow0 + m0);
    f32x4_t acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    mx_few_sums<2, BS>(w, s, up32(ra.I) / 32, l, n, k0, k1, [&] {
      mx_few_stage<64 * NW>(l, n, nI, ra.I, [&](int r) { return (const float*)a.w.hf + (row0 + r) * ra.I; });
    }, acc);
#pragma unroll
    for (int f = 0; f < 2; ++f) red[(wave_id() * 2 + f) * 64 + lane] = acc[f];
    __syncthreads();
    // 16 lanes per row, two columns each
    for (int r = threadIdx.x >> 4; r < n; r += 4 * NW) {
      const int c = (threadIdx.x & 15) * 2;
      if (n0 + c >= d) break;
      const float v0 = mx_few_sum<2, NW>(red, c >> 4, r, c & 15), v1 = mx_few_sum<2, NW>(red, c >> 4, r, (c & 15) + 1);
      *(FM_GLOBAL uint32_t*)((uint16_t*)a.O + (row0 + r) * d + n0 + c) = pk_bf16(v0, v1);
    }
    __syncthreads();   // red and the rows are read
  }
}

// Whether a call takes the kernels for a few tokens.  us there and on 64-row tiles, replayed
// from a graph: d = 4096, I = 688, 16 slots, top-4: 1 token 11, 22; 4 tokens 19, 24; 8 27,
// 26.  d = 2048, I = 1408, 64 + 2 slots, top-6 (calls among others): 1 token (1408 blocks)
// 16, 20; 2 (2464) 22, 23; 4 (4576) 33, 26.  d = 512, I = 256, 8 slots, top-2: 1 token 6.4,
// 11.3; 8 7.3, 11.0.  d = 128, I = 64: 6.3, 10.5.  A block's rows have to fit the LDS.
bool mx_few_tokens(const moe_layer_mx4* L, int T, long active) {
  return T <= MX_FEW && active * (L->I / 8) <= 2048 && T * mx_few_row_bytes(up128(L->d) / 128) <= 56 * 1024 &&
         T * mx_few_row_bytes(up128(L->I) / 128) <= 52 * 1024;
}
// Whether it takes 256 x 256 tiles, one block of 8 waves per compute unit, rather than
// 128 x 128 ones (64 x 128 where few rows are left), two of 4 waves, whose blocks run
// over each other's tile boundaries but request twice as much per MFMA: with very many
// rows per slot.  us of the small and the large tiles: d = 4096, I = 1024, 64 slots, top-8:
// 2048 rows per slot 1421, 1273; 512 401, 403; the first layer above at 375 rows per
// slot 80, 81; 175 46, 54; 83 38, 35; the second at 384 297, 298; 159 145, 166; 74 102, 114;
// the third at 8192 58, 68.
bool mx_large_tiles(const moe_layer_mx4* L, int T, int k, long active) {
  const double r = (double)T * (k + L->S_shared) / active;
  return r >= 1000 && active * (r / 256 + 0.5) * ((L->I + 127) / 128) >= 1024;
}

template <class C, class HALF> void mx_tiles(const MxArgs& a, const bf16* X, hipStream_t st) {
  const RowArgs& ra = a.ra;
  const int nb = act_blocks(ra.d);
  hipLaunchKernelGGL(k_mx_prep, dim3(cdiv((long)ra.Tn * nb, 16) + 1), dim3(256), 0, st, X, ra, C::RA, nb, a.w.xq, a.w.xs,
                     a.w.mbase);
  hipLaunchKernelGGL((k_mx_tiles<C, HALF, false>), tile_grid<C>(ra, cdiv(ra.I, C::RB / 2)), dim3(64 * C::NW), 0, st, a);
  hipLaunchKernelGGL((k_mx_tiles<C, HALF, true>), tile_grid<C>(ra, cdiv(ra.d, C::RB)), dim3(64 * C::NW), 0, st, a);
}

int check_rows(const void* a, const char* an, const void* b, const char* bn, const void* c, const char* cn, long rows,
               int cols) {
  if (rows <= 0 || cols <= 0) return fail(MOE_ERR_ARG, "rows=%ld cols=%d", rows, cols);
  if (cols % 8 || cols > 1 << 30) return fail(MOE_ERR_UNSUPPORTED, "cols=%d not a multiple of 8 up to 2^30", cols);
  FM_TRY(need(a, an)); FM_TRY(need(b, bn)); FM_TRY(need(c, cn));
  FM_TRY(need_aligned(a, an)); FM_TRY(need_aligned(b, bn)); FM_TRY(need_aligned(c, cn));
  return MOE_OK;
}

// Slots that may hold rows.
long mx_active(const moe_layer_mx4* L, int T, int k) {
  const long R = (long)T * k;
  return (R < L->S_routed ? R : L->S_routed) + L->S_shared;
}

}  // namespace

int mx4_tile(const moe_layer_mx4* L, int T, int k) {
  const long active = mx_active(L, T, k);
  return mx_few_tokens(L, T, active) ? 0 : mx_large_tiles(L, T, k, active) ? 256 : 128;
}

}  // namespace fm

using namespace fm;

extern "C" int moe_quantize_mxfp4(const void* W, int dtype, long rows, int cols, uint8_t* codes, uint8_t* scale,
                                  void* stream) {
  clear_error();
  FM_TRY(need_dtype_float(dtype, "dtype"));
  FM_TRY(check_rows(W, "W", codes, "codes", scale, "scale", rows, cols));
  const int nb = up128(cols) / 128, es = esize(dtype);
  // launches of at most 2^27 items: 16 threads each, and a launch of 2^32 threads or more
  // runs some of them only, without an error
  const long step = (1L << 27) / nb;   // nb <= 2^23
  for (long r = 0; r < rows; r += step) {
    const uint32_t items = (uint32_t)((rows - r < step ? rows - r : step) * nb);
    const char* w = (const char*)W + (size_t)r * cols * es;
    uint8_t* q = codes + (size_t)r * (up32(cols) / 2);
    uint8_t* s = scale + (size_t)r * nb * 4;
    if (dtype == MOE_BF16)
      hipLaunchKernelGGL(k_quantize_mx<bf16>, dim3(cdiv(items, 16)), dim3(256), 0, as_stream(stream), (const bf16*)w,
                         items, cols, nb, q, s);
    else
      hipLaunchKernelGGL(k_quantize_mx<float>, dim3(cdiv(items, 16)), dim3(256), 0, as_stream(stream), (const float*)w,
                         items, cols, nb, q, s);
  }
  return check_launch("moe_quantize_mxfp4");
}

extern "C" int moe_dequant_mxfp4(const uint8_t* codes, const uint8_t* scale, long rows, int cols, int out_dtype,
                                 void* out, void* stream) {
  clear_error();
  FM_TRY(need_dtype_float(out_dtype, "out_dtype"));
  FM_TRY(check_rows(codes, "codes", scale, "scale", out, "out", rows, cols));
  const int n8 = cols / 8, es = esize(out_dtype);
  // launches of less than 2^31 items, a thread each, so that the kernel divides 32-bit numbers
  const long step = 0x7FFFFFF0L / n8;
  for (long r = 0; r < rows; r += step) {
    const uint32_t items = (uint32_t)((rows - r < step ? rows - r : step) * n8);
    const uint8_t* q = codes + (size_t)r * (up32(cols) / 2);
    const uint8_t* s = scale + (size_t)r * (up128(cols) / 32);
    char* o = (char*)out + (size_t)r * cols * es;
    if (out_dtype == MOE_BF16)
      hipLaunchKernelGGL(k_dequant_mx<bf16>, dim3(cdiv(items, 256)), dim3(256), 0, as_stream(stream), q, s, items, cols,
                         n8, (bf16*)o);
    else
      hipLaunchKernelGGL(k_dequant_mx<float>, dim3(cdiv(items, 256)), dim3(256), 0, as_stream(stream), q, s, items, cols,
                         n8, (float*)o);
  }
  return check_launch("moe_dequant_mxfp4");
}

extern "C" size_t moe_grouped_swiglu_fwd_mx4_workspace_size(const moe_layer_mx4* L, int T, int k) {
  if (!L || T < 0 || k <= 0 || L->d <= 0 || L->I <= 0 || L->S_routed < 0 || L->S_shared < 0) return 0;
  size_t bytes;
  mx_ws_at(nullptr, L, T, k, &bytes);
  return bytes;
}

extern "C" int moe_grouped_swiglu_fwd_mx4(const moe_layer_mx4* L, const void* X, const int32_t* perm_token,
                                          const int32_t* offsets, int T, int k, void* O, void* ws, size_t ws_bytes,
                                          void* stream) {
  clear_error();
  if (!L) return fail(MOE_ERR_ARG, "layer must not be NULL");
  if (L->d <= 0 || L->I <= 0) return fail(MOE_ERR_ARG, "layer d=%d I=%d", L->d, L->I);
  if (L->d % 8 || L->I % 8 || L->d > 1 << 30 || L->I > 1 << 30)
    return fail(MOE_ERR_UNSUPPORTED, "4-bit layer d=%d I=%d must be multiples of 8 up to 2^30", L->d, L->I);
  if (L->S_routed < 0 || L->S_shared < 0 || L->S_routed + L->S_shared < 1 || L->S_routed > 512 || L->S_shared > 511)
    return fail(MOE_ERR_ARG, "layer S_routed=%d S_shared=%d", L->S_routed, L->S_shared);
  // byte offsets within a matrix, and of a token's packed row, are 32 bits wide
  if ((long long)up128(L->d) * up128(L->I) > (1LL << 32))
    return fail(MOE_ERR_UNSUPPORTED, "4-bit layer d=%d I=%d: more than 2^32 weights in a matrix", L->d, L->I);
  FM_TRY(need(L->q_gate, "layer q_gate")); FM_TRY(need(L->q_up, "layer q_up")); FM_TRY(need(L->q_down, "layer q_down"));
  FM_TRY(need(L->s_gate, "layer s_gate")); FM_TRY(need(L->s_up, "layer s_up")); FM_TRY(need(L->s_down, "layer s_down"));
  if (T < 0 || k <= 0 || k > 16) return fail(MOE_ERR_ARG, "T=%d k=%d", T, k);
  if ((long long)T * up128(L->d) > (1LL << 32))
    return fail(MOE_ERR_UNSUPPORTED, "T=%d tokens of d=%d: more than 2^32 values", T, L->d);
  if (T == 0) return MOE_OK;
  FM_TRY(need(X, "X")); FM_TRY(need(offsets, "offsets")); FM_TRY(need(O, "O")); FM_TRY(need(ws, "ws"));
  if (L->S_routed > 0) FM_TRY(need(perm_token, "perm_token"));
  FM_TRY(need_aligned(X, "X")); FM_TRY(need_aligned(perm_token, "perm_token")); FM_TRY(need_aligned(offsets, "offsets"));
  FM_TRY(need_aligned(O, "O")); FM_TRY(need_aligned(ws, "ws"));
  size_t bytes;
  const MxWs w = mx_ws_at(ws, L, T, k, &bytes);
  if (ws_bytes < bytes) return fail(MOE_ERR_WORKSPACE, "workspace %zu < %zu bytes", ws_bytes, bytes);
  hipStream_t st = as_stream(stream);
  if (debug_checks() && L->S_routed > 0) {
    int rows = 0;
    FM_TRY(debug_check_offsets(offsets, L->S_routed, T, k, st));
    FM_TRY(debug_rows(offsets, L->S_routed, st, &rows));
    FM_TRY(debug_check_tokens(perm_token, rows, T, st));
  }
  const RowArgs ra{offsets, w.mbase, L->S_routed, L->S_routed + L->S_shared, T, k, L->d, L->I, L->I};
  const MxArgs a{{L->q_gate, L->q_up, L->q_down, L->s_gate, L->s_up, L->s_down}, w, perm_token, ra, (bf16*)O};
  const int nb = up128(L->d) / 128;
  const bf16* const Xb = (const bf16*)X;
  const int tile = mx4_tile(L, T, k);
  if (tile == 0) {
    const long active = mx_active(L, T, k);
    const int ng = L->I / 8, nd = cdiv(L->d, 32);
    hipLaunchKernelGGL((k_mx_few_gate_up<4, 4>), dim3(active * ng), dim3(256), T * mx_few_row_bytes(nb) + 4 * 1024, st, a,
                       Xb, ng, T);
    hipLaunchKernelGGL((k_mx_few_down<4, 2>), dim3(active * nd), dim3(256),
                       T * mx_few_row_bytes(up128(L->I) / 128) + 4 * 2048, st, a, nd, T);
    return check_launch("moe_grouped_swiglu_fwd_mx4");
  }
  if (tile == 256) mx_tiles<M256, M128>(a, Xb, st);
  else mx_tiles<Q128, Q64>(a, Xb, st);
  return check_launch("moe_grouped_swiglu_fwd_mx4");
}
