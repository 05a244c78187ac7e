// 4-bit microscaled floating point: packing, unpacking, and the product on the scaled matrix instruction of gfx950
// (clt_mx4_quantise, clt_mx4_dequantise, clt_mx4_product; the packed layout is described in include/clt.h).
#include "common.h"

#include <type_traits>

namespace clt {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

// Byte offsets of block `kb` (32 elements, counted from the start of the row) of row r in a packed matrix of KS steps
__device__ __forceinline__ size_t code_offset(int r, int kb, int KS) {
  return (((size_t)(r >> 4) * KS + (kb >> 2)) << 10) + (((kb & 3) * 16 + (r & 15)) << 4);
}
__device__ __forceinline__ size_t scale_offset(int r, int kb, int KS) {
  return (((size_t)(r >> 6) * KS + (kb >> 2)) << 8) + (((kb & 3) * 16 + (r & 15)) << 2) + ((r >> 4) & 3);
}

// Scale byte of a block whose largest magnitude has this fp32 image (a largest of 1.75 * 2^e or more takes the next power)
__device__ __forceinline__ uint32_t block_scale(uint32_t top) {
  return top >= 0x7f800000u ? 255u : (uint32_t)max((int)((top + 0x200000u) >> 23) - 2, 0);
}

// Eight floats -> eight codes.  The conversion instruction rounds to nearest even and saturates; its scale is a float, 2^(s-127), which
// for s = 0 is the denormal 2^-127: such blocks are multiplied by 2^64 first and converted with 2^(s-127+64).
__device__ __forceinline__ uint32_t to_codes(const float* x, uint32_t s) {
  const bool small = s < 64u;
  const float scale = __uint_as_float((small ? s + 64u : s) << 23), up = small ? 0x1p64f : 1.f;
  float y[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) y[j] = x[j] * up;
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[0], y[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[2], y[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[4], y[5], scale, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[6], y[7], scale, 3);
  return s == 255u ? 0u : w;
}

__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  v = max(v, dpp_move<0xB1>(v));          // quad_perm [1,0,3,2]
  return max(v, dpp_move<0x4E>(v));       // quad_perm [2,3,0,1]
}

// 4 x 4 words across the lanes of a quad: word j of lane i <-> word i of lane j
__device__ __forceinline__ void quad_transpose(uint32_t (&w)[4], int i) {
  const bool odd = i & 1, high = i & 2;
  uint32_t a[4];
#pragma unroll
  for (int j = 0; j < 4; j += 2) {      // lanes i, i ^ 1
    const uint32_t x = dpp_move<0xB1>(odd ? w[j] : w[j + 1]);
    a[j] = odd ? x : w[j];
    a[j + 1] = odd ? w[j + 1] : x;
  }
#pragma unroll
  for (int j = 0; j < 2; ++j) {         // lanes i, i ^ 2
    const uint32_t x = dpp_move<0x4E>(high ? a[j] : a[j + 2]);
    w[j] = high ? x : a[j];
    w[j + 2] = high ? a[j + 2] : x;
  }
}

// Eight consecutive elements as they come out of memory, and as floats
template <typename TE> struct Eight;
template <> struct Eight<float> {
  f32x4 a, b;
  __device__ __forceinline__ void load(const float* p) { a = *reinterpret_cast<const f32x4*>(p); b = *reinterpret_cast<const f32x4*>(p + 4); }
  __device__ __forceinline__ void zero() { a = b = f32x4{0.f, 0.f, 0.f, 0.f}; }
  __device__ __forceinline__ float get(int j) const { return j < 4 ? a[j] : b[j - 4]; }
};
template <> struct Eight<bf16_t> {
  u32x4 a;
  __device__ __forceinline__ void load(const bf16_t* p) { a = *reinterpret_cast<const u32x4*>(p); }
  __device__ __forceinline__ void zero() { a = u32x4{0u, 0u, 0u, 0u}; }
  __device__ __forceinline__ float get(int j) const { return __uint_as_float(j & 1 ? a[j >> 1] & 0xffff0000u : a[j >> 1] << 16); }
};
template <> struct Eight<int8_t> {
  uint2 a;
  __device__ __forceinline__ void load(const int8_t* p) { a = *reinterpret_cast<const uint2*>(p); }
  __device__ __forceinline__ void zero() { a = make_uint2(0u, 0u); }
  __device__ __forceinline__ float get(int j) const { return (float)(int8_t)((j < 4 ? a.x : a.y) >> (8 * (j & 3))); }
};

// Rows along the contraction.  A wavefront packs 16 rows by one step (1 KB of codes): four lanes share a block, eight elements each, so
// loads are 16 bytes of bf16 per lane and a block's largest element is two maxima inside a quad away; its four blocks of a row come
// one after the other, their loads in flight together.  A workgroup is a panel of 64 rows (whose scales share 256 bytes) by
// QUANTISE_STEPS steps.  Bound by memory: 16 layers of 4096 rows of 2048 bf16 (340 MB) 60 us, 5.7 TB/s (64 us with one step).  Small calls are not: 6 layers of
// 1037 int8 rows of 2056 (20 MB) take 8.4 us, twice their bytes' time, in about seven instructions an element, the maximum and the exchange inside a
// quad among them.
constexpr int QUANTISE_STEPS = 2;
template <typename TE>
__global__ __launch_bounds__(256) void mx4_quantise_kernel(int rows, int K, int KS, int chunks, const TE* __restrict__ a,
                                                           const float* __restrict__ a_scale, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
  const int lane = threadIdx.x & 63, sub = threadIdx.x >> 6, panels = (rows + 63) >> 6, l = blockIdx.y;
  const int panel = blockIdx.x / chunks, ks0 = (blockIdx.x - panel * chunks) * QUANTISE_STEPS;
  const int part = lane & 3, r = panel * 64 + sub * 16 + (lane >> 2);
  if (r >= rows) return;
  const TE* row = a + ((size_t)l * rows + r) * K;
  const float s = a_scale ? a_scale[(size_t)l * rows + r] : 1.f;
  uint8_t* tile = codes + (((size_t)(l * panels + panel) * 4 + sub) * KS << 10) + part * 256 + (lane >> 2) * 16;
  uint8_t* sc = scales + ((size_t)(l * panels + panel) * KS << 8) + ((part * 16 + (lane >> 2)) << 2) + sub;
  Eight<TE> in[QUANTISE_STEPS][4];
#pragma unroll
  for (int t = 0; t < QUANTISE_STEPS; ++t)
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
      const int k = (ks0 + t) * 128 + kb * 32 + part * 8;      // K is a multiple of 8
      if (k < K) in[t][kb].load(row + k);
      else in[t][kb].zero();
    }
#pragma unroll
  for (int t = 0; t < QUANTISE_STEPS; ++t) {
    if (ks0 + t >= KS) return;
    uint32_t mine = 0, w[4];
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
      float x[8];
      uint32_t top = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        x[j] = in[t][kb].get(j) * s;
        top = max(top, __float_as_uint(x[j]) & 0x7fffffffu);
      }
      const uint32_t e = block_scale(quad_max(top));
      w[kb] = to_codes(x, e);
      mine = part == kb ? e : mine;
    }
    quad_transpose(w, part);      // this lane: the four words of block `part`
    *reinterpret_cast<u32x4*>(tile + ((size_t)(ks0 + t) << 10)) = u32x4{w[0], w[1], w[2], w[3]};
    sc[(size_t)(ks0 + t) << 8] = (uint8_t)mine;
  }
}

// Columns along the contraction (a is [K][rows]).  A lane takes one dword of columns (two of bf16, one of fp32) and the 32 elements of
// one block of each, so that a wavefront's loads are 256 consecutive bytes; the wavefronts of a workgroup take the four blocks of a step.
// 12 matrices of 768 by 6144 bf16 (143 MB): 21.6 us, 6.6 TB/s out of the Infinity Cache in part.
template <typename TE>
__global__ __launch_bounds__(256) void mx4_quantise_transposed_kernel(int rows, int K, int KS, const TE* __restrict__ a, uint8_t* __restrict__ codes,
                                                                      uint8_t* __restrict__ scales) {
  constexpr int C = 4 / sizeof(TE);
  const int lane = threadIdx.x & 63, panels = (rows + 63) >> 6, l = blockIdx.z, kb = blockIdx.y * 4 + (threadIdx.x >> 6);
  const int r = (blockIdx.x * 64 + lane) * C;      // rows is a multiple of 8
  if (r >= rows) return;
  const TE* p = a + ((size_t)l * K + (size_t)kb * 32) * rows + r;
  uint32_t in[32];
#pragma unroll
  for (int j = 0; j < 32; ++j) {
    in[j] = 0;
    if (kb * 32 + j < K) in[j] = *reinterpret_cast<const uint32_t*>(p + (size_t)j * rows);
  }
#pragma unroll
  for (int c = 0; c < C; ++c) {
    float x[32];
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 32; ++j) {
      const uint32_t u = C == 1 ? in[j] : c ? in[j] & 0xffff0000u : in[j] << 16;
      x[j] = __uint_as_float(u);
      top = max(top, u & 0x7fffffffu);
    }
    const uint32_t e = block_scale(top);
    const u32x4 w = {to_codes(x, e), to_codes(x + 8, e), to_codes(x + 16, e), to_codes(x + 24, e)};
    *reinterpret_cast<u32x4*>(codes + ((size_t)l * panels * 4 * KS << 10) + code_offset(r + c, kb, KS)) = w;
    scales[((size_t)l * panels * KS << 8) + scale_offset(r + c, kb, KS)] = (uint8_t)e;
  }
}

// The way back, cut as the way there: a wavefront takes 16 rows by one step; the lanes of a quad exchange the words of their four blocks, so that each
// has eight consecutive elements of each block.  12 layers of 6144 rows of 768 into bf16 (143 MB): 22.8 us, 6.3 TB/s.
template <typename T>
__global__ __launch_bounds__(256) void mx4_dequantise_kernel(int rows, int K, int KS, int chunks, Mx4 a, T* __restrict__ out) {
  const int lane = threadIdx.x & 63, sub = threadIdx.x >> 6, panels = (rows + 63) >> 6, l = blockIdx.y;
  const int panel = blockIdx.x / chunks, ks0 = (blockIdx.x - panel * chunks) * QUANTISE_STEPS;
  const int part = lane & 3, r = panel * 64 + sub * 16 + (lane >> 2);
  if (r >= rows) return;
  const uint8_t* tile = a.codes + (((size_t)(l * panels + panel) * 4 + sub) * KS << 10) + part * 256 + (lane >> 2) * 16;
  const uint8_t* sc = a.scales + ((size_t)(l * panels + panel) * KS << 8) + ((part * 16 + (lane >> 2)) << 2) + sub;
  T* row = out + ((size_t)l * rows + r) * K;
  u32x4 in[QUANTISE_STEPS];
  uint32_t mine[QUANTISE_STEPS];
#pragma unroll
  for (int t = 0; t < QUANTISE_STEPS; ++t) {
    const int ks = min(ks0 + t, KS - 1);
    in[t] = *reinterpret_cast<const u32x4*>(tile + ((size_t)ks << 10));
    mine[t] = sc[(size_t)ks << 8];
  }
#pragma unroll
  for (int t = 0; t < QUANTISE_STEPS; ++t) {
    uint32_t w[4] = {in[t][0], in[t][1], in[t][2], in[t][3]};
    quad_transpose(w, part);
    const float f = scale_value(mine[t]);
    const float scale[4] = {__uint_as_float(dpp_move<0x00>(__float_as_uint(f))), __uint_as_float(dpp_move<0x55>(__float_as_uint(f))),
                            __uint_as_float(dpp_move<0xAA>(__float_as_uint(f))), __uint_as_float(dpp_move<0xFF>(__float_as_uint(f)))};
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
      const int k = (ks0 + t) * 128 + kb * 32 + part * 8;
      if (k >= K) continue;
      const auto x = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[kb], 1.0f, 0), y = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[kb], 1.0f, 1);
      const auto z = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[kb], 1.0f, 2), u = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[kb], 1.0f, 3);
      Elem<T>::store4(row + k, make_float4(x[0] * scale[kb], x[1] * scale[kb], y[0] * scale[kb], y[1] * scale[kb]));
      Elem<T>::store4(row + k + 4, make_float4(z[0] * scale[kb], z[1] * scale[kb], u[0] * scale[kb], u[1] * scale[kb]));
    }
  }
}

// ---- product -------------------------------------------------------------------------------------------------------
//
// v_mfma_scale_f32_16x16x128: a lane's operand is the 32 elements (16 bytes) of one block, row lane % 16, block lane / 16,
// with the block's scale in one byte of a register that the instruction selects: what a packed tile of 16 rows holds at byte
// 16 * lane, and what a panel's step holds of scales at byte 4 * lane.  The rows of B (features) are the instruction's first
// operand, those of A (tokens) its second, so a lane's four results are four consecutive features of one token.

// Loads of 16 or 4 bytes per lane, consecutive lanes, from `offset` bytes on: through buffer descriptors, which keep everything but
// the lane's own offset (one register for all loads) in scalar registers.  A panel of K <= 2^22 is at most 2^27 bytes.
struct Source {
  __amdgpu_buffer_rsrc_t d;
  __device__ __forceinline__ Source(const uint8_t* base) : d(__builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base), 0, 0x7fffffff, 0x00027000)) {}
  __device__ __forceinline__ u32x4 lanes16(uint32_t lane, uint32_t offset) const {
    return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(d, (int)(lane * 16), (int)offset, 0));
  }
  __device__ __forceinline__ uint32_t lanes4(uint32_t lane, uint32_t offset) const {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_raw_buffer_load_b32(d, (int)(lane * 4), (int)offset, 0));
  }
};

// Operands of one panel (64 rows) and step
struct PanelFrag { u32x4 c[4]; uint32_t s; };
struct Panel {
  Source codes, scales; int KS;
  __device__ __forceinline__ Panel(Mx4 b, size_t panel, int KS) : codes(b.codes + ((panel * 4 * KS) << 10)), scales(b.scales + ((panel * KS) << 8)), KS(KS) {}
  __device__ __forceinline__ u32x4 tile(int j, int ks, uint32_t lane) const { return codes.lanes16(lane, (uint32_t)(j * KS + ks) << 10); }
  __device__ __forceinline__ uint32_t scale(int ks, uint32_t lane) const { return scales.lanes4(lane, (uint32_t)ks << 8); }
};

template <int OB, int OA> __device__ __forceinline__ f32x4 mfma(u32x4 b, uint32_t bs, u32x4 a, uint32_t as, f32x4 c) {
  const i32x8 A = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0}, B = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(B, A, c, 4, 4, OB, (int)bs, OA, (int)as);
}
// one tile of tokens, whose scales are in byte i of their panel's, by the four tiles of a panel of features
template <int I> __device__ __forceinline__ void mfma4(const PanelFrag& b, u32x4 a, uint32_t as, f32x4 (&c)[4]) {
  c[0] = mfma<0, I>(b.c[0], b.s, a, as, c[0]);
  c[1] = mfma<1, I>(b.c[1], b.s, a, as, c[1]);
  c[2] = mfma<2, I>(b.c[2], b.s, a, as, c[2]);
  c[3] = mfma<3, I>(b.c[3], b.s, a, as, c[3]);
}
__device__ __forceinline__ void mfma4(int i, const PanelFrag& b, u32x4 a, uint32_t as, f32x4 (&c)[4]) {
  switch (i & 3) {
    case 0: mfma4<0>(b, a, as, c); break;
    case 1: mfma4<1>(b, a, as, c); break;
    case 2: mfma4<2>(b, a, as, c); break;
    default: mfma4<3>(b, a, as, c);
  }
}

// Lanes 8..15 of each row of 16 get `b` of the lane eight before them, the others keep `a`; and the other way round.
__device__ __forceinline__ uint32_t upper_from(uint32_t a, uint32_t b) { return (uint32_t)__builtin_amdgcn_update_dpp((int)a, (int)b, 0x128, 0xF, 0xC, false); }
__device__ __forceinline__ uint32_t lower_from(uint32_t a, uint32_t b) { return (uint32_t)__builtin_amdgcn_update_dpp((int)a, (int)b, 0x128, 0xF, 0x3, false); }

// Stores of sixteen tokens' features.  v[j]: features 16 j + 4 q .. + 3 (q = lane / 16) of token lane % 16 of the panel and tile at o (rows
// `stride` apart); `features` and `tokens` are inside the matrix.  The output is written once and large, so the stores are
// streaming ones, and those only pay in whole 128-byte lines (16 layers of 4096 tokens by 8192 features by K = 128, all stores: 613 us in pieces of
// 32 bytes, 237 through the L2).  So the lanes first exchange what they hold, in registers.
// bf16: the lanes of q = 0, 1 (and 2, 3) swap halves, so that each has eight consecutive features of two tiles, w[0] of tile 0 (even q) or 2
// and w[1] of tile 1 or 3; then tokens t and t + 8 swap, so that one store holds the lines of tokens 0..7 and the other of 8..15.
__device__ __forceinline__ void store_tile(bf16_t* o, size_t stride, const f32x4 (&v)[4], int lane, int features, int tokens) {
  const int q = lane >> 4, t = lane & 7, j = (lane >> 3) & 1;
  uint32_t w[2][4];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const auto x = __builtin_amdgcn_permlane16_swap(pack_bf16x2(v[i][2 * h], v[i][2 * h + 1]), pack_bf16x2(v[i + 2][2 * h], v[i + 2][2 * h + 1]), false, false);
      w[i][h] = x[0];
      w[i][2 + h] = x[1];
    }
  u32x4 a, b;
#pragma unroll
  for (int h = 0; h < 4; ++h) { a[h] = upper_from(w[0][h], w[1][h]); b[h] = lower_from(w[1][h], w[0][h]); }
  const int f = 16 * j + 32 * (q & 1) + 8 * (q >> 1);
  bf16_t* p = o + t * stride + f;
  if (f < features && t < tokens) __builtin_nontemporal_store(a, reinterpret_cast<u32x4*>(p));
  if (f < features && t + 8 < tokens) __builtin_nontemporal_store(b, reinterpret_cast<u32x4*>(p + 8 * stride));
}
// fp32: tokens t and t + 8 swap tiles 1 and 0, and 3 and 2
__device__ __forceinline__ void store_tile(float* o, size_t stride, const f32x4 (&v)[4], int lane, int features, int tokens) {
  const int q = lane >> 4, t = lane & 7, j = (lane >> 3) & 1;
#pragma unroll
  for (int i = 0; i < 4; i += 2) {
    u32x4 a, b;
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      const uint32_t x = __float_as_uint(v[i][h]), y = __float_as_uint(v[i + 1][h]);
      a[h] = upper_from(x, y);
      b[h] = lower_from(y, x);
    }
    const int f = 16 * (i + j) + 4 * q;
    float* p = o + t * stride + f;
    if (f < features && t < tokens) __builtin_nontemporal_store(a, reinterpret_cast<u32x4*>(p));
    if (f < features && t + 8 < tokens) __builtin_nontemporal_store(b, reinterpret_cast<u32x4*>(p + 8 * stride));
  }
}

template <int i> using I = std::integral_constant<int, i>;
struct ProductArgs { int M, N, KS; Mx4 a, b; const float* bias; const float* theta; void* out; };

// Accumulators of MT tiles of 16 tokens by one panel of features begin at the features' bias: an addition that costs nothing.
template <int MT>
__device__ __forceinline__ void begin(const ProductArgs& p, int l, int panel, int lane, f32x4 (&acc)[MT][4]) {
  const int f = panel * 64 + 4 * (lane >> 4);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    f32x4 b = {0.f, 0.f, 0.f, 0.f};
    if (p.bias && f + 16 * j < p.N) b = *reinterpret_cast<const f32x4*>(p.bias + (size_t)l * p.N + f + 16 * j);      // N is a multiple of 8
#pragma unroll
    for (int i = 0; i < MT; ++i) acc[i][j] = b;
  }
}
// Threshold, rounding and stores
template <typename T, bool THETA, int MT>
__device__ __forceinline__ void finish(const ProductArgs& p, int l, int token0, int panel, int lane, const f32x4 (&acc)[MT][4]) {
  const int f = panel * 64 + 4 * (lane >> 4);
  f32x4 theta[4];
  if (THETA) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      theta[j] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (f + 16 * j < p.N) theta[j] = *reinterpret_cast<const f32x4*>(p.theta + (size_t)l * p.N + f + 16 * j);
    }
  }
  T* o = static_cast<T*>(p.out) + ((size_t)l * p.M + token0) * p.N + panel * 64;
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int m = token0 + i * 16;
    if (m >= p.M) break;
    f32x4 v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int k = 0; k < 4; ++k) v[j][k] = !THETA || acc[i][j][k] > theta[j][k] ? acc[i][j][k] : 0.f;
    store_tile(o + (size_t)(i * 16) * p.N, p.N, v, lane, p.N - panel * 64, p.M - m);
  }
}

// Many tokens: a workgroup takes tiles of 128 tokens by 256 features one after the other, each of its four wavefronts one panel of 64
// features by all the tokens (8 x 4 accumulators of 16 x 16).  A panel is read by one wavefront only and goes from memory into its
// registers, one step ahead; the tokens are fetched three steps ahead and staged in LDS, in three stages of one step each.  Both run on
// into the next tile.  Two workgroups share a compute unit, so that one's epilogue runs under the other's matrix instructions.
// Measured: 16 layers of 4096 by 8192 by K = 2048, bf16 results, 590 to 610 us in a loop of 100 (two cards), 3.6 to 3.7 PFLOP/s, and 615 to 660 behind other work;
// fp32 results 739.  A bare loop of the instruction on random operands reaches 7.2, with the LDS reads and the barrier 6.5; at K = 32768 this kernel 4.5 on random
// numbers and 5.3 on zeros, where power is no limit.  No one unit bounds it: of the cycles of a step, 1024 are matrix instructions of a compute unit's eight
// wavefronts, 860 the operands' way through the vector cache (64 bytes a cycle, 6.75 KB a wavefront), 40 % the LDS, and they do not overlap altogether.  With
// parts left out, of 632 us in that run: half of the features' loads 600, the scales' 602, all of the features' 566, the tokens' as well 533; with all loads,
// of 619: no stores 551, nor the results' way through LDS 534, nor the threshold 519, and that on zeros 443.  A tile of 128 by 128 to a wavefront would need a third fewer
// operands and all registers of a SIMD, with no second workgroup for the epilogue to hide under.
constexpr int PT = 8;             // tiles of 16 tokens
constexpr int AHEAD = 3;          // of these, the operands under way from LDS
constexpr int WORKGROUPS = 512;   // two on each of 256 compute units

// Quotients n / d for n < 2^31 by a multiplication (Granlund and Montgomery's division by invariant integers): m = floor(2^(31+s) / d) + 1 with 2^(s-1) < d <= 2^s is too large by less than 2^s / 2^(31+s)
// of itself.  (Division instructions do not exist; a wavefront would spend as long on three quotients as on two steps.)
struct Quotient {
  uint32_t m, s;
  explicit Quotient(uint32_t d) : s(0) {
    while ((1ull << s) < d) ++s;
    m = (uint32_t)((1ull << (31 + s)) / d) + 1;
  }
  __device__ __forceinline__ uint32_t of(uint32_t n) const { return (uint32_t)(((uint64_t)n * m) >> (31 + s)); }
};
// The order of the tiles: layer by layer; eight tiles of tokens at a time (fewer in the last group) through all the features
struct TileOrder {
  uint32_t tiles, per_layer, per_group; int tiles_m; Quotient layer, group, last_rows;
  TileOrder(int L, int tiles_m, int tiles_n) : tiles((uint32_t)((size_t)L * tiles_m * tiles_n)), per_layer((uint32_t)tiles_m * tiles_n), per_group(8 * tiles_n),
    tiles_m(tiles_m), layer(per_layer), group(per_group), last_rows((tiles_m & 7) ? tiles_m & 7 : 8) {}
};
// Where a workgroup stands: a step of one of its tiles
struct Cursor {
  uint32_t t; int ks, l, tm, panel; bool ok;
};
//
// Results leave a wavefront in one of two ways.  Directly: at the end of a tile its 16 or 32 stores are issued at once, and because loads and
// stores are counted in order, the first operands of the next tile are waited for together with all of them.  STAGED (bf16): the results are put into
// LDS (rounded, 14 KB a wavefront, and 2 KB in the stage that is free at that moment, which makes 80 KB for a workgroup), and every step of the next tile
// reads one sixteen tokens' worth back as whole lines and stores it behind its loads, so that a store has a step's time; bias and threshold are fetched with the
// tile's first features.  The stores go through a buffer descriptor that ends with the tile's last token: what lies beyond is not written, without a branch.
// (The place is in the descriptor's base: a 16-byte store whose offset was in a scalar register has lost its first word to the next
// instruction's write of that register, for which the compiler waits only in the other form.)
template <typename T, bool THETA, bool STAGED>
__global__ __launch_bounds__(256, 2) void mx4_product_kernel(ProductArgs p, TileOrder order) {
  static_assert(!STAGED || sizeof(T) == 2, "an fp32 tile does not fit");
  constexpr int STAGE = PT * 64;
  __shared__ u32x4 lds[(STAGED ? 3 + PT - 1 : 3) * STAGE];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int KS = p.KS, panels_m = (p.M + 63) >> 6, panels_n = (p.N + 63) >> 6;
  // Workgroups are dealt to the eight XCDs in turn: each XCD takes a run of consecutive tiles, which go through the features for
  // eight tiles of tokens at a time, so that the tiles at work on an XCD share their operands in its L2.
  const uint32_t xcd = blockIdx.x & 7, per_xcd = gridDim.x >> 3;      // the grid is a multiple of 8
  const uint32_t first = xcd * (order.tiles >> 3) + min(xcd, order.tiles & 7), end = first + (order.tiles >> 3) + (xcd < (order.tiles & 7) ? 1 : 0);
  auto locate = [&](Cursor& c) __attribute__((always_inline)) {
    c.ok = c.t < end;
    const uint32_t t = c.ok ? c.t : first;
    c.l = order.layer.of(t);
    const uint32_t r = t - c.l * order.per_layer, group = order.group.of(r), in_group = r - group * order.per_group;
    const int rows = min(8, order.tiles_m - (int)group * 8), tn = rows == 8 ? in_group >> 3 : order.last_rows.of(in_group);
    c.tm = group * 8 + in_group - tn * rows;
    c.panel = tn * 4 + wave;
  };
  Cursor at{first + (blockIdx.x >> 3), 0, 0, 0, 0, false};
  locate(at);
  if (!at.ok) return;
  // (tiles and panels beyond the matrix: the last one again; what it gives is not stored)
  auto panel_of = [&](const Cursor& c) __attribute__((always_inline)) { return Panel(p.b, (size_t)c.l * panels_n + min(c.panel, panels_n - 1), KS); };
  struct Tokens { Source codes, scales; uint32_t a1, s1; };
  auto tokens_of = [&](const Cursor& c) __attribute__((always_inline)) {
    const uint32_t second = c.tm * 2 + 1 < panels_m ? 1 : 0;      // the second panel of tokens
    return Tokens{Source(p.a.codes + (((size_t)c.l * panels_m * 4 + c.tm * PT) * KS << 10)),
                  Source(p.a.scales + (((size_t)c.l * panels_m + c.tm * 2) * KS << 8)), (second * 4 * KS) << 10, (second * KS) << 8};
  };
  Cursor ca = at, cb = at;      // of the next fetch of tokens and of features (behind the last tile they fetch the first of this XCD, for nothing)
  Panel B = panel_of(cb);
  Tokens A = tokens_of(ca), S = A;      // S: for the tokens' scales, which go with the features
  f32x4 acc[PT][4];
  u32x4 next[2], fa[4];
  PanelFrag fb[2];
  uint32_t sa[2][2];
  auto load_a = [&]() __attribute__((always_inline)) {
    next[0] = A.codes.lanes16(lane, (uint32_t)(wave * KS + ca.ks) << 10);
    next[1] = A.codes.lanes16(lane, A.a1 + ((uint32_t)(wave * KS + ca.ks) << 10));
  };
  auto advance_a = [&]() __attribute__((always_inline)) {
    if (__builtin_expect(++ca.ks == KS, 0)) {
      ca.ks = 0;
      ca.t += per_xcd;
      locate(ca);
      A = tokens_of(ca);
    }
  };
  auto load_b = [&](int buf, int j) __attribute__((always_inline)) { fb[buf].c[j] = B.tile(j, cb.ks, lane); };
  // STAGED: bias and threshold of the next tile, feature `lane` of the panel, fetched when cb comes to it
  float bias_next = 0.f, theta_next = 0.f, theta_now = 0.f;
  auto load_vectors = [&]() __attribute__((always_inline)) {
    const size_t f = (size_t)cb.l * p.N + min(cb.panel * 64 + lane, p.N - 1);
    if (p.bias) bias_next = p.bias[f];
    if (THETA) theta_next = p.theta[f];
  };
  auto spread = [&](float v, int j, int k) __attribute__((always_inline)) { return __uint_as_float((uint32_t)__builtin_amdgcn_ds_bpermute((16 * j + 4 * (lane >> 4) + k) * 4, (int)__float_as_uint(v))); };
  auto start = [&]() __attribute__((always_inline)) {
    if constexpr (STAGED) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float b = spread(bias_next, j, k);
#pragma unroll
          for (int i = 0; i < PT; ++i) acc[i][j][k] = b;
        }
      theta_now = theta_next;
    } else begin(p, at.l, at.panel, lane, acc);
  };
  auto load_scales = [&](int buf) __attribute__((always_inline)) {
    fb[buf].s = B.scale(cb.ks, lane);
    sa[buf][0] = S.scales.lanes4(lane, (uint32_t)cb.ks << 8);
    sa[buf][1] = S.scales.lanes4(lane, S.s1 + ((uint32_t)cb.ks << 8));
  };
  auto advance_b = [&]() __attribute__((always_inline)) {
    if (__builtin_expect(++cb.ks == KS, 0)) {
      cb.ks = 0;
      cb.t += per_xcd;
      locate(cb);
      B = panel_of(cb);
      S = tokens_of(cb);
      if (STAGED) load_vectors();
    }
  };
  auto put = [&](int st) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 2; ++i) lds[st * STAGE + (wave + 4 * i) * 64 + lane] = next[i];
  };
  load_a(); advance_a(); put(0);
  load_a(); advance_a(); put(1);
  load_a();
  for (int j = 0; j < 4; ++j) load_b(0, j);
  load_scales(0);
  if (STAGED) load_vectors();
  start();
  __syncthreads();
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) fa[i] = lds[i * 64 + lane];
  // One step: the features of the next step are fetched, the tokens of two steps on go to LDS (into the stage that the step before read)
  // and those of three steps on are fetched, one or two instructions of this at a time between the matrix instructions, which leave twelve
  // cycles each for others to issue.  Each tile's operand is read three tiles ahead, across the barrier as well: what is read before it
  // belongs to the next step and was written before the last barrier.
  int s0 = 0, s1 = 1, s2 = 2;
  // STAGED, results under way: the next tile of 16 tokens to store, where it goes, and the bytes from there on that the buffer has
  int out_next = PT, out_bytes = 0;
  const int row_bytes = p.N * 2;
  const char* out_at = static_cast<const char*>(p.out);
  uint32_t out_lane = 0;      // offset of a lane's 16 bytes; beyond the buffer where its features are
  const int out_lds = wave * 64 + ((lane & 56) | ((lane & 7) ^ (lane >> 3)));
  u32x4 out[2];
  auto out_read = [&]() __attribute__((always_inline)) {
    const int at0 = (out_next == 0 ? s2 : 2 + min(out_next, PT - 1)) * STAGE + out_lds;
    out[0] = lds[at0];
    out[1] = lds[at0 + STAGE / 2];
  };
  auto out_store = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const auto d = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(out_at + h * 8 * (size_t)row_bytes), 0, max(out_bytes - h * 8 * row_bytes, 0), 0x00027000);
      __builtin_amdgcn_raw_buffer_store_b128(out[h], d, (int)out_lane, 0, 2);      // (2: non-temporal)
    }
    ++out_next;
    out_at += 16 * (size_t)row_bytes;
    out_bytes = max(out_bytes - 16 * row_bytes, 0);
  };
  auto step = [&](auto i2) __attribute__((always_inline)) {
    constexpr int b = decltype(i2)::value;
    // (The branches of a step come before its matrix instructions: the compiler moved them into the block behind a branch, past the barrier.)
    advance_a();
    advance_b();
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < PT; ++i) {
      const int r = i + AHEAD;
      if (i == 0) load_scales(b ^ 1);
      if (i < 4) load_b(b ^ 1, i);
      if (i == PT - AHEAD - 1) put(s2);      // (at least AHEAD reads come behind it)
      if (i == 5) load_a();
      if (STAGED && i == 0) out_read();
      if (STAGED && i == PT - 1) out_store();
      fa[r & 3] = lds[(r < PT ? s0 : s1) * STAGE + (r & (PT - 1)) * 64 + lane];
      mfma4(i, fb[b], fa[i & 3], sa[b][i >> 2], acc[i]);
      __builtin_amdgcn_sched_barrier(0);
    }
    // Not __syncthreads(), which waits for the reads under way as well: all but the last AHEAD of this wavefront's LDS accesses, its
    // writes among them, are done here (they complete in order).
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F | AHEAD << 8);      // lgkmcnt(AHEAD)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    const int s = s0;
    s0 = s1; s1 = s2; s2 = s;
    if (__builtin_expect(++at.ks < KS, 1)) return true;
    if constexpr (STAGED) {
      while (out_next < PT) { out_read(); out_store(); }
      f32x4 theta[4];
      if (THETA) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int k = 0; k < 4; ++k) theta[j][k] = spread(theta_now, j, k);
      }
      const int t = lane & 7, q = lane >> 4, token0 = at.tm * PT * 16, f0 = at.panel * 64;
#pragma unroll
      for (int i = 0; i < PT; ++i) {
        const int base = (i == 0 ? s2 : 2 + i) * STAGE + ((lane >> 3) & 1) * (STAGE / 2) + wave * 64 + t * 8;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float v[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) v[k] = !THETA || acc[i][j][k] > theta[j][k] ? acc[i][j][k] : 0.f;
          reinterpret_cast<u32x2*>(lds + base + ((2 * j + (q >> 1)) ^ t))[q & 1] = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
        }
      }
      out_next = 0;
      out_at = static_cast<const char*>(p.out) + (((size_t)at.l * p.M + token0) * p.N + f0) * 2;
      out_bytes = min(p.M - token0, PT * 16) * row_bytes;
      out_lane = (lane & 7) * 8 < p.N - f0 ? (uint32_t)((lane >> 3) * row_bytes + (lane & 7) * 16) : 0x80000000u;
    } else finish<T, THETA>(p, at.l, at.tm * PT * 16, at.panel, lane, acc);
    at.ks = 0;
    at.t += per_xcd;
    locate(at);
    if (at.ok) start();
    return at.ok;
  };
  while (step(I<0>()) && step(I<1>())) {}
  if (STAGED)
    while (out_next < PT) { out_read(); out_store(); }
}

// Few tokens: bound by the bytes of B.  One workgroup takes one panel of 64 features by MT tiles of 16 tokens; its four wavefronts take
// every fourth step of the contraction, straight from memory, two steps in flight, and add up in LDS in a fixed order.  One token, 16 layers of 8192
// features by 2048 (143 MB): 22.8 us, 6.3 TB/s.
template <typename T, bool THETA, int MT>
__global__ __launch_bounds__(256) void mx4_product_few_kernel(ProductArgs p) {
  __shared__ f32x4 part[3][MT * 4][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int KS = p.KS, panels_m = (p.M + 63) >> 6, panels_n = (p.N + 63) >> 6, panel = blockIdx.x, token0 = blockIdx.y * MT * 16, l = blockIdx.z;
  const Panel B(p.b, (size_t)l * panels_n + panel, KS);
  const Source ac(p.a.codes + (((size_t)l * panels_m * 4 + (token0 >> 4)) * KS << 10)), as(p.a.scales + (((size_t)l * panels_m + (token0 >> 6)) * KS << 8));
  f32x4 acc[MT][4];
  begin(p, l, panel, lane, acc);
  if (wave > 0) {
#pragma unroll
    for (int i = 0; i < MT * 4; ++i) acc[i >> 2][i & 3] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  PanelFrag fb[2];
  u32x4 fa[2][MT];
  uint32_t sa[2];
  auto fetch = [&](int ks, int buf) {
#pragma unroll
    for (int j = 0; j < 4; ++j) fb[buf].c[j] = B.tile(j, ks, lane);
    fb[buf].s = B.scale(ks, lane);
#pragma unroll
    for (int i = 0; i < MT; ++i) fa[buf][i] = ac.lanes16(lane, (uint32_t)(i * KS + ks) << 10);
    sa[buf] = as.lanes4(lane, (uint32_t)ks << 8);
  };
  auto compute = [&](int buf) {
    const uint32_t s = sa[buf] >> (8 * ((token0 >> 4) & 3));      // (MT = 2: token0 is a multiple of 32)
#pragma unroll
    for (int i = 0; i < MT; ++i) mfma4(i, fb[buf], fa[buf][i], s, acc[i]);
  };
  if (wave < KS) fetch(wave, 0);
  for (int ks = wave; ks < KS; ks += 8) {
    if (ks + 4 < KS) fetch(ks + 4, 1);
    compute(0);
    if (ks + 4 < KS) {
      if (ks + 8 < KS) fetch(ks + 8, 0);
      compute(1);
    }
  }
  if (wave > 0) {
#pragma unroll
    for (int i = 0; i < MT * 4; ++i) part[wave - 1][i][lane] = acc[i >> 2][i & 3];
  }
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int i = 0; i < MT * 4; ++i) {
    const f32x4 x = part[0][i][lane], y = part[1][i][lane], z = part[2][i][lane];
    acc[i >> 2][i & 3] = (acc[i >> 2][i & 3] + x) + (y + z);
  }
  finish<T, THETA>(p, l, token0, panel, lane, acc);
}

template <typename T, bool THETA>
hipError_t launch_product(hipStream_t s, int L, const ProductArgs& p) {
  const int panels_n = (p.N + 63) / 64, tiles_m = (p.M + PT * 16 - 1) / (PT * 16), tiles_n = (panels_n + 3) / 4;
  // The kernel for few tokens: up to 32 of them, and where tiles are too few for the chip.  us with it and with the other one (L, M, N, K):
  // 16, 1, 8192, 2048 22.0 / 22.4; 1, 64, 8192, 2048 (32 tiles) 4.9 / 11.2; 1, 300, 2048, 8192 (24) 11.1 / 32.7; 4, 128, 6144, 768 (96) 6.5 / 8.3;
  // 1, 512, 8192, 2048 (128) 12.2 / 13.0; 1, 768, 8192, 2048 (192) 17.2 / 13.6; 8, 128, 8192, 2048 (256) 22.3 / 14.9; 12, 64, 6144, 768 (288) 8.7 / 10.2;
  // 16, 48, 8192, 2048 (512) 25.5 / 24.5.  (The rule counts tiles, not how full they are: at 33 to 64 tokens of few steps, as in the last but one, the
  // kernel that is taken is the slower one.)  Two tiles of tokens instead of one at 17 to 32 tokens: 12 layers of 6144, K = 768 6.2 and 6.6.
  if (p.M <= 16) {
    hipLaunchKernelGGL((mx4_product_few_kernel<T, THETA, 1>), dim3(panels_n, 1, L), dim3(256), 0, s, p);
    return hipGetLastError();
  }
  if (p.M <= 32 || (double)L * tiles_m * tiles_n < 160.0) {
    hipLaunchKernelGGL((mx4_product_few_kernel<T, THETA, 2>), dim3(panels_n, (p.M + 31) / 32, L), dim3(256), 0, s, p);
    return hipGetLastError();
  }
  const TileOrder order(L, tiles_m, tiles_n);
  const uint32_t grid = order.tiles >= WORKGROUPS ? WORKGROUPS : (order.tiles + 7) / 8 * 8;
  // Results through LDS where workgroups have four tiles and more, so that there is a next tile to store under, of up to 20 steps: beyond the
  // eight that store something the others still read LDS in vain.  us staged / directly (L, M, N, K): 16, 4096, 8192, 128 201 / 224; the same, 512 239 / 258,
  // 1024 363 / 384, 2048 610 / 617; 12, 4096, 6144, 768 176 / 195; the same, 2560 421 / 427; 16, 2048, 4096, 4096 295 / 289;
  // 1, 16384, 2048, 256 (two tiles each) 20.2 / 19.3; 1, 4096, 2048, 768 (one) 11.7 / 9.7.
  if constexpr (sizeof(T) == 2) {
    if (order.tiles >= 4 * WORKGROUPS && p.KS <= 20) {
      hipLaunchKernelGGL((mx4_product_kernel<T, THETA, true>), dim3(grid), dim3(256), 0, s, p, order);
      return hipGetLastError();
    }
  }
  hipLaunchKernelGGL((mx4_product_kernel<T, THETA, false>), dim3(grid), dim3(256), 0, s, p, order);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_mx4_quantise(hipStream_t s, bool bf16, bool int8, bool transposed, int L, int rows, int K, const void* a,
                               const float* a_scale, uint8_t* codes, uint8_t* scales) {
  const int KS = mx4_steps(K), chunks = (KS + QUANTISE_STEPS - 1) / QUANTISE_STEPS;
  const dim3 grid(mx4_panels(rows) * chunks, L), wg(256);
  const dim3 columns((rows * (bf16 ? 1 : 2) + 127) / 128, KS, L);
  if (int8) hipLaunchKernelGGL(mx4_quantise_kernel<int8_t>, grid, wg, 0, s, rows, K, KS, chunks, (const int8_t*)a, a_scale, codes, scales);
  else if (bf16 && transposed) hipLaunchKernelGGL(mx4_quantise_transposed_kernel<bf16_t>, columns, wg, 0, s, rows, K, KS, (const bf16_t*)a, codes, scales);
  else if (bf16) hipLaunchKernelGGL(mx4_quantise_kernel<bf16_t>, grid, wg, 0, s, rows, K, KS, chunks, (const bf16_t*)a, a_scale, codes, scales);
  else if (transposed) hipLaunchKernelGGL(mx4_quantise_transposed_kernel<float>, columns, wg, 0, s, rows, K, KS, (const float*)a, codes, scales);
  else hipLaunchKernelGGL(mx4_quantise_kernel<float>, grid, wg, 0, s, rows, K, KS, chunks, (const float*)a, a_scale, codes, scales);
  return hipGetLastError();
}

hipError_t launch_mx4_dequantise(hipStream_t s, bool bf16, int L, int rows, int K, Mx4 a, void* out) {
  const int KS = mx4_steps(K), chunks = (KS + QUANTISE_STEPS - 1) / QUANTISE_STEPS;
  const dim3 grid(mx4_panels(rows) * chunks, L), wg(256);
  if (bf16) hipLaunchKernelGGL(mx4_dequantise_kernel<bf16_t>, grid, wg, 0, s, rows, K, KS, chunks, a, (bf16_t*)out);
  else hipLaunchKernelGGL(mx4_dequantise_kernel<float>, grid, wg, 0, s, rows, K, KS, chunks, a, (float*)out);
  return hipGetLastError();
}

hipError_t launch_mx4_product(hipStream_t s, bool bf16, int L, int M, int N, int K, Mx4 a, Mx4 b, const float* bias, const float* theta,
                              void* out) {
  const ProductArgs p{M, N, mx4_steps(K), a, b, bias, theta, out};
  if (bf16) return theta ? launch_product<bf16_t, true>(s, L, p) : launch_product<bf16_t, false>(s, L, p);
  return theta ? launch_product<float, true>(s, L, p) : launch_product<float, false>(s, L, p);
}

}  // namespace clt
