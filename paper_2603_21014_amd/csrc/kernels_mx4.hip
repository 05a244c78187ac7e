// 4-bit microscaled floating point: packing, unpacking, and the product on the scaled matrix instruction of gfx950
// (clt_mx4_quantise, clt_mx4_dequantise, clt_mx4_product; the packed layout is described in include/clt.h).
#include "common.h"

namespace clt {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
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
  const float scale = __uint_as_float((small ? s + 64u : s) << 23);
  float y[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) y[j] = small ? x[j] * 0x1p64f : x[j];
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[0], y[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[2], y[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[4], y[5], scale, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[6], y[7], scale, 3);
  return s == 255u ? 0u : w;
}

template <int CTRL> __device__ __forceinline__ uint32_t dpp_move(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, true);
}
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  v = max(v, dpp_move<0xB1>(v));          // quad_perm [1,0,3,2]
  return max(v, dpp_move<0x4E>(v));       // quad_perm [2,3,0,1]
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
// QUANTISE_STEPS steps.
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
  uint8_t* tile = codes + (((size_t)(l * panels + panel) * 4 + sub) * KS << 10) + lane * 4;
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
    uint32_t mine = 0;
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
      *reinterpret_cast<uint32_t*>(tile + ((size_t)(ks0 + t) << 10) + kb * 256) = to_codes(x, e);
      mine = part == kb ? e : mine;
    }
    sc[(size_t)(ks0 + t) << 8] = (uint8_t)mine;
  }
}

// Columns along the contraction (a is [K][rows]).  A lane takes one dword of columns (two of bf16, one of fp32) and the 32 elements of
// one block of each, so that a wavefront's loads are 256 consecutive bytes; the wavefronts of a workgroup take the four blocks of a step.
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

__device__ __forceinline__ float from_code(uint32_t c) {      // E2M1
  const uint32_t m = c & 7u;
  const float v = m < 2u ? 0.5f * m : __uint_as_float((126u + (m >> 1)) << 23 | (m & 1u) << 22);
  return c & 8u ? -v : v;
}

template <typename T>
__global__ __launch_bounds__(256) void mx4_dequantise_kernel(int rows, int K, int KS, Mx4 a, T* __restrict__ out) {
  const int l = blockIdx.y, nb = (K + 7) / 8;
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;      // eight elements
  const int r = (int)(i / nb), k = (int)(i % nb) * 8;
  if (r >= rows) return;
  const int panels = (rows + 63) >> 6, kb = k >> 5;
  const uint32_t w = *reinterpret_cast<const uint32_t*>(a.codes + (((size_t)l * panels * 4 * KS) << 10) + code_offset(r, kb, KS) + ((k & 31) >> 1));
  const uint32_t s = a.scales[(((size_t)l * panels * KS) << 8) + scale_offset(r, kb, KS)];
  float v[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = s == 255u ? __uint_as_float(0x7fc00000u) : __builtin_amdgcn_ldexpf(from_code(w >> (4 * j)), (int)s - 127);
  T* o = out + ((size_t)l * rows + r) * K + k;
  Elem<T>::store4(o, make_float4(v[0], v[1], v[2], v[3]));
  Elem<T>::store4(o + 4, make_float4(v[4], v[5], v[6], v[7]));
}

// ---- product -------------------------------------------------------------------------------------------------------
//
// v_mfma_scale_f32_16x16x128: a lane's operand is the 32 elements (16 bytes) of one block, row lane % 16, block lane / 16,
// with the block's scale in one byte of a register that the instruction selects: what a packed tile of 16 rows holds at byte
// 16 * lane.  The rows of B (features) are the instruction's first operand, those of A (tokens) its second, so a lane's
// four results are four features of one token.  The sixteen rows that make up the j-th of a panel's four operands are free;
// with rows 16 a + 4 j + b (a, b = 0..3) at lane 4 a + b, a lane ends up with sixteen consecutive features of its token:
// 32 bytes of bf16 to store, and the four lanes of a token a whole 128-byte line.  The price are four byte loads of scales for a
// panel's step instead of one dword.

// B operands of one panel (64 rows) and step
struct PanelFrag { u32x4 c[4]; uint32_t s[4]; };
struct PanelPtr {
  const uint8_t* codes; const uint8_t* scales;
  __device__ __forceinline__ PanelPtr(Mx4 b, size_t panel, int KS, int lane) {
    const int kb = lane >> 4, a = (lane >> 2) & 3, r = lane & 3;
    codes = b.codes + (((panel * 4 + a) * KS) << 10) + ((kb * 16 + r) << 4);
    scales = b.scales + ((panel * KS) << 8) + ((kb * 16 + r) << 2) + a;
  }
  __device__ __forceinline__ void load(PanelFrag& f, int ks) const {
    const uint8_t *c = codes + ((size_t)ks << 10), *s = scales + ((size_t)ks << 8);
#pragma unroll
    for (int j = 0; j < 4; ++j) f.c[j] = *reinterpret_cast<const u32x4*>(c + 64 * j);
#pragma unroll
    for (int j = 0; j < 4; ++j) f.s[j] = s[16 * j];
  }
};

template <int OP> __device__ __forceinline__ f32x4 mfma(u32x4 b, uint32_t bs, u32x4 a, uint32_t as, f32x4 c) {
  const i32x8 A = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0}, B = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(B, A, c, 4, 4, 0, (int)bs, OP, (int)as);
}
// tile i of a 64-row panel of A has its scales in byte i
__device__ __forceinline__ f32x4 mfma(int i, u32x4 b, uint32_t bs, u32x4 a, uint32_t as, f32x4 c) {
  switch (i & 3) {
    case 0: return mfma<0>(b, bs, a, as, c);
    case 1: return mfma<1>(b, bs, a, as, c);
    case 2: return mfma<2>(b, bs, a, as, c);
    default: return mfma<3>(b, bs, a, as, c);
  }
}

// Sixteen consecutive features, n of them (0, 8 or 16, or less than 0) inside the matrix
__device__ __forceinline__ void store_features(bf16_t* o, const float (&v)[16], int n) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const u32x4 w = {pack_bf16x2(v[8 * h], v[8 * h + 1]), pack_bf16x2(v[8 * h + 2], v[8 * h + 3]), pack_bf16x2(v[8 * h + 4], v[8 * h + 5]),
                     pack_bf16x2(v[8 * h + 6], v[8 * h + 7])};
    if (n >= 8 * (h + 1)) *reinterpret_cast<u32x4*>(o + 8 * h) = w;
  }
}
__device__ __forceinline__ void store_features(float* o, const float (&v)[16], int n) {
#pragma unroll
  for (int h = 0; h < 4; ++h)
    if (n >= 4 * (h + 1)) *reinterpret_cast<float4*>(o + 4 * h) = make_float4(v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]);
}
__device__ __forceinline__ void load_features(const float* p, float (&v)[16], int n, float none) {
#pragma unroll
  for (int h = 0; h < 4; ++h) {
    float4 x = make_float4(none, none, none, none);
    if (p && n >= 4 * (h + 1)) x = *reinterpret_cast<const float4*>(p + 4 * h);
    v[4 * h] = x.x; v[4 * h + 1] = x.y; v[4 * h + 2] = x.z; v[4 * h + 3] = x.w;
  }
}

struct ProductArgs { int M, N, KS; Mx4 a, b; const float* bias; const float* theta; void* out; };

// Bias, threshold, rounding and the stores of MT tiles of 16 tokens by one panel of features
template <typename T, int MT>
__device__ __forceinline__ void finish(const ProductArgs& p, int l, int token0, int panel, int lane, const f32x4 (&acc)[MT][4]) {
  const int n0 = panel * 64 + (lane >> 4) * 16, n = p.N - n0;
  if (n <= 0) return;
  float bias[16], theta[16];
  load_features(p.bias ? p.bias + (size_t)l * p.N + n0 : nullptr, bias, n, 0.f);
  load_features(p.theta ? p.theta + (size_t)l * p.N + n0 : nullptr, theta, n, 0.f);
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int m = token0 + i * 16 + (lane & 15);
    if (m >= p.M) continue;
    float v[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      v[j] = acc[i][j >> 2][j & 3] + bias[j];
      if (p.theta && !(v[j] > theta[j])) v[j] = 0.f;
    }
    store_features(static_cast<T*>(p.out) + ((size_t)l * p.M + m) * p.N + n0, v, n);
  }
}

// Many tokens: one workgroup takes 128 tokens by 256 features, each of its four wavefronts one panel of 64 features by all the
// tokens (8 x 4 accumulators of 16 x 16).  A panel is read by one wavefront only and goes from memory into its registers; the tokens
// are staged in LDS in two stages of one step each.  Two workgroups share a compute unit, so that one's prologue and epilogue
// run under the other's matrix instructions.
constexpr int PT = 8;      // tiles of 16 tokens
template <typename T>
__global__ __launch_bounds__(256, 2) void mx4_product_kernel(ProductArgs p, int tiles_m, int tiles_n) {
  __shared__ u32x4 stage[2][PT * 64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int KS = p.KS, panels_m = (p.M + 63) >> 6, panels_n = (p.N + 63) >> 6;
  // Workgroups are dealt to the eight XCDs in turn: each XCD takes a run of consecutive tiles, which go through the features for
  // eight tiles of tokens at a time, so that the tiles at work on an XCD share their operands in its L2.
  const uint32_t n = gridDim.x, x = blockIdx.x & 7, t = x * (n >> 3) + min(x, n & 7) + (blockIdx.x >> 3), per_layer = (uint32_t)tiles_m * tiles_n;
  const int l = t / per_layer, r = t - l * per_layer, group = r / (8 * tiles_n), rows = min(8, tiles_m - group * 8), in_group = r - group * 8 * tiles_n;
  const int tm = group * 8 + in_group % rows, tn = in_group / rows;
  const int panel = tn * 4 + wave;
  // (tiles and panels beyond the matrix: the last one again; what it gives is not stored)
  const PanelPtr B(p.b, (size_t)l * panels_n + min(panel, panels_n - 1), KS, lane);
  const uint8_t* ac[2];
  const uint32_t* as[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    ac[i] = p.a.codes + (((size_t)l * panels_m * 4 + min(tm * PT + wave + 4 * i, panels_m * 4 - 1)) * KS << 10) + lane * 16;
    as[i] = reinterpret_cast<const uint32_t*>(p.a.scales + (((size_t)l * panels_m + min(tm * 2 + i, panels_m - 1)) * KS << 8)) + lane;
  }
  f32x4 acc[PT][4];
#pragma unroll
  for (int i = 0; i < PT; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  u32x4 next[2];
  PanelFrag fb[2];
  uint32_t sa[2][2];
  auto fetch_a = [&](int ks) {
#pragma unroll
    for (int i = 0; i < 2; ++i) next[i] = *reinterpret_cast<const u32x4*>(ac[i] + ((size_t)ks << 10));
  };
  auto fetch_b = [&](int ks, int buf) {
    B.load(fb[buf], ks);
#pragma unroll
    for (int i = 0; i < 2; ++i) sa[buf][i] = as[i][ks << 6];
  };
  auto put = [&](int buf) {
#pragma unroll
    for (int i = 0; i < 2; ++i) stage[buf][(wave + 4 * i) * 64 + lane] = next[i];
  };
  fetch_a(0);
  fetch_b(0, 0);
  put(0);
  if (KS > 1) fetch_a(1);
  __syncthreads();
  auto step = [&](int ks, int buf) {
    if (ks + 1 < KS) {
      put(buf ^ 1);
      fetch_b(ks + 1, buf ^ 1);
      if (ks + 2 < KS) fetch_a(ks + 2);
    }
#pragma unroll
    for (int i = 0; i < PT; ++i) {
      const u32x4 a = stage[buf][i * 64 + lane];
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = mfma(i, fb[buf].c[j], fb[buf].s[j], a, sa[buf][i >> 2], acc[i][j]);
    }
    __syncthreads();
  };
  int ks = 0;
  for (; ks + 2 <= KS; ks += 2) { step(ks, 0); step(ks + 1, 1); }
  if (ks < KS) step(ks, 0);
  finish<T, PT>(p, l, tm * PT * 16, panel, lane, acc);
}

// Few tokens: bound by the bytes of B.  One workgroup takes one panel of 64 features by MT tiles of 16 tokens; its four wavefronts take
// every fourth step of the contraction, straight from memory, two steps in flight, and add up in LDS in a fixed order.
template <typename T, int MT>
__global__ __launch_bounds__(256) void mx4_product_few_kernel(ProductArgs p) {
  __shared__ f32x4 part[3][MT * 4][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int KS = p.KS, panels_m = (p.M + 63) >> 6, panels_n = (p.N + 63) >> 6, panel = blockIdx.x, token0 = blockIdx.y * MT * 16, l = blockIdx.z;
  const PanelPtr B(p.b, (size_t)l * panels_n + panel, KS, lane);
  const uint8_t* ac = p.a.codes + (((size_t)l * panels_m * 4 + (token0 >> 4)) * KS << 10) + lane * 16;
  const uint32_t* as = reinterpret_cast<const uint32_t*>(p.a.scales + (((size_t)l * panels_m + (token0 >> 6)) * KS << 8)) + lane;
  f32x4 acc[MT][4];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  PanelFrag fb[2];
  u32x4 fa[2][MT];
  uint32_t sa[2];
  auto fetch = [&](int ks, int buf) {
    B.load(fb[buf], ks);
#pragma unroll
    for (int i = 0; i < MT; ++i) fa[buf][i] = *reinterpret_cast<const u32x4*>(ac + (((size_t)i * KS + ks) << 10));
    sa[buf] = as[ks << 6];
  };
  auto compute = [&](int buf) {
    const uint32_t s = MT == 4 ? sa[buf] : sa[buf] >> (8 * ((token0 >> 4) & 3));
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = mfma(i, fb[buf].c[j], fb[buf].s[j], fa[buf][i], s, acc[i][j]);
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
  finish<T, MT>(p, l, token0, panel, lane, acc);
}

template <typename T>
hipError_t launch_product(hipStream_t s, int L, const ProductArgs& p) {
  const int panels_n = (p.N + 63) / 64;
  if (p.M <= 64) {
    const dim3 wg(256);
    if (p.M <= 16) hipLaunchKernelGGL((mx4_product_few_kernel<T, 1>), dim3(panels_n, 1, L), wg, 0, s, p);
    else if (p.M <= 32) hipLaunchKernelGGL((mx4_product_few_kernel<T, 2>), dim3(panels_n, 1, L), wg, 0, s, p);
    else hipLaunchKernelGGL((mx4_product_few_kernel<T, 4>), dim3(panels_n, 1, L), wg, 0, s, p);
    return hipGetLastError();
  }
  const int tiles_m = (p.M + PT * 16 - 1) / (PT * 16), tiles_n = (panels_n + 3) / 4;
  hipLaunchKernelGGL(mx4_product_kernel<T>, dim3((uint32_t)((size_t)L * tiles_m * tiles_n)), dim3(256), 0, s, p, tiles_m, tiles_n);
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
  const dim3 grid((uint32_t)(((size_t)rows * ((K + 7) / 8) + 255) / 256), L), wg(256);
  if (bf16) hipLaunchKernelGGL(mx4_dequantise_kernel<bf16_t>, grid, wg, 0, s, rows, K, mx4_steps(K), a, (bf16_t*)out);
  else hipLaunchKernelGGL(mx4_dequantise_kernel<float>, grid, wg, 0, s, rows, K, mx4_steps(K), a, (float*)out);
  return hipGetLastError();
}

hipError_t launch_mx4_product(hipStream_t s, bool bf16, int L, int M, int N, int K, Mx4 a, Mx4 b, const float* bias, const float* theta,
                              void* out) {
  const ProductArgs p{M, N, mx4_steps(K), a, b, bias, theta, out};
  return bf16 ? launch_product<bf16_t>(s, L, p) : launch_product<float>(s, L, p);
}

}  // namespace clt
