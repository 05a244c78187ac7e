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

// 32 floats -> 16 bytes.  The conversion instruction rounds to nearest even and saturates; its scale is a float, 2^(s-127), which
// for s = 0 is the denormal 2^-127: such blocks are multiplied by 2^64 first and converted with 2^(s-127+64).
__device__ __forceinline__ u32x4 to_codes(const float (&x)[32], uint32_t s) {
  u32x4 c = {0u, 0u, 0u, 0u};
  if (s == 255u) return c;
  const bool small = s < 64u;
  const float scale = __uint_as_float((small ? s + 64u : s) << 23);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float y[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = small ? x[8 * i + j] * 0x1p64f : x[8 * i + j];
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[0], y[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[2], y[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[4], y[5], scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[6], y[7], scale, 3);
    c[i] = w;
  }
  return c;
}

template <typename TE> __device__ __forceinline__ float value(TE x);
template <> __device__ __forceinline__ float value<float>(float x) { return x; }
template <> __device__ __forceinline__ float value<bf16_t>(bf16_t x) { return bf16_to_f32(x); }
template <> __device__ __forceinline__ float value<int8_t>(int8_t x) { return (float)x; }

// One lane per block of 32 elements.  TRANSPOSED: a is [K][rows].
template <typename TE, bool TRANSPOSED>
__global__ __launch_bounds__(256) void mx4_quantise_kernel(int rows, int K, int KS, const TE* __restrict__ a, const float* __restrict__ a_scale,
                                                           uint8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
  const int l = blockIdx.z;
  const int i = blockIdx.x * 256 + threadIdx.x;
  const int r = TRANSPOSED ? i : i / (KS * 4), kb = TRANSPOSED ? blockIdx.y : i % (KS * 4);
  if (r >= rows) return;
  a += (size_t)l * rows * K;
  float x[32];
  uint32_t top = 0;
  const float s = a_scale ? a_scale[(size_t)l * rows + r] : 1.f;
#pragma unroll
  for (int j = 0; j < 32; ++j) {
    const int k = kb * 32 + j;
    x[j] = k < K ? value<TE>(a[TRANSPOSED ? (size_t)k * rows + r : (size_t)r * K + k]) * s : 0.f;
    top = max(top, __float_as_uint(x[j]) & 0x7fffffffu);
  }
  const uint32_t e = block_scale(top);
  const int panels = (rows + 63) >> 6;
  *reinterpret_cast<u32x4*>(codes + (((size_t)l * panels * 4 * KS) << 10) + code_offset(r, kb, KS)) = to_codes(x, e);
  scales[(((size_t)l * panels * KS) << 8) + scale_offset(r, kb, KS)] = (uint8_t)e;
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

// One wavefront per 16 x 16 outputs, operands straight from memory.  The product is formed with B as the instruction's
// first operand, so that a lane holds four consecutive columns of one row.
template <typename T>
__global__ __launch_bounds__(64) void mx4_product_kernel(int M, int N, int KS, Mx4 a, Mx4 b, const float* __restrict__ bias,
                                                         const float* __restrict__ theta, T* __restrict__ out) {
  const int lane = threadIdx.x, l = blockIdx.z, tm = blockIdx.y, tn = blockIdx.x;
  const int pm = (M + 63) >> 6, pn = (N + 63) >> 6;
  const uint8_t* ac = a.codes + (((size_t)(l * pm * 4 + tm) * KS) << 10) + lane * 16;
  const uint8_t* bc = b.codes + (((size_t)(l * pn * 4 + tn) * KS) << 10) + lane * 16;
  const uint8_t* as = a.scales + (((size_t)(l * pm + (tm >> 2)) * KS) << 8) + lane * 4 + (tm & 3);
  const uint8_t* bs = b.scales + (((size_t)(l * pn + (tn >> 2)) * KS) << 8) + lane * 4 + (tn & 3);
  f32x4 c = {0.f, 0.f, 0.f, 0.f};
  for (int k = 0; k < KS; ++k) {
    const u32x4 x = *reinterpret_cast<const u32x4*>(ac + ((size_t)k << 10)), y = *reinterpret_cast<const u32x4*>(bc + ((size_t)k << 10));
    const i32x8 A = {(int)x[0], (int)x[1], (int)x[2], (int)x[3], 0, 0, 0, 0}, B = {(int)y[0], (int)y[1], (int)y[2], (int)y[3], 0, 0, 0, 0};
    c = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(B, A, c, 4, 4, 0, (int)bs[(size_t)k << 8], 0, (int)as[(size_t)k << 8]);
  }
  const int m = tm * 16 + (lane & 15), n = tn * 16 + (lane >> 4) * 4;
  if (m >= M || n >= N) return;      // N is a multiple of 8
  float v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = c[i] + (bias ? bias[(size_t)l * N + n + i] : 0.f);
    if (theta && !(v[i] > theta[(size_t)l * N + n + i])) v[i] = 0.f;
  }
  Elem<T>::store4(out + ((size_t)l * M + m) * N + n, make_float4(v[0], v[1], v[2], v[3]));
}

}  // namespace

hipError_t launch_mx4_quantise(hipStream_t s, bool bf16, bool int8, bool transposed, int L, int rows, int K, const void* a,
                               const float* a_scale, uint8_t* codes, uint8_t* scales) {
  const int KS = mx4_steps(K);
  const dim3 grid(transposed ? (rows + 255) / 256 : (uint32_t)(((size_t)rows * KS * 4 + 255) / 256), transposed ? KS * 4 : 1, L), wg(256);
  if (int8) hipLaunchKernelGGL((mx4_quantise_kernel<int8_t, false>), grid, wg, 0, s, rows, K, KS, (const int8_t*)a, a_scale, codes, scales);
  else if (bf16 && transposed) hipLaunchKernelGGL((mx4_quantise_kernel<bf16_t, true>), grid, wg, 0, s, rows, K, KS, (const bf16_t*)a, a_scale, codes, scales);
  else if (bf16) hipLaunchKernelGGL((mx4_quantise_kernel<bf16_t, false>), grid, wg, 0, s, rows, K, KS, (const bf16_t*)a, a_scale, codes, scales);
  else if (transposed) hipLaunchKernelGGL((mx4_quantise_kernel<float, true>), grid, wg, 0, s, rows, K, KS, (const float*)a, a_scale, codes, scales);
  else hipLaunchKernelGGL((mx4_quantise_kernel<float, false>), grid, wg, 0, s, rows, K, KS, (const float*)a, a_scale, codes, scales);
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
  const dim3 grid((N + 15) / 16, (M + 15) / 16, L);
  if (bf16) hipLaunchKernelGGL(mx4_product_kernel<bf16_t>, grid, dim3(64), 0, s, M, N, mx4_steps(K), a, b, bias, theta, (bf16_t*)out);
  else hipLaunchKernelGGL(mx4_product_kernel<float>, grid, dim3(64), 0, s, M, N, mx4_steps(K), a, b, bias, theta, (float*)out);
  return hipGetLastError();
}

}  // namespace clt
