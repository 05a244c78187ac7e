// Root-mean-square norm of residual streams with the residual's addition, as T or as int8 codes with a scale per row, and its
// backward pass (clt_rms_norm, clt_rms_norm_backward).
#include "common.h"

namespace clt {
namespace {

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
  return v;
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, off, 64));
  return v;
}

// Rows whose largest |h w| is below this count as all-zero (127 / max must not overflow).
constexpr float ROW_IS_ZERO = 0x1p-100f;

// One workgroup per row, the row read twice.
template <typename T>
__global__ __launch_bounds__(256) void rms_norm_kernel(int B, int d, RmsNormArgs a) {
  __shared__ float sums[4];
  __shared__ uint32_t tops[4];
  const size_t row = blockIdx.x, o = row * d;
  const float* w = a.weight + row / B * d;
  const T* x = static_cast<const T*>(a.x) + o;
  T* hs = static_cast<T*>(a.h);
  float s = 0.f;
  uint32_t top = 0;
  for (int i = threadIdx.x * 4; i < d; i += 1024) {
    float4 h = Elem<T>::load4(x + i);
    if (a.residual) {
      const float4 r = Elem<T>::load4(static_cast<const T*>(a.residual) + o + i);
      const typename Elem<T>::Raw4 raw = Elem<T>::narrow4(make_float4(h.x + r.x, h.y + r.y, h.z + r.z, h.w + r.w));
      *reinterpret_cast<typename Elem<T>::Raw4*>(hs + o + i) = raw;
      h = Elem<T>::widen4(raw);
    }
    const float4 w4 = *reinterpret_cast<const float4*>(w + i);
    s = fmaf(h.x, h.x, fmaf(h.y, h.y, fmaf(h.z, h.z, fmaf(h.w, h.w, s))));
    const uint32_t t0 = max(__float_as_uint(h.x * w4.x) & 0x7fffffffu, __float_as_uint(h.y * w4.y) & 0x7fffffffu);
    const uint32_t t1 = max(__float_as_uint(h.z * w4.z) & 0x7fffffffu, __float_as_uint(h.w * w4.w) & 0x7fffffffu);
    top = max(top, max(t0, t1));
  }
  s = wave_sum(s);
  top = wave_max(top);
  if ((threadIdx.x & 63) == 0) { sums[threadIdx.x >> 6] = s; tops[threadIdx.x >> 6] = top; }
  __syncthreads();
  s = (sums[0] + sums[1]) + (sums[2] + sums[3]);
  top = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
  const float rstd = 1.0f / sqrtf(s / (float)d + a.eps);
  const float amax = __uint_as_float(top);
  const bool broken = top >= 0x7f800000u, zero = amax < ROW_IS_ZERO;
  const float k = broken || zero ? 0.f : 127.0f / amax;
  if (threadIdx.x == 0) {
    if (a.rstd) a.rstd[row] = rstd;
    if (a.q) a.q_scale[row] = broken ? __uint_as_float(0x7fc00000u) : zero ? 1.f : amax * rstd / 127.0f;
  }
  const T* h = a.residual ? hs + o : x;
  for (int i = threadIdx.x * 4; i < d; i += 1024) {
    const float4 h4 = Elem<T>::load4(h + i), w4 = *reinterpret_cast<const float4*>(w + i);
    const float t[4] = {h4.x * w4.x, h4.y * w4.y, h4.z * w4.z, h4.w * w4.w};
    if (a.y) Elem<T>::store4(static_cast<T*>(a.y) + o + i, make_float4(t[0] * rstd, t[1] * rstd, t[2] * rstd, t[3] * rstd));
    if (a.q) {
      uint32_t c = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) c |= ((uint32_t)(int)(broken ? 0.f : rintf(t[j] * k)) & 255u) << (8 * j);
      *reinterpret_cast<uint32_t*>(a.q + o + i) = c;
    }
  }
}

// dx: one workgroup per row, the row read twice
template <typename T>
__global__ __launch_bounds__(256) void rms_norm_dx_kernel(int B, int d, RmsNormBackwardArgs a) {
  __shared__ float sums[4];
  const size_t row = blockIdx.x, o = row * d;
  const float* w = a.weight + row / B * d;
  const T *h = static_cast<const T*>(a.h) + o, *dy = static_cast<const T*>(a.dy) + o;
  const float r = a.rstd[row];
  float s = 0.f;
  for (int i = threadIdx.x * 4; i < d; i += 1024) {
    const float4 h4 = Elem<T>::load4(h + i), g4 = Elem<T>::load4(dy + i), w4 = *reinterpret_cast<const float4*>(w + i);
    s += (h4.x * (w4.x * g4.x) + h4.y * (w4.y * g4.y)) + (h4.z * (w4.z * g4.z) + h4.w * (w4.w * g4.w));
  }
  s = wave_sum(s);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = s;
  __syncthreads();
  const float c = ((sums[0] + sums[1]) + (sums[2] + sums[3])) / (float)d * r * r * r;
  for (int i = threadIdx.x * 4; i < d; i += 1024) {
    const float4 h4 = Elem<T>::load4(h + i), g4 = Elem<T>::load4(dy + i), w4 = *reinterpret_cast<const float4*>(w + i);
    float4 e = make_float4(0.f, 0.f, 0.f, 0.f);
    if (a.dh) e = Elem<T>::load4(static_cast<const T*>(a.dh) + o + i);
    Elem<T>::store4(static_cast<T*>(a.dx) + o + i,
                    make_float4(fmaf(r, w4.x * g4.x, fmaf(-c, h4.x, e.x)), fmaf(r, w4.y * g4.y, fmaf(-c, h4.y, e.y)),
                                fmaf(r, w4.z * g4.z, fmaf(-c, h4.z, e.z)), fmaf(r, w4.w * g4.w, fmaf(-c, h4.w, e.w))));
  }
}

constexpr int DW_ROWS = 32;      // rows of a partial sum
inline int dw_blocks(int B) { return (B + DW_ROWS - 1) / DW_ROWS; }

// dweight, first pass: sums over DW_ROWS rows; grid = (columns / 256, row blocks, layers)
template <typename T>
__global__ __launch_bounds__(256) void rms_norm_dw_kernel(int B, int d, RmsNormBackwardArgs a) {
  const int c = blockIdx.x * 256 + threadIdx.x, l = blockIdx.z;
  if (c >= d) return;
  const int end = min(B, (int)(blockIdx.y + 1) * DW_ROWS);
  float s = 0.f;
  for (int b = blockIdx.y * DW_ROWS; b < end; ++b) {
    const size_t row = (size_t)l * B + b;
    s = fmaf(Elem<T>::load(static_cast<const T*>(a.dy) + row * d + c) * a.rstd[row], Elem<T>::load(static_cast<const T*>(a.h) + row * d + c), s);
  }
  a.part[((size_t)l * gridDim.y + blockIdx.y) * d + c] = s;
}
__global__ __launch_bounds__(256) void rms_norm_dw_finish_kernel(int blocks, int d, const float* __restrict__ part, float* __restrict__ dweight) {
  const int c = blockIdx.x * 256 + threadIdx.x, l = blockIdx.y;
  if (c >= d) return;
  float s = 0.f;
  for (int b = 0; b < blocks; ++b) s += part[((size_t)l * blocks + b) * d + c];
  dweight[(size_t)l * d + c] = s;
}

}  // namespace

hipError_t launch_rms_norm(hipStream_t s, bool bf16, int L, int B, int d, const RmsNormArgs& a) {
  const dim3 grid((uint32_t)((size_t)L * B));
  if (bf16) hipLaunchKernelGGL(rms_norm_kernel<bf16_t>, grid, dim3(256), 0, s, B, d, a);
  else hipLaunchKernelGGL(rms_norm_kernel<float>, grid, dim3(256), 0, s, B, d, a);
  return hipGetLastError();
}

size_t rms_norm_backward_floats(int L, int B, int d) { return (size_t)L * dw_blocks(B) * d; }

hipError_t launch_rms_norm_backward(hipStream_t s, bool bf16, int L, int B, int d, const RmsNormBackwardArgs& a) {
  const dim3 rows((uint32_t)((size_t)L * B)), cols((d + 255) / 256, dw_blocks(B), L);
  if (a.dweight) {      // before dx, which may overwrite dy
    if (bf16) hipLaunchKernelGGL(rms_norm_dw_kernel<bf16_t>, cols, dim3(256), 0, s, B, d, a);
    else hipLaunchKernelGGL(rms_norm_dw_kernel<float>, cols, dim3(256), 0, s, B, d, a);
    hipLaunchKernelGGL(rms_norm_dw_finish_kernel, dim3((d + 255) / 256, L), dim3(256), 0, s, dw_blocks(B), d, a.part, a.dweight);
  }
  if (bf16) hipLaunchKernelGGL(rms_norm_dx_kernel<bf16_t>, rows, dim3(256), 0, s, B, d, a);
  else hipLaunchKernelGGL(rms_norm_dx_kernel<float>, rows, dim3(256), 0, s, B, d, a);
  return hipGetLastError();
}

}  // namespace clt
