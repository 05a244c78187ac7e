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

// Rows whose largest |h w| is below this count as all-zero (1 / max must not overflow).
constexpr float ROW_IS_ZERO = 0x1p-100f;

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
template <typename T> struct Vec16 { static constexpr int N = 16 / sizeof(T); };      // elements in 16 bytes
__device__ __forceinline__ void widen16(u32x4 r, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(r[i] << 16); f[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u); }
}
__device__ __forceinline__ void widen16(u32x4 r, float (&f)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ u32x4 narrow16(const float (&f)[8]) {
  return u32x4{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])};
}
__device__ __forceinline__ u32x4 narrow16(const float (&f)[4]) {
  return u32x4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
}

// A row whose sum of squares, or whose products with the weights, are beyond fp32 is multiplied by the power of two that brings its largest |h|
// into [1/2, 1), which is exact, and normalised in that form, where no product is above its weight; only rstd gets the power back.  hmax: that |h|'s image.
__device__ __forceinline__ bool beyond(float sum, uint32_t top) { return !(sum < __uint_as_float(0x7f800000u)) || top >= 0x7f800000u; }
__device__ __forceinline__ float power_below(uint32_t hmax) {      // 1 where it would not help: an infinity, a NaN, a weight that is one
  return hmax < 0x3f800000u || hmax >= 0x7f800000u ? 1.f : __builtin_amdgcn_ldexpf(1.f, 126 - (int)(hmax >> 23));
}

// What the codes and the scale of a row follow from; sum and top are those of the row times `down`
struct RowScale { float norm, rstd, k, scale; bool broken; };
__device__ __forceinline__ RowScale row_scale(float sum, uint32_t top, float eps, int d, float down) {
  RowScale r;
  r.norm = 1.0f / sqrtf(sum / (float)d + eps * down * down);
  r.rstd = r.norm * down;
  const float amax = __uint_as_float(top);
  const bool zero = amax < fmaxf(ROW_IS_ZERO * down, 0x1p-118f);
  r.broken = top >= 0x7f800000u;
  r.k = r.broken || zero ? 0.f : 1.0f / amax * 127.0f;
  r.scale = r.broken ? __uint_as_float(0x7fc00000u) : zero ? 1.f : amax * r.norm / 127.0f;
  return r;
}
__device__ __forceinline__ uint32_t code(float t, const RowScale& r) { return (uint32_t)(int)(r.broken ? 0.f : rintf(t * r.k)) & 255u; }

// A row is held in registers by one wavefront (W = 1, four rows at a time in a workgroup) or by a workgroup (W = 4), NV pieces of 16
// bytes per lane, so that it is read once: the sum of squares and the largest |h weight| come from the same pass, and the codes
// 127 y / max|y| need no second one because rstd cancels in them.  The weights stay in registers over the rows of a wavefront (they are
// four bytes where a bf16 element is two).  Bound by memory: 16 layers of 4096 rows of 2048 in bf16, residual in, sum and codes out (940 MB): 168 us,
// 5.6 TB/s.  (Fetching a row ahead of the one at work: 16 layers of 4096 rows of 768 75 -> 69 us, of 256 rows of 2048 11.6 -> 13.2, else the same.)
template <typename T, int NV, int W, bool STREAM>
__global__ __launch_bounds__(256) void rms_norm_kernel(int B, int d, int rows_each, RmsNormArgs a) {
  constexpr int N = Vec16<T>::N;
  __shared__ float sums[4][4];
  __shared__ uint32_t tops[4][4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = blockIdx.y;
  const int b0 = (W == 1 ? blockIdx.x * 4 + wave : blockIdx.x) * rows_each, b1 = min(B, b0 + rows_each);
  int e[NV];      // first element of each piece
#pragma unroll
  for (int v = 0; v < NV; ++v) e[v] = ((W == 1 ? 0 : wave * NV * 64) + v * 64 + lane) * N;
  float w[NV][N];
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
      if (e[v] < d) x = *reinterpret_cast<const float4*>(a.weight + (size_t)l * d + e[v] + i);
      w[v][i] = x.x; w[v][i + 1] = x.y; w[v][i + 2] = x.z; w[v][i + 3] = x.w;
    }
  for (int b = b0; b < b1; ++b) {
    const size_t row = (size_t)l * B + b, o = row * d;
    const T *x = static_cast<const T*>(a.x) + o, *res = static_cast<const T*>(a.residual) + o;
    u32x4 raw[NV], add[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      raw[v] = add[v] = u32x4{0u, 0u, 0u, 0u};
      if (e[v] < d) {
        raw[v] = take<STREAM, u32x4>(x + e[v]);
        if (a.residual) add[v] = take<STREAM, u32x4>(res + e[v]);
      }
    }
    float t[NV][N], s = 0.f, down = 1.f;
    uint32_t top = 0;
    auto measure = [&](const float (&h)[N], int v) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        s = fmaf(h[i], h[i], s);
        t[v][i] = h[i] * w[v][i];
        top = max(top, __float_as_uint(t[v][i]) & 0x7fffffffu);
      }
    };
    auto join = [&](int buf) __attribute__((always_inline)) {
      s = wave_sum(s);
      top = wave_max(top);
      if (W == 4) {
        if (lane == 0) { sums[buf][wave] = s; tops[buf][wave] = top; }
        __syncthreads();
        s = (sums[buf][0] + sums[buf][1]) + (sums[buf][2] + sums[buf][3]);
        top = max(max(tops[buf][0], tops[buf][1]), max(tops[buf][2], tops[buf][3]));
      }
    };
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float h[N], r[N];
      widen16(raw[v], h);
      if (a.residual) {
        widen16(add[v], r);
#pragma unroll
        for (int i = 0; i < N; ++i) h[i] += r[i];
        raw[v] = narrow16(h);      // the norm is that of the stored sum, as a model that reads it again would have it
        widen16(raw[v], h);
        if (e[v] < d) give<STREAM>(static_cast<T*>(a.h) + o + e[v], raw[v]);
      }
      measure(h, v);
    }
    join(b & 1);      // (two buffers in turn: one barrier per row)
    if (__builtin_expect(beyond(s, top), 0)) {      // (the same for all lanes of the row; it is read again, so that nobody else has to keep it)
      const T* again = (a.residual ? static_cast<const T*>(a.h) : static_cast<const T*>(a.x)) + o;
      auto load = [&](float (&h)[N], int v) __attribute__((always_inline)) {
        widen16(e[v] < d ? *reinterpret_cast<const u32x4*>(again + e[v]) : u32x4{0u, 0u, 0u, 0u}, h);
#pragma unroll
        for (int i = 0; i < N; ++i) h[i] *= down;
      };
      s = 0.f;
      top = 0;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        float h[N];
        load(h, v);
#pragma unroll
        for (int i = 0; i < N; ++i) top = max(top, __float_as_uint(h[i]) & 0x7fffffffu);
      }
      join(2);
      down = power_below(top);
      top = 0;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        float h[N];
        load(h, v);
        measure(h, v);
      }
      join(3);
    }
    const RowScale r = row_scale(s, top, a.eps, d, down);
    if ((W == 1 ? lane : threadIdx.x) == 0) {
      if (a.rstd) a.rstd[row] = r.rstd;
      if (a.q) a.q_scale[row] = r.scale;
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      if (e[v] >= d) continue;
      if (a.y) {
        float y[N];
#pragma unroll
        for (int i = 0; i < N; ++i) y[i] = t[v][i] * r.norm;
        give<STREAM>(static_cast<T*>(a.y) + o + e[v], narrow16(y));
      }
      if (a.q) {
        uint32_t c[N / 4];
#pragma unroll
        for (int i = 0; i < N; i += 4) c[i / 4] = code(t[v][i], r) | code(t[v][i + 1], r) << 8 | code(t[v][i + 2], r) << 16 | code(t[v][i + 3], r) << 24;
        if (N == 8) give<STREAM>(a.q + o + e[v], u32x2{c[0], c[N / 4 - 1]});
        else give<STREAM>(a.q + o + e[v], c[0]);
      }
    }
  }
}

// Rows too wide for that: one workgroup per row, the row read twice.
template <typename T>
__global__ __launch_bounds__(256) void rms_norm_wide_kernel(int B, int d, RmsNormArgs a) {
  __shared__ float sums[2][4];
  __shared__ uint32_t tops[3][4];
  const size_t row = blockIdx.x, o = row * d;
  const float* w = a.weight + row / B * d;
  const T* x = static_cast<const T*>(a.x) + o;
  T* hs = static_cast<T*>(a.h);
  const T* h = a.residual ? hs + o : x;
  float s = 0.f, down = 1.f;
  uint32_t top = 0;
  auto add = [&](float4 v, int i) __attribute__((always_inline)) {
    const float4 w4 = *reinterpret_cast<const float4*>(w + i);
    s = fmaf(v.x, v.x, fmaf(v.y, v.y, fmaf(v.z, v.z, fmaf(v.w, v.w, s))));
    const uint32_t t0 = max(__float_as_uint(v.x * w4.x) & 0x7fffffffu, __float_as_uint(v.y * w4.y) & 0x7fffffffu);
    const uint32_t t1 = max(__float_as_uint(v.z * w4.z) & 0x7fffffffu, __float_as_uint(v.w * w4.w) & 0x7fffffffu);
    top = max(top, max(t0, t1));
  };
  auto largest = [&](int buf) __attribute__((always_inline)) {      // of all lanes' top
    top = wave_max(top);
    if ((threadIdx.x & 63) == 0) tops[buf][threadIdx.x >> 6] = top;
    __syncthreads();
    top = max(max(tops[buf][0], tops[buf][1]), max(tops[buf][2], tops[buf][3]));
  };
  auto join = [&](int buf) __attribute__((always_inline)) {
    s = wave_sum(s);
    if ((threadIdx.x & 63) == 0) sums[buf][threadIdx.x >> 6] = s;
    largest(buf);
    s = (sums[buf][0] + sums[buf][1]) + (sums[buf][2] + sums[buf][3]);
  };
  auto load = [&](int i) __attribute__((always_inline)) {
    float4 v = Elem<T>::load4(h + i);
    v.x *= down; v.y *= down; v.z *= down; v.w *= down;
    return v;
  };
  for (int i = threadIdx.x * 4; i < d; i += 1024) {
    float4 v = Elem<T>::load4(x + i);
    if (a.residual) {
      const float4 r = Elem<T>::load4(static_cast<const T*>(a.residual) + o + i);
      const typename Elem<T>::Raw4 raw = Elem<T>::narrow4(make_float4(v.x + r.x, v.y + r.y, v.z + r.z, v.w + r.w));
      *reinterpret_cast<typename Elem<T>::Raw4*>(hs + o + i) = raw;
      v = Elem<T>::widen4(raw);
    }
    add(v, i);
  }
  join(0);
  if (__builtin_expect(beyond(s, top), 0)) {      // (the same for the whole workgroup)
    top = 0;
    for (int i = threadIdx.x * 4; i < d; i += 1024) {
      const float4 v = load(i);
      const uint32_t t0 = max(__float_as_uint(v.x) & 0x7fffffffu, __float_as_uint(v.y) & 0x7fffffffu);
      top = max(top, max(t0, max(__float_as_uint(v.z) & 0x7fffffffu, __float_as_uint(v.w) & 0x7fffffffu)));
    }
    largest(2);
    down = power_below(top);
    s = 0.f;
    top = 0;
    for (int i = threadIdx.x * 4; i < d; i += 1024) add(load(i), i);
    join(1);
  }
  const RowScale r = row_scale(s, top, a.eps, d, down);
  if (threadIdx.x == 0) {
    if (a.rstd) a.rstd[row] = r.rstd;
    if (a.q) a.q_scale[row] = r.scale;
  }
  for (int i = threadIdx.x * 4; i < d; i += 1024) {
    const float4 h4 = load(i), w4 = *reinterpret_cast<const float4*>(w + i);
    const float t[4] = {h4.x * w4.x, h4.y * w4.y, h4.z * w4.z, h4.w * w4.w};
    if (a.y) Elem<T>::store4(static_cast<T*>(a.y) + o + i, make_float4(t[0] * r.norm, t[1] * r.norm, t[2] * r.norm, t[3] * r.norm));
    if (a.q) *reinterpret_cast<uint32_t*>(a.q + o + i) = code(t[0], r) | code(t[1], r) << 8 | code(t[2], r) << 16 | code(t[3], r) << 24;
  }
}

// ---- backward pass ---------------------------------------------------------------------------------------------------
//
// Rows of very large numbers: with a small rstd its cube leaves fp32 (from 2^-42 on), and so do products of h and dy.  From 2^-30 on h is
// multiplied by the power of two at or below rstd and rstd divided by it, both exact, so that the products are those of a row of ordinary
// size; the factor of the projection gets the power back at its end.
struct RowPower { float down, rn; };      // that power, rstd over it; 1 and rstd itself for ordinary rows
__device__ __forceinline__ RowPower row_power(float rstd) {
  if (!(rstd > 0.f && rstd < 0x1p-30f)) return {1.f, rstd};
  const uint32_t e = max(__float_as_uint(rstd) >> 23, 1u);
  return {__uint_as_float(e << 23), rstd * __uint_as_float((254u - e) << 23)};
}

// The same arrangement: h, dy (and dh) of a row are read once, for dx and for the row's share of dweight, which the lanes add up in
// registers over all rows of their wavefront.  A workgroup leaves one partial sum of dweight, a second kernel adds those in order.
// 16 layers of 4096 rows of 2048 in bf16 with dh (1.07 GB): 182 us, 5.9 TB/s; 300 rows of 2056: 4.5 us and 4.2 for the partial sums.
template <typename T, int NV, int W, bool STREAM>
__global__ __launch_bounds__(256) void rms_norm_backward_kernel(int B, int d, int rows_each, RmsNormBackwardArgs a) {
  constexpr int N = Vec16<T>::N;
  __shared__ float sums[2][4];
  __shared__ float part[W == 1 ? 3 : 1][NV * 64 * N];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = blockIdx.y;
  const int b0 = (W == 1 ? blockIdx.x * 4 + wave : blockIdx.x) * rows_each, b1 = min(B, b0 + rows_each);
  int e[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) e[v] = ((W == 1 ? 0 : wave * NV * 64) + v * 64 + lane) * N;
  float w[NV][N], dw[NV][N];
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
      if (e[v] < d) x = *reinterpret_cast<const float4*>(a.weight + (size_t)l * d + e[v] + i);
      w[v][i] = x.x; w[v][i + 1] = x.y; w[v][i + 2] = x.z; w[v][i + 3] = x.w;
      dw[v][i] = dw[v][i + 1] = dw[v][i + 2] = dw[v][i + 3] = 0.f;
    }
  for (int b = b0; b < b1; ++b) {
    const size_t row = (size_t)l * B + b, o = row * d;
    u32x4 rh[NV], rg[NV], re[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      rh[v] = rg[v] = re[v] = u32x4{0u, 0u, 0u, 0u};
      if (e[v] < d) {
        rh[v] = take<STREAM, u32x4>(static_cast<const T*>(a.h) + o + e[v]);
        rg[v] = take<STREAM, u32x4>(static_cast<const T*>(a.dy) + o + e[v]);
        if (a.dh) re[v] = take<STREAM, u32x4>(static_cast<const T*>(a.dh) + o + e[v]);
      }
    }
    const float r = __uint_as_float((uint32_t)__builtin_amdgcn_readfirstlane((int)__float_as_uint(a.rstd[row])));      // (one row to a wavefront)
    const RowPower p = row_power(r);
    if (__builtin_expect(p.down != 1.f, 0)) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        float h[N];
        widen16(rh[v], h);
#pragma unroll
        for (int i = 0; i < N; ++i) h[i] *= p.down;
        rh[v] = narrow16(h);
      }
    }
    float s = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float h[N], g[N];
      widen16(rh[v], h);
      widen16(rg[v], g);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float gh = g[i] * h[i];
        s = fmaf(w[v][i], gh, s);
        dw[v][i] = fmaf(gh, p.rn, dw[v][i]);
      }
    }
    s = wave_sum(s);
    if (W == 4) {
      const int buf = b & 1;
      if (lane == 0) sums[buf][wave] = s;
      __syncthreads();
      s = (sums[buf][0] + sums[buf][1]) + (sums[buf][2] + sums[buf][3]);
    }
    const float c = s / (float)d * p.rn * p.rn * p.rn * p.down;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float h[N], g[N], x[N];
      widen16(rh[v], h);
      widen16(rg[v], g);
      widen16(re[v], x);
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = fmaf(r, w[v][i] * g[i], fmaf(-c, h[i], x[i]));
      if (e[v] < d) give<STREAM>(static_cast<T*>(a.dx) + o + e[v], narrow16(x));
    }
  }
  if (!a.dweight) return;
  if (W == 1) {      // the four wavefronts' sums, in order
    if (wave > 0) {
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int i = 0; i < N; ++i) part[wave - 1][(v * N + i) * 64 + lane] = dw[v][i];
    }
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int k = (v * N + i) * 64 + lane;
        dw[v][i] = (dw[v][i] + part[0][k]) + (part[1][k] + part[2][k]);
      }
  }
  float* out = a.part + ((size_t)l * gridDim.x + blockIdx.x) * d;
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int i = 0; i < N; i += 4)
      if (e[v] < d) *reinterpret_cast<float4*>(out + e[v] + i) = make_float4(dw[v][i], dw[v][i + 1], dw[v][i + 2], dw[v][i + 3]);
}

// Rows too wide for that.  dx: one workgroup per row, the row read twice; dweight: sums over dw_rows(B) rows, a lane per column
template <typename T>
__global__ __launch_bounds__(256) void rms_norm_dx_kernel(int B, int d, RmsNormBackwardArgs a) {
  __shared__ float sums[4];
  const size_t row = blockIdx.x, o = row * d;
  const float* w = a.weight + row / B * d;
  const T *h = static_cast<const T*>(a.h) + o, *dy = static_cast<const T*>(a.dy) + o;
  const float r = a.rstd[row];
  const RowPower p = row_power(r);
  auto load_h = [&](int i) __attribute__((always_inline)) {
    const float4 v = Elem<T>::load4(h + i);
    return make_float4(v.x * p.down, v.y * p.down, v.z * p.down, v.w * p.down);
  };
  float s = 0.f;
  for (int i = threadIdx.x * 4; i < d; i += 1024) {
    const float4 h4 = load_h(i), g4 = Elem<T>::load4(dy + i), w4 = *reinterpret_cast<const float4*>(w + i);
    s += (h4.x * (w4.x * g4.x) + h4.y * (w4.y * g4.y)) + (h4.z * (w4.z * g4.z) + h4.w * (w4.w * g4.w));
  }
  s = wave_sum(s);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = s;
  __syncthreads();
  const float c = ((sums[0] + sums[1]) + (sums[2] + sums[3])) / (float)d * p.rn * p.rn * p.rn * p.down;
  for (int i = threadIdx.x * 4; i < d; i += 1024) {
    const float4 h4 = load_h(i), g4 = Elem<T>::load4(dy + i), w4 = *reinterpret_cast<const float4*>(w + i);
    float4 e = make_float4(0.f, 0.f, 0.f, 0.f);
    if (a.dh) e = Elem<T>::load4(static_cast<const T*>(a.dh) + o + i);
    Elem<T>::store4(static_cast<T*>(a.dx) + o + i,
                    make_float4(fmaf(r, w4.x * g4.x, fmaf(-c, h4.x, e.x)), fmaf(r, w4.y * g4.y, fmaf(-c, h4.y, e.y)),
                                fmaf(r, w4.z * g4.z, fmaf(-c, h4.z, e.z)), fmaf(r, w4.w * g4.w, fmaf(-c, h4.w, e.w))));
  }
}

inline int dw_rows(int B) { return B <= 1 << 20 ? 32 : (B + 32767) / 32768; }      // rows of a partial sum (a grid has 65535 blocks along its second axis)
inline int dw_blocks(int B) { return (B + dw_rows(B) - 1) / dw_rows(B); }

// grid = (columns / 256, row blocks, layers)
template <typename T>
__global__ __launch_bounds__(256) void rms_norm_dw_kernel(int B, int d, int rows, RmsNormBackwardArgs a) {
  const int c = blockIdx.x * 256 + threadIdx.x, l = blockIdx.z;
  if (c >= d) return;
  const int end = min(B, (int)(blockIdx.y + 1) * rows);
  float s = 0.f;
  for (int b = blockIdx.y * rows; b < end; ++b) {
    const size_t row = (size_t)l * B + b;
    const RowPower p = row_power(a.rstd[row]);
    s = fmaf(Elem<T>::load(static_cast<const T*>(a.dy) + row * d + c) * p.rn, Elem<T>::load(static_cast<const T*>(a.h) + row * d + c) * p.down, s);
  }
  a.part[((size_t)l * gridDim.y + blockIdx.y) * d + c] = s;
}
// The partial sums of 64 columns: sixteen wavefronts take every sixteenth each, eight loads in flight, and their sums are added in
// order.  (One lane for all 300 partial sums of a column: 10 us, most of the whole backward pass of 300 rows.)
constexpr int FINISH = 16;
__global__ __launch_bounds__(64 * FINISH) void rms_norm_dw_finish_kernel(int blocks, int d, const float* __restrict__ part, float* __restrict__ dweight) {
  __shared__ float sum[FINISH][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x * 64 + lane, l = blockIdx.y;
  float s[8] = {};
  if (c < d) {
    const float* p = part + (size_t)l * blocks * d + c;
    int b = wave;
    for (; b + 7 * FINISH < blocks; b += 8 * FINISH) {
#pragma unroll
      for (int i = 0; i < 8; ++i) s[i] += p[(size_t)(b + i * FINISH) * d];
    }
#pragma unroll
    for (int i = 0; i < 7; ++i)
      if (b + i * FINISH < blocks) s[i] += p[(size_t)(b + i * FINISH) * d];
  }
  sum[wave][lane] = ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7]));
  __syncthreads();
  if (wave > 0 || c >= d) return;
  float t = 0.f;
#pragma unroll
  for (int i = 0; i < FINISH; ++i) t += sum[i][lane];
  dweight[(size_t)l * d + c] = t;
}

// How rows are cut: NV pieces of 16 bytes per lane of one wavefront (W = 1) or of four.  A wavefront takes up to 2048 elements of bf16 or
// 1024 of fp32 (32 values and 32 weights in registers), a workgroup four times that; pieces 0: neither, the wide kernels.
// us forward / backward, bf16, by a wavefront, a workgroup and the wide kernels: 16 layers of 4096 rows of 2048 174 / 183, 177 / 205, 253 / 386; 12 of
// 1037 of 768 13.8 / 18.4, 25.5 / 24.0, 20.9 / 30.8; by a workgroup and the wide kernels: 4 of 4096 of 8192 181 / 216, 238 / 422; 64 rows of 8192 4.8 / 8.6, 7.8 / 13.0.
struct RowCut { int pieces, waves; };
inline RowCut row_cut(bool bf16, int d) {
  const int per = bf16 ? 512 : 256;      // elements of one piece of all lanes
  for (int w = 1; w <= 4; w *= 4)
    for (int nv = 1; nv <= 4; nv *= 2)
      if (d <= per * nv * w) return {nv, w};
  return {0, 0};
}
// Rows of a wavefront (or of a workgroup of four): enough wavefronts to fill the chip first, then rows that share the weights.
inline int rows_each(int L, int B, int waves, int most) {
  const int64_t n = ((int64_t)L * B * waves + 8191) / 8192;      // 8192 wavefronts: eight for every SIMD
  return (int)(n < 1 ? 1 : n > most ? most : n);
}

}  // namespace

#define ROW_KERNELS(KERNEL, T, STREAM)                                                                                              \
  do {                                                                                                                              \
    if (cut.waves == 1) {                                                                                                           \
      if (cut.pieces == 1) hipLaunchKernelGGL((KERNEL<T, 1, 1, STREAM>), grid, dim3(256), 0, s, B, d, each, a);                     \
      else if (cut.pieces == 2) hipLaunchKernelGGL((KERNEL<T, 2, 1, STREAM>), grid, dim3(256), 0, s, B, d, each, a);                \
      else hipLaunchKernelGGL((KERNEL<T, 4, 1, STREAM>), grid, dim3(256), 0, s, B, d, each, a);                                     \
    } else if (cut.pieces == 2) hipLaunchKernelGGL((KERNEL<T, 2, 4, STREAM>), grid, dim3(256), 0, s, B, d, each, a);                \
    else hipLaunchKernelGGL((KERNEL<T, 4, 4, STREAM>), grid, dim3(256), 0, s, B, d, each, a);                                       \
  } while (0)
#define ROW_KERNELS_T(KERNEL, bytes)                                                                                                \
  do {                                                                                                                              \
    if (bf16 && streams(bytes)) ROW_KERNELS(KERNEL, bf16_t, true);                                                                  \
    else if (bf16) ROW_KERNELS(KERNEL, bf16_t, false);                                                                              \
    else if (streams(bytes)) ROW_KERNELS(KERNEL, float, true);                                                                      \
    else ROW_KERNELS(KERNEL, float, false);                                                                                         \
  } while (0)
// Streaming accesses where a call touches more than the Infinity Cache (256 MB) holds.  us with them / without, forward and backward: 16 layers of 4096
// rows of 2048 in bf16 174 / 186, 183 / 206; 16 of 256 (59 and 67 MB) 11.5 / 11.7, 21.6 / 21.0; 12 of 1037 of 768 in fp32 (124 and 153 MB) 22.3 / 20.9, 31.8 / 28.8.
static bool streams(double bytes) { return bytes > 256e6; }

hipError_t launch_rms_norm(hipStream_t s, bool bf16, int L, int B, int d, const RmsNormArgs& a) {
  const RowCut cut = row_cut(bf16, d);
  if (!cut.pieces) {
    const dim3 grid((uint32_t)((size_t)L * B));
    if (bf16) hipLaunchKernelGGL(rms_norm_wide_kernel<bf16_t>, grid, dim3(256), 0, s, B, d, a);
    else hipLaunchKernelGGL(rms_norm_wide_kernel<float>, grid, dim3(256), 0, s, B, d, a);
    return hipGetLastError();
  }
  // (8 rows that share the weights; more of them where the grid, of 2^32 threads at most, would not hold a wavefront for every eight)
  const int each = rows_each(L, B, cut.waves, B <= 1 << 28 ? 8 : 32), per = each * (cut.waves == 1 ? 4 : 1);
  const dim3 grid((B + per - 1) / per, L);
  const double n = (double)L * B * d, e = bf16 ? 2 : 4;
  ROW_KERNELS_T(rms_norm_kernel, n * (e * (1 + (a.residual ? 2 : 0) + (a.y ? 1 : 0)) + (a.q ? 1 : 0)));
  return hipGetLastError();
}

// (the larger of both types' needs: the room is asked for without the type)
static int dw_parts(bool bf16, int L, int B, int d) {
  const RowCut cut = row_cut(bf16, d);
  if (!cut.pieces) return dw_blocks(B);
  const int per = rows_each(L, B, cut.waves, B) * (cut.waves == 1 ? 4 : 1);
  return (B + per - 1) / per;
}
size_t rms_norm_backward_floats(int L, int B, int d) {
  const int n = dw_parts(true, L, B, d), m = dw_parts(false, L, B, d);
  return (size_t)L * (n > m ? n : m) * d;
}

hipError_t launch_rms_norm_backward(hipStream_t s, bool bf16, int L, int B, int d, const RmsNormBackwardArgs& a) {
  const RowCut cut = row_cut(bf16, d);
  const int parts = dw_parts(bf16, L, B, d);
  if (cut.pieces) {
    const int each = rows_each(L, B, cut.waves, B);
    const dim3 grid(parts, L);
    ROW_KERNELS_T(rms_norm_backward_kernel, (double)L * B * d * (bf16 ? 2 : 4) * (a.dh ? 4 : 3));
  } else {
    const dim3 rows((uint32_t)((size_t)L * B)), cols((d + 255) / 256, parts, L);
    if (a.dweight) {      // before dx, which may overwrite dy
      if (bf16) hipLaunchKernelGGL(rms_norm_dw_kernel<bf16_t>, cols, dim3(256), 0, s, B, d, dw_rows(B), a);
      else hipLaunchKernelGGL(rms_norm_dw_kernel<float>, cols, dim3(256), 0, s, B, d, dw_rows(B), a);
    }
    if (bf16) hipLaunchKernelGGL(rms_norm_dx_kernel<bf16_t>, rows, dim3(256), 0, s, B, d, a);
    else hipLaunchKernelGGL(rms_norm_dx_kernel<float>, rows, dim3(256), 0, s, B, d, a);
  }
  if (a.dweight) hipLaunchKernelGGL(rms_norm_dw_finish_kernel, dim3((d + 63) / 64, L), dim3(64 * FINISH), 0, s, parts, d, a.part, a.dweight);
  return hipGetLastError();
}

}  // namespace clt
