// AdamW over a list of tensors in one launch, moments in fp32 or in 8 bits (clt_adamw_step).
//
// Sixteen lanes with eight elements each hold one block of 128 moments.  The block's power of two comes from the largest
// magnitude (four maxima across the sixteen lanes).  Both 8-bit formats are images of a float cut short: scaled by
// ldexp so that the format's smallest exponent is the smallest exponent of an fp32 number, the top bits of the fp32
// image ARE the 8-bit float, denormals included, and adding random bits below the cut before cutting rounds without bias.
//
// m' and v' are formed by single multiplications and additions (no fused ones): every rounding of the state is then
// one that any IEEE arithmetic repeats, and the codes can be compared bit for bit.
//
// Bound by memory: 10.03 bytes an element with bf16 weights and 8-bit moments, 22 with 32-bit ones.  The 8-bit form is not far from
// the vector units' limit either (38 instructions an element; the two multiplications of the random
// bits, the root and the reciprocal take four cycles each): with moments
// unpacked and packed by shifts and selects (52) it was bound by them.  Measured: 738 M elements with 8-bit moments 1178 us, 6.3 TB/s
// (1349 with 52 instructions and plain accesses); 425 M with 32-bit moments 1640 us, 5.7 TB/s (1754 with plain accesses).
#include "../../include/clt.h"
#include "common.h"

namespace clt {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Mixes 32 bits: two rounds of xor-shift and multiplication by an odd constant (digits of the golden ratio and of pi).
__host__ __device__ __forceinline__ uint32_t mix32(uint32_t x) {
  x ^= x >> 16;
  x *= 0x9E3779B1u;
  x ^= x >> 15;
  x *= 0x85A308D3u;
  return x ^ (x >> 16);
}

__device__ __forceinline__ uint32_t row16_max(uint32_t v) {      // as row16_sum
  v = max(v, dpp_move<0xB1>(v));
  v = max(v, dpp_move<0x4E>(v));
  v = max(v, dpp_move<0x141>(v));
  return max(v, dpp_move<0x140>(v));
}

// 8-bit floats of MANT mantissa bits whose exponent has bias BIAS and whose largest finite value is 1.75 * 2^TOP
// (E4M3: 3, 7, 8; E5M2: 2, 15, 15).
template <int MANT, int BIAS, int TOP> struct Float8 {
  static constexpr int CUT = 23 - MANT;
  // scale byte of a block whose largest magnitude has this fp32 image: 2^(s-127) brings the largest into (0.875, 1.75] * 2^TOP,
  // so no rounding up leaves the format; 255 where the image is an infinity or a NaN
  static __device__ __forceinline__ uint32_t scale(uint32_t top) {
    const int e = (int)((top + 0x1FFFFFu) >> 23);
    return top >= 0x7f800000u || e >= 255 ? 255u : (uint32_t)max(e - TOP, 0);
  }
  // fp32 image of x / 2^(s-127), its exponent field and mantissa moved down so that the code is what is left of bit CUT, with random bits
  // (16 of them) added below: the code of the neighbour below, or above with the probability of the distance from below.  The sign stays at the
  // top.  (Of a block with s = 255 the codes mean nothing.)
  static __device__ __forceinline__ uint32_t image(float x, uint32_t s, uint32_t random) {
    return __float_as_uint(__builtin_amdgcn_ldexpf(x, BIAS - (int)s)) + (random << (CUT - 16)) + (1u << (CUT - 17));
  }
};
typedef Float8<3, 7, 8> E4M3;
typedef Float8<2, 15, 15> E5M2;
// the top bytes of four words
__device__ __forceinline__ uint32_t top_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  const uint32_t lo = __builtin_amdgcn_perm(b, a, 0x0c0c0703u), hi = __builtin_amdgcn_perm(d, c, 0x07030c0cu);
  return lo | hi;
}
// four codes -> values
__device__ __forceinline__ void decode_m(uint32_t c, float f, float* x) {
  const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
  x[0] = a[0] * f; x[1] = a[1] * f; x[2] = b[0] * f; x[3] = b[1] * f;
}
__device__ __forceinline__ void decode_v(uint32_t c, float f, float* x) {
  const auto a = __builtin_amdgcn_cvt_pk_f32_bf8((int)c, false), b = __builtin_amdgcn_cvt_pk_f32_bf8((int)c, true);
  x[0] = a[0] * f; x[1] = a[1] * f; x[2] = b[0] * f; x[3] = b[1] * f;
}

// Eight elements of a lane from or to memory.  ROW: consecutive ones (a block of 8-bit moments is sixteen such lanes); else two runs of four
// elements, HALF apart, which are 16 bytes of fp32 each and neighbours of the next lane's.  WHOLE: all eight are inside the tensor; else
// those before `left` are.
constexpr int HALF = ADAMW_CHUNK / 2;
template <bool ROW> __device__ __forceinline__ constexpr int place(int i) { return ROW || i < 4 ? i : HALF + i - 4; }
__device__ __forceinline__ void widen4(u32x4 r, float* f) {
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void widen2(uint32_t r, float* f) { f[0] = __uint_as_float(r << 16); f[1] = __uint_as_float(r & 0xffff0000u); }
template <bool ROW, bool WHOLE, bool STREAM> __device__ __forceinline__ void load8(const float* p, int64_t left, float (&f)[8]) {
  if (!WHOLE) {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = place<ROW>(i) < left ? p[place<ROW>(i)] : 0.f;
    return;
  }
  widen4(take<STREAM, u32x4>(p), f);
  widen4(take<STREAM, u32x4>(p + place<ROW>(4)), f + 4);
}
template <bool ROW, bool WHOLE, bool STREAM> __device__ __forceinline__ void load8(const bf16_t* p, int64_t left, float (&f)[8]) {
  if (!WHOLE) {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = place<ROW>(i) < left ? bf16_to_f32(p[place<ROW>(i)]) : 0.f;
  } else if (ROW) {
    const u32x4 r = take<STREAM, u32x4>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) widen2(r[i], f + 2 * i);
  } else {
    const u32x2 a = take<STREAM, u32x2>(p), b = take<STREAM, u32x2>(p + HALF);
    widen2(a[0], f); widen2(a[1], f + 2); widen2(b[0], f + 4); widen2(b[1], f + 6);
  }
}
template <bool ROW, bool WHOLE, bool STREAM> __device__ __forceinline__ void store8(float* p, int64_t left, const float (&f)[8]) {
  if (!WHOLE) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (place<ROW>(i) < left) p[place<ROW>(i)] = f[i];
    return;
  }
  const f32x4 a = {f[0], f[1], f[2], f[3]}, b = {f[4], f[5], f[6], f[7]};
  give<STREAM>(p, a);
  give<STREAM>(p + place<ROW>(4), b);
}
template <bool ROW, bool WHOLE, bool STREAM> __device__ __forceinline__ void store8(bf16_t* p, int64_t left, const float (&f)[8]) {
  if (!WHOLE) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (place<ROW>(i) < left) p[place<ROW>(i)] = f32_to_bf16(f[i]);
    return;
  }
  const u32x4 r = {pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])};
  if (ROW) give<STREAM>(p, r);
  else {
    give<STREAM>(p, u32x2{r[0], r[1]});
    give<STREAM>(p + HALF, u32x2{r[2], r[3]});
  }
}
template <bool WHOLE, bool STREAM> __device__ __forceinline__ u32x2 load_bytes(const uint8_t* p, int64_t left) {
  if (WHOLE) return take<STREAM, u32x2>(p);
  u32x2 w = {0u, 0u};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < left) w[i >> 2] |= (uint32_t)p[i] << (8 * (i & 3));
  return w;
}
template <bool WHOLE, bool STREAM> __device__ __forceinline__ void store_bytes(uint8_t* p, int64_t left, u32x2 w) {
  if (WHOLE) { give<STREAM>(p, w); return; }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < left) p[i] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
}

__device__ __forceinline__ void update_moments(float& m, float& v, float g, const AdamScalars& a) {
#pragma clang fp contract(off)
  const float m0 = a.b1 * m, m1 = a.omb1 * g, v0 = a.b2 * v, v1 = (a.omb2 * g) * g;
  m = m0 + m1;
  v = v0 + v1;
}

template <bool ROW, bool WHOLE, bool STREAM> __device__ __forceinline__ void load_gp(const AdamWTensor& t, int64_t i0, float (&g)[8], float (&p)[8]) {
  const int64_t left = t.n - i0;
  if (t.grad_bf16) load8<ROW, WHOLE, STREAM>(static_cast<const bf16_t*>(t.g) + i0, left, g);
  else load8<ROW, WHOLE, STREAM>(static_cast<const float*>(t.g) + i0, left, g);
  if (t.master) load8<ROW, WHOLE, STREAM>(t.master + i0, left, p);
  else if (t.bf16) load8<ROW, WHOLE, STREAM>(static_cast<const bf16_t*>(t.p) + i0, left, p);
  else load8<ROW, WHOLE, STREAM>(static_cast<const float*>(t.p) + i0, left, p);
}
template <bool ROW, bool WHOLE, bool STREAM> __device__ __forceinline__ void store_p(const AdamWTensor& t, int64_t i0, const float (&p)[8]) {
  const int64_t left = t.n - i0;
  if (t.master) store8<ROW, WHOLE, STREAM>(t.master + i0, left, p);
  if (t.bf16) store8<ROW, WHOLE, STREAM>(static_cast<bf16_t*>(t.p) + i0, left, p);
  else store8<ROW, WHOLE, STREAM>(static_cast<float*>(t.p) + i0, left, p);
}
// The square root's unit takes denormal numbers for zeros.  Beside an eps of 2^-39 and more the root of one, below 2^-63, is less than
// the sum's rounding; beside a smaller eps (SMALL) it decides the step, and small arguments are scaled by 2^64.
constexpr float SMALL_EPS = 0x1p-39f;
template <bool SMALL> __device__ __forceinline__ float root(float x) {
  if (!SMALL) return __builtin_amdgcn_sqrtf(x);
  const bool low = x < 0x1p-96f;
  return __builtin_amdgcn_sqrtf(low ? x * 0x1p64f : x) * (low ? 0x1p-32f : 1.f);
}
template <bool SMALL> __device__ __forceinline__ void update(float (&p)[8], float (&m)[8], float (&v)[8], const float (&g)[8], float keep, const AdamScalars& a) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    update_moments(m[i], v[i], g[i], a);
    // (square root and reciprocal: one unit each, as in adam_element)
    const float den = root<SMALL>(v[i] * a.inv_bc2) + a.eps;
    p[i] = fmaf(a.neg_lr_over_bc1 * m[i], __builtin_amdgcn_rcpf(den), p[i] * keep);
  }
}

template <bool WHOLE, bool STREAM, bool SMALL> __device__ __forceinline__ void chunk32(const AdamWTensor& t, int64_t base, const AdamScalars& a) {
  const int64_t i0 = base + threadIdx.x * 4, left = t.n - i0;
  float g[8], p[8], m[8], v[8];
  load_gp<false, WHOLE, STREAM>(t, i0, g, p);
  load8<false, WHOLE, STREAM>(static_cast<const float*>(t.m) + i0, left, m);
  load8<false, WHOLE, STREAM>(static_cast<const float*>(t.v) + i0, left, v);
  update<SMALL>(p, m, v, g, t.keep, a);
  store8<false, WHOLE, STREAM>(static_cast<float*>(t.m) + i0, left, m);
  store8<false, WHOLE, STREAM>(static_cast<float*>(t.v) + i0, left, v);
  store_p<false, WHOLE, STREAM>(t, i0, p);
}

template <bool WHOLE, bool STREAM, bool SMALL> __device__ __forceinline__ void chunk8(const AdamWTensor& t, int64_t base, const AdamScalars& a) {
  const int64_t i0 = base + threadIdx.x * 8, left = t.n - i0;
  const int64_t block = (WHOLE || left > 0 ? i0 : base) / CLT_ADAMW_BLOCK;      // (lanes behind the end: any block; they hold zeros)
  float g[8], p[8], m[8], v[8];
  load_gp<true, WHOLE, STREAM>(t, i0, g, p);
  uint32_t ms = t.m_scale[block], vs = t.v_scale[block];
  if (!WHOLE && left <= 0) ms = vs = 0u;
  const u32x2 mc = load_bytes<WHOLE, STREAM>(static_cast<const uint8_t*>(t.m) + i0, left), vc = load_bytes<WHOLE, STREAM>(static_cast<const uint8_t*>(t.v) + i0, left);
  const float mf = scale_value(ms), vf = scale_value(vs);
  decode_m(mc[0], mf, m); decode_m(mc[1], mf, m + 4);
  decode_v(vc[0], vf, v); decode_v(vc[1], vf, v + 4);
  update<SMALL>(p, m, v, g, t.keep, a);
  uint32_t mtop = 0, vtop = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    mtop = max(mtop, __float_as_uint(m[i]) & 0x7fffffffu);
    vtop = max(vtop, __float_as_uint(v[i]));      // (never negative; a NaN's image is above an infinity's with either sign)
  }
  ms = E4M3::scale(row16_max(mtop));
  vs = E5M2::scale(row16_max(vtop));
  uint32_t mi[8], vi[8];
  const uint32_t key = t.key + (uint32_t)((uint64_t)i0 >> 32) * 0x85A308D3u;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t r = mix32(((uint32_t)i0 + i) ^ key);
    const uint32_t x = E4M3::image(m[i], ms, r & 0xffffu);      // sign, four zeros, the code's seven bits
    mi[i] = (x & 0x80000000u) | (x << 4 & 0x7fffffffu);
    const uint32_t y = E5M2::image(v[i], vs, r >> 16);          // three zeros, the code's seven bits, its sign zero
    vi[i] = max(y, v[i] > 0.f ? 1u << E5M2::CUT : 0u) << 3;
  }
  const u32x2 mw = {top_bytes(mi[0], mi[1], mi[2], mi[3]), top_bytes(mi[4], mi[5], mi[6], mi[7])};
  const u32x2 vw = {top_bytes(vi[0], vi[1], vi[2], vi[3]), top_bytes(vi[4], vi[5], vi[6], vi[7])};
  store_bytes<WHOLE, STREAM>(static_cast<uint8_t*>(t.m) + i0, left, mw);
  store_bytes<WHOLE, STREAM>(static_cast<uint8_t*>(t.v) + i0, left, vw);
  if ((threadIdx.x & 15) == 0 && (WHOLE || left > 0)) { t.m_scale[block] = (uint8_t)ms; t.v_scale[block] = (uint8_t)vs; }
  store_p<true, WHOLE, STREAM>(t, i0, p);
}

// One workgroup per ADAMW_CHUNK elements of one tensor.
template <bool STREAM, bool SMALL>
__global__ __launch_bounds__(256) void adamw_kernel(AdamWList q) {
  int k = 0;
  while (k + 1 < q.count && q.t[k + 1].chunk0 <= blockIdx.x) ++k;
  const AdamWTensor& t = q.t[k];
  const int64_t base = (int64_t)(blockIdx.x - t.chunk0) * ADAMW_CHUNK;
  const bool whole = base + ADAMW_CHUNK <= t.n;
  if (t.state8) {
    if (whole) chunk8<true, STREAM, SMALL>(t, base, q.a);
    else chunk8<false, STREAM, SMALL>(t, base, q.a);
  } else {
    if (whole) chunk32<true, STREAM, SMALL>(t, base, q.a);
    else chunk32<false, STREAM, SMALL>(t, base, q.a);
  }
}

}  // namespace

uint32_t adamw_mix(uint32_t x) { return mix32(x); }

// Streaming accesses where the launch's tensors are more than the Infinity Cache (256 MB) holds.  Both sides, us a step with plain / streaming
// ones: bf16 weights, 32-bit moments, 400 M elements 1642 / 1552, 10 M (120 MB) 32.5 / 35.7; fp32, 200 M 1053 / 977, 2 M 7.3 / 9.4.
hipError_t launch_adamw(hipStream_t s, const AdamWList& q) {
  double bytes = 0.0;
  for (int i = 0; i < q.count; ++i) {
    const AdamWTensor& t = q.t[i];
    bytes += (double)t.n * ((t.bf16 ? 2 : 4) + (t.grad_bf16 ? 2 : 4) + (t.state8 ? 2 : 8) + (t.master ? 4 : 0));
  }
  const bool stream = bytes > 256e6, small = q.a.eps < SMALL_EPS;
  if (stream && small) hipLaunchKernelGGL((adamw_kernel<true, true>), dim3(q.chunks), dim3(256), 0, s, q);
  else if (stream) hipLaunchKernelGGL((adamw_kernel<true, false>), dim3(q.chunks), dim3(256), 0, s, q);
  else if (small) hipLaunchKernelGGL((adamw_kernel<false, true>), dim3(q.chunks), dim3(256), 0, s, q);
  else hipLaunchKernelGGL((adamw_kernel<false, false>), dim3(q.chunks), dim3(256), 0, s, q);
  return hipGetLastError();
}

}  // namespace clt
