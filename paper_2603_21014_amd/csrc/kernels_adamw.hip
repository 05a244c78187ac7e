// AdamW over a list of tensors in one launch, moments in fp32 or in 8 bits (clt_adamw_step).
//
// Sixteen lanes with eight elements each hold one block of 128 moments.  The block's power of two comes from the largest
// magnitude (four maxima across the sixteen lanes), and both 8-bit formats are images of a float cut short: scaled by
// ldexp so that the format's smallest exponent is the smallest exponent of an fp32 number, the top bits of the fp32
// image ARE the 8-bit float, denormals included, and adding random bits below the cut before cutting rounds without bias.
//
// m' and v' are formed by single multiplications and additions (no fused ones): every rounding of the state is then
// one that any IEEE arithmetic repeats, and the codes can be compared bit for bit.
#include "../../include/clt.h"
#include "common.h"

namespace clt {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

// Mixes 32 bits: two rounds of xor-shift and multiplication by an odd constant (digits of the golden ratio and of pi).
__host__ __device__ __forceinline__ uint32_t mix32(uint32_t x) {
  x ^= x >> 16;
  x *= 0x9E3779B1u;
  x ^= x >> 15;
  x *= 0x85A308D3u;
  return x ^ (x >> 16);
}

template <int CTRL> __device__ __forceinline__ uint32_t dpp_move(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, true);
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
  static __device__ __forceinline__ float decode(uint32_t code, uint32_t s) {      // magnitude
    const float x = __builtin_amdgcn_ldexpf(__uint_as_float(code << CUT), (int)s - BIAS);
    return s == 255u ? __uint_as_float(0x7fc00000u) : x;
  }
  // nearest below or above, above with the probability of the distance from below; random: 16 bits
  static __device__ __forceinline__ uint32_t encode(float x, uint32_t s, uint32_t random) {
    const uint32_t y = __float_as_uint(__builtin_amdgcn_ldexpf(x, BIAS - (int)s));
    return s == 255u ? 0u : (y + (random << (CUT - 16)) + (1u << (CUT - 17))) >> CUT;
  }
};
typedef Float8<3, 7, 8> E4M3;
typedef Float8<2, 15, 15> E5M2;

// eight consecutive elements from or to memory, `left` of them inside the tensor
template <typename T> __device__ __forceinline__ void load8(const T* p, int left, float (&f)[8]) {
  if (left >= 8) {
    const float4 a = Elem<T>::load4(p), b = Elem<T>::load4(p + 4);
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = i < left ? Elem<T>::load(p + i) : 0.f;
  }
}
template <typename T> __device__ __forceinline__ void store8(T* p, int left, const float (&f)[8]) {
  if (left >= 8) {
    Elem<T>::store4(p, make_float4(f[0], f[1], f[2], f[3]));
    Elem<T>::store4(p + 4, make_float4(f[4], f[5], f[6], f[7]));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < left) Elem<T>::store(p + i, f[i]);
  }
}
__device__ __forceinline__ uint2 load_bytes(const uint8_t* p, int left) {
  if (left >= 8) return *reinterpret_cast<const uint2*>(p);
  uint32_t w[2] = {0u, 0u};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < left) w[i >> 2] |= (uint32_t)p[i] << (8 * (i & 3));
  return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ void store_bytes(uint8_t* p, int left, const uint32_t (&w)[2]) {
  if (left >= 8) { *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]); return; }
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

__global__ __launch_bounds__(256) void adamw_kernel(AdamWList q) {
  int k = 0;
  while (k + 1 < q.count && q.t[k + 1].chunk0 <= blockIdx.x) ++k;
  const AdamWTensor& t = q.t[k];
  const int64_t i0 = (int64_t)(blockIdx.x - t.chunk0) * ADAMW_CHUNK + threadIdx.x * 8;
  const int left = (int)min((int64_t)8, t.n - i0);      // none: this lane only takes part in its block's maxima
  float g[8] = {}, p[8] = {}, m[8] = {}, v[8] = {};
  const int64_t block = i0 / CLT_ADAMW_BLOCK;
  uint2 mc = make_uint2(0u, 0u);
  if (left > 0) {
    if (t.grad_bf16) load8(static_cast<const bf16_t*>(t.g) + i0, left, g);
    else load8(static_cast<const float*>(t.g) + i0, left, g);
    if (t.master) load8(t.master + i0, left, p);
    else if (t.bf16) load8(static_cast<const bf16_t*>(t.p) + i0, left, p);
    else load8(static_cast<const float*>(t.p) + i0, left, p);
    if (t.state8) {
      const uint32_t ms = t.m_scale[block], vs = t.v_scale[block];
      mc = load_bytes(static_cast<const uint8_t*>(t.m) + i0, left);
      const uint2 vc = load_bytes(static_cast<const uint8_t*>(t.v) + i0, left);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t cm = (i < 4 ? mc.x : mc.y) >> (8 * (i & 3)) & 255u, cv = (i < 4 ? vc.x : vc.y) >> (8 * (i & 3)) & 255u;
        m[i] = E4M3::decode(cm & 127u, ms);
        if (cm & 128u) m[i] = -m[i];
        v[i] = E5M2::decode(cv, vs);
      }
    } else {
      load8(static_cast<const float*>(t.m) + i0, left, m);
      load8(static_cast<const float*>(t.v) + i0, left, v);
    }
  }
  uint32_t mtop = 0, vtop = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    update_moments(m[i], v[i], g[i], q.a);
    const float den = __builtin_amdgcn_sqrtf(v[i] * q.a.inv_bc2) + q.a.eps;
    p[i] = fmaf(q.a.neg_lr_over_bc1 * m[i], __builtin_amdgcn_rcpf(den), p[i] * t.keep);
    mtop = max(mtop, __float_as_uint(m[i]) & 0x7fffffffu);
    vtop = max(vtop, __float_as_uint(v[i]) & 0x7fffffffu);
  }
  if (t.state8) {
    const uint32_t ms = E4M3::scale(row16_max(mtop)), vs = E5M2::scale(row16_max(vtop));
    if (left > 0) {
      uint32_t mw[2] = {0u, 0u}, vw[2] = {0u, 0u};
      const uint32_t key = t.key + (uint32_t)((uint64_t)i0 >> 32) * 0x85A308D3u;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t r = mix32(((uint32_t)i0 + i) ^ key);
        mw[i >> 2] |= (E4M3::encode(fabsf(m[i]), ms, r & 0xffffu) | (m[i] < 0.f ? 128u : 0u)) << (8 * (i & 3));
        uint32_t c = E5M2::encode(v[i], vs, r >> 16);
        if (v[i] > 0.f && c == 0u && vs != 255u) c = 1u;
        vw[i >> 2] |= c << (8 * (i & 3));
      }
      store_bytes(static_cast<uint8_t*>(t.m) + i0, left, mw);
      store_bytes(static_cast<uint8_t*>(t.v) + i0, left, vw);
      if ((threadIdx.x & 15) == 0) { t.m_scale[block] = (uint8_t)ms; t.v_scale[block] = (uint8_t)vs; }
    }
  } else if (left > 0) {
    store8(static_cast<float*>(t.m) + i0, left, m);
    store8(static_cast<float*>(t.v) + i0, left, v);
  }
  if (left > 0) {
    if (t.master) store8(t.master + i0, left, p);
    if (t.bf16) store8(static_cast<bf16_t*>(t.p) + i0, left, p);
    else store8(static_cast<float*>(t.p) + i0, left, p);
  }
}

}  // namespace

uint32_t adamw_mix(uint32_t x) { return mix32(x); }

hipError_t launch_adamw(hipStream_t s, const AdamWList& q) {
  hipLaunchKernelGGL(adamw_kernel, dim3(q.chunks), dim3(256), 0, s, q);
  return hipGetLastError();
}

}  // namespace clt
