// Eight-element vectors in registers: loads, stores and conversions shared by the bandwidth-bound kernels.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace osdp {

// A kernel that is launched over the end of the one before it may find written by that one whatever it reads after pdl_wait():
// inputs, scales, statistics, parameters that a step has just changed.  Such data is read with ordinary loads, never
// through the read-only path (whose data must not change while the kernel runs, and it runs before the wait).
__device__ __forceinline__ void pdl_launch_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// 32 bytes in one access (256-bit global accesses need a 32-byte aligned address).  The data of these kernels is
// streamed: nothing of it is kept in L1.
__device__ __forceinline__ void load32(const void *p, uint32_t (&w)[8]) {
  asm volatile("ld.global.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
               : "l"(p)
               : "memory");
}
__device__ __forceinline__ void store32(void *p, const uint32_t (&w)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
               : "memory");
}
__device__ __forceinline__ uint4 load16(const void *p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
  return v;
}

__device__ __forceinline__ void widen8(const uint4 &u, float (&f)[8]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    f[2 * j] = __uint_as_float(w[j] << 16);
    f[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ uint4 narrow8(const float (&f)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * j], f[2 * j + 1]);
    w[j] = *reinterpret_cast<const uint32_t *>(&h);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// Two fp32 values side by side: sm_100 multiplies and adds such pairs in one instruction, which is what lets the
// element-wise kernels keep up with the memory.
struct f2 {
  unsigned long long v;
};
__device__ __forceinline__ f2 pack2(float a, float b) {
  f2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 split2(f2 a) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(a.v));
  return r;
}
__device__ __forceinline__ f2 both(float a) { return pack2(a, a); }
__device__ __forceinline__ f2 mul2(f2 a, f2 b) {
  f2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ f2 add2(f2 a, f2 b) {
  f2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) {
  f2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}
__device__ __forceinline__ float sum2(f2 a) {
  const float2 s = split2(a);
  return s.x + s.y;
}
__device__ __forceinline__ void widen4(const uint4 &u, f2 (&f)[4]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) f[j] = pack2(__uint_as_float(w[j] << 16), __uint_as_float(w[j] & 0xFFFF0000u));
}
__device__ __forceinline__ uint4 narrow4(const f2 (&f)[4]) {
  uint32_t w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 v = split2(f[j]);
    const __nv_bfloat162 h = __floats2bfloat162_rn(v.x, v.y);
    w[j] = *reinterpret_cast<const uint32_t *>(&h);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// Eight fp32 values from two 16-byte pieces, and back to memory as T.
__device__ __forceinline__ void join4(const float4 &lo, const float4 &hi, f2 (&f)[4]) {
  f[0] = pack2(lo.x, lo.y);
  f[1] = pack2(lo.z, lo.w);
  f[2] = pack2(hi.x, hi.y);
  f[3] = pack2(hi.z, hi.w);
}
template <typename T>
__device__ __forceinline__ void store4(T *p, const f2 (&f)[4]) {
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<uint4 *>(p) = narrow4(f);
  } else {
    uint32_t w[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 v = split2(f[j]);
      w[2 * j] = __float_as_uint(v.x);
      w[2 * j + 1] = __float_as_uint(v.y);
    }
    store32(p, w);
  }
}

// Eight consecutive elements of type T (__nv_bfloat16: 16-byte aligned, float: 32-byte aligned) <-> fp32.
template <typename T>
__device__ __forceinline__ void load8(const T *p, float (&f)[8]) {
  if constexpr (sizeof(T) == 2) {
    widen8(load16(p), f);
  } else {
    uint32_t w[8];
    load32(p, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = __uint_as_float(w[j]);
  }
}
template <typename T>
__device__ __forceinline__ void store8(T *p, const float (&f)[8]) {
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<uint4 *>(p) = narrow8(f);
  } else {
    uint32_t w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = __float_as_uint(f[j]);
    store32(p, w);
  }
}
__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T>
__device__ __forceinline__ T from_f32(float v) {
  if constexpr (sizeof(T) == 2) return __float2bfloat16_rn(v);
  else return v;
}

// Eight e4m3 codes (8 bytes) <-> fp32.  Round to nearest, ties to even; beyond +-448 saturates; NaN stays NaN.
__device__ __forceinline__ void decode_e4m3x8(const uint2 &c, f2 (&f)[4]) {
  const uint32_t w[2] = {c.x, c.y};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[j >> 1] >> (16 * (j & 1))), __NV_E4M3);
    const float2 v = __half22float2(*reinterpret_cast<const __half2 *>(&h));
    f[j] = pack2(v.x, v.y);
  }
}
__device__ __forceinline__ uint2 encode_e4m3x8(const f2 (&f)[4]) {
  uint32_t w[2] = {0u, 0u};
#pragma unroll
  for (int j = 0; j < 4; ++j)
    w[j >> 1] |= (uint32_t)__nv_cvt_float2_to_fp8x2(split2(f[j]), __NV_SATFINITE, __NV_E4M3) << (16 * (j & 1));
  return make_uint2(w[0], w[1]);
}

// Largest of three magnitudes; a NaN wins.
__device__ __forceinline__ float max_abs3(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(fabsf(a)), "f"(fabsf(b)), "f"(fabsf(c)));
  return r;
}
// Smallest of `a` >= 0 and two magnitudes; a NaN loses.
__device__ __forceinline__ float min_abs3(float a, float b, float c) {
  float r;
  asm("min.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(fabsf(b)), "f"(fabsf(c)));
  return r;
}
// Square root and reciprocals of the special-function unit (relative error about 2^-22; denormals count as zero in the
// reciprocals).
__device__ __forceinline__ float fast_sqrt(float x) {
  float r;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float fast_rsqrt(float x) {
  float r;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float fast_rcp(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// int8 rows: scale = (largest magnitude) / 127; a row whose largest magnitude is below 2^-100 (its reciprocal could
// overflow) is stored as zeros with scale 0.  An infinity or a NaN goes into the scale.
__device__ __forceinline__ float int8_scale(float top) { return top < 7.888609052210118e-31f ? 0.f : __fdiv_rn(top, 127.0f); }
__device__ __forceinline__ float int8_inverse(float scale) { return scale == 0.f ? 0.f : __frcp_rn(scale); }
// Eight values / scale, rounded to the nearest integers (ties to even), as int8; zeros if the scale is not finite.
// `inv` = int8_inverse(scale).  Adding 1.5 * 2^23 rounds to an integer and leaves it in the last byte (a conversion runs at a
// quarter of the rate).  value * inv is within 127 * 2^-23 + 2^-24 of the quotient, so that it decides unless it is that close to
// the middle of two integers; those, one in some thousand vectors, are divided.
__device__ __forceinline__ uint2 to_int8x8(const float (&f)[8], float scale, float inv) {
  constexpr float round = 12582912.0f;
  const f2 inv2 = both(inv), up = both(round), down = both(-round), minus = both(-1.0f);
  uint32_t q[8];
  float furthest = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const f2 t = mul2(pack2(f[2 * j], f[2 * j + 1]), inv2), s = add2(t, up);
    const float2 off = split2(fma2(add2(s, down), minus, t)), i = split2(s);
    furthest = max_abs3(furthest, off.x, off.y);
    q[2 * j] = __float_as_uint(i.x);
    q[2 * j + 1] = __float_as_uint(i.y);
  }
  if (furthest > 0.4999f) {
#pragma unroll
    for (int j = 0; j < 8; ++j) q[j] = __float_as_uint(__fadd_rn(__fdiv_rn(f[j], scale), round));
  }
  uint32_t w[2];
#pragma unroll
  for (int h = 0; h < 2; ++h)
    w[h] = __byte_perm(__byte_perm(q[4 * h], q[4 * h + 1], 0x0040), __byte_perm(q[4 * h + 2], q[4 * h + 3], 0x0040), 0x5410);
  return scale < __int_as_float(0x7F800000) ? make_uint2(w[0], w[1]) : make_uint2(0u, 0u);
}

// Epilogue of the int8 products.  Both kernels that have it round every operation by itself, whatever flags they are compiled
// with, so that a token's outputs do not depend on how many tokens come with it.
__device__ __forceinline__ float dequantise1(int sum, float row_scale, float col_scale) {
  return __fmul_rn(__fmul_rn((float)sum, row_scale), col_scale);
}
// act(x) with the ABI's activation codes (0 none, 1 GeLU tanh form, 2 GeLU erf form).  0.5 (1 + tanh u) = 1 / (1 + exp(-2 u)): the
// special-function unit's power of two and reciprocal are good to 2^-22, and a small output keeps its digits.
__device__ __forceinline__ float gelu1(float x, int act) {
  if (act == 1) {
    constexpr float k = -2.0f * 1.4426950408889634f * 0.7978845608028654f;   // -2 log2(e) sqrt(2 / pi)
    float e, h;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(__fmul_rn(x, __fmaf_rn(__fmul_rn(x, x), k * 0.044715f, k))));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(h) : "f"(__fadd_rn(1.0f, e)));
    return __fmul_rn(x, h);
  }
  if (act == 2) return __fmul_rn(__fmul_rn(0.5f, x), __fadd_rn(1.0f, erff(__fmul_rn(x, 0.7071067811865476f))));
  return x;
}

// The same for the experts' products, whose erf form keeps the digits of a small output too: 1 + erf(y) = erfc(-y).  Both of their
// kernels have it, so that a token's activation does not depend on how many tokens come with it.
__device__ __forceinline__ float expert_gelu1(float x, int act) {
  if (act == 2) return __fmul_rn(__fmul_rn(0.5f, x), erfcf(__fmul_rn(x, -0.7071067811865476f)));
  return gelu1(x, act);
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  return v;
}
// Largest magnitude in the warp, `a` >= 0 or NaN (which wins: the bit patterns of non-negative floats are ordered
// and a NaN's lies above infinity's).
__device__ __forceinline__ float warp_max_abs(float a) {
  return __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(a) & 0x7FFFFFFFu));
}

}  // namespace osdp
