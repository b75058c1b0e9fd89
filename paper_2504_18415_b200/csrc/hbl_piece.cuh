// Eight consecutive elements of a head, as the kernels over heads load and store them.
#pragma once

#include "hbl_common.cuh"

namespace hbl {

// Eight consecutive elements, as loaded.
template <typename T>
struct Piece;
template <>
struct Piece<__nv_bfloat16> {
  uint4 w;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { w = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void store(__nv_bfloat16* p) const { *reinterpret_cast<uint4*>(p) = w; }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(u[i] << 16);
      f[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
    }
  }
  __device__ __forceinline__ void set(const float (&f)[8]) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
      u[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    w = make_uint4(u[0], u[1], u[2], u[3]);
  }
};
template <>
struct Piece<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = *reinterpret_cast<const float4*>(p);
    b = *reinterpret_cast<const float4*>(p + 4);
  }
  __device__ __forceinline__ void store(float* p) const {
    *reinterpret_cast<float4*>(p) = a;
    *reinterpret_cast<float4*>(p + 4) = b;
  }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  }
  __device__ __forceinline__ void set(const float (&f)[8]) {
    a = make_float4(f[0], f[1], f[2], f[3]);
    b = make_float4(f[4], f[5], f[6], f[7]);
  }
};

// Two fp32 operations to an instruction, each rounded as on its own; sums one by one, because a product and a sum that are both
// packed come out contracted to one rounding.
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  asm("{\n .reg .b64 u, v;\n mov.b64 u, {%0, %1};\n mov.b64 v, {%2, %3};\n mul.rn.f32x2 u, u, v;\n mov.b64 {%0, %1}, u;\n}"
      : "+f"(a.x), "+f"(a.y) : "f"(b.x), "f"(b.y));
  return a;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) { return make_float2(__fadd_rn(a.x, b.x), __fadd_rn(a.y, b.y)); }
__device__ __forceinline__ float2 sub2(float2 a, float2 b) { return make_float2(__fsub_rn(a.x, b.x), __fsub_rn(a.y, b.y)); }
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  asm("{\n .reg .b64 u, v, w;\n mov.b64 u, {%0, %1};\n mov.b64 v, {%2, %3};\n mov.b64 w, {%4, %5};\n fma.rn.f32x2 u, u, v, w;\n mov.b64 {%0, %1}, u;\n}"
      : "+f"(a.x), "+f"(a.y) : "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return a;
}
__device__ __forceinline__ void copy_async16(uint4* dst, const uint4* src) {         // to shared memory
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}

// Gains of 8 consecutive elements; NULL: ones.
__device__ __forceinline__ void load_gain(const void* gain, int bf16, int d, float (&g)[8]) {
  if (gain == nullptr) {
#pragma unroll
    for (int i = 0; i < 8; ++i) g[i] = 1.f;
  } else if (bf16) {
    Piece<__nv_bfloat16> p;
    p.load(static_cast<const __nv_bfloat16*>(gain) + d);
    p.get(g);
  } else {
    Piece<float> p;
    p.load(static_cast<const float*>(gain) + d);
    p.get(g);
  }
}
// 1 / sqrt(v) rounded to fp32: two steps of Newton's iteration y (3 - v y^2) / 2 from an fp32 value (off by 2^-22, 2^-43
// after one step).  What fp32 cannot start from (0, infinities, NaN, and far out) goes the long way.
__device__ __forceinline__ float inverse_root(double v) {
  if (!(v > 1e-30 && v < 1e30)) return (float)(1.0 / sqrt(v));
  double y = rsqrtf((float)v);
#pragma unroll
  for (int i = 0; i < 2; ++i) y = fma(0.5 * y, fma(-v * y, y, 1.0), y);
  return (float)y;
}

}  // namespace hbl
