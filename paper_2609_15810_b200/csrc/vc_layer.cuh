// Pieces shared by the operators around the quantized attention: element types, strides, vector loads and stores of
// eight elements.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <utility>

#include "vc_internal.h"
#include "vc_launch.h"
#include "vc_sm100.cuh"

namespace vc {
namespace layer {

inline int elem_size(int dtype) { return dtype == VC_DTYPE_FP32 ? 4 : 2; }
inline bool bad_dtype(int dtype) { return dtype < VC_DTYPE_BF16 || dtype > VC_DTYPE_FP32; }
inline bool misaligned16(const void* p) { return ((uintptr_t)p & 15) != 0; }

// Strides of [B][H][N][d] with the packed default filled in; those of dimensions of one entry are never used and are
// made harmless.  Refuses rows off a 16-byte boundary and tokens that overlap, for outputs any two rows that might: taken by
// stride, each dimension must step over what the smaller ones span (a broadcast, stride 0, does not).  Strides stay below 2^40
// bytes, so that the span of an output (2^22 tokens, 65535 heads and batches at most) stays below 2^63.
inline bool resolve_strides(const vc_strides& in, int64_t B, int64_t H, int64_t N, int64_t d, int es, bool output, vc_strides* out) {
  vc_strides s = in;
  if (!s.b && !s.h && !s.n) { s.n = d; s.h = N * d; s.b = H * N * d; }
  if (B == 1) s.b = 0;
  if (H == 1) s.h = 0;
  if (N == 1) s.n = d;
  const int64_t per16 = 16 / es, most = (1ll << 40) / es;
  if (s.b < 0 || s.h < 0 || s.n < d) return false;
  if (s.b >= most || s.h >= most || s.n >= most) return false;
  if (s.b % per16 || s.h % per16 || s.n % per16) return false;
  if (output) {
    struct { int64_t count, stride; } dim[3] = {{B, s.b}, {H, s.h}, {N, s.n}};
    for (int i = 0; i < 2; ++i)
      for (int j = 0; j < 2 - i; ++j)
        if (dim[j].stride > dim[j + 1].stride) std::swap(dim[j], dim[j + 1]);
    int64_t span = d;
    for (const auto& m : dim) {
      if (m.count == 1) continue;
      if (m.stride < span) return false;
      span += (m.count - 1) * m.stride;
    }
  }
  *out = s;
  return true;
}

#ifdef __CUDACC__
template <typename T> __device__ __forceinline__ float2 unpack16(uint32_t v);
template <> __device__ __forceinline__ float2 unpack16<__nv_bfloat16>(uint32_t v) {
  return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
}
template <> __device__ __forceinline__ float2 unpack16<__half>(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2*>(&v)); }
template <typename T> __device__ __forceinline__ uint32_t pack16(float a, float b);
template <> __device__ __forceinline__ uint32_t pack16<__nv_bfloat16>(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
template <> __device__ __forceinline__ uint32_t pack16<__half>(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// Eight consecutive elements as they lie in memory (16-byte aligned).
template <typename T> struct Raw8 {
  uint4 v;
  __device__ __forceinline__ void load(const T* p) { v = __ldcs(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void load_again(const T* p) { v = __ldg(reinterpret_cast<const uint4*>(p)); }     // (read by many CTAs)
  __device__ __forceinline__ void get(float (&f)[8]) const {
    const float2 a = unpack16<T>(v.x), b = unpack16<T>(v.y), c = unpack16<T>(v.z), d = unpack16<T>(v.w);
    f[0] = a.x; f[1] = a.y; f[2] = b.x; f[3] = b.y; f[4] = c.x; f[5] = c.y; f[6] = d.x; f[7] = d.y;
  }
  __device__ __forceinline__ void zero() { v = make_uint4(0, 0, 0, 0); }
};
template <> struct Raw8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = __ldcs(reinterpret_cast<const float4*>(p));
    b = __ldcs(reinterpret_cast<const float4*>(p) + 1);
  }
  __device__ __forceinline__ void load_again(const float* p) {
    a = __ldg(reinterpret_cast<const float4*>(p));
    b = __ldg(reinterpret_cast<const float4*>(p) + 1);
  }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  }
  __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
};
template <typename T> __device__ __forceinline__ void store8(T* p, const float (&f)[8]) {
  *reinterpret_cast<uint4*>(p) = make_uint4(pack16<T>(f[0], f[1]), pack16<T>(f[2], f[3]), pack16<T>(f[4], f[5]), pack16<T>(f[6], f[7]));
}
template <> __device__ __forceinline__ void store8<float>(float* p, const float (&f)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
}
// f times a number, f times g, two products an instruction.
__device__ __forceinline__ void times(float (&f)[8], float g) {
#pragma unroll
  for (int e = 0; e < 8; e += 2) sm100::unpack2(sm100::mul2(sm100::pack_f32x2(f[e], f[e + 1]), sm100::pack_f32x2(g, g)), f[e], f[e + 1]);
}
__device__ __forceinline__ void times(float (&f)[8], const float (&g)[8]) {
#pragma unroll
  for (int e = 0; e < 8; e += 2) sm100::unpack2(sm100::mul2(sm100::pack_f32x2(f[e], f[e + 1]), sm100::pack_f32x2(g[e], g[e + 1])), f[e], f[e + 1]);
}
// One element / eight elements of an array whose type is an argument.
__device__ __forceinline__ float load1(const void* p, int dtype, int64_t i) {
  if (dtype == VC_DTYPE_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
  if (dtype == VC_DTYPE_FP16) return __half2float(static_cast<const __half*>(p)[i]);
  return static_cast<const float*>(p)[i];
}
__device__ __forceinline__ void load8(const void* p, int dtype, int64_t i, float (&f)[8]) {
  if (dtype == VC_DTYPE_FP32) {
    const float4 a = __ldg(reinterpret_cast<const float4*>(static_cast<const float*>(p) + i)), b = __ldg(reinterpret_cast<const float4*>(static_cast<const float*>(p) + i) + 1);
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  } else {
    const uint4 u = __ldg(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + i));
    if (dtype == VC_DTYPE_BF16) Raw8<__nv_bfloat16>{u}.get(f);
    else Raw8<__half>{u}.get(f);
  }
}
#endif

}  // namespace layer
}  // namespace vc
