// vc_quant_fp8: a matrix as E4M3 codes with one FP32 scale per block of 128 columns and 1 or 128 rows.
//
// Bound by memory: two or four bytes in, one out.  block_rows 1: eight lanes hold the 128 columns of a row's block, sixteen
// each, so the codes leave 16 bytes at a time and the maximum is three shuffles; a CTA takes 32 rows, whose scales
// lie side by side.  block_rows 128: a CTA holds its block in registers between the maximum and the codes.
//
// 40 heads x 32760 x 128 in bf16 (508 MB): 89 us, 88 % of the measured copy rate; the issue slots are 67 % taken, the ALU half.  One block of
// columns in flight a thread or four, CTAs of 128 or 512 threads: no better over the sizes.
#include <cuda_fp8.h>

#include "vc_layer.cuh"

namespace vc {
namespace {

using namespace layer;

constexpr int kThreads = 256, kRows = kThreads / 8;
constexpr float kTop = 448.0f, kLeast = 448.0f / 1.2676506002282294e30f;     // the largest code; 448 * 2^-100

struct QuantArgs {
  const void* x;
  uint8_t* codes;
  float* scale;
  vc_strides in;
  unsigned long long mul_d;       // ceil(2^40 / d): column / d by one multiplication (columns below 2^20)
  int N, d, rows, cols, blocks;
};

__device__ __forceinline__ float max_nan(float a, float b) {      // a NaN stays
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
template <typename T> __device__ __forceinline__ float amax8(const Raw8<T>& raw) {
  float f[8], m = 0.f;
  raw.get(f);
#pragma unroll
  for (int e = 0; e < 8; ++e) m = max_nan(m, fabsf(f[e]));
  return m;
}
template <typename T> __device__ __forceinline__ uint2 codes8(const Raw8<T>& raw, float inv) {
  float f[8];
  raw.get(f);
  uint32_t w[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = __nv_cvt_float2_to_fp8x2(make_float2(f[2 * e] * inv, f[2 * e + 1] * inv), __NV_SATFINITE, __NV_E4M3);
  return make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
}
// Sixteen columns from `col` on of a row (two groups of eight, which may belong to different heads).
template <typename T> __device__ __forceinline__ void load16(const QuantArgs& a, const T* row, int col, Raw8<T>& lo, Raw8<T>& hi) {
  lo.zero(); hi.zero();
  if (col < a.cols) {               // (the width is a multiple of 16)
    const int h0 = (int)(((unsigned long long)col * a.mul_d) >> 40), h1 = (int)(((unsigned long long)(col + 8) * a.mul_d) >> 40);
    lo.load(row + h0 * a.in.h + (col - h0 * a.d));
    hi.load(row + h1 * a.in.h + (col + 8 - h1 * a.d));
  }
}
template <typename T> __device__ __forceinline__ const T* row_of(const QuantArgs& a, int r) {
  const int b = r / a.N;
  return static_cast<const T*>(a.x) + b * a.in.b + (int64_t)(r - b * a.N) * a.in.n;
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
quant_rows_kernel(const __grid_constant__ QuantArgs a) {
  const int lane = threadIdx.x & 7, r = blockIdx.x * kRows + (threadIdx.x >> 3);
  const bool live = r < a.rows;
  pdl_wait();
  const T* row = row_of<T>(a, live ? r : a.rows - 1);
  constexpr int kBatch = 2;         // blocks in flight: 64 bytes a thread at 16 bits
  for (int kb0 = blockIdx.y; kb0 < a.blocks; kb0 += kBatch * gridDim.y) {
    Raw8<T> lo[kBatch], hi[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) load16(a, row, min(kb0 + i * (int)gridDim.y, a.blocks) * 128 + 16 * lane, lo[i], hi[i]);
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int kb = kb0 + i * gridDim.y, col = kb * 128 + 16 * lane;
      float m = max_nan(amax8(lo[i]), amax8(hi[i]));
#pragma unroll
      for (int s = 4; s > 0; s >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, s));
      m = max_nan(m, kLeast);
      const float inv = kTop / m;
      const uint2 c0 = codes8(lo[i], inv), c1 = codes8(hi[i], inv);
      if (live && kb < a.blocks) {
        if (col < a.cols) *reinterpret_cast<uint4*>(a.codes + (int64_t)r * a.cols + col) = make_uint4(c0.x, c0.y, c1.x, c1.y);
        if (lane == 0) a.scale[(int64_t)kb * a.rows + r] = m / kTop;
      }
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
quant_tiles_kernel(const __grid_constant__ QuantArgs a) {
  __shared__ float part[kThreads / 32];
  const int lane = threadIdx.x & 7, r0 = blockIdx.x * 128 + (threadIdx.x >> 3), col = blockIdx.y * 128 + 16 * lane;
  pdl_wait();
  constexpr int kTimes = 128 / kRows;
  Raw8<T> lo[kTimes], hi[kTimes];
  float m = kLeast;
#pragma unroll
  for (int i = 0; i < kTimes; ++i) {
    const int r = r0 + i * kRows;
    load16(a, row_of<T>(a, min(r, a.rows - 1)), r < a.rows ? col : a.cols, lo[i], hi[i]);
  }
#pragma unroll
  for (int i = 0; i < kTimes; ++i) m = max_nan(m, max_nan(amax8(lo[i]), amax8(hi[i])));
#pragma unroll
  for (int s = 16; s > 0; s >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, s));
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kThreads / 32; ++i) m = max_nan(m, part[i]);
  const float inv = kTop / m;
#pragma unroll
  for (int i = 0; i < kTimes; ++i) {
    const int r = r0 + i * kRows;
    const uint2 c0 = codes8(lo[i], inv), c1 = codes8(hi[i], inv);
    if (r < a.rows && col < a.cols) *reinterpret_cast<uint4*>(a.codes + (int64_t)r * a.cols + col) = make_uint4(c0.x, c0.y, c1.x, c1.y);
  }
  if (threadIdx.x == 0) a.scale[(int64_t)blockIdx.x * a.blocks + blockIdx.y] = m / kTop;
}

template <typename T>
cudaError_t launch_quant(const QuantArgs& a, int block_rows, cudaStream_t s) {
  if (block_rows == 128) return launch_overlapped(quant_tiles_kernel<T>, dim3((unsigned)((a.rows + 127) / 128), (unsigned)a.blocks), kThreads, 0, s, a);
  const int tiles = (a.rows + kRows - 1) / kRows;
  int split = (8 * sm_count() + tiles - 1) / tiles;             // few rows: their blocks go to several CTAs
  if (split > a.blocks) split = a.blocks;
  return launch_overlapped(quant_rows_kernel<T>, dim3((unsigned)tiles, (unsigned)split), kThreads, 0, s, a);
}

}  // namespace
}  // namespace vc

using namespace vc;

extern "C" vc_status vc_quant_fp8(const vc_quant_params* p, const void* x, void* codes, float* scale, void* stream) {
  if (!p || !x || !codes || !scale) return VC_ERR_INVALID_ARG;
  if (misaligned16(x) || misaligned16(codes) || misaligned16(scale)) return VC_ERR_INVALID_ARG;
  if (p->B < 1 || p->H < 1 || p->N < 1 || p->d < 8 || p->d % 8 || bad_dtype(p->dtype)) return VC_ERR_INVALID_ARG;
  const int64_t rows = (int64_t)p->B * p->N, cols = (int64_t)p->H * p->d;
  if (rows > INT32_MAX - 128 || cols > (1 << 20) || cols % 16) return VC_ERR_INVALID_ARG;
  if (p->block_rows != 1 && p->block_rows != 128) return VC_ERR_INVALID_ARG;
  QuantArgs a{};
  if (!resolve_strides(p->x, p->B, p->H, p->N, p->d, elem_size(p->dtype), false, &a.in)) return VC_ERR_INVALID_ARG;
  a.x = x; a.codes = (uint8_t*)codes; a.scale = scale;
  a.mul_d = ((1ull << 40) + p->d - 1) / p->d;
  a.N = p->N; a.d = p->d; a.rows = (int)rows; a.cols = (int)cols; a.blocks = (int)((cols + 127) / 128);
  cudaStream_t s = (cudaStream_t)stream;
  const cudaError_t e = p->dtype == VC_DTYPE_BF16   ? launch_quant<__nv_bfloat16>(a, p->block_rows, s)
                        : p->dtype == VC_DTYPE_FP16 ? launch_quant<__half>(a, p->block_rows, s)
                                                    : launch_quant<float>(a, p->block_rows, s);
  if (e != cudaSuccess) return VC_ERR_CUDA;
  count_launches(1);
  return VC_OK;
}
