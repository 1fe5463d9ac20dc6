// vc_qk_norm_rope: RMS norm of queries and keys (per head, or per token over all heads) and the position rotation.
//
// Bound by memory: every element is read once and written once.  A thread owns eight channels of one token and
// walks over that token's heads, so the angles of a token are formed once for all its heads (a table of the CTA's tokens in
// shared memory), loads and stores are 16 bytes, and a head's sum of squares is a shuffle within its lanes.  The norm over
// a token keeps the thread's part of the token in registers between the sum and the rotation: one pass over memory.
#include <cmath>

#include "vc_layer.cuh"

namespace vc {
namespace {

using namespace layer;

constexpr int kThreads = 256, kKeep = 8, kMaxPairs = 128, kBatch = 4;

struct QkArgs {
  const void *x[2], *w[2];
  void* y[2];
  const int32_t* positions;
  vc_strides in[2], out[2];
  int H[2];
  int N, tiles, chunks, log_lanes, log_hl, weight_dtype;
  int pairs, pair_end[3];          // rotated pairs; where each axis's pairs end
  int grid_h, grid_w, start[3];
  float eps, inv_count[2], mult;
  double turns[kMaxPairs];         // frequency of a pair in turns per position
};

// Angles of the CTA's tokens.  The product is formed in FP64: in FP32 the angle of position 10^5 is off by 10^-2.
// Whole turns are taken off there too, and sincospi sees |x| <= 1.
__device__ __forceinline__ void fill_table(const QkArgs& a, float2* tab, int b, int n0, int tokens) {
  for (int i = threadIdx.x; i < tokens * a.pairs; i += kThreads) {
    const int tt = i / a.pairs, p = i - tt * a.pairs, n = min(n0 + tt, a.N - 1);
    const int axis = (p >= a.pair_end[0]) + (p >= a.pair_end[1]);
    int pos;
    if (a.positions) {
      pos = a.positions[((int64_t)b * a.N + n) * 3 + axis];
    } else {
      const int row = n / a.grid_w;
      pos = a.start[axis] + (axis == 2 ? n - row * a.grid_w : axis == 1 ? row % a.grid_h : row / a.grid_h);
    }
    const double t = (double)pos * a.turns[p];
    float s, c;
    sincospif(2.0f * (float)(t - rint(t)), &s, &c);
    tab[i] = make_float2(c * a.mult, s * a.mult);
  }
}

template <typename T, int NORM, int ROT>
__global__ void __launch_bounds__(kThreads)
qk_norm_kernel(const __grid_constant__ QkArgs a) {
  extern __shared__ float2 tab[];                       // [tokens][pairs]
  __shared__ float xch[ROT == VC_ROTARY_HALF ? kThreads * 8 : 1];
  __shared__ float part[NORM == VC_NORM_TOKEN ? kThreads : 1];
  const int lanes = 1 << a.log_lanes, hls = 1 << a.log_hl, rows = kThreads >> a.log_lanes, tokens = rows >> a.log_hl;
  const int c = threadIdx.x & (lanes - 1), r = threadIdx.x >> a.log_lanes, hl = r & (hls - 1), tt = r >> a.log_hl;
  const int b = blockIdx.x / a.tiles, n0 = (blockIdx.x - b * a.tiles) * tokens, n = n0 + tt;
  const bool live = n < a.N && c < a.chunks;
  pdl_wait();
  // cos and sin of my channels; where a channel is not rotated, bit e of `still` is set
  constexpr int kAngles = ROT == VC_ROTARY_HALF ? 8 : 4;
  float cs[kAngles], sn[kAngles];
  int src[ROT == VC_ROTARY_HALF ? 8 : 1];
  uint32_t still = 0;
  if constexpr (ROT != VC_ROTARY_NONE) {
    fill_table(a, tab, b, n0, tokens);
    __syncthreads();
    const float2* mine = tab + tt * a.pairs;
#pragma unroll
    for (int e = 0; e < kAngles; ++e) {
      cs[e] = 1.f; sn[e] = 0.f;
      if constexpr (ROT == VC_ROTARY_INTERLEAVED) {
        const int p = 4 * c + e;
        if (p < a.pairs) { cs[e] = mine[p].x; sn[e] = mine[p].y; } else still |= 1u << e;
      } else {
        const int ch = 8 * c + e;
        src[e] = e * lanes + c;
        if (ch < 2 * a.pairs) {
          const int axis = (ch >= 2 * a.pair_end[0]) + (ch >= 2 * a.pair_end[1]);
          const int p0 = axis ? a.pair_end[axis - 1] : 0, half = a.pair_end[axis] - p0, i = ch - 2 * p0;
          const bool low = i < half;
          const int other = low ? ch + half : ch - half;
          const float2 t = mine[p0 + (low ? i : i - half)];
          cs[e] = t.x; sn[e] = low ? -t.y : t.y;
          src[e] = (other & 7) * lanes + (other >> 3);
        } else {
          still |= 1u << e;
        }
      }
    }
  }
  auto rotate = [&](float (&f)[8]) {
    if constexpr (ROT == VC_ROTARY_INTERLEAVED) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float f0 = f[2 * e], f1 = f[2 * e + 1];
        const bool keep = still >> e & 1;
        f[2 * e] = keep ? f0 : f0 * cs[e] - f1 * sn[e];
        f[2 * e + 1] = keep ? f1 : f0 * sn[e] + f1 * cs[e];
      }
    } else if constexpr (ROT == VC_ROTARY_HALF) {
      // a pair's halves are half an axis apart, in another lane as a rule: the head's channels change places in
      // shared memory, element-major so that the lanes of an access lie side by side
      float* row = xch + r * 8 * lanes;
      __syncwarp();
#pragma unroll
      for (int e = 0; e < 8; ++e) row[e * lanes + c] = f[e];
      __syncwarp();
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float g = row[src[e]];
        f[e] = still >> e & 1 ? f[e] : f[e] * cs[e] + g * sn[e];
      }
    }
  };
  auto lanes_sum = [&](float v) {
    for (int s = lanes >> 1; s > 0; s >>= 1) v += __shfl_xor_sync(0xffffffffu, v, s);
    return v;
  };
  auto squares = [](const Raw8<T>& raw) {
    float f[8], s = 0.f;
    raw.get(f);
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fmaf(f[e], f[e], s);
    return s;
  };

#pragma unroll 1
  for (int t = 0; t < 2; ++t) {
    const int H = a.H[t];
    if (H == 0) continue;
    const T* x = static_cast<const T*>(a.x[t]) + b * a.in[t].b + (int64_t)n * a.in[t].n + 8 * c;
    T* y = static_cast<T*>(a.y[t]) + b * a.out[t].b + (int64_t)n * a.out[t].n + 8 * c;
    const int64_t sh = a.in[t].h, oh = a.out[t].h;
    const void* w = a.w[t];
    float wt[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) wt[e] = 1.f;
    if constexpr (NORM == VC_NORM_TOKEN) {
      Raw8<T> raw[kKeep];
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < kKeep; ++i) {
        const int h = hl + (i << a.log_hl);
        raw[i].zero();
        if (live && h < H) raw[i].load(x + h * sh);
      }
#pragma unroll
      for (int i = 0; i < kKeep; ++i) ss += squares(raw[i]);
      for (int h = hl + (kKeep << a.log_hl); h < H; h += hls) {      // more heads than the registers hold: read twice
        Raw8<T> more;
        more.zero();
        if (live) more.load(x + h * sh);
        ss += squares(more);
      }
      ss = lanes_sum(ss);
      __syncthreads();                                               // (the sums of Q have been read)
      if (c == 0) part[r] = ss;
      __syncthreads();
      float sum = 0.f;
      for (int i = 0; i < hls; ++i) sum += part[tt * hls + i];       // one order for every thread of the token
      const float inv = rsqrtf(fmaf(sum, a.inv_count[t], a.eps));
      auto finish = [&](const Raw8<T>& v, int h) {
        float f[8];
        v.get(f);
        if (w && live && h < H) load8(w, a.weight_dtype, ((int64_t)h * a.chunks + c) * 8, wt);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = f[e] * inv * wt[e];
        rotate(f);
        if (live && h < H) store8<T>(y + h * oh, f);
      };
#pragma unroll
      for (int i = 0; i < kKeep; ++i)
        if ((i << a.log_hl) < H) finish(raw[i], hl + (i << a.log_hl));
      for (int h0 = kKeep << a.log_hl; h0 < H; h0 += hls) {
        Raw8<T> more;
        more.zero();
        if (live && h0 + hl < H) more.load(x + (h0 + hl) * sh);
        finish(more, h0 + hl);
      }
    } else {
      if (NORM == VC_NORM_HEAD && w && c < a.chunks) load8(w, a.weight_dtype, 8 * c, wt);
      const int step = hls * gridDim.y;
      for (int h0 = blockIdx.y * hls; h0 < H; h0 += kBatch * step) {
        Raw8<T> raw[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
          const int h = h0 + i * step + hl;
          raw[i].zero();
          if (live && h < H) raw[i].load(x + h * sh);
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
          const int h = h0 + i * step + hl;
          if (h0 + i * step >= H) break;
          float f[8];
          raw[i].get(f);
          if constexpr (NORM == VC_NORM_HEAD) {
            const float inv = rsqrtf(fmaf(lanes_sum(squares(raw[i])), a.inv_count[t], a.eps));
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = f[e] * inv * wt[e];
          }
          rotate(f);
          if (live && h < H) store8<T>(y + h * oh, f);
        }
      }
    }
  }
}

template <typename T, int NORM>
cudaError_t launch_rot(int rot, const QkArgs& a, dim3 grid, size_t smem, cudaStream_t s) {
  if (rot == VC_ROTARY_NONE) return launch_overlapped(qk_norm_kernel<T, NORM, VC_ROTARY_NONE>, grid, kThreads, smem, s, a);
  if (rot == VC_ROTARY_INTERLEAVED) return launch_overlapped(qk_norm_kernel<T, NORM, VC_ROTARY_INTERLEAVED>, grid, kThreads, smem, s, a);
  return launch_overlapped(qk_norm_kernel<T, NORM, VC_ROTARY_HALF>, grid, kThreads, smem, s, a);
}
template <typename T>
cudaError_t launch_norm(int norm, int rot, const QkArgs& a, dim3 grid, size_t smem, cudaStream_t s) {
  if (norm == VC_NORM_NONE) return launch_rot<T, VC_NORM_NONE>(rot, a, grid, smem, s);
  if (norm == VC_NORM_HEAD) return launch_rot<T, VC_NORM_HEAD>(rot, a, grid, smem, s);
  return launch_rot<T, VC_NORM_TOKEN>(rot, a, grid, smem, s);
}

constexpr double kTwoPi = 6.283185307179586476925286766559;

// Frequencies of an axis's pairs in turns per position.  Powers by repeated multiplication in extended precision: 64 steps
// of 2^-64 each, against one call of pow() per pair (a call's host time: 1.1 us instead of 4.6 for 64 pairs).
bool axis_frequencies(const vc_qk_params* p, int n, double factor, int original, double theta, double* out) {
  if (n == 0) return true;
  const int pairs = n / 2;
  if (p->rope_scaling == VC_ROPE_SCALING_NTK && n > 2) theta *= std::pow(factor, (double)n / (n - 2));
  if (!(theta > 0.0) || !std::isfinite(theta)) return false;
  const long double ratio = std::pow((long double)theta, -2.0L / n);
  double lo = 0, hi = 1;
  if (p->rope_scaling == VC_ROPE_SCALING_YARN) {
    const double fast = p->yarn_beta_fast != 0.f ? p->yarn_beta_fast : 32.0, slow = p->yarn_beta_slow != 0.f ? p->yarn_beta_slow : 1.0;
    const double per = n / (2.0 * std::log(theta));
    lo = std::floor(per * std::log(original / (kTwoPi * fast)));
    hi = std::ceil(per * std::log(original / (kTwoPi * slow)));
    lo = lo > 0 ? lo : 0;
    hi = hi < n - 1 ? hi : n - 1;
    if (hi - lo < 0.001) hi = lo + 0.001;
  }
  long double f = 1.0L / (long double)kTwoPi;
  for (int i = 0; i < pairs; ++i, f *= ratio) {
    double v = (double)f;
    if (p->rope_scaling == VC_ROPE_SCALING_LINEAR) v /= factor;
    if (p->rope_scaling == VC_ROPE_SCALING_YARN) {
      double r = (i - lo) / (hi - lo);
      r = r < 0 ? 0 : (r > 1 ? 1 : r);
      v = v * (1.0 - r) + v / factor * r;
    }
    out[i] = v;
  }
  return true;
}

bool not_positive(float v) { return v != 0.f && !(v > 0.f && std::isfinite(v)); }

}  // namespace
}  // namespace vc

using namespace vc;

extern "C" vc_status vc_qk_norm_rope(const vc_qk_params* p, const void* q, const void* k, const void* q_weight,
                                     const void* k_weight, const int32_t* positions, void* q_out, void* k_out, void* stream) {
  if (!p) return VC_ERR_INVALID_ARG;
  if (p->B < 1 || p->B > 65535 || p->N < 1 || p->N > (1 << 22)) return VC_ERR_INVALID_ARG;
  if (p->d < 8 || p->d > 256 || p->d % 8) return VC_ERR_INVALID_ARG;
  if (p->H_q < 0 || p->H_q > 65535 || p->H_k < 0 || p->H_k > 65535 || p->H_q + p->H_k == 0) return VC_ERR_INVALID_ARG;
  if (bad_dtype(p->dtype) || bad_dtype(p->weight_dtype)) return VC_ERR_INVALID_ARG;
  if (p->norm < VC_NORM_NONE || p->norm > VC_NORM_TOKEN || p->rotary < VC_ROTARY_NONE || p->rotary > VC_ROTARY_HALF) return VC_ERR_INVALID_ARG;
  if (!(p->eps >= 0.f) || !std::isfinite(p->eps)) return VC_ERR_INVALID_ARG;
  QkArgs a{};
  const int es = elem_size(p->dtype);
  const struct { int H; const void *x, *w; void* y; const vc_strides *in, *out; } side[2] = {
      {p->H_q, q, q_weight, q_out, &p->q, &p->q_out}, {p->H_k, k, k_weight, k_out, &p->k, &p->k_out}};
  for (int t = 0; t < 2; ++t) {
    a.H[t] = side[t].H;
    if (side[t].H == 0) continue;
    if (!side[t].x || !side[t].y || misaligned16(side[t].x) || misaligned16(side[t].y) || misaligned16(side[t].w)) return VC_ERR_INVALID_ARG;
    if (!resolve_strides(*side[t].in, p->B, side[t].H, p->N, p->d, es, false, &a.in[t]) ||
        !resolve_strides(*side[t].out, p->B, side[t].H, p->N, p->d, es, true, &a.out[t]))
      return VC_ERR_INVALID_ARG;
    if (side[t].x == side[t].y && (a.in[t].b != a.out[t].b || a.in[t].h != a.out[t].h || a.in[t].n != a.out[t].n)) return VC_ERR_INVALID_ARG;
    a.x[t] = side[t].x; a.y[t] = side[t].y;
    a.w[t] = p->norm == VC_NORM_NONE ? nullptr : side[t].w;
    a.inv_count[t] = 1.0f / ((float)p->d * (p->norm == VC_NORM_TOKEN ? side[t].H : 1));
  }
  int rot = p->rotary;
  if (rot != VC_ROTARY_NONE) {
    int dims[3] = {p->rope_dim_t, p->rope_dim_h, p->rope_dim_w};
    if (!dims[0] && !dims[1] && !dims[2]) { dims[1] = dims[2] = 2 * (p->d / 6); dims[0] = p->d - 2 * dims[1]; }
    const float factors[3] = {p->rope_factor_t, p->rope_factor_h, p->rope_factor_w};
    const int original[3] = {p->rope_original_t, p->rope_original_h, p->rope_original_w};
    const double theta = p->rope_theta != 0.f ? p->rope_theta : 10000.0;
    if (!(theta > 1.0) || !std::isfinite(theta)) return VC_ERR_INVALID_ARG;
    if (p->rope_scaling < VC_ROPE_SCALING_NONE || p->rope_scaling > VC_ROPE_SCALING_YARN) return VC_ERR_INVALID_ARG;
    if (not_positive(p->yarn_beta_fast) || not_positive(p->yarn_beta_slow) || not_positive(p->rope_attention_factor)) return VC_ERR_INVALID_ARG;
    double largest = 1.0;
    int pairs = 0;
    for (int i = 0; i < 3; ++i) {
      if (dims[i] < 0 || dims[i] % 2 || dims[i] > p->d || not_positive(factors[i])) return VC_ERR_INVALID_ARG;
      if (2 * pairs + dims[i] > p->d) return VC_ERR_INVALID_ARG;
      const double factor = factors[i] != 0.f ? factors[i] : 1.0;
      if (dims[i] && p->rope_scaling == VC_ROPE_SCALING_YARN && original[i] < 1) return VC_ERR_INVALID_ARG;
      if (!axis_frequencies(p, dims[i], factor, original[i], theta, a.turns + pairs)) return VC_ERR_INVALID_ARG;
      if (dims[i] && factor > largest) largest = factor;
      pairs += dims[i] / 2;
      a.pair_end[i] = pairs;
    }
    a.pairs = pairs;
    a.mult = p->rope_attention_factor != 0.f ? p->rope_attention_factor
             : p->rope_scaling == VC_ROPE_SCALING_YARN ? (float)(0.1 * std::log(largest) + 1.0) : 1.0f;
    if (positions) {
      if (misaligned16(positions)) return VC_ERR_INVALID_ARG;
    } else {
      if (p->grid_t < 1 || p->grid_h < 1 || p->grid_w < 1 || p->grid_h > (1 << 22) || p->grid_w > (1 << 22)) return VC_ERR_INVALID_ARG;
      if ((int64_t)p->grid_h * p->grid_w > (1 << 22) || (int64_t)p->grid_t * p->grid_h * p->grid_w != p->N) return VC_ERR_INVALID_ARG;
      const int start[3] = {p->start_t, p->start_h, p->start_w}, grid[3] = {p->grid_t, p->grid_h, p->grid_w};
      for (int i = 0; i < 3; ++i)
        if ((int64_t)start[i] + grid[i] > INT32_MAX) return VC_ERR_INVALID_ARG;
      a.positions = nullptr;
      a.grid_h = p->grid_h; a.grid_w = p->grid_w;
      for (int i = 0; i < 3; ++i) a.start[i] = start[i];
    }
    a.positions = positions;
    if (pairs == 0) rot = VC_ROTARY_NONE;
  }
  a.N = p->N;
  a.chunks = p->d / 8;
  a.weight_dtype = p->weight_dtype;
  a.eps = p->eps != 0.f ? p->eps : 1e-6f;
  while ((1 << a.log_lanes) < a.chunks) ++a.log_lanes;
  const int rows = kThreads >> a.log_lanes, heads = a.H[0] > a.H[1] ? a.H[0] : a.H[1];
  // Rows of a CTA side by side: `1 << log_hl` heads of each token.  The norm over a token takes as many as bring the heads that
  // a thread keeps down to kKeep; else as many as a short sequence leaves without a token.
  if (p->norm == VC_NORM_TOKEN)
    while ((1 << a.log_hl) < rows && (heads > kKeep << a.log_hl || (rows >> a.log_hl) >= 2 * p->N)) ++a.log_hl;
  else
    while ((1 << a.log_hl) < rows && (rows >> a.log_hl) >= 2 * p->N) ++a.log_hl;
  const int tokens = rows >> a.log_hl;
  a.tiles = (p->N + tokens - 1) / tokens;
  const int64_t ctas = (int64_t)p->B * a.tiles;
  if (ctas > INT32_MAX) return VC_ERR_UNSUPPORTED;
  int split = 1;
  if (p->norm != VC_NORM_TOKEN) {            // few tokens: their heads go to several CTAs
    const int64_t most = (heads + (1 << a.log_hl) - 1) >> a.log_hl, want = (8 * sm_count() + ctas - 1) / ctas;
    split = (int)(want < most ? want : most);
  }
  const dim3 grid((unsigned)ctas, (unsigned)split);
  const size_t smem = rot == VC_ROTARY_NONE ? 0 : (size_t)tokens * a.pairs * sizeof(float2);
  cudaStream_t s = (cudaStream_t)stream;
  const cudaError_t e = p->dtype == VC_DTYPE_BF16   ? launch_norm<__nv_bfloat16>(p->norm, rot, a, grid, smem, s)
                        : p->dtype == VC_DTYPE_FP16 ? launch_norm<__half>(p->norm, rot, a, grid, smem, s)
                                                    : launch_norm<float>(p->norm, rot, a, grid, smem, s);
  if (e != cudaSuccess) return VC_ERR_CUDA;
  count_launches(1);
  return VC_OK;
}
