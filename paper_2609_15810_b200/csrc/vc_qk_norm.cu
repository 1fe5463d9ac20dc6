// vc_qk_norm_rope: RMS norm of queries and keys (per head, or per token over all heads) and the position rotation.
//
// Bound by memory: every element is read once and written once.  A thread owns sixteen channels of one token and
// walks over that token's heads, so the angles of a token are formed once for all its heads (a table of the CTA's tokens in
// shared memory), loads and stores are 16 bytes, and a head's sum of squares is a shuffle within its lanes.  The norm over
// a token keeps the thread's part of the token in registers between the sum and the rotation: one pass over memory.
//
// 32760 tokens of d128, interleaved, 40 + 40 / 12 + 12 heads, calls that follow one another: rotation alone 213 / 66 us (97 / 94 % of the measured copy rate),
// with the norm per head 229-236 / 85, per token 253-256 / 92 (1342 / 403 MB; a CTA's loads stand still while a token's sum is formed, and the angles cost 14 to 19).  Eight
// channels a thread instead of 16: 302 for 260 at that time (angles, addresses and shuffles per row cost twice as much); CTAs of 256 threads: 282 (more
// warps wait for a token's slowest); five or six CTAs an SM: 284 and 326 (spills), with three heads a thread 12 heads 98 for 105, 40 heads 333.
// Halves whose axes are multiples of 16 channels: 24 + 24 heads with the norm per head 153 us (floor 124).  Other axes, the default split of d 64 and 128 among
// them: 24 + 24 heads 262, 40 + 40 heads 420 (floor 206); the change of places in shared memory bounds it, head after head.  Under the token norm
// the 16-bit form of these spills 64 bytes of stores and 32 of loads a thread.
#include <cmath>

#include "vc_layer.cuh"

namespace vc {
namespace {

using namespace layer;

constexpr int kThreads = 128, kMaxPairs = 128;
// Halves whose axes are multiples of 16 channels: a pair's two channels lie in whole groups of eight, and one thread owns both groups.
constexpr int kRotaryWhole = VC_ROTARY_HALF + 1;

// Heads whose channels a thread holds in registers: four CTAs an SM then fit the register file.
__host__ __device__ constexpr int heads_held(int elem_bytes, int rotary) { return rotary == VC_ROTARY_HALF ? (elem_bytes == 2 ? 3 : 1) : (elem_bytes == 2 ? 5 : 2); }

struct QkArgs {
  const void *x[2], *w[2];
  void* y[2];
  const int32_t* positions;
  vc_strides in[2], out[2];
  int H[2], first;                 // first: 1 if there is no Q
  bool both;                       // a CTA takes its tokens' Q, then their K (else blockIdx.z is one of them)
  int N, chunks, log_lanes, log_hl, log_pairs, weight_dtype;     // log_pairs: 2^log_pairs >= pairs
  bool same_type;                  // weights are of the tensors' type
  bool partial;                    // some channels are not rotated
  // The two groups of eight channels of a lane (255: none), and (kRotaryWhole) their first pair (255: not rotated).
  uint8_t lo[16], hi[16], first_pair[16];
  int pairs, pair_end[3];          // rotated pairs; where each axis's pairs end
  int grid_h, grid_w, start[3];
  float inv_w, inv_h;              // about 1 / grid_w, 1 / grid_h
  float eps, inv_count[2], mult;
  uint64_t turns[kMaxPairs];       // frequency of a pair in turns per position, 64 bits behind the point
};

// n / by for n and by up to 2^22, inv about 1 / by: the quotient in FP32 is off by one at most.
__device__ __forceinline__ int quotient(int n, int by, float inv) {
  const int q = __float2int_rd((float)n * inv), r = n - q * by;
  return q + (r >= by) - (r < 0);
}

// Angles of the CTA's tokens.  The product of position and frequency is formed in 64-bit fixed point, whose overflow takes off the whole
// turns: at position p it is off by |p| 2^-64 turns, and by p times what the frequency is off by (see axis_frequencies; together below 2^-27 at
// position 2^31).  Rounding it to FP32 for the sine, up to 2^-26 turns, is more.  (In FP32 the angle of position 10^5 is off by 10^-2; in FP64, with the
// integer divisions of the position, a table took twice as long: 12 + 12 heads x 32760 x 128, norm per head, 94.3 us instead of 85.2.)
__device__ __forceinline__ void fill_table(const QkArgs& a, float2* tab, int b, int n0, int tokens) {
  const int p = threadIdx.x & ((1 << a.log_pairs) - 1);
  if (p >= a.pairs) return;
  const int axis = (p >= a.pair_end[0]) + (p >= a.pair_end[1]);
  const uint64_t turns = a.turns[p];
  for (int tt = threadIdx.x >> a.log_pairs; tt < tokens; tt += kThreads >> a.log_pairs) {
    const int n = min(n0 + tt, a.N - 1);
    int pos;
    if (a.positions) {
      pos = a.positions[((int64_t)b * a.N + n) * 3 + axis];
    } else {
      const int row = quotient(n, a.grid_w, a.inv_w), t = quotient(row, a.grid_h, a.inv_h);
      pos = a.start[axis] + (axis == 2 ? n - row * a.grid_w : axis == 1 ? row - t * a.grid_h : t);
    }
    const uint64_t t = (uint64_t)(int64_t)pos * turns;
    float s, c;
    sincospif((float)(int32_t)(t >> 32) * 0x1p-31f, &s, &c);      // half turns, in [-1, 1]
    tab[tt * a.pairs + p] = make_float2(c * a.mult, s * a.mult);
  }
}

// f times eight weights.  Their type is an argument; as a rule it is the tensors'.
template <typename T> __device__ __forceinline__ void times_weights(float (&f)[8], const QkArgs& a, const void* w, int64_t at) {
  float wt[8];
  if (a.same_type) {
    Raw8<T> raw;
    raw.load_again(static_cast<const T*>(w) + at);
    raw.get(wt);
  } else {
    load8(w, a.weight_dtype, at, wt);
  }
  times(f, wt);
}

template <typename T, int NORM, int ROT>
__global__ void __launch_bounds__(kThreads, 4)
qk_norm_kernel(const __grid_constant__ QkArgs a) {
  extern __shared__ __align__(16) float2 tab[];         // [tokens of the CTA][pairs]
  __shared__ float xch[ROT == VC_ROTARY_HALF ? kThreads * 16 + 1 : 1];  // (the last one is 0)
  __shared__ float part[NORM == VC_NORM_TOKEN ? 2 : 1][kThreads / 32];
  constexpr int kKeep = heads_held(sizeof(T), ROT);
  const int lanes = 1 << a.log_lanes, tokens = kThreads >> (a.log_lanes + a.log_hl);
  const int c = threadIdx.x & (lanes - 1), r = threadIdx.x >> a.log_lanes, hl = r & ((1 << a.log_hl) - 1), tt = r >> a.log_hl;
  const int b = blockIdx.y, n0 = blockIdx.x * tokens, n = n0 + tt;
  const int first = a.both ? 0 : blockIdx.z + a.first, last = a.both ? 1 : first;       // Q, K or (the norm over a token alone) Q and then K
  // My channels: two groups of eight.
  const int lo = a.lo[c], hi = a.hi[c];
  const bool ch0 = lo != 255, ch1 = hi != 255;
  const int at0 = 8 * (ch0 ? lo : 0), at1 = 8 * (ch1 ? hi : 0), step = at1 - at0;
  const bool live0 = n < a.N && ch0, live1 = n < a.N && ch1;
  // cos and sin of my channels.  One that is not rotated keeps its value whatever its neighbour holds: bit e of `still`, or 0 in the
  // place of the other half (with as many bits to test the predicate registers run out).
  constexpr int kAngles = ROT >= VC_ROTARY_HALF ? 8 : 4;
  float cs[2][kAngles], sn[2][kAngles];
  int src[2][ROT == VC_ROTARY_HALF ? 8 : 1];
  uint32_t still = 0;
  const bool turned = ROT == kRotaryWhole && a.first_pair[c] != 255;

  auto lanes_sum = [](float v, int count) {
    for (int s = count >> 1; s > 0; s >>= 1) v += __shfl_xor_sync(0xffffffffu, v, s);
    return v;
  };
  auto squares = [](const Raw8<T>& v) {
    float f[8], even, odd;
    uint64_t s = 0;
    v.get(f);
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const uint64_t f2 = sm100::pack_f32x2(f[e], f[e + 1]);
      s = sm100::fma2(f2, f2, s);
    }
    sm100::unpack2(s, even, odd);
    return even + odd;
  };
  auto side = [&](const int t) {
    const int H = a.H[t];
    const void* w = a.w[t];
    // My heads: hl, hl + hls, ..., `rows` of them, the last one perhaps behind H.  (What lies outside reads another place and is
    // neither summed nor stored.)
    const int rows = (H + (1 << a.log_hl) - 1) >> a.log_hl;
    const bool last_in = hl + ((rows - 1) << a.log_hl) < H;
    const int64_t sx = a.in[t].h << a.log_hl, sy = a.out[t].h << a.log_hl;
    const T* x = static_cast<const T*>(a.x[t]) + (b * a.in[t].b + (hl < H ? hl : 0) * a.in[t].h + (int64_t)min(n, a.N - 1) * a.in[t].n + at0);
    T* y = static_cast<T*>(a.y[t]) + (b * a.out[t].b + hl * a.out[t].h + (int64_t)n * a.out[t].n + at0);
    if (t == first) pdl_wait();
    Raw8<T> raw[kKeep][2];
    auto load_rows = [&](int i0) {                        // heads i0, i0 + 1, ... of mine
      const T* from = x + i0 * sx;
#pragma unroll
      for (int i = 0; i < kKeep; ++i) {
        if (i0 + i >= rows) break;
        if (i0 + i + 1 == rows && !last_in) from = x;
        raw[i][0].load(from);
        raw[i][1].load(from + step);
        from += sx;
      }
    };
    load_rows(0);                                         // (on their way while the angles are formed)
    float wt[2][8];
#pragma unroll
    for (int e = 0; e < 8; ++e) wt[0][e] = wt[1][e] = 1.f;
    if (NORM == VC_NORM_HEAD && w) {
      times_weights<T>(wt[0], a, w, at0);
      times_weights<T>(wt[1], a, w, at1);
    }
    if (ROT != VC_ROTARY_NONE && t == first) {
      fill_table(a, tab, b, n0, tokens);
      if (ROT == VC_ROTARY_HALF && threadIdx.x == 0) xch[kThreads * 16] = 0.f;
      if constexpr (NORM != VC_NORM_TOKEN) __syncthreads();
    }

    float inv = 1.f;
    if constexpr (NORM == VC_NORM_TOKEN) {
      float ss0 = 0.f, ss1 = 0.f;
      for (int i0 = 0;;) {
#pragma unroll
        for (int i = 0; i < kKeep; ++i) {
          if (i0 + i >= rows) break;
          const float q0 = squares(raw[i][0]), q1 = squares(raw[i][1]);
          if (i0 + i + 1 < rows || last_in) { ss0 += q0; ss1 += q1; }
        }
        i0 += kKeep;
        if (i0 >= rows) break;
        load_rows(i0);
      }
      float ss = lanes_sum((ch0 ? ss0 : 0.f) + (ch1 ? ss1 : 0.f), min(lanes << a.log_hl, 32));   // a token's lanes in this warp
      if ((threadIdx.x & 31) == 0) part[t][threadIdx.x >> 5] = ss;
      __syncthreads();
      const int warps = lanes << a.log_hl >> 5;                          // of a token; 0 or 1: its sum is at hand
      if (warps > 1) {
        ss = 0.f;
        for (int i = 0; i < warps; ++i) ss += part[t][(threadIdx.x >> 5 & -warps) + i];   // one order for every thread of the token
      }
      inv = rsqrtf(fmaf(ss, a.inv_count[t], a.eps));
      if (rows > kKeep) load_rows(0);                                 // more heads than the registers hold: read twice
    }

    if (t == first) {
      const float2* mine = tab + tt * a.pairs;
      if constexpr (ROT == kRotaryWhole) {
        const float4* from = reinterpret_cast<const float4*>(mine + (turned ? a.first_pair[c] : 0));      // (a multiple of eight pairs on)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float4 v = from[e];
          cs[0][2 * e] = v.x; sn[0][2 * e] = v.y; cs[0][2 * e + 1] = v.z; sn[0][2 * e + 1] = v.w;
        }
      } else if constexpr (ROT != VC_ROTARY_NONE) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const int cq = c + q * lanes;
#pragma unroll
          for (int e = 0; e < kAngles; ++e) {
            cs[q][e] = 1.f; sn[q][e] = 0.f;
            if constexpr (ROT == VC_ROTARY_INTERLEAVED) {
              const int p = 4 * cq + e;
              if (p < a.pairs) { cs[q][e] = mine[p].x; sn[q][e] = mine[p].y; } else still |= 1u << (4 * q + e);
            } else {
              const int ch = 8 * cq + e;
              src[q][e] = kThreads * 16 - r * 16 * lanes;
              if (ch < 2 * a.pairs) {
                const int axis = (ch >= 2 * a.pair_end[0]) + (ch >= 2 * a.pair_end[1]);
                const int p0 = axis ? a.pair_end[axis - 1] : 0, half = a.pair_end[axis] - p0, i = ch - 2 * p0;
                const bool low = i < half;
                const int other = low ? ch + half : ch - half;
                const float2 cosine_sine = mine[p0 + (low ? i : i - half)];
                cs[q][e] = cosine_sine.x; sn[q][e] = low ? -cosine_sine.y : cosine_sine.y;
                src[q][e] = (other & 7) * 2 * lanes + (other >> 3);
              }
            }
          }
        }
      }
    }
    auto rotate = [&](float (&f)[2][8]) {
      if constexpr (ROT == kRotaryWhole) {
        if (turned) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float f0 = f[0][e], f1 = f[1][e];
            f[0][e] = f0 * cs[0][e] - f1 * sn[0][e];
            f[1][e] = f0 * sn[0][e] + f1 * cs[0][e];
          }
        }
      } else if constexpr (ROT == VC_ROTARY_INTERLEAVED) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          float g[8];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            g[2 * e] = f[q][2 * e] * cs[q][e] - f[q][2 * e + 1] * sn[q][e];
            g[2 * e + 1] = f[q][2 * e] * sn[q][e] + f[q][2 * e + 1] * cs[q][e];
          }
          if (a.partial) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (still >> (4 * q + e / 2) & 1) g[e] = f[q][e];
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) f[q][e] = g[e];
        }
      } else if constexpr (ROT == VC_ROTARY_HALF) {
        // a pair's halves are half an axis apart, in another lane as a rule: the head's channels change places in
        // shared memory, element-major so that the lanes of an access lie side by side
        float* row = xch + r * 16 * lanes;
        __syncwarp();
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          row[e * 2 * lanes + c] = f[0][e];
          row[e * 2 * lanes + c + lanes] = f[1][e];
        }
        __syncwarp();
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
          for (int e = 0; e < 8; ++e) f[q][e] = f[q][e] * cs[q][e] + row[src[q][e]] * sn[q][e];
      }
    };

    int64_t w_at = (int64_t)hl * a.chunks * 8 + at0;
    for (int i0 = 0; i0 < rows;) {
#pragma unroll
      for (int i = 0; i < kKeep; ++i) {
        if (i0 + i >= rows) break;
        const bool in = i0 + i + 1 < rows || last_in;
        float f[2][8];
        raw[i][0].get(f[0]);
        raw[i][1].get(f[1]);
        if constexpr (NORM == VC_NORM_HEAD) {
          const float q0 = squares(raw[i][0]), q1 = squares(raw[i][1]);
          inv = rsqrtf(fmaf(lanes_sum((ch0 ? q0 : 0.f) + (ch1 ? q1 : 0.f), lanes), a.inv_count[t], a.eps));
        }
        if constexpr (NORM != VC_NORM_NONE) {
          times(f[0], inv);
          times(f[1], inv);
        }
        if constexpr (NORM == VC_NORM_HEAD) {
          times(f[0], wt[0]);
          times(f[1], wt[1]);
        }
        if constexpr (NORM == VC_NORM_TOKEN) {
          if (w && in) {
            times_weights<T>(f[0], a, w, w_at);
            times_weights<T>(f[1], a, w, w_at + step);
          }
          w_at += (int64_t)a.chunks * 8 << a.log_hl;
        }
        rotate(f);
        if (in) {
          if (live0) store8<T>(y, f[0]);
          if (live1) store8<T>(y + step, f[1]);
        }
        y += sy;
      }
      i0 += kKeep;
      if (i0 < rows) load_rows(i0);
    }
  };
  if constexpr (NORM == VC_NORM_TOKEN) {
#pragma unroll 1
    for (int t = first; t <= last; ++t) side(t);
  } else {
    side(first);
  }
}

template <typename T, int NORM>
cudaError_t launch_rot(int rot, const QkArgs& a, dim3 grid, size_t smem, cudaStream_t s) {
  if (rot == VC_ROTARY_NONE) return launch_overlapped(qk_norm_kernel<T, NORM, VC_ROTARY_NONE>, grid, kThreads, smem, s, a);
  if (rot == VC_ROTARY_INTERLEAVED) return launch_overlapped(qk_norm_kernel<T, NORM, VC_ROTARY_INTERLEAVED>, grid, kThreads, smem, s, a);
  if (rot == kRotaryWhole) return launch_overlapped(qk_norm_kernel<T, NORM, kRotaryWhole>, grid, kThreads, smem, s, a);
  return launch_overlapped(qk_norm_kernel<T, NORM, VC_ROTARY_HALF>, grid, kThreads, smem, s, a);
}
template <typename T>
cudaError_t launch_norm(int norm, int rot, const QkArgs& a, dim3 grid, size_t smem, cudaStream_t s) {
  if (norm == VC_NORM_NONE) return launch_rot<T, VC_NORM_NONE>(rot, a, grid, smem, s);
  if (norm == VC_NORM_HEAD) return launch_rot<T, VC_NORM_HEAD>(rot, a, grid, smem, s);
  return launch_rot<T, VC_NORM_TOKEN>(rot, a, grid, smem, s);
}

constexpr double kTwoPi = 6.283185307179586476925286766559;

// v^n for n >= 1, off by n 2^-64 of itself at most in 64 bits of fraction.
long double whole_power(long double v, int n) {
  long double r = 1;
  for (; n > 1; n >>= 1, v *= v)
    if (n & 1) r *= v;
  return r * v;
}

// Frequencies of an axis's pairs in turns per position, in long double (64 bits of fraction on x86: in double they alone turn position 2^31
// by 2^-25).  Powers by repeated multiplication, one call of pow() instead of one a pair, in double and made exact by a step of Newton's method towards
// ratio^pairs base = 1: three axes of 64 pairs together take 0.8 us of host time, as in double (with pow() in long double 1.7; one such call a pair 23).  Pair i
// is off by (2 i + 8) 2^-64 of its frequency at most, the fixed point by another 2^-64 of a turn.
bool axis_frequencies(const vc_qk_params* p, int n, double factor, int original, double theta, uint64_t* out) {
  if (n == 0) return true;
  const int pairs = n / 2;
  long double base = theta;
  if (p->rope_scaling == VC_ROPE_SCALING_NTK && n > 2 && factor != 1.0) base *= std::pow((long double)factor, (long double)n / (n - 2));
  if (!(base > 0) || !std::isfinite((double)base)) return false;
  const long double near = std::pow((double)base, -2.0 / n);
  const long double ratio = near - near * (whole_power(near, pairs) * base - 1) / pairs;
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
  long double f = 0.159154943091895335768883763372514362L;      // 1 / (2 pi)
  for (int i = 0; i < pairs; ++i, f *= ratio) {
    long double v = f;
    if (p->rope_scaling == VC_ROPE_SCALING_LINEAR) v /= factor;
    if (p->rope_scaling == VC_ROPE_SCALING_YARN) {
      long double r = ((long double)i - lo) / ((long double)hi - lo);
      r = r < 0 ? 0 : (r > 1 ? 1 : r);
      v = v * (1 - r) + v / factor * r;
    }
    if (v >= 1) v -= std::floor(v);
    out[i] = (uint64_t)(v * 18446744073709551616.0L);           // (2^64; exact, and below it: v is below 1)
  }
  return true;
}

bool not_positive(double v) { return v != 0.0 && !(v > 0.0 && std::isfinite(v)); }

vc_status qk_norm_rope(const vc_qk_params* p, const vc_rope_values& rope, const void* q, const void* k, const void* q_weight, const void* k_weight,
                       const int32_t* positions, void* q_out, void* k_out, void* stream) {
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
    a.inv_count[t] = 1.0f / ((float)p->d * (p->norm == VC_NORM_TOKEN && side[t].H ? side[t].H : 1));
    if (side[t].H == 0) continue;
    if (!side[t].x || !side[t].y || misaligned16(side[t].x) || misaligned16(side[t].y) || misaligned16(side[t].w)) return VC_ERR_INVALID_ARG;
    if (!resolve_strides(*side[t].in, p->B, side[t].H, p->N, p->d, es, false, &a.in[t]) ||
        !resolve_strides(*side[t].out, p->B, side[t].H, p->N, p->d, es, true, &a.out[t]))
      return VC_ERR_INVALID_ARG;
    if (side[t].x == side[t].y && (a.in[t].b != a.out[t].b || a.in[t].h != a.out[t].h || a.in[t].n != a.out[t].n)) return VC_ERR_INVALID_ARG;
    a.x[t] = side[t].x; a.y[t] = side[t].y;
    a.w[t] = p->norm == VC_NORM_NONE ? nullptr : side[t].w;
  }
  int rot = p->rotary;
  if (rot != VC_ROTARY_NONE) {
    int dims[3] = {p->rope_dim_t, p->rope_dim_h, p->rope_dim_w};
    if (!dims[0] && !dims[1] && !dims[2]) { dims[1] = dims[2] = 2 * (p->d / 6); dims[0] = p->d - 2 * dims[1]; }
    const double factors[3] = {rope.factor_t, rope.factor_h, rope.factor_w};
    const int original[3] = {p->rope_original_t, p->rope_original_h, p->rope_original_w};
    const double theta = rope.theta != 0.0 ? rope.theta : 10000.0;
    if (!(theta > 1.0) || !std::isfinite(theta)) return VC_ERR_INVALID_ARG;
    if (p->rope_scaling < VC_ROPE_SCALING_NONE || p->rope_scaling > VC_ROPE_SCALING_YARN) return VC_ERR_INVALID_ARG;
    if (not_positive(p->yarn_beta_fast) || not_positive(p->yarn_beta_slow) || not_positive(p->rope_attention_factor)) return VC_ERR_INVALID_ARG;
    double largest = 1.0;
    int pairs = 0;
    for (int i = 0; i < 3; ++i) {
      if (dims[i] < 0 || dims[i] % 2 || dims[i] > p->d || not_positive(factors[i])) return VC_ERR_INVALID_ARG;
      if (2 * pairs + dims[i] > p->d) return VC_ERR_INVALID_ARG;
      const double factor = factors[i] != 0.0 ? factors[i] : 1.0;
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
      a.inv_h = 1.0f / p->grid_h; a.inv_w = 1.0f / p->grid_w;
      for (int i = 0; i < 3; ++i) a.start[i] = start[i];
    }
    a.positions = positions;
    if (pairs == 0) rot = VC_ROTARY_NONE;
    if (rot == VC_ROTARY_HALF && dims[0] % 16 == 0 && dims[1] % 16 == 0 && dims[2] % 16 == 0) rot = kRotaryWhole;
  }
  a.N = p->N;
  a.chunks = p->d / 8;
  a.same_type = p->weight_dtype == p->dtype;
  a.partial = 2 * a.pairs < p->d;
  a.weight_dtype = p->weight_dtype;
  a.eps = p->eps != 0.f ? p->eps : 1e-6f;
  while ((2 << a.log_lanes) < a.chunks) ++a.log_lanes;
  for (int i = 0; i < 16; ++i) {
    const int lanes = 1 << a.log_lanes;
    a.lo[i] = (uint8_t)(i < lanes && i < a.chunks ? i : 255);
    a.hi[i] = (uint8_t)(i < lanes && i + lanes < a.chunks ? i + lanes : 255);
    a.first_pair[i] = 255;
  }
  if (rot == kRotaryWhole) {                 // lanes for the pairs of every axis, then for the channels behind them
    int lane = 0, chunk = 0, pair = 0;
    for (int axis = 0; axis < 3; ++axis) {
      const int groups = (a.pair_end[axis] - pair) / 8;
      for (int i = 0; i < groups; ++i, ++lane, pair += 8) {
        a.lo[lane] = (uint8_t)(chunk + i); a.hi[lane] = (uint8_t)(chunk + groups + i); a.first_pair[lane] = (uint8_t)pair;
      }
      chunk += 2 * groups;
    }
    for (; lane < 16; ++lane, chunk += 2) {
      a.lo[lane] = (uint8_t)(chunk < a.chunks ? chunk : 255); a.hi[lane] = (uint8_t)(chunk + 1 < a.chunks ? chunk + 1 : 255);
      a.first_pair[lane] = 255;
    }
  }
  const int rows = kThreads >> a.log_lanes, heads = a.H[0] > a.H[1] ? a.H[0] : a.H[1], keep = heads_held(es, rot);
  const int tensors = (a.H[0] > 0) + (a.H[1] > 0);
  a.first = a.H[0] == 0;
  while ((1 << a.log_pairs) < a.pairs) ++a.log_pairs;
  // Rows of a CTA side by side: `1 << log_hl` heads of each token.  The norm over a token takes as many as bring the heads that
  // a thread holds down to `keep`; beyond that as many as leave four CTAs an SM, or a short sequence without a token.
  auto ctas = [&] { return (int64_t)p->B * tensors * ((p->N + (rows >> a.log_hl) - 1) / (rows >> a.log_hl)); };
  while ((1 << a.log_hl) < rows && ((p->norm == VC_NORM_TOKEN && heads > keep << a.log_hl) || (heads >= 2 << a.log_hl && ctas() < 4 * sm_count()) ||
                                    (rows >> a.log_hl) >= 2 * p->N))
    ++a.log_hl;
  const int tokens = rows >> a.log_hl, tiles = (p->N + tokens - 1) / tokens;
  // Long sequences under the norm over a token: one table of angles for Q and K (12 + 12 heads x 32760 x 128 99.9 -> 91.8 us; with the norm
  // per head, where a CTA's phases are shorter, 85.2 -> 88.5).
  a.both = p->norm == VC_NORM_TOKEN && tensors == 2 && (int64_t)p->B * tiles >= 16 * sm_count();
  const dim3 grid((unsigned)tiles, (unsigned)p->B, a.both ? 1u : (unsigned)tensors);
  const size_t smem = rot == VC_ROTARY_NONE ? 0 : (size_t)tokens * a.pairs * sizeof(float2);
  cudaStream_t s = (cudaStream_t)stream;
  const cudaError_t e = p->dtype == VC_DTYPE_BF16   ? launch_norm<__nv_bfloat16>(p->norm, rot, a, grid, smem, s)
                        : p->dtype == VC_DTYPE_FP16 ? launch_norm<__half>(p->norm, rot, a, grid, smem, s)
                                                    : launch_norm<float>(p->norm, rot, a, grid, smem, s);
  if (e != cudaSuccess) return VC_ERR_CUDA;
  count_launches(1);
  return VC_OK;
}

}  // namespace
}  // namespace vc

using namespace vc;

extern "C" vc_status vc_qk_norm_rope_with_values(const vc_qk_params* p, const vc_rope_values* rope, const void* q, const void* k, const void* q_weight,
                                                 const void* k_weight, const int32_t* positions, void* q_out, void* k_out, void* stream) {
  if (!p) return VC_ERR_INVALID_ARG;
  vc_rope_values v = {p->rope_theta, p->rope_factor_t, p->rope_factor_h, p->rope_factor_w};
  if (rope) {
    if (rope->theta != 0.0) v.theta = rope->theta;
    if (rope->factor_t != 0.0) v.factor_t = rope->factor_t;
    if (rope->factor_h != 0.0) v.factor_h = rope->factor_h;
    if (rope->factor_w != 0.0) v.factor_w = rope->factor_w;
  }
  return qk_norm_rope(p, v, q, k, q_weight, k_weight, positions, q_out, k_out, stream);
}

extern "C" vc_status vc_qk_norm_rope(const vc_qk_params* p, const void* q, const void* k, const void* q_weight,
                                     const void* k_weight, const int32_t* positions, void* q_out, void* k_out, void* stream) {
  return vc_qk_norm_rope_with_values(p, nullptr, q, k, q_weight, k_weight, positions, q_out, k_out, stream);
}
