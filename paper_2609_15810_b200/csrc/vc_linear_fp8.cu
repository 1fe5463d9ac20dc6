// vc_linear_fp8: product of two E4M3 matrices with an FP32 scale per block of 128, on the tensor cores.
//
//   y[m][n] = sum_kb xs[kb][m] ws[n / 128][kb] S_kb[m][n] + bias[n],   S_kb = the product over the block's 128 columns
//
// The scales are arbitrary FP32 numbers and differ from block to block of the common width, so no accumulator can run over
// blocks: each S_kb is a product of its own (4 instructions of 32 columns into a tensor-memory buffer) and two
// warpgroups add it, scaled, to sums in registers, 128 columns of a row a thread at most.  The two scales are multiplied first: one FMA an element.
// (Scales whose product FP32 does not hold, applied one after the other behind a test per block: right, but 737 -> 763 us at 32760 x 5120 x 5120, and
// 11.1 -> 11.9 at 64 rows; the header asks for products that it holds.)
//
// Three shapes: tiles of 256 x 256 by two CTAs of a cluster (each 128 rows of A and half of B in shared memory, 128 rows of sums), where
// these fill the SMs; tiles of 128 x 128; and up to 64 rows of x as B with 128 weight rows as A, which is bound by reading the weights.  With
// fewer tiles than SMs the blocks of K are split between CTAs and the parts joined in a fixed order: up to 64 rows by a cluster of the CTAs, from shared
// memory, else by a second launch.
//
// What bounds the large ones: a block takes 836 cycles, at any clock (clock reads around the waits in a scratch build): an adding warp reads and adds
// for 505 of them and waits 221 for the product, a tile's end comes to 110 (4400 a tile of 40 blocks).  The tensor cores need 512, but there are two buffers
// only (256 columns each of 512): an issuing warp waits for its buffer to be free for half of its time, 844 of 1670 cycles a buffer.
// 32760 x 5120 x 5120 is 1.175e6 cycles: 726-743 us in the first ten calls (1.6 GHz), 840-855 behind a hundred (1.38 GHz, the power cap).
// Tried (first calls / behind many): a CTA by itself on 128 x 256 (48 KB copied and 48 KB read per block and 512 cycles
// from a shared memory that gives 128 bytes a cycle) 808 / 880 us; one issuing warp instead of two that take every other block (a group of products
// begins 150 cycles behind the end of the one in front if the same warp issued it) 781, and the same under the cap; four buffers of
// 128 columns (two products of 256 x 128 a block, A read twice) 794 / 868; a release or acquire of
// cluster scope at the buffers' barriers 1490 (it waits for every load in flight); packed additions 860 (a move and a half each, the products
// arrive in registers that do not pair up); four warpgroups of 64 columns, scales four blocks ahead: no gain.
// The 256 x 256 form spills 164 bytes of stores and 80 of loads a thread; builds with 92 and 100, and with 68 and 52, were 2 % slower.
// 5120 x 5120 with weights in L2: one row 7.8 us (26 MB at the copy rate 4.0), 64 rows 11, 512 rows 22, 1024 rows 40, 2048 rows 62: from 65 rows to
// some thousands whole tiles leave SMs without work (512 rows: 40 tiles of a pair on 74 pairs; 1024: 320 of a CTA, two rounds and 24 more).
#include "vc_attn_shared.cuh"
#include "vc_layer.cuh"
#include "vc_sm100.cuh"

namespace vc {
namespace {

using namespace layer;
using namespace sm100;

constexpr int kThreads = 384;
constexpr int kCluster = 8;                  // CTAs of a portable cluster
constexpr int kSms = 148;                    // what the rule for splits counts on: the workspace's size must not vary

struct LinearArgs {
  const float *xs, *ws;
  const void* bias;
  void* out;
  float* part;                               // [splits][M][ldp]
  uint32_t* status;
  int64_t ldo, ldp;
  int M, N, blocks, tiles_b, splits, items;  // blocks: of 128 columns of K; tiles_b: tiles along B
  int out_dtype, bias_dtype;
  bool vec;                                  // rows of out start on 16-byte boundaries
  bool copies;                               // and end on them: they leave by TMA
  bool joined;                               // the CTAs of a tile's splits are a cluster and join their sums themselves
  uint32_t limit, nonblocking;
};

// SWAP: A = weights (128 rows), B = TN rows of x.  Else A = 128 rows of x, B = TN weights.
// TN 256: two CTAs of a cluster work on a tile of 256 x 256, each with 128 rows of A and, in shared memory, half of B.
template <bool SWAP, int TN> struct Cfg {
  static constexpr bool kPair = TN == 256;
  static constexpr int kGroups = TN >= 128 ? 2 : 1;            // warpgroups that add
  static constexpr int kCols = TN / kGroups;                   // columns of a thread
  static constexpr int kBufs = TN == 256 ? 2 : 4;
  static constexpr int kTmem = kBufs * TN;                     // 512, 512, 256, 64
  static constexpr uint32_t kA = 128 * 128, kB = (kPair ? TN / 2 : TN) * 128, kStage = kA + kB;
  static constexpr int kStages = TN >= 128 ? 6 : 8;
  static constexpr uint32_t kOut = SWAP ? 0 : 8 * 32 * 128;    // 128 bytes of each warp's 32 rows
};

template <int STAGES, int BUFS> struct Smem {
  uint64_t full[STAGES], empty[STAGES], acc_full[BUFS], acc_free[BUFS], drain[2];
  uint32_t tmem_base;
  volatile int abort;
  float touched[32];                         // (never read)
};

template <class S>
__device__ __forceinline__ bool wait(uint64_t* bar, uint32_t parity, S* sh, const LinearArgs& a, uint32_t code) {
  if (__all_sync(0xffffffffu, mbar_test_wait(bar, parity))) return true;
#pragma unroll 1
  for (uint32_t i = 0; i < a.limit; ++i) {
    if (__all_sync(0xffffffffu, a.nonblocking ? mbar_test_wait(bar, parity) : mbar_try_wait(bar, parity))) return true;
    if ((i & 63u) == 63u && __any_sync(0xffffffffu, sh->abort)) return false;
  }
  sh->abort = 1;
  __nanosleep(20000);                        // (CTA 0 clears the word when it starts)
  atomicExch(a.status, kStatusTimeout | code);
  return false;
}

__device__ __forceinline__ void tma_load_2d(void* dst, const CUtensorMap* m, uint64_t* bar, int c0, int c1) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(smem_u32(dst)),
               "l"(reinterpret_cast<uint64_t>(m)), "r"(smem_u32(bar)), "r"(c0), "r"(c1)
               : "memory");
}

// A pair of CTAs: the copy counts at a barrier of the leader's (`bar` is an address in the cluster), the product reads both
// CTAs' shared memory and writes both CTAs' tensor memory, and its completion counts at the barrier of both.
__device__ __forceinline__ void tma_load_2d_pair(void* dst, const CUtensorMap* m, uint32_t bar, int c0, int c1) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%3, %4}], [%2];" ::"r"(smem_u32(dst)),
               "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(c0), "r"(c1)
               : "memory");
}
__device__ __forceinline__ void mma_f8_pair(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
               "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
               : "memory");
}
__device__ __forceinline__ void mma_commit_leader(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void mma_commit_pair(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)), "h"((uint16_t)3) : "memory");
}
__device__ __forceinline__ uint32_t in_leader(const void* p) {       // the address of the leader's copy of `p`
  uint32_t at;
  asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(at) : "r"(smem_u32(p)));
  return at;
}
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ float4 load_cluster(const float4* p, int rank) {    // from the same place of the cluster's CTA `rank`
  uint32_t at;
  float4 v;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(p)), "r"(rank));
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}

struct Item { int a0, b0, split, kb0, kb1; };                  // first rows in A (this CTA's) and B (the tile's); blocks of K
template <int TN> __device__ __forceinline__ Item item_of(const LinearArgs& a, int idx, int rank) {
  Item w;
  const int tile = idx / a.splits, ta = tile / a.tiles_b;
  w.split = idx - tile * a.splits;
  w.a0 = TN == 256 ? ta * 256 + rank * 128 : ta * 128;
  w.b0 = (tile - ta * a.tiles_b) * TN;
  w.kb0 = (int)((int64_t)a.blocks * w.split / a.splits);
  w.kb1 = (int)((int64_t)a.blocks * (w.split + 1) / a.splits);
  return w;
}

// The warp's 32 rows of `COLS` FP32 sums -> rows of O in memory, 128 bytes of each at a time through shared memory.
template <typename O> __device__ __forceinline__ uint4 pack_chunk(const float* f);
template <> __device__ __forceinline__ uint4 pack_chunk<float>(const float* f) {
  return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}
template <> __device__ __forceinline__ uint4 pack_chunk<__nv_bfloat16>(const float* f) {
  return make_uint4(pack16<__nv_bfloat16>(f[0], f[1]), pack16<__nv_bfloat16>(f[2], f[3]), pack16<__nv_bfloat16>(f[4], f[5]), pack16<__nv_bfloat16>(f[6], f[7]));
}
template <> __device__ __forceinline__ uint4 pack_chunk<__half>(const float* f) {
  return make_uint4(pack16<__half>(f[0], f[1]), pack16<__half>(f[2], f[3]), pack16<__half>(f[4], f[5]), pack16<__half>(f[6], f[7]));
}
// The same as one copy of the warp's 32 rows at a time, where rows of `out` start and end on 16-byte boundaries; what lies outside of it the copy
// leaves out.  (It leaves out 16 bytes at a time: behind a row that ends in between it writes zeros up to the boundary.)
template <typename O, int COLS>
__device__ __forceinline__ void emit_copies(const float (&y)[COLS], uint32_t tile, const CUtensorMap* map, int col0, int row0, int rows, int lane) {
  using Out = attn::OutTile<64>;
  constexpr int kPer = 16 / sizeof(O), kPass = 8 * kPer;
#pragma unroll
  for (int p = 0; p < COLS / kPass; ++p) {
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");        // the copy in front has read the tile
    __syncwarp();
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      const uint4 v = pack_chunk<O>(y + p * kPass + c * kPer);
      sts128(Out::chunk(tile, lane, c), v.x, v.y, v.z, v.w);
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0 && rows > 0) {
      asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];" ::"l"(reinterpret_cast<uint64_t>(map)), "r"(tile),
                   "r"(col0 + p * kPass), "r"(row0)
                   : "memory");
      asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
  }
}
template <typename O, int COLS>
__device__ __forceinline__ void emit_rows(const float (&y)[COLS], uint32_t tile, O* dst, int64_t ld, int rows, int cols, bool vec, int lane) {
  using Out = attn::OutTile<64>;                               // (128 bytes a row, whatever the type)
  constexpr int kPer = 16 / sizeof(O), kPass = 8 * kPer;       // elements of 16 and of 128 bytes
#pragma unroll
  for (int p = 0; p < COLS / kPass; ++p) {
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      const uint4 v = pack_chunk<O>(y + p * kPass + c * kPer);
      sts128(Out::chunk(tile, lane, c), v.x, v.y, v.z, v.w);
    }
    __syncwarp();
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int r = 4 * k + (lane >> 3), c = lane & 7, col = p * kPass + c * kPer;
      if (r < rows && col < cols) {
        const float4 v = lds128(Out::chunk(tile, r, c));
        O* at = dst + r * ld + col;
        if (vec && col + kPer <= cols) {
          *reinterpret_cast<float4*>(at) = v;
        } else {
          const O* e = reinterpret_cast<const O*>(&v);
#pragma unroll
          for (int i = 0; i < kPer; ++i)
            if (col + i < cols) at[i] = e[i];
        }
      }
    }
    __syncwarp();
  }
}

template <bool SWAP, int TN>
__global__ void __launch_bounds__(kThreads, 1)
linear_fp8_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_b,
                  const __grid_constant__ CUtensorMap tm_o, const __grid_constant__ LinearArgs a) {
  using C = Cfg<SWAP, TN>;
  using S = Smem<C::kStages, C::kBufs>;
  constexpr int kRegAdd = 216, kRegCtl = 72;
  static_assert(2 * kRegAdd + kRegCtl <= 3 * 168, "register budget exceeds the CTA's allocation");
  static_assert(C::kStages * C::kStage + C::kOut + sizeof(S) <= 227 * 1024, "shared memory of the kernel exceeds the SM");
  extern __shared__ __align__(1024) unsigned char smem[];
  unsigned char* sOut = smem + C::kStages * C::kStage;
  S* sh = reinterpret_cast<S*>(sOut + C::kOut);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = C::kPair ? blockIdx.x & 1 : 0, first = C::kPair ? blockIdx.x >> 1 : blockIdx.x, stride = C::kPair ? gridDim.x >> 1 : gridDim.x;
  if (tid == 0) {
    for (int i = 0; i < C::kStages; ++i) { mbar_init(&sh->full[i], 1); mbar_init(&sh->empty[i], 1); }
    for (int i = 0; i < C::kBufs; ++i) { mbar_init(&sh->acc_full[i], 1); mbar_init(&sh->acc_free[i], C::kPair ? 16 : 128 * C::kGroups); }
    mbar_init(&sh->drain[0], 1); mbar_init(&sh->drain[1], 1);
    sh->abort = 0;
    mbar_fence_init();
    tma_prefetch_desc(&tm_a); tma_prefetch_desc(&tm_b);
  }
  pdl_wait();
  if (warp == 10) {
    if constexpr (C::kPair) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh->tmem_base)), "n"(C::kTmem) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      tmem_alloc<C::kTmem>(&sh->tmem_base);
      tmem_relinquish();
    }
  }
  if (tid == 0 && blockIdx.x == 0) *a.status = 0;
  if (a.splits > 1 && !a.joined) pdl_allow();               // (what follows then is the launch that joins the parts: it may stand by)
  tc_fence_before();
  if constexpr (C::kPair) cluster_sync(); else __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sh->tmem_base;

  if (warp >= 8) {
    reg_dec<kRegCtl>();
    if (warp == 8) {
      // -------------------------------------------------------------------------------- loads
      int n = 0;
      bool ok = true;
      const uint32_t full = in_leader(&sh->full[0]);
      for (int idx = first; ok && idx < a.items; idx += stride) {
        const Item w = item_of<TN>(a, idx, rank);
        for (int kb = w.kb0; kb < w.kb1; ++kb, ++n) {
          const int st = n % C::kStages;
          if (!(ok = wait(&sh->empty[st], ((n / C::kStages) & 1) ^ 1, sh, a, 1))) break;
          if (elect_one()) {
            unsigned char* base = smem + st * C::kStage;
            if constexpr (C::kPair) {
              if (rank == 0) mbar_expect_tx(&sh->full[st], 2 * C::kStage);
              tma_load_2d_pair(base, &tm_a, full + 8 * st, kb * 128, w.a0);
              tma_load_2d_pair(base + C::kA, &tm_b, full + 8 * st, kb * 128, w.b0 + 128 * rank);
            } else {
              mbar_expect_tx(&sh->full[st], C::kStage);
              tma_load_2d(base, &tm_a, &sh->full[st], kb * 128, w.a0);
              tma_load_2d(base + C::kA, &tm_b, &sh->full[st], kb * 128, w.b0);
            }
          }
          __syncwarp();
          // The block's scales into the first-level cache: the adding warps fetch them one block ahead, less than the latency of L2
          // (257 x 5120 x 13824 48.5 -> 35.9 us, 8192 x 5120 x 5120 196 -> 187; two or four blocks ahead into registers: 37, and others +5 %).
          const float* scale = lane < 17 ? a.xs + (int64_t)kb * a.M + min((SWAP ? w.b0 : w.a0) + min(8 * lane, SWAP ? TN - 1 : 127), a.M - 1)
                                         : a.ws + (int64_t)min(((SWAP ? w.a0 : w.b0) >> 7) + (lane & 1), (a.N - 1) >> 7) * a.blocks + kb;
          asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(&sh->touched[lane])), "l"(scale) : "memory");
        }
      }
      asm volatile("cp.async.wait_all;" ::: "memory");
      // Every copy issued has landed before the CTA may end (at once on a normal run).  A pair's land at the leader's barriers: what
      // says so in both is that they have been read; where a wait has given up, time.
      if constexpr (C::kPair) {
        for (int i = n > C::kStages ? n - C::kStages : 0; ok && i < n; ++i) ok = wait(&sh->empty[i % C::kStages], (i / C::kStages) & 1, sh, a, 2);
        if (!ok)
          for (int i = 0; i < 10; ++i) __nanosleep(20000);
      } else
      for (int i = n > C::kStages ? n - C::kStages : 0; i < n; ++i) mbar_wait(&sh->full[i % C::kStages], (i / C::kStages) & 1, attn::kDrainLimit);
    } else if ((warp == 9 || warp == 11) && rank == 0) {
      // -------------------------------------------------------------------------------- products: two warps, every other block each
      const int mine = warp >> 1 & 1;
      constexpr uint32_t idesc = idesc_e4m3(C::kPair ? 256 : 128, TN);
      int n = 0;
      bool ok = true;
      for (int idx = first; ok && idx < a.items; idx += stride) {
        const Item w = item_of<TN>(a, idx, rank);
        for (int kb = w.kb0; kb < w.kb1; ++kb, ++n) {
          if ((n & 1) != mine) continue;             // (stages and buffers are even in number: each has one of the warps)
          const int st = n % C::kStages, buf = n % C::kBufs;
          if (!(ok = wait(&sh->full[st], (n / C::kStages) & 1, sh, a, 10)) || !(ok = wait(&sh->acc_free[buf], ((n / C::kBufs) & 1) ^ 1, sh, a, 11))) break;
          if (elect_one()) {
            tc_fence_after();
            const uint64_t da = smem_desc_kmajor(smem_u32(smem + st * C::kStage), 128), db = smem_desc_kmajor(smem_u32(smem + st * C::kStage + C::kA), 128);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              if constexpr (C::kPair) mma_f8_pair(tmem + buf * TN, da + 2 * k, db + 2 * k, idesc, k > 0);
              else mma_f8_ss(tmem + buf * TN, da + 2 * k, db + 2 * k, idesc, k > 0);
            }
            if constexpr (C::kPair) {
              mma_commit_pair(&sh->empty[st]);
              mma_commit_pair(&sh->acc_full[buf]);
            } else {
              mma_commit(&sh->empty[st]);
              mma_commit(&sh->acc_full[buf]);
            }
          }
          __syncwarp();
        }
      }
      if (elect_one()) {
        if constexpr (C::kPair) mma_commit_leader(&sh->drain[mine]); else mma_commit(&sh->drain[mine]);
      }
      __syncwarp();
      mbar_wait(&sh->drain[mine], 0, attn::kDrainLimit);
    }
  } else if (warp < 4 * C::kGroups) {
    // ---------------------------------------------------------------------------------- sums
    reg_inc<kRegAdd>();
    constexpr int kCols = C::kCols, kChunk = kCols < 32 ? kCols : 32, kChunks = kCols / kChunk;
    const int group = warp >> 2, row = (warp & 3) * 32 + lane;
    const uint32_t lane_base = tmem + ((uint32_t)((warp & 3) * 32) << 16) + group * kCols;
    constexpr int kBias = SWAP ? 1 : (kCols + 31) / 32;
    const bool whole = a.splits == 1;
    // An item's scales (of one block of K) and biases, fetched ahead: while the block in front is added, or the item in front written.
    // xa: of my row, or (SWAP) of row `lane` of my columns, xb of row 32 + lane; bias: of my columns lane, 32 + lane, ..., or (SWAP) of my row.
    float xa = 0.f, xb = 0.f, wv = 0.f, bias[kBias] = {};
    int xb_at = 0;
    const float *xp = a.xs, *wp = a.ws;                        // where the next block's are (of a row outside: any, never stored)
    auto fetch = [&] {
      if (!SWAP || lane < kCols) xa = __ldg(xp);
      if constexpr (SWAP && kCols > 32) xb = __ldg(xp + xb_at);
      wv = __ldg(wp);
      xp += a.M;
      ++wp;
    };
    auto fetch_item = [&](const Item& w) {
      const int m = SWAP ? w.b0 + lane : w.a0 + row;
      const int n0 = SWAP ? w.a0 : w.b0 + group * kCols;       // my (first) weight row; all of mine lie in its block of 128
      xp = a.xs + (int64_t)w.kb0 * a.M + min(m, a.M - 1);
      xb_at = min(m + 32, a.M - 1) - min(m, a.M - 1);
      wp = a.ws + (int64_t)min(n0 >> 7, (a.N - 1) >> 7) * a.blocks + w.kb0;
      fetch();
      if (whole && a.bias) {
#pragma unroll
        for (int i = 0; i < kBias; ++i) {
          const int col = SWAP ? w.a0 + row : w.b0 + group * kCols + 32 * i + lane;
          bias[i] = col < a.N ? load1(a.bias, a.bias_dtype, col) : 0.f;
        }
      }
    };
    int n = 0;
    bool ok = true;
    const uint32_t acc_free = in_leader(&sh->acc_free[0]);
    Item w = item_of<TN>(a, first, rank);
    fetch_item(w);
    for (int idx = first; ok && idx < a.items; idx += stride) {
      float y[kCols];
#pragma unroll
      for (int i = 0; i < kCols; ++i) y[i] = 0.f;
      const int m0 = SWAP ? w.b0 : w.a0 + row, n0 = SWAP ? w.a0 : w.b0 + group * kCols;
      for (int kb = w.kb0; kb < w.kb1; ++kb, ++n) {
        const int buf = n % C::kBufs;
        const float fa = xa * wv, fb = xb * wv;
        if (kb + 1 < w.kb1) fetch();
        if (!(ok = wait(&sh->acc_full[buf], (n / C::kBufs) & 1, sh, a, 20))) break;
        tc_fence_after();
        const uint32_t at = lane_base + buf * TN;
        uint32_t r[2][kChunk];
        auto load = [&](int c) {
          if constexpr (kChunk == 32) tmem_ld32(at + 32 * c, r[c & 1]);
          else tmem_ld16(at, r[c & 1]);
        };
        load(0);
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
          tmem_wait_ld();
          if (c + 1 < kChunks) {
            load(c + 1);
          } else {
            tc_fence_before();
            if constexpr (C::kPair) {
              __syncwarp();
              if (lane == 0) mbar_arrive_cluster(acc_free + 8 * buf);
            } else {
              mbar_arrive(&sh->acc_free[buf]);
            }
          }
#pragma unroll
          for (int i = 0; i < kChunk; ++i) {
            float f = fa;
            if constexpr (SWAP) f = __shfl_sync(0xffffffffu, c == 0 ? fa : fb, i);
            y[c * kChunk + i] = fmaf(__uint_as_float(r[c & 1][i]), f, y[c * kChunk + i]);
          }
        }
      }
      if (!ok) break;
      float mine[kBias];
#pragma unroll
      for (int i = 0; i < kBias; ++i) mine[i] = bias[i];
      const Item now = w;
      if (idx + stride < a.items) {
        w = item_of<TN>(a, idx + stride, rank);
        fetch_item(w);
      }
      if constexpr (SWAP) {
        const int col = now.a0 + row;
        if (a.joined) {                            // (the last product is complete: the stages are free)
#pragma unroll
          for (int i = 0; i < kCols; ++i) reinterpret_cast<float*>(smem)[i * 128 + row] = y[i];
        } else if (col < a.N) {
#pragma unroll
          for (int i = 0; i < kCols; ++i) {
            if (m0 + i >= a.M) break;
            const float v = y[i] + mine[0];
            if (!whole) a.part[((int64_t)now.split * a.M + m0 + i) * a.ldp + col] = v;
            else if (a.out_dtype == VC_DTYPE_BF16) static_cast<__nv_bfloat16*>(a.out)[(m0 + i) * a.ldo + col] = __float2bfloat16_rn(v);
            else if (a.out_dtype == VC_DTYPE_FP16) static_cast<__half*>(a.out)[(m0 + i) * a.ldo + col] = __float2half_rn(v);
            else static_cast<float*>(a.out)[(m0 + i) * a.ldo + col] = v;
          }
        }
      } else {
        const int row0 = now.a0 + (warp & 3) * 32, rows = min(32, a.M - row0), cols = min(kCols, a.N - n0);
        const uint32_t tile = smem_u32(sOut) + warp * 4096;
        if (whole && a.bias) {
#pragma unroll
          for (int i = 0; i < kCols; ++i) y[i] += __shfl_sync(0xffffffffu, mine[i / 32], i % 32);
        }
        if (whole && a.copies) {
          if (a.out_dtype == VC_DTYPE_BF16) emit_copies<__nv_bfloat16, kCols>(y, tile, &tm_o, n0, row0, cols > 0 ? rows : 0, lane);
          else if (a.out_dtype == VC_DTYPE_FP16) emit_copies<__half, kCols>(y, tile, &tm_o, n0, row0, cols > 0 ? rows : 0, lane);
          else emit_copies<float, kCols>(y, tile, &tm_o, n0, row0, cols > 0 ? rows : 0, lane);
          continue;
        }
        if (!whole) emit_rows<float, kCols>(y, tile, a.part + ((int64_t)now.split * a.M + row0) * a.ldp + n0, a.ldp, rows, cols, true, lane);
        else if (a.out_dtype == VC_DTYPE_BF16) emit_rows<__nv_bfloat16, kCols>(y, tile, static_cast<__nv_bfloat16*>(a.out) + row0 * a.ldo + n0, a.ldo, rows, cols, a.vec, lane);
        else if (a.out_dtype == VC_DTYPE_FP16) emit_rows<__half, kCols>(y, tile, static_cast<__half*>(a.out) + row0 * a.ldo + n0, a.ldo, rows, cols, a.vec, lane);
        else emit_rows<float, kCols>(y, tile, static_cast<float*>(a.out) + row0 * a.ldo + n0, a.ldo, rows, cols, a.vec, lane);
      }
    }
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");       // the rows have left shared memory before the CTA may end
  }
  tc_fence_before();
  if (SWAP && a.joined) {
    // A sum's parts in the order of the splits, from the shared memory of the cluster's CTAs, each of which takes some of the sums.
    const Item w = item_of<TN>(a, first, rank);
    const int rows = min(TN, a.M - w.b0);
    cluster_sync();
    for (int e = w.split * kThreads + tid; e < rows * 32; e += a.splits * kThreads) {        // four columns of a row
      const int col = w.a0 + 4 * (e & 31);
      if (col >= a.N) continue;
      float4 v[kCluster];
      float y[4] = {};
#pragma unroll
      for (int i = 0; i < kCluster; ++i)
        if (i < a.splits) v[i] = load_cluster(reinterpret_cast<const float4*>(smem) + e, i);
#pragma unroll
      for (int i = 0; i < kCluster; ++i)
        if (i < a.splits) { y[0] += v[i].x; y[1] += v[i].y; y[2] += v[i].z; y[3] += v[i].w; }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (col + j >= a.N) break;
        if (a.bias) y[j] += load1(a.bias, a.bias_dtype, col + j);
        const int64_t at = (w.b0 + (e >> 5)) * a.ldo + col + j;
        if (a.out_dtype == VC_DTYPE_BF16) static_cast<__nv_bfloat16*>(a.out)[at] = __float2bfloat16_rn(y[j]);
        else if (a.out_dtype == VC_DTYPE_FP16) static_cast<__half*>(a.out)[at] = __float2half_rn(y[j]);
        else static_cast<float*>(a.out)[at] = y[j];
      }
    }
    cluster_sync();                            // (a CTA stays until its peers have read it)
    if (warp == 10) tmem_dealloc<C::kTmem>(tmem);
    return;
  }
  if constexpr (C::kPair) {
    cluster_sync();                            // (neither CTA ends, nor gives its tensor memory back, while the other's products or signals reach it)
    if (warp == 10) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(C::kTmem) : "memory");
  } else {
    __syncthreads();
    if (warp == 10) tmem_dealloc<C::kTmem>(tmem);
  }
}

// The parts of every sum in the order of the splits, the bias, the rounding.  A thread takes four columns of a row.
__global__ void __launch_bounds__(256) linear_join_kernel(const __grid_constant__ LinearArgs a) {
  pdl_wait();
  const int quads = (a.N + 3) / 4;
  const int64_t total = (int64_t)a.M * quads;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t m = i / quads;
    const int n = (int)(i - m * quads) * 4;
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s = 0; s < a.splits; ++s) {
      const float4 v = *reinterpret_cast<const float4*>(a.part + ((int64_t)s * a.M + m) * a.ldp + n);
      y.x += v.x; y.y += v.y; y.z += v.z; y.w += v.w;
    }
    const float e[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (n + j >= a.N) break;
      const float v = e[j] + (a.bias ? load1(a.bias, a.bias_dtype, n + j) : 0.f);
      if (a.out_dtype == VC_DTYPE_BF16) static_cast<__nv_bfloat16*>(a.out)[m * a.ldo + n + j] = __float2bfloat16_rn(v);
      else if (a.out_dtype == VC_DTYPE_FP16) static_cast<__half*>(a.out)[m * a.ldo + n + j] = __float2half_rn(v);
      else static_cast<float*>(a.out)[m * a.ldo + n + j] = v;
    }
  }
}

struct Plan {
  bool swap, joined;
  int tn, tiles_b, splits, blocks;
  int64_t items, ldp;
  size_t total;
};

// Clusters of n CTAs with an SM each that run side by side: eight GPCs of 18 SMs or more.
inline int clusters_at_once(int n) { return 8 * (18 / n); }

vc_status resolve(const vc_linear_params* p, vc_linear_params* out, Plan* plan) {
  if (!p) return VC_ERR_INVALID_ARG;
  vc_linear_params r = *p;
  if (r.M < 1 || r.N < 1 || r.M > (1 << 30) || r.N > (1 << 30) || r.K < 16 || r.K % 16 || r.K > (1 << 20)) return VC_ERR_INVALID_ARG;
  if (bad_dtype(r.out_dtype) || bad_dtype(r.bias_dtype) || r.k_splits < 0 || r.k_splits > 64) return VC_ERR_INVALID_ARG;
  if (r.M == 1 || r.ldx == 0) r.ldx = r.K;
  if (r.N == 1 || r.ldw == 0) r.ldw = r.K;
  if (r.M == 1 || r.ldo == 0) r.ldo = r.N;
  if (r.ldx < r.K || r.ldw < r.K || r.ldo < r.N || r.ldx % 16 || r.ldw % 16 || r.ldx >= 1ll << 38 || r.ldw >= 1ll << 38 || r.ldo >= 1ll << 32) return VC_ERR_INVALID_ARG;
  Plan pl{};
  pl.blocks = (r.K + 127) / 128;
  // Up to 64 rows: weights are A.  Else a pair of CTAs takes 0.53 us for a block of 256 x 256, a CTA 0.33 for one of 128 x 128: the shape whose
  // rounds over the SMs cost less (512 x 5120 x 5120: 40 tiles of a pair 22.2 us, 160 of a CTA 26.8; 257 x 13824 x 5120: 49.0, 41.1).
  pl.swap = r.M <= 64;
  if (pl.swap) pl.tn = r.M <= 16 ? 16 : 64;
  else {
    auto rounds = [&](int64_t t, int at_once) { return (((r.M + t - 1) / t) * ((r.N + t - 1) / t) + at_once - 1) / at_once; };
    pl.tn = 8 * rounds(256, kSms / 2) <= 5 * rounds(128, kSms) ? 256 : 128;
  }
  const int64_t ta = pl.swap ? (r.N + 127) / 128 : pl.tn == 256 ? (r.M + 255) / 256 : (r.M + 127) / 128;
  pl.tiles_b = (int)(((pl.swap ? r.M : r.N) + (int64_t)pl.tn - 1) / pl.tn);
  const int64_t tiles = ta * pl.tiles_b, ctas = pl.tn == 256 ? 2 : 1;        // (of a tile)
  pl.splits = r.k_splits;
  if (pl.splits == 0) {
    const int64_t room = kSms / (tiles * ctas);
    pl.splits = 1;
    if (room > 1 && pl.blocks >= 8) pl.splits = (int)(room < pl.blocks / 4 ? room : pl.blocks / 4);
    if (pl.swap) {                             // no more than clusters of as many CTAs find room for at a time
      if (pl.splits > kCluster) pl.splits = kCluster;
      while (pl.splits > 1 && tiles > clusters_at_once(pl.splits)) --pl.splits;
    }
  }
  if (pl.splits > pl.blocks) pl.splits = pl.blocks;
  if (pl.splits > 64) pl.splits = 64;
  // Few rows: the splits of a tile are a cluster and need no second launch (one row of 5120 x 5120 8.2 -> 7.7 us, 64 rows 11.8 -> 10.8,
  // one row of 1536 x 8960 7.8 -> 6.7).
  pl.joined = pl.swap && pl.splits > 1 && pl.splits <= kCluster && tiles <= clusters_at_once(pl.splits);
  pl.items = tiles * pl.splits;
  if (pl.items > INT32_MAX) return VC_ERR_UNSUPPORTED;
  pl.ldp = (r.N + 3) / 4 * 4ll;
  if (pl.splits > 1 && r.M * pl.ldp > 1ll << 40) return VC_ERR_UNSUPPORTED;      // (the parts' bytes stay far below 2^64)
  // (The parts have their place also where a cluster joins them in shared memory: the size goes by the splits alone.)
  pl.total = 256 + (pl.splits > 1 ? (size_t)pl.splits * r.M * pl.ldp * 4 : 0);
  *out = r;
  *plan = pl;
  return VC_OK;
}

bool make_map8(CUtensorMap* m, const void* base, int rows, int K, int64_t ld, int box_rows) {
  attn::EncodeTiledFn fn = attn::encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)K, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld};
  const cuuint32_t box[2] = {128, (cuuint32_t)box_rows}, step[2] = {1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool make_map_out(CUtensorMap* m, void* out, const vc_linear_params& r) {
  attn::EncodeTiledFn fn = attn::encode_fn();
  if (!fn) return false;
  const int es = elem_size(r.out_dtype);
  const cuuint64_t dims[2] = {(cuuint64_t)r.N, (cuuint64_t)r.M}, strides[1] = {(cuuint64_t)r.ldo * es};
  const cuuint32_t box[2] = {(cuuint32_t)(128 / es), 32}, step[2] = {1, 1};
  const CUtensorMapDataType type = r.out_dtype == VC_DTYPE_FP32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                   : r.out_dtype == VC_DTYPE_FP16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
  return fn(m, type, 2, out, dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool SWAP, int TN>
cudaError_t launch_linear(const vc_linear_params& r, const Plan& pl, const LinearArgs& a, const void* x, const void* w, cudaStream_t s) {
  using C = Cfg<SWAP, TN>;
  alignas(64) CUtensorMap ta, tb, to;
  if (!make_map8(&ta, SWAP ? w : x, SWAP ? r.N : r.M, r.K, SWAP ? r.ldw : r.ldx, 128) ||
      !make_map8(&tb, SWAP ? x : w, SWAP ? r.M : r.N, r.K, SWAP ? r.ldx : r.ldw, C::kPair ? TN / 2 : TN))
    return cudaErrorUnknown;
  to = ta;                                   // (read where rows leave by copies alone)
  if (!SWAP && a.copies && pl.splits == 1 && !make_map_out(&to, a.out, r)) return cudaErrorUnknown;
  cudaError_t e = allow_smem<linear_fp8_kernel<SWAP, TN>>();
  if (e != cudaSuccess) return e;
  const int ctas = C::kPair ? 2 : pl.joined ? pl.splits : 1, room = sm_count() / (C::kPair ? 2 : 1);
  const int grid = pl.joined ? (int)pl.items : (C::kPair ? 2 : 1) * (pl.items < room ? (int)pl.items : room);       // (joined: an item a CTA)
  constexpr size_t smem = C::kStages * C::kStage + C::kOut + sizeof(Smem<C::kStages, C::kBufs>);
  e = launch_clusters(linear_fp8_kernel<SWAP, TN>, dim3((unsigned)grid), ctas, kThreads, smem, s, ta, tb, to, a);
  if (e != cudaSuccess) return e;
  count_launches(1);
  if (pl.splits > 1 && !pl.joined) {
    const int64_t work = ((int64_t)r.M * ((r.N + 3) / 4) + 255) / 256, most = 8 * sm_count();
    e = launch_overlapped(linear_join_kernel, dim3((unsigned)(work < most ? work : most)), 256, 0, s, a);
    if (e != cudaSuccess) return e;
    count_launches(1);
  }
  return cudaSuccess;
}

}  // namespace
}  // namespace vc

using namespace vc;

extern "C" size_t vc_linear_workspace_bytes(const vc_linear_params* p) {
  vc_linear_params r;
  Plan pl;
  return resolve(p, &r, &pl) == VC_OK ? pl.total : 0;
}

extern "C" vc_status vc_linear_fp8(const vc_linear_params* p, const void* x_codes, const float* x_scale, const void* w_codes, const float* w_scale,
                                   const void* bias, void* out, void* workspace, void* stream) {
  vc_linear_params r;
  Plan pl;
  const vc_status st = resolve(p, &r, &pl);
  if (st != VC_OK) return st;
  if (!x_codes || !x_scale || !w_codes || !w_scale || !out || !workspace) return VC_ERR_INVALID_ARG;
  if (misaligned16(x_codes) || misaligned16(x_scale) || misaligned16(w_codes) || misaligned16(w_scale) || misaligned16(bias) || misaligned16(out) ||
      misaligned16(workspace))
    return VC_ERR_INVALID_ARG;
  LinearArgs a{};
  a.xs = x_scale; a.ws = w_scale; a.bias = bias; a.out = out;
  a.status = (uint32_t*)workspace;
  a.part = (float*)((uint8_t*)workspace + 256);
  a.ldo = r.ldo; a.ldp = pl.ldp;
  a.M = r.M; a.N = r.N; a.blocks = pl.blocks; a.tiles_b = pl.tiles_b; a.splits = pl.splits; a.joined = pl.joined; a.items = (int)pl.items;
  a.out_dtype = r.out_dtype; a.bias_dtype = r.bias_dtype;
  a.vec = r.ldo * elem_size(r.out_dtype) % 16 == 0;
  a.copies = a.vec && (int64_t)r.N * elem_size(r.out_dtype) % 16 == 0;
  a.limit = attn::attn_wait_limit();
  a.nonblocking = attn::attn_wait_nonblocking();
  cudaStream_t s = (cudaStream_t)stream;
  const cudaError_t e = pl.swap ? (pl.tn == 16 ? launch_linear<true, 16>(r, pl, a, x_codes, w_codes, s) : launch_linear<true, 64>(r, pl, a, x_codes, w_codes, s))
                        : pl.tn == 256 ? launch_linear<false, 256>(r, pl, a, x_codes, w_codes, s)
                                       : launch_linear<false, 128>(r, pl, a, x_codes, w_codes, s);
  return e == cudaSuccess ? VC_OK : VC_ERR_CUDA;
}
