// vc_cross_attn: attention of queries to an encoder's keys and values, at 16 bits on the tensor cores.
//
// A persistent CTA works through items: one or two 128-row query tiles of a head against the head's key tiles (128 keys each), or a
// part of them.  Warp 0 loads, 1 and 3 issue the products of the two query tiles, 2 clears value rows of masked keys; 4-7 and
// 8-11 are the softmax of the two query tiles, 12-15 the epilogue.
//
//   S_t = Q_t K^T    both operands in shared memory, K-major, FP32 accumulators in 128 columns of tensor memory
//   P_t = 2^(s S_t - m)  in registers, a thread a row; written back as 16-bit values over S_t's own columns: both operands of a product have
//                        one type, and P in two parts would double the second product.  (Error against 64 bits in bf16 0.0022 of the outputs' 2-norm,
//                        where rounding the outputs alone gives 0.0017; fp16 0.00024 and 0.00021.)
//   O_t += P_t V     P_t from tensor memory, V as it was loaded ([key][channel], read MN-major)
//
// The running maximum m of a row is a reference, not the exact maximum: O_t and the row sum are rescaled only when a tile
// exceeds it by a factor of 2^8 (P_t then holds values up to 2^8, which both types do).  The first tile sets it,
// so a rescale is rare, and the softmax warps do it themselves: S_t(j) complete says that the product of tile j - 1,
// issued in front of it, is complete too.
//
// What bounds it: per query tile the chain S_t -> softmax (1900 cycles) -> O_t product and next S_t (1024 at d = 128, 1300 with the
// hand-overs), two of which overlap; a pair of query tiles takes 3550 cycles for 128 keys, where the tensor cores need
// 2048 and the exponentials as many, and an item's ends take 1300 more (512 keys 15510 an item, 128 keys 6440: there nothing covers them).  B1 H40 32760 x 512
// d128 is 556000 cycles at any clock: 320-340 us in the first ten calls (1.65 GHz; 1010 to 1075 TFLOP/s), 365-395 behind hundreds (1.4 to 1.5 GHz, the
// power cap); 8192 x 4096 577-605 and 660; 32760 x 512 d64 280-292 in both.  Tried and slower there (first calls): one warp that issues
// for both tiles 332 us (its waits and descriptors lie between the products; 567 at 4096 keys), two that do not take turns (both tiles in the same phase),
// the turn passed at half of a tile's scores 344, two threads a row and 24 warps 358, a polynomial for one exponential in 8 / 4 / 3: 344 / 360 / 372,
// scores read twice from tensor memory instead of held in registers 363 (650 at 4096), the second half of P handed over on its own 343,
// exponentials in front of the tile's maximum 433.  Output rows by TMA instead of by the epilogue's own stores: 403 -> 363.
#include <cmath>
#include <type_traits>

#include "vc_attn_shared.cuh"
#include "vc_layer.cuh"
#include "vc_sm100.cuh"

namespace vc {
namespace {

using namespace layer;
using namespace sm100;

constexpr int kThreads = 512, kStages = 4;
constexpr int kSms = 148;                         // what the rule for splits counts on: the workspace's size must not vary
constexpr float kRescale = 8.0f;                  // log2 of the factor a row may exceed its reference by
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct CrossArgs {
  void* o;
  float *lse, *part_o, *part_lse;                 // part_*: [splits][B * H][N_q] of keys split between CTAs
  const int32_t* kv_len;
  const uint8_t* key_mask;
  uint32_t* status;
  vc_strides so;
  int heads, H, group, Nq, Nkv;                   // heads: B * H
  int qtiles, qitems, tiles_per_item, splits, items;
  int q_b, q_h, k_b, k_h, v_b, v_h;               // 1, or 0 for a dimension that is broadcast: multiplies the copy's coordinate
  float sl;                                       // softmax_scale * log2(e)
  bool joined;                                    // the CTAs of a tile's splits are a cluster and join their parts themselves
  uint32_t limit, nonblocking;
};

struct Smem {
  uint64_t full[kStages], empty[kStages], fixed[2];
  uint64_t q_full[2], q_free[2], s_full[2], p_full[2], o_full[2], o_free[2], turn[2], drain[2];
  alignas(16) uint32_t bits[4][4];                // kept keys of a tile
  float2 ml[2][2][128];                           // [a tile's items in turn][query tile][row]: reference, row sum
  uint32_t tmem_base;
  volatile int abort;
};

struct Item {
  int b, h, q0, split, t0, nt, len;
  bool two;
  // Is there work for query tile t (half t of the keys, with g key tiles of the CTA's in front of the item)?
  __device__ __forceinline__ bool has(int t, bool halves, int g) const { return halves ? nt > (t ^ (g & 1)) : t == 0 || two; }
};

__device__ __forceinline__ Item item_of(const CrossArgs& a, int idx) {
  Item w;
  const int u = idx / a.splits, bh = u / a.qitems;
  w.split = idx - u * a.splits;
  w.q0 = (u - bh * a.qitems) * a.tiles_per_item;
  w.b = bh / a.H;
  w.h = bh - w.b * a.H;
  w.two = a.tiles_per_item == 2 && w.q0 + 1 < a.qtiles;
  w.len = a.kv_len ? min(max(__ldg(a.kv_len + w.b), 0), a.Nkv) : a.Nkv;
  const int tiles = (w.len + 127) >> 7, per = (tiles + a.splits - 1) / a.splits;
  w.t0 = w.split * per;
  w.nt = max(0, min(per, tiles - w.t0));
  return w;
}

// Bounded wait of a whole warp (see warp_wait2 of the quantized kernels: a bare test in front, one vote a poll).
__device__ __forceinline__ bool wait(uint64_t* bar, uint32_t parity, Smem* sh, const CrossArgs& a, uint32_t code) {
  if (__all_sync(0xffffffffu, mbar_test_wait(bar, parity))) return true;
#pragma unroll 1
  for (uint32_t i = 0; i < a.limit; ++i) {
    if (__all_sync(0xffffffffu, a.nonblocking ? mbar_test_wait(bar, parity) : mbar_try_wait(bar, parity))) return true;
    if ((i & 63u) == 63u && __any_sync(0xffffffffu, sh->abort)) return false;
  }
  sh->abort = 1;
  // CTA 0 clears the word when it starts; a wait that gave up started later and took longer, but for a test's tiny limit
  __nanosleep(20000);
  atomicExch(a.status, kStatusTimeout | code);
  return false;
}

__device__ __forceinline__ void tma_load_4d(void* dst, const CUtensorMap* m, uint64_t* bar, int c0, int c1, int c2, int c3) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(m)), "r"(smem_u32(bar)), "r"(c0), "r"(c1), "r"(c2), "r"(c3)
      : "memory");
}

// MN-major operand in the 128-byte swizzle: rows of 64 channels of one key, 8 keys a kilobyte, the next 64 channels a panel on.
__device__ __forceinline__ uint64_t desc_mnmajor(uint32_t saddr, uint32_t panel_bytes) {
  return (uint64_t)((saddr & 0x3FFFF) >> 4) | (uint64_t)(panel_bytes >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
template <typename T> __device__ constexpr uint32_t idesc16(int M, int N) {       // T x T -> FP32, both K-major
  return (1u << 4) | (std::is_same<T, __nv_bfloat16>::value ? (1u << 7) | (1u << 10) : 0u) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
// N floats from the same place of the shared memory of the cluster's CTA `rank`.
template <int N> __device__ __forceinline__ void load_cluster(const float* p, int rank, float (&v)[N]) {
  uint32_t at;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(p)), "r"(rank));
  if constexpr (N == 4) asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]) : "r"(at) : "memory");
  else if constexpr (N == 2) asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v[0]), "=f"(v[1]) : "r"(at) : "memory");
  else asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v[0]) : "r"(at) : "memory");
}

constexpr int kCluster = 8;                       // CTAs of a portable cluster
constexpr uint32_t kPanel = 128 * 128;            // 128 rows of 64 16-bit channels

template <int D> struct Lay {
  static constexpr uint32_t kTile = kPanel * (D / 64);         // a query, key or value tile
  static constexpr uint32_t kOut = kPanel;                     // 64 channels of an output tile
  static constexpr uint32_t kSmem = 2 * kTile + kStages * kTile + kOut + (uint32_t)sizeof(Smem);
  // S_t at 128 t (P_t over its first half), O_t behind
  static constexpr uint32_t kO = 256, kOStride = D;
};

// HALVES: one query tile an item; the CTA's even and its odd key tiles take the places of two query tiles, and the epilogue joins an
// item's.  (Counted over all items of the CTA: a half that passed over key tiles would wait for a barrier's phase two ahead of
// it, which reads as complete.)
template <typename T, int D, bool HALVES>
__global__ void __launch_bounds__(kThreads, 1)
cross_attn_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                  const __grid_constant__ CUtensorMap tm_o, const __grid_constant__ CrossArgs a) {
  using L = Lay<D>;
  constexpr int kRegSoftmax = 176, kRegEpi = 80, kRegCtl = 80;
  constexpr int kPartRow = D + 4;              // floats from row to row of a part in shared memory: no bank conflicts
  static_assert((128 * kPartRow + 128) * 4 <= kStages * L::kTile, "a part exceeds the ring");
  static_assert(2 * kRegSoftmax + kRegEpi + kRegCtl <= 4 * 128, "register budget exceeds the CTA's allocation");
  static_assert(L::kSmem <= 227 * 1024, "shared memory of the kernel exceeds the SM");
  extern __shared__ __align__(1024) unsigned char smem[];
  unsigned char* sQ = smem;
  unsigned char* sKV = smem + 2 * L::kTile;
  unsigned char* sOut = sKV + kStages * L::kTile;
  Smem* sh = reinterpret_cast<Smem*>(sOut + L::kOut);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const bool masked = a.kv_len || a.key_mask;       // some value row may have to be cleared

  if (tid == 0) {
    for (int i = 0; i < kStages; ++i) { mbar_init(&sh->full[i], 1); mbar_init(&sh->empty[i], 2); }
    for (int t = 0; t < 2; ++t) {
      mbar_init(&sh->fixed[t], 1); mbar_init(&sh->turn[t], 1);
      mbar_init(&sh->q_full[t], 1); mbar_init(&sh->q_free[t], 1);
      mbar_init(&sh->s_full[t], 1); mbar_init(&sh->p_full[t], 128);
      mbar_init(&sh->o_full[t], 1); mbar_init(&sh->o_free[t], 128);
    }
    mbar_init(&sh->drain[0], 1); mbar_init(&sh->drain[1], 1);
    sh->abort = 0;
    mbar_fence_init();
    tma_prefetch_desc(&tm_q); tma_prefetch_desc(&tm_k); tma_prefetch_desc(&tm_v);
  }
  pdl_wait();
  if (warp == 2) { tmem_alloc<512>(&sh->tmem_base); tmem_relinquish(); }
  if (tid == 0 && blockIdx.x == 0) *a.status = 0;
  if (a.splits > 1 && !a.joined) pdl_allow();               // (what follows then is the launch that joins the parts: it may stand by)
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sh->tmem_base;
  const uint32_t lane_base = tmem + ((uint32_t)((warp & 3) * 32) << 16);

  if (warp < 4) {
    reg_dec<kRegCtl>();
    if (warp == 0) {
      // -------------------------------------------------------------------------------- loads
      int g = 0;                                    // key tiles
      int issued = 0, n[2] = {0, 0};                // ring slots filled, query tiles loaded
      bool ok = true;
      auto fill = [&](const CUtensorMap* m, int row, int ch, int cb) {
        const int st = issued % kStages;
        if (elect_one()) {
          mbar_expect_tx(&sh->full[st], L::kTile);
          for (int c = 0; c < D / 64; ++c) tma_load_4d(sKV + st * L::kTile + c * kPanel, m, &sh->full[st], 64 * c, row, ch, cb);
        }
        __syncwarp();
        ++issued;
      };
      auto room = [&] { return ok = wait(&sh->empty[issued % kStages], ((issued / kStages) & 1) ^ 1, sh, a, 1); };
      for (int idx = blockIdx.x; ok && idx < a.items; idx += gridDim.x) {
        const Item w = item_of(a, idx);
        const int hk = w.h / a.group;
        for (int j = 0; j < w.nt; ++j, ++g) {
          const int row = (w.t0 + j) * 128;
          uint32_t words[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int key = row + 32 * i + lane;
            bool keep = key < w.len;
            if (a.key_mask && keep) keep = __ldg(a.key_mask + (int64_t)w.b * a.Nkv + key) != 0;
            words[i] = __ballot_sync(0xffffffffu, keep);
          }
          if (!room()) break;
          // (the words' last readers are four key tiles back, and this slot's keys were read two tiles back)
          if (lane < 4) sh->bits[g & 3][lane] = lane == 0 ? words[0] : lane == 1 ? words[1] : lane == 2 ? words[2] : words[3];
          __syncwarp();
          fill(&tm_k, row, hk * a.k_h, w.b * a.k_b);
          if (j == 0) {                             // queries, each tile's when its predecessor's last scores are complete
            for (int t = 0; t < 2; ++t) {
              if (!w.has(t, HALVES, g)) continue;
              if (!(ok = wait(&sh->q_free[t], (n[t] & 1) ^ 1, sh, a, 3))) break;
              if (elect_one()) {
                mbar_expect_tx(&sh->q_full[t], L::kTile);
                for (int c = 0; c < D / 64; ++c)
                  tma_load_4d(sQ + t * L::kTile + c * kPanel, &tm_q, &sh->q_full[t], 64 * c, (HALVES ? w.q0 : w.q0 + t) * 128, w.h * a.q_h, w.b * a.q_b);
              }
              __syncwarp();
              ++n[t];
            }
            if (!ok) break;
          }
          if (!room()) break;
          fill(&tm_v, row, hk * a.v_h, w.b * a.v_b);
        }
      }
      for (int t = 0; t < 2; ++t)
        if (n[t]) mbar_wait(&sh->q_full[t], (n[t] - 1) & 1, attn::kDrainLimit);
      // every copy issued has landed before the CTA may end (at once on a normal run)
      for (int i = issued > kStages ? issued - kStages : 0; i < issued; ++i) mbar_wait(&sh->full[i % kStages], (i / kStages) & 1, attn::kDrainLimit);
    } else if (warp == 1 || warp == 3) {
      // -------------------------------------------------------------------------------- products, one warp a query tile
      // (with one warp for both, each group of products began 200 cycles behind the end of the one in front)
      constexpr uint32_t idesc_s = idesc16<T>(128, 128), idesc_o = idesc16<T>(128, D) | (1u << 16);
      const int t = warp >> 1;
      const uint32_t s_at = tmem + 128 * t, o_at = tmem + L::kO + L::kOStride * t;
      const uint64_t dq = smem_desc_kmajor(smem_u32(sQ + t * L::kTile), 128), dk0 = smem_desc_kmajor(smem_u32(sKV), 128), dv0 = desc_mnmajor(smem_u32(sKV), kPanel);
      int g = 0, items = 0, uses = 0;               // key tiles of the CTA; items and key tiles of this query tile
      bool ok = true;
      // The two warps take turns: [P_0 V, next S_0], [P_1 V, next S_1], ...  Left alone their products mix, both tiles' scores are
      // complete at the same time, both softmax groups want the special-function unit at once and the tensor cores wait for them.
      int turns = 0;
      auto my_turn = [&] { return ok = HALVES || t == 0 && turns == 0 ? true : wait(&sh->turn[t], (t == 0 ? turns - 1 : turns) & 1, sh, a, 16); };
      auto pass = [&] { if (!HALVES) mbar_arrive(&sh->turn[t ^ 1]); };
      auto scores = [&](bool first, bool last_of_item, bool alone) {
        const int slot = 2 * g, st = slot % kStages;
        if (!(ok = wait(&sh->full[st], (slot / kStages) & 1, sh, a, 10))) return;
        if (first && !(ok = wait(&sh->q_full[t], items & 1, sh, a, 11))) return;
        // (no fence: what these columns held was read in front of the hand-over that the product issued last has waited for)
        if (elect_one()) {
          const uint64_t dk = dk0 + st * (L::kTile >> 4);
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            const uint32_t at = (k / 4) * (kPanel >> 4) + 2 * (k % 4);
            mma_f16_ss(s_at, dq + at, dk + at, idesc_s, k > 0);
          }
          mma_commit(&sh->s_full[t]);
          pass();
          if (last_of_item) mma_commit(&sh->q_free[t]);
          mma_commit(&sh->empty[st]);
          if (alone) mma_commit(&sh->empty[st]);    // for the query tile that is not there
        }
        __syncwarp();
      };
      auto outputs = [&](bool first, bool last_of_item, bool alone) {
        const int slot = 2 * g + 1, st = slot % kStages;
        if (!(ok = wait(&sh->full[st], (slot / kStages) & 1, sh, a, 12))) return;
        if (masked && !(ok = wait(&sh->fixed[g & 1], (g >> 1) & 1, sh, a, 13))) return;
        if (first && !(ok = wait(&sh->o_free[t], (items & 1) ^ 1, sh, a, 14))) return;
        if (!(ok = wait(&sh->p_full[t], uses & 1, sh, a, 15))) return;
        if (!my_turn()) return;
        ++turns;
        if (elect_one()) {
          tc_fence_after();
          const uint64_t dv = dv0 + st * (L::kTile >> 4);
#pragma unroll
          for (int k = 0; k < 8; ++k) mma_f16_ts(o_at, s_at + 8 * k, dv + 128 * k, idesc_o, !first | (k > 0));
          if (last_of_item) mma_commit(&sh->o_full[t]);
          mma_commit(&sh->empty[st]);
          if (alone) mma_commit(&sh->empty[st]);
        }
        __syncwarp();
      };
      Item w, x;
      auto next_item = [&](int from, Item& it) {    // the next item that has keys
        for (; from < a.items; from += gridDim.x) {
          it = item_of(a, from);
          if (it.nt > 0) break;
        }
        return from;
      };
      int idx;
      if constexpr (HALVES) {
        // My key tiles one by one, and no turns: a tile's keys and values have one reader.
        int before = 0, j0 = t;                     // key tiles in front of the item, its first one of mine
        auto find = [&](int from) {                 // the next item that has one
          for (idx = next_item(from, w); idx < a.items && w.nt <= (j0 = t ^ (before & 1)); idx = next_item(idx + gridDim.x, w)) before += w.nt;
          g = before + j0;
        };
        find(blockIdx.x);
        if (idx < a.items) scores(true, w.nt <= j0 + 2, true);
        for (int j = j0; ok && idx < a.items;) {
          const bool end = j + 2 >= w.nt;
          outputs(j == j0, end, true);
          ++uses;
          if (!ok) break;
          if (end) {
            ++items;
            before += w.nt;
            find(idx + gridDim.x);
            j = j0;
          } else {
            g += 2;
            j += 2;
          }
          if (idx < a.items) scores(j == j0, j + 2 >= w.nt, true);
        }
      } else {
        // S(0), [P(0) V, S(1)], [P(1) V, S(2)], ... across items.  A turn for every key tile, also where this query tile is not there.
        auto here = [&](const Item& it) { return t == 0 || it.two; };
        idx = next_item(blockIdx.x, w);
        if (idx < a.items) {
          if (!my_turn()) {
          } else if (++turns, here(w)) {
            scores(true, w.nt == 1, !w.two);
          } else if (elect_one()) {
            pass();
          }
        }
        while (ok && idx < a.items) {
          const int nidx = next_item(idx + gridDim.x, x);
          for (int j = 0; ok && j < w.nt; ++j) {
            const bool end = j + 1 == w.nt, nx_here = end ? nidx < a.items && here(x) : here(w);
            if (here(w)) {
              outputs(j == 0, end, !w.two);
              ++uses;
              if (end) ++items;
            } else if (my_turn()) {
              ++turns;
            }
            ++g;
            if (!ok) break;
            if (nx_here) scores(end, end ? x.nt == 1 : j + 2 == w.nt, end ? !x.two : !w.two);
            else if (elect_one()) pass();
            __syncwarp();
          }
          w = x;
          idx = nidx;
        }
      }
      if (elect_one()) mma_commit(&sh->drain[t]);
      __syncwarp();
      mbar_wait(&sh->drain[t], 0, attn::kDrainLimit);
    } else if (warp == 2 && masked) {
      // -------------------------------------------------------------------------------- value rows of masked keys
      // 0 times an infinity or NaN is NaN: rows whose probability is 0 must hold numbers.
      int g = 0;
      bool ok = true;
      for (int idx = blockIdx.x; ok && idx < a.items; idx += gridDim.x) {
        const Item w = item_of(a, idx);
        for (int j = 0; j < w.nt; ++j, ++g) {
          const int slot = 2 * g + 1, st = slot % kStages;
          if (!(ok = wait(&sh->full[st], (slot / kStages) & 1, sh, a, 20))) break;
          const uint4 kept = *reinterpret_cast<const uint4*>(sh->bits[g & 3]);       // (written in front of the keys' copy)
          if ((kept.x & kept.y & kept.z & kept.w) != 0xffffffffu) {
            unsigned char* tile = sKV + st * L::kTile;
#pragma unroll 1
            for (int r = lane >> 3; r < 128; r += 4) {                               // eight lanes a row
              const uint32_t word = r < 64 ? (r < 32 ? kept.x : kept.y) : (r < 96 ? kept.z : kept.w);
              if (!(word >> (r & 31) & 1))
                for (int c = 0; c < D / 64; ++c) *reinterpret_cast<uint4*>(tile + c * kPanel + r * 128 + 16 * (lane & 7)) = make_uint4(0, 0, 0, 0);
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");             // the stores -> tensor-core reads
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(&sh->fixed[g & 1]);
          __syncwarp();
        }
      }
    }
  } else if (warp < 12) {
    reg_inc<kRegSoftmax>();
    // ---------------------------------------------------------------------------------- softmax, one query tile a warpgroup
    const int t = (warp >> 2) - 1, row = (warp & 3) * 32 + lane;
    const uint32_t s_col = lane_base + 128 * t, o_col = lane_base + L::kO + L::kOStride * t;
    int g = 0, uses = 0, items = 0;
    bool ok = true;
    for (int idx = blockIdx.x; ok && idx < a.items; idx += gridDim.x) {
      const Item w = item_of(a, idx);
      if (w.nt == 0) continue;
      if (!w.has(t, HALVES, g)) { g += w.nt; continue; }
      float m = -INFINITY, l = 0.f;                 // reference (log2 domain) and row sum
      const int step = HALVES ? 2 : 1, j0 = HALVES ? t ^ (g & 1) : 0;
      for (int j = j0; j < w.nt; j += step) {
        if (!(ok = wait(&sh->s_full[t], uses & 1, sh, a, 30))) break;
        ++uses;
        tc_fence_after();
        uint32_t s0[32], s1[32], s2[32], s3[32];
        tmem_ld32(s_col, s0); tmem_ld32(s_col + 32, s1); tmem_ld32(s_col + 64, s2); tmem_ld32(s_col + 96, s3);
        tmem_wait_ld();
        if (w.len - (w.t0 + j) * 128 < 128 || a.key_mask) {
          const uint4 kept = *reinterpret_cast<const uint4*>(sh->bits[(g + j) & 3]);
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            if (!(kept.x >> i & 1)) s0[i] = 0xff800000u;
            if (!(kept.y >> i & 1)) s1[i] = 0xff800000u;
            if (!(kept.z >> i & 1)) s2[i] = 0xff800000u;
            if (!(kept.w >> i & 1)) s3[i] = 0xff800000u;
          }
        }
        float mx[4] = {__uint_as_float(s0[0]), __uint_as_float(s1[0]), __uint_as_float(s2[0]), __uint_as_float(s3[0])};
#pragma unroll
        for (int i = 1; i < 31; i += 2) {
          mx[0] = max3(mx[0], __uint_as_float(s0[i]), __uint_as_float(s0[i + 1]));
          mx[1] = max3(mx[1], __uint_as_float(s1[i]), __uint_as_float(s1[i + 1]));
          mx[2] = max3(mx[2], __uint_as_float(s2[i]), __uint_as_float(s2[i + 1]));
          mx[3] = max3(mx[3], __uint_as_float(s3[i]), __uint_as_float(s3[i + 1]));
        }
        const float top = a.sl * max3(max3(mx[0], __uint_as_float(s0[31]), mx[1]), max3(__uint_as_float(s1[31]), mx[2], __uint_as_float(s2[31])), fmaxf(mx[3], __uint_as_float(s3[31])));
        if (j == j0) {
          m = top;
        } else if (__any_sync(0xffffffffu, top > m + kRescale)) {
          const float m_new = fmaxf(m, top), alpha = m == m_new ? 1.f : ex2_approx(m - m_new);
          l *= alpha;
          m = m_new;
          uint32_t r[16];
#pragma unroll 1
          for (int c = 0; c < D / 16; ++c) {
            tmem_ld16(o_col + 16 * c, r);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 16; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) * alpha);
            tmem_st16(o_col + 16 * c, r);
          }
        }
        // (a row without a kept key so far: every score is -infinity, and so is the reference)
        const float ms = m == -INFINITY ? 0.f : m;
        const uint64_t sl2 = pack_f32x2(a.sl, a.sl), nm2 = pack_f32x2(-ms, -ms);
        uint64_t sum0 = 0, sum1 = 0;
        auto part = [&](const uint32_t (&s)[32], int q) {
          uint32_t out[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            float x0, x1;
            unpack2(fma2(pack_b32x2(s[2 * i], s[2 * i + 1]), sl2, nm2), x0, x1);
            const float p0 = ex2_approx(x0), p1 = ex2_approx(x1);
            const uint64_t pp = pack_f32x2(p0, p1);
            if (i & 1) sum1 = add2(sum1, pp); else sum0 = add2(sum0, pp);
            out[i] = pack16<T>(p0, p1);
          }
          tmem_st16(s_col + 16 * q, out);
        };
        part(s0, 0); part(s1, 1); part(s2, 2); part(s3, 3);
        float a0, a1;
        unpack2(add2(sum0, sum1), a0, a1);
        l += a0 + a1;
        // In front of the last hand-over: the product behind it, when complete, says that these are there too.  Two slots do: the
        // tile's next item but one gets here only when the next one's first product has seen the epilogue of this one.
        if (j + step >= w.nt) sh->ml[items & 1][t][row] = make_float2(m, l);
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive(&sh->p_full[t]);
      }
      g += w.nt;
      ++items;
    }
  } else {
    reg_dec<kRegEpi>();
    // ---------------------------------------------------------------------------------- epilogue
    using Out = attn::OutTile<64>;                  // rows leave in lines of 128 bytes
    const int quarter = warp & 3;
    const uint32_t tile = smem_u32(sOut) + quarter * 32 * Out::ROW;
    int uses[2] = {0, 0}, g = 0;
    bool ok = true;
    for (int idx = blockIdx.x; ok && idx < a.items; idx += gridDim.x) {
      const Item w = item_of(a, idx);
      const int half = HALVES ? g & 1 : 0;              // the half that has the item's first key tile
      g += w.nt;
#pragma unroll 1
      for (int t = 0; t < (w.two ? 2 : 1); ++t) {       // (the halves of the keys are joined in one pass)
        const int row0 = (w.q0 + t) * 128 + quarter * 32, rows = min(32, a.Nq - row0);
        const bool both = HALVES && w.nt > 1;
        const int u = HALVES ? half : t;
        float inv = 0.f, inv1 = 0.f, lse2 = -INFINITY;
        // my row of the outputs' [B * H][N_q], behind those of the splits in front of this one
        const int64_t line = ((int64_t)w.split * a.heads + w.b * a.H + w.h) * a.Nq + row0 + lane;
        if (w.nt > 0) {
          if (!(ok = wait(&sh->o_full[u], uses[u] & 1, sh, a, 40)) || (both && !(ok = wait(&sh->o_full[u ^ 1], uses[u ^ 1] & 1, sh, a, 41)))) break;
          float2 ml = sh->ml[uses[u] & 1][u][quarter * 32 + lane];
          ++uses[u];
          float f0 = 1.f, f1 = 0.f;
          if (both) {                                 // o = (2^(m0 - m) O_0 + 2^(m1 - m) O_1) / (2^(m0 - m) l0 + 2^(m1 - m) l1)
            const float2 ml1 = sh->ml[uses[u ^ 1] & 1][u ^ 1][quarter * 32 + lane];
            ++uses[u ^ 1];
            const float m = fmaxf(ml.x, ml1.x), ms = m == -INFINITY ? 0.f : m;
            f0 = ex2_approx(ml.x - ms);
            f1 = ex2_approx(ml1.x - ms);
            ml = make_float2(m, f0 * ml.y + f1 * ml1.y);
          }
          const float total = ml.y > 0.f || ml.y != ml.y ? 1.0f / ml.y : 0.f;     // (a sum of NaN makes a row of NaN)
          inv = f0 * total;
          inv1 = f1 * total;
          lse2 = ml.y == 0.f ? -INFINITY : ml.x + log2f(ml.y);
          tc_fence_after();
        }
        const uint32_t o_col = lane_base + L::kO + L::kOStride * u, o_col1 = lane_base + L::kO + L::kOStride * (u ^ 1);
#pragma unroll 1
        for (int c = 0; c < D / 32; ++c) {                            // 32 channels
          uint32_t r[32];
          if (w.nt > 0) {
            tmem_ld32(o_col + 32 * c, r);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 32; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) * inv);
            if (both) {
#pragma unroll
              for (int q = 0; q < 2; ++q) {
                uint32_t r1[16];
                tmem_ld16(o_col1 + 32 * c + 16 * q, r1);
                tmem_wait_ld();
#pragma unroll
                for (int i = 0; i < 16; ++i) r[16 * q + i] = __float_as_uint(fmaf(__uint_as_float(r1[i]), inv1, __uint_as_float(r[16 * q + i])));
              }
            }
            if (c == D / 32 - 1) {
              tc_fence_before();
              mbar_arrive(&sh->o_free[u]);
              if (both) mbar_arrive(&sh->o_free[u ^ 1]);
            }
          } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) r[i] = 0;
          }
          if (a.splits > 1) {
            // (joined: the last product is complete, the ring is free)
            float4* po = reinterpret_cast<float4*>(a.joined ? reinterpret_cast<float*>(sKV) + (quarter * 32 + lane) * kPartRow + 32 * c : a.part_o + line * D + 32 * c);
            if (lane < rows)
#pragma unroll
              for (int i = 0; i < 32; i += 4)
                po[i / 4] = make_float4(__uint_as_float(r[i]), __uint_as_float(r[i + 1]), __uint_as_float(r[i + 2]), __uint_as_float(r[i + 3]));
            continue;
          }
          if ((c & 1) == 0) {
            if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");        // the copy in front has read the rows
            __syncwarp();
          }
          auto two = [&](int i) { return pack16<T>(__uint_as_float(r[i]), __uint_as_float(r[i + 1])); };
#pragma unroll
          for (int i = 0; i < 4; ++i) sts128(Out::chunk(tile, lane, 4 * (c & 1) + i), two(8 * i), two(8 * i + 2), two(8 * i + 4), two(8 * i + 6));
          if (c & 1) {
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0 && rows > 0) {               // (rows behind the last query are left as they are)
              asm volatile("cp.async.bulk.tensor.4d.global.shared::cta.bulk_group [%0, {%2, %3, %4, %5}], [%1];" ::"l"(reinterpret_cast<uint64_t>(&tm_o)),
                           "r"(tile), "r"(32 * c - 32), "r"(row0), "r"(w.h), "r"(w.b)
                           : "memory");
              asm volatile("cp.async.bulk.commit_group;" ::: "memory");
            }
          }
        }
        if (lane < rows) {
          if (a.joined) reinterpret_cast<float*>(sKV)[128 * kPartRow + quarter * 32 + lane] = lse2;
          else if (a.splits > 1) a.part_lse[line] = lse2;
          else if (a.lse) a.lse[line] = lse2 * kLn2;
        }
      }
    }
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");       // the rows have left shared memory before the CTA may end
  }
  tc_fence_before();
  if (HALVES && a.joined) {
    // A row's parts in the order of the splits (as cross_join_kernel), from the shared memory of the cluster's CTAs.  A warp a row.
    constexpr int kPer = D / 32;
    const Item w = item_of(a, blockIdx.x);
    const int rows = min(128, a.Nq - w.q0 * 128);
    const float* part = reinterpret_cast<const float*>(sKV);
    cluster_sync();
    for (int r = w.split * (kThreads / 32) + warp; r < rows; r += a.splits * (kThreads / 32)) {
      float lse[kCluster][1], po[kCluster][kPer], top = -INFINITY, acc[kPer] = {}, sum = 0.f;
#pragma unroll
      for (int i = 0; i < kCluster; ++i)
        if (i < a.splits) {
          load_cluster<1>(part + 128 * kPartRow + r, i, lse[i]);
          load_cluster<kPer>(part + r * kPartRow + lane * kPer, i, po[i]);
        }
#pragma unroll
      for (int i = 0; i < kCluster; ++i)
        if (i < a.splits) top = lse[i][0] != lse[i][0] || top != top ? NAN : fmaxf(top, lse[i][0]);
      const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
      for (int i = 0; i < kCluster; ++i)
        if (i < a.splits) {
          const float wt = exp2f(lse[i][0] - base);
          sum += wt;
#pragma unroll
          for (int j = 0; j < kPer; ++j) acc[j] = fmaf(wt, po[i][j], acc[j]);
        }
      const float inv = sum == 0.f ? 0.f : 1.0f / sum;
      T* dst = static_cast<T*>(a.o) + w.b * a.so.b + w.h * a.so.h + (int64_t)(w.q0 * 128 + r) * a.so.n + lane * kPer;
#pragma unroll
      for (int j = 0; j < kPer; j += 2) reinterpret_cast<uint32_t*>(dst)[j / 2] = pack16<T>(acc[j] * inv, acc[j + 1] * inv);
      if (a.lse && lane == 0) a.lse[((int64_t)w.b * a.H + w.h) * a.Nq + w.q0 * 128 + r] = sum == 0.f ? -INFINITY : (base + log2f(sum)) * kLn2;
    }
    cluster_sync();                            // (a CTA stays until its peers have read it)
    if (warp == 2) tmem_dealloc<512>(tmem);
    return;
  }
  __syncthreads();
  if (warp == 2) tmem_dealloc<512>(tmem);
}

// Joins the parts of a row: o = sum w_s o_s / sum w_s, w_s = 2^(lse_s - max lse), in the order of the splits.  A warp a row.
template <typename T, int D>
__global__ void __launch_bounds__(256)
cross_join_kernel(const __grid_constant__ CrossArgs a, int64_t rows) {
  constexpr int kPer = D / 32;
  const int lane = threadIdx.x & 31;
  const int64_t r = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  pdl_wait();
  if (r >= rows) return;
  float top = -INFINITY;
  for (int s = 0; s < a.splits; ++s) {
    const float v = a.part_lse[s * rows + r];
    top = v != v ? v : fmaxf(top, v);
    if (v != v) break;
  }
  const float base = top == -INFINITY ? 0.f : top;
  float acc[kPer] = {}, sum = 0.f;
  for (int s = 0; s < a.splits; ++s) {
    const float wt = exp2f(a.part_lse[s * rows + r] - base);
    sum += wt;
    const float* po = a.part_o + (s * rows + r) * D + lane * kPer;
#pragma unroll
    for (int i = 0; i < kPer; ++i) acc[i] = fmaf(wt, po[i], acc[i]);
  }
  const float inv = sum == 0.f ? 0.f : 1.0f / sum;
  const int64_t bh = r / a.Nq, n = r - bh * a.Nq, b = bh / a.H, h = bh - b * a.H;
  T* dst = static_cast<T*>(a.o) + b * a.so.b + h * a.so.h + n * a.so.n + lane * kPer;
#pragma unroll
  for (int i = 0; i < kPer; i += 2) reinterpret_cast<uint32_t*>(dst)[i / 2] = pack16<T>(acc[i] * inv, acc[i + 1] * inv);
  if (a.lse && lane == 0) a.lse[r] = sum == 0.f ? -INFINITY : (base + log2f(sum)) * kLn2;
}

// Clusters of n CTAs with an SM each that run side by side: eight GPCs of 18 SMs or more.
inline int clusters_at_once(int n) { return 8 * (18 / n); }

struct Plan {
  bool joined;
  int qtiles, tiles_per_item, qitems, splits;
  int64_t rows, items;
  size_t part_o, part_lse, total;
};

vc_status resolve(const vc_cross_params* p, vc_cross_params* out, Plan* plan) {
  if (!p) return VC_ERR_INVALID_ARG;
  vc_cross_params r = *p;
  if (r.B < 1 || r.H < 1 || r.H_kv < 1 || r.H % r.H_kv || (int64_t)r.B * r.H > 65535) return VC_ERR_INVALID_ARG;
  if (r.N_q < 1 || r.N_q > (1 << 22) || r.N_kv < 0 || r.N_kv > (1 << 22)) return VC_ERR_INVALID_ARG;
  if (r.d != 64 && r.d != 128) return VC_ERR_INVALID_ARG;
  if (r.dtype != VC_DTYPE_BF16 && r.dtype != VC_DTYPE_FP16) return VC_ERR_INVALID_ARG;
  if (r.key_splits < 0 || r.key_splits > 64) return VC_ERR_INVALID_ARG;
  if (r.softmax_scale == 0.f) r.softmax_scale = 1.0f / std::sqrt((float)r.d);
  if (!(r.softmax_scale > 0.f) || !std::isfinite(r.softmax_scale)) return VC_ERR_INVALID_ARG;
  const int nk = r.N_kv > 0 ? r.N_kv : 1;
  if (!resolve_strides(p->q, r.B, r.H, r.N_q, r.d, 2, false, &r.q) || !resolve_strides(p->k, r.B, r.H_kv, nk, r.d, 2, false, &r.k) ||
      !resolve_strides(p->v, r.B, r.H_kv, nk, r.d, 2, false, &r.v) || !resolve_strides(p->o, r.B, r.H, r.N_q, r.d, 2, true, &r.o))
    return VC_ERR_INVALID_ARG;
  Plan pl{};
  pl.rows = (int64_t)r.B * r.H * r.N_q;
  pl.qtiles = (r.N_q + 127) / 128;
  const int64_t bh = (int64_t)r.B * r.H;
  // Two query tiles an item share the keys' copies and keep the tensor cores busy in turn; a pair takes about 1.3 times a tile alone.
  // With so few pairs that twice as many tiles still fit the SMs, every tile has a CTA of its own; so has a head's only tile, which
  // would be alone in a pair's place (B8 H40, one token against 512 keys 28.5 -> 21.4 us, 128 against 4096 178 -> 135).
  pl.tiles_per_item = pl.qtiles > 1 && 2 * bh * ((pl.qtiles + 1) / 2) > kSms ? 2 : 1;
  pl.qitems = (pl.qtiles + pl.tiles_per_item - 1) / pl.tiles_per_item;
  const int ktiles = (r.N_kv + 127) / 128;
  pl.splits = r.key_splits;
  if (pl.splits == 0) {
    const int64_t room = kSms / (bh * pl.qitems);
    pl.splits = 1;
    if (room > 1 && ktiles >= 8) pl.splits = (int)(room < ktiles / 4 ? room : ktiles / 4);
  }
  if (pl.splits > ktiles) pl.splits = ktiles > 0 ? ktiles : 1;
  if (pl.splits > 64) pl.splits = 64;
  // Few parts: the splits of a tile are a cluster and need no second launch (B2 H16, one token against 16384 keys 50.5 -> 49.1 us, B4 H8 against 2048
  // 12.7 -> 11.4, B1 H12, 100 against 2048 14.3 -> 13.6), up to two rows a warp of the cluster (four, 128 rows in two parts: 11.8 -> 12.9).
  pl.joined = pl.tiles_per_item == 1 && pl.splits > 1 && pl.splits <= kCluster && bh * pl.qitems <= clusters_at_once(pl.splits) &&
              (r.N_q < 128 ? r.N_q : 128) <= 32 * pl.splits;
  pl.items = bh * pl.qitems * pl.splits;
  if (pl.items > INT32_MAX) return VC_ERR_UNSUPPORTED;
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  // (The parts have their place also where a cluster joins them in shared memory: the size goes by the splits alone.)
  pl.part_o = 256;
  pl.part_lse = pl.part_o + (pl.splits > 1 ? up((size_t)pl.splits * pl.rows * r.d * 4) : 0);
  pl.total = pl.part_lse + (pl.splits > 1 ? up((size_t)pl.splits * pl.rows * 4) : 0);
  *out = r;
  *plan = pl;
  return VC_OK;
}

// [B][H][N][d] of 16-bit elements, boxes of 64 channels x `box_rows` in the 128-byte swizzle.  A broadcast dimension becomes one
// entry (its coordinate is multiplied by 0).
bool make_map16(CUtensorMap* m, const void* base, const vc_strides& s, int B, int H, int N, int d, int box_rows, int* mul_b, int* mul_h) {
  attn::EncodeTiledFn fn = attn::encode_fn();
  if (!fn) return false;
  *mul_b = s.b != 0; *mul_h = s.h != 0;
  const cuuint64_t dims[4] = {(cuuint64_t)d, (cuuint64_t)N, (cuuint64_t)(s.h ? H : 1), (cuuint64_t)(s.b ? B : 1)};
  const cuuint64_t strides[3] = {(cuuint64_t)s.n * 2, (cuuint64_t)(s.h ? s.h : s.n) * 2, (cuuint64_t)(s.b ? s.b : s.n) * 2};
  const cuuint32_t box[4] = {64, (cuuint32_t)box_rows, 1, 1}, step[4] = {1, 1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int D, bool HALVES>
cudaError_t launch_cross(const vc_cross_params& r, const Plan& pl, CrossArgs& a, const void* q, const void* k, const void* v, cudaStream_t s) {
  alignas(64) CUtensorMap tq, tk, tv, to;
  const bool any = r.N_kv > 0;                      // without keys nothing is loaded, and any valid map will do
  int one_b, one_h;
  if (!make_map16(&tq, q, r.q, r.B, r.H, r.N_q, D, 128, &a.q_b, &a.q_h) || !make_map16(&to, a.o, r.o, r.B, r.H, r.N_q, D, 32, &one_b, &one_h)) return cudaErrorUnknown;
  tk = tv = tq;
  if (any && (!make_map16(&tk, k, r.k, r.B, r.H_kv, r.N_kv, D, 128, &a.k_b, &a.k_h) || !make_map16(&tv, v, r.v, r.B, r.H_kv, r.N_kv, D, 128, &a.v_b, &a.v_h)))
    return cudaErrorUnknown;
  cudaError_t e = allow_smem<cross_attn_kernel<T, D, HALVES>>();
  if (e != cudaSuccess) return e;
  const int grid = pl.joined || pl.items < sm_count() ? (int)pl.items : sm_count();       // (joined: an item a CTA)
  e = launch_clusters(cross_attn_kernel<T, D, HALVES>, dim3((unsigned)grid), pl.joined ? pl.splits : 1, kThreads, Lay<D>::kSmem, s, tq, tk, tv, to, a);
  if (e != cudaSuccess) return e;
  count_launches(1);
  if (pl.splits > 1 && !pl.joined) {
    e = launch_overlapped(cross_join_kernel<T, D>, dim3((unsigned)((pl.rows + 7) / 8)), 256, 0, s, a, pl.rows);
    if (e != cudaSuccess) return e;
    count_launches(1);
  }
  return cudaSuccess;
}

template <typename T, int D>
cudaError_t launch_halves(const vc_cross_params& r, const Plan& pl, CrossArgs& a, const void* q, const void* k, const void* v, cudaStream_t s) {
  return pl.tiles_per_item == 1 ? launch_cross<T, D, true>(r, pl, a, q, k, v, s) : launch_cross<T, D, false>(r, pl, a, q, k, v, s);
}

}  // namespace
}  // namespace vc

using namespace vc;

extern "C" size_t vc_cross_workspace_bytes(const vc_cross_params* p) {
  vc_cross_params r;
  Plan pl;
  return resolve(p, &r, &pl) == VC_OK ? pl.total : 0;
}

extern "C" vc_status vc_cross_attn(const vc_cross_params* p, const void* q, const void* k, const void* v, const int32_t* kv_len,
                                   const uint8_t* key_mask, void* o, float* lse, void* workspace, void* stream) {
  vc_cross_params r;
  Plan pl;
  const vc_status st = resolve(p, &r, &pl);
  if (st != VC_OK) return st;
  if (!q || !o || !workspace || (r.N_kv > 0 && (!k || !v))) return VC_ERR_INVALID_ARG;
  if (misaligned16(q) || misaligned16(k) || misaligned16(v) || misaligned16(o) || misaligned16(workspace) || ((uintptr_t)kv_len & 3) ||
      ((uintptr_t)lse & 3))
    return VC_ERR_INVALID_ARG;
  CrossArgs a{};
  a.o = o; a.lse = lse; a.kv_len = kv_len; a.key_mask = key_mask;
  a.status = (uint32_t*)workspace;
  a.part_o = (float*)((uint8_t*)workspace + pl.part_o);
  a.part_lse = (float*)((uint8_t*)workspace + pl.part_lse);
  a.so = r.o;
  a.heads = r.B * r.H; a.H = r.H; a.group = r.H / r.H_kv; a.Nq = r.N_q; a.Nkv = r.N_kv;
  a.qtiles = pl.qtiles; a.qitems = pl.qitems; a.tiles_per_item = pl.tiles_per_item; a.splits = pl.splits; a.joined = pl.joined; a.items = (int)pl.items;
  a.sl = r.softmax_scale * kLog2e;
  a.limit = attn::attn_wait_limit();
  a.nonblocking = attn::attn_wait_nonblocking();
  cudaStream_t s = (cudaStream_t)stream;
  cudaError_t e;
  if (r.dtype == VC_DTYPE_BF16) e = r.d == 128 ? launch_halves<__nv_bfloat16, 128>(r, pl, a, q, k, v, s) : launch_halves<__nv_bfloat16, 64>(r, pl, a, q, k, v, s);
  else e = r.d == 128 ? launch_halves<__half, 128>(r, pl, a, q, k, v, s) : launch_halves<__half, 64>(r, pl, a, q, k, v, s);
  return e == cudaSuccess ? VC_OK : VC_ERR_CUDA;
}
