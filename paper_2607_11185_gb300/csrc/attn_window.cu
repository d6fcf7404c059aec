// attn_window.cu - causal grouped-query attention with a sliding window and sinks, forward, over packed
// variable-length segments, for sm_103a (tcgen05 + TMEM + TMA).
//
// Token i of a segment sees token j of it for j <= i and (i - j < window or j < sinks):
//   s_ij = scale <q_i, k_j>,  o_i = sum_j softmax_j(s_ij) v_j,  lse_i = ln sum_j exp(s_ij)
// over the visible j.  Every row sees itself, so no row is empty.
//
// Work unit: two 128-row query tiles that stream the same key tiles.  Where a kv head serves two or more
// query heads they are the same rows of two heads, whose key tiles are the same ones; of an odd group's
// last head, or a single head, they are two consecutive row tiles (m, m + 1), which share all but one
// tile at each end of the window.  A block of two row tiles of one kv head is G units either way.
// A unit's key tiles: those of the sinks, then those from the window of its first row to the diagonal.
// Masked element-wise: the diagonal tile, the tiles the window's edge crosses, and the sinks' tiles
// outside the window.
//
// What bounds it is the chain of one tile, softmax, P V and next S, beside the other tile's: about 1.6 us a step
// at 28/4/128 of 1.1 that the MMAs of both take, and 2.6 us a unit besides, for which a CTA of its own took longer
// (512 segments of 256: 0.84 ms in the causal kernel, 0.46 here).  So
// a CTA stays on its SM and takes every grid-th unit: barriers and TMEM are set up once, the ring of K/V
// tiles runs on across units, the next unit's Q is loaded once the last S of this one is complete, and
// warps of their own write its O while the softmax warps are at the next one's first tile.
// 28/4/128, 32 segments of 4,096, window 128 / 1,024: 0.55 / 1.41 ms (0.78 / 1.66 with O written by the softmax
// warps, masks compared column by column and one issuer).
//
// Warp roles (512 threads):
//   warp 0      TMA producer: Q0/Q1 of a unit, K and V tiles into a ring (K runs one tile ahead of V)
//   warp 1      TMEM allocator and tcgen05.mma issuer of tile 0; at d = 64 of both tiles' S
//   warp 2      issuer of tile 1; at d = 64 of both tiles' P V
//   warps 4-7   softmax of tile 0 (thread = query row);  warps 8-11 of tile 1
//   warps 12-15 O of both tiles, out of TMEM, scaled, through shared memory, by a bulk copy a row
// TMEM (512 columns): S0, S1 (128 each), O0 and O1 from 256 and 384 on.  d = 128: P_k goes over the first
// 64 columns of S_k; d = 64: it has 64 columns of its own behind O_k.  P is read straight from TMEM.
// d = 128, step j of a tile: O_k += P_k(j) V_j, then S_k(j+1), which overwrites P_k(j): the MMAs of one issuer
// execute in order, as the causal kernel relies on too, so S_k(j+1) complete also says that P_k(j) has been
// consumed, O_k is up to date and V_j no longer read by the tile.  d = 64: S_k(j+1) as soon as S_k(j)
// has been read, by one warp, and P V by another.
#include <cfloat>
#include <cstdint>

#include "internal.h"
#include "sm100.cuh"

namespace vcs {
namespace {

using namespace dev;

constexpr int kThreads = 512;
constexpr int kRegLaunch = 128;  // registers per thread of the block, which its warpgroups then trade
constexpr float kRescaleThreshold = 8.0f;  // log2 units a row's maximum may grow before O is rescaled
constexpr float kHidden = -INFINITY;

template <int D>
struct Win {
  static constexpr int BM = 128;
  static constexpr int BN = 128;
  static constexpr int KB = D / 64;                 // 128-byte column blocks per row
  static constexpr int TILE = BM * D * 2;           // bytes of a 128 x D bf16 tile
  static constexpr int BLOCK = BM * 128;            // bytes of one 128 x 64 column block
  static constexpr bool OWN_P = D == 64;            // P in TMEM columns of its own
  static constexpr int NSLOT = OWN_P ? 8 : 4;
  static constexpr int NGRP = 4;                    // ring-item group barriers
  static constexpr int OFF_Q0 = 0;
  static constexpr int OFF_Q1 = TILE;
  static constexpr int OFF_KV = 2 * TILE;
  // A tile's O on its way out.  Rows are 16 bytes apart, so that threads on neighbouring rows write to other
  // banks; the 16 bytes hold the row's 1 / l of each tile.
  static constexpr int OFF_OUT = OFF_KV + NSLOT * TILE;
  static constexpr int OUT_ROW = D * 2 + 16;
  static constexpr int OFF_BAR = OFF_OUT + BM * OUT_ROW;
  static constexpr int SMEM = OFF_BAR + 512;
  static constexpr int TM_S0 = 0, TM_S1 = 128, TM_O0 = 256, TM_O1 = 384;
  static constexpr int TM_P0 = OWN_P ? TM_O0 + 64 : TM_S0, TM_P1 = OWN_P ? TM_O1 + 64 : TM_S1;
  static constexpr uint32_t IDESC_S = idesc_bf16(128, 128, 0, 0);   // Q (K-major) x K^T (K-major)
  static constexpr uint32_t IDESC_PV = idesc_bf16(128, D, 0, 1);    // P (TMEM) x V (MN-major)
  // with 64 for the issuers a d = 128 step took 10% longer while one warp issued for both tiles
  static constexpr int REG_CTRL = 80, REG_OUT = 48, REG_SOFTMAX = 192;
  static_assert(REG_CTRL + REG_OUT + 2 * REG_SOFTMAX <= 4 * kRegLaunch,
                "setmaxnreg targets exceed the launch registers");
};
static_assert(Win<64>::SMEM <= 232448 && Win<128>::SMEM <= 232448, "shared memory budget");

struct Bars {
  uint64_t q_full;       // a unit's Q tiles landed
  uint64_t q_free;       // its last S is complete
  uint64_t kv_full[8];   // per ring slot (OWN_P)
  uint64_t kv_empty[8];
  uint64_t grp_full[4];  // per group of ring items consumed in one step (without OWN_P)
  uint64_t s_full[2];
  uint64_t s_read[2];    // OWN_P: S(j) is in the softmax warps' registers
  uint64_t p_full[2];
  uint64_t o_done[2];    // the unit's last P V is complete; OWN_P: every step's
  uint64_t l_full[2];    // the unit's 1 / l are written (and, OWN_P, all but the last o_done have passed)
  uint64_t o_free[2];    // the unit's O has been read out of TMEM
  uint32_t tmem_base;
  int32_t abort;
};
static_assert(sizeof(Bars) <= 512, "barrier space");

// workspace header: the number of listed work units sits after the status word
constexpr size_t kWsItemTotal = 128;

// Bulk copies of a thread's own: shared memory to global (16-byte aligned), and the wait until all that it
// has committed have been read from shared memory.
__device__ __forceinline__ void bulk_store(void* dst, uint32_t src, uint32_t bytes) {
  asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(src), "r"(bytes)
               : "memory");
}
__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
__device__ __forceinline__ void bulk_wait_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }

__device__ __forceinline__ void on_timeout(Bars* b, int32_t* status) {
  set_status(status, VCS_ERR_DEVICE_TIMEOUT);
  *reinterpret_cast<volatile int32_t*>(&b->abort) = 1;
}
__device__ __forceinline__ bool aborted(Bars* b) { return *reinterpret_cast<volatile int32_t*>(&b->abort) != 0; }

// S = Q K^T; qd, kd are K-major descriptors of the Q tile and the K tile.
template <int D>
__device__ __forceinline__ void issue_s(uint32_t tmem_d, uint64_t qd, uint64_t kd) {
  using C = Win<D>;
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) {
    const uint32_t off = (kk >> 2) * C::BLOCK + (kk & 3) * 32;
    tc_mma_ss(tmem_d, desc_at(qd, off), desc_at(kd, off), C::IDESC_S, kk > 0);
  }
}

// O (+)= P V with P (128 x 128 keys, bf16) in TMEM; vd is the MN-major descriptor of the V tile.
template <int D>
__device__ __forceinline__ void issue_pv(uint32_t tmem_d, uint32_t p_tmem, uint64_t vd, bool accumulate) {
  using C = Win<D>;
  const uint32_t acc0 = accumulate ? 1u : 0u;
#pragma unroll
  for (int kk = 0; kk < C::BN / 16; ++kk)
    tc_mma_ts(tmem_d, p_tmem + kk * 8, desc_at(vd, kk * 16 * 128), C::IDESC_PV, kk > 0 ? 1u : acc0);
}

// ------------------------------------------------------------------ work units
// A unit as listed: {segment start, segment end, 2 * (row tile of tile 0) + (its tiles are two heads), head
// of tile 0}.
__device__ __forceinline__ long long seg_units(const int32_t* __restrict__ cu_seqlens, int32_t num_segments,
                                         int32_t num_tokens, int32_t max_seqlen, int32_t G, int s, int32_t* status) {
  const int start = cu_seqlens[s], end = cu_seqlens[s + 1];
  if (start < 0 || end < start || end > num_tokens || end - start > max_seqlen || (s == 0 && start != 0) ||
      (s == num_segments - 1 && end != num_tokens)) {
    set_status(status, VCS_ERR_DEVICE_CHECK);
    return 0;
  }
  const int tiles = (end - start + 127) / 128;
  return (long long)(tiles >> 1) * G + (tiles & 1) * ((G + 1) >> 1);  // of one kv head
}

// The units of segment s at items[base ..], by threads tid of n: kv head by kv head, blocks of two row tiles in order,
// so that the units running together share their key tiles in L2.  A segment whose units would pass the capacity
// writes none.
__device__ __forceinline__ void write_units(const int32_t* __restrict__ cu_seqlens, int32_t num_segments,
                                            int32_t num_tokens, int32_t max_seqlen, int32_t hkv, int32_t G,
                                            int32_t capacity, long long base, int4* __restrict__ items,
                                            int32_t* status, int s, int tid, int n) {
  const long long one = seg_units(cu_seqlens, num_segments, num_tokens, max_seqlen, G, s, status);
  const long long units = hkv * one;
  if (one == 0 || base + units > capacity) return;
  const int per = (int)one;
  const int start = cu_seqlens[s], end = cu_seqlens[s + 1];
  const int tiles = (end - start + 127) / 128, pairs = G >> 1;
  for (int i = tid; i < (int)units; i += n) {
    const int g = i / per, u = i - g * per;
    const int p = u / G, r = u - p * G;                 // block of two row tiles, unit of it
    const bool half = 2 * p + 1 >= tiles;               // the last block may be one tile
    const int pair = half ? r : r >> 1;                 // (an odd group's last head has r = 2 * pairs, or pairs)
    const bool two = pair < pairs;
    const int m = 2 * p + (two && !half ? r & 1 : 0);
    items[base + i] = make_int4(start, end, 2 * m + (two ? 1 : 0), g * G + 2 * pair);
  }
}

// off[s] = units of segments 0 .. s-1 (clipped to the capacity), *total = their sum, or 0 where it passes the
// capacity: only segments that overlap, which inconsistent bounds describe, list so many, and no CTA then
// reads a unit that was not written.  The call's first kernel: it clears the status word.  items != nullptr:
// it writes the units too, a warp a segment.
__global__ void __launch_bounds__(1024) window_unit_scan(const int32_t* __restrict__ cu_seqlens, int32_t num_segments,
                                                         int32_t num_tokens, int32_t max_seqlen, int32_t hkv, int32_t G,
                                                         int32_t capacity, int32_t* off, int32_t* __restrict__ total,
                                                         int4* __restrict__ items, int32_t* status) {
  __shared__ long long wsum[32];
  __shared__ long long carry;
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  if (threadIdx.x == 0) {
    carry = 0;
    *reinterpret_cast<volatile int32_t*>(status) = VCS_OK;
  }
  __syncthreads();
  for (int base = 0; base < num_segments; base += 1024) {
    const int s = base + (int)threadIdx.x;
    const long long cnt =
        s < num_segments
            ? hkv * seg_units(cu_seqlens, num_segments, num_tokens, max_seqlen, G, s, status)
            : 0;
    long long x = cnt;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    if (lane == 31) wsum[wid] = x;
    __syncthreads();
    if (wid == 0) {
      long long w = wsum[lane];
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long y = __shfl_up_sync(0xffffffffu, w, o);
        if (lane >= o) w += y;
      }
      wsum[lane] = w;
    }
    __syncthreads();
    const long long incl = carry + (wid > 0 ? wsum[wid - 1] : 0) + x;
    if (s < num_segments) off[s] = (int32_t)(incl - cnt < capacity ? incl - cnt : capacity);
    __syncthreads();
    if (threadIdx.x == 1023) carry = incl;
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    const int32_t t = carry <= capacity ? (int32_t)carry : 0;
    if (carry > capacity) set_status(status, VCS_ERR_DEVICE_CHECK);
    off[num_segments] = t;
    *total = t;
  }
  if (items == nullptr) return;
  __syncthreads();
  for (int s = wid; s < num_segments; s += 32)
    write_units(cu_seqlens, num_segments, num_tokens, max_seqlen, hkv, G, capacity, off[s], items, status, s, lane, 32);
}

__global__ void __launch_bounds__(256) window_unit_fill(const int32_t* __restrict__ cu_seqlens, int32_t num_segments,
                                                        int32_t num_tokens, int32_t max_seqlen, int32_t hkv, int32_t G,
                                                        int32_t capacity, const int32_t* __restrict__ off,
                                                        int4* __restrict__ items, int32_t* status) {
  for (int s = blockIdx.x; s < num_segments; s += gridDim.x)
    write_units(cu_seqlens, num_segments, num_tokens, max_seqlen, hkv, G, capacity, off[s], items, status, s,
                threadIdx.x, blockDim.x);
}

// What every role derives from a listed unit.  Step j takes key tile kt(j): the sinks' first `ns` tiles, then
// lo, lo + 1, ...  Tile 0 takes steps j < n0; tile 1 (if has1) all but `skip`, the window's first tile where
// two row tiles share a unit and none of its keys is visible to the second.
struct Unit {
  int start, L, h[2], m[2], ns, lo, nkv, n0, skip;
  bool has1;
  __device__ __forceinline__ Unit(int4 e, int window, int sinks) {
    start = e.x;
    L = e.y - e.x;
    const bool two = e.z & 1;
    m[0] = e.z >> 1;
    m[1] = two ? m[0] : m[0] + 1;
    h[0] = e.w;
    h[1] = two ? e.w + 1 : e.w;
    has1 = two || m[1] * 128 < L;
    const int last = has1 ? m[1] : m[0];
    lo = max(0, m[0] * 128 - window + 1) >> 7;
    ns = min((sinks >> 7) + ((sinks & 127) != 0), lo);
    nkv = ns + last - lo + 1;
    n0 = nkv - (last - m[0]);
    skip = !two && has1 && (max(0, m[1] * 128 - window + 1) >> 7) > lo && lo * 128 >= sinks ? ns : -1;
  }
  __device__ __forceinline__ int kt(int j) const { return j < ns ? j : j - ns + lo; }
  __device__ __forceinline__ bool active(int t, int j) const { return t == 0 ? j < n0 : has1 && j != skip; }
  __device__ __forceinline__ int end(int t) const { return t == 0 ? n0 : nkv; }       // behind the tile's last step
  __device__ __forceinline__ int after(int t, int j) const { return t == 1 && j + 1 == skip ? j + 2 : j + 1; }
  // ring items of the unit in load order: K0, K1, V0, K2, V1, ..., K_{n-1}, V_{n-2}, V_{n-1}
  __device__ __forceinline__ int k_item(int j) const { return j == 0 ? 0 : 2 * j - 1; }
  __device__ __forceinline__ int v_item(int j) const { return j == nkv - 1 ? 2 * nkv - 1 : 2 * j + 2; }
};

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
    attn_window_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                       const __grid_constant__ CUtensorMap tm_v, const int4* __restrict__ items,
                       const int32_t* __restrict__ item_total, int32_t num_tokens, int32_t hq, int32_t hkv,
                       int32_t window, int32_t sinks, float scale_log2, __nv_bfloat16* __restrict__ out,
                       float* __restrict__ lse, int32_t* status) {
  using C = Win<D>;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = smem_raw;
  Bars* bars = reinterpret_cast<Bars*>(smem + C::OFF_BAR);

  const int G = hq / hkv;
  const int total = *item_total;
  const int st = *reinterpret_cast<volatile int32_t*>(status);
  if ((int)blockIdx.x >= total) return;  // the grid is bounded by an upper bound of the listed units
  // Once any CTA of this launch has given up on a wait, those not started stand down.  The word may be set between two
  // threads' reads: one of them decides for all.
  if (__syncthreads_or(threadIdx.x == 0 && st == VCS_ERR_DEVICE_TIMEOUT)) return;
  // The tiles' 128-byte swizzle wants 1,024-byte aligned blocks.  A kernel without static shared memory gets
  // its dynamic shared memory so aligned; there is no room to align it here.
  if (smem_u32(smem) & 1023u) {
    if (threadIdx.x == 0) set_status(status, VCS_ERR_CUDA);
    return;
  }

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t sbase = smem_u32(smem);

  if (threadIdx.x == 0) {
    mbar_init(&bars->q_full, 1);
    mbar_init(&bars->q_free, C::OWN_P ? 1 : 2);
    for (int i = 0; i < C::NSLOT; ++i) {
      mbar_init(&bars->kv_full[i], 1);
      mbar_init(&bars->kv_empty[i], 2);  // one for each tile
    }
    for (int i = 0; i < C::NGRP; ++i) mbar_init(&bars->grp_full[i], 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bars->s_full[i], 1);
      mbar_init(&bars->s_read[i], 4);
      mbar_init(&bars->p_full[i], 128);
      mbar_init(&bars->o_done[i], 1);
      mbar_init(&bars->l_full[i], 128);
      mbar_init(&bars->o_free[i], 4);
    }
    bars->abort = 0;
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc(&bars->tmem_base, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = bars->tmem_base;

  // Every role walks the same units and counts what it has passed: ring items (`ib`) and groups (`gb`) before
  // the unit, units (`un`), and per tile the steps taken.
  if (warp < 4) {
    setmaxnreg_dec<C::REG_CTRL>();
    if (warp == 0 && lane == 0) {
    // ------------------------------------------------------------ producer
      tma_prefetch_desc(&tm_q);
      tma_prefetch_desc(&tm_k);
      tma_prefetch_desc(&tm_v);
      const uint64_t keep_l2 = l2_policy_evict_last();
      uint32_t ib = 0, gb = 0, un = 0;
      bool go = true;
      int4 e = items[blockIdx.x];
      for (int i = blockIdx.x; go && i < total; i += gridDim.x) {
        const Unit u(e, window, sinks);
        if (i + (int)gridDim.x < total) e = items[i + gridDim.x];
        for (int c = 0; c < 2 * u.nkv; ++c) {
          const bool is_v = c == 2 * u.nkv - 1 || (c > 0 && (c & 1) == 0);
          const int j = c == 2 * u.nkv - 1 ? u.nkv - 1 : (is_v ? (c - 2) >> 1 : (c + 1) >> 1);
          const uint32_t it = ib + c, slot = it % C::NSLOT;
          if ((it >= C::NSLOT && !mbar_wait(&bars->kv_empty[slot], (it / C::NSLOT - 1) & 1))) {
            on_timeout(bars, status);
            go = false;
            break;
          }
          if (aborted(bars)) {
            go = false;
            break;
          }
          // Without OWN_P items 2m-1, 2m of the unit (K_m, V_{m-1}), which step m-1 consumes, complete one
          // barrier, armed for both by the first; group 0 (K_0) and group nkv (V_{nkv-1}) hold one item
          const int m = (c + 1) >> 1;
          uint64_t* bar = C::OWN_P ? &bars->kv_full[slot] : &bars->grp_full[(gb + m) % C::NGRP];
          if (C::OWN_P)
            mbar_arrive_expect_tx(bar, C::TILE);
          else if (c == 0 || (c & 1))
            mbar_arrive_expect_tx(bar, (m == 0 || m == u.nkv ? 1 : 2) * C::TILE);
          const CUtensorMap* tm = is_v ? &tm_v : &tm_k;
#pragma unroll
          for (int kb = 0; kb < C::KB; ++kb)
            tma_load_3d_hint(smem + C::OFF_KV + slot * C::TILE + kb * C::BLOCK, tm, bar, kb * 64, u.h[0] / G,
                             u.start + u.kt(j) * C::BN, keep_l2);
          if (c == 0) {  // Q behind the first K, which needs no wait for the unit before
            if (un > 0 && !mbar_wait(&bars->q_free, (un - 1) & 1)) {
              on_timeout(bars, status);
              go = false;
              break;
            }
            mbar_arrive_expect_tx(&bars->q_full, (u.has1 ? 2 : 1) * C::TILE);
#pragma unroll
            for (int kb = 0; kb < C::KB; ++kb) {
              tma_load_3d(smem + C::OFF_Q0 + kb * C::BLOCK, &tm_q, &bars->q_full, kb * 64, u.h[0],
                          u.start + u.m[0] * C::BM);
              if (u.has1)
                tma_load_3d(smem + C::OFF_Q1 + kb * C::BLOCK, &tm_q, &bars->q_full, kb * 64, u.h[1],
                            u.start + u.m[1] * C::BM);
            }
          }
        }
        ib += 2 * u.nkv;
        gb += u.nkv + 1;
        ++un;
      }
    } else if (C::OWN_P && (warp == 1 || warp == 2)) {
    // ---------------------------------------------------- MMA issuers (S; P V)
      const uint64_t q0d = smem_desc(sbase + C::OFF_Q0, 16, 1024);
      const uint64_t kv_kmaj = smem_desc(sbase + C::OFF_KV, 16, 1024);
      const uint64_t kv_mnmaj = smem_desc(sbase + C::OFF_KV, C::BLOCK, 1024);
      // A wait can run out between two lanes' reads, so no lane's answer decides where the warp goes:
      // every lane runs every step, one that has given up waits no more, and the elected lane issues as
      // long as its own waits were met.  A vote a unit ends the walk.
      bool ok = true;
      uint32_t ib = 0, un = 0, steps[2] = {0, 0}, outs[2] = {0, 0};
      int4 e = items[blockIdx.x];
      for (int i = blockIdx.x; i < total; i += gridDim.x) {
        const Unit u(e, window, sinks);
        if (i + (int)gridDim.x < total) e = items[i + gridDim.x];
        if (warp == 1) ok = ok && mbar_wait(&bars->q_full, un & 1);
        if (!__all_sync(0xffffffffu, ok)) break;
        for (int j = 0; j < u.nkv; ++j) {
          const uint32_t it = ib + (warp == 1 ? u.k_item(j) : u.v_item(j)), slot = it % C::NSLOT;
          ok = ok && mbar_wait(&bars->kv_full[slot], (it / C::NSLOT) & 1);
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            if (!u.active(t, j)) continue;
            if (warp == 1) {
              if (steps[t] > 0) ok = ok && mbar_wait(&bars->s_read[t], (steps[t] - 1) & 1);
              tc_fence_after();
              if (elect_one() && ok) {
                issue_s<D>(tmem + (t ? C::TM_S1 : C::TM_S0), desc_at(q0d, t * C::TILE),
                           desc_at(kv_kmaj, slot * C::TILE));
                tc_commit(&bars->s_full[t]);
              }
            } else {
              const bool more = j > (t == 1 && u.skip == 0 ? 1 : 0);
              ok = ok && mbar_wait(&bars->p_full[t], steps[t] & 1);
              if (!more) {  // O of the unit before has been read
                if (outs[t] > 0) ok = ok && mbar_wait(&bars->o_free[t], (outs[t] - 1) & 1);
                ++outs[t];
              }
              tc_fence_after();
              if (elect_one() && ok) {
                issue_pv<D>(tmem + (t ? C::TM_O1 : C::TM_O0), tmem + (t ? C::TM_P1 : C::TM_P0),
                            desc_at(kv_mnmaj, slot * C::TILE), more);
                tc_commit(&bars->o_done[t]);
              }
            }
            __syncwarp();
            ++steps[t];
          }
        }
        if (warp == 1) {
          if (elect_one() && ok) tc_commit(&bars->q_free);
          __syncwarp();
        }
        ib += 2 * u.nkv;
        ++un;
      }
      if (!ok) on_timeout(bars, status);
    } else if (!C::OWN_P && (warp == 1 || warp == 2)) {
    // ---------------------------------------------------- MMA issuers (tile 0; tile 1)
    // The whole warp runs the loop and one elected lane issues, so that descriptors and addresses stay in
    // uniform registers.  As above, no lane's answer decides where the warp goes; here a vote a step does.
    // A warp a tile: a barrier wait takes its thread 200 to 300 cycles while the pipe streams from shared
    // memory, and there are two or three a step, which the other tile's MMAs now cover.
      const int t = warp - 1;
      bool ok = true;
      const uint64_t qd = desc_at(smem_desc(sbase + C::OFF_Q0, 16, 1024), t * C::TILE);
      const uint64_t kv_kmaj = smem_desc(sbase + C::OFF_KV, 16, 1024);
      const uint64_t kv_mnmaj = smem_desc(sbase + C::OFF_KV, C::BLOCK, 1024);
      const uint32_t tm_s = tmem + (t ? C::TM_S1 : C::TM_S0), tm_o = tmem + (t ? C::TM_O1 : C::TM_O0);
      uint32_t ib = 0, gb = 0, un = 0, steps = 0, outs = 0;  // outs: units that have this tile
      auto acquire_group = [&](uint32_t g) {
        ok &= mbar_wait(&bars->grp_full[g % C::NGRP], (g / C::NGRP) & 1);
        tc_fence_after();
      };
      int4 e = items[blockIdx.x];
      for (int i = blockIdx.x; i < total; i += gridDim.x) {
        const Unit u(e, window, sinks);
        if (i + (int)gridDim.x < total) e = items[i + gridDim.x];
        auto slot_off = [&](int item) { return (uint32_t)(((ib + item) % C::NSLOT) * C::TILE); };
        ok &= mbar_wait(&bars->q_full, un & 1);
        const int first = t == 1 && u.skip == 0 ? 1 : 0, end = u.end(t);
        if (t == 0 || u.has1) {
          acquire_group(gb + first);
          if (!__all_sync(0xffffffffu, ok)) break;
          // S of the first step overwrites the P that the last P V of the unit before, issued before, reads
          if (elect_one() && ok) {
            issue_s<D>(tm_s, qd, desc_at(kv_kmaj, slot_off(u.k_item(first))));
            tc_commit(&bars->s_full[t]);
            if (u.after(t, first) >= end) tc_commit(&bars->q_free);
          }
          __syncwarp();
          for (int j = first; j < end; j = u.after(t, j)) {
            // O += P(j) V_j, then S of the tile's next step; K and V are in groups j + 1 and, of a step that was
            // skipped to, next
            const int next = u.after(t, j);
            acquire_group(gb + j + 1);
            if (next < end && next > j + 1) acquire_group(gb + next);
            ok &= mbar_wait(&bars->p_full[t], steps++ & 1);
            if (j == first && outs > 0) ok &= mbar_wait(&bars->o_free[t], (outs - 1) & 1);  // O of the unit before read
            if (!__all_sync(0xffffffffu, ok)) break;
            tc_fence_after();
            const uint32_t vaddr = slot_off(u.v_item(j)), kaddr = next < end ? slot_off(u.k_item(next)) : 0u;
            if (elect_one() && ok) {
              issue_pv<D>(tm_o, tm_s, desc_at(kv_mnmaj, vaddr), j > first);
              if (next < end) {
                issue_s<D>(tm_s, qd, desc_at(kv_kmaj, kaddr));
                tc_commit(&bars->s_full[t]);
                if (u.after(t, next) >= end) tc_commit(&bars->q_free);  // the unit's last S
              } else {
                tc_commit(&bars->o_done[t]);
              }
            }
            __syncwarp();
          }
          ++outs;
        } else {
          if (elect_one() && ok) mbar_arrive(&bars->q_free);
          __syncwarp();
        }
        if (!__all_sync(0xffffffffu, ok)) break;
        ib += 2 * u.nkv;
        gb += u.nkv + 1;
        ++un;
      }
      if (!ok) on_timeout(bars, status);
    }
  } else if (warp < 12) {
    // ------------------------------------------------------------ softmax
    setmaxnreg_inc<C::REG_SOFTMAX>();
    const int wg = (warp - 4) >> 2;
    const int quad = warp & 3;
    const int r = quad * 32 + lane;  // query row within the tile
    const uint32_t trow = tmem + ((uint32_t)(quad * 32) << 16);
    const uint32_t s_col = wg == 0 ? C::TM_S0 : C::TM_S1;
    const uint32_t o_col = wg == 0 ? C::TM_O0 : C::TM_O1;
    const uint32_t p_col = wg == 0 ? C::TM_P0 : C::TM_P1;
    const uint64_t sc2 = f2pack(scale_log2, scale_log2);
    float* inv_s = reinterpret_cast<float*>(smem + C::OFF_OUT + r * C::OUT_ROW + D * 2) + wg;
    uint32_t ib = 0, steps = 0, un = 0;
    bool ok = true;
    int4 e = items[blockIdx.x];
    for (int i = blockIdx.x; ok && i < total; i += gridDim.x) {
      const Unit u(e, window, sinks);
      if (i + (int)gridDim.x < total) e = items[i + gridDim.x];
      if (wg == 1 && !u.has1) {
        ib += 2 * u.nkv;
        continue;
      }
      const int mt = u.m[wg];
      float m_run = kHidden, l = 0.f;
      // The ring slots are handed back from here rather than by commits of the MMA threads (a commit holds its thread
      // about as long as an MMA): once S(j) of a tile is complete, so is what its issuer issued before, which with
      // K_j is done, and without OWN_P with the V of the tile's step before (with it, o_done says so of V).  A slot
      // is free when both tiles have given it back, each for the steps it takes, or twice if it takes one alone.
      const bool releaser = quad == 0 && lane == 0;
      auto release = [&](int item, int j) {
        mbar_arrive(&bars->kv_empty[(ib + item) % C::NSLOT]);
        if (!u.active(wg ^ 1, j)) mbar_arrive(&bars->kv_empty[(ib + item) % C::NSLOT]);
      };
      int prev = -1;  // the tile's step before
      bool first = true;
      for (int j = 0; j < u.nkv; ++j) {
        if (!u.active(wg, j)) continue;
        // Without OWN_P, S(j) complete also means that the P before it was consumed and O is up to date.  The
        // wait's outcome is the warp's: the TMEM loads and votes below are warp-collective.
        if (!mbar_wait_warp(&bars->s_full[wg], steps & 1)) { ok = false; break; }
        ++steps;
        if (releaser) {
          release(u.k_item(j), j);
          if (!C::OWN_P && prev >= 0) release(u.v_item(prev), prev);
        }
        tc_fence_after();
        uint32_t s[128];
#pragma unroll
        for (int c = 0; c < 4; ++c)
          tmem_ld_32x32b_x32(trow + s_col + c * 32, *reinterpret_cast<uint32_t(*)[32]>(&s[c * 32]));
        tmem_ld_wait();
        reg_fence<128>(s);
        if constexpr (C::OWN_P) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&bars->s_read[wg]);
        }
        // Column c of key tile kt is ahead of row r if c > r + ahead, and behind its window if
        // c <= r + ahead - window, unless it is a sink (c < keep).  A bit a column says what the row sees, so that a
        // masked tile takes two instructions an element and shares the rest of the code with the others: code of
        // its own for masked tiles, which leaves out the exponentials of hidden columns, made the warps wait for
        // instructions (28/4/128, 32 segments of 4,096, window 256: 1.09 ms against 0.77).
        const int kt = u.kt(j);
        const int ahead = (mt - kt) * 128, keep = sinks - kt * 128;
        if (ahead == 0 || (ahead + 127 >= window && keep < 128)) {
          auto low = [](int n) { return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u; };
          const int last = r + ahead;
#pragma unroll
          for (int ch = 0; ch < 4; ++ch) {
            const int c0 = 32 * ch;
            const uint32_t seen = low(last + 1 - c0) & (~low(last - window + 1 - c0) | low(keep - c0));
#pragma unroll
            for (int c = 0; c < 32; ++c)
              if (!(seen >> c & 1)) s[c0 + c] = __float_as_uint(kHidden);
          }
        }
        // row maximum: 8 independent three-input chains
        float pm[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) pm[x] = fmaxf(__uint_as_float(s[2 * x]), __uint_as_float(s[2 * x + 1]));
#pragma unroll
        for (int c = 16; c < 128; c += 16)
#pragma unroll
          for (int x = 0; x < 8; ++x)
            pm[x] = fmax3(pm[x], __uint_as_float(s[c + 2 * x]), __uint_as_float(s[c + 2 * x + 1]));
        const float mx = fmax3(fmax3(pm[0], pm[1], pm[2]), fmax3(pm[3], pm[4], pm[5]), fmaxf(pm[6], pm[7]));
        const float mx2 = mx * scale_log2;
        float alpha = 1.f;
        bool rescale = false;
        if (first) {
          m_run = mx2;
        } else if (mx2 > m_run + kRescaleThreshold) {
          alpha = ex2(m_run - mx2);  // 0 where the tiles before were hidden from the row
          m_run = mx2;
          rescale = true;
        }
        // P = exp2(s*scale*log2e - m) as bf16 pairs, the type of V, which the tensor pipe multiplies it with; l sums
        // it unrounded.  The roundings, half a step each, are as many as the row's keys and average out: o is 2.1e-3
        // in norm from 64 bits where its own last rounding alone leaves 1.6e-3.  A row that has seen nothing yet
        // subtracts 0 and gets zeros.
        const float shift = m_run == kHidden ? 0.f : -m_run;
        const uint64_t nm2 = f2pack(shift, shift);
        uint64_t acc[4] = {0ull, 0ull, 0ull, 0ull};
#pragma unroll
        for (int c2 = 0; c2 < 64; ++c2) {
          float x0, x1;
          f2unpack(ffma2(f2pack(__uint_as_float(s[2 * c2]), __uint_as_float(s[2 * c2 + 1])), sc2, nm2), x0, x1);
          const float p0 = ex2(x0), p1 = ex2(x1);
          acc[c2 & 3] = fadd2(acc[c2 & 3], f2pack(p0, p1));
          s[c2] = pack_bf16(p0, p1);
        }
        float a0, a1, b0, b1;
        f2unpack(fadd2(acc[0], acc[1]), a0, a1);
        f2unpack(fadd2(acc[2], acc[3]), b0, b1);
        l = l * alpha + ((a0 + a1) + (b0 + b1));
        if (C::OWN_P && steps > 1) {  // the P V before is complete: P's columns are free and O is up to date
          if (!mbar_wait_warp(&bars->o_done[wg], steps & 1)) { ok = false; break; }
          if (releaser && prev >= 0) release(u.v_item(prev), prev);
          tc_fence_after();
        }
        tmem_st_32x32b_x32(trow + p_col, *reinterpret_cast<uint32_t(*)[32]>(&s[0]));
        tmem_st_32x32b_x32(trow + p_col + 32, *reinterpret_cast<uint32_t(*)[32]>(&s[32]));
        if (!first && __any_sync(0xffffffffu, rescale)) {
          const uint64_t al2 = f2pack(alpha, alpha);
#pragma unroll
          for (int c = 0; c < D / 32; ++c) {
            uint32_t o[32];
            tmem_ld_32x32b_x32(trow + o_col + c * 32, o);
            tmem_ld_wait();
            reg_fence<32>(o);
#pragma unroll
            for (int x = 0; x < 32; x += 2) {
              float x0, x1;
              f2unpack(fmul2(f2pack(__uint_as_float(o[x]), __uint_as_float(o[x + 1])), al2), x0, x1);
              o[x] = __float_as_uint(x0);
              o[x + 1] = __float_as_uint(x1);
            }
            tmem_st_32x32b_x32(trow + o_col + c * 32, o);
          }
        }
        tmem_st_wait();
        tc_fence_before();
        mbar_arrive(&bars->p_full[wg]);
        first = false;
        prev = j;
      }
      // another role's giving up is looked for once a unit; the waits are bounded without it
      if (ok && __any_sync(0xffffffffu, aborted(bars))) ok = false;
      // 1 / l of the unit before has been read, and its l_full waited for
      if (ok && un > 0) ok = mbar_wait_warp(&bars->o_free[wg], (un - 1) & 1);
      if (!ok) break;
      ib += 2 * u.nkv;
      *inv_s = 1.f / l;
      mbar_arrive(&bars->l_full[wg]);
      ++un;
      const int row = mt * C::BM + r;
      if (row < u.L)
        lse[(size_t)u.h[wg] * num_tokens + u.start + row] = (m_run + lg2(l)) * 0.69314718055994531f;
    }
    if (!ok) on_timeout(bars, status);
  } else {
    // ------------------------------------------------------------ O
    setmaxnreg_dec<C::REG_OUT>();
    const int quad = warp & 3;
    const int r = quad * 32 + lane;
    const uint32_t trow = tmem + ((uint32_t)(quad * 32) << 16);
    const uint32_t stage = sbase + C::OFF_OUT + r * C::OUT_ROW;
    uint32_t ib = 0, un[2] = {0, 0}, steps[2] = {0, 0};
    bool ok = true;
    int4 e = items[blockIdx.x];
    for (int i = blockIdx.x; ok && i < total; i += gridDim.x) {
      const Unit u(e, window, sinks);
      if (i + (int)gridDim.x < total) e = items[i + gridDim.x];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if (t == 1 && !u.has1) continue;
        steps[t] += t == 0 ? u.n0 : u.nkv - (u.skip >= 0 ? 1 : 0);
        // o_done of the unit's last step: behind l_full, all phases before it have passed
        if (!mbar_wait_warp(&bars->l_full[t], un[t] & 1) ||
            !mbar_wait_warp(&bars->o_done[t], (C::OWN_P ? steps[t] - 1 : un[t]) & 1)) {
          ok = false;
          break;
        }
        tc_fence_after();
        // the tile is done with its last V
        if (quad == 0 && lane == 0) {
          const int j = u.end(t) - 1;
          mbar_arrive(&bars->kv_empty[(ib + u.v_item(j)) % C::NSLOT]);
          if (!u.active(t ^ 1, j)) mbar_arrive(&bars->kv_empty[(ib + u.v_item(j)) % C::NSLOT]);
        }
        const float inv_l = reinterpret_cast<const float*>(smem + C::OFF_OUT + r * C::OUT_ROW + D * 2)[t];
        const uint64_t il2 = f2pack(inv_l, inv_l);
        bulk_wait_read();  // the thread's row of the tile before has left the staging buffer
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          uint32_t o[32];
          tmem_ld_32x32b_x32(trow + (t ? C::TM_O1 : C::TM_O0) + c * 32, o);
          tmem_ld_wait();
          reg_fence<32>(o);
          if (c == D / 32 - 1) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars->o_free[t]);
          }
          uint32_t pk[16];
#pragma unroll
          for (int x = 0; x < 16; ++x) {
            float x0, x1;
            f2unpack(fmul2(f2pack(__uint_as_float(o[2 * x]), __uint_as_float(o[2 * x + 1])), il2), x0, x1);
            pk[x] = pack_bf16(x0, x1);
          }
#pragma unroll
          for (int v4 = 0; v4 < 4; ++v4)
            st_shared_v4(stage + c * 64 + v4 * 16, pk[4 * v4], pk[4 * v4 + 1], pk[4 * v4 + 2], pk[4 * v4 + 3]);
        }
        fence_proxy_async_smem();
        const int row = u.m[t] * C::BM + r;
        if (row < u.L)
          bulk_store(out + ((size_t)(u.start + row) * hq + u.h[t]) * D, stage, D * 2);
        bulk_commit();
        ++un[t];
      }
      ib += 2 * u.nkv;
    }
    bulk_wait_read();  // shared memory outlives the copies that read it
    if (!ok) on_timeout(bars, status);
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

inline size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

// Upper bound of a launch's units: a segment of t row tiles lists hkv (G floor(t / 2) + (t odd) ceil(G / 2))
// <= hq (L / 256 + 1), so they fit the causal forward's list of hq (T / 256 + S + 1).
template <int D>
cudaError_t launch_window_d(const AttnArgs& a, void* o, float* lse, void* ws, cudaStream_t st) {
  using C = Win<D>;
  alignas(64) CUtensorMap tq, tk, tv;
  if (!encode_tma_3d_bf16(&tq, a.q, D, a.hq, a.num_tokens, 64, 128) ||
      !encode_tma_3d_bf16(&tk, a.k, D, a.hkv, a.num_tokens, 64, 128) ||
      !encode_tma_3d_bf16(&tv, a.v, D, a.hkv, a.num_tokens, 64, 128))
    return cudaErrorInvalidValue;
  static std::atomic<int> regs_cache{-1};
  bool regs_ok = false;
  if (cudaError_t e = launch_regs_match(reinterpret_cast<const void*>(attn_window_kernel<D>), kRegLaunch, &regs_cache,
                                        &regs_ok);
      e != cudaSuccess)
    return e;
  if (!regs_ok) return cudaErrorInvalidConfiguration;
  cudaError_t e = cudaFuncSetAttribute(attn_window_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
  if (e != cudaSuccess) return e;
  const int64_t max_items = (int64_t)a.hq * (a.num_tokens / 256 + (int64_t)a.num_segments + 1);
  if (max_items > INT32_MAX) return cudaErrorInvalidConfiguration;
  char* w = static_cast<char*>(ws);
  int32_t* total = reinterpret_cast<int32_t*>(w + kWsItemTotal);
  int32_t* off = reinterpret_cast<int32_t*>(w + kWsHeader);
  int4* items = reinterpret_cast<int4*>(w + kWsHeader + align256(((size_t)a.num_segments + 1) * 4));
  // small launches list their units in the scan's launch, as the causal forward does
  const bool one = max_items <= 2048 && a.num_segments <= 64;
  const int G = a.hq / a.hkv;
  window_unit_scan<<<1, 1024, 0, st>>>(a.cu_seqlens, a.num_segments, (int32_t)a.num_tokens, a.max_seqlen, a.hkv, G,
                                       (int32_t)max_items, off, total, one ? items : nullptr, a.status);
  if (!one) {
    const int fill_blocks = a.num_segments < 152 * 8 ? a.num_segments : 152 * 8;
    window_unit_fill<<<fill_blocks, 256, 0, st>>>(a.cu_seqlens, a.num_segments, (int32_t)a.num_tokens, a.max_seqlen,
                                                  a.hkv, G, (int32_t)max_items, off, items, a.status);
  }
  const unsigned grid = (unsigned)(max_items < 152 ? max_items : 152);
  const int32_t longest = a.max_seqlen > 1 ? a.max_seqlen : 1;  // as far as either reaches; the kernel's sums stay in range
  const int32_t window = a.window < longest ? a.window : longest, sinks = a.sinks < longest ? a.sinks : longest;
  attn_window_kernel<D><<<grid, kThreads, C::SMEM, st>>>(
      tq, tk, tv, items, total, (int32_t)a.num_tokens, a.hq, a.hkv, window, sinks, a.scale * 1.4426950408889634f,
      static_cast<__nv_bfloat16*>(o), lse, a.status);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_attn_fwd_window(const AttnArgs& a, void* o, float* lse, void* ws, cudaStream_t st) {
  if (a.d == 64) return launch_window_d<64>(a, o, lse, ws, st);
  return launch_window_d<128>(a, o, lse, ws, st);
}

}  // namespace vcs
