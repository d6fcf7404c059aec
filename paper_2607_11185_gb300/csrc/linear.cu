// linear.cu - linear attention with a decay for each key/value head, over packed variable-length segments, sm_103a.
//
// With lam = exp(log_decay) of the head, over the tokens t of a segment:
//   S_t = lam S_{t-1} + k_t v_t^T,   o_t = scale q_t^T S_t
// Its gradients are sums of the same kind: with R_t = lam R_{t+1} + sum_group q_t do_t^T,
//   dq_t = scale S_t do_t   (the same call: queries do, keys v, values k)
//   dk_t = scale R_t v_t,  dv_t = scale R_t^T k_t   (linear_back, from the last token to the first)
//
// Chunks of 128 tokens.  From the state S before a chunk's first token, for its n tokens i, j = 0 .. n - 1:
//   o_i = scale [ lam^(i+1) q_i S + sum_{j <= i} lam^(i-j) (q_i . k_j) v_j ],
//   S'  = lam^n S + sum_j lam^(n-1-j) k_j v_j^T
// four 128-wide products a chunk on the tensor pipe.
//
// Operands of the tensor pipe are bf16: the inputs as they are, the products between a chunk's tokens, the factor that the
// decay weighs, and the copy of the state that a chunk's queries read.  Between a chunk's tokens two such roundings meet an
// output, through the state two others; with its own they leave 0.0029 of a result's norm where its own alone leaves 0.0017.
// One of each less leaves 0.0024 and was measured in two forms, over one rollout of 246,616 tokens at 40 / 8 heads of 128,
// forward, where this takes 1,055 us, and a training step over 102,936 at 14 / 2 of 64, 441: a second bf16 term of the
// weighted V in a tile of its own (at D = 128 in the place of the next chunk's K), 1,338 and 474; the decay's factors in P, V
// as it is, and K weighted late with its second term over the state's copy, 1,203 and 482.  Neither helps dK and dV at
// D = 128, where shared memory has no room.  The state itself, all sums and the states that are results are fp32.
//
// A "sequence" is one segment of one head.  The chunks of all sequences, one after another, are divided evenly among
// the CTAs; a sequence that a CTA's range ends in goes on in the next one, which needs the state at the cut.
// linear_states adds up the keys and values before every cut, as far back as the decay leaves anything in fp32, in
// parts of equal size spread over the chip, and linear_join makes the cuts' states of them.  So a cut costs its
// piece's keys and values read twice.  (A CTA that adds up the piece before its own cut takes as long as the head that
// forgets slowest: the three passes of a training step over the rollout above 955 us, the parts 480 with what joins them.)
//
// That rollout, us: the outputs 940 (6.06 GB, 6.45 TB/s), the states at the cuts 74 for K and V, 283 for a
// group's Q and dO (about 6 TB/s of what the decays leave of them) and 16 to join them, dK and dV 1,465.

#include <cfloat>
#include <cstdint>

#include "internal.h"
#include "sm100.cuh"

namespace vcs {
namespace {

using namespace dev;
using bf16 = __nv_bfloat16;

constexpr int kGrid = 152;   // a CTA an SM
constexpr int kChunk = 128;
// Sequences up to this many chunks are not cut where all are: a CTA takes those that start in its range.
constexpr int kWhole = 16;

// (the lowest decays would be -inf as a log2, and not a number times 0 tokens)
__device__ __forceinline__ float log2_decay(float g) { return fmaxf(g * 1.4426950408889634f, -1e30f); }
__device__ __forceinline__ bool decay_ok(float g) { return g <= 0.f && g >= -FLT_MAX; }

// ------------------------------------------------------------------ division of the work
constexpr int kFade = 150;   // a weight of 2^-150 and less is 0 in fp32
constexpr int kWaves = 3;    // parts to a CTA, at most
constexpr int kPartCost = 3; // of a part, in chunks: its first loads and its sum's way out

// Chunks of a head with the log2 decay l2 behind which a key's weight is 0.
__device__ __forceinline__ int fade_chunks(float l2) {
  const float far = kFade / fabsf(l2 * kChunk);   // l2 = 0: infinite
  return far < 1e8f ? (int)far + 2 : 1 << 30;
}

struct Plan {        // in the workspace, behind the header
  int64_t total;     // chunks of all sequences
  int64_t range;     // of a CTA
  int32_t cut;       // sequences are cut at the ranges' ends
  int32_t part[2];   // chunks of a part, in order and the other way in time
  int32_t pad;
  // Of the cut behind range t: chunks whose keys and values its state needs, and the parts before it (the last: all).
  int32_t need[2][kGrid], first[2][kGrid + 1];
};

__device__ __forceinline__ int seg_chunks(const int32_t* __restrict__ cu, int32_t num_tokens, int s, int32_t* status) {
  const int start = cu[s], end = cu[s + 1];
  if (start < 0 || end < start || end > num_tokens) {
    set_status(status, VCS_ERR_DEVICE_CHECK);
    return 0;
  }
  return (end - start + kChunk - 1) / kChunk;
}

// off[s] = chunks of segments 0 .. s - 1, and the plan.  The call's first kernel: it clears the status word.
__global__ void __launch_bounds__(1024) linear_plan(const int32_t* __restrict__ cu, int32_t num_segments,
                                                    int32_t num_tokens, int32_t heads, int32_t grid,
                                                    const float* __restrict__ log_decay, int32_t* off, Plan* plan,
                                                    int32_t* status) {
  __shared__ long long wsum[32], s_total, s_range;
  __shared__ int need[2][kGrid], s_part[2][kWaves];
  __shared__ long long carry;
  __shared__ int longest;
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  if (threadIdx.x == 0) {
    carry = 0;
    longest = 0;
    *reinterpret_cast<volatile int32_t*>(status) = VCS_OK;
  }
  __syncthreads();
  const long long most = (long long)num_tokens / kChunk + num_segments;  // segments that overlap may pass it
  for (int base = 0; base < num_segments; base += 1024) {
    const int s = base + (int)threadIdx.x;
    const int n = s < num_segments ? seg_chunks(cu, num_tokens, s, status) : 0;
    if (n > 0) atomicMax(&longest, n);
    long long x = n;
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
    if (s < num_segments) off[s] = (int32_t)(incl - n < most ? incl - n : most);
    __syncthreads();
    if (threadIdx.x == 1023) carry = incl;
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    if (carry > most) set_status(status, VCS_ERR_DEVICE_CHECK);
    const long long all = carry > most ? 0 : carry * heads;
    off[num_segments] = (int32_t)(carry > most ? 0 : carry);
    s_total = plan->total = all;
    s_range = plan->range = (all + grid - 1) / grid;
    plan->cut = longest > kWhole;
  }
  if (num_tokens <= kWhole * kChunk) return;   // no sequence is so long
  __syncthreads();
  const long long total = s_total, range = s_range;
  const bool cut = longest > kWhole;
  if (threadIdx.x < kGrid) {
    const int t = threadIdx.x;
    const long long g = range * (t + 1);
    int fwd = 0, bwd = 0;
    if (cut && g < total) {   // the sequence that chunk g is in
      const int q = (int)(g / heads);
      int lo = 0, up = num_segments;
      while (up - lo > 1) {
        const int mid = (lo + up) >> 1;
        if (off[mid] <= q) lo = mid;
        else up = mid;
      }
      const int first = off[lo], nch = off[lo + 1] - first;
      const long long rest = g - (long long)first * heads, base = (long long)first * heads + rest / nch * nch;
      const float ld = log_decay[rest / nch], l2 = log2_decay(ld);
      if (g > base && decay_ok(ld)) {
        const int keep = fade_chunks(l2);
        const long long back = g - (g - range > base ? g - range : base);
        const long long end = base + nch < total ? base + nch : total, ahead = (g + range < end ? g + range : end) - g;
        fwd = (int)(back < keep ? back : keep);
        bwd = (int)(ahead < keep ? ahead : keep);
      }
    }
    need[0][t] = plan->need[0][t] = fwd;
    need[1][t] = plan->need[1][t] = bwd;
  }
  __syncthreads();
  // The smallest parts that make one, two or three to a CTA: a warp each, for both directions.
  const int d = wid & 1;
  if (wid < 2 * kWaves) {
    const int most_parts = (wid / 2 + 1) * grid;
    int lo = 4, up = 4;   // up is enough: no more than one part a cut
    for (int t = lane; t < kGrid; t += 32) up = max(up, need[d][t]);
    up = __reduce_max_sync(0xffffffffu, up);
    while (lo < up) {
      const int mid = (lo + up) >> 1;
      int n = 0;
      for (int t = lane; t < kGrid; t += 32) n += (need[d][t] + mid - 1) / mid;
      n = __reduce_add_sync(0xffffffffu, n);
      if (n <= most_parts) up = mid;
      else lo = mid + 1;
    }
    if (lane == 0) s_part[d][wid / 2] = up;
  }
  __syncthreads();
  if (wid < 2) {
    int part = s_part[d][0];
    for (int i = 1, best = part + kPartCost; i < kWaves; ++i)
      if ((i + 1) * (s_part[d][i] + kPartCost) < best) {
        part = s_part[d][i];
        best = (i + 1) * (part + kPartCost);
      }
    int carry = 0;
    for (int t0 = 0; t0 < kGrid; t0 += 32) {
      const int t = t0 + lane, n = t < kGrid ? (need[d][t] + part - 1) / part : 0;
      int x = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
      }
      if (t < kGrid) plan->first[d][t] = carry + x - n;
      carry += __shfl_sync(0xffffffffu, x, 31);
    }
    if (lane == 0) {
      plan->first[d][kGrid] = carry;
      plan->part[d] = part;
    }
  }
}

struct Common {
  const float* log_decay;
  const int32_t* cu;
  const int32_t* off;
  const Plan* plan;
  int32_t num_segments, num_tokens, heads;
  int32_t* status;
};

// The pieces of CTA b's range, one after another: chunks c0 .. c1 of a sequence.
struct Walk {
  const Common& a;
  int64_t g, hi, base, range;
  int seg, head, nch, start, len, c0, c1;
  float l2;     // log2 of the decay
  bool cut, located;
  __device__ __forceinline__ Walk(const Common& a, int b) : a(a) {
    const int64_t total = a.plan->total;
    range = a.plan->range;
    cut = a.plan->cut != 0;
    g = range * b < total ? range * b : total;
    hi = range * (b + 1) < total ? range * (b + 1) : total;
    located = false;
  }
  __device__ __forceinline__ void locate(int64_t at) {  // the sequence that holds chunk `at` < total
    const int q = (int)(at / a.heads);
    int lo = 0, up = a.num_segments;  // off[lo] <= q < off[up]
    while (up - lo > 1) {
      const int mid = (lo + up) >> 1;
      if (__ldg(&a.off[mid]) <= q) lo = mid;
      else up = mid;
    }
    seg = lo;
    const int first = __ldg(&a.off[seg]);
    nch = __ldg(&a.off[seg + 1]) - first;
    const int64_t rest = at - (int64_t)first * a.heads;
    head = (int)(rest / nch);
    base = (int64_t)first * a.heads + (int64_t)head * nch;
    bounds();
    located = true;
  }
  __device__ __forceinline__ void bounds() {
    start = __ldg(&a.cu[seg]);
    len = __ldg(&a.cu[seg + 1]) - start;
  }
  __device__ __forceinline__ bool next() {
    while (true) {
      if (g >= hi) return false;
      if (!located) {
        locate(g);
        if (!cut && g != base) {  // it started in an earlier range
          g = base + nch;
          if (g >= hi) return false;
          advance();
        }
      } else {
        advance();
      }
      c0 = (int)(g - base);
      c1 = cut && hi - base < nch ? (int)(hi - base) : nch;
      g = base + c1;
      const float ld = __ldg(&a.log_decay[head]);
      l2 = log2_decay(ld);
      if (decay_ok(ld)) return true;
      set_status(a.status, VCS_ERR_DEVICE_CHECK);
    }
  }
  __device__ __forceinline__ void advance() {  // to the sequence behind this one
    base += nch;
    if (++head < a.heads) return;
    head = 0;
    do ++seg;
    while (__ldg(&a.off[seg + 1]) == __ldg(&a.off[seg]));
    nch = __ldg(&a.off[seg + 1]) - __ldg(&a.off[seg]);
    bounds();
  }
  __device__ __forceinline__ int rows(int c) const { return min(kChunk, len - c * kChunk); }
};

// ------------------------------------------------------------------ shared pieces
__device__ __forceinline__ void tma_store_3d(const void* map, uint32_t src, int x, int y, int z) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(map),
               "r"(src), "r"(x), "r"(y), "r"(z)
               : "memory");
}
__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
__device__ __forceinline__ void bulk_wait_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }

__device__ __forceinline__ void set_abort(int32_t* abort, int32_t* status) {
  set_status(status, VCS_ERR_DEVICE_TIMEOUT);
  *reinterpret_cast<volatile int32_t*>(abort) = 1;
}

// What a block has under way when it has given up on a wait ends before it.  (Otherwise somebody has waited for all of it.)
// Of `n` loads into `slots` slots, the last ones:
__device__ __forceinline__ void finish_loads(uint64_t* full, uint32_t n, uint32_t slots) {
  for (uint32_t i = n > slots ? n - slots : 0; i < n; ++i) mbar_wait(&full[i % slots], (i / slots) & 1);
}
__device__ __forceinline__ void finish_mmas(uint64_t* idle) {   // the issuer's whole warp
  if (elect_one()) tc_commit(idle);
  __syncwarp();
  mbar_wait(idle, 0);
}

__device__ __forceinline__ float lo_f(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Row r of a 128 x D tile (64-column blocks of 128-byte rows) set to zero.
template <int D>
__device__ __forceinline__ void zero_row(uint32_t tile, int r) {
#pragma unroll
  for (int kb = 0; kb < D / 64; ++kb)
#pragma unroll
    for (int u = 0; u < 8; ++u) st_shared_v4(tile + kb * 16384 + r * 128 + (((u + r) & 7) << 4), 0u, 0u, 0u, 0u);
}

// ------------------------------------------------------------------ states of the pieces
// TERMS: bf16 terms that a weighted key is split into.  Where the states are results (state_out) there are three,
// which hold its 24 bits; where queries read them, rounded to bf16 themselves, one.
struct StateArgs {
  Common c;
  float* slots;            // [parts][D][D]; state_out != nullptr: every piece of the ranges, a slot a CTA
  const float* state_in;
  float* state_out;
  int32_t group;           // key heads of a state
  bool back;
};

template <int D, int TERMS>
struct Sta {
  static constexpr int TILE = kChunk * D * 2;
  static constexpr int NKV = (TERMS == 1 ? 3 : 2) * (D == 64 ? 2 : 1);
  static constexpr int OFF_KV = 0;
  static constexpr int OFF_TERM = NKV * 2 * TILE;        // second and third term of a weighted key tile
  // at D = 64 the upper lanes of an MMA (see Lin) read a tile further than the last term
  static constexpr int OFF_BAR = OFF_TERM + (TERMS == 1 ? 0 : D == 64 ? 3 : 2) * TILE;
  static constexpr int SMEM = OFF_BAR + 512;
  static constexpr uint32_t IDESC_U = idesc_bf16(128, D, 1, 1);
  static constexpr int REG_CTRL = 80, REG_ROWS = 96, REG_STATE = 224;
  static_assert(REG_CTRL + 2 * REG_ROWS + REG_STATE <= 512, "setmaxnreg targets exceed the launch registers");
  static_assert(SMEM <= 232448, "shared memory budget");
};

struct StaBars {
  uint64_t kv_full[6], kv_empty[6];
  uint64_t kt_full[6][2];  // the weighted keys of a slot's first and second 64 tokens are written
  uint64_t term_free[2];   // and read
  uint64_t u_full[2], u_free[2];
  uint64_t idle;           // given up: all MMAs are complete
  uint32_t loads;
  uint32_t tmem_base;
  int32_t abort;
};
static_assert(sizeof(StaBars) <= 512, "barrier space");

constexpr int kStaThreads = 512;

template <int D, int TERMS>
__global__ void __launch_bounds__(kStaThreads, 1)
    linear_states(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                  const __grid_constant__ StateArgs p) {
  using C = Sta<D, TERMS>;
  extern __shared__ __align__(1024) uint8_t smem[];
  StaBars* bars = reinterpret_cast<StaBars*>(smem + C::OFF_BAR);
  Walk w(p.c, blockIdx.x);
  const bool all = p.state_out != nullptr;
  const Plan& plan = *p.c.plan;
  const int parts = all || !w.cut ? 0 : plan.first[p.back][kGrid];
  if (all ? w.g >= w.hi : (int)blockIdx.x >= parts) return;
  if (smem_u32(smem) & 1023u) {
    if (threadIdx.x == 0) set_status(p.c.status, VCS_ERR_CUDA);
    return;
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t sbase = smem_u32(smem);
  if (threadIdx.x == 0) {
    for (int i = 0; i < C::NKV; ++i) {
      mbar_init(&bars->kv_full[i], 1);
      mbar_init(&bars->kv_empty[i], 1);
      mbar_init(&bars->kt_full[i][0], 128);
      mbar_init(&bars->kt_full[i][1], 128);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bars->term_free[i], 1);
      mbar_init(&bars->u_full[i], 1);
      mbar_init(&bars->u_free[i], 4);
    }
    mbar_init(&bars->idle, 1);
    bars->abort = 0;
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc(&bars->tmem_base, 256);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = bars->tmem_base;
  auto gave_up = [&] { return *reinterpret_cast<volatile int32_t*>(&bars->abort) != 0; };
  // The next piece: of the CTA's range, or every grid-th part of what the cuts need, from the cut outwards.
  int slot = (int)blockIdx.x - (int)gridDim.x;
  auto next = [&] {
    if (all) {
      slot = blockIdx.x;
      if (!w.next()) return false;
      w.c0 = max(w.c0, w.c1 - fade_chunks(w.l2));   // (what lies before a fade adds 0, a state that goes in too)
      return true;
    }
    slot += gridDim.x;
    if (slot >= parts) return false;
    int lo = 0, up = kGrid;   // first[lo] <= slot < first[up]
    while (up - lo > 1) {
      const int mid = (lo + up) >> 1;
      if (__ldg(&plan.first[p.back][mid]) <= slot) lo = mid;
      else up = mid;
    }
    const int64_t g = plan.range * (lo + 1);
    w.locate(g);
    w.l2 = log2_decay(__ldg(&p.c.log_decay[w.head]));
    const int size = plan.part[p.back], j = slot - __ldg(&plan.first[p.back][lo]), e = (int)(g - w.base);
    const int near = j * size, far = min(near + size, __ldg(&plan.need[p.back][lo]));
    w.c0 = p.back ? e + near : e - far;
    w.c1 = p.back ? e + far : e - near;
    return true;
  };

  if (warp < 4) {
    setmaxnreg_dec<C::REG_CTRL>();
    if (warp == 0) {
      // ---------------------------------------------------------- producer
      if (lane == 0) {
        bool go = true;
        uint32_t it = 0;
        while (go && next())
          for (int n = 0; go && n < w.c1 - w.c0; ++n) {
            const int c = p.back ? w.c1 - 1 - n : w.c0 + n;
            for (int h = 0; h < p.group; ++h, ++it) {
              const uint32_t slot = it % C::NKV;
              if ((it >= C::NKV && !mbar_wait(&bars->kv_empty[slot], (it / C::NKV - 1) & 1)) || gave_up()) {
                set_abort(&bars->abort, p.c.status);
                go = false;
                break;
              }
              mbar_arrive_expect_tx(&bars->kv_full[slot], 2 * C::TILE);
#pragma unroll
              for (int kb = 0; kb < D / 64; ++kb) {
                uint8_t* dst = smem + C::OFF_KV + slot * 2 * C::TILE + kb * 16384;
                tma_load_3d(dst, &tm_k, &bars->kv_full[slot], kb * 64, w.head * p.group + h, w.start + c * kChunk);
                tma_load_3d(dst + C::TILE, &tm_v, &bars->kv_full[slot], kb * 64, w.head * p.group + h,
                            w.start + c * kChunk);
              }
            }
          }
        bars->loads = it;
      }
    } else if (warp == 1) {
      // ---------------------------------------------------------- MMA issuer
      // Every lane runs every step and no lane's answer to a wait decides where the warp goes; a vote an item does.
      const uint64_t kd = smem_desc(sbase + C::OFF_KV, 16384, 1024), td = smem_desc(sbase + C::OFF_TERM, 16384, 1024);
      bool ok = true, go = true;
      uint32_t it = 0, un = 0;
      while (go && next())
        for (int n = 0; go && n < w.c1 - w.c0; ++n, ++un)
          for (int h = 0; h < p.group; ++h, ++it) {
            const uint32_t slot = it % C::NKV, buf = un & 1;
            if (h == 0 && un >= 2) ok = ok && mbar_wait(&bars->u_free[buf], (un / 2 - 1) & 1);
            for (int half = 0; half < 2; ++half) {
              ok = ok && mbar_wait(&bars->kt_full[slot][half], (it / C::NKV) & 1);
              tc_fence_after();
              if (elect_one() && ok) {
                const uint64_t a0 = desc_at(kd, slot * 2 * C::TILE + half * 8192), b = desc_at(a0, C::TILE);
#pragma unroll
                for (int t = TERMS - 1; t >= 0; --t)   // the smallest term first
#pragma unroll
                  for (int kk = 0; kk < 4; ++kk)
                    tc_mma_ss(tmem + buf * 128,
                              desc_at(t == 0 ? a0 : desc_at(td, (t - 1) * C::TILE + half * 8192), kk * 2048),
                              desc_at(b, kk * 2048), C::IDESC_U, h > 0 || half > 0 || t < TERMS - 1 || kk > 0);
                if (TERMS > 1) tc_commit(&bars->term_free[half]);
                if (half == 1) tc_commit(&bars->kv_empty[slot]);
                if (half == 1 && h == p.group - 1) tc_commit(&bars->u_full[buf]);
              }
              __syncwarp();
            }
            go = __all_sync(0xffffffffu, ok);
            if (!go) break;
          }
      if (!go) set_abort(&bars->abort, p.c.status);
    }
  } else if (warp < 12) {
    // ---------------------------------------------------------- weighted keys: a warpgroup's 64 tokens, two threads each
    setmaxnreg_dec<C::REG_ROWS>();
    const int half = warp < 8 ? 0 : 1, r = half * 64 + (threadIdx.x & 63), part = threadIdx.x >> 6 & 1;
    bool go = true;
    uint32_t it = 0;
    while (go && next())
      for (int n = 0; go && n < w.c1 - w.c0; ++n) {
        const int c = p.back ? w.c1 - 1 - n : w.c0 + n;
        const int rows = w.rows(c);
        const float wt = r < rows ? exp2f(w.l2 * (float)(p.back ? r : rows - 1 - r)) : 0.f;
        for (int h = 0; h < p.group; ++h, ++it) {
          const uint32_t slot = it % C::NKV, tile = sbase + C::OFF_KV + slot * 2 * C::TILE, term = sbase + C::OFF_TERM;
          if (!mbar_wait_warp(&bars->kv_full[slot], (it / C::NKV) & 1) ||
              (TERMS > 1 && it > 0 && !mbar_wait_warp(&bars->term_free[half], (it - 1) & 1)) ||
              __any_sync(0xffffffffu, gave_up())) {
            go = false;
            break;
          }
          // its part of a row: 8 vectors of the one 64-column block or the other, or 4 of the only one
          const uint32_t row = (D == 128 ? part * 16384 : 0) + r * 128;
          const int u0 = D == 128 ? 0 : part * 4;
#pragma unroll
          for (int i8 = 0; i8 < D / 16; ++i8) {
            const uint32_t at = row + (((u0 + i8 + r) & 7) << 4);
            if (r >= rows) {  // rows of the next segment, which may hold anything
              st_shared_v4(tile + at, 0u, 0u, 0u, 0u);
              st_shared_v4(tile + C::TILE + at, 0u, 0u, 0u, 0u);
#pragma unroll
              for (int t = 1; t < TERMS; ++t) st_shared_v4(term + (t - 1) * C::TILE + at, 0u, 0u, 0u, 0u);
              continue;
            }
            const uint4 x = ld_shared_v4(tile + at);
            const uint32_t in[4] = {x.x, x.y, x.z, x.w};
            uint32_t y[3][4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float a = lo_f(in[i]) * wt, b = hi_f(in[i]) * wt;
#pragma unroll
              for (int t = 0; t < TERMS; ++t) {
                y[t][i] = pack_bf16(a, b);
                a -= lo_f(y[t][i]);
                b -= hi_f(y[t][i]);
              }
            }
            st_shared_v4(tile + at, y[0][0], y[0][1], y[0][2], y[0][3]);
#pragma unroll
            for (int t = 1; t < TERMS; ++t)
              st_shared_v4(term + (t - 1) * C::TILE + at, y[t][0], y[t][1], y[t][2], y[t][3]);
          }
          fence_proxy_async_smem();
          mbar_arrive(&bars->kt_full[slot][half]);
        }
      }
    if (!go) set_abort(&bars->abort, p.c.status);
  } else {
    // ---------------------------------------------------------- sums, a thread a row of the state
    setmaxnreg_inc<C::REG_STATE>();
    const int quad = warp & 3, r = quad * 32 + lane;
    const uint32_t trow = tmem + ((uint32_t)(quad * 32) << 16);
    bool go = true;
    uint32_t un = 0;
    while (go && next()) {
      float s[D];
#pragma unroll
      for (int i = 0; i < D; ++i) s[i] = 0.f;
      const int last = min(w.len, w.c1 * kChunk);
      for (int n = 0; n < w.c1 - w.c0; ++n, ++un) {
        const int c = p.back ? w.c1 - 1 - n : w.c0 + n;
        // from the chunk's end to the piece's (or between their beginnings), at once: the factors do not add up errors
        const int gap = p.back ? (c - w.c0) * kChunk : last - (c * kChunk + w.rows(c));
        const float f = exp2f(w.l2 * (float)gap);
        if (!mbar_wait_warp(&bars->u_full[un & 1], (un / 2) & 1) || __any_sync(0xffffffffu, gave_up())) {
          go = false;
          break;
        }
        tc_fence_after();
        if (D == 128 || quad < 2) {
#pragma unroll
          for (int g = 0; g < D / 32; ++g) {
            uint32_t u[32];
            tmem_ld_32x32b_x32(trow + (un & 1) * 128 + g * 32, u);
            tmem_ld_wait();
            reg_fence<32>(u);
#pragma unroll
            for (int i = 0; i < 32; ++i) s[g * 32 + i] = fmaf(f, __uint_as_float(u[i]), s[g * 32 + i]);
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars->u_free[un & 1]);
      }
      if (!go) break;
      if (D == 128 || quad < 2) {
        float* dst;
        const size_t state = ((size_t)w.seg * p.c.heads + w.head) * D * D + (size_t)r * D;
        if (!all || w.c1 < w.nch) {   // for the cut
          dst = p.slots + ((size_t)slot * D + r) * D;
        } else {
          dst = p.state_out + state;
          if (p.state_in != nullptr && w.c0 == 0) {
            const float f = exp2f(w.l2 * (float)w.len);
#pragma unroll
            for (int i = 0; i < D; i += 4) {
              const float4 x = *reinterpret_cast<const float4*>(p.state_in + state + i);
              s[i] = fmaf(f, x.x, s[i]);
              s[i + 1] = fmaf(f, x.y, s[i + 1]);
              s[i + 2] = fmaf(f, x.z, s[i + 2]);
              s[i + 3] = fmaf(f, x.w, s[i + 3]);
            }
          }
        }
#pragma unroll
        for (int i = 0; i < D; i += 4)
          *reinterpret_cast<float4*>(dst + i) = make_float4(s[i], s[i + 1], s[i + 2], s[i + 3]);
      }
    }
    if (!go) set_abort(&bars->abort, p.c.status);
  }
  tc_fence_before();
  __syncthreads();
  if (gave_up()) {
    if (threadIdx.x == 0) finish_loads(bars->kv_full, bars->loads, C::NKV);
    if (warp == 1) finish_mmas(&bars->idle);
    __syncthreads();
  }
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem, 256);
  }
}

// ------------------------------------------------------------------ states at the cuts
struct JoinArgs {
  Common c;
  const float* slots;
  const float* state_in;
  float* starts;   // [grid][D][D]: of the cut behind range t
  bool back, all;  // all: a slot a CTA, the sum of its last piece
};

// A block a cut and 1,024 elements: the parts before it, the nearest first, until they have faded.
template <int D>
__global__ void __launch_bounds__(256) linear_join(const __grid_constant__ JoinArgs p) {
  const Plan& plan = *p.c.plan;
  const int t = blockIdx.x;
  if (!plan.cut || plan.need[p.back][t] == 0) return;
  Walk w(p.c, t);
  const int64_t g = plan.range * (t + 1);
  w.locate(g);
  const float l2 = log2_decay(__ldg(&p.c.log_decay[w.head]));
  const int size = plan.part[p.back], e = (int)(g - w.base);
  const size_t at = (size_t)blockIdx.y * 1024 + threadIdx.x * 4;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [&](const float* src, float f) {
    const float4 x = *reinterpret_cast<const float4*>(src + at);
    s.x = fmaf(f, x.x, s.x);
    s.y = fmaf(f, x.y, s.y);
    s.z = fmaf(f, x.z, s.z);
    s.w = fmaf(f, x.w, s.w);
  };
  bool faded = false;
  for (int x = t; !faded && x >= 0 && x < kGrid; p.back ? ++x : --x) {
    const int64_t gap = p.back ? plan.range * (x + 1) - g : g - plan.range * (x + 1);   // chunks between the cuts
    // in another sequence
    if (p.back ? plan.range * (x + 1) >= w.base + w.nch : plan.range * (x + 1) <= w.base) break;
    const int first = p.all ? x : plan.first[p.back][x], end = p.all ? x + 1 : plan.first[p.back][x + 1];
    for (int i = first; i < end; ++i) {
      const float f = exp2f(l2 * (float)((gap + (int64_t)(i - first) * size) * kChunk));
      faded = f == 0.f;
      if (faded) break;
      add(p.slots + (size_t)i * D * D, f);
    }
  }
  if (p.state_in != nullptr && !faded)
    add(p.state_in + ((size_t)w.seg * p.c.heads + w.head) * D * D, exp2f(l2 * (float)((int64_t)e * kChunk)));
  *reinterpret_cast<float4*>(p.starts + (size_t)t * D * D + at) = s;
}

// ------------------------------------------------------------------ outputs
struct OutArgs {
  Common c;
  const float* starts;     // the states at the cuts
  const float* state_in;
  float* state_out;
  int32_t group;           // query heads of a state
  float scale;
  bool wide;               // out is 32-byte aligned
  bf16* out;
};

// ONE: one query head to a key head, else a group of them.
template <int D, bool ONE>
struct Lin {
  static constexpr int TILE = kChunk * D * 2;
  // Tiles of Q, and of K and V, which take turns.  A load takes 2 to 4 thousand cycles under way and an item the
  // memory 3 to 6, so that what streams has to have two to three tiles on its way: a group of query heads streams Q,
  // one head of each K and V too.
  static constexpr int NQ = D == 64 ? 4 : ONE ? 1 : 2;
  static constexpr int NT = D == 64 ? 8 : ONE ? 4 : 3;
  // Buffers of Q K^T and P: two if K^T V and two outputs leave room.  Outputs: two.
  static constexpr int NP = D == 64 ? 2 : 1;
  static constexpr int NB = 2;
  static constexpr int OFF_Q = 0;
  static constexpr int OFF_T = NQ * TILE;
  static constexpr int OFF_O = OFF_T + NT * TILE;
  static constexpr int OFF_S = OFF_O + TILE;  // the state, D rows of k's dims, like a V tile
  static constexpr int OFF_TAB = OFF_S + D * D * 2;      // 32 powers of the decay for each warp that makes P
  static constexpr int OFF_BAR = OFF_TAB + 8 * 128;
  static constexpr int SMEM = OFF_BAR + 512;
  static constexpr int TM_P = 0, TM_B = NP * 128, TM_U = TM_B + NB * D;
  static constexpr uint32_t IDESC_S = idesc_bf16(128, 128, 0, 0);  // Q (K-major) x K^T (K-major)
  static constexpr uint32_t IDESC_A = idesc_bf16(128, D, 0, 1);    // Q (K-major) x S (MN-major)
  static constexpr uint32_t IDESC_B = idesc_bf16(128, D, 0, 1);    // P (TMEM) x V (MN-major)
  // K^T (MN-major) x V (MN-major).  M = 128 at D = 64 too, whose lanes 64 .. 127 take the tile behind K's (or the
  // state) and are not read: an M of 64 lies in other lanes.
  static constexpr uint32_t IDESC_U = idesc_bf16(128, D, 1, 1);
  static constexpr int REG_CTRL = 96, REG_ROWS = 104, REG_STATE = 208;
  static_assert(REG_CTRL + 2 * REG_ROWS + REG_STATE <= 512, "setmaxnreg targets exceed the launch registers");
  static_assert(SMEM <= 232448 && TM_U + D <= 512, "shared memory and TMEM budgets");
  static_assert(D == 128 || NT % 2 == 0, "behind a K tile lies another tile");
};

struct LinBars {
  uint64_t q_full[4], q_empty[4], t_full[8], t_empty[8];
  // Of an item or an output of one warpgroup and of the other:
  uint64_t s_full[2];  // Q K^T
  uint64_t p_full[2];  // its P is in TMEM
  uint64_t a_full[2];  // Q S, for the warpgroup that scales its rows
  uint64_t o_full[2];  // the products of an output are complete
  uint64_t o_free[2];  // and in registers
  uint64_t out_full;   // an output is in its tile, or its rows are written
  uint64_t out_free[2];  // and on its way, of one warpgroup's or the other's (each waits for the other's, in turn)
  uint64_t k_done;     // a K that is to be weighted is no longer read as it was loaded
  uint64_t wt_full[4]; // a pair's V, or K, is weighted; four, as the warps that do it may be some pairs ahead
  uint64_t u_full;     // the chunk's K^T V
  uint64_t u_free;     // and in registers
  uint64_t s_ready;    // the state that the chunk's queries read is in shared memory
  uint64_t s_read;     // and has been read
  uint64_t idle[2];    // given up: all MMAs of an issuer are complete
  uint32_t loads[2];   // of Q, and of K and V
  uint32_t tmem_base;
  int32_t abort;
};
static_assert(sizeof(LinBars) <= 512, "barrier space");

constexpr int kThreads = 512;
constexpr int kRegLaunch = 128;

// 32 bytes at p, which is 32-byte aligned (wide) or 16.
__device__ __forceinline__ void st_global_32(void* p, const uint32_t (&x)[8], bool wide) {
  if (!wide) {
    static_cast<uint4*>(p)[0] = make_uint4(x[0], x[1], x[2], x[3]);
    static_cast<uint4*>(p)[1] = make_uint4(x[4], x[5], x[6], x[7]);
    return;
  }
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(x[0]), "r"(x[1]), "r"(x[2]),
               "r"(x[3]), "r"(x[4]), "r"(x[5]), "r"(x[6]), "r"(x[7])
               : "memory");
}

// O is one accumulator for both terms: Q S first, then P V on top.  With m = 64, the middle of a chunk,
//   o_i = scale lam^(i+1-m) [ q_i (lam^m S) + sum_{j <= i} (q_i . k_j) w_j ],  w_j = lam^(m-1-j) v_j,
//   S'  = lam^n S + lam^(n-m) sum_j k_j w_j^T
// so that P = Q K^T below the diagonal has no factors at all, V is weighted once for both products, as soon as it is
// loaded, and the row's factor comes last, as long as lam^-m stays in range: 2^64 at most (kSlow).  For a head that
// forgets faster P has the exact powers, the rows of Q S are scaled in TMEM, and K is weighted for the state when Q
// K^T has read it.
constexpr int kMiddle = 64;
constexpr float kSlow = -1.0f;   // log2 of the decay

// An item is a chunk with one query head.  What bounds it is memory: Q in and O out, 64 KB an item at D = 128, 3,400
// cycles at the copy rate, of which the MMAs take 1,700.  Two warps issue them, as one is held up by its waits and
// commits (90 cycles a wait that is met): 975 -> 940 us a pass over one rollout at 40 / 8 heads of 128, 97 -> 86 over
// eight short ones at 14 / 2 of 64, where an item is 1,500 cycles of memory and takes 2,000.
// Warp roles:
//   warp 0       loads;  warp 2  O out of shared memory
//   warps 1, 3   MMAs: Q K^T and K^T V (and TMEM);  Q S and P V
//   warps 4-11   two warpgroups, for every other item: P below the diagonal, in bf16 for P V (a thread a query), then
//                O out of TMEM, scaled
//   warps 12-15  the weighted tiles, and the state in registers (a thread a row), its bf16 copy in shared memory
template <int D, bool ONE>
__global__ void __launch_bounds__(kThreads, 1)
    linear_out(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
               const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_o,
               const __grid_constant__ OutArgs p) {
  using C = Lin<D, ONE>;
  extern __shared__ __align__(1024) uint8_t smem[];
  LinBars* bars = reinterpret_cast<LinBars*>(smem + C::OFF_BAR);
  Walk w(p.c, blockIdx.x);
  // sequences without a token: their states go through
  if (p.state_out != nullptr)
    for (int s = blockIdx.x; s < p.c.num_segments; s += gridDim.x)
      if (p.c.cu[s] == p.c.cu[s + 1] && p.c.cu[s] >= 0 && p.c.cu[s] <= p.c.num_tokens) {
        const size_t n = (size_t)p.c.heads * D * D / 4, at = n * s;
        for (size_t i = threadIdx.x; i < n; i += kThreads) {
          const int head = (int)(i / (D * D / 4));
          if (!decay_ok(p.c.log_decay[head])) {
            set_status(p.c.status, VCS_ERR_DEVICE_CHECK);
            continue;
          }
          reinterpret_cast<float4*>(p.state_out)[at + i] =
              p.state_in != nullptr ? reinterpret_cast<const float4*>(p.state_in)[at + i]
                                    : make_float4(0.f, 0.f, 0.f, 0.f);
        }
      }
  if (w.g >= w.hi) return;
  // Once any CTA of this call has given up on a wait, those not started stand down.  The word may be set between two
  // threads' reads: one of them decides for all.
  if (__syncthreads_or(threadIdx.x == 0 && *reinterpret_cast<volatile int32_t*>(p.c.status) == VCS_ERR_DEVICE_TIMEOUT))
    return;
  if (smem_u32(smem) & 1023u) {  // the tiles' swizzle wants 1,024-byte aligned blocks
    if (threadIdx.x == 0) set_status(p.c.status, VCS_ERR_CUDA);
    return;
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t sbase = smem_u32(smem);
  if (threadIdx.x == 0) {
    for (int i = 0; i < C::NQ; ++i) {
      mbar_init(&bars->q_full[i], 1);
      mbar_init(&bars->q_empty[i], 2);
    }
    for (int i = 0; i < C::NT; ++i) {
      mbar_init(&bars->t_full[i], 1);
      mbar_init(&bars->t_empty[i], 2);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bars->s_full[i], 1);
      mbar_init(&bars->p_full[i], 4);
      mbar_init(&bars->a_full[i], 1);
      mbar_init(&bars->o_full[i], 1);
      mbar_init(&bars->o_free[i], 4);
      mbar_init(&bars->out_free[i], 1);
      mbar_init(&bars->idle[i], 1);
    }
    for (int i = 0; i < 4; ++i) mbar_init(&bars->wt_full[i], 128);
    mbar_init(&bars->k_done, 1);
    mbar_init(&bars->s_read, 1);
    mbar_init(&bars->out_full, 128);
    mbar_init(&bars->u_free, 4);
    mbar_init(&bars->u_full, 1);
    mbar_init(&bars->s_ready, 128);
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
  auto gave_up = [&] { return *reinterpret_cast<volatile int32_t*>(&bars->abort) != 0; };
  const int group = ONE ? 1 : p.group;
  // Every role walks the same items and counts what it has passed.

  if (warp < 4) {
    setmaxnreg_dec<C::REG_CTRL>();
    if (warp == 0 && lane == 0) {
      // -------------------------------------------------------- producer
      bool go = true;
      uint32_t qi = 0, ti = 0;
      auto load = [&](int off, uint64_t* full, uint64_t* empty, uint32_t& i, uint32_t n, const CUtensorMap* tm, int head,
                      int tok) {
        const uint32_t slot = i % n;
        if (!go || (i >= n && !mbar_wait(&empty[slot], (i / n - 1) & 1)) || gave_up()) {
          go = false;
          return;
        }
        mbar_arrive_expect_tx(&full[slot], C::TILE);
#pragma unroll
        for (int kb = 0; kb < D / 64; ++kb)
          tma_load_3d(smem + off + slot * C::TILE + kb * 16384, tm, &full[slot], kb * 64, head, tok);
        ++i;
      };
      while (go && w.next())
        for (int n = 0; go && n < w.c1 - w.c0; ++n) {
          const int tok = w.start + (w.c0 + n) * kChunk;
          for (int h = 0; go && h < group; ++h) {
            if (h == 0) load(C::OFF_T, bars->t_full, bars->t_empty, ti, C::NT, &tm_k, w.head, tok);
            load(C::OFF_Q, bars->q_full, bars->q_empty, qi, C::NQ, &tm_q, w.head * group + h, tok);
            if (h == 0) load(C::OFF_T, bars->t_full, bars->t_empty, ti, C::NT, &tm_v, w.head, tok);
          }
        }
      if (!go) set_abort(&bars->abort, p.c.status);
      bars->loads[0] = qi;
      bars->loads[1] = ti;
    } else if (warp == 1) {
      // -------------------------------------------------------- MMAs of Q K^T and of the state
      // Every lane of an issuer runs every step, no lane's answer to a wait decides where the warp goes, and a vote an
      // item ends the walk.  A chunk's K^T V comes behind its second item's Q K^T (its only one's): V is weighted by
      // then, and the next chunk's state is made while this one's queries are worked on; for a head that forgets fast
      // behind the last item's, when K is weighted.
      const uint64_t qd = smem_desc(sbase + C::OFF_Q, 16, 1024);
      const uint64_t kd = smem_desc(sbase + C::OFF_T, 16, 1024), kt = smem_desc(sbase + C::OFF_T, 16384, 1024);
      bool ok = true, go = true;
      uint32_t it = 0, ki = 0, us = 0;
      while (go && w.next()) {
        const int chunks = w.c1 - w.c0;
        const bool fast = w.l2 < kSlow;
        for (int n = 0; go && n < chunks; ++n, ++ki) {
          const bool weigh = n < chunks - 1;
          const uint32_t ks = 2 * ki % C::NT, vs = (2 * ki + 1) % C::NT;
          for (int h = 0; h < group; ++h, ++it) {
            const bool last = h == group - 1, state = weigh && h == (fast || group == 1 ? group - 1 : 1);
            const uint32_t q = it % C::NQ;
            if (h == 0) ok = ok && mbar_wait(&bars->t_full[ks], (2 * ki / C::NT) & 1);
            ok = ok && mbar_wait(&bars->q_full[q], (it / C::NQ) & 1);
            // its P was read
            if (it >= C::NP) ok = ok && mbar_wait(&bars->o_full[(it - C::NP) & 1], ((it - C::NP) >> 1) & 1);
            go = __all_sync(0xffffffffu, ok);
            if (!go) break;
            tc_fence_after();
            if (elect_one()) {
              const uint64_t a = desc_at(qd, q * C::TILE), d = desc_at(kd, ks * C::TILE);
#pragma unroll
              for (int kk = 0; kk < D / 16; ++kk) {
                const uint32_t off = (kk >> 2) * 16384 + (kk & 3) * 32;
                tc_mma_ss(tmem + C::TM_P + it % C::NP * 128, desc_at(a, off), desc_at(d, off), C::IDESC_S, kk > 0);
              }
              tc_commit(&bars->s_full[it & 1]);
              tc_commit(&bars->q_empty[q]);
              if (fast && weigh && last) tc_commit(&bars->k_done);
            }
            __syncwarp();
            if (state) {
              // (of a head that forgets fast K is weighted, and V may still be on its way)
              if (fast) ok = ok && mbar_wait(&bars->t_full[vs], ((2 * ki + 1) / C::NT) & 1);
              ok = ok && mbar_wait(&bars->wt_full[ki & 3], (ki >> 2) & 1);
              if (us++ > 0) ok = ok && mbar_wait(&bars->u_free, us & 1);
              tc_fence_after();
              if (elect_one() && ok) {
                const uint64_t a = desc_at(kt, ks * C::TILE), d = desc_at(kt, vs * C::TILE);
#pragma unroll
                for (int kk = 0; kk < 8; ++kk)
                  tc_mma_ss(tmem + C::TM_U, desc_at(a, kk * 2048), desc_at(d, kk * 2048), C::IDESC_U, kk > 0);
                tc_commit(&bars->u_full);
                tc_commit(&bars->t_empty[vs]);
              }
              __syncwarp();
            }
            if (last && elect_one() && ok) {   // a tile's slot takes two arrivals
              tc_commit(&bars->t_empty[ks]);
              tc_commit(&bars->t_empty[ks]);
              if (!weigh) tc_commit(&bars->t_empty[vs]);
            }
            __syncwarp();
          }
        }
      }
      go = __all_sync(0xffffffffu, ok);
      if (!go) set_abort(&bars->abort, p.c.status);
    } else if (warp == 3) {
      // -------------------------------------------------------- MMAs of the outputs: P V, Q S of the next item
      const uint64_t qd = smem_desc(sbase + C::OFF_Q, 16, 1024), vd = smem_desc(sbase + C::OFF_T, 16384, 1024);
      const uint64_t sd = smem_desc(sbase + C::OFF_S, D * 128, 1024);
      bool ok = true, go = true, more = w.next();
      uint32_t it = 0, ki = 0, qi = 0, ck = 0;   // items and chunks of P V, of Q S
      auto issue_a = [&](int h) {   // B = Q S
        const bool fast = w.l2 < kSlow;
        const uint32_t q = qi % C::NQ;
        if (h == 0) ok = ok && mbar_wait(&bars->s_ready, ck++ & 1);
        // the output before is in registers
        if (qi >= 2) ok = ok && mbar_wait(&bars->o_free[qi & 1], ((qi - 2) >> 1) & 1);
        ok = ok && mbar_wait(&bars->q_full[q], (qi / C::NQ) & 1);
        tc_fence_after();
        if (elect_one() && ok) {
          const uint64_t a = desc_at(qd, q * C::TILE);
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk)
            tc_mma_ss(tmem + C::TM_B + (qi & 1) * D, desc_at(a, (kk >> 2) * 16384 + (kk & 3) * 32), desc_at(sd, kk * 2048),
                      C::IDESC_A, kk > 0);
          tc_commit(&bars->q_empty[q]);
          if (fast) tc_commit(&bars->a_full[qi & 1]);
          if (h == group - 1) tc_commit(&bars->s_read);
        }
        __syncwarp();
        ++qi;
      };
      if (more) issue_a(0);
      while (go && more) {
        const int chunks = w.c1 - w.c0;
        const bool fast = w.l2 < kSlow;
        for (int n = 0; go && n < chunks; ++n, ++ki) {
          const bool weigh = n < chunks - 1;
          const uint32_t vs = (2 * ki + 1) % C::NT;
          for (int h = 0; h < group; ++h, ++it) {
            const bool last = h == group - 1;
            if (h == 0 && fast) ok = ok && mbar_wait(&bars->t_full[vs], ((2 * ki + 1) / C::NT) & 1);
            // (a fast head's last V is not weighted, but its slot is not given back before the warps that do it have
            // passed it)
            if (h == 0 && !(fast && weigh)) ok = ok && mbar_wait(&bars->wt_full[ki & 3], (ki >> 2) & 1);
            ok = ok && mbar_wait(&bars->p_full[it & 1], (it >> 1) & 1);
            go = __all_sync(0xffffffffu, ok);
            if (!go) break;
            tc_fence_after();
            if (elect_one()) {   // B += P V
              const uint64_t d = desc_at(vd, vs * C::TILE);
#pragma unroll
              for (int kk = 0; kk < 8; ++kk)
                tc_mma_ts(tmem + C::TM_B + (it & 1) * D, tmem + C::TM_P + it % C::NP * 128 + kk * 8, desc_at(d, kk * 2048),
                          C::IDESC_B, 1);
              tc_commit(&bars->o_full[it & 1]);
              if (last) tc_commit(&bars->t_empty[vs]);
            }
            __syncwarp();
            if (last && !weigh) more = w.next();
            if (!last || more) issue_a(last ? 0 : h + 1);
          }
        }
      }
      go = __all_sync(0xffffffffu, ok);
      if (!go) set_abort(&bars->abort, p.c.status);
    } else if (warp == 2 && lane == 0) {
      // -------------------------------------------------------- O out of shared memory
      bool go = true;
      uint32_t oi = 0;
      while (go && w.next())
        for (int n = 0; go && n < w.c1 - w.c0; ++n) {
          const int c = w.c0 + n;
          for (int h = 0; h < group; ++h, ++oi) {
            if (!mbar_wait(&bars->out_full, oi & 1) || gave_up()) {
              go = false;
              break;
            }
            if (w.rows(c) == kChunk) {
#pragma unroll
              for (int kb = 0; kb < D / 64; ++kb)
                tma_store_3d(&tm_o, sbase + C::OFF_O + kb * 16384, kb * 64, w.head * group + h, w.start + c * kChunk);
              bulk_commit();
              bulk_wait_read();
            }
            mbar_arrive(&bars->out_free[oi & 1]);
          }
        }
      if (!go) set_abort(&bars->abort, p.c.status);
    }
  } else if (warp < 12) {
    // ---------------------------------------------------------- P and O
    setmaxnreg_dec<C::REG_ROWS>();
    const uint32_t mine = warp < 8 ? 0 : 1;
    const int quad = warp & 3, r = quad * 32 + lane;
    const uint32_t trow = tmem + ((uint32_t)(quad * 32) << 16);
    float* tab = reinterpret_cast<float*>(smem + C::OFF_TAB) + (warp - 4) * 32;
    const uint32_t tab_at = smem_u32(tab);
    bool go = true;
    uint32_t it = 0, ki = 0, oi = 0, fasts = 0;   // oi: outputs
    while (go && w.next()) {
      const bool fast = w.l2 < kSlow;
      __syncwarp();
      tab[lane] = exp2f(w.l2 * (float)(31 - lane));
      __syncwarp();
      const uint64_t slope = f2pack(w.l2, w.l2);
      for (int n = 0; go && n < w.c1 - w.c0; ++n) {
        const int c = w.c0 + n;
        const int rows = w.rows(c);
        const float f_out = fast ? p.scale : p.scale * exp2f(w.l2 * (float)(r + 1 - kMiddle));
        for (int h = 0; h < group; ++h, ++it) {
          if ((it & 1) == mine) {
            const uint32_t tp = trow + C::TM_P + it % C::NP * 128;
            if (!mbar_wait_warp(&bars->s_full[mine], (it >> 1) & 1) || __any_sync(0xffffffffu, gave_up())) {
              go = false;
              break;
            }
            tc_fence_after();
            // Loops over columns are not unrolled: the roles' code together outgrows the instruction cache.  P goes
            // over columns of Q K^T that have been read.
            if (!fast) {
#pragma unroll 1
              for (int g = 0; g < 4; ++g) {
                const int c0 = g * 32;
                uint32_t s[32];
                if (g > quad) {   // nothing seen
#pragma unroll
                  for (int i = 0; i < 16; ++i) s[i] = 0u;
                } else {
                  tmem_ld_32x32b_x32(tp + c0, s);
                  tmem_ld_wait();
                  reg_fence<32>(s);
                  if (g == quad) {
                    // columns of the group that the row takes, a bit each
                    const uint32_t seen = 0xffffffffu >> (31 - lane);
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                      if (!(seen >> i & 1)) s[i] = 0u;
                  }
#pragma unroll
                  for (int i = 0; i < 16; ++i)
                    s[i] = pack_bf16(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1]));
                }
                tmem_st_32x32b_x16(tp + g * 16, *reinterpret_cast<uint32_t(*)[16]>(&s[0]));
              }
            } else {
              // lam^|r - c|: in a group of 32 columns that the diagonal does not cross a power for the row, from the
              // group's near end, times one of 32 for the column, at most 1 both; in the diagonal's, powers of the
              // exact distances, so that a token sees itself with weight 1.
#pragma unroll 1
              for (int g = 0; g < 4; ++g) {
                uint32_t pk[16];
                if (g > quad) {   // nothing seen
#pragma unroll
                  for (int i = 0; i < 16; ++i) pk[i] = 0u;
                } else {
                  uint32_t s[32];
                  tmem_ld_32x32b_x32(tp + g * 32, s);
                  if (g == quad) {
                    const uint32_t seen = 0xffffffffu >> (31 - lane);
                    const float gap = (float)(r - g * 32);
                    const uint64_t at = f2pack(gap, gap);
                    tmem_ld_wait();
                    reg_fence<32>(s);
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                      float e0, e1, x0, x1;
                      f2unpack(fmul2(slope, fadd2(at, f2pack(-2.f * i, -2.f * i - 1.f))), e0, e1);
                      f2unpack(fmul2(f2pack(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1])),
                                     f2pack(ex2(e0), ex2(e1))),
                               x0, x1);
                      pk[i] = pack_bf16(seen >> (2 * i) & 1 ? x0 : 0.f, seen >> (2 * i + 1) & 1 ? x1 : 0.f);
                    }
                  } else {
                    const float rf = ex2(w.l2 * (float)(r - g * 32 - 31));
                    const uint64_t rf2 = f2pack(rf, rf);
                    tmem_ld_wait();
                    reg_fence<32>(s);
#pragma unroll
                    for (int i = 0; i < 16; i += 2) {
                      const uint4 f = ld_shared_v4(tab_at + i * 8);
                      float x0, x1;
                      f2unpack(fmul2(f2pack(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1])),
                                     fmul2(rf2, f2pack(__uint_as_float(f.x), __uint_as_float(f.y)))),
                               x0, x1);
                      pk[i] = pack_bf16(x0, x1);
                      f2unpack(fmul2(f2pack(__uint_as_float(s[2 * i + 2]), __uint_as_float(s[2 * i + 3])),
                                     fmul2(rf2, f2pack(__uint_as_float(f.z), __uint_as_float(f.w)))),
                               x0, x1);
                      pk[i + 1] = pack_bf16(x0, x1);
                    }
                  }
                }
                tmem_st_32x32b_x16(tp + g * 16, pk);
              }
            }
            if (fast) {   // the rows of Q S
              if (!mbar_wait_warp(&bars->a_full[mine], fasts & 1)) {
                go = false;
                break;
              }
              tc_fence_after();
              const float f = exp2f(w.l2 * (float)(r + 1));
              const uint64_t f2 = f2pack(f, f);
              const uint32_t tb = trow + C::TM_B + oi % C::NB * D;
#pragma unroll 1
              for (int g = 0; g < D / 32; ++g) {
                uint32_t s[32];
                tmem_ld_32x32b_x32(tb + g * 32, s);
                tmem_ld_wait();
                reg_fence<32>(s);
#pragma unroll
                for (int i = 0; i < 32; i += 2) {
                  float x0, x1;
                  f2unpack(fmul2(f2pack(__uint_as_float(s[i]), __uint_as_float(s[i + 1])), f2), x0, x1);
                  s[i] = __float_as_uint(x0);
                  s[i + 1] = __float_as_uint(x1);
                }
                tmem_st_32x32b_x32(tb + g * 32, s);
              }
              ++fasts;
            }
            if (fast && h == 0 && rows < kChunk) {  // V's rows of the next segment, which may hold anything
              const uint32_t v = 2 * ki + 1;
              if (!mbar_wait_warp(&bars->t_full[v % C::NT], (v / C::NT) & 1)) {
                go = false;
                break;
              }
              if (r >= rows) zero_row<D>(sbase + C::OFF_T + v % C::NT * C::TILE, r);
              fence_proxy_async_smem();
            }
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars->p_full[mine]);
          }
          if (h == group - 1) ++ki;
          // Through a tile and a bulk copy: rows stored from registers, a line to a lane, kept the load/store unit so
          // busy that every wait of the other warps took a thousand cycles (40/8/128, one long rollout: 1,260 us).
          // They are where a chunk ends inside the tile.
          if ((oi & 1) == mine) {
            if (!mbar_wait_warp(&bars->o_full[mine], (oi >> 1) & 1)) {
              go = false;
              break;
            }
            tc_fence_after();
            const int head = w.head * group + h;
            bf16* row = p.out + ((size_t)(w.start + c * kChunk + r) * ((size_t)p.c.heads * group) + head) * D;
            const uint64_t f2 = f2pack(f_out, f_out);
            const uint32_t tb = trow + C::TM_B + oi % C::NB * D;
            const bool staged = rows == kChunk;
            const uint32_t tile = sbase + C::OFF_O + r * 128;
            // the output before has left the tile (and this one's place in the order of out_full)
            if (oi > 0 && !mbar_wait_warp(&bars->out_free[(oi - 1) & 1], ((oi - 1) >> 1) & 1)) {
              go = false;
              break;
            }
#pragma unroll 1
            for (int g = 0; g < D / 32; ++g) {
              uint32_t b[32];
              tmem_ld_32x32b_x32(tb + g * 32, b);
              tmem_ld_wait();
              reg_fence<32>(b);
              if (g == D / 32 - 1) {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&bars->o_free[mine]);
              }
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                float x0, x1;
                f2unpack(fmul2(f2, f2pack(__uint_as_float(b[2 * i]), __uint_as_float(b[2 * i + 1]))), x0, x1);
                b[i] = pack_bf16(x0, x1);
              }
              if (staged) {
#pragma unroll
                for (int u = 0; u < 4; ++u)
                  st_shared_v4(tile + (g >> 1) * 16384 + ((((g & 1) * 4 + u) ^ (r & 7)) << 4), b[4 * u], b[4 * u + 1],
                               b[4 * u + 2], b[4 * u + 3]);
              } else if (r < rows) {
                st_global_32(row + g * 32, *reinterpret_cast<const uint32_t(*)[8]>(&b[0]), p.wide);
                st_global_32(row + g * 32 + 16, *reinterpret_cast<const uint32_t(*)[8]>(&b[8]), p.wide);
              }
            }
            fence_proxy_async_smem();
            mbar_arrive(&bars->out_full);
          }
          ++oi;
        }
      }
    }
    if (!go) set_abort(&bars->abort, p.c.status);
  } else {
    // ---------------------------------------------------------- state
    setmaxnreg_inc<C::REG_STATE>();
    const int quad = warp & 3, r = quad * 32 + lane;
    const uint32_t trow = tmem + ((uint32_t)(quad * 32) << 16);
    const bool mine = D == 128 || quad < 2;   // a row of the state
    bool go = true;
    uint32_t ki = 0, ch = 0, handed = 0, sums = 0;   // ki: the next pair to weight;  sums: K^T V read
    while (go && w.next()) {
      const int chunks = w.c1 - w.c0;
      float s[D];
      if (mine) {
#pragma unroll
        for (int i = 0; i < D; ++i) s[i] = 0.f;
        auto add = [&](const float* src, float f) {
#pragma unroll
          for (int i = 0; i < D; i += 4) {
            const float4 x = *reinterpret_cast<const float4*>(src + i);
            s[i] = fmaf(f, x.x, s[i]);
            s[i + 1] = fmaf(f, x.y, s[i + 1]);
            s[i + 2] = fmaf(f, x.z, s[i + 2]);
            s[i + 3] = fmaf(f, x.w, s[i + 3]);
            if (i % 32 == 28) asm volatile("" ::: "memory");   // not all loads ahead: the registers are the state's
          }
        };
        const size_t state = ((size_t)w.seg * p.c.heads + w.head) * D * D + (size_t)r * D;
        if (w.c0 > 0) add(p.starts + ((size_t)(blockIdx.x - 1) * D + r) * D, 1.f);
        else if (p.state_in != nullptr) add(p.state_in + state, 1.f);
        if (p.state_out != nullptr && w.c0 > 0 && w.c1 == w.nch) {  // its last piece's own sum is there
          float* dst = p.state_out + state;
          const float f = exp2f(w.l2 * (float)(w.len - w.c0 * kChunk));
#pragma unroll
          for (int i = 0; i < D; i += 4) {
            float4 x = *reinterpret_cast<const float4*>(dst + i);
            x.x = fmaf(f, s[i], x.x);
            x.y = fmaf(f, s[i + 1], x.y);
            x.z = fmaf(f, s[i + 2], x.z);
            x.w = fmaf(f, s[i + 3], x.w);
            *reinterpret_cast<float4*>(dst + i) = x;
            if (i % 32 == 28) asm volatile("" ::: "memory");
          }
        }
      }
      const bool fast = w.l2 < kSlow;
      for (int n = 0; go && n < chunks; ++n, ++ch) {
        const bool weigh = n < chunks - 1;
        // the copy that the chunk's queries read, when the one before has been read
        if (ch > 0 && !mbar_wait_warp(&bars->s_read, (ch - 1) & 1)) {
          go = false;
          break;
        }
        if (mine) {
          const float f = fast ? 1.f : exp2f(w.l2 * (float)kMiddle);
          const uint64_t f2 = f2pack(f, f);
          const uint32_t dst = sbase + C::OFF_S + r * 128;
#pragma unroll
          for (int i = 0; i < D / 8; ++i) {
            uint32_t y[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              float a, b;
              f2unpack(fmul2(f2, f2pack(s[8 * i + 2 * j], s[8 * i + 2 * j + 1])), a, b);
              y[j] = pack_bf16(a, b);
            }
            st_shared_v4(dst + (i >> 3) * (D * 128) + (((i & 7) ^ (r & 7)) << 4), y[0], y[1], y[2], y[3]);
          }
        }
        fence_proxy_async_smem();
        mbar_arrive(&bars->s_ready);
        // the chunk's V weighted, or its K when Q K^T has read it
        const int rows = w.rows(w.c0 + n);
        const uint32_t at = 2 * ki + (fast ? 0 : 1), tile = sbase + C::OFF_T + at % C::NT * C::TILE + r * 128;
        if ((fast && weigh && !mbar_wait_warp(&bars->k_done, handed++ & 1)) ||
            (fast && !weigh ? !mbar_wait_warp(&bars->t_full[(2 * ki + 1) % C::NT], ((2 * ki + 1) / C::NT) & 1)
                            : !mbar_wait_warp(&bars->t_full[at % C::NT], (at / C::NT) & 1)) ||
            __any_sync(0xffffffffu, gave_up())) {
          go = false;
          break;
        }
        if (!fast || weigh) {   // (no state comes behind a piece's last chunk)
          const float wt = exp2f(w.l2 * (float)(fast ? kChunk - 1 - r : kMiddle - 1 - r));
          const uint64_t wt2 = f2pack(wt, wt);
#pragma unroll 1
          for (int kb = 0; kb < D / 32; ++kb) {   // four loads under way
            uint4 x[4];
            const uint32_t row = tile + (kb >> 1) * 16384;
            const int u0 = (kb & 1) * 4 + r;
#pragma unroll
            for (int u = 0; u < 4; ++u) x[u] = ld_shared_v4(row + (((u0 + u) & 7) << 4));
#pragma unroll
            for (int u = 0; u < 4; ++u) {
              const uint32_t in[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
              uint32_t y[4];
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                float a, b;
                f2unpack(fmul2(f2pack(lo_f(in[i]), hi_f(in[i])), wt2), a, b);
                y[i] = r < rows ? pack_bf16(a, b) : 0u;   // rows of the next segment may hold anything
              }
              st_shared_v4(row + (((u0 + u) & 7) << 4), y[0], y[1], y[2], y[3]);
            }
          }
          fence_proxy_async_smem();
        }
        mbar_arrive(&bars->wt_full[ki++ & 3]);
        if (!go || !weigh) continue;
        if (!mbar_wait_warp(&bars->u_full, sums++ & 1)) {
          go = false;
          break;
        }
        tc_fence_after();
        if (mine) {
          const float f = exp2f(w.l2 * (float)kChunk), fu = fast ? 1.f : exp2f(w.l2 * (float)(kChunk - kMiddle));
          const uint64_t f2 = f2pack(f, f), fu2 = f2pack(fu, fu);
#pragma unroll
          for (int g = 0; g < D / 16; ++g) {
            uint32_t u[16];
            tmem_ld_32x32b_x16(trow + C::TM_U + g * 16, u);
            tmem_ld_wait();
            reg_fence<16>(u);
#pragma unroll
            for (int i = 0; i < 16; i += 2)
              f2unpack(ffma2(f2, f2pack(s[g * 16 + i], s[g * 16 + i + 1]),
                             fmul2(fu2, f2pack(__uint_as_float(u[i]), __uint_as_float(u[i + 1])))),
                       s[g * 16 + i], s[g * 16 + i + 1]);
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars->u_free);
      }
    }
    if (!go) set_abort(&bars->abort, p.c.status);
  }
  tc_fence_before();
  __syncthreads();
  if (gave_up()) {
    if (threadIdx.x == 0) {
      finish_loads(bars->q_full, bars->loads[0], C::NQ);
      finish_loads(bars->t_full, bars->loads[1], C::NT);
    }
    if (warp == 1 || warp == 3) finish_mmas(&bars->idle[warp >> 1]);
    __syncthreads();
  }
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

// ------------------------------------------------------------------ gradients of keys and values
struct BackArgs {
  Common c;
  const float* starts;     // the states at the cuts
  int32_t group;
  float scale;
  bool wide;               // dk and dv are 32-byte aligned
  bf16 *dk, *dv;
};

template <int D>
struct Bck {
  static constexpr int TILE = kChunk * D * 2;
  static constexpr int NKV = D == 64 ? 2 : 1;    // tiles of a chunk's K and V
  static constexpr int NQ = D == 64 ? 4 : 2;     // of an item's Q and dO
  // Queries of a step: at D = 128 TMEM has room for two products of 64 queries beside dK, dV and Q^T dO.
  static constexpr int QN = D == 64 ? 128 : 64, NS = kChunk / QN;
  static constexpr int OFF_K = 0, OFF_V = NKV * TILE, OFF_Q = 2 * NKV * TILE, OFF_D = OFF_Q + NQ * TILE;
  static constexpr int OFF_S = OFF_D + NQ * TILE;        // the state, a row a dim of q
  static constexpr int OFF_TAB = OFF_S + D * D * 2;      // 32 powers of the decay for each warp that makes P
  static constexpr int OFF_BAR = OFF_TAB + 8 * 128;
  static constexpr int SMEM = OFF_BAR + 512;
  static constexpr int TM_O = 2 * QN, TM_U = TM_O + 2 * D;   // dV, dK; before them K Q^T, V dO^T
  static constexpr uint32_t IDESC_S = idesc_bf16(128, QN, 0, 0);   // K (K-major) x Q^T (K-major), V x dO^T
  static constexpr uint32_t IDESC_V = idesc_bf16(128, D, 0, 1);    // K (K-major) x S (MN-major), P (TMEM) x dO or Q
  static constexpr uint32_t IDESC_K = idesc_bf16(128, D, 0, 0);    // V (K-major) x S^T (K-major)
  static constexpr uint32_t IDESC_U = idesc_bf16(128, D, 1, 1);    // Q^T (MN-major) x dO (MN-major); see Lin for M
  static constexpr int REG_CTRL = 96, REG_ROWS = 104, REG_STATE = 208;
  static_assert(REG_CTRL + 2 * REG_ROWS + REG_STATE <= 512, "setmaxnreg targets exceed the launch registers");
  static_assert(SMEM <= 232448 && TM_U + D <= 512, "shared memory and TMEM budgets");
};

struct BckBars {
  uint64_t k_full[2][2], k_empty[2][2];   // K and V
  uint64_t q_full[4], q_empty[4];   // an item's Q and dO
  uint64_t wt_full[4];              // and Q is weighted, rows behind the segment's end are cleared in both
  uint64_t k_done, wt2[4];          // of a head that forgets fast: Q has been read as it was loaded; it is weighted
  // Of dV's products and of dK's:
  uint64_t s_full[2], p_full[2];    // of a step: K Q^T, V dO^T, and its P in TMEM
  uint64_t a_full[2];               // the product with the state, for the warps that scale its rows
  uint64_t o_full[2], o_free[2];    // a chunk's sum is complete, and in registers
  uint64_t u_full, u_free;          // the chunk's Q^T dO, and in registers
  uint64_t s_ready, s_read;         // the state that the chunk's keys read is in shared memory, and has been read
  uint64_t idle[3];                 // given up: all MMAs of an issuer are complete
  uint32_t loads[3];                // of Q and dO, of K and of V
  uint32_t tmem_base;
  int32_t abort;
  int32_t steps;           // of dV whose K Q^T is there
};
static_assert(sizeof(BckBars) <= 512, "barrier space");

// dK and dV of a chunk together, from the last chunk to the first: with m = 64 and w_i = lam^(i-m) q_i, weighted in
// place as soon as it is loaded,
//   dv_j = scale lam^(m-j) [ k_j (lam^(n-m) R) + sum_{i >= j} (k_j . w_i) do_i ]
//   dk_j = scale lam^(m-j) [ v_j (lam^(n-m) R)^T + sum_{i >= j} (v_j . do_i) w_i ]
//   R'   = lam^n R + lam^m sum_i w_i do_i^T
// with one load of q and do and one state for both.  (A pass each loads them twice and has six products an item, not
// five: 2,166 us over one rollout of 246,616 tokens at 40 / 8 heads of 128, this 1,472.)  Both factors are at most
// 2^64 (kSlow); for a head that forgets faster both P have the exact powers, the rows of the products with R are
// scaled in TMEM, and Q is weighted when they have read it.
//
// An item is a chunk with one query head; a step an item's QN queries.  Three warps issue MMAs, each its own chain and
// in order: dV's  P dO, K Q^T of the next step;  dK's  P Q, V dO^T of the next step;  the state's  Q^T dO of an item.
// A chunk's products with R come in its second item (of one, the first): R has had an item's time.  One warp for all
// is held up by its waits and commits: 1,940 us of the rollout above.  What bounds it now is the chain of a step, a
// product's P into TMEM and back: 2,400 cycles, of which the MMAs of both chains and the state take 1,536 and memory
// 1,690.  (At D = 64 a second buffer of steps does not shorten it: 2,600 cycles an item of 1,408 with one or two.)
//   warp 0  loads;  warps 1, 3  MMAs of dV and of dK;  warp 2  TMEM, MMAs of the state
//   warps 4-7    P of K Q^T, dV;  warps 8-11  P of V dO^T, dK  (a thread a key)
//   warps 12-15  weighted Q, and the state in registers (a thread a row), its bf16 copy in shared memory
template <int D>
__global__ void __launch_bounds__(kThreads, 1)
    linear_back(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_do,
                const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                const __grid_constant__ BackArgs p) {
  using C = Bck<D>;
  extern __shared__ __align__(1024) uint8_t smem[];
  BckBars* bars = reinterpret_cast<BckBars*>(smem + C::OFF_BAR);
  Walk w(p.c, blockIdx.x);
  if (w.g >= w.hi) return;
  if (__syncthreads_or(threadIdx.x == 0 && *reinterpret_cast<volatile int32_t*>(p.c.status) == VCS_ERR_DEVICE_TIMEOUT))
    return;
  if (smem_u32(smem) & 1023u) {
    if (threadIdx.x == 0) set_status(p.c.status, VCS_ERR_CUDA);
    return;
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, group = p.group;
  const uint32_t sbase = smem_u32(smem);
  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      for (int j = 0; j < 2; ++j) {
        mbar_init(&bars->k_full[i][j], 1);
        mbar_init(&bars->k_empty[i][j], 1);
      }
      mbar_init(&bars->s_full[i], 1);
      mbar_init(&bars->p_full[i], 4);
      mbar_init(&bars->a_full[i], 1);
      mbar_init(&bars->o_full[i], 1);
      mbar_init(&bars->o_free[i], 4);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(&bars->q_full[i], 1);
      mbar_init(&bars->q_empty[i], 3);
      mbar_init(&bars->wt_full[i], 128);
      mbar_init(&bars->wt2[i], 128);
    }
    mbar_init(&bars->k_done, 2);
    mbar_init(&bars->u_full, 1);
    mbar_init(&bars->u_free, 4);
    mbar_init(&bars->s_ready, 128);
    mbar_init(&bars->s_read, 2);
    for (int i = 0; i < 3; ++i) mbar_init(&bars->idle[i], 1);
    bars->abort = 0;
    bars->steps = 0;
    fence_mbar_init();
  }
  if (warp == 2) {
    tmem_alloc(&bars->tmem_base, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = bars->tmem_base;
  auto gave_up = [&] { return *reinterpret_cast<volatile int32_t*>(&bars->abort) != 0; };

  if (warp < 4) {
    setmaxnreg_dec<C::REG_CTRL>();
    if (warp == 0) {
      // -------------------------------------------------------- loads
      bool go = lane == 0;
      uint32_t it = 0, ck = 0, loads[2] = {0, 0};   // of K and of V
      while (go && w.next())
        for (int n = 0; go && n < w.c1 - w.c0; ++n, ++ck) {
          const int tok = w.start + (w.c1 - 1 - n) * kChunk;
          auto load = [&](int off, const CUtensorMap* tm, uint64_t* full, int head) {
#pragma unroll
            for (int kb = 0; kb < D / 64; ++kb) tma_load_3d(smem + off + kb * 16384, tm, full, kb * 64, head, tok);
          };
          for (int h = 0; go && h < group; ++h, ++it) {
            const uint32_t slot = it % C::NQ, kv = ck % C::NKV;
            go = (it < C::NQ || mbar_wait(&bars->q_empty[slot], (it / C::NQ - 1) & 1)) && !gave_up();
            if (!go) break;
            mbar_arrive_expect_tx(&bars->q_full[slot], 2 * C::TILE);
            load(C::OFF_Q + slot * C::TILE, &tm_q, &bars->q_full[slot], w.head * group + h);
            load(C::OFF_D + slot * C::TILE, &tm_do, &bars->q_full[slot], w.head * group + h);
            if (h > 0) continue;
            for (int x = 0; x < 2; ++x) {
              go = go && (ck < C::NKV || mbar_wait(&bars->k_empty[x][kv], (ck / C::NKV - 1) & 1));
              if (!go) break;
              mbar_arrive_expect_tx(&bars->k_full[x][kv], C::TILE);
              load((x ? C::OFF_V : C::OFF_K) + kv * C::TILE, x ? &tm_v : &tm_k, &bars->k_full[x][kv], w.head);
              ++loads[x];
            }
          }
        }
      if (lane == 0) {
        if (!go) set_abort(&bars->abort, p.c.status);
        bars->loads[0] = it;
        bars->loads[1] = loads[0];
        bars->loads[2] = loads[1];
      }
    } else if (warp == 2) {
      // -------------------------------------------------------- MMAs of the state (see linear_out for the issuers' form)
      const uint64_t qt = smem_desc(sbase + C::OFF_Q, 16384, 1024);
      bool ok = true, go = true;
      uint32_t it = 0, us = 0, fasts = 0;
      while (go && w.next()) {
        const bool fast = w.l2 < kSlow;
        const int chunks = w.c1 - w.c0;
        for (int n = 0; go && n < chunks; ++n)
          for (int h = 0; h < group; ++h, ++it) {
            const uint32_t q = it % C::NQ;
            const bool weigh = n < chunks - 1;
            if (weigh && fast) {
              ok = ok && mbar_wait(&bars->wt2[fasts & 3], (fasts >> 2) & 1);
              ++fasts;
            } else {
              ok = ok && mbar_wait(&bars->wt_full[q], (it / C::NQ) & 1);
            }
            if (weigh && h == 0 && us++ > 0) ok = ok && mbar_wait(&bars->u_free, us & 1);
            go = __all_sync(0xffffffffu, ok) && !__any_sync(0xffffffffu, gave_up());
            if (!go) break;
            tc_fence_after();
            if (elect_one()) {
              if (weigh) {
                const uint64_t a = desc_at(qt, q * C::TILE), d = desc_at(a, C::NQ * C::TILE);
#pragma unroll
                for (int kk = 0; kk < 8; ++kk)
                  tc_mma_ss(tmem + C::TM_U, desc_at(a, kk * 2048), desc_at(d, kk * 2048), C::IDESC_U, kk > 0 || h > 0);
                if (h == group - 1) tc_commit(&bars->u_full);
              }
              tc_commit(&bars->q_empty[q]);
            }
            __syncwarp();
          }
      }
      if (!go) set_abort(&bars->abort, p.c.status);
    } else {
      // -------------------------------------------------------- MMAs of dV (x = 0) and of dK (1)
      const int x = warp >> 1;
      const uint32_t ts = tmem + x * C::QN, to = tmem + C::TM_O + x * D;
      uint64_t *k_full = bars->k_full[x], *k_empty = bars->k_empty[x];
      const uint64_t kd = smem_desc(sbase + (x ? C::OFF_V : C::OFF_K), 16, 1024);      // K or V
      const uint64_t qd = smem_desc(sbase + (x ? C::OFF_D : C::OFF_Q), 16, 1024);      // x Q^T or dO^T
      const uint64_t pd = smem_desc(sbase + (x ? C::OFF_Q : C::OFF_D), 16384, 1024);   // P x dO or Q
      const uint64_t rd = x ? smem_desc(sbase + C::OFF_S, 16, 1024) : smem_desc(sbase + C::OFF_S, D * 128, 1024);
      const uint32_t r_step = x ? 32 : 2048, r_block = x ? D * 128 : 4 * 2048, r_idesc = x ? C::IDESC_K : C::IDESC_V;
      bool ok = true, go = true, more = w.next();
      uint32_t t = 0, it = 0, ck = 0;   // steps, items, chunks
      // The step whose product comes next: its item and chunk, and place in them.
      uint32_t nit = 0, nck = 0;
      int ns = 0, nh = 0;
      auto issue_s = [&] {
        if (ns == 0) {
          ok = ok && mbar_wait(&bars->wt_full[nit % C::NQ], (nit / C::NQ) & 1);
          if (w.l2 < kSlow) ok = ok && mbar_wait(&bars->q_full[nit % C::NQ], (nit / C::NQ) & 1);
          if (nh == 0) ok = ok && mbar_wait(&k_full[nck % C::NKV], (nck / C::NKV) & 1);
          // Both chains wait for the same Q and dO.  In step they want the pipe at once and leave it idle at once, so dK's
          // begins an item when dV's first product is there, or 500 cycles after (300 to 800 are as good, 1,500 half as
          // good): 1,570 -> 1,472 us of one rollout at 40 / 8 heads of 128; with the forward 1,256 -> 1,198 us of two of
          // 40,000 tokens at 16 / 16.  At D = 64, where the pipe is no bound, without: with the forward 894 -> 878 us of four
          // of 60,000 tokens at 14 / 2, 510 -> 505 of 64 short ones at 16 / 2, 765 either way at 6 / 6.
          if (D == 128 && x == 1) {
            const long long t0 = clock64();
            while (*reinterpret_cast<volatile int32_t*>(&bars->steps) <= (int)t && clock64() - t0 < 500) {
            }
          }
        }
        tc_fence_after();
        if (elect_one() && ok) {
          const uint64_t a = desc_at(kd, nck % C::NKV * C::TILE);
          const uint64_t d = desc_at(qd, nit % C::NQ * C::TILE + ns * C::QN * 128);
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk) {
            const uint32_t off = (kk >> 2) * 16384 + (kk & 3) * 32;
            tc_mma_ss(ts, desc_at(a, off), desc_at(d, off), C::IDESC_S, kk > 0);
          }
          tc_commit(&bars->s_full[x]);
          if (C::NKV == 1 && ns == C::NS - 1 && nh == group - 1) tc_commit(&k_empty[0]);
        }
        __syncwarp();
      };
      if (more) issue_s();
      while (go && more) {
        const int chunks = w.c1 - w.c0;
        const bool fast = w.l2 < kSlow;
        const int hr = fast || group == 1 ? 0 : 1;   // the item that the product with R comes in
        for (int n = 0; go && n < chunks; ++n) {
          const bool weigh = n < chunks - 1;
          for (int h = 0; go && h < group; ++h)
            for (int s = 0; s < C::NS; ++s) {
              const bool first = h == 0 && s == 0, item = s == C::NS - 1, end = item && h == group - 1;
              const uint32_t q = it % C::NQ, kv = ck % C::NKV;
              if (first && ck > 0) ok = ok && mbar_wait(&bars->o_free[x], (ck - 1) & 1);
              if (h == hr && s == 0) {   // dV += K R, dK += V R^T
                ok = ok && mbar_wait(&bars->s_ready, ck & 1);
                tc_fence_after();
                if (elect_one() && ok) {
                  const uint64_t a = desc_at(kd, kv * C::TILE);
#pragma unroll
                  for (int kk = 0; kk < D / 16; ++kk)
                    tc_mma_ss(to, desc_at(a, (kk >> 2) * 16384 + (kk & 3) * 32),
                              desc_at(rd, (kk >> 2) * r_block + (kk & 3) * r_step), r_idesc, kk > 0 || !first);
                  if (fast) tc_commit(&bars->a_full[x]);
                  tc_commit(&bars->s_read);
                }
                __syncwarp();
              }
              ok = ok && mbar_wait(&bars->p_full[x], t & 1);
              go = __all_sync(0xffffffffu, ok);
              if (!go) break;
              tc_fence_after();
              if (elect_one()) {   // dV += P dO, dK += P Q
                const uint64_t d = desc_at(pd, q * C::TILE + s * C::QN * 128);
#pragma unroll
                for (int kk = 0; kk < C::QN / 16; ++kk)
                  tc_mma_ts(to, ts + kk * 8, desc_at(d, kk * 2048), C::IDESC_V, kk > 0 || !(first && hr > 0));
                if (item) {
                  tc_commit(&bars->q_empty[q]);
                  if (fast && weigh) tc_commit(&bars->k_done);
                }
                if (end) {
                  tc_commit(&bars->o_full[x]);
                  if (C::NKV > 1) tc_commit(&k_empty[kv]);
                }
              }
              __syncwarp();
              bool next = true;
              ns = s + 1;
              ++t;
              if (item) {
                ns = 0;
                ++nit, ++it;
                nh = h + 1;
                if (end) {
                  nh = 0;
                  ++nck, ++ck;
                  if (!weigh) next = more = w.next();
                }
              }
              if (next) issue_s();
            }
        }
      }
      go = __all_sync(0xffffffffu, ok);
      if (!go) set_abort(&bars->abort, p.c.status);
    }
  } else if (warp < 12) {
    // ---------------------------------------------------------- P, dV and dK
    setmaxnreg_dec<C::REG_ROWS>();
    const int x = warp < 8 ? 0 : 1;
    const int quad = warp & 3, r = quad * 32 + lane;
    const uint32_t trow = tmem + ((uint32_t)(quad * 32) << 16), tp = trow + x * C::QN, tb = trow + C::TM_O + x * D;
    bf16* out = x ? p.dk : p.dv;
    float* tab = reinterpret_cast<float*>(smem + C::OFF_TAB) + (warp - 4) * 32;
    const uint32_t tab_at = smem_u32(tab);
    bool go = true;
    uint32_t t = 0, ck = 0, fasts = 0;
    while (go && w.next()) {
      const bool fast = w.l2 < kSlow;
      __syncwarp();
      tab[lane] = exp2f(w.l2 * (float)lane);
      __syncwarp();
      const uint64_t slope = f2pack(-w.l2, -w.l2);
      for (int n = 0; go && n < w.c1 - w.c0; ++n, ++ck) {
        const int c = w.c1 - 1 - n, rows = w.rows(c);
        const float f_out = fast ? p.scale : p.scale * exp2f(w.l2 * (float)(kMiddle - r));
        if (fast) {   // the rows of the product with R
          if (!mbar_wait_warp(&bars->a_full[x], fasts++ & 1)) {
            go = false;
            break;
          }
          tc_fence_after();
          const float f = exp2f(w.l2 * (float)max(rows - r, 0));
          const uint64_t f2 = f2pack(f, f);
#pragma unroll 1
          for (int g = 0; g < D / 32; ++g) {
            uint32_t s[32];
            tmem_ld_32x32b_x32(tb + g * 32, s);
            tmem_ld_wait();
            reg_fence<32>(s);
#pragma unroll
            for (int i = 0; i < 32; i += 2) {
              float x0, x1;
              f2unpack(fmul2(f2pack(__uint_as_float(s[i]), __uint_as_float(s[i + 1])), f2), x0, x1);
              s[i] = __float_as_uint(x0);
              s[i + 1] = __float_as_uint(x1);
            }
            tmem_st_32x32b_x32(tb + g * 32, s);
          }
        }
        for (int st = 0; go && st < group * C::NS; ++st, ++t) {
          if (!mbar_wait_warp(&bars->s_full[x], t & 1) || __any_sync(0xffffffffu, gave_up())) {
            go = false;
            break;
          }
          if (D == 128 && threadIdx.x == 128) *reinterpret_cast<volatile int32_t*>(&bars->steps) = (int)t + 1;
          tc_fence_after();
          // P goes over columns that have been read.  Loops are not unrolled: see linear_out.
#pragma unroll 1
          for (int g = 0; g < C::QN / 32; ++g) {
            const int q0 = (st % C::NS) * C::QN + g * 32;   // the group's first query
            uint32_t s[32];
            if (q0 + 31 < quad * 32 || q0 >= rows) {   // nothing seen
#pragma unroll
              for (int i = 0; i < 16; ++i) s[i] = 0u;
            } else {
              tmem_ld_32x32b_x32(tp + g * 32, s);
              uint32_t seen = 0xffffffffu;   // queries of the group that the key is seen by, a bit each
              if (q0 == quad * 32) seen = 0xffffffffu << lane;
              if (rows - q0 < 32) seen &= (1u << (rows - q0)) - 1u;
              const bool all = q0 > quad * 32 && rows - q0 >= 32;
              tmem_ld_wait();
              reg_fence<32>(s);
              if (!fast) {
                if (!all) {
#pragma unroll
                  for (int i = 0; i < 32; ++i)
                    if (!(seen >> i & 1)) s[i] = 0u;
                }
#pragma unroll
                for (int i = 0; i < 16; ++i)
                  s[i] = pack_bf16(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1]));
              } else if (!all) {   // lam^(query - key): powers of the exact distances (see linear_out)
                const float gap = (float)(r - q0);
                const uint64_t at = f2pack(gap, gap);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                  float e0, e1, x0, x1;
                  f2unpack(fmul2(slope, fadd2(at, f2pack(-2.f * i, -2.f * i - 1.f))), e0, e1);
                  f2unpack(fmul2(f2pack(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1])),
                                 f2pack(ex2(e0), ex2(e1))),
                           x0, x1);
                  s[i] = pack_bf16(seen >> (2 * i) & 1 ? x0 : 0.f, seen >> (2 * i + 1) & 1 ? x1 : 0.f);
                }
              } else {
                const float rf = ex2(w.l2 * (float)(q0 - r));
                const uint64_t rf2 = f2pack(rf, rf);
#pragma unroll
                for (int i = 0; i < 16; i += 2) {
                  const uint4 f = ld_shared_v4(tab_at + i * 8);
                  float x0, x1;
                  f2unpack(fmul2(f2pack(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1])),
                                 fmul2(rf2, f2pack(__uint_as_float(f.x), __uint_as_float(f.y)))),
                           x0, x1);
                  s[i] = pack_bf16(x0, x1);
                  f2unpack(fmul2(f2pack(__uint_as_float(s[2 * i + 2]), __uint_as_float(s[2 * i + 3])),
                                 fmul2(rf2, f2pack(__uint_as_float(f.z), __uint_as_float(f.w)))),
                           x0, x1);
                  s[i + 1] = pack_bf16(x0, x1);
                }
              }
            }
            tmem_st_32x32b_x16(tp + g * 16, *reinterpret_cast<uint32_t(*)[16]>(&s[0]));
          }
          tmem_st_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&bars->p_full[x]);
        }
        if (!go || !mbar_wait_warp(&bars->o_full[x], ck & 1)) {
          go = false;
          break;
        }
        tc_fence_after();
        bf16* row = out + ((size_t)(w.start + c * kChunk + r) * p.c.heads + w.head) * D;
        const uint64_t f2 = f2pack(f_out, f_out);
#pragma unroll 1
        for (int g = 0; g < D / 32; ++g) {
          uint32_t b[32];
          tmem_ld_32x32b_x32(tb + g * 32, b);
          tmem_ld_wait();
          reg_fence<32>(b);
          if (g == D / 32 - 1) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars->o_free[x]);
          }
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            float x0, x1;
            f2unpack(fmul2(f2, f2pack(__uint_as_float(b[2 * i]), __uint_as_float(b[2 * i + 1]))), x0, x1);
            b[i] = pack_bf16(x0, x1);
          }
          if (r < rows) {
            st_global_32(row + g * 32, *reinterpret_cast<const uint32_t(*)[8]>(&b[0]), p.wide);
            st_global_32(row + g * 32 + 16, *reinterpret_cast<const uint32_t(*)[8]>(&b[8]), p.wide);
          }
        }
      }
    }
    if (!go) set_abort(&bars->abort, p.c.status);
  } else {
    // ---------------------------------------------------------- weighted Q, state
    setmaxnreg_inc<C::REG_STATE>();
    const int quad = warp & 3, r = quad * 32 + lane;
    const uint32_t trow = tmem + ((uint32_t)(quad * 32) << 16);
    const bool mine = D == 128 || quad < 2;   // a row of the state
    bool go = true;
    uint32_t it = 0, ck = 0, fasts = 0, sums = 0;
    while (go && w.next()) {
      const int chunks = w.c1 - w.c0;
      const bool fast = w.l2 < kSlow;
      float s[D];
      if (mine) {
        const float* src = p.starts + ((size_t)blockIdx.x * D + r) * D;
#pragma unroll
        for (int i = 0; i < D; i += 4) {
          float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
          if (w.c1 < w.nch) x = *reinterpret_cast<const float4*>(src + i);
          s[i] = x.x;
          s[i + 1] = x.y;
          s[i + 2] = x.z;
          s[i + 3] = x.w;
          if (i % 32 == 28) asm volatile("" ::: "memory");   // not all loads ahead: the registers are the state's
        }
      }
      const int64_t items = (int64_t)chunks * group;
      int64_t done = 0;
      for (int n = 0; go && n < chunks; ++n, ++ck) {
        if (ck > 0 && !mbar_wait_warp(&bars->s_read, (ck - 1) & 1)) {
          go = false;
          break;
        }
        if (mine) {
          const float f = fast ? 1.f : exp2f(w.l2 * (float)(w.rows(w.c1 - 1 - n) - kMiddle));
          const uint64_t f2 = f2pack(f, f);
          const uint32_t dst = sbase + C::OFF_S + r * 128;
#pragma unroll
          for (int i = 0; i < D / 8; ++i) {
            uint32_t y[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              float a, b;
              f2unpack(fmul2(f2, f2pack(s[8 * i + 2 * j], s[8 * i + 2 * j + 1])), a, b);
              y[j] = pack_bf16(a, b);
            }
            st_shared_v4(dst + (i >> 3) * (D * 128) + (((i & 7) ^ (r & 7)) << 4), y[0], y[1], y[2], y[3]);
          }
        }
        fence_proxy_async_smem();
        mbar_arrive(&bars->s_ready);
        // Items up to this chunk's and, as K Q^T runs a step ahead, the next one's first (which for a fast head waits).
        int64_t target = (int64_t)(n + 1) * group + (fast ? 0 : 1);
        if (target > items) target = items;
        for (; done < target; ++done, ++it) {
          const int m = (int)(done / group), rows = w.rows(w.c1 - 1 - m);
          const uint32_t slot = it % C::NQ, tile = sbase + C::OFF_Q + slot * C::TILE;
          if (!mbar_wait_warp(&bars->q_full[slot], (it / C::NQ) & 1) || __any_sync(0xffffffffu, gave_up())) {
            go = false;
            break;
          }
          if (r >= rows) {   // rows of the next segment, which may hold anything
            zero_row<D>(tile, r);
            zero_row<D>(tile + C::NQ * C::TILE, r);
          }
          if (fast) {
            fence_proxy_async_smem();
            mbar_arrive(&bars->wt_full[slot]);
            if (m == chunks - 1) continue;   // no state comes behind the last chunk
            if (!mbar_wait_warp(&bars->k_done, fasts & 1)) {
              go = false;
              break;
            }
          }
          const float wt = exp2f(w.l2 * (float)(fast ? r : r - kMiddle));
          const uint64_t wt2 = f2pack(wt, wt);
          if (r < rows) {
#pragma unroll 1
            for (int kb = 0; kb < D / 32; ++kb) {   // four loads under way
              uint4 x[4];
              const uint32_t row = tile + (kb >> 1) * 16384 + r * 128;
              const int u0 = (kb & 1) * 4 + r;
#pragma unroll
              for (int u = 0; u < 4; ++u) x[u] = ld_shared_v4(row + (((u0 + u) & 7) << 4));
#pragma unroll
              for (int u = 0; u < 4; ++u) {
                const uint32_t in[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
                uint32_t y[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  float a, b;
                  f2unpack(fmul2(f2pack(lo_f(in[i]), hi_f(in[i])), wt2), a, b);
                  y[i] = pack_bf16(a, b);
                }
                st_shared_v4(row + (((u0 + u) & 7) << 4), y[0], y[1], y[2], y[3]);
              }
            }
          }
          fence_proxy_async_smem();
          mbar_arrive(fast ? &bars->wt2[fasts++ & 3] : &bars->wt_full[slot]);
        }
        if (!go || n == chunks - 1) continue;
        if (!mbar_wait_warp(&bars->u_full, sums++ & 1)) {
          go = false;
          break;
        }
        tc_fence_after();
        if (mine) {
          const float f = exp2f(w.l2 * (float)w.rows(w.c1 - 1 - n));
          const float fu = fast ? 1.f : exp2f(w.l2 * (float)kMiddle);
          const uint64_t f2 = f2pack(f, f), fu2 = f2pack(fu, fu);
#pragma unroll
          for (int g = 0; g < D / 16; ++g) {
            uint32_t u[16];
            tmem_ld_32x32b_x16(trow + C::TM_U + g * 16, u);
            tmem_ld_wait();
            reg_fence<16>(u);
#pragma unroll
            for (int i = 0; i < 16; i += 2)
              f2unpack(ffma2(f2, f2pack(s[g * 16 + i], s[g * 16 + i + 1]),
                             fmul2(fu2, f2pack(__uint_as_float(u[i]), __uint_as_float(u[i + 1])))),
                       s[g * 16 + i], s[g * 16 + i + 1]);
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars->u_free);
      }
    }
    if (!go) set_abort(&bars->abort, p.c.status);
  }
  tc_fence_before();
  __syncthreads();
  if (gave_up()) {
    if (threadIdx.x == 0) {
      finish_loads(bars->q_full, bars->loads[0], C::NQ);
      for (int x = 0; x < 2; ++x) finish_loads(bars->k_full[x], bars->loads[1 + x], C::NKV);
    }
    if (warp > 0 && warp < 4) finish_mmas(&bars->idle[warp - 1]);
    __syncthreads();
  }
  if (warp == 2) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

// ------------------------------------------------------------------ single tokens
// A block takes COLS columns of one head's state: a row's lanes hold four columns each, and a thread R rows, all
// loaded before the first is used.  The state is read and written once: what bounds it is memory (512 sequences at 40
// / 8 heads of 128, 537 MB: 84 us, 6.4 TB/s).
struct StepArgs {
  const bf16 *q, *k, *v;
  const float* log_decay;
  int32_t hkv, group;
  float scale;
  float* states;
  bf16* o;
  int32_t* status;
};

constexpr int kStepThreads = 256;
constexpr int kStepHeads = 8;   // query heads at a time
constexpr int kStepCols = 64;

template <int D, int COLS>
__global__ void __launch_bounds__(kStepThreads) linear_step(const __grid_constant__ StepArgs a) {
  constexpr int LANES = COLS / 4, RG = kStepThreads / LANES, R = D / RG, W = kStepThreads / 32;
  static_assert(LANES <= 32 && R >= 1, "a warp holds whole rows");
  __shared__ float sk[D], sq[kStepHeads * D], red[kStepHeads][W][COLS];
  const int slices = D / COLS;
  const int64_t unit = blockIdx.x / slices;
  const int col0 = blockIdx.x % slices * COLS;
  const float ld = a.log_decay[unit % a.hkv];
  if (!decay_ok(ld)) {
    if (threadIdx.x == 0) set_status(a.status, VCS_ERR_DEVICE_CHECK);
    return;
  }
  const int lane = threadIdx.x % LANES, rg = threadIdx.x / LANES, wid = threadIdx.x >> 5;
  float4* p = reinterpret_cast<float4*>(a.states + ((size_t)unit * D + rg) * D + col0) + lane;
  float4 s[R];
#pragma unroll
  for (int i = 0; i < R; ++i) s[i] = __ldcs(p + (size_t)i * RG * (D / 4));
  const uint2 v = *reinterpret_cast<const uint2*>(a.v + (size_t)unit * D + col0 + lane * 4);
  if (threadIdx.x < D) sk[threadIdx.x] = __bfloat162float(a.k[(size_t)unit * D + threadIdx.x]);
  const bf16* q = a.q + (size_t)unit * a.group * D;
  auto stage = [&](int h0) {
    const int n = min(kStepHeads, a.group - h0) * D;
    for (int i = threadIdx.x; i < n; i += kStepThreads) sq[i] = __bfloat162float(q[(size_t)h0 * D + i]);
  };
  stage(0);
  const float lam = expf(ld), v0 = lo_f(v.x), v1 = hi_f(v.x), v2 = lo_f(v.y), v3 = hi_f(v.y);
  __syncthreads();
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const float k = sk[rg + i * RG];
    s[i].x = lam * s[i].x + k * v0;
    s[i].y = lam * s[i].y + k * v1;
    s[i].z = lam * s[i].z + k * v2;
    s[i].w = lam * s[i].w + k * v3;
    __stcs(p + (size_t)i * RG * (D / 4), s[i]);
  }
  for (int h0 = 0; h0 < a.group; h0 += kStepHeads) {
    const int heads = min(kStepHeads, a.group - h0);
    if (h0 > 0) {
      __syncthreads();   // the sums and the queries before have been read
      stage(h0);
      __syncthreads();
    }
    for (int h = 0; h < heads; ++h) {
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const float y = sq[h * D + rg + i * RG];
        x.x += y * s[i].x;
        x.y += y * s[i].y;
        x.z += y * s[i].z;
        x.w += y * s[i].w;
      }
#pragma unroll
      for (int o = LANES; o < 32; o <<= 1) {   // the warp's rows
        x.x += __shfl_xor_sync(0xffffffffu, x.x, o);
        x.y += __shfl_xor_sync(0xffffffffu, x.y, o);
        x.z += __shfl_xor_sync(0xffffffffu, x.z, o);
        x.w += __shfl_xor_sync(0xffffffffu, x.w, o);
      }
      if ((threadIdx.x & 31) < LANES) *reinterpret_cast<float4*>(&red[h][wid][lane * 4]) = x;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < heads * COLS; i += kStepThreads) {
      const int h = i / COLS, c = i % COLS;
      float y = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) y += red[h][w][c];
      a.o[((size_t)unit * a.group + h0 + h) * D + col0 + c] = __float2bfloat16(a.scale * y);
    }
  }
}

}  // namespace

namespace {

inline size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

// Workspace: header (status word), the plan, the segments' chunk offsets, and, where a sequence may be cut, the parts'
// sums (three to a CTA at most) and the states at the cuts.
int32_t grid_of(int32_t num_segments, int64_t num_tokens, int32_t hkv) {
  const int64_t chunks = hkv * (num_tokens / kChunk + (int64_t)num_segments);   // no fewer than the sequences'
  return (int32_t)(chunks < kGrid ? chunks : kGrid);
}
bool may_cut(int64_t num_tokens) { return num_tokens > kWhole * kChunk; }
size_t ws_plan() { return align256(sizeof(Plan)); }
size_t ws_off(int32_t num_segments) { return align256(((size_t)num_segments + 1) * 4); }
size_t ws_bytes(int32_t num_segments, int64_t num_tokens, int32_t hkv, int32_t d) {
  const size_t states = may_cut(num_tokens) ? 4 * (size_t)grid_of(num_segments, num_tokens, hkv) : 0;
  return kWsHeader + ws_plan() + ws_off(num_segments) + states * d * d * 4;
}

struct Work {
  Common c;
  float *slots, *starts;
  int32_t grid;
  bool cut;
};

Work make_work(const LinearArgs& a, void* ws) {
  Work w;
  char* p = static_cast<char*>(ws);
  w.grid = grid_of(a.num_segments, a.num_tokens, a.hkv);
  w.cut = may_cut(a.num_tokens);
  w.c.log_decay = a.log_decay;
  w.c.cu = a.cu_seqlens;
  w.c.plan = reinterpret_cast<Plan*>(p + kWsHeader);
  w.c.off = reinterpret_cast<int32_t*>(p + kWsHeader + ws_plan());
  w.c.num_segments = a.num_segments;
  w.c.num_tokens = (int32_t)a.num_tokens;
  w.c.heads = a.hkv;
  w.c.status = static_cast<int32_t*>(ws);
  w.slots = reinterpret_cast<float*>(p + kWsHeader + ws_plan() + ws_off(a.num_segments));
  w.starts = w.slots + 3 * (size_t)w.grid * a.d * a.d;
  return w;
}

// A tensor map of [tokens, heads, D].  Without tokens nothing is read and the pointer may be null: any address that is
// aligned as a map's has to be serves, such as the workspace's.
bool encode(CUtensorMap* map, const void* base, int d, int64_t heads, const LinearArgs& a, const Work& w) {
  return encode_tma_3d_bf16(map, a.num_tokens > 0 ? base : w.c.status, d, heads, a.num_tokens, 64, 128);
}

cudaError_t launch_plan(const Work& w, cudaStream_t st) {
  linear_plan<<<1, 1024, 0, st>>>(w.c.cu, w.c.num_segments, w.c.num_tokens, w.c.heads, w.grid, w.c.log_decay,
                                  const_cast<int32_t*>(w.c.off), const_cast<Plan*>(w.c.plan), w.c.status);
  return cudaGetLastError();
}

// The states at the cuts (and, with state_out, behind the segments, but for what pieces before the last add to them).
template <int D, int TERMS>
cudaError_t launch_states(const Work& w, const LinearArgs& a, const void* k, const void* v, int group, bool back,
                          const float* state_in, float* state_out, cudaStream_t st) {
  using C = Sta<D, TERMS>;
  if (!w.cut && state_out == nullptr) return cudaSuccess;
  alignas(64) CUtensorMap tk, tv;
  const int64_t heads = (int64_t)a.hkv * group;
  if (!encode(&tk, k, D, heads, a, w) || !encode(&tv, v, D, heads, a, w)) return cudaErrorInvalidValue;
  static std::atomic<int> regs_cache{-1};
  bool regs_ok = false;
  cudaError_t e = launch_regs_match(reinterpret_cast<const void*>(linear_states<D, TERMS>), kRegLaunch, &regs_cache, &regs_ok);
  if (e != cudaSuccess) return e;
  if (!regs_ok) return cudaErrorInvalidConfiguration;
  e = cudaFuncSetAttribute(linear_states<D, TERMS>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
  if (e != cudaSuccess) return e;
  StateArgs p;
  p.c = w.c;
  p.slots = w.slots;
  p.state_in = state_in;
  p.state_out = state_out;
  p.group = group;
  p.back = back;
  linear_states<D, TERMS><<<w.grid, kStaThreads, C::SMEM, st>>>(tk, tv, p);
  if (e = cudaGetLastError(); e != cudaSuccess || !w.cut) return e;
  JoinArgs j;
  j.c = w.c;
  j.slots = w.slots;
  j.state_in = state_in;
  j.starts = w.starts;
  j.back = back;
  j.all = state_out != nullptr;
  linear_join<D><<<dim3(w.grid, D * D / 1024), 256, 0, st>>>(j);
  return cudaGetLastError();
}

template <int D, bool ONE>
cudaError_t launch_out(const Work& w, const LinearArgs& a, const void* q, const void* k, const void* v, int group,
                       const float* state_in, float* state_out, void* out, cudaStream_t st) {
  using C = Lin<D, ONE>;
  alignas(64) CUtensorMap tq, tk, tv, to;
  if (!encode(&tq, q, D, a.hq, a, w) || !encode(&tk, k, D, a.hkv, a, w) || !encode(&tv, v, D, a.hkv, a, w) ||
      !encode(&to, out, D, a.hq, a, w))
    return cudaErrorInvalidValue;
  const void* fn = reinterpret_cast<const void*>(linear_out<D, ONE>);
  static std::atomic<int> regs_cache{-1};
  bool regs_ok = false;
  if (cudaError_t e = launch_regs_match(fn, kRegLaunch, &regs_cache, &regs_ok); e != cudaSuccess) return e;
  if (!regs_ok) return cudaErrorInvalidConfiguration;
  cudaError_t e = cudaFuncSetAttribute(linear_out<D, ONE>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
  if (e != cudaSuccess) return e;
  OutArgs p;
  p.c = w.c;
  p.starts = w.starts;
  p.state_in = state_in;
  p.state_out = state_out;
  p.group = group;
  p.scale = a.scale;
  p.out = static_cast<bf16*>(out);
  p.wide = (reinterpret_cast<uintptr_t>(out) & 31u) == 0;
  linear_out<D, ONE><<<w.grid, kThreads, C::SMEM, st>>>(tq, tk, tv, to, p);
  return cudaGetLastError();
}

template <int D>
cudaError_t launch_forth(const Work& w, const LinearArgs& a, const void* q, const void* k, const void* v, int group,
                         const float* state_in, float* state_out, void* out, cudaStream_t st) {
  return group == 1 ? launch_out<D, true>(w, a, q, k, v, 1, state_in, state_out, out, st)
                    : launch_out<D, false>(w, a, q, k, v, group, state_in, state_out, out, st);
}

template <int D>
cudaError_t launch_back(const Work& w, const LinearArgs& a, const void* dout, void* dk, void* dv, int group,
                        cudaStream_t st) {
  using C = Bck<D>;
  alignas(64) CUtensorMap tq, td, tk, tv;
  if (!encode(&tq, a.q, D, a.hq, a, w) || !encode(&td, dout, D, a.hq, a, w) || !encode(&tk, a.k, D, a.hkv, a, w) ||
      !encode(&tv, a.v, D, a.hkv, a, w))
    return cudaErrorInvalidValue;
  const void* fn = reinterpret_cast<const void*>(linear_back<D>);
  static std::atomic<int> regs_cache{-1};
  bool regs_ok = false;
  if (cudaError_t e = launch_regs_match(fn, kRegLaunch, &regs_cache, &regs_ok); e != cudaSuccess) return e;
  if (!regs_ok) return cudaErrorInvalidConfiguration;
  cudaError_t e = cudaFuncSetAttribute(linear_back<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
  if (e != cudaSuccess) return e;
  BackArgs p;
  p.c = w.c;
  p.starts = w.starts;
  p.group = group;
  p.scale = a.scale;
  p.wide = ((reinterpret_cast<uintptr_t>(dk) | reinterpret_cast<uintptr_t>(dv)) & 31u) == 0;
  p.dk = static_cast<bf16*>(dk);
  p.dv = static_cast<bf16*>(dv);
  linear_back<D><<<w.grid, kThreads, C::SMEM, st>>>(tq, td, tk, tv, p);
  return cudaGetLastError();
}

template <int D>
cudaError_t launch_fwd(const LinearArgs& a, const float* state_in, float* state_out, void* o, void* ws,
                       cudaStream_t st) {
  const Work w = make_work(a, ws);
  cudaError_t e = launch_plan(w, st);
  if (e != cudaSuccess) return e;
  e = state_out != nullptr ? launch_states<D, 3>(w, a, a.k, a.v, 1, false, state_in, state_out, st)
                           : launch_states<D, 1>(w, a, a.k, a.v, 1, false, state_in, nullptr, st);
  if (e != cudaSuccess) return e;
  return launch_forth<D>(w, a, a.q, a.k, a.v, a.hq / a.hkv, state_in, state_out, o, st);
}

template <int D>
cudaError_t launch_bwd(const LinearArgs& a, const void* dout, void* dq, void* dk, void* dv, void* ws,
                       cudaStream_t st) {
  const Work w = make_work(a, ws);
  const int group = a.hq / a.hkv;
  cudaError_t e = launch_plan(w, st);
  if (e == cudaSuccess) e = launch_states<D, 1>(w, a, a.v, a.k, 1, false, nullptr, nullptr, st);
  if (e == cudaSuccess) e = launch_forth<D>(w, a, dout, a.v, a.k, group, nullptr, nullptr, dq, st);
  if (e == cudaSuccess) e = launch_states<D, 1>(w, a, a.q, dout, group, true, nullptr, nullptr, st);
  if (e == cudaSuccess) e = launch_back<D>(w, a, dout, dk, dv, group, st);
  return e;
}

}  // namespace

size_t linear_fwd_ws_bytes(int32_t num_segments, int64_t num_tokens, int32_t, int32_t hkv, int32_t d) {
  return ws_bytes(num_segments, num_tokens, hkv, d);
}
size_t linear_bwd_ws_bytes(int32_t num_segments, int64_t num_tokens, int32_t, int32_t hkv, int32_t d) {
  return ws_bytes(num_segments, num_tokens, hkv, d);
}

cudaError_t launch_linear_fwd(const LinearArgs& a, const float* state_in, float* state_out, void* o, void* ws,
                              cudaStream_t st) {
  return a.d == 64 ? launch_fwd<64>(a, state_in, state_out, o, ws, st) : launch_fwd<128>(a, state_in, state_out, o, ws, st);
}

cudaError_t launch_linear_bwd(const LinearArgs& a, const void* dout, void* dq, void* dk, void* dv, void* ws,
                              cudaStream_t st) {
  return a.d == 64 ? launch_bwd<64>(a, dout, dq, dk, dv, ws, st) : launch_bwd<128>(a, dout, dq, dk, dv, ws, st);
}

template <int D>
static cudaError_t launch_step(const StepArgs& s, int64_t num_seqs, cudaStream_t st) {
  const int64_t blocks = num_seqs * s.hkv * (D / kStepCols);
  if (blocks > INT32_MAX) return cudaErrorInvalidConfiguration;
  linear_step<D, kStepCols><<<(unsigned)blocks, kStepThreads, 0, st>>>(s);
  return cudaGetLastError();
}

cudaError_t launch_linear_step(const LinearArgs& a, float* states, void* o, int32_t* status, cudaStream_t st) {
  StepArgs s;
  s.q = static_cast<const bf16*>(a.q);
  s.k = static_cast<const bf16*>(a.k);
  s.v = static_cast<const bf16*>(a.v);
  s.log_decay = a.log_decay;
  s.hkv = a.hkv;
  s.group = a.hq / a.hkv;
  s.scale = a.scale;
  s.states = states;
  s.o = static_cast<bf16*>(o);
  s.status = status;
  return a.d == 64 ? launch_step<64>(s, a.num_tokens, st) : launch_step<128>(s, a.num_tokens, st);
}

}  // namespace vcs
