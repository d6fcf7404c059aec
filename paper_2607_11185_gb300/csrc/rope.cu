// rope.cu - rotary positions with several axes over training segments, sm_103a.
//
// A fresh stream (App. C.1) starts its positions over, so a trajectory token stands at other
// positions in every segment that copies it, and the rotation belongs on the way from the trajectory
// rows to the segment rows:
//   stream_positions   pos[a][n], a = time, height, width, of every segment token
//   gather_rope        q[n] = R(pos[., n]) q_traj[tok_gather[n]], k alike, v copied
//   gather_rope_bwd    dq_traj[t] = sum over the copies n of t of R(-pos[., n]) dq[n], dk alike, dv summed
// R turns pair i, dims (a, b), by the angle x = inv_freq[i] * pos[axis[i]]:
//   (a, b) -> (a cos x - b sin x, b cos x + a sin x).
//
// The angle is reduced in integers: inv_freq / 2 pi is a 64-bit fraction of a turn, its product with the
// position modulo 2^64 is the fraction of a turn the angle ends at, and the upper 32 bits of that go to
// sincospi as a float, off by up to 2^-26 of a turn.  What grows with the position is the rounding of
// inv_freq / 2 pi, a double: up to 2^-52 of the turns passed, 8e-8 of a turn at a position of 2^31 and a radian a
// position (a product in fp32 would be off by 4e-3 radians at 67,000).
//
// All three are bound by HBM.  The rotation reads and writes each row once; a pass of its own over
// the gathered rows would double that.
#include <cmath>
#include <cstdint>

#include "internal.h"
#include "rope_table.h"
#include "sm100.cuh"

namespace vcs {
namespace {

using dev::set_status;

// i / c by the magic 2^32 / c + 1, exactly for i < 2^32 / c; c = 1 has none
__device__ __forceinline__ int div_by(int i, int c, uint32_t magic) {
  return c == 1 ? i : (int)__umulhi((uint32_t)i, magic);
}

// ------------------------------------------------------------------ positions
constexpr int kPosThreads = 256;
constexpr int kPosChunk = 8192;  // tokens of a segment a block writes

// One block: tokens [chunk * kPosChunk, + kPosChunk) of segment blockIdx.x.  The segment's steps in
// tiles of a step a thread: a step's run of tokens starts at the lower bound of its index in
// tok_src_step (non-decreasing within a segment), how far it moves the position follows from the run's
// length (text only, or screenshot and text), and a block scan gives each run's first position.  Every
// chunk of a segment repeats the scan of the steps before it: the searches' latency against a launch and a
// workspace.  That suits segments of one or a few tiles of steps: steps of 15 tokens on average, 299,355 and
// 11,996,577 tokens of them, take 0.03 and 0.16 ms in segments of 50 steps and 0.7 and 67 ms in a single one.  A search
// is one of 256 samples of the segment in shared memory, then four lanes' probes at a time: 5 loads that wait on one
// another for a segment of 46,176 tokens, where halving takes 16.  15.8 M tokens: 54 us, 71 with searches by halving
// and without the loads ahead.
__global__ void __launch_bounds__(kPosThreads, 6)
    stream_positions_kernel(const int32_t* __restrict__ cu_seqlens, int32_t num_segments, int32_t num_tokens,
                            const int32_t* __restrict__ src_step, const int32_t* __restrict__ step_img,
                            const int32_t* __restrict__ step_txt, const int32_t* __restrict__ step_grid,
                            int32_t num_steps, int32_t* __restrict__ pos, int32_t* status) {
  __shared__ int32_t run_at[kPosThreads + 1];   // first token of the step's run
  __shared__ int32_t run_pos[kPosThreads];      // its first position
  __shared__ int32_t run_img[kPosThreads];      // screenshot tokens of the run, 0 if it is text only
  __shared__ int32_t run_skip[kPosThreads];     // positions the screenshot takes
  __shared__ int32_t run_h[kPosThreads], run_w[kPosThreads];
  __shared__ uint32_t run_hm[kPosThreads], run_wm[kPosThreads];  // magics of div_by; 0: divide
  __shared__ int32_t wsum[kPosThreads / 32];
  __shared__ int32_t carry_s;
  __shared__ int32_t sample[kPosThreads];
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  const size_t N = (size_t)num_tokens;
  const bool vec =
      num_tokens % 4 == 0 && ((reinterpret_cast<uintptr_t>(src_step) | reinterpret_cast<uintptr_t>(pos)) & 15u) == 0;
  for (int seg = blockIdx.x; seg < num_segments; seg += gridDim.x) {
    const int start = cu_seqlens[seg], end = cu_seqlens[seg + 1];
    if (start < 0 || end < start || end > num_tokens || (seg == 0 && start != 0) ||
        (seg == num_segments - 1 && end != num_tokens)) {
      if (tid == 0 && blockIdx.y == 0) set_status(status, VCS_ERR_DEVICE_CHECK);
      continue;
    }
    if (start + (int64_t)blockIdx.y * kPosChunk >= end) continue;
    const int first = src_step[start], last = src_step[end - 1];
    const int apart = (end - start - 1) / kPosThreads + 1;  // tokens between samples
    __syncthreads();  // the last segment's searches
    sample[tid] = start + (int64_t)tid * apart < end ? src_step[start + tid * apart] : INT32_MAX;
    __syncthreads();
    if (first < 0 || last < first || last >= num_steps) {
      if (tid == 0) set_status(status, VCS_ERR_DEVICE_CHECK);
      continue;
    }
    for (int64_t c0 = start + (int64_t)blockIdx.y * kPosChunk; c0 < end; c0 += (int64_t)gridDim.y * kPosChunk) {
      const int lo_tok = (int)c0, hi_tok = (int)(c0 + kPosChunk < end ? c0 + kPosChunk : end);
      int carry = 0;  // position at the tile's first run
      for (int64_t s0 = first; s0 <= last; s0 += kPosThreads) {
        const int64_t s = s0 + tid;
        // lower bounds of s0, ... in src_step[start, end), that of s0 + kPosThreads too; end behind the last step
        for (int i0 = 0; i0 <= kPosThreads; i0 += kPosThreads / 4) {
          const int i = i0 + tid / 4;
          const int64_t want = s0 + i;
          int a = end, b = end;
          if (i <= kPosThreads && want <= last) {
            int x = 0;  // samples below it
#pragma unroll
            for (int o = kPosThreads / 2; o > 0; o >>= 1)
              if (sample[x + o - 1] < want) x += o;
            x += x < kPosThreads && sample[x] < want;
            a = x == 0 ? start : start + (x - 1) * apart + 1;
            b = x == kPosThreads || end - start <= (int64_t)x * apart ? end : start + x * apart;
          }
          while (__any_sync(0xffffffffu, a < b)) {
            const int d = b - a, q = lane & 3, step = d / 5, rest = d - 5 * step;
            auto probe = [&](int k) { return a + (k + 1) * step + ((k + 1) * rest) / 5; };
            const bool less = d > 0 && __ldg(&src_step[probe(q)]) < want;
            const int below = __popc(__ballot_sync(0xffffffffu, less) >> (lane & ~3) & 15u);
            if (d > 0) {
              const int a1 = below > 0 ? probe(below - 1) + 1 : a;
              b = below < 4 ? probe(below) : b;
              a = a1;
            }
          }
          if (i <= kPosThreads && (lane & 3) == 0) run_at[i] = a;
          if (s0 + i0 + kPosThreads / 4 > (int64_t)last + 1 && i0 + kPosThreads / 4 <= kPosThreads) {
            // no step that is left is in the segment
            for (int k = i0 + kPosThreads / 4 + tid; k <= kPosThreads; k += kPosThreads) run_at[k] = end;
            break;
          }
        }
        __syncthreads();
        const int lo = run_at[tid], len = run_at[tid + 1] - lo;
        // Of steps that are not in order the first one's lower bound may be behind tokens that no run then holds.  From
        // it on every token is compared with the run that it is in.
        if (tid == 0 && s0 == first && lo != start) set_status(status, VCS_ERR_DEVICE_CHECK);
        int adv = 0;
        if (s <= last) {
          const int img = step_img[s], txt = step_txt[s];
          int im = 0, skip = 0, h = 1, w = 1;
          bool ok = len == 0 || len == txt || (int64_t)len == (int64_t)img + txt;
          if (len > 0 && img > 0 && (int64_t)len == (int64_t)img + txt) {
            const int t = step_grid[3 * s];
            h = step_grid[3 * s + 1];
            w = step_grid[3 * s + 2];
            // the grid holds the screenshot's tokens: then every product below is at most img
            ok = t > 0 && h > 0 && w > 0 && t <= img && h <= img && w <= img && (int64_t)h * w <= img &&
                 (int64_t)t * (h * w) == img;
            if (ok) {
              im = img;
              skip = max(t, max(h, w));
            } else {
              h = w = 1;
            }
          }
          if (!ok) set_status(status, VCS_ERR_DEVICE_CHECK);  // its tokens are counted like text
          adv = len - im + skip;
          run_img[tid] = im;
          run_skip[tid] = skip;
          run_h[tid] = h;
          run_w[tid] = w;
          // exact below 2^32 / c
          run_hm[tid] = h > 1 && (int64_t)img * h < (1ll << 32) ? 0xffffffffu / (uint32_t)h + 1u : 0u;
          run_wm[tid] = w > 1 && (int64_t)img * w < (1ll << 32) ? 0xffffffffu / (uint32_t)w + 1u : 0u;
        }
        int x = adv;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int y = __shfl_up_sync(0xffffffffu, x, o);
          if (lane >= o) x += y;
        }
        if (lane == 31) wsum[wid] = x;
        __syncthreads();
        int before = carry;
        for (int i = 0; i < wid; ++i) before += wsum[i];
        run_pos[tid] = before + x - adv;
        if (tid == kPosThreads - 1) carry_s = before + x;
        __syncthreads();
        carry = carry_s;
        const int n0 = max(lo_tok, run_at[0]), n1 = min(hi_tok, run_at[kPosThreads]);
        const int step0 = (int)s0;
        // token k of run r: a screenshot's by its grid, or text
        auto place = [&](int r, int k, int& frame, int& line, int& col) {
          const int h = run_h[r], w = run_w[r];
          const uint32_t hm = run_hm[r], wm = run_wm[r];
          line = wm != 0u ? div_by(k, w, wm) : k / w;
          col = k - line * w;
          frame = hm != 0u ? div_by(line, h, hm) : line / h;
          line -= frame * h;
        };
        auto whole = [&](int64_t m) { return vec && m >= n0 && m + 4 <= n1; };
        auto steps_at = [&](int64_t m) {
          return whole(m) ? __ldg(reinterpret_cast<const int4*>(src_step + m)) : make_int4(0, 0, 0, 0);
        };
        int4 ahead = steps_at((n0 & ~3) + 4 * tid);
        for (int64_t m64 = (n0 & ~3) + 4 * tid; m64 < n1; m64 += 4 * kPosThreads) {
          const int m = (int)m64;
          const int4 step = ahead;
          ahead = steps_at(m64 + 4 * kPosThreads);  // the next ones' load is under way while these are written
          // four tokens of one run, of its screenshot or of its text, in 16-byte accesses and with one division
          if (whole(m)) {
            const int r = step.x - step0;
            if (step.y == step.x && step.z == step.x && step.w == step.x && r >= 0 && r < kPosThreads &&
                m >= run_at[r] && m + 3 < run_at[r + 1]) {
              const int k = m - run_at[r], im = run_img[r], p = run_pos[r];
              if (k >= im) {
                const int t = p + run_skip[r] + k - im;
                const int4 x = make_int4(t, t + 1, t + 2, t + 3);
                *reinterpret_cast<int4*>(pos + m) = *reinterpret_cast<int4*>(pos + N + m) =
                    *reinterpret_cast<int4*>(pos + 2 * N + m) = x;
                continue;
              }
              if (k + 3 < im) {
                int f[4], l[4], c[4];
                place(r, k, f[0], l[0], c[0]);
#pragma unroll
                for (int v = 1; v < 4; ++v) {
                  const bool wrap = c[v - 1] + 1 == run_w[r], next = wrap && l[v - 1] + 1 == run_h[r];
                  c[v] = wrap ? 0 : c[v - 1] + 1;
                  l[v] = next ? 0 : l[v - 1] + wrap;
                  f[v] = f[v - 1] + next;
                }
                *reinterpret_cast<int4*>(pos + m) = make_int4(p + f[0], p + f[1], p + f[2], p + f[3]);
                *reinterpret_cast<int4*>(pos + N + m) = make_int4(p + l[0], p + l[1], p + l[2], p + l[3]);
                *reinterpret_cast<int4*>(pos + 2 * N + m) = make_int4(p + c[0], p + c[1], p + c[2], p + c[3]);
                continue;
              }
            }
          }
          for (int n = max(m, n0); n < min(m + 4, n1); ++n) {
            const int r = __ldg(&src_step[n]) - step0;
            if (r < 0 || r >= kPosThreads || n < run_at[r] || n >= run_at[r + 1]) {
              set_status(status, VCS_ERR_DEVICE_CHECK);  // tok_src_step decreases within the segment
              continue;
            }
            const int k = n - run_at[r], im = run_img[r], p = run_pos[r];
            int f, l, c;
            if (k < im)
              place(r, k, f, l, c);
            else
              f = l = c = run_skip[r] + k - im;
            pos[n] = p + f;
            pos[N + n] = p + l;
            pos[2 * N + n] = p + c;
          }
        }
        const int tile_end = run_at[kPosThreads];
        __syncthreads();
        if (tile_end >= hi_tok) break;
      }
    }
  }
}

// ------------------------------------------------------------------ inverse map
// For every trajectory token t the segment tokens that are copies of it, in order, whatever the map; no atomic
// decides an order.  A layout's map is made of stretches of consecutive tokens, so what is sorted is not its keys but
// runs: up to 512 neighbouring consecutive keys within one group of 2^shift trajectory tokens, as one word (group,
// length - 1) and the place of the first.  inverse_runs finds them and counts every group's runs and keys; a
// stable radix sort by 8-bit digits of the group brings a group's runs together, in order; then a warp takes a group:
// the ends of its runs give the tokens' counts, their scan inv_off and where each token's next copy goes.  The map is
// read once, and once more where runs begin.  15.8 M keys of long rollouts: 125 us (a sort of the keys themselves by
// three digits and a search of the offsets took 400); random keys, which are runs of one, take 770 against 430.
// A group of more than kChunk runs, which no layout of few segments has, is split among warps: the copies in each
// chunk, a scan, the places (5 M copies of one token: 4.1 ms, with one warp 204).  Far fewer keys than tokens, where
// the groups would be too wide or too many, are sorted by themselves.
// Keys outside [0, T) become T, behind all others.
constexpr int kSortThreads = 256;
constexpr int kPerThread = 16;
constexpr int kTile = kSortThreads * kPerThread;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int64_t kSmallOffsets = 8192;  // trajectory tokens whose searches take the one block about a launch's time
constexpr int kRunBits = 9;              // a run is within a warp's 512 keys
// Keys a group, on average.  A layout of 15.8 M keys takes 180, 135 and 130 us at 128, 256 and 512 (a call from
// Python), a map with as many trajectory tokens as keys 125 and 588 at 256 and 512: with 512 it would need groups of
// more than kCounters tokens, and its keys are sorted by themselves.
constexpr int kGroupKeys = 256;
constexpr int kGroups = 256;             // but one digit of groups at least
constexpr int kMostGroups = 4096;        // and up to these where a group would pass kCounters tokens
constexpr int kCounters = 512;           // trajectory tokens of a group at most
constexpr int kChunk = 1024;             // runs of a group that one warp takes; a group of more is split
constexpr int kGroupTile = 4096;         // groups scanned by a block
constexpr int kLongRun = 8;              // keys of a run, on average of 32, from which runs are taken one by one
constexpr int kAhead = 4;                // of a run's keys, loads before their stores
constexpr int kHeavyBlocks = 152;        // for the chunks of heavy groups
constexpr int kSortBlocks = 152 * 4;     // blocks, of as many tiles each as it takes

// Keys at, at + step, ... before n.  All loads first (the check of a key, which may report, would hold up the next
// one's load: a pass over 15.8 M keys took 140 us with it in between).
template <int STEP>
__device__ __forceinline__ void load_keys(const int32_t* __restrict__ keys, int64_t at, int64_t n, uint32_t T,
                                          int32_t* status, uint32_t (&key)[kPerThread]) {
  if (at + (kPerThread - 1) * STEP < n) {  // a whole tile: one address
    const int32_t* p = keys + at;
#pragma unroll
    for (int u = 0; u < kPerThread; ++u) key[u] = (uint32_t)__ldg(p + u * STEP);
  } else {
#pragma unroll
    for (int u = 0; u < kPerThread; ++u) key[u] = (uint32_t)__ldg(&keys[at + u * STEP < n ? at + u * STEP : n - 1]);
  }
  bool bad = false;
#pragma unroll
  for (int u = 0; u < kPerThread; ++u)
    if (key[u] >= T) {
      key[u] = T;
      bad = bad || at + u * STEP < n;
    }
  if (bad) set_status(status, VCS_ERR_DEVICE_CHECK);
}

// Exclusive sum over the block's threads of v.
__device__ __forceinline__ int block_before(int v, int32_t* wsum) {
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) wsum[wid] = x;
  __syncthreads();
  int at = x - v;
  for (int i = 0; i < wid; ++i) at += wsum[i];
  __syncthreads();
  return at;
}

// The runs of a block's `each` tiles, packed at the block's own places of run_key and run_at; how many of each first
// digit; and what they add to their groups (runs above 32 bits, keys below).
__global__ void __launch_bounds__(kSortThreads)
    inverse_runs(const int32_t* __restrict__ keys, int64_t n, uint32_t T, int shift, int each,
                 uint32_t* __restrict__ run_key, int32_t* __restrict__ run_at, int32_t* __restrict__ block_runs,
                 int32_t* __restrict__ counts, unsigned long long* __restrict__ groups, int32_t* status) {
  __shared__ int32_t c[256];
  __shared__ int32_t wsum[2][kSortWarps];
  constexpr int kRounds = kPerThread / 4;
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  c[tid] = 0;
  int64_t base = (int64_t)blockIdx.x * each * kTile;
  run_key += base;
  run_at += base;
  int runs = 0;
  const bool vec = (reinterpret_cast<uintptr_t>(keys) & 15u) == 0;
  for (int t = 0; t < each && base < n; ++t, base += kTile) {
    const int off = wid * (32 * kPerThread), here = (int)(n - base < kTile ? n - base : kTile);
    const int live = min(32 * kPerThread, here - off);  // keys of the warp, possibly less than none
    // the warp's keys 128 u + 4 lane + j
    const int64_t mine = base + off + 4 * lane;
    uint32_t key[kRounds][4], heads[kRounds][4];
    if (vec && live == 32 * kPerThread) {
#pragma unroll
      for (int u = 0; u < kRounds; ++u) {
        const int4 k = __ldg(reinterpret_cast<const int4*>(keys + mine) + 32 * u);
        key[u][0] = k.x, key[u][1] = k.y, key[u][2] = k.z, key[u][3] = k.w;
      }
    } else {
#pragma unroll
      for (int u = 0; u < kRounds; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j) key[u][j] = (uint32_t)__ldg(&keys[min(mine + 128 * u + j, n - 1)]);
    }
    bool bad = false;
    int found = 0;
#pragma unroll
    for (int u = 0; u < kRounds; ++u) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        bad = bad || key[u][j] >= T;  // the last key's copies behind n tell the same
        key[u][j] = min(key[u][j], T);
      }
      uint32_t last = __shfl_up_sync(0xffffffffu, key[u][3], 1);
      if (u > 0) {
        const uint32_t end = __shfl_sync(0xffffffffu, key[u - 1][3], 31);
        if (lane == 0) last = end;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bool head = key[u][j] != last + 1 || (key[u][j] & ((1u << shift) - 1u)) == 0;
        last = key[u][j];
        heads[u][j] = __ballot_sync(0xffffffffu, (head || 128 * u + 4 * lane + j == 0) &&
                                                     128 * u + 4 * lane + j < live);
        found += __popc(heads[u][j]);
      }
    }
    if (bad) set_status(status, VCS_ERR_DEVICE_CHECK);
    if (lane == 0) wsum[t & 1][wid] = found;
    __syncthreads();
    int at = runs + found;  // behind the warp's runs
#pragma unroll
    for (int w = 0; w < kSortWarps; ++w) {
      if (w < wid) at += wsum[t & 1][w];
      runs += wsum[t & 1][w];
    }
    int next = live;  // the first place behind the run
    const uint32_t below = (1u << lane) - 1u, above = ~(2u * below + 1u);
    // the place of a lane's first head
    auto first_of = [](const uint32_t (&h)[4], int lane_of) {
      return 4 * lane_of + (h[0] >> lane_of & 1 ? 0 : h[1] >> lane_of & 1 ? 1 : h[2] >> lane_of & 1 ? 2 : 3);
    };
#pragma unroll
    for (int u = kRounds - 1; u >= 0; --u) {
      const uint32_t any = heads[u][0] | heads[u][1] | heads[u][2] | heads[u][3];
      if (any == 0) continue;
      at -= __popc(heads[u][0]) + __popc(heads[u][1]) + __popc(heads[u][2]) + __popc(heads[u][3]);
      if (any >> lane & 1) {
        int to = at + __popc(heads[u][0] & below) + __popc(heads[u][1] & below) + __popc(heads[u][2] & below) +
                 __popc(heads[u][3] & below);
        const int then = (any & above) != 0 ? 128 * u + first_of(heads[u], __ffs(any & above) - 1) : next;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (heads[u][j] >> lane & 1) {
            const int place = 128 * u + 4 * lane + j;
            int upto = then;
#pragma unroll
            for (int i = 3; i > j; --i)
              if (heads[u][i] >> lane & 1) upto = 128 * u + 4 * lane + i;
            const uint32_t group = key[u][j] >> shift;
            run_key[to] = group << kRunBits | (uint32_t)(upto - place - 1);
            run_at[to++] = (int32_t)(base + off + place);
            atomicAdd(&c[group & 255u], 1);
            atomicAdd(&groups[group], 1ull << 32 | (unsigned long long)(upto - place));
          }
      }
      next = 128 * u + first_of(heads[u], __ffs(any) - 1);
    }
  }
  __syncthreads();
  counts[(size_t)tid * gridDim.x + blockIdx.x] = c[tid];
  if (tid == 0) block_runs[blockIdx.x] = runs;
}

// Packed runs that a block takes, of n by so many blocks: few runs are spread over more blocks than tiles would.
__device__ __forceinline__ int64_t packed_part(int64_t n, int blocks) {
  constexpr int64_t kLeast = kTile / 4;
  return ((n + kLeast - 1) / kLeast + blocks - 1) / blocks * kLeast;
}

// Digit counts of packed runs.
__global__ void __launch_bounds__(kSortThreads)
    inverse_count(const uint32_t* __restrict__ run_key, const int32_t* __restrict__ num_runs, int shift,
                  int32_t* __restrict__ counts) {
  __shared__ int32_t c[256];
  const int64_t n = *num_runs, part = packed_part(n, gridDim.x), base = blockIdx.x * part;
  if (base >= n) return;
  c[threadIdx.x] = 0;
  __syncthreads();
  const int here = (int)min(n - base, part);
  run_key += base;
#pragma unroll 8
  for (int i = threadIdx.x; i < here; i += kSortThreads) atomicAdd(&c[run_key[i] >> shift & 255u], 1);
  __syncthreads();
  counts[(size_t)threadIdx.x * gridDim.x + blockIdx.x] = c[threadIdx.x];
}

// Exclusive scan of v over the block's 1,024 threads; all is its sum.
template <typename T>
__device__ __forceinline__ T scan_1024(T v, T* wsum, T& all) {
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  T x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const T y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) wsum[wid] = x;
  __syncthreads();
  T w = wsum[lane];
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const T y = __shfl_up_sync(0xffffffffu, w, o);
    if (lane >= o) w += y;
  }
  const T before = __shfl_sync(0xffffffffu, w, wid > 0 ? wid - 1 : 0);
  all = __shfl_sync(0xffffffffu, w, 31);
  __syncthreads();
  return x - v + (wid > 0 ? before : T(0));
}

// The groups of more than kChunk runs: their chunks stand at `slot` and behind it.
struct HeavyList {
  int32_t* num;     // chunks, groups
  int2* group;      // group, its first slot
  int2* chunk;      // of a slot: its group, the chunk's number there
  int32_t* counts;  // of a slot: the chunk's copies of the group's tokens, then their first places
};

// Block b < 256: the exclusive scan of digit b's counts over the blocks that counted (with packed runs, as many as
// num_runs fill), and their sum.
// A block behind them: that of kGroupTile groups, and their sum; and the list of heavy groups.
__global__ void __launch_bounds__(1024)
    inverse_scan(int32_t* __restrict__ counts, int blocks, const int32_t* __restrict__ num_runs,
                 int32_t* __restrict__ totals, unsigned long long* __restrict__ groups, int num_groups,
                 unsigned long long* __restrict__ group_sums, HeavyList heavy) {
  if (blockIdx.x < 256) {
    __shared__ int32_t wsum[32];
    int32_t* c = counts + (size_t)blockIdx.x * blocks;
    int live = blocks;
    if (num_runs != nullptr) {
      const int64_t n = *num_runs, part = packed_part(n, blocks);
      live = (int)((n + part - 1) / part);
    }
    int carry = 0, all;
    for (int base = 0; base < live; base += 1024) {
      const int i = base + (int)threadIdx.x;
      const int x = scan_1024(i < live ? c[i] : 0, wsum, all);
      if (i < live) c[i] = carry + x;
      carry += all;
    }
    if (threadIdx.x == 0) totals[blockIdx.x] = carry;
  } else {
    __shared__ unsigned long long wsum[32];
    constexpr int kEach = kGroupTile / 1024;
    const int at = ((int)blockIdx.x - 256) * kGroupTile + (int)threadIdx.x * kEach;
    unsigned long long v[kEach], sum = 0, all;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      v[i] = at + i < num_groups ? groups[at + i] : 0ull;
      sum += v[i];
    }
    unsigned long long x = scan_1024(sum, wsum, all);
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      if (at + i < num_groups) groups[at + i] = x;
      x += v[i];
      if (v[i] >> 32 > kChunk) {  // where its chunks stand among the others' makes no difference
        const int chunks = (int)(((v[i] >> 32) + kChunk - 1) / kChunk), slot = atomicAdd(&heavy.num[0], chunks);
        heavy.group[atomicAdd(&heavy.num[1], 1)] = make_int2(at + i, slot);
        for (int c = 0; c < chunks; ++c) heavy.chunk[slot + c] = make_int2(at + i, c);
      }
    }
    if (threadIdx.x == 0) group_sums[blockIdx.x - 256] = all;
  }
}

struct SortTile {
  int32_t seen[kSortWarps][256];  // keys of each digit that a warp has passed; then where its next one goes
  int32_t wsum[kSortWarps];
  int32_t to[256];                // from a place in the tile to the digit's place in the output
  uint32_t key[kTile + kTile / 16];  // at skew(place)
  int32_t val[kTile + kTile / 16];
};
// A tile has some 16 keys a digit, so that a warp's keys of consecutive digits go 16 places apart, all to two banks: a
// word of space behind every 16 spreads them.
__device__ __forceinline__ int skew(int i) { return i + (i >> 4); }

// Places of the tile's keys sorted by a digit.  Warp w has its keys [32 rounds w, + 32 rounds) in order, 32 at a
// time (key u of a thread is there if 32 u < live, and u < rounds): a key's
// rank among the warp's equal digits is the count of them before it, by votes on the digit's bits (a match
// instruction takes several times as long) and a running count.
// Returns the first place of the thread's digit, and how many keys have it.
__device__ __forceinline__ int place_tile(SortTile& s, const uint32_t (&key)[kPerThread], int live, int rounds,
                                          int shift, int (&place)[kPerThread], int& count) {
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
#pragma unroll
  for (int w = 0; w < kSortWarps; ++w) s.seen[w][tid] = 0;
  __syncthreads();
  uint32_t same[kPerThread];
#pragma unroll
  for (int u = 0; u < kPerThread; ++u) {
    if (u >= rounds) break;
    const bool on = 32 * u < live;
    const uint32_t dg = (key[u] >> shift) & 255u;
    same[u] = __ballot_sync(0xffffffffu, on);
#pragma unroll
    for (int b = 0; b < 8; ++b) {
      const bool bit = dg >> b & 1;
      const uint32_t v = __ballot_sync(0xffffffffu, bit);
      same[u] &= bit ? v : ~v;
    }
    // the first lane of each digit adds; a warp's additions to shared memory are done in order
    place[u] = 0;
    if (on && (same[u] & ((1u << lane) - 1u)) == 0) place[u] = atomicAdd(&s.seen[wid][dg], __popc(same[u]));
  }
#pragma unroll
  for (int u = 0; u < kPerThread; ++u) {
    if (u >= rounds) break;
    place[u] = __shfl_sync(0xffffffffu, place[u], (__ffs(same[u]) - 1) & 31) + __popc(same[u] & ((1u << lane) - 1u));
  }
  __syncthreads();
  count = 0;
#pragma unroll
  for (int w = 0; w < kSortWarps; ++w) count += s.seen[w][tid];
  const int first = block_before(count, s.wsum);
  int at = first;
#pragma unroll
  for (int w = 0; w < kSortWarps; ++w) {
    const int c = s.seen[w][tid];
    s.seen[w][tid] = at;
    at += c;
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < kPerThread; ++u)
    if (u < rounds) place[u] += s.seen[wid][(key[u] >> shift) & 255u];
  return first;
}

// A pass of the runs' sort.  The first one's blocks have block_runs runs each, and it says how many there are; later
// ones' are packed.  A tile is sorted in shared memory first, so that a digit's runs leave together.
__global__ void __launch_bounds__(kSortThreads, 3)
    inverse_scatter(const uint32_t* __restrict__ keys, const int32_t* __restrict__ vals, int shift, int each,
                    const int32_t* __restrict__ counts, const int32_t* __restrict__ totals,
                    const int32_t* __restrict__ block_runs, int32_t* __restrict__ num_runs,
                    uint32_t* __restrict__ keys_out, int32_t* __restrict__ vals_out) {
  __shared__ SortTile s;
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  int64_t base = (int64_t)blockIdx.x * each * kTile;
  int all;
  if (block_runs != nullptr) {
    all = block_runs[blockIdx.x];
  } else {
    const int64_t n = *num_runs, part = packed_part(n, gridDim.x);
    base = blockIdx.x * part;
    if (base >= n) return;
    all = (int)min(n - base, part);
  }
  keys += base;
  vals += base;
  int to = block_before(totals[tid], s.wsum);  // of the thread's digit
  if (block_runs != nullptr && blockIdx.x == 0 && tid == kSortThreads - 1) *num_runs = to + totals[tid];
  to += counts[(size_t)tid * gridDim.x + blockIdx.x];
  for (int done = 0; done < all; done += kTile) {
    const int here = min(all - done, kTile), rounds = (here + kSortThreads - 1) / kSortThreads;
    const int off = wid * (32 * rounds) + lane, live = here - off;  // run u of the thread: off + 32 u < here
    uint32_t key[kPerThread];
    int val[kPerThread], place[kPerThread];
#pragma unroll
    for (int u = 0; u < kPerThread; ++u) {
      const bool on = u < rounds && 32 * u < live;
      key[u] = on ? __ldg(&keys[done + off + 32 * u]) : 0u;
      val[u] = on ? __ldg(&vals[done + off + 32 * u]) : 0;
    }
    int count;
    s.to[tid] = to - place_tile(s, key, live, rounds, shift, place, count);
    to += count;
#pragma unroll
    for (int u = 0; u < kPerThread; ++u)
      if (u < rounds && 32 * u < live) {
        s.key[skew(place[u])] = key[u];
        s.val[skew(place[u])] = val[u];
      }
    __syncthreads();
    for (int i = tid; i < here; i += kSortThreads) {
      const uint32_t k = s.key[skew(i)];
      const int at = s.to[k >> shift & 255u] + i;
      keys_out[at] = k;
      vals_out[at] = s.val[skew(i)];
    }
    __syncthreads();
  }
}

// Up to one tile of keys of few trajectory tokens: sorted by one block in shared memory, and the offsets by searches
// there.
__global__ void __launch_bounds__(kSortThreads)
    inverse_small(const int32_t* __restrict__ keys, int32_t n, uint32_t T, int passes, int32_t* __restrict__ off,
                  int32_t* __restrict__ vals_out, int32_t* status) {
  __shared__ SortTile s;
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  const int rounds = (n + kSortThreads - 1) / kSortThreads;
  const int at = wid * 32 * rounds + lane, live = n - at;
  uint32_t key[kPerThread];
  int val[kPerThread], place[kPerThread];
  load_keys<32>(keys, at, n, T, status, key);
#pragma unroll
  for (int u = 0; u < kPerThread; ++u) val[u] = at + 32 * u;
  for (int p = 0; p < passes; ++p) {
    int count;
    place_tile(s, key, live, rounds, 8 * p, place, count);
#pragma unroll
    for (int u = 0; u < kPerThread; ++u)
      if (u < rounds && 32 * u < live) {
        s.key[skew(place[u])] = key[u];
        s.val[skew(place[u])] = val[u];
      }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kPerThread; ++u)
      if (u < rounds && 32 * u < live) {
        key[u] = s.key[skew(at + 32 * u)];
        val[u] = s.val[skew(at + 32 * u)];
      }
    __syncthreads();
  }
  for (int i = tid; i < n; i += kSortThreads) vals_out[i] = s.val[skew(i)];
  for (uint32_t t = tid; t <= T; t += kSortThreads) {
    int a = 0, b = n;
    while (a < b) {
      const int mid = (a + b) >> 1;
      if (s.key[skew(mid)] < t) a = mid + 1;
      else b = mid;
    }
    off[t] = a;
  }
}

// A group's runs and its first place in inv_tok.
struct Group {
  const uint32_t* run_key;
  const int32_t* run_at;
  int runs, first;
  uint32_t token;  // its first
  int width;       // tokens
};
__device__ __forceinline__ Group group_at(int g, uint32_t T, int shift, const uint32_t* run_key, const int32_t* run_at,
                                          const unsigned long long* groups, int num_groups,
                                          const unsigned long long* group_sums) {
  unsigned long long before = 0;
  for (int i = threadIdx.x & 31; i < g / kGroupTile; i += 32) before += group_sums[i];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) before += __shfl_xor_sync(0xffffffffu, before, o);
  const unsigned long long in_tile = groups[g];
  const unsigned long long end = (g + 1) % kGroupTile == 0 || g + 1 == num_groups ? group_sums[g / kGroupTile]
                                                                                  : groups[g + 1];
  before += in_tile;
  Group r;
  r.runs = (int)((end >> 32) - (in_tile >> 32));
  r.run_key = run_key + (before >> 32);
  r.run_at = run_at + (before >> 32);
  r.first = (int)(uint32_t)before;
  r.token = (uint32_t)g << shift;
  r.width = (int)min(1u << shift, T + 1 - r.token);
  return r;
}

// Chunk c of the group's runs, as a group.
__device__ __forceinline__ Group chunk_of(Group g, int c) {
  g.run_key += (int64_t)c * kChunk;
  g.run_at += (int64_t)c * kChunk;
  g.runs = min(g.runs - c * kChunk, kChunk);
  return g;
}

__device__ __forceinline__ int warp_scan(int x) {  // inclusive
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  return x;
}

// Sums of c[0], ... in its place, from `carry` on: of those before (places of counts), or with the own (counts of
// changes).  256 at a time, eight a lane: a scan over the warp for every 32 was half of inverse_place's instructions.
constexpr int kSpan = 256;
template <bool BEFORE>
__device__ __forceinline__ void sums(int32_t* c, int width, int carry) {
  const int lane = threadIdx.x & 31;
  for (int i0 = 0; i0 < width; i0 += kSpan) {
    int4* at = reinterpret_cast<int4*>(c + i0) + 2 * lane;
    const int4 lo = at[0], hi = at[1];
    int v[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w}, sum = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += v[i];
    const int upto = warp_scan(sum) + carry;
    int x = upto - sum;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int own = v[i];
      v[i] = BEFORE ? x : x + own;
      x += own;
    }
    at[0] = make_int4(v[0], v[1], v[2], v[3]);
    at[1] = make_int4(v[4], v[5], v[6], v[7]);
    carry = __shfl_sync(0xffffffffu, upto, 31);
  }
  __syncwarp();
}

// The copies of the group's tokens into c, from where its runs begin and end.
__device__ __forceinline__ void count_copies(const Group& g, const int32_t* __restrict__ keys, uint32_t T, int32_t* c) {
  const int lane = threadIdx.x & 31;
  for (int i = 4 * lane; i < g.width; i += 128) *reinterpret_cast<int4*>(c + i) = make_int4(0, 0, 0, 0);
  for (int i = g.width + lane; i < (g.width + kSpan - 1) / kSpan * kSpan; i += 32) c[i] = 0;
  __syncwarp();
  for (int r = lane; r < g.runs; r += 32) {
    const int first = (int)(min((uint32_t)__ldg(&keys[g.run_at[r]]), T) - g.token);
    const int end = first + (int)(g.run_key[r] & ((1u << kRunBits) - 1u)) + 1;
    atomicAdd(&c[first], 1);
    if (end < g.width) atomicAdd(&c[end], -1);
  }
  __syncwarp();
  sums<false>(c, g.width, 0);
}

// The runs' segment tokens, in order, to their tokens' places c.  A run's tokens differ, so long runs are taken one by
// one; the keys of short ones are taken 32 at a time, and those of one token told apart by votes on the bits.
__device__ __forceinline__ void place_copies(const Group& g, const int32_t* __restrict__ keys, uint32_t T, int shift,
                                             int32_t* c, int32_t* __restrict__ inv_tok) {
  const int lane = threadIdx.x & 31;
  for (int r = 0; r < g.runs; r += 32) {
    const bool there = r + lane < g.runs;
    const int at = there ? g.run_at[r + lane] : 0;
    const int len = there ? (int)(g.run_key[r + lane] & ((1u << kRunBits) - 1u)) + 1 : 0;
    const int first = there ? (int)(min((uint32_t)__ldg(&keys[at]), T) - g.token) : 0;
    const int upto = warp_scan(len);  // keys of the runs up to this one
    const int all = __shfl_sync(0xffffffffu, upto, 31), here = min(g.runs - r, 32);
    if (all >= here * kLongRun) {
      for (int j = 0; j < here; ++j) {
        const int f = __shfl_sync(0xffffffffu, first, j), l = __shfl_sync(0xffffffffu, len, j);
        const int a = __shfl_sync(0xffffffffu, at, j);
        for (int e = lane; e < l; e += 32 * kAhead) {
          int to[kAhead];
#pragma unroll
          for (int u = 0; u < kAhead; ++u)
            if (e + 32 * u < l) to[u] = c[f + e + 32 * u];
#pragma unroll
          for (int u = 0; u < kAhead; ++u)
            if (e + 32 * u < l) {
              inv_tok[to[u]] = a + e + 32 * u;
              c[f + e + 32 * u] = to[u] + 1;
            }
        }
        __syncwarp();
      }
    } else {
      for (int b = 0; b < all; b += 32) {
        const int e = b + lane;
        int j = 0;  // runs that end at or before key e
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
          if (__shfl_sync(0xffffffffu, upto, j + o - 1) <= e) j += o;
        const int in_run = e - __shfl_sync(0xffffffffu, upto - len, j);
        const int i = __shfl_sync(0xffffffffu, first, j) + in_run, a = __shfl_sync(0xffffffffu, at, j) + in_run;
        const bool on = e < all;
        uint32_t same = __ballot_sync(0xffffffffu, on);
        for (int k = 0; k < shift; ++k) {
          const bool bit = i >> k & 1;
          const uint32_t v = __ballot_sync(0xffffffffu, bit);
          same &= bit ? v : ~v;
        }
        const int to = on ? c[i] + __popc(same & ((1u << lane) - 1u)) : 0;
        __syncwarp();
        if (on) {
          inv_tok[to] = a;
          if (same >> lane == 1u) c[i] = to + 1;  // the last of its token
        }
        __syncwarp();
      }
    }
  }
}

// A warp a group of up to kChunk runs: its tokens' copies, their scan, and the copies to their places.  The warps of
// the blocks behind them: the copies in the chunks of the other groups.
__global__ void __launch_bounds__(kSortThreads, 5)
    inverse_place(const int32_t* __restrict__ keys, uint32_t T, int shift, const uint32_t* __restrict__ run_key,
                  const int32_t* __restrict__ run_at, const unsigned long long* __restrict__ groups, int num_groups,
                  const unsigned long long* __restrict__ group_sums, HeavyList heavy, int32_t* __restrict__ inv_off,
                  int32_t* __restrict__ inv_tok) {
  __shared__ __align__(16) int32_t counters[kSortWarps][kCounters];
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, blocks = (num_groups + kSortWarps - 1) / kSortWarps;
  int32_t* c = counters[wid];
  if ((int)blockIdx.x < blocks) {
    const int g = blockIdx.x * kSortWarps + wid;
    if (g >= num_groups) return;
    const Group group = group_at(g, T, shift, run_key, run_at, groups, num_groups, group_sums);
    if (group.runs > kChunk) return;
    count_copies(group, keys, T, c);
    sums<true>(c, group.width, group.first);
    for (int i = lane; i < group.width; i += 32) inv_off[(size_t)group.token + i] = c[i];
    __syncwarp();
    place_copies(group, keys, T, shift, c, inv_tok);
  } else {
    const int chunks = heavy.num[0];
    for (int k = ((int)blockIdx.x - blocks) * kSortWarps + wid; k < chunks; k += kHeavyBlocks * kSortWarps) {
      const int2 which = heavy.chunk[k];
      const Group group = group_at(which.x, T, shift, run_key, run_at, groups, num_groups, group_sums);
      int32_t* to = heavy.counts + (size_t)k * kCounters;
      count_copies(chunk_of(group, which.y), keys, T, c);
      for (int i = lane; i < group.width; i += 32) to[i] = c[i];
      __syncwarp();
    }
  }
}

// A block a heavy group, a thread a token: the scan of the tokens' copies, then where each chunk's first one goes.
__global__ void __launch_bounds__(kCounters)
    inverse_heavy_scan(uint32_t T, int shift, const uint32_t* __restrict__ run_key, const int32_t* __restrict__ run_at,
                       const unsigned long long* __restrict__ groups, int num_groups,
                       const unsigned long long* __restrict__ group_sums, HeavyList heavy,
                       int32_t* __restrict__ inv_off) {
  __shared__ int32_t wsum[kCounters / 32];
  const int tid = threadIdx.x;
  for (int k = blockIdx.x; k < heavy.num[1]; k += gridDim.x) {
    const int2 which = heavy.group[k];
    const Group group = group_at(which.x, T, shift, run_key, run_at, groups, num_groups, group_sums);
    const int chunks = (group.runs + kChunk - 1) / kChunk;
    int32_t* counts = heavy.counts + (size_t)which.y * kCounters + tid;
    const bool on = tid < group.width;
    int copies = 0;
#pragma unroll 8
    for (int c = 0; c < chunks; ++c)
      if (on) copies += counts[(size_t)c * kCounters];
    int next = group.first + block_before(copies, wsum);
    if (on) inv_off[(size_t)group.token + tid] = next;
    for (int c0 = 0; c0 < chunks; c0 += 8) {
      int v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) v[u] = on && c0 + u < chunks ? counts[(size_t)(c0 + u) * kCounters] : 0;
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        if (on && c0 + u < chunks) counts[(size_t)(c0 + u) * kCounters] = next;
        next += v[u];
      }
    }
  }
}

// A warp a chunk of a heavy group: its copies to their places.
__global__ void __launch_bounds__(kSortThreads)
    inverse_heavy_place(const int32_t* __restrict__ keys, uint32_t T, int shift, const uint32_t* __restrict__ run_key,
                        const int32_t* __restrict__ run_at, const unsigned long long* __restrict__ groups,
                        int num_groups, const unsigned long long* __restrict__ group_sums, HeavyList heavy,
                        int32_t* __restrict__ inv_tok) {
  __shared__ int32_t counters[kSortWarps][kCounters];
  const int wid = threadIdx.x >> 5, chunks = heavy.num[0];
  int32_t* c = counters[wid];
  for (int k = blockIdx.x * kSortWarps + wid; k < chunks; k += gridDim.x * kSortWarps) {
    const int2 which = heavy.chunk[k];
    const Group group = group_at(which.x, T, shift, run_key, run_at, groups, num_groups, group_sums);
    __syncwarp();
    for (int i = threadIdx.x & 31; i < group.width; i += 32) c[i] = heavy.counts[(size_t)k * kCounters + i];
    __syncwarp();
    place_copies(chunk_of(group, which.y), keys, T, shift, c, inv_tok);
  }
}

// Single keys as what is sorted: for more trajectory tokens than kCounters a group.
__global__ void __launch_bounds__(kSortThreads)
    inverse_keys(const int32_t* __restrict__ keys, int64_t n, uint32_t T, uint32_t* __restrict__ key_out,
                 int32_t* __restrict__ at_out, int32_t* __restrict__ num, int32_t* status) {
  const int64_t i = (int64_t)blockIdx.x * kSortThreads + threadIdx.x;
  if (i == 0) *num = (int32_t)n;
  if (i >= n) return;
  const uint32_t k = (uint32_t)keys[i];
  if (k >= T) set_status(status, VCS_ERR_DEVICE_CHECK);
  key_out[i] = min(k, T);
  at_out[i] = (int32_t)i;
}

// off[t] = first place of a key >= t in the sorted keys, for t in a block's 1,024: two searches bound
// the block's keys; counts of them in shared memory and a scan give the rest, or searches where there are many.
constexpr int kOffTile = 1024;
__global__ void __launch_bounds__(256) inverse_offsets(const uint32_t* __restrict__ keys, int32_t n, int64_t T,
                                                       int32_t* __restrict__ off) {
  __shared__ int32_t c[kOffTile];
  __shared__ int32_t bound[2];
  __shared__ int32_t wsum[8];
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  const int64_t t0 = (int64_t)blockIdx.x * kOffTile;
#pragma unroll
  for (int u = 0; u < kOffTile / 256; ++u) c[u * 256 + tid] = 0;
  if (wid < 2) {  // a warp a search: the keys from `a` on, 32 probes at a time
    const int64_t t = t0 + wid * (int64_t)kOffTile;
    int a = 0, len = n;
    while (len > 0) {
      const int step = (len + 31) / 32;
      const int at = a + lane * step;
      const bool less = lane * step < len && __ldg(&keys[at]) < t;
      const int c = __popc(__ballot_sync(0xffffffffu, less));  // the probes of smaller keys come first
      if (c == 0) break;
      const int from = (c - 1) * step + 1;  // past the last smaller one
      len = min(step - 1, len - from);
      a += from;
    }
    if (lane == 0) bound[wid] = a;
  }
  __syncthreads();
  const int lo = bound[0], hi = bound[1];
  if (hi - lo > 4 * kOffTile) {
    for (int64_t t = t0 + tid; t < t0 + kOffTile && t <= T; t += 256) {
      int a = lo, b = hi;
      while (a < b) {
        const int mid = a + ((b - a) >> 1);
        if (keys[mid] < t) a = mid + 1;
        else b = mid;
      }
      off[t] = a;
    }
    return;
  }
  for (int i = lo + tid; i < hi; i += 256) atomicAdd(&c[keys[i] - t0], 1);
  __syncthreads();
  int v[kOffTile / 256], sum = 0;
#pragma unroll
  for (int u = 0; u < kOffTile / 256; ++u) {
    v[u] = c[tid * (kOffTile / 256) + u];
    sum += v[u];
  }
  int x = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) wsum[wid] = x;
  __syncthreads();
  int at = lo + x - sum;
  for (int i = 0; i < wid; ++i) at += wsum[i];
#pragma unroll
  for (int u = 0; u < kOffTile / 256; ++u) {
    const int64_t t = t0 + tid * (kOffTile / 256) + u;
    if (t <= T) off[t] = at;
    at += v[u];
  }
}

// ------------------------------------------------------------------ rotation
constexpr int kRopeThreads = 32 * kRopeWarps;
constexpr int kBatch = kRopeCopies;
constexpr int kMaxPairs = VCS_ROPE_MAX_PAIRS;

struct RopeArgs {
  const int4 *q_in, *k_in, *v_in;
  int4 *q_out, *k_out, *v_out;
  int64_t rows_in, rows_out;     // tokens of the inputs and of the outputs
  const int32_t* pos;            // [axes][segment tokens]
  int64_t pos_stride;
  const int32_t* map;            // forward: tok_gather; backward: inv_tok (nullptr: token n is row n)
  const int32_t* off;            // backward: inv_off
  int32_t hq, hkv;
  int32_t chunks;                // 16-byte chunks of a row
  int32_t per;                   // rows a warp takes together
  int32_t turned;                // items of a row that are rotated (pairs of chunks, or chunks if interleaved)
  int32_t plain;                 // and its chunks that are not
  uint32_t turned_magic, plain_magic;  // of div_by
  int32_t* status;
  uint64_t turn[kMaxPairs];      // inv_freq / 2 pi in 2^-64 turns
  uint8_t axis[kMaxPairs];
};

__device__ __forceinline__ int4 ld_stream(const int4* p) {
  int4 r;
  asm volatile("ld.global.nc.L1::no_allocate.v4.s32 {%0, %1, %2, %3}, [%4];"
               : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w)
               : "l"(p));
  return r;
}
__device__ __forceinline__ void st_stream(int4* p, int4 v) {
  asm volatile("st.global.cs.v4.s32 [%0], {%1, %2, %3, %4};" ::"l"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w)
               : "memory");
}

// the two bf16 of a word, exactly
__device__ __forceinline__ float lo_f(int w) { return __uint_as_float((uint32_t)w << 16); }
__device__ __forceinline__ float hi_f(int w) { return __uint_as_float((uint32_t)w & 0xffff0000u); }
__device__ __forceinline__ int& word(int4& x, int i) { return i == 0 ? x.x : i == 1 ? x.y : i == 2 ? x.z : x.w; }
__device__ __forceinline__ int pack2(uint64_t f) {
  float a, b;
  dev::f2unpack(f, a, b);
  return (int)dev::pack_bf16(a, b);
}

// A warp takes `per` consecutive output tokens, one where a row is some 8 KB or more.  Lane l computes the
// angles of pairs l, l + 32, ... of all their copies into the warp's table (forward: a token has one copy), then
// the lanes take each row's items in turn.  An item is, with pairs (i, i + rot/2), the chunks of eight dims c and
// c + rot/16, which hold eight whole pairs; with neighbouring pairs, one chunk of four.  The table holds two
// pairs (cos, cos, sin, sin) in 16 bytes, the operands of packed fp32 arithmetic, at [pair of the item / 2][item of
// the row], so that lanes on neighbouring items read neighbouring 16 bytes.
template <int NP, bool INTER, bool BWD>
__global__ void __launch_bounds__(kRopeThreads, 8) rope_rows(const __grid_constant__ RopeArgs a) {
  constexpr int B = kBatch;
  constexpr int H = INTER ? 2 : 4;         // two pairs each: an item's table entries
  constexpr int IC = INTER ? 1 : 2;        // chunks of an item
  constexpr int U = INTER ? 2 : 1;         // items a lane has in flight
  extern __shared__ float4 table[];        // rope_table.h
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  float4* tab = table + rope_copy_at<NP>(wid, BWD ? B : a.per, 0);
  uint64_t turn[NP];
  int axis[NP], slot[NP];                  // slot: of the pair's cosine in the table, as floats; -1: none
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    const int pair = lane + 32 * p, item = pair / (2 * H), k = pair % (2 * H);
    turn[p] = a.turn[pair];
    axis[p] = a.axis[pair];
    slot[p] = pair < a.turned * 2 * H ? 4 * rope_entry(k >> 1, a.turned, item) + (k & 1) : -1;
  }
  const int heads = a.hq + a.hkv;
  const int turned = heads * a.turned, plain = heads * a.plain;
  const int q_row = a.hq * a.chunks, kv_row = a.hkv * a.chunks;  // chunks of a token
  const int64_t stride = (int64_t)gridDim.x * kRopeWarps * a.per;
  for (int64_t r0 = (blockIdx.x * (int64_t)kRopeWarps + wid) * a.per; r0 < a.rows_out; r0 += stride) {
    const int rows = (int)(a.rows_out - r0 < a.per ? a.rows_out - r0 : a.per);
    // held: on lane j, the input row of copy j of the batch, -1 for none
    int held = -1;
    // of `count` copies; their positions are those of tokens first + j (forward) or of the rows held
    auto angles = [&](int count, int64_t first) {
      __syncwarp();
      for (int j = 0; j < count; ++j) {
        const int64_t n = BWD ? __shfl_sync(0xffffffffu, held, j) : first + j;
        if (n < 0) continue;
        float* t = reinterpret_cast<float*>(tab + rope_copy_at<NP>(0, 0, j));
#pragma unroll
        for (int p = 0; p < NP; ++p) {
          const uint64_t ph = (uint64_t)(int64_t)__ldg(&a.pos[axis[p] * a.pos_stride + n]) * turn[p];
          float s, c;
          sincospif((float)(int32_t)(ph >> 32) * 0x1p-31f, &s, &c);
          if (slot[p] >= 0) {
            t[slot[p]] = c;
            t[slot[p] + 2] = BWD ? -s : s;
          }
        }
      }
      __syncwarp();
    };
    // a batch of copies: on lanes j < count, row j of the list (or, without one, rows r0 + j themselves)
    auto hold = [&](const int32_t* list, int count) {
      const bool mine = lane < count;
      held = !mine ? -1 : list != nullptr ? __ldg(&list[lane]) : (int)r0 + lane;
      if (mine && (held < 0 || held >= a.rows_in)) {
        set_status(a.status, VCS_ERR_DEVICE_CHECK);
        held = -1;
      }
    };
    // backward: lane i <= rows holds where row i's copies start in the inverse's list; of an inconsistent
    // list there are none
    int start = lane;
    if (BWD && a.off != nullptr) start = lane <= rows ? __ldg(&a.off[r0 + lane]) : 0;
    const int64_t most = BWD && a.off != nullptr ? a.rows_in : B;
    const int next = __shfl_down_sync(0xffffffffu, start, 1);
    const bool bad = lane < rows && (start < 0 || next < start || next > most);
    if (bad) set_status(a.status, VCS_ERR_DEVICE_CHECK);
    // All the rows' copies as one batch if they are few, else a row's at a time.
    const int begin = __shfl_sync(0xffffffffu, start, 0);
    const int all = __shfl_sync(0xffffffffu, start, rows) - begin;
    const bool together = !__any_sync(0xffffffffu, bad) && all <= B;
    if (together) {
      hold(BWD ? (a.off != nullptr ? a.map + begin : nullptr) : a.map != nullptr ? a.map + r0 : nullptr, all);
      angles(all, r0);
    }
    for (int i = 0; i < rows; ++i) {
      const int64_t r = r0 + i;
      // the row's copies [lo, lo + m) of the list; j of the batch at b0 is on lane at0 + j
      const int lo = __shfl_sync(0xffffffffu, start, i), hi = __shfl_sync(0xffffffffu, start, i + 1);
      const int m = lo >= 0 && hi >= lo && hi <= most ? hi - lo : 0;
      const int at0 = together ? lo - begin : 0;
      auto copy = [&](int j) { return __shfl_sync(0xffffffffu, held, at0 + j); };
      if (!BWD && copy(0) < 0) continue;
      bool ready = together;
      for (int i0 = 0; i0 < turned; i0 += 32 * U) {
        uint64_t acc[U][H][2];  // two pairs' first and second dims
        int at[U];              // chunk of the item in its token's row of q or k
        int entry[U];           // item of its head's row
        bool live[U], is_q[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int i = i0 + 32 * u + lane, h = div_by(i, a.turned, a.turned_magic);
          live[u] = i < turned;
          is_q[u] = h < a.hq;
          entry[u] = i - h * a.turned;
          at[u] = (is_q[u] ? h : h - a.hq) * a.chunks + entry[u];
#pragma unroll
          for (int k = 0; k < H; ++k) acc[u][k][0] = acc[u][k][1] = 0ull;
        }
        for (int b0 = 0; b0 < m; b0 += B) {
          const int cnt = m - b0 < B ? m - b0 : B;
          if (!ready || m > B) {
            hold(a.map + lo + b0, cnt);
            angles(cnt, 0);
            ready = true;
          }
          for (int j = 0; j < cnt; ++j) {
            const int n = copy(j);
            if (n < 0) continue;
            const int4* qs = a.q_in + (int64_t)n * q_row;
            const int4* ks = a.k_in + (int64_t)n * kv_row;
            int4 x[U][IC];
#pragma unroll
            for (int u = 0; u < U; ++u)
              if (live[u]) {
                const int4* src = (is_q[u] ? qs : ks) + at[u];
#pragma unroll
                for (int e = 0; e < IC; ++e) x[u][e] = ld_stream(src + e * a.turned);
              }
            const float4* t0 = tab + rope_copy_at<NP>(0, 0, at0 + j);
#pragma unroll
            for (int u = 0; u < U; ++u)
              if (live[u]) {
#pragma unroll
                for (int k = 0; k < H; ++k) {
                  const float4 cs = t0[rope_entry(k, a.turned, entry[u])];
                  const uint64_t c = dev::f2pack(cs.x, cs.y), s = dev::f2pack(cs.z, cs.w);
                  const uint64_t ns = s ^ 0x8000000080000000ull;
                  uint64_t f, g;  // first and second dims of two pairs
                  if constexpr (INTER) {
                    const int w0 = word(x[u][0], 2 * k), w1 = word(x[u][0], 2 * k + 1);
                    f = dev::f2pack(lo_f(w0), lo_f(w1));
                    g = dev::f2pack(hi_f(w0), hi_f(w1));
                  } else {
                    const int w0 = word(x[u][0], k), w1 = word(x[u][IC - 1], k);
                    f = dev::f2pack(lo_f(w0), hi_f(w0));
                    g = dev::f2pack(lo_f(w1), hi_f(w1));
                  }
                  acc[u][k][0] = dev::ffma2(g, ns, BWD ? dev::ffma2(f, c, acc[u][k][0]) : dev::fmul2(f, c));
                  acc[u][k][1] = dev::ffma2(f, s, BWD ? dev::ffma2(g, c, acc[u][k][1]) : dev::fmul2(g, c));
                }
              }
          }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (live[u]) {
            int4* dst = (is_q[u] ? a.q_out + r * q_row : a.k_out + r * kv_row) + at[u];
            int4 y[IC];
#pragma unroll
            for (int k = 0; k < H; ++k) {
              if constexpr (INTER) {
                float f0, f1, g0, g1;
                dev::f2unpack(acc[u][k][0], f0, f1);
                dev::f2unpack(acc[u][k][1], g0, g1);
                word(y[0], 2 * k) = (int)dev::pack_bf16(f0, g0);
                word(y[0], 2 * k + 1) = (int)dev::pack_bf16(f1, g1);
              } else {
                word(y[0], k) = pack2(acc[u][k][0]);
                word(y[IC - 1], k) = pack2(acc[u][k][1]);
              }
            }
#pragma unroll
            for (int e = 0; e < IC; ++e) st_stream(dst + e * a.turned, y[e]);
          }
      }
      // chunks that are not rotated: the ends of the rows of q and k, and v
      const int rest = plain + kv_row;
      for (int i0 = 0; i0 < rest; i0 += 64) {
        const int4* src[2];
        int4* dst[2];
        int stride[2];
        bool live[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int i = i0 + 32 * u + lane;
          live[u] = i < rest;
          if (i < plain) {
            const int h = div_by(i, a.plain, a.plain_magic);
            const bool is_q = h < a.hq;
            const int c = (is_q ? h : h - a.hq) * a.chunks + IC * a.turned + i - h * a.plain;
            stride[u] = is_q ? q_row : kv_row;
            src[u] = (is_q ? a.q_in : a.k_in) + c;
            dst[u] = (is_q ? a.q_out : a.k_out) + c;
          } else {
            stride[u] = kv_row;
            src[u] = a.v_in + (i - plain);
            dst[u] = a.v_out + (i - plain);
          }
          dst[u] += r * stride[u];
        }
        if (!ready) {
          hold(a.map + lo, min(m, B));
          ready = true;
        }
        if (!BWD || m == 1) {  // a copy, bit for bit
          const int n = copy(0);
          int4 x[2];
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            x[u] = make_int4(0, 0, 0, 0);
            if (live[u] && n >= 0) x[u] = ld_stream(src[u] + (int64_t)n * stride[u]);
          }
#pragma unroll
          for (int u = 0; u < 2; ++u)
            if (live[u]) st_stream(dst[u], x[u]);
          continue;
        }
        uint64_t acc[2][4];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[u][e] = 0ull;
        for (int b0 = 0; b0 < m; b0 += B) {
          const int cnt = m - b0 < B ? m - b0 : B;
          if (m > B) hold(a.map + lo + b0, cnt);
          for (int j = 0; j < cnt; ++j) {
            const int n = copy(j);
            if (n < 0) continue;
            int4 x[2];
#pragma unroll
            for (int u = 0; u < 2; ++u)
              if (live[u]) x[u] = ld_stream(src[u] + (int64_t)n * stride[u]);
#pragma unroll
            for (int u = 0; u < 2; ++u)
              if (live[u])
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  acc[u][e] = dev::fadd2(acc[u][e], dev::f2pack(lo_f(word(x[u], e)), hi_f(word(x[u], e))));
          }
        }
#pragma unroll
        for (int u = 0; u < 2; ++u)
          if (live[u])
            st_stream(dst[u], make_int4(pack2(acc[u][0]), pack2(acc[u][1]), pack2(acc[u][2]), pack2(acc[u][3])));
      }
    }
  }
}

inline size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

int key_passes(int64_t traj_tokens) {  // 8-bit digits of the keys 0 .. traj_tokens
  int p = 1;
  while (p < 4 && (traj_tokens >> (8 * p)) != 0) ++p;
  return p;
}

template <int NP, bool INTER, bool BWD>
cudaError_t launch_rope_rows(RopeArgs a, cudaStream_t st) {
  // Rows of some 8 KB are a warp's each; of smaller ones it takes up to eight together, so that the latencies of
  // the map, the positions and the sines are met once for all, while enough warps for every SM remain.
  const int64_t chunks = (int64_t)(a.hq + 2 * a.hkv) * a.chunks;
  a.per = 1;
  while (a.per < kBatch && 2 * a.per * chunks <= 512 && a.rows_out >= 2 * a.per * 152 * 32) a.per *= 2;
  // Backward, a row takes as long as it has copies: a block for every few rows, which the SMs take as they get
  // free.  One long rollout at 40/8/128, step by step at 14/2/64 (up to 50 copies), us: 1,042 and 613; with blocks
  // that walk rows in a fixed stride, eight an SM, 1,324 and 925.
  int64_t blocks = (a.rows_out + kRopeWarps * a.per - 1) / (kRopeWarps * a.per);
  if (!BWD && blocks > 152 * 32) blocks = 152 * 32;
  static_assert(rope_table_bytes<NP>(kBatch) <= 48 * 1024, "a launch of more asks for it first");
  rope_rows<NP, INTER, BWD><<<(unsigned)blocks, kRopeThreads, rope_table_bytes<NP>(BWD ? kBatch : a.per), st>>>(a);
  return cudaGetLastError();
}

template <bool INTER, bool BWD>
cudaError_t launch_rope(const RopeArgs& a, int pairs, cudaStream_t st) {
  const int np = rope_lane_pairs(pairs);
  if (np == 1) return launch_rope_rows<1, INTER, BWD>(a, st);
  if (np == 2) return launch_rope_rows<2, INTER, BWD>(a, st);
  return launch_rope_rows<4, INTER, BWD>(a, st);
}

}  // namespace

cudaError_t launch_stream_positions(const int32_t* cu_seqlens, int32_t num_segments, int32_t num_tokens,
                                    const int32_t* src_step, const int32_t* step_img, const int32_t* step_txt,
                                    const int32_t* step_grid, int32_t num_steps, int32_t* pos, int32_t* status,
                                    cudaStream_t st) {
  if (num_segments == 0 || num_tokens == 0) return cudaSuccess;
  // A block per segment and chunk: all the chunks that one segment can have while that is a few blocks an
  // SM, else those of the average segment; a longer one's are taken in turn.
  const int64_t all = ((int64_t)num_tokens + kPosChunk - 1) / kPosChunk, few = 152 * 64 / num_segments;
  int64_t chunks = num_tokens / num_segments / kPosChunk + 1;
  if (chunks < few) chunks = few;
  if (chunks > all) chunks = all;
  if (chunks > 65535) chunks = 65535;
  dim3 grid((unsigned)num_segments, (unsigned)chunks);
  stream_positions_kernel<<<grid, kPosThreads, 0, st>>>(cu_seqlens, num_segments, num_tokens, src_step, step_img,
                                                        step_txt, step_grid, num_steps, pos, status);
  return cudaGetLastError();
}

// Groups that the workspace has room for.
int64_t group_limit(int64_t num_tokens) {
  return num_tokens / kGroupKeys > kMostGroups ? num_tokens / kGroupKeys : kMostGroups;
}

// A group's trajectory tokens as a power of two; T, the token of the keys that are out of range, is in the last one.
// -1: there are too many for groups.
int group_shift(int64_t num_tokens, int64_t T) {
  const int64_t want = num_tokens / kGroupKeys > kGroups ? num_tokens / kGroupKeys : kGroups;
  int shift = 0;
  while ((T >> shift) + 1 > want) ++shift;
  if (1ll << shift <= kCounters) return shift;
  for (shift = 0; 1 << shift < kCounters;) ++shift;
  return (T >> shift) + 1 <= group_limit(num_tokens) ? shift : -1;
}

// Chunks of heavy groups, each of which has more than kChunk runs.
int64_t chunk_limit(int64_t num_tokens) { return num_tokens / (kChunk / 2) + 1; }

struct SortGrid {
  int each, blocks;  // tiles a block
};
SortGrid sort_grid(int64_t num_tokens) {
  const int64_t tiles = (num_tokens + kTile - 1) / kTile, each = (tiles + kSortBlocks - 1) / kSortBlocks;
  return {(int)each, each == 0 ? 0 : (int)((tiles + each - 1) / each)};
}

// Workspace: digit counts of the blocks, their totals and the blocks' runs; the groups' counts, their sums and the
// heavy ones' list; the runs twice, but for one array (inv_tok).
size_t gather_inverse_ws_bytes(int64_t num_tokens) {
  const int64_t blocks = sort_grid(num_tokens).blocks, groups = group_limit(num_tokens);
  return align256((size_t)blocks * 256 * 4) + align256(257 * 4) + align256((size_t)blocks * 4) +
         align256((size_t)groups * 8 + 8) + align256((size_t)(groups / kGroupTile + 1) * 8) +
         2 * align256((size_t)chunk_limit(num_tokens) * 8) + 3 * align256((size_t)num_tokens * 4) + 256;
}

cudaError_t launch_gather_inverse(const int32_t* tok_gather, int64_t num_tokens, int64_t traj_tokens, int32_t* inv_off,
                                  int32_t* inv_tok, void* ws, int32_t* status, cudaStream_t st) {
  if (num_tokens == 0) {
    return cudaMemsetAsync(inv_off, 0, ((size_t)traj_tokens + 1) * 4, st);
  }
  const SortGrid grid = sort_grid(num_tokens);
  const uint32_t T = (uint32_t)traj_tokens;
  if (num_tokens <= kTile && traj_tokens <= kSmallOffsets) {
    inverse_small<<<1, kSortThreads, 0, st>>>(tok_gather, (int32_t)num_tokens, T, key_passes(traj_tokens), inv_off,
                                              inv_tok, status);
    return cudaGetLastError();
  }
  const int64_t limit = group_limit(num_tokens);
  const int shift = group_shift(num_tokens, traj_tokens);
  char* w = static_cast<char*>(ws);
  auto take = [&w](size_t bytes) {
    char* at = w;
    w += align256(bytes);
    return at;
  };
  auto* counts = reinterpret_cast<int32_t*>(take((size_t)grid.blocks * 256 * 4));
  auto* totals = reinterpret_cast<int32_t*>(take(257 * 4));
  int32_t* num_runs = totals + 256;
  auto* block_runs = reinterpret_cast<int32_t*>(take((size_t)grid.blocks * 4));
  auto* groups = reinterpret_cast<unsigned long long*>(take((size_t)limit * 8 + 8));  // behind heavy.num
  auto* group_sums = reinterpret_cast<unsigned long long*>(take((size_t)(limit / kGroupTile + 1) * 8));
  HeavyList heavy;
  heavy.num = reinterpret_cast<int32_t*>(groups++);
  heavy.group = reinterpret_cast<int2*>(take((size_t)chunk_limit(num_tokens) * 8));
  heavy.chunk = reinterpret_cast<int2*>(take((size_t)chunk_limit(num_tokens) * 8));
  const size_t nb = (size_t)num_tokens * 4;
  uint32_t* key[2] = {reinterpret_cast<uint32_t*>(take(nb)), reinterpret_cast<uint32_t*>(take(nb))};
  auto* spare = reinterpret_cast<int32_t*>(take(nb));
  const bool runs = shift >= 0;
  const int num_groups = runs ? (int)((traj_tokens >> shift) + 1) : 0;
  const int passes = key_passes(runs ? num_groups - 1 : traj_tokens), last = passes & 1;
  // sorted keys' places are inv_tok; runs that are sorted last must not be where inverse_place writes
  int32_t* at[2];
  at[last] = runs ? spare : inv_tok;
  at[last ^ 1] = runs ? inv_tok : spare;
  heavy.counts = reinterpret_cast<int32_t*>(key[last ^ 1]);
  if (runs) {
    const cudaError_t err = cudaMemsetAsync(heavy.num, 0, (size_t)num_groups * 8 + 8, st);
    if (err != cudaSuccess) return err;
    inverse_runs<<<grid.blocks, kSortThreads, 0, st>>>(tok_gather, num_tokens, T, shift, grid.each, key[0], at[0],
                                                       block_runs, counts, groups, status);
  } else {
    inverse_keys<<<(unsigned)((num_tokens + kSortThreads - 1) / kSortThreads), kSortThreads, 0, st>>>(
        tok_gather, num_tokens, T, key[0], at[0], num_runs, status);
  }
  for (int p = 0; p < passes; ++p) {
    const bool first = runs && p == 0;  // inverse_runs has counted
    const int digit = 8 * p + (runs ? kRunBits : 0), in = p & 1;
    if (!first) inverse_count<<<grid.blocks, kSortThreads, 0, st>>>(key[in], num_runs, digit, counts);
    inverse_scan<<<256 + (first ? (num_groups + kGroupTile - 1) / kGroupTile : 0), 1024, 0, st>>>(
        counts, grid.blocks, first ? nullptr : num_runs, totals, groups, num_groups, group_sums, heavy);
    inverse_scatter<<<grid.blocks, kSortThreads, 0, st>>>(key[in], at[in], digit, grid.each, counts, totals,
                                                          first ? block_runs : nullptr, num_runs, key[in ^ 1],
                                                          at[in ^ 1]);
  }
  if (!runs) {
    inverse_offsets<<<(unsigned)((traj_tokens + kOffTile) / kOffTile), 256, 0, st>>>(key[last], (int32_t)num_tokens,
                                                                                    traj_tokens, inv_off);
    return cudaGetLastError();
  }
  const bool split = num_tokens > kChunk;  // a group may be heavy
  inverse_place<<<(num_groups + kSortWarps - 1) / kSortWarps + (split ? kHeavyBlocks : 0), kSortThreads, 0, st>>>(
      tok_gather, T, shift, key[last], at[last], groups, num_groups, group_sums, heavy, inv_off, inv_tok);
  if (split) {
    inverse_heavy_scan<<<kHeavyBlocks, kCounters, 0, st>>>(T, shift, key[last], at[last], groups, num_groups,
                                                           group_sums, heavy, inv_off);
    inverse_heavy_place<<<kHeavyBlocks * 4, kSortThreads, 0, st>>>(tok_gather, T, shift, key[last], at[last], groups,
                                                                   num_groups, group_sums, heavy, inv_tok);
  }
  return cudaGetLastError();
}

cudaError_t launch_gather_rope(const void* q_in, const void* k_in, const void* v_in, int64_t rows_in, int64_t rows_out,
                               const int32_t* pos, int64_t pos_stride, const int32_t* map, const int32_t* off,
                               bool backward, int32_t hq, int32_t hkv, int32_t d, const vcs_rope& rope, void* q_out,
                               void* k_out, void* v_out, int32_t* status, cudaStream_t st) {
  if (rows_out == 0) return cudaSuccess;
  RopeArgs a;
  a.q_in = static_cast<const int4*>(q_in);
  a.k_in = static_cast<const int4*>(k_in);
  a.v_in = static_cast<const int4*>(v_in);
  a.q_out = static_cast<int4*>(q_out);
  a.k_out = static_cast<int4*>(k_out);
  a.v_out = static_cast<int4*>(v_out);
  a.rows_in = rows_in;
  a.rows_out = rows_out;
  a.pos = pos;
  a.pos_stride = pos_stride;
  a.map = map;
  a.off = off;
  a.hq = hq;
  a.hkv = hkv;
  a.chunks = d / 8;
  a.turned = rope.interleaved ? rope.rot_dim / 8 : rope.rot_dim / 16;
  a.plain = (d - rope.rot_dim) / 8;
  auto magic = [](int32_t c) { return c > 1 ? (uint32_t)((1ull << 32) / (uint32_t)c + 1) : 0u; };
  a.turned_magic = magic(a.turned);
  a.plain_magic = magic(a.plain);
  a.status = status;
  const int pairs = rope.rot_dim / 2;
  for (int i = 0; i < kMaxPairs; ++i) {
    a.turn[i] = 0;
    a.axis[i] = 0;
    if (i >= pairs) continue;
    // of the size, whose fraction is exact: that of a small negative number would be rounded next to 1
    const double turns = std::fabs(rope.inv_freq[i]) * 0.15915494309189533577;
    const uint64_t turn = (uint64_t)((turns - std::floor(turns)) * 18446744073709551616.0);
    a.turn[i] = rope.inv_freq[i] < 0.0 ? 0 - turn : turn;
    a.axis[i] = (uint8_t)rope.pair_axis[i];
  }
  if (backward)
    return rope.interleaved ? launch_rope<true, true>(a, pairs, st) : launch_rope<false, true>(a, pairs, st);
  return rope.interleaved ? launch_rope<true, false>(a, pairs, st) : launch_rope<false, false>(a, pairs, st);
}

}  // namespace vcs
