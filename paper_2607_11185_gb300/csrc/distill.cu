// distill.cu - divergence of rows of logits from a teacher's top entries, and its gradient, sm_103a.
//
// Row r with logits z, temperature T and weight w; its list of entries (id_j, t_j):
//   p_j = softmax_j(t_j / T),  log q_v = z_v / T - L,  L = ln sum_v exp(z_v / T)
//   kl = sum_j p_j (ln p_j - log q_{id_j}),  loss = sum_r w kl,  dz_v = w / T (q_v - sum_{j: id_j = v} p_j)
#include <algorithm>
#include <cfloat>
#include <cstdint>

#include "cluster_counts.h"
#include "internal.h"
#include "sm100.cuh"

namespace vcs {
namespace {

using namespace dev;
using bf16 = __nv_bfloat16;

constexpr int kMaxTop = VCS_DISTILL_MAX_TOP;
constexpr int kBytes = 16;   // of a vector
constexpr int64_t kShort = 16384;       // bytes of a row for small blocks
constexpr int64_t kShare = 65536;       // of a CTA's share of a row, so that three run on an SM
constexpr int64_t kMostShare = 212992;  // and the largest

struct Args {
  const void* z;
  int64_t rows, vocab, ld;
  const int32_t* ids;
  const float* t;
  int32_t top;
  int64_t lists;
  const int32_t* map;
  const float* weights;
  float inv_t, k;     // 1 / T, log2(e) / T
  float* loss;
  float* row_kl;
  void* dz;
  int64_t ldg;
  double* terms;      // [rows] w kl
  int32_t* status;
  uint32_t* done;     // blocks that have written their rows' terms
};

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(bf16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(bf16* p, float x) { *p = __float2bfloat16(x); }

// A vector's elements as fp32, and back.
template <class T>
struct Vec {
  static constexpr int N = kBytes / (int)sizeof(T);
  static __device__ __forceinline__ void open(const uint4& v, float (&x)[N]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (N == 8) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      } else {
        x[i] = __uint_as_float(w[i]);
      }
    }
  }
  static __device__ __forceinline__ uint4 close(const float (&x)[N]) {
    if constexpr (N == 8)
      return make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
    else
      return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
};

// exp((x - m) / T) of pairs; k = log2(e) / T.  The difference comes first: it is exact where it matters, near the maximum.
__device__ __forceinline__ void exp_pair(float x0, float x1, uint64_t minus_m, uint64_t k, float& e0, float& e1) {
  float a, b;
  f2unpack(fmul2(fadd2(f2pack(x0, x1), minus_m), k), a, b);
  e0 = ex2(a);
  e1 = ex2(b);
}

// ln x to 2^-24 absolute: the exponent's part in fp64, the fraction's, at most ln 2 / 2, in fp32.  (fp64 is slow here: its
// own logarithm took a lane 5 us.)
__device__ __forceinline__ double ln(float x) {
  const int e = ((__float_as_int(x) - 0x3f3504f3) >> 23);       // x / 2^e from sqrt(1/2) to sqrt(2)
  if (!(x > 0.f) || x > FLT_MAX || x < FLT_MIN) return (double)logf(x);
  return e * 0.69314718055994531 + (double)logf(__int_as_float(__float_as_int(x) - (e << 23)));
}

// Largest logit and sum of exponentials, taken together in one pass.  Before the first finite logit the exponentials are
// taken from 0: nothing but -inf sums to 0.  A vector's exponentials are added up by themselves and then to the sum; LONG:
// with what that addition rounds off kept beside it (Knuth's two-sum), as a row of a million equal logits would be rounded
// the same way a thousand times.  (A share in shared memory is 52 vectors a thread at most: there it would cost 3%.)
template <bool LONG>
struct Sum {
  float m = -INFINITY, s = 0.f, rest = 0.f;
  uint64_t neg = 0ull;   // -m, twice
  __device__ __forceinline__ void join(float m2, float s2, float k) {
    const float top = fmaxf(m, m2), base = top == -INFINITY ? 0.f : top;
    s = s * ex2((m - base) * k) + s2 * ex2((m2 - base) * k);
    m = top;
  }
  template <int N>
  __device__ __forceinline__ void add(const float (&x)[N], float k, uint64_t kk) {
    float top = fmaxf(x[0], x[1]);
#pragma unroll
    for (int i = 2; i < N; i += 2) top = fmax3(top, x[i], x[i + 1]);
    if (top > m) {   // rarely, after the first elements
      const float f = ex2((m - top) * k);
      s *= f;
      if (LONG) rest *= f;
      m = top;
      neg = f2pack(-m, -m);
    }
    float a, b;
    exp_pair(x[0], x[1], neg, kk, a, b);
    uint64_t acc = f2pack(a, b);
#pragma unroll
    for (int i = 2; i < N; i += 2) {
      exp_pair(x[i], x[i + 1], neg, kk, a, b);
      acc = fadd2(acc, f2pack(a, b));
    }
    f2unpack(acc, a, b);
    const float v = a + b, sum = s + v, back = sum - s;
    if (LONG) rest += (s - (sum - back)) + (v - back);
    s = sum;
  }
  __device__ __forceinline__ void close() {
    if (LONG) s += rest;
  }
};

// Maximum and sum of the warps' pairs, in order.
template <int W>
__device__ __forceinline__ void join_warps(const float* m, const float* s, float k, float& top, float& sum) {
  top = m[0];
#pragma unroll
  for (int i = 1; i < W; ++i) top = fmaxf(top, m[i]);
  const float base = top == -INFINITY ? 0.f : top;
  sum = 0.f;
#pragma unroll
  for (int i = 0; i < W; ++i) sum += s[i] * ex2((m[i] - base) * k);
}

// Zeros at dst .. dst + n.
template <class T, int THREADS>
__device__ __forceinline__ void clear(T* dst, int64_t n) {
  constexpr int N = Vec<T>::N;
  const int64_t lead = min(n, (int64_t)((kBytes - (reinterpret_cast<uintptr_t>(dst) & (kBytes - 1))) / sizeof(T)) % N);
  const int64_t m = (n - lead) / N;
  for (int64_t v = threadIdx.x; v < m; v += THREADS) reinterpret_cast<uint4*>(dst + lead)[v] = make_uint4(0u, 0u, 0u, 0u);
  if (threadIdx.x < lead) put(dst + threadIdx.x, 0.f);
  for (int64_t e = lead + m * N + threadIdx.x; e < n; e += THREADS) put(dst + e, 0.f);
}

// The words `off` bytes on from one vector to the next.
__device__ __forceinline__ uint4 join_vectors(const uint4& lo, const uint4& hi, uint32_t off) {
  const uint32_t words[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
  uint32_t o[4];
#pragma unroll
  for (int q = 0; q < 4; ++q)
    if (off >> 2 == q)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = __funnelshift_r(words[q + i], words[(q + i + 1) & 7], (off & 3) * 8);
  return make_uint4(o[0], o[1], o[2], o[3]);
}

// c q of a vector of logits.
template <class T>
__device__ __forceinline__ uint4 gradient(const uint4& x, uint64_t neg, uint64_t kk, uint64_t gg) {
  constexpr int N = Vec<T>::N;
  float f[N];
  Vec<T>::open(x, f);
#pragma unroll
  for (int i = 0; i < N; i += 2) {
    float e0, e1;
    exp_pair(f[i], f[i + 1], neg, kk, e0, e1);
    f2unpack(fmul2(f2pack(e0, e1), gg), f[i], f[i + 1]);
  }
  return Vec<T>::close(f);
}

// A list's entries, `E` to a thread (j = threadIdx.x + i THREADS), and what is made of them.
template <int THREADS, int E>
struct Entries {
  int id[E];
  float t[E], p[E], keep[E];
  __device__ __forceinline__ void load(const Args& a, int64_t list) {   // under way while the row is read
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int j = threadIdx.x + i * THREADS;
      id[i] = -1;
      t[i] = -INFINITY;
      if (j < a.top && list >= 0) {
        id[i] = __ldg(&a.ids[list * a.top + j]);
        t[i] = __ldg(&a.t[list * a.top + j]);
      }
    }
  }
  // Checks the ids, takes the entries' logits (before any is overwritten: dz may be z); the largest t, where a NaN counts as
  // infinite, so that it goes through (fmaxf drops it, the sums do not).
  template <class Logit>
  __device__ __forceinline__ float check(const Args& a, int32_t* ids, Logit logit) {
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int j = threadIdx.x + i * THREADS;
      if (id[i] < -1 || id[i] >= a.vocab) {
        set_status(a.status, VCS_ERR_DEVICE_CHECK);
        id[i] = -1;
      }
      keep[i] = 0.f;
      if (id[i] >= 0) keep[i] = logit(id[i]);
      else t[i] = -INFINITY;
      top = fmaxf(top, t[i] != t[i] ? INFINITY : t[i]);
      if (j < ((a.top + 3) & ~3)) ids[j] = id[i];
    }
    return top;
  }
  __device__ __forceinline__ float weigh(const Args& a, float tmax) {   // the thread's sum of unnormalised p
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      t[i] = t[i] == -INFINITY ? t[i] : t[i] - tmax;   // (+inf - +inf is a NaN)
      p[i] = t[i] == -INFINITY ? 0.f : expf(t[i] * a.inv_t);
      sum += p[i];
    }
    return sum;
  }
  __device__ __forceinline__ void normalise(const Args& a, float psum, float* ps) {
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int j = threadIdx.x + i * THREADS;
      p[i] = t[i] == -INFINITY ? 0.f : p[i] / psum;
      if (j < a.top) ps[j] = p[i];
    }
  }
  // Of entry i: 0 if it is none or its id came before, 1 if it comes once, 2 if it comes again.
  __device__ __forceinline__ int place(const Args& a, const int32_t* ids, int i) const {
    if (id[i] < 0) return 0;
    int count = 0;
    for (int m = 0; m < a.top; m += 4) {   // (ids are written up to a multiple of 4)
      const int4 x = *reinterpret_cast<const int4*>(ids + m);
      count += (x.x == id[i]) + (x.y == id[i]) + (x.z == id[i]) + (x.w == id[i]);
    }
    if (count == 1) return 1;
    const int j = threadIdx.x + i * THREADS;
    for (int m = 0; m < j; ++m)
      if (ids[m] == id[i]) return 0;
    return 2;
  }
  __device__ __forceinline__ float mass(const Args& a, const int32_t* ids, const float* ps, int i, int place) const {
    if (place == 1) return p[i];
    float sum = 0.f;
    for (int m = 0; m < a.top; ++m)
      if (ids[m] == id[i]) sum += ps[m];
    return sum;
  }
  // The thread's terms of the divergence, of entries that are `mine`: ln p - log q is the difference of the two differences
  // from the maxima and of the two logarithms.
  template <class Mine>
  __device__ __forceinline__ float divergence(const Args& a, float zmax, float logs, Mine mine) const {
    float kl = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (p[i] != 0.f && mine(id[i])) kl = fmaf(p[i], fmaf(t[i] - (keep[i] - zmax), a.inv_t, logs), kl);
    return kl;
  }
};

template <int THREADS, class T>
__device__ __forceinline__ T block_sum(T x, T* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = x;
  __syncthreads();
  x = red[0];
#pragma unroll
  for (int i = 1; i < THREADS / 32; ++i) x += red[i];
  return x;
}

// A block a row at a time.  Without a gradient one pass over its logits; with it a second, for short rows, which are in
// L1 or L2 by then, and for those that do not fit the shared memory of a cluster.
template <class T, int THREADS, int E>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) distill_rows(const __grid_constant__ Args a) {
  constexpr int N = Vec<T>::N, U = 4, W = THREADS / 32;   // U: vectors a thread has under way
  __shared__ __align__(16) int32_t ids[kMaxTop];
  __shared__ __align__(16) float ps[kMaxTop];
  __shared__ double red64[W];
  __shared__ float red_m[W], red_s[W], red_t[W], red_p[W], red_k[W];
  __shared__ bool last;
  const float k = a.k;
  const uint64_t kk = f2pack(k, k);
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, warps = min(W, (a.top + 31) / 32);   // with entries
  float w_next = a.weights[blockIdx.x];
  int list_next = a.map == nullptr ? (int)blockIdx.x : a.map[blockIdx.x];
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T* z = static_cast<const T*>(a.z) + r * a.ld;
    T* dz = a.dz == nullptr ? nullptr : static_cast<T*>(a.dz) + r * a.ldg;
    const float w = w_next;
    int64_t list = list_next;
    if (r + gridDim.x < a.rows) {
      w_next = __ldg(&a.weights[r + gridDim.x]);
      list_next = a.map == nullptr ? (int)(r + gridDim.x) : __ldg(&a.map[r + gridDim.x]);
    }
    if (w == 0.f) {   // not read
      if (threadIdx.x == 0) a.row_kl[r] = 0.f, a.terms[r] = 0.0;
      if (dz != nullptr) clear<T, THREADS>(dz, a.vocab);
      continue;
    }
    if (list < 0 || list >= a.lists) {
      if (threadIdx.x == 0) set_status(a.status, VCS_ERR_DEVICE_CHECK);
      list = -1;
    }
    Entries<THREADS, E> en;
    en.load(a, list);
    // ---- statistics of the row
    Sum<true> sum;
    {
      const int64_t head = min(a.vocab, (int64_t)((kBytes - (reinterpret_cast<uintptr_t>(z) & (kBytes - 1))) / sizeof(T)) % N);
      const int64_t vecs = (a.vocab - head) / N;
      const uint4* zv = reinterpret_cast<const uint4*>(z + head);   // (plain loads: the gradient may go over them)
      int64_t v = threadIdx.x;
      for (; v + (U - 1) * THREADS < vecs; v += U * THREADS) {
        uint4 x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = zv[v + u * THREADS];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          float f[N];
          Vec<T>::open(x[u], f);
          sum.add<N>(f, k, kk);
        }
      }
      for (; v < vecs; v += THREADS) {
        float f[N];
        Vec<T>::open(zv[v], f);
        sum.add<N>(f, k, kk);
      }
      const int64_t rest = a.vocab - head - vecs * N;   // with the head, fewer than two vectors
      if (threadIdx.x < head + rest) {
        const float x = to_float(z[threadIdx.x < head ? threadIdx.x : vecs * N + threadIdx.x]);
        const float f[2] = {x, -INFINITY};
        sum.add<2>(f, k, kk);
      }
    }
    sum.close();
    float tmax = en.check(a, ids, [&](int v) { return to_float(z[v]); });
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      sum.join(__shfl_xor_sync(0xffffffffu, sum.m, o), __shfl_xor_sync(0xffffffffu, sum.s, o), k);
      tmax = fmaxf(tmax, __shfl_xor_sync(0xffffffffu, tmax, o));
    }
    if (lane == 0) {
      red_m[wid] = sum.m;
      red_s[wid] = sum.s;
      red_t[wid] = tmax;
    }
    __syncthreads();
    tmax = red_t[0];
#pragma unroll
    for (int i = 1; i < W; ++i) tmax = fmaxf(tmax, red_t[i]);
    join_warps<W>(red_m, red_s, k, sum.m, sum.s);
    const bool empty = tmax == -INFINITY;                    // nothing to learn from
    const float zmax = sum.m == -INFINITY ? NAN : sum.m;     // nothing but -inf: no distribution
    float mine = en.weigh(a, tmax);
    if (wid < warps) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
      if (lane == 0) red_p[wid] = mine;
    }
    __syncthreads();
    float psum = 0.f;
    for (int i = 0; i < warps; ++i) psum += red_p[i];
    en.normalise(a, psum, ps);
    if (wid < warps) {
      float kl = en.divergence(a, zmax, (float)(ln(sum.s) - ln(psum)), [](int) { return true; });
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) kl += __shfl_xor_sync(0xffffffffu, kl, o);
      if (lane == 0) red_k[wid] = kl;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      float kl = 0.f;
      for (int i = 0; i < warps; ++i) kl += red_k[i];
      a.row_kl[r] = empty ? 0.f : kl;
      a.terms[r] = empty ? 0.0 : (double)w * kl;
    }
    if (dz == nullptr) continue;
    if (empty) {
      clear<T, THREADS>(dz, a.vocab);
      continue;
    }
    // ---- gradient
    const float c = w * a.inv_t, inv = 1.f / sum.s, g = c * inv;
    const uint64_t neg = f2pack(-zmax, -zmax), gg = f2pack(g, g);
    // bytes from a vector of the gradient's back to one of the logits': 0 where the rows are aligned alike
    const uint32_t shift = (uint32_t)((reinterpret_cast<uintptr_t>(z) - reinterpret_cast<uintptr_t>(dz)) & (kBytes - 1));
    int64_t head = min(a.vocab, (int64_t)((kBytes - (reinterpret_cast<uintptr_t>(dz) & (kBytes - 1))) / sizeof(T)) % N);
    int64_t vecs = (a.vocab - head) / N;
    if (shift != 0) {   // vectors whose two of the logits lie in the row
      while (vecs > 0 && head * (int64_t)sizeof(T) < (int64_t)shift) head += N, --vecs;
      while (vecs > 0 && (head + vecs * N) * (int64_t)sizeof(T) - shift + kBytes > a.vocab * (int64_t)sizeof(T)) --vecs;
    }
    const uint4* zv = reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(z + head) - shift);
    uint4* gv = reinterpret_cast<uint4*>(dz + head);
    auto fetch = [&](int64_t v) {   // (plain loads: in place the gradient follows)
      const uint4 lo = zv[v];
      return shift == 0 ? lo : join_vectors(lo, zv[v + 1], shift);
    };
    int64_t v = threadIdx.x;
    for (; v + (U - 1) * THREADS < vecs; v += U * THREADS) {
      uint4 x[U];
#pragma unroll
      for (int u = 0; u < U; ++u) x[u] = fetch(v + u * THREADS);
#pragma unroll
      for (int u = 0; u < U; ++u) __stcs(gv + v + u * THREADS, gradient<T>(x[u], neg, kk, gg));
    }
    for (; v < vecs; v += THREADS) __stcs(gv + v, gradient<T>(fetch(v), neg, kk, gg));
    const int64_t rest = a.vocab - head - vecs * N;
    for (int64_t i = threadIdx.x; i < head + rest; i += THREADS) {
      const int64_t e = i < head ? i : vecs * N + i;
      put(dz + e, ex2((to_float(z[e]) - zmax) * k) * g);
    }
    __syncthreads();
    // the entries again, less their p: one that comes twice by its first place, with the sum of both
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int place = en.place(a, ids, i);
      if (place > 0)
        put(dz + en.id[i], c * (ex2((en.keep[i] - zmax) * k) * inv - en.mass(a, ids, ps, i, place)));
    }
    __syncthreads();   // the lists are read
  }
  // the block that finishes last adds the rows' terms in an order of its threads, so that the loss does not depend on scheduling
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    last = atomicAdd(a.done, 1u) == gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
  __threadfence();
  double x = 0.0;
  for (int64_t r = threadIdx.x; r < a.rows; r += THREADS) x += __ldcg(&a.terms[r]);
  x = block_sum<THREADS>(x, red64);
  if (threadIdx.x == 0) *a.loss = (float)x;
}

// ------------------------------------------------------------------ rows held in shared memory
// A cluster of `size` CTAs a row, each with its share of the row in shared memory: every logit is read once.  A share is
// at most 64 KB where it can be, so that three CTAs run on an SM and one's loads, all under way at once, go with another's
// stores.
constexpr int kHeldThreads = 256;
constexpr int kParts = 4;    // of a share, each with a barrier of its own

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// {x, y} at `dst` of a CTA of the cluster, whose barrier counts the 8 bytes (addresses as in this CTA).
__device__ __forceinline__ void send(float* dst, uint64_t* bar, uint32_t rank, float x, float y) {
  uint32_t at, on;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(dst)), "r"(rank));
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(on) : "r"(smem_u32(bar)), "r"(rank));
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];" ::"r"(at), "f"(x),
               "f"(y), "r"(on)
               : "memory");
}
// mbar_wait for what other CTAs of the cluster have sent.
__device__ __forceinline__ bool mbar_wait_cluster(uint64_t* bar, uint32_t parity) {
  const long long t0 = clock64();
  while (true) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
    if (ok != 0) return true;
    if (clock64() - t0 > kWaitLimitCycles) return false;
  }
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
               "l"(src), "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}

template <class T, int E>
__global__ void __launch_bounds__(kHeldThreads, 3) distill_held(const __grid_constant__ Args a, int log_size) {
  constexpr int N = Vec<T>::N, THREADS = kHeldThreads, W = THREADS / 32, U = 4;
  extern __shared__ __align__(128) uint8_t held[];
  __shared__ __align__(16) int32_t ids[kMaxTop];
  __shared__ __align__(16) float ps[kMaxTop];
  __shared__ double red64[W];
  __shared__ float red_m[W], red_s[W], red_t[W], red_p[W], red_k[W];
  __shared__ __align__(16) float peer[2][8][2];   // the CTAs' maxima and sums, by turns
  __shared__ __align__(16) float terms[2][8][W][2];  // the first CTA's: the others' terms of the divergence, a warp's each
  __shared__ uint64_t full[kParts], met[2], added[2];
  __shared__ bool last;
  const float k = a.k;
  const uint64_t kk = f2pack(k, k);
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, warps = min(W, (a.top + 31) / 32);
  const int size = 1 << log_size, rank = (int)cluster_rank(), clusters = (int)gridDim.x >> log_size;
  const uint32_t base_s = smem_u32(held);
  if (threadIdx.x == 0) {
    for (int i = 0; i < kParts; ++i) mbar_init(&full[i], 1);
    for (int i = 0; i < 2; ++i) mbar_init(&met[i], 1), mbar_init(&added[i], 1);
    fence_mbar_init();
  }
  __syncthreads();
  if (size > 1) {   // the others' barriers are there
    cluster_arrive();
    cluster_wait();
  }
  // A row's vectors, from its first 16-byte boundary on, and this CTA's share of them.
  struct Row {
    const T* z;
    int head, vecs, v0, n;
    __device__ __forceinline__ Row(const Args& a, int64_t r, int rank, int log_size) {
      z = static_cast<const T*>(a.z) + r * a.ld;
      head = (int)min(a.vocab, (int64_t)((kBytes - (reinterpret_cast<uintptr_t>(z) & (kBytes - 1))) / sizeof(T)) % N);
      vecs = (int)((a.vocab - head) / N);
      v0 = (int)((int64_t)vecs * rank >> log_size);
      n = (int)((int64_t)vecs * (rank + 1) >> log_size) - v0;
    }
    __device__ __forceinline__ int part(int i) const { return n * i / kParts; }
  };
  // Sets the next row with a weight on its way, from row r of weight w on, as soon as the one before has been read.
  auto fetch = [&](int64_t r, float w) {
    if (threadIdx.x != 0) return;
    while (r < a.rows && w == 0.f) {
      r += clusters;
      if (r < a.rows) w = __ldg(&a.weights[r]);
    }
    if (r >= a.rows) return;
    const Row row(a, r, rank, log_size);
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
      const uint32_t bytes = (uint32_t)(row.part(i + 1) - row.part(i)) * kBytes;
      mbar_arrive_expect_tx(&full[i], bytes);
      if (bytes > 0)
        bulk_load(base_s + row.part(i) * kBytes, reinterpret_cast<const uint4*>(row.z + row.head) + row.v0 + row.part(i),
                  bytes, &full[i]);
    }
  };
  int64_t r = blockIdx.x >> log_size;
  float w_next = r < a.rows ? a.weights[r] : 0.f;
  int list_next = r < a.rows && a.map != nullptr ? a.map[r] : (int)r;
  fetch(r, w_next);
  uint32_t turn = 0;
  bool ok = true, go = true;
  // A row whose divergence waits for the other CTAs' terms: they have sent them before their sums of the next row, so that
  // the first CTA takes them when it has met those.  (Waiting in the row itself: 4,096 rows of 131,072 bf16 388 us, so 381;
  // 1,024 of fp32 188 and 185.)
  int64_t open_row = -1;
  float open_kl = 0.f, open_w = 0.f;
  auto finish = [&](uint32_t t) {
    if (open_row < 0) return;
    ok = ok && mbar_wait_cluster(&added[t & 1], t >> 1 & 1);
    for (int c = 1; c < size; ++c)
      for (int i = 0; i < warps; ++i) open_kl += terms[t & 1][c][i][0];
    a.row_kl[open_row] = open_kl;
    a.terms[open_row] = (double)open_w * open_kl;
    open_row = -1;
  };
  for (; r < a.rows; r += clusters) {
    const Row row(a, r, rank, log_size);
    T* dz = static_cast<T*>(a.dz) + r * a.ldg;
    const float w = w_next;
    int64_t list = list_next;
    if (r + clusters < a.rows) {
      w_next = __ldg(&a.weights[r + clusters]);
      list_next = a.map == nullptr ? (int)(r + clusters) : __ldg(&a.map[r + clusters]);
    }
    const int64_t e0 = rank == 0 ? 0 : row.head + (int64_t)row.v0 * N;   // elements whose gradient this CTA clears
    const int64_t e1 = rank == size - 1 ? a.vocab : row.head + (int64_t)(row.v0 + row.n) * N;
    if (w == 0.f) {   // not read
      if (rank == 0 && threadIdx.x == 0) a.row_kl[r] = 0.f, a.terms[r] = 0.0;
      clear<T, THREADS>(dz + e0, e1 - e0);
      continue;
    }
    if (list < 0 || list >= a.lists) {
      if (rank == 0 && threadIdx.x == 0) set_status(a.status, VCS_ERR_DEVICE_CHECK);
      list = -1;
    }
    Entries<THREADS, E> en;
    en.load(a, list);
    // the few elements outside the vectors: the first CTA's, a thread each
    const int loose = rank == 0 ? (int)(a.vocab - (int64_t)row.vecs * N) : 0;
    const int64_t my_loose = (int)threadIdx.x < row.head ? (int64_t)threadIdx.x : (int64_t)row.vecs * N + threadIdx.x;
    const float x_loose = (int)threadIdx.x < loose ? to_float(row.z[my_loose]) : -INFINITY;
    // ---- statistics
    Sum<false> sum;
#pragma unroll 1
    for (int i = 0; i < kParts; ++i) {
      const int e = row.part(i + 1);
      ok = ok && mbar_wait(&full[i], turn & 1);
      int v = row.part(i) + threadIdx.x;
      for (; v + (U - 1) * THREADS < e; v += U * THREADS) {
        uint4 x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = ld_shared_v4(base_s + (v + u * THREADS) * kBytes);
#pragma unroll
        for (int u = 0; u < U; ++u) {
          float f[N];
          Vec<T>::open(x[u], f);
          sum.add<N>(f, k, kk);
        }
      }
      for (; v < e; v += THREADS) {
        float f[N];
        Vec<T>::open(ld_shared_v4(base_s + v * kBytes), f);
        sum.add<N>(f, k, kk);
      }
    }
    if ((int)threadIdx.x < loose) {
      const float f[2] = {x_loose, -INFINITY};
      sum.add<2>(f, k, kk);
    }
    // An entry's logit is taken, and its gradient written, by the CTA whose element it is: in place another CTA's loads would
    // have to be waited for.
    const int s0 = row.head + row.v0 * N, s1 = s0 + row.n * N, tail = row.head + row.vecs * N;   // (a row held is short)
    auto outside = [&](int v) { return rank == 0 && (v < s0 || v >= tail); };
    auto owned = [&](int v) { return (v >= s0 && v < s1) || outside(v); };
    float tmax = en.check(a, ids, [&](int v) {
      return outside(v) ? to_float(row.z[v]) : v >= s0 && v < s1 ? to_float(reinterpret_cast<const T*>(held)[v - s0]) : 0.f;
    });
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      sum.join(__shfl_xor_sync(0xffffffffu, sum.m, o), __shfl_xor_sync(0xffffffffu, sum.s, o), k);
      tmax = fmaxf(tmax, __shfl_xor_sync(0xffffffffu, tmax, o));
    }
    if (lane == 0) {
      red_m[wid] = sum.m;
      red_s[wid] = sum.s;
      red_t[wid] = tmax;
    }
    __syncthreads();
    tmax = red_t[0];
#pragma unroll
    for (int i = 1; i < W; ++i) tmax = fmaxf(tmax, red_t[i]);
    join_warps<W>(red_m, red_s, k, sum.m, sum.s);
    // Each CTA's maximum and sum to all of them: no store of a gradient is waited for, as a barrier of the cluster does.  By
    // turns: whoever writes a turn's words again has met all that read them.
    if (size > 1) {
      if (threadIdx.x == 0) mbar_arrive_expect_tx(&met[turn & 1], 8 * size);
      if ((int)threadIdx.x < size) send(peer[turn & 1][rank], &met[turn & 1], threadIdx.x, sum.m, sum.s);
    }
    float mine = en.weigh(a, tmax);
    if (wid < warps) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
      if (lane == 0) red_p[wid] = mine;
    }
    int place[E];   // while the others arrive
#pragma unroll
    for (int i = 0; i < E; ++i) place[i] = en.place(a, ids, i);
    if (size > 1) {
      ok = ok && mbar_wait_cluster(&met[turn & 1], turn >> 1 & 1);
      float m[8], s[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        m[i] = i < size ? peer[turn & 1][i][0] : -INFINITY;
        s[i] = i < size ? peer[turn & 1][i][1] : 0.f;
      }
      join_warps<8>(m, s, k, sum.m, sum.s);
    }
    // (The predicate takes the words, which so have been read when this CTA sends its next ones.)
    go = __syncthreads_and(ok && !(sum.s < 0.f));
    if (!go) break;
    if (rank == 0 && threadIdx.x == 0) finish(turn - 1);
    ++turn;
    const bool empty = tmax == -INFINITY;                    // nothing to learn from
    const float zmax = sum.m == -INFINITY ? NAN : sum.m;     // nothing but -inf: no distribution
    float psum = 0.f;
    for (int i = 0; i < warps; ++i) psum += red_p[i];
    en.normalise(a, psum, ps);
    const float c = w * a.inv_t, inv = 1.f / sum.s, g = c * inv;
    if (empty) {
      clear<T, THREADS>(dz + e0, e1 - e0);
    } else {
      // ---- gradient
      const uint64_t neg = f2pack(-zmax, -zmax), gg = f2pack(g, g);
      T* out = dz + row.head + (int64_t)row.v0 * N;   // of the held elements
      // elements of them before the gradient's first vector
      const int lead = min(row.n * N, (int)((kBytes - (reinterpret_cast<uintptr_t>(out) & (kBytes - 1))) / sizeof(T)) % N);
      uint4* gv = reinterpret_cast<uint4*>(out + lead);
      if (lead == 0) {
        int v = threadIdx.x;
        for (; v + (U - 1) * THREADS < row.n; v += U * THREADS) {
          uint4 x[U];
#pragma unroll
          for (int u = 0; u < U; ++u) x[u] = ld_shared_v4(base_s + (v + u * THREADS) * kBytes);
#pragma unroll
          for (int u = 0; u < U; ++u) __stcs(gv + v + u * THREADS, gradient<T>(x[u], neg, kk, gg));
        }
        for (; v < row.n; v += THREADS) __stcs(gv + v, gradient<T>(ld_shared_v4(base_s + v * kBytes), neg, kk, gg));
      } else {   // aligned otherwise than the logits: a vector's words from two of the held
        for (int v = threadIdx.x; v < row.n - 1; v += THREADS)
          __stcs(gv + v, gradient<T>(join_vectors(ld_shared_v4(base_s + v * kBytes), ld_shared_v4(base_s + (v + 1) * kBytes),
                                                  lead * (uint32_t)sizeof(T)),
                                     neg, kk, gg));
        if ((int)threadIdx.x < N) {   // `lead` elements in front, the others behind
          const int e = (int)threadIdx.x < lead ? (int)threadIdx.x : (row.n - 1) * N + (int)threadIdx.x;
          put(out + e, ex2((to_float(reinterpret_cast<const T*>(held)[e]) - zmax) * k) * g);
        }
      }
      if ((int)threadIdx.x < loose) put(dz + my_loose, ex2((x_loose - zmax) * k) * g);
    }
    __syncthreads();
    fetch(r + clusters, w_next);   // everybody is done with the share
    // the entries again, less their p, by the CTA whose elements they are: one that comes twice by its first place, with the
    // sum of both
#pragma unroll
    for (int i = 0; i < E; ++i) {
      if (place[i] == 0 || empty || !owned(en.id[i])) continue;
      put(dz + en.id[i], c * (ex2((en.keep[i] - zmax) * k) * inv - en.mass(a, ids, ps, i, place[i])));
    }
    // ---- the divergence: each CTA's terms to the first, which adds them up in order (turn is the next row's by now)
    if (wid < warps) {
      float kl = en.divergence(a, zmax, (float)(ln(sum.s) - ln(psum)), owned);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) kl += __shfl_xor_sync(0xffffffffu, kl, o);
      if (lane == 0 && rank == 0) red_k[wid] = kl;
      if (lane == 0 && rank > 0) send(terms[~turn & 1][rank][wid], &added[~turn & 1], 0, kl, 0.f);
    }
    if (rank == 0) {
      __syncthreads();
      if (threadIdx.x == 0) {
        float kl = 0.f;
        for (int i = 0; i < warps; ++i) kl += red_k[i];
        const float weight = empty ? 0.f : w;   // (without entries kl is 0)
        if (size == 1) {
          a.row_kl[r] = kl;
          a.terms[r] = (double)weight * kl;
        } else {
          mbar_arrive_expect_tx(&added[~turn & 1], 8 * (size - 1) * warps);
          open_row = r;
          open_kl = kl;
          open_w = weight;
        }
      }
    }
    __syncthreads();   // the lists are read
  }
  if (rank == 0 && threadIdx.x == 0 && go) finish(turn - 1);
  __syncwarp();
  if (!ok) set_status(a.status, VCS_ERR_DEVICE_TIMEOUT);
  if (!go && threadIdx.x == 0)   // a wait has run out: the row's loads, once more with a limit
    for (int i = 0; i < kParts; ++i) mbar_wait(&full[i], turn & 1);
  __syncwarp();
  if (size > 1) {   // what this CTA sent has arrived before the others end, and they have its words
    cluster_arrive();
    cluster_wait();
  }
  // the block that finishes last adds the rows' terms in an order of its threads, so that the loss does not depend on scheduling
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    last = atomicAdd(a.done, 1u) == gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
  __threadfence();
  double x = 0.0;
  for (int64_t i = threadIdx.x; i < a.rows; i += THREADS) x += __ldcg(&a.terms[i]);
  x = block_sum<THREADS>(x, red64);
  if (threadIdx.x == 0) *a.loss = (float)x;
}

template <class T, int E>
cudaError_t launch_held(const Args& a, int log_size, size_t share, cudaStream_t st) {
  cudaError_t e = cudaFuncSetAttribute(distill_held<T, E>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostShare);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(152u << log_size);
  cfg.blockDim = dim3(kHeldThreads);
  cfg.dynamicSmemBytes = share;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 1u << log_size;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  // As many clusters as run at a time: the SMs of a part of the chip are no multiple of a cluster, and two clusters that
  // started when the others were done took as long again.  The answer is kept: asking takes microseconds.
  static ClusterCounts known[4];
  int device = 0;
  if (e = cudaGetDevice(&device); e != cudaSuccess) return e;
  int n = known[log_size].find(device, (uint32_t)share);
  if (n == 0) {
    if (e = cudaOccupancyMaxActiveClusters(&n, distill_held<T, E>, &cfg); e != cudaSuccess) return e;
    if (n < 1) return cudaErrorInvalidConfiguration;
    known[log_size].keep(device, (uint32_t)share, n);
  }
  cfg.gridDim = dim3((unsigned)std::min<int64_t>(n, a.rows) << log_size);
  return cudaLaunchKernelEx(&cfg, distill_held<T, E>, a, log_size);
}

template <class T, int THREADS>
cudaError_t launch_block(const Args& a, cudaStream_t st) {
  const int64_t most = 152 * (1024 / THREADS);
  const unsigned grid = (unsigned)(a.rows < most ? a.rows : most);
  if (a.top <= THREADS) distill_rows<T, THREADS, 1><<<grid, THREADS, 0, st>>>(a);
  else distill_rows<T, THREADS, (kMaxTop + THREADS - 1) / THREADS><<<grid, THREADS, 0, st>>>(a);
  return cudaGetLastError();
}

template <class T>
cudaError_t launch_rows(const Args& a, cudaStream_t st) {
  const int64_t bytes = a.vocab * (int64_t)sizeof(T);
  // A short row leaves most of a large block without work, and its fixed time shows: small blocks, more of them.
  if (bytes <= kShort) return launch_block<T, 128>(a, st);
  if (a.dz != nullptr) {
    int l = 0;
    while (l < 3 && bytes > kShare << l) ++l;
    while (l < 3 && a.rows << (l + 1) <= 152 && bytes > 8192 << l) ++l;   // few rows: over the chip
    const int64_t share = ((bytes >> l) + 2 * kBytes) & ~(int64_t)(kBytes - 1);
    if (share <= kMostShare)
      return a.top <= kHeldThreads ? launch_held<T, 1>(a, l, (size_t)share, st)
                                   : launch_held<T, (kMaxTop + kHeldThreads - 1) / kHeldThreads>(a, l, (size_t)share, st);
  }
  // Between a row's last load and the next one's first lie its sums and its list.  With more rows than large blocks smaller
  // ones take turns at that (us, blocks of 128, 256 and 512 threads: 20,000 rows of 10,000 fp32 167, 194, 302; 4,096 of
  // 131,072 bf16 193, 188, 202; 512 of 99,991 fp32 65, 54, 57), with fewer a large one has more loads under way (304 of
  // these 58, 44, 38).
  if (a.dz == nullptr && a.rows > 2 * 152) return bytes <= kShare ? launch_block<T, 128>(a, st) : launch_block<T, 256>(a, st);
  return launch_block<T, 512>(a, st);
}

}  // namespace

size_t distill_ws_bytes(int64_t rows) { return kWsHeader + (size_t)rows * sizeof(double); }

cudaError_t launch_distill(const DistillArgs& d, void* ws, cudaStream_t st) {
  if (cudaError_t e = cudaMemsetAsync(ws, 0, kWsHeader, st); e != cudaSuccess) return e;
  if (d.rows == 0) return cudaMemsetAsync(d.loss, 0, sizeof(float), st);
  Args a;
  a.z = d.logits;
  a.rows = d.rows;
  a.vocab = d.vocab;
  a.ld = d.stride;
  a.ids = d.ids;
  a.t = d.teacher;
  a.top = d.top;
  a.lists = d.lists;
  a.map = d.map;
  a.weights = d.weights;
  a.inv_t = 1.f / d.temperature;
  a.k = (float)(1.4426950408889634 / (double)d.temperature);   // rounded once: it multiplies every argument
  a.loss = d.loss;
  a.row_kl = d.row_kl;
  a.dz = d.dlogits;
  a.ldg = d.grad_stride;
  a.status = static_cast<int32_t*>(ws);
  a.done = reinterpret_cast<uint32_t*>(ws) + 1;
  a.terms = reinterpret_cast<double*>(static_cast<char*>(ws) + kWsHeader);
  return d.f32 ? launch_rows<float>(a, st) : launch_rows<bf16>(a, st);
}

}  // namespace vcs
