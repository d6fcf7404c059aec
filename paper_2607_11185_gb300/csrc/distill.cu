// distill.cu - divergence of rows of logits from a teacher's top entries, and its gradient, sm_103a.
//
// Row r with logits z, temperature T and weight w; its list of entries (id_j, t_j):
//   p_j = softmax_j(t_j / T),  log q_v = z_v / T - L,  L = ln sum_v exp(z_v / T)
//   kl = sum_j p_j (ln p_j - log q_{id_j}),  loss = sum_r w kl,  dz_v = w / T (q_v - sum_{j: id_j = v} p_j)
#include <cfloat>
#include <cstdint>

#include "internal.h"
#include "sm100.cuh"

namespace vcs {
namespace {

using namespace dev;
using bf16 = __nv_bfloat16;

constexpr int kMaxTop = VCS_DISTILL_MAX_TOP;
constexpr int kBytes = 16;   // of a vector

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

// Largest logit and sum of exponentials, taken together in one pass.
struct Sum {
  float m, s;
  __device__ __forceinline__ void join(float m2, float s2, float k) {
    const float top = fmaxf(m, m2), base = top == -INFINITY ? 0.f : top;   // nothing but -inf so far: sums of 0
    s = s * ex2((m - base) * k) + s2 * ex2((m2 - base) * k);
    m = top;
  }
  template <int N>
  __device__ __forceinline__ void add(const float (&x)[N], float k) {
    float top = x[0];
#pragma unroll
    for (int i = 1; i + 1 < N; i += 2) top = fmax3(top, x[i], x[i + 1]);
    if (N % 2 == 0) top = fmaxf(top, x[N - 1]);
    if (top > m) {   // rarely, after the first elements
      s *= ex2((m - top) * k);
      m = top;
    }
    const float base = m == -INFINITY ? 0.f : m;
    const uint64_t mm = f2pack(-base, -base), kk = f2pack(k, k);
    uint64_t acc = 0ull;
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      float a, b;
      exp_pair(x[i], x[i + 1], mm, kk, a, b);
      acc = fadd2(acc, f2pack(a, b));
    }
    float a, b;
    f2unpack(acc, a, b);
    s += a + b;
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

// A block a row at a time, in two passes over its logits: the statistics, then the gradient, whose read finds the row in
// L2 (the rows under way, a few hundred, are at most half of it).  What bounds it is memory: 4,096 rows of 131,072 bf16
// logits with their gradient move 2.15 GB.
template <class T, int THREADS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) distill_rows(const __grid_constant__ Args a) {
  constexpr int N = Vec<T>::N, U = 4;                  // vectors a thread has under way
  constexpr int E = (kMaxTop + THREADS - 1) / THREADS; // entries of a thread
  __shared__ __align__(16) int32_t ids[kMaxTop];
  __shared__ __align__(16) float ps[kMaxTop];
  constexpr int W = THREADS / 32;
  __shared__ double red64[W], logs[2];
  __shared__ float red_m[W], red_s[W], red_t[W], red_p[W];
  __shared__ bool last;
  const float k = a.k;
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  // Warps with entries.  fp64 is slow here (a log of every thread's took 13 us a row): the logarithms are one lane's, of
  // the last warp, and the sums of entries their warps'.
  const int warps = min(W, (a.top + 31) / 32);
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
      if (dz != nullptr) {
        const int64_t head = min(a.vocab, (int64_t)((kBytes - (reinterpret_cast<uintptr_t>(dz) & (kBytes - 1))) / sizeof(T)) % N);
        const int64_t vecs = (a.vocab - head) / N;
        for (int64_t v = threadIdx.x; v < vecs; v += THREADS)
          reinterpret_cast<uint4*>(dz + head)[v] = make_uint4(0u, 0u, 0u, 0u);
        if (threadIdx.x < head) put(dz + threadIdx.x, 0.f);
        for (int64_t v = head + vecs * N + threadIdx.x; v < a.vocab; v += THREADS) put(dz + v, 0.f);
      }
      continue;
    }
    if (list < 0 || list >= a.lists) {
      if (threadIdx.x == 0) set_status(a.status, VCS_ERR_DEVICE_CHECK);
      list = -1;
    }
    // the list's entries, under way while the row is read
    int my_id[E];
    float my_t[E];
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int j = threadIdx.x + i * THREADS;
      my_id[i] = -1;
      my_t[i] = -INFINITY;
      if (j < a.top && list >= 0) {
        my_id[i] = __ldg(&a.ids[list * a.top + j]);
        my_t[i] = __ldg(&a.t[list * a.top + j]);
      }
    }
    // ---- statistics of the row
    Sum sum{-INFINITY, 0.f};
    {
      const int64_t head = min(a.vocab, (int64_t)((kBytes - (reinterpret_cast<uintptr_t>(z) & (kBytes - 1))) / sizeof(T)) % N);
      const int64_t vecs = (a.vocab - head) / N;
      const uint4* zv = reinterpret_cast<const uint4*>(z + head);
      int64_t v = threadIdx.x;
      for (; v + (U - 1) * THREADS < vecs; v += U * THREADS) {
        uint4 x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = __ldg(zv + v + u * THREADS);
#pragma unroll
        for (int u = 0; u < U; ++u) {
          float f[N];
          Vec<T>::open(x[u], f);
          sum.add<N>(f, k);
        }
      }
      for (; v < vecs; v += THREADS) {
        float f[N];
        Vec<T>::open(__ldg(zv + v), f);
        sum.add<N>(f, k);
      }
      const int64_t rest = a.vocab - head - vecs * N;   // with the head, fewer than two vectors
      if (threadIdx.x < head + rest) {
        const float x = to_float(z[threadIdx.x < head ? threadIdx.x : vecs * N + threadIdx.x]);
        const float f[2] = {x, -INFINITY};
        sum.add<2>(f, k);
      }
    }
    // ---- and of the list; a NaN goes through (fmaxf drops it, the sums do not)
    float tmax = -INFINITY;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int j = threadIdx.x + i * THREADS;
      if (my_id[i] < -1 || my_id[i] >= a.vocab) {
        set_status(a.status, VCS_ERR_DEVICE_CHECK);
        my_id[i] = -1;
      }
      if (my_id[i] < 0) my_t[i] = -INFINITY;
      tmax = fmaxf(tmax, my_t[i] != my_t[i] ? INFINITY : my_t[i]);
      if (j < a.top) ids[j] = my_id[i];
    }
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
    sum.m = red_m[0];
#pragma unroll
    for (int i = 1; i < W; ++i) {
      sum.m = fmaxf(sum.m, red_m[i]);
      tmax = fmaxf(tmax, red_t[i]);
    }
    const bool empty = tmax == -INFINITY;                    // nothing to learn from
    const float zmax = sum.m == -INFINITY ? NAN : sum.m;     // nothing but -inf: no distribution
    sum.s = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) sum.s += red_s[i] * ex2((red_m[i] - zmax) * k);
    float mine = 0.f, p_of[E];
#pragma unroll
    for (int i = 0; i < E; ++i) {
      my_t[i] = my_t[i] == -INFINITY ? my_t[i] : my_t[i] - tmax;   // (+inf - +inf is a NaN)
      p_of[i] = my_t[i] == -INFINITY ? 0.f : expf(my_t[i] * a.inv_t);
      mine += p_of[i];
    }
    if (wid < warps) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
      if (lane == 0) red_p[wid] = mine;
    }
    // the entries' logits, before any is overwritten (dz may be z)
    float keep[E];
#pragma unroll
    for (int i = 0; i < E; ++i) keep[i] = my_id[i] >= 0 ? to_float(z[my_id[i]]) : 0.f;
    __syncthreads();
    float psum = 0.f;
    for (int i = 0; i < warps; ++i) psum += red_p[i];
    if (threadIdx.x == THREADS - 1) {
      logs[0] = log((double)sum.s);
      logs[1] = log((double)psum);
    }
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int j = threadIdx.x + i * THREADS;
      p_of[i] = p_of[i] / psum;
      if (j < a.top) ps[j] = my_t[i] == -INFINITY ? 0.f : p_of[i];
    }
    // the divergence, when the logarithms are there, and the sum of its terms
    auto divergence = [&] {
      double kl = 0.0;
      if (wid < warps) {
#pragma unroll
        for (int i = 0; i < E; ++i)
          if (my_id[i] >= 0 && my_t[i] != -INFINITY && p_of[i] != 0.f) {
            const double logp = (double)my_t[i] * a.inv_t - logs[1];
            const double logq = ((double)keep[i] - zmax) * a.inv_t - logs[0];
            kl += p_of[i] * (logp - logq);
          }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) kl += __shfl_xor_sync(0xffffffffu, kl, o);
        if (lane == 0) red64[wid] = kl;
      }
      __syncthreads();
      if (threadIdx.x == 0) {
        for (int i = 1; i < warps; ++i) kl += red64[i];
        a.row_kl[r] = empty ? 0.f : (float)kl;
        a.terms[r] = empty ? 0.0 : (double)w * kl;
      }
    };
    if (dz == nullptr) {
      __syncthreads();
      divergence();
      continue;
    }
    // ---- gradient
    const float c = empty ? 0.f : w * a.inv_t, inv = empty ? 0.f : 1.f / sum.s, g = c * inv, base = empty ? 0.f : zmax;
    const uint64_t mm = f2pack(-base, -base), kk = f2pack(k, k), gg = f2pack(g, g);
    auto grad = [&](float x) { return empty ? 0.f : ex2((x - base) * k) * g; };
    const uint32_t at = reinterpret_cast<uintptr_t>(dz) & (kBytes - 1);
    // bytes from a vector of the gradient's back to one of the logits': 0 where the rows are aligned alike
    const uint32_t shift = (uint32_t)((reinterpret_cast<uintptr_t>(z) - reinterpret_cast<uintptr_t>(dz)) & (kBytes - 1));
    int64_t head = min(a.vocab, (int64_t)((kBytes - at) / sizeof(T)) % N);
    int64_t vecs = (a.vocab - head) / N;
    if (shift != 0) {   // vectors whose two of the logits lie in the row
      while (vecs > 0 && head * (int64_t)sizeof(T) < (int64_t)shift) head += N, --vecs;
      while (vecs > 0 && (head + vecs * N) * (int64_t)sizeof(T) - shift + kBytes > a.vocab * (int64_t)sizeof(T)) --vecs;
    }
    const uint4* zv = reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(z + head) - shift);
    uint4* gv = reinterpret_cast<uint4*>(dz + head);
    // words of the logits under a vector of the gradient, from two vectors
    auto fetch = [&](int64_t v) {
      const uint4 lo = zv[v];
      if (shift == 0) return lo;
      const uint4 hi = zv[v + 1];
      const uint32_t words[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
      uint32_t o[4];
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (shift >> 2 == q)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[i] = __funnelshift_r(words[q + i], words[(q + i + 1) & 7], (shift & 3) * 8);
      return make_uint4(o[0], o[1], o[2], o[3]);
    };
    auto store = [&](int64_t v, const uint4& x) {
      float f[N];
      Vec<T>::open(x, f);
#pragma unroll
      for (int i = 0; i < N; i += 2) {
        float e0, e1;
        exp_pair(f[i], f[i + 1], mm, kk, e0, e1);
        f2unpack(fmul2(f2pack(e0, e1), gg), f[i], f[i + 1]);
        if (empty) f[i] = f[i + 1] = 0.f;
      }
      __stcs(gv + v, Vec<T>::close(f));
    };
    // (rows aligned otherwise in place: a vector's second read may be another thread's write, so all of a block's are read
    // before any is written; dz == z has shift 0)
    int64_t v = threadIdx.x;
    for (; v + (U - 1) * THREADS < vecs; v += U * THREADS) {
      uint4 x[U];
#pragma unroll
      for (int u = 0; u < U; ++u) x[u] = fetch(v + u * THREADS);
#pragma unroll
      for (int u = 0; u < U; ++u) store(v + u * THREADS, x[u]);
    }
    for (; v < vecs; v += THREADS) store(v, fetch(v));
    const int64_t rest = a.vocab - head - vecs * N;
    for (int64_t i = threadIdx.x; i < head + rest; i += THREADS) {
      const int64_t e = i < head ? i : vecs * N + i;
      put(dz + e, grad(to_float(z[e])));
    }
    __syncthreads();
    // the entries again, less their p: one that comes twice by its first place, with the sum of both
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int j = threadIdx.x + i * THREADS;
      if (my_id[i] < 0) continue;
      float p = 0.f;
      bool first = true;
      for (int m = 0; m < a.top; ++m)
        if (ids[m] == my_id[i]) {
          p += ps[m];
          first &= m >= j;
        }
      if (first) put(dz + my_id[i], empty ? 0.f : c * (ex2((keep[i] - base) * k) * inv - p));
    }
    divergence();
  }
  // the block that finishes last adds the rows' terms, in row order, so that the loss does not depend on scheduling
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

template <class T>
cudaError_t launch_rows(const Args& a, cudaStream_t st) {
  // A row of few vectors leaves most of a large block without work, and its fixed time shows: small blocks, more of them.
  if (a.vocab * (int64_t)sizeof(T) <= 32768) {
    const unsigned grid = (unsigned)(a.rows < 152 * 8 ? a.rows : 152 * 8);
    distill_rows<T, 128><<<grid, 128, 0, st>>>(a);
  } else {
    const unsigned grid = (unsigned)(a.rows < 152 * 2 ? a.rows : 152 * 2);
    distill_rows<T, 512><<<grid, 512, 0, st>>>(a);
  }
  return cudaGetLastError();
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
