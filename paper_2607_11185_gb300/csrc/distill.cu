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

using dev::set_status;
using bf16 = __nv_bfloat16;

constexpr int kThreads = 512;
constexpr int kMaxTop = VCS_DISTILL_MAX_TOP;

struct Args {
  const void* z;
  int64_t rows, vocab, ld;
  const int32_t* ids;
  const float* t;
  int32_t top;
  int64_t lists;
  const int32_t* map;
  const float* weights;
  float inv_t;
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

// Sum and maximum over the block; every thread gets them.
__device__ __forceinline__ float block_max(float x, float* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = x;
  __syncthreads();
  x = red[0];
  for (int i = 1; i < kThreads / 32; ++i) x = fmaxf(x, red[i]);
  return x;
}
template <class T>
__device__ __forceinline__ T block_sum(T x, T* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = x;
  __syncthreads();
  x = red[0];
  for (int i = 1; i < kThreads / 32; ++i) x += red[i];
  return x;
}

// A block a row: the maximum, the sum, the list, the gradient, and the gradient again at the list's entries.
template <class T>
__global__ void __launch_bounds__(kThreads) distill_rows(const __grid_constant__ Args a) {
  __shared__ int32_t ids[kMaxTop];
  __shared__ float ps[kMaxTop];
  __shared__ double red64[kThreads / 32];
  __shared__ float red[kThreads / 32];
  __shared__ bool last;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T* z = static_cast<const T*>(a.z) + r * a.ld;
    T* dz = a.dz == nullptr ? nullptr : static_cast<T*>(a.dz) + r * a.ldg;
    const float w = a.weights[r];
    int64_t list = a.map == nullptr ? r : a.map[r];
    if (list < 0 || list >= a.lists) {
      if (threadIdx.x == 0) set_status(a.status, VCS_ERR_DEVICE_CHECK);
      list = -1;
    }
    float tmax = -INFINITY;
    __syncthreads();
    if (w != 0.f && list >= 0) {
      for (int j = threadIdx.x; j < a.top; j += kThreads) {
        int id = a.ids[list * a.top + j];
        if (id < -1 || id >= a.vocab) {
          set_status(a.status, VCS_ERR_DEVICE_CHECK);
          id = -1;
        }
        const float t = id < 0 ? -INFINITY : a.t[list * a.top + j];
        ids[j] = id;
        ps[j] = t;
        tmax = t != t ? t : fmaxf(tmax, t);
      }
    }
    // NaN goes through: fmaxf drops it, so it is counted apart
    const bool bad = __syncthreads_or(tmax != tmax);
    tmax = block_max(tmax, red);
    if (w == 0.f || list < 0 || (tmax == -INFINITY && !bad)) {  // nothing to learn from
      if (threadIdx.x == 0) a.row_kl[r] = 0.f, a.terms[r] = 0.0;
      if (dz != nullptr)
        for (int64_t v = threadIdx.x; v < a.vocab; v += kThreads) put(dz + v, 0.f);
      continue;
    }
    if (bad) tmax = NAN;
    float zmax = -INFINITY;
    bool nan = false;
    for (int64_t v = threadIdx.x; v < a.vocab; v += kThreads) {
      const float x = to_float(z[v]);
      nan |= x != x;
      zmax = fmaxf(zmax, x);
    }
    nan = __syncthreads_or(nan);
    zmax = nan ? NAN : block_max(zmax, red);
    float sum = 0.f;
    for (int64_t v = threadIdx.x; v < a.vocab; v += kThreads) sum += expf((to_float(z[v]) - zmax) * a.inv_t);
    sum = block_sum(sum, red);
    float psum = 0.f;
    for (int j = threadIdx.x; j < a.top; j += kThreads) psum += ps[j] == -INFINITY ? 0.f : expf((ps[j] - tmax) * a.inv_t);
    psum = block_sum(psum, red);
    const double lnorm = log((double)sum), lp = log((double)psum);
    double kl = 0.0;
    for (int j = threadIdx.x; j < a.top; j += kThreads) {
      if (ids[j] < 0 || ps[j] == -INFINITY) {
        ps[j] = 0.f;
        continue;
      }
      const float p = expf((ps[j] - tmax) * a.inv_t) / psum;
      const double logp = ((double)ps[j] - tmax) * a.inv_t - lp;
      const double logq = ((double)to_float(z[ids[j]]) - zmax) * a.inv_t - lnorm;
      ps[j] = p;
      if (p != 0.f) kl += p * (logp - logq);
    }
    kl = block_sum(kl, red64);
    if (threadIdx.x == 0) a.row_kl[r] = (float)kl, a.terms[r] = (double)w * kl;
    if (dz == nullptr) continue;
    const float c = w * a.inv_t, inv = 1.f / sum;
    // the listed entries' logits before any is overwritten (dz may be z)
    float keep[kMaxTop / kThreads];
#pragma unroll
    for (int i = 0; i < kMaxTop / kThreads; ++i) {
      const int j = threadIdx.x + i * kThreads;
      keep[i] = j < a.top && ids[j] >= 0 ? to_float(z[ids[j]]) : 0.f;
    }
    __syncthreads();
    for (int64_t v = threadIdx.x; v < a.vocab; v += kThreads)
      put(dz + v, c * (expf((to_float(z[v]) - zmax) * a.inv_t) * inv));
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kMaxTop / kThreads; ++i) {
      const int j = threadIdx.x + i * kThreads;
      if (j >= a.top || ids[j] < 0) continue;
      float p = 0.f;
      bool first = true;
      for (int m = 0; m < a.top; ++m)
        if (ids[m] == ids[j]) {
          p += ps[m];
          first &= m >= j;
        }
      if (first) put(dz + ids[j], c * (expf((keep[i] - zmax) * a.inv_t) * inv - p));
    }
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
  for (int64_t r = threadIdx.x; r < a.rows; r += kThreads) x += __ldcg(&a.terms[r]);
  x = block_sum(x, red64);
  if (threadIdx.x == 0) *a.loss = (float)x;
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
  a.loss = d.loss;
  a.row_kl = d.row_kl;
  a.dz = d.dlogits;
  a.ldg = d.grad_stride;
  a.status = static_cast<int32_t*>(ws);
  a.done = reinterpret_cast<uint32_t*>(ws) + 1;
  a.terms = reinterpret_cast<double*>(static_cast<char*>(ws) + kWsHeader);
  const unsigned grid = (unsigned)(d.rows < 152 * 4 ? d.rows : 152 * 4);
  if (d.f32)
    distill_rows<float><<<grid, kThreads, 0, st>>>(a);
  else
    distill_rows<bf16><<<grid, kThreads, 0, st>>>(a);
  return cudaGetLastError();
}

}  // namespace vcs
