// linear.cu - linear attention with a decay for each key/value head, over packed variable-length segments, sm_103a.
//
// With lam = exp(log_decay) of the head, over the tokens t of a segment:
//   S_t = lam S_{t-1} + k_t v_t^T,   o_t = scale q_t^T S_t
// Its gradients are calls of the same kind: with R_t = lam R_{t+1} + sum_group q_t do_t^T,
//   dq_t = scale S_t do_t   (queries do, keys v, values k)
//   dk_t = scale R_t v_t    (queries v, keys do, values q, from the last token to the first)
//   dv_t = scale R_t^T k_t  (queries k, keys q, values do, likewise)
// where the first has a group of query heads to a state, the others a group of key heads.
#include <cfloat>
#include <cstdint>

#include "internal.h"
#include "sm100.cuh"

namespace vcs {
namespace {

using namespace dev;
using bf16 = __nv_bfloat16;

__device__ __forceinline__ bool decay_ok(float g) { return g <= 0.f && g >= -FLT_MAX; }

struct WalkArgs {
  const bf16 *q, *k, *v;  // [tokens, state heads * gq], [tokens, state heads * gk] twice
  const float* log_decay;
  const int32_t* cu_seqlens;
  int32_t num_segments, num_tokens, heads, gq, gk;
  float scale;
  bool back;  // from each segment's last token to its first
  const float* state_in;
  float* state_out;
  bf16* o;
  int32_t* status;
};

constexpr int kCols = 32, kGroups = 8;

// Token by token.  A block holds 32 columns of one head's state in registers, thread (g, c) rows g D/8 .. of column c.
template <int D>
__global__ void __launch_bounds__(256) linear_walk(const __grid_constant__ WalkArgs a) {
  constexpr int R = D / kGroups;
  __shared__ float sk[D], sq[D], sv[kCols], red[kGroups * kCols];
  const int slices = D / kCols;
  const int unit = blockIdx.x / slices, col0 = blockIdx.x % slices * kCols;
  const int seg = unit / a.heads, head = unit % a.heads;
  const int c = threadIdx.x & 31, g = threadIdx.x >> 5;
  const int start = a.cu_seqlens[seg], end = a.cu_seqlens[seg + 1];
  const float ld = a.log_decay[head];
  if (start < 0 || end < start || end > a.num_tokens || !decay_ok(ld)) {
    if (threadIdx.x == 0) set_status(a.status, VCS_ERR_DEVICE_CHECK);
    return;
  }
  const float lam = expf(ld);
  float s[R];
  const size_t at = ((size_t)unit * D + g * R) * D + col0 + c;
#pragma unroll
  for (int i = 0; i < R; ++i) s[i] = a.state_in != nullptr ? a.state_in[at + (size_t)i * D] : 0.f;
  for (int n = 0; n < end - start; ++n) {
    const size_t t = a.back ? end - 1 - n : start + n;
#pragma unroll
    for (int i = 0; i < R; ++i) s[i] *= lam;
    for (int h = 0; h < a.gk; ++h) {
      const size_t row = (t * a.heads + head) * a.gk + h;
      __syncthreads();
      if (threadIdx.x < D) sk[threadIdx.x] = __bfloat162float(a.k[row * D + threadIdx.x]);
      if (threadIdx.x < kCols) sv[threadIdx.x] = __bfloat162float(a.v[row * D + col0 + threadIdx.x]);
      __syncthreads();
#pragma unroll
      for (int i = 0; i < R; ++i) s[i] += sk[g * R + i] * sv[c];
    }
    for (int h = 0; h < a.gq; ++h) {
      const size_t row = (t * a.heads + head) * a.gq + h;
      if (threadIdx.x < D) sq[threadIdx.x] = __bfloat162float(a.q[row * D + threadIdx.x]);
      __syncthreads();
      float x = 0.f;
#pragma unroll
      for (int i = 0; i < R; ++i) x += sq[g * R + i] * s[i];
      red[g * kCols + c] = x;
      __syncthreads();
      if (g == 0) {
#pragma unroll
        for (int i = 1; i < kGroups; ++i) x += red[i * kCols + c];
        a.o[row * D + col0 + c] = __float2bfloat16(a.scale * x);
      }
      __syncthreads();
    }
  }
  if (a.state_out != nullptr)
#pragma unroll
    for (int i = 0; i < R; ++i) a.state_out[at + (size_t)i * D] = s[i];
}

template <int D>
cudaError_t launch_walk(const WalkArgs& a, cudaStream_t st) {
  const int64_t blocks = (int64_t)a.num_segments * a.heads * (D / kCols);
  if (blocks > INT32_MAX) return cudaErrorInvalidConfiguration;
  if (blocks > 0) linear_walk<D><<<(unsigned)blocks, 256, 0, st>>>(a);
  return cudaGetLastError();
}

// One token of a sequence.  A block takes 4 SLICE_LANES columns of one head's state: lane l of a row's lanes holds four
// columns of every row its thread has, all loaded before the first is used.
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

template <int D, int COLS>
__global__ void __launch_bounds__(kStepThreads) linear_step(const __grid_constant__ StepArgs a) {
  constexpr int LANES = COLS / 4;                // threads of a row
  constexpr int RG = kStepThreads / LANES;       // row groups
  constexpr int R = D / RG;                      // rows of a thread: rg, rg + RG, ...
  __shared__ float sk[D], sq[D];
  __shared__ float4 red[kStepThreads];
  const int slices = D / COLS;
  const int64_t unit = blockIdx.x / slices;
  const int col0 = blockIdx.x % slices * COLS;
  const int head = (int)(unit % a.hkv);
  const float ld = a.log_decay[head];
  if (!decay_ok(ld)) {
    if (threadIdx.x == 0) set_status(a.status, VCS_ERR_DEVICE_CHECK);
    return;
  }
  const int lane = threadIdx.x % LANES, rg = threadIdx.x / LANES;
  float4* p = reinterpret_cast<float4*>(a.states + ((size_t)unit * D + rg) * D + col0) + lane;
  float4 s[R];
#pragma unroll
  for (int i = 0; i < R; ++i) s[i] = p[(size_t)i * RG * (D / 4)];
  const bf16* vp = a.v + (size_t)unit * D + col0 + lane * 4;
  const float v0 = __bfloat162float(vp[0]), v1 = __bfloat162float(vp[1]), v2 = __bfloat162float(vp[2]),
              v3 = __bfloat162float(vp[3]);
  if (threadIdx.x < D) sk[threadIdx.x] = __bfloat162float(a.k[(size_t)unit * D + threadIdx.x]);
  const float lam = expf(ld);
  __syncthreads();
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const float k = sk[rg + i * RG];
    s[i].x = lam * s[i].x + k * v0;
    s[i].y = lam * s[i].y + k * v1;
    s[i].z = lam * s[i].z + k * v2;
    s[i].w = lam * s[i].w + k * v3;
    p[(size_t)i * RG * (D / 4)] = s[i];
  }
  for (int h = 0; h < a.group; ++h) {
    const size_t row = (size_t)unit * a.group + h;
    if (threadIdx.x < D) sq[threadIdx.x] = __bfloat162float(a.q[row * D + threadIdx.x]);
    __syncthreads();
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const float q = sq[rg + i * RG];
      x.x += q * s[i].x;
      x.y += q * s[i].y;
      x.z += q * s[i].z;
      x.w += q * s[i].w;
    }
    red[threadIdx.x] = x;
    __syncthreads();
    if (threadIdx.x < COLS) {
      float y = 0.f;
      for (int i = 0; i < RG; ++i) y += reinterpret_cast<const float*>(red)[i * COLS + threadIdx.x];
      a.o[row * D + col0 + threadIdx.x] = __float2bfloat16(a.scale * y);
    }
    __syncthreads();
  }
}

}  // namespace

size_t linear_fwd_ws_bytes(int32_t, int64_t, int32_t, int32_t, int32_t) { return kWsHeader; }
size_t linear_bwd_ws_bytes(int32_t, int64_t, int32_t, int32_t, int32_t) { return kWsHeader; }

cudaError_t launch_linear_fwd(const LinearArgs& a, const float* state_in, float* state_out, void* o, void* ws,
                              cudaStream_t st) {
  if (cudaError_t e = cudaMemsetAsync(ws, 0, kWsHeader, st); e != cudaSuccess) return e;
  WalkArgs w{};
  w.q = static_cast<const bf16*>(a.q);
  w.k = static_cast<const bf16*>(a.k);
  w.v = static_cast<const bf16*>(a.v);
  w.log_decay = a.log_decay;
  w.cu_seqlens = a.cu_seqlens;
  w.num_segments = a.num_segments;
  w.num_tokens = (int32_t)a.num_tokens;
  w.heads = a.hkv;
  w.gq = a.hq / a.hkv;
  w.gk = 1;
  w.scale = a.scale;
  w.state_in = state_in;
  w.state_out = state_out;
  w.o = static_cast<bf16*>(o);
  w.status = static_cast<int32_t*>(ws);
  return a.d == 64 ? launch_walk<64>(w, st) : launch_walk<128>(w, st);
}

cudaError_t launch_linear_bwd(const LinearArgs& a, const void* dout, void* dq, void* dk, void* dv, void* ws,
                              cudaStream_t st) {
  if (cudaError_t e = cudaMemsetAsync(ws, 0, kWsHeader, st); e != cudaSuccess) return e;
  const bf16 *q = static_cast<const bf16*>(a.q), *k = static_cast<const bf16*>(a.k),
             *v = static_cast<const bf16*>(a.v), *g = static_cast<const bf16*>(dout);
  WalkArgs w{};
  w.log_decay = a.log_decay;
  w.cu_seqlens = a.cu_seqlens;
  w.num_segments = a.num_segments;
  w.num_tokens = (int32_t)a.num_tokens;
  w.heads = a.hkv;
  w.scale = a.scale;
  w.status = static_cast<int32_t*>(ws);
  auto run = [&](const bf16* x, const bf16* y, const bf16* z, int gq, int gk, bool back, void* out) {
    w.q = x;
    w.k = y;
    w.v = z;
    w.gq = gq;
    w.gk = gk;
    w.back = back;
    w.o = static_cast<bf16*>(out);
    return a.d == 64 ? launch_walk<64>(w, st) : launch_walk<128>(w, st);
  };
  const int group = a.hq / a.hkv;
  cudaError_t e = run(g, v, k, group, 1, false, dq);
  if (e == cudaSuccess) e = run(v, g, q, 1, group, true, dk);
  if (e == cudaSuccess) e = run(k, q, g, 1, group, true, dv);
  return e;
}

template <int D>
static cudaError_t launch_step(const StepArgs& s, int64_t num_seqs, cudaStream_t st) {
  const int64_t units = num_seqs * s.hkv;
  if (units * (D / 32) > INT32_MAX) return cudaErrorInvalidConfiguration;
  if (units < 304)
    linear_step<D, 32><<<(unsigned)(units * (D / 32)), kStepThreads, 0, st>>>(s);
  else
    linear_step<D, D><<<(unsigned)units, kStepThreads, 0, st>>>(s);
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
