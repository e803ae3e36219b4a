// logit_controls.cu -- penalties for repeated tokens, biases and grammar masks
// on logits (sm_103a).
//
//   x > 0 ? x / r : x r (tokens of the history), - f count - p (generated ones), + bias, -inf where not allowed
//
// A row is cut into slices of the vocabulary, a CTA each.  The slice's logits stream
// through with the mask applied, which is what counts: they are on their way from the
// start, before the history is looked at.  The few tokens that a penalty or a bias
// applies to are then put right one by one.  How often each occurs is counted in a
// table in shared memory with an entry for each token of the slice, of which only the
// entries of tokens that occur are ever set to zero, so that a short history costs
// little whatever the vocabulary.  The first thread that claims an entry writes the
// token's logit.  Every CTA reads the whole history, and takes what falls in its slice.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "decode_internal.h"
#include "stride_device.cuh"

namespace stride {
namespace {

constexpr int kThreads = 512;
constexpr int kHeld = 8;      // tokens of the history that a thread keeps
constexpr int kAhead = 6;     // vectors of logits that a thread has on their way
constexpr uint32_t kPrompt = 0x80000000u, kClaimed = 0xffffffffu;

__device__ __forceinline__ float value(float x) { return x; }
__device__ __forceinline__ float value(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float value(__half x) { return __half2float(x); }
template <typename T>
__device__ __forceinline__ T rounded(float x);
template <>
__device__ __forceinline__ float rounded<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 rounded<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <>
__device__ __forceinline__ __half rounded<__half>(float x) { return __float2half_rn(x); }

// -inf in the places of a 16-byte vector whose bit is clear.
template <typename T>
__device__ __forceinline__ uint4 masked(uint4 v, uint32_t bits) {
  uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      if (!((bits >> i) & 1)) w[i] = 0xff800000u;
    } else {
      constexpr uint32_t kInf = std::is_same<T, __half>::value ? 0xfc00u : 0xff80u;
      if (!((bits >> (2 * i)) & 1)) w[i] = (w[i] & 0xffff0000u) | kInf;
      if (!((bits >> (2 * i + 1)) & 1)) w[i] = (w[i] & 0xffffu) | kInf << 16;
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// Blocks: row * slices + slice.  Shared memory: `slice` counts and, where there are biases, as many places of the last entry.
template <typename T>
__global__ void __launch_bounds__(kThreads) controls_kernel(const __grid_constant__ ControlParams p, const int slice, const int slices) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  extern __shared__ uint32_t table[];
  constexpr int kVec = 16 / (int)sizeof(T);
  uint32_t* const count = table;
  uint32_t* const entry = table + slice;
  const int row = blockIdx.x / slices, tid = threadIdx.x;
  const int c0 = (blockIdx.x - row * slices) * slice, c1 = min(p.V, c0 + slice);  // (V is below 2^30 and a slice more)
  const stride_logit_rules& r = p.how;
  const T* const x = static_cast<const T*>(p.x) + row * p.ld;
  T* const out = static_cast<T*>(p.out) + row * p.ld_out;
  const bool in_place = p.x == p.out;
  const uint32_t* const allowed = r.allowed ? r.allowed + row * r.allowed_stride : nullptr;

  // ---- what applies to the row ----
  float rep = 1.f, freq = 0.f, pres = 0.f;
  int n = 0, prompt = 0, bias0 = 0, biases = 0, bad = 0;
  if (r.history) {
    n = __ldg(r.history_len + row);
    prompt = r.prompt_len ? __ldg(r.prompt_len + row) : 0;
    rep = r.repetition ? __ldg(r.repetition + row) : r.repetition_all;
    freq = r.frequency ? __ldg(r.frequency + row) : r.frequency_all;
    pres = r.presence ? __ldg(r.presence + row) : r.presence_all;
    if (n < 0 || n > r.history_most) bad |= STRIDE_DEV_BAD_LAYOUT;
    if (!(rep > 0.f && isfinite(rep)) || !isfinite(freq) || !isfinite(pres)) bad |= STRIDE_DEV_BAD_CONTROL;
  }
  if (r.bias_off) {
    bias0 = __ldg(r.bias_off + row);
    const int end = __ldg(r.bias_off + row + 1);
    if (bias0 < 0 || end < bias0 || end > r.n_bias) bad |= STRIDE_DEV_BAD_LAYOUT;
    biases = end - bias0;
  }
  if (bad) {  // (all of the row's CTAs alike)
    for (int c = c0 + tid; c < c1; c += kThreads) out[c] = rounded<T>(NAN);
    if (tid == 0) set_status(p.dev_status, bad);
    return;
  }

  // ---- logits on their way, where they are copied as whole vectors ----
  const bool stream = !in_place || allowed;
  const bool same = ((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(out)) & 15) == 0;
  const int shift = (int)(((16 - (reinterpret_cast<uintptr_t>(x + c0) & 15)) & 15) / sizeof(T));  // elements before the first vector
  const int head = !same ? c1 : min(c1, c0 + shift);  // elements up to here, and those past the last vector, are taken one by one
  const int vecs = (c1 - head) / kVec;
  uint4 v[kAhead];
#pragma unroll
  for (int u = 0; u < kAhead; ++u) {
    const int i = tid + u * kThreads;
    if (stream && i < vecs) v[u] = *(reinterpret_cast<const uint4*>(x + head) + i);
  }

  // ---- counts ----
  const int32_t* const history = r.history + row * r.history_stride;
  const uint32_t wide = (uint32_t)(c1 - c0);
  int held[kHeld];
#pragma unroll
  for (int u = 0; u < kHeld; ++u) {
    const int i = tid + u * kThreads;
    held[u] = i < n ? __ldg(history + i) : -1;
  }
  // f(i, place in the slice) for this thread's tokens of the history that are in the slice
  const auto each = [&](auto&& f) {
#pragma unroll
    for (int u = 0; u < kHeld; ++u)
      if (held[u] >= 0 && (uint32_t)(held[u] - c0) < wide) f(tid + u * kThreads, held[u] - c0);
    for (int64_t i = tid + kHeld * kThreads; i < n; i += kThreads) {
      const int t = __ldg(history + i);
      if (t >= 0 && (uint32_t)(t - c0) < wide) f((int)i, t - c0);
    }
  };
  const auto each_bias = [&](auto&& f) {
    for (int64_t i = tid; i < biases; i += kThreads) {
      const int t = __ldg(r.bias_token + bias0 + i);
      if (t >= 0 && (uint32_t)(t - c0) < wide) f((uint32_t)i + 1, t - c0);
      if (c0 == 0 && t >= p.V) set_status(p.dev_status, STRIDE_DEV_TOKEN_RANGE);
    }
  };
  if (c0 == 0) {
#pragma unroll
    for (int u = 0; u < kHeld; ++u)
      if (held[u] >= p.V) set_status(p.dev_status, STRIDE_DEV_TOKEN_RANGE);
    for (int64_t i = tid + kHeld * kThreads; i < n; i += kThreads)
      if (__ldg(history + i) >= p.V) set_status(p.dev_status, STRIDE_DEV_TOKEN_RANGE);
  }
  const bool any = n > 0 || biases > 0;
  if (any) {
    each([&](int, int t) {
      count[t] = 0;
      if (biases) entry[t] = 0;
    });
    each_bias([&](uint32_t, int t) {
      count[t] = 0;
      entry[t] = 0;
    });
    __syncthreads();
    each([&](int i, int t) {
      if (i < prompt)
        atomicOr(&count[t], kPrompt);
      else
        atomicAdd(&count[t], 1u);
    });
    each_bias([&](uint32_t i, int t) { atomicMax(&entry[t], i); });
  }

  // ---- the slice with the mask ----
  const auto bits_from = [&](int c) {  // of columns c, c + 1, ... of a vector
    const uint32_t lo = __ldg(allowed + (c >> 5));
    const int s = c & 31;
    return s + kVec > 32 && ((c >> 5) + 1) * 32 < p.V ? __funnelshift_r(lo, __ldg(allowed + (c >> 5) + 1), s) : lo >> s;
  };
  if (stream) {
    constexpr uint32_t kFull = (1u << kVec) - 1;
    for (int i0 = tid; i0 < vecs; i0 += kAhead * kThreads) {
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int i = i0 + u * kThreads;
        if (i0 != tid && i < vecs) v[u] = *(reinterpret_cast<const uint4*>(x + head) + i);
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int i = i0 + u * kThreads;
        if (i >= vecs) continue;
        const uint32_t bits = allowed ? bits_from(head + i * kVec) & kFull : kFull;
        if (bits != kFull)
          v[u] = masked<T>(v[u], bits);
        else if (in_place)
          continue;
        *(reinterpret_cast<uint4*>(out + head) + i) = v[u];
      }
    }
    const auto one = [&](int c) {
      const bool ok = !allowed || (__ldg(allowed + (c >> 5)) >> (c & 31)) & 1;
      if (!ok)
        out[c] = rounded<T>(-INFINITY);
      else if (!in_place)
        out[c] = x[c];
    };
    for (int c = c0 + tid; c < head; c += kThreads) one(c);
    for (int c = head + vecs * kVec + tid; c < c1; c += kThreads) one(c);
  }
  if (!any) return;
  __syncthreads();

  // ---- the tokens that something applies to ----
  const auto fix = [&](int t) {
    const uint32_t seen = atomicExch(&count[t], kClaimed);
    if (seen == kClaimed) return;
    const int c = c0 + t;
    if (allowed && !((__ldg(allowed + (c >> 5)) >> (c & 31)) & 1)) return;
    float y = value(x[c]);
    if (seen) y = y > 0.f ? __fdiv_rn(y, rep) : y * rep;
    const uint32_t made = seen & ~kPrompt;
    if (made) y = y - freq * (float)made - pres;
    if (biases && entry[t]) y += __ldg(r.bias + bias0 + entry[t] - 1);
    out[c] = rounded<T>(y);
  };
  each([&](int, int t) { fix(t); });
  each_bias([&](uint32_t, int t) { fix(t); });
}

template <typename T>
cudaError_t run(const ControlParams& p, cudaStream_t stream) {
  // entries of a slice's tables: two CTAs on an SM
  const int per = p.how.bias_off ? 8 : 4, most = 98304 / per;
  const int about = (p.V + most - 1) / most, slice = ((p.V + about - 1) / about + 63) & ~63, slices = (p.V + slice - 1) / slice;
  if ((int64_t)slices * p.rows > INT32_MAX) return cudaErrorInvalidValue;
  const auto kern = controls_kernel<T>;
  const size_t smem = p.how.history || p.how.bias_off ? (size_t)slice * per : 0;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 98304 + 1024);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(p.rows * slices);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  e = cudaLaunchKernelEx(&cfg, kern, p, slice, slices);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

cudaError_t launch_logit_controls(const ControlParams& p, int dtype, int, cudaStream_t stream) {
  if (dtype == STRIDE_DTYPE_BF16) return run<__nv_bfloat16>(p, stream);
  if (dtype == STRIDE_DTYPE_F16) return run<__half>(p, stream);
  return run<float>(p, stream);
}

}  // namespace stride
