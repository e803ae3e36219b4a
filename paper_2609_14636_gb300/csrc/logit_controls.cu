// logit_controls.cu -- penalties for repeated tokens, biases and grammar masks
// on logits (sm_103a).
//
//   x > 0 ? x / r : x r (tokens of the history), - f count - p (generated ones), + bias, -inf where not allowed
//
// A row is cut into slices of the vocabulary, a CTA each, as many as run at once.
// What counts is that the slice streams through, with the mask applied: the CTA's warps
// take runs of it in turn, the next one's logits on their way.  Half of them first
// find what else applies to the slice: a bit for each token of the vocabulary
// that occurs, the number of bits before each word (so that a token's place among
// those that occur needs no search: a hash table's exchanges took 20,000
// clocks for 4,096 tokens), and a count and a last bias at each place.  The logits listed so
// are then put right, fetched while the slice is still in L2 (by a kernel of its
// own after the copy they came from memory again, 61 us beside the copy's 24 for 256
// rows of 151,936).  In place and without a mask only they are read.
//
// Measured, us (floor: of bytes at 6,683 GB/s): 256 rows of 151,936 bf16 with a mask, histories of up to 4,096 and 100 biases 36.5
// (24.5; 4.5 TB/s: the listed logits, after the slice, with few CTAs left to hide their latency); 512 rows of 32,000 fp32 without a
// mask 25.3 (20); one row 5.6 in a graph (a chain of eight steps between barriers).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "decode_internal.h"
#include "stride_device.cuh"

namespace stride {
namespace {

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

__device__ __forceinline__ const uint32_t* mask_row(const stride_logit_rules& r, int row) {
  return r.allowed ? r.allowed + row * r.allowed_stride : nullptr;
}
__device__ __forceinline__ bool is_allowed(const uint32_t* mask, int c) { return !mask || (__ldg(mask + (c >> 5)) >> (c & 31)) & 1; }

// -inf in the places of a 16-byte vector whose bit is clear.
template <typename T>
__device__ __forceinline__ uint4 masked(uint4 v, uint32_t bits) {
  uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      w[i] = (bits >> i) & 1 ? w[i] : 0xff800000u;
    } else {
      constexpr uint32_t kInf = std::is_same<T, __half>::value ? 0xfc00fc00u : 0xff80ff80u;
      const uint32_t keep = ((bits >> (2 * i)) & 1 ? 0xffffu : 0u) | ((bits >> (2 * i + 1)) & 1 ? 0xffff0000u : 0u);
      w[i] = (w[i] & keep) | (kInf & ~keep);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

constexpr int kThreads = 512;
constexpr int kCounters = 256;    // of them, those that count first (256 rows of 151,936, us: 36.8, all 42.1; one row in a graph 5.6, 5.9)
constexpr int kAhead = 3;         // vectors of a lane in a run (256 rows of 151,936, us: 2 38.3, 3 36.8, 4 38.5)
constexpr int kMostWords = 8192;  // of a slice's bits
constexpr int kWindow = 4096;     // places that have counts at a time
constexpr uint32_t kPrompt = 0x80000000u, kBias = 0x40000000u;  // flags of a count

// What applies to a row.
struct Applies {
  float rep, freq, pres;
  int n, prompt, bias0, biases, bad;
};
__device__ __forceinline__ Applies applies_to(const stride_logit_rules& r, int row) {
  Applies a = {1.f, 0.f, 0.f, 0, 0, 0, 0, 0};
  if (r.history) {
    a.n = __ldg(r.history_len + row);
    a.prompt = r.prompt_len ? __ldg(r.prompt_len + row) : 0;
    a.rep = r.repetition ? __ldg(r.repetition + row) : r.repetition_all;
    a.freq = r.frequency ? __ldg(r.frequency + row) : r.frequency_all;
    a.pres = r.presence ? __ldg(r.presence + row) : r.presence_all;
    if (a.n < 0 || a.n > r.history_most) a.bad |= STRIDE_DEV_BAD_LAYOUT;
    if (!(a.rep > 0.f && isfinite(a.rep)) || !isfinite(a.freq) || !isfinite(a.pres)) a.bad |= STRIDE_DEV_BAD_CONTROL;
  }
  if (r.bias_off) {
    a.bias0 = __ldg(r.bias_off + row);
    const int end = __ldg(r.bias_off + row + 1);
    if (a.bias0 < 0 || end < a.bias0 || end > r.n_bias) a.bad |= STRIDE_DEV_BAD_LAYOUT;
    a.biases = end - a.bias0;
  }
  return a;
}

// A run of a lane: kAhead vectors, 32 lanes' side by side, and the words of the mask that they need.
struct Run {
  int first;  // the lane's first vector; past the last: none
  uint4 v[kAhead];
  uint32_t lo[kAhead], hi[kAhead];
};

// Blocks: row * slices + slice.  Shared memory: the bits and their prefix sums, counts, tokens and last biases of a window.
template <typename T>
__global__ void __launch_bounds__(kThreads, 2) controls_kernel(const __grid_constant__ ControlParams p, const int slice, const int slices) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  constexpr int kVec = 16 / (int)sizeof(T);
  constexpr uint32_t kFull = (1u << kVec) - 1;
  extern __shared__ __align__(16) uint32_t smem[];
  __shared__ Applies s_applies;
  __shared__ int s_run, s_total, s_part[kThreads / 32];
  const int words = slice / 32;
  uint32_t* const bits = smem;
  uint32_t* const before = bits + words;
  uint32_t* const count = before + words;
  int32_t* const token = reinterpret_cast<int32_t*>(count + kWindow);
  uint32_t* const entry = count + 2 * kWindow;
  const int row = blockIdx.x / slices, tid = threadIdx.x, lane = tid & 31;
  const int c0 = (blockIdx.x - row * slices) * slice, c1 = min(p.V, c0 + slice);  // (V is below 2^30 and a slice more)
  const stride_logit_rules& r = p.how;
  const T* const x = static_cast<const T*>(p.x) + row * p.ld;
  T* const out = static_cast<T*>(p.out) + row * p.ld_out;
  const bool in_place = p.x == p.out;
  const uint32_t* const mask = mask_row(r, row);
  if (tid == 0) s_run = 0;
  __syncthreads();

  // ---- a first run of the slice on its way ----
  const bool streams = !in_place || mask;
  const uintptr_t at = reinterpret_cast<uintptr_t>(x + c0);
  const bool apart = ((at ^ reinterpret_cast<uintptr_t>(out + c0)) & 15) != 0;  // (no vector of one is one of the other)
  const int head = min(c1, c0 + (int)(((16 - (at & 15)) & 15) / sizeof(T))), vecs = streams && !apart ? (c1 - head) / kVec : 0;
  const auto take = [&](Run& u) {  // the next run
    int k = 0;
    if (lane == 0) k = atomicAdd(&s_run, 1);
    u.first = __shfl_sync(0xffffffffu, k, 0) * 32 * kAhead + lane;
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int i = u.first + 32 * j;
      if (i < vecs) u.v[j] = *(reinterpret_cast<const uint4*>(x + head) + i);
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int i = u.first + 32 * j, c = head + i * kVec, w = c >> 5;
      u.lo[j] = u.hi[j] = 0xffffffffu;
      if (!mask || i >= vecs) continue;
      u.lo[j] = __ldg(mask + w);
      if ((c & 31) + kVec > 32 && (w + 1) * 32 < p.V) u.hi[j] = __ldg(mask + w + 1);
    }
  };
  Run a;
  take(a);

  const int32_t* const history = r.history + row * r.history_stride;
  // f(i, place in the slice) for this thread's tokens of a list, of `by` threads
  constexpr int kOnce = 8;
  const auto each = [&](const int32_t* list, int64_t from, int len, int by, auto&& f) {  // (from: this thread's first)
    for (int64_t i0 = from; i0 < len; i0 += kOnce * by) {
      int t[kOnce];
#pragma unroll
      for (int u = 0; u < kOnce; ++u) t[u] = i0 + (int64_t)u * by < len ? __ldg(list + i0 + (int64_t)u * by) : -1;
#pragma unroll
      for (int u = 0; u < kOnce; ++u) f((int)(i0 + u * by), t[u]);
    }
  };
  const auto inside = [&](int t) { return t >= c0 && t < c1; };
  const auto place = [&](int t) { return before[t >> 5] + __popc(bits[t >> 5] & ((1u << (t & 31)) - 1)); };
  // Counts, tokens and biases of places w0 .. w0 + kWindow - 1, by all of `by` threads; `sync` between its steps.  held: this
  // thread's first tokens of the history, if it has them, at first, first + by, ...
  const auto fill = [&](const Applies& h, uint32_t w0, int me, int by, const int* held, auto&& sync) {
    for (int i = me; i < kWindow / 4; i += by) {
      reinterpret_cast<uint4*>(count)[i] = make_uint4(0, 0, 0, 0);
      if (h.biases) reinterpret_cast<uint4*>(entry)[i] = make_uint4(0, 0, 0, 0);
    }
    sync();
    const auto count_one = [&](int i, int t) {
      if (!inside(t)) return;
      const uint32_t k = place(t - c0) - w0;
      if (k >= kWindow) return;
      token[k] = t;
      if (i < h.prompt)
        atomicOr(&count[k], kPrompt);
      else
        atomicAdd(&count[k], 1u);
    };
    if (held)
#pragma unroll
      for (int u = 0; u < kOnce; ++u) count_one(me + u * by, held[u]);
    each(history, me + (held ? (int64_t)kOnce * by : 0), h.n, by, count_one);
    each(r.bias_token + h.bias0, me, h.biases, by, [&](int i, int t) {
      if (!inside(t)) return;
      const uint32_t k = place(t - c0) - w0;
      if (k >= kWindow) return;
      token[k] = t;
      atomicOr(&count[k], kBias);
      atomicMax(&entry[k], (uint32_t)i + 1);  // (of several entries the last)
    });
  };

  // ---- which tokens occur, and how often ----
  const bool fixes = r.history || r.bias_off;
  if (fixes && tid < kCounters) {
    const auto sync = [&] { asm volatile("bar.sync 1, %0;" ::"r"(kCounters) : "memory"); };
    int held[kOnce];  // (on their way with what says how many count)
#pragma unroll
    for (int u = 0; u < kOnce; ++u) {
      const int64_t i = tid + (int64_t)u * kCounters;
      held[u] = r.history && i < r.history_most ? __ldg(history + i) : -1;
    }
    const Applies h = applies_to(r, row);
#pragma unroll
    for (int u = 0; u < kOnce; ++u)
      if (tid + u * kCounters >= h.n) held[u] = -1;
    if (tid == 0) s_applies = h;
    const bool any = !h.bad && (h.n > 0 || h.biases > 0);
    if (tid == 0) s_total = 0;
    if (any) {
      for (int i = tid; i < words / 4; i += kCounters) reinterpret_cast<uint4*>(bits)[i] = make_uint4(0, 0, 0, 0);
      sync();
      const auto set = [&](int, int t) {
        if (inside(t))
          atomicOr(&bits[(t - c0) >> 5], 1u << ((t - c0) & 31));
        else if (t >= p.V && c0 == 0)
          set_status(p.dev_status, STRIDE_DEV_TOKEN_RANGE);
      };
#pragma unroll
      for (int u = 0; u < kOnce; ++u) set(0, held[u]);
      each(history, tid + (int64_t)kOnce * kCounters, h.n, kCounters, set);
      each(r.bias_token + h.bias0, tid, h.biases, kCounters, set);
      sync();
      // bits before each word: a warp's run of words by itself, four words of a lane at a time, then the warps' sums
      const int warp = tid >> 5, warps = kCounters >> 5, run = (words + 128 * warps - 1) / (128 * warps) * 128;
      const int i1 = min(words, (warp + 1) * run);
      int base = 0;
      for (int i0 = warp * run; i0 < i1; i0 += 128) {
        const int i = i0 + lane * 4;
        uint4 w = make_uint4(0, 0, 0, 0);
        if (i < i1) w = *reinterpret_cast<const uint4*>(bits + i);
        const int c[4] = {__popc(w.x), __popc(w.y), __popc(w.z), __popc(w.w)};
        const int own = c[0] + c[1] + c[2] + c[3];
        int upto = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int v = __shfl_up_sync(0xffffffffu, upto, o);
          if (lane >= o) upto += v;
        }
        const int first = base + upto - own;
        if (i < i1) *reinterpret_cast<uint4*>(before + i) = make_uint4(first, first + c[0], first + c[0] + c[1], first + c[0] + c[1] + c[2]);
        base += __shfl_sync(0xffffffffu, upto, 31);
      }
      if (lane == 0) s_part[warp] = base;
      sync();
      int others = 0, all = 0;
#pragma unroll
      for (int w = 0; w < kThreads / 32; ++w) {
        const int v = w < warps ? s_part[w] : 0;
        if (w < warp) others += v;
        all += v;
      }
      for (int i = warp * run + lane * 4; i < i1; i += 128) {
        uint4 w = *reinterpret_cast<const uint4*>(before + i);
        w.x += others;
        w.y += others;
        w.z += others;
        w.w += others;
        *reinterpret_cast<uint4*>(before + i) = w;
      }
      if (tid == 0) s_total = all;
      sync();
      fill(h, 0, tid, kCounters, held, sync);
    }
  }

  // ---- the slice with the mask ----
  if (apart) {  // (an element at a time: 256 rows of 151,936 under a mask 147 us, 44 where both are alike, L2 flushed)
    T v[8];
    for (int c = c0 + tid; c < c1; c += 8 * kThreads) {
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (c + u * kThreads < c1) v[u] = x[c + u * kThreads];
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (c + u * kThreads < c1) out[c + u * kThreads] = is_allowed(mask, c + u * kThreads) ? v[u] : rounded<T>(-INFINITY);
    }
  } else if (streams) {
    const auto put = [&](const Run& u) {
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int i = u.first + 32 * j;
        if (i >= vecs) continue;
        const uint32_t ok = __funnelshift_r(u.lo[j], u.hi[j], (head + i * kVec) & 31) & kFull;
        if (!(in_place && ok == kFull)) *(reinterpret_cast<uint4*>(out + head) + i) = masked<T>(u.v[j], ok);
      }
    };
    Run b;
    while (__any_sync(0xffffffffu, a.first < vecs)) {
      take(b);
      put(a);
      if (!__any_sync(0xffffffffu, b.first < vecs)) break;
      take(a);
      put(b);
    }
    const auto one = [&](int c) {
      if (!is_allowed(mask, c))
        out[c] = rounded<T>(-INFINITY);
      else if (!in_place)
        out[c] = x[c];
    };
    if (c0 + tid < head) one(c0 + tid);
    const int tail = head + vecs * kVec + tid;
    if (tail < c1) one(tail);
  }
  if (!fixes) return;
  __syncthreads();

  // ---- the tokens that something applies to ----
  const Applies h = s_applies;
  if (h.bad) {  // (all of the row's CTAs alike)
    for (int c = c0 + tid; c < c1; c += kThreads) out[c] = rounded<T>(NAN);
    if (tid == 0) set_status(p.dev_status, h.bad);
    return;
  }
  const auto sync = [] { __syncthreads(); };
  for (int w0 = 0; w0 < s_total; w0 += kWindow) {
    const int here = min(kWindow, s_total - w0);
    constexpr int kOnce = 4;  // logits of a thread on their way
    for (int i0 = tid; i0 < here; i0 += kOnce * kThreads) {
      float y[kOnce], bias[kOnce];
      uint32_t word[kOnce];
#pragma unroll
      for (int u = 0; u < kOnce; ++u) {
        const int i = i0 + u * kThreads;
        if (i >= here) continue;
        const int t = token[i];
        y[u] = value(x[t]);
        word[u] = mask ? __ldg(mask + (t >> 5)) : 0xffffffffu;
        bias[u] = count[i] & kBias ? __ldg(r.bias + h.bias0 + entry[i] - 1) : 0.f;
      }
#pragma unroll
      for (int u = 0; u < kOnce; ++u) {
        const int i = i0 + u * kThreads;
        if (i >= here) continue;
        const int t = token[i];
        if (!(word[u] >> (t & 31) & 1)) continue;
        const uint32_t seen = count[i], made = seen & ~(kPrompt | kBias);
        if (seen & ~kBias) y[u] = y[u] > 0.f ? __fdiv_rn(y[u], h.rep) : y[u] * h.rep;
        if (made) y[u] = y[u] - h.freq * (float)made - h.pres;
        if (seen & kBias) y[u] += bias[u];
        out[t] = rounded<T>(y[u]);
      }
    }
    if (w0 + kWindow >= s_total) break;
    __syncthreads();
    fill(h, w0 + kWindow, tid, kThreads, nullptr, sync);
    __syncthreads();
  }
}

template <typename T>
cudaError_t run(const ControlParams& p, int sms, cudaStream_t stream) {
  // twice as many slices as run at once (256 rows of 151,936, us: as many 39.6, twice 36.8, four times 46.6), of 8,192 tokens at least
  // and as many as there are bits for at most
  const int64_t most = (int64_t)p.V + 8191, wanted = std::max<int64_t>(1, 4 * sms / p.rows);
  const int64_t about = std::max<int64_t>(std::min<int64_t>(wanted, most / 8192), (p.V + kMostWords * 32 - 1) / (kMostWords * 32));
  const int slice = (int)(((p.V + about - 1) / about + 1023) & ~1023), slices = (p.V + slice - 1) / slice;
  if ((int64_t)slices * p.rows > INT32_MAX) return cudaErrorInvalidValue;
  const auto kern = controls_kernel<T>;
  const size_t smem = p.how.history || p.how.bias_off ? (size_t)slice / 4 + kWindow * (p.how.bias_off ? 12 : 8) : 0;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostWords * 8 + kWindow * 12);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)slices * p.rows);
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

cudaError_t launch_logit_controls(const ControlParams& p, int dtype, int sms, cudaStream_t stream) {
  if (dtype == STRIDE_DTYPE_BF16) return run<__nv_bfloat16>(p, sms, stream);
  if (dtype == STRIDE_DTYPE_F16) return run<__half>(p, sms, stream);
  return run<float>(p, sms, stream);
}

}  // namespace stride
