// sample.cu -- tokens from logits with temperature, top-k, top-p and min-p and
// given random numbers (sm_103a).
//
//   d_i = (x_i - max) / T, w_i = exp d_i; kept: the largest tokens (ties: lowest
//   index first) up to top_k, then up to top_p of their mass, then w >= min_p;
//   token = argmax over the kept of w_i / noise_i (an exponential race).
//
// A row is read from memory once, by a thread-block cluster whose CTAs keep
// their shares of it in shared memory.  What is kept is all above a threshold
// and, at it, the first few by index; the threshold is found without sorting:
// a histogram over the ordered bit patterns of the logits in the range that can
// hold it (counts for top-k, masses for top-p), summed over the cluster, gives
// the bin where the running count or mass crosses its target; that bin is the
// next range.  Masses are fixed-point integers (2^-40 of the largest weight), so
// the atomics' order changes nothing.  One pass over the share then races the
// kept tokens; noise is read for those alone.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include "decode_internal.h"
#include "stride_device.cuh"

namespace cg = cooperative_groups;

namespace stride {
namespace {

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kBins = 2048;
constexpr int kMaxCluster = 8;

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float widen(__half x) { return __half2float(x); }

// Order-preserving bits of a logit, both zeros alike, and back.
template <typename T>
struct Key;
template <>
struct Key<float> {
  static __device__ __forceinline__ uint32_t of(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
  }
  static __device__ __forceinline__ float value(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }
};
template <typename T>
struct Key16 {
  static __device__ __forceinline__ uint32_t of(T x) {
    uint32_t b = *reinterpret_cast<const uint16_t*>(&x);
    if (b == 0x8000u) b = 0;
    return b & 0x8000u ? ~b & 0xffffu : b | 0x8000u;
  }
  static __device__ __forceinline__ float value(uint32_t k) {
    const uint16_t b = (uint16_t)(k & 0x8000u ? k & 0x7fffu : ~k);
    return widen(*reinterpret_cast<const T*>(&b));
  }
};
template <>
struct Key<__nv_bfloat16> : Key16<__nv_bfloat16> {};
template <>
struct Key<__half> : Key16<__half> {};

template <typename T>
struct Vec {
  static constexpr int N = 16 / sizeof(T);
  alignas(16) T e[N];
};

template <typename T>
__device__ __forceinline__ T lowest();
template <>
__device__ __forceinline__ float lowest() { return -INFINITY; }
template <>
__device__ __forceinline__ __nv_bfloat16 lowest() { return __float2bfloat16_rn(-INFINITY); }
template <>
__device__ __forceinline__ __half lowest() { return __float2half_rn(-INFINITY); }

struct Best {  // the larger value, the lower index on ties
  float v;
  int32_t i;
};
__device__ __forceinline__ void take(Best& a, float v, int32_t i) {
  if (v > a.v || (v == a.v && i < a.i)) a = {v, i};
}

struct Shared {
  uint32_t cnt[kBins], lo[kBins], hi[kBins];
  // exchanged with the cluster
  Best top;
  int32_t bad;
  float sum;
  uint32_t total_cnt;
  uint64_t total_mass;
  uint32_t found_bin, found_cnt, found_at;  // the crossing bin, its count, the count above it
  uint64_t found_mass;                      // the mass above it
  Best race;
  float kept;
  // of the CTA
  Best wb[kWarps];
  float wf[kWarps];
  int32_t wi[kWarps];
  uint32_t wc[kWarps];
  uint64_t wm[kWarps];
  int32_t cutoff;
};

// A CTA's share of a row: whole 16-byte vectors (of the row's frame, which
// starts at the vector that holds its first logit), the first `cap` of them in
// shared memory.
template <typename T>
struct Share {
  const T* row;
  Vec<T>* held;
  int32_t shift;  // elements of the frame's first vector before the row
  int32_t V, first, end, cap;

  __device__ __forceinline__ int32_t index(int32_t v) const { return v * Vec<T>::N - shift; }
  __device__ __forceinline__ Vec<T> load(int32_t v) const {
    const int32_t i = index(v);
    Vec<T> x;
    if (i >= 0 && i + Vec<T>::N <= V) {
      *reinterpret_cast<uint4*>(&x) = ld_stream(reinterpret_cast<const uint4*>(row + i));
    } else {
#pragma unroll
      for (int e = 0; e < Vec<T>::N; ++e) x.e[e] = i + e >= 0 && i + e < V ? row[i + e] : lowest<T>();
    }
    return x;
  }
  __device__ __forceinline__ Vec<T> get(int32_t v) const { return v - first < cap ? held[v - first] : load(v); }
};

struct Weight {
  float m, T;
  __device__ __forceinline__ float log(float x) const { return T == 1.f ? x - m : (x - m) / T; }
  __device__ __forceinline__ float operator()(float x) const { return expf(log(x)); }
};

__device__ __forceinline__ float block_sum(float x, Shared& s) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  if ((threadIdx.x & 31) == 0) s.wf[threadIdx.x >> 5] = x;
  __syncthreads();
  float t = 0.f;
  for (int w = 0; w < kWarps; ++w) t += s.wf[w];
  __syncthreads();
  return t;
}

__device__ __forceinline__ Best block_best(Best b, Shared& s) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float v = __shfl_xor_sync(0xffffffffu, b.v, o);
    const int32_t i = __shfl_xor_sync(0xffffffffu, b.i, o);
    take(b, v, i);
  }
  if ((threadIdx.x & 31) == 0) s.wb[threadIdx.x >> 5] = b;
  __syncthreads();
  b = s.wb[0];
  for (int w = 1; w < kWarps; ++w) take(b, s.wb[w].v, s.wb[w].i);
  __syncthreads();
  return b;
}

// Exclusive prefix over the block of (c, m) in thread order; the totals in *tc, *tm.
__device__ __forceinline__ void block_scan(uint32_t& c, uint64_t& m, uint32_t* tc, uint64_t* tm, Shared& s) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t c0 = c;
  const uint64_t m0 = m;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t a = __shfl_up_sync(0xffffffffu, c, o);
    const uint64_t b = __shfl_up_sync(0xffffffffu, m, o);
    if (lane >= o) {
      c += a;
      m += b;
    }
  }
  if (lane == 31) {
    s.wc[warp] = c;
    s.wm[warp] = m;
  }
  __syncthreads();
  uint32_t bc = 0, t = 0;
  uint64_t bm = 0, u = 0;
  for (int w = 0; w < kWarps; ++w) {
    if (w == warp) {
      bc = t;
      bm = u;
    }
    t += s.wc[w];
    u += s.wm[w];
  }
  c += bc - c0;
  m += bm - m0;
  *tc = t;
  *tm = u;
  __syncthreads();
}

// Where a search ended: a key, the range's tokens that have it, and the count
// and mass of those above it.
struct Cut {
  uint32_t key, ties, above;
  uint64_t mass_above;
};

// The key in [lo, hi] at which the count (by_mass false) or the mass of the
// tokens from the largest down first reaches the target (at most the range's
// total: a larger target is lowered to it).
template <typename T>
__device__ Cut search(const Share<T>& sh, const Weight& weight, uint32_t lo, uint32_t hi, bool by_mass, uint64_t target, bool masses,
                      Shared& s, cg::cluster_group& cluster) {
  const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  uint32_t above = 0;
  uint64_t mass_above = 0;
  while (true) {
    int shift = 0;
    while (((hi - lo) >> shift) >= (uint32_t)kBins) ++shift;
    for (int b = threadIdx.x; b < kBins; b += kThreads) s.cnt[b] = s.lo[b] = s.hi[b] = 0;
    __syncthreads();
    for (int32_t v = sh.first + threadIdx.x; v < sh.end; v += kThreads) {
      const Vec<T> x = sh.get(v);
#pragma unroll
      for (int e = 0; e < Vec<T>::N; ++e) {
        const uint32_t k = Key<T>::of(x.e[e]);
        if (k < lo || k > hi) continue;
        const uint32_t b = (hi - k) >> shift;
        atomicAdd(&s.cnt[b], 1u);
        if (masses) {
          const float w = weight(widen(x.e[e])) * 256.f, whole = floorf(w);
          const uint32_t q = __float2uint_rz((w - whole) * 4294967296.f);
          const uint32_t old = atomicAdd(&s.lo[b], q);
          const uint32_t up = (uint32_t)whole + (old + q < old ? 1u : 0u);
          if (up) atomicAdd(&s.hi[b], up);
        }
      }
    }
    cluster.sync();
    // the cluster's sums of this CTA's slice of the bins, a run of them per thread
    const int slice = kBins / C, per = (slice + kThreads - 1) / kThreads, b0 = rank * slice + threadIdx.x * per;
    const bool mine = (int)threadIdx.x * per < slice;
    uint32_t c[kBins / kThreads];
    uint64_t m[kBins / kThreads];
    uint32_t tc = 0;
    uint64_t tm = 0;
    for (int j = 0; j < per; ++j) {
      c[j] = 0;
      m[j] = 0;
      if (mine)
        for (int r = 0; r < C; ++r) {
          const Shared* o = cluster.map_shared_rank(&s, r);
          c[j] += o->cnt[b0 + j];
          if (masses) m[j] += ((uint64_t)o->hi[b0 + j] << 32) + o->lo[b0 + j];
        }
      tc += c[j];
      tm += m[j];
    }
    uint32_t ec = tc, all_c;
    uint64_t em = tm, all_m;
    block_scan(ec, em, &all_c, &all_m, s);
    if (threadIdx.x == 0) {
      s.total_cnt = all_c;
      s.total_mass = all_m;
    }
    cluster.sync();
    uint64_t sum = by_mass ? mass_above : above, range = sum;
    for (int r = 0; r < C; ++r) {
      const Shared* o = cluster.map_shared_rank(&s, r);
      range += by_mass ? o->total_mass : o->total_cnt;
    }
    if (target > range) target = range;
    int owner = 0;
    uint32_t base_c = above;
    uint64_t base_m = mass_above;
    for (; owner < C - 1; ++owner) {
      const Shared* o = cluster.map_shared_rank(&s, owner);
      const uint64_t next = sum + (by_mass ? o->total_mass : o->total_cnt);
      if (next >= target) break;
      sum = next;
      base_c += o->total_cnt;
      base_m += o->total_mass;
    }
    if (rank == owner) {
      ec += base_c;
      em += base_m;
      for (int j = 0; j < per && mine; ++j) {
        const uint64_t before = by_mass ? em : ec, after = before + (by_mass ? m[j] : c[j]);
        if (before < target && after >= target) {
          s.found_bin = b0 + j;
          s.found_cnt = c[j];
          s.found_at = ec;
          s.found_mass = em;
        }
        ec += c[j];
        em += m[j];
      }
    }
    cluster.sync();
    const Shared* o = cluster.map_shared_rank(&s, owner);
    const uint32_t bin = o->found_bin;
    above = o->found_at;
    mass_above = o->found_mass;
    hi -= bin << shift;
    if (shift == 0) return {hi, o->found_cnt, above, mass_above};
    const uint32_t width = (1u << shift) - 1;
    if (hi - lo > width) lo = hi - width;
  }
}

// The index below which this share's tokens with the given key are kept, if the
// row's first `keep` of them (in order of index) are.
template <typename T>
__device__ int32_t tie_cutoff(const Share<T>& sh, uint32_t key, uint32_t keep, Shared& s, cg::cluster_group& cluster) {
  const auto tied = [&](const Vec<T>& x) {
    uint32_t n = 0;
#pragma unroll
    for (int e = 0; e < Vec<T>::N; ++e) n += Key<T>::of(x.e[e]) == key;
    return n;
  };
  uint32_t n = 0, own;
  uint64_t z = 0, zt;
  for (int32_t v = sh.first + threadIdx.x; v < sh.end; v += kThreads) n += tied(sh.get(v));
  block_scan(n, z, &own, &zt, s);
  if (threadIdx.x == 0) s.total_cnt = own;
  cluster.sync();
  uint32_t before = 0;
  for (int o = 0; o < (int)cluster.block_rank(); ++o) before += cluster.map_shared_rank(&s, o)->total_cnt;
  if (before >= keep) return -1;
  const uint32_t want = keep - before;
  if (own <= want) return INT32_MAX;
  uint32_t seen = 0;  // the want-th of this share is the last kept: a round covers consecutive vectors
  for (int32_t v0 = sh.first; seen < want; v0 += kThreads) {
    const int32_t v = v0 + threadIdx.x;
    Vec<T> x;
    uint32_t c = 0, all;
    if (v < sh.end) {
      x = sh.get(v);
      c = tied(x);
    }
    uint32_t at = c;
    z = 0;
    block_scan(at, z, &all, &zt, s);
    if (c && seen + at < want && seen + at + c >= want) {
      uint32_t left = want - seen - at;
#pragma unroll
      for (int e = 0; e < Vec<T>::N; ++e)
        if (Key<T>::of(x.e[e]) == key && --left == 0) s.cutoff = sh.index(v) + e + 1;
    }
    seen += all;
  }
  __syncthreads();
  return s.cutoff;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) sample_kernel(const SampleParams p, const int cap) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  extern __shared__ __align__(16) unsigned char dyn[];
  Shared& s = *reinterpret_cast<Shared*>(dyn);
  cg::cluster_group cluster = cg::this_cluster();
  const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int32_t r = blockIdx.x / C;
  constexpr int N = Vec<T>::N;

  Share<T> sh;
  sh.row = static_cast<const T*>(p.x) + (int64_t)r * p.ld;
  sh.held = reinterpret_cast<Vec<T>*>(dyn + ((sizeof(Shared) + 15) & ~(size_t)15));
  sh.shift = (int32_t)((reinterpret_cast<uintptr_t>(sh.row) & 15) / sizeof(T));
  sh.V = p.V;
  const int64_t vecs = ((int64_t)p.V + sh.shift + N - 1) / N;
  sh.first = (int32_t)(vecs * rank / C);
  sh.end = (int32_t)(vecs * (rank + 1) / C);
  sh.cap = cap;
  const float* noise = p.noise + (int64_t)r * p.ld_noise;
  const float temp = p.how.temperature ? __ldg(p.how.temperature + r) : p.how.temperature_all;
  const int32_t top_k = p.how.top_k ? __ldg(p.how.top_k + r) : p.how.top_k_all;
  const float top_p = p.how.top_p ? __ldg(p.how.top_p + r) : p.how.top_p_all;
  const float min_p = p.how.min_p ? __ldg(p.how.min_p + r) : p.how.min_p_all;  // (over 1: as 1)

  // the share into shared memory, and its largest logit
  Best top = {-INFINITY, INT32_MAX};
  bool bad = false;
  for (int32_t v0 = sh.first; v0 < sh.end; v0 += 4 * kThreads) {
    Vec<T> x[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int32_t v = v0 + u * kThreads + threadIdx.x;
      if (v < sh.end) x[u] = sh.load(v);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int32_t v = v0 + u * kThreads + threadIdx.x;
      if (v >= sh.end) continue;
      if (v - sh.first < cap) sh.held[v - sh.first] = x[u];
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float f = widen(x[u].e[e]);
        bad |= !(f < INFINITY);
        if (f > top.v) top = {f, sh.index(v) + e};
      }
    }
  }
  top = block_best(top, s);
  bad = __syncthreads_or(bad);
  if (threadIdx.x == 0) {
    s.top = top;
    s.bad = bad;
  }
  cluster.sync();
  for (int o = 0; o < C; ++o) {
    const Shared* t = cluster.map_shared_rank(&s, o);
    take(top, t->top.v, t->top.i);
    bad |= t->bad != 0;
  }
  const Weight weight = {top.v, temp};

  int32_t token = -1;
  float logp = NAN;
  const bool sound = !bad && top.v > -INFINITY && temp >= 0.f && temp < INFINITY && !isnan(top_p) && !isnan(min_p);
  if (!sound) {
    // no token
  } else if (temp == 0.f) {
    token = top.i;
    logp = 0.f;
  } else {
    // what is kept: keys above `key`, and of those at it the ones of index below `cutoff`
    const uint32_t none = Key<T>::of(lowest<T>()), first = Key<T>::of(static_cast<T>(top.v));
    uint32_t key = none;
    int32_t cutoff = 0;
    const bool cut_k = top_k > 0 && top_k < p.V, cut_p = top_p < 1.f;
    if (cut_k || cut_p) {
      constexpr double kOne = 1099511627776.0;  // 2^40, the fixed-point 1
      Cut cut = {none, 0, 0, 0};
      uint32_t ties = 0;  // of the tokens at the cut, the first so many are kept
      double mass = 0.0;
      if (cut_k) {  // (all tokens that are not ruled out, where those are fewer)
        cut = search(sh, weight, none + 1, first, false, (uint64_t)top_k, cut_p, s, cluster);
        ties = min((uint32_t)top_k - cut.above, cut.ties);
        mass = (double)cut.mass_above + kOne * ties * weight(Key<T>::value(cut.key));
      } else {
        float t = 0.f;
        for (int32_t v = sh.first + threadIdx.x; v < sh.end; v += kThreads) {
          const Vec<T> x = sh.get(v);
#pragma unroll
          for (int e = 0; e < N; ++e) t += weight(widen(x.e[e]));
        }
        t = block_sum(t, s);
        if (threadIdx.x == 0) s.sum = t;
        cluster.sync();
        for (int o = 0; o < C; ++o) mass += kOne * cluster.map_shared_rank(&s, o)->sum;
      }
      if (cut_p) {
        const double goal = fmax(ceil((double)top_p * mass), 1.0);
        const Cut by_mass = search(sh, weight, cut_k ? cut.key : none + 1, first, true, (uint64_t)goal, true, s, cluster);
        const uint32_t most = cut_k && by_mass.key == cut.key ? ties : by_mass.ties;
        const double one = fmax((double)weight(Key<T>::value(by_mass.key)) * kOne, 1.0);
        const double need = ceil((goal - (double)by_mass.mass_above) / one);
        ties = need < 1.0 ? 1u : need < (double)most ? (uint32_t)need : most;
        cut = by_mass;
      }
      key = cut.key;
      cutoff = INT32_MAX;
      if (ties < cut.ties) cutoff = tie_cutoff(sh, key, ties, s, cluster);
    }
    // the race
    const float least = fminf(min_p, 1.f);
    Best best = {-1.f, INT32_MAX};
    float kept = 0.f;
    for (int32_t v = sh.first + threadIdx.x; v < sh.end; v += kThreads) {
      const Vec<T> x = sh.get(v);
      const int32_t i0 = sh.index(v);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const uint32_t k = Key<T>::of(x.e[e]);
        if (k < key || (k == key && i0 + e >= cutoff)) continue;
        const float w = weight(widen(x.e[e]));
        if (w < least) continue;
        kept += w;
        take(best, w / __ldg(noise + i0 + e), i0 + e);
      }
    }
    best = block_best(best, s);
    kept = block_sum(kept, s);
    if (threadIdx.x == 0) {
      s.race = best;
      s.kept = kept;
    }
    cluster.sync();
    if (rank == 0 && threadIdx.x == 0) {
      float z = 0.f;
      for (int o = 0; o < C; ++o) {
        const Shared* t = cluster.map_shared_rank(&s, o);
        take(best, t->race.v, t->race.i);
        z += t->kept;
      }
      if (best.v > 0.f) {
        token = best.i;
        logp = weight.log(widen(sh.row[token])) - logf(z);
      }
    }
  }
  if (rank == 0 && threadIdx.x == 0) {
    p.tokens[r] = token;
    if (p.logp) p.logp[r] = logp;
    if (token < 0) set_status(p.dev_status, STRIDE_DEV_NO_TOKEN);
  }
  cluster.sync();  // no CTA leaves while another may read its shared memory
}

template <typename T>
cudaError_t run(const SampleParams& p, cudaStream_t stream) {
  int C = kMaxCluster;
  while (C > 1 && p.V < 2048 * C) C /= 2;
  const int64_t vecs = ((int64_t)p.V * sizeof(T) + 15) / 16 + 1;
  const int64_t share = (vecs + C - 1) / C + 1;
  const int64_t most = (220 * 1024 - (int64_t)sizeof(Shared) - 16) / 16;
  const int cap = (int)(share < most ? share : most);
  const size_t smem = ((sizeof(Shared) + 15) & ~(size_t)15) + (size_t)cap * 16;
  cudaError_t e = cudaFuncSetAttribute(sample_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((int64_t)p.rows * C));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = C;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  e = cudaLaunchKernelEx(&cfg, sample_kernel<T>, p, cap);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

cudaError_t launch_sample(const SampleParams& p, int dtype, int, cudaStream_t stream) {
  if (p.rows > INT32_MAX / kMaxCluster) return cudaErrorInvalidConfiguration;
  if (dtype == STRIDE_DTYPE_BF16) return run<__nv_bfloat16>(p, stream);
  if (dtype == STRIDE_DTYPE_F16) return run<__half>(p, stream);
  return run<float>(p, stream);
}

}  // namespace stride
