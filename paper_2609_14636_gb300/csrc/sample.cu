// sample.cu -- tokens from logits with temperature, top-k, top-p and min-p and
// given random numbers (sm_103a).
//
//   d_i = (x_i - max) / T, w_i = exp d_i; kept: the largest tokens (ties: lowest
//   index first) up to top_k, then up to top_p of their mass, then w >= min_p;
//   token = argmax over the kept of w_i / noise_i (an exponential race).
//
// A row is read from memory once, by a thread-block cluster whose CTAs keep
// their shares of it in shared memory.  Three ways from there:
// - nothing is cut off: the race is run while the row streams in, each thread's
//   ratios relative to the largest logit it has met;
// - what is kept lies among the few largest tokens (a top_k of up to some
//   hundreds; a top_p whose mass they hold): of groups of lanes each one's
//   largest logit is known from the load, and the R-th largest of those is a
//   bound that at least R tokens reach and few more do.  The tokens that reach it
//   go to the cluster's first CTA, which ranks them by (logit, index) and does the
//   rest on that list, while the other CTAs make room for the next rows;
// - else the threshold is found without sorting: a histogram over the ordered
//   bit patterns of the logits in the range that can hold it (counts for top-k,
//   masses for top-p), summed over the cluster, gives the bin where the running
//   count or mass crosses its target; that bin is the next range.  Masses are
//   fixed-point integers (2^-40 of the largest weight), so the atomics' order
//   changes nothing.  What is kept is all above the threshold and, at it, the
//   first few by index; one pass over the share races them.
// Noise is read for kept tokens alone.
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
constexpr int kBins = 1024;
constexpr int kLoads = 5;      // vectors that a thread has in flight while it loads its share
constexpr int kGroups = 1024;  // groups of lanes at most
constexpr int kList = 1024;    // tokens that the first CTA ranks at most
constexpr int kUsual = 96;     // groups that a top_p without top_k asks to reach the bound
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
  union {
    struct {
      uint32_t cnt[kBins], lo[kBins], hi[kBins];
    };
    struct {
      float group[kGroups];  // the largest logits of the cluster's groups
      uint64_t list[kList];  // (key, ~index) of the tokens that reach the bound; the first CTA's, ranked
    };
  };
  // exchanged with the cluster
  float own_group[kThreads];
  uint64_t pushed[kList];  // the first CTA's: the tokens, in one segment per CTA
  Best top[kWarps];        // of the warps
  int32_t bad;
  uint32_t listed[kMaxCluster];
  float sum_all[kMaxCluster], sum_listed[kMaxCluster];
  float sum;
  uint32_t total_cnt;
  uint64_t total_mass;
  uint32_t found_bin, found_cnt, found_at;  // the crossing bin, its count, the count above it
  uint64_t found_mass;                      // the mass above it
  Best race[kMaxCluster];                   // the first CTA's
  float kept[kMaxCluster], largest[kMaxCluster];
  // of the CTA
  Best wb[kWarps];
  float wf[kWarps];
  uint32_t wc[kWarps];
  uint64_t wm[kWarps];
  int32_t cutoff;
  uint32_t count;
  float bound;
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
    uint32_t c[(kBins + kThreads - 1) / kThreads];
    uint64_t m[(kBins + kThreads - 1) / kThreads];
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

// A remote CTA's copy of a member of Shared.
template <typename M>
__device__ __forceinline__ M* at_rank(M* p, int rank, cg::cluster_group& cluster) {
  return cluster.map_shared_rank(p, rank);
}

// The noise of a vector's tokens (1 where there is no token).
template <int N>
__device__ __forceinline__ void load_noise(float (&e)[N], const float* noise, int32_t i, int32_t V, bool whole) {
  if (whole && i >= 0 && i + N <= V) {
#pragma unroll
    for (int x = 0; x < N; x += 4) {
      const uint4 u = ld_stream(reinterpret_cast<const uint4*>(noise + i + x));
      e[x] = __uint_as_float(u.x);
      e[x + 1] = __uint_as_float(u.y);
      e[x + 2] = __uint_as_float(u.z);
      e[x + 3] = __uint_as_float(u.w);
    }
  } else {
#pragma unroll
    for (int x = 0; x < N; ++x) e[x] = i + x >= 0 && i + x < V ? __ldg(noise + i + x) : 1.f;
  }
}

// Nothing is cut off: one pass over logits and noise together.  A thread keeps
// its largest logit m, sum exp((x - m) / T) and its best ratio exp((x - m) / T) /
// noise, rescaled where m grows.  Exponentials and quotients on the way are the
// approximate ones (2^-22); the threads' best that come within 1e-5 of the largest
// then race again with exact ones.
template <typename T>
__device__ void race_all(const SampleParams& p, const Share<T>& sh, const float* noise, float temp, int32_t r, Shared& s,
                         cg::cluster_group& cluster) {
  constexpr int N = Vec<T>::N, U = N == 8 ? 2 : 4;
  const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank(), tid = threadIdx.x;
  const float scale = kLog2e / temp;
  const bool whole = (reinterpret_cast<uintptr_t>(noise + sh.index(0)) & 15) == 0;
  Best best = {-1.f, INT32_MAX};
  float m = -INFINITY, z = 0.f;
  bool bad = false;
  for (int32_t v0 = sh.first; v0 < sh.end; v0 += U * kThreads) {
    Vec<T> x[U];
    float e[U][N];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int32_t v = v0 + u * kThreads + tid;
      if (v < sh.end) {
        x[u] = sh.load(v);
        load_noise<N>(e[u], noise, sh.index(v), sh.V, whole);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int32_t v = v0 + u * kThreads + tid;
      if (v >= sh.end) continue;
      float f[N], mx = m;
#pragma unroll
      for (int k = 0; k < N; ++k) {
        f[k] = widen(x[u].e[k]);
        bad |= !(f[k] < INFINITY);
        mx = fmaxf(mx, f[k]);
      }
      if (mx > m) {
        const float by = ex2((m - mx) * scale);
        z *= by;
        if (best.v < INFINITY) best.v *= by;  // (a thread without a token has -1 or -0: still no ratio)
        m = mx;
      }
      if (m == -INFINITY) continue;
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const float w = ex2((f[k] - m) * scale);
        z += w;
        const float q = __fdividef(w, e[u][k]);
        if (q > best.v && w > 0.f) best = {q, sh.index(v) + k};
      }
    }
  }
  // the row's largest logit, then everything relative to it
  float top = m;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  if ((tid & 31) == 0) s.wf[tid >> 5] = top;
  bad = __syncthreads_or(bad);
  for (int w = 0; w < kWarps; ++w) top = fmaxf(top, s.wf[w]);
  if (tid == 0) {
    s.sum = top;
    s.bad = bad;
  }
  cluster.sync();
  for (int o = 0; o < C; ++o) {
    top = fmaxf(top, *at_rank(&s.sum, o, cluster));
    bad |= *at_rank(&s.bad, o, cluster) != 0;
  }
  const float by = m == -INFINITY ? 0.f : ex2((m - top) * scale);
  z = block_sum(z * by, s);
  if (best.i == INT32_MAX)
    best.v = -1.f;
  else if (best.v < INFINITY)
    best.v *= by;
  const Best lead = block_best(best, s);
  // (the CTA's near-best race exactly; those of a CTA that is not near the row's best lose either way)
  const Weight weight = {top, temp};
  Best exact = {-1.f, INT32_MAX};
  if (best.i != INT32_MAX && best.v >= lead.v * 0.99999f)
    exact = {best.v < INFINITY ? weight(widen(sh.row[best.i])) / __ldg(noise + best.i) : INFINITY, best.i};
  exact = block_best(exact, s);
  if (tid == 0) {
    *at_rank(&s.race[rank], 0, cluster) = exact;
    *at_rank(&s.kept[rank], 0, cluster) = z;
  }
  cluster.sync();
  if (rank == 0 && tid == 0) {
    z = 0.f;
    for (int o = 0; o < C; ++o) {
      take(exact, s.race[o].v, s.race[o].i);
      z += s.kept[o];
    }
    const bool found = !bad && exact.v > 0.f && exact.i != INT32_MAX;
    p.tokens[r] = found ? exact.i : -1;
    if (p.logp) p.logp[r] = found ? weight.log(widen(sh.row[exact.i])) - logf(z) : NAN;
    if (!found) set_status(p.dev_status, STRIDE_DEV_NO_TOKEN);
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) sample_kernel(const SampleParams p, const int cap) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  extern __shared__ __align__(16) unsigned char dyn[];
  Shared& s = *reinterpret_cast<Shared*>(dyn);
  cg::cluster_group cluster = cg::this_cluster();
  const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
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
  const float min_p = p.how.min_p ? __ldg(p.how.min_p + r) : p.how.min_p_all;
  const bool cut_k = top_k > 0 && top_k < p.V, cut_p = top_p < 1.f;
  const bool params = temp >= 0.f && temp < INFINITY && !isnan(top_p) && !isnan(min_p);

  if (params && temp > 0.f && !cut_k && !cut_p && min_p <= 0.f) {
    race_all(p, sh, noise, temp, r, s, cluster);
    return;
  }

  // the share into shared memory, and its largest logits
  Best top = {-INFINITY, INT32_MAX};
  bool bad = false;
  for (int32_t v0 = sh.first; v0 < sh.end; v0 += kLoads * kThreads) {
    Vec<T> x[kLoads];
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int32_t v = v0 + u * kThreads + tid;
      if (v < sh.end) x[u] = sh.load(v);
    }
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int32_t v = v0 + u * kThreads + tid;
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
  const float own_top = top.v;
  // groups of `per` lanes: at least 128 of them, and a third more than the bound asks for
  const uint32_t reach = cut_k ? (uint32_t)top_k : (uint32_t)kUsual;
  int per = 32;
  while (per > 1 && (uint32_t)(C * kThreads / per) < max(reach + reach / 3, 128u)) per /= 2;
  const int groups = C * kThreads / per, own_groups = kThreads / per;
  const bool by_list = (cut_k || cut_p) && groups <= kGroups && (uint32_t)groups >= reach;
  Best b = top;
  for (int o = 1; o < 32; o <<= 1) {
    if (by_list && o == per && lane % per == 0) s.own_group[tid / per] = b.v;
    const float v = __shfl_xor_sync(0xffffffffu, b.v, o);
    const int32_t i = __shfl_xor_sync(0xffffffffu, b.i, o);
    take(b, v, i);
  }
  if (by_list && per == 32 && lane == 0) s.own_group[warp] = b.v;
  if (lane == 0) s.top[warp] = b;
  if (tid == 0) s.count = 0;
  bad = __syncthreads_or(bad);
  if (tid == 0) s.bad = bad;
  cluster.sync();
  // every warp reads all warps' best
  bool any_bad = false;
  top = {-INFINITY, INT32_MAX};
  for (int j = lane; j < C * kWarps; j += 32) {
    const Best o = *at_rank(&s.top[j % kWarps], j / kWarps, cluster);
    take(top, o.v, o.i);
  }
  if (lane < C) any_bad = *at_rank(&s.bad, lane, cluster) != 0;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float v = __shfl_xor_sync(0xffffffffu, top.v, o);
    const int32_t i = __shfl_xor_sync(0xffffffffu, top.i, o);
    take(top, v, i);
  }
  any_bad = __any_sync(0xffffffffu, any_bad);
  const Weight weight = {top.v, temp};

  const auto answer = [&](int32_t token, float logp) {
    p.tokens[r] = token;
    if (p.logp) p.logp[r] = logp;
    if (token < 0) set_status(p.dev_status, STRIDE_DEV_NO_TOKEN);
  };
  const bool sound = !any_bad && top.v > -INFINITY && params;
  if (!sound || temp == 0.f) {
    if (rank == 0 && tid == 0) answer(sound ? top.i : -1, sound ? 0.f : NAN);
    cluster.sync();  // no CTA leaves while another may read its shared memory
    return;
  }
  const float least = fminf(min_p, 1.f);
  const uint32_t none = Key<T>::of(lowest<T>()), first = Key<T>::of(static_cast<T>(top.v));

  if (by_list) {
    for (int j = tid; j < groups; j += kThreads) s.group[j] = *at_rank(&s.own_group[j % own_groups], j / own_groups, cluster);
    __syncthreads();
    // the bound: the smallest of them that fewer than `reach` exceed
    for (int j = tid; j < groups; j += kThreads) {
      const float f = s.group[j];
      uint32_t greater = 0, equal_before = 0;
      for (int k = 0; k < groups; ++k) {
        greater += s.group[k] > f;
        equal_before += s.group[k] == f && k < j;
      }
      if (greater + equal_before == reach - 1) s.bound = f;
    }
    __syncthreads();
    const float bound = s.bound;
    float all = 0.f, listed = 0.f;
    const bool need_all = !cut_k;
    if (need_all || own_top >= bound) {
      for (int32_t v = sh.first + tid; v < sh.end; v += kThreads) {
        const Vec<T> x = sh.get(v);
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const float f = widen(x.e[e]);
          const float w = need_all ? weight(f) : 0.f;
          all += w;
          if (f >= bound && f > -INFINITY) {
            listed += w;
            const uint32_t at = atomicAdd(&s.count, 1u);
            if (at < kList) s.list[at] = (uint64_t)Key<T>::of(x.e[e]) << 32 | (uint32_t)~(sh.index(v) + e);
          }
        }
      }
    }
    if (need_all) {
      all = block_sum(all, s);
      listed = block_sum(listed, s);
    } else {
      __syncthreads();
    }
    const uint32_t n_own = s.count, segment = kList / C;
    for (uint32_t j = tid; j < min(n_own, segment); j += kThreads) *at_rank(&s.pushed[rank * segment + j], 0, cluster) = s.list[j];
    if (tid < C) {
      *at_rank(&s.listed[rank], tid, cluster) = n_own;
      *at_rank(&s.sum_all[rank], tid, cluster) = all;
      *at_rank(&s.sum_listed[rank], tid, cluster) = listed;
    }
    cluster.sync();
    bool held = true;
    uint32_t n = 0;
    float z = 0.f, zl = 0.f;
    for (int o = 0; o < C; ++o) {
      held = held && s.listed[o] <= segment;
      n += s.listed[o];
      z += s.sum_all[o];
      zl += s.sum_listed[o];
    }
    // the list holds what is kept: top_k of the largest; or more than top_p of the mass, or all of w >= min_p
    if (held && (cut_k || zl > top_p * z * 1.00001f || weight(bound) < least)) {
      if (rank == 0) {
        for (uint32_t j = tid; j < n; j += kThreads) {
          uint32_t o = 0, k = j;
          while (k >= s.listed[o]) k -= s.listed[o++];
          s.list[j] = s.pushed[o * segment + k];
        }
        __syncthreads();
        // ranks by (logit, index): at most kList / kThreads tokens a thread
        uint64_t mine[kList / kThreads];
        uint32_t place[kList / kThreads];
#pragma unroll
        for (int u = 0; u < kList / kThreads; ++u) {
          const uint32_t j = tid + u * kThreads;
          place[u] = 0;
          if (j < n) {
            mine[u] = s.list[j];
            for (uint32_t k = 0; k < n; ++k) place[u] += s.list[k] > mine[u];
          }
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kList / kThreads; ++u)
          if (tid + u * kThreads < n) s.list[place[u]] = mine[u];
        __syncthreads();
        constexpr int kPer = kList / kThreads;  // consecutive ranks of a thread
        const uint32_t kept_k = cut_k ? min((uint32_t)top_k, n) : n;
        float w[kPer], e[kPer], mass = 0.f;
        int32_t idx[kPer];
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
          const uint32_t j = tid * kPer + u;
          w[u] = 0.f;
          e[u] = 1.f;
          if (j < kept_k) {
            const uint64_t q = s.list[j];
            idx[u] = (int32_t)~(uint32_t)q;
            e[u] = __ldg(noise + idx[u]);
            w[u] = weight(Key<T>::value((uint32_t)(q >> 32)));
          }
          mass += w[u];
        }
        // the mass before each thread's first token
        float before = mass;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const float v = __shfl_up_sync(0xffffffffu, before, o);
          if (lane >= o) before += v;
        }
        if (lane == 31) s.wf[warp] = before;
        before -= mass;
        __syncthreads();
        float total = 0.f;
        for (int k = 0; k < kWarps; ++k) {
          if (k == warp) before += total;
          total += s.wf[k];
        }
        __syncthreads();
        const float goal = top_p * (cut_k ? total : z);
        Best best = {-1.f, INT32_MAX};
        float kept = 0.f;
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
          const uint32_t j = tid * kPer + u;
          if (j < kept_k && (!cut_p || j == 0 || before < goal) && w[u] >= least) {
            kept += w[u];
            take(best, w[u] / e[u], idx[u]);
          }
          before += w[u];
        }
        best = block_best(best, s);
        kept = block_sum(kept, s);
        if (tid == 0) {
          if (best.v > 0.f)
            answer(best.i, weight.log(widen(sh.row[best.i])) - logf(kept));
          else
            answer(-1, NAN);
        }
      }
      return;  // (nothing of another CTA is read after the last cluster.sync)
    }
    cluster.sync();  // s.list and s.group make room for the histogram
  }

  // what is kept: keys above `key`, and of those at it the ones of index below `cutoff`
  uint32_t key = none;
  int32_t cutoff = 0;
  if (cut_k || cut_p) {
    constexpr double kOne = 1099511627776.0;  // 2^40, the fixed-point 1
    Cut cut = {none, 0, 0, 0};
    uint32_t ties = 0;  // of the tokens at the cut, the first so many are kept
    uint32_t from = none + 1;
    double mass = 0.0;
    if (cut_k) {  // (all tokens that are not ruled out, where those are fewer)
      cut = search(sh, weight, from, first, false, (uint64_t)top_k, cut_p, s, cluster);
      ties = min((uint32_t)top_k - cut.above, cut.ties);
      mass = (double)cut.mass_above + kOne * ties * weight(Key<T>::value(cut.key));
      from = cut.key;
    } else {
      float t = 0.f;
      for (int32_t v = sh.first + tid; v < sh.end; v += kThreads) {
        const Vec<T> x = sh.get(v);
#pragma unroll
        for (int e = 0; e < N; ++e) t += weight(widen(x.e[e]));
      }
      t = block_sum(t, s);
      if (tid == 0) s.sum = t;
      cluster.sync();
      double z = 0.0;
      for (int o = 0; o < C; ++o) z += *at_rank(&s.sum, o, cluster);
      mass = kOne * z;
      // The tokens of w < (1 - top_p) z / (2 V) hold less than half of what may be left out: none of them is needed.
      const float low = top.v + temp * logf(fmaxf((1.f - fmaxf(top_p, 0.f)) * (float)z / (2.f * (float)p.V), 1e-30f));
      const uint32_t k = Key<T>::of(static_cast<T>(fmaxf(low, -1e30f)));
      if (k > from + 1 && k <= first) from = k - 1;  // (a step below: the conversion may have rounded up)
    }
    if (cut_p) {
      const double goal = fmax(ceil((double)top_p * mass), 1.0);
      const Cut by_mass = search(sh, weight, from, first, true, (uint64_t)goal, true, s, cluster);
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
  Best best = {-1.f, INT32_MAX};
  float kept = 0.f;
  for (int32_t v = sh.first + tid; v < sh.end; v += kThreads) {
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
  if (tid == 0) {
    *at_rank(&s.race[rank], 0, cluster) = best;
    *at_rank(&s.kept[rank], 0, cluster) = kept;
  }
  cluster.sync();
  if (rank == 0 && tid == 0) {
    float z = 0.f;
    for (int o = 0; o < C; ++o) {
      take(best, s.race[o].v, s.race[o].i);
      z += s.kept[o];
    }
    if (best.v > 0.f)
      answer(best.i, weight.log(widen(sh.row[best.i])) - logf(z));
    else
      answer(-1, NAN);
  }
}

template <typename T>
cudaError_t run(const SampleParams& p, cudaStream_t stream) {
  int C = kMaxCluster;
  while (C > 1 && p.V < 4096 * C) C /= 2;
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
