// sample.cu -- tokens from logits with temperature, top-k, top-p and min-p and
// given random numbers (sm_103a).
//
//   d_i = (x_i - max) / T, w_i = exp d_i; kept: the largest tokens (ties: lowest
//   index first) up to top_k, then up to top_p of their mass, then w >= min_p;
//   token = argmax over the kept of w_i / noise_i (an exponential race).
//
// A row belongs to a thread-block cluster of 1 to 8 CTAs, each of which takes a
// share of it (run() below says how many).  The row comes from memory once;
// what is read again comes from L2.  Three ways:
// - nothing is cut off: the race is run while the row streams in, each thread's
//   ratios relative to the largest logit it has met;
// - what is kept lies among the few largest tokens (a top_k of up to some
//   hundreds; a top_p whose mass they hold): the first pass leaves each thread's
//   largest logit (and the sum of weights, for a top_p of the whole row); of
//   groups of threads, the R-th largest of their maxima is a bound that at least R
//   tokens reach and few more do.  The threads that reach it look their tokens
//   up again, and send those to the cluster's first CTA, which sorts them by
//   (logit, index) and does the rest on that list, while the other CTAs make room
//   for the next rows;
// - else the last kept token is bracketed, for a count by a histogram of the
//   logits by their distance from the largest, for a mass by the masses above a
//   few pivots, three times (sums in registers: an atomic sum per token of the tail
//   took 25 us a row where this takes 5); the tokens of the bracket are sorted as
//   above, and the last kept one is found among them.  Where they are too many for
//   that (ties), the threshold is found by histograms over the ordered bit
//   patterns, each level the next one's range, and the ties kept at it by
//   counting.  One more pass races what is kept.
//   All sums that atomics make are integers: their order changes nothing.
// Noise is read for kept tokens alone.  GB300, rows of 151,936 bf16 logits: one row
// with a top_k of 20 and a top_p 9.2 us; 256 with a top_k of 50 37 (2.1 TB/s); 256 of
// mixed parameters 92; 256 with a top_p alone 233; 512 uncut rows of 32,000 fp32 45
// (2.9 TB/s).
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <float.h>
#include <math.h>

#include "decode_internal.h"
#include "stride_device.cuh"

namespace cg = cooperative_groups;

namespace stride {
namespace {

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kBins = 1024;
constexpr int kLoads = 6;      // vectors that a thread has in flight
constexpr int kDepth = 6;
constexpr int kGroups = 1024;  // groups of threads at most
constexpr int kList = 1024;    // tokens that the first CTA sorts at most
constexpr float kOne = 1099511627776.f;  // 2^40, the fixed-point 1 of masses (weights are at most 1)
static_assert((uint64_t)STRIDE_MAX_TOP_P_VOCAB << 40 <= (uint64_t)1 << 63, "a row's mass fits in 64 bits, with room for rounding");
constexpr int kPivots = 7;
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

struct Pick {  // the last kept token, by falling key and rising index
  uint32_t key;
  int32_t i;
};

struct Found {  // where a search's target falls: a bin, its count, the count and the mass above it
  uint32_t bin, cnt, above, pad;
  uint64_t mass_above;
};

struct Shared {
  union {
    struct {
      uint32_t cnt[kBins], lo[kBins], hi[kBins];
    };
    uint64_t list[kList];  // (key, ~index) of the tokens that reach the bound; the first CTA's, sorted
  };
  // exchanged with the cluster
  float own_group[kThreads];
  uint64_t pushed[kList];  // the first CTA's: the tokens, in one segment per CTA
  float top;
  uint32_t listed[kMaxCluster];
  float sum_all[kMaxCluster], sum_listed[kMaxCluster];
  int32_t lowest[kMaxCluster];
  uint32_t total_cnt[kMaxCluster];  // of the CTAs' slices of a histogram
  uint64_t total_mass[kMaxCluster];
  Found found;
  Best race[kMaxCluster];                   // the first CTA's
  float kept[kMaxCluster];
  // of the CTA
  Best wb[kWarps];
  float wf[kWarps];
  uint32_t wc[kWarps];
  uint64_t wm[kWarps];
  int32_t cutoff;
  uint32_t count, bound;
  int32_t first_row;
  Pick pick;
  float pivot[kMaxCluster][kPivots], part[kWarps][kPivots];
};

// The CTA's.  (A function called out of line that had it as an argument would
// make its atomics generic ones, an order of magnitude slower.)
__device__ __forceinline__ Shared& shared() {
  __shared__ Shared s;
  return s;
}

// Whether a token of a row comes no later than the last kept one.
__device__ __forceinline__ bool kept_by(const Pick& last, uint32_t key, int32_t i) { return key > last.key || (key == last.key && i <= last.i); }


// A CTA's share of a row: whole 16-byte vectors of the row's frame, which starts
// at the vector that holds its first logit.
template <typename T>
struct Share {
  const T* row;
  int32_t shift;  // elements of the frame's first vector before the row
  int32_t V, first, end;

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
  // f(v, x) for this thread's vectors, U of them in flight.
  template <int U, typename F>
  __device__ __forceinline__ void each(F&& f) const {
    for (int32_t v0 = first + threadIdx.x; v0 < end; v0 += U * kThreads) {
      Vec<T> x[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (v0 + u * kThreads < end) x[u] = load(v0 + u * kThreads);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (v0 + u * kThreads < end) f(v0 + u * kThreads, x[u]);
    }
  }
  // The same with kDepth of them on their way through shared memory: one copy of
  // f's code, for passes that do more than a few operations a token.
  template <typename F>
  __device__ __forceinline__ void stream(F&& f) const {
    extern __shared__ uint4 ring[];  // [kDepth][kThreads], each thread its own
    uint4* slot = ring + threadIdx.x;
    int32_t ahead = first + threadIdx.x;
    const auto ask = [&](int k) {
      if (ahead < end) {
        const int32_t i = index(ahead);
        if (i >= 0 && i + Vec<T>::N <= V) {
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(slot + k * kThreads)), "l"(row + i)
                       : "memory");
        } else {
          const Vec<T> x = load(ahead);
          slot[k * kThreads] = *reinterpret_cast<const uint4*>(&x);
        }
        ahead += kThreads;
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll 1
    for (int k = 0; k < kDepth; ++k) ask(k);
    int k = 0;
#pragma unroll 1
    for (int32_t v = first + threadIdx.x; v < end; v += kThreads) {
      asm volatile("cp.async.wait_group %0;" ::"n"(kDepth - 1) : "memory");
      const uint4 u = slot[k * kThreads];
      f(v, *reinterpret_cast<const Vec<T>*>(&u));
      ask(k);
      k = k + 1 == kDepth ? 0 : k + 1;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
  }
  // f(v, x) for the vectors of the warp's threads that want them: the warp takes
  // a few such threads' vectors together, one per lane, so that it waits for
  // memory once.
  template <typename F>
  __device__ __forceinline__ void each_of(bool wanted, F&& f) const {
    unsigned who = __ballot_sync(0xffffffffu, wanted);
    if (__popc(who) > 8) {
      if (wanted) stream(f);
      return;
    }
    const int lane = threadIdx.x & 31;
    const int32_t base = first + (int32_t)(threadIdx.x - lane), stride = 32 * kThreads;
    // the next vector is on its way while one is looked at
    int32_t v = 0, next = 0;
    Vec<T> x, xn;
    bool have = false;
    for (; who; who &= who - 1)
      for (int32_t v0 = base + __ffs(who) - 1; v0 < end; v0 += stride) {
        next = v0 + lane * kThreads;
        if (next < end) xn = load(next);
        if (have && v < end) f(v, x);
        v = next;
        x = xn;
        have = true;
      }
    if (have && v < end) f(v, x);
  }
};

// The larger, or NaN if one is.
__device__ __forceinline__ float max_nan(float a, float b) {
  float c;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(c) : "f"(a), "f"(b));
  return c;
}
__device__ __forceinline__ float vec_max(const Vec<float>& x) { return max_nan(max_nan(x.e[0], x.e[1]), max_nan(x.e[2], x.e[3])); }
template <typename P>
__device__ __forceinline__ float pair_max(const uint4& u, P) {
  const P* h = reinterpret_cast<const P*>(&u);
  const P m = __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3]));
  return max_nan(widen(m.x), widen(m.y));
}
__device__ __forceinline__ float vec_max(const Vec<__nv_bfloat16>& x) { return pair_max(*reinterpret_cast<const uint4*>(&x), __nv_bfloat162()); }
__device__ __forceinline__ float vec_max(const Vec<__half>& x) { return pair_max(*reinterpret_cast<const uint4*>(&x), __half2()); }

// Element e of a vector (e not known when compiled).
__device__ __forceinline__ float pick(const Vec<float>& x, int e) {
  const float a = e & 1 ? x.e[1] : x.e[0], b = e & 1 ? x.e[3] : x.e[2];
  return e & 2 ? b : a;
}
template <typename T>
__device__ __forceinline__ T pick(const Vec<T>& x, int e) {
  const uint4 u = *reinterpret_cast<const uint4*>(&x);
  const uint32_t a = e & 2 ? u.y : u.x, b = e & 2 ? u.w : u.z, w = e & 4 ? b : a;
  const uint16_t h = (uint16_t)(e & 1 ? w >> 16 : w & 0xffffu);
  return *reinterpret_cast<const T*>(&h);
}

// does(x, e) for a vector's elements that are(x, e): what few elements need is
// written, and stands in the instruction cache, once.
template <typename T, typename P, typename F>
__device__ __forceinline__ void visit(const Vec<T>& x, P&& are, F&& does) {
  unsigned in = 0;
#pragma unroll
  for (int e = 0; e < Vec<T>::N; ++e)
    if (are(x.e[e], e)) in |= 1u << e;
  for (; in; in &= in - 1) {
    const int e = __ffs(in) - 1;
    does(pick(x, e), e);
  }
}

struct Weight {
  float m, T;
  __device__ __forceinline__ float log(float x) const { return T == 1.f ? x - m : (x - m) / T; }
  __device__ __forceinline__ float operator()(float x) const { return expf(log(x)); }
};

// What a difference of logits is multiplied with for an exponent of 2.  (Below a temperature of 2^-127 the quotient is infinite,
// and times a difference of 0 not a number: the largest finite one leaves the largest logits alone as well.)
__device__ __forceinline__ float exponent_scale(float T) { return fminf(kLog2e / T, FLT_MAX); }

__device__ __forceinline__ float block_sum(float x) {
  Shared& s = shared();
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  if ((threadIdx.x & 31) == 0) s.wf[threadIdx.x >> 5] = x;
  __syncthreads();
  float t = 0.f;
  for (int w = 0; w < kWarps; ++w) t += s.wf[w];
  __syncthreads();
  return t;
}

__device__ __forceinline__ Best block_best(Best b) {
  Shared& s = shared();
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
__device__ __forceinline__ void block_scan(uint32_t& c, uint64_t& m, uint32_t* tc, uint64_t* tm) {
  Shared& s = shared();
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

// A remote CTA's copy of a member of Shared.
template <typename M>
__device__ __forceinline__ M* at_rank(M* p, int rank, cg::cluster_group& cluster) {
  return cluster.map_shared_rank(p, rank);
}

// The bin of the cluster's summed histograms at which the running count or mass,
// from `above` and `mass_above` on, first reaches the target (lowered to the
// total where that is less).  mass_of(bin, count, sum of lo and hi): a bin's mass.
template <typename F>
__device__ __forceinline__ Found crossing(uint32_t above, uint64_t mass_above, bool by_mass, bool masses, uint64_t& target, cg::cluster_group& cluster, F&& mass_of) {
  Shared& s = shared();
  constexpr int kPer = (kBins + kThreads - 1) / kThreads;
  const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  cluster.sync();
  // this CTA's slice of the bins, a run of them per thread
  const int slice = kBins / C, per = (slice + kThreads - 1) / kThreads, b0 = rank * slice + threadIdx.x * per;
  const bool mine = (int)threadIdx.x * per < slice;
  uint32_t c[kPer], tc = 0;
  uint64_t m[kPer], tm = 0;
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    c[j] = 0;
    m[j] = 0;
    if (mine && j < per) {  // (the CTAs' parts asked for together)
      uint32_t pc[kMaxCluster], pl[kMaxCluster], ph[kMaxCluster];
#pragma unroll
      for (int r = 0; r < kMaxCluster; ++r) {
        const Shared* o = cluster.map_shared_rank(&s, r < C ? r : 0);
        pc[r] = r < C ? o->cnt[b0 + j] : 0u;
        pl[r] = masses && r < C ? o->lo[b0 + j] : 0u;
        ph[r] = masses && r < C ? o->hi[b0 + j] : 0u;
      }
#pragma unroll
      for (int r = 0; r < kMaxCluster; ++r) {
        c[j] += pc[r];
        m[j] += ((uint64_t)ph[r] << 32) + pl[r];
      }
      m[j] = masses && c[j] ? mass_of((uint32_t)(b0 + j), c[j], m[j]) : 0;
    }
    tc += c[j];
    tm += m[j];
  }
  uint32_t ec = tc, all_c;
  uint64_t em = tm, all_m;
  block_scan(ec, em, &all_c, &all_m);
  if (threadIdx.x < C) {
    *at_rank(&s.total_cnt[rank], threadIdx.x, cluster) = all_c;
    *at_rank(&s.total_mass[rank], threadIdx.x, cluster) = all_m;
  }
  cluster.sync();
  uint64_t sum = by_mass ? mass_above : above, range = sum;
  for (int r = 0; r < C; ++r) range += by_mass ? s.total_mass[r] : s.total_cnt[r];
  if (target > range) target = range;
  int owner = 0;
  uint32_t base_c = above;
  uint64_t base_m = mass_above;
  for (; owner < C - 1; ++owner) {
    const uint64_t next = sum + (by_mass ? s.total_mass[owner] : s.total_cnt[owner]);
    if (next >= target) break;
    sum = next;
    base_c += s.total_cnt[owner];
    base_m += s.total_mass[owner];
  }
  if (rank == owner) {
    ec += base_c;
    em += base_m;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const uint64_t before = by_mass ? em : ec, after = before + (by_mass ? m[j] : c[j]);
      if (before < target && after >= target) {
        const Found f = {(uint32_t)(b0 + j), c[j], ec, 0, em};
        for (int r = 0; r < C; ++r) *at_rank(&s.found, r, cluster) = f;
      }
      ec += c[j];
      em += m[j];
    }
  }
  cluster.sync();
  return s.found;
}

// Where a search ended: a key, the range's tokens that have it, and the count
// and mass of those above it.
struct Cut {
  uint32_t key, ties, above;
  uint64_t mass_above;
};

// The key in [lo, hi] at which the count (by_mass false) or the mass of the
// tokens from the largest down first reaches the target (at most the range's
// total: a larger target is lowered to it), of tokens up to `last` alone.  own:
// the key of this thread's largest logit.
template <typename T>
__device__ Cut search(const Share<T>& sh, const Weight& weight, const Pick& last, uint32_t own, uint32_t lo, uint32_t hi, bool by_mass, uint64_t target, bool masses,
                      cg::cluster_group& cluster) {
  Shared& s = shared();
  uint32_t above = 0;
  uint64_t mass_above = 0;
  while (true) {
    int shift = 0;
    while (((hi - lo) >> shift) >= (uint32_t)kBins) ++shift;
    for (int b = threadIdx.x; b < kBins; b += kThreads) s.cnt[b] = s.lo[b] = s.hi[b] = 0;
    __syncthreads();
    sh.each_of(own >= lo, [&](int32_t v, const Vec<T>& x) {
      visit(
          x, [&](T y, int e) { const uint32_t k = Key<T>::of(y); return k >= lo && k <= hi && kept_by(last, k, sh.index(v) + e); },
          [&](T y, int) {
            const uint32_t b = (hi - Key<T>::of(y)) >> shift;
            atomicAdd(&s.cnt[b], 1u);
            if (masses && shift > 0) {  // (in a bin of one key all weigh the same)
              const float w = weight(widen(y)) * 256.f, whole = floorf(w);
              const uint32_t q = __float2uint_rz((w - whole) * 4294967296.f);
              const uint32_t old = atomicAdd(&s.lo[b], q);
              const uint32_t up = (uint32_t)whole + (old + q < old ? 1u : 0u);
              if (up) atomicAdd(&s.hi[b], up);
            }
          });
    });
    const Found f = crossing(above, mass_above, by_mass, masses, target, cluster, [&](uint32_t b, uint32_t c, uint64_t q) {
      return shift > 0 ? q : c * (uint64_t)(weight(Key<T>::value(hi - b)) * kOne);
    });
    above = f.above;
    mass_above = f.mass_above;
    hi -= f.bin << shift;
    if (shift == 0) return {hi, f.cnt, above, mass_above};
    const uint32_t width = (1u << shift) - 1;
    if (hi - lo > width) lo = hi - width;
  }
}

// The index below which this share's tokens with the given key are kept, if the
// row's first `keep` of them (in order of index) are.
template <typename T>
__device__ int32_t tie_cutoff(const Share<T>& sh, uint32_t own_key, uint32_t key, uint32_t keep, cg::cluster_group& cluster) {
  Shared& s = shared();
  const auto tied = [&](const Vec<T>& x) {
    uint32_t n = 0;
#pragma unroll
    for (int e = 0; e < Vec<T>::N; ++e) n += Key<T>::of(x.e[e]) == key;
    return n;
  };
  uint32_t n = 0, own;
  uint64_t z = 0, zt;
  sh.each_of(own_key >= key, [&](int32_t, const Vec<T>& x) { n += tied(x); });
  block_scan(n, z, &own, &zt);
  const int rank = (int)cluster.block_rank();
  if (threadIdx.x < cluster.num_blocks()) *at_rank(&s.total_cnt[rank], threadIdx.x, cluster) = own;
  cluster.sync();
  uint32_t before = 0;
  for (int o = 0; o < rank; ++o) before += s.total_cnt[o];
  if (before >= keep) return -1;
  const uint32_t want = keep - before;
  if (own <= want) return INT32_MAX;
  uint32_t seen = 0;  // the want-th of this share is the last kept: a round covers consecutive vectors
  for (int32_t v0 = sh.first; seen < want; v0 += kLoads * kThreads) {
    uint32_t c[kLoads];
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int32_t v = v0 + u * kThreads + threadIdx.x;
      c[u] = v < sh.end && own_key >= key ? tied(sh.load(v)) : 0u;
    }
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      if (seen >= want) continue;
      uint32_t at = c[u], all;
      z = 0;
      block_scan(at, z, &all, &zt);
      if (c[u] && seen + at < want && seen + at + c[u] >= want) {
        const int32_t v = v0 + u * kThreads + threadIdx.x;
        const Vec<T> x = sh.load(v);
        uint32_t left = want - seen - at;
#pragma unroll
        for (int e = 0; e < Vec<T>::N; ++e)
          if (Key<T>::of(x.e[e]) == key && --left == 0) s.cutoff = sh.index(v) + e + 1;
      }
      seen += all;
    }
  }
  __syncthreads();
  return s.cutoff;
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

// A thread's largest logit, and the sum of exp((x - m) / T) over its tokens.
struct Running {
  float m = -INFINITY, z = 0.f, off = 0.f;  // off = m * scale
};

// Takes a vector into it: w[] = exp((x - m) / T) of its tokens relative to the
// new m; the factor by which what was relative to the old one shrinks.
template <typename T>
__device__ __forceinline__ float run_on(Running& a, const Vec<T>& x, float (&w)[Vec<T>::N], float scale) {
  const float mx = max_nan(a.m, vec_max(x));
  float by = 1.f;
  if (!(mx == a.m)) {  // (also once, and from then on, where there is a NaN)
    by = a.m == -INFINITY ? 0.f : ex2((a.m - mx) * scale);
    a.m = mx;
    a.z *= by;
    a.off = mx * scale;
  }
  if (fabsf(a.off) < 64.f) {  // (one rounding of at most 2^-19 of the exponent's unit, the same for all the thread's tokens)
#pragma unroll
    for (int k = 0; k < Vec<T>::N; ++k) w[k] = ex2(fmaf(widen(x.e[k]), scale, -a.off));
  } else {  // (no token yet, or logits of a size that would lose more)
#pragma unroll
    for (int k = 0; k < Vec<T>::N; ++k) w[k] = a.m == -INFINITY ? 0.f : ex2((widen(x.e[k]) - a.m) * scale);
  }
#pragma unroll
  for (int k = 0; k < Vec<T>::N; ++k) a.z += w[k];
  return by;
}

// The largest of the cluster's threads' values, NaN if one is.
__device__ __forceinline__ float cluster_top(float top, cg::cluster_group& cluster) {
  Shared& s = shared();
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
  if (lane == 0) s.wf[threadIdx.x >> 5] = top;
  __syncthreads();
  top = s.wf[lane % kWarps];
#pragma unroll
  for (int o = kWarps / 2; o > 0; o >>= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
  if (threadIdx.x == 0) s.top = top;
  cluster.sync();
  top = *at_rank(&s.top, lane % (int)cluster.num_blocks(), cluster);
#pragma unroll
  for (int o = kMaxCluster / 2; o > 0; o >>= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
  return top;
}

__device__ __forceinline__ void answer(const SampleParams& p, int32_t r, int32_t token, float logp) {
  p.tokens[r] = token;
  if (p.logp) p.logp[r] = logp;
  if (token < 0) set_status(p.dev_status, STRIDE_DEV_NO_TOKEN);
}

// The CTAs' winners race each other; the first CTA answers.
template <typename T>
__device__ __forceinline__ void finish(const SampleParams& p, const Share<T>& sh, int32_t r, const Weight& weight, bool sound, Best best,
                                       float kept, cg::cluster_group& cluster) {
  Shared& s = shared();
  const int rank = (int)cluster.block_rank();
  if (threadIdx.x == 0) {
    *at_rank(&s.race[rank], 0, cluster) = best;
    *at_rank(&s.kept[rank], 0, cluster) = kept;
  }
  cluster.sync();
  if (rank != 0 || threadIdx.x != 0) return;
  kept = 0.f;
  for (int o = 0; o < (int)cluster.num_blocks(); ++o) {
    take(best, s.race[o].v, s.race[o].i);
    kept += s.kept[o];
  }
  if (sound && best.v > 0.f)
    answer(p, r, best.i, weight.log(widen(sh.row[best.i])) - logf(kept));
  else
    answer(p, r, -1, NAN);
}

// The threads' best ratios (no token: INT32_MAX), of approximate exponentials and
// quotients (2^-22, and the rounding of an exponent of up to 64), race again with
// exact ones where they come within 1e-5 of the CTA's largest; kept: the threads'
// sums of weights.
template <typename T>
__device__ __forceinline__ void exact_race(const SampleParams& p, const Share<T>& sh, const float* noise, int32_t r, const Weight& weight,
                                           bool sound, Best best, float kept, cg::cluster_group& cluster) {
  if (best.i == INT32_MAX) best.v = -1.f;
  const Best lead = block_best(best);
  kept = block_sum(kept);
  Best exact = {-1.f, INT32_MAX};
  if (sound && best.i != INT32_MAX && best.v >= lead.v * 0.99999f)
    exact = {best.v < INFINITY ? weight(widen(sh.row[best.i])) / __ldg(noise + best.i) : INFINITY, best.i};
  exact = block_best(exact);
  finish(p, sh, r, weight, sound, exact, kept, cluster);
}

// Nothing is cut off: one pass over logits and noise together.  A thread keeps
// its largest logit m, sum exp((x - m) / T) and its best ratio exp((x - m) / T) /
// noise, rescaled where m grows.
template <typename T>
__device__ __noinline__ void race_all(const SampleParams& p, const Share<T>& sh, const float* noise, float temp, int32_t r, cg::cluster_group& cluster) {
  Shared& s = shared();
  constexpr int N = Vec<T>::N, U = N == 8 ? 2 : 4;
  const int tid = threadIdx.x;
  const float scale = exponent_scale(temp);
  const bool whole = (reinterpret_cast<uintptr_t>(noise + sh.index(0)) & 15) == 0;
  Best best = {0.f, INT32_MAX};
  Running a;
  for (int32_t v0 = sh.first + tid; v0 < sh.end; v0 += U * kThreads) {
    Vec<T> x[U];
    float e[U][N];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (v0 + u * kThreads < sh.end) {
        x[u] = sh.load(v0 + u * kThreads);
        load_noise<N>(e[u], noise, sh.index(v0 + u * kThreads), sh.V, whole);
      }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (v0 + u * kThreads >= sh.end) continue;
      float w[N], mx = 0.f;
      const float by = run_on(a, x[u], w, scale);
      if (best.v < INFINITY) best.v *= by;
#pragma unroll
      for (int k = 0; k < N; ++k) {
        w[k] = __fdividef(w[k], e[u][k]);  // (NaN, from a NaN noise or 0 / 0, wins nothing)
        mx = fmaxf(mx, w[k]);
      }
      if (mx > best.v) {
        best.v = mx;
#pragma unroll
        for (int k = N - 1; k >= 0; --k)
          if (w[k] == mx) best.i = sh.index(v0 + u * kThreads) + k;
      }
    }
  }
  const float top = cluster_top(a.m, cluster);
  const bool sound = top > -INFINITY && top < INFINITY;
  const float by = a.m == -INFINITY ? 0.f : ex2((a.m - top) * scale);
  if (best.v < INFINITY) best.v *= by;
  exact_race(p, sh, noise, r, Weight{top, temp}, sound, best, a.m == -INFINITY ? 0.f : a.z * by, cluster);
}

// The first CTA's list from the segments that the cluster's CTAs pushed, sorted.
__device__ __forceinline__ void sort_list(uint32_t n);
__device__ __forceinline__ void gather_list(uint32_t n, uint32_t segment) {
  Shared& s = shared();
  for (uint32_t j = threadIdx.x; j < n; j += kThreads) {
    uint32_t o = 0, k = j;
    while (k >= s.listed[o]) k -= s.listed[o++];
    s.list[j] = s.pushed[o * segment + k];
  }
  sort_list(n);
}

// Sorts s.list[0, n) (distinct values) from the largest down; n <= kList.  Up to
// 256 values each one's rank is counted, by several threads a value; the passes of
// a bitonic sort cost less above.
__device__ __forceinline__ void sort_list(uint32_t n) {
  Shared& s = shared();
  __syncthreads();
  if (n <= 256) {
    uint32_t P = 32;
    while (P < n) P *= 2;
    const uint32_t team = kThreads / P, j = threadIdx.x / team, part = threadIdx.x % team;
    const uint64_t mine = j < n ? s.list[j] : 0;
    uint32_t place = 0;
    for (uint32_t k = part; k < n; k += team) place += s.list[k] > mine;
    for (uint32_t o = 1; o < team; o *= 2) place += __shfl_xor_sync(0xffffffffu, place, o);
    __syncthreads();
    if (j < n && part == 0) s.list[place] = mine;
    __syncthreads();
    return;
  }
  uint32_t P = 512;
  while (P < n) P *= 2;
  for (uint32_t j = n + threadIdx.x; j < P; j += kThreads) s.list[j] = 0;
  __syncthreads();
  for (uint32_t run = 2; run <= P; run *= 2)
    for (uint32_t d = run / 2; d > 0; d /= 2) {
      for (uint32_t q = threadIdx.x; q < P / 2; q += kThreads) {
        const uint32_t i = 2 * q - (q & (d - 1)), j = i + d;
        const uint64_t a = s.list[i], b = s.list[j];
        if ((a < b) == ((i & run) == 0)) {
          s.list[i] = b;
          s.list[j] = a;
        }
      }
      __syncthreads();
    }
}

// The last kept token, among those up to `last` that in(x) holds for (none of a
// thread that `any` is false for): the first of them, in order, where base plus the
// count or mass up to it reaches the target.  False where they are too many to be
// sorted.
template <typename T, typename In>
__device__ __forceinline__ bool pick_among(const Share<T>& sh, const Weight& weight, bool any, In&& in, bool by_mass, uint64_t base,
                                           uint64_t target, Pick& last, cg::cluster_group& cluster) {
  Shared& s = shared();
  const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const Pick limit = last;
  const bool all = limit.key == Key<T>::of(lowest<T>());  // (no limit yet; its index alone does not say so: see tie_cutoff)
  __syncthreads();
  if (threadIdx.x == 0) s.count = 0;
  __syncthreads();
  sh.each_of(any, [&](int32_t v, const Vec<T>& x) {
    visit(
        x, [&](T y, int e) { return in(widen(y)) && (all || kept_by(limit, Key<T>::of(y), sh.index(v) + e)); },
        [&](T y, int e) {
          const uint32_t j = atomicAdd(&s.count, 1u);
          if (j < kList) s.list[j] = (uint64_t)Key<T>::of(y) << 32 | (uint32_t)~(sh.index(v) + e);
        });
  });
  __syncthreads();
  const uint32_t own_n = s.count, segment = kList / C;
  for (uint32_t j = threadIdx.x; j < min(own_n, segment); j += kThreads) *at_rank(&s.pushed[rank * segment + j], 0, cluster) = s.list[j];
  if (threadIdx.x < C) *at_rank(&s.listed[rank], threadIdx.x, cluster) = own_n;
  cluster.sync();
  uint32_t n = 0;
  bool fits = true;
  for (int o = 0; o < C; ++o) {
    fits = fits && s.listed[o] <= segment;
    n += s.listed[o];
  }
  if (!fits || n == 0) return false;
  if (rank == 0) {
    gather_list(n, segment);
    constexpr int kPer = kList / kThreads;
    uint32_t c = 0, tc;
    uint64_t m = 0, tm, w[kPer];
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      const uint32_t j = threadIdx.x * kPer + u;
      w[u] = j < n ? (by_mass ? (uint64_t)(weight(Key<T>::value((uint32_t)(s.list[j] >> 32))) * kOne) : 1) : 0;
      m += w[u];
    }
    block_scan(c, m, &tc, &tm);
    const auto tell = [&](uint32_t j) {
      const Pick q = {(uint32_t)(s.list[j] >> 32), (int32_t)~(uint32_t)s.list[j]};
      for (int o = 0; o < C; ++o) *at_rank(&s.pick, o, cluster) = q;
    };
    m += base;
    const bool reached = tm + base >= target;
    if (!reached && threadIdx.x == 0) tell(n - 1);  // (by the sums' rounding: all of them are kept)
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      if (reached && w[u] && m < target && m + w[u] >= target) tell(threadIdx.x * kPer + u);
      if (reached && threadIdx.x == 0 && u == 0 && m >= target) tell(0);
      m += w[u];
    }
  }
  cluster.sync();
  last = s.pick;
  return true;
}

// The `target`-th token: a histogram of 1,024 bins of the 32 units below the
// largest logit (the last one takes all below), then the tokens of one bin.
template <typename T>
__device__ __forceinline__ bool last_by_count(const Share<T>& sh, const Weight& weight, float own, uint64_t target, Pick& last,
                                              cg::cluster_group& cluster) {
  Shared& s = shared();
  // (the order of bins is that of the logits: each operation is monotone)
  const auto bin_of = [&](float x) { return (uint32_t)fminf((weight.m - x) * (kBins / 32.f), (float)(kBins - 1)); };
  for (int b = threadIdx.x; b < kBins; b += kThreads) s.cnt[b] = 0;
  __syncthreads();
  sh.each_of(own > -INFINITY, [&](int32_t, const Vec<T>& x) {
    visit(
        x, [&](T y, int) { return widen(y) > -INFINITY; }, [&](T y, int) { atomicAdd(&s.cnt[bin_of(widen(y))], 1u); });
  });
  const Found f = crossing(0, 0, false, false, target, cluster, [](uint32_t, uint32_t, uint64_t) { return uint64_t(0); });
  if (f.cnt > kList) return false;
  return pick_among(
      sh, weight, own > -INFINITY && bin_of(own) <= f.bin, [&](float x) { return x > -INFINITY && bin_of(x) == f.bin; }, false, f.above,
      target, last, cluster);
}

// A thread's sums become the cluster's (in a fixed order) in every CTA.
__device__ __forceinline__ void cluster_sums(float (&sum)[kPivots], cg::cluster_group& cluster) {
  Shared& s = shared();
  const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank(), lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int j = 0; j < kPivots; ++j) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum[j] += __shfl_xor_sync(0xffffffffu, sum[j], o);
    if (lane == j) s.part[warp][j] = sum[j];
  }
  __syncthreads();
  if (threadIdx.x < kPivots * C) {
    const int j = threadIdx.x % kPivots;
    float q = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) q += s.part[w][j];
    *at_rank(&s.pivot[rank][j], threadIdx.x / kPivots, cluster) = q;
  }
  cluster.sync();
#pragma unroll
  for (int j = 0; j < kPivots; ++j) {
    sum[j] = 0.f;
    for (int o = 0; o < C; ++o) sum[j] += s.pivot[o][j];
  }
  cluster.sync();  // (they make room for the next)
}

// The token where the mass of those up to `last` reaches the goal (in 2^-40).
// Tokens below `low` are not needed for it.  The masses above 7 pivots leave an
// eighth of the range, and twice those of the tokens in it above 7 more an eighth
// of that.
template <typename T>
__device__ __forceinline__ bool last_by_mass(const Share<T>& sh, const Weight& weight, float own, float low, uint64_t goal, Pick& last,
                                             cg::cluster_group& cluster) {
  const float scale = exponent_scale(weight.T), want = (float)goal * (1.f / kOne);
  const Pick limit = last;
  const bool all = limit.key == Key<T>::of(lowest<T>());  // (no limit yet; its index alone does not say so: see tie_cutoff)
  float lo = low, hi = INFINITY, above = 0.f;  // mass(x >= hi) = above < goal <= mass(x >= lo)
  for (int pass = 0; pass < 3; ++pass) {
    const float step = ((hi < INFINITY ? hi : weight.m) - lo) * (1.f / (kPivots + 1));
    float t[kPivots], sum[kPivots];
#pragma unroll
    for (int j = 0; j < kPivots; ++j) {
      t[j] = lo + step * (j + 1);
      sum[j] = 0.f;
    }
    const auto add = [&](float f, float w) {
#pragma unroll
      for (int j = 0; j < kPivots; ++j) sum[j] += f >= t[j] ? w : 0.f;
    };
    if (pass == 0) {
      sh.each_of(own >= lo, [&](int32_t v, const Vec<T>& x) {
#pragma unroll
        for (int e = 0; e < Vec<T>::N; ++e) {
          const float f = widen(x.e[e]);
          add(f, all || kept_by(limit, Key<T>::of(x.e[e]), sh.index(v) + e) ? ex2((f - weight.m) * scale) : 0.f);
        }
      });
    } else {
      sh.each_of(own >= lo, [&](int32_t v, const Vec<T>& x) {
        visit(
            x, [&](T y, int e) { return widen(y) >= lo && widen(y) < hi && (all || kept_by(limit, Key<T>::of(y), sh.index(v) + e)); },
            [&](T y, int) { add(widen(y), ex2((widen(y) - weight.m) * scale)); });
      });
    }
    cluster_sums(sum, cluster);
    float next_lo = lo, next_hi = hi, next_above = above;
    bool below = false;
#pragma unroll
    for (int j = kPivots - 1; j >= 0; --j) {
      if (below) continue;
      if (above + sum[j] >= want) {
        next_lo = t[j];
        below = true;
      } else {
        next_hi = t[j];
        next_above = above + sum[j];
      }
    }
    lo = next_lo;
    hi = next_hi;
    above = next_above;
  }
  return pick_among(
      sh, weight, own >= lo, [&](float x) { return x >= lo && x < hi; }, true, (uint64_t)(above * kOne), goal, last, cluster);
}

// What the first passes leave of a row.
struct Row {
  float temp, top_p, least, own, z;  // own: the thread's largest logit; z: the row's mass (of a top_p without top_k)
  int32_t top_k, r;
  bool cut_k, cut_p;
};

// The general way: the threshold by histograms, then the race.  (Its weights are approximate, also those that min_p is compared
// with and that the kept mass sums up: 2^-22, and the rounding of an exponent of up to 128. The winner's is computed again.)
template <typename T>
__device__ __noinline__ void race_above(const SampleParams& p, const Share<T>& sh, const float* noise, const Weight& weight, const Row& q,
                                        cg::cluster_group& cluster) {
  Shared& s = shared();
  constexpr int N = Vec<T>::N;
  const uint32_t none = Key<T>::of(lowest<T>()), first = Key<T>::of(static_cast<T>(weight.m)), own_key = Key<T>::of(static_cast<T>(q.own));
  Pick last = {none, -1};  // (all that are not ruled out)
  if (q.cut_k) {
    const uint64_t target = (uint64_t)q.top_k;
    if (!last_by_count(sh, weight, q.own, target, last, cluster)) {
      cluster.sync();
      const Cut cut = search(sh, weight, last, own_key, none + 1, first, false, target, false, cluster);
      const uint32_t ties = min((uint32_t)target - cut.above, cut.ties);
      last = {cut.key, ties < cut.ties ? tie_cutoff(sh, own_key, cut.key, ties, cluster) - 1 : INT32_MAX};
    }
  }
  if (q.cut_p) {
    float z = q.z;
    if (q.cut_k) {  // the mass of what top_k leaves
      float t = 0.f;
      sh.each_of(own_key >= last.key && own_key > none, [&](int32_t v, const Vec<T>& x) {
        visit(
            x, [&](T y, int e) { return kept_by(last, Key<T>::of(y), sh.index(v) + e); }, [&](T y, int) { t += weight(widen(y)); });
      });
      t = block_sum(t);
      cluster.sync();
      if (threadIdx.x < cluster.num_blocks()) *at_rank(&s.sum_all[cluster.block_rank()], threadIdx.x, cluster) = t;
      cluster.sync();
      z = 0.f;
      for (int o = 0; o < (int)cluster.num_blocks(); ++o) z += s.sum_all[o];
    }
    const uint64_t goal = (uint64_t)fmax(ceil((double)q.top_p * z * kOne), 1.0);
    // The tokens of w < (1 - top_p) z / (2 V) hold less than half of what may be left out: none of them is needed.
    const float low = weight.m + q.temp * logf(fmaxf((1.f - fmaxf(q.top_p, 0.f)) * z / (2.f * (float)p.V), 1e-30f));
    if (!last_by_mass(sh, weight, q.own, low, goal, last, cluster)) {
      cluster.sync();
      const Cut cut = search(sh, weight, last, own_key, none + 1, first, true, goal, true, cluster);
      const uint64_t one = max((uint64_t)(weight(Key<T>::value(cut.key)) * kOne), uint64_t(1));
      const uint64_t need = goal > cut.mass_above ? (goal - cut.mass_above + one - 1) / one : 1;
      const uint32_t ties = (uint32_t)min(need, (uint64_t)cut.ties);
      const int32_t at = ties < cut.ties ? tie_cutoff(sh, own_key, cut.key, ties, cluster) - 1 : INT32_MAX;
      if (cut.key > last.key || at < last.i) last = {cut.key, at};
    }
  }
  Best best = {0.f, INT32_MAX};
  float kept = 0.f;
  const float scale = exponent_scale(q.temp);
  sh.each_of(own_key >= last.key && q.own > -INFINITY && ex2((q.own - weight.m) * scale) >= q.least, [&](int32_t v, const Vec<T>& x) {
    const int32_t i0 = sh.index(v);
    float w[N], e[N];  // (the noise of the kept ones, asked for together)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      w[i] = ex2((widen(x.e[i]) - weight.m) * scale);
      if (!kept_by(last, Key<T>::of(x.e[i]), i0 + i) || w[i] < q.least) w[i] = 0.f;
      e[i] = w[i] > 0.f ? __ldg(noise + i0 + i) : 1.f;
    }
    float mx = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      kept += w[i];
      w[i] = __fdividef(w[i], e[i]);
      mx = fmaxf(mx, w[i]);
    }
    if (mx > 0.f && mx >= best.v) {  // (a lane's vectors come in no order of index: see each_of)
      int32_t at = INT32_MAX;
#pragma unroll
      for (int i = N - 1; i >= 0; --i)
        if (w[i] == mx) at = i0 + i;
      take(best, mx, at);
    }
  });
  exact_race(p, sh, noise, q.r, weight, true, best, kept, cluster);
}

// The n-th row of the call (of kThreads at most: a thread tells each row's kind) if
// those without a top_k come first.  With a top_p they take several times as long as
// the others: started last, they were what the call waited for.  (Nothing is lost
// where they are short after all; a row whose top_k is past the list is long, too, and
// comes in its turn.)
__device__ __forceinline__ int32_t long_first(const SampleParams& p, int32_t n) {
  Shared& s = shared();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int32_t k = tid < p.rows ? __ldg(p.how.top_k + tid) : 1;
  const bool is_long = k <= 0 || k >= p.V;
  const unsigned those = __ballot_sync(0xffffffffu, is_long);
  if (lane == 0) s.wc[warp] = __popc(those);
  __syncthreads();
  int32_t before = __popc(those & ((1u << lane) - 1)), all = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) before += s.wc[w];
    all += s.wc[w];
  }
  if (tid < p.rows && (is_long ? before : all + tid - before) == n) s.first_row = tid;
  __syncthreads();
  return s.first_row;
}

template <typename T>
__global__ void __launch_bounds__(kThreads, 2) sample_kernel(const SampleParams p) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  Shared& s = shared();
  cg::cluster_group cluster = cg::this_cluster();
  const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int32_t r = p.long_first ? long_first(p, blockIdx.x / C) : blockIdx.x / C;
  constexpr int N = Vec<T>::N;

  Share<T> sh;
  sh.row = static_cast<const T*>(p.x) + (int64_t)r * p.ld;
  sh.shift = (int32_t)((reinterpret_cast<uintptr_t>(sh.row) & 15) / sizeof(T));
  sh.V = p.V;
  const int64_t vecs = ((int64_t)p.V + sh.shift + N - 1) / N;
  sh.first = (int32_t)(vecs * rank / C);
  sh.end = (int32_t)(vecs * (rank + 1) / C);
  if (tid == 0 && sh.end > sh.first) {  // on its way while the row's parameters are
    const int32_t i0 = max(sh.index(sh.first), 0), i1 = min(sh.index(sh.end), p.V);
    prefetch_l2(sh.row + i0, (int64_t)(i1 - i0) * sizeof(T));
  }
  const float* noise = p.noise + (int64_t)r * p.ld_noise;
  const float temp = p.how.temperature ? __ldg(p.how.temperature + r) : p.how.temperature_all;
  const int32_t top_k = p.how.top_k ? __ldg(p.how.top_k + r) : p.how.top_k_all;
  const float top_p = p.how.top_p ? __ldg(p.how.top_p + r) : p.how.top_p_all;
  const float min_p = p.how.min_p ? __ldg(p.how.min_p + r) : p.how.min_p_all;
  const bool cut_k = top_k > 0 && top_k < p.V, cut_p = top_p < 1.f;
  const bool params = temp >= 0.f && temp < INFINITY && !isnan(top_p) && !isnan(min_p);

  if (params && temp > 0.f && !cut_k && !cut_p && min_p <= 0.f) {
    race_all(p, sh, noise, temp, r, cluster);
    return;
  }

  // each thread's largest logit (NaN if it has one) and, for a top_p of the whole row, its sum of weights
  const bool need_all = params && temp > 0.f && cut_p && !cut_k;
  Running a;
  if (need_all)
    sh.template each<kLoads>([&](int32_t, const Vec<T>& x) {
      float w[N];
      run_on(a, x, w, exponent_scale(temp));
    });
  else
    sh.template each<kLoads>([&](int32_t, const Vec<T>& x) { a.m = max_nan(a.m, vec_max(x)); });
  const float own = a.m;
  // groups of `per` threads: at least 128 of them, and a third more than the bound asks for
  const uint32_t reach = cut_k ? (uint32_t)top_k : (uint32_t)kUsual;
  int per = 32;
  while (per > 1 && (uint32_t)(C * kThreads / per) < max(reach + reach / 3, 128u)) per /= 2;
  const int groups = C * kThreads / per, own_groups = kThreads / per;
  const bool by_list = (cut_k || cut_p) && groups <= kGroups && (uint32_t)groups >= reach;
  if (by_list) {
    float g = own;
    for (int o = 1; o < per; o <<= 1) g = max_nan(g, __shfl_xor_sync(0xffffffffu, g, o));
    if (lane % per == 0) s.own_group[tid / per] = g;
  }
  if (tid == 0) {
    s.count = 0;
    s.cutoff = INT32_MAX;
  }
  const float top = cluster_top(own, cluster);
  const Weight weight = {top, temp};

  const bool sound = params && top > -INFINITY && top < INFINITY;
  if (!sound || temp == 0.f) {
    if (sound) {  // the first of the largest
      sh.each_of(own == top, [&](int32_t v, const Vec<T>& x) {
#pragma unroll
        for (int e = 0; e < N; ++e)
          if (widen(x.e[e]) == top) atomicMin(&s.cutoff, sh.index(v) + e);
      });
      __syncthreads();
      if (tid == 0) *at_rank(&s.lowest[rank], 0, cluster) = s.cutoff;
    }
    cluster.sync();  // (no CTA leaves while another may read its shared memory)
    if (rank == 0 && tid == 0) {
      int32_t token = INT32_MAX;
      for (int o = 0; sound && o < C; ++o) token = min(token, s.lowest[o]);
      answer(p, r, sound ? token : -1, sound ? 0.f : NAN);
    }
    return;
  }
  const float least = fminf(min_p, 1.f);
  const uint32_t none = Key<T>::of(lowest<T>()), first = Key<T>::of(static_cast<T>(top)), own_key = Key<T>::of(static_cast<T>(own));
  float all = 0.f, z = 0.f;  // the mass of the share's tokens, of the row's
  if (need_all) all = block_sum(own == -INFINITY ? 0.f : a.z * ex2((own - top) * exponent_scale(temp)));

  if (by_list) {
    // The bound: the largest key that at least `reach` of the groups reach (to within an eighth of them), by bisection;
    // one warp's work where it holds all groups (four a lane).
    constexpr int kMine = kGroups / kThreads;
    uint32_t lo = none, hi = first + 1;  // (all groups reach lo; fewer than `reach` reach hi, or hi is past the largest)
    const auto group = [&](int j) {
      return j < groups ? Key<T>::of(static_cast<T>(*at_rank(&s.own_group[j % own_groups], j / own_groups, cluster))) : 0u;
    };
    if (groups <= 128) {
      if (warp == 0) {
        uint32_t g[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) g[u] = group(lane + u * 32);
        while (hi - lo > 1) {
          const uint32_t mid = lo + (hi - lo) / 2;
          uint32_t n = 0;
#pragma unroll
          for (int u = 0; u < 4; ++u) n += __popc(__ballot_sync(0xffffffffu, g[u] >= mid));
          if (n >= reach) {
            lo = mid;
            if (n <= reach + reach / 8) break;
          } else {
            hi = mid;
          }
        }
        if (lane == 0) s.bound = lo;
      }
      __syncthreads();
      lo = s.bound;
    } else {
      uint32_t g[kMine];
#pragma unroll
      for (int u = 0; u < kMine; ++u) g[u] = group(tid + u * kThreads);
      while (hi - lo > 1) {
        const uint32_t mid = lo + (hi - lo) / 2;
        uint32_t n = 0;
#pragma unroll
        for (int u = 0; u < kMine; ++u)
          if (u * kThreads < groups) n += __syncthreads_count(g[u] >= mid);
        if (n >= reach) {
          lo = mid;
          if (n <= reach + reach / 8) break;
        } else {
          hi = mid;
        }
      }
    }
    const uint32_t bound = max(lo, none + 1);  // (tokens of -inf are none)
    float listed = 0.f;
    sh.each_of(own_key >= bound, [&](int32_t v, const Vec<T>& x) {
      visit(
          x, [&](T y, int) { return Key<T>::of(y) >= bound; },
          [&](T y, int e) {
            if (need_all) listed += weight(widen(y));
            const uint32_t at = atomicAdd(&s.count, 1u);
            if (at < kList) s.list[at] = (uint64_t)Key<T>::of(y) << 32 | (uint32_t)~(sh.index(v) + e);
          });
    });
    if (need_all)
      listed = block_sum(listed);
    else
      __syncthreads();
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
    float zl = 0.f;
    for (int o = 0; o < C; ++o) {
      held = held && s.listed[o] <= segment;
      n += s.listed[o];
      z += s.sum_all[o];
      zl += s.sum_listed[o];
    }
    // the list holds what is kept: top_k of the largest; or more than top_p of the mass, or all of w >= min_p
    if (held && (cut_k || zl > top_p * z * 1.00001f || weight(Key<T>::value(bound)) < least)) {
      if (rank == 0) {
        gather_list(n, segment);
        constexpr int kPer = kList / kThreads;  // consecutive ranks of a thread
        const uint32_t kept_k = cut_k ? min((uint32_t)top_k, n) : n;
        float w[kPer], e[kPer], d[kPer], mass = 0.f;
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
            d[u] = weight.log(Key<T>::value((uint32_t)(q >> 32)));
            w[u] = expf(d[u]);
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
        const Best mine = best;
        best = block_best(best);
        kept = block_sum(kept);
        if (best.v > 0.f) {
#pragma unroll
          for (int u = 0; u < kPer; ++u)
            if (mine.i == best.i && idx[u] == best.i && tid * kPer + u < kept_k) answer(p, r, best.i, d[u] - logf(kept));
        } else if (tid == 0) {
          answer(p, r, -1, NAN);
        }
      }
      return;  // (nothing of another CTA is read after the last cluster.sync)
    }
    cluster.sync();  // s.list makes room for the histogram
  }

  const Row row = {temp, top_p, least, own, z, top_k, r, cut_k, cut_p};
  race_above(p, sh, noise, weight, row, cluster);
}

template <typename T>
cudaError_t run(SampleParams p, int sms, cudaStream_t stream) {
  // CTAs of a row: 8 where all run at once (two on an SM); else, at least a vector per thread,
  // - with a top_k of each row's own, 4 up to the 512 rows that long_first() orders: the longest row counts (us, rows of 151,936
  //   bf16 logits, with 8 / 4 / 2 / 1, 90 rows of mixed parameters: 46 / 47 / 67 / 112; 256: 87 / 88 / 129 / 217; 500: 160 /
  //   110 / 140 / 233);
  // - with one small top_k for all, what runs at once (top_k 50, 64 rows: 25 / 15 / 17 / 27; 90: 30 / 23 / 17 / 29; 256: 75 / 46 /
  //   34 / 35; 500: 144 / 86 / 69 / 62);
  // - else 4 up to two rows an SM, and 1 (top_p 0.9, 90 rows: 133 / 110 / 156 / 272; 256: 318 / 231 / 220 / 307; 512 uncut rows of
  //   32,000 fp32: 144 / 81 / 60 / 48).
  const int64_t rows = p.rows, at_once = 2 * sms;
  int C = 1;
  if (rows * kMaxCluster <= at_once)
    C = kMaxCluster;
  else if (p.how.top_k)
    C = rows <= kThreads ? 4 : 1;
  else if (p.how.top_k_all > 0 && p.how.top_k_all <= 128)
    C = rows * 4 <= at_once ? 4 : rows <= at_once ? 2 : 1;
  else
    C = rows <= at_once ? 4 : 1;
  while (C > 1 && p.V < C * kThreads * Vec<T>::N) C /= 2;
  p.long_first = p.how.top_k && p.rows <= kThreads && (int64_t)p.rows * C > 2 * sms;  // (several waves of CTAs)
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((int64_t)p.rows * C));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kDepth * kThreads * 16;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = C;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  cudaError_t e = cudaFuncSetAttribute(sample_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, kDepth * kThreads * 16);
  if (e != cudaSuccess) return e;
  e = cudaLaunchKernelEx(&cfg, sample_kernel<T>, p);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

cudaError_t launch_sample(const SampleParams& p, int dtype, int sms, cudaStream_t stream) {
  if (p.rows > INT32_MAX / kMaxCluster) return cudaErrorInvalidConfiguration;
  if (dtype == STRIDE_DTYPE_BF16) return run<__nv_bfloat16>(p, sms, stream);
  if (dtype == STRIDE_DTYPE_F16) return run<__half>(p, sms, stream);
  return run<float>(p, sms, stream);
}

}  // namespace stride
