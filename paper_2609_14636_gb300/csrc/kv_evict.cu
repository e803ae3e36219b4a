// kv_evict.cu -- the slots of most attention weight of a cache, copied in order
// into fewer pages (sm_103a).
//
// Two kernels.  The first finds, for each sequence and kv head, which slots remain:
// the m-th largest mass digit by digit (its ordered bits, eight at a time, counted
// in shared memory), then the slots above it and the first ones equal to it,
// numbered by a prefix sum in the slots' order.  A unit (sequence, head) is taken by a
// cluster of CTAs, more where there are fewer units; their counts meet in
// distributed shared memory.  The masses stay in registers from the first digit on,
// as far as they fit.  The second copies the rows, which is what counts: pages are
// looked up and offsets computed once for a CTA's rows, then threads move 16 bytes at
// a time, several loads each on their way.
#include <cooperative_groups.h>

#include <algorithm>

#include "decode_internal.h"
#include "stride_device.cuh"

namespace cg = cooperative_groups;

namespace stride {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kHeld = 16;  // masses of a thread that stay in registers
constexpr int kMaxCluster = 16;

// Rises with x; a NaN is below all, zeros are alike.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t b = x == 0.f ? 0 : __float_as_uint(x);
  return isnan(x) ? 0 : (b >> 31) ? ~b : b | 0x80000000u;
}

// What remains of a sequence.
struct Plan {
  int32_t n, m, sink, recent;
  bool out, bad;  // left out; a length that does not fit
};
__device__ __forceinline__ Plan plan_of(const EvictParams& p, int b) {
  Plan r;
  r.n = __ldg(p.from.ctx_len + b);
  const int budget = p.how.budget ? __ldg(p.how.budget + b) : p.how.budget_all;
  r.out = budget < 0;
  r.m = min(r.n, budget);
  r.sink = min(r.m, p.how.sink);
  r.recent = min(r.m - r.sink, p.how.recent);
  r.bad = r.n < 0 || r.n > p.mass.slots || r.n > p.from.table_stride * p.from.page_size || r.m > p.how.most ||
          r.m > p.to.table_stride * p.to.page_size;
  return r;
}

// Blocks: unit * cluster + rank.
__global__ void __launch_bounds__(kThreads) select_kernel(const __grid_constant__ EvictParams p) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  __shared__ uint32_t s_count[4][256];  // of each digit's pass
  __shared__ uint32_t s_sum[256];       // a pass's counts of all CTAs
  __shared__ int2 s_total;              // slots above the threshold, equal to it, of this CTA
  __shared__ int2 s_warp[kWarps];
  const cg::cluster_group cluster = cg::this_cluster();
  const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int unit = blockIdx.x / C, b = unit / p.from.n_heads, head = unit - b * p.from.n_heads;
  const Plan plan = plan_of(p, b);
  if (plan.out || plan.bad) {  // (all of the cluster alike)
    if (head == 0 && rank == 0 && tid == 0) {
      p.new_len[b] = plan.out ? plan.n : -1;
      if (!plan.out) set_status(p.dev_status, STRIDE_DEV_BAD_LAYOUT);
    }
    return;
  }
  if (head == 0 && rank == 0 && tid == 0) p.new_len[b] = plan.m;

  const float* mass = p.mass.data + b * p.mass.seq_stride + head * p.mass.head_stride;
  // A warp's slots: a run of `steps` times 32.
  const int steps = (plan.n + C * kThreads - 1) / (C * kThreads);
  const int64_t first = (int64_t)(rank * kWarps + warp) * steps * 32 + lane;
  const int lo = plan.sink, hi = plan.n - plan.recent;  // between them the masses decide
  float held[kHeld];
#pragma unroll
  for (int j = 0; j < kHeld; ++j) {
    const int64_t slot = first + j * 32;
    held[j] = j < steps && slot < plan.n ? __ldg(mass + slot) : 0.f;
  }
  // f(j, slot, mass) for each of this lane's slots below n.
  const auto each = [&](auto&& f) {
#pragma unroll
    for (int j = 0; j < kHeld; ++j) f(j, first + j * 32, held[j]);
    for (int j = kHeld; j < steps; ++j) {
      const int64_t slot = first + j * 32;
      f(j, slot, slot < plan.n ? __ldg(mass + slot) : 0.f);
    }
  };

  int need = plan.m - plan.sink - plan.recent;  // of those between
  const bool all = need == hi - lo, none = need == 0;
  uint32_t threshold = 0;
  if (!all && !none) {
    for (int i = tid; i < 4 * 256; i += kThreads) s_count[i / 256][i % 256] = 0;
    __syncthreads();
#pragma unroll
    for (int pass = 0; pass < 4; ++pass) {
      const int shift = 24 - 8 * pass;
      each([&](int j, int64_t slot, float x) {
        if (j >= steps || slot < lo || slot >= hi) return;
        const uint32_t key = ordered(x);
        if (pass == 0 || (key ^ threshold) >> (shift + 8) == 0) atomicAdd(&s_count[pass][(key >> shift) & 255], 1u);
      });
      cluster.sync();
      if (tid < 256) {
        uint32_t sum = 0;
        for (int r = 0; r < C; ++r) sum += *cluster.map_shared_rank(&s_count[pass][tid], r);
        s_sum[tid] = sum;
      }
      __syncthreads();
      // the digit at which the counts from the top reach `need`, found by each warp: a lane has eight digits
      uint32_t c[8], own = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        c[i] = s_sum[255 - (lane * 8 + i)];
        own += c[i];
      }
      uint32_t upto = own;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t v = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += v;
      }
      const int l = __ffs(__ballot_sync(0xffffffffu, upto >= (uint32_t)need)) - 1;
      uint32_t above = upto - own;
      int digit = 0, left = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (above < (uint32_t)need && above + c[i] >= (uint32_t)need) {
          digit = 255 - (lane * 8 + i);
          left = need - (int)above;
        }
        above += c[i];
      }
      threshold |= (uint32_t)__shfl_sync(0xffffffffu, digit, l) << shift;
      need = __shfl_sync(0xffffffffu, left, l);
      __syncthreads();  // (s_sum is read)
    }
  }
  // `need` of those equal to the threshold remain, the first ones.
  const auto above = [&](int64_t slot, float x) {
    return slot < plan.n && (slot < lo || slot >= hi || all || (!none && ordered(x) > threshold));
  };
  const auto equal = [&](int64_t slot, float x) { return slot >= lo && slot < hi && !all && !none && ordered(x) == threshold; };
  int2 mine = make_int2(0, 0);
  each([&](int j, int64_t slot, float x) {
    if (j >= steps) return;
    mine.x += __popc(__ballot_sync(0xffffffffu, above(slot, x)));
    mine.y += __popc(__ballot_sync(0xffffffffu, equal(slot, x)));
  });
  if (lane == 0) s_warp[warp] = mine;
  __syncthreads();
  if (tid == 0) {
    int2 sum = make_int2(0, 0);
    for (int w = 0; w < kWarps; ++w) {
      const int2 v = s_warp[w];
      s_warp[w] = sum;
      sum.x += v.x;
      sum.y += v.y;
    }
    s_total = sum;
  }
  if (C > 1)
    cluster.sync();
  else
    __syncthreads();
  int2 before = s_warp[warp];
  for (int r = 0; r < rank; ++r) {
    const int2 v = *cluster.map_shared_rank(&s_total, r);
    before.x += v.x;
    before.y += v.y;
  }
  const int64_t row = (int64_t)unit * p.how.most;
  float* mass_to = p.mass_to.data ? p.mass_to.data + b * p.mass_to.seq_stride + head * p.mass_to.head_stride : nullptr;
  each([&](int j, int64_t slot, float x) {
    if (j >= steps) return;
    const bool up = above(slot, x), eq = equal(slot, x);
    const unsigned ups = __ballot_sync(0xffffffffu, up), eqs = __ballot_sync(0xffffffffu, eq), below = (1u << lane) - 1;
    const int e = before.y + __popc(eqs & below);
    if (up || (eq && e < need)) {
      const int i = before.x + __popc(ups & below) + min(e, need);
      p.kept[row + i] = (int32_t)slot;
      if (mass_to) mass_to[i] = x;
    }
    before.x += __popc(ups);
    before.y += __popc(eqs);
  });
  if (C > 1) cluster.sync();  // (no CTA leaves while its counts may be read)
}

constexpr int kRows = 64;          // rows of a CTA at a time
constexpr int kCopyThreads = 256;

// Blocks: unit * splits + part, which takes every splits-th run of kRows rows.
template <typename V>
__global__ void __launch_bounds__(kCopyThreads) copy_kernel(const __grid_constant__ EvictParams p, const int elem, const int splits) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  __shared__ int64_t s_from[kRows], s_to[kRows];  // bytes; -1: not copied
  const int unit = blockIdx.x / splits, part = blockIdx.x - unit * splits, b = unit / p.from.n_heads, head = unit - b * p.from.n_heads;
  if (p.how.budget ? __ldg(p.how.budget + b) < 0 : p.how.budget_all < 0) return;
  const int m = p.new_len[b];
  const int per = p.row_bytes / (int)sizeof(V), tid = threadIdx.x;  // vectors of a row
  for (int64_t r0 = (int64_t)part * kRows; r0 < m; r0 += (int64_t)splits * kRows) {
    const int have = (int)min((int64_t)kRows, m - r0);
    if (tid < have) {
      const int i = (int)r0 + tid, slot = p.kept[(int64_t)unit * p.how.most + i];
      const int e = slot / p.from.page_size, f = i / p.to.page_size;
      const int32_t page = __ldg(p.from.block_table + (int64_t)b * p.from.table_stride + e);
      const int32_t there = __ldg(p.to.block_table + (int64_t)b * p.to.table_stride + f);
      const bool ok = page >= 0 && page < p.from.n_pages && there >= 0 && there < p.to.n_pages;
      if (!ok) set_status(p.dev_status, STRIDE_DEV_BAD_LAYOUT);
      s_from[tid] = (page * p.from.page_stride + (slot - e * p.from.page_size) * p.from.row_stride + head * p.from.head_stride) * elem;
      s_to[tid] = ok ? (there * p.to.page_stride + (i - f * p.to.page_size) * p.to.row_stride + head * p.to.head_stride) * elem : -1;
    }
    __syncthreads();
    constexpr int kAhead = 4;
    for (int v0 = tid; v0 < have * per; v0 += kAhead * kCopyThreads) {
      V k[kAhead], w[kAhead];
      int64_t to[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int v = v0 + u * kCopyThreads, r = v / per, c = (v - r * per) * (int)sizeof(V);
        to[u] = v < have * per ? s_to[r] : -1;
        if (to[u] < 0) continue;
        k[u] = *reinterpret_cast<const V*>(static_cast<const char*>(p.from.k) + s_from[r] + c);
        w[u] = *reinterpret_cast<const V*>(static_cast<const char*>(p.from.v) + s_from[r] + c);
        to[u] += c;
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (to[u] < 0) continue;
        *reinterpret_cast<V*>(static_cast<char*>(p.to.k) + to[u]) = k[u];
        *reinterpret_cast<V*>(static_cast<char*>(p.to.v) + to[u]) = w[u];
      }
    }
    __syncthreads();
  }
}

}  // namespace

cudaError_t launch_kv_evict(const EvictParams& p, int elem, int chunk, int sms, cudaStream_t stream) {
  const int units = p.from.n_seqs * p.from.n_heads;
  const int64_t slots = std::min<int64_t>(p.mass.slots, p.from.table_stride * (int64_t)p.from.page_size);
  int C = 1;
  while (C < kMaxCluster && (int64_t)units * C * 2 <= sms && slots > (int64_t)C * kThreads * 2) C *= 2;
  cudaError_t e = cudaFuncSetAttribute(select_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(units * C);
  cfg.blockDim = dim3(kThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = C;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  e = cudaLaunchKernelEx(&cfg, select_kernel, p);
  if (e != cudaSuccess) return e;
  const int64_t most = std::min<int64_t>(std::min<int64_t>(p.how.most, slots), p.to.table_stride * (int64_t)p.to.page_size);
  const int64_t parts = std::min<int64_t>((most + kRows - 1) / kRows, ((int64_t)sms * 64 + units - 1) / units);
  const int splits = (int)std::max<int64_t>(1, parts);
  if (chunk == 16) return launch_dependent(copy_kernel<uint4>, units * splits, kCopyThreads, stream, p, elem, splits);
  if (chunk == 4) return launch_dependent(copy_kernel<uint32_t>, units * splits, kCopyThreads, stream, p, elem, splits);
  return launch_dependent(copy_kernel<uint16_t>, units * splits, kCopyThreads, stream, p, elem, splits);
}

}  // namespace stride
