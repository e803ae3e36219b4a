// kv_evict.cu -- the slots of most attention weight of a cache, copied in order
// into fewer pages (sm_103a).
//
// Two kernels.  The first finds, for each sequence and kv head, which slots remain:
// the m-th largest mass digit by digit (its ordered bits, eight at a time, counted
// in shared memory, with a cluster's counts added up in distributed shared memory), then the slots above it and the first ones equal to it,
// numbered by a prefix sum in the slots' order.  A unit (sequence, head) is taken by a
// cluster of CTAs, more where there are fewer units.  The masses stay in registers from the first digit on,
// as far as they fit.  The second copies the rows, which is what counts: pages are
// looked up and offsets computed once for a CTA's rows, then threads move 16 bytes at
// a time, several loads each on their way.
//
// Measured, us (floor: of bytes at 6,683 GB/s): 256 sequences of up to 4,096 slots to 1,024, 8 heads of 128, 343 (310: the copy 300,
// before it the selection); one of 131,072 to 16,384 45 (21: the copy 20, the selection's exchanges in clusters of 16 before it 22);
// three of up to 323 9.6 (two launches and the digits' passes).  Rows that remain for sure copied by CTAs of the first kernel: 420
// and 48.
#include <cooperative_groups.h>

#include <algorithm>

#include "decode_internal.h"
#include "stride_device.cuh"

namespace cg = cooperative_groups;

namespace stride {
namespace {

constexpr int kMaxCluster = 16;
// Copies of the first digit's counts, by lane: nearly all masses have one of a few exponents, and lanes that count alike wait for
// one another.
constexpr int kCopies = 8;

// Rises with x; a NaN is below all, zeros are alike.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t b = x == 0.f ? 0 : __float_as_uint(x);
  return isnan(x) ? 0 : (b >> 31) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float mass_of(uint32_t key) {
  return key == 0 ? NAN : __uint_as_float(key >> 31 ? key & 0x7fffffffu : ~key);
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

// Blocks: unit * cluster + rank.  kHeld: masses of a thread that stay in registers; kBlocks: CTAs on an SM.
template <int kThreads, int kHeld, int kBlocks>
__global__ void __launch_bounds__(kThreads, kBlocks) select_kernel(const __grid_constant__ EvictParams p) {
  constexpr int kWarps = kThreads / 32;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  __shared__ __align__(16) uint32_t s_first[256 * kCopies];  // the first digit's counts, a digit's copies side by side
  __shared__ uint32_t s_count[4][256];                       // of each digit's pass
  __shared__ uint32_t s_part[8], s_digit, s_left;
  __shared__ int2 s_total;  // slots above the threshold, equal to it, of this CTA
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
  // A warp's slots: a run of `steps` times 32.  (Below 2^31 and some thousands: unsigned.)
  const int steps = (int)(((int64_t)plan.n + C * kThreads - 1) / (C * kThreads));
  const uint32_t first = (uint32_t)(rank * kWarps + warp) * steps * 32 + lane, n = plan.n;
  const uint32_t lo = plan.sink, between = plan.n - plan.recent - plan.sink;  // from lo on, so many slots that the masses decide about
  int need = plan.m - plan.sink - plan.recent;                                // that remain of them
  const bool all = need == (int)between, decide = !all && need > 0;
  // The first kHeld of this lane's masses, in order, and which of them are still to be decided about; later ones are read again.
  // (All on their way at once: a load behind each slot's own branch took 19,000 clocks for sixteen.)
  uint32_t held[kHeld], open = 0;
  const uint32_t end = n > 0 ? n - 1 : 0;
  if (n > 0) {
    float x[kHeld];
#pragma unroll
    for (int j = 0; j < kHeld; ++j) x[j] = __ldg(mass + min(first + j * 32, end));
#pragma unroll
    for (int j = 0; j < kHeld; ++j) held[j] = ordered(x[j]);
  }
  if (decide) {
#pragma unroll
    for (int j = 0; j < kHeld; ++j)
      if (j < steps && first + j * 32 - lo < between) open |= 1u << j;
  }
  // f(key) for the keys of this lane's undecided slots that share the threshold's bits above `shift` + 8
  uint32_t threshold = 0;
  const auto each = [&](int shift, auto&& f) {
#pragma unroll
    for (int j = 0; j < kHeld; ++j)
      if (open >> j & 1) {
        if (shift < 24 && (held[j] ^ threshold) >> (shift + 8))
          open &= ~(1u << j);
        else
          f(held[j]);
      }
    for (int j = kHeld; j < steps; ++j) {
      const uint32_t slot = first + j * 32;
      if (slot - lo >= between) continue;
      const uint32_t key = ordered(__ldg(mass + slot));
      if (shift == 24 || (key ^ threshold) >> (shift + 8) == 0) f(key);
    }
  };
  const auto cluster_sync = [&] {
    if (C > 1)
      cluster.sync();
    else
      __syncthreads();
  };
  if (decide) {
    for (int i = tid; i < 256 * kCopies; i += kThreads) s_first[i] = 0;
    for (int i = tid; i < 3 * 256; i += kThreads) s_count[1 + i / 256][i % 256] = 0;
    __syncthreads();
    each(24, [&](uint32_t key) { atomicAdd(&s_first[(key >> 24) * kCopies + (lane & (kCopies - 1))], 1u); });
    __syncthreads();
    if (tid < 256) {
      const uint4 u = reinterpret_cast<const uint4*>(s_first)[2 * tid], v = reinterpret_cast<const uint4*>(s_first)[2 * tid + 1];
      s_count[0][tid] = u.x + u.y + u.z + u.w + v.x + v.y + v.z + v.w;
    }
#pragma unroll 1
    for (int pass = 0; pass < 4; ++pass) {
      const int shift = 24 - 8 * pass;
      if (pass > 0) each(shift, [&](uint32_t key) { atomicAdd(&s_count[pass][(key >> shift) & 255], 1u); });
      cluster_sync();
      // the digit at which the counts from the top reach `need`: a thread has a digit, the highest first
      const int digit = 255 - tid;
      uint32_t sum = 0, upto = 0;
      if (tid < 256) {
        if (C == 1) {
          sum = s_count[pass][digit];
        } else {
          for (int r0 = 0; r0 < C; r0 += 8) {  // (eight CTAs' on their way at once; C is a power of two)
            uint32_t v[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) v[r] = *cluster.map_shared_rank(&s_count[pass][digit], (r0 + r) & (C - 1));
#pragma unroll
            for (int r = 0; r < 8; ++r) sum += r0 + r < C ? v[r] : 0;
          }
        }
        upto = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const uint32_t v = __shfl_up_sync(0xffffffffu, upto, o);
          if (lane >= o) upto += v;
        }
        if (lane == 31) s_part[warp] = upto;
      }
      __syncthreads();
      if (tid < 256) {
        for (int w = 0; w < warp; ++w) upto += s_part[w];
        if (upto >= (uint32_t)need && upto - sum < (uint32_t)need) {
          s_digit = digit;
          s_left = need - (upto - sum);
        }
      }
      __syncthreads();
      threshold |= s_digit << shift;
      need = (int)s_left;
      // (the next write of these is behind two barriers)
    }
  }
  // `need` of those equal to the threshold remain, the first ones.
  const auto above = [&](uint32_t slot, uint32_t key) {
    return slot < n && (slot - lo >= between || all || (decide && key > threshold));
  };
  const auto equal = [&](uint32_t slot, uint32_t key) { return decide && slot - lo < between && key == threshold; };
  uint32_t ups = 0, eqs = 0;  // bits: the first kHeld slots
  int2 mine = make_int2(0, 0);
#pragma unroll
  for (int j = 0; j < kHeld; ++j) {
    if (j >= steps) break;
    const uint32_t slot = first + j * 32;
    if (above(slot, held[j])) ups |= 1u << j;
    if (equal(slot, held[j])) eqs |= 1u << j;
  }
  mine.x = __popc(ups);
  mine.y = __popc(eqs);
  for (int j = kHeld; j < steps; ++j) {
    const uint32_t slot = first + j * 32, key = slot < n ? ordered(__ldg(mass + slot)) : 0;
    mine.x += above(slot, key);
    mine.y += equal(slot, key);
  }
  mine.x = __reduce_add_sync(0xffffffffu, mine.x);
  mine.y = __reduce_add_sync(0xffffffffu, mine.y);
  if (lane == 0) s_warp[warp] = mine;
  __syncthreads();
  int2 before = make_int2(0, 0);
  for (int w = 0; w < warp; ++w) {
    before.x += s_warp[w].x;
    before.y += s_warp[w].y;
  }
  if (tid == kThreads - 1) s_total = make_int2(before.x + s_warp[warp].x, before.y + s_warp[warp].y);
  if (C > 1) {
    cluster.sync();
    int2 v = make_int2(0, 0);
    if (lane < rank) v = *cluster.map_shared_rank(&s_total, lane);  // (a lane's CTA)
    before.x += __reduce_add_sync(0xffffffffu, v.x);
    before.y += __reduce_add_sync(0xffffffffu, v.y);
  }
  int32_t* const kept = p.kept + (int64_t)unit * p.how.most;
  float* const mass_to = p.mass_to.data ? p.mass_to.data + b * p.mass_to.seq_stride + head * p.mass_to.head_stride : nullptr;
  const auto put = [&](uint32_t slot, uint32_t key, bool up, bool eq) {
    const unsigned up_lanes = __ballot_sync(0xffffffffu, up), eq_lanes = __ballot_sync(0xffffffffu, eq), below = (1u << lane) - 1;
    const int e = before.y + __popc(eq_lanes & below);
    if (up || (eq && e < need)) {
      const int i = before.x + __popc(up_lanes & below) + min(e, need);
      kept[i] = (int32_t)slot;
      if (mass_to) mass_to[i] = mass_of(key);
    }
    before.x += __popc(up_lanes);
    before.y += __popc(eq_lanes);
  };
#pragma unroll
  for (int j = 0; j < kHeld; ++j) {
    if (j >= steps) break;
    put(first + j * 32, held[j], ups >> j & 1, eqs >> j & 1);
  }
  for (int j = kHeld; j < steps; ++j) {
    const uint32_t slot = first + j * 32, key = slot < n ? ordered(__ldg(mass + slot)) : 0;
    put(slot, key, above(slot, key), equal(slot, key));
  }
  if (C > 1) cluster.sync();  // (no CTA leaves while its counts may be read)
}

constexpr int kRows = 64;          // rows of a CTA at a time
constexpr int kCopyThreads = 256;
constexpr int64_t kNowhere = INT64_MIN;  // (an offset may be negative: a pool's strides may)

// Blocks: unit * splits + part, which takes every splits-th run of kRows rows.
template <typename V>
__global__ void __launch_bounds__(kCopyThreads) copy_kernel(const __grid_constant__ EvictParams p, const int elem, const int splits) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  __shared__ int64_t s_from[kRows], s_to[kRows];  // bytes; kNowhere: not copied
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
      s_to[tid] = ok ? (there * p.to.page_stride + (i - f * p.to.page_size) * p.to.row_stride + head * p.to.head_stride) * elem : kNowhere;
    }
    __syncthreads();
    constexpr int kAhead = 4;
    for (int v0 = tid; v0 < have * per; v0 += kAhead * kCopyThreads) {
      V k[kAhead], w[kAhead];
      int64_t to[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int v = v0 + u * kCopyThreads, r = v / per, c = (v - r * per) * (int)sizeof(V);
        to[u] = v < have * per ? s_to[r] : kNowhere;
        if (to[u] == kNowhere) continue;
        k[u] = *reinterpret_cast<const V*>(static_cast<const char*>(p.from.k) + s_from[r] + c);
        w[u] = *reinterpret_cast<const V*>(static_cast<const char*>(p.from.v) + s_from[r] + c);
        to[u] += c;
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (to[u] == kNowhere) continue;
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
  while (C < kMaxCluster && (int64_t)units * C * 2 <= sms && slots > (int64_t)C * 1024) C *= 2;
  // (256 sequences of up to 4,096 slots, us: 256 threads of 16 masses each 343, 512 of 8 368; a cluster's, of up to 131,072 slots:
  // 512 threads 45, 256 78.  By what there is room for, as the host does not know the lengths: 256 of 4,096 with room for 32,768 take
  // 402, with room for as many 375, L2 flushed.  Masses past 16 a thread are read again in each pass: eight of 131,072 355, one 50)
  const bool few = C == 1 && slots <= 4096;
  const auto kern = few ? select_kernel<256, 16, 5> : select_kernel<512, 16, 2>;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(units * C);
  cfg.blockDim = dim3(few ? 256 : 512);
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = C;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  e = cudaLaunchKernelEx(&cfg, kern, p);
  if (e != cudaSuccess) return e;
  const int64_t most = std::min<int64_t>(std::min<int64_t>(p.how.most, slots), p.to.table_stride * (int64_t)p.to.page_size);
  const int64_t parts = std::min<int64_t>((most + kRows - 1) / kRows, ((int64_t)sms * 64 + units - 1) / units);
  const int splits = (int)std::max<int64_t>(1, parts);
  if (chunk == 16) return launch_dependent(copy_kernel<uint4>, units * splits, kCopyThreads, stream, p, elem, splits);
  if (chunk == 4) return launch_dependent(copy_kernel<uint32_t>, units * splits, kCopyThreads, stream, p, elem, splits);
  return launch_dependent(copy_kernel<uint16_t>, units * splits, kCopyThreads, stream, p, elem, splits);
}

}  // namespace stride
