// tree_attention_many.cu -- attention of many rows at a time over a paged cache:
// drafted trees, chains of new tokens (sm_103a).
//
// Blocks of 128 rows by tiles of 64 slots on the tensor cores.  One CTA on an SM
// takes a share of the line of tiles (attention_line.cuh); its warps:
//   4     looks up a tile's pages and starts their tensor copies (a box of up to
//         64 slots by 128 bytes, swizzled), up to five tiles ahead;
//   5     one thread issues the products: scores Q K^T of the next tile, then
//         output += P V of this one (tcgen05, accumulators in tensor memory);
//   0-3   a thread for each row: scores from tensor memory, running maximum and
//         sum, weights P back into tensor memory, where the second product reads
//         them.  Scores and weights have two buffers each, so the products of one
//         tile run while the weights of the next are formed.
// The output is rescaled only where a row's maximum has grown by more than 2^8
// since it was last (weights up to 256 fit both types as well as weights up to 1;
// maximum and sum stay consistent either way).  Slots past the end, and new tokens
// that no row of the block sees, may hold anything: their values are zeroed in
// shared memory before the second product, their scores are masked.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <atomic>
#include <type_traits>

#include "attention_line.cuh"
#include "mbarrier.cuh"

namespace stride {
namespace {

constexpr int kRows = 128;
constexpr int kSlots = 64;
constexpr int kThreads = 192;
constexpr int kMaxWorkers = 152;
constexpr float kGrowth = 8.f;  // log2

// ---- tensor memory and tcgen05 ----
__device__ __forceinline__ void tmem_load32(uint32_t (&r)[32], uint32_t addr) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(addr));
}
__device__ __forceinline__ void tmem_store32(uint32_t addr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(addr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void tmem_wait_load() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_store() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// The barrier's phase ends when all products issued so far by this thread are done.
__device__ __forceinline__ void commit(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
  asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a), "l"(b),
               "r"(idesc), "r"((uint32_t)add)
               : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool add) {
  asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d), "r"(a), "l"(b),
               "r"(idesc), "r"((uint32_t)add)
               : "memory");
}
// A matrix in shared memory of 128-byte rows, swizzled in groups of eight:
// `next` bytes lie between 64-component groups (where components are the rows).
__device__ __forceinline__ uint64_t matrix(uint32_t addr, uint32_t next) {
  return (uint64_t)((addr & 0x3ffff) >> 4) | (uint64_t)(next >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
// Both operands of type T, 32-bit results of M = 128 by N; b_rows: B's rows, not
// its columns, run along the summed dimension.
template <typename T>
__host__ __device__ constexpr uint32_t product(int N, bool b_rows) {
  const uint32_t type = sizeof(T) == 2 && std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
  return 1u << 4 | type << 7 | type << 10 | (b_rows ? 1u << 16 : 0u) | (uint32_t)(N >> 3) << 17 | (uint32_t)(kRows >> 4) << 24;
}

__device__ __forceinline__ void copy_box(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, int c3, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
      "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(smem_u32(bar))
      : "memory");
}

template <typename T>
__device__ __forceinline__ uint32_t pack(float lo, float hi);
template <>
__device__ __forceinline__ uint32_t pack<__nv_bfloat16>(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
template <>
__device__ __forceinline__ uint32_t pack<__half>(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

template <int D>
struct Plan {
  static constexpr int kHalves = D / 64;                    // 128-byte column groups of a row
  static constexpr int kQ = kHalves * kRows * 128;          // bytes
  static constexpr int kKeys = kHalves * kSlots * 128;
  static constexpr int kStage = 2 * kKeys;                  // keys, then values
  static constexpr int kStages = 5;
  static constexpr size_t kSmem = kQ + (size_t)kStages * kStage + 1024;  // (the base rounded up to 1,024)
  // columns of tensor memory: scores (two buffers), output, weights (two)
  static constexpr int kO = 2 * kSlots, kP = kO + D, kColumns = kP + kSlots <= 256 ? 256 : 512;
};

struct Barriers {
  uint64_t full[8], empty[8], scores[2], weights[2], output[2], queries, drained;
};

// What the rows of a unit's block see of its tiles.
struct RowView {
  int lim;        // chain: slots below it
  uint64_t bits;  // tree: new tokens
};

template <typename T, int D>
__global__ void __launch_bounds__(kThreads, 1)
    attention_many_kernel(const AttentionParams p, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map,
                          const int box) {
  using L = Plan<D>;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  extern __shared__ unsigned char dyn[];
  __shared__ int64_t line[kLineSeqs], part[kThreads / 32];
  __shared__ Barriers bars;
  __shared__ int32_t s_lost[8];  // the tile (1-based, of the share) in a stage that has a slot without a page
  __shared__ int32_t s_abort;
  __shared__ uint32_t s_tmem;

  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const Grouping g = {p.Hq / p.cache.n_heads, kRows, kSlots, p.tree_mask == nullptr};
  const PagedCache& pc = p.cache;
  const uint32_t q_smem = (smem_u32(dyn) + 1023) & ~1023u, stages = q_smem + L::kQ;

  if (tid == 0) {
    for (int i = 0; i < L::kStages; ++i) {
      mbar_init(&bars.full[i], 1);
      mbar_init(&bars.empty[i], 1);
      s_lost[i] = 0;
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bars.scores[i], 1);
      mbar_init(&bars.weights[i], 4);
      mbar_init(&bars.output[i], 1);
    }
    mbar_init(&bars.queries, 4);
    mbar_init(&bars.drained, 1);
    s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  const int64_t total = lay_line<kThreads>(p, g, line, part);
  const Span span = span_of(total, blockIdx.x, gridDim.x);
  const Slots slots(p.workspace, gridDim.x, kRows, D);
  if (tid == 0) slots.joined[blockIdx.x] = {0, 0, 0, 0};
  if (span.begin >= span.end) return;  // (all threads alike)
  if (warp == 5) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"(L::kColumns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    fence_before();
  }
  Cursor at = place_in_line(p, g, line, span.begin);
  __syncthreads();
  fence_after();
  const uint32_t tmem = s_tmem;
  const int n = (int)(span.end - span.begin);
  // Waits end: after two seconds, or once another warp's wait has run out.
  const auto wait = [&](uint64_t* bar, uint32_t parity) { return mbar_wait(bar, parity, kWaitTimeoutNs, &s_abort); };
  bool ok = true;

  if (warp == 4) {
    // ---- copies ----
    const int boxes = kSlots / box;  // of a tile's slots: at most 8, so that a lane has one copy
    int t = 0;
    for (; t < n; ++t) {
      const int st = t % L::kStages;
      if (t >= L::kStages) {
        ok = __all_sync(0xffffffffu, wait(&bars.empty[st], (t / L::kStages - 1) & 1));
        if (!ok) break;
      }
      const int end = at.s.bad ? 0 : g.end(at.s, at.block);
      int32_t page = -1;
      int row = 0;
      bool real = false, lost = false;
      if (lane < boxes) {
        const int slot = at.tile * kSlots + lane * box;
        if (slot < end) {
          const int e = slot / pc.page_size;
          row = slot - e * pc.page_size;
          page = __ldg(pc.block_table + (int64_t)at.b * pc.table_stride + e);
          real = page >= 0 && page < pc.n_pages;
          lost = !real;
        }
      }
      const unsigned who = __ballot_sync(0xffffffffu, real);
      if (__any_sync(0xffffffffu, lost) && lane == 0) s_lost[st] = t + 1;
      if (lane == 0) mbar_arrive_expect_tx(&bars.full[st], (uint32_t)(__popc(who) * 2 * L::kHalves * box * 128));
      __syncwarp();
      const int bx = lane % boxes, which = lane / boxes, half = which >> 1;
      page = __shfl_sync(0xffffffffu, page, bx);
      row = __shfl_sync(0xffffffffu, row, bx);
      if (which < 2 * L::kHalves && (who >> bx & 1)) {
        const uint32_t dst = stages + st * L::kStage + (which & 1) * L::kKeys + half * kSlots * 128 + bx * box * 128;
        copy_box(dst, which & 1 ? &v_map : &k_map, half * 64, row, at.head, page, &bars.full[st]);
      }
      at.next(p, g);
    }
    if (!ok) {  // (never seen.  No copy may outlive the CTA: those on their way end, or take their time)
      if (lane == 0) s_abort = 1;
      volatile int32_t go_on = 0;
      for (int k = t < L::kStages ? 0 : t - L::kStages; k < t; ++k)
        mbar_wait_warp(&bars.full[k % L::kStages], (k / L::kStages) & 1, kWaitTimeoutNs, &go_on);
    }
  } else if (warp == 5) {
    // ---- products ----
    if (lane == 0) {
      constexpr uint32_t qk = product<T>(kSlots, false), pv = product<T>(D, true);
      Cursor ahead = at;
      int segment = 0;
      const auto scores = [&](int t, bool first) {
        if (first) ok = ok && wait(&bars.queries, segment++ & 1);
        ok = ok && wait(&bars.full[t % L::kStages], (t / L::kStages) & 1);
        if (!ok) return;
        fence_after();
        const uint32_t k = stages + (t % L::kStages) * L::kStage;
#pragma unroll
        for (int x = 0; x < D / 16; ++x)
          mma_ss(tmem + (t & 1) * kSlots, matrix(q_smem + (x / 4) * kRows * 128 + (x % 4) * 32, 16),
                 matrix(k + (x / 4) * kSlots * 128 + (x % 4) * 32, 16), qk, x > 0);
        commit(&bars.scores[t & 1]);
      };
      scores(0, true);
      bool first = true;
      for (int t = 0; t < n && ok; ++t) {
        const bool last = ahead.tile + 1 == ahead.tiles;  // of its unit
        ahead.next(p, g);
        if (t + 1 < n && !last) scores(t + 1, false);
        ok = ok && wait(&bars.weights[t & 1], (t >> 1) & 1);
        if (!ok) break;
        fence_after();
        const uint32_t v = stages + (t % L::kStages) * L::kStage + L::kKeys;
#pragma unroll
        for (int x = 0; x < kSlots / 16; ++x)
          mma_ts(tmem + L::kO, tmem + L::kP + (t & 1) * (kSlots / 2) + x * 8, matrix(v + x * 16 * 128, kSlots * 128), pv, !first || x > 0);
        commit(&bars.empty[t % L::kStages]);
        commit(&bars.output[t & 1]);
        first = last;
        if (t + 1 < n && last) scores(t + 1, true);
      }
      if (!ok) {
        s_abort = 1;
        volatile int32_t go_on = 0;
        commit(&bars.drained);
        mbar_wait(&bars.drained, 0, kWaitTimeoutNs, &go_on);
      }
    }
    __syncwarp();
  } else {
    // ---- rows ----
    const uint32_t my = tmem + ((uint32_t)(warp * 32) << 16);  // this warp's lanes of tensor memory
    const float scale2 = p.scale * kLog2e;
    RowView view = {0, 0};
    float m = -INFINITY, l = 0.f;
    bool nan = false;
    int first_tile = 0;
    // This thread's row of a unit's queries into shared memory.
    const auto take_queries = [&](const Cursor& u) {
      const int64_t rr = (int64_t)u.block * kRows + tid;
      const int i = (int)(rr / g.group);
      const bool have = i < u.s.n;
      const T* q = static_cast<const T*>(p.q) + (u.s.off + (have ? i : 0)) * p.q_tok + (u.head * g.group + rr % g.group) * p.q_head;
#pragma unroll
      for (int c = 0; c < D / 8; ++c) {
        uint4 x = make_uint4(0, 0, 0, 0);
        if (have && c * 8 < p.D) x = *reinterpret_cast<const uint4*>(q + c * 8);
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(q_smem + (c / 8) * kRows * 128 + tid * 128 + (((c % 8) ^ (tid & 7)) << 4)),
                     "r"(x.x), "r"(x.y), "r"(x.z), "r"(x.w)
                     : "memory");
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars.queries);
    };
    take_queries(at);
    bool fresh = true;
    for (int t = 0; t < n; ++t) {
      const int st = t % L::kStages, b = t & 1;
      if (fresh) {
        fresh = false;
        m = -INFINITY;
        l = 0.f;
        nan = at.s.bad;
        first_tile = at.tile;
        const int i = (int)(((int64_t)at.block * kRows + tid) / g.group);
        const bool have = i < at.s.n;
        view.lim = at.s.ctx + (have ? i + 1 : 0);
        view.bits = have && !g.chain ? __ldg(p.tree_mask + at.s.off + i) : 0;
      }
      ok = wait(&bars.full[st], (t / L::kStages) & 1) && wait(&bars.scores[b], (t >> 1) & 1);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      fence_after();
      nan |= s_lost[st] == t + 1;
      float s[kSlots];
      {
        uint32_t r0[32], r1[32];
        tmem_load32(r0, my + b * kSlots);
        tmem_load32(r1, my + b * kSlots + 32);
        tmem_wait_load();
#pragma unroll
        for (int j = 0; j < 32; ++j) {
          s[j] = __uint_as_float(r0[j]);
          s[32 + j] = __uint_as_float(r1[j]);
        }
      }
      if (at.tile * kSlots + kSlots > at.s.ctx) {  // some slots are new tokens', or past the end
        const int slot0 = at.tile * kSlots;
#pragma unroll
        for (int j = 0; j < kSlots; ++j) {
          const int back = slot0 + j - at.s.ctx;
          const bool seen = g.chain ? slot0 + j < view.lim : back < 0 || (back < at.s.n && ((view.bits >> (back & 63)) & 1));
          if (!seen) s[j] = -INFINITY;
        }
        // values that no row uses become zeros
        const int end = at.s.bad ? 0 : g.end(at.s, at.block), slot = slot0 + (tid & 63), back = slot - at.s.ctx;
        bool out = slot >= end;
        if (!out && !g.chain && back >= 0) {
          uint64_t any = 0;
          const int i0 = (int)((int64_t)at.block * kRows / g.group), i1 = min(at.s.n, (int)(((int64_t)(at.block + 1) * kRows - 1) / g.group) + 1);
          for (int i = i0; i < i1; ++i) any |= __ldg(p.tree_mask + at.s.off + i);
          out = !((any >> (back & 63)) & 1);
        }
        if (out && tid / 64 < L::kHalves) {
          const uint32_t v = stages + st * L::kStage + L::kKeys + (tid / 64) * kSlots * 128 + (tid & 63) * 128;
#pragma unroll
          for (int c = 0; c < 8; ++c) asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(v + c * 16), "r"(0) : "memory");
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      }
      float mx = s[0];
#pragma unroll
      for (int j = 1; j < kSlots; ++j) mx = fmaxf(mx, s[j]);
      mx *= scale2;
      if (scale2 <= 0.f) {  // (the largest score is the smallest product)
        mx = -INFINITY;
#pragma unroll
        for (int j = 0; j < kSlots; ++j) mx = fmaxf(mx, s[j] == -INFINITY ? -INFINITY : s[j] * scale2);
      }
      // the row's reference grows at its first tile that sees anything, then by 2^8 at least
      const bool grows = mx > m + kGrowth || (m == -INFINITY && mx > -INFINITY);
      float by = 1.f;
      if (grows) {
        by = ex2(m - mx);
        m = mx;
        l *= by;
      }
      if (t > 0 && at.tile != first_tile && __any_sync(0xffffffffu, grows)) {
        ok = __all_sync(0xffffffffu, wait(&bars.output[b ^ 1], ((t - 1) >> 1) & 1));
        if (!ok) break;
        fence_after();
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          uint32_t r[32];
          tmem_load32(r, my + L::kO + c * 32);
          tmem_wait_load();
#pragma unroll
          for (int j = 0; j < 32; ++j) r[j] = __float_as_uint(__uint_as_float(r[j]) * by);
          tmem_store32(my + L::kO + c * 32, r);
        }
        tmem_wait_store();
      }
      const float ref = m == -INFINITY ? 0.f : m;
      uint32_t w[32];
#pragma unroll
      for (int j = 0; j < 32; ++j) {
        float a = ex2(fmaf(s[2 * j], scale2, -ref)), c = ex2(fmaf(s[2 * j + 1], scale2, -ref));
        if (scale2 <= 0.f) {  // (a masked score times it is not -inf)
          a = s[2 * j] == -INFINITY ? 0.f : a;
          c = s[2 * j + 1] == -INFINITY ? 0.f : c;
        }
        l += a + c;
        w[j] = pack<T>(a, c);
      }
      if (t >= 2) {  // the product that read this buffer's last weights is done
        ok = __all_sync(0xffffffffu, wait(&bars.output[b], ((t - 2) >> 1) & 1));
        if (!ok) break;
      }
      tmem_store32(my + L::kP + b * (kSlots / 2), w);
      tmem_wait_store();
      fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars.weights[b]);

      const bool unit_ends = at.tile + 1 == at.tiles;
      const Cursor was = at;
      at.next(p, g);
      if (unit_ends || t + 1 == n) {
        if (t + 1 < n) take_queries(at);  // (the scores of the unit's last tile are done with the old ones)
        ok = __all_sync(0xffffffffu, wait(&bars.output[b], (t >> 1) & 1));
        if (!ok) break;
        fence_after();
        const bool starts = first_tile == 0, whole = unit_ends && starts;
        const int64_t rr = (int64_t)was.block * kRows + tid;
        const int i = (int)(rr / g.group);
        const bool have = i < was.s.n;
        const int64_t token = was.s.off + i;
        const int head = was.head * g.group + (int)(rr % g.group);
        float* slot = slots.of(blockIdx.x, starts);
        if (nan) l = NAN;
        const float inv = l == 0.f ? 0.f : 1.f / l;
        T* out = static_cast<T*>(p.out) + (have ? token * p.out_tok + head * p.out_head : 0);
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          uint32_t r[32];
          tmem_load32(r, my + L::kO + c * 32);
          tmem_wait_load();
          if (have && !whole) {
#pragma unroll
            for (int j = 0; j < 32; j += 4)
              *reinterpret_cast<uint4*>(slot + (size_t)tid * D + c * 32 + j) = make_uint4(r[j], r[j + 1], r[j + 2], r[j + 3]);
          } else if (have) {
#pragma unroll
            for (int j = 0; j < 32; j += 8) {
              uint32_t h[4];
#pragma unroll
              for (int x = 0; x < 4; ++x) h[x] = pack<T>(__uint_as_float(r[j + 2 * x]) * inv, __uint_as_float(r[j + 2 * x + 1]) * inv);
              if (c * 32 + j < p.D) *reinterpret_cast<uint4*>(out + c * 32 + j) = make_uint4(h[0], h[1], h[2], h[3]);
            }
          }
          __syncwarp();
        }
        if (have && !whole) {
          slot[(size_t)kRows * D + tid] = m;
          slot[(size_t)kRows * D + kRows + tid] = l;
        } else if (have && p.lse) {
          p.lse[token * p.Hq + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
        }
        fence_before();
        if (tid == 0) {
          if (nan) set_status(p.dev_status, STRIDE_DEV_BAD_LAYOUT);
          if (starts && !unit_ends)
            slots.joined[blockIdx.x] = {last_worker(span, blockIdx.x, span.begin + t + was.tiles - was.tile), was.b, was.block, was.head};
        }
        fresh = true;
      }
    }
    if (!ok && lane == 0) {
      s_abort = 1;
      set_status(p.dev_status, STRIDE_DEV_TIMEOUT);
    }
  }
  fence_before();
  __syncthreads();
  if (warp == 5) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(L::kColumns) : "memory");
  }
}

// cuTensorMapEncodeTiled, from the driver that the runtime has loaded.
using Encode = decltype(&cuTensorMapEncodeTiled);
Encode encoder() {
  static std::atomic<Encode> known{nullptr};
  Encode f = known.load(std::memory_order_relaxed);
  if (f) return f;
  void* sym = nullptr;
  cudaDriverEntryPointQueryResult found;
  if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &sym, 12000, cudaEnableDefault, &found) != cudaSuccess ||
      found != cudaDriverEntryPointSuccess)
    return nullptr;
  f = reinterpret_cast<Encode>(sym);
  known.store(f, std::memory_order_relaxed);
  return f;
}

// The cache as components x rows of a page x heads x pages, read in boxes of 64
// components (128 bytes, swizzled) by `box` rows; components past D are zeros.
bool describe(CUtensorMap* map, const void* base, const AttentionParams& p, int dtype, int box) {
  const Encode encode = encoder();
  if (!encode) return false;
  const PagedCache& c = p.cache;
  const cuuint64_t dims[4] = {(cuuint64_t)p.D, (cuuint64_t)c.page_size, (cuuint64_t)c.n_heads, (cuuint64_t)c.n_pages};
  const cuuint64_t row = (cuuint64_t)((p.D * 2 + 15) / 16 * 16);  // (any stride will do where there is one of a kind)
  const cuuint64_t strides[3] = {c.page_size > 1 ? (cuuint64_t)c.row_stride * 2 : row, c.n_heads > 1 ? (cuuint64_t)c.head_stride * 2 : row,
                                 c.n_pages > 1 ? (cuuint64_t)c.page_stride * 2 : row};
  const cuuint32_t boxes[4] = {64, (cuuint32_t)box, 1, 1}, steps[4] = {1, 1, 1, 1};
  return encode(map, dtype == STRIDE_DTYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, const_cast<void*>(base),
                dims, strides, boxes, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int slots_of_a_box(int page_size) {
  int box = kSlots;
  while (box > 1 && page_size % box != 0) box /= 2;
  return box;
}

template <typename T, int D>
cudaError_t run(const AttentionParams& p, int dtype, int sms, cudaStream_t stream) {
  using L = Plan<D>;
  auto kern = attention_many_kernel<T, D>;
  const int box = slots_of_a_box(p.cache.page_size);
  CUtensorMap k_map, v_map;
  if (!describe(&k_map, p.cache.k, p, dtype, box) || !describe(&v_map, p.cache.v, p, dtype, box)) return cudaErrorInvalidValue;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)L::kSmem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  const int grid = sms < kMaxWorkers ? sms : kMaxWorkers;
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = L::kSmem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  e = cudaLaunchKernelEx(&cfg, kern, p, k_map, v_map, box);
  if (e != cudaSuccess) return e;
  if (p.cache.table_stride * p.cache.page_size <= kSlots) return cudaGetLastError();  // (no unit has two tiles)
  return launch_attention_join(p, dtype, grid, kRows, stream);
}

}  // namespace

size_t attention_many_bytes(int D) {
  return slots_offset(kMaxWorkers) + 2 * kMaxWorkers * slot_floats(kRows, D <= 64 ? 64 : 128) * sizeof(float);
}

bool attention_many_takes(const AttentionParams& p) {
  const PagedCache& c = p.cache;
  const int64_t most = (int64_t)1 << 38;  // (strides of a tensor map: under 2^40 bytes)
  return c.page_size % 8 == 0 && (c.row_stride > 0 && c.row_stride < most) && (c.n_heads == 1 || (c.head_stride > 0 && c.head_stride < most)) &&
         (c.n_pages == 1 || (c.page_stride > 0 && c.page_stride < most));
}

cudaError_t launch_attention_many(const AttentionParams& p, int dtype, int sms, cudaStream_t stream) {
  if (dtype == STRIDE_DTYPE_BF16)
    return p.D <= 64 ? run<__nv_bfloat16, 64>(p, dtype, sms, stream) : run<__nv_bfloat16, 128>(p, dtype, sms, stream);
  return p.D <= 64 ? run<__half, 64>(p, dtype, sms, stream) : run<__half, 128>(p, dtype, sms, stream);
}

}  // namespace stride
