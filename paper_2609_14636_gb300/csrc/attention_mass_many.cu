// attention_mass_many.cu -- attention weight of cached slots from many rows at a
// time: drafted trees, chains of new tokens (sm_103a).
//
// The product of 128 slots by up to 128 rows on the tensor cores, turned so that a slot is
// a lane of tensor memory: a slot's sum over the rows is then a thread's own, and
// nothing is joined but two halves of the columns at most.  One CTA on an SM takes a share of
// the tiles of 128 slots, two at a time; its warps:
//   16   looks up tiles' pages, a run of tiles ahead, and starts the tensor copies of the keys
//        (boxes of slots by 128 bytes, swizzled);
//   17   starts the copies of the rows, a block of whole tokens at a time, and leaves
//        what a column needs beside them: -lse, and which columns count;
//   18, 19  one thread each issues a tile's products, of up to 64 of a block's columns each;
//   0-15 keys from shared memory into tensor memory, where they are the first operand
//        of all the unit's blocks (from shared memory they would be read again for each,
//        which is more of its bandwidth than there is), and scores from tensor
//        memory, weights, sums.
// Where units have many rows (kWide) the exponentials count: each of the sixteen does both, four
// for each tile and half of the columns, whose waits for their next product are filled
// by the three others of a scheduler.  Where they have few blocks, a tile costs its
// way through the CTA: eight bring keys, two steps ahead, eight add up (all sixteen doing
// both, one after the other: 32 trees of 13 tokens 87 us, 79).
// The rows of a unit that fit in one block are copied once for all its tiles.
//
// Measured, us (floor: of bytes at 6,683 GB/s, of products at 1,981 TFLOP/s): 32 trees of 13 tokens, 32 / 8 heads of 128, over up to
// 8,000 slots 78 (55; 4.7 TB/s: the weights' chain of waits, 3,600 clocks for two tiles); 4 chains of 511 over up to 6,000 90
// (35, the exponentials 30 at 32 a clock and SM; 0.78 PFLOP/s: without the exponentials 70, product, scores and sums one after the
// other).  The simple kernel of mma.sync took 313 and 1,126.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cfloat>

#include "attention_line.cuh"
#include "tensor_core.cuh"

namespace stride {
namespace {

constexpr int kSlots = 128;        // of a tile
constexpr int kCols = 128;         // rows of a block at most
constexpr int kPart = 64;          // of them, those of a product at most
constexpr int kTeamWarps = 8;      // of a tile's
constexpr int kWarps = 2 * kTeamWarps + 4, kThreads = kWarps * 32;
constexpr int kMaxStages = 12;
constexpr int kInfos = 4;          // steps that weights may be behind the keys

// kWide: a team's products take three places for their scores in turn, so that two are on their way while one is worked on, and its
// keys have one; else two places each, as the keys count.
template <int D, bool kWide>
struct Plan {
  static constexpr int kHalves = D / 64;  // 128-byte column groups of a row
  static constexpr int kStage = kHalves * kSlots * 128;  // bytes: a tile of keys, a block of rows
  static constexpr int kStages = D == 128 ? 6 : 12;
  static constexpr size_t kSmem = (size_t)kStages * kStage + 1024;  // (the base rounded up to 1,024)
  static constexpr int kKeyPlaces = kWide ? 1 : 2, kScorePlaces = kWide ? 3 : 2;
  // columns of tensor memory: keys of two tiles, scores of two tiles
  static constexpr int kKeys = D / 2, kScores = 2 * kKeyPlaces * kKeys, kColumns = 512;
  static_assert(kScores + 2 * kScorePlaces * kPart <= kColumns, "tensor memory");
};

struct Barriers {
  uint64_t k_full[kMaxStages], k_empty[kMaxStages], q_full[kMaxStages], q_empty[kMaxStages], keys[2][2], read[2][2], scores[2][3], taken[2][3], sums[2], joined[2], info_full[kInfos], info_empty[kInfos], landed, drained[2];
};

// A place in a ring, and the parity of its barriers' phase.
struct Place {
  int st = 0;
  uint32_t parity = 0;
  __device__ __forceinline__ void on(int stages) {
    if (++st == stages) {
      st = 0;
      parity ^= 1;
    }
  }
};

// A sequence's tiles of a head, and what one costs: its blocks, and three at least where all warps take part in a step's start and end
// (two chains of 511 tokens among six of 40 over 4,000 slots, us: at least 1 95, 2 95, 3 79, 4 91; a chain of 1,000 among seven of 13
// over 6,000: 181, 113, 124, 125).  Elsewhere that is done beside the blocks (31 of 8 tokens and a chain of 300 over 4,000: 1 87, 2
// 140, 4 224).
struct Unit {
  int32_t ctx, n, off, tiles, blocks, cost;
  bool bad;
};
template <bool kWide>
__device__ __forceinline__ Unit unit_of(const MassParams& p, int b, int tokens) {
  const Seq s = sequence(p.a, b);
  Unit u = {s.ctx, s.n, s.off, 0, 0, 0, s.bad || (s.n > 0 && (int64_t)s.ctx + s.n > p.mass.slots)};
  if (!u.bad && u.n > 0) {
    u.tiles = (u.ctx + u.n + kSlots - 1) / kSlots;
    u.blocks = (u.n + tokens - 1) / tokens;
    u.cost = max(kWide ? 3 : 1, u.blocks);
  }
  return u;
}

// A place among the tiles of the call: sequences, of one the heads, of one the tiles.
template <bool kWide>
struct Cursor2 {
  int32_t b, head, tile;
  int64_t pos;  // the cost of what lies before it
  Unit u;

  __device__ __forceinline__ void on(const MassParams& p, int tokens, int by) {
    pos += (int64_t)by * u.cost;
    tile += by;
    if (tile < u.tiles) return;
    tile = 0;
    if (++head < p.a.cache.n_heads) return;
    head = 0;
    do {
      if (++b >= p.a.cache.n_seqs) return;  // (past the last tile: pos is the call's cost)
      u = unit_of<kWide>(p, b, tokens);
    } while (u.tiles == 0);
  }
  // Tiles of the step here: two where the unit and the share, which ends at `end`, have them.
  __device__ __forceinline__ int step(int64_t end) const { return tile + 1 < u.tiles && pos + u.cost < end ? 2 : 1; }
  // The block of the first row that may see the step's slots.
  __device__ __forceinline__ int first_block(bool chain, int tokens) const {
    const int back = tile * kSlots - u.ctx;
    return chain && back > 0 ? back / tokens : 0;
  }
  // The step of `by` tiles is the share's last of the unit.
  __device__ __forceinline__ bool run_ends(int by, int64_t end) const { return tile + by >= u.tiles || pos + (int64_t)by * u.cost >= end; }
};

// Columns of a block's halves.
__device__ __forceinline__ int part_of(int cols) { return cols > kPart ? kPart : kPart / 2; }

// A step, as the warps that add up its weights need it.
struct __align__(16) Step {
  int64_t mass;   // where its first slot's is
  int32_t back;   // of the first slot: its place among the new tokens
  int32_t n, off, blk0, blocks;
  int32_t flags;  // tiles, 4: the share's last step of the unit, 8: the share's last
};

// The same, of both tiles, where other warps than those of the weights have its keys.
struct __align__(16) Info {
  Step step;
  uint32_t lost[2];
};

// Sum over the CTA's threads before this one, and of all.
__device__ __forceinline__ int64_t block_scan(int64_t v, int64_t& all, int64_t* part) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int64_t incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t w = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += w;
  }
  __syncthreads();
  if (lane == 31) part[warp] = incl;
  __syncthreads();
  int64_t before = 0;
  all = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) before += part[w];
    all += part[w];
  }
  return before + incl - v;
}

// tokens: of a block, whose rows are `tokens` times the group; k_stages: of the ring's stages, those of keys; both: a copy takes
// both halves of a key's components.
template <typename T, int D, bool kWide>
__global__ void __launch_bounds__(kThreads, 1)
    mass_many_kernel(const __grid_constant__ MassParams p, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap q_map,
                     const int box, const int page_shift, const int tokens, const int k_stages, const bool both) {
  using L = Plan<D, kWide>;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  extern __shared__ unsigned char dyn[];
  __shared__ Barriers bars;
  __shared__ __align__(16) float s_lse[kMaxStages][kCols];  // -lse log2 e of a block's columns
  __shared__ __align__(16) uint32_t s_counts[kMaxStages][kCols / 32];  // columns that count
  __shared__ Step s_step[kMaxStages];         // of the step that starts with a tile
  __shared__ float s_sum[2][kSlots];
  __shared__ uint32_t s_lost[kMaxStages];                // boxes of a tile that have no page
  __shared__ Info s_info[kInfos];                        // of a step (not kWide)
  __shared__ int64_t s_scan[kWarps], s_pos;
  __shared__ int32_t s_seq, s_abort;
  __shared__ uint32_t s_tmem;

  const AttentionParams& a = p.a;
  const PagedCache& pc = a.cache;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int group = a.Hq / pc.n_heads, q_stages = L::kStages - k_stages;
  const bool chain = a.tree_mask == nullptr;
  const uint32_t k_ring = (smem_u32(dyn) + 1023) & ~1023u, q_ring = k_ring + k_stages * L::kStage;

  if (tid == 0) {
    for (int i = 0; i < kMaxStages; ++i) {
      mbar_init(&bars.k_full[i], 1);
      mbar_init(&bars.k_empty[i], kWide ? 2 * kTeamWarps : kTeamWarps);
      mbar_init(&bars.q_full[i], 2);
      mbar_init(&bars.q_empty[i], (kWide ? 2 * kTeamWarps : kTeamWarps) + 2);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bars.keys[0][i], kWide ? kTeamWarps : kTeamWarps / 2);
      mbar_init(&bars.keys[1][i], kWide ? kTeamWarps : kTeamWarps / 2);
      for (int j = 0; j < 2; ++j) mbar_init(&bars.read[i][j], 1);
      for (int j = 0; j < 3; ++j) {
        mbar_init(&bars.scores[i][j], 2);
        mbar_init(&bars.taken[i][j], kTeamWarps / 2);
      }
      if (i == 0) mbar_init(&bars.landed, 1);
      mbar_init(&bars.sums[i], kTeamWarps / 2);
      mbar_init(&bars.joined[i], kTeamWarps / 2);
      mbar_init(&bars.drained[i], 1);
    }
    for (int i = 0; i < kInfos; ++i) {
      mbar_init(&bars.info_full[i], 1);
      mbar_init(&bars.info_empty[i], kTeamWarps);
    }
    s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  // ---- this CTA's share ----
  int64_t total = 0, first = 0, of_all;
  const auto cost_of = [&](int b) -> int64_t {
    if (b >= pc.n_seqs) return 0;
    const Unit u = unit_of<kWide>(p, b, tokens);
    if (u.bad && blockIdx.x == 0) set_status(a.dev_status, STRIDE_DEV_BAD_LAYOUT);
    return (int64_t)u.tiles * u.cost * pc.n_heads;
  };
  int64_t own = cost_of(tid);
  first = block_scan(own, total, s_scan);
  for (int b0 = kThreads; b0 < pc.n_seqs; b0 += kThreads) {
    block_scan(cost_of(b0 + tid), of_all, s_scan);
    total += of_all;
  }
  const int64_t begin = total * blockIdx.x / gridDim.x, end = total * (blockIdx.x + 1) / gridDim.x;
  if (begin >= end) return;  // (all threads alike)
  int64_t before = 0;
  for (int b0 = 0; b0 < pc.n_seqs; b0 += kThreads) {  // (the costs of one round of sequences are at hand)
    if (pc.n_seqs > kThreads) {
      own = cost_of(b0 + tid);
      first = before + block_scan(own, of_all, s_scan);
      before += of_all;
    }
    if (begin >= first && begin < first + own) {
      s_seq = b0 + tid;
      s_pos = first;
    }
  }
  if (warp == kWarps - 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"(L::kColumns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    fence_before();
  }
  __syncthreads();
  fence_after();
  constexpr uint32_t tmem = 0;  // (all columns are this CTA's)
  Cursor2<kWide> at;
  at.b = s_seq;
  at.u = unit_of<kWide>(p, at.b, tokens);
  {  // the first tile that starts at `begin` or after it
    const int64_t tile = (begin - s_pos + at.u.cost - 1) / at.u.cost;
    at.head = (int)(tile / at.u.tiles);
    at.tile = (int)(tile - (int64_t)at.head * at.u.tiles);
    at.pos = s_pos + tile * at.u.cost;
    if (at.head >= pc.n_heads) {  // (past the sequence's last)
      at.head = pc.n_heads - 1;
      at.tile = at.u.tiles;
      at.on(p, tokens, 0);
    }
  }
  // Waits end: after two seconds, or once another warp's wait has run out.
  const auto wait = [&](uint64_t* bar, uint32_t parity) { return mbar_wait(bar, parity, kWaitTimeoutNs, &s_abort); };
  bool ok = true;

  if (warp == kWarps - 4) {
    // ---- copies of keys ----
    const int boxes = kSlots / box;  // of a tile: at most 16
    const int run_tiles = 32 / boxes, my_tile = lane / boxes, bx = lane & (boxes - 1);
    // A run of tiles of a unit and the pages of their boxes, one a lane, looked up a run ahead.
    struct Run {
      Step step;               // of its first tile, without blk0 and flags
      int32_t len, left, head;  // tiles; the share's of the unit from here on
      int32_t page, row;       // (the page's first row of the box)
      bool some, last;         // there is something to read; the share ends with the unit's
    };
    int left = 0;  // tiles of the share in the unit here
    bool last = true;
    const auto enter = [&] {
      if (at.pos >= end) return;
      left = at.u.tiles - at.tile;
      const int64_t cost = end - at.pos;
      last = cost <= (int64_t)left * at.u.cost;
      if (last) left = (int)((cost + at.u.cost - 1) / at.u.cost);
    };
    const auto look_up = [&](Run& x) {
      x.len = min(run_tiles, left);
      x.some = false;
      if (left == 0) return;
      x.left = left;
      x.last = last;
      x.head = at.head;
      x.step = {at.b * p.mass.seq_stride + at.head * p.mass.head_stride + at.tile * kSlots, at.tile * kSlots - at.u.ctx, at.u.n, at.u.off, 0, at.u.blocks, 0};
      x.page = 0;
      const int slot = (at.tile + my_tile) * kSlots + bx * box;
      x.some = my_tile < x.len && slot < at.u.ctx + at.u.n;
      if (x.some) {
        const int e = page_shift >= 0 ? slot >> page_shift : slot / pc.page_size;
        x.row = slot - e * pc.page_size;
        x.page = __ldg(pc.block_table + (int64_t)at.b * pc.table_stride + e);
      }
      at.on(p, tokens, x.len);
      left -= x.len;
      if (left == 0 && !last) enter();
    };
    Place k;
    int t = 0;
    const auto copy = [&](Run& run) {
      const bool real = run.some && run.page >= 0 && run.page < pc.n_pages;
      const unsigned gone = __ballot_sync(0xffffffffu, run.some && !real), who = __ballot_sync(0xffffffffu, real);
      for (int i = 0; i < run.len; ++i) {
        const int rest = run.left - i, by = rest > 1 ? 2 : 1;
        run.step.blk0 = chain && run.step.back > 0 ? run.step.back / tokens : 0;
        run.step.flags = by | (rest <= by ? 4 : 0) | (rest <= by && run.last ? 8 : 0);
        if (t >= k_stages) {
          ok = __all_sync(0xffffffffu, wait(&bars.k_empty[k.st], k.parity ^ 1));
          if (!ok) return;
        }
        uint64_t* bar = &bars.k_full[k.st];
        // (a lane for each box: 1,000 clocks for eight of 16 slots, all by one thread, with the pages from the lanes, 1,400; 32 trees of
        // 13 tokens 87 us, 96)
        if (elect_one()) {
          const unsigned mine = (1u << boxes) - 1;
          // (before the arrival, which publishes them: a tile without pages has no bytes to come, and its phase ends there)
          s_lost[k.st] = gone >> (i * boxes) & mine;
          s_step[k.st] = run.step;
          mbar_arrive_expect_tx(bar, (uint32_t)(__popc(who >> (i * boxes) & mine) * L::kHalves * box * 128));
        }
        __syncwarp();
        if (my_tile == i && real) {
          const uint32_t there = k_ring + k.st * L::kStage + bx * L::kHalves * box * 128;  // (a box's halves side by side)
          if (L::kHalves == 2 && both) {
            copy_box(there, &k_map, 0, run.row, 0, run.head, run.page, bar);
          } else {
#pragma unroll
            for (int half = 0; half < L::kHalves; ++half) copy_box(there + half * box * 128, &k_map, half * 64, run.row, run.head, run.page, bar);
          }
        }
        __syncwarp();
        run.step.mass += kSlots;
        run.step.back += kSlots;
        k.on(k_stages);
        ++t;
      }
    };
    enter();
    Run x0, x1;  // (by name: registers that move wait for their loads)
    look_up(x0);
    while (true) {
      look_up(x1);
      copy(x0);
      if (!ok || !x1.len) break;
      look_up(x0);
      copy(x1);
      if (!ok || !x0.len) break;
    }
    if (!ok && lane == 0) s_abort = 1;
    {  // (no copy may outlive the CTA, whatever the others did: those on their way end, or take their time)
      volatile int32_t go_on = 0;
      for (int i = t < k_stages ? 0 : t - k_stages; i < t; ++i) mbar_wait_warp(&bars.k_full[i % k_stages], (i / k_stages) & 1, kWaitTimeoutNs, &go_on);
    }
  } else if (warp == kWarps - 3) {
    // ---- copies of rows ----
    // (A block's -lse are on their way while the one before waits for its stage.)
    int at_lse[kCols / 32];  // of a column: where its lse is past the block's first
#pragma unroll
    for (int j = 0; j < kCols / 32; ++j) {
      const int col = lane + 32 * j, i = col / group;
      at_lse[j] = i * a.Hq + col - i * group;
    }
    Place q;
    int t = 0;
    bool fresh = true;
    // The block at hand; the next.
    int blk = 0, by = 0;
    const auto enter = [&] {  // the step at `at`
      if (at.pos >= end) return false;
      by = at.step(end);
      blk = at.first_block(chain, tokens);
      return true;
    };
    const auto fetch = [&](float (&lse)[kCols / 32]) {
      const int cols = min(tokens, at.u.n - blk * tokens) * group;
      const float* from = p.lse + (int64_t)(at.u.off + blk * tokens) * a.Hq + at.head * group;
#pragma unroll
      for (int j = 0; j < kCols / 32; ++j) {
        lse[j] = -INFINITY;
        if (lane + 32 * j < cols) lse[j] = __ldg(from + at_lse[j]);
      }
    };
    // On to the next block that is copied; false: none.
    const auto on = [&] {
      if (++blk < at.u.blocks) return true;
      while (true) {
        fresh = at.run_ends(by, end);
        at.on(p, tokens, by);
        if (!enter()) return false;
        if (at.u.blocks > 1 || fresh) return true;
      }
    };
    float lse[kCols / 32], next[kCols / 32];
    bool more = enter();
    if (more) fetch(lse);
    uint32_t landed_parity = 0;
    while (more) {
      const int head = at.head * group, token0 = at.u.off + blk * tokens, cols = min(tokens, at.u.n - blk * tokens) * group;
      more = on();
      if (more) fetch(next);
      if (t >= q_stages) {
        ok = __all_sync(0xffffffffu, wait(&bars.q_empty[q.st], q.parity ^ 1));
        if (!ok) break;
      }
      // Rows past the block's last, up to a whole run of 32 columns, are its last again, and their columns' -lse is the lowest number:
      // weights of 0.  They are added only where all rows of the run count and see the slot, the last among them, so that a score
      // of theirs that is infinite or NaN makes the sum no other than that row's own does.  (Zeros, or a row that need not see the
      // slot, would make NaN of a key's infinities.)
      uint64_t* bar = &bars.q_full[q.st];
      const bool ragged = cols % 32 != 0;
      const uint32_t to = q_ring + q.st * L::kStage;
      if (elect_one()) {
        uint64_t* land = ragged ? &bars.landed : bar;
        mbar_arrive_expect_tx(land, (uint32_t)(tokens * group * L::kHalves * 128));
#pragma unroll
        for (int half = 0; half < L::kHalves; ++half) copy_box(to + half * kCols * 128, &q_map, half * 64, head, token0, 0, land);
      }
      __syncwarp();
#pragma unroll
      for (int j = 0; j < kCols / 32; ++j) {
        const unsigned counts = __ballot_sync(0xffffffffu, lse[j] != -INFINITY);
        s_lse[q.st][lane + 32 * j] = lane + 32 * j < cols ? -lse[j] * kLog2e : -FLT_MAX;
        if (lane == 0) s_counts[q.st][j] = counts;
        lse[j] = next[j];
      }
      if (ragged) {
        ok = __all_sync(0xffffffffu, wait(&bars.landed, landed_parity));
        landed_parity ^= 1;
        if (!ok) {
          ++t;
          break;
        }
        const int last = cols - 1;
        for (int i = cols * 8 + lane; i < ((cols + 31) & ~31) * 8; i += 32) {
          const int chunk = last * 8 + ((i ^ i >> 3 ^ last) & 7);  // (a row's chunks are exchanged by its number)
#pragma unroll
          for (int half = 0; half < L::kHalves; ++half) {
            uint32_t w[4];
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
                         : "r"(to + half * kCols * 128 + chunk * 16)
                         : "memory");
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + half * kCols * 128 + i * 16), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3])
                         : "memory");
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(bar);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(bar);
      q.on(q_stages);
      ++t;
    }
    if (!ok && lane == 0) s_abort = 1;
    {
      volatile int32_t go_on = 0;
      for (int i = t < q_stages ? 0 : t - q_stages; i < t; ++i) mbar_wait_warp(&bars.q_full[i % q_stages], (i / q_stages) & 1, kWaitTimeoutNs, &go_on);
    }
  } else if (warp >= kWarps - 2) {
    // ---- products ----
    if (elect_one()) {
      const int team = warp - (kWarps - 2);
      const uint32_t q0 = matrix(q_ring, 16);
      Place q;
      uint32_t keys_parity = 0;  // bits: places of keys
      Place score;               // of the next product
      int buffer = 0;
      bool fresh = true;
      while (at.pos < end && ok) {
        const int by = at.step(end);
        const bool many = at.u.blocks > 1, run_ends = at.run_ends(by, end), mine = team < by;
        if (mine) {
          ok = wait(&bars.keys[buffer][team], keys_parity >> buffer & 1);
          keys_parity ^= 1u << buffer;
        }
        for (int blk = at.first_block(chain, tokens); blk < at.u.blocks && ok; ++blk) {
          if (many || fresh) ok = wait(&bars.q_full[q.st], q.parity);
          const int cols = min(tokens, at.u.n - blk * tokens) * group, wide = kWide ? part_of(cols) : kPart;
          if (!mine) {
            if (ok && (many || run_ends)) mbar_arrive(&bars.q_empty[q.st]);
          } else {
#pragma unroll
            for (int part = 0; part < 2; ++part) {
              const int c = part * wide;
              if (c >= cols || !ok) break;
              const int place = score.st;
              ok = wait(&bars.taken[team][place], score.parity ^ 1);
              if (!ok) break;
              fence_after();
              const uint32_t idesc = product<T>((min(cols - c, wide) + 31) & ~31, false);
              const uint32_t b = q0 + q.st * (L::kStage >> 4) + (c * 128 >> 4), k = tmem + (2 * buffer + team) * L::kKeys;
              const uint32_t d = tmem + L::kScores + (team * L::kScorePlaces + place) * kPart;
#pragma unroll
              for (int x = 0; x < D / 16; ++x) mma_ts(d, k + x * 8, b + (x / 4) * (kCols * 128 >> 4) + (x % 4) * 2, idesc, x > 0);
              // (the stage and the keys first: whoever has seen the last scores knows that nothing more arrives)
              if (c + wide >= cols) {
                if (many || run_ends) commit(&bars.q_empty[q.st]);
                if (blk + 1 >= at.u.blocks) commit(&bars.read[buffer][team]);
              }
              commit(&bars.scores[team][place]);
              mbar_arrive(&bars.scores[team][place]);  // (what this thread knows, that -lse are there, goes with them)
              score.on(L::kScorePlaces);
            }
          }
          if (many || run_ends) q.on(q_stages);
        }
        fresh = run_ends;
        buffer ^= L::kKeyPlaces - 1;
        at.on(p, tokens, by);
      }
      if (!ok) s_abort = 1;
      volatile int32_t go_on = 0;  // (nor a product tensor memory)
      commit(&bars.drained[team]);
      mbar_wait(&bars.drained[team], 0, kWaitTimeoutNs, &go_on);
    }
    __syncwarp();
  } else {
    // ---- weights ----
    // tile of the step, half of the columns (kWide; else whether the keys' or the weights'), slot of the tile
    const int team = (warp >> 2) & 1, part = warp >> 3, row = (warp & 3) * 32 + lane;
    const int box_shift = __ffs(box) - 1;
    const uint32_t my = tmem + ((uint32_t)(warp & 3) << 21);  // this warp's lanes of tensor memory
    const float2 scale2 = make_float2(a.scale * kLog2e, a.scale * kLog2e);
    Place k, q;
    // What is at hand of a step.
    struct Now {
      float* mass;                // of this thread's slot
      int32_t back, n, off, blk0, blocks, flags;
      bool lost;                  // the slot has no page
    };
    const auto now_of = [&](const Step& s) {
      const Now x = {p.mass.data + s.mass + team * kSlots + row, s.back + team * kSlots + row, s.n, s.off, s.blk0, s.blocks, s.flags, false};
      return x;
    };
    // Half of the components of this thread's slot, from the stage at hand into tensor memory.
    const auto move = [&](int half, int buffer) {
      constexpr int kRegs = D / 4;  // D / 2 components
      uint32_t r[kRegs];
      const uint32_t from = k_ring + k.st * L::kStage + (((row >> box_shift) * L::kHalves + (D == 128 ? half : 0)) * box + (row & (box - 1))) * 128;
#pragma unroll
      for (int c = 0; c < kRegs / 4; ++c) {
        const int chunk = (D == 128 ? 0 : half * 4) + c;
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(r[4 * c]), "=r"(r[4 * c + 1]), "=r"(r[4 * c + 2]), "=r"(r[4 * c + 3])
                     : "r"(from + ((chunk ^ (row & 7)) << 4))
                     : "memory");
      }
      tmem_store(my + (2 * buffer + team) * L::kKeys + half * kRegs, r);
    };
    // The next step, its keys of this team's tile into tensor memory, where products have read the ones before them.
    // Every warp waits for every tile and lets go of it, in order: a stage's barriers are never a lap ahead of a team that has
    // no tile in a step.
    uint32_t read_parity = 3;  // bits: a buffer (nothing to wait for at first)
    const auto convert = [&](int buffer, Info* info) {
      Now x = {};
      int by = 1;
      for (int i = 0; i < by; ++i, k.on(k_stages)) {
        ok = ok && __all_sync(0xffffffffu, wait(&bars.k_full[k.st], k.parity));
        if (!ok) return x;
        if (i == 0) {
          x = now_of(s_step[k.st]);
          by = x.flags & 3;
          if (info) info->step = s_step[k.st];
        }
        if (info) info->lost[i] = s_lost[k.st];
        if (i == team) {
          ok = __all_sync(0xffffffffu, wait(&bars.read[buffer][team], read_parity >> buffer & 1));
          read_parity ^= 1u << buffer;
          if (!ok) return x;
          fence_after();
          if (kWide) {
            move(part, buffer);
          } else {
            move(0, buffer);
            move(1, buffer);
          }
          x.lost = (s_lost[k.st] >> (row >> box_shift)) & 1;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars.k_empty[k.st]);
      }
      if (team < by) {
        tmem_wait_store();
        fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars.keys[buffer][team]);
      }
      return x;
    };
    float2 sum[2];  // of this thread's slot
    // Adds the weights of columns [c0, c1) of a block, up to 64 of one product, whose scores are in `place`.
    const auto weigh = [&](const Now& now, int blk, int cols, int c0, int c1, int place) {
      const int back = now.back, token0 = blk * tokens;
      const bool whole = back - row + kSlots <= 0;
      uint64_t* const taken = &bars.taken[team][place];
      const uint32_t my_scores = my + L::kScores + (team * L::kScorePlaces + place) * kPart;
      fence_after();
      // (log2 e is in scale's and lse's factors: their roundings make 2^-24 (|score| + |lse|) of a weight, as lse's own in 32 bits does
      // and a score's.  The difference first, its product after it: 32 trees of 13 tokens 82 us instead of 78, 4 chains of 511 94
      // instead of 91; a factor of each column for what lse's leaves 82 and 98.)
      const auto add = [&](const uint32_t (&r)[32], const float4* lse) {
#pragma unroll
        for (int j = 0; j < 32; j += 4) {
          const float4 l = lse[j / 4];
          const float2 x0 = __ffma2_rn(make_float2(__uint_as_float(r[j]), __uint_as_float(r[j + 1])), scale2, make_float2(l.x, l.y));
          const float2 x1 = __ffma2_rn(make_float2(__uint_as_float(r[j + 2]), __uint_as_float(r[j + 3])), scale2, make_float2(l.z, l.w));
          sum[0] = __fadd2_rn(sum[0], make_float2(ex2(x0.x), ex2(x0.y)));
          sum[1] = __fadd2_rn(sum[1], make_float2(ex2(x1.x), ex2(x1.y)));
        }
      };
      // all columns count for all of the warp's slots (in a chain: those of tokens past the last of them)
      bool all = kWide && c1 - c0 > 32 && s_counts[q.st][c0 / 32] == 0xffffffffu && s_counts[q.st][c0 / 32 + 1] == 0xffffffffu >> (c0 + kPart - c1);
      if (all && !whole) all = __all_sync(0xffffffffu, back < 0 || (chain && back <= token0 + c0 / group));
      if (all) {
        uint32_t r0[32], r1[32];
        tmem_load32(r0, my_scores);
        tmem_load32(r1, my_scores + 32);
        tmem_wait_load();
        fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(taken);
        add(r0, reinterpret_cast<const float4*>(&s_lse[q.st][c0]));
        add(r1, reinterpret_cast<const float4*>(&s_lse[q.st][c0 + 32]));
      } else
#pragma unroll 1
      for (int c = c0; c < c1; c += 32) {
        const uint32_t from = my_scores + c - c0;
        const float4* lse = reinterpret_cast<const float4*>(&s_lse[q.st][c]);
        const int n = min(c1 - c, 32);  // columns
        const bool last = c + 32 >= c1;
        const uint32_t every = 0xffffffffu >> (32 - n);
        uint32_t see = s_counts[q.st][c / 32];
        bool full = see == every, none = see == 0;
        if (!whole) {
          if (back >= 0) {
            if (chain) {  // from the first column of a token that is as far on as the slot
              const int first = back > token0 ? min(back - token0, tokens) * group - c : 0;
              see = first >= 32 ? 0 : first > 0 ? see >> first << first : see;
            } else {
              const int last_token = (min(c + 32, cols) - 1) / group;
              uint32_t by_bits = 0;
              for (int i = c / group; i <= last_token; ++i) {  // (tokens with a column among these)
                const int first = max(i * group - c, 0), upto = min((i + 1) * group - c, 32);
                if (__ldg(a.tree_mask + now.off + token0 + i) >> (back & 63) & 1) by_bits |= (0xffffffffu >> (32 - (upto - first))) << first;
              }
              see &= by_bits;
            }
          }
          full = __all_sync(0xffffffffu, see == every);
          none = __all_sync(0xffffffffu, see == 0);
        }
        if (none) {
          if (last) {
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(taken);
          }
          continue;
        }
        if (full) {  // (columns past the last have weights of 0)
          uint32_t r[32];
          tmem_load32(r, from);
          tmem_wait_load();
          if (last) {
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(taken);
          }
          add(r, lse);
          continue;
        }
        // (eight columns at a time, in a loop: unrolled with the others' this took so many registers that the whole kernel
        // was slower: 32 trees of 13 tokens 147 us)
#pragma unroll 1
        for (int j = 0; j < n; j += 8) {
          uint32_t r[8];
          __syncwarp();
          tmem_load8(r, from + j);
          tmem_wait_load();
          if (last && j + 8 >= n) {
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(taken);
          }
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float e = ex2(fmaf(__uint_as_float(r[i]), scale2.x, reinterpret_cast<const float*>(lse)[j + i]));
            sum[i & 1].x += see >> (j + i) & 1 ? e : 0.f;
          }
        }
      }
    };
    // (A load behind a branch was waited for there.)
    const auto old_mass = [&](const Now& now, bool mine) {
      float x = 0.f;
      asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %2, 0;\n @p ld.global.f32 %0, [%1];\n}"
                   : "+f"(x)
                   : "l"(now.mass), "r"((uint32_t)(mine && p.decay != 0.f && now.back < 0))
                   : "memory");
      return x;
    };
    const auto put = [&](const Now& now, float w, float old) {
      if (now.back < 0 && p.decay != 0.f) w = fmaf(p.decay, old, w);
      if (now.back < now.n) *now.mass = now.lost ? NAN : w;
      if (now.lost && now.back < now.n) set_status(a.dev_status, STRIDE_DEV_BAD_LAYOUT);
    };
    Place score;  // of the team's next product
    bool fresh = true;
    if (kWide) {
      uint32_t sums_parity = part;  // (the second half's: the first half's have been read)
      if (at.pos < end) {
        Now now = convert(0, nullptr), next = now;
        while (ok) {
          const bool ends = now.flags & 8, many = now.blocks > 1, run_ends = now.flags & 4, mine = team < (now.flags & 3);
          const float old = old_mass(now, mine && part == 0);
          sum[0] = sum[1] = make_float2(0.f, 0.f);
          for (int blk = now.blk0; blk < now.blocks && ok; ++blk) {
            const int cols = min(tokens, now.n - blk * tokens) * group;
            const int wide = part_of(cols), c0 = part * wide, c1 = min(cols, c0 + wide);  // this warp's columns: up to 32 or 64
            // (Where a half has no columns, in a unit's last block, the keys of the team's next step wait for all products of this
            // one: a place's barrier is never a lap ahead of a half.)
            Place own = score;  // of this half's product
            if (part == 1) own.on(L::kScorePlaces);
            if (mine && c0 < c1)
              ok = __all_sync(0xffffffffu, wait(&bars.scores[team][own.st], own.parity));
            else if (many || fresh)
              ok = __all_sync(0xffffffffu, wait(&bars.q_full[q.st], q.parity));
            if (!ok) break;
            if (mine) {
              score.on(L::kScorePlaces);
              if (cols > wide) score.on(L::kScorePlaces);
              if (c0 < c1) weigh(now, blk, cols, c0, c1, own.st);
            }
            if (many || run_ends) {
              __syncwarp();
              if (lane == 0) mbar_arrive(&bars.q_empty[q.st]);
              q.on(q_stages);
            }
          }
          if (!ends) next = convert(0, nullptr);
          if (!ok) break;
          fresh = run_ends;
          if (mine) {  // the columns' halves meet
            float w = (sum[0].x + sum[1].x) + (sum[0].y + sum[1].y);
            ok = __all_sync(0xffffffffu, wait(part == 0 ? &bars.sums[team] : &bars.joined[team], sums_parity));
            sums_parity ^= 1;
            if (!ok) break;
            if (part == 1) {
              s_sum[team][row] = w;
              __syncwarp();
              if (lane == 0) mbar_arrive(&bars.sums[team]);
            } else {
              w += s_sum[team][row];
              __syncwarp();
              if (lane == 0) mbar_arrive(&bars.joined[team]);
              put(now, w, old);
            }
          }
          if (ends) break;
          now = next;
        }
      }
    } else if (at.pos < end) {
      Place info;
      if (part == 1) {  // keys, up to two steps ahead of their products
        bool ends = false;
        for (int buffer = 0; !ends; buffer ^= 1) {
          Info x;
          const Now now = convert(buffer, &x);
          if (!ok) break;
          ends = now.flags & 8;
          if (warp == kTeamWarps) {  // (one warp leaves what the weights need: the stages are let go of)
            ok = __all_sync(0xffffffffu, wait(&bars.info_empty[info.st], info.parity ^ 1));
            if (!ok) break;
            if (lane == 0) {
              s_info[info.st] = x;
              mbar_arrive(&bars.info_full[info.st]);
            }
            __syncwarp();
            info.on(kInfos);
          }
        }
      } else {
        bool ends = false;
        while (!ends) {
          ok = __all_sync(0xffffffffu, wait(&bars.info_full[info.st], info.parity));
          if (!ok) break;
          Now now = now_of(s_info[info.st].step);
          now.lost = (s_info[info.st].lost[team] >> (row >> box_shift)) & 1;
          __syncwarp();
          if (lane == 0) mbar_arrive(&bars.info_empty[info.st]);
          info.on(kInfos);
          ends = now.flags & 8;
          const bool many = now.blocks > 1, run_ends = now.flags & 4, mine = team < (now.flags & 3);
          const float old = old_mass(now, mine);
          sum[0] = sum[1] = make_float2(0.f, 0.f);
          for (int blk = now.blk0; blk < now.blocks && ok; ++blk) {
            const int cols = min(tokens, now.n - blk * tokens) * group;
            if (mine) {
              for (int c0 = 0; c0 < cols && ok; c0 += kPart) {
                ok = __all_sync(0xffffffffu, wait(&bars.scores[team][score.st], score.parity));
                if (ok) weigh(now, blk, cols, c0, min(cols, c0 + kPart), score.st);
                score.on(L::kScorePlaces);
              }
            } else if (many || fresh) {
              ok = __all_sync(0xffffffffu, wait(&bars.q_full[q.st], q.parity));
            }
            if (!ok) break;
            if (many || run_ends) {
              __syncwarp();
              if (lane == 0) mbar_arrive(&bars.q_empty[q.st]);
              q.on(q_stages);
            }
          }
          if (!ok) break;
          fresh = run_ends;
          if (mine) put(now, (sum[0].x + sum[1].x) + (sum[0].y + sum[1].y), old);
        }
      }
    }
    if (!ok && lane == 0) {
      s_abort = 1;
      set_status(a.dev_status, STRIDE_DEV_TIMEOUT);
    }
  }
  fence_before();
  __syncthreads();
  if (warp == kWarps - 1) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(L::kColumns) : "memory");
  }
}

int slots_of_a_box(int page_size) {
  int box = kSlots;
  while (box > 1 && page_size % box != 0) box /= 2;
  return box;
}

template <typename T, int D, bool kWide>
cudaError_t run(const MassParams& p, bool bf16, int sms, cudaStream_t stream) {
  using L = Plan<D, kWide>;
  const auto kern = mass_many_kernel<T, D, kWide>;
  const PagedCache& c = p.a.cache;
  const int box = slots_of_a_box(c.page_size), group = p.a.Hq / c.n_heads, tokens = kCols / group;
  CUtensorMap k_map, q_map;
  const bool both = p.a.D == 128;  // (of fewer components what follows them would be read)
  if (!(both ? describe<5>(&k_map, c.k, bf16, {64, c.page_size, 2, c.n_heads, c.n_pages}, {c.row_stride, 64, c.head_stride, c.page_stride},
                           {box, 2, 1, 1})
             : describe<4>(&k_map, c.k, bf16, {p.a.D, c.page_size, c.n_heads, c.n_pages}, {c.row_stride, c.head_stride, c.page_stride},
                           {box, 1, 1})) ||
      !describe<4>(&q_map, p.a.q, bf16, {p.a.D, p.a.Hq, p.a.n_tokens, 1}, {p.a.q_head, p.a.q_tok, 0}, {group, tokens, 1}))
    return cudaErrorInvalidValue;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)L::kSmem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)std::min<int64_t>(sms, most_tiles(p.a, 1 << 30, kSlots)));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = L::kSmem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  // units of several blocks stream the rows past the keys, others the keys past the rows (chains of 511 tokens, us: 2 stages of keys 97,
  // 3 99, 4 105; trees of 13 72, 68, 68, of 5 70)
  const int64_t mean = (p.a.n_tokens + c.n_seqs - 1) / c.n_seqs;
  const int k_stages = mean > tokens ? L::kStages / 3 : L::kStages * 2 / 3;
  e = cudaLaunchKernelEx(&cfg, kern, p, k_map, q_map, box, page_shift(c.page_size), tokens, k_stages, both);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

bool attention_mass_many_takes(const MassParams& p) {
  const PagedCache& c = p.a.cache;
  const int64_t most = (int64_t)1 << 38;  // (strides of a tensor map: under 2^40 bytes)
  const auto fits = [&](int64_t stride, int64_t n) { return n <= 1 || (stride > 0 && stride < most); };
  return c.page_size % 8 == 0 && p.a.Hq / c.n_heads <= kCols && fits(c.row_stride, c.page_size) && fits(c.head_stride, c.n_heads) &&
         fits(c.page_stride, c.n_pages) && fits(p.a.q_head, p.a.Hq) && fits(p.a.q_tok, p.a.n_tokens);
}

cudaError_t launch_attention_mass_many(const MassParams& p, int dtype, int sms, cudaStream_t stream) {
  // By the mean of rows a sequence: all warps add up from two blocks on (a sequence's rows, us else, so: 64 68 106, 128 78 111, 256
  // 124 139, 384 97 94, 512 122 109, 2,044 130 97; 4 to 32 sequences of 4,000 slots).
  const bool wide = ((p.a.n_tokens + p.a.cache.n_seqs - 1) / p.a.cache.n_seqs) * (p.a.Hq / p.a.cache.n_heads) > 2 * kCols;
  const bool bf16 = dtype == STRIDE_DTYPE_BF16;
  const auto of = [&](auto type) {
    using T = decltype(type);
    if (p.a.D <= 64) return wide ? run<T, 64, true>(p, bf16, sms, stream) : run<T, 64, false>(p, bf16, sms, stream);
    return wide ? run<T, 128, true>(p, bf16, sms, stream) : run<T, 128, false>(p, bf16, sms, stream);
  };
  return bf16 ? of(__nv_bfloat16()) : of(__half());
}

}  // namespace stride
