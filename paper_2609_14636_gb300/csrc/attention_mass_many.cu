// attention_mass_many.cu -- attention weight of cached slots from many rows at a
// time: drafted trees, chains of new tokens (sm_103a).
//
// The product of 128 slots by up to 128 rows on the tensor cores, turned so that a slot is
// a lane of tensor memory: a slot's sum over the rows is then a thread's own, and
// nothing is joined but two halves of the columns.  One CTA on an SM takes a share of
// the tiles of 128 slots, two at a time; its warps:
//   16   looks up a tile's pages and starts the tensor copies of its keys (boxes of
//        slots by 128 bytes, swizzled), some tiles ahead;
//   17   starts the copies of the rows, a block of whole tokens at a time, and leaves
//        what a column needs beside them: -lse, and which columns count;
//   18   one thread issues the products;
//   0-15 keys from shared memory into tensor memory, where they are the first operand
//        of all the unit's blocks (from shared memory they would be read again for each,
//        which is more of its bandwidth than there is); then scores from tensor
//        memory, weights, sums.  Eight warps for each of the two tiles, four for each
//        half of a block's columns.
// The rows of a unit that fit in one block are copied once for all its tiles.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "attention_line.cuh"
#include "tensor_core.cuh"

namespace stride {
namespace {

constexpr int kSlots = 128;        // of a tile
constexpr int kCols = 128;         // rows of a block at most
constexpr int kTeamWarps = 8;      // of a tile's
constexpr int kWarps = 2 * kTeamWarps + 3, kThreads = kWarps * 32;
constexpr int kMaxStages = 12;
constexpr int kTileCost = 4;       // what a tile costs at least, in blocks

template <int D>
struct Plan {
  static constexpr int kHalves = D / 64;  // 128-byte column groups of a row
  static constexpr int kStage = kHalves * kSlots * 128;  // bytes: a tile of keys, a block of rows
  static constexpr int kStages = D == 128 ? 6 : 12;
  static constexpr size_t kSmem = (size_t)kStages * kStage + 1024;  // (the base rounded up to 1,024)
  // columns of tensor memory: keys of two steps' two tiles, scores of two tiles
  static constexpr int kKeys = D / 2, kScores = 4 * kKeys, kColumns = 512;
  static_assert(kScores + 2 * kCols <= kColumns, "tensor memory");
};

struct Barriers {
  uint64_t k_full[kMaxStages], k_empty[kMaxStages], q_full[kMaxStages], q_empty[kMaxStages], keys[2][2], scores[2], taken[2], drained;
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

// A sequence's tiles of a head, and what one costs.
struct Unit {
  int32_t ctx, n, off, tiles, blocks, cost;
  bool bad;
};
__device__ __forceinline__ Unit unit_of(const MassParams& p, int b, int tokens) {
  const Seq s = sequence(p.a, b);
  Unit u = {s.ctx, s.n, s.off, 0, 0, 0, s.bad || (s.n > 0 && (int64_t)s.ctx + s.n > p.mass.slots)};
  if (!u.bad && u.n > 0) {
    u.tiles = (u.ctx + u.n + kSlots - 1) / kSlots;
    u.blocks = (u.n + tokens - 1) / tokens;
    u.cost = max(kTileCost, u.blocks);
  }
  return u;
}

// A place among the tiles of the call: sequences, of one the heads, of one the tiles.
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
      u = unit_of(p, b, tokens);
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

// tokens: of a block, whose rows are `tokens` times the group; k_stages: of the ring's stages, those of keys.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads, 1)
    mass_many_kernel(const __grid_constant__ MassParams p, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap q_map,
                     const int box, const int page_shift, const int tokens, const int k_stages) {
  using L = Plan<D>;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  extern __shared__ unsigned char dyn[];
  __shared__ Barriers bars;
  __shared__ __align__(16) float s_lse[kMaxStages][kCols];  // -lse log2 e of a block's columns
  __shared__ uint32_t s_counts[kMaxStages][kCols / 32];  // columns that count
  __shared__ uint32_t s_lost[kMaxStages];                // boxes of a tile that have no page
  __shared__ float s_part[2][2][kSlots];
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
      mbar_init(&bars.k_empty[i], 2 * kTeamWarps);
      mbar_init(&bars.q_full[i], 1);
      mbar_init(&bars.q_empty[i], 2 * kTeamWarps + 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bars.keys[0][i], kTeamWarps);
      mbar_init(&bars.keys[1][i], kTeamWarps);
      mbar_init(&bars.scores[i], 1);
      mbar_init(&bars.taken[i], kTeamWarps);
    }
    mbar_init(&bars.drained, 1);
    s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  // ---- this CTA's share ----
  int64_t total = 0, first = 0, of_all;
  const auto cost_of = [&](int b) -> int64_t {
    if (b >= pc.n_seqs) return 0;
    const Unit u = unit_of(p, b, tokens);
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
  Cursor2 at;
  at.b = s_seq;
  at.u = unit_of(p, at.b, tokens);
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

  if (warp == kWarps - 3) {
    // ---- copies of keys ----
    const int boxes = kSlots / box;  // of a tile: at most 16
    const int bx = lane & (boxes - 1);
    int32_t page = 0;
    int row = 0;
    bool some = false;
    const auto look_up = [&](const Cursor2& c) {
      const int slot = c.tile * kSlots + bx * box;
      some = slot < c.u.ctx + c.u.n;
      if (some) {
        const int e = page_shift >= 0 ? slot >> page_shift : slot / pc.page_size;
        row = slot - e * pc.page_size;
        page = __ldg(pc.block_table + (int64_t)c.b * pc.table_stride + e);
      }
    };
    Place k;
    int t = 0;
    if (at.pos < end) look_up(at);
    for (; at.pos < end; ++t) {
      const bool real = some && page >= 0 && page < pc.n_pages, lost = some && !real;
      const int now = page, now_row = row, head = at.head;
      at.on(p, tokens, 1);
      if (at.pos < end) look_up(at);  // (the next tile's, on its way while this one waits for its stage)
      if (t >= k_stages) {
        ok = __all_sync(0xffffffffu, wait(&bars.k_empty[k.st], k.parity ^ 1));
        if (!ok) break;
      }
      const unsigned mine = (1u << boxes) - 1;
      const unsigned gone = __ballot_sync(0xffffffffu, lost) & mine, who = __ballot_sync(0xffffffffu, real) & mine;
      if (lane == 0) {
        s_lost[k.st] = gone;
        mbar_arrive_expect_tx(&bars.k_full[k.st], (uint32_t)(__popc(who) * L::kHalves * box * 128));
      }
      __syncwarp();
      if (lane < boxes && real)
#pragma unroll
        for (int half = 0; half < L::kHalves; ++half)
          copy_box(k_ring + k.st * L::kStage + half * kSlots * 128 + bx * box * 128, &k_map, half * 64, now_row, head, now, &bars.k_full[k.st]);
      __syncwarp();
      k.on(k_stages);
    }
    if (!ok) {  // (never seen.  No copy may outlive the CTA: those on their way end, or take their time)
      if (lane == 0) s_abort = 1;
      volatile int32_t go_on = 0;
      for (int i = t < k_stages ? 0 : t - k_stages; i < t; ++i) mbar_wait_warp(&bars.k_full[i % k_stages], (i / k_stages) & 1, kWaitTimeoutNs, &go_on);
    }
  } else if (warp == kWarps - 2) {
    // ---- copies of rows ----
    Place q;
    int t = 0;
    bool fresh = true;
    while (at.pos < end && ok) {
      const int by = at.step(end);
      if (at.u.blocks > 1 || fresh)
        for (int blk = at.first_block(chain, tokens); blk < at.u.blocks; ++blk, ++t) {
          const int token0 = at.u.off + blk * tokens, cols = min(tokens, at.u.n - blk * tokens) * group;
          float lse[kCols / 32];
#pragma unroll
          for (int j = 0; j < kCols / 32; ++j) {
            const int col = lane + 32 * j, i = col / group;
            lse[j] = -INFINITY;
            if (col < cols) lse[j] = __ldg(p.lse + (int64_t)(token0 + i) * a.Hq + at.head * group + col - i * group);
          }
          if (t >= q_stages) {
            ok = __all_sync(0xffffffffu, wait(&bars.q_empty[q.st], q.parity ^ 1));
            if (!ok) break;
          }
#pragma unroll
          for (int j = 0; j < kCols / 32; ++j) {
            const unsigned counts = __ballot_sync(0xffffffffu, lse[j] != -INFINITY);
            s_lse[q.st][lane + 32 * j] = -lse[j] * kLog2e;
            if (lane == 0) s_counts[q.st][j] = counts;
          }
          __syncwarp();
          if (elect_one()) {
            uint64_t* bar = &bars.q_full[q.st];
            mbar_arrive_expect_tx(bar, (uint32_t)(tokens * group * L::kHalves * 128));
#pragma unroll
            for (int half = 0; half < L::kHalves; ++half)
              copy_box(q_ring + q.st * L::kStage + half * kCols * 128, &q_map, half * 64, at.head * group, token0, 0, bar);
          }
          __syncwarp();
          q.on(q_stages);
        }
      fresh = at.run_ends(by, end);
      at.on(p, tokens, by);
    }
    if (!ok) {
      if (lane == 0) s_abort = 1;
      volatile int32_t go_on = 0;
      for (int i = t < q_stages ? 0 : t - q_stages; i < t; ++i) mbar_wait_warp(&bars.q_full[i % q_stages], (i / q_stages) & 1, kWaitTimeoutNs, &go_on);
    }
  } else if (warp == kWarps - 1) {
    // ---- products ----
    if (elect_one()) {
      const uint32_t q0 = matrix(q_ring, 16);
      Place q;
      uint32_t keys_parity = 0, taken_parity = 0, used = 0;  // bits: buffer and tile; tile
      int buffer = 0;
      bool fresh = true;
      while (at.pos < end && ok) {
        const int by = at.step(end);
        const bool many = at.u.blocks > 1, run_ends = at.run_ends(by, end);
        const int blk0 = at.first_block(chain, tokens);
        for (int blk = blk0; blk < at.u.blocks && ok; ++blk) {
          if (many || fresh) ok = wait(&bars.q_full[q.st], q.parity);
          const uint32_t idesc = product<T>((min(tokens, at.u.n - blk * tokens) * group + 15) & ~15, false);
          for (int h = 0; h < by && ok; ++h) {
            if (blk == blk0) {
              ok = wait(&bars.keys[buffer][h], (keys_parity >> (2 * buffer + h)) & 1);
              keys_parity ^= 1u << (2 * buffer + h);
            }
            if (used >> h & 1) {
              ok = ok && wait(&bars.taken[h], (taken_parity >> h) & 1);
              taken_parity ^= 1u << h;
            }
            if (!ok) break;
            used |= 1u << h;
            fence_after();
            const uint32_t b = q0 + q.st * (L::kStage >> 4), k = tmem + (2 * buffer + h) * L::kKeys, d = tmem + L::kScores + h * kCols;
#pragma unroll
            for (int x = 0; x < D / 16; ++x) mma_ts(d, k + x * 8, b + (x / 4) * (kCols * 128 >> 4) + (x % 4) * 2, idesc, x > 0);
            // (the rows' stage first: whoever has seen the last scores knows that nothing more arrives)
            if (h == by - 1 && (many || run_ends)) commit(&bars.q_empty[q.st]);
            commit(&bars.scores[h]);
          }
          if (many || run_ends) q.on(q_stages);
        }
        fresh = run_ends;
        buffer ^= 1;
        at.on(p, tokens, by);
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
    // ---- weights ----
    const int team = (warp >> 2) & 1, part = warp >> 3, row = (warp & 3) * 32 + lane;  // tile of the step, half of the columns, slot of the tile
    const uint32_t my = tmem + ((uint32_t)(warp & 3) << 21);  // this warp's lanes of tensor memory
    const float scale2 = a.scale * kLog2e;
    Place k, q;
    // Keys of the step's tile of this team into tensor memory (a half of the components); whether this thread's slot has no page.
    // Every warp waits for every tile and lets go of it, in order: a stage's barriers are never a lap ahead of a team that has
    // no tile in a step.
    const auto convert = [&](int by, int buffer) {
      bool lost = false;
      for (int i = 0; i < by; ++i, k.on(k_stages)) {
        if (ok) ok = __all_sync(0xffffffffu, wait(&bars.k_full[k.st], k.parity));
        if (!ok) continue;
        if (i != team) {
          if (lane == 0) mbar_arrive(&bars.k_empty[k.st]);
          continue;
        }
        constexpr int kRegs = D / 4;  // D / 2 components
        uint32_t x[kRegs];
        const uint32_t from = k_ring + k.st * L::kStage + (D == 128 ? part * kSlots * 128 : 0) + row * 128;
#pragma unroll
        for (int c = 0; c < kRegs / 4; ++c) {
          const int chunk = (D == 128 ? 0 : part * 4) + c;
          asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                       : "=r"(x[4 * c]), "=r"(x[4 * c + 1]), "=r"(x[4 * c + 2]), "=r"(x[4 * c + 3])
                       : "r"(from + ((chunk ^ (row & 7)) << 4))
                       : "memory");
        }
        lost = (s_lost[k.st] >> (row / box)) & 1;
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars.k_empty[k.st]);
        tmem_store(my + (2 * buffer + team) * L::kKeys + part * kRegs, x);
        tmem_wait_store();
        fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars.keys[buffer][team]);
      }
      return lost;
    };
    uint32_t scores_parity = 0;
    int buffer = 0;
    bool fresh = true, lost = false, lost_ahead = false;
    Cursor2 ahead = at;
    if (at.pos < end) {
      lost = convert(at.step(end), 0);
      ahead.on(p, tokens, at.step(end));
    }
    // (a warp whose wait has run out goes on without waiting, to the barriers that the others are at)
    while (at.pos < end) {
      const int by = at.step(end);
      if (ahead.pos < end) {
        const int next = ahead.step(end);
        lost_ahead = convert(next, buffer ^ 1);
        ahead.on(p, tokens, next);
      }
      const bool many = at.u.blocks > 1, run_ends = at.run_ends(by, end), mine = team < by;
      const int slot0 = (at.tile + team) * kSlots, back = slot0 + row - at.u.ctx;
      const bool whole = slot0 + kSlots <= at.u.ctx;
      float* const mass = p.mass.data + at.b * p.mass.seq_stride + at.head * p.mass.head_stride + slot0 + row;
      float old = 0.f;
      if (mine && part == 0 && p.decay != 0.f && back < 0) old = *mass;
      float2 sum[2] = {};
      for (int blk = at.first_block(chain, tokens); blk < at.u.blocks && ok; ++blk) {
        const int token0 = blk * tokens, cols = min(tokens, at.u.n - token0) * group;
        const int half = (cols + 63) / 64 * 32, c0 = part * half;  // this warp's columns: 32 or 64 from c0 on
        if (many || fresh) ok = wait(&bars.q_full[q.st], q.parity);
        if (mine) {
          ok = ok && wait(&bars.scores[team], scores_parity);
          scores_parity ^= 1;
        }
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        if (mine) {
          fence_after();
          const float2 sc = make_float2(scale2, scale2);
          const int c1 = min(cols, c0 + half);
#pragma unroll 1
          for (int c = c0; c < c1; c += 32) {
            uint32_t r[32];
            tmem_load32(r, my + L::kScores + team * kCols + c);
            tmem_wait_load();
            if (c + 32 >= c1) {  // (the last)
              fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(&bars.taken[team]);
            }
            uint32_t see = s_counts[q.st][c / 32];
            if (!whole && back >= 0) {
              if (chain) {  // from the first column of a token that is as far on as the slot
                const int from = back > token0 ? min(back - token0, tokens) * group - c : 0;
                see = from >= 32 ? 0 : from > 0 ? see >> from << from : see;
              } else {
                for (uint32_t left = see; left; left &= left - 1) {
                  const int j = __ffs(left) - 1;
                  if (back >= at.u.n || !(__ldg(a.tree_mask + at.u.off + token0 + (c + j) / group) >> back & 1)) see &= ~(1u << j);
                }
              }
            }
            const float4* lse = reinterpret_cast<const float4*>(&s_lse[q.st][c]);
            const bool all_seen = __all_sync(0xffffffffu, see == 0xffffffffu);
#pragma unroll
            for (int j = 0; j < 32; j += 4) {
              const float4 l = lse[j / 4];
              const float2 x0 = __ffma2_rn(make_float2(__uint_as_float(r[j]), __uint_as_float(r[j + 1])), sc, make_float2(l.x, l.y));
              const float2 x1 = __ffma2_rn(make_float2(__uint_as_float(r[j + 2]), __uint_as_float(r[j + 3])), sc, make_float2(l.z, l.w));
              float2 e0 = make_float2(ex2(x0.x), ex2(x0.y)), e1 = make_float2(ex2(x1.x), ex2(x1.y));
              if (!all_seen) {
                e0 = make_float2(see >> j & 1 ? e0.x : 0.f, see >> (j + 1) & 1 ? e0.y : 0.f);
                e1 = make_float2(see >> (j + 2) & 1 ? e1.x : 0.f, see >> (j + 3) & 1 ? e1.y : 0.f);
              }
              sum[0] = __fadd2_rn(sum[0], e0);
              sum[1] = __fadd2_rn(sum[1], e1);
            }
          }
          if (c0 >= c1) {  // (no columns: nothing to read)
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars.taken[team]);
          }
        }
        if (many || run_ends) {
          __syncwarp();
          if (lane == 0) mbar_arrive(&bars.q_empty[q.st]);
          q.on(q_stages);
        }
      }
      if (!ok && lane == 0) s_abort = 1;
      fresh = run_ends;
      // the columns' halves meet
      float w = (sum[0].x + sum[1].x) + (sum[0].y + sum[1].y);
      if (part == 1) s_part[buffer][team][row] = w;
      asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "n"(kTeamWarps * 32) : "memory");
      if (mine && part == 0 && ok) {
        w += s_part[buffer][team][row];
        if (back < 0 && p.decay != 0.f) w = fmaf(p.decay, old, w);
        if (back < at.u.n) *mass = lost ? NAN : w;
        if (lost && back < at.u.n) set_status(a.dev_status, STRIDE_DEV_BAD_LAYOUT);
      }
      lost = lost_ahead;
      buffer ^= 1;
      at.on(p, tokens, by);
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

template <typename T, int D>
cudaError_t run(const MassParams& p, bool bf16, int sms, cudaStream_t stream) {
  using L = Plan<D>;
  const auto kern = mass_many_kernel<T, D>;
  const PagedCache& c = p.a.cache;
  const int box = slots_of_a_box(c.page_size), group = p.a.Hq / c.n_heads, tokens = kCols / group;
  CUtensorMap k_map, q_map;
  if (!describe(&k_map, c.k, bf16, {p.a.D, c.page_size, c.n_heads, c.n_pages}, {c.row_stride, c.head_stride, c.page_stride}, {box, 1, 1}) ||
      !describe(&q_map, p.a.q, bf16, {p.a.D, p.a.Hq, p.a.n_tokens, 1}, {p.a.q_head, p.a.q_tok, 0}, {group, tokens, 1}))
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
  // units of several blocks stream the rows past the keys, others the keys past the rows
  const int64_t mean = (p.a.n_tokens + c.n_seqs - 1) / c.n_seqs;
  const int k_stages = mean > tokens ? L::kStages / 3 : L::kStages * 2 / 3;
  e = cudaLaunchKernelEx(&cfg, kern, p, k_map, q_map, box, page_shift(c.page_size), tokens, k_stages);
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
  if (dtype == STRIDE_DTYPE_BF16)
    return p.a.D <= 64 ? run<__nv_bfloat16, 64>(p, true, sms, stream) : run<__nv_bfloat16, 128>(p, true, sms, stream);
  return p.a.D <= 64 ? run<__half, 64>(p, false, sms, stream) : run<__half, 128>(p, false, sms, stream);
}

}  // namespace stride
