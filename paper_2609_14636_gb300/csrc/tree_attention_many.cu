// tree_attention_many.cu -- attention of many rows at a time over a paged cache:
// drafted trees, chains of new tokens (sm_103a).
//
// Blocks of 128 rows by tiles of 64 slots on the tensor cores.  One CTA on an SM
// takes a share of the line of tiles (attention_line.cuh); its warps:
//   8, 9  look up a tile's pages and start the tensor copies of its keys and its
//         values (boxes of up to 64 slots by 128 bytes, swizzled), up to six tiles
//         ahead;
//   10    one thread issues the products: scores Q K^T two tiles ahead, as soon as
//         their place is free, and output += P V (tcgen05, accumulators in tensor
//         memory).  The queries are an operand in tensor memory too: read from
//         shared memory for each tile they took more of its bandwidth than the
//         keys;
//   0-7   two teams of a thread for each row, which take the even and the odd
//         tiles: scores from tensor memory, running maximum and sum, weights P
//         back into tensor memory, where the second product reads them.  Each
//         team has scores, weights and an output of its own, as if the tiles were
//         two sequences, joined where the unit or the share ends: nothing of one
//         tile waits for the other's.
// The output is rescaled only where a row's maximum has grown by more than 2^8 (half:
// 2^2, see kGrowth) since it was last: maximum and sum stay consistent either way.
// The weights are rounded to the values' type, as tcgen05 wants both operands of one
// type; their sum is of the unrounded ones.  (What the rounding leaves, as a second
// operand, has no place in tensor memory, and its product would be half as much work
// again.)  Slots past the end, and new tokens that no row of the block sees, may hold
// anything: their values are zeroed in shared memory before the second product, their
// scores are masked.  What bounds it is the latency of a team's chain of steps for a
// tile (wait, load, maximum, exponentials, store, arrive): in chains the tensor pipe
// is 40 % busy, at 1.5 instructions a clock.  GB300, 32 / 8 heads of 128, bf16: 32
// trees of 13 tokens over up to 8,000 slots 128 us (5.5 TB/s), 4 chains of 511 over up
// to 6,000 170 us (825 TFLOP/s).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <type_traits>

#include "attention_line.cuh"
#include "mbarrier.cuh"
#include "tensor_core.cuh"

namespace stride {
namespace {

constexpr int kRows = 128;
constexpr int kShift = 6, kSlots = 1 << kShift;
constexpr int kRowWarps = 8;
constexpr int kThreads = (kRowWarps + 3) * 32;
constexpr int kExtra = 10;  // tiles that a unit's start and end cost (32 trees of 13 tokens: 2 145 us, 6 138, 8 130, 10 128, 14 129)
constexpr int kMaxWorkers = 152;

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

// What a row's maximum may have grown by (log2) before its reference follows, so that weights are up to 2^kGrowth; a factor of
// the weights that go into a product.  Half loses bits below 2^-14 and all of them below 2^-25: as they are, slots that score
// some 17 below the row's reference would be lost, and a long prefix may hold its whole mass there.  So its weights go in as
// large as they may be, which leaves them whole from 2^-27 of the largest on.
template <typename T>
constexpr int kGrowth = std::is_same<T, __half>::value ? 2 : 8;
template <typename T>
constexpr float kWeight = std::is_same<T, __half>::value ? (float)(1 << (15 - kGrowth<T>)) : 1.f;
template <typename T>
__device__ __forceinline__ uint32_t pack_weights(float2 e) {
  if constexpr (kWeight<T> != 1.f) e = __fmul2_rn(e, make_float2(kWeight<T>, kWeight<T>));
  return pack<T>(e.x, e.y);
}

template <int D>
struct Plan {
  static constexpr int kHalves = D / 64;                    // 128-byte column groups of a row
  static constexpr int kKeys = kHalves * kSlots * 128;      // bytes
  static constexpr int kStage = 2 * kKeys;                  // keys, then values
  static constexpr int kStages = 6;
  static constexpr size_t kSmem = (size_t)kStages * kStage + 1024;  // (the base rounded up to 1,024)
  // columns of tensor memory: scores, outputs, weights of the two teams; queries
  static constexpr int kO = 2 * kSlots, kP = kO + 2 * D, kQ = kP + kSlots, kColumns = 512;
  static_assert(kQ + D / 2 <= kColumns, "tensor memory");
};

// A place in the ring of stages, and the parity of its barriers' phase.
template <int kStages>
struct Place {
  int st = 0;
  uint32_t parity = 0;
  __device__ __forceinline__ void on() {
    if (++st == kStages) {
      st = 0;
      parity ^= 1;
    }
  }
};

struct Barriers {
  uint64_t full[8], empty[8], scores[2], taken[2], weights[2], output[2], queries, drained;
};

// What the rows of a unit's block see of its tiles.
struct RowView {
  int lim;        // chain: slots below it
  uint64_t bits;  // tree: new tokens
};

template <typename T, int D>
__global__ void __launch_bounds__(kThreads, 1)
    attention_many_kernel(const __grid_constant__ AttentionParams p, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map,
                          const int box, const int page_shift) {
  using L = Plan<D>;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  extern __shared__ unsigned char dyn[];
  __shared__ Line line;
  __shared__ Barriers bars;
  __shared__ int32_t s_lost[8];  // the tile (1-based, of the share) in a stage that has a slot without a page
  __shared__ int32_t s_abort;
  __shared__ int32_t s_wild;  // the last tile (1-based, of the share) with values that are not finite and some rows may not see
  __shared__ uint32_t s_tmem;
  __shared__ float s_m[2][kRows], s_l[2][kRows];  // the teams' maxima and sums, where they are joined

  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const Grouping g = {p.Hq / p.cache.n_heads, kRows, kShift, p.tree_mask == nullptr};
  const PagedCache& pc = p.cache;
  const uint32_t stages = (smem_u32(dyn) + 1023) & ~1023u;

  if (tid == 0) {
    for (int i = 0; i < L::kStages; ++i) {
      mbar_init(&bars.full[i], 2);
      mbar_init(&bars.empty[i], 1);
      s_lost[i] = 0;
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bars.scores[i], 1);
      mbar_init(&bars.taken[i], 4);
      mbar_init(&bars.weights[i], 4);
      mbar_init(&bars.output[i], 1);
    }
    mbar_init(&bars.queries, kRowWarps);
    mbar_init(&bars.drained, 1);
    s_abort = 0;
    s_wild = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  const Length all = lay_line<kThreads>(p, g, line);
  const Span span = span_of(all, blockIdx.x, gridDim.x, kExtra);
  const Slots slots(p.workspace, gridDim.x, kRows, D);
  if (tid == 0) slots.joined[blockIdx.x] = {0, 0, 0, 0};
  if (span.begin >= span.end) return;  // (all threads alike)
  if (warp == kRowWarps + 2) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"(L::kColumns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    fence_before();
  }
  const Start start = place_in_line(p, g, line, all, span, span.begin);
  const int n = (int)(place_in_line(p, g, line, all, span, span.end).index - start.index);  // tiles of the share
  Cursor at = start.at;
  __syncthreads();
  fence_after();
  constexpr uint32_t tmem = 0;  // (all columns are this CTA's)
  // Waits end: after two seconds, or once another warp's wait has run out.
  const auto wait = [&](uint64_t* bar, uint32_t parity) { return mbar_wait(bar, parity, kWaitTimeoutNs, &s_abort); };
  bool ok = true;

  if (warp == kRowWarps || warp == kRowWarps + 1) {
    // ---- copies ----
    const int boxes = kSlots / box;  // of a tile's slots: at most 8, so that a lane has one copy
    const bool values = warp == kRowWarps + 1;
    const int bx = lane & (boxes - 1);  // (a lane looks up a box; lanes past the last repeat the first ones')
    const uint32_t dst = stages + (values ? L::kKeys : 0);
    const CUtensorMap* map = values ? &v_map : &k_map;
    // The page of this lane's box of a tile, where there is something to read, and its first row there.
    int32_t page = 0;
    int row = 0;
    bool some = false;
    const auto look_up = [&](const Cursor& u) {
      const int slot = u.tile * kSlots + bx * box;
      some = slot < u.end;
      if (some) {
        const int e = page_shift >= 0 ? slot >> page_shift : slot / pc.page_size;
        row = slot - e * pc.page_size;
        page = __ldg(pc.block_table + (int64_t)u.b * pc.table_stride + e);
      }
    };
    Place<L::kStages> at_stage;
    int t = 0;
    look_up(at);
    for (; t < n; ++t) {
      const bool real = some && page >= 0 && page < pc.n_pages, lost = some && !real;
      const int now = page, now_row = row, head = at.head;
      at.next(p, g);
      if (t + 1 < n) look_up(at);  // (the next tile's, on its way while this one waits for its stage)
      if (t >= L::kStages) {
        ok = __all_sync(0xffffffffu, wait(&bars.empty[at_stage.st], at_stage.parity ^ 1));
        if (!ok) break;
      }
      const bool any_lost = __any_sync(0xffffffffu, lost);
      const unsigned who = __ballot_sync(0xffffffffu, real) & ((1u << boxes) - 1);
      int pages[8], rows[8];
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        pages[x] = __shfl_sync(0xffffffffu, now, x);
        rows[x] = __shfl_sync(0xffffffffu, now_row, x);
      }
      if (elect_one()) {
        uint64_t* bar = &bars.full[at_stage.st];
        const uint32_t to = dst + at_stage.st * L::kStage;
        if (any_lost) s_lost[at_stage.st] = t + 1;  // (by the thread whose arrival publishes it)
        mbar_arrive_expect_tx(bar, (uint32_t)(__popc(who) * L::kHalves * box * 128));
#pragma unroll
        for (int x = 0; x < 8; ++x)
          if (who >> x & 1)
#pragma unroll
            for (int half = 0; half < L::kHalves; ++half)
              copy_box(to + half * kSlots * 128 + x * box * 128, map, half * 64, rows[x], head, pages[x], bar);
      }
      __syncwarp();
      at_stage.on();
    }
    if (!ok) {  // (never seen.  No copy may outlive the CTA: those on their way end, or take their time)
      if (lane == 0) s_abort = 1;
      volatile int32_t go_on = 0;
      for (int k = t < L::kStages ? 0 : t - L::kStages; k < t; ++k)
        mbar_wait_warp(&bars.full[k % L::kStages], (k / L::kStages) & 1, kWaitTimeoutNs, &go_on);
    }
  } else if (warp == kRowWarps + 2) {
    // ---- products ----
    if (elect_one()) {
      constexpr uint32_t qk = product<T>(kSlots, false), pv = product<T>(D, true);
      const uint32_t k0 = matrix(stages, 16), v0 = matrix(stages + L::kKeys, kSlots * 128);
      Place<L::kStages> ahead, here;  // of the scores, of the output
      uint32_t team_ahead = 0, team = 0, weights_parity = 0, queries_parity = 0;
      const auto scores = [&] {
        ok = wait(&bars.full[ahead.st], ahead.parity);
        if (!ok) return;
        fence_after();
        const uint32_t k = k0 + ahead.st * (L::kStage >> 4), d = tmem + team_ahead * kSlots;
#pragma unroll
        for (int x = 0; x < D / 16; ++x)
          mma_ts(d, tmem + L::kQ + x * 8, k + (x / 4) * (kSlots * 128 >> 4) + (x % 4) * 2, qk, x > 0);
        commit(&bars.scores[team_ahead]);
        team_ahead ^= 1;
        ahead.on();
      };
      for (int left = n; left > 0 && ok;) {
        const int len = min(left, at.tiles - at.tile);  // of the unit, in this share
        left -= len;
        ok = wait(&bars.queries, queries_parity);
        queries_parity ^= 1;
        if (ok) scores();
        if (ok && len > 1) scores();
        for (int u = 0; u < len && ok; ++u) {
          if (u + 2 < len) {  // the team's next scores, as soon as it has these
            ok = wait(&bars.taken[team], weights_parity);
            if (!ok) break;
            scores();
          }
          ok = ok && wait(&bars.weights[team], weights_parity);
          if (!ok) break;
          fence_after();
          const uint32_t v = v0 + here.st * (L::kStage >> 4), d = tmem + L::kO + team * D, w = tmem + L::kP + team * (kSlots / 2);
#pragma unroll
          for (int x = 0; x < kSlots / 16; ++x) mma_ts(d, w + x * 8, v + x * (16 * 128 >> 4), pv, x > 0 || u >= 2);
          commit(&bars.empty[here.st]);
          commit(&bars.output[team]);
          here.on();
          weights_parity ^= team;
          team ^= 1;
        }
        at.skip(p, g, len);
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
    const int team = warp / 4, row = tid % kRows;
    const uint32_t my = tmem + ((uint32_t)(warp % 4 * 32) << 16);  // this warp's lanes of tensor memory
    const uint32_t my_scores = my + team * kSlots, my_out = my + L::kO + team * D, my_weights = my + L::kP + team * (kSlots / 2);
    const float scale2 = p.scale * kLog2e;
    RowView view = {0, 0};
    float m = -INFINITY, l = 0.f;
    bool nan = false;
    const auto all_rows = [&] { asm volatile("bar.sync 1, %0;" ::"n"(kRowWarps * 32) : "memory"); };
    // Row `row` of a unit's block: token of the sequence, query head.
    const auto token_of = [&](const Cursor& u) { return (int)((uint32_t)(u.block * kRows + row) / (uint32_t)g.group); };
    // This thread's row of a unit's queries into tensor memory (a team takes half of the columns).
    const auto take_queries = [&](const Cursor& u) {
      const int i = token_of(u);
      const bool have = i < u.s.n;
      const T* q = static_cast<const T*>(p.q) + (u.s.off + (have ? i : 0)) * p.q_tok + (u.head * g.group + u.block * kRows + row - i * g.group) * p.q_head;
      uint32_t x[D / 4];
#pragma unroll
      for (int c = 0; c < D / 16; ++c) {
        uint4 v = make_uint4(0, 0, 0, 0);
        const int col = team * (D / 2) + c * 8;
        if (have && col < p.D) v = __ldg(reinterpret_cast<const uint4*>(q + col));
        x[4 * c] = v.x;
        x[4 * c + 1] = v.y;
        x[4 * c + 2] = v.z;
        x[4 * c + 3] = v.w;
      }
      __syncwarp();
      tmem_store(my + L::kQ + team * (D / 4), x);
      tmem_wait_store();
      fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars.queries);
    };
    take_queries(at);
    Place<L::kStages> at_stage;       // of this team's next tile
    if (team == 1) at_stage.on();
    uint32_t parity = 0;              // of this team's scores, weights and output
    bool any_yet = false;             // this team has had a tile
    int64_t unit = start.unit;        // the cost at which the unit starts
    for (int t0 = 0; t0 < n;) {       // a unit, or what of it falls to this share
      const int len = min(n - t0, at.tiles - at.tile), first_tile = at.tile;
      const bool unit_ends = at.tile + len == at.tiles;
      const int first_u = (t0 ^ team) & 1;  // this team's first tile of it
      m = -INFINITY;
      l = 0.f;
      nan = at.s.bad;
      {
        const int i = token_of(at);
        const bool have = i < at.s.n;
        view.lim = at.s.ctx + (have ? i + 1 : 0);
        view.bits = have && !g.chain ? __ldg(p.tree_mask + at.s.off + i) : 0;
      }
      // (a warp whose wait has run out goes on without waiting, to the barriers that the others are at)
      for (int u = first_u; u < len && ok; u += 2) {
        const int st = at_stage.st;
        ok = wait(&bars.full[st], at_stage.parity) && wait(&bars.scores[team], parity);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        fence_after();
        nan |= s_lost[st] == t0 + u + 1;
        float s[kSlots];
        {
          uint32_t r0[32], r1[32];
          tmem_load32(r0, my_scores);
          tmem_load32(r1, my_scores + 32);
          tmem_wait_load();
          fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&bars.taken[team]);
#pragma unroll
          for (int j = 0; j < 32; ++j) {
            s[j] = __uint_as_float(r0[j]);
            s[32 + j] = __uint_as_float(r1[j]);
          }
        }
        const int slot0 = (first_tile + u) * kSlots;
        if (slot0 + kSlots > at.s.ctx) {  // some slots are new tokens', or past the end
#pragma unroll
          for (int j = 0; j < kSlots; ++j) {
            const int back = slot0 + j - at.s.ctx;
            const bool seen = g.chain ? slot0 + j < view.lim : back < 0 || (back < at.s.n && ((view.bits >> (back & 63)) & 1));
            if (!seen) s[j] = -INFINITY;
          }
          // values that no row uses become zeros
          const int slot = slot0 + (row & 63), back = slot - at.s.ctx;
          bool out = slot >= at.end;
          if (!out && !g.chain && back >= 0) {
            uint64_t any = 0;
            const int i0 = at.block * kRows / g.group, i1 = min(at.s.n, ((at.block + 1) * kRows - 1) / g.group + 1);
            for (int i = i0; i < i1; ++i) any |= __ldg(p.tree_mask + at.s.off + i);
            out = !((any >> (back & 63)) & 1);
          }
          const uint32_t v = stages + st * L::kStage + L::kKeys + (row / 64) * kSlots * 128 + (row & 63) * 128;
          if (row / 64 >= L::kHalves) {
          } else if (!out && slot >= first_apart(g, at.s, at.block)) {
            bool was = false;
#pragma unroll
            for (int c = 0; c < 8; ++c) was |= make_finite16<T>(v + c * 16);
            if (was) atomicMax(&s_wild, t0 + u + 1);
          } else if (out) {
#pragma unroll
            for (int c = 0; c < 8; ++c) asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(v + c * 16), "r"(0) : "memory");
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        float mx;
        if (scale2 > 0.f) {
          float x[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
          for (int j = 4; j < kSlots; ++j) x[j & 3] = fmaxf(x[j & 3], s[j]);
          mx = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])) * scale2;
        } else {  // (the largest score is the smallest product)
          mx = -INFINITY;
#pragma unroll
          for (int j = 0; j < kSlots; ++j) mx = fmaxf(mx, s[j] == -INFINITY ? -INFINITY : s[j] * scale2);
        }
        // the row's reference grows at its first tile that sees anything, then by 2^kGrowth at least
        // (a difference: a sum may round to a larger reference, and half has no room for larger weights)
        const bool grows = mx - m > (float)kGrowth<T>;
        float by = 1.f;
        if (grows) {
          by = ex2(m - mx);
          m = mx;
          l *= by;
        }
        const float ref = m == -INFINITY ? 0.f : m;
        uint32_t w[32];
        if (scale2 > 0.f) {
          const float2 sc = make_float2(scale2, scale2), nr = make_float2(-ref, -ref);
          float2 sum[4] = {make_float2(l, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
          for (int j = 0; j < 32; ++j) {
            const float2 x = __ffma2_rn(make_float2(s[2 * j], s[2 * j + 1]), sc, nr);
            const float2 e = make_float2(ex2(x.x), ex2(x.y));
            sum[j & 3] = __fadd2_rn(sum[j & 3], e);
            w[j] = pack_weights<T>(e);
          }
          sum[0] = __fadd2_rn(__fadd2_rn(sum[0], sum[1]), __fadd2_rn(sum[2], sum[3]));
          l = sum[0].x + sum[0].y;
        } else {
#pragma unroll
          for (int j = 0; j < 32; ++j) {  // (a masked score times it is not -inf)
            const float a = s[2 * j] == -INFINITY ? 0.f : ex2(fmaf(s[2 * j], scale2, -ref));
            const float c = s[2 * j + 1] == -INFINITY ? 0.f : ex2(fmaf(s[2 * j + 1], scale2, -ref));
            l += a + c;
            w[j] = pack_weights<T>(make_float2(a, c));
          }
        }
        if (any_yet) {  // the product that read this team's last weights, and added to its output, is done
          ok = __all_sync(0xffffffffu, wait(&bars.output[team], parity ^ 1));
          if (!ok) break;
          fence_after();
        }
        if (u >= 2 && __any_sync(0xffffffffu, grows)) {
#pragma unroll
          for (int c = 0; c < D / 32; ++c) {
            uint32_t r[32];
            tmem_load32(r, my_out + c * 32);
            tmem_wait_load();
#pragma unroll
            for (int j = 0; j < 32; ++j) r[j] = __float_as_uint(__uint_as_float(r[j]) * by);
            tmem_store32(my_out + c * 32, r);
          }
        }
        tmem_store32(my_weights, w);
        tmem_wait_store();
        fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars.weights[team]);
        any_yet = true;
        parity ^= 1;
        at_stage.on();
        at_stage.on();
      }
      if (!ok && lane == 0) s_abort = 1;

      // The teams' parts of the rows become one; out it goes, or into a slot.
      const Cursor was = at;
      at.skip(p, g, len);
      s_m[team][row] = m;
      s_l[team][row] = nan ? NAN : l;
      all_rows();
      if (ok && t0 + len < n) take_queries(at);  // (the scores of the unit's last tile are done with the old ones)
      const int last = t0 + len - 1;
      bool part_of[2];  // whether a team had a tile of it
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int tb = last - ((last ^ b) & 1);  // its last tile
        part_of[b] = tb >= t0;
        if (ok && part_of[b]) ok = wait(&bars.output[b], (tb >> 1) & 1);
      }
      ok = __all_sync(0xffffffffu, ok);
      if (!ok && lane == 0) s_abort = 1;
      if (ok) {
        fence_after();
        const bool starts = first_tile == 0, whole = unit_ends && starts, wild = s_wild > t0;
        const int i = token_of(was);
        const bool have = i < was.s.n;
        const int64_t token = was.s.off + i;
        const int head = was.head * g.group + was.block * kRows + row - i * g.group;
        float* slot = slots.of(blockIdx.x, starts);
        const float m0 = s_m[0][row], m1 = s_m[1][row], M = fmaxf(m0, m1);
        const float f0 = M == -INFINITY ? 1.f : ex2(m0 - M), f1 = M == -INFINITY ? 1.f : ex2(m1 - M);
        const float o0 = f0 * (1.f / kWeight<T>), o1 = f1 * (1.f / kWeight<T>);
        const float sum = s_l[0][row] * f0 + s_l[1][row] * f1, inv = sum == 0.f ? 0.f : 1.f / sum;
        T* out = static_cast<T*>(p.out) + (have ? token * p.out_tok + head * p.out_head : 0);
#pragma unroll
        for (int x = 0; x < D / 64; ++x) {  // (a team writes half of the columns)
          const int c = team * (D / 64) + x;
          uint32_t r0[32], r1[32];
          tmem_load32(r0, my + L::kO + c * 32);
          tmem_load32(r1, my + L::kO + D + c * 32);
          tmem_wait_load();
          float v[32];
#pragma unroll
          for (int j = 0; j < 32; ++j)
            v[j] = (part_of[0] ? __uint_as_float(r0[j]) * o0 : 0.f) + (part_of[1] ? __uint_as_float(r1[j]) * o1 : 0.f);
          if (have && !whole) {
#pragma unroll
            for (int j = 0; j < 32; j += 8) store32(slot + (size_t)row * D + c * 32 + j, v + j);
          } else if (have) {
#pragma unroll
            for (int j = 0; j < 32; j += 8) {
              uint32_t h[4];
#pragma unroll
              for (int y = 0; y < 4; ++y) h[y] = pack<T>(v[j + 2 * y] * inv, v[j + 2 * y + 1] * inv);
              if (c * 32 + j < p.D) *reinterpret_cast<uint4*>(out + c * 32 + j) = make_uint4(h[0], h[1], h[2], h[3]);
            }
          }
          __syncwarp();
        }
        if (wild && have)
          add_wild<T>(p, was.b, was.head, was.s.ctx, max(first_apart(g, was.s, was.block), first_tile * kSlots),
                      min(was.end, (first_tile + len) * kSlots), view.lim, view.bits, whole ? out : nullptr,
                      whole ? nullptr : slot + (size_t)row * D, team * (D / 2), (team + 1) * (D / 2), 2);
        if (team == 0 && have && !whole) {
          slot[(size_t)kRows * D + row] = M;
          slot[(size_t)kRows * D + kRows + row] = sum;
        } else if (team == 0 && have && p.lse) {
          p.lse[token * p.Hq + head] = sum == 0.f ? -INFINITY : (M + log2f(sum)) * kLn2;
        }
        fence_before();
        if (nan && row == 0) set_status(p.dev_status, STRIDE_DEV_BAD_LAYOUT);
        if (tid == 0 && starts && !unit_ends)
          slots.joined[blockIdx.x] = {last_worker(span, blockIdx.x, unit + span.extra + was.tiles), was.b, was.block, was.head};
      }
      all_rows();  // (outputs, maxima and sums make room for the next unit's)
      t0 += len;
      unit += span.extra + was.tiles;
    }
    if (!ok && lane == 0) set_status(p.dev_status, STRIDE_DEV_TIMEOUT);
  }
  fence_before();
  __syncthreads();
  if (warp == kRowWarps + 2) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(L::kColumns) : "memory");
  }
}

// The cache as components x rows of a page x heads x pages, read in boxes of `box` rows.
bool describe_cache(CUtensorMap* map, const void* base, const AttentionParams& p, int dtype, int box) {
  const PagedCache& c = p.cache;
  return describe<4>(map, base, dtype == STRIDE_DTYPE_BF16, {p.D, c.page_size, c.n_heads, c.n_pages}, {c.row_stride, c.head_stride, c.page_stride},
                  {box, 1, 1});
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
  if (!describe_cache(&k_map, p.cache.k, p, dtype, box) || !describe_cache(&v_map, p.cache.v, p, dtype, box)) return cudaErrorInvalidValue;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)L::kSmem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  const int grid = (int)std::min<int64_t>(std::min(sms, kMaxWorkers), most_tiles(p, kRows, kSlots));
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = L::kSmem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  e = cudaLaunchKernelEx(&cfg, kern, p, k_map, v_map, box, page_shift(p.cache.page_size));
  if (e != cudaSuccess) return e;
  if (p.cache.table_stride * p.cache.page_size <= kSlots) return cudaGetLastError();  // (no unit has two tiles)
  return launch_attention_join(p, dtype, grid, kRows, 16, stream);
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
