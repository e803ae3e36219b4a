// attention_line.cuh -- the line of tiles that attention over a paged cache is
// cut into, shared by its kernels (sm_103a).
//
// A unit is a sequence, a block of its rows (new tokens times the query heads of
// one key/value head) and a kv head; its tiles are runs of slots.  The units'
// tiles, one unit after the other, form a line, of which every worker (a warp or
// a CTA) takes an equal share whatever the sequences' lengths: of the line's cost,
// where a unit counts as some tiles more than it has for what it takes to start
// and to end it (`extra`; a share has at least one tile).  Where a unit is
// cut between workers each leaves its part (largest score, sum, unnormalised
// output, in 32 bits) in a slot of the workspace, and the worker where it starts
// leaves a Joined record for the kernel that joins them, in the line's order.
#pragma once

#include <cuda_bf16.h>
#include <math.h>

#include <type_traits>

#include "decode_internal.h"
#include "stride_device.cuh"

namespace stride {

constexpr int kLineSeqs = 1024;  // sequences whose places in the line fit in shared memory

// A sequence of the call.
struct Seq {
  int32_t ctx, n, off;  // committed tokens, new tokens, the first new token's row
  bool bad;             // its rows are NaN
};

__device__ __forceinline__ Seq sequence(const AttentionParams& p, int b) {
  Seq s;
  s.off = __ldg(p.cache.tok_off + b);
  s.n = __ldg(p.cache.tok_off + b + 1) - s.off;
  s.ctx = __ldg(p.cache.ctx_len + b);
  s.bad = false;
  if (s.off < 0 || s.n < 0 || (int64_t)s.off + s.n > p.n_tokens) {
    s.n = 0;  // (no rows of the call: nothing to write)
    s.bad = true;
  }
  if (s.ctx < 0 || (int64_t)s.ctx + s.n > (int64_t)p.cache.table_stride * p.cache.page_size || (int64_t)s.ctx + s.n > INT32_MAX - 256 ||
      (p.tree_mask && s.n > STRIDE_MAX_TREE))
    s.bad = true;
  return s;
}

// How rows and slots are grouped: row = token * group + head within the kv
// head's query heads.
struct Grouping {
  int32_t group, rows, shift;  // query heads per kv head, rows of a block, 2^shift slots of a tile (n * group fits in 31 bits with room)
  bool chain;                 // no tree mask: each token sees the new ones up to itself
  __device__ __forceinline__ int blocks(const Seq& s) const { return (s.n * group + rows - 1) / rows; }
  // One past the last slot that a block's rows may see.
  __device__ __forceinline__ int end(const Seq& s, int block) const {
    if (!chain) return s.ctx + s.n;
    return s.ctx + (min((block + 1) * rows, s.n * group) - 1) / group + 1;
  }
  __device__ __forceinline__ int tiles(const Seq& s, int block) const { return s.bad ? 1 : (end(s, block) + (1 << shift) - 1) >> shift; }
  // The tiles of one head of all blocks.
  __device__ __forceinline__ int64_t all_tiles(const Seq& s) const {
    const int nb = blocks(s);
    if (nb == 0) return 0;
    if (!chain || s.bad || nb == 1) return (int64_t)nb * tiles(s, 0);
    int64_t t = 0;
    for (int k = 0; k < nb; ++k) t += tiles(s, k);
    return t;
  }
};

// A place in the line.
struct Cursor {
  int32_t b, block, head, tile, tiles;
  int32_t end;  // one past the last slot that the block's rows may see; 0 where the sequence is bad
  Seq s;

  __device__ __forceinline__ void enter(const Grouping& g) {
    end = s.bad ? 0 : g.end(s, block);
    tiles = s.bad ? 1 : (end + (1 << g.shift) - 1) >> g.shift;
  }

  __device__ __forceinline__ void next(const AttentionParams& p, const Grouping& g) {
    if (++tile < tiles) return;
    tile = 0;
    if (++head < p.cache.n_heads) return;
    head = 0;
    if (++block >= g.blocks(s)) {
      block = 0;
      do {
        if (++b >= p.cache.n_seqs) return;  // (past the last tile of the line)
        s = sequence(p, b);
      } while (s.n == 0);
    }
    enter(g);
  }
  // The place `n` tiles on, at most one past the last tile of this unit and head.
  __device__ __forceinline__ void skip(const AttentionParams& p, const Grouping& g, int n) {
    tile += n - 1;
    next(p, g);
  }
};

// Sequences' places in the line: the tiles and the units before sequence b + 1,
// for the first kLineSeqs, and the line's length.
struct Line {
  int64_t tiles[kLineSeqs];
  int32_t units[kLineSeqs];
  int64_t part_tiles[32];
  int64_t part_units[32];
};
struct Length {
  int64_t tiles, units;
};

// Called by all of a CTA's threads.
template <int kThreads>
__device__ __forceinline__ Length lay_line(const AttentionParams& p, const Grouping& g, Line& line) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  Length all = {0, 0};
  for (int b0 = 0; b0 < p.cache.n_seqs; b0 += kThreads) {
    const int b = b0 + tid;
    int64_t t = 0, u = 0;
    if (b < p.cache.n_seqs) {
      const Seq s = sequence(p, b);
      if (s.bad && blockIdx.x == 0) set_status(p.dev_status, STRIDE_DEV_BAD_LAYOUT);
      t = g.all_tiles(s) * p.cache.n_heads;
      u = (int64_t)g.blocks(s) * p.cache.n_heads;
    }
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t v = __shfl_up_sync(0xffffffffu, t, o), w = __shfl_up_sync(0xffffffffu, u, o);
      if (lane >= o) {
        t += v;
        u += w;
      }
    }
    __syncthreads();
    if (lane == 31) {
      line.part_tiles[warp] = t;
      line.part_units[warp] = u;
    }
    __syncthreads();
    t += all.tiles;
    u += all.units;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) {
      if (w < warp) {
        t += line.part_tiles[w];
        u += line.part_units[w];
      }
      all.tiles += line.part_tiles[w];
      all.units += line.part_units[w];
    }
    if (b < p.cache.n_seqs && b < kLineSeqs) {
      line.tiles[b] = t;
      line.units[b] = (int32_t)u;
    }
  }
  __syncthreads();
  return all;
}

// A worker's share of the line.
struct Span {
  int64_t begin, end, cost;  // of the worker (begin = end: none), of the line
  int32_t workers, extra;    // that have a share; tiles that a unit counts as beyond its own
};
__device__ __forceinline__ Span span_of(const Length& all, int worker, int workers, int most_extra) {
  Span s;
  s.workers = (int)(all.tiles < workers ? all.tiles : workers);
  const int64_t each = s.workers ? all.tiles / s.workers : 0;
  s.extra = (int)(each <= most_extra ? (each > 0 ? each - 1 : 0) : most_extra);
  s.cost = all.tiles + s.extra * all.units;
  s.begin = worker < s.workers ? s.cost * worker / s.workers : 0;
  s.end = worker < s.workers ? s.cost * (worker + 1) / s.workers : 0;
  return s;
}
// The last worker that has tiles of a unit that ends at unit_end (in cost).
__device__ __forceinline__ int last_worker(const Span& s, int worker, int64_t unit_end) {
  int64_t last = unit_end * s.workers / s.cost;
  if (last >= s.workers) last = s.workers - 1;
  while (last > worker && s.cost * last / s.workers >= unit_end) --last;
  while (s.cost * (last + 1) / s.workers < unit_end) ++last;
  return (int)last;
}

// A place in the line by its cost, for a whole warp alike: the cursor there, the
// cost at which its unit starts, and the tile's index in the line.
struct Start {
  Cursor at;
  int64_t unit, index;
};
__device__ __forceinline__ Start place_in_line(const AttentionParams& p, const Grouping& g, const Line& line, const Length& all,
                                               const Span& span, int64_t x) {
  const int lane = threadIdx.x & 31, n = p.cache.n_seqs, m = min(n, kLineSeqs);
  Start r;
  r.index = all.tiles;
  r.unit = x;
  if (x >= span.cost) return r;  // (the line's end: its index alone)
  const auto cost = [&](int b) { return line.tiles[b] + (int64_t)span.extra * line.units[b]; };
  Cursor& c = r.at;
  int64_t inside = 0, tiles = 0;
  if (x < cost(m - 1)) {
    int lo = 0, hi = m - 1;  // the first sequence whose end lies past x
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (cost(mid) > x)
        hi = mid;
      else
        lo = mid + 1;
    }
    c.b = lo;
    inside = x - (lo ? cost(lo - 1) : 0);
    tiles = lo ? line.tiles[lo - 1] : 0;
  } else {
    int64_t before = cost(m - 1);
    tiles = line.tiles[m - 1];
    c.b = m;
    for (int b0 = m; b0 < n; b0 += 32) {
      const int b = b0 + lane;
      int64_t own = 0, own_tiles = 0;
      if (b < n) {
        const Seq s = sequence(p, b);
        own_tiles = g.all_tiles(s) * p.cache.n_heads;
        own = own_tiles + (int64_t)span.extra * g.blocks(s) * p.cache.n_heads;
      }
      int64_t incl = own, incl_tiles = own_tiles;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int64_t v = __shfl_up_sync(0xffffffffu, incl, o), w = __shfl_up_sync(0xffffffffu, incl_tiles, o);
        if (lane >= o) {
          incl += v;
          incl_tiles += w;
        }
      }
      const unsigned past = __ballot_sync(0xffffffffu, before + incl > x);
      if (past) {
        const int l = __ffs(past) - 1;
        c.b = b0 + l;
        inside = x - before - __shfl_sync(0xffffffffu, incl - own, l);
        tiles += __shfl_sync(0xffffffffu, incl_tiles - own_tiles, l);
        break;
      }
      before += __shfl_sync(0xffffffffu, incl, 31);
      tiles += __shfl_sync(0xffffffffu, incl_tiles, 31);
    }
  }
  c.s = sequence(p, c.b);
  c.block = 0;
  while (true) {
    c.enter(g);
    const int64_t of_block = (int64_t)(c.tiles + span.extra) * p.cache.n_heads;
    if (inside < of_block) break;
    inside -= of_block;
    tiles += (int64_t)c.tiles * p.cache.n_heads;
    ++c.block;
  }
  c.head = (int)(inside / (c.tiles + span.extra));
  const int off = (int)(inside - (int64_t)c.head * (c.tiles + span.extra));
  c.tile = max(off - span.extra, 0);
  r.unit = x - off;
  r.index = tiles + (int64_t)c.head * c.tiles + c.tile;
  return r;
}

// ---- values that are not finite ----
// A weight of 0 times such a value is NaN in a product, so that a new token that
// only some of a block's rows see would reach the others.  Where that can be, the
// components that are not finite are taken out of the values' copy, and added to
// the outputs of the rows that see them, which gives what the sum gives.

// The first slot that some of a block's rows may not see.
__device__ __forceinline__ int first_apart(const Grouping& g, const Seq& s, int block) {
  return s.n <= 1 ? INT32_MAX : s.ctx + (g.chain ? block * g.rows / g.group + 1 : 0);
}
// Two components: those that are not finite become zeros.  True where one was.
template <typename T>
__device__ __forceinline__ bool make_finite(uint32_t& w) {
  constexpr uint32_t kExponent = std::is_same<T, __nv_bfloat16>::value ? 0x7f807f80u : 0x7c007c00u;
  const uint32_t wild = __vcmpeq2(w & kExponent, kExponent);
  w &= ~wild;
  return wild != 0;
}
// 16 bytes in shared memory, likewise.
template <typename T>
__device__ __forceinline__ bool make_finite16(uint32_t addr) {
  uint32_t w[4];
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(addr) : "memory");
  bool any = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) any |= make_finite<T>(w[i]);
  if (any) asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
  return any;
}
// Adds those of slots [j0, j1) of a sequence that a row sees (chain: below lim; tree: new tokens `bits`) to what has been
// stored of the row, an output or a part: to components first, first + 1, then `step` on, below last.
template <typename T>
__device__ __noinline__ void add_wild(const AttentionParams& p, int b, int head, int ctx, int j0, int j1, int lim, uint64_t bits, T* out,
                                      float* part, int first, int last, int step) {
  const PagedCache& pc = p.cache;
  for (int j = j0; j < j1; ++j) {
    if (p.tree_mask ? !((bits >> (j - ctx)) & 1) : j >= lim) continue;
    const int e = j / pc.page_size;
    const int32_t page = __ldg(pc.block_table + (int64_t)b * pc.table_stride + e);
    if (page < 0 || page >= pc.n_pages) continue;
    const T* v = static_cast<const T*>(pc.v) + page * pc.page_stride + (j - e * pc.page_size) * pc.row_stride + head * pc.head_stride;
    for (int c = first; c < last && c < p.D; c += step)
      for (int x = c; x < c + 2; ++x) {
        const float a = (float)v[x];
        if (isfinite(a)) continue;
        if (part)
          part[x] += a;
        else
          out[x] = (T)((float)out[x] + a);
      }
  }
}

// What a worker leaves: the unit that starts in its share and goes on in those
// of the workers after it, up to `last` (none: last 0).
struct Joined {
  int32_t last, seq, block, head;
};

// Workspace: a Joined per worker, then two slots a worker (of the unit that it
// starts with and the one that it ends with, if cut): rows x D outputs, the rows'
// largest scores (in units of ln 2), their sums.
__host__ __device__ inline size_t slot_floats(int rows, int D) { return (size_t)rows * (D + 2); }
__host__ __device__ inline size_t slots_offset(int workers) { return ((size_t)workers * sizeof(Joined) + 255) & ~(size_t)255; }
struct Slots {
  Joined* joined;
  float* base;
  size_t size;
  __device__ __forceinline__ Slots(void* workspace, int workers, int rows, int D)
      : joined(static_cast<Joined*>(workspace)),
        base(reinterpret_cast<float*>(static_cast<char*>(workspace) + slots_offset(workers))),
        size(slot_floats(rows, D)) {}
  // starts: the unit starts in this worker's share
  __device__ __forceinline__ float* of(int worker, bool starts) const { return base + (size_t)(2 * worker + (starts ? 1 : 0)) * size; }
};

constexpr float kLn2 = 0.6931471805599453f;

cudaError_t launch_attention_few(const AttentionParams& p, int dtype, int sms, cudaStream_t stream);
cudaError_t launch_attention_many(const AttentionParams& p, int dtype, int sms, cudaStream_t stream);
// Whether the kernel for many rows takes the cache (its copies are boxes of 8 slots at least).
bool attention_many_takes(const AttentionParams& p);
size_t attention_few_bytes(int D);
size_t attention_many_bytes(int D);
// Joins the cut units of a kernel of `workers` workers and blocks of `rows` rows,
// each with so many CTAs.
cudaError_t launch_attention_join(const AttentionParams& p, int dtype, int workers, int rows, int ctas, cudaStream_t stream);

// No call's line is longer (sequences are as long as the block table holds).
inline int64_t most_tiles(const AttentionParams& p, int rows, int tile) {
  const int64_t group = p.Hq / p.cache.n_heads, blocks = p.cache.n_seqs + p.n_tokens * group / rows;
  const int64_t slots = p.cache.table_stride * (int64_t)p.cache.page_size, most = INT64_MAX / 4;
  const int64_t per = slots > most / p.cache.n_heads ? most : ((slots + tile - 1) / tile) * p.cache.n_heads;
  return per > most / blocks ? most : per * blocks;
}

}  // namespace stride
