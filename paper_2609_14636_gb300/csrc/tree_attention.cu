// tree_attention.cu -- attention of new tokens (one, a chain, a drafted tree)
// over a paged cache of keys and values (sm_103a).
//
//   s_j = scale q.k_j over the slots that a row may see, out = softmax(s) V,
//   lse = ln sum exp s
//
// A sequence's new tokens times the query heads of one key/value head are the
// rows of one product: they read the same keys and values, once.  The work is
// cut into tiles of 64 slots: units (sequence, block of rows, kv head) one after
// the other, each a run of tiles.  Every CTA takes an equal share of that line
// of tiles, whatever the sequences' lengths, and walks over it with the running
// maximum and sum of a softmax; where a unit is cut between CTAs each writes its
// part (maximum, sum, unnormalised output, in 32 bits) to the workspace and a
// second kernel joins them in the order of the line.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include "decode_internal.h"
#include "mbarrier.cuh"
#include "stride_device.cuh"

namespace stride {
namespace {

constexpr int kTile = 64;          // slots of a tile
constexpr int kStages = 3;         // tiles in shared memory
constexpr int kMaxCtas = 304;      // two for each of 152 SMs
constexpr int kMaxRows = 64;       // rows of a block at most

// What CTA c leaves to the second kernel: the unit that starts in its share and
// goes on in those of CTAs c + 1 .. last.
struct Joined {
  int32_t last;  // 0: none
  int32_t seq, block, head;
};

__host__ __device__ inline size_t slot_floats(int rows, int D) { return (size_t)rows * (D + 2); }

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool real) {
  const int n = real ? 16 : 0;
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a));
}
__device__ __forceinline__ void ldmatrix4t(uint32_t (&r)[4], uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a));
}
template <typename T>
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma<__nv_bfloat16>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma<__half>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
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
  if (s.ctx < 0 || (int64_t)s.ctx + s.n > (int64_t)p.cache.table_stride * p.cache.page_size ||
      (int64_t)s.ctx + s.n > INT32_MAX - kTile || (p.tree_mask && s.n > STRIDE_MAX_TREE))
    s.bad = true;
  return s;
}

// Rows of a unit's block: token * group + head within the kv head's group.
struct Grouping {
  int32_t group, rows;  // query heads per kv head, rows of a block
  __device__ __forceinline__ int blocks(const Seq& s) const { return (s.n * group + rows - 1) / rows; }
  // One past the last slot that a block's rows may see.
  __device__ __forceinline__ int end(const Seq& s, int block, bool chain) const {
    const int last = min((block + 1) * rows, s.n * group) - 1;
    return s.ctx + (chain ? last / group + 1 : s.n);
  }
  __device__ __forceinline__ int tiles(const Seq& s, int block, bool chain) const {
    return s.bad ? 1 : (end(s, block, chain) + kTile - 1) / kTile;
  }
  // The tiles of one head of all blocks.
  __device__ __forceinline__ int64_t all_tiles(const Seq& s, bool chain) const {
    int64_t t = 0;
    const int nb = blocks(s);
    if (!chain || s.bad) return (int64_t)nb * (nb ? tiles(s, 0, false) : 0);
    for (int k = 0; k < nb; ++k) t += tiles(s, k, true);
    return t;
  }
};

// A place in the line of tiles.
struct Cursor {
  int32_t b, block, head, tile, tiles;
  Seq s;

  __device__ __forceinline__ void enter(const AttentionParams& p, const Grouping& g) {
    tiles = g.tiles(s, block, p.tree_mask == nullptr);
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
    enter(p, g);
  }
};

template <typename T, int D, int WM, int WN>
struct Shape {
  static constexpr int kWarps = WM * WN, kThreads = kWarps * 32, kRows = WM * 16;
  static constexpr int kSlots = kTile / WN;  // slots of a tile that one warp takes
  static constexpr int kStageBytes = 2 * kTile * D * 2;
  static constexpr int kMergeFloats = WN * kRows * 33;
  static constexpr size_t smem() { return (size_t)kStages * kStageBytes + kMergeFloats * 4 + 2 * WN * kRows * 4; }
};

template <typename T, int D, int WM, int WN>
__global__ void __launch_bounds__(WM* WN * 32) attention_kernel(const AttentionParams p) {
  using S = Shape<T, D, WM, WN>;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  extern __shared__ __align__(128) unsigned char smem[];
  float* merge = reinterpret_cast<float*>(smem + kStages * S::kStageBytes);
  float* row_m = merge + S::kMergeFloats;  // [WN][rows]
  float* row_l = row_m + WN * S::kRows;
  __shared__ int64_t s_part[S::kWarps];
  __shared__ int32_t s_bad[kStages];  // the tile (1-based, of the share) in a stage that has a slot without a page

  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, wm = warp / WN, wn = warp % WN;
  const bool chain = p.tree_mask == nullptr;
  const Grouping g = {p.Hq / p.cache.n_heads, S::kRows};
  const int Hk = p.cache.n_heads, n_seqs = p.cache.n_seqs;

  // The line's length, and the place where this CTA's share starts.
  int64_t total = 0;
  for (int b0 = 0; b0 < n_seqs; b0 += S::kThreads) {
    const int b = b0 + tid;
    int64_t t = 0;
    if (b < n_seqs) {
      const Seq s = sequence(p, b);
      if (s.bad && blockIdx.x == 0) set_status(p.dev_status, STRIDE_DEV_BAD_LAYOUT);
      t = g.all_tiles(s, chain) * Hk;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
    __syncthreads();
    if (lane == 0) s_part[warp] = t;
    __syncthreads();
    for (int w = 0; w < S::kWarps; ++w) total += s_part[w];
  }
  const int c = blockIdx.x, ctas = (int)(total < gridDim.x ? total : gridDim.x);  // each of them has a tile
  const int64_t t0 = c < ctas ? total * c / ctas : 0, t1 = c < ctas ? total * (c + 1) / ctas : 0;
  Joined* joined = static_cast<Joined*>(p.workspace);
  float* slots = reinterpret_cast<float*>(joined + kMaxCtas);
  const size_t slot_size = slot_floats(S::kRows, D);
  if (t0 >= t1) {
    if (tid == 0) joined[c].last = 0;
    return;
  }
  Cursor at;
  {
    int64_t before = 0;
    int found = -1;
    int64_t inside = 0;
    for (int b0 = 0; b0 < n_seqs && found < 0; b0 += 32) {  // each warp alike
      const int b = b0 + lane;
      const int64_t t = b < n_seqs ? g.all_tiles(sequence(p, b), chain) * Hk : 0;
      int64_t incl = t;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int64_t v = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += v;
      }
      const unsigned m = __ballot_sync(0xffffffffu, before + incl > t0);
      if (m) {
        const int l = __ffs(m) - 1;
        found = b0 + l;
        inside = t0 - before - __shfl_sync(0xffffffffu, incl - t, l);
      } else {
        before += __shfl_sync(0xffffffffu, incl, 31);
      }
    }
    at.b = found;
    at.s = sequence(p, found);
    at.block = 0;
    while (true) {
      const int64_t n = (int64_t)g.tiles(at.s, at.block, chain) * Hk;
      if (inside < n) break;
      inside -= n;
      ++at.block;
    }
    at.enter(p, g);
    at.head = (int)(inside / at.tiles);
    at.tile = (int)(inside % at.tiles);
  }
  if (tid < kStages) s_bad[tid] = 0;
  __syncthreads();

  const PagedCache& pc = p.cache;
  const int chunks = p.D / 8;  // 16-byte chunks of a row that exist
  const uint32_t base = smem_u32(smem);
  // Starts the copy of a tile's keys and values into a stage.
  const auto load = [&](const Cursor& u, int64_t t) {
    const int stage = (int)((t - t0) % kStages);
    const int end = u.s.bad ? 0 : g.end(u.s, u.block, chain);
    constexpr int kChunks = D / 8, kPer = S::kThreads / kChunks;
    const int ch = tid % kChunks;
    const uint32_t kb = base + stage * S::kStageBytes, vb = kb + kTile * D * 2;
    uint64_t seen = ~0ull;  // new tokens that some row of the unit sees
    if (!chain && u.tile * kTile + kTile > u.s.ctx && !u.s.bad) {
      seen = 0;
      const int i0 = u.block * S::kRows / g.group, i1 = min(u.s.n, ((u.block + 1) * S::kRows - 1) / g.group + 1);
      for (int i = i0; i < i1; ++i) seen |= __ldg(p.tree_mask + u.s.off + i);
    }
#pragma unroll 4
    for (int r = tid / kChunks; r < kTile; r += kPer) {
      const int slot = u.tile * kTile + r;
      bool real = slot < end && ch < chunks;
      if (real && slot >= u.s.ctx && !chain) real = (seen >> ((slot - u.s.ctx) & 63)) & 1;
      int64_t off = 0;
      if (real) {
        const int e = slot / pc.page_size;
        const int32_t page = __ldg(pc.block_table + (int64_t)u.b * pc.table_stride + e);
        if (page >= 0 && page < pc.n_pages) {
          off = page * pc.page_stride + (slot - e * pc.page_size) * pc.row_stride + u.head * pc.head_stride + ch * 8;
        } else {
          real = false;
          s_bad[stage] = (int32_t)(t - t0) + 1;
        }
      }
      const uint32_t d = (uint32_t)(r * D * 2 + ((ch ^ (r & 7)) << 4));
      cp_async16(kb + d, static_cast<const T*>(pc.k) + off, real);
      cp_async16(vb + d, static_cast<const T*>(pc.v) + off, real);
    }
  };

  Cursor ahead = at;
  int64_t next = t0;
#pragma unroll
  for (int st = 0; st < kStages - 1; ++st) {
    if (next < t1) {
      load(ahead, next);
      ahead.next(p, g);
      ++next;
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  }

  uint32_t qf[D / 16][4];
  float o[D / 8][4];
  float m[2], l[2];
  int lim[2];         // chain: slots below it are seen
  uint64_t bits[2];   // tree: new tokens seen
  const float scale2 = p.scale * kLog2e;
  bool fresh = true, nan = false;
  int first_tile = 0;

  for (int64_t t = t0; t < t1; ++t) {
    if (fresh) {  // a unit (or what of it falls to this CTA) starts
      fresh = false;
      nan = at.s.bad;
      first_tile = at.tile;
#pragma unroll
      for (int n = 0; n < D / 8; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        m[h] = -INFINITY;
        l[h] = 0.f;
        const int r = at.block * S::kRows + wm * 16 + lane / 4 + h * 8;
        const int i = r / g.group;
        const bool have = i < at.s.n;
        lim[h] = at.s.ctx + (have ? i + 1 : 0);
        bits[h] = have && !chain ? __ldg(p.tree_mask + at.s.off + i) : 0;
        const T* q = static_cast<const T*>(p.q) + (at.s.off + (have ? i : 0)) * p.q_tok + (at.head * g.group + r % g.group) * p.q_head;
#pragma unroll
        for (int k = 0; k < D / 16; ++k)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const int col = k * 16 + x * 8 + (lane % 4) * 2;
            qf[k][h + 2 * x] = have && col < p.D ? *reinterpret_cast<const uint32_t*>(q + col) : 0u;
          }
      }
    }
    asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
    __syncthreads();
    const int stage = (int)((t - t0) % kStages);
    if (next < t1) {
      load(ahead, next);
      ahead.next(p, g);
      ++next;
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    nan |= s_bad[stage] == (int32_t)(t - t0) + 1;

    // scores of this warp's slots
    const uint32_t kb = base + stage * S::kStageBytes, vb = kb + kTile * D * 2;
    constexpr int kN = S::kSlots / 8;
    float s[kN][4];
#pragma unroll
    for (int n = 0; n < kN; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
#pragma unroll
      for (int n = 0; n < kN; n += 2) {
        // two 8-slot groups by 16 components: matrices (slots n, k lo), (n, k hi), (n + 1, lo), (n + 1, hi)
        const int r = wn * S::kSlots + n * 8 + (lane & 7) + ((lane >> 4) << 3), ch = k * 2 + ((lane >> 3) & 1);
        uint32_t f[4];
        ldmatrix4(f, kb + r * D * 2 + ((ch ^ (r & 7)) << 4));
        mma<T>(s[n], qf[k], f[0], f[1]);
        mma<T>(s[n + 1], qf[k], f[2], f[3]);
      }
    }
    const int slot0 = at.tile * kTile + wn * S::kSlots + (lane % 4) * 2;
    const bool edge = at.tile * kTile + kTile > at.s.ctx;
    float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int n = 0; n < kN; ++n)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        float v = s[n][x] * scale2;
        if (edge) {
          const int j = slot0 + n * 8 + (x & 1), h = x >> 1;
          const int back = j - at.s.ctx;
          const bool ok = chain ? j < lim[h] : back < 0 || (back < at.s.n && ((bits[h] >> (back & 63)) & 1));
          v = ok ? v : -INFINITY;
        }
        s[n][x] = v;
        mx[x >> 1] = fmaxf(mx[x >> 1], v);
      }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], 1));
      mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], 2));
      const float was = m[h];
      m[h] = fmaxf(was, mx[h]);
      const float ref = m[h] == -INFINITY ? 0.f : m[h];
      const float f = ex2(was - ref);
      l[h] *= f;
#pragma unroll
      for (int n = 0; n < D / 8; ++n) {
        o[n][2 * h] *= f;
        o[n][2 * h + 1] *= f;
      }
#pragma unroll
      for (int n = 0; n < kN; ++n)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          s[n][2 * h + x] = ex2(s[n][2 * h + x] - ref);
          l[h] += s[n][2 * h + x];
        }
    }
    // output
#pragma unroll
    for (int k = 0; k < kN / 2; ++k) {
      const uint32_t a[4] = {pack<T>(s[2 * k][0], s[2 * k][1]), pack<T>(s[2 * k][2], s[2 * k][3]),
                             pack<T>(s[2 * k + 1][0], s[2 * k + 1][1]), pack<T>(s[2 * k + 1][2], s[2 * k + 1][3])};
#pragma unroll
      for (int n = 0; n < D / 8; n += 2) {
        const int r = wn * S::kSlots + k * 16 + (lane & 15), ch = n + (lane >> 4);
        uint32_t f[4];
        ldmatrix4t(f, vb + r * D * 2 + ((ch ^ (r & 7)) << 4));
        mma<T>(o[n], a, f[0], f[1]);
        mma<T>(o[n + 1], a, f[2], f[3]);
      }
    }

    const bool unit_ends = at.tile + 1 == at.tiles;
    if (unit_ends || t + 1 == t1) {
      // The warps' parts of the rows become one; out it goes, or into a slot.
      const bool whole = unit_ends && first_tile == 0;
      float* slot = slots + (size_t)(2 * c + (first_tile == 0 ? 1 : 0)) * slot_size;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
        l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
        if (lane % 4 == 0) {
          const int r = wm * 16 + lane / 4 + h * 8;
          row_m[wn * S::kRows + r] = m[h];
          row_l[wn * S::kRows + r] = l[h];
        }
      }
      __syncthreads();
      float f[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int r = wm * 16 + lane / 4 + h * 8;
        float M = row_m[r];
        for (int w = 1; w < WN; ++w) M = fmaxf(M, row_m[w * S::kRows + r]);
        f[h] = M == -INFINITY ? 0.f : ex2(m[h] - M);
      }
#pragma unroll
      for (int q = 0; q < D / 32; ++q) {
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const int h = x >> 1, r = wm * 16 + lane / 4 + h * 8;
            merge[(wn * S::kRows + r) * 33 + n * 8 + (lane % 4) * 2 + (x & 1)] = o[q * 4 + n][x] * f[h];
          }
        __syncthreads();
        for (int r = warp; r < S::kRows; r += S::kWarps) {
          float M = row_m[r], L = 0.f, v = 0.f;
          for (int w = 1; w < WN; ++w) M = fmaxf(M, row_m[w * S::kRows + r]);
          for (int w = 0; w < WN; ++w) {
            L += M == -INFINITY ? 0.f : row_l[w * S::kRows + r] * ex2(row_m[w * S::kRows + r] - M);
            v += merge[(w * S::kRows + r) * 33 + lane];
          }
          if (nan) L = NAN;
          const int col = q * 32 + lane;
          if (!whole) {
            slot[(size_t)r * D + col] = v;
            if (q == 0 && lane == 0) {
              slot[(size_t)S::kRows * D + r] = M;
              slot[(size_t)S::kRows * D + S::kRows + r] = L;
            }
          } else {
            const int rr = at.block * S::kRows + r, i = rr / g.group;
            if (i < at.s.n) {
              const int64_t token = at.s.off + i;
              const int head = at.head * g.group + rr % g.group;
              const float y = L == 0.f ? 0.f : v / L;
              if (col < p.D) static_cast<T*>(p.out)[token * p.out_tok + head * p.out_head + col] = static_cast<T>(y);
              if (p.lse && q == 0 && lane == 0)
                p.lse[token * p.Hq + head] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
            }
          }
        }
        __syncthreads();
      }
      if (nan && tid == 0) set_status(p.dev_status, STRIDE_DEV_BAD_LAYOUT);
      if (t + 1 == t1 && tid == 0) {
        Joined j = {0, at.b, at.block, at.head};
        if (!unit_ends && first_tile == 0) {  // the last CTA that has tiles of it
          const int64_t unit_end = t + at.tiles - at.tile;
          int64_t last = unit_end * ctas / total;
          while (last > c && total * last / ctas >= unit_end) --last;
          while (total * (last + 1) / ctas < unit_end) ++last;
          j.last = (int)last;
        }
        joined[c] = j;
      }
      fresh = true;
    }
    at.next(p, g);
  }
}

// Joins the parts of the units that are cut between CTAs: block (c, y) joins
// rows y * 4 .. y * 4 + 3 of the unit that starts in CTA c's share, a warp each.
template <typename T, int D>
__global__ void __launch_bounds__(128) join_kernel(const AttentionParams p, const int rows) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int c = blockIdx.x, lane = threadIdx.x & 31, r = blockIdx.y * 4 + (threadIdx.x >> 5);
  const Joined* joined = static_cast<const Joined*>(p.workspace);
  const Joined j = joined[c];
  if (j.last <= c) return;
  const float* slots = reinterpret_cast<const float*>(joined + kMaxCtas);
  const size_t slot_size = slot_floats(rows, D);
  const Seq s = sequence(p, j.seq);
  const int group = p.Hq / p.cache.n_heads;
  const int rr = j.block * rows + r, i = rr / group;
  if (i >= s.n) return;
  float M = -INFINITY;
  for (int k = c + lane; k <= j.last; k += 32)
    M = fmaxf(M, slots[(size_t)(2 * k + (k == c ? 1 : 0)) * slot_size + (size_t)rows * D + r]);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
  float L = 0.f, v[D / 32];
#pragma unroll
  for (int x = 0; x < D / 32; ++x) v[x] = 0.f;
#pragma unroll 4
  for (int k = c; k <= j.last; ++k) {
    const float* slot = slots + (size_t)(2 * k + (k == c ? 1 : 0)) * slot_size;
    const float m = slot[(size_t)rows * D + r], l = slot[(size_t)rows * D + rows + r];
    const float f = m == -INFINITY ? 0.f : ex2(m - M);
    L += l * f;
#pragma unroll
    for (int x = 0; x < D / 32; ++x) v[x] += slot[(size_t)r * D + x * 32 + lane] * f;
  }
  const int64_t token = s.off + i;
  const int head = j.head * group + rr % group;
#pragma unroll
  for (int x = 0; x < D / 32; ++x)
    if (x * 32 + lane < p.D)
      static_cast<T*>(p.out)[token * p.out_tok + head * p.out_head + x * 32 + lane] = static_cast<T>(L == 0.f ? 0.f : v[x] / L);
  if (p.lse && lane == 0) p.lse[token * p.Hq + head] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
}

template <typename T, int D, int WM, int WN>
cudaError_t run(const AttentionParams& p, int sms, cudaStream_t stream) {
  using S = Shape<T, D, WM, WN>;
  auto kern = attention_kernel<T, D, WM, WN>;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S::smem());
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  const int grid = 2 * sms < kMaxCtas ? 2 * sms : kMaxCtas;
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(S::kThreads);
  cfg.dynamicSmemBytes = S::smem();
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  e = cudaLaunchKernelEx(&cfg, kern, p);
  if (e != cudaSuccess) return e;
  if (p.cache.table_stride * p.cache.page_size > kTile) {  // (else no unit has two tiles)
    cfg.gridDim = dim3(grid, S::kRows / 4);
    cfg.blockDim = dim3(128);
    cfg.dynamicSmemBytes = 0;
    e = cudaLaunchKernelEx(&cfg, join_kernel<T, D>, p, (int)S::kRows);
    if (e != cudaSuccess) return e;
  }
  return cudaGetLastError();
}

template <typename T, int D>
cudaError_t of_rows(const AttentionParams& p, int sms, cudaStream_t stream) {
  const int64_t rows = ((p.n_tokens + p.cache.n_seqs - 1) / p.cache.n_seqs) * (p.Hq / p.cache.n_heads);
  if (rows <= 16) return run<T, D, 1, 4>(p, sms, stream);
  if (rows <= 32) return run<T, D, 2, 2>(p, sms, stream);
  return run<T, D, 4, 1>(p, sms, stream);
}

template <typename T>
cudaError_t of_type(const AttentionParams& p, int sms, cudaStream_t stream) {
  return p.D <= 64 ? of_rows<T, 64>(p, sms, stream) : of_rows<T, 128>(p, sms, stream);
}

}  // namespace

size_t attention_workspace_bytes(int64_t, int, int, int D) {
  const size_t d = D <= 64 ? 64 : 128;
  return (sizeof(Joined) * kMaxCtas + 2 * kMaxCtas * slot_floats(kMaxRows, d) * sizeof(float) + 255) & ~(size_t)255;
}

cudaError_t launch_tree_attention(const AttentionParams& p, int dtype, int sms, cudaStream_t stream) {
  if (dtype == STRIDE_DTYPE_BF16) return of_type<__nv_bfloat16>(p, sms, stream);
  return of_type<__half>(p, sms, stream);
}

}  // namespace stride
