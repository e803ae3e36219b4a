// attention_mass.cu -- the attention weight that each cached slot gets from a
// call's new tokens, added up over steps (sm_103a).
//
//   w_j = sum over a sequence's rows (new tokens that see slot j, query heads of one
//   kv head) of exp(scale q.k_j - lse),  mass_j = decay mass_j + w_j
//
// With lse known the weights need no maximum and no second pass, and a slot's sum is
// its own: the slots are what is spread over workers, each reads a key once and
// takes all rows past it, so that nothing is joined and no order depends on anything
// but the slot's own sequence.
//
// This kernel takes up to 16 rows at a time, where reading the keys is what counts.
// Every warp has a share of the line of tiles (attention_line.cuh; a unit is a
// sequence and a kv head) and loads a tile of 16 slots, two rows of keys for each
// quad of lanes, straight into the registers of mma.sync's first operand (m16n8k16):
// the order of the summed components is free as long as both operands have the
// same, so a lane takes whole 16-byte vectors and no shuffle or shared memory is
// needed.  The next tile's keys are on their way meanwhile.  The rows are the
// second operand and stay in registers where a unit has no more than the kernel takes
// at once; a result's two columns are added in the lane, the quad's by shuffles.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "attention_line.cuh"

namespace stride {
namespace {

constexpr int kShift = 4, kSlots = 1 << kShift;
constexpr int kWarps = 16;
constexpr int kExtra = 1;  // tiles that a unit's start costs

template <typename T>
__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma<__nv_bfloat16>(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma<__half>(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// What a lane holds of a tile: 16-byte chunks t, t + 4, ... (t its place in the quad) of the keys of slots s and s + 8 of the
// tile, s the quad; their old masses (the quad's first and second lane).
template <int kVec>
struct Tile {
  uint4 k[2][kVec];
  float old;
  bool lost[2];
};

// Eight rows of a unit, likewise, and what the lane's two columns of the result need.
template <int kVec>
struct RowGroup {
  uint4 q[kVec];
  float lse[2];
  int token[2];  // -1: no row, or one that sees nothing
};

// kVec: chunks of a key that a lane has (D up to 32 kVec); kGroups: groups of eight rows taken at once.
template <typename T, int kVec, int kGroups>
__global__ void __launch_bounds__(kWarps * 32, 1) mass_few_kernel(const __grid_constant__ MassParams p, const int page_shift) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  __shared__ Line line;
  const AttentionParams& a = p.a;
  const PagedCache& pc = a.cache;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, quad = lane >> 2, t = lane & 3;
  const Grouping g = {a.Hq / pc.n_heads, 1 << 30, kShift, a.tree_mask == nullptr};
  const Length all = lay_line<kWarps * 32>(a, g, line);
  // (a CTA's warps are workers far apart, so that few tiles are spread over the SMs)
  const Span span = span_of(all, warp * gridDim.x + blockIdx.x, gridDim.x * kWarps, kExtra);
  if (span.begin >= span.end) return;
  const Start start = place_in_line(a, g, line, all, span, span.begin);
  const int n = (int)(place_in_line(a, g, line, all, span, span.end).index - start.index);  // tiles of the share
  const int chunks = a.D / 8;

  // The pages of this lane's two slots of a tile (-1: past the end).
  const auto look_up = [&](const Cursor& u, int32_t (&page)[2]) {
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int slot = u.tile * kSlots + quad + 8 * r;
      page[r] = 0;
      if (slot < u.end) page[r] = __ldg(pc.block_table + (int64_t)u.b * pc.table_stride + (page_shift >= 0 ? slot >> page_shift : slot / pc.page_size));
    }
  };
  const auto load = [&](const Cursor& u, const int32_t (&page)[2], Tile<kVec>& x) {
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int slot = u.tile * kSlots + quad + 8 * r;
      const bool in = slot < u.end, real = in && page[r] >= 0 && page[r] < pc.n_pages;
      x.lost[r] = in && !real;
      const int row = page_shift >= 0 ? slot & ((1 << page_shift) - 1) : slot % pc.page_size;
      const T* k = static_cast<const T*>(pc.k) + page[r] * pc.page_stride + row * pc.row_stride + u.head * pc.head_stride;
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        const int c = t + 4 * i;
        x.k[r][i] = real && c < chunks ? ld_stream(reinterpret_cast<const uint4*>(k) + c) : make_uint4(0, 0, 0, 0);
      }
    }
    x.old = 0.f;
    const int slot = u.tile * kSlots + quad + 8 * t;
    if (t < 2 && p.decay != 0.f && slot < u.s.ctx && slot < u.end && u.end <= p.mass.slots)
      x.old = p.mass.data[u.b * p.mass.seq_stride + u.head * p.mass.head_stride + slot];
  };
  RowGroup<kVec> rows[kGroups];
  const auto load_rows = [&](const Cursor& u, int row0) {
    const int have = u.s.n * g.group;
#pragma unroll
    for (int y = 0; y < kGroups; ++y) {
      const int r = row0 + 8 * y + quad, i = r / g.group;
      const T* q = static_cast<const T*>(a.q) + (u.s.off + i) * a.q_tok + (u.head * g.group + r - i * g.group) * a.q_head;
#pragma unroll
      for (int x = 0; x < kVec; ++x) {
        const int c = t + 4 * x;
        rows[y].q[x] = r < have && c < chunks ? __ldg(reinterpret_cast<const uint4*>(q) + c) : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int col = row0 + 8 * y + 2 * t + x, j = col / g.group;
        rows[y].token[x] = -1;
        rows[y].lse[x] = 0.f;
        if (col < have) {
          rows[y].lse[x] = __ldg(p.lse + (int64_t)(u.s.off + j) * a.Hq + u.head * g.group + col - j * g.group);
          if (rows[y].lse[x] != -INFINITY) rows[y].token[x] = j;
        }
      }
    }
  };

  Cursor at = start.at, ahead = at;  // the tile at hand, the one whose pages are looked up
  int32_t page[2];
  Tile<kVec> now, next;
  bool fresh = true;  // a unit's first tile of the share
  look_up(ahead, page);
  load(ahead, page, now);
  if (n > 1) {
    ahead.next(a, g);
    look_up(ahead, page);
  }
  for (int u = 0; u < n; ++u) {
    if (u + 1 < n) load(ahead, page, next);
    if (u + 2 < n) {
      ahead.next(a, g);
      look_up(ahead, page);
    }
    const int have = at.s.n * g.group, slot0 = at.tile * kSlots + quad;
    const bool whole = slot0 - quad + kSlots <= at.s.ctx;  // all slots committed
    float w[2] = {0.f, 0.f};
    for (int row0 = 0; row0 < have; row0 += 8 * kGroups) {
      if (fresh || have > 8 * kGroups) load_rows(at, row0);
#pragma unroll
      for (int y = 0; y < kGroups; ++y) {
        float c[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int x = 0; x < kVec; ++x) {
          mma<T>(c, now.k[0][x].x, now.k[1][x].x, now.k[0][x].y, now.k[1][x].y, rows[y].q[x].x, rows[y].q[x].y);
          mma<T>(c, now.k[0][x].z, now.k[1][x].z, now.k[0][x].w, now.k[1][x].w, rows[y].q[x].z, rows[y].q[x].w);
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int token = rows[y].token[x];
          bool see[2] = {token >= 0, token >= 0};
          if (!whole && token >= 0) {
            const uint64_t bits = g.chain ? 0 : __ldg(a.tree_mask + at.s.off + token);
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              const int back = slot0 + 8 * r - at.s.ctx;
              see[r] = back < 0 || (g.chain ? back <= token : (bits >> (back & 63)) & 1);
            }
          }
          // (the difference first: its rounding is that of the score)
#pragma unroll
          for (int r = 0; r < 2; ++r)
            w[r] += see[r] ? ex2(fmaf(c[2 * r + x], a.scale, -rows[y].lse[x]) * kLog2e) : 0.f;
        }
      }
    }
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      w[r] += __shfl_xor_sync(0xffffffffu, w[r], 1);
      w[r] += __shfl_xor_sync(0xffffffffu, w[r], 2);
    }
    if (at.end > p.mass.slots) {
      if (lane == 0) set_status(a.dev_status, STRIDE_DEV_BAD_LAYOUT);
    } else if (t < 2) {
      const int slot = slot0 + 8 * t;
      const bool lost = t ? now.lost[1] : now.lost[0];
      float m = t ? w[1] : w[0];
      if (p.decay != 0.f && slot < at.s.ctx) m = fmaf(p.decay, now.old, m);
      if (slot < at.end) p.mass.data[at.b * p.mass.seq_stride + at.head * p.mass.head_stride + slot] = lost ? NAN : m;
      if (lost) set_status(a.dev_status, STRIDE_DEV_BAD_LAYOUT);
    }
    const int b = at.b, head = at.head;
    at.next(a, g);
    fresh = at.b != b || at.head != head;
    now = next;
  }
}

template <typename T, int kVec, int kGroups>
cudaError_t run(const MassParams& p, int sms, cudaStream_t stream) {
  int page_shift = -1;  // not a power of two
  for (int k = 0; k < 31; ++k)
    if (p.a.cache.page_size == 1 << k) page_shift = k;
  const int grid = (int)std::min<int64_t>(sms, most_tiles(p.a, 1 << 30, kSlots));
  return launch_dependent(mass_few_kernel<T, kVec, kGroups>, grid, kWarps * 32, stream, p, page_shift);
}

template <typename T>
cudaError_t run(const MassParams& p, bool few, int sms, cudaStream_t stream) {
  if (p.a.D <= 64) return few ? run<T, 2, 1>(p, sms, stream) : run<T, 2, 2>(p, sms, stream);
  return few ? run<T, 4, 1>(p, sms, stream) : run<T, 4, 2>(p, sms, stream);
}

}  // namespace

cudaError_t launch_attention_mass(const MassParams& p, int dtype, int sms, cudaStream_t stream) {
  // By the mean of rows a sequence, as only the device knows how many each has.
  const int64_t rows = ((p.a.n_tokens + p.a.cache.n_seqs - 1) / p.a.cache.n_seqs) * (p.a.Hq / p.a.cache.n_heads);
  if (rows > 16 && attention_mass_many_takes(p)) return launch_attention_mass_many(p, dtype, sms, stream);
  return dtype == STRIDE_DTYPE_BF16 ? run<__nv_bfloat16>(p, rows <= 8, sms, stream) : run<__half>(p, rows <= 8, sms, stream);
}

}  // namespace stride
