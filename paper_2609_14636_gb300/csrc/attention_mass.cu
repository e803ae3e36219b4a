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
// sequence and a kv head) and takes 16 slots of it at a time through a ring of stages in
// shared memory, filled by asynchronous copies some tiles ahead.  A lane copies what
// it will need itself, whole 16-byte vectors of two keys: mma.sync's first operand
// (m16n8k16), as the order of the summed components is free where both operands have
// the same.  So there is no exchange between lanes and nothing to wait for but the lane's
// own copies.  (Held in registers a tile ahead: 248 us for 256 sequences of up to 4,096
// slots, as registers bound what is on its way.)  The rows are the second operand and stay
// in registers where a unit has no more than the kernel takes at once; a result's two
// columns are added in the lane, the quad's by shuffles.
//
// Measured, us (floor: of bytes at 6,683 GB/s): 256 sequences, a token each over up to 4,096 slots, 32 / 8 heads of 128, 224 (212; 6.3
// TB/s: memory); one token over 131,072 48.8 (41; the ramp and the last tiles of 7 us); over 37 4.9 (a launch and a chain of four
// loads).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "attention_line.cuh"
#include "mbarrier.cuh"

namespace stride {
namespace {

constexpr int kShift = 4, kSlots = 1 << kShift;
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

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool real) {
  const int n = real ? 16 : 0;  // (0: zeros)
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t dst, const void* src, bool real) {
  const int n = real ? 4 : 0;
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}

// Warps of a CTA, of which two share an SM, and their rings.  What is done for a tile takes as many warps as fit (one CTA, us for 256
// sequences of up to 4,096 slots: 16 warps of 3 stages 221, 12 of 4 249, 8 of 6 334; two of 8 of 3 224, and a call of 37 slots 5.0
// instead of 5.5).  A stage: 16-byte chunks t, t + 4, ... (t its place in the quad) of the keys of slots s and s + 8
// of the tile (s the quad) of each lane, side by side for the warp; the old masses of the slots.
template <int kVec>
struct Ring {
  static constexpr int kWarps = 8, kStages = kVec == 4 ? 3 : 5;
  static constexpr int kStage = 2 * kVec * 512 + 64;
  static constexpr size_t kSmem = (size_t)kWarps * kStages * kStage;
};

// Eight rows of a unit, the same chunks of them, and what the lane's two columns of the result need.
template <int kVec>
struct RowGroup {
  uint4 q[kVec];
  float lse[2];
  int token[2];  // -1: no row, or one that sees nothing
};

// kVec: chunks of a key that a lane has (D up to 32 kVec); kGroups: groups of eight rows taken at once.
template <typename T, int kVec, int kGroups>
__global__ void __launch_bounds__(Ring<kVec>::kWarps * 32, 2) mass_few_kernel(const __grid_constant__ MassParams p, const int page_shift) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  using R = Ring<kVec>;
  constexpr int kWarps = R::kWarps, kStages = R::kStages;
  extern __shared__ __align__(128) unsigned char dyn[];
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
  const uint32_t ring = smem_u32(dyn) + warp * kStages * R::kStage;
  // Starts the copies of a tile; its bits: whether the lane's slots have no page.
  const auto load = [&](const Cursor& u, const int32_t (&page)[2], uint32_t stage) {
    uint32_t lost = 0;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int slot = u.tile * kSlots + quad + 8 * r;
      const bool in = slot < u.end, real = in && page[r] >= 0 && page[r] < pc.n_pages;
      lost |= (uint32_t)(in && !real) << r;
      const int row = page_shift >= 0 ? slot & ((1 << page_shift) - 1) : slot % pc.page_size;
      const T* k = static_cast<const T*>(pc.k) + (real ? page[r] * pc.page_stride + row * pc.row_stride + u.head * pc.head_stride : 0);
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        const bool some = real && t + 4 * i < chunks;
        copy16(stage + (r * kVec + i) * 512 + lane * 16, some ? k + (t + 4 * i) * 8 : k, some);
      }
    }
    if (t < 2 && p.decay != 0.f) {
      const int slot = u.tile * kSlots + quad + 8 * t;
      const bool some = slot < u.s.ctx && slot < u.end && u.end <= p.mass.slots;
      copy4(stage + 2 * kVec * 512 + (quad + 8 * t) * 4,
            some ? p.mass.data + u.b * p.mass.seq_stride + u.head * p.mass.head_stride + slot : p.mass.data, some);
    }
    return lost;
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

  // Tiles are started kStages - 1 ahead; each has a group of copies, and so has each turn when none are left.
  Cursor at = start.at, ahead = at;  // the tile at hand, the one whose pages are looked up
  int32_t page[2];
  uint32_t lost = 0;  // two bits a stage
  int started = 0, to = 0, st = 0;
  bool fresh = true;  // a unit's first tile of the share
  look_up(ahead, page);
  const auto start_one = [&] {
    if (started < n) {
      lost = (lost & ~(3u << (2 * to))) | load(ahead, page, ring + to * R::kStage) << (2 * to);
      if (++started < n) {
        ahead.next(a, g);
        look_up(ahead, page);
      }
    }
    to = to + 1 == kStages ? 0 : to + 1;
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int i = 0; i < kStages - 1; ++i) start_one();
  for (int u = 0; u < n; ++u) {
    start_one();
    asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
    const uint32_t stage = ring + st * R::kStage;
    const int have = at.s.n * g.group, slot0 = at.tile * kSlots + quad;
    const bool whole = slot0 - quad + kSlots <= at.s.ctx;  // all slots committed
    float w[2] = {0.f, 0.f};
    for (int row0 = 0; row0 < have; row0 += 8 * kGroups) {
      if (fresh || have > 8 * kGroups) load_rows(at, row0);
      float scores[kGroups][4] = {};
#pragma unroll
      for (int x = 0; x < kVec; ++x) {
        uint32_t k0[4], k1[4];
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(k0[0]), "=r"(k0[1]), "=r"(k0[2]), "=r"(k0[3]) : "r"(stage + x * 512 + lane * 16) : "memory");
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(k1[0]), "=r"(k1[1]), "=r"(k1[2]), "=r"(k1[3]) : "r"(stage + (kVec + x) * 512 + lane * 16) : "memory");
#pragma unroll
        for (int y = 0; y < kGroups; ++y) {
          mma<T>(scores[y], k0[0], k1[0], k0[1], k1[1], rows[y].q[x].x, rows[y].q[x].y);
          mma<T>(scores[y], k0[2], k1[2], k0[3], k1[3], rows[y].q[x].z, rows[y].q[x].w);
        }
      }
#pragma unroll
      for (int y = 0; y < kGroups; ++y) {
        const float (&c)[4] = scores[y];
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
      const bool gone = lost >> (2 * st + t) & 1;
      float m = t ? w[1] : w[0];
      if (p.decay != 0.f && slot < at.s.ctx) {
        float old;
        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(old) : "r"(stage + 2 * kVec * 512 + (quad + 8 * t) * 4) : "memory");
        m = fmaf(p.decay, old, m);
      }
      if (slot < at.end) p.mass.data[at.b * p.mass.seq_stride + at.head * p.mass.head_stride + slot] = gone ? NAN : m;
      if (gone) set_status(a.dev_status, STRIDE_DEV_BAD_LAYOUT);
    }
    const int b = at.b, head = at.head;
    at.next(a, g);
    fresh = at.b != b || at.head != head;
    st = st + 1 == kStages ? 0 : st + 1;
  }
}

template <typename T, int kVec, int kGroups>
cudaError_t run(const MassParams& p, int sms, cudaStream_t stream) {
  int page_shift = -1;  // not a power of two
  for (int k = 0; k < 31; ++k)
    if (p.a.cache.page_size == 1 << k) page_shift = k;
  using R = Ring<kVec>;
  const auto kern = mass_few_kernel<T, kVec, kGroups>;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)R::kSmem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)std::min<int64_t>(2 * sms, most_tiles(p.a, 1 << 30, kSlots)));
  cfg.blockDim = dim3(R::kWarps * 32);
  cfg.dynamicSmemBytes = R::kSmem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  e = cudaLaunchKernelEx(&cfg, kern, p, page_shift);
  return e != cudaSuccess ? e : cudaGetLastError();
}

template <typename T>
cudaError_t run(const MassParams& p, bool few, int sms, cudaStream_t stream) {
  if (p.a.D <= 64) return few ? run<T, 2, 1>(p, sms, stream) : run<T, 2, 2>(p, sms, stream);
  return few ? run<T, 4, 1>(p, sms, stream) : run<T, 4, 2>(p, sms, stream);
}

}  // namespace

cudaError_t launch_attention_mass(const MassParams& p, int dtype, int sms, cudaStream_t stream) {
  // By the mean of rows a sequence, as only the device knows how many each has.  Up to 16 this kernel takes them at once (16 rows,
  // us: over 100,000 slots 23, the other 25; over 37 11 and 13; 256 times 2,000 71 and 66), more a group of 16 after the other (20
  // rows, 16 times 1,000 slots: 29 and 22; 32 times 4,000 130 and 66; 4 times 500 13 and 15).  A share's tiles count alike whatever
  // rows they have: a chain of 511 over 6,000 among 255 single tokens over 1,000 takes 7,940, in two calls 111 and 52.
  const int64_t rows = ((p.a.n_tokens + p.a.cache.n_seqs - 1) / p.a.cache.n_seqs) * (p.a.Hq / p.a.cache.n_heads);
  if (rows > 16 && attention_mass_many_takes(p)) return launch_attention_mass_many(p, dtype, sms, stream);
  return dtype == STRIDE_DTYPE_BF16 ? run<__nv_bfloat16>(p, rows <= 8, sms, stream) : run<__half>(p, rows <= 8, sms, stream);
}

}  // namespace stride
