// tree_attention_few.cu -- attention of up to 16 rows at a time over a paged
// cache: decode steps of one token, small trees (sm_103a).
//
// Each byte of keys and values is used by at most 16 rows, so reading them is
// what counts.  Every warp works alone: it has a share of the line of tiles
// (attention_line.cuh) and a ring of stages in shared memory, which it fills with
// 16-byte asynchronous copies a tile ahead; a lane looks up one slot's page for
// all.  (Bulk copies of a key or a value each, 256 bytes, took some 22 clocks
// apiece however many were in flight: 3.3 TB/s.)  Rows are padded by 16 bytes,
// which keeps ldmatrix free of bank conflicts.  16 rows by 32 slots go through
// mma.sync (m16n8k16: a tcgen05 product would have 128 rows, most of them empty,
// and an accumulator to fetch); maximum, sum and output stay in registers until the
// unit or the share ends.  GB300, 32 / 8 heads of 128, bf16: 256 sequences of up to
// 4,096 slots 467 us (5.9 TB/s), one of 131,072 102 us (5.2 TB/s), with 16 / 2
// heads one of 37 7.8 us.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "attention_line.cuh"
#include "mbarrier.cuh"

namespace stride {
namespace {

constexpr int kRows = 16;
constexpr int kShift = 5, kSlots = 1 << kShift;  // of a tile: one for each lane
constexpr int kExtra = 1;   // tiles that a unit's start and end cost
constexpr int kSms = 152;

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

// A factor of the weights (at most 1) that go into a product.  Half loses bits below 2^-14 and all of them below 2^-25: as they
// are, slots that score some 17 below the largest would be lost, and a long prefix may hold its whole mass there.  Times 2^15
// they are whole from 2^-29 on.
template <typename T>
constexpr float kWeight = std::is_same<T, __half>::value ? 32768.f : 1.f;
template <typename T>
__device__ __forceinline__ uint32_t pack_weights(float lo, float hi) {
  return pack<T>(lo * kWeight<T>, hi * kWeight<T>);
}

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool real) {
  const int n = real ? 16 : 0;  // (0: zeros)
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}

template <int D>
struct Ring {
  static constexpr int kPitch = D * 2 + 16;             // bytes of a slot's key or value
  static constexpr int kStage = 2 * kSlots * kPitch;    // keys, then values
  // what shared memory holds: the more warps the better, at two stages each (D = 128, us for 256 sequences of up to 4,096
  // slots: 4 warps of 3 stages 481, 6 of 2 463)
  static constexpr int kWarps = D == 128 ? 6 : 10, kStages = 2;
  static constexpr int kMaxWorkers = kSms * kWarps;
  static constexpr size_t kSmem = (size_t)kWarps * kStages * kStage;
};

template <typename T, int D>
__global__ void __launch_bounds__(Ring<D>::kWarps * 32, 1) attention_few_kernel(const __grid_constant__ AttentionParams p, const int page_shift,
                                                                              const int line_shift) {
  using R = Ring<D>;
  constexpr int kWarps = R::kWarps;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ Line line;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const Grouping g = {p.Hq / p.cache.n_heads, kRows, kShift, p.tree_mask == nullptr};
  const PagedCache& pc = p.cache;
  if (p.D < D)  // (columns past p.D are read as zeros: nothing writes them)
    for (uint32_t i = tid * 16; i < R::kSmem; i += kWarps * 32 * 16)
      *reinterpret_cast<uint4*>(smem + i) = make_uint4(0, 0, 0, 0);
  // (line_shift: of the slots that the line counts as a tile, kSlots or more than any unit has)
  const bool whole_units = line_shift > kShift;
  const Grouping lg = {g.group, kRows, line_shift, g.chain};
  const Length all = lay_line<kWarps * 32>(p, lg, line);

  const int workers = gridDim.x * kWarps, worker = blockIdx.x * kWarps + warp;
  const Span span = span_of(all, worker, workers, whole_units ? 0 : kExtra);
  const Slots slots(p.workspace, workers, kRows, D);
  if (lane == 0) slots.joined[worker] = {0, 0, 0, 0};
  if (span.begin >= span.end) return;
  const Start start = place_in_line(p, lg, line, all, span, span.begin);
  int count = (int)(place_in_line(p, lg, line, all, span, span.end).index - start.index);  // tiles of the share
  Cursor at = start.at;
  if (whole_units) {
    at.enter(g);
    Cursor c = at;
    for (int units = count, u = count = 0; u < units; ++u) {
      count += c.tiles;
      c.skip(p, g, c.tiles);
    }
  }
  int64_t unit = start.unit;  // the cost at which the unit starts

  const uint32_t base = smem_u32(smem) + warp * R::kStages * R::kStage;
  const int row_chunks = p.D / 8;  // 16-byte chunks of a key or a value
  // Starts the copies of a tile; true where a slot has no page.
  const auto load = [&](const Cursor& u, int stage) {
    const int slot = u.tile * kSlots + lane;
    bool real = slot < u.end;
    if (!g.chain && slot >= u.s.ctx && real) {  // a new token that no row of the unit sees is left out
      uint64_t seen = 0;
      const int i0 = u.block * kRows / g.group, i1 = min(u.s.n, ((u.block + 1) * kRows - 1) / g.group + 1);
      for (int i = i0; i < i1; ++i) seen |= __ldg(p.tree_mask + u.s.off + i);
      real = (seen >> ((slot - u.s.ctx) & 63)) & 1;
    }
    int64_t off = 0;
    bool lost = false;
    if (real) {
      const int e = page_shift >= 0 ? slot >> page_shift : slot / pc.page_size;
      const int32_t page = __ldg(pc.block_table + (int64_t)u.b * pc.table_stride + e);
      lost = page < 0 || page >= pc.n_pages;
      off = page * pc.page_stride + (slot - e * pc.page_size) * pc.row_stride + u.head * pc.head_stride;
      real = !lost;
    }
    // (a lane's chunk of two slots at a time; row_chunks are powers of two or leave lanes idle)
    const uint32_t k = base + stage * R::kStage;
    constexpr int kChunks = D / 8, kAtOnce = 32 / kChunks;
    const int ch = lane % kChunks, sub = lane / kChunks;
    const unsigned who = __ballot_sync(0xffffffffu, real);
#pragma unroll
    for (int r0 = 0; r0 < kSlots; r0 += kAtOnce) {
      const int r = r0 + sub;
      const int64_t o = __shfl_sync(0xffffffffu, off, r) + ch * 8;
      const bool have = (who >> r) & 1;
      if (ch < row_chunks) {
        copy16(k + r * R::kPitch + ch * 16, static_cast<const T*>(pc.k) + o, have);
        copy16(k + (kSlots + r) * R::kPitch + ch * 16, static_cast<const T*>(pc.v) + o, have);
      }
    }
    return lost;
  };

  Cursor ahead = at;
  int next = 0;
  int into = 0, from = 0;        // stages: the next to load, the next to use
  unsigned lost_in = 0;          // stages (bits) that miss a page
  const auto load_next = [&] {
    if (next < count) {
      const bool lost = __any_sync(0xffffffffu, load(ahead, into));
      lost_in = (lost_in & ~(1u << into)) | (lost ? 1u << into : 0u);
      ahead.next(p, g);
      ++next;
      into = into + 1 == R::kStages ? 0 : into + 1;
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  for (int st = 0; st < R::kStages - 1; ++st) load_next();

  uint32_t qf[D / 16][4];
  float o[D / 8][4], m[2], l[2];
  int lim[2];        // chain: slots below it are seen
  uint64_t bits[2];  // tree: new tokens seen
  const float scale2 = p.scale * kLog2e;
  bool fresh = true, nan = false, wild = false;  // wild: the unit has had values that are not finite and some rows may not see
  int first_tile = 0;

  for (int t = 0; t < count; ++t) {
    if (fresh) {  // a unit (or what of it falls to this warp) starts
      fresh = false;
      nan = at.s.bad;
      wild = false;
      first_tile = at.tile;
#pragma unroll
      for (int n = 0; n < D / 8; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        m[h] = -INFINITY;
        l[h] = 0.f;
        const int r = at.block * kRows + lane / 4 + h * 8, i = r / g.group;
        const bool have = i < at.s.n;
        lim[h] = at.s.ctx + (have ? i + 1 : 0);
        bits[h] = have && !g.chain ? __ldg(p.tree_mask + at.s.off + i) : 0;
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
    load_next();
    asm volatile("cp.async.wait_group %0;" ::"n"(R::kStages - 1) : "memory");
    __syncwarp();
    nan |= (lost_in >> from) & 1;

    const uint32_t kb = base + from * R::kStage, vb = kb + kSlots * R::kPitch;
    if (const int apart = first_apart(g, at.s, at.block); at.tile * kSlots + kSlots > apart) {
      bool was = false;
      if (at.tile * kSlots + lane >= apart)
        for (int c = 0; c < row_chunks; ++c) was |= make_finite16<T>(vb + lane * R::kPitch + c * 16);
      wild |= __any_sync(0xffffffffu, was);
      __syncwarp();  // (other lanes read the values: a vote alone orders no memory)
    }
    constexpr int kN = kSlots / 8;
    float s[kN][4];
#pragma unroll
    for (int n = 0; n < kN; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
#pragma unroll
    for (int k = 0; k < D / 16; ++k)
#pragma unroll
      for (int n = 0; n < kN; n += 2) {
        // matrices: (slots n, components lo), (n, hi), (n + 1, lo), (n + 1, hi)
        uint32_t f[4];
        ldmatrix4(f, kb + (n * 8 + (lane & 7) + ((lane >> 4) << 3)) * R::kPitch + k * 32 + ((lane >> 3) & 1) * 16);
        mma<T>(s[n], qf[k], f[0], f[1]);
        mma<T>(s[n + 1], qf[k], f[2], f[3]);
      }
    const int slot0 = at.tile * kSlots + (lane % 4) * 2;
    float mx[2] = {-INFINITY, -INFINITY};
    if (at.tile * kSlots + kSlots > at.s.ctx) {
#pragma unroll
      for (int n = 0; n < kN; ++n)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int j = slot0 + n * 8 + (x & 1), h = x >> 1, back = j - at.s.ctx;
          const bool seen = g.chain ? j < lim[h] : back < 0 || (back < at.s.n && ((bits[h] >> (back & 63)) & 1));
          if (!seen) s[n][x] = -INFINITY;
          else s[n][x] *= scale2;
          mx[h] = fmaxf(mx[h], s[n][x]);
        }
    } else {
#pragma unroll
      for (int n = 0; n < kN; ++n)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          s[n][x] *= scale2;
          mx[x >> 1] = fmaxf(mx[x >> 1], s[n][x]);
        }
    }
    float ref[2], f[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], 1));
      mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], 2));
      mx[h] = fmaxf(mx[h], m[h]);
      ref[h] = mx[h] == -INFINITY ? 0.f : mx[h];
      f[h] = ex2(m[h] - ref[h]);
    }
    if (__any_sync(0xffffffffu, mx[0] > m[0] || mx[1] > m[1])) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        l[h] *= f[h];
        m[h] = mx[h];
#pragma unroll
        for (int n = 0; n < D / 8; ++n) {
          o[n][2 * h] *= f[h];
          o[n][2 * h + 1] *= f[h];
        }
      }
    }
#pragma unroll
    for (int n = 0; n < kN; ++n)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        s[n][x] = ex2(s[n][x] - ref[x >> 1]);
        l[x >> 1] += s[n][x];
      }
    // The weights are rounded to the values' type, as mma.sync wants both operands of one type (a product of what the rounding
    // leaves would be half as many instructions again).  Their sum is of the unrounded ones.
#pragma unroll
    for (int k = 0; k < kN / 2; ++k) {
      const uint32_t a[4] = {pack_weights<T>(s[2 * k][0], s[2 * k][1]), pack_weights<T>(s[2 * k][2], s[2 * k][3]),
                             pack_weights<T>(s[2 * k + 1][0], s[2 * k + 1][1]), pack_weights<T>(s[2 * k + 1][2], s[2 * k + 1][3])};
#pragma unroll
      for (int n = 0; n < D / 8; n += 2) {
        uint32_t b[4];
        ldmatrix4t(b, vb + (k * 16 + (lane & 15)) * R::kPitch + (n + (lane >> 4)) * 16);
        mma<T>(o[n], a, b[0], b[1]);
        mma<T>(o[n + 1], a, b[2], b[3]);
      }
    }
    __syncwarp();  // (the stage is read: it may be loaded again)
    from = from + 1 == R::kStages ? 0 : from + 1;

    const bool unit_ends = at.tile + 1 == at.tiles;
    if (unit_ends || t + 1 == count) {
      const bool starts = first_tile == 0, whole = unit_ends && starts;
      float* slot = slots.of(worker, starts);
      const int apart = max(first_apart(g, at.s, at.block), first_tile * kSlots), wild_end = min(at.end, (at.tile + 1) * kSlots);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
        l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
        if (nan) l[h] = NAN;
        const int r = lane / 4 + h * 8, rr = at.block * kRows + r, i = rr / g.group;
        if (!whole) {
#pragma unroll
          for (int n = 0; n < D / 8; ++n)
            *reinterpret_cast<float2*>(slot + (size_t)r * D + n * 8 + (lane % 4) * 2) =
                make_float2(o[n][2 * h] * (1.f / kWeight<T>), o[n][2 * h + 1] * (1.f / kWeight<T>));
          if (wild) add_wild<T>(p, at.b, at.head, at.s.ctx, apart, wild_end, lim[h], bits[h], nullptr, slot + (size_t)r * D, (lane % 4) * 2, D, 8);
          if (lane % 4 == 0) {
            slot[(size_t)kRows * D + r] = m[h];
            slot[(size_t)kRows * D + kRows + r] = l[h];
          }
        } else if (i < at.s.n) {
          const int64_t token = at.s.off + i;
          const int head = at.head * g.group + rr % g.group;
          const float by = l[h] == 0.f ? 0.f : (1.f / kWeight<T>) / l[h];
          T* out = static_cast<T*>(p.out) + token * p.out_tok + head * p.out_head;
#pragma unroll
          for (int n = 0; n < D / 8; ++n) {
            const int col = n * 8 + (lane % 4) * 2;
            if (col < p.D) *reinterpret_cast<uint32_t*>(out + col) = pack<T>(o[n][2 * h] * by, o[n][2 * h + 1] * by);
          }
          if (wild) add_wild<T>(p, at.b, at.head, at.s.ctx, apart, wild_end, lim[h], bits[h], out, nullptr, (lane % 4) * 2, D, 8);
          if (p.lse && lane % 4 == 0) p.lse[token * p.Hq + head] = l[h] == 0.f ? -INFINITY : (m[h] + log2f(l[h])) * kLn2;
        }
      }
      if (lane == 0) {
        if (nan) set_status(p.dev_status, STRIDE_DEV_BAD_LAYOUT);
        if (starts && !unit_ends) slots.joined[worker] = {last_worker(span, worker, unit + span.extra + at.tiles), at.b, at.block, at.head};
      }
      fresh = true;
      unit += span.extra + at.tiles;
    }
    at.next(p, g);
  }
}

template <typename T, int D>
cudaError_t run(const AttentionParams& p, int dtype, int sms, cudaStream_t stream) {
  using R = Ring<D>;
  auto kern = attention_few_kernel<T, D>;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)R::kSmem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  constexpr int kWarps = R::kWarps;
  // Where no unit has more than two tiles, and each can have a warp of its own, none is cut: there is nothing to join, a launch
  // less.  (One token over up to 38 slots, 4 kv heads, us cut / whole: 1 sequence 9.8 / 8.0, 64 11.4 / 10.8, 228, a unit for
  // each warp, 16.5 / 17.0; 1 sequence of 100 slots, four tiles: 10.1 / 10.8.)
  constexpr int kUncut = 30;
  const bool whole = p.cache.table_stride * p.cache.page_size <= 2 * kSlots && 2 * most_tiles(p, kRows, 1 << kUncut) <= R::kMaxWorkers;
  const int line_shift = whole ? kUncut : kShift;
  const int64_t need = (most_tiles(p, kRows, 1 << line_shift) + kWarps - 1) / kWarps;
  const int grid = (int)std::min<int64_t>(std::min(sms, kSms), need);
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(kWarps * 32);
  cfg.dynamicSmemBytes = R::kSmem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  int shift = -1;
  for (int k = 0; k < 31; ++k)
    if (p.cache.page_size == 1 << k) shift = k;
  e = cudaLaunchKernelEx(&cfg, kern, p, shift, line_shift);
  if (e != cudaSuccess) return e;
  if (whole) return cudaGetLastError();
  return launch_attention_join(p, dtype, grid * kWarps, kRows, 4, stream);
}

}  // namespace

size_t attention_few_bytes(int D) {
  const int workers = D <= 64 ? Ring<64>::kMaxWorkers : Ring<128>::kMaxWorkers;
  return slots_offset(workers) + 2 * (size_t)workers * slot_floats(kRows, D <= 64 ? 64 : 128) * sizeof(float);
}

cudaError_t launch_attention_few(const AttentionParams& p, int dtype, int sms, cudaStream_t stream) {
  if (dtype == STRIDE_DTYPE_BF16)
    return p.D <= 64 ? run<__nv_bfloat16, 64>(p, dtype, sms, stream) : run<__nv_bfloat16, 128>(p, dtype, sms, stream);
  return p.D <= 64 ? run<__half, 64>(p, dtype, sms, stream) : run<__half, 128>(p, dtype, sms, stream);
}

}  // namespace stride
