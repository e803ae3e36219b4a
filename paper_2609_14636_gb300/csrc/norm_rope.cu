// norm_rope.cu -- norms of queries and keys for each head with the position
// rotation in the same pass, its backward pass, and the append to a paged
// cache with both on the way (sm_103a).
//
//   r = (mean(x^2) + eps)^(-1/2), n = r x, u = n w, y = R u
//   du = R^T dy, dw = sum du n, g = du w, dx = r (g - n mean(g n))
//
// A head row is a few hundred bytes that is read once and written once, so the
// memory system bounds it.  A row belongs to a group of 1 to 32 lanes; a lane
// holds two chunks of it, A and B, of at most 16 bytes each, chosen so that
// both members of every rotated pair are its own: the rotation needs no
// exchange, the norm one or two shuffle sums.  A warp works on one token, its
// groups on that token's heads, so the angles are loaded once for all of them.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include "decode_internal.h"
#include "stride_device.cuh"

namespace stride {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;

template <typename T>
__device__ __forceinline__ float as_f32(T x);
template <>
__device__ __forceinline__ float as_f32(float x) { return x; }
template <>
__device__ __forceinline__ float as_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
template <>
__device__ __forceinline__ float as_f32(__half x) { return __half2float(x); }

template <typename T>
__device__ __forceinline__ T from_f32(float x);
template <>
__device__ __forceinline__ float from_f32(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32(float x) { return __float2bfloat16_rn(x); }
template <>
__device__ __forceinline__ __half from_f32(float x) { return __float2half_rn(x); }

// CH elements as one load or store.
template <typename T, int CH>
struct alignas(sizeof(T) * CH) Chunk {
  T e[CH];
};

template <typename T, int CH>
__device__ __forceinline__ Chunk<T, CH> load_chunk(const T* p) {
  return *reinterpret_cast<const Chunk<T, CH>*>(p);
}
template <typename T, int CH>
__device__ __forceinline__ void store_chunk(T* p, const float (&f)[CH]) {
  Chunk<T, CH> c;
#pragma unroll
  for (int i = 0; i < CH; ++i) c.e[i] = from_f32<T>(f[i]);
  *reinterpret_cast<Chunk<T, CH>*>(p) = c;
}

// Where a lane's two chunks lie in a row, and the rotation of its pairs
// (cos 1, sin 0 where a component is not rotated).
template <int CH>
struct Lane {
  int a, b;     // first component of each chunk; >= D: the lane has none
  bool across;  // pairs are (A[i], B[i]); else (A[2i], A[2i+1]) and (B[2i], B[2i+1])
  float c[CH], s[CH];
};

// Chunks of item `it` of a row.  Rotary halves: chunk `it` of the first half
// and its partner of the second; the rest of the row, and interleaved rows,
// two neighbours.  One-component chunks put an interleaved pair in A and B.
template <int CH>
__device__ __forceinline__ void place(Lane<CH>& l, int it, int D, int R, bool inter) {
  const int half = R / 2;
  if (!inter && it * CH < half) {
    l.a = it * CH;
    l.b = half + it * CH;
    l.across = true;
  } else {
    const int base = inter ? 0 : R, item = inter ? it : it - half / CH;
    l.a = base + 2 * item * CH;
    l.b = l.a + CH;
    l.across = CH == 1;
  }
  if (l.a >= D) l.a = D;
  if (l.b >= D) l.b = D;
}

template <int CH>
__device__ __forceinline__ void angles(Lane<CH>& l, const NormRopeParams& p, int64_t row, bool good) {
  const int half = p.rot_dim / 2;
  const float* ct = p.cos_table + row * half;
  const float* st = p.sin_table + row * half;
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    int k;  // the angle of pair i of this lane
    if (l.across)
      k = p.interleaved ? l.a / 2 + i : l.a + i;
    else
      k = i < CH / 2 ? l.a / 2 + i : l.b / 2 + (i - CH / 2);
    const bool turned = (l.across && !p.interleaved ? l.b : 2 * k) < p.rot_dim && l.a < p.rot_dim;
    l.c[i] = turned && good ? __ldg(ct + k) : 1.f;
    l.s[i] = turned && good ? __ldg(st + k) : 0.f;
  }
}

// (A, B) rotated by the lane's angles, or by their negatives.
template <int CH>
__device__ __forceinline__ void rotate(const Lane<CH>& l, float (&A)[CH], float (&B)[CH], float sign) {
  if (l.across) {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const float a = A[i], b = B[i], s = sign * l.s[i];
      A[i] = a * l.c[i] - b * s;
      B[i] = a * s + b * l.c[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < CH / 2; ++i) {
      float a = A[2 * i], b = A[2 * i + 1], c = l.c[i], s = sign * l.s[i];
      A[2 * i] = a * c - b * s;
      A[2 * i + 1] = a * s + b * c;
      a = B[2 * i], b = B[2 * i + 1], c = l.c[CH / 2 + i], s = sign * l.s[CH / 2 + i];
      B[2 * i] = a * c - b * s;
      B[2 * i + 1] = a * s + b * c;
    }
  }
}

__device__ __forceinline__ float group_sum(float x, int lanes) {
  for (int o = lanes >> 1; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

// The sequence of token i (the last one whose tok_off is at most i), for a
// whole warp at once: each round narrows the range to a 32nd.
__device__ __forceinline__ int sequence_of(const int32_t* tok_off, int n_seqs, int64_t i, int lane) {
  int lo = 0, n = n_seqs;  // the answer is in [lo, lo + n)
  while (n > 1) {
    const int step = (n + 31) / 32;
    const int at = lo + lane * step;
    const bool le = lane * step < n && __ldg(tok_off + at) <= i;
    const unsigned m = __ballot_sync(0xffffffffu, le);
    const int last = m ? 31 - __clz(m) : 0;
    n = min(step, n - last * step);
    lo += last * step;
  }
  return lo;
}

struct Shape {
  int lanes;           // lanes of a row's group (a power of two)
  int warps_per_token;
};

// One warp per token and share of its heads.
template <typename T, int CH, int IT, bool kAppend>
__global__ void __launch_bounds__(kThreads) norm_rope_kernel(const NormRopeParams p, const Shape sh) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int lane = threadIdx.x & 31;
  const int64_t w = ((int64_t)blockIdx.x * kThreads + threadIdx.x) >> 5;
  const int64_t token = w / sh.warps_per_token;
  const int part = (int)(w % sh.warps_per_token);
  if (token >= p.n_tokens) return;
  const int groups = 32 / sh.lanes, group = lane / sh.lanes, sub = lane % sh.lanes;
  const int step = groups * sh.warps_per_token;

  Lane<CH> l[IT];
#pragma unroll
  for (int it = 0; it < IT; ++it) place(l[it], sub + it * 32, p.D, p.rot_dim, p.interleaved != 0);
  bool good = true;
  int64_t row = 0;
  if (p.rot_dim > 0) {
    row = __ldg(p.pos + token);
    good = row >= 0 && row < p.table_rows;
    if (!good && part == 0 && lane == 0) set_status(p.dev_status, STRIDE_DEV_POSITION);
  }
  int64_t slot_off = 0;
  bool kept = true;
  if constexpr (kAppend) {
    const PagedCache& c = p.cache;
    const int b = sequence_of(c.tok_off, c.n_seqs, token, lane);
    const int64_t slot = (int64_t)__ldg(c.ctx_len + b) + (token - __ldg(c.tok_off + b));
    const int64_t entry = slot / c.page_size;
    int32_t page = -1;
    if (slot >= 0 && entry < c.table_stride) page = __ldg(c.block_table + (int64_t)b * c.table_stride + entry);
    kept = page >= 0 && page < c.n_pages && token < __ldg(c.tok_off + b + 1);
    if (!kept && part == 0 && lane == 0) set_status(p.dev_status, STRIDE_DEV_BAD_LAYOUT);
    slot_off = (int64_t)page * c.page_stride + (slot - entry * c.page_size) * c.row_stride;
  }
#pragma unroll
  for (int it = 0; it < IT; ++it) angles(l[it], p, row, good);

  const int total = p.q.heads + p.k.heads + (kAppend ? p.k.heads : 0);
  for (int h0 = part * groups; h0 < total; h0 += step) {
    const int h = h0 + group;
    const bool is_q = h < p.q.heads, is_v = kAppend && h >= p.q.heads + p.k.heads;
    const bool have = h < total && (is_q || !kAppend || kept);
    const int hh = is_q ? h : is_v ? h - p.q.heads - p.k.heads : h - p.q.heads;
    const T* x;
    T* y;
    const T* wt = nullptr;
    if (is_q) {
      x = static_cast<const T*>(p.q.x) + token * p.q.x_tok + hh * p.q.x_head;
      y = static_cast<T*>(p.q.y) + token * p.q.y_tok + hh * p.q.y_head;
      wt = static_cast<const T*>(p.q.w);
    } else {
      x = is_v ? static_cast<const T*>(p.v) + token * p.v_tok + hh * p.v_head
               : static_cast<const T*>(p.k.x) + token * p.k.x_tok + hh * p.k.x_head;
      if constexpr (kAppend)
        y = static_cast<T*>(is_v ? p.cache.v : p.cache.k) + slot_off + hh * p.cache.head_stride;
      else
        y = static_cast<T*>(p.k.y) + token * p.k.y_tok + hh * p.k.y_head;
      if (!is_v) wt = static_cast<const T*>(p.k.w);
    }
    float A[IT][CH], B[IT][CH];
    float ss = 0.f;
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      Chunk<T, CH> ca = {}, cb = {};
      if (have && l[it].a < p.D) ca = load_chunk<T, CH>(x + l[it].a);
      if (have && l[it].b < p.D) cb = load_chunk<T, CH>(x + l[it].b);
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        A[it][i] = as_f32<T>(ca.e[i]);
        B[it][i] = as_f32<T>(cb.e[i]);
        ss = fmaf(A[it][i], A[it][i], fmaf(B[it][i], B[it][i], ss));
      }
    }
    ss = group_sum(ss, sh.lanes);
    if (!is_v) {
      const float r = good ? (wt ? rsqrtf(ss / (float)p.D + p.eps) : 1.f) : NAN;
#pragma unroll
      for (int it = 0; it < IT; ++it) {
        Chunk<T, CH> wa = {}, wb = {};
        if (wt && l[it].a < p.D) wa = load_chunk<T, CH>(wt + l[it].a);
        if (wt && l[it].b < p.D) wb = load_chunk<T, CH>(wt + l[it].b);
#pragma unroll
        for (int i = 0; i < CH; ++i) {
          A[it][i] *= wt ? r * as_f32<T>(wa.e[i]) : r;
          B[it][i] *= wt ? r * as_f32<T>(wb.e[i]) : r;
        }
        if (p.rot_dim > 0) rotate(l[it], A[it], B[it], 1.f);
      }
    }
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      if (have && l[it].a < p.D) store_chunk<T, CH>(y + l[it].a, A[it]);
      if (have && l[it].b < p.D) store_chunk<T, CH>(y + l[it].b, B[it]);
    }
  }
}

// Blocks [0, q_blocks) take the query rows, the others the key rows; each warp
// walks over tokens and sums its rows' share of the weight gradient in
// registers, the block in a fixed order.
template <typename T, int CH, int IT>
__global__ void __launch_bounds__(kThreads) norm_rope_backward_kernel(const NormRopeParams p, const Shape sh, const int q_blocks) {
  extern __shared__ float s_dw[];  // [kWarps][D]
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const bool is_q = (int)blockIdx.x < q_blocks;
  const RowSet rs = is_q ? p.q : p.k;
  const int block = is_q ? blockIdx.x : blockIdx.x - q_blocks, blocks = is_q ? q_blocks : (int)gridDim.x - q_blocks;
  const int groups = 32 / sh.lanes, group = lane / sh.lanes, sub = lane % sh.lanes;
  const T* wt = static_cast<const T*>(rs.w);
  const bool want = (is_q ? p.dq_weight : p.dk_weight) != nullptr && wt != nullptr;

  Lane<CH> l[IT];
  float wA[IT][CH], wB[IT][CH], dA[IT][CH], dB[IT][CH];
#pragma unroll
  for (int it = 0; it < IT; ++it) {
    place(l[it], sub + it * 32, p.D, p.rot_dim, p.interleaved != 0);
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      wA[it][i] = wt && l[it].a < p.D ? as_f32<T>(wt[l[it].a + i]) : 1.f;
      wB[it][i] = wt && l[it].b < p.D ? as_f32<T>(wt[l[it].b + i]) : 1.f;
      dA[it][i] = dB[it][i] = 0.f;
    }
  }
  const float inv_d = 1.f / (float)p.D;
  for (int64_t token = (int64_t)block * kWarps + warp; token < p.n_tokens; token += (int64_t)blocks * kWarps) {
    int64_t row = 0;
    bool good = true;
    if (p.rot_dim > 0) {
      row = __ldg(p.pos + token);
      good = row >= 0 && row < p.table_rows;
      if (!good && lane == 0) set_status(p.dev_status, STRIDE_DEV_POSITION);
    }
#pragma unroll
    for (int it = 0; it < IT; ++it) angles(l[it], p, row, good);
    for (int h0 = 0; h0 < rs.heads; h0 += groups) {
      const int h = h0 + group;
      const bool have = h < rs.heads;
      const T* x = static_cast<const T*>(rs.x) + token * rs.x_tok + h * rs.x_head;
      const T* dy = static_cast<const T*>(rs.dy) + token * rs.dy_tok + h * rs.dy_head;
      T* dx = static_cast<T*>(rs.y) + token * rs.y_tok + h * rs.y_head;
      float A[IT][CH], B[IT][CH], gA[IT][CH], gB[IT][CH];
      float ss = 0.f, gx = 0.f;
#pragma unroll
      for (int it = 0; it < IT; ++it) {
        Chunk<T, CH> xa = {}, xb = {}, ya = {}, yb = {};
        if (have && l[it].a < p.D) {
          ya = load_chunk<T, CH>(dy + l[it].a);
          if (wt) xa = load_chunk<T, CH>(x + l[it].a);
        }
        if (have && l[it].b < p.D) {
          yb = load_chunk<T, CH>(dy + l[it].b);
          if (wt) xb = load_chunk<T, CH>(x + l[it].b);
        }
#pragma unroll
        for (int i = 0; i < CH; ++i) {
          A[it][i] = as_f32<T>(xa.e[i]);
          B[it][i] = as_f32<T>(xb.e[i]);
          gA[it][i] = as_f32<T>(ya.e[i]);
          gB[it][i] = as_f32<T>(yb.e[i]);
        }
        if (p.rot_dim > 0) rotate(l[it], gA[it], gB[it], -1.f);  // du
      }
      if (wt) {
#pragma unroll
        for (int it = 0; it < IT; ++it)
#pragma unroll
          for (int i = 0; i < CH; ++i) {
            ss = fmaf(A[it][i], A[it][i], fmaf(B[it][i], B[it][i], ss));
            gx = fmaf(gA[it][i] * wA[it][i], A[it][i], fmaf(gB[it][i] * wB[it][i], B[it][i], gx));
          }
        ss = group_sum(ss, sh.lanes);
        gx = group_sum(gx, sh.lanes);
      }
      const float r = !good ? NAN : wt ? rsqrtf(ss * inv_d + p.eps) : 1.f;
      const float m = wt ? gx * r * r * inv_d : 0.f;  // mean(g n) r
#pragma unroll
      for (int it = 0; it < IT; ++it) {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
          if (want && have) {
            dA[it][i] = fmaf(gA[it][i], A[it][i] * r, dA[it][i]);
            dB[it][i] = fmaf(gB[it][i], B[it][i] * r, dB[it][i]);
          }
          gA[it][i] = r * (gA[it][i] * wA[it][i] - A[it][i] * m);
          gB[it][i] = r * (gB[it][i] * wB[it][i] - B[it][i] * m);
        }
        if (have && l[it].a < p.D) store_chunk<T, CH>(dx + l[it].a, gA[it]);
        if (have && l[it].b < p.D) store_chunk<T, CH>(dx + l[it].b, gB[it]);
      }
    }
  }
  if (!want) return;
  // lanes of equal place in the warp's groups, then the block's warps
#pragma unroll
  for (int it = 0; it < IT; ++it)
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      for (int o = sh.lanes; o < 32; o <<= 1) {
        dA[it][i] += __shfl_xor_sync(0xffffffffu, dA[it][i], o);
        dB[it][i] += __shfl_xor_sync(0xffffffffu, dB[it][i], o);
      }
      if (group == 0) {
        if (l[it].a < p.D) s_dw[warp * p.D + l[it].a + i] = dA[it][i];
        if (l[it].b < p.D) s_dw[warp * p.D + l[it].b + i] = dB[it][i];
      }
    }
  __syncthreads();
  for (int d = threadIdx.x; d < p.D; d += kThreads) {
    float t = 0.f;
    for (int k = 0; k < kWarps; ++k) t += s_dw[k * p.D + d];
    p.partials[(int64_t)blockIdx.x * p.D + d] = t;
  }
}

// Sums the blocks' partial weight gradients: blockIdx.y 0 the queries', 1 the
// keys'; 32 columns per block, 32 strided partial sums per column.
__global__ void __launch_bounds__(1024) weight_gradient_kernel(const float* partials, int D, int q_blocks, int blocks, float* dq, float* dk) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  __shared__ float s[32][33];
  const bool is_q = blockIdx.y == 0;
  float* out = is_q ? dq : dk;
  if (!out) return;
  const int d = blockIdx.x * 32 + threadIdx.x, first = is_q ? 0 : q_blocks, end = is_q ? q_blocks : blocks;
  float t = 0.f;
  if (d < D)
    for (int b = first + threadIdx.y; b < end; b += 32) t += partials[(int64_t)b * D + d];
  s[threadIdx.y][threadIdx.x] = t;
  __syncthreads();
  t = s[threadIdx.x][threadIdx.y];  // (transposed: a warp per column)
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
  const int col = blockIdx.x * 32 + threadIdx.y;
  if (threadIdx.x == 0 && col < D) out[col] = t;
}

// A row's items (pairs of chunks) and the lanes that hold them.
int group_lanes(int D, int chunk) {
  const int items = (D + 2 * chunk - 1) / (2 * chunk);
  int lanes = 1;
  while (lanes < items && lanes < 32) lanes *= 2;
  return lanes;
}

template <typename T, int CH, int IT>
cudaError_t run_forward(const NormRopeParams& p, bool append, int sms, cudaStream_t stream) {
  Shape sh;
  sh.lanes = group_lanes(p.D, CH);
  const int rows = p.q.heads + p.k.heads * (append ? 2 : 1), groups = 32 / sh.lanes;
  const int most = (rows + groups - 1) / groups;  // one pass over the heads per warp
  const int64_t warps = (int64_t)sms * 64;
  int64_t share = (warps + p.n_tokens - 1) / p.n_tokens;
  sh.warps_per_token = (int)(share < 1 ? 1 : share > most ? most : share);
  const int64_t blocks = (p.n_tokens * sh.warps_per_token + kWarps - 1) / kWarps;
  if (blocks > INT32_MAX) return cudaErrorInvalidConfiguration;
  if (append) return launch_dependent(norm_rope_kernel<T, CH, IT, true>, (unsigned)blocks, kThreads, stream, p, sh);
  return launch_dependent(norm_rope_kernel<T, CH, IT, false>, (unsigned)blocks, kThreads, stream, p, sh);
}

cudaError_t launch_with(void (*kern)(const NormRopeParams, const Shape, const int), unsigned grid, size_t smem, cudaStream_t stream,
                        const NormRopeParams& p, const Shape& sh, int q_blocks) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kern, p, sh, q_blocks);
  return e != cudaSuccess ? e : cudaGetLastError();
}

template <typename T, int CH, int IT>
cudaError_t run_backward(const NormRopeParams& p, cudaStream_t stream) {
  Shape sh;
  sh.lanes = group_lanes(p.D, CH);
  sh.warps_per_token = 1;
  // blocks in proportion to the rows, at least one for each that has rows
  const int64_t need = (p.n_tokens + kWarps - 1) / kWarps;
  const int64_t heads = p.q.heads + p.k.heads;
  int64_t qb = p.q.heads ? (int64_t)kNormRopeBackwardBlocks * p.q.heads / heads : 0;
  if (p.q.heads && qb < 1) qb = 1;
  if (p.k.heads && qb > kNormRopeBackwardBlocks - 1) qb = kNormRopeBackwardBlocks - 1;
  int64_t kb = p.k.heads ? kNormRopeBackwardBlocks - qb : 0;
  if (qb > need) qb = need;
  if (kb > need) kb = need;
  const bool want = (p.dq_weight && p.q.w) || (p.dk_weight && p.k.w);
  cudaError_t e = cudaSuccess;
  if (qb + kb > 0)
    e = launch_with(norm_rope_backward_kernel<T, CH, IT>, (unsigned)(qb + kb), want ? (size_t)kWarps * p.D * sizeof(float) : 0, stream,
                    p, sh, (int)qb);
  if (e != cudaSuccess || !want) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((p.D + 31) / 32), 2);
  cfg.blockDim = dim3(32, 32);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  e = cudaLaunchKernelEx(&cfg, weight_gradient_kernel, (const float*)p.partials, (int)p.D, (int)qb, (int)(qb + kb),
                         p.dq_weight, p.dk_weight);
  return e != cudaSuccess ? e : cudaGetLastError();
}

// Chunks of 8 elements hold rows of up to 512 components in 32 lanes, of 4 up
// to 256; longer rows, and those that no such chunk divides, go by single
// components, 16 pairs a lane (1,024 components).
template <typename T>
int usable_chunk(int chunk, int D) {
  if (chunk >= 8 && sizeof(T) == 2 && D <= 512) return 8;
  if (chunk >= 4 && D <= 256) return 4;
  return 1;
}

template <typename T>
cudaError_t forward_of(const NormRopeParams& p, int chunk, bool append, int sms, cudaStream_t stream) {
  switch (usable_chunk<T>(chunk, p.D)) {
    case 8:
      if constexpr (sizeof(T) == 2) return run_forward<T, 8, 1>(p, append, sms, stream);
    case 4: return run_forward<T, 4, 1>(p, append, sms, stream);
    default: return run_forward<T, 1, 16>(p, append, sms, stream);
  }
}

template <typename T>
cudaError_t backward_of(const NormRopeParams& p, int chunk, cudaStream_t stream) {
  switch (usable_chunk<T>(chunk, p.D)) {
    case 8:
      if constexpr (sizeof(T) == 2) return run_backward<T, 8, 1>(p, stream);
    case 4: return run_backward<T, 4, 1>(p, stream);
    default: return run_backward<T, 1, 16>(p, stream);
  }
}

}  // namespace

cudaError_t launch_norm_rope(const NormRopeParams& p, int dtype, int chunk, bool append, int sms, cudaStream_t stream) {
  if (dtype == STRIDE_DTYPE_BF16) return forward_of<__nv_bfloat16>(p, chunk, append, sms, stream);
  if (dtype == STRIDE_DTYPE_F16) return forward_of<__half>(p, chunk, append, sms, stream);
  return forward_of<float>(p, chunk, append, sms, stream);
}

cudaError_t launch_norm_rope_backward(const NormRopeParams& p, int dtype, int chunk, cudaStream_t stream) {
  if (dtype == STRIDE_DTYPE_BF16) return backward_of<__nv_bfloat16>(p, chunk, stream);
  if (dtype == STRIDE_DTYPE_F16) return backward_of<__half>(p, chunk, stream);
  return backward_of<float>(p, chunk, stream);
}

}  // namespace stride
