// tree_attention.cu -- attention of new tokens (one, a chain, a drafted tree)
// over a paged cache of keys and values (sm_103a): which kernel runs, and the one
// that joins what they cut.
//
//   s_j = scale q.k_j over the slots that a row may see, out = softmax(s) V,
//   lse = ln sum exp s
//
// A sequence's new tokens times the query heads of one key/value head are the
// rows of one product, which reads the keys and values once.  Up to 16 of them:
// tree_attention_few.cu, a stream of keys and values through warps; more:
// tree_attention_many.cu, tcgen05 products of 128 rows.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "attention_line.cuh"

namespace stride {
namespace {

constexpr int kJoinWarps = 8;

// Blocks (c, y): the unit that starts in worker c's share.  Its rows are spread
// over the blocks' warps; where there are fewer rows, a power of two of a block's
// warps shares a row's parts.
template <typename T, int D>
__global__ void __launch_bounds__(kJoinWarps * 32) join_kernel(const AttentionParams p, const int workers, const int rows) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  __shared__ float s_m[kJoinWarps], s_l[kJoinWarps], s_v[kJoinWarps][D];
  const int c = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const Slots slots(p.workspace, workers, rows, D);
  const Joined j = slots.joined[c];
  if (j.last <= c) return;
  const Seq s = sequence(p, j.seq);
  const int group = p.Hq / p.cache.n_heads;
  const int64_t all = (int64_t)s.n * group - (int64_t)j.block * rows;
  const int have = all < rows ? (int)all : rows, parts = j.last - c + 1;
  int team = kJoinWarps;  // warps of a row
  while (team > 1 && (have * team > (int)gridDim.y * kJoinWarps || team > parts)) team /= 2;
  const int r = (blockIdx.y * kJoinWarps + warp) / team, member = warp % team;
  if (blockIdx.y * kJoinWarps / team >= have) return;  // (the block's first row)
  constexpr int kCols = D / 32;
  // a warp's parts: running maximum, sum and output
  float m = -INFINITY, l = 0.f, v[kCols];
#pragma unroll
  for (int x = 0; x < kCols; ++x) v[x] = 0.f;
  for (int k0 = c + member; k0 <= j.last && r < have; k0 += 4 * team) {
    float pm[4], pl[4], pv[4][kCols];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int k = k0 + u * team;
      pm[u] = -INFINITY;
      if (k > j.last) continue;
      const float* slot = slots.of(k, k == c);
      pm[u] = slot[(size_t)rows * D + r];
      pl[u] = slot[(size_t)rows * D + rows + r];
#pragma unroll
      for (int x = 0; x < kCols; ++x) pv[u][x] = slot[(size_t)r * D + x * 32 + lane];
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (k0 + u * team > j.last) continue;
      const float mx = fmaxf(m, pm[u]), ref = mx == -INFINITY ? 0.f : mx, f = ex2(m - ref), g = ex2(pm[u] - ref);
      m = mx;
      l = l * f + pl[u] * g;
#pragma unroll
      for (int x = 0; x < kCols; ++x) v[x] = v[x] * f + pv[u][x] * g;
    }
  }
  if (lane == 0) {
    s_m[warp] = m;
    s_l[warp] = l;
  }
#pragma unroll
  for (int x = 0; x < kCols; ++x) s_v[warp][x * 32 + lane] = v[x];
  __syncthreads();
  if (member != 0 || r >= have) return;
  const int64_t row = (int64_t)j.block * rows + r, token = s.off + row / group;
  const int head = j.head * group + (int)(row % group);
  float M = m, L = 0.f;
  for (int w = 1; w < team; ++w) M = fmaxf(M, s_m[warp + w]);
#pragma unroll
  for (int x = 0; x < kCols; ++x) v[x] = 0.f;
  for (int w = 0; w < team; ++w) {
    const float f = M == -INFINITY ? 1.f : ex2(s_m[warp + w] - M);
    L += s_l[warp + w] * f;
#pragma unroll
    for (int x = 0; x < kCols; ++x) v[x] += s_v[warp + w][x * 32 + lane] * f;
  }
#pragma unroll
  for (int x = 0; x < kCols; ++x)
    if (x * 32 + lane < p.D)
      static_cast<T*>(p.out)[token * p.out_tok + head * p.out_head + x * 32 + lane] = static_cast<T>(L == 0.f ? 0.f : v[x] / L);
  if (p.lse && lane == 0) p.lse[token * p.Hq + head] = L == 0.f ? -INFINITY : (M + log2f(L)) * kLn2;
}

template <typename T, int D>
cudaError_t join(const AttentionParams& p, int workers, int rows, int ctas, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(workers, ctas);
  cfg.blockDim = dim3(kJoinWarps * 32);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, join_kernel<T, D>, p, workers, rows);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

cudaError_t launch_attention_join(const AttentionParams& p, int dtype, int workers, int rows, int ctas, cudaStream_t stream) {
  if (dtype == STRIDE_DTYPE_BF16)
    return p.D <= 64 ? join<__nv_bfloat16, 64>(p, workers, rows, ctas, stream) : join<__nv_bfloat16, 128>(p, workers, rows, ctas, stream);
  return p.D <= 64 ? join<__half, 64>(p, workers, rows, ctas, stream) : join<__half, 128>(p, workers, rows, ctas, stream);
}

size_t attention_workspace_bytes(int64_t, int, int, int D) {
  const size_t few = attention_few_bytes(D), many = attention_many_bytes(D);
  return ((few > many ? few : many) + 255) & ~(size_t)255;
}

cudaError_t launch_tree_attention(const AttentionParams& p, int dtype, int sms, cudaStream_t stream) {
  // By the mean of rows a sequence, as only the device knows how many each has.  Where they are very unequal the kernel for few
  // rows takes long chains, too, and reads their prefixes once for 16 rows: a chain of 511 tokens over 6,000 slots 84 us, 255
  // single tokens over 1,000 217, both in one call 542.
  const int64_t rows = ((p.n_tokens + p.cache.n_seqs - 1) / p.cache.n_seqs) * (p.Hq / p.cache.n_heads);
  if (rows > 16 && attention_many_takes(p)) return launch_attention_many(p, dtype, sms, stream);
  return launch_attention_few(p, dtype, sms, stream);
}

}  // namespace stride
