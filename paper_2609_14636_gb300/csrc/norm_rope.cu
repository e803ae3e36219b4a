// norm_rope.cu -- norms of queries and keys for each head with the position
// rotation in the same pass, its backward pass, and the append to a paged
// cache with both on the way (sm_103a).
//
//   r = (mean(x^2) + eps)^(-1/2), n = r x, u = n w, y = R u
//   du = R^T dy, dw = sum du n, g = du w, dx = r (g - n mean(g n))
//
// A head row is a few hundred bytes that is read once and written once, so the
// memory system bounds it.  A row belongs to a group of 1 to 32 lanes; a lane
// holds two chunks of it, A and B, of at most 16 bytes each, chosen so that both
// members of every rotated pair are its own: the rotation needs no exchange, the
// norm one or two shuffle sums.  A warp works on one token, its groups on that
// token's heads, so the angles are loaded once for all of them; the next rows are
// on their way while these are worked on, and two components at a time go through
// packed fp32 operations (component by component, the rows' arithmetic took 426
// instructions an iteration of a warp, and twice the time).  Rows that no chunk of
// four components divides, or of more than 512 (fp32: 256), go by single
// components, a warp each.  GB300, 16,384 tokens, 32 + 8 heads of 128, bf16:
// forward 65 us (5.2 TB/s), backward 108 (4.7 TB/s); 13 sequences of 640 tokens
// into pages 30.5 us (4.4 TB/s); 256 tokens 4.4 us.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include <type_traits>

#include "decode_internal.h"
#include "stride_device.cuh"

namespace stride {
namespace {

constexpr int kThreads = 128;
constexpr int kWarps = kThreads / 32;
constexpr int kAhead = 1;  // rows of a group on their way (backward of 16,384 tokens: one 108 us, two 143)

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

// CH elements as one load or store: whole words, so that none is taken apart by
// halves.
template <typename T, int CH>
struct Chunk {
  static constexpr int kWords = CH * sizeof(T) / 4;
  uint32_t w[kWords];
};

template <typename T, int CH>
__device__ __forceinline__ Chunk<T, CH> load_chunk(const T* p) {
  Chunk<T, CH> c;
  if constexpr (Chunk<T, CH>::kWords == 4) {
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    c.w[0] = v.x, c.w[1] = v.y, c.w[2] = v.z, c.w[3] = v.w;
  } else {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    c.w[0] = v.x, c.w[1] = v.y;
  }
  return c;
}
template <typename T, int CH>
__device__ __forceinline__ void save_chunk(T* p, const Chunk<T, CH>& c) {
  if constexpr (Chunk<T, CH>::kWords == 4)
    *reinterpret_cast<uint4*>(p) = make_uint4(c.w[0], c.w[1], c.w[2], c.w[3]);
  else
    *reinterpret_cast<uint2*>(p) = make_uint2(c.w[0], c.w[1]);
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

// Chunks of CH components as pairs.
template <int CH>
struct Pairs {
  float2 v[CH / 2];
};
template <typename T, int CH>
__device__ __forceinline__ Pairs<CH> widen(const Chunk<T, CH>& c) {
  Pairs<CH> p;
#pragma unroll
  for (int i = 0; i < CH / 2; ++i) {
    if constexpr (std::is_same<T, __nv_bfloat16>::value) {
      p.v[i] = make_float2(bf16_lo(c.w[i]), bf16_hi(c.w[i]));
    } else if constexpr (std::is_same<T, __half>::value) {
      __half2 h;
      *reinterpret_cast<uint32_t*>(&h) = c.w[i];
      p.v[i] = __half22float2(h);
    } else {
      p.v[i] = make_float2(__uint_as_float(c.w[2 * i]), __uint_as_float(c.w[2 * i + 1]));
    }
  }
  return p;
}
template <typename T, int CH>
__device__ __forceinline__ void store_pairs(T* out, const Pairs<CH>& p) {
  Chunk<T, CH> c;
#pragma unroll
  for (int i = 0; i < CH / 2; ++i) {
    if constexpr (std::is_same<T, __nv_bfloat16>::value) {
      const __nv_bfloat162 h = __float22bfloat162_rn(p.v[i]);
      c.w[i] = *reinterpret_cast<const uint32_t*>(&h);
    } else if constexpr (std::is_same<T, __half>::value) {
      const __half2 h = __float22half2_rn(p.v[i]);
      c.w[i] = *reinterpret_cast<const uint32_t*>(&h);
    } else {
      c.w[2 * i] = __float_as_uint(p.v[i].x);
      c.w[2 * i + 1] = __float_as_uint(p.v[i].y);
    }
  }
  save_chunk(out, c);
}

// A lane's place in a row, and its angles.
template <int CH>
struct Place {
  int a, b;        // first component of each chunk; D: the lane has none
  Pairs<CH> c, s;  // of the rotated pairs: (A[i], B[i]), or, interleaved, of A's CH / 2, then of B's
};

// Halves of the rotated part against each other, neighbours elsewhere.
template <int CH>
__device__ __forceinline__ void find(Place<CH>& l, int item, int D, int R, bool inter) {
  const int half = inter ? 0 : R / 2;
  if (item * CH < half) {
    l.a = item * CH;
    l.b = half + item * CH;
  } else {
    l.a = 2 * half + 2 * (item - half / CH) * CH;
    l.b = l.a + CH;
  }
  if (l.a >= D) l.a = D;
  if (l.b >= D) l.b = D;
}

// The token's angles (cos 1, sin 0 where nothing is rotated).
template <int CH>
__device__ __forceinline__ void turn_to(Place<CH>& l, const NormRopeParams& p, int64_t row, bool good) {
  const int half = p.rot_dim / 2;
  const float* ct = p.cos_table + row * half;
  const float* st = p.sin_table + row * half;
  float c[CH], s[CH];
  if (!p.interleaved) {
    const bool turned = good && l.a < half;  // (half is a multiple of CH)
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      c[i] = turned ? __ldg(ct + l.a + i) : 1.f;
      s[i] = turned ? __ldg(st + l.a + i) : 0.f;
    }
  } else {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int k = i < CH / 2 ? l.a / 2 + i : l.b / 2 + (i - CH / 2);
      const bool turned = good && k < half;
      c[i] = turned ? __ldg(ct + k) : 1.f;
      s[i] = turned ? __ldg(st + k) : 0.f;
    }
  }
#pragma unroll
  for (int i = 0; i < CH / 2; ++i) {
    l.c.v[i] = make_float2(c[2 * i], c[2 * i + 1]);
    l.s.v[i] = make_float2(s[2 * i], s[2 * i + 1]);
  }
}

__device__ __forceinline__ float2 negative(float2 x) { return make_float2(-x.x, -x.y); }

// (A, B) rotated by the lane's angles; back: by their negatives.  Components from R
// on stay as they are (a product with a sine of 0 would make an infinity of one NaN in
// the other).
template <int CH, bool kBack>
__device__ __forceinline__ void turn(const Place<CH>& l, Pairs<CH>& A, Pairs<CH>& B, int R, bool inter) {
  if (!inter) {
    if (2 * l.a >= R) return;  // (half of R is a multiple of CH)
#pragma unroll
    for (int i = 0; i < CH / 2; ++i) {
      const float2 a = A.v[i], b = B.v[i], c = l.c.v[i], s = kBack ? negative(l.s.v[i]) : l.s.v[i];
      A.v[i] = __ffma2_rn(a, c, negative(__fmul2_rn(b, s)));
      B.v[i] = __ffma2_rn(a, s, __fmul2_rn(b, c));
    }
  } else {
#pragma unroll
    for (int i = 0; i < CH / 2; ++i) {
      const int k = CH / 4 + i / 2;
      const float ca = i & 1 ? l.c.v[i / 2].y : l.c.v[i / 2].x, ua = i & 1 ? l.s.v[i / 2].y : l.s.v[i / 2].x;
      const float cb = i & 1 ? l.c.v[k].y : l.c.v[k].x, ub = i & 1 ? l.s.v[k].y : l.s.v[k].x;
      const float sa = kBack ? -ua : ua, sb = kBack ? -ub : ub;
      const float2 a = A.v[i], b = B.v[i];
      if (l.a + 2 * i < R) A.v[i] = make_float2(fmaf(a.x, ca, -(a.y * sa)), fmaf(a.x, sa, a.y * ca));
      if (l.b + 2 * i < R) B.v[i] = make_float2(fmaf(b.x, cb, -(b.y * sb)), fmaf(b.x, sb, b.y * cb));
    }
  }
}

template <int CH>
__device__ __forceinline__ float dot(const Pairs<CH>& a, const Pairs<CH>& b, const Pairs<CH>& c, const Pairs<CH>& d) {
  float2 t = __fmul2_rn(a.v[0], b.v[0]);
#pragma unroll
  for (int i = 1; i < CH / 2; ++i) t = __ffma2_rn(a.v[i], b.v[i], t);
#pragma unroll
  for (int i = 0; i < CH / 2; ++i) t = __ffma2_rn(c.v[i], d.v[i], t);
  return t.x + t.y;
}
template <int CH>
__device__ __forceinline__ void times(Pairs<CH>& a, const Pairs<CH>& b) {
#pragma unroll
  for (int i = 0; i < CH / 2; ++i) a.v[i] = __fmul2_rn(a.v[i], b.v[i]);
}
template <int CH>
__device__ __forceinline__ void times(Pairs<CH>& a, float r) {
#pragma unroll
  for (int i = 0; i < CH / 2; ++i) a.v[i] = __fmul2_rn(a.v[i], make_float2(r, r));
}

// A token's slot in the cache: the offset of its page's row, for a whole warp.
// One token per sequence is the common call: the first guess says so.
__device__ __forceinline__ int64_t slot_of(const PagedCache& c, int64_t token, int lane, bool& kept) {
  int b = (int)min(token, (int64_t)c.n_seqs - 1);
  int32_t first = __ldg(c.tok_off + b), end = __ldg(c.tok_off + b + 1), ctx = __ldg(c.ctx_len + b);
  if (token < first || token >= end) {
    b = sequence_of(c.tok_off, c.n_seqs, token, lane);
    first = __ldg(c.tok_off + b);
    end = __ldg(c.tok_off + b + 1);
    ctx = __ldg(c.ctx_len + b);
  }
  const int64_t slot = (int64_t)ctx + (token - first);
  kept = ctx >= 0 && token >= first && token < end && slot <= INT32_MAX;
  const int32_t at = kept ? (int32_t)slot : 0, entry = at / c.page_size;
  int32_t page = -1;
  if (kept && entry < c.table_stride) page = __ldg(c.block_table + (int64_t)b * c.table_stride + entry);
  kept = page >= 0 && page < c.n_pages;
  return (int64_t)page * c.page_stride + (int64_t)(at - entry * c.page_size) * c.row_stride;
}

// A head row's input, output and weight: heads of q, of k, then of v (append:
// k and v into the cache, at its token's slot).
template <typename T>
struct Row {
  const T* x;
  T* y;
  const T* w;
  bool value;
};
template <typename T, bool kAppend>
__device__ __forceinline__ Row<T> row_of(const NormRopeParams& p, int64_t token, int h, int64_t slot) {
  Row<T> r;
  r.value = kAppend && h >= p.q.heads + p.k.heads;
  if (h < p.q.heads) {
    r.x = static_cast<const T*>(p.q.x) + token * p.q.x_tok + h * p.q.x_head;
    r.y = static_cast<T*>(p.q.y) + token * p.q.y_tok + h * p.q.y_head;
    r.w = static_cast<const T*>(p.q.w);
    return r;
  }
  const int hh = h - p.q.heads - (r.value ? p.k.heads : 0);
  r.x = r.value ? static_cast<const T*>(p.v) + token * p.v_tok + hh * p.v_head
                : static_cast<const T*>(p.k.x) + token * p.k.x_tok + hh * p.k.x_head;
  if constexpr (kAppend)
    r.y = static_cast<T*>(r.value ? p.cache.v : p.cache.k) + slot + hh * p.cache.head_stride;
  else
    r.y = static_cast<T*>(p.k.y) + token * p.k.y_tok + hh * p.k.y_head;
  r.w = r.value ? nullptr : static_cast<const T*>(p.k.w);
  return r;
}

// One warp per token and share of its heads.
template <typename T, int CH, bool kAppend>
__global__ void __launch_bounds__(kThreads, 6) norm_rope_kernel(const NormRopeParams p, const Shape sh) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int lane = threadIdx.x & 31;
  const int64_t w = ((int64_t)blockIdx.x * kThreads + threadIdx.x) >> 5;
  const uint32_t token = (uint32_t)w / (uint32_t)sh.warps_per_token, part = (uint32_t)w % (uint32_t)sh.warps_per_token;
  if (token >= p.n_tokens) return;
  const int groups = 32 / sh.lanes, group = lane / sh.lanes, sub = lane % sh.lanes;
  const int step = groups * sh.warps_per_token, total = p.q.heads + p.k.heads * (kAppend ? 2 : 1);
  const bool inter = p.interleaved != 0;

  Place<CH> l;
  find(l, sub, p.D, p.rot_dim, inter);
  const bool has_a = l.a < p.D, has_b = l.b < p.D;
  Chunk<T, CH> xa[kAhead], xb[kAhead];  // the next rows'
  const auto ask = [&](int h, Chunk<T, CH>& a, Chunk<T, CH>& b) {
    a = b = Chunk<T, CH>{};
    if (h >= total) return;
    const T* x = row_of<T, kAppend>(p, token, h, 0).x;
    if (has_a) a = load_chunk<T, CH>(x + l.a);
    if (has_b) b = load_chunk<T, CH>(x + l.b);
  };
#pragma unroll
  for (int u = 0; u < kAhead; ++u) ask(part * groups + group + u * step, xa[u], xb[u]);
  bool good = true, kept = true;
  int64_t row = 0, slot = 0;
  if (p.rot_dim > 0) {
    row = __ldg(p.pos + token);
    good = row >= 0 && row < p.table_rows;
    if (!good && part == 0 && lane == 0) set_status(p.dev_status, STRIDE_DEV_POSITION);
  }
  if constexpr (kAppend) {
    slot = slot_of(p.cache, token, lane, kept);
    if (!kept && part == 0 && lane == 0) set_status(p.dev_status, STRIDE_DEV_BAD_LAYOUT);
  }
  turn_to(l, p, row, good);

  const T* weight = nullptr;  // whose chunks are in wa, wb
  Pairs<CH> wa, wb;
  for (int h0 = part * groups; h0 < total; h0 += kAhead * step)
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int h = h0 + u * step + group;
      if (h0 + u * step >= total) break;  // (the warp alike)
      Pairs<CH> A = widen(xa[u]), B = widen(xb[u]);
      const Chunk<T, CH> va = xa[u], vb = xb[u];  // (values go as they are)
      if (h0 + (u + kAhead) * step < total) ask(h + kAhead * step, xa[u], xb[u]);
      const float ss = group_sum(dot(A, A, B, B), sh.lanes);
      if (h >= total || (h >= p.q.heads && !kept)) continue;
      const Row<T> r = row_of<T, kAppend>(p, token, h, slot);
      if (r.value) {
        if (has_a) save_chunk(r.y + l.a, va);
        if (has_b) save_chunk(r.y + l.b, vb);
        continue;
      }
      if (r.w) {
        if (r.w != weight) {
          weight = r.w;
          wa = widen(has_a ? load_chunk<T, CH>(r.w + l.a) : Chunk<T, CH>{});
          wb = widen(has_b ? load_chunk<T, CH>(r.w + l.b) : Chunk<T, CH>{});
        }
        times(A, wa);
        times(B, wb);
      }
      if (p.rot_dim > 0) turn<CH, false>(l, A, B, p.rot_dim, inter);
      if (r.w || !good) {
        const float by = good ? rsqrtf(ss / (float)p.D + p.eps) : NAN;
        times(A, by);
        times(B, by);
      }
      if (has_a) store_pairs(r.y + l.a, A);
      if (has_b) store_pairs(r.y + l.b, B);
    }
}

// Blocks [0, q_blocks) take the query rows, the others the key rows; each warp
// walks over tokens and sums its rows' share of the weight gradient in
// registers, the block in a fixed order.
constexpr int kBackThreads = 128, kBackWarps = kBackThreads / 32;
template <typename T, int CH>
__global__ void __launch_bounds__(kBackThreads, 4) norm_rope_backward_kernel(const NormRopeParams p, const Shape sh, const int q_blocks) {
  extern __shared__ float s_dw[];  // [kBackWarps][D]
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const bool is_q = (int)blockIdx.x < q_blocks, inter = p.interleaved != 0;
  const RowSet& rs = is_q ? p.q : p.k;
  const int block = is_q ? blockIdx.x : blockIdx.x - q_blocks, blocks = is_q ? q_blocks : (int)gridDim.x - q_blocks;
  const int groups = 32 / sh.lanes, group = lane / sh.lanes, sub = lane % sh.lanes, heads = rs.heads;
  const T* wt = static_cast<const T*>(rs.w);
  const bool want = (is_q ? p.dq_weight : p.dk_weight) != nullptr && wt != nullptr;

  Place<CH> l;
  find(l, sub, p.D, p.rot_dim, inter);
  const bool has_a = l.a < p.D, has_b = l.b < p.D;
  Pairs<CH> wa, wb, da, db;
#pragma unroll
  for (int i = 0; i < CH / 2; ++i) {
    wa.v[i] = wb.v[i] = make_float2(1.f, 1.f);
    da.v[i] = db.v[i] = make_float2(0.f, 0.f);
    if (wt && has_a) wa.v[i] = make_float2(as_f32<T>(wt[l.a + 2 * i]), as_f32<T>(wt[l.a + 2 * i + 1]));
    if (wt && has_b) wb.v[i] = make_float2(as_f32<T>(wt[l.b + 2 * i]), as_f32<T>(wt[l.b + 2 * i + 1]));
  }
  const float inv_d = 1.f / (float)p.D;
  struct Next {  // a row's x and dy on their way
    Chunk<T, CH> xa, xb, ya, yb;
  } next[kAhead];
  const int64_t first = (int64_t)block * kBackWarps + warp, stride = (int64_t)blocks * kBackWarps;
  int64_t ahead = first;  // the row that is asked for next: its token, its group's first head
  int ahead_h = 0;
  const auto ask = [&](Next& q) {
    q = Next{};
    const int h = ahead_h + group;
    if (ahead < p.n_tokens && h < heads) {
      const T* x = static_cast<const T*>(rs.x) + ahead * rs.x_tok + h * rs.x_head;
      const T* dy = static_cast<const T*>(rs.dy) + ahead * rs.dy_tok + h * rs.dy_head;
      if (has_a) {
        q.ya = load_chunk<T, CH>(dy + l.a);
        if (wt) q.xa = load_chunk<T, CH>(x + l.a);
      }
      if (has_b) {
        q.yb = load_chunk<T, CH>(dy + l.b);
        if (wt) q.xb = load_chunk<T, CH>(x + l.b);
      }
    }
    ahead_h += groups;
    if (ahead_h >= heads) {
      ahead_h = 0;
      ahead += stride;
    }
  };
#pragma unroll
  for (int u = 0; u < kAhead; ++u) ask(next[u]);
  int64_t token = first;
  int h0 = 0;
  bool good = true;
  while (token < p.n_tokens)
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (token >= p.n_tokens) break;
      if (h0 == 0) {
        int64_t row = 0;
        if (p.rot_dim > 0) {
          row = __ldg(p.pos + token);
          good = row >= 0 && row < p.table_rows;
          if (!good && lane == 0) set_status(p.dev_status, STRIDE_DEV_POSITION);
        }
        turn_to(l, p, row, good);
      }
      const int h = h0 + group;
      const Pairs<CH> A = widen(next[u].xa), B = widen(next[u].xb);
      Pairs<CH> ga = widen(next[u].ya), gb = widen(next[u].yb);
      ask(next[u]);  // (a row's own loads are done before its gradient is stored: dx may be dy)
      if (p.rot_dim > 0) turn<CH, true>(l, ga, gb, p.rot_dim, inter);  // du
      if (wt) {
        const float ss = group_sum(dot(A, A, B, B), sh.lanes), r = good ? rsqrtf(ss * inv_d + p.eps) : NAN;
        const float2 rr = make_float2(r, r);
        if (want && h < heads) {  // dw += du n
#pragma unroll
          for (int i = 0; i < CH / 2; ++i) {
            da.v[i] = __ffma2_rn(ga.v[i], __fmul2_rn(A.v[i], rr), da.v[i]);
            db.v[i] = __ffma2_rn(gb.v[i], __fmul2_rn(B.v[i], rr), db.v[i]);
          }
        }
        times(ga, wa);
        times(gb, wb);
        const float m = -group_sum(dot(ga, A, gb, B), sh.lanes) * r * r * inv_d;  // dx = r (g + x m)
        const float2 mm = make_float2(m, m);
#pragma unroll
        for (int i = 0; i < CH / 2; ++i) {
          ga.v[i] = __fmul2_rn(__ffma2_rn(A.v[i], mm, ga.v[i]), rr);
          gb.v[i] = __fmul2_rn(__ffma2_rn(B.v[i], mm, gb.v[i]), rr);
        }
      } else if (!good) {
        times(ga, NAN);
        times(gb, NAN);
      }
      if (h < heads) {
        T* dx = static_cast<T*>(rs.y) + token * rs.y_tok + h * rs.y_head;
        if (has_a) store_pairs(dx + l.a, ga);
        if (has_b) store_pairs(dx + l.b, gb);
      }
      h0 += groups;
      if (h0 >= heads) {
        h0 = 0;
        token += stride;
      }
    }
  if (!want) return;
  // lanes of equal place in the warp's groups, then the block's warps
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    float a = i & 1 ? da.v[i / 2].y : da.v[i / 2].x, b = i & 1 ? db.v[i / 2].y : db.v[i / 2].x;
    for (int o = sh.lanes; o < 32; o <<= 1) {
      a += __shfl_xor_sync(0xffffffffu, a, o);
      b += __shfl_xor_sync(0xffffffffu, b, o);
    }
    if (group == 0 && has_a) s_dw[warp * p.D + l.a + i] = a;
    if (group == 0 && has_b) s_dw[warp * p.D + l.b + i] = b;
  }
  __syncthreads();
  for (int d = threadIdx.x; d < p.D; d += kBackThreads) {
    float sum = 0.f;
    for (int x = 0; x < kBackWarps; ++x) sum += s_dw[x * p.D + d];
    p.partials[(int64_t)blockIdx.x * p.D + d] = sum;
  }
}

// ---- single components: a warp per row, a lane every 32nd pair ----

// The components and the angle of item `it` of a row: rotated pairs, then what is
// left, one by one (b: none).
struct Item {
  int a, b;
  float c, s;
};
__device__ __forceinline__ int items_of(const NormRopeParams& p) { return p.D - p.rot_dim / 2; }
__device__ __forceinline__ Item item_of(const NormRopeParams& p, int it, int64_t row, bool good) {
  const int half = p.rot_dim / 2;
  if (it >= half) return {p.rot_dim + it - half, -1, 1.f, 0.f};
  Item r = p.interleaved ? Item{2 * it, 2 * it + 1, 1.f, 0.f} : Item{it, half + it, 1.f, 0.f};
  if (good) {
    r.c = __ldg(p.cos_table + row * half + it);
    r.s = __ldg(p.sin_table + row * half + it);
  }
  return r;
}

template <typename T, bool kAppend>
__global__ void __launch_bounds__(kThreads) norm_rope_single_kernel(const NormRopeParams p) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int lane = threadIdx.x & 31, total = p.q.heads + p.k.heads * (kAppend ? 2 : 1);
  const int64_t w = ((int64_t)blockIdx.x * kThreads + threadIdx.x) >> 5, token = w / total;
  const int h = (int)(w - token * total);
  if (token >= p.n_tokens) return;
  bool good = true, kept = true;
  int64_t row = 0, slot = 0;
  if (p.rot_dim > 0) {
    row = __ldg(p.pos + token);
    good = row >= 0 && row < p.table_rows;
    if (!good && h == 0 && lane == 0) set_status(p.dev_status, STRIDE_DEV_POSITION);
  }
  if constexpr (kAppend) {
    slot = slot_of(p.cache, token, lane, kept);
    if (!kept && h == 0 && lane == 0) set_status(p.dev_status, STRIDE_DEV_BAD_LAYOUT);
  }
  if (h >= p.q.heads && !kept) return;
  const Row<T> r = row_of<T, kAppend>(p, token, h, slot);
  if (r.value) {
    for (int d = lane; d < p.D; d += 32) r.y[d] = r.x[d];
    return;
  }
  float ss = 0.f;
  for (int d = lane; r.w && d < p.D; d += 32) ss = fmaf(as_f32<T>(r.x[d]), as_f32<T>(r.x[d]), ss);
  ss = group_sum(ss, 32);
  const float by = !good ? NAN : r.w ? rsqrtf(ss / (float)p.D + p.eps) : 1.f;
  for (int it = lane; it < items_of(p); it += 32) {
    const Item i = item_of(p, it, row, good);
    const float a = as_f32<T>(r.x[i.a]) * by * (r.w ? as_f32<T>(r.w[i.a]) : 1.f);
    const float b = i.b < 0 ? 0.f : as_f32<T>(r.x[i.b]) * by * (r.w ? as_f32<T>(r.w[i.b]) : 1.f);
    r.y[i.a] = from_f32<T>(a * i.c - b * i.s);
    if (i.b >= 0) r.y[i.b] = from_f32<T>(a * i.s + b * i.c);
  }
}

// As norm_rope_backward_kernel; a lane's components of the weight gradient are
// summed in shared memory, which no other lane or warp touches.
template <typename T>
__global__ void __launch_bounds__(kBackThreads) norm_rope_backward_single_kernel(const NormRopeParams p, const int q_blocks) {
  extern __shared__ float s_dw[];  // [kBackWarps][D]
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const bool is_q = (int)blockIdx.x < q_blocks;
  const RowSet& rs = is_q ? p.q : p.k;
  const int block = is_q ? blockIdx.x : blockIdx.x - q_blocks, blocks = is_q ? q_blocks : (int)gridDim.x - q_blocks;
  const T* wt = static_cast<const T*>(rs.w);
  const bool want = (is_q ? p.dq_weight : p.dk_weight) != nullptr && wt != nullptr;
  float* dw = s_dw + warp * p.D;
  if (want)
    for (int it = lane; it < items_of(p); it += 32) {
      const Item i = item_of(p, it, 0, false);
      dw[i.a] = 0.f;
      if (i.b >= 0) dw[i.b] = 0.f;
    }
  for (int64_t token = (int64_t)block * kBackWarps + warp; token < p.n_tokens; token += (int64_t)blocks * kBackWarps) {
    int64_t row = 0;
    bool good = true;
    if (p.rot_dim > 0) {
      row = __ldg(p.pos + token);
      good = row >= 0 && row < p.table_rows;
      if (!good && lane == 0) set_status(p.dev_status, STRIDE_DEV_POSITION);
    }
    for (int h = 0; h < rs.heads; ++h) {
      const T* x = static_cast<const T*>(rs.x) + token * rs.x_tok + h * rs.x_head;
      const T* dy = static_cast<const T*>(rs.dy) + token * rs.dy_tok + h * rs.dy_head;
      T* dx = static_cast<T*>(rs.y) + token * rs.y_tok + h * rs.y_head;
      const auto du = [&](const Item& i, float& a, float& b) {
        const float ya = as_f32<T>(dy[i.a]), yb = i.b < 0 ? 0.f : as_f32<T>(dy[i.b]);
        a = ya * i.c + yb * i.s;
        b = yb * i.c - ya * i.s;
      };
      float ss = 0.f, gx = 0.f;
      for (int it = lane; wt && it < items_of(p); it += 32) {
        const Item i = item_of(p, it, row, good);
        float a, b;
        du(i, a, b);
        const float xa = as_f32<T>(x[i.a]), xb = i.b < 0 ? 0.f : as_f32<T>(x[i.b]);
        ss = fmaf(xa, xa, fmaf(xb, xb, ss));
        gx = fmaf(a * as_f32<T>(wt[i.a]), xa, gx);
        if (i.b >= 0) gx = fmaf(b * as_f32<T>(wt[i.b]), xb, gx);
      }
      ss = group_sum(ss, 32);
      gx = group_sum(gx, 32);
      const float r = !good ? NAN : wt ? rsqrtf(ss / (float)p.D + p.eps) : 1.f, m = wt ? gx * r * r / (float)p.D : 0.f;
      for (int it = lane; it < items_of(p); it += 32) {
        const Item i = item_of(p, it, row, good);
        float a, b;
        du(i, a, b);
        if (!wt) {
          dx[i.a] = from_f32<T>(a * r);
          if (i.b >= 0) dx[i.b] = from_f32<T>(b * r);
          continue;
        }
        const float xa = as_f32<T>(x[i.a]), xb = i.b < 0 ? 0.f : as_f32<T>(x[i.b]);
        if (want) {
          dw[i.a] = fmaf(a, xa * r, dw[i.a]);
          if (i.b >= 0) dw[i.b] = fmaf(b, xb * r, dw[i.b]);
        }
        dx[i.a] = from_f32<T>(r * (a * as_f32<T>(wt[i.a]) - xa * m));
        if (i.b >= 0) dx[i.b] = from_f32<T>(r * (b * as_f32<T>(wt[i.b]) - xb * m));
      }
    }
  }
  if (!want) return;
  __syncthreads();
  for (int d = threadIdx.x; d < p.D; d += kBackThreads) {
    float sum = 0.f;
    for (int k = 0; k < kBackWarps; ++k) sum += s_dw[k * p.D + d];
    p.partials[(int64_t)blockIdx.x * p.D + d] = sum;
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

template <typename... K, typename... A>
cudaError_t launch(void (*kern)(K...), dim3 grid, dim3 block, size_t smem, cudaStream_t stream, A... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kern, static_cast<K>(args)...);
  return e != cudaSuccess ? e : cudaGetLastError();
}

// CH: components of a chunk; 1: single components.
template <typename T, int CH>
cudaError_t run_forward(const NormRopeParams& p, bool append, int sms, cudaStream_t stream) {
  const int rows = p.q.heads + p.k.heads * (append ? 2 : 1);
  Shape sh = {group_lanes(p.D, CH), rows};
  if constexpr (CH > 1) {
    const int groups = 32 / sh.lanes, most = (rows + groups - 1) / groups;  // one pass over the heads per warp
    // as many warps as run at once, if there are so few tokens: what a token needs is then read once (640 tokens each of 13
    // sequences, warps an SM: 24 30.5 us, 48 to 64 33.0, 192 41.0; 256 tokens: 16 5.0, 24 to 192 4.4)
    const int64_t share = ((int64_t)sms * 24 + p.n_tokens - 1) / p.n_tokens;
    sh.warps_per_token = (int)(share < 1 ? 1 : share > most ? most : share);
  }
  const int64_t blocks = (p.n_tokens * sh.warps_per_token + kWarps - 1) / kWarps;
  if (blocks > INT32_MAX / kWarps) return cudaErrorInvalidConfiguration;
  const dim3 grid((unsigned)blocks);
  if constexpr (CH > 1)
    return append ? launch(norm_rope_kernel<T, CH, true>, grid, kThreads, 0, stream, p, sh)
                  : launch(norm_rope_kernel<T, CH, false>, grid, kThreads, 0, stream, p, sh);
  else
    return append ? launch(norm_rope_single_kernel<T, true>, grid, kThreads, 0, stream, p)
                  : launch(norm_rope_single_kernel<T, false>, grid, kThreads, 0, stream, p);
}

template <typename T, int CH>
cudaError_t run_backward(const NormRopeParams& p, cudaStream_t stream) {
  // blocks in proportion to the rows, at least one for each that has rows
  const int64_t need = (p.n_tokens + kBackWarps - 1) / kBackWarps;
  const int64_t heads = p.q.heads + p.k.heads;
  int64_t qb = p.q.heads ? (int64_t)kNormRopeBackwardBlocks * p.q.heads / heads : 0;
  if (p.q.heads && qb < 1) qb = 1;
  if (p.k.heads && qb > kNormRopeBackwardBlocks - 1) qb = kNormRopeBackwardBlocks - 1;
  int64_t kb = p.k.heads ? kNormRopeBackwardBlocks - qb : 0;
  if (qb > need) qb = need;
  if (kb > need) kb = need;
  const bool want = p.dq_weight || p.dk_weight;  // (given with their weights alone)
  const size_t smem = want ? (size_t)kBackWarps * p.D * sizeof(float) : 0;
  cudaError_t e = cudaSuccess;
  if (qb + kb > 0) {
    if constexpr (CH > 1)
      e = launch(norm_rope_backward_kernel<T, CH>, (unsigned)(qb + kb), kBackThreads, smem, stream, p, Shape{group_lanes(p.D, CH), 1}, (int)qb);
    else
      e = launch(norm_rope_backward_single_kernel<T>, (unsigned)(qb + kb), kBackThreads, smem, stream, p, (int)qb);
  }
  if (e != cudaSuccess || !want) return e;
  return launch(weight_gradient_kernel, dim3((unsigned)((p.D + 31) / 32), 2), dim3(32, 32), 0, stream, (const float*)p.partials, (int)p.D,
                (int)qb, (int)(qb + kb), p.dq_weight, p.dk_weight);
}

// Chunks of 8 components hold rows of up to 512 in 32 lanes, of 4 up to 256.
template <typename T>
int usable_chunk(int chunk, int D) {
  if (chunk >= 8 && sizeof(T) == 2 && D <= 512) return 8;
  if (chunk >= 4 && D <= 256) return 4;
  return 1;
}

template <typename T>
cudaError_t forward_of(const NormRopeParams& p, int chunk, bool append, int sms, cudaStream_t stream) {
  const int c = usable_chunk<T>(chunk, p.D);
  if constexpr (sizeof(T) == 2)
    if (c == 8) return run_forward<T, 8>(p, append, sms, stream);
  return c == 4 ? run_forward<T, 4>(p, append, sms, stream) : run_forward<T, 1>(p, append, sms, stream);
}

template <typename T>
cudaError_t backward_of(const NormRopeParams& p, int chunk, cudaStream_t stream) {
  const int c = usable_chunk<T>(chunk, p.D);
  if constexpr (sizeof(T) == 2)
    if (c == 8) return run_backward<T, 8>(p, stream);
  return c == 4 ? run_backward<T, 4>(p, stream) : run_backward<T, 1>(p, stream);
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
