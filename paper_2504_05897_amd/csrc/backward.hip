// Gradients of the layer around its experts: of the weighted sum (hmoe_combine_backward), of the gates
// (hmoe_route_backward) and of the router's product (hmoe_router_backward).  The row gather's gradient is the weighted sum
// without weights (hmoe_permute_backward in combine.hip).  Every sum is taken in a fixed order; no atomics.
#include <algorithm>

#include "common.h"

namespace hmoe {

__device__ __forceinline__ float sum_over_wave(float v) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off);
  return v;
}

// Pieces of a row: 16 bytes (VEC of N elements), or one fp32 element where rows are no multiple of that.
template <class VEC>
struct Piece;
template <>
struct Piece<u32x4> {  // bfloat16
  static constexpr int N = 8;
  static __device__ __forceinline__ void dot(float (&sum)[2], const u32x4& a, const u32x4& b) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      sum[0] = fmaf(__uint_as_float(a[i] << 16), __uint_as_float(b[i] << 16), sum[0]);
      sum[1] = fmaf(__uint_as_float(a[i] & 0xffff0000u), __uint_as_float(b[i] & 0xffff0000u), sum[1]);
    }
  }
  static __device__ __forceinline__ u32x4 times(const u32x4& a, float w) {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = f32_to_bf16_pair(w * __uint_as_float(a[i] << 16), w * __uint_as_float(a[i] & 0xffff0000u));
    return r;
  }
};
template <>
struct Piece<f32x4_t> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void dot(float (&sum)[2], const f32x4_t& a, const f32x4_t& b) {
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[i % 2] = fmaf(a[i], b[i], sum[i % 2]);
  }
  static __device__ __forceinline__ f32x4_t times(const f32x4_t& a, float w) { return a * w; }
};
template <>
struct Piece<float> {
  static constexpr int N = 1;
  static __device__ __forceinline__ void dot(float (&sum)[2], float a, float b) { sum[0] = fmaf(a, b, sum[0]); }
  static __device__ __forceinline__ float times(float a, float w) { return a * w; }
};

// d_o_perm[p] = w dy[t], d_topk_w = dy[t] . o_perm[p]: one wavefront per assignment, whose neighbours find dy[t] in the caches.
// Bound by the rows' trips to memory and back; four pieces per lane are on their way at a time.  STREAM: rows that no cache will
// hold go past them.  16384 tokens of 2048, top 6: 150 us, 5.8 TB/s (element by element 480).  d_o_perm may be o_perm: a lane reads its pieces before it writes
// them.
template <class VEC, bool ROWS, bool WEIGHTS, bool STREAM>
__global__ __launch_bounds__(256) void combine_backward_kernel(const VEC* dy, const VEC* o_perm, const int32_t* inv_perm,
                                                               const float* topk_w, int n_assign, int top_k, int row_vec, VEC* d_o_perm,
                                                               float* d_topk_w) {
  constexpr int AHEAD = 4;
  const int a = blockIdx.x * 4 + threadIdx.x / 64, lane = threadIdx.x % 64;
  if (a >= n_assign) return;
  const int p = inv_perm[a];
  const float w = ROWS ? topk_w[a] : 0.0f;
  float sum[2] = {0.0f, 0.0f};
  if ((unsigned)p < (unsigned)n_assign) {
    const VEC* g_row = dy + (size_t)(a / top_k) * row_vec;
    const VEC* o_row = WEIGHTS ? o_perm + (size_t)p * row_vec : nullptr;
    VEC* d_row = ROWS ? d_o_perm + (size_t)p * row_vec : nullptr;
    for (int c0 = lane; c0 < row_vec; c0 += 64 * AHEAD) {
      VEC g[AHEAD], o[AHEAD];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        const int c = c0 + 64 * i;
        if (c >= row_vec) continue;
        g[i] = g_row[c];
        if (WEIGHTS) o[i] = STREAM ? __builtin_nontemporal_load(o_row + c) : o_row[c];
      }
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        const int c = c0 + 64 * i;
        if (c >= row_vec) continue;
        if (WEIGHTS) Piece<VEC>::dot(sum, g[i], o[i]);
        if (ROWS) {
          const VEC r = Piece<VEC>::times(g[i], w);
          if (STREAM) __builtin_nontemporal_store(r, d_row + c);
          else d_row[c] = r;
        }
      }
    }
  }
  if (!WEIGHTS) return;
  const float dot = sum_over_wave(sum[0] + sum[1]);
  if (lane == 0) d_topk_w[a] = dot;
}

// d_logits: a group of G lanes per token, lane l of it takes experts l, l + G, ...
template <int G>
__global__ __launch_bounds__(256) void route_backward_kernel(const int32_t* __restrict__ topk_idx, const float* __restrict__ topk_w,
                                                             const float* __restrict__ d_topk_w, int n_tokens, int top_k, int n_experts,
                                                             float* __restrict__ d_logits) {
  const int t = (blockIdx.x * 256 + threadIdx.x) / G, l = threadIdx.x % G;
  if (t >= n_tokens) return;  // uniform over the group
  int id = -1;
  float w = 0.0f, dw = 0.0f;
  if (l < top_k) {
    id = topk_idx[(size_t)t * top_k + l];
    w = topk_w[(size_t)t * top_k + l];
    dw = d_topk_w[(size_t)t * top_k + l];
  }
  float mean = w * dw;
#pragma unroll
  for (int off = G / 2; off >= 1; off >>= 1) mean += __shfl_xor(mean, off, G);
  const float own = w * (dw - mean);
  for (int e0 = 0; e0 < n_experts; e0 += G) {
    const int e = e0 + l;
    float v = 0.0f;
    for (int j = 0; j < top_k; ++j) {
      // (a token per wavefront: through scalar registers)
      const int named = G == 64 ? __builtin_amdgcn_readlane(id, j) : __shfl(id, j, G);
      const float part = G == 64 ? __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(own), j)) : __shfl(own, j, G);
      if (named == e) v += part;
    }
    if (e < n_experts) d_logits[(size_t)t * n_experts + e] = v;
  }
}

// ---- the router's product --------------------------------------------------------------------
// dx = d_logits . W_g (sum over experts) and d_w_g = d_logits^T . x (sum over tokens), both on matrix instructions whose
// summed index is the slow one of W_g and x in memory.  No operand is transposed through LDS: lane l of a wave loads 16 bytes,
// a piece of consecutive columns 16 / sizeof(T) * (l % 16) .., of each of the rows that its k block needs, and column i of every
// lane's piece makes an operand of its own, for the columns {16 / sizeof(T) * n + i}.  A lane's results are then consecutive
// columns again.
//   bfloat16 layers: 16x16x32 instructions; d_logits, fp32, goes in as a sum of three bfloat16 pieces, each what is left of the
//     value cut to its upper 8 bits: together all 24 bits, so that the products are exact.  (Two would do for a dx that is rounded
//     to bfloat16, but not where its terms or `add` cancel.)  The fp32 instruction would take 27 us for each product of 16384 x 64 x 2048.
//   fp32 layers: 16x16x4 fp32 instructions.

// N of 16-bit pairs: operand dwords (rows 2 d, 2 d + 1) of the lower / upper halves of one dword column of eight rows
__device__ __forceinline__ void transpose_halves(const uint32_t (&rows)[8], u32x4& lower, u32x4& upper) {
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    lower[d] = __builtin_amdgcn_perm(rows[2 * d + 1], rows[2 * d], 0x05040100u);
    upper[d] = __builtin_amdgcn_perm(rows[2 * d + 1], rows[2 * d], 0x07060302u);
  }
}
// The next piece of eight values: their upper halves as an operand, which are taken out of the values.  (What is its own upper
// half leaves nothing, an infinity too, whose difference with itself would be a NaN.)
__device__ __forceinline__ u32x4 take_piece(float (&v)[8]) {
  u32x4 piece;
#pragma unroll
  for (int d = 0; d < 4; ++d)
    piece[d] = __builtin_amdgcn_perm(__float_as_uint(v[2 * d + 1]), __float_as_uint(v[2 * d]), 0x07060302u);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float upper = __uint_as_float(__float_as_uint(v[i]) & 0xffff0000u);
    v[i] = v[i] == upper ? 0.0f : v[i] - upper;
  }
  return piece;
}
__device__ __forceinline__ u32x4 round_piece(const float (&v)[8]) {
  return u32x4{f32_to_bf16_pair(v[0], v[1]), f32_to_bf16_pair(v[2], v[3]), f32_to_bf16_pair(v[4], v[5]), f32_to_bf16_pair(v[6], v[7])};
}
// Values i0 .. i0 + 4 of a row of n; past its end other values of the row, whose results are not stored or meet zeros.  (Always
// loaded: a load behind a condition makes the wave wait for those before it.)  WHOLE: n is a multiple of 4, and rows 16-byte
// aligned.
template <bool WHOLE>
__device__ __forceinline__ f32x4_t load_4(const float* row, int i0, int n) {
  if (WHOLE) return *(const f32x4_t*)(row + min(i0, n - 4));
  f32x4_t v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = row[min(i0 + i, n - 1)];
  return v;
}
__device__ __forceinline__ f32x4_t mfma_16x16x4_f32(float a, float b, f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

// Number formats: columns of a wave (16 pieces of 16 bytes), values per piece, tokens of a d_w_g step.
struct DwBf16 {
  typedef bf16_t T;
  static constexpr int COLS = 128, PIECE = 8, STEP = 32;
};
struct DwF32 {
  typedef float T;
  static constexpr int COLS = 64, PIECE = 4, STEP = 16;
};

// dx, bfloat16: a wave has 16 tokens x 128 columns (slice) and goes through the experts 32 at a time.
//
// W_g rows e .. + 8 of the lane's k block, eight columns from col_at, as operands.  Past the last expert both factors are cleared:
// the clamped loads bring values of other rows there, and of the token's own, and zero times an infinity is none.
__device__ __forceinline__ void load_w_rows(u32x4 (&w)[8], const bf16_t* __restrict__ w_g, int e, int n_experts, int hidden, int col_at) {
#pragma unroll
  for (int k = 0; k < 8; ++k) w[k] = *(const u32x4*)(w_g + (size_t)min(e + k, n_experts - 1) * hidden + col_at);
}
__device__ __forceinline__ void w_operands(u32x4 (&w)[8], u32x4 (&op)[8], int e0, int kblk, int n_experts) {
  if (e0 + 32 > n_experts) {  // uniform
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (e0 + 8 * kblk + k >= n_experts) w[k] = u32x4{0, 0, 0, 0};
  }
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    const uint32_t rows[8] = {w[0][p], w[1][p], w[2][p], w[3][p], w[4][p], w[5][p], w[6][p], w[7][p]};
    transpose_halves(rows, op[2 * p], op[2 * p + 1]);
  }
}
// e0: of the 32 experts at hand
__device__ __forceinline__ void add_experts(f32x4_t (&acc)[8], const f32x4_t& d0, const f32x4_t& d1, const u32x4 (&op)[8], int e0, int kblk,
                                            int n_experts) {
  float v[8] = {d0[0], d0[1], d0[2], d0[3], d1[0], d1[1], d1[2], d1[3]};
  if (e0 + 32 > n_experts) {  // uniform
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (e0 + 8 * kblk + i >= n_experts) v[i] = 0.0f;
  }
#pragma unroll
  for (int piece = 0; piece < 3; ++piece) {
    const u32x4 a = take_piece(v);
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] = mfma_16x16x32_bf16(a, op[i], acc[i]);
  }
}
// what is added to rows t0 + 4 kblk .. + 4
__device__ __forceinline__ void load_more(u32x4 (&more)[4], const bf16_t* add, int t0, int kblk, int n_tokens, int hidden, int col_at) {
#pragma unroll
  for (int r = 0; r < 4; ++r)
    more[r] = __builtin_nontemporal_load((const u32x4*)(add + (size_t)min(t0 + 4 * kblk + r, n_tokens - 1) * hidden + col_at));
}
// register r of lane (n, kblk) is token 4 kblk + r, operand i column 8 n + i
__device__ __forceinline__ void store_dx(const f32x4_t (&acc)[8], const u32x4 (&more)[4], bool added, bf16_t* dx, int t0, int kblk, int n_tokens,
                                         int hidden, int col) {
  if (col >= hidden) return;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int t = t0 + 4 * kblk + r;
    if (t >= n_tokens) continue;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = acc[i][r];
    if (added) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] += __uint_as_float(more[r][i] << 16);
        v[2 * i + 1] += __uint_as_float(more[r][i] & 0xffff0000u);
      }
    }
    __builtin_nontemporal_store(round_piece(v), (u32x4*)(dx + (size_t)t * hidden + col));
  }
}

template <bool WHOLE>
__device__ __forceinline__ void router_dx_wave(const bf16_t* __restrict__ w_g, const float* __restrict__ d_logits, const bf16_t* add,
                                               int n_tokens, int n_experts, int hidden, bf16_t* dx, int t0, int slice) {
  const int lane = threadIdx.x % 64, n = lane % 16, kblk = lane / 16;
  const int col = slice * DwBf16::COLS + 8 * n, col_at = min(col, hidden - 8);  // clamped: never stored
  f32x4_t acc[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) acc[i] = f32x4_t{0, 0, 0, 0};
  u32x4 more[4];  // on its way while the experts are multiplied
  if (add) load_more(more, add, t0, kblk, n_tokens, hidden, col_at);
  const float* row = d_logits + (size_t)min(t0 + n, n_tokens - 1) * n_experts;
  for (int e0 = 0; e0 < n_experts; e0 += 32) {
    const int e = e0 + 8 * kblk;
    u32x4 w[8], op[8];
    load_w_rows(w, w_g, e, n_experts, hidden, col_at);
    const f32x4_t d0 = load_4<WHOLE>(row, e, n_experts), d1 = load_4<WHOLE>(row, e + 4, n_experts);
    w_operands(w, op, e0, kblk, n_experts);
    add_experts(acc, d0, d1, op, e0, kblk, n_experts);
  }
  store_dx(acc, more, add != nullptr, dx, t0, kblk, n_tokens, hidden, col);
}

// Large batches over at most 32 EC experts: a wave keeps its columns of W_g as operands and goes from one 16 tokens to another,
// the next ones on their way.  16384 tokens, 64 experts of 2048, from memory: 31 us, 4.5 TB/s; with W_g read
// for every 16 tokens 39.
template <int EC, bool WHOLE>
__global__ __launch_bounds__(256, EC <= 2 ? 2 : 1) void router_dx_walk_kernel(const bf16_t* __restrict__ w_g, const float* __restrict__ d_logits,
                                                                              const bf16_t* add, int n_tokens, int n_experts, int hidden,
                                                                              bf16_t* dx) {
  const int lane = threadIdx.x % 64, n = lane % 16, kblk = lane / 16;
  const int col = blockIdx.y * DwBf16::COLS + 8 * n, col_at = min(col, hidden - 8);
  struct Tokens {
    f32x4_t d[EC][2];
    u32x4 more[4];
  } now, next;
  auto load = [&](Tokens& k, int t0) {
    const float* row = d_logits + (size_t)min(t0 + n, n_tokens - 1) * n_experts;
#pragma unroll
    for (int c = 0; c < EC; ++c)
#pragma unroll
      for (int i = 0; i < 2; ++i) k.d[c][i] = load_4<WHOLE>(row, 32 * c + 8 * kblk + 4 * i, n_experts);
    if (add) load_more(k.more, add, t0, kblk, n_tokens, hidden, col_at);
  };
  const int stride = gridDim.x * 64;
  int t0 = (blockIdx.x * 4 + threadIdx.x / 64) * 16;
  if (t0 >= n_tokens) return;
  u32x4 op[EC][8];
  load(next, t0);
#pragma unroll
  for (int c = 0; c < EC; ++c) {
    u32x4 w[8];
    load_w_rows(w, w_g, 32 * c + 8 * kblk, n_experts, hidden, col_at);
    w_operands(w, op[c], 32 * c, kblk, n_experts);
  }
  for (; t0 < n_tokens; t0 += stride) {
    now = next;
    load(next, min(t0 + stride, n_tokens - 1));  // (past the end: its last token again, unused)
    __builtin_amdgcn_sched_barrier(0);
    f32x4_t acc[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] = f32x4_t{0, 0, 0, 0};
#pragma unroll
    for (int c = 0; c < EC; ++c) add_experts(acc, now.d[c][0], now.d[c][1], op[c], 32 * c, kblk, n_experts);
    store_dx(acc, now.more, add != nullptr, dx, t0, kblk, n_tokens, hidden, col);
  }
}

// dx, fp32: 16 tokens x 64 columns, the experts 16 at a time; instruction s of a step has experts 4 (l / 16) + s.
template <bool WHOLE>
__device__ __forceinline__ void router_dx_wave(const float* __restrict__ w_g, const float* __restrict__ d_logits, const float* add, int n_tokens,
                                               int n_experts, int hidden, float* dx, int t0, int slice) {
  const int lane = threadIdx.x % 64, n = lane % 16, kblk = lane / 16;
  const int col = slice * DwF32::COLS + 4 * n;
  f32x4_t acc[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) acc[i] = f32x4_t{0, 0, 0, 0};
  const float* row = d_logits + (size_t)min(t0 + n, n_tokens - 1) * n_experts;
  for (int e0 = 0; e0 < n_experts; e0 += 16) {
    const int e = e0 + 4 * kblk;
    f32x4_t w[4];
#pragma unroll
    for (int s = 0; s < 4; ++s)
      w[s] = load_4<WHOLE>(w_g + (size_t)min(e + s, n_experts - 1) * hidden, col, hidden);
    f32x4_t d = load_4<WHOLE>(row, e, n_experts);
    if (e0 + 16 > n_experts) {  // uniform
#pragma unroll
      for (int s = 0; s < 4; ++s)
        if (e + s >= n_experts) {  // (both, as above)
          w[s] = f32x4_t{0, 0, 0, 0};
          d[s] = 0.0f;
        }
    }
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i] = mfma_16x16x4_f32(d[s], w[s][i], acc[i]);
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int t = t0 + 4 * kblk + r;
    if (t >= n_tokens) continue;
    f32x4_t v = {acc[0][r], acc[1][r], acc[2][r], acc[3][r]};
    if (add) v += load_4<WHOLE>(add + (size_t)t * hidden, col, hidden);
    float* out = dx + (size_t)t * hidden;
    if (WHOLE) {
      if (col < hidden) *(f32x4_t*)(out + col) = v;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (col + i < hidden) out[col + i] = v[i];
    }
  }
}

// dx of large batches: four waves per block
template <class NUM, bool WHOLE>
__global__ __launch_bounds__(256, 4) void router_dx_kernel(const typename NUM::T* __restrict__ w_g, const float* __restrict__ d_logits,
                                                                         const typename NUM::T* add, int n_tokens, int n_experts, int hidden,
                                                                         typename NUM::T* dx) {
  const int t0 = (blockIdx.x * 4 + threadIdx.x / 64) * 16;
  if (t0 < n_tokens) router_dx_wave<WHOLE>(w_g, d_logits, add, n_tokens, n_experts, hidden, dx, t0, blockIdx.y);
}

// d_w_g: a block takes 16 M experts x NUM::COLS columns over some of the tokens, its waves a step of STEP tokens each
// in turn.  The waves' sums meet in LDS, the blocks' of several chunks of the tokens in router_dw_sum_kernel, all in a
// fixed order.  M = 4: a step's x serves 64 experts; M = 1: four times the blocks, for batches that make few.
//
// The operands of a step.  Tokens past the end are cleared where they are multiplied, in the step that has some: behind the
// loads it would be a wait for them.  Operand m of lane n has expert e + m, e = e0 + M n.
template <class NUM, int M, bool WHOLE>
struct DwStep;
template <int M, bool WHOLE>
__device__ __forceinline__ void load_logits(float (&v)[M], const float* row, int e, int n_experts) {
  if constexpr (M == 4) {
    const f32x4_t q = load_4<WHOLE>(row, e, n_experts);
#pragma unroll
    for (int m = 0; m < 4; ++m) v[m] = q[m];
  } else {
    v[0] = row[min(e, n_experts - 1)];
  }
}
template <int M, bool WHOLE>
struct DwStep<DwBf16, M, WHOLE> {
  u32x4 x[8];
  float d[8][M];
  __device__ __forceinline__ void load(const bf16_t* __restrict__ x_in, const float* __restrict__ d_logits, int t0, int t_end, int col_at,
                                       int e, int n_experts, int hidden, int kblk) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int at = min(t0 + 8 * kblk + k, t_end - 1);
      x[k] = *(const u32x4*)(x_in + (size_t)at * hidden + col_at);
      load_logits<M, WHOLE>(d[k], d_logits + (size_t)at * n_experts, e, n_experts);
    }
  }
  // left: tokens from t0 to the end
  __device__ __forceinline__ void multiply(f32x4_t (&acc)[M][8], int left, int kblk) {
    if (left < DwBf16::STEP) {  // uniform
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (8 * kblk + k >= left) {  // (both: zero times an infinity is none)
          x[k] = u32x4{0, 0, 0, 0};
#pragma unroll
          for (int m = 0; m < M; ++m) d[k][m] = 0.0f;
        }
    }
    u32x4 op[8];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const uint32_t rows[8] = {x[0][p], x[1][p], x[2][p], x[3][p], x[4][p], x[5][p], x[6][p], x[7][p]};
      transpose_halves(rows, op[2 * p], op[2 * p + 1]);
    }
#pragma unroll
    for (int m = 0; m < M; ++m) {
      float v[8] = {d[0][m], d[1][m], d[2][m], d[3][m], d[4][m], d[5][m], d[6][m], d[7][m]};
#pragma unroll
      for (int piece = 0; piece < 3; ++piece) {
        const u32x4 a = take_piece(v);
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[m][i] = mfma_16x16x32_bf16(a, op[i], acc[m][i]);
      }
    }
  }
};
template <int M, bool WHOLE>
struct DwStep<DwF32, M, WHOLE> {
  f32x4_t x[4];
  float d[4][M];
  __device__ __forceinline__ void load(const float* __restrict__ x_in, const float* __restrict__ d_logits, int t0, int t_end, int col_at, int e,
                                       int n_experts, int hidden, int kblk) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int at = min(t0 + 4 * k + kblk, t_end - 1);
      x[k] = load_4<WHOLE>(x_in + (size_t)at * hidden, col_at, hidden);
      load_logits<M, WHOLE>(d[k], d_logits + (size_t)at * n_experts, e, n_experts);
    }
  }
  __device__ __forceinline__ void multiply(f32x4_t (&acc)[M][4], int left, int kblk) {
    if (left < DwF32::STEP) {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (4 * k + kblk >= left) {
          x[k] = f32x4_t{0, 0, 0, 0};
#pragma unroll
          for (int m = 0; m < M; ++m) d[k][m] = 0.0f;
        }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int m = 0; m < M; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[m][i] = mfma_16x16x4_f32(d[k][m], x[k][i], acc[m][i]);
  }
};

template <class NUM, int WAVES>
using DwRed = float[WAVES][NUM::PIECE * 4][64];

// experts 16 M tile .., columns of `slice`, tokens t_begin .. t_end -> out [E, H]
// AHEAD steps per wave are on their way while one is multiplied.
template <class NUM, int M, int WAVES, int AHEAD, bool WHOLE>
__device__ __forceinline__ void router_dw_block(const typename NUM::T* __restrict__ x, const float* __restrict__ d_logits, int n_experts,
                                                int hidden, int slice, int tile, int t_begin, int t_end, float* __restrict__ out,
                                                DwRed<NUM, WAVES>& red) {
  constexpr int PIECE = NUM::PIECE;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, n = lane % 16, kblk = lane / 16;
  const int col = slice * NUM::COLS + PIECE * n;
  const int col_at = PIECE == 8 ? min(col, hidden - 8) : col;  // (fp32 rows of any length are checked where they are read)
  const int e0 = 16 * M * tile, e = e0 + M * n;
  f32x4_t acc[M][PIECE];
#pragma unroll
  for (int m = 0; m < M; ++m)
#pragma unroll
    for (int i = 0; i < PIECE; ++i) acc[m][i] = f32x4_t{0, 0, 0, 0};
  constexpr int STRIDE = WAVES * NUM::STEP, RING = AHEAD + 1;
  int t = t_begin + wave * NUM::STEP;
  if (t < t_end) {
    DwStep<NUM, M, WHOLE> ring[RING];
    // (steps past the end load its last token; nothing multiplies them)
    auto load = [&](DwStep<NUM, M, WHOLE>& step, int t0) {
      step.load(x, d_logits, t0, t_end, col_at, e, n_experts, hidden, kblk);
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) load(ring[i], t + i * STRIDE);
    for (bool more = true; more;) {
#pragma unroll
      for (int i = 0; i < RING; ++i) {
        if (more) {
          load(ring[(i + AHEAD) % RING], t + AHEAD * STRIDE);
          __builtin_amdgcn_sched_barrier(0);  // (left alone, the loads move down to their uses)
          ring[i].multiply(acc, t_end - t, kblk);
          t += STRIDE;
          more = t < t_end;
        }
      }
    }
  }
  // register r of lane (n, kblk) is row 4 kblk + r of the instruction: expert e0 + M (4 kblk + r) + m; operand i column PIECE n + i
#pragma unroll
  for (int m = 0; m < M; ++m) {
    if (m > 0) __syncthreads();
#pragma unroll
    for (int i = 0; i < PIECE; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) red[wave][i * 4 + r][lane] = acc[m][i][r];
    __syncthreads();
    // a thread per row and some of its piece of columns
    constexpr int SOME = PIECE * 4 / WAVES;
    static_assert(WAVES % 4 == 0 && SOME >= 1, "");
    const int r = wave % 4, i0 = wave / 4 * SOME, to = e0 + M * (4 * kblk + r) + m;
    float v[SOME];
#pragma unroll
    for (int i = 0; i < SOME; ++i) {
      v[i] = red[0][(i0 + i) * 4 + r][lane];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) v[i] += red[w][(i0 + i) * 4 + r][lane];
    }
    if (to < n_experts) {
      float* row = out + (size_t)to * hidden;
      if constexpr (PIECE == 8) {  // (columns come in eights)
#pragma unroll
        for (int i = 0; i < SOME; i += 4)
          if (col < hidden) *(f32x4_t*)(row + col + i0 + i) = f32x4_t{v[i], v[i + 1], v[i + 2], v[i + 3]};
      } else {
#pragma unroll
        for (int i = 0; i < SOME; ++i)
          if (col + i0 + i < hidden) row[col + i0 + i] = v[i];
      }
    }
  }
}

// One wave per SIMD with two steps ahead (16384 tokens, 64 experts of 2048, from memory: 22 us; two waves without: 37).
constexpr int DW_WAVES = 4;
template <class NUM, bool WHOLE>
__global__ __launch_bounds__(64 * DW_WAVES, 1) void router_dw_kernel(const typename NUM::T* __restrict__ x, const float* __restrict__ d_logits,
                                                                     int n_tokens, int n_experts, int hidden, int chunk_tokens,
                                                                     float* __restrict__ out) {
  __shared__ DwRed<NUM, DW_WAVES> red;
  const int t_begin = blockIdx.y * chunk_tokens;
  router_dw_block<NUM, 4, DW_WAVES, 2, WHOLE>(x, d_logits, n_experts, hidden, blockIdx.x, blockIdx.z, t_begin, min(t_begin + chunk_tokens, n_tokens),
                          out + (size_t)blockIdx.y * n_experts * hidden, red);
}

// Batches of up to SMALL_TOKENS: both results in one launch, d_w_g without chunks.  The first dw_blocks blocks are d_w_g's (they
// take longest), the others eight waves of dx.
constexpr int SMALL_WAVES = 8;
template <class NUM, bool WHOLE>
__global__ __launch_bounds__(64 * SMALL_WAVES, 2) void router_backward_small_kernel(const typename NUM::T* __restrict__ x,
                                                                                 const typename NUM::T* __restrict__ w_g,
                                                                                 const float* __restrict__ d_logits, int n_tokens, int n_experts,
                                                                                 int hidden, const typename NUM::T* add, typename NUM::T* dx,
                                                                                 float* __restrict__ d_w_g, int slices, int dw_blocks) {
  __shared__ DwRed<NUM, SMALL_WAVES> red;
  const int b = blockIdx.x;
  if (b < dw_blocks) {
    router_dw_block<NUM, 1, SMALL_WAVES, 1, WHOLE>(x, d_logits, n_experts, hidden, b % slices, b / slices, 0, n_tokens, d_w_g, red);
  } else {
    const int i = b - dw_blocks, t0 = (i / slices * SMALL_WAVES + threadIdx.x / 64) * 16;
    if (t0 < n_tokens) router_dx_wave<WHOLE>(w_g, d_logits, add, n_tokens, n_experts, hidden, dx, t0, i % slices);
  }
}

// d_w_g = sum of the chunks' parts
__global__ __launch_bounds__(256) void router_dw_sum_kernel(const float* __restrict__ parts, int n_chunks, long n, float* __restrict__ out) {
  const long i = ((long)blockIdx.x * 256 + threadIdx.x) * 4;
  if (i >= n) return;
  if (n % 4 == 0) {
    f32x4_t v = *(const f32x4_t*)(parts + i);
#pragma unroll 8
    for (int c = 1; c < n_chunks; ++c) v += *(const f32x4_t*)(parts + (long)c * n + i);
    *(f32x4_t*)(out + i) = v;
  } else {
    for (long k = i; k < i + 4 && k < n; ++k) {
      float v = parts[k];
      for (int c = 1; c < n_chunks; ++c) v += parts[(long)c * n + k];
      out[k] = v;
    }
  }
}

// Up to this many tokens one launch does everything (us, this launch / those of larger batches, bfloat16: 64 experts of 2048, 1003 and
// 2048 tokens 7.0 / 14.8, 10.6 / 18.7; 160 of 4096 20.3 / 24.0, 33.2 / 34.5; 256 of 4096 23.3 / 27.2, 43.3 / 42.3, but 256 tokens 16.5 / 14.9).
// In fp32, with twice the bytes and steps half as long, the two meet earlier (64 of 2048 16.5 / 17.7, 32.1 / 24.9; 256 of 4096, 64 and 256
// tokens 12.8 / 13.7, 25.5 / 17.7, 2048 tokens 139.7 / 95.7): a border that knew the type and the experts would lie lower there.
constexpr int SMALL_TOKENS = 2048;
// Beyond: chunks of the tokens in the d_w_g launch, as many as give every CU a block.
struct DwPlan {
  int slices, tiles, chunks, chunk_tokens;
  int most;  // chunks of this many tokens or fewer, at most
};
static DwPlan dw_plan(const hmoe_layer_desc& d, int T) {
  DwPlan p;
  const int cols = d.dtype == HMOE_F32 ? DwF32::COLS : DwBf16::COLS;
  p.slices = (d.hidden + cols - 1) / cols;
  p.tiles = (d.n_experts + 63) / 64;
  const long blocks = (long)p.slices * p.tiles;
  p.most = T <= SMALL_TOKENS ? 1 : (int)std::max(1l, std::min(256 / blocks, (T + 255l) / 256));
  p.chunk_tokens = (int)std::min(0x7fffff00l, std::max(256l, (T + p.most - 1l) / p.most + 255) / 256 * 256);
  p.chunks = (int)std::max(1l, ((long)T + p.chunk_tokens - 1) / p.chunk_tokens);
  return p;
}

template <class NUM, bool WHOLE>
static void launch_router_backward(const hmoe_layer_desc& d, const typename NUM::T* x, const typename NUM::T* w_g, const float* d_logits, int T,
                                   const typename NUM::T* add, typename NUM::T* dx, float* d_w_g, float* workspace, hipStream_t s) {
  const int E = d.n_experts, H = d.hidden;
  const DwPlan p = dw_plan(d, T);
  if (T <= SMALL_TOKENS) {
    const int dw_blocks = d_w_g ? p.slices * ((E + 15) / 16) : 0, dx_blocks = dx ? p.slices * ((T + 16 * SMALL_WAVES - 1) / (16 * SMALL_WAVES)) : 0;
    if (dw_blocks + dx_blocks > 0)
      hipLaunchKernelGGL((router_backward_small_kernel<NUM, WHOLE>), dim3((unsigned)(dw_blocks + dx_blocks)), dim3(64 * SMALL_WAVES), 0, s, x, w_g, d_logits,
                         T, E, H, add, dx, d_w_g, p.slices, dw_blocks);
    return;
  }
  if (dx) {
    const unsigned blocks = (unsigned)((T + 63) / 64);
    auto launch = [&](auto kernel, unsigned most) {
      hipLaunchKernelGGL(kernel, dim3(std::min(blocks, most), (unsigned)p.slices), dim3(256), 0, s, w_g, d_logits, add, T, E, H, dx);
    };
    const unsigned per_slice = (unsigned)std::max(1, 512 / p.slices);  // two blocks per CU
    if constexpr (NUM::PIECE == 8) {
      if (E <= 32) launch(&router_dx_walk_kernel<1, WHOLE>, per_slice);
      else if (E <= 64) launch(&router_dx_walk_kernel<2, WHOLE>, per_slice);
      else if (E <= 128) launch(&router_dx_walk_kernel<4, WHOLE>, (per_slice + 1) / 2);
      else launch(&router_dx_kernel<NUM, WHOLE>, blocks);
    } else {
      launch(&router_dx_kernel<NUM, WHOLE>, blocks);
    }
  }
  if (d_w_g) {
    const dim3 grid((unsigned)p.slices, (unsigned)p.chunks, (unsigned)p.tiles);
    hipLaunchKernelGGL((router_dw_kernel<NUM, WHOLE>), grid, dim3(64 * DW_WAVES), 0, s, x, d_logits, T, E, H, p.chunk_tokens,
                       p.chunks > 1 ? workspace : d_w_g);
    if (p.chunks > 1) {
      const long n = (long)E * H;
      hipLaunchKernelGGL(router_dw_sum_kernel, dim3((unsigned)((n + 1023) / 1024)), dim3(256), 0, s, workspace, p.chunks, n, d_w_g);
    }
  }
}

}  // namespace hmoe

using namespace hmoe;

extern "C" int32_t hmoe_combine_backward(const hmoe_layer_desc* desc, const void* dy, const void* o_perm, const int32_t* inv_perm,
                                         const float* topk_w, int32_t T, void* d_o_perm, float* d_topk_w, void* stream) {
  int rc = check_desc(desc);
  if (rc != HMOE_OK) return rc;
  if (T < 0 || T > 0x7fffffff / desc->top_k) return HMOE_ERR_INVALID_ARG;
  if (T == 0) return HMOE_OK;
  if (!dy || !inv_perm || (!d_o_perm && !d_topk_w) || (d_o_perm && !topk_w) || (d_topk_w && !o_perm)) return HMOE_ERR_INVALID_ARG;
  if (!aligned16(dy) || (d_topk_w && !aligned16(o_perm)) || (d_o_perm && !aligned16(d_o_perm))) return HMOE_ERR_INVALID_ARG;
  if (!aligned4(inv_perm) || !aligned4(topk_w) || !aligned4(d_topk_w)) return HMOE_ERR_INVALID_ARG;
  if (desc->dtype != HMOE_F32 && desc->hidden % 8 != 0) return HMOE_ERR_UNSUPPORTED;
  const int n_assign = T * desc->top_k, H = desc->hidden;
  auto launch = [&](auto type) {
    typedef decltype(type) VEC;
    const int row_vec = H / Piece<VEC>::N;
    const bool stream_past = (size_t)n_assign * row_vec * sizeof(VEC) >= (size_t)64 << 20;
    const auto kernel = d_o_perm && d_topk_w ? (stream_past ? &combine_backward_kernel<VEC, true, true, true> : &combine_backward_kernel<VEC, true, true, false>)
                        : d_o_perm           ? (stream_past ? &combine_backward_kernel<VEC, true, false, true> : &combine_backward_kernel<VEC, true, false, false>)
                                             : (stream_past ? &combine_backward_kernel<VEC, false, true, true> : &combine_backward_kernel<VEC, false, true, false>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(((long)n_assign + 3) / 4)), dim3(256), 0, (hipStream_t)stream, (const VEC*)dy, (const VEC*)o_perm,
                       inv_perm, topk_w, n_assign, desc->top_k, row_vec, (VEC*)d_o_perm, d_topk_w);
  };
  if (desc->dtype != HMOE_F32) launch(u32x4{});
  else if (H % 4 == 0) launch(f32x4_t{});
  else launch(0.0f);
  HMOE_HIP(hipGetLastError());
  return HMOE_OK;
}

extern "C" int32_t hmoe_route_backward(const hmoe_layer_desc* desc, const int32_t* topk_idx, const float* topk_w, const float* d_topk_w,
                                       int32_t T, float* d_logits, void* stream) {
  int rc = check_desc(desc);
  if (rc != HMOE_OK) return rc;
  if (T < 0 || T > 0x7fffffff / desc->top_k) return HMOE_ERR_INVALID_ARG;
  if (T == 0) return HMOE_OK;
  if (!topk_idx || !topk_w || !d_topk_w || !d_logits) return HMOE_ERR_INVALID_ARG;
  if (!aligned4(topk_idx) || !aligned4(topk_w) || !aligned4(d_topk_w) || !aligned4(d_logits)) return HMOE_ERR_INVALID_ARG;
  hipStream_t s = (hipStream_t)stream;
  // a group has a lane for every choice; top_k <= n_experts, so one as wide as the experts up to 64 does
  auto launch = [&](auto kernel, int g) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)(((long)T * g + 255) / 256)), dim3(256), 0, s, topk_idx, topk_w, d_topk_w, T, desc->top_k,
                       desc->n_experts, d_logits);
  };
  if (desc->n_experts <= 8) launch(&route_backward_kernel<8>, 8);
  else if (desc->n_experts <= 16) launch(&route_backward_kernel<16>, 16);
  else if (desc->n_experts <= 32) launch(&route_backward_kernel<32>, 32);
  else launch(&route_backward_kernel<64>, 64);
  HMOE_HIP(hipGetLastError());
  return HMOE_OK;
}

extern "C" size_t hmoe_router_backward_workspace_bytes(const hmoe_layer_desc* desc, int32_t T) {
  if (check_desc(desc) != HMOE_OK || T < 0) return 0;
  const DwPlan p = dw_plan(*desc, T);
  return p.most > 1 ? (size_t)p.most * desc->n_experts * desc->hidden * sizeof(float) : 16;  // (what holds T tokens holds fewer)
}

extern "C" int32_t hmoe_router_backward(const hmoe_layer_desc* desc, const void* x, const void* w_g, const float* d_logits, int32_t T,
                                        const void* add, void* dx, float* d_w_g, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check_desc(desc);
  if (rc != HMOE_OK) return rc;
  if (T < 0 || T > 0x7fffffff / desc->top_k || T > 0x7fff0000) return HMOE_ERR_INVALID_ARG;  // (token numbers past the last tile fit)
  if (!dx && !d_w_g) return HMOE_ERR_INVALID_ARG;
  if (T > 0 && (!d_logits || (dx && !w_g) || (d_w_g && !x))) return HMOE_ERR_INVALID_ARG;
  if (!aligned16(d_logits) || (dx && (!aligned16(dx) || !aligned16(w_g) || !aligned16(add))) || (d_w_g && (!aligned16(d_w_g) || !aligned16(x))))
    return HMOE_ERR_INVALID_ARG;
  if (desc->dtype != HMOE_F32 && desc->hidden % 16 != 0) return HMOE_ERR_UNSUPPORTED;
  if (!workspace || workspace_bytes < hmoe_router_backward_workspace_bytes(desc, T)) return HMOE_ERR_WORKSPACE;
  if (!aligned16(workspace)) return HMOE_ERR_INVALID_ARG;
  hipStream_t s = (hipStream_t)stream;
  auto launch = [&](auto num, auto launch_of) {
    typedef typename decltype(num)::T V;
    launch_of(*desc, (const V*)x, (const V*)w_g, d_logits, T, (const V*)add, (V*)dx, d_w_g, (float*)workspace, s);
  };
  const bool rows_of_4 = desc->n_experts % 4 == 0 && desc->hidden % 4 == 0;
  if (desc->dtype == HMOE_F32) launch(DwF32{}, rows_of_4 ? &launch_router_backward<DwF32, true> : &launch_router_backward<DwF32, false>);
  else launch(DwBf16{}, rows_of_4 ? &launch_router_backward<DwBf16, true> : &launch_router_backward<DwBf16, false>);
  HMOE_HIP(hipGetLastError());
  return HMOE_OK;
}
