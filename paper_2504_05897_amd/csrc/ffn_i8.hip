// Expert FFN in 8-bit integers (HMOE_BF16_I8): what its paths share (quantisation of rows), and the reference path.
//
// A call is four launches: the tokens' rows, in sorted order, become codes and scales; gate/up products and SwiGLU leave h in
// fp32; the rows of h become codes and scales; the down projection rounds to bfloat16.  h cannot be quantised where it is
// made: the scale of a row is known when its last value is.  It stays in fp32 until then, since a code is decided by where
// 127 h / amax lies between two halves: 16 bits for it would move one code in a thousand, which is as large an error of the
// result as its final rounding.
#include "i8_rows.h"

namespace hmoe {

struct I8Ctx {
  const int32_t* offsets;
  const int32_t* slot_of;
  const char* slots;
  size_t slot_bytes;
  ActiveMask active;
  bool all_active;
  int n_experts, hidden, ffn;
  const int32_t* row_map;
  int map_div;
};

// expert that owns sorted row p: offsets[e] <= p < offsets[e+1]
__device__ __forceinline__ int i8_expert_of(const int32_t* __restrict__ offsets, int n_experts, int p) {
  int lo = 0, hi = n_experts;  // invariant: offsets[lo] <= p < offsets[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (offsets[mid] <= p) lo = mid; else hi = mid;
  }
  return lo;
}

// Whether sorted row p takes part in the launch: a caller may only know how many rows there are at most, and a call over some
// experts leaves the others' rows to their own calls.
__device__ __forceinline__ bool row_takes_part(const I8Ctx& c, int p) {
  if (p >= c.offsets[c.n_experts]) return false;
  if (c.all_active) return true;
  const int e = i8_expert_of(c.offsets, c.n_experts, p);
  return c.active.test(e) && c.slot_of[e] >= 0;
}

// Codes and scale of a row by a wavefront, which holds its values in registers between their maximum and the codes.
template <class T, int HELD>
__device__ __forceinline__ void quantize_row_wave(const T* __restrict__ row, int K, int8_t* __restrict__ out, float* __restrict__ scale) {
  const int lane = threadIdx.x % 64;
  float v[HELD][8];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < HELD; ++i) {
    const int k = 8 * (i * 64 + lane);
    if (k < K) load_8(row + k, v[i]);
  }
#pragma unroll
  for (int i = 0; i < HELD; ++i)
    if (8 * (i * 64 + lane) < K) m = max(m, magnitude_bits(v[i]));
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, off));
  const RowQuant q = row_quant(m);
#pragma unroll
  for (int i = 0; i < HELD; ++i) {
    const int k = 8 * (i * 64 + lane);
    if (k < K) *(uint2*)(out + k) = codes_of(v[i], q);
  }
  if (lane == 0) *scale = q.scale;
}

// codes[p] and scales[p] of sorted row p of `in` (through the row map if there is one).  Rows of up to 64 * 8 * HELD values: a
// wavefront each, four per block and no barrier.
template <class T, int HELD>
__global__ __launch_bounds__(256) void quantize_rows_wave_kernel(I8Ctx c, const T* __restrict__ in, int n_rows, int K,
                                                                 int8_t* __restrict__ codes, float* __restrict__ scales) {
  const int p = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + threadIdx.x / 64);
  if (p >= n_rows || !row_takes_part(c, p)) return;
  quantize_row_wave<T, HELD>(in + (size_t)mapped_row(c.row_map, c.map_div, p) * K, K, codes + (size_t)p * K, scales + p);
}

// Longer rows: a block of 1024 threads each.  What is beyond 16 values per thread is read twice.
template <class T>
__global__ __launch_bounds__(1024) void quantize_rows_block_kernel(I8Ctx c, const T* __restrict__ in, int K, int8_t* __restrict__ codes,
                                                                   float* __restrict__ scales) {
  __shared__ uint32_t wave_max[16];
  __shared__ float scale;
  const int p = blockIdx.x;
  if (!row_takes_part(c, p)) return;
  own_row_codes<16, 2>(in + (size_t)mapped_row(c.row_map, c.map_div, p) * K, K, codes + (size_t)p * K, &scale, wave_max);
  if (threadIdx.x == 0) scales[p] = scale;  // (the thread that wrote it)
}

template <class T>
static void launch_quantize(const I8Ctx& c, int n_rows, const T* in, int K, int8_t* codes, float* scales, hipStream_t s) {
  auto waves = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)((n_rows + 3l) / 4)), dim3(256), 0, s, c, in, n_rows, K, codes, scales);
  };
  if (K <= 512) waves(&quantize_rows_wave_kernel<T, 1>);
  else if (K <= 1024) waves(&quantize_rows_wave_kernel<T, 2>);
  else if (K <= 1536) waves(&quantize_rows_wave_kernel<T, 3>);
  else if (K <= 2048) waves(&quantize_rows_wave_kernel<T, 4>);
  else if (K <= 4096) waves(&quantize_rows_wave_kernel<T, 8>);
  else hipLaunchKernelGGL(quantize_rows_block_kernel<T>, dim3((unsigned)n_rows), dim3(1024), 0, s, c, in, K, codes, scales);
}

// ---- one row of codes per token ---------------------------------------------------------------
// A batch with a row map reads every token top_k times.  Its codes once per token are a K-th of the traffic (16384 tokens of
// 2048, top 6: 100 -> 34 us), and the tiles find them through code_row as they find bfloat16 rows through the row map.  Only rows
// that the map names are read, whatever it names: a first launch notes for each token one sorted row that names it, and a
// second quantises the tokens whose note is true (memory that nothing was noted in may hold anything).  Tokens past the
// expected number, as calls over some of the assignments may name, get a row per sorted row behind the others.
__global__ __launch_bounds__(256) void note_tokens_kernel(I8Ctx c, int n_tokens, int32_t* __restrict__ code_row, int32_t* __restrict__ owner) {
  const int p = blockIdx.x * 256 + threadIdx.x;
  if (p >= c.offsets[c.n_experts]) return;
  const int t = c.row_map[p] / c.map_div;
  const bool by_token = (unsigned)t < (unsigned)n_tokens;
  code_row[p] = by_token ? t : n_tokens + p;
  if (by_token) __hip_atomic_store(owner + t, p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // (one of them, whichever)
}

constexpr int FAR_BLOCKS = 64;  // in front: they look through the row map for tokens past the expected number
template <int HELD>
__global__ __launch_bounds__(256) void quantize_tokens_kernel(I8Ctx c, const bf16_t* __restrict__ x, int n_tokens, const int32_t* __restrict__ owner,
                                                              int8_t* __restrict__ codes, float* __restrict__ scales) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, H = c.hidden;
  const int n = c.offsets[c.n_experts];
  if (blockIdx.x >= FAR_BLOCKS) {
    const int t = (blockIdx.x - FAR_BLOCKS) * 4 + wave;
    if (t >= n_tokens) return;
    const int p = owner[t];
    if ((unsigned)p >= (unsigned)n || c.row_map[p] / c.map_div != t) return;
    quantize_row_wave<bf16_t, HELD>(x + (size_t)t * H, H, codes + (size_t)t * H, scales + t);
    return;
  }
  for (int p0 = (blockIdx.x * 4 + wave) * 64; p0 < n; p0 += FAR_BLOCKS * 256) {
    const int t = p0 + lane < n ? c.row_map[p0 + lane] / c.map_div : 0;
    for (uint64_t far = __ballot(t >= n_tokens); far; far &= far - 1) {
      const int l = __ffsll((long long)far) - 1;
      const size_t to = (size_t)n_tokens + p0 + l;
      quantize_row_wave<bf16_t, HELD>(x + (size_t)__builtin_amdgcn_readlane(t, l) * H, H, codes + to * H, scales + to);
    }
  }
}

// ---- the reference path: one wavefront per output element ------------------------------------
__device__ __forceinline__ int dot_16(const int4& a, const int4& b, int acc) {
  acc = __builtin_amdgcn_sdot4(a.x, b.x, acc, false);
  acc = __builtin_amdgcn_sdot4(a.y, b.y, acc, false);
  acc = __builtin_amdgcn_sdot4(a.z, b.z, acc, false);
  return __builtin_amdgcn_sdot4(a.w, b.w, acc, false);
}
__device__ __forceinline__ int wave_sum_int(int v) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off);
  return v;
}
__device__ __forceinline__ const char* i8_row_slot(const I8Ctx& c, int p) {
  if (p >= c.offsets[c.n_experts]) return nullptr;
  const int e = i8_expert_of(c.offsets, c.n_experts, p);
  const int s = c.slot_of[e];
  return c.active.test(e) && s >= 0 ? c.slots + (size_t)s * c.slot_bytes : nullptr;
}

__global__ __launch_bounds__(256) void ref_gateup_i8(I8Ctx c, const int8_t* __restrict__ x, const float* __restrict__ x_scales,
                                                     float* __restrict__ h) {
  const int p = blockIdx.x, wave = threadIdx.x / 64, lane = threadIdx.x % 64;
  const int f = blockIdx.y * 4 + wave;
  const char* slot = i8_row_slot(c, p);
  if (!slot || f >= c.ffn) return;
  const I8Offsets off = i8_offsets((size_t)c.hidden, (size_t)c.ffn);
  const int n_gate = 2 * TILE_N * (f / TILE_N) + f % TILE_N, n_up = n_gate + TILE_N;
  const int8_t* xr = x + (size_t)p * c.hidden;
  int g = 0, u = 0;
  for (int k = 16 * lane; k < c.hidden; k += 16 * 64) {
    const int4 xv = *(const int4*)(xr + k);
    g = dot_16(*(const int4*)(slot + i8_packed_index(n_gate, k, c.hidden)), xv, g);
    u = dot_16(*(const int4*)(slot + i8_packed_index(n_up, k, c.hidden)), xv, u);
  }
  g = wave_sum_int(g);
  u = wave_sum_int(u);
  if (lane == 0) {
    const float sx = x_scales[p];
    const float gf = i8_product(g, sx, ((const float*)(slot + off.gate_scales))[f]);
    const float uf = i8_product(u, sx, ((const float*)(slot + off.up_scales))[f]);
    h[(size_t)p * c.ffn + f] = gf / (1.0f + expf(-gf)) * uf;
  }
}

__global__ __launch_bounds__(256) void ref_down_i8(I8Ctx c, const int8_t* __restrict__ h, const float* __restrict__ h_scales,
                                                   bf16_t* __restrict__ o) {
  const int p = blockIdx.x, wave = threadIdx.x / 64, lane = threadIdx.x % 64;
  const int n = blockIdx.y * 4 + wave;
  const char* slot = i8_row_slot(c, p);
  if (!slot || n >= c.hidden) return;
  const I8Offsets off = i8_offsets((size_t)c.hidden, (size_t)c.ffn);
  const int8_t* hr = h + (size_t)p * c.ffn;
  int acc = 0;
  for (int k = 16 * lane; k < c.ffn; k += 16 * 64)
    acc = dot_16(*(const int4*)(slot + off.down + i8_packed_index(n, k, c.ffn)), *(const int4*)(hr + k), acc);
  acc = wave_sum_int(acc);
  if (lane == 0)
    o[(size_t)p * c.hidden + n] = f32_to_bf16_any(i8_product(acc, h_scales[p], ((const float*)(slot + off.down_scales))[n]));
}

static I8Ctx i8_ctx(const FfnArgs& a) {
  return I8Ctx{a.offsets, a.slot_of, a.slots, a.slot_bytes, a.active, a.all_active, a.desc->n_experts, a.desc->hidden, a.desc->ffn,
               a.row_map, a.map_div};
}
void launch_quantize_x_i8(const FfnArgs& a) {
  const I8Work w = i8_work(*a.desc, a.n_rows);
  launch_quantize(i8_ctx(a), a.n_rows, (const bf16_t*)a.x_perm, a.desc->hidden, (int8_t*)a.h + w.codes, (float*)((char*)a.h + w.scales),
                  a.stream);
}
void launch_quantize_h_i8(const FfnArgs& a) {
  const I8Work w = i8_work(*a.desc, a.n_rows);
  I8Ctx c = i8_ctx(a);
  c.row_map = nullptr;  // h is in sorted order
  launch_quantize(c, a.n_rows, (const float*)a.h, a.desc->ffn, (int8_t*)a.h + w.codes, (float*)((char*)a.h + w.scales), a.stream);
}

bool i8_shares_rows(const FfnArgs& a) {
  // (rows of more than 4096 values are quantised by whole blocks; a few MiB of codes are not worth a launch)
  return a.row_map && a.map_div > 1 && a.desc->hidden <= 4096 && (size_t)a.n_rows * a.desc->hidden >= (size_t)8 << 20;
}
void launch_quantize_shared_x_i8(const FfnArgs& a) {
  const I8Ctx c = i8_ctx(a);
  const I8Work w = i8_work(*a.desc, a.n_rows);
  int32_t* code_row = (int32_t*)((char*)a.h + w.code_row);
  int32_t* owner = (int32_t*)((char*)a.h + w.owner);
  const int T = (int)w.tokens, H = a.desc->hidden;
  hipLaunchKernelGGL(note_tokens_kernel, dim3((unsigned)((a.n_rows + 255l) / 256)), dim3(256), 0, a.stream, c, T, code_row, owner);
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)(FAR_BLOCKS + (T + 3l) / 4)), dim3(256), 0, a.stream, c, (const bf16_t*)a.x_perm, T, owner,
                       (int8_t*)a.h + w.codes, (float*)((char*)a.h + w.scales));
  };
  if (H <= 1024) launch(&quantize_tokens_kernel<2>);
  else if (H <= 2048) launch(&quantize_tokens_kernel<4>);
  else launch(&quantize_tokens_kernel<8>);
}

int launch_ffn_reference_i8(const FfnArgs& a) {
  const hmoe_layer_desc& d = *a.desc;
  if (a.n_rows == 0) return HMOE_OK;
  if ((d.ffn + 3) / 4 > 65535 || (d.hidden + 3) / 4 > 65535) return HMOE_ERR_UNSUPPORTED;
  const I8Ctx c = i8_ctx(a);
  const I8Work w = i8_work(d, a.n_rows);
  const int8_t* codes = (const int8_t*)a.h + w.codes;
  const float* scales = (const float*)((const char*)a.h + w.scales);
  launch_quantize_x_i8(a);
  probe_before(a.stream);
  hipLaunchKernelGGL(ref_gateup_i8, dim3((unsigned)a.n_rows, (unsigned)((d.ffn + 3) / 4)), dim3(256), 0, a.stream, c, codes, scales,
                     (float*)a.h);
  probe_after(a.stream);
  launch_quantize_h_i8(a);
  probe_before(a.stream);
  hipLaunchKernelGGL(ref_down_i8, dim3((unsigned)a.n_rows, (unsigned)((d.hidden + 3) / 4)), dim3(256), 0, a.stream, c, codes, scales,
                     (bf16_t*)a.o_perm);
  probe_after(a.stream);
  HMOE_HIP(hipGetLastError());
  return HMOE_OK;
}

}  // namespace hmoe
