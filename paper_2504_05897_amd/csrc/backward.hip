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

__device__ __forceinline__ float to_f32(bf16_t v) { return bf16_to_f32(v); }
__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ void from_f32(bf16_t& o, float v) { o = f32_to_bf16_any(v); }
__device__ __forceinline__ void from_f32(float& o, float v) { o = v; }

// d_o_perm[p] = w dy[t], d_topk_w = dy[t] . o_perm[p]: one wavefront per assignment.  d_o_perm may be o_perm: a lane reads
// its elements before it writes them.
template <class T>
__global__ __launch_bounds__(256) void combine_backward_kernel(const T* dy, const T* o_perm, const int32_t* inv_perm, const float* topk_w,
                                                               int n_assign, int top_k, int hidden, T* d_o_perm, float* d_topk_w) {
  const int a = blockIdx.x * 4 + threadIdx.x / 64, lane = threadIdx.x % 64;
  if (a >= n_assign) return;
  const int p = inv_perm[a];
  const bool has_row = (unsigned)p < (unsigned)n_assign;
  float dot = 0.0f;
  if (has_row) {
    const T* g = dy + (size_t)(a / top_k) * hidden;
    const float w = d_o_perm ? topk_w[a] : 0.0f;
    for (int c = lane; c < hidden; c += 64) {
      const float v = to_f32(g[c]);
      if (d_topk_w) dot += v * to_f32(o_perm[(size_t)p * hidden + c]);
      if (d_o_perm) from_f32(d_o_perm[(size_t)p * hidden + c], w * v);
    }
  }
  if (!d_topk_w) return;
  dot = sum_over_wave(dot);
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
      const int named = __shfl(id, j, G);
      const float part = __shfl(own, j, G);
      if (named == e) v += part;
    }
    if (e < n_experts) d_logits[(size_t)t * n_experts + e] = v;
  }
}

// dx[t] = sum_e d_logits[t, e] w_g[e] (+ add[t]): one thread per element
template <class T>
__global__ __launch_bounds__(256) void router_dx_kernel(const T* __restrict__ w_g, const float* __restrict__ d_logits, const T* add,
                                                        int n_experts, int hidden, T* dx) {
  const size_t t = blockIdx.x;
  const int c = blockIdx.y * 256 + threadIdx.x;
  if (c >= hidden) return;
  float acc = 0.0f;
  for (int e = 0; e < n_experts; ++e) acc = fmaf(d_logits[t * n_experts + e], to_f32(w_g[(size_t)e * hidden + c]), acc);
  if (add) acc += to_f32(add[t * hidden + c]);
  from_f32(dx[t * hidden + c], acc);
}

// d_w_g[e] = sum_t d_logits[t, e] x[t]: one thread per element
template <class T>
__global__ __launch_bounds__(256) void router_dw_kernel(const T* __restrict__ x, const float* __restrict__ d_logits, int n_tokens,
                                                        int n_experts, int hidden, float* __restrict__ d_w_g) {
  const int e = blockIdx.y, c = blockIdx.x * 256 + threadIdx.x;
  if (c >= hidden) return;
  float acc = 0.0f;
  for (int t = 0; t < n_tokens; ++t) acc = fmaf(d_logits[(size_t)t * n_experts + e], to_f32(x[(size_t)t * hidden + c]), acc);
  d_w_g[(size_t)e * hidden + c] = acc;
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
  const dim3 grid((unsigned)(((long)n_assign + 3) / 4));
  hipStream_t s = (hipStream_t)stream;
  if (desc->dtype == HMOE_F32)
    hipLaunchKernelGGL(combine_backward_kernel<float>, grid, dim3(256), 0, s, (const float*)dy, (const float*)o_perm, inv_perm, topk_w, n_assign,
                       desc->top_k, H, (float*)d_o_perm, d_topk_w);
  else
    hipLaunchKernelGGL(combine_backward_kernel<bf16_t>, grid, dim3(256), 0, s, (const bf16_t*)dy, (const bf16_t*)o_perm, inv_perm, topk_w,
                       n_assign, desc->top_k, H, (bf16_t*)d_o_perm, d_topk_w);
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
  return 256;
}

extern "C" int32_t hmoe_router_backward(const hmoe_layer_desc* desc, const void* x, const void* w_g, const float* d_logits, int32_t T,
                                        const void* add, void* dx, float* d_w_g, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check_desc(desc);
  if (rc != HMOE_OK) return rc;
  const int E = desc->n_experts, H = desc->hidden;
  if (T < 0) return HMOE_ERR_INVALID_ARG;
  if (!dx && !d_w_g) return HMOE_ERR_INVALID_ARG;
  if (T > 0 && (!d_logits || (dx && !w_g) || (d_w_g && !x))) return HMOE_ERR_INVALID_ARG;
  if (!aligned16(d_logits) || (dx && (!aligned16(dx) || !aligned16(w_g) || !aligned16(add))) || (d_w_g && (!aligned16(d_w_g) || !aligned16(x))))
    return HMOE_ERR_INVALID_ARG;
  if (desc->dtype != HMOE_F32 && H % 16 != 0) return HMOE_ERR_UNSUPPORTED;
  if (!workspace || workspace_bytes < hmoe_router_backward_workspace_bytes(desc, T)) return HMOE_ERR_WORKSPACE;
  if (!aligned16(workspace)) return HMOE_ERR_INVALID_ARG;
  hipStream_t s = (hipStream_t)stream;
  const unsigned columns = (unsigned)((H + 255) / 256);
  if (dx && T > 0) {
    const dim3 grid((unsigned)T, columns);
    if (desc->dtype == HMOE_F32)
      hipLaunchKernelGGL(router_dx_kernel<float>, grid, dim3(256), 0, s, (const float*)w_g, d_logits, (const float*)add, E, H, (float*)dx);
    else
      hipLaunchKernelGGL(router_dx_kernel<bf16_t>, grid, dim3(256), 0, s, (const bf16_t*)w_g, d_logits, (const bf16_t*)add, E, H, (bf16_t*)dx);
  }
  if (d_w_g) {
    const dim3 grid(columns, (unsigned)E);
    if (desc->dtype == HMOE_F32)
      hipLaunchKernelGGL(router_dw_kernel<float>, grid, dim3(256), 0, s, (const float*)x, d_logits, T, E, H, d_w_g);
    else
      hipLaunchKernelGGL(router_dw_kernel<bf16_t>, grid, dim3(256), 0, s, (const bf16_t*)x, d_logits, T, E, H, d_w_g);
  }
  HMOE_HIP(hipGetLastError());
  return HMOE_OK;
}
