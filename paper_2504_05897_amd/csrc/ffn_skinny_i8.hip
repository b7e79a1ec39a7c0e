// Decode FFN in 8-bit integers (HMOE_BF16_I8, HMOE_FFN_SKINNY): every touched expert's codes are streamed from HBM once,
// straight into MFMA operand registers.
//
// A block owns one packed 32-row group of the down projection, or the gate and the up group of 32 features, of one busy
// expert.  The matrix instruction is v_mfma_i32_16x16x64_i8: up to 16 rows of tokens x 16 weight rows x 64 k.  Codes are packed
// for the 32x32x32 instruction of the prefill tiles (1 KiB per 32 k: lane l has row l % 32, k 16 (l / 32) .. + 16); two
// consecutive tiles are 32 rows x 64 k, and which lane holds which 16 bytes of them is a matter of where it loads from: for
// the lower or upper 16 rows lane l takes row l % 16 and k block l / 16, so a load is four runs of 256 bytes and both loads
// together are 2 KiB on end.
//   * K is dealt to the NW waves in steps of 64, round-robin, so that the block sweeps one contiguous stretch; DEPTH steps are
//     in flight per wave.  Loads go through buffer descriptors: one lane offset, a scalar offset per load; a lane without a
//     token fetches nothing and gets zeros, which add nothing to integer sums.
//   * In small calls (in_blocks below) a block quantises the rows it needs itself, into LDS, while its first codes are on
//     their way: two launches instead of four, and the rows' maxima cost each block a trip to the L2 that holds them.
//   * The waves' sums meet in LDS; they are exact, so neither the split nor its order shows in the result.
#include <algorithm>

#include "i8_rows.h"

namespace hmoe {

struct SkinnyI8Ctx {
  const int32_t* offsets;
  const int32_t* slot_of;
  const char* slots;
  size_t slot_bytes;
  ActiveMask active;
  int n_experts, hidden, ffn;
  uint32_t in_bytes;       // of the codes of all rows
  int own_rows;            // rows per pass of a block that quantises them itself, up to SKINNY_I8_ROWS
  const int32_t* row_map;  // rows quantised in the gate/up launch: input row of sorted row p is row_map[p] / map_div
  int map_div;
};

// The `want`-th expert (ascending) that is active, resident and has rows: its cache slot and sorted rows [first, end), uniform
// over the wave; false if there are fewer.
__device__ __forceinline__ bool nth_busy_expert_i8(const SkinnyI8Ctx& c, int want, int lane, int& slot, int& first, int& end) {
  for (int base = 0; base < c.n_experts; base += 64) {
    const int e = base + lane, at = min(e, c.n_experts - 1);
    const int s = c.slot_of[at], b = c.offsets[at], n = c.offsets[at + 1];
    uint64_t m = __ballot(e < c.n_experts && c.active.test(at) && s >= 0 && n > b);
    const int busy = __popcll(m);
    if (want < busy) {
      for (int i = 0; i < want; ++i) m &= m - 1;
      const int l = __ffsll((long long)m) - 1;
      slot = __builtin_amdgcn_readlane(s, l);
      first = __builtin_amdgcn_readlane(b, l);
      end = __builtin_amdgcn_readlane(n, l);
      return true;
    }
    want -= busy;
  }
  return false;
}

constexpr int SKINNY_I8_ROWS = 8;       // rows per pass of a block that quantises them itself
constexpr int SKINNY_I8_ROW_PAD = 16;   // bytes between their codes in LDS

// GATEUP: codes of the tokens [A, H] -> h [A, F] fp32;  else: codes of h [A, F] -> o_perm [A, H] bfloat16.
// OWN: `in` holds the rows themselves, of bfloat16 tokens (through the row map) or fp32 h, and the block makes the codes.
// NW waves per block, XF fragments of 16 rows per pass.
template <bool GATEUP, int NW, int XF, int DEPTH, bool OWN>
__global__ __launch_bounds__(64 * NW) void ffn_skinny_i8_kernel(SkinnyI8Ctx c, const void* __restrict__ in,
                                                                 const float* __restrict__ row_scales, void* __restrict__ out) {
  static_assert(!OWN || XF == 1, "");
  extern __shared__ __attribute__((aligned(16))) int8_t own_codes[];  // [own_rows][K + pad]
  __shared__ float own_scales[SKINNY_I8_ROWS];
  __shared__ uint32_t own_max[NW];
  constexpr int NMAT = GATEUP ? 2 : 1;
  constexpr int NU = 2 * NMAT;  // 16-row units per block
  __shared__ i32x4_t red[(NW > 1 ? NW - 1 : 1) * NU * XF * 64];

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
  int cache_slot, row_first, row_end;
  if (!nth_busy_expert_i8(c, blockIdx.y, lane, cache_slot, row_first, row_end)) return;  // uniform over the block
  const int K = GATEUP ? c.hidden : c.ffn;      // reduction length
  const int n_out = GATEUP ? c.ffn : c.hidden;  // row length of `out`
  const int fb = blockIdx.x;                    // features [32 fb, 32 fb + 32) of `out`
  const int j = lane % 16, kblk = lane / 16;
  const char* slot = c.slots + (size_t)cache_slot * c.slot_bytes;
  const I8Offsets off = i8_offsets((size_t)c.hidden, (size_t)c.ffn);
  const size_t group_bytes = (size_t)TILE_N * K;
  const char* group = slot + (GATEUP ? 0 : off.down) + (size_t)NMAT * fb * group_bytes;
  __amdgpu_buffer_rsrc_t w_rsrc[NMAT];
#pragma unroll
  for (int m = 0; m < NMAT; ++m)
    w_rsrc[m] = __builtin_amdgcn_make_buffer_rsrc((void*)(group + m * group_bytes), 0, (int)group_bytes, 0x00027000);
  const __amdgpu_buffer_rsrc_t x_rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)in, 0, c.in_bytes, 0x00027000);
  const uint32_t w_lane = (uint32_t)(kblk / 2 * 1024 + (kblk % 2 * 32 + j) * 16);
  const int n_steps = K / 64, per_wave = (n_steps + NW - 1) / NW;  // steps per wave (the last ones may lie past the end)
  constexpr uint32_t NO_ROW = 0xF0000000u;

  const int PASS = OWN ? c.own_rows : 16 * XF;
  for (int row0 = row_first + (int)blockIdx.z * PASS; row0 < row_end; row0 += PASS * (int)gridDim.z) {
    const int rows = min(PASS, row_end - row0);
    uint32_t xin[XF];
#pragma unroll
    for (int x = 0; x < XF; ++x)
      xin[x] = 16 * x + j < rows ? (uint32_t)(row0 + 16 * x + j) * (uint32_t)K + 16 * kblk : NO_ROW;

    u32x4 w[DEPTH][NU], xa[DEPTH][XF];
    // (rows past the last repeat one in LDS: what a row of tokens holds shows in its own results only)
    const int8_t* own_row = own_codes + min(j, rows - 1) * (K + SKINNY_I8_ROW_PAD) + 16 * kblk;
    auto load_tokens = [&](int ring, int i) {
      const int want = i * NW + wave, step = min(want, n_steps - 1);
      if constexpr (OWN) {
        const u32x4 v = *(const u32x4*)(own_row + step * 64);
        xa[ring][0] = want < n_steps ? v : u32x4{0, 0, 0, 0};
      } else {
#pragma unroll
        for (int x = 0; x < XF; ++x)
          xa[ring][x] = __builtin_amdgcn_raw_buffer_load_b128(x_rsrc, want < n_steps ? xin[x] : NO_ROW, step * 64, 0);
      }
    };
    auto load_step = [&](int ring, int i) {
      // A step past the end of K is the last one again with nothing for tokens.  (A descriptor checks the lane's offset against
      // its end, not the scalar one.)
      const int step = min(i * NW + wave, n_steps - 1);
#pragma unroll
      for (int u = 0; u < NU; ++u)
        w[ring][u] = __builtin_amdgcn_raw_buffer_load_b128(w_rsrc[u / 2], w_lane + u % 2 * 256, step * 2048, 2);
    };
    i32x4_t acc[NU][XF];
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
      for (int x = 0; x < XF; ++x) acc[u][x] = i32x4_t{0, 0, 0, 0};
    // (the scheduling barriers keep the loads where they are written, and with them the lookahead)
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) load_step(d, d);
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (OWN) {
      for (int r = 0; r < rows; ++r) {
        if constexpr (GATEUP)
          own_row_codes<NW, 2>((const bf16_t*)in + (size_t)mapped_row(c.row_map, c.map_div, row0 + r) * K, K,
                               own_codes + r * (K + SKINNY_I8_ROW_PAD), &own_scales[r], own_max);
        else
          own_row_codes<NW, 4>((const float*)in + (size_t)(row0 + r) * K, K, own_codes + r * (K + SKINNY_I8_ROW_PAD), &own_scales[r], own_max);
      }
      __syncthreads();
    }
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) load_tokens(d, d);
    __builtin_amdgcn_sched_barrier(0);
    for (int i = 0; i < per_wave; i += DEPTH) {
#pragma unroll
      for (int d = 0; d < DEPTH; ++d) {
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
          for (int x = 0; x < XF; ++x) acc[u][x] = mfma_16x16x64_i8(xa[d][x], w[d][u], acc[u][x]);
        __builtin_amdgcn_sched_barrier(0);
        load_step(d, i + d + DEPTH);
        load_tokens(d, i + d + DEPTH);
        __builtin_amdgcn_sched_barrier(0);
      }
    }

    // accumulator register r of lane (j, kblk) is row 4 kblk + r of its fragment, weight row j of its unit
    if (NW > 1 && wave > 0) {
#pragma unroll
      for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int x = 0; x < XF; ++x) red[((wave - 1) * NU * XF + u * XF + x) * 64 + lane] = acc[u][x];
    }
    if (NW > 1) __syncthreads();
    if (wave == 0) {
#pragma unroll 1
      for (int v = 0; v < NW - 1; ++v)
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
          for (int x = 0; x < XF; ++x) acc[u][x] += red[(v * NU * XF + u * XF + x) * 64 + lane];
      const float* scales = (const float*)(slot + (GATEUP ? off.gate_scales : off.down_scales)) + 32 * fb + j;
#pragma unroll
      for (int x = 0; x < XF; ++x)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int m = 16 * x + 4 * kblk + r;
          if (m >= rows) continue;
          const float rs = OWN ? own_scales[m % SKINNY_I8_ROWS] : row_scales[row0 + m];
          const size_t at = (size_t)(row0 + m) * n_out + 32 * fb + j;
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            if (GATEUP) {
              const float g = i8_product(acc[s][x][r], rs, scales[16 * s]);
              const float u = i8_product(acc[2 % NU + s][x][r], rs, scales[c.ffn + 16 * s]);
              ((float*)out)[at + 16 * s] = silu_f32(g) * u;
            } else {
              ((bf16_t*)out)[at + 16 * s] = f32_to_bf16(i8_product(acc[s][x][r], rs, scales[16 * s]));
            }
          }
        }
    }
    __syncthreads();  // the reduction area and the codes in LDS are reused by the next row pass
  }
}

// Waves per block: about 16 steps of K each, 2 to 8 of them (launches, us, 2 / 4 / 8 waves: gate/up over 32 steps, 35 experts,
// 37.8 / 37.0 / 38.9, over 64 steps, 2 experts, 40.5 / 39.7 / 41.2; down over 22 steps 21.7 / 22.5 / 27.4, over 224 steps, 2
// experts, 38.6 / 25.7 / 22.4).
template <bool GATEUP, int XF, bool OWN>
static void launch_stage_i8(const SkinnyI8Ctx& c, int busy_max, int max_rows, const void* in, const float* row_scales, void* out,
                            hipStream_t s) {
  // (an expert's passes side by side, so that one with many rows does not take as many times as long)
  const unsigned passes = OWN ? 1 : (unsigned)std::min(8, (max_rows + 16 * XF - 1) / (16 * XF));
  const dim3 grid((unsigned)((GATEUP ? c.ffn : c.hidden) / TILE_N), (unsigned)busy_max, passes);
  const int K = GATEUP ? c.hidden : c.ffn, n_steps = K / 64;
  const size_t lds = OWN ? (size_t)c.own_rows * (K + SKINNY_I8_ROW_PAD) : 0;
  auto launch = [&](auto kernel, int nw) { hipLaunchKernelGGL(kernel, grid, dim3(64 * nw), lds, s, c, in, row_scales, out); };
  if (n_steps < 48) launch(&ffn_skinny_i8_kernel<GATEUP, 2, XF, 4, OWN>, 2);
  else if (n_steps < 112) launch(&ffn_skinny_i8_kernel<GATEUP, 4, XF, 4, OWN>, 4);
  else launch(&ffn_skinny_i8_kernel<GATEUP, 8, XF, 2, OWN>, 8);
}

// What HMOE_FFN_AUTO chooses (calls, us, these kernels / the prefill tiles): up to 16 tokens (64 experts of 3584 x 2560, top 8, 16 tokens
// 246 / 256, 32 tokens 288 / 277; 8 of 4096 x 14336, top 2, 20 tokens 226 / 226; 64 of 2048 x 1408, top 6, 20 tokens 93 / 88; one of 3584 x
// 20480, 16 tokens 65 / 75, 32 tokens 82 / 77).  Small layers, whose calls are a few launches' latency, up to 256 tokens while that is no
// more than a few rounds of blocks (16 of 1024 x 640, top 2, 77 / 200 tokens 19.6 / 22.2, 23.8 / 22.9, with skewed routing 21.3 / 22.0, 27.3 /
// 34.3; one of 2048 x 2816, 48 / 256 tokens 24 / 30, 38 / 49; one of 2048 x 8192, 64 / 128 tokens 39 / 43, 48 / 54; but 71 of 2304 x 128, top 3, 229
// tokens, 40896 blocks, 48 / 44; 85 of 128 x 1792, top 7, 24 tokens, 4760 blocks, 26 / 23, 187 tokens, 28560 blocks, 75 / 37), whose
// passes of 32 rows do not read the weights too often (one of 4096 x 5120, 64 / 200 tokens 43 / 48, 98 / 82).
bool ffn_skinny_i8_takes(const hmoe_layer_desc& d, int n_rows) {
  const int T = n_rows / d.top_k;
  if (T <= 16) return true;
  const long passes = (T + 31) / 32, bytes = 3l * d.hidden * d.ffn * d.n_experts;
  if (T > 256 || bytes > (64l << 20) || bytes * passes > (256l << 20)) return false;
  return (long)(std::max(d.hidden, d.ffn) / TILE_N) * std::min(d.n_experts, n_rows) * passes <= 4096;
}

int launch_ffn_skinny_i8(const FfnArgs& a) {
  const hmoe_layer_desc& d = *a.desc;
  if (d.dtype != HMOE_BF16_I8) return HMOE_ERR_UNSUPPORTED;
  if (a.n_rows == 0) return HMOE_OK;
  // offsets of 32 bits, and a margin in which lanes without a token stay past the end at every step
  const size_t x_bytes = (size_t)a.n_rows * d.hidden, h_bytes = (size_t)a.n_rows * d.ffn;
  if (std::max(x_bytes, h_bytes) > 0xE0000000u) return launch_ffn_tiled_i8(a);
  SkinnyI8Ctx c{a.offsets, a.slot_of, a.slots, a.slot_bytes, a.active, d.n_experts, d.hidden, d.ffn, (uint32_t)x_bytes, 0, a.row_map, a.map_div};
  const int busy_max = std::min(d.n_experts, a.n_rows);          // every busy expert has at least one row
  const int max_rows = std::max(1, a.n_rows / d.top_k);          // a token names an expert at most once
  const I8Work w = i8_work(d, a.n_rows);
  const int8_t* codes = (const int8_t*)a.h + w.codes;
  const float* scales = (const float*)((const char*)a.h + w.scales);
  // Rows quantised by the blocks that read them (max_rows of them per pass, in LDS) or by a launch of its own.  The launch
  // costs 3 to 4 us; in a block it costs time per row, and that again in every round of blocks.  Calls, own launches / in the
  // blocks, us: 64 experts of 2048 x 1408, top 6, 1 / 4 / 8 tokens 19.0 / 16.5, 39.6 / 35.6, 61.0 / 58.7; 16 of 4096 x 1024, top 2, 8 tokens
  // 32.2 / 27.7; 8 of 4096 x 14336, top 2, 2 tokens (28672 values of h per pass) 115.0 / 112.4, 4 tokens (57344) 143.8 / 146.2, 8 tokens
  // (3584 blocks in gate/up) 198.4 / 206.2; 64 of 3584 x 2560, top 8, 8 tokens (5120 blocks) 198.1 / 199.4.  Those have one or two rows per
  // expert; one expert of 2048 x 2816, 8 tokens and rows 21 / 33.
  auto in_blocks = [&](int K, int n_out) {
    return max_rows <= SKINNY_I8_ROWS && a.n_rows <= 2 * d.n_experts && max_rows * K <= 32768 && (long)(n_out / TILE_N) * busy_max <= 3000;
  };
  const bool own_x = in_blocks(d.hidden, d.ffn), own_h = in_blocks(d.ffn, d.hidden);
  const bool two = max_rows > 16;
  c.own_rows = max_rows;
  if (!own_x) launch_quantize_x_i8(a);
  probe_before(a.stream);
  if (own_x) launch_stage_i8<true, 1, true>(c, busy_max, max_rows, a.x_perm, nullptr, a.h, a.stream);
  else (two ? launch_stage_i8<true, 2, false> : launch_stage_i8<true, 1, false>)(c, busy_max, max_rows, codes, scales, a.h, a.stream);
  probe_after(a.stream);
  if (!own_h) launch_quantize_h_i8(a);
  c.in_bytes = (uint32_t)h_bytes;
  probe_before(a.stream);
  if (own_h) launch_stage_i8<false, 1, true>(c, busy_max, max_rows, a.h, nullptr, a.o_perm, a.stream);
  else (two ? launch_stage_i8<false, 2, false> : launch_stage_i8<false, 1, false>)(c, busy_max, max_rows, codes, scales, a.o_perm, a.stream);
  probe_after(a.stream);
  HMOE_HIP(hipGetLastError());
  return HMOE_OK;
}

}  // namespace hmoe
