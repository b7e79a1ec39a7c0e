// Prefill FFN in 8-bit integers (HMOE_BF16_I8, HMOE_FFN_TILED): the tiles of stream_tile.h on the 32x32x32 int8 matrix
// instruction, between the launches that quantise the tokens' rows and the rows of h (ffn_i8.hip).
//
// A fragment of codes is 16 bytes per lane like one of bfloat16 and holds twice the k, so a tile does twice the products per
// byte that moves and per matrix instruction.  Sums are integers; the epilogue multiplies them by the scale of the row (from
// the quantiser) and of the column (from the slot) and goes on in fp32: SwiGLU into h, or bfloat16 into o_perm.
#include <stdlib.h>

#include <algorithm>

#include "stream_tile.h"

namespace hmoe {

template <class TILE, class OUT>
__device__ __forceinline__ void run_tile_i8(const TiledCtx& c, const bf16_t* __restrict__ in, const float* __restrict__ row_scales,
                                            OUT* __restrict__ out, const TileLoc& loc, u32x4* lds) {
  typename TILE::Acc acc;
#pragma unroll
  for (int i = 0; i < TILE::FM; ++i)
#pragma unroll
    for (int j = 0; j < TILE::FN; ++j) acc[i][j] = i32x16_t{0};
  TILE::mainloop(c, in, loc, 0, TILE::k_units(c) / TILE::BKT, lds, acc);
  // scales of the lane's column in each of the wave's groups (of group 0 for groups past N: never stored)
  const int wave = threadIdx.x / 64, col = threadIdx.x % 32;
  const char* slot = c.slots + (size_t)loc.slot * c.slot_bytes;
  const I8Offsets off = i8_offsets((size_t)c.hidden, (size_t)c.ffn);
  const int n_groups = (TILE::GATEUP ? 2 * c.ffn : c.hidden) / TILE_N;
  float col_scales[TILE::FN];
#pragma unroll
  for (int j = 0; j < TILE::FN; ++j) {
    int g = loc.nt * (TILE::BN / TILE_N) + wave * TILE::FN + j;
    if (g >= n_groups) g = 0;
    const float* scales = (const float*)(slot + (!TILE::GATEUP ? off.down_scales : g % 2 ? off.up_scales : off.gate_scales));
    col_scales[j] = scales[(TILE::GATEUP ? g / 2 : g) * TILE_N + col];
  }
  typename TILE::Sums sums;
  TILE::scale_sums(loc, row_scales, col_scales, acc, lds, sums);
  if constexpr (TILE::GATEUP && TILE::FN == 2) TILE::epilogue_h_f32(c, out, loc, sums);
  else if constexpr (TILE::GATEUP) TILE::epilogue_pairs(c, out, loc, sums, lds);
  else if constexpr (TILE::FN == 2) TILE::epilogue_lines_down(c, out, loc, sums, lds);
  else TILE::epilogue_lines_block(c, out, loc, sums, lds);
}

template <bool GATEUP, int BM, int NWV, bool NT, int RING, int FM, int FN>
using TileI8 = StreamTile<GATEUP, BM, NWV, 4, NT, RING, FM, FN, false, false, StreamI8>;

// Tiles of up to 128 rows, two weight groups per wave (see ffn_tile_fit_kernel).
template <bool GATEUP, int NWV, bool NT, class OUT>
__global__ __launch_bounds__(64 * NWV, 2) void ffn_tile_i8_kernel(TiledCtx c, const bf16_t* __restrict__ in,
                                                                const float* __restrict__ row_scales, OUT* __restrict__ out) {
  constexpr int RING = NWV == 4 ? 4 : 8;
  typedef TileI8<GATEUP, 128, NWV, NT, RING, 4, 2> FULL;
  __shared__ u32x4 lds[FULL::LDS_VEC];
  TileLoc loc;
  if (!locate_tile<128>(c, loc)) return;  // uniform over the block
  const int tiles = (loc.m_rows + 127) / 128;
  const int fragments = ((loc.m_rows + tiles - 1) / tiles + 31) / 32;  // per m-tile, 1..4; uniform
  if (fragments == 4) run_tile_i8<FULL>(c, in, row_scales, out, loc, lds);
  else if (fragments == 3) run_tile_i8<TileI8<GATEUP, 128, NWV, NT, RING, 3, 2>>(c, in, row_scales, out, loc, lds);
  else if (fragments == 2) run_tile_i8<TileI8<GATEUP, 128, NWV, NT, RING, 2, 2>>(c, in, row_scales, out, loc, lds);
  else run_tile_i8<TileI8<GATEUP, 128, NWV, NT, RING, 1, 2>>(c, in, row_scales, out, loc, lds);
}

// Tiles of up to 256 rows, one weight group per wave (see ffn_tile_fit256_kernel).
template <bool GATEUP, int NWV, bool NT, class OUT>
__global__ __launch_bounds__(64 * NWV) void ffn_tile256_i8_kernel(TiledCtx c, const bf16_t* __restrict__ in,
                                                                   const float* __restrict__ row_scales, OUT* __restrict__ out) {
  typedef TileI8<GATEUP, 256, NWV, NT, 8, 8, 1> FULL;
  __shared__ u32x4 lds[FULL::LDS_VEC];
  TileLoc loc;
  if (!locate_tile<256>(c, loc)) return;  // uniform over the block
  const int tiles = (loc.m_rows + 255) / 256;
  const int fragments = ((loc.m_rows + tiles - 1) / tiles + 31) / 32;  // per m-tile, 1..8; uniform
  if (fragments > 6) run_tile_i8<FULL>(c, in, row_scales, out, loc, lds);
  else if (fragments > 4) run_tile_i8<TileI8<GATEUP, 256, NWV, NT, 8, 6, 1>>(c, in, row_scales, out, loc, lds);
  else if (fragments > 2) run_tile_i8<TileI8<GATEUP, 256, NWV, NT, 8, 4, 1>>(c, in, row_scales, out, loc, lds);
  else run_tile_i8<TileI8<GATEUP, 256, NWV, NT, 8, 2, 1>>(c, in, row_scales, out, loc, lds);
}

enum { I8_FIT = 0, I8_FIT_PLAIN = 1, I8_FIT4 = 2, I8_FIT4_PLAIN = 3, I8_FIT256 = 4, I8_FIT256_PLAIN = 5 };

template <bool GATEUP, class OUT>
static void launch_stage_i8(TiledCtx c, int variant, int n_rows, const bf16_t* in, const float* row_scales, OUT* out, hipStream_t s) {
  const int n_total = GATEUP ? 2 * c.ffn : c.hidden;
  auto launch = [&](auto kernel, int bm, int bn, int threads) {
    c.n_tiles_n = (n_total + bn - 1) / bn;
    c.grid_padded = (int)((tiles_upper_bound(c, n_rows, bm) + 7) / 8 * 8);
    hipLaunchKernelGGL(kernel, dim3((unsigned)c.grid_padded), dim3(threads), 0, s, c, in, row_scales, out);
  };
  constexpr int NW256 = GATEUP ? 8 : 4;
  switch (variant) {
    case I8_FIT: launch(&ffn_tile_i8_kernel<GATEUP, 8, true, OUT>, 128, 512, 512); break;
    case I8_FIT_PLAIN: launch(&ffn_tile_i8_kernel<GATEUP, 8, false, OUT>, 128, 512, 512); break;
    case I8_FIT4: launch(&ffn_tile_i8_kernel<GATEUP, 4, true, OUT>, 128, 256, 256); break;
    case I8_FIT4_PLAIN: launch(&ffn_tile_i8_kernel<GATEUP, 4, false, OUT>, 128, 256, 256); break;
    case I8_FIT256: launch(&ffn_tile256_i8_kernel<GATEUP, NW256, true, OUT>, 256, 32 * NW256, 64 * NW256); break;
    default: launch(&ffn_tile256_i8_kernel<GATEUP, NW256, false, OUT>, 256, 32 * NW256, 64 * NW256); break;
  }
}

int launch_ffn_tiled_i8(const FfnArgs& a) {
  const hmoe_layer_desc& d = *a.desc;
  if (d.dtype != HMOE_BF16_I8) return HMOE_ERR_UNSUPPORTED;
  if (a.n_rows == 0) return HMOE_OK;
  TiledCtx c{a.offsets, a.slot_of, a.slots, a.slot_bytes, a.active, d.n_experts, d.hidden, d.ffn, 0, 0, nullptr, 1};
  const I8Work w = i8_work((size_t)a.n_rows, (size_t)d.hidden, (size_t)d.ffn);
  const bf16_t* codes = (const bf16_t*)((const char*)a.h + w.codes);
  const float* scales = (const float*)((const char*)a.h + w.scales);
  int v_gate_up = I8_FIT, v_down = I8_FIT;
  if (a.n_rows / d.n_experts >= 192) v_gate_up = v_down = I8_FIT4_PLAIN;
  if (const char* env = getenv("HMOE_I8_VARIANT")) {  // tuning: "<gate/up><down>"
    if (env[0] >= '0' && env[0] <= '5') v_gate_up = env[0] - '0';
    if (env[0] && env[1] >= '0' && env[1] <= '5') v_down = env[1] - '0';
  }
  launch_quantize_x_i8(a);
  probe_before(a.stream);
  launch_stage_i8<true>(c, v_gate_up, a.n_rows, codes, scales, (float*)a.h, a.stream);
  probe_after(a.stream);
  launch_quantize_h_i8(a);
  probe_before(a.stream);
  launch_stage_i8<false>(c, v_down, a.n_rows, codes, scales, (bf16_t*)a.o_perm, a.stream);
  probe_after(a.stream);
  HMOE_HIP(hipGetLastError());
  return HMOE_OK;
}

}  // namespace hmoe
