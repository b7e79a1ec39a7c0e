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

template <class TILE>
__device__ __forceinline__ void clear_sums(typename TILE::Acc& acc) {
#pragma unroll
  for (int i = 0; i < TILE::FM; ++i)
#pragma unroll
    for (int j = 0; j < TILE::FN; ++j) acc[i][j] = i32x16_t{0};
}

// The tile's integer sums times their scales, to `out` as h or o_perm.
template <class TILE, class OUT>
__device__ __forceinline__ void finish_tile_i8(const TiledCtx& c, const float* __restrict__ row_scales, OUT* __restrict__ out, const TileLoc& loc,
                                               const typename TILE::Acc& acc, u32x4* lds) {
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
  TILE::scale_sums(c, loc, row_scales, col_scales, acc, lds, sums);
  if constexpr (TILE::GATEUP && TILE::FN == 2) TILE::epilogue_h_f32(c, out, loc, sums);
  else if constexpr (TILE::GATEUP) TILE::epilogue_pairs(c, out, loc, sums, lds);
  else if constexpr (TILE::FN == 2) TILE::epilogue_lines_down(c, out, loc, sums, lds);
  else TILE::epilogue_lines_block(c, out, loc, sums, lds);
}

template <class TILE, class OUT>
__device__ __forceinline__ void run_tile_i8(const TiledCtx& c, const bf16_t* __restrict__ in, const float* __restrict__ row_scales,
                                            OUT* __restrict__ out, const TileLoc& loc, u32x4* lds) {
  typename TILE::Acc acc;
  clear_sums<TILE>(acc);
  TILE::mainloop(c, in, loc, 0, TILE::k_units(c) / TILE::BKT, lds, acc);
  finish_tile_i8<TILE>(c, row_scales, out, loc, acc, lds);
}

template <bool GATEUP, int BM, int NWV, bool NT, int RING, int FM, int FN>
using TileI8 = StreamTile<GATEUP, BM, NWV, 4, NT, RING, FM, FN, false, false, StreamI8>;

// Tiles of up to 128 rows, two weight groups per wave (see ffn_tile_fit_kernel).
template <bool GATEUP, int NWV, bool NT, class OUT>
__global__ __launch_bounds__(64 * NWV, 2) void ffn_tile_i8_kernel(TiledCtx c, const bf16_t* __restrict__ in,
                                                                const float* __restrict__ row_scales, OUT* __restrict__ out) {
  constexpr int RING = 4;
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

// Down launches with a long K and a tile or less per CU: tiles of up to 160 rows x 128 columns, by two sets of four waves that take
// half of K each (with one set, a SIMD has one wave, and nothing hides what that waits for).  The second set hands its sums to the
// first, exact as they are, and ends.
template <bool NT, int FM>
using SplitI8 = StreamTile<false, 160, 4, 3, NT, 8, FM, 1, false, false, StreamI8>;
constexpr int SPLIT_LDS = 2 * SplitI8<false, 5>::LDS_VEC;

template <class TILE>
__device__ __forceinline__ void run_split_i8(const TiledCtx& c, const bf16_t* __restrict__ in, const float* __restrict__ row_scales,
                                             bf16_t* __restrict__ out, const TileLoc& loc, u32x4* lds) {
  static_assert(TILE::FM * 16 * 256 <= SPLIT_LDS * 4 && TILE::FN == 1, "the sums must fit");
  const int set = __builtin_amdgcn_readfirstlane(threadIdx.x / 256), tid = threadIdx.x % 256;
  const int half = TILE::k_units(c) / TILE::BKT / 2;
  typename TILE::Acc acc;
  clear_sums<TILE>(acc);
  TILE::mainloop_of_set(c, in, loc, set * half, half, lds + set * TILE::LDS_VEC, acc, tid);
  i32x4_t* sums = (i32x4_t*)lds + tid;
  __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
  block_barrier();  // every wave has read its last activation fragments
  if (set == 1) {
#pragma unroll
    for (int i = 0; i < TILE::FM * 4; ++i)
      sums[i * 256] = i32x4_t{acc[i / 4][0][i % 4 * 4], acc[i / 4][0][i % 4 * 4 + 1], acc[i / 4][0][i % 4 * 4 + 2], acc[i / 4][0][i % 4 * 4 + 3]};
  }
  __syncthreads();
  if (set == 1) return;
#pragma unroll
  for (int i = 0; i < TILE::FM * 4; ++i) {
    const i32x4_t v = sums[i * 256];
#pragma unroll
    for (int t = 0; t < 4; ++t) acc[i / 4][0][i % 4 * 4 + t] += v[t];
  }
  __builtin_amdgcn_s_waitcnt(0xC07F);  // before the barrier after which others write over the sums
  finish_tile_i8<TILE>(c, row_scales, out, loc, acc, lds);
}

template <bool NT>
__global__ __launch_bounds__(512) void ffn_tile_split_i8_kernel(TiledCtx c, const bf16_t* __restrict__ in, const float* __restrict__ row_scales,
                                                                bf16_t* __restrict__ out) {
  __shared__ u32x4 lds[SPLIT_LDS];
  TileLoc loc;
  if (!locate_tile<160>(c, loc)) return;  // uniform over the block
  const int tiles = (loc.m_rows + 159) / 160;
  const int fragments = ((loc.m_rows + tiles - 1) / tiles + 31) / 32;  // per m-tile, 1..5; uniform
  if (fragments == 5) run_split_i8<SplitI8<NT, 5>>(c, in, row_scales, out, loc, lds);
  else if (fragments == 4) run_split_i8<SplitI8<NT, 4>>(c, in, row_scales, out, loc, lds);
  else if (fragments == 3) run_split_i8<SplitI8<NT, 3>>(c, in, row_scales, out, loc, lds);
  else run_split_i8<SplitI8<NT, 2>>(c, in, row_scales, out, loc, lds);
}

// The 224x256 tile in blocks that work through several tiles, one wave per SIMD (see ffn_tile_walk_kernel).  A tile's last
// two K steps issue the first loads of the block's next tile, which an int8 tile, with half as many K steps, gains more from.
// The scales of a tile's rows and columns travel to LDS with two copies issued by hand at its start; the waits of its K steps,
// which are more than any of them leaves in flight, see them through.
constexpr int WALK_ROWS = 8;  // per thread in LDS: the input rows of its seven copies, and the row whose scale it copies
template <bool GATEUP, int FM, bool NT>
using WalkI8 = StreamTile<GATEUP, 224, 4, 3, NT, 8, FM, 2, true, true, StreamI8>;

struct WalkI8Lds {
  u32x4 ring[WalkI8<true, 7, false>::LDS_VEC];
  u32x4 staging[4 * 64 * 8];
  float row_scales[2][256], col_scales[2][256];  // of the tile at hand and the next
  int table[TileWalk<4>::TABLE_INTS];
  int rows[WALK_ROWS * 256];
};

// the sorted row whose scale this thread copies: that of row `tid` of the tile
__device__ __forceinline__ int walk_scale_row(const TiledCtx& c, const TileLoc& loc, int tid) {
  return loc.row_first + min(loc.m0 + tid, loc.m_rows - 1);
}

// One tile of fm == FM fragments whose first K step lies in half START of the weight ring.  In: loc, ring and stage describe the
// tile, whose first loads have landed; w.rows (gate/up) its input rows.  Out: the same for the block's next tile.
template <bool GATEUP, bool NT, bool ODD, int START, int FM, class OUT>
__device__ __forceinline__ void walk_one_tile_i8(const TiledCtx& c, const bf16_t* __restrict__ in, const float* __restrict__ row_scales,
                                                 OUT* __restrict__ out, const TileWalk<4>& walk, int xcd, int stride, int wave, int lane,
                                                 int k_steps, WalkI8Lds& w, uint32_t lds0, TileLoc& loc, int& idx, int& fm, bool& more,
                                                 int& stage, int& turn, u32x4 (&ring)[8][2]) {
  typedef WalkI8<GATEUP, FM, NT> TILE;
  typedef WalkI8<GATEUP, 7, NT> FULL;
  const TileLoc done = loc;
  idx += stride;
  more = walk.at(xcd, idx, loc);  // leaves loc as it is when there is no further tile
  fm = loc.fm;
  int lane_rows = lane;  // (opaque copies of the lane id: what is derived from it is recomputed where it is used)
  asm volatile("" : "+v"(lane_rows));
  const int tid_rows = wave * 64 + lane_rows;
  int* const rows_lds = w.rows + tid_rows;
  int rows[7], rows_next[7], scale_row, scale_row_next = 0;
  if constexpr (GATEUP) {
#pragma unroll
    for (int i = 0; i < 7; ++i) rows[i] = rows_lds[i * 256];
    scale_row = rows_lds[7 * 256];
    FULL::fetch_rows(c, loc, loc.m0, wave, lane_rows, rows_next);
    scale_row_next = walk_scale_row(c, loc, tid_rows);
    if (c.row_map) scale_row_next = c.row_map[scale_row_next];
  } else {
    FULL::fetch_rows(c, done, done.m0, wave, lane_rows, rows);
    scale_row = walk_scale_row(c, done, tid_rows);
  }
  typename TILE::Acc acc;
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) acc[i][j] = i32x16_t{0};
  if constexpr (GATEUP) {
    // The lookups are waited for here, before the first load issued by hand.
#pragma unroll
    for (int i = 0; i < 7; ++i) asm volatile("" : "+v"(rows_next[i]));
    asm volatile("" : "+v"(scale_row_next));
    FULL::input_rows(c, rows_next);
    if (c.row_map) scale_row_next = div_by_map(c, scale_row_next);
#pragma unroll
    for (int i = 0; i < 7; ++i) rows_lds[i * 256] = rows_next[i];
    rows_lds[7 * 256] = scale_row_next;
  }
  // the tile's scales, into the half of their buffers that the tile before the last used
  turn ^= 1;
  {
    const char* slot = c.slots + (size_t)done.slot * c.slot_bytes;
    const I8Offsets off = i8_offsets((size_t)c.hidden, (size_t)c.ffn);
    const int n_groups = (GATEUP ? 2 * c.ffn : c.hidden) / TILE_N;
    int g = done.nt * 8 + tid_rows / 32;
    if (g >= n_groups) g = 0;  // (never stored)
    const float* scales = (const float*)(slot + (!GATEUP ? off.down_scales : g % 2 ? off.up_scales : off.gate_scales));
    load_to_lds_4(row_scales + scale_row, (uint32_t)(uintptr_t)(__attribute__((address_space(3))) float*)&w.row_scales[turn][wave * 64]);
    load_to_lds_4(scales + (GATEUP ? g / 2 : g) * TILE_N + tid_rows % 32,
                  (uint32_t)(uintptr_t)(__attribute__((address_space(3))) float*)&w.col_scales[turn][wave * 64]);
  }
  int lane_steps = lane;
  asm volatile("" : "+v"(lane_steps));
  auto then = [&]() __attribute__((always_inline)) {
    int lane_then = lane;
    asm volatile("" : "+v"(lane_then));
    if constexpr (GATEUP) {
#pragma unroll
      for (int i = 0; i < 7; ++i) {
        rows_next[i] = w.rows[i * 256 + wave * 64 + lane_then];
        asm volatile("" : "+v"(rows_next[i]));
      }
    } else {
      FULL::fetch_rows(c, loc, loc.m0, wave, lane_then, rows_next);
    }
    return TILE::row_sources(c, in, loc, rows_next, wave, lane_then);
  };
  TILE::template steps_walk<START, ODD>(TILE::row_sources(c, in, done, rows, wave, lane_steps), then, w.ring, wave, lane_steps, k_steps,
                                        stage, ring, acc);
  int lane_there = lane;
  asm volatile("" : "+v"(lane_there));
  TILE::epilogue_walk_i8(c, out, done, acc, w.staging, w.row_scales[turn], w.col_scales[turn] + wave * 64, wave, lane_there);
  walk_wait_ring(ring);
  // A next tile that is higher than this one: its last rows were not copied (this tile's steps copy FM row blocks).
  if (fm > FM) {  // uniform
    const int s0 = stage, s1 = stage + 1 == 3 ? 0 : stage + 1;
#pragma unroll
    for (int op = FM; op < 7; ++op)
      if (op < fm) {
        const typename FULL::RowSrc src = FULL::row_sources(c, in, loc, rows_next, wave, lane_there);
        FULL::copy_to_stage(src.a_at(op, 0), lds0, wave, s0, op);
        FULL::copy_to_stage(src.a_at(op, 8), lds0, wave, s1, op);
      }
    wait_vmcnt<0>();
  }
}

// ODD: an odd number of K steps, every other tile of a block then starts in the other half of the weight ring.
template <bool GATEUP, bool NT, bool ODD, class OUT>
__global__ __launch_bounds__(256) void ffn_tile_walk_i8_kernel(TiledCtx c, const bf16_t* __restrict__ in, const float* __restrict__ row_scales,
                                                               OUT* __restrict__ out) {
  typedef WalkI8<GATEUP, 7, NT> FULL;
  __shared__ WalkI8Lds w;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) u32x4*)w.ring;
  const int tid = threadIdx.x, lane = tid % 64;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
  TileWalk<4> walk;
  walk.init(c, w.table);
  const int xcd = blockIdx.x % 8, stride = gridDim.x / 8;
  int idx = blockIdx.x / 8;
  TileLoc loc;
  if (!walk.at(xcd, idx, loc)) return;  // uniform over the block
  const int k_steps = FULL::k_units(c) / 64;
  int rows[7];  // input rows of the thread's copies
  u32x4 ring[8][2];
  int fm = loc.fm, stage = 0, turn = 0;
  FULL::fetch_rows(c, loc, loc.m0, wave, lane, rows);
  FULL::input_rows(c, rows);
  int scale_row = walk_scale_row(c, loc, tid);
  if (GATEUP && c.row_map) scale_row = div_by_map(c, c.row_map[scale_row]);
#pragma unroll
  for (int i = 0; i < 7; ++i) w.rows[i * 256 + tid] = rows[i];
  w.rows[7 * 256 + tid] = scale_row;
  walk_issue_prologue<FULL>(FULL::row_sources(c, in, loc, rows, wave, lane), lds0, wave, fm, ring);
  walk_wait_ring(ring);
  bool more = true;
#define HMOE_WALK_TILE(START, FM_) \
  walk_one_tile_i8<GATEUP, NT, ODD, START, FM_>(c, in, row_scales, out, walk, xcd, stride, wave, lane, k_steps, w, lds0, loc, idx, fm, more, \
                                            stage, turn, ring)
#define HMOE_WALK_HEIGHTS(START)              \
  if (fm == 7) HMOE_WALK_TILE(START, 7);      \
  else if (fm == 6) HMOE_WALK_TILE(START, 6); \
  else if (fm == 5) HMOE_WALK_TILE(START, 5); \
  else HMOE_WALK_TILE(START, 4)
  while (more) {
    HMOE_WALK_HEIGHTS(0);
    if constexpr (ODD) {
      if (!more) break;
      HMOE_WALK_HEIGHTS(1);
    }
  }
#undef HMOE_WALK_HEIGHTS
#undef HMOE_WALK_TILE
}

// Tile shapes.  nt: weight loads that are not kept in the caches.
enum { I8_FIT4 = 0, I8_FIT256 = 1, I8_WALK = 2, I8_SPLIT = 6 };  // (the last: down only, a multiple of four K steps)

template <bool GATEUP, class OUT>
static void launch_stage_i8(TiledCtx c, int shape, bool nt, int n_rows, const bf16_t* in, const float* row_scales, OUT* out, hipStream_t s) {
  const int n_total = GATEUP ? 2 * c.ffn : c.hidden;
  auto launch = [&](auto kernel, int bm, int bn, int threads, long most) {
    c.n_tiles_n = (n_total + bn - 1) / bn;
    c.grid_padded = (int)std::min(most, (tiles_upper_bound(c, n_rows, bm) + 7) / 8 * 8);
    hipLaunchKernelGGL(kernel, dim3((unsigned)c.grid_padded), dim3(threads), 0, s, c, in, row_scales, out);
  };
  constexpr int NW256 = GATEUP ? 8 : 4;
  constexpr long ALL = 0x7ffffff8;
  if (shape == I8_WALK) {
    const bool odd = (GATEUP ? c.hidden : c.ffn) / 128 % 2;
    c.walk_bm = 224;
    const auto kernel = odd ? (nt ? &ffn_tile_walk_i8_kernel<GATEUP, true, true, OUT> : &ffn_tile_walk_i8_kernel<GATEUP, false, true, OUT>)
                            : (nt ? &ffn_tile_walk_i8_kernel<GATEUP, true, false, OUT> : &ffn_tile_walk_i8_kernel<GATEUP, false, false, OUT>);
    launch(kernel, 224, 256, 256, 256);  // one block per CU
  } else if (shape == I8_SPLIT) {
    if constexpr (!GATEUP) launch(nt ? &ffn_tile_split_i8_kernel<true> : &ffn_tile_split_i8_kernel<false>, 160, 128, 512, ALL);
  } else if (shape == I8_FIT256) {
    launch(nt ? &ffn_tile256_i8_kernel<GATEUP, NW256, true, OUT> : &ffn_tile256_i8_kernel<GATEUP, NW256, false, OUT>, 256, 32 * NW256,
           64 * NW256, ALL);
  } else {
    launch(nt ? &ffn_tile_i8_kernel<GATEUP, 4, true, OUT> : &ffn_tile_i8_kernel<GATEUP, 4, false, OUT>, 128, 256, 256, ALL);
  }
}

// Which shape a launch takes (us; 64 experts of 2048 x 1408 top 6, 8 of 4096 x 14336 top 2, 64 of 3584 x 2560 top 8, 16 of 1024 x 640
// top 2, rows per expert on average):
//   * 60 rows or more (down 96): walking blocks; for a gate/up launch against the better of the other two shapes 84 / 89 and 100 /
//     104 (66 and 140 rows of the first), 207 / 226 (128 of the second), 232 / 245 (62 of the third), 37 / 51 (1000 of the fourth); one
//     expert of 3584 x 20480, 200 rows 41 / 50; but 20 rows of the second 167 / 157.  A down launch (66 rows of the first 49 / 44) has
//     half the columns or fewer and needs a tile for every CU: 200 rows of the second, 128 tiles, 154 / 130; 300 rows, 256 tiles, 145 / 186.
//   * A down launch of fewer tiles than CUs, 96 rows or more and a long K: halves of K (one expert of 3584 x 20480, 200 / 1000 rows 113 / 62,
//     127 / 94; of 2048 x 2048, 500 rows 22 / 15; but 64 rows of the former 45 / 48, and 130 rows of the second layer, 256 tiles, 116 / 117).
//   * Few tiles: up to 256 rows by 32 columns per wave, each wave of a tile then multiplies as little as it can and an
//     expert's weights are read once: fourth, 40 tokens 11.4 / 12.4; with a long K also when there are more tiles, since a tile's
//     time is what counts (down, 75 rows of the second 98 / 126).  But 90 experts of 768 x 768, 26 rows 42 / 30.
//   * Else 128 x 256, two blocks per CU.
// Weights that do not stay in the 256 MiB behind the L2s from call to call anyway are loaded past the caches while one
// tile holds all rows of an expert (down, 4.5 rows of the first 33 / 38; 40 tokens of the fourth, in the caches, 10.0 / 9.2).
struct I8Choice {
  int shape;
  bool nt;
};
static I8Choice choose_i8(const hmoe_layer_desc& d, int n_rows, bool gate_up) {
  const long K = gate_up ? d.hidden : d.ffn, n_total = gate_up ? 2l * d.ffn : d.hidden;
  const long busy = std::min(d.n_experts, n_rows), per_expert = n_rows / d.n_experts;
  const long k_steps = K / 128;
  const bool far = 3l * d.hidden * d.ffn * d.n_experts > (256l << 20);
  const long walk_tiles = (n_rows / 224 + busy) * ((n_total + 255) / 256);
  if (per_expert >= (gate_up ? 60 : 96) && k_steps >= 6 + k_steps % 2 && (gate_up || walk_tiles >= 256)) return {I8_WALK, far && per_expert <= 224};
  if (!gate_up && k_steps % 4 == 0 && K >= 2048 && per_expert >= 96 && (n_rows / 160 + busy) * ((n_total + 127) / 128) <= 256)
    return {I8_SPLIT, false};
  const long tiles = (n_rows / 128 + busy) * ((n_total + 255) / 256);
  if (tiles <= 128 || (tiles <= 320 && K >= 4096)) return {I8_FIT256, far && per_expert <= 192};
  return {I8_FIT4, far && per_expert <= 96};
}

int launch_ffn_tiled_i8(const FfnArgs& a) {
  const hmoe_layer_desc& d = *a.desc;
  if (d.dtype != HMOE_BF16_I8) return HMOE_ERR_UNSUPPORTED;
  if (a.n_rows == 0) return HMOE_OK;
  TiledCtx c{a.offsets, a.slot_of, a.slots, a.slot_bytes, a.active, d.n_experts, d.hidden, d.ffn, 0, 0, nullptr, 1};
  const I8Work w = i8_work(d, a.n_rows);
  const bf16_t* codes = (const bf16_t*)((const char*)a.h + w.codes);
  const float* scales = (const float*)((const char*)a.h + w.scales);
  I8Choice gate_up = choose_i8(d, a.n_rows, true), down = choose_i8(d, a.n_rows, false);
  if (const char* env = getenv("HMOE_I8_TILES")) {  // tuning and tests: "<gate/up><down>", 0 .. 2 the shapes, 3 .. 5 the same past the caches, 6 and 7 down in halves of K
    auto forced = [&](char c, int k, I8Choice otherwise, bool is_down) {
      const int v = c - '0';
      if (v == 6 || v == 7) return is_down && k / 128 % 4 == 0 ? I8Choice{I8_SPLIT, v == 7} : otherwise;
      if (v < 0 || v > 5 || (v % 3 == I8_WALK && k / 128 < 6 + k / 128 % 2)) return otherwise;
      return I8Choice{v % 3, v >= 3};
    };
    gate_up = forced(env[0], d.hidden, gate_up, false);
    if (env[0]) down = forced(env[1], d.ffn, down, true);
  }
  if (i8_shares_rows(a)) {
    launch_quantize_shared_x_i8(a);
    c.row_map = (const int32_t*)((const char*)a.h + w.code_row);
  } else {
    launch_quantize_x_i8(a);
  }
  probe_before(a.stream);
  launch_stage_i8<true>(c, gate_up.shape, gate_up.nt, a.n_rows, codes, scales, (float*)a.h, a.stream);
  probe_after(a.stream);
  launch_quantize_h_i8(a);
  probe_before(a.stream);
  launch_stage_i8<false>(c, down.shape, down.nt, a.n_rows, codes, scales, (bf16_t*)a.o_perm, a.stream);
  probe_after(a.stream);
  HMOE_HIP(hipGetLastError());
  return HMOE_OK;
}

}  // namespace hmoe
