// Prefill FFN (HMOE_FFN_TILED): grouped GEMM on bf16 MFMA, weights streamed past LDS.
//
// Two launches per call:  h = silu(X Wgate^T) * (X Wup^T)   and   O = h Wdown^T,
// each a grouped GEMM  C[rows of expert e, N] = A[rows, K] * W_e[N, K]^T  over the ragged row
// groups that the permutation produced (expert_offsets), with W_e found through the
// expert-id -> slot table.  All dispatch happens on the device: a block turns its index into
// (expert, m-tile, n-tile) by walking expert_offsets, so the host never reads the routing result.
//
// A block owns a tile of up to BM rows and 32 * FN * waves columns; every wave spans all rows and owns
// FN 32-row weight groups, as 32x32x16 bf16 MFMA fragments with fp32 accumulators.
//   * Weights arrive pre-tiled (packed slot layout): a 32-row x 16-k tile is 1 KiB in MFMA operand
//     order.  Each wave streams the tiles of its groups straight from global memory into a ring of
//     registers, DB k-substeps ahead; they never touch LDS.
//   * Activation tiles travel global -> LDS without passing through registers (global_load_lds_dwordx4:
//     every lane supplies a global address, the wave's 64 x 16 bytes land contiguously in LDS), into a
//     ring of SA stages; one barrier per K step of 64.  Rows are row-major; the lane that fills LDS chunk
//     (row, slot) fetches global chunk slot ^ f(row), an XOR swizzle that spreads the fragment reads over
//     all banks.
//   * Rows past the end of an expert and weight groups past N are loaded from a clamped (valid)
//     address instead of being zero-filled; their products land in accumulators that are never
//     stored.
//   * Gate and up rows are interleaved in 32-row groups, so with FN = 2 a wave's even fragments are gate
//     and its odd fragments the matching up columns: SwiGLU is applied to registers.
//   * Tiles are numbered expert-major, then n-tile, then m-tile, and block ids are dealt to the
//     8 XCDs in contiguous ranges so that blocks sharing a weight panel share an L2.
#include <stdlib.h>
#include <string.h>

#include <algorithm>
#include <type_traits>

#include "stream_tile.h"

namespace hmoe {

// ---------------------------------------------------------------------------------------------
// Kernels over a tile type.

template <class TILE>
__device__ __forceinline__ void zero_acc(typename TILE::Acc& acc) {
#pragma unroll
  for (int i = 0; i < TILE::FM; ++i)
#pragma unroll
    for (int j = 0; j < TILE::FN; ++j) acc[i][j] = f32x16_t{0};
}

template <class TILE>
__device__ __forceinline__ void run_tile(const TiledCtx& c, const bf16_t* __restrict__ in, bf16_t* __restrict__ out,
                                         const TileLoc& loc, u32x4* lds) {
  typename TILE::Acc acc;
  zero_acc<TILE>(acc);
  // A 224-row tile with two weight groups per wave keeps its accumulators in the second half of the register file
  // (one wave per SIMD, 512 registers).  A fitted instantiation needs fewer of them than the full tile, and the
  // register allocator would park weight-ring values in the free ones -- copying a register whose hand-issued load
  // has not landed.  Holding the unused accumulator registers over the tile leaves it nowhere to park.
  constexpr int HELD = TILE::BM == 224 && TILE::FN == 2 ? 14 - TILE::FM * TILE::FN : 0;
  f32x16_t held[HELD > 0 ? HELD : 1];
#pragma unroll
  for (int i = 0; i < HELD; ++i) asm volatile("" : "=a"(held[i]));
  TILE::mainloop(c, in, loc, 0, (TILE::GATEUP ? c.hidden : c.ffn) / TILE::BKT, lds, acc);
  TILE::epilogue(c, out, loc, acc, lds);
#pragma unroll
  for (int i = 0; i < HELD; ++i) asm volatile("" ::"a"(held[i]));
}

// One block per tile, tile height fitted to the expert.  An expert of R rows has ceil(R / 128) m-tiles whatever
// their height; instead of 128 rows each (the last one mostly padding when R is just above a multiple of 128)
// they all get ceil(R / tiles) rows, rounded up to whole 32-row fragments, and the block runs the tile type
// that multiplies that many fragments.  The m-tiles of one weight panel stay equally long -- their blocks run
// side by side and share the panel through L2, which uneven tiles would break -- and the padding rows that are
// multiplied drop from up to 127 to at most 31 per m-tile.
//
// Two waves per SIMD either way (the second launch bound caps the kernel at 256 registers): one block of 8 waves, or
// two blocks of 4 waves whose ring fill and epilogue overlap each other's main loop.  Left to itself the compiler
// gives the 4-wave kernel 480 registers and the CU a single block.  With 256 registers the 4-wave tile has room for
// a weight ring of one K step only.
template <bool GATEUP, int NWV, bool NT>
__global__ __launch_bounds__(64 * NWV, 2) void ffn_tile_fit_kernel(TiledCtx c, const bf16_t* __restrict__ in,
                                                                 bf16_t* __restrict__ out) {
  constexpr int RING = NWV == 4 ? 4 : 8;
  typedef StreamTile<GATEUP, 128, NWV, 4, NT, RING, 4> FULL;
  __shared__ u32x4 lds[FULL::LDS_VEC];
  TileLoc loc;
  if (!locate_tile<128>(c, loc)) return;  // uniform over the block
  const int tiles = (loc.m_rows + 127) / 128;
  const int fragments = ((loc.m_rows + tiles - 1) / tiles + 31) / 32;  // per m-tile, 1..4; uniform
  if (fragments == 4) run_tile<FULL>(c, in, out, loc, lds);
  else if (fragments == 3) run_tile<StreamTile<GATEUP, 128, NWV, 4, NT, RING, 3>>(c, in, out, loc, lds);
  else if (fragments == 2) run_tile<StreamTile<GATEUP, 128, NWV, 4, NT, RING, 2>>(c, in, out, loc, lds);
  else run_tile<StreamTile<GATEUP, 128, NWV, 4, NT, RING, 1>>(c, in, out, loc, lds);
}

template <bool GATEUP, int NWV, bool NT>
static void launch_tiles_fit(TiledCtx c, int n_rows, const bf16_t* in, bf16_t* out, hipStream_t s) {
  const int n_total = GATEUP ? 2 * c.ffn : c.hidden;
  c.n_tiles_n = (n_total + NWV * 64 - 1) / (NWV * 64);
  c.grid_padded = (int)((tiles_upper_bound(c, n_rows, 128) + 7) / 8 * 8);
  hipLaunchKernelGGL((ffn_tile_fit_kernel<GATEUP, NWV, NT>), dim3((unsigned)c.grid_padded), dim3(64 * NWV), 0, s, c, in, out);
}

// The same with tiles of up to 256 rows and one weight group per wave (tile width 32 * NWV columns): an expert of
// 129..256 rows takes one m-tile instead of two.  Heights come in steps of two fragments.
template <bool GATEUP, int NWV, bool NT>
__global__ __launch_bounds__(64 * NWV) void ffn_tile_fit256_kernel(TiledCtx c, const bf16_t* __restrict__ in,
                                                                    bf16_t* __restrict__ out) {
  typedef StreamTile<GATEUP, 256, NWV, 4, NT, 8, 8, 1> FULL;
  __shared__ u32x4 lds[FULL::LDS_VEC];
  TileLoc loc;
  if (!locate_tile<256>(c, loc)) return;  // uniform over the block
  const int tiles = (loc.m_rows + 255) / 256;
  const int fragments = ((loc.m_rows + tiles - 1) / tiles + 31) / 32;  // per m-tile, 1..8; uniform
  if (fragments > 6) run_tile<FULL>(c, in, out, loc, lds);
  else if (fragments > 4) run_tile<StreamTile<GATEUP, 256, NWV, 4, NT, 8, 6, 1>>(c, in, out, loc, lds);
  else if (fragments > 2) run_tile<StreamTile<GATEUP, 256, NWV, 4, NT, 8, 4, 1>>(c, in, out, loc, lds);
  else run_tile<StreamTile<GATEUP, 256, NWV, 4, NT, 8, 2, 1>>(c, in, out, loc, lds);
}

template <bool GATEUP, int NWV, bool NT>
static void launch_tiles_fit256(TiledCtx c, int n_rows, const bf16_t* in, bf16_t* out, hipStream_t s) {
  const int n_total = GATEUP ? 2 * c.ffn : c.hidden;
  c.n_tiles_n = (n_total + NWV * 32 - 1) / (NWV * 32);
  c.grid_padded = (int)((tiles_upper_bound(c, n_rows, 256) + 7) / 8 * 8);
  hipLaunchKernelGGL((ffn_tile_fit256_kernel<GATEUP, NWV, NT>), dim3((unsigned)c.grid_padded), dim3(64 * NWV), 0, s, c, in, out);
}

// Tiles of up to 224 rows with TWO weight groups per wave: 224x256 with four waves, one wave per SIMD, the 224
// accumulator registers of a wave in the second half of its register file (256 rows would fill that half to the last
// register, which the register allocator does not manage without spilling).  A CU then pulls (224 + 256) * 2 bytes
// per k for 224 x 256 products, against (128 + 256) * 2 for 128 x 256 with two resident 128x256 blocks.  With one
// wave per SIMD nothing hides what a wave issues between its matrix instructions: see ILV in StreamTile::steps.
// Gate/up only (a tuning variant; the walking blocks below are what the library chooses).
template <bool GATEUP, bool NT>
__global__ __launch_bounds__(256) void ffn_tile_fit256w_kernel(TiledCtx c, const bf16_t* __restrict__ in,
                                                                bf16_t* __restrict__ out) {
  typedef StreamTile<GATEUP, 224, 4, 4, NT, 8, 7, 2, true> FULL;
  __shared__ u32x4 lds[FULL::LDS_VEC];
  TileLoc loc;
  if (!locate_tile<224>(c, loc)) return;  // uniform over the block
  const int tiles = (loc.m_rows + 223) / 224;
  const int fragments = ((loc.m_rows + tiles - 1) / tiles + 31) / 32;  // per m-tile, 1..7; uniform
  if (fragments > 6) run_tile<FULL>(c, in, out, loc, lds);
  else if (fragments > 5) run_tile<StreamTile<GATEUP, 224, 4, 4, NT, 8, 6, 2, true>>(c, in, out, loc, lds);
  else if (fragments > 4) run_tile<StreamTile<GATEUP, 224, 4, 4, NT, 8, 5, 2, true>>(c, in, out, loc, lds);
  else run_tile<StreamTile<GATEUP, 224, 4, 4, NT, 8, 4, 2, true>>(c, in, out, loc, lds);
}

template <bool GATEUP, bool NT>
static void launch_tiles_fit256w(TiledCtx c, int n_rows, const bf16_t* in, bf16_t* out, hipStream_t s) {
  const int n_total = GATEUP ? 2 * c.ffn : c.hidden;
  c.n_tiles_n = (n_total + 255) / 256;
  c.grid_padded = (int)((tiles_upper_bound(c, n_rows, 224) + 7) / 8 * 8);
  hipLaunchKernelGGL((ffn_tile_fit256w_kernel<GATEUP, NT>), dim3((unsigned)c.grid_padded), dim3(256), 0, s, c, in, out);
}

// The 224x256 tile in a block that works through several tiles (one block per CU, every eighth of the tile list dealt
// to the blocks of one XCD in turn).  A tile's last two K steps issue the first loads and copies of the block's next
// tile (see StreamTile::steps_walk), so their latency passes under those steps and the epilogue instead of in front of
// the next K loop.  The activation ring has three stages of the full tile height whatever the tile's own, and the
// epilogue a staging region of its own; every vector-memory operation of the kernel after the tile table is issued
// by hand, except the row-map lookups at the start of a tile, where nothing else is in flight.
//
// One tile of fm == FM fragments.  In: loc, ring, stage and the thread's seven input rows at rows_lds (a slot of its own
// per thread and copy, in LDS: registers are short over the K loop) describe the tile, whose first loads have landed.
// Out: the same for the block's next tile (more: whether there is one), its first loads landed as well.
template <bool GATEUP, bool NT, int FM>
__device__ __forceinline__ void walk_one_tile(const TiledCtx& c, const bf16_t* __restrict__ in, bf16_t* __restrict__ out,
                                              const TileWalk<4>& walk, int xcd, int stride, int wave, int lane, int k_steps,
                                              u32x4* lds, uint32_t lds0, TileLoc& loc, int& idx, int& fm, bool& more, int& stage,
                                              int* rows_lds, u32x4 (&ring)[8][2]) {
  typedef StreamTile<GATEUP, 224, 4, 3, NT, 8, FM, 2, true, true> TILE;
  typedef StreamTile<GATEUP, 224, 4, 3, NT, 8, 7, 2, true, true> FULL;
  // The next tile is looked up before this tile's K loop, and the row-map entries of its copies are requested here,
  // where nothing issued by hand is in flight.  A block at its last tile looks that tile up once more, and its last
  // K steps load that tile's first steps once more, unused.
  const TileLoc done = loc;
  idx += stride;
  more = walk.at(xcd, idx, loc);  // leaves loc as it is when there is no further tile
  fm = loc.fm;
  // Input rows of this tile's copies and of the next tile's.  Gate/up (rows looked up in the row map): this tile's
  // come from the thread's slots in LDS, where the next tile's then go until the K loop's other steps are through.
  // Down projection: plain arithmetic, done where the rows are needed.
  int rows[7], rows_next[7];
  if constexpr (GATEUP) {
#pragma unroll
    for (int i = 0; i < 7; ++i) rows[i] = rows_lds[i * 256];
    int lane_rows = lane;  // (opaque copies of the lane id: what is derived from it is recomputed where it is used)
    asm volatile("" : "+v"(lane_rows));
    FULL::fetch_rows(c, loc, loc.m0, wave, lane_rows, rows_next);
  } else {
    int lane_rows = lane;
    asm volatile("" : "+v"(lane_rows));
    FULL::fetch_rows(c, done, done.m0, wave, lane_rows, rows);
  }
  typename TILE::Acc acc;
  zero_acc<TILE>(acc);
  if constexpr (GATEUP) {
    // The lookups are waited for here, before the first load issued by hand (a wait of the compiler's further down
    // would count the hand-issued loads as its own and drain them), and turned into input rows.
#pragma unroll
    for (int i = 0; i < 7; ++i) asm volatile("" : "+v"(rows_next[i]));
    FULL::input_rows(c, rows_next);
#pragma unroll
    for (int i = 0; i < 7; ++i) rows_lds[i * 256] = rows_next[i];
  }
  int lane_steps = lane;
  asm volatile("" : "+v"(lane_steps));
  auto then = [&]() __attribute__((always_inline)) {
    // (made here, so that the next tile's addresses are not held over this tile's other steps)
    int lane_then = lane;
    asm volatile("" : "+v"(lane_then));
    if constexpr (GATEUP) {
#pragma unroll
      for (int i = 0; i < 7; ++i) {
        rows_next[i] = rows_lds[i * 256];
        asm volatile("" : "+v"(rows_next[i]));
      }
    } else {
      FULL::fetch_rows(c, loc, loc.m0, wave, lane_then, rows_next);
    }
    return TILE::row_sources(c, in, loc, rows_next, wave, lane_then);
  };
  TILE::steps_walk(TILE::row_sources(c, in, done, rows, wave, lane_steps), then, lds, wave, lane_steps, k_steps, stage, ring, acc);
  int lane_there = lane;
  asm volatile("" : "+v"(lane_there));
  if constexpr (GATEUP) TILE::epilogue_lines_walk_tr(c, out, done, acc, lds + FULL::LDS_VEC, wave, lane_there);
  else TILE::epilogue_lines_down_walk_tr(c, out, done, acc, lds + FULL::LDS_VEC, wave, lane_there);
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

// DENSE: the launch is a single expert over all rows (a layer's shared experts).  The code is the same; the two are
// separate kernels so that traces and counter runs tell the shared experts' launches from the routed ones, which
// have the same grid.
template <bool GATEUP, bool NT, bool DENSE>
__global__ __launch_bounds__(256) void ffn_tile_walk_kernel(TiledCtx c, const bf16_t* __restrict__ in,
                                                             bf16_t* __restrict__ out) {
  typedef StreamTile<GATEUP, 224, 4, 3, NT, 8, 7, 2, true, true> FULL;
  constexpr int STAGING = 2 * 7 * 32 * 8;  // two [224][64] bf16 blocks, in 16-byte units
  __shared__ u32x4 lds[FULL::LDS_VEC + STAGING];
  __shared__ int walk_table[TileWalk<4>::TABLE_INTS];
  __shared__ int walk_rows[7 * 256];  // input rows of the copies of the tile at hand, then of the next: [copy][thread]
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) u32x4*)lds;
  const int tid = threadIdx.x, lane = tid % 64;
  const int wave = __builtin_amdgcn_readfirstlane(tid / 64);
  TileWalk<4> walk;
  walk.init(c, walk_table);
  const int xcd = blockIdx.x % 8, stride = gridDim.x / 8;
  int idx = blockIdx.x / 8;
  TileLoc loc;
  if (!walk.at(xcd, idx, loc)) return;  // uniform over the block
  const int k_steps = (GATEUP ? c.hidden : c.ffn) / 64;  // even, at least 6 (the launch sees to it)
  int rows[7];  // input rows of the thread's copies
  u32x4 ring[8][2];
  int fm = loc.fm;
  int stage = 0;
  FULL::fetch_rows(c, loc, loc.m0, wave, lane, rows);
  FULL::input_rows(c, rows);
#pragma unroll
  for (int i = 0; i < 7; ++i) walk_rows[i * 256 + tid] = rows[i];
  walk_issue_prologue<FULL>(FULL::row_sources(c, in, loc, rows, wave, lane), lds0, wave, fm, ring);
  walk_wait_ring(ring);
  bool more = true;
#define HMOE_WALK_TILE(FM_) \
  walk_one_tile<GATEUP, NT, FM_>(c, in, out, walk, xcd, stride, wave, lane, k_steps, lds, lds0, loc, idx, fm, more, stage, \
                                 walk_rows + tid, ring)
  while (more) {
    if (fm == 7) HMOE_WALK_TILE(7);
    else if (fm == 6) HMOE_WALK_TILE(6);
    else if (fm == 5) HMOE_WALK_TILE(5);
    else HMOE_WALK_TILE(4);
  }
#undef HMOE_WALK_TILE
}

template <bool GATEUP, bool NT>
static void launch_tiles_walk(TiledCtx c, int n_rows, const bf16_t* in, bf16_t* out, hipStream_t s) {
  const int n_total = GATEUP ? 2 * c.ffn : c.hidden;
  c.n_tiles_n = (n_total + 255) / 256;
  // The most fragments an m-tile may have.  Lower heights for launches of few rounds (whose partly filled last round
  // weighs more) were measured: a dense expert alone gains 10-23 %, routed experts lose 8 %, and the layer, whose
  // two FFNs overlap, stays where it is; 7 is kept.
  int cap = 7;
  if (const char* env = getenv("HMOE_WALK_CAP")) {  // tuning
    const int want = atoi(env);
    if (want >= 4 && want <= 7) cap = want;
  }
  c.walk_bm = 32 * cap;
  if ((GATEUP ? c.hidden : c.ffn) % 128 != 0 || (GATEUP ? c.hidden : c.ffn) < 384) {  // they need an even number of K steps, 6 or more
    launch_tiles_fit<GATEUP, 4, NT>(c, n_rows, in, out, s);
    return;
  }
  const long bound = (tiles_upper_bound(c, n_rows, c.walk_bm) + 7) / 8 * 8;
  long blocks = bound < 256 ? bound : 256;  // one per CU
  if (const char* env = getenv("HMOE_WALK_BLOCKS")) {  // tuning and tests: fewer blocks, more tiles each
    const long want = atol(env) / 8 * 8;
    if (want >= 8 && want < blocks) blocks = want;
  }
  c.grid_padded = (int)blocks;
  if (!NT && c.n_experts == 1)  // (what the library itself chooses for shared experts: plain loads)
    hipLaunchKernelGGL((ffn_tile_walk_kernel<GATEUP, false, true>), dim3((unsigned)c.grid_padded), dim3(256), 0, s, c, in, out);
  else
    hipLaunchKernelGGL((ffn_tile_walk_kernel<GATEUP, NT, false>), dim3((unsigned)c.grid_padded), dim3(256), 0, s, c, in, out);
}

// Tile shapes built into the library.  hmoe picks one from the average rows per expert; the
// environment variable HMOE_TILED_VARIANT (an index into this table) overrides the choice for
// tuning runs.
typedef void (*tiled_launch_fn)(TiledCtx, int, const bf16_t*, bf16_t*, hipStream_t);
struct TiledVariant {
  const char* name;
  tiled_launch_fn gate_up, down;
};
#define HMOE_STREAM_FIT(NAME, NWV, NT) { NAME, launch_tiles_fit<true, NWV, NT>, launch_tiles_fit<false, NWV, NT> }
#define HMOE_STREAM_FIT256(NAME, NWV_GU, NWV_D, NT) \
  { NAME, launch_tiles_fit256<true, NWV_GU, NT>, launch_tiles_fit256<false, NWV_D, NT> }
enum {
  V_FIT = 0,            // 128x512 tile, 8 waves, tile height fitted to the expert, non-temporal weight loads
  V_FIT_PLAIN = 1,      //   ... with plain weight loads
  V_FIT4 = 2,           // 128x256 tile, 4 waves, half the weight ring: two blocks per CU
  V_FIT4_PLAIN = 3,
  V_FIT256 = 4,         // tiles of up to 256 rows, one weight group per wave: 256x256 (gate/up, 8 waves), 256x128 (down, 4 waves)
  V_FIT256_PLAIN = 5,
  V_FIT256W = 6,        // gate/up: 224x256, 4 waves, two weight groups per wave, one wave per SIMD (down: as 0 / 1)
  V_FIT256W_PLAIN = 7,
  V_WALK = 8,           // the same tile in blocks that work through several tiles each
  V_WALK_PLAIN = 9
};
static const TiledVariant kVariants[] = {
    HMOE_STREAM_FIT("stream 128x512 fit", 8, true),
    HMOE_STREAM_FIT("stream 128x512 fit plain", 8, false),
    HMOE_STREAM_FIT("stream 128x256 fit, 4 waves", 4, true),
    HMOE_STREAM_FIT("stream 128x256 fit, 4 waves, plain", 4, false),
    HMOE_STREAM_FIT256("stream 256x256/128 fit", 8, 4, true),
    HMOE_STREAM_FIT256("stream 256x256/128 fit plain", 8, 4, false),
    {"stream 224x256, 4 waves", launch_tiles_fit256w<true, true>, launch_tiles_fit<false, 8, true>},
    {"stream 224x256, 4 waves, plain", launch_tiles_fit256w<true, false>, launch_tiles_fit<false, 8, false>},
    {"stream 224x256, walking blocks", launch_tiles_walk<true, true>, launch_tiles_walk<false, true>},
    {"stream 224x256, walking blocks, plain", launch_tiles_walk<true, false>, launch_tiles_walk<false, false>},
};
constexpr int kNumVariants = sizeof(kVariants) / sizeof(kVariants[0]);

int launch_ffn_tiled(const FfnArgs& a) {
  const hmoe_layer_desc& d = *a.desc;
  if (d.dtype != HMOE_BF16) return HMOE_ERR_UNSUPPORTED;
  if (a.n_rows == 0) return HMOE_OK;
  TiledCtx c{a.offsets, a.slot_of, a.slots, a.slot_bytes, a.active, d.n_experts, d.hidden, d.ffn, 0, 0, a.row_map, a.map_div};
  set_map_div(c);
  const bf16_t* x = (const bf16_t*)a.x_perm;
  bf16_t* h = (bf16_t*)a.h;
  bf16_t* o = (bf16_t*)a.o_perm;
  // Kernel choice (measured on the workload shapes and on batch-size sweeps of them; the tile counts are the
  // launch's upper bounds).
  //  * Experts of fewer than 192 rows on average stream each weight byte about once: 128x512 tiles with 8 waves,
  //    the tile height fitted to the expert, non-temporal weight loads.  When such a launch has too few tiles to
  //    fill the CUs, the time of one tile is what counts and it takes tiles of up to 256 rows and 32 columns per
  //    wave: each wave multiplies as little as the expert needs, and an expert of up to 256 rows streams its
  //    weights once.  Gate/up over a short K range (hidden < 4096) with experts of at most 32 rows on average takes
  //    the 128x256 tile with 4 waves, two blocks per CU: 2-10 % on the DeepSeek-style and Qwen2-style shapes up
  //    to 256 tokens (with a long K range the deeper weight ring of the 8-wave tile is worth more; with larger
  //    experts under skewed routing the non-temporal loads of several m-tiles per panel cost more than it gains).
  //  * Experts of 192 rows or more (a shared expert at a prefill batch, large routed experts) have several
  //    m-tiles that share their weight panel through L2: plain loads, and 128x256 tiles with 4 waves, two blocks
  //    per CU, so that one block's ring fill and epilogue overlap the other's main loop (4-14 % over the 8-wave
  //    tile on compute-bound launches).  The down projection keeps the 128x512 tile when its K range is short
  //    and its tiles are plenty (F < 4096: the stress and Qwen2 shapes, 1-2 % either way).
  const long m_tiles = (long)a.n_rows / 128 + std::min(d.n_experts, a.n_rows);
  const long tiles_down = m_tiles * ((d.hidden + 511) / 512);
  const bool few_gate_up = m_tiles * ((2 * d.ffn + 255) / 256) <= 128;
  const bool shared_panels = a.n_rows / d.n_experts >= 192;
  int v_gate_up = V_FIT, v_down = V_FIT;
  if (shared_panels) {
    v_gate_up = V_FIT4_PLAIN;
    v_down = tiles_down < 256 || d.ffn >= 4096 ? V_FIT4_PLAIN : V_FIT_PLAIN;
    // A dense expert with a very long K range: a few tiles of the down projection, each a chain of 192 K steps or more,
    // are what the layer's last launch waits for, the more so when the routed experts' launches got the CUs before
    // them.  Tiles of 256x128 halve the reads of weights per row and so the chain.  Shared expert of 3584 x 20480 beside 64
    // experts, top 8 (layer): 286 tokens 750 -> 716 us, 400 tokens 848 -> 770 us, 1003 tokens 1234 -> 1108 us; 4096 x
    // 14336 beside 16, top 2, 300 tokens 344 -> 306 us.  Up to 256 rows they are no more tiles than 128x256, but twice as
    // high (5 % slower at 220 rows), with 192 and more of them the many smaller ones are as fast, and for shorter K
    // (shared experts of 4096 to 8192) the layer is 25 % faster to 7 % slower, by how the two FFNs' blocks happen to meet.
    const long tiles_256 = ((long)a.n_rows + 255) / 256 * ((d.hidden + 127) / 128);
    if (d.n_experts == 1 && d.ffn >= 12288 && a.n_rows > 256 && tiles_256 <= 192) v_down = V_FIT256_PLAIN;
    // A layer whose routed experts make at least seven rounds of 224x256 tiles (a large batch) takes that tile with
    // one wave per SIMD, in blocks that walk through their tiles -- for both projections, and for the layer's shared
    // experts too (hmoe_cache_set_layer tells their launches which layer they run beside): stress shape -3.5 % per
    // layer, Qwen2 shape unchanged.  A block of these fills its CU, one of the other kernels half of one, and
    // launches of both kinds next to each other on two streams keep each other waiting (+2 %); alone, a dense
    // expert of a few rounds is 3-25 % slower with the large tile (its last, partly filled round).
    const hmoe_layer_desc& lay = a.beside ? *a.beside : d;
    const long lay_rows = a.beside ? (long)a.n_rows * lay.top_k : a.n_rows;
    const long m_tiles_224 = lay_rows / 224 + std::min((long)lay.n_experts, lay_rows);
    long min_rounds = 7;
    if (const char* env = getenv("HMOE_WALK_MIN_ROUNDS")) min_rounds = atol(env);  // tuning
    if (lay_rows / lay.n_experts >= 192 &&
        m_tiles_224 * ((2 * lay.ffn + 255) / 256) >= min_rounds * 256) v_gate_up = v_down = V_WALK_PLAIN;
  } else {
    if (few_gate_up) v_gate_up = V_FIT256;
    else if (d.hidden < 4096 && a.n_rows <= 32 * d.n_experts) v_gate_up = V_FIT4;
    // Experts of 96 to 191 rows on average: gate/up in walking blocks (non-temporal loads), whose weight stream does
    // not stop between tiles -- Mixtral shape at 512 tokens 405 -> 357 us, Qwen2 shape at 1024 tokens 480 -> 427 us,
    // DeepSeek-style at 1024 tokens 186 -> 181 us; below 96 rows the fitted tiles are faster (fewer padded rows).
    else if ((long)a.n_rows >= 96L * d.n_experts) v_gate_up = V_WALK;
    if (tiles_down < 256) v_down = V_FIT256;
  }
  if (const char* env = getenv("HMOE_TILED_VARIANT")) {
    // "<index>" for both projections or "<gate/up index>,<down index>"
    const int want_gate_up = atoi(env);
    const char* comma = strchr(env, ',');
    const int want_down = comma ? atoi(comma + 1) : want_gate_up;
    if (want_gate_up >= 0 && want_gate_up < kNumVariants) v_gate_up = want_gate_up;
    if (want_down >= 0 && want_down < kNumVariants) v_down = want_down;
  }
  probe_before(a.stream);
  kVariants[v_gate_up].gate_up(c, a.n_rows, x, h, a.stream);
  probe_after(a.stream);
  probe_before(a.stream);
  kVariants[v_down].down(c, a.n_rows, h, o, a.stream);
  probe_after(a.stream);
  HMOE_HIP(hipGetLastError());
  return HMOE_OK;
}

}  // namespace hmoe
