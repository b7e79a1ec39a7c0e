// The tile of the prefill FFN kernels (ffn_tiled.hip, ffn_tiled_i8.hip): a block's part of a grouped GEMM, with the weights
// streamed from global memory to registers and the activations through a ring of stages in LDS.
#pragma once

#include "common.h"
#include "tile_locate.h"

namespace hmoe {

// Number formats.  Both operands of a matrix instruction are 16 bytes per lane and its result 16 registers, whatever the
// format: a tile counts K in units of 16 bits, which hold PER_UNIT operands each.
struct StreamBf16 {
  static constexpr int PER_UNIT = 1;
  typedef f32x16_t acc_t;
  static __device__ __forceinline__ acc_t mfma(u32x4 a, u32x4 b, acc_t c) { return mfma_32x32x16_bf16(a, b, c); }
};
struct StreamI8 {
  static constexpr int PER_UNIT = 2;
  typedef i32x16_t acc_t;
  static __device__ __forceinline__ acc_t mfma(u32x4 a, u32x4 b, acc_t c) { return mfma_32x32x32_i8(a, b, c); }
};

// One 16-byte global -> LDS copy per lane; the wave's 64 chunks land at lds_base .. +1024 in lane
// order.  lds_base must be wave-uniform.  Completion is tracked by vmcnt like any vector load.
__device__ __forceinline__ void load_to_lds_16(const void* gptr, uint32_t lds_base) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off"
               :
               : "v"(gptr), "s"(__builtin_amdgcn_readfirstlane(lds_base))
               : "memory", "m0");
}
// One 4-byte copy per lane likewise: the wave's 64 values land at lds_base .. + 256.
__device__ __forceinline__ void load_to_lds_4(const void* gptr, uint32_t lds_base) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off"
               :
               : "v"(gptr), "s"(__builtin_amdgcn_readfirstlane(lds_base))
               : "memory", "m0");
}
// 16-byte global store issued by hand (a kernel that keeps hand-issued loads in flight across its epilogue issues
// every vector-memory operation itself, so that the compiler never waits for, or counts, any of them)
__device__ __forceinline__ void store_16(void* gptr, const u32x4& v) {
  asm volatile("global_store_dwordx4 %0, %1, off" ::"v"(gptr), "v"(v) : "memory");
}
template <int N>
__device__ __forceinline__ void wait_vmcnt() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// The two marks below put no instruction into the kernel; they are comments in the device assembly that the
// build's listing check (asm_check.py) reads to recount the hand-counted waits: where the copies of one activation
// stage end, and which wait opens a stage of a ring of SA.
__device__ __forceinline__ void mark_stage_issued() { asm volatile("; hmoe: activation stage issued" ::: "memory"); }
template <int N, int SA>
__device__ __forceinline__ void wait_vmcnt_opens_stage() {
  asm volatile("s_waitcnt vmcnt(%0) ; hmoe: opens an activation stage, ring of %1" ::"n"(N), "n"(SA) : "memory");
}
// Workgroup barrier that the compiler may not move LDS accesses across.  (No fence instruction:
// the waits that make the data visible are issued explicitly by the caller.)
__device__ __forceinline__ void block_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// ---------------------------------------------------------------------------------------------
// The tile.
//
// All NWV waves of a block span the whole BM rows; a wave owns 64 packed weight rows (one gate/up
// pair, or 64 output columns of the down projection; 32 with FN = 1).  Activation tiles go through the
// LDS ring (every wave needs all of them); weight tiles are 1 KiB each in MFMA operand order, so each wave
// streams its own straight from global memory into a ring of DB register slots, DB k-substeps ahead.
// Compared with staging both operands in LDS this removes the LDS fill and the LDS reads of the weight
// operand (about 40 % of the LDS traffic of a 256x256 tile) and keeps DB KiB per matrix in flight per wave,
// which is what the weight-streaming shapes need.
//
// Every vector-memory operation is issued by hand in a fixed order per k-substep
//   [FN weight-tile loads for substep s+DB] [this substep's share of the LDS copies for step t+SA-1]
// so the number of younger operations at each wait is a compile-time constant: N_B for a weight tile,
// N_A for an activation stage.  In the last steps the same operations are still issued, with the
// step clamped (their results are never used), which keeps the counts valid.
//
// NT: weight loads carry the non-temporal hint.  It pays when an expert has one or two m-tiles (each
// weight byte is used about once); with many m-tiles per expert the blocks of an XCD share the panel
// through L2 and plain loads are faster.
template <bool NT>
__device__ __forceinline__ u32x4 load_stream_16(const void* gptr) {
  u32x4 v;
  if (NT)
    asm volatile("global_load_dwordx4 %0, %1, off nt" : "=v"(v) : "v"(gptr) : "memory");
  else
    asm volatile("global_load_dwordx4 %0, %1, off" : "=v"(v) : "v"(gptr) : "memory");
  return v;
}
// the same from a wave-uniform address (held in scalar registers) plus a byte offset per lane
template <bool NT>
__device__ __forceinline__ u32x4 load_stream_16(const void* uniform, uint32_t lane_bytes) {
  u32x4 v;
  if (NT)
    asm volatile("global_load_dwordx4 %0, %1, %2 nt" : "=v"(v) : "v"(lane_bytes), "s"(uniform) : "memory");
  else
    asm volatile("global_load_dwordx4 %0, %1, %2" : "=v"(v) : "v"(lane_bytes), "s"(uniform) : "memory");
  return v;
}
// wait until at most N younger vector-memory operations are outstanding; the operands tie the wait
// to the registers whose loads it covers, so their uses cannot be scheduled above it
template <int N>
__device__ __forceinline__ void wait_vmcnt_regs(u32x4& a, u32x4& b) {
  asm volatile("s_waitcnt vmcnt(%2)" : "+v"(a), "+v"(b) : "n"(N) : "memory");
}
template <int N>
__device__ __forceinline__ void wait_vmcnt_regs(u32x4& a) {
  asm volatile("s_waitcnt vmcnt(%1)" : "+v"(a) : "n"(N) : "memory");
}

// FMC (0: off): the tile multiplies only its first FMC 32-row fragments and consecutive m-tiles of an expert
// start 32 * FMC rows apart (the activation copies still move BM rows).  The kernel picks FMC per expert so
// that the expert's m-tiles are equally high (see ffn_tile_fit_kernel).
//
// FN_ (2 or 1): 32-row weight groups per wave.  With one group a wave needs half the accumulators per row, which is
// what lets a tile span 256 rows (an expert of up to 256 rows then reads its weights once, in one block, instead of
// twice in two blocks that must keep pace to share them through L2); the gate and the up half of a SwiGLU pair then
// sit in neighbouring waves and meet through LDS in the epilogue.  Tiles higher than 128 rows copy only the rows
// they multiply (rounded up to what one copy instruction per thread moves).
// TR (with ILV): the weight tile is the first operand of the matrix instruction, so the accumulators hold the transposed
// block: a lane owns one row per fragment and, per weight group, four runs of four consecutive columns, which the
// epilogues turn into 8-byte pieces of an output row (a quarter of the conversions and LDS writes of the other form).
// NUM: the number format of the operands (StreamBf16, StreamI8).
template <bool GATEUP_, int BM_, int NWV, int SA, bool NT, int DB = 8, int FMC = 0, int FN_ = 2, bool ILV = false, bool TR = false,
          class NUM = StreamBf16>
struct StreamTile {
  static constexpr bool GATEUP = GATEUP_;
  static constexpr int BM = BM_;
  static constexpr int FN = FN_, BN = NWV * 32 * FN, BKT = 64, KK = 4;
  static constexpr int FM = FMC > 0 ? FMC : BM / 32;   // fragments multiplied
  static constexpr int MSTRIDE = 32 * FM;              // rows between the starts of consecutive m-tiles
  static_assert(FM * 32 <= BM && (FN == 1 || FN == 2) && (!TR || (ILV && FN == 2)), "");
  static_assert(DB % KK == 0, "the weight ring holds whole K steps");
  static constexpr int CPR = BKT / 8, RP = 256 / (BKT * 2);
  static constexpr int ROWS_PER_OP = 64 * NWV / CPR;   // rows one copy instruction of every thread moves
  static constexpr int A_ROWS = BM > 128 ? (FM * 32 + ROWS_PER_OP - 1) / ROWS_PER_OP * ROWS_PER_OP : BM;
  static constexpr int A_CHUNKS = A_ROWS * CPR;
  static constexpr int A_OPS = A_CHUNKS / (64 * NWV);
  static_assert(A_OPS >= 1 && A_OPS * 64 * NWV == A_CHUNKS, "activation tile must split evenly over the waves");
  static_assert(SA >= 3, "the activation ring needs three stages");
  static constexpr int OPS3 = A_OPS - A_OPS * 3 / KK;  // copies issued in the last substep of a step
  static constexpr int N_B = (DB - 1) * FN + (DB / KK) * A_OPS;
  static constexpr int N_A = (SA - 3) * (KK * FN + A_OPS) + 3 * FN + A_OPS - OPS3;
  static_assert(N_B <= 63 && N_A + FN - 1 <= 63, "vmcnt range");
  // ILV (one wave per SIMD): the substep's work is issued between its matrix instructions, in the order [weight group
  // 0] [copies] [weight group 1]; a wait for both groups of a ring slot then has one substep's copies fewer behind it.
  // The count uses the largest piece of copies, so it is exact or one operation stricter.
  static constexpr int N_B_ILV = N_B - (A_OPS + KK - 1) / KK;
  static constexpr int THREADS = 64 * NWV;
  // 16-byte units between ring stages: the tile's own rows, or with TR (blocks that go from tile to tile, whose next
  // tile is already being copied in while this one is multiplied) the rows of the highest tile, whatever FM is
  static constexpr int STAGE_CHUNKS = TR ? BM * CPR : A_CHUNKS;
  static constexpr int LDS_VEC = SA * STAGE_CHUNKS;  // 16-byte units
  typedef typename NUM::acc_t Acc[FM][FN];
  typedef f32x16_t Sums[FM][FN];  // what the epilogues take

  // length of a row of the input in units of 16 bits
  static __device__ __forceinline__ int k_units(const TiledCtx& c) { return (GATEUP ? c.hidden : c.ffn) / NUM::PER_UNIT; }

  // Where a thread's copies and weight loads start: a_src[i] is the 16-byte chunk of the activation tile that copy i
  // of this thread moves (rows past the expert's end clamped to its last row), b_src[j] the thread's piece of the
  // first weight tile of the wave's group j (groups past N clamped to group 0).  m0 is the tile's first row within
  // the expert.  NA may exceed A_OPS (a caller that serves tile types of several heights with one set of pointers).
  // In two steps, so that a caller can put other work between the lookups and their use.
  //
  // Sorted rows of the thread's copies, and with a row map (the gather folded into gate/up) what the map holds for
  // them: all lookups are issued before the first is used, one trip to memory per tile.
  template <int NA>
  static __device__ __forceinline__ void fetch_rows(const TiledCtx& c, const TileLoc& loc, int m0, int wave, int lane,
                                                    int (&rows)[NA]) {
#pragma unroll
    for (int i = 0; i < NA; ++i) {
      const int r = ((i * NWV + wave) * 64 + lane) / CPR;
      rows[i] = loc.row_first + (m0 + r < loc.m_rows ? m0 + r : loc.m_rows - 1);
    }
    if (GATEUP && c.row_map) {
#pragma unroll
      for (int i = 0; i < NA; ++i) rows[i] = c.row_map[rows[i]];
    }
  }
  // ... the input rows from what the map holds
  template <int NA>
  static __device__ __forceinline__ void input_rows(const TiledCtx& c, int (&rows)[NA]) {
    if (GATEUP && c.row_map) {
#pragma unroll
      for (int i = 0; i < NA; ++i) rows[i] = div_by_map(c, rows[i]);
    }
  }
  // ... and the pointers from the input rows
  template <int NA>
  static __device__ __forceinline__ void set_sources_from(const TiledCtx& c, const bf16_t* __restrict__ in, const TileLoc& loc,
                                                          const int (&rows)[NA], int k_begin, int wave, int lane,
                                                          const u32x4* (&a_src)[NA], const u32x4* (&b_src)[FN]) {
    const int K = k_units(c);
    const int n_groups = (GATEUP ? 2 * c.ffn : c.hidden) / TILE_N;
    const int kt16 = K / TILE_K;
    const char* slot = c.slots + (size_t)loc.slot * c.slot_bytes;
    const u32x4* w = GATEUP ? (const u32x4*)slot : (const u32x4*)(slot + 4 / NUM::PER_UNIT * (size_t)c.ffn * c.hidden);
#pragma unroll
    for (int i = 0; i < NA; ++i) {
      const int ci = (i * NWV + wave) * 64 + lane;
      const int r = ci / CPR, sl = ci % CPR;
      const int chunk = sl ^ ((r / RP) % CPR);
      a_src[i] = (const u32x4*)(in + (size_t)rows[i] * K) + chunk + (size_t)k_begin * CPR;
    }
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      const int g = loc.nt * (BN / TILE_N) + wave * FN + j;
      b_src[j] = w + ((size_t)(g < n_groups ? g : 0) * kt16 + (size_t)k_begin * KK) * 64 + lane;
    }
  }
  template <int NA>
  static __device__ __forceinline__ void set_sources(const TiledCtx& c, const bf16_t* __restrict__ in, const TileLoc& loc,
                                                     int m0, int k_begin, int wave, int lane, const u32x4* (&a_src)[NA],
                                                     const u32x4* (&b_src)[FN]) {
    int rows[NA];
    fetch_rows(c, loc, m0, wave, lane, rows);
    input_rows(c, rows);
    set_sources_from(c, in, loc, rows, k_begin, wave, lane, a_src, b_src);
  }
  // copy `op` of this thread for K step `kstep` (clamped to the last step) into ring stage `stage`
  template <int NA>
  static __device__ __forceinline__ void issue_a_op(const u32x4* (&a_src)[NA], uint32_t lds0, int wave, int k_steps,
                                                    int stage, int kstep, int op) {
    copy_to_stage(a_src[op] + (size_t)(kstep < k_steps ? kstep : k_steps - 1) * CPR, lds0, wave, stage, op);
  }
  // copy `op` of this thread, from `from`, into ring stage `stage`
  static __device__ __forceinline__ void copy_to_stage(const u32x4* from, uint32_t lds0, int wave, int stage, int op) {
    const uint32_t base = lds0 + (uint32_t)stage * STAGE_CHUNKS * 16;
    load_to_lds_16(from, base + (uint32_t)((op * NWV + wave) * 64) * 16);
  }
  // piece `piece` (of KK) of the copies of one stage
  template <int NA>
  static __device__ __forceinline__ void issue_a_piece(const u32x4* (&a_src)[NA], uint32_t lds0, int wave, int k_steps,
                                                       int stage, int kstep, int piece) {
#pragma unroll
    for (int op = 0; op < A_OPS; ++op)
      if (op >= A_OPS * piece / KK && op < A_OPS * (piece + 1) / KK) issue_a_op(a_src, lds0, wave, k_steps, stage, kstep, op);
    if (piece == KK - 1) mark_stage_issued();
  }
  // The start of a tile: fill the weight ring and SA-1 activation stages.  Nothing is waited for.
  template <int NA>
  static __device__ __forceinline__ void issue_prologue(const u32x4* (&a_src)[NA], const u32x4* (&b_src)[FN], uint32_t lds0,
                                                        int wave, int k_steps, u32x4 (&ring)[DB][FN]) {
    const int n_sub = k_steps * KK;
#pragma unroll
    for (int s = 0; s < DB; ++s)
#pragma unroll
      for (int j = 0; j < FN; ++j) ring[s][j] = load_stream_16<NT>(b_src[j] + (size_t)(s < n_sub ? s : n_sub - 1) * 64);
#pragma unroll
    for (int st = 0; st < SA - 1; ++st)
#pragma unroll
      for (int p = 0; p < KK; ++p) issue_a_piece(a_src, lds0, wave, k_steps, st, st, p);
  }

  // acc += A[rows of the tile, k range] * W[columns of the tile, k range]^T for the k_steps steps of BKT
  // that start at step k_begin.  On return every copy into LDS has landed.
  static __device__ __forceinline__ void mainloop(const TiledCtx& c, const bf16_t* __restrict__ in, const TileLoc& loc,
                                                  int k_begin, int k_steps, u32x4* lds, Acc& acc) {
    const int tid = threadIdx.x, lane = tid % 64;
    const int wave = __builtin_amdgcn_readfirstlane(tid / 64);  // uniform: LDS bases and weight groups stay scalar
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) u32x4*)lds;
    const u32x4* a_src[A_OPS];
    const u32x4* b_src[FN];
    set_sources(c, in, loc, loc.mt * MSTRIDE, k_begin, wave, lane, a_src, b_src);
    u32x4 ring[DB][FN];
    issue_prologue(a_src, b_src, lds0, wave, k_steps, ring);
    steps(a_src, b_src, lds, wave, lane, k_steps, ring, acc);
  }
  // ... by a set of waves of a larger block, for an even number of steps: tid is the thread's number in the set, lds the set's
  // own.  (The barriers are the block's: every set takes as many steps.)
  static __device__ __forceinline__ void mainloop_of_set(const TiledCtx& c, const bf16_t* __restrict__ in, const TileLoc& loc, int k_begin,
                                                         int k_steps, u32x4* lds, Acc& acc, int tid) {
    const int lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) u32x4*)lds;
    const u32x4* a_src[A_OPS];
    const u32x4* b_src[FN];
    set_sources(c, in, loc, loc.mt * MSTRIDE, k_begin, wave, lane, a_src, b_src);
    u32x4 ring[DB][FN];
    issue_prologue(a_src, b_src, lds0, wave, k_steps, ring);
    steps<true>(a_src, b_src, lds, wave, lane, k_steps, ring, acc);
  }

  // fragment i (rows 32 i ..) of k-substep kk of a ring stage, for the lane that owns (half, col) of the operand
  static __device__ __forceinline__ u32x4 read_fragment(const u32x4* lds, int stage, int kk, int i, int half, int col) {
    const int r = i * 32 + col;
    return lds[stage * STAGE_CHUNKS + r * CPR + ((kk * 2 + half) ^ ((r / RP) % CPR))];
  }
  // One k-substep of a wave that has its SIMD to itself (ILV): nothing else fills the matrix pipe while this wave issues
  // anything else, so all other work of the substep sits between its matrix instructions, one piece behind each: the
  // next substep's fragment reads behind the first FM, which multiply weight group 0; then the reload of group 0's
  // ring slot, this substep's activation copies, and behind the last one the reload of group 1.  Vector-memory order
  // per substep: [group 0] [copies] [group 1].  kk: substep within the K step; sl: its ring slot; w_next: where the
  // reloads read (16-byte units from b_src); koff: where the copies read (from a_src), into fill_stage.
  // Where the operands of a tile come from.  As pointers per thread: a[op] is the thread's 16 bytes of copy op at the
  // tile's first K step, b[j] its piece of the first weight tile of group j.
  template <int NA>
  struct PtrSrc {
    const u32x4* (&a)[NA];
    const u32x4* (&b)[FN];
    __device__ __forceinline__ const u32x4* a_at(int op, size_t koff) const { return a[op] + koff; }
    __device__ __forceinline__ u32x4 b_at(int j, size_t w) const { return load_stream_16<NT>(b[j] + w); }
  };
  // Or, for a block that goes from tile to tile and holds two tiles' sources over a K loop, in half the registers:
  // the input ROW of each copy (the thread's place within a row, a_lane, is the same for every copy and tile), and
  // wave-uniform weight addresses in scalar registers with the lane's offset added by the load.
  struct RowSrc {
    const u32x4* a_lane;  // input + the thread's chunk within a row
    uint32_t pitch;       // 16-byte units per input row
    const int (&rows)[7];
    const u32x4* b[2];    // wave-uniform
    uint32_t lane_bytes;
    __device__ __forceinline__ const u32x4* a_at(int op, size_t koff) const {
      return a_lane + ((size_t)(uint32_t)rows[op] * pitch + koff);
    }
    __device__ __forceinline__ u32x4 b_at(int j, size_t w) const { return load_stream_16<NT>(b[j] + w, lane_bytes); }
  };
  template <class SRC, int NF>
  static __device__ __forceinline__ void ilv_substep(int kk, int sl, int stage, int next_stage, int fill_stage, size_t w_next,
                                                     size_t koff, const SRC& src, const u32x4* lds, uint32_t lds0, int wave,
                                                     int half, int col, u32x4 (&ring)[DB][FN], u32x4 (&fa)[NF][FM],
                                                     Acc& acc) {
    static_assert(FN == 2 && NF == 2, "");
    wait_vmcnt_regs<N_B_ILV>(ring[sl][0], ring[sl][1]);
#pragma unroll
    for (int m = 0; m < 2 * FM; ++m) {
      const int i = m % FM, j = m / FM;
      acc[i][j] = TR ? NUM::mfma(ring[sl][j], fa[kk & 1][i], acc[i][j])
                     : NUM::mfma(fa[kk & 1][i], ring[sl][j], acc[i][j]);
      if (m < FM)
        fa[(kk + 1) & 1][m] = kk == KK - 1 ? read_fragment(lds, next_stage, 0, m, half, col)
                                           : read_fragment(lds, stage, kk + 1, m, half, col);
      if (m == FM) ring[sl][0] = src.b_at(0, w_next);
#pragma unroll
      for (int op = 0; op < A_OPS; ++op)
        if (op >= A_OPS * kk / KK && op < A_OPS * (kk + 1) / KK) {
          const int at = FM + 1 + (op - A_OPS * kk / KK);
          if (m == (at < 2 * FM - 1 ? at : 2 * FM - 1)) copy_to_stage(src.a_at(op, koff), lds0, wave, fill_stage, op);
        }
      if (m == 2 * FM - 1) {
        if (kk == KK - 1) mark_stage_issued();
        ring[sl][1] = src.b_at(1, w_next);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  // The K loop of a tile whose prologue has been issued (by this thread, into `ring` and the first SA-1 stages).
  // On return every vector-memory operation of the thread has completed.
  // EVEN: k_steps is even, and the ring holds two steps.
  template <bool EVEN = false, int NA>
  static __device__ __forceinline__ void steps(const u32x4* (&a_src)[NA], const u32x4* (&b_src)[FN], u32x4* lds, int wave,
                                               int lane, int k_steps, u32x4 (&ring)[DB][FN], Acc& acc) {
    const int half = lane / 32, col = lane % 32;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) u32x4*)lds;
    const int n_sub = k_steps * KK;
    // Activation fragments: two sets with two weight groups per wave (the next substep's set is read while this one
    // is multiplied); one set with one group, where a fragment feeds a single MFMA and is refilled right behind it.
    constexpr int FA_SETS = FN == 1 ? 1 : 2;
    u32x4 fa[FA_SETS][FM];
    auto read_frag = [&](int stage, int kk, int i) { return read_fragment(lds, stage, kk, i, half, col); };
    auto read_a = [&](int buf, int stage, int kk) {
      const u32x4* sa = lds + stage * STAGE_CHUNKS;
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        const int r = i * 32 + col;
        fa[buf][i] = sa[r * CPR + ((kk * 2 + half) ^ ((r / RP) % CPR))];
      }
    };

    // ---- the prologue's loads and copies: wait for all of them ----
    wait_vmcnt<0>();
    block_barrier();
    read_a(0, 0, 0);

    int stage = 0;  // ring stage of step tt
    // one K step; hc carries h, the step's place in the weight ring (a compile-time constant: the ring is registers)
    auto k_step = [&](int tt, auto hc) __attribute__((always_inline)) {
        constexpr int h = decltype(hc)::value;
        {
          const int next_stage = stage + 1 == SA ? 0 : stage + 1;
          const int fill_stage = stage == 0 ? SA - 1 : stage - 1;  // held step tt-1, free since this step opened
#pragma unroll
          for (int kk = 0; kk < KK; ++kk) {
            if (kk == KK - 1) {
              // open step tt+1: its activation tile has landed once at most N_A younger operations are out
              wait_vmcnt_opens_stage<ILV ? N_A + FN - 1 : N_A, SA>();
              __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0): this step's last fragments are in registers
              block_barrier();
              if constexpr (FN == 2 && !ILV) read_a((kk + 1) & 1, next_stage, 0);
            } else {
              if constexpr (FN == 2 && !ILV) read_a((kk + 1) & 1, stage, kk + 1);
            }
            __builtin_amdgcn_sched_barrier(0);
            const int sl = h * KK + kk;  // ring slot of substep 4*tt + kk
            if constexpr (FN == 2 && ILV) {
              const int s_next = tt * KK + kk + DB;
              const int copy_step = tt + SA - 1;
              ilv_substep(kk, sl, stage, next_stage, fill_stage, (size_t)(s_next < n_sub ? s_next : n_sub - 1) * 64,
                          (size_t)(copy_step < k_steps ? copy_step : k_steps - 1) * CPR, PtrSrc<NA>{a_src, b_src}, lds, lds0, wave,
                          half, col, ring, fa, acc);
            } else if constexpr (FN == 2) {
              wait_vmcnt_regs<N_B>(ring[sl][0], ring[sl][1]);
#pragma unroll
              for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) acc[i][j] = NUM::mfma(fa[kk & 1][i], ring[sl][j], acc[i][j]);
            } else {
              wait_vmcnt_regs<N_B>(ring[sl][0]);
#pragma unroll
              for (int i = 0; i < FM; ++i) {
                acc[i][0] = NUM::mfma(fa[0][i], ring[sl][0], acc[i][0]);
                fa[0][i] = kk == KK - 1 ? read_frag(next_stage, 0, i) : read_frag(stage, kk + 1, i);
              }
            }
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (!ILV) {
              const int s_next = tt * KK + kk + DB;
#pragma unroll
              for (int j = 0; j < FN; ++j)
                ring[sl][j] = load_stream_16<NT>(b_src[j] + (size_t)(s_next < n_sub ? s_next : n_sub - 1) * 64);
              issue_a_piece(a_src, lds0, wave, k_steps, fill_stage, tt + SA - 1, kk);
            }
          }
          stage = next_stage;
        }
    };
    static_assert(DB / KK == 1 || DB / KK == 2, "the weight ring holds one or two K steps");
    if constexpr (ILV && DB / KK == 2) {
      // Pairs of steps without a condition inside the loop, then the odd step if there is one: accumulators that
      // pass through a conditional block inside the loop are more than the register allocator handles when they
      // fill the second register file.
      int t = 0;
      for (; t + 2 <= k_steps; t += 2) {
        k_step(t, std::integral_constant<int, 0>{});
        k_step(t + 1, std::integral_constant<int, 1>{});
      }
      if (t < k_steps) k_step(t, std::integral_constant<int, 0>{});
    } else if constexpr (EVEN) {
      static_assert(DB / KK == 2, "");
      int t = 0;
      do {
        k_step(t, std::integral_constant<int, 0>{});
        k_step(t + 1, std::integral_constant<int, 1>{});
        t += 2;
      } while (t < k_steps);
    } else {
      for (int t = 0; t < k_steps; t += DB / KK) {
        k_step(t, std::integral_constant<int, 0>{});
        if constexpr (DB / KK == 2)
          if (t + 1 < k_steps) k_step(t + 1, std::integral_constant<int, 1>{});
      }
    }
    wait_vmcnt<0>();  // the clamped tail copies must not outlive the block's LDS
    // The tail's weight loads are never multiplied.  The compiler knows nothing of their latency: without a use
    // after the wait it may give two of them the same destination, or build the next address in a register that
    // a load still in flight is about to overwrite.  Keeping every ring slot alive up to here rules that out.
#pragma unroll
    for (int s = 0; s < DB; ++s)
#pragma unroll
      for (int j = 0; j < FN; ++j) asm volatile("" ::"v"(ring[s][j]));
  }

  // The K loop of a block that goes from tile to tile (TR).  On entry the weight ring and the first two activation
  // stages of the tile have landed (the thread's own part; a barrier here covers the other waves'): they were issued
  // by the previous tile's last two K steps, or by the block's first prologue.  The last two K steps of this tile in
  // turn issue the first loads of the NEXT tile, from the sources that `then()` returns (called when the other steps
  // are through), in place of loads this tile has no use for: they run the same code with their step numbers counted
  // from the next tile's start.  No operation changes its place in the
  // vector-memory order, so every hand-counted wait stands.  The ring holds two K steps: START is the half of it that holds
  // the tile's first one.  k_steps is even and at least 6, or with ODD odd and at least 7; the next tile then starts in the
  // other half.
  // stage: the ring stage of the tile's first step, on return that of the next tile's first step.
  // On return the next tile's first loads and copies are in flight.
  template <int START = 0, bool ODD = false, class THEN>
  static __device__ __forceinline__ void steps_walk(const RowSrc& now, THEN then, u32x4* lds, int wave, int lane, int k_steps,
                                                    int& stage, u32x4 (&ring)[DB][FN], Acc& acc) {
    static_assert(TR && ILV && FN == 2 && DB == 2 * KK && SA == 3, "");
    const int half = lane / 32, col = lane % 32;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) u32x4*)lds;
    u32x4 fa[2][FM];
    block_barrier();  // the copies of every wave into the first stage have landed (each waited for its own)
#pragma unroll
    for (int i = 0; i < FM; ++i) fa[0][i] = read_fragment(lds, stage, 0, i, half, col);
    // one K step; hc: its place in the weight ring; first: the step that src counts from
    auto k_step = [&](int tt, auto hc, const RowSrc& src, int first) __attribute__((always_inline)) {
      constexpr int h = decltype(hc)::value;
      const int next_stage = stage + 1 == SA ? 0 : stage + 1;
      const int fill_stage = stage == 0 ? SA - 1 : stage - 1;  // held step tt-1, free since this step opened
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        if (kk == KK - 1) {
          wait_vmcnt_opens_stage<N_A + FN - 1, SA>();  // open step tt+1
          __builtin_amdgcn_s_waitcnt(0xC07F);          // lgkmcnt(0): this step's last fragments are in registers
          block_barrier();
        }
        __builtin_amdgcn_sched_barrier(0);
        ilv_substep(kk, h * KK + kk, stage, next_stage, fill_stage, (size_t)((tt - first) * KK + kk + DB) * 64,
                    (size_t)(tt - first + SA - 1) * CPR, src, lds, lds0, wave, half, col, ring, fa, acc);
        __builtin_amdgcn_sched_barrier(0);
      }
      stage = next_stage;
    };
    // The first two steps stand apart: the accumulators start at zero (the caller's zero_acc), so their first matrix
    // instructions take the constant as their addend and nothing has to be cleared.
    std::integral_constant<int, START> here;
    std::integral_constant<int, 1 - START> there;
    k_step(0, here, now, 0);
    k_step(1, there, now, 0);
    // (a loop that always runs: with a way round it, registers with loads in flight would meet at the far end)
    int t = 2;
#pragma nounroll
    do {
      k_step(t, here, now, 0);
      k_step(t + 1, there, now, 0);
      t += 2;
    } while (t + 2 < k_steps - (ODD ? 1 : 0));
    if constexpr (ODD) {
      k_step(t, here, now, 0);
      const RowSrc after = then();
      k_step(t + 1, there, after, k_steps);
      k_step(t + 2, here, after, k_steps);
    } else {
      const RowSrc after = then();
      k_step(t, here, after, k_steps);
      k_step(t + 1, there, after, k_steps);
    }
  }
  // The sources of a tile, given the input rows of its copies
  static __device__ __forceinline__ RowSrc row_sources(const TiledCtx& c, const bf16_t* __restrict__ in, const TileLoc& loc,
                                                       const int (&rows)[7], int wave, int lane) {
    const int K = k_units(c);
    const int n_groups = (GATEUP ? 2 * c.ffn : c.hidden) / TILE_N;
    const int kt16 = K / TILE_K;
    const char* slot = c.slots + (size_t)loc.slot * c.slot_bytes;
    const u32x4* w = GATEUP ? (const u32x4*)slot : (const u32x4*)(slot + 4 / NUM::PER_UNIT * (size_t)c.ffn * c.hidden);
    // the thread's chunk within a row: the same for every copy (32 rows apart, and the swizzle repeats every 16 rows)
    const int ci = wave * 64 + lane;
    const int chunk = (ci % CPR) ^ (((ci / CPR) / RP) % CPR);
    const int g0 = loc.nt * (BN / TILE_N) + wave * FN;
    return RowSrc{(const u32x4*)in + chunk, (uint32_t)(K / 8), rows,
                  {w + (size_t)(g0 < n_groups ? g0 : 0) * kt16 * 64, w + (size_t)(g0 + 1 < n_groups ? g0 + 1 : 0) * kt16 * 64},
                  (uint32_t)lane * 16};
  }

  static __device__ __forceinline__ void epilogue(const TiledCtx& c, bf16_t* __restrict__ out, const TileLoc& loc,
                                                  const Sums& acc, u32x4* lds) {
    if constexpr (GATEUP && FN == 1) epilogue_pairs(c, out, loc, acc, lds);
    else if constexpr (GATEUP) epilogue_lines(c, out, loc, acc, lds);
    else if constexpr (FN == 2) epilogue_lines_down(c, out, loc, acc, lds);
    else epilogue_lines_block(c, out, loc, acc, lds);
  }
  // Gate/up with one weight group per wave: wave 2p holds the gate half and wave 2p+1 the up half of pair p, for all
  // rows.  The gate wave finishes the first HALF fragments and the up wave the others; each passes the partner the
  // accumulators the partner finishes, through the (now idle) activation ring in LDS.
  static constexpr int HALF = (FM + 1) / 2;
  template <class H>
  static __device__ __forceinline__ void epilogue_pairs(const TiledCtx& c, H* __restrict__ out, const TileLoc& loc,
                                                        const Sums& acc, u32x4* lds) {
    static_assert(NWV % 2 == 0 && NWV * HALF * 1024 <= LDS_VEC * 4, "the exchange must fit the activation ring");
    const int row_first = loc.row_first, m_rows = loc.m_rows, nt = loc.nt;
    const int n_out = c.ffn;
    const int m0 = loc.mt * MSTRIDE;
    const int tid = threadIdx.x, wave = tid / 64, lane = tid % 64;
    const int half = lane / 32, col = lane % 32;
    const bool up_wave = wave & 1;
    float* mine = (float*)lds + (size_t)wave * HALF * 1024;          // what this wave hands over
    const float* theirs = (const float*)lds + (size_t)(wave ^ 1) * HALF * 1024;
    block_barrier();  // every wave has read its last activation fragments
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      if ((i < HALF) == up_wave) {  // uniform per wave: a fragment the partner finishes
        const int fi = i < HALF ? i : i - HALF;
#pragma unroll
        for (int r = 0; r < 16; ++r) mine[(fi * 16 + r) * 64 + lane] = acc[i][0][r];
      }
    }
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
    block_barrier();
    const int f = (nt * (BN / 64) + wave / 2) * 32 + col;
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      if ((i < HALF) != up_wave) {
        const int fi = i < HALF ? i : i - HALF;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float other = theirs[(fi * 16 + r) * 64 + lane];
          const float g = up_wave ? other : acc[i][0][r];
          const float u = up_wave ? acc[i][0][r] : other;
          const int m = m0 + i * 32 + (r / 4) * 8 + half * 4 + (r % 4);
          if constexpr (sizeof(H) == 2) {
            if (m < m_rows && f < n_out) out[(size_t)(row_first + m) * n_out + f] = f32_to_bf16(silu_f32(g) * u);
          } else {
            if (m < m_rows && f < n_out) out[(size_t)(row_first + m) * n_out + f] = silu_f32(g) * u;
          }
        }
      }
    }
  }
  // Gate/up with two weight groups per wave: a wave's SwiGLU results are 32 columns wide, half a 128-byte line of h,
  // and written as such they cost the launch 6-10 % (partial lines, the other half arriving from another wave at
  // another time).  Waves 2p and 2p+1 own neighbouring columns: both put their results into one [rows][64] block in
  // the idle activation ring, then each stores half of the rows as whole lines, 16 bytes per lane.
  static __device__ __forceinline__ void epilogue_lines(const TiledCtx& c, bf16_t* __restrict__ out, const TileLoc& loc,
                                                        const Sums& acc, u32x4* lds) {
    static_assert(NWV % 2 == 0 && (NWV / 2) * FM * 32 * 8 <= LDS_VEC, "the staging blocks must fit the activation ring");
    const int row_first = loc.row_first, m_rows = loc.m_rows, nt = loc.nt;
    const int n_out = c.ffn;
    const int m0 = loc.mt * MSTRIDE;
    const int tid = threadIdx.x, wave = tid / 64, lane = tid % 64;
    const int half = lane / 32, col = lane % 32;
    bf16_t* block = (bf16_t*)(lds + (wave / 2) * FM * 32 * 8);  // [FM * 32 rows][64 columns]
    block_barrier();  // every wave has read its last activation fragments
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int row = i * 32 + (r / 4) * 8 + half * 4 + (r % 4);
        block[row * 64 + (wave % 2) * 32 + col] = f32_to_bf16(silu_f32(acc[i][0][r]) * acc[i][1][r]);
      }
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
    block_barrier();
    const int f = nt * (BN / 2) + (wave / 2) * 64 + (lane % 8) * 8;
#pragma unroll
    for (int k = 0; k < 2 * FM; ++k) {
      const int row = (wave % 2) * FM * 16 + k * 8 + lane / 8;
      const u32x4 v = *(const u32x4*)(block + row * 64 + (lane % 8) * 8);
      const int m = m0 + row;
      if (m < m_rows && f < n_out) *(u32x4*)(out + (size_t)(row_first + m) * n_out + f) = v;
    }
  }
  // Integer sums times the scales of their rows and columns.  row_scales: per input row; they reach the lanes through LDS, four
  // consecutive rows at a time (a lane's 16 sums per fragment are four runs of four rows).  col_scales: of the lane's column of
  // each group.
  static __device__ __forceinline__ void scale_sums(const TiledCtx& c, const TileLoc& loc, const float* __restrict__ row_scales,
                                                    const float (&col_scales)[FN], const Acc& acc, u32x4* lds, Sums& sums) {
    const int tid = threadIdx.x, half = tid % 64 / 32;
    const int m0 = loc.mt * MSTRIDE;
    float* staged = (float*)lds;
    block_barrier();  // every wave has read its last activation fragments
    if (tid < FM * 32) {
      int row = loc.row_first + (m0 + tid < loc.m_rows ? m0 + tid : loc.m_rows - 1);
      if (GATEUP && c.row_map) row = div_by_map(c, c.row_map[row]);
      staged[tid] = row_scales[row];
    }
    static_assert(FM * 32 <= THREADS, "a thread per row");
    __syncthreads();
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x4_t rs = *(const f32x4_t*)(staged + i * 32 + q * 8 + half * 4);
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
          for (int t = 0; t < 4; ++t) sums[i][j][q * 4 + t] = i8_product(acc[i][j][q * 4 + t], rs[t], col_scales[j]);
      }
    __builtin_amdgcn_s_waitcnt(0xC07F);  // the scales are in registers before the barrier after which others write over them
  }
  // Gate/up with two weight groups per wave and h in fp32: the wave's 32 columns are a whole line, which each store fills
  // for two rows.
  static __device__ __forceinline__ void epilogue_h_f32(const TiledCtx& c, float* __restrict__ out, const TileLoc& loc,
                                                        const Sums& acc) {
    const int n_out = c.ffn;
    const int m0 = loc.mt * MSTRIDE;
    const int tid = threadIdx.x, wave = tid / 64, lane = tid % 64;
    const int half = lane / 32, col = lane % 32;
    const int f = loc.nt * (BN / 2) + wave * 32 + col;
    float* at = out + (size_t)loc.row_first * n_out + f;
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int m = m0 + i * 32 + (r / 4) * 8 + half * 4 + (r % 4);
        if (m < loc.m_rows && f < n_out) at[(size_t)m * n_out] = silu_f32(acc[i][0][r]) * acc[i][1][r];
      }
  }
  // Down projection with two weight groups per wave: the wave's 64 columns are one 128-byte line per row.  The wave
  // turns its accumulators into rows in a block of its own in the idle activation ring, two fragments (64 rows) at a
  // time, and stores whole lines, 16 bytes per lane.  (LDS serves a wave's accesses in order: no barrier in between.)
  static __device__ __forceinline__ void epilogue_lines_down(const TiledCtx& c, bf16_t* __restrict__ out, const TileLoc& loc,
                                                             const Sums& acc, u32x4* lds) {
    static_assert(NWV * 64 * 8 <= LDS_VEC, "the staging blocks must fit the activation ring");
    const int row_first = loc.row_first, m_rows = loc.m_rows, nt = loc.nt;
    const int n_out = c.hidden;
    const int m0 = loc.mt * MSTRIDE;
    const int tid = threadIdx.x, wave = tid / 64, lane = tid % 64;
    const int half = lane / 32, col = lane % 32;
    bf16_t* block = (bf16_t*)(lds + wave * 64 * 8);  // [64 rows][64 columns]
    const int n = nt * BN + wave * 64 + (lane % 8) * 8;
    block_barrier();  // every wave has read its last activation fragments
#pragma unroll
    for (int pass = 0; pass < (FM + 1) / 2; ++pass) {
#pragma unroll
      for (int ii = 0; ii < 2; ++ii) {
        const int i = pass * 2 + ii;
        if (i < FM) {
#pragma unroll
          for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r)
              block[(ii * 32 + (r / 4) * 8 + half * 4 + (r % 4)) * 64 + j * 32 + col] = f32_to_bf16(acc[i][j][r]);
        }
      }
      __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int row = k * 8 + lane / 8;
        if (pass * 2 + row / 32 < FM) {  // uniform per k: the second fragment of the last pass may not exist
          const u32x4 v = *(const u32x4*)(block + row * 64 + (lane % 8) * 8);
          const int m = m0 + pass * 64 + row;
          if (m < m_rows && n < n_out) *(u32x4*)(out + (size_t)(row_first + m) * n_out + n) = v;
        }
      }
      __builtin_amdgcn_s_waitcnt(0xC07F);  // the rows are in registers before the next pass overwrites the block
    }
  }
  // The two epilogues of a block that goes on to another tile (transposed product, TR).  The staging blocks lie in a
  // region of their own (`staging`: the activation ring is already being filled for the next tile) and the stores are
  // issued by hand; the previous tile's reads of the staging blocks are separated from these writes by that tile's
  // whole K loop.  The accumulators are pinned where they are on entry: without that the compiler starts to copy them
  // out of the second register file before the next tile's loads are issued, into registers it frees by moving
  // others; the scheduling fences keep the tile's arithmetic from spreading over the registers of loads in flight.
  // Staging blocks are rows of 128 bytes in eight 16-byte slots; row r keeps slot s at s ^ ((r / 2) % 8), so that the 8-byte writes of a wave (32 rows, two
  // neighbouring half slots each) and the 16-byte reads (8 rows x 8 slots) both spread over all banks.
  static __device__ __forceinline__ uint32_t staged_at(int row, int slot) {
    return (uint32_t)(row * 128 + ((slot ^ ((row >> 1) & 7)) << 4));
  }
  static __device__ __forceinline__ void epilogue_lines_walk_tr(const TiledCtx& c, bf16_t* __restrict__ out, const TileLoc& loc,
                                                                Acc& acc, u32x4* staging, int wave, int lane) {
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) asm volatile("" : "+a"(acc[i][j]));
    const int row_first = loc.row_first, m_rows = loc.m_rows, nt = loc.nt;
    const int n_out = c.ffn;
    const int m0 = loc.m0;
    const int half = lane / 32, rl = lane % 32;
    char* block = (char*)(staging + (wave / 2) * FM * 32 * 8);  // [FM * 32 rows][64 columns] of waves 2p, 2p+1
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      const int row = i * 32 + rl;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float v[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) v[t] = silu_f32(acc[i][0][q * 4 + t]) * acc[i][1][q * 4 + t];
        uint2 pk;
        pk.x = f32_to_bf16_pair(v[0], v[1]);
        pk.y = f32_to_bf16_pair(v[2], v[3]);
        *(uint2*)(block + staged_at(row, (wave % 2) * 4 + q) + half * 8) = pk;
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
    block_barrier();
    // (the reads of up to four rows are issued together, then their stores: one trip to LDS per batch, not per store)
    const int f = nt * (BN / 2) + (wave / 2) * 64 + (lane % 8) * 8;
#pragma unroll
    for (int k0 = 0; k0 < 2 * FM; k0 += 4) {
      u32x4 v[4];
#pragma unroll
      for (int k = k0; k < k0 + 4 && k < 2 * FM; ++k)
        v[k - k0] = *(const u32x4*)(block + staged_at((wave % 2) * FM * 16 + k * 8 + lane / 8, lane % 8));
      __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int k = k0; k < k0 + 4 && k < 2 * FM; ++k) {
        const int m = m0 + (wave % 2) * FM * 16 + k * 8 + lane / 8;
        if (m < m_rows && f < n_out) store_16(out + (size_t)(row_first + m) * n_out + f, v[k - k0]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  static __device__ __forceinline__ void epilogue_lines_down_walk_tr(const TiledCtx& c, bf16_t* __restrict__ out,
                                                                     const TileLoc& loc, Acc& acc, u32x4* staging, int wave,
                                                                     int lane) {
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) asm volatile("" : "+a"(acc[i][j]));
    const int row_first = loc.row_first, m_rows = loc.m_rows, nt = loc.nt;
    const int n_out = c.hidden;
    const int m0 = loc.m0;
    const int half = lane / 32, rl = lane % 32;
    char* block = (char*)(staging + wave * 64 * 8);  // two [32 rows][64 columns] halves, the wave's own
    const int n = nt * BN + wave * 64 + (lane % 8) * 8;
    // Fragment by fragment through the two halves in turn: the next fragment is converted and written while the reads
    // of this one are on their way, so the trips to LDS overlap the conversions instead of following them.  (LDS
    // serves a wave's accesses in order: the reads see the writes before them, and a half is written again only
    // after its reads have come back, two fragments later.)
    auto write_fragment = [&](int i) {
      const int row = (i % 2) * 32 + rl;
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          uint2 pk;
          pk.x = f32_to_bf16_pair(acc[i][j][q * 4 + 0], acc[i][j][q * 4 + 1]);
          pk.y = f32_to_bf16_pair(acc[i][j][q * 4 + 2], acc[i][j][q * 4 + 3]);
          *(uint2*)(block + staged_at(row, j * 4 + q) + half * 8) = pk;
        }
    };
    write_fragment(0);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      u32x4 v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = *(const u32x4*)(block + staged_at((i % 2) * 32 + k * 8 + lane / 8, lane % 8));
      __builtin_amdgcn_sched_barrier(0);
      if (i + 1 < FM) write_fragment(i + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int m = m0 + i * 32 + k * 8 + lane / 8;
        if (m < m_rows && n < n_out) store_16(out + (size_t)(row_first + m) * n_out + n, v[k]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  // The same for integer sums (NUM = StreamI8): times the scales of their rows and columns, which lie in LDS (row_scales: the
  // tile's rows; col_scales: the wave's 64 packed columns), then SwiGLU into fp32 rows of 32 columns, or bfloat16 rows of 64:
  // 128 bytes of a row per wave in both.
  template <class OUT>
  static __device__ __forceinline__ void epilogue_walk_i8(const TiledCtx& c, OUT* __restrict__ out, const TileLoc& loc, Acc& acc,
                                                          u32x4* staging, const float* row_scales, const float* col_scales, int wave,
                                                          int lane) {
    static_assert(GATEUP == (sizeof(OUT) == 4), "h in fp32, o_perm in bfloat16");
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) asm volatile("" : "+a"(acc[i][j]));
    const int row_first = loc.row_first, m_rows = loc.m_rows, nt = loc.nt;
    const int n_out = GATEUP ? c.ffn : c.hidden;
    const int m0 = loc.m0;
    const int half = lane / 32, rl = lane % 32;
    char* block = (char*)(staging + wave * 64 * 8);  // two [32 rows][128 bytes] halves, the wave's own
    constexpr int PER = 16 / sizeof(OUT);
    const int n = nt * (GATEUP ? BN / 2 : BN) + wave * 8 * PER + (lane % 8) * PER;
    f32x4_t cs[FN][4];
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) cs[j][q] = *(const f32x4_t*)(col_scales + j * 32 + q * 8 + half * 4);
    auto write_fragment = [&](int i) {
      const int row = (i % 2) * 32 + rl;
      const float rs = row_scales[i * 32 + rl];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        f32x4_t v[FN];
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
          for (int t = 0; t < 4; ++t) v[j][t] = i8_product(acc[i][j][q * 4 + t], rs, cs[j][q][t]);
        if constexpr (GATEUP) {
#pragma unroll
          for (int t = 0; t < 4; ++t) v[0][t] = silu_f32(v[0][t]) * v[1][t];
          *(f32x4_t*)(block + staged_at(row, q * 2 + half)) = v[0];
        } else {
#pragma unroll
          for (int j = 0; j < FN; ++j) {
            uint2 pk;
            pk.x = f32_to_bf16_pair(v[j][0], v[j][1]);
            pk.y = f32_to_bf16_pair(v[j][2], v[j][3]);
            *(uint2*)(block + staged_at(row, j * 4 + q) + half * 8) = pk;
          }
        }
      }
    };
    write_fragment(0);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      u32x4 v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = *(const u32x4*)(block + staged_at((i % 2) * 32 + k * 8 + lane / 8, lane % 8));
      __builtin_amdgcn_sched_barrier(0);
      if (i + 1 < FM) write_fragment(i + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int m = m0 + i * 32 + k * 8 + lane / 8;
        if (m < m_rows && n < n_out) store_16(out + (size_t)(row_first + m) * n_out + n, v[k]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  // Down projection with one weight group per wave: a wave's 32 columns are a quarter of a line.  The block collects
  // the tile's bf16 results in the idle activation ring, [rows][32 * NWV columns], and every thread stores whole
  // 16-byte pieces of whole lines.
  static __device__ __forceinline__ void epilogue_lines_block(const TiledCtx& c, bf16_t* __restrict__ out, const TileLoc& loc,
                                                              const Sums& acc, u32x4* lds) {
    static_assert(FM * 32 * BN * 2 <= LDS_VEC * 16, "the tile's results must fit the activation ring");
    const int row_first = loc.row_first, m_rows = loc.m_rows, nt = loc.nt;
    const int n_out = c.hidden;
    const int m0 = loc.mt * MSTRIDE;
    const int tid = threadIdx.x, wave = tid / 64, lane = tid % 64;
    const int half = lane / 32, col = lane % 32;
    bf16_t* staged = (bf16_t*)lds;
    block_barrier();  // every wave has read its last activation fragments
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        staged[(i * 32 + (r / 4) * 8 + half * 4 + (r % 4)) * BN + wave * 32 + col] = f32_to_bf16(acc[i][0][r]);
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
    block_barrier();
#pragma unroll
    for (int id = tid; id < FM * 32 * BN / 8; id += THREADS) {
      const int row = id / (BN / 8), cc = (id % (BN / 8)) * 8;
      const int m = m0 + row, n = nt * BN + cc;
      if (m < m_rows && n < n_out)
        *(u32x4*)(out + (size_t)(row_first + m) * n_out + n) = *(const u32x4*)(staged + row * BN + cc);
    }
  }
};

// Blocks that go from tile to tile (StreamTile::steps_walk): first loads and copies of a block's first tile (fm copies per thread and stage, into stages 0 and 1)
template <class TILE>
__device__ __forceinline__ void walk_issue_prologue(const typename TILE::RowSrc& src, uint32_t lds0, int wave, int fm,
                                                    u32x4 (&ring)[8][2]) {
#pragma unroll
  for (int s = 0; s < 8; ++s)
#pragma unroll
    for (int j = 0; j < 2; ++j) ring[s][j] = src.b_at(j, (size_t)s * 64);
#pragma unroll
  for (int st = 0; st < 2; ++st)
#pragma unroll
    for (int op = 0; op < 7; ++op)
      if (op < fm) TILE::copy_to_stage(src.a_at(op, (size_t)st * 8), lds0, wave, st, op);  // uniform
}
// every vector-memory operation of the thread has completed; the operands tie the weight ring to the wait
__device__ __forceinline__ void walk_wait_ring(u32x4 (&r)[8][2]) {
  asm volatile("s_waitcnt vmcnt(0)"
               : "+v"(r[0][0]), "+v"(r[0][1]), "+v"(r[1][0]), "+v"(r[1][1]), "+v"(r[2][0]), "+v"(r[2][1]), "+v"(r[3][0]),
                 "+v"(r[3][1]), "+v"(r[4][0]), "+v"(r[4][1]), "+v"(r[5][0]), "+v"(r[5][1]), "+v"(r[6][0]), "+v"(r[6][1]),
                 "+v"(r[7][0]), "+v"(r[7][1])
               :
               : "memory");
}

}  // namespace hmoe
