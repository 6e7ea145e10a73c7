// bf16 MFMA GEMM tiles for gfx950: what a workgroup does for a tile of C[i][j] = sum_r X(i, r) * Y(r, j), fp32 accumulation.
//
// A workgroup of 4 waves owns a tile of C, 256 x 256 elements at most; wave (wi, wj) owns a quarter of
// it as accumulator blocks of the 32x32x16 MFMA (256 accumulator registers and one wave per SIMD for the large
// tile), computed transposed (the MFMA's row index is j) so that a lane owns one row i of C and stores
// consecutive j.  The contraction runs in stages of 32 or 64: each stage's X and Y tiles are copied
// global -> LDS asynchronously AHEAD stages before their use (the scheme of the attention kernels, deeper
// because a stage is shorter).  An operand whose contraction index is contiguous in memory sits in LDS
// as [outer][STEP] and is read with ds_read_b128; one whose contraction index is the row of the
// stored matrix sits as [STEP][128] tiles and is read with the transposing LDS read.  Operand reads are issued
// one sub-step (16 contraction indices) ahead.
#pragma once
#include "helix_common.hpp"
#include "kernels.hpp"
#include <type_traits>

namespace helix {
namespace {

constexpr int kWaves = 4;                     // 2 x 2 waves

// Geometry of a workgroup tile: TI x TJ elements of C, contraction in stages of STEP, NST stage buffers.
// A wave owns TI/2 x TJ/2 elements.
template <int TI_, int TJ_, int STEP_, int NST_>
struct Tile {
  static constexpr int TI = TI_, TJ = TJ_, STEP = STEP_, NST = NST_;
  static constexpr int BI = TI / 64, BJ = TJ / 64;   // 32-wide blocks per wave in i and in j
  static constexpr int XBYTES = TI * STEP * 2, YBYTES = TJ * STEP * 2;
  static constexpr int STAGE = XBYTES + YBYTES;
  static constexpr int AHEAD = NST - 1;              // a stage's copy is issued this many iterations before its use
  static constexpr int LDS = NST * STAGE;
  static constexpr int WORKGROUPS = LDS > 80 * 1024 ? 1 : 2;   // on a compute unit
};
using Tile256 = Tile<256, 256, 32, 5>;        // 160 KB of LDS: one workgroup per compute unit
using Tile128 = Tile<128, 128, 32, 5>;        // 80 KB: two
using Tile64ShortStages = Tile<64, 64, 32, 8>;
using Tile64 = Tile<64, 64, 64, 5>;           // 80 KB: two

__device__ __forceinline__ void copy_16_bytes_per_lane(uint32_t lane_byte_off, const __bf16* base, uint32_t lds_dst) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" :: "v"(lane_byte_off), "s"(base), "s"(lds_dst) : "memory");
}

// Operand whose stored rows are the outer index (i or j) and whose contraction index is
// contiguous: LDS tile [OUTER][STEP].  Rows past the edge of the matrix are clamped to its last row once,
// here, because the outer index of a workgroup never changes: a stage's copy is nothing but its copy instructions.
template <int OUTER, int STEP>
struct ContiguousOperand {
  using Loader = TileLoader<STEP, OUTER, kWaves>;
  static constexpr int DMA = Loader::N;              // copy instructions per wave and stage
  uint32_t off[DMA];
  const __bf16* ptr;                                 // element (outer0, first contraction index of the next stage to copy)
  uint32_t piece0;                                   // this wave's first 1 KB piece of the LDS tile
  __device__ __forceinline__ ContiguousOperand(const __bf16* p, long long ld, int outer0, int outer_n, int r0, int lane, int wave)
      : piece0((uint32_t)wave * 1024) {
    const Loader loader(lane, wave, (int)ld);
    const int last = outer_n - 1 - outer0;
#pragma unroll
    for (int i = 0; i < DMA; i++) {
      const int row = (wave + kWaves * i) * Loader::ROWS_PER_KB + loader.lane_row;
      off[i] = loader.off[i] - (uint32_t)(row > last ? row - last : 0) * loader.row_bytes;
    }
    ptr = uniform_ptr(p + (size_t)outer0 * ld + r0);
  }
  // Copy instruction i of the next stage; `next` after the last one.
  __device__ __forceinline__ void copy(int i, uint32_t lds) const { copy_16_bytes_per_lane(off[i], ptr, lds + piece0 + i * kWaves * 1024); }
  __device__ __forceinline__ void next() { ptr += STEP; }
  // lane addresses of the operand of a 32-row block starting at tile row blk0, one per sub-step of 16
  static constexpr int NADDR = STEP / 16;
  __device__ __forceinline__ static void addresses(int lane, int blk0, uint32_t (&a)[NADDR]) {
    const int row = blk0 + (lane & 31), half = lane >> 5;
#pragma unroll
    for (int ks = 0; ks < NADDR; ks++) a[ks] = lds_chunk_off<STEP>(row, 2 * ks + half);
  }
  __device__ __forceinline__ static bf16x8 read(const uint32_t (&a)[NADDR], int ks) { return lds_b128(a[ks], 0); }
};

// Operand whose stored rows are the contraction index: LDS holds [STEP][W] tiles side by side (W = 128, or 64
// for 64 outer indices), read with the transposing LDS read so that contraction slot e of lane half h is row 8h + e.
template <int OUTER, int STEP, int W_ = (OUTER < 128 ? OUTER : 128)>
struct TransposedOperand {
  static constexpr int W = W_, SUBS = OUTER / W;
  using Loader = TileLoader<W, STEP, kWaves>;
  static constexpr int DMA = SUBS * Loader::N;
  uint32_t off[Loader::N];
  const __bf16* ptr[SUBS];   // element (first contraction index of the next stage, first outer index of the sub-tile)
  uint32_t piece0;
  long long stage_elems;
  __device__ __forceinline__ TransposedOperand(const __bf16* p, long long ld, int outer0, int outer_n, int r0, int lane, int wave)
      : piece0((uint32_t)wave * 1024), stage_elems(STEP * ld) {
    const Loader loader(lane, wave, (int)ld);
#pragma unroll
    for (int i = 0; i < Loader::N; i++) off[i] = loader.off[i];
#pragma unroll
    for (int b = 0; b < SUBS; b++)   // a sub-tile past the edge falls back to the first one; its results are not stored
      ptr[b] = uniform_ptr(p + (size_t)r0 * ld + (outer0 + b * W < outer_n ? outer0 + b * W : outer0));
  }
  __device__ __forceinline__ void copy(int i, uint32_t lds) const {
    const int sub = i / Loader::N, piece = i % Loader::N;
    copy_16_bytes_per_lane(off[piece], ptr[sub], lds + sub * (W * STEP * 2) + piece0 + piece * kWaves * 1024);
  }
  __device__ __forceinline__ void next() {
#pragma unroll
    for (int b = 0; b < SUBS; b++) ptr[b] += stage_elems;
  }
  // The next stage ends with the row `last` of it: later rows are read as that one (their products are with zeros).
  __device__ __forceinline__ void clamp(long long ld, int lane, int wave, int last) {
    const Loader loader(lane, wave, (int)ld);
#pragma unroll
    for (int i = 0; i < Loader::N; i++) {
      const int row = (wave + kWaves * i) * Loader::ROWS_PER_KB + loader.lane_row;
      off[i] -= (uint32_t)(row > last ? row - last : 0) * loader.row_bytes;
    }
  }
  static constexpr int NADDR = 2;
  __device__ __forceinline__ static void addresses(int lane, int blk0, uint32_t (&a)[NADDR]) {
    const int i = lane & 15;
    const int c = (blk0 & (W - 1)) + ((lane >> 4) & 1) * 16 + (i & 3) * 4;
    const int r = (lane >> 5) * 8 + (i >> 2);
    const int sub = (blk0 / W) * (W * STEP * 2);
    a[0] = sub + lds_chunk_off<W>(r, c >> 3) + (c & 7) * 2;
    a[1] = sub + lds_chunk_off<W>(r + 4, c >> 3) + (c & 7) * 2;
  }
  // rows 16*ks + ...: the swizzle has period 16 in the row, so the sub-step is an immediate
  __device__ __forceinline__ static bf16x8 read(const uint32_t (&a)[NADDR], int ks) { return lds_tr_pair(a[0], a[1], ks * 16 * W * 2); }
};

// The fp32 counterparts of put_rows and store_rows in helix_common.hpp: 32 rows of W floats in this wave's own LDS, 16-byte
// chunks permuted by the row so that neither access has bank conflicts.
template <int W>
__device__ __forceinline__ int float_chunk_off(int row, int chunk) {
  return row * (W * 4) + ((chunk ^ (W == 32 ? (row >> 1) & 7 : row & 15)) << 4);
}
template <int W>
__device__ __forceinline__ void put_rows(char* tile, int lane, int block, const f32x16& acc, float) {
  pin(lane);
#pragma unroll
  for (int g = 0; g < 4; g++) {
    const f32x4 x = {acc[4 * g], acc[4 * g + 1], acc[4 * g + 2], acc[4 * g + 3]};
    *reinterpret_cast<f32x4*>(tile + float_chunk_off<W>(lane & 31, 8 * block + 2 * g + (lane >> 5))) = x;
  }
}
template <int W>
__device__ __forceinline__ void put_rows(char* tile, int lane, int block, const f32x16& acc, __bf16) { helix::put_rows<W>(tile, lane, block, acc); }
// One 32 x 32 block from the lanes, 16 bytes at a time.
__device__ __forceinline__ void store_block(float* row, int half, const f32x16& acc) {
#pragma unroll
  for (int g = 0; g < 4; g++) {
    const f32x4 x = {acc[4 * g], acc[4 * g + 1], acc[4 * g + 2], acc[4 * g + 3]};
    *reinterpret_cast<f32x4*>(row + 8 * g + 4 * half) = x;
  }
}
__device__ __forceinline__ void store_block(__bf16* row, int half, const f32x16& acc) {
  for_each_chunk(half, acc, [&](int chunk, const u32x4& x) __attribute__((always_inline)) { *reinterpret_cast<u32x4*>(row + 8 * chunk) = x; });
}
// Stores the tile; `rows` of its rows and `cols` of its columns (a multiple of 32) exist.  ONCE: the caches need not keep them.
template <int W, bool ONCE = false, typename T>
__device__ __forceinline__ void store_rows(const char* tile, int lane, T* row0, long long row_stride, int rows, int cols) {
  constexpr int PER_CHUNK = 16 / sizeof(T), CH = W / PER_CHUNK, PER = 64 / CH;   // elements of a chunk, chunks of a row, rows of a piece
  pin(lane);
  const int r0 = lane / CH, chunk = lane % CH;
  const uint32_t lane_off = (uint32_t)(r0 * (int)row_stride + chunk * PER_CHUNK) * (uint32_t)sizeof(T);   // below 2^30: the row pitch is bounded
#pragma unroll
  for (int i = 0; i < 32 / PER; i++) {
    const int r = i * PER + r0;
    const int off = sizeof(T) == 4 ? float_chunk_off<W>(r, chunk) : lds_chunk_off<W>(r, chunk);
    const u32x4 x = *reinterpret_cast<const u32x4*>(tile + off);
    char* const rows_i = const_cast<char*>(uniform_ptr(reinterpret_cast<const char*>(row0 + (size_t)(i * PER) * row_stride)));
    if (r < rows && chunk * PER_CHUNK < cols) {
      if constexpr (ONCE) __builtin_nontemporal_store(x, reinterpret_cast<u32x4*>(rows_i + lane_off));
      else *reinterpret_cast<u32x4*>(rows_i + lane_off) = x;
    }
  }
}
// All but the N newest vector memory operations of this wave are done, and every wave of the workgroup has got here.
// LDS reads may stay in flight across it: the reads of a stage are consumed by MFMAs of that stage's own iteration, and
// its buffer is not copied into before the one after.
template <int N>
__device__ __forceinline__ void stage_barrier() {
  wait_tile_loads_except<N>();
  asm volatile("s_barrier" ::: "memory");
}

// The place of tile t in a grid of tiles: all column tiles of a row tile one after the other, or of `side` row tiles together, column by column.  With more
// column tiles than an XCD has compute units the workgroups that run at the same time then share panels of both operands: `side` rows x 32 / side
// columns of tiles read side + 32 / side panels instead of 33.
__device__ __forceinline__ void place_tile(int t, int tiles_i, int tiles_j, int side, int& ti, int& tj) {
  if (side < 2) {
    ti = t / tiles_j;
    tj = t - ti * tiles_j;
    return;
  }
  const int first = t / (side * tiles_j) * side, rows = tiles_i - first < side ? tiles_i - first : side;
  t -= first * tiles_j;
  tj = t / rows;
  ti = first + t - tj * rows;
}

// One product C = X Y, with its tiles and the parts its contraction is cut into.
template <typename OutT>
struct Gemm {
  const __bf16 *X, *Y;
  OutT* C;
  long long ldx, ldy, ldc, part_stride;   // a part's partial result goes to C + part * part_stride
  int I, J, R, tiles_i, tiles_j, parts, r_per_part;
  int side;   // of a RAGGED product: row tiles side by side in the order of tiles (below 2: one after the other)
  // Workgroups of a part: all tiles, rounded up so that the XCD of a workgroup is its number mod 8 in every part.
  __host__ __device__ int blocks_per_part() const { return (tiles_i * tiles_j + 7) & ~7; }
};

// Where block b of a wave's BJ blocks of columns lies in the workgroup's tile: side by side.
struct BlocksSideBySide {
  __device__ __forceinline__ static constexpr int column(int BJ, int wj, int b) { return 32 * (BJ * wj + b); }
};

// What a wave asks of memory when the last copies of its stages have landed: loads that nothing waits for before the sums are complete.
struct NothingBeforeTheEnd {
  __device__ __forceinline__ void operator()() const {}
};

// The sums of a wave over nk stages.  RAGGED: the last stage of X (stored by rows of the contraction index, `ldx` elements apart) ends with its row `last`.
template <typename G, typename XOp, typename YOp, typename YBlocks, bool RAGGED, typename Before = NothingBeforeTheEnd>
__device__ __forceinline__ void gemm_sums(XOp& xsrc, YOp& ysrc, int nk, uint32_t base, int lane, int w, f32x16 (&acc)[G::BJ][G::BI], long long ldx = 0, int last = 0,
                                          Before&& before_the_end = Before()) {
  constexpr int BI = G::BI, BJ = G::BJ, NS = G::STEP / 16, AHEAD = G::AHEAD, NST = G::NST, STAGE = G::STAGE;
  const int wi = w & 1, wj = w >> 1;
  constexpr int NDMA = XOp::DMA + YOp::DMA;
  auto copy = [&](int n, uint32_t lds) __attribute__((always_inline)) {   // copy instruction n of the next stage
    if (n < XOp::DMA) xsrc.copy(n, lds);
    else ysrc.copy(n - XOp::DMA, lds + G::XBYTES);
  };
#pragma unroll
  for (int k = 0; k < AHEAD; k++)
    if (k < nk) {
      if constexpr (RAGGED)
        if (k == nk - 1) xsrc.clamp(ldx, lane, w, last);
#pragma unroll
      for (int n = 0; n < NDMA; n++) copy(n, base + k * STAGE);
      xsrc.next();
      ysrc.next();
    }
  // iteration k reads stages k and k+1: the first two must be complete, the others may still fly
  if (nk >= AHEAD) stage_barrier<(AHEAD - 2) * NDMA>();   // all AHEAD copies are out: the newest may fly
  else stage_barrier<0>();

  uint32_t xa[BI][XOp::NADDR], ya[BJ][YOp::NADDR];
#pragma unroll
  for (int b = 0; b < BI; b++) {
    XOp::addresses(lane, 32 * (BI * wi + b), xa[b]);
#pragma unroll
    for (int e = 0; e < XOp::NADDR; e++) xa[b][e] += base;
  }
#pragma unroll
  for (int b = 0; b < BJ; b++) {
    YOp::addresses(lane, YBlocks::column(BJ, wj, b), ya[b]);
#pragma unroll
    for (int e = 0; e < YOp::NADDR; e++) ya[b][e] += base + G::XBYTES;
  }

#pragma unroll
  for (int jb = 0; jb < BJ; jb++)
#pragma unroll
    for (int ib = 0; ib < BI; ib++)
#pragma unroll
      for (int e = 0; e < 16; e++) acc[jb][ib][e] = 0.f;

  // Operands are read a sub-step ahead into the other of two sets.  With a single MFMA to a sub-step (the 64 x 64 tile) that is not
  // ahead enough: there a set for every sub-step is refilled behind its MFMA, a whole stage ahead (64 tokens x 2048 x 768 forward
  // 8.8 -> 7.8 us; the larger tiles lose 5 to 10 % that way, by 14 registers more and reads in bursts).
  constexpr bool STAGE_AHEAD = BI * BJ == 1;
  constexpr int SETS = STAGE_AHEAD ? NS : 2;
  bf16x8 xo[SETS][BI], yo[SETS][BJ];
#pragma unroll
  for (int ks = 0; ks < (STAGE_AHEAD ? NS : 1); ks++) {
#pragma unroll
    for (int b = 0; b < BI; b++) xo[ks][b] = XOp::read(xa[b], ks);
#pragma unroll
    for (int b = 0; b < BJ; b++) yo[ks][b] = YOp::read(ya[b], ks);
  }

  // One stage: NS sub-steps of BI * BJ MFMAs; behind each MFMA its share of the operand reads (of the next sub-step, in the last one from
  // the next buffer; or of the same sub-step of the next stage) and of the copies of stage k + AHEAD, which replaces stage k - 1.
  int buf = 0;
  auto stage = [&](auto copying, auto reading) __attribute__((always_inline)) {
    constexpr bool COPY = decltype(copying)::value, READ = decltype(reading)::value;
    constexpr int MM = BI * BJ, SLOTS = NS * MM, READS = BI + BJ;
    const int step = (buf == NST - 1) ? -(NST - 1) * STAGE : STAGE;
    const uint32_t dst = base + (buf == 0 ? NST - 1 : buf - 1) * STAGE;
#pragma unroll
    for (int ks = 0; ks < NS; ks++) {
      if (ks == (STAGE_AHEAD ? 0 : NS - 1)) {
#pragma unroll
        for (int b = 0; b < BI; b++)
#pragma unroll
          for (int e = 0; e < XOp::NADDR; e++) xa[b][e] += step;
#pragma unroll
        for (int b = 0; b < BJ; b++)
#pragma unroll
          for (int e = 0; e < YOp::NADDR; e++) ya[b][e] += step;
      }
#pragma unroll
      for (int m = 0; m < MM; m++) {
        const int jb = m / BI, ib = m % BI, set = STAGE_AHEAD ? ks : ks & 1;
        acc[jb][ib] = mfma32(yo[set][jb], xo[set][ib], acc[jb][ib]);
        // reads go behind the first MFMAs of a sub-step, one each where there are enough of them
        const int to = STAGE_AHEAD ? ks : (ks & 1) ^ 1, next_ks = STAGE_AHEAD ? ks : (ks + 1) % NS;
#pragma unroll
        for (int q = 0; q < READS; q++) {
          if (!READ || (MM >= READS ? q : q * MM / READS) != m) continue;
          if (q < BI) xo[to][q] = XOp::read(xa[q], next_ks);
          else yo[to][q - BI] = YOp::read(ya[q - BI], next_ks);
        }
        if constexpr (COPY) {
#pragma unroll
          for (int n = 0; n < NDMA; n++)
            if (n * SLOTS / NDMA == ks * MM + m) copy(n, dst);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    if constexpr (COPY) {
      xsrc.next();
      ysrc.next();
    }
    buf = (buf == NST - 1) ? 0 : buf + 1;
  };
  int k = 0;
  // stages up to k+2 must have landed before the next iteration starts (it reads k+1 and k+2);
  // the copies of stages k+3 .. k+AHEAD may stay in flight
  for (; k + AHEAD < nk; k++) {
    if constexpr (RAGGED)
      if (k + AHEAD == nk - 1) xsrc.clamp(ldx, lane, w, last);
    stage(std::true_type{}, std::true_type{});
    stage_barrier<(AHEAD - 2) * NDMA>();
  }
  if constexpr (std::is_same<typename std::decay<Before>::type, NothingBeforeTheEnd>::value) {
    for (; k < (STAGE_AHEAD ? nk - 1 : nk); k++) {
      stage(std::false_type{}, std::true_type{});
      stage_barrier<0>();
    }
  } else {
    // The loads go out behind the barrier that has waited for the last copies, all of them, and the barriers after it wait for no memory: which copies have landed does not
    // depend on how many load instructions the compiler makes or where it puts them.
    static_assert(!STAGE_AHEAD, "the last stage is one of those below");
    stage(std::false_type{}, std::true_type{});
    stage_barrier<0>();
    before_the_end();
    for (k++; k < nk; k++) {
      stage(std::false_type{}, std::true_type{});
      asm volatile("s_barrier" ::: "memory");
    }
  }
  // The last stage has nothing to read ahead and, as the tile leaves from the registers, nobody to wait for: its reads held up the workgroup beside this one (forward of
  // 12480 x 128 x 128 3.39 -> 3.27 us, 4256 x 512 x 256 4.91 -> 4.84).
  if constexpr (STAGE_AHEAD) stage(std::false_type{}, std::false_type{});
}

// The tile of workgroup `block`.
template <typename G, bool X_ROWS_ARE_R, bool Y_ROWS_ARE_R, typename OutT, bool RAGGED = false>
__device__ __forceinline__ void gemm_block(int block, const Gemm<OutT>& g) {
  using XOp = typename std::conditional<X_ROWS_ARE_R, TransposedOperand<G::TI, G::STEP>, ContiguousOperand<G::TI, G::STEP>>::type;
  using YOp = typename std::conditional<Y_ROWS_ARE_R, TransposedOperand<G::TJ, G::STEP>, ContiguousOperand<G::TJ, G::STEP>>::type;
  constexpr int BI = G::BI, BJ = G::BJ;
  extern __shared__ __align__(16) char smem[];

  // workgroup id mod 8 is the XCD: each XCD takes a contiguous run of tiles, all column tiles of a row tile
  // one after the other, so an X panel reaches one L2 only
  const int per_part = g.blocks_per_part();
  // (one part, as in every forward: no division in front of the first copies, 0.12 us of a short call's 2.6)
  const int part = g.parts == 1 ? 0 : block / per_part, n = block - part * per_part;
  const int t = (n & 7) * (per_part >> 3) + (n >> 3);
  if (t >= g.tiles_i * g.tiles_j) return;
  int ti, tj;
  place_tile(t, g.tiles_i, g.tiles_j, RAGGED ? g.side : 1, ti, tj);
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wi = w & 1, wj = w >> 1;
  const int i0 = ti * G::TI, j0 = tj * G::TJ;
  const uint32_t base = lds_base(smem);

  const int r_begin = part * g.r_per_part;
  const int r_n = g.R - r_begin < g.r_per_part ? g.R - r_begin : g.r_per_part;
  const int nk = RAGGED ? (r_n + G::STEP - 1) / G::STEP : r_n / G::STEP;
  XOp xsrc(g.X, g.ldx, i0, g.I, r_begin, lane, w);
  YOp ysrc(g.Y, g.ldy, j0, g.J, r_begin, lane, w);
  f32x16 acc[BJ][BI];
  gemm_sums<G, XOp, YOp, BlocksSideBySide, RAGGED>(xsrc, ysrc, nk, base, lane, w, acc, g.ldx, RAGGED ? r_n - 1 - (nk - 1) * G::STEP : 0);

  // A lane owns row i of C: on the larger tiles 32 rows at a time go through LDS (free since the last barrier), this wave's part of it, and leave as whole
  // rows.  Stored from the lanes, 16 bytes of 32 or 64 rows an instruction, a 256 x 256 tile takes 4 to 5 us (fp32 7) in which the
  // compute unit has nothing else to do, of 21 us for a contraction of 768.
  if constexpr (BI * BJ == 16) {   // 256 sums stay in accumulator registers: moved to the others all at once, they push the lane's index out to memory
#pragma unroll
    for (int jb = 0; jb < BJ; jb++)
#pragma unroll
      for (int ib = 0; ib < BI; ib++) asm volatile("" : "+a"(acc[jb][ib]));
  }
  constexpr int W = 32 * BJ;
  const int i_wave = i0 + 32 * BI * wi, j_wave = j0 + W * wj;
  if constexpr (BI * BJ == 1) {   // one block to a wave: straight from the lanes is the shorter way (0.28 against 0.45 us at the end of a short call)
    const int half = lane >> 5, i = i_wave + (lane & 31);
    if (i < g.I && j_wave < g.J) store_block(g.C + (size_t)part * g.part_stride + (size_t)i * g.ldc + j_wave, half, acc[0][0]);
    return;
  }
  char* const out = smem + w * (32 * W * (int)sizeof(OutT));
#pragma unroll
  for (int ib = 0; ib < BI; ib++) {
#pragma unroll
    for (int jb = 0; jb < BJ; jb++) {
      put_rows<W>(out, lane, jb, acc[jb][ib], OutT());
      __builtin_amdgcn_sched_barrier(0);   // keeps the registers of one block in flight, not of all
    }
    store_rows<W>(out, lane, g.C + (size_t)part * g.part_stride + (size_t)(i_wave + 32 * ib) * g.ldc + j_wave, g.ldc,
                  g.I - i_wave - 32 * ib, g.J - j_wave);
    __builtin_amdgcn_sched_barrier(0);
  }
}

}  // namespace
}  // namespace helix
