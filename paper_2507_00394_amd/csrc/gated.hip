// The gated feed-forward projections, forward and backward, on the tiles of gemm.hpp:
//
//     [g u] = a w,   h = act(g) * u              a [M][K], w [K][2F]: the gate's F columns, then the other projection's
//     dg = dh * u * act'(g),   du = dh * act(g),   da = [dg du] w^T,   dw = a^T [dg du]
//
// Forward: a workgroup's tile holds the SAME columns of both projections, half of its columns from either half of w, and a wave its
// blocks of both, so that activation and product happen in registers: g and u reach memory only if the caller wants to keep them for the
// backward.  The backward either reads them (gated_grad_kernel, bound by bytes) or does the product again with an epilogue that turns g, u and dh
// into dg and du (recomputation: 4MKF FLOPs more, 2F elements a token less to keep).  da and dw are then the linear layer's two gradient products.
//
// dg and du are rounded to bf16, the type in which the matrix pipes take them; sums are fp32; dw is rounded to the weights' type once, from the whole fp32 sum.
#include "gated_math.hpp"
#include "gemm.hpp"
#include "helix_common.hpp"
#include "kernels.hpp"
#include <algorithm>

namespace helix {
namespace {

// Tiles of h: 256 x 128, 128 x 64 and 64 x 64 elements, twice as many columns of the product.
using Wide = Tile<256, 256, 32, 5>;     // 160 KB of LDS: one workgroup per compute unit
using Middle = Tile<128, 128, 32, 5>;   // 80 KB: two
using Short = Tile<64, 128, 32, 6>;     // 72 KB: two

// The columns j0 .. of either half of w, in sub-tiles of 64 columns.  Sub-tiles past the edge (F is a multiple of 64) fall back to the first one; their
// results are not stored.
template <int OUTER, int STEP>
struct GatedOperand : TransposedOperand<OUTER, STEP, 64> {
  using Base = TransposedOperand<OUTER, STEP, 64>;
  __device__ __forceinline__ GatedOperand(const __bf16* w, long long ldw, int j0, int F, int lane, int wave) : Base(w, ldw, 0, 64, 0, lane, wave) {
#pragma unroll
    for (int b = 0; b < Base::SUBS; b++) {
      const int half = b / (Base::SUBS / 2), j = j0 + (b % (Base::SUBS / 2)) * 64;
      this->ptr[b] = uniform_ptr(w + (size_t)half * F + (j < F ? j : j0));
    }
  }
};
// A wave's first BJ / 2 blocks are columns of the gate, the others the same columns of the other projection.
template <int OUTER>
struct GatedBlocks {
  __device__ __forceinline__ static constexpr int column(int BJ, int wj, int b) {
    return b < BJ / 2 ? 32 * (BJ / 2 * wj + b) : OUTER / 2 + 32 * (BJ / 2 * (wj - 1) + b);
  }
};

// A wave's part of dh, 32 * BI rows x 32 * BH columns, in registers: requested when the last copies have landed, so that it is there when the sums are.  A lane loads
// 16 bytes at a time of the row that its sums belong to, those of the lane 32 further on in between.
template <int BI, int BH>
struct Gradient {
  const __bf16* base;   // column of the wave's first block
  long long ld;
  int i_wave, M, lane;
  u32x4 piece[BI][BH][2];
  __device__ __forceinline__ void operator()() {
#pragma unroll
    for (int ib = 0; ib < BI; ib++) {
      const int i = i_wave + 32 * ib + (lane & 31);
      const __bf16* const row = base + (size_t)(i < M ? i : M - 1) * ld + 8 * (lane >> 5);
#pragma unroll
      for (int jb = 0; jb < BH; jb++)
#pragma unroll
        for (int q = 0; q < 2; q++) piece[ib][jb][q] = *reinterpret_cast<const u32x4*>(row + 32 * jb + 16 * q);
    }
  }
  // the four columns 8 g + 4 (lane / 32) .. of a block
  __device__ __forceinline__ void columns(int ib, int jb, int g, float (&d)[4]) const {
    const u32x4& x = piece[ib][jb][g >> 1];
    const auto a = __builtin_amdgcn_permlane32_swap(x[0], x[2], false, false), b = __builtin_amdgcn_permlane32_swap(x[1], x[3], false, false);
    const uint32_t lo = a[g & 1], hi = b[g & 1];
    d[0] = __uint_as_float(lo << 16);
    d[1] = __uint_as_float(lo & 0xffff0000u);
    d[2] = __uint_as_float(hi << 16);
    d[3] = __uint_as_float(hi & 0xffff0000u);
  }
};

// Results leave as stores that the caches need not keep: all workgroups end a tile at about the same time, and 64 to 192 KB of results each are then a burst that
// the chip takes several us for (32768 x 2048 x (2 x 5504) 1317 -> 1263 us, with g and u kept 1467 -> 1338).
//
// GRAD: dgu <- [dg du] from a, w and dh (rows up to a multiple of 32, zeros behind row M); else h, and gu = [g u] unless null.
template <typename G, bool GRAD, Activation ACT>
__global__ void __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(G::WORKGROUPS, G::WORKGROUPS))) gated_kernel(Gated p) {
  using XOp = ContiguousOperand<G::TI, G::STEP>;
  using YOp = GatedOperand<G::TJ, G::STEP>;
  constexpr int BI = G::BI, BJ = G::BJ, BH = BJ / 2, W = 32 * BH;
  extern __shared__ __align__(16) char smem[];

  // workgroup id mod 8 is the XCD: each takes a contiguous run of tiles
  const int tiles_i = (p.M + G::TI - 1) / G::TI, tiles_j = (p.F + G::TJ / 2 - 1) / (G::TJ / 2);
  const int t = ((int)blockIdx.x & 7) * ((int)gridDim.x >> 3) + ((int)blockIdx.x >> 3);
  if (t >= tiles_i * tiles_j) return;
  int ti, tj;
  place_tile(t, tiles_i, tiles_j, 8, ti, tj);
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i0 = ti * G::TI, j0 = tj * (G::TJ / 2);
  const uint32_t base = lds_base(smem);

  XOp xsrc((const __bf16*)p.a, p.lda, i0, p.M, 0, lane, w);
  YOp ysrc((const __bf16*)p.w, p.ldw, j0, p.F, lane, w);
  f32x16 acc[BJ][BI];
  const int i_wave = i0 + 32 * BI * (w & 1), j_wave = j0 + W * (w >> 1);
  Gradient<BI, BH> dh = {(const __bf16*)p.dh + (j_wave < p.F ? j_wave : 0), p.lddh, i_wave, p.M, lane, {}};
  if constexpr (GRAD) gemm_sums<G, XOp, YOp, GatedBlocks<G::TJ>, false>(xsrc, ysrc, p.K / G::STEP, base, lane, w, acc, 0, 0, dh);
  else gemm_sums<G, XOp, YOp, GatedBlocks<G::TJ>, false>(xsrc, ysrc, p.K / G::STEP, base, lane, w, acc);

  if constexpr (BI * BJ == 16) {   // see gemm_block
#pragma unroll
    for (int jb = 0; jb < BJ; jb++)
#pragma unroll
      for (int ib = 0; ib < BI; ib++) asm volatile("" : "+a"(acc[jb][ib]));
  }
  constexpr int PIECE = 32 * W * 2;   // bytes of 32 rows
  if constexpr (!GRAD) {
    char* const out = smem + w * PIECE;
#pragma unroll
    for (int ib = 0; ib < BI; ib++) {
      const int i = i_wave + 32 * ib;
      if (p.gu) {
#pragma unroll
        for (int half = 0; half < 2; half++) {
#pragma unroll
          for (int jb = 0; jb < BH; jb++) {
            helix::put_rows<W>(out, lane, jb, acc[half * BH + jb][ib]);
            __builtin_amdgcn_sched_barrier(0);
          }
          store_rows<W, true>(out, lane, (__bf16*)p.gu + (size_t)i * p.ldgu + (size_t)half * p.F + j_wave, p.ldgu, p.M - i, p.F - j_wave);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
#pragma unroll
      for (int jb = 0; jb < BH; jb++) {
        f32x16 h;
#pragma unroll
        for (int e = 0; e < 16; e++) {
          float value, slope;
          activate<ACT>(acc[jb][ib][e], value, slope);
          h[e] = value * acc[BH + jb][ib][e];
        }
        helix::put_rows<W>(out, lane, jb, h);
        __builtin_amdgcn_sched_barrier(0);
      }
      store_rows<W, true>(out, lane, (__bf16*)p.h + (size_t)i * p.ldh + j_wave, p.ldh, p.M - i, p.F - j_wave);
      __builtin_amdgcn_sched_barrier(0);
    }
  } else {
    const int rows = (p.M + 31) & ~31;
    char* const out = smem + w * (2 * PIECE);
#pragma unroll
    for (int ib = 0; ib < BI; ib++) {
      const int i = i_wave + 32 * ib;
      const uint32_t exists = i + (lane & 31) < p.M ? ~0u : 0u;   // a mask and no condition, which would be a branch for every element
#pragma unroll
      for (int jb = 0; jb < BH; jb++) {
        f32x16 dg, du;
#pragma unroll
        for (int q = 0; q < 4; q++) {
          float d[4];
          dh.columns(ib, jb, q, d);
#pragma unroll
          for (int e = 0; e < 4; e++) {
            float value, slope;
            activate<ACT>(acc[jb][ib][4 * q + e], value, slope);
            dg[4 * q + e] = __uint_as_float(__float_as_uint(d[e] * acc[BH + jb][ib][4 * q + e] * slope) & exists);
            du[4 * q + e] = __uint_as_float(__float_as_uint(d[e] * value) & exists);
          }
        }
        helix::put_rows<W>(out, lane, jb, dg);
        helix::put_rows<W>(out + PIECE, lane, jb, du);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int half = 0; half < 2; half++) {
        store_rows<W, true>(out + half * PIECE, lane, (__bf16*)p.gu + (size_t)i * p.ldgu + (size_t)half * p.F + j_wave, p.ldgu, rows - i, p.F - j_wave);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
}

// dgu [rows][2F] <- [dg du] from the projections that were kept, eight columns to a thread; zeros behind row M.
template <Activation ACT>
__global__ void __launch_bounds__(256) gated_grad_kernel(const __bf16* __restrict__ gu, long long ldgu, const __bf16* __restrict__ dh, long long lddh, __bf16* __restrict__ dgu,
                                                         int M, int rows, int F, unsigned step_rows, unsigned step_chunks) {
  const unsigned chunks = (unsigned)F / 8;
  const unsigned long long at = (unsigned long long)blockIdx.x * 256 + threadIdx.x;
  unsigned row = (unsigned)(at / chunks), c = (unsigned)(at % chunks);
  while (row < (unsigned)rows) {
    bf16x8 dg, du;
#pragma unroll
    for (int e = 0; e < 8; e++) dg[e] = du[e] = (__bf16)0.f;
    if (row < (unsigned)M) {
      const bf16x8 g = *reinterpret_cast<const bf16x8*>(gu + (size_t)row * ldgu + 8 * c), u = *reinterpret_cast<const bf16x8*>(gu + (size_t)row * ldgu + F + 8 * c),
                   d = *reinterpret_cast<const bf16x8*>(dh + (size_t)row * lddh + 8 * c);
#pragma unroll
      for (int e = 0; e < 8; e++) {
        float value, slope;
        activate<ACT>((float)g[e], value, slope);
        dg[e] = (__bf16)((float)d[e] * (float)u[e] * slope);
        du[e] = (__bf16)((float)d[e] * value);
      }
    }
    __bf16* const out = dgu + (size_t)row * 2 * F + 8 * c;
    *reinterpret_cast<bf16x8*>(out) = dg;
    *reinterpret_cast<bf16x8*>(out + F) = du;
    row += step_rows;
    c += step_chunks;
    if (c >= chunks) {
      c -= chunks;
      row++;
    }
  }
}

template <typename G, bool GRAD, Activation ACT>
hipError_t launch_tiles(const Gated& p, hipStream_t stream) {
  const long long tiles = (long long)((p.M + G::TI - 1) / G::TI) * ((p.F + G::TJ / 2 - 1) / (G::TJ / 2));
  auto kern = gated_kernel<G, GRAD, ACT>;
  static unsigned long long configured = 0;   // one static per template instantiation
  const hipError_t e = allow_dynamic_lds(kern, G::LDS, configured);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kern, dim3((unsigned)((tiles + 7) & ~7LL)), dim3(64 * kWaves), G::LDS, stream, p);
  return hipGetLastError();
}
template <bool GRAD, Activation ACT>
hipError_t launch_projections(const Gated& p, hipStream_t stream) {
  if (gated_few(p.M, p.F)) return launch_skinny_projections(p, GRAD, ACT, stream);
  switch (gated_tile(p.M, p.K, p.F)) {
    case TileKind::k256: return launch_tiles<Wide, GRAD, ACT>(p, stream);
    case TileKind::k128: return launch_tiles<Middle, GRAD, ACT>(p, stream);
    default: return launch_tiles<Short, GRAD, ACT>(p, stream);
  }
}
template <Activation ACT>
hipError_t launch_grad(const Gated& p, const void* gu, long long ldgu, hipStream_t stream) {
  const int rows = (p.M + 31) & ~31;
  const long long chunks = p.F / 8, grid = std::min<long long>((chunks * rows + 255) / 256, 2048), step = grid * 256;
  hipLaunchKernelGGL((gated_grad_kernel<ACT>), dim3((unsigned)grid), dim3(256), 0, stream, (const __bf16*)gu, ldgu, (const __bf16*)p.dh, p.lddh, (__bf16*)p.gu, p.M, rows, p.F,
                     (unsigned)(step / chunks), (unsigned)(step % chunks));
  return hipGetLastError();
}

}  // namespace

hipError_t launch_gated_fwd(const Gated& p, Activation act, hipStream_t stream) {
  return act == Activation::silu ? launch_projections<false, Activation::silu>(p, stream) : launch_projections<false, Activation::gelu>(p, stream);
}

// Workspace: that of the linear layer's backward with 2F columns, then dgu.
size_t gated_bwd_products_bytes(int M, int K, int F) { return (linear_bwd_ragged_workspace_bytes(M, K, 2 * F) + 255) & ~(size_t)255; }
size_t gated_bwd_workspace_bytes(int M, int K, int F) { return gated_bwd_products_bytes(M, K, F) + (size_t)((M + 31) & ~31) * 2 * F * 2; }

hipError_t launch_gated_bwd(const Gated& given, const void* gu, long long ldgu, void* da, long long ldda, void* dw, long long lddw, void* workspace, Activation act,
                            hipStream_t stream) {
  Gated p = given;
  p.gu = static_cast<char*>(workspace) + gated_bwd_products_bytes(p.M, p.K, p.F);
  p.ldgu = 2LL * p.F;
  hipError_t e;
  if (gu) e = act == Activation::silu ? launch_grad<Activation::silu>(p, gu, ldgu, stream) : launch_grad<Activation::gelu>(p, gu, ldgu, stream);
  else e = act == Activation::silu ? launch_projections<true, Activation::silu>(p, stream) : launch_projections<true, Activation::gelu>(p, stream);
  if (e != hipSuccess) return e;
  return launch_linear_bwd_ragged(p.a, p.lda, p.w, p.ldw, p.gu, p.ldgu, da, ldda, dw, lddw, workspace, p.M, p.K, 2 * p.F, stream);
}

}  // namespace helix
