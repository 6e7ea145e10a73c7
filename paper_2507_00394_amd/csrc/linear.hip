// The QKV linear layer next to attention (Section 4.2: HelixPipe ships the layer's input and
// weights to the attention stage and runs the layer there) and its two backward products,
// as one bf16 MFMA GEMM kernel for gfx950:
//
//     C[i][j] = sum_r X(i, r) * Y(r, j),       fp32 accumulation
//
//   forward          qkv[M][N] = a[M][K]    * w[K][N]      X stored [i][r],  Y stored [r][j]
//   backward input   da[M][K]  = dqkv[M][N] * w[K][N]^T    X stored [i][r],  Y stored [r][j] after a transposing copy of w
//   backward weight  dw[K][N]  = a[M][K]^T  * dqkv[M][N]   X stored [r][i],  Y stored [r][j]
//
// A workgroup (gemm.hpp) owns a 256 x 256, 128 x 128 or 64 x 64 tile of C (linear_tile and linear_gradient_tiles in dispatch.hpp say which: a
// large tile reads less per MFMA, a small one fills the chip when C is small).
//
// What bounds it: at one GPU's share of a 7B layer (131072 x 4096 x 1536) the power limit, as in the attention
// kernels; with few tokens the latency of the copies and barriers.  The copies are spread behind the MFMAs, each one
// instruction with running scalar pointers; in front of the stage (as address arithmetic, an edge test and
// eight copies in a row, with no MFMA in flight) they cost 14 %: forward 1571 -> 1365 us (1050 -> 1208 TFLOP/s),
// da 1853 -> 1570, dw 1785 -> 1578.
#include "gemm.hpp"
#include "helix_common.hpp"
#include "kernels.hpp"
#include <algorithm>
#include <cmath>

namespace helix {

template <typename G, bool X_ROWS_ARE_R, bool Y_ROWS_ARE_R, typename OutT, bool RAGGED>
__global__ void __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(G::WORKGROUPS, G::WORKGROUPS)))
gemm_kernel(Gemm<OutT> g) {
  gemm_block<G, X_ROWS_ARE_R, Y_ROWS_ARE_R, OutT, RAGGED>(blockIdx.x, g);
}

// Both gradients in one launch (see launch_linear_bwd): the first `weight_blocks` workgroups take the weight gradient.
template <typename GI, bool WT, typename GW, typename WeightT, bool RAGGED>
__global__ void __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(GI::WORKGROUPS, GI::WORKGROUPS)))
linear_bwd_kernel(Gemm<__bf16> input, Gemm<WeightT> weight, int weight_blocks) {
  static_assert(GI::WORKGROUPS == GW::WORKGROUPS, "tiles that share a compute unit alike");
  const int block = (int)blockIdx.x;
  if (block < weight_blocks) gemm_block<GW, true, true, WeightT, RAGGED>(block, weight);
  else gemm_block<GI, false, WT, __bf16>(block - weight_blocks, input);
}

// dst[e] = sum over `parts` slabs of src, `n` elements each (n a multiple of 4).
template <typename T>
__global__ void __launch_bounds__(256) sum_parts_kernel(const float* __restrict__ src, T* __restrict__ dst, long long ld_dst,
                                                        int rows, int cols, int parts) {
  const long long quad = (long long)blockIdx.x * 256 + threadIdx.x;
  const int qpr = cols / 4;
  if (quad >= (long long)rows * qpr) return;
  const int r = (int)(quad / qpr), c = (int)(quad % qpr) * 4;
  const size_t slab = (size_t)rows * cols;
  f32x4 acc = *reinterpret_cast<const f32x4*>(src + (size_t)r * cols + c);
  for (int p = 1; p < parts; p++) acc += *reinterpret_cast<const f32x4*>(src + p * slab + (size_t)r * cols + c);
  typedef T Quad __attribute__((ext_vector_type(4)));
  *reinterpret_cast<Quad*>(dst + (size_t)r * ld_dst + c) = __builtin_convertvector(acc, Quad);
}

template <typename G, typename OutT>
static long long set_tiles(Gemm<OutT>& g) {
  g.tiles_i = (g.I + G::TI - 1) / G::TI;
  g.tiles_j = (g.J + G::TJ - 1) / G::TJ;
  return (long long)g.blocks_per_part() * g.parts;
}
template <typename G, bool XR, bool YR, bool RAGGED = false, typename OutT>
static hipError_t launch_gemm_tile(Gemm<OutT> g, hipStream_t stream) {
  const unsigned grid = (unsigned)set_tiles<G>(g);
  auto kern = gemm_kernel<G, XR, YR, OutT, RAGGED>;
  static unsigned long long configured = 0;   // one static per template instantiation
  hipError_t e = allow_dynamic_lds(kern, G::LDS, configured);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kern, dim3(grid), dim3(64 * kWaves), G::LDS, stream, g);
  return hipGetLastError();
}
template <typename GI, bool WT, typename GW, bool RAGGED, typename WeightT>
static hipError_t launch_gradients(Gemm<__bf16> input, Gemm<WeightT> weight, hipStream_t stream) {
  const long long weight_blocks = set_tiles<GW>(weight), input_blocks = set_tiles<GI>(input);
  const size_t lds = GI::LDS > GW::LDS ? GI::LDS : GW::LDS;
  auto kern = linear_bwd_kernel<GI, WT, GW, WeightT, RAGGED>;
  static unsigned long long configured = 0;   // one static per template instantiation
  hipError_t e = allow_dynamic_lds(kern, lds, configured);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kern, dim3((unsigned)(weight_blocks + input_blocks)), dim3(64 * kWaves), lds, stream, input, weight, (int)weight_blocks);
  return hipGetLastError();
}

hipError_t launch_linear_fwd(const void* a, long long lda, const void* w, long long ldw, void* out, long long ldo,
                             int M, int K, int N, hipStream_t stream) {
  const Gemm<__bf16> g = {(const __bf16*)a, (const __bf16*)w, (__bf16*)out, lda, ldw, ldo, 0, M, N, K, 0, 0, 1, K};
  switch (linear_tile(M, K, N)) {
    case TileKind::k256: return launch_gemm_tile<Tile256, false, true>(g, stream);
    case TileKind::k128: return launch_gemm_tile<Tile128, false, true>(g, stream);
    default: return launch_gemm_tile<Tile64, false, true>(g, stream);
  }
}
// out[c][r] = in[r][c] for a [rows][cols] bf16 matrix (both extents multiples of 64).
__global__ void __launch_bounds__(256) transpose_kernel(const __bf16* __restrict__ in, long long ld_in,
                                                        __bf16* __restrict__ out, long long ld_out) {
  __shared__ __bf16 tile[64][66];
  const int tx = threadIdx.x & 63, ty = threadIdx.x >> 6;
  const size_t r0 = (size_t)blockIdx.y * 64, c0 = (size_t)blockIdx.x * 64;
#pragma unroll
  for (int i = 0; i < 16; i++) tile[ty * 16 + i][tx] = in[(r0 + ty * 16 + i) * ld_in + c0 + tx];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 16; i++) out[(c0 + ty * 16 + i) * ld_out + r0 + tx] = tile[tx][ty * 16 + i];
}

// Workspace of the backward: w^T (bf16 [N][K], rounded up to 256 bytes), then the partial weight gradients.
size_t linear_bwd_wt_bytes(int K, int N) { return ((size_t)K * N * 2 + 255) & ~(size_t)255; }
size_t linear_bwd_workspace_bytes(int M, int K, int N) {
  const int parts = linear_bwd_weight_parts(M, K, N);
  return linear_bwd_wt_bytes(K, N) + (parts > 1 ? (size_t)parts * K * N * sizeof(float) : 0);
}

// With the input gradient in parts (linear_bwd with RAGGED only): the slabs hold either's partial results.  No less than fewer rows need.
size_t linear_bwd_ragged_workspace_bytes(int M, int K, int N) {
  const int parts = split_weight_parts(M, K, N);
  return linear_bwd_wt_bytes(K, N) + std::max(parts > 1 ? (size_t)parts * K * N * sizeof(float) : 0, (size_t)split_input_rows(M, K, N) * K * sizeof(float));
}

// Input gradient da = dout * w^T.  With w as stored ([K][N], contraction index n contiguous) both
// operands would reach LDS in 64-byte row pieces, the least efficient pattern of the copy path
// (measured 30 % slower than the forward product); on the large tile a transposed copy of the small weight matrix
// (w^T [N][K], in the workspace) turns it into the forward's operand combination.
// Weight gradient dw = a^T * dout, in parts.
//
// The two need nothing of each other, so they go in one launch where their tiles share a compute unit alike, the weight gradient's longer
// workgroups first: the last round of one is filled by the other, and a small layer pays for one start.
template <bool RAGGED, typename WeightT>
static hipError_t launch_products(TilePair kind, const Gemm<__bf16>& in, const Gemm<WeightT>& grad_w, hipStream_t stream) {
  if (kind.input == TileKind::k256) return launch_gradients<Tile256, true, Tile256, RAGGED>(in, grad_w, stream);   // which the weight gradient then has too
  if (kind.weight == TileKind::k256) {   // tiles that do not share a compute unit alike: a launch each
    const hipError_t e = launch_gemm_tile<Tile256, true, true, RAGGED>(grad_w, stream);
    if (e != hipSuccess) return e;
    return kind.input == TileKind::k128 ? launch_gemm_tile<Tile128, false, false>(in, stream) : launch_gemm_tile<Tile64, false, false>(in, stream);
  }
  if (kind.input == TileKind::k128)
    return kind.weight == TileKind::k128 ? launch_gradients<Tile128, false, Tile128, RAGGED>(in, grad_w, stream)
                                         : launch_gradients<Tile128, false, Tile64ShortStages, RAGGED>(in, grad_w, stream);
  return kind.weight == TileKind::k128 ? launch_gradients<Tile64, false, Tile128, RAGGED>(in, grad_w, stream)
                                       : launch_gradients<Tile64, false, Tile64ShortStages, RAGGED>(in, grad_w, stream);
}

template <bool RAGGED, typename WeightT>
static hipError_t launch_weight(TileKind kind, const Gemm<WeightT>& grad_w, hipStream_t stream) {
  return kind == TileKind::k256 ? launch_gemm_tile<Tile256, true, true, RAGGED>(grad_w, stream) : launch_gemm_tile<Tile128, true, true, RAGGED>(grad_w, stream);
}
template <typename T>
static hipError_t launch_sum_parts(const float* slabs, T* dst, long long ld_dst, int rows, int cols, int parts, hipStream_t stream) {
  const long long quads = (long long)rows * cols / 4;
  hipLaunchKernelGGL(sum_parts_kernel<T>, dim3((unsigned)((quads + 255) / 256)), dim3(256), 0, stream, slabs, dst, ld_dst, rows, cols, parts);
  return hipGetLastError();
}

// RAGGED: any M; dout then has rows of zeros up to the next multiple of 32.
template <bool RAGGED, typename WeightT>
static hipError_t linear_bwd(const void* a, long long lda, const void* w, long long ldw, const void* dout, long long ldd, void* da, long long ldda, WeightT* dw,
                             long long lddw, void* workspace, int M, int K, int N, int side, hipStream_t stream) {
  __bf16* const wt = (__bf16*)workspace;
  float* const slabs = reinterpret_cast<float*>(static_cast<char*>(workspace) + linear_bwd_wt_bytes(K, N));
  const int parts = RAGGED ? split_weight_parts(M, K, N) : linear_bwd_weight_parts(M, K, N);
  const int per = parts == 1 ? M : (((M + 31) / 32 + parts - 1) / parts) * 32;    // tokens per part, a multiple of the stage length
  Gemm<__bf16> in = {(const __bf16*)dout, (const __bf16*)w, (__bf16*)da, ldd, ldw, ldda, 0, M, K, N, 0, 0, 1, N, 1};
  TilePair kind = linear_gradient_tiles(M, K, N, parts);
  const int input_parts = RAGGED ? split_input_parts(M, K, N) : 1;
  if (input_parts > 1) {   // the input gradient's contraction in parts too, whose sums come before the weight gradient takes the slabs
    const int per_in = (N / 64 + input_parts - 1) / input_parts * 64;
    const Gemm<float> in_parts = {(const __bf16*)dout, (const __bf16*)w, slabs, ldd, ldw, K, (long long)M * K, M, K, N, 0, 0, (N + per_in - 1) / per_in, per_in, 1};
    hipError_t e = split_input_tile(M) == TileKind::k64 ? launch_gemm_tile<Tile64, false, false>(in_parts, stream) : launch_gemm_tile<Tile128, false, false>(in_parts, stream);
    if (e != hipSuccess) return e;
    if ((e = launch_sum_parts(slabs, (__bf16*)da, ldda, M, K, in_parts.parts, stream)) != hipSuccess) return e;
  } else if (kind.input == TileKind::k256) {
    hipLaunchKernelGGL(transpose_kernel, dim3((unsigned)(N / 64), (unsigned)(K / 64)), dim3(256), 0, stream, (const __bf16*)w, ldw, wt, (long long)K);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    in.Y = wt;
    in.ldy = K;
  }
  if (parts == 1) {
    const Gemm<WeightT> grad_w = {(const __bf16*)a, (const __bf16*)dout, dw, lda, ldd, lddw, 0, K, N, M, 0, 0, 1, per, side};
    return input_parts > 1 ? launch_weight<RAGGED>(kind.weight, grad_w, stream) : launch_products<RAGGED>(kind, in, grad_w, stream);
  }
  const Gemm<float> grad_w = {(const __bf16*)a, (const __bf16*)dout, slabs, lda, ldd, N, (long long)K * N, K, N, M, 0, 0, parts, per, side};
  const hipError_t e = input_parts > 1 ? launch_weight<RAGGED>(kind.weight, grad_w, stream) : launch_products<RAGGED>(kind, in, grad_w, stream);
  return e != hipSuccess ? e : launch_sum_parts(slabs, dw, lddw, K, N, parts, stream);
}

hipError_t launch_linear_bwd(const void* a, long long lda, const void* w, long long ldw, const void* dout, long long ldd, void* da,
                             long long ldda, float* dw, long long lddw, void* workspace, int M, int K, int N, hipStream_t stream) {
  return linear_bwd<false>(a, lda, w, ldw, dout, ldd, da, ldda, dw, lddw, workspace, M, K, N, 0, stream);
}
hipError_t launch_linear_bwd_ragged(const void* a, long long lda, const void* w, long long ldw, const void* dout, long long ldd, void* da,
                                    long long ldda, void* dw, long long lddw, void* workspace, int M, int K, int N, hipStream_t stream) {
  return linear_bwd<true>(a, lda, w, ldw, dout, ldd, da, ldda, (__bf16*)dw, lddw, workspace, M, K, N, 8, stream);
}

}  // namespace helix
