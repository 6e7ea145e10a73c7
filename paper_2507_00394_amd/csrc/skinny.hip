// The gated projections of at most 32 rows (tokens).
//
// The bytes of the weights are all that counts, and a compute unit fetches them as fast as it has requests on their way: the tiles of gated.hip spend half of
// them on rows of a that do not exist, and their waves meet at a barrier for every 12 KB.  Here a workgroup has 64 columns of both projections, 128 bytes of
// a row, and its waves share the contraction: each streams its own range of it through its own ring of LDS stages, three of 10 KB on their way,
// and waits for nobody; the partial sums are added up in LDS at the end, in a fixed order.
#include "gated_math.hpp"
#include "gemm.hpp"
#include "helix_common.hpp"
#include "kernels.hpp"

namespace helix {
namespace {

constexpr int kSkinnyWaves = 4;
// A wave's stage: 32 rows of a and 64 columns of either projection, 32 contraction indices each.
struct Skinny {
  static constexpr int STEP = 32, XBYTES = 32 * STEP * 2, YBYTES = 64 * STEP * 2, STAGE = XBYTES + 2 * YBYTES, NST = 4, RING = NST * STAGE;
  static constexpr int LDS = kSkinnyWaves * RING;   // 160 KB: one workgroup on a compute unit
  static_assert(RING >= 4 * 4096 && LDS <= 160 * 1024, "the partial sums of a wave, four blocks, lie in its ring");
};

template <bool GRAD, Activation ACT>
__global__ void __launch_bounds__(64 * kSkinnyWaves) skinny_kernel(Gated p) {
  using S = Skinny;
  using XLoader = TileLoader<32, 32, 1>;
  using YLoader = TileLoader<64, 32, 1>;
  constexpr int NDMA = XLoader::N + 2 * YLoader::N, AHEAD = S::NST - 1;
  extern __shared__ __align__(16) char smem[];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
  const int j0 = 64 * (int)blockIdx.x;

  const int nk = p.K / S::STEP, k_begin = nk * w / kSkinnyWaves, n = nk * (w + 1) / kSkinnyWaves - k_begin;
  const XLoader xload(lane, 0, (int)p.lda);
  const YLoader yload(lane, 0, (int)p.ldw);
  uint32_t xoff[XLoader::N];
#pragma unroll
  for (int i = 0; i < XLoader::N; i++) {   // rows behind the last one are the last one: their results are not stored
    const int row = i * XLoader::ROWS_PER_KB + xload.lane_row;
    xoff[i] = xload.off[i] - (uint32_t)(row > p.M - 1 ? row - (p.M - 1) : 0) * xload.row_bytes;
  }
  const __bf16* xptr = uniform_ptr((const __bf16*)p.a + (size_t)k_begin * S::STEP);
  const __bf16* yptr[2];
#pragma unroll
  for (int b = 0; b < 2; b++) yptr[b] = uniform_ptr((const __bf16*)p.w + (size_t)k_begin * S::STEP * p.ldw + (size_t)b * p.F + j0);
  const long long ystep = S::STEP * p.ldw;
  const uint32_t ring = lds_base(smem) + w * S::RING;
  auto copy = [&](uint32_t stage) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < XLoader::N; i++) copy_16_bytes_per_lane(xoff[i], xptr, stage + i * 1024);
#pragma unroll
    for (int b = 0; b < 2; b++)
#pragma unroll
      for (int i = 0; i < YLoader::N; i++) copy_16_bytes_per_lane(yload.off[i], yptr[b], stage + S::XBYTES + b * S::YBYTES + i * 1024);
    xptr += S::STEP;
#pragma unroll
    for (int b = 0; b < 2; b++) yptr[b] += ystep;
  };

  // lane addresses inside a stage: a's for each 16 contraction indices; the weights' a pair for each 32 columns
  uint32_t straight[2], crossed[2][2];
#pragma unroll
  for (int ks = 0; ks < 2; ks++) straight[ks] = lds_chunk_off<32>(lane & 31, 2 * ks + half);
#pragma unroll
  for (int jb = 0; jb < 2; jb++) {
    const int i = lane & 15, c = 32 * jb + ((lane >> 4) & 1) * 16 + (i & 3) * 4, r = half * 8 + (i >> 2);
    crossed[jb][0] = lds_chunk_off<64>(r, c >> 3) + (c & 7) * 2;
    crossed[jb][1] = lds_chunk_off<64>(r + 4, c >> 3) + (c & 7) * 2;
  }
  f32x16 acc[2][2];   // projection, 32 columns
#pragma unroll
  for (int b = 0; b < 2; b++)
#pragma unroll
    for (int jb = 0; jb < 2; jb++)
#pragma unroll
      for (int e = 0; e < 16; e++) acc[b][jb][e] = 0.f;
  auto multiply = [&](uint32_t stage) __attribute__((always_inline)) {
    bf16x8 x[2], y[2][2][2];
#pragma unroll
    for (int ks = 0; ks < 2; ks++) {
      x[ks] = lds_b128(stage + straight[ks]);
#pragma unroll
      for (int b = 0; b < 2; b++)
#pragma unroll
        for (int jb = 0; jb < 2; jb++) {
          const uint32_t at = stage + S::XBYTES + b * S::YBYTES;
          y[ks][b][jb] = lds_tr_pair(at + crossed[jb][0], at + crossed[jb][1], ks * 16 * 128);
        }
    }
#pragma unroll
    for (int ks = 0; ks < 2; ks++)
#pragma unroll
      for (int b = 0; b < 2; b++)
#pragma unroll
        for (int jb = 0; jb < 2; jb++) acc[b][jb] = mfma32(y[ks][b][jb], x[ks], acc[b][jb]);
  };

  // Stage k + AHEAD goes where stage k - 1 was, whose operands are in registers by then: the MFMAs that take them have been issued.
  uint32_t to = ring, from = ring;
  auto next = [&](uint32_t& stage) __attribute__((always_inline)) { stage = stage == ring + (S::NST - 1) * S::STAGE ? ring : stage + S::STAGE; };
  for (int k = 0; k < AHEAD && k < n; k++) {
    copy(to);
    next(to);
  }
  int k = 0;
  for (; k + AHEAD < n; k++) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the reads of stage k - 1, before it is overwritten
    copy(to);
    next(to);
    wait_tile_loads_except<AHEAD * NDMA>();
    multiply(from);
    next(from);
  }
  wait_tile_loads();
  for (; k < n; k++) {
    multiply(from);
    next(from);
  }

  // The partial sums through LDS, each wave's in its own part; then every wave adds up 8 columns of 32 rows at a time.
#pragma unroll
  for (int b = 0; b < 2; b++)
#pragma unroll
    for (int jb = 0; jb < 2; jb++) lds_put_block(smem + w * S::RING + (2 * b + jb) * 4096, lane, acc[b][jb]);
  __syncthreads();
#pragma unroll
  for (int u = 0; u < 8 / kSkinnyWaves; u++) {
    const int jb = u, g = w;
    f32x4 sum[2];
#pragma unroll
    for (int b = 0; b < 2; b++) {
      const char* const at = smem + (2 * b + jb) * 4096 + 1024 * g + 16 * lane;
      sum[b] = *reinterpret_cast<const f32x4*>(at);
#pragma unroll
      for (int v = 1; v < kSkinnyWaves; v++) sum[b] += *reinterpret_cast<const f32x4*>(at + v * S::RING);
    }
    const int i = lane & 31, j = j0 + 32 * jb + 8 * g + 4 * half;
    f32x4 value, slope;
#pragma unroll
    for (int e = 0; e < 4; e++) {
      float v, s;
      activate<ACT>(sum[0][e], v, s);
      value[e] = v;
      slope[e] = s;
    }
    if constexpr (!GRAD) {
      if (i >= p.M) continue;
      *reinterpret_cast<bf16x4*>((__bf16*)p.h + (size_t)i * p.ldh + j) = __builtin_convertvector(value * sum[1], bf16x4);
      if (p.gu)
#pragma unroll
        for (int b = 0; b < 2; b++) *reinterpret_cast<bf16x4*>((__bf16*)p.gu + (size_t)i * p.ldgu + (size_t)b * p.F + j) = __builtin_convertvector(sum[b], bf16x4);
    } else {   // zeros behind row M
      f32x4 dg = 0.f, du = 0.f;
      if (i < p.M) {
        const f32x4 d = __builtin_convertvector(*reinterpret_cast<const bf16x4*>((const __bf16*)p.dh + (size_t)i * p.lddh + j), f32x4);
        dg = d * sum[1] * slope;
        du = d * value;
      }
      *reinterpret_cast<bf16x4*>((__bf16*)p.gu + (size_t)i * p.ldgu + j) = __builtin_convertvector(dg, bf16x4);
      *reinterpret_cast<bf16x4*>((__bf16*)p.gu + (size_t)i * p.ldgu + p.F + j) = __builtin_convertvector(du, bf16x4);
    }
  }
}

template <bool GRAD, Activation ACT>
hipError_t launch(const Gated& p, hipStream_t stream) {
  auto kern = skinny_kernel<GRAD, ACT>;
  static unsigned long long configured = 0;   // one static per template instantiation
  const hipError_t e = allow_dynamic_lds(kern, Skinny::LDS, configured);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kern, dim3((unsigned)(p.F / 64)), dim3(64 * kSkinnyWaves), (int)Skinny::LDS, stream, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_skinny_projections(const Gated& p, bool grad, Activation act, hipStream_t stream) {
  if (act == Activation::silu) return grad ? launch<true, Activation::silu>(p, stream) : launch<false, Activation::silu>(p, stream);
  return grad ? launch<true, Activation::gelu>(p, stream) : launch<false, Activation::gelu>(p, stream);
}

}  // namespace helix
