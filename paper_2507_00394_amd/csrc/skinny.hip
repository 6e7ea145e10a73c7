// The gated projections of at most 32 rows (tokens).
//
// The bytes of the weights are all that counts.  A compute unit has only so many lines on their way, about 450 whatever asks for them (a workgroup takes 2.8 us for 1024
// rows of w from the last cache, with 64 columns of both projections or 32, through LDS or into registers, with 96 or 256 KB asked for), so what helps is more compute units: a
// workgroup has 32 columns of either projection, and neighbours, which share lines, are on one XCD.  Its waves share the contraction.  Each streams its own range of it straight into
// registers, DEPTH groups of 32 rows of w ahead, and waits for nobody: a lane loads four columns of eight rows, which with the elements of two rows put side by side (one
// byte permutation) are the contraction indices of four operands of the 16x16x32 MFMA.  An operand's 16 rows are every fourth column: the first eight of the gate, the
// others the same columns of the other projection.  The partial sums are added up in LDS at the end, in a fixed order.
//
// One token, us (64 columns to a workgroup and stages in LDS / so): 2048 x 5504 11.5 / 10.2, 4.4 TB/s; 4096 x 4096 21.6 / 20.3; 1024 x 2752 7.1 / 5.9; 512 x 640 5.0 / 3.7.
#include "gated_math.hpp"
#include "helix_common.hpp"
#include "kernels.hpp"

namespace helix {
namespace {

constexpr int kFewWaves = 8, kFewColumns = 32, kFewGroup = 32;
typedef uint32_t Piece __attribute__((ext_vector_type(2)));   // four columns of a row of w

// From a base in scalar registers and a lane's offset.
template <typename T>
__device__ __forceinline__ T load_global(const __bf16* base, uint32_t off) {
  typedef const __attribute__((address_space(1))) char* Bytes;
  typedef const __attribute__((address_space(1))) T* Values;
  return *(Values)((Bytes)uniform_ptr(base) + off);
}

// TB blocks of 16 tokens.
template <int TB, bool GRAD, Activation ACT>
__global__ void __launch_bounds__(64 * kFewWaves) skinny_kernel(Gated p) {
  constexpr int DEPTH = 6;
  constexpr int BLOCK = 1024, SUMS = 4 * TB * BLOCK;   // bytes of a wave's partial sums: 16 x 16 for each operand and block of tokens
  extern __shared__ __align__(16) char smem[];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int id = (int)blockIdx.x, block = 2 * ((id >> 4) * 8 + (id & 7)) + ((id >> 3) & 1);   // the XCD is the id mod 8
  const int j0 = kFewColumns * block;
  if (j0 >= p.F) return;

  const int nk = p.K / kFewGroup, k_begin = nk * w / kFewWaves, n = nk * (w + 1) / kFewWaves - k_begin;
  const int slot = lane & 15, rows8 = 8 * (lane >> 4);   // operand row, first contraction index inside a group
  // below 2^29: the pitch is at most 2^22
  uint32_t woff = ((uint32_t)rows8 * (uint32_t)p.ldw + (slot & 8 ? (uint32_t)p.F : 0) + 4 * (slot & 7)) * 2;
  uint32_t xoff[TB];
#pragma unroll
  for (int t = 0; t < TB; t++) {   // rows behind the last one are the last one: their results are not stored
    const int row = 16 * t + slot;
    xoff[t] = ((uint32_t)(row < p.M ? row : p.M - 1) * (uint32_t)p.lda + rows8) * 2;
  }
  const __bf16* xptr = (const __bf16*)p.a + (size_t)k_begin * kFewGroup;
  const __bf16* wptr = (const __bf16*)p.w + (size_t)k_begin * kFewGroup * p.ldw + j0;

  Piece piece[DEPTH][8];
  bf16x8 x[DEPTH][TB];
  f32x4 acc[4][TB];
#pragma unroll
  for (int c = 0; c < 4; c++)
#pragma unroll
    for (int t = 0; t < TB; t++) acc[c][t] = 0.f;
  auto load = [&](int d) __attribute__((always_inline)) {
    pin(woff);   // widened here, where the load takes it as it is, not in front of the loop
#pragma unroll
    for (int t = 0; t < TB; t++) {
      pin(xoff[t]);
      x[d][t] = load_global<bf16x8>(xptr, xoff[t]);
    }
#pragma unroll
    for (int r = 0; r < 8; r++) piece[d][r] = load_global<Piece>(wptr + r * p.ldw, woff);
    xptr += kFewGroup;
    wptr += kFewGroup * p.ldw;
    __builtin_amdgcn_sched_barrier(0);
  };
  auto multiply = [&](int d) __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < 4; c++) {
      u32x4 y;
#pragma unroll
      for (int i = 0; i < 4; i++) y[i] = __builtin_amdgcn_perm(piece[d][2 * i + 1][c / 2], piece[d][2 * i][c / 2], c & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
      for (int t = 0; t < TB; t++) acc[c][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, y), x[d][t], acc[c][t], 0, 0, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  };

  if (n >= DEPTH) {
#pragma unroll
    for (int d = 0; d < DEPTH; d++) load(d);
    int left = n - DEPTH;   // groups not yet asked for
    for (; left >= DEPTH; left -= DEPTH)
#pragma unroll
      for (int d = 0; d < DEPTH; d++) {
        multiply(d);
        load(d);
      }
#pragma unroll
    for (int d = 0; d < DEPTH; d++) {
      multiply(d);
      if (d < left) load(d);
    }
#pragma unroll
    for (int d = 0; d < DEPTH; d++)
      if (d < left) multiply(d);
  } else {
#pragma unroll
    for (int d = 0; d < DEPTH; d++)
      if (d < n) load(d);
#pragma unroll
    for (int d = 0; d < DEPTH; d++)
      if (d < n) multiply(d);
  }

  // acc[c][t]: token 16 t + lane % 16, element e the operand row 4 (lane / 16) + e, which is column 4 (row % 8) + c of one projection
#pragma unroll
  for (int c = 0; c < 4; c++)
#pragma unroll
    for (int t = 0; t < TB; t++) *reinterpret_cast<f32x4*>(smem + w * SUMS + (c * TB + t) * BLOCK + 16 * lane) = acc[c][t];
  __syncthreads();
  // a thread takes two columns of a token; the first half of the threads is enough for 16 tokens
  if (const int u = threadIdx.x; u < TB * 256) {
    const int token = u & 15, row = (u >> 4) & 7, pair = (u >> 7) & 1, t = u >> 8;
    float sum[2][2];   // projection, column
#pragma unroll
    for (int b = 0; b < 2; b++)
#pragma unroll
      for (int c = 0; c < 2; c++) {
        const int r = row + 8 * b;
        const char* const at = smem + ((2 * pair + c) * TB + t) * BLOCK + 16 * (token + 16 * (r >> 2)) + 4 * (r & 3);
        float s = *reinterpret_cast<const float*>(at);
#pragma unroll
        for (int v = 1; v < kFewWaves; v++) s += *reinterpret_cast<const float*>(at + v * SUMS);
        sum[b][c] = s;
      }
    const int i = 16 * t + token, j = j0 + 4 * row + 2 * pair;
    float value[2], slope[2];
#pragma unroll
    for (int c = 0; c < 2; c++) activate<ACT>(sum[0][c], value[c], slope[c]);
    auto put = [&](void* base, long long ld, int column, float a, float b) __attribute__((always_inline)) {
      *reinterpret_cast<uint32_t*>((__bf16*)base + (size_t)i * ld + column) = pack_bf16_pair(a, b);
    };
    if constexpr (!GRAD) {
      if (i < p.M) {
        put(p.h, p.ldh, j, value[0] * sum[1][0], value[1] * sum[1][1]);
        if (p.gu)
#pragma unroll
          for (int b = 0; b < 2; b++) put(p.gu, p.ldgu, b * p.F + j, sum[b][0], sum[b][1]);
      }
    } else {   // zeros behind row M
      float dg[2] = {0.f, 0.f}, du[2] = {0.f, 0.f};
      if (i < p.M) {
        const uint32_t both = *reinterpret_cast<const uint32_t*>((const __bf16*)p.dh + (size_t)i * p.lddh + j);
        const float d[2] = {__uint_as_float(both << 16), __uint_as_float(both & 0xffff0000u)};
#pragma unroll
        for (int c = 0; c < 2; c++) {
          dg[c] = d[c] * sum[1][c] * slope[c];
          du[c] = d[c] * value[c];
        }
      }
      put(p.gu, p.ldgu, j, dg[0], dg[1]);
      put(p.gu, p.ldgu, p.F + j, du[0], du[1]);
    }
  }
  if constexpr (GRAD && TB == 1) {   // dgu has rows up to a multiple of 32: two columns of each projection to a thread, 16 rows
    if (const int u = threadIdx.x; u < 256) {
      const int i = 16 + (u >> 4), j = j0 + 2 * (u & 15);
#pragma unroll
      for (int b = 0; b < 2; b++) *reinterpret_cast<uint32_t*>((__bf16*)p.gu + (size_t)i * p.ldgu + (size_t)b * p.F + j) = 0;
    }
  }
}

template <int TB, bool GRAD, Activation ACT>
hipError_t launch_few(const Gated& p, hipStream_t stream) {
  constexpr int LDS = kFewWaves * 4 * TB * 1024;
  static_assert(LDS <= 64 * 1024, "no more than a kernel has without being asked for");
  hipLaunchKernelGGL((skinny_kernel<TB, GRAD, ACT>), dim3((unsigned)(p.F / kFewColumns + 15) & ~15u), dim3(64 * kFewWaves), LDS, stream, p);
  return hipGetLastError();
}
template <bool GRAD, Activation ACT>
hipError_t launch(const Gated& p, hipStream_t stream) {
  return p.M <= 16 ? launch_few<1, GRAD, ACT>(p, stream) : launch_few<2, GRAD, ACT>(p, stream);
}

}  // namespace

hipError_t launch_skinny_projections(const Gated& p, bool grad, Activation act, hipStream_t stream) {
  if (act == Activation::silu) return grad ? launch<true, Activation::silu>(p, stream) : launch<false, Activation::silu>(p, stream);
  return grad ? launch<true, Activation::gelu>(p, stream) : launch<false, Activation::gelu>(p, stream);
}

}  // namespace helix
