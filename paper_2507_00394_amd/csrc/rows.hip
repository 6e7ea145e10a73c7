// The row-wise operators around the attention stage, for activations of M rows (tokens) and E columns:
//
//   dropout and sum   out = r + keep * x * scale
//   layer norm        y = (x - mean) * rstd * gamma + beta,   mean and rstd = (var + eps)^-1/2 over a row
//   both              s = r + keep * x * scale,  y = layer norm of s
//
// and their gradients.  All are bound by the bytes they move; the arithmetic (fp32) has to stay out of the way.
//
// A thread owns 8 consecutive columns at a time ("chunk", 16 bytes of a 2-byte type), the unit of the random numbers too.
//
// Random numbers: Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011) with the
// seed as its key and the counter (chunk, first_row + row, offset): 128 bits, 16 to each column of the chunk.  A column is kept where its
// 16 bits are no less than round(p * 2^16).  Nothing of the mask is stored: the backward pass, or a forward pass that is run again,
// makes the same bits.  16 bits and not 32 because the generator would otherwise be the bound: two 32 x 32 bit products a round take 16
// cycles each, 320 cycles of a wave for a block, at 512 elements a block 2.6 * 10^12 elements/s on the chip (15 TB/s of bf16 traffic), at
// 256 half of that.
#include "helix_common.hpp"
#include "kernels.hpp"
#include <algorithm>

namespace helix {
namespace {

// Eight elements with the alignment of one: rows of any width and pitch are read and written 16 bytes at a time.
template <typename T>
struct Chunk {
  typedef T Vec __attribute__((ext_vector_type(8), aligned(sizeof(T))));
  Vec v;
};
// `n` of the 8 elements exist; the others are read as zero and not written.
template <typename T>
__device__ __forceinline__ Chunk<T> load_chunk(const T* p, int n) {
  Chunk<T> c;
  c.v = (T)0.f;
  if (n >= 8) {
    c.v = *reinterpret_cast<const typename Chunk<T>::Vec*>(p);
  } else if (n > 0) {
#pragma unroll
    for (int e = 0; e < 7; e++)
      if (e < n) c.v[e] = p[e];
  }
  return c;
}
template <typename T>
__device__ __forceinline__ void store_chunk(T* p, int n, const f32x8& x) {
  const auto v = __builtin_convertvector(x, typename Chunk<T>::Vec);
  if (n >= 8) {
    *reinterpret_cast<typename Chunk<T>::Vec*>(p) = v;
  } else if (n > 0) {
#pragma unroll
    for (int e = 0; e < 7; e++)
      if (e < n) p[e] = v[e];
  }
}
template <typename T>
__device__ __forceinline__ f32x8 widen(const Chunk<T>& c) { return __builtin_convertvector(c.v, f32x8); }

// The generator of one call.  `cut` = round(p * 2^16).
struct Generator {
  uint32_t k0, k1, o0, o1, first_row, cut;
  float scale;
  __device__ __forceinline__ explicit Generator(const Dropout& d) : k0(0), k1(0), o0(0), o1(0), first_row(d.first_row), cut(d.cut), scale(d.scale) {
    if (cut) {
      const uint64_t seed = d.rng[0], offset = d.rng[1];
      k0 = (uint32_t)seed;
      k1 = (uint32_t)(seed >> 32);
      o0 = (uint32_t)offset;
      o1 = (uint32_t)(offset >> 32);
    }
  }
  __device__ __forceinline__ u32x4 block(uint32_t chunk, uint32_t row) const {
    uint32_t c0 = chunk, c1 = first_row + row, c2 = o0, c3 = o1, a = k0, b = k1;
#pragma unroll
    for (int round = 0; round < 10; round++) {
      const uint64_t p0 = (uint64_t)0xD2511F53u * c0, p1 = (uint64_t)0xCD9E8D57u * c2;
      c0 = (uint32_t)(p1 >> 32) ^ c1 ^ a;
      c2 = (uint32_t)(p0 >> 32) ^ c3 ^ b;
      c1 = (uint32_t)p1;
      c3 = (uint32_t)p0;
      a += 0x9E3779B9u;
      b += 0xBB67AE85u;
    }
    return u32x4{c0, c1, c2, c3};
  }
  // keep * x * scale.  What is dropped is zero whatever it was.
  __device__ __forceinline__ f32x8 apply(const f32x8& x, uint32_t chunk, uint32_t row) const {
    if (!cut) return x;
    const u32x4 bits = block(chunk, row);
    f32x8 y;
#pragma unroll
    for (int e = 0; e < 8; e++) {
      const uint32_t u = e & 1 ? bits[e / 2] >> 16 : bits[e / 2] & 0xffffu;
      y[e] = u >= cut ? x[e] * scale : 0.f;
    }
    return y;
  }
};

// ---------------------------------------------------------------- dropout and sum

// Chunks of all rows one after the other; a thread steps over `step_rows` rows and `step_chunks` chunks, without a division.
template <typename T>
__global__ void __launch_bounds__(256) dropout_add_kernel(const T* x, long long ldx, const T* r, long long ldr, T* out, long long ldo, unsigned rows, int cols,
                                                          Dropout drop, unsigned step_rows, unsigned step_chunks) {
  const Generator gen(drop);
  const unsigned chunks = (unsigned)(cols + 7) / 8;
  const unsigned long long at = (unsigned long long)blockIdx.x * 256 + threadIdx.x;
  unsigned row = (unsigned)(at / chunks), c = (unsigned)(at % chunks);
  while (row < rows) {
    const int n = cols - (int)(8 * c);
    const Chunk<T> xc = load_chunk(x + (size_t)row * ldx + 8 * (size_t)c, n);
    f32x8 y;
    if (r) {
      const Chunk<T> rc = load_chunk(r + (size_t)row * ldr + 8 * (size_t)c, n);
      y = widen(rc) + gen.apply(widen(xc), c, row);
    } else {
      y = gen.apply(widen(xc), c, row);
    }
    store_chunk(out + (size_t)row * ldo + 8 * (size_t)c, n, y);
    row += step_rows;
    c += step_chunks;
    if (c >= chunks) {
      c -= chunks;
      row++;
    }
  }
}

// ---------------------------------------------------------------- layer norm

// N sums over the L lanes of a row (16, 64, or whole waves of a workgroup of L threads); every lane gets the same bits.  `red`: N floats for each wave,
// which may be written again once all waves have passed another barrier.
template <int CTRL>
__device__ __forceinline__ float dpp_add(float x) {
  return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
template <int L>
__device__ __forceinline__ float wave_sum(float x) {
  x = dpp_add<0xB1>(x);    // lane ^ 1
  x = dpp_add<0x4E>(x);    // lane ^ 2
  x = dpp_add<0x141>(x);   // the other four of eight
  x = dpp_add<0x140>(x);   // the other eight of sixteen
  if constexpr (L >= 64) {
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = half_sum(__uint_as_float(p[0]) + __uint_as_float(p[1]));
  }
  return x;
}
template <int L, int N>
__device__ __forceinline__ void row_sums(float (&x)[N], float (*red)[N]) {
#pragma unroll
  for (int k = 0; k < N; k++) x[k] = wave_sum<L>(x[k]);
  if constexpr (L > 64) {
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int k = 0; k < N; k++) red[threadIdx.x >> 6][k] = x[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; k++) x[k] = red[0][k];
#pragma unroll
    for (int w = 1; w < L / 64; w++)
#pragma unroll
      for (int k = 0; k < N; k++) x[k] += red[w][k];
  }
}

constexpr int row_threads(int L) { return L > 256 ? L : 256; }
// L lanes hold a row, NC chunks each: lane l the chunks l, l + L, ...
template <int L, int NC>
struct Rows {
  static constexpr int THREADS = row_threads(L), PER_GROUP = THREADS / L, WAVES = THREADS / 64, COLS = 8 * L * NC;
};

template <typename T, int L, int NC, bool SUM>
__global__ void __launch_bounds__(row_threads(L)) layer_norm_fwd_kernel(NormFwd a) {
  using R = Rows<L, NC>;
  __shared__ float red[2][R::WAVES][1];
  const int l = threadIdx.x % L, sub = threadIdx.x / L;
  const T *const x = (const T*)a.x, *const r = (const T*)a.r;
  T *const s = (T*)a.s, *const y = (T*)a.y;
  int n[NC];
  f32x8 gamma[NC], beta[NC];
#pragma unroll
  for (int i = 0; i < NC; i++) {
    n[i] = a.cols - 8 * (l + L * i);
    gamma[i] = widen(load_chunk(a.gamma + 8 * (l + L * i), n[i]));
    beta[i] = widen(load_chunk(a.beta + 8 * (l + L * i), n[i]));
  }
  const Generator gen(a.drop);
  const float over = 1.f / (float)a.cols;
  for (unsigned row = blockIdx.x * R::PER_GROUP + sub; row < (unsigned)a.rows; row += gridDim.x * R::PER_GROUP) {
    f32x8 v[NC];
    Chunk<T> xc[NC], rc[NC];
#pragma unroll
    for (int i = 0; i < NC; i++) {
      xc[i] = load_chunk(x + (size_t)row * a.ldx + 8 * (l + L * i), n[i]);
      if (SUM) rc[i] = load_chunk(r + (size_t)row * a.ldr + 8 * (l + L * i), n[i]);
    }
    float sum[1] = {0.f}, var[1] = {0.f};
#pragma unroll
    for (int i = 0; i < NC; i++) {
      v[i] = widen(xc[i]);
      if (SUM) {
        v[i] = widen(rc[i]) + gen.apply(v[i], l + L * i, row);
        store_chunk(s + (size_t)row * a.lds + 8 * (l + L * i), n[i], v[i]);
      }
#pragma unroll
      for (int e = 0; e < 8; e++) sum[0] += v[i][e];   // columns that do not exist are zero
    }
    // the statistics are those of the fp32 sum, not of its rounded copy in s; two passes over registers: no cancellation
    row_sums<L>(sum, red[0]);
    const float mean = sum[0] * over;
#pragma unroll
    for (int i = 0; i < NC; i++)
#pragma unroll
      for (int e = 0; e < 8; e++) {
        v[i][e] -= mean;
        if (e < n[i]) var[0] = fmaf(v[i][e], v[i][e], var[0]);
      }
    row_sums<L>(var, red[1]);
    const float rstd = 1.f / sqrtf(fmaf(var[0], over, a.eps));
#pragma unroll
    for (int i = 0; i < NC; i++) store_chunk(y + (size_t)row * a.ldy + 8 * (l + L * i), n[i], v[i] * rstd * gamma[i] + beta[i]);
    if (l == 0 && a.mean) a.mean[row] = mean;
    if (l == 0 && a.rstd) a.rstd[row] = rstd;
  }
}

// Gradient.  With xh = (x - mean) * rstd and g = dy * gamma:
//   dx = rstd * (g - mean(g) - xh * mean(g * xh)),   dgamma = sum over rows of dy * xh,   dbeta = sum over rows of dy.
// SUM (x is the sum s): what came to s directly, ds, is added, and dx = keep * scale * dr for the branch that was dropped out.
// A thread keeps its columns' sums over the rows of its workgroup; they go to `partial` [gridDim.x][2][cols], which
// sum_partials_kernel adds up in a fixed order.
template <typename T, int L, int NC, bool SUM>
__global__ void __launch_bounds__(row_threads(L)) layer_norm_bwd_kernel(NormBwd a) {
  using R = Rows<L, NC>;
  __shared__ float red[2][R::WAVES][2];
  const int l = threadIdx.x % L, sub = threadIdx.x / L;
  const T *const x = (const T*)a.x, *const dy = (const T*)a.dy, *const ds = (const T*)a.ds;
  T *const dx = (T*)a.dx, *const dr = (T*)a.dr;
  int n[NC];
  f32x8 dgamma[NC], dbeta[NC];
  // 1024 threads have 128 registers each, too few for gamma beside the sums: there it waits in LDS, 16 bytes to a lane and access
  constexpr bool IN_LDS = L == 1024;
  __shared__ f32x4 gamma_lds[IN_LDS ? 2 * NC : 1][IN_LDS ? L : 1];
  f32x8 gamma_reg[IN_LDS ? 1 : NC];
#pragma unroll
  for (int i = 0; i < NC; i++) {
    n[i] = a.cols - 8 * (l + L * i);
    const f32x8 g = widen(load_chunk(a.gamma + 8 * (l + L * i), n[i]));
    if constexpr (IN_LDS) {   // a lane reads what it wrote itself: no barrier
      gamma_lds[2 * i][l] = __builtin_shufflevector(g, g, 0, 1, 2, 3);
      gamma_lds[2 * i + 1][l] = __builtin_shufflevector(g, g, 4, 5, 6, 7);
    } else {
      gamma_reg[i] = g;
    }
    dgamma[i] = dbeta[i] = 0.f;
  }
  constexpr bool LATE = IN_LDS;   // for the same reason ds is read where it is added
  auto gamma = [&](int i) __attribute__((always_inline)) {
    if constexpr (IN_LDS) return __builtin_shufflevector(gamma_lds[2 * i][l], gamma_lds[2 * i + 1][l], 0, 1, 2, 3, 4, 5, 6, 7);
    else return gamma_reg[i];
  };
  const Generator gen(a.drop);
  const float over = 1.f / (float)a.cols;
  int turn = 0;
  for (unsigned row = blockIdx.x * R::PER_GROUP + sub; row < (unsigned)a.rows; row += gridDim.x * R::PER_GROUP) {
    Chunk<T> xc[NC], gc[NC], sc[NC];
    const float mean = a.mean[row], rstd = a.rstd[row];
#pragma unroll
    for (int i = 0; i < NC; i++) {
      gc[i] = load_chunk(dy + (size_t)row * a.lddy + 8 * (l + L * i), n[i]);
      xc[i] = load_chunk(x + (size_t)row * a.ldx + 8 * (l + L * i), n[i]);
      if (SUM && !LATE && ds) sc[i] = load_chunk(ds + (size_t)row * a.ldds + 8 * (l + L * i), n[i]);
    }
    float sums[2] = {0.f, 0.f};   // of g and of g * xh
#pragma unroll
    for (int i = 0; i < NC; i++) {
      const f32x8 d = widen(gc[i]), xh = (widen(xc[i]) - mean) * rstd, gm = gamma(i);
      dbeta[i] += d;
#pragma unroll
      for (int e = 0; e < 8; e++) {   // dy and gamma are zero in columns that do not exist
        dgamma[i][e] = fmaf(d[e], xh[e], dgamma[i][e]);
        const float g = d[e] * gm[e];
        sums[0] += g;
        sums[1] = fmaf(g, xh[e], sums[1]);
      }
    }
    row_sums<L>(sums, red[turn]);
    turn ^= 1;
    const float mean_g = sums[0] * over, mean_gx = sums[1] * over;
#pragma unroll
    for (int i = 0; i < NC; i++) {
      f32x8 d = (widen(gc[i]) * gamma(i) - mean_g - (widen(xc[i]) - mean) * rstd * mean_gx) * rstd;
      if (SUM) {
        if (LATE && ds) sc[i] = load_chunk(ds + (size_t)row * a.ldds + 8 * (l + L * i), n[i]);
        if (ds) d += widen(sc[i]);
        store_chunk(dr + (size_t)row * a.lddr + 8 * (l + L * i), n[i], d);
        d = gen.apply(d, l + L * i, row);
      }
      store_chunk(dx + (size_t)row * a.lddx + 8 * (l + L * i), n[i], d);
    }
  }
  float* const out = a.partial + (size_t)blockIdx.x * 2 * a.cols;
  if constexpr (R::PER_GROUP == 1) {
#pragma unroll
    for (int i = 0; i < NC; i++) {
      store_chunk(out + 8 * (l + L * i), n[i], dgamma[i]);
      store_chunk(out + a.cols + 8 * (l + L * i), n[i], dbeta[i]);
    }
  } else {
    __shared__ float all[R::PER_GROUP][R::COLS];
#pragma unroll
    for (int which = 0; which < 2; which++) {
      if (which) __syncthreads();
#pragma unroll
      for (int i = 0; i < NC; i++)
#pragma unroll
        for (int e = 0; e < 8; e++) all[sub][8 * (l + L * i) + e] = which ? dbeta[i][e] : dgamma[i][e];
      __syncthreads();
      for (int c = threadIdx.x; c < a.cols; c += R::THREADS) {
        float t = all[0][c];
#pragma unroll
        for (int g = 1; g < R::PER_GROUP; g++) t += all[g][c];
        out[which * a.cols + c] = t;
      }
    }
  }
}

// dgamma and dbeta: the sums of `groups` slabs of 2 * cols floats.  32 columns to a workgroup, eight threads to a column.
__global__ void __launch_bounds__(256) sum_partials_kernel(const float* __restrict__ partial, int groups, int cols, float* __restrict__ dgamma, float* __restrict__ dbeta) {
  __shared__ float all[8][32];
  const int lane = threadIdx.x & 31, part = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + lane;
  float t = 0.f;
  if (c < 2 * cols)
    for (int g = part; g < groups; g += 8) t += partial[(size_t)g * 2 * cols + c];
  all[part][lane] = t;
  __syncthreads();
  if (part == 0 && c < 2 * cols) {
#pragma unroll
    for (int p = 1; p < 8; p++) t += all[p][lane];
    if (c < cols) dgamma[c] = t;
    else dbeta[c - cols] = t;
  }
}

template <typename T, int L, int NC>
hipError_t launch_fwd_rows(const NormFwd& a, hipStream_t stream) {
  using R = Rows<L, NC>;
  const long long groups = ((long long)a.rows + R::PER_GROUP - 1) / R::PER_GROUP;
  const unsigned grid = (unsigned)std::min<long long>(groups, norm_groups_at_once(R::THREADS));
  if (a.s) hipLaunchKernelGGL((layer_norm_fwd_kernel<T, L, NC, true>), dim3(grid), dim3(R::THREADS), 0, stream, a);
  else hipLaunchKernelGGL((layer_norm_fwd_kernel<T, L, NC, false>), dim3(grid), dim3(R::THREADS), 0, stream, a);
  return hipGetLastError();
}
template <typename T, int L, int NC>
hipError_t launch_bwd_rows(const NormBwd& a, hipStream_t stream) {
  using R = Rows<L, NC>;
  const unsigned grid = (unsigned)norm_bwd_groups(a.rows, a.cols);
  if (a.dr) hipLaunchKernelGGL((layer_norm_bwd_kernel<T, L, NC, true>), dim3(grid), dim3(R::THREADS), 0, stream, a);
  else hipLaunchKernelGGL((layer_norm_bwd_kernel<T, L, NC, false>), dim3(grid), dim3(R::THREADS), 0, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(sum_partials_kernel, dim3((unsigned)((2 * a.cols + 31) / 32)), dim3(256), 0, stream, a.partial, (int)grid, a.cols, a.dgamma, a.dbeta);
  return hipGetLastError();
}

template <typename T>
hipError_t norm_fwd(const NormFwd& a, hipStream_t stream) {
  switch (norm_rows(a.cols)) {
    case NormRows::k16x2: return launch_fwd_rows<T, 16, 2>(a, stream);
    case NormRows::k64x2: return launch_fwd_rows<T, 64, 2>(a, stream);
    case NormRows::k256x1: return launch_fwd_rows<T, 256, 1>(a, stream);
    case NormRows::k256x2: return launch_fwd_rows<T, 256, 2>(a, stream);
    case NormRows::k512x2: return launch_fwd_rows<T, 512, 2>(a, stream);
    default: return launch_fwd_rows<T, 1024, 2>(a, stream);
  }
}
template <typename T>
hipError_t norm_bwd(const NormBwd& a, hipStream_t stream) {
  switch (norm_rows(a.cols)) {
    case NormRows::k16x2: return launch_bwd_rows<T, 16, 2>(a, stream);
    case NormRows::k64x2: return launch_bwd_rows<T, 64, 2>(a, stream);
    case NormRows::k256x1: return launch_bwd_rows<T, 256, 1>(a, stream);
    case NormRows::k256x2: return launch_bwd_rows<T, 256, 2>(a, stream);
    case NormRows::k512x2: return launch_bwd_rows<T, 512, 2>(a, stream);
    default: return launch_bwd_rows<T, 1024, 2>(a, stream);
  }
}

template <typename T>
hipError_t dropout_add(const void* x, long long ldx, const void* r, long long ldr, void* out, long long ldo, int rows, int cols, const Dropout& drop, hipStream_t stream) {
  const long long chunks = (cols + 7) / 8, total = chunks * rows;
  const long long grid = std::min<long long>((total + 255) / 256, 2048);
  const long long step = grid * 256;
  hipLaunchKernelGGL((dropout_add_kernel<T>), dim3((unsigned)grid), dim3(256), 0, stream, (const T*)x, ldx, (const T*)r, ldr, (T*)out, ldo, (unsigned)rows, cols, drop,
                     (unsigned)(step / chunks), (unsigned)(step % chunks));
  return hipGetLastError();
}

}  // namespace

hipError_t launch_dropout_add(const void* x, long long ldx, const void* r, long long ldr, void* out, long long ldo, int rows, int cols, ElementType type,
                              const Dropout& drop, hipStream_t stream) {
  switch (type) {
    case ElementType::bf16: return dropout_add<__bf16>(x, ldx, r, ldr, out, ldo, rows, cols, drop, stream);
    case ElementType::f16: return dropout_add<_Float16>(x, ldx, r, ldr, out, ldo, rows, cols, drop, stream);
    default: return dropout_add<float>(x, ldx, r, ldr, out, ldo, rows, cols, drop, stream);
  }
}
hipError_t launch_norm_fwd(const NormFwd& a, ElementType type, hipStream_t stream) {
  switch (type) {
    case ElementType::bf16: return norm_fwd<__bf16>(a, stream);
    case ElementType::f16: return norm_fwd<_Float16>(a, stream);
    default: return norm_fwd<float>(a, stream);
  }
}
hipError_t launch_norm_bwd(const NormBwd& a, ElementType type, hipStream_t stream) {
  switch (type) {
    case ElementType::bf16: return norm_bwd<__bf16>(a, stream);
    case ElementType::f16: return norm_bwd<_Float16>(a, stream);
    default: return norm_bwd<float>(a, stream);
  }
}

}  // namespace helix
