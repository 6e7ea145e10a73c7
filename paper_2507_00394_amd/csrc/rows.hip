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
// `n` of the 8 elements exist; the others are read as zero and not written.  A lane's 16 bytes go past the caches, which have no use for them (dropout and sum of
// 32768 x 4096 bf16 158 -> 143 us); the 32 bytes of a 4-byte type are two accesses to a line, which they had better join (20000 x 4001 fp32 197 us, 218 past them).
template <typename T>
__device__ __forceinline__ Chunk<T> load_chunk(const T* p, int n) {
  Chunk<T> c;
  c.v = (T)0.f;
  if (n >= 8) {
    const auto* const q = reinterpret_cast<const typename Chunk<T>::Vec*>(p);
    if constexpr (sizeof(T) == 2) c.v = __builtin_nontemporal_load(q);
    else c.v = *q;
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
    auto* const q = reinterpret_cast<typename Chunk<T>::Vec*>(p);
    if constexpr (sizeof(T) == 2) __builtin_nontemporal_store(v, q);
    else *q = v;
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
__device__ __forceinline__ void row_sums(float (&x)[N], float (*red)[N]) {   // red: this row's
#pragma unroll
  for (int k = 0; k < N; k++) x[k] = wave_sum<L>(x[k]);
  if constexpr (L > 64) {
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int k = 0; k < N; k++) red[threadIdx.x % L >> 6][k] = x[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; k++) x[k] = red[0][k];
#pragma unroll
    for (int w = 1; w < L / 64; w++)
#pragma unroll
      for (int k = 0; k < N; k++) x[k] += red[w][k];
  }
}

// L lanes hold a row of the matrix, NC chunks each: lane l the chunks l, l + L, ... as far as they are whole.  The columns behind the last whole chunk, seven at
// most, are one each with the first lanes ("tail"): what a lane does for a chunk has no case for a part of one, which would be most of the code.
template <int L, int NC>
struct Columns {
  int l, tail, tail_at;   // tail_at: column of this lane's element behind the chunks
  bool has[NC], has_tail;
  uint32_t first;         // column of its first chunk
  __device__ __forceinline__ explicit Columns(int cols) : l(threadIdx.x % L), tail(cols & 7), tail_at((cols & ~7) + l), has_tail(l < tail), first(8 * l) {
#pragma unroll
    for (int i = 0; i < NC; i++) has[i] = 8 * (l + L * i) + 8 <= cols;
  }
  template <typename T>
  __device__ __forceinline__ Chunk<T> load(const T* row, int i) const {
    Chunk<T> c;
    c.v = (T)0.f;
    if (has[i]) c.v = *reinterpret_cast<const typename Chunk<T>::Vec*>(row + (first + 8 * L * i));
    return c;
  }
  // ONCE: results that the caches need not keep, as in store_chunk (8192 x 5001 50 -> 35 us, dropout, sum and norm of 20000 x 900 36 -> 28).  Loads past the caches are no
  // gain here: 192 -> 183 us for dropout, sum and norm of 32768 x 4096, but 35 -> 47 at 8192 x 5001, whose lines two lanes or two waves read.
  template <bool ONCE = false, typename T>
  __device__ __forceinline__ void store(T* row, int i, const f32x8& x) const {
    auto* const p = reinterpret_cast<typename Chunk<T>::Vec*>(row + (first + 8 * L * i));
    const auto v = __builtin_convertvector(x, typename Chunk<T>::Vec);
    if (has[i]) {
      if constexpr (ONCE && sizeof(T) == 2) __builtin_nontemporal_store(v, p);
      else *p = v;
    }
  }
  template <typename T>
  __device__ __forceinline__ float load_tail(const T* row) const { return has_tail ? (float)row[tail_at] : 0.f; }
  template <typename T>
  __device__ __forceinline__ void store_tail(T* row, float x) const {
    if (has_tail) row[tail_at] = (T)x;
  }
  __device__ __forceinline__ uint32_t chunk(int i) const { return l + L * i; }
  // keep * x * scale for this lane's element of the tail
  __device__ __forceinline__ float apply_tail(const Generator& gen, float x, uint32_t row) const {
    if (!gen.cut) return x;
    const u32x4 bits = gen.block(tail_at >> 3, row);
    const uint32_t w = tail_at & 4 ? (tail_at & 2 ? bits[3] : bits[2]) : (tail_at & 2 ? bits[1] : bits[0]);
    return (tail_at & 1 ? w >> 16 : w & 0xffffu) >= gen.cut ? x * gen.scale : 0.f;
  }
};
// Which of a workgroup's rows this lane works on: in a scalar register where a wave has no other, and with it the rows' addresses.
template <int L>
__device__ __forceinline__ int row_of_lane() {
  if constexpr (L >= 64) return __builtin_amdgcn_readfirstlane(threadIdx.x / L);
  else return threadIdx.x / L;
}
constexpr int row_threads(int L) { return L > 256 ? L : 256; }

template <typename T, int L, int NC, bool SUM>
__global__ void __launch_bounds__(row_threads(L)) __attribute__((amdgpu_waves_per_eu(norm_fwd_waves(L, NC, SUM), norm_fwd_waves(L, NC, SUM)))) layer_norm_fwd_kernel(NormFwd a) {
  constexpr int TOGETHER = row_threads(L) / L;
  __shared__ float red[2][row_threads(L) / 64][1];
  const int sub = row_of_lane<L>();
  const Columns<L, NC> at(a.cols);
  f32x8 gamma[NC], beta[NC];
#pragma unroll
  for (int i = 0; i < NC; i++) {
    gamma[i] = widen(at.load(a.gamma, i));
    beta[i] = widen(at.load(a.beta, i));
  }
  const float gamma_tail = at.load_tail(a.gamma), beta_tail = at.load_tail(a.beta);
  const Generator gen(a.drop);
  const float over = 1.f / (float)a.cols;
  for (unsigned row = blockIdx.x * TOGETHER + sub; row < (unsigned)a.rows; row += gridDim.x * TOGETHER) {
    const T *const x = (const T*)a.x + (size_t)row * a.ldx, *const r = (const T*)a.r + (size_t)row * a.ldr;
    T *const s = (T*)a.s + (size_t)row * a.lds, *const y = (T*)a.y + (size_t)row * a.ldy;
    f32x8 v[NC];
    float vt = 0.f;
    Chunk<T> xc[NC], rc[NC];
#pragma unroll
    for (int i = 0; i < NC; i++) {
      xc[i] = at.load(x, i);
      if (SUM) rc[i] = at.load(r, i);
    }
    if (at.tail) {
      vt = at.load_tail(x);
      if (SUM) {
        vt = at.load_tail(r) + at.apply_tail(gen, vt, row);
        at.store_tail(s, vt);
      }
    }
    float sum[1] = {vt}, var[1] = {0.f};
#pragma unroll
    for (int i = 0; i < NC; i++) {
      v[i] = widen(xc[i]);
      if (SUM) {
        v[i] = widen(rc[i]) + gen.apply(v[i], at.chunk(i), row);
        at.template store<true>(s, i, v[i]);
      }
#pragma unroll
      for (int e = 0; e < 8; e++) sum[0] += v[i][e];   // columns that do not exist are zero
    }
    // the statistics are those of the fp32 sum, not of its rounded copy in s; two passes over registers: no cancellation
    row_sums<L>(sum, red[0]);
    const float mean = sum[0] * over;
#pragma unroll
    for (int i = 0; i < NC; i++) {
      v[i] -= mean;
      if (at.has[i])
#pragma unroll
        for (int e = 0; e < 8; e++) var[0] = fmaf(v[i][e], v[i][e], var[0]);
    }
    vt -= mean;
    if (at.has_tail) var[0] = fmaf(vt, vt, var[0]);
    row_sums<L>(var, red[1]);
    const float rstd = 1.f / sqrtf(fmaf(var[0], over, a.eps));
#pragma unroll
    for (int i = 0; i < NC; i++) at.template store<true>(y, i, v[i] * rstd * gamma[i] + beta[i]);
    if (at.tail) at.store_tail(y, vt * rstd * gamma_tail + beta_tail);
    if (at.l == 0 && a.mean) a.mean[row] = mean;
    if (at.l == 0 && a.rstd) a.rstd[row] = rstd;
  }
}

// Gradient.  With xh = (x - mean) * rstd and g = dy * gamma:
//   dx = rstd * (g - mean(g) - xh * mean(g * xh)),   dgamma = sum over rows of dy * xh,   dbeta = sum over rows of dy.
// SUM (x is the sum s): what came to s directly, ds, is added, and dx = keep * scale * dr for the branch that was dropped out.
//
// A lane keeps its columns' sums over all rows that it works on.  A compute unit has one workgroup, of as many rows at a time as it has waves for, so that
// few partial sums are left: the workgroup adds up its rows' and leaves one slab, `partial` [gridDim.x][2][cols], and sum_partials_kernel adds the slabs up in a fixed
// order (16384 x 2048 bf16: 73 us with four workgroups of 256 threads on a compute unit, 1024 slabs and a thread's loads of them one after the other, 45 now, 4.9 TB/s of
// the main kernel; 131072 x 4096 with dropout and sum 985, 5.45 TB/s).  Up to 1024 columns a row is in one wave at most and needs no barrier.  gamma waits in LDS for all
// rows: its registers are the sums'.
template <typename T, int L, int NC, bool SUM>
__global__ void __launch_bounds__(kNormBwdThreads) layer_norm_bwd_kernel(NormBwd a) {
  constexpr int COLS = 8 * L * NC, MOST = kNormBwdThreads / L;   // MOST rows at a time
  __shared__ __align__(16) float lds[(MOST > 1 ? 2 * (MOST / 2) : 1) * COLS];   // gamma; at the end the sums of half of the rows
  __shared__ float red[2][kNormBwdThreads / 64][2], tails[2][MOST][8];
  const int sub = row_of_lane<L>(), together = blockDim.x / L;
  const Columns<L, NC> at(a.cols);
  f32x8 dgamma[NC], dbeta[NC];
  // a chunk is two halves of 16 bytes, L lanes' first halves one behind the other, then their second ones
  if (sub == 0)
#pragma unroll
    for (int i = 0; i < NC; i++) {
      const f32x8 g = widen(at.load(a.gamma, i));
      f32x4* const to = reinterpret_cast<f32x4*>(lds) + 2 * i * L + at.l;
      to[0] = __builtin_shufflevector(g, g, 0, 1, 2, 3);
      to[L] = __builtin_shufflevector(g, g, 4, 5, 6, 7);
    }
  auto gamma_of = [&](int i, int lane) __attribute__((always_inline)) {
    const f32x4* const p = reinterpret_cast<const f32x4*>(lds) + 2 * i * L + lane;
    return __builtin_shufflevector(p[0], p[L], 0, 1, 2, 3, 4, 5, 6, 7);
  };
#pragma unroll
  for (int i = 0; i < NC; i++) dgamma[i] = dbeta[i] = 0.f;
  const float gamma_tail = at.load_tail(a.gamma);
  float dgamma_tail = 0.f, dbeta_tail = 0.f;
  const Generator gen(a.drop);
  const float over = 1.f / (float)a.cols;
  int turn = 0;
  __syncthreads();
  for (unsigned first = blockIdx.x * together; first < (unsigned)a.rows; first += gridDim.x * together) {
    const unsigned row = first + sub;
    if (row >= (unsigned)a.rows) {   // in the last turn only
      if constexpr (L > 64) __syncthreads();   // that of row_sums
      continue;
    }
    const T *const dy = (const T*)a.dy + (size_t)row * a.lddy, *const x = (const T*)a.x + (size_t)row * a.ldx;
    Chunk<T> xc[NC], gc[NC];
    float xt = 0.f, gt = 0.f;
    const float mean = a.mean[row], rstd = a.rstd[row];
#pragma unroll
    for (int i = 0; i < NC; i++) {
      gc[i] = at.load(dy, i);
      xc[i] = at.load(x, i);
    }
    float sums[2] = {0.f, 0.f};   // of g and of g * xh
    int lane = at.l;
    pin(lane);   // gamma is read here, not once for all rows into registers
    if (at.tail) {
      xt = at.has_tail ? (at.load_tail(x) - mean) * rstd : 0.f;
      gt = at.load_tail(dy);
      dgamma_tail = fmaf(gt, xt, dgamma_tail);
      dbeta_tail += gt;
      gt *= gamma_tail;
      sums[0] = gt;
      sums[1] = gt * xt;
    }
#pragma unroll
    for (int i = 0; i < NC; i++) {
      // in columns that do not exist dy, gamma and xh are zero: mean * rstd may leave the range of fp32 where no x - mean does
      const f32x8 d = widen(gc[i]), xh = (widen(xc[i]) - (at.has[i] ? mean : 0.f)) * rstd, gamma = gamma_of(i, lane);
      dbeta[i] += d;
#pragma unroll
      for (int e = 0; e < 8; e++) {
        dgamma[i][e] = fmaf(d[e], xh[e], dgamma[i][e]);
        const float g = d[e] * gamma[e];
        sums[0] += g;
        sums[1] = fmaf(g, xh[e], sums[1]);
      }
      pin(dgamma[i]);   // added here, not when the row is finished
      pin(dbeta[i]);
    }
    row_sums<L>(sums, red[turn] + (L > 64 ? sub * (L / 64) : 0));
    turn ^= 1;
    T* const dx = (T*)a.dx + (size_t)row * a.lddx;
    const float mean_g = sums[0] * over, mean_gx = sums[1] * over;
    pin(lane);
#pragma unroll
    for (int i = 0; i < NC; i++) {   // what is made of them above is made again: it would take twice their registers
      pin(xc[i].v);
      pin(gc[i].v);
    }
#pragma unroll
    for (int i = 0; i < NC; i++) {
      f32x8 d = (widen(gc[i]) * gamma_of(i, lane) - mean_g - (widen(xc[i]) - mean) * rstd * mean_gx) * rstd;
      if (SUM) {
        if (a.ds) d += widen(at.load((const T*)a.ds + (size_t)row * a.ldds, i));
        at.template store<true>((T*)a.dr + (size_t)row * a.lddr, i, d);
        d = gen.apply(d, at.chunk(i), row);
      }
      at.template store<true>(dx, i, d);
    }
    if (at.tail) {
      float d = (gt - mean_g - xt * mean_gx) * rstd;
      if (SUM) {
        if (a.ds) d += at.load_tail((const T*)a.ds + (size_t)row * a.ldds);
        at.store_tail((T*)a.dr + (size_t)row * a.lddr, d);
        d = at.apply_tail(gen, d, row);
      }
      at.store_tail(dx, d);
    }
  }
  const bool alone = gridDim.x == 1;   // these are the results
  if (at.has_tail) {
    tails[0][sub][at.l] = dgamma_tail;
    tails[1][sub][at.l] = dbeta_tail;
  }
  for (int left = together; left > 1; left = (left + 1) / 2) {   // the upper half of the rows' sums is added to the lower
    const int half = (left + 1) / 2;
    __syncthreads();
    f32x4* const mine = reinterpret_cast<f32x4*>(lds) + (size_t)(sub >= half ? sub - half : sub) * (COLS / 2) + at.l;
    if (sub >= half && sub < left)
#pragma unroll
      for (int i = 0; i < 2 * NC; i++) {
        const f32x8& sum = i < NC ? dgamma[i % NC] : dbeta[i % NC];
        mine[2 * i * L] = __builtin_shufflevector(sum, sum, 0, 1, 2, 3);
        mine[(2 * i + 1) * L] = __builtin_shufflevector(sum, sum, 4, 5, 6, 7);
      }
    __syncthreads();
    if (sub + half < left)
#pragma unroll
      for (int i = 0; i < 2 * NC; i++) (i < NC ? dgamma[i % NC] : dbeta[i % NC]) += __builtin_shufflevector(mine[2 * i * L], mine[(2 * i + 1) * L], 0, 1, 2, 3, 4, 5, 6, 7);
  }
  if (sub != 0) return;
#pragma unroll
  for (int which = 0; which < 2; which++) {
    float* const out = alone ? (which ? a.dbeta : a.dgamma) : a.partial + ((size_t)blockIdx.x * 2 + which) * a.cols;
#pragma unroll
    for (int i = 0; i < NC; i++) at.store(out, i, which ? dbeta[i] : dgamma[i]);
    if (at.has_tail) {   // written above, in front of a barrier unless this is the only row
      float t = tails[which][0][at.l];
      for (int g = 1; g < together; g++) t += tails[which][g][at.l];
      at.store_tail(out, t);
    }
  }
}

// dgamma and dbeta: the sums of `groups` slabs of 2 * cols floats.  32 columns to a workgroup, 32 threads to a column, eight loads of each in flight: it is
// latency that counts here (eight threads to a column and a load at a time: 33 us for 1024 slabs of 2 x 2048 columns).
constexpr int kSumParts = 32;
__global__ void __launch_bounds__(32 * kSumParts) sum_partials_kernel(const float* __restrict__ partial, int groups, int cols, float* __restrict__ dgamma, float* __restrict__ dbeta) {
  __shared__ float all[kSumParts][32];
  const int lane = threadIdx.x & 31, part = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + lane;
  float t[8] = {};
  if (c < 2 * cols)
    for (int g = part; g < groups; g += 8 * kSumParts)
#pragma unroll
      for (int u = 0; u < 8; u++)
        if (g + u * kSumParts < groups) t[u] += partial[(size_t)(g + u * kSumParts) * 2 * cols + c];
  all[part][lane] = ((t[0] + t[1]) + (t[2] + t[3])) + ((t[4] + t[5]) + (t[6] + t[7]));
  __syncthreads();
  if (part == 0 && c < 2 * cols) {
    float sum = all[0][lane];
#pragma unroll
    for (int p = 1; p < kSumParts; p++) sum += all[p][lane];
    if (c < cols) dgamma[c] = sum;
    else dbeta[c - cols] = sum;
  }
}

template <typename T, int L, int NC>
hipError_t launch_fwd_rows(const NormFwd& a, hipStream_t stream) {
  constexpr int THREADS = row_threads(L), TOGETHER = THREADS / L;
  const long long groups = ((long long)a.rows + TOGETHER - 1) / TOGETHER;
  const unsigned grid = (unsigned)std::min<long long>(groups, groups_at_once(THREADS, norm_fwd_waves(L, NC, a.s != nullptr)));
  if (a.s) hipLaunchKernelGGL((layer_norm_fwd_kernel<T, L, NC, true>), dim3(grid), dim3(THREADS), 0, stream, a);
  else hipLaunchKernelGGL((layer_norm_fwd_kernel<T, L, NC, false>), dim3(grid), dim3(THREADS), 0, stream, a);
  return hipGetLastError();
}
template <typename T, int L, int NC>
hipError_t launch_bwd_rows(const NormBwd& a, hipStream_t stream) {
  const int together = norm_bwd_together(a.rows, a.cols), grid = norm_bwd_groups(a.rows, a.cols);
  if (a.dr) hipLaunchKernelGGL((layer_norm_bwd_kernel<T, L, NC, true>), dim3((unsigned)grid), dim3((unsigned)(together * L)), 0, stream, a);
  else hipLaunchKernelGGL((layer_norm_bwd_kernel<T, L, NC, false>), dim3((unsigned)grid), dim3((unsigned)(together * L)), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || grid == 1) return e;
  hipLaunchKernelGGL(sum_partials_kernel, dim3((unsigned)((2 * a.cols + 31) / 32)), dim3(32 * kSumParts), 0, stream, a.partial, grid, a.cols, a.dgamma, a.dbeta);
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
  switch (norm_bwd_rows(a.cols)) {
    case NormBwdRows::k16x2: return launch_bwd_rows<T, 16, 2>(a, stream);
    case NormBwdRows::k64x2: return launch_bwd_rows<T, 64, 2>(a, stream);
    case NormBwdRows::k128x2: return launch_bwd_rows<T, 128, 2>(a, stream);
    case NormBwdRows::k256x2: return launch_bwd_rows<T, 256, 2>(a, stream);
    case NormBwdRows::k512x2: return launch_bwd_rows<T, 512, 2>(a, stream);
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
