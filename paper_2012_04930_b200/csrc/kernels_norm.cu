// Layer norm over the rows of a matrix, forward and backward, and 8-bit checkpoints of activations (pack8_device.h).
//
// All of these read and write whole matrices once and compute little, so memory bounds them: a row is loaded once, stays in
// registers through its sums, and is written once.  A row belongs to a team of T threads (8, 16 or 32 lanes, or a block of
// 256) that holds NV float4 of it each; a warp works on 32 / T rows at a time, times R where rows are short.
#include <cuda_runtime.h>

#include <algorithm>

#include "internal.h"
#include "launch.h"
#include "pack8_device.h"

namespace gcnsa {

namespace {

constexpr unsigned kFull = 0xffffffffu;
constexpr int kNormThreads = 256;
constexpr int kNormMaxCols = 8192;  // columns that 256 threads hold in registers

// Column k of chunk v of thread t: four neighbours to a thread where rows take 16-byte accesses, neighbouring threads
// otherwise (one scalar access covers 128 bytes of a warp, and 32 / T of them by a narrower team are one block of a checkpoint).
template <int T, bool VEC>
__device__ __forceinline__ int col_of(int v, int k, int t) {
  return VEC ? 4 * (v * T + t) + k : (4 * v + k) * T + t;
}

template <int T, int NV, bool VEC>
__device__ __forceinline__ void load_row(const float* row, int f, int t, float (&x)[4 * NV]) {
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    if constexpr (VEC) {
      const int c = col_of<T, VEC>(v, 0, t);
      const float4 a = c < f ? *reinterpret_cast<const float4*>(row + c) : make_float4(0.f, 0.f, 0.f, 0.f);
      x[4 * v] = a.x;
      x[4 * v + 1] = a.y;
      x[4 * v + 2] = a.z;
      x[4 * v + 3] = a.w;
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int c = col_of<T, VEC>(v, k, t);
        x[4 * v + k] = c < f ? row[c] : 0.f;
      }
    }
  }
}
// ... and, when all loads of a row are under way, zeros for the pad columns in it, which may hold anything
template <int T, int NV, bool VEC>
__device__ __forceinline__ void clear_pads(int f, int t, float (&x)[4 * NV]) {
  if (VEC && (f & 3))
#pragma unroll
    for (int i = 0; i < 4 * NV; ++i) x[i] = col_of<T, VEC>(i / 4, i % 4, t) < f ? x[i] : 0.f;
}
// the row's pad columns up to the next multiple of 4 come out as zeros (n_pad)
template <int T, int NV, bool VEC>
__device__ __forceinline__ void store_row(float* row, int f, int n_pad, int t, const float (&x)[4 * NV]) {
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    if constexpr (VEC) {
      const int c = col_of<T, VEC>(v, 0, t);
      float4 a = make_float4(x[4 * v], x[4 * v + 1], x[4 * v + 2], x[4 * v + 3]);
      if (f & 3) {
        a.y = c + 1 < f ? a.y : 0.f;
        a.z = c + 2 < f ? a.z : 0.f;
        a.w = c + 3 < f ? a.w : 0.f;
      }
      if (c < f) *reinterpret_cast<float4*>(row + c) = a;
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int c = col_of<T, VEC>(v, k, t);
        if (c < n_pad) row[c] = c < f ? x[4 * v + k] : 0.f;
      }
    }
  }
}
// a row of a checkpoint; q rows lie on 16-byte boundaries and their pad columns up to the next multiple of 16 are zeros
struct PackedRows {
  int8_t* q = nullptr;
  int64_t ldq = 0;
  uint8_t* e = nullptr;
  int64_t lde = 0;
};
template <int T, int NV, bool VEC>
__device__ __forceinline__ void load_packed(const PackedRows& p, int64_t row, int f, int t, float (&x)[4 * NV]) {
  const int8_t* q = p.q + row * p.ldq;
  const uint8_t* e = p.e + row * p.lde;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    if constexpr (VEC) {
      const int c = col_of<T, VEC>(v, 0, t);
      const uint32_t q4 = c < f ? *reinterpret_cast<const uint32_t*>(q + c) : 0u;
      const float step = c < f ? pack8_step(e[c / kPackBlock]) : 0.f;
      float a[4];
      pack8_open(q4, a);  // (pad bytes are zeros)
#pragma unroll
      for (int k = 0; k < 4; ++k) x[4 * v + k] = a[k] * step;
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int c = col_of<T, VEC>(v, k, t);
        x[4 * v + k] = c < f ? (float)q[c] * pack8_step(e[c / kPackBlock]) : 0.f;
      }
    }
  }
}
// Every lane of the warp comes here (shuffles), `in` or not.
template <int T, int NV, bool VEC>
__device__ __forceinline__ void store_packed(const PackedRows& p, int64_t row, bool in, int f, int t, const float (&x)[4 * NV]) {
  int8_t* q = p.q + row * p.ldq;
  uint8_t* e = p.e + row * p.lde;
  const int f16 = (f + 15) / 16 * 16;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    if constexpr (VEC) {  // eight lanes hold a block
      const int c = col_of<T, VEC>(v, 0, t);
      float b[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) b[k] = c + k < f ? x[4 * v + k] : 0.f;
      uint32_t m = pack8_magnitude(b);
#pragma unroll
      for (int o = 1; o < 8; o <<= 1) m = max(m, __shfl_xor_sync(kFull, m, o));
      const uint32_t ex = pack8_exponent(m);
      if (in && c < f16) *reinterpret_cast<uint32_t*>(q + c) = pack8_bytes(b, ex);
      if (in && c < f && (t & 7) == 0) e[c / kPackBlock] = (uint8_t)ex;
    } else if constexpr (T < 32) {  // PK values of a team's lanes are a block
      constexpr int PK = 32 / T;
#pragma unroll
      for (int k0 = 0; k0 < 4; k0 += PK) {
        float a[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < PK; ++k) a[k] = col_of<T, VEC>(v, k0 + k, t) < f ? x[4 * v + k0 + k] : 0.f;
        uint32_t m = pack8_magnitude(a);
#pragma unroll
        for (int o = 1; o < T; o <<= 1) m = max(m, __shfl_xor_sync(kFull, m, o));
        const uint32_t ex = pack8_exponent(m);
        const uint32_t b = pack8_bytes(a, ex);
#pragma unroll
        for (int k = 0; k < PK; ++k) {
          const int c = col_of<T, VEC>(v, k0 + k, t);
          if (in && c < f16) q[c] = (int8_t)(b >> (8 * k));
        }
        const int c = col_of<T, VEC>(v, k0, t);
        if (in && c < f && t == 0) e[c / kPackBlock] = (uint8_t)ex;
      }
    } else {  // a warp holds a block
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int c = col_of<T, VEC>(v, k, t);
        const float a = c < f ? x[4 * v + k] : 0.f;
        const uint32_t ex = pack8_exponent(__reduce_max_sync(kFull, __float_as_uint(a) & 0x7fffffffu));
        const float b[4] = {a, 0.f, 0.f, 0.f};
        if (in && c < f16) q[c] = (int8_t)pack8_bytes(b, ex);
        if (in && c < f && (t & 31) == 0) e[c / kPackBlock] = (uint8_t)ex;
      }
    }
  }
}

// What the ReLU let through, a bit per value: bit c % 32 of word c / 32 of a row.
struct BitRows {
  uint32_t* w = nullptr;
  int64_t ld = 0;
};
// Every lane of the warp comes here (shuffles), `in` or not.
template <int T, int NV, bool VEC>
__device__ __forceinline__ void store_bits(const BitRows& p, int64_t row, bool in, int f, int t, const float (&y)[4 * NV]) {
  uint32_t* w = p.w + row * p.ld;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    if constexpr (VEC) {
      const int c = col_of<T, VEC>(v, 0, t);
      uint32_t b = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) b |= (c + k < f && y[4 * v + k] > 0.f ? 1u : 0u) << ((c + k) & 31);
#pragma unroll
      for (int o = 1; o < 8; o <<= 1) b |= __shfl_xor_sync(kFull, b, o);
      if (in && c < f && (t & 7) == 0) w[c / 32] = b;
    } else if constexpr (T < 32) {
      constexpr int PK = 32 / T;
#pragma unroll
      for (int k0 = 0; k0 < 4; k0 += PK) {
        uint32_t b = 0;
#pragma unroll
        for (int k = 0; k < PK; ++k) {
          const int c = col_of<T, VEC>(v, k0 + k, t);
          b |= (c < f && y[4 * v + k0 + k] > 0.f ? 1u : 0u) << (c & 31);
        }
#pragma unroll
        for (int o = 1; o < T; o <<= 1) b |= __shfl_xor_sync(kFull, b, o);
        const int c = col_of<T, VEC>(v, k0, t);
        if (in && c < f && t == 0) w[c / 32] = b;
      }
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int c = col_of<T, VEC>(v, k, t);
        const uint32_t b = __ballot_sync(kFull, c < f && y[4 * v + k] > 0.f);
        if (in && c < f && (t & 31) == 0) w[c / 32] = b;
      }
    }
  }
}
__device__ __forceinline__ bool bit_at(const BitRows& p, int64_t row, int64_t c) { return (p.w[row * p.ld + c / 32] >> (c & 31)) & 1u; }

// Sums over the team, the same in every thread of it.  A team of a block uses shared memory, two slots in turn: a slot is
// written again only after a barrier that follows its last reading.
template <int T, int COUNT>
__device__ __forceinline__ void team_sum(float (&v)[COUNT], float (*sh)[COUNT][kNormThreads / 32], int& slot) {
#pragma unroll
  for (int o = (T < 32 ? T : 32) / 2; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < COUNT; ++i) v[i] += __shfl_xor_sync(kFull, v[i], o);
  if constexpr (T > 32) {
    const int warp = threadIdx.x >> 5;
    if ((threadIdx.x & 31) == 0)
#pragma unroll
      for (int i = 0; i < COUNT; ++i) sh[slot][i][warp] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
      v[i] = 0.f;
#pragma unroll
      for (int w = 0; w < kNormThreads / 32; ++w) v[i] += sh[slot][i][w];
    }
    slot ^= 1;
  }
}

// y = ((x - mean) rstd) gamma + beta, then ReLU; a NaN stays one
__device__ __forceinline__ float norm_value(float xh, float gamma, float beta) { return fmaf(xh, gamma, beta); }

// gamma or beta of a thread's columns, kept in registers from row to row (`none` where the pointer is NULL)
template <int T, int NV, bool VEC>
__device__ __forceinline__ void load_cols(const float* __restrict__ w, float none, int f, int t, float (&o)[4 * NV]) {
#pragma unroll
  for (int i = 0; i < 4 * NV; ++i) {
    const int c = col_of<T, VEC>(i / 4, i % 4, t);
    o[i] = w && c < f ? __ldg(w + c) : none;
  }
}

// The mean is corrected by the mean of what is left after subtracting it, and the variance is taken around the corrected
// one: y and rstd of a row 1e4 off zero with a spread of 1 then lose no digits, as the differences x - mean are exact.  (The mean is
// handed to the backward pass in 32 bits, half a unit of it off, and xh is shifted by as much there: 5e-4 in such a row.)
//
// A short row is the chain load - two sums across lanes - store: a warp that holds few float4 of a row works on R at a time
// (200 000 x 100: 66 us with one, 56 with four); two rows share a block's barriers (33 333 x 1 500: 121 and 109; by 4-byte
// accesses two cost registers, 168 and 187 for 48 543 x 1 030).  The rest is registers, for enough warps: 83 194 x 601 takes 147 us with 172 a
// thread, 94 with 128 and a few spilled; 48 543 x 1 030 by 4-byte accesses 433 with 148, 168 with 64.  The grid is what the SMs
// hold at once (twice as many blocks: 83 194 x 601 96, 50 003 x 1 001 72 for 70).
GCNSA_HD constexpr int norm_rows_at_once(int t, int nv, bool vec) {
  return t > 32 ? (vec && nv == 2 ? 2 : 1) : t < 32 ? 2 : nv == 1 ? 4 : nv == 2 ? 2 : 1;
}
constexpr int norm_blocks_per_sm(int t, int nv) { return nv <= 2 ? 4 : t <= 32 && nv <= 4 ? 3 : 2; }
template <int T, int NV, bool VEC>
__global__ void __launch_bounds__(kNormThreads, norm_blocks_per_sm(T, NV))
layer_norm_rows(int64_t n, int f, const float* x, int64_t ldx, const float* __restrict__ gamma, const float* __restrict__ beta,
                float eps, int relu, float* y, int64_t ldy, float* __restrict__ mean_out, float* __restrict__ rstd_out,
                PackedRows x8, PackedRows y8, BitRows bits) {
  wait_for_predecessors();
  constexpr int R = norm_rows_at_once(T, NV, VEC), TEAMS = kNormThreads / T;
  __shared__ float sh1[2][R][kNormThreads / 32], sh2[2][2 * R][kNormThreads / 32];
  const int t = threadIdx.x % T, team = threadIdx.x / T;
  const int n_pad = (int)min(ldy, (int64_t)((f + 3) / 4 * 4));
  const float inv_f = 1.f / (float)f;
  int s1 = 0, s2 = 0;
  float ga[4 * NV], be[4 * NV];
  load_cols<T, NV, VEC>(gamma, 1.f, f, t, ga);
  load_cols<T, NV, VEC>(beta, 0.f, f, t, be);
  // all lanes of a warp stay together (shuffles): rows past the end are computed on zeros and not written
  for (int64_t base = (int64_t)blockIdx.x * TEAMS * R; base < n; base += (int64_t)gridDim.x * TEAMS * R) {
    float a[R][4 * NV], s[R], d[2 * R];
#pragma unroll
    for (int q = 0; q < R; ++q) {
      const int64_t row = base + q * TEAMS + team;
      load_row<T, NV, VEC>(x + row * ldx, row < n ? f : 0, t, a[q]);
    }
#pragma unroll
    for (int q = 0; q < R; ++q) {
      const int64_t row = base + q * TEAMS + team;
      clear_pads<T, NV, VEC>(f, t, a[q]);
      if (x8.q) store_packed<T, NV, VEC>(x8, row, row < n, f, t, a[q]);
      s[q] = 0.f;
#pragma unroll
      for (int i = 0; i < 4 * NV; ++i) s[q] += a[q][i];
    }
    team_sum<T, R>(s, sh1, s1);
#pragma unroll
    for (int q = 0; q < R; ++q) {
      const float m0 = s[q] * inv_f;
      d[2 * q] = d[2 * q + 1] = 0.f;
#pragma unroll
      for (int i = 0; i < 4 * NV; ++i) {
        a[q][i] = col_of<T, VEC>(i / 4, i % 4, t) < f ? a[q][i] - m0 : 0.f;
        d[2 * q] += a[q][i];
        d[2 * q + 1] = fmaf(a[q][i], a[q][i], d[2 * q + 1]);
      }
    }
    team_sum<T, 2 * R>(d, sh2, s2);
#pragma unroll
    for (int q = 0; q < R; ++q) {
      const int64_t row = base + q * TEAMS + team;
      const bool in = row < n;
      const float dm = d[2 * q] * inv_f;
      // (max drops a NaN, which has to reach rstd)
      const float var = fmaf(-dm, dm, d[2 * q + 1] * inv_f), r = 1.f / sqrtf((var < 0.f ? 0.f : var) + eps);
#pragma unroll
      for (int i = 0; i < 4 * NV; ++i) a[q][i] = norm_value((a[q][i] - dm) * r, ga[i], be[i]);
      if (relu)
#pragma unroll
        for (int i = 0; i < 4 * NV; ++i) a[q][i] = a[q][i] < 0.f ? 0.f : a[q][i];
      if (y8.q) store_packed<T, NV, VEC>(y8, row, in, f, t, a[q]);
      if (bits.w) store_bits<T, NV, VEC>(bits, row, in, f, t, a[q]);
      if (in) {
        store_row<T, NV, VEC>(y + row * ldy, f, n_pad, t, a[q]);
        if (t == 0) {
          if (mean_out) mean_out[row] = s[q] * inv_f + dm;
          if (rstd_out) rstd_out[row] = r;
        }
      }
    }
  }
}

// Where v = xh gamma + beta lies within its own rounding error of zero the sign is taken in 64 bits: a gradient is kept or
// dropped by it.  xh is off by 3 half units of 2^-23 and v by one more: by at most 2.4e-7 (|xh gamma| + |v|), and as |xh gamma|
// <= |v| + |beta| its sign is certain where |v| is above 2.5e-7 |beta|.
__device__ __forceinline__ bool near_zero(float v, float beta) { return !(fabsf(v) > 1e-6f * fabsf(beta)); }
__device__ __forceinline__ bool exactly_positive(float x, float mean, float rstd, float gamma, float beta) {
  return ((double)x - mean) * rstd * gamma + beta > 0.0;
}
__device__ __forceinline__ bool norm_positive(float x, float mean, float rstd, float xh, float gamma, float beta) {
  const float v = fmaf(xh, gamma, beta);
  return near_zero(v, beta) ? exactly_positive(x, mean, rstd, gamma, beta) : v > 0.f;
}

// dx = rstd (u - mean(u) - xh mean(u xh)), u = g gamma where the ReLU let the value through; every block leaves the column
// sums of g xh and g over its rows in its row of `partial` (2 f floats), which norm_sums adds in block order.
//
// Registers decide how many rows are on the way: with 127 a thread (the compiler's choice for T = 32, NV = 2) two blocks an SM,
// 269 498 x 256 takes 158 us; at most 80 make it three, 148.  (The next row's loads before this row's sums: 156.)
constexpr int grad_blocks_per_sm(int nv) { return nv <= 1 ? 4 : nv <= 2 ? 3 : nv <= 4 ? 2 : 1; }
template <int T, int NV, bool VEC, bool X8>
__global__ void __launch_bounds__(kNormThreads, grad_blocks_per_sm(NV))
layer_norm_grad(int64_t n, int f, const float* g, int64_t ldg, const float* x, int64_t ldx, PackedRows x8,
                const float* __restrict__ mean, const float* __restrict__ rstd, const float* __restrict__ gamma,
                const float* __restrict__ beta, int relu, BitRows bits, float* dx, int64_t lddx,
                float* __restrict__ partial) {
  wait_for_predecessors();
  __shared__ float sh2[2][2][kNormThreads / 32];
  __shared__ float4 sums[T > 32 ? 1 : kNormThreads];
  constexpr int TEAMS = kNormThreads / T;
  const int t = threadIdx.x % T, team = threadIdx.x / T;
  const int n_pad = (int)min(lddx, (int64_t)((f + 3) / 4 * 4));
  const float inv_f = 1.f / (float)f;
  int s2 = 0;
  float dg[4 * NV], db[4 * NV];
#pragma unroll
  for (int i = 0; i < 4 * NV; ++i) dg[i] = db[i] = 0.f;
  float ga[4 * NV], be[4 * NV];
  load_cols<T, NV, VEC>(gamma, 1.f, f, t, ga);
  load_cols<T, NV, VEC>(beta, 0.f, f, t, be);
  for (int64_t base = (int64_t)blockIdx.x * TEAMS; base < n; base += (int64_t)gridDim.x * TEAMS) {
    const int64_t row = base + team;
    const bool in = row < n;
    float a[4 * NV], u[4 * NV];
    if constexpr (X8) load_packed<T, NV, VEC>(x8, row, in ? f : 0, t, a);
    else load_row<T, NV, VEC>(x + row * ldx, in ? f : 0, t, a);
    load_row<T, NV, VEC>(g + row * ldg, in ? f : 0, t, u);
    const float mu = in ? mean[row] : 0.f, r = in ? rstd[row] : 0.f;
    if constexpr (!X8) clear_pads<T, NV, VEC>(f, t, a);
    clear_pads<T, NV, VEC>(f, t, u);
    if (relu) {
      if (bits.w) {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
          const int c0 = col_of<T, VEC>(v, 0, t);
          const uint32_t word = VEC && in && c0 < f ? bits.w[row * bits.ld + c0 / 32] >> (c0 & 31) : 0u;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int c = col_of<T, VEC>(v, k, t);
            const bool keep = VEC ? (word >> k) & 1u : in && c < f && bit_at(bits, row, c);
            u[4 * v + k] = keep ? u[4 * v + k] : 0.f;
          }
        }
      } else {
        bool close = false;
#pragma unroll
        for (int i = 0; i < 4 * NV; ++i) {
          const float v = fmaf((a[i] - mu) * r, ga[i], be[i]);
          const bool zero = near_zero(v, be[i]);
          close |= zero;
          u[i] = zero || v > 0.f ? u[i] : 0.f;
        }
        if (close)
#pragma unroll
          for (int i = 0; i < 4 * NV; ++i)
            if (near_zero(fmaf((a[i] - mu) * r, ga[i], be[i]), be[i]) && !exactly_positive(a[i], mu, r, ga[i], be[i])) u[i] = 0.f;
      }
    }
    // Columns past the end: u is 0, and what xh is there enters nothing that is written, as long as it is finite.  (It is -mu r in all
    // of them; a select per value instead of this question per row costs 4 to 7 % at 1 030 columns.)
    if (isinf(mu * r))
#pragma unroll
      for (int i = 0; i < 4 * NV; ++i) a[i] = col_of<T, VEC>(i / 4, i % 4, t) < f ? a[i] : mu;
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4 * NV; ++i) {
      a[i] = (a[i] - mu) * r;
      dg[i] = fmaf(u[i], a[i], dg[i]);
      db[i] += u[i];
      u[i] *= ga[i];
      s[0] += u[i];
      s[1] = fmaf(u[i], a[i], s[1]);
    }
    team_sum<T, 2>(s, sh2, s2);
    const float c1 = s[0] * inv_f, c2 = s[1] * inv_f;
#pragma unroll
    for (int i = 0; i < 4 * NV; ++i) a[i] = r * (u[i] - fmaf(a[i], c2, c1));
    if (in) store_row<T, NV, VEC>(dx + row * lddx, f, n_pad, t, a);
  }
  if (!partial) return;
  float* out = partial + (int64_t)blockIdx.x * 2 * f;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const float* w = h ? db + 4 * v : dg + 4 * v;
      if constexpr (T > 32) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int c = col_of<T, VEC>(v, k, t);
          if (c < f) out[h * f + c] = w[k];
        }
      } else {  // the block's teams in a fixed order
        __syncthreads();
        sums[threadIdx.x] = make_float4(w[0], w[1], w[2], w[3]);
        __syncthreads();
        if (team == 0) {
          float4 z = sums[t];
          for (int q = 1; q < TEAMS; ++q) {
            const float4 o = sums[q * T + t];
            z.x += o.x; z.y += o.y; z.z += o.z; z.w += o.w;
          }
          const float zz[4] = {z.x, z.y, z.z, z.w};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int c = col_of<T, VEC>(v, k, t);
            if (c < f) out[h * f + c] = zz[k];
          }
        }
      }
    }
  }
}

// Rows of at most 8 columns, a thread per row, in 64 bits: what the projections leave of a row of two columns is eps rstd^2
// of it, which 32 bits would lose.
constexpr int kNarrowCols = 8;
template <bool X8>
__global__ void __launch_bounds__(kNormThreads)
layer_norm_grad_narrow(int64_t n, int f, const float* g, int64_t ldg, const float* x, int64_t ldx, PackedRows x8,
                       const float* __restrict__ mean, const float* __restrict__ rstd, const float* __restrict__ gamma,
                       const float* __restrict__ beta, int relu, BitRows bits, float* dx, int64_t lddx,
                float* __restrict__ partial) {
  wait_for_predecessors();
  __shared__ double sh[kNormThreads / 32];
  const int n_pad = (int)min(lddx, (int64_t)((f + 3) / 4 * 4));
  double dg[kNarrowCols], db[kNarrowCols];
#pragma unroll
  for (int c = 0; c < kNarrowCols; ++c) dg[c] = db[c] = 0.0;
  for (int64_t row = (int64_t)blockIdx.x * kNormThreads + threadIdx.x; row < n; row += (int64_t)gridDim.x * kNormThreads) {
    const double mu = mean[row], r = rstd[row];
    const float step = X8 ? pack8_step(x8.e[row * x8.lde]) : 0.f;
    double xh[kNarrowCols], u[kNarrowCols], s0 = 0.0, s1 = 0.0;
#pragma unroll
    for (int c = 0; c < kNarrowCols; ++c) {
      xh[c] = u[c] = 0.0;
      if (c < f) {
        const float a = X8 ? (float)x8.q[row * x8.ldq + c] * step : x[row * ldx + c];
        const double ga = gamma ? (double)gamma[c] : 1.0;
        xh[c] = (a - mu) * r;
        double v = g[row * ldg + c];
        if (relu && !(bits.w ? bit_at(bits, row, c) : xh[c] * ga + (beta ? (double)beta[c] : 0.0) > 0.0)) v = 0.0;
        dg[c] += v * xh[c];
        db[c] += v;
        u[c] = v * ga;
        s0 += u[c];
        s1 += u[c] * xh[c];
      }
    }
    s0 /= f;
    s1 /= f;
#pragma unroll
    for (int c = 0; c < kNarrowCols; ++c)
      if (c < n_pad) dx[row * lddx + c] = c < f ? (float)(r * (u[c] - s0 - xh[c] * s1)) : 0.f;
  }
  if (!partial) return;
  float* out = partial + (int64_t)blockIdx.x * 2 * f;
#pragma unroll
  for (int i = 0; i < 2 * kNarrowCols; ++i) {
    const int c = i % kNarrowCols;
    if (c >= f) continue;
    double v = i < kNarrowCols ? dg[c] : db[c];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
    __syncthreads();
    if (threadIdx.x == 0) {
      double z = 0.0;
      for (int w = 0; w < kNormThreads / 32; ++w) z += sh[w];
      out[(i < kNarrowCols ? 0 : f) + c] = (float)z;
    }
  }
}

// Rows wider than the registers of a block hold: a block per row, the row read once per sum (out of the caches).
__global__ void __launch_bounds__(kNormThreads)
layer_norm_wide(int64_t n, int f, const float* x, int64_t ldx, const float* __restrict__ gamma, const float* __restrict__ beta,
                float eps, int relu, float* y, int64_t ldy, float* __restrict__ mean_out, float* __restrict__ rstd_out,
                PackedRows x8, PackedRows y8, BitRows bits) {
  wait_for_predecessors();
  __shared__ float sh1[2][1][kNormThreads / 32], sh2[2][2][kNormThreads / 32];
  const int t = threadIdx.x, n_pad = (int)min(ldy, (int64_t)f + (4 - f % 4) % 4);
  const int f_all = (f + kNormThreads - 1) / kNormThreads * kNormThreads;  // whole warps (shuffles)
  const float inv_f = 1.f / (float)f;
  int s1 = 0, s2 = 0;
  for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
    const float* a = x + row * ldx;
    float s[1] = {0.f}, d[2] = {0.f, 0.f};
    for (int c = t; c < f; c += kNormThreads) s[0] += a[c];
    team_sum<kNormThreads, 1>(s, sh1, s1);
    const float m0 = s[0] * inv_f;
    for (int c = t; c < f; c += kNormThreads) {
      const float v = a[c] - m0;
      d[0] += v;
      d[1] = fmaf(v, v, d[1]);
    }
    team_sum<kNormThreads, 2>(d, sh2, s2);
    const float dm = d[0] * inv_f;
    const float var = fmaf(-dm, dm, d[1] * inv_f), r = 1.f / sqrtf((var < 0.f ? 0.f : var) + eps);
    for (int c = t; c < f_all; c += kNormThreads) {
      const float in = c < f ? a[c] : 0.f;
      const float o = norm_value(((in - m0) - dm) * r, gamma && c < f ? gamma[c] : 1.f, beta && c < f ? beta[c] : 0.f);
      const float out[4] = {c >= f ? 0.f : relu && o < 0.f ? 0.f : o, 0.f, 0.f, 0.f}, src[4] = {in, 0.f, 0.f, 0.f};
      const int chunk = c - t;  // a warp's 32 columns are a block of a checkpoint
      if (x8.q) store_packed<kNormThreads, 1, false>(PackedRows{x8.q + chunk, x8.ldq, x8.e + chunk / kPackBlock, x8.lde}, row, true, min(f - chunk, kNormThreads), t, src);
      if (y8.q) store_packed<kNormThreads, 1, false>(PackedRows{y8.q + chunk, y8.ldq, y8.e + chunk / kPackBlock, y8.lde}, row, true, min(f - chunk, kNormThreads), t, out);
      if (bits.w) store_bits<kNormThreads, 1, false>(BitRows{bits.w + chunk / 32, bits.ld}, row, true, min(f - chunk, kNormThreads), t, out);
      if (c < n_pad) y[row * ldy + c] = out[0];
    }
    if (t == 0) {
      if (mean_out) mean_out[row] = m0 + dm;
      if (rstd_out) rstd_out[row] = r;
    }
  }
}

struct WideRow {  // an element of x or of its checkpoint
  const float* x;
  int64_t ldx;
  PackedRows p;
  __device__ __forceinline__ float at(int64_t row, int64_t c) const {
    return p.q ? (float)p.q[row * p.ldq + c] * pack8_step(p.e[row * p.lde + c / kPackBlock]) : x[row * ldx + c];
  }
};
// A block owns the rows blockIdx.x, blockIdx.x + gridDim.x, ...; its row of `partial` is its own to add to.
__global__ void __launch_bounds__(kNormThreads)
layer_norm_grad_wide(int64_t n, int f, const float* g, int64_t ldg, WideRow x, const float* __restrict__ mean,
                     const float* __restrict__ rstd, const float* __restrict__ gamma, const float* __restrict__ beta, int relu,
                     BitRows bits, float* dx, int64_t lddx, float* __restrict__ partial) {
  wait_for_predecessors();
  __shared__ float sh2[2][2][kNormThreads / 32];
  const int t = threadIdx.x, n_pad = (int)min(lddx, (int64_t)f + (4 - f % 4) % 4);
  const float inv_f = 1.f / (float)f;
  int s2 = 0;
  float* out = partial ? partial + (int64_t)blockIdx.x * 2 * f : nullptr;
  bool first = true;
  for (int64_t row = blockIdx.x; row < n; row += gridDim.x, first = false) {
    const float mu = mean[row], r = rstd[row];
    float s[2] = {0.f, 0.f};
    for (int c = t; c < f; c += kNormThreads) {
      const float a = x.at(row, c), xh = (a - mu) * r, ga = gamma ? gamma[c] : 1.f;
      float v = g[row * ldg + c];
      if (relu && !(bits.w ? bit_at(bits, row, c) : norm_positive(a, mu, r, xh, ga, beta ? beta[c] : 0.f))) v = 0.f;
      if (out) {
        out[c] = first ? v * xh : fmaf(v, xh, out[c]);
        out[(int64_t)f + c] = first ? v : out[(int64_t)f + c] + v;
      }
      s[0] += v * ga;
      s[1] = fmaf(v * ga, xh, s[1]);
    }
    team_sum<kNormThreads, 2>(s, sh2, s2);
    const float c1 = s[0] * inv_f, c2 = s[1] * inv_f;
    for (int c = t; c < n_pad; c += kNormThreads) {
      float o = 0.f;
      if (c < f) {
        const float a = x.at(row, c), xh = (a - mu) * r, ga = gamma ? gamma[c] : 1.f;
        float v = g[row * ldg + c];
        if (relu && !(bits.w ? bit_at(bits, row, c) : norm_positive(a, mu, r, xh, ga, beta ? beta[c] : 0.f))) v = 0.f;
        o = r * (v * ga - fmaf(xh, c2, c1));
      }
      dx[row * lddx + c] = o;  // (this thread was the only one to read dx[c] where dx is g or x)
    }
  }
}

// dgamma[j] (+)= sum over blocks of partial[b][j], dbeta[j] of partial[b][f + j]; a block covers 32 columns, its 16 warps add
// every 16th row, and the 16 sums are added in warp order.
constexpr int kSumWarps = 16;
__global__ void __launch_bounds__(kSumWarps * 32)
norm_sums(int f, int blocks, const float* __restrict__ partial, float* __restrict__ dgamma, float* __restrict__ dbeta, int accumulate) {
  wait_for_predecessors();
  __shared__ float sh[kSumWarps][32];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int64_t j = (int64_t)blockIdx.x * 32 + lane;
  float s = 0.f;
  if (j < 2 * (int64_t)f)
#pragma unroll 8
    for (int b = w; b < blocks; b += kSumWarps) s += partial[(int64_t)b * 2 * f + j];
  sh[w][lane] = s;
  __syncthreads();
  if (w != 0 || j >= 2 * (int64_t)f) return;
  float z = sh[0][lane];
#pragma unroll
  for (int q = 1; q < kSumWarps; ++q) z += sh[q][lane];
  float* dst = j < f ? (dgamma ? dgamma + j : nullptr) : (dbeta ? dbeta + (j - f) : nullptr);
  if (dst) *dst = accumulate ? *dst + z : z;
}

// ---- checkpoints: eight lanes to a block, four blocks of any rows to a warp at a time --------------------------------
// (row, block of the row) of a lane's blocks, one grid stride after the other.  A row is 32 bits, so that its place costs two
// multiplications.
struct BlockWalk {
  uint32_t row, drow;
  int b, db, nb;
  __device__ __forceinline__ BlockWalk(int nb_, uint64_t first, uint64_t stride)
      : row((uint32_t)(first / nb_)), drow((uint32_t)(stride / nb_)), b((int)(first % nb_)), db((int)(stride % nb_)), nb(nb_) {}
  __device__ __forceinline__ void next() {
    row += drow;
    b += db;
    if (b >= nb) {
      b -= nb;
      ++row;
    }
  }
};
// kPackUnroll blocks of a lane are on the way at a time, and the grid is what the SMs hold at once.  552 000 x 256: packing takes
// 126 us with six blocks an SM (40 registers), 135 with a grid of eight of which five fit, 147 with eight (32, spilled);
// unpacking 129 with five blocks of four and four blocks of eight, 150 with eight at a time and three blocks.
constexpr int kPackUnroll = 4, kPackBlocks = 6, kUnpackBlocks = 5;
template <bool VEC>
__global__ void __launch_bounds__(256, kPackBlocks)
pack8_rows(uint32_t n, int f, int nb, const float* __restrict__ x, int64_t ldx, PackedRows p) {
  wait_for_predecessors();
  const int g = threadIdx.x & 7, f16 = (f + 15) / 16 * 16;
  BlockWalk at(nb, ((uint64_t)blockIdx.x * 256 + threadIdx.x) / 8, (uint64_t)gridDim.x * 32);
  // (a warp's four groups run on together until the last of them is past the end)
  while (__any_sync(kFull, at.row < n)) {
    float a[kPackUnroll][4];
    BlockWalk to = at;
#pragma unroll
    for (int i = 0; i < kPackUnroll; ++i) {
      const int c = 32 * at.b + 4 * g;
      const float* src = x + at.row * ldx + c;
      if constexpr (VEC) {
        const float4 v = at.row < n && c < f ? __ldg(reinterpret_cast<const float4*>(src)) : make_float4(0.f, 0.f, 0.f, 0.f);
        a[i][0] = v.x; a[i][1] = v.y; a[i][2] = v.z; a[i][3] = v.w;
        if (c + 3 >= f)
#pragma unroll
          for (int k = 1; k < 4; ++k) a[i][k] = c + k < f ? a[i][k] : 0.f;
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) a[i][k] = at.row < n && c + k < f ? __ldg(src + k) : 0.f;
      }
      at.next();
    }
#pragma unroll
    for (int i = 0; i < kPackUnroll; ++i) {
      uint32_t m = pack8_magnitude(a[i]);
#pragma unroll
      for (int o = 1; o < 8; o <<= 1) m = max(m, __shfl_xor_sync(kFull, m, o));
      const uint32_t ex = pack8_exponent(m);
      const int c = 32 * to.b + 4 * g;
      if (to.row < n) {
        if (c < f16) *reinterpret_cast<uint32_t*>(p.q + to.row * p.ldq + c) = pack8_bytes(a[i], ex);
        if (g == 0) p.e[to.row * p.lde + to.b] = (uint8_t)ex;
      }
      to.next();
    }
  }
}
template <bool VEC>
__global__ void __launch_bounds__(256, kUnpackBlocks)
unpack8_rows(uint32_t n, int f, int nb, PackedRows p, float* __restrict__ x, int64_t ldx) {
  wait_for_predecessors();
  const int g = threadIdx.x & 7, n_pad = (int)min(ldx, (int64_t)f + (4 - f % 4) % 4);
  BlockWalk at(nb, ((uint64_t)blockIdx.x * 256 + threadIdx.x) / 8, (uint64_t)gridDim.x * 32);
  while (at.row < n) {
    uint32_t q[kPackUnroll], ex[kPackUnroll];
    BlockWalk to = at;
#pragma unroll
    for (int i = 0; i < kPackUnroll; ++i) {
      const int c = 32 * at.b + 4 * g;
      const bool in = at.row < n && c < f;
      q[i] = in ? __ldg(reinterpret_cast<const uint32_t*>(p.q + at.row * p.ldq + c)) : 0u;
      ex[i] = in ? __ldg(p.e + at.row * p.lde + at.b) : 0u;
      at.next();
    }
#pragma unroll
    for (int i = 0; i < kPackUnroll; ++i) {
      const int c = 32 * to.b + 4 * g;
      if (to.row < n && c < f) {
        float a[4];
        pack8_open(q[i], a);
        const float step = pack8_step(ex[i]);
#pragma unroll
        for (int k = 0; k < 4; ++k) a[k] *= step;
        if (c + 3 >= f)
#pragma unroll
          for (int k = 1; k < 4; ++k) a[k] = c + k < f ? a[k] : 0.f;
        float* dst = x + to.row * ldx + c;
        if constexpr (VEC) {
          *reinterpret_cast<float4*>(dst) = make_float4(a[0], a[1], a[2], a[3]);
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (c + k < n_pad) dst[k] = a[k];
        }
      }
      to.next();
    }
  }
}

bool vec_rows(const void* p, int64_t ld) { return ((uintptr_t)p & 15) == 0 && ld % 4 == 0; }
PackedRows rows_of(const gcnsa_packed8* p) {
  return p ? PackedRows{p->q, p->ldq, p->e, p->lde} : PackedRows{};
}
// How a row of f columns is held: threads of a team, and float4 of it to each.  Lanes of a warp as far as registers go (up to
// `lane_vecs` float4 each, backward twice as many values are kept): a block's barriers cost a row more than its waiting
// lanes (50 003 x 1 001 forward: 70 us with a warp to a row, 228 with a block).
struct RowTeam {
  int t, nv;
};
constexpr int kNormLaneVecs = 8, kGradLaneVecs = 4;
RowTeam row_team(int32_t f, int lane_vecs) {
  const int vecs = (f + 3) / 4, lane = (vecs + 31) / 32, thread = (vecs + kNormThreads - 1) / kNormThreads;
  if (vecs <= 16) return {vecs <= 8 ? 8 : 16, 1};
  if (lane <= lane_vecs) return {32, lane <= 4 ? lane : lane <= 6 ? 6 : 8};
  return {kNormThreads, thread <= 2 ? thread : thread <= 4 ? 4 : 8};
}
int row_blocks(int64_t n, int64_t rows_per_block, int64_t most) { return (int)std::max<int64_t>(1, std::min((n + rows_per_block - 1) / rows_per_block, most)); }
// blocks of the backward pass; sizes alone decide (the scratch holds a line for each)
int grad_blocks(int64_t n, int32_t f) {
  if (f <= kNarrowCols) return row_blocks(n, kNormThreads, 148 * 4);
  // rows too wide for registers: a block's partial sums are as wide, and all of them take at most 256 MB
  if (f > kNormMaxCols) return row_blocks(n, 1, std::max<int64_t>(1, std::min<int64_t>(148 * 4, (int64_t(256) << 20) / (8 * (int64_t)f))));
  const RowTeam m = row_team(f, kGradLaneVecs);
  return row_blocks(n, kNormThreads / m.t, 148 * grad_blocks_per_sm(m.nv));
}

}  // namespace

int launch_layer_norm(void* stream, int64_t n, int32_t f, const float* x, int64_t ldx, const float* gamma, const float* beta,
                      float eps, int32_t relu, float* y, int64_t ldy, float* mean, float* rstd, const gcnsa_packed8* x8,
                      const gcnsa_packed8* y8, uint32_t* bits, int64_t ldbits) {
  if (n <= 0) return 0;
  cudaStream_t s = (cudaStream_t)stream;
  const bool vec = vec_rows(x, ldx) && vec_rows(y, ldy);
  const PackedRows px = rows_of(x8), py = rows_of(y8);
  auto run = [&](auto kernel, int blocks) {
    launch(kernel, blocks, kNormThreads, 0, s, n, f, x, ldx, gamma, beta, eps, relu, y, ldy, mean, rstd, px, py, BitRows{bits, ldbits});
  };
  if (f > kNormMaxCols) {
    run(layer_norm_wide, row_blocks(n, 1, 148 * 8));
  } else {
    const RowTeam m = row_team(f, kNormLaneVecs);
    const int blocks = row_blocks(n, kNormThreads / m.t * norm_rows_at_once(m.t, m.nv, vec), 148 * norm_blocks_per_sm(m.t, m.nv));
#define GCNSA_NORM(T, NV) (vec ? run(layer_norm_rows<T, NV, true>, blocks) : run(layer_norm_rows<T, NV, false>, blocks))
    if (m.t == 8) GCNSA_NORM(8, 1);
    else if (m.t == 16) GCNSA_NORM(16, 1);
    else if (m.t == 32 && m.nv == 1) GCNSA_NORM(32, 1);
    else if (m.t == 32 && m.nv == 2) GCNSA_NORM(32, 2);
    else if (m.t == 32 && m.nv == 3) GCNSA_NORM(32, 3);
    else if (m.t == 32 && m.nv == 4) GCNSA_NORM(32, 4);
    else if (m.t == 32 && m.nv == 6) GCNSA_NORM(32, 6);
    else if (m.t == 32) GCNSA_NORM(32, 8);
    else if (m.nv == 2) GCNSA_NORM(256, 2);
    else if (m.nv == 4) GCNSA_NORM(256, 4);
    else GCNSA_NORM(256, 8);
#undef GCNSA_NORM
  }
  note_launch();
  return (int)cudaGetLastError();
}

size_t layer_norm_grad_scratch(int64_t n, int32_t f) { return (size_t)grad_blocks(n, f) * 2 * (size_t)f * sizeof(float); }

int launch_layer_norm_grad(void* stream, int64_t n, int32_t f, const float* g, int64_t ldg, const float* x, int64_t ldx,
                           const gcnsa_packed8* x8, const float* mean, const float* rstd, const float* gamma, const float* beta,
                           int32_t relu, const uint32_t* bits, int64_t ldbits, float* dx, int64_t lddx, float* dgamma, float* dbeta,
                           int32_t accumulate, void* scratch) {
  cudaStream_t s = (cudaStream_t)stream;
  const int blocks = n > 0 ? grad_blocks(n, f) : 0;
  float* partial = dgamma || dbeta ? (float*)scratch : nullptr;
  if (n > 0) {
    const bool vec = (x8 || vec_rows(x, ldx)) && vec_rows(g, ldg) && vec_rows(dx, lddx);
    const PackedRows p = rows_of(x8);
    const BitRows through{const_cast<uint32_t*>(bits), ldbits};
    const RowTeam m = row_team(f, kGradLaneVecs);
    auto run = [&](auto kernel) {
      launch(kernel, blocks, kNormThreads, 0, s, n, f, g, ldg, x, ldx, p, mean, rstd, gamma, beta, relu, through, dx, lddx, partial);
    };
#define GCNSA_NORM_GRAD(T, NV)                                                                                        \
  (vec ? (x8 ? run(layer_norm_grad<T, NV, true, true>) : run(layer_norm_grad<T, NV, true, false>))                    \
       : (x8 ? run(layer_norm_grad<T, NV, false, true>) : run(layer_norm_grad<T, NV, false, false>)))
    if (f <= kNarrowCols) x8 ? run(layer_norm_grad_narrow<true>) : run(layer_norm_grad_narrow<false>);
    else if (f > kNormMaxCols)
      launch(layer_norm_grad_wide, blocks, kNormThreads, 0, s, n, f, g, ldg, WideRow{x, ldx, p}, mean, rstd, gamma, beta, relu,
             through, dx, lddx, partial);
    else if (m.t == 8) GCNSA_NORM_GRAD(8, 1);
    else if (m.t == 16) GCNSA_NORM_GRAD(16, 1);
    else if (m.t == 32 && m.nv == 1) GCNSA_NORM_GRAD(32, 1);
    else if (m.t == 32 && m.nv == 2) GCNSA_NORM_GRAD(32, 2);
    else if (m.t == 32 && m.nv == 3) GCNSA_NORM_GRAD(32, 3);
    else if (m.t == 32) GCNSA_NORM_GRAD(32, 4);
    else if (m.nv == 1) GCNSA_NORM_GRAD(256, 1);
    else if (m.nv == 2) GCNSA_NORM_GRAD(256, 2);
    else if (m.nv == 4) GCNSA_NORM_GRAD(256, 4);
    else GCNSA_NORM_GRAD(256, 8);
#undef GCNSA_NORM_GRAD
    note_launch();
  }
  if (partial && !(n <= 0 && accumulate)) {
    launch(norm_sums, (unsigned)((2 * (int64_t)f + 31) / 32), kSumWarps * 32, 0, s, f, blocks, (const float*)partial, dgamma, dbeta, accumulate);
    note_launch();
  }
  return (int)cudaGetLastError();
}

static int pack_blocks(int64_t groups, int per_sm) { return row_blocks(groups, 32 * kPackUnroll, 148 * per_sm); }

int launch_pack8(void* stream, int64_t n, int32_t f, const float* x, int64_t ldx, const gcnsa_packed8* p) {
  if (n <= 0) return 0;
  const int nb = (f + kPackBlock - 1) / kPackBlock, blocks = pack_blocks(n * nb, kPackBlocks);
  auto run = [&](auto kernel) { launch(kernel, blocks, 256, 0, (cudaStream_t)stream, n, f, nb, x, ldx, rows_of(p)); };
  vec_rows(x, ldx) ? run(pack8_rows<true>) : run(pack8_rows<false>);
  note_launch();
  return (int)cudaGetLastError();
}

int launch_unpack8(void* stream, int64_t n, int32_t f, const gcnsa_packed8* p, float* x, int64_t ldx) {
  if (n <= 0) return 0;
  const int nb = (f + kPackBlock - 1) / kPackBlock, blocks = pack_blocks(n * nb, kUnpackBlocks);
  auto run = [&](auto kernel) { launch(kernel, blocks, 256, 0, (cudaStream_t)stream, n, f, nb, rows_of(p), x, ldx); };
  vec_rows(x, ldx) ? run(unpack8_rows<true>) : run(unpack8_rows<false>);
  note_launch();
  return (int)cudaGetLastError();
}

}  // namespace gcnsa
