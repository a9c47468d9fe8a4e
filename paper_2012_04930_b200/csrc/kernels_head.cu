// The weight gradient of a layer whose input is an 8-bit checkpoint, and the softmax cross-entropy of an output layer
// over many classes without its logits.
#include <cuda_runtime.h>

#include <algorithm>

#include "internal.h"
#include "launch.h"
#include "pack8_device.h"

namespace gcnsa {

namespace {

constexpr unsigned kFull = 0xffffffffu;
size_t up256(size_t b) { return (b + 255) / 256 * 256; }

// ---- dw = X^T G, X packed: 32 x 32 tiles of dw, a slice of the rows per block ---------------------------------------
constexpr int kTile = 32;
__global__ void __launch_bounds__(256)
packed8_product(int64_t n, int f, int c, gcnsa_packed8 x, const float* __restrict__ g, int64_t ldg, int64_t rows_per_slice,
                float* __restrict__ partial, int64_t ldp) {
  wait_for_predecessors();
  __shared__ float xs[kTile][kTile + 1], gs[kTile][kTile + 1];
  const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
  const int f0 = blockIdx.x * kTile, c0 = blockIdx.y * kTile;
  const int64_t r0 = (int64_t)blockIdx.z * rows_per_slice, r1 = min(n, r0 + rows_per_slice);
  float acc[4] = {0.f, 0.f, 0.f, 0.f};
  for (int64_t r = r0; r < r1; r += kTile) {
    for (int k = ty; k < kTile; k += 8) {
      const int64_t row = r + k;
      xs[k][tx] = row < r1 && f0 + tx < f ? (float)x.q[row * x.ldq + f0 + tx] * pack8_step(x.e[row * x.lde + f0 / kPackBlock]) : 0.f;
      gs[k][tx] = row < r1 && c0 + tx < c ? g[row * ldg + c0 + tx] : 0.f;
    }
    __syncthreads();
#pragma unroll 8
    for (int k = 0; k < kTile; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i] = fmaf(xs[k][ty + 8 * i], gs[k][tx], acc[i]);
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (f0 + ty + 8 * i < f && c0 + tx < c) partial[((int64_t)blockIdx.z * f + f0 + ty + 8 * i) * ldp + c0 + tx] = acc[i];
}
int packed8_slices(int64_t n, int32_t f, int32_t c) {
  const int64_t tiles = (((int64_t)f + kTile - 1) / kTile) * (((int64_t)c + kTile - 1) / kTile);
  return (int)std::max<int64_t>(1, std::min<int64_t>({(n + 255) / 256, 148 * 8 / tiles, 1024}));
}

// ---- softmax cross-entropy over pieces of the classes: z of a piece is in memory, rows carry their running maximum and
// sum of exponentials (m, s) and their label's logit ------------------------------------------------------------------
struct RowState {
  float *m, *s, *zy;
};
__global__ void __launch_bounds__(256)
ce_piece_stats(int64_t n, int c0, int width, const float* __restrict__ z, int64_t ldz, const int32_t* __restrict__ y, RowState st) {
  wait_for_predecessors();
  const int lane = threadIdx.x & 31;
  for (int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); row < n; row += (int64_t)gridDim.x * 8) {
    const float* r = z + row * ldz;
    float m = -INFINITY;
    for (int j = lane; j < width; j += 32) m = fmaxf(m, r[j]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(kFull, m, o));
    float s = 0.f;
    for (int j = lane; j < width; j += 32) s += expf(r[j] - m);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(kFull, s, o);
    if (lane == 0) {
      if (c0 > 0) {
        const float m0 = st.m[row], m1 = fmaxf(m0, m);
        s = st.s[row] * expf(m0 - m1) + s * expf(m - m1);
        m = m1;
      } else {
        st.zy[row] = NAN;  // no label met yet
      }
      st.m[row] = m;
      st.s[row] = s;
      const int64_t at = (int64_t)y[row] - c0;
      if (at >= 0 && at < width) st.zy[row] = r[at];
    }
  }
}
__global__ void __launch_bounds__(256)
ce_piece_grad(int64_t n, int c0, int width, int pad, float* __restrict__ z, int64_t ldz, const int32_t* __restrict__ y,
              const uint8_t* __restrict__ mask, float inv_nt, RowState st) {
  wait_for_predecessors();
  const int lane = threadIdx.x & 31;
  for (int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); row < n; row += (int64_t)gridDim.x * 8) {
    float* r = z + row * ldz;
    const bool on = !mask || mask[row] != 0;
    const float m = st.m[row], inv = 1.f / st.s[row];
    const int yi = y[row];
    for (int j = lane; j < pad; j += 32)
      r[j] = on && j < width ? (expf(r[j] - m) * inv - (c0 + j == yi ? 1.f : 0.f)) * inv_nt : 0.f;
  }
}
// sum of the masked rows' losses and their number, in a fixed order
__global__ void __launch_bounds__(1024)
ce_loss(int64_t n, const uint8_t* __restrict__ mask, RowState st, int64_t n_train, float* __restrict__ loss) {
  wait_for_predecessors();
  __shared__ double sh[32];
  __shared__ long long shc[32];
  double s = 0.0;
  long long count = 0;
  for (int64_t row = threadIdx.x; row < n; row += 1024)
    if (!mask || mask[row]) {
      s += (double)(st.m[row] + logf(st.s[row])) - st.zy[row];
      ++count;
    }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    s += __shfl_xor_sync(kFull, s, o);
    count += __shfl_xor_sync(kFull, count, o);
  }
  if ((threadIdx.x & 31) == 0) {
    sh[threadIdx.x >> 5] = s;
    shc[threadIdx.x >> 5] = count;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 32; ++w) {
      s += sh[w];
      count += shc[w];
    }
    *loss = count != n_train ? NAN : n_train > 0 ? (float)(s / (double)n_train) : 0.f;
  }
}

int64_t piece_of(int64_t n, int32_t c) {
  const int64_t fit = (int64_t(64) << 20) / 4 / std::max<int64_t>(n, 1) / 128 * 128;
  return std::min<int64_t>((c + 3) / 4 * 4, std::max<int64_t>(fit, 128));
}

}  // namespace

size_t gemm_packed8_workspace(int64_t n, int32_t f, int32_t c) {
  return up256((size_t)packed8_slices(n, f, c) * f * (((size_t)c + 3) / 4 * 4) * sizeof(float));
}

int launch_gemm_packed8(void* stream, int64_t n, int32_t f, int32_t c, const gcnsa_packed8* x, const float* g, int64_t ldg,
                        float* dw, int64_t lddw, int32_t accumulate, void* workspace) {
  const int64_t ldp = ((int64_t)c + 3) / 4 * 4;
  const int slices = n > 0 ? packed8_slices(n, f, c) : 0;
  if (n > 0) {
    const dim3 grid((f + kTile - 1) / kTile, (c + kTile - 1) / kTile, slices);
    launch(packed8_product, grid, 256, 0, (cudaStream_t)stream, n, f, c, *x, g, ldg, (n + slices - 1) / slices, (float*)workspace, ldp);
    note_launch();
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return (int)e;
  }
  return launch_splitk_reduce(stream, f, c, slices, (const float*)workspace, ldp, dw, lddw, accumulate, GCNSA_EPI_NONE, nullptr, 0);
}

size_t linear_ce_workspace(int64_t n, int32_t d, int32_t c) {
  const int64_t piece = piece_of(n, c);
  return up256((size_t)n * piece * 4) + 3 * up256((size_t)n * 4) + up256(colsum_scratch(n, (int32_t)piece)) +
         up256(std::max({gemm_workspace(GCNSA_GEMM_FP32, 0, 0, n, piece, d), gemm_workspace(GCNSA_GEMM_FP32, 0, 1, n, d, piece),
                         gemm_workspace(GCNSA_GEMM_FP32, 1, 0, d, piece, n)}));
}

int launch_linear_ce(void* stream, const LinearCe& a, void* workspace) {
  cudaStream_t s = (cudaStream_t)stream;
  const int64_t n = a.n, piece = piece_of(n, a.c);
  uint8_t* ws = (uint8_t*)workspace;
  auto take = [&](size_t bytes) { uint8_t* p = ws; ws += up256(bytes); return p; };
  float* z = (float*)take((size_t)n * piece * 4);
  RowState st;
  st.m = (float*)take((size_t)n * 4);
  st.s = (float*)take((size_t)n * 4);
  st.zy = (float*)take((size_t)n * 4);
  void* sums = take(colsum_scratch(n, (int32_t)piece));
  void* gw = ws;
  const size_t gwb = (size_t)((uint8_t*)workspace + linear_ce_workspace(n, a.d, a.c) - ws);
  const float inv_nt = a.n_train > 0 ? 1.f / (float)a.n_train : 0.f;
  const int blocks = (int)std::max<int64_t>(1, std::min<int64_t>((n + 7) / 8, 148 * 8));
#define GCNSA_STEP(call)              \
  do {                                \
    const int rc_ = (call);           \
    if (rc_ != 0) return rc_;         \
  } while (0)
  auto logits = [&](int64_t c0, int64_t width) {
    return launch_gemm(stream, GCNSA_GEMM_FP32, 0, 0, n, width, a.d, a.h, a.ldh, a.w + c0, a.ldw, z, piece, 0, a.bias ? GCNSA_EPI_BIAS : GCNSA_EPI_NONE,
                       a.bias ? a.bias + c0 : nullptr, 0, gw, gwb);
  };
  if (n > 0)
    for (int64_t c0 = 0; c0 < a.c; c0 += piece) {
      const int64_t width = std::min<int64_t>(piece, a.c - c0);
      GCNSA_STEP(logits(c0, width));
      launch(ce_piece_stats, blocks, 256, 0, s, n, (int)c0, (int)width, (const float*)z, piece, a.y, st);
      note_launch();
    }
  launch(ce_loss, 1, 1024, 0, s, n, a.mask, st, a.n_train, a.loss);
  note_launch();
  GCNSA_STEP((int)cudaGetLastError());
  if (!a.dh && !a.dw && !a.db) return 0;
  for (int64_t c0 = 0; c0 < a.c; c0 += piece) {
    const int64_t width = std::min<int64_t>(piece, a.c - c0);
    if (n > 0) {
      if (piece < a.c) GCNSA_STEP(logits(c0, width));
      launch(ce_piece_grad, blocks, 256, 0, s, n, (int)c0, (int)width, (int)((width + 3) / 4 * 4), z, piece, a.y, a.mask, inv_nt, st);
      note_launch();
      if (a.dh) GCNSA_STEP(launch_gemm(stream, GCNSA_GEMM_FP32, 0, 1, n, a.d, width, z, piece, a.w + c0, a.ldw, a.dh, a.lddh, c0 > 0, GCNSA_EPI_NONE, nullptr, 0, gw, gwb));
    }
    if (a.dw) GCNSA_STEP(launch_gemm(stream, GCNSA_GEMM_FP32, 1, 0, a.d, width, n, a.h, a.ldh, z, piece, a.dw + c0, a.lddw, a.accumulate, GCNSA_EPI_NONE, nullptr, 0, gw, gwb));
    if (a.db) GCNSA_STEP(launch_colsum(stream, n, (int32_t)width, z, piece, a.db + c0, a.accumulate, sums));
  }
#undef GCNSA_STEP
  return 0;
}

}  // namespace gcnsa
