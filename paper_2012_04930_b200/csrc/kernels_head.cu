// The weight gradient of a layer whose input is an 8-bit checkpoint, and the softmax cross-entropy of an output layer
// over many classes without its logits.  Both are products of kernels_terms.h.
//
// Output layer: z = H W + b, G = (softmax(z) - onehot) / n_train, dH = G W^T, dW = H^T G, db = 1^T G.  z is made tile by
// tile and never leaves the SM; G is written transposed (thread = row, so a class is a line of memory), which is how both
// gradient products want it: dH^T = W G^T and dW^T = G^T H have a K-major left and an MN-major right operand, and their
// results, written transposed, are dH and dW.  db falls out of the second one, whose left operand passes through registers.
//  - c <= 128: a tile holds whole rows of z, so softmax, loss and G come from one pass over the products.
//  - c > 128: one pass keeps a running maximum and sum of exponentials per row (8 bytes per row and run of tiles), then, a
//    piece of the classes at a time, z is made again and turned into G.  Rows that
//    do not count are left out of all products: the others are gathered first.
// Rows that do not count may hold anything: up to 128 classes they are rows of zeros in G, and in H^T G rows of zeros of H too.
// The two gradient products of a piece are independent and run as one launch, the slices of dW^T before the tiles of dH^T.
#include <cuda_runtime.h>

#include <algorithm>

#include "debug_check.h"
#include "internal.h"
#include "kernels_terms.h"
#include "launch.h"

namespace gcnsa {

namespace {

constexpr unsigned kFull = 0xffffffffu;
size_t up256(size_t b) { return (b + 255) / 256 * 256; }
int64_t up4(int64_t n) { return (n + 3) / 4 * 4; }
int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Slices of the inner dimension: as many as make the rounds of tiles x slices items over the SMs shortest, a slice costing
// about six k-blocks on top of its own (its share of the sums written and read again, an accumulator's start and end).
template <class Cost>
int cheapest_slices(int64_t tiles, int64_t units, Cost cost) {
  const int most = (int)std::min<int64_t>(units, std::max<int64_t>(1, 2 * sm_count() / tiles));
  int best = 1;
  int64_t best_cost = INT64_MAX;
  for (int s = 1; s <= most; s += std::max(1, s / 16)) {  // (one in 16 apart: the search runs in every call)
    const int64_t len = div_up(units, s), c = cost(div_up(units, len), len);
    if (c < best_cost) {
      best = s;
      best_cost = c;
    }
  }
  return (int)div_up(units, div_up(units, best));
}
int pick_slices(int64_t tiles, int64_t units) {
  return cheapest_slices(tiles, units, [&](int64_t s, int64_t len) { return div_up(tiles * s, sm_count()) * (len + 6); });
}
// The same for a product whose items are followed in a launch by `others` items of other_units k-blocks.  Block b takes items b,
// b + grid, ...: what the fullest block gets, which is the first one or the first with an item less of either kind.
int balanced_slices(int64_t tiles, int64_t units, int64_t others, int64_t other_units) {
  return cheapest_slices(tiles, units, [&](int64_t s, int64_t len) {
    const int64_t items = tiles * s, total = items + others, grid = std::min<int64_t>(total, sm_count());
    int64_t most = 0;
    for (const int64_t b : {int64_t(0), items % grid, total % grid}) {
      const int64_t mine = items > b ? div_up(items - b, grid) : 0, all = div_up(total - b, grid);
      most = std::max(most, mine * (len + 6) + (all - mine) * (other_units + 6));
    }
    return most;
  });
}
void set_slices(Product& p, int bn, int slices) {
  p.tiles_m = (int)div_up(p.M, BM);
  p.tiles_n = (int)div_up(p.N, bn);
  p.per_slice = (int)div_up(p.units, slices);
  p.items = p.tiles_m * p.tiles_n * slices;
}

// ---- dw = X^T G: dw^T = G^T X, tiles of 128 columns of G x 64 or 128 features --------------------------------------
struct PackedPlan {
  int bn, slices;
  int64_t ldp;
};
PackedPlan packed_plan(int64_t n, int32_t f, int32_t c) {
  PackedPlan p;
  p.bn = f <= 64 ? 64 : 128;
  p.slices = pick_slices(div_up(c, BM) * div_up(f, p.bn), div_up(n, BK));
  p.ldp = up4(c);
  return p;
}
template <int BN, ASrc A>
cudaError_t run_packed(cudaStream_t s, const TermArgs& a, int grid) {
  return run_terms<TermShape<BN, A, true, Out::transposed>>(s, a, grid);
}

// ---- rows that count ---------------------------------------------------------------------------------------------------
constexpr int kRowsPerBlock = 1024;
__global__ void __launch_bounds__(kRowsPerBlock) mask_counts(int64_t n, const uint8_t* __restrict__ mask, int* __restrict__ counts) {
  wait_for_predecessors();
  const int64_t i = (int64_t)blockIdx.x * kRowsPerBlock + threadIdx.x;
  const int c = __syncthreads_count(i < n && mask[i] != 0);
  if (threadIdx.x == 0) counts[blockIdx.x] = c;
}
// place[i] = how many counted rows lie before row i, -1 where i does not count or is beyond the `room` places; rows[place] = i
// (-1 behind the last one), *total = all that count.
__global__ void __launch_bounds__(kRowsPerBlock)
mask_places(int64_t n, const uint8_t* __restrict__ mask, const int* __restrict__ counts, int64_t room, int32_t* __restrict__ place,
            int32_t* __restrict__ rows, int* __restrict__ total) {
  wait_for_predecessors();
  __shared__ int sh[32];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  int before = 0;  // rows that count in the blocks before
  for (int b = threadIdx.x; b < (int)blockIdx.x; b += kRowsPerBlock) before += counts[b];
  before = __reduce_add_sync(kFull, before);
  if (lane == 0) sh[w] = before;
  __syncthreads();
  before = __reduce_add_sync(kFull, sh[lane]);
  __syncthreads();
  const int64_t i = (int64_t)blockIdx.x * kRowsPerBlock + threadIdx.x;
  const bool on = i < n && mask[i] != 0;
  const unsigned set = __ballot_sync(kFull, on);
  if (lane == 0) sh[w] = __popc(set);
  __syncthreads();
  const int mine = sh[lane];
  int warps = __reduce_add_sync(kFull, lane < w ? mine : 0), all = __reduce_add_sync(kFull, mine);
  const int64_t at = (int64_t)before + warps + __popc(set & ((1u << lane) - 1));
  if (i < n) place[i] = on && at < room ? (int32_t)at : -1;
  if (on && at < room) rows[at] = (int32_t)i;
  if (blockIdx.x == gridDim.x - 1) {
    const int64_t count = (int64_t)before + all;
    if (threadIdx.x == 0) *total = (int)count;
    for (int64_t k = count + threadIdx.x; k < room; k += kRowsPerBlock) rows[k] = -1;
  }
}
// A warp per row: counted rows of h and their labels to their places, rows of dh that do not count to zero.  Places behind
// the last counted row (n_train larger than the mask says) become rows of zeros without a label.
__global__ void __launch_bounds__(256)
gather_rows(int64_t n, int d, const float* __restrict__ h, int64_t ldh, const int32_t* __restrict__ y, const int32_t* __restrict__ place,
            const int* __restrict__ total, int64_t room, float* __restrict__ hc, int64_t ldc, int32_t* __restrict__ yc, float* __restrict__ dh, int64_t lddh) {
  wait_for_predecessors();
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const bool vec = ((uintptr_t)h & 15) == 0 && ldh % 4 == 0;
  const int pad = (int)min(lddh, (int64_t)(d + 3) / 4 * 4);
  for (int64_t i = (int64_t)blockIdx.x * 8 + w; i < n; i += (int64_t)gridDim.x * 8) {
    const int at = place[i];
    if (at >= 0) {
#if GCNSA_DBG
      if (!dbg_in(&g_dbg_head, at, 0, room, kDbgGatherPlace)) continue;
#endif
      const float* src = h + i * ldh;
      float* dst = hc + at * ldc;
      const int d4 = vec ? d / 4 : 0;
      for (int j = lane; j < d4; j += 32) reinterpret_cast<float4*>(dst)[j] = __ldg(reinterpret_cast<const float4*>(src) + j);
      for (int j = 4 * d4 + lane; j < d; j += 32) dst[j] = __ldg(src + j);
      if (lane == 0) yc[at] = y[i];
    } else if (dh) {
      for (int j = lane; j < pad; j += 32) dh[i * lddh + j] = 0.f;
    }
  }
  for (int64_t k = (int64_t)*total + (int64_t)blockIdx.x * 8 + w; k < room; k += (int64_t)gridDim.x * 8) {
    for (int j = lane; j < d; j += 32) hc[k * ldc + j] = 0.f;
    if (lane == 0) yc[k] = -1;
  }
}

// The loss from the sums of warps or blocks, in a fixed order: 256 threads.
__device__ __forceinline__ void finish_loss(int n, const LossSum* __restrict__ sums, const int* __restrict__ total, int64_t n_train, float* __restrict__ loss) {
  __shared__ double shl[8];
  __shared__ long long shc[8];
  LossSum a = {0.0, 0};
#pragma unroll 4
  for (int i = threadIdx.x; i < n; i += 256) {
    a.loss += sums[i].loss;
    a.count += sums[i].count;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    a.loss += __shfl_xor_sync(kFull, a.loss, o);
    a.count += __shfl_xor_sync(kFull, a.count, o);
  }
  if ((threadIdx.x & 31) == 0) {
    shl[threadIdx.x >> 5] = a.loss;
    shc[threadIdx.x >> 5] = a.count;
  }
  __syncthreads();
  if (threadIdx.x != 0) return;
  for (int w = 1; w < 8; ++w) {
    a.loss += shl[w];
    a.count += shc[w];
  }
  const long long count = total ? *total : a.count;
  *loss = count != n_train ? NAN : n_train > 0 ? (float)(a.loss / (double)n_train) : 0.f;
}
__global__ void __launch_bounds__(256) loss_total(int n, const LossSum* __restrict__ sums, const int* __restrict__ total, int64_t n_train, float* __restrict__ loss) {
  wait_for_predecessors();
  finish_loss(n, sums, total, n_train, loss);
}
// Maximum and 1 / sum of exponentials of every row from the runs that crossed its tile, and a block's sum of losses.  The two are
// kept apart: as one number, the maximum plus the sum's logarithm, they would be off by half a unit of the maximum, which a
// probability near 1 has above its distance from 1 (logits near 1 000: 3e-5 of p - 1).
__global__ void __launch_bounds__(256)
row_finish(int64_t rows, int c, int tiles_n, int total, int grid, const float* __restrict__ part_m, const float* __restrict__ part_s,
           const int32_t* __restrict__ y, const float* __restrict__ zy, float2* __restrict__ top, LossSum* __restrict__ losses) {
  wait_for_predecessors();
  __shared__ double sh[8];
  const int64_t r = (int64_t)blockIdx.x * 256 + threadIdx.x;
  double loss = 0.0;
  if (r < rows) {
    const int t = (int)(r / BM);
    const int b0 = term_owner(t * tiles_n, total, grid), b1 = term_owner((t + 1) * tiles_n - 1, total, grid);
    float m = -INFINITY, s = 0.f;
    for (int b = b0; b <= b1; ++b)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int64_t slot = ((int64_t)(b + t) * 2 + h) * BM + r % BM;
        const float pm = part_m[slot], larger = fmaxf(m, pm), base = larger == -INFINITY ? 0.f : larger;
        s = s * expf(m - base) + part_s[slot] * expf(pm - base);
        m = larger;
      }
    const int label = y[r];
    top[r] = make_float2(m, 1.f / s);
    loss = label >= 0 && label < c ? ((double)m - zy[r]) + logf(s) : NAN;  // (no class was a label outside)
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) loss += __shfl_xor_sync(kFull, loss, o);
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = loss;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 8; ++w) loss += sh[w];
    losses[blockIdx.x] = LossSum{loss, (long long)min((int64_t)256, rows - (int64_t)blockIdx.x * 256)};
  }
}
// what finish_loss is given
struct LossEnd {
  int n = 0;
  const LossSum* sums = nullptr;
  const int* total = nullptr;
  int64_t n_train = 0;
  float* loss = nullptr;  // NULL: not to be written
};
// The slices of a product added up, and with them the sums that its left operand left: row r of c (+)= sum over the slices of
// partial[z][r][.] for r < rows, and sums_out (+)= sum over `lines` lines of sums; with them the loss, where it is still to be
// made.  A block has 128 columns of a row; its 8 warps
// take every 8th slice each, a float4 to a lane, and are added in warp order.
__global__ void __launch_bounds__(256)
add_slices(int rows, int n, int slices, const float* __restrict__ partial, int64_t ldp, float* __restrict__ c, int64_t ldc, int n_pad, int lines,
           const float* __restrict__ sums, float* __restrict__ sums_out, int accumulate, LossEnd end) {
  wait_for_predecessors();
  if (end.loss && blockIdx.y == gridDim.y - 1) {  // a line of blocks of its own
    if (blockIdx.x == 0) finish_loss(end.n, end.sums, end.total, end.n_train, end.loss);
    return;
  }
  const int lines_y = gridDim.y - (end.loss != nullptr);
  __shared__ float4 sh[8][32];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, j = 128 * blockIdx.x + 4 * lane;
  for (int r = blockIdx.y; r < rows + (sums_out != nullptr); r += lines_y) {
    const bool tail = r == rows;
    const float* src = tail ? sums + j : partial + r * ldp + j;
    const int64_t step = tail ? ldp : rows * ldp;
    const int count = tail ? lines : slices;
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
    if (j < n) {
#pragma unroll 8
      for (int z = w; z < count; z += 8) {
        const float4 v = __ldg(reinterpret_cast<const float4*>(src + z * step));
        a.x += v.x; a.y += v.y; a.z += v.z; a.w += v.w;
      }
    }
    sh[w][lane] = a;
    __syncthreads();
    if (threadIdx.x < 128) {
      const int k = threadIdx.x, col = 128 * blockIdx.x + k;
      float s = 0.f;
#pragma unroll
      for (int q = 0; q < 8; ++q) s += reinterpret_cast<const float*>(sh[q])[k];
      float* const dst = tail ? sums_out + col : c + r * ldc + col;
      if (col < n) *dst = accumulate ? *dst + s : s;
      else if (!tail && col < n_pad && !accumulate) *dst = 0.f;
    }
    __syncthreads();
  }
}
// (pitch of both partial and sums: ldp)
int launch_add_slices(cudaStream_t s, int64_t rows, int64_t n, int slices, const float* partial, int64_t ldp, float* c, int64_t ldc, int64_t n_pad,
                      int lines, const float* sums, float* sums_out, int accumulate, const LossEnd& end = LossEnd{}) {
  const dim3 grid((unsigned)((n_pad + 127) / 128), (unsigned)std::min<int64_t>(rows + (sums_out != nullptr), 65000) + (end.loss != nullptr));
  const cudaError_t e = launch(add_slices, grid, 256, 0, s, rows, n, slices, partial, ldp, c, ldc, n_pad, lines, sums, sums_out, accumulate, end);
  note_launch();
  return (int)e;
}

// ---- plan of a call: sizes that hold for every count of rows up to n -------------------------------------------------
constexpr int kSumLines = TermShape<128, ASrc::kMajor, false, Out::transposed>::AG;  // of a_sums, per slice
constexpr int kWholeCols = 128;                    // classes that one tile holds
// Floats of G^T at most (a piece has 128 classes at least): 160 MB.  Three launches a piece cost about 30 us on top of their work, more than
// it costs that G^T is then read from HBM in part: 20 011 x 256 x 10 007 with 64 / 96 / 192 MB 1 922 / 1 793 / 1 722 us.
constexpr int64_t kPieceFloats = int64_t(40) << 20;
struct CePlan {
  int64_t gt_floats, partial_floats, sums_floats, slots;
  size_t gt, partial, sums, hc, wc, yc, rows, place, counts, total, zy, top, part, losses, end;
};
CePlan ce_plan(int64_t n, int32_t d, int32_t c) {
  CePlan p;
  const int64_t n4 = up4(n), c128 = div_up(c, 128) * 128, sms = sm_count();
  const bool whole = c <= kWholeCols;
  p.gt_floats = whole ? c * n4 : std::min(c128 * n4, std::max(kPieceFloats, 128 * n4));
  // at most 2 x SMs items of slices of dW^T (pick_slices)
  p.partial_floats = n > 0 ? std::min(2 * sms, std::max<int64_t>(div_up(n, BK), 1) * div_up(d, 128) * (c128 / 128)) * 128 * 128 : 0;
  p.sums_floats = n > 0 ? kSumLines * std::max<int64_t>(2 * sms * 128, c128) : 0;  // a line per slice and group
  p.slots = sms + div_up(n, BM);
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t o = at; at += up256(bytes); return o; };
  p.gt = take((size_t)p.gt_floats * 4);
  p.partial = take((size_t)p.partial_floats * 4);
  p.sums = take((size_t)p.sums_floats * 4);
  p.hc = take((size_t)n * up4(d) * 4);
  p.wc = take((size_t)d * up4(c) * 4);
  p.yc = take((size_t)n * 4);
  p.rows = take((size_t)n * 4);
  p.place = take((size_t)n * 4);
  p.counts = take((size_t)div_up(n, kRowsPerBlock) * 4);
  p.total = take(4);
  p.zy = take((size_t)n * 4);
  p.top = take((size_t)n * sizeof(float2));
  p.part = take((size_t)p.slots * 2 * BM * 2 * 4);
  p.losses = take((size_t)std::max<int64_t>(sms * kFoldWarps, div_up(n, 256)) * sizeof(LossSum));
  p.end = at;
  return p;
}
// Classes of a piece: the multiple of 128 whose G^T fits its room and with which the rounds of z's tiles over the SMs and the
// launches (about 30 k-blocks' time a piece) cost least.
int64_t piece_classes(const CePlan& p, int64_t rows, int32_t d, int32_t c) {
  const int64_t all = div_up(c, 128), most = std::max<int64_t>(1, std::min(all, p.gt_floats / (128 * up4(rows)))), tiles_m = div_up(rows, BM), sms = sm_count();
  int64_t best = most, best_cost = INT64_MAX;
  for (int64_t k = most; k >= std::max<int64_t>(1, most / 2); --k) {
    const int64_t pieces = div_up(all, k), last = all - (pieces - 1) * k;
    const int64_t cost = ((pieces - 1) * div_up(tiles_m * k, sms) + div_up(tiles_m * last, sms)) * (div_up(d, BK) + 2) + pieces * 30;
    if (cost < best_cost) {
      best = k;
      best_cost = cost;
    }
  }
  return best * 128;
}

#define GCNSA_STEP(...)                           \
  do {                                            \
    const int rc_ = (int)(__VA_ARGS__);           \
    if (rc_ != 0) return rc_;                     \
  } while (0)

}  // namespace

size_t gemm_packed8_workspace(int64_t n, int32_t f, int32_t c) {
  const PackedPlan p = packed_plan(n, f, c);
  return p.slices > 1 ? up256((size_t)p.slices * f * p.ldp * sizeof(float)) : 0;
}

int launch_gemm_packed8(void* stream, int64_t n, int32_t f, int32_t c, const gcnsa_packed8* x, const float* g, int64_t ldg,
                        float* dw, int64_t lddw, int32_t accumulate, void* workspace) {
  if (n <= 0) return launch_add_slices((cudaStream_t)stream, f, c, 0, nullptr, up4(c), dw, lddw, std::min<int64_t>(lddw, up4(c)), 0, nullptr, nullptr, accumulate);
  const PackedPlan pl = packed_plan(n, f, c);
  const bool tma = ((uintptr_t)g & 15) == 0 && ldg % 4 == 0;
  TermArgs a = {};
  Product& p = a.p[0];
  if (!term_map(&p.map_b, x->q, true, n, f, x->ldq, pl.bn, BK, false) || (tma && !term_map(&p.map_a, g, false, n, c, ldg, 32, BK, false)))
    return (int)cudaErrorNotSupported;
  p.M = c;
  p.N = f;
  p.units = (int)div_up(n, BK);
  set_slices(p, pl.bn, pl.slices);
  const bool split = pl.slices > 1;
  p.c = split ? (float*)workspace : dw;
  p.ldc = split ? pl.ldp : lddw;
  p.slice_stride = split ? f * pl.ldp : 0;
  p.accumulate = split ? 0 : accumulate;
  p.m_pad = (int)std::min<int64_t>(p.ldc, up4(c));
  p.write = 1;
  p.a = g;
  p.lda = ldg;
  p.k_rows = n;
  p.e = x->e;
  p.lde = x->lde;
  p.e_blocks = (int)div_up(f, kPackBlock);
  a.total = p.items;
  const int grid = std::min(a.total, sm_count());
  cudaStream_t s = (cudaStream_t)stream;
  GCNSA_STEP(pl.bn == 64 ? (tma ? run_packed<64, ASrc::mnMajor>(s, a, grid) : run_packed<64, ASrc::direct>(s, a, grid))
                         : (tma ? run_packed<128, ASrc::mnMajor>(s, a, grid) : run_packed<128, ASrc::direct>(s, a, grid)));
  note_launch();
  if (split) return launch_add_slices(s, f, c, pl.slices, (const float*)workspace, pl.ldp, dw, lddw, std::min<int64_t>(lddw, up4(c)), 0, nullptr, nullptr, accumulate);
  return 0;
}

size_t linear_ce_workspace(int64_t n, int32_t d, int32_t c) { return ce_plan(n, d, c).end; }

int launch_linear_ce(void* stream, const LinearCe& a, void* workspace) {
  cudaStream_t s = (cudaStream_t)stream;
  const CePlan pl = ce_plan(a.n, a.d, a.c);
  uint8_t* const ws = (uint8_t*)workspace;
  auto f_at = [&](size_t o) { return (float*)(ws + o); };
  const int sms = sm_count();
  const bool whole = a.c <= kWholeCols, grads = a.dh || a.dw || a.db;
  const float inv_nt = a.n_train > 0 ? 1.f / (float)a.n_train : 0.f;
  const int *total = nullptr;
  const int32_t *rows = nullptr, *y = a.y;
  const float *h = a.h, *w = a.w;
  int64_t ldh = a.ldh, ldw = a.ldw, R = a.n;  // rows of the products

  const bool gather = !whole && a.mask && a.n > 0;
  if (gather) {
    const int blocks = (int)div_up(a.n, kRowsPerBlock);
    R = a.n_train;
    GCNSA_STEP(launch(mask_counts, blocks, kRowsPerBlock, 0, s, a.n, a.mask, (int*)(ws + pl.counts)));
    GCNSA_STEP(launch(mask_places, blocks, kRowsPerBlock, 0, s, a.n, a.mask, (const int*)(ws + pl.counts), R, (int32_t*)(ws + pl.place),
                      (int32_t*)(ws + pl.rows), (int*)(ws + pl.total)));
    GCNSA_STEP(launch(gather_rows, (int)std::min<int64_t>(div_up(a.n, 8), 148 * 8), 256, 0, s, a.n, a.d, a.h, a.ldh, a.y,
                      (const int32_t*)(ws + pl.place), (const int*)(ws + pl.total), R, f_at(pl.hc), up4(a.d), (int32_t*)(ws + pl.yc), a.dh, a.lddh));
    note_launch(3);
    h = f_at(pl.hc);
    ldh = up4(a.d);
    y = (const int32_t*)(ws + pl.yc);
    rows = (const int32_t*)(ws + pl.rows);
    total = (const int*)(ws + pl.total);
  } else if (a.n > 0 && (((uintptr_t)h & 15) || ldh % 4)) {  // TMA wants lines on 16-byte boundaries
    GCNSA_STEP(launch_copy_rows(stream, a.n, a.d, a.h, a.ldh, f_at(pl.hc), up4(a.d)));
    h = f_at(pl.hc);
    ldh = up4(a.d);
  }
  if (R > 0 && (((uintptr_t)w & 15) || ldw % 4)) {
    GCNSA_STEP(launch_copy_rows(stream, a.d, a.c, a.w, a.ldw, f_at(pl.wc), up4(a.c)));
    w = f_at(pl.wc);
    ldw = up4(a.c);
  }

  const int64_t ldg = up4(R);
  TermArgs t = {};  // z
  t.ce.bias = a.bias;
  t.ce.y = y;
  t.ce.ldg = (int)ldg;
  t.ce.inv_nt = inv_nt;
  if (R > 0) {
    Product& p = t.p[0];
    if (!term_map(&p.map_a, h, false, R, a.d, ldh, BK, BM, true) || !term_map(&p.map_b, w, false, a.d, a.c, ldw, 32, BK, false))
      return (int)cudaErrorNotSupported;
    p.M = (int)R;
    p.N = a.c;
    p.units = (int)div_up(a.d, BK);
    p.k_rows = a.d;
  }
  // loss: sums of warps or blocks, which the first launch of add_slices finishes
  LossSum* const losses = (LossSum*)(ws + pl.losses);
  LossEnd end;
  end.sums = losses;
  end.total = total;
  end.n_train = a.n_train;
  end.loss = a.loss;
  if (R > 0 && whole) {
    t.ce.mask = a.mask;
    t.ce.gt = grads ? f_at(pl.gt) : nullptr;
    t.ce.losses = losses;
    set_slices(t.p[0], a.c <= 64 ? 64 : 128, 1);
    t.total = t.p[0].items;
    const int grid = std::min(t.total, sms);
    end.n = grid * kFoldWarps;
    GCNSA_STEP(a.c <= 64 ? run_terms<TermShape<64, ASrc::kMajor, false, Out::whole>>(s, t, grid)
                         : run_terms<TermShape<128, ASrc::kMajor, false, Out::whole>>(s, t, grid));
    note_launch();
  } else if (R > 0) {
    t.ce.zy = f_at(pl.zy);
    t.ce.part_m = f_at(pl.part);
    t.ce.part_s = f_at(pl.part) + pl.slots * 2 * BM;
    set_slices(t.p[0], 128, 1);
    t.total = t.p[0].items;
    const int grid = std::min(t.total, sms);
    GCNSA_STEP((run_terms<TermShape<128, ASrc::kMajor, false, Out::stats>>(s, t, grid)));
    end.n = (int)div_up(R, 256);
    GCNSA_STEP(launch(row_finish, end.n, 256, 0, s, R, a.c, t.p[0].tiles_n, t.total, grid, (const float*)t.ce.part_m, (const float*)t.ce.part_s,
                      y, (const float*)t.ce.zy, (float2*)(ws + pl.top), losses));
    note_launch(2);
    t.ce.top = (const float2*)(ws + pl.top);
  }
  if (!grads || R == 0 || (!a.dw && !a.db)) {  // no launch of add_slices to come
    GCNSA_STEP(launch(loss_total, 1, 256, 0, s, end.n, (const LossSum*)losses, total, a.n_train, a.loss));
    note_launch();
    end.loss = nullptr;
  }
  if (!grads) return 0;
  if (R == 0) {  // nothing counts: sums of nothing
    if (a.dw || a.db)
      GCNSA_STEP(launch_add_slices(s, a.dw ? a.d : 0, a.c, 0, nullptr, up4(a.c), a.dw, a.lddw, a.dw ? std::min<int64_t>(a.lddw, up4(a.c)) : a.c, 0, nullptr, a.db, a.accumulate));
    return 0;
  }
  const int64_t piece = whole ? a.c : piece_classes(pl, R, a.d, a.c);
  for (int64_t c0 = 0; c0 < a.c; c0 += piece) {
    const int64_t width = std::min<int64_t>(piece, a.c - c0);
    if (!whole) {
      if (!term_map(&t.p[0].map_b, w + c0, false, a.d, width, ldw, 32, BK, false)) return (int)cudaErrorNotSupported;
      t.p[0].N = (int)width;
      t.ce.c0 = (int)c0;
      t.ce.gt = f_at(pl.gt);
      set_slices(t.p[0], 128, 1);
      t.total = t.p[0].items;
      GCNSA_STEP((run_terms<TermShape<128, ASrc::kMajor, false, Out::grad>>(s, t, std::min(t.total, sms))));
      note_launch();
    }
    TermArgs b = {};
    Product &pw = b.p[0], &ph = b.p[1];
    const bool weights = a.dw || a.db;
    // pad columns belong to the last piece
    const int64_t dw_pad = a.dw && c0 + width == a.c ? std::min<int64_t>(a.lddw - c0, up4(width)) : width;
    int slices = 1;
    if (weights) {
      if (!term_map(&pw.map_a, f_at(pl.gt), false, width, R, ldg, BK, BM, true) || !term_map(&pw.map_b, h, false, R, a.d, ldh, 32, BK, false))
        return (int)cudaErrorNotSupported;
      pw.M = (int)width;
      pw.N = a.d;
      pw.units = (int)div_up(R, BK);
      // (also where dh is not asked for: the same slices, the same bits)
      slices = balanced_slices(div_up(width, BM) * div_up(a.d, 128), pw.units, div_up(a.d, BM) * div_up(R, 128), div_up(width, BK));
      set_slices(pw, 128, slices);
      const bool split = slices > 1;
      pw.write = a.dw != nullptr;
      pw.c = split ? f_at(pl.partial) : a.dw + (a.dw ? c0 : 0);
      pw.ldc = split ? up4(width) : a.lddw;
      pw.slice_stride = split ? a.d * up4(width) : 0;
      pw.accumulate = split ? 0 : a.accumulate;
      pw.m_pad = (int)(split ? up4(width) : dw_pad);
      pw.k_rows = R;
      pw.k_mask = whole ? a.mask : nullptr;  // (rows that do not count are still there: 0 in G, but 0 x NaN is NaN)
      if (a.db) {
        pw.a_sums = f_at(pl.sums);
        pw.sums_pitch = up4(width);
      }
    }
    if (a.dh) {
      if (!term_map(&ph.map_a, w + c0, false, a.d, width, ldw, BK, BM, true) || !term_map(&ph.map_b, f_at(pl.gt), false, width, R, ldg, 32, BK, false))
        return (int)cudaErrorNotSupported;
      ph.M = a.d;
      ph.N = (int)R;
      ph.units = (int)div_up(width, BK);
      set_slices(ph, 128, 1);
      ph.write = 1;
      ph.c = a.dh;
      ph.ldc = a.lddh;
      ph.row_map = rows;
      ph.map_rows = a.n;
      ph.accumulate = c0 > 0;
      ph.m_pad = (int)std::min<int64_t>(a.lddh, up4(a.d));
      ph.k_rows = width;
    }
    b.total = pw.items + ph.items;
    GCNSA_STEP((run_terms<TermShape<128, ASrc::kMajor, false, Out::transposed>>(s, b, std::min(b.total, sms))));
    note_launch();
    const bool add = a.dw && slices > 1;
    if (add || a.db || end.loss) {
      GCNSA_STEP(launch_add_slices(s, add ? a.d : 0, width, slices, f_at(pl.partial), up4(width), add ? a.dw + c0 : nullptr, a.lddw, add ? dw_pad : width,
                                   kSumLines * slices, f_at(pl.sums), a.db ? a.db + c0 : nullptr, a.accumulate, end));
      end.loss = nullptr;
    }
  }
  return 0;
}

int debug_word_head(unsigned long long* out, bool clear) {
  *out = 0ull;
#if GCNSA_DBG
  cudaError_t e = cudaMemcpyFromSymbol(out, g_dbg_head, sizeof(*out));
  if (e == cudaSuccess && clear) {
    const unsigned long long zero = 0ull;
    e = cudaMemcpyToSymbol(g_dbg_head, &zero, sizeof(zero));
  }
  return (int)e;
#else
  (void)clear;
  return 0;
#endif
}

int tc_status_head(int* out) {
  int v = 0;
  cudaError_t e = cudaMemcpyFromSymbol(&v, g_tc_error, sizeof(int));
  if (e != cudaSuccess) return (int)e;
  *out = v;
  return 0;
}

int tc_clear_head() {
  const int zero = 0;
  return (int)cudaMemcpyToSymbol(g_tc_error, &zero, sizeof(int));
}

}  // namespace gcnsa
