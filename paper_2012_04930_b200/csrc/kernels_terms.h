// D = A B on the 5th-generation tensor cores from bf16 terms, with sums that keep fp32 accuracy however long they are.
//
// A fp32 value is the exact sum of three bf16 terms (24 significant bits cut into 8 + 8 + 8); of the nine products of two
// such operands the three smallest are left out (each below 2^-21 of the product, about 2^-24 on average).  An operand that is an 8-bit checkpoint
// is one bf16 term.  The tensor core cuts a sum off at 24 bits, always toward zero, where an fp32 addition rounds, so an
// accumulator may not live long: the products of the leading terms go into one of two accumulators in turn, two
// instructions per 32 k, and after 256 k its sum is added to running sums in registers (rounded), while the
// MMAs go on in the other one.  The products of the smaller terms have a third accumulator; what is cut off there is
// 2^-8 of that, and it is folded every kSmallFolds folds.  (One accumulator for everything over 245 000 rows would be
// 1e-4 off.)
//
// One CTA per SM works on tiles of 128 x BN.  Warps 0 and 2 stream boxes of A and B into rings of shared memory with TMA.
// Groups of four warps make the terms, a k-block of an operand each at a time: two for A (three where B is packed and its
// terms are ready sooner), three terms in tensor memory (a lane per row of the tile, two k per 32-bit column), and two for B, one
// or three terms in MN-major tiles with the 128-byte swizzle.  (With both operands of a k-block in one group's hands, a stage that the MMAs had
// given back stood empty for 1 700 clocks.)  Warp 1 issues the MMAs, and eight warps (two per lane quarter of tensor memory,
// half the columns each) fold the accumulators and write the result: thread = row of the tile, so a result that is
// wanted transposed, D[m, n] at c[n * ldc + m], is written in lines of 128 bytes without a turn through shared memory.
// Every product of this file is arranged so that this is the layout it needs.
//
// A k-block of 32 of a 128 x 128 tile keeps the tensor pipe busy for 768 clocks (12 MMAs) and shared memory for about
// 1 090 (boxes in 256, both read for the split 256, terms of B out 192, B read by the MMAs 384, at 128 bytes a clock).
// Counters of the passes over 20 011 x 256 x 10 007 classes: tensor pipe 50-58 % busy, issue slots 66-74 %, ALUs 60-65 %, DRAM at
// most 28 %; of a weight gradient from a checkpoint (245 000 rows, 256 x 256): 40 %, 74 %, 58 %, 36 %.  Making terms, not
// the MMAs, is what these products wait for.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>

#include "debug_check.h"
#include "launch.h"
#include "pack8_device.h"
#include "register_split.h"
#include "tc_device.h"
#include "tma_host.h"

namespace gcnsa {
namespace {

#if GCNSA_DBG
GCNSA_DBG_WORD(g_dbg_head);
#endif

constexpr int BM = 128, BK = 32;
constexpr int kAWarp0 = 4, kFoldWarps = 8;
constexpr int kSmallFolds = 8, kRetired = 8;
constexpr int A_SLOT = BM * BK * 4;

// A: K-major (k contiguous in memory), MN-major (rows of D contiguous), or MN-major without the alignment that TMA needs
// (read with plain loads)
enum class ASrc { kMajor, mnMajor, direct };
enum class Out { transposed, stats, grad, whole };

// D[m, n] = sum_k A[m, k] B[k, n], B MN-major
struct Product {
  CUtensorMap map_a, map_b;
  int M, N, units, per_slice, tiles_m, tiles_n, items;  // units: k-blocks of 32; items = tiles x slices
  float* c;                // element (m, n) at c[z * slice_stride + row(n) * ldc + m]
  int64_t ldc, slice_stride;
  const int32_t* row_map;  // row(n), nullable; negative: not written
  int64_t map_rows;        // rows that row_map leads to
  int accumulate, m_pad;   // columns [M, m_pad) of a line are written as zeros (left as they are with accumulate)
  float* a_sums;           // nullable: sums of A's rows (over k) of slice z, k-blocks of group g: a_sums[(AG z + g) * sums_pitch + m]
  int64_t sums_pitch;
  int write;               // 0: only a_sums are wanted
  const float* a;          // ASrc::direct
  int64_t lda, k_rows;
  const uint8_t* k_mask;   // nullable [k_rows], B as floats: lines of B whose byte is 0 count as zeros, whatever they hold
  const uint8_t* e;        // steps of a packed B
  int64_t lde;
  int e_blocks;
};
// Sum of row losses and number of rows that count.
struct LossSum {
  double loss;
  long long count;
};
// The epilogues of the output layer; D[m, n] is a logit without its bias, m a row, n a class of the piece from c0 on.
struct CeTile {
  const float* bias;     // nullable, of the whole layer
  const int32_t* y;      // [M]
  const uint8_t* mask;   // nullable [M] (Out::whole)
  int c0, ldg;
  float inv_nt;
  float* gt;             // G^T: [class of the piece][ldg]; nullable (Out::whole)
  const float2* top;     // [M] maximum and 1 / sum of exponentials of a row (Out::grad)
  float *part_m, *part_s, *zy;  // (Out::stats) running maximum and sum of a CTA's run in a row tile, the label's logit
  LossSum* losses;       // (Out::whole) a sum per fold warp of the grid
};
struct TermArgs {
  Product p[2];
  CeTile ce;
  int total;  // items of both
};

__device__ __forceinline__ void tma_load_2d(void* dst, const CUtensorMap* map, int x, int y, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(
          smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(smem_u32(bar))
      : "memory");
}
// MN-major tile of 16-bit elements, 128-byte swizzle: blocks of 64 n x 32 k (4 096 bytes apart), in a block the 64 elements of
// one k are 128 contiguous bytes and 8 k are a swizzle group of 1 024 bytes.
__device__ __forceinline__ uint64_t desc_b(uint32_t smem_addr) {
  uint64_t d = 0;
  d |= (uint64_t)((smem_addr & 0x3FFFF) >> 4);
  d |= (uint64_t)(4096 >> 4) << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}
__device__ __forceinline__ void umma_bf16_ta(uint32_t tmem_d, uint32_t tmem_a, uint64_t bdesc, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n"
      " .reg .pred p;\n"
      " setp.ne.b32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n"
      "}\n" ::"r"(tmem_d),
      "r"(tmem_a), "l"(bdesc), "r"(idesc), "r"(acc)
      : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
      "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
      "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
      : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
        "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
      : "r"(taddr)
      : "memory");
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}
// Bounded wait as mbar_wait, for phases that last microseconds: the thread asks to be put aside for up to 2 us at a time, as 12
// warps that poll take a third of the issue slots from those that split and fold.
__device__ __forceinline__ bool mbar_wait_long(uint64_t* bar, uint32_t parity, int code) {
  if (mbar_try_wait(bar, parity)) return true;
  const long long t0 = clock64();
  for (;;) {
    uint32_t ok;
    asm volatile(
        "{\n"
        " .reg .pred p;\n"
        " mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, 2000;\n"
        " selp.u32 %0, 1, 0, p;\n"
        "}\n"
        : "=r"(ok)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
    if (ok) return true;
    if (tc_error_now() != 0) return false;
    if (clock64() - t0 > kSpinCycles) {
      atomicCAS(&g_tc_error, 0, code);
      return false;
    }
  }
}
// 2^x (2 units in the last place; 0 for -infinity, NaN for NaN)
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
constexpr float kLog2e = 1.44269504088896340736f;
// Two values as three pairs of bf16 terms, the first value in the lower halves.  Every term is what its upper 16 bits say (cut
// off, not rounded: no finite value becomes an infinity, and a byte permute packs two of them, where cvt.rn.bf16x2 has a
// fraction of that rate); 8 + 8 + 8 bits are all that a value has.  An infinity leaves a NaN as its second term: products with
// one are NaN.  (To keep it would take a test per value, and infinity times a second term of 0 is NaN all the same.)
__device__ __forceinline__ void split3(float x0, float x1, uint32_t& t0, uint32_t& t1, uint32_t& t2) {
  auto upper = [](float v) { return __uint_as_float(__float_as_uint(v) & 0xffff0000u); };
  t0 = __byte_perm(__float_as_uint(x0), __float_as_uint(x1), 0x7632);
  x0 -= upper(x0);
  x1 -= upper(x1);
  t1 = __byte_perm(__float_as_uint(x0), __float_as_uint(x1), 0x7632);
  x0 -= upper(x0);
  x1 -= upper(x1);
  t2 = __byte_perm(__float_as_uint(x0), __float_as_uint(x1), 0x7632);
}

template <int BN_, ASrc A_, bool P8_, Out OUT_>
struct TermShape {
  static constexpr int BN = BN_;
  static constexpr ASrc A = A_;
  static constexpr bool P8 = P8_;
  static constexpr Out OUT = OUT_;
  static constexpr int NTB = P8 ? 1 : 3;                 // terms of B
  static constexpr int AG = P8 ? 3 : 2, BG = 2;          // groups of four warps that make terms of A, of B
  static constexpr int BWARP0 = kAWarp0 + 4 * AG, FWARP0 = BWARP0 + 4 * BG, THREADS = 32 * (FWARP0 + kFoldWarps);
  // registers per thread by role, in multiples of 8; their sum over the warpgroups is at most what the launch gives
  static constexpr int REGS = P8 ? 64 : 72;              // (the compiler's, with that many threads; run_terms asks)
  static constexpr int REGS_ISSUE = P8 ? 24 : 32, REGS_A = 72, REGS_B = P8 ? 48 : 64, REGS_FOLD = P8 ? 88 : 96;
  static constexpr bool A_INC = REGS_A > REGS;
  static constexpr RegisterShare SHARES[4] = {{1, REGS_ISSUE, false}, {AG, REGS_A, A_INC}, {BG, REGS_B, false}, {kFoldWarps / 4, REGS_FOLD, true}};
  static_assert(registers_hold(REGS, SHARES), "setmaxnreg draws on the registers of the launch");
  static constexpr int HALF = BN / 2;                    // columns of a fold warp
  // With one term of B all three products of a k-block share an accumulator, which is folded twice as often; the columns of
  // the third one hold more stages of A.
  static constexpr bool SMALL = !P8;
  static constexpr int FOLD = SMALL ? 8 : 4;             // k-blocks to a fold
  static constexpr int A_COLS = 48, A_COL0 = (SMALL ? 3 : 2) * BN, TMEM_COLS = 512;  // tensor-memory columns
  static constexpr int NSA = (TMEM_COLS - A_COL0) / A_COLS < 5 ? (TMEM_COLS - A_COL0) / A_COLS : 5, NSB = P8 ? 6 : 3;  // stages of terms
  static constexpr int B_SLOT = BK * BN * (P8 ? 1 : 4), B_TERM = BK * BN * 2;
  // Landing slots, a multiple of the groups: a slot's boxes are then all read by one group, in order.  (A wait by parity cannot
  // tell a phase from the one two before it, and boxes land out of order: with four slots and three groups a group could
  // take a slot whose box before the last was still on its way for one that had landed.)
  static constexpr int NA = A == ASrc::direct ? 0 : P8 ? 6 : 4, NB = P8 ? 6 : 4;
  static constexpr int B_OFF = NA * A_SLOT, T_OFF = B_OFF + NB * B_SLOT, X_OFF = T_OFF + NSB * NTB * B_TERM;
  // biases of the fold warps' classes; maxima and sums of the halves of a row
  static constexpr int X_BYTES = (OUT != Out::transposed ? kFoldWarps * HALF * 4 : 0) + (OUT == Out::whole ? 2 * 2 * BM * 4 : 0);
  static constexpr int BAR_OFF = X_OFF + X_BYTES;
  // more than half of an SM's shared memory: a second CTA, which would wait for tensor memory, never shares the SM
  static constexpr int NEED = BAR_OFF + 512 + 1024;
  static constexpr int SMEM_BYTES = NEED > 118 * 1024 ? NEED : 118 * 1024;
  static_assert(NA % AG == 0 && NB % BG == 0, "a slot belongs to one group");
  // A group that waits for the MMAs of k-block g - NS has seen those of g - NS - (its groups) retire, so the phase before the
  // last of that barrier, k-block g - NS - kRetired, has ended.
  static_assert(kRetired >= AG && kRetired >= BG, "the phase before the last of a retire barrier has ended");
  static_assert(A_COL0 + NSA * A_COLS <= TMEM_COLS, "tensor memory has 512 columns");
  static_assert(SMEM_BYTES <= 227 * 1024, "shared memory of one CTA");
};

struct TermWork {
  int prob, m0, n0, z, kb0, n_kb;
};
__device__ __forceinline__ TermWork term_work(const TermArgs& a, int w, int bn) {
  TermWork k;
  k.prob = w >= a.p[0].items;
  if (k.prob) w -= a.p[0].items;
  const Product& p = a.p[k.prob];
  const int tiles = p.tiles_m * p.tiles_n;
  k.z = w / tiles;
  w -= k.z * tiles;
  k.m0 = w / p.tiles_n * BM;
  k.n0 = w % p.tiles_n * bn;
  k.kb0 = k.z * p.per_slice;
  k.n_kb = max(min(p.units, k.kb0 + p.per_slice) - k.kb0, 0);
  return k;
}
// The items of a CTA: every gridDim.x-th, or (Out::stats) a run of neighbours, which lie in one row tile or a few.
template <class S>
__device__ __forceinline__ void term_items(int total, int& first, int& end, int& step) {
  if constexpr (S::OUT == Out::stats) {
    first = (int)((int64_t)total * blockIdx.x / gridDim.x);
    end = (int)((int64_t)total * (blockIdx.x + 1) / gridDim.x);
    step = 1;
  } else {
    first = blockIdx.x;
    end = total;
    step = gridDim.x;
  }
}
// the CTA whose run has item i
__host__ __device__ inline int term_owner(int i, int total, int grid) { return (int)(((int64_t)(i + 1) * grid - 1) / total); }

// A group's k-block of B.  Loaded as a whole before the first term is written: the compiler cannot tell that the boxes and the terms
// do not overlap, and line by line every load would wait for the stores before it.
template <class S, bool P8 = S::P8>
struct TermB {  // a lane has four neighbouring n of line(i), i below COUNT
  static constexpr int LANES = S::BN / 4, LINES = 32 / LANES, COUNT = 8 / LINES;  // lanes of a line, lines per instruction
  float4 x[COUNT];
  static __device__ __forceinline__ int line(int i, int wq, int lane) { return wq * 8 + i * LINES + lane / LANES; }
  __device__ __forceinline__ void load(const uint8_t* raw, int wq, int lane) {
    const int n = 4 * (lane % LANES);
#pragma unroll
    for (int i = 0; i < COUNT; ++i) x[i] = *reinterpret_cast<const float4*>(raw + (n / 32) * 4096 + line(i, wq, lane) * 128 + (n & 31) * 4);
  }
  // zeros for the lines wq * 8 + k with bit k of `lines`
  __device__ __forceinline__ void clear(uint32_t lines, int lane) {
#pragma unroll
    for (int i = 0; i < COUNT; ++i)
      if ((lines >> line(i, 0, lane)) & 1u) x[i] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  __device__ __forceinline__ void store(uint8_t* terms, int wq, int lane, uint32_t) const {
    const int n = 4 * (lane % LANES);
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
      const int k = line(i, wq, lane);
      uint8_t* dst = terms + (n / 64) * 4096 + k * 128 + ((((n & 63) >> 3) ^ (k & 7)) << 4) + (n & 7) * 2;
      uint2 t0, t1, t2;
      split3(x[i].x, x[i].y, t0.x, t1.x, t2.x);
      split3(x[i].z, x[i].w, t0.y, t1.y, t2.y);
      *reinterpret_cast<uint2*>(dst) = t0;
      *reinterpret_cast<uint2*>(dst + S::B_TERM) = t1;
      *reinterpret_cast<uint2*>(dst + 2 * S::B_TERM) = t2;
    }
  }
};
template <class S>
struct TermB<S, true> {  // a lane has 16 neighbouring n, half a block of the checkpoint
  static constexpr int LANES = S::BN / 16, LINES = 32 / LANES, COUNT = 8 / LINES;
  uint4 q[COUNT];
  static __device__ __forceinline__ int line(int i, int wq, int lane) { return wq * 8 + i * LINES + lane / LANES; }
  __device__ __forceinline__ void load(const uint8_t* raw, int wq, int lane) {
#pragma unroll
    for (int i = 0; i < COUNT; ++i) q[i] = *reinterpret_cast<const uint4*>(raw + line(i, wq, lane) * S::BN + 16 * (lane % LANES));
  }
  // e8: the step of line wq * 8 + lane / (BN / 32), block lane % (BN / 32)
  __device__ __forceinline__ void store(uint8_t* terms, int wq, int lane, uint32_t e8) const {
    const int n = 16 * (lane % LANES);
    const bool odd = n >= 64;  // the second block's lanes write their halves the other way round: all banks, once each
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
      const int k = line(i, wq, lane);
      const float step = pack8_step(__shfl_sync(0xffffffffu, e8, (k & 7) * (S::BN / 32) + n / 32));
      uint8_t* dst = terms + (n / 64) * 4096 + k * 128;
      const uint32_t half[2][2] = {{odd ? q[i].z : q[i].x, odd ? q[i].w : q[i].y}, {odd ? q[i].x : q[i].z, odd ? q[i].y : q[i].w}};
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t w[4];
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          float v[4];
          pack8_open(half[h][p], v);
          w[2 * p] = __byte_perm(__float_as_uint(v[0] * step), __float_as_uint(v[1] * step), 0x7632);
          w[2 * p + 1] = __byte_perm(__float_as_uint(v[2] * step), __float_as_uint(v[3] * step), 0x7632);
        }
        const int chunk = ((n & 63) >> 3) + (h ^ (odd ? 1 : 0));
        *reinterpret_cast<uint4*>(dst + ((chunk ^ (k & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
  }
};

template <class S>
__global__ void __launch_bounds__(S::THREADS, 1) term_product(const __grid_constant__ TermArgs args) {
  constexpr int BN = S::BN, NA = S::NA, NB = S::NB, NSA = S::NSA, NSB = S::NSB, NTB = S::NTB, HALF = S::HALF;
  constexpr bool A_TMA = S::A != ASrc::direct;
  extern __shared__ uint8_t smem_raw[];
  // (an offset, not a rounded pointer: the compiler then knows that this is shared memory and need not use generic accesses)
  uint8_t* const smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
  uint64_t* full_a = reinterpret_cast<uint64_t*>(smem + S::BAR_OFF);  // box landed
  uint64_t* free_a = full_a + (NA ? NA : 1);                           // slot read
  uint64_t* full_b = free_a + (NA ? NA : 1);
  uint64_t* free_b = full_b + NB;
  uint64_t* ready_a = free_b + NB;        // [NSA] terms in place
  uint64_t* ready_b = ready_a + NSA;      // [NSB]
  uint64_t* retired = ready_b + NSB;      // [kRetired] MMAs of k-block g have read their operands: barrier g % kRetired
  uint64_t* acc_full = retired + kRetired;  // [2]
  uint64_t* acc_empty = acc_full + 2;     // [2] read back by the fold warps
  uint64_t* small_empty = acc_empty + 2;
  uint64_t* pair = small_empty + 1;       // [4] the two fold warps of a lane quarter (Out::whole)
  uint64_t* drain = pair + 4;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 1);
  int* abort_slot = reinterpret_cast<int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // a wait ran out in an earlier launch or in another CTA of this one: nothing is allocated, nothing is computed
  if (threadIdx.x == 0) *abort_slot = tc_error_now();
  __syncthreads();
  if (*abort_slot != 0) {
    wait_for_predecessors();
    return;
  }
  if (threadIdx.x == 0) {
    for (int i = 0; i < NA; ++i) {
      mbar_init(&full_a[i], 1);
      mbar_init(&free_a[i], 4);
    }
    for (int i = 0; i < NB; ++i) {
      mbar_init(&full_b[i], 1);
      mbar_init(&free_b[i], 4);
    }
    for (int i = 0; i < NSB; ++i) {
      mbar_init(&ready_b[i], 4);
    }
    for (int i = 0; i < NSA; ++i) mbar_init(&ready_a[i], 4);
    for (int i = 0; i < kRetired; ++i) mbar_init(&retired[i], 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(&acc_full[i], 1);
      mbar_init(&acc_empty[i], kFoldWarps);
    }
    mbar_init(small_empty, kFoldWarps);
    for (int i = 0; i < 4; ++i) mbar_init(&pair[i], 2);
    mbar_init(drain, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)),
                 "r"(S::TMEM_COLS)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem_base = *tmem_slot;
  wait_for_predecessors();  // barriers and tensor memory are up; from here on global memory is read

  int w0, w_end, w_step;
  term_items<S>(args.total, w0, w_end, w_step);

  if (warp < kAWarp0) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(S::REGS_ISSUE));
    if ((warp == 0 && A_TMA) || warp == 2) {
      // ---------------- TMA producers: warp 0 streams A, warp 2 streams B ----------------
      if (elect_one()) {
        const bool is_a = warp == 0;
        const uint32_t ring = is_a ? (NA ? NA : 1) : NB;
        uint64_t* full = is_a ? full_a : full_b;
        uint64_t* freed = is_a ? free_a : free_b;
        uint32_t g = 0;  // k-blocks issued so far, over all items
        bool ok = true;
        for (int w = w0; ok && w < w_end; w += w_step) {
          const TermWork wk = term_work(args, w, BN);
          const Product& p = args.p[wk.prob];
          for (int it = 0; it < wk.n_kb; ++it, ++g) {
            const uint32_t s = g % ring, ph = (g / ring) & 1;
            ok = mbar_wait_long(&freed[s], ph ^ 1, is_a ? 41 : 42);
            if (!ok) break;
            const int kx = (wk.kb0 + it) * BK;
            if (is_a) {
              uint8_t* dst = smem + s * A_SLOT;
              mbar_expect_tx(&full[s], A_SLOT);
              if (S::A == ASrc::kMajor) {
                tma_load_2d(dst, &p.map_a, kx, wk.m0, &full[s]);
              } else {
#pragma unroll
                for (int j = 0; j < BM / 32; ++j) tma_load_2d(dst + j * 4096, &p.map_a, wk.m0 + 32 * j, kx, &full[s]);
              }
            } else {
              uint8_t* dst = smem + S::B_OFF + s * S::B_SLOT;
              mbar_expect_tx(&full[s], S::B_SLOT);
              if (S::P8) {
                tma_load_2d(dst, &p.map_b, wk.n0, kx, &full[s]);
              } else {
#pragma unroll
                for (int j = 0; j < BN / 32; ++j) tma_load_2d(dst + j * 4096, &p.map_b, wk.n0 + 32 * j, kx, &full[s]);
              }
            }
          }
        }
        if (!ok || tc_error_now() != 0) {  // wind down: let the copies already issued land before the CTA exits
          const long long t0 = clock64();
          for (uint32_t gi = g > ring ? g - ring : 0; gi < g; ++gi) {
            const uint32_t ph = (gi / ring) & 1;
            while (!mbar_try_wait(&full[gi % ring], ph) && clock64() - t0 < kSpinCycles) {
            }
          }
        }
      }
    } else if (warp == 1) {
      // ---------------- MMA issuer ----------------
      // (the whole warp walks the k-blocks and one elected thread issues, so that addresses stay in uniform registers)
      const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(BN >> 3) << 17) | (8u << 24);
      const uint32_t tm = __shfl_sync(0xffffffffu, tmem_base, 0);
      const uint64_t b0 = desc_b(smem_u32(smem + S::T_OFF));
      uint32_t g = 0, folds = 0, smalls = 0;  // k-blocks, folds of the main and of the small accumulator so far
      bool ok = true;
      for (int w = w0; ok && w < w_end; w += w_step) {
        const TermWork wk = term_work(args, w, BN);
        for (int it = 0; it < wk.n_kb; ++it, ++g) {
          const uint32_t sa = g % NSA, pa = (g / NSA) & 1, sb = g % NSB, pb = (g / NSB) & 1;
          const int in_fold = it % S::FOLD, in_small = it % (S::FOLD * kSmallFolds);
          // (the questions are asked at once, their answers take 30 clocks each; only a no leads to a wait)
          const bool have_b = mbar_try_wait(&ready_b[sb], pb), have_a = mbar_try_wait(&ready_a[sa], pa);
          if (in_fold == 0) ok = mbar_wait(&acc_empty[folds & 1], ((folds >> 1) & 1) ^ 1, 46);
          if (S::SMALL && ok && in_small == 0) ok = mbar_wait(small_empty, (smalls & 1) ^ 1, 47);
          if (!have_b) ok = ok && mbar_wait(&ready_b[sb], pb, 43);
          if (!have_a) ok = ok && mbar_wait(&ready_a[sa], pa, 52);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const bool last_fold = in_fold == S::FOLD - 1 || it == wk.n_kb - 1;
          const bool last_small = in_small == S::FOLD * kSmallFolds - 1 || it == wk.n_kb - 1;
          const uint32_t d_main = tm + (folds & 1) * BN, d_small = S::SMALL ? tm + 2 * BN : d_main, ta = tm + S::A_COL0 + sa * S::A_COLS;
          const uint64_t bs = b0 + (uint64_t)((sb * NTB * S::B_TERM) >> 4);
          if (elect_one()) {
#pragma unroll
            for (int kk = 0; kk < BK / 16; ++kk) {
              const uint64_t bk = bs + (uint64_t)((kk * 2048) >> 4);
              constexpr uint64_t term = S::B_TERM >> 4;
              const uint32_t a0 = ta + 8 * kk, a1 = a0 + 16, a2 = a0 + 32;
              // small terms first, the smallest before all
              umma_bf16_ta(d_small, a2, bk, idesc, kk != 0 || (S::SMALL ? in_small : in_fold) != 0);
              if constexpr (NTB == 3) {
                umma_bf16_ta(d_small, a0, bk + 2 * term, idesc, 1);
                umma_bf16_ta(d_small, a1, bk + term, idesc, 1);
                umma_bf16_ta(d_small, a0, bk + term, idesc, 1);
              }
              umma_bf16_ta(d_small, a1, bk, idesc, 1);
              umma_bf16_ta(d_main, a0, bk, idesc, !S::SMALL || kk != 0 || in_fold != 0);
            }
            umma_commit(&retired[g % kRetired]);  // arrives when the MMAs above have read their operands
            if (last_fold) umma_commit(&acc_full[folds & 1]);
          }
          __syncwarp();
          if (last_fold) ++folds;
          if (last_small) ++smalls;
        }
      }
      if (!ok && g > 0) {
        // a wait ran out: the MMAs issued so far must have retired before tensor memory is given back
        if (elect_one()) umma_commit(drain);
        const long long t0 = clock64();
        while (!mbar_try_wait(drain, 0) && clock64() - t0 < kSpinCycles) {
        }
      }
    }
  } else if (warp < S::BWARP0) {
    // ---------------- terms of A: every AG-th k-block to a group ----------------
    if constexpr (S::A_INC) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(S::REGS_A));
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(S::REGS_A));
    const int q = warp & 3, group = (warp - kAWarp0) >> 2, row = 32 * q + lane;  // row of the tile
    uint32_t g = 0;
    bool ok = true;
    for (int w = w0; ok && w < w_end; w += w_step) {
      const TermWork wk = term_work(args, w, BN);
      const Product& p = args.p[wk.prob];
      float a_sum = 0.f;
      const bool sums = p.a_sums != nullptr && wk.n0 == 0;
      // (fields of p are copied where a loop uses them: with the product's index a variable each would be a load every time)
      const float* const a_at = A_TMA ? nullptr : p.a + wk.m0 + row;
      const int64_t lda = p.lda, k_rows = p.k_rows;
      const bool in_m = wk.m0 + row < p.M;
      int it = (int)((group + S::AG - g % S::AG) % S::AG);  // first k-block of this group in the item
      g += it;
      for (; it < wk.n_kb; it += S::AG, g += S::AG) {
        float x[32];
        if constexpr (!A_TMA) {
          const int64_t k0 = (int64_t)(wk.kb0 + it) * BK;
          const float* src = a_at + k0 * lda;
#pragma unroll
          for (int k = 0; k < 32; ++k) x[k] = in_m && k0 + k < k_rows ? __ldg(src + k * lda) : 0.f;
        } else {
          ok = __all_sync(0xffffffffu, mbar_wait_long(&full_a[g % NA], (g / NA) & 1, 48));  // the warp gives up as a whole
          if (!ok) break;
          const uint8_t* slot = smem + (g % NA) * A_SLOT;
          if constexpr (S::A == ASrc::kMajor) {
            // 128-byte swizzle: the 16-byte chunk c of row r sits at chunk position c ^ (r % 8)
            const uint8_t* arow = slot + (row >> 3) * 1024 + (row & 7) * 128;
#pragma unroll
            for (int c = 0; c < 8; ++c) {
              const float4 v = *reinterpret_cast<const float4*>(arow + ((c ^ (row & 7)) << 4));
              x[4 * c] = v.x; x[4 * c + 1] = v.y; x[4 * c + 2] = v.z; x[4 * c + 3] = v.w;
            }
          } else {
            const uint8_t* s = slot + q * 4096 + lane * 4;
#pragma unroll
            for (int k = 0; k < 32; ++k) x[k] = *reinterpret_cast<const float*>(s + k * 128);
          }
        }
        if (sums) {
          float s8[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) s8[k] = (x[k] + x[k + 8]) + (x[k + 16] + x[k + 24]);
          a_sum += ((s8[0] + s8[1]) + (s8[2] + s8[3])) + ((s8[4] + s8[5]) + (s8[6] + s8[7]));
        }
        uint32_t t0[16], t1[16], t2[16];
#pragma unroll
        for (int k = 0; k < 16; ++k) split3(x[2 * k], x[2 * k + 1], t0[k], t1[k], t2[k]);
        const uint32_t sa = g % NSA;
        if (g >= NSA) ok = __all_sync(0xffffffffu, mbar_wait(&retired[(g - NSA) % kRetired], ((g - NSA) / kRetired) & 1, 49));
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint32_t ta = tmem_base + ((uint32_t)(32 * q) << 16) + (uint32_t)(S::A_COL0 + sa * S::A_COLS);
        tmem_st16(ta, t0);
        tmem_st16(ta + 16, t1);
        tmem_st16(ta + 32, t2);
        if constexpr (A_TMA) {
          __syncwarp();
          // A slot is given back when what was made of it has been stored, not when it has been loaded: nothing keeps the
          // loads themselves in front of the arrival (with it straight behind them results changed from run to run).
          if (lane == 0) mbar_arrive(&free_a[g % NA]);
        }
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(&ready_a[sa]);
      }
      if (!ok) break;
      g -= it - wk.n_kb;  // k-blocks of all groups
      if (sums && in_m) p.a_sums[(S::AG * (int64_t)wk.z + group) * p.sums_pitch + wk.m0 + row] = a_sum;
    }
  } else if (warp < S::FWARP0) {
    // ---------------- terms of B ----------------
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(S::REGS_B));
    const int q = warp & 3, group = (warp - S::BWARP0) >> 2;
    uint32_t g = 0;
    bool ok = true;
    for (int w = w0; ok && w < w_end; w += w_step) {
      const TermWork wk = term_work(args, w, BN);
      const Product& p = args.p[wk.prob];
      // steps of a packed B: a lane has the one of line q * 8 + lane / (BN / 32) of the k-block, block lane % (BN / 32) of the
      // tile; fetched three k-blocks (of this group) ahead
      constexpr int EB = BN / 32;
      const int64_t lde = p.lde, k_left = p.k_rows - ((int64_t)wk.kb0 * BK + q * 8 + lane / EB);
      const uint8_t* const e_at = p.e + (p.k_rows - k_left) * lde + wk.n0 / 32 + lane % EB;
      const bool e_in = S::P8 && lane < 8 * EB && wk.n0 / 32 + lane % EB < p.e_blocks;
      auto step_of = [&](int it) { return e_in && it < wk.n_kb && it * BK < k_left ? __ldg(e_at + (int64_t)it * BK * lde) : 0u; };
      // lines of B that do not count: a lane has the byte of line q * 8 + lane % 8, fetched one k-block (of this group) ahead
      constexpr bool MASKED = !S::P8 && S::OUT == Out::transposed;
      const uint8_t* const k_mask = MASKED ? p.k_mask : nullptr;
      auto counts = [&](int it) {
        const int64_t k = (int64_t)(wk.kb0 + it) * BK + q * 8 + (lane & 7);
        return !k_mask || it >= wk.n_kb || k >= p.k_rows ? 1u : (uint32_t)__ldg(k_mask + k);
      };
      int it = (int)((group + S::BG - g % S::BG) % S::BG);
      g += it;
      uint32_t counts_next = MASKED ? counts(it) : 1u;
      uint32_t e_next[3];
#pragma unroll
      for (int i = 0; i < 3; ++i) e_next[i] = step_of(it + i * S::BG);
      for (; it < wk.n_kb; it += S::BG, g += S::BG) {
        const uint32_t sb = g % NSB, e8 = e_next[0];
        e_next[0] = e_next[1];
        e_next[1] = e_next[2];
        e_next[2] = step_of(it + 3 * S::BG);
        const uint32_t left_out = MASKED ? __ballot_sync(0xffffffffu, counts_next == 0) & 0xffu : 0u;
        if constexpr (MASKED) counts_next = counts(it + S::BG);
        ok = __all_sync(0xffffffffu, mbar_wait_long(&full_b[g % NB], (g / NB) & 1, 44));
        if (!ok) break;
        TermB<S> tb;
        tb.load(smem + S::B_OFF + (g % NB) * S::B_SLOT, q, lane);
        if constexpr (MASKED)
          if (left_out) tb.clear(left_out, lane);
        if (g >= NSB) ok = __all_sync(0xffffffffu, mbar_wait(&retired[(g - NSB) % kRetired], ((g - NSB) / kRetired) & 1, 45));
        if (!ok) break;
        tb.store(smem + S::T_OFF + sb * NTB * S::B_TERM, q, lane, e8);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // generic-proxy writes -> visible to the MMA
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&free_b[g % NB]);
          mbar_arrive(&ready_b[sb]);
        }
      }
      if (!ok) break;
      g -= it - wk.n_kb;
    }
  } else {
    // ---------------- folds and results ----------------
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(S::REGS_FOLD));
    const int quad = warp & 3, half = (warp - S::FWARP0) >> 2;
    const uint32_t lanes = tmem_base + ((uint32_t)(quad * 32) << 16) + half * HALF;
    uint32_t folds = 0;
    float run_m = -INFINITY, run_s = 0.f;  // (Out::stats)
    uint32_t met = 0;                      // (Out::whole) meetings of the two warps of a quarter
    LossSum mine = {0.0, 0};
    bool ok = true;
    auto meet = [&]() {  // what either wrote to shared memory before is there for the other one; false: a wait ran out
      __syncwarp();
      if (lane == 0) mbar_arrive(&pair[quad]);
      const bool there = __all_sync(0xffffffffu, mbar_wait(&pair[quad], met & 1, 51));
      ++met;
      return there;
    };
    for (int w = w0; ok && w < w_end; w += w_step) {
      const TermWork wk = term_work(args, w, BN);
      const Product& p = args.p[wk.prob];
      const int m = wk.m0 + quad * 32 + lane, nb = wk.n0 + half * HALF;
      const bool row_in = m < p.M;
      // what the epilogue needs of its row, on the way while the sums are made
      int label = -1;
      float2 top = {0.f, 0.f};
      bool on = row_in;
      if constexpr (S::OUT != Out::transposed) {
        if (row_in) label = max(__ldg(args.ce.y + m), -1);
        if constexpr (S::OUT == Out::grad)
          if (row_in) top = __ldg(args.ce.top + m);
        if constexpr (S::OUT == Out::whole) on = row_in && (!args.ce.mask || __ldg(args.ce.mask + m) != 0);
      }
      float sum[HALF];
#pragma unroll
      for (int j = 0; j < HALF; ++j) sum[j] = 0.f;
      for (int it = 0; it < wk.n_kb; it += S::FOLD, ++folds) {
        ok = __all_sync(0xffffffffu, mbar_wait_long(&acc_full[folds & 1], (folds >> 1) & 1, 50));
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const int done = it + S::FOLD;
        const bool small = S::SMALL && (done >= wk.n_kb || done % (S::FOLD * kSmallFolds) == 0);
        auto fold = [&](uint32_t acc) {
#pragma unroll
          for (int c0 = 0; c0 < HALF; c0 += 16) {
            uint32_t v[16];
            tmem_ld16(acc + c0, v);
#pragma unroll
            for (int j = 0; j < 16; ++j) sum[c0 + j] += __uint_as_float(v[j]);
          }
        };
        if (small) {  // first: the MMAs of the next item wait for it, while they have another accumulator for the leading terms
          fold(lanes + 2 * BN);
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
          __syncwarp();
          if (lane == 0) mbar_arrive(small_empty);
        }
        fold(lanes + (folds & 1) * BN);
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(&acc_empty[folds & 1]);
      }
      if (!ok) break;
      if constexpr (S::OUT == Out::transposed) {
        const bool add = p.accumulate != 0;
        if (p.write && m < (add ? p.M : p.m_pad)) {
          if (!row_in)  // (not the accumulator: 0 x NaN where B has one)
#pragma unroll
            for (int j = 0; j < HALF; ++j) sum[j] = 0.f;
          // (with what is there added) 8 lines at a time: where they go, what is there, then the stores (one by one every load would wait for the store
          // before it, as the compiler cannot tell that the lines differ)
          float* const dst = p.c + wk.z * p.slice_stride + m;
          const int32_t* const row_map = p.row_map;
          const int64_t ldc = p.ldc;
          const int left = p.N - nb;
          if (!row_map && !add) {
            float* at = dst + nb * ldc;
#pragma unroll
            for (int j = 0; j < HALF; ++j, at += ldc)
              if (j < left) *at = sum[j];
          } else {
#pragma unroll
            for (int j0 = 0; j0 < HALF; j0 += 8) {
              if (j0 >= left) break;
              int r[8];
#pragma unroll
              for (int j = 0; j < 8; ++j) r[j] = j0 + j >= left ? -1 : row_map ? __ldg(row_map + nb + j0 + j) : nb + j0 + j;
#if GCNSA_DBG
              if (row_map)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                  if (r[j] >= 0 && !dbg_in(&g_dbg_head, r[j], 0, p.map_rows, kDbgResultRow)) r[j] = -1;
#endif
              if (add) {
                float was[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) was[j] = r[j] >= 0 ? dst[r[j] * ldc] : 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) sum[j0 + j] += was[j];
              }
#pragma unroll
              for (int j = 0; j < 8; ++j)
                if (r[j] >= 0) dst[r[j] * ldc] = sum[j0 + j];
            }
          }
        }
      } else {
        const int cols = min(HALF, p.N - nb);  // classes of this half (may be below 1)
        const int c0 = args.ce.c0 + nb;
        if (args.ce.bias) {
          float* const xb = reinterpret_cast<float*>(smem + S::X_OFF) + (warp - S::FWARP0) * HALF;
#pragma unroll
          for (int j = 0; j < HALF; j += 32) xb[j + lane] = j + lane < cols ? __ldg(args.ce.bias + c0 + j + lane) : 0.f;
          __syncwarp();
#pragma unroll
          for (int j = 0; j < HALF; j += 4) {
            const float4 b = *reinterpret_cast<const float4*>(xb + j);
            sum[j] += b.x; sum[j + 1] += b.y; sum[j + 2] += b.z; sum[j + 3] += b.w;
          }
          __syncwarp();
        }
        if (cols < HALF) {
#pragma unroll
          for (int j = 0; j < HALF; ++j)
            if (j >= cols) sum[j] = -INFINITY;
        }
        label -= c0;  // relative to this half
        const bool here = row_in && label >= 0 && label < cols;
        const bool any_here = __any_sync(0xffffffffu, here);  // (few of the tiles have a label of a warp's rows)
        if constexpr (S::OUT == Out::grad) {
          const float scale = top.y * args.ce.inv_nt;
          float own = 0.f;
#pragma unroll
          for (int j = 0; j < HALF; ++j) sum[j] = exp2_fast((sum[j] - top.x) * kLog2e);
          if (any_here)
#pragma unroll
            for (int j = 0; j < HALF; ++j) own = j == label ? sum[j] : own;
#pragma unroll
          for (int j = 0; j < HALF; ++j) sum[j] *= scale;
          if (any_here) {  // the label's: p is rounded once, with the 1 taken off
            own = fmaf(own, top.y, -1.f) * args.ce.inv_nt;
#pragma unroll
            for (int j = 0; j < HALF; ++j) sum[j] = j == label ? own : sum[j];
          }
          if (row_in) {
            const int64_t ldg = args.ce.ldg;
            float* at = args.ce.gt + nb * ldg + m;
#pragma unroll
            for (int j = 0; j < HALF; ++j, at += ldg)
              if (j < cols) *at = sum[j];
          }
        } else {
          float mx = -INFINITY, zy = 0.f;
#pragma unroll
          for (int j = 0; j < HALF; ++j) mx = fmaxf(mx, sum[j]);
          if (any_here)
#pragma unroll
            for (int j = 0; j < HALF; ++j) zy = j == label ? sum[j] : zy;
          if constexpr (S::OUT == Out::stats) {
            if (here) args.ce.zy[m] = zy;
            // the run's maximum and sum go on; a maximum of -infinity has nothing to be subtracted from
            const float top = fmaxf(run_m, mx), base = top == -INFINITY ? 0.f : top;
            float s4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < HALF; ++j) s4[j & 3] += exp2_fast((sum[j] - base) * kLog2e);
            run_s = run_s * exp2_fast((run_m - base) * kLog2e) + ((s4[0] + s4[1]) + (s4[2] + s4[3]));
            run_m = top;
            const int next = w + 1;
            if (next >= w_end || next / p.tiles_n != w / p.tiles_n) {
              const int64_t slot = ((int64_t)(blockIdx.x + w / p.tiles_n) * 2 + half) * BM + quad * 32 + lane;
              args.ce.part_m[slot] = run_m;
              args.ce.part_s[slot] = run_s;
              run_m = -INFINITY;
              run_s = 0.f;
            }
          } else {
            // both halves of a row: maxima, then sums and the label's logit, through shared memory
            float* xm = reinterpret_cast<float*>(smem + S::X_OFF) + kFoldWarps * HALF;
            float* xs = xm + 2 * BM;
            const int r = quad * 32 + lane;
            xm[half * BM + r] = mx;
            ok = meet();
            if (!ok) break;
            const float top = fmaxf(xm[r], xm[BM + r]), base = top == -INFINITY ? 0.f : top;
            float s4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < HALF; ++j) {
              sum[j] = exp2_fast((sum[j] - base) * kLog2e);
              s4[j & 3] += sum[j];
            }
            float s = (s4[0] + s4[1]) + (s4[2] + s4[3]);
            xs[half * BM + r] = s;
            ok = meet();
            if (!ok) break;
            s = xs[r] + xs[BM + r];
            if (row_in) {
              const float inv = 1.f / s;
              // the half that has the label's logit adds the row's loss (a label outside all classes: no loss is a number)
              // (its distance from the maximum first: log(s) added to a large maximum would lose its digits)
              if (on && here) mine.loss += (base - zy) + logf(s);
              if (on && half == 0) {
                if (label + c0 < 0 || label + c0 >= p.N) mine.loss = NAN;
                ++mine.count;
              }
              if (args.ce.gt) {
                const int64_t ldg = args.ce.ldg;
                float* at = args.ce.gt + nb * ldg + m;
#pragma unroll
                for (int j = 0; j < HALF; ++j, at += ldg)
                  if (j < cols) *at = on ? (sum[j] * inv - (j == label ? 1.f : 0.f)) * args.ce.inv_nt : 0.f;
              }
            }
          }
        }
      }
    }
    if constexpr (S::OUT == Out::whole) {  // (a fixed order; written also where a wait ran out, as all of them are read)
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        mine.loss += __shfl_xor_sync(0xffffffffu, mine.loss, o);
        mine.count += __shfl_xor_sync(0xffffffffu, mine.count, o);
      }
      if (lane == 0) args.ce.losses[blockIdx.x * kFoldWarps + warp - S::FWARP0] = mine;
    }
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (warp == 1) {
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(S::TMEM_COLS) : "memory");
  }
}

// ---- host side ---------------------------------------------------------------------------------------------------------
// fp32 matrix with `inner` contiguous elements per line and `outer` lines, pitch ld; zero fill outside.  K-major: boxes of 32 k
// x `box_outer` lines, 128-byte swizzle; MN-major: boxes of 32 x 32 as they are.
inline bool term_map(CUtensorMap* map, const void* base, bool bytes, int64_t outer, int64_t inner, int64_t ld, int box_inner, int box_outer, bool swizzle) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[2] = {(cuuint64_t)inner, (cuuint64_t)outer};
  cuuint64_t strides[1] = {(cuuint64_t)ld * (bytes ? 1 : sizeof(float))};
  cuuint32_t box[2] = {(cuuint32_t)box_inner, (cuuint32_t)box_outer};
  cuuint32_t estr[2] = {1, 1};
  return fn(map, bytes ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2, (void*)base, dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE,
            CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Whether the compiled kernel has the registers that its warps divide (asked once).
template <class S>
cudaError_t registers_given() {
  static std::atomic<bool> held{false};
  if (held.load(std::memory_order_relaxed)) return cudaSuccess;
  cudaFuncAttributes f;
  const cudaError_t e = cudaFuncGetAttributes(&f, term_product<S>);
  if (e != cudaSuccess) return e;
  if (!registers_hold(f.numRegs, S::SHARES)) return cudaErrorInvalidKernelImage;
  held.store(true, std::memory_order_relaxed);
  return cudaSuccess;
}

template <class S>
cudaError_t run_terms(cudaStream_t s, const TermArgs& a, int grid) {
  cudaError_t e = registers_given<S>();
  if (e != cudaSuccess) return e;
  e = cudaFuncSetAttribute(term_product<S>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM_BYTES);
  if (e != cudaSuccess) return e;
  return launch(term_product<S>, grid, S::THREADS, S::SMEM_BYTES, s, a);
}

}  // namespace
}  // namespace gcnsa
