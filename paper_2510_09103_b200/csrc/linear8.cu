// The products of a linear layer in 8 bits:
//
//   forward      y[t, n]  = xs[t] ws[n] sum_k x8[t, k] w8[n, k]       whole numbers (tcgen05 kind::i8, sums in 32 bits), scaled at the end
//   input grad   dx[t, k] = sum_n dy[t, n] (ws[n] w8[n, k])           bf16 x codes
//   weight grad  dw[n, k] = sum_t dy[t, n] (xs[t] x8[t, k])           bf16 x codes
//
// The scale of a gradient's codes stands beside an index of K, so it cannot wait for the end as in the forward product: code x scale is
// made a bf16 number first (which rounds nothing where the scale is a power of two), by a launch of its own, and then multiplied
// (kind::f16, sums in fp32).  Where the scale is no power of two, that is a rounding per term, as large as the one of a bf16 result: the error's norm is 2.4e-3 of the
// result's, 1.7e-3 without (input gradient 8192 x 14336 x 4096).  A second bf16 number for what it leaves would double the product (700 us and more), so that only results
// that it would spoil have one: gradients of few columns, and in fp32.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <mutex>
#include <type_traits>

#include "codes.cuh"
#include "linear8_plan.h"
#include "tc_engine.cuh"
#include "tc_host.h"

namespace adapm {
namespace {

using namespace linear8;
using namespace tc;

constexpr int kOperandBytes = 16384;             // of one CTA and stage: 128 rows or columns of an operand, 128 bytes of K (or the reverse)
constexpr int kStageBytes = 2 * kOperandBytes;
constexpr int kSegLong = 4, kSegShort = 64;      // stages of 64 K between two sums in registers: gradients in fp32, long ones in bf16

// WIDE: boxes of results with rows of 128 bytes (see Outlet); only without LONG.
template <int OP, bool LONG, bool WIDE>
struct Shape {
  static constexpr bool kGrad = OP != FORWARD;
  static constexpr int kDrain = LONG ? 8 : 16;   // warps that drain, after four that issue
  static constexpr int kThreads = 32 * (4 + kDrain);
  static constexpr int kStages = WIDE ? 5 : 6, kBox = WIDE ? 4096 : 2048;
  static constexpr int kSmem = kStages * kStageBytes + kDrain * kBox + 1024;
};
// LONG: registers of the launch, and as the first four and the other eight warps divide them (the eight keep 128 sums each).
constexpr int kLongRegs = 168, kLongIssue = 88, kLongDrain = 208;
static_assert(4 * kLongIssue + 8 * kLongDrain <= 12 * kLongRegs, "a block has the registers that it was launched with");

struct Args {
  CUtensorMap a, b, o;           // b of a gradient: [planes][K][cols]; o: the result, or the parts of K [parts][rows][cols]
  Plan plan;
  const float *a_scale, *b_scale;      // forward: xs, ws
  void* out;
  int32_t* status;
  const int32_t* scale_words;    // a gradient in fp32: not all zero where B has three planes
  int64_t out_ld;
  int32_t pairs, out_f32, accumulate, seg;      // accumulate: not where K has parts
};

template <int OP, bool LONG, bool WIDE>
struct __align__(8) Shared {
  using S = Shape<OP, LONG, WIDE>;
  uint64_t full[S::kStages], empty[S::kStages], tfull[2], tempty[2], old_full[S::kDrain];
  uint32_t tmem_base;
  int abort;
};

// Instruction descriptor of kind::i8: signed 8-bit operands, K-major, 32-bit sums.
__device__ __forceinline__ uint32_t i8_idesc(int n, int m) {
  return 2u << 4 | 1u << 7 | 1u << 10 | (uint32_t)(n >> 3) << 17 | (uint32_t)(m >> 4) << 24;
}
template <bool PAIR>
__device__ __forceinline__ void mma_i8(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  if (PAIR)
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n}" ::"r"(d_tmem), "l"(a_desc),
                 "l"(b_desc), "r"(idesc), "r"(accumulate)
                 : "memory");
  else
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n}" ::"r"(d_tmem), "l"(a_desc),
                 "l"(b_desc), "r"(idesc), "r"(accumulate)
                 : "memory");
}

__device__ __forceinline__ void put4(void* p, const uint32_t* v) { *reinterpret_cast<uint4*>(p) = make_uint4(v[0], v[1], v[2], v[3]); }

// What a bf16 number leaves of x (nothing where it is not finite).
__device__ __forceinline__ float2 left_of_bf16(float2 x) {
  const uint32_t w = pack_bf16x2_rn(x.x, x.y);
  const float hi[2] = {__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)};
  return make_float2(fabsf(hi[0]) <= 3.402823466e38f ? x.x - hi[0] : 0.f, fabsf(hi[1]) <= 3.402823466e38f ? x.y - hi[1] : 0.f);
}

// x += 32 bf16 numbers of a row of which those below n (a multiple of 8) exist.
__device__ __forceinline__ void add_row32(const uint16_t* from, float* x, int n) {
#pragma unroll
  for (int h = 0; h < 4; ++h) {
    if (8 * h >= n) continue;
    const uint4 u = *reinterpret_cast<const uint4*>(from + 8 * h);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[8 * h + 2 * e] += __uint_as_float(w[e] << 16);
      x[8 * h + 2 * e + 1] += __uint_as_float(w[e] & 0xffff0000u);
    }
  }
}

// A warp's way out: 32 rows of 64 bytes (16 columns in fp32, 32 in bf16), or (WIDE) of 128, are put into its box in shared memory, with the
// swizzle of as many, and stored as a whole by TMA, which leaves out what the result does not have.  (Every thread storing 32 bytes of a row of its
// own: weight gradient of 1 x 14336 x 4096 36 to 42 us, with a box 27.  Eight warps with boxes of 128 bytes for 128 columns each instead of
// sixteen for 64: forward 8192 x 14336 x 512 92 us for 76.  Two boxes of 64 bytes to a warp: no faster.)
// Wide boxes are for results in bf16 whose rows do not all start on 32 bytes: of a row of 64 bytes two sectors of three are then written in two
// pieces (input gradient 10166 x 144 x 12408 112 us, wide 87; 12416 columns without 67; forward 15697 x 7576 x 280 95 and 72).  Two warps that fill a
// wide box together, which leaves the sixth stage: 87 and 78, and 8 % more where rows start on 32 bytes.
// Results that are added to what is there: in fp32 by TMA; in bf16, where the sum is to be rounded once, the box holds what is there before its results
// come (`old`), for which it is wide.  (Every thread reading its row of it: weight gradient 512 x 14336 x 4096 111 us, 31 x 3576 x 4104 in fp32 48; now 74 and 29.)
template <bool LONG, bool WIDE>
struct Outlet {
  const CUtensorMap* map;
  uint8_t* box;
  int lane;
  bool add;                      // LONG, fp32
  // 32 columns from column `col` on of the rows from `row0` on, the lane's own in x; `part`: of K; `half`: whether they are the second 32 of 64.
  __device__ __forceinline__ void put32(float* x, int half, int col, int row0, int part, bool f32, int rows, int cols, bool old = false) {
    uint8_t* const line = box + lane * (WIDE ? 128 : 64);
    const int swap = WIDE ? lane & 7 : (lane >> 1) & 3, first = WIDE ? 4 * half : 0;      // (a wide box takes two turns)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if ((WIDE || !f32) && h == 1) break;
      if (first == 0 && !(WIDE && old)) {
        if (lane == 0) bulk_wait_group_read<0>();
        __syncwarp();
      }
      if (!WIDE && f32) {
#pragma unroll
        for (int c = 0; c < 4; ++c)
          *reinterpret_cast<float4*>(line + ((c ^ swap) * 16)) = make_float4(x[16 * h + 4 * c], x[16 * h + 4 * c + 1], x[16 * h + 4 * c + 2], x[16 * h + 4 * c + 3]);
      } else {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint8_t* const to = line + (((first + c) ^ swap) * 16);
          if (WIDE && old) {
            const uint4 o = *reinterpret_cast<const uint4*>(to);
            const uint32_t v[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              x[8 * c + 2 * e] += __uint_as_float(v[e] << 16);
              x[8 * c + 2 * e + 1] += __uint_as_float(v[e] & 0xffff0000u);
            }
          }
          uint32_t w[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) w[e] = pack_bf16x2_rn(x[8 * c + 2 * e], x[8 * c + 2 * e + 1]);
          put4(to, w);
        }
      }
      if (WIDE && half == 0) continue;
      fence_async_smem();
      __syncwarp();
      if (lane == 0) {
        const int from = col + 16 * h - 8 * first;
        if (row0 < rows && from < cols) {
          if (LONG && add) tma_add_box3(map, from, row0, part, box);
          else tma_store_box3(map, from, row0, part, box);
        }
        bulk_commit_group();
      }
    }
  }
};

// What a gradient's item does with 32 columns of its sums.
template <bool LONG, bool WIDE>
__device__ __forceinline__ void finish32(const Args& a, const Cut& t, Outlet<LONG, WIDE>& out, int half, int row0, int col, float* x, bool old) {
  const int row = row0 + out.lane;
  if (LONG && a.accumulate && !a.out_f32 && row < a.plan.rows) add_row32(static_cast<const uint16_t*>(a.out) + (int64_t)row * a.out_ld + col, x, a.plan.cols - col);
  __syncwarp();
  out.put32(x, half, col, row0, t.part, a.plan.parts > 1 || a.out_f32, a.plan.rows, a.plan.cols, old);
}

// An item's K in segments of even length: how many, and the stages of each but the last.
__device__ __forceinline__ void segments(int stages, int most, int& n, int& each) {
  n = (stages + most - 1) / most;
  each = (stages + n - 1) / n;
  n = (stages + each - 1) / each;
}

// Pairs of CTAs (cta_group::2), tiles of 256 x 256 (192, 128 columns).  Warp 0 loads A, warp 2 B, warp 1 issues the MMAs, the others drain the
// accumulators.
// What bounds it: the tensor cores, and with them the power cap.  8192 x 14336 x 4096: forward 285 to 350 us = 2.7 to 3.4 P operations/s (the
// library's 8-bit integer product alone 314 to 355), gradients with the decoding of their codes (16 to 30 us) 690 to 850 us = 1.1 to 1.4 PFLOP/s (the
// library's bf16 products alone 620 to 940 and 670 to 760).  With short K a tile's way out: forward 8192 x 14336 x 512 70 to 80 us, in fp32 97 to 119, is 2.9 us for a round
// of tiles whose products take 1.1.  That is not memory's doing, since dequant8_kernel writes the same 235 MB, and reads 117 besides, in 54 us; which part of the way is
// to blame is open.  With few tiles the rounds of them, and a start and an end that nothing runs beside.
// Not kept: codes made bf16 numbers by warps of this kernel on their way into shared memory, which the CTA of rank 1 has to tell the one of rank
// 0: an arrival that releases at cluster scope takes 1000 to 1800 cycles, twice to three times what a stage does (8192 x 14336 x 4096 1230 us, by a
// warp that does nothing else 1660, with a relaxed one, which does not order the codes, 980).
// LONG: K in segments that the epilogue adds up in registers, because the tensor cores cut every partial sum off toward zero (a K step of 16 leaves
// an accumulator up to 2^-23 of itself too small).  For gradients in fp32, and for sums above 16384 terms.
template <int OP, bool LONG, bool WIDE>
__global__ void __launch_bounds__(Shape<OP, LONG, WIDE>::kThreads, 1) linear8_kernel(const __grid_constant__ Args a) {
  using S = Shape<OP, LONG, WIDE>;
  extern __shared__ uint8_t dyn_smem[];
  __shared__ Shared<OP, LONG, WIDE> sh;
  let_next_kernel_start();
  const uint32_t rank = cluster_rank();
  uint8_t* const ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(dyn_smem) + 1023) & ~(uintptr_t)1023);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, pair = (int)(blockIdx.x >> 1);
  volatile int* const abort = &sh.abort;
  int32_t* const status = a.status + pair;

  if (threadIdx.x == 0) {
    for (int i = 0; i < S::kStages; ++i) {
      mbar_init(&sh.full[i], 2);                    // A and B, those of rank 0 for both CTAs
      mbar_init(&sh.empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) { mbar_init(&sh.tfull[i], 1); mbar_init(&sh.tempty[i], 2 * S::kDrain); }
    for (int i = 0; i < S::kDrain; ++i) mbar_init(&sh.old_full[i], 1);
    sh.abort = 0;
    mbar_fence_init();
  }
  wait_for_what_is_before();
  if (warp == 1) {
    tmem_alloc<true>(&sh.tmem_base, 512);
    tmem_relinquish<true>();
  }
  tc_fence_before();
  if (rank == 0 && threadIdx.x == 0) *status = 0;      // (the cluster barrier orders it before what either CTA adds)
  if (blockIdx.x == 0)
    for (int i = a.pairs + (int)threadIdx.x; i < kMostWords; i += S::kThreads) a.status[i] = 0;      // words of no pair
  int planes = 1;
  if (LONG) planes = __syncthreads_or(a.scale_words && threadIdx.x < kScaleWords ? a.scale_words[threadIdx.x] : 0) ? kPlanesF32 : 1;
  else __syncthreads();
  cluster_sync();
  tc_fence_after();
  const uint32_t tmem_base = sh.tmem_base;
  Cut t;

  if (warp < 4) {
    if (LONG) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kLongIssue));
    if (warp == 0 || warp == 2) {
      // ------------------------------------------------------------------ producers (all lanes run, one issues)
      const bool leader = elect_one(), is_a = warp == 0;
      const uint32_t pair_full = uniform(shared_of(sh.full, 0));
      const bool along_y = is_a ? OP == WEIGHT_GRAD : S::kGrad;      // rows are K: boxes of 64 columns
      constexpr int kStep = OP == FORWARD ? 128 : 64;
      int stage = 0;
      uint32_t phase = 0, issued = 0;
      bool ok = true;
      for (int i = pair; ok && a.plan.item(i, t); i += a.pairs) {
        const CUtensorMap* const map = is_a ? &a.a : &a.b;
        const int mine = uniform(is_a ? t.m0 + (int)rank * 128 : t.n0 + (int)rank * (t.bn / 2));
        const int count = uniform(t.count);
        const bool two = is_a || t.bn > 128;
        const uint32_t bytes = along_y && !two ? kOperandBytes : 2 * kOperandBytes;
        const int first = uniform(t.k0) * kStep;
        int k = first, plane = 0;
        for (int left = count * planes; left > 0; --left) {
          if (!mbar_wait_warp<WAIT_PAIR>(&sh.empty[stage], phase ^ 1u, abort, status, ST_WAIT_EMPTY, kWaitSpinDefault)) { ok = false; break; }
          uint8_t* const dst = ring + stage * kStageBytes + (is_a ? 0 : kOperandBytes);
          if (leader) {
            if (rank == 0) mbar_arrive_expect_tx(&sh.full[stage], bytes);
            const uint32_t bar = pair_full + 8u * (uint32_t)stage;
            if (S::kGrad && !is_a) {
              tma_load_box3_pair(dst, map, mine, k, plane, bar);
              if (two) tma_load_box3_pair(dst + kOperandBytes / 2, map, mine + 64, k, plane, bar);
            } else if (along_y) {
              tma_load_box_pair(dst, map, mine, k, bar);
              tma_load_box_pair(dst + kOperandBytes / 2, map, mine + 64, k, bar);
            } else {
              tma_load_box_pair(dst, map, k, mine, bar);
            }
          }
          __syncwarp();
          ++issued;
          if (++stage == S::kStages) { stage = 0; phase ^= 1u; }
          k += kStep;
          if (LONG && k == first + count * kStep) { k = first; ++plane; }          // the next plane of B, the same A again
        }
      }
      if (!ok) drain_ring<true>(sh.full, stage, phase, issued, S::kStages, rank);
    } else if (warp == 1 && rank == 0) {
      // ------------------------------------------------------------------ MMA issuer (all lanes run, one issues)
      const bool leader = elect_one();
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      const uint32_t ring0 = uniform(smem_u32(ring)), d0 = uniform(tmem_base), dhi = desc_hi();
      // per K step: 32 bytes inside a K-major row, 16 rows of 128 bytes of an MN-major box (in 16-byte units)
      constexpr bool kAmn = OP == WEIGHT_GRAD, kBmn = S::kGrad;
      constexpr uint32_t kAstep = kAmn ? 128u : 2u, kBstep = kBmn ? 128u : 2u;
      uint32_t run = 0;
      for (int i = pair; ok && a.plan.item(i, t); i += a.pairs) {
        const uint32_t idesc = uniform(S::kGrad ? make_idesc(t.bn, kAmn, kBmn, false, 256) : i8_idesc(t.bn, 256));
        int left = uniform(t.count) * planes, n_seg = 1, each = left;
        if (LONG) segments(left, a.seg, n_seg, each);
        for (; left > 0 && ok; left -= each, ++run) {
          const int acc = (int)(run & 1);
          if (!mbar_wait_warp<WAIT_PAIR_TC>(&sh.tempty[acc], ((run >> 1) & 1u) ^ 1u, abort, status, ST_WAIT_TMEM_EMPTY, kWaitSpinDefault)) { ok = false; break; }
          tc_fence_after();
          const uint32_t d = d0 + (uint32_t)(acc * kTile);
          uint32_t accumulate = 0;
          for (int n = min(each, left); n > 0; --n) {
            if (!mbar_wait_warp<WAIT_PAIR>(&sh.full[stage], phase, abort, status, ST_WAIT_FULL, kWaitSpinDefault)) { ok = false; break; }
            tc_fence_after();
            const uint32_t slot = ring0 + (uint32_t)(stage * kStageBytes);
            const uint32_t alo = desc_lo(slot, kAmn ? kOperandBytes / 2 : 16u), blo = desc_lo(slot + kOperandBytes, kBmn ? kOperandBytes / 2 : 16u);
            if (leader) {
#pragma unroll
              for (int q = 0; q < 4; ++q) {
                const uint64_t da = desc_join(alo + q * kAstep, dhi), db = desc_join(blo + q * kBstep, dhi);
                if (S::kGrad) mma_bf16<true>(d, da, db, idesc, q ? 1u : accumulate);
                else mma_i8<true>(d, da, db, idesc, q ? 1u : accumulate);
              }
              mma_commit<true>(&sh.empty[stage]);
            }
            __syncwarp();
            accumulate = 1;
            if (++stage == S::kStages) { stage = 0; phase ^= 1u; }
          }
          if (ok && leader) mma_commit<true>(&sh.tfull[acc]);
          __syncwarp();
        }
      }
    }
  } else {
    if (LONG) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kLongDrain));
    // ------------------------------------------------------------------ epilogue: a thread has one row of the tile and, by its
    // group of four warps, 64 (LONG: 128) of the columns
    const int q = 32 * (warp & 3) + lane, grp = (warp - 4) >> 2;
    const uint32_t lane_addr = (uint32_t)(32 * (warp & 3)) << 16;
    Outlet<LONG, WIDE> out = {&a.o, ring + S::kStages * kStageBytes + (warp - 4) * S::kBox, lane, LONG && a.accumulate && a.out_f32};
    // what is there already of this warp's box of an item: asked for as soon as the box is free of the item before
    const bool old = OP == WEIGHT_GRAD && WIDE && a.accumulate;
    uint64_t* const old_bar = &sh.old_full[warp - 4];
    uint32_t old_phase = 0;
    bool asked = false;
    auto ask = [&](int i) {
      Cut n;
      asked = old && a.plan.item(i, n) && 64 * grp < n.bn;
      if (asked && lane == 0) {
        bulk_wait_group_read<0>();
        mbar_arrive_expect_tx(old_bar, S::kBox);
        tma_load_box3(out.box, &a.o, n.n0 + 64 * grp, n.m0 + (int)rank * 128 + 32 * (warp & 3), 0, old_bar);
      }
      __syncwarp();
    };
    if (WIDE) ask(pair);
    uint32_t run = 0;
    bool ok = true;
    auto wait_full = [&](int acc) {
      if (lane == 0) ok = mbar_wait<WAIT_PAIR_TC>(&sh.tfull[acc], (run >> 1) & 1u, abort, status, ST_WAIT_TMEM_FULL, kWaitSpinDefault);
      ok = __shfl_sync(0xffffffffu, ok, 0);
      tc_fence_after();
    };
    auto release = [&](int acc) {
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_relaxed_at(shared_of(&sh.tempty[acc], 0));
    };
    for (int i = pair; ok && a.plan.item(i, t); i += a.pairs) {
      const int row = t.m0 + (int)rank * 128 + q, col0 = t.n0 + grp * (LONG ? 128 : 64);
      if (LONG) {
        const int mine = grp ? t.bn - 128 : min(t.bn, 128);
        float v[128];
        int n_seg, each;
        segments(t.count * planes, a.seg, n_seg, each);
#pragma unroll 1
        for (int s = 0; s < n_seg; ++s, ++run) {
          const int acc = (int)(run & 1);
          wait_full(acc);
          if (!ok) break;
          const uint32_t at = tmem_base + lane_addr + (uint32_t)(acc * kTile + grp * 128);
          if (s == 0) {
#pragma unroll
            for (int c = 0; c < 128; c += 16)
              if (c < mine) tmem_ld16(at + c, v + c);
            tmem_ld_wait();
          } else {
#pragma unroll
            for (int c = 0; c < 128; c += 32) {
              if (c < mine) {
                float x[32];
                tmem_ld16(at + c, x);
                tmem_ld16(at + c + 16, x + 16);
                tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 32; ++e) v[c + e] += x[e];
              }
            }
          }
          release(acc);
        }
        if (!ok) break;
#pragma unroll
        for (int c = 0; c < 128; c += 32)
          if (c < mine) finish32(a, t, out, c / 32 % 2, row - lane, col0 + c, v + c, false);
      } else {
        const int acc = (int)(run & 1);
        const float xs = OP == FORWARD && row < a.plan.rows ? a.a_scale[row] : 0.f;
        // (the columns' scales are asked for sixteen columns ahead: forward 2048 x 2736 x 1024 13.3 -> 10.3 us; 32 ahead, which does not fit the registers, 10.6)
        float4 ws[4];
        auto scales_of = [&](int col) {
#pragma unroll
          for (int e = 0; e < 4; ++e) ws[e] = col + 4 * e < a.plan.cols ? __ldg(reinterpret_cast<const float4*>(a.b_scale + col + 4 * e)) : make_float4(0.f, 0.f, 0.f, 0.f);
        };
        if (OP == FORWARD) scales_of(col0);
        wait_full(acc);
        if (!ok) break;
        const uint32_t at = tmem_base + lane_addr + (uint32_t)(acc * kTile + grp * 64);
        if (64 * grp < t.bn) {                         // (tiles are multiples of 64 wide)
          if (WIDE && old) {
            ok = mbar_wait_warp(old_bar, old_phase, abort, status, ST_WAIT_FULL, kWaitSpinDefault);
            if (!ok) break;
            old_phase ^= 1u;
            asked = false;
          }
#pragma unroll
          for (int c = 0; c < 64; c += 32) {
            __syncwarp();
            float v[32];
            tmem_ld16(at + c, v);
            tmem_ld16(at + c + 16, v + 16);
            tmem_ld_wait();
            if (c == 32) release(acc);
            if (OP == FORWARD) {
#pragma unroll
              for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  float* const to = v + 16 * h + 4 * e;
                  to[0] = (float)__float_as_int(to[0]) * xs * ws[e].x;
                  to[1] = (float)__float_as_int(to[1]) * xs * ws[e].y;
                  to[2] = (float)__float_as_int(to[2]) * xs * ws[e].z;
                  to[3] = (float)__float_as_int(to[3]) * xs * ws[e].w;
                }
                if (c + 16 * h < 48) scales_of(col0 + c + 16 * h + 16);
              }
              out.put32(v, c / 32, col0 + c, row - lane, 0, a.out_f32, a.plan.rows, a.plan.cols);
            } else {
              finish32(a, t, out, c / 32, row - lane, col0 + c, v, old);
            }
          }
        } else {
          release(acc);
        }
        if (WIDE) ask(i + a.pairs);
        ++run;
      }
    }
    if (WIDE && asked)                                 // (a wait ran out: the box is not left before what was asked for has come)
      for (uint32_t spin = 0; spin < kDrainSpins && !mbar_try_wait<WAIT_CTA>(old_bar, old_phase); ++spin) __nanosleep(64);
    if (lane == 0) bulk_wait_group<0>();
    __syncwarp();
  }

  tc_fence_before();
  __syncthreads();
  cluster_sync();      // neither CTA leaves while the other may still reach into it
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc<true>(tmem_base, 512);
  }
}

// ---- codes to bf16 numbers for a gradient in fp32 -------------------------------------------------------------------
// One bf16 number has 8 of the up to 32 bits of code x scale: enough where the scale is a power of two, and about as good as a bf16
// gradient's own rounding where not; an fp32 gradient then takes three, which have the 24 bits of the product in fp32.

// Up to so many scales every CTA of linear8_planes_kernel looks through by itself, which takes less time than a launch.
constexpr int64_t kFewScales = 4096;

// words[i] != 0: some scale that CTA i has seen is no power of two.
__global__ void __launch_bounds__(256) linear8_scales_kernel(const float* scales, int64_t n, int32_t* words) {
  wait_for_previous_kernel();
  int others = 0;
#pragma unroll 8
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) others |= __float_as_int(scales[i]) & 0x7fffff;
  others = __syncthreads_or(others);
  if (threadIdx.x == 0) words[blockIdx.x] = others;
  if (blockIdx.x == 0)
    for (int i = (int)(gridDim.x + threadIdx.x); i < kScaleWords; i += 256) words[i] = 0;      // of no CTA
}

struct PlanesArgs {
  const uint8_t* codes;
  const float* scales;
  int32_t* words;
  uint16_t* out;                 // [planes][rows][ld]
  int64_t codes_ld, ld, rows, scan;  // scan: scales to look through, 0: the words say it
  int32_t cols, groups;          // cols: a multiple of eight; scales per row
};

template <bool E4M3>
__global__ void __launch_bounds__(256) linear8_planes_kernel(const PlanesArgs a) {
  wait_for_previous_kernel();
  static_assert(kScaleWords == 256, "a thread has a word");
  int others = a.scan ? 0 : a.words[threadIdx.x];
#pragma unroll 16
  for (int64_t i = threadIdx.x; i < a.scan; i += 256) others |= __float_as_int(a.scales[i]) & 0x7fffff;
  others = __syncthreads_or(others);
  if (a.scan && blockIdx.x == 0) a.words[threadIdx.x] = others;
  const int planes = others ? kPlanesF32 : 1, eights = a.cols / 8;
  const int64_t chunks = a.rows * eights, plane = a.rows * a.ld;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < chunks; i += (int64_t)gridDim.x * 256) {
    const int64_t row = chunks <= UINT32_MAX ? (int64_t)((uint32_t)i / (uint32_t)eights) : i / eights;
    const int c = 8 * (int)(i - row * eights);
    const uint2 q = *reinterpret_cast<const uint2*>(a.codes + row * a.codes_ld + c);
    const float s = a.scales[a.groups > 1 ? row * a.groups + c / 128 : row];
    float x[8];
    unpack4<E4M3>(q.x, x);
    unpack4<E4M3>(q.y, x + 4);
    float2 v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = make_float2(x[2 * e] * s, x[2 * e + 1] * s);
    for (int p = 0; p < planes; ++p) {
      uint32_t w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        w[e] = pack_bf16x2_rn(v[e].x, v[e].y);
        v[e] = left_of_bf16(v[e]);
      }
      put4(a.out + p * plane + row * a.ld + c, w);
    }
  }
}

// ---- a gradient whose K was cut: its parts, put together ------------------------------------------------------------

struct SumArgs {
  const float* part;
  void* out;
  int64_t out_ld, places, part_elems;      // fours of columns; elements of a part
  int32_t fours, parts, f32, accumulate;
};

__global__ void __launch_bounds__(256) linear8_sum_kernel(const SumArgs a) {
  wait_for_previous_kernel();
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < a.places; i += (int64_t)gridDim.x * 256) {
    const int64_t row = a.places <= UINT32_MAX ? (int64_t)((uint32_t)i / (uint32_t)a.fours) : i / a.fours, c = (i - row * a.fours) * 4;
    const float* p = a.part + i * 4;
    float4 x = __ldcg(reinterpret_cast<const float4*>(p));
#pragma unroll 8
    for (int u = 1; u < a.parts; ++u) {
      const float4 v = __ldcg(reinterpret_cast<const float4*>(p + u * a.part_elems));
      x.x += v.x; x.y += v.y; x.z += v.z; x.w += v.w;
    }
    const int64_t at = row * a.out_ld + c;
    if (a.f32) {
      float4* const to = reinterpret_cast<float4*>(static_cast<float*>(a.out) + at);
      if (a.accumulate) { const float4 o = *to; x.x += o.x; x.y += o.y; x.z += o.z; x.w += o.w; }
      *to = x;
    } else {
      uint2* const to = reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + at);
      if (a.accumulate) {
        const uint2 o = *to;
        x.x += __uint_as_float(o.x << 16); x.y += __uint_as_float(o.x & 0xffff0000u);
        x.z += __uint_as_float(o.y << 16); x.w += __uint_as_float(o.y & 0xffff0000u);
      }
      *to = make_uint2(pack_bf16x2_rn(x.x, x.y), pack_bf16x2_rn(x.z, x.w));
    }
  }
}

// ---- strips: few columns, or few tiles -----------------------------------------------------------------------------------
// A CTA has 128 features of the 8-bit operand (the rows of an MMA, so that few tokens cost few products) and up to 256 columns of the
// other one; the CTAs of a cluster take parts of K, whose sums they add up through each other's shared memory, in a fixed order.
//   forward       output features of w8 x tokens of x8         both read as they lie (kind::i8)
//   input grad    input features of w8 x tokens of dy          codes made bf16 numbers on their way: sixteen warps, four to a stage,
//   weight grad   input features of x8 x output features of dy     write them into shared memory, times their scales
// The result lies across: out[column][feature].
// FOLD (up to 16 columns, or a gradient in fp32): code x scale rounded to bf16 would be a rounding per term that few terms do not average out,
// or too coarse.  The scale is a number per index of K, so it may as well go into the other operand, as far as its size is not in the way: scale = 2^e m, 1/2 < m <= 1,
// the codes are bf16 numbers times 2^e, which rounds nothing, and dy x m is carried as two bf16 numbers (three for fp32), next to one another as columns of
// one product, whose sums are added at the end.  Where all scales of the CTA's part of K are powers of two, m is 1 and dy goes in as it is; where all lie between
// 2^-30 and 1, 2^e stays with m (1 x 14336 x 4096 34 us; apart 41), which beyond would leave bf16's range where code x scale does not.  K is taken in segments
// that are added up in registers, as above.

struct StripArgs {
  CUtensorMap codes, other;
  StripPlan plan;
  const float *xs, *ws;          // forward: of a column, of a feature
  const float* scale;            // gradients: of a row of K [K][scale_groups]
  void* out;
  int32_t* status;
  int64_t out_ld;
  int32_t columns, features, k, scale_groups, f32, accumulate, e4m3;
};

template <int OP, bool FOLD>
struct StripShape {
  static constexpr bool kGrad = OP != FORWARD;
  static constexpr int kThreads = kGrad ? 768 : 256;       // warp 0 loads, 1 issues the MMAs, 4 to 7 drain, 8 to 23 make numbers of codes
  static constexpr int kAccs = FOLD ? 2 : 1;
};
// FOLD: registers of the launch, and as the four warps that issue, the four that drain and the sixteen that decode divide them.
constexpr int kStripRegs = 80, kStripIssue = 72, kStripDrain = 152, kStripDecode = 64;
static_assert(4 * kStripIssue + 4 * kStripDrain + 16 * kStripDecode <= 24 * kStripRegs, "a block has the registers that it was launched with");

struct __align__(8) StripShared {
  uint64_t full[kStripRing], empty[kStripRing], raw_full[kStripRing], raw_empty[kStripRing], tfull[2], tempty[2];
  uint32_t tmem_base;
  int abort;
};

__device__ __forceinline__ int4 load_shared4_at(uint32_t at) {
  int4 v;
  asm volatile("ld.shared::cluster.v4.s32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}

// Eight codes of one row, times its scale, as bf16 numbers: 16 bytes.
template <bool E4M3>
__device__ __forceinline__ void decode8(uint32_t c0, uint32_t c1, float s, uint32_t* w) {
  float x[8];
  unpack4<E4M3>(c0, x);
  unpack4<E4M3>(c1, x + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 t = mul2(make_float2(x[2 * i], x[2 * i + 1]), make_float2(s, s));
    w[i] = pack_bf16x2_rn(t.x, t.y);
  }
}
// ... without a scale, which rounds nothing.  int8: the lower seven bits become those of a bf16 number from 128 on, the upper one says whether 128
// or 256 is taken off again.
template <bool E4M3>
__device__ __forceinline__ void decode8(uint32_t c0, uint32_t c1, uint32_t* w) {
  if (E4M3) {
    float x[8];
    unpack4<E4M3>(c0, x);
    unpack4<E4M3>(c1, x + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = pack_bf16x2_rn(x[2 * i], x[2 * i + 1]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t two = __byte_perm(i < 2 ? c0 : c1, 0u, i & 1 ? 0x4342u : 0x4140u);          // in the lower halves of 16 bits each
      asm("add.rn.bf16x2 %0, %1, %2;" : "=r"(w[i]) : "r"((two & 0x007f007fu) | 0x43004300u), "r"((two & 0x00800080u) | 0xc300c300u));
    }
  }
}

// scale = power x m: the power of two as two bf16 numbers of a register, with the scale's sign, and m from above 1/2 to 1 (1 to 2 for scales above 2^127,
// whose next power has no number).  A NaN is one in the power; an infinity, or zero, is a power.
struct Split { uint32_t power; float m; };
__device__ __forceinline__ Split split_scale(float s) {
  const uint32_t bits = __float_as_uint(s), size = bits & 0x7fffffffu, fraction = size & 0x7fffffu;
  const int e = (int)(size >> 23), up = min(254, e + (fraction ? 1 : 0));
  const uint32_t power = size >= 0x7f800000u ? size >> 16 | (fraction ? 0x40u : 0u) : (uint32_t)up << 7;
  Split r;
  r.power = (power | (bits >> 16 & 0x8000u)) * 0x10001u;
  // (the reciprocal of 2^127 is subnormal)
  r.m = fraction == 0 || e == 255 ? 1.f : __uint_as_float(size) * __uint_as_float(up < 254 ? (uint32_t)(254 - up) << 23 : 0x400000u);
  return r;
}
__device__ __forceinline__ uint32_t times_bf16x2(uint32_t x, uint32_t y) {
  uint32_t r;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(y));
  return r;
}

// A CTA puts its share of the features together, a thread four of them, for every few columns: eight loads of four sums on their way
// at a time.
template <int OP, bool FOLD, int SPLIT>
__device__ __forceinline__ void put_together(const StripArgs& a, const uint8_t* sums, int rank, int f0, int c0) {
  constexpr int kShare = 128 / SPLIT, kFours = kShare / 4, kStep = StripShape<OP, FOLD>::kThreads / kFours, kAtOnce = 8 / SPLIT;
  const int mine = rank * kShare + 4 * ((int)threadIdx.x % kFours), f = f0 + mine, columns = min(a.plan.width, a.columns - c0);
  if (f >= a.features) return;
  float4 ws = make_float4(1.f, 1.f, 1.f, 1.f);
  if (OP == FORWARD) ws = *reinterpret_cast<const float4*>(a.ws + f);
  uint32_t from[SPLIT];
#pragma unroll
  for (int r = 0; r < SPLIT; ++r) from[r] = SPLIT > 1 ? shared_of(sums + 4 * mine, (uint32_t)r) : smem_u32(sums + 4 * mine);
  for (int c = (int)threadIdx.x / kFours; c < columns; c += kAtOnce * kStep) {
    int4 v[kAtOnce][SPLIT];
    float xs[kAtOnce];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      const int at = min(c + u * kStep, columns - 1);
      xs[u] = OP == FORWARD ? a.xs[c0 + at] : 1.f;
#pragma unroll
      for (int r = 0; r < SPLIT; ++r) v[u][r] = load_shared4_at(from[r] + 512u * (uint32_t)at);
    }
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      if (c + u * kStep >= columns) continue;
      const int64_t to = (int64_t)(c0 + c + u * kStep) * a.out_ld + f;
      float y[4];
      if (OP == FORWARD) {
        int4 sum = v[u][0];
#pragma unroll
        for (int r = 1; r < SPLIT; ++r) { sum.x += v[u][r].x; sum.y += v[u][r].y; sum.z += v[u][r].z; sum.w += v[u][r].w; }
        y[0] = (float)sum.x * xs[u] * ws.x; y[1] = (float)sum.y * xs[u] * ws.y; y[2] = (float)sum.z * xs[u] * ws.z; y[3] = (float)sum.w * xs[u] * ws.w;
      } else {
        y[0] = __int_as_float(v[u][0].x); y[1] = __int_as_float(v[u][0].y); y[2] = __int_as_float(v[u][0].z); y[3] = __int_as_float(v[u][0].w);
#pragma unroll
        for (int r = 1; r < SPLIT; ++r) {
          y[0] += __int_as_float(v[u][r].x); y[1] += __int_as_float(v[u][r].y); y[2] += __int_as_float(v[u][r].z); y[3] += __int_as_float(v[u][r].w);
        }
        if (a.f32 && a.accumulate) {
          const float4 o = *reinterpret_cast<const float4*>(static_cast<const float*>(a.out) + to);
          y[0] += o.x; y[1] += o.y; y[2] += o.z; y[3] += o.w;
        } else if (a.accumulate) {
          const uint2 o = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(a.out) + to);
          y[0] += __uint_as_float(o.x << 16); y[1] += __uint_as_float(o.x & 0xffff0000u);
          y[2] += __uint_as_float(o.y << 16); y[3] += __uint_as_float(o.y & 0xffff0000u);
        }
      }
      if (a.f32) *reinterpret_cast<float4*>(static_cast<float*>(a.out) + to) = make_float4(y[0], y[1], y[2], y[3]);
      else *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + to) = make_uint2(pack_bf16x2_rn(y[0], y[1]), pack_bf16x2_rn(y[2], y[3]));
    }
  }
}

template <int OP, bool FOLD>
__global__ void __launch_bounds__(StripShape<OP, FOLD>::kThreads, 1) linear8_strip_kernel(const __grid_constant__ StripArgs a) {
  using S = StripShape<OP, FOLD>;
  constexpr int kStep = S::kGrad ? 64 : 128;                       // K of a stage
  extern __shared__ uint8_t dyn_smem[];
  __shared__ StripShared sh;
  let_next_kernel_start();
  const StripPlan& p = a.plan;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, split = p.split, rank = split > 1 ? (int)cluster_rank() : 0;
  const int tile = (int)blockIdx.x / split, c_tile = tile / p.f_tiles, f0 = (tile - c_tile * p.f_tiles) * 128, c0 = c_tile * p.width;
  const int k0 = p.first(rank), count = p.first(rank + 1) - k0, bytes = p.stage_bytes;
  uint8_t* const ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(dyn_smem) + 1023) & ~(uintptr_t)1023);
  uint8_t* const raw = ring + p.ring * bytes;
  volatile int* const abort = &sh.abort;
  int32_t* const status = a.status + blockIdx.x;
  const int widest = p.width * p.planes;
  const uint32_t acc_cols = widest <= 32 ? 32 : widest <= 64 ? 64 : widest <= 128 ? 128 : 256, tmem_cols = S::kAccs * acc_cols;

  if (threadIdx.x == 0) {
    for (int i = 0; i < p.ring; ++i) { mbar_init(&sh.full[i], (FOLD ? 0 : 1) + (S::kGrad ? 4 : 0)); mbar_init(&sh.empty[i], 1); }
    if (S::kGrad)
      for (int i = 0; i < p.raw; ++i) { mbar_init(&sh.raw_full[i], 1); mbar_init(&sh.raw_empty[i], 4); }
    for (int i = 0; i < S::kAccs; ++i) { mbar_init(&sh.tfull[i], 1); mbar_init(&sh.tempty[i], 4); }
    sh.abort = 0;
    mbar_fence_init();
  }
  wait_for_what_is_before();
  if (warp == 1) {
    tmem_alloc(&sh.tmem_base, tmem_cols);
    tmem_relinquish();
  }
  tc_fence_before();
  if (threadIdx.x == 0) *status = 0;
  if (blockIdx.x == 0)
    for (int i = (int)gridDim.x + (int)threadIdx.x; i < kMostWords; i += S::kThreads) a.status[i] = 0;      // words of no CTA
  int planes = 1;
  bool apart = FOLD;
  if (FOLD) {                          // whether all scales of this CTA's part of K are powers of two, or between 2^-30 and 1
    int others = 0, far = 0;
    const float* const scale = a.scale + (a.scale_groups > 1 ? f0 / 128 : 0);
    for (int k = 64 * k0 + (int)threadIdx.x; k < min(a.k, 64 * (k0 + count)); k += S::kThreads) {
      const float s = scale[(int64_t)k * a.scale_groups];
      others |= __float_as_int(s) & 0x7fffff;
      far |= !(fabsf(s) >= 9.31322575e-10f && fabsf(s) <= 1.f);
    }
    planes = __syncthreads_or(others) ? p.planes : 1;
    if (planes > 1) apart = __syncthreads_or(far);
  } else {
    __syncthreads();
  }
  tc_fence_after();
  const uint32_t tmem_base = sh.tmem_base;
  if (warp < 4) {
    if (FOLD) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kStripIssue));
    if (warp == 0 && !FOLD) {
      // ------------------------------------------------------------------ the operands (forward), the other operand (gradients)
      const bool leader = elect_one();
      int stage = 0;
      uint32_t phase = 0, issued = 0;
      bool ok = true;
      for (int i = 0; i < count; ++i) {
        if (!mbar_wait_warp(&sh.empty[stage], phase ^ 1u, abort, status, ST_WAIT_EMPTY, kWaitSpinDefault)) { ok = false; break; }
        if (leader) {
          uint8_t* const dst = ring + stage * bytes;
          uint64_t* const bar = &sh.full[stage];
          const int k = (k0 + i) * kStep;
          mbar_arrive_expect_tx(bar, (uint32_t)(S::kGrad ? bytes - 16384 : bytes));
          if (OP == FORWARD) tma_load_box(dst, &a.codes, k, f0, bar);
          if (OP == WEIGHT_GRAD) {
            for (int c = 0; c < p.width; c += 64) tma_load_box(dst + 16384 + c * 128, &a.other, c0 + c, k, bar);
          } else {
            tma_load_box(dst + 16384, &a.other, k, c0, bar);
          }
        }
        __syncwarp();
        ++issued;
        if (++stage == p.ring) { stage = 0; phase ^= 1u; }
      }
      if (!ok) drain_ring<false>(sh.full, stage, phase, issued, p.ring, 0);
    } else if (S::kGrad && warp == 2) {
      // ------------------------------------------------------------------ codes, and what scales go into, as they lie
      const bool leader = elect_one();
      int stage = 0;
      uint32_t phase = 0, issued = 0;
      bool ok = true;
      for (int i = 0; i < count; ++i) {
        if (!mbar_wait_warp(&sh.raw_empty[stage], phase ^ 1u, abort, status, ST_WAIT_EMPTY, kWaitSpinDefault)) { ok = false; break; }
        if (leader) {
          uint8_t* const dst = raw + stage * p.raw_bytes;
          uint64_t* const bar = &sh.raw_full[stage];
          const int k = (k0 + i) * kStep;
          mbar_arrive_expect_tx(bar, (uint32_t)p.raw_bytes);
          tma_load_box(dst, &a.codes, f0, k, bar);
          if (FOLD) {
            if (OP == WEIGHT_GRAD) tma_load_box(dst + kStripRawBytes, &a.other, c0, k, bar);
            else tma_load_box(dst + kStripRawBytes, &a.other, k, c0, bar);
          }
        }
        __syncwarp();
        ++issued;
        if (++stage == p.raw) { stage = 0; phase ^= 1u; }
      }
      if (!ok) drain_ring<false>(sh.raw_full, stage, phase, issued, p.raw, 0);
    } else if (warp == 1) {
      // ------------------------------------------------------------------ MMA issuer (all lanes run, one issues)
      const bool leader = elect_one();
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      constexpr bool kAmn = S::kGrad, kBmn = OP == WEIGHT_GRAD;
      constexpr uint32_t kAstep = kAmn ? 128u : 2u, kBstep = kBmn ? 128u : 2u;
      const uint32_t ring0 = uniform(smem_u32(ring)), d0 = uniform(tmem_base), dhi = desc_hi();
      const uint32_t idesc = uniform(S::kGrad ? make_idesc(p.width * planes, kAmn, kBmn, false, 128) : i8_idesc(p.width, 128));
      const int each = FOLD ? kSegLong : count;
      uint32_t run = 0;
      for (int at = 0; at < count && ok; at += each, ++run) {
        const int acc = FOLD ? (int)(run & 1) : 0;
        if (FOLD && !mbar_wait_warp(&sh.tempty[acc], ((run >> 1) & 1u) ^ 1u, abort, status, ST_WAIT_TMEM_EMPTY, kWaitSpinDefault)) { ok = false; break; }
        if (FOLD) tc_fence_after();
        const uint32_t d = d0 + (uint32_t)acc * acc_cols;
        for (int i = 0; i < min(each, count - at); ++i) {
          if (!mbar_wait_warp(&sh.full[stage], phase, abort, status, ST_WAIT_FULL, kWaitSpinDefault)) { ok = false; break; }
          tc_fence_after();
          const uint32_t slot = ring0 + (uint32_t)(stage * bytes), alo = desc_lo(slot, kAmn ? 8192u : 16u), blo = desc_lo(slot + 16384, kBmn ? 8192u : 16u);
          if (leader) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const uint64_t da = desc_join(alo + q * kAstep, dhi), db = desc_join(blo + q * kBstep, dhi);
              if (S::kGrad) mma_bf16<false>(d, da, db, idesc, i || q ? 1u : 0u);
              else mma_i8<false>(d, da, db, idesc, i || q ? 1u : 0u);
            }
            mma_commit(&sh.empty[stage]);
          }
          __syncwarp();
          if (++stage == p.ring) { stage = 0; phase ^= 1u; }
        }
        if (ok && leader) mma_commit(&sh.tfull[acc]);
        __syncwarp();
      }
    }
  } else if (S::kGrad && warp >= 8) {
    if (FOLD) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kStripDecode));
    // ------------------------------------------------------------------ codes to bf16 numbers: the teams take turns; a warp has
    // four of every sixteen rows of K, eight lanes to a row, 16 codes to a lane
    const int team = (warp - 8) >> 2, row0 = 4 * (warp & 3) + (lane >> 3), j = lane & 7, sub = row0 & 7;
    // the 128-byte swizzle; lanes 4 to 7 write their second chunk first, so that eight lanes meet no bank twice
    const int odd = j >> 2, from = row0 * 128 + 16 * j, to = odd * 8192 + row0 * 128;
    const int at0 = to + ((2 * (j & 3) + odd) ^ sub) * 16, at1 = to + ((2 * (j & 3) + 1 - odd) ^ sub) * 16;
    // scales, a turn ahead: one of its row's four to a lane, or (FOLD, where K runs along a row of dy) those of its chunk of eight, or both
    constexpr bool kAlong = FOLD && OP == INPUT_GRAD;
    constexpr int kChunk = kAlong ? 8 : 1;
    const float* const scale = a.scale + (a.scale_groups > 1 ? f0 / 128 : 0);
    auto scale_at = [&](int i, int at) {
      const int k = (k0 + i) * 64 + at;
      return i < count && k < a.k ? __ldg(scale + (int64_t)k * a.scale_groups) : 0.f;
    };
    // (the form is chosen once: asked for in every stage, 1 x 14336 x 4096 takes 39.5 us for 34)
    auto decode = [&](auto form) {
      constexpr bool kApart = FOLD && decltype(form)::value;
      float next = 0.f, next_of[kChunk] = {};
      auto scales_of = [&](int i) {
        if (kApart || !kAlong) next = j < 4 ? scale_at(i, 16 * j + row0) : 0.f;
        if (kAlong && planes > 1) {
#pragma unroll
          for (int e = 0; e < kChunk; ++e) next_of[e] = scale_at(i, 8 * j + e);
        }
      };
      int stage = team, rs = team;           // (either ring has at least as many stages as there are teams)
      uint32_t phase = 0, raw_phase = 0;
      scales_of(team);
      for (int i = team; i < count; i += kStripTeams) {
        const float mine = next;
        const Split own = kApart ? split_scale(mine) : Split{0u, mine};
        float m_of[kChunk];
#pragma unroll
        for (int e = 0; e < kChunk; ++e) m_of[e] = kApart && planes > 1 ? split_scale(next_of[e]).m : next_of[e];
        scales_of(i + kStripTeams);
        if (!mbar_wait_warp(&sh.raw_full[rs], raw_phase, abort, status, ST_WAIT_FULL, kWaitSpinDefault)) break;
        const uint8_t* const src = raw + rs * p.raw_bytes;
        uint4 q[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) q[r] = *reinterpret_cast<const uint4*>(src + from + r * 2048);
        if (!mbar_wait_warp(&sh.empty[stage], phase ^ 1u, abort, status, ST_WAIT_EMPTY, kWaitSpinDefault)) break;
        uint8_t* const dst = ring + stage * bytes;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const uint32_t c0 = odd ? q[r].z : q[r].x, c1 = odd ? q[r].w : q[r].y, c2 = odd ? q[r].x : q[r].z, c3 = odd ? q[r].y : q[r].w;
          uint32_t u[4], v[4];
          if (FOLD) {
            if (a.e4m3) { decode8<true>(c0, c1, u); decode8<true>(c2, c3, v); }
            else { decode8<false>(c0, c1, u); decode8<false>(c2, c3, v); }
            if (kApart) {
              const uint32_t power = __shfl_sync(0xffffffffu, own.power, (lane & 24) | r);
#pragma unroll
              for (int e = 0; e < 4; ++e) { u[e] = times_bf16x2(u[e], power); v[e] = times_bf16x2(v[e], power); }
            }
          } else {
            const float s = __shfl_sync(0xffffffffu, mine, (lane & 24) | r);
            if (a.e4m3) { decode8<true>(c0, c1, s, u); decode8<true>(c2, c3, s, v); }
            else { decode8<false>(c0, c1, s, u); decode8<false>(c2, c3, s, v); }
          }
          put4(dst + at0 + r * 2048, u);
          put4(dst + at1 + r * 2048, v);
        }
        if (FOLD) {
          // the other operand times m, a chunk of eight at a time, from where TMA has put it to the same place of each plane
          const int o = row0 * 128 + ((j ^ sub) * 16);
#pragma unroll 1
          for (int r = 0; r < p.width / 16; ++r) {
            const uint4 b = *reinterpret_cast<const uint4*>(src + kStripRawBytes + o + r * 2048);
            const uint32_t w[4] = {b.x, b.y, b.z, b.w};
            if (kApart && planes == 1) {
              put4(dst + 16384 + o + r * 2048, w);
              continue;
            }
            const float row_m = kAlong ? 0.f : __shfl_sync(0xffffffffu, own.m, (lane & 24) | (r & 3));
            float2 x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
              x[e] = mul2(make_float2(__uint_as_float(w[e] << 16), __uint_as_float(w[e] & 0xffff0000u)),
                          kAlong ? make_float2(m_of[2 * e % kChunk], m_of[(2 * e + 1) % kChunk]) : make_float2(row_m, row_m));
            for (int n = 0; n < planes; ++n) {
              uint32_t u[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) u[e] = pack_bf16x2_rn(x[e].x, x[e].y);
              put4(dst + 16384 + n * p.width * 128 + o + r * 2048, u);
              if (n + 1 < planes) {
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = left_of_bf16(x[e]);
              }
            }
          }
        }
        fence_async_smem();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&sh.raw_empty[rs]);
          mbar_arrive(&sh.full[stage]);
        }
        stage += kStripTeams;
        if (stage >= p.ring) { stage -= p.ring; phase ^= 1u; }
        rs += kStripTeams;
        if (rs >= p.raw) { rs -= p.raw; raw_phase ^= 1u; }
      }
    };
    if (apart) decode(std::true_type{});
    else decode(std::false_type{});
  } else {
    if (FOLD) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kStripDrain));
    // ------------------------------------------------------------------ this CTA's sums [columns][128], over the ring once all that was
    // in it has been multiplied
    bool ok = true;
    const uint32_t lane_addr = tmem_base + ((uint32_t)(32 * (warp & 3)) << 16);
    int* const sums = reinterpret_cast<int*>(ring) + 32 * (warp & 3) + lane;
    auto wait_full = [&](int acc, uint32_t parity) {
      if (lane == 0) ok = mbar_wait(&sh.tfull[acc], parity, abort, status, ST_WAIT_TMEM_FULL, kWaitSpinDefault);
      ok = __shfl_sync(0xffffffffu, ok, 0);
      tc_fence_after();
    };
    if (FOLD) {
      float v[kFoldWidth];
#pragma unroll
      for (int e = 0; e < kFoldWidth; ++e) v[e] = 0.f;
      const int n_seg = (count + kSegLong - 1) / kSegLong;
#pragma unroll 1
      for (int s = 0; s < n_seg && ok; ++s) {
        const int acc = s & 1;
        wait_full(acc, (uint32_t)(s >> 1) & 1u);
        if (!ok) break;
#pragma unroll 1
        for (int n = planes - 1; n >= 0; --n) {                      // (the smallest first)
#pragma unroll
          for (int c = 0; c < kFoldWidth; c += 16) {
            if (c < p.width) {
              float x[16];
              tmem_ld16(lane_addr + (uint32_t)acc * acc_cols + (uint32_t)(n * p.width + c), x);
              tmem_ld_wait();
#pragma unroll
              for (int e = 0; e < 16; ++e) v[c + e] += x[e];
            }
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.tempty[acc]);
      }
#pragma unroll
      for (int c = 0; c < kFoldWidth; ++c)
        if (ok && c < p.width) sums[c * 128] = __float_as_int(v[c]);
    } else {
      wait_full(0, 0);
      if (ok) {
        for (int c = 0; c < p.width; c += 16) {
          float v[16];
          tmem_ld16(lane_addr + (uint32_t)c, v);
          tmem_ld_wait();
#pragma unroll
          for (int e = 0; e < 16; ++e) sums[(c + e) * 128] = __float_as_int(v[e]);
        }
      }
    }
    tc_fence_before();
    __syncwarp();
    if (FOLD) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kStripRegs));
  }
  __syncthreads();
  // (not before: the warps that drain have taken theirs and given them back by now, so that nobody waits for registers of a warp that waits here)
  if (FOLD && (warp < 4 || warp >= 8)) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kStripRegs));
  if (split > 1) cluster_sync();
  if (split == 1) put_together<OP, FOLD, 1>(a, ring, rank, f0, c0);
  else if (split == 2) put_together<OP, FOLD, 2>(a, ring, rank, f0, c0);
  else if (split == 4) put_together<OP, FOLD, 4>(a, ring, rank, f0, c0);
  else put_together<OP, FOLD, 8>(a, ring, rank, f0, c0);
  __syncwarp();
  if (split > 1) cluster_sync();      // no CTA leaves while another may still read its sums
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, tmem_cols);
  }
}

// ---- forward, one or two tokens --------------------------------------------------------------------------------------
// The weight once past the tokens: a warp has kRowsOfWarp rows of the weight, 512 bytes of each at a time, which a lane multiplies four codes at a
// time (dp4a) with those of every token; `split` warps of a CTA share a row's K.  Bound by HBM: the rows are read end to end, which
// the strips' boxes of 128 x 128 bytes do not do (1 x 14336 x 4096, codes from HBM: 13.2 -> 11.5 us = 5.1 TB/s).  With more tokens the
// products take longer than the rows' way (4 tokens 15.5 us from L2, strips 10.5).
constexpr int kRowsOfWarp = 4, kLineThreads = 256;

struct LineArgs {
  const uint8_t *x, *w;
  const float *xs, *ws;
  void* y;
  int32_t* status;
  int64_t y_ld;
  int32_t x_ld, w_ld, out, in, split, f32;
};

// The 16 codes of a row from byte k on, as far as the row goes (rows are multiples of eight long).
__device__ __forceinline__ uint4 codes16(const uint8_t* row, int k, int n) {
  if (k + 16 <= n) return __ldg(reinterpret_cast<const uint4*>(row + k));
  uint4 q = make_uint4(0, 0, 0, 0);
  if (k + 8 <= n) { const uint2 h = __ldg(reinterpret_cast<const uint2*>(row + k)); q.x = h.x; q.y = h.y; }
  return q;
}
__device__ __forceinline__ int dot16(const uint4& a, const uint4& b, int sum) {
  sum = __dp4a((int)a.x, (int)b.x, sum);
  sum = __dp4a((int)a.y, (int)b.y, sum);
  sum = __dp4a((int)a.z, (int)b.z, sum);
  return __dp4a((int)a.w, (int)b.w, sum);
}

template <int TOKENS>
__global__ void __launch_bounds__(kLineThreads) linear8_line_kernel(const LineArgs a) {
  __shared__ int part[8][kRowsOfWarp][TOKENS];
  wait_for_previous_kernel();
  if (blockIdx.x == 0)
    for (int i = threadIdx.x; i < kMostWords; i += kLineThreads) a.status[i] = 0;      // (nothing here waits)
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, groups = 8 / a.split, group = warp / a.split, share = warp - group * a.split;
  const int n0 = ((int)blockIdx.x * groups + group) * kRowsOfWarp;
  const uint8_t* rows[kRowsOfWarp];
#pragma unroll
  for (int r = 0; r < kRowsOfWarp; ++r) rows[r] = a.w + (int64_t)min(n0 + r, a.out - 1) * a.w_ld;
  int sum[kRowsOfWarp][TOKENS] = {};
  const int step = 512 * a.split;
  auto add = [&](const uint4* w, int k) {
#pragma unroll
    for (int t = 0; t < TOKENS; ++t) {
      const uint4 x = codes16(a.x + (int64_t)t * a.x_ld, k, a.in);
#pragma unroll
      for (int r = 0; r < kRowsOfWarp; ++r) sum[r][t] = dot16(w[r], x, sum[r][t]);
    }
  };
  if (n0 < a.out) {
    int k = 512 * share + 16 * lane;
    for (; k + step < a.in; k += 2 * step) {            // two pieces of every row on their way
      uint4 w[2][kRowsOfWarp];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int r = 0; r < kRowsOfWarp; ++r) w[u][r] = codes16(rows[r], k + u * step, a.in);
      add(w[0], k);
      add(w[1], k + step);
    }
    if (k < a.in) {
      uint4 w[kRowsOfWarp];
#pragma unroll
      for (int r = 0; r < kRowsOfWarp; ++r) w[r] = codes16(rows[r], k, a.in);
      add(w, k);
    }
  }
#pragma unroll
  for (int r = 0; r < kRowsOfWarp; ++r)
#pragma unroll
    for (int t = 0; t < TOKENS; ++t) {
      const int all = __reduce_add_sync(0xffffffffu, sum[r][t]);
      if (lane == 0) part[warp][r][t] = all;
    }
  __syncthreads();
  for (int i = threadIdx.x; i < groups * kRowsOfWarp * TOKENS; i += kLineThreads) {
    const int r = i % kRowsOfWarp, t = i / kRowsOfWarp % TOKENS, g = i / (kRowsOfWarp * TOKENS);
    const int n = ((int)blockIdx.x * groups + g) * kRowsOfWarp + r;
    if (n >= a.out) continue;
    int all = 0;
    for (int s = 0; s < a.split; ++s) all += part[g * a.split + s][r][t];
    const float y = (float)all * a.xs[t] * a.ws[n];
    if (a.f32) static_cast<float*>(a.y)[(int64_t)t * a.y_ld + n] = y;
    else static_cast<uint16_t*>(a.y)[(int64_t)t * a.y_ld + n] = (uint16_t)pack_bf16x2_rn(y, 0.f);
  }
}

// ---- host ----------------------------------------------------------------------------------------------------------

// `planes` matrices of bf16 numbers [rows, cols], one behind the other, in boxes of 64 columns x 64 rows.
bool encode_planes(CUtensorMap* out, const void* base, int64_t planes, int64_t rows, int64_t cols, int64_t pitch) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (!fn) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)planes};
  const cuuint64_t strides[2] = {(cuuint64_t)pitch * 2, (cuuint64_t)(rows * pitch) * 2};
  const cuuint32_t box[3] = {64, 64, 1};
  const cuuint32_t estr[3] = {1, 1, 1};
  return fn(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// `parts` results [rows, cols], one behind the other, in boxes of 32 rows of 64 bytes, or `wide` of 128, with the swizzle of as many.
bool encode_result(CUtensorMap* out, void* base, int64_t parts, int64_t rows, int64_t cols, int64_t pitch, bool f32, bool wide) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (!fn) return false;
  const cuuint64_t bytes = f32 ? 4 : 2, line = (cuuint64_t)pitch * bytes;
  const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)parts};
  const cuuint64_t strides[2] = {line, parts > 1 ? (cuuint64_t)rows * line : line};
  const cuuint32_t box[3] = {(cuuint32_t)((wide ? 128 : 64) / bytes), 32, 1};
  const cuuint32_t estr[3] = {1, 1, 1};
  return fn(out, f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, base, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            wide ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Whether some row of a result starts inside a sector of 32 bytes.
bool off_sectors(const void* out, int64_t pitch, bool f32) { return !f32 && ((uintptr_t)out % 32 || pitch % 16); }

// A row-major matrix of bytes in boxes of 128 columns x box_rows rows, with the 128-byte swizzle or as they lie.
bool encode_bytes(CUtensorMap* out, const void* base, uint64_t rows, uint64_t cols, uint64_t pitch, uint32_t box_rows, bool swizzle = true) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (!fn) return false;
  const cuuint64_t dims[2] = {cols, rows};
  const cuuint64_t strides[1] = {pitch};
  const cuuint32_t box[2] = {128, box_rows};
  const cuuint32_t estr[2] = {1, 1};
  return fn(out, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            swizzle ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int OP, bool LONG, bool WIDE>
int allow(int* resident, int sms) {
  using S = Shape<OP, LONG, WIDE>;
  ADAPM_CUDA(cudaFuncSetAttribute(linear8_kernel<OP, LONG, WIDE>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem));
  if (LONG) {
    cudaFuncAttributes fa;                  // (with fewer registers at launch the split above would wait for ever)
    ADAPM_CUDA(cudaFuncGetAttributes(&fa, linear8_kernel<OP, LONG, WIDE>));
    if (fa.numRegs < kLongRegs) {
      set_error_text("linear8_kernel was built with fewer registers than it divides among its warps");
      return ADAPM_EUNSUPPORTED;
    }
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(sms / 2 * 2); cfg.blockDim = dim3(S::kThreads); cfg.dynamicSmemBytes = S::kSmem;
  cudaLaunchAttribute at;
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = 2; at.val.clusterDim.y = 1; at.val.clusterDim.z = 1;
  cfg.attrs = &at; cfg.numAttrs = 1;
  int n = 0;
  ADAPM_CUDA(cudaOccupancyMaxActiveClusters(&n, linear8_kernel<OP, LONG, WIDE>, &cfg));
  *resident = std::min(*resident, n);
  return ADAPM_OK;
}

template <int OP, bool LONG>
int allow_strips() {
  ADAPM_CUDA(cudaFuncSetAttribute(linear8_strip_kernel<OP, LONG>, cudaFuncAttributeMaxDynamicSharedMemorySize, kStripSmem + 1024));
  if (LONG) {
    cudaFuncAttributes fa;                  // (as above)
    ADAPM_CUDA(cudaFuncGetAttributes(&fa, linear8_strip_kernel<OP, LONG>));
    if (fa.numRegs < kStripRegs) {
      set_error_text("linear8_strip_kernel was built with fewer registers than it divides among its warps");
      return ADAPM_EUNSUPPORTED;
    }
  }
  return ADAPM_OK;
}

// Pairs of CTAs that run at the same time on this device; the kernels' shared memory is allowed on the way.  (Once per device.)
int pairs_of(int device, int* pairs) {
  static std::mutex mu;
  static int known[64] = {};
  if (device < 0 || device >= 64) return ADAPM_ERANGE;
  std::lock_guard<std::mutex> lock(mu);
  if (!known[device]) {
    int sms = 0;
    ADAPM_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device));
    int n = std::min(sms / 2, (int)kMostWords);
    int rc = allow<FORWARD, false, false>(&n, sms);
    if (rc == ADAPM_OK) rc = allow<FORWARD, false, true>(&n, sms);
    if (rc == ADAPM_OK) rc = allow<INPUT_GRAD, false, false>(&n, sms);
    if (rc == ADAPM_OK) rc = allow<INPUT_GRAD, false, true>(&n, sms);
    if (rc == ADAPM_OK) rc = allow<INPUT_GRAD, true, false>(&n, sms);
    if (rc == ADAPM_OK) rc = allow<WEIGHT_GRAD, false, false>(&n, sms);
    if (rc == ADAPM_OK) rc = allow<WEIGHT_GRAD, false, true>(&n, sms);
    if (rc == ADAPM_OK) rc = allow<WEIGHT_GRAD, true, false>(&n, sms);
    if (rc == ADAPM_OK) rc = allow_strips<FORWARD, false>();
    if (rc == ADAPM_OK) rc = allow_strips<INPUT_GRAD, false>();
    if (rc == ADAPM_OK) rc = allow_strips<INPUT_GRAD, true>();
    if (rc == ADAPM_OK) rc = allow_strips<WEIGHT_GRAD, false>();
    if (rc == ADAPM_OK) rc = allow_strips<WEIGHT_GRAD, true>();
    if (rc != ADAPM_OK) return rc;
    known[device] = std::max(1, n);
  }
  *pairs = known[device];
  return ADAPM_OK;
}

template <int OP, bool LONG, bool WIDE>
cudaError_t launch(const Args& a, cudaStream_t s) {
  using S = Shape<OP, LONG, WIDE>;
  return launch_clusters(true, 2, linear8_kernel<OP, LONG, WIDE>, 2 * (unsigned)a.pairs, S::kThreads, S::kSmem, s, a);
}
template <int OP>
cudaError_t launch_short(const Args& a, bool wide, cudaStream_t s) { return wide ? launch<OP, false, true>(a, s) : launch<OP, false, false>(a, s); }

struct Buffer { const void* p; int64_t align; Place at; };

// What the three calls check of their buffers: `in` are read, `out` is written, as is the scratch.
int check_buffers(std::initializer_list<Buffer> in, const Buffer& out, void* scratch, size_t scratch_bytes, int64_t needed, const char* overlap, int* device) {
  for (const Buffer& b : in)
    if (!b.p) return ADAPM_EINVAL;
  if (!out.p || !scratch) return ADAPM_EINVAL;
  for (const Buffer& b : in)
    if ((uintptr_t)b.p % (uintptr_t)b.align) return ADAPM_EALIGN;
  if ((uintptr_t)out.p % (uintptr_t)out.align || (uintptr_t)scratch % 256) return ADAPM_EALIGN;
  if (scratch_bytes < (size_t)needed) return ADAPM_ENOWORKSPACE;
  const Place own = vector_at(scratch, needed, 1);
  bool apart = !share(own, out.at);
  for (const Buffer& b : in) apart = apart && !share(out.at, b.at) && !share(own, b.at);
  if (!apart) {
    set_error_text(overlap);
    return ADAPM_EINVAL;
  }
  const Buffer* const at = in.begin();
  return check_on_this_device({out.p, scratch, at[0].p, at[1].p, at[2].p, in.size() > 3 ? at[3].p : nullptr}, device);
}

int64_t room_of(size_t scratch_bytes) { return (int64_t)std::min<size_t>(scratch_bytes, (size_t)INT64_MAX); }

Buffer bf16_or_f32(const void* p, int64_t rows, int64_t ld, int64_t cols, int32_t dtype) { return Buffer{p, 16, matrix_at(p, rows, ld, cols, type_bytes(dtype))}; }
Buffer codes_at(const void* p, int64_t rows, int64_t ld, int64_t cols) { return Buffer{p, 16, matrix_at(p, rows, ld, cols, 1)}; }
Buffer floats_at(const float* p, int64_t n, int64_t align) { return Buffer{p, align, vector_at(p, n, 4)}; }

template <int OP, bool LONG>
cudaError_t launch_strips(const StripArgs& a, cudaStream_t s) {
  const size_t smem = (size_t)a.plan.ring * a.plan.stage_bytes + (size_t)a.plan.raw * a.plan.raw_bytes + 1024;
  return launch_clusters(true, (unsigned)a.plan.split, linear8_strip_kernel<OP, LONG>, (unsigned)a.plan.ctas, (unsigned)StripShape<OP, LONG>::kThreads, smem, s, a);
}

// A gradient: [rows, cols] = A [rows, K] (or its transpose) times codes [K, cols].
int gradient(const adapm_linear8& d, int32_t which, const void* dy, const void* codes, const float* scales, void* out, int32_t out_dtype, int64_t out_ld,
             void* scratch, const Form& form, int pairs, cudaStream_t s) {
  const bool weight = which == WEIGHT_GRAD;
  const StripPlan& strip = form.strip;
  const Plan& plan = form.plan;
  if (form.form == STRIPS) {
    StripArgs t;
    std::memset(&t, 0, sizeof(t));
    t.plan = strip;
    t.k = (int32_t)(weight ? d.tokens : d.out_features);
    if (!encode_bytes(&t.codes, codes, t.k, d.in_features, weight ? d.x8_ld : d.w8_ld, 64, false) ||
        !encode_bf16_matrix(&t.other, dy, d.tokens, d.out_features, d.y_ld, weight ? 64 : (uint32_t)strip.width)) {
      set_error_text("cuTensorMapEncodeTiled failed for a gradient of linear8");
      return ADAPM_ECUDA;
    }
    t.scale = scales; t.scale_groups = weight && d.x_group ? (int32_t)((d.in_features + 127) / 128) : 1;
    t.out = out; t.out_ld = out_ld; t.status = (int32_t*)scratch;
    t.columns = (int32_t)(weight ? d.out_features : d.tokens); t.features = (int32_t)d.in_features;
    t.f32 = out_dtype == ADAPM_TYPE_F32; t.accumulate = weight && d.accumulate != 0; t.e4m3 = weight && d.x_code == ADAPM_CODE_E4M3;
    ADAPM_CUDA(strip.fold ? (weight ? launch_strips<WEIGHT_GRAD, true>(t, s) : launch_strips<INPUT_GRAD, true>(t, s))
                          : (weight ? launch_strips<WEIGHT_GRAD, false>(t, s) : launch_strips<INPUT_GRAD, false>(t, s)));
    return ADAPM_OK;
  }
  Args a;
  std::memset(&a, 0, sizeof(a));
  a.plan = plan;
  void* const decoded = (char*)scratch + kHeadBytes;
  adapm_codes8 q;
  q.rows = weight ? d.tokens : d.out_features; q.cols = d.in_features; q.x_ld = decoded_pitch(d.in_features); q.codes_ld = weight ? d.x8_ld : d.w8_ld;
  q.dtype = ADAPM_TYPE_BF16; q.code = weight ? d.x_code : ADAPM_CODE_INT8; q.group = weight ? d.x_group : 0; q.pow2 = 0;
  const int planes = out_dtype == ADAPM_TYPE_F32 ? kPlanesF32 : 1;
  if (!encode_bf16_matrix(&a.a, dy, d.tokens, d.out_features, d.y_ld, weight ? 64 : 128) || !encode_planes(&a.b, decoded, planes, q.rows, q.cols, q.x_ld)) {
    set_error_text("cuTensorMapEncodeTiled failed for a gradient of linear8");
    return ADAPM_ECUDA;
  }
  a.out = out; a.out_ld = out_ld;
  a.status = (int32_t*)scratch;
  float* const parts = (float*)((char*)scratch + plan.part_at);
  a.out_f32 = out_dtype == ADAPM_TYPE_F32;
  const bool accumulate = weight && d.accumulate != 0;
  a.accumulate = accumulate && plan.parts == 1;
  a.pairs = std::min(pairs, plan.items);
  a.seg = a.out_f32 ? kSegLong : kSegShort;
  const bool is_long = a.out_f32 || plan.each > kShortStages;
  const bool wide = !is_long && plan.parts == 1 && (a.accumulate || off_sectors(out, out_ld, a.out_f32));
  if (!(plan.parts > 1 ? encode_result(&a.o, parts, plan.parts, plan.rows, plan.cols, plan.cols, true, wide)
                       : encode_result(&a.o, out, 1, plan.rows, plan.cols, out_ld, a.out_f32, wide))) {
    set_error_text("cuTensorMapEncodeTiled failed for a gradient of linear8");
    return ADAPM_ECUDA;
  }
  if (a.out_f32) {
    int32_t* const words = (int32_t*)scratch + kMostWords;
    a.scale_words = words;
    const int64_t n = q.rows * (q.group ? (q.cols + 127) / 128 : 1);
    if (n > kFewScales) ADAPM_CUDA(launch_chained(true, linear8_scales_kernel, (unsigned)std::min<int64_t>(kScaleWords, (n + 2047) / 2048), 256, 0, s, scales, n, words));
    PlanesArgs p;
    p.codes = static_cast<const uint8_t*>(codes); p.scales = scales; p.words = words; p.out = (uint16_t*)decoded;
    p.scan = n > kFewScales ? 0 : n;
    p.codes_ld = q.codes_ld; p.ld = q.x_ld; p.rows = q.rows; p.cols = (int32_t)q.cols; p.groups = q.group ? (int32_t)((q.cols + 127) / 128) : 1;
    const int64_t chunks = q.rows * (q.cols / 8);
    const unsigned grid = (unsigned)std::min<int64_t>((chunks + 255) / 256, 148 * 16);
    ADAPM_CUDA(q.code == ADAPM_CODE_E4M3 ? launch_chained(true, linear8_planes_kernel<true>, grid, 256, 0, s, p) : launch_chained(true, linear8_planes_kernel<false>, grid, 256, 0, s, p));
  } else {
    const int rc = launch_dequant8(q, codes, scales, decoded, s);
    if (rc != ADAPM_OK) return rc;
  }
  ADAPM_CUDA(weight ? (is_long ? launch<WEIGHT_GRAD, true, false>(a, s) : launch_short<WEIGHT_GRAD>(a, wide, s))
                    : (is_long ? launch<INPUT_GRAD, true, false>(a, s) : launch_short<INPUT_GRAD>(a, wide, s)));
  if (plan.parts == 1) return ADAPM_OK;
  SumArgs u;
  u.part = parts; u.out = out; u.out_ld = out_ld; u.fours = plan.cols / 4; u.places = (int64_t)plan.rows * u.fours;
  u.part_elems = (int64_t)plan.rows * plan.cols; u.parts = plan.parts; u.f32 = a.out_f32; u.accumulate = accumulate;
  ADAPM_CUDA(launch_chained(true, linear8_sum_kernel, (unsigned)std::min<int64_t>((u.places + 255) / 256, 148 * 8), 256, 0, s, u));
  return ADAPM_OK;
}

}  // namespace
}  // namespace adapm

using namespace adapm;

extern "C" size_t adapm_linear8_scratch_bytes(const adapm_linear8* d, int32_t which) {
  if (!d || check_desc(*d, which) != ADAPM_OK) return 0;
  return (size_t)form_of(*d, which).bytes;
}

extern "C" int adapm_linear8_forward(const adapm_linear8* d, const void* x8, const float* xs, const void* w8, const float* ws, void* y,
                                     void* scratch, size_t scratch_size, adapm_stream stream) {
  if (!d) return ADAPM_EINVAL;
  int rc = check_desc(*d, FORWARD);
  if (rc != ADAPM_OK || d->tokens == 0) return rc;
  const Form form = form_of(*d, FORWARD, room_of(scratch_size));
  const Plan& plan = form.plan;
  int device, pairs;
  rc = check_buffers({codes_at(x8, d->tokens, d->x8_ld, d->in_features), floats_at(xs, d->tokens, 4), codes_at(w8, d->out_features, d->w8_ld, d->in_features),
                      floats_at(ws, d->out_features, 16)},
                     bf16_or_f32(y, d->tokens, d->y_ld, d->out_features, d->y_dtype), scratch, scratch_size, form.bytes,
                     "adapm_linear8_forward: the output or the scratch overlaps another buffer", &device);
  if (rc == ADAPM_OK) rc = pairs_of(device, &pairs);
  if (rc != ADAPM_OK) return rc;
  if (form.form == LINES) {
    LineArgs l;
    l.x = static_cast<const uint8_t*>(x8); l.w = static_cast<const uint8_t*>(w8); l.xs = xs; l.ws = ws; l.y = y;
    l.status = (int32_t*)scratch; l.y_ld = d->y_ld; l.x_ld = (int32_t)d->x8_ld; l.w_ld = (int32_t)d->w8_ld;
    l.out = (int32_t)d->out_features; l.in = (int32_t)d->in_features; l.f32 = d->y_dtype == ADAPM_TYPE_F32;
    // as many warps as give every SM sixteen, a piece of K for each
    const int64_t row_groups = (d->out_features + kRowsOfWarp - 1) / kRowsOfWarp;
    l.split = 1;
    while (l.split < 8 && row_groups * l.split < 2 * kPlannedPairs * 16 && 512 * l.split < d->in_features) l.split *= 2;
    const unsigned grid = (unsigned)((row_groups * l.split + 7) / 8);
    cudaStream_t s = (cudaStream_t)stream;
    ADAPM_CUDA(d->tokens == 1 ? launch_chained(true, linear8_line_kernel<1>, grid, kLineThreads, 0, s, l)
                             : launch_chained(true, linear8_line_kernel<2>, grid, kLineThreads, 0, s, l));
    return ADAPM_OK;
  }
  if (form.form == STRIPS) {
    const StripPlan& strip = form.strip;
    StripArgs t;
    std::memset(&t, 0, sizeof(t));
    t.plan = strip;
    if (!encode_bytes(&t.codes, w8, d->out_features, d->in_features, d->w8_ld, 128) ||
        !encode_bytes(&t.other, x8, d->tokens, d->in_features, d->x8_ld, (uint32_t)strip.width)) {
      set_error_text("cuTensorMapEncodeTiled failed for linear8");
      return ADAPM_ECUDA;
    }
    t.xs = xs; t.ws = ws; t.out = y; t.out_ld = d->y_ld; t.status = (int32_t*)scratch;
    t.columns = (int32_t)d->tokens; t.features = (int32_t)d->out_features; t.f32 = d->y_dtype == ADAPM_TYPE_F32;
    ADAPM_CUDA((launch_strips<FORWARD, false>(t, (cudaStream_t)stream)));
    return ADAPM_OK;
  }
  Args a;
  std::memset(&a, 0, sizeof(a));
  a.plan = plan;
  const bool wide = off_sectors(y, d->y_ld, d->y_dtype == ADAPM_TYPE_F32);
  if (!encode_bytes(&a.a, x8, d->tokens, d->in_features, d->x8_ld, 128) || !encode_bytes(&a.b, w8, d->out_features, d->in_features, d->w8_ld, 128) ||
      !encode_result(&a.o, y, 1, d->tokens, d->out_features, d->y_ld, d->y_dtype == ADAPM_TYPE_F32, wide)) {
    set_error_text("cuTensorMapEncodeTiled failed for linear8");
    return ADAPM_ECUDA;
  }
  a.a_scale = xs; a.b_scale = ws;
  a.out = y; a.out_ld = d->y_ld; a.out_f32 = d->y_dtype == ADAPM_TYPE_F32;
  a.status = (int32_t*)scratch;
  a.pairs = std::min(pairs, plan.items);
  ADAPM_CUDA(launch_short<FORWARD>(a, wide, (cudaStream_t)stream));
  return ADAPM_OK;
}

extern "C" int adapm_linear8_input_grad(const adapm_linear8* d, const void* dy, const void* w8, const float* ws, void* dx, void* scratch,
                                        size_t scratch_size, adapm_stream stream) {
  if (!d) return ADAPM_EINVAL;
  int rc = check_desc(*d, INPUT_GRAD);
  if (rc != ADAPM_OK || d->tokens == 0) return rc;
  const Form form = form_of(*d, INPUT_GRAD, room_of(scratch_size));
  int device, pairs;
  rc = check_buffers({bf16_or_f32(dy, d->tokens, d->y_ld, d->out_features, ADAPM_TYPE_BF16), codes_at(w8, d->out_features, d->w8_ld, d->in_features),
                      floats_at(ws, d->out_features, 4)},
                     bf16_or_f32(dx, d->tokens, d->dx_ld, d->in_features, d->dx_dtype), scratch, scratch_size, form.bytes,
                     "adapm_linear8_input_grad: the output or the scratch overlaps another buffer", &device);
  if (rc == ADAPM_OK) rc = pairs_of(device, &pairs);
  if (rc != ADAPM_OK) return rc;
  return gradient(*d, INPUT_GRAD, dy, w8, ws, dx, d->dx_dtype, d->dx_ld, scratch, form, pairs, (cudaStream_t)stream);
}

extern "C" int adapm_linear8_weight_grad(const adapm_linear8* d, const void* dy, const void* x8, const float* xs, void* dweight, void* scratch,
                                         size_t scratch_size, adapm_stream stream) {
  if (!d) return ADAPM_EINVAL;
  int rc = check_desc(*d, WEIGHT_GRAD);
  if (rc != ADAPM_OK) return rc;
  if (!dweight) return ADAPM_EINVAL;
  cudaStream_t s = (cudaStream_t)stream;
  int device, pairs;
  if (d->tokens == 0) {                        // no token: the gradient is zero
    if (d->accumulate) return ADAPM_OK;
    if ((uintptr_t)dweight % 16) return ADAPM_EALIGN;
    rc = check_on_this_device({dweight}, &device);
    if (rc != ADAPM_OK) return rc;
    const int64_t gb = type_bytes(d->dweight_dtype);
    ADAPM_CUDA(cudaMemset2DAsync(dweight, (size_t)(d->dweight_ld * gb), 0, (size_t)(d->in_features * gb), (size_t)d->out_features, s));
    return ADAPM_OK;
  }
  const Form form = form_of(*d, WEIGHT_GRAD, room_of(scratch_size));
  const int64_t groups = d->x_group ? (d->in_features + 127) / 128 : 1;
  rc = check_buffers({bf16_or_f32(dy, d->tokens, d->y_ld, d->out_features, ADAPM_TYPE_BF16), codes_at(x8, d->tokens, d->x8_ld, d->in_features),
                      floats_at(xs, d->tokens * groups, 4)},
                     bf16_or_f32(dweight, d->out_features, d->dweight_ld, d->in_features, d->dweight_dtype), scratch, scratch_size, form.bytes,
                     "adapm_linear8_weight_grad: the output or the scratch overlaps another buffer", &device);
  if (rc == ADAPM_OK) rc = pairs_of(device, &pairs);
  if (rc != ADAPM_OK) return rc;
  return gradient(*d, WEIGHT_GRAD, dy, x8, xs, dweight, d->dweight_dtype, d->dweight_ld, scratch, form, pairs, s);
}

extern "C" int adapm_linear8_status(const void* scratch, adapm_stream stream, int32_t* status) {
  if (!scratch || !status) return ADAPM_EINVAL;
  int32_t words[kMostWords], all = 0;
  ADAPM_CUDA(cudaMemcpyAsync(words, scratch, sizeof(words), cudaMemcpyDeviceToHost, (cudaStream_t)stream));
  ADAPM_CUDA(cudaStreamSynchronize((cudaStream_t)stream));
  for (int32_t w : words) all |= w;
  *status = all;
  return all == 0 ? ADAPM_OK : ADAPM_EDEVICE;
}
