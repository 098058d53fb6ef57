// The products of a linear layer in 8 bits:
//
//   forward      y[t, n]  = xs[t] ws[n] sum_k x8[t, k] w8[n, k]       whole numbers (tcgen05 kind::i8, sums in 32 bits), scaled at the end
//   input grad   dx[t, k] = sum_n dy[t, n] (ws[n] w8[n, k])           bf16 x codes
//   weight grad  dw[n, k] = sum_t dy[t, n] (xs[t] x8[t, k])           bf16 x codes
//
// The gradients' codes travel as bytes as far as shared memory; there eight warps turn them into bf16 numbers, times their scales,
// in the order that the tensor cores read (kind::f16, sums in fp32).  The scale stands beside an index of K, so it cannot wait for
// the end as in the forward product; where it is a power of two, code x scale is a bf16 number and nothing is rounded.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <mutex>

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
constexpr int kRawBytes = 64 * 128;              // codes of a CTA's half of a stage
constexpr int kSegLong = 4, kSegShort = 64;      // stages of 64 K between two sums in registers: gradients in fp32, long ones in bf16

template <int OP, bool LONG>
struct Shape {
  static constexpr bool kGrad = OP != FORWARD;
  static constexpr int kConvert = !kGrad ? 0 : LONG ? 4 : 8;         // warps that make bf16 numbers of codes
  static constexpr int kWarps = 12 + kConvert;                      // after four that issue and eight that drain
  static constexpr int kThreads = 32 * kWarps;
  static constexpr int kStages = kGrad ? 5 : 6;
  static constexpr int kRawStages = kGrad ? 6 : 0;
  static constexpr int kSmem = kStages * kStageBytes + kRawStages * kRawBytes + 1024;
};
// LONG: registers as the four groups of four warps divide those of the launch (the eight that drain keep 128 sums each).
constexpr int kLongRegs = 128, kLongIssue = 48, kLongConvert = 48, kLongDrain = 208;
static_assert(kLongIssue + kLongConvert + 2 * kLongDrain <= 4 * kLongRegs, "a block has the registers that it was launched with");

struct Args {
  CUtensorMap a, b;              // b: K-major (forward) or the codes as they lie (gradients)
  Plan plan;
  const float* a_scale;          // forward: xs
  const float* b_scale;          // ws, or xs of the weight's gradient [K][b_groups]
  void* out;
  float* part;                   // [parts][rows][cols], where K is cut
  int32_t* status;
  int64_t out_ld;
  int32_t k, b_groups, pairs, out_f32, wide, accumulate, seg, e4m3;
};

template <int OP, bool LONG>
struct __align__(8) Shared {
  using S = Shape<OP, LONG>;
  uint64_t full[S::kStages], empty[S::kStages], raw_full[S::kRawStages + 1], raw_empty[S::kRawStages + 1], tfull[2], tempty[2];
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

// Arrives at the barrier of another CTA of the cluster (address from shared_of) and makes what this thread wrote, or saw written,
// visible to who waits there.
__device__ __forceinline__ void mbar_arrive_release_at(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

__device__ __forceinline__ void put4(void* p, const uint32_t* v) { *reinterpret_cast<uint4*>(p) = make_uint4(v[0], v[1], v[2], v[3]); }

// 16 values of a row of which those below n (a multiple of 8) exist, to addresses that are multiples of 32 (wide) or 16 bytes.
__device__ __forceinline__ void store_row16(void* base, int64_t at, const float* x, int n, bool f32, bool wide) {
  if (f32) {
    float* p = static_cast<float*>(base) + at;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (8 * h < n) {
        if (wide) st_f32x8(p + 8 * h, x + 8 * h);
        else {
          *reinterpret_cast<float4*>(p + 8 * h) = make_float4(x[8 * h], x[8 * h + 1], x[8 * h + 2], x[8 * h + 3]);
          *reinterpret_cast<float4*>(p + 8 * h + 4) = make_float4(x[8 * h + 4], x[8 * h + 5], x[8 * h + 6], x[8 * h + 7]);
        }
      }
    }
    return;
  }
  uint16_t* p = static_cast<uint16_t*>(base) + at;
  uint32_t w[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) w[e] = pack_bf16x2_rn(x[2 * e], x[2 * e + 1]);
  if (wide && n >= 16) st_b32x8(p, w);
  else {
    if (n > 0) put4(p, w);
    if (n > 8) put4(p + 8, w + 4);
  }
}
// x += 16 values of a row of which those below n exist.
__device__ __forceinline__ void add_row16(const void* base, int64_t at, float* x, int n, bool f32) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if (8 * h >= n) continue;
    if (f32) {
      const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(base) + at + 8 * h);
      const float4 u = *p, v = *(p + 1);
      x[8 * h] += u.x; x[8 * h + 1] += u.y; x[8 * h + 2] += u.z; x[8 * h + 3] += u.w;
      x[8 * h + 4] += v.x; x[8 * h + 5] += v.y; x[8 * h + 6] += v.z; x[8 * h + 7] += v.w;
    } else {
      const uint4 u = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(base) + at + 8 * h);
      const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[8 * h + 2 * e] += __uint_as_float(w[e] << 16);
        x[8 * h + 2 * e + 1] += __uint_as_float(w[e] & 0xffff0000u);
      }
    }
  }
}

// What a gradient's item does with 16 columns of its sums.
__device__ __forceinline__ void finish16(const Args& a, const Cut& t, int row, int col, float* x) {
  if (row >= a.plan.rows) return;
  const int n = a.plan.cols - col;
  if (a.plan.parts > 1) {
    store_row16(a.part, ((int64_t)t.part * a.plan.rows + row) * a.plan.cols + col, x, n, true, true);
    return;
  }
  const int64_t at = (int64_t)row * a.out_ld + col;
  if (a.accumulate) add_row16(a.out, at, x, n, a.out_f32);
  store_row16(a.out, at, x, n, a.out_f32, a.wide);
}

// 16 codes of one row, times its scale, as bf16 numbers: two chunks of 16 bytes.
template <bool E4M3>
__device__ __forceinline__ void decode16(const uint4& q, float s, uint32_t* w) {
  const uint32_t c[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float x[4];
    unpack4<E4M3>(c[i], x);
    w[2 * i] = pack_bf16x2_rn(x[0] * s, x[1] * s);
    w[2 * i + 1] = pack_bf16x2_rn(x[2] * s, x[3] * s);
  }
}

// An item's K in segments of even length: how many, and the stages of each but the last.
__device__ __forceinline__ void segments(int stages, int most, int& n, int& each) {
  n = (stages + most - 1) / most;
  each = (stages + n - 1) / n;
  n = (stages + each - 1) / each;
}

// Pairs of CTAs (cta_group::2), 256 x 256 tiles.  Warp 0 loads A, warp 2 loads B or the codes, warp 1 issues the MMAs, warps 4 to 11
// drain the accumulators; gradients have 8 more (LONG: 4) that turn codes into bf16 numbers.
// LONG: K in segments that the epilogue adds up in registers, because the tensor cores cut every partial sum off toward zero (a K step of 16 leaves
// an accumulator up to 2^-23 of itself too small).  For gradients in fp32, and for sums above 16384 terms.
template <int OP, bool LONG>
__global__ void __launch_bounds__(Shape<OP, LONG>::kThreads, 1) linear8_kernel(const __grid_constant__ Args a) {
  using S = Shape<OP, LONG>;
  extern __shared__ uint8_t dyn_smem[];
  __shared__ Shared<OP, LONG> sh;
  wait_for_previous_kernel();
  const uint32_t rank = cluster_rank();
  uint8_t* const ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(dyn_smem) + 1023) & ~(uintptr_t)1023);
  uint8_t* const raw = ring + S::kStages * kStageBytes;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, pair = (int)(blockIdx.x >> 1);
  volatile int* const abort = &sh.abort;
  int32_t* const status = a.status + pair;

  if (threadIdx.x == 0) {
    for (int i = 0; i < S::kStages; ++i) {
      mbar_init(&sh.full[i], S::kGrad ? 1 + 2 * S::kConvert : 2);
      mbar_init(&sh.empty[i], 1);
    }
    for (int i = 0; i < S::kRawStages; ++i) { mbar_init(&sh.raw_full[i], 1); mbar_init(&sh.raw_empty[i], S::kConvert); }
    for (int i = 0; i < 2; ++i) { mbar_init(&sh.tfull[i], 1); mbar_init(&sh.tempty[i], 16); }
    sh.abort = 0;
    if (rank == 0) *status = 0;                        // (the cluster barrier below orders it before what either CTA adds)
    mbar_fence_init();
  }
  if (blockIdx.x == 0)
    for (int i = a.pairs + (int)threadIdx.x; i < kMostWords; i += S::kThreads) a.status[i] = 0;      // words of no pair
  if (warp == 1) {
    tmem_alloc<true>(&sh.tmem_base, 512);
    tmem_relinquish<true>();
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();
  tc_fence_after();
  const uint32_t tmem_base = sh.tmem_base;
  Cut t;

  if (warp < 4) {
    if (LONG) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kLongIssue));
    if (warp == 0 || (warp == 2 && !S::kGrad)) {
      // ------------------------------------------------------------------ operands that are multiplied as they lie
      const bool leader = elect_one(), is_a = warp == 0;
      const uint32_t pair_full = uniform(shared_of(sh.full, 0));
      constexpr bool kAlongY = OP == WEIGHT_GRAD;      // rows are K: two boxes of 64 columns
      constexpr int kStep = OP == FORWARD ? 128 : 64;
      int stage = 0;
      uint32_t phase = 0, issued = 0;
      bool ok = true;
      for (int i = pair; ok && a.plan.item(i, t); i += a.pairs) {
        const CUtensorMap* const map = is_a ? &a.a : &a.b;
        const int mine = uniform(is_a ? t.m0 + (int)rank * 128 : t.n0 + (int)rank * (t.bn / 2));
        const int count = uniform(t.count);
        int k = uniform(t.k0) * kStep;
        for (int left = count; left > 0; --left, k += kStep) {
          if (!mbar_wait_warp<WAIT_PAIR>(&sh.empty[stage], phase ^ 1u, abort, status, ST_WAIT_EMPTY, kWaitSpinDefault)) { ok = false; break; }
          uint8_t* const dst = ring + stage * kStageBytes + (is_a ? 0 : kOperandBytes);
          if (leader) {
            if (rank == 0) mbar_arrive_expect_tx(&sh.full[stage], 2 * kOperandBytes);
            const uint32_t bar = pair_full + 8u * (uint32_t)stage;
            if (kAlongY) {
              tma_load_box_pair(dst, map, mine, k, bar);
              tma_load_box_pair(dst + kOperandBytes / 2, map, mine + 64, k, bar);
            } else {
              tma_load_box_pair(dst, map, k, mine, bar);
            }
          }
          __syncwarp();
          ++issued;
          if (++stage == S::kStages) { stage = 0; phase ^= 1u; }
        }
      }
      if (!ok) drain_ring<true>(sh.full, stage, phase, issued, S::kStages, rank);
    } else if (warp == 2) {
      // ------------------------------------------------------------------ codes, into a ring of their own
      const bool leader = elect_one();
      int stage = 0;
      uint32_t phase = 0, issued = 0;
      bool ok = true;
      for (int i = pair; ok && a.plan.item(i, t); i += a.pairs) {
        const int x = uniform(t.n0 + (int)rank * (t.bn / 2)), count = uniform(t.count);
        int y = uniform(t.k0) * 64;
        for (int left = count; left > 0; --left, y += 64) {
          if (!mbar_wait_warp(&sh.raw_empty[stage], phase ^ 1u, abort, status, ST_WAIT_EMPTY, kWaitSpinDefault)) { ok = false; break; }
          if (leader) {
            mbar_arrive_expect_tx(&sh.raw_full[stage], kRawBytes);
            tma_load_box(raw + stage * kRawBytes, &a.b, x, y, &sh.raw_full[stage]);
          }
          __syncwarp();
          ++issued;
          if (++stage == S::kRawStages) { stage = 0; phase ^= 1u; }
        }
      }
      if (!ok) drain_ring<false>(sh.raw_full, stage, phase, issued, S::kRawStages, rank);
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
        int left = uniform(t.count), n_seg = 1, each = left;
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
  } else if (S::kGrad && warp >= 12) {
    if (LONG) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kLongConvert));
    // ------------------------------------------------------------------ codes to bf16 numbers: a warp has four rows of K at a time,
    // eight lanes to a row, 16 codes to a lane
    constexpr int kPasses = S::kGrad ? 64 / (4 * (S::kConvert ? S::kConvert : 1)) : 1;
    const int row0 = 4 * (warp - 12) + (lane >> 3), j = lane & 7;
    const uint32_t pair_full = shared_of(sh.full, 0);
    int stage = 0, rs = 0;
    uint32_t phase = 0, raw_phase = 0;
    bool ok = true;
    for (int i = pair; ok && a.plan.item(i, t); i += a.pairs) {
      const int half = t.bn / 2, group = a.b_groups > 1 ? (t.n0 + (int)rank * half) / 128 : 0;
      const bool live = 16 * j < half && group < a.b_groups;
      const float* const scale = a.b_scale + group;
      int k = t.k0 * 64 + row0;
      float s[kPasses];
      auto scales = [&]() {
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
          const int at = k + p * 4 * S::kConvert;
          s[p] = live && at < a.k ? __ldg(scale + (int64_t)at * a.b_groups) : 0.f;
        }
      };
      scales();
      for (int left = t.count; left > 0; --left) {
        float now[kPasses];
#pragma unroll
        for (int p = 0; p < kPasses; ++p) now[p] = s[p];
        k += 64;
        if (left > 1) scales();                        // of the next stage
        if (!mbar_wait_warp(&sh.raw_full[rs], raw_phase, abort, status, ST_WAIT_FULL, kWaitSpinDefault)) { ok = false; break; }
        uint4 q[kPasses];
#pragma unroll
        for (int p = 0; p < kPasses; ++p) q[p] = *reinterpret_cast<const uint4*>(raw + rs * kRawBytes + (row0 + p * 4 * S::kConvert) * 128 + 16 * j);
        if (!mbar_wait_warp<WAIT_PAIR>(&sh.empty[stage], phase ^ 1u, abort, status, ST_WAIT_EMPTY, kWaitSpinDefault)) { ok = false; break; }
        uint8_t* const dst = ring + stage * kStageBytes + kOperandBytes + (j >> 2) * (kOperandBytes / 2);
        if (16 * j < half) {
#pragma unroll
          for (int p = 0; p < kPasses; ++p) {
            const int row = row0 + p * 4 * S::kConvert;
            uint32_t w[8];
            if (a.e4m3) decode16<true>(q[p], now[p], w);
            else decode16<false>(q[p], now[p], w);
            // the 128-byte swizzle; lanes 4 to 7 write their second chunk first, so that eight lanes meet no bank twice
            const int c = 2 * (j & 3), odd = j >> 2;
            uint8_t* const line = dst + row * 128;
            put4(line + ((c + odd) ^ (row & 7)) * 16, odd ? w + 4 : w);
            put4(line + ((c + 1 - odd) ^ (row & 7)) * 16, odd ? w : w + 4);
          }
        }
        fence_async_smem();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&sh.raw_empty[rs]);
          mbar_arrive_release_at(pair_full + 8u * (uint32_t)stage);
        }
        if (++rs == S::kRawStages) { rs = 0; raw_phase ^= 1u; }
        if (++stage == S::kStages) { stage = 0; phase ^= 1u; }
      }
    }
  } else {
    if (LONG) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kLongDrain));
    // ------------------------------------------------------------------ epilogue: a thread has one row of the tile and, by its
    // group of four warps, the lower or upper half of the columns
    const int q = 32 * (warp & 3) + lane, grp = (warp - 4) >> 2;
    const uint32_t lane_addr = (uint32_t)(32 * (warp & 3)) << 16;
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
      const int row = t.m0 + (int)rank * 128 + q, half = t.bn / 2, col0 = t.n0 + grp * half;
      if (LONG) {
        float v[128];
        int n_seg, each;
        segments(t.count, a.seg, n_seg, each);
#pragma unroll 1
        for (int s = 0; s < n_seg; ++s, ++run) {
          const int acc = (int)(run & 1);
          wait_full(acc);
          if (!ok) break;
          const uint32_t at = tmem_base + lane_addr + (uint32_t)(acc * kTile + grp * half);
          if (s == 0) {
#pragma unroll
            for (int c = 0; c < 128; c += 16)
              if (c < half) tmem_ld16(at + c, v + c);
            tmem_ld_wait();
          } else {
#pragma unroll
            for (int c = 0; c < 128; c += 32) {
              if (c < half) {
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
        for (int c = 0; c < 128; c += 16)
          if (c < half) finish16(a, t, row, col0 + c, v + c);
      } else {
        const int acc = (int)(run & 1);
        const float xs = OP == FORWARD && row < a.plan.rows ? a.a_scale[row] : 0.f;
        wait_full(acc);
        if (!ok) break;
        const uint32_t at = tmem_base + lane_addr + (uint32_t)(acc * kTile + grp * half);
#pragma unroll
        for (int c = 0; c < 128; c += 32) {
          if (c >= half) continue;
          __syncwarp();
          float v[32];
          tmem_ld16(at + c, v);
          tmem_ld16(at + c + 16, v + 16);
          tmem_ld_wait();
          if (c + 32 >= half) release(acc);
#pragma unroll
          for (int h = 0; h < 32; h += 16) {
            float* const x = v + h;
            const int col = col0 + c + h;
            if (OP == FORWARD) {
              const int n = a.plan.cols - col;
              if (row >= a.plan.rows || n <= 0) continue;
#pragma unroll
              for (int e = 0; e < 16; e += 4) {
                if (e >= n) continue;
                const float4 ws = __ldg(reinterpret_cast<const float4*>(a.b_scale + col + e));
                x[e] = (float)__float_as_int(x[e]) * xs * ws.x;
                x[e + 1] = (float)__float_as_int(x[e + 1]) * xs * ws.y;
                x[e + 2] = (float)__float_as_int(x[e + 2]) * xs * ws.z;
                x[e + 3] = (float)__float_as_int(x[e + 3]) * xs * ws.w;
              }
              store_row16(a.out, (int64_t)row * a.out_ld + col, x, n, a.out_f32, a.wide);
            } else {
              finish16(a, t, row, col, x);
            }
          }
        }
        ++run;
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  cluster_sync();      // neither CTA leaves while the other may still reach into it
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc<true>(tmem_base, 512);
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

// ---- host ----------------------------------------------------------------------------------------------------------

// A row-major matrix of bytes in boxes of 128 columns x box_rows rows, with the 128-byte swizzle or as it lies.
bool encode_bytes(CUtensorMap* out, const void* base, uint64_t rows, uint64_t cols, uint64_t pitch, uint32_t box_rows, bool swizzle) {
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

template <int OP, bool LONG>
int allow(int* resident, int sms) {
  using S = Shape<OP, LONG>;
  ADAPM_CUDA(cudaFuncSetAttribute(linear8_kernel<OP, LONG>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem));
  if (LONG) {
    cudaFuncAttributes fa;                  // (with fewer registers at launch the split above would wait for ever)
    ADAPM_CUDA(cudaFuncGetAttributes(&fa, linear8_kernel<OP, LONG>));
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
  ADAPM_CUDA(cudaOccupancyMaxActiveClusters(&n, linear8_kernel<OP, LONG>, &cfg));
  *resident = std::min(*resident, n);
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
    int rc = allow<FORWARD, false>(&n, sms);
    if (rc == ADAPM_OK) rc = allow<INPUT_GRAD, false>(&n, sms);
    if (rc == ADAPM_OK) rc = allow<INPUT_GRAD, true>(&n, sms);
    if (rc == ADAPM_OK) rc = allow<WEIGHT_GRAD, false>(&n, sms);
    if (rc == ADAPM_OK) rc = allow<WEIGHT_GRAD, true>(&n, sms);
    if (rc != ADAPM_OK) return rc;
    known[device] = std::max(1, n);
  }
  *pairs = known[device];
  return ADAPM_OK;
}

template <int OP, bool LONG>
cudaError_t launch(const Args& a, cudaStream_t s) {
  using S = Shape<OP, LONG>;
  return launch_clusters(true, 2, linear8_kernel<OP, LONG>, 2 * (unsigned)a.pairs, S::kThreads, S::kSmem, s, a);
}

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
  int rc = check_on_this_device({out.p, scratch}, device);
  for (const Buffer& b : in)
    if (rc == ADAPM_OK) rc = check_on_this_device({b.p}, device);
  return rc;
}

Buffer bf16_or_f32(const void* p, int64_t rows, int64_t ld, int64_t cols, int32_t dtype) { return Buffer{p, 16, matrix_at(p, rows, ld, cols, type_bytes(dtype))}; }
Buffer codes_at(const void* p, int64_t rows, int64_t ld, int64_t cols) { return Buffer{p, 16, matrix_at(p, rows, ld, cols, 1)}; }
Buffer floats_at(const float* p, int64_t n, int64_t align) { return Buffer{p, align, vector_at(p, n, 4)}; }

// A gradient: [rows, cols] = A [rows, K] (or its transpose) times codes [K, cols].
int gradient(const adapm_linear8& d, int32_t which, const void* dy, const void* codes, const float* scales, void* out, int32_t out_dtype, int64_t out_ld,
             void* scratch, const Plan& plan, int pairs, cudaStream_t s) {
  const bool weight = which == WEIGHT_GRAD;
  Args a;
  std::memset(&a, 0, sizeof(a));
  a.plan = plan;
  a.k = (int32_t)(weight ? d.tokens : d.out_features);
  const int64_t codes_ld = weight ? d.x8_ld : d.w8_ld;
  if (!encode_bf16_matrix(&a.a, dy, d.tokens, d.out_features, d.y_ld, weight ? 64 : 128) ||
      !encode_bytes(&a.b, codes, a.k, d.in_features, codes_ld, 64, false)) {
    set_error_text("cuTensorMapEncodeTiled failed for a gradient of linear8");
    return ADAPM_ECUDA;
  }
  a.b_scale = scales;
  a.b_groups = weight && d.x_group ? (int32_t)((d.in_features + 127) / 128) : 1;
  a.out = out; a.out_ld = out_ld;
  a.status = (int32_t*)scratch;
  a.part = (float*)((char*)scratch + kHeadBytes);
  a.out_f32 = out_dtype == ADAPM_TYPE_F32;
  a.wide = (uintptr_t)out % 32 == 0 && (a.out_f32 || out_ld % 16 == 0);
  a.accumulate = weight && d.accumulate != 0;
  a.e4m3 = weight && d.x_code == ADAPM_CODE_E4M3;
  a.pairs = std::min(pairs, plan.items);
  a.seg = a.out_f32 ? kSegLong : kSegShort;
  const bool is_long = a.out_f32 || plan.each > kShortStages;
  ADAPM_CUDA(weight ? (is_long ? launch<WEIGHT_GRAD, true>(a, s) : launch<WEIGHT_GRAD, false>(a, s))
                    : (is_long ? launch<INPUT_GRAD, true>(a, s) : launch<INPUT_GRAD, false>(a, s)));
  if (plan.parts == 1) return ADAPM_OK;
  SumArgs u;
  u.part = a.part; u.out = out; u.out_ld = out_ld; u.fours = plan.cols / 4; u.places = (int64_t)plan.rows * u.fours;
  u.part_elems = (int64_t)plan.rows * plan.cols; u.parts = plan.parts; u.f32 = a.out_f32; u.accumulate = a.accumulate;
  ADAPM_CUDA(launch_chained(true, linear8_sum_kernel, (unsigned)std::min<int64_t>((u.places + 255) / 256, 148 * 8), 256, 0, s, u));
  return ADAPM_OK;
}

}  // namespace
}  // namespace adapm

using namespace adapm;

extern "C" size_t adapm_linear8_scratch_bytes(const adapm_linear8* d, int32_t which) {
  if (!d || check_desc(*d, which) != ADAPM_OK) return 0;
  return (size_t)scratch_bytes(plan_of(*d, which));
}

extern "C" int adapm_linear8_forward(const adapm_linear8* d, const void* x8, const float* xs, const void* w8, const float* ws, void* y,
                                     void* scratch, size_t scratch_size, adapm_stream stream) {
  if (!d) return ADAPM_EINVAL;
  int rc = check_desc(*d, FORWARD);
  if (rc != ADAPM_OK || d->tokens == 0) return rc;
  const Plan plan = plan_of(*d, FORWARD);
  int device, pairs;
  rc = check_buffers({codes_at(x8, d->tokens, d->x8_ld, d->in_features), floats_at(xs, d->tokens, 4), codes_at(w8, d->out_features, d->w8_ld, d->in_features),
                      floats_at(ws, d->out_features, 16)},
                     bf16_or_f32(y, d->tokens, d->y_ld, d->out_features, d->y_dtype), scratch, scratch_size, scratch_bytes(plan),
                     "adapm_linear8_forward: the output or the scratch overlaps another buffer", &device);
  if (rc == ADAPM_OK) rc = pairs_of(device, &pairs);
  if (rc != ADAPM_OK) return rc;
  Args a;
  std::memset(&a, 0, sizeof(a));
  a.plan = plan;
  if (!encode_bytes(&a.a, x8, d->tokens, d->in_features, d->x8_ld, 128, true) || !encode_bytes(&a.b, w8, d->out_features, d->in_features, d->w8_ld, 128, true)) {
    set_error_text("cuTensorMapEncodeTiled failed for linear8");
    return ADAPM_ECUDA;
  }
  a.a_scale = xs; a.b_scale = ws; a.b_groups = 1; a.k = (int32_t)d->in_features;
  a.out = y; a.out_ld = d->y_ld; a.out_f32 = d->y_dtype == ADAPM_TYPE_F32;
  a.wide = (uintptr_t)y % 32 == 0 && (a.out_f32 || d->y_ld % 16 == 0);
  a.status = (int32_t*)scratch;
  a.pairs = std::min(pairs, plan.items);
  ADAPM_CUDA((launch<FORWARD, false>(a, (cudaStream_t)stream)));
  return ADAPM_OK;
}

extern "C" int adapm_linear8_input_grad(const adapm_linear8* d, const void* dy, const void* w8, const float* ws, void* dx, void* scratch,
                                        size_t scratch_size, adapm_stream stream) {
  if (!d) return ADAPM_EINVAL;
  int rc = check_desc(*d, INPUT_GRAD);
  if (rc != ADAPM_OK || d->tokens == 0) return rc;
  const Plan plan = plan_of(*d, INPUT_GRAD);
  int device, pairs;
  rc = check_buffers({bf16_or_f32(dy, d->tokens, d->y_ld, d->out_features, ADAPM_TYPE_BF16), codes_at(w8, d->out_features, d->w8_ld, d->in_features),
                      floats_at(ws, d->out_features, 4)},
                     bf16_or_f32(dx, d->tokens, d->dx_ld, d->in_features, d->dx_dtype), scratch, scratch_size, scratch_bytes(plan),
                     "adapm_linear8_input_grad: the output or the scratch overlaps another buffer", &device);
  if (rc == ADAPM_OK) rc = pairs_of(device, &pairs);
  if (rc != ADAPM_OK) return rc;
  return gradient(*d, INPUT_GRAD, dy, w8, ws, dx, d->dx_dtype, d->dx_ld, scratch, plan, pairs, (cudaStream_t)stream);
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
  const Plan plan = plan_of(*d, WEIGHT_GRAD);
  const int64_t groups = d->x_group ? (d->in_features + 127) / 128 : 1;
  rc = check_buffers({bf16_or_f32(dy, d->tokens, d->y_ld, d->out_features, ADAPM_TYPE_BF16), codes_at(x8, d->tokens, d->x8_ld, d->in_features),
                      floats_at(xs, d->tokens * groups, 4)},
                     bf16_or_f32(dweight, d->out_features, d->dweight_ld, d->in_features, d->dweight_dtype), scratch, scratch_size, scratch_bytes(plan),
                     "adapm_linear8_weight_grad: the output or the scratch overlaps another buffer", &device);
  if (rc == ADAPM_OK) rc = pairs_of(device, &pairs);
  if (rc != ADAPM_OK) return rc;
  return gradient(*d, WEIGHT_GRAD, dy, x8, xs, dweight, d->dweight_dtype, d->dweight_ld, scratch, plan, pairs, s);
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
