// Softmax cross entropy of a language model's output head, and its gradient, from the hidden states and the head's weight, in
// pieces of the vocabulary: neither the logits nor their gradient exist as a whole.
//
//   z = h W^T    lse_t = log sum_v exp z_tv    loss_t = lse_t - (1-e) z_ty - (e/V) sum_v z_tv + zl lse_t^2
//   g_tv = dloss_t [ p_tv (1 + 2 zl lse_t) - (1-e) [v = y_t] - e/V ],  p = exp(z - lse)
//   dh_t = scale sum_v g_tv W_v        dW_v = scale sum_t g_tv h_t
//
// One kernel (head_items_kernel) does all the products, on pairs of CTAs (tcgen05, cta_group::2, 256 x 256 tiles of the
// result, K = 64 per stage) with the softmax in its epilogue; its items are
//   logits -> partial (max, sum) of a row over 128 columns         forward
//   logits -> g, rounded, into one of two buffers of a piece       backward, piece i + 1
//   g W and g^T h -> dh (summed over the pieces in fp32) and dW    backward, piece i, in the same launch
// The three kinds of items of a launch do not depend on one another, so that the many short logits items fill what the long
// ones of the two gradients leave at the end.  Tokens without a target are taken out first (head_prepare_kernel): no product is made
// for them, and whatever their hidden states hold (a padded batch's may be NaN) reaches neither gradient.  A forward call of at most
// a tile of tokens leaves them in: no row's loss depends on another row, and theirs are replaced at the end.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <mutex>

#include "head_plan.h"
#include "op_checks.h"
#include "tc_engine.cuh"
#include "tc_host.h"

namespace adapm {
namespace {

using namespace head;
using namespace tc;

constexpr int kHeadThreads = 384;            // warp 0 loads A, 2 loads B, 1 issues the MMAs, 4-11 drain the accumulators
// Registers per thread: of the launch, and as the first four and the other eight warps divide them (the eight keep 128 values each).
constexpr int kHeadRegs = 168, kIssueRegs = 88, kDrainRegs = 208;
static_assert(4 * kIssueRegs + 8 * kDrainRegs <= 12 * kHeadRegs, "a block has the registers that it was launched with");
constexpr int kOperandBytes = 128 * kStageK * 2;        // of one CTA and stage: 128 rows or columns of A, as many of B
constexpr int kHeadStages = 6;
constexpr int kHeadSmem = kHeadStages * 2 * kOperandBytes + 1024;
constexpr float kLog2e = 1.4426950408889634f;
// The tensor cores cut every partial sum off toward zero (a K step of 16 leaves an accumulator up to 2^-23 of itself too small),
// so that a long sum shrinks with its length: with the whole K in one accumulator an fp32 gradient was off by 1.3e-5 at K = 12288
// (three planes of 4096) and by 2e-3 at K = 234222.  An item's K is therefore cut into segments, which the epilogue adds up in
// registers, rounded to nearest; the next segment runs meanwhile in the other accumulator.
constexpr int kSegForward = 8, kSegF32 = 4, kSegBf16 = 64;      // stages of 64 K: for the losses, for gradients in fp32 and in bf16

struct HeadArgs {
  CUtensorMap hk, hn, ck, cn, wk, wn, gk, gn;      // hidden, its compacted copy, weight, g; boxes of 64 x 128 (K-major use) and 64 x 64
  int32_t* head;                 // HD_*
  const Walk* walk;              // of this launch, on the device; null: own_walk
  Walk own_walk;
  const int32_t* token;          // of a compacted row
  const int32_t* target;         // of a compacted row
  const int64_t* targets;        // forward over at most a tile of tokens, which are not compacted: the caller's (else null)
  const float* lse;              // of a compacted row
  const float* dloss;            // of a compacted row, or null: 1
  float2* part;                  // forward: (exponent, sum) [2 n_tiles][t_pad]
  float* part_sum;               // forward with smoothing: sum of the logits, same layout
  float* z_target;               // forward: logit of the target of a compacted row
  uint16_t* g;                   // [2 buffers][g_rows][piece]: the planes of the walk one behind the other
  float* dh_acc;                 // [split_dh][t_pad][hidden], between two pieces and before the splits (and planes) are added up
  float* dw_acc;                 // [split_dw][vocab][hidden], before the splits are added up
  void* dh;
  void* dw;
  int64_t hidden_ld, weight_ld;
  int32_t tokens, vocab, hidden, t_pad, piece, g_rows;
  int32_t g_begin, g_cols, g_buf;          // piece whose g this launch makes (g_cols = 0: none)
  int32_t o_begin, o_cols, o_buf;          // piece whose gradients it makes (o_cols = 0: none)
  int32_t first, last;                     // of the pieces, for dh
  int32_t split_dh, split_dw;              // parts that K is cut into, at most; 1: not cut
  int32_t dh_f32, dw_f32, accumulate, dh_wide, dw_wide;      // wide: rows start on 32 bytes
  int32_t seg_logits, seg_dh, seg_dw;      // longest segments, in stages
  float scale, smooth, z_loss;
};

struct __align__(8) HeadShared {
  uint64_t full[kHeadStages], empty[kHeadStages], tfull[2], tempty[2];
  uint32_t tmem_base;
  int abort, skip;
  Walk walk;                     // here and not in every thread's registers
};

// Two fp32 operations per instruction (the same roundings as one at a time).
__device__ __forceinline__ void fma2(float& d0, float& d1, float a0, float a1, float b, float c) {
  asm("{\n.reg .b64 x, y, z, w;\nmov.b64 x, {%2, %3};\nmov.b64 y, {%4, %4};\nmov.b64 z, {%5, %5};\nfma.rn.f32x2 w, x, y, z;\nmov.b64 {%0, %1}, w;\n}"
      : "=f"(d0), "=f"(d1) : "f"(a0), "f"(a1), "f"(b), "f"(c));
}
__device__ __forceinline__ void add2(float& d0, float& d1, float a0, float a1) {
  asm("{\n.reg .b64 x, y, z;\nmov.b64 x, {%0, %1};\nmov.b64 y, {%2, %3};\nadd.rn.f32x2 z, x, y;\nmov.b64 {%0, %1}, z;\n}"
      : "+f"(d0), "+f"(d1) : "f"(a0), "f"(a1));
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ void st_b32x4(void* p, const uint32_t* v) {
  *reinterpret_cast<uint4*>(p) = make_uint4(v[0], v[1], v[2], v[3]);
}

// 16 values of one row of a gradient, of which those below n (a multiple of 8) exist: as fp32 or bf16, to addresses that are
// multiples of 32 (wide) or 16 bytes.
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
    if (n > 0) st_b32x4(p, w);
    if (n > 8) st_b32x4(p + 8, w + 4);
  }
}
__device__ __forceinline__ void load_row16(const void* base, int64_t at, float* x, int n, bool f32) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if (8 * h >= n) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[8 * h + e] = 0.f;
    } else if (f32) {
      const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(base) + at + 8 * h);
      const float4 u = __ldcg(p), v = __ldcg(p + 1);
      x[8 * h] = u.x; x[8 * h + 1] = u.y; x[8 * h + 2] = u.z; x[8 * h + 3] = u.w;
      x[8 * h + 4] = v.x; x[8 * h + 5] = v.y; x[8 * h + 6] = v.z; x[8 * h + 7] = v.w;
    } else {
      const uint4 u = __ldcg(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(base) + at + 8 * h));
      const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[8 * h + 2 * e] = __uint_as_float(w[e] << 16);
        x[8 * h + 2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
      }
    }
  }
}

// An item's K in segments of even length: how many, and the stages of each but the last.
__device__ __forceinline__ void segments(int stages, int most, int& n, int& each) {
  n = (stages + most - 1) / most;
  each = (stages + n - 1) / n;
  n = (stages + each - 1) / each;
}

// `half` columns of this thread's row of an accumulator: v = them, or v += them.
__device__ __forceinline__ void take(uint32_t taddr, int half, float* v) {
#pragma unroll
  for (int c = 0; c < 128; c += 16)
    if (c < half) tmem_ld16(taddr + c, v + c);
  tmem_ld_wait();
}
__device__ __forceinline__ void take_add(uint32_t taddr, int half, float* v) {
#pragma unroll
  for (int c = 0; c < 128; c += 32) {
    if (c < half) {
      float t[32];
      tmem_ld16(taddr + c, t);
      if (c + 16 < half) tmem_ld16(taddr + c + 16, t + 16);
      tmem_ld_wait();
#pragma unroll
      for (int e = 0; e < 16; e += 2) add2(v[c + e], v[c + e + 1], t[e], t[e + 1]);
      if (c + 16 < half) {
#pragma unroll
        for (int e = 16; e < 32; e += 2) add2(v[c + e], v[c + e + 1], t[e], t[e + 1]);
      }
    }
  }
}

// v[y] for a y that the compiler does not know.
__device__ __forceinline__ float pick(const float* v, int y) {
  float x = 0.f;
#pragma unroll
  for (int c = 0; c < 128; c += 16) {
    if ((unsigned)(y - c) < 16u) {
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (y - c == e) x = v[c + e];
    }
  }
  return x;
}

// The sum of exp over 128 logits of a row is made as sum * 2^k, k a whole number: z log2(e) - k is then one multiply-add with one
// rounding, and the sums of different columns are scaled by powers of two only.  k is the greatest of the first 16 logits in
// base 2: any k near the greatest one does, and one that is known early lets the maxima be found beside the exponentials.
// Where the exponential of a logit is above 2^(k + 64) after all, or all 16 are -inf, the sum is made again with the greatest of
// all.  NaN and +inf logits make the sum NaN.
__device__ __forceinline__ float exponent_of(float top) { return fmaxf(-INFINITY, rintf(top * kLog2e)); }      // (NaN: -inf)
__device__ __forceinline__ void sum_exponentials(const float* z, float shift, float* s) {
  s[0] = s[1] = s[2] = s[3] = 0.f;
#pragma unroll
  for (int e = 0; e < 128; e += 2) {
    float p0, p1;
    fma2(p0, p1, z[e], z[e + 1], kLog2e, -shift);
    add2(s[e & 2], s[(e & 2) + 1], ex2(p0), ex2(p1));
  }
}
template <int FROM, int TO>
__device__ __forceinline__ float greatest(const float* z) {
  float top[4] = {z[FROM], z[FROM + 1], z[FROM + 2], z[FROM + 3]};
#pragma unroll
  for (int e = FROM + 4; e < TO; ++e) top[e & 3] = fmaxf(top[e & 3], z[e]);
  return fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
}
// Columns from n on count as -inf; returns the sum of the others.
__device__ __forceinline__ float cut_row(float* z, int n) {
  float t = 0.f;
#pragma unroll
  for (int e = 0; e < 128; ++e) {
    if (e < n) t += z[e];
    else z[e] = -INFINITY;
  }
  return t;
}

// What bounds it: the tensor cores, and with them the power cap, where there are a few hundred tokens or more.  8192 x 50257 x 1600
// forward 0.95 ms = 1.38 PFLOP/s (cuBLAS sustains 1.38 on this card, 1.62 in a burst), both gradients 3.25 to 3.4 ms = 1.16 to
// 1.22, with half the tokens of 8192 x 128256 x 4096 10.0 to 10.3 ms = 1.25 to 1.29; tensor pipe 82 % active in the forward
// launch, 76 to 78 % in those of the gradients, DRAM 10 and 30 %.  With few tokens the weight's way from memory and back (100 tokens of
// 128256 x 4096: both gradients 0.98 ms for 3.2 GB), and below a few ten microseconds the launches themselves.  With D = 256 the
// exponentials: a tile of 256 x 256 is multiplied in 2 thousand cycles, and its epilogue takes 4 (2 of them the pipe that
// makes 16 exponentials a cycle).
// Not kept: an epilogue that reads the accumulator column by column as it goes (smaller code, but its multiply-segment form
// spilled: 1150 us forward against 955); rows turned in shared memory so that stores cover 64 bytes of a row (no change for
// bf16, 49 against 43 us on 512 tokens in fp32).
template <bool BACKWARD>
__global__ void __launch_bounds__(kHeadThreads, 1) head_items_kernel(const __grid_constant__ HeadArgs a) {
  extern __shared__ uint8_t dyn_smem[];
  __shared__ HeadShared sh;
  wait_for_previous_kernel();
  const uint32_t rank = cluster_rank();
  uint8_t* const stages = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(dyn_smem) + 1023) & ~(uintptr_t)1023);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  volatile int* const abort = &sh.abort;
  // forward: a word of this pair's own, so that nothing has to be cleared before the launch
  int32_t* const status = a.head + (BACKWARD ? HD_STATUS : HD_PAIRS + (int)(blockIdx.x >> 1));

  if (threadIdx.x == 0) {
    for (int i = 0; i < kHeadStages; ++i) {
      mbar_init(&sh.full[i], 2);                    // A and B, those of rank 0 for both CTAs
      mbar_init(&sh.empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) { mbar_init(&sh.tfull[i], 1); mbar_init(&sh.tempty[i], 16); }
    sh.abort = 0;
    if (!BACKWARD && rank == 0) *status = 0;          // (the cluster barrier below orders it before what either CTA adds)
    sh.skip = BACKWARD && *reinterpret_cast<volatile int32_t*>(status) != 0;
    mbar_fence_init();
  }
  if (threadIdx.x >= 64 && threadIdx.x < 64 + sizeof(Walk) / 4)
    reinterpret_cast<int*>(&sh.walk)[threadIdx.x - 64] = reinterpret_cast<const int*>(a.walk ? a.walk : &a.own_walk)[threadIdx.x - 64];
  if (warp == 1) {
    tmem_alloc<true>(&sh.tmem_base, 512);
    tmem_relinquish<true>();
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();
  tc_fence_after();
  const uint32_t tmem_base = sh.tmem_base;
  const bool skip = load_shared_of(&sh.skip, 0) != 0;       // an earlier launch gave up: the pair decides together
  const int tv = uniform(sh.walk.tv), pair = (int)(blockIdx.x >> 1);
  const bool compacted = tv != a.tokens;
  const Walk& walk = sh.walk;
  HeadItem t;

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kIssueRegs));
    if (skip) {
      // nothing
    } else if (warp == 0 || warp == 2) {
      // ------------------------------------------------------------------ producers (all lanes run, one issues)
      const bool leader = elect_one(), is_a = warp == 0;
      const uint32_t pair_full = uniform(shared_of(sh.full, 0));
      int stage = 0;
      uint32_t phase = 0, issued = 0;
      bool ok = true;
      const int plane_rows = uniform(walk.plane_rows);          // (read anew for every item: 100 x 128256 x 4096 988 us for 971)
      for (int seq = 0; ok && walk.item_uniform<BACKWARD>(pair, seq, t); ++seq) {
        const CUtensorMap* map;
        int x, y, n_box = 1;                 // K-major: one box of 128 rows, x runs; MN-major: boxes of 64 columns, y runs
        const int half = t.bn / 2, o_row = a.o_buf * a.g_rows;
        if (is_a) {
          if (t.cls == CLS_DW) { map = &a.gn; x = t.m0 + (int)rank * 128; y = o_row; n_box = 2; }
          else if (t.cls == CLS_DH) { map = &a.gk; x = 0; y = o_row + t.m0 + (int)rank * 128; }
          else { map = compacted ? &a.ck : &a.hk; x = 0; y = t.m0 + (int)rank * 128; }
        } else {
          if (t.cls == CLS_LOGITS) { map = &a.wk; x = 0; y = (BACKWARD ? a.g_begin : 0) + t.n0 + (int)rank * 128; }
          else {
            map = t.cls == CLS_DH ? &a.wn : (compacted ? &a.cn : &a.hn);
            x = t.n0 + (int)rank * half; y = t.cls == CLS_DH ? a.o_begin : 0; n_box = half > 64 ? 2 : 1;
          }
        }
        const bool along_y = is_a ? t.cls == CLS_DW : t.cls != CLS_LOGITS;
        const uint32_t bytes = along_y ? (uint32_t)n_box * (kOperandBytes / 2) : kOperandBytes;
        const int plane_step = is_a && t.cls != CLS_LOGITS ? plane_rows : 0;
        const int plane0 = t.k0 / t.per_plane, kx = along_y ? 0 : kStageK, ky = along_y ? kStageK : 0;
        int k = t.k0 - plane0 * t.per_plane;
        y += plane0 * plane_step + k * ky;
        x += k * kx;
        for (int left = t.count; left > 0; --left) {
          if (!mbar_wait_warp<WAIT_PAIR>(&sh.empty[stage], phase ^ 1u, abort, status, ST_WAIT_EMPTY, kWaitSpinDefault)) { ok = false; break; }
          uint8_t* const dst = stages + stage * (2 * kOperandBytes) + (is_a ? 0 : kOperandBytes);
          if (leader) {
            if (rank == 0) mbar_arrive_expect_tx(&sh.full[stage], 2 * bytes);
            const uint32_t bar = pair_full + 8u * (uint32_t)stage;
            tma_load_box_pair(dst, map, x, y, bar);
            if (n_box == 2) tma_load_box_pair(dst + kOperandBytes / 2, map, x + 64, y, bar);
          }
          __syncwarp();
          x += kx;
          y += ky;
          if (++k == t.per_plane) {                 // the next plane of A, the same B again
            k = 0;
            x -= kx * t.per_plane;
            y += plane_step - ky * t.per_plane;
          }
          ++issued;
          if (++stage == kHeadStages) { stage = 0; phase ^= 1u; }
        }
      }
      if (!ok) drain_ring<true>(sh.full, stage, phase, issued, kHeadStages, rank);
    } else if (warp == 1 && rank == 0) {
      // ------------------------------------------------------------------ MMA issuer (all lanes run, one issues)
      const bool leader = elect_one();
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      const uint32_t ring = uniform(smem_u32(stages)), d0 = uniform(tmem_base), dhi = desc_hi();
      uint32_t run = 0;                     // segments so far
      for (int seq = 0; ok && walk.item_uniform<BACKWARD>(pair, seq, t); ++seq) {
        const bool a_mn = t.cls == CLS_DW, b_mn = t.cls != CLS_LOGITS;
        const uint32_t idesc = uniform(make_idesc(t.bn, a_mn, b_mn, false, 256));
        // per K step of 16: 32 bytes inside a K-major row, 16 rows of 128 bytes of an MN-major box (in 16-byte units)
        const uint32_t a_step = a_mn ? 128u : 2u, b_step = b_mn ? 128u : 2u;
        int left = t.count, n_seg, each;
        segments(left, t.cls == CLS_LOGITS ? a.seg_logits : t.cls == CLS_DH ? a.seg_dh : a.seg_dw, n_seg, each);
        for (; left > 0 && ok; left -= each, ++run) {
          const int acc = (int)(run & 1);
          if (!mbar_wait_warp<WAIT_PAIR_TC>(&sh.tempty[acc], ((run >> 1) & 1u) ^ 1u, abort, status, ST_WAIT_TMEM_EMPTY, kWaitSpinDefault)) { ok = false; break; }
          tc_fence_after();
          const uint32_t d = d0 + (uint32_t)(acc * kTile);
          uint32_t accumulate = 0;
          for (int i = min(each, left); i > 0; --i) {
            if (!mbar_wait_warp<WAIT_PAIR>(&sh.full[stage], phase, abort, status, ST_WAIT_FULL, kWaitSpinDefault)) { ok = false; break; }
            tc_fence_after();
            const uint32_t slot = ring + (uint32_t)(stage * 2 * kOperandBytes);
            const uint32_t alo = desc_lo(slot, a_mn ? kOperandBytes / 2 : 16u);
            const uint32_t blo = desc_lo(slot + kOperandBytes, b_mn ? kOperandBytes / 2 : 16u);
            if (leader) {
#pragma unroll
              for (int q = 0; q < kStageK / 16; ++q)
                mma_bf16<true>(d, desc_join(alo + q * a_step, dhi), desc_join(blo + q * b_step, dhi), idesc, q ? 1u : accumulate);
              mma_commit<true>(&sh.empty[stage]);
            }
            __syncwarp();
            accumulate = 1;
            if (++stage == kHeadStages) { stage = 0; phase ^= 1u; }
          }
          if (ok && leader) mma_commit<true>(&sh.tfull[acc]);
          __syncwarp();
        }
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kDrainRegs));
    // ------------------------------------------------------------------ epilogue: a thread has one row of the tile and, by its
    // group of four warps, the lower or upper half of the columns, all of them in registers
    const int q = 32 * (warp & 3) + lane, grp = (warp - 4) >> 2;
    const uint32_t lane_addr = (uint32_t)(32 * (warp & 3)) << 16;
    uint32_t run = 0;
    bool ok = true;
    // what a row needs is asked for an item ahead
    struct Row { int y, token; float lse, dl; };
    auto fetch = [&](const HeadItem& t) {
      Row r = {-1, 0, 0.f, 0.f};
      const int row = t.m0 + (int)rank * 128 + q;
      if (row >= tv) return r;
      if (t.cls == CLS_LOGITS) {
        if (!BACKWARD && a.targets) {
          const int64_t wide_y = a.targets[row];
          r.y = wide_y >= 0 && wide_y < a.vocab ? (int)wide_y : -(1 << 30);
        } else {
          r.y = a.target[row];
        }
        if (BACKWARD) {
          r.lse = a.lse[row];
          r.dl = a.dloss ? a.dloss[row] : 1.f;
        }
      } else if (BACKWARD && t.cls == CLS_DH && a.last && a.split_dh == 1) {
        r.token = a.token[row];
      }
      return r;
    };
    bool more = !skip && walk.item<BACKWARD>(pair, 0, t);
    Row here = {-1, 0, 0.f, 0.f};
    if (more) here = fetch(t);
    for (int seq = 1; more; ++seq) {
      const int cls = t.cls, m0 = t.m0, n0 = t.n0, split = t.split, count = t.count;
      const int row = m0 + (int)rank * 128 + q, half = t.bn / 2;
      const Row now = here;
      more = walk.item<BACKWARD>(pair, seq, t);
      if (more) here = fetch(t);
      const int y = row < tv ? now.y - (BACKWARD ? a.g_begin : 0) - n0 - 128 * grp : -1, token = now.token;
      const float lse = now.lse, dl = now.dl;
      float v[128];
      int n_seg, each;
      segments(count, cls == CLS_LOGITS ? a.seg_logits : cls == CLS_DH ? a.seg_dh : a.seg_dw, n_seg, each);
#pragma unroll 1
      for (int i = 0; i < n_seg; ++i, ++run) {
        const int acc = (int)(run & 1);
        if (lane == 0) ok = mbar_wait<WAIT_PAIR_TC>(&sh.tfull[acc], (run >> 1) & 1u, abort, status, ST_WAIT_TMEM_FULL, kWaitSpinDefault);
        ok = __shfl_sync(0xffffffffu, ok, 0);
        if (!ok) break;
        tc_fence_after();
        const uint32_t at = tmem_base + lane_addr + (uint32_t)(acc * kTile + grp * half);
        if (i > 0) take_add(at, half, v);
        else take(at, half, v);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_relaxed_at(shared_of(&sh.tempty[acc], 0));
      }
      if (!ok) break;
      if (!BACKWARD) {
        const int n = min(128, a.vocab - n0 - 128 * grp);
        if ((unsigned)y < 128u && y < n) a.z_target[row] = pick(v, y);
        float total = 0.f, s[4];
        if (n < 128) {
          total = cut_row(v, n);
        } else if (a.smooth != 0.f) {
          float t[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int e = 0; e < 128; e += 2) add2(t[e & 2], t[(e & 2) + 1], v[e], v[e + 1]);
          total = (t[0] + t[1]) + (t[2] + t[3]);
        }
        float k = exponent_of(greatest<0, 16>(v));
        sum_exponentials(v, k == -INFINITY ? 0.f : k, s);
        const float all = exponent_of(greatest<16, 128>(v));
        if (all > k && (all > k + 64.f || k == -INFINITY)) {
          k = all;
          sum_exponentials(v, k, s);
        }
        const float sum = (s[0] + s[1]) + (s[2] + s[3]);
        if (row < tv) {
          const int64_t at = (int64_t)(n0 / 128 + grp) * a.t_pad + row;
          a.part[at] = make_float2(k, sum);
          if (a.smooth != 0.f) a.part_sum[at] = total;
        }
      } else if (cls == CLS_LOGITS) {
        if (m0 + (int)rank * 128 + 32 * (warp & 3) >= ((tv + kStageK - 1) & -kStageK)) continue;      // rows that nothing reads
        // p = exp(z - lse) = 2^(z log2(e) - k) 2^(k - lse log2(e)) with k whole: the first exponent is one multiply-add
        // with one rounding, the second factor belongs to the row
        const float k = rintf(lse * kLog2e);
        const float rest = fmaf(lse, kLog2e, -k) + lse * (float)(1.44269504088896340736 - (double)kLog2e);
        const float up = dl * ex2(-rest) * fmaf(2.f * a.z_loss, lse, 1.f);
        const float down = dl * (a.smooth / (float)a.vocab), at_y = dl * (1.f - a.smooth);
        const int n = row < tv ? a.vocab - a.g_begin - n0 - 128 * grp : 0;            // columns that exist
        uint16_t* const dst = a.g + ((int64_t)a.g_buf * a.g_rows + row) * a.piece + n0 + 128 * grp;
        const int planes = walk.planes;
        const int64_t plane = (int64_t)walk.plane_rows * a.piece;
#pragma unroll
        for (int c = 0; c < 128; c += 16) {
          float* const z = v + c;
#pragma unroll
          for (int e = 0; e < 16; e += 2) {
            float p0, p1;
            fma2(p0, p1, z[e], z[e + 1], kLog2e, -k);
            fma2(z[e], z[e + 1], ex2(p0), ex2(p1), up, -down);
          }
          if ((unsigned)(y - c) < 16u) {
#pragma unroll
            for (int e = 0; e < 16; ++e)
              if (y - c == e) z[e] -= at_y;
          }
          if (c + 16 > n) {
#pragma unroll
            for (int e = 0; e < 16; ++e)
              if (c + e >= n) z[e] = 0.f;
          }
          // g in bf16 (off by 2^-8 of itself at most, like the gradients it makes), or as the sum of two bf16 numbers (2^-16), or,
          // where a gradient is wanted in fp32, of three, which have its 24 bits
          for (int p = 0;;) {
            uint32_t w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = pack_bf16x2_rn(z[2 * e], z[2 * e + 1]);
            st_b32x8(dst + p * plane + c, w);
            if (++p == planes) break;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              z[2 * e] -= __uint_as_float(w[e] << 16);
              z[2 * e + 1] -= __uint_as_float(w[e] & 0xffff0000u);
            }
          }
        }
      } else {
        const int col0 = n0 + grp * half;
        const bool is_dh = cls == CLS_DH;
        const bool stacked = is_dh && walk.stacked;
        const bool row_ok = row < (stacked ? 2 * kFewTokens : is_dh ? tv : a.o_cols), none = tv == 0;
        const bool cut = is_dh ? stacked || a.split_dh > 1 : a.split_dw > 1;
        const bool to_acc = cut || (is_dh && !a.last), from_acc = is_dh && !a.first, from_out = !to_acc && !is_dh && a.accumulate;
        const int64_t out_row = is_dh ? (int64_t)token * a.hidden_ld : (int64_t)(a.o_begin + row) * a.weight_ld;
        float* const acc_row = is_dh ? a.dh_acc + ((int64_t)split * a.t_pad + row) * a.hidden : a.dw_acc + ((int64_t)split * a.vocab + row) * a.hidden;
        // where the result goes, and where what it is added to comes from
        const bool to_f32 = to_acc || (is_dh ? a.dh_f32 : a.dw_f32), with_old = from_acc || from_out;
        void* const to = to_acc ? (void*)acc_row : to_f32 ? (void*)(static_cast<float*>(is_dh ? a.dh : a.dw) + out_row)
                                                          : (void*)(static_cast<uint16_t*>(is_dh ? a.dh : a.dw) + out_row);
        const bool wide = to_acc || (is_dh ? a.dh_wide : a.dw_wide);
        const float scale = to_acc ? 1.f : a.scale, old_scale = from_acc ? scale : 1.f;
#pragma unroll
        for (int c = 0; c < 128; c += 16) {
          if (c < half) {
            const int n = row_ok ? a.hidden - col0 - c : 0;
            float* const x = v + c;
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] = none ? 0.f : x[e] * scale;
            if (with_old) {
              float old[16];
              load_row16(from_acc ? acc_row : to, col0 + c, old, n, from_acc || to_f32);
#pragma unroll
              for (int e = 0; e < 16; ++e) x[e] = fmaf(old[e], old_scale, x[e]);
            }
            store_row16(to, col0 + c, x, n, to_f32, wide);
          }
        }
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

// ---- tokens with a target ----------------------------------------------------------------------------

struct PrepareArgs {
  const int64_t* targets;
  const uint16_t* hidden;
  uint16_t* compact;             // [t_pad][width]
  int32_t* head;
  int32_t* token;
  int32_t* target;
  const float* lse_in; float* lse;          // backward
  const float* dloss_in; float* dloss;      // backward, may be null
  float* loss; float* lse_out;              // forward: what tokens without a target get
  void* dh;                                 // backward: its rows of tokens without a target become zero; may be null
  Walk* walks;                   // of the launches that follow
  Plan plan;
  int64_t hidden_ld, ignore;
  int32_t tokens, vocab, width, per_cta, dh_f32, n_walks;
};

// Every CTA counts the targets of all tokens (8 bytes each, from L2; cheaper than a second launch: 4 us for 8192 tokens, all of it
// latency), then writes what belongs to
// its own ones: the row number among those with a target, the copies that the products read, the answers of the others.
__global__ void __launch_bounds__(256) head_prepare_kernel(const PrepareArgs a) {
  __shared__ int counts[2][8];
  __shared__ int at[256];
  wait_for_previous_kernel();
  const int begin = (int)blockIdx.x * a.per_cta, end = min(a.tokens, begin + a.per_cta);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  auto has_target = [&](int64_t y) { return y != a.ignore && y >= 0 && y < a.vocab; };
  int before = 0, all = 0;
#pragma unroll 4
  for (int t = threadIdx.x; t < a.tokens; t += 256) {
    const int v = has_target(a.targets[t]) ? 1 : 0;
    all += v;
    before += t < begin ? v : 0;
  }
  before = __reduce_add_sync(0xffffffffu, before);
  all = __reduce_add_sync(0xffffffffu, all);
  if (lane == 0) { counts[0][warp] = before; counts[1][warp] = all; }
  __syncthreads();
  before = all = 0;
  for (int w = 0; w < 8; ++w) { before += counts[0][w]; all += counts[1][w]; }
  if (blockIdx.x == 0 && threadIdx.x == 0) { a.head[HD_STATUS] = 0; a.head[HD_COUNT] = all; }
  for (int i = (int)(gridDim.x - 1 - blockIdx.x) * 256 + (int)threadIdx.x; i < a.n_walks; i += (int)gridDim.x * 256) a.walks[i].make(a.plan, i, all);
  const bool copy = all != a.tokens;
  const int vec = a.width >> 3;
  for (int t0 = begin; t0 < end; t0 += 256) {
    const int t = t0 + (int)threadIdx.x;
    const int64_t y = t < end ? a.targets[t] : a.ignore;
    const bool valid = t < end && has_target(y);
    const unsigned votes = __ballot_sync(0xffffffffu, valid);
    __syncthreads();                              // (counts and at of the round before have been read)
    if (lane == 0) counts[0][warp] = __popc(votes);
    __syncthreads();
    int row = before + __popc(votes & ((1u << lane) - 1));
    for (int w = 0; w < 8; ++w) {
      if (w < warp) row += counts[0][w];
      before += counts[0][w];
    }
    at[threadIdx.x] = valid ? row : -1;
    if (valid) {
      a.token[row] = t;
      a.target[row] = (int32_t)y;
      if (a.lse_in) a.lse[row] = a.lse_in[t];
      if (a.dloss_in) a.dloss[row] = a.dloss_in[t];
    } else if (t < end && a.loss) {
      const float x = y == a.ignore ? 0.f : __int_as_float(0x7fffffff);
      a.loss[t] = x;
      a.lse_out[t] = x;
    }
    __syncthreads();
    for (int i = warp; i < min(256, end - t0); i += 8) {
      const int r = at[i];
      const int64_t src_row = (int64_t)(t0 + i) * a.hidden_ld;
      if (r >= 0 && copy) {
        const uint4* src = reinterpret_cast<const uint4*>(a.hidden + src_row);
        uint4* dst = reinterpret_cast<uint4*>(a.compact + (int64_t)r * a.width);
#pragma unroll 4
        for (int v = lane; v < vec; v += 32) dst[v] = src[v];
      } else if (r < 0 && a.dh) {
        uint4* dst = reinterpret_cast<uint4*>(a.dh_f32 ? (void*)(static_cast<float*>(a.dh) + src_row) : (void*)(static_cast<uint16_t*>(a.dh) + src_row));
        for (int v = lane; v < (a.dh_f32 ? 2 * vec : vec); v += 32) dst[v] = make_uint4(0, 0, 0, 0);
      }
    }
  }
  // the last stage of a product over the tokens reads whole groups of 64 rows
  if (copy && blockIdx.x == gridDim.x - 1) {
    const int64_t stop = ((int64_t)max(all, 1) + 63) / 64 * 64 * vec;
    for (int64_t v = (int64_t)all * vec + threadIdx.x; v < stop; v += 256) reinterpret_cast<uint4*>(a.compact)[v] = make_uint4(0, 0, 0, 0);
  }
}

// ---- what the forward items left of a row, put together ------------------------------------------------

struct FinalArgs {
  int32_t* head;
  const int32_t* token;
  const int64_t* targets;        // tokens that were not compacted: the caller's (else null)
  const float2* part;
  const float* part_sum;
  const float* z_target;
  float* loss;
  float* lse;
  int64_t ignore;
  int32_t n_parts, t_pad, tokens, vocab, pairs;
  float smooth, z_loss;
};

// A CTA has 32 rows (its lanes), eight warps share the parts of each, eight at a time (one after the other, each with its own
// rescaling: 20 us for 8192 tokens of 50257 columns, 8 now; 8 bytes per 128 columns are read).
__global__ void __launch_bounds__(256) head_final_kernel(const FinalArgs a) {
  __shared__ float ks[8][32], sums[8][32], totals[8][32];
  wait_for_previous_kernel();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, row = (int)blockIdx.x * 32 + lane;
  const int tv = a.targets ? a.tokens : a.head[HD_COUNT];
  const bool gave_up = __syncthreads_or((int)threadIdx.x < a.pairs ? a.head[HD_PAIRS + threadIdx.x] : 0) != 0;
  if (blockIdx.x == 0 && threadIdx.x < 32) {
    int word = 0;
    for (int p = lane; p < a.pairs; p += 32) word |= a.head[HD_PAIRS + p];
    word = __reduce_or_sync(0xffffffffu, (unsigned)word);
    if (lane == 0) a.head[HD_STATUS] = word;
  }
  float k = -INFINITY, sum = 0.f, total = 0.f;
  auto add = [&](float pk, float ps) {             // (a part whose logits are all -inf or NaN has k = -inf and counts as it is)
    const float top = fmaxf(k, pk);
    sum = (k == top ? sum : sum * ex2(k - top)) + (pk == top || pk == -INFINITY ? ps : ps * ex2(pk - top));
    k = top;
  };
  if (row < tv) {
    for (int i0 = warp; i0 < a.n_parts; i0 += 64) {
      float2 p[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) p[u] = i0 + 8 * u < a.n_parts ? a.part[(int64_t)(i0 + 8 * u) * a.t_pad + row] : make_float2(-INFINITY, 0.f);
      float top = p[0].x, ps = 0.f;
#pragma unroll
      for (int u = 1; u < 8; ++u) top = fmaxf(top, p[u].x);
#pragma unroll
      for (int u = 0; u < 8; ++u) ps += p[u].x == -INFINITY ? p[u].y : p[u].y * ex2(p[u].x - top);
      add(top, ps);
      if (a.smooth != 0.f) {
#pragma unroll
        for (int u = 0; u < 8; ++u)
          if (i0 + 8 * u < a.n_parts) total += a.part_sum[(int64_t)(i0 + 8 * u) * a.t_pad + row];
      }
    }
  }
  ks[warp][lane] = k; sums[warp][lane] = sum; totals[warp][lane] = total;
  __syncthreads();
  if (warp != 0 || row >= tv) return;
  for (int w = 1; w < 8; ++w) { add(ks[w][lane], sums[w][lane]); total += totals[w][lane]; }
  int t = row;
  float none = 0.f;
  bool left_out = false;
  if (a.targets) {
    const int64_t y = a.targets[row];
    left_out = y == a.ignore || y < 0 || y >= a.vocab;
    none = y == a.ignore ? 0.f : __int_as_float(0x7fffffff);
  } else {
    t = a.token[row];
  }
  // the sum of k and the logarithm in 64 bits: what is rounded is the result
  double lse = ((double)k + (double)log2f(sum)) * 0.69314718055994530942;
  if (gave_up) lse = __longlong_as_double(0x7ff8000000000000ll);       // a wait ran out: nothing of this call holds
  const double loss = lse - (1.0 - (double)a.smooth) * (double)a.z_target[row] - (double)a.smooth * (double)total / a.vocab +
                      (double)a.z_loss * lse * lse;
  a.loss[t] = left_out ? none : (float)loss;
  a.lse[t] = left_out ? none : (float)lse;
}

// ---- a gradient whose K was cut: its parts, put together ------------------------------------------------

struct SumArgs {
  const int32_t* head;
  const Walk* walk;              // of the launch that made the gradients of the first piece
  const int32_t* token;
  struct Job {
    const float* acc;            // [parts][pitch of a part in rows][hidden]
    void* out;
    int64_t ld, part_rows;
    int32_t rows;                // of dw; < 0: dh, of the tokens with a target, whose places in `out` are `token`
    int32_t most;                // parts, at most
    int32_t may_stack;           // dh in bf16
    int32_t f32, accumulate;
  } job[2];
  int32_t hidden, ctas[2];       // ... of each job
  float scale;
};

__global__ void __launch_bounds__(256) head_sum_kernel(const SumArgs a) {
  __shared__ float4 sums[8][32];
  wait_for_previous_kernel();
  if (a.head[HD_STATUS] != 0) return;
  const int job = (int)blockIdx.x < a.ctas[0] ? 0 : 1, cta = (int)blockIdx.x - (job ? a.ctas[0] : 0);
  const SumArgs::Job& j = a.job[job];
  const int tv = a.head[HD_COUNT], rows = j.rows < 0 ? tv : j.rows, vec = a.hidden / 4;
  // two planes of dh as rows of one tile are summed like parts: the second is kFewTokens rows behind the first
  const int n = j.rows < 0 ? a.walk->parts_dh : a.walk->parts_dw, planes = j.may_stack && a.walk->stacked ? 2 : 1;
  if (j.most * planes == 1) return;
  const int64_t part = j.part_rows * a.hidden, total = (int64_t)rows * vec;
  // many parts: the eight warps of a CTA share those of 32 places; few: a thread has a place to itself
  const bool shared = n >= 8;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, each_cta = shared ? 32 : 256;
  const int64_t stride = (int64_t)a.ctas[job] * each_cta;
  for (int64_t i0 = (int64_t)cta * each_cta; i0 < total; i0 += stride) {
    const int64_t i = i0 + (shared ? lane : (int)threadIdx.x);
    const bool live = i < total;
    const int64_t row = !live ? 0 : total <= UINT32_MAX ? (int64_t)((uint32_t)i / (uint32_t)vec) : i / vec;
    const int c = live ? (int)(i - row * vec) * 4 : 0, step = shared ? 8 : 1;
    float x[4] = {0.f, 0.f, 0.f, 0.f};
    const float* p = j.acc + row * a.hidden + c;
    auto add_parts = [&](const float* p) {
      for (int u = shared ? warp : 0; u < n; u += 4 * step) {
        float4 v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = __ldcg(reinterpret_cast<const float4*>(p + min(u + k * step, n - 1) * part));      // (the last one again past the end)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const bool counts = u + k * step < n;
          x[0] += counts ? v[k].x : 0.f; x[1] += counts ? v[k].y : 0.f; x[2] += counts ? v[k].z : 0.f; x[3] += counts ? v[k].w : 0.f;
        }
      }
    };
    add_parts(p);
    if (planes == 2) add_parts(p + (int64_t)kFewTokens * a.hidden);
    if (shared) {
      __syncthreads();
      sums[warp][lane] = make_float4(x[0], x[1], x[2], x[3]);
      __syncthreads();
      if (warp != 0) continue;
      for (int w = 1; w < 8; ++w) {
        const float4 o = sums[w][lane];
        x[0] += o.x; x[1] += o.y; x[2] += o.z; x[3] += o.w;
      }
    }
    if (!live) continue;
    const int64_t at = (j.rows < 0 ? (int64_t)a.token[row] : row) * j.ld + c;
    if (j.f32) {
      float4* const to = reinterpret_cast<float4*>(static_cast<float*>(j.out) + at);
      const float4 o = j.accumulate ? *to : make_float4(0.f, 0.f, 0.f, 0.f);
      *to = make_float4(fmaf(x[0], a.scale, o.x), fmaf(x[1], a.scale, o.y), fmaf(x[2], a.scale, o.z), fmaf(x[3], a.scale, o.w));
    } else {
      uint2* const to = reinterpret_cast<uint2*>(static_cast<uint16_t*>(j.out) + at);
      const uint2 o = j.accumulate ? *to : make_uint2(0, 0);
      *to = make_uint2(pack_bf16x2_rn(fmaf(x[0], a.scale, __uint_as_float(o.x << 16)), fmaf(x[1], a.scale, __uint_as_float(o.x & 0xffff0000u))),
                       pack_bf16x2_rn(fmaf(x[2], a.scale, __uint_as_float(o.y << 16)), fmaf(x[3], a.scale, __uint_as_float(o.y & 0xffff0000u))));
    }
  }
}

// ---- host ----------------------------------------------------------------------------------------------

// Pairs of CTAs that run at the same time on this device; the kernels' shared memory is allowed on the way.  (Once per device.)
int pairs_of(int device, int* pairs) {
  static std::mutex mu;
  static int known[64] = {};
  if (device < 0 || device >= 64) return ADAPM_ERANGE;
  std::lock_guard<std::mutex> lock(mu);
  if (!known[device]) {
    int sms = 0;
    ADAPM_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device));
    for (const void* kernel : {(const void*)head_items_kernel<false>, (const void*)head_items_kernel<true>}) {
      cudaFuncAttributes fa;                  // (with fewer registers at launch the split above would wait for ever)
      ADAPM_CUDA(cudaFuncGetAttributes(&fa, kernel));
      if (fa.numRegs < kHeadRegs) {
        set_error_text("head_items_kernel was built with fewer registers than it divides among its warps");
        return ADAPM_EUNSUPPORTED;
      }
    }
    ADAPM_CUDA(cudaFuncSetAttribute(head_items_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kHeadSmem));
    ADAPM_CUDA(cudaFuncSetAttribute(head_items_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kHeadSmem));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(sms / 2 * 2); cfg.blockDim = dim3(kHeadThreads); cfg.dynamicSmemBytes = kHeadSmem;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = 2; at.val.clusterDim.y = 1; at.val.clusterDim.z = 1;
    cfg.attrs = &at; cfg.numAttrs = 1;
    int resident = 0;
    ADAPM_CUDA(cudaOccupancyMaxActiveClusters(&resident, head_items_kernel<true>, &cfg));
    known[device] = std::max(1, std::min({resident, sms / 2, kMostPairs}));
  }
  *pairs = known[device];
  return ADAPM_OK;
}

// Tensor maps of the operands.  (Half a microsecond of the host's time each: only those that the call reads.)
bool maps_of_operands(HeadArgs& a, const adapm_head_loss& d, const void* hidden, const void* weight, const void* compact, int64_t t_pad,
                      bool direct, bool backward) {
  bool ok = encode_bf16_matrix(&a.hk, hidden, d.tokens, d.hidden, d.hidden_ld, 128) && encode_bf16_matrix(&a.wk, weight, d.vocab, d.hidden, d.weight_ld, 128);
  if (!direct) ok = ok && encode_bf16_matrix(&a.ck, compact, t_pad, d.hidden, d.hidden, 128);
  if (backward)
    ok = ok && encode_bf16_matrix(&a.hn, hidden, d.tokens, d.hidden, d.hidden_ld, 64) && encode_bf16_matrix(&a.cn, compact, t_pad, d.hidden, d.hidden, 64) &&
         encode_bf16_matrix(&a.wn, weight, d.vocab, d.hidden, d.weight_ld, 64);
  return ok;
}

int launch_prepare(const adapm_head_loss& d, PrepareArgs p, cudaStream_t s) {
  p.ignore = d.ignore_index;
  p.hidden_ld = d.hidden_ld;
  p.tokens = (int32_t)d.tokens; p.vocab = (int32_t)d.vocab; p.width = (int32_t)d.hidden;
  p.n_walks = p.plan.backward ? p.plan.n_pieces + 1 : 1;
  p.per_cta = (int32_t)std::max<int64_t>(8, (d.tokens + 295) / 296);
  const unsigned grid = (unsigned)((d.tokens + p.per_cta - 1) / p.per_cta);
  ADAPM_CUDA(launch_chained(true, head_prepare_kernel, grid, 256, 0, s, p));
  return ADAPM_OK;
}

}  // namespace
}  // namespace adapm

using namespace adapm;

extern "C" size_t adapm_head_loss_scratch_bytes(const adapm_head_loss* d, int32_t backward) {
  Layout l;
  return d && plan(*d, backward != 0, l) == ADAPM_OK ? (size_t)l.bytes : 0;
}

extern "C" int adapm_head_loss_forward(const adapm_head_loss* d, const void* hidden, const void* weight, const int64_t* targets, float* loss,
                                       float* lse, void* scratch, size_t scratch_bytes, adapm_stream stream) {
  if (!d) return ADAPM_EINVAL;
  Layout l;
  int rc = plan(*d, false, l);
  if (rc != ADAPM_OK || d->tokens == 0) return rc;
  if (!hidden || !weight || !targets || !loss || !lse || !scratch) return ADAPM_EINVAL;
  if ((uintptr_t)hidden % 16 || (uintptr_t)weight % 16 || (uintptr_t)targets % 8 || (uintptr_t)loss % 4 || (uintptr_t)lse % 4 || (uintptr_t)scratch % 256) return ADAPM_EALIGN;
  if (scratch_bytes < (size_t)l.bytes) return ADAPM_ENOWORKSPACE;
  const Place ph = matrix_at(hidden, d->tokens, d->hidden_ld, d->hidden, 2), pw = matrix_at(weight, d->vocab, d->weight_ld, d->hidden, 2),
              pt = vector_at(targets, d->tokens, 8), ploss = vector_at(loss, d->tokens, 4), plse = vector_at(lse, d->tokens, 4),
              own = vector_at(scratch, l.bytes, 1);
  bool apart = !share(ploss, plse) && !share(own, ploss) && !share(own, plse);
  for (const Place& in : {ph, pw, pt}) apart = apart && !share(ploss, in) && !share(plse, in) && !share(own, in);
  if (!apart) {
    set_error_text("adapm_head_loss_forward: the losses, their lse or the scratch overlap another buffer");
    return ADAPM_EINVAL;
  }
  int device, pairs;
  rc = check_on_this_device({hidden, weight, targets, loss, lse, scratch}, &device);
  if (rc == ADAPM_OK) rc = pairs_of(device, &pairs);
  if (rc != ADAPM_OK) return rc;
  cudaStream_t s = (cudaStream_t)stream;
  char* const base = static_cast<char*>(scratch);

  HeadArgs a;
  std::memset(&a, 0, sizeof(a));
  if (!maps_of_operands(a, *d, hidden, weight, base + l.compact, l.t_pad, l.direct, false)) {
    set_error_text("cuTensorMapEncodeTiled failed for the head");
    return ADAPM_ECUDA;
  }
  a.head = (int32_t*)base;
  a.token = (int32_t*)(base + l.token); a.target = (int32_t*)(base + l.target);
  a.targets = l.direct ? targets : nullptr;
  a.part = (float2*)(base + l.part); a.part_sum = (float*)(base + l.part_sum); a.z_target = (float*)(base + l.z_target);
  a.tokens = (int32_t)d->tokens; a.vocab = (int32_t)d->vocab; a.hidden = (int32_t)d->hidden; a.t_pad = (int32_t)l.t_pad;
  a.split_dh = a.split_dw = 1;
  a.seg_logits = kSegForward;
  a.smooth = d->label_smoothing; a.z_loss = d->z_loss;

  const Plan plan = plan_of(*d, l, false, false, false, pairs);
  if (l.direct) {
    a.own_walk.make(plan, 0, a.tokens);
  } else {
    a.walk = (const Walk*)(base + l.walks);
    PrepareArgs p;
    std::memset(&p, 0, sizeof(p));
    p.walks = (Walk*)(base + l.walks); p.plan = plan;
    p.targets = targets; p.hidden = (const uint16_t*)hidden; p.compact = (uint16_t*)(base + l.compact);
    p.head = a.head; p.token = (int32_t*)(base + l.token); p.target = (int32_t*)(base + l.target); p.loss = loss; p.lse_out = lse;
    rc = launch_prepare(*d, p, s);
    if (rc != ADAPM_OK) return rc;
  }
  const int used = plan.used(0);
  ADAPM_CUDA(launch_clusters(true, 2, head_items_kernel<false>, 2 * (unsigned)used, kHeadThreads, kHeadSmem, s, a));
  FinalArgs f;
  f.head = a.head; f.token = a.token; f.targets = a.targets; f.part = a.part; f.part_sum = a.part_sum; f.z_target = a.z_target; f.loss = loss; f.lse = lse;
  f.ignore = d->ignore_index; f.n_parts = (int32_t)(2 * l.n_tiles); f.t_pad = (int32_t)l.t_pad; f.tokens = a.tokens; f.vocab = a.vocab; f.pairs = used;
  f.smooth = d->label_smoothing; f.z_loss = d->z_loss;
  ADAPM_CUDA(launch_chained(true, head_final_kernel, (unsigned)((d->tokens + 31) / 32), 256, 0, s, f));
  return ADAPM_OK;
}

extern "C" int adapm_head_loss_backward(const adapm_head_loss* d, const void* hidden, const void* weight, const int64_t* targets, const float* lse,
                                        const float* dloss, float scale, void* dhidden, void* dweight, void* scratch, size_t scratch_bytes,
                                        adapm_stream stream) {
  if (!d) return ADAPM_EINVAL;
  Layout l;
  int rc = plan(*d, true, l);
  if (rc != ADAPM_OK) return rc;
  if (!dhidden && !dweight) return ADAPM_EINVAL;
  cudaStream_t s = (cudaStream_t)stream;
  if ((uintptr_t)hidden % 16 || (uintptr_t)weight % 16 || (uintptr_t)targets % 8 || (uintptr_t)lse % 4 || (uintptr_t)dloss % 4 ||
      (uintptr_t)dhidden % 16 || (uintptr_t)dweight % 16 || (uintptr_t)scratch % 256) return ADAPM_EALIGN;
  const int64_t dw_row = d->weight_ld * type_bytes(d->dweight_dtype);
  int device, pairs;
  if (d->tokens == 0) {                        // no token: the gradient of the weight is zero
    if (!dweight || d->accumulate) return ADAPM_OK;
    rc = check_on_this_device({dweight}, &device);
    if (rc != ADAPM_OK) return rc;
    ADAPM_CUDA(cudaMemset2DAsync(dweight, (size_t)dw_row, 0, (size_t)(d->hidden * type_bytes(d->dweight_dtype)), (size_t)d->vocab, s));
    return ADAPM_OK;
  }
  if (!hidden || !weight || !targets || !lse || !scratch) return ADAPM_EINVAL;
  if (scratch_bytes < (size_t)l.bytes) return ADAPM_ENOWORKSPACE;
  const Place ph = matrix_at(hidden, d->tokens, d->hidden_ld, d->hidden, 2), pw = matrix_at(weight, d->vocab, d->weight_ld, d->hidden, 2),
              pt = vector_at(targets, d->tokens, 8), plse = vector_at(lse, d->tokens, 4), pdl = vector_at(dloss, d->tokens, 4),
              pdh = matrix_at(dhidden, d->tokens, d->hidden_ld, d->hidden, type_bytes(d->dhidden_dtype)),
              pdw = matrix_at(dweight, d->vocab, d->weight_ld, d->hidden, type_bytes(d->dweight_dtype));
  const Place own = vector_at(scratch, l.bytes, 1);
  bool apart = !share(pdh, pdw) && !share(own, pdh) && !share(own, pdw);
  for (const Place& in : {ph, pw, pt, plse, pdl}) apart = apart && !share(pdh, in) && !share(pdw, in) && !share(own, in);
  if (!apart) {
    set_error_text("adapm_head_loss_backward: a gradient or the scratch overlaps another buffer");
    return ADAPM_EINVAL;
  }
  rc = check_on_this_device({hidden, weight, targets, lse, dloss, dhidden, dweight, scratch}, &device);
  if (rc == ADAPM_OK) rc = pairs_of(device, &pairs);
  if (rc != ADAPM_OK) return rc;
  char* const base = static_cast<char*>(scratch);

  HeadArgs a;
  std::memset(&a, 0, sizeof(a));
  uint16_t* const g = (uint16_t*)(base + l.g);
  const int64_t g_rows = l.n_buf * l.g_rows;
  if (!maps_of_operands(a, *d, hidden, weight, base + l.compact, l.t_pad, false, true) || !encode_bf16_matrix(&a.gk, g, g_rows, l.piece, l.piece, 128) ||
      !encode_bf16_matrix(&a.gn, g, g_rows, l.piece, l.piece, 64)) {
    set_error_text("cuTensorMapEncodeTiled failed for the head");
    return ADAPM_ECUDA;
  }
  a.head = (int32_t*)base;
  a.token = (int32_t*)(base + l.token); a.target = (int32_t*)(base + l.target);
  a.lse = (float*)(base + l.lse); a.dloss = dloss ? (float*)(base + l.dloss) : nullptr;
  a.g = g; a.dh_acc = (float*)(base + l.dh_acc); a.dw_acc = (float*)(base + l.dw_acc); a.dh = dhidden; a.dw = dweight;
  a.hidden_ld = d->hidden_ld; a.weight_ld = d->weight_ld;
  a.tokens = (int32_t)d->tokens; a.vocab = (int32_t)d->vocab; a.hidden = (int32_t)d->hidden; a.t_pad = (int32_t)l.t_pad; a.piece = (int32_t)l.piece;
  a.g_rows = (int32_t)l.g_rows;
  a.split_dh = (int32_t)l.split_dh; a.split_dw = (int32_t)l.split_dw;
  a.dh_f32 = d->dhidden_dtype == ADAPM_TYPE_F32; a.dw_f32 = d->dweight_dtype == ADAPM_TYPE_F32;
  a.dh_wide = (uintptr_t)dhidden % 32 == 0 && (a.dh_f32 || d->hidden_ld % 16 == 0);
  a.dw_wide = (uintptr_t)dweight % 32 == 0 && (a.dw_f32 || d->weight_ld % 16 == 0);
  a.accumulate = d->accumulate != 0;
  a.seg_logits = a.dh_f32 || a.dw_f32 ? kSegF32 : kSegBf16;
  a.seg_dh = a.dh_f32 ? kSegF32 : kSegBf16; a.seg_dw = a.dw_f32 ? kSegF32 : kSegBf16;
  a.scale = scale; a.smooth = d->label_smoothing; a.z_loss = d->z_loss;

  const Plan plan = plan_of(*d, l, true, dhidden != nullptr, dweight != nullptr, pairs);
  PrepareArgs p;
  std::memset(&p, 0, sizeof(p));
  p.walks = (Walk*)(base + l.walks); p.plan = plan;
  p.targets = targets; p.hidden = (const uint16_t*)hidden; p.compact = (uint16_t*)(base + l.compact);
  p.head = a.head; p.token = (int32_t*)(base + l.token); p.target = (int32_t*)(base + l.target);
  p.lse_in = lse; p.lse = (float*)(base + l.lse); p.dloss_in = dloss; p.dloss = (float*)(base + l.dloss);
  p.dh = dhidden; p.dh_f32 = a.dh_f32;
  rc = launch_prepare(*d, p, s);
  if (rc != ADAPM_OK) return rc;

  for (int i = 0; i <= plan.n_pieces; ++i) {
    a.walk = (const Walk*)(base + l.walks) + i;
    a.g_begin = i * plan.piece; a.g_buf = i & 1; a.g_cols = plan.cols(i);
    a.o_begin = (i - 1) * plan.piece; a.o_buf = (i + 1) & 1; a.o_cols = plan.cols(i - 1);
    a.first = i == 1; a.last = i == plan.n_pieces;
    ADAPM_CUDA(launch_clusters(true, 2, head_items_kernel<true>, 2 * (unsigned)plan.used(i), kHeadThreads, kHeadSmem, s, a));
  }
  // (whether two planes of dh are to be summed is known on the device alone)
  const bool sum_dh = dhidden && (l.split_dh > 1 || !a.dh_f32), sum_dw = dweight && l.split_dw > 1;
  if (!sum_dh && !sum_dw) return ADAPM_OK;
  SumArgs u;
  std::memset(&u, 0, sizeof(u));
  u.head = a.head; u.walk = (const Walk*)(base + l.walks) + 1; u.token = a.token; u.hidden = a.hidden; u.scale = scale;
  int jobs = 0;
  if (sum_dh) u.job[jobs++] = {a.dh_acc, dhidden, d->hidden_ld, l.t_pad, -1, a.split_dh, !a.dh_f32, a.dh_f32, 0};
  if (sum_dw) u.job[jobs++] = {a.dw_acc, dweight, d->weight_ld, d->vocab, a.vocab, a.split_dw, 0, a.dw_f32, a.accumulate};
  for (int i = 0; i < jobs; ++i) {
    const int64_t rows = u.job[i].rows >= 0 ? d->vocab : l.split_dh > 1 ? d->tokens : std::min<int64_t>(d->tokens, kFewTokens);
    const int64_t places = rows * (d->hidden / 4), each = u.job[i].most >= 8 ? 32 : 256;
    u.ctas[i] = (int32_t)std::min<int64_t>((places + each - 1) / each, 4096);
  }
  ADAPM_CUDA(launch_chained(true, head_sum_kernel, (unsigned)(u.ctas[0] + u.ctas[1]), 256, 0, s, u));
  return ADAPM_OK;
}

extern "C" int adapm_head_loss_status(const void* scratch, adapm_stream stream, int32_t* status) {
  if (!scratch || !status) return ADAPM_EINVAL;
  int32_t word = 0;
  ADAPM_CUDA(cudaMemcpyAsync(&word, static_cast<const int32_t*>(scratch) + HD_STATUS, sizeof(word), cudaMemcpyDeviceToHost, (cudaStream_t)stream));
  ADAPM_CUDA(cudaStreamSynchronize((cudaStream_t)stream));
  *status = word;
  return word == 0 ? ADAPM_OK : ADAPM_EDEVICE;
}
