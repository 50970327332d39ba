// Dense products on the 5th-generation tensor cores, each with its epilogue:
//   forward   y  = act(x W^T s_x s_w + bias) + residual   x, W K-major, bf16 or e4m3 with scales
//   dx        dx = dp W (+ dx_residual)                   W MN-major
//   dW        dW (+)= dp^T x                              both MN-major, fp32 out
// Three forms: CTA pairs with tiles of 256 x 256 or 256 x 128, and a kernel for few tokens (below); the rule is linear_form.  dx and dW may
// share a launch of CTA pairs (linear_dw_plan_tc).
//
// linear_pair_kernel: persistent CTA pairs as in the grouped kernels (expert_tc.cu): 256 x 256 tiles, M = 256 over both CTAs'
// tensor memory, six 32 KB operand stages a CTA, accumulators double-buffered so that a tile's epilogue runs beside the next
// one's products.  Sixteen epilogue warps, four to a TMEM lane quarter with 64 columns each: a chunk of 32 x 32 is a chain of
// waits (tensor memory, shared memory, proxy fence, TMA) of a microsecond, which it takes four warps on a scheduler to hide behind
// the products of 768 inputs, the special-function unit (two instructions an element of silu and gelu) being busy for 2.2 of
// the 3.1 us that they take.
// Long contractions of many tokens are bound by the tensor pipe (operands through shared memory; see expert_tc.cu) and, held for long, by power:
// 32768 tokens 4096 -> 1536 345 us (1.2 PFLOP/s held), 9001 tokens 1536 -> 4096 79 us (1.44 PFLOP/s).  Short ones, and 8 bits, whose products
// take half the time, by the epilogue (the pipe 56 % busy in both): 9001 tokens 1536 -> 4096 in e4m3 50 us (2.28 PFLOP/s), 56 to 66 with bias and silu;
// 16384 tokens 768 -> 2048 42 us, with gelu 46, with p stored too 52 to 61.  Few tiles of a long contraction by what the L2
// delivers (1501 tokens 4096 -> 1536: 72 tiles of 256 x 128, 26 us).
// 18 warps leave 96 registers to a thread, and some of them spill: dx beside dW with a residual on 256 columns 76 bytes stored and 140 loaded a
// thread, the forward ones up to 36 and 48; the times above are with that.
#include <cuda.h>

#include <algorithm>
#include <type_traits>

#include "common.cuh"
#include "linear_act.cuh"
#include "tc_maps.cuh"
#include "tc_ptx.cuh"

namespace unipool {

namespace {

enum LinearKind { kLinFwd, kLinFwd8, kLinDx, kLinDw, kLinBoth };   // kLinBoth: dW's tiles, then dx's, in one launch

constexpr uint32_t kLinHalf = 128 * 128;                 // 128 rows (columns) x 128 bytes of one operand
constexpr uint32_t kLinBars = 229376;                    // operand stages and staging tiles fill this much
constexpr uint32_t kLinSmem = kLinBars + 512 + 1024;
constexpr int kLinEpiWarps = 16;
constexpr int kLinThreads = 64 + 32 * kLinEpiWarps;
constexpr int kLinChunk = 32;                            // columns that an epilogue warp has in hand
constexpr uint32_t kLinTile = 32 * kLinChunk * 2;        // a chunk of 32 rows in bf16, rows of 64 bytes
// The tensor core truncates the sums it adds to: over K terms of both signs they lose 1.1e-9 K of their magnitude (measured, 512 to 32768
// rows), over terms of one sign 5e-9 to 7e-9 K in bf16 (16384 to 1048576), which at 262144 is a third of half a bf16 step and at
// 2097152 three of them.  The weight gradient, an fp32 result of a sum over all tokens, is therefore taken from the accumulator every
// 768 tokens and added up in registers, where it is rounded to nearest; the other products every 16384 terms (32768 in 8 bits), which
// leaves 1e-4 at most and costs contractions of up to so many nothing.
constexpr int kLinSegment = 12;                          // k-blocks of 64 tokens
constexpr int kLinLong = 256;                            // k-blocks of 128 bytes

struct LinearGrid {
  int M, N;                          // rows and columns of the result
  int n_mt, n_nt, units, kb_total, kb_split;
};
struct LinearParams {
  LinearGrid g, w;                   // w: of the weight gradient in kLinBoth
  int act;
  const float *bias, *x_scale, *w_scale;
  bool pre;                          // the value before the activation is stored too
  bool vec;                          // bias and w_scale are 16-byte aligned
  const __nv_bfloat16* residual;     // [M, N] or NULL
  float* dw;                         // weight gradient: [splits, M, N]
  bool add;                          // ... +=
  bool wide, wide_dw;                // residual, and dw, are 32-byte aligned
  int32_t* status;
};

struct LinearMaps { CUtensorMap a, b, c, r, p, wa, wb; };  // operands, result, residual, value before the activation; kLinBoth: dW's operands

struct LinearUnit { int mt, nt, split, kb0, kb1; };
__device__ __forceinline__ LinearUnit linear_unit(const LinearGrid& p, int u) {
  LinearUnit t;
  const int per = p.n_mt * p.n_nt;
  t.split = u / per;
  const int rem = u - t.split * per;
  t.mt = rem / p.n_nt;
  t.nt = rem - t.mt * p.n_nt;
  t.kb0 = t.split * p.kb_split;
  t.kb1 = min(p.kb_total, t.kb0 + p.kb_split);
  return t;
}

__device__ __forceinline__ void linear_timeout(int32_t* status, volatile int* abort, int site) {
  *abort = 1;
  if (atomicCAS(status, 0, kStatusTimeout) == 0) {
    status[1] = site;
    status[2] = (int)blockIdx.x;
  }
}

// 32 bytes at p, a sector (`wide`: p is 32-byte aligned, else 16).
__device__ __forceinline__ void st_sector(void* p, const uint32_t* v, bool wide) {
  if (wide) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]),
                 "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
                 : "memory");
  } else {
    static_cast<uint4*>(p)[0] = make_uint4(v[0], v[1], v[2], v[3]);
    static_cast<uint4*>(p)[1] = make_uint4(v[4], v[5], v[6], v[7]);
  }
}
__device__ __forceinline__ void ld_sector(const void* p, uint32_t* v, bool wide) {
  if (wide) {
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
                 : "l"(p)
                 : "memory");
  } else {
    const uint4 a = static_cast<const uint4*>(p)[0], b = static_cast<const uint4*>(p)[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
}
// 16-byte piece q of row r of a staging tile in the layout of the 64-byte TMA swizzle
__device__ __forceinline__ uint4* piece(uint8_t* tile, int r, int q) {
  return reinterpret_cast<uint4*>(tile + r * 64 + ((q ^ ((r >> 1) & 3)) << 4));
}
__device__ __forceinline__ void put_row(uint8_t* tile, int r, const float (&v)[32]) {
#pragma unroll
  for (int q = 0; q < 4; ++q)
    *piece(tile, r, q) = make_uint4(tc::pack_bf16(v[8 * q], v[8 * q + 1]), tc::pack_bf16(v[8 * q + 2], v[8 * q + 3]),
                                    tc::pack_bf16(v[8 * q + 4], v[8 * q + 5]), tc::pack_bf16(v[8 * q + 6], v[8 * q + 7]));
}
// 32 consecutive values, the same in all lanes
struct Columns {
  float4 v[8];
  __device__ __forceinline__ void load(const float* p, bool vec) {
#pragma unroll
    for (int q = 0; q < 8; ++q)
      v[q] = vec ? __ldg(reinterpret_cast<const float4*>(p) + q)
                 : make_float4(__ldg(p + 4 * q), __ldg(p + 4 * q + 1), __ldg(p + 4 * q + 2), __ldg(p + 4 * q + 3));
  }
  __device__ __forceinline__ float at(int i) const { return i % 4 == 0 ? v[i / 4].x : i % 4 == 1 ? v[i / 4].y : i % 4 == 2 ? v[i / 4].z : v[i / 4].w; }
};
__device__ __forceinline__ void activate(float (&v)[32], int act) {
#define UP_ACT(a)                                                          \
  case a:                                                                  \
    _Pragma("unroll") for (int i = 0; i < 32; ++i) v[i] = act_value<true>(v[i], a); \
    break;
  switch (act) {
    UP_ACT(UNIPOOL_ACT_RELU)
    UP_ACT(UNIPOOL_ACT_SILU)
    UP_ACT(UNIPOOL_ACT_GELU)
  }
#undef UP_ACT
}

// kRes: a residual is added.  All of it is asked for before the accumulator is waited for: the first chunk's comes by TMA into
// the staging tile, the second's into registers (a second tile for it would take an operand stage: 16384 tokens, 2048 -> 768 48.7
// us instead of 44.8).  kPre: the value before the activation is stored too (one kernel with and without it where no residual is).
// kN: columns of a tile, 256 or 128.  kLong: a contraction of several parts of kLinLong k-blocks (a kernel of its own: the parts' sums and the branch
// cost the others up to 5 %, 9001 tokens 1536 -> 4096 in e4m3 67.8 us instead of 66.2).
template <int KIND, int kN, bool kRes, bool kPre, bool kLong>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kLinThreads, 1)
linear_pair_kernel(const __grid_constant__ LinearMaps m, LinearParams p) {
  constexpr uint32_t kStage = kLinHalf + kN * 64;         // 128 rows of A, kN / 2 of B
  constexpr int kStages = KIND == kLinDw ? 7 : kN == 256 ? 6 : 8;
  constexpr uint32_t kStaging = KIND == kLinDw ? 0 : kLinTile;
  static_assert(kStages * kStage + kLinEpiWarps * kStaging == kLinBars, "shared memory");
  static_assert(kN == 256 || (kN == 128 && KIND != kLinDw), "columns of a tile");
  constexpr bool kBoth = KIND == kLinBoth, kDw = KIND == kLinDw || kBoth;
  constexpr int kPart = kN / 4, kChunks = kPart / kLinChunk;   // columns of an epilogue warp, its chunks
  constexpr bool kBMn = KIND == kLinDx || kDw;
  constexpr int kKb = KIND == kLinFwd8 ? 128 : 64;       // elements of a k-block
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* full_bar = reinterpret_cast<uint64_t*>(smem + kLinBars);
  uint64_t* empty_bar = full_bar + kStages;
  uint64_t* tmem_full = empty_bar + kStages;
  uint64_t* tmem_empty = tmem_full + 2;
  uint64_t* res_bar = tmem_empty + 2;                    // [16] a chunk of the residual has landed
  uint32_t* tmem_ptr = reinterpret_cast<uint32_t*>(res_bar + (kRes ? kLinEpiWarps : 0));
  volatile int* abort = reinterpret_cast<volatile int*>(tmem_ptr + 1);
  static_assert((2 * kStages + 4 + kLinEpiWarps) * 8 + 8 <= 512, "barrier block");

  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int rank = (int)tc::cluster_ctarank();           // 0 = leader
  const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) { tc::mbar_init(&full_bar[s], 1); tc::mbar_init(&empty_bar[s], 1); }
    for (int a = 0; a < 2; ++a) { tc::mbar_init(&tmem_full[a], 1); tc::mbar_init(&tmem_empty[a], 2 * kLinEpiWarps); }
    if constexpr (kRes)
      for (int i = 0; i < kLinEpiWarps; ++i) tc::mbar_init(&res_bar[i], 1);
    *abort = 0;
    tc::fence_barrier_init();
    tc::tma_prefetch_desc(&m.a);
    tc::tma_prefetch_desc(&m.b);
  }
  if (warp == 1) {
    tc::tmem_alloc_pair(tmem_ptr, 512);
    tc::tmem_relinquish_pair();
  }
  tc::tc_fence_before_sync();
  __syncthreads();
  tc::cluster_sync();                                    // both CTAs' barriers exist before any remote use
  tc::tc_fence_after_sync();
  const uint32_t tmem_base = *tmem_ptr;
  grid_wait(p.bias, p.x_scale, p.w_scale, p.residual);
  const int units = p.g.units + (kBoth ? p.w.units : 0);
  auto is_dw = [&](int u) { return KIND == kLinDw || (kBoth && u < p.w.units); };
  auto unit = [&](int u) { return kBoth ? (u < p.w.units ? linear_unit(p.w, u) : linear_unit(p.g, u - p.w.units)) : linear_unit(p.g, u); };

  if (warp == 0) {
    // ------------------------------------------------------------ TMA producer (one in each CTA)
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int u = pair; u < units && ok; u += n_pairs) {
        const LinearUnit t = unit(u);
        const bool dw = is_dw(u);
        for (int kb = t.kb0; kb < t.kb1; ++kb) {
          if (!tc::mbar_wait(&empty_bar[stage], phase ^ 1u, abort)) { linear_timeout(p.status, abort, 41); ok = false; break; }
          uint8_t* sA = smem + stage * kStage;
          uint8_t* sB = sA + kLinHalf;
          if (rank == 0) tc::mbar_expect_tx(&full_bar[stage], 2 * kStage);         // both CTAs' bytes
          const CUtensorMap *ma = kBoth && dw ? &m.wa : &m.a, *mb = kBoth && dw ? &m.wb : &m.b;
          if (kDw && dw) tc::tma_load_3d_pair(sA, ma, &full_bar[stage], 0, kb * kKb, t.mt * 4 + rank * 2);
          else tc::tma_load_2d_pair(sA, ma, &full_bar[stage], kb * kKb, t.mt * 256 + rank * 128);
          if constexpr (kBMn) tc::tma_load_3d_pair(sB, mb, &full_bar[stage], 0, kb * kKb, (t.nt * 2 + rank) * (kN / 128));
          else tc::tma_load_2d_pair(sB, mb, &full_bar[stage], kb * kKb, t.nt * kN + rank * (kN / 2));
          if (++stage == kStages) { stage = 0; phase ^= 1u; }
        }
      }
      if (!ok)
        for (int i = 0; i < 200; ++i) __nanosleep(1000);  // let loads already in flight land before the CTA retires
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMA issuer (leader CTA only)
    if (lane == 0 && rank == 0) {
      constexpr uint32_t b_lbo = kBMn ? kLinHalf / 2 : 16, b_step = (kBMn ? 16 * 128 : 32) >> 4;
      int stage = 0, local = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int u = pair; u < units && ok; u += n_pairs) {
        const LinearUnit t = unit(u);
        const bool dw = is_dw(u);
        const bool a_mn = kDw && dw;
        const uint32_t idesc = KIND == kLinFwd8 ? tc::instr_desc_e4m3(kN, 256) : tc::instr_desc_bf16(kN, a_mn, kBMn, 256);
        const uint32_t a_lbo = a_mn ? kLinHalf / 2 : 16, a_step = (a_mn ? 16 * 128 : 32) >> 4;
        for (int kb = t.kb0; kb < t.kb1 && ok;) {
          const int end = a_mn ? min(t.kb1, kb + kLinSegment) : kLong ? min(t.kb1, kb + kLinLong) : t.kb1;
          const int acc = local & 1;
          if (!tc::mbar_wait(&tmem_empty[acc], ((local >> 1) & 1) ^ 1u, abort)) { linear_timeout(p.status, abort, 42); ok = false; break; }
          ++local;
          tc::tc_fence_after_sync();
          const uint32_t d_tmem = tmem_base + acc * 256;
          uint32_t accumulate = 0;
          for (; kb < end; ++kb) {
            if (!tc::mbar_wait(&full_bar[stage], phase, abort)) { linear_timeout(p.status, abort, 43); ok = false; break; }
            tc::tc_fence_after_sync();
            const uint32_t a = tc::smem_u32(smem + stage * kStage);
            const uint64_t adesc = tc::smem_desc_sw128(a, a_lbo, 1024);
            const uint64_t bdesc = tc::smem_desc_sw128(a + kLinHalf, b_lbo, 1024);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              if constexpr (KIND == kLinFwd8) tc::umma_e4m3_pair(d_tmem, adesc + j * a_step, bdesc + j * b_step, idesc, accumulate);
              else tc::umma_bf16_pair(d_tmem, adesc + j * a_step, bdesc + j * b_step, idesc, accumulate);
              accumulate = 1;
            }
            tc::umma_commit_pair(&empty_bar[stage], 3);   // frees the stage in both CTAs
            if (++stage == kStages) { stage = 0; phase ^= 1u; }
          }
          if (ok) tc::umma_commit_pair(&tmem_full[acc], 3);   // accumulator complete, both CTAs
        }
      }
    }
  } else {
    // ------------------------------------------------------------ epilogue: 32 rows and a quarter of the tile's columns to a warp
    const int quarter = warp & 3, ew = warp - 2, part = ew >> 2;
    uint8_t* stg = smem + kStages * kStage + ew * kStaging;
    const uint32_t lanes = static_cast<uint32_t>(quarter * 32) << 16;
    int local = 0;
    uint32_t turn = 0;                                    // chunks of the residual that have landed in the staging tile
    bool ok = true;
    auto release = [&](int acc) {
      tc::tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) {                                    // the leader's MMA thread waits for both CTAs' epilogue warps
        if (rank == 0) tc::mbar_arrive(&tmem_empty[acc]);
        else tc::mbar_arrive_leader(&tmem_empty[acc]);
      }
    };
    auto wait_full = [&](int acc) {
      const bool got = tc::mbar_wait_warp(&tmem_full[acc], (local >> 1) & 1, abort);
      if (!got && lane == 0) linear_timeout(p.status, abort, 44);
      ++local;
      tc::tc_fence_after_sync();
      return got;
    };
    for (int u = pair; u < units && ok; u += n_pairs) {
      const LinearUnit t = unit(u);
      const bool dw = is_dw(u);
      const LinearGrid& g = kBoth && dw ? p.w : p.g;
      const int row0 = t.mt * 256 + rank * 128 + quarter * 32, col0 = t.nt * kN + part * kPart;
      const int nch = row0 < g.M ? max(0, min(kChunks, (g.N - col0) / kLinChunk)) : 0;
      if (kDw && dw) {
        float sum[kPart / 16][16];
#pragma unroll
        for (int q = 0; q < kPart / 16; ++q)
#pragma unroll
          for (int i = 0; i < 16; ++i) sum[q][i] = 0.f;
#pragma unroll 1
        for (int kb = t.kb0; kb < t.kb1 && ok; kb += kLinSegment) {
          const int acc = local & 1;
          ok = wait_full(acc);
          if (!ok) break;
#pragma unroll
          for (int q = 0; q < kPart / 16; ++q) {
            uint32_t rr[16];
            tc::tmem_ld_32x16(tmem_base + lanes + acc * 256 + part * kPart + q * 16, rr);
            tc::tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 16; ++i) sum[q][i] += __uint_as_float(rr[i]);
          }
          release(acc);
        }
        if (!ok) break;
        float* out = &p.dw[((int64_t)t.split * g.M + row0 + lane) * g.N + col0];
#pragma unroll
        for (int ch = 0; ch < kChunks; ++ch) {
          if (ch >= nch) continue;                        // (row0 < M: then all of the warp's rows are, M being a multiple of 64)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            float(&v)[16] = sum[2 * ch + q / 2];
            float* o = out + ch * kLinChunk + 8 * q;
            uint32_t w[8];
            if (p.add) {
              ld_sector(o, w, p.wide_dw);
#pragma unroll
              for (int i = 0; i < 8; ++i) v[q % 2 * 8 + i] += __uint_as_float(w[i]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(v[q % 2 * 8 + i]);
            st_sector(o, w, p.wide_dw);
          }
        }
      }
      if (KIND != kLinDw && !(kBoth && dw)) {
        const bool mine = row0 + lane < g.M;
        uint32_t r1[16];
        if constexpr (kRes) {
          if (lane == 0 && nch > 0) {
            tc::bulk_wait_read<0>();                      // what last left from there
            tc::mbar_expect_tx(&res_bar[ew], kLinTile);
            tc::tma_load_2d(stg, &m.r, &res_bar[ew], col0, row0);
          }
          if (kChunks > 1 && mine && nch > 1) {
            const __nv_bfloat16* r = p.residual + ((int64_t)(row0 + lane) * g.N + col0 + kLinChunk);
            ld_sector(r, r1, p.wide);
            ld_sector(r + 16, r1 + 8, p.wide);
          }
          __syncwarp();
        }
        float xs = 1.f;
        if (KIND == kLinFwd8 && mine) xs = __ldg(p.x_scale + row0 + lane);
        float held[kLong ? kPart : 1];                    // sums of the parts but the last (indexed by a variable: local memory, no registers)
        if constexpr (kLong) {
#pragma unroll 1
          for (int kb = t.kb0; kb + kLinLong < t.kb1; kb += kLinLong) {
            const int a = local & 1;
            ok = wait_full(a);
            if (!ok) break;
#pragma unroll 1
            for (int c = 0; c < kPart; c += 16) {
              uint32_t rr[16];
              tc::tmem_ld_32x16(tmem_base + lanes + a * 256 + part * kPart + c, rr);
              tc::tmem_ld_wait();
#pragma unroll
              for (int i = 0; i < 16; ++i) held[c + i] = (kb > t.kb0 ? held[c + i] : 0.f) + __uint_as_float(rr[i]);
            }
            release(a);
          }
          if (!ok) break;
        }
        const int acc = local & 1;
        ok = wait_full(acc);
        if (!ok) break;
#pragma unroll
        for (int ch = 0; ch < kChunks; ++ch) {
          if (ch >= nch) continue;
          const int col = col0 + ch * kLinChunk;
          uint32_t rr[32];
          Columns c;                                      // on their way while the accumulator is
          tc::tmem_ld_32x32(tmem_base + lanes + acc * 256 + part * kPart + ch * kLinChunk, rr);
          // (with a residual too there are no registers for that)
          if (KIND == kLinFwd8 && !kRes) c.load(p.w_scale + col, p.vec);
          if (KIND == kLinFwd && !kRes && p.bias != nullptr) c.load(p.bias + col, p.vec);
          tc::tmem_ld_wait();
          if (ch + 1 == nch) release(acc);                // the accumulator is in registers
          float v[32];
#pragma unroll
          for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(rr[i]);
          if constexpr (kLong) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] += held[ch * kLinChunk + i];
          }
          if constexpr (KIND == kLinFwd8) {
            if (kRes) c.load(p.w_scale + col, p.vec);
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = v[i] * xs * c.at(i);   // one after the other: their product may leave fp32's range
          }
          if ((KIND == kLinFwd8 || (KIND == kLinFwd && kRes)) && p.bias != nullptr) c.load(p.bias + col, p.vec);
          if (KIND != kLinDx && !kBoth && p.bias != nullptr) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] += c.at(i);
          }
          uint32_t r0[16];
          auto take = [&] {                               // the first chunk's residual, out of the tile
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const uint4 w = *piece(stg, lane, q);
              r0[4 * q] = w.x; r0[4 * q + 1] = w.y; r0[4 * q + 2] = w.z; r0[4 * q + 3] = w.w;
            }
          };
          if constexpr (kRes) {
            if (ch == 0) {
              ok = tc::mbar_wait_warp(&res_bar[ew], turn & 1, abort);
              if (!ok) {
                if (lane == 0) linear_timeout(p.status, abort, 45);
                break;
              }
              ++turn;
              if (kPre) take();
            }
          }
          if constexpr (KIND != kLinDx && !kBoth) {
            if (kPre || (!kRes && p.pre)) {               // leaves first, from the same tile
              if ((!kRes || ch == 1) && lane == 0) tc::bulk_wait_read<0>();
              __syncwarp();
              put_row(stg, lane, v);
              tc::fence_proxy_async();
              __syncwarp();
              if (lane == 0) { tc::tma_store_2d(&m.p, stg, col, row0); tc::bulk_commit(); }
            }
            activate(v, p.act);
          }
          if constexpr (kRes) {
            if (ch == 0 && !kPre) take();
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const uint32_t w = ch == 0 ? r0[i] : r1[i];
              v[2 * i] += __uint_as_float(w << 16);
              v[2 * i + 1] += __uint_as_float(w & 0xffff0000u);
            }
          }
          if ((!kRes || kPre || ch == 1) && lane == 0) tc::bulk_wait_read<0>();
          __syncwarp();
          put_row(stg, lane, v);
          tc::fence_proxy_async();
          __syncwarp();
          if (lane == 0) { tc::tma_store_2d(&m.c, stg, col, row0); tc::bulk_commit(); }
        }
        if (!ok) break;
        if (nch == 0) release(acc);
      }
    }
    if (!ok && lane == 0)
      for (int i = 0; i < 200; ++i) __nanosleep(1000);
    if (lane == 0) tc::bulk_wait<0>();
    __syncwarp();
  }

  tc::tc_fence_before_sync();
  __syncthreads();
  tc::cluster_sync();                                    // neither CTA leaves while the other may still signal it
  if (warp == 1) {
    tc::tc_fence_after_sync();
    tc::tmem_dealloc_pair(tmem_base, 512);
  }
}

LinearGrid linear_grid(int M, int N, int tile_n, int kb_total, int splits) {
  LinearGrid g{};
  g.M = M; g.N = N;
  g.n_mt = (M + 255) / 256; g.n_nt = (N + tile_n - 1) / tile_n;
  g.kb_total = kb_total;
  g.kb_split = (kb_total + splits - 1) / splits;
  g.units = g.n_mt * g.n_nt * ((kb_total + g.kb_split - 1) / g.kb_split);
  return g;
}

template <int KIND, int kN, bool kRes, bool kPre>
int launch_linear(unipool_ctx* ctx, int phase, const LinearMaps& m, const LinearParams& p, cudaStream_t s) {
  PhaseTimer pt(ctx, phase, 1, s);
  auto run = [&](auto kern) {
    UP_CUDA(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kLinSmem));
    const int pairs = ctx->sm_count / 2, units = p.g.units + p.w.units;
    UP_KERNEL(kern, 2 * (units < pairs ? units : pairs), kLinThreads, kLinSmem, s, m, p);
    return (int)UNIPOOL_OK;
  };
  if constexpr (KIND != kLinDw) {
    if (p.g.kb_split > kLinLong) return run(linear_pair_kernel<KIND, kN, kRes, kPre, true>);
  }
  return run(linear_pair_kernel<KIND, kN, kRes, kPre, false>);
}

template <typename... P> bool aligned(uintptr_t n, P... p) { return ((... | reinterpret_cast<uintptr_t>(p)) & (n - 1)) == 0; }

#define UP_TRY(call)                     \
  do {                                   \
    const int rc__ = (call);             \
    if (rc__ != UNIPOOL_OK) return rc__; \
  } while (0)

// ---------------------------------------------------------------- few tokens
// The weights on the M side: a CTA holds 128 features (A) against all of up to 128 tokens (N in steps of 16), S CTAs of a cluster
// share a tile's contraction and add up through each other's shared memory, in the order of their ranks; each then finishes every
// S-th token.  Bound by the weights' bytes and, below some megabytes of them, by latency: every CTA asks for all of its weights
// at once as far as they fit its stages.
// No CTA waits for another one while it holds tensor memory: the columns go back as soon as the sums lie in shared memory, in front of the
// first wait for the cluster.  (CTAs of several calls share an SM where those run on several streams, and an allocation waits until
// columns are free: one that is held until the cluster is complete could wait for a CTA that itself waits for columns, round in a ring.)
// And every launch asks for so much shared memory that no more CTAs lie on an SM than it has columns for.
constexpr int kFewTokens = 128, kFewMaxStages = 12;
constexpr uint32_t kFewBars = 512;
constexpr int kFewLong = 1024;                           // k-blocks of a CTA at most: 65536 terms in bf16, which lose 5e-4 at most (kLinSegment)
constexpr uint32_t kFewColumns = 128;                    // of the SM's 512: one accumulator of up to 128 tokens
constexpr uint32_t kFewSmemLeast = 46080;                // (with the system's 1 KB, five CTAs are more than an SM's 228 KB)
static_assert(kFewColumns >= kFewTokens && (512 / kFewColumns + 1) * (kFewSmemLeast + 1024) > 228 * 1024, "tensor memory of an SM");

struct FewParams {
  int T, M, N;                       // tokens of the call and of a tile (a multiple of 16); features of the result
  int kb_total, stages, act;
  const float *bias, *x_scale, *w_scale;
  const __nv_bfloat16* residual;
  __nv_bfloat16 *pre, *y;            // [T, M]
  int32_t* status;
};

__device__ __forceinline__ float4 ld_cluster(uint32_t addr, uint32_t rank) {    // 16 bytes at `addr` of CTA `rank`
  uint32_t remote;
  float4 v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(addr), "r"(rank));
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(remote) : "memory");
  return v;
}
__device__ __forceinline__ void store_bf16x4(__nv_bfloat16* p, const float (&v)[4]) {
  *reinterpret_cast<uint2*>(p) = make_uint2(tc::pack_bf16(v[0], v[1]), tc::pack_bf16(v[2], v[3]));
}

// E epilogue warps: four or sixteen (few_shape).
template <int KIND, int S, int E>
__global__ void __cluster_dims__(S, 1, 1) __launch_bounds__(64 + 32 * E)
linear_few_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX, FewParams p) {
  constexpr bool kAMn = KIND == kLinDx;
  constexpr int kKb = KIND == kLinFwd8 ? 128 : 64;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* full_bar = reinterpret_cast<uint64_t*>(smem);
  uint64_t* empty_bar = full_bar + kFewMaxStages;
  uint64_t* done_bar = empty_bar + kFewMaxStages;
  uint32_t* tmem_ptr = reinterpret_cast<uint32_t*>(done_bar + 1);
  volatile int* abort = reinterpret_cast<volatile int*>(tmem_ptr + 1);
  static_assert((2 * kFewMaxStages + 1) * 8 + 8 <= kFewBars, "barrier block");
  uint8_t* ring = smem + 1024;
  float* sums = reinterpret_cast<float*>(ring);            // [N][128], once the products are complete
  const uint32_t stage_bytes = kLinHalf + p.N * 128;

  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int rank = S > 1 ? (int)tc::cluster_ctarank() : 0;
  const int m0 = blockIdx.x / S * 128, t0 = blockIdx.y * p.N;
  const int kb0 = (int)((int64_t)p.kb_total * rank / S), n = (int)((int64_t)p.kb_total * (rank + 1) / S) - kb0;
  if (threadIdx.x == 0) {
    for (int s = 0; s < p.stages; ++s) { tc::mbar_init(&full_bar[s], 1); tc::mbar_init(&empty_bar[s], 1); }
    tc::mbar_init(done_bar, 1);
    *abort = 0;
    tc::fence_barrier_init();
    tc::tma_prefetch_desc(&tmW);
    tc::tma_prefetch_desc(&tmX);
  }
  if (warp == 1) {
    tc::tmem_alloc(tmem_ptr, kFewColumns);
    tc::tmem_relinquish();
  }
  tc::tc_fence_before_sync();
  __syncthreads();
  tc::tc_fence_after_sync();
  const uint32_t tmem = *tmem_ptr;
  grid_wait(p.bias, p.x_scale, p.w_scale, p.residual);

  if (warp == 0) {
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int i = 0; i < n; ++i) {
        ok = tc::mbar_wait(&empty_bar[stage], phase ^ 1u, abort);
        if (!ok) { linear_timeout(p.status, abort, 51); break; }
        uint8_t* sW = ring + stage * stage_bytes;
        const int k = (kb0 + i) * kKb;
        tc::mbar_expect_tx(&full_bar[stage], stage_bytes);
        if constexpr (kAMn) tc::tma_load_3d(sW, &tmW, &full_bar[stage], 0, k, m0 / 64);
        else tc::tma_load_2d(sW, &tmW, &full_bar[stage], k, m0);
        tc::tma_load_2d(sW + kLinHalf, &tmX, &full_bar[stage], k, t0);
        if (++stage == p.stages) { stage = 0; phase ^= 1u; }
      }
      if (!ok)
        for (int i = 0; i < 200; ++i) __nanosleep(1000);
    }
    __syncwarp();
  } else if (warp == 1) {
    if (lane == 0 && n > 0) {
      const uint32_t idesc = KIND == kLinFwd8 ? tc::instr_desc_e4m3(p.N, 128) : tc::instr_desc_bf16(p.N, kAMn, false, 128);
      constexpr uint32_t a_lbo = kAMn ? kLinHalf / 2 : 16, a_step = (kAMn ? 16 * 128 : 32) >> 4;
      int stage = 0;
      uint32_t phase = 0, accumulate = 0;
      bool ok = true;
      for (int i = 0; i < n; ++i) {
        ok = tc::mbar_wait(&full_bar[stage], phase, abort);
        if (!ok) { linear_timeout(p.status, abort, 52); break; }
        tc::tc_fence_after_sync();
        const uint32_t a = tc::smem_u32(ring + stage * stage_bytes);
        const uint64_t adesc = tc::smem_desc_sw128(a, a_lbo, 1024), bdesc = tc::smem_desc_sw128(a + kLinHalf, 16, 1024);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if constexpr (KIND == kLinFwd8) tc::umma_e4m3(tmem, adesc + j * a_step, bdesc + j * 2, idesc, accumulate);
          else tc::umma_bf16(tmem, adesc + j * a_step, bdesc + j * 2, idesc, accumulate);
          accumulate = 1;
        }
        tc::umma_commit(&empty_bar[stage]);
        if (++stage == p.stages) { stage = 0; phase ^= 1u; }
      }
      if (ok) tc::umma_commit(done_bar);
    }
    __syncwarp();
  } else {
    const int quarter = warp & 3, f = quarter * 32 + lane;
    bool some = n > 0;
    if (some) {
      some = tc::mbar_wait_warp(done_bar, 0, abort);
      if (!some && lane == 0) linear_timeout(p.status, abort, 53);
      tc::tc_fence_after_sync();
    }
    for (int c = (warp - 2) / 4 * 16; c < p.N; c += E * 4) {
      uint32_t rr[16];
      if (some) {
        tc::tmem_ld_32x16(tmem + (static_cast<uint32_t>(quarter * 32) << 16) + c, rr);
        tc::tmem_ld_wait();
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) sums[(c + i) * 128 + f] = some ? __uint_as_float(rr[i]) : 0.f;
    }
    tc::tc_fence_before_sync();
  }
  __syncthreads();                                       // this CTA's sums are there
  if (warp == 1) {
    tc::tc_fence_after_sync();
    tc::tmem_dealloc(tmem, kFewColumns);                  // (before any other CTA is waited for)
  }
  if constexpr (S > 1) tc::cluster_sync();               // every CTA's are

  // Four features to a lane, a token to a warp: of the cluster's (2 + E) S warps each takes every (2 + E) S-th token.
  const int m = m0 + 4 * lane;
  if (m < p.M) {
    float4 b = make_float4(0.f, 0.f, 0.f, 0.f), ws = b;
    if (KIND != kLinDx && p.bias != nullptr)
      b = make_float4(__ldg(p.bias + m), __ldg(p.bias + m + 1), __ldg(p.bias + m + 2), __ldg(p.bias + m + 3));
    if (KIND == kLinFwd8)
      ws = make_float4(__ldg(p.w_scale + m), __ldg(p.w_scale + m + 1), __ldg(p.w_scale + m + 2), __ldg(p.w_scale + m + 3));
    const uint32_t mine = tc::smem_u32(sums) + lane * 16;
    constexpr int kWarps = 2 + E;
#pragma unroll 2
    for (int t = rank * kWarps + warp; t < p.N && t0 + t < p.T; t += S * kWarps) {
      const int64_t at = (int64_t)(t0 + t) * p.M + m;
      uint2 r = make_uint2(0u, 0u);
      if (p.residual != nullptr) r = *reinterpret_cast<const uint2*>(&p.residual[at]);
      const float xs = KIND == kLinFwd8 ? __ldg(p.x_scale + (t0 + t)) : 1.f;
      float4 part[S];
#pragma unroll
      for (int q = 0; q < S; ++q) part[q] = S > 1 ? ld_cluster(mine + t * 512, q) : *reinterpret_cast<const float4*>(&sums[t * 128 + 4 * lane]);
#pragma unroll
      for (int q = 1; q < S; ++q) {
        part[0].x += part[q].x; part[0].y += part[q].y; part[0].z += part[q].z; part[0].w += part[q].w;
      }
      float v[4] = {part[0].x, part[0].y, part[0].z, part[0].w};
      if constexpr (KIND == kLinFwd8) {
        v[0] = v[0] * xs * ws.x; v[1] = v[1] * xs * ws.y; v[2] = v[2] * xs * ws.z; v[3] = v[3] * xs * ws.w;
      }
      if constexpr (KIND != kLinDx) {
        v[0] += b.x; v[1] += b.y; v[2] += b.z; v[3] += b.w;
        if (p.pre != nullptr) store_bf16x4(&p.pre[at], v);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = act_value<true>(v[i], p.act);
      }
      v[0] += __uint_as_float(r.x << 16); v[1] += __uint_as_float(r.x & 0xffff0000u);
      v[2] += __uint_as_float(r.y << 16); v[3] += __uint_as_float(r.y & 0xffff0000u);
      store_bf16x4(&p.y[at], v);
    }
  }
  if constexpr (S > 1) tc::cluster_sync();               // no CTA leaves while another reads its sums
}

template <int KIND, int S, int E>
int launch_few(unipool_ctx* ctx, int phase, const CUtensorMap& tmW, const CUtensorMap& tmX, const FewParams& p, uint32_t smem,
               cudaStream_t s) {
  PhaseTimer pt(ctx, phase, 1, s);
  auto kern = linear_few_kernel<KIND, S, E>;
  UP_CUDA(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 232448));
  UP_KERNEL(kern, dim3((p.M + 127) / 128 * S, (p.T + p.N - 1) / p.N), 64 + 32 * E, smem, s, tmW, tmX, p);
  return UNIPOOL_OK;
}

// How a call runs on the kernel for few tokens: a cluster of eight or four lies inside one GPC of 16 to 18 SMs, so that with two
// CTAs on an SM 32 clusters of eight run at a time, 64 of four, 144 of two, and half as many with one (one more than that, and the
// last come second: 384 tokens, 4096 -> 1536 on 36 clusters 19 us instead of 12).
struct FewShape { int N, tiles, splits; bool half, wide; };   // half: two CTAs share an SM's memory; wide: sixteen epilogue warps
FewShape few_shape(int T, int M, int kb_total) {
  FewShape f;
  f.N = T < kFewTokens ? (T + 15) / 16 * 16 : kFewTokens;
  f.tiles = (int)((int64_t)((M + 127) / 128) * ((T + f.N - 1) / f.N));
  f.splits = f.tiles <= 28 ? 8 : f.tiles <= 60 ? 4 : f.tiles <= 140 ? 2 : 1;
  while (f.splits > kb_total) f.splits /= 2;
  // (each CTA finishes its share of the tokens in rounds of as many as it has warps, some 0.35 us each: 128 -> 4096, 128 tokens 8.3 us with
  // four epilogue warps and 6.4 with sixteen; where a cluster of eight shares them, 9.2 and 10.0)
  f.wide = f.N > 32 && f.splits <= 2;
  f.half = f.tiles > (f.splits == 8 ? 16 : f.splits == 4 ? 32 : f.splits == 2 ? 72 : 148);
  return f;
}

// Which kernel and which tile, by what they take for the call (us; M tokens, N features, k-blocks of 128 bytes).  The pairs: rounds of
// tiles, 0.29 to 0.38 us a k-block (what shared memory moves; less while half the chip is idle), a start and an end.  The kernel
// for few tokens: the bytes that its CTAs bring into an SM (85 a ns for one, 120 for two), and adding up.  Measured in us, few
// tokens / 128 columns / 256 columns, bf16 with a residual:
//   768 -> 2048   1 token 5.1/9.3/11.5    128 9.2/10.1/12.7   512 8.3/10.5/12.8   2048 13.5/15.2/13.5   8000 47.7/38.3/31.4
//   4096 -> 1536  1 token 6.1/23.7/26.0   128 9.7/24.5/27.2   512 15.0/24.9/27.4  1501 27.9/26.0/28.7   8000 105/123/79
//   4096 -> 128   1 token 6.0/23.2/24.5   512 8.9/24.2/25.0   8000 18.3/25.3/27.1
//   128 -> 4096   1 token 3.9/6.6/8.8     512 8.9/7.6/10.2    8000 66.3/47.8/47.5
enum LinearForm { kFew, kPairs128, kPairs256 };
constexpr double kLaunchUs = 2.0;                        // from one kernel of a call to the next
struct FormTime { LinearForm form; double us; };
FormTime linear_form(const unipool_ctx* ctx, int M, int N, int kb, bool plain) {
  const int pairs = ctx->sm_count / 2;
  auto by_pairs = [&](int n, double busy, double alone, double rest) {
    const int64_t rounds = ((int64_t)((M + 255) / 256) * ((N + n - 1) / n) + pairs - 1) / pairs;
    return (double)rounds * (kb * (rounds > 1 ? busy : alone) + 1.0) + rest;
  };
  const double p128 = by_pairs(128, 0.33, 0.30, plain ? 3.3 : 5.0), p256 = by_pairs(256, 0.38, 0.29, plain ? 4.1 : 8.0);
  if (M <= 16 * 1024) {
    const FewShape f = few_shape(M, N, kb);
    const double ctas = (double)f.tiles * f.splits / ctx->sm_count, each = (kb + f.splits - 1) / f.splits * (16.0 + f.N / 8.0);
    const double few = 3.2 + (f.wide ? 0.02 : 0.03) * f.N + (ctas > 1.0 ? 1.7 + ctas * each / 120.0 : each / 85.0);
    // (several rounds of its CTAs never were the fastest; and one accumulator for all of a CTA's contraction)
    if (ctas <= 2.0 && few < p128 && few < p256 && (kb + f.splits - 1) / f.splits <= kFewLong) return {kFew, few};
  }
  return p128 < p256 ? FormTime{kPairs128, p128} : FormTime{kPairs256, p256};
}

template <int KIND>
int few_as(unipool_ctx* ctx, int phase, const CUtensorMap& tmW, const CUtensorMap& tmX, FewParams p, cudaStream_t s) {
  const FewShape f = few_shape(p.T, p.M, p.kb_total);
  const int splits = f.splits;
  const uint32_t room = (f.half ? 113000u : 232448u) - 2048u, stage = kLinHalf + p.N * 128;
  const int most = (int)(room / stage), need = (p.kb_total + splits - 1) / splits;
  p.stages = most < kFewMaxStages ? most : kFewMaxStages;
  if (p.stages > need) p.stages = need;
  const uint32_t bytes = p.stages * stage > p.N * 512u ? p.stages * stage : p.N * 512u;   // the sums lie there too
  auto as = [&](auto e) {
    constexpr int E = decltype(e)::value;
    auto run = splits == 2 ? launch_few<KIND, 2, E> : launch_few<KIND, 1, E>;
    if constexpr (E == 4) {                              // (few_shape takes sixteen warps for no more than two CTAs)
      if (splits == 8) run = launch_few<KIND, 8, E>;
      if (splits == 4) run = launch_few<KIND, 4, E>;
    }
    return run(ctx, phase, tmW, tmX, p, std::max(2048 + bytes, kFewSmemLeast), s);
  };
  return f.wide ? as(std::integral_constant<int, 16>()) : as(std::integral_constant<int, 4>());
}

}  // namespace

static int linear_few(unipool_ctx* ctx, const LinearArgs& a, cudaStream_t s) {
  const bool q8 = a.x_scale != nullptr;
  const int kb = q8 ? 128 : 64;
  FewParams p{};
  p.T = a.T; p.M = a.n_out;
  p.kb_total = (a.n_in + kb - 1) / kb;
  p.N = few_shape(p.T, p.M, p.kb_total).N;
  p.act = a.act;
  p.bias = a.bias; p.x_scale = a.x_scale; p.w_scale = a.w_scale;
  p.residual = static_cast<const __nv_bfloat16*>(a.residual);
  p.pre = static_cast<__nv_bfloat16*>(a.pre); p.y = static_cast<__nv_bfloat16*>(a.y);
  p.status = ctx->ws.status;
  CUtensorMap tmW, tmX;
  const MapKind kind = q8 ? kMapByteOperand : kMapOperand;
  UP_TRY(map_2d(ctx, &tmW, a.W, a.n_in, a.n_out, kb, 128, kind));
  UP_TRY(map_2d(ctx, &tmX, a.x, a.n_in, a.T, kb, p.N, kind));
  return q8 ? few_as<kLinFwd8>(ctx, UNIPOOL_PH_LINEAR, tmW, tmX, p, s) : few_as<kLinFwd>(ctx, UNIPOOL_PH_LINEAR, tmW, tmX, p, s);
}

static int linear_few_dx(unipool_ctx* ctx, const LinearBwdArgs& a, const void* dp, cudaStream_t s) {
  FewParams p{};
  p.T = a.T; p.M = a.n_in;
  p.kb_total = a.n_out / 64;
  p.N = few_shape(p.T, p.M, p.kb_total).N;
  p.residual = static_cast<const __nv_bfloat16*>(a.dx_residual);
  p.y = static_cast<__nv_bfloat16*>(a.dx);
  p.status = ctx->ws.status;
  CUtensorMap tmW, tmX;
  UP_TRY(map_mn(ctx, &tmW, a.W, a.n_in, a.n_out, 2));
  UP_TRY(map_2d(ctx, &tmX, dp, a.n_out, a.T, 64, p.N));
  return few_as<kLinDx>(ctx, UNIPOOL_PH_LINEAR_BWD, tmW, tmX, p, s);
}

int linear_fwd_tc(unipool_ctx* ctx, const LinearArgs& a, cudaStream_t s) {
  const bool q8 = a.x_scale != nullptr;
  const int kb = q8 ? 128 : 64;
  const LinearForm form = linear_form(ctx, a.T, a.n_out, (a.n_in + kb - 1) / kb, a.bias == nullptr && a.act == UNIPOOL_ACT_NONE).form;
  if (form == kFew) return linear_few(ctx, a, s);
  const int tile_n = form == kPairs128 ? 128 : 256;
  LinearParams p{};
  p.g = linear_grid(a.T, a.n_out, tile_n, (a.n_in + kb - 1) / kb, 1);
  p.status = ctx->ws.status;
  p.act = a.act;
  p.bias = a.bias; p.x_scale = a.x_scale; p.w_scale = a.w_scale;
  p.pre = a.pre != nullptr;
  p.vec = aligned(16, a.bias, a.w_scale);
  p.residual = static_cast<const __nv_bfloat16*>(a.residual);
  p.wide = aligned(32, a.residual);
  LinearMaps m{};
  const MapKind kind = q8 ? kMapByteOperand : kMapOperand;
  UP_TRY(map_2d(ctx, &m.a, a.x, a.n_in, a.T, kb, 128, kind));
  UP_TRY(map_2d(ctx, &m.b, a.W, a.n_in, a.n_out, kb, tile_n / 2, kind));
  UP_TRY(map_2d(ctx, &m.c, a.y, a.n_out, a.T, kLinChunk, 32, kMapBf16Chunk));
  if (a.residual != nullptr) UP_TRY(map_2d(ctx, &m.r, a.residual, a.n_out, a.T, kLinChunk, 32, kMapBf16Chunk));
  if (a.pre != nullptr) UP_TRY(map_2d(ctx, &m.p, a.pre, a.n_out, a.T, kLinChunk, 32, kMapBf16Chunk));
  auto as = [&](auto n) {
    constexpr int N = decltype(n)::value;
    auto run = a.residual == nullptr ? (q8 ? launch_linear<kLinFwd8, N, false, false> : launch_linear<kLinFwd, N, false, false>)
               : a.pre == nullptr    ? (q8 ? launch_linear<kLinFwd8, N, true, false> : launch_linear<kLinFwd, N, true, false>)
                                     : (q8 ? launch_linear<kLinFwd8, N, true, true> : launch_linear<kLinFwd, N, true, true>);
    return run(ctx, UNIPOOL_PH_LINEAR, m, p, s);
  };
  return tile_n == 256 ? as(std::integral_constant<int, 256>()) : as(std::integral_constant<int, 128>());
}

namespace {

int dx_maps(unipool_ctx* ctx, LinearMaps& m, const LinearBwdArgs& a, const void* dp, int tile_n) {
  UP_TRY(map_2d(ctx, &m.a, dp, a.n_out, a.T, 64, 128));
  UP_TRY(map_mn(ctx, &m.b, a.W, a.n_in, a.n_out, tile_n / 128));
  UP_TRY(map_2d(ctx, &m.c, a.dx, a.n_in, a.T, kLinChunk, 32, kMapBf16Chunk));
  if (a.dx_residual != nullptr) UP_TRY(map_2d(ctx, &m.r, a.dx_residual, a.n_in, a.T, kLinChunk, 32, kMapBf16Chunk));
  return UNIPOOL_OK;
}
int dw_maps(unipool_ctx* ctx, CUtensorMap& ma, CUtensorMap& mb, const LinearBwdArgs& a, const void* dp, int tile_n) {
  UP_TRY(map_mn(ctx, &ma, dp, a.n_out, a.T, 2));
  return map_mn(ctx, &mb, a.x, a.n_in, a.T, tile_n / 128);
}
LinearParams bwd_params(const unipool_ctx* ctx, const LinearBwdArgs& a, float* out, bool add) {
  LinearParams p{};
  p.status = ctx->ws.status;
  p.residual = static_cast<const __nv_bfloat16*>(a.dx_residual);
  p.wide = aligned(32, a.dx_residual);
  p.add = add;
  p.dw = out;
  p.wide_dw = aligned(32, out);
  return p;
}

}  // namespace

int linear_dx_tc(unipool_ctx* ctx, const LinearBwdArgs& a, const void* dp, cudaStream_t s) {
  const LinearForm form = linear_form(ctx, a.T, a.n_in, a.n_out / 64, true).form;
  if (form == kFew) return linear_few_dx(ctx, a, dp, s);
  const int tile_n = form == kPairs128 ? 128 : 256;
  LinearParams p = bwd_params(ctx, a, nullptr, false);
  p.g = linear_grid(a.T, a.n_in, tile_n, a.n_out / 64, 1);
  LinearMaps m{};
  UP_TRY(dx_maps(ctx, m, a, dp, tile_n));
  auto as = [&](auto n) {
    constexpr int N = decltype(n)::value;
    auto run = a.dx_residual != nullptr ? launch_linear<kLinDx, N, true, false> : launch_linear<kLinDx, N, false, false>;
    return run(ctx, UNIPOOL_PH_LINEAR_BWD, m, p, s);
  };
  return tile_n == 256 ? as(std::integral_constant<int, 256>()) : as(std::integral_constant<int, 128>());
}

// How the weight gradient is taken: the parts of the tokens, so that its tiles fill the CTA pairs, and whether dx's tiles go into the same
// launch behind its own (short tiles after long ones).  Each by its time in us: a pair's tiles (0.29 us a k-block, 0.38 while all pairs are
// busy, an epilogue at least), the parts' sums (6 bytes a ns written and read, and a launch), a launch between two kernels.  Measured
// in us (tokens, n_in, n_out), two launches / one with 128 columns / with 256:
//   8 192 3584 13/21/22      128 2048 768 18/9/11     493 1408 960 20/11/12     820 4096 1536 32/36/27   1501 768 2048 28/24/17
//   1501 1536 4096 49/50/36  4000 256 512 20/12/14    4000 1536 4096 96/128/78  16384 768 2048 88/127/88  32768 1536 1536 239/338/239
LinearDwPlan linear_dw_plan_tc(const unipool_ctx* ctx, int T, int n_in, int n_out, bool with_dx) {
  const int kb = (T + 63) / 64, pairs = ctx->sm_count / 2, kb_x = n_out / 64;
  LinearDwPlan best{1, 0};
  double least = 0.0;
  const double apart = with_dx ? linear_form(ctx, T, n_in, kb_x, true).us + kLaunchUs + 3.3 : 0.0;
  auto consider = [&](int tile, bool together) {
    const int across = (n_in + tile - 1) / tile, tiles = ((n_out + 255) / 256) * across;
    const int64_t units_x = together ? ((int64_t)T + 255) / 256 * across : 0;
    const double end = tile == 256 ? 3.5 : 2.0;
    for (int splits = 1; splits <= 64 && splits <= kb && (splits == 1 || tiles * (splits - 1) < 2 * pairs); ++splits) {
      const int len = (kb + splits - 1) / splits, parts = (kb + len - 1) / len;
      if (parts != splits) continue;
      // pair q takes units q, q + pairs, ...; the last to end is the first of one of these
      const int64_t units_w = (int64_t)tiles * splits, all = units_w + units_x;
      double us = 0.0;
      for (const int64_t q : {(int64_t)0, units_w % pairs, all % pairs}) {
        const int64_t n = (all - q + pairs - 1) / pairs, w = q < units_w ? (units_w - q + pairs - 1) / pairs : 0;
        const double busy = ((double)units_w * len + (double)units_x * kb_x) / ((double)pairs * (double)(w * len + (n - w) * kb_x));
        const double each = 0.29 + 0.09 * std::min(1.0, busy * busy);
        us = std::max(us, w * std::max(len * each + 1.0, end) + (n - w) * std::max(kb_x * each + 1.0, end));
      }
      us += together ? (tile == 256 ? 6.3 : 4.4) : with_dx ? apart : 0.0;
      if (splits > 1) us += 3.0 + 8.0 * splits * n_in * n_out / 6.0e6;
      if (least == 0.0 || us < least) { best = {splits, together ? tile : 0}; least = us; }
    }
  };
  consider(256, false);
  if (with_dx) {
    consider(128, true);
    consider(256, true);
  }
  return best;
}

// out [splits, n_out, n_in]: the parts' sums, or with one part the gradient.
int linear_dw_tc(unipool_ctx* ctx, const LinearBwdArgs& a, const void* dp, float* out, const LinearDwPlan& plan, bool add, cudaStream_t s) {
  const int kb = (a.T + 63) / 64, tile_n = plan.dx_tile == 128 ? 128 : 256;
  LinearParams p = bwd_params(ctx, a, out, add);
  LinearMaps m{};
  const LinearGrid w = linear_grid(a.n_out, a.n_in, tile_n, kb, plan.splits);
  if (plan.dx_tile == 0) {
    p.g = w;
    UP_TRY(dw_maps(ctx, m.a, m.b, a, dp, tile_n));
    return launch_linear<kLinDw, 256, false, false>(ctx, UNIPOOL_PH_LINEAR_BWD, m, p, s);
  }
  p.w = w;
  p.g = linear_grid(a.T, a.n_in, tile_n, a.n_out / 64, 1);
  UP_TRY(dx_maps(ctx, m, a, dp, tile_n));
  UP_TRY(dw_maps(ctx, m.wa, m.wb, a, dp, tile_n));
  auto as = [&](auto n) {
    constexpr int N = decltype(n)::value;
    auto run = a.dx_residual != nullptr ? launch_linear<kLinBoth, N, true, false> : launch_linear<kLinBoth, N, false, false>;
    return run(ctx, UNIPOOL_PH_LINEAR_BWD, m, p, s);
  };
  return tile_n == 256 ? as(std::integral_constant<int, 256>()) : as(std::integral_constant<int, 128>());
}

}  // namespace unipool
