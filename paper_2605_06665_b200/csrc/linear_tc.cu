// Dense products on the 5th-generation tensor cores, each with its epilogue:
//   forward   y  = act(x W^T s_x s_w + bias) + residual   x, W K-major, bf16 or e4m3 with scales
//   dx        dx = dp W (+ dx_residual)                   W MN-major
//   dW        dW (+)= dp^T x                              both MN-major, fp32 out
//
// linear_pair_kernel: persistent CTA pairs as in the grouped kernels (expert_tc.cu): 256 x 256 tiles, M = 256 over both CTAs'
// tensor memory, six 32 KB operand stages a CTA, accumulators double-buffered so that a tile's epilogue runs beside the next
// one's products.  Eight epilogue warps, two to a TMEM lane quarter with 128 columns each: an activation costs two
// special-function instructions an element, which four warps could not hide behind the products of 768 inputs.
// The residual comes by TMA into the staging tile that the result leaves from, a chunk of 32 x 32 ahead.
// Bound by the tensor pipe (operands through shared memory; see expert_tc.cu) and, held for long, by power.
#include <cuda.h>

#include "common.cuh"
#include "linear_act.cuh"
#include "tc_maps.cuh"
#include "tc_ptx.cuh"

namespace unipool {

namespace {

enum LinearKind { kLinFwd, kLinFwd8, kLinDx, kLinDw };

constexpr uint32_t kLinHalf = 128 * 128;                 // 128 rows (columns) x 128 bytes of one operand
constexpr uint32_t kLinStage = 2 * kLinHalf;
constexpr uint32_t kLinBars = 229376;                    // operand stages + staging fill this much
constexpr uint32_t kLinSmem = kLinBars + 512 + 1024;
constexpr int kLinEpiWarps = 8;
constexpr int kLinThreads = 64 + 32 * kLinEpiWarps;
constexpr int kLinChunk = 32;
constexpr uint32_t kLinBf16Chunk = 32 * kLinChunk * 2, kLinF32Chunk = 32 * kLinChunk * 4;
// The tensor core truncates the sums it adds to: a sum over K terms loses 1.1e-9 K of itself (measured, 512 to 32768 rows).  The
// weight gradient, an fp32 result of a sum over all tokens, is therefore taken from the accumulator every 768 tokens and
// added up in registers, where it is rounded to nearest.
constexpr int kLinSegment = 12;                          // k-blocks of 64 tokens

struct LinearParams {
  int M, N;                          // rows and columns of the result
  int n_mt, n_nt, units, kb_total, kb_split;
  int act;
  const float *bias, *x_scale, *w_scale;
  bool residual, add, vec;           // vec: bias and w_scale are 16-byte aligned
  int32_t* status;
};

struct LinearUnit { int mt, nt, split, kb0, kb1; };
__device__ __forceinline__ LinearUnit linear_unit(const LinearParams& p, int u) {
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

// 16-byte piece q of row r of a staging tile in the layout of the TMA swizzle: rows of 64 bytes, rows of 128.
__device__ __forceinline__ uint4* piece64(uint8_t* tile, int r, int q) {
  return reinterpret_cast<uint4*>(tile + r * 64 + ((q ^ ((r >> 1) & 3)) << 4));
}
__device__ __forceinline__ uint4* piece128(uint8_t* tile, int r, int q) {
  return reinterpret_cast<uint4*>(tile + r * 128 + ((q ^ (r & 7)) << 4));
}
__device__ __forceinline__ void put_row(uint8_t* tile, int r, const float (&v)[32]) {
#pragma unroll
  for (int q = 0; q < 4; ++q)
    *piece64(tile, r, q) = make_uint4(tc::pack_bf16(v[8 * q], v[8 * q + 1]), tc::pack_bf16(v[8 * q + 2], v[8 * q + 3]),
                                      tc::pack_bf16(v[8 * q + 4], v[8 * q + 5]), tc::pack_bf16(v[8 * q + 6], v[8 * q + 7]));
}
__device__ __forceinline__ void add_row(uint8_t* tile, int r, float (&v)[32]) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const uint4 w = *piece64(tile, r, q);
    const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[8 * q + 2 * i] += __uint_as_float(ww[i] << 16);
      v[8 * q + 2 * i + 1] += __uint_as_float(ww[i] & 0xffff0000u);
    }
  }
}
// v = f(v, column's number) for the 32 columns from `p` on, the same in all lanes
template <typename F> __device__ __forceinline__ void by_column(const float* p, bool vec, float (&v)[32], F f) {
#pragma unroll
  for (int q = 0; q < 8; ++q) {
    const float4 b = vec ? __ldg(reinterpret_cast<const float4*>(p) + q)
                         : make_float4(__ldg(p + 4 * q), __ldg(p + 4 * q + 1), __ldg(p + 4 * q + 2), __ldg(p + 4 * q + 3));
    v[4 * q] = f(v[4 * q], b.x);
    v[4 * q + 1] = f(v[4 * q + 1], b.y);
    v[4 * q + 2] = f(v[4 * q + 2], b.z);
    v[4 * q + 3] = f(v[4 * q + 3], b.w);
  }
}
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

// kPre: the value before the activation is stored too; two more staging tiles a warp take an operand stage.
template <int KIND, bool kPre>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kLinThreads, 1)
linear_pair_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                   const __grid_constant__ CUtensorMap tmC, const __grid_constant__ CUtensorMap tmR,
                   const __grid_constant__ CUtensorMap tmP, LinearParams p) {
  constexpr int kStages = kPre ? 5 : 6;
  constexpr uint32_t kStaging = (kLinBars - kStages * kLinStage) / kLinEpiWarps;
  static_assert(kStaging >= (kPre ? 4 : 2) * kLinBf16Chunk && kStaging >= kLinF32Chunk, "staging tiles");
  constexpr bool kAMn = KIND == kLinDw, kBMn = KIND == kLinDx || KIND == kLinDw;
  constexpr int kKb = KIND == kLinFwd8 ? 128 : 64;       // elements of a k-block
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* full_bar = reinterpret_cast<uint64_t*>(smem + kLinBars);
  uint64_t* empty_bar = full_bar + kStages;
  uint64_t* tmem_full = empty_bar + kStages;
  uint64_t* tmem_empty = tmem_full + 2;
  uint64_t* res_bar = tmem_empty + 2;                    // [8][2] a chunk of the residual has landed
  uint32_t* tmem_ptr = reinterpret_cast<uint32_t*>(res_bar + 2 * kLinEpiWarps);
  volatile int* abort = reinterpret_cast<volatile int*>(tmem_ptr + 1);
  static_assert((2 * kStages + 4 + 2 * kLinEpiWarps) * 8 + 8 <= 512, "barrier block");

  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int rank = (int)tc::cluster_ctarank();           // 0 = leader
  const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) { tc::mbar_init(&full_bar[s], 1); tc::mbar_init(&empty_bar[s], 1); }
    for (int a = 0; a < 2; ++a) { tc::mbar_init(&tmem_full[a], 1); tc::mbar_init(&tmem_empty[a], 2 * kLinEpiWarps); }
    for (int i = 0; i < 2 * kLinEpiWarps; ++i) tc::mbar_init(&res_bar[i], 1);
    *abort = 0;
    tc::fence_barrier_init();
    tc::tma_prefetch_desc(&tmA);
    tc::tma_prefetch_desc(&tmB);
    tc::tma_prefetch_desc(&tmC);
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
  grid_wait(p.bias, p.x_scale, p.w_scale);

  if (warp == 0) {
    // ------------------------------------------------------------ TMA producer (one in each CTA)
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int u = pair; u < p.units && ok; u += n_pairs) {
        const LinearUnit t = linear_unit(p, u);
        for (int kb = t.kb0; kb < t.kb1; ++kb) {
          if (!tc::mbar_wait(&empty_bar[stage], phase ^ 1u, abort)) { linear_timeout(p.status, abort, 41); ok = false; break; }
          uint8_t* sA = smem + stage * kLinStage;
          uint8_t* sB = sA + kLinHalf;
          if (rank == 0) tc::mbar_expect_tx(&full_bar[stage], 2 * kLinStage);      // both CTAs' bytes
          if constexpr (kAMn) tc::tma_load_3d_pair(sA, &tmA, &full_bar[stage], 0, kb * kKb, t.mt * 4 + rank * 2);
          else tc::tma_load_2d_pair(sA, &tmA, &full_bar[stage], kb * kKb, t.mt * 256 + rank * 128);
          if constexpr (kBMn) tc::tma_load_3d_pair(sB, &tmB, &full_bar[stage], 0, kb * kKb, t.nt * 4 + rank * 2);
          else tc::tma_load_2d_pair(sB, &tmB, &full_bar[stage], kb * kKb, t.nt * 256 + rank * 128);
          if (++stage == kStages) { stage = 0; phase ^= 1u; }
        }
      }
      if (!ok)
        for (int i = 0; i < 200; ++i) __nanosleep(1000);  // let loads already in flight land before the CTA retires
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMA issuer (leader CTA only)
    if (lane == 0 && rank == 0) {
      constexpr uint32_t idesc = KIND == kLinFwd8 ? tc::instr_desc_e4m3(256, 256) : tc::instr_desc_bf16(256, kAMn, kBMn, 256);
      constexpr uint32_t a_lbo = kAMn ? kLinHalf / 2 : 16, b_lbo = kBMn ? kLinHalf / 2 : 16;
      constexpr uint32_t a_step = (kAMn ? 16 * 128 : 32) >> 4, b_step = (kBMn ? 16 * 128 : 32) >> 4;
      int stage = 0, local = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int u = pair; u < p.units && ok; u += n_pairs) {
        const LinearUnit t = linear_unit(p, u);
        for (int kb = t.kb0; kb < t.kb1 && ok;) {
          const int end = KIND == kLinDw ? min(t.kb1, kb + kLinSegment) : t.kb1;
          const int acc = local & 1;
          if (!tc::mbar_wait(&tmem_empty[acc], ((local >> 1) & 1) ^ 1u, abort)) { linear_timeout(p.status, abort, 42); ok = false; break; }
          ++local;
          tc::tc_fence_after_sync();
          const uint32_t d_tmem = tmem_base + acc * 256;
          uint32_t accumulate = 0;
          for (; kb < end; ++kb) {
            if (!tc::mbar_wait(&full_bar[stage], phase, abort)) { linear_timeout(p.status, abort, 43); ok = false; break; }
            tc::tc_fence_after_sync();
            const uint32_t a = tc::smem_u32(smem + stage * kLinStage);
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
    // ------------------------------------------------------------ epilogue: 32 rows and 128 columns of the tile to a warp
    const int quarter = warp & 3, ew = warp - 2, half = ew >> 2;
    uint8_t* stg = smem + kStages * kLinStage + ew * kStaging;
    uint64_t* my_res = res_bar + 2 * ew;
    const uint32_t lanes = static_cast<uint32_t>(quarter * 32) << 16;
    int local = 0;
    uint32_t chunk = 0, loaded = 0;                       // chunks staged, chunks of the residual asked for
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
    for (int u = pair; u < p.units && ok; u += n_pairs) {
      const LinearUnit t = linear_unit(p, u);
      const int row0 = t.mt * 256 + rank * 128 + quarter * 32, col0 = t.nt * 256 + half * 128;
      const int nch = row0 < p.M ? max(0, min(4, (p.N - col0 + kLinChunk - 1) / kLinChunk)) : 0;
      if constexpr (KIND == kLinDw) {
        float sum[4][32];
        for (int kb = t.kb0, first = 1; kb < t.kb1 && ok; kb += kLinSegment, first = 0) {
          const int acc = local & 1;
          ok = wait_full(acc);
          if (!ok) break;
#pragma unroll
          for (int ch = 0; ch < 4; ++ch) {
            uint32_t rr[32];
            tc::tmem_ld_32x32(tmem_base + lanes + acc * 256 + half * 128 + ch * kLinChunk, rr);
            tc::tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 32; ++i) sum[ch][i] = first ? __uint_as_float(rr[i]) : sum[ch][i] + __uint_as_float(rr[i]);
          }
          release(acc);
        }
        if (!ok) break;
#pragma unroll
        for (int ch = 0; ch < 4; ++ch) {
          if (ch >= nch) continue;
          if (lane == 0) tc::bulk_wait_read<0>();
          __syncwarp();
#pragma unroll
          for (int q = 0; q < 8; ++q)
            *piece128(stg, lane, q) = make_uint4(__float_as_uint(sum[ch][4 * q]), __float_as_uint(sum[ch][4 * q + 1]),
                                                 __float_as_uint(sum[ch][4 * q + 2]), __float_as_uint(sum[ch][4 * q + 3]));
          tc::fence_proxy_async();
          __syncwarp();
          if (lane == 0) {
            // (rows of the splits lie one after the other, M each: a tile that reaches beyond M ends at a warp's edge, M being
            // a multiple of 64)
            const int col = col0 + ch * kLinChunk, row = t.split * p.M + row0;
            if (p.add) tc::tma_reduce_add_2d(&tmC, stg, col, row);
            else tc::tma_store_2d(&tmC, stg, col, row);
            tc::bulk_commit();
          }
        }
      } else {
        const int acc = local & 1;
        auto ask = [&](int ch) {                          // lane 0: chunk ch of the residual into its staging tile
          tc::bulk_wait_read<0>();                        // the store that last left from there
          uint64_t* bar = &my_res[loaded & 1];
          tc::mbar_expect_tx(bar, kLinBf16Chunk);
          tc::tma_load_2d(stg + (loaded & 1) * kLinBf16Chunk, &tmR, bar, col0 + ch * kLinChunk, row0);
        };
        if (p.residual && nch > 0) {
          if (lane == 0) ask(0);
          ++loaded;
        }
        float xs = 1.f;
        if (KIND == kLinFwd8 && row0 + lane < p.M) xs = __ldg(p.x_scale + row0 + lane);
        ok = wait_full(acc);
        if (!ok) break;
#pragma unroll 1
        for (int ch = 0; ch < nch; ++ch, ++chunk) {
          const int col = col0 + ch * kLinChunk;
          uint32_t rr[32];
          tc::tmem_ld_32x32(tmem_base + lanes + acc * 256 + half * 128 + ch * kLinChunk, rr);
          if (p.residual && ch + 1 < nch) {
            if (lane == 0) ask(ch + 1);
            ++loaded;
          }
          tc::tmem_ld_wait();
          float v[32];
#pragma unroll
          for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(rr[i]);
          if constexpr (KIND == kLinFwd8) by_column(p.w_scale + col, p.vec, v, [&](float a, float s) { return a * (xs * s); });
          uint8_t* buf = stg + (chunk & 1) * kLinBf16Chunk;
          if constexpr (KIND != kLinDx) {
            if (p.bias != nullptr) by_column(p.bias + col, p.vec, v, [](float a, float b) { return a + b; });
            if constexpr (kPre) {
              if (lane == 1) tc::bulk_wait_read<1>();     // the store of two chunks ago
              __syncwarp();
              put_row(buf + 2 * kLinBf16Chunk, lane, v);
            }
            activate(v, p.act);
          }
          if (p.residual) {
            ok = tc::mbar_wait_warp(&my_res[chunk & 1], (chunk >> 1) & 1, abort);
            if (!ok) {
              if (lane == 0) linear_timeout(p.status, abort, 45);
              break;
            }
            add_row(buf, lane, v);
          } else {
            if (lane == 0) tc::bulk_wait_read<1>();
            __syncwarp();
          }
          put_row(buf, lane, v);
          tc::fence_proxy_async();
          __syncwarp();
          if (lane == 0) { tc::tma_store_2d(&tmC, buf, col, row0); tc::bulk_commit(); }
          if (kPre && lane == 1) { tc::tma_store_2d(&tmP, buf + 2 * kLinBf16Chunk, col, row0); tc::bulk_commit(); }
        }
        if (!ok) break;
        release(acc);
      }
    }
    if (!ok && lane == 0)
      for (int i = 0; i < 200; ++i) __nanosleep(1000);
    if (lane < 2) tc::bulk_wait<0>();
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

LinearParams linear_params(const unipool_ctx* ctx, int M, int N, int kb_total, int splits) {
  LinearParams p{};
  p.M = M; p.N = N;
  p.n_mt = (M + 255) / 256; p.n_nt = (N + 255) / 256;
  p.kb_total = kb_total;
  p.kb_split = (kb_total + splits - 1) / splits;
  p.units = p.n_mt * p.n_nt * ((kb_total + p.kb_split - 1) / p.kb_split);
  p.status = ctx->ws.status;
  return p;
}

template <int KIND, bool kPre>
int launch_linear(unipool_ctx* ctx, int phase, const CUtensorMap& tmA, const CUtensorMap& tmB, const CUtensorMap& tmC,
                  const CUtensorMap& tmR, const CUtensorMap& tmP, const LinearParams& p, cudaStream_t s) {
  PhaseTimer pt(ctx, phase, 1, s);
  auto kern = linear_pair_kernel<KIND, kPre>;
  UP_CUDA(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kLinSmem));
  const int pairs = ctx->sm_count / 2;
  UP_KERNEL(kern, 2 * (p.units < pairs ? p.units : pairs), kLinThreads, kLinSmem, s, tmA, tmB, tmC, tmR, tmP, p);
  return UNIPOOL_OK;
}

#define UP_TRY(call)                     \
  do {                                   \
    const int rc__ = (call);             \
    if (rc__ != UNIPOOL_OK) return rc__; \
  } while (0)

}  // namespace

int linear_fwd_tc(unipool_ctx* ctx, const LinearArgs& a, cudaStream_t s) {
  const bool q8 = a.x_scale != nullptr;
  const int kb = q8 ? 128 : 64;
  LinearParams p = linear_params(ctx, a.T, a.n_out, (a.n_in + kb - 1) / kb, 1);
  p.act = a.act;
  p.bias = a.bias; p.x_scale = a.x_scale; p.w_scale = a.w_scale;
  p.residual = a.residual != nullptr;
  p.vec = ((reinterpret_cast<uintptr_t>(a.bias) | reinterpret_cast<uintptr_t>(a.w_scale)) & 15) == 0;
  CUtensorMap tmA, tmB, tmC, tmR, tmP;
  const MapKind kind = q8 ? kMapByteOperand : kMapOperand;
  UP_TRY(map_2d(ctx, &tmA, a.x, a.n_in, a.T, kb, 128, kind));
  UP_TRY(map_2d(ctx, &tmB, a.W, a.n_in, a.n_out, kb, 128, kind));
  UP_TRY(map_2d(ctx, &tmC, a.y, a.n_out, a.T, kLinChunk, 32, kMapBf16Chunk));
  tmR = tmP = tmC;
  if (a.residual != nullptr) UP_TRY(map_2d(ctx, &tmR, a.residual, a.n_out, a.T, kLinChunk, 32, kMapBf16Chunk));
  if (a.pre != nullptr) UP_TRY(map_2d(ctx, &tmP, a.pre, a.n_out, a.T, kLinChunk, 32, kMapBf16Chunk));
  if (q8) return a.pre ? launch_linear<kLinFwd8, true>(ctx, UNIPOOL_PH_LINEAR, tmA, tmB, tmC, tmR, tmP, p, s)
                       : launch_linear<kLinFwd8, false>(ctx, UNIPOOL_PH_LINEAR, tmA, tmB, tmC, tmR, tmP, p, s);
  return a.pre ? launch_linear<kLinFwd, true>(ctx, UNIPOOL_PH_LINEAR, tmA, tmB, tmC, tmR, tmP, p, s)
               : launch_linear<kLinFwd, false>(ctx, UNIPOOL_PH_LINEAR, tmA, tmB, tmC, tmR, tmP, p, s);
}

int linear_dx_tc(unipool_ctx* ctx, const LinearBwdArgs& a, const void* dp, cudaStream_t s) {
  LinearParams p = linear_params(ctx, a.T, a.n_in, a.n_out / 64, 1);
  p.residual = a.dx_residual != nullptr;
  CUtensorMap tmA, tmB, tmC, tmR;
  UP_TRY(map_2d(ctx, &tmA, dp, a.n_out, a.T, 64, 128));
  UP_TRY(map_mn(ctx, &tmB, a.W, a.n_in, a.n_out, 2));
  UP_TRY(map_2d(ctx, &tmC, a.dx, a.n_in, a.T, kLinChunk, 32, kMapBf16Chunk));
  tmR = tmC;
  if (a.dx_residual != nullptr) UP_TRY(map_2d(ctx, &tmR, a.dx_residual, a.n_in, a.T, kLinChunk, 32, kMapBf16Chunk));
  return launch_linear<kLinDx, false>(ctx, UNIPOOL_PH_LINEAR_BWD, tmA, tmB, tmC, tmR, tmC, p, s);
}

// Parts of the tokens that the weight gradient is taken in, so that its tiles fill the CTA pairs: the number with the least
// time for its rounds of tiles (0.3 us a k-block) and for writing and reading the parts' sums (6 bytes a ns).
int linear_dw_splits_tc(const unipool_ctx* ctx, int T, int n_in, int n_out) {
  const int tiles = ((n_out + 255) / 256) * ((n_in + 255) / 256), kb = (T + 63) / 64, pairs = ctx->sm_count / 2;
  int best = 1;
  double least = 0.0;
  for (int splits = 1; splits <= 64 && splits <= kb; ++splits) {
    const int len = (kb + splits - 1) / splits, parts = (kb + len - 1) / len;
    if (parts != splits) continue;
    const int rounds = (tiles * splits + pairs - 1) / pairs;
    const double ns = rounds * (len * 300.0 + 1000.0) + (splits > 1 ? 3000.0 + 8.0 * splits * n_in * n_out / 6.0e3 : 0.0);
    if (splits == 1 || ns < least) { best = splits; least = ns; }
  }
  return best;
}

// out [splits, n_out, n_in]: the parts' sums, or with one part the gradient.
int linear_dw_tc(unipool_ctx* ctx, const LinearBwdArgs& a, const void* dp, float* out, int splits, bool add, cudaStream_t s) {
  LinearParams p = linear_params(ctx, a.n_out, a.n_in, (a.T + 63) / 64, splits);
  p.add = add;
  CUtensorMap tmA, tmB, tmC;
  UP_TRY(map_mn(ctx, &tmA, dp, a.n_out, a.T, 2));
  UP_TRY(map_mn(ctx, &tmB, a.x, a.n_in, a.T, 2));
  UP_TRY(map_2d(ctx, &tmC, out, a.n_in, (uint64_t)splits * a.n_out, kLinChunk, 32, kMapF32Chunk));
  return launch_linear<kLinDw, false>(ctx, UNIPOOL_PH_LINEAR_BWD, tmA, tmB, tmC, tmC, tmC, p, s);
}

}  // namespace unipool
