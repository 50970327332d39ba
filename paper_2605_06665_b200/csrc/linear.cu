// Dense products with an epilogue and their backward pass: the calls, the fp32 path on CUDA cores, and the element-wise
// kernels beside both paths.
//   forward   p = x W^T + bias,  y = act(p) + residual
//   backward  dp = dy act'(p),  dx = dp W (+ dx_residual),  dW (+)= dp^T x,  dbias (+)= sum_t dp
#include <cooperative_groups.h>

#include <algorithm>
#include <type_traits>

#include "common.cuh"
#include "linear_act.cuh"
#include "simt_gemm.cuh"
#include "vec.cuh"

namespace unipool {

namespace {

// ---------------------------------------------------------------- dp and the sums for dbias
// dp = dy act'(p), rounded to the element type, and the column sums of the unrounded dp over the block's rows, into parts
// [gridDim.y, N] (one row block: the gradient itself).  A thread owns V columns and every eighth row of the block's run;
// eight rows' threads are added up in their order.  Bound by HBM (dy, p in, dp out: 201 MB of 16384 x 2048 bf16 in 29 us, 7 TB/s with
// part of dp still in L2), with silu and gelu by the special-function unit beside it (two instructions an element, 15 us).
constexpr int kDpRows = 8, kDpAhead = 4;                 // rows of a block's warps, rows that each has in flight

struct DpParams {
  const void *dy, *p;
  void* dp;
  float* parts;
  int T, N, rows, act;                                   // rows: of a block's run
  bool add;                                              // one row block: dbias +=
};

// the rows of a thread, from t on
template <typename E, int V, bool kFast, int ACT>
__device__ __forceinline__ void dp_run(const DpParams& a, int t, int t1, int c, float (&sum)[V]) {
  const E* gy = static_cast<const E*>(a.dy) + c;
  const E* gp = static_cast<const E*>(a.p) + c;
  for (; t < t1; t += kDpRows * kDpAhead) {
    Vec<E, V> dy[kDpAhead], pre[kDpAhead];
#pragma unroll
    for (int u = 0; u < kDpAhead; ++u) {
      const int row = t + u * kDpRows;
      dy[u].zero();
      if (row >= t1) continue;
      dy[u].load(gy + (int64_t)row * a.N);
      if (ACT != UNIPOOL_ACT_NONE) pre[u].load(gp + (int64_t)row * a.N);
    }
#pragma unroll
    for (int u = 0; u < kDpAhead; ++u) {
      const int row = t + u * kDpRows;
      float d[V], p[V];
      dy[u].get(d);
      if (ACT != UNIPOOL_ACT_NONE && row < t1) {
        pre[u].get(p);
#pragma unroll
        for (int j = 0; j < V; ++j) d[j] *= act_slope<kFast>(p[j], ACT);
        Vec<E, V>::store(static_cast<E*>(a.dp) + ((int64_t)row * a.N + c), d);
      }
#pragma unroll
      for (int j = 0; j < V; ++j) sum[j] += d[j];
    }
  }
}

// Four blocks to an SM, as dp_row_blocks counts (70 registers in fp32 without the bound: 16384 x 2048 gelu 86 us instead of 69).
// C > 1: the row blocks are one cluster, which adds its sums up through each other's shared memory, in the order of the ranks.
template <typename E, int V, bool kFast, int C>
__global__ void __cluster_dims__(1, C, 1) __launch_bounds__(256, 4) linear_dp_kernel(DpParams a) {
  grid_wait(a.dy, a.p);
  __shared__ float s[kDpRows][32 * V];
  __shared__ float sums[C > 1 ? 32 * V : 1];
  const int g = threadIdx.x / 32, lane = threadIdx.x % 32, c = (blockIdx.x * 32 + lane) * V;
  const int t0 = blockIdx.y * a.rows, t1 = min(a.T, t0 + a.rows);
  float sum[V];
#pragma unroll
  for (int j = 0; j < V; ++j) sum[j] = 0.f;
  if (c < a.N) {
    switch (a.act) {
      case UNIPOOL_ACT_NONE: dp_run<E, V, kFast, UNIPOOL_ACT_NONE>(a, t0 + g, t1, c, sum); break;
      case UNIPOOL_ACT_RELU: dp_run<E, V, kFast, UNIPOOL_ACT_RELU>(a, t0 + g, t1, c, sum); break;
      case UNIPOOL_ACT_SILU: dp_run<E, V, kFast, UNIPOOL_ACT_SILU>(a, t0 + g, t1, c, sum); break;
      case UNIPOOL_ACT_GELU: dp_run<E, V, kFast, UNIPOOL_ACT_GELU>(a, t0 + g, t1, c, sum); break;
    }
  }
  if (a.parts == nullptr) return;
#pragma unroll
  for (int j = 0; j < V; ++j) s[g][j * 32 + lane] = sum[j];
  __syncthreads();
  for (int i = threadIdx.x; i < 32 * V; i += 256) {
    const int col = (blockIdx.x * 32 + i % 32) * V + i / 32;
    if (col >= a.N) continue;
    float v = s[0][i];
#pragma unroll
    for (int q = 1; q < kDpRows; ++q) v += s[q][i];
    if constexpr (C > 1) {
      sums[i] = v;
    } else {
      float* out = a.parts + (int64_t)blockIdx.y * a.N + col;
      *out = a.add ? *out + v : v;
    }
  }
  if constexpr (C > 1) {
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    cluster.sync();
    for (int i = blockIdx.y * (32 * V / C) + threadIdx.x; i < (int)(blockIdx.y + 1) * (32 * V / C); i += 256) {
      const int col = (blockIdx.x * 32 + i % 32) * V + i / 32;
      if (col >= a.N) continue;
      float v = *cluster.map_shared_rank(&sums[i], 0);
#pragma unroll
      for (int q = 1; q < C; ++q) v += *cluster.map_shared_rank(&sums[i], q);
      float* out = a.parts + col;
      *out = a.add ? *out + v : v;
    }
    cluster.sync();                                      // no block leaves while another reads its sums
  }
}

constexpr int kDpOneBlock = 3 * kDpRows * kDpAhead;      // so many rows go to one block
// With dbias, up to kDpClusterRows go to a cluster of eight: some steps more in its blocks, but no launch behind them that adds up parts, and no
// scratch (300 x 2048 bf16 relu 3.6 us with it and 3.9 with parts, gelu 4.6 and 4.6, 512 rows 4.0 and 3.9, gelu 5.3 and 4.7; the
// launch and the memory are 3.5 us of the host's time).
constexpr int kDpCluster = 8, kDpClusterRows = 512;
// Rows of each of n row blocks: whole steps of the loop.
int dp_rows(int T, int n) { return ((T + n - 1) / n + kDpRows * kDpAhead - 1) / (kDpRows * kDpAhead) * (kDpRows * kDpAhead); }
// Row blocks of the kernel, of 32 rows at least: four blocks to an SM, as its registers allow, where the special-function unit is to be
// kept busy, three where the rows' bytes are all (16384 x 2048 bf16 with the sum behind it: gelu 35.4 us with four and 37.4 with
// three, relu 35.0 and 33.3); few rows on one, which leaves nothing to add up behind it.
int dp_row_blocks(const unipool_ctx* ctx, int T, int N, int cols_per_block, int act) {
  const int across = (N + cols_per_block - 1) / cols_per_block;
  if (T <= kDpOneBlock) return 1;
  int n = (act == UNIPOOL_ACT_SILU || act == UNIPOOL_ACT_GELU ? 4 : 3) * ctx->sm_count / across;
  if (n > (T + 31) / 32) n = (T + 31) / 32;
  if (n < 1) n = 1;
  return (T + dp_rows(T, n) - 1) / dp_rows(T, n);
}

// ---------------------------------------------------------------- sums of parts, in their order
// out [width] (+)= the sum over n parts [n, width] of type P.
template <typename P> struct PartSum { const P* parts; int n; int64_t width; float* out; bool add; };

// Blocks [0, wide_blocks): few parts of many columns (a weight gradient's), four columns to a thread, 16 bytes at a time.  The others:
// many parts of few columns, a sector of them to a block, whose 32 groups of eight threads take every 32nd part.
template <typename P>
__global__ void __launch_bounds__(256) part_sum_kernel(PartSum<float> wide, int wide_blocks, PartSum<P> tall) {
  grid_wait(wide.parts, tall.parts);
  if ((int)blockIdx.x < wide_blocks) {
    const int64_t c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (c >= wide.width) return;
    float4 v = __ldg(reinterpret_cast<const float4*>(wide.parts + c));
#pragma unroll 4
    for (int i = 1; i < wide.n; ++i) {
      const float4 o = __ldg(reinterpret_cast<const float4*>(wide.parts + i * wide.width + c));
      v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w;
    }
    float* out = &wide.out[c];
    if (wide.add) v = make_float4(v.x + out[0], v.y + out[1], v.z + out[2], v.w + out[3]);
    st4(out, v, (reinterpret_cast<uintptr_t>(out) & 15) == 0);
    return;
  }
  constexpr int V = 4 / (int)sizeof(P);                  // columns of a thread
  __shared__ float s[8][8 * V];
  const int lane = threadIdx.x % 32, g = threadIdx.x / 8;
  const int64_t c = ((int64_t)(blockIdx.x - wide_blocks) * 8 + threadIdx.x % 8) * V;
  float v[V];
#pragma unroll
  for (int j = 0; j < V; ++j) v[j] = 0.f;
  if (c < tall.width) {
#pragma unroll 8
    for (int i = g; i < tall.n; i += 32) {
      Vec<P, V> r;
      float u[V];
      r.load(tall.parts + i * tall.width + c);
      r.get(u);
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] += u[j];
    }
  }
#pragma unroll
  for (int j = 0; j < V; ++j) {
    v[j] += __shfl_xor_sync(0xffffffffu, v[j], 8);
    v[j] += __shfl_xor_sync(0xffffffffu, v[j], 16);
    if (lane < 8) s[threadIdx.x / 32][lane * V + j] = v[j];
  }
  __syncthreads();
  const int64_t col = (int64_t)(blockIdx.x - wide_blocks) * 8 * V + threadIdx.x;
  if (threadIdx.x >= 8 * V || col >= tall.width) return;
  float sum = s[0][threadIdx.x];
#pragma unroll
  for (int i = 1; i < 8; ++i) sum += s[i][threadIdx.x];
  tall.out[col] = tall.add ? tall.out[col] + sum : sum;
}
template <typename P> int part_sum(const PartSum<float>& wide, const PartSum<P>& tall, cudaStream_t s) {   // (one of n = 0: none)
  constexpr int kCols = 8 * 4 / (int)sizeof(P);
  const int a = wide.n > 0 ? (int)((wide.width / 4 + 255) / 256) : 0, b = tall.n > 0 ? (int)((tall.width + kCols - 1) / kCols) : 0;
  if (a + b > 0) UP_KERNEL(part_sum_kernel<P>, a + b, 256, 0, s, wide, a, tall);
  return UNIPOOL_OK;
}

// ---------------------------------------------------------------- fp32 products on CUDA cores
struct SimtLinear {
  const float *A, *B;
  float *C, *P;                                          // P: the value before the activation, or NULL
  const float *bias, *residual;
  int M, N, K, act;                                      // C [M, N]
  int k_len;                                             // dW: tokens of a part
  bool vec_a, vec_b, vec_c, add;                         // 16-byte aligned operands; vec_c: everything of the epilogue
};

template <typename Tile> constexpr int tile_cols = kSimtN;
template <> constexpr int tile_cols<SimtWideTile> = SimtWideTile::kCols;

// C = act(A B + bias) + residual; B along K (forward) or across it (dx).  S blocks of a cluster share a tile by taking runs of its
// contraction and add up through each other's shared memory, in the order of their ranks (few tiles of a long contraction leave
// most SMs idle otherwise: 16 tokens 2048 -> 1728 35 us with one block to a tile, 12 with eight).
template <typename Tile, Major BM, int S>
__global__ void __cluster_dims__(1, 1, S) __launch_bounds__(Tile::kThreads, Tile::kBlocks) linear_rows_kernel(SimtLinear p) {
  grid_wait(p.A, p.B, p.bias, p.residual);
  extern __shared__ float4 smem_raw[];
  typename Tile::Smem& sm = *reinterpret_cast<typename Tile::Smem*>(smem_raw);
  const int m0 = blockIdx.x * Tile::kRows, n0 = blockIdx.y * tile_cols<Tile>;
  const int all = p.K / kSimtKC, c0 = all * (int)blockIdx.z / S, c1 = all * ((int)blockIdx.z + 1) / S;
  Tile t;
  t.template run<kAlongK, BM>(
      sm, c1 - c0, p.vec_a, p.vec_b, p.A, [](int) {},
      [&](int c, int i, int k) { return m0 + i < p.M ? p.A + (int64_t)(m0 + i) * p.K + (c0 + c) * kSimtKC + k : nullptr; },
      [&](int c, int i, int k) -> const float* {
        const int kk = (c0 + c) * kSimtKC + k;
        if (tile_cols<Tile> > kSimtN && n0 + i >= p.N) return nullptr;
        return BM == kAlongK ? p.B + (int64_t)(n0 + i) * p.K + kk : p.B + (int64_t)kk * p.N + n0 + i;
      });
  auto put = [&](int i, int j, float4 v) {
    if (m0 + i >= p.M || (tile_cols<Tile> > kSimtN && n0 + j >= p.N)) return;
    const int n = n0 + j;
    const int64_t at = (int64_t)(m0 + i) * p.N + n;
    if (p.bias != nullptr) {
      const float4 b = ld4(p.bias + n, p.vec_c);
      v = make_float4(v.x + b.x, v.y + b.y, v.z + b.z, v.w + b.w);
    }
    if (p.P != nullptr) st4(p.P + at, v, p.vec_c);
    v = make_float4(act_value<false>(v.x, p.act), act_value<false>(v.y, p.act), act_value<false>(v.z, p.act),
                    act_value<false>(v.w, p.act));
    if (p.residual != nullptr) {
      // (C may be the residual itself: a thread's own elements, and no read-only load)
      const float* r = p.residual + at;
      const float4 b = p.vec_c ? *reinterpret_cast<const float4*>(r) : make_float4(r[0], r[1], r[2], r[3]);
      v = make_float4(v.x + b.x, v.y + b.y, v.z + b.z, v.w + b.w);
    }
    st4(p.C + at, v, p.vec_c);
  };
  if constexpr (S == 1) {
    t.each4(sm, put);
  } else {
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    float* mine = sm.w[0].sums;
    t.each4(sm, [&](int i, int j, float4 v) { *reinterpret_cast<float4*>(&mine[i * kSimtLd + j]) = v; });
    cluster.sync();
    constexpr int kQuads = Tile::kRows * kSimtN / 4;
    for (int q = kQuads / S * (int)blockIdx.z + threadIdx.x; q < kQuads / S * ((int)blockIdx.z + 1); q += Tile::kThreads) {
      const int i = q / (kSimtN / 4), j = q % (kSimtN / 4) * 4;
      float4 part[S];
#pragma unroll
      for (int o = 0; o < S; ++o) part[o] = *reinterpret_cast<const float4*>(&cluster.map_shared_rank(mine, o)[i * kSimtLd + j]);
#pragma unroll
      for (int o = 1; o < S; ++o) {
        part[0].x += part[o].x; part[0].y += part[o].y; part[0].z += part[o].z; part[0].w += part[o].w;
      }
      put(i, j, part[0]);
    }
    cluster.sync();                                      // no block leaves while another reads its sums
  }
}

// C [M, N] (+)= sum over the tokens of a part of A[t, m] B[t, n]; part z of C behind the one before it.
using LinearDwTile = SimtBlockTile<2>;
__global__ void __launch_bounds__(LinearDwTile::kThreads, LinearDwTile::kBlocks) linear_dw_kernel(SimtLinear p) {
  grid_wait(p.A, p.B);
  extern __shared__ float4 smem_raw[];
  LinearDwTile::Smem& sm = *reinterpret_cast<LinearDwTile::Smem*>(smem_raw);
  const int m0 = blockIdx.x * LinearDwTile::kRows, n0 = blockIdx.y * kSimtN;
  const int k0 = blockIdx.z * p.k_len, k1 = min(p.K, k0 + p.k_len);
  LinearDwTile t;
  t.run<kAcrossK, kAcrossK>(
      sm, (k1 - k0 + kSimtKC - 1) / kSimtKC, p.vec_a, p.vec_b, p.A, [](int) {},
      [&](int c, int i, int k) -> const float* {
        const int tok = k0 + c * kSimtKC + k;
        return tok < k1 ? p.A + (int64_t)tok * p.M + m0 + i : nullptr;
      },
      [&](int c, int i, int k) -> const float* {
        const int tok = k0 + c * kSimtKC + k;
        return tok < k1 ? p.B + (int64_t)tok * p.N + n0 + i : nullptr;
      });
  t.each4(sm, [&](int i, int j, float4 v) {
    float* o = p.C + ((int64_t)blockIdx.z * p.M + m0 + i) * p.N + n0 + j;
    if (p.add) v = make_float4(v.x + o[0], v.y + o[1], v.z + o[2], v.w + o[3]);
    st4(o, v, p.vec_c);
  });
}

template <typename Tile, Major BM, int S> int rows_as(unipool_ctx* ctx, int phase, const SimtLinear& p, cudaStream_t s) {
  PhaseTimer pt(ctx, phase, 1, s);
  auto kern = linear_rows_kernel<Tile, BM, S>;
  constexpr int smem = (int)sizeof(typename Tile::Smem);
  UP_CUDA(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
  UP_KERNEL(kern, dim3((p.M + Tile::kRows - 1) / Tile::kRows, (p.N + tile_cols<Tile> - 1) / tile_cols<Tile>, S), Tile::kThreads, smem, s, p);
  return UNIPOOL_OK;
}
template <Major BM> int rows_simt(unipool_ctx* ctx, int phase, const SimtLinear& p, cudaStream_t s) {
  const int64_t tiles = (int64_t)((p.M + kSimtM - 1) / kSimtM) * (p.N / kSimtN);
  // Tiles of four warps, three to an SM: as many to a tile as run at a time (a cluster of eight inside one GPC of 16 SMs), while each
  // warp has two chunks.
  const int chunks = p.K / kSimtKC;
  auto fits = [&](int n) { return tiles * n <= (n == 8 ? 5 : 6) * ctx->sm_count / 2 && chunks >= 8 * n; };
  if (2 * tiles <= ctx->sm_count) {
    if (fits(8)) return rows_as<SimtTile<4>, BM, 8>(ctx, phase, p, s);
    if (fits(4)) return rows_as<SimtTile<4>, BM, 4>(ctx, phase, p, s);
    if (fits(2)) return rows_as<SimtTile<4>, BM, 2>(ctx, phase, p, s);
  }
  if (tiles <= ctx->sm_count) return rows_as<SimtTile<8>, BM, 1>(ctx, phase, p, s);
  // Halves of tiles, where they leave half a tile less to the fullest SM than whole ones: 640 tokens 1024 -> 704 (220 tiles on 148 SMs) 27 us
  // instead of 35, 1024 -> 1152 (360) 45 instead of 50, 2880 -> 1536 (480) 157 instead of 175.
  const int64_t whole = (tiles + ctx->sm_count - 1) / ctx->sm_count, halves = (2 * tiles + ctx->sm_count - 1) / ctx->sm_count;
  if (whole <= 5 && halves < 2 * whole && chunks >= 32) return rows_as<SimtTile<4>, BM, 2>(ctx, phase, p, s);
  // Tiles of 128 x 128 where they give three of four SMs two blocks and little of them lies outside.  us, forward and dx, with / without:
  // 4000 tokens 1024 -> 1024 213/244, 201/224; 16384 768 -> 1024 536/585, 566/571; 3000 4096 -> 1536 798/878, 842/842; 8000 1024 -> 1024
  // 415/400, 391/377 (1.7 rounds of blocks)
  const int64_t wide = (int64_t)((p.M + 127) / 128) * ((p.N + 127) / 128);
  if (2 * wide >= 3 * ctx->sm_count && 20 * (int64_t)p.M * p.N >= 17 * wide * 128 * 128)
    return rows_as<SimtWideTile, BM, 1>(ctx, phase, p, s);
  if (tiles <= 6 * ctx->sm_count) return rows_as<SimtTile<4>, BM, 1>(ctx, phase, p, s);
  return rows_as<SimtBlockTile<1>, BM, 1>(ctx, phase, p, s);
}

// Tokens of a part of the weight gradient: the number of parts with the least time, by the blocks on the fullest SM (a block of 64 x 64
// takes 24 ns a token beside two others, 27 beside one and 33 alone), their starts, and writing and reading the parts' sums (8 bytes a
// ns).  us with one part / two blocks to an SM / this: 2183 tokens 1728 x 256 78/60/49, 2000 2048 x 1024 203/203/175, 16384 768 x 1024
// 882/622/525, 512 256 x 512 20/13/9.  (Tiles of 128 x 128 were no faster.)
int dw_length_simt(const unipool_ctx* ctx, int T, int n_in, int n_out) {
  const int64_t tiles = (int64_t)(n_out / 64) * (n_in / 64);
  int best = 0;
  double least = 0.0;
  for (int n = 1; n <= 64 && n <= (T + 63) / 64; ++n) {
    const int len = ((T + n - 1) / n + kSimtKC - 1) / kSimtKC * kSimtKC;
    if ((T + len - 1) / len != n) continue;
    const double k = (double)((tiles * n + ctx->sm_count - 1) / ctx->sm_count);
    double us = k * (len * (k > 2.0 ? 0.025 : k > 1.0 ? 0.027 : 0.033) + 0.35);
    if (n > 1) us += 2.0 + (double)n * n_in * n_out / 1.0e6;
    if (best == 0 || us < least) { best = len; least = us; }
  }
  return best;
}
int dw_splits_simt(const unipool_ctx* ctx, int T, int n_in, int n_out) {
  const int len = dw_length_simt(ctx, T, n_in, n_out);
  return (T + len - 1) / len;
}
int dw_simt(unipool_ctx* ctx, const LinearBwdArgs& a, const void* dp, float* out, int splits, bool add, cudaStream_t s) {
  SimtLinear p{};
  p.A = static_cast<const float*>(dp); p.B = static_cast<const float*>(a.x); p.C = out;
  p.M = a.n_out; p.N = a.n_in; p.K = a.T; p.add = add;
  p.k_len = dw_length_simt(ctx, a.T, a.n_in, a.n_out);
  p.vec_a = aligned16(p.A); p.vec_b = aligned16(p.B); p.vec_c = aligned16(p.C);
  PhaseTimer pt(ctx, UNIPOOL_PH_LINEAR_BWD, 1, s);
  UP_CUDA(cudaFuncSetAttribute(linear_dw_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(LinearDwTile::Smem)));
  UP_KERNEL(linear_dw_kernel, dim3(a.n_out / LinearDwTile::kRows, a.n_in / kSimtN, splits), LinearDwTile::kThreads,
            sizeof(LinearDwTile::Smem), s, p);
  return UNIPOOL_OK;
}

constexpr int kDyRows = 512;             // so few rows of dy are summed without a kernel of their own

bool tensor_cores(const unipool_ctx* ctx) { return ctx->cfg.dtype == UNIPOOL_BF16; }
LinearDwPlan dw_plan(const unipool_ctx* ctx, int T, int n_in, int n_out, bool with_dx) {
  return tensor_cores(ctx) ? linear_dw_plan_tc(ctx, T, n_in, n_out, with_dx) : LinearDwPlan{dw_splits_simt(ctx, T, n_in, n_out), 0};
}

template <typename E, int V, bool kFast>
int dp_as(unipool_ctx* ctx, const LinearBwdArgs& a, int* blocks, float* parts, cudaStream_t s) {
  const bool cluster = a.dbias != nullptr && a.T > kDpOneBlock && a.T <= kDpClusterRows;
  const int n = cluster ? kDpCluster : dp_row_blocks(ctx, a.T, a.n_out, 32 * V, a.act);
  DpParams p{a.dy, a.pre, a.act != UNIPOOL_ACT_NONE ? a.dp : nullptr, nullptr, a.T, a.n_out,
             cluster ? ((a.T + n - 1) / n + kDpRows - 1) / kDpRows * kDpRows : dp_rows(a.T, n), a.act, false};
  if (a.dbias != nullptr) {
    *blocks = cluster ? 1 : n;
    p.parts = *blocks > 1 ? parts : a.dbias;
    p.add = *blocks == 1 && !a.overwrite;
  }
  PhaseTimer pt(ctx, UNIPOOL_PH_LINEAR_BWD, 1, s);
  const dim3 grid((a.n_out + 32 * V - 1) / (32 * V), n);
  if (cluster) UP_KERNEL((linear_dp_kernel<E, V, kFast, kDpCluster>), grid, 256, 0, s, p);
  else UP_KERNEL((linear_dp_kernel<E, V, kFast, 1>), grid, 256, 0, s, p);
  return UNIPOOL_OK;
}

}  // namespace

int column_sum_launch(const float* parts, int n_parts, int64_t width, float* out, bool add, cudaStream_t s) {
  return part_sum(PartSum<float>{}, PartSum<float>{parts, n_parts, width, out, add}, s);
}

int linear_launch(unipool_ctx* ctx, const LinearArgs& a, cudaStream_t s) {
  if (a.T == 0) return UNIPOOL_OK;
  if (tensor_cores(ctx)) return linear_fwd_tc(ctx, a, s);
  SimtLinear p{};
  p.A = static_cast<const float*>(a.x); p.B = static_cast<const float*>(a.W); p.C = static_cast<float*>(a.y);
  p.P = static_cast<float*>(a.pre); p.bias = a.bias; p.residual = static_cast<const float*>(a.residual);
  p.M = a.T; p.N = a.n_out; p.K = a.n_in; p.act = a.act;
  p.vec_a = aligned16(p.A); p.vec_b = aligned16(p.B); p.vec_c = aligned16(p.C, p.P, p.bias, p.residual);
  return rows_simt<kAlongK>(ctx, UNIPOOL_PH_LINEAR, p, s);
}

// Scratch: the parts of dbias, then those of dW.
static size_t dw_parts(int splits, int n_in, int n_out) { return splits > 1 ? (size_t)splits * n_in * n_out : 0; }
static size_t db_parts(const unipool_ctx* ctx, int T, int n_out) {
  if (T <= kDpClusterRows) return 0;
  int sums = 0;                                          // (the widest call: any activation, and in fp32 any alignment)
  for (const int act : {UNIPOOL_ACT_NONE, UNIPOOL_ACT_GELU})
    for (const int cols : {32 * (tensor_cores(ctx) ? 8 : 4), 32}) sums = std::max(sums, dp_row_blocks(ctx, T, n_out, cols, act));
  return sums > 1 ? (size_t)sums * n_out : 0;
}
size_t linear_bwd_scratch(const unipool_ctx* ctx, int T, int n_in, int n_out) {
  const int splits = std::max(dw_plan(ctx, T, n_in, n_out, false).splits, dw_plan(ctx, T, n_in, n_out, true).splits);
  return (db_parts(ctx, T, n_out) + dw_parts(splits, n_in, n_out)) * sizeof(float);
}

int linear_bwd_launch(unipool_ctx* ctx, const LinearBwdArgs& args, cudaStream_t s) {
  LinearBwdArgs a = args;
  if (a.T == 0) {
    if (a.overwrite && a.dW != nullptr) UP_CUDA(cudaMemsetAsync(a.dW, 0, (size_t)a.n_in * a.n_out * sizeof(float), s));
    if (a.overwrite && a.dbias != nullptr) UP_CUDA(cudaMemsetAsync(a.dbias, 0, (size_t)a.n_out * sizeof(float), s));
    return UNIPOOL_OK;
  }
  const bool tc = tensor_cores(ctx), act = a.act != UNIPOOL_ACT_NONE;
  const void* dp = act ? a.dp : a.dy;
  int rc = UNIPOOL_OK;
  PartSum<float> dW{}, db{};                             // what is left to add up
  // (few rows of dy itself are added up beside dW's parts: one launch less)
  const bool dy_rows = !act && a.dbias != nullptr && a.T <= kDyRows;
  if (act && a.dx != nullptr && a.dx_residual == a.dp) {   // (x + act(x W^T): both dy) dp overwrites what dx still adds
    UP_CUDA(cudaMemcpyAsync(a.dx, a.dx_residual, (size_t)a.T * a.n_in * ctx->elem_bytes, cudaMemcpyDeviceToDevice, s));
    a.dx_residual = a.dx;
  }
  if (act || (a.dbias != nullptr && !dy_rows)) {
    int blocks = 1;
    rc = tc ? dp_as<__nv_bfloat16, 8, true>(ctx, a, &blocks, a.scratch, s)
         : aligned16(a.dy, a.pre, act ? a.dp : nullptr) ? dp_as<float, 4, false>(ctx, a, &blocks, a.scratch, s)
                                                        : dp_as<float, 1, false>(ctx, a, &blocks, a.scratch, s);
    if (rc != UNIPOOL_OK) return rc;
    if (a.dbias != nullptr && blocks > 1) db = {a.scratch, blocks, a.n_out, a.dbias, !a.overwrite};
  }
  const LinearDwPlan plan = a.dW != nullptr ? dw_plan(ctx, a.T, a.n_in, a.n_out, a.dx != nullptr) : LinearDwPlan{1, 0};
  if (a.dx != nullptr && plan.dx_tile == 0) {
    if (tc) {
      rc = linear_dx_tc(ctx, a, dp, s);
    } else {
      SimtLinear p{};
      p.A = static_cast<const float*>(dp); p.B = static_cast<const float*>(a.W); p.C = static_cast<float*>(a.dx);
      p.residual = static_cast<const float*>(a.dx_residual);
      p.M = a.T; p.N = a.n_in; p.K = a.n_out; p.act = UNIPOOL_ACT_NONE;
      p.vec_a = aligned16(p.A); p.vec_b = aligned16(p.B); p.vec_c = aligned16(p.C, p.residual);
      rc = rows_simt<kAcrossK>(ctx, UNIPOOL_PH_LINEAR_BWD, p, s);
    }
    if (rc != UNIPOOL_OK) return rc;
  }
  if (a.dW != nullptr) {
    const int splits = plan.splits;
    float* out = splits > 1 ? a.scratch + db_parts(ctx, a.T, a.n_out) : a.dW;
    const bool add = splits == 1 && !a.overwrite;
    rc = tc ? linear_dw_tc(ctx, a, dp, out, plan, add, s) : dw_simt(ctx, a, dp, out, splits, add, s);
    if (rc != UNIPOOL_OK) return rc;
    if (splits > 1) dW = {out, splits, (int64_t)a.n_in * a.n_out, a.dW, !a.overwrite};
  }
  if (dW.n == 0 && db.n == 0 && !dy_rows) return UNIPOOL_OK;
  PhaseTimer pt(ctx, UNIPOOL_PH_LINEAR_BWD, 1, s);
  if (!dy_rows) return part_sum(dW, db, s);
  if (tc) return part_sum(dW, PartSum<__nv_bfloat16>{static_cast<const __nv_bfloat16*>(a.dy), a.T, a.n_out, a.dbias, !a.overwrite}, s);
  return part_sum(dW, PartSum<float>{static_cast<const float*>(a.dy), a.T, a.n_out, a.dbias, !a.overwrite}, s);
}

}  // namespace unipool
