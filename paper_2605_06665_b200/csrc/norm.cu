// RMS norm of a residual stream, with the addition in front of it and 8-bit output behind it, and its backward pass.
//
//   r = x + y,  n_t = 1 / sqrt(mean_j r_tj^2 + eps),  h = r n_t w;   q = e4m3(h / s_t),  s_t = max_j |h_tj| / 448
//   backward of h (gradient dh) and of r itself (dr):  with xhat = r n_t,
//     dx = n_t (w dh - xhat mean_j(w dh xhat)) + dr,   dw_j += sum_t dh_tj xhat_tj
// (xhat is of size one whatever the row's scale: no power of n_t over- or underflows)
//
// Bound by HBM: forward 2 (x, h) to 4 (y, r too) passes over the stream, backward 3 to 4, next to no arithmetic.  A row stays
// in the registers of the threads that share it, so that it is read once: a warp up to 256 vectors of 16 bytes (2048 bf16
// columns), four, eight or sixteen beyond; all of a thread's loads are issued before the first is used.  Rows whose bytes are no
// multiple of 16, and misaligned tensors, go two elements or one at a time through the same kernels (one, four, five, eight, ten or sixteen
// warps to a row).  16384 x 768 bf16 with residual 17 us
// (5.9 TB/s), 32768 x 1536 with 8 bits too 71 us (6.4 TB/s); backward of 16384 x 768 with dr 22 us, 4 of them for adding up dw.
// Sums of squares, the statistics and the gradient of w are fp32; h is formed from the unrounded sum r.
#include <cooperative_groups.h>
#include <cuda_fp8.h>

#include <type_traits>

#include "common.cuh"
#include "tc_ptx.cuh"
#include "vec.cuh"

namespace unipool {

namespace {

constexpr float kE4m3Max = 448.f;
constexpr float kSmallestScale = 1.17549435e-38f;        // 2^-126: its reciprocal is finite, a row of zeros keeps zeros

template <int V> __device__ __forceinline__ void load_w(const float* w, float (&v)[V]) {
  if constexpr (V == 1) {
    v[0] = __ldg(w);
  } else if constexpr (V == 2) {
    const float2 f = __ldg(reinterpret_cast<const float2*>(w));
    v[0] = f.x; v[1] = f.y;
  } else {
#pragma unroll
    for (int i = 0; i < V; i += 4) {
      const float4 f = __ldg(reinterpret_cast<const float4*>(w + i));
      v[i] = f.x; v[i + 1] = f.y; v[i + 2] = f.z; v[i + 3] = f.w;
    }
  }
}

template <int V> __device__ __forceinline__ void store_e4m3(uint8_t* q, const float (&v)[V]) {
  if constexpr (V == 1) {
    *q = __nv_cvt_float_to_fp8(v[0], __NV_SATFINITE, __NV_E4M3);
  } else if constexpr (V == 2) {
    *reinterpret_cast<uint16_t*>(q) = __nv_cvt_float2_to_fp8x2(make_float2(v[0], v[1]), __NV_SATFINITE, __NV_E4M3);
  } else {
    uint32_t w[V / 4];
#pragma unroll
    for (int i = 0; i < V / 4; ++i) {
      const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(v[4 * i], v[4 * i + 1]), __NV_SATFINITE, __NV_E4M3);
      const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(v[4 * i + 2], v[4 * i + 3]), __NV_SATFINITE, __NV_E4M3);
      w[i] = lo | hi << 16;
    }
    if constexpr (V == 8) *reinterpret_cast<uint2*>(q) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<uint32_t*>(q) = w[0];
  }
}

// The row's value of op over the TPR threads that share it, the same in all of them: a warp, or the block (`part`: one value per warp,
// not read by anyone any more).
template <int TPR, typename F> __device__ __forceinline__ float row_reduce(float v, float* part, F op) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, o));
  if constexpr (TPR > 32) {
    if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int i = 1; i < TPR / 32; ++i) v = op(v, part[i]);
  }
  return v;
}

struct NormParams {
  const void *x, *y;
  const float* w;
  void *r, *h;
  float* rstd;
  uint8_t* q;
  float* q_scale;
  int T, width;
  float eps;
};

template <int TPR> constexpr int kNormThreads = TPR == 32 ? 128 : TPR;

// TPR threads share a row, VPT vectors of V elements each.  kNorm = false: rows to 8 bits as they are.
template <typename E, int V, int TPR, int VPT, bool kNorm>
__global__ void __launch_bounds__(kNormThreads<TPR>) rmsnorm_kernel(NormParams p) {
  grid_wait(p.x, p.y, p.w);
  __shared__ float part[2][TPR > 32 ? TPR / 32 : 1];
  const int row = blockIdx.x * (kNormThreads<TPR> / TPR) + threadIdx.x / TPR, t = threadIdx.x % TPR;
  if (TPR == 32 && row >= p.T) return;
  const int64_t at = (int64_t)row * p.width;
  const E* x = static_cast<const E*>(p.x) + at;
  const E* y = static_cast<const E*>(p.y) + at;
  Vec<E, V> a[VPT], b[VPT];
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int c = (i * TPR + t) * V;
    a[i].zero();
    if (c < p.width) a[i].load(x + c);
  }
  if (kNorm && p.y != nullptr) {
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int c = (i * TPR + t) * V;
      b[i].zero();
      if (c < p.width) b[i].load(y + c);
    }
  }
  float v[VPT][V];
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    a[i].get(v[i]);
    if (kNorm && p.y != nullptr) {
      float u[V];
      b[i].get(u);
#pragma unroll
      for (int j = 0; j < V; ++j) v[i][j] += u[j];
    }
#pragma unroll
    for (int j = 0; j < V; ++j) ss = fmaf(v[i][j], v[i][j], ss);
  }
  float amax = 0.f;
  if constexpr (kNorm) {
    ss = row_reduce<TPR>(ss, part[0], [](float m, float n) { return m + n; });
    const float n = 1.f / sqrtf(ss / (float)p.width + p.eps);
    if (t == 0 && p.rstd != nullptr) p.rstd[row] = n;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int c = (i * TPR + t) * V;
      if (c >= p.width) continue;
      if (p.r != nullptr) Vec<E, V>::store(static_cast<E*>(p.r) + at + c, v[i]);
      float w[V];
      load_w<V>(p.w + c, w);
#pragma unroll
      for (int j = 0; j < V; ++j) v[i][j] = v[i][j] * n * w[j];      // (n w may leave fp32's range where h does not)
      if (p.h != nullptr) Vec<E, V>::store(static_cast<E*>(p.h) + at + c, v[i]);
    }
  }
  if (p.q == nullptr) return;
#pragma unroll
  for (int i = 0; i < VPT; ++i)
#pragma unroll
    for (int j = 0; j < V; ++j) amax = max_nan(amax, fabsf(v[i][j]));
  amax = row_reduce<TPR>(amax, part[1], [](float m, float n) { return max_nan(m, n); });
  const float scale = max_nan(amax / kE4m3Max, kSmallestScale);
  const float inv = 1.f / scale;
  if (t == 0) p.q_scale[row] = scale;
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int c = (i * TPR + t) * V;
    if (c >= p.width) continue;
#pragma unroll
    for (int j = 0; j < V; ++j) v[i][j] *= inv;
    store_e4m3<V>(p.q + at + c, v[i]);
  }
}

// ---------------------------------------------------------------- backward
struct NormBwdParams {
  const void *dh, *r, *dr;
  const float *w, *rstd;
  void* dx;
  float* dw;        // [blocks, width] sums of the blocks; one block: the gradient itself
  int T, width, stages;
  bool add;         // one block: add to what dw holds
  int32_t* status;
};

// Bytes of the ring for a run of so many: it may begin and end inside 16 bytes.
__host__ __device__ constexpr uint32_t norm_bwd_slot(uint32_t run) { return (run + 30) / 16 * 16; }

// The sums over the warp of each of R values: the lane's own value of row row_of_lane<R>(lane) on return.  A lane hands half of its
// values over at each step, until it has one.
template <int R> __device__ __forceinline__ float reduce_rows(float (&v)[R], int lane) {
  static_assert(R == 1 || R == 2 || R == 4 || R == 8, "rows");
  if constexpr (R == 8) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float give = lane & 16 ? v[k] : v[k + 4];
      v[k] = (lane & 16 ? v[k + 4] : v[k]) + __shfl_xor_sync(0xffffffffu, give, 16);
    }
  }
  if constexpr (R >= 4) {
    constexpr int o = R == 8 ? 8 : 16;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const float give = lane & o ? v[k] : v[k + 2];
      v[k] = (lane & o ? v[k + 2] : v[k]) + __shfl_xor_sync(0xffffffffu, give, o);
    }
  }
  if constexpr (R >= 2) {
    constexpr int o = 32 / R;
    const float give = lane & o ? v[0] : v[1];
    v[0] = (lane & o ? v[1] : v[0]) + __shfl_xor_sync(0xffffffffu, give, o);
  }
#pragma unroll
  for (int o = 16 / R; o > 0; o >>= 1) v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
  return v[0];
}
template <int R> __device__ __forceinline__ int row_of_lane(int lane) { return lane / (32 / R); }

// A block takes R rows at a time and a thread VPT vectors of the same columns of each: it keeps w and its sums for dw in
// registers over all its rows, and the rows' dot products cost one barrier for R of them.  (With a row to a warp the sums of a whole
// row lay in every warp's registers and had to be added up at the end: 16384 rows of 768 bf16 22.5 us instead of 18.7.)
// kRing: R rows are one run of bytes in memory; runs are copied, from the 16-byte boundary below to the one above, into a ring in
// shared memory some stages ahead, so that reads go on while rows are worked on and whatever the rows' alignment (16384 rows of
// 770 bf16 read element by element 69 us, through the ring 35).  Without it (arrays off 16 bytes, rows too long for two stages) the loads go
// from memory into registers.
// The sums' order depends on the sizes, the number of arrays and their alignment (norm_bwd_shape).  C > 1: the blocks are one cluster, which adds its sums for dw up through each other's shared
// memory, in the order of the ranks.
template <typename E, int V, int VPT, int R, bool kRing, int C>
__global__ void __cluster_dims__(C, 1, 1) __launch_bounds__(512, V * sizeof(E) == 16 ? 1 : 2) rmsnorm_bwd_kernel(NormBwdParams p) {
  extern __shared__ __align__(128) uint8_t ring[];       // [stages][dh, r, dr][R rows], then the barriers
  __shared__ float part[2][16][R];
  __shared__ int abort_word;
  constexpr bool kKeepW = VPT * V <= 16;                 // else w comes from the cache again
  const int t = threadIdx.x, n_warps = blockDim.x / 32;
  const uint32_t run = (uint32_t)(R * p.width * (int)sizeof(E)), slot = norm_bwd_slot(run);
  const int arrays = p.dr != nullptr ? 3 : 2;
  uint64_t* full = reinterpret_cast<uint64_t*>(ring + (size_t)p.stages * arrays * slot);
  volatile int* abort = &abort_word;
  if constexpr (kRing) {
    if (t == 0) {
      for (int s = 0; s < p.stages; ++s) tc::mbar_init(&full[s], 1);
      *abort = 0;
      tc::fence_barrier_init();
    }
    __syncthreads();
  }
  grid_wait(p.dh, p.r, p.dr, p.w, p.rstd);
  const int64_t groups = ((int64_t)p.T + R - 1) / R;
  // Rows of group g into its stage: by the copy engine, but for the last ones, where that would reach beyond the array's end.
  const int64_t total = (int64_t)p.T * p.width * (int)sizeof(E);
  auto end_of = [&](int64_t g) { return (min((g + 1) * (int64_t)run, total) + 15) / 16 * 16; };
  auto fetch = [&](int64_t g, int stage) {
    const int64_t from = g * run / 16 * 16;
    if (end_of(g) > total) return;
    const uint32_t n = (uint32_t)(end_of(g) - from);
    uint8_t* to = ring + (size_t)stage * arrays * slot;
    tc::mbar_expect_tx(&full[stage], arrays * n);
    tc::bulk_load(to, static_cast<const uint8_t*>(p.dh) + from, n, &full[stage]);
    tc::bulk_load(to + slot, static_cast<const uint8_t*>(p.r) + from, n, &full[stage]);
    if (arrays == 3) tc::bulk_load(to + 2 * slot, static_cast<const uint8_t*>(p.dr) + from, n, &full[stage]);
  };
  if (kRing && t == 0) {
    int64_t g = blockIdx.x;
    for (int s = 0; s < p.stages && g < groups; ++s, g += gridDim.x) fetch(g, s);
  }
  auto column = [&](int i) { return (i * (int)blockDim.x + t) * V; };
  float dw[VPT][V], w[kKeepW ? VPT : 1][V];
#pragma unroll
  for (int i = 0; i < VPT; ++i)
#pragma unroll
    for (int j = 0; j < V; ++j) dw[i][j] = 0.f;
  if constexpr (kKeepW) {
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
#pragma unroll
      for (int j = 0; j < V; ++j) w[i][j] = 0.f;
      if (column(i) < p.width) load_w<V>(p.w + column(i), w[i]);
    }
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j) w[0][j] = 0.f;
  }
  const float inv_width = 1.f / (float)p.width;
  int turn = 0, stage = 0;
  uint32_t phase = 0;
  float n_next[R];                                       // rstd of the next rows
  auto load_rstd = [&](int64_t g) {
#pragma unroll
    for (int k = 0; k < R; ++k) n_next[k] = g * R + k < p.T ? __ldg(p.rstd + (g * R + k)) : 0.f;
  };
  load_rstd(blockIdx.x);
  for (int64_t group = blockIdx.x; group < groups; group += gridDim.x, turn ^= 1) {
    const int64_t row0 = group * R;
    uint8_t* at_stage = ring + (size_t)stage * arrays * slot + group * run % 16;
    if constexpr (kRing) {
      if (end_of(group) <= total) {
        // (a wait that runs out is reported, and no later one waits; the block goes on to its end)
        if (!*abort && !tc::mbar_wait(&full[stage], phase, abort)) {
          *abort = 1;
          if (atomicCAS(p.status, 0, kStatusTimeout) == 0) { p.status[1] = 61; p.status[2] = (int)blockIdx.x; }
        }
      } else {
        const int64_t from = row0 * p.width;
        const int n = (int)min((int64_t)R, p.T - row0) * p.width;
        for (int c = t; c < n; c += blockDim.x) {
          reinterpret_cast<E*>(at_stage)[c] = static_cast<const E*>(p.dh)[from + c];
          reinterpret_cast<E*>(at_stage + slot)[c] = static_cast<const E*>(p.r)[from + c];
          if (arrays == 3) reinterpret_cast<E*>(at_stage + 2 * slot)[c] = static_cast<const E*>(p.dr)[from + c];
        }
        __syncthreads();
      }
    }
    // g = w dh and xhat stay in registers from one side of the barrier to the other
    Vec<E, V> d[R][VPT];
    float g[R][VPT][V], xhat[R][VPT][V], n[R], dot[R];
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const bool live = row0 + k < p.T;
      n[k] = n_next[k];
      dot[k] = 0.f;
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        const int c = column(i);
        Vec<E, V> a, b;
        a.zero();
        b.zero();
        d[k][i].zero();
        if (live && c < p.width) {
          const E *x, *y, *z;
          if constexpr (kRing) {
            x = reinterpret_cast<const E*>(at_stage) + (k * p.width + c);
            y = reinterpret_cast<const E*>(at_stage + slot) + (k * p.width + c);
            z = reinterpret_cast<const E*>(at_stage + 2 * slot) + (k * p.width + c);
          } else {
            const int64_t at = (row0 + k) * p.width + c;
            x = static_cast<const E*>(p.dh) + at;
            y = static_cast<const E*>(p.r) + at;
            z = static_cast<const E*>(p.dr) + at;
          }
          a.load(x);
          b.load(y);
          if (p.dr != nullptr) d[k][i].load(z);
        }
        a.get(g[k][i]);
        b.get(xhat[k][i]);
      }
    }
    load_rstd(group + gridDim.x);
#pragma unroll
    for (int k = 0; k < R; ++k)
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        float(&wi)[V] = w[kKeepW ? i : 0];
        if (!kKeepW && column(i) < p.width) load_w<V>(p.w + column(i), wi);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          xhat[k][i][j] *= n[k];
          dw[i][j] = fmaf(g[k][i][j], xhat[k][i][j], dw[i][j]);
          g[k][i][j] *= wi[j];
          dot[k] = fmaf(g[k][i][j], xhat[k][i][j], dot[k]);
        }
      }
    {
      const float sum = reduce_rows<R>(dot, t % 32);
      if (t % (32 / R) == 0) part[turn][t / 32][row_of_lane<R>(t % 32)] = sum;
    }
    __syncthreads();                                     // (two arrays in turn: the next rows' sums need no second barrier)
    if constexpr (kRing) {                               // the stage is in registers: on to the rows that lie `stages` further
      if (t == 0 && group + (int64_t)p.stages * gridDim.x < groups && !*abort) fetch(group + (int64_t)p.stages * gridDim.x, stage);
      if (++stage == p.stages) { stage = 0; phase ^= 1u; }
    }
    if (n_warps <= 4) {
#pragma unroll
      for (int k = 0; k < R; ++k) dot[k] = part[turn][0][k];
      for (int q = 1; q < n_warps; ++q)
#pragma unroll
        for (int k = 0; k < R; ++k) dot[k] += part[turn][q][k];
    } else {                                             // a warp's sum to a lane, half of the rows to either half of the lanes
      constexpr int H = R > 1 ? R / 2 : 1;
      const int q = t % 16, first = R > 1 ? (t / 16 % 2) * H : 0;
      float half[H];
#pragma unroll
      for (int k = 0; k < H; ++k) half[k] = q < n_warps ? part[turn][q][first + k] : 0.f;
#pragma unroll
      for (int o = 8; o > 0; o >>= 1)
#pragma unroll
        for (int k = 0; k < H; ++k) half[k] += __shfl_xor_sync(0xffffffffu, half[k], o);
#pragma unroll
      for (int k = 0; k < H; ++k) {
        const float other = __shfl_xor_sync(0xffffffffu, half[k], 16);
        dot[k] = first == 0 ? half[k] : other;
        if constexpr (R > 1) dot[H + k] = first == 0 ? other : half[k];
      }
    }
#pragma unroll
    for (int k = 0; k < R; ++k) {
      if (row0 + k >= p.T) break;
      const float mean = dot[k] * inv_width;
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        const int c = column(i);
        if (c >= p.width) continue;
        float u[V];
        d[k][i].get(u);                                  // (zeros without dr)
#pragma unroll
        for (int j = 0; j < V; ++j) u[j] = fmaf(n[k], fmaf(-xhat[k][i][j], mean, g[k][i][j]), u[j]);
        Vec<E, V>::store(static_cast<E*>(p.dx) + (row0 + k) * p.width + c, u);
      }
    }
  }
  if (kRing && *abort)
    for (int i = 0; i < 200; ++i) __nanosleep(1000);     // let copies already in flight land before the block retires
  if (p.dw == nullptr) return;
  float* out = C > 1 ? reinterpret_cast<float*>(ring) : &p.dw[(int64_t)blockIdx.x * p.width];
  const bool add = C == 1 && p.add;
  if (C > 1) __syncthreads();                            // (the rows in the ring are worked on)
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int c = column(i);
    if (c >= p.width) continue;
#pragma unroll
    for (int j = 0; j < V; ++j) out[c + j] = add ? out[c + j] + dw[i][j] : dw[i][j];
  }
  if constexpr (C > 1) {
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    cluster.sync();
    const int each = (p.width + C - 1) / C, c0 = (int)blockIdx.x * each, c1 = min(p.width, c0 + each);
    for (int c = c0 + t; c < c1; c += blockDim.x) {
      float v = cluster.map_shared_rank(out, 0)[c];
#pragma unroll
      for (int q = 1; q < C; ++q) v += cluster.map_shared_rank(out, q)[c];
      float* o = &p.dw[c];
      *o = p.add ? *o + v : v;
    }
    cluster.sync();                                      // no block leaves while another reads its sums
  }
}

// How the backward kernel runs: elements of a vector, vectors of a thread, threads and rows of a block, blocks, stages of the ring
// (0: none) and its bytes; whether with dw a cluster takes the rows instead.
constexpr int kNormBwdCluster = 8;
struct NormBwdShape { int v, vpt, threads, rows, blocks, stages; uint32_t smem; bool cluster; };
constexpr int norm_bwd_rows(int V, int bytes, int vpt) {   // 48 registers of elements, 24 of narrower vectors
  return V * bytes == 16 ? (vpt >= 4 ? 1 : 4 / vpt) : vpt >= 8 ? 1 : 8 / (vpt * (V * bytes == 8 ? 2 : 1));
}
NormBwdShape norm_bwd_shape_of(const unipool_ctx* ctx, int T, int width, int v, bool aligned, int arrays) {
  const int e = (int)ctx->elem_bytes, n = (width + v - 1) / v;
  NormBwdShape s;
  s.v = v;
  // (many rows of narrow vectors: smaller blocks, more of which overlap on an SM, though there are more sums to add up behind them.  16384 x 770
  // bf16 34 -> 29 us, x 1001 57 -> 52)
  const int wide = v <= 2 && T > 32 * ctx->sm_count ? 256 : 512;
  s.vpt = n <= wide ? 1 : n <= 2 * wide ? 2 : n <= 2048 ? 4 : n <= 4096 ? 8 : 32;
  s.threads = ((n + s.vpt - 1) / s.vpt + 31) / 32 * 32;
  s.rows = norm_bwd_rows(v, e, s.vpt);
  const int64_t stage = (int64_t)norm_bwd_slot((uint32_t)(s.rows * width * e)) * arrays;
  const int threads = v * e == 16 ? 640 : 1024;          // on an SM, by their registers
  int per_sm = 2 * s.threads <= threads ? threads / s.threads : 1;
  per_sm = per_sm > 16 ? 16 : per_sm;
  s.stages = 0;
  if (aligned && s.vpt <= 8) {
    auto fit = [&](int blocks) { return (int)((220 * 1024 / blocks - 2304) / stage); };     // (2304: barriers, sums, the system's)
    while (per_sm > 1 && fit(per_sm) < 2) --per_sm;
    s.stages = fit(per_sm) > 4 ? 4 : fit(per_sm) < 2 ? 0 : fit(per_sm);
  }
  s.smem = s.stages > 0 ? (uint32_t)(s.stages * stage + 64) : 0;
  // (few rows on one block: no sums to add up behind it, which costs as much as three steps of a block)
  const int64_t all = ((int64_t)T + s.rows - 1) / s.rows;
  const int most = ctx->sm_count * per_sm;
  s.blocks = all <= 4 ? 1 : all < most ? (int)all : most;
  // (some more on a cluster of eight: a step or two of its blocks, but no launch behind them and no scratch, 4.5 us of the host's time.  48 rows
  // of 768 bf16 5.0 us on a cluster and 4.5 in two launches, 96 rows 6.2 and 4.5)
  s.cluster = all > 4 && all <= (s.rows > 1 ? 2 : 1) * kNormBwdCluster && s.vpt <= 8;
  return s;
}
NormBwdShape norm_bwd_shape(const unipool_ctx* ctx, int T, int width, bool aligned, int arrays) {
  const int e = (int)ctx->elem_bytes;
  if (aligned && width * e % 16 == 0) return norm_bwd_shape_of(ctx, T, width, 16 / e, true, arrays);
  if (aligned && width % 2 == 0) {
    const NormBwdShape s = norm_bwd_shape_of(ctx, T, width, 2, true, arrays);
    if (s.stages > 0) return s;
  }
  return norm_bwd_shape_of(ctx, T, width, 1, aligned, arrays);
}

template <int N> using Int = std::integral_constant<int, N>;

template <bool kNorm, typename E> int norm_as(unipool_ctx* ctx, const NormParams& p, cudaStream_t s) {
  constexpr int V = 16 / (int)sizeof(E);
  const uintptr_t rows = reinterpret_cast<uintptr_t>(p.x) | reinterpret_cast<uintptr_t>(p.y) | reinterpret_cast<uintptr_t>(p.r) |
                         reinterpret_cast<uintptr_t>(p.h) | reinterpret_cast<uintptr_t>(p.w);
  auto run = [&](auto v, auto tpr, auto vpt) {
    constexpr int kTpr = decltype(tpr)::value, kRows = kNormThreads<kTpr> / kTpr;
    PhaseTimer pt(ctx, UNIPOOL_PH_RMSNORM, 1, s);
    UP_KERNEL((rmsnorm_kernel<E, decltype(v)::value, kTpr, decltype(vpt)::value, kNorm>), (unsigned)(((int64_t)p.T + kRows - 1) / kRows),
              kNormThreads<kTpr>, 0, s, p);
    return UNIPOOL_OK;
  };
  // vectors of v elements whose number and rows' alignment allow them
  auto fits = [&](int v) { return p.width % v == 0 && rows % (v * sizeof(E)) == 0 && rows % (v * 4 < 16 ? v * 4 : 16) == 0 &&
                                  reinterpret_cast<uintptr_t>(p.q) % v == 0; };
  if (fits(V)) {
    const int n = p.width / V;
    if (n <= 32) return run(Int<V>(), Int<32>(), Int<1>());
    if (n <= 64) return run(Int<V>(), Int<32>(), Int<2>());
    if (n <= 96) return run(Int<V>(), Int<32>(), Int<3>());
    if (n <= 128) return run(Int<V>(), Int<32>(), Int<4>());
    if (n <= 192) return run(Int<V>(), Int<32>(), Int<6>());
    if (n <= 256) return run(Int<V>(), Int<32>(), Int<8>());
    if (n <= 512) return run(Int<V>(), Int<128>(), Int<4>());
    if (n <= 1024) return run(Int<V>(), Int<256>(), Int<4>());
    if constexpr (V == 4) {                              // (no row has more than 2048 vectors of eight)
      if (n > 2048) return run(Int<V>(), Int<512>(), Int<8>());
    }
    return run(Int<V>(), Int<512>(), Int<4>());
  }
  auto narrow = [&](auto v) {
    const int n = p.width / decltype(v)::value;
    // Sixteen vectors to a thread leave fewer rows in work at a time, with more bytes under way for each: better for many rows (us, eight and
    // sixteen vectors: 16384 x 301 bf16 16.2 and 10.4, 24702 x 2187 100 and 86, 4096 x 3001 24 and 22), worse for few (1 x 1001 2.9
    // and 4.3) and for rows of 513 to 2048 (16384 x 1001 fp32 42 and 50).
    const bool many = p.T > 8 * ctx->sm_count;
    if (n <= 256) return run(v, Int<32>(), Int<8>());
    if (n <= 512 && many) return run(v, Int<32>(), Int<16>());
    if (n <= 1024) return run(v, Int<128>(), Int<8>());
    if (n <= 2048) return run(v, Int<256>(), Int<8>());
    if (n <= 2560) return many ? run(v, Int<160>(), Int<16>()) : run(v, Int<320>(), Int<8>());
    if (n <= 4096) return many ? run(v, Int<256>(), Int<16>()) : run(v, Int<512>(), Int<8>());
    return run(v, Int<512>(), Int<32>());
  };
  return fits(2) ? narrow(Int<2>()) : narrow(Int<1>());
}

template <typename E, int V, int VPT, bool kRing>
int norm_bwd_run(const NormBwdShape& f, const NormBwdParams& p, cudaStream_t s) {
  auto run = [&](auto c) {
    constexpr int C = decltype(c)::value;
    auto kern = rmsnorm_bwd_kernel<E, V, VPT, norm_bwd_rows(V, (int)sizeof(E), VPT), kRing, C>;
    const uint32_t sums = C > 1 ? p.width * 4u : 0u;     // they lie where the ring was
    if (kRing || C > 1) UP_CUDA(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 223 * 1024));
    UP_KERNEL(kern, C > 1 ? C : f.blocks, f.threads, f.smem > sums ? f.smem : sums, s, p);
    return (int)UNIPOOL_OK;
  };
  if constexpr (VPT <= 8) {                              // (norm_bwd_shape takes no cluster for more)
    if (f.cluster) return run(std::integral_constant<int, kNormBwdCluster>());
  }
  return run(std::integral_constant<int, 1>());
}

template <typename E> int norm_bwd_as(unipool_ctx* ctx, NormBwdParams p, bool aligned, float* scratch, bool overwrite, cudaStream_t s) {
  constexpr int V = 16 / (int)sizeof(E);
  NormBwdShape f = norm_bwd_shape(ctx, p.T, p.width, aligned, p.dr != nullptr ? 3 : 2);
  float* dw = p.dw;
  f.cluster = f.cluster && dw != nullptr;
  const bool split = dw != nullptr && f.blocks > 1 && !f.cluster;
  p.add = !overwrite && !split;
  p.stages = f.stages;
  if (split) p.dw = scratch;
  PhaseTimer pt(ctx, UNIPOOL_PH_RMSNORM_BWD, split ? 2 : 1, s);
  auto by_vpt = [&](auto v, auto ring) {
    constexpr int kV = decltype(v)::value;
    constexpr bool kRing = decltype(ring)::value;
    if (f.vpt == 1) return norm_bwd_run<E, kV, 1, kRing>(f, p, s);
    if (f.vpt == 2) return norm_bwd_run<E, kV, 2, kRing>(f, p, s);
    if (f.vpt == 4) return norm_bwd_run<E, kV, 4, kRing>(f, p, s);
    if constexpr (kV <= 4) {                             // (no row has so many vectors of eight)
      if (f.vpt == 8) return norm_bwd_run<E, kV, 8, kRing>(f, p, s);
    }
    if constexpr (kV == 1 && !kRing) return norm_bwd_run<E, 1, 32, false>(f, p, s);
    return (int)UNIPOOL_ERR_UNSUPPORTED;
  };
  int rc;
  if (f.stages > 0) rc = f.v == V ? by_vpt(Int<V>(), std::true_type()) : f.v == 1 ? by_vpt(Int<1>(), std::true_type()) : by_vpt(Int<2>(), std::true_type());
  else if (f.v == 1) rc = by_vpt(Int<1>(), std::false_type());
  else if constexpr (V == 4) rc = norm_bwd_run<E, 4, 8, false>(f, p, s);   // fp32 rows of 9288 and more with dr, 13936 without: two do not fit
  else rc = UNIPOOL_ERR_UNSUPPORTED;                     // (every bf16 row's do)
  return rc == UNIPOOL_OK && split ? column_sum_launch(scratch, f.blocks, p.width, dw, !overwrite, s) : rc;
}

}  // namespace

// (The most that any alignment and number of arrays takes.)
size_t rmsnorm_bwd_scratch(const unipool_ctx* ctx, int T, int width) {
  int most = 0;
  for (int k = 0; k < 4; ++k) {
    const NormBwdShape f = norm_bwd_shape(ctx, T, width, (k & 1) != 0, k < 2 ? 2 : 3);
    if (!f.cluster && f.blocks > most) most = f.blocks;
  }
  return most > 1 ? (size_t)most * width * sizeof(float) : 0;
}

int rmsnorm_launch(unipool_ctx* ctx, const void* x, const void* y, int T, int width, const float* w, float eps, void* r,
                   float* rstd, void* h, uint8_t* q, float* q_scale, cudaStream_t s) {
  if (T == 0) return UNIPOOL_OK;
  const NormParams p{x, y, w, r, h, rstd, q, q_scale, T, width, eps};
  return ctx->cfg.dtype == UNIPOOL_BF16 ? norm_as<true, __nv_bfloat16>(ctx, p, s) : norm_as<true, float>(ctx, p, s);
}

int quantize_rows_launch(unipool_ctx* ctx, const void* x, int T, int width, uint8_t* q, float* q_scale, cudaStream_t s) {
  if (T == 0) return UNIPOOL_OK;
  const NormParams p{x, nullptr, nullptr, nullptr, nullptr, nullptr, q, q_scale, T, width, 0.f};
  return ctx->cfg.dtype == UNIPOOL_BF16 ? norm_as<false, __nv_bfloat16>(ctx, p, s) : norm_as<false, float>(ctx, p, s);
}

int rmsnorm_bwd_launch(unipool_ctx* ctx, const void* dh, const void* r, int T, int width, const float* w, const float* rstd,
                       const void* dr, void* dx, float* dw, float* scratch, bool overwrite, cudaStream_t s) {
  if (T == 0) {
    if (dw != nullptr && overwrite) UP_CUDA(cudaMemsetAsync(dw, 0, (size_t)width * sizeof(float), s));
    return UNIPOOL_OK;
  }
  const NormBwdParams p{dh, r, dr, w, rstd, dx, dw, T, width, 0, false, ctx->ws.status};
  const uintptr_t all = reinterpret_cast<uintptr_t>(dh) | reinterpret_cast<uintptr_t>(r) | reinterpret_cast<uintptr_t>(dr) |
                        reinterpret_cast<uintptr_t>(dx) | reinterpret_cast<uintptr_t>(w);
  return ctx->cfg.dtype == UNIPOOL_BF16 ? norm_bwd_as<__nv_bfloat16>(ctx, p, all % 16 == 0, scratch, overwrite, s)
                                        : norm_bwd_as<float>(ctx, p, all % 16 == 0, scratch, overwrite, s);
}

}  // namespace unipool
