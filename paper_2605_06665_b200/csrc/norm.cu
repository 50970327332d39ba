// RMS norm of a residual stream, with the addition in front of it and 8-bit output behind it, and its backward pass.
//
//   r = x + y,  n_t = 1 / sqrt(mean_j r_tj^2 + eps),  h = r n_t w;   q = e4m3(h / s_t),  s_t = max_j |h_tj| / 448
//   backward of h (gradient dh) and of r itself (dr):  with c_t = sum_j dh_tj w_j r_tj,
//     dx = n_t w dh - r n_t^3 c_t / width + dr,        dw_j += sum_t dh_tj n_t r_tj
//
// Bound by HBM: forward 2 (x, h) to 4 (y, r too) passes over the stream, backward 3 to 4, next to no arithmetic.  A row stays
// in the registers of the threads that share it, so that it is read once: a warp up to 256 vectors of 16 bytes (2048 bf16
// columns), four or sixteen warps beyond; all of a thread's loads are issued before the first is used.  Rows whose bytes are no
// multiple of 16, and misaligned tensors, go element by element through the same kernels.
// Sums of squares, the statistics and the gradient of w are fp32; h is formed from the unrounded sum r.
#include <cuda_fp8.h>

#include <type_traits>

#include "common.cuh"

namespace unipool {

namespace {

constexpr int kNormMaxWidth = 16384;
constexpr float kE4m3Max = 448.f;
constexpr float kSmallestScale = 1.17549435e-38f;        // 2^-126: its reciprocal is finite, a row of zeros keeps zeros

// V consecutive elements as they lie in memory: 16 bytes, or a single element where those do not fit.
template <typename E, int V> struct Vec;
template <> struct Vec<__nv_bfloat16, 8> {
  uint4 raw;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { raw = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void zero() { raw = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  __device__ __forceinline__ static void store(__nv_bfloat16* p, const float (&v)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&b);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  }
};
template <> struct Vec<float, 4> {
  float4 raw;
  __device__ __forceinline__ void load(const float* p) { raw = *reinterpret_cast<const float4*>(p); }
  __device__ __forceinline__ void zero() { raw = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ void get(float (&v)[4]) const { v[0] = raw.x; v[1] = raw.y; v[2] = raw.z; v[3] = raw.w; }
  __device__ __forceinline__ static void store(float* p, const float (&v)[4]) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  }
};
template <typename E> struct Vec<E, 1> {
  E raw;
  __device__ __forceinline__ void load(const E* p) { raw = *p; }
  __device__ __forceinline__ void zero() { raw = from_f32<E>(0.f); }
  __device__ __forceinline__ void get(float (&v)[1]) const { v[0] = to_f32(raw); }
  __device__ __forceinline__ static void store(E* p, const float (&v)[1]) { *p = from_f32<E>(v[0]); }
};

template <int V> __device__ __forceinline__ void load_w(const float* w, float (&v)[V]) {
  if constexpr (V == 1) {
    v[0] = __ldg(w);
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

// The row's value of op over the TPR threads that share it, the same in all of them.  (TPR > 32: the block; `part` one
// value per warp, not read by anyone any more.)
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
      for (int j = 0; j < V; ++j) v[i][j] *= n * w[j];
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
  int T, width;
  bool add;         // one block: add to what dw holds
};

template <int TPR> constexpr int kNormBwdThreads = TPR == 32 ? 256 : TPR;

// Blocks walk over the rows; a thread sums dw of its columns over its rows, a block over its warps in their order, so that the
// result does not depend on who is first.
template <typename E, int V, int TPR, int VPT>
__global__ void __launch_bounds__(kNormBwdThreads<TPR>) rmsnorm_bwd_kernel(NormBwdParams p) {
  grid_wait(p.dh, p.r, p.dr, p.w, p.rstd);
  extern __shared__ float sums[];                        // [width] (TPR = 32)
  __shared__ float part[2][TPR > 32 ? TPR / 32 : 1];
  constexpr int kRows = kNormBwdThreads<TPR> / TPR;
  const int t = threadIdx.x % TPR;
  float dw[VPT][V];
#pragma unroll
  for (int i = 0; i < VPT; ++i)
#pragma unroll
    for (int j = 0; j < V; ++j) dw[i][j] = 0.f;
  int turn = 0;
  for (int64_t row = blockIdx.x * kRows + threadIdx.x / TPR; row < p.T; row += (int64_t)gridDim.x * kRows, turn ^= 1) {
    const int64_t at = row * p.width;
    const E* dh = static_cast<const E*>(p.dh) + at;
    const E* r = static_cast<const E*>(p.r) + at;
    const E* dr = static_cast<const E*>(p.dr) + at;
    Vec<E, V> a[VPT], b[VPT], d[VPT];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int c = (i * TPR + t) * V;
      a[i].zero();
      b[i].zero();
      if (c < p.width) { a[i].load(dh + c); b[i].load(r + c); }
    }
    if (p.dr != nullptr) {
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        const int c = (i * TPR + t) * V;
        d[i].zero();
        if (c < p.width) d[i].load(dr + c);
      }
    }
    const float n = __ldg(p.rstd + row);
    float dot = 0.f;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int c = (i * TPR + t) * V;
      if (c >= p.width) continue;
      float u[V], v[V], w[V];
      a[i].get(u);
      b[i].get(v);
      load_w<V>(p.w + c, w);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        dw[i][j] = fmaf(u[j], v[j] * n, dw[i][j]);
        dot = fmaf(u[j] * w[j], v[j], dot);
      }
    }
    dot = row_reduce<TPR>(dot, part[turn], [](float m, float o) { return m + o; });   // (two, for the next row's writers)
    const float k = n * n * n * (dot / (float)p.width);
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int c = (i * TPR + t) * V;
      if (c >= p.width) continue;
      float u[V], v[V], w[V];
      a[i].get(u);
      b[i].get(v);
      load_w<V>(p.w + c, w);
#pragma unroll
      for (int j = 0; j < V; ++j) u[j] = n * w[j] * u[j] - v[j] * k;
      if (p.dr != nullptr) {
        d[i].get(v);
#pragma unroll
        for (int j = 0; j < V; ++j) u[j] += v[j];
      }
      Vec<E, V>::store(static_cast<E*>(p.dx) + at + c, u);
    }
  }
  if (p.dw == nullptr) return;
  float* out = &p.dw[(int64_t)blockIdx.x * p.width];
  if constexpr (TPR == 32) {
    for (int g = 0; g < kRows; ++g) {
      if ((int)threadIdx.x / 32 == g) {
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
          const int c = (i * TPR + t) * V;
          if (c >= p.width) continue;
#pragma unroll
          for (int j = 0; j < V; ++j) sums[c + j] = g == 0 ? dw[i][j] : sums[c + j] + dw[i][j];
        }
      }
      __syncthreads();
    }
    for (int c = threadIdx.x; c < p.width; c += blockDim.x) out[c] = p.add ? out[c] + sums[c] : sums[c];
  } else {
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int c = (i * TPR + t) * V;
      if (c >= p.width) continue;
#pragma unroll
      for (int j = 0; j < V; ++j) out[c + j] = p.add ? out[c + j] + dw[i][j] : dw[i][j];
    }
  }
}

// Calls f(TPR, VPT) as compile-time numbers for rows of `n` vectors.
template <int N> using Int = std::integral_constant<int, N>;
template <bool kScalar, typename F> int by_width(int n, F f) {
  if constexpr (!kScalar) {
    if (n <= 32) return f(Int<32>(), Int<1>());
    if (n <= 64) return f(Int<32>(), Int<2>());
    if (n <= 96) return f(Int<32>(), Int<3>());
    if (n <= 128) return f(Int<32>(), Int<4>());
    if (n <= 192) return f(Int<32>(), Int<6>());
    if (n <= 256) return f(Int<32>(), Int<8>());
    if (n <= 512) return f(Int<128>(), Int<4>());
    if (n <= 1024) return f(Int<128>(), Int<8>());
    if (n <= 2048) return f(Int<512>(), Int<4>());
    return f(Int<512>(), Int<8>());
  } else {
    if (n <= 256) return f(Int<32>(), Int<8>());
    if (n <= 1024) return f(Int<128>(), Int<8>());
    if (n <= 4096) return f(Int<512>(), Int<8>());
    return f(Int<512>(), Int<32>());
  }
}

// Calls f(E, V, TPR, VPT) for the element type and what of the rows fits 16-byte accesses.
template <typename E, typename F> int by_row(bool vec, int width, F f) {
  constexpr int V = 16 / (int)sizeof(E);
  if (vec) return by_width<false>(width / V, [&](auto tpr, auto vpt) { return f(E(), Int<V>(), tpr, vpt); });
  return by_width<true>(width, [&](auto tpr, auto vpt) { return f(E(), Int<1>(), tpr, vpt); });
}

template <bool kNorm, typename E> int norm_as(unipool_ctx* ctx, const NormParams& p, cudaStream_t s) {
  const uintptr_t rows = reinterpret_cast<uintptr_t>(p.x) | reinterpret_cast<uintptr_t>(p.y) | reinterpret_cast<uintptr_t>(p.r) |
                         reinterpret_cast<uintptr_t>(p.h) | reinterpret_cast<uintptr_t>(p.w);
  const bool vec = (int64_t)p.width * sizeof(E) % 16 == 0 && rows % 16 == 0 && reinterpret_cast<uintptr_t>(p.q) % 8 == 0;
  return by_row<E>(vec, p.width, [&](auto e, auto v, auto tpr, auto vpt) {
    constexpr int kRows = kNormThreads<tpr> / tpr;
    PhaseTimer pt(ctx, UNIPOOL_PH_RMSNORM, 1, s);
    UP_KERNEL((rmsnorm_kernel<decltype(e), v, tpr, vpt, kNorm>), (p.T + kRows - 1) / kRows, kNormThreads<tpr>, 0, s, p);
    return UNIPOOL_OK;
  });
}

// Blocks of the backward kernel: up to two to an SM, each with a row for every warp.
int norm_bwd_blocks(const unipool_ctx* ctx, int T, int rows) {
  const int most = 2 * ctx->sm_count, all = (T + rows - 1) / rows;
  return all < most ? all : most;
}

template <typename E> int norm_bwd_as(unipool_ctx* ctx, NormBwdParams p, float* scratch, bool overwrite, cudaStream_t s) {
  const uintptr_t rows = reinterpret_cast<uintptr_t>(p.dh) | reinterpret_cast<uintptr_t>(p.r) | reinterpret_cast<uintptr_t>(p.dr) |
                         reinterpret_cast<uintptr_t>(p.dx) | reinterpret_cast<uintptr_t>(p.w);
  const bool vec = (int64_t)p.width * sizeof(E) % 16 == 0 && rows % 16 == 0;
  return by_row<E>(vec, p.width, [&](auto e, auto v, auto tpr, auto vpt) {
    constexpr int kRows = kNormBwdThreads<tpr> / tpr;
    const int blocks = norm_bwd_blocks(ctx, p.T, kRows);
    float* dw = p.dw;
    const bool split = dw != nullptr && blocks > 1;
    NormBwdParams a = p;
    a.add = !overwrite && !split;
    if (split) a.dw = scratch;
    PhaseTimer pt(ctx, UNIPOOL_PH_RMSNORM_BWD, split ? 2 : 1, s);
    auto kern = rmsnorm_bwd_kernel<decltype(e), v, tpr, vpt>;
    UP_KERNEL(kern, blocks, kNormBwdThreads<tpr>, tpr == 32 ? p.width * sizeof(float) : 0, s, a);
    return split ? column_sum_launch(scratch, blocks, p.width, dw, !overwrite, s) : UNIPOOL_OK;
  });
}

}  // namespace

int norm_max_width() { return kNormMaxWidth; }

// (The most blocks that any width and alignment takes.)
size_t rmsnorm_bwd_scratch(const unipool_ctx* ctx, int T, int width) {
  const int most = 2 * ctx->sm_count;
  return (size_t)(T < most ? T : most) * width * sizeof(float);
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
  const NormBwdParams p{dh, r, dr, w, rstd, dx, dw, T, width, false};
  return ctx->cfg.dtype == UNIPOOL_BF16 ? norm_bwd_as<__nv_bfloat16>(ctx, p, scratch, overwrite, s)
                                        : norm_bwd_as<float>(ctx, p, scratch, overwrite, s);
}

}  // namespace unipool
