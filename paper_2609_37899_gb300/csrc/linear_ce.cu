// linear_ce.cu -- linear cross entropy and its gradients in pieces of the
// vocabulary (soma_linear_ce_* in include/soma_api.h have the formulas).
#include <cmath>

#define SOMA_CHECK_FILE 10
#include "checked.cuh"
#include "numeric.cuh"
#include "soma_api.h"
#include "soma_launch.h"

namespace soma {

namespace {

constexpr int kTile = 64, kDepth = 16;
constexpr size_t kPieceBytes = (size_t)256 << 20;  // of the logits of one piece

// What a row takes part with: its target, or -1 for a row without gradient.
struct RowInfo {
  float lse, g;
  int64_t y;
};

__device__ __forceinline__ bool row_live(int64_t y, int64_t ignore, int64_t vocab, float lse) {
  return y != ignore && y >= 0 && y < vocab && isfinite(lse);
}

// C[m][n] = sum_k A[m][k] B[k][n] on a 64 x 64 tile: A, B by row and column
// strides; `rows` (may be null) masks the k (transposed A) whose row is dead.
template <typename TA, typename TB, typename F>
__device__ __forceinline__ void tile_product(const TA* a, int64_t am, int64_t ak, const TB* b,
                                             int64_t bk, int64_t bn, int64_t M, int64_t N,
                                             int64_t K, F f) {
  __shared__ float sa[kDepth][kTile + 1], sb[kDepth][kTile + 1];
  const int64_t m0 = (int64_t)blockIdx.y * kTile, n0 = (int64_t)blockIdx.x * kTile;
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  float acc[4][4] = {};
  for (int64_t k0 = 0; k0 < K; k0 += kDepth) {
    for (int j = threadIdx.x; j < kDepth * kTile; j += 256) {
      const int k = j % kDepth, m = j / kDepth;
      sa[k][m] = m0 + m < M && k0 + k < K ? to_f32(a[(m0 + m) * am + (k0 + k) * ak]) : 0.f;
      const int kk = j / kTile, n = j % kTile;
      sb[kk][n] = n0 + n < N && k0 + kk < K ? to_f32(b[(k0 + kk) * bk + (n0 + n) * bn]) : 0.f;
    }
    __syncthreads();
    for (int k = 0; k < kDepth; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          acc[i][j] = fmaf(sa[k][ty * 4 + i], sb[k][tx * 4 + j], acc[i][j]);
    __syncthreads();
  }
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const int64_t m = m0 + ty * 4 + i, n = n0 + tx * 4 + j;
      if (m < M && n < N) f(m, n, acc[i][j]);
    }
}

template <typename T>
__global__ void __launch_bounds__(256)
logits_kernel(const T* h, int64_t hs, const T* emb, int64_t es, int64_t rows, int64_t width,
              int64_t dim, float* out) {
  tile_product(h, hs, 1, emb, 1, es, rows, width, dim,
               [&](int64_t m, int64_t n, float x) { out[m * width + n] = x; });
}

// Joins one piece's logits of a row to its running maximum and sum.
__global__ void stats_kernel(const float* logits, int64_t width, int64_t v0, int64_t vocab,
                             const int64_t* targets, int64_t ignore, float* top, float* sum,
                             float* own, float* loss, float* lse, int* status) {
  const int64_t n = blockIdx.x;
  const int64_t y = targets[n];
  const float* x = logits + n * width;
  float m = v0 ? top[n] : -INFINITY;
  __shared__ float red[8];
  float mx = -INFINITY;
  for (int64_t j = threadIdx.x; j < width; j += 256) mx = fmaxf(mx, x[j]);
  for (int s = 16; s; s >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, s));
  if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = mx;
  __syncthreads();
  float now = m;
  for (int j = 0; j < 8; ++j) now = fmaxf(now, red[j]);
  __syncthreads();
  const float ref = isinf(now) ? 0.f : now;
  float s = 0.f;
  for (int64_t j = threadIdx.x; j < width; j += 256) s += expf(x[j] - ref);
  for (int k = 16; k; k >>= 1) s += __shfl_xor_sync(0xffffffffu, s, k);
  if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = s;
  __syncthreads();
  if (threadIdx.x) return;
  s = v0 ? sum[n] * expf(m - ref) : 0.f;
  for (int j = 0; j < 8; ++j) s += red[j];
  top[n] = now;
  sum[n] = s;
  if (y >= v0 && y < v0 + width) own[n] = x[y - v0];
  if (v0 + width < vocab) return;
  if (y == ignore) {
    loss[n] = lse[n] = 0.f;
    return;
  }
  const float l = now + logf(s);
  const float r = y >= 0 && y < vocab ? l - own[n] : NAN;
  lse[n] = l;
  loss[n] = isfinite(r) ? r : NAN;
  if (!isfinite(r)) atomicCAS(status, 0, SOMA_ERR_NONFINITE);
}

// Per row: lse, gradient and target where it takes part; a copy of h with
// the other rows zeroed.
template <typename T>
__global__ void rows_kernel(const T* h, int64_t hs, int64_t dim, const int64_t* targets,
                            int64_t ignore, int64_t vocab, const float* lse, const float* dloss,
                            RowInfo* info, T* copy, int64_t cs, float* top) {
  const int64_t n = blockIdx.x;
  const int64_t y = targets[n];
  const bool live = row_live(y, ignore, vocab, lse[n]);
  if (threadIdx.x == 0) {
    info[n] = {lse[n], live ? dloss[n] : 0.f, live ? y : -1};
    // non-negative floats order as their bits do
    if (live && isfinite(dloss[n]))
      atomicMax(reinterpret_cast<int*>(top), __float_as_int(fabsf(dloss[n])));
  }
  for (int64_t j = threadIdx.x; j < cs; j += blockDim.x)
    copy[n * cs + j] = live && j < dim ? h[n * hs + j] : from_f32<T>(0.f);
}

// The power of two that the 16-bit G is scaled by.
template <typename T>
__device__ __forceinline__ float g_scale(float) { return 1.f; }
template <>
__device__ __forceinline__ float g_scale<__half>(float top) {
  int e = 0;
  frexpf(top, &e);  // top in [2^(e-1), 2^e)
  return top > 0.f ? exp2f((float)(14 - e)) : 1.f;
}

template <typename T>
__global__ void __launch_bounds__(256)
grad_kernel(const T* h, int64_t hs, const T* emb, int64_t es, int64_t rows, int64_t width,
            int64_t dim, int64_t v0, const RowInfo* info, const float* top, T* G) {
  const float scale = g_scale<T>(*top);
  tile_product(h, hs, 1, emb, 1, es, rows, width, dim, [&](int64_t m, int64_t n, float x) {
    const RowInfo r = info[m];
    float g = 0.f;
    if (r.y >= 0) g = scale * r.g * (expf(x - r.lse) - (r.y == v0 + n ? 1.f : 0.f));
    G[m * width + n] = from_f32<T>(g);
  });
}

template <typename T>
__global__ void __launch_bounds__(256)
dh_kernel(const T* G, int64_t width, const T* emb, int64_t es, int64_t rows, int64_t dim,
          bool first, const RowInfo* info, float* acc) {
  tile_product(G, width, 1, emb, es, 1, rows, dim, width, [&](int64_t m, int64_t n, float x) {
    if (info[m].y < 0) x = 0.f;
    acc[m * dim + n] = first ? x : acc[m * dim + n] + x;
  });
}

template <typename T>
__global__ void dh_round_kernel(const float* acc, int64_t rows, int64_t dim, const float* top,
                                T* dh, int64_t ds) {
  const int64_t n = blockIdx.x;
  const float unscale = 1.f / g_scale<T>(*top);
  for (int64_t j = threadIdx.x; j < dim; j += blockDim.x)
    dh[n * ds + j] = from_f32<T>(acc[n * dim + j] * unscale);
}

template <typename T>
__global__ void __launch_bounds__(256)
demb_kernel(const T* G, int64_t width, const T* h, int64_t hs, int64_t rows, int64_t dim,
            const float* top, T* demb, int64_t ds) {
  const float unscale = 1.f / g_scale<T>(*top);
  tile_product(G, 1, width, h, hs, 1, width, dim, rows, [&](int64_t m, int64_t n, float x) {
    demb[m * ds + n] = from_f32<T>(x * unscale);
  });
}

size_t round256(size_t x) { return (x + 255) / 256 * 256; }

struct Plan {
  int64_t piece;  // vocabulary entries of one piece
  size_t logits, top, sum, own;           // forward
  size_t g, info, copy, acc, gtop, total;  // backward
};

bool dims_ok(const soma_linear_ce_dims& d) {
  return d.rows >= 0 && d.rows <= (1 << 30) && d.vocab >= 1 && d.vocab <= (1 << 30) &&
         d.dim >= 1 && d.dim <= 65536 && d.h_stride >= d.dim && d.emb_stride >= d.dim &&
         d.h_stride <= ((int64_t)1 << 32) && d.emb_stride <= ((int64_t)1 << 32) &&
         (d.dtype == SOMA_BF16 || d.dtype == SOMA_FP16);
}

Plan plan(const soma_linear_ce_dims& d, bool backward) {
  Plan p = {};
  size_t at = 0;
  const auto take = [&](size_t bytes) {
    const size_t o = at;
    at += round256(bytes);
    return o;
  };
  const int64_t rows = d.rows ? d.rows : 1;
  p.piece = (int64_t)(kPieceBytes / 4) / rows / kTile * kTile;
  if (p.piece < kTile) p.piece = kTile;
  if (p.piece > d.vocab) p.piece = d.vocab;
  if (!backward) {
    p.logits = take((size_t)rows * p.piece * 4);
    p.top = take((size_t)rows * 4);
    p.sum = take((size_t)rows * 4);
    p.own = take((size_t)rows * 4);
  } else {
    p.g = take((size_t)rows * p.piece * 2);
    p.info = take((size_t)rows * sizeof(RowInfo));
    p.copy = take((size_t)rows * ((d.dim + 7) / 8 * 8) * 2);
    p.acc = take((size_t)rows * d.dim * 4);
    p.gtop = take(4);
  }
  p.total = at;
  return p;
}

bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

dim3 tiles(int64_t m, int64_t n) {
  return dim3((unsigned)((n + kTile - 1) / kTile), (unsigned)((m + kTile - 1) / kTile));
}

template <typename T>
cudaError_t forward(const T* h, const T* emb, const soma_linear_ce_dims& d, const int64_t* targets,
                    int64_t ignore, float* loss, float* lse, uint8_t* ws, int* status,
                    cudaStream_t st) {
  const Plan p = plan(d, false);
  float* logits = reinterpret_cast<float*>(ws + p.logits);
  for (int64_t v0 = 0; v0 < d.vocab; v0 += p.piece) {
    const int64_t width = d.vocab - v0 < p.piece ? d.vocab - v0 : p.piece;
    logits_kernel<T><<<tiles(d.rows, width), 256, 0, st>>>(
        h, d.h_stride, emb + v0 * d.emb_stride, d.emb_stride, d.rows, width, d.dim, logits);
    stats_kernel<<<(unsigned)d.rows, 256, 0, st>>>(
        logits, width, v0, d.vocab, targets, ignore, reinterpret_cast<float*>(ws + p.top),
        reinterpret_cast<float*>(ws + p.sum), reinterpret_cast<float*>(ws + p.own), loss, lse,
        status);
  }
  return cudaGetLastError();
}

template <typename T>
cudaError_t backward(const T* h, const T* emb, const soma_linear_ce_dims& d,
                     const int64_t* targets, int64_t ignore, const float* lse, const float* dloss,
                     T* dh, int64_t dhs, T* demb, int64_t des, uint8_t* ws, cudaStream_t st) {
  const Plan p = plan(d, true);
  RowInfo* info = reinterpret_cast<RowInfo*>(ws + p.info);
  T* copy = reinterpret_cast<T*>(ws + p.copy);
  T* G = reinterpret_cast<T*>(ws + p.g);
  float* top = reinterpret_cast<float*>(ws + p.gtop);
  float* acc = reinterpret_cast<float*>(ws + p.acc);
  const int64_t cs = (d.dim + 7) / 8 * 8;
  cudaMemsetAsync(top, 0, 4, st);
  if (d.rows)
    rows_kernel<T><<<(unsigned)d.rows, 128, 0, st>>>(h, d.h_stride, d.dim, targets, ignore,
                                                     d.vocab, lse, dloss, info, copy, cs, top);
  for (int64_t v0 = 0; v0 < d.vocab; v0 += p.piece) {
    const int64_t width = d.vocab - v0 < p.piece ? d.vocab - v0 : p.piece;
    const T* e = emb + v0 * d.emb_stride;
    if (d.rows) {
      grad_kernel<T><<<tiles(d.rows, width), 256, 0, st>>>(
          copy, cs, e, d.emb_stride, d.rows, width, d.dim, v0, info, top, G);
      dh_kernel<T><<<tiles(d.rows, d.dim), 256, 0, st>>>(G, width, e, d.emb_stride, d.rows, d.dim,
                                                         v0 == 0, info, acc);
    }
    demb_kernel<T><<<tiles(width, d.dim), 256, 0, st>>>(G, width, copy, cs, d.rows, d.dim, top,
                                                        demb + v0 * des, des);
  }
  if (d.rows)
    dh_round_kernel<T><<<(unsigned)d.rows, 128, 0, st>>>(acc, d.rows, d.dim, top, dh, dhs);
  return cudaGetLastError();
}

}  // namespace

}  // namespace soma

using namespace soma;

extern "C" {

size_t soma_linear_ce_workspace_bytes(soma_linear_ce_dims d, int backward) {
  if (!dims_ok(d)) return 0;
  return plan(d, backward != 0).total;
}

int soma_linear_ce_forward(const void* h, const void* emb, soma_linear_ce_dims d,
                           const int64_t* targets, int64_t ignore_index, float* loss, float* lse,
                           void* workspace, size_t workspace_bytes, void* stream) {
  if (!dims_ok(d)) return SOMA_ERR_UNSUPPORTED;
  if (d.rows == 0) return SOMA_OK;
  if (!h || !emb || !targets || !loss || !lse || !aligned(h, 16) || !aligned(emb, 16) ||
      !aligned(targets, 8) || !aligned(loss, 4) || !aligned(lse, 4))
    return SOMA_ERR_INVALID_ARG;
  if (!workspace || !aligned(workspace, 16) || workspace_bytes < plan(d, false).total)
    return SOMA_ERR_WORKSPACE;
  int* status = status_ptr();
  if (!status) return SOMA_ERR_CUDA;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  const cudaStream_t st = (cudaStream_t)stream;
  trace_begin(SOMA_TRACE_HEAD, st);
  const cudaError_t e =
      d.dtype == SOMA_BF16
          ? forward(static_cast<const __nv_bfloat16*>(h), static_cast<const __nv_bfloat16*>(emb),
                    d, targets, ignore_index, loss, lse, ws, status, st)
          : forward(static_cast<const __half*>(h), static_cast<const __half*>(emb), d, targets,
                    ignore_index, loss, lse, ws, status, st);
  trace_end(SOMA_TRACE_HEAD, st);
  return e == cudaSuccess ? SOMA_OK : SOMA_ERR_CUDA;
}

int soma_linear_ce_backward(const void* h, const void* emb, soma_linear_ce_dims d,
                            const int64_t* targets, int64_t ignore_index, const float* lse,
                            const float* dloss, void* dh, int64_t dh_stride, void* demb,
                            int64_t demb_stride, void* workspace, size_t workspace_bytes,
                            void* stream) {
  if (!dims_ok(d)) return SOMA_ERR_UNSUPPORTED;
  if (!emb || !demb || !aligned(emb, 16) || !aligned(h, 16) || !aligned(demb, 2) ||
      !aligned(dh, 2) || !aligned(targets, 8) || !aligned(lse, 4) || !aligned(dloss, 4) ||
      dh_stride < d.dim || demb_stride < d.dim || dh_stride > ((int64_t)1 << 32) ||
      demb_stride > ((int64_t)1 << 32) || (d.rows && (!h || !targets || !lse || !dloss || !dh)))
    return SOMA_ERR_INVALID_ARG;
  if (!workspace || !aligned(workspace, 16) || workspace_bytes < plan(d, true).total)
    return SOMA_ERR_WORKSPACE;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  const cudaStream_t st = (cudaStream_t)stream;
  trace_begin(SOMA_TRACE_HEAD, st);
  const cudaError_t e =
      d.dtype == SOMA_BF16
          ? backward(static_cast<const __nv_bfloat16*>(h), static_cast<const __nv_bfloat16*>(emb),
                     d, targets, ignore_index, lse, dloss, static_cast<__nv_bfloat16*>(dh),
                     dh_stride, static_cast<__nv_bfloat16*>(demb), demb_stride, ws, st)
          : backward(static_cast<const __half*>(h), static_cast<const __half*>(emb), d, targets,
                     ignore_index, lse, dloss, static_cast<__half*>(dh), dh_stride,
                     static_cast<__half*>(demb), demb_stride, ws, st);
  trace_end(SOMA_TRACE_HEAD, st);
  return e == cudaSuccess ? SOMA_OK : SOMA_ERR_CUDA;
}

}  // extern "C"
