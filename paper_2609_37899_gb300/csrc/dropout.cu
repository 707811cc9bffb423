// dropout.cu -- dropout with the residual's addition, the mask from the
// counter-based generator (soma_dropout in include/soma_api.h).
//
// Eight elements of a row-major count share a Philox block, 16 bits each, so a
// thread owns such a group: 60 instructions of generator for 8 elements.
// 65536 x 1376 bf16, after a flush of L2: 84 us with a residual and 68 without, 6.4 and
// 5.3 TB/s (in fp32 158 and 109 us, 6.9 and 6.6 TB/s): two streams of 16 bits do not
// quite hide the generator.  Comparing halves where they are instead of making a mask, and packed
// conversions, were 2 to 6 us slower.
#include <cmath>

#define SOMA_CHECK_FILE 12
#include "checked.cuh"
#include "numeric.cuh"
#include "pdl.cuh"
#include "soma_api.h"
#include "soma_launch.h"

namespace soma {

namespace {

constexpr int kThreads = 256;
constexpr uint32_t kDomain = 0x80000003u;  // counter word 3: disjoint from all other streams

struct Dropout {
  int64_t xs, rs, ys;         // elements between rows
  int64_t rows, cols, count;  // count = rows * cols
  uint32_t k0, k1;            // seed halves
  uint64_t offset;
  const uint64_t* counter;
  uint32_t drop;              // an element whose 16 bits are below this is dropped
  float scale;
  int* status;
};

// Bit j: whether element 8 q + j is kept.
__device__ __forceinline__ uint32_t kept(const Dropout& d, uint32_t q, uint64_t call) {
  const uint4 w = philox4x32_10(make_uint4(q, (uint32_t)call, (uint32_t)(call >> 32), kDomain),
                                d.k0, d.k1);
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t v = word_of(w, j);
    m |= ((v & 0xffffu) >= d.drop ? 1u : 0u) << (2 * j);
    m |= ((v >> 16) >= d.drop ? 1u : 0u) << (2 * j + 1);
  }
  return m;
}

// Groups that lie in one row, 16-byte aligned on every side.
template <typename T, bool RESIDUAL>
__global__ void __launch_bounds__(kThreads)
dropout_groups_kernel(const T* x, const T* residual, T* y, const Dropout d, uint32_t row_groups) {
  admit_successor();
  after_predecessor();
  const int64_t q = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (q * 8 >= d.count) return;
  // no division where all is one row
  const uint32_t row = row_groups == UINT32_MAX ? 0 : (uint32_t)q / row_groups;
  const int64_t at = (int64_t)((uint32_t)q - row * row_groups) * 8;
  if (!SOMA_CHECK(row < d.rows && at >= 0 && at + 8 <= d.cols, d.status)) return;
  float a[8], r[8], o[8];
  load8(x + row * d.xs + at, a);
  if (RESIDUAL) load8(residual + row * d.rs + at, r);
  const uint32_t m = kept(d, (uint32_t)q, d.offset + (d.counter ? *d.counter : 0));
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float v = m >> j & 1u ? a[j] * d.scale : 0.f;
    o[j] = RESIDUAL ? v + r[j] : v;
  }
  store8(y + row * d.ys + at, o);
}

// Any strides: a warp owns 256 elements in a row-major count, each lane the mask
// of one group.  Lane l reads elements l, 32 + l, ... and gets their groups'
// masks from the lanes that made them.  One element per lane and access: 3001 x 681
// fp16 14 us with a residual, 60000 x 681 143 us, 1.7 TB/s.
template <typename T, bool RESIDUAL>
__global__ void __launch_bounds__(kThreads)
dropout_kernel(const T* x, const T* residual, T* y, const Dropout d) {
  admit_successor();
  after_predecessor();
  const int lane = threadIdx.x % 32;
  const int64_t first = ((int64_t)blockIdx.x * (kThreads / 32) + threadIdx.x / 32) * 256;
  if (first >= d.count) return;
  const uint32_t mask =
      kept(d, (uint32_t)(first / 8) + lane, d.offset + (d.counter ? *d.counter : 0));
  const int64_t e = first + lane;  // 64-bit divisions only where they are needed
  int64_t row = d.count <= UINT32_MAX ? (uint32_t)e / (uint32_t)d.cols : e / d.cols;
  int64_t col = e - row * d.cols;
  const int64_t down = d.cols > 32 ? 0 : 32 / (uint32_t)d.cols;  // 32 elements further
  const int64_t right = 32 - down * d.cols;
  float a[8], r[8];
  int64_t to[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const bool there = first + 32 * j + lane < d.count &&
                       SOMA_CHECK(row >= 0 && row < d.rows && col >= 0 && col < d.cols, d.status);
    to[j] = there ? row * d.ys + col : -1;
    a[j] = there ? to_f32(x[row * d.xs + col]) : 0.f;
    r[j] = RESIDUAL && there ? to_f32(residual[row * d.rs + col]) : 0.f;
    row += down;
    col += right;
    if (col >= d.cols) {
      col -= d.cols;
      ++row;
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t m = __shfl_sync(0xffffffffu, mask, 4 * j + lane / 8);
    const float v = m >> (lane & 7) & 1u ? a[j] * d.scale : 0.f;
    if (to[j] >= 0) y[to[j]] = from_f32<T>(RESIDUAL ? v + r[j] : v);
  }
}

bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

template <typename T, bool RESIDUAL>
cudaError_t launch(const void* x, const void* residual, void* y, Dropout d, cudaStream_t st) {
  const T *px = static_cast<const T*>(x), *pr = static_cast<const T*>(residual);
  T* py = static_cast<T*>(y);
  constexpr int piece = 16 / sizeof(T);  // elements of a 16-byte access
  const bool wide = aligned(x, 16) && aligned(y, 16) && aligned(residual, 16);
  if (d.xs == d.cols && d.ys == d.cols && (!RESIDUAL || d.rs == d.cols) && d.count % 8 == 0) {
    d.cols = d.count;  // no gaps: one row
    d.rows = 1;
  }
  const bool rows_wide = d.rows <= 1 || (d.xs % piece == 0 && d.ys % piece == 0 &&
                                         (!RESIDUAL || d.rs % piece == 0));
  const int64_t groups = (d.count + 7) / 8;
  if (wide && rows_wide && d.cols % 8 == 0)
    return launch_overlapped(dropout_groups_kernel<T, RESIDUAL>,
                             dim3((unsigned)((groups + kThreads - 1) / kThreads)), kThreads, 0, st,
                             px, pr, py, d, (uint32_t)(d.rows <= 1 ? UINT32_MAX : d.cols / 8));
  return launch_overlapped(dropout_kernel<T, RESIDUAL>,
                           dim3((unsigned)((groups + kThreads - 1) / kThreads)), kThreads, 0, st,
                           px, pr, py, d);
}

template <typename T>
cudaError_t run(const void* x, const void* residual, void* y, const Dropout& d, cudaStream_t st) {
  return residual ? launch<T, true>(x, residual, y, d, st) : launch<T, false>(x, residual, y, d, st);
}

}  // namespace
}  // namespace soma

using namespace soma;

extern "C" int soma_dropout(const void* x, int64_t x_stride, const void* residual,
                            int64_t residual_stride, void* y, int64_t y_stride, int dtype,
                            int64_t rows, int64_t cols, double p, uint64_t seed, uint64_t offset,
                            const uint64_t* counter, void* stream) {
  const int64_t most = (int64_t)1 << 34;
  if (rows < 0 || cols < 0 || (cols && rows > most / cols)) return SOMA_ERR_UNSUPPORTED;
  if (dtype != SOMA_FP32 && dtype != SOMA_BF16 && dtype != SOMA_FP16) return SOMA_ERR_INVALID_ARG;
  const size_t width = dtype == SOMA_FP32 ? 4 : 2;
  if (!(p >= 0 && p <= 1) || x_stride < cols || y_stride < cols ||
      (residual && residual_stride < cols) || !aligned(x, width) || !aligned(y, width) ||
      !aligned(residual, width) || !aligned(counter, 8))
    return SOMA_ERR_INVALID_ARG;
  if (rows == 0 || cols == 0) return SOMA_OK;
  if (!x || !y) return SOMA_ERR_INVALID_ARG;
  int* status = status_ptr();
  if (!status) return SOMA_ERR_CUDA;
  Dropout d = {};
  d.status = status;
  d.xs = x_stride;
  d.rs = residual_stride;
  d.ys = y_stride;
  d.rows = rows;
  d.cols = cols;
  d.count = rows * cols;
  d.k0 = (uint32_t)seed;
  d.k1 = (uint32_t)(seed >> 32);
  d.offset = offset;
  d.counter = counter;
  d.drop = (uint32_t)std::nearbyint(p * 65536.0);  // to even, as Python's round()
  d.scale = d.drop < 65536 ? (float)(65536.0 / (65536.0 - d.drop)) : 0.f;
  const cudaStream_t st = (cudaStream_t)stream;
  trace_begin(SOMA_TRACE_DROPOUT, st);
  const cudaError_t e = dtype == SOMA_FP32   ? run<float>(x, residual, y, d, st)
                        : dtype == SOMA_BF16 ? run<__nv_bfloat16>(x, residual, y, d, st)
                                             : run<__half>(x, residual, y, d, st);
  trace_end(SOMA_TRACE_DROPOUT, st);
  return e == cudaSuccess ? SOMA_OK : SOMA_ERR_CUDA;
}
