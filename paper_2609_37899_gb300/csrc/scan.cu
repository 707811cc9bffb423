// scan.cu -- the gated linear recurrence: forward, backward and the one-token
// form (soma_scan_* in include/soma_api.h have the formulas).
#define SOMA_CHECK_FILE 9
#include "checked.cuh"
#include "numeric.cuh"
#include "soma_api.h"
#include "soma_launch.h"

namespace soma {

namespace {

constexpr int kSegment = 16;  // steps between two checkpoints

__device__ __forceinline__ float sigmoid(float x) { return 1.f / (1.f + expf(-x)); }

struct Gates {
  float i, f, g, o;
};

template <typename T>
__device__ __forceinline__ Gates load_gates(const T* p, int64_t stride) {
  return {sigmoid(to_f32(p[0])), sigmoid(to_f32(p[stride])), tanhf(to_f32(p[2 * stride])),
          sigmoid(to_f32(p[3 * stride]))};
}

struct Scan {
  soma_scan_dims d;
  soma_scan_strides gs, hs, ds;
  const float* c0;
  const int32_t* lengths;
  const uint8_t* resets;
  float* c_last;
  float* marks;  // [batch][ceil(steps / kSegment)][dim]
};

__device__ __forceinline__ int64_t length_of(const Scan& s, int64_t b) {
  if (!s.lengths) return s.d.steps;
  const int64_t n = s.lengths[b];
  return n < 0 ? 0 : (n < s.d.steps ? n : s.d.steps);
}

// One thread per (sequence, channel) walks the steps in order.
template <typename T>
__global__ void scan_forward_kernel(const T* __restrict__ gates, Scan s, T* __restrict__ h) {
  const int64_t at = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (at >= s.d.batch * s.d.dim) return;
  const int64_t b = at / s.d.dim, ch = at % s.d.dim;
  const int64_t n = length_of(s, b), marks = (s.d.steps + kSegment - 1) / kSegment;
  float c = s.c0 ? s.c0[at] : 0.f;
  for (int64_t t = 0; t < s.d.steps; ++t) {
    if (s.marks && t % kSegment == 0) s.marks[(b * marks + t / kSegment) * s.d.dim + ch] = c;
    float y = 0.f;
    if (t < n) {
      const Gates a = load_gates(gates + b * s.gs.b + t * s.gs.t + ch, s.gs.g);
      if (s.resets && s.resets[b * s.d.steps + t]) c = 0.f;
      c = a.f * c + a.i * a.g;
      y = a.o * tanhf(c);
    }
    h[b * s.hs.b + t * s.hs.t + ch] = from_f32<T>(y);
  }
  if (s.c_last) s.c_last[at] = c;
}

// One thread per (sequence, channel) walks the segments backwards; a
// segment's states are computed again from its checkpoint.
template <typename T>
__global__ void scan_backward_kernel(const T* __restrict__ gates, Scan s,
                                     const T* __restrict__ dh, const float* __restrict__ dc_last,
                                     T* __restrict__ dgates, float* __restrict__ dc0) {
  const int64_t at = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (at >= s.d.batch * s.d.dim) return;
  const int64_t b = at / s.d.dim, ch = at % s.d.dim;
  const int64_t n = length_of(s, b), marks = (s.d.steps + kSegment - 1) / kSegment;
  float dc = dc_last ? dc_last[at] : 0.f;
  for (int64_t seg = marks - 1; seg >= 0; --seg) {
    const int64_t t0 = seg * kSegment;
    float prev[kSegment], next[kSegment];  // the states that a step takes and leaves
    float c = s.marks[(b * marks + seg) * s.d.dim + ch];
    for (int j = 0; j < kSegment; ++j) {
      const int64_t t = t0 + j;
      if (t >= n) break;
      const Gates a = load_gates(gates + b * s.gs.b + t * s.gs.t + ch, s.gs.g);
      prev[j] = s.resets && s.resets[b * s.d.steps + t] ? 0.f : c;
      next[j] = c = a.f * prev[j] + a.i * a.g;
    }
    for (int j = kSegment - 1; j >= 0; --j) {
      const int64_t t = t0 + j;
      if (t >= s.d.steps) continue;
      float d[4] = {0.f, 0.f, 0.f, 0.f};
      if (t < n) {
        const Gates a = load_gates(gates + b * s.gs.b + t * s.gs.t + ch, s.gs.g);
        const float y = to_f32(dh[b * s.hs.b + t * s.hs.t + ch]);
        const float th = tanhf(next[j]);
        dc += y * a.o * (1.f - th * th);
        d[0] = dc * a.g * a.i * (1.f - a.i);
        d[1] = dc * prev[j] * a.f * (1.f - a.f);
        d[2] = dc * a.i * (1.f - a.g * a.g);
        d[3] = y * th * a.o * (1.f - a.o);
        dc = s.resets && s.resets[b * s.d.steps + t] ? 0.f : dc * a.f;
      }
      for (int k = 0; k < 4; ++k)
        dgates[b * s.ds.b + t * s.ds.t + k * s.ds.g + ch] = from_f32<T>(d[k]);
    }
  }
  if (dc0) dc0[at] = dc;
}

template <typename T>
__global__ void scan_step_kernel(const T* __restrict__ gates, Scan s, float* __restrict__ c,
                                 T* __restrict__ h) {
  const int64_t at = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (at >= s.d.batch * s.d.dim) return;
  const int64_t b = at / s.d.dim, ch = at % s.d.dim;
  const Gates a = load_gates(gates + b * s.gs.b + ch, s.gs.g);
  const float x = a.f * c[at] + a.i * a.g;
  c[at] = x;
  h[b * s.hs.b + ch] = from_f32<T>(a.o * tanhf(x));
}

constexpr int kScanThreads = 64;

unsigned blocks(const soma_scan_dims& d) {
  return (unsigned)((d.batch * d.dim + kScanThreads - 1) / kScanThreads);
}

bool dims_ok(const soma_scan_dims& d) {
  return d.batch >= 0 && d.steps >= 0 && d.dim >= 0 && d.batch <= INT32_MAX &&
         d.steps <= INT32_MAX && d.dim <= (1 << 24) &&
         (d.dim == 0 || d.batch <= ((int64_t)1 << 36) / d.dim);
}

bool strides_ok(const soma_scan_strides& s) { return s.b >= 0 && s.t >= 0 && s.g >= 0; }

bool dtype_ok(int t) { return t == SOMA_FP32 || t == SOMA_BF16 || t == SOMA_FP16; }

// null pointers pass
bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

size_t width(int dtype) { return dtype == SOMA_FP32 ? 4 : 2; }

template <typename F>
cudaError_t with_type(int dtype, F f) {
  if (dtype == SOMA_FP32) f(float());
  else if (dtype == SOMA_BF16) f(__nv_bfloat16());
  else f(__half());
  return cudaGetLastError();
}

}  // namespace

}  // namespace soma

using namespace soma;

extern "C" {

int64_t soma_scan_checkpoint_count(soma_scan_dims d) {
  if (!dims_ok(d)) return -1;
  return d.batch * d.dim * ((d.steps + kSegment - 1) / kSegment);
}

int soma_scan_forward(const void* gates, soma_scan_strides gate_strides, int dtype,
                      soma_scan_dims d, const float* c0, const int32_t* lengths,
                      const uint8_t* resets, void* h, soma_scan_strides h_strides,
                      float* c_last, float* checkpoints, void* stream) {
  if (!dims_ok(d)) return SOMA_ERR_UNSUPPORTED;
  if (!dtype_ok(dtype) || !strides_ok(gate_strides) || !strides_ok(h_strides) ||
      !aligned(gates, width(dtype)) || !aligned(h, width(dtype)) || !aligned(c0, 4) ||
      !aligned(lengths, 4) || !aligned(c_last, 4) || !aligned(checkpoints, 4))
    return SOMA_ERR_INVALID_ARG;
  if (d.batch == 0 || d.dim == 0) return SOMA_OK;
  if (d.steps > 0 && (!gates || !h)) return SOMA_ERR_INVALID_ARG;
  const Scan s = {d, gate_strides, h_strides, {0, 0, 0}, c0, lengths, resets, c_last, checkpoints};
  const cudaStream_t st = (cudaStream_t)stream;
  trace_begin(SOMA_TRACE_GATE, st);
  const cudaError_t e = with_type(dtype, [&](auto x) {
    using T = decltype(x);
    scan_forward_kernel<<<blocks(d), kScanThreads, 0, st>>>(static_cast<const T*>(gates), s,
                                                             static_cast<T*>(h));
  });
  trace_end(SOMA_TRACE_GATE, st);
  return e == cudaSuccess ? SOMA_OK : SOMA_ERR_CUDA;
}

int soma_scan_backward(const void* gates, soma_scan_strides gate_strides, int dtype,
                       soma_scan_dims d, const float* checkpoints, const int32_t* lengths,
                       const uint8_t* resets, const void* dh, soma_scan_strides dh_strides,
                       const float* dc_last, void* dgates, soma_scan_strides dgate_strides,
                       float* dc0, void* stream) {
  if (!dims_ok(d)) return SOMA_ERR_UNSUPPORTED;
  if (!dtype_ok(dtype) || !strides_ok(gate_strides) || !strides_ok(dh_strides) ||
      !strides_ok(dgate_strides) || !aligned(gates, width(dtype)) || !aligned(dh, width(dtype)) ||
      !aligned(dgates, width(dtype)) || !aligned(checkpoints, 4) || !aligned(lengths, 4) ||
      !aligned(dc_last, 4) || !aligned(dc0, 4))
    return SOMA_ERR_INVALID_ARG;
  if (d.batch == 0 || d.dim == 0) return SOMA_OK;
  if (d.steps > 0 && (!gates || !dh || !dgates || !checkpoints)) return SOMA_ERR_INVALID_ARG;
  const Scan s = {d,       gate_strides, dh_strides, dgate_strides, nullptr,
                  lengths, resets,       nullptr,    const_cast<float*>(checkpoints)};
  const cudaStream_t st = (cudaStream_t)stream;
  trace_begin(SOMA_TRACE_GATE, st);
  const cudaError_t e = with_type(dtype, [&](auto x) {
    using T = decltype(x);
    scan_backward_kernel<<<blocks(d), kScanThreads, 0, st>>>(
        static_cast<const T*>(gates), s, static_cast<const T*>(dh), dc_last,
        static_cast<T*>(dgates), dc0);
  });
  trace_end(SOMA_TRACE_GATE, st);
  return e == cudaSuccess ? SOMA_OK : SOMA_ERR_CUDA;
}

int soma_scan_step(const void* gates, soma_scan_strides gate_strides, int dtype, int64_t batch,
                   int64_t dim, float* c, void* h, soma_scan_strides h_strides, void* stream) {
  const soma_scan_dims d = {batch, 1, dim};
  if (!dims_ok(d)) return SOMA_ERR_UNSUPPORTED;
  if (!dtype_ok(dtype) || !strides_ok(gate_strides) || !strides_ok(h_strides) ||
      !aligned(gates, width(dtype)) || !aligned(h, width(dtype)) || !aligned(c, 4))
    return SOMA_ERR_INVALID_ARG;
  if (batch == 0 || dim == 0) return SOMA_OK;
  if (!gates || !c || !h) return SOMA_ERR_INVALID_ARG;
  const Scan s = {d, gate_strides, h_strides, {0, 0, 0}, nullptr, nullptr, nullptr, nullptr,
                  nullptr};
  const cudaStream_t st = (cudaStream_t)stream;
  trace_begin(SOMA_TRACE_GATE, st);
  const cudaError_t e = with_type(dtype, [&](auto x) {
    using T = decltype(x);
    scan_step_kernel<<<blocks(d), kScanThreads, 0, st>>>(static_cast<const T*>(gates), s, c,
                                                          static_cast<T*>(h));
  });
  trace_end(SOMA_TRACE_GATE, st);
  return e == cudaSuccess ? SOMA_OK : SOMA_ERR_CUDA;
}

}  // extern "C"
