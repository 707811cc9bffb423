// linear_attn.cu -- linear attention with a decay for each head: the entry
// points, the kernels of fp32 arithmetic and the one-token form
// (soma_linear_attn_* in include/soma_api.h have the formulas).
#include <cmath>

#define SOMA_CHECK_FILE 14
#include "checked.cuh"
#include "linear_attn.cuh"
#include "numeric.cuh"
#include "pdl.cuh"

namespace soma {
namespace attn {

namespace {

constexpr int kTile = 16;       // steps that are staged at once
constexpr int kRows = 16;       // rows of the state that a thread holds, in four runs of four
constexpr int kCols = 4;        // and columns
constexpr int kStepThreads = 256;

// exp(g) by fp32 numbers that have it as their mean: `up` is due `share` / 2^32 of
// the steps, `low` in the others.  The nearest fp32 number would be off by up to
// 2^-25 every time in the same direction, 3e-5 after a thousand steps.
struct Decay {
  float low, up;
  uint32_t share;
  __device__ __forceinline__ float at(int64_t step) const {
    return (uint32_t)(step + 1) * share < share ? up : low;
  }
};
__device__ Decay split_decay(float g) {
  const double l = exp((double)g);
  Decay d;
  d.low = __double2float_rd(l);
  d.up = __double2float_ru(l);
  d.share = d.up > d.low ? (uint32_t)((l - d.low) / ((double)d.up - d.low) * 4294967295.0) : 0;
  return d;
}

// The recurrence step by step in fp32: one CTA per problem, sequence and head,
// the state in registers, 16 x 4 of it per thread.  Threads of `groups`
// neighbouring lanes hold the rows of the same columns.
template <typename T>
__global__ void __launch_bounds__(256)
plain_kernel(const __grid_constant__ Call call, int groups) {
  extern __shared__ __align__(16) float smem[];
  admit_successor();
  after_predecessor();
  const int64_t rows_all = call.batch * call.heads;
  const Problem& p = call.p[blockIdx.x / rows_all];
  const int64_t bh = blockIdx.x % rows_all, b = bh / call.heads, h = bh % call.heads;
  const int64_t len = length_of(call, b);
  __shared__ Decay decay;
  if (threadIdx.x == 0) decay = split_decay(decay_of(call, h));
  const int rows = groups * kRows, cols = (p.c + kCols - 1) / kCols * kCols;
  float* sx = smem;
  float* sy = sx + kTile * rows;
  float* sz = sy + kTile * rows;
  float* sm = sz + kTile * cols;
  const int group = threadIdx.x % groups, c0 = threadIdx.x / groups * kCols;
  const bool holds = c0 < cols;
  const T* x = static_cast<const T*>(p.x) + b * p.xs.b + h * p.xs.h;
  const T* y = static_cast<const T*>(p.y) + b * p.ys.b + h * p.ys.h;
  const T* z = static_cast<const T*>(p.z) + b * p.zs.b + h * p.zs.h;
  T* out = static_cast<T*>(p.out) + b * p.os.b + h * p.os.h;
  const uint8_t* resets = call.resets ? call.resets + b * call.steps : nullptr;

  // row of register r: runs of four, `groups` runs apart
  const auto row_of = [&](int r) { return (r / 4 * groups + group) * 4 + r % 4; };
  float S[kRows][kCols];
#pragma unroll
  for (int r = 0; r < kRows; ++r)
#pragma unroll
    for (int j = 0; j < kCols; ++j) {
      const int i = row_of(r), c = c0 + j;
      S[r][j] = p.s_in && i < p.a && c < p.c
                    ? p.s_in[bh * call.state + i * p.in_row + c * p.in_col]
                    : 0.f;
    }

  for (int64_t n0 = 0; n0 < len; n0 += kTile) {
    const int n = len - n0 < kTile ? (int)(len - n0) : kTile;
    const auto step_of = [&](int k) { return p.reversed ? len - 1 - n0 - k : n0 + k; };
    __syncthreads();
    for (int e = threadIdx.x; e < n * rows; e += blockDim.x) {
      const int k = e / rows, i = e % rows;
      const int64_t t = step_of(k);
      sx[e] = i < p.a ? to_f32(x[t * p.xs.t + i]) : 0.f;
      sy[e] = i < p.a ? to_f32(y[t * p.ys.t + i]) : 0.f;
    }
    for (int e = threadIdx.x; e < n * cols; e += blockDim.x) {
      const int k = e / cols, i = e % cols;
      sz[e] = i < p.c ? p.f * to_f32(z[step_of(k) * p.zs.t + i]) : 0.f;
    }
    if ((int)threadIdx.x < n) {
      const int64_t t = step_of(threadIdx.x);
      float m = decay.at(n0 + threadIdx.x);
      if (p.reversed) {
        if (t == len - 1) m = 1.f;
        else if (resets && resets[t + 1]) m = 0.f;
      } else if (resets && resets[t]) {
        m = 0.f;
      }
      sm[threadIdx.x] = m;
    }
    __syncthreads();
    for (int k = 0; k < n; ++k) {
      const float m = sm[k];
      float o[kCols] = {0.f, 0.f, 0.f, 0.f};
      if (holds) {
        const float4 v4 = *reinterpret_cast<const float4*>(sz + k * cols + c0);
        const float v[kCols] = {v4.x, v4.y, v4.z, v4.w};
        if (m == 0.f) {  // nothing passes, whatever it is
#pragma unroll
          for (int r = 0; r < kRows; ++r)
#pragma unroll
            for (int j = 0; j < kCols; ++j) S[r][j] = 0.f;
        }
#pragma unroll
        for (int q = 0; q < kRows / 4; ++q) {
          const int at = k * rows + (q * groups + group) * 4;
          const float4 y4 = *reinterpret_cast<const float4*>(sy + at);
          const float4 x4 = *reinterpret_cast<const float4*>(sx + at);
          const float yr[4] = {y4.x, y4.y, y4.z, y4.w}, xr[4] = {x4.x, x4.y, x4.z, x4.w};
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < kCols; ++j) {
              float& s = S[4 * q + r][j];
              s = fmaf(m, s, yr[r] * v[j]);
              o[j] = fmaf(xr[r], s, o[j]);
            }
        }
      }
      for (int s = 1; s < groups; s <<= 1)
#pragma unroll
        for (int j = 0; j < kCols; ++j) o[j] += __shfl_xor_sync(0xffffffffu, o[j], s);
      if (holds) {
        T* to = out + step_of(k) * p.os.t + c0;
#pragma unroll
        for (int j = 0; j < kCols; ++j)
          if (j % groups == group && c0 + j < p.c) to[j] = from_f32<T>(p.g * o[j]);
      }
    }
  }
  // past the end
  for (int64_t e = len * p.c + threadIdx.x; e < call.steps * p.c; e += blockDim.x)
    out[e / p.c * p.os.t + e % p.c] = from_f32<T>(0.f);
  if (!p.s_out || !holds) return;
  const float last = !p.reversed || len == 0 ? 1.f : resets && resets[0] ? 0.f : decay.at(len);
#pragma unroll
  for (int r = 0; r < kRows; ++r)
#pragma unroll
    for (int j = 0; j < kCols; ++j) {
      const int i = row_of(r), c = c0 + j;
      if (i < p.a && c < p.c)
        p.s_out[bh * call.state + i * p.out_row + c * p.out_col] =
            last == 0.f ? 0.f : last * S[r][j];
    }
}

// One token: a CTA per sequence and head, V adjacent columns per thread, the rows
// dealt out to `lanes` threads of the same columns.  The state's bytes bound it.
template <typename T, int V>
__global__ void __launch_bounds__(kStepThreads)
step_kernel(const __grid_constant__ Call call, int lanes) {
  __shared__ float sx[128], sy[128];
  __shared__ float part[kStepThreads * V];
  admit_successor();
  after_predecessor();
  const Problem& p = call.p[0];
  const int64_t bh = blockIdx.x, b = bh / call.heads, h = bh % call.heads;
  const int columns = p.c / V, col = threadIdx.x % columns * V, first = threadIdx.x / columns;
  float* s = p.s_out + bh * call.state;
  constexpr int kAhead = 4;
  // the state's first rows are on their way while x and y are staged
  float v[kAhead][V];
  const auto fetch = [&](int i) {
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (i + k * lanes < p.a) {
        const float* at = s + (i + k * lanes) * p.c + col;
        if (V == 4) {
          const float4 w = *reinterpret_cast<const float4*>(at);
          v[k][0] = w.x; v[k][V - 3] = w.y; v[k][V - 2] = w.z; v[k][V - 1] = w.w;
        } else {
          v[k][0] = *at;
        }
      }
  };
  if (first < lanes) fetch(first);
  const T* x = static_cast<const T*>(p.x) + b * p.xs.b + h * p.xs.h;
  const T* y = static_cast<const T*>(p.y) + b * p.ys.b + h * p.ys.h;
  const T* z = static_cast<const T*>(p.z) + b * p.zs.b + h * p.zs.h;
  for (int i = threadIdx.x; i < p.a; i += kStepThreads) {
    sx[i] = to_f32(x[i]);
    sy[i] = to_f32(y[i]);
  }
  // exp(g) as a sum whose error is 2^-24 of 1 - exp(g), not of exp(g): over the
  // steps that a state lasts it stays 2^-24
  const float g = decay_of(call, h);
  const bool slow = g > -0.5f;
  const float keep = slow ? 1.f : expf(g), change = slow ? expm1f(g) : 0.f;
  float zc[V], o[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    zc[j] = first < lanes ? to_f32(z[col + j]) : 0.f;
    o[j] = 0.f;
  }
  __syncthreads();
  if (first < lanes) {
    for (int i = first; i < p.a; i += kAhead * lanes) {
      if (i != first) fetch(i);
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int r = i + k * lanes;
        if (r >= p.a) break;
#pragma unroll
        for (int j = 0; j < V; ++j) {
          // a decay of 0 keeps nothing, whatever it is
          const float new_part = sy[r] * zc[j];
          v[k][j] = keep == 0.f ? new_part : fmaf(keep, v[k][j], fmaf(change, v[k][j], new_part));
          o[j] = fmaf(sx[r], v[k][j], o[j]);
        }
        float* at = s + r * p.c + col;
        if (V == 4)
          *reinterpret_cast<float4*>(at) = make_float4(v[k][0], v[k][V - 3], v[k][V - 2], v[k][V - 1]);
        else
          *at = v[k][0];
      }
    }
#pragma unroll
    for (int j = 0; j < V; ++j) part[first * p.c + col + j] = o[j];
  }
  __syncthreads();
  T* out = static_cast<T*>(p.out) + b * p.os.b + h * p.os.h;
  for (int c = threadIdx.x; c < p.c; c += kStepThreads) {
    float t = 0.f;
    for (int k = 0; k < lanes; ++k) t += part[k * p.c + c];
    out[c] = from_f32<T>(p.g * t);
  }
}

// ------------------------------------------------------------------- host --

bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

bool dims_ok(const soma_attn_dims& d) {
  return d.batch >= 0 && d.steps >= 0 && d.heads >= 0 && d.batch <= INT32_MAX &&
         d.steps <= INT32_MAX && d.heads <= (1 << 16) &&
         (d.heads == 0 || d.batch <= (1 << 29) / d.heads) && d.key_dim >= 1 && d.key_dim <= 128 &&
         d.value_dim >= 1 && d.value_dim <= 128;
}

bool dtype_ok(int t) { return t == SOMA_FP32 || t == SOMA_BF16 || t == SOMA_FP16; }

size_t width(int dtype) { return dtype == SOMA_FP32 ? 4 : 2; }

bool tensor_ok(const void* p, const soma_attn_strides& s, int dtype) {
  return aligned(p, width(dtype)) && s.b >= 0 && s.t >= 0 && s.h >= 0;
}

bool overlap(const float* p, const float* q, int64_t count) {
  if (!p || !q) return false;
  const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
  return (a < b ? b - a : a - b) < (uintptr_t)count * sizeof(float);
}

template <typename T>
cudaError_t plain(const Call& call, cudaStream_t st) {
  int widest = 0, wide_c = 0;
  for (int k = 0; k < call.problems; ++k) {
    if (call.p[k].a > widest) widest = call.p[k].a;
    if (call.p[k].c > wide_c) wide_c = call.p[k].c;
  }
  int groups = 1;
  while (groups * kRows < widest) groups *= 2;
  const int cols = (wide_c + kCols - 1) / kCols * kCols;
  const int threads = (groups * (cols / kCols) + 31) / 32 * 32;
  const size_t smem = sizeof(float) * (kTile * (2 * groups * kRows + cols) + kTile);
  return launch_overlapped(plain_kernel<T>, dim3((unsigned)(call.problems * call.batch * call.heads)),
                           threads, smem, st, call, groups);
}

template <typename T>
cudaError_t step(const Call& call, cudaStream_t st) {
  const Problem& p = call.p[0];
  const dim3 grid((unsigned)(call.batch * call.heads));
  if (p.c % 4 == 0 && aligned(p.s_out, 16))
    return launch_overlapped(step_kernel<T, 4>, grid, kStepThreads, 0, st, call,
                             kStepThreads / (p.c / 4));
  return launch_overlapped(step_kernel<T, 1>, grid, kStepThreads, 0, st, call, kStepThreads / p.c);
}

// Whether the tensor-core kernels can read and write a tensor.
bool tiled(const void* p, const soma_attn_strides& s) {
  return aligned(p, 16) && s.b % 8 == 0 && s.t % 8 == 0 && s.h % 8 == 0;
}

// The cut with the least estimated time, in chunks of one CTA: states of all
// segments but the last first (half the work of a chunk), then the outputs.
Cut cut_of(const soma_attn_dims& d, int dtype, int problems) {
  Cut best = {};
  best.segments = 1;
  best.chunks = (d.steps + kChunk - 1) / kChunk;
  if (dtype == SOMA_FP32 || d.key_dim % 8 || d.value_dim % 8) return best;
  const int64_t rows = d.batch * d.heads * problems, chunks = best.chunks;
  const int64_t resident = d.key_dim <= 64 && d.value_dim <= 64 ? 304 : 152;
  const auto waves = [&](int64_t n) { return (double)((n + resident - 1) / resident); };
  double least = waves(rows) * (chunks + 2);
  for (int64_t n = 2; n <= chunks && n <= 1024; ++n) {
    const int64_t each = (chunks + n - 1) / n;
    if ((chunks + each - 1) / each != n) continue;
    const double cost =
        waves(rows * n) * (each + 2) + waves(rows * (n - 1)) * (0.5 * each + 2) + 4;
    if (cost < least) {
      least = cost;
      best.segments = (int32_t)n;
      best.chunks = each;
    }
  }
  return best;
}

// Where a cut's parts lie in the workspace, with the checked build's gaps.
struct Parts {
  size_t starts, fades, bytes;
  Gaps gaps;
};
Parts parts_of(const soma_attn_dims& d, const Cut& cut, int problems) {
  Parts p = {};
  if (cut.segments < 2) return p;
  const size_t n = (size_t)(d.batch * d.heads) * problems * cut.segments;
  p.starts = kGuard;
  p.fades = p.starts + (n * d.key_dim * d.value_dim * sizeof(float) + 15) / 16 * 16 + kGuard;
  p.bytes = p.fades + (n * sizeof(float2) + 15) / 16 * 16 + kGuard;
  p.gaps.n = 3;
  p.gaps.off[0] = 0;
  p.gaps.off[1] = p.fades - kGuard;
  p.gaps.off[2] = p.bytes - kGuard;
  return p;
}

cudaError_t run(const Call& call, const Cut& cut, int dtype, cudaStream_t st) {
  bool chunked = dtype != SOMA_FP32 && call.steps > 0;
  for (int k = 0; k < call.problems; ++k) {
    const Problem& p = call.p[k];
    chunked = chunked && p.a % 8 == 0 && p.c % 8 == 0 && tiled(p.x, p.xs) && tiled(p.y, p.ys) &&
              tiled(p.z, p.zs) && tiled(p.out, p.os);
  }
  cudaError_t e;
  if (chunked && launch_chunks(call, cut, dtype, st, &e)) return e;
  return dtype == SOMA_FP32   ? plain<float>(call, st)
         : dtype == SOMA_BF16 ? plain<__nv_bfloat16>(call, st)
                              : plain<__half>(call, st);
}

Call make_call(const soma_attn_dims& d, const float* log_decay, const int32_t* lengths,
               const uint8_t* resets, int* status) {
  Call c = {};
  c.heads = (int32_t)d.heads;
  c.batch = d.batch;
  c.steps = d.steps;
  c.state = (int64_t)d.key_dim * d.value_dim;
  c.log_decay = log_decay;
  c.lengths = lengths;
  c.resets = resets;
  c.status = status;
  return c;
}

void put_workspace(Cut* cut, const Parts& parts, void* workspace) {
  if (!parts.bytes) return;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  cut->starts = reinterpret_cast<float*>(ws + parts.starts);
  cut->fades = reinterpret_cast<float2*>(ws + parts.fades);
}

int traced(const Call& call, const Cut& cut, const Parts& parts, int dtype, void* workspace,
           cudaStream_t st) {
  if (parts.bytes && gaps_fill(parts.gaps, workspace, st) != cudaSuccess) return SOMA_ERR_CUDA;
  trace_begin(SOMA_TRACE_LINEAR_ATTN, st);
  cudaError_t e = run(call, cut, dtype, st);
  trace_end(SOMA_TRACE_LINEAR_ATTN, st);
  if (parts.bytes && e == cudaSuccess) e = gaps_check(parts.gaps, workspace, call.status, st);
  return e == cudaSuccess ? SOMA_OK : SOMA_ERR_CUDA;
}

// States are [key_dim][value_dim]; `turned`: the problem's rows are its columns.
void put_states(Problem* p, const soma_attn_dims& d, bool turned, const float* in, float* out) {
  p->s_in = in;
  p->s_out = out;
  p->in_row = p->out_row = turned ? 1 : d.value_dim;
  p->in_col = p->out_col = turned ? d.value_dim : 1;
}

}  // namespace
}  // namespace attn
}  // namespace soma

using namespace soma;
using namespace soma::attn;

extern "C" {

int64_t soma_linear_attn_workspace_bytes(soma_attn_dims d, int dtype, int backward) {
  if (!dims_ok(d) || !dtype_ok(dtype) || (backward != 0 && backward != 1)) return -1;
  const int problems = backward ? 3 : 1;
  return (int64_t)parts_of(d, cut_of(d, dtype, problems), problems).bytes;
}

int soma_linear_attn_forward(const void* q, soma_attn_strides q_strides, const void* k,
                             soma_attn_strides k_strides, const void* v,
                             soma_attn_strides v_strides, int dtype, soma_attn_dims d,
                             const float* log_decay, float scale, const float* s0,
                             const int32_t* lengths, const uint8_t* resets, void* o,
                             soma_attn_strides o_strides, float* s_last, void* workspace,
                             size_t workspace_bytes, void* stream) {
  if (!dims_ok(d)) return SOMA_ERR_UNSUPPORTED;
  if (!dtype_ok(dtype) || !tensor_ok(q, q_strides, dtype) || !tensor_ok(k, k_strides, dtype) ||
      !tensor_ok(v, v_strides, dtype) || !tensor_ok(o, o_strides, dtype) ||
      !std::isfinite(scale) || !aligned(log_decay, 4) || !aligned(s0, 4) || !aligned(lengths, 4) ||
      !aligned(s_last, 4))
    return SOMA_ERR_INVALID_ARG;
  if (d.batch == 0 || d.heads == 0) return SOMA_OK;
  if (!log_decay || (d.steps > 0 && (!q || !k || !v || !o))) return SOMA_ERR_INVALID_ARG;
  if (overlap(s0, s_last, d.batch * d.heads * d.key_dim * d.value_dim)) return SOMA_ERR_INVALID_ARG;
  Cut cut = cut_of(d, dtype, 1);
  const Parts parts = parts_of(d, cut, 1);
  if (parts.bytes && (!workspace || !aligned(workspace, 16) || workspace_bytes < parts.bytes))
    return SOMA_ERR_WORKSPACE;
  put_workspace(&cut, parts, workspace);
  int* status = status_ptr();
  if (!status) return SOMA_ERR_CUDA;
  Call call = make_call(d, log_decay, lengths, resets, status);
  call.problems = 1;
  Problem& p = call.p[0];
  p = {q, k, v, o, q_strides, k_strides, v_strides, o_strides, d.key_dim, d.value_dim};
  p.f = 1.f;
  p.g = scale;
  put_states(&p, d, false, s0, s_last);
  return traced(call, cut, parts, dtype, workspace, (cudaStream_t)stream);
}

int soma_linear_attn_backward(const void* q, soma_attn_strides q_strides, const void* k,
                              soma_attn_strides k_strides, const void* v,
                              soma_attn_strides v_strides, int dtype, soma_attn_dims d,
                              const float* log_decay, float scale, const float* s0,
                              const int32_t* lengths, const uint8_t* resets, const void* d_out,
                              soma_attn_strides do_strides, const float* ds_last, void* dq,
                              soma_attn_strides dq_strides, void* dk,
                              soma_attn_strides dk_strides, void* dv,
                              soma_attn_strides dv_strides, float* ds0, void* workspace,
                              size_t workspace_bytes, void* stream) {
  if (!dims_ok(d)) return SOMA_ERR_UNSUPPORTED;
  if (!dtype_ok(dtype) || !tensor_ok(q, q_strides, dtype) || !tensor_ok(k, k_strides, dtype) ||
      !tensor_ok(v, v_strides, dtype) || !tensor_ok(d_out, do_strides, dtype) ||
      !tensor_ok(dq, dq_strides, dtype) || !tensor_ok(dk, dk_strides, dtype) ||
      !tensor_ok(dv, dv_strides, dtype) || !std::isfinite(scale) || !aligned(log_decay, 4) ||
      !aligned(s0, 4) || !aligned(lengths, 4) || !aligned(ds_last, 4) || !aligned(ds0, 4))
    return SOMA_ERR_INVALID_ARG;
  if (d.batch == 0 || d.heads == 0) return SOMA_OK;
  if (!log_decay || (d.steps > 0 && (!q || !k || !v || !d_out || !dq || !dk || !dv)))
    return SOMA_ERR_INVALID_ARG;
  const int64_t states = d.batch * d.heads * d.key_dim * d.value_dim;
  if (overlap(s0, ds0, states) || overlap(ds_last, ds0, states)) return SOMA_ERR_INVALID_ARG;
  Cut cut = cut_of(d, dtype, 3);
  const Parts parts = parts_of(d, cut, 3);
  if (parts.bytes && (!workspace || !aligned(workspace, 16) || workspace_bytes < parts.bytes))
    return SOMA_ERR_WORKSPACE;
  put_workspace(&cut, parts, workspace);
  int* status = status_ptr();
  if (!status) return SOMA_ERR_CUDA;
  Call call = make_call(d, log_decay, lengths, resets, status);
  call.problems = 3;
  Problem &pq = call.p[0], &pk = call.p[1], &pv = call.p[2];
  pq = {d_out, v, k, dq, do_strides, v_strides, k_strides, dq_strides, d.value_dim, d.key_dim};
  pk = {v, d_out, q, dk, v_strides, do_strides, q_strides, dk_strides, d.value_dim, d.key_dim};
  pv = {k, q, d_out, dv, k_strides, q_strides, do_strides, dv_strides, d.key_dim, d.value_dim};
  pq.f = pk.g = pv.g = 1.f;
  pq.g = pk.f = pv.f = scale;
  pk.reversed = pv.reversed = 1;
  put_states(&pq, d, true, s0, nullptr);
  put_states(&pk, d, true, ds_last, nullptr);
  put_states(&pv, d, false, ds_last, ds0);
  return traced(call, cut, parts, dtype, workspace, (cudaStream_t)stream);
}

int soma_linear_attn_step(const void* q, soma_attn_strides q_strides, const void* k,
                          soma_attn_strides k_strides, const void* v,
                          soma_attn_strides v_strides, int dtype, soma_attn_dims d,
                          const float* log_decay, float scale, float* s, void* o,
                          soma_attn_strides o_strides, void* stream) {
  if (!dims_ok(d)) return SOMA_ERR_UNSUPPORTED;
  if (!dtype_ok(dtype) || !tensor_ok(q, q_strides, dtype) || !tensor_ok(k, k_strides, dtype) ||
      !tensor_ok(v, v_strides, dtype) || !tensor_ok(o, o_strides, dtype) ||
      !std::isfinite(scale) || !aligned(log_decay, 4) || !aligned(s, 4))
    return SOMA_ERR_INVALID_ARG;
  if (d.batch == 0 || d.heads == 0) return SOMA_OK;
  if (!log_decay || !q || !k || !v || !o || !s) return SOMA_ERR_INVALID_ARG;
  int* status = status_ptr();
  if (!status) return SOMA_ERR_CUDA;
  Call call = make_call(d, log_decay, nullptr, nullptr, status);
  call.problems = 1;
  Problem& p = call.p[0];
  p = {q, k, v, o, q_strides, k_strides, v_strides, o_strides, d.key_dim, d.value_dim};
  p.f = 1.f;
  p.g = scale;
  put_states(&p, d, false, s, s);
  const cudaStream_t st = (cudaStream_t)stream;
  trace_begin(SOMA_TRACE_LINEAR_ATTN, st);
  const cudaError_t e = dtype == SOMA_FP32   ? step<float>(call, st)
                        : dtype == SOMA_BF16 ? step<__nv_bfloat16>(call, st)
                                             : step<__half>(call, st);
  trace_end(SOMA_TRACE_LINEAR_ATTN, st);
  return e == cudaSuccess ? SOMA_OK : SOMA_ERR_CUDA;
}

}  // extern "C"
