// scan.cu -- the gated linear recurrence: forward, backward and the one-token
// form (soma_scan_* in include/soma_api.h have the formulas).
//
// c_t = f_t c_{t-1} + u_t with u = i g.  Steps t0 .. t1 together are the map
// c -> A c + B with A the product of their f and B what they make of c = 0, so
// the time axis is cut into segments of kSegment steps: every warp turns its
// segment's gates into f and u in registers, the (A, B) of the segments are
// joined, and each warp runs its steps again from the state that reaches it.
// The gates are read once.  A warp holds 32 lanes' channels of one segment; a
// CTA's warps hold consecutive segments, a cluster's CTAs consecutive groups of
// them, and the cluster walks the sequence, its next gates on their way while
// it joins (through shared memory and distributed shared memory).  Backward is
// the same with r_t = f_t (dh_t o_t tanh'(c_t) + r_{t+1}) from the right, the
// states of a segment run again from the forward call's checkpoint.
//
// Bytes bound it: per element of 16 bits 8 read and 2 written forward, 10 read
// and 8 written backward, next to 6 (10) operations of the special function
// unit.
#define SOMA_CHECK_FILE 9
#include "checked.cuh"
#include "numeric.cuh"
#include "soma_api.h"
#include "soma_launch.h"
#include "tc_tiles.cuh"

namespace soma {

namespace {

constexpr int kSegment = 8;     // steps of a warp, and between two checkpoints
constexpr int kMaxWarps = 8;    // of a CTA
constexpr int kMaxCluster = 8;
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Minimum and maximum that pass NaN on.
__device__ __forceinline__ float min_nan(float a, float b) {
  float y;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}

// 1 + exp(-x): its reciprocal is sigmoid(x).
__device__ __forceinline__ float one_exp(float x) { return 1.f + tc::ex2(-kLog2e * x); }

// tanh(x) = num / den, a rational function of degrees 9 and 8 fitted to
// tanh(x)/x in x^2 by iteratively reweighted least squares of the relative
// error on [0, 8.7] (1.5e-8; in fp32 with the division 3.2e-7, also near 0,
// where 1 - 2/(1 + e^2x) would lose all digits).  Beyond 8.7 tanh is 1 within
// 6e-8.  The division is left to the caller, who has another one to share.
__device__ __forceinline__ void tanh_parts(float x, float& num, float& den) {
  x = min_nan(max_nan(x, -8.7f), 8.7f);
  const float s = x * x;
  num = x * fmaf(fmaf(fmaf(fmaf(0x1.dd859ep-27f, s, 0x1.60381ep-16f), s, 0x1.cd359ap-9f), s,
                      0x1.12710ep-3f), s, 1.f);
  den = fmaf(fmaf(fmaf(fmaf(0x1.ad4ff2p-21f, s, 0x1.5c82aep-12f), s, 0x1.a968bap-6f), s,
                  0x1.de8dd4p-2f), s, 1.f);
}

// sigmoid(x) and its derivative, both good relative to their size.
__device__ __forceinline__ void sigmoid_slope(float x, float& y, float& dy) {
  const float e = tc::ex2(-kLog2e * fabsf(x)), r = rcp(1.f + e);
  y = x >= 0.f ? r : e * r;
  dy = e * r * r;
}

// tanh(x) and its derivative: by e = exp(-2 |x|), which gives the derivative
// relative to its size, and below 0.3 by the Taylor series to x^9 (5e-8).
__device__ __forceinline__ void tanh_slope(float x, float& y, float& dy) {
  const float e = tc::ex2(-2.f * kLog2e * fabsf(x)), r = rcp(1.f + e);
  const float s = x * x;
  const float near = x * fmaf(fmaf(fmaf(fmaf(0x1.664f48p-6f, s, -0x1.ba1ba2p-5f), s,
                                        0x1.111112p-3f), s, -0x1.555556p-2f), s, 1.f);
  y = fabsf(x) < 0.3f ? near : copysignf((1.f - e) * r, x);
  dy = 4.f * e * r * r;
}

struct Scan {
  soma_scan_dims d;
  soma_scan_strides gs, hs, ds;
  const float* c0;
  const int32_t* lengths;
  const uint8_t* resets;
  float* c_last;
  float* marks;      // [batch][ceil(steps / kSegment)][dim]: the state before each segment
  int64_t blocks;    // blocks of 32 V channels
  int32_t cluster;   // CTAs along the time axis
};

__device__ __forceinline__ int64_t length_of(const Scan& s, int64_t b) {
  if (!s.lengths) return s.d.steps;
  const int64_t n = s.lengths[b];
  return n < 0 ? 0 : (n < s.d.steps ? n : s.d.steps);
}

// V adjacent elements as one register of bits.
template <typename T, int V>
struct Bits;
template <>
struct Bits<float, 1> {
  using type = uint32_t;
};
template <typename T>
struct Bits<T, 1> {
  using type = uint16_t;
};
template <typename T>
struct Bits<T, 2> {
  using type = uint32_t;
};

template <typename T, int V>
__device__ __forceinline__ void unpack(typename Bits<T, V>::type b, float (&x)[V]) {
  union {
    typename Bits<T, V>::type b;
    T t[V];
  } u;
  u.b = b;
#pragma unroll
  for (int v = 0; v < V; ++v) x[v] = to_f32(u.t[v]);
}

template <typename T, int V>
__device__ __forceinline__ typename Bits<T, V>::type pack(const float (&x)[V]) {
  union {
    typename Bits<T, V>::type b;
    T t[V];
  } u;
#pragma unroll
  for (int v = 0; v < V; ++v) u.t[v] = from_f32<T>(x[v]);
  return u.b;
}

// The map c -> a c + b.
template <int V>
struct Map {
  float a[V], b[V];
};

// A map applied; a = 0 forgets the state altogether, a NaN one too.
__device__ __forceinline__ float apply(float a, float b, float c) {
  return a == 0.f ? b : fmaf(a, c, b);
}

template <int V>
__device__ __forceinline__ void apply(const Map<V>& m, float (&c)[V]) {
#pragma unroll
  for (int v = 0; v < V; ++v) c[v] = apply(m.a[v], m.b[v], c[v]);
}

template <int V>
struct Joint {
  Map<V> warp[2][kMaxWarps][32];
  Map<V> cta[2][kMaxCluster][32];
};

// Joins the maps of a cluster's segments (in time order; `reverse`: from the
// last to the first).  c: in, what reaches the cluster's first (last) segment,
// the same in all its warps; out, what leaves its last (first).  `in` becomes
// what reaches this warp's.
template <int V, bool REVERSE>
__device__ __forceinline__ void join(Joint<V>& sh, const Map<V>& mine, int round, int cluster,
                                     uint32_t rank, float (&c)[V], float (&in)[V]) {
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, warps = blockDim.x / 32;
  const int buf = round & 1;
  __syncwarp();  // lanes past the last channel left the round early
  sh.warp[buf][warp][lane] = mine;
  __syncthreads();
  const auto at = [](int j, int n) { return REVERSE ? n - 1 - j : j; };
  if (cluster > 1) {
    Map<V> all = sh.warp[buf][at(0, warps)][lane];
    for (int j = 1; j < warps; ++j) {
      const Map<V> m = sh.warp[buf][at(j, warps)][lane];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        all.b[v] = apply(m.a[v], m.b[v], all.b[v]);
        all.a[v] *= m.a[v];
      }
    }
    for (int to = warp; to < cluster; to += warps) {
      uint32_t addr;
      asm("mapa.shared::cluster.u32 %0, %1, %2;"
          : "=r"(addr)
          : "r"(tc::smem_u32(&sh.cta[buf][rank][lane])), "r"(to));
#pragma unroll
      for (int v = 0; v < V; ++v) {
        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr + 4 * v), "f"(all.a[v])
                     : "memory");
        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr + 4 * (V + v)), "f"(all.b[v])
                     : "memory");
      }
    }
    tc::cluster_sync();
    for (int j = 0; j < cluster; ++j) {
      const int r = at(j, cluster);
      if (r == (int)rank) {
#pragma unroll
        for (int v = 0; v < V; ++v) in[v] = c[v];
      }
      apply(sh.cta[buf][r][lane], c);
    }
    for (int j = 0; j < warps; ++j) {
      const int w = at(j, warps);
      if (w == warp) break;
      apply(sh.warp[buf][w][lane], in);
    }
  } else {
    for (int j = 0; j < warps; ++j) {
      const int w = at(j, warps);
      if (w == warp) {
#pragma unroll
        for (int v = 0; v < V; ++v) in[v] = c[v];
      }
      apply(sh.warp[buf][w][lane], c);
    }
  }
}

// RAGGED: lengths or resets are given.
template <typename T, int V, bool RAGGED>
__global__ void __launch_bounds__(32 * kMaxWarps, 2)
scan_forward_kernel(const T* __restrict__ gates, const __grid_constant__ Scan s,
                    T* __restrict__ h) {
  using B = typename Bits<T, V>::type;
  __shared__ Joint<V> sh;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, warps = blockDim.x / 32;
  const int C = s.cluster;
  const uint32_t rank = C > 1 ? tc::pair_rank() : 0;
  const int64_t span = (int64_t)C * warps * kSegment;  // steps of the cluster's round
  const int64_t marks = (s.d.steps + kSegment - 1) / kSegment;
  int round = 0;
  for (int64_t item = blockIdx.x / C; item < s.d.batch * s.blocks; item += gridDim.x / C) {
    const int64_t b = item / s.blocks, ch = (item % s.blocks) * 32 * V + lane * V;
    const bool on = ch < s.d.dim;  // V divides dim or is 1
    const int64_t n = length_of(s, b);
    float c[V];
#pragma unroll
    for (int v = 0; v < V; ++v) c[v] = on && s.c0 ? s.c0[b * s.d.dim + ch + v] : 0.f;

    int64_t t0 = (int64_t)(rank * warps + warp) * kSegment;
    B next[kSegment][4];
    const auto fetch = [&](int64_t t) {
      const T* p = gates + b * s.gs.b + t * s.gs.t + ch;
#pragma unroll
      for (int j = 0; j < kSegment; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          next[j][k] = 0;
          if (on && t + j < n)
            next[j][k] = *reinterpret_cast<const B*>(p + j * s.gs.t + k * s.gs.g);
        }
    };
    fetch(t0);
    for (int64_t start = 0; start < s.d.steps; start += span, t0 += span, ++round) {
      float f[kSegment][V], u[kSegment][V];
      B o[kSegment];
      Map<V> m;
#pragma unroll
      for (int v = 0; v < V; ++v) m.a[v] = 1.f, m.b[v] = 0.f;
#pragma unroll
      for (int j = 0; j < kSegment; ++j) {
        float ai[V], af[V], ag[V];
        unpack<T, V>(next[j][0], ai);
        unpack<T, V>(next[j][1], af);
        unpack<T, V>(next[j][2], ag);
        o[j] = next[j][3];
        const bool live = t0 + j < n;
        bool reset = false;
        if (RAGGED && s.resets && live) reset = s.resets[b * s.d.steps + t0 + j] != 0;
#pragma unroll
        for (int v = 0; v < V; ++v) {
          float num, den;
          tanh_parts(ag[v], num, den);
          u[j][v] = num * rcp(den * one_exp(ai[v]));
          f[j][v] = rcp(one_exp(af[v]));
          if (RAGGED && reset) f[j][v] = 0.f;
          if (!live) f[j][v] = 1.f, u[j][v] = 0.f;
          m.b[v] = RAGGED ? apply(f[j][v], u[j][v], m.b[v]) : fmaf(f[j][v], m.b[v], u[j][v]);
          m.a[v] *= f[j][v];
        }
      }
      fetch(t0 + span);
      float in[V];
      join<V, false>(sh, m, round, C, rank, c, in);
      if (!on) continue;
      if (s.marks && t0 < s.d.steps) {
        float* p = s.marks + (b * marks + t0 / kSegment) * s.d.dim + ch;
#pragma unroll
        for (int v = 0; v < V; ++v) p[v] = in[v];
      }
      T* p = h + b * s.hs.b + t0 * s.hs.t + ch;
#pragma unroll
      for (int j = 0; j < kSegment; ++j) {
        float ao[V], y[V];
        unpack<T, V>(o[j], ao);
#pragma unroll
        for (int v = 0; v < V; ++v) {
          in[v] = RAGGED ? apply(f[j][v], u[j][v], in[v]) : fmaf(f[j][v], in[v], u[j][v]);
          float num, den;
          tanh_parts(in[v], num, den);
          y[v] = num * rcp(den * one_exp(ao[v]));
          if (t0 + j >= n) y[v] = 0.f;
        }
        if (t0 + j < s.d.steps) *reinterpret_cast<B*>(p + j * s.hs.t) = pack<T, V>(y);
      }
    }
    if (s.c_last && on && rank == 0 && warp == 0)
#pragma unroll
      for (int v = 0; v < V; ++v) s.c_last[b * s.d.dim + ch + v] = c[v];
  }
}

template <typename T, int V, bool RAGGED>
__global__ void __launch_bounds__(32 * kMaxWarps, 1)
scan_backward_kernel(const T* __restrict__ gates, const __grid_constant__ Scan s,
                     const T* __restrict__ dh, const float* __restrict__ dc_last,
                     T* __restrict__ dgates, float* __restrict__ dc0) {
  using B = typename Bits<T, V>::type;
  __shared__ Joint<V> sh;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, warps = blockDim.x / 32;
  const int C = s.cluster;
  const uint32_t rank = C > 1 ? tc::pair_rank() : 0;
  const int64_t span = (int64_t)C * warps * kSegment;
  const int64_t marks = (s.d.steps + kSegment - 1) / kSegment;
  int round = 0;
  for (int64_t item = blockIdx.x / C; item < s.d.batch * s.blocks; item += gridDim.x / C) {
    const int64_t b = item / s.blocks, ch = (item % s.blocks) * 32 * V + lane * V;
    const bool on = ch < s.d.dim;
    const int64_t n = length_of(s, b);
    float r[V];
#pragma unroll
    for (int v = 0; v < V; ++v) r[v] = on && dc_last ? dc_last[b * s.d.dim + ch + v] : 0.f;

    const int64_t rounds = (s.d.steps + span - 1) / span;
    int64_t t0 = (rounds - 1) * span + (int64_t)(rank * warps + warp) * kSegment;
    B next[kSegment][5];
    float mark[V];
    const auto fetch = [&](int64_t t) {
      const T* p = gates + b * s.gs.b + t * s.gs.t + ch;
      const T* q = dh + b * s.hs.b + t * s.hs.t + ch;
#pragma unroll
      for (int j = 0; j < kSegment; ++j) {
        const bool live = on && t >= 0 && t + j < n;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          next[j][k] = 0;
          if (live) next[j][k] = *reinterpret_cast<const B*>(p + j * s.gs.t + k * s.gs.g);
        }
        next[j][4] = 0;
        if (live) next[j][4] = *reinterpret_cast<const B*>(q + j * s.hs.t);
      }
#pragma unroll
      for (int v = 0; v < V; ++v)
        mark[v] = on && t >= 0 && t < n
                      ? s.marks[(b * marks + t / kSegment) * s.d.dim + ch + v] : 0.f;
    };
    fetch(t0);
    for (int64_t left = rounds; left > 0; --left, t0 -= span, ++round) {
      // what each step adds to r, its f, and the factors that turn the gradient
      // of its state into those of i, f and g
      float add[kSegment][V], f[kSegment][V], ki[kSegment][V], kf[kSegment][V], kg[kSegment][V];
      float c[V];
#pragma unroll
      for (int v = 0; v < V; ++v) c[v] = mark[v];
      T* p = dgates + b * s.ds.b + t0 * s.ds.t + ch;
#pragma unroll
      for (int j = 0; j < kSegment; ++j) {
        float ai[V], af[V], ag[V], ao[V], y[V], od[V];
        unpack<T, V>(next[j][0], ai);
        unpack<T, V>(next[j][1], af);
        unpack<T, V>(next[j][2], ag);
        unpack<T, V>(next[j][3], ao);
        unpack<T, V>(next[j][4], y);
        const bool live = t0 + j < n;
        bool reset = false;
        if (RAGGED && s.resets && live) reset = s.resets[b * s.d.steps + t0 + j] != 0;
#pragma unroll
        for (int v = 0; v < V; ++v) {
          float i, di, fg, df, g, dg, o, d_o, th, dth;
          sigmoid_slope(ai[v], i, di);
          sigmoid_slope(af[v], fg, df);
          tanh_slope(ag[v], g, dg);
          sigmoid_slope(ao[v], o, d_o);
          const float prev = RAGGED && reset ? 0.f : c[v];
          c[v] = fmaf(fg, prev, i * g);
          tanh_slope(c[v], th, dth);
          add[j][v] = live ? y[v] * o * dth : 0.f;
          f[j][v] = live ? (RAGGED && reset ? 0.f : fg) : 1.f;
          ki[j][v] = live ? g * di : 0.f;
          kf[j][v] = live ? prev * df : 0.f;
          kg[j][v] = live ? i * dg : 0.f;
          od[v] = live ? y[v] * th * d_o : 0.f;
        }
        if (on && t0 + j < s.d.steps)
          *reinterpret_cast<B*>(p + j * s.ds.t + 3 * s.ds.g) = pack<T, V>(od);
      }
      Map<V> m;
#pragma unroll
      for (int v = 0; v < V; ++v) m.a[v] = 1.f, m.b[v] = 0.f;
#pragma unroll
      for (int j = kSegment - 1; j >= 0; --j)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const float at = f[j][v] * add[j][v];
          m.b[v] = RAGGED ? apply(f[j][v], at, m.b[v]) : fmaf(f[j][v], m.b[v], at);
          m.a[v] *= f[j][v];
        }
      fetch(t0 - span);
      float in[V];
      join<V, true>(sh, m, round, C, rank, r, in);
      if (!on) continue;
#pragma unroll
      for (int j = kSegment - 1; j >= 0; --j) {
        float di[V], df[V], dg[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const float dc = add[j][v] + in[v];
          di[v] = dc * ki[j][v];
          df[v] = dc * kf[j][v];
          dg[v] = dc * kg[j][v];
          if (t0 + j >= n) di[v] = df[v] = dg[v] = 0.f;
          in[v] = RAGGED ? apply(f[j][v], 0.f, dc) : f[j][v] * dc;
        }
        if (t0 + j < s.d.steps) {
          *reinterpret_cast<B*>(p + j * s.ds.t) = pack<T, V>(di);
          *reinterpret_cast<B*>(p + j * s.ds.t + s.ds.g) = pack<T, V>(df);
          *reinterpret_cast<B*>(p + j * s.ds.t + 2 * s.ds.g) = pack<T, V>(dg);
        }
      }
    }
    if (dc0 && on && rank == 0 && warp == 0)
#pragma unroll
      for (int v = 0; v < V; ++v) dc0[b * s.d.dim + ch + v] = r[v];
  }
}

template <typename T, int V>
__global__ void __launch_bounds__(128)
scan_step_kernel(const T* __restrict__ gates, const __grid_constant__ Scan s,
                 float* __restrict__ c, T* __restrict__ h) {
  using B = typename Bits<T, V>::type;
  const int64_t at = ((int64_t)blockIdx.x * 128 + threadIdx.x) * V;
  if (at >= s.d.batch * s.d.dim) return;
  const int64_t b = at / s.d.dim, ch = at % s.d.dim;
  const T* p = gates + b * s.gs.b + ch;
  float a[4][V], x[V], y[V];
#pragma unroll
  for (int k = 0; k < 4; ++k)
    unpack<T, V>(*reinterpret_cast<const B*>(p + k * s.gs.g), a[k]);
#pragma unroll
  for (int v = 0; v < V; ++v) {
    float num, den;
    tanh_parts(a[2][v], num, den);
    x[v] = fmaf(rcp(one_exp(a[1][v])), c[at + v], num * rcp(den * one_exp(a[0][v])));
    tanh_parts(x[v], num, den);
    y[v] = num * rcp(den * one_exp(a[3][v]));
  }
#pragma unroll
  for (int v = 0; v < V; ++v) c[at + v] = x[v];
  *reinterpret_cast<B*>(h + b * s.hs.b + ch) = pack<T, V>(y);
}

// ------------------------------------------------------------------- host --

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

// Whether a 16-bit tensor can be read in pairs of channels.
bool pairs(const void* p, const soma_scan_strides& s) {
  return aligned(p, 4) && s.b % 2 == 0 && s.t % 2 == 0 && s.g % 2 == 0;
}

struct Shape {
  int warps;
  unsigned grid;
};

// Warps of a CTA cover the steps as far as they go; CTAs are put together
// along the time axis while the channels alone leave SMs without work.
Shape shape(Scan* s, int V) {
  s->blocks = (s->d.dim + 32 * V - 1) / (32 * V);
  const int64_t items = s->d.batch * s->blocks;
  Shape f;
  f.warps = 1;
  while (f.warps < kMaxWarps && f.warps * kSegment < s->d.steps) f.warps *= 2;
  s->cluster = 1;
  while (s->cluster < kMaxCluster && items * s->cluster < 2 * 152 &&
         (int64_t)s->cluster * f.warps * kSegment < s->d.steps)
    s->cluster *= 2;
  const int64_t most = 1 << 20;
  f.grid = (unsigned)((items < most ? items : most) * s->cluster);
  return f;
}

template <typename K, typename... A>
cudaError_t launch(K kernel, const Shape& f, int cluster, cudaStream_t st, A... args) {
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = (unsigned)cluster;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(f.grid);
  cfg.blockDim = dim3(32u * f.warps);
  cfg.stream = st;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <typename T, int V>
cudaError_t forward(const void* gates, Scan s, void* h, cudaStream_t st) {
  const Shape f = shape(&s, V);
  const bool ragged = s.lengths || s.resets;
  return launch(ragged ? scan_forward_kernel<T, V, true> : scan_forward_kernel<T, V, false>, f,
                s.cluster, st, static_cast<const T*>(gates), s, static_cast<T*>(h));
}

template <typename T, int V>
cudaError_t backward(const void* gates, Scan s, const void* dh, const float* dc_last,
                     void* dgates, float* dc0, cudaStream_t st) {
  const Shape f = shape(&s, V);
  const bool ragged = s.lengths || s.resets;
  return launch(ragged ? scan_backward_kernel<T, V, true> : scan_backward_kernel<T, V, false>, f,
                s.cluster, st, static_cast<const T*>(gates), s, static_cast<const T*>(dh), dc_last,
                static_cast<T*>(dgates), dc0);
}

template <typename T, int V>
cudaError_t step(const void* gates, const Scan& s, float* c, void* h, cudaStream_t st) {
  const int64_t threads = s.d.batch * s.d.dim / V;
  scan_step_kernel<T, V><<<(unsigned)((threads + 127) / 128), 128, 0, st>>>(
      static_cast<const T*>(gates), s, c, static_cast<T*>(h));
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
  h_strides.g = 0;
  const Scan s = {d,       gate_strides, h_strides, {0, 0, 0},   c0,
                  lengths, resets,       c_last,    checkpoints, 0, 1};
  const cudaStream_t st = (cudaStream_t)stream;
  const bool two = d.dim % 2 == 0 && pairs(gates, gate_strides) && pairs(h, h_strides);
  trace_begin(SOMA_TRACE_GATE, st);
  cudaError_t e;
  if (dtype == SOMA_FP32) e = forward<float, 1>(gates, s, h, st);
  else if (dtype == SOMA_BF16)
    e = two ? forward<__nv_bfloat16, 2>(gates, s, h, st) : forward<__nv_bfloat16, 1>(gates, s, h, st);
  else
    e = two ? forward<__half, 2>(gates, s, h, st) : forward<__half, 1>(gates, s, h, st);
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
  dh_strides.g = 0;
  const Scan s = {d,       gate_strides, dh_strides, dgate_strides,
                  nullptr, lengths,      resets,     nullptr,
                  const_cast<float*>(checkpoints), 0, 1};
  const cudaStream_t st = (cudaStream_t)stream;
  const bool two = d.dim % 2 == 0 && pairs(gates, gate_strides) && pairs(dh, dh_strides) &&
                   pairs(dgates, dgate_strides);
  trace_begin(SOMA_TRACE_GATE, st);
  cudaError_t e;
  if (dtype == SOMA_FP32) e = backward<float, 1>(gates, s, dh, dc_last, dgates, dc0, st);
  else if (dtype == SOMA_BF16)
    e = two ? backward<__nv_bfloat16, 2>(gates, s, dh, dc_last, dgates, dc0, st)
            : backward<__nv_bfloat16, 1>(gates, s, dh, dc_last, dgates, dc0, st);
  else
    e = two ? backward<__half, 2>(gates, s, dh, dc_last, dgates, dc0, st)
            : backward<__half, 1>(gates, s, dh, dc_last, dgates, dc0, st);
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
  gate_strides.t = h_strides.t = h_strides.g = 0;
  const Scan s = {d,       gate_strides, h_strides, {0, 0, 0}, nullptr,
                  nullptr, nullptr,      nullptr,   nullptr,   0, 1};
  const cudaStream_t st = (cudaStream_t)stream;
  const bool two = dim % 2 == 0 && pairs(gates, gate_strides) && pairs(h, h_strides);
  trace_begin(SOMA_TRACE_GATE, st);
  cudaError_t e;
  if (dtype == SOMA_FP32) e = step<float, 1>(gates, s, c, h, st);
  else if (dtype == SOMA_BF16)
    e = two ? step<__nv_bfloat16, 2>(gates, s, c, h, st) : step<__nv_bfloat16, 1>(gates, s, c, h, st);
  else
    e = two ? step<__half, 2>(gates, s, c, h, st) : step<__half, 1>(gates, s, c, h, st);
  trace_end(SOMA_TRACE_GATE, st);
  return e == cudaSuccess ? SOMA_OK : SOMA_ERR_CUDA;
}

}  // extern "C"
