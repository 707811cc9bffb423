// scan.cu -- the gated linear recurrence: forward, backward and the one-token
// form (soma_scan_* in include/soma_api.h have the formulas).
//
// c_t = f_t c_{t-1} + u_t with u = i g.  Steps t0 .. t1 together are the map
// c -> A c + B with A the product of their f and B what they make of c = 0, so
// the time axis is cut into segments of kSegment steps: every warp turns its
// segment's gates into f and u in registers, the (A, B) of the segments are
// joined, and each warp runs its steps again from the state that reaches it.
// The gates are read once.  A CTA's warps hold consecutive segments, a
// cluster's CTAs consecutive groups of them, and the cluster walks the
// sequence, joining through shared memory and distributed shared memory.
// Backward is the same with r_t = f_t (dh_t o_t tanh'(c_t) + r_{t+1}) from the
// right, the states of a segment run again from the forward call's checkpoint.
//
// Tiled kernels: a lane holds two channels in packed fp32 arithmetic, the gates
// come as TMA boxes into a ring of shared-memory stages.  Plain kernels: one
// channel per lane and loads of single elements, for tensors that a tensor map
// cannot describe.
//
// Bytes bound it: per element of 16 bits 8 read and 2 written forward, 10 read
// and 8 written backward.  The instructions come close: 113 per element (one
// channel at a time, a 64-bit address and a bounds check per load) took 2.7
// times the bytes' time.
#include <cmath>
#include <initializer_list>

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

// Two fp32 values for the packed instructions.
struct Two {
  float2 v;
};
__device__ __forceinline__ Two two(float a, float b) { return {make_float2(a, b)}; }
__device__ __forceinline__ Two two(float a) { return two(a, a); }
__device__ __forceinline__ void split(Two x, float& a, float& b) {
  a = x.v.x;
  b = x.v.y;
}
__device__ __forceinline__ Two operator*(Two a, Two b) { return {__fmul2_rn(a.v, b.v)}; }
__device__ __forceinline__ Two operator+(Two a, Two b) { return {__fadd2_rn(a.v, b.v)}; }
__device__ __forceinline__ Two fma2(Two a, Two b, Two c) { return {__ffma2_rn(a.v, b.v, c.v)}; }
template <typename F>
__device__ __forceinline__ Two each(Two x, F f) {
  float a, b;
  split(x, a, b);
  return two(f(a), f(b));
}
__device__ __forceinline__ Two rcp2(Two x) {
  return each(x, [](float y) { return rcp(y); });
}
__device__ __forceinline__ Two ex22(Two x) {
  return each(x, [](float y) { return tc::ex2(y); });
}
__device__ __forceinline__ Two one_exp2(Two x) { return ex22(x * two(-kLog2e)) + two(1.f); }
__device__ __forceinline__ void tanh_parts2(Two x, Two& num, Two& den) {
  x = each(x, [](float y) { return min_nan(max_nan(y, -8.7f), 8.7f); });
  const Two s = x * x;
  num = x * fma2(fma2(fma2(fma2(two(0x1.dd859ep-27f), s, two(0x1.60381ep-16f)), s,
                           two(0x1.cd359ap-9f)), s, two(0x1.12710ep-3f)), s, two(1.f));
  den = fma2(fma2(fma2(fma2(two(0x1.ad4ff2p-21f), s, two(0x1.5c82aep-12f)), s,
                       two(0x1.a968bap-6f)), s, two(0x1.de8dd4p-2f)), s, two(1.f));
}
// sigmoid and y (1 - y): the derivative good to 1 u of 1.
__device__ __forceinline__ void sigmoid_slope2(Two x, Two& y, Two& dy) {
  y = rcp2(one_exp2(x));
  dy = fma2(y * two(-1.f), y, y);
}
// tanh by e = exp(-2 |x|), which gives the derivative 4 e / (1 + e)^2 good
// relative to its size, and below 0.1 by the Taylor series to x^5 (6e-8).
__device__ __forceinline__ void tanh_slope2(Two x, Two& y, Two& dy) {
  const Two e = each(x, [](float z) { return tc::ex2(-2.f * kLog2e * fabsf(z)); });
  const Two r = rcp2(e + two(1.f));
  const Two s = x * x;
  const Two near = x * fma2(fma2(two(0x1.111112p-3f), s, two(-0x1.555556p-2f)), s, two(1.f));
  const Two far = fma2(e, two(-1.f), two(1.f)) * r;
  float x0, x1, n0, n1, f0, f1;
  split(x, x0, x1);
  split(near, n0, n1);
  split(far, f0, f1);
  y = two(fabsf(x0) < 0.1f ? n0 : copysignf(f0, x0), fabsf(x1) < 0.1f ? n1 : copysignf(f1, x1));
  dy = (e * two(4.f)) * (r * r);
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
  int32_t depth;     // stages of the ring
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
struct __align__(8 * V) Map {
  float a[V], b[V];
};

// A map applied; a = 0 forgets the state altogether, a NaN one too.
__device__ __forceinline__ float apply(float a, float b, float c) {
  return a == 0.f ? b : fmaf(a, c, b);
}

template <bool RAGGED, int V>
__device__ __forceinline__ void apply(const Map<V>& m, float (&c)[V]) {
#pragma unroll
  for (int v = 0; v < V; ++v)
    c[v] = RAGGED ? apply(m.a[v], m.b[v], c[v]) : fmaf(m.a[v], c[v], m.b[v]);
}

// Where the maps are exchanged: [2][warps][32] of this CTA, and in clusters
// [2][CTAs][32] that every CTA writes into all of them.
template <int V>
struct Joint {
  Map<V>* warp;
  Map<V>* cta;
};

template <int V>
__host__ __device__ constexpr size_t joint_bytes(int warps, int cluster) {
  return sizeof(Map<V>) * 64 * (warps + (cluster > 1 ? cluster : 0));
}

template <int V>
__device__ __forceinline__ Joint<V> joint_at(void* p, int warps) {
  Map<V>* const m = static_cast<Map<V>*>(p);
  return {m, m + 64 * warps};
}

// Joins the maps of a cluster's segments (in time order; REVERSE: from the
// last to the first).  c: in, what reaches the cluster's first (last) segment,
// the same in all its warps; out, what leaves its last (first).  `in` becomes
// what reaches this warp's.
template <bool REVERSE, bool RAGGED, int WARPS, int V>
__device__ __forceinline__ void join(const Joint<V>& sh, const Map<V>& mine, int round,
                                     int cluster, uint32_t rank, float (&c)[V], float (&in)[V]) {
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, warps = blockDim.x / 32;
  Map<V>* const of_warp = sh.warp + (round & 1) * warps * 32 + lane;
  Map<V>* const of_cta = sh.cta + (round & 1) * cluster * 32 + lane;
  __syncwarp();  // lanes past the last channel left the round early
  of_warp[warp * 32] = mine;
  __syncthreads();
  const auto at = [](int j, int n) { return REVERSE ? n - 1 - j : j; };
  if (cluster > 1) {
    if (warp < cluster) {
      Map<V> all = of_warp[at(0, warps) * 32];
#pragma unroll
      for (int j = 1; j < WARPS; ++j) {
        if (j >= warps) break;
        const Map<V> m = of_warp[at(j, warps) * 32];
        apply<RAGGED>(m, all.b);
#pragma unroll
        for (int v = 0; v < V; ++v) all.a[v] *= m.a[v];
      }
      for (int to = warp; to < cluster; to += warps) {
        uint32_t addr;
        asm("mapa.shared::cluster.u32 %0, %1, %2;"
            : "=r"(addr)
            : "r"(tc::smem_u32(of_cta + rank * 32)), "r"(to));
        if (V == 2)
          asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(addr),
                       "f"(all.a[0]), "f"(all.a[V - 1]), "f"(all.b[0]), "f"(all.b[V - 1])
                       : "memory");
        else
          asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(addr), "f"(all.a[0]),
                       "f"(all.b[0])
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
      apply<RAGGED>(of_cta[r * 32], c);
    }
#pragma unroll
    for (int j = 0; j < WARPS - 1; ++j) {
      const int w = at(j, warps);
      if (j >= warps || w == warp) break;
      apply<RAGGED>(of_warp[w * 32], in);
    }
  } else {
#pragma unroll
    for (int j = 0; j < WARPS; ++j) {
      const int w = at(j, warps);
      if (j >= warps) break;
      if (w == warp) {
#pragma unroll
        for (int v = 0; v < V; ++v) in[v] = c[v];
      }
      apply<RAGGED>(of_warp[w * 32], c);
    }
  }
}

// RAGGED: lengths or resets are given.
template <typename T, int V, bool RAGGED>
__global__ void __launch_bounds__(32 * kMaxWarps, 2)
scan_forward_kernel(const T* __restrict__ gates, const __grid_constant__ Scan s,
                    T* __restrict__ h) {
  using B = typename Bits<T, V>::type;
  extern __shared__ __align__(16) uint8_t raw[];
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, warps = blockDim.x / 32;
  const int C = s.cluster;
  const uint32_t rank = C > 1 ? tc::pair_rank() : 0;
  const Joint<V> sh = joint_at<V>(raw, warps);
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
      join<false, RAGGED, kMaxWarps>(sh, m, round, C, rank, c, in);
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
  extern __shared__ __align__(16) uint8_t raw[];
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, warps = blockDim.x / 32;
  const int C = s.cluster;
  const uint32_t rank = C > 1 ? tc::pair_rank() : 0;
  const Joint<V> sh = joint_at<V>(raw, warps);
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
      join<true, RAGGED, kMaxWarps>(sh, m, round, C, rank, r, in);
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

// ---- tiled ----------------------------------------------------------------
constexpr int kBlock = 64;  // channels of a CTA: 32 lanes of two
// Stages of the ring: one is read to the end of its round (forward) or being
// stored (backward), so one less is in flight.  A call whose CTAs have an SM to
// themselves takes more of them, as nothing else covers a copy's latency.
constexpr int kMaxDepth = 4;
// CTAs of so many warps that an SM's registers hold.
constexpr int forward_resident(int warps) { return 20 / warps; }
constexpr int backward_resident(int warps) { return 12 / warps; }

// The tensors of a call as boxes of 64 channels by the CTA's steps: one map
// per gate, then dh.
struct Maps {
  CUtensorMap in[5], out[4];
  int32_t t_inner;  // whether steps are the second dimension of the maps, sequences the third
};

__device__ __forceinline__ void box_g2s(void* dst, const CUtensorMap* map, int x, int y, int z,
                                        uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(tc::smem_u32(dst)),
      "l"(map), "r"(x), "r"(y), "r"(z), "r"(tc::smem_u32(bar))
      : "memory");
}
__device__ __forceinline__ void box_s2g(const CUtensorMap* map, int x, int y, int z,
                                        const void* src) {
  asm volatile(
      "cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(
          map),
      "r"(x), "r"(y), "r"(z), "r"(tc::smem_u32(src))
      : "memory");
}

// A lane's two channels in shared memory.
__device__ __forceinline__ Two load_two(const float* p) {
  const float2 x = *reinterpret_cast<const float2*>(p);
  return two(x.x, x.y);
}
__device__ __forceinline__ Two load_two(const __nv_bfloat16* p) {
  const uint32_t x = *reinterpret_cast<const uint32_t*>(p);
  return two(__uint_as_float(x << 16), __uint_as_float(x & 0xFFFF0000u));
}
__device__ __forceinline__ Two load_two(const __half* p) {
  const float2 x = __half22float2(*reinterpret_cast<const __half2*>(p));
  return two(x.x, x.y);
}
__device__ __forceinline__ void store_two(float* p, Two x) {
  float a, b;
  split(x, a, b);
  *reinterpret_cast<float2*>(p) = make_float2(a, b);
}
__device__ __forceinline__ void store_two(__nv_bfloat16* p, Two x) {
  float a, b;
  split(x, a, b);
  *reinterpret_cast<__nv_bfloat162*>(p) = __floats2bfloat162_rn(a, b);
}
__device__ __forceinline__ void store_two(__half* p, Two x) {
  float a, b;
  split(x, a, b);
  *reinterpret_cast<__half2*>(p) = __floats2half2_rn(a, b);
}

__device__ __forceinline__ Two apply2(Two a, Two b, Two c) {
  float a0, a1, b0, b1, c0, c1;
  split(a, a0, a1);
  split(b, b0, b1);
  split(c, c0, c1);
  return two(apply(a0, b0, c0), apply(a1, b1, c1));
}

struct Ring {
  uint64_t full[kMaxDepth];
  volatile int abort;
};

__device__ __forceinline__ void ring_wait(Ring& r, int stage, uint32_t parity, int* status) {
  if (r.abort || tc::mbar_wait(&r.full[stage], parity)) return;
  r.abort = 1;
  atomicCAS(status, 0, SOMA_ERR_TIMEOUT);
}

// RAGGED: lengths or resets are given.  h is written directly: a row of a
// warp's store is 128 bytes.
template <typename T, bool RAGGED, int WARPS>
__global__ void __launch_bounds__(32 * WARPS, forward_resident(WARPS))
scan_forward_tiled_kernel(const __grid_constant__ Maps maps, const __grid_constant__ Scan s,
                          T* __restrict__ h, int* status) {
  extern __shared__ uint8_t raw[];
  const int depth = s.depth;
  __shared__ Ring ring;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, warps = blockDim.x / 32;
  const int C = s.cluster;
  const uint32_t rank = C > 1 ? tc::pair_rank() : 0;
  const int rows = warps * kSegment;                // steps of the CTA's round
  const int64_t span = (int64_t)C * rows;           // ... of the cluster's
  const int64_t marks = (s.d.steps + kSegment - 1) / kSegment;
  const int stage_elems = 4 * rows * kBlock;
  T* const stages = reinterpret_cast<T*>(raw + (128 - (tc::smem_u32(raw) & 127)) % 128);
  const Joint<2> sh = joint_at<2>(stages + (size_t)depth * stage_elems, warps);
  if (threadIdx.x == 0) {
    for (int i = 0; i < depth; ++i) tc::mbar_init(&ring.full[i], 1);
    tc::mbar_fence_init();
    ring.abort = 0;
  }
  __syncthreads();
  int filled = 0, st = 0;          // the next stage to fill, and to use
  uint32_t parity = 0, turn = 0;
  for (int64_t item = blockIdx.x / C; item < s.d.batch * s.blocks; item += gridDim.x / C) {
    const int64_t b = item / s.blocks;
    const int ch0 = (int)(item % s.blocks) * kBlock;
    const int64_t ch = ch0 + 2 * lane;
    const bool on = ch < s.d.dim;
    const int64_t n = length_of(s, b);
    const int64_t rounds = (n + span - 1) / span;
    if (item >= gridDim.x / C) __syncthreads();  // the last item's stages have been read
    float c[2] = {0.f, 0.f};
    if (on && s.c0) c[0] = s.c0[b * s.d.dim + ch], c[1] = s.c0[b * s.d.dim + ch + 1];

    const auto fill = [&](int64_t round) {  // warp 0
      const int st = filled;
      filled = filled + 1 == depth ? 0 : filled + 1;
      if (lane == 0) tc::mbar_arrive_expect_tx(&ring.full[st], stage_elems * sizeof(T));
      __syncwarp();
      if (lane < 4) {
        const int t = (int)(round * span) + (int)rank * rows;
        box_g2s(stages + (size_t)st * stage_elems + lane * rows * kBlock, &maps.in[lane], ch0,
                maps.t_inner ? t : (int)b, maps.t_inner ? (int)b : t, &ring.full[st]);
      }
    };
    // one stage less in flight than there are: the newest is read to the end of
    // its round
    if (warp == 0)
      for (int64_t q = 0; q < depth - 1 && q < rounds; ++q) fill(q);

    int64_t t0 = (int64_t)(rank * warps + warp) * kSegment;
    for (int64_t round = 0; round < rounds; ++round, t0 += span) {
      ring_wait(ring, st, parity, status);
      const T* p = stages + (size_t)st * stage_elems + warp * kSegment * kBlock + 2 * lane;
      const int gate = rows * kBlock;
      Two f[kSegment], u[kSegment];
      Two A = two(1.f), B = two(0.f);
      // steps of this segment that exist: nearly always all of them, and the
      // whole warp takes the branch without their checks
      const int live = n - t0 >= kSegment ? kSegment : n > t0 ? (int)(n - t0) : 0;
#pragma unroll
      for (int j = 0; j < kSegment; ++j) {
        const Two ai = load_two(p + j * kBlock), af = load_two(p + gate + j * kBlock);
        const Two ag = load_two(p + 2 * gate + j * kBlock);
        Two num, den;
        tanh_parts2(ag, num, den);
        u[j] = num * rcp2(den * one_exp2(ai));
        f[j] = rcp2(one_exp2(af));
      }
      if (RAGGED && s.resets) {
#pragma unroll
        for (int j = 0; j < kSegment; ++j)
          if (j < live && s.resets[b * s.d.steps + t0 + j]) f[j] = two(0.f);
      }
      if (live < kSegment) {
#pragma unroll
        for (int j = 0; j < kSegment; ++j)
          if (j >= live) f[j] = two(1.f), u[j] = two(0.f);
      }
#pragma unroll
      for (int j = 0; j < kSegment; ++j) {
        B = RAGGED ? apply2(f[j], u[j], B) : fma2(f[j], B, u[j]);
        A = A * f[j];
      }
      Map<2> m;
      split(A, m.a[0], m.a[1]);
      split(B, m.b[0], m.b[1]);
      float in[2];
      join<false, RAGGED, WARPS>(sh, m, (int)(turn & 1), C, rank, c, in);
      // every warp is through with the stage of the round before
      if (warp == 0 && round + depth - 1 < rounds) fill(round + depth - 1);
      if (on) {
        if (s.marks && t0 < s.d.steps)
          *reinterpret_cast<float2*>(s.marks + (b * marks + t0 / kSegment) * s.d.dim + ch) =
              make_float2(in[0], in[1]);
        T* q = h + b * s.hs.b + t0 * s.hs.t + ch;
        Two x = two(in[0], in[1]);
#pragma unroll
        for (int j = 0; j < kSegment; ++j) {
          x = RAGGED ? apply2(f[j], u[j], x) : fma2(f[j], x, u[j]);
          Two num, den;
          tanh_parts2(x, num, den);
          const Two y = num * rcp2(den * one_exp2(load_two(p + 3 * gate + j * kBlock)));
          if (live == kSegment) store_two(q, y);
          else if (t0 + j < s.d.steps) store_two(q, j < live ? y : two(0.f));
          q += s.hs.t;
        }
      }
      __syncwarp();
      if (++st == depth) st = 0, parity ^= 1;
      ++turn;
    }
    // rounds past the sequence's end
    if (RAGGED && on)
      for (; t0 < s.d.steps; t0 += span)
        for (int j = 0; j < kSegment && t0 + j < s.d.steps; ++j)
          store_two(h + b * s.hs.b + (t0 + j) * s.hs.t + ch, two(0.f));
    __syncwarp();
    if (s.c_last && on && rank == 0 && warp == 0)
      s.c_last[b * s.d.dim + ch] = c[0], s.c_last[b * s.d.dim + ch + 1] = c[1];
  }
}

// The gradients of the gates take their places in the stage and are stored
// from there as boxes.
template <typename T, bool RAGGED, int WARPS>
__global__ void __launch_bounds__(32 * WARPS, backward_resident(WARPS))
scan_backward_tiled_kernel(const __grid_constant__ Maps maps, const __grid_constant__ Scan s,
                           const float* __restrict__ dc_last, float* __restrict__ dc0,
                           int* status) {
  extern __shared__ uint8_t raw[];
  const int depth = s.depth;
  __shared__ Ring ring;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, warps = blockDim.x / 32;
  const int C = s.cluster;
  const uint32_t rank = C > 1 ? tc::pair_rank() : 0;
  const int rows = warps * kSegment;
  const int64_t span = (int64_t)C * rows;
  const int64_t marks = (s.d.steps + kSegment - 1) / kSegment;
  const int stage_elems = 5 * rows * kBlock;
  T* const stages = reinterpret_cast<T*>(raw + (128 - (tc::smem_u32(raw) & 127)) % 128);
  const Joint<2> sh = joint_at<2>(stages + (size_t)depth * stage_elems, warps);
  if (threadIdx.x == 0) {
    for (int i = 0; i < depth; ++i) tc::mbar_init(&ring.full[i], 1);
    tc::mbar_fence_init();
    ring.abort = 0;
  }
  __syncthreads();
  int filled = 0, st = 0;
  uint32_t parity = 0, turn = 0;
  for (int64_t item = blockIdx.x / C; item < s.d.batch * s.blocks; item += gridDim.x / C) {
    const int64_t b = item / s.blocks;
    const int ch0 = (int)(item % s.blocks) * kBlock;
    const int64_t ch = ch0 + 2 * lane;
    const bool on = ch < s.d.dim;
    const int64_t n = length_of(s, b);
    const int64_t rounds = (s.d.steps + span - 1) / span;  // the last ones may be past the end
    float r[2] = {0.f, 0.f};
    if (on && dc_last) r[0] = dc_last[b * s.d.dim + ch], r[1] = dc_last[b * s.d.dim + ch + 1];

    // warp 0; of the stores that this thread has made, the newest may still read
    // its stage: the stage filled here is an older one, except at an item's start
    const auto fill = [&](int64_t round, bool start) {
      const int st = filled;
      filled = filled + 1 == depth ? 0 : filled + 1;
      if (lane == 0) {
        if (start) tc::bulk_wait_read();
        else asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
        tc::mbar_arrive_expect_tx(&ring.full[st], stage_elems * sizeof(T));
      }
      __syncwarp();
      if (lane < 5) {
        const int t = (int)(round * span) + (int)rank * rows;
        box_g2s(stages + (size_t)st * stage_elems + lane * rows * kBlock, &maps.in[lane], ch0,
                maps.t_inner ? t : (int)b, maps.t_inner ? (int)b : t, &ring.full[st]);
      }
    };
    // one stage less in flight than there are: the newest is being stored
    if (warp == 0)
      for (int64_t q = 0; q < depth - 1 && q < rounds; ++q) fill(rounds - 1 - q, true);

    const auto mark_at = [&](int64_t t) {
      float2 x = make_float2(0.f, 0.f);
      if (on && t >= 0 && t < n)
        x = *reinterpret_cast<const float2*>(s.marks + (b * marks + t / kSegment) * s.d.dim + ch);
      return two(x.x, x.y);
    };
    int64_t t0 = (rounds - 1) * span + (int64_t)(rank * warps + warp) * kSegment;
    Two next_mark = mark_at(t0);
    for (int64_t round = rounds - 1; round >= 0; --round, t0 -= span) {
      const Two mark = next_mark;
      next_mark = mark_at(t0 - span);
      ring_wait(ring, st, parity, status);
      T* p = stages + (size_t)st * stage_elems + warp * kSegment * kBlock + 2 * lane;
      const int gate = rows * kBlock;
      // what each step adds to r, its f, and the factors that turn the gradient
      // of its state into those of i, f and g
      Two add[kSegment], f[kSegment], ki[kSegment], kf[kSegment], kg[kSegment];
      Two c = mark;
      const int live = n - t0 >= kSegment ? kSegment : n > t0 ? (int)(n - t0) : 0;
#pragma unroll
      for (int j = 0; j < kSegment; ++j) {
        const Two ai = load_two(p + j * kBlock), af = load_two(p + gate + j * kBlock);
        const Two ag = load_two(p + 2 * gate + j * kBlock);
        const Two ao = load_two(p + 3 * gate + j * kBlock);
        const Two y = load_two(p + 4 * gate + j * kBlock);
        Two i, di, fg, df, g, dg, o, d_o, th, dth;
        sigmoid_slope2(ai, i, di);
        sigmoid_slope2(af, fg, df);
        tanh_slope2(ag, g, dg);
        sigmoid_slope2(ao, o, d_o);
        const bool reset =
            RAGGED && s.resets && j < live && s.resets[b * s.d.steps + t0 + j] != 0;
        const Two prev = reset ? two(0.f) : c;
        c = fma2(fg, prev, i * g);
        tanh_slope2(c, th, dth);
        add[j] = y * o * dth;
        f[j] = reset ? two(0.f) : fg;
        ki[j] = g * di;
        kf[j] = prev * df;
        kg[j] = i * dg;
        store_two(p + 3 * gate + j * kBlock, y * th * d_o);
      }
      if (live < kSegment) {
#pragma unroll
        for (int j = 0; j < kSegment; ++j)
          if (j >= live) {
            add[j] = ki[j] = kf[j] = kg[j] = two(0.f);
            f[j] = two(1.f);
            store_two(p + 3 * gate + j * kBlock, two(0.f));
          }
      }
      Two A = two(1.f), B = two(0.f);
#pragma unroll
      for (int j = kSegment - 1; j >= 0; --j) {
        B = RAGGED ? apply2(f[j], f[j] * add[j], B) : f[j] * (add[j] + B);
        A = A * f[j];
      }
      Map<2> m;
      split(A, m.a[0], m.a[1]);
      split(B, m.b[0], m.b[1]);
      float in[2];
      join<true, RAGGED, WARPS>(sh, m, (int)(turn & 1), C, rank, r, in);
      Two x = two(in[0], in[1]);
#pragma unroll
      for (int j = kSegment - 1; j >= 0; --j) {
        const Two dc = add[j] + x;
        store_two(p + j * kBlock, dc * ki[j]);
        store_two(p + gate + j * kBlock, dc * kf[j]);
        store_two(p + 2 * gate + j * kBlock, dc * kg[j]);
        x = RAGGED ? apply2(f[j], two(0.f), dc) : f[j] * dc;
      }
      if (live < kSegment) {  // an infinite dc times 0 is no gradient
#pragma unroll
        for (int j = 0; j < kSegment; ++j)
          if (j >= live)
            for (int k = 0; k < 3; ++k) store_two(p + k * gate + j * kBlock, two(0.f));
      }
      tc::fence_async_smem();
      __syncthreads();
      if (warp == 0) {
        if (lane == 0) {
          const int t = (int)(round * span) + (int)rank * rows;
          if (t < s.d.steps) {
            for (int k = 0; k < 4; ++k)
              box_s2g(&maps.out[k], ch0, maps.t_inner ? t : (int)b, maps.t_inner ? (int)b : t,
                      stages + (size_t)st * stage_elems + k * gate);
          }
          tc::bulk_commit();
        }
        __syncwarp();
        if (round >= depth - 1) fill(round - (depth - 1), false);
      }
      if (++st == depth) st = 0, parity ^= 1;
      ++turn;
    }
    if (dc0 && on && rank == 0 && warp == 0)
      dc0[b * s.d.dim + ch] = r[0], dc0[b * s.d.dim + ch + 1] = r[1];
    __syncwarp();
  }
  if (threadIdx.x == 0) tc::bulk_wait();
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
  int warps, most;  // of a CTA, and of the kernel compiled for it
  unsigned grid;
  bool alone;       // no SM has two CTAs
};

// How the work is cut: CTAs of up to `most` warps (resident[k] of `most >> k`
// fit an SM) along the steps, and CTAs of a cluster.  All CTAs of a call
// together on the GPU finish soonest: 704 items (32 x 2048 x 1376) in CTAs of
// eight warps are 2.3 waves of 304 and took three (222 us forward), in CTAs of
// four they are one of 760.  What is left is the SM with the most CTAs, too
// few warps to fill an SM, and the price of a cluster's barrier (clusters of
// eight of the same work, 18.5 waves: 290 us).
Shape shape(Scan* s, int V, int most, std::initializer_list<int> resident) {
  s->blocks = (s->d.dim + 32 * V - 1) / (32 * V);
  const int64_t items = s->d.batch * s->blocks;
  Shape best = {1, 1, 1, false};
  double least = 1e300;
  for (const int fit : resident) {
    int warps = 1;
    while (warps < most && warps * kSegment < s->d.steps) warps *= 2;
    for (int c = 1; c <= kMaxCluster; c *= 2) {
      if (c > 1 && (int64_t)c / 2 * warps * kSegment >= s->d.steps) break;
      const double n = (double)items * c, slots = 152.0 * fit;
      const double waves = n > slots ? std::ceil(n / slots) * slots / n
                                     : std::ceil(n / 152) * 152 / n;
      const double held = (n < slots ? n : slots) * warps / 152;
      const double cost = waves * (held < 10 ? 10 / held : 1) * (c > 1 ? 1.4 : 1);
      if (cost < least * 0.98) {
        least = cost;
        best.warps = warps;
        best.most = most;
        s->cluster = c;
      }
    }
    most /= 2;
  }
  const int64_t cap = 1 << 20;
  best.grid = (unsigned)((items < cap ? items : cap) * s->cluster);
  best.alone = best.grid <= 152;
  return best;
}

template <typename K, typename... A>
cudaError_t launch(K kernel, const Shape& f, int cluster, size_t smem, cudaStream_t st, A... args) {
  cudaError_t e =
      cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = (unsigned)cluster;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(f.grid);
  cfg.blockDim = dim3(32u * f.warps);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// A [batch][steps][dim] tensor as a tensor map: its steps inside the sequences
// (t_inner) or the other way round.
struct Layout3 {
  int64_t size[3], stride[2];
};

bool layout(const soma_scan_dims& d, const soma_scan_strides& s, bool t_inner, int dtype,
            Layout3* l) {
  const int64_t unit = dtype == SOMA_FP32 ? 4 : 8;  // elements of 16 bytes
  const int64_t n1 = t_inner ? d.steps : d.batch, n2 = t_inner ? d.batch : d.steps;
  int64_t s1 = t_inner ? s.t : s.b, s2 = t_inner ? s.b : s.t;
  if (n1 == 1) s1 = (d.dim + unit - 1) / unit * unit;  // never stepped over
  if (n2 == 1) s2 = n1 * s1;
  *l = {{d.dim, n1, n2}, {s1, s2}};
  return s1 % unit == 0 && s2 % unit == 0 && s1 >= d.dim && s2 >= n1 * s1 && s2 % s1 == 0 &&
         s1 < ((int64_t)1 << 37) && s2 < ((int64_t)1 << 37);
}

bool mappable(const void* p, const soma_scan_dims& d, const soma_scan_strides& s, bool gates,
              bool t_inner, int dtype) {
  const int64_t unit = dtype == SOMA_FP32 ? 4 : 8;
  Layout3 l;
  return aligned(p, 16) && (!gates || s.g % unit == 0) && layout(d, s, t_inner, dtype, &l);
}

// Maps of one tensor's gates (or of the tensor itself), boxes of 64 channels
// by `rows` steps of one sequence.
bool map_all(CUtensorMap* maps, int count, const void* p, const soma_scan_dims& d,
             const soma_scan_strides& s, bool t_inner, int dtype, int rows) {
  Layout3 l;
  if (!layout(d, s, t_inner, dtype, &l)) return false;
  const int box[3] = {kBlock, t_inner ? rows : 1, t_inner ? 1 : rows};
  for (int k = 0; k < count; ++k)
    if (!make_box_map(&maps[k], static_cast<const uint8_t*>(p) + k * s.g * (int64_t)width(dtype),
                      dtype, l.size, l.stride, box))
      return false;
  return true;
}

template <typename T>
constexpr int dtype_of() {
  return std::is_same<T, float>::value ? SOMA_FP32
         : std::is_same<T, __half>::value ? SOMA_FP16 : SOMA_BF16;
}

template <typename T>
size_t tiled_bytes(int depth, int boxes, int warps, int cluster) {
  return (size_t)depth * boxes * warps * kSegment * kBlock * sizeof(T) + 128 +
         joint_bytes<2>(warps, cluster);
}

template <typename T>
cudaError_t forward(const void* gates, Scan s, void* h, int* status, cudaStream_t st) {
  constexpr int dtype = dtype_of<T>();
  const bool ragged = s.lengths || s.resets;
  // h and the checkpoints are written two channels at a time
  const bool direct = s.d.dim % 2 == 0 && aligned(h, 2 * sizeof(T)) && s.hs.b % 2 == 0 &&
                      s.hs.t % 2 == 0 && aligned(s.marks, 8);
  for (const bool t_inner : {true, false}) {
    if (s.d.steps < 1 || !direct || !mappable(gates, s.d, s.gs, true, t_inner, dtype)) continue;
    // eight warps' stages of fp32 fit an SM only once
    const Shape f = sizeof(T) == 4 ? shape(&s, 2, 4, {3, 5}) : shape(&s, 2, 8, {2, 5});
    Maps maps;
    maps.t_inner = t_inner;
    if (!map_all(maps.in, 4, gates, s.d, s.gs, t_inner, dtype, f.warps * kSegment))
      return cudaErrorInvalidValue;
    const auto kernel = f.most == 8   ? ragged ? scan_forward_tiled_kernel<T, true, 8>
                                               : scan_forward_tiled_kernel<T, false, 8>
                        : f.most == 4 ? ragged ? scan_forward_tiled_kernel<T, true, 4>
                                               : scan_forward_tiled_kernel<T, false, 4>
                                      : ragged ? scan_forward_tiled_kernel<T, true, 2>
                                               : scan_forward_tiled_kernel<T, false, 2>;
    s.depth = f.alone ? 4 : 2;
    return launch(kernel, f, s.cluster, tiled_bytes<T>(s.depth, 4, f.warps, s.cluster), st, maps, s,
                  static_cast<T*>(h), status);
  }
  const Shape f = shape(&s, 1, kMaxWarps, {2});
  return launch(ragged ? scan_forward_kernel<T, 1, true> : scan_forward_kernel<T, 1, false>, f,
                s.cluster, joint_bytes<1>(f.warps, s.cluster), st, static_cast<const T*>(gates), s,
                static_cast<T*>(h));
}

template <typename T>
cudaError_t backward(const void* gates, Scan s, const void* dh, const float* dc_last,
                     void* dgates, float* dc0, int* status, cudaStream_t st) {
  constexpr int dtype = dtype_of<T>();
  const bool ragged = s.lengths || s.resets;
  for (const bool t_inner : {true, false}) {
    if (s.d.steps < 1 || s.d.dim % 2 || !aligned(s.marks, 8) ||
        !mappable(gates, s.d, s.gs, true, t_inner, dtype) ||
        !mappable(dh, s.d, s.hs, false, t_inner, dtype) ||
        !mappable(dgates, s.d, s.ds, true, t_inner, dtype))
      continue;
    const Shape f = sizeof(T) == 4 ? shape(&s, 2, 2, {3, 6}) : shape(&s, 2, 4, {3, 6});
    const int rows = f.warps * kSegment;
    Maps maps;
    maps.t_inner = t_inner;
    if (!map_all(maps.in, 4, gates, s.d, s.gs, t_inner, dtype, rows) ||
        !map_all(maps.in + 4, 1, dh, s.d, s.hs, t_inner, dtype, rows) ||
        !map_all(maps.out, 4, dgates, s.d, s.ds, t_inner, dtype, rows))
      return cudaErrorInvalidValue;
    const auto kernel = f.most == 4   ? ragged ? scan_backward_tiled_kernel<T, true, 4>
                                               : scan_backward_tiled_kernel<T, false, 4>
                        : f.most == 2 ? ragged ? scan_backward_tiled_kernel<T, true, 2>
                                               : scan_backward_tiled_kernel<T, false, 2>
                                      : ragged ? scan_backward_tiled_kernel<T, true, 1>
                                               : scan_backward_tiled_kernel<T, false, 1>;
    s.depth = f.alone ? 4 : 3;
    return launch(kernel, f, s.cluster, tiled_bytes<T>(s.depth, 5, f.warps, s.cluster), st, maps, s,
                  dc_last, dc0, status);
  }
  const Shape f = shape(&s, 1, kMaxWarps, {1});
  return launch(ragged ? scan_backward_kernel<T, 1, true> : scan_backward_kernel<T, 1, false>, f,
                s.cluster, joint_bytes<1>(f.warps, s.cluster), st, static_cast<const T*>(gates), s, static_cast<const T*>(dh),
                dc_last, static_cast<T*>(dgates), dc0);
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
                  lengths, resets,       c_last,    checkpoints, 0, 1, 2};
  const cudaStream_t st = (cudaStream_t)stream;
  int* status = status_ptr();
  if (!status) return SOMA_ERR_CUDA;
  trace_begin(SOMA_TRACE_GATE, st);
  const cudaError_t e = dtype == SOMA_FP32   ? forward<float>(gates, s, h, status, st)
                        : dtype == SOMA_BF16 ? forward<__nv_bfloat16>(gates, s, h, status, st)
                                             : forward<__half>(gates, s, h, status, st);
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
                  const_cast<float*>(checkpoints), 0, 1, 2};
  const cudaStream_t st = (cudaStream_t)stream;
  int* status = status_ptr();
  if (!status) return SOMA_ERR_CUDA;
  trace_begin(SOMA_TRACE_GATE, st);
  const cudaError_t e =
      dtype == SOMA_FP32   ? backward<float>(gates, s, dh, dc_last, dgates, dc0, status, st)
      : dtype == SOMA_BF16 ? backward<__nv_bfloat16>(gates, s, dh, dc_last, dgates, dc0, status, st)
                           : backward<__half>(gates, s, dh, dc_last, dgates, dc0, status, st);
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
                  nullptr, nullptr,      nullptr,   nullptr,   0, 1, 2};
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
