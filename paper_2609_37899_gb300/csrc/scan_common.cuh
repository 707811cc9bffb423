// scan_common.cuh -- what the kernels of the gated linear recurrence share
// (scan_forward.cu, scan_backward.cu; soma_scan_* in include/soma_api.h have
// the formulas).
//
// c_t = f_t c_{t-1} + u_t with u = i g.  Steps t0 .. t1 together are the map
// c -> A c + B with A the product of their f and B what they make of c = 0, so
// the time axis can be cut: every warp turns the gates of a segment of kSegment
// steps into f and u in registers, a CTA's warps hold consecutive segments and
// join their (A, B) through shared memory, and each warp runs its steps again
// from the state that reaches it.  The CTA walks the steps so, a round at a
// time, and the gates are read once.  Backward is the same with
// r_t = f_t (dh_t o_t tanh'(c_t) + r_{t+1}) from the right, the states of a
// segment run again from the forward call's checkpoint.
//
// Where the channels alone do not occupy the GPU, the steps are cut into
// chunks as well: one launch forms the chunks' maps (it reads what the maps
// need and writes nothing else), and in the next each CTA applies the maps of
// the chunks before its own to the state that enters and runs its chunk.  The
// first of the two goes through a chunk the other way round: what it read last
// is what the second wants first, and still in L2.
//
// Tiled kernels: a lane holds two channels in packed fp32 arithmetic, the gates
// come as TMA boxes into a ring of shared-memory stages.  Plain kernels: one
// channel per lane and loads of single elements, for tensors that a tensor map
// cannot describe.
#pragma once

#include <cmath>
#include <cstring>
#include <type_traits>

#include "numeric.cuh"
#include "pdl.cuh"
#include "soma_api.h"
#include "soma_launch.h"
#include "tc_tiles.cuh"

namespace soma {
namespace scan {

constexpr int kSegment = 8;  // steps of a warp, and between two checkpoints
constexpr int kBlock = 64;   // channels of a tiled CTA: 32 lanes of two
constexpr int kSms = 152;
constexpr float kLog2e = 1.4426950408889634f;

// The special function unit's reciprocal and power of two: within an ulp or two
// of the rounded ones.  h, the states and the gradients are allowed 32 half
// ulps of their terms per step for all of it.
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

// Forget gates, and products of them, are never taken as less than this, the
// least fp32 number: 0 times a state that is infinite would be NaN, and which
// products underflow depends on how the steps are cut.  Of a finite state it
// leaves less than 2^-21 (2^-49 of one up to 2^100).  So 0 stands for a reset
// alone.
constexpr float kLeast = 0x1p-149f;
__device__ __forceinline__ float open(float f) { return max_nan(f, kLeast); }

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
// sigmoid and its derivative e / (1 + e)^2 with e = exp(-x), both good relative
// to their size on either side: y - y^2 would be good to half an ulp of 1 only,
// and a saturated gate's is far below.  e stays finite (0 times infinity); the
// reciprocal of 2^127 is flushed to 0.
__device__ __forceinline__ void sigmoid_slope2(Two x, Two& y, Two& dy) {
  const Two e = each(x * two(-kLog2e), [](float z) { return tc::ex2(min_nan(z, 127.f)); });
  y = rcp2(e + two(1.f));
  dy = (e * y) * y;
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

__device__ __forceinline__ Two open2(Two f) {
  return each(f, [](float x) { return open(x); });
}

struct Scan {
  soma_scan_dims d;
  soma_scan_strides gs, hs, ds;
  const float* c0;
  const int32_t* lengths;
  const uint8_t* resets;
  float* c_last;
  float* marks;      // [batch][ceil(steps / kSegment)][dim]: the state before each segment
  int64_t blocks;    // blocks of a CTA's channels
  int64_t chunks;    // of the steps, `chunk` steps each
  int64_t chunk;
  float2* maps;      // [batch][chunks][dim]: (A, B) of the chunks
  int* status;
  int32_t depth;     // stages of the ring (tiled)
};

__device__ __forceinline__ int64_t length_of(const Scan& s, int64_t b) {
  if (!s.lengths) return s.d.steps;
  const int64_t n = s.lengths[b];
  return n < 0 ? 0 : (n < s.d.steps ? n : s.d.steps);
}

// What the checked build asks of an access: steps [t, t + n) of sequence b,
// channels [ch, ch + v).
__device__ __forceinline__ bool inside(const Scan& s, int64_t b, int64_t t, int64_t n, int64_t ch,
                                       int v) {
  return b >= 0 && b < s.d.batch && t >= 0 && t + n <= s.d.steps && ch >= 0 && ch + v <= s.d.dim;
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

// A map applied; a = 0 forgets the state altogether, a NaN one too (resets).
// So a map with a reset among its steps has a = 0, whatever the product of its
// other gates is (NaN * 0 is not): a document that is not finite ends with it.
// Without one a is at least kLeast, also where a gate is NaN: b is NaN then.
__device__ __forceinline__ float apply(float a, float b, float c) {
  return a == 0.f ? b : fmaf(a, c, b);
}

template <bool RAGGED, int V>
__device__ __forceinline__ void apply(const Map<V>& m, float (&c)[V]) {
#pragma unroll
  for (int v = 0; v < V; ++v)
    c[v] = RAGGED ? apply(m.a[v], m.b[v], c[v]) : fmaf(m.a[v], c[v], m.b[v]);
}

// `later` after `m`.
template <bool RAGGED, int V>
__device__ __forceinline__ void follow(Map<V>& m, const Map<V>& later) {
  apply<RAGGED>(later, m.b);
#pragma unroll
  for (int v = 0; v < V; ++v)
    m.a[v] = RAGGED && (m.a[v] == 0.f || later.a[v] == 0.f)
                 ? 0.f : fmaxf(m.a[v] * later.a[v], kLeast);
}

template <int V>
__device__ __forceinline__ Map<V> identity() {
  Map<V> m;
#pragma unroll
  for (int v = 0; v < V; ++v) m.a[v] = 1.f, m.b[v] = 0.f;
  return m;
}

// Joins the maps of a CTA's warps (in time order; REVERSE: from the last to the
// first).  shared: [2][warps][32], used alternately.  c: in, what reaches the
// first (last) warp, the same in all of them; out, what leaves the last
// (first).  `in` becomes what reaches this warp.
template <bool REVERSE, bool RAGGED, int WARPS, int V>
__device__ __forceinline__ void join(Map<V>* shared, const Map<V>& mine, uint32_t turn,
                                     float (&c)[V], float (&in)[V]) {
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, warps = blockDim.x / 32;
  Map<V>* const of_warp = shared + (turn & 1) * warps * 32 + lane;
  __syncwarp();  // lanes past the last channel left the round early
  of_warp[warp * 32] = mine;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < WARPS; ++j) {
    if (j >= warps) break;
    const int w = REVERSE ? warps - 1 - j : j;
    if (w == warp) {
#pragma unroll
      for (int v = 0; v < V; ++v) in[v] = c[v];
    }
    apply<RAGGED>(of_warp[w * 32], c);
  }
}

// The same for a CTA that forms its chunk's map, from its end (REVERSE: from
// its beginning) on: all of its warps' maps go before `total`.
template <bool REVERSE, bool RAGGED, int WARPS, int V>
__device__ __forceinline__ void join_total(Map<V>* shared, const Map<V>& mine, uint32_t turn,
                                           Map<V>& total) {
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, warps = blockDim.x / 32;
  Map<V>* const of_warp = shared + (turn & 1) * warps * 32 + lane;
  __syncwarp();
  of_warp[warp * 32] = mine;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < WARPS; ++j) {
    if (j >= warps) break;
    Map<V> m = of_warp[(REVERSE ? j : warps - 1 - j) * 32];
    follow<RAGGED>(m, total);
    total = m;
  }
}

// Takes c over the chunks [from, to) (REVERSE: from the last of them to the
// first): each warp composes its share, and the warps are joined.
template <bool REVERSE, bool RAGGED, int WARPS, int V>
__device__ __forceinline__ void over_chunks(const Scan& s, int64_t b, int64_t ch, bool on,
                                            int64_t from, int64_t to, Map<V>* shared,
                                            uint32_t turn, float (&c)[V]) {
  if (from >= to) return;
  const int warp = threadIdx.x / 32, warps = blockDim.x / 32;
  const int64_t n = to - from;
  const int64_t w = REVERSE ? warps - 1 - warp : warp;
  Map<V> m = identity<V>();
  // w: this warp's place in the order of application
  const int64_t first = n * w / warps, last = n * (w + 1) / warps;
#pragma unroll 4
  for (int64_t j = first; j < last; ++j) {
    const int64_t k = REVERSE ? to - 1 - j : from + j;
    Map<V> x = identity<V>();
    if (on && SOMA_CHECK(k >= 0 && k < s.chunks && inside(s, b, 0, 0, ch, V), s.status)) {
      const float2* p = s.maps + (b * s.chunks + k) * s.d.dim + ch;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const float2 q = p[v];
        x.a[v] = q.x;
        x.b[v] = q.y;
      }
    }
    follow<RAGGED>(m, x);
  }
  float in[V];
  join<REVERSE, RAGGED, WARPS>(shared, m, turn, c, in);
}

template <int V>
__device__ __forceinline__ void write_map(const Scan& s, int64_t b, int64_t k, int64_t ch,
                                          const Map<V>& m) {
  if (!SOMA_CHECK(k >= 0 && k < s.chunks && inside(s, b, 0, 0, ch, V), s.status)) return;
  float2* p = s.maps + (b * s.chunks + k) * s.d.dim + ch;
#pragma unroll
  for (int v = 0; v < V; ++v) p[v] = make_float2(m.a[v], m.b[v]);
}

// ---- tiled ----------------------------------------------------------------
constexpr int kMaxDepth = 4;

// The tensors of a call as boxes of 64 channels by the CTA's steps: one map
// per gate, then dh; the gradients.
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

// A lane's two channels in shared memory, as they are and as fp32.
__device__ __forceinline__ float2 load_raw(const float* p) {
  return *reinterpret_cast<const float2*>(p);
}
template <typename T>
__device__ __forceinline__ uint32_t load_raw(const T* p) {
  return *reinterpret_cast<const uint32_t*>(p);
}
template <typename T>
__device__ __forceinline__ Two widen(float2 x) { return two(x.x, x.y); }
template <typename T>
__device__ __forceinline__ Two widen(uint32_t x) {
  if (std::is_same<T, __nv_bfloat16>::value)
    return two(__uint_as_float(x << 16), __uint_as_float(x & 0xFFFF0000u));
  __half2 h;
  memcpy(&h, &x, 4);
  const float2 f = __half22float2(h);
  return two(f.x, f.y);
}
template <typename T>
__device__ __forceinline__ Two load_two(const T* p) { return widen<T>(load_raw(p)); }
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

// The bytes [at, at + n) of the CTA's dynamic shared memory.
__device__ __forceinline__ bool in_dynamic(const void* raw, const void* at, size_t n) {
  uint32_t size;
  asm("mov.u32 %0, %%dynamic_smem_size;" : "=r"(size));
  return tc::smem_u32(at) >= tc::smem_u32(raw) && tc::smem_u32(at) + n <= tc::smem_u32(raw) + size;
}

struct Ring {
  uint64_t full[kMaxDepth];
  volatile int abort;
};

__device__ __forceinline__ void ring_init(Ring& r, int depth) {
  if (threadIdx.x == 0) {
    for (int i = 0; i < depth; ++i) tc::mbar_init(&r.full[i], 1);
    tc::mbar_fence_init();
    r.abort = 0;
  }
  __syncthreads();
}

// A wait that runs out records the timeout and raises the abort flag: from
// then on no stage is filled and no wait is made, and the rest of the CTA's
// work runs through on whatever the stages hold.
__device__ __forceinline__ void ring_wait(Ring& r, int stage, uint32_t parity, int* status,
                                          uint32_t max_polls = 1u << 22) {
  if (r.abort || tc::mbar_wait(&r.full[stage], parity, max_polls)) return;
  r.abort = 1;
  atomicCAS(status, 0, SOMA_ERR_TIMEOUT);
}

// Whether the loading warp (all of it) may arm another stage: after an abort
// the stage's last copy may still be on its way, and its barrier not free.
__device__ __forceinline__ bool ring_may_fill(const Ring& r) {
  return !__any_sync(0xffffffffu, r.abort);
}

// One thread, at the end of a CTA: after an abort the copies on their way land
// before the CTA leaves its shared memory to another.  fills: the stages filled
// in all, one after another around the ring, so that stage i's last copy
// completes phase (its number of fills) - 1.
__device__ __forceinline__ void ring_drain(Ring& r, int depth, uint32_t fills) {
  if (!r.abort) return;
  for (int i = 0; i < depth; ++i) {
    const uint32_t n = (fills + depth - 1 - i) / depth;
    if (n) tc::mbar_wait(&r.full[i], (n - 1) & 1);
  }
}

// ------------------------------------------------------------------- host --

inline bool dims_ok(const soma_scan_dims& d) {
  return d.batch >= 0 && d.steps >= 0 && d.dim >= 0 && d.batch <= INT32_MAX &&
         d.steps <= INT32_MAX && d.dim <= (1 << 24) &&
         (d.dim == 0 || d.batch <= ((int64_t)1 << 36) / d.dim);
}

inline bool strides_ok(const soma_scan_strides& s) { return s.b >= 0 && s.t >= 0 && s.g >= 0; }

inline bool dtype_ok(int t) { return t == SOMA_FP32 || t == SOMA_BF16 || t == SOMA_FP16; }

// null pointers pass
inline bool aligned(const void* p, size_t to) {
  return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0;
}

// Whether two states [batch][dim] share memory (null pointers: no).  A call
// reads one all along its chunks and writes the other as soon as its first or
// last chunk is done.
inline bool overlap(const float* p, const float* q, const soma_scan_dims& d) {
  if (!p || !q) return false;
  const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
  return (a < b ? b - a : a - b) < (uintptr_t)(d.batch * d.dim) * sizeof(float);
}

inline size_t width(int dtype) { return dtype == SOMA_FP32 ? 4 : 2; }

// How a call is cut.
struct Shape {
  int warps;                     // of a CTA
  int64_t blocks, chunks, chunk; // of the channels, of the steps; steps of a chunk
  unsigned grid;
  double cost;                   // estimated time, relative to other cuts of the same call
};

// CTAs of up to `most` warps, `fit` of which an SM holds, each over V * 32
// channels.  The time is that of the SM with the most of them, longer where
// their warps do not fill it; with chunks, half as much again for the launch
// that forms the maps (it reads 6 bytes of 10 forward, 10 of 18 backward), and
// what it takes to join them: as long as `join` steps for each of the chunks.
// The alternative for 1 x 32768 x 960 (15 blocks), clusters of eight CTAs that
// joined over distributed shared memory every round, took 170 us forward and
// 350 us backward.
// No CTA of the next launch is admitted before the end of the present ones:
// early ones would sit where there is room and leave the rest badly spread.
inline Shape shape(const soma_scan_dims& d, int V, int most, int fit, double join) {
  Shape f;
  f.blocks = (d.dim + 32 * V - 1) / (32 * V);
  f.warps = 1;
  while (f.warps < most && f.warps * kSegment < d.steps) f.warps *= 2;
  const int64_t items = d.batch * f.blocks, rows = f.warps * kSegment;
  const int64_t slots = (int64_t)kSms * fit;
  const auto cost = [&](int64_t chunks, int64_t chunk) {
    const double n = (double)items * chunks;
    const double waves = n > slots ? std::ceil(n / slots) * slots / n
                                   : std::ceil(n / kSms) * kSms / n;
    const double held = (n < slots ? n : slots) * f.warps / kSms;
    const double enough = fit * f.warps < 16 ? fit * f.warps : 16;
    return waves * (held < enough ? enough / held : 1) *
           (chunks > 1 ? 1.5 + join * (double)chunks / (double)chunk : 1);
  };
  f.chunks = 1;
  f.chunk = d.steps > 0 ? d.steps : 1;
  f.cost = cost(1, f.chunk);
  // two rounds a chunk at least, and no more chunks than are quickly joined
  for (int64_t n = 2; n <= 256 && n * 2 * rows <= d.steps && items * n <= 2 * slots; ++n) {
    const int64_t chunk = (d.steps + n * rows - 1) / (n * rows) * rows;
    const int64_t chunks = (d.steps + chunk - 1) / chunk;
    const double c = cost(chunks, chunk) * (double)(chunk * chunks) / (double)d.steps;
    if (c < f.cost * 0.98) {
      f.cost = c;
      f.chunks = chunks;
      f.chunk = chunk;
    }
  }
  const int64_t cap = (int64_t)1 << 30;
  const int64_t ctas = items * f.chunks;
  f.grid = (unsigned)(ctas < cap ? ctas : cap);
  return f;
}

// Workspace of a call cut like this: its chunks' maps (the checked build's
// canary gaps go around it).
inline size_t maps_bytes(const soma_scan_dims& d, const Shape& f) {
  return f.chunks > 1 ? (size_t)d.batch * f.chunks * d.dim * sizeof(float2) : 0;
}

inline size_t guarded(size_t need) {
  return need && kGuard ? (need + 255) / 256 * 256 + 2 * kGuard : need;
}
inline Gaps gaps_around(size_t need) { return {2, {0, guarded(need) - kGuard}}; }

inline void put(const Shape& f, Scan* s) {
  s->blocks = f.blocks;
  s->chunks = f.chunks;
  s->chunk = f.chunk;
}

template <typename K, typename... A>
cudaError_t launch(K kernel, const Shape& f, size_t smem, cudaStream_t st, A... args) {
  if (smem > (48 << 10)) {  // more than a kernel has unasked
    const cudaError_t e =
        cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
  }
  return launch_overlapped(kernel, dim3(f.grid), 32 * f.warps, smem, st, args...);
}

// A [batch][steps][dim] tensor as a tensor map: its steps inside the sequences
// (t_inner) or the other way round.
struct Layout3 {
  int64_t size[3], stride[2];
};

inline bool layout(const soma_scan_dims& d, const soma_scan_strides& s, bool t_inner, int dtype,
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

inline bool mappable(const void* p, const soma_scan_dims& d, const soma_scan_strides& s,
                     bool gates, bool t_inner, int dtype) {
  const int64_t unit = dtype == SOMA_FP32 ? 4 : 8;
  Layout3 l;
  return aligned(p, 16) && (!gates || s.g % unit == 0) && layout(d, s, t_inner, dtype, &l);
}

// Maps of one tensor's gates (or of the tensor itself), boxes of 64 channels
// by `rows` steps of one sequence.
inline bool map_all(CUtensorMap* maps, int count, const void* p, const soma_scan_dims& d,
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

template <int V>
size_t joint_bytes(int warps) { return sizeof(Map<V>) * 64 * warps; }

template <typename T>
size_t tiled_bytes(int depth, int boxes, int warps) {
  return (size_t)depth * boxes * warps * kSegment * kBlock * sizeof(T) + 128 +
         joint_bytes<2>(warps);
}

// Workspace of the two directions (the larger of the tiled and the plain
// kernels').
size_t forward_workspace(const soma_scan_dims& d);
size_t backward_workspace(const soma_scan_dims& d);

}  // namespace scan
}  // namespace soma
