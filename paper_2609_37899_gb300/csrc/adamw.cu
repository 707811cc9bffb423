// adamw.cu -- AdamW over many tensors in one launch, moments in 32 bits or in
// 8 (soma_adamw_step in include/soma_api.h has the formulas).
//
// Work is cut into chunks of kChunk elements of one tensor, one CTA each, which
// finds its tensor in a table in the kernel's parameters.  (Resident CTAs that
// took chunks in turn were slower: 100M parameters in 32 bits 451 us against
// 368, the copy rate of the memory being 383.)  A thread owns eight consecutive elements, so every stream is read and
// written in 8- to 32-byte pieces, and a warp owns 256: exactly one block of the
// 8-bit state, whose new scale is the warp's maximum.
//
// Bytes bound the 32-bit form: 200M fp32 parameters with bf16 gradients in 300
// tensors, 26 bytes each, take 733 us (7.1 TB/s).  The 8-bit form has about 70
// instructions for 14 to 16 bytes an element and comes to 0.85 of the copy rate:
// 150M bf16 parameters with masters in 120 tensors 418 us (5.7 TB/s).
#include <cfloat>
#include <cmath>
#include <cuda_fp8.h>

#define SOMA_CHECK_FILE 11
#include "checked.cuh"
#include "numeric.cuh"
#include "soma_api.h"
#include "soma_launch.h"

namespace soma {

namespace {

constexpr int kThreads = 128;
constexpr int kGroup = 8;                          // elements of one thread
constexpr int kBlock8 = 256;                       // elements that share a scale
constexpr int kChunk = kThreads * kGroup;          // elements of one CTA
constexpr int kMaxTensors = 360;                   // table rows of one launch
static_assert(kBlock8 == 32 * kGroup, "a warp owns one block of the 8-bit state");

constexpr float kE4M3Max = 448.f;      // largest e4m3 value
constexpr float kE4M3Normal = 0x1p-6f; // smallest normal one; the step below it is 2^-9
constexpr float kE4M3Least = 0x1p-9f;  // smallest above zero

struct Row {
  void* p;
  const void* g;
  void* m;
  void* v;
  float* ms;
  float* vs;
  float* master;
  int64_t n;
  float decay;    // lr * weight_decay
  int32_t index;  // of the tensor in the caller's list
  int64_t first;  // its first chunk
  int64_t vec;    // every address allows 8-element accesses
};

constexpr int kBuckets = 256;

struct Table {
  int32_t rows;
  int32_t shift;  // chunks of a bucket: 2^shift
  int64_t chunks;
  uint16_t row_of[kBuckets + 1];  // the row of a bucket's first chunk
  Row row[kMaxTensors];
};
static_assert(sizeof(Table) + 256 <= 32764, "kernel parameter space");

struct Args {
  float b1, c1, b2, c2;  // beta and 1 - beta
  float lr, s2, eps;     // lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
  uint32_t key[20], t;   // the ten Philox rounds' keys, update
};

// The two rounding forms of y = |x| / scale in [0, 448] to its e4m3 neighbour,
// up or down at random.  Adding 16 random bits (here at their place) right below
// the last kept mantissa bit and cutting the rest off rounds up with the odds
// of the cut-off part.
__device__ __forceinline__ uint32_t round_normal(float y, uint32_t random) {
  return (__float_as_uint(y) + random) & 0xFFF00000u;
}
// Below the smallest normal value the grid has the step 2^-9, which is the
// step of [2^-6, 2^-5): the value is moved there and back.  `floor`: what is
// above zero stays above zero.
__device__ __forceinline__ uint32_t round_any(float y, uint32_t random, bool floor) {
  const float low = y < kE4M3Normal ? kE4M3Normal : 0.f;
  float r = __fsub_rn(__uint_as_float(round_normal(__fadd_rn(y, low), random)), low);
  if (floor && y > 0.f) r = fmaxf(r, kE4M3Least);
  return __float_as_uint(r);
}

// philox4x32_10 with the rounds' keys given.
__device__ __forceinline__ uint4 random_block(uint4 ctr, const uint32_t (&key)[20]) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t p = (uint64_t)0xD2511F53u * ctr.x, q = (uint64_t)0xCD9E8D57u * ctr.z;
    ctr = make_uint4((uint32_t)(q >> 32) ^ ctr.y ^ key[2 * r], (uint32_t)q,
                     (uint32_t)(p >> 32) ^ ctr.w ^ key[2 * r + 1], (uint32_t)p);
  }
  return ctr;
}

// Rounds the warp's 256 values x, the largest magnitude of which is `top`, and
// returns this lane's eight bytes; the scale goes to *scale.  FLOOR: the values
// are roots, none is negative, and what is above zero stays above zero.
template <bool FLOOR>
__device__ __forceinline__ uint2 pack_block(const float (&x)[8], float top,
                                            const uint32_t (&random)[8], float* scale) {
  // below 2^-100 the reciprocal could overflow: such a block is zero
  const bool some = top > 0x1p-100f;
  const float inv = some ? __fdiv_rn(kE4M3Max, top) : 0.f;
  if ((threadIdx.x & 31) == 0) *scale = some ? __fdiv_rn(top, kE4M3Max) : 0.f;
  float y[8], z[8], least = kE4M3Max;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    y[j] = __fmul_rn(fabsf(x[j]), inv);
    least = fminf(least, y[j]);
  }
  // one value in ten thousand of a normal distribution is below the normal
  // ones: the others do without its steps
  if (least >= kE4M3Normal) {
#pragma unroll
    for (int j = 0; j < 8; ++j) z[j] = __uint_as_float(round_normal(y[j], random[j]));
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) z[j] = __uint_as_float(round_any(y[j], random[j], FLOOR));
  }
  if (!FLOOR)
#pragma unroll
    for (int j = 0; j < 8; ++j)
      z[j] = __uint_as_float(__float_as_uint(z[j]) | (__float_as_uint(x[j]) & 0x80000000u));
  // z is on the e4m3 grid, or the step above it where the product was rounded
  // above 448: the conversion is exact or saturates
  uint32_t h[4];
#pragma unroll
  for (int j = 0; j < 4; ++j)
    h[j] = __nv_cvt_float2_to_fp8x2(make_float2(z[2 * j], z[2 * j + 1]), __NV_SATFINITE, __NV_E4M3);
  return make_uint2(h[0] | (h[1] << 16), h[2] | (h[3] << 16));
}

__device__ __forceinline__ float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ void unpack8(const uint2& b, float scale, float (&x)[8]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t w = (j < 2 ? b.x : b.y) >> (16 * (j & 1));
    const __half2 h = __half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w & 0xFFFFu), __NV_E4M3));
    const float2 f = __half22float2(h);
    x[2 * j] = __fmul_rn(f.x, scale);
    x[2 * j + 1] = __fmul_rn(f.y, scale);
  }
}

// The eight elements from p, or the first n of them one by one (FULL: all, by
// wide accesses).
template <bool FULL, typename T>
__device__ __forceinline__ void load_n(const T* p, int n, float (&x)[8]) {
  if (FULL) {
    load8(p, x);
  } else {
#pragma unroll
    for (int j = 0; j < kGroup; ++j) x[j] = j < n ? to_f32(p[j]) : 0.f;
  }
}

template <bool FULL, typename T>
__device__ __forceinline__ void store_n(T* p, int n, const float (&x)[8]) {
  if (FULL) {
    store8(p, x);
  } else {
#pragma unroll
    for (int j = 0; j < kGroup; ++j)
      if (j < n) p[j] = from_f32<T>(x[j]);
  }
}

template <bool FULL>
__device__ __forceinline__ uint2 load_bytes(const uint8_t* p, int n) {
  if (FULL) return *reinterpret_cast<const uint2*>(p);
  uint32_t w[2] = {0u, 0u};
#pragma unroll
  for (int j = 0; j < kGroup; ++j)
    if (j < n) w[j >> 2] |= (uint32_t)p[j] << (8 * (j & 3));
  return make_uint2(w[0], w[1]);
}

template <bool FULL>
__device__ __forceinline__ void store_bytes(uint8_t* p, int n, const uint2& b) {
  if (FULL) {
    *reinterpret_cast<uint2*>(p) = b;
  } else {
#pragma unroll
    for (int j = 0; j < kGroup; ++j)
      if (j < n) p[j] = (uint8_t)((j < 4 ? b.x : b.y) >> (8 * (j & 3)));
  }
}

// The eight elements' new moments (r: the second one's root) and parameters.
// Each operation of the moments is rounded by itself, which makes the 8-bit
// states a matter of the formulas alone.  The parameter's quotient is one of
// the special function unit in the 8-bit form (good to 2^-23), where
// instructions are scarce.
template <bool EIGHT>
__device__ __forceinline__ void update_one(const Args& a, float decay, float x, float& w, float& m,
                                           float& v, float& r) {
  if (EIGHT) v = __fmul_rn(r, r);
  m = __fadd_rn(__fmul_rn(m, a.b1), __fmul_rn(x, a.c1));
  v = __fadd_rn(__fmul_rn(v, a.b2), __fmul_rn(__fmul_rn(x, x), a.c2));
  r = __fsqrt_rn(v);
  float step;
  if (EIGHT) step = m * rcp_approx(fmaf(r, a.s2, a.eps));
  else step = __fdiv_rn(m, __fadd_rn(__fmul_rn(r, a.s2), a.eps));
  // w - decay w in one rounding: 1 - decay would be rounded before the product
  w = __fmaf_rn(-step, a.lr, __fmaf_rn(-w, decay, w));
}

// A thread's eight bytes of the 8-bit state with those set to e4m3's NaN whose
// moments are NaN and stay it.
__device__ __forceinline__ uint2 with_nan(uint2 b, uint32_t which) {
#pragma unroll
  for (int j = 0; j < kGroup; ++j)
    if ((which >> j) & 1u) (j < 4 ? b.x : b.y) |= 0x7Fu << (8 * (j & 3));
  return b;
}

// The thread's eight elements from i on, n of which exist.  FULL: all of the
// warp's exist and are aligned.  Returns whether an element's new moments were
// not finite: it keeps what it had.
template <typename P, typename G, bool MASTER, bool EIGHT, bool FULL>
__device__ __forceinline__ bool eight_elements(const Row& t, const Args& a, float gs, int64_t i,
                                               int n) {
  const int64_t block = (int64_t)((uint64_t)i / kBlock8);
  float g[8], w[8], m[8], v[8], r[8];
  const auto load_state = [&] {
    if (MASTER) load_n<FULL>(t.master + i, n, w);
    else load_n<FULL>(static_cast<const P*>(t.p) + i, n, w);
    if (EIGHT) {
      const uint2 bm = load_bytes<FULL>(static_cast<const uint8_t*>(t.m) + i, n);
      const uint2 bv = load_bytes<FULL>(static_cast<const uint8_t*>(t.v) + i, n);
      const float ms = t.ms[block], vs = t.vs[block];
      unpack8(bm, ms, m);
      unpack8(bv, vs, r);
    } else {
      load_n<FULL>(static_cast<const float*>(t.m) + i, n, m);
      load_n<FULL>(static_cast<const float*>(t.v) + i, n, v);
    }
  };
  load_n<FULL>(static_cast<const G*>(t.g) + i, n, g);
  load_state();
  bool bad = false;
  if (EIGHT) {
#pragma unroll
    for (int j = 0; j < kGroup; ++j)
      update_one<true>(a, t.decay, __fmul_rn(g[j], gs), w[j], m[j], v[j], r[j]);
    // The bits of non-negative floats order as the floats do, NaN above all:
    // one reduction gives the scale and whether all of the block are finite.
    const auto largest = [](const float (&x)[8]) {
      uint32_t top = 0u;
#pragma unroll
      for (int j = 0; j < kGroup; ++j) top = max(top, __float_as_uint(x[j]) & 0x7FFFFFFFu);
      return __reduce_max_sync(0xffffffffu, top);
    };
    uint32_t top_r = largest(r), top_m = largest(m);
    // lost: elements whose stored moment is NaN, eight bits for m and eight for r
    const auto store_all = [&](uint32_t lost) {
      if (MASTER) store_n<FULL>(t.master + i, n, w);
      store_n<FULL>(static_cast<P*>(t.p) + i, n, w);
      const uint64_t q = (uint64_t)i / kGroup;
      const uint4 rnd =
          random_block(make_uint4((uint32_t)q, (uint32_t)t.index, a.t, 0x80000002u), a.key);
      uint32_t random[8];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        random[2 * j] = (word_of(rnd, j) << 4) & 0xFFFF0u;
        random[2 * j + 1] = (word_of(rnd, j) >> 12) & 0xFFFF0u;
      }
      const uint2 bm = pack_block<false>(m, __uint_as_float(top_m), random, t.ms + block);
      const uint2 bv = pack_block<true>(r, __uint_as_float(top_r), random, t.vs + block);
      store_bytes<FULL>(static_cast<uint8_t*>(t.m) + i, n, with_nan(bm, lost));
      store_bytes<FULL>(static_cast<uint8_t*>(t.v) + i, n, with_nan(bv, lost >> 8));
    };
    if (max(top_r, top_m) >= 0x7F800000u) {  // the whole warp
      // a gradient that is not finite, or whose square is not, or a stored moment
      if (!isfinite(t.ms[block]) || !isfinite(t.vs[block])) return true;  // no element has moments
      uint32_t keep = 0, lost = 0;
      float new_w[8], new_m[8], new_r[8];
#pragma unroll
      for (int j = 0; j < kGroup; ++j) {
        if (!isfinite(r[j]) || !isfinite(m[j])) keep |= 1u << j;
        new_w[j] = w[j], new_m[j] = m[j], new_r[j] = r[j];
      }
      load_state();
#pragma unroll
      for (int j = 0; j < kGroup; ++j) {
        if (!((keep >> j) & 1u)) w[j] = new_w[j], m[j] = new_m[j], r[j] = new_r[j];
        // the scales are those of the others
        if (!isfinite(m[j])) lost |= 1u << j, m[j] = 0.f;
        if (!isfinite(r[j])) lost |= 256u << j, r[j] = 0.f;
      }
      top_r = largest(r);
      top_m = largest(m);
      store_all(lost);  // apart, so that the common path holds no `lost`
      return keep != 0;
    }
    store_all(0u);
  } else {
#pragma unroll
    for (int j = 0; j < kGroup; ++j) {
      float w1 = w[j], m1 = m[j], v1 = v[j];
      update_one<false>(a, t.decay, __fmul_rn(g[j], gs), w1, m1, v1, r[j]);
      if (isfinite(m1) && isfinite(v1)) w[j] = w1, m[j] = m1, v[j] = v1;
      else bad = true;
    }
    if (MASTER) store_n<FULL>(t.master + i, n, w);
    store_n<FULL>(static_cast<P*>(t.p) + i, n, w);
    store_n<FULL>(static_cast<float*>(t.m) + i, n, m);
    store_n<FULL>(static_cast<float*>(t.v) + i, n, v);
  }
  return bad;
}

// In 8 bits nine CTAs an SM: with eight its loads cover one another less (277 us
// against 269 for 100M bf16 parameters with masters), with ten registers spill
// (275 us).
template <typename P, typename G, bool MASTER, bool EIGHT>
__global__ void __launch_bounds__(kThreads, EIGHT ? 9 : 8)
adamw_kernel(const __grid_constant__ Table tab, const __grid_constant__ Args a,
             const float* __restrict__ grad_scale, int* status) {
  const float gs = grad_scale ? *grad_scale : 1.f;
  if (!isfinite(gs)) {
    if (blockIdx.x == 0 && threadIdx.x == 0) atomicCAS(status, 0, SOMA_ERR_NONFINITE);
    return;
  }
  bool bad = false;
  for (int64_t chunk = blockIdx.x; chunk < tab.chunks; chunk += gridDim.x) {
    // the last row whose first chunk is <= chunk, from the bucket's rows on: over
    // all of 120 rows the search took an eighth of the 8-bit kernel's time
    const int bucket = (int)(chunk >> tab.shift);
    int lo = tab.row_of[bucket], hi = tab.row_of[bucket + 1];
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (tab.row[mid].first <= chunk) lo = mid; else hi = mid - 1;
    }
    if (!SOMA_CHECK(bucket < kBuckets && lo >= 0 && lo < tab.rows && tab.row[lo].first <= chunk,
                    status))
      continue;
    const Row& t = tab.row[lo];
    const int64_t i = (chunk - t.first) * kChunk + (int64_t)threadIdx.x * kGroup;
    const int64_t warp_i = i - (threadIdx.x & 31) * kGroup;
    if (warp_i >= t.n) continue;
    if (!SOMA_CHECK(warp_i >= 0 && warp_i % kBlock8 == 0, status)) continue;
    if (t.vec && warp_i + 32 * kGroup <= t.n) {
      bad |= eight_elements<P, G, MASTER, EIGHT, true>(t, a, gs, i, kGroup);
    } else {
      const int n = i >= t.n ? 0 : (int)(t.n - i < kGroup ? t.n - i : kGroup);
      const bool in = SOMA_CHECK(n >= 0 && n <= kGroup && (n == 0 || i + n <= t.n), status);
      bad |= eight_elements<P, G, MASTER, EIGHT, false>(t, a, gs, i, in ? n : 0);
    }
  }
  if (bad) atomicCAS(status, 0, SOMA_ERR_NONFINITE);
}

using Kernel = void (*)(const Table, const Args, const float*, int*);

template <typename P, typename G>
Kernel pick(bool master, bool eight) {
  if (master) return eight ? adamw_kernel<P, G, true, true> : adamw_kernel<P, G, true, false>;
  return eight ? adamw_kernel<P, G, false, true> : adamw_kernel<P, G, false, false>;
}

template <typename P>
Kernel pick(int grad, bool master, bool eight) {
  if (grad == SOMA_FP32) return pick<P, float>(master, eight);
  if (grad == SOMA_BF16) return pick<P, __nv_bfloat16>(master, eight);
  return pick<P, __half>(master, eight);
}

Kernel pick(int param, int grad, bool master, bool eight) {
  if (param == SOMA_FP32) return pick<float>(grad, false, eight);
  if (param == SOMA_BF16) return pick<__nv_bfloat16>(grad, master, eight);
  return pick<__half>(grad, master, eight);
}

int width(int dtype) { return dtype == SOMA_FP32 ? 4 : 2; }

bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

}  // namespace

}  // namespace soma

using namespace soma;

extern "C" int soma_adamw_step(const soma_adamw_tensor* tensors, int n_tensors,
                               soma_adamw_config cfg, const float* grad_scale, void* stream) {
  const auto dtype_ok = [](int d) { return d == SOMA_FP32 || d == SOMA_BF16 || d == SOMA_FP16; };
  if (n_tensors < 0 || (n_tensors > 0 && !tensors) || !dtype_ok(cfg.param_dtype) ||
      !dtype_ok(cfg.grad_dtype) || (cfg.state_bits != 8 && cfg.state_bits != 32) || cfg.t < 1 ||
      !std::isfinite(cfg.lr) || !(cfg.beta1 >= 0 && cfg.beta1 < 1) ||
      !(cfg.beta2 >= 0 && cfg.beta2 < 1) || !((float)cfg.eps > 0.f) ||
      !std::isfinite((float)cfg.eps) || !aligned(grad_scale, 4))
    return SOMA_ERR_INVALID_ARG;
  const bool eight = cfg.state_bits == 8;
  // the 8-bit form's reciprocal takes a subnormal denominator for 0, and an
  // element with zero moments would get 0 times infinity
  if (eight && (float)cfg.eps < FLT_MIN) return SOMA_ERR_INVALID_ARG;
  const int pw = width(cfg.param_dtype), gw = width(cfg.grad_dtype), sw = eight ? 1 : 4;
  bool master = false, plain = false;
  for (int k = 0; k < n_tensors; ++k) {
    const soma_adamw_tensor& t = tensors[k];
    if (t.count < 0 || t.count > ((int64_t)1 << 40) || !(t.weight_decay >= 0) ||
        !std::isfinite(t.weight_decay))
      return SOMA_ERR_INVALID_ARG;
    if (t.count == 0) continue;
    if (!t.param || !t.grad || !t.m || !t.v || !aligned(t.param, pw) || !aligned(t.grad, gw) ||
        !aligned(t.m, sw) || !aligned(t.v, sw) || !aligned(t.master, 4) ||
        !aligned(t.m_scale, 4) || !aligned(t.v_scale, 4) ||
        (eight ? !t.m_scale || !t.v_scale : t.m_scale || t.v_scale) ||
        (t.master && cfg.param_dtype == SOMA_FP32))
      return SOMA_ERR_INVALID_ARG;
    (t.master ? master : plain) = true;
  }
  if (master && plain) return SOMA_ERR_INVALID_ARG;  // masters for all tensors or for none
  int* status = status_ptr();
  if (!status) return SOMA_ERR_CUDA;

  Args a;
  a.b1 = (float)cfg.beta1;
  a.c1 = (float)(1.0 - cfg.beta1);
  a.b2 = (float)cfg.beta2;
  a.c2 = (float)(1.0 - cfg.beta2);
  a.lr = (float)(cfg.lr / (1.0 - std::pow(cfg.beta1, (double)cfg.t)));
  a.s2 = (float)(1.0 / std::sqrt(1.0 - std::pow(cfg.beta2, (double)cfg.t)));
  a.eps = (float)cfg.eps;
  for (uint32_t r = 0; r < 10; ++r) {  // the key advances by the Weyl constants (philox4x32_10)
    a.key[2 * r] = (uint32_t)cfg.seed + r * 0x9E3779B9u;
    a.key[2 * r + 1] = (uint32_t)(cfg.seed >> 32) + r * 0xBB67AE85u;
  }
  a.t = (uint32_t)cfg.t;
  const Kernel kernel = pick(cfg.param_dtype, cfg.grad_dtype, master, eight);

  Table tab;
  int k = 0;
  while (k < n_tensors) {
    tab.rows = 0;
    tab.chunks = 0;
    for (; k < n_tensors && tab.rows < kMaxTensors; ++k) {
      const soma_adamw_tensor& t = tensors[k];
      if (t.count == 0) continue;
      Row& r = tab.row[tab.rows++];
      r.p = t.param;
      r.g = t.grad;
      r.m = t.m;
      r.v = t.v;
      r.ms = t.m_scale;
      r.vs = t.v_scale;
      r.master = t.master;
      r.n = t.count;
      r.decay = (float)(cfg.lr * t.weight_decay);
      r.index = k;
      r.first = tab.chunks;
      r.vec = aligned(t.param, 16) && aligned(t.grad, 16) && aligned(t.m, eight ? 8 : 16) &&
              aligned(t.v, eight ? 8 : 16) && aligned(t.master, 16);
      tab.chunks += (t.count + kChunk - 1) / kChunk;
    }
    if (!tab.rows) break;
    tab.shift = 0;
    while (((tab.chunks - 1) >> tab.shift) >= kBuckets) ++tab.shift;
    for (int j = 0, r = 0; j <= kBuckets; ++j) {
      while (r + 1 < tab.rows && tab.row[r + 1].first <= (int64_t)j << tab.shift) ++r;
      tab.row_of[j] = (uint16_t)r;
    }
    const int64_t most = (int64_t)1 << 30;
    const unsigned grid = (unsigned)(tab.chunks < most ? tab.chunks : most);
    trace_begin(SOMA_TRACE_ADAMW, (cudaStream_t)stream);
    kernel<<<grid, kThreads, 0, (cudaStream_t)stream>>>(tab, a, grad_scale, status);
    trace_end(SOMA_TRACE_ADAMW, (cudaStream_t)stream);
    if (cudaGetLastError() != cudaSuccess) return SOMA_ERR_CUDA;
  }
  return SOMA_OK;
}
