// sample.cu -- one token per row of logits by temperature, top-k, top-p and min-p
// from given random numbers (soma_sample in include/soma_api.h).
//
// A cluster of up to eight CTAs shares a row, each with a part of the vocabulary
// in its shared memory, so that the logits are read once (above 131,072 of them, or
// seven fewer where rows do not begin at 16 bytes, from L2 or memory in every pass).  The ranking is never made: top-k and top-p
// each need one cut in it, which is found as a radix selection finds it, by
// counts (or weights) per bin, the bin that the cut lies in, then the logits of
// that one: sorted in a list where they are few, by finer bins where not (equal
// logits, as a rule).  The first bins are equal steps of (max - l) / T.
//
// Weights are whole numbers, so sums do not depend on their order and every CTA
// of a cluster comes to the same cut by itself.
//
// Few rows are bound by latency, one step after another, six meetings of the cluster
// among them: 1 x 131072 bf16, top-k 50 and top-p 0.9: 19 us a call (25 after a flush
// of L2); 64 x 50021 with settings per row 33 to 38.  Many by
// instruction issue, some 300 per logit over two evaluations of its weight and four
// scans: 256 x 131072 fp32, top-p alone, 413 us, 0.05 of the copy rate.
#include <cmath>

#define SOMA_CHECK_FILE 13
#include "checked.cuh"
#include "numeric.cuh"
#include "pdl.cuh"
#include "soma_api.h"
#include "soma_launch.h"
#include "tc_tiles.cuh"

namespace soma {

namespace {

using u64 = unsigned long long;

constexpr int kBins = 2048;
constexpr int kMaxCluster = 8;
constexpr int kSlots = 24;                 // exchanges between the CTAs of a row
constexpr int kHeld = 32;                  // logits of a thread that shared memory holds
constexpr int kMostVocab = 1 << 20;
constexpr int kMostPart = kMostVocab / kMaxCluster + 8;  // logits of a CTA, at most
constexpr float kDeepest = 28.5f;          // 2^40 exp(-28.42) = 1/2: weights further down are 0
constexpr float kStep = kDeepest / kBins;
constexpr float kLeastTemperature = 0x1p-100f, kMostTemperature = 0x1p100f;

// 2^(-j/64) as the sum of two fp32 numbers.
__device__ const float2 kRoots[64] = {
    {1.f, 0.f}, {0.98922801f, 3.01636316e-09f}, {0.978572071f, -8.51090221e-09f},
    {0.96803087f, 2.67853615e-08f}, {0.957603276f, 4.92266405e-09f}, {0.947287977f, 1.40516923e-08f},
    {0.93708384f, -2.33150281e-08f}, {0.926989555f, 7.18280591e-09f}, {0.917004049f, -5.61963898e-09f},
    {0.907126069f, 1.86812912e-08f}, {0.897354543f, -5.70752245e-09f}, {0.88768822f, 2.67159894e-08f},
    {0.878126085f, -4.61788519e-09f}, {0.868666947f, -2.92511171e-08f}, {0.859309673f, -2.4248088e-08f},
    {0.850053191f, -1.43257362e-08f}, {0.840896428f, -1.23776633e-08f}, {0.83183831f, -1.96014938e-08f},
    {0.822877765f, -2.56248605e-08f}, {0.81401372f, -8.63004157e-09f}, {0.805245161f, 4.91810859e-09f},
    {0.796571076f, -2.45156839e-10f}, {0.787990451f, -2.83051271e-08f}, {0.779502213f, -1.28823325e-08f},
    {0.771105409f, 4.03545242e-09f}, {0.762799084f, -8.81428441e-09f}, {0.754582226f, -1.24796866e-08f},
    {0.746453881f, -1.71181007e-08f}, {0.738413095f, -2.25044943e-08f}, {0.730458915f, -1.81432878e-08f},
    {0.722590387f, 1.66209997e-08f}, {0.714806676f, -6.71496458e-09f}, {0.707106769f, 1.21016175e-08f},
    {0.699489832f, 4.34471703e-09f}, {0.69195497f, -2.93778868e-08f}, {0.684501231f, -1.92294092e-08f},
    {0.677127779f, -5.06167463e-09f}, {0.669833779f, -1.73083698e-08f}, {0.662618339f, -1.74818666e-08f},
    {0.655480623f, -1.74828578e-08f}, {0.648419797f, -2.00949977e-08f}, {0.641435027f, -1.90831084e-08f},
    {0.634525478f, 7.09666659e-10f}, {0.627690375f, 3.66111874e-09f}, {0.620928884f, 2.24841905e-08f},
    {0.614240289f, -2.06810018e-08f}, {0.607623696f, -1.63369744e-08f}, {0.601078391f, -2.53487826e-08f},
    {0.594603539f, 1.89881764e-08f}, {0.588198483f, 1.28348754e-08f}, {0.58186245f, -2.02572075e-08f},
    {0.575594604f, 1.09611413e-08f}, {0.56939429f, 2.69311116e-08f}, {0.563260794f, 1.56182072e-08f},
    {0.557193398f, -2.71777001e-08f}, {0.55119127f, 2.130251e-08f}, {0.545253873f, -6.53876997e-09f},
    {0.539380372f, 2.73079728e-08f}, {0.53357023f, -2.96687599e-08f}, {0.527822614f, -2.45358471e-08f},
    {0.522136867f, 2.41673508e-08f}, {0.516512454f, -1.40454466e-08f}, {0.510948598f, -2.40577993e-08f},
    {0.505444646f, -2.85580271e-09f}};

// The weight of a token whose logit l is at most kDeepest temperatures below
// max; inv = 1 / T as the sum of two fp32 numbers.  x = (l - max) / T is split
// into -k ln2/64 + r with |r| < 0.0055, and exp(x) = 2^-(k/64) (1 + r + r^2/2 +
// ...), with what fp32 rounds off the large terms carried along.  The whole number is
// less than 4 from 2^40 exp(x): 3.1 at most among 2 10^7 logits, at temperatures
// from 1/400 to 400.
__device__ __forceinline__ u64 weight(float l, float max, float2 inv, const float2* roots) {
  // l - max = d + e (Knuth's two-sum), times inv
  const float d = __fsub_rn(l, max), b = __fsub_rn(d, l);
  const float e = __fsub_rn(__fsub_rn(l, __fsub_rn(d, b)), __fadd_rn(max, b));
  const float xh = __fmul_rn(d, inv.x);
  const float xl = fmaf(d, inv.y, fmaf(e, inv.x, fmaf(d, inv.x, -xh)));
  // ln2 / 64 in parts of 12 bits, whose products with k (12 bits) are exact
  const float k = fminf(rintf(-xh * 92.3324826f), 4095.f);
  const float r = fmaf(k, 0x1.62ep-7f, xh);
  const float m = __fmul_rn(k, 0x1.0bep-21f);
  const float rh = __fadd_rn(r, m);
  const float rl = __fadd_rn(__fsub_rn(m, __fsub_rn(rh, r)), fmaf(k, 0x1.be8e7cp-33f, xl));
  const float q = fmaf(rh * rh, fmaf(rh, fmaf(rh, 1.f / 24, 1.f / 6), 0.5f),
                       fmaf(rl, rh, rl));
  const int n = (int)k;
  const float2 t = roots[n & 63];
  const float p = __fmul_rn(t.x, rh);
  const float s = __fadd_rn(t.x, p);
  const float lo = __fadd_rn(__fsub_rn(p, __fsub_rn(s, t.x)),
                             fmaf(t.x, q, fmaf(t.x, rh, -p)) + fmaf(t.y, rh, t.y));
  // to units of 2^-40, the upper 20 bits apart
  const float up = __fmul_rn(s, 0x1p20f);
  const int whole = (int)up;
  const float rest = __fsub_rn(up, (float)whole);
  const long long w = ((long long)whole << 20) +
                      (int)rintf(__fmul_rn(fmaf(lo, 0x1p20f, rest), 0x1p20f));
  const int shift = n >> 6;
  return shift ? (u64)(w + (1ll << (shift - 1))) >> shift : (u64)w;
}

// A number that orders as the logits do, and the logit of such a number.
// 16-bit types have at most 19 significant bits in it, which 22 hold.
template <typename T>
constexpr int kKeyBits = sizeof(T) == 4 ? 32 : 22;
template <typename T>
__device__ __forceinline__ uint32_t key_of(float l) {
  const uint32_t b = __float_as_uint(__fadd_rn(l, 0.f));  // -0 as 0
  return (b >> 31 ? ~b : b | 0x80000000u) >> (32 - kKeyBits<T>);
}
template <typename T>
__device__ __forceinline__ float logit_of(uint32_t key) {
  const uint32_t b = key << (32 - kKeyBits<T>);
  const uint32_t low = (1u << (32 - kKeyBits<T>)) - 1;
  return __uint_as_float(b >> 31 ? b & 0x7fffffffu : ~(b | low));
}

struct Sample {
  int64_t stride, rows;
  int32_t vocab;
  int32_t part;  // elements of a CTA
  soma_sample_config cfg;
  const float* u;
  int64_t* tokens;
  float* logprobs;
};

// Logits that one CTA finishes alone.
__host__ __device__ constexpr int list_of(int threads) { return 2 * threads; }

// Logits of a thread: neighbouring ones, in eights.
__host__ __device__ constexpr int each_of(int part, int threads) {
  return (part + 8 * threads - 1) / (8 * threads) * 8;
}

template <int THREADS>
struct __align__(16) Shared {
  uint32_t hist[3][kBins];
  float2 roots[64];
  u64 slot[kSlots][3];         // sums of this CTA, for the others
  u64 part[3][THREADS / 32];
  float2 inv;
  u64 found[3], need;
  u64 list[list_of(THREADS)];     // rank 0's: key and index, sorted
  u64 weights[list_of(THREADS)];  // running sums of the list's weights
  uint32_t listed;
  int lo, hi;
};

__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t n;
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(n));
  return n;
}
__device__ __forceinline__ uint32_t at_rank(const void* p, uint32_t rank) {
  uint32_t a;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(tc::smem_u32(p)), "r"(rank));
  return a;
}
__device__ __forceinline__ uint32_t remote32(const uint32_t* p, uint32_t rank) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(at_rank(p, rank)) : "memory");
  return v;
}
__device__ __forceinline__ void set_remote64(u64* p, uint32_t rank, u64 v) {
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(at_rank(p, rank)), "l"(v) : "memory");
}
__device__ __forceinline__ u64 remote64(const u64* p, uint32_t rank) {
  u64 v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(at_rank(p, rank)) : "memory");
  return v;
}

// The same variable of all CTAs (at most N), on their way together.
template <int N>
__device__ __forceinline__ void remote_all(const u64* p, uint32_t ranks, u64 (&v)[N]) {
#pragma unroll
  for (uint32_t r = 0; r < N; ++r) v[r] = remote64(p, min(r, ranks - 1));
#pragma unroll
  for (uint32_t r = 0; r < N; ++r)
    if (r >= ranks) v[r] = 0;
}

// One row's work in one CTA.
template <typename T, int THREADS, bool HELD>
struct Row {
  using S = Shared<THREADS>;
  static constexpr int kWarps = THREADS / 32;
  static constexpr int kOwn = kBins / THREADS;  // bins of a thread
  static constexpr int kList = list_of(THREADS);
  static constexpr int kMost = THREADS < 512 ? 1 : kMaxCluster;  // CTAs of a row
  S& sh;
  const T* row;        // 16-byte aligned, `shift` elements before the first logit
  int shift, end;      // end: one behind the last logit, counted from `row`
  int vocab;
  int* status;
  int first, stop;     // this thread's
  uint32_t rank, ranks;
  int slots = 0;
  float max = 0.f, inv = 0.f;
  float2 inv2 = {0.f, 0.f};
  uint32_t cut = 0;    // what is ranked above this key remains, and ...
  u64 ties = 0;        // ... so many of this key

  __device__ Row(S& s) : sh(s) {}

  // Where the checked build looks: an exchange, a bin, a place in the list, a group of
  // eight held logits, and logits of the row.
  __device__ __forceinline__ bool slot_ok() const {
    return SOMA_CHECK(slots >= 0 && slots < kSlots, status);
  }
  __device__ __forceinline__ bool bin_ok(int b) const {
    return SOMA_CHECK(b >= 0 && b < kBins, status);
  }
  __device__ __forceinline__ bool listed_ok(int i) const {
    return SOMA_CHECK(i >= 0 && i < kList, status);
  }
  __device__ __forceinline__ bool held_ok(int group) const {
    return SOMA_CHECK(HELD && group >= 0 && group < kHeld / 8, status);
  }
  __device__ __forceinline__ bool logits_ok(int i, int n) const {
    return SOMA_CHECK(i >= shift && i - shift + n <= vocab, status);
  }

  // The sum of a variable over the CTAs before `upto`.
  __device__ __forceinline__ u64 remote_sum(const u64* p, uint32_t upto) const {
    u64 v[kMost], t = 0;
    remote_all(p, ranks, v);
#pragma unroll
    for (uint32_t r = 0; r < kMost; ++r) t += r < upto ? v[r] : 0;
    return t;
  }

  // Eight logits in shared memory: 16-byte pieces of neighbouring threads side by
  // side.  What lies outside the row is -infinity.
  static constexpr int kPieces = sizeof(T) / 2;
  uint4* held;
  __device__ __forceinline__ void hold(int group, const float (&v)[8]) {
    union {
      T t[8];
      uint4 u[kPieces];
    } w;
#pragma unroll
    for (int j = 0; j < 8; ++j) w.t[j] = from_f32<T>(v[j]);  // exact
#pragma unroll
    for (int k = 0; k < kPieces; ++k)
      if (held_ok(group)) held[(group * kPieces + k) * THREADS + threadIdx.x] = w.u[k];
  }
  __device__ __forceinline__ void load(int i, float (&v)[8]) const {
    if (HELD) {
      union {
        T t[8];
        uint4 u[kPieces];
      } w;
      const int group = (i - first) / 8;
#pragma unroll
      for (int k = 0; k < kPieces; ++k)
        w.u[k] = held[(held_ok(group) ? group * kPieces + k : 0) * THREADS + threadIdx.x];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = to_f32(w.t[j]);
    } else {
      fetch(i, v);
    }
  }
  __device__ __forceinline__ void fetch(int i, float (&v)[8]) const {
    if (i >= shift && i + 8 <= end && logits_ok(i, 8)) {
      load8(row + i, v);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        v[j] = i + j >= shift && i + j < end && logits_ok(i + j, 1) ? to_f32(row[i + j]) : -INFINITY;
    }
  }
  // f(logit, index from `row`) for this thread's logits in order.
  template <typename F>
  __device__ __forceinline__ void each(F f) const {
    for (int i = first; i < stop; i += 8) {
      float v[8];
      load(i, v);
#pragma unroll
      for (int j = 0; j < 8; ++j) f(v[j], i + j);
    }
  }
  // The first pass: the same over the logits in memory, which shared memory holds
  // from then on.
  template <typename F>
  __device__ __forceinline__ void first_pass(F f) {
#pragma unroll
    for (int g = 0; g < kHeld / 8; g += 2) {
      float v[2][8];
#pragma unroll
      for (int u = 0; u < 2; ++u)
        if (first + 8 * (g + u) < stop) fetch(first + 8 * (g + u), v[u]);
#pragma unroll
      for (int u = 0; u < 2; ++u)
        if (first + 8 * (g + u) < stop) {
          hold(g + u, v[u]);
#pragma unroll
          for (int j = 0; j < 8; ++j) f(v[u][j], 0);
        }
    }
  }
  // f(logit, index, depth) for those whose weight may be above 0.  The depth, in
  // bins, orders as the logits do: bin b has those of [b, b + 1).
  template <typename F>
  __device__ __forceinline__ void each_weighted(F f) const {
    each([&](float l, int i) {
      const float depth = __fmul_rn(__fmul_rn(__fsub_rn(max, l), inv), 1.f / kStep);
      if (depth < kBins) f(l, i, depth);
    });
  }
  __device__ __forceinline__ static bool in(float depth, int bin) {
    return depth >= bin && depth < bin + 1;
  }
  // whether a top-k cut leaves it, but for those at the cut itself
  __device__ __forceinline__ bool above_cut(float l) const {
    return cut == 0 || key_of<T>(l) > cut;
  }
  __device__ __forceinline__ u64 weight_of(float l) const {
    return weight(l, max, inv2, sh.roots);
  }

  // The largest over the row's CTAs.
  __device__ u64 largest(u64 v) {
#pragma unroll
    for (int k = 16; k; k >>= 1) {
      const u64 o = __shfl_xor_sync(0xffffffffu, v, k);
      v = o > v ? o : v;
    }
    if (threadIdx.x % 32 == 0) sh.part[0][threadIdx.x / 32] = v;
    __syncthreads();
    if (threadIdx.x == 0) {
      for (int w = 1; w < kWarps; ++w) v = sh.part[0][w] > v ? sh.part[0][w] : v;
      if (slot_ok()) sh.slot[slots][0] = v;
    }
    tc::cluster_sync();
    u64 o[kMost];
    remote_all(&sh.slot[slots][0], ranks, o);
#pragma unroll
    for (uint32_t r = 0; r < kMost; ++r) v = r == 0 || o[r] > v ? o[r] : v;
    ++slots;
    return v;
  }

  // ---- bins: those of all CTAs have been read when find() or band() returns ----
  __device__ void clear(int arrays) {
    for (int a = 0; a < arrays; ++a)
      for (int b = threadIdx.x; b < kBins; b += THREADS) sh.hist[a][b] = 0;
    __syncthreads();
  }
  __device__ __forceinline__ void count(int b) {
    if (bin_ok(b)) atomicAdd(&sh.hist[0][b], 1u);
  }
  // weights go by 14 bits, whose sums over a CTA's logits fit 32 bits
  static_assert(((u64)kMostPart << 14) - kMostPart <= 0xffffffffu, "sums of 14 bits");
  __device__ __forceinline__ void add(int b, u64 w) {
    if (!bin_ok(b)) return;
    atomicAdd(&sh.hist[0][b], (uint32_t)w & 0x3fffu);
    atomicAdd(&sh.hist[1][b], (uint32_t)(w >> 14) & 0x3fffu);
    atomicAdd(&sh.hist[2][b], (uint32_t)(w >> 28));
  }
  template <bool WEIGHTS>
  __device__ __forceinline__ u64 in_bin(int b) const {
    uint32_t v[kMost][WEIGHTS ? 3 : 1];
    if (!bin_ok(b)) return 0;
#pragma unroll
    for (uint32_t r = 0; r < kMost; ++r)
#pragma unroll
      for (int a = 0; a < (WEIGHTS ? 3 : 1); ++a) v[r][a] = remote32(&sh.hist[a][b], min(r, ranks - 1));
    u64 t = 0;
#pragma unroll
    for (uint32_t r = 0; r < kMost; ++r)
      if (r < ranks) {
        t += v[r][0];
        if (WEIGHTS) t += ((u64)v[r][WEIGHTS ? 1 : 0] << 14) + ((u64)v[r][WEIGHTS ? 2 : 0] << 28);
      }
    return t;
  }
  // Every CTA adds up a slice of the bins over all of them.  A thread's bins of it:
  __device__ __forceinline__ int slice_bins() const {  // 0: none
    const int per = kBins / (int)ranks;
    return per >= THREADS ? per / THREADS : (int)threadIdx.x < per ? 1 : 0;
  }
  __device__ __forceinline__ int slice_first() const {
    const int per = kBins / (int)ranks;
    return (int)rank * per + (int)threadIdx.x * (per >= THREADS ? per / THREADS : 1);
  }
  // The sum of `v` over the threads before this one; *all: over all of them.
  template <typename V>
  __device__ __forceinline__ V before_me(V v, V* parts, V* all) {
    V run = v;
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
#pragma unroll
    for (int k = 1; k < 32; k <<= 1) {
      const V o = __shfl_up_sync(0xffffffffu, run, k);
      if (lane >= k) run += o;
    }
    if (lane == 31) parts[warp] = run;
    __syncthreads();
    run -= v;
    V total = 0;
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) run += parts[w];
      total += parts[w];
    }
    *all = total;
    return run;
  }
  // The bin where the running sum over the row's bins reaches need_of(the sum of
  // all), which is at least 1; the sum before it and what it holds.  False if none
  // does.
  template <bool WEIGHTS, typename F>
  __device__ bool find(F need_of, int* bin, u64* need, u64* before, u64* held_there) {
    if (threadIdx.x == 0) sh.found[0] = ~0ull;
    tc::cluster_sync();
    const int bins = slice_bins(), b0 = slice_first();
    u64 own[kOwn], total = 0, all;
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      own[j] = j < bins ? in_bin<WEIGHTS>(b0 + j) : 0;
      total += own[j];
    }
    u64 run = before_me(total, sh.part[0], &all);
    if (threadIdx.x == 0 && slot_ok()) sh.slot[slots][0] = all;
    tc::cluster_sync();
    run += remote_sum(&sh.slot[slots][0], rank);
    if (threadIdx.x == 0) sh.need = need_of(remote_sum(&sh.slot[slots][0], ranks));
    __syncthreads();
    *need = sh.need;
    ++slots;
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      if (j < bins && run < *need && run + own[j] >= *need)
        for (uint32_t r = 0; r < ranks; ++r) {
          set_remote64(&sh.found[0], r, (u64)(b0 + j));
          set_remote64(&sh.found[1], r, run);
          set_remote64(&sh.found[2], r, own[j]);
        }
      run += own[j];
    }
    tc::cluster_sync();
    *bin = (int)sh.found[0];
    *before = sh.found[1];
    *held_there = sh.found[2];
    return sh.found[0] != ~0ull;
  }
  // ---- a list of few logits in rank 0 ----
  // Those for which f says so, kList at most, sorted by logit and index.
  template <typename F>
  __device__ void gather(F f) {
    if (threadIdx.x == 0) sh.listed = 0;
    tc::cluster_sync();
    each_weighted([&](float l, int i, float depth) {
      if (!f(l, depth)) return;
      uint32_t at;
      asm volatile("atom.shared::cluster.add.u32 %0, [%1], 1;"
                   : "=r"(at)
                   : "r"(at_rank(&sh.listed, 0))
                   : "memory");
      if (listed_ok((int)at) && at < kList)  // as many as were counted, or estimated
        set_remote64(&sh.list[at], 0, (u64)key_of<T>(l) << 32 | (~(uint32_t)i));
    });
    tc::cluster_sync();
    if (rank == 0) sort((int)min(sh.listed, (uint32_t)kList));
  }
  // Sorts rank 0's list downwards: bitonic, past its end zeros.
  __device__ void sort(int count) {
    int n = 2;
    while (n < count) n *= 2;
    if (!listed_ok(n - 1)) return;
    for (int i = count + threadIdx.x; i < n; i += THREADS) sh.list[i] = 0;
    __syncthreads();
    for (int size = 2; size <= n; size *= 2)
      for (int step = size / 2; step > 0; step /= 2) {
        for (int t = threadIdx.x; t < n / 2; t += THREADS) {
          const int a = 2 * t - (t & (step - 1)), b = a + step;
          const u64 x = sh.list[a], y = sh.list[b];
          if ((x < y) == ((a & size) == 0)) {
            sh.list[a] = y;
            sh.list[b] = x;
          }
        }
        __syncthreads();
      }
  }
  // Running sums over f(position) of the list into sh.weights.
  template <typename F>
  __device__ u64 run_over(int count, F f) {
    constexpr int kEach = (kList + THREADS - 1) / THREADS;
    u64 own[kEach], total = 0, all;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      const int i = threadIdx.x * kEach + j;
      total += own[j] = i < count ? f(i) : 0;
    }
    u64 run = before_me(total, sh.part[0], &all);
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      run += own[j];
      if (threadIdx.x * kEach + j < kList) sh.weights[threadIdx.x * kEach + j] = run;
    }
    __syncthreads();
    return all;
  }
  // The first of `count` positions whose running sum is at least `need`, or count.
  __device__ int reaches(int count, u64 need) {
    if (threadIdx.x == 0) sh.lo = count;
    __syncthreads();
    for (int i = threadIdx.x; i < count; i += THREADS)
      if (sh.weights[i] >= need && (i == 0 || sh.weights[i - 1] < need)) sh.lo = i;
    __syncthreads();
    const int at = sh.lo;
    __syncthreads();
    return at;
  }
  __device__ __forceinline__ uint32_t listed_key(int i) const {
    return listed_ok(i) ? (uint32_t)(sh.list[i] >> 32) : 0u;
  }

  // The key in bin `bin` of depth at which the running count (or weight) of the
  // bin, which has `held_there` of it, reaches `need`; what is left of `need` at
  // that key is returned.
  template <bool WEIGHTS>
  __device__ u64 refine(int bin, u64 held_there, u64 need, uint32_t* key) {
    // a bin's weights are known to 1.4%, and their roundings to whole numbers to
    // 1.3% where they are 40 or more: how many they are at most
    const float deep = kStep * (bin + 1);
    const float most = WEIGHTS ? (float)held_there * 0x1p-40f * __expf(deep) * 1.03f + 2.f
                               : (float)held_there;
    if (most <= kList && (!WEIGHTS || deep < 24.f)) {
      gather([&](float l, float depth) { return in(depth, bin) && above_cut(l); });
      if (rank == 0) {
        const int n = (int)min(sh.listed, (uint32_t)kList);
        run_over(n, [&](int i) { return WEIGHTS ? weight_of(logit_of<T>(listed_key(i))) : 1ull; });
        const int at = min(reaches(n, need), n - 1);
        // back to the first of this key
        if (threadIdx.x == 0) {
          int first_equal = at;
          while (first_equal > 0 && listed_key(first_equal - 1) == listed_key(at)) --first_equal;
          const u64 left = need - (first_equal ? sh.weights[first_equal - 1] : 0);
          for (uint32_t r = 0; r < ranks; ++r) {
            set_remote64(&sh.found[0], r, listed_key(at));
            set_remote64(&sh.found[1], r, left);
          }
        }
      }
      tc::cluster_sync();
      *key = (uint32_t)sh.found[0];
      return sh.found[1];
    }
    // many, of few keys as a rule: by digits of the keys
    uint32_t prefix = 0;
    int left = kKeyBits<T>;
    while (left > 0) {
      const int bits = left < 11 ? left : 11;
      const uint32_t mask = (1u << bits) - 1;
      clear(WEIGHTS ? 3 : 1);
      each_weighted([&](float l, int, float depth) {
        if (!in(depth, bin)) return;
        const uint32_t k = key_of<T>(l);
        if (k <= cut || (left < kKeyBits<T> && k >> left != prefix)) return;
        const int b = (int)(mask - (k >> (left - bits) & mask));  // larger keys first
        if (WEIGHTS) add(b, weight_of(l));
        else count(b);
      });
      int at;
      u64 before, held_now;
      const u64 wanted = need;
      find<WEIGHTS>([&](u64) { return wanted; }, &at, &need, &before, &held_now);
      need -= before;
      prefix = prefix << bits | (mask - (uint32_t)at);
      left -= bits;
    }
    *key = prefix;
    return need;
  }

  // ---- the two cuts ----
  // Few logits are left by top-k (the first `count` of the ranking hold it): rank 0
  // does the rest alone.  The answer's index, or -1, in rank 0.
  struct Answer {
    int token;
    float logit;
    u64 total;
  };
  __device__ Answer finish(int count, u64 k, float top_p, u64 least, float u) {
    int n = (int)min((u64)count, k);
    u64 total = run_over(n, [&](int i) { return weight_of(logit_of<T>(listed_key(i))); });
    if (top_p < 1.f) {
      if (threadIdx.x == 0) sh.found[0] = share_of(top_p, total);
      __syncthreads();
      const u64 need = sh.found[0];
      __syncthreads();
      n = min(n, reaches(n, need) + 1);
    }
    if (least) {  // weights fall: those from some place on are out
      if (threadIdx.x == 0) sh.hi = n;
      __syncthreads();
      for (int i = threadIdx.x; i < n; i += THREADS)
        if (sh.weights[i] - (i ? sh.weights[i - 1] : 0) < least) atomicMin(&sh.hi, i);
      __syncthreads();
      n = min(n, sh.hi);
    }
    total = sh.weights[n - 1];
    __syncthreads();
    // by index, their order for the choice
    for (int i = threadIdx.x; i < n; i += THREADS) {
      const u64 e = sh.list[i];
      sh.list[i] = e << 32 | e >> 32;
    }
    __syncthreads();
    sort(n);
    run_over(n, [&](int i) { return weight_of(logit_of<T>((uint32_t)sh.list[i])); });
    if (threadIdx.x == 0) {
      const u64 at = (u64)((double)u * (double)total);
      sh.found[0] = (at >= total ? total - 1 : at) + 1;
    }
    __syncthreads();
    const int at = min(reaches(n, sh.found[0]), n - 1);
    const u64 e = sh.list[at];
    return {(int)~(uint32_t)(e >> 32), logit_of<T>((uint32_t)e), total};
  }
  __device__ __forceinline__ static u64 share_of(float p, u64 total) {
    const double want = ceil((double)p * (double)total);
    return want < 1.0 ? 1 : (u64)want;
  }

  // True if few logits hold the first k: they are in rank 0's list then.
  __device__ bool top_k(u64 k, int* few) {
    clear(1);
    each_weighted([&](float, int, float depth) { count((int)depth); });
    int bin;
    u64 need, before, held_there;
    if (!find<false>([&](u64) { return k; }, &bin, &need, &before, &held_there)) return false;  // fewer have a weight at all
    if (before + held_there <= kList) {
      *few = (int)(before + held_there);
      gather([&](float, float depth) { return depth < bin + 1; });
      return true;
    }
    uint32_t key;
    ties = refine<false>(bin, held_there, k - before, &key);
    cut = key;
    return false;
  }
  __device__ void top_p(float p) {
    clear(3);
    each_weighted([&](float l, int, float depth) {
      if (above_cut(l)) add((int)depth, weight_of(l));
    });
    const u64 tie = ties ? weight_of(logit_of<T>(cut)) : 0, tied = ties * tie;
    int bin;
    u64 need, before, held_there;
    if (!find<true>([&](u64 all) { return share_of(p, all + tied); }, &bin, &need, &before,
                    &held_there)) {
      // the cut stays at the key of the first one, with as many of that key as it takes
      if (tie) {
        const u64 over = remote_sum(&sh.slot[slots - 1][0], ranks);
        ties = min(ties, (need - over + tie - 1) / tie);
      }
      return;
    }
    uint32_t key;
    need = refine<true>(bin, held_there, need - before, &key);
    const u64 w = weight_of(logit_of<T>(key));
    cut = key;
    ties = w ? (need + w - 1) / w : 0;
  }
};

template <typename T, int THREADS, bool HELD>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS)
sample_kernel(const T* logits, const Sample s, int* status) {
  extern __shared__ __align__(16) uint8_t raw[];
  auto& sh = *reinterpret_cast<Shared<THREADS>*>(raw);
  Row<T, THREADS, HELD> r(sh);
  r.held = reinterpret_cast<uint4*>(raw + sizeof(Shared<THREADS>));
  r.ranks = cluster_size();
  r.rank = tc::pair_rank();
  const int64_t n = blockIdx.x / r.ranks;
  if (threadIdx.x < 64) sh.roots[threadIdx.x] = kRoots[threadIdx.x];
  admit_successor();
  after_predecessor();

  const float temperature = s.cfg.temperatures ? s.cfg.temperatures[n] : s.cfg.temperature;
  const float top_p = s.cfg.top_ps ? s.cfg.top_ps[n] : s.cfg.top_p;
  const float min_p = s.cfg.min_ps ? s.cfg.min_ps[n] : s.cfg.min_p;
  const int top_k = s.cfg.top_ks ? s.cfg.top_ks[n] : s.cfg.top_k;
  const float u = s.u[n];
  const T* row = logits + n * s.stride;
  r.shift = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
  r.row = row - r.shift;
  r.end = r.shift + s.vocab;
  r.vocab = s.vocab;
  r.status = status;
  if (!SOMA_CHECK(n < s.rows && (int)(r.ranks * s.part) >= r.end, status)) return;  // the cluster
  const int part_end = min(r.end, (int)(r.rank + 1) * s.part);
  const int each = each_of(s.part, THREADS);
  r.first = (int)r.rank * s.part + (int)threadIdx.x * each;
  r.stop = min(r.first + each, part_end);

  // the largest logit, as an ordered number; NaN above all
  uint32_t own_top = 0;
  const auto upper = [&](float l, int) {
    const uint32_t b = __float_as_uint(__fadd_rn(l, 0.f));
    const uint32_t k = isnan(l) ? 0xffffffffu : (b >> 31 ? ~b : b | 0x80000000u);
    own_top = max(own_top, k);
  };
  if (HELD) r.first_pass(upper);
  else r.each(upper);
  const u64 top = r.largest(own_top);
  const uint32_t lowest = ~0xff800000u;  // of -infinity
  const bool nothing = top <= lowest;
  const bool bad = top >= (0x7f800000u | 0x80000000u) || !(temperature >= 0.f) || isnan(top_p) ||
                   isnan(min_p) || !(u >= 0.f && u < 1.f);
  if (bad || nothing) {  // the whole cluster
    if (r.rank == 0 && threadIdx.x == 0) {
      s.tokens[n] = -1;
      if (s.logprobs) s.logprobs[n] = NAN;
      if (bad) atomicCAS(status, 0, SOMA_ERR_NONFINITE);
    }
    tc::cluster_sync();
    return;
  }
  r.max = __uint_as_float(top >> 31 ? (uint32_t)top & 0x7fffffffu : ~(uint32_t)top);

  if (temperature < kLeastTemperature) {
    u64 at = 0;  // the first of the largest: the largest of 2^32 - index
    r.each([&](float l, int i) {
      if (l == r.max) at = max(at, (1ull << 32) - (u64)i);
    });
    at = r.largest(at);
    if (r.rank == 0 && threadIdx.x == 0) {
      s.tokens[n] = (int64_t)((1ull << 32) - at) - r.shift;
      if (s.logprobs) s.logprobs[n] = 0.f;
    }
    tc::cluster_sync();
    return;
  }

  if (threadIdx.x == 0) {
    const double inv = 1.0 / (double)fminf(temperature, kMostTemperature);
    const float hi = (float)inv;
    sh.inv = make_float2(hi, (float)(inv - (double)hi));
  }
  __syncthreads();
  r.inv2 = sh.inv;
  r.inv = r.inv2.x;
  const auto logprob = [&](float l, u64 total) {
    return (float)(((double)l - (double)r.max) / (double)fminf(temperature, kMostTemperature) -
                   log((double)total * 0x1p-40));
  };
  const u64 least = min_p > 0.f ? (u64)ceil((double)fminf(min_p, 1.f) * 0x1p40) : 0;
  int few;
  if (top_k > 0 && top_k < s.vocab && r.top_k((u64)top_k, &few)) {
    if (r.rank == 0) {
      const auto a = r.finish(few, (u64)top_k, top_p, least, u);
      if (threadIdx.x == 0) {
        s.tokens[n] = a.token - r.shift;
        if (s.logprobs) s.logprobs[n] = logprob(a.logit, a.total);
      }
    }
    return;  // the others' last access to its memory was before its last meeting
  }
  if (top_p < 1.f) r.top_p(top_p);

  // what remains, in the order of the indexes
  const u64 tie = r.ties ? r.weight_of(logit_of<T>(r.cut)) : 0;
  const bool tied = r.ties && tie >= least;
  u64 own = 0, equal = 0;
  r.each_weighted([&](float l, int, float) {
    const uint32_t k = key_of<T>(l);
    if (k > r.cut) {
      const u64 w = r.weight_of(l);
      if (w >= least) own += w;
    } else if (tied && k == r.cut) {
      ++equal;
    }
  });
  // equal ones before this thread's, in the CTA and in the CTAs before it
  u64 all;
  u64 room = 0;
  if (tied) {
    u64 equal_before = r.before_me(equal, sh.part[0], &all);
    if (threadIdx.x == 0 && r.slot_ok()) sh.slot[r.slots][0] = all;
    tc::cluster_sync();
    equal_before += r.remote_sum(&sh.slot[r.slots][0], r.rank);
    room = r.ties > equal_before ? r.ties - equal_before : 0;
    own += min(room, equal) * tie;
  }
  u64 before = r.before_me(own, sh.part[1], &all);
  if (threadIdx.x == 0 && r.slot_ok()) sh.slot[r.slots][1] = all;
  tc::cluster_sync();
  before += r.remote_sum(&sh.slot[r.slots][1], r.rank);
  const u64 total = r.remote_sum(&sh.slot[r.slots][1], r.ranks);
  u64 at = (u64)((double)u * (double)total);
  if (at >= total) at = total - 1;
  if (at >= before && at - before < own) {
    // the token is this thread's
    u64 run = before;
    int token = -1;
    float chosen = 0.f;
    r.each_weighted([&](float l, int i, float) {
      if (token >= 0) return;
      const uint32_t k = key_of<T>(l);
      u64 w = 0;
      if (k > r.cut) {
        w = r.weight_of(l);
        if (w < least) w = 0;
      } else if (k == r.cut && room) {
        w = tie;
        --room;
      }
      run += w;
      if (run > at) {
        token = i - r.shift;
        chosen = l;
      }
    });
    s.tokens[n] = token;
    if (s.logprobs) s.logprobs[n] = logprob(chosen, total);
  }
  tc::cluster_sync();  // no CTA leaves while another may read its sums
}

// Logits of one of n CTAs; `before`: elements that may come before a row's first
// one, as rows are read from 16-byte boundaries.
int part_of(int64_t vocab, int before, int n) {
  return (int)(((vocab + before + n - 1) / n + 7) / 8 * 8);
}

// CTAs of a row: as many as hold its logits in shared memory; twice as many while
// that leaves SMs idle and each 2048 logits or more.
int cluster_of(int64_t rows, int64_t vocab, int before) {
  int n = 1;
  while (n < kMaxCluster && (each_of(part_of(vocab, before, n), 512) > kHeld ||
                             (rows * n < 152 && vocab / (2 * n) >= 2048)))
    n *= 2;
  return n;
}

template <typename T, int THREADS, bool HELD>
cudaError_t launch(const void* logits, Sample s, int n, int* status, cudaStream_t st) {
  constexpr int most = sizeof(Shared<THREADS>) + (HELD ? THREADS * kHeld * sizeof(T) : 0);
  const cudaError_t e = allow_shared<sample_kernel<T, THREADS, HELD>>(most);
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)n;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(s.rows * n));
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = most;
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, sample_kernel<T, THREADS, HELD>, static_cast<const T*>(logits), (const Sample)s, status);
}

bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

template <typename T>
cudaError_t run(const void* logits, Sample s, int* status, cudaStream_t st) {
  constexpr int piece = 16 / sizeof(T);
  const int before = aligned(logits, 16) && (s.rows == 1 || s.stride % piece == 0) ? 0 : piece - 1;
  const bool few = s.vocab <= 2048;
  const int n = few ? 1 : cluster_of(s.rows, s.vocab, before);
  s.part = part_of(s.vocab, before, n);
  if (few) return launch<T, 128, true>(logits, s, n, status, st);
  return each_of(s.part, 512) <= kHeld ? launch<T, 512, true>(logits, s, n, status, st)
                                       : launch<T, 512, false>(logits, s, n, status, st);
}


}  // namespace
}  // namespace soma

using namespace soma;

extern "C" int soma_sample(const void* logits, int64_t stride, int dtype, int64_t rows,
                           int64_t vocab, soma_sample_config cfg, const float* u, int64_t* tokens,
                           float* logprobs, void* stream) {
  if (rows < 0 || rows > (1 << 24) || vocab < 1 || vocab > kMostVocab)
    return SOMA_ERR_UNSUPPORTED;
  if (dtype != SOMA_FP32 && dtype != SOMA_BF16 && dtype != SOMA_FP16) return SOMA_ERR_INVALID_ARG;
  if (stride < vocab || !aligned(logits, dtype == SOMA_FP32 ? 4 : 2) || !aligned(u, 4) ||
      !aligned(tokens, 8) || !aligned(logprobs, 4) || !aligned(cfg.temperatures, 4) ||
      !aligned(cfg.top_ps, 4) || !aligned(cfg.min_ps, 4) || !aligned(cfg.top_ks, 4) ||
      (!cfg.temperatures && !(cfg.temperature >= 0.f)) ||
      (!cfg.top_ps && std::isnan(cfg.top_p)) || (!cfg.min_ps && std::isnan(cfg.min_p)))
    return SOMA_ERR_INVALID_ARG;
  if (rows == 0) return SOMA_OK;
  if (!logits || !u || !tokens) return SOMA_ERR_INVALID_ARG;
  int* status = status_ptr();
  if (!status) return SOMA_ERR_CUDA;
  Sample s = {};
  s.stride = stride;
  s.rows = rows;
  s.vocab = (int32_t)vocab;
  s.cfg = cfg;
  s.u = u;
  s.tokens = tokens;
  s.logprobs = logprobs;
  const cudaStream_t st = (cudaStream_t)stream;
  trace_begin(SOMA_TRACE_SAMPLE, st);
  const cudaError_t e = dtype == SOMA_FP32   ? run<float>(logits, s, status, st)
                        : dtype == SOMA_BF16 ? run<__nv_bfloat16>(logits, s, status, st)
                                             : run<__half>(logits, s, status, st);
  trace_end(SOMA_TRACE_SAMPLE, st);
  return e == cudaSuccess ? SOMA_OK : SOMA_ERR_CUDA;
}
