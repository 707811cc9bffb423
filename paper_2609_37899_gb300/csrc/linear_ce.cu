// linear_ce.cu -- linear cross entropy and its gradients in pieces of the
// vocabulary (soma_linear_ce_* in include/soma_api.h have the formulas).
//
// Every product is a tcgen05 one of 128 x 256 tiles: a persistent kernel whose
// CTAs copy operand tiles with TMA into a ring of shared-memory stages,
// multiply them into one of two accumulators in tensor memory, and read the
// other one back in the epilogue.  What differs is the epilogue:
//   stats  h emb^T        per row the running maximum and sum of the exponentials
//                         over a range of the vocabulary, and the target's logit
//   grad   h emb^T        G of one piece of the vocabulary, in 16 bits
//   dh     G emb          added to fp32 sums over the pieces
//   demb   G^T h          the piece's rows of demb
#include <cmath>

#define SOMA_CHECK_FILE 10
#include "checked.cuh"
#include "numeric.cuh"
#include "soma_api.h"
#include "soma_launch.h"
#include "tc_tiles.cuh"

namespace soma {

bool make_tile_map(CUtensorMap* map, const void* base, bool bf16, int64_t rows, int64_t cols,
                   int64_t stride, int box_rows) {
  using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*,
                              const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                              const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                              CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  static const Encode encode = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault,
                                         &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess)
      f = nullptr;
    return reinterpret_cast<Encode>(f);
  }();
  if (!encode) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)stride * 2};
  const cuuint32_t box[2] = {(cuuint32_t)tc::kBoxCols, (cuuint32_t)box_rows};
  const cuuint32_t step[2] = {1, 1};
  return encode(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2,
                const_cast<void*>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

namespace {

constexpr int kSms = 152;
constexpr int kM = 128, kN = 256;             // one accumulator tile
constexpr int kStages = 4;
constexpr uint32_t kABytes = kM * 128, kBBytes = kN * 128;
constexpr uint32_t kStageBytes = kABytes + kBBytes;
constexpr int kEpilogueWarps = 8;
constexpr int kThreads = 128 + 32 * kEpilogueWarps;
constexpr size_t kSmem = kStages * kStageBytes + 1024;  // and what aligns the stages
constexpr size_t kPieceBytes = (size_t)256 << 20;       // of G of one piece
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

enum Kind { kStats, kGrad, kDh, kDemb };
__host__ __device__ constexpr bool a_mn(int kind) { return kind == kDemb; }
__host__ __device__ constexpr bool b_mn(int kind) { return kind == kDh || kind == kDemb; }

// What a row of the backward call takes part with; y = -1: no part.
struct RowInfo {
  float lse2, g;  // lse in powers of two, the scaled gradient of the loss
  int64_t y;
};

// One launch.  Stats: unit (m, split) covers the n tiles of the split.  Grad
// and demb: a unit is one tile.  Dh: the depth of all tiles laid end to end is
// cut into equal shares, one per CTA; a tile that several CTAs share is summed
// in as many slots.
struct Work {
  int32_t m_tiles, n_tiles, k_stages, splits;
  int32_t ctas;
  int64_t M, N;               // rows and columns that exist
  int32_t x_a, y_a, x_b, y_b; // first column or row of the operands' depth-free axis (pieces)
  // stats
  const int64_t* targets;
  float2* partial;            // [2 splits][M]: maximum (powers of two), sum
  float* own;                 // [M] logit of the target
  // grad
  const RowInfo* info;
  void* out;                  // G, or demb
  int64_t out_stride;
  int64_t v0;                 // first vocabulary entry of the piece
  int32_t vec;                // rows of out allow 16-byte stores
  // dh
  float* acc;                 // [slots][M][N4]
  int64_t acc_stride, slot_stride;
  int32_t add;                // add to acc instead of writing it
  const float* top;           // largest |dloss|
};

__device__ __forceinline__ int64_t share_start(int64_t c, int64_t total, int64_t ctas) {
  return c * total / ctas;
}
// The CTA whose share holds depth stage x.
__host__ __device__ __forceinline__ int64_t share_owner(int64_t x, int64_t total, int64_t ctas) {
  return ((x + 1) * ctas - 1) / total;
}

// A stretch of one CTA's work: stages [k0, k1) of tile (m, n).
struct Span {
  int32_t m, n, k0, k1;
};

// The spans of CTA `cta` in order.
template <int KIND>
struct Walk {
  const Work& w;
  int64_t at, end;
  int32_t n, n_end;

  __device__ Walk(const Work& work, int cta) : w(work) {
    if (KIND == kDh) {
      const int64_t total = (int64_t)w.m_tiles * w.n_tiles * w.k_stages;
      at = share_start(cta, total, w.ctas);
      end = share_start(cta + 1, total, w.ctas);
    } else {
      at = cta;
      end = (int64_t)w.m_tiles * (KIND == kStats ? w.splits : w.n_tiles);
    }
    n = n_end = 0;
  }
  // first / last: whether the span begins / ends a unit (stats)
  __device__ bool next(Span& s, bool& first, bool& last) {
    if (KIND == kDh) {
      if (at >= end) return false;
      const int64_t tile = at / w.k_stages;
      s.n = (int32_t)(tile % w.n_tiles);
      s.m = (int32_t)(tile / w.n_tiles);
      s.k0 = (int32_t)(at - tile * w.k_stages);
      const int64_t left = end - at;
      s.k1 = left < w.k_stages - s.k0 ? (int32_t)(s.k0 + left) : w.k_stages;
      at += s.k1 - s.k0;
      first = last = true;
      return true;
    }
    s.k0 = 0;
    s.k1 = w.k_stages;
    if (KIND == kStats) {
      first = n == n_end;
      if (first) {
        if (at >= end) return false;
        const int64_t split = at / w.m_tiles;
        n = (int32_t)(split * w.n_tiles / w.splits);
        n_end = (int32_t)((split + 1) * w.n_tiles / w.splits);
      }
      s.m = (int32_t)(at % w.m_tiles);
      s.n = n++;
      last = n == n_end;
      if (last) at += w.ctas;
      return true;
    }
    if (at >= end) return false;
    if (KIND == kGrad) {  // CTAs that run together share columns of emb
      s.m = (int32_t)(at % w.m_tiles);
      s.n = (int32_t)(at / w.m_tiles);
    } else {              // ... columns of G
      s.n = (int32_t)(at % w.n_tiles);
      s.m = (int32_t)(at / w.n_tiles);
    }
    at += w.ctas;
    first = last = true;
    return true;
  }
  __device__ int64_t unit_split() const { return (at - w.ctas) / w.m_tiles; }  // after `last`
};

// The power of two that the 16-bit G is scaled by.
template <typename T>
__device__ __forceinline__ float g_scale(float) { return 1.f; }
template <>
__device__ __forceinline__ float g_scale<__half>(float top) {
  int e = 0;
  frexpf(top, &e);  // top in [2^(e-1), 2^e)
  return top > 0.f ? exp2f((float)(14 - e)) : 1.f;
}

struct Shared {
  uint64_t full[kStages], empty[kStages], acc_full[2], acc_empty[2], done;
  uint32_t tmem;
  volatile int abort;
};

// A bounded wait; on running out it records the timeout and raises the CTA's
// abort flag.
__device__ __forceinline__ bool wait_or_abort(uint64_t* bar, uint32_t parity, Shared* sh,
                                              int* status, uint32_t max_polls = 1u << 22) {
  if (sh->abort) return false;
  if (tc::mbar_wait(bar, parity, max_polls)) return true;
  sh->abort = 1;
  atomicCAS(status, 0, SOMA_ERR_TIMEOUT);
  return false;
}

template <typename T>
__device__ __forceinline__ void store16(T* p, const float (&x)[32], int from) {
  float a[8];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
#pragma unroll
    for (int j = 0; j < 8; ++j) a[j] = x[from + 8 * h + j];
    store8(p + 8 * h, a);
  }
}

template <int KIND, typename T>
__global__ void __launch_bounds__(kThreads, 1)
product_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
               const __grid_constant__ Work w, int* status) {
  extern __shared__ uint8_t raw[];
  __shared__ Shared sh;
  uint8_t* stages = raw + (1024 - (tc::smem_u32(raw) & 1023)) % 1024;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;

  if (warp == 0 && lane == 0) {
    for (int i = 0; i < kStages; ++i) {
      tc::mbar_init(&sh.full[i], 1);
      tc::mbar_init(&sh.empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      tc::mbar_init(&sh.acc_full[i], 1);
      tc::mbar_init(&sh.acc_empty[i], kEpilogueWarps);
    }
    tc::mbar_init(&sh.done, 1);
    tc::mbar_fence_init();
    sh.abort = 0;
    tc::prefetch_map(&map_a);
    tc::prefetch_map(&map_b);
  }
  if (warp == 2) tc::tmem_alloc(&sh.tmem, 512);
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem = sh.tmem;

  Walk<KIND> walk(w, blockIdx.x);
  Span s;
  bool first, last;

  if (warp == 0) {
    // loader
    if (lane == 0) {
      uint32_t it = 0;
      bool ok = true;
      while (ok && walk.next(s, first, last)) {
        for (int k = s.k0; k < s.k1; ++k, ++it) {
          const uint32_t slot = it % kStages, round = it / kStages;
          if (!wait_or_abort(&sh.empty[slot], (round & 1) ^ 1, &sh, status)) {
            ok = false;
            break;
          }
          uint8_t* a = stages + slot * kStageBytes;
          uint8_t* b = a + kABytes;
          uint64_t* bar = &sh.full[slot];
          tc::mbar_arrive_expect_tx(bar, kStageBytes);
          if (a_mn(KIND)) {
            for (int j = 0; j < kM / 64; ++j)
              tc::tile_g2s(a + j * tc::kBoxBytes, &map_a, w.x_a + s.m * kM + j * 64,
                           w.y_a + k * tc::kDepth, bar);
          } else {
            tc::tile_g2s(a, &map_a, w.x_a + k * tc::kDepth, w.y_a + s.m * kM, bar);
          }
          if (b_mn(KIND)) {
            for (int j = 0; j < kN / 64; ++j)
              tc::tile_g2s(b + j * tc::kBoxBytes, &map_b, w.x_b + s.n * kN + j * 64,
                           w.y_b + k * tc::kDepth, bar);
          } else {
            tc::tile_g2s(b, &map_b, w.x_b + k * tc::kDepth, w.y_b + s.n * kN, bar);
          }
        }
      }
      // an aborting CTA leaves only after its copies have landed
      if (!ok)
        for (uint32_t j = it > kStages ? it - kStages : 0; j < it; ++j)
          tc::mbar_wait(&sh.full[j % kStages], (j / kStages) & 1);
    }
  } else if (warp == 1) {
    // MMA issuer: the whole warp waits, one elected thread issues
    constexpr uint32_t idesc = tc::idesc_16(kM, kN, sizeof(T) == 2 && !std::is_same<T, __half>::value,
                                            a_mn(KIND), b_mn(KIND));
    uint32_t it = 0, n_acc = 0;
    bool ok = true;
    while (ok && walk.next(s, first, last)) {
      const uint32_t buf = n_acc & 1;
      if (!wait_or_abort(&sh.acc_empty[buf], ((n_acc >> 1) & 1) ^ 1, &sh, status)) break;
      tc::tc_fence_after();
      const uint32_t d = tmem + buf * kN;
      for (int k = s.k0; k < s.k1; ++k, ++it) {
        const uint32_t slot = it % kStages;
        if (!wait_or_abort(&sh.full[slot], (it / kStages) & 1, &sh, status)) {
          ok = false;
          break;
        }
        tc::tc_fence_after();
        const uint32_t a = tc::smem_u32(stages + slot * kStageBytes);
        const uint32_t a_lo = tc::desc_lo(a, a_mn(KIND));
        const uint32_t b_lo = tc::desc_lo(a + kABytes, b_mn(KIND));
        if (tc::elect_one()) {
#pragma unroll
          for (int j = 0; j < tc::kDepth / 16; ++j)
            tc::mma_f16_ss_lohi(d, a_lo + j * tc::desc_step(a_mn(KIND)), tc::kDescHi,
                                b_lo + j * tc::desc_step(b_mn(KIND)), tc::kDescHi, idesc,
                                k > s.k0 || j > 0);
          tc::mma_commit(&sh.empty[slot]);
        }
        __syncwarp();
      }
      if (ok && tc::elect_one()) tc::mma_commit(&sh.acc_full[buf]);
      __syncwarp();
      ++n_acc;
    }
    if (tc::elect_one()) tc::mma_commit(&sh.done);
    __syncwarp();
    if (!tc::mbar_wait(&sh.done, 0)) atomicCAS(status, 0, SOMA_ERR_TIMEOUT);
  } else if (warp >= 4) {
    // epilogue: warp w reads lane quarter w % 4 (a warp can read no other) and
    // columns half (w - 4) / 4; a thread has one row
    const int quarter = warp % 4, half = (warp - 4) / 4;
    const int row = quarter * 32 + lane;
    uint32_t n_acc = 0;
    float top = -INFINITY, sum = 0.f;  // stats
    int64_t y = -1;
    RowInfo info = {0.f, 0.f, -1};
    float scale = 1.f;
    if (KIND == kGrad) scale = g_scale<T>(*w.top);
    if (KIND == kDemb) scale = 1.f / g_scale<T>(*w.top);
    while (walk.next(s, first, last)) {
      const int64_t m = (int64_t)s.m * kM + row;
      const bool live = m < w.M;
      if (KIND == kStats && first) {
        top = -INFINITY;
        sum = 0.f;
        y = live ? w.targets[m] : -1;
      }
      if (KIND == kGrad) {
        info = {0.f, 0.f, -1};
        if (live) info = w.info[m];
      }
      const uint32_t buf = n_acc & 1;
      // a tile's whole depth may lie before this: allow it more time
      if (!wait_or_abort(&sh.acc_full[buf], (n_acc >> 1) & 1, &sh, status, 1u << 27)) break;
      tc::tc_fence_after();
      const uint32_t src = tmem + buf * kN + half * (kN / 2) + ((uint32_t)(quarter * 32) << 16);
      const int64_t n0 = (int64_t)s.n * kN + half * (kN / 2);
      for (int c = 0; c < kN / 2; c += 32) {
        float x[32];
        tc::tmem_ld32_nowait(src + c, x);
        tc::tmem_wait_ld();
        const int64_t n = n0 + c;
        if (n >= w.N) continue;  // columns that do not exist (the whole warp)
        if (KIND == kStats) {
          const int64_t hit = y - n;
          if (hit >= 0 && hit < 32) {
            float v = 0.f;
#pragma unroll
            for (int j = 0; j < 32; ++j) v = j == hit ? x[j] : v;
            if (y < w.N) w.own[m] = v;
          }
          if (n + 32 > w.N) {
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (n + j >= w.N) x[j] = -INFINITY;
          }
          float mx = x[0];
#pragma unroll
          for (int j = 1; j < 32; ++j) mx = fmaxf(mx, x[j]);
          const float now = fmaxf(top, mx * kLog2e);
          const float ref = now == -INFINITY ? 0.f : now;
          float t = 0.f;
#pragma unroll
          for (int j = 0; j < 32; ++j) t += tc::ex2(fmaf(x[j], kLog2e, -ref));
          sum = fmaf(sum, tc::ex2(top - ref), t);
          top = now;
        } else if (KIND == kGrad) {
          const int64_t hit = info.y - w.v0 - n;
          const float g = info.y >= 0 ? scale * info.g : 0.f;
#pragma unroll
          for (int j = 0; j < 32; ++j) {
            const float p = tc::ex2(fmaf(x[j], kLog2e, -info.lse2));
            x[j] = info.y >= 0 && n + j < w.N ? g * (p - (j == hit ? 1.f : 0.f)) : 0.f;
          }
          if (live) {
            T* p = static_cast<T*>(w.out) + m * w.out_stride + n;
            store16(p, x, 0);
            store16(p + 16, x, 16);
          }
        } else if (KIND == kDemb) {
          if (live) {
            T* p = static_cast<T*>(w.out) + m * w.out_stride + n;
#pragma unroll
            for (int j = 0; j < 32; ++j) x[j] *= scale;
            if (w.vec && n + 32 <= w.N) {
              store16(p, x, 0);
              store16(p + 16, x, 16);
            } else {
#pragma unroll
              for (int j = 0; j < 32; ++j)
                if (n + j < w.N) p[j] = from_f32<T>(x[j]);
            }
          }
        } else {
          const int64_t tile = (int64_t)s.m * w.n_tiles + s.n;
          const int64_t slot =
              blockIdx.x - share_owner(tile * w.k_stages,
                                       (int64_t)w.m_tiles * w.n_tiles * w.k_stages, w.ctas);
          if (live) {
            float4* p = reinterpret_cast<float4*>(w.acc + slot * w.slot_stride +
                                                  m * w.acc_stride + n);
#pragma unroll
            for (int j = 0; j < 8; ++j)
              if (n + 4 * j < w.acc_stride) {
                float4 v = make_float4(x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3]);
                if (w.add) {
                  const float4 o = p[j];
                  v = make_float4(v.x + o.x, v.y + o.y, v.z + o.z, v.w + o.w);
                }
                p[j] = v;
              }
          }
        }
      }
      tc::tc_fence_before();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&sh.acc_empty[buf]);
      ++n_acc;
      if (KIND == kStats && last && live)
        w.partial[(walk.unit_split() * 2 + half) * w.M + m] = make_float2(top, sum);
    }
  }
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  if (warp == 2) tc::tmem_dealloc(tmem, 512);
}

// Joins a row's partial statistics: one warp per row.
__global__ void __launch_bounds__(256)
join_kernel(const float2* partial, int parts, const float* own, const int64_t* targets,
            int64_t ignore, int64_t rows, int64_t vocab, float* loss, float* lse, int* status) {
  const int64_t n = (int64_t)blockIdx.x * 8 + threadIdx.x / 32;
  if (n >= rows) return;
  const int lane = threadIdx.x % 32;
  float top = -INFINITY, sum = 0.f;
  for (int j = lane; j < parts; j += 32) {
    const float2 p = partial[(int64_t)j * rows + n];
    const float now = fmaxf(top, p.x), ref = now == -INFINITY ? 0.f : now;
    sum = sum * tc::ex2(top - ref) + p.y * tc::ex2(p.x - ref);
    top = now;
  }
#pragma unroll
  for (int k = 16; k; k >>= 1) {
    const float ot = __shfl_xor_sync(0xffffffffu, top, k);
    const float os = __shfl_xor_sync(0xffffffffu, sum, k);
    const float now = fmaxf(top, ot), ref = now == -INFINITY ? 0.f : now;
    // the same two terms on both sides of the exchange: commutative, so the
    // order is the same in every lane
    sum = sum * tc::ex2(top - ref) + os * tc::ex2(ot - ref);
    top = now;
  }
  if (lane) return;
  const int64_t y = targets[n];
  if (y == ignore) {
    loss[n] = lse[n] = 0.f;
    return;
  }
  const float l = fmaf(top, kLn2, logf(sum));
  const float r = y >= 0 && y < vocab ? l - own[n] : NAN;
  lse[n] = l;
  loss[n] = isfinite(r) ? r : NAN;
  if (!isfinite(r)) atomicCAS(status, 0, SOMA_ERR_NONFINITE);
}

// Per row: what it takes part with, and a copy of h in rows of a multiple of
// eight elements with the rows that take no part zeroed (their h may hold
// anything, and 0 * NaN would reach demb).
template <typename T>
__global__ void __launch_bounds__(128)
rows_kernel(const T* h, int64_t hs, int64_t dim, const int64_t* targets, int64_t ignore,
            int64_t vocab, const float* lse, const float* dloss, RowInfo* info, T* copy,
            int64_t cs, float* top) {
  const int64_t n = blockIdx.x;
  const int64_t y = targets[n];
  const float l = lse[n];
  const bool live = y != ignore && y >= 0 && y < vocab && isfinite(l);
  if (threadIdx.x == 0) {
    const float g = live ? dloss[n] : 0.f;
    info[n] = {l * kLog2e, g, live ? y : -1};
    // non-negative floats order as their bits do
    if (top && isfinite(g)) atomicMax(reinterpret_cast<int*>(top), __float_as_int(fabsf(g)));
  }
  const bool vec = hs % 8 == 0;
  for (int64_t j = threadIdx.x * 8; j < cs; j += 128 * 8) {
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (live) {
      if (vec && j + 8 <= dim) {
        v = *reinterpret_cast<const uint4*>(h + n * hs + j);
      } else {
        T t[8];
        for (int k = 0; k < 8; ++k) t[k] = j + k < dim ? h[n * hs + j + k] : from_f32<T>(0.f);
        memcpy(&v, t, 16);
      }
    }
    *reinterpret_cast<uint4*>(copy + n * cs + j) = v;
  }
}

// A matrix whose row stride is no multiple of eight, copied to rows that are.
template <typename T>
__global__ void __launch_bounds__(128)
pack_kernel(const T* x, int64_t xs, int64_t dim, T* copy, int64_t cs) {
  const int64_t n = blockIdx.x;
  for (int64_t j = threadIdx.x; j < cs; j += 128)
    copy[n * cs + j] = j < dim ? x[n * xs + j] : from_f32<T>(0.f);
}

// dh from the fp32 sums: the slots of a row's tile in order.
template <typename T>
__global__ void __launch_bounds__(128)
dh_kernel(const float* acc, int64_t acc_stride, int64_t slot_stride, int slots, int per_tile,
          Work w, int64_t dim, const RowInfo* info, const float* top, T* dh, int64_t ds) {
  const int64_t n = blockIdx.x;
  const bool live = info[n].y >= 0;
  const float unscale = 1.f / g_scale<T>(*top);
  const int64_t total = (int64_t)w.m_tiles * w.n_tiles * w.k_stages;
  for (int64_t j = threadIdx.x; j < dim; j += 128) {
    int used = slots;
    if (per_tile) {  // one piece: only the slots that its tile has were written
      const int64_t tile = n / kM * w.n_tiles + j / kN;
      used = (int)(share_owner((tile + 1) * w.k_stages - 1, total, w.ctas) -
                   share_owner(tile * w.k_stages, total, w.ctas)) + 1;
    }
    float x = 0.f;
    if (live)
      for (int k = 0; k < used; ++k) x += acc[k * slot_stride + n * acc_stride + j];
    dh[n * ds + j] = from_f32<T>(x * unscale);
  }
}

// ------------------------------------------------------------------- host --

size_t round256(size_t x) { return (x + 255) / 256 * 256; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
int64_t round8(int64_t x) { return (x + 7) / 8 * 8; }

bool dims_ok(const soma_linear_ce_dims& d) {
  return d.rows >= 0 && d.rows <= (1 << 30) && d.vocab >= 1 && d.vocab <= (1 << 30) &&
         d.dim >= 1 && d.dim <= 65536 && d.h_stride >= d.dim && d.emb_stride >= d.dim &&
         d.h_stride <= ((int64_t)1 << 32) && d.emb_stride <= ((int64_t)1 << 32) &&
         (d.dtype == SOMA_BF16 || d.dtype == SOMA_FP16);
}

struct Plan {
  int32_t splits;              // forward
  int64_t piece;               // backward: vocabulary entries of one piece
  int64_t g_stride, acc_stride, slots;
  size_t h, emb, partial, own; // offsets; h, emb: copies (emb only where its stride asks for it)
  size_t g, info, acc, top, total;
};

// Shares of the depth of dh's tiles.
void share_plan(const soma_linear_ce_dims& d, int64_t width, Work* w) {
  w->m_tiles = (int32_t)ceil_div(d.rows, kM);
  w->n_tiles = (int32_t)ceil_div(d.dim, kN);
  w->k_stages = (int32_t)ceil_div(width, tc::kDepth);
  const int64_t total = (int64_t)w->m_tiles * w->n_tiles * w->k_stages;
  w->ctas = (int32_t)(total < kSms ? total : kSms);
}

// Slots that a tile can need: its depth touches at most this many shares.
int64_t slots_of(const Work& w) {
  const int64_t total = (int64_t)w.m_tiles * w.n_tiles * w.k_stages;
  const int64_t share = total / w.ctas;
  const int64_t n = ceil_div(w.k_stages, share) + 1;
  return n < w.ctas ? n : w.ctas;
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
  if (backward || d.h_stride % 8) p.h = take((size_t)rows * round8(d.dim) * 2);
  if (d.emb_stride % 8) p.emb = take((size_t)d.vocab * round8(d.dim) * 2);
  const int64_t mt = ceil_div(rows, kM), vt = ceil_div(d.vocab, kN);
  if (!backward) {
    // rounds of CTAs times the tiles of a unit, least first
    int64_t best = INT64_MAX;
    for (int64_t s = 1; s <= vt && s <= 4 * kSms; ++s) {
      const int64_t cost = ceil_div(mt * s, kSms) * ceil_div(vt, s);
      if (cost < best) {
        best = cost;
        p.splits = (int32_t)s;
      }
    }
    p.partial = take((size_t)rows * 2 * p.splits * sizeof(float2));
    p.own = take((size_t)rows * 4);
  } else {
    p.piece = (int64_t)(kPieceBytes / 2) / rows / kN * kN;
    if (p.piece < kN) p.piece = kN;
    if (p.piece > d.vocab) p.piece = d.vocab;
    p.g_stride = ceil_div(p.piece, kN) * kN;
    p.acc_stride = ceil_div(d.dim, 4) * 4;
    p.g = take((size_t)rows * p.g_stride * 2);
    p.info = take((size_t)rows * sizeof(RowInfo));
    soma_linear_ce_dims one = d;
    one.rows = rows;
    Work w = {};
    for (int64_t width : {p.piece, d.vocab - (d.vocab - 1) / p.piece * p.piece}) {
      share_plan(one, width, &w);
      const int64_t n = slots_of(w);
      if (n > p.slots) p.slots = n;
    }
    p.acc = take((size_t)p.slots * rows * p.acc_stride * 4);
    p.top = take(4);
  }
  p.total = at;
  return p;
}

bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

template <int KIND, typename T>
cudaError_t launch(const CUtensorMap& a, const CUtensorMap& b, Work w, int64_t units, int* status,
                   cudaStream_t st) {
  const cudaError_t ready = cudaFuncSetAttribute(
      product_kernel<KIND, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem);
  if (ready != cudaSuccess) return ready;
  if (KIND != kDh) w.ctas = (int32_t)(units < kSms ? units : kSms);
  product_kernel<KIND, T><<<w.ctas, kThreads, kSmem, st>>>(a, b, w, status);
  return cudaGetLastError();
}

template <typename T>
constexpr bool is_bf16() { return !std::is_same<T, __half>::value; }

template <typename T>
cudaError_t forward(const T* h, const T* emb, const soma_linear_ce_dims& d, const int64_t* targets,
                    int64_t ignore, float* loss, float* lse, uint8_t* ws, int* status,
                    cudaStream_t st) {
  const Plan p = plan(d, false);
  int64_t hs = d.h_stride, es = d.emb_stride;
  if (hs % 8) {
    T* copy = reinterpret_cast<T*>(ws + p.h);
    pack_kernel<T><<<(unsigned)d.rows, 128, 0, st>>>(h, hs, d.dim, copy, round8(d.dim));
    h = copy;
    hs = round8(d.dim);
  }
  if (es % 8) {
    T* copy = reinterpret_cast<T*>(ws + p.emb);
    pack_kernel<T><<<(unsigned)d.vocab, 128, 0, st>>>(emb, es, d.dim, copy, round8(d.dim));
    emb = copy;
    es = round8(d.dim);
  }
  CUtensorMap ma, mb;
  if (!make_tile_map(&ma, h, is_bf16<T>(), d.rows, d.dim, hs, kM) ||
      !make_tile_map(&mb, emb, is_bf16<T>(), d.vocab, d.dim, es, kN))
    return cudaErrorInvalidValue;
  Work w = {};
  w.m_tiles = (int32_t)ceil_div(d.rows, kM);
  w.n_tiles = (int32_t)ceil_div(d.vocab, kN);
  w.k_stages = (int32_t)ceil_div(d.dim, tc::kDepth);
  w.splits = p.splits;
  w.M = d.rows;
  w.N = d.vocab;
  w.targets = targets;
  w.partial = reinterpret_cast<float2*>(ws + p.partial);
  w.own = reinterpret_cast<float*>(ws + p.own);
  const cudaError_t e =
      launch<kStats, T>(ma, mb, w, (int64_t)w.m_tiles * w.splits, status, st);
  if (e != cudaSuccess) return e;
  join_kernel<<<(unsigned)ceil_div(d.rows, 8), 256, 0, st>>>(w.partial, 2 * p.splits, w.own,
                                                             targets, ignore, d.rows, d.vocab,
                                                             loss, lse, status);
  return cudaGetLastError();
}

template <typename T>
cudaError_t backward(const T* h, const T* emb, const soma_linear_ce_dims& d,
                     const int64_t* targets, int64_t ignore, const float* lse, const float* dloss,
                     T* dh, int64_t dhs, T* demb, int64_t des, uint8_t* ws, int* status,
                     cudaStream_t st) {
  if (d.rows == 0)
    return cudaMemset2DAsync(demb, des * 2, 0, d.dim * 2, d.vocab, st);
  const Plan p = plan(d, true);
  RowInfo* info = reinterpret_cast<RowInfo*>(ws + p.info);
  T* copy = reinterpret_cast<T*>(ws + p.h);
  T* G = reinterpret_cast<T*>(ws + p.g);
  float* top = reinterpret_cast<float*>(ws + p.top);
  float* acc = reinterpret_cast<float*>(ws + p.acc);
  const int64_t cs = round8(d.dim);
  int64_t es = d.emb_stride;
  cudaError_t e = cudaMemsetAsync(top, 0, 4, st);
  if (e != cudaSuccess) return e;
  rows_kernel<T><<<(unsigned)d.rows, 128, 0, st>>>(h, d.h_stride, d.dim, targets, ignore, d.vocab,
                                                   lse, dloss, info, copy, cs,
                                                   is_bf16<T>() ? nullptr : top);
  if (es % 8) {
    T* packed = reinterpret_cast<T*>(ws + p.emb);
    pack_kernel<T><<<(unsigned)d.vocab, 128, 0, st>>>(emb, es, d.dim, packed, cs);
    emb = packed;
    es = cs;
  }
  const bool many = p.piece < d.vocab;
  if (many) {
    e = cudaMemsetAsync(acc, 0, (size_t)p.slots * d.rows * p.acc_stride * 4, st);
    if (e != cudaSuccess) return e;
  }
  CUtensorMap h_k, h_mn, e_k, e_mn;
  if (!make_tile_map(&h_k, copy, is_bf16<T>(), d.rows, d.dim, cs, kM) ||
      !make_tile_map(&h_mn, copy, is_bf16<T>(), d.rows, d.dim, cs, 64) ||
      !make_tile_map(&e_k, emb, is_bf16<T>(), d.vocab, d.dim, es, kN) ||
      !make_tile_map(&e_mn, emb, is_bf16<T>(), d.vocab, d.dim, es, 64))
    return cudaErrorInvalidValue;
  Work dhw = {};
  for (int64_t v0 = 0; v0 < d.vocab; v0 += p.piece) {
    const int64_t width = d.vocab - v0 < p.piece ? d.vocab - v0 : p.piece;
    CUtensorMap g_k, g_mn;
    if (!make_tile_map(&g_k, G, is_bf16<T>(), d.rows, width, p.g_stride, kM) ||
        !make_tile_map(&g_mn, G, is_bf16<T>(), d.rows, width, p.g_stride, 64))
      return cudaErrorInvalidValue;
    Work w = {};
    w.m_tiles = (int32_t)ceil_div(d.rows, kM);
    w.n_tiles = (int32_t)ceil_div(width, kN);
    w.k_stages = (int32_t)ceil_div(d.dim, tc::kDepth);
    w.M = d.rows;
    w.N = width;
    w.y_b = (int32_t)v0;
    w.info = info;
    w.out = G;
    w.out_stride = p.g_stride;
    w.v0 = v0;
    w.top = top;
    e = launch<kGrad, T>(h_k, e_k, w, (int64_t)w.m_tiles * w.n_tiles, status, st);
    if (e != cudaSuccess) return e;

    w = {};
    share_plan(d, width, &w);
    w.M = d.rows;
    w.N = d.dim;
    w.y_b = (int32_t)v0;
    w.acc = acc;
    w.acc_stride = p.acc_stride;
    w.slot_stride = d.rows * p.acc_stride;
    w.add = many;
    w.top = top;
    dhw = w;
    e = launch<kDh, T>(g_k, e_mn, w, 0, status, st);
    if (e != cudaSuccess) return e;

    w = {};
    w.m_tiles = (int32_t)ceil_div(width, kM);
    w.n_tiles = (int32_t)ceil_div(d.dim, kN);
    w.k_stages = (int32_t)ceil_div(d.rows, tc::kDepth);
    w.M = width;
    w.N = d.dim;
    w.out = demb + v0 * des;
    w.out_stride = des;
    w.vec = des % 8 == 0 && aligned(demb, 16);
    w.top = top;
    e = launch<kDemb, T>(g_mn, h_mn, w, (int64_t)w.m_tiles * w.n_tiles, status, st);
    if (e != cudaSuccess) return e;
  }
  dh_kernel<T><<<(unsigned)d.rows, 128, 0, st>>>(acc, p.acc_stride, d.rows * p.acc_stride,
                                                 (int)p.slots, !many, dhw, d.dim, info, top, dh,
                                                 dhs);
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
  int* status = status_ptr();
  if (!status) return SOMA_ERR_CUDA;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  const cudaStream_t st = (cudaStream_t)stream;
  trace_begin(SOMA_TRACE_HEAD, st);
  const cudaError_t e =
      d.dtype == SOMA_BF16
          ? backward(static_cast<const __nv_bfloat16*>(h), static_cast<const __nv_bfloat16*>(emb),
                     d, targets, ignore_index, lse, dloss, static_cast<__nv_bfloat16*>(dh),
                     dh_stride, static_cast<__nv_bfloat16*>(demb), demb_stride, ws, status, st)
          : backward(static_cast<const __half*>(h), static_cast<const __half*>(emb), d, targets,
                     ignore_index, lse, dloss, static_cast<__half*>(dh), dh_stride,
                     static_cast<__half*>(demb), demb_stride, ws, status, st);
  trace_end(SOMA_TRACE_HEAD, st);
  return e == cudaSuccess ? SOMA_OK : SOMA_ERR_CUDA;
}

}  // extern "C"
