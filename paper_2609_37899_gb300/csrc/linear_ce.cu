// linear_ce.cu -- linear cross entropy and its gradients in pieces of the
// vocabulary (soma_linear_ce_* in include/soma_api.h have the formulas).
//
// Every product is a tcgen05 one of 256 x 256 tiles: a persistent kernel of
// CTA pairs that copy operand tiles with TMA into a ring of shared-memory
// stages, multiply them into one of two accumulators in tensor memory, and
// read the other one back in the epilogue.  What differs is the epilogue:
//   stats  h emb^T        per row the running maximum and sum of the exponentials
//                         over a range of the vocabulary, and the target's logit
//   grad   h emb^T        G of one piece of the vocabulary, in 16 bits
//   demb   G^T h          the piece's rows of demb
//   dh     G emb          the rows of dh, where one piece holds the vocabulary
//   demb_sums, dh_sums    fp32 sums over pieces, or over parts of the depth where
//                         there are too few tiles to occupy the GPU otherwise;
//                         sums_kernel rounds them
//
// The tensor cores bound large sizes: 16385 x 32768 x 1376 forward 865 us (1710
// TFLOP/s, the rate that the power limit lets a long run keep), 8192 x 131072 x
// 1024 forward and backward 5.6 ms (1575); the tensor pipe is 91% busy in stats
// and 77 to 80% in the others at 4096 x 65536 x 1024.  emb's bytes bound few
// rows (64 x 32768 x 960 forward: 18 us, 3.4 TB/s), the launches small sizes
// (8192 x 256 x 960 forward and backward: 63 us).
#include <atomic>
#include <cmath>

#define SOMA_CHECK_FILE 8
#include "checked.cuh"
#include "numeric.cuh"
#include "pdl.cuh"
#include "soma_api.h"
#include "soma_launch.h"
#include "tc_tiles.cuh"

namespace soma {

namespace {

constexpr int kPairs = 76;                    // CTA pairs that are resident: 152 SMs
constexpr int kTile = 256;                    // rows and columns of a pair's tile
constexpr int kHalf = 128;                    // rows of A, and of B, that one CTA stages
constexpr int kStages = 6;
constexpr uint32_t kOperandBytes = kHalf * 128;
constexpr uint32_t kStageBytes = 2 * kOperandBytes;
constexpr int kEpilogueWarps = 8;
constexpr uint32_t kOutBytes = 32 * 128;      // a warp's output box: 32 rows of 128 bytes
constexpr int kThreads = 128 + 32 * kEpilogueWarps;
constexpr size_t kSmem =                      // and what aligns the stages
    kStages * kStageBytes + kEpilogueWarps * kOutBytes + 1024;
// Of G of one piece, at most, while a piece has kTile vocabulary entries at
// least: above 524,288 rows G takes 512 bytes a row.  Smaller pieces would stay
// in the 129 MB L2 but make dh's sums and the launches more (8192 x 131072 x
// 1024, both calls: 6.4 ms at 48 MB, 5.6 at 96, 5.25 at 256, 5.5 at 512).
constexpr size_t kPieceBytes = (size_t)256 << 20;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

enum Kind { kStats, kGrad, kDemb, kDh, kDembSums, kDhSums };
__host__ __device__ constexpr bool a_mn(int kind) { return kind == kDemb || kind == kDembSums; }
__host__ __device__ constexpr bool b_mn(int kind) { return kind >= kDemb; }
__host__ __device__ constexpr bool sums(int kind) { return kind >= kDembSums; }
// demb's product reads nothing of dh's, which is launched right before it: it
// starts on the SMs that dh's last tiles leave and waits for dh's end at its own.
// What both read is complete by then, as dh's kernels admit their successor
// after their own wait (8192 x 256 x 960, dh's 128 tiles on 76 pairs: both calls
// 68 us where demb waits, 65 so).
__host__ __device__ constexpr bool is_demb(int kind) { return kind == kDemb || kind == kDembSums; }
// The successors of these rely on all that came before.
__host__ __device__ constexpr bool admits_late(int kind) {
  return kind == kDh || kind == kDhSums || kind == kStats;
}

// rows_kernel leaves the largest |dloss| of each of its blocks, and every
// epilogue warp of grad reads them all while its first products run.
constexpr int64_t kMostTops = 1024;

// What a row of the backward call takes part with; y = -1: no part.  The
// entry of G at the target is by far the row's largest, and its rounding to 16
// bits would be most of dh's error: what the rounding took off is kept, and dh
// gets it back times the target's row of emb.
struct __align__(16) RowInfo {
  float lse2;  // lse in powers of two
  float g;     // gradient of the loss
  float rest;  // p - 1 of the target, by fp32 multiply-adds (rows_kernel); from
               // grad on, what its rounding took off the (scaled) entry of G
  int32_t y;
};

// One launch.  Stats: unit (m, split) covers the n tiles of the split.  Grad
// and demb: a unit is one tile.  Sums: `columns` pairs form a group that works
// on the same rows and depth, one n tile each (then n + columns, ...); the
// depth of all m tiles laid end to end is cut into equal shares, one per
// group, and a tile that several groups share is summed in as many slots.
struct Work {
  int32_t m_tiles, n_tiles, k_stages;
  int32_t tile_n;             // columns of a tile: kTile, or fewer (stats, grad)
  int32_t rows_a;             // rows of A's box; fewer than 128: the odd CTA has none
  int32_t splits;             // stats
  int32_t pairs;              // of the grid
  int32_t columns, groups;    // sums
  int64_t M, N;               // rows and columns that exist
  int32_t y_b;                // first row of B (the piece's place in emb)
  // stats
  const int64_t* targets;
  float2* partial;            // [M][2 splits]: maximum (powers of two), sum
  float* own;                 // [M] logit of the target
  int32_t low;                // grad: rows to where G's second half goes, or 0
  // grad, dh
  RowInfo* info;
  const void* emb;            // dh: 16-byte aligned rows of emb
  int64_t emb_stride;
  int64_t v0;                 // first vocabulary entry of the piece
  float* top;                 // largest |dloss|; after it those of rows_kernel's blocks
  int32_t tops;               // grad: how many
  // demb, dh: where its rows are not 16-byte aligned, or null; grad: G
  void* out;
  int64_t out_stride;
  // sums
  int32_t slot_rows;          // rows of one slot
  int32_t add;                // add to the sums instead of writing them
};

// The first depth stage of share g, and the share that holds stage x.
__host__ __device__ __forceinline__ int64_t share_start(int64_t g, int64_t total, int64_t groups) {
  return g * total / groups;
}
__host__ __device__ __forceinline__ int64_t share_owner(int64_t x, int64_t total, int64_t groups) {
  return ((x + 1) * groups - 1) / total;
}

// A stretch of one pair's work: stages [k0, k1) of tile (m, n).
struct Span {
  int32_t m, n, k0, k1;
  int32_t part;     // stats: the split; sums: the slot
  bool first, last; // stats: whether the span begins / ends its unit
};

// The spans of one pair in order; every warp role walks them by itself.
template <int KIND>
struct Walk {
  const Work& w;
  int64_t at, end;
  int32_t n, n_end;

  __device__ Walk(const Work& work, int pair) : w(work), n_end(0) {
    if (sums(KIND)) {
      const int64_t total = (int64_t)w.m_tiles * w.k_stages;
      const int g = pair / w.columns;
      at = share_start(g, total, w.groups);
      end = share_start(g + 1, total, w.groups);
      n = pair % w.columns;
    } else {
      at = pair;
      end = (int64_t)w.m_tiles * (KIND == kStats ? w.splits : w.n_tiles);
      n = 0;
    }
  }
  __device__ bool next(Span& s, int pair) {
    s.k0 = 0;
    s.k1 = w.k_stages;
    s.part = 0;
    if (sums(KIND)) {
      const int64_t total = (int64_t)w.m_tiles * w.k_stages;
      const int64_t g = pair / w.columns;
      if (at >= end) {  // the next n tile of this pair, from the share's start
        n += w.columns;
        at = share_start(g, total, w.groups);
      }
      if (n >= w.n_tiles || at >= end) return false;
      s.m = (int32_t)(at / w.k_stages);
      s.n = n;
      const int64_t begin = (int64_t)s.m * w.k_stages;
      s.k0 = (int32_t)(at - begin);
      if (end - at < w.k_stages - s.k0) s.k1 = (int32_t)(s.k0 + (end - at));
      s.part = (int32_t)(g - share_owner(begin, total, w.groups));
      at += s.k1 - s.k0;
    } else if (KIND == kStats) {
      s.first = n == n_end;
      if (s.first) {
        if (at >= end) return false;
        const int64_t split = at / w.m_tiles;
        n = (int32_t)(split * w.n_tiles / w.splits);
        n_end = (int32_t)((split + 1) * w.n_tiles / w.splits);
      }
      s.m = (int32_t)(at % w.m_tiles);
      s.n = n++;
      s.part = (int32_t)(at / w.m_tiles);
      s.last = n == n_end;
      if (s.last) at += w.pairs;
    } else {
      if (at >= end) return false;
      if (KIND == kGrad) {  // pairs that run together share rows of emb
        s.m = (int32_t)(at % w.m_tiles);
        s.n = (int32_t)(at / w.m_tiles);
      } else {              // ... the part of G
        s.n = (int32_t)(at % w.n_tiles);
        s.m = (int32_t)(at / w.n_tiles);
      }
      at += w.pairs;
    }
    return true;
  }
};

// What the 16-bit G is scaled by: the largest |dloss| becomes 1, or 2^14 in fp16.
// Most calls have one dloss for all rows; -dloss (1 - p) is then next to a power
// of two and exact for small p.  Without the scaling those entries were all off
// by the same up to 2^-8 of themselves in bf16, and demb with them (1.5 times
// the error that its own rounding has).  One scale serves all rows, as demb adds
// over them: in fp16 a row whose |dloss| is far below the largest has its small
// entries among the subnormals, 2^-39 of the largest |dloss| off at most.
template <typename T>
__device__ __forceinline__ float g_scale(float top) {
  const float to = std::is_same<T, __half>::value ? 16384.f : 1.f;
  return to / fminf(fmaxf(top, 0x1p-100f), 0x1p126f);
}

struct Shared {
  uint64_t full[kStages], empty[kStages], acc_full[2], acc_empty[2], done;
  uint32_t tmem;
  volatile int abort;
};

// A bounded wait of a whole warp, with one answer for all its lanes; on
// running out it records the timeout and raises the CTA's abort flag.
__device__ __forceinline__ bool wait_or_abort(uint64_t* bar, uint32_t parity, Shared* sh,
                                              int* status, uint32_t max_polls = 1u << 22) {
  const bool ok = !sh->abort && tc::mbar_wait(bar, parity, max_polls);
  if (__all_sync(0xffffffffu, ok)) return true;
  if (!sh->abort) atomicCAS(status, 0, SOMA_ERR_TIMEOUT);
  sh->abort = 1;
  return false;
}

// Eight elements from column j of a row of `dim`; zeros past its end.
template <typename T>
__device__ __forceinline__ uint4 row_piece(const T* row, int64_t j, int64_t dim, bool vec) {
  if (vec && j + 8 <= dim) return *reinterpret_cast<const uint4*>(row + j);
  union {
    T t[8];
    uint4 u;
  } v;
#pragma unroll
  for (int k = 0; k < 8; ++k) v.t[k] = j + k < dim ? row[j + k] : from_f32<T>(0.f);
  return v.u;
}

// One 128-byte row of a warp's output box: 16-byte piece j of row r lies at
// piece j ^ (r % 8), as the tiled store expects it.
__device__ __forceinline__ uint4* box_piece(uint8_t* box, int row, int j) {
  return reinterpret_cast<uint4*>(box + row * 128 + ((j ^ (row & 7)) << 4));
}

template <typename T>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  union {
    T t[2];
    uint32_t u;
  } w;
  w.t[0] = from_f32<T>(a);
  w.t[1] = from_f32<T>(b);
  return w.u;
}

// The first `cols` of 64 columns of a box's rows to memory that a tiled store
// cannot address: a warp writes a row at a time, a 4-byte word per lane.  Where
// a row starts between two words (odd), a lane's word is made of its own lower
// half and its neighbour's upper one, and the row's ends go by themselves.
template <typename T>
__device__ __forceinline__ void store_box(T* out, int64_t stride, uint8_t* box, int rows, int cols,
                                          int lane) {
  uint16_t* q = reinterpret_cast<uint16_t*>(out) + 2 * lane;  // this lane's first column
#pragma unroll 4
  for (int r = 0; r < rows; ++r, q += stride) {
    const uint32_t own =
        *reinterpret_cast<const uint32_t*>(reinterpret_cast<uint8_t*>(box_piece(box, r, lane / 4)) +
                                           (lane % 4) * 4);
    const uint32_t before = __shfl_up_sync(0xffffffffu, own, 1);
    const int odd = (int)(reinterpret_cast<uintptr_t>(q) >> 1) & 1;
    const int first = 2 * lane - odd, last = cols - 1;
    if (first >= 0 && first < last)
      *reinterpret_cast<uint32_t*>(q - odd) = odd ? __funnelshift_r(before, own, 16) : own;
    if (first < 0) q[0] = (uint16_t)own;
    if (((cols ^ odd) & 1) && lane == last / 2)
      q[last & 1] = (uint16_t)(last & 1 ? own >> 16 : own);
  }
}

template <int KIND, typename T>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
product_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
               const __grid_constant__ CUtensorMap map_out, const __grid_constant__ Work w,
               int* status) {
  extern __shared__ uint8_t raw[];
  __shared__ Shared sh;
  uint8_t* stages = raw + (1024 - (tc::smem_u32(raw) & 1023)) % 1024;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int pair = blockIdx.x / 2;
  const uint32_t rank = tc::pair_rank();

  if (warp == 0 && lane == 0) {
    for (int i = 0; i < kStages; ++i) {
      tc::mbar_init(&sh.full[i], 1);
      tc::mbar_init(&sh.empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      tc::mbar_init(&sh.acc_full[i], 1);
      tc::mbar_init(&sh.acc_empty[i], 2 * kEpilogueWarps);
    }
    tc::mbar_init(&sh.done, 1);
    tc::mbar_fence_init();
    sh.abort = 0;
    tc::prefetch_map(&map_a);
    tc::prefetch_map(&map_b);
    if (KIND != kStats) tc::prefetch_map(&map_out);
  }
  if (!admits_late(KIND)) admit_successor();
  if (warp == 2) tc::tmem_alloc_pair(&sh.tmem, 512);
  tc::tc_fence_before();
  __syncthreads();
  tc::cluster_sync();
  tc::tc_fence_after();
  if (!is_demb(KIND)) after_predecessor();
  if (admits_late(KIND)) admit_successor();
  const uint32_t tmem = sh.tmem;

  Walk<KIND> walk(w, pair);
  Span s;

  if (warp == 0) {
    // loader: lanes 0 and 1 copy this CTA's half of A, lanes 2 and 3 that of B,
    // in one instruction (boxes of several lanes are fetched at once, those of
    // consecutive instructions one after another).  A K-major half is one box
    // (two of 64 rows took 10% longer), an MN-major one two.  Both CTAs' bytes
    // count on the even CTA's barrier.
    const bool is_b = lane >= 2;
    const int sub = (lane & 1) * 64;
    const CUtensorMap* map = is_b ? &map_b : &map_a;
    const bool mn = is_b ? b_mn(KIND) : a_mn(KIND);
    // Few rows (K-major A): the box ends with them, as boxes that reach past a
    // matrix's end are slow, and the odd CTA copies none.  What the products
    // make of the stage's other rows is not read.
    const bool few = !a_mn(KIND) && w.rows_a < kHalf;
    const bool copies = lane < 4 && (mn || !sub) && !(few && !is_b && rank);
    const int half_n = w.tile_n / 2;  // rows of B that one CTA stages
    const uint32_t bytes = (few ? w.rows_a * 128 : 2 * kOperandBytes) + 2 * half_n * 128;
    const int y0 = is_b ? w.y_b : 0;
    uint32_t it = 0;
    bool ok = true;
    while (ok && walk.next(s, pair)) {
      const int r0 = (is_b ? s.n * w.tile_n + (int)rank * half_n
                           : s.m * kTile + (int)rank * kHalf) + sub;
      for (int k = s.k0; k < s.k1; ++k, ++it) {
        const uint32_t slot = it % kStages, round = it / kStages;
        if (!wait_or_abort(&sh.empty[slot], (round & 1) ^ 1, &sh, status)) {
          ok = false;
          break;
        }
        if (rank == 0 && lane == 0) tc::mbar_arrive_expect_tx(&sh.full[slot], bytes);
        __syncwarp();
        const int kx = k * tc::kDepth;
        // a box starts inside its matrix's tiles, on 16 bytes, and fits the stage
        if (copies &&
            SOMA_CHECK(r0 % 8 == 0 && r0 >= 0 && kx >= 0 && k < w.k_stages &&
                           s.m < w.m_tiles && s.n < w.n_tiles &&
                           slot * kStageBytes + lane * tc::kBoxBytes +
                                   (mn ? tc::kBoxBytes : kOperandBytes) <= kStages * kStageBytes,
                       status)) {
          tc::tile_g2s_pair(stages + slot * kStageBytes + lane * tc::kBoxBytes, map,
                            mn ? r0 : kx, y0 + (mn ? kx : r0), tc::leader_addr(&sh.full[slot]));
        }
      }
    }
    // an aborting CTA leaves only after its copies have landed (the even
    // CTA's barriers count both CTAs' copies)
    if (!ok && rank == 0)
      for (uint32_t j = it > kStages ? it - kStages : 0; j < it; ++j)
        tc::mbar_wait(&sh.full[j % kStages], (j / kStages) & 1);
  } else if (warp == 1 && rank == 0) {
    // MMA issuer of the pair: the whole warp waits, one elected thread issues
    const uint32_t idesc =
        tc::idesc_16(kTile, w.tile_n, !std::is_same<T, __half>::value, a_mn(KIND), b_mn(KIND));
    uint32_t it = 0, n_acc = 0;
    bool ok = true;
    while (ok && walk.next(s, pair)) {
      const uint32_t buf = n_acc & 1;
      if (!wait_or_abort(&sh.acc_empty[buf], ((n_acc >> 1) & 1) ^ 1, &sh, status)) break;
      tc::tc_fence_after();
      const uint32_t d = tmem + buf * kTile;
      for (int k = s.k0; k < s.k1; ++k, ++it) {
        const uint32_t slot = it % kStages;
        if (!wait_or_abort(&sh.full[slot], (it / kStages) & 1, &sh, status)) {
          ok = false;
          break;
        }
        tc::tc_fence_after();
        const uint32_t a = tc::smem_u32(stages + slot * kStageBytes);
        const uint32_t a_lo = tc::desc_lo(a, a_mn(KIND));
        const uint32_t b_lo = tc::desc_lo(a + kOperandBytes, b_mn(KIND));
        if (tc::elect_one() &&
            SOMA_CHECK(buf * kTile + w.tile_n <= 512 &&
                           (slot + 1) * kStageBytes <= kStages * kStageBytes,
                       status)) {
#pragma unroll
          for (int j = 0; j < tc::kDepth / 16; ++j)
            tc::mma_f16_ss_pair(d, a_lo + j * tc::desc_step(a_mn(KIND)),
                                b_lo + j * tc::desc_step(b_mn(KIND)), tc::kDescHi, idesc,
                                k > s.k0 || j > 0);
          tc::mma_commit_pair(&sh.empty[slot]);
        }
        __syncwarp();
      }
      if (ok && tc::elect_one()) tc::mma_commit_pair(&sh.acc_full[buf]);
      __syncwarp();
      ++n_acc;
    }
    if (tc::elect_one()) tc::mma_commit_pair(&sh.done);
    __syncwarp();
    if (!tc::mbar_wait(&sh.done, 0)) atomicCAS(status, 0, SOMA_ERR_TIMEOUT);
  } else if (warp >= 4) {
    // epilogue: warp w reads lane quarter w % 4 (a warp can read no other) and
    // columns half (w - 4) / 4; a thread has one row
    const int quarter = warp % 4, half = (warp - 4) / 4;
    const int m_in = (int)rank * kHalf + quarter * 32;  // the warp's first row in the tile
    uint8_t* box = stages + kStages * kStageBytes + (warp - 4) * kOutBytes;
    const uint32_t empty_bar[2] = {tc::leader_addr(&sh.acc_empty[0]),
                                   tc::leader_addr(&sh.acc_empty[1])};
    uint32_t n_acc = 0;
    float top = -INFINITY, sum = 0.f;  // stats
    int64_t y = -1;
    RowInfo info = {0.f, 0.f, 0.f, -1};
    float scale = 1.f;
    if (KIND == kGrad) {
      int largest = 0;  // non-negative floats order as their bits do
#pragma unroll 8
      for (int j = lane; j < w.tops; j += 32)
        largest = max(largest, __float_as_int(w.top[1 + j]));
      const float g = __int_as_float(__reduce_max_sync(0xffffffffu, largest));
      scale = g_scale<T>(g);
      if (blockIdx.x == 0 && warp == 4 && lane == 0) *w.top = g;  // for the kernels that follow
    }
    if (KIND == kDemb || KIND == kDh) scale = 1.f / g_scale<T>(__ldcg(w.top));
    while (walk.next(s, pair)) {
      const int64_t m0 = (int64_t)s.m * kTile + m_in, m = m0 + lane;
      const bool live = m < w.M;
      if (KIND == kStats && s.first) {
        top = -INFINITY;
        sum = 0.f;
        y = live && SOMA_CHECK(m >= 0, status) ? w.targets[m] : -1;
      }
      if (KIND == kGrad || KIND == kDh) {
        info = {0.f, 0.f, 0.f, -1};
        if (live) info = w.info[m];
      }
      // dh: the target's row of emb, 32 columns ahead of their use
      const T* e_row = nullptr;
      uint4 e_next[4];
      const auto fetch_e = [&](int64_t n) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          e_next[j] = make_uint4(0u, 0u, 0u, 0u);
          if (info.y >= 0 && n + 8 * j < w.N) e_next[j] = row_piece(e_row, n + 8 * j, w.N, true);
        }
      };
      if (KIND == kDh) {
        if (!SOMA_CHECK(info.y < (int64_t)w.k_stages * tc::kDepth, status)) info.y = -1;
        e_row = static_cast<const T*>(w.emb) + (info.y < 0 ? 0 : info.y) * w.emb_stride;
        fetch_e((int64_t)s.n * w.tile_n + half * (w.tile_n / 2));
      }
      const uint32_t buf = n_acc & 1;
      // a tile's whole depth may lie before this: allow it more time
      if (!wait_or_abort(&sh.acc_full[buf], (n_acc >> 1) & 1, &sh, status, 1u << 27)) break;
      tc::tc_fence_after();
      const int half_n = w.tile_n / 2;
      const uint32_t src = tmem + buf * kTile + half * half_n + ((uint32_t)(quarter * 32) << 16);
      const int64_t n0 = (int64_t)s.n * w.tile_n + half * half_n;
      const int64_t n_end = n0 + half_n < w.N ? n0 + half_n : w.N;
      // 32 columns at a time, the next ones on their way while these are used
      float next[32];
      if (n0 < n_end && m0 < w.M) tc::tmem_ld32_nowait(src, next);
#pragma unroll
      for (int c = 0; c < kHalf; c += 32) {
        const int64_t n = n0 + c;
        if (n >= n_end || m0 >= w.M) break;  // nothing there (the whole warp)
        if (!SOMA_CHECK(buf * kTile + half * half_n + c + 32 <= 512 && quarter * 32 + 32 <= 128,
                        status))
          break;
        tc::tmem_wait_ld32(next);
        float x[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) x[j] = next[j];
        if (c + 32 < kHalf && n + 32 < n_end) tc::tmem_ld32_nowait(src + c + 32, next);
        if (KIND == kStats) {
          const int64_t hit = y - n;
          if (hit >= 0 && hit < 32) {
            float v = 0.f;
#pragma unroll
            for (int j = 0; j < 32; ++j) v = j == hit ? x[j] : v;
            if (y < n_end && SOMA_CHECK(m >= 0 && m < w.M, status)) w.own[m] = v;
          }
          if (n + 32 > n_end) {
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (n + j >= n_end) x[j] = -INFINITY;
          }
          // four chains each: one would wait for itself
          float mx[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
          for (int j = 4; j < 32; ++j) mx[j % 4] = fmaxf(mx[j % 4], x[j]);
          const float now =
              fmaxf(top, fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * kLog2e);
          const float ref = now == -INFINITY ? 0.f : now;
          float t[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int j = 0; j < 32; ++j) t[j % 4] += tc::ex2(fmaf(x[j], kLog2e, -ref));
          sum = fmaf(sum, tc::ex2(top - ref), (t[0] + t[1]) + (t[2] + t[3]));
          top = now;
          continue;
        }
        if (KIND == kGrad) {
          if (info.y >= 0) {
            const int64_t hit = info.y - w.v0 - n;
            const float g = scale * info.g;
            if (hit >= 0 && hit < 32) {
              const int at = (int)hit;
              float rest = 0.f;
#pragma unroll
              for (int j = 0; j < 32; ++j) {
                const float p = tc::ex2(fmaf(x[j], kLog2e, -info.lse2));
                x[j] = g * (j == at ? info.rest : p);
                rest = j == at ? x[j] - to_f32(from_f32<T>(x[j])) : rest;
              }
              if (SOMA_CHECK(m >= 0 && m < w.M, status)) w.info[m].rest = rest;
            } else {
#pragma unroll
              for (int j = 0; j < 32; ++j) x[j] = g * tc::ex2(fmaf(x[j], kLog2e, -info.lse2));
            }
          } else {
#pragma unroll
            for (int j = 0; j < 32; ++j) x[j] = 0.f;
          }
        }
        if (KIND == kDemb) {
#pragma unroll
          for (int j = 0; j < 32; ++j) x[j] *= scale;
        }
        if (KIND == kDh) {
          uint4 e[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) e[j] = e_next[j];
          if (c + 32 < kHalf) fetch_e(n + 32);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            union {
              uint4 u;
              T t[8];
            } v;
            v.u = e[j];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              float& o = x[8 * j + k];
              o = info.y >= 0 ? scale * fmaf(info.rest, to_f32(v.t[k]), o) : 0.f;
            }
          }
        }
        if (KIND == kGrad && w.low) {
          // few rows: what the rounding takes off each entry, for demb, right away
          // (32 columns, 64 bytes a row, at a time)
          if (live) {
            T* q = static_cast<T*>(w.out) + (m + w.low) * w.out_stride + n;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              float rest[8];
#pragma unroll
              for (int k = 0; k < 8; ++k)
                rest[k] = x[8 * j + k] - to_f32(from_f32<T>(x[8 * j + k]));
              if (n + 8 * j < w.N &&
                  SOMA_CHECK(n + 8 * j + 8 <= w.out_stride && m < w.low, status))
                store8(q + 8 * j, rest);
            }
          }
        }
        if (sums(KIND) || c % 64 == 0) {  // the last box has been read before this is written
          if (lane == 0) tc::bulk_wait_read();
          __syncwarp();
        }
        if (sums(KIND)) {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            *box_piece(box, lane, j) =
                make_uint4(__float_as_uint(x[4 * j]), __float_as_uint(x[4 * j + 1]),
                           __float_as_uint(x[4 * j + 2]), __float_as_uint(x[4 * j + 3]));
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            *box_piece(box, lane, (c % 64) / 8 + j) =
                make_uint4(pack2<T>(x[8 * j], x[8 * j + 1]), pack2<T>(x[8 * j + 2], x[8 * j + 3]),
                           pack2<T>(x[8 * j + 4], x[8 * j + 5]),
                           pack2<T>(x[8 * j + 6], x[8 * j + 7]));
        }
        if (!sums(KIND) && c % 64 == 0 && n + 32 < n_end) continue;  // half a box so far
        const int bx = (int)(sums(KIND) ? n : n - c % 64);
        if (!sums(KIND) && KIND != kGrad && w.out) {
          __syncwarp();
          const int rows = w.M - m0 < 32 ? (int)(w.M - m0) : 32;
          const int cols = n_end - bx < 64 ? (int)(n_end - bx) : 64;
          if (!SOMA_CHECK(m0 >= 0 && rows >= 0 && m0 + rows <= w.M && bx >= 0 && cols >= 0 &&
                              bx + cols <= w.N,
                          status))
            continue;
          store_box(static_cast<T*>(w.out) + m0 * w.out_stride + bx, w.out_stride, box, rows, cols,
                    lane);
          __syncwarp();
          continue;
        }
        tc::fence_async_smem();
        __syncwarp();
        if (lane == 0 &&
            SOMA_CHECK(m0 >= 0 && m0 < w.M && bx >= 0 && bx < w.N && bx % 8 == 0 &&
                           (!sums(KIND) || (s.part >= 0 && s.part < w.groups)),
                       status)) {
          if (!sums(KIND)) tc::tile_s2g(&map_out, bx, (int)m0, box);
          else if (w.add) tc::tile_add_s2g(&map_out, bx, s.part * w.slot_rows + (int)m0, box);
          else tc::tile_s2g(&map_out, bx, s.part * w.slot_rows + (int)m0, box);
          tc::bulk_commit();
        }
      }
      tc::tc_fence_before();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive_cluster(empty_bar[buf]);
      ++n_acc;
      if (KIND == kStats && s.last && live &&
          SOMA_CHECK(m >= 0 && m < w.M && s.part >= 0 && s.part < w.splits, status))
        w.partial[m * 2 * w.splits + 2 * s.part + half] = make_float2(top, sum);
    }
    if (KIND != kStats && lane == 0) tc::bulk_wait();
  }
  __syncwarp();
  if (is_demb(KIND)) after_predecessor();
  tc::tc_fence_before();
  __syncthreads();
  tc::cluster_sync();  // no CTA leaves while its pair may still signal or read it
  tc::tc_fence_after();
  if (warp == 2) tc::tmem_dealloc_pair(tmem, 512);
}

// Joins a row's partial statistics: one warp per row.
//
// The tensor cores cut an fp32 sum off instead of rounding it, so a logit comes
// out short by about 1e-8 of itself for every 16 of its depth, several times
// that where its products are of one sign, as the target's are.  That matters
// for the target's, which is large and enters the loss twice (960 deep: the
// loss was off by 1.2e-6 of itself): it is computed here once more by fp32
// multiply-adds and takes the other one's place in the sum and in the loss.
// lse and the target's logit are several times the loss: their difference is
// taken before the small terms are added.
template <typename T>
__global__ void __launch_bounds__(256)
join_kernel(const float2* partial, int parts, const float* own, const T* h, int64_t hs,
            const T* emb, int64_t es, const int64_t* targets, int64_t ignore, int64_t rows,
            int64_t vocab, int64_t dim, float* loss, float* lse, int* status) {
  admit_successor();
  const int64_t n = (int64_t)blockIdx.x * 8 + threadIdx.x / 32;
  if (n >= rows) return;
  const int lane = threadIdx.x % 32;
  // the call's inputs are there since before stats: it admits this kernel after
  // its own wait, and CTAs that find room next to it compute this meanwhile
  // (from L2, where what earlier kernels wrote is)
  const int64_t y = __ldcg(reinterpret_cast<const long long*>(targets) + n);
  const bool has_target = y != ignore && y >= 0 && y < vocab &&
                          SOMA_CHECK(hs >= dim && es >= dim && hs % 8 == 0 && es % 8 == 0, status);
  float logit = 0.f;
  if (has_target) {
    const T* a = h + n * hs;
    const T* b = emb + y * es;
    const int64_t whole = dim / 8 * 8;
    for (int64_t j0 = lane * 8; j0 < whole; j0 += 1024) {
      union {
        uint4 u;
        T t[8];
      } p[4], q[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool there = j0 + 256 * i < whole;
        p[i].u = q[i].u = make_uint4(0u, 0u, 0u, 0u);
        if (there) p[i].u = __ldcg(reinterpret_cast<const uint4*>(a + j0 + 256 * i));
        if (there) q[i].u = __ldcg(reinterpret_cast<const uint4*>(b + j0 + 256 * i));
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int k = 0; k < 8; ++k) logit = fmaf(to_f32(p[i].t[k]), to_f32(q[i].t[k]), logit);
    }
    if (whole + lane < dim)
      logit = fmaf(to_f32(__ldcg(a + whole + lane)), to_f32(__ldcg(b + whole + lane)), logit);
#pragma unroll
    for (int k = 16; k; k >>= 1) logit += __shfl_xor_sync(0xffffffffu, logit, k);
  }
  after_predecessor();  // no CTA ends before stats has
  if (y == ignore) {
    if (lane == 0) loss[n] = lse[n] = 0.f;
    return;
  }
  constexpr int kAhead = 4;
  float2 ahead[kAhead];
#pragma unroll
  for (int i = 0; i < kAhead; ++i)
    ahead[i] = lane + 32 * i < parts ? partial[n * parts + lane + 32 * i]
                                     : make_float2(-INFINITY, 0.f);
  const float was = own[n];
  float top = ahead[0].x, sum = 0.f;
#pragma unroll
  for (int i = 1; i < kAhead; ++i) top = fmaxf(top, ahead[i].x);
  {
    const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) sum = fmaf(ahead[i].y, tc::ex2(ahead[i].x - ref), sum);
  }
#pragma unroll 4
  for (int j = lane + 32 * kAhead; j < parts; j += 32) {
    const float2 p = partial[n * parts + j];
    const float now = fmaxf(top, p.x), ref = now == -INFINITY ? 0.f : now;
    sum = sum * tc::ex2(top - ref) + p.y * tc::ex2(p.x - ref);
    top = now;
  }
#pragma unroll
  for (int k = 16; k; k >>= 1) {
    const float ot = __shfl_xor_sync(0xffffffffu, top, k);
    const float os = __shfl_xor_sync(0xffffffffu, sum, k);
    const float now = fmaxf(top, ot), ref = now == -INFINITY ? 0.f : now;
    sum = sum * tc::ex2(top - ref) + os * tc::ex2(ot - ref);
    top = now;
  }
  if (lane) return;
  if (has_target) {
    const float instead =
        tc::ex2(fmaf(logit, kLog2e, -top)) - tc::ex2(fmaf(was, kLog2e, -top));
    sum += instead;
  }
  const float hi = top * kLn2, lo = fmaf(top, kLn2, -hi) + logf(sum);
  const float r = has_target ? (hi - logit) + lo : NAN;
  lse[n] = hi + lo;
  loss[n] = isfinite(r) ? r : NAN;
  if (!isfinite(r)) atomicCAS(status, 0, SOMA_ERR_NONFINITE);
}

// Per row, one warp: what it takes part with, and a copy of h in rows of a
// multiple of 64 elements with the rows that take no part zeroed (their h
// may hold anything, and 0 * NaN would reach demb).
//
// The target's p - 1 is taken from the logit that is in lse, which is not the
// tensor cores' (join_kernel): that one is short by so much that a row sure of
// its target would get several times its gradient, always the same way (960
// deep at a logit of 22: p short by 5e-5 in bf16, 1.3e-4 in fp16, where the
// loss is 1.5e-5).
template <typename T>
__global__ void __launch_bounds__(256)
rows_kernel(const T* h, const T* emb, soma_linear_ce_dims d, const int64_t* targets, int64_t ignore,
            const float* lse, const float* dloss, RowInfo* info, T* copy, int64_t cs, int halves,
            float* top, int* status) {
  __shared__ int largest;
  if (threadIdx.x == 0) largest = 0;
  __syncthreads();
  admit_successor();
  after_predecessor();
  const int lane = threadIdx.x % 32;
  for (int64_t n = (int64_t)blockIdx.x * 8 + threadIdx.x / 32; n < d.rows; n += 8 * gridDim.x) {
    const int64_t y = targets[n];
    const float l = lse[n];
    const bool live = y != ignore && y >= 0 && y < d.vocab && isfinite(l);
    const bool vec = d.h_stride % 8 == 0, vec_e = d.emb_stride % 8 == 0;
    const T* e = emb + (live ? y : 0) * d.emb_stride;
    float logit = 0.f;
    for (int64_t j = lane * 8; j < cs; j += 256) {
      if (!SOMA_CHECK(j + 8 <= cs && n >= 0 && n < d.rows, status)) break;
      union {
        uint4 u;
        T t[8];
      } v, w;
      v.u = w.u = make_uint4(0u, 0u, 0u, 0u);
      if (live) {
        v.u = row_piece(h + n * d.h_stride, j, d.dim, vec);
        w.u = row_piece(e, j, d.dim, vec_e);
      }
      *reinterpret_cast<uint4*>(copy + n * cs + j) = v.u;
      if (halves == 2) *reinterpret_cast<uint4*>(copy + (d.rows + n) * cs + j) = v.u;
#pragma unroll
      for (int k = 0; k < 8; ++k) logit = fmaf(to_f32(v.t[k]), to_f32(w.t[k]), logit);
    }
#pragma unroll
    for (int k = 16; k; k >>= 1) logit += __shfl_xor_sync(0xffffffffu, logit, k);
    if (lane == 0) {
      RowInfo r = {l * kLog2e, 0.f, 0.f, -1};
      if (live) {
        r.rest = expm1f(logit - l);
        r.g = dloss[n];
        r.y = (int32_t)y;
        // non-negative floats order as their bits do
        if (isfinite(r.g)) atomicMax(&largest, __float_as_int(fabsf(r.g)));
      }
      info[n] = r;
    }
  }
  __syncthreads();
  if (threadIdx.x == 0 && SOMA_CHECK(blockIdx.x < kMostTops, status))
    top[1 + blockIdx.x] = __int_as_float(largest);
}

// A matrix copied to rows of cs elements, zeros after the first dim; eight
// elements per thread.
template <typename T>
__global__ void __launch_bounds__(256)
pack_kernel(const T* x, int64_t xs, int64_t rows, int64_t dim, T* copy, int64_t cs, int* status) {
  admit_successor();
  after_predecessor();
  const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  const int64_t n = at / cs, j = at - n * cs;
  if (n < rows && SOMA_CHECK(at >= 0 && at + 8 <= rows * cs && j + 8 <= cs, status))
    *reinterpret_cast<uint4*>(copy + at) = row_piece(x + n * xs, j, dim, xs % 8 == 0);
}

// The rows of dh (info) or demb (no info) from their fp32 sums, the slots in
// order.  used = 0: the slots that the row's tile has (w's shares).
template <typename T>
__global__ void __launch_bounds__(128)
sums_kernel(const float* acc, int64_t acc_stride, int used, const __grid_constant__ Work w,
            const RowInfo* info, T* out, int64_t stride, int vec, int* status) {
  after_predecessor();
  admit_successor();  // only now: the product of demb may follow
  const int64_t n = blockIdx.x;
  const float f = 1.f / g_scale<T>(*w.top);
  if (!used) {
    const int64_t total = (int64_t)w.m_tiles * w.k_stages, begin = n / kTile * w.k_stages;
    used = (int)(share_owner(begin + w.k_stages - 1, total, w.groups) -
                 share_owner(begin, total, w.groups)) + 1;
  }
  RowInfo r = {0.f, 0.f, 0.f, 0};
  if (info) r = info[n];
  const T* e = static_cast<const T*>(w.emb) + (r.y < 0 ? 0 : r.y) * w.emb_stride;
  const int64_t j = ((int64_t)blockIdx.y * 128 + threadIdx.x) * 4;
  if (!SOMA_CHECK(n < w.M && used >= 1 && used <= kPairs && (j >= w.N || j + 4 <= acc_stride),
                  status))
    return;
  if (j < w.N) {
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    if (r.y >= 0) {
#pragma unroll 8
      for (int k = 0; k < used; ++k) {
        const float4 v = *reinterpret_cast<const float4*>(
            acc + ((int64_t)k * w.slot_rows + n) * acc_stride + j);
        x = make_float4(x.x + v.x, x.y + v.y, x.z + v.z, x.w + v.w);
      }
      if (info) {
        float* o = &x.x;
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (j + k < w.N) o[k] = fmaf(r.rest, to_f32(e[j + k]), o[k]);
      }
    }
    T* p = out + n * stride + j;
    if (vec && j + 4 <= w.N) {
      *reinterpret_cast<uint2*>(p) = make_uint2(pack2<T>(x.x * f, x.y * f), pack2<T>(x.z * f, x.w * f));
    } else {
      const float v[4] = {x.x, x.y, x.z, x.w};
      for (int k = 0; k < 4 && j + k < w.N; ++k) p[k] = from_f32<T>(v[k] * f);
    }
  }
}

// ------------------------------------------------------------------- host --

size_t round256(size_t x) { return (x + 255) / 256 * 256; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
int64_t round8(int64_t x) { return (x + 7) / 8 * 8; }
int64_t round64(int64_t x) { return (x + 63) / 64 * 64; }

bool dims_ok(const soma_linear_ce_dims& d) {
  return d.rows >= 0 && d.rows <= (1 << 30) && d.vocab >= 1 && d.vocab <= (1 << 30) &&
         d.dim >= 1 && d.dim <= 65536 && d.h_stride >= d.dim && d.emb_stride >= d.dim &&
         d.h_stride <= ((int64_t)1 << 32) && d.emb_stride <= ((int64_t)1 << 32) &&
         (d.dtype == SOMA_BF16 || d.dtype == SOMA_FP16);
}

// Times of the backward call's parts, in units of a pair's stage (about 0.4 us
// at the rate of a large product): what a launch costs besides its stages, and
// the fp32 bytes that one unit reads or writes.
constexpr int64_t kLaunchStages = 18;
constexpr int64_t kBytesPerStage = 2700000;

// With no more rows than this, the rounding of G to 16 bits does not average
// out in demb (a row of it may be a single entry times a single state: its norm
// was off by up to 1.6 times what rounding the result costs).  G is stored in
// two halves then, what the rounding took off as further rows that meet h's
// rows once more.  demb is bound by its own bytes at such sizes.
constexpr int64_t kFewRows = 128;

// Rows of the boxes of a K-major A of M rows.
int box_rows(int64_t M) { return M <= kHalf - 8 ? (int)round8(M) : kHalf; }

// M x N sums over a depth, cut into shares.
Work shares(int64_t M, int64_t N, int64_t depth) {
  Work w = {};
  w.M = M;
  w.N = N;
  w.m_tiles = (int32_t)ceil_div(M, kTile);
  w.tile_n = kTile;
  w.rows_a = box_rows(M);
  w.n_tiles = (int32_t)ceil_div(N, kTile);
  w.k_stages = (int32_t)ceil_div(depth, tc::kDepth);
  w.columns = w.n_tiles < kPairs ? w.n_tiles : kPairs;
  const int64_t total = (int64_t)w.m_tiles * w.k_stages;
  w.groups = (int32_t)(total < kPairs / w.columns ? total : kPairs / w.columns);
  w.pairs = w.groups * w.columns;
  w.slot_rows = w.m_tiles * kTile;
  return w;
}

// Slots that a tile can need: its depth touches at most this many shares.
int64_t slots_of(const Work& w) {
  const int64_t share = (int64_t)w.m_tiles * w.k_stages / w.groups;
  const int64_t n = ceil_div(w.k_stages, share) + 1;
  return n < w.groups ? n : w.groups;
}

int64_t sums_cost(const Work& w, bool add) {
  const int64_t bytes = (int64_t)w.M * w.N * 4;
  return ceil_div((int64_t)w.m_tiles * w.k_stages, w.groups) * ceil_div(w.n_tiles, w.columns) +
         kLaunchStages + bytes * (add ? 2 : 1) / kBytesPerStage;
}
int64_t tiles_cost(int64_t M, int64_t N, int64_t depth) {
  return ceil_div(ceil_div(M, kTile) * ceil_div(N, kTile), kPairs) * ceil_div(depth, tc::kDepth) +
         kLaunchStages;
}

// Stats and grad take tiles of half the columns where those occupy the GPU
// better: 8192 x 256 x 960 is 32 whole tiles or 64 half ones for 76 pairs (grad
// 14 -> 12 us).  A half tile's stage takes 0.7 of a whole one's: its copies,
// half of which are A's, not its products.  Widths in between were tried where
// they divide the vocabulary evenly among the pairs (64 x 32768 in 147 tiles of
// 224) and were slower, 19.7 us against 18.4.
constexpr double kHalfTile = 0.7;

// Whether a matrix of `copied` rows is copied to rows of a multiple of 64
// elements before `rows` rows are multiplied by it: a stride that is no
// multiple of 8 cannot be read in boxes at all, and one that is no multiple of
// 16 puts a box's 128-byte rows across five 32-byte sectors, which makes the
// products take 1.35 times as long (3001 x 50021 x 680 forward: 182 us at a
// stride of 680 or 712, 133 us at 704).  The copy is worth its time (4 bytes
// per element moved) from about 2000 rows in the forward call, and a third of
// that in the backward call with its three products.
bool copied(int64_t stride, int64_t rows, bool backward) {
  return stride % 8 != 0 || (stride % 16 != 0 && rows >= (backward ? 700 : 2000));
}

// Blocks of rows_kernel.
unsigned row_blocks(const soma_linear_ce_dims& d) {
  const int64_t n = ceil_div(d.rows, 8);
  return (unsigned)(n < kMostTops ? n : kMostTops);
}

struct Plan {
  int32_t splits, tile_n;        // forward
  int64_t piece;                 // backward: vocabulary entries of one piece
  bool dh_sums, demb_sums;       // which kernels the products take
  int64_t halves;                // rows of G and of h's copy per row: 2 with G's second half
  int64_t g_stride, acc_stride, dh_slots, demb_slots;
  bool copy_h, copy_emb;
  size_t h, emb, partial, own;   // offsets; h, emb: copies
  size_t g, info, dh_acc, demb_acc, top, total;
  Gaps gaps;                     // of the checked build
};

// The backward call's pieces: as few as G's share of the workspace allows, or
// somewhat more where the tiles then fill the last round of pairs better.
void plan_pieces(const soma_linear_ce_dims& d, Plan* p) {
  int64_t most = (int64_t)(kPieceBytes / 2) / (d.rows * p->halves) / kTile * kTile;
  if (most < kTile) most = kTile;
  const int64_t fewest = ceil_div(d.vocab, most);
  int64_t best = INT64_MAX;
  // one piece has no sums over pieces, and then more would only add launches
  for (int64_t n = fewest; n < fewest + (fewest == 1 ? 1 : 24); ++n) {
    int64_t width = n == 1 ? d.vocab : ceil_div(ceil_div(d.vocab, n), kTile) * kTile;
    if (width > d.vocab) width = d.vocab;
    const int64_t full = d.vocab / width, rest = d.vocab % width;
    const bool one = full == 1 && !rest;
    int64_t cost = 0;
    bool dh_sums = true, demb_sums = false;
    for (int64_t w : {width, rest}) {
      if (!w) continue;
      const int64_t dh_by_sums =
          sums_cost(shares(d.rows, d.dim, w), !one) + (one ? kLaunchStages : 0);
      const int64_t dh_by_tiles = tiles_cost(d.rows, d.dim, w);
      int64_t demb = tiles_cost(w, d.dim, d.rows * p->halves);
      if (one) {
        dh_sums = dh_by_sums < dh_by_tiles;
        const int64_t by_sums =
            sums_cost(shares(w, d.dim, d.rows * p->halves), false) + kLaunchStages;
        demb_sums = by_sums < demb;
        if (demb_sums) demb = by_sums;
      }
      cost += (w == width ? full : 1) *
              (tiles_cost(d.rows, w, d.dim) + demb + (dh_sums ? dh_by_sums : dh_by_tiles));
    }
    if (cost < best) {
      best = cost;
      p->piece = width;
      p->dh_sums = dh_sums;
      p->demb_sums = demb_sums;
    }
    if (width == kTile) break;
  }
}

Plan plan(soma_linear_ce_dims d, bool backward) {
  Plan p = {};
  size_t at = 0;
  const auto take = [&](size_t bytes) {
    p.gaps.off[p.gaps.n++] = at;
    const size_t o = at + kGuard;
    at = o + round256(bytes);
    return o;
  };
  if (!d.rows) d.rows = 1;
  p.halves = backward && d.rows <= kFewRows ? 2 : 1;
  p.copy_h = backward || copied(d.h_stride, d.rows, false);
  p.copy_emb = copied(d.emb_stride, d.rows, backward);
  if (p.copy_h) p.h = take((size_t)d.rows * p.halves * round64(d.dim) * 2);
  if (p.copy_emb) p.emb = take((size_t)d.vocab * round64(d.dim) * 2);
  if (!backward) {
    // rounds of pairs times the tiles of a unit, least first
    const int64_t mt = ceil_div(d.rows, kTile);
    double best = 1e300;
    for (const int tile_n : {kTile, kTile / 2}) {
      const int64_t vt = ceil_div(d.vocab, tile_n);
      // as many splits as fit r rounds of the pairs
      for (int64_t r = ceil_div(mt, kPairs), tried = 0; tried < 64; ++r, ++tried) {
        const int64_t fit = r * kPairs / mt;
        const int64_t s = fit < vt ? fit : vt;
        if (tried && s > 4 * kPairs) break;
        const double cost =
            (double)(r * ceil_div(vt, s)) * (tile_n == kTile ? 1 : kHalfTile);
        if (cost < best * 0.995) {
          best = cost;
          p.splits = (int32_t)s;
          p.tile_n = tile_n;
        }
        if (s == vt) break;
      }
    }
    p.partial = take((size_t)d.rows * 2 * p.splits * sizeof(float2));
    p.own = take((size_t)d.rows * 4);
  } else {
    plan_pieces(d, &p);
    p.g_stride = round8(p.piece);
    p.acc_stride = ceil_div(d.dim, 4) * 4;
    p.g = take((size_t)d.rows * p.halves * p.g_stride * 2);
    p.info = take((size_t)d.rows * sizeof(RowInfo));
    if (p.dh_sums) {
      for (int64_t width : {p.piece, d.vocab % p.piece}) {
        if (!width) continue;
        const int64_t n = slots_of(shares(d.rows, d.dim, width));
        if (n > p.dh_slots) p.dh_slots = n;
      }
      p.dh_acc = take((size_t)p.dh_slots * ceil_div(d.rows, kTile) * kTile * p.acc_stride * 4);
    }
    if (p.demb_sums) {
      p.demb_slots = slots_of(shares(d.vocab, d.dim, d.rows * p.halves));
      p.demb_acc = take((size_t)p.demb_slots * ceil_div(d.vocab, kTile) * kTile * p.acc_stride * 4);
    }
    p.top = take((1 + kMostTops) * 4);
  }
  p.gaps.off[p.gaps.n++] = at;
  p.total = at + kGuard;
  return p;
}

bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

template <typename T>
constexpr int dtype_of() { return std::is_same<T, __half>::value ? SOMA_FP16 : SOMA_BF16; }

// x copied to rows of a multiple of 64 elements; *stride becomes theirs.
template <typename T>
const T* pack(const T* x, int64_t rows, int64_t dim, int64_t* stride, T* copy, int* status,
              cudaStream_t st) {
  const int64_t cs = round64(dim);
  const cudaError_t e = launch_overlapped(pack_kernel<T>, (unsigned)ceil_div(rows * cs, 256 * 8),
                                          256, 0, st, x, *stride, rows, dim, copy, cs, status);
  *stride = cs;
  return e == cudaSuccess ? copy : nullptr;
}

// A launch of `units` units, or of w.pairs pairs (sums).
template <int KIND, typename T>
cudaError_t launch(const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& out, Work w,
                   int64_t units, int* status, cudaStream_t st) {
  // the attribute stays with the kernel: asked for once per device
  static std::atomic<uint64_t> ready{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = dev < 64 ? (uint64_t)1 << dev : 0;
  if (!(ready.load(std::memory_order_relaxed) & bit) || !bit) {
    e = cudaFuncSetAttribute(product_kernel<KIND, T>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             (int)kSmem);
    if (e != cudaSuccess) return e;
    ready.fetch_or(bit, std::memory_order_relaxed);
  }
  if (!sums(KIND)) w.pairs = (int32_t)(units < kPairs ? units : kPairs);
  return launch_overlapped(product_kernel<KIND, T>, 2 * w.pairs, kThreads, kSmem, st, a, b, out, w,
                           status);
}

template <typename T>
cudaError_t forward(const Plan& p, const T* h, const T* emb, const soma_linear_ce_dims& d,
                    const int64_t* targets, int64_t ignore, float* loss, float* lse, uint8_t* ws,
                    int* status, cudaStream_t st) {
  int64_t hs = d.h_stride, es = d.emb_stride;
  if (p.copy_h) h = pack(h, d.rows, d.dim, &hs, reinterpret_cast<T*>(ws + p.h), status, st);
  if (p.copy_emb)
    emb = pack(emb, d.vocab, d.dim, &es, reinterpret_cast<T*>(ws + p.emb), status, st);
  if (!h || !emb) return cudaErrorLaunchFailure;
  CUtensorMap ma, mb;
  if (!make_tile_map(&ma, h, dtype_of<T>(), d.rows, d.dim, hs, box_rows(d.rows)) ||
      !make_tile_map(&mb, emb, dtype_of<T>(), d.vocab, d.dim, es, p.tile_n / 2))
    return cudaErrorInvalidValue;
  Work w = {};
  w.m_tiles = (int32_t)ceil_div(d.rows, kTile);
  w.tile_n = p.tile_n;
  w.rows_a = box_rows(d.rows);
  w.n_tiles = (int32_t)ceil_div(d.vocab, p.tile_n);
  w.k_stages = (int32_t)ceil_div(d.dim, tc::kDepth);
  w.splits = p.splits;
  w.M = d.rows;
  w.N = d.vocab;
  w.targets = targets;
  w.partial = reinterpret_cast<float2*>(ws + p.partial);
  w.own = reinterpret_cast<float*>(ws + p.own);
  const cudaError_t e =
      launch<kStats, T>(ma, mb, ma, w, (int64_t)w.m_tiles * w.splits, status, st);
  if (e != cudaSuccess) return e;
  return launch_overlapped(join_kernel<T>, (unsigned)ceil_div(d.rows, 8), 256, 0, st, w.partial,
                           2 * p.splits, w.own, h, hs, emb, es, targets, ignore, d.rows, d.vocab,
                           d.dim, loss, lse, status);
}

template <typename T>
cudaError_t backward(const Plan& p, const T* h, const T* emb, const soma_linear_ce_dims& d,
                     const int64_t* targets, int64_t ignore, const float* lse, const float* dloss,
                     T* dh, int64_t dhs, T* demb, int64_t des, uint8_t* ws, int* status,
                     cudaStream_t st) {
  if (d.rows == 0)
    return cudaMemset2DAsync(demb, des * 2, 0, d.dim * 2, d.vocab, st);
  constexpr int dtype = dtype_of<T>();
  RowInfo* info = reinterpret_cast<RowInfo*>(ws + p.info);
  T* copy = reinterpret_cast<T*>(ws + p.h);
  T* G = reinterpret_cast<T*>(ws + p.g);
  float* top = reinterpret_cast<float*>(ws + p.top);
  float* dh_acc = reinterpret_cast<float*>(ws + p.dh_acc);
  float* demb_acc = reinterpret_cast<float*>(ws + p.demb_acc);
  const int64_t cs = round64(d.dim);
  int64_t es = d.emb_stride;
  cudaError_t e = cudaSuccess;
  if (p.dh_sums && p.piece < d.vocab && e == cudaSuccess)
    e = cudaMemsetAsync(dh_acc, 0,
                        (size_t)p.dh_slots * ceil_div(d.rows, kTile) * kTile * p.acc_stride * 4, st);
  if (e == cudaSuccess)
    e = launch_overlapped(rows_kernel<T>, row_blocks(d), 256, 0, st, h, emb, d, targets, ignore,
                          lse, dloss, info, copy, cs, (int)p.halves, top, status);
  if (e != cudaSuccess) return e;
  if (p.copy_emb)
    emb = pack(emb, d.vocab, d.dim, &es, reinterpret_cast<T*>(ws + p.emb), status, st);
  if (!emb) return cudaErrorLaunchFailure;
  const bool many = p.piece < d.vocab;
  const bool dh_tiled = dhs % 8 == 0 && aligned(dh, 16);
  const bool demb_tiled = des % 8 == 0 && aligned(demb, 16);
  CUtensorMap h_k, h_mn, e_k, e_k_half, e_mn, dh_out, demb_sum;
  bool ok = make_tile_map(&h_k, copy, dtype, d.rows, d.dim, cs, box_rows(d.rows)) &&
            make_tile_map(&h_mn, copy, dtype, d.rows * p.halves, d.dim, cs, 64) &&
            make_tile_map(&e_k, emb, dtype, d.vocab, d.dim, es, kHalf) &&
            make_tile_map(&e_k_half, emb, dtype, d.vocab, d.dim, es, kHalf / 2) &&
            make_tile_map(&e_mn, emb, dtype, d.vocab, d.dim, es, 64);
  if (p.dh_sums)
    ok = ok && make_tile_map(&dh_out, dh_acc, SOMA_FP32,
                             p.dh_slots * ceil_div(d.rows, kTile) * kTile, p.acc_stride,
                             p.acc_stride, 32);
  else if (dh_tiled)
    ok = ok && make_tile_map(&dh_out, dh, dtype, d.rows, d.dim, dhs, 32);
  else
    dh_out = h_k;  // not used
  if (p.demb_sums)
    ok = ok && make_tile_map(&demb_sum, demb_acc, SOMA_FP32,
                             p.demb_slots * ceil_div(d.vocab, kTile) * kTile, p.acc_stride,
                             p.acc_stride, 32);
  if (!ok) return cudaErrorInvalidValue;
  for (int64_t v0 = 0; v0 < d.vocab; v0 += p.piece) {
    const int64_t width = d.vocab - v0 < p.piece ? d.vocab - v0 : p.piece;
    CUtensorMap g_k, g_mn, g_out, demb_out = h_k;
    if (!make_tile_map(&g_k, G, dtype, d.rows, width, p.g_stride, box_rows(d.rows)) ||
        !make_tile_map(&g_mn, G, dtype, d.rows * p.halves, width, p.g_stride, 64) ||
        !make_tile_map(&g_out, G, dtype, d.rows, width, p.g_stride, 32) ||
        (demb_tiled && !p.demb_sums &&
         !make_tile_map(&demb_out, demb + v0 * des, dtype, width, d.dim, des, 32)))
      return cudaErrorInvalidValue;
    Work w = {};
    w.M = d.rows;
    w.N = width;
    w.rows_a = box_rows(d.rows);
    w.m_tiles = (int32_t)ceil_div(w.M, kTile);
    const auto rounds = [&](int64_t tile_n) {
      return (double)ceil_div(w.m_tiles * ceil_div(width, tile_n), kPairs);
    };
    w.tile_n = kHalfTile * rounds(kTile / 2) < rounds(kTile) ? kTile / 2 : kTile;
    w.n_tiles = (int32_t)ceil_div(w.N, w.tile_n);
    w.k_stages = (int32_t)ceil_div(d.dim, tc::kDepth);
    w.y_b = (int32_t)v0;
    w.info = info;
    w.v0 = v0;
    w.top = top;
    w.out = G;
    w.out_stride = p.g_stride;
    w.tops = (int32_t)row_blocks(d);
    w.low = p.halves == 2 ? (int32_t)d.rows : 0;
    e = launch<kGrad, T>(h_k, w.tile_n == kTile ? e_k : e_k_half, g_out, w,
                         (int64_t)w.m_tiles * w.n_tiles, status, st);
    if (e != cudaSuccess) return e;

    w = shares(d.rows, d.dim, width);
    w.y_b = (int32_t)v0;
    w.info = info;
    w.emb = emb;
    w.emb_stride = es;
    w.top = top;
    if (p.dh_sums) {
      w.add = many;
      e = launch<kDhSums, T>(g_k, e_mn, dh_out, w, 0, status, st);
      if (e == cudaSuccess && v0 + width == d.vocab)
        e = launch_overlapped(sums_kernel<T>, dim3((unsigned)d.rows, (unsigned)ceil_div(d.dim, 512)),
                              128, 0, st, dh_acc, p.acc_stride,
                              many ? (int)p.dh_slots : 0, w, info, dh, dhs,
                              dhs % 4 == 0 && aligned(dh, 8), status);
    } else {
      w.out = dh_tiled ? nullptr : dh;
      w.out_stride = dhs;
      e = launch<kDh, T>(g_k, e_mn, dh_out, w, (int64_t)w.m_tiles * w.n_tiles, status, st);
    }
    if (e != cudaSuccess) return e;

    w = shares(width, d.dim, d.rows * p.halves);
    w.top = top;
    if (p.demb_sums) {
      e = launch<kDembSums, T>(g_mn, h_mn, demb_sum, w, 0, status, st);
      if (e == cudaSuccess)
        e = launch_overlapped(sums_kernel<T>, dim3((unsigned)d.vocab, (unsigned)ceil_div(d.dim, 512)),
                              128, 0, st, demb_acc,
                              p.acc_stride, 0, w, nullptr, demb, des,
                              des % 4 == 0 && aligned(demb, 8), status);
    } else {
      w.out = demb_tiled ? nullptr : demb + v0 * des;
      w.out_stride = des;
      e = launch<kDemb, T>(g_mn, h_mn, demb_out, w, (int64_t)w.m_tiles * w.n_tiles, status, st);
    }
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
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
  const Plan p = plan(d, false);
  if (!workspace || !aligned(workspace, 16) || workspace_bytes < p.total)
    return SOMA_ERR_WORKSPACE;
  int* status = status_ptr();
  if (!status) return SOMA_ERR_CUDA;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  const cudaStream_t st = (cudaStream_t)stream;
  if (gaps_fill(p.gaps, ws, st) != cudaSuccess) return SOMA_ERR_CUDA;
  trace_begin(SOMA_TRACE_LINEAR_CE, st);
  cudaError_t e =
      d.dtype == SOMA_BF16
          ? forward(p, static_cast<const __nv_bfloat16*>(h), static_cast<const __nv_bfloat16*>(emb),
                    d, targets, ignore_index, loss, lse, ws, status, st)
          : forward(p, static_cast<const __half*>(h), static_cast<const __half*>(emb), d, targets,
                    ignore_index, loss, lse, ws, status, st);
  trace_end(SOMA_TRACE_LINEAR_CE, st);
  if (e == cudaSuccess) e = gaps_check(p.gaps, ws, status, st);
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
  const Plan p = plan(d, true);
  if (!workspace || !aligned(workspace, 16) || workspace_bytes < p.total)
    return SOMA_ERR_WORKSPACE;
  int* status = status_ptr();
  if (!status) return SOMA_ERR_CUDA;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  const cudaStream_t st = (cudaStream_t)stream;
  if (gaps_fill(p.gaps, ws, st) != cudaSuccess) return SOMA_ERR_CUDA;
  trace_begin(SOMA_TRACE_LINEAR_CE, st);
  cudaError_t e =
      d.dtype == SOMA_BF16
          ? backward(p, static_cast<const __nv_bfloat16*>(h), static_cast<const __nv_bfloat16*>(emb),
                     d, targets, ignore_index, lse, dloss, static_cast<__nv_bfloat16*>(dh),
                     dh_stride, static_cast<__nv_bfloat16*>(demb), demb_stride, ws, status, st)
          : backward(p, static_cast<const __half*>(h), static_cast<const __half*>(emb), d, targets,
                     ignore_index, lse, dloss, static_cast<__half*>(dh), dh_stride,
                     static_cast<__half*>(demb), demb_stride, ws, status, st);
  trace_end(SOMA_TRACE_LINEAR_CE, st);
  if (e == cudaSuccess) e = gaps_check(p.gaps, ws, status, st);
  return e == cudaSuccess ? SOMA_OK : SOMA_ERR_CUDA;
}

}  // extern "C"
