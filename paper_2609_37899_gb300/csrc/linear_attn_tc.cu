// linear_attn_tc.cu -- linear attention with a decay per head on the tensor
// cores (linear_attn.cuh has the recurrences that it computes).
//
// A CTA takes the steps of one recurrence in chunks of 128.  With D_ij = l^|i-j|
// for the pairs that see one another, w the decays from a step to the chunk's
// end and r those from its start, a chunk is four products:
//   P  = X Y^T                      [steps][steps]
//   O1 = X S                        what earlier chunks add, S the state so far
//   O2 = (f g D o P) Z              what the chunk's own steps add
//   dS = Y^T (f w Z)                S <- l^n S + dS
//   out = g r O1 + O2
// Two warps issue them (tcgen05, operands in 128-byte-swizzled shared memory,
// accumulators and D o P in tensor memory), one copies X, Y and Z with TMA (two
// that copied 16 bytes a lane took 12,000 cycles a chunk).  Two groups of warps
// do the rest side by side: D o P and out, and w Z and S, which stays in
// registers in fp32.  P of the next chunk runs under out.
//
// bf16, 16 x 4096 x 8 heads of 128 x 128: 129 to 135 us forward and 385 backward after
// a flush of L2 (floors of their bytes 80 and 139; three problems of four tensors each
// are read there).  Of 16 x 2048 x 8's time the tensor pipe is active for 23% forward
// and 22% backward, issue slots are busy for 33 and 30%, shared memory's data pipe for
// 39 and 34%: products and the groups of warps wait for one another in turn, and with
// chunks of 128 steps the 224 KB of shared memory have no room for a second X or Z
// that would take them apart (shorter chunks were not tried).  A chunk takes 4 us; a
// CTA's begin and end, with cold caches, 8 us.
//
// Long sequences of few heads are cut into segments: one launch for the state
// that each segment adds, one that joins them, one for the outputs.
#include <atomic>
#include <cmath>

#define SOMA_CHECK_FILE 15
#include "checked.cuh"
#include "linear_attn.cuh"
#include "numeric.cuh"
#include "pdl.cuh"
#include "tc_tiles.cuh"

namespace soma {
namespace attn {

namespace {

constexpr uint32_t kBox = kChunk * 128;  // 64 columns of a tile: 128 rows of 128 bytes
constexpr int kCols = 64;                // columns of a tile that a worker holds

// Shared memory: tiles of 128 steps by W columns.
template <int W>
struct Layout {
  static constexpr uint32_t tile = kChunk * W * 2;
  // scaled: w Z in 16 bits; rest: what that rounding took off
  static constexpr uint32_t x = 0, y = tile, z = 3 * tile, scaled = 4 * tile, rest = 5 * tile;
  static constexpr uint32_t state = 6 * tile;
  static constexpr uint32_t state_box = W * 128;
  static constexpr uint32_t bytes = state + W * W * 2;
  // tensor memory, in columns: D o P takes the place of P
  static constexpr uint32_t p = 0, o1 = kChunk, o2 = W == 64 ? 64 : 256, ds = W == 64 ? 192 : 384;
  static constexpr uint32_t columns = W == 64 ? 256 : 512;
  // Warps: a group for the outputs, one for the states, then those that copy and
  // the one that issues products.  A warp can read the 32 tensor-memory lanes of
  // its place among four, so a group is four warps for each half of W columns.
  static constexpr int halves = W / kCols, group = 4 * halves;
  static constexpr int loader = 2 * group, issuer = loader + 1;
  static constexpr int state_issuer = issuer + 1, threads = 32 * (2 * group + 4);
  // Registers of a thread, of each kind of warps.  All were launched with `launched`
  // (what ptxas takes from the launch bounds), and the sums must not exceed that.
  static constexpr int launched = W == 64 ? 80 : 96;
  static constexpr int out_regs = W == 64 ? 80 : 88, state_regs = W == 64 ? 112 : 128;
  static constexpr int rest_regs = W == 64 ? 48 : 40;
  static_assert(32 * (group * (out_regs + state_regs) + 4 * rest_regs) <= threads * launched,
                "setmaxnreg would wait for registers that the CTA does not have");
  // Columns of the state of a thread of the states' group.  64 rows fill half of
  // the lanes: dS then has them twice, for the other half of the columns.
  static constexpr int state_cols = W == 64 ? 32 : kCols;
};

struct Shared {
  uint64_t x_full, x_empty, y_full[2], y_empty[2], z_full, z_empty;
  uint64_t p_done, x_done, o_done, s_done;           // products (x_done: O1)
  uint64_t p_ready, o_free, z_ready, s_ready, done, done_s;  // what the workers made, or have read
  float power[kChunk + 1];                  // l^e
  float pair[2 * kChunk];                   // f g D_ij at kChunk + i - j
  float row_top[2][kChunk];                 // fp16: the largest of a half row of D o P
  float s_scale[2];                         // fp16: of the state in 16 bits
  uint32_t top[4];                          // fp16: the largest of a tile
  uint32_t tmem;
  volatile int abort;
};

// A bounded wait of a whole warp; on running out it records the timeout and
// raises the CTA's abort flag, after which no wait waits.
__device__ __forceinline__ bool wait(uint64_t* bar, uint32_t parity, Shared* sh, int* status,
                                     uint32_t max_polls = 1u << 22) {
  if (__all_sync(0xffffffffu, tc::mbar_try_wait(bar, parity))) return true;
  const bool ok = !sh->abort && tc::mbar_wait(bar, parity, max_polls);
  if (__all_sync(0xffffffffu, ok)) return true;
  if (!sh->abort) atomicCAS(status, 0, SOMA_ERR_TIMEOUT);
  sh->abort = 1;
  return false;
}

// The tiles that a CTA has asked for; those of y go to its two places in turn.  A
// place is handed back only by who has seen its copy land, also after an abort (the
// products' issuers break off then, and the states' warps keep z), so what has been
// handed back may be copied into, and one copy at most is under way in each place.
struct Copies {
  uint32_t x, y, z;
};

// The loading warp's last act: the last copy into each place has landed before the
// CTA leaves its shared memory to another.  In a whole run the products have waited
// for it; after an abort, whoever gave up, it may be on its way.
__device__ __forceinline__ void land(Shared& sh, const Copies& c) {
  if (c.x) tc::mbar_wait(&sh.x_full, (c.x - 1) & 1);
  for (uint32_t i = 0; i < 2; ++i) {
    const uint32_t n = (c.y + 1 - i) / 2;
    if (n) tc::mbar_wait(&sh.y_full[i], (n - 1) & 1);
  }
  if (c.z) tc::mbar_wait(&sh.z_full, (c.z - 1) & 1);
}

// How a tensor [batch][steps][heads][width] is seen by its tensor map, 64 columns
// wide and up to 128 steps high boxes of which the loader copies.
enum Form : int32_t {
  kHeadsInner,  // (column, head, step, sequence)
  kStepsInner,  // (column, step, head, sequence)
  kRows         // (column of all heads, step, sequence): rows of any heads' stride
};
struct Source {
  CUtensorMap map;
  int32_t form;
  int32_t head, sequence;  // 0 where all heads (sequences) are the same; kRows: columns of a head
};
struct Sources {
  Source x[kMaxProblems], y[kMaxProblems], z[kMaxProblems];
  int32_t box_rows;
};

__device__ __forceinline__ void load_box(void* dst, const Source& s, int column, int t, int b, int h,
                                         uint64_t* bar) {
  const int seq = b * s.sequence, head = h * s.head;
  const int x = s.form == kRows ? column + head : column;
  const int c1 = s.form == kHeadsInner ? head : t;
  const int c2 = s.form == kHeadsInner ? t : s.form == kStepsInner ? head : seq;
  const int c3 = s.form == kRows ? 0 : seq;
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], "
      "[%1, {%2, %3, %4, %5}], [%6];" ::"r"(tc::smem_u32(dst)),
      "l"(&s.map), "r"(x), "r"(c1), "r"(c2), "r"(c3), "r"(tc::smem_u32(bar))
      : "memory");
}

// 32 aligned bytes by one thread.
__device__ __forceinline__ void store32(void* p, const uint32_t (&u)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(u[0]),
               "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7])
               : "memory");
}
template <int N>
__device__ __forceinline__ void more_registers() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
}
template <int N>
__device__ __forceinline__ void fewer_registers() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}
__device__ __forceinline__ void sync_threads(int id, int threads) {
  asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}

// Low word of a swizzled operand descriptor: K-major, or MN-major with `box`
// bytes between blocks of 64 columns.
__device__ __forceinline__ uint32_t desc_k(uint32_t saddr) {
  return ((saddr & 0x3FFFFu) >> 4) | (1u << 16);
}
__device__ __forceinline__ uint32_t desc_mn(uint32_t saddr, uint32_t box) {
  return ((saddr & 0x3FFFFu) >> 4) | ((box >> 4) << 16);
}

// Shared address of piece 0 of a tile's row; piece j of its first 64 columns lies
// at this address with its bits 4 to 6 xor-ed with j.
__device__ __forceinline__ uint32_t row_address(const uint8_t* tile, int row) {
  return tc::smem_u32(tile) + row * 128 + ((row & 7) << 4);
}
__device__ __forceinline__ uint4 load_piece(uint32_t row, int j) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "r"(row ^ (j << 4))
               : "memory");
  return v;
}
__device__ __forceinline__ void store_piece(uint32_t row, int j, uint4 v) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(row ^ (j << 4)), "r"(v.x), "r"(v.y),
               "r"(v.z), "r"(v.w)
               : "memory");
}

// Two values in one conversion (one at a time they take four times as long).
template <typename T>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  union {
    __nv_bfloat162 b;
    __half2 h;
    uint32_t u;
  } w;
  if (std::is_same<T, __half>::value) w.h = __floats2half2_rn(a, b);
  else w.b = __floats2bfloat162_rn(a, b);
  return w.u;
}
template <typename T>
__device__ __forceinline__ void unpack2(uint32_t u, float& a, float& b) {
  if (std::is_same<T, __half>::value) {
    const __half2 h = *reinterpret_cast<const __half2*>(&u);
    const float2 f = __half22float2(h);
    a = f.x;
    b = f.y;
  } else {
    a = __uint_as_float(u << 16);
    b = __uint_as_float(u & 0xffff0000u);
  }
}

// fp16 has 5 bits of exponent: what is rounded to it is scaled by a power of two
// that brings the largest value to [2^13, 2^14) first.  Its reciprocal is a normal
// number, and the scale of a zero is 1.
__device__ __forceinline__ float range_scale(float top) {
  const int e = (int)(__float_as_uint(top) >> 23);  // biased exponent
  const int s = e == 0 || e == 255 ? 127 : 127 + 13 - (e - 127);
  return __uint_as_float((uint32_t)(s < 1 ? 1 : s > 253 ? 253 : s) << 23);
}
__device__ __forceinline__ float reciprocal(float scale) {  // of a power of two
  return __uint_as_float((254u << 23) - __float_as_uint(scale));
}

// Which steps of a chunk start a document, as bits.
struct Starts {
  uint32_t m[4];
  __device__ __forceinline__ bool any() const { return (m[0] | m[1] | m[2] | m[3]) != 0; }
  // the last one at or before i, or -1; the first one after i, or n
  __device__ __forceinline__ int at_or_before(int i) const {
    for (int q = i >> 5; q >= 0; --q) {
      const uint32_t w = q == i >> 5 ? m[q] & (0xffffffffu >> (31 - (i & 31))) : m[q];
      if (w) return q * 32 + 31 - __clz((int)w);
    }
    return -1;
  }
  __device__ __forceinline__ int after(int i, int n) const {
    for (int q = i >> 5; q < 4; ++q) {
      const uint32_t w = q == i >> 5 ? m[q] & (0xfffffffeu << (i & 31)) : m[q];
      if (w) return q * 32 + __ffs((int)w) - 1;
    }
    return n;
  }
};

template <typename T, int W, bool OUT>
__global__ void __launch_bounds__(Layout<W>::threads, W == 64 ? 2 : 1)
chunk_kernel(const __grid_constant__ Sources sources, const __grid_constant__ Call call,
             const __grid_constant__ Cut cut) {
  using L = Layout<W>;
  constexpr bool kHalfType = std::is_same<T, __half>::value;
  extern __shared__ __align__(1024) uint8_t smem[];
  Shared& sh = *reinterpret_cast<Shared*>(smem + L::bytes);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  int* status = call.status;
  if (tc::smem_u32(smem) & 1023) {  // the swizzle goes by addresses; the whole grid leaves
    atomicCAS(status, 0, SOMA_ERR_CUDA);
    return;
  }

  if (threadIdx.x == 0) {
    tc::mbar_init(&sh.x_full, 1);
    tc::mbar_init(&sh.x_empty, 1);
    for (int k = 0; k < 2; ++k) {
      tc::mbar_init(&sh.y_full[k], 1);
      tc::mbar_init(&sh.y_empty[k], OUT ? 2 : 1);  // P and dS
    }
    tc::mbar_init(&sh.z_full, 1);
    tc::mbar_init(&sh.z_empty, L::group + (OUT ? 1 : 0));  // the states' warps, and O2
    tc::mbar_init(&sh.p_done, 1);
    tc::mbar_init(&sh.x_done, 1);
    tc::mbar_init(&sh.o_done, 1);
    tc::mbar_init(&sh.s_done, 1);
    tc::mbar_init(&sh.p_ready, L::group);
    tc::mbar_init(&sh.o_free, L::group);
    tc::mbar_init(&sh.z_ready, L::group);
    tc::mbar_init(&sh.s_ready, L::group);
    tc::mbar_init(&sh.done, 1);
    tc::mbar_init(&sh.done_s, 1);
    tc::mbar_fence_init();
    sh.abort = 0;
    for (int k = 0; k < 4; ++k) sh.top[k] = 0;
  }
  if (warp == L::issuer) tc::tmem_alloc(&sh.tmem, L::columns);
  admit_successor();
  after_predecessor();

  const int problem = blockIdx.x % call.problems;
  const int64_t rest = blockIdx.x / call.problems;
  const int seg = (int)(rest % cut.launched);  // in the order in which they follow one another
  const int64_t bh = rest / cut.launched, b = bh / call.heads, h = bh % call.heads;
  const Problem& p = call.p[problem];
  const int len = (int)length_of(call, b);
  const bool reversed = p.reversed;
  const float g = decay_of(call, h);
  if ((int)threadIdx.x <= kChunk) {
    const float l = power_of(g, (float)threadIdx.x);
    sh.power[threadIdx.x] = l;
    // D is 0 above its diagonal, or, reversed, below
    const int up = reversed ? -(int)threadIdx.x : (int)threadIdx.x;
    if (threadIdx.x < kChunk) sh.pair[kChunk + up] = p.f * p.g * l;
    if (threadIdx.x > 0 && threadIdx.x < kChunk) sh.pair[kChunk - up] = 0.f;
  }
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem = sh.tmem;

  // this segment's chunks [first, last) in time
  const int place = reversed ? cut.segments - 1 - seg : seg;
  const int all = (int)(((int64_t)len + kChunk - 1) / kChunk);
  const int chunks = (int)(cut.steps / kChunk);
  const int first = min(all, place * chunks), last = min(all, first + chunks);
  const int count = last - first;
  const bool final_one = seg == cut.segments - 1;
  // whether the state after the segment is wanted; of each chunk but the last it is
  const bool state_wanted = !OUT || (final_one && p.s_out);
  const int a16 = (p.a + 15) / 16 * 16, c16 = (p.c + 15) / 16 * 16;
  const auto start_of = [&](int k) { return (reversed ? last - 1 - k : first + k) * kChunk; };
  const auto arrive = [&](uint64_t* bar) {
    __syncwarp();
    if (lane == 0) tc::mbar_arrive(bar);
  };

  // which steps of chunk k start a document: four steps' flags of each lane
  const auto flags_of = [&](int k) {
    uint32_t f = 0;
    if (call.resets && k < count) {
      const int t0 = start_of(k);
      const uint8_t* at = call.resets + b * call.steps + t0;
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (t0 + q * 32 + lane < len && at[q * 32 + lane]) f |= 1u << q;
    }
    return f;
  };
  const auto starts_of = [&](uint32_t flags) {
    Starts s;
#pragma unroll
    for (int q = 0; q < 4; ++q) s.m[q] = __ballot_sync(0xffffffffu, flags >> q & 1);
    return s;
  };

  if (warp < L::group) {
    // ---- outputs -------------------------------------------------------------
    fewer_registers<L::out_regs>();
    // No worker leaves early, as they meet at named barriers.
    if (OUT) {
      const int quarter = warp % 4, half = warp / 4;
      const int row = quarter * 32 + lane;  // step of the chunk
      const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16);
      constexpr int kPairs = kChunk / L::halves;  // columns of P
      const int j0 = half * kPairs;
      const auto meet = [&] {  // with the other half of these rows
        if (L::halves > 1) sync_threads(1 + quarter, 64);
      };
      T* const out = static_cast<T*>(p.out) + b * p.os.b + h * p.os.h;
      // rows whose whole sectors one lane can write
      const bool wide = (reinterpret_cast<uintptr_t>(out) & 31) == 0 && p.os.t % 16 == 0;
      uint32_t flags = flags_of(0);
      for (int k = 0; k < count; ++k) {
        const uint32_t odd = k & 1;
        const int t0 = start_of(k), n = min(kChunk, len - t0);
        // a sequence that ends before its tensor: the rest of the boxes may hold anything
        const bool ends = n < kChunk && len < call.steps;
        bool split = ends, sees = true;
        int lo = reversed ? row : 0, hi = reversed ? n - 1 : row;
        if (call.resets) {
          const Starts starts = starts_of(flags);
          flags = flags_of(k + 1);
          if (starts.any()) {
            split = true;
            const int doc = starts.at_or_before(row), next = row < n ? starts.after(row, n) : n;
            lo = reversed ? row : max(doc, 0);
            hi = reversed ? next - 1 : row;
            sees = reversed ? next >= n : doc < 0;  // the state before the chunk
          }
        }

        // D o P in 16 bits, in the place of P, 32 columns at a time
        const float* pair = sh.pair + kChunk + row - j0;
        // blocks that no row of this warp sees are zeros
        const auto unseen = [&](int q) {
          const int c = j0 + 32 * q;
          return reversed ? c + 31 < quarter * 32 : c > quarter * 32 + 31;
        };
        const auto block = [&](int q, float (&v)[32]) {
          tc::tmem_ld32_nowait(lanes + L::p + j0 + 32 * q, v);
          tc::tmem_wait_ld32(v);
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] *= pair[-(32 * q + j)];
          if (split) {
#pragma unroll
            for (int j = 0; j < 32; ++j) {
              const int c = j0 + 32 * q + j;
              if (c < lo || c > hi) v[j] = 0.f;
            }
          }
        };
        const auto pack = [&](float scale, const float (&v)[32], uint32_t (&u)[16]) {
#pragma unroll
          for (int j = 0; j < 16; ++j)
            u[j] = kHalfType ? pack2<T>(v[2 * j] * scale, v[2 * j + 1] * scale)
                             : pack2<T>(v[2 * j], v[2 * j + 1]);
        };
        wait(&sh.p_done, odd, &sh, status);
        tc::tc_fence_after();
        float p_scale = 1.f;
        if (kHalfType) {
          float top = 0.f;
#pragma unroll 1
          for (int q = 0; q < kPairs / 32; ++q)
            if (!unseen(q)) {
              float v[32];
              block(q, v);
#pragma unroll
              for (int j = 0; j < 32; ++j)  // what lies past the end was not computed
                top = j0 + 32 * q + j < n ? fmaxf(top, fabsf(v[j])) : top;
            }
          if (L::halves > 1) {
            sh.row_top[half][row] = top;
            meet();
            top = fmaxf(sh.row_top[0][row], sh.row_top[1][row]);
          }
          p_scale = range_scale(top);
        }
        const auto packed = [&](int q, uint32_t (&u)[16]) {
          if (unseen(q)) {
#pragma unroll
            for (int j = 0; j < 16; ++j) u[j] = 0;
          } else {
            float v[32];
            block(q, v);
            pack(p_scale, v, u);
          }
        };
        if (L::halves == 1) {
          // what is written lies in columns that have been read
#pragma unroll 1
          for (int q = 0; q < kPairs / 32; ++q) {
            uint32_t u[16];
            packed(q, u);
            tc::tmem_st16(lanes + L::p + q * 16, u);
          }
        } else {
          uint32_t u0[16], u1[16];
          packed(0, u0);
          packed(1, u1);
          tc::tc_fence_before();
          meet();  // both halves have read P
          tc::tc_fence_after();
          tc::tmem_st16(lanes + L::p + half * 32, u0);
          tc::tmem_st16(lanes + L::p + half * 32 + 16, u1);
        }
        tc::tmem_wait_st();
        tc::tc_fence_before();
        const int n16 = (n + 15) / 16 * 16;
        if (ends) {  // the steps that O2 goes through
          wait(&sh.z_full, odd, &sh, status);
          if (row >= n && row < n16)
            for (int j = 0; j < kCols / 8; ++j)
              store_piece(row_address(smem + L::z + half * kBox, row), j, make_uint4(0u, 0u, 0u, 0u));
          tc::fence_async_smem();
        }
        arrive(&sh.p_ready);

        // out = g r O1 + O2
        float r = p.g * sh.power[min(max(reversed ? n - 1 - row : row + 1, 0), kChunk)];
        const float back = reciprocal(p_scale);
        wait(&sh.o_done, odd, &sh, status);
        // written before s_ready, which O1's issuer has waited for (this warp could
        // find that barrier a phase further on)
        if (kHalfType) r *= reciprocal(*(volatile float*)&sh.s_scale[odd]);
        tc::tc_fence_after();
        T* const to = out + (t0 + row) * p.os.t + half * kCols;
#pragma unroll
        for (int c = 0; c < kCols; c += 16) {
          const int col = half * kCols + c;
          float o1[16], o2[16];
          tc::tmem_ld16(lanes + L::o1 + col, o1);
          tc::tmem_ld16(lanes + L::o2 + col, o2);
          uint32_t u[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            float v[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const float own = kHalfType ? o2[2 * j + i] * back : o2[2 * j + i];
              v[i] = sees ? fmaf(r, o1[2 * j + i], own) : own;
            }
            u[j] = pack2<T>(v[0], v[1]);
          }
          if (row < n &&
              SOMA_CHECK(b < call.batch && t0 >= 0 && t0 + row < call.steps &&
                             (wide && col + 16 <= p.c ? (reinterpret_cast<uintptr_t>(to + c) & 31) == 0
                                                      : (reinterpret_cast<uintptr_t>(to + c) & 15) == 0),
                         status)) {
            T* at = to + c;
            if (wide && col + 16 <= p.c) {
              store32(at, u);
            } else {
              if (col + 8 <= p.c)
                *reinterpret_cast<uint4*>(at) = make_uint4(u[0], u[1], u[2], u[3]);
              if (col + 16 <= p.c)
                *reinterpret_cast<uint4*>(at + 8) = make_uint4(u[4], u[5], u[6], u[7]);
            }
          }
        }
        tc::tc_fence_before();
        arrive(&sh.o_free);
      }
      // rows past the sequence's end, this segment's share of them
      const int64_t share = cut.steps;
      const int64_t from_step = max((int64_t)len, place * share);
      const int64_t to_step = min(call.steps, (place + 1) * share);
      const int per = p.c / 8;
      for (int64_t e = threadIdx.x; e < (to_step - from_step) * per; e += 32 * L::group)
        if (SOMA_CHECK(from_step + e / per >= len && from_step + e / per < call.steps, status))
          *reinterpret_cast<uint4*>(out + (from_step + e / per) * p.os.t + e % per * 8) =
              make_uint4(0u, 0u, 0u, 0u);
    }
  } else if (warp < 2 * L::group) {
    // ---- states --------------------------------------------------------------
    more_registers<L::state_regs>();
    const int quarter = warp % 4, half = (warp - L::group) / 4;
    const int row = quarter * 32 + lane;  // step of the chunk
    const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16);
    constexpr int kOwn = L::state_cols;
    const int s_row = W == 64 ? row % 64 : row;                  // of the state
    const int c0 = W == 64 ? row / 64 * kOwn : half * kOwn;      // first column
    const uint32_t z_row = row_address(smem + L::z + half * kBox, row);
    uint32_t tops = 0;
    // fp16: the largest over the group's values
    const auto largest = [&](float v) {
      const uint32_t t = __reduce_max_sync(0xffffffffu, __float_as_uint(v));
      if (lane == 0) atomicMax(&sh.top[tops & 3], t);
      sync_threads(5, 32 * L::group);
      const float r = __uint_as_float(*(volatile uint32_t*)&sh.top[tops & 3]);
      if (warp == L::group && lane == 0) sh.top[(tops + 2) & 3] = 0;
      ++tops;
      return r;
    };

    // Segments' own states start at 0.
    const bool joined = cut.starts && seg > 0;
    const float* from =
        joined ? cut.starts + ((bh * call.problems + problem) * cut.segments + seg) * call.state
               : p.s_in ? p.s_in + bh * call.state : nullptr;
    if (!OUT) from = nullptr;
    const int64_t from_row = joined ? p.c : p.in_row, from_col = joined ? 1 : p.in_col;
    float S[kOwn];
    if (from && from_col == 1 && (reinterpret_cast<uintptr_t>(from) & 15) == 0) {
#pragma unroll
      for (int j = 0; j < kOwn; j += 4) {
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (s_row < p.a && c0 + j < p.c &&
            SOMA_CHECK(s_row * from_row + c0 + j + 4 <= call.state && bh < call.batch * call.heads,
                       status))
          v = *reinterpret_cast<const float4*>(from + s_row * from_row + c0 + j);
        S[j] = v.x; S[j + 1] = v.y; S[j + 2] = v.z; S[j + 3] = v.w;
      }
    } else {
#pragma unroll
      for (int j = 0; j < kOwn; ++j)
        S[j] = from && s_row < p.a && c0 + j < p.c &&
                       SOMA_CHECK(s_row * from_row + (c0 + j) * from_col < call.state, status)
                   ? from[s_row * from_row + (c0 + j) * from_col]
                   : 0.f;
    }
    const uint32_t state_row = row_address(smem + L::state + c0 / kCols * L::state_box, s_row);
    // The state in 16 bits, for O1 of chunk k.
    const auto put_state = [&](int k) {
      float scale = 1.f;
      if (kHalfType) {
        float top = 0.f;
#pragma unroll
        for (int j = 0; j < kOwn; ++j) top = fmaxf(top, fabsf(S[j]));
        scale = range_scale(largest(top));
        if (warp == L::group && lane == 0) sh.s_scale[k & 1] = scale;
      }
      if (s_row < a16)
#pragma unroll
        for (int j = 0; j < kOwn / 8; ++j) {
          uint32_t u[4];
#pragma unroll
          for (int i = 0; i < 4; ++i)
            u[i] = kHalfType ? pack2<T>(S[8 * j + 2 * i] * scale, S[8 * j + 2 * i + 1] * scale)
                             : pack2<T>(S[8 * j + 2 * i], S[8 * j + 2 * i + 1]);
          store_piece(state_row, c0 % kCols / 8 + j, make_uint4(u[0], u[1], u[2], u[3]));
        }
      tc::fence_async_smem();
      arrive(&sh.s_ready);
    };
    if (OUT && count > 0) put_state(0);

    uint32_t flags = flags_of(0);
    bool whole = true;  // no document started in this segment
    bool landed = true;  // every z so far has been seen
    const Fade full = fade_of(g, (float)kChunk);
    for (int k = 0; k < count; ++k) {
      if (k + 1 == count && !state_wanted) break;
      const uint32_t odd = k & 1, s = k & 1, round = (k >> 1) & 1;
      const int t0 = start_of(k), n = min(kChunk, len - t0);
      bool split = false, counts = row < n;
      if (call.resets) {
        const Starts starts = starts_of(flags);
        flags = flags_of(k + 1);
        split = starts.any();
        // whether the state after the chunk sees this step
        if (split)
          counts = counts && (reversed ? starts.at_or_before(row) < 0 : starts.after(row, n) >= n);
        if (split) whole = false;
      }

      // w Z in 16 bits, and what their rounding takes off.  The last chunk's dS has
      // been waited for: their places are free.
      const float w = counts ? p.f * sh.power[reversed ? row + 1 : n - 1 - row] : 0.f;
      float z_scale = 1.f;
      landed = wait(&sh.z_full, odd, &sh, status) && landed;
      const auto fetch = [&](int j) {
        const uint4 v = load_piece(z_row, j);
        return counts ? v : make_uint4(0u, 0u, 0u, 0u);  // whatever it is
      };
      if (kHalfType) {
        __half2 top = __float2half2_rn(0.f);
#pragma unroll
        for (int j = 0; j < kCols / 8; ++j) {
          const uint4 z = fetch(j);
          const uint32_t e[4] = {z.x, z.y, z.z, z.w};
#pragma unroll
          for (int i = 0; i < 4; ++i)  // columns past the width hold anything
            if (half * kCols + j * 8 < p.c)
              top = __hmax2(top, __habs2(*reinterpret_cast<const __half2*>(&e[i])));
        }
        z_scale = range_scale(largest(fabsf(w) * fmaxf(__low2float(top), __high2float(top))));
      }
      const float by = w * z_scale;
#pragma unroll
      for (int j0 = 0; j0 < kCols / 8; j0 += 4) {
        uint4 z[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) z[j] = fetch(j0 + j);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t e[4] = {z[j].x, z[j].y, z[j].z, z[j].w};
          uint32_t u[4], v[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float f0, f1, r0, r1;
            unpack2<T>(e[i], f0, f1);
            f0 *= by;
            f1 *= by;
            u[i] = pack2<T>(f0, f1);
            unpack2<T>(u[i], r0, r1);
            v[i] = pack2<T>(f0 - r0, f1 - r1);
          }
          store_piece(z_row + (L::scaled - L::z), j0 + j, make_uint4(u[0], u[1], u[2], u[3]));
          store_piece(z_row + (L::rest - L::z), j0 + j, make_uint4(v[0], v[1], v[2], v[3]));
        }
      }
      if (n < kChunk && len < call.steps) {  // the steps that dS goes through
        wait(&sh.y_full[s], round, &sh, status);
        if (row >= n && row < (n + 15) / 16 * 16)
          for (int j = 0; j < kCols / 8; ++j)
            store_piece(z_row - L::z + L::y + s * L::tile, j, make_uint4(0u, 0u, 0u, 0u));
      }
      tc::fence_async_smem();
      arrive(&sh.z_ready);
      if (landed) arrive(&sh.z_empty);

      const Fade fade = n == kChunk ? full : fade_of(g, (float)n);
      const float back = reciprocal(z_scale);
      const bool gone = split || fade.keep == 0.f;  // keeps nothing, whatever it is
      wait(&sh.s_done, odd, &sh, status);
      tc::tc_fence_after();
#pragma unroll
      for (int c = 0; c < kOwn; c += 16) {
        float d[16];
        tc::tmem_ld16(lanes + L::ds + c0 + c, d);
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const float add = kHalfType ? d[j] * back : d[j];
          S[c + j] = gone ? add : fmaf(fade.keep, S[c + j], fmaf(fade.change, S[c + j], add));
        }
      }
      // what lies past the widths is not the state's
      if (s_row >= p.a || c0 + kOwn > p.c)
#pragma unroll
        for (int j = 0; j < kOwn; ++j)
          if (s_row >= p.a || c0 + j >= p.c) S[j] = 0.f;
      tc::tc_fence_before();
      if (OUT && k + 1 < count) {
        wait(&sh.x_done, odd, &sh, status);  // O1 has read the state before
        put_state(k + 1);
      }
    }

    float* to = nullptr;
    int64_t to_row = p.c, to_col = 1;
    if (!OUT) {
      // the state that the segment adds, and what it leaves of the one before it
      const int64_t at = (bh * call.problems + problem) * cut.segments + seg;
      if (SOMA_CHECK(at + 1 < call.batch * call.heads * call.problems * cut.segments, status))
        to = cut.starts + (at + 1) * call.state;
      if (warp == L::group && lane == 0) {
        const int64_t end = min((int64_t)len, (int64_t)last * kChunk);  // up to 2^31
        const Fade f = fade_of(g, count > 0 ? (float)(end - (int64_t)first * kChunk) : 0.f);
        cut.fades[at] = whole ? make_float2(f.keep, f.change) : make_float2(0.f, 0.f);
      }
    } else if (final_one && p.s_out) {
      to = p.s_out + bh * call.state;
      to_row = p.out_row;
      to_col = p.out_col;
    }
    if (to && s_row < p.a) {
      if (to_col == 1 && (reinterpret_cast<uintptr_t>(to) & 15) == 0) {
#pragma unroll
        for (int j = 0; j < kOwn; j += 4)
          if (c0 + j < p.c && SOMA_CHECK(s_row * to_row + c0 + j + 4 <= call.state, status))
            *reinterpret_cast<float4*>(to + s_row * to_row + c0 + j) =
                make_float4(S[j], S[j + 1], S[j + 2], S[j + 3]);
      } else {
#pragma unroll
        for (int j = 0; j < kOwn; ++j)
          if (c0 + j < p.c && SOMA_CHECK(s_row * to_row + (c0 + j) * to_col < call.state, status))
            to[s_row * to_row + (c0 + j) * to_col] = S[j];
      }
    }
  } else if (fewer_registers<L::rest_regs>(); warp == L::loader) {
    // ---- copies: one thread ----------------------------------------------------
    const Source &sx = sources.x[problem], &sy = sources.y[problem], &sz = sources.z[problem];
    const auto load = [&](uint32_t tile, const Source& src, int width, int t0, uint64_t* bar) {
      const int boxes = (width + 63) / 64;
      if (lane == 0) {
        tc::mbar_arrive_expect_tx(bar, boxes * sources.box_rows * 128);
        for (int j = 0; j < boxes; ++j)
          if (SOMA_CHECK(t0 >= 0 && t0 % kChunk == 0 && t0 < len && j * 64 < W &&
                             tile + j * kBox + sources.box_rows * 128 <= L::state,
                         status))
            load_box(smem + tile + j * kBox, src, j * 64, t0, (int)b, (int)h, bar);
      }
      __syncwarp();
    };
    Copies copies = {};
    for (int k = 0; k < count; ++k) {
      const int t0 = start_of(k);
      const uint32_t s = k & 1, round = (k >> 1) & 1;
      if (OUT) {
        if (!wait(&sh.x_empty, (k & 1) ^ 1, &sh, status)) break;
        load(L::x, sx, p.a, t0, &sh.x_full);
        ++copies.x;
      }
      if (!wait(&sh.y_empty[s], round ^ 1, &sh, status)) break;
      load(L::y + s * L::tile, sy, p.a, t0, &sh.y_full[s]);
      ++copies.y;
      if (!wait(&sh.z_empty, (k & 1) ^ 1, &sh, status)) break;
      load(L::z, sz, p.c, t0, &sh.z_full);
      ++copies.z;
    }
    land(sh, copies);
  } else if (warp == L::issuer) {
    // ---- P, O1 and O2: the whole warp waits, one elected thread issues ---------
    if (OUT) {
      const uint32_t xa = tc::smem_u32(smem + L::x), sa = tc::smem_u32(smem + L::state);
      const uint32_t za = tc::smem_u32(smem + L::z);
      const uint32_t id_o = tc::idesc_16(kChunk, c16, !kHalfType, false, true);
      for (int k = 0; k < count; ++k) {
        const uint32_t s = k & 1, round = (k >> 1) & 1, odd = k & 1;
        const int n16 = (min(kChunk, len - start_of(k)) + 15) / 16 * 16;
        const uint32_t ya = tc::smem_u32(smem + L::y + s * L::tile);
        if (!wait(&sh.x_full, odd, &sh, status)) break;
        if (!wait(&sh.y_full[s], round, &sh, status)) break;
        // O2 of the last chunk has read D o P, which P overwrites
        if (k > 0 && !wait(&sh.o_done, odd ^ 1, &sh, status)) break;
        // ... and with 64 columns O2 itself
        if (W == 64 && k > 0 && !wait(&sh.o_free, odd ^ 1, &sh, status)) break;
        tc::tc_fence_after();
        if (tc::elect_one()) {
          const uint32_t id_p = tc::idesc_16(kChunk, n16, !kHalfType, false, false);
          for (int j = 0; j < a16 / 16; ++j) {
            const uint32_t off = (j >> 2) * kBox + (j & 3) * 32;
            tc::mma_f16_ss_lohi(tmem + L::p, desc_k(xa + off), tc::kDescHi, desc_k(ya + off),
                                tc::kDescHi, id_p, j > 0);
          }
          tc::mma_commit(&sh.p_done);
          tc::mma_commit(&sh.y_empty[s]);
        }
        __syncwarp();
        if (!wait(&sh.s_ready, odd, &sh, status)) break;
        if (W != 64 && k > 0 && !wait(&sh.o_free, odd ^ 1, &sh, status)) break;
        tc::tc_fence_after();
        if (tc::elect_one()) {
          for (int j = 0; j < a16 / 16; ++j)
            tc::mma_f16_ss_lohi(tmem + L::o1, desc_k(xa + (j >> 2) * kBox + (j & 3) * 32),
                                tc::kDescHi, desc_mn(sa + j * 2048, L::state_box), tc::kDescHi, id_o,
                                j > 0);
          tc::mma_commit(&sh.x_done);
          tc::mma_commit(&sh.x_empty);
        }
        __syncwarp();
        if (!wait(&sh.z_full, odd, &sh, status)) break;
        if (!wait(&sh.p_ready, odd, &sh, status)) break;
        tc::tc_fence_after();
        if (tc::elect_one()) {
          for (int j = 0; j < n16 / 16; ++j)
            tc::mma_f16_ts_lohi(tmem + L::o2, tmem + L::p + j * 8, desc_mn(za + j * 2048, kBox),
                                tc::kDescHi, id_o, j > 0);
          tc::mma_commit(&sh.o_done);
          tc::mma_commit(&sh.z_empty);
        }
        __syncwarp();
      }
    }
    if (tc::elect_one()) tc::mma_commit(&sh.done);
    __syncwarp();
    if (!tc::mbar_wait(&sh.done, 0)) atomicCAS(status, 0, SOMA_ERR_TIMEOUT);
  } else if (warp == L::state_issuer) {
    // ---- dS, by a warp of its own: it is not to wait for D o P -------------------
    const uint32_t wa = tc::smem_u32(smem + L::scaled), ra = tc::smem_u32(smem + L::rest);
    const uint32_t id_s = tc::idesc_16(kChunk, c16, !kHalfType, true, true);
    for (int k = 0; k < count; ++k) {
      if (k + 1 == count && !state_wanted) break;
      const uint32_t s = k & 1, round = (k >> 1) & 1, odd = k & 1;
      const int n16 = (min(kChunk, len - start_of(k)) + 15) / 16 * 16;
      const uint32_t ya = tc::smem_u32(smem + L::y + s * L::tile);
      if (!wait(&sh.y_full[s], round, &sh, status)) break;
      if (!wait(&sh.z_ready, odd, &sh, status)) break;
      tc::tc_fence_after();
      if (tc::elect_one()) {
        // with 64 columns the rows of dS come twice (no bytes between blocks)
        for (int half = 0; half < 2; ++half)
          for (int j = 0; j < n16 / 16; ++j)
            tc::mma_f16_ss_lohi(tmem + L::ds, desc_mn(ya + j * 2048, W == 64 ? 0 : kBox), tc::kDescHi,
                                desc_mn((half ? ra : wa) + j * 2048, kBox), tc::kDescHi, id_s,
                                half > 0 || j > 0);
        tc::mma_commit(&sh.s_done);
        tc::mma_commit(&sh.y_empty[s]);
      }
      __syncwarp();
    }
    if (tc::elect_one()) tc::mma_commit(&sh.done_s);
    __syncwarp();
    if (!tc::mbar_wait(&sh.done_s, 0)) atomicCAS(status, 0, SOMA_ERR_TIMEOUT);
  }
  __syncwarp();
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  if (warp == L::issuer) tc::tmem_dealloc(tmem, L::columns);
}

// A wait of the loader's that runs out, with copies under way: x, both places of y
// and z are filled from src, y's first place is waited for and filled again, z's is
// never handed back.  out: the four tiles as they are when the CTA would leave, then
// the copies made of each.
constexpr int kTimeoutTest = 256;  // floats of a tile
__global__ void __launch_bounds__(32)
copies_timeout_kernel(const float* src, float* out, uint32_t max_polls, int* status) {
  __shared__ __align__(128) float tiles[4][kTimeoutTest];
  __shared__ Shared sh;
  if (threadIdx.x == 0) {
    tc::mbar_init(&sh.x_full, 1);
    tc::mbar_init(&sh.y_full[0], 1);
    tc::mbar_init(&sh.y_full[1], 1);
    tc::mbar_init(&sh.z_full, 1);
    tc::mbar_init(&sh.z_empty, 1);
    tc::mbar_fence_init();
    sh.abort = 0;
  }
  __syncwarp();
  Copies copies = {};
  const auto copy = [&](int tile, int from, uint64_t* bar, uint32_t& count) {
    ++count;
    if (threadIdx.x == 0) {
      tc::mbar_arrive_expect_tx(bar, sizeof(tiles[0]));
      tc::bulk_g2s(tiles[tile], src + from * kTimeoutTest, sizeof(tiles[0]), bar);
    }
    __syncwarp();
  };
  copy(0, 0, &sh.x_full, copies.x);
  copy(1, 1, &sh.y_full[0], copies.y);
  copy(2, 2, &sh.y_full[1], copies.y);
  copy(3, 3, &sh.z_full, copies.z);
  if (wait(&sh.y_full[0], 0, &sh, status)) copy(1, 4, &sh.y_full[0], copies.y);
  if (wait(&sh.z_empty, 0, &sh, status, max_polls)) copy(3, 0, &sh.z_full, copies.z);
  land(sh, copies);
  __syncwarp();
  for (int i = threadIdx.x; i < 4 * kTimeoutTest; i += 32) out[i] = tiles[i / kTimeoutTest][i % kTimeoutTest];
  if (threadIdx.x == 0) {
    out[4 * kTimeoutTest] = (float)copies.x;
    out[4 * kTimeoutTest + 1] = (float)copies.y;
    out[4 * kTimeoutTest + 2] = (float)copies.z;
  }
}

// ------------------------------------------------------------------- host --

// The tensor map of a tensor, if one of the forms describes it: strides are
// multiples of 16 bytes, each a multiple of the one before it, and no dimension
// is longer than the next stride.
bool make_source(Source* s, const void* base, const soma_attn_strides& st, int64_t batch,
                 int64_t steps, int64_t heads, int width, int box_rows, int dtype) {
  s->head = heads > 1 && st.h ? 1 : 0;
  s->sequence = batch > 1 && st.b ? 1 : 0;
  const int64_t H = s->head ? heads : 1, B = s->sequence ? batch : 1;
  if (steps > 1 && st.t == 0) return false;
  const auto nested = [](int64_t inner_size, int64_t inner, int64_t outer) {
    return outer % inner == 0 && outer / inner >= inner_size;
  };
  for (int form : {kHeadsInner, kStepsInner, kRows}) {
    int64_t size[4] = {width, 1, 1, 1}, stride[3] = {0, 0, 0};
    if (form == kHeadsInner) {
      size[1] = H; size[2] = steps; size[3] = B;
      stride[0] = st.h; stride[1] = st.t; stride[2] = st.b;
    } else if (form == kStepsInner) {
      size[1] = steps; size[2] = H; size[3] = B;
      stride[0] = st.t; stride[1] = st.h; stride[2] = st.b;
    } else {
      // what lies next to a head is read for it: only whole steps of 16 columns
      if (width % 16) return false;
      size[0] = (H - 1) * st.h + width; size[1] = steps; size[2] = B;
      stride[0] = st.t; stride[1] = st.b;
    }
    bool fits = true;
    int64_t inner_size = size[0], inner = 1;
    for (int i = 0; i < 3; ++i) {
      // the stride of a single element may be any that fits
      if (size[i + 1] == 1) stride[i] = (inner_size * inner + 7) / 8 * 8;
      fits = fits && stride[i] % 8 == 0 && nested(inner_size, inner, stride[i]) &&
             stride[i] < ((int64_t)1 << 38) && size[i] < ((int64_t)1 << 31);
      inner_size = size[i + 1];
      inner = stride[i];
    }
    if (!fits) continue;
    s->form = form;
    if (form == kRows && s->head) {
      if (st.h > INT32_MAX / heads) return false;
      s->head = (int32_t)st.h;
    }
    const int rows[4] = {64, form == kHeadsInner ? 1 : box_rows, form == kHeadsInner ? box_rows : 1,
                         1};
    return make_swizzled_map(&s->map, base, dtype, size, stride, rows);
  }
  return false;
}

// Whether a kernel's threads are launched with so many registers: its warps share
// those among them (setmaxnreg), and would wait for ever for more.  Another number
// than the launch bounds give here is an error of the build, which is said, not
// served by the kernels without tensor cores.  A failed query is not remembered.
template <auto KERNEL>
cudaError_t launched_with(int registers) {
  static std::atomic<int> known{0};
  int has = known.load(std::memory_order_relaxed);
  if (has == 0) {
    cudaFuncAttributes a;
    const cudaError_t e = cudaFuncGetAttributes(&a, KERNEL);
    if (e != cudaSuccess) return e;
    has = a.numRegs;
    known.store(has, std::memory_order_relaxed);
  }
  return has == registers ? cudaSuccess : cudaErrorInvalidConfiguration;
}

template <typename T, int W>
cudaError_t launch(const Sources& sources, const Call& call, Cut cut, cudaStream_t st) {
  constexpr size_t smem = Layout<W>::bytes + sizeof(Shared);
  static_assert(smem <= 227 * 1024, "shared memory of a CTA");
  cudaError_t e = launched_with<chunk_kernel<T, W, true>>(Layout<W>::launched);
  if (e == cudaSuccess) e = launched_with<chunk_kernel<T, W, false>>(Layout<W>::launched);
  if (e == cudaSuccess) e = allow_shared<chunk_kernel<T, W, true>>(smem);
  if (e == cudaSuccess) e = allow_shared<chunk_kernel<T, W, false>>(smem);
  if (e != cudaSuccess) return e;
  const int64_t rows = call.batch * call.heads * call.problems;
  if (cut.segments > 1) {
    cut.launched = cut.segments - 1;
    e = launch_overlapped(chunk_kernel<T, W, false>, dim3((unsigned)(rows * cut.launched)),
                          Layout<W>::threads, smem, st, sources, call, cut);
    if (e != cudaSuccess) return e;
    e = launch_join(call, cut, st);
    if (e != cudaSuccess) return e;
  } else {
    cut.starts = nullptr;
  }
  cut.launched = cut.segments;
  return launch_overlapped(chunk_kernel<T, W, true>, dim3((unsigned)(rows * cut.segments)), Layout<W>::threads,
                           smem, st, sources, call, cut);
}

}  // namespace

bool launch_chunks(const Call& call, const Cut& cut, int dtype, cudaStream_t st, cudaError_t* e) {
  Sources s;
  s.box_rows = call.steps < kChunk ? (int)(call.steps + 15) / 16 * 16 : kChunk;
  const int64_t B = call.batch, T = call.steps, H = call.heads;
  for (int k = 0; k < call.problems; ++k) {
    const Problem& p = call.p[k];
    if (!make_source(&s.x[k], p.x, p.xs, B, T, H, p.a, s.box_rows, dtype) ||
        !make_source(&s.y[k], p.y, p.ys, B, T, H, p.a, s.box_rows, dtype) ||
        !make_source(&s.z[k], p.z, p.zs, B, T, H, p.c, s.box_rows, dtype))
      return false;
  }
  const bool narrow = call.p[0].a <= 64 && call.p[0].c <= 64;
  *e = dtype == SOMA_BF16
           ? narrow ? launch<__nv_bfloat16, 64>(s, call, cut, st)
                    : launch<__nv_bfloat16, 128>(s, call, cut, st)
           : narrow ? launch<__half, 64>(s, call, cut, st) : launch<__half, 128>(s, call, cut, st);
  return true;
}

}  // namespace attn
}  // namespace soma

using namespace soma;
using namespace soma::attn;

extern "C" int soma_debug_attn_timeout(const float* src, float* out, uint32_t max_polls,
                                       void* stream) {
  if (!src || !out || (reinterpret_cast<uintptr_t>(src) & 15) ||
      (reinterpret_cast<uintptr_t>(out) & 3) || max_polls < 1 || max_polls > (1u << 22))
    return SOMA_ERR_INVALID_ARG;
  int* status = status_ptr();
  if (!status) return SOMA_ERR_CUDA;
  copies_timeout_kernel<<<1, 32, 0, (cudaStream_t)stream>>>(src, out, max_polls, status);
  return cudaGetLastError() == cudaSuccess ? SOMA_OK : SOMA_ERR_CUDA;
}
