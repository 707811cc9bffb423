// linear_attn.cu -- linear attention with a decay for each head: the entry
// points, the kernels of fp32 arithmetic and the one-token form
// (soma_linear_attn_* in include/soma_api.h have the formulas).
#include <cmath>
#include <type_traits>

#define SOMA_CHECK_FILE 14
#include "checked.cuh"
#include "linear_attn.cuh"
#include "numeric.cuh"
#include "pdl.cuh"
#include "tc_primitives.cuh"

namespace soma {
namespace attn {

namespace {

constexpr int kTile = 16;       // steps that are staged at once
constexpr int kAtOnce = 2;      // and gone through in one go
constexpr int kCols = 4;        // and columns
constexpr int kSums = kAtOnce * kCols;
constexpr int kStepThreads = 256;
constexpr int kMostWidth = 128;  // of keys and values
constexpr int kLoaders = 128;
// Log decays from here up are put off to a tile's end: z is multiplied by up to
// exp(0.5 * 15) = 1808 then, which fp32's range allows.
constexpr float kMildest = -0.5f;

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
__device__ Decay split_decay(double g) {
  const double l = exp(g);
  Decay d;
  d.low = __double2float_rd(l);
  d.up = __double2float_ru(l);
  d.share = d.up > d.low ? (uint32_t)((l - d.low) * (1.f / (d.up - d.low)) * 4294967295.0) : 0;
  return d;
}

// Threads that an SM's registers are shared among: two CTAs where heads are narrow.
__host__ __device__ constexpr int most_threads(int runs) { return runs == 4 ? 512 : 640; }

// Shared memory of the plain kernel: three tiles of steps, two of them on their way.
constexpr int kTiles = 3;
struct Tile {
  int rows, cols;
  float* at;
  __device__ float* x(int buf) const { return at + buf * kTile * (2 * rows + cols); }
  __device__ float* y(int buf) const { return x(buf) + kTile * rows; }
  __device__ float* z(int buf) const { return y(buf) + kTile * rows; }
  // whether n floats from p on lie in the CTA's dynamic shared memory
  __device__ bool holds(const float* p, int n) const {
    uint32_t size;
    asm("mov.u32 %0, %%dynamic_smem_size;" : "=r"(size));
    return p >= at && (uint32_t)((p - at) + n) * 4 <= size;
  }
};

// Adds what a lane and its partner hold: the first N sums for the lower of them,
// the next N for the upper.
template <int N>
__device__ __forceinline__ void fold(float (&o)[kSums], bool upper, int partner) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float sent = upper ? o[i] : o[i + N];
    o[i] = (upper ? o[i + N] : o[i]) + __shfl_xor_sync(0xffffffffu, sent, partner);
  }
}

// The recurrence step by step in fp32: one CTA per problem, segment, sequence and
// head, the state in registers, RUNS runs of four rows by four columns per thread.
// Up to eight neighbouring lanes (`groups`) hold the rows of the same columns.  A few steps at a
// time: what they read and the sums over their rows do not wait for one another, only
// the state itself does.
// Within a tile the state is kept as S l^-k, k steps into the tile, so that it is
// decayed once per tile and the decays go into the factors of z and of the output: two
// fp32 instructions per element of the state and step.  Strong decays, whose powers
// would cost range, are applied at each step, a third instruction.
// 16 x 2048 x 8 heads of 128 x 128 in fp32: 788 us forward, 2285 backward, in some
// runs up to 909 and 2390 (floors of their bytes 80 and 139).  Instruction issue bounds
// it (67% of the slots, half of them multiply-adds), and shared memory is busy for 42%
// of the time: few warps fit beside the state to cover latencies.  Packed pairs
// (fma.rn.f32x2) were no faster.  In bf16, for layouts that the tensor cores do not
// take: 1378 and 3929; 64 x 64: 819 and 1657.
template <typename T, int RUNS, bool OUT>
__global__ void __launch_bounds__(most_threads(RUNS))
plain_kernel(const __grid_constant__ Call call, const __grid_constant__ Cut cut, int loaders) {
  constexpr int kRows = 4 * RUNS;
  extern __shared__ __align__(16) float smem[];
  __shared__ Decay decay;
  __shared__ float multiplier[kTiles][kTile];  // of the state, before a step
  __shared__ float2 factor[kTile];             // of z and of the output
  __shared__ float first_decay;
  admit_successor();
  after_predecessor();
  // the last `loaders` threads stage, or if there are none, all
  const int workers = blockDim.x - loaders;
  const bool loads = !loaders || (int)threadIdx.x >= workers;
  const Problem& p = call.p[blockIdx.x % call.problems];
  const int64_t rest = blockIdx.x / call.problems;
  const int seg = (int)(rest % cut.launched);
  const int64_t bh = rest / cut.launched, b = bh / call.heads, h = bh % call.heads;
  int groups = 1;  // of this problem: the CTA's threads are those of the widest
  while (groups * kRows < p.a) groups *= 2;
  const int64_t which = bh * call.problems + blockIdx.x % call.problems;
  const int64_t len = length_of(call, b);
  const float g = decay_of(call, h);
  const bool put_off = g >= kMildest;  // the decays of a tile
  if (threadIdx.x == 0) {
    decay = split_decay(put_off ? kTile * (double)g : (double)g);
    first_decay = expf(g);
  }
  if (threadIdx.x < kTile) {
    const float e = put_off ? (float)threadIdx.x : 0.f;
    factor[threadIdx.x] = make_float2(p.f * power_of(-g, e), p.g * power_of(g, e));
  }
  // this segment's steps [first, last) in time, and how many of the sequence come
  // before them in the recurrence's order
  const int place = p.reversed ? cut.segments - 1 - seg : seg;
  const int64_t first = min(len, place * cut.steps);
  const int64_t last = min(len, (place + 1) * cut.steps);
  const int64_t count = last - first, done = p.reversed ? len - last : first;
  const Tile tile = {groups * kRows, (p.c + kCols - 1) / kCols * kCols, smem};
  const uint8_t* resets = call.resets ? call.resets + b * call.steps : nullptr;
  const auto step_of = [&](int64_t k) { return p.reversed ? last - 1 - k : first + k; };
  // whether n elements of step k of the segment, from column i on, are a tensor's
  const auto within = [&](int64_t k, int i, int n, int width) {
    return b < call.batch && step_of(k) >= 0 && step_of(k) < call.steps && i >= 0 && i + n <= width;
  };

  // steps k0 .. of the segment, rows and columns and steps past the end as zeros
  bool fresh = false;  // a document started in what this thread has seen
  const auto stage = [&](int64_t k0, int buf) {
    const int thread = threadIdx.x - (loaders ? workers : 0);
    const int all = loaders ? loaders : blockDim.x;
    const int n = count - k0 < kTile ? (int)(count - k0) : kTile;
    const auto copy = [&](const void* base, const soma_attn_strides& s, int width, int wide,
                          float* to) {
      const T* from = static_cast<const T*>(base) + b * s.b + h * s.h;
      const int64_t stride = s.t;
      if (std::is_same<T, float>::value) {
        // asynchronous: whole tiles are on their way
        const bool pieces = width % 4 == 0 && stride % 4 == 0 &&
                            (reinterpret_cast<uintptr_t>(from) & 15) == 0;
        const int each = pieces ? 4 : 1, across = wide / each;
        const int at_once = min(across, all), per = all / at_once;
        const int64_t next = (p.reversed ? -per : per) * stride;
        const int k1 = thread / at_once;
        if (k1 >= per) return;
        for (int i = thread % at_once * each; i < wide; i += at_once * each) {
          const int upto = i < width ? n : 0;
          const T* src = from + step_of(k0 + k1) * stride + i;
          uint32_t dst = tc::smem_u32(to + k1 * wide + i);
#pragma unroll 2
          for (int k = k1; k < kTile; k += per, src += next, dst += per * wide * 4) {
            if (!SOMA_CHECK(tile.holds(to + k * wide + i, each) && dst == tc::smem_u32(to + k * wide + i),
                            call.status))
              break;
            const bool there = k < upto &&  // zeros otherwise
                               SOMA_CHECK(within(k0 + k, i, each, width) &&
                                              src == from + step_of(k0 + k) * stride + i,
                                          call.status);
            if (pieces)
              asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst),
                           "l"(there ? src : from), "r"(there ? 16 : 0)
                           : "memory");
            else
              asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst),
                           "l"(there ? src : from), "r"(there ? 4 : 0)
                           : "memory");
          }
        }
      } else {
        // 16 loads are on their way before the first is stored
        constexpr int kAhead = 16;
        const int i = thread % wide, per = all / wide;
        if (thread >= per * wide) return;
        for (int k = thread / wide; k < kTile; k += per * kAhead) {
          T v[kAhead];
#pragma unroll
          for (int u = 0; u < kAhead; ++u) {
            const int s = k + u * per;
            const bool there = s < n && i < width &&
                               SOMA_CHECK(within(k0 + s, i, 1, width), call.status);
            v[u] = from[there ? step_of(k0 + s) * stride + i : 0];
          }
#pragma unroll
          for (int u = 0; u < kAhead; ++u) {
            const int s = k + u * per;
            if (s < kTile && SOMA_CHECK(tile.holds(to + s * wide + i, 1), call.status))
              to[s * wide + i] = s < n && i < width ? to_f32(v[u]) : 0.f;
          }
        }
      }
    };
#pragma unroll 1
    for (int w = OUT ? 0 : 1; w < 3; ++w)
      copy(w == 0 ? p.x : w == 1 ? p.y : p.z, w == 0 ? p.xs : w == 1 ? p.ys : p.zs,
           w == 2 ? p.c : p.a, w == 2 ? tile.cols : tile.rows,
           w == 0 ? tile.x(buf) : w == 1 ? tile.y(buf) : tile.z(buf));
    if (thread < kTile) {
      float m = 1.f;
      if (thread < n) {
        const int64_t t = step_of(k0 + thread);
        const bool none = p.reversed && t == len - 1;  // the decay that belongs to no step
        if (!put_off) m = none ? 1.f : decay.at(done + k0 + thread);
        else if (thread == 0) m = k0 ? decay.at(k0 / kTile) : none ? 1.f : first_decay;
        if (resets && !none && resets[p.reversed ? t + 1 : t]) m = 0.f;
        fresh = fresh || m == 0.f;
      }
      multiplier[buf][thread] = m;
    }
  };

  // row of register r: runs of four, `groups` runs apart
  const int group = threadIdx.x % groups, c0 = threadIdx.x / groups * kCols;
  const bool holds = (!loaders || !loads) && c0 < tile.cols;
  const bool works = __any_sync(0xffffffffu, holds);
  const auto row_of = [&](int r) { return (r / 4 * groups + group) * 4 + r % 4; };
  const bool joined = cut.segments > 1 && seg > 0;
  const int64_t states = call.batch * call.heads * call.problems * cut.segments;  // of the workspace
  const float* from = joined ? cut.starts + (which * cut.segments + seg) * call.state
                      : p.s_in ? p.s_in + bh * call.state : nullptr;
  if (!OUT) from = nullptr;  // what the segment adds
  const int64_t from_row = joined ? p.c : p.in_row, from_col = joined ? 1 : p.in_col;
  float S[kRows][kCols];
#pragma unroll
  for (int r = 0; r < kRows; ++r)
#pragma unroll
    for (int j = 0; j < kCols; ++j) S[r][j] = 0.f;
  if (from && holds)
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
      for (int j = 0; j < kCols; ++j) {
        const int i = row_of(r), c = c0 + j;
        if (i < p.a && c < p.c &&
            SOMA_CHECK(i * from_row + c * from_col < call.state &&
                           (!joined || which * cut.segments + seg < states),
                       call.status))
          S[r][j] = from[i * from_row + c * from_col];
      }
  // Of the sums of kAtOnce steps (in rows of kCols), a lane gets kSums / groups from
  // `mine` on, `mine_cols` of them or fewer in its columns.
  const int mine = (group & 1) * 4 + (group & 2) + (group >> 2);
  const int mine_cols = holds ? p.c - c0 - mine % kCols : 0;

  __syncthreads();  // the decay
  T* out = static_cast<T*>(p.out) + b * p.os.b + h * p.os.h;
  const auto arrived = [&](bool all) {  // this thread's copies, but those of the last tile
    if (all) asm volatile("cp.async.wait_all;" ::: "memory");
    else asm volatile("cp.async.wait_group 1;" ::: "memory");
  };
  const auto stage_next = [&](int64_t k0, int buf) {
    if (k0 < count) stage(k0, buf);
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  int buf = kTiles - 2;
  const int64_t next_out = p.reversed ? -p.os.t : p.os.t;
  // a tile's steps; kEach: every step decays the state, which is whole then
  const auto go = [&](auto each, int n, int64_t k0, T* to) {
    constexpr bool kEach = decltype(each)::value;
    if (!kEach) {
      const float m = multiplier[buf][0];
#pragma unroll
      for (int r = 0; r < kRows; ++r)
#pragma unroll
        for (int j = 0; j < kCols; ++j) S[r][j] *= m;
    }
    for (int k = 0; k < n; k += kAtOnce) {
      float o[kSums];
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        const float m = multiplier[buf][k + u], f = factor[k + u].x;
        const float* z = tile.z(buf) + (k + u) * tile.cols + c0;
        const float4 v4 =
            holds ? *reinterpret_cast<const float4*>(z) : make_float4(0.f, 0.f, 0.f, 0.f);
        const float v[kCols] = {f * v4.x, f * v4.y, f * v4.z, f * v4.w};
        if (m == 0.f) {  // nothing passes, whatever it is
#pragma unroll
          for (int r = 0; r < kRows; ++r)
#pragma unroll
            for (int j = 0; j < kCols; ++j) S[r][j] = 0.f;
        }
#pragma unroll
        for (int j = 0; j < kCols; ++j) o[u * kCols + j] = 0.f;
#pragma unroll
        for (int q = 0; q < RUNS; ++q) {
          const int at = (k + u) * tile.rows + (q * groups + group) * 4;
          const float4 y4 = *reinterpret_cast<const float4*>(tile.y(buf) + at);
          const float yr[4] = {y4.x, y4.y, y4.z, y4.w};
          float xr[4];
          if (OUT) {
            const float4 x4 = *reinterpret_cast<const float4*>(tile.x(buf) + at);
            xr[0] = x4.x; xr[1] = x4.y; xr[2] = x4.z; xr[3] = x4.w;
          }
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < kCols; ++j) {
              float& s = S[4 * q + r][j];
              s = kEach ? fmaf(m, s, yr[r] * v[j]) : fmaf(yr[r], v[j], s);
              if (OUT) o[u * kCols + j] = fmaf(xr[r], s, o[u * kCols + j]);
            }
        }
      }
      if (OUT) {
        if (groups > 1) fold<4>(o, group & 1, 1);
        if (groups > 2) fold<2>(o, group & 2, 2);
        if (groups > 4) fold<1>(o, group & 4, 4);
#pragma unroll
        for (int i = 0; i < kSums; ++i) {
          const int u = k + mine / kCols + i / kCols;
          if (i * groups < kSums && i % kCols < mine_cols && u < n &&
              SOMA_CHECK(within(k0 + u, c0 + mine % kCols + i % kCols, 1, p.c) &&
                             to + i % kCols + i / kCols * next_out ==
                                 out + step_of(k0 + u) * p.os.t + c0 + mine % kCols + i % kCols,
                         call.status))
            to[i % kCols + i / kCols * next_out] = from_f32<T>(factor[u].y * o[i]);
        }
        to += kAtOnce * next_out;
      }
    }
  };
  // Two tiles ahead of use; the copying code is there once, as cold instructions
  // are much of a short call's time (4 x 777 x 7 heads of 33 x 65: 69 us, with the first
  // two tiles' copies and each operand's written out 84).
  for (int64_t k0 = -2 * kTile; k0 < count; k0 += kTile) {
    if (loads) {
      stage_next(k0 + 2 * kTile, (buf + 2) % kTiles);
      arrived(false);
    }
    if (works && k0 >= 0) {
      const int n = count - k0 < kTile ? (int)(count - k0) : kTile;
      T* to = out + step_of(k0) * p.os.t + c0 + mine / kCols * next_out + mine % kCols;
      if (put_off) go(std::false_type(), n, k0, to);
      else go(std::true_type(), n, k0, to);
    }
    __syncthreads();
    buf = (buf + 1) % kTiles;
  }
  if (loads) arrived(true);
  if (put_off && count > 0) {  // the state itself
    const float l = power_of(decay_of(call, h), (float)((count - 1) % kTile));
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
      for (int j = 0; j < kCols; ++j) S[r][j] *= l;
  }

  if (!OUT) {
    // what the segment adds, and what it leaves of the state before it: the
    // reversed recurrence's decays come one step later
    const bool any = __syncthreads_or(fresh) != 0;
    float* to = cut.starts + (which * cut.segments + seg + 1) * call.state;
    if (threadIdx.x == 0) {
      const int64_t decays = p.reversed && last == len && count > 0 ? count - 1 : count;
      const Fade f = fade_of(g, (float)decays);
      cut.fades[which * cut.segments + seg] = any ? make_float2(0.f, 0.f)
                                                  : make_float2(f.keep, f.change);
    }
    if (holds)
#pragma unroll
      for (int r = 0; r < kRows; ++r)
#pragma unroll
        for (int j = 0; j < kCols; ++j) {
          const int i = row_of(r), c = c0 + j;
          if (i < p.a && c < p.c &&
              SOMA_CHECK(which * cut.segments + seg + 1 < states && i * p.c + c < call.state,
                         call.status))
            to[i * p.c + c] = S[r][j];
        }
    return;
  }
  // past the end, this segment's share
  const int64_t begin = max(len, place * cut.steps);
  const int64_t end = min(call.steps, (place + 1) * cut.steps);
  for (int64_t e = threadIdx.x; e < (end - begin) * p.c; e += blockDim.x)
    if (SOMA_CHECK(begin + e / p.c >= len && begin + e / p.c < call.steps, call.status))
      out[(begin + e / p.c) * p.os.t + e % p.c] = from_f32<T>(0.f);
  if (!p.s_out || !holds || seg != cut.segments - 1) return;
  const float left = !p.reversed || len == 0 ? 1.f
                     : resets && resets[0]     ? 0.f
                     : put_off                 ? first_decay
                                               : decay.at(len);
#pragma unroll
  for (int r = 0; r < kRows; ++r)
#pragma unroll
    for (int j = 0; j < kCols; ++j) {
      const int i = row_of(r), c = c0 + j;
      if (i < p.a && c < p.c &&
          SOMA_CHECK(bh < call.batch * call.heads && i * p.out_row + c * p.out_col < call.state,
                     call.status))
        p.s_out[bh * call.state + i * p.out_row + c * p.out_col] =
            left == 0.f ? 0.f : left * S[r][j];
    }
}

// Turns the segments' states into those that they start from, in place: state
// s + 1 is what segment s adds to what it leaves of state s.
__global__ void __launch_bounds__(256)
join_kernel(const __grid_constant__ Call call, const __grid_constant__ Cut cut) {
  admit_successor();
  after_predecessor();
  const int64_t parts = (call.state + 255) / 256, which = blockIdx.x / parts;
  const int64_t bh = which / call.problems;
  const Problem& p = call.p[which % call.problems];
  const int64_t e = blockIdx.x % parts * 256 + threadIdx.x;
  if (e >= call.state) return;
  const int64_t i = e / p.c, c = e % p.c;
  if (!SOMA_CHECK(bh < call.batch * call.heads && i < p.a && c < p.c &&
                      (!p.s_in || i * p.in_row + c * p.in_col < call.state),
                  call.status))
    return;
  float s = p.s_in ? p.s_in[bh * call.state + i * p.in_row + c * p.in_col] : 0.f;
  float* at = cut.starts + which * cut.segments * call.state + e;
  const float2* fades = cut.fades + which * cut.segments;
  constexpr int kAhead = 8;
  for (int k0 = 1; k0 < cut.segments; k0 += kAhead) {
    float add[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      add[j] = k0 + j < cut.segments ? at[(k0 + j) * call.state] : 0.f;
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      if (k0 + j < cut.segments) {
        const float2 f = fades[k0 + j - 1];
        s = f.x == 0.f ? add[j] : fmaf(f.x, s, fmaf(f.y, s, add[j]));
        at[(k0 + j) * call.state] = s;
      }
  }
}

// One token: a CTA per sequence and head, V adjacent columns per thread, the rows
// dealt out to `lanes` threads of the same columns.  The state's bytes bound it:
// 960 states of 64 x 64 (31 MB in and out) in 9 us with cold caches, 0.5 of the copy
// rate, the rest the kernel's begin and end.
template <typename T, int V>
__global__ void __launch_bounds__(kStepThreads)
step_kernel(const __grid_constant__ Call call, int lanes) {
  __shared__ float sx[kMostWidth], sy[kMostWidth];
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
      if (i + k * lanes < p.a &&
          SOMA_CHECK((i + k * lanes) * p.c + col + V <= call.state && bh < call.batch * call.heads,
                     call.status)) {
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
  for (int i = threadIdx.x; i < p.a && SOMA_CHECK(i < kMostWidth, call.status); i += kStepThreads) {
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
        if (r >= p.a || !SOMA_CHECK(r * p.c + col + V <= call.state, call.status)) break;
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
    for (int j = 0; j < V; ++j)
      if (SOMA_CHECK(first * p.c + col + j < kStepThreads * V && col + j < p.c, call.status))
        part[first * p.c + col + j] = o[j];
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
         (d.heads == 0 || d.batch <= (1 << 29) / d.heads) && d.key_dim >= 1 &&
         d.key_dim <= kMostWidth && d.value_dim >= 1 && d.value_dim <= kMostWidth;
}

bool dtype_ok(int t) { return t == SOMA_FP32 || t == SOMA_BF16 || t == SOMA_FP16; }

size_t width(int dtype) { return dtype == SOMA_FP32 ? 4 : 2; }

bool tensor_ok(const void* p, const soma_attn_strides& s, int dtype) {
  return aligned(p, width(dtype)) && s.b >= 0 && s.t >= 0 && s.h >= 0;
}

// An output's rows lie apart.
bool apart(const soma_attn_strides& s, const soma_attn_dims& d, int width) {
  return (d.batch < 2 || s.b >= width) && (d.steps < 2 || s.t >= width) &&
         (d.heads < 2 || s.h >= width);
}

bool overlap(const float* p, const float* q, int64_t count) {
  if (!p || !q) return false;
  const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
  return (a < b ? b - a : a - b) < (uintptr_t)count * sizeof(float);
}

constexpr size_t kSharedOfSm = 228 * 1024;

// Threads of a CTA of the plain kernel: `groups` of them share columns, each with
// `runs` runs of four rows, as few as hold all rows.
struct Spread {
  int groups, runs, cols;
};
Spread spread_of(int rows, int columns) {
  Spread s = {1, 0, (columns + kCols - 1) / kCols * kCols};
  while (s.groups * 16 < rows) s.groups *= 2;  // 8 at most: key and value dims end at 128
  s.runs = (rows + 4 * s.groups - 1) / (4 * s.groups);
  return s;
}
size_t shared_of(const Spread& s) {
  return sizeof(float) * kTiles * kTile * (2 * s.groups * 4 * s.runs + s.cols);
}
// Threads that stage the next steps while the others work.  None in fp32 with few
// threads, where all of them do it: the copies are asynchronous, and the registers
// of four more warps would keep another CTA away (64 x 64: 302 us instead of 445 for
// 16 x 2048 x 8; 33 x 65, backward, 4 x 777 x 7: 146 instead of 177).  With eight
// warps at work it is the other way round (128 x 128: 1093 and 788 us).
int loaders_of(const Spread& s, int dtype) {
  return dtype == SOMA_FP32 && s.groups * (s.cols / kCols) <= 160 ? 0 : kLoaders;
}
int threads_of(const Spread& s, int dtype) {
  return (s.groups * (s.cols / kCols) + 31) / 32 * 32 + loaders_of(s, dtype);
}

template <typename T, int RUNS>
cudaError_t plain(const Call& call, Cut cut, const Spread& s, cudaStream_t st) {
  const size_t smem = shared_of(s);
  constexpr int most = sizeof(float) * kTiles * kTile * (2 * 128 + 128);
  cudaError_t e = allow_shared<plain_kernel<T, RUNS, true>>(most);
  if (e == cudaSuccess) e = allow_shared<plain_kernel<T, RUNS, false>>(most);
  if (e != cudaSuccess) return e;
  const int64_t rows = call.problems * call.batch * call.heads;
  const int dtype = std::is_same<T, float>::value ? SOMA_FP32 : SOMA_BF16;
  const int loaders = loaders_of(s, dtype);
  if (cut.segments > 1) {
    cut.launched = cut.segments - 1;
    e = launch_overlapped(plain_kernel<T, RUNS, false>, dim3((unsigned)(rows * cut.launched)),
                          threads_of(s, dtype), smem, st, call, cut, loaders);
    if (e == cudaSuccess) e = launch_join(call, cut, st);
    if (e != cudaSuccess) return e;
  }
  cut.launched = cut.segments;
  return launch_overlapped(plain_kernel<T, RUNS, true>, dim3((unsigned)(rows * cut.segments)),
                           threads_of(s, dtype), smem, st, call, cut, loaders);
}

template <typename T>
cudaError_t plain(const Call& call, const Cut& cut, cudaStream_t st) {
  int rows = 0, columns = 0;
  for (int k = 0; k < call.problems; ++k) {
    if (call.p[k].a > rows) rows = call.p[k].a;
    if (call.p[k].c > columns) columns = call.p[k].c;
  }
  const Spread s = spread_of(rows, columns);
  return s.runs == 1   ? plain<T, 1>(call, cut, s, st)
         : s.runs == 2 ? plain<T, 2>(call, cut, s, st)
         : s.runs == 3 ? plain<T, 3>(call, cut, s, st)
                       : plain<T, 4>(call, cut, s, st);
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

// Whether the tensor-core kernels can read and write a tensor of `call`.  The
// stride of a dimension of one element leads nowhere and may be any.
bool tiled(const Call& call, const void* p, const soma_attn_strides& s) {
  const auto pieces = [](int64_t size, int64_t stride) { return size < 2 || stride % 8 == 0; };
  return aligned(p, 16) && pieces(call.batch, s.b) && pieces(call.steps, s.t) &&
         pieces(call.heads, s.h);
}

bool chunked_widths(const soma_attn_dims& d, int dtype) {
  return dtype != SOMA_FP32 && d.key_dim % 8 == 0 && d.value_dim % 8 == 0;
}

// CTAs that the GPU holds at once.
int64_t resident_of(const soma_attn_dims& d, int dtype, int problems) {
  if (chunked_widths(d, dtype)) return d.key_dim <= 64 && d.value_dim <= 64 ? 304 : 152;
  const int wide = d.key_dim > d.value_dim ? d.key_dim : d.value_dim;
  const Spread s = spread_of(problems > 1 ? wide : d.key_dim, problems > 1 ? wide : d.value_dim);
  const int by_threads = most_threads(s.runs) / threads_of(s, dtype);
  const int by_shared = (int)(kSharedOfSm / (shared_of(s) + 2048));
  return 152 * (by_threads < by_shared ? by_threads : by_shared);
}

// The cut with the least estimated time, in units of one CTA's work: a chunk on
// the tensor cores, a tile of steps elsewhere.  The states of all segments but
// the last come first (half the work), then the outputs; a CTA's begin and end
// take about two units, the join between the launches as much.
Cut cut_of(const soma_attn_dims& d, int dtype, int problems) {
  const int unit = chunked_widths(d, dtype) ? kChunk : kTile, ends = 2;
  const int64_t resident = resident_of(d, dtype, problems);
  Cut best = {};
  best.segments = 1;
  const int64_t rows = d.batch * d.heads * problems, units = (d.steps + unit - 1) / unit;
  best.steps = units * unit;
  const auto waves = [&](int64_t n) { return (double)((n + resident - 1) / resident); };
  double least = waves(rows) * (units + ends);
  for (int64_t n = 2; n <= units && n <= 1024; ++n) {
    const int64_t each = (units + n - 1) / n;
    if ((units + each - 1) / each != n) continue;
    const double cost =
        waves(rows * n) * (each + ends) + waves(rows * (n - 1)) * (0.5 * each + ends) + 2 * ends;
    if (cost < least) {
      least = cost;
      best.segments = (int32_t)n;
      best.steps = each * unit;
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
    chunked = chunked && p.a % 8 == 0 && p.c % 8 == 0 && tiled(call, p.x, p.xs) &&
              tiled(call, p.y, p.ys) && tiled(call, p.z, p.zs) && tiled(call, p.out, p.os);
  }
  cudaError_t e;
  if (chunked && launch_chunks(call, cut, dtype, st, &e)) return e;
  return dtype == SOMA_FP32   ? plain<float>(call, cut, st)
         : dtype == SOMA_BF16 ? plain<__nv_bfloat16>(call, cut, st)
                              : plain<__half>(call, cut, st);
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

cudaError_t launch_join(const Call& call, const Cut& cut, cudaStream_t st) {
  const int64_t rows = call.batch * call.heads * call.problems;
  return launch_overlapped(join_kernel, dim3((unsigned)(rows * ((call.state + 255) / 256))), 256, 0,
                           st, call, cut);
}

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

int64_t soma_linear_attn_workspace_bytes_upto(soma_attn_dims d, int dtype, int backward) {
  if (soma_linear_attn_workspace_bytes(d, dtype, backward) < 0) return -1;
  // A call of three rounds of CTAs or more is not cut.  With x rounds and n segments
  // the launches cost at least (1.5 - 0.5 / n) x of one segment's time, which from
  // n = 3 on is more than ceil(x); two segments cost ceil(2 x) / 2 + ceil(x) / 4,
  // which is at least ceil(x) from two rounds on.
  const int problems = backward ? 3 : 1;
  const int64_t rows = 3 * resident_of(d, dtype, problems), batch = d.batch;
  int64_t most = 0;
  for (d.batch = 1; d.batch <= batch && (d.batch - 1) * d.heads * problems <= rows; ++d.batch) {
    const int64_t bytes = (int64_t)parts_of(d, cut_of(d, dtype, problems), problems).bytes;
    if (bytes > most) most = bytes;
    if (d.heads == 0) break;
  }
  return most;
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
  if (!log_decay || (d.steps > 0 && (!q || !k || !v || !o)) ||
      !apart(o_strides, d, d.value_dim))
    return SOMA_ERR_INVALID_ARG;
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
  if (!log_decay || (d.steps > 0 && (!q || !k || !v || !d_out || !dq || !dk || !dv)) ||
      !apart(dq_strides, d, d.key_dim) || !apart(dk_strides, d, d.key_dim) ||
      !apart(dv_strides, d, d.value_dim))
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
  d.steps = 1;
  if (!log_decay || !q || !k || !v || !o || !s || !apart(o_strides, d, d.value_dim))
    return SOMA_ERR_INVALID_ARG;
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
