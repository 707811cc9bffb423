// scan_forward.cu -- the gated linear recurrence forward, and its one-token
// form (scan_common.cuh says how the work is cut).
//
// Bytes bound the forward kernels: per element of 16 bits 8 read and 2 written,
// and half a byte for the checkpoints.  The instructions come close: 113 per
// element (one channel at a time, a 64-bit address and a bounds check per
// load) took 2.7 times the bytes' time.  As it is, 32 x 2048 x 1376 in bf16
// takes 188 us (5.0 TB/s; 67% of the issue slots, DRAM 61%), 1 x 32768 x 960,
// whose gates are read twice, 103 us.
//
// Warps of a CTA and CTAs of an SM, those two sizes, before forget gates were
// kept above zero (1% more now): 4 and 5 186 and 103 us, 3 and 7 213 and 108, 4
// and 6 202 and 108, 5 and 5 229 and 113, 6 and 4 212 and 115, 8 and 3 196 and
// 112.
#define SOMA_CHECK_FILE 9
#include "checked.cuh"
#include "scan_common.cuh"

namespace soma {
namespace scan {

namespace {

constexpr int kWarps = 4;     // of a CTA
constexpr int kResident = 5;  // such CTAs fit an SM
constexpr double kJoin = 0.8; // steps that joining a chunk's map is worth (8 x 1024 x 480 in fp32:
                              // 25.0 us with 0, 23.2 with this)

constexpr int kRingTest = 1024;  // floats of a stage of ring_timeout_kernel

// RAGGED: lengths or resets are given.  MAPS: the chunks' maps instead of h.
template <typename T, bool RAGGED, bool MAPS>
__global__ void __launch_bounds__(32 * kWarps, kResident)
forward_kernel(const T* __restrict__ gates, const __grid_constant__ Scan s, T* __restrict__ h) {
  extern __shared__ __align__(16) uint8_t raw[];
  Map<1>* const shared = reinterpret_cast<Map<1>*>(raw);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, warps = blockDim.x / 32;
  const int rows = warps * kSegment;  // steps of a round
  const int64_t marks = (s.d.steps + kSegment - 1) / kSegment;
  constexpr int kGates = MAPS ? 3 : 4;
  uint32_t turn = 0;
  after_predecessor();
  for (int64_t at = blockIdx.x; at < s.d.batch * s.blocks * s.chunks; at += gridDim.x) {
    const int64_t item = at / s.chunks, k = at % s.chunks;
    const int64_t b = item / s.blocks, ch = (item % s.blocks) * 32 + lane;
    const bool on = ch < s.d.dim;
    const int64_t n = length_of(s, b);
    const int64_t end = s.d.steps - k * s.chunk < s.chunk ? s.d.steps : (k + 1) * s.chunk;
    float c[1] = {on && s.c0 ? s.c0[b * s.d.dim + ch] : 0.f};
    Map<1> total = identity<1>();
    if (!MAPS) over_chunks<false, RAGGED, kWarps>(s, b, ch, on, 0, k, shared, turn++, c);

    const int64_t begin = k * s.chunk, stop = n < end ? n : end;
    const int64_t at_ch = on ? ch : s.d.dim - 1;  // lanes past the last channel read along
    // maps: from the chunk's last round to its first
    const int64_t step = MAPS ? -rows : rows;
    int64_t t0 = begin + warp * kSegment + (MAPS ? (end - begin - 1) / rows * rows : 0);
    T next[kSegment][kGates];
    const auto fetch = [&](int64_t t) {
      const T* p = gates + b * s.gs.b + t * s.gs.t + at_ch;
      if ((!MAPS || t >= begin) && t + kSegment <= stop) {
#pragma unroll
        for (int j = 0; j < kSegment; ++j, p += s.gs.t)
#pragma unroll
          for (int g = 0; g < kGates; ++g)
            if (SOMA_CHECK(inside(s, b, t + j, 1, at_ch, 1), s.status)) next[j][g] = p[g * s.gs.g];
      } else {
#pragma unroll
        for (int j = 0; j < kSegment; ++j)
#pragma unroll
          for (int g = 0; g < kGates; ++g)
            next[j][g] = (!MAPS || t >= begin) && t + j < stop &&
                                 SOMA_CHECK(inside(s, b, t + j, 1, at_ch, 1), s.status)
                             ? p[j * s.gs.t + g * s.gs.g] : from_f32<T>(0.f);
      }
    };
    fetch(t0);
    for (int64_t start = begin; start < end; start += rows, t0 += step) {
      float f[kSegment], u[kSegment];
      T o[kSegment];
      Map<1> m = identity<1>();
      const int live = stop - t0 >= kSegment ? kSegment : stop > t0 ? (int)(stop - t0) : 0;
#pragma unroll
      for (int j = 0; j < kSegment; ++j) {
        o[j] = next[j][kGates - 1];
        float num, den;
        tanh_parts(to_f32(next[j][2]), num, den);
        u[j] = num * rcp(den * one_exp(to_f32(next[j][0])));
        f[j] = open(rcp(one_exp(to_f32(next[j][1]))));
      }
      fetch(t0 + step);
      bool cut = false;  // a reset in the segment
      if (RAGGED && s.resets) {
#pragma unroll
        for (int j = 0; j < kSegment; ++j)
          if (j < live && s.resets[b * s.d.steps + t0 + j]) f[j] = 0.f, cut = true;
      }
      if (live < kSegment) {
#pragma unroll
        for (int j = 0; j < kSegment; ++j)
          if (j >= live) f[j] = 1.f, u[j] = 0.f;
      }
#pragma unroll
      for (int j = 0; j < kSegment; ++j) {
        m.b[0] = RAGGED ? apply(f[j], u[j], m.b[0]) : fmaf(f[j], m.b[0], u[j]);
        m.a[0] *= f[j];
      }
      m.a[0] = RAGGED && cut ? 0.f : fmaxf(m.a[0], kLeast);
      if (MAPS) {
        join_total<false, RAGGED, kWarps>(shared, m, turn++, total);
        continue;
      }
      float in[1];
      join<false, RAGGED, kWarps>(shared, m, turn++, c, in);
      if (!on) continue;
      if (s.marks && t0 < end &&
          SOMA_CHECK(t0 % kSegment == 0 && inside(s, b, t0, 1, ch, 1), s.status))
        s.marks[(b * marks + t0 / kSegment) * s.d.dim + ch] = in[0];
      T* p = h + b * s.hs.b + t0 * s.hs.t + ch;
#pragma unroll
      for (int j = 0; j < kSegment; ++j, p += s.hs.t) {
        in[0] = RAGGED ? apply(f[j], u[j], in[0]) : fmaf(f[j], in[0], u[j]);
        float num, den;
        tanh_parts(in[0], num, den);
        const T y = from_f32<T>(num * rcp(den * one_exp(to_f32(o[j]))));
        if (t0 + j < end && !SOMA_CHECK(inside(s, b, t0 + j, 1, ch, 1), s.status)) continue;
        if (live == kSegment) *p = y;
        else if (t0 + j < end) *p = j < live ? y : from_f32<T>(0.f);
      }
    }
    __syncwarp();
    if (MAPS) {
      if (on && warp == 0) write_map(s, b, k, ch, total);
    } else if (s.c_last && on && k == s.chunks - 1 && warp == 0) {
      s.c_last[b * s.d.dim + ch] = c[0];
    }
    __syncthreads();
  }
  admit_successor();
}

// h is written directly: a row of a warp's store is 128 bytes.
template <typename T, bool RAGGED, bool MAPS>
__global__ void __launch_bounds__(32 * kWarps, kResident)
forward_tiled_kernel(const __grid_constant__ Maps maps, const __grid_constant__ Scan s,
                     T* __restrict__ h, int* status) {
  extern __shared__ uint8_t raw[];
  __shared__ Ring ring;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, warps = blockDim.x / 32;
  const int rows = warps * kSegment;  // steps of a round
  const int64_t marks = (s.d.steps + kSegment - 1) / kSegment;
  constexpr int kGates = MAPS ? 3 : 4;
  const int gate = rows * kBlock, stage_elems = kGates * gate, depth = s.depth;
  T* const stages = reinterpret_cast<T*>(raw + (128 - (tc::smem_u32(raw) & 127)) % 128);
  Map<2>* const shared = reinterpret_cast<Map<2>*>(stages + (size_t)depth * stage_elems);
  ring_init(ring, depth);
  int filled = 0, st = 0;  // the next stage to fill, and to use
  uint32_t parity = 0, turn = 0, fills = 0;
  after_predecessor();
  for (int64_t at = blockIdx.x; at < s.d.batch * s.blocks * s.chunks; at += gridDim.x) {
    const int64_t item = at / s.chunks, k = at % s.chunks;
    const int64_t b = item / s.blocks;
    const int ch0 = (int)(item % s.blocks) * kBlock;
    const int64_t ch = ch0 + 2 * lane;
    const bool on = ch < s.d.dim;
    const int64_t n = length_of(s, b), begin = k * s.chunk;
    const int64_t end = s.d.steps - begin < s.chunk ? s.d.steps : begin + s.chunk;
    const int64_t stop = n < end ? n : end;  // of the steps that exist
    const int64_t rounds = stop > begin ? (stop - begin + rows - 1) / rows : 0;

    const auto fill = [&](int64_t round) {  // warp 0
      if (!ring_may_fill(ring)) return;
      const int t = (int)(begin + (MAPS ? rounds - 1 - round : round) * rows);
      if (!SOMA_CHECK(ch0 % kBlock == 0 && inside(s, b, t, 1, ch0, 1) && filled < depth &&
                          in_dynamic(raw, stages + (size_t)filled * stage_elems,
                                     stage_elems * sizeof(T)),
                      s.status))
        return;
      ++fills;
      const int to = filled;
      filled = filled + 1 == depth ? 0 : filled + 1;
      if (lane == 0) tc::mbar_arrive_expect_tx(&ring.full[to], stage_elems * sizeof(T));
      __syncwarp();
      if (lane < kGates) {
        box_g2s(stages + (size_t)to * stage_elems + lane * gate, &maps.in[lane], ch0,
                maps.t_inner ? t : (int)b, maps.t_inner ? (int)b : t, &ring.full[to]);
      }
    };
    if (warp == 0)
      for (int64_t q = 0; q < depth && q < rounds; ++q) fill(q);
    float c[2] = {0.f, 0.f};
    if (on && s.c0) c[0] = s.c0[b * s.d.dim + ch], c[1] = s.c0[b * s.d.dim + ch + 1];
    Map<2> total = identity<2>();
    if (!MAPS) over_chunks<false, RAGGED, kWarps>(s, b, ch, on, 0, k, shared, turn++, c);

    // maps: from the last round to the first
    int64_t t0 = begin + warp * kSegment + (MAPS ? (rounds - 1) * rows : 0);
    for (int64_t round = 0; round < rounds; ++round, t0 += MAPS ? -rows : rows) {
      ring_wait(ring, st, parity, status);
      const T* p = stages + (size_t)st * stage_elems + warp * kSegment * kBlock + 2 * lane;
      Two f[kSegment], u[kSegment];
      decltype(load_raw(p)) o[kSegment];  // kept, so that the stage is free after the join
      Two A = two(1.f), B = two(0.f);
      // steps of this segment that exist: nearly always all of them, and the
      // whole warp takes the branch without their checks
      const int live = stop - t0 >= kSegment ? kSegment : stop > t0 ? (int)(stop - t0) : 0;
#pragma unroll
      for (int j = 0; j < kSegment; ++j) {
        const Two ai = load_two(p + j * kBlock), af = load_two(p + gate + j * kBlock);
        const Two ag = load_two(p + 2 * gate + j * kBlock);
        if (!MAPS) o[j] = load_raw(p + 3 * gate + j * kBlock);
        Two num, den;
        tanh_parts2(ag, num, den);
        u[j] = num * rcp2(den * one_exp2(ai));
        f[j] = open2(rcp2(one_exp2(af)));
      }
      bool cut = false;  // a reset in the segment
      if (RAGGED && s.resets) {
#pragma unroll
        for (int j = 0; j < kSegment; ++j)
          if (j < live && s.resets[b * s.d.steps + t0 + j]) f[j] = two(0.f), cut = true;
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
#pragma unroll
      for (int v = 0; v < 2; ++v) m.a[v] = RAGGED && cut ? 0.f : fmaxf(m.a[v], kLeast);
      split(B, m.b[0], m.b[1]);
      float in[2];
      if (MAPS) join_total<false, RAGGED, kWarps>(shared, m, turn++, total);
      else join<false, RAGGED, kWarps>(shared, m, turn++, c, in);
      // every warp has read the stage
      if (warp == 0 && round + depth < rounds) fill(round + depth);
      if (!MAPS && on) {
        if (s.marks && t0 < end &&
            SOMA_CHECK(t0 % kSegment == 0 && inside(s, b, t0, 1, ch, 2), s.status))
          *reinterpret_cast<float2*>(s.marks + (b * marks + t0 / kSegment) * s.d.dim + ch) =
              make_float2(in[0], in[1]);
        T* q = h + b * s.hs.b + t0 * s.hs.t + ch;
        Two x = two(in[0], in[1]);
#pragma unroll
        for (int j = 0; j < kSegment; ++j) {
          x = RAGGED ? apply2(f[j], u[j], x) : fma2(f[j], x, u[j]);
          Two num, den;
          tanh_parts2(x, num, den);
          const Two y = num * rcp2(den * one_exp2(widen<T>(o[j])));
          if (t0 + j < end && !SOMA_CHECK(inside(s, b, t0 + j, 1, ch, 2), s.status)) continue;
          if (live == kSegment) store_two(q, y);
          else if (t0 + j < end) store_two(q, j < live ? y : two(0.f));
          q += s.hs.t;
        }
      }
      __syncwarp();
      if (++st == depth) st = 0, parity ^= 1;
    }
    // rounds past the sequence's end
    if (RAGGED && !MAPS && on)
      for (; t0 < end; t0 += rows)
        for (int j = 0; j < kSegment && t0 + j < end; ++j)
          if (SOMA_CHECK(inside(s, b, t0 + j, 1, ch, 2), s.status))
            store_two(h + b * s.hs.b + (t0 + j) * s.hs.t + ch, two(0.f));
    __syncwarp();
    if (MAPS) {
      if (on && warp == 0) write_map(s, b, k, ch, total);
    } else if (s.c_last && on && k == s.chunks - 1 && warp == 0) {
      s.c_last[b * s.d.dim + ch] = c[0], s.c_last[b * s.d.dim + ch + 1] = c[1];
    }
    __syncthreads();  // the stages have been read
  }
  if (threadIdx.x == 0) ring_drain(ring, depth, fills);
  admit_successor();
}

// A wait of the ring that runs out, with a copy under way: stage 0 is filled
// from src, stage 1 is waited for and never filled.  out: stage 0 as it is
// when the CTA would leave, then the stages filled (a fill after the timeout is
// refused).
__global__ void __launch_bounds__(64)
ring_timeout_kernel(const float* src, float* out, uint32_t max_polls, int* status) {
  __shared__ __align__(128) float stages[2][kRingTest];
  __shared__ Ring ring;
  uint32_t fills = 0;
  ring_init(ring, 2);
  const auto fill = [&](int to) {
    if (!ring_may_fill(ring)) return;
    ++fills;
    if (threadIdx.x) return;
    tc::mbar_arrive_expect_tx(&ring.full[to], sizeof(stages[0]));
    tc::bulk_g2s(stages[to], src, sizeof(stages[0]), &ring.full[to]);
  };
  if (threadIdx.x < 32) fill(0);
  ring_wait(ring, 1, 0, status, max_polls);
  __syncthreads();
  if (threadIdx.x < 32) fill(1);
  if (threadIdx.x == 0) ring_drain(ring, 2, fills);
  __syncthreads();
  for (int i = threadIdx.x; i < kRingTest; i += 64) out[i] = stages[0][i];
  if (threadIdx.x == 0) out[kRingTest] = (float)fills;
}

template <typename T, int V>
__global__ void __launch_bounds__(128)
scan_step_kernel(const T* __restrict__ gates, const __grid_constant__ Scan s,
                 float* __restrict__ c, T* __restrict__ h) {
  using B = typename Bits<T, V>::type;
  admit_successor();
  after_predecessor();
  const int64_t at = ((int64_t)blockIdx.x * 128 + threadIdx.x) * V;
  if (at >= s.d.batch * s.d.dim) return;
  const int64_t b = at / s.d.dim, ch = at % s.d.dim;
  if (!SOMA_CHECK(inside(s, b, 0, 1, ch, V), s.status)) return;
  const T* p = gates + b * s.gs.b + ch;
  float a[4][V], x[V], y[V];
#pragma unroll
  for (int k = 0; k < 4; ++k)
    unpack<T, V>(*reinterpret_cast<const B*>(p + k * s.gs.g), a[k]);
#pragma unroll
  for (int v = 0; v < V; ++v) {
    float num, den;
    tanh_parts(a[2][v], num, den);
    x[v] = fmaf(open(rcp(one_exp(a[1][v]))), c[at + v], num * rcp(den * one_exp(a[0][v])));
    tanh_parts(x[v], num, den);
    y[v] = num * rcp(den * one_exp(a[3][v]));
  }
#pragma unroll
  for (int v = 0; v < V; ++v) c[at + v] = x[v];
  *reinterpret_cast<B*>(h + b * s.hs.b + ch) = pack<T, V>(y);
}

// ------------------------------------------------------------------- host --

Shape tiled_shape(const soma_scan_dims& d, size_t width) {
  return shape(d, 2, kWarps, width == 4 ? 3 : kResident, kJoin);  // fp32: what shared memory holds
}
Shape plain_shape(const soma_scan_dims& d) { return shape(d, 1, kWarps, kResident, kJoin); }

template <typename T>
cudaError_t forward(const void* gates, Scan s, void* h, int* status, cudaStream_t st) {
  constexpr int dtype = dtype_of<T>();
  const bool ragged = s.lengths || s.resets;
  // h and the checkpoints are written two channels at a time
  const bool direct = s.d.dim % 2 == 0 && aligned(h, 2 * sizeof(T)) && s.hs.b % 2 == 0 &&
                      s.hs.t % 2 == 0 && aligned(s.marks, 8);
  for (const bool t_inner : {true, false}) {
    if (s.d.steps < 1 || !direct || !mappable(gates, s.d, s.gs, true, t_inner, dtype)) continue;
    const Shape f = tiled_shape(s.d, sizeof(T));
    put(f, &s);
    Maps maps;
    maps.t_inner = t_inner;
    if (!map_all(maps.in, 4, gates, s.d, s.gs, t_inner, dtype, f.warps * kSegment))
      return cudaErrorInvalidValue;
    s.depth = 2;
    const size_t smem = tiled_bytes<T>(s.depth, 4, f.warps);
    if (f.chunks > 1) {
      const cudaError_t e =
          launch(ragged ? forward_tiled_kernel<T, true, true> : forward_tiled_kernel<T, false, true>,
                 f, smem, st, maps, s, static_cast<T*>(h), status);
      if (e != cudaSuccess) return e;
    }
    return launch(
        ragged ? forward_tiled_kernel<T, true, false> : forward_tiled_kernel<T, false, false>, f,
        smem, st, maps, s, static_cast<T*>(h), status);
  }
  const Shape f = plain_shape(s.d);
  put(f, &s);
  const size_t smem = joint_bytes<1>(f.warps);
  if (f.chunks > 1) {
    const cudaError_t e =
        launch(ragged ? forward_kernel<T, true, true> : forward_kernel<T, false, true>, f, smem, st,
               static_cast<const T*>(gates), s, static_cast<T*>(h));
    if (e != cudaSuccess) return e;
  }
  return launch(ragged ? forward_kernel<T, true, false> : forward_kernel<T, false, false>, f, smem,
                st, static_cast<const T*>(gates), s, static_cast<T*>(h));
}

template <typename T, int V>
cudaError_t step(const void* gates, const Scan& s, float* c, void* h, cudaStream_t st) {
  const int64_t threads = s.d.batch * s.d.dim / V;
  return launch_overlapped(scan_step_kernel<T, V>, dim3((unsigned)((threads + 127) / 128)), 128, 0,
                           st, static_cast<const T*>(gates), s, c, static_cast<T*>(h));
}

// Whether a 16-bit tensor can be read in pairs of channels.
bool pairs(const void* p, const soma_scan_strides& s) {
  return aligned(p, 4) && s.b % 2 == 0 && s.t % 2 == 0 && s.g % 2 == 0;
}

}  // namespace

size_t forward_workspace(const soma_scan_dims& d) {
  size_t most = maps_bytes(d, plain_shape(d));
  for (size_t w : {2, 4}) {
    const size_t n = maps_bytes(d, tiled_shape(d, w));
    if (n > most) most = n;
  }
  return most;
}

}  // namespace scan
}  // namespace soma

using namespace soma;
using namespace soma::scan;

extern "C" {

int64_t soma_scan_checkpoint_count(soma_scan_dims d) {
  if (!dims_ok(d)) return -1;
  return d.batch * d.dim * ((d.steps + kSegment - 1) / kSegment);
}

int64_t soma_scan_workspace_bytes(soma_scan_dims d) {
  if (!dims_ok(d)) return -1;
  if (d.batch == 0 || d.dim == 0) return 0;
  const size_t f = forward_workspace(d), b = backward_workspace(d);
  return (int64_t)guarded(f > b ? f : b);
}

int soma_scan_forward(const void* gates, soma_scan_strides gate_strides, int dtype,
                      soma_scan_dims d, const float* c0, const int32_t* lengths,
                      const uint8_t* resets, void* h, soma_scan_strides h_strides,
                      float* c_last, float* checkpoints, void* workspace, size_t workspace_bytes,
                      void* stream) {
  if (!dims_ok(d)) return SOMA_ERR_UNSUPPORTED;
  if (!dtype_ok(dtype) || !strides_ok(gate_strides) || !strides_ok(h_strides) ||
      !aligned(gates, width(dtype)) || !aligned(h, width(dtype)) || !aligned(c0, 4) ||
      !aligned(lengths, 4) || !aligned(c_last, 4) || !aligned(checkpoints, 4))
    return SOMA_ERR_INVALID_ARG;
  if (d.batch == 0 || d.dim == 0) return SOMA_OK;
  if (d.steps > 0 && (!gates || !h)) return SOMA_ERR_INVALID_ARG;
  if (overlap(c0, c_last, d)) return SOMA_ERR_INVALID_ARG;
  const size_t need = forward_workspace(d);
  if (need && (!workspace || !aligned(workspace, 16) || workspace_bytes < guarded(need)))
    return SOMA_ERR_WORKSPACE;
  h_strides.g = 0;
  Scan s = {};
  s.d = d;
  s.gs = gate_strides;
  s.hs = h_strides;
  s.c0 = c0;
  s.lengths = lengths;
  s.resets = resets;
  s.c_last = c_last;
  s.marks = checkpoints;
  if (need) s.maps = reinterpret_cast<float2*>(static_cast<uint8_t*>(workspace) + kGuard);
  const cudaStream_t st = (cudaStream_t)stream;
  int* status = s.status = status_ptr();
  if (!status) return SOMA_ERR_CUDA;
  if (need && gaps_fill(gaps_around(need), workspace, st) != cudaSuccess) return SOMA_ERR_CUDA;
  trace_begin(SOMA_TRACE_SCAN, st);
  cudaError_t e = dtype == SOMA_FP32   ? forward<float>(gates, s, h, status, st)
                  : dtype == SOMA_BF16 ? forward<__nv_bfloat16>(gates, s, h, status, st)
                                       : forward<__half>(gates, s, h, status, st);
  trace_end(SOMA_TRACE_SCAN, st);
  if (need && e == cudaSuccess) e = gaps_check(gaps_around(need), workspace, status, st);
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
  Scan s = {};
  s.d = d;
  s.gs = gate_strides;
  s.hs = h_strides;
  s.status = status_ptr();
  if (!s.status) return SOMA_ERR_CUDA;
  const cudaStream_t st = (cudaStream_t)stream;
  const bool two = dim % 2 == 0 && pairs(gates, gate_strides) && pairs(h, h_strides);
  trace_begin(SOMA_TRACE_SCAN, st);
  cudaError_t e;
  if (dtype == SOMA_FP32) e = step<float, 1>(gates, s, c, h, st);
  else if (dtype == SOMA_BF16)
    e = two ? step<__nv_bfloat16, 2>(gates, s, c, h, st) : step<__nv_bfloat16, 1>(gates, s, c, h, st);
  else
    e = two ? step<__half, 2>(gates, s, c, h, st) : step<__half, 1>(gates, s, c, h, st);
  trace_end(SOMA_TRACE_SCAN, st);
  return e == cudaSuccess ? SOMA_OK : SOMA_ERR_CUDA;
}

int soma_debug_scan_timeout(const float* src, float* out, uint32_t max_polls, void* stream) {
  if (!src || !out || !aligned(src, 16) || !aligned(out, 4) || max_polls < 1 ||
      max_polls > (1u << 22))
    return SOMA_ERR_INVALID_ARG;
  int* status = status_ptr();
  if (!status) return SOMA_ERR_CUDA;
  ring_timeout_kernel<<<1, 64, 0, (cudaStream_t)stream>>>(src, out, max_polls, status);
  return cudaGetLastError() == cudaSuccess ? SOMA_OK : SOMA_ERR_CUDA;
}

}  // extern "C"
