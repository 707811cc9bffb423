// scan_backward.cu -- the gated linear recurrence backward (scan_common.cuh
// says how the work is cut).
//
// Per element of 16 bits 10 bytes read, 8 written and half a byte of the
// checkpoints.  Instructions bound it, with the 168 registers a thread that a
// segment's factors take and so at most 12 warps an SM: 32 x 2048 x 1376 in
// bf16 takes 339 us (4.9 TB/s), 1 x 32768 x 960, read twice, 172 us.  Before
// forget gates were kept above zero and sigmoid' good relative to its size,
// which cost 4%, with 128 registers (16 warps), where they spill: 371 and 240 us
// against 325 and 167.
#define SOMA_CHECK_FILE 10
#include "checked.cuh"
#include "scan_common.cuh"

namespace soma {
namespace scan {

namespace {

constexpr int kWarps = 4;     // of a CTA, at most
constexpr int kResident = 3;  // such CTAs fit an SM
constexpr double kJoin = 0.2; // steps that joining a chunk's map is worth

template <typename T, bool RAGGED, bool MAPS>
__global__ void __launch_bounds__(32 * kWarps, kResident)
backward_kernel(const T* __restrict__ gates, const __grid_constant__ Scan s,
                const T* __restrict__ dh, const float* __restrict__ dc_last,
                T* __restrict__ dgates, float* __restrict__ dc0) {
  extern __shared__ __align__(16) uint8_t raw[];
  Map<1>* const shared = reinterpret_cast<Map<1>*>(raw);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, warps = blockDim.x / 32;
  const int rows = warps * kSegment;
  const int64_t marks = (s.d.steps + kSegment - 1) / kSegment;
  uint32_t turn = 0;
  after_predecessor();
  for (int64_t at = blockIdx.x; at < s.d.batch * s.blocks * s.chunks; at += gridDim.x) {
    const int64_t item = at / s.chunks, k = at % s.chunks;
    const int64_t b = item / s.blocks, ch = (item % s.blocks) * 32 + lane;
    const bool on = ch < s.d.dim;
    const int64_t n = length_of(s, b), begin = k * s.chunk;
    const int64_t end = s.d.steps - begin < s.chunk ? s.d.steps : begin + s.chunk;
    float r[1] = {on && dc_last ? dc_last[b * s.d.dim + ch] : 0.f};
    Map<1> total = identity<1>();
    if (!MAPS) over_chunks<true, RAGGED, kWarps>(s, b, ch, on, k + 1, s.chunks, shared, turn++, r);

    const int64_t stop = n < end ? n : end;
    const int64_t at_ch = on ? ch : s.d.dim - 1;  // lanes past the last channel read along
    const int64_t rounds = (end - begin + rows - 1) / rows;
    // maps: from the chunk's first round to its last
    const int64_t step = MAPS ? rows : -rows;
    int64_t t0 = begin + (MAPS ? 0 : rounds - 1) * rows + warp * kSegment;
    T next[kSegment][5];
    float next_mark;
    const auto fetch = [&](int64_t t) {
      const T* p = gates + b * s.gs.b + t * s.gs.t + at_ch;
      const T* q = dh + b * s.hs.b + t * s.hs.t + at_ch;
      if (t >= begin && t + kSegment <= stop) {
#pragma unroll
        for (int j = 0; j < kSegment; ++j, p += s.gs.t, q += s.hs.t) {
          if (!SOMA_CHECK(inside(s, b, t + j, 1, at_ch, 1), s.status)) continue;
#pragma unroll
          for (int g = 0; g < 4; ++g) next[j][g] = p[g * s.gs.g];
          next[j][4] = *q;
        }
      } else {
#pragma unroll
        for (int j = 0; j < kSegment; ++j) {
          const bool there = t >= begin && t + j < stop &&
                             SOMA_CHECK(inside(s, b, t + j, 1, at_ch, 1), s.status);
#pragma unroll
          for (int g = 0; g < 4; ++g)
            next[j][g] = there ? p[j * s.gs.t + g * s.gs.g] : from_f32<T>(0.f);
          next[j][4] = there ? q[j * s.hs.t] : from_f32<T>(0.f);
        }
      }
      next_mark = t >= begin && t < stop &&
                          SOMA_CHECK(t % kSegment == 0 && inside(s, b, t, 1, at_ch, 1), s.status)
                      ? s.marks[(b * marks + t / kSegment) * s.d.dim + at_ch] : 0.f;
    };
    fetch(t0);
    for (int64_t left = rounds; left > 0; --left, t0 += step) {
      float add[kSegment], f[kSegment], ki[kSegment], kf[kSegment], kg[kSegment], od[kSegment];
      float c = next_mark;
      bool cut = false;  // a reset in the segment
      const int live = stop - t0 >= kSegment ? kSegment : stop > t0 ? (int)(stop - t0) : 0;
#pragma unroll
      for (int j = 0; j < kSegment; ++j) {
        const float y = to_f32(next[j][4]);
        const bool reset =
            RAGGED && s.resets && j < live && s.resets[b * s.d.steps + t0 + j] != 0;
        float i, di, fg, df, g, dg, o, d_o, th, dth;
        sigmoid_slope(to_f32(next[j][0]), i, di);
        sigmoid_slope(to_f32(next[j][1]), fg, df);
        fg = open(fg);
        tanh_slope(to_f32(next[j][2]), g, dg);
        sigmoid_slope(to_f32(next[j][3]), o, d_o);
        cut |= reset;
        const float prev = reset ? 0.f : c;
        c = fmaf(fg, prev, i * g);
        tanh_slope(c, th, dth);
        add[j] = y * o * dth;
        f[j] = reset ? 0.f : fg;
        ki[j] = g * di;
        kf[j] = prev * df;
        kg[j] = i * dg;
        od[j] = y * th * d_o;
      }
      fetch(t0 + step);
      if (live < kSegment) {
#pragma unroll
        for (int j = 0; j < kSegment; ++j)
          if (j >= live) {
            add[j] = ki[j] = kf[j] = kg[j] = od[j] = 0.f;
            f[j] = 1.f;
          }
      }
      Map<1> m = identity<1>();
#pragma unroll
      for (int j = kSegment - 1; j >= 0; --j) {
        // past a reset nothing goes on, not a NaN of its own document either
        m.b[0] = RAGGED ? apply(f[j], 0.f, add[j] + m.b[0]) : fmaf(f[j], m.b[0], f[j] * add[j]);
        m.a[0] *= f[j];
      }
      m.a[0] = RAGGED && cut ? 0.f : fmaxf(m.a[0], kLeast);
      if (MAPS) {
        join_total<true, RAGGED, kWarps>(shared, m, turn++, total);
        continue;
      }
      float in[1];
      join<true, RAGGED, kWarps>(shared, m, turn++, r, in);
      if (!on) continue;
      T* w = dgates + b * s.ds.b + (t0 + kSegment - 1) * s.ds.t + ch;
#pragma unroll
      for (int j = kSegment - 1; j >= 0; --j, w -= s.ds.t) {
        const float dc = add[j] + in[0];
        in[0] = RAGGED ? apply(f[j], 0.f, dc) : f[j] * dc;
        if (live < kSegment && t0 + j >= end) continue;
        if (!SOMA_CHECK(inside(s, b, t0 + j, 1, ch, 1), s.status)) continue;
        const bool dead = live < kSegment && j >= live;  // an infinite dc times 0 is no gradient
        w[0] = from_f32<T>(dead ? 0.f : dc * ki[j]);
        w[s.ds.g] = from_f32<T>(dead ? 0.f : dc * kf[j]);
        w[2 * s.ds.g] = from_f32<T>(dead ? 0.f : dc * kg[j]);
        w[3 * s.ds.g] = from_f32<T>(od[j]);
      }
    }
    __syncwarp();
    if (MAPS) {
      if (on && warp == 0) write_map(s, b, k, ch, total);
    } else if (dc0 && on && k == 0 && warp == 0) {
      dc0[b * s.d.dim + ch] = r[0];
    }
    __syncthreads();
  }
  admit_successor();
}

// The gradients of the gates take their places in the stage and are stored
// from there as boxes.
template <typename T, bool RAGGED, bool MAPS>
__global__ void __launch_bounds__(32 * kWarps, kResident)
backward_tiled_kernel(const __grid_constant__ Maps maps, const __grid_constant__ Scan s,
                      const float* __restrict__ dc_last, float* __restrict__ dc0, int* status) {
  extern __shared__ uint8_t raw[];
  __shared__ Ring ring;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, warps = blockDim.x / 32;
  const int rows = warps * kSegment;
  const int64_t marks = (s.d.steps + kSegment - 1) / kSegment;
  const int gate = rows * kBlock, stage_elems = 5 * gate, depth = s.depth;
  T* const stages = reinterpret_cast<T*>(raw + (128 - (tc::smem_u32(raw) & 127)) % 128);
  Map<2>* const shared = reinterpret_cast<Map<2>*>(stages + (size_t)depth * stage_elems);
  ring_init(ring, depth);
  int filled = 0, st = 0;
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
    const int64_t stop = n < end ? n : end;
    // the last rounds may be past the sequence's end: their gradients are zeros
    const int64_t rounds = (end - begin + rows - 1) / rows;

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
      if (lane < 5) {
        box_g2s(stages + (size_t)to * stage_elems + lane * gate, &maps.in[lane], ch0,
                maps.t_inner ? t : (int)b, maps.t_inner ? (int)b : t, &ring.full[to]);
      }
    };
    // one stage less in flight than there are: the newest is being stored
    if (warp == 0)
      for (int64_t q = 0; q < depth - 1 && q < rounds; ++q) fill(rounds - 1 - q);
    float r[2] = {0.f, 0.f};
    if (on && dc_last) r[0] = dc_last[b * s.d.dim + ch], r[1] = dc_last[b * s.d.dim + ch + 1];
    Map<2> total = identity<2>();
    if (!MAPS) over_chunks<true, RAGGED, kWarps>(s, b, ch, on, k + 1, s.chunks, shared, turn++, r);

    const auto mark_at = [&](int64_t t) {
      float2 x = make_float2(0.f, 0.f);
      if (on && t >= begin && t < stop &&
          SOMA_CHECK(t % kSegment == 0 && inside(s, b, t, 1, ch, 2), s.status))
        x = *reinterpret_cast<const float2*>(s.marks + (b * marks + t / kSegment) * s.d.dim + ch);
      return two(x.x, x.y);
    };
    // maps: from the first round to the last
    const int64_t step = MAPS ? rows : -rows;
    int64_t t0 = begin + (MAPS ? 0 : rounds - 1) * rows + warp * kSegment;
    Two next_mark = mark_at(t0);
    for (int64_t round = rounds - 1; round >= 0; --round, t0 += step) {
      const Two mark = next_mark;
      next_mark = mark_at(t0 + step);
      ring_wait(ring, st, parity, status);
      T* p = stages + (size_t)st * stage_elems + warp * kSegment * kBlock + 2 * lane;
      // what each step adds to r, its f, and the factors that turn the gradient
      // of its state into those of i, f and g
      Two add[kSegment], f[kSegment], ki[kSegment], kf[kSegment], kg[kSegment];
      Two c = mark;
      bool cut = false;  // a reset in the segment
      const int live = stop - t0 >= kSegment ? kSegment : stop > t0 ? (int)(stop - t0) : 0;
#pragma unroll
      for (int j = 0; j < kSegment; ++j) {
        const Two ai = load_two(p + j * kBlock), af = load_two(p + gate + j * kBlock);
        const Two ag = load_two(p + 2 * gate + j * kBlock);
        const Two ao = load_two(p + 3 * gate + j * kBlock);
        const Two y = load_two(p + 4 * gate + j * kBlock);
        Two i, di, fg, df, g, dg, o, d_o, th, dth;
        sigmoid_slope2(ai, i, di);
        sigmoid_slope2(af, fg, df);
        fg = open2(fg);
        tanh_slope2(ag, g, dg);
        sigmoid_slope2(ao, o, d_o);
        const bool reset =
            RAGGED && s.resets && j < live && s.resets[b * s.d.steps + t0 + j] != 0;
        cut |= reset;
        const Two prev = reset ? two(0.f) : c;
        c = fma2(fg, prev, i * g);
        tanh_slope2(c, th, dth);
        add[j] = y * o * dth;
        f[j] = reset ? two(0.f) : fg;
        if (MAPS) continue;
        ki[j] = g * di;
        kf[j] = prev * df;
        kg[j] = i * dg;
        store_two(p + 3 * gate + j * kBlock, y * th * d_o);
      }
      if (live < kSegment) {
#pragma unroll
        for (int j = 0; j < kSegment; ++j)
          if (j >= live) {
            add[j] = two(0.f);
            f[j] = two(1.f);
            if (MAPS) continue;
            ki[j] = kf[j] = kg[j] = two(0.f);
            store_two(p + 3 * gate + j * kBlock, two(0.f));
          }
      }
      Two A = two(1.f), B = two(0.f);
#pragma unroll
      for (int j = kSegment - 1; j >= 0; --j) {
        // past a reset nothing goes on, not a NaN of its own document either
        B = RAGGED ? apply2(f[j], two(0.f), add[j] + B) : f[j] * (add[j] + B);
        A = A * f[j];
      }
      Map<2> m;
      split(A, m.a[0], m.a[1]);
#pragma unroll
      for (int v = 0; v < 2; ++v) m.a[v] = RAGGED && cut ? 0.f : fmaxf(m.a[v], kLeast);
      split(B, m.b[0], m.b[1]);
      float in[2];
      if (MAPS) {
        join_total<true, RAGGED, kWarps>(shared, m, turn++, total);
      } else {
        if (lane == 0) tc::bulk_wait_read();  // this warp's stores of the round before
        join<true, RAGGED, kWarps>(shared, m, turn++, r, in);
      }
      // every warp is through with the stage of the round before
      if (warp == 0 && round >= depth - 1) fill(round - (depth - 1));
      if (!MAPS) {
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
              for (int g = 0; g < 3; ++g) store_two(p + g * gate + j * kBlock, two(0.f));
        }
        // each warp stores its own steps: no barrier of the CTA
        tc::fence_async_smem();
        __syncwarp();
        if (lane == 0 && t0 < end &&
            SOMA_CHECK(inside(s, b, t0, 1, ch0, 1) &&
                           in_dynamic(raw, p - 2 * lane, 3 * (size_t)gate * sizeof(T) +
                                                             kSegment * kBlock * sizeof(T)),
                       s.status)) {
          for (int g = 0; g < 4; ++g)
            box_s2g(&maps.out[g], ch0, maps.t_inner ? (int)t0 : (int)b,
                    maps.t_inner ? (int)b : (int)t0, p - 2 * lane + g * gate);
          tc::bulk_commit();
        }
      }
      if (++st == depth) st = 0, parity ^= 1;
    }
    __syncwarp();
    if (MAPS) {
      if (on && warp == 0) write_map(s, b, k, ch, total);
    } else if (dc0 && on && k == 0 && warp == 0) {
      dc0[b * s.d.dim + ch] = r[0], dc0[b * s.d.dim + ch + 1] = r[1];
    }
    if (!MAPS && lane == 0) tc::bulk_wait_read();
    __syncthreads();  // the stages are free
  }
  if (threadIdx.x == 0) ring_drain(ring, depth, fills);
  admit_successor();
  if (!MAPS && lane == 0) tc::bulk_wait();
}

// ------------------------------------------------------------------- host --

// CTAs of two warps, or of four and half as many: the larger ones take fewer
// chunks (1 x 32768 x 960: 183 us with two warps, 167 with four) and keep an SM
// full where two-warp ones are too few to (32 x 2048 x 1376: 348 and 325);
// elsewhere the smaller ones spread better (4 x 4096 x 960: 89 and 98).  All of
// these are some 3% more now, as said at the top.
Shape shape_of(const soma_scan_dims& d, int V, int fit) {
  const Shape a = shape(d, V, kWarps / 2, fit, kJoin), b = shape(d, V, kWarps, fit / 2, kJoin);
  return b.cost < 0.98 * a.cost ? b : a;
}
Shape tiled_shape(const soma_scan_dims& d, size_t width) {
  return shape_of(d, 2, width == 4 ? 5 : 2 * kResident);  // fp32: as many as shared memory holds
}
Shape plain_shape(const soma_scan_dims& d) { return shape_of(d, 1, 2 * kResident); }

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
    const Shape f = tiled_shape(s.d, sizeof(T));
    put(f, &s);
    const int rows = f.warps * kSegment;
    Maps maps;
    maps.t_inner = t_inner;
    if (!map_all(maps.in, 4, gates, s.d, s.gs, t_inner, dtype, rows) ||
        !map_all(maps.in + 4, 1, dh, s.d, s.hs, t_inner, dtype, rows) ||
        !map_all(maps.out, 4, dgates, s.d, s.ds, t_inner, dtype, kSegment))
      return cudaErrorInvalidValue;
    s.depth = sizeof(T) == 4 ? 2 : 3;
    const size_t smem = tiled_bytes<T>(s.depth, 5, f.warps);
    if (f.chunks > 1) {
      const cudaError_t e = launch(
          ragged ? backward_tiled_kernel<T, true, true> : backward_tiled_kernel<T, false, true>, f,
          smem, st, maps, s, dc_last, dc0, status);
      if (e != cudaSuccess) return e;
    }
    return launch(
        ragged ? backward_tiled_kernel<T, true, false> : backward_tiled_kernel<T, false, false>, f,
        smem, st, maps, s, dc_last, dc0, status);
  }
  const Shape f = plain_shape(s.d);
  put(f, &s);
  const size_t smem = joint_bytes<1>(f.warps);
  if (f.chunks > 1) {
    const cudaError_t e =
        launch(ragged ? backward_kernel<T, true, true> : backward_kernel<T, false, true>, f, smem,
               st, static_cast<const T*>(gates), s, static_cast<const T*>(dh), dc_last,
               static_cast<T*>(dgates), dc0);
    if (e != cudaSuccess) return e;
  }
  return launch(ragged ? backward_kernel<T, true, false> : backward_kernel<T, false, false>, f,
                smem, st, static_cast<const T*>(gates), s, static_cast<const T*>(dh), dc_last,
                static_cast<T*>(dgates), dc0);
}

}  // namespace

size_t backward_workspace(const soma_scan_dims& d) {
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

extern "C" int soma_scan_backward(const void* gates, soma_scan_strides gate_strides, int dtype,
                                  soma_scan_dims d, const float* checkpoints,
                                  const int32_t* lengths, const uint8_t* resets, const void* dh,
                                  soma_scan_strides dh_strides, const float* dc_last, void* dgates,
                                  soma_scan_strides dgate_strides, float* dc0, void* workspace,
                                  size_t workspace_bytes, void* stream) {
  if (!dims_ok(d)) return SOMA_ERR_UNSUPPORTED;
  if (!dtype_ok(dtype) || !strides_ok(gate_strides) || !strides_ok(dh_strides) ||
      !strides_ok(dgate_strides) || !aligned(gates, width(dtype)) || !aligned(dh, width(dtype)) ||
      !aligned(dgates, width(dtype)) || !aligned(checkpoints, 4) || !aligned(lengths, 4) ||
      !aligned(dc_last, 4) || !aligned(dc0, 4))
    return SOMA_ERR_INVALID_ARG;
  if (d.batch == 0 || d.dim == 0) return SOMA_OK;
  if (d.steps > 0 && (!gates || !dh || !dgates || !checkpoints)) return SOMA_ERR_INVALID_ARG;
  if (overlap(dc_last, dc0, d)) return SOMA_ERR_INVALID_ARG;
  const size_t need = backward_workspace(d);
  if (need && (!workspace || !aligned(workspace, 16) || workspace_bytes < guarded(need)))
    return SOMA_ERR_WORKSPACE;
  dh_strides.g = 0;
  Scan s = {};
  s.d = d;
  s.gs = gate_strides;
  s.hs = dh_strides;
  s.ds = dgate_strides;
  s.lengths = lengths;
  s.resets = resets;
  s.marks = const_cast<float*>(checkpoints);
  if (need) s.maps = reinterpret_cast<float2*>(static_cast<uint8_t*>(workspace) + kGuard);
  const cudaStream_t st = (cudaStream_t)stream;
  int* status = s.status = status_ptr();
  if (!status) return SOMA_ERR_CUDA;
  if (need && gaps_fill(gaps_around(need), workspace, st) != cudaSuccess) return SOMA_ERR_CUDA;
  trace_begin(SOMA_TRACE_SCAN, st);
  cudaError_t e =
      dtype == SOMA_FP32   ? backward<float>(gates, s, dh, dc_last, dgates, dc0, status, st)
      : dtype == SOMA_BF16 ? backward<__nv_bfloat16>(gates, s, dh, dc_last, dgates, dc0, status, st)
                           : backward<__half>(gates, s, dh, dc_last, dgates, dc0, status, st);
  trace_end(SOMA_TRACE_SCAN, st);
  if (need && e == cudaSuccess) e = gaps_check(gaps_around(need), workspace, status, st);
  return e == cudaSuccess ? SOMA_OK : SOMA_ERR_CUDA;
}
