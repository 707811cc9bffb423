// linear_attn.cuh -- what the kernels of linear attention with a decay per head
// share.
//
// One recurrence serves the forward call and each gradient.  With the roles x
// (asks), y (is asked) and z (answers) it is
//   S <- m_t S + f y_t z_t^T,   out_t = g S^T x_t,   S: [a][c]
// over the steps in order, or, reversed, from the last to the first:
//             x    y    z          S            f      g
//   o         q    k    v          S            1      scale
//   dq        do   v    k          S^T          1      scale
//   dk        v    do   q          dS^T         scale  1     reversed
//   dv        k    q    do         dS           scale  1     reversed
// m_t is the decay, or 0 where a document starts.  The reversed recurrence has
// the state's gradient after step t where the other has the state before it:
// its first step decays nothing, and a last decay comes after step 0.
#pragma once

#include <cstdint>

#include "soma_api.h"
#include "soma_launch.h"

namespace soma {
namespace attn {

// One of the recurrences of a call.
struct Problem {
  const void *x, *y, *z;
  void* out;
  soma_attn_strides xs, ys, zs, os;
  int32_t a, c;              // widths of x and y, and of z and out
  const float* s_in;         // state before the first step, or null: element (row, column)
  float* s_out;              // state after the last, or null
  int64_t in_row, in_col;    // ... lies at row * in_row + column * in_col of its head's
  int64_t out_row, out_col;
  int32_t reversed;
  float f, g;
};

constexpr int kMaxProblems = 3;

struct Call {
  Problem p[kMaxProblems];
  int32_t problems;
  int32_t heads;
  int64_t batch, steps;
  int64_t state;             // elements of one head's state
  const float* log_decay;
  const int32_t* lengths;
  const uint8_t* resets;
  int* status;
};

// Steps of a chunk of the tensor-core kernels, and how the steps of a call are
// cut into segments (there, of whole chunks).
constexpr int kChunk = 128;
struct Cut {
  int32_t segments;
  int32_t launched;  // segments of the launch
  int64_t steps;     // of a segment
  float* starts;     // [batch * heads][problems][segments] states; where segments > 1
  float2* fades;     // ... what a segment keeps of the state before it
};

// exp(e g) with the product's rounding carried along.  A NaN stays one where
// nothing decays: it reaches all that a head's steps do.
__device__ __forceinline__ float power_of(float g, float e) {
  if (e == 0.f) return isnan(g) ? g : 1.f;
  const float y = g * e;
  if (y < -104.f) return 0.f;
  return expf(y) * (1.f + fmaf(g, e, -y));
}
// S times exp(e g) is keep S + change S, so written that its error is 2^-24 of
// what is taken off where that is little: over many chunks it adds up.
struct Fade {
  float keep, change;
};
__device__ __forceinline__ Fade fade_of(float g, float e) {
  if (e == 0.f) return {1.f, 0.f};  // no steps: the state as it is, whatever g
  const float y = g * e;
  if (!(y > -0.5f)) return {power_of(g, e), 0.f};
  return {1.f, expm1f(y) + fmaf(g, e, -y)};
}

// Joins the segments' states of `call` (after the launch that made them).
cudaError_t launch_join(const Call& call, const Cut& cut, cudaStream_t st);

// The recurrences of a call on the tensor cores (16-bit types; widths, strides
// and addresses of whole 16-byte pieces; steps > 0).  False, and nothing is
// launched, if the strides do not nest as a tensor map wants it.
bool launch_chunks(const Call& call, const Cut& cut, int dtype, cudaStream_t st, cudaError_t* e);

__device__ __forceinline__ int64_t length_of(const Call& c, int64_t b) {
  if (!c.lengths) return c.steps;
  const int64_t n = c.lengths[b];
  return n < 0 ? 0 : n < c.steps ? n : c.steps;
}

// The head's log decay; NaN, with a record of it, where it is above 0 or NaN.
__device__ __forceinline__ float decay_of(const Call& c, int64_t h) {
  const float g = c.log_decay[h];
  if (g <= 0.f) return g;
  atomicCAS(c.status, 0, SOMA_ERR_NONFINITE);
  return NAN;
}

}  // namespace attn
}  // namespace soma
