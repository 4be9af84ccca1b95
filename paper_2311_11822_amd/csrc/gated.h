// What the kernels of gated feed-forward layers share: arguments, activations, and what becomes of each product's values.
#pragma once

#include <type_traits>

#include "dp_internal.h"
#include "piece.h"

namespace dpbk {

struct GatedArgs {
  const void *x, *w_gate, *w_up, *b_gate, *b_up;       // forward: [rows, d], [d, f], [d, f], [f] or null
  const void *dy, *w_down;                             // backward: [rows, d_out], [f, d_out]; w_down null: dy is [rows, f]
  void *gate, *up, *h;                                 // [rows, f]: results (gate and up may be null); the first two backward's inputs
  void *dgate, *dup, *dx;                              // [rows, f], [rows, f], [rows, d] or null
  int rows, d, f, d_out;
  int act;
  float* partial;                                      // sums of tiles whose contraction is dealt to several workgroups
};

// The products: x with both weights; dy with w_down; dgate and dup with theirs.
enum GatedPass { kForward, kHidden, kInput };
dp_status launch_gated_tiles(const GatedArgs& a, dp_dtype dt, GatedPass pass, hipStream_t s);      // 16-bit types (gated_tiles.hip)
// How a pass is launched: the kernel, its tiles of one workgroup each, large and small, and those that several share.
enum GatedKernel { kGatedTiles16 = 0, kGatedFew = 1, kGatedTiles32 = 2 };
struct GatedLaunches {
  int kernel;
  int64_t large, small, dealt;
  int parts, side;                                     // of the dealt ones
};
GatedLaunches gated_tiles_launches(GatedPass pass, int rows, int d, int f, int d_out);
GatedLaunches gated_launches(dp_dtype dt, GatedPass pass, int rows, int d, int f, int d_out);
size_t gated_tiles_workspace(GatedPass pass, int rows, int d, int f, int d_out);                   // bytes of `partial`
size_t gated_workspace(dp_dtype dt, GatedPass pass, int rows, int d, int f, int d_out);            // of any type
constexpr int kGatedFewRows = 64;
dp_status launch_gated_few(const GatedArgs& a, dp_dtype dt, GatedPass pass, hipStream_t s);        // up to kGatedFewRows of them (gated_few.hip)
dp_status launch_gated_forward(const GatedArgs& a, dp_dtype dt, hipStream_t s);
dp_status launch_gated_backward(const GatedArgs& a, dp_dtype dt, hipStream_t s);

// The gate's activation: its value and, where asked for, its slope.  All but relu are shares of their argument (sigmoid: the share itself).
//
// EXACT, for fp32 results: written with exp(-|v|), so that neither a share nor its complement is a difference.  For 16-bit ones some 2^-23 of 1 is
// enough of a share, which takes half the instructions (not of sigmoid's slope, which is all there is where the share is next to 1: as the exact one);
// gelu's is then Hastings' approximation of the normal distribution's tail (Abramowitz and Stegun, 7.1.26: within 1.5e-7), whose exponential is its
// slope's as well.
template <int ACT, bool EXACT, bool SLOPE>
__device__ __forceinline__ float activation(float x, float& slope) {
  constexpr float kLog2e = 1.44269504088896340736f;
  if constexpr (ACT == DP_ACT_RELU) {
    slope = x > 0.f ? 1.f : 0.f;
    return x < 0.f ? 0.f : x;
  } else if constexpr (ACT == DP_ACT_GELU) {
    constexpr float kDensity = 0.39894228040143267794f, kRoot = 0.70710678118654752440f;
    if constexpr (EXACT) {
      const float share = 0.5f * erfcf(-kRoot * x);
      if (SLOPE) slope = fmaf(x * kDensity, expf(-0.5f * x * x), share);
      return x * share;
    } else {
      const float e = __builtin_amdgcn_exp2f(-0.5f * kLog2e * x * x), t = __builtin_amdgcn_rcpf(fmaf(0.3275911f * kRoot, fabsf(x), 1.f));
      float tail = fmaf(t, 0.5f * 1.061405429f, 0.5f * -1.453152027f);
      tail = fmaf(t, tail, 0.5f * 1.421413741f);
      tail = fmaf(t, tail, 0.5f * -0.284496736f);
      tail = fmaf(t, tail, 0.5f * 0.254829592f) * t * e;
      const float share = x < 0.f ? tail : 1.f - tail;
      if (SLOPE) slope = fmaf(x * kDensity, e, share);
      return x * share;
    }
  } else {
    float v = x, dv = 1.f;
    if constexpr (ACT == DP_ACT_GELU_TANH) {           // 1 + tanh(u) = 2 share(2 u)
      constexpr float c = 1.59576912160573071176f, c3 = c * 0.044715f;
      v = x * fmaf(c3, x * x, c);
      dv = fmaf(3.f * c3, fminf(x * x, 1e30f), c);     // (finite: it meets shares of zero)
    }
    float share, rise;
    if constexpr (EXACT) {
      const float e = expf(-fabsf(v)), r = 1.f / (1.f + e);
      share = v < 0.f ? e * r : r;
      rise = e * r * r * dv;                           // share (1 - share) dv
    } else if constexpr (ACT == DP_ACT_SIGMOID && SLOPE) {
      const float e = __builtin_amdgcn_exp2f(-kLog2e * fabsf(v)), r = __builtin_amdgcn_rcpf(1.f + e);
      share = v < 0.f ? e * r : r;
      rise = e * r * r;
    } else {
      share = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * v));
      rise = fmaf(-share, share, share) * dv;
    }
    if constexpr (ACT == DP_ACT_SIGMOID) {
      slope = rise;
      return share;
    } else {
      slope = fmaf(x, rise, share);
      return x * share;
    }
  }
}

// f(std::integral_constant<int, act>): the branch is taken once for all of a kernel's values.
template <class F>
__device__ __forceinline__ void with_activation(int act, F f) {
  if (act == DP_ACT_SILU)
    f(std::integral_constant<int, DP_ACT_SILU>{});
  else if (act == DP_ACT_GELU)
    f(std::integral_constant<int, DP_ACT_GELU>{});
  else if (act == DP_ACT_GELU_TANH)
    f(std::integral_constant<int, DP_ACT_GELU_TANH>{});
  else if (act == DP_ACT_RELU)
    f(std::integral_constant<int, DP_ACT_RELU>{});
  else
    f(std::integral_constant<int, DP_ACT_SIGMOID>{});
}

}  // namespace dpbk
