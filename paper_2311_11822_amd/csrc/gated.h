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
  float* partial;                                      // dx: [parts, rows, d] where the contraction is dealt to several workgroups
};

// The products: x with both weights; dy with w_down; dgate and dup with theirs.
enum GatedPass { kForward, kHidden, kInput };
dp_status launch_gated_tiles(const GatedArgs& a, dp_dtype dt, GatedPass pass, hipStream_t s);      // 16-bit types (gated_tiles.hip)
size_t gated_input_workspace(int rows, int d, int f, int d_out);                                   // of their input gradients: `partial`
constexpr int kGatedFewRows = 64;
dp_status launch_gated_few(const GatedArgs& a, dp_dtype dt, GatedPass pass, hipStream_t s);        // up to kGatedFewRows of them (gated_few.hip)
dp_status launch_gated_forward(const GatedArgs& a, dp_dtype dt, hipStream_t s);
dp_status launch_gated_backward(const GatedArgs& a, dp_dtype dt, hipStream_t s);

// The gate's activation: its value and, where asked for, its slope.  All but relu are shares of their argument (sigmoid: the share
// itself), written with exp(-|v|) so that neither a share nor its complement is a difference.
template <bool EXACT>                                  // fp32 results; 16-bit ones round more than the shorter exponential errs
__device__ __forceinline__ float act_exp(float x) {
  return EXACT ? expf(x) : __expf(x);
}
template <bool EXACT, bool SLOPE>
__device__ __forceinline__ float activation(int act, float x, float& slope) {
  if (act == DP_ACT_RELU) {
    slope = x > 0.f ? 1.f : 0.f;
    return x < 0.f ? 0.f : x;
  }
  if (act == DP_ACT_GELU) {
    const float share = 0.5f * erfcf(-0.70710678118654752440f * x);
    if (SLOPE) slope = fmaf(x * 0.39894228040143267794f, act_exp<EXACT>(-0.5f * x * x), share);
    return x * share;
  }
  float v = x, dv = 1.f;
  if (act == DP_ACT_GELU_TANH) {                       // 1 + tanh(u) = 2 share(2 u)
    constexpr float c = 1.59576912160573071176f, c3 = c * 0.044715f;
    v = x * fmaf(c3, x * x, c);
    dv = fmaf(3.f * c3, x * x, c);
  }
  const float e = act_exp<EXACT>(-fabsf(v)), r = EXACT ? 1.f / (1.f + e) : __builtin_amdgcn_rcpf(1.f + e);
  const float share = v < 0.f ? e * r : r;
  const float rise = e * r * r * dv;                   // share (1 - share) dv
  if (act == DP_ACT_SIGMOID) {
    slope = rise;
    return share;
  }
  slope = fmaf(x, rise, share);
  return x * share;
}

}  // namespace dpbk
