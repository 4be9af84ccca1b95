// Entry points of what gated transformer blocks run besides: heads' rotation and norms, gated feed-forward layers, orthogonalised updates.
// Arguments are checked here, on the host, before anything is launched.
#include <float.h>
#include <math.h>

#include <algorithm>

#include "gated.h"
#include "heads.h"
#include "muon.h"

using namespace dpbk;

namespace {

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
bool dtype_ok(dp_dtype dt) { return dt == DP_F32 || dt == DP_BF16 || dt == DP_F16; }
uintptr_t alignment(dp_dtype dt) { return dt == DP_F32 ? 4 : 16; }
bool there(const void* p, dp_dtype dt) { return p && aligned(p, alignment(dt)); }

// Both sides' sizes and strides; `backward`: results are read and inputs written.
dp_status heads_args(const dp_heads_shape* p, dp_dtype dt, bool backward, HeadsArgs& a) {
  if (!p || !dtype_ok(dt)) return DP_ERR_INVALID_ARG;
  const dp_heads_shape& s = *p;
  if (s.B <= 0 || s.T <= 0 || s.H <= 0 || s.H_kv < 0 || s.D <= 0) return DP_ERR_INVALID_ARG;
  if (s.rotary < 0 || s.rotary > s.D || s.rotary % 2 || (s.interleaved != 0 && s.interleaved != 1)) return DP_ERR_INVALID_ARG;
  if (s.rotary && (!s.turns || !aligned(s.turns, 8) || !isfinite(s.amplitude))) return DP_ERR_INVALID_ARG;
  if (!aligned(s.position, 4) || !aligned(s.len, 4) || (dt != DP_F32 && s.D % 8)) return DP_ERR_INVALID_ARG;
  const int64_t* strides[] = {s.q_stride, s.k_stride, s.q_out_stride, s.k_out_stride};
  for (int n = 0; n < 4; ++n) {
    if (n % 2 && s.H_kv == 0) continue;
    for (int i = 0; i < 3; ++i)
      if (strides[n][i] < 0 || strides[n][i] > (int64_t)1 << 40 || (dt != DP_F32 && strides[n][i] % 8)) return DP_ERR_INVALID_ARG;
  }
  if (s.D > kHeadsMaxWidth || s.B > kHeadsMostSamples || (int64_t)s.B * s.T > INT32_MAX || (int64_t)s.H + s.H_kv > 1 << 20) return DP_ERR_UNSUPPORTED;
  a = HeadsArgs{};
  a.heads[0] = s.H;
  a.heads[1] = s.H_kv;
  a.B = s.B;
  a.T = s.T;
  a.D = s.D;
  a.turn = s.rotary;
  a.interleaved = s.interleaved;
  a.amplitude = s.amplitude;
  a.turns = s.turns;
  a.position = s.position;
  a.len = s.len;
  for (int w = 0; w < (s.H_kv ? 2 : 1); ++w) {
    const int64_t *in = strides[w], *out = strides[2 + w];
    a.in_stride[w] = {in[0], in[1], in[2]};
    a.out_stride[w] = {out[0], out[1], out[2]};
    if (backward) std::swap(a.in_stride[w], a.out_stride[w]);
    // what is written does not overlap itself: by growing stride, each axis steps over all that the ones before span
    struct { int64_t stride, n; } axes[] = {{a.out_stride[w].sample, s.B}, {a.out_stride[w].token, s.T}, {a.out_stride[w].head, a.heads[w]}};
    std::sort(axes, axes + 3, [](const auto& x, const auto& y) { return x.stride < y.stride; });
    __int128 span = s.D;
    for (const auto& axis : axes) {
      if (axis.n == 1) continue;
      if (axis.stride < span) return DP_ERR_INVALID_ARG;
      span += (__int128)axis.stride * (axis.n - 1);
    }
  }
  return DP_OK;
}

bool sides_there(const HeadsArgs& a, dp_dtype dt, const void* q, const void* k) { return there(q, dt) && (a.heads[1] == 0 || there(k, dt)); }

// Sums of a chunk's gains: a side's chunks are no more than its bound and one more for each sample, nor than tokens.
size_t head_norm_workspace(const HeadsArgs& a) {
  const int64_t chunks = std::min((int64_t)a.B * a.T, (int64_t)kHeadsGradChunks + a.B);
  return (size_t)chunks * (a.heads[1] ? 2 : 1) * a.D * sizeof(float);
}

dp_status rotate(const dp_heads_shape* shape, dp_dtype dt, bool backward, const void* q, const void* k, void* q_out, void* k_out, void* stream) {
  HeadsArgs a;
  const dp_status st = heads_args(shape, dt, backward, a);
  if (st != DP_OK) return st;
  if (!sides_there(a, dt, q, k) || !sides_there(a, dt, q_out, k_out)) return DP_ERR_INVALID_ARG;
  a.in[0] = q;
  a.in[1] = k;
  a.out[0] = q_out;
  a.out[1] = k_out;
  a.back = backward;
  return launch_heads(a, dt, kRotate, static_cast<hipStream_t>(stream));
}

constexpr int kGatedMost = 1 << 20;

dp_status gated_shape(dp_dtype dt, int rows, int d, int f, int d_out) {
  if (!dtype_ok(dt) || rows <= 0 || d <= 0 || f <= 0 || d_out <= 0) return DP_ERR_INVALID_ARG;
  if (dt != DP_F32 && (d % 8 || f % 8 || d_out % 8)) return DP_ERR_INVALID_ARG;
  if (d > kGatedMost || f > kGatedMost || d_out > kGatedMost || rows > 1 << 28) return DP_ERR_UNSUPPORTED;
  // workgroups of the smallest tiles
  if (((int64_t)rows + 63) / 64 * ((std::max(d, f) + 63) / 64) > INT32_MAX || (int64_t)rows * f / 256 > INT32_MAX) return DP_ERR_UNSUPPORTED;
  return DP_OK;
}
// Both passes use the same memory, one after the other.
size_t gated_backward_workspace(dp_dtype dt, int rows, int d, int f, int d_out, bool input) {
  return std::max(d_out ? gated_workspace(dt, kHidden, rows, d, f, d_out) : 0, input ? gated_workspace(dt, kInput, rows, d, f, d_out) : 0);
}
dp_status scratch_ok(const void* ws, size_t ws_bytes, size_t need) {
  if (need == 0) return DP_OK;
  if (!ws || ws_bytes < need) return DP_ERR_WORKSPACE;
  return aligned(ws, 16) ? DP_OK : DP_ERR_INVALID_ARG;
}
bool act_ok(dp_activation act) { return act >= DP_ACT_SILU && act <= DP_ACT_SIGMOID; }

// Matrices of a step, as far as their sizes go.
dp_status muon_sizes(const dp_muon_tensor* tensors, int n) {
  if (!tensors || n <= 0) return DP_ERR_INVALID_ARG;
  for (int i = 0; i < n; ++i) {
    const int rows = tensors[i].rows, cols = tensors[i].cols;
    if (rows <= 0 || cols <= 0) return DP_ERR_INVALID_ARG;
    if (rows > kMuonMostSide || cols > kMuonMostSide || std::min(rows, cols) > kMuonMostShort) return DP_ERR_UNSUPPORTED;
  }
  return n <= 1 << 20 ? DP_OK : DP_ERR_UNSUPPORTED;
}

// The matrices in runs of as many as travel together, those that one workgroup holds by themselves; weight decay and scale where the launcher
// wants what comes of them.
template <class F>
dp_status muon_runs(const dp_muon_tensor* tensors, int n, F run) {
  MuonTensor t[kMuonGroup];
  for (const bool small : {false, true}) {
    int total = 0, done = 0, count = 0;
    for (int i = 0; i < n; ++i) total += muon_is_small(tensors[i].rows, tensors[i].cols) == small;
    const int runs = (total + kMuonGroup - 1) / kMuonGroup, per = total ? (total + runs - 1) / runs : 0;
    for (int i = 0; i < n; ++i) {
      const dp_muon_tensor& from = tensors[i];
      if (muon_is_small(from.rows, from.cols) != small) continue;
      t[count++] = {from.param, from.grad, from.m, from.copy, from.rows, from.cols, from.weight_decay, from.scale};
      if (++done < total && count < per) continue;
      const dp_status st = run(t, count, small);
      if (st != DP_OK) return st;
      count = 0;
    }
  }
  return DP_OK;
}

// Where singular values from [0, 1] go under x <- a x + b x^3 + c x^5: x, x^2 and a + b x^2 + c x^4 stay within what two halves hold.
bool muon_values_fit(const double* abc, int iterations) {
  double most = 1.;
  for (int k = 0; k < iterations; ++k) {
    const double a = abc[3 * k], b = abc[3 * k + 1], c = abc[3 * k + 2], end = most * most;
    if (!(fabs(a) <= FLT_MAX && fabs(b) <= FLT_MAX && fabs(c) <= FLT_MAX && end <= kMuonMost)) return false;      // (kernels take fp32; NaN as well)
    double next = 0., poly = 0.;
    auto at = [&](double s) {                          // s = x^2
      if (!(s >= 0. && s <= end)) return;
      const double p = a + s * (b + c * s);
      poly = std::max(poly, fabs(p));
      next = std::max(next, sqrt(s) * fabs(p));
    };
    at(0.);
    at(end);
    // where the polynomial of A turns, and where x's does: a + 3 b s + 5 c s^2 = 0, by the sum of two terms of one sign, so that neither
    // root is lost where c is next to nothing
    if (c != 0.) at(-b / (2. * c));
    const double q = -0.5 * (3. * b + copysign(sqrt(std::max(0., 9. * b * b - 20. * a * c)), b));
    if (c != 0.) at(q / (5. * c));
    if (q != 0.) at(a / q);
    if (!(poly <= kMuonMost && next <= kMuonMost)) return false;
    most = next * 1.001;                               // what rounding adds
  }
  return true;
}

}  // namespace

extern "C" {

dp_status dp_rotary_turns(double* turns, int rotary, double base, dp_rotary_scaling scaling, double factor, double original, double slow,
                          double fast) {
  if (!turns || rotary < 0 || rotary % 2 || !(base > 0.) || isinf(base)) return DP_ERR_INVALID_ARG;
  if (scaling < DP_ROTARY_PLAIN || scaling > DP_ROTARY_PARTS) return DP_ERR_INVALID_ARG;
  if (scaling != DP_ROTARY_PLAIN && (!(factor > 0.) || isinf(factor))) return DP_ERR_INVALID_ARG;
  if (scaling == DP_ROTARY_PARTS && (!(original > 0.) || isinf(original) || !(slow < fast) || isinf(slow) || isinf(fast))) return DP_ERR_INVALID_ARG;
  if (scaling == DP_ROTARY_BASE && rotary > 2) base *= pow(factor, rotary / (rotary - 2.));
  for (int i = 0; i < rotary / 2; ++i) {
    const double t = pow(base, -2. * i / rotary) / 6.283185307179586476925;
    turns[i] = t;
    if (scaling == DP_ROTARY_LINEAR) turns[i] = t / factor;
    if (scaling == DP_ROTARY_PARTS) {
      const double keep = std::min(1., std::max(0., (t * original - slow) / (fast - slow)));
      turns[i] = t / factor * (1. - keep) + t * keep;
    }
  }
  return DP_OK;
}

dp_status dp_rotary(const dp_heads_shape* shape, dp_dtype dt, const void* q, const void* k, void* q_out, void* k_out, void* stream) {
  return rotate(shape, dt, false, q, k, q_out, k_out, stream);
}

dp_status dp_rotary_backward(const dp_heads_shape* shape, dp_dtype dt, const void* dq_out, const void* dk_out, void* dq, void* dk,
                             void* stream) {
  return rotate(shape, dt, true, dq_out, dk_out, dq, dk, stream);
}

dp_status dp_head_norm(const dp_heads_shape* shape, dp_dtype dt, const void* q, const void* k, const float* q_gain, const float* k_gain,
                       float eps, void* q_out, void* k_out, void* stream) {
  HeadsArgs a;
  const dp_status st = heads_args(shape, dt, false, a);
  if (st != DP_OK) return st;
  if (!sides_there(a, dt, q, k) || !sides_there(a, dt, q_out, k_out) || !aligned(q_gain, 4) || !aligned(k_gain, 4)) return DP_ERR_INVALID_ARG;
  if (!(eps >= 0.f) || isinf(eps)) return DP_ERR_INVALID_ARG;
  a.in[0] = q;
  a.in[1] = k;
  a.out[0] = q_out;
  a.out[1] = k_out;
  a.gain[0] = q_gain;
  a.gain[1] = k_gain;
  a.eps = eps;
  return launch_heads(a, dt, kNorm, static_cast<hipStream_t>(stream));
}

size_t dp_head_norm_workspace_bytes(const dp_heads_shape* shape, dp_dtype dt) {
  HeadsArgs a;
  return heads_args(shape, dt, true, a) == DP_OK ? head_norm_workspace(a) : 0;
}

dp_status dp_head_norm_backward(const dp_heads_shape* shape, dp_dtype dt, const void* q, const void* k, const void* dq_out,
                                const void* dk_out, const float* q_gain, const float* k_gain, float eps, void* dq, void* dk, float* kept,
                                float* sqnorm_out, void* ws, size_t ws_bytes, void* stream) {
  HeadsArgs a;
  const dp_status st = heads_args(shape, dt, true, a);
  if (st != DP_OK) return st;
  if (!sides_there(a, dt, q, k) || !sides_there(a, dt, dq_out, dk_out) || !sides_there(a, dt, dq, dk)) return DP_ERR_INVALID_ARG;
  if (!aligned(q_gain, 4) || !aligned(k_gain, 4) || !kept != !sqnorm_out || !aligned(kept, 4) || !aligned(sqnorm_out, 4)) return DP_ERR_INVALID_ARG;
  if (!(eps >= 0.f) || isinf(eps)) return DP_ERR_INVALID_ARG;
  if (kept) {
    if (!ws || ws_bytes < head_norm_workspace(a)) return DP_ERR_WORKSPACE;
    if (!aligned(ws, 16)) return DP_ERR_INVALID_ARG;
  }
  for (int w = 0; w < 2; ++w) {
    a.dy_stride[w] = a.in_stride[w];                 // (heads_args: results' strides)
    a.in_stride[w] = a.out_stride[w];
  }
  a.in[0] = q;
  a.in[1] = k;
  a.dy[0] = dq_out;
  a.dy[1] = dk_out;
  a.out[0] = dq;
  a.out[1] = dk;
  a.gain[0] = q_gain;
  a.gain[1] = k_gain;
  a.eps = eps;
  a.back = 1;
  a.kept = kept;
  a.sqnorm = sqnorm_out;
  a.partial = static_cast<float*>(ws);
  return launch_heads(a, dt, kNormGrad, static_cast<hipStream_t>(stream));
}

size_t dp_gated_workspace_bytes(dp_dtype dt, int rows, int d, int f) {
  return gated_shape(dt, rows, d, f, d) == DP_OK ? gated_workspace(dt, kForward, rows, d, f, d) : 0;
}

dp_status dp_gated(const void* x, dp_dtype dt, int rows, int d, int f, const void* w_gate, const void* w_up, const void* b_gate,
                   const void* b_up, dp_activation act, void* gate, void* up, void* h, void* ws, size_t ws_bytes, void* stream) {
  const dp_status st = gated_shape(dt, rows, d, f, d);
  if (st != DP_OK) return st;
  if (!act_ok(act) || !there(x, dt) || !there(w_gate, dt) || !there(w_up, dt) || !there(h, dt) || !gate != !up) return DP_ERR_INVALID_ARG;
  for (const void* p : {b_gate, b_up, (const void*)gate, (const void*)up})
    if (!aligned(p, alignment(dt))) return DP_ERR_INVALID_ARG;
  const dp_status scratch = scratch_ok(ws, ws_bytes, gated_workspace(dt, kForward, rows, d, f, d));
  if (scratch != DP_OK) return scratch;
  GatedArgs a = {};
  a.partial = static_cast<float*>(ws);
  a.x = x;
  a.w_gate = w_gate;
  a.w_up = w_up;
  a.b_gate = b_gate;
  a.b_up = b_up;
  a.gate = gate;
  a.up = up;
  a.h = h;
  a.rows = rows;
  a.d = d;
  a.f = f;
  a.act = act;
  return launch_gated_forward(a, dt, static_cast<hipStream_t>(stream));
}

size_t dp_gated_backward_workspace_bytes(dp_dtype dt, int rows, int d, int f, int d_out) {
  if (gated_shape(dt, rows, d, f, d_out == 0 ? d : d_out) != DP_OK) return 0;
  return gated_backward_workspace(dt, rows, d, f, d_out, true);
}

dp_status dp_gated_backward(const void* dy, const void* w_down, int d_out, const void* gate, const void* up, dp_dtype dt, int rows, int d,
                            int f, const void* w_gate, const void* w_up, dp_activation act, void* dgate, void* dup, void* dx, void* ws,
                            size_t ws_bytes, void* stream) {
  const dp_status st = gated_shape(dt, rows, d, f, w_down ? d_out : d);
  if (st != DP_OK) return st;
  if (!act_ok(act) || !aligned(w_down, alignment(dt)) || !aligned(dx, alignment(dt))) return DP_ERR_INVALID_ARG;
  for (const void* p : {dy, gate, up, (const void*)dgate, (const void*)dup})
    if (!there(p, dt)) return DP_ERR_INVALID_ARG;
  if (dx && (!there(w_gate, dt) || !there(w_up, dt))) return DP_ERR_INVALID_ARG;
  const dp_status scratch = scratch_ok(ws, ws_bytes, gated_backward_workspace(dt, rows, d, f, w_down ? d_out : 0, dx != nullptr));
  if (scratch != DP_OK) return scratch;
  GatedArgs a = {};
  a.dy = dy;
  a.w_down = w_down;
  a.d_out = d_out;
  a.gate = const_cast<void*>(gate);
  a.up = const_cast<void*>(up);
  a.w_gate = w_gate;
  a.w_up = w_up;
  a.dgate = dgate;
  a.dup = dup;
  a.dx = dx;
  a.partial = static_cast<float*>(ws);
  a.rows = rows;
  a.d = d;
  a.f = f;
  a.act = act;
  return launch_gated_backward(a, dt, static_cast<hipStream_t>(stream));
}

dp_status dp_gated_launches(dp_dtype dt, int rows, int d, int f, int d_out, int pass, int32_t* launches) {
  const dp_status st = gated_shape(dt, rows, d, f, pass == kHidden ? d_out : d);
  if (st != DP_OK) return st;
  if (pass < kForward || pass > kInput || !launches) return DP_ERR_INVALID_ARG;
  const GatedLaunches l = gated_launches(dt, (GatedPass)pass, rows, d, f, d_out);
  const int64_t all[6] = {l.kernel, l.large, l.small, l.dealt, l.parts, l.side};
  for (int i = 0; i < 6; ++i) launches[i] = (int32_t)std::min<int64_t>(all[i], INT32_MAX);
  return DP_OK;
}

size_t dp_muon_workspace_bytes(const dp_muon_tensor* tensors, int n_tensors) {
  if (muon_sizes(tensors, n_tensors) != DP_OK) return 0;
  size_t most = 0;
  muon_runs(tensors, n_tensors, [&](const MuonTensor* run, int n, bool small) {
    most = std::max(most, small ? (size_t)16 : muon_workspace(run, n));
    return DP_OK;
  });
  return most;
}

dp_status dp_muon_launches(const dp_muon_tensor* tensors, int n_tensors, int32_t* launches) {
  const dp_status st = muon_sizes(tensors, n_tensors);
  if (st != DP_OK) return st;
  if (!launches) return DP_ERR_INVALID_ARG;
  std::fill(launches, launches + 7, 0);
  int runs = 0;
  muon_runs(tensors, n_tensors, [&](const MuonTensor* run, int n, bool small) {
    if (small) {
      launches[0] += n;
    } else if (++runs == 1) {
      MuonLaunches steps[3];
      muon_launches(run, n, steps);
      for (int i = 0; i < 3; ++i) launches[1 + 2 * i] = steps[i].side, launches[2 + 2 * i] = steps[i].parts;
    }
    return DP_OK;
  });
  return DP_OK;
}

dp_status dp_muon_multi(const dp_muon_tensor* tensors, int n_tensors, dp_dtype grad_dt, dp_dtype copy_dt, double lr, double beta, int nesterov,
                        double grad_scale, double eps, const double* coefficients, int iterations, void* ws, size_t ws_bytes, void* stream) {
  if (!dtype_ok(grad_dt) || !dtype_ok(copy_dt) || !coefficients || iterations < 1 || iterations > kMuonMostIterations) return DP_ERR_INVALID_ARG;
  if (nesterov != 0 && nesterov != 1) return DP_ERR_INVALID_ARG;
  if (!(lr >= 0.) || isinf(lr) || !(beta >= 0. && beta < 1.) || !(eps >= 0.) || isinf(eps) || !isfinite(grad_scale)) return DP_ERR_INVALID_ARG;
  dp_status st = muon_sizes(tensors, n_tensors);
  if (st != DP_OK) return st;
  const uintptr_t grad_size = grad_dt == DP_F32 ? 4 : 2;
  for (int i = 0; i < n_tensors; ++i) {
    const dp_muon_tensor& t = tensors[i];
    if (!t.param || !t.grad || !t.m || !aligned(t.param, 4) || !aligned(t.grad, grad_size) || !aligned(t.m, 4)) return DP_ERR_INVALID_ARG;
    if (copy_dt != DP_F32 && (!t.copy || !aligned(t.copy, 2))) return DP_ERR_INVALID_ARG;
    if (!isfinite(t.weight_decay) || !isfinite(t.scale)) return DP_ERR_INVALID_ARG;
  }
  if (!muon_values_fit(coefficients, iterations)) return DP_ERR_UNSUPPORTED;
  if (!ws || ws_bytes < dp_muon_workspace_bytes(tensors, n_tensors)) return DP_ERR_WORKSPACE;
  if (!aligned(ws, 16)) return DP_ERR_INVALID_ARG;
  MuonArgs a = {};
  a.beta = (float)beta;
  a.ahead = nesterov ? (float)beta : -1.f;
  a.grad_scale = (float)grad_scale;
  a.eps = (float)eps;
  a.iterations = iterations;
  a.coefficients = coefficients;
  return muon_runs(tensors, n_tensors, [&](MuonTensor* run, int n, bool small) {
    for (int i = 0; i < n; ++i) run[i].keep = (float)(1. - lr * (double)run[i].keep), run[i].rate = (float)(lr * (double)run[i].rate);
    if (small) return launch_muon_small(run, n, a, grad_dt, copy_dt, static_cast<hipStream_t>(stream));
    return launch_muon(run, n, a, grad_dt, copy_dt, ws, static_cast<hipStream_t>(stream));
  });
}

}  // extern "C"
