// Entry points of what stands around the linear layers: layer norms, attention, the optimizer.  Arguments are checked here, on the
// host, before anything is launched.
#include <math.h>

#include <algorithm>

#include "attention.h"
#include "train.h"

using namespace dpbk;

namespace {

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
bool dtype_ok(dp_dtype dt) { return dt == DP_F32 || dt == DP_BF16 || dt == DP_F16; }

// DP_OK where a layer norm of these sizes has a kernel.
dp_status norm_shape(dp_dtype dt, int B, int T, int d) {
  if (!dtype_ok(dt) || B <= 0 || T <= 0 || d <= 0) return DP_ERR_INVALID_ARG;
  if (d > kNormMaxWidth || (int64_t)B * T > INT32_MAX) return DP_ERR_UNSUPPORTED;
  return DP_OK;
}

size_t norm_workspace(dp_dtype dt, int B, int T, int d) {
  const int chunks = layer_norm_chunks(dt, B, T, d);
  return chunks > 1 ? (size_t)B * chunks * 2 * d * sizeof(float) : 16;
}

// Fills in what the two attention calls have in common.
dp_status attention_args(const dp_attention_shape* p, dp_dtype dt, AttnArgs& a) {
  if (!p || !dtype_ok(dt)) return DP_ERR_INVALID_ARG;
  const dp_attention_shape& s = *p;
  if (s.B <= 0 || s.H <= 0 || s.H_kv <= 0 || s.Tq <= 0 || s.Tk <= 0 || s.D <= 0 || s.H % s.H_kv) return DP_ERR_INVALID_ARG;
  if (s.causal != 0 && s.causal != 1) return DP_ERR_INVALID_ARG;
  if (!(s.scale > 0.f) || isinf(s.scale)) return DP_ERR_INVALID_ARG;
  const int64_t* strides[] = {s.q_stride, s.k_stride, s.v_stride, s.o_stride};
  const int32_t tokens[] = {s.Tq, s.Tk, s.Tk, s.Tq};
  for (int n = 0; n < 4; ++n) {
    for (int i = 0; i < 3; ++i)
      if (strides[n][i] < 0 || (dt != DP_F32 && strides[n][i] % 8)) return DP_ERR_INVALID_ARG;
    if (tokens[n] > 1 && strides[n][1] < s.D) return DP_ERR_INVALID_ARG;
  }
  if (!aligned(s.q_len, 4) || !aligned(s.k_len, 4)) return DP_ERR_INVALID_ARG;
  if (dt != DP_F32 && s.D % 8) return DP_ERR_INVALID_ARG;
  if (s.D > 128 || s.Tq > 1 << 30 || s.Tk > 1 << 30) return DP_ERR_UNSUPPORTED;
  for (int n = 0; n < 4; ++n)
    // 128 rows of 16 bits, 64 of fp32, lie within 2^31 bytes: what a tile is at most, but for the split forms, whose rule looks at strides itself
    if (tokens[n] > 1 && strides[n][1] > 1 << 23) return DP_ERR_UNSUPPORTED;
  const int64_t rows = s.Tq > s.Tk ? s.Tq : s.Tk;
  if ((int64_t)s.B * s.H > (1 << 30) || ((int64_t)s.B * s.H + 7) * ((rows + 3) / 4) > INT32_MAX) return DP_ERR_UNSUPPORTED;
  a = AttnArgs{};
  a.q_len = s.q_len;
  a.k_len = s.k_len;
  a.B = s.B;
  a.H = s.H;
  a.H_kv = s.H_kv;
  a.share = s.H / s.H_kv;
  a.Tq = s.Tq;
  a.Tk = s.Tk;
  a.D = s.D;
  a.causal = s.causal;
  a.scale = s.scale;
  a.scale2 = s.scale * kLog2e;
  AttnSide* sides[] = {&a.qs, &a.ks, &a.vs, &a.os};
  for (int i = 0; i < 4; ++i) *sides[i] = {strides[i][0], tokens[i] > 1 ? strides[i][1] : s.D, strides[i][2]};
  return DP_OK;
}

// The backward pass's workspace: rows' corrections, in whole 16 bytes, then partial sums.
int64_t padded_rows(const AttnArgs& a) { return ((int64_t)2 * a.B * a.H * a.Tq + 3) / 4 * 4; }
int parts_of(const AttnArgs& a, dp_dtype dt) { return dt != DP_F32 || whole_pieces(a) ? attention_parts(a) : 1; }
size_t backward_workspace(const AttnArgs& a, dp_dtype dt) {
  return (size_t)(padded_rows(a) + (parts_of(a, dt) > 1 ? attention_partial_floats(a) : 0)) * sizeof(float);
}

// No two elements of an array that is written share a place: by growing stride, each axis steps over all that the ones before span.
bool apart(const AttnSide& s, int B, int T, int H, int D) {
  struct { int64_t stride, n; } axes[] = {{s.sample, B}, {s.token, T}, {s.head, H}};
  std::sort(axes, axes + 3, [](const auto& a, const auto& b) { return a.stride < b.stride; });
  int64_t span = D;
  for (const auto& axis : axes) {
    if (axis.n == 1) continue;
    if (axis.stride < span) return false;
    span += axis.stride * (axis.n - 1);
  }
  return true;
}

template <class... P>
bool all_there(uintptr_t to, P... p) {
  return ((p && aligned(p, to)) && ...);
}
uintptr_t attention_alignment(dp_dtype dt) { return dt == DP_F32 ? 4 : 16; }

}  // namespace

extern "C" {

dp_status dp_layer_norm(const void* x, const void* add, dp_dtype dt, int B, int T, int d, const float* gain, const float* bias,
                        float eps, void* sum, void* y, float* mean, float* rstd, void* stream) {
  if (!all_there(16, x, y) || !aligned(add, 16) || !aligned(sum, 16) || !add != !sum) return DP_ERR_INVALID_ARG;
  if (!aligned(gain, 4) || !aligned(bias, 4) || !aligned(mean, 4) || !aligned(rstd, 4)) return DP_ERR_INVALID_ARG;
  if (!(eps >= 0.f) || isinf(eps)) return DP_ERR_INVALID_ARG;
  const dp_status st = norm_shape(dt, B, T, d);
  if (st != DP_OK) return st;
  NormArgs a = {};
  a.x = x;
  a.add = add;
  a.sum = sum;
  a.out = y;
  a.gain = gain;
  a.bias = bias;
  a.mean = mean;
  a.rstd = rstd;
  a.B = B;
  a.T = T;
  a.d = d;
  a.eps = eps;
  return launch_layer_norm(a, dt, static_cast<hipStream_t>(stream));
}

size_t dp_layer_norm_workspace_bytes(dp_dtype dt, int B, int T, int d) {
  return norm_shape(dt, B, T, d) == DP_OK ? norm_workspace(dt, B, T, d) : 0;
}

dp_status dp_layer_norm_backward(const void* x, const void* dy, const void* add, dp_dtype dt, int B, int T, int d, const float* gain,
                                 const float* mean, const float* rstd, void* dx, float* kept, float* sqnorm_out, void* ws,
                                 size_t ws_bytes, void* stream) {
  if (!all_there(16, x, dy) || !mean || !rstd || (!dx && !kept) || !kept != !sqnorm_out || (add && !dx)) return DP_ERR_INVALID_ARG;
  if (!aligned(add, 16) || !aligned(dx, 16) || !aligned(kept, 16)) return DP_ERR_INVALID_ARG;
  if (!aligned(gain, 4) || !aligned(mean, 4) || !aligned(rstd, 4) || !aligned(sqnorm_out, 4)) return DP_ERR_INVALID_ARG;
  const dp_status st = norm_shape(dt, B, T, d);
  if (st != DP_OK) return st;
  if (kept) {
    if (!ws || ws_bytes < norm_workspace(dt, B, T, d)) return DP_ERR_WORKSPACE;
    if (!aligned(ws, 16)) return DP_ERR_INVALID_ARG;
  }
  NormArgs a = {};
  a.x = x;
  a.dy = dy;
  a.add = add;
  a.out = dx;
  a.gain = gain;
  a.mean = const_cast<float*>(mean);
  a.rstd = const_cast<float*>(rstd);
  a.kept = kept;
  a.partial = static_cast<float*>(ws);
  a.sqnorm = sqnorm_out;
  a.B = B;
  a.T = T;
  a.d = d;
  return launch_layer_norm_backward(a, dt, static_cast<hipStream_t>(stream));
}

size_t dp_attention_workspace_bytes(const dp_attention_shape* shape, dp_dtype dt) {
  AttnArgs a;
  if (attention_args(shape, dt, a) != DP_OK) return 0;
  attention_key_parts(a, dt);
  return (size_t)attention_key_floats(a) * sizeof(float);
}

dp_status dp_attention(const dp_attention_shape* shape, dp_dtype dt, const void* q, const void* k, const void* v, void* o, float* lse,
                       void* ws, size_t ws_bytes, void* stream) {
  AttnArgs a;
  const dp_status st = attention_args(shape, dt, a);
  if (st != DP_OK) return st;
  if (!all_there(attention_alignment(dt), q, k, v, o) || !lse || !aligned(lse, 4) || !apart(a.os, a.B, a.Tq, a.H, a.D)) return DP_ERR_INVALID_ARG;
  a.q = q;
  a.k = k;
  a.v = v;
  a.out = o;
  a.lse = lse;
  a.key_parts = 1;
  a.part_keys = a.Tk;
  if (ws) {
    if (!aligned(ws, 16)) return DP_ERR_INVALID_ARG;
    attention_key_parts(a, dt);
    if (ws_bytes < (size_t)attention_key_floats(a) * sizeof(float)) return DP_ERR_WORKSPACE;
    a.partial = static_cast<float*>(ws);
  }
  return launch_attention_forward(a, dt, static_cast<hipStream_t>(stream));
}

dp_status dp_attention_tile_rows(const dp_attention_shape* shape, dp_dtype dt, int32_t* rows) {
  AttnArgs a;
  if (!rows) return DP_ERR_INVALID_ARG;
  const dp_status st = attention_args(shape, dt, a);
  if (st != DP_OK) return st;
  a.parts = parts_of(a, dt);
  int queries, keys;
  attention_backward_tiles(a, dt, queries, keys);
  rows[0] = attention_forward_tile(a, dt);
  rows[1] = queries;
  rows[2] = keys;
  return DP_OK;
}

size_t dp_attention_backward_workspace_bytes(const dp_attention_shape* shape, dp_dtype dt) {
  AttnArgs a;
  return attention_args(shape, dt, a) == DP_OK ? backward_workspace(a, dt) : 0;
}

dp_status dp_attention_backward(const dp_attention_shape* shape, dp_dtype dt, const void* q, const void* k, const void* v,
                                const void* o, const float* lse, const void* dout, void* dq, void* dk, void* dv, void* ws,
                                size_t ws_bytes, void* stream) {
  AttnArgs a;
  const dp_status st = attention_args(shape, dt, a);
  if (st != DP_OK) return st;
  if (!all_there(attention_alignment(dt), q, k, v, o, dout, dq, dk, dv) || !lse || !aligned(lse, 4))
    return DP_ERR_INVALID_ARG;
  if (!apart(a.qs, a.B, a.Tq, a.H, a.D) || !apart(a.ks, a.B, a.Tk, a.H_kv, a.D) || !apart(a.vs, a.B, a.Tk, a.H_kv, a.D))
    return DP_ERR_INVALID_ARG;
  const int64_t rows = (int64_t)a.B * a.H * a.Tq;
  if (!ws || ws_bytes < backward_workspace(a, dt)) return DP_ERR_WORKSPACE;
  if (!aligned(ws, 16)) return DP_ERR_INVALID_ARG;
  a.q = q;
  a.k = k;
  a.v = v;
  a.o = o;
  a.lse = const_cast<float*>(lse);
  a.dout = dout;
  a.dq = dq;
  a.dk = dk;
  a.dv = dv;
  a.lse2 = static_cast<float*>(ws);
  a.delta = a.lse2 + rows;
  a.parts = parts_of(a, dt);
  a.partial = a.lse2 + padded_rows(a);
  return launch_attention_backward(a, dt, static_cast<hipStream_t>(stream));
}

dp_status dp_adamw_multi(const dp_adamw_tensor* tensors, int n_tensors, dp_dtype grad_dt, int state_bits, dp_dtype copy_dt, double lr,
                         double beta1, double beta2, double eps, double grad_scale, uint64_t step, void* stream) {
  if (!tensors || n_tensors <= 0 || !dtype_ok(grad_dt) || !dtype_ok(copy_dt) || step == 0) return DP_ERR_INVALID_ARG;
  if (state_bits != 8 && state_bits != 32) return DP_ERR_INVALID_ARG;
  if (!(lr >= 0.) || isinf(lr) || !(eps >= 0.) || isinf(eps) || !isfinite(grad_scale)) return DP_ERR_INVALID_ARG;
  if (!(beta1 >= 0. && beta1 < 1.) || !(beta2 >= 0. && beta2 < 1.)) return DP_ERR_INVALID_ARG;
  const uintptr_t grad_size = grad_dt == DP_F32 ? 4 : 2, state_size = state_bits / 8;
  for (int i = 0; i < n_tensors; ++i) {
    const dp_adamw_tensor& t = tensors[i];
    if (t.n == 0) continue;
    if (!t.param || !t.grad || !t.m || !t.v || !isfinite(t.weight_decay)) return DP_ERR_INVALID_ARG;
    if (!aligned(t.param, 4) || !aligned(t.grad, grad_size) || !aligned(t.m, state_size) || !aligned(t.v, state_size))
      return DP_ERR_INVALID_ARG;
    if (state_bits == 8 && (!t.m_scale || !t.v_scale || !aligned(t.m_scale, 4) || !aligned(t.v_scale, 4))) return DP_ERR_INVALID_ARG;
    if (copy_dt != DP_F32 && (!t.copy || !aligned(t.copy, 2))) return DP_ERR_INVALID_ARG;
    if (t.n > (uint64_t)1 << 42) return DP_ERR_UNSUPPORTED;
  }
  AdamArgs a = {};
  a.grad_scale = (float)grad_scale;
  a.beta1 = (float)beta1;
  a.beta2 = (float)beta2;
  a.rest1 = (float)(1. - beta1);
  a.rest2 = (float)(1. - beta2);
  a.lr = (float)lr;
  a.fix1 = 1.f / (float)(1. - pow(beta1, (double)step));
  a.fix2 = 1.f / (float)(1. - pow(beta2, (double)step));
  a.eps = (float)eps;
  a.dither = (uint32_t)step * 0x9E3779B1u;
  int64_t blocks = 0;
  auto flush = [&] {
    if (a.n_tensors == 0) return DP_OK;
    const dp_status st = launch_adamw(a, blocks, grad_dt, state_bits, copy_dt, static_cast<hipStream_t>(stream));
    a.n_tensors = 0;
    blocks = 0;
    return st;
  };
  for (int i = 0; i < n_tensors; ++i) {
    const dp_adamw_tensor& t = tensors[i];
    if (t.n == 0) continue;
    const int64_t more = (int64_t)((t.n + kAdamChunk - 1) / kAdamChunk);
    if (a.n_tensors == kAdamTensors || blocks + more > INT32_MAX) {
      const dp_status st = flush();
      if (st != DP_OK) return st;
    }
    AdamTensor& to = a.t[a.n_tensors];
    to.param = t.param;
    to.grad = t.grad;
    to.m = t.m;
    to.v = t.v;
    to.m_scale = t.m_scale;
    to.v_scale = t.v_scale;
    to.copy = t.copy;
    to.n = t.n;
    to.keep = (float)(1. - lr * (double)t.weight_decay);
    to.whole = aligned(t.param, 16) && aligned(t.grad, 4 * grad_size) && aligned(t.m, 4 * state_size) && aligned(t.v, 4 * state_size) &&
               (copy_dt == DP_F32 || aligned(t.copy, 8));
    a.begin[a.n_tensors++] = (unsigned)blocks;
    blocks += more;
  }
  return flush();
}

}  // extern "C"
