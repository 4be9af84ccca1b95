// Gated feed-forward layers, fp32 forms: products on the fp32 matrix instructions, tiles through registers into LDS, any sizes.
//   gate = x Wg + bg,  up = x Wu + bu,  h = act(gate) up;
//   dh = dy Wd',  dgate = dh up act'(gate),  dup = dh act(gate),  dx = dgate Wg' + dup Wu'.
#include "gated.h"

namespace dpbk {

namespace {

constexpr int kThreads = 256, kRows = 64, kCols = 64, kDepth = 16;     // a tile: 64 rows, two sets of 64 columns; 16 terms at a time

// Two sets of columns side by side: forward the gate's and up's, else a product's at n0 and n0 + 64.  A wave has 32 rows and 32 columns of
// each set.  As [row][k], columns' operands [k][column] as they lie (forward) or [column][k].
template <int PASS>
__global__ void __launch_bounds__(kThreads) gated_f32_kernel(const GatedArgs a, int tiles_n) {
  constexpr int PITCH = kDepth + 1;
  __shared__ float la[kRows * PITCH], lb[2][PASS == kForward ? kDepth * kCols : kCols * PITCH];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int tm = blockIdx.x / (unsigned)tiles_n, tn = blockIdx.x - tm * tiles_n;
  const int m0 = tm * kRows, n0 = tn * (PASS == kForward ? kCols : 2 * kCols);
  const int N = PASS == kInput ? a.d : a.f, K = PASS == kForward ? a.d : PASS == kHidden ? a.d_out : a.f;
  auto value = [](const void* base, int64_t at) { return static_cast<const float*>(base)[at]; };
  f32x16 acc[2];
#pragma unroll
  for (int s = 0; s < 2; ++s)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[s][r] = 0.f;
  const int segments = PASS == kInput ? 2 : 1;
  for (int seg = 0; seg < segments; ++seg) {
    const void* const A = PASS == kForward ? a.x : PASS == kHidden ? a.dy : seg ? a.dup : a.dgate;
    const void* const W = PASS == kHidden ? a.w_down : seg ? a.w_up : a.w_gate;
    for (int k0 = 0; k0 < K; k0 += kDepth) {
      float ra[4], rb[2][4];
      {
        const int m = m0 + tid / 4, k = k0 + 4 * (tid % 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) ra[i] = m < a.rows && k + i < K ? value(A, (int64_t)m * K + k + i) : 0.f;
      }
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (PASS == kForward) {
            const int k = k0 + tid / 16, n = n0 + 4 * (tid % 16) + i;
            rb[s][i] = k < K && n < N ? value(s ? a.w_up : a.w_gate, (int64_t)k * N + n) : 0.f;
          } else {
            const int n = n0 + kCols * s + tid / 4, k = k0 + 4 * (tid % 4) + i;
            rb[s][i] = k < K && n < N ? value(W, (int64_t)n * K + k) : 0.f;
          }
        }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 4; ++i) la[tid / 4 * PITCH + 4 * (tid % 4) + i] = ra[i];
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          lb[s][PASS == kForward ? tid / 16 * kCols + 4 * (tid % 16) + i : tid / 4 * PITCH + 4 * (tid % 4) + i] = rb[s][i];
      __syncthreads();
#pragma unroll
      for (int k = 0; k < kDepth; k += 2) {
        const int kk = k + (lane >> 5), c = 32 * (wave & 1) + (lane & 31);
        const float fa = la[(32 * (wave >> 1) + (lane & 31)) * PITCH + kk];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const float fb = lb[s][PASS == kForward ? kk * kCols + c : c * PITCH + kk];
          acc[s] = __builtin_amdgcn_mfma_f32_32x32x2f32(fa, fb, acc[s], 0, 0, 0);
        }
      }
    }
  }
  // lane: column 32 (wave & 1) + lane % 32; register r: row 8 (r / 4) + 4 (lane / 32) + r % 4 of the wave's 32
  auto put = [](void* base, int64_t at, float x) { static_cast<float*>(base)[at] = x; };
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int m = m0 + 32 * (wave >> 1) + 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3);
    if (m >= a.rows) continue;
    const int n = n0 + 32 * (wave & 1) + (lane & 31);
    float slope;
    if (PASS == kForward) {
      if (n >= N) continue;
      const int64_t at = (int64_t)m * N + n;
      const float gate = acc[0][r] + (a.b_gate ? value(a.b_gate, n) : 0.f), up = acc[1][r] + (a.b_up ? value(a.b_up, n) : 0.f);
      if (a.gate) {
        put(a.gate, at, gate);
        put(a.up, at, up);
      }
      put(a.h, at, activation<true, false>(a.act, gate, slope) * up);
    } else {
#pragma unroll
      for (int s = 0; s < 2; ++s)
        if (n + kCols * s < N) {
          const int64_t at = (int64_t)m * N + n + kCols * s;
          if (PASS == kInput) {
            put(a.dx, at, acc[s][r]);
          } else {
            const float dh = acc[s][r], v = activation<true, true>(a.act, value(a.gate, at), slope);
            put(a.dgate, at, dh * value(a.up, at) * slope);
            put(a.dup, at, dh * v);
          }
        }
    }
  }
}

// dgate and dup where dh is given, VEC values a thread.
template <int DT, int VEC>
__global__ void __launch_bounds__(kThreads) gated_slopes_kernel(const GatedArgs a, int64_t n) {
  const int64_t at = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * VEC;
  if (at >= n) return;
  Values<DT, VEC> dh, gate, up;
  dh.load(a.dy, at);
  gate.load(a.gate, at);
  up.load(a.up, at);
  float dg[VEC], du[VEC];
#pragma unroll
  for (int k = 0; k < VEC; ++k) {
    float slope;
    const float v = activation<DT == DP_F32, true>(a.act, gate.get(k), slope);
    dg[k] = dh.get(k) * up.get(k) * slope;
    du[k] = dh.get(k) * v;
  }
  gate.set(dg);
  up.set(du);
  gate.store(a.dgate, at);
  up.store(a.dup, at);
}

template <int DT>
dp_status launch_slopes(const GatedArgs& a, hipStream_t s) {
  const int64_t n = (int64_t)a.rows * a.f;
  constexpr int WIDE = DT == DP_F32 ? 4 : 8;
  const uintptr_t all = (uintptr_t)a.dy | (uintptr_t)a.gate | (uintptr_t)a.up | (uintptr_t)a.dgate | (uintptr_t)a.dup;
  const bool wide = all % 16 == 0 && n % WIDE == 0;
  const int64_t threads = wide ? n / WIDE : n, blocks = (threads + kThreads - 1) / kThreads;
  if (wide)
    gated_slopes_kernel<DT, WIDE><<<dim3((unsigned)blocks), kThreads, 0, s>>>(a, n);
  else
    gated_slopes_kernel<DT, 1><<<dim3((unsigned)blocks), kThreads, 0, s>>>(a, n);
  return hip_status(hipGetLastError());
}

template <int PASS>
dp_status launch_f32(const GatedArgs& a, hipStream_t s) {
  const int N = PASS == kInput ? a.d : a.f, width = PASS == kForward ? kCols : 2 * kCols;
  const int64_t tiles_n = (N + width - 1) / width, tiles_m = (a.rows + kRows - 1) / kRows;
  gated_f32_kernel<PASS><<<dim3((unsigned)(tiles_m * tiles_n)), kThreads, 0, s>>>(a, (int)tiles_n);
  return hip_status(hipGetLastError());
}

}  // namespace

dp_status launch_gated_forward(const GatedArgs& a, dp_dtype dt, hipStream_t s) {
  return dt == DP_F32 ? launch_f32<kForward>(a, s) : launch_gated_tiles(a, dt, kForward, s);
}

dp_status launch_gated_backward(const GatedArgs& a, dp_dtype dt, hipStream_t s) {
  dp_status st;
  if (!a.w_down)
    st = dt == DP_F32 ? launch_slopes<DP_F32>(a, s) : dt == DP_BF16 ? launch_slopes<DP_BF16>(a, s) : launch_slopes<DP_F16>(a, s);
  else
    st = dt == DP_F32 ? launch_f32<kHidden>(a, s) : launch_gated_tiles(a, dt, kHidden, s);
  if (st != DP_OK || !a.dx) return st;
  return dt == DP_F32 ? launch_f32<kInput>(a, s) : launch_gated_tiles(a, dt, kInput, s);
}

}  // namespace dpbk
