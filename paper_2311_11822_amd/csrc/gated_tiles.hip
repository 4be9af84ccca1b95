// Gated feed-forward layers, 16-bit forms: products on the matrix cores (product.h), what becomes of them in the tiles' epilogues.
//   forward   one tile has the same columns of the gate's projection and up's, so that h = act(gate) up leaves with them
//   hidden    dh = dy Wd' exists in registers alone: dgate and dup leave, with gate and up read there
//   input     dx = dgate Wg' + dup Wu', one contraction over both
#include <algorithm>

#include "gated.h"
#include "product.h"

namespace dpbk {

namespace {

template <int DT>
__device__ __forceinline__ void gated_forward_rows(const GatedArgs& a, int64_t at, int n, const float (&v)[2][8]) {
  Values<DT, 8> out, bias;
  float gate[8], up[8], h[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) gate[k] = v[0][k], up[k] = v[1][k];
  if (a.b_gate) {
    bias.load(a.b_gate, n);
#pragma unroll
    for (int k = 0; k < 8; ++k) gate[k] += bias.get(k);
  }
  if (a.b_up) {
    bias.load(a.b_up, n);
#pragma unroll
    for (int k = 0; k < 8; ++k) up[k] += bias.get(k);
  }
  float slope;
#pragma unroll
  for (int k = 0; k < 8; ++k) h[k] = activation<false, false>(a.act, gate[k], slope) * up[k];
  if (a.gate) {
    out.set(gate);
    out.store(a.gate, at);
    out.set(up);
    out.store(a.up, at);
  }
  out.set(h);
  out.store(a.h, at);
}

template <int DT>
struct GateAndUp {
  Values<DT, 8> gate, up;
};
template <int DT>
__device__ __forceinline__ void gated_hidden_rows(const GatedArgs& a, int64_t at, const float (&dh)[8], GateAndUp<DT>& in) {
  Values<DT, 8>&gate = in.gate, &up = in.up;
  float dg[8], du[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    float slope;
    const float v = activation<false, true>(a.act, gate.get(k), slope);
    dg[k] = dh[k] * up.get(k) * slope;
    du[k] = dh[k] * v;
  }
  gate.set(dg);
  up.set(du);
  gate.store(a.dgate, at);
  up.store(a.dup, at);
}

template <int PASS, class S, int DT>
__global__ void __launch_bounds__(S::NT, 163840 / S::LDS_BYTES) gated_tile_kernel(const GatedArgs a, int tiles_m, int tiles_n, int parts) {
  extern __shared__ __attribute__((aligned(1024))) unsigned char lds_raw[];
  const unsigned lds0 = (unsigned)(uintptr_t)lds_raw;
  ProductShape p;
  p.M = a.rows;
  p.N = PASS == kInput ? a.d : a.f;
  p.K = PASS == kForward ? a.d : PASS == kHidden ? a.d_out : a.f;
  p.terms = p.K;
  p.lda = p.K;
  p.ldb = PASS == kForward ? p.N : p.K;
  p.segments = PASS == kInput ? 2 : 1;
  if constexpr (PASS == kForward) p.s[0] = {a.x, a.w_gate, a.w_up};
  if constexpr (PASS == kHidden) p.s[0] = {a.dy, a.w_down, nullptr};
  if constexpr (PASS == kInput) p.s[0] = {a.dgate, a.w_gate, nullptr};
  p.s[1] = PASS == kInput ? ProductSegment{a.dup, a.w_up, nullptr} : p.s[0];
  const int tiles = tiles_m * tiles_n, id = grad_logical_tile(blockIdx.x, tiles * parts);
  int tm, tn, part = 0;
  if constexpr (PASS == kInput) part = id / tiles;
  grad_tile_of(tiles_m, tiles_n, id - part * tiles, tm, tn);
  const int64_t stages = p.segments * ((p.K + kProductTerms - 1) / kProductTerms);
  p.first = (int)(part * stages / parts);
  p.stages = (int)((part + 1) * stages / parts) - p.first;
  const int m0 = tm * S::BM, n = tn * (S::SETS ? S::BN / 2 : S::BN), n0[2] = {n, n};
  f32x4 acc[S::TM][S::TN];
  product_tile<S, DT == DP_F16>(p, m0, n0, lds0, acc);
  auto place = [&](int row, int col) { return (int64_t)(m0 + row) * p.N + n + col; };
  auto inside = [&](int row, int col) { return m0 + row < p.M && n + col < p.N; };
  if constexpr (PASS == kHidden) {
    auto load = [&](int row, int col, int) {
      GateAndUp<DT> in;
      if (inside(row, col)) {
        in.gate.load(a.gate, place(row, col));
        in.up.load(a.up, place(row, col));
      }
      return in;
    };
    product_rows<S, false>(acc, lds0, load, [&](int row, int col, int, const float (&v)[2][8], GateAndUp<DT>& in) {
      if (inside(row, col)) gated_hidden_rows<DT>(a, place(row, col), v[0], in);
    });
  } else {
    product_rows<S, PASS == kForward>(acc, lds0, NoLoad{}, [&](int row, int col, int, const float (&v)[2][8], Nothing) {
      if (!inside(row, col)) return;
      if constexpr (PASS == kForward) gated_forward_rows<DT>(a, place(row, col), n + col, v);
      if constexpr (PASS == kInput) {
        if (parts > 1) {
          f32x4* const to = reinterpret_cast<f32x4*>(a.partial + (int64_t)part * p.M * p.N + place(row, col));
          to[0] = f32x4{v[0][0], v[0][1], v[0][2], v[0][3]};
          to[1] = f32x4{v[0][4], v[0][5], v[0][6], v[0][7]};
          return;
        }
        Values<DT, 8> out;
        out.set(v[0]);
        out.store(a.dx, place(row, col));
      }
    });
  }
}

// The parts' sums, in their order.
template <int DT>
__global__ void __launch_bounds__(256) gated_join_kernel(const float* partial, void* dx, int64_t n, int parts) {
  const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (at >= n) return;
  float v[8] = {};
  for (int p = 0; p < parts; ++p) {
    const f32x4* from = reinterpret_cast<const f32x4*>(partial + p * n + at);
    const f32x4 x = from[0], y = from[1];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] += x[k], v[4 + k] += y[k];
  }
  Values<DT, 8> out;
  out.set(v);
  out.store(dx, at);
}

template <int PASS, class S, int DT>
dp_status launch_tiles(const GatedArgs& a, int parts, hipStream_t s) {
  static ReadyTable ready;
  dp_status st = allow_big_lds(gated_tile_kernel<PASS, S, DT>, S::LDS_BYTES, ready);
  if (st != DP_OK) return st;
  const int N = PASS == kInput ? a.d : a.f, width = S::SETS ? S::BN / 2 : S::BN;
  const int tiles_m = (a.rows + S::BM - 1) / S::BM, tiles_n = (N + width - 1) / width;
  gated_tile_kernel<PASS, S, DT><<<dim3((unsigned)tiles_m * tiles_n * parts), S::NT, S::LDS_BYTES, s>>>(a, tiles_m, tiles_n, parts);
  st = hip_status(hipGetLastError());
  if (st != DP_OK || parts == 1) return st;
  const int64_t n = (int64_t)a.rows * a.d;
  gated_join_kernel<DT><<<dim3((unsigned)((n / 8 + 255) / 256)), 256, 0, s>>>(a.partial, a.dx, n, parts);
  return hip_status(hipGetLastError());
}

// A pass's kernel: few rows, or large or small tiles, the latter in parts.
//
// 256 large tiles are resident at a time and start and end together: 1.5 us to a stage of 64 terms, and what comes before and after.  Small ones,
// two to a compute unit, run into each other, one's epilogue beside the other's products: 0.45 us a stage alone on a unit, 0.8 two at a time (0.9
// with all units full).  Both as measured, us, large and small: forward 4096 x 768 x 2048 31.5, 36.3; 4728 x 784 x 2096 57.4, 50.9;
// 4096 x 4096 x 11008 609, 728; hidden 16384 x 768 x 2048 112, 97; 4096 x 4096 x 11008 369, 371; input 4096 x 4096 x 11008 517, 752; 2048 x 4096 x
// 4096 145, 118.
// Input gradients contract over 2 f and have few tiles: where small ones leave compute units idle their contraction is dealt to `parts`
// workgroups, whose sums go through memory (4 bytes an element and part, there and back, at some 6 TB/s) and one more launch.  1, 2, 4, 8 and 16
// parts, us: 128 x 768 x 2048 27.5, 15.9, 9.9, 7.9, 9.4; 256 x 4096 x 11008 162, 89, 55, 54, 81; 4096 x 1280 x 3456 87.5, 90.6, 95.4, 137, 233.
// Few rows, there and on tiles (in parts), us: forward 64 x 1280 x 3456 9.7, 16.3; 32 x 4096 x 11008 54.6, 44.1; hidden 32 x 4096 x 11008 26.6, 37.6;
// 64 x 12288 x 32768 407, 198; input 32 x 768 x 2048 3.3, 6.6; 16 x 4096 x 11008 27.9, 32.4; 64 x 4096 x 11008 62.1, 34.8.
struct Choice {
  bool few, large;
  int parts;
};
Choice choose(GatedPass pass, int rows, int d, int f, int d_out) {
  const int64_t N = pass == kInput ? d : f, K = pass == kForward ? d : pass == kHidden ? d_out : f;
  const int stages = (int)((K + kProductTerms - 1) / kProductTerms) * (pass == kInput ? 2 : 1);
  auto tiles = [&](int side) { return ((int64_t)rows + side - 1) / side * ((N * (pass == kForward ? 2 : 1) + side - 1) / side); };
  Choice c = {false, true, 1};
  if (rows <= kGatedFewRows) {
    const double products = (double)rows * (double)K * (double)N;
    c.few = pass == kForward ? tiles(128) < 160 : rows <= 16 || products <= (pass == kHidden ? 3e9 : 1.5e8);
    if (c.few) return c;
  }
  const float big_rest = pass == kForward ? 10.f : pass == kHidden ? 30.f : 8.f, mid_rest = pass == kForward ? 9.f : pass == kHidden ? 18.f : 8.f;
  float best = (float)((tiles(256) + 255) / 256) * (1.5f * stages + big_rest);
  for (int parts = 1; parts <= (pass == kInput ? 64 : 1) && (parts == 1 || 4 * parts <= stages); ++parts) {
    const float n = (float)tiles(128) * parts;
    const float stage = n <= 256.f ? 0.45f : n <= 512.f ? 0.8f : n <= 768.f ? 1.2f : 0.9f / 512.f * n;
    float cost = stage * stages / parts + std::max(1.f, n / 512.f) * mid_rest;
    if (parts > 1) cost += 4.f + (2 * parts + 0.5f) * ((float)rows * d * 4e-6f / 6.f);
    if (cost < best) {
      best = cost;
      c.large = false;
      c.parts = parts;
    }
  }
  return c;
}

template <int PASS, int DT>
dp_status launch_pass(const GatedArgs& a, hipStream_t s) {
  constexpr ProductB B = PASS == kForward ? kColumnSets : kRowsOfTerms;
  const Choice c = choose((GatedPass)PASS, a.rows, a.d, a.f, a.d_out);
  if (c.few) return launch_gated_few(a, (dp_dtype)DT, (GatedPass)PASS, s);
  return c.large ? launch_tiles<PASS, BigProduct<B>, DT>(a, 1, s) : launch_tiles<PASS, MidProduct<B>, DT>(a, c.parts, s);
}

}  // namespace

size_t gated_input_workspace(int rows, int d, int f, int d_out) {
  const Choice c = choose(kInput, rows, d, f, d_out);
  return c.parts > 1 ? (size_t)c.parts * rows * d * sizeof(float) : 0;
}

dp_status launch_gated_tiles(const GatedArgs& a, dp_dtype dt, GatedPass pass, hipStream_t s) {
  if (dt == DP_BF16)
    return pass == kForward ? launch_pass<kForward, DP_BF16>(a, s) : pass == kHidden ? launch_pass<kHidden, DP_BF16>(a, s) : launch_pass<kInput, DP_BF16>(a, s);
  return pass == kForward ? launch_pass<kForward, DP_F16>(a, s) : pass == kHidden ? launch_pass<kHidden, DP_F16>(a, s) : launch_pass<kInput, DP_F16>(a, s);
}

}  // namespace dpbk
