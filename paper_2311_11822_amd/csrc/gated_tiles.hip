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
__global__ void __launch_bounds__(S::NT, 163840 / S::LDS_BYTES) gated_tile_kernel(const GatedArgs a, int tiles_m, int tiles_n) {
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
  p.s[2] = p.s[0];
  int tm, tn;
  grad_tile_of(tiles_m, tiles_n, grad_logical_tile(blockIdx.x, tiles_m * tiles_n), tm, tn);
  const int m0 = tm * S::BM, n = tn * (S::COLUMNS ? S::BN / 2 : S::BN), n0[2] = {n, n};
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
        Values<DT, 8> out;
        out.set(v[0]);
        out.store(a.dx, place(row, col));
      }
    });
  }
}

template <int PASS, class S, int DT>
dp_status launch_tiles(const GatedArgs& a, hipStream_t s) {
  static ReadyTable ready;
  const dp_status st = allow_big_lds(gated_tile_kernel<PASS, S, DT>, S::LDS_BYTES, ready);
  if (st != DP_OK) return st;
  const int N = PASS == kInput ? a.d : a.f, width = S::COLUMNS ? S::BN / 2 : S::BN;
  const int tiles_m = (a.rows + S::BM - 1) / S::BM, tiles_n = (N + width - 1) / width;
  gated_tile_kernel<PASS, S, DT><<<dim3((unsigned)tiles_m * tiles_n), S::NT, S::LDS_BYTES, s>>>(a, tiles_m, tiles_n);
  return hip_status(hipGetLastError());
}

// Large tiles or small ones.  256 large tiles are resident at a time and start and end together: 1.5 us to a stage of 64 terms, and what comes
// before and after; 512 small ones, two to a compute unit, whose rounds run into each other: 0.9 us, and less beside it, since one's epilogue
// runs beside the other's products.  Both as measured, us, large and small: forward 4096 x 768 x 2048 31.5, 36.3; 4728 x 784 x 2096 57.4,
// 50.9; 4096 x 4096 x 11008 609, 728; hidden 16384 x 768 x 2048 112, 97; 4096 x 4096 x 11008 369, 371; input 4096 x 4096 x 11008 517, 752;
// 2048 x 4096 x 4096 145, 118.
template <int PASS, int DT>
dp_status launch_pass(const GatedArgs& a, hipStream_t s) {
  constexpr bool COLUMNS = PASS == kForward;
  constexpr float kBigRest = PASS == kForward ? 10.f : PASS == kHidden ? 30.f : 8.f, kMidRest = PASS == kForward ? 9.f : PASS == kHidden ? 18.f : 8.f;
  const int64_t N = PASS == kInput ? a.d : a.f, K = PASS == kForward ? a.d : PASS == kHidden ? a.d_out : a.f;
  const float stages = (float)((K + 63) / 64 * (PASS == kInput ? 2 : 1));
  auto tiles = [&](int side) { return ((int64_t)a.rows + side - 1) / side * ((N * (COLUMNS ? 2 : 1) + side - 1) / side); };
  const float big = (float)((tiles(256) + 255) / 256) * (1.5f * stages + kBigRest);
  const float mid = std::max(1.f, (float)tiles(128) / 512.f) * (0.9f * stages + kMidRest);
  return big <= mid ? launch_tiles<PASS, BigProduct<COLUMNS>, DT>(a, s) : launch_tiles<PASS, MidProduct<COLUMNS>, DT>(a, s);
}

}  // namespace

dp_status launch_gated_tiles(const GatedArgs& a, dp_dtype dt, GatedPass pass, hipStream_t s) {
  if (dt == DP_BF16)
    return pass == kForward ? launch_pass<kForward, DP_BF16>(a, s) : pass == kHidden ? launch_pass<kHidden, DP_BF16>(a, s) : launch_pass<kInput, DP_BF16>(a, s);
  return pass == kForward ? launch_pass<kForward, DP_F16>(a, s) : pass == kHidden ? launch_pass<kHidden, DP_F16>(a, s) : launch_pass<kInput, DP_F16>(a, s);
}

}  // namespace dpbk
