// Gated feed-forward layers, 16-bit forms: products on the matrix cores (product.h), what becomes of them in the tiles' epilogues.
//   forward   one tile has the same columns of the gate's projection and up's, so that h = act(gate) up leaves with them
//   hidden    dh = dy Wd' exists in registers alone: dgate and dup leave, with gate and up read there
//   input     dx = dgate Wg' + dup Wu', one contraction over both
#include <algorithm>

#include "gated.h"
#include "product.h"

namespace dpbk {

namespace {

template <int ACT, int DT>
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
  for (int k = 0; k < 8; ++k) h[k] = activation<ACT, false, false>(gate[k], slope) * up[k];
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
template <int ACT, int DT>
__device__ __forceinline__ void gated_hidden_rows(const GatedArgs& a, int64_t at, const float (&dh)[8], GateAndUp<DT>& in) {
  Values<DT, 8>&gate = in.gate, &up = in.up;
  float dg[8], du[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    float slope;
    const float v = activation<ACT, false, true>(gate.get(k), slope);
    dg[k] = dh[k] * up.get(k) * slope;
    du[k] = dh[k] * v;
  }
  gate.set(dg);
  up.set(du);
  gate.store(a.dgate, at);
  up.store(a.dup, at);
}

// The tiles of a launch: a grid of m x n, or, small ones, what the large tiles from `cut` on of a grid of large ones are cut into, four each.  The first
// `whole` have a workgroup each, the others `parts`.
struct Tiles {
  int m, n, cut, whole, parts;
  __host__ __device__ int count() const { return cut < 0 ? m * n : 4 * (m * n - cut); }
  __device__ __forceinline__ void place(int tile, int& tm, int& tn) const {
    if (cut < 0) return grad_tile_of(m, n, tile, tm, tn);
    grad_tile_of(m, n, cut + tile / 4, tm, tn);
    tm = 2 * tm + (tile >> 1 & 1);
    tn = 2 * tn + (tile & 1);
  }
};

template <int PASS, class S, int DT>
__global__ void __launch_bounds__(S::NT, 163840 / S::LDS_BYTES) gated_tile_kernel(const GatedArgs a, const Tiles tiles) {
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
  const int rest = tiles.count() - tiles.whole, id = grad_logical_tile(blockIdx.x, tiles.whole + rest * tiles.parts);
  const bool dealt = id >= tiles.whole;
  const int part = dealt ? (id - tiles.whole) / rest : 0, tile = id - part * rest, shares = dealt ? tiles.parts : 1;
  int tm, tn;
  tiles.place(tile, tm, tn);
  const int64_t stages = p.segments * ((p.K + kProductTerms - 1) / kProductTerms);
  p.first = (int)(part * stages / shares);
  p.stages = (int)((part + 1) * stages / shares) - p.first;
  const int m0 = tm * S::BM, n = tn * (S::SETS ? S::BN / 2 : S::BN), n0[2] = {n, n};
  if (m0 >= p.M || n >= p.N) return;                   // of a large tile at the edge
  f32x4 acc[S::TM][S::TN];
  // a part's sums: [row][column], of two sets one beside the other
  float* const partial = a.partial + ((int64_t)part * rest + tile - tiles.whole) * (S::BM * S::BN);
  auto keep = [&](int row, int col, int, const float (&v)[2][8], Nothing) {
#pragma unroll
    for (int set = 0; set < (S::SETS ? 2 : 1); ++set) {
      f32x4* const to = reinterpret_cast<f32x4*>(partial + row * S::BN + set * (S::BN / 2) + col);
      to[0] = f32x4{v[set][0], v[set][1], v[set][2], v[set][3]};
      to[1] = f32x4{v[set][4], v[set][5], v[set][6], v[set][7]};
    }
  };
  auto place = [&](int row, int col) { return (int64_t)(m0 + row) * p.N + n + col; };
  auto inside = [&](int row, int col) { return m0 + row < p.M && n + col < p.N; };
  if constexpr (PASS == kHidden) {
    auto load = [&](int row, int col, int) {
      GateAndUp<DT> in;
      if (!dealt && inside(row, col)) {
        in.gate.load(a.gate, place(row, col));
        in.up.load(a.up, place(row, col));
      }
      return in;
    };
    ProductAhead<S, false, decltype(load)> ahead(load);
    product_tile<S, DT == DP_F16>(p, m0, n0, lds0, acc);
    if (dealt) {
      NothingAhead<S, false> none(NoLoad{});
      product_rows<S, false>(acc, lds0, none, keep);
      return;
    }
    with_activation(a.act, [&](auto act) {
      product_rows<S, false>(acc, lds0, ahead, [&](int row, int col, int, const float (&v)[2][8], GateAndUp<DT>& in) {
        if (inside(row, col)) gated_hidden_rows<decltype(act)::value, DT>(a, place(row, col), v[0], in);
      });
    });
  } else if constexpr (PASS == kForward) {
    product_tile<S, DT == DP_F16>(p, m0, n0, lds0, acc);
    NothingAhead<S, true> ahead(NoLoad{});
    if (dealt) {
      product_rows<S, true>(acc, lds0, ahead, keep);
      return;
    }
    with_activation(a.act, [&](auto act) {
      product_rows<S, true>(acc, lds0, ahead, [&](int row, int col, int, const float (&v)[2][8], Nothing) {
        if (inside(row, col)) gated_forward_rows<decltype(act)::value, DT>(a, place(row, col), n + col, v);
      });
    });
  } else {
    product_tile<S, DT == DP_F16>(p, m0, n0, lds0, acc);
    NothingAhead<S, false> ahead(NoLoad{});
    if (dealt) {
      product_rows<S, false>(acc, lds0, ahead, keep);
      return;
    }
    product_rows<S, false>(acc, lds0, ahead, [&](int row, int col, int, const float (&v)[2][8], Nothing) {
      if (!inside(row, col)) return;
      Values<DT, 8> out;
      out.set(v[0]);
      out.store(a.dx, place(row, col));
    });
  }
}

// The parts' sums of the tiles from `whole` on, in their order, and what becomes of them: eight columns (of both sets) to a thread.
template <int PASS, int SIDE>
constexpr int kJoinGroups = SIDE * SIDE / (PASS == kForward ? 2 : 1) / 2048;      // workgroups to a tile
template <int PASS, int SIDE, int DT>
__global__ void __launch_bounds__(256) gated_join_kernel(const GatedArgs a, const Tiles tiles) {
  constexpr int SETS = PASS == kForward ? 2 : 1, WIDTH = SIDE / SETS, GROUPS = kJoinGroups<PASS, SIDE>;
  const int rest = tiles.count() - tiles.whole, t = blockIdx.x / GROUPS, at = (blockIdx.x % GROUPS * 256 + threadIdx.x) * 8;
  int tm, tn;
  tiles.place(tiles.whole + t, tm, tn);
  const int N = PASS == kInput ? a.d : a.f, row = tm * SIDE + at / WIDTH, col = tn * WIDTH + at % WIDTH;
  if (row >= a.rows || col >= N) return;
  const int64_t to = (int64_t)row * N + col;
  float v[2][8] = {};
  for (int p = 0; p < tiles.parts; ++p) {
    const float* const from = a.partial + ((int64_t)p * rest + t) * (SIDE * SIDE) + at / WIDTH * SIDE + at % WIDTH;
#pragma unroll
    for (int set = 0; set < SETS; ++set) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(from + set * WIDTH), y = *reinterpret_cast<const f32x4*>(from + set * WIDTH + 4);
#pragma unroll
      for (int k = 0; k < 4; ++k) v[set][k] += x[k], v[set][4 + k] += y[k];
    }
  }
  if constexpr (PASS == kForward) {
    with_activation(a.act, [&](auto act) { gated_forward_rows<decltype(act)::value, DT>(a, to, col, v); });
  } else if constexpr (PASS == kHidden) {
    GateAndUp<DT> in;
    in.gate.load(a.gate, to);
    in.up.load(a.up, to);
    with_activation(a.act, [&](auto act) { gated_hidden_rows<decltype(act)::value, DT>(a, to, v[0], in); });
  } else {
    Values<DT, 8> out;
    out.set(v[0]);
    out.store(a.dx, to);
  }
}

template <int PASS, class S>
Tiles grid_of(const GatedArgs& a, int cut) {
  const int N = PASS == kInput ? a.d : a.f, width = S::SETS ? S::BN / 2 : S::BN;
  return {(a.rows + S::BM - 1) / S::BM, (N + width - 1) / width, cut, 0, 1};
}

// The first `blocks` workgroups of these tiles.
template <int PASS, class S, int DT>
dp_status launch_tiles(const GatedArgs& a, const Tiles& tiles, int64_t blocks, hipStream_t s) {
  static ReadyTable ready;
  const dp_status st = allow_big_lds(gated_tile_kernel<PASS, S, DT>, S::LDS_BYTES, ready);
  if (st != DP_OK) return st;
  gated_tile_kernel<PASS, S, DT><<<dim3((unsigned)blocks), S::NT, S::LDS_BYTES, s>>>(a, tiles);
  return hip_status(hipGetLastError());
}

// A pass's kernel: few rows; or large tiles, and small ones for what is left of whole rounds of them, or for all, some of them in parts.
//
// 256 large tiles are resident at a time and start and end together: 1.5 us to a stage of 64 terms, and what comes before and after.  Small ones,
// two to a compute unit, run into each other, one's epilogue beside the other's products: 0.45 us a stage alone on a unit, 0.8 two at a time (0.9
// with all units full).  Both as measured, us, large and small: forward 4096 x 768 x 2048 30.0, 35.0; 1000 x 1024 x 2816 28.6, 20.5;
// 4096 x 4096 x 11008 616, 743; hidden 4096 x 1280 x 3456 47.0, 54.1; 16384 x 768 x 2048 92, 90; 2048 x 1280 x 3456 39.4, 28.4; input 4096 x 4096 x
// 11008 517, 752; 2048 x 4096 x 4096 145, 118.
// Weights that come from memory arrive later than small tiles have asked for them: 0.7 us a stage alone, 1.1 to 1.2 two at a time; large ones, which
// need half as many bytes to a product, hardly feel it.  Where they come from is not known here; the forward pass and input gradients take these costs
// (`far`) from f = 5120 on, where what they lose if a cache has the weights after all meets what they win if none has.  The other costs and these, us,
// from memory and, behind the semicolon, from caches: input gradients 1014 x 2048 x 4096 58.7, 51.8; 43.7, 45.9.  x 4608 64.9, 58.8; 48.1, 53.3.
// x 5112 76.3, 67.8; 62.0, 60.3.  x 5120 71.8, 61.8; 52.5, 56.6.  x 6144 83.0, 66.6; 61.9, 61.8.  2048 x 4096 x 4096 137, 128; 123, 123.  x 5120 173, 155;
// 154, 148.  Forward 1014 x 2048 x 4096 47.0, 47.9; 40.2, 40.4.  x 5120 65.2, 55.0; 54.5, 52.3.  (Rows of 5112 values begin inside of lines, at any rule.)
// Where tiles leave compute units idle, as most input gradients', which contract over 2 f, their contraction is dealt to `parts`
// workgroups, whose sums go through memory (4 bytes an element and part, there and back, at some 6 TB/s) and one more launch.  Input gradients in
// 1, 2, 4, 8 and 16 parts of small tiles, us: 128 x 768 x 2048 27.5, 15.9, 9.9, 7.9, 9.4; 4096 x 1280 x 3456 95.0, 90.2, 94.4, 136, 229, and 76.2 with 256 of
// its 320 tiles whole and the others, which would be a second one on some units, in four parts; 1014 x 4096 x 11008, weights from memory, 254, 211,
// 223, 246, and of large ones 441, 238, 160, 183, 242; 512 x 4096 x 11008 120 in 4 parts of small tiles, 95 in 8 of large ones.  Other passes, whole and in
// parts: forward 1014 x 7416 x 216 70, 24; 256 x 4096 x 1024 39, 20; 200 x 16384 x 8192 199 (small tiles), 147 (large ones); hidden, d_out 4096,
// 1014 x 1024 35, 22.
// Few rows, there and on tiles (in parts), weights from caches, us: forward 16 x 4096 x 2048 14.4, 17.8; 64 x 2048 x 4096 15.2, 17.7; 16 x 7424 x 768
// 26.3, 17.8; 64 x 4096 x 4096 25.3, 21.8 (from memory 63 or 64 x 2048 x 4096 20.7, 20.6, x 4096 x 2048 33.6, 21.2: the rule ends between those rows);
// hidden, d_out first, 16 x 8192 x 11008 35.6, 38.8; 64 x 2048 x 4096 10.9, 16.1; 64 x 7424 x 2048 22.5, 18.1; input, 2 f last, 16 x 4096 x 16384 18.0,
// 23.1; 64 x 4096 x 2048 3.5, 9.5; 64 x 11008 x 4096 33.6, 20.5; 64 x 216 x 7424 18.9, 10.6.
struct Choice {
  bool few;
  int64_t large, whole;             // large tiles and, of what is left, small ones that one workgroup has each
  int parts, side;                  // of the others, whose sides these are
  int64_t dealt;                    // how many those are
};
Choice choose(GatedPass pass, int rows, int d, int f, int d_out) {
  const int64_t N = pass == kInput ? d : f, K = pass == kForward ? d : pass == kHidden ? d_out : f;
  const int stages = (int)((K + kProductTerms - 1) / kProductTerms) * (pass == kInput ? 2 : 1);
  auto tiles = [&](int side) { return ((int64_t)rows + side - 1) / side * ((N * (pass == kForward ? 2 : 1) + side - 1) / side); };
  const int64_t all_large = tiles(256), all_small = tiles(128);
  Choice c = {false, all_large, 0, 1, 128, 0};
  if (rows <= kGatedFewRows) {
    const double weights = (double)stages * kProductTerms * (double)N;
    if (pass == kForward)
      c.few = K <= 4096 && (rows + 32) * weights <= 8e8;
    else
      c.few = (double)rows * rows * weights <= 4e10 && (pass == kHidden || rows * stages <= 4096);
    if (c.few) return c;
  }
  const float big_rest = pass == kForward ? 9.f : pass == kHidden ? 19.f : 8.f, mid_rest = pass == kHidden ? 13.f : 8.f;
  const bool far = pass != kHidden && f >= 5120;
  const float big_stage = far && pass == kForward ? 1.65f : 1.5f, mid_stage = !far ? 0.4f : pass == kForward ? 0.55f : 0.6f, alone = far ? 0.15f : 0.05f;
  auto joined = [&](int parts, int64_t dealt, float tile_bytes) {
    if (dealt == 0 || parts == 1) return 0.f;
    const float bytes = (float)dealt * tile_bytes;                             // (hidden: its epilogue is the join's)
    return (pass == kForward && far ? 8.f : 4.f) + (2 * parts + 0.5f) * bytes / (pass == kInput && far ? 4.5e6f : 6e6f) + (pass == kHidden ? 1.3e-6f * bytes : 0.f);
  };
  auto rounds = [&](int64_t large) { return (float)((large + 255) / 256) * (big_stage * stages + big_rest); };
  float best = rounds(all_large);
  auto consider = [&](int64_t large, int64_t whole, int parts) {
    const int64_t total = large ? 4 * (all_large - large) : all_small, dealt = total - whole, pieces = dealt * parts, n = whole + pieces;
    float cost = large ? rounds(large) - 6.f : 0.f;
    if (n > 768) {
      cost += (far ? 1.1f : 0.9f + 0.0004f * stages) / 512.f * stages * (float)total;
    } else {
      // a compute unit's workgroups, and more where one runs alone
      const float longest = whole ? (float)stages : (float)stages / parts;
      const float all = (float)((whole + 255) / 256) * stages + (float)((pieces + 255) / 256) * stages / parts;
      cost += mid_stage * all + alone * std::max(0.f, 2.f * longest - all);
    }
    cost += std::max(1.f, (float)n / 512.f) * ((float)whole * mid_rest + (float)pieces * 8.f) / (float)n;
    cost += joined(parts, dealt, 65536.f);
    if (cost < best) {
      best = cost;
      c.large = large;
      c.whole = whole;
      c.side = 128;
      c.parts = parts;
      c.dealt = dealt;
    }
  };
  auto deal_large = [&](int parts) {
    const float cost = big_stage * stages / parts + big_rest + joined(parts, all_large, 262144.f);
    if (cost < best) {
      best = cost;
      c.large = c.whole = 0;
      c.parts = parts;
      c.side = 256;
      c.dealt = all_large;
    }
  };
  for (const int64_t large : {(int64_t)0, all_large / 256 * 256}) {
    if (large == all_large) continue;
    const int64_t total = large ? 4 * (all_large - large) : all_small;
    consider(large, total, 1);
    for (const int parts : {2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 48, 64}) {
      if (4 * parts > stages) break;
      consider(large, 0, parts);
      if (total > 256 && total % 256) consider(large, total / 256 * 256, parts);
      if (large == 0 && pass != kHidden && all_large * parts <= 256) deal_large(parts);
    }
  }
  return c;
}

template <int PASS, int DT>
dp_status launch_pass(const GatedArgs& a, hipStream_t s) {
  constexpr ProductB B = PASS == kForward ? kColumnSets : kRowsOfTerms;
  typedef BigProduct<B> Big;
  typedef MidProduct<B> Mid;
  const Choice c = choose((GatedPass)PASS, a.rows, a.d, a.f, a.d_out);
  if (c.few) return launch_gated_few(a, (dp_dtype)DT, (GatedPass)PASS, s);
  Tiles tiles = grid_of<PASS, Big>(a, -1);
  const int all_large = tiles.count();
  auto join = [&](auto side) {
    const unsigned blocks = (unsigned)c.dealt * kJoinGroups<PASS, decltype(side)::value>;
    gated_join_kernel<PASS, decltype(side)::value, DT><<<dim3(blocks), 256, 0, s>>>(a, tiles);
    return hip_status(hipGetLastError());
  };
  dp_status st = DP_OK;
  if (c.large > 0) {
    tiles.whole = all_large;
    st = launch_tiles<PASS, Big, DT>(a, tiles, c.large, s);
  }
  if (st != DP_OK || c.large == all_large) return st;
  if (c.large > 0 || c.side == 128) tiles = c.large > 0 ? grid_of<PASS, Big>(a, (int)c.large) : grid_of<PASS, Mid>(a, -1);
  tiles.whole = (int)c.whole;
  tiles.parts = c.parts;
  const int64_t blocks = c.whole + c.dealt * c.parts;
  if constexpr (PASS != kHidden)
    if (c.side == 256) {
      st = launch_tiles<PASS, Big, DT>(a, tiles, blocks, s);
      return st == DP_OK ? join(std::integral_constant<int, 256>{}) : st;
    }
  st = launch_tiles<PASS, Mid, DT>(a, tiles, blocks, s);
  return st == DP_OK && c.dealt > 0 ? join(std::integral_constant<int, 128>{}) : st;
}

}  // namespace

GatedLaunches gated_tiles_launches(GatedPass pass, int rows, int d, int f, int d_out) {
  const Choice c = choose(pass, rows, d, f, d_out);
  if (c.few) return {kGatedFew, 0, 0, 0, 0, 0};
  return {kGatedTiles16, c.large, c.whole, c.dealt, c.dealt ? c.parts : 0, c.dealt ? c.side : 0};
}

size_t gated_tiles_workspace(GatedPass pass, int rows, int d, int f, int d_out) {
  const Choice c = choose(pass, rows, d, f, d_out);
  return c.few ? 0 : (size_t)c.parts * c.dealt * (c.side * c.side) * sizeof(float);
}

dp_status launch_gated_tiles(const GatedArgs& a, dp_dtype dt, GatedPass pass, hipStream_t s) {
  if (dt == DP_BF16)
    return pass == kForward ? launch_pass<kForward, DP_BF16>(a, s) : pass == kHidden ? launch_pass<kHidden, DP_BF16>(a, s) : launch_pass<kInput, DP_BF16>(a, s);
  return pass == kForward ? launch_pass<kForward, DP_F16>(a, s) : pass == kHidden ? launch_pass<kHidden, DP_F16>(a, s) : launch_pass<kInput, DP_F16>(a, s);
}

}  // namespace dpbk
