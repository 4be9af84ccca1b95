// Gated feed-forward layers, fp32 forms: products on the fp32 matrix instructions, any sizes and alignments.
//   gate = x Wg + bg,  up = x Wu + bu,  h = act(gate) up;
//   dh = dy Wd',  dgate = dh up act'(gate),  dup = dh act(gate),  dx = dgate Wg' + dup Wu'.
#include <algorithm>

#include "gated.h"
#include "lds_dma.h"
#include "tile_order.h"

namespace dpbk {

namespace {

constexpr int kThreads = 256, kWaves = 4, kTerms = 32;         // terms of a stage: 128 bytes of a row

// 16384 x 512 x 1024 forward: 320 us, 107 TFLOP/s (the library's product alone, without what comes of it: 135).
// A tile of 32 W x 32 W by four waves of 16 W x 16 W.  Its columns: forward two sets of half as many, the gate's and up's, else those of one product.
// Memory -> LDS without registers, 4 bytes a lane, so that no row need begin anywhere in particular: 256 loads of 256 bytes to 64 KiB of a
// stage cost a hundredth of the matrix instructions' time, which is 16 times that of 16-bit ones.  Two stages: one is multiplied, one on its way.
// LDS holds [row][32 terms], 16-byte pieces XORed with row / 2, read 16 bytes a lane: four instructions take one of the four terms each, for both
// operands the same.  Columns' operands [term][columns], pieces XORed with term / 4, are read term by term.
template <int W, bool SETS>
struct F32Tile {
  static constexpr int SIDE = 32 * W, OPERAND_BYTES = SIDE * 128, STAGE_BYTES = 2 * OPERAND_BYTES, LOADS = OPERAND_BYTES / 256 / kWaves;
  static constexpr int SET = SIDE / 2;                         // columns of a set
};

// All loads into LDS have landed, in the other waves' too, and every wave is through with its reads.
__device__ __forceinline__ void landed() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

template <int PASS>
__device__ __forceinline__ float bias_of(const void* b, int n) { return PASS == kForward && b ? static_cast<const float*>(b)[n] : 0.f; }
// What becomes of a value of the products (forward: of both, with their biases).
template <int PASS, int ACT>
__device__ __forceinline__ void finish_value(const GatedArgs& a, int m, int n, int N, float v0, float v1, float b_gate, float b_up) {
  const int64_t place = (int64_t)m * N + n;
  auto at = [&](const void* base, int64_t i) { return static_cast<const float*>(base)[i]; };
  auto put = [&](void* base, float x) { static_cast<float*>(base)[place] = x; };
  float slope;
  if constexpr (PASS == kForward) {
    const float gate = v0 + b_gate, up = v1 + b_up;
    if (a.gate) {
      put(a.gate, gate);
      put(a.up, up);
    }
    put(a.h, activation<ACT, true, false>(gate, slope) * up);
  } else if constexpr (PASS == kHidden) {
    const float up = at(a.up, place), v = activation<ACT, true, true>(at(a.gate, place), slope);
    put(a.dgate, v0 * up * slope);
    put(a.dup, v0 * v);
  } else {
    put(a.dx, v0);
  }
}
template <int PASS, class F>
__device__ __forceinline__ void with_activation_of(int act, F f) {
  if constexpr (PASS == kInput)
    f(std::integral_constant<int, DP_ACT_RELU>{});     // (not used)
  else
    with_activation(act, f);
}

// A workgroup has one of a tile's `parts` shares of the contraction; of several, its sums go to memory: [part][tile][row][column], of two sets
// one beside the other.
template <int PASS, int W>
__global__ void __launch_bounds__(kThreads, 2) gated_f32_kernel(const GatedArgs a, int tiles_m, int tiles_n, int parts) {
  constexpr bool SETS = PASS == kForward;
  typedef F32Tile<W, SETS> S;
  extern __shared__ __attribute__((aligned(1024))) unsigned char lds_raw[];
  const unsigned lds0 = (unsigned)(uintptr_t)lds_raw;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int tm, tn;
  const int tiles = tiles_m * tiles_n, id = grad_logical_tile(blockIdx.x, tiles * parts), part = id / tiles, tile = id - part * tiles;
  grad_tile_of(tiles_m, tiles_n, tile, tm, tn);
  const int m0 = tm * S::SIDE, n0 = tn * (SETS ? S::SET : S::SIDE);
  const int N = PASS == kInput ? a.d : a.f, K = PASS == kForward ? a.d : PASS == kHidden ? a.d_out : a.f;
  const int per = (K + kTerms - 1) / kTerms, stages = per * (PASS == kInput ? 2 : 1);
  const int first = (int)((int64_t)part * stages / parts), end = (int)((int64_t)(part + 1) * stages / parts);
  const unsigned a_pitch = 4u * K, b_pitch = 4u * (SETS ? N : K);

  // A load brings two rows' terms; a lane's place in them, and the term that lies there, by the load's parity
  const int half = lane >> 5, at = lane & 31;
  int term[2];
#pragma unroll
  for (int odd = 0; odd < 2; ++odd) term[odd] = ((at >> 2) ^ ((4 * odd + wave) & 7)) * 4 + (at & 3);
  auto scalar = [](i32x4 r) {
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __builtin_amdgcn_readfirstlane(r[i]);
    return r;
  };
  auto ask = [&](int st, unsigned to) __attribute__((always_inline)) {
    const int seg = PASS == kInput && st >= per ? 1 : 0, k = (st - seg * per) * kTerms;
    const char* const pa = static_cast<const char*>(PASS == kForward ? a.x : PASS == kHidden ? a.dy : seg ? a.dup : a.dgate);
    const char* const pb = static_cast<const char*>(PASS == kHidden ? a.w_down : seg ? a.w_up : a.w_gate);
    auto rows = [&](const char* base, int row0, int row_end, unsigned pitch, unsigned lds) __attribute__((always_inline)) {
      const i32x4 r = scalar(make_rsrc(base + (uint64_t)row0 * pitch + 4ull * k, st < end ? (unsigned)imax(imin(row_end - row0, S::SIDE), 0) * pitch : 0));
#pragma unroll
      for (int l = 0; l < S::LOADS; ++l) {
        const unsigned row = 2 * (l * kWaves + wave) + half;
        load_dword_to_lds(r, k + term[l & 1] < K ? row * pitch + 4 * term[l & 1] : OOB, lds + (l * kWaves + wave) * 256);
      }
    };
    rows(pa, m0, a.rows, a_pitch, to);
    if constexpr (!SETS) {
      rows(pb, n0, N, b_pitch, to + S::OPERAND_BYTES);
    } else {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const char* const w = static_cast<const char*>(s ? a.w_up : a.w_gate);
        const i32x4 r = scalar(make_rsrc(w + (uint64_t)k * b_pitch, st < end ? (unsigned)imin(K - k, kTerms) * b_pitch : 0));
        constexpr int PER = 64 / S::SET;                       // terms of a load
#pragma unroll
        for (int l = 0; l < S::LOADS / 2; ++l) {
          const int kk = (l * kWaves + wave) * PER + lane / S::SET, c = lane % S::SET;
          const int col = n0 + (((c >> 2) ^ (((kk >> 2) & 3) << (S::SET == 64 ? 2 : 1))) << 2) + (c & 3);
          load_dword_to_lds(r, col < N ? kk * b_pitch + 4u * col : OOB, to + S::OPERAND_BYTES + s * S::OPERAND_BYTES / 2 + (l * kWaves + wave) * 256);
        }
      }
    }
  };
  f32x4 acc[W][W], sum[W][W];
#pragma unroll
  for (int i = 0; i < W; ++i)
#pragma unroll
    for (int k = 0; k < W; ++k) sum[i][k] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int r16 = lane & 15, h = lane >> 4, wm = (wave >> 1) * 16 * W, wc = wave & 1;
  typedef __attribute__((address_space(3))) const f32x4* Four;
  typedef __attribute__((address_space(3))) const float* One;
  ask(first, lds0);
  landed();
  auto stage = [&](int st, auto fresh) __attribute__((always_inline)) {
    const unsigned from = lds0 + (st & 1) * S::STAGE_BYTES;
    ask(first + st + 1, lds0 + (~st & 1) * S::STAGE_BYTES);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      f32x4 fa[W], fb[W];
      const unsigned place = ((4 * ks + h) ^ (r16 >> 1)) << 4;
#pragma unroll
      for (int x = 0; x < W; ++x) fa[x] = *(Four)(uintptr_t)(from + (wm + 16 * x + r16) * 128 + place);
#pragma unroll
      for (int y = 0; y < W; ++y) {
        if constexpr (!SETS) {
          fb[y] = *(Four)(uintptr_t)(from + S::OPERAND_BYTES + (16 * W * wc + 16 * y + r16) * 128 + place);
        } else {
          // frags 0 .. W / 2 - 1 of the gate's set, the others of up's
          const int set = y / (W / 2), c = 8 * W * wc + 16 * (y % (W / 2)) + r16;
          const unsigned piece = (unsigned)((c >> 2) ^ (h << (S::SET == 64 ? 2 : 1)));
#pragma unroll
          for (int e = 0; e < 4; ++e)
            fb[y][e] = *(One)(uintptr_t)(from + S::OPERAND_BYTES + set * S::OPERAND_BYTES / 2 + (16 * ks + 4 * h + e) * 4 * S::SET + piece * 16 + 4 * (c & 3));
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int x = 0; x < W; ++x)
#pragma unroll
          for (int y = 0; y < W; ++y)
            acc[x][y] = __builtin_amdgcn_mfma_f32_16x16x4f32(fa[x][e], fb[y][e], fresh && ks + e == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : acc[x][y], 0, 0, 0);
    }
    landed();
  };
  // Sums of 64 terms, then of those: the error grows with the root of either number.  2048 terms 1.7e-7 off, chains of 256 2.9e-7 (and no faster:
  // a chain begins from the zero that its first instructions take).
  for (int st = 0; st < end - first; ++st) {
    stage(st, std::true_type{});
    if (++st < end - first) stage(st, std::false_type{});
#pragma unroll
    for (int i = 0; i < W; ++i)
#pragma unroll
      for (int k = 0; k < W; ++k) sum[i][k] += acc[i][k];
  }

  // lane: column lane % 16 of a fragment; register r: row 4 (lane / 16) + r
  constexpr int COLS = SETS ? W / 2 : W;
  if (parts > 1) {
    float* const to = a.partial + ((int64_t)part * tiles + tile) * (S::SIDE * S::SIDE) + (wm + 4 * h) * S::SIDE + 16 * COLS * wc + r16;
#pragma unroll
    for (int y = 0; y < W; ++y)
#pragma unroll
      for (int x = 0; x < W; ++x)
#pragma unroll
        for (int r = 0; r < 4; ++r) to[(16 * x + r) * S::SIDE + y / COLS * S::SET + 16 * (y % COLS)] = sum[x][y][r];
    return;
  }
  with_activation_of<PASS>(a.act, [&](auto act) {
#pragma unroll
    for (int y = 0; y < COLS; ++y) {
      const int n = n0 + 16 * COLS * wc + 16 * y + r16;
      if (n >= N) continue;
      const float bg = bias_of<PASS>(a.b_gate, n), bu = bias_of<PASS>(a.b_up, n);
#pragma unroll
      for (int x = 0; x < W; ++x)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int m = m0 + wm + 16 * x + 4 * h + r;
          if (m < a.rows) finish_value<PASS, decltype(act)::value>(a, m, n, N, sum[x][y][r], sum[x][SETS ? y + W / 2 : y][r], bg, bu);
        }
    }
  });
}

// The parts' sums, in their order, a value (of both sets) to a thread.
template <int PASS, int SIDE>
__global__ void __launch_bounds__(kThreads) gated_f32_join_kernel(const GatedArgs a, int tiles_m, int tiles_n, int parts) {
  constexpr int SETS = PASS == kForward ? 2 : 1, WIDTH = SIDE / SETS, GROUPS = SIDE * WIDTH / kThreads;
  const int tiles = tiles_m * tiles_n, tile = blockIdx.x / GROUPS, at = blockIdx.x % GROUPS * kThreads + threadIdx.x;
  int tm, tn;
  grad_tile_of(tiles_m, tiles_n, tile, tm, tn);
  const int N = PASS == kInput ? a.d : a.f, m = tm * SIDE + at / WIDTH, n = tn * WIDTH + at % WIDTH;
  if (m >= a.rows || n >= N) return;
  const float* from = a.partial + (int64_t)tile * (SIDE * SIDE) + at / WIDTH * SIDE + at % WIDTH;
  float v[2] = {0.f, 0.f};
#pragma unroll 4
  for (int p = 0; p < parts; ++p, from += (int64_t)tiles * (SIDE * SIDE))
#pragma unroll
    for (int set = 0; set < SETS; ++set) v[set] += from[set * WIDTH];
  const float bg = bias_of<PASS>(a.b_gate, n), bu = bias_of<PASS>(a.b_up, n);
  with_activation_of<PASS>(a.act, [&](auto act) { finish_value<PASS, decltype(act)::value>(a, m, n, N, v[0], v[1], bg, bu); });
}

// dgate and dup where dh is given, VEC values a thread at a time.  Bound by memory.
template <int DT, int VEC>
__global__ void __launch_bounds__(kThreads) gated_slopes_kernel(const GatedArgs a, int64_t n) {
  for (int64_t at = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * VEC; at < n; at += (int64_t)gridDim.x * kThreads * VEC) {
    Values<DT, VEC> dh, gate, up;
    dh.load(a.dy, at);
    gate.load(a.gate, at);
    up.load(a.up, at);
    float dg[VEC], du[VEC];
    with_activation(a.act, [&](auto act) {
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        float slope;
        const float v = activation<decltype(act)::value, DT == DP_F32, true>(gate.get(k), slope);
        dg[k] = dh.get(k) * up.get(k) * slope;
        du[k] = dh.get(k) * v;
      }
    });
    gate.set(dg);
    up.set(du);
    gate.store(a.dgate, at);
    up.store(a.dup, at);
  }
}

template <int DT>
dp_status launch_slopes(const GatedArgs& a, hipStream_t s) {
  const int64_t n = (int64_t)a.rows * a.f;
  constexpr int WIDE = DT == DP_F32 ? 4 : 8;
  const uintptr_t all = (uintptr_t)a.dy | (uintptr_t)a.gate | (uintptr_t)a.up | (uintptr_t)a.dgate | (uintptr_t)a.dup;
  const bool wide = all % 16 == 0 && n % WIDE == 0;
  const int64_t threads = wide ? n / WIDE : n, blocks = std::min<int64_t>((threads + kThreads - 1) / kThreads, 1 << 20);
  if (wide)
    gated_slopes_kernel<DT, WIDE><<<dim3((unsigned)blocks), kThreads, 0, s>>>(a, n);
  else
    gated_slopes_kernel<DT, 1><<<dim3((unsigned)blocks), kThreads, 0, s>>>(a, n);
  return hip_status(hipGetLastError());
}

// Tiles of 128 x 128 where they are one to a compute unit at least, else of 64 x 64; of few small ones the contraction is dealt to several
// workgroups: a stage is 0.9 us of one alone on a compute unit, 0.65 of each of several, and the join a launch and its traffic.
// Rows x d x f, one workgroup to a tile and several, us: input gradients 12 x 768 x 2048 103, 14; 512 x 768 x 2048 105, 41; forward
// 512 x 7416 x 216 222, 49.
struct F32Choice {
  bool large;
  int tiles_m, tiles_n, parts;
};
F32Choice choose_f32(GatedPass pass, int rows, int d, int f, int d_out) {
  const int N = pass == kInput ? d : f, K = pass == kForward ? d : pass == kHidden ? d_out : f, sets = pass == kForward ? 2 : 1;
  const int stages = (K + kTerms - 1) / kTerms * (pass == kInput ? 2 : 1);
  F32Choice c = {(int64_t)((rows + 127) / 128) * (((int64_t)N * sets + 127) / 128) >= 256, 0, 0, 1};
  const int side = c.large ? 128 : 64;
  c.tiles_m = (rows + side - 1) / side;
  c.tiles_n = (int)(((int64_t)N * sets + side - 1) / side);
  if (c.large) return c;
  const int64_t tiles = (int64_t)c.tiles_m * c.tiles_n;
  float best = 0.f;
  for (const int parts : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}) {
    if (parts > 1 && 2 * parts > stages) break;
    float cost = (float)((stages + parts - 1) / parts) * std::max(0.9f, 0.65f * (float)((tiles * parts + 255) / 256));
    if (parts > 1) cost += 5.f + (float)tiles * (float)parts * 0.012f;
    if (parts > 1 && cost >= best) continue;
    best = cost;
    c.parts = parts;
  }
  return c;
}

template <int PASS, int W>
dp_status launch_f32_tiles(const GatedArgs& a, const F32Choice& c, hipStream_t s) {
  typedef F32Tile<W, PASS == kForward> S;
  static ReadyTable ready;
  dp_status st = allow_big_lds(gated_f32_kernel<PASS, W>, 2 * S::STAGE_BYTES, ready);
  if (st != DP_OK) return st;
  const unsigned tiles = (unsigned)c.tiles_m * c.tiles_n;
  gated_f32_kernel<PASS, W><<<dim3(tiles * c.parts), kThreads, 2 * S::STAGE_BYTES, s>>>(a, c.tiles_m, c.tiles_n, c.parts);
  st = hip_status(hipGetLastError());
  if constexpr (W == 2) {
    if (st != DP_OK || c.parts == 1) return st;
    constexpr unsigned GROUPS = S::SIDE * S::SIDE / kThreads / (PASS == kForward ? 2 : 1);
    gated_f32_join_kernel<PASS, S::SIDE><<<dim3(tiles * GROUPS), kThreads, 0, s>>>(a, c.tiles_m, c.tiles_n, c.parts);
    st = hip_status(hipGetLastError());
  }
  return st;
}

template <int PASS>
dp_status launch_f32(const GatedArgs& a, hipStream_t s) {
  const F32Choice c = choose_f32((GatedPass)PASS, a.rows, a.d, a.f, a.d_out);
  return c.large ? launch_f32_tiles<PASS, 4>(a, c, s) : launch_f32_tiles<PASS, 2>(a, c, s);
}

}  // namespace

GatedLaunches gated_launches(dp_dtype dt, GatedPass pass, int rows, int d, int f, int d_out) {
  if (dt != DP_F32) return gated_tiles_launches(pass, rows, d, f, d_out);
  const F32Choice c = choose_f32(pass, rows, d, f, d_out);
  const int64_t tiles = (int64_t)c.tiles_m * c.tiles_n;
  return {kGatedTiles32, c.large ? tiles : 0, !c.large && c.parts == 1 ? tiles : 0, c.parts > 1 ? tiles : 0, c.parts > 1 ? c.parts : 0, c.parts > 1 ? 64 : 0};
}

size_t gated_workspace(dp_dtype dt, GatedPass pass, int rows, int d, int f, int d_out) {
  if (dt != DP_F32) return gated_tiles_workspace(pass, rows, d, f, d_out);
  const F32Choice c = choose_f32(pass, rows, d, f, d_out);
  return c.parts == 1 ? 0 : (size_t)c.parts * c.tiles_m * c.tiles_n * (64 * 64) * sizeof(float);
}

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
