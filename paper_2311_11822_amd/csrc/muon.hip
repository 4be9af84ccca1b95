// An optimizer step on matrices whose update is orthogonalised:
//   m = beta m + g,  u = g + beta m (or m),  X = u / (|u| + eps);  so many times  X <- (a + b A + c A^2) X,  A = X X';
//   param = keep param - rate X.
// X is taken with its shorter side as rows (turned on the way in and out), so A is the smaller square.
//
// Products next to fp32's (X 0.6 to 0.8 times as far off as with those for random matrices, up to 2.3 times where singular values span four decades) at
// the rate of 16-bit ones: a value v is kept as two fp16 numbers, h = fp16(2^12 v) and l = fp16(2^12 v - h),
// together within 2^-23 of v (2^-37 of 1 where v is next to nothing), and h h' + h l' + l h' is added up in fp32; l l', 2^-24 of it, is left
// out.  A row is lines of 32 columns' h and l (product.h).  2^12 keeps the halves of entries from 2^-15 up out of fp16's subnormal range;
// entries are bounded by singular values, which the host has followed through the polynomials.  (fp32 matrix instructions have 1/16 of the 16-bit
// ones' rate, three products for one have 1/3.)
// A, the square and the polynomial of A are symmetric: tiles on and above the diagonal are formed, and leave turned as well.
// Matrices travel together: a launch does one step of up to 64 of them.  60 matrices of 768 x 768 to 768 x 2304 (85 M elements), us: momentum 190,
// start 250, five times A 205, polynomial 127 and update 363, parameters 270; the elementwise passes move 3.2 GB, 650 us of a copy, the products are
// 468 us an iteration at the rate of a large library product.
#include <math.h>

#include <algorithm>

#include "muon.h"
#include "piece.h"
#include "product.h"

namespace dpbk {

namespace {

constexpr int kThreads = 256, kSide = 64;            // elementwise passes: squares of 64 x 64
constexpr float kScale = 4096.f;

struct Matrix {
  float* param;
  const void* grad;
  float* momentum;
  void* copy;
  _Float16 *x[2], *gram, *poly;                      // [m][n or m, to a multiple of 32][2]: 32 h, 32 l, 32 h ...
  int rows, cols;
  float keep, rate;
  int parts;                                         // partial sums of |u|^2, at `partial`
  unsigned begin;                                    // first workgroup
  float* partial;
};
struct Group {
  int n;
  float beta, ahead, grad_scale, eps;
  float a, b, c;
  int from;                                          // x[from] is X, x[1 - from] what comes of it
  float* sums;                                       // of A's tiles whose contraction is dealt to several workgroups
  Matrix t[kMuonGroup];
};

__host__ __device__ inline int blocks_of(int n) { return (n + 31) & ~31; }
// Where h of a row's column is; l is 32 on.
__host__ __device__ inline int64_t half_at(int row, int col, int width) { return (int64_t)row * 2 * width + (col >> 5) * 64 + (col & 31); }
__host__ __device__ inline int64_t part_values(int64_t size) {
  const int64_t per = (size + kMuonParts - 1) / kMuonParts;
  return per < 4096 ? 4096 : (per + 1023) / 1024 * 1024;
}

// The matrix that owns workgroup `id`; whole waves call.
__device__ __forceinline__ int owner(const Group& g, unsigned id) {
  static_assert(kMuonGroup <= 64, "a lane to a matrix");
  const int lane = threadIdx.x & 63;
  const unsigned begin = g.t[lane < g.n ? lane : 0].begin;
  return __builtin_amdgcn_readfirstlane(__builtin_popcountll(__ballot(lane < g.n && begin <= id)) - 1);
}

__device__ __forceinline__ float block_sum(float x, float* red) {
  for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) s += red[w];
  return s;
}

// m = beta m + g, and a part's sum of u^2.  Bound by memory.
template <int DT>
__global__ void __launch_bounds__(kThreads) muon_momentum_kernel(const Group g) {
  __shared__ float red[kThreads / 64];
  const Matrix& t = g.t[owner(g, blockIdx.x)];
  const int part = blockIdx.x - t.begin;
  const int64_t size = (int64_t)t.rows * t.cols, per = part_values(size), first = part * per, end = first + per < size ? first + per : size;
  float sum = 0.f;
  for (int64_t i = first + threadIdx.x; i < end; i += kThreads) {
    Values<DT, 1> v;
    v.load(t.grad, i);
    const float grad = v.get(0) * g.grad_scale, m = fmaf(g.beta, t.momentum[i], grad);
    t.momentum[i] = m;
    const float u = g.ahead < 0.f ? m : fmaf(g.ahead, m, grad);
    sum = fmaf(u, u, sum);
  }
  sum = block_sum(sum, red);
  if (threadIdx.x == 0) t.partial[part] = sum;
}

struct Halves {
  _Float16 h, l;
  __device__ __forceinline__ explicit Halves(float v) : h((_Float16)v), l((_Float16)(v - (float)h)) {}
};

// A square of X = u / (|u| + eps), turned where the matrix is higher than wide; zeros behind its columns.
template <int DT>
__global__ void __launch_bounds__(kThreads) muon_start_kernel(const Group g) {
  __shared__ float red[kThreads / 64], tile[kSide][kSide + 1];
  const Matrix& t = g.t[owner(g, blockIdx.x)];
  const bool turned = t.rows > t.cols;
  const int m = turned ? t.cols : t.rows, n = turned ? t.rows : t.cols, pitch = blocks_of(n), across = (pitch + kSide - 1) / kSide;
  float sum = 0.f;
  for (int i = threadIdx.x; i < t.parts; i += kThreads) sum += t.partial[i];
  const float norm = sqrtf(block_sum(sum, red)) + g.eps;            // (0: all of u is, and X with it)
  const int id = blockIdx.x - t.begin, r0 = id / across * kSide, c0 = (id - id / across * across) * kSide;       // of X
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  auto value = [&](int64_t i) {
    Values<DT, 1> v;
    v.load(t.grad, i);
    const float m1 = t.momentum[i];
    return g.ahead < 0.f ? m1 : fmaf(g.ahead, m1, v.get(0) * g.grad_scale);
  };
#pragma unroll
  for (int k = wave; k < kSide; k += kThreads / 64) {            // rows of the matrix as it lies
    const int row = (turned ? c0 : r0) + k, col = (turned ? r0 : c0) + lane;
    tile[k][lane] = row < t.rows && col < t.cols ? value((int64_t)row * t.cols + col) : 0.f;
  }
  __syncthreads();
  _Float16* const x = t.x[g.from];
  for (int k = wave; k < kSide; k += kThreads / 64) {
    const int r = r0 + k, c = c0 + lane;
    if (r < m && c < pitch) {
      const float u = turned ? tile[lane][k] : tile[k][lane];
      const Halves v(norm == 0.f ? 0.f : u / norm * kScale);
      const int64_t at = half_at(r, c, pitch);
      x[at] = v.h;
      x[at + 32] = v.l;
    }
  }
}

// param = keep param - rate X, and its 16-bit copy.
template <int DT>                                    // of the copy; DP_F32: none
__global__ void __launch_bounds__(kThreads) muon_apply_kernel(const Group g) {
  __shared__ float tile[kSide][kSide + 1];
  const Matrix& t = g.t[owner(g, blockIdx.x)];
  const bool turned = t.rows > t.cols;
  const int m = turned ? t.cols : t.rows, n = turned ? t.rows : t.cols, pitch = blocks_of(n), across = (n + kSide - 1) / kSide;
  const int id = blockIdx.x - t.begin, r0 = id / across * kSide, c0 = (id - id / across * across) * kSide;       // of X
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const _Float16* const x = t.x[g.from];
  constexpr int WAVES = kThreads / 64, PER = kSide / WAVES;
  float param[PER];                                  // on its way while X is turned
  const int col = (turned ? r0 : c0) + lane;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int row = (turned ? c0 : r0) + wave + i * WAVES;
    param[i] = row < t.rows && col < t.cols ? t.param[(int64_t)row * t.cols + col] : 0.f;
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int k = wave + i * WAVES, r = r0 + k, c = c0 + lane;
    if (r < m && c < n) {
      const int64_t at = half_at(r, c, pitch);
      tile[k][lane] = ((float)x[at] + (float)x[at + 32]) * (1.f / kScale);
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int k = wave + i * WAVES, row = (turned ? c0 : r0) + k;
    if (row < t.rows && col < t.cols) {
      const int64_t at = (int64_t)row * t.cols + col;
      float w = fmaf(t.keep, param[i], -t.rate * (turned ? tile[lane][k] : tile[k][lane]));
      asm("" : "+v"(w));                              // the copy is the parameter rounded, not the sum (v_fma_mixlo_f16)
      t.param[at] = w;
      if constexpr (DT != DP_F32) {
        Values<DT, 1> v;
        v.set({w});
        v.store(t.copy, at);
      }
    }
  }
}

enum MuonStep { kGram, kPoly, kUpdate };

// Eight values of a row as halves; col is a multiple of 8.
__device__ __forceinline__ void put_halves(_Float16* out, int pitch, int row, int col, const float (&v)[8]) {
  f16x8 h, l;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const Halves w(v[k]);
    h[k] = w.h;
    l[k] = w.l;
  }
  f16x8* const to = reinterpret_cast<f16x8*>(out + half_at(row, col, pitch));
  to[0] = h;
  to[4] = l;
}

// Where a symmetric result's tile lies: tile row by tile row from the diagonal on.
__device__ __forceinline__ void place_above(int tiles_m, int rest, int& tm, int& tn) {
  for (tm = 0; rest >= tiles_m - tm; ++tm) rest -= tiles_m - tm;
  tn = tm + rest;
}

constexpr int kDealtSide = 128;                      // of tiles that are dealt in parts

// Tiles of one step.  DEALT: each has `parts` workgroups, whose sums go to memory: [part][tile][row][column].
template <int STEP, class S, bool DEALT>
__global__ void __launch_bounds__(S::NT, 163840 / S::LDS_BYTES) muon_product_kernel(const Group g, int total, int parts) {
  extern __shared__ __attribute__((aligned(1024))) unsigned char lds_raw[];
  const unsigned lds0 = (unsigned)(uintptr_t)lds_raw;
  const int id = grad_logical_tile(blockIdx.x, DEALT ? total * parts : total), part = DEALT ? id / total : 0, logical = id - part * total;
  const Matrix& t = g.t[owner(g, logical)];
  const int m = imin(t.rows, t.cols), mp = blocks_of(m), np = blocks_of(imax(t.rows, t.cols));
  const int tiles_m = (m + S::BM - 1) / S::BM;
  int tm, tn, rest = logical - (int)t.begin;
  if constexpr (STEP == kUpdate) {
    grad_tile_of(tiles_m, (np + S::BN - 1) / S::BN, rest, tm, tn);
  } else {
    place_above(tiles_m, rest, tm, tn);
  }
  const int m0 = tm * S::BM, n = tn * S::BN, n0[2] = {n, n};
  const _Float16 *a, *b;
  ProductShape p;
  p.M = m;
  p.N = STEP == kUpdate ? np : m;
  p.segments = 1;
  p.terms = m;
  p.first = 0;
  if constexpr (STEP == kGram) {
    a = b = t.x[g.from];
    p.K = p.lda = p.ldb = 2 * np;
  } else if constexpr (STEP == kPoly) {
    a = b = t.gram;
    p.K = p.lda = p.ldb = 2 * mp;
  } else {
    a = t.poly;
    b = t.x[g.from];
    p.ldb = 2 * np;
    p.K = p.lda = 2 * mp;
  }
  p.stages = p.K / kProductTerms;
  if constexpr (DEALT) {
    p.first = part * p.stages / parts;
    p.stages = (part + 1) * p.stages / parts - p.first;
  }
  p.s[0] = p.s[1] = {a, b, b};
  f32x4 acc[S::TM][S::TN];
  product_tile<S, true>(p, m0, n0, lds0, acc);
  _Float16* const out = STEP == kGram ? t.gram : STEP == kPoly ? t.poly : t.x[1 - g.from];
  const int pitch = STEP == kUpdate ? np : mp;
  if constexpr (DEALT) {
    float* const sums = g.sums + ((int64_t)part * total + logical) * (S::BM * S::BN);
    NothingAhead<S, false> ahead(NoLoad{});
    product_rows<S, false>(acc, lds0, ahead, [&](int row, int col, int, const float (&acc8)[2][8], Nothing) {
      f32x4* const to = reinterpret_cast<f32x4*>(sums + row * S::BN + col);
      to[0] = f32x4{acc8[0][0], acc8[0][1], acc8[0][2], acc8[0][3]};
      to[1] = f32x4{acc8[0][4], acc8[0][5], acc8[0][6], acc8[0][7]};
    });
    return;
  }
  // what is stored of eight values of the product
  auto finish = [&](int row, int col, const float (&acc8)[8], float (&v)[8]) {
    if constexpr (STEP == kPoly) {
      const f16x8* const from = reinterpret_cast<const f16x8*>(t.gram + half_at(row, col, mp));
      const f16x8 h = from[0], l = from[4];
#pragma unroll
      for (int k = 0; k < 8; ++k)
        v[k] = fmaf(g.c / kScale, acc8[k], g.b * ((float)h[k] + (float)l[k])) + (row == col + k ? g.a * kScale : 0.f);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = acc8[k] * (1.f / kScale);
    }
  };
  auto store = [&](int row, int col, int, const float (&acc8)[2][8], Nothing) {
    const int r = m0 + row, c = n + col;
    if (r >= m || c >= pitch) return;
    float v[8];
    finish(r, c, acc8[0], v);
    put_halves(out, pitch, r, c, v);
  };
  if constexpr (STEP == kUpdate) {
    NothingAhead<S, false> ahead(NoLoad{});
    product_rows<S, false>(acc, lds0, ahead, store);
  } else {
    // below the diagonal: rows of the tile's columns
    auto across = [&](int row, int col, const float (&acc8)[8]) {
      const int r = n + col, c = m0 + row;
      if (r >= m || c >= mp) return;
      float v[8];
      finish(r, c, acc8, v);
      put_halves(out, pitch, r, c, v);
    };
    NothingAhead<S, false> ahead(NoLoad{});
    product_rows<S, false>(acc, lds0, ahead, store, tm != tn, across);
  }
}

// The parts' sums of A's tiles, in their order: four workgroups to a tile, a square of 64 x 64 each.
__global__ void __launch_bounds__(kThreads) muon_join_kernel(const Group g, int total, int parts) {
  __shared__ float square[kSide][kSide + 1];
  const int logical = blockIdx.x / 4, quarter = blockIdx.x % 4;
  const Matrix& t = g.t[owner(g, logical)];
  const int m = imin(t.rows, t.cols), pitch = blocks_of(m);
  int tm, tn;
  place_above((m + kDealtSide - 1) / kDealtSide, logical - (int)t.begin, tm, tn);
  const int r0 = (quarter >> 1) * kSide, c0 = (quarter & 1) * kSide;
  const float* const from = g.sums + (int64_t)logical * (kDealtSide * kDealtSide);
#pragma unroll
  for (int i = 0; i < kSide * kSide / 8 / kThreads; ++i) {
    const int piece = threadIdx.x + i * kThreads, row = piece / 8, col = piece % 8 * 8;
    float v[8] = {};
#pragma unroll 4
    for (int p = 0; p < parts; ++p) {
      const f32x4* const at = reinterpret_cast<const f32x4*>(from + (int64_t)p * total * (kDealtSide * kDealtSide) + (r0 + row) * kDealtSide + c0 + col);
      const f32x4 x = at[0], y = at[1];
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] += x[k], v[4 + k] += y[k];
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) square[row][col + k] = v[k] *= 1.f / kScale;
    const int r = tm * kDealtSide + r0 + row, c = tn * kDealtSide + c0 + col;
    if (r < m && c < pitch) put_halves(t.gram, pitch, r, c, v);
  }
  if (tm == tn) return;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kSide * kSide / 8 / kThreads; ++i) {         // below the diagonal
    const int piece = threadIdx.x + i * kThreads, row = piece / 8, col = piece % 8 * 8;
    const int r = tn * kDealtSide + c0 + row, c = tm * kDealtSide + r0 + col;
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = square[col + k][row];
    if (r < m && c < pitch) put_halves(t.gram, pitch, r, c, v);
  }
}

template <class F>
unsigned lay_out(Group& g, F workgroups) {
  unsigned total = 0;
  for (int i = 0; i < g.n; ++i) {
    g.t[i].begin = total;
    total += (unsigned)workgroups(g.t[i]);
  }
  return total;
}

template <int STEP, int SIDE, class T>
int64_t tiles_of(const T& t) {
  const int64_t m = std::min(t.rows, t.cols), n = blocks_of(std::max(t.rows, t.cols)), tm = (m + SIDE - 1) / SIDE;
  return STEP == kUpdate ? tm * ((n + SIDE - 1) / SIDE) : tm * (tm + 1) / 2;
}

// Large tiles or small ones, and of how many workgroups each.  256 large ones are resident, 2.2 us to a stage of 32 terms; 512 small ones, 1.2 us, or
// 256 at 0.6; and what comes before and after a contraction.  Workgroups are dealt out in order, the longest first: a launch takes their sum over
// those that are resident, and some of the longest besides.  A of few matrices, whose rows are long, has few tiles: their contraction is dealt to
// `parts` workgroups, for one more launch and the sums' way through memory.  A step of one matrix, its contractions whole and in parts, us:
// 768 x 2304 507, 352; 1280 x 3456 812, 615; 300 x 5000 671, 271; 8 x 4096 459, 152; 128 x 32768 3160, 285; 768 x 50264 5880, 1820.
struct StepChoice {
  bool large;
  int parts;
  int64_t tiles;
};
template <int STEP, class T>
StepChoice choose_step(const T* t, int n) {
  constexpr float kBigStage = 2.2f, kBigRest = STEP == kUpdate ? 12.f : 30.f, kMidStage = 1.2f, kMidRest = STEP == kUpdate ? 10.f : 18.f;
  int64_t big = 0, mid = 0, big_stages = 0, mid_stages = 0, longest = 0, shortest = INT64_MAX;
  for (int i = 0; i < n; ++i) {
    const int64_t stages = ((STEP == kGram ? std::max(t[i].rows, t[i].cols) : std::min(t[i].rows, t[i].cols)) + kHalfTerms - 1) / kHalfTerms;
    big += tiles_of<STEP, 256>(t[i]);
    mid += tiles_of<STEP, 128>(t[i]);
    big_stages += stages * tiles_of<STEP, 256>(t[i]);
    mid_stages += stages * tiles_of<STEP, 128>(t[i]);
    longest = std::max(longest, stages);
    shortest = std::min(shortest, stages);
  }
  auto cost = [&](int64_t tiles, int64_t tile_stages, float stage, float rest, float resident) {
    const float one = (float)longest * stage + rest;
    return (float)tiles <= resident ? one : ((float)tile_stages * stage + (float)tiles * rest) / resident + one / 2;
  };
  const float large = cost(big, big_stages, kBigStage, kBigRest, 256.f);
  const float small = mid <= 256 ? 0.6f * (float)longest + 7.f : cost(mid, mid_stages, kMidStage, kMidRest, 512.f);
  StepChoice c = {large <= small, 1, mid};
  if constexpr (STEP == kGram) {
    float best = std::min(large, small);
    for (const int parts : {2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64, 96, 128}) {
      const int64_t pieces = mid * parts;
      if (pieces > 512 || 4 * parts > shortest) break;
      const float dealt = (pieces <= 256 ? 0.6f : 1.2f) * (float)longest / parts + 13.f + 0.02f * (float)pieces + 0.3f * (float)parts;
      if (dealt >= best) continue;
      best = dealt;
      c.large = false;
      c.parts = parts;
    }
  }
  return c;
}

template <int STEP, class S, bool DEALT = false>
dp_status launch_product(Group& g, int parts, hipStream_t s) {
  static ReadyTable ready;
  const dp_status st = allow_big_lds(muon_product_kernel<STEP, S, DEALT>, S::LDS_BYTES, ready);
  if (st != DP_OK) return st;
  const unsigned total = lay_out(g, [](const Matrix& t) { return tiles_of<STEP, S::BM>(t); });
  muon_product_kernel<STEP, S, DEALT><<<dim3(total * parts), S::NT, S::LDS_BYTES, s>>>(g, (int)total, parts);
  if constexpr (DEALT) muon_join_kernel<<<dim3(total * 4), kThreads, 0, s>>>(g, (int)total, parts);
  return hip_status(hipGetLastError());
}

template <int STEP>
dp_status launch_step(Group& g, hipStream_t s) {
  constexpr ProductB B = STEP == kUpdate ? kSplitColumns : kRowsOfTerms;
  const StepChoice c = choose_step<STEP>(g.t, g.n);
  if constexpr (STEP == kGram)
    if (c.parts > 1) return launch_product<STEP, MidProduct<B, true>, true>(g, c.parts, s);
  return c.large ? launch_product<STEP, BigProduct<B, true>>(g, 1, s) : launch_product<STEP, MidProduct<B, true>>(g, 1, s);
}

// Bytes of a matrix's two X, A, polynomial and partial sums.
size_t matrix_bytes(int rows, int cols, size_t (&at)[5]) {
  const int64_t m = std::min(rows, cols), n = std::max(rows, cols);
  const size_t x = (size_t)4 * m * blocks_of((int)n), square = (size_t)4 * m * blocks_of((int)m), sizes[5] = {x, x, square, square, kMuonParts * 4};
  size_t total = 0;
  for (int i = 0; i < 5; ++i) {
    at[i] = total;
    total += (sizes[i] + 255) / 256 * 256;
  }
  return total;
}

}  // namespace

void muon_launches(const MuonTensor* tensors, int n, MuonLaunches (&steps)[3]) {
  const StepChoice c[3] = {choose_step<kGram>(tensors, n), choose_step<kPoly>(tensors, n), choose_step<kUpdate>(tensors, n)};
  for (int i = 0; i < 3; ++i) steps[i] = {c[i].large ? 256 : kDealtSide, c[i].parts};
}

size_t muon_workspace(const MuonTensor* tensors, int n) {
  size_t total = 0, at[5];
  for (int i = 0; i < n; ++i) total += matrix_bytes(tensors[i].rows, tensors[i].cols, at);
  const StepChoice c = choose_step<kGram>(tensors, n);
  return total + (c.parts > 1 ? (size_t)c.parts * c.tiles * (kDealtSide * kDealtSide) * sizeof(float) : 0);
}

dp_status launch_muon(const MuonTensor* tensors, int n, const MuonArgs& a, dp_dtype grad_dt, dp_dtype copy_dt, void* ws, hipStream_t s) {
  Group g = {};
  g.n = n;
  g.beta = a.beta;
  g.ahead = a.ahead;
  g.grad_scale = a.grad_scale;
  g.eps = a.eps;
  char* base = static_cast<char*>(ws);
  int order[kMuonGroup];                             // the longest contractions first: others fill in behind them
  for (int i = 0; i < n; ++i) order[i] = i;
  std::stable_sort(order, order + n, [&](int i, int j) {
    return std::max(tensors[i].rows, tensors[i].cols) > std::max(tensors[j].rows, tensors[j].cols);
  });
  for (int i = 0; i < g.n; ++i) {
    const MuonTensor& from = tensors[order[i]];
    Matrix& t = g.t[i];
    size_t at[5];
    const size_t bytes = matrix_bytes(from.rows, from.cols, at);
    t.param = from.param;
    t.grad = from.grad;
    t.momentum = from.momentum;
    t.copy = from.copy;
    t.rows = from.rows;
    t.cols = from.cols;
    t.keep = from.keep;
    t.rate = from.rate;
    t.x[0] = reinterpret_cast<_Float16*>(base + at[0]);
    t.x[1] = reinterpret_cast<_Float16*>(base + at[1]);
    t.gram = reinterpret_cast<_Float16*>(base + at[2]);
    t.poly = reinterpret_cast<_Float16*>(base + at[3]);
    t.partial = reinterpret_cast<float*>(base + at[4]);
    const int64_t size = (int64_t)t.rows * t.cols;
    t.parts = (int)((size + part_values(size) - 1) / part_values(size));
    base += bytes;
  }
  g.sums = reinterpret_cast<float*>(base);
  auto launch = [&](auto kernel, unsigned total) {
    kernel<<<dim3(total), kThreads, 0, s>>>(g);
    return hip_status(hipGetLastError());
  };
  unsigned total = lay_out(g, [](const Matrix& t) { return t.parts; });
  dp_status st = launch(grad_dt == DP_F32    ? muon_momentum_kernel<DP_F32>
                        : grad_dt == DP_BF16 ? muon_momentum_kernel<DP_BF16>
                                             : muon_momentum_kernel<DP_F16>,
                        total);
  if (st != DP_OK) return st;
  auto squares = [](const Matrix& t, bool padded) {
    const int64_t m = std::min(t.rows, t.cols), c = std::max(t.rows, t.cols);
    return ((m + kSide - 1) / kSide) * (((padded ? blocks_of((int)c) : c) + kSide - 1) / kSide);
  };
  total = lay_out(g, [&](const Matrix& t) { return squares(t, true); });
  st = launch(grad_dt == DP_F32 ? muon_start_kernel<DP_F32> : grad_dt == DP_BF16 ? muon_start_kernel<DP_BF16> : muon_start_kernel<DP_F16>, total);
  for (int k = 0; k < a.iterations && st == DP_OK; ++k) {
    g.a = (float)a.coefficients[3 * k];
    g.b = (float)a.coefficients[3 * k + 1];
    g.c = (float)a.coefficients[3 * k + 2];
    st = launch_step<kGram>(g, s);
    if (st == DP_OK) st = launch_step<kPoly>(g, s);
    if (st == DP_OK) st = launch_step<kUpdate>(g, s);
    g.from = 1 - g.from;
  }
  if (st != DP_OK) return st;
  total = lay_out(g, [&](const Matrix& t) { return squares(t, false); });
  st = launch(copy_dt == DP_F32 ? muon_apply_kernel<DP_F32> : copy_dt == DP_BF16 ? muon_apply_kernel<DP_BF16> : muon_apply_kernel<DP_F16>, total);
  return st;
}

}  // namespace dpbk
