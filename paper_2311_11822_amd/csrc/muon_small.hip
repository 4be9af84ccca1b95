// The step of muon.hip for matrices that one workgroup holds: all of it in one launch, X, A and its polynomial in LDS as fp32, products on the
// fp32 matrix instructions.  What counts there is the chain of 3 products an iteration, each behind a barrier: five matrices of 24 x 24 to
// 24 x 72 took 112 us in 18 launches.
#include <algorithm>

#include "muon.h"
#include "piece.h"

namespace dpbk {

namespace {

constexpr int kThreads = 512, kWaves = kThreads / 64, kPartBytes = kWaves * 1024, kLds = 160 * 1024 - 64 - kPartBytes;

struct SmallGroup {
  int n, iterations, grad_dt, copy_dt;
  float beta, ahead, grad_scale, eps;
  float abc[kMuonMostIterations][3];
  MuonTensor t[kMuonGroup];
};

__host__ __device__ inline int sixteens(int n) { return (n + 15) & ~15; }
// Floats from one row to the next: 16-byte reads of sixteen rows fall on different banks.
__host__ __device__ inline int pitch_of(int n) { return sixteens(n) + 4; }
__host__ __device__ inline int64_t small_floats(int m, int n) { return (int64_t)sixteens(m) * (pitch_of(n) + 2 * pitch_of(m)); }

// Whether waves share the tiles of A (one or four of them): 8 x 1000 56 us without, 39 with; 16 x 16 8.1 and 8.7.
__host__ __device__ inline bool is_long(int m, int n) { return m <= 32 && n > 240; }

__device__ __forceinline__ float value(const void* base, int dt, int64_t at) {
  if (dt == DP_F32) return static_cast<const float*>(base)[at];
  const uint16_t bits = static_cast<const uint16_t*>(base)[at];
  return dt == DP_BF16 ? __uint_as_float((uint32_t)bits << 16) : (float)__builtin_bit_cast(_Float16, bits);
}

// acc += rows i0 .. of p times rows j0 .. of q, k terms (a multiple of 16).  A lane has row lane % 16 of both and 4 terms of every 16: which terms an
// instruction adds is the same for both.  Result: row i0 + 4 (lane / 16) + r, column j0 + lane % 16.
__device__ __forceinline__ f32x4 rows_product(const float* p, const float* q, int pitch_p, int pitch_q, int i0, int j0, int k, int lane) {
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  const float* a = p + (i0 + (lane & 15)) * pitch_p + 4 * (lane >> 4);
  const float* b = q + (j0 + (lane & 15)) * pitch_q + 4 * (lane >> 4);
#pragma unroll 4
  for (int c = 0; c < k; c += 16) {
    const f32x4 x = *reinterpret_cast<const f32x4*>(a + c), y = *reinterpret_cast<const f32x4*>(b + c);
#pragma unroll
    for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], y[e], acc, 0, 0, 0);
  }
  return acc;
}

// LONG: some matrix's A has few tiles of a long contraction, which several waves share.
template <bool LONG>
__global__ void __launch_bounds__(kThreads) muon_small_kernel(const SmallGroup g) {
  extern __shared__ __align__(16) float lds[];
  __shared__ float red[kWaves], part[LONG ? kWaves : 1][256];
  const MuonTensor& t = g.t[blockIdx.x];
  const bool turned = t.rows > t.cols;
  const int m = turned ? t.cols : t.rows, n = turned ? t.rows : t.cols, mp = sixteens(m), np = sixteens(n), px = pitch_of(n), pa = pitch_of(m);
  float *const X = lds, *const A = X + mp * px, *const P = A + mp * pa;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, size = t.rows * t.cols;
  for (int i = tid; i < mp * px; i += kThreads) X[i] = 0.f;
  __syncthreads();
  float sum = 0.f;
  for (int i = tid; i < size; i += kThreads) {
    const int row = i / t.cols, col = i - row * t.cols;
    const float grad = value(t.grad, g.grad_dt, i) * g.grad_scale, mom = fmaf(g.beta, t.momentum[i], grad);
    t.momentum[i] = mom;
    const float u = g.ahead < 0.f ? mom : fmaf(g.ahead, mom, grad);
    X[turned ? col * px + row : row * px + col] = u;
    sum = fmaf(u, u, sum);
  }
  for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off);
  if (lane == 0) red[wave] = sum;
  __syncthreads();
  sum = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) sum += red[w];
  const float norm = sqrtf(sum) + g.eps;
  for (int i = tid; i < mp * px; i += kThreads) X[i] = norm == 0.f ? 0.f : X[i] / norm;
  __syncthreads();
  const int tiles = mp / 16, shares = LONG && is_long(m, n) ? kWaves / (tiles * tiles) : 1, tile = wave / shares, share = wave - tile * shares;
  const int begin = share * (np / 16) / shares * 16, end = (share + 1) * (np / 16) / shares * 16;
  for (int it = 0; it < g.iterations; ++it) {
    const float a = g.abc[it][0], b = g.abc[it][1], c = g.abc[it][2];
    for (int k = tile; k < tiles * tiles; k += kWaves) {
      const int i0 = k / tiles * 16, j0 = (k - k / tiles * tiles) * 16;
      const f32x4 acc = rows_product(X + begin, X + begin, px, px, i0, j0, end - begin, lane);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int i = 4 * (lane >> 4) + r, j = lane & 15;
        if (shares > 1)
          part[wave][i * 16 + j] = acc[r];
        else
          A[(i0 + i) * pa + j0 + j] = acc[r];
      }
    }
    __syncthreads();
    if (shares > 1) {
      for (int e = tid; e < tiles * tiles * 256; e += kThreads) {
        const int k = e >> 8, i0 = k / tiles * 16, j0 = (k - k / tiles * tiles) * 16;
        float s = 0.f;
        for (int w = 0; w < shares; ++w) s += part[k * shares + w][e & 255];
        A[(i0 + (e >> 4 & 15)) * pa + j0 + (e & 15)] = s;
      }
      __syncthreads();
    }
    for (int k = wave; k < tiles * tiles; k += kWaves) {
      const int i0 = k / tiles * 16, j0 = (k - k / tiles * tiles) * 16;
      const f32x4 acc = rows_product(A, A, pa, pa, i0, j0, mp, lane);          // A is symmetric
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int i = i0 + 4 * (lane >> 4) + r, j = j0 + (lane & 15);
        P[i * pa + j] = fmaf(c, acc[r], b * A[i * pa + j]) + (i == j ? a : 0.f);
      }
    }
    __syncthreads();
    // sixteen columns of X to a wave, in place; its row tiles four at a time
    for (int s = wave; s < np / 16; s += kWaves) {
      float* const x = X + 16 * s + (lane & 15);
      f32x4 acc[kMuonSmallTiles];
#pragma unroll
      for (int i = 0; i < kMuonSmallTiles; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      for (int k = 0; k < mp; k += 16) {
        f32x4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = x[(k + 4 * (lane >> 4) + e) * px];
#pragma unroll
        for (int i = 0; i < kMuonSmallTiles; ++i)
          if (i < tiles) {
            const f32x4 p = *reinterpret_cast<const f32x4*>(P + (16 * i + (lane & 15)) * pa + k + 4 * (lane >> 4));
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(p[e], y[e], acc[i], 0, 0, 0);
          }
      }
#pragma unroll
      for (int i = 0; i < kMuonSmallTiles; ++i)
        if (i < tiles)
#pragma unroll
          for (int r = 0; r < 4; ++r) x[(16 * i + 4 * (lane >> 4) + r) * px] = acc[i][r];
    }
    __syncthreads();
  }
  for (int i = tid; i < size; i += kThreads) {
    const int row = i / t.cols, col = i - row * t.cols;
    float w = fmaf(t.keep, t.param[i], -t.rate * X[turned ? col * px + row : row * px + col]);
    asm("" : "+v"(w));                                // the copy is the parameter rounded, not the sum
    t.param[i] = w;
    if (g.copy_dt == DP_BF16) static_cast<__bf16*>(t.copy)[i] = (__bf16)w;
    if (g.copy_dt == DP_F16) static_cast<_Float16*>(t.copy)[i] = (_Float16)w;
  }
}

template <bool LONG>
dp_status launch(const SmallGroup& g, int64_t floats, hipStream_t s) {
  static ReadyTable ready;
  const dp_status st = allow_big_lds(muon_small_kernel<LONG>, kLds, ready);
  if (st != DP_OK) return st;
  muon_small_kernel<LONG><<<dim3((unsigned)g.n), kThreads, (size_t)floats * 4, s>>>(g);
  return hip_status(hipGetLastError());
}

}  // namespace

// One compute unit's fp32 matrix instructions take some 2 us to 2^20 multiply-adds of an iteration.
bool muon_is_small(int rows, int cols) {
  const int m = std::min(rows, cols), n = std::max(rows, cols);
  return m <= 16 * kMuonSmallTiles && n <= 8192 && small_floats(m, n) * 4 <= kLds && (int64_t)sixteens(m) * sixteens(m) * sixteens(n) <= 1 << 20;
}

dp_status launch_muon_small(const MuonTensor* tensors, int n, const MuonArgs& a, dp_dtype grad_dt, dp_dtype copy_dt, hipStream_t s) {
  SmallGroup g = {};
  g.n = n;
  g.iterations = a.iterations;
  g.grad_dt = grad_dt;
  g.copy_dt = copy_dt;
  g.beta = a.beta;
  g.ahead = a.ahead;
  g.grad_scale = a.grad_scale;
  g.eps = a.eps;
  for (int k = 0; k < a.iterations; ++k)
    for (int i = 0; i < 3; ++i) g.abc[k][i] = (float)a.coefficients[3 * k + i];
  int64_t floats = 0;
  bool any_long = false;
  for (int i = 0; i < n; ++i) {
    g.t[i] = tensors[i];
    const int rows = std::min(tensors[i].rows, tensors[i].cols), cols = std::max(tensors[i].rows, tensors[i].cols);
    floats = std::max(floats, small_floats(rows, cols));
    any_long = any_long || is_long(rows, cols);
  }
  return any_long ? launch<true>(g, floats, s) : launch<false>(g, floats, s);
}

}  // namespace dpbk
