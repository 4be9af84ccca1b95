// Layer norm, forward and backward, with the clipped parameters' per-sample gradients.
//   y = h gain + bias,  h = (x - mean) rstd;   dx = rstd (u - mean(u) - h mean(u h)),  u = dy gain;
//   kept_i = (sum_t dy h, sum_t dy) of sample i,  sqnorm_i = |kept_i|^2.
// Streams over memory: a row is read once and held in registers (as stored) between its statistics and its result; the gradients of
// gain and bias grow in the registers of the lanes that hold their columns while a workgroup goes through its rows.
#include <algorithm>
#include <type_traits>

#include "train.h"

namespace dpbk {

namespace {

constexpr int kThreads = 512;

// P values a thread as pieces of VEC: piece n of thread t holds columns VEC (n TPR + t) ...
template <int DT, int VEC>
struct Piece {                                     // VEC values as stored, 16 bytes
  static constexpr int WORDS = 4, SIZE = DT == DP_F32 ? 4 : 2;
  uint32_t w[WORDS];
  __device__ __forceinline__ void load(const void* base, int64_t at) {
    const uint4 v = *reinterpret_cast<const uint4*>(static_cast<const char*>(base) + at * SIZE);
    w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
  }
  // The same where the array may end within the piece, `left` values on.
  __device__ __forceinline__ void load(const void* base, int64_t at, int64_t left) {
    if (left >= VEC) return load(base, at);
#pragma unroll
    for (int i = 0; i < WORDS; ++i) w[i] = 0;
#pragma unroll
    for (int k = 0; k < VEC; ++k)
      if (k < left) {
        if constexpr (DT == DP_F32)
          w[k] = static_cast<const uint32_t*>(base)[at + k];
        else
          w[k / 2] |= (uint32_t) static_cast<const uint16_t*>(base)[at + k] << (16 * (k & 1));
      }
  }
  __device__ __forceinline__ void store(void* base, int64_t at) const {
    *reinterpret_cast<uint4*>(static_cast<char*>(base) + at * SIZE) = make_uint4(w[0], w[1], w[2], w[3]);
  }
  // Values from..to - 1 of it.
  __device__ __forceinline__ void store(void* base, int64_t at, int from, int to) const {
    if (from <= 0 && to >= VEC) return store(base, at);
#pragma unroll
    for (int k = 0; k < VEC; ++k)
      if (k >= from && k < to) {
        if constexpr (DT == DP_F32)
          static_cast<uint32_t*>(base)[at + k] = w[k];
        else
          static_cast<uint16_t*>(base)[at + k] = (uint16_t)(w[k / 2] >> (16 * (k & 1)));
      }
  }
  __device__ __forceinline__ float get(int k) const {
    if constexpr (DT == DP_F32) return __uint_as_float(w[k]);
    const uint32_t pair = w[k / 2];
    if constexpr (DT == DP_BF16) return __uint_as_float(k & 1 ? pair & 0xFFFF0000u : pair << 16);
    return (float)__builtin_bit_cast(_Float16, (uint16_t)(k & 1 ? pair >> 16 : pair & 0xFFFFu));
  }
  // Rounded to nearest even, the only rounding of a result.
  __device__ __forceinline__ void set(const float (&x)[VEC]) {
    if constexpr (DT == DP_F32) {
#pragma unroll
      for (int k = 0; k < VEC; ++k) w[k] = __float_as_uint(x[k]);
    } else {
#pragma unroll
      for (int k = 0; k < WORDS; ++k) {
        const float lo = x[2 * k], hi = x[2 * k + 1];
        typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
        typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
        if constexpr (DT == DP_BF16)
          w[k] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)lo, (__bf16)hi});
        else
          w[k] = __builtin_bit_cast(uint32_t, f16x2{(_Float16)lo, (_Float16)hi});
      }
    }
  }
};

// Sums of N values over the TPR threads of a row, in every one of them.
template <int TPR, int N>
__device__ __forceinline__ void row_sums(float (&x)[N], float (*red)[N]) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1)
#pragma unroll
    for (int n = 0; n < N; ++n) x[n] += __shfl_xor(x[n], off);
  if constexpr (TPR > 64) {
    constexpr int WAVES = TPR / 64;
    const int wave = threadIdx.x >> 6;
    __syncthreads();                               // the last sums have been read
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int n = 0; n < N; ++n) red[wave][n] = x[n];
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) {
      x[n] = 0.f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) x[n] += red[w][n];
    }
  }
}

// A parameter's values of columns col ..; those outside of a row of d are whatever.
template <int VEC, bool SHIFT>
__device__ __forceinline__ void load_params(float (&v)[VEC], const float* p, int col, int d, float none) {
  typedef f32x4 Four __attribute__((aligned(4)));
  if (!p) {
#pragma unroll
    for (int k = 0; k < VEC; ++k) v[k] = none;
  } else if (!SHIFT || (col >= 0 && col + VEC <= d)) {
#pragma unroll
    for (int k = 0; k < VEC; k += 4) {
      const f32x4 four = *reinterpret_cast<const Four*>(p + col + k);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[k + i] = four[i];
    }
  } else {
#pragma unroll
    for (int k = 0; k < VEC; ++k) v[k] = p[min(max(col + k, 0), d - 1)];
  }
}

// A wave to a row of up to 2048 values, else a workgroup; registers hold the row between the two sums and the result (variance around
// the mean, not from a sum of squares: no cancellation).  Bound by memory: 8 x 512 rows of 1280 bf16 values with the residual sum, 42 MB in
// 8.9 us; 4 x 2048 x 12288 80 us, 5.0 TB/s, with the sum 147 us, 5.5 TB/s.
// SHIFT: rows of no whole number of pieces.  Pieces lie at 16 bytes all the same, the first `ahead` values of a row's first one belong to the
// row before; what a row does not own is loaded (where the array has it) but takes no part, and its own are stored one by one there.
// (2048 x 12289 fp16: 26 us, and 58 an element at a time.)
template <int DT, int VEC, int TPR, int P, bool SHIFT>
__global__ void __launch_bounds__(kThreads) layer_norm_kernel(const NormArgs a, int64_t rows, int first_block) {
  constexpr int N = P / VEC, GROUPS = kThreads / TPR;
  __shared__ float red[kThreads / 64][1];
  const int t = threadIdx.x % TPR;
  const int64_t row = ((int64_t)first_block + blockIdx.x) * GROUPS + threadIdx.x / TPR;
  if (TPR == 64 && row >= rows) return;            // (a whole workgroup's row otherwise: always there)
  const int64_t at = row * a.d, total = rows * a.d;
  const int ahead = SHIFT ? (int)(at & (VEC - 1)) : 0;
  auto own = [&](int col, int k) { return !SHIFT || (unsigned)(col + k) < (unsigned)a.d; };
  auto load = [&](Piece<DT, VEC>& p, const void* from, int col) {
    if constexpr (SHIFT)
      p.load(from, at + col, total - (at + col));
    else
      p.load(from, at + col);
  };
  auto store = [&](const Piece<DT, VEC>& p, void* to, int col) {
    if constexpr (SHIFT)
      p.store(to, at + col, -col, a.d - col);
    else
      p.store(to, at + col);
  };
  Piece<DT, VEC> x[N];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int col = VEC * (n * TPR + t) - ahead;
    if (col < a.d) load(x[n], a.x, col);
  }
  if (a.add) {
    Piece<DT, VEC> y[N];
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int col = VEC * (n * TPR + t) - ahead;
      if (col < a.d) load(y[n], a.add, col);
    }
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int col = VEC * (n * TPR + t) - ahead;
      if (col < a.d) {
        float s[VEC];
#pragma unroll
        for (int k = 0; k < VEC; ++k) s[k] = x[n].get(k) + y[n].get(k);
        x[n].set(s);                               // the stream as it is kept is what is normalised
        store(x[n], a.sum, col);
      }
    }
  }
  float sum[1] = {0.f};
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int col = VEC * (n * TPR + t) - ahead;
    if (col < a.d)
#pragma unroll
      for (int k = 0; k < VEC; ++k) sum[0] += own(col, k) ? x[n].get(k) : 0.f;
  }
  row_sums<TPR>(sum, red);
  const float mean = sum[0] / a.d;
  float square[1] = {0.f};
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int col = VEC * (n * TPR + t) - ahead;
    if (col < a.d)
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        const float c = own(col, k) ? x[n].get(k) - mean : 0.f;
        square[0] = fmaf(c, c, square[0]);
      }
  }
  row_sums<TPR>(square, red);
  const float rstd = 1.f / sqrtf(square[0] / a.d + a.eps);
  if (t == 0) {
    if (a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int col = VEC * (n * TPR + t) - ahead;
    if (col < a.d) {
      float gain[VEC], bias[VEC], y[VEC];
      load_params<VEC, SHIFT>(gain, a.gain, col, a.d, 1.f);
      load_params<VEC, SHIFT>(bias, a.bias, col, a.d, 0.f);
#pragma unroll
      for (int k = 0; k < VEC; ++k) y[k] = fmaf((x[n].get(k) - mean) * rstd, gain[k], bias[k]);
      Piece<DT, VEC> out;
      out.set(y);
      store(out, a.out, col);
    }
  }
}

// Workgroup (chunk, sample): its row groups take rows in turn, the next one's values on their way while one is worked on; gain is in LDS
// (read again for every row, it would be as many bytes out of L2 as the rows themselves).  The gradients of gain and bias stay in the
// registers of the lanes that hold their columns and are then added over the groups through LDS, in their order.  Bound by memory: the
// rows, and the chunks' sums, written and read once more.  4 x 2048 rows of 12288 bf16 values: 166 us with the join, 3.6 TB/s of the rows
// alone (140 us where only dx is asked for); 214 us with loads where they are used and gain out of L2.  16 x 256 rows of 768: 12 us,
// most of it two launches and a wave's two or three turns to memory.  Shifted rows: 2048 x 12289 fp16 81 us, an element at a time 319.
template <int DT, int VEC, int TPR, int P, int THREADS, bool SHIFT>
__global__ void __launch_bounds__(THREADS, THREADS == 1024 || P <= (DT == DP_F32 ? 8 : SHIFT ? 16 : 24) ? 4 : 2)
layer_norm_backward_kernel(const NormArgs a, int first_block) {
  constexpr int N = P / VEC, GROUPS = THREADS / TPR;
  constexpr bool AHEAD = P <= 32;                  // (no registers for it beyond)
  extern __shared__ __align__(16) float lds[];     // gain; then, in the same place, sums over groups
  __shared__ float red[THREADS / 64][2];
  float* const gains = lds + (SHIFT ? VEC : 0);    // (read up to a piece before its first and behind its last)
  const int t = threadIdx.x % TPR, group = threadIdx.x / TPR;
  const unsigned id = first_block + blockIdx.x;
  const int chunk = id % (unsigned)a.chunks, b = id / (unsigned)a.chunks;
  // Rows first + group, + step, ... below end.  With SHIFT a group's rows are all ahead by the same: a multiple of VEC apart.
  const int phases = SHIFT && GROUPS == 1 ? min(VEC, a.T) : 1, step = GROUPS * phases;
  const int first = chunk / phases * a.chunk_rows + chunk % phases, end = min(chunk / phases * a.chunk_rows + a.chunk_rows, a.T);
  const int ahead = SHIFT ? (int)((((int64_t)b * a.T + first + group) * a.d) & (VEC - 1)) : 0;
  const int64_t total = (int64_t)a.B * a.T * a.d;
  auto own = [&](int col, int k) { return !SHIFT || (unsigned)(col + k) < (unsigned)a.d; };
  auto load_piece = [&](Piece<DT, VEC>& p, const void* from, int64_t at) {
    if constexpr (SHIFT)
      p.load(from, at, total - at);
    else
      p.load(from, at);
  };
  struct Row {
    Piece<DT, VEC> x[N], dy[N];
    float mean, rstd;
  };
  auto load = [&](Row& r, int in_sample) {
    const int64_t row = (int64_t)b * a.T + in_sample, at = row * a.d;
    r.mean = a.mean[row];
    r.rstd = a.rstd[row];
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int col = VEC * (n * TPR + t) - ahead;
      if (col < a.d) {
        load_piece(r.x[n], a.x, at + col);
        load_piece(r.dy[n], a.dy, at + col);
      }
    }
  };
  Row row;
  if (first + group < end) load(row, first + group);
  for (int k = threadIdx.x; k < a.d; k += THREADS) gains[k] = a.gain ? a.gain[k] : 1.f;
  if (SHIFT && threadIdx.x < VEC) lds[threadIdx.x] = gains[a.d + threadIdx.x] = 0.f;
  __syncthreads();
  float dgain[N][VEC] = {}, dbias[N][VEC] = {};
  const float width = 1.f / a.d;
  for (int r = first; r < end; r += step) {
    const bool there = GROUPS == 1 || r + group < end;
    Row next;
    if (AHEAD && r + group + step < end) load(next, r + group + step);
    float sums[2] = {0.f, 0.f};
    if (there) {
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const int col = VEC * (n * TPR + t) - ahead;
        if (col < a.d)
#pragma unroll
          for (int k = 0; k < VEC; ++k) {
            const float h = own(col, k) ? (row.x[n].get(k) - row.mean) * row.rstd : 0.f, g = own(col, k) ? row.dy[n].get(k) : 0.f;
            const float u = g * gains[col + k];
            dgain[n][k] = fmaf(g, h, dgain[n][k]);
            dbias[n][k] += g;
            sums[0] += u;
            sums[1] = fmaf(u, h, sums[1]);
          }
      }
    }
    if (a.out) {
      row_sums<TPR>(sums, red);
      const float mean_u = sums[0] * width, mean_uh = sums[1] * width;
      if (there) {
        const int64_t at = ((int64_t)b * a.T + r + group) * a.d;
#pragma unroll
        for (int n = 0; n < N; ++n) {
          const int col = VEC * (n * TPR + t) - ahead;
          if (col < a.d) {
            Piece<DT, VEC> add, out;
            if (a.add) load_piece(add, a.add, at + col);
            float dx[VEC];
#pragma unroll
            for (int k = 0; k < VEC; ++k) {
              const float h = (row.x[n].get(k) - row.mean) * row.rstd, u = row.dy[n].get(k) * gains[col + k];
              dx[k] = (u - mean_u - h * mean_uh) * row.rstd;
              if (a.add) dx[k] += add.get(k);
            }
            out.set(dx);
            if constexpr (SHIFT)
              out.store(a.out, at + col, -col, a.d - col);
            else
              out.store(a.out, at + col);
          }
        }
      }
    }
    if (AHEAD)
      row = next;
    else if (r + group + step < end)
      load(row, r + group + step);
  }
  if (!a.kept) return;
  float* to = a.chunks > 1 ? a.partial + (int64_t)id * 2 * a.d : a.kept + (int64_t)b * 2 * a.d;
  float square[1] = {0.f};
  if constexpr (GROUPS == 1) {
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        const int col = VEC * (n * TPR + t) - ahead + k;
        if (own(col, 0) && col < a.d) {
          to[col] = dgain[n][k];
          to[(int64_t)a.d + col] = dbias[n][k];
          square[0] = fmaf(dgain[n][k], dgain[n][k], fmaf(dbias[n][k], dbias[n][k], square[0]));
        }
      }
  } else if constexpr (SHIFT) {
    // A group's pieces lie `ahead` columns before where its columns are: each group's sums as they lie, and the shift where they are read.
    const int region = (a.d + 2 * VEC - 1) / VEC * VEC;
    for (int half = 0; half < 2; ++half) {
      __syncthreads();
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const int col = VEC * (n * TPR + t);
        if (col < region)
#pragma unroll
          for (int k = 0; k < VEC; ++k) lds[group * region + col + k] = half ? dbias[n][k] : dgain[n][k];
      }
      __syncthreads();
      for (int c = threadIdx.x; c < a.d; c += THREADS) {
        float v = 0.f;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g)
          v += lds[g * region + c + (int)((((int64_t)b * a.T + first + g) * a.d) & (VEC - 1))];
        to[half * a.d + c] = v;
        square[0] = fmaf(v, v, square[0]);
      }
    }
  } else {
    constexpr int SUMS = 2 * VEC * TPR;            // of a group
#pragma unroll
    for (int n = 0; n < N; ++n) {
      __syncthreads();
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        lds[group * SUMS + VEC * t + k] = dgain[n][k];
        lds[group * SUMS + VEC * (TPR + t) + k] = dbias[n][k];
      }
      __syncthreads();
      for (int c = threadIdx.x; c < SUMS; c += THREADS) {
        const int half = c / (VEC * TPR), col = n * VEC * TPR + c % (VEC * TPR);
        if (col < a.d) {
          float v = 0.f;
#pragma unroll
          for (int g = 0; g < GROUPS; ++g) v += lds[g * SUMS + c];
          to[(int64_t)half * a.d + col] = v;
          square[0] = fmaf(v, v, square[0]);
        }
      }
    }
  }
  if (a.chunks == 1) {
    row_sums<THREADS>(square, reinterpret_cast<float(*)[1]>(red));
    if (threadIdx.x == 0) a.sqnorm[b] = square[0];
  }
}

// The sum of a column over chunks c, c + step ..., in their order, eight loads in flight.
__device__ __forceinline__ float add_chunks(const float* p, int c, int step, int chunks, int width) {
  float v = 0.f;
  for (; c + 7 * step < chunks; c += 8 * step) {
    float x[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) x[q] = p[(int64_t)(c + q * step) * width];
#pragma unroll
    for (int q = 0; q < 8; ++q) v += x[q];
  }
  for (; c < chunks; c += step) v += p[(int64_t)c * width];
  return v;
}

// kept[i, k] = the sample's chunks added up; strips of 64 columns, `strips` to a sample, the chunks dealt to 16 waves.  (One sample of 512
// chunks of 8192 values, a thread to a column: 30 us, all latency.)
constexpr int kJoinThreads = 1024;
__global__ void __launch_bounds__(kJoinThreads) layer_norm_join_kernel(const float* __restrict__ partial, int chunks, int width, int strips,
                                                                       int first_block, float* __restrict__ kept) {
  __shared__ float part[kJoinThreads / 64][64];
  const unsigned id = first_block + blockIdx.x, b = id / (unsigned)strips, k = id % (unsigned)strips * 64 + (threadIdx.x & 63);
  const int wave = threadIdx.x >> 6;
  if (k < (unsigned)width)
    part[wave][threadIdx.x & 63] = add_chunks(partial + (int64_t)b * chunks * width + k, wave, kJoinThreads / 64, chunks, width);
  __syncthreads();
  if (wave == 0 && k < (unsigned)width) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kJoinThreads / 64; ++w) v += part[w][threadIdx.x];
    kept[(int64_t)b * width + k] = v;
  }
}

// The same and the squared norm in one launch, a workgroup to a sample, where a sample's chunks are few values.
constexpr int kJoinValues = 1 << 16;
__global__ void __launch_bounds__(kJoinThreads) layer_norm_join_norm_kernel(const float* __restrict__ partial, int chunks, int width,
                                                                            int first_block, float* __restrict__ kept,
                                                                            float* __restrict__ sqnorm) {
  __shared__ float red[kJoinThreads / 64];
  const unsigned b = first_block + blockIdx.x;
  float square = 0.f;
  for (int k = threadIdx.x; k < width; k += kJoinThreads) {
    const float v = add_chunks(partial + (int64_t)b * chunks * width + k, 0, 1, chunks, width);
    kept[(int64_t)b * width + k] = v;
    square = fmaf(v, v, square);
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) square += __shfl_xor(square, off);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = square;
  __syncthreads();
  if (threadIdx.x == 0) {
    float total = 0.f;
#pragma unroll
    for (int w = 0; w < kJoinThreads / 64; ++w) total += red[w];
    sqnorm[b] = total;
  }
}

// Values to a piece, and the values that a row's pieces cover at most.
constexpr int piece_values(int dt) { return dt == DP_F32 ? 4 : 8; }
int covered(dp_dtype dt, int d) { return d % piece_values(dt) == 0 ? d : d + piece_values(dt) - 1; }
constexpr int kWaveWidth = 2048;                   // of rows that a wave takes alone

// Calls f with the form for rows that cover `width` values: threads to a row and values to a thread.
template <int THREADS, bool SHIFT, class F>
dp_status by_width(int width, F f) {
  using std::integral_constant;
  const int per = width <= kWaveWidth ? (width + 63) / 64 : (width + THREADS - 1) / THREADS;
  if (width <= kWaveWidth) {
    const integral_constant<int, 64> tpr{};
    if (per <= 8) return f(tpr, integral_constant<int, 8>{});
    if (THREADS == 1024 || per <= 16) return f(tpr, integral_constant<int, 16>{});
    if constexpr (THREADS == 512) return per <= 24 ? f(tpr, integral_constant<int, 24>{}) : f(tpr, integral_constant<int, 32>{});
  }
  const integral_constant<int, THREADS> tpr{};
  if (per <= 8) return f(tpr, integral_constant<int, 8>{});
  if (THREADS == 1024 || per <= 16) return f(tpr, integral_constant<int, 16>{});
  if constexpr (THREADS == 512) {
    if (per <= 24) return f(tpr, integral_constant<int, 24>{});
    if (per <= 32) return f(tpr, integral_constant<int, 32>{});
    return f(tpr, integral_constant<int, SHIFT ? 72 : 64>{});
  }
  return DP_ERR_UNSUPPORTED;
}

// Calls f with the type and whether rows are shifted.
template <class F>
dp_status by_type(dp_dtype dt, int d, F f) {
  using std::integral_constant;
  auto go = [&](auto type) {
    return d % piece_values(decltype(type)::value) ? f(type, std::true_type{}) : f(type, std::false_type{});
  };
  if (dt == DP_F32) return go(integral_constant<int, DP_F32>{});
  return dt == DP_F16 ? go(integral_constant<int, DP_F16>{}) : go(integral_constant<int, DP_BF16>{});
}

// Threads to a workgroup of the backward pass: 512, of which a compute unit has two, or 1024, one, where a thread's part of a row is at most 32
// bytes (64 of narrow fp32 rows; twice the waves leave it 128 registers) and that brings something: wide rows leave half as many sums to be joined (4 x
// 2048 x 12288 bf16: 166 us, with 512 threads 184), waves that take rows alone have one each where two were (32 x 197 x 768: 12.8 and 16.1; a
// sample of up to 8 rows has none for the other waves: 512 x 1 x 1024, 10.6 and 9.8).  Beyond, 2 x 1000 x 32768: 206 us with 1024, 183.
// Both sides of the lines, us with 512 and 1024 threads.  Wide, 4 x 2048 (fp32: 4 x 1024) rows: bf16 of 4096 54 and 72, 8192 117 and 124, 8200 134 and 136,
// 9216 144 and 139, 10240 153 and 148, 14336 221 and 189, 16384 254 and 207; fp32 of 4096 44 and 51, 4100 58 and 54, 5120 70 and 59, 8192 116 and 102; shifted
// bf16 of 8195 196 and 221, 12289 253 and 251, 16377 306 and 283.  (2 x 300 and 16 x 128 rows: 1024 ahead from 8200 and 4100 on, by up to 15 %.)
// Narrow: bf16 32 x 197 rows of 520 14.1 and 11.5, 1024 17.3 and 13.7, 16 x 256 and 1 x 4096 the same within 3 %; 512 x 4 rows of 768 8.1 and 10.2; fp32 32 x
// 197 of 768 22.2 and 16.5, 1024 26.6 and 20.4, but 16 x 256 of 1024 14.9 and 16.5.  It loses where few rows are shifted in fp32 (16 x 256 of 513: 12.4 and
// 19.1; 32 x 197: 21.1 and 21.2).
int backward_threads(dp_dtype dt, int T, int d) {
  const int width = covered(dt, d), bytes = width * (dt == DP_F32 ? 4 : 2);
  if (width <= 1024) return T > 8 ? 1024 : 512;
  return bytes > 16384 && bytes <= 32768 ? 1024 : 512;
}

}  // namespace

dp_status launch_layer_norm(const NormArgs& a, dp_dtype dt, hipStream_t s) {
  const int64_t rows = (int64_t)a.B * a.T;
  return by_type(dt, a.d, [&](auto type, auto shift) {
    return by_width<kThreads, decltype(shift)::value>(covered(dt, a.d), [&](auto tpr, auto per) {
      constexpr int DT = decltype(type)::value, GROUPS = kThreads / decltype(tpr)::value;
      return launch_in_runs((rows + GROUPS - 1) / GROUPS, [&](dim3 grid, int first) {
        hipLaunchKernelGGL((layer_norm_kernel<DT, piece_values(DT), decltype(tpr)::value, decltype(per)::value, decltype(shift)::value>),
                           grid, dim3(kThreads), 0, s, a, rows, first);
      });
    });
  });
}

namespace {

// How a sample's T rows are dealt to workgroups: chunks of `rows` rows, a whole number of phases (the rows of a chunk that are shifted
// alike make a workgroup where one works on one row at a time).
struct Dealt {
  int chunks, rows;
};
Dealt deal(dp_dtype dt, int B, int T, int d) {
  const int64_t all = (int64_t)B * T;
  const int threads = backward_threads(dt, T, d), units = 262144 / threads;      // 512 threads: two workgroups to a compute unit, 1024: one
  const bool alone = covered(dt, d) <= kWaveWidth;
  const int phases = !alone && d % piece_values(dt) ? std::min(piece_values(dt), T) : 1;
  int64_t per = std::max<int64_t>((all + units - 1) / units, alone ? 16 : 8);         // to a workgroup
  const int64_t strips = std::max<int64_t>(1, (T + per * phases - 1) / (per * phases));
  const int64_t rows = ((T + strips - 1) / strips + phases - 1) / phases * phases;
  return {(int)((T + rows - 1) / rows * phases), (int)rows};
}

}  // namespace

int layer_norm_chunks(dp_dtype dt, int B, int T, int d) { return deal(dt, B, T, d).chunks; }

dp_status launch_layer_norm_backward(NormArgs a, dp_dtype dt, hipStream_t s) {
  const Dealt dealt = deal(dt, a.B, a.T, a.d);
  a.chunks = dealt.chunks;
  a.chunk_rows = dealt.rows;
  dp_status st = by_type(dt, a.d, [&](auto type, auto shift) {
    auto by_threads = [&](auto threads) {
      constexpr int THREADS = decltype(threads)::value;
      return by_width<THREADS, decltype(shift)::value>(covered(dt, a.d), [&](auto tpr, auto per) {
        constexpr int DT = decltype(type)::value, VEC = piece_values(DT), TPR = decltype(tpr)::value, GROUPS = THREADS / TPR;
        constexpr bool SHIFT = decltype(shift)::value;
        auto kernel = layer_norm_backward_kernel<DT, VEC, TPR, decltype(per)::value, THREADS, SHIFT>;
        const int sums = GROUPS == 1 ? 0 : SHIFT ? GROUPS * ((a.d + 2 * VEC - 1) / VEC * VEC) : GROUPS * 2 * VEC * TPR;
        const int lds = 4 * std::max(a.d + (SHIFT ? 2 * VEC : 0), sums);
        static ReadyTable done;
        if (lds > 65536) {
          const dp_status ready = allow_big_lds(kernel, 4 * (kNormMaxWidth + 16), done);
          if (ready != DP_OK) return ready;
        }
        return launch_in_runs((int64_t)a.B * a.chunks, [&](dim3 grid, int first) {
          hipLaunchKernelGGL(kernel, grid, dim3(THREADS), lds, s, a, first);
        });
      });
    };
    return backward_threads(dt, a.T, a.d) == 1024 ? by_threads(std::integral_constant<int, 1024>{})
                                                  : by_threads(std::integral_constant<int, 512>{});
  });
  if (st != DP_OK || !a.kept || a.chunks == 1) return st;
  if ((int64_t)a.chunks * 2 * a.d <= kJoinValues)
    return launch_in_runs(a.B, [&](dim3 grid, int first) {
      hipLaunchKernelGGL(layer_norm_join_norm_kernel, grid, dim3(kJoinThreads), 0, s, a.partial, a.chunks, 2 * a.d, first, a.kept, a.sqnorm);
    });
  const int strips = (2 * a.d + 63) / 64;
  st = launch_in_runs((int64_t)a.B * strips, [&](dim3 grid, int first) {
    hipLaunchKernelGGL(layer_norm_join_kernel, grid, dim3(kJoinThreads), 0, s, a.partial, a.chunks, 2 * a.d, strips, first, a.kept);
  });
  return st != DP_OK ? st : launch_row_sqnorm(a.kept, a.B, 2 * a.d, a.sqnorm, s);
}

}  // namespace dpbk
