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

// P values a thread as VEC-wide pieces: piece n of thread t holds columns VEC (n TPR + t) ...
template <int DT, int VEC>
struct Piece {                                     // VEC values as stored
  static constexpr int WORDS = DT == DP_F32 ? VEC : (VEC + 1) / 2;
  uint32_t w[WORDS];
  __device__ __forceinline__ void load(const void* base, int64_t at) {
    if constexpr (DT != DP_F32 && VEC == 1) {
      w[0] = static_cast<const uint16_t*>(base)[at];
    } else if constexpr (WORDS == 1) {
      w[0] = static_cast<const uint32_t*>(base)[at];
    } else {
      const uint4 v = *reinterpret_cast<const uint4*>(static_cast<const char*>(base) + at * (DT == DP_F32 ? 4 : 2));
      w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
    }
  }
  __device__ __forceinline__ void store(void* base, int64_t at) const {
    if constexpr (DT != DP_F32 && VEC == 1) {
      static_cast<uint16_t*>(base)[at] = (uint16_t)w[0];
    } else if constexpr (WORDS == 1) {
      static_cast<uint32_t*>(base)[at] = w[0];
    } else {
      *reinterpret_cast<uint4*>(static_cast<char*>(base) + at * (DT == DP_F32 ? 4 : 2)) = make_uint4(w[0], w[1], w[2], w[3]);
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
        const float lo = x[2 * k], hi = VEC == 1 ? 0.f : x[(2 * k + 1) % VEC];
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

template <int VEC>
__device__ __forceinline__ void load_params(float (&v)[VEC], const float* p, int col, float none) {
#pragma unroll
  for (int k = 0; k < VEC; ++k) v[k] = p ? p[col + k] : none;
}

template <int DT, int VEC, int TPR, int P>
__global__ void __launch_bounds__(kThreads) layer_norm_kernel(const NormArgs a, int64_t rows, int first_block) {
  constexpr int N = P / VEC, GROUPS = kThreads / TPR;
  __shared__ float red[kThreads / 64][1];
  const int t = threadIdx.x % TPR;
  const int64_t row = ((int64_t)first_block + blockIdx.x) * GROUPS + threadIdx.x / TPR;
  if (TPR == 64 && row >= rows) return;            // (a whole workgroup's row otherwise: always there)
  const int64_t at = row * a.d;
  Piece<DT, VEC> x[N];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int col = VEC * (n * TPR + t);
    if (col < a.d) x[n].load(a.x, at + col);
  }
  if (a.add) {
    Piece<DT, VEC> y[N];
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int col = VEC * (n * TPR + t);
      if (col < a.d) y[n].load(a.add, at + col);
    }
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int col = VEC * (n * TPR + t);
      if (col < a.d) {
        float s[VEC];
#pragma unroll
        for (int k = 0; k < VEC; ++k) s[k] = x[n].get(k) + y[n].get(k);
        x[n].set(s);                               // the stream as it is kept is what is normalised
        x[n].store(a.sum, at + col);
      }
    }
  }
  float sum[1] = {0.f};
#pragma unroll
  for (int n = 0; n < N; ++n)
    if (VEC * (n * TPR + t) < a.d)
#pragma unroll
      for (int k = 0; k < VEC; ++k) sum[0] += x[n].get(k);
  row_sums<TPR>(sum, red);
  const float mean = sum[0] / a.d;
  float square[1] = {0.f};
#pragma unroll
  for (int n = 0; n < N; ++n)
    if (VEC * (n * TPR + t) < a.d)
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        const float c = x[n].get(k) - mean;
        square[0] = fmaf(c, c, square[0]);
      }
  row_sums<TPR>(square, red);
  const float rstd = 1.f / sqrtf(square[0] / a.d + a.eps);
  if (t == 0) {
    if (a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int col = VEC * (n * TPR + t);
    if (col < a.d) {
      float gain[VEC], bias[VEC], y[VEC];
      load_params<VEC>(gain, a.gain, col, 1.f);
      load_params<VEC>(bias, a.bias, col, 0.f);
#pragma unroll
      for (int k = 0; k < VEC; ++k) y[k] = fmaf((x[n].get(k) - mean) * rstd, gain[k], bias[k]);
      Piece<DT, VEC> out;
      out.set(y);
      out.store(a.out, at + col);
    }
  }
}

// Workgroup (chunk, sample): its row groups take rows in turn, the next one's values on their way while one is worked on; gain is in LDS
// (read again for every row, it would be as many bytes out of L2 as the rows themselves).  The gradients of gain and bias are then
// added over the groups through LDS, in their order.  4 x 2048 rows of 12288 bf16 values: 214 us with loads where they are used and
// gain out of L2.
template <int DT, int VEC, int TPR, int P>
__global__ void __launch_bounds__(kThreads, P <= (DT == DP_F32 ? 8 : VEC > 1 ? 24 : 0) ? 4 : 2) layer_norm_backward_kernel(const NormArgs a, int first_block) {
  constexpr int N = P / VEC, GROUPS = kThreads / TPR;
  constexpr bool AHEAD = P <= 32;                  // (no registers for it beyond)
  extern __shared__ __align__(16) float gains[];   // then, in the same place, the groups' sums
  __shared__ float red[kThreads / 64][2];
  const int t = threadIdx.x % TPR, group = threadIdx.x / TPR;
  const unsigned id = first_block + blockIdx.x;
  const int chunk = id % (unsigned)a.chunks, b = id / (unsigned)a.chunks;
  const int first = chunk * a.chunk_rows, end = min(first + a.chunk_rows, a.T);
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
      const int col = VEC * (n * TPR + t);
      if (col < a.d) {
        r.x[n].load(a.x, at + col);
        r.dy[n].load(a.dy, at + col);
      }
    }
  };
  Row row;
  if (first + group < end) load(row, first + group);
  for (int k = threadIdx.x; k < a.d; k += kThreads) gains[k] = a.gain ? a.gain[k] : 1.f;
  __syncthreads();
  float dgain[N][VEC] = {}, dbias[N][VEC] = {};
  const float width = 1.f / a.d;
  for (int r = first; r < end; r += GROUPS) {
    const bool there = GROUPS == 1 || r + group < end;
    Row next;
    if (AHEAD && r + group + GROUPS < end) load(next, r + group + GROUPS);
    float sums[2] = {0.f, 0.f};
    if (there) {
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const int col = VEC * (n * TPR + t);
        if (col < a.d)
#pragma unroll
          for (int k = 0; k < VEC; ++k) {
            const float h = (row.x[n].get(k) - row.mean) * row.rstd, g = row.dy[n].get(k), u = g * gains[col + k];
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
          const int col = VEC * (n * TPR + t);
          if (col < a.d) {
            Piece<DT, VEC> add, out;
            if (a.add) add.load(a.add, at + col);
            float dx[VEC];
#pragma unroll
            for (int k = 0; k < VEC; ++k) {
              const float h = (row.x[n].get(k) - row.mean) * row.rstd, u = row.dy[n].get(k) * gains[col + k];
              dx[k] = (u - mean_u - h * mean_uh) * row.rstd;
              if (a.add) dx[k] += add.get(k);
            }
            out.set(dx);
            out.store(a.out, at + col);
          }
        }
      }
    }
    if (AHEAD)
      row = next;
    else if (r + group + GROUPS < end)
      load(row, r + group + GROUPS);
  }
  if (!a.kept) return;
  float* to = a.chunks > 1 ? a.partial + (int64_t)id * 2 * a.d : a.kept + (int64_t)b * 2 * a.d;
  float square[1] = {0.f};
#pragma unroll
  for (int n = 0; n < N; ++n) {
    if constexpr (GROUPS > 1) {
      constexpr int SUMS = 2 * VEC * TPR;          // of a group
      __syncthreads();
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        gains[group * SUMS + VEC * t + k] = dgain[n][k];
        gains[group * SUMS + VEC * (TPR + t) + k] = dbias[n][k];
      }
      __syncthreads();
      for (int c = threadIdx.x; c < SUMS; c += kThreads) {
        const int half = c / (VEC * TPR), col = n * VEC * TPR + c % (VEC * TPR);
        if (col < a.d) {
          float v = 0.f;
#pragma unroll
          for (int g = 0; g < GROUPS; ++g) v += gains[g * SUMS + c];
          to[(int64_t)half * a.d + col] = v;
          square[0] = fmaf(v, v, square[0]);
        }
      }
    } else {
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        const int col = VEC * (n * TPR + t) + k;
        if (col < a.d) {
          to[col] = dgain[n][k];
          to[(int64_t)a.d + col] = dbias[n][k];
          square[0] = fmaf(dgain[n][k], dgain[n][k], fmaf(dbias[n][k], dbias[n][k], square[0]));
        }
      }
    }
  }
  if (a.chunks == 1) {
    row_sums<kThreads>(square, reinterpret_cast<float(*)[1]>(red));
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

// Calls f with the form for rows of width d: threads to a row and values to a thread.
template <class F>
dp_status by_width(int d, F f) {
  using std::integral_constant;
  const int per = d <= 2048 ? (d + 63) / 64 : (d + kThreads - 1) / kThreads;
  auto go = [&](auto tpr) {
    if (per <= 8) return f(tpr, integral_constant<int, 8>{});
    if (per <= 16) return f(tpr, integral_constant<int, 16>{});
    if (per <= 24) return f(tpr, integral_constant<int, 24>{});
    return f(tpr, integral_constant<int, 32>{});
  };
  if (d <= 2048) return go(integral_constant<int, 64>{});
  if (per <= 32) return go(integral_constant<int, kThreads>{});
  return f(integral_constant<int, kThreads>{}, integral_constant<int, 64>{});
}

template <class F>
dp_status by_type(dp_dtype dt, int d, F f) {
  using std::integral_constant;
  if (dt == DP_F32) {
    if (d % 4 == 0) return f(integral_constant<int, DP_F32>{}, integral_constant<int, 4>{});
    return f(integral_constant<int, DP_F32>{}, integral_constant<int, 1>{});
  }
  const bool whole = d % 8 == 0;
  if (dt == DP_F16) {
    if (whole) return f(integral_constant<int, DP_F16>{}, integral_constant<int, 8>{});
    return f(integral_constant<int, DP_F16>{}, integral_constant<int, 1>{});
  }
  if (whole) return f(integral_constant<int, DP_BF16>{}, integral_constant<int, 8>{});
  return f(integral_constant<int, DP_BF16>{}, integral_constant<int, 1>{});
}

}  // namespace

dp_status launch_layer_norm(const NormArgs& a, dp_dtype dt, hipStream_t s) {
  const int64_t rows = (int64_t)a.B * a.T;
  return by_type(dt, a.d, [&](auto type, auto vec) {
    return by_width(a.d, [&](auto tpr, auto per) {
      constexpr int GROUPS = kThreads / decltype(tpr)::value;
      return launch_in_runs((rows + GROUPS - 1) / GROUPS, [&](dim3 grid, int first) {
        hipLaunchKernelGGL((layer_norm_kernel<decltype(type)::value, decltype(vec)::value, decltype(tpr)::value, decltype(per)::value>),
                           grid, dim3(kThreads), 0, s, a, rows, first);
      });
    });
  });
}

int layer_norm_chunks(dp_dtype, int B, int T, int d) {
  const int64_t rows = (int64_t)B * T;
  const int groups = d <= 2048 ? kThreads / 64 : 1;
  int64_t per = (rows + 511) / 512;                // two workgroups to a compute unit
  per = per < 2 * groups ? 2 * groups : per;
  per = per < 16 ? 16 : per;
  return (int)((T + per - 1) / per);
}

dp_status launch_layer_norm_backward(NormArgs a, dp_dtype dt, hipStream_t s) {
  a.chunks = layer_norm_chunks(dt, a.B, a.T, a.d);
  a.chunk_rows = (a.T + a.chunks - 1) / a.chunks;
  dp_status st = by_type(dt, a.d, [&](auto type, auto vec) {
    return by_width(a.d, [&](auto tpr, auto per) {
      constexpr int VEC = decltype(vec)::value, TPR = decltype(tpr)::value, GROUPS = kThreads / TPR;
      auto kernel = layer_norm_backward_kernel<decltype(type)::value, VEC, TPR, decltype(per)::value>;
      const int lds = 4 * std::max(a.d, GROUPS > 1 ? GROUPS * 2 * VEC * TPR : 0);
      static ReadyTable done;
      if (lds > 65536) {
        const dp_status ready = allow_big_lds(kernel, 4 * kNormMaxWidth, done);
        if (ready != DP_OK) return ready;
      }
      return launch_in_runs((int64_t)a.B * a.chunks, [&](dim3 grid, int first) {
        hipLaunchKernelGGL(kernel, grid, dim3(kThreads), lds, s, a, first);
      });
    });
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
