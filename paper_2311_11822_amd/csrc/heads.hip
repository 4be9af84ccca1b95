// Heads of queries and keys between their projection and attention: position rotation, alone or behind a norm of each head, and the
// norm's backward pass with its gains' per-sample gradients.
//   y = R(x),  or  y = R(h gain),  h = x r,  r = 1 / sqrt(mean(x^2) + eps);
//   R turns pair i of columns, (x1, x2) -> amplitude (x1 cos - x2 sin, x2 cos + x1 sin), by position * turns[i] whole turns;
//   dy comes back through R' (the angle's sign changed):  g = R'(dy),  u = g gain,  dx = r (u - h mean(u h)),  kept_i = sum_{t, heads} g h.
// Streams over memory: a lane holds the pieces that turn together, so nothing is exchanged but the sums of a norm; a token's angles are
// worked out once, in 64 bits as far as whole turns go, and kept in LDS for all of its heads.
#include <algorithm>

#include "heads.h"
#include "piece.h"

namespace dpbk {

namespace {

constexpr int kThreads = 256;

// Sum over the 2^lanes lanes of a row, in each of them.
__device__ __forceinline__ float lanes_sum(float x, int lanes) {
  for (int n = 0; n < lanes; ++n) x += __shfl_xor(x, 1 << n);
  return x;
}

// Cosine and sine of each pair at the tokens first .. first + n - 1 of sample b.  What counts of an angle is its fraction of a turn:
// taken in 64 bits, it is exact to 2^-33 of a turn at any 32-bit position.
__device__ __forceinline__ void work_out_angles(const HeadsArgs& a, int b, int first, int n, float2* angle) {
  const int half = a.turn / 2;
  for (int k = threadIdx.x; k < n * half; k += kThreads) {
    const int token = k / half, i = k - token * half, t = first + token;
    const double at = a.position ? (double)a.position[(int64_t)b * a.T + t] : (double)t;
    const double turned = at * a.turns[i];
    float sine, cosine;
    sincospif(2.f * (float)(turned - rint(turned)), &sine, &cosine);
    angle[k] = make_float2(cosine * a.amplitude, (a.back ? -sine : sine) * a.amplitude);
  }
}

// Where a lane's values lie.  Unit u of a row is two pieces of VEC columns that turn together: u and u + h of the h pieces of each half, or
// two adjacent ones (interleaved pairs, and columns that do not turn).
template <int VEC>
struct Unit {
  int first, second;                 // columns; a second one at or past D is not there
  bool halves;                       // the two pieces turn with each other
  __device__ __forceinline__ void init(const HeadsArgs& a, int u) {
    const int h = a.interleaved ? 0 : a.turn / 2 / VEC;
    halves = u < h || (VEC == 1 && a.interleaved && 2 * u < a.turn);
    first = VEC * (u < h ? u : 2 * u);
    second = u < h ? first + a.turn / 2 : first + VEC;
  }
  __device__ __forceinline__ void turn(const HeadsArgs& a, const float2* angle, float (&x)[VEC], float (&y)[VEC]) const {
    if (halves) {
      const float2* at = angle + (VEC == 1 && a.interleaved ? first / 2 : first);
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        const float2 w = at[k];
        const float x1 = x[k], x2 = y[k];
        x[k] = x1 * w.x - x2 * w.y;
        y[k] = x2 * w.x + x1 * w.y;
      }
    } else if (VEC > 1 && a.interleaved) {
#pragma unroll
      for (int k = 0; k < VEC; k += 2) {
        if (first + k < a.turn) pair(angle[(first + k) / 2], x[k], x[k + 1 < VEC ? k + 1 : k]);
        if (second + k < a.turn) pair(angle[(second + k) / 2], y[k], y[k + 1 < VEC ? k + 1 : k]);
      }
    }
  }
  __device__ static __forceinline__ void pair(float2 w, float& x1, float& x2) {
    const float before = x1;
    x1 = before * w.x - x2 * w.y;
    x2 = x2 * w.x + before * w.y;
  }
};

template <int DT, int VEC, int KIND>
__global__ void __launch_bounds__(kThreads) heads_kernel(const HeadsArgs a) {
  constexpr int N = VEC == 1 ? 2 : 1;                  // units of a lane: rows are 64 lanes at most
  extern __shared__ __align__(16) float2 angle[];      // then, in the same place, sums over row groups
  const int row_lanes = 1 << a.lanes, t = threadIdx.x & (row_lanes - 1), group = threadIdx.x >> a.lanes, groups = kThreads >> a.lanes;
  const unsigned id = blockIdx.x;
  const int b = id / (unsigned)a.chunks, chunk = id - b * a.chunks, half = a.turn / 2;
  const int length = a.len ? min(max(a.len[b], 0), a.T) : a.T;
  const int begin = min(chunk * a.chunk_tokens, length), end = min(begin + a.chunk_tokens, length);
  Unit<VEC> unit[N];
  bool there[N][2];
  float gain[2][N][2][VEC], sum[2][N][2][VEC];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    unit[n].init(a, t + n * row_lanes);
    there[n][0] = unit[n].first < a.D;
    there[n][1] = there[n][0] && unit[n].second < a.D;
    if constexpr (KIND != kRotate) {
#pragma unroll
      for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
          for (int k = 0; k < VEC; ++k) {
            gain[w][n][p][k] = there[n][p] && a.gain[w] ? a.gain[w][(p ? unit[n].second : unit[n].first) + k] : 1.f;
            sum[w][n][p][k] = 0.f;
          }
    }
  }
  const float width = 1.f / a.D;

  for (int first = begin; first < end; first += a.block_tokens) {
    const int tokens = min(a.block_tokens, end - first);
    if (first > begin) __syncthreads();                // the last ones' angles have been read
    if (half) {
      work_out_angles(a, b, first, tokens, angle);
      __syncthreads();
    }
    auto side = [&](auto w_tag) {
      constexpr int w = decltype(w_tag)::value;
      const int heads = a.heads[w], token_step = groups / max(heads, 1), head_step = groups - token_step * heads;
      if (heads == 0) return;
      int token = group / heads, head = group - token * heads;
      for (; token < tokens; token += token_step, head += head_step) {
        if (head >= heads) {
          head -= heads;
          if (++token >= tokens) break;
        }
        const int64_t in_row = b * a.in_stride[w].sample + (first + token) * a.in_stride[w].token + head * a.in_stride[w].head;
        const int64_t out_row = b * a.out_stride[w].sample + (first + token) * a.out_stride[w].token + head * a.out_stride[w].head;
        const float2* const at = angle + token * half;
        float x[N][2][VEC];
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
          for (int p = 0; p < 2; ++p) {
            Values<DT, VEC> v;
            if (there[n][p]) v.load(a.in[w], in_row + (p ? unit[n].second : unit[n].first));
#pragma unroll
            for (int k = 0; k < VEC; ++k) x[n][p][k] = there[n][p] ? v.get(k) : 0.f;
          }
        float dy[N][2][VEC];
        if constexpr (KIND == kNormGrad) {
          const int64_t row = b * a.dy_stride[w].sample + (first + token) * a.dy_stride[w].token + head * a.dy_stride[w].head;
#pragma unroll
          for (int n = 0; n < N; ++n) {
#pragma unroll
            for (int p = 0; p < 2; ++p) {
              Values<DT, VEC> v;
              if (there[n][p]) v.load(a.dy[w], row + (p ? unit[n].second : unit[n].first));
#pragma unroll
              for (int k = 0; k < VEC; ++k) dy[n][p][k] = there[n][p] ? v.get(k) : 0.f;
            }
            unit[n].turn(a, at, dy[n][0], dy[n][1]);
          }
        }
        float r = 1.f, mean_uh = 0.f;
        if constexpr (KIND != kRotate) {
          float square = 0.f;
#pragma unroll
          for (int n = 0; n < N; ++n)
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
              for (int k = 0; k < VEC; ++k) square = fmaf(x[n][p][k], x[n][p][k], square);
          r = 1.f / sqrtf(lanes_sum(square, a.lanes) * width + a.eps);
        }
        if constexpr (KIND == kNormGrad) {
          float uh = 0.f;
#pragma unroll
          for (int n = 0; n < N; ++n)
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
              for (int k = 0; k < VEC; ++k) {
                const float h = x[n][p][k] * r, u = dy[n][p][k] * gain[w][n][p][k];
                sum[w][n][p][k] = fmaf(dy[n][p][k], h, sum[w][n][p][k]);
                uh = fmaf(u, h, uh);
              }
          mean_uh = lanes_sum(uh, a.lanes) * width;
        }
#pragma unroll
        for (int n = 0; n < N; ++n) {
          if constexpr (KIND == kNorm) {
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
              for (int k = 0; k < VEC; ++k) x[n][p][k] = x[n][p][k] * r * gain[w][n][p][k];
          }
          if constexpr (KIND == kNormGrad) {
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
              for (int k = 0; k < VEC; ++k) x[n][p][k] = r * (dy[n][p][k] * gain[w][n][p][k] - x[n][p][k] * r * mean_uh);
          } else {
            unit[n].turn(a, at, x[n][0], x[n][1]);
          }
#pragma unroll
          for (int p = 0; p < 2; ++p)
            if (there[n][p]) {
              Values<DT, VEC> v;
              v.set(x[n][p]);
              v.store(a.out[w], out_row + (p ? unit[n].second : unit[n].first));
            }
        }
      }
    };
    side(std::integral_constant<int, 0>{});
    side(std::integral_constant<int, 1>{});
  }

  if constexpr (KIND == kNormGrad) {
    if (!a.kept) return;
    // the row groups' sums, one after the other
    float* const red = reinterpret_cast<float*>(angle);                // [groups][D]
    const int sides = a.heads[1] ? 2 : 1;
    float* const to = a.partial + ((int64_t)b * a.chunks + chunk) * sides * a.D;
    auto join = [&](auto w_tag) {
      constexpr int w = decltype(w_tag)::value;
      __syncthreads();
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
          for (int k = 0; k < VEC; ++k)
            if (there[n][p]) red[group * a.D + (p ? unit[n].second : unit[n].first) + k] = sum[w][n][p][k];
      __syncthreads();
      for (int c = threadIdx.x; c < a.D; c += kThreads) {
        float s = 0.f;
        for (int g = 0; g < groups; ++g) s += red[g * a.D + c];
        to[w * a.D + c] = s;
      }
    };
    join(std::integral_constant<int, 0>{});
    if (a.heads[1]) join(std::integral_constant<int, 1>{});
  }
}

// A workgroup to a sample: its chunks' sums, in their order by sixteenths, and the square of all of them.
constexpr int kJoinThreads = 1024, kJoinParts = 16;
__global__ void __launch_bounds__(kJoinThreads) heads_join_kernel(const float* partial, float* kept, float* sqnorm, int chunks, int columns) {
  __shared__ float part[kJoinParts][64], square[kJoinParts];
  const int b = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const float* from = partial + (int64_t)b * chunks * columns;
  float total = 0.f;                                                   // of wave 0's lanes
  for (int c0 = 0; c0 < columns; c0 += 64) {
    const int c = c0 + lane;
    float s = 0.f;
    if (c < columns)
      for (int k = wave; k < chunks; k += kJoinParts) s += from[(int64_t)k * columns + c];
    part[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && c < columns) {
      float v = 0.f;
#pragma unroll
      for (int w = 0; w < kJoinParts; ++w) v += part[w][lane];
      kept[(int64_t)b * columns + c] = v;
      total = fmaf(v, v, total);
    }
    __syncthreads();
  }
  if (wave == 0) {
    for (int off = 32; off > 0; off >>= 1) total += __shfl_xor(total, off);
    if (lane == 0) sqnorm[b] = total;
  }
}

template <int DT, int VEC>
dp_status launch(const HeadsArgs& a, HeadsKind kind, size_t lds, hipStream_t s) {
  const dim3 grid((unsigned)a.B * a.chunks);
  if (kind == kRotate)
    heads_kernel<DT, VEC, kRotate><<<grid, kThreads, lds, s>>>(a);
  else if (kind == kNorm)
    heads_kernel<DT, VEC, kNorm><<<grid, kThreads, lds, s>>>(a);
  else
    heads_kernel<DT, VEC, kNormGrad><<<grid, kThreads, lds, s>>>(a);
  return hip_status(hipGetLastError());
}

}  // namespace

// Accesses of 16 bytes where rows begin at such and the pieces of two halves that turn together do, else the largest that fit: 8, 4 or 2.
void heads_layout(HeadsArgs& a, dp_dtype dt, HeadsKind kind, int& vec) {
  vec = dt == DP_F32 ? 4 : 8;
  const int size = dt == DP_F32 ? 4 : 2;
  int64_t all = a.D | (a.interleaved ? 0 : a.turn / 2);
  for (int w = 0; w < 2; ++w)
    if (a.heads[w]) {
      const HeadStrides* sides[] = {&a.in_stride[w], &a.dy_stride[w], &a.out_stride[w]};
      for (const HeadStrides* st : sides) all |= st->sample | st->token | st->head;
      const void* arrays[] = {a.in[w], a.dy[w], a.out[w]};
      for (const void* p : arrays) all |= (int64_t)(reinterpret_cast<uintptr_t>(p) / size);
    }
  while (vec > 1 && all % vec) vec /= 2;
  const int pieces = (a.D + vec - 1) / vec, units = (pieces + 1) / 2, per_lane = vec == 1 ? 2 : 1;
  a.lanes = 0;
  while ((1 << a.lanes) * per_lane < units) ++a.lanes;
  const int groups = kThreads >> a.lanes, heads = a.heads[0] + a.heads[1];
  // two turns of the workgroup's row groups at least, and no more angles than 16 KiB
  a.block_tokens = std::max(1, std::min({(2 * groups + heads - 1) / heads, 2048 / std::max(1, a.turn / 2), a.T}));
  const int64_t blocks = (int64_t)((a.T + a.block_tokens - 1) / a.block_tokens) * a.B;
  const int64_t most = kind == kNormGrad ? 1024 : 4096;
  a.chunk_tokens = a.block_tokens * (int)((blocks + most - 1) / most);
  a.chunks = (a.T + a.chunk_tokens - 1) / a.chunk_tokens;
}

dp_status launch_heads(HeadsArgs a, dp_dtype dt, HeadsKind kind, hipStream_t s) {
  int vec;
  heads_layout(a, dt, kind, vec);
  size_t lds = (size_t)a.block_tokens * (a.turn / 2) * sizeof(float2);
  if (kind == kNormGrad && a.kept) lds = std::max(lds, (size_t)(kThreads >> a.lanes) * a.D * sizeof(float));
  dp_status st;
#define DP_LAUNCH(DT, VEC) \
  if (dt == DT && vec == VEC) st = launch<DT, VEC>(a, kind, lds, s);
  DP_LAUNCH(DP_F32, 4)
  else DP_LAUNCH(DP_F32, 2)
  else DP_LAUNCH(DP_F32, 1)
  else DP_LAUNCH(DP_BF16, 8)
  else DP_LAUNCH(DP_BF16, 4)
  else DP_LAUNCH(DP_BF16, 2)
  else DP_LAUNCH(DP_BF16, 1)
  else DP_LAUNCH(DP_F16, 8)
  else DP_LAUNCH(DP_F16, 4)
  else DP_LAUNCH(DP_F16, 2)
  else DP_LAUNCH(DP_F16, 1)
  else return DP_ERR_UNSUPPORTED;
#undef DP_LAUNCH
  if (st != DP_OK || kind != kNormGrad || !a.kept) return st;
  heads_join_kernel<<<dim3(a.B), kJoinThreads, 0, s>>>(a.partial, a.kept, a.sqnorm, a.chunks, (a.heads[1] ? 2 : 1) * a.D);
  return hip_status(hipGetLastError());
}

}  // namespace dpbk
