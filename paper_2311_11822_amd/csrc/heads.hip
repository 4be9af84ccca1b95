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

// Sum over the 2^lanes lanes of a row, in each of them; up to sixteen without LDS: within four lanes, then eights and sixteens turned around.
template <int CONTROL>
__device__ __forceinline__ float lane_of(float x) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), CONTROL, 0xF, 0xF, true));
}
__device__ __forceinline__ float lanes_sum(float x, int lanes) {
  if (lanes > 0) x += lane_of<0xB1>(x);                // quad_perm 1 0 3 2
  if (lanes > 1) x += lane_of<0x4E>(x);                // quad_perm 2 3 0 1
  if (lanes > 2) x += lane_of<0x141>(x);               // row_half_mirror
  if (lanes > 3) x += lane_of<0x140>(x);               // row_mirror
  if (lanes > 4) x += __shfl_xor(x, 16);
  if (lanes > 5) x += __shfl_xor(x, 32);
  return x;
}

// Within one unit in the last place; the instruction itself takes subnormal numbers (eps of zero) for zeros.
__device__ __forceinline__ float inverse_root(float x) {
  const bool low = x < 0x1p-126f;
  return __builtin_amdgcn_rsqf(low ? x * 0x1p64f : x) * (low ? 0x1p32f : 1.f);
}

// Cosine and sine of each pair at the tokens first .. first + n - 1 of sample b.  What counts of an angle is its fraction of a turn.  Whole
// turns come off the exact product of position and turns, so the fraction is right to 2^-54 of a turn at any 32-bit position (off the product's
// nearest 64-bit number: to 2^-25 near 2^31).  Its nearest fp32 number goes to the library's functions, and what that leaves, up to 2^-26 of a turn,
// turns their results by the small angle it is: 1.1e-7 of error without, a few units in the last place of either with it.
__device__ __forceinline__ void work_out_angles(const HeadsArgs& a, int b, int first, int n, float2* angle) {
  const int half = a.turn / 2;
  for (int k = threadIdx.x; k < n * half; k += kThreads) {
    const int token = k / half, i = k - token * half, t = first + token;
    const double at = a.position ? (double)a.position[(int64_t)b * a.T + t] : (double)t;
    const double per = a.turns[i], part = fma(at, per, -rint(at * per));
    const float near = (float)part, rest = 6.28318530717958647692f * (float)(part - (double)near);
    float s, c;
    sincospif(2.f * near, &s, &c);
    const float sine = fmaf(c, rest, s), cosine = fmaf(-s, rest, c);
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

// A workgroup has one side (queries or keys) of a run of tokens; its row groups take rows in turn, the next one's values on their way while
// one is worked on.  Bound by memory: gradients of 32760 tokens of 16 + 4 heads of 128 (335 MB) 71 us; a norm's backward pass of 4 x 2048 tokens of
// 96 + 96 heads of 128 (1.2 GB) 248 us, 4.9 TB/s.  (Both sides' heads of a token in one workgroup: 419 us there, rows of two widths left
// lanes idle.)
template <int DT, int VEC, int KIND>
__global__ void __launch_bounds__(kThreads) heads_kernel(const HeadsArgs a) {
  constexpr int N = VEC == 1 ? 2 : 1;                  // units of a lane: rows are 64 lanes at most
  constexpr bool GRAD = KIND == kNormGrad;
  extern __shared__ __align__(16) float2 angle[];      // then, in the same place, sums over row groups
  const int row_lanes = 1 << a.lanes, t = threadIdx.x & (row_lanes - 1), group = threadIdx.x >> a.lanes, groups = kThreads >> a.lanes;
  const int w = blockIdx.x >= a.begin;
  const HeadsPlan plan = a.plan[w];
  const unsigned id = blockIdx.x - (w ? a.begin : 0);
  const int b = id / (unsigned)plan.chunks, chunk = id - b * plan.chunks, half = a.turn / 2, heads = a.heads[w];
  const int length = a.len ? min(max(a.len[b], 0), a.T) : a.T;
  const int begin = min(chunk * plan.chunk_tokens, length), end = begin + min(plan.chunk_tokens, length - begin);      // (up to 2^31 - 1)
  const HeadStrides in_stride = a.in_stride[w], out_stride = a.out_stride[w], dy_stride = a.dy_stride[w];
  Unit<VEC> unit[N];
  bool there[N][2];
  float gain[N][2][VEC], sum[N][2][VEC];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    unit[n].init(a, t + n * row_lanes);
    there[n][0] = unit[n].first < a.D;
    there[n][1] = there[n][0] && unit[n].second < a.D;
    if constexpr (KIND != kRotate) {
#pragma unroll
      for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
          gain[n][p][k] = there[n][p] && a.gain[w] ? a.gain[w][(p ? unit[n].second : unit[n].first) + k] : 1.f;
          sum[n][p][k] = 0.f;
        }
    }
  }
  const float width = 1.f / a.D;
  const int token_step = groups / heads, head_step = groups - token_step * heads;
  struct Row {                                         // as stored
    Values<DT, VEC> x[N][2], dy[GRAD ? N : 1][2];
  };
  const void *const in = a.in[w], *const dy_in = a.dy[w];
  // Where a row lies, and from one of a group's rows to the next: a step, or one past the last head.
  struct Place {
    int64_t at, step, wrapped;
    __device__ __forceinline__ void init(const HeadStrides& st, int b, int token, int head, int token_step, int head_step, int heads) {
      at = b * st.sample + token * st.token + head * st.head;
      step = token_step * st.token + head_step * st.head;
      wrapped = step + st.token - heads * st.head;
    }
    __device__ __forceinline__ void next(bool wrap) { at += wrap ? wrapped : step; }
  };
  auto load = [&](Row& row, int64_t at, int64_t dy_at) {
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int p = 0; p < 2; ++p)
        if (there[n][p]) {
          row.x[n][p].load(in, at + (p ? unit[n].second : unit[n].first));
          if constexpr (GRAD) row.dy[n][p].load(dy_in, dy_at + (p ? unit[n].second : unit[n].first));
        }
  };

  for (int done = 0; done < end - begin; done += plan.block_tokens) {
    const int first = begin + done, tokens = min(plan.block_tokens, end - first);
    int token = group / heads, head = group - token * heads;
    Place x_at, dy_at, out_at;
    x_at.init(in_stride, b, first + token, head, token_step, head_step, heads);
    dy_at.init(dy_stride, b, first + token, head, token_step, head_step, heads);
    out_at.init(out_stride, b, first + token, head, token_step, head_step, heads);
    Row row;
    if (token < tokens) load(row, x_at.at, dy_at.at);
    if (half) {
      if (done > 0) __syncthreads();              // the last ones' angles have been read
      work_out_angles(a, b, first, tokens, angle);
      __syncthreads();
    }
    while (token < tokens) {
      const bool wrap = head + head_step >= heads;
      const int next_token = token + token_step + wrap, next_head = head + head_step - (wrap ? heads : 0);
      x_at.next(wrap);
      dy_at.next(wrap);
      Row next;
      if (next_token < tokens) load(next, x_at.at, dy_at.at);
      const float2* const at = angle + token * half;
      float x[N][2][VEC], dy[N][2][VEC];
#pragma unroll
      for (int n = 0; n < N; ++n) {
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
          for (int k = 0; k < VEC; ++k) {
            x[n][p][k] = there[n][p] ? row.x[n][p].get(k) : 0.f;
            if constexpr (GRAD) dy[n][p][k] = there[n][p] ? row.dy[n][p].get(k) : 0.f;
          }
        if constexpr (GRAD) unit[n].turn(a, at, dy[n][0], dy[n][1]);
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
        r = inverse_root(lanes_sum(square, a.lanes) * width + a.eps);
      }
      if constexpr (GRAD) {
        float uh = 0.f;
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
          for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int k = 0; k < VEC; ++k) {
              x[n][p][k] *= r;
              sum[n][p][k] = fmaf(dy[n][p][k], x[n][p][k], sum[n][p][k]);
              dy[n][p][k] *= gain[n][p][k];
              uh = fmaf(dy[n][p][k], x[n][p][k], uh);
            }
        mean_uh = lanes_sum(uh, a.lanes) * width;
      }
#pragma unroll
      for (int n = 0; n < N; ++n) {
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
          for (int k = 0; k < VEC; ++k) {
            if constexpr (KIND == kNorm) x[n][p][k] = x[n][p][k] * r * gain[n][p][k];
            if constexpr (GRAD) x[n][p][k] = r * (dy[n][p][k] - x[n][p][k] * mean_uh);
          }
        if constexpr (!GRAD) unit[n].turn(a, at, x[n][0], x[n][1]);
#pragma unroll
        for (int p = 0; p < 2; ++p)
          if (there[n][p]) {
            Values<DT, VEC> v;
            v.set(x[n][p]);
            v.store(a.out[w], out_at.at + (p ? unit[n].second : unit[n].first));
          }
      }
      out_at.next(wrap);
      row = next;
      token = next_token;
      head = next_head;
    }
  }

  if constexpr (GRAD) {
    if (!a.kept) return;
    // the row groups' sums, one after the other
    float* const red = reinterpret_cast<float*>(angle);                // [groups][D]
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int k = 0; k < VEC; ++k)
          if (there[n][p]) red[group * a.D + (p ? unit[n].second : unit[n].first) + k] = sum[n][p][k];
    __syncthreads();
    float* const to = a.partial + (w ? (int64_t)a.B * a.plan[0].chunks * a.D : 0) + (int64_t)id * a.D;
    for (int c = threadIdx.x; c < a.D; c += kThreads) {
      float s = 0.f;
      for (int g = 0; g < groups; ++g) s += red[g * a.D + c];
      to[c] = s;
    }
  }
}

// A workgroup to a sample: its chunks' sums, VEC columns to a thread, by parts that are added in their order, and the square of all of them.
// 94 chunks of 2 x 128 columns of each of four samples 5 us, 1024 of one sample 7 (one column to a thread 11).
constexpr int kJoinThreads = 1024, kJoinParts = 32;
template <int VEC>
__global__ void __launch_bounds__(kJoinThreads) heads_join_kernel(const HeadsArgs a) {
  __shared__ __align__(16) float part[kJoinThreads * VEC];
  __shared__ float square[kJoinThreads / 64];
  const int b = blockIdx.x, sides = a.heads[1] ? 2 : 1, columns = sides * a.D, units = columns / VEC;           // up to 512 columns
  const int parts = min(kJoinThreads / units, kJoinParts), p = threadIdx.x / units, c = (threadIdx.x - p * units) * VEC, w = c >= a.D;
  const HeadsPlan plan = a.plan[w];
  typedef __attribute__((ext_vector_type(VEC))) float Columns;
  Columns s = {};
  if (p < parts) {
    const float* from = a.partial + (w ? (int64_t)a.B * a.plan[0].chunks * a.D : 0) + (int64_t)b * plan.chunks * a.D + (c - w * a.D);
#pragma unroll 8
    for (int k = p; k < plan.chunks; k += parts) s += *reinterpret_cast<const Columns*>(from + (int64_t)k * a.D);
    *reinterpret_cast<Columns*>(part + p * columns + c) = s;
  }
  __syncthreads();
  float v = 0.f;
  if (threadIdx.x < columns) {
#pragma unroll 8
    for (int k = 0; k < parts; ++k) v += part[k * columns + threadIdx.x];
    a.kept[(int64_t)b * columns + threadIdx.x] = v;
  }
  v *= v;
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
  if ((threadIdx.x & 63) == 0) square[threadIdx.x >> 6] = v;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int k = 1; k < kJoinThreads / 64; ++k) v += square[k];
    a.sqnorm[b] = v;
  }
}

// Accesses of 16 bytes where rows begin at such and the pieces of two halves that turn together do, else the largest that fit: 8, 4 or 2.
int access_width(const HeadsArgs& a, dp_dtype dt) {
  int vec = dt == DP_F32 ? 4 : 8;
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
  return vec;
}

// A side's tokens by workgroup: of a block's rows as few as can be leave row groups idle in their last turn (of two at least), no more angles
// than 16 KiB, and no more workgroups than `most` and one to a sample.
HeadsPlan plan_side(const HeadsArgs& a, int w, int most) {
  const int groups = kThreads >> a.lanes, heads = a.heads[w];
  const int turns = (int64_t)a.B * a.T * heads >= (int64_t)2048 * groups ? 2 : 1;          // (few rows: all of them on their way at once)
  const int least = std::max(1, std::min((turns * groups + heads - 1) / heads, a.T)), limit = std::max(1, std::min(2048 / std::max(1, a.turn / 2), a.T));
  HeadsPlan plan = {};
  double best = -1.;
  for (int tokens = std::min(least, limit); tokens <= std::min(limit, 4 * least); ++tokens) {
    const int64_t rows = (int64_t)tokens * heads, taken = (rows + groups - 1) / groups;
    const double filled = (double)rows / (double)(taken * groups);
    if (filled > best + (turns == 1 ? 0.2 : 0.02)) {
      best = filled;
      plan.block_tokens = tokens;
    }
  }
  // (in 64 bits: tokens are up to 2^31 - 1)
  const int64_t blocks = ((int64_t)a.T + plan.block_tokens - 1) / plan.block_tokens * a.B;
  plan.chunk_tokens = (int)std::min<int64_t>(plan.block_tokens * ((blocks + most - 1) / most), a.T);
  plan.chunks = (int)(((int64_t)a.T + plan.chunk_tokens - 1) / plan.chunk_tokens);
  return plan;
}

template <int DT, int VEC>
dp_status launch(const HeadsArgs& a, HeadsKind kind, unsigned blocks, size_t lds, hipStream_t s) {
  if (kind == kRotate)
    heads_kernel<DT, VEC, kRotate><<<dim3(blocks), kThreads, lds, s>>>(a);
  else if (kind == kNorm)
    heads_kernel<DT, VEC, kNorm><<<dim3(blocks), kThreads, lds, s>>>(a);
  else
    heads_kernel<DT, VEC, kNormGrad><<<dim3(blocks), kThreads, lds, s>>>(a);
  return hip_status(hipGetLastError());
}

}  // namespace

dp_status launch_heads(HeadsArgs a, dp_dtype dt, HeadsKind kind, hipStream_t s) {
  const int vec = access_width(a, dt);
  const int pieces = (a.D + vec - 1) / vec, units = (pieces + 1) / 2, per_lane = vec == 1 ? 2 : 1;
  while ((1 << a.lanes) * per_lane < units) ++a.lanes;
  int tokens = 0;
  unsigned blocks = 0;
  for (int w = 0; w < 2; ++w) {
    if (w == 1) a.begin = blocks;
    if (!a.heads[w]) continue;
    // A norm's backward pass: pieces of eight values leave registers for three workgroups to a compute unit: one round of those, but for a side of half as many
    // heads as the other, whose small chunks fill in.  Each side up to 768 workgroups and both together, us: 16 x 256 tokens, 12 + 12 heads of 64 16.0, 14.3;
    // 8 x 512, 20 + 20 19.5, 17.9; 1 x 4096, 16 + 4 of 128 17.6, 19.1; pieces of four, 7 x 991, 2 + 2 of 152 15.3, 16.4.
    const int others = a.heads[1 - w];
    const bool apart = vec < 8 || 2 * a.heads[w] <= others;
    const int share = apart ? kHeadsGradChunks : (int)((int64_t)kHeadsGradChunks * a.heads[w] / (a.heads[w] + others)) + 1;
    a.plan[w] = plan_side(a, w, kind == kNormGrad ? share : kHeadsChunks);
    blocks += (unsigned)(a.B * a.plan[w].chunks);
    tokens = std::max(tokens, a.plan[w].block_tokens);
  }
  size_t lds = (size_t)tokens * (a.turn / 2) * sizeof(float2);
  if (kind == kNormGrad && a.kept) lds = std::max(lds, (size_t)(kThreads >> a.lanes) * a.D * sizeof(float));
  dp_status st;
#define DP_LAUNCH(DT, VEC) \
  if (dt == DT && vec == VEC) st = launch<DT, VEC>(a, kind, blocks, lds, s);
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
  if (a.D % 4 == 0)
    heads_join_kernel<4><<<dim3(a.B), kJoinThreads, 0, s>>>(a);
  else
    heads_join_kernel<1><<<dim3(a.B), kJoinThreads, 0, s>>>(a);
  return hip_status(hipGetLastError());
}

}  // namespace dpbk
