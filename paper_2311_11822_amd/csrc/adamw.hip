// One AdamW step over many tensors (decoupled weight decay):
//   m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2,  g = grad_scale * grad,
//   w = w (1 - lr decay) - lr (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps).
// A stream over memory: 28 bytes an element with 32-bit states and gradients, 16 with 8-bit states.  A stack of 85 million parameters, 32 bits
// and a bf16 copy, in two launches: 500 us, 5.1 TB/s, what a copy reaches.  226 million with 8-bit states: 784 to 840 us by card and run, 4.3 to 4.6 TB/s,
// some 130 vector instructions an element beside it.
//
// 8-bit states are e4m3 numbers in units of their block's largest / 448, m itself and the root of v (whose range they cover where
// they would not that of v).  Rounding to nearest would lose the small steps of a slow average, so values are rounded up where
// their rest is above one minus a dither, which is spread evenly over an element's steps (and a step's elements): fractional
// parts of multiples of sqrt(2) - 1 and of the golden ratio, in 32-bit integers.  The root's rest is taken between the squares of its
// neighbours, so that v is rounded without a bias (between the roots themselves v came out 3.5 % too large after 2000 steps with beta2 =
// 0.999).  A value above zero is not rounded to zero: m / sqrt(v) stays bounded.
//
// Every operation is rounded on its own, none fused: what is computed is defined to the bit (a code at the edge of its dither does not
// depend on how a compiler fuses, and plain fp32 code elsewhere reproduces a step).
#include <type_traits>

#include "train.h"

#pragma clang fp contract(off)

namespace dpbk {

namespace {

typedef __attribute__((ext_vector_type(2))) float f32x2v;
constexpr int kThreads = 256, kBlocks = 4;         // blocks of 256 values that a wave has in flight
static_assert(kThreads / 64 * kBlocks * kAdamScaleBlock == kAdamChunk, "a workgroup's values");

template <int DT>
__device__ __forceinline__ float load_grad(const void* g, uint64_t at) {
  if constexpr (DT == DP_F32) return static_cast<const float*>(g)[at];
  const uint16_t w = static_cast<const uint16_t*>(g)[at];
  if constexpr (DT == DP_BF16) return __uint_as_float((uint32_t)w << 16);
  return (float)__builtin_bit_cast(_Float16, w);
}

template <int DT>
__device__ __forceinline__ uint16_t to_half(float x) {
  if constexpr (DT == DP_BF16) return __builtin_bit_cast(uint16_t, (__bf16)x);
  return __builtin_bit_cast(uint16_t, (_Float16)x);
}

// Four values of one block in a thread: neighbours (VEC), or 64 apart.
template <bool VEC>
__device__ __forceinline__ int element(int lane, int i) {
  return VEC ? 4 * lane + i : lane + 64 * i;
}

template <bool VEC>
__device__ __forceinline__ void load4(float (&x)[4], const float* p, uint64_t at, int lane, int64_t left) {
  if (VEC && left >= kAdamScaleBlock) {
    const f32x4 v = *reinterpret_cast<const f32x4*>(p + at + 4 * lane);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = v[i];
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = element<VEC>(lane, i) < left ? p[at + element<VEC>(lane, i)] : 0.f;
  }
}

template <bool VEC>
__device__ __forceinline__ void store4(const float (&x)[4], float* p, uint64_t at, int lane, int64_t left) {
  if (VEC && left >= kAdamScaleBlock) {
    *reinterpret_cast<f32x4*>(p + at + 4 * lane) = f32x4{x[0], x[1], x[2], x[3]};
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (element<VEC>(lane, i) < left) p[at + element<VEC>(lane, i)] = x[i];
  }
}

template <bool VEC, int DT>
__device__ __forceinline__ void load_grad4(float (&x)[4], const void* g, uint64_t at, int lane, int64_t left) {
  if constexpr (DT == DP_F32) {
    load4<VEC>(x, static_cast<const float*>(g), at, lane, left);
  } else if (VEC && left >= kAdamScaleBlock) {
    const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(g) + at + 4 * lane);
    const uint32_t u[2] = {w.x, w.y};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t pair = u[i / 2];
      if (DT == DP_BF16)
        x[i] = __uint_as_float(i & 1 ? pair & 0xFFFF0000u : pair << 16);
      else
        x[i] = (float)__builtin_bit_cast(_Float16, (uint16_t)(i & 1 ? pair >> 16 : pair & 0xFFFFu));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = element<VEC>(lane, i) < left ? load_grad<DT>(g, at + element<VEC>(lane, i)) : 0.f;
  }
}

template <bool VEC>
__device__ __forceinline__ uint32_t load_codes(const void* p, uint64_t at, int lane, int64_t left) {
  const uint8_t* c = static_cast<const uint8_t*>(p) + at;
  if (VEC && left >= kAdamScaleBlock) return reinterpret_cast<const uint32_t*>(c)[lane];
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (element<VEC>(lane, i) < left) w |= (uint32_t)c[element<VEC>(lane, i)] << (8 * i);
  return w;
}

template <bool VEC>
__device__ __forceinline__ void store_codes(uint32_t w, void* p, uint64_t at, int lane, int64_t left) {
  uint8_t* c = static_cast<uint8_t*>(p) + at;
  if (VEC && left >= kAdamScaleBlock) {
    reinterpret_cast<uint32_t*>(c)[lane] = w;
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (element<VEC>(lane, i) < left) c[element<VEC>(lane, i)] = (uint8_t)(w >> (8 * i));
}

__device__ __forceinline__ void decode(float (&x)[4], uint32_t w, float scale) {
  const f32x2v lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
  x[0] = lo[0] * scale;
  x[1] = lo[1] * scale;
  x[2] = hi[0] * scale;
  x[3] = hi[1] * scale;
}

// A wave's 8-bit step is bound by its instructions, divisions and square roots for the most part, which as the compiler has them
// serve all of fp32's range.  These round as they do, to nearest even, where nothing is lost below fp32's smallest numbers: the remainder
// of a quotient (or of a root's square) is exact there.  Quotients by their remainder over a corrected reciprocal is Markstein's method; a root
// whose remainders against both neighbours decide is Tuckerman's test.
__device__ __forceinline__ float reciprocal(float d) {
  const float r = __builtin_amdgcn_rcpf(d);
  return fmaf(fmaf(-d, r, 1.f), r, r);
}
__device__ __forceinline__ float divide(float n, float d, float r) {          // r: reciprocal(d)
  const float q = n * r;
  return fmaf(fmaf(-d, q, n), r, q);
}
__device__ __forceinline__ float root_of(float x) {                            // 0, or from 2^-96 on; the instruction is off by a unit at most
  const float s = __builtin_amdgcn_sqrtf(x), down = __uint_as_float(__float_as_uint(s) - 1), up = __uint_as_float(__float_as_uint(s) + 1);
  const float to_down = fmaf(-down, s, x), to_up = fmaf(-up, s, x);
  return to_up > 0.f ? up : to_down <= 0.f ? down : s;
}

// Codes of a block of 256 values (four to a lane) and its scale.  dither: in [0, 1), a value for each element.
template <bool ROOT>
__device__ __forceinline__ uint32_t encode(const float (&x)[4], const float (&dither)[4], float& scale) {
  uint32_t top = 0;                                // of magnitudes as integers: what is no number stays the largest
#pragma unroll
  for (int i = 0; i < 4; ++i) top = max(top, __float_as_uint(x[i]) & 0x7FFFFFFFu);
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, off));
  scale = __uint_as_float(top) * (1.f / 448.f);
  const float unit = scale > 0.f ? scale : 1.f;
  float c[4], quotient[4];
  if (__builtin_amdgcn_readfirstlane(unit > 0x1p-60f && unit < 0x1p60f)) {
    const float r = reciprocal(unit);
#pragma unroll
    for (int i = 0; i < 4; ++i) quotient[i] = divide(fabsf(x[i]), unit, r);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) quotient[i] = fabsf(x[i]) / unit;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float a = quotient[i];
    const int e = max(__builtin_amdgcn_frexp_expf(a) - 1, -6) - 3;
    const float y = ldexpf(a, -e), low = floorf(y), between = 2.f * low + 1.f;
    const float rest = ROOT ? divide((y - low) * (y + low), between, reciprocal(between)) : y - low;
    const float q = ldexpf(low + floorf(rest + dither[i]), e);
    c[i] = a > 0.f ? copysignf(fminf(fmaxf(q, 0x1p-9f), 448.f), x[i]) : 0.f;
  }
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(c[0], c[1], 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c[2], c[3], w, true);
}

// One block of 256 values, `left` of them there.
template <bool VEC, int GRAD, int BITS, int COPY>
struct Block {
  float w[4], g[4], m[4], v[4];
  uint32_t mc, vc;
  float ms, vs;
  __device__ __forceinline__ void load(const AdamTensor& t, uint64_t at, int lane, int64_t left) {
    load4<VEC>(w, t.param, at, lane, left);
    load_grad4<VEC, GRAD>(g, t.grad, at, lane, left);
    if constexpr (BITS == 32) {
      load4<VEC>(m, static_cast<const float*>(t.m), at, lane, left);
      load4<VEC>(v, static_cast<const float*>(t.v), at, lane, left);
    } else {
      mc = load_codes<VEC>(t.m, at, lane, left);
      vc = load_codes<VEC>(t.v, at, lane, left);
      ms = t.m_scale[at / kAdamScaleBlock];
      vs = t.v_scale[at / kAdamScaleBlock];
    }
  }
  __device__ __forceinline__ void step(const AdamArgs& a, const AdamTensor& t, uint64_t at, int lane, int64_t left) {
    if constexpr (BITS == 8) {
      decode(m, mc, ms);
      decode(v, vc, vs);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] *= v[i];
    }
    float root[4], fixed[4];                       // roots of v and of v / (1 - beta2^t)
    uint32_t least = ~0u;                          // of v but zeros
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      g[i] *= a.grad_scale;
      m[i] = a.beta1 * m[i] + a.rest1 * g[i];
      v[i] = a.beta2 * v[i] + a.rest2 * g[i] * g[i];
      least = min(least, __float_as_uint(v[i]) - 1);
    }
    if (BITS == 8 && !__any(least < __float_as_uint(0x1p-96f) - 1)) {          // (fix2 is at least 1)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        root[i] = root_of(v[i]);
        fixed[i] = root_of(v[i] * a.fix2);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        root[i] = sqrtf(v[i]);
        fixed[i] = sqrtf(v[i] * a.fix2);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = w[i] * t.keep - a.lr * (m[i] * a.fix1 / (fixed[i] + a.eps));
    store4<VEC>(w, t.param, at, lane, left);
    if constexpr (COPY != DP_F32) {
      uint16_t* c = static_cast<uint16_t*>(t.copy) + at;
      if (VEC && left >= kAdamScaleBlock) {
        uint16_t h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = to_half<COPY>(w[i]);
        *reinterpret_cast<uint2*>(c + 4 * lane) = make_uint2(h[0] | (uint32_t)h[1] << 16, h[2] | (uint32_t)h[3] << 16);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (element<VEC>(lane, i) < left) c[element<VEC>(lane, i)] = to_half<COPY>(w[i]);
      }
    }
    if constexpr (BITS == 32) {
      store4<VEC>(m, static_cast<float*>(t.m), at, lane, left);
      store4<VEC>(v, static_cast<float*>(t.v), at, lane, left);
    } else {
      float dither[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t e = (uint32_t)at + element<VEC>(lane, i);
        dither[i] = (float)((e * 0x6A09E667u + a.dither) >> 8) * 0x1p-24f;
        if (element<VEC>(lane, i) >= left) m[i] = root[i] = 0.f;
      }
      float scale;
      const uint32_t m_new = encode<false>(m, dither, scale);
      store_codes<VEC>(m_new, t.m, at, lane, left);
      if (lane == 0) t.m_scale[at / kAdamScaleBlock] = scale;
      const uint32_t v_new = encode<true>(root, dither, scale);
      store_codes<VEC>(v_new, t.v, at, lane, left);
      if (lane == 0) t.v_scale[at / kAdamScaleBlock] = scale;
    }
  }
};

template <bool VEC, int GRAD, int BITS, int COPY>
__device__ __forceinline__ void update(const AdamArgs& a, const AdamTensor& t, uint64_t first) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  Block<VEC, GRAD, BITS, COPY> block[kBlocks];
#pragma unroll
  for (int q = 0; q < kBlocks; ++q) {
    const uint64_t at = first + (q * (kThreads / 64) + wave) * kAdamScaleBlock;
    if (at < t.n) block[q].load(t, at, lane, (int64_t)(t.n - at));
  }
#pragma unroll
  for (int q = 0; q < kBlocks; ++q) {
    const uint64_t at = first + (q * (kThreads / 64) + wave) * kAdamScaleBlock;
    if (at < t.n) block[q].step(a, t, at, lane, (int64_t)(t.n - at));
  }
}

template <int GRAD, int BITS, int COPY>
__global__ void __launch_bounds__(kThreads) adamw_kernel(const AdamArgs a) {
  // The tensor that owns this workgroup: the last whose first workgroup is not past it, a lane to each of 64.
  const unsigned id = a.first + blockIdx.x;
  const int lane = threadIdx.x & 63;
  int owner = -1;
#pragma unroll
  for (int k = 0; k < kAdamTensors; k += 64)
    owner += __builtin_popcountll(__ballot(k + lane < a.n_tensors && a.begin[min(k + lane, kAdamTensors - 1)] <= id));
  owner = __builtin_amdgcn_readfirstlane(owner);
  const AdamTensor t = a.t[owner];
  const uint64_t first = (uint64_t)(id - a.begin[owner]) * kAdamChunk;
  if (t.whole)
    update<true, GRAD, BITS, COPY>(a, t, first);
  else
    update<false, GRAD, BITS, COPY>(a, t, first);
}

}  // namespace

dp_status launch_adamw(const AdamArgs& a, int64_t blocks, dp_dtype grad_dt, int state_bits, int copy_dt, hipStream_t s) {
  using std::integral_constant;
  auto launch = [&](auto grad, auto bits, auto copy) {
    return launch_in_runs(blocks, [&](dim3 grid, int first) {
      AdamArgs run = a;
      run.first = (unsigned)first;
      hipLaunchKernelGGL((adamw_kernel<decltype(grad)::value, decltype(bits)::value, decltype(copy)::value>), grid, dim3(kThreads), 0, s, run);
    });
  };
  auto by_copy = [&](auto grad, auto bits) {
    if (copy_dt == DP_BF16) return launch(grad, bits, integral_constant<int, DP_BF16>{});
    if (copy_dt == DP_F16) return launch(grad, bits, integral_constant<int, DP_F16>{});
    return launch(grad, bits, integral_constant<int, DP_F32>{});
  };
  auto by_bits = [&](auto grad) {
    return state_bits == 8 ? by_copy(grad, integral_constant<int, 8>{}) : by_copy(grad, integral_constant<int, 32>{});
  };
  if (grad_dt == DP_BF16) return by_bits(integral_constant<int, DP_BF16>{});
  if (grad_dt == DP_F16) return by_bits(integral_constant<int, DP_F16>{});
  return by_bits(integral_constant<int, DP_F32>{});
}

}  // namespace dpbk
