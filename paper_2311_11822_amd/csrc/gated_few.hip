// Gated feed-forward layers of few rows (single tokens of some sequences), 16-bit types: what counts is how fast the weights come.
//
// A workgroup has 16 columns (forward: of both weights) and all rows; its eight waves take eighths of the contraction, each on its own: a ring of
// blocks of 32 terms in LDS that no other wave reads, so there is no barrier before the eight sums are added, in their order.  A block is one
// load of 16 bytes a lane for each 16 rows and each 16 columns; as many as LDS holds are on their way.  Workgroups of adjacent columns are on one
// XCD, whose L2 has the other parts of their lines.
#include "gated.h"
#include "lds_dma.h"
#include "tile_order.h"

namespace dpbk {

namespace {

constexpr int kWaves = 8, kThreads = 64 * kWaves, kTerms = 32;

// TM: sixteens of rows; SETS: sets of 16 columns.
template <int TM, int SETS>
struct Few {
  static constexpr int LOADS = TM + SETS, BLOCK_BYTES = 1024 * LOADS, DEPTH = 163840 / kWaves / BLOCK_BYTES, RING_BYTES = DEPTH * BLOCK_BYTES;
  static constexpr int LDS_BYTES = kWaves * RING_BYTES;
  static_assert(kWaves * TM * SETS * 1024 <= LDS_BYTES && DEPTH * LOADS <= 60, "sums; vmcnt counts up to 63");
};

template <int PASS, int TM, int DT>
__global__ void __launch_bounds__(kThreads) gated_few_kernel(const GatedArgs a, int groups) {
  constexpr bool COLUMNS = PASS == kForward;
  constexpr int SETS = COLUMNS ? 2 : 1;
  typedef Few<TM, SETS> F;
  extern __shared__ __attribute__((aligned(1024))) unsigned char lds_raw[];
  const unsigned lds0 = (unsigned)(uintptr_t)lds_raw;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int N = PASS == kInput ? a.d : a.f, K = COLUMNS ? a.d : PASS == kHidden ? a.d_out : a.f;
  const int n0 = 16 * contiguous_eighth(blockIdx.x, groups);
  const unsigned a_pitch = 2u * K, b_pitch = 2u * (COLUMNS ? N : K), ring = lds0 + wave * F::RING_BYTES;

  // a row operand's 1 KiB: 16 rows of 32 terms, the 16-byte places of a row XORed with row / 4; a columns operand's: 32 terms of 16 columns
  const int row = lane >> 2, chunk = (lane & 3) ^ (row >> 2);
  const unsigned va = row * a_pitch + chunk * 16;
  const int column = n0 + 8 * (lane & 1);
  const unsigned vb = COLUMNS ? (column < N ? (lane >> 1) * b_pitch + 2u * column : OOB) : row * b_pitch + chunk * 16;

  // this wave's blocks, of all segments one behind the other
  const int per = (K + kTerms - 1) / kTerms, total = per * (PASS == kInput ? 2 : 1), share = (total + kWaves - 1) / kWaves;
  const int first = imin(wave * share, total), count = imin(share, total - first);
  i32x4 ra[TM], rb[SETS];
  int seg = first >= per ? 1 : 0, k = (first - seg * per) * kTerms, left = count;      // of the block to ask for next
  auto scalar = [](i32x4 r) {
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __builtin_amdgcn_readfirstlane(r[i]);
    return r;
  };
  auto open = [&]() {
    const char* const x = static_cast<const char*>(PASS == kForward ? a.x : PASS == kHidden ? a.dy : seg ? a.dup : a.dgate);
#pragma unroll
    for (int m = 0; m < TM; ++m) ra[m] = make_rsrc(x + (uint64_t)16 * m * a_pitch, (unsigned)imax(imin(a.rows - 16 * m, 16), 0) * a_pitch);
    if constexpr (COLUMNS) {
      rb[0] = make_rsrc(a.w_gate, 0);
      rb[SETS - 1] = make_rsrc(a.w_up, 0);
    } else {
      const char* const w = static_cast<const char*>(PASS == kHidden ? a.w_down : seg ? a.w_up : a.w_gate);
      rb[0] = make_rsrc(w + (uint64_t)n0 * b_pitch, (unsigned)imin(N - n0, 16) * b_pitch);
    }
  };
  auto ask = [&](int place) {                          // a block past the last one is asked for as zeros, so that loads can be counted
    const unsigned to = ring + place * F::BLOCK_BYTES;
    const bool there = left > 0, in = there && k + 8 * chunk < K;
#pragma unroll
    for (int m = 0; m < TM; ++m) load_to_lds(scalar(ra[m]), in ? va : OOB, 2u * k, to + 1024 * m);
#pragma unroll
    for (int s = 0; s < SETS; ++s) {
      if constexpr (COLUMNS) {
        const uint64_t at = (uint64_t)(s ? a.w_up : a.w_gate) + (uint64_t)k * b_pitch;
        const i32x4 r = make_rsrc((const void*)at, there ? (unsigned)imin(K - k, kTerms) * b_pitch : 0);
        load_to_lds(scalar(r), vb, 0, to + 1024 * (TM + s));
      } else {
        load_to_lds(scalar(rb[s]), in ? vb : OOB, 2u * k, to + 1024 * (TM + s));
      }
    }
    --left;
    k += kTerms;
    if (k >= K && left > 0) {
      seg = 1;
      k = 0;
      open();
    }
  };
  open();
  f32x4 acc[TM][SETS];
#pragma unroll
  for (int m = 0; m < TM; ++m)
#pragma unroll
    for (int s = 0; s < SETS; ++s) acc[m][s] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int r16 = lane & 15, h = lane >> 4;
  const unsigned a_rd = ring + r16 * 64 + ((h ^ (r16 >> 2)) << 4);
  const unsigned b_rd = ring + 1024 * TM + (COLUMNS ? (8 * h + (r16 >> 2)) * 32 + 8 * (r16 & 3) : r16 * 64 + ((h ^ (r16 >> 2)) << 4));
  for (int i = 0; i < F::DEPTH - 1; ++i) ask(i);
  int place = 0;
  for (int i = 0; i < count; ++i) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");         // the place that is asked for next has been read
    ask(place == 0 ? F::DEPTH - 1 : place - 1);
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((F::DEPTH - 1) * F::LOADS) : "memory");
    const unsigned at = place * F::BLOCK_BYTES;
    Frag fa[TM], fb[SETS];
    typedef __attribute__((address_space(3))) const bf16x8* Lds;
#pragma unroll
    for (int m = 0; m < TM; ++m) fa[m].v = *(Lds)(uintptr_t)(a_rd + at + 1024 * m);
#pragma unroll
    for (int s = 0; s < SETS; ++s) {
      if constexpr (COLUMNS) {
        fb[s].h[0] = lds_read_tr(b_rd + at + 1024 * s);
        fb[s].h[1] = lds_read_tr(b_rd + at + 1024 * s + 4 * 32);
      } else {
        fb[s].v = *(Lds)(uintptr_t)(b_rd + at + 1024 * s);
      }
    }
#pragma unroll
    for (int m = 0; m < TM; ++m)
#pragma unroll
      for (int s = 0; s < SETS; ++s) acc[m][s] = mfma16<DT == DP_F16>(fb[s].v, fa[m].v, acc[m][s]);
    place = place + 1 == F::DEPTH ? 0 : place + 1;
  }
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  __syncthreads();

  // The waves' sums: [m][s][wave][row 16][column 16]; a lane has row lane % 16, four columns from 4 (lane / 16) on.
  float* const sums = reinterpret_cast<float*>(lds_raw);
#pragma unroll
  for (int m = 0; m < TM; ++m)
#pragma unroll
    for (int s = 0; s < SETS; ++s) *reinterpret_cast<f32x4*>(sums + ((m * SETS + s) * kWaves + wave) * 256 + r16 * 16 + 4 * h) = acc[m][s];
  __syncthreads();
  auto finish = [&](auto act) {
    for (int e = tid; e < TM * 256; e += kThreads) {
      const int m = e >> 8, at = e & 255, r = 16 * m + (at >> 4), n = n0 + (at & 15);
      if (r >= a.rows || n >= N) continue;
      float v[SETS];
#pragma unroll
      for (int s = 0; s < SETS; ++s) {
        v[s] = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) v[s] += sums[((m * SETS + s) * kWaves + w) * 256 + at];
      }
      const int64_t to = (int64_t)r * N + n;
      float slope;
      Values<DT, 1> one;
      auto value = [&](const void* from, int64_t place) {
        Values<DT, 1> x;
        x.load(from, place);
        return x.get(0);
      };
      auto put = [&](void* out, float x) {
        one.set({x});
        one.store(out, to);
      };
      if constexpr (PASS == kForward) {
        const float gate = v[0] + (a.b_gate ? value(a.b_gate, n) : 0.f), up = v[SETS - 1] + (a.b_up ? value(a.b_up, n) : 0.f);
        if (a.gate) {
          put(a.gate, gate);
          put(a.up, up);
        }
        put(a.h, activation<decltype(act)::value, false, false>(gate, slope) * up);
      } else if constexpr (PASS == kHidden) {
        const float up = value(a.up, to), x = activation<decltype(act)::value, false, true>(value(a.gate, to), slope);
        put(a.dgate, v[0] * up * slope);
        put(a.dup, v[0] * x);
      } else {
        put(a.dx, v[0]);
      }
    }
  };
  if constexpr (PASS == kInput)
    finish(std::integral_constant<int, DP_ACT_RELU>{});
  else
    with_activation(a.act, finish);
}

template <int PASS, int TM, int DT>
dp_status launch(const GatedArgs& a, hipStream_t s) {
  typedef Few<TM, PASS == kForward ? 2 : 1> F;
  static ReadyTable ready;
  const dp_status st = allow_big_lds(gated_few_kernel<PASS, TM, DT>, F::LDS_BYTES, ready);
  if (st != DP_OK) return st;
  const int groups = ((PASS == kInput ? a.d : a.f) + 15) / 16;
  gated_few_kernel<PASS, TM, DT><<<dim3((unsigned)groups), kThreads, F::LDS_BYTES, s>>>(a, groups);
  return hip_status(hipGetLastError());
}

template <int PASS, int DT>
dp_status launch_rows(const GatedArgs& a, hipStream_t s) {
  return a.rows <= 16 ? launch<PASS, 1, DT>(a, s) : a.rows <= 32 ? launch<PASS, 2, DT>(a, s) : launch<PASS, 4, DT>(a, s);
}

template <int DT>
dp_status launch_pass(const GatedArgs& a, GatedPass pass, hipStream_t s) {
  return pass == kForward ? launch_rows<kForward, DT>(a, s) : pass == kHidden ? launch_rows<kHidden, DT>(a, s) : launch_rows<kInput, DT>(a, s);
}

}  // namespace

dp_status launch_gated_few(const GatedArgs& a, dp_dtype dt, GatedPass pass, hipStream_t s) {
  return dt == DP_BF16 ? launch_pass<DP_BF16>(a, pass, s) : launch_pass<DP_F16>(a, pass, s);
}

}  // namespace dpbk
