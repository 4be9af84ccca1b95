// Attention, forward: o_i = sum_j p_ij v_j with p_ij = exp(scale q_i k_j - lse_i) over the keys j that row i sees, in one pass over keys and
// values with a running maximum and sum.
#include <type_traits>

#include "attention.h"

namespace dpbk {

namespace {

#ifndef FWD_OCC
#define FWD_OCC(DP) (DP <= 64 ? 3 : 2)
#endif
#ifndef FWD_PIPE
#define FWD_PIPE (DP > 64)
#endif
constexpr int kKeys = 64;                         // of a tile
constexpr float kLazy = 8.f;                      // a maximum may be passed by 2^8 before sums are expressed in a new one

template <bool F16, int DP, int NW, bool PIPE>
__global__ void __launch_bounds__(64 * NW, FWD_OCC(DP)) attention_kernel(const AttnArgs a) {
  extern __shared__ __align__(1024) char smem[];
  constexpr int TILE = kKeys * HeadTile<DP>::ROW_BYTES;
  int pair, block;
  attn_unit(a, a.first + blockIdx.x, pair, block);
  if (pair >= a.heads) return;
  const int b = pair / a.H, h = pair % a.H;
  if (a.causal) block = a.blocks - 1 - block;     // the longest first
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n_q = valid_rows(a.q_len, b, a.Tq), n_k = valid_rows(a.k_len, b, a.Tk), shift = n_k - n_q;
  const int row0 = block * 32 * NW, own0 = row0 + 32 * wave, row = own0 + (lane & 31);
  const unsigned lds = (unsigned)(uintptr_t)DP_LDS(char, smem);

  // Keys that the workgroup's, this wave's and the lane's rows see: below these.
  const int last = min(row0 + 32 * NW, n_q) - 1, own_last = min(own0 + 32, n_q) - 1;
  const int end = row0 >= n_q ? 0 : a.causal ? min(n_k, last + shift + 1) : n_k;
  const int own_end = own0 >= n_q ? 0 : a.causal ? min(n_k, own_last + shift + 1) : n_k;
  const int lane_end = row >= n_q ? 0 : a.causal ? min(n_k, row + shift + 1) : n_k;

  const uint16_t* q = static_cast<const uint16_t*>(a.q) + b * a.qs.sample + h * a.qs.head;
  TileLoader<DP, kKeys, NW> k_tiles, v_tiles;
  k_tiles.init(static_cast<const uint16_t*>(a.k) + b * a.ks.sample + h / a.share * a.ks.head, a.ks.token, a.D, wave, lane);
  v_tiles.init(static_cast<const uint16_t*>(a.v) + b * a.vs.sample + h / a.share * a.vs.head, a.vs.token, a.D, wave, lane);
  constexpr int KS = DP / 16, CB = DP / 32;
  constexpr int V = 2 * TILE;                     // two stages of keys, then two of values
  if (end > 0) {
    k_tiles.load(0, n_k, lds, wave);
    if (PIPE) k_tiles.load(kKeys, n_k, lds + TILE, wave);
    v_tiles.load(0, n_k, lds + V, wave);
  }
  bf16x8 qf[KS];
  load_own<DP>(qf, q, a.qs.token, row, row < n_q, a.D, lane);
  TileReader<DP> read;
  read.init(lds, lane);

  f32x16 o[CB];
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) o[cb] = zeros16();
  float most = -3.4028235e38f, total = 0.f;       // of scale2 * score; total: of this half's keys
  auto scores = [&](f32x16 (&to)[2], int tile) {
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      to[kb] = zeros16();
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) to[kb] = mfma16<F16>(read.rows(tile, 32 * kb, ks), qf[ks], to[kb]);
    }
  };
  const int all_see = a.causal ? min(n_k, own0 + shift + 1) : n_k;       // keys that each of the wave's rows sees
  // One tile, in stage STAGE.  PIPE: s has its scores, and next gets those of the tile behind it (behind the last one: of what LDS holds,
  // and not used).
  auto step = [&](f32x16 (&s)[2], f32x16 (&next)[2], int j0, auto stage_tag) {
    constexpr int STAGE = decltype(stage_tag)::value, HERE = STAGE * TILE, THERE = TILE - HERE;
    tiles_landed();
    if (PIPE) {
      if (j0 + 2 * kKeys < end) k_tiles.load(j0 + 2 * kKeys, n_k, lds + HERE, wave);
    } else {
      if (j0 + kKeys < end) k_tiles.load(j0 + kKeys, n_k, lds + THERE, wave);
    }
    if (j0 + kKeys < end) v_tiles.load(j0 + kKeys, n_k, lds + V + THERE, wave);
    if (j0 >= own_end) return;
    if (!PIPE) scores(s, HERE);
    if (j0 + kKeys > all_see) {
      const int seen = lane_end - j0 - 4 * (lane >> 5);
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (32 * kb + 8 * (r >> 2) + (r & 3) >= seen) s[kb][r] = -INFINITY;
    }
    float top = s[0][0];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) top = fmaxf(top, s[kb][r]);
    top = fmaxf(top, other_half(top, lane)) * a.scale2;
    if (__any(top > most + kLazy)) {
      const float higher = fmaxf(most, top), fix = __builtin_amdgcn_exp2f(most - higher);
      most = higher;
      total *= fix;
#pragma unroll
      for (int cb = 0; cb < CB; ++cb)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[cb][r] *= fix;
    }
    if (PIPE) scores(next, THERE);
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[kb][r] = __builtin_amdgcn_exp2f(fmaf(s[kb][r], a.scale2, -most));
        total += s[kb][r];
      }
#pragma unroll
    for (int ks = 0; ks < kKeys / 16; ++ks) {
      const bf16x8 p = round8<F16>(s[ks >> 1], 8 * (ks & 1));
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) o[cb] = mfma16<F16>(read.columns(V + HERE, 16 * ks, cb), p, o[cb]);
    }
  };
  if (end > 0) {
    f32x16 s[2], t[2];
    if (PIPE) {
      tiles_landed();
      scores(s, 0);                               // (the next barrier says that all waves are through with these keys)
    }
    for (int j0 = 0;;) {
      step(s, t, j0, std::integral_constant<int, 0>{});
      if ((j0 += kKeys) >= end) break;
      step(t, s, j0, std::integral_constant<int, 1>{});
      if ((j0 += kKeys) >= end) break;
    }
  }
  total += other_half(total, lane);
  const bool there = lane_end > 0 && total != 0.f;
  store_rows16<F16, DP>(o, 1.f / total, there, static_cast<uint16_t*>(a.out) + b * a.os.sample + h * a.os.head, a.os.token, row,
                        a.Tq, a.D, lane);
  if (lane < 32 && row < a.Tq)
    a.lse[((int64_t)b * a.H + h) * a.Tq + row] = there ? most * kLn2 + logf(total) : -INFINITY;
  // A zero probability times an infinity is no number: rows beside a token that they do not see.
  if (a.causal && __any(there && (not_finite(o) || !(fabsf(total) < INFINITY)))) {
    const AttnRows<typename Half<F16>::T> rows(a, b, h, lane);
    for (int i = own0; i < min(own0 + 32, n_q); ++i) rows.forward(i);
  }
}

__global__ void __launch_bounds__(256) attention_f32_kernel(const AttnArgs a) {
  int pair, block;
  attn_unit(a, a.first + blockIdx.x, pair, block);
  if (pair >= a.heads) return;
  const AttnRows<float> rows(a, pair / a.H, pair % a.H, threadIdx.x & 63);
  const int i = block * 4 + (threadIdx.x >> 6);
  if (i < a.Tq) rows.forward(i);
}

template <bool F16, int DP, int NW>
dp_status launch(AttnArgs a, hipStream_t s) {
  a.heads = a.B * a.H;
  a.blocks = (a.Tq + 32 * NW - 1) / (32 * NW);
  constexpr int LDS = 4 * kKeys * HeadTile<DP>::ROW_BYTES;
  auto kernel = attention_kernel<F16, DP, NW, FWD_PIPE>;
  static ReadyTable done;
  if (LDS > 65536) {
    const dp_status st = allow_big_lds(kernel, LDS, done);
    if (st != DP_OK) return st;
  }
  return launch_attention(kernel, a, 64 * NW, LDS, s);
}

#ifndef FWD_NW
#define FWD_NW 4
#endif
template <bool F16, int DP>
dp_status launch(const AttnArgs& a, hipStream_t s) {
  if (a.Tq <= 32) return launch<F16, DP, 1>(a, s);
  if (a.Tq <= 64) return launch<F16, DP, 2>(a, s);
  return launch<F16, DP, FWD_NW>(a, s);
}

template <bool F16>
dp_status launch(const AttnArgs& a, hipStream_t s) {
  if (a.D <= 32) return launch<F16, 32>(a, s);
  if (a.D <= 64) return launch<F16, 64>(a, s);
  if (a.D <= 96) return launch<F16, 96>(a, s);
  return launch<F16, 128>(a, s);
}

}  // namespace

dp_status launch_attention_forward(const AttnArgs& args, dp_dtype dt, hipStream_t s) {
  if (dt != DP_F32) return dt == DP_F16 ? launch<true>(args, s) : launch<false>(args, s);
  AttnArgs a = args;
  a.heads = a.B * a.H;
  a.blocks = (a.Tq + 3) / 4;
  return launch_attention(attention_f32_kernel, a, 256, 0, s);
}

}  // namespace dpbk
