// Attention, backward.  With p_ij = exp(scale q_i k_j - lse_i) formed again from the forward pass's lse:
//   dv_j = sum_i p_ij do_i,   ds_ij = p_ij (do_i v_j - delta_i),   delta_i = do_i o_i,
//   dq_i = scale sum_j ds_ij k_j,   dk_j = scale sum_i ds_ij q_i     (over the query heads that share the key head, too).
// Two kernels, one that owns queries and one that owns keys, so that every sum has one owner and a fixed order: no atomics, no
// partial sums in memory.  The price is that scores and do v' are formed in both, seven products for five.
#include "attention.h"

namespace dpbk {

namespace {

// dq, and for the other kernel delta and lse in units of log 2.
constexpr int kKeys = 64;
template <bool F16, int DP, int NW>
__global__ void __launch_bounds__(64 * NW, 2) attention_query_grad_kernel(const AttnArgs a) {
  extern __shared__ __align__(1024) char smem[];
  constexpr int TILE = kKeys * HeadTile<DP>::ROW_BYTES, STAGE = 2 * TILE;
  int pair, block;
  attn_unit(a, a.first + blockIdx.x, pair, block);
  if (pair >= a.heads) return;
  const int b = pair / a.H, h = pair % a.H;
  if (a.causal) block = a.blocks - 1 - block;     // the longest first
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n_q = valid_rows(a.q_len, b, a.Tq), n_k = valid_rows(a.k_len, b, a.Tk), shift = n_k - n_q;
  const int row0 = block * 32 * NW, own0 = row0 + 32 * wave, row = own0 + (lane & 31);
  const unsigned lds = (unsigned)(uintptr_t)DP_LDS(char, smem);
  const int last = min(row0 + 32 * NW, n_q) - 1, own_last = min(own0 + 32, n_q) - 1;
  const int end = row0 >= n_q ? 0 : a.causal ? min(n_k, last + shift + 1) : n_k;
  const int own_end = own0 >= n_q ? 0 : a.causal ? min(n_k, own_last + shift + 1) : n_k;
  const int lane_end = row >= n_q ? 0 : a.causal ? min(n_k, row + shift + 1) : n_k;

  TileLoader<DP, kKeys, NW> k_tiles, v_tiles;
  k_tiles.init(static_cast<const uint16_t*>(a.k) + b * a.ks.sample + h / a.share * a.ks.head, a.ks.token, a.D, wave, lane);
  v_tiles.init(static_cast<const uint16_t*>(a.v) + b * a.vs.sample + h / a.share * a.vs.head, a.vs.token, a.D, wave, lane);
  if (end > 0) {
    k_tiles.load(0, n_k, lds, wave);
    v_tiles.load(0, n_k, lds + TILE, wave);
  }
  bf16x8 qf[DP / 16], df[DP / 16];
  load_own<DP>(qf, static_cast<const uint16_t*>(a.q) + b * a.qs.sample + h * a.qs.head, a.qs.token, row, row < n_q, a.D, lane);
  load_own<DP>(df, static_cast<const uint16_t*>(a.dout) + b * a.os.sample + h * a.os.head, a.os.token, row, row < n_q, a.D, lane);
  // delta: the diagonal of o do', formed as do v' is: a row that sees one key alone has the same products in both, and zero
  // gradients of its scores, not what two orders of adding leave.
  float delta = 0.f;
  {
    bf16x8 of[DP / 16];
    load_own<DP>(of, static_cast<const uint16_t*>(a.o) + b * a.os.sample + h * a.os.head, a.os.token, row, row < n_q, a.D, lane);
    f32x16 od = zeros16();
#pragma unroll
    for (int ks = 0; ks < DP / 16; ++ks) od = mfma16<F16>(of[ks], df[ks], od);
#pragma unroll
    for (int r = 0; r < 16; ++r)
      if (8 * (r >> 2) + 4 * (lane >> 5) + (r & 3) == (lane & 31)) delta = od[r];
    const float there = other_half(delta, lane);
    if (((lane >> 2) & 1) != lane >> 5) delta = there;
  }
  const int64_t at = ((int64_t)b * a.H + h) * a.Tq + row;
  float lse2 = INFINITY;                          // a row that sees nothing
  if (lane_end > 0) {
    lse2 = a.lse[at] * kLog2e;
    if (lse2 == -INFINITY) lse2 = INFINITY;
  }
  if (lane_end == 0) delta = 0.f;

  f32x16 dq[DP / 32];
#pragma unroll
  for (int cb = 0; cb < DP / 32; ++cb) dq[cb] = zeros16();
  for (int j0 = 0, stage = 0; j0 < end; j0 += kKeys, stage ^= 1) {
    tiles_landed();
    const unsigned kt = lds + stage * STAGE, vt = kt + TILE;
    if (j0 + kKeys < end) {
      k_tiles.load(j0 + kKeys, n_k, lds + (stage ^ 1) * STAGE, wave);
      v_tiles.load(j0 + kKeys, n_k, lds + (stage ^ 1) * STAGE + TILE, wave);
    }
    if (j0 >= own_end) continue;
    const bool mask = j0 + kKeys > (a.causal ? min(n_k, own0 + shift + 1) : n_k);
    // Probabilities and do v' of 32 keys.
    auto products = [&](int kb, f32x16& p, f32x16& dp) {
      p = dp = zeros16();
#pragma unroll
      for (int ks = 0; ks < DP / 16; ++ks) p = mfma16<F16>(read_rows<DP>(kt, 32 * kb, ks, lane), qf[ks], p);
#pragma unroll
      for (int ks = 0; ks < DP / 16; ++ks) dp = mfma16<F16>(read_rows<DP>(vt, 32 * kb, ks, lane), df[ks], dp);
#pragma unroll
      for (int r = 0; r < 16; ++r) p[r] = __builtin_amdgcn_exp2f(fmaf(p[r], a.scale2, -lse2));
    };
    auto hide = [&](int kb, f32x16& x) {          // a select: what is not seen may be no number
      const int seen = lane_end - j0 - 32 * kb - 4 * (lane >> 5);
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (8 * (r >> 2) + (r & 3) >= seen) x[r] = 0.f;
    };
    if (own_end <= kKeys) {
      // All that these rows see is at hand: delta from the probabilities, free of o's rounding, which counts where few keys share a
      // row (2-norm of dq's error against 64 bits, fp16, 18 x 591 tokens: 3.1e-4 with o's alone).
      float sum = 0.f;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        f32x16 p, dp;
        products(kb, p, dp);
#pragma unroll
        for (int r = 0; r < 16; ++r) p[r] *= dp[r];
        hide(kb, p);
#pragma unroll
        for (int r = 0; r < 16; ++r) sum += p[r];
      }
      sum += other_half(sum, lane);
      if (lane_end > 1) delta = sum;
    }
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      f32x16 s, dp;
      products(kb, s, dp);
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] *= dp[r] - delta;
      if (mask) hide(kb, s);
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        const bf16x8 ds = round8<F16>(s, 8 * ks);
#pragma unroll
        for (int cb = 0; cb < DP / 32; ++cb) dq[cb] = mfma16<F16>(read_columns<DP>(kt, 32 * kb + 16 * ks, cb, lane), ds, dq[cb]);
      }
    }
  }
  if (lane < 32 && row < a.Tq) {
    a.lse2[at] = lse2;
    a.delta[at] = delta;
  }
  store_rows16<F16, DP>(dq, a.scale, lane_end > 0, static_cast<uint16_t*>(a.dq) + b * a.qs.sample + h * a.qs.head, a.qs.token, row,
                        a.Tq, a.D, lane);
  if (a.causal && __any(lane_end > 0 && not_finite(dq))) {
    const AttnRows<typename Half<F16>::T> rows(a, b, h, lane);
    for (int i = own0; i < min(own0 + 32, n_q); ++i) rows.query_gradient(i);
  }
}

// dk and dv.  A wave owns 32 keys; tiles of queries and their output gradients go through LDS, with lse and delta.
constexpr int kRows = 64;
template <bool F16, int DP, int NW>
__global__ void __launch_bounds__(64 * NW, DP == 128 ? 1 : 2) attention_key_grad_kernel(const AttnArgs a) {
  extern __shared__ __align__(1024) char smem[];
  constexpr int TILE = kRows * HeadTile<DP>::ROW_BYTES, STAGE = 2 * TILE + 512;
  int pair, block;
  attn_unit(a, a.first + blockIdx.x, pair, block);
  if (pair >= a.heads) return;
  const int b = pair / a.H_kv, h = pair % a.H_kv;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n_q = valid_rows(a.q_len, b, a.Tq), n_k = valid_rows(a.k_len, b, a.Tk), shift = n_k - n_q;
  const int key0 = block * 32 * NW, own0 = key0 + 32 * wave, key = own0 + (lane & 31);
  const unsigned lds = (unsigned)(uintptr_t)DP_LDS(char, smem);
  // Queries from here on see a key of the workgroup, of this wave; and the first that sees the lane's.
  const int begin = a.causal ? max(key0 - shift, 0) & ~31 : 0;
  const int own_begin = a.causal ? max(own0 - shift, 0) : 0, lane_begin = a.causal ? key - shift : 0;
  const int tiles = key0 < n_k && begin < n_q ? (n_q - begin + kRows - 1) / kRows : 0;

  const int64_t kv = b * a.ks.sample + h * a.ks.head, vv = b * a.vs.sample + h * a.vs.head;
  bf16x8 kf[DP / 16], vf[DP / 16];
  load_own<DP>(kf, static_cast<const uint16_t*>(a.k) + kv, a.ks.token, key, key < n_k, a.D, lane);
  load_own<DP>(vf, static_cast<const uint16_t*>(a.v) + vv, a.vs.token, key, key < n_k, a.D, lane);
  TileLoader<DP, kRows, NW> q_tiles, d_tiles;
  q_tiles.init(static_cast<const uint16_t*>(a.q) + b * a.qs.sample + h * a.share * a.qs.head, a.qs.token, a.D, wave, lane);
  d_tiles.init(static_cast<const uint16_t*>(a.dout) + b * a.os.sample + h * a.share * a.os.head, a.os.token, a.D, wave, lane);
  const int64_t at = ((int64_t)b * a.H + h * a.share) * a.Tq;
  auto load = [&](int head, int i0, int stage) {
    const unsigned to = lds + stage * STAGE;
    const uint64_t q_head = 2 * (uint64_t)(head * a.qs.head), d_head = 2 * (uint64_t)(head * a.os.head);
    TileLoader<DP, kRows, NW> q = q_tiles, d = d_tiles;
    q.base += q_head;
    d.base += d_head;
    q.load(i0, n_q, to, wave);
    d.load(i0, n_q, to + TILE, wave);
    if (wave == 0) {                              // 64 values of either, zeros past the tensor's end
      const unsigned bytes = 4 * min(a.Tq - i0, kRows);
      const int64_t first = at + (int64_t)head * a.Tq + i0;
      load_dword_to_lds(make_rsrc(a.lse2 + first, bytes), 4 * lane, to + 2 * TILE);
      load_dword_to_lds(make_rsrc(a.delta + first, bytes), 4 * lane, to + 2 * TILE + 256);
    }
  };

  f32x16 dk[DP / 32], dv[DP / 32];
#pragma unroll
  for (int cb = 0; cb < DP / 32; ++cb) dk[cb] = dv[cb] = zeros16();
  const int steps = tiles * a.share;
  int head = 0, i0 = begin;                       // of the tile that is loaded next
  auto advance = [&] {
    i0 += kRows;
    if (i0 >= n_q) {
      i0 = begin;
      ++head;
    }
  };
  if (steps > 0) {
    load(0, i0, 0);
    advance();
  }
  int here = begin;                               // first query of the tile at hand
  for (int step = 0, stage = 0; step < steps; ++step, stage ^= 1) {
    tiles_landed();
    const unsigned qt = lds + stage * STAGE, dt = qt + TILE;
    if (step + 1 < steps) load(head, i0, stage ^ 1);
    const int i_here = here;
    here = i0;
    advance();
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) {
      const int first = i_here + 32 * qb;
      if (own0 >= n_k || first >= n_q || first + 31 < own_begin) continue;
      f32x16 s = zeros16(), dp = zeros16();
#pragma unroll
      for (int ks = 0; ks < DP / 16; ++ks) s = mfma16<F16>(read_rows<DP>(qt, 32 * qb, ks, lane), kf[ks], s);
#pragma unroll
      for (int ks = 0; ks < DP / 16; ++ks) dp = mfma16<F16>(read_rows<DP>(dt, 32 * qb, ks, lane), vf[ks], dp);
      const auto* lse2 = (__attribute__((address_space(3))) const f32x4*)(uintptr_t)(dt + TILE + 128 * qb + 16 * (lane >> 5));
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 l = lse2[2 * g], d = lse2[16 + 2 * g];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          s[4 * g + i] = __builtin_amdgcn_exp2f(fmaf(s[4 * g + i], a.scale2, -l[i]));
          dp[4 * g + i] = s[4 * g + i] * (dp[4 * g + i] - d[i]);
        }
      }
      if (a.causal && first < own0 + 31 - shift) {
        const int hidden = lane_begin - first - 4 * (lane >> 5);
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (8 * (r >> 2) + (r & 3) < hidden) s[r] = dp[r] = 0.f;
      }
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        const bf16x8 p = round8<F16>(s, 8 * ks), ds = round8<F16>(dp, 8 * ks);
#pragma unroll
        for (int cb = 0; cb < DP / 32; ++cb) {
          dv[cb] = mfma16<F16>(read_columns<DP>(dt, 32 * qb + 16 * ks, cb, lane), p, dv[cb]);
          dk[cb] = mfma16<F16>(read_columns<DP>(qt, 32 * qb + 16 * ks, cb, lane), ds, dk[cb]);
        }
      }
    }
  }
  store_rows16<F16, DP>(dk, a.scale, key < n_k, static_cast<uint16_t*>(a.dk) + kv, a.ks.token, key, a.Tk, a.D, lane);
  store_rows16<F16, DP>(dv, 1.f, key < n_k, static_cast<uint16_t*>(a.dv) + vv, a.vs.token, key, a.Tk, a.D, lane);
  if (a.causal && __any(key < n_k && (not_finite(dk) || not_finite(dv)))) {
    const AttnRows<typename Half<F16>::T> rows(a, b, h, lane);
    for (int j = own0; j < min(own0 + 32, n_k); ++j) rows.key_gradient(j);
  }
}

__global__ void __launch_bounds__(256) attention_query_grad_f32_kernel(const AttnArgs a) {
  int pair, block;
  attn_unit(a, a.first + blockIdx.x, pair, block);
  if (pair >= a.heads) return;
  const AttnRows<float> rows(a, pair / a.H, pair % a.H, threadIdx.x & 63);
  const int i = block * 4 + (threadIdx.x >> 6);
  if (i < a.Tq) rows.query_gradient(i);
}

__global__ void __launch_bounds__(256) attention_key_grad_f32_kernel(const AttnArgs a) {
  int pair, block;
  attn_unit(a, a.first + blockIdx.x, pair, block);
  if (pair >= a.heads) return;
  const AttnRows<float> rows(a, pair / a.H_kv, pair % a.H_kv, threadIdx.x & 63);
  const int j = block * 4 + (threadIdx.x >> 6);
  if (j < a.Tk) rows.key_gradient(j);
}

template <bool F16, int DP, int NW>
dp_status launch_queries(AttnArgs a, hipStream_t s) {
  a.heads = a.B * a.H;
  a.blocks = (a.Tq + 32 * NW - 1) / (32 * NW);
  constexpr int LDS = 4 * kKeys * HeadTile<DP>::ROW_BYTES;
  auto kernel = attention_query_grad_kernel<F16, DP, NW>;
  static ReadyTable done;
  if (LDS > 65536) {
    const dp_status st = allow_big_lds(kernel, LDS, done);
    if (st != DP_OK) return st;
  }
  return launch_attention(kernel, a, 64 * NW, LDS, s);
}

template <bool F16, int DP, int NW>
dp_status launch_keys(AttnArgs a, hipStream_t s) {
  a.heads = a.B * a.H_kv;
  a.blocks = (a.Tk + 32 * NW - 1) / (32 * NW);
  constexpr int LDS = 2 * (2 * kRows * HeadTile<DP>::ROW_BYTES + 512);
  auto kernel = attention_key_grad_kernel<F16, DP, NW>;
  static ReadyTable done;
  if (LDS > 65536) {
    const dp_status st = allow_big_lds(kernel, LDS, done);
    if (st != DP_OK) return st;
  }
  return launch_attention(kernel, a, 64 * NW, LDS, s);
}

template <bool F16, int DP>
dp_status launch(const AttnArgs& a, hipStream_t s) {
  const dp_status st = a.Tq <= 32 ? launch_queries<F16, DP, 1>(a, s) : launch_queries<F16, DP, 4>(a, s);
  if (st != DP_OK) return st;
  return a.Tk <= 32 ? launch_keys<F16, DP, 1>(a, s) : launch_keys<F16, DP, 4>(a, s);
}

template <bool F16>
dp_status launch(const AttnArgs& a, hipStream_t s) {
  if (a.D <= 32) return launch<F16, 32>(a, s);
  if (a.D <= 64) return launch<F16, 64>(a, s);
  if (a.D <= 96) return launch<F16, 96>(a, s);
  return launch<F16, 128>(a, s);
}

}  // namespace

dp_status launch_attention_backward(const AttnArgs& args, dp_dtype dt, hipStream_t s) {
  if (dt != DP_F32) return dt == DP_F16 ? launch<true>(args, s) : launch<false>(args, s);
  AttnArgs a = args;
  a.heads = a.B * a.H;
  a.blocks = (a.Tq + 3) / 4;
  const dp_status st = launch_attention(attention_query_grad_f32_kernel, a, 256, 0, s);
  if (st != DP_OK) return st;
  a.heads = a.B * a.H_kv;
  a.blocks = (a.Tk + 3) / 4;
  return launch_attention(attention_key_grad_f32_kernel, a, 256, 0, s);
}

}  // namespace dpbk
