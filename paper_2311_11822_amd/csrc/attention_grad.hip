// Attention, backward.  With p_ij = exp(scale q_i k_j - lse_i) formed again from the forward pass's lse:
//   dv_j = sum_i p_ij do_i,   ds_ij = p_ij (do_i v_j - delta_i),   delta_i = do_i o_i,
//   dq_i = scale sum_j ds_ij k_j,   dk_j = scale sum_i ds_ij q_i     (over the query heads that share the key head, too).
// Two kernels, one that owns queries and one that owns keys, so that every sum has one owner and a fixed order, without atomics.  The price is
// that scores and do v' are formed in both, seven products for five.  Where key heads are too few to fill the device the query heads
// that share one are dealt to several workgroups: their fp32 sums of dk and dv lie in the workspace and a third kernel joins them, in a fixed order
// too.
#include "attention.h"

namespace dpbk {

namespace {

// Both kernels go through tiles of 32 rows of the other side, in two stages, a barrier a tile.  Bound by the turn of a tile, not by the
// matrix cores' rate: its products depend on each other through the exponentials, and registers allow two or three workgroups to a unit to fill the
// gaps.  4 x 2048 causal tokens, 96 heads of 128, bf16: 1520 to 1610 us by card and run (dq 44 % of it), 1.0e12 operations that count (1.4e12 done): 640 to
// 680 TFLOP/s, half of a large product's rate.  8 x 512, 20 heads of 64: 21 and 24 us for the 17 that the tensors take from memory.  fp16's powers of two
// (Raised) take 7 to 9 %: both passes of 4 x 1024 tokens, 12 heads of 64, 57 us, without them 52.
// The key kernel at its full registers keeps 12 (width 64) and 16 bytes (128) of a lane in scratch, fp16 24 and 8.
// Tried without gain: a ring of four stages; the next tile's scores beside the exponentials, as in the forward pass (there are registers for two
// workgroups of width 64 instead of three: 2 x 4096 tokens, 12 heads, 7 % faster at the time, 8 x 512 17 % slower); two and eight waves; one
// wave to a SIMD with 512 registers.
constexpr int kRows = 32;
constexpr int kPartUnits = 256;                   // compute units
// Workgroups to a compute unit, as registers allow; operands asked for ahead: what is left of them.
constexpr int grad_workgroups(int DT, int DP) { return DT == DP_F32 ? (DP <= 64 ? 2 : 1) : DP <= 64 ? 3 : 2; }
constexpr int grad_waves(int DT, int DP, int SPLIT) { return SPLIT == 8 ? 2 : SPLIT > 1 ? 1 : grad_workgroups(DT, DP); }     // to a SIMD
constexpr int grad_ahead(int DT, int DP) { return DT == DP_F32 || DP <= 64 ? 2 : 4; }
// Own keys and values, two sums, scores and their gradients are 224 registers at a width of 128: there the values stay in LDS.
constexpr bool values_in_lds(int DT, int DP) { return DT != DP_F32 && DP == 128; }

// dq, and for the other kernel lse in units of log 2 and delta.  A wave owns 32 queries (SPLIT waves the same ones).
template <int DT, int DP, int NW, int SPLIT>
__global__ void __launch_bounds__(64 * NW * SPLIT, grad_waves(DT, DP, SPLIT))
attention_query_grad_kernel(const AttnArgs a) {
  extern __shared__ __align__(1024) char smem[];
  typedef Ops<DT> O;
  typedef typename O::E E;
  constexpr int KS = HeadTile<DT, DP>::CHUNKS / 2, CB = DP / 32, TILE = SPLIT * kRows * HeadTile<DT, DP>::ROW_BYTES, STAGE = 2 * TILE;
  constexpr int SUB = kRows * HeadTile<DT, DP>::ROW_BYTES;           // one wave's tile of a stage's
  typedef TileLoader<DT, DP, SPLIT * kRows, NW * SPLIT> Loader;
  int pair, block;
  attn_unit(a, a.first + blockIdx.x, pair, block);
  if (pair >= a.heads) return;
  const int b = pair / a.H, h = pair % a.H;
  if (a.causal) block = a.blocks - 1 - block;     // the longest first
  const int lane = threadIdx.x & 63, id = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = id % NW, turn = id / NW;
  const int n_q = valid_rows(a.q_len, b, a.Tq), n_k = valid_rows(a.k_len, b, a.Tk), shift = n_k - n_q;
  const int row0 = block * 32 * NW, own0 = row0 + 32 * wave, row = own0 + (lane & 31);
  const unsigned lds = (unsigned)(uintptr_t)DP_LDS(char, smem);
  const int last = min(row0 + 32 * NW, n_q) - 1, own_last = min(own0 + 32, n_q) - 1;
  const int end = row0 >= n_q ? 0 : a.causal ? min(n_k, last + shift + 1) : n_k;
  const int own_end = own0 >= n_q ? 0 : a.causal ? min(n_k, own_last + shift + 1) : n_k;
  const int lane_end = row >= n_q ? 0 : a.causal ? min(n_k, row + shift + 1) : n_k;
  const int all_see = a.causal ? min(n_k, own0 + shift + 1) : n_k;       // keys that each of the wave's rows sees

  typename O::Row qf[KS], df[KS];
  load_own<DT>(qf, static_cast<const E*>(a.q) + b * a.qs.sample + h * a.qs.head, a.qs.token, row, row < n_q, a.D, lane);
  load_own<DT>(df, static_cast<const E*>(a.dout) + b * a.os.sample + h * a.os.head, a.os.token, row, row < n_q, a.D, lane);
  float delta = 0.f;
  {
    typename O::Row of[KS];
    load_own<DT>(of, static_cast<const E*>(a.o) + b * a.os.sample + h * a.os.head, a.os.token, row, row < n_q, a.D, lane);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int i = 0; i < O::EL; ++i) delta = fmaf(O::get(df[ks], i), O::get(of[ks], i), delta);
    delta += other_half(delta, lane);
  }
  const int64_t at = ((int64_t)b * a.H + h) * a.Tq + row;
  float lse2 = INFINITY;                          // a row that sees nothing
  if (lane_end > 0) {
    lse2 = a.lse[at] * kLog2e;
    if (lse2 == -INFINITY) lse2 = INFINITY;
  }
  if (lane_end <= 0) delta = 0.f;
  // The scores of a row that sees one key have no gradient: zero probabilities here, not what two orders of adding leave.
  const float own_lse2 = lane_end == 1 ? INFINITY : lse2;

  Loader k_tiles, v_tiles;
  k_tiles.init(static_cast<const E*>(a.k) + b * a.ks.sample + h / a.share * a.ks.head, a.ks.token, a.D, id, lane);
  v_tiles.init(static_cast<const E*>(a.v) + b * a.vs.sample + h / a.share * a.vs.head, a.vs.token, a.D, id, lane);
  TileReader<DT, DP> read;
  read.init(lds + turn * SUB, lane);
  auto load = [&](int tile, int stage) {
    const unsigned to = lds + stage * STAGE;
    k_tiles.load(tile * SPLIT * kRows, n_k, to, id);
    v_tiles.load(tile * SPLIT * kRows, n_k, to + TILE, id);
  };
  // Scores, and do v' - delta (the sums begin at -delta).
  auto products = [&](f32x16& s, f32x16& dp, int at, const f32x16& begin) {
    auto operand = [&](int m) { return read.rows(at + m / KS * TILE, 0, m % KS); };
    Stretch<typename O::Row, 2 * KS, grad_ahead(DT, DP)> run;
    run.begin(operand);
    run.run(operand,
            [&](int m, typename O::Row f) {
              const int ks = m % KS;
              if (m < KS)
                s = O::rows(f, qf[ks], ks == 0 ? zeros16() : s);
              else
                dp = O::rows(f, df[ks], ks == 0 ? begin : dp);
            });
  };
  constexpr bool F16 = DT == DP_F16;
  Raised raised;
  auto probability = [&](float s, float raise) { return __builtin_amdgcn_exp2f(fmaf(s, a.scale2, raise - own_lse2)); };      // times 2^raise
  auto hide = [&](f32x16& x, int tile) {          // a select: what is not seen may be no number
    const int seen = lane_end - tile * kRows - 4 * (lane >> 5);
#pragma unroll
    for (int r = 0; r < 16; ++r)
      if (8 * (r >> 2) + (r & 3) >= seen) x[r] = 0.f;
  };

  f32x16 dq[CB], begin;
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) dq[cb] = zeros16();
  const int tiles = (end + SPLIT * kRows - 1) / (SPLIT * kRows), own_tiles = (own_end + kRows - 1) / kRows;
  if (tiles > 0) {
    load(0, 0);
    load(1, 1);
    constexpr bool ROUNDED = DT != DP_F32;        // o is
    if (ROUNDED && end <= 2 * kRows + 32 * NW) tiles_landed();       // some wave's rows may end within two tiles
    if (ROUNDED && own_end <= 2 * kRows) {
      // All that these rows see is at hand: delta from the probabilities, free of o's rounding, which counts where few keys share a
      // row (2-norm of dq's error against 64 bits, fp16, 18 x 591 tokens: 3.1e-4 with o's alone, 3.0e-4 so).
      float sum = 0.f;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        f32x16 s, dp;
        products(s, dp, SPLIT > 1 ? (t - turn) * SUB : t * STAGE, zeros16());
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = probability(s[r], 0.f) * dp[r];
        hide(s, t);
#pragma unroll
        for (int r = 0; r < 16; ++r) sum += s[r];
      }
      sum += other_half(sum, lane);
      if (lane_end > 1) delta = sum;
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) begin[r] = -delta;
  }
  two_stages(tiles, [&](int t, auto stage) {
    constexpr int HERE = decltype(stage)::value;
    tiles_landed();
    if (t > 0 && t + 1 < tiles) load(t + 1, HERE ^ 1);
    const int tile = t * SPLIT + turn;
    if (tile >= own_tiles) return;
    f32x16 s, dp;
    products(s, dp, HERE * STAGE, begin);
    auto operand = [&](int m) { return read.columns(HERE * STAGE, 16 * (m / CB), m % CB); };
    Stretch<typename O::Column, 2 * CB, grad_ahead(DT, DP)> run;
    run.begin(operand);
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = probability(s[r], F16 ? (float)raised.raise : 0.f) * dp[r];
    if ((tile + 1) * kRows > all_see) hide(s, tile);
    typename O::Column ds[2] = {O::weights(s, 0), O::weights(s, 8)};
    if constexpr (F16)
      if (raised.outgrown(ds)) {
        raised.lower(s, dq, lane);
        ds[0] = O::weights(s, 0), ds[1] = O::weights(s, 8);
      }
    run.run(operand, [&](int m, typename O::Column f) { dq[m % CB] = O::columns(f, ds[m / CB], dq[m % CB]); });
  });
  if constexpr (F16) raised.take_out(dq);
  tiles_landed();                                 // LDS is free
  if constexpr (SPLIT > 1) {
    constexpr int EACH = handed_floats(16 * CB);
    float* const mine = reinterpret_cast<float*>(smem) + id * EACH;
    if (turn > 0) hand_over(dq, mine, lane);
    tiles_landed();
    if (turn > 0) return;
#pragma unroll
    for (int w = 1; w < SPLIT; ++w) take_over(dq, mine + w * NW * EACH, lane);
  }
  if (lane < 32 && row < a.Tq) {
    a.lse2[at] = lse2 - kGain<E>;
    a.delta[at] = -delta;
  }
  store_rows<DT, DP>(dq, a.scale, lane_end > 0, static_cast<E*>(a.dq) + b * a.qs.sample + h * a.qs.head, a.qs.token, own0,
                        a.Tq, a.D, lds + wave * 32 * HeadTile<DT, DP>::ROW_BYTES, lane);
  if (a.causal && __any(lane_end > 0 && not_finite(dq))) {
    const AttnRows<E> rows(a, reinterpret_cast<float*>(smem + wave * 32 * HeadTile<DT, DP>::ROW_BYTES), b, h, lane);
    for (int i = own0; i < min(own0 + 32, n_q); ++i) rows.query_gradient(i);
  }
}

// dk and dv.  A wave owns 32 keys (SPLIT waves the same ones); tiles of queries and their output gradients go through LDS, with lse and delta.
template <int DT, int DP, int NW, int SPLIT>
__global__ void __launch_bounds__(64 * NW * SPLIT, grad_waves(DT, DP, SPLIT))
attention_key_grad_kernel(const AttnArgs a) {
  extern __shared__ __align__(1024) char smem[];
  typedef Ops<DT> O;
  typedef typename O::E E;
  constexpr int KS = HeadTile<DT, DP>::CHUNKS / 2, CB = DP / 32, TILE = SPLIT * kRows * HeadTile<DT, DP>::ROW_BYTES, STAGE = 2 * TILE + 512 * SPLIT;
  constexpr int SUB = kRows * HeadTile<DT, DP>::ROW_BYTES;
  constexpr bool V_IN_LDS = values_in_lds(DT, DP);
  typedef TileLoader<DT, DP, SPLIT * kRows, NW * SPLIT> Loader;
  int pair, block;
  attn_unit(a, a.first + blockIdx.x, pair, block);
  if (pair >= a.heads) return;
  // (A unit is a sample, a key head and a part of the query heads that share it.)
  const int part = pair % a.parts, b = pair / a.parts / a.H_kv, h = pair / a.parts % a.H_kv;
  const int heads = a.share / a.parts, q_head = h * a.share + part * heads;
  const int lane = threadIdx.x & 63, id = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = id % NW, turn = id / NW;
  const int n_q = valid_rows(a.q_len, b, a.Tq), n_k = valid_rows(a.k_len, b, a.Tk), shift = n_k - n_q;
  const int key0 = block * 32 * NW, own0 = key0 + 32 * wave, key = own0 + (lane & 31);
  const unsigned lds = (unsigned)(uintptr_t)DP_LDS(char, smem);
  // Queries from here on see a key of the workgroup, of this wave; and the first that sees the lane's.
  const int begin = a.causal ? max(key0 - shift, 0) & ~31 : 0;
  const int own_begin = own0 >= n_k ? INT32_MAX : a.causal ? max(own0 - shift, 0) : 0, lane_begin = a.causal ? key - shift : 0;
  const int tiles = key0 < n_k && begin < n_q ? (n_q - begin + SPLIT * kRows - 1) / (SPLIT * kRows) : 0;       // of one query head

  const int64_t kv = b * a.ks.sample + h * a.ks.head, vv = b * a.vs.sample + h * a.vs.head;
  typename O::Row kf[KS], vf[V_IN_LDS ? 1 : KS];
  load_own<DT>(kf, static_cast<const E*>(a.k) + kv, a.ks.token, key, key < n_k, a.D, lane);
  if constexpr (V_IN_LDS) {
    // Own keys and values, two sums, scores and their gradients are 224 registers at a width of 128: the values stay in LDS.
    TileLoader<DT, DP, 32 * NW, NW * SPLIT> own;
    own.init(static_cast<const E*>(a.v) + vv, a.vs.token, a.D, id, lane);
    own.load(key0, n_k, lds + 2 * STAGE, id);
  } else {
    load_own<DT>(vf, static_cast<const E*>(a.v) + vv, a.vs.token, key, key < n_k, a.D, lane);
  }
  TileReader<DT, DP> read;
  read.init(lds + turn * SUB, lane);
  const unsigned own_values = 2 * STAGE + wave * SUB - turn * SUB;
  Loader q_tiles, d_tiles;
  q_tiles.init(static_cast<const E*>(a.q) + b * a.qs.sample + q_head * a.qs.head, a.qs.token, a.D, id, lane);
  d_tiles.init(static_cast<const E*>(a.dout) + b * a.os.sample + q_head * a.os.head, a.os.token, a.D, id, lane);
  int64_t corr = ((int64_t)b * a.H + q_head) * a.Tq;
  // Tiles of the part's query heads, one behind the other; first row of the one that is loaded next.
  int next_row = begin;
  auto load = [&](int stage) {
    const unsigned to = lds + stage * STAGE;
    q_tiles.load(next_row, n_q, to, id);
    d_tiles.load(next_row, n_q, to + TILE, id);
    const int corr_row = min(next_row + turn * kRows, a.Tq), bytes = 4 * min(a.Tq - corr_row, kRows);
    if (wave == 0)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      i32x4 r = make_rsrc((k ? a.delta : a.lse2) + corr + corr_row, bytes);
#pragma unroll
      for (int i = 0; i < 3; ++i) r[i] = __builtin_amdgcn_readfirstlane(r[i]);
      load_dword_to_lds(r, 4 * lane, to + 2 * TILE + 512 * turn + 256 * k);
    }
    next_row += SPLIT * kRows;
    if (next_row >= n_q) {
      next_row = begin;
      q_tiles.base += O::SIZE * a.qs.head;
      d_tiles.base += O::SIZE * a.os.head;
      corr += a.Tq;
    }
  };
  const unsigned pairs = lds + 2 * TILE + 512 * turn + 16 * (lane >> 5);
  auto four = [&](int at) { return *(__attribute__((address_space(3))) const f32x4*)(uintptr_t)(pairs + at); };
  // Scores, and do v' - delta.
  auto products = [&](f32x16& s, f32x16& dp, int stage) {
    // The operands of LDS in the order of their instructions: Q's rows, then do's (and the values).
    constexpr int PER = V_IN_LDS ? 2 : 1;
    auto operand = [&](int m) {
      const int n = m - KS;
      if (m < KS) return read.rows(stage * STAGE, 0, m);
      return V_IN_LDS && n % PER ? read.rows(own_values, 0, n / PER) : read.rows(stage * STAGE + TILE, 0, n / PER);
    };
    Stretch<typename O::Row, KS + PER * KS, grad_ahead(DT, DP)> run;
    run.begin(operand);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const f32x4 d = four(stage * STAGE + 256 + 32 * g);
#pragma unroll
      for (int i = 0; i < 4; ++i) dp[4 * g + i] = d[i];
    }
    run.run(operand,
            [&](int m, typename O::Row f) {
              const int n = m - KS, ks = m < KS ? m : n / PER;
              if (m < KS)
                s = O::rows(f, kf[ks], ks == 0 ? zeros16() : s);
              else if (!V_IN_LDS)
                dp = O::rows(f, vf[V_IN_LDS ? 0 : ks], dp);
              else if (n % PER)
                dp = O::rows(run.f[m - 1], f, dp);
            });
  };

  f32x16 dk[CB], dv[CB];
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) dk[cb] = dv[cb] = zeros16();
  constexpr bool F16 = DT == DP_F16;
  Raised raised;
  const int steps = tiles * heads;
  if (steps > 0) load(0);
  int first = begin;                              // of the tile at hand
  two_stages(steps, [&](int t, auto stage) {
    constexpr int HERE = decltype(stage)::value;
    tiles_landed();
    if (t + 1 < steps) load(HERE ^ 1);
    const int i0 = first + turn * kRows;
    first = first + SPLIT * kRows < n_q ? first + SPLIT * kRows : begin;
    if (i0 + 31 < own_begin || i0 >= n_q) return;         // no query of the tile sees a key of the wave
    f32x16 p, ds;
    products(p, ds, HERE);
    // Instruction m: columns m / 2 % CB of rows 16 (m / 2 / CB) on, of dv or of dk.
    auto operand = [&](int m) { return read.columns(HERE * STAGE + (m & 1 ? 0 : TILE), 16 * (m / 2 / CB), m / 2 % CB); };
    Stretch<typename O::Column, 4 * CB, grad_ahead(DT, DP)> run;
    run.begin(operand);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const f32x4 l = four(HERE * STAGE + 32 * g);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = 4 * g + i;
        p[r] = __builtin_amdgcn_exp2f(fmaf(p[r], a.scale2, -l[i]));
        ds[r] *= p[r];
      }
    }
    if ((a.causal && i0 < own0 + 31 - shift) || n_k == 1) {
      // The scores of a row that sees one key have no gradient: every row's of a single key, under the mask the first row's.
      const int hidden = lane_begin - i0 - 4 * (lane >> 5);
      const int hidden_ds = n_k == 1 ? INT32_MAX : max(hidden, 1 - shift - i0 - 4 * (lane >> 5));
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int i = 8 * (r >> 2) + (r & 3);
        p[r] = i < hidden ? 0.f : p[r];
        ds[r] = i < hidden_ds ? 0.f : ds[r];
      }
    }
    if constexpr (F16) {
      const float f = raised.factor((int)kGain<E>);
#pragma unroll
      for (int r = 0; r < 16; ++r) ds[r] *= f;
    }
    const typename O::Column pr[2] = {O::weights(p, 0), O::weights(p, 8)};
    typename O::Column dr[2] = {O::weights(ds, 0), O::weights(ds, 8)};
    if constexpr (F16)
      if (raised.outgrown(dr)) {
        raised.lower(ds, dk, lane);
        dr[0] = O::weights(ds, 0), dr[1] = O::weights(ds, 8);
      }
    run.run(operand,
            [&](int m, typename O::Column f) {
              const int cb = m / 2 % CB, ks = m / 2 / CB;
              if (m & 1)
                dk[cb] = O::columns(f, dr[ks], dk[cb]);
              else
                dv[cb] = O::columns(f, pr[ks], dv[cb]);
            });
  });
  if constexpr (F16) {
    raised.take_out(dk);
    Raised::lower_by(dv, (int)kGain<E>);
  }
  tiles_landed();                                 // LDS is free
  if constexpr (SPLIT > 1) {
    constexpr int EACH = handed_floats(32 * CB);
    float* const mine = reinterpret_cast<float*>(smem) + (id - NW) * EACH;
    if (turn > 0) {
      hand_over(dk, mine, lane);
      hand_over(dv, mine + EACH / 2, lane);
    }
    tiles_landed();
    if (turn > 0) return;
#pragma unroll
    for (int w = 1; w < SPLIT; ++w) {
      take_over(dk, mine + w * NW * EACH, lane);
      take_over(dv, mine + w * NW * EACH + EACH / 2, lane);
    }
  }
  float *dk_part = nullptr, *dv_part = nullptr;
  if (a.parts > 1) {
    dk_part = a.partial + (((int64_t)part * a.B + b) * a.H_kv + h) * a.Tk * a.D;
    dv_part = dk_part + (int64_t)a.parts * a.B * a.H_kv * a.Tk * a.D;
    store_partial<DP>(dk, key < n_k, dk_part, key, a.Tk, a.D, lane);
    store_partial<DP>(dv, key < n_k, dv_part, key, a.Tk, a.D, lane);
  } else {
    const unsigned own_rows = lds + wave * 32 * HeadTile<DT, DP>::ROW_BYTES;
    store_rows<DT, DP>(dk, a.scale, key < n_k, static_cast<E*>(a.dk) + kv, a.ks.token, own0, a.Tk, a.D, own_rows, lane);
    store_rows<DT, DP>(dv, 1.f, key < n_k, static_cast<E*>(a.dv) + vv, a.vs.token, own0, a.Tk, a.D, own_rows, lane);
  }
  if (a.causal && __any(key < n_k && (not_finite(dk) || not_finite(dv)))) {
    const AttnRows<E> rows(a, reinterpret_cast<float*>(smem + wave * 32 * HeadTile<DT, DP>::ROW_BYTES), b, h, lane);
    for (int j = own0; j < min(own0 + 32, n_k); ++j) rows.key_gradient(j, q_head, q_head + heads, dk_part, dv_part);
  }
}

// dk and dv from the parts' sums, in their order; four columns a thread.
template <class E>
__global__ void __launch_bounds__(256) attention_join_kernel(const AttnArgs a, int64_t pieces) {
  typedef __attribute__((ext_vector_type(4))) E E4;
  const int64_t id = ((int64_t)a.first + blockIdx.x) * 256 + threadIdx.x;
  if (id >= 2 * pieces) return;
  const bool values = id >= pieces;
  const int64_t at = values ? id - pieces : id, size = 4 * pieces;              // elements of a part
  const float* p = a.partial + (values ? size * a.parts : 0) + 4 * at;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  for (int part = 0; part < a.parts; ++part) sum += *reinterpret_cast<const f32x4*>(p + part * size);
  const int64_t row = 4 * at / a.D;                                             // of [B][H_kv][Tk]
  const int col = (int)(4 * at - row * a.D), j = (int)(row % a.Tk), h = (int)(row / a.Tk % a.H_kv), b = (int)(row / a.Tk / a.H_kv);
  const AttnSide& s = values ? a.vs : a.ks;
  const float f = values ? 1.f : a.scale;
  E4 y;
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = (E)(sum[i] * f);
  *reinterpret_cast<E4*>(static_cast<E*>(values ? a.dv : a.dk) + b * s.sample + h * s.head + j * s.token + col) = y;
}

__global__ void __launch_bounds__(256) attention_query_grad_rows_kernel(const AttnArgs a) {
  int pair, block;
  attn_unit(a, a.first + blockIdx.x, pair, block);
  if (pair >= a.heads) return;
  __shared__ __align__(16) float own[4 * kRowFloats];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = block * 4 + wave;
  const AttnRows<float> rows(a, own + wave * kRowFloats, pair / a.H, pair % a.H, threadIdx.x & 63);
  if (i < a.Tq) rows.query_gradient(i);
}

__global__ void __launch_bounds__(256) attention_key_grad_rows_kernel(const AttnArgs a) {
  int pair, block;
  attn_unit(a, a.first + blockIdx.x, pair, block);
  if (pair >= a.heads) return;
  __shared__ __align__(16) float own[4 * kRowFloats];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), j = block * 4 + wave;
  const AttnRows<float> rows(a, own + wave * kRowFloats, pair / a.H_kv, pair % a.H_kv, threadIdx.x & 63);
  if (j < a.Tk) rows.key_gradient(j, rows.h * a.share, (rows.h + 1) * a.share, nullptr, nullptr);
}

template <int DT, int DP, int NW, int SPLIT>
dp_status launch_queries(AttnArgs a, hipStream_t s) {
  a.heads = a.B * a.H;
  a.blocks = (a.Tq + 32 * NW - 1) / (32 * NW);
  constexpr int LDS = 4 * SPLIT * kRows * HeadTile<DT, DP>::ROW_BYTES;
  auto kernel = attention_query_grad_kernel<DT, DP, NW, SPLIT>;
  static ReadyTable done;
  if (LDS > 65536) {
    const dp_status st = allow_big_lds(kernel, LDS, done);
    if (st != DP_OK) return st;
  }
  return launch_attention(kernel, a, (int64_t)2 * Ops<DT>::SIZE * a.Tk * a.D, 64 * NW * SPLIT, LDS, s);
}

template <int DT, int DP, int NW, int SPLIT>
dp_status launch_keys(AttnArgs a, hipStream_t s) {
  a.heads = a.B * a.H_kv * a.parts;
  a.blocks = (a.Tk + 32 * NW - 1) / (32 * NW);
  constexpr int ROW = HeadTile<DT, DP>::ROW_BYTES;
  constexpr int LDS = 2 * SPLIT * (2 * kRows * ROW + 512) + (values_in_lds(DT, DP) ? 32 * NW * ROW : 0);
  auto kernel = attention_key_grad_kernel<DT, DP, NW, SPLIT>;
  static ReadyTable done;
  dp_status st = DP_OK;
  if (LDS > 65536) st = allow_big_lds(kernel, LDS, done);
  if (st == DP_OK) st = launch_attention(kernel, a, (int64_t)2 * Ops<DT>::SIZE * a.Tq * a.D * (a.share / a.parts), 64 * NW * SPLIT, LDS, s);
  if (st != DP_OK || a.parts == 1) return st;
  const int64_t pieces = (int64_t)a.B * a.H_kv * a.Tk * a.D / 4;
  return launch_in_runs((2 * pieces + 255) / 256, [&](dim3 grid, int first) {
    AttnArgs run = a;
    run.first = (unsigned)first;
    hipLaunchKernelGGL(attention_join_kernel<typename Ops<DT>::E>, grid, dim3(256), 0, s, run, pieces);
  });
}

template <int DT, int DP>
dp_status launch(const AttnArgs& a, hipStream_t s) {
  constexpr int SPLIT = split_waves(HeadTile<DT, DP>::ROW_BYTES);
  // (One wave for few rows: 512 x 32 tokens, 12 heads of 64: 64 us, with four 95.)
  const dp_status st = split_queries<DT, DP>(a) ? launch_queries<DT, DP, 1, SPLIT>(a, s)
                       : a.Tq <= 32             ? launch_queries<DT, DP, 1, 1>(a, s)
                                                : launch_queries<DT, DP, 4, 1>(a, s);
  if (st != DP_OK) return st;
  if (split_keys<DT, DP>(a)) return launch_keys<DT, DP, 1, SPLIT>(a, s);
  return a.Tk <= 32 ? launch_keys<DT, DP, 1, 1>(a, s) : launch_keys<DT, DP, 4, 1>(a, s);
}

template <int DT>
dp_status launch(const AttnArgs& a, hipStream_t s) {
  return by_head_width<DT>(a.D, [&](auto width) { return launch<DT, decltype(width)::value>(a, s); });
}

template <int DT>
void tile_rows(const AttnArgs& a, int& queries, int& keys) {
  by_head_width<DT>(a.D, [&](auto width) {
    constexpr int DP = decltype(width)::value, SPLIT = split_waves(HeadTile<DT, DP>::ROW_BYTES);
    queries = kRows * (split_queries<DT, DP>(a) ? SPLIT : 1);
    keys = kRows * (split_keys<DT, DP>(a) ? SPLIT : 1);
  });
}

}  // namespace

// Where key heads are few, a workgroup to each of their blocks leaves compute units idle while it goes through its query heads one after the
// other: these are dealt to several, in as many parts as fill the units, whose sums are then joined.  2 x 128 tokens, fp32, 48 heads of
// 128 that share 6: 312 us in one part.
int attention_parts(const AttnArgs& a) {
  const int64_t units = (int64_t)a.B * a.H_kv * ((a.Tk + 127) / 128);
  int parts = 1;
  for (int p = 2; p <= a.share && units * parts < kPartUnits; ++p)
    if (a.share % p == 0) parts = p;
  return parts;
}

int64_t attention_partial_floats(const AttnArgs& a) {
  const int parts = attention_parts(a);
  return parts > 1 ? (int64_t)2 * parts * a.B * a.H_kv * a.Tk * a.D : 0;
}

void attention_backward_tiles(const AttnArgs& a, dp_dtype dt, int& queries, int& keys) {
  queries = keys = 1;
  if (dt != DP_F32)
    tile_rows<DP_BF16>(a, queries, keys);
  else if (whole_pieces(a))
    tile_rows<DP_F32>(a, queries, keys);
}

dp_status launch_attention_backward(const AttnArgs& args, dp_dtype dt, hipStream_t s) {
  if (dt == DP_BF16) return launch<DP_BF16>(args, s);
  if (dt == DP_F16) return launch<DP_F16>(args, s);
  if (whole_pieces(args)) return launch<DP_F32>(args, s);
  AttnArgs a = args;
  a.heads = a.B * a.H;
  a.blocks = (a.Tq + 3) / 4;
  const dp_status st = launch_attention(attention_query_grad_rows_kernel, a, (int64_t)8 * a.Tk * a.D, 256, 0, s);
  if (st != DP_OK) return st;
  a.heads = a.B * a.H_kv;
  a.blocks = (a.Tk + 3) / 4;
  return launch_attention(attention_key_grad_rows_kernel, a, (int64_t)8 * a.Tq * a.D * a.share, 256, 0, s);
}

}  // namespace dpbk
