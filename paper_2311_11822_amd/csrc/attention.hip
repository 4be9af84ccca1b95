// Attention, forward: o_i = sum_j p_ij v_j with p_ij = exp(scale q_i k_j - lse_i) over the keys j that row i sees, in one pass over keys and
// values with a running maximum and sum.
#include "attention.h"

#include <algorithm>

namespace dpbk {

namespace {

constexpr float kLazy = 8.f;                      // a maximum may be passed by 2^8 before sums are expressed in a new one

// NW waves of 32 queries each (SPLIT waves the same ones, whose turns at the tiles are joined at the end), tiles of KEYS keys in two stages.
// A pair's keys and values come out of L2 for all blocks but the first; what is left is work on scores: four matrix instructions a tile for
// D = 64 and as many issue cycles of exponentials, maxima and roundings beside them, with a barrier a tile, three workgroups to a
// unit.  2 x 4096 causal tokens, 12 heads of 64, bf16: 70 to 75 us by card and run, 690 to 740 TFLOP/s of the 1400 of a large product.  16 x 256: 10 us and 32 x 197
// (fp16, all seen) 14 to 15 us for the 5 and 8 that q, k, v and o take from memory: a launch, and a workgroup's loads, few tiles and stores one after
// the other.  Tried without gain: four stages, two and eight waves, operands asked for ahead in a fixed order.
template <int DT, int DP, int NW, int SPLIT, int KEYS>
__global__ void __launch_bounds__(64 * NW * SPLIT, 2) attention_kernel(const AttnArgs a) {
  extern __shared__ __align__(1024) char smem[];
  typedef Ops<DT> O;
  typedef typename O::E E;
  constexpr int KS = HeadTile<DT, DP>::CHUNKS / 2, CB = DP / 32, KB = KEYS / 32, TILE = SPLIT * KEYS * HeadTile<DT, DP>::ROW_BYTES;
  constexpr int V = 2 * TILE;                     // two stages of keys, then two of values
  int pair, block;
  attn_unit(a, a.first + blockIdx.x, pair, block);
  if (pair >= a.heads) return;
  const int b = pair / a.H, h = pair % a.H;
  if (a.causal) block = a.blocks - 1 - block;     // the longest first
  const int part = SPLIT > 1 ? block % a.key_parts : 0;
  if (SPLIT > 1) block /= a.key_parts;
  const int part_begin = SPLIT > 1 ? part * a.part_keys : 0;
  const int lane = threadIdx.x & 63, id = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = id % NW, turn = id / NW;
  const int n_q = valid_rows(a.q_len, b, a.Tq), n_k = valid_rows(a.k_len, b, a.Tk), shift = n_k - n_q;
  const int row0 = block * 32 * NW, own0 = row0 + 32 * wave, row = own0 + (lane & 31);
  const unsigned lds = (unsigned)(uintptr_t)DP_LDS(char, smem);

  // Keys that the workgroup's, this wave's and the lane's rows see: below these.
  const int last = min(row0 + 32 * NW, n_q) - 1, own_last = min(own0 + 32, n_q) - 1;
  const int there_k = SPLIT > 1 ? min(n_k, part_begin + a.part_keys) : n_k;         // (the part's)
  const int end = row0 >= n_q ? 0 : a.causal ? min(there_k, last + shift + 1) : there_k;
  const int own_end = own0 >= n_q ? 0 : a.causal ? min(there_k, own_last + shift + 1) : there_k;
  const int lane_end = row >= n_q ? 0 : a.causal ? min(n_k, row + shift + 1) : n_k;

  const E* q = static_cast<const E*>(a.q) + b * a.qs.sample + h * a.qs.head;
  TileLoader<DT, DP, SPLIT * KEYS, NW * SPLIT> k_tiles, v_tiles;
  k_tiles.init(static_cast<const E*>(a.k) + b * a.ks.sample + h / a.share * a.ks.head, a.ks.token, a.D, id, lane);
  v_tiles.init(static_cast<const E*>(a.v) + b * a.vs.sample + h / a.share * a.vs.head, a.vs.token, a.D, id, lane);
  // A tile's scores are formed beside the exponentials of the tile before it, so its keys are loaded a step before its values.
  auto load_keys = [&](int tile, int stage) { k_tiles.load(part_begin + tile * SPLIT * KEYS, there_k, lds + stage * TILE, id); };
  auto load_values = [&](int tile, int stage) { v_tiles.load(part_begin + tile * SPLIT * KEYS, there_k, lds + V + stage * TILE, id); };
  const int tiles = (max(end - part_begin, 0) + SPLIT * KEYS - 1) / (SPLIT * KEYS);
  if (tiles > 0) {
    load_keys(0, 0);
    if (tiles > 1) load_keys(1, 1);
    load_values(0, 0);
  }
  typename O::Row qf[KS];
  load_own<DT>(qf, q, a.qs.token, row, row < n_q, a.D, lane);
  have(qf);
  TileReader<DT, DP> read;
  read.init(lds + turn * KEYS * HeadTile<DT, DP>::ROW_BYTES, lane);

  f32x16 o[CB];
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) o[cb] = zeros16();
  float most = -3.4028235e38f, total = 0.f;       // of scale2 * score; total: of this half's keys
  auto scores = [&](f32x16 (&to)[KB], int tile) {
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      to[kb] = zeros16();
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) to[kb] = O::rows(read.rows(tile, 32 * kb, ks), qf[ks], to[kb]);
    }
  };
  const int all_see = a.causal ? min(n_k, own0 + shift + 1) : n_k;       // keys that each of the wave's rows sees
  f32x16 both[2][KB];
  if (tiles > 0) {
    tiles_landed();
    scores(both[0], 0);                           // (the next barrier says that all waves are through with these keys)
  }
  two_stages(tiles, [&](int t, auto stage) {
    constexpr int HERE = decltype(stage)::value, NEXT = HERE ^ 1;
    f32x16(&s)[KB] = both[HERE], (&next)[KB] = both[NEXT];
    const int j0 = part_begin + (t * SPLIT + turn) * KEYS;
    tiles_landed();
    if (t + 2 < tiles) load_keys(t + 2, HERE);
    if (t + 1 < tiles) load_values(t + 1, NEXT);
    if (j0 >= own_end) return;
    if (j0 + KEYS > all_see) {
      const int seen = lane_end - j0 - 4 * (lane >> 5);
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (32 * kb + 8 * (r >> 2) + (r & 3) >= seen) s[kb][r] = -INFINITY;
    }
    float top = s[0][0];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
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
    scores(next, NEXT * TILE);                    // (behind the last tile: of what LDS holds, and not used)
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[kb][r] = __builtin_amdgcn_exp2f(fmaf(s[kb][r], a.scale2, -most));
        total += s[kb][r];
      }
#pragma unroll
    for (int ks = 0; ks < KEYS / 16; ++ks) {
      const typename O::Column p = O::weights(s[ks >> 1], 8 * (ks & 1));
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) o[cb] = O::columns(read.columns(V + HERE * TILE, 16 * ks, cb), p, o[cb]);
    }
  });
  total += other_half(total, lane);
  if constexpr (SPLIT > 1) {
    constexpr int EACH = handed_floats(16 * CB + 2);
    float* const mine = reinterpret_cast<float*>(smem) + id * EACH;
    tiles_landed();
    if (turn > 0) {
      hand_over(o, mine, lane);
      mine[16 * CB * 64 + lane] = most;
      mine[(16 * CB + 1) * 64 + lane] = total;
    }
    tiles_landed();
    if (turn > 0) return;
#pragma unroll
    for (int w = 1; w < SPLIT; ++w) {
      const float* theirs = mine + w * NW * EACH;
      const float higher = fmaxf(most, theirs[16 * CB * 64 + lane]);
      const float fix = __builtin_amdgcn_exp2f(most - higher), their_fix = __builtin_amdgcn_exp2f(theirs[16 * CB * 64 + lane] - higher);
      most = higher;
      total = total * fix + theirs[(16 * CB + 1) * 64 + lane] * their_fix;
#pragma unroll
      for (int cb = 0; cb < CB; ++cb)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[cb][r] = o[cb][r] * fix + theirs[(16 * cb + r) * 64 + lane] * their_fix;
    }
  }
  const bool there = lane_end > 0 && total != 0.f;
  if (SPLIT > 1 && a.key_parts > 1) {
    const int64_t rows = (int64_t)part * a.B * a.H * a.Tq + (int64_t)pair * a.Tq;
    store_partial<DP>(o, there, a.partial + rows * a.D, row, a.Tq, a.D, lane);
    float* stats = a.partial + (int64_t)a.key_parts * a.B * a.H * a.Tq * a.D + 2 * (rows + row);
    if (lane < 32 && row < a.Tq) {
      stats[0] = most;
      stats[1] = there ? total : 0.f;
    }
    return;
  }
  if (SPLIT == 1) tiles_landed();                 // LDS is free
  store_rows<DT, DP>(o, 1.f / total, there, static_cast<E*>(a.out) + b * a.os.sample + h * a.os.head, a.os.token, own0,
                        a.Tq, a.D, lds + wave * 32 * HeadTile<DT, DP>::ROW_BYTES, lane);
  if (lane < 32 && row < a.Tq)
    a.lse[((int64_t)b * a.H + h) * a.Tq + row] = there ? most * kLn2 + logf(total) : -INFINITY;
  // A zero probability times an infinity is no number: rows beside a token that they do not see.
  if (a.causal && __any(there && (not_finite(o) || !(fabsf(total) < INFINITY)))) {
    const AttnRows<E> rows(a, reinterpret_cast<float*>(smem + wave * 32 * HeadTile<DT, DP>::ROW_BYTES), b, h, lane);
    for (int i = own0; i < min(own0 + 32, n_q); ++i) rows.forward(i);
  }
}

// Rows from the sums of their parts, in their order; four to a workgroup, columns lane and lane + 64 to a lane.
template <class E>
__global__ void __launch_bounds__(256) attention_join_parts_kernel(const AttnArgs a) {
  __shared__ __align__(16) float own[4 * kRowFloats];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t row = ((int64_t)a.first + blockIdx.x) * 4 + wave, rows = (int64_t)a.B * a.H * a.Tq;
  if (row >= rows) return;
  const float* stats = a.partial + a.key_parts * rows * a.D;
  float most = -3.4028235e38f, total = 0.f, acc[2] = {0.f, 0.f};
  for (int p = 0; p < a.key_parts; ++p) most = fmaxf(most, stats[2 * (p * rows + row)]);
  for (int p = 0; p < a.key_parts; ++p) {
    const int64_t at = p * rows + row;
    const float fix = __builtin_amdgcn_exp2f(stats[2 * at] - most);
    total = fmaf(stats[2 * at + 1], fix, total);
#pragma unroll
    for (int c = 0; c < 2; ++c)
      if (lane + 64 * c < a.D) acc[c] = fmaf(a.partial[at * a.D + lane + 64 * c], fix, acc[c]);
  }
  const int pair = (int)(row / a.Tq), i = (int)(row - (int64_t)pair * a.Tq), b = pair / a.H, h = pair % a.H;
  if (a.causal && __any(!(fabsf(total) < INFINITY) || !(fabsf(acc[0]) < INFINITY) || !(fabsf(acc[1]) < INFINITY))) {
    AttnRows<E>(a, own + wave * kRowFloats, b, h, lane).forward(i);
    return;
  }
  store_row(acc, total != 0.f ? 1.f / total : 0.f, static_cast<E*>(a.out) + b * a.os.sample + h * a.os.head + i * a.os.token, a.D, lane);
  if (lane == 0) a.lse[row] = total != 0.f ? most * kLn2 + logf(total) : -INFINITY;
}

// fp32 rows of no whole 16-byte pieces, four to a workgroup.
__global__ void __launch_bounds__(256) attention_rows_kernel(const AttnArgs a) {
  int pair, block;
  attn_unit(a, a.first + blockIdx.x, pair, block);
  if (pair >= a.heads) return;
  __shared__ __align__(16) float own[4 * kRowFloats];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i = block * 4 + wave;
  const AttnRows<float> rows(a, own + wave * kRowFloats, pair / a.H, pair % a.H, threadIdx.x & 63);
  if (i < a.Tq) rows.forward(i);
}

template <int DT, int DP, int NW, int SPLIT, int KEYS>
dp_status launch(AttnArgs a, hipStream_t s) {
  a.heads = a.B * a.H;
  a.blocks = (a.Tq + 32 * NW - 1) / (32 * NW) * (SPLIT > 1 ? a.key_parts : 1);
  constexpr int LDS = 4 * SPLIT * KEYS * HeadTile<DT, DP>::ROW_BYTES;
  auto kernel = attention_kernel<DT, DP, NW, SPLIT, KEYS>;
  static ReadyTable done;
  if (LDS > 65536) {
    const dp_status st = allow_big_lds(kernel, LDS, done);
    if (st != DP_OK) return st;
  }
  const dp_status st = launch_attention(kernel, a, (int64_t)2 * Ops<DT>::SIZE * a.Tk * a.D, 64 * NW * SPLIT, LDS, s);
  if (SPLIT == 1 || a.key_parts == 1 || st != DP_OK) return st;
  return launch_in_runs(((int64_t)a.heads * a.Tq + 3) / 4, [&](dim3 grid, int first) {
    AttnArgs run = a;
    run.first = (unsigned)first;
    hipLaunchKernelGGL(attention_join_parts_kernel<typename Ops<DT>::E>, grid, dim3(256), 0, s, run);
  });
}

// Calls f with waves, waves on the same rows and keys to a tile.
template <int DT, int DP, class F>
auto by_form(const AttnArgs& a, F f) {
  using std::integral_constant;
  constexpr int LONG = DT == DP_F32 ? 32 : 64;
  const integral_constant<int, 1> one{};
  const integral_constant<int, 2> two{};
  const integral_constant<int, 4> four{};
  const integral_constant<int, 32> tile{};
  if (split_queries<DT, DP>(a)) return f(one, integral_constant<int, split_waves(HeadTile<DT, DP>::ROW_BYTES)>{}, tile);
  // One wave for few queries (512 x 32 tokens, 12 heads of 64: 20 us, with four 40), two up to 64 (256 x 48: 17 and 24).  Tiles of 64 keys hide
  // more of a turn's latency (1 x 3000 tokens, 9 heads: 39 us, of 32 keys 48), but leave more of a short row's last tile empty (64 x 128: 13.7 and
  // 12.4; 32 x 197 14.7 and 13.8; 18 x 591 34 and 36).
  if (a.Tq <= 32) return f(one, one, tile);
  if (a.Tq <= 64) return f(two, one, tile);
  if (a.Tk <= 256) return f(four, one, tile);
  return f(four, one, integral_constant<int, LONG>{});
}

template <int DT>
dp_status launch(const AttnArgs& a, hipStream_t s) {
  return by_head_width<DT>(a.D, [&](auto width) {
    constexpr int DP = decltype(width)::value;
    return by_form<DT, DP>(a, [&](auto waves, auto split, auto keys) {
      return launch<DT, DP, decltype(waves)::value, decltype(split)::value, decltype(keys)::value>(a, s);
    });
  });
}

template <int DT>
int tile_rows(const AttnArgs& a) {
  return by_head_width<DT>(a.D, [&](auto width) {
    return by_form<DT, decltype(width)::value>(a, [](auto, auto split, auto keys) { return split * keys; });
  });
}

template <int DT>
bool queries_are_split(const AttnArgs& a) {
  return by_head_width<DT>(a.D, [&](auto width) { return split_queries<DT, decltype(width)::value>(a); });
}

}  // namespace

// Where split blocks of queries are still few, their keys are dealt to as many workgroups as fill the compute units, from 512 keys to each; the
// sums are joined.  One query, 32 heads of 128 on 8, 32768 keys: 88 us, in one part 303; 8 heads of 64, 4096 keys: 15.6 and 20.1; fp32, 4 heads of
// 32: 17 and 49.  Below four parts it is not worth the second launch (300 queries, 6 heads, 2000 keys in three: 15.0 and 14.1).
void attention_key_parts(AttnArgs& a, dp_dtype dt) {
  const int64_t heads = (int64_t)a.B * a.H, workgroups = heads * ((a.Tq + 31) / 32);
  a.key_parts = 1;
  a.part_keys = a.Tk;
  if (!(dt == DP_F32 ? whole_pieces(a) && queries_are_split<DP_F32>(a) : queries_are_split<DP_BF16>(a))) return;
  const int64_t parts = std::min<int64_t>(256 / workgroups, a.Tk / 512);
  if (parts < 4) return;
  a.part_keys = (int)((a.Tk + parts - 1) / parts + 255) / 256 * 256;            // whole turns of every form
  a.key_parts = (a.Tk + a.part_keys - 1) / a.part_keys;
}

int64_t attention_key_floats(const AttnArgs& a) {
  return a.key_parts > 1 ? (int64_t)a.key_parts * a.B * a.H * a.Tq * (a.D + 2) : 0;
}

int attention_forward_tile(const AttnArgs& a, dp_dtype dt) {
  return dt != DP_F32 ? tile_rows<DP_BF16>(a) : whole_pieces(a) ? tile_rows<DP_F32>(a) : 1;
}

dp_status launch_attention_forward(const AttnArgs& args, dp_dtype dt, hipStream_t s) {
  if (dt == DP_BF16) return launch<DP_BF16>(args, s);
  if (dt == DP_F16) return launch<DP_F16>(args, s);
  if (whole_pieces(args)) return launch<DP_F32>(args, s);
  AttnArgs a = args;
  a.heads = a.B * a.H;
  a.blocks = (a.Tq + 3) / 4;
  return launch_attention(attention_rows_kernel, a, (int64_t)8 * a.Tk * a.D, 256, 0, s);
}

}  // namespace dpbk
