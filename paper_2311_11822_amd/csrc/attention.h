// What the attention kernels share: arguments, the order of their workgroups, key and value tiles on their way into LDS, and the
// row-wise form in fp32.
//
// Operands on the matrix cores.  A wave holds its 32 rows of one side (queries; in the key gradients, keys) as the second
// operand in registers, and the tiles of the other side go through LDS.  A product's 32 x 32 result has that side's index in
// the register (8 (r / 4) + 4 (lane / 32) + r % 4) and the wave's own row in the lane (lane % 32), so that
//  * a softmax over keys is a reduction within a lane and one exchange between its halves, and maxima, sums and their
//    corrections are one value a lane;
//  * sixteen such values, rounded to 16 bits (fp32: as they are), are the second operand of the next product as they lie: lane half h holds
//    rows 4 h .. 4 h + 3 and 8 + 4 h .. 8 + 4 h + 3 of every 16.  A sum does not care for its order, so the first operand is
//    read in the same one (two transposing LDS reads, of rows 4 h and 8 + 4 h on), and no probability passes through LDS.
// Rounding a probability or a score's gradient to the type costs half a unit of it, independently of the others: as much as the result's own
// rounding; sums, maxima, lse and delta are fp32.  fp16 has that unit from 2^-14 to 65504 only, which scores' gradients leave at both ends: they
// are held times a power of two (Raised).  So are the key gradients' probabilities (kGain), which are 1 / n in a row of n equal scores; the forward
// pass has them in units of the largest.
//
// LDS holds rows of a head (DP columns) as they come from memory, 16-byte chunks XOR-swizzled by row such that eight
// rows' reads of one column and the transposing reads of four rows fall on different banks.
#pragma once

#include <type_traits>

#include "dp_internal.h"
#include "lds_dma.h"

namespace dpbk {

struct AttnSide {                 // element strides of sample, token and head
  int64_t sample, token, head;
};

struct AttnArgs {
  const void *q, *k, *v, *o, *dout;
  void *out, *dq, *dk, *dv;
  float* lse;                     // [B, H, Tq]
  float *lse2, *delta;            // backward, [B, H, Tq]: lse in units of log 2, less kGain (+inf: the row counts for nothing), and -delta
  const int32_t *q_len, *k_len;   // [B] or null
  int B, H, H_kv, share;          // share: query heads to a key head
  int Tq, Tk, D;
  int causal;
  int parts;                      // key gradients: the query heads of a key head are dealt to this many workgroups
  float* partial;                 // parts > 1: [2 (dk, dv)][parts][B][H_kv][Tk][D]; key_parts > 1: [key_parts][B][H][Tq][D], then maximum and sum
  int key_parts, part_keys;       // forward: the keys of a block of queries are dealt to this many workgroups, so many to each
  float scale, scale2;            // scale2: scale * log2(e)
  AttnSide qs, ks, vs, os;
  int heads, blocks;              // of the launch: (sample, head) pairs and their blocks of rows
  int spread, group;              // attn_unit
  unsigned first;                 // number of the launch's first workgroup
};

// Arrays that begin at 16 bytes (16-bit ones always do).
__host__ __device__ inline bool aligned_arrays(const AttnArgs& a) {
  return ((uintptr_t)a.q & 15) == 0 && ((uintptr_t)a.k & 15) == 0 && ((uintptr_t)a.v & 15) == 0 && ((uintptr_t)a.o & 15) == 0 &&
         ((uintptr_t)a.out & 15) == 0 && ((uintptr_t)a.dout & 15) == 0 && ((uintptr_t)a.dq & 15) == 0 &&
         ((uintptr_t)a.dk & 15) == 0 && ((uintptr_t)a.dv & 15) == 0;
}

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// What the key gradients' kernel has of probabilities: them times 2^kGain, at most 2^15 in fp16.  (4 queries on 60000 keys: the 2-norm of dv's error
// 6.7e-4 without, 2.9e-4 with it.)
template <class E>
constexpr float kGain = std::is_same_v<E, _Float16> ? 15.f : 0.f;

// Operands and products by storage type DT.  A row operand is 16 bytes of a row, EL columns to each lane half: one matrix instruction of
// 16-bit values, four of fp32.  A column operand is 16 rows of a column, 8 to each half, against eight weights a lane: one instruction, or
// eight (whose two halves are the two rows that it adds, in the order in which the weights lie anyway).
typedef __attribute__((ext_vector_type(8))) float f32x8;
template <int DT>
struct Ops {
  static constexpr bool F16 = DT == DP_F16;
  static constexpr int EL = 8, SIZE = 2;
  typedef bf16x8 Row;
  typedef bf16x8 Column;
  typedef std::conditional_t<F16, _Float16, __bf16> E;
  __device__ static __forceinline__ f32x16 rows(Row a, Row b, f32x16 c) { return mfma16<F16>(a, b, c); }
  __device__ static __forceinline__ f32x16 columns(Column a, Column w, f32x16 c) { return mfma16<F16>(a, w, c); }
  // Eight values rounded to nearest even.
  __device__ static __forceinline__ Column weights(const f32x16& x, int first) {
    typedef __attribute__((ext_vector_type(8))) E E8;
    E8 y;
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = (E)x[first + i];
    return __builtin_bit_cast(bf16x8, y);
  }
  __device__ static __forceinline__ float get(Row x, int i) {
    typedef __attribute__((ext_vector_type(8))) E E8;
    return (float)__builtin_bit_cast(E8, x)[i];
  }
};
template <>
struct Ops<DP_F32> {
  static constexpr int EL = 4, SIZE = 4;
  typedef f32x4 Row;
  typedef f32x8 Column;
  typedef float E;
  __device__ static __forceinline__ f32x16 rows(Row a, Row b, f32x16 c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], c, 0, 0, 0);
    return c;
  }
  __device__ static __forceinline__ f32x16 columns(Column a, Column w, f32x16 c) {
#pragma unroll
    for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], w[i], c, 0, 0, 0);
    return c;
  }
  __device__ static __forceinline__ Column weights(const f32x16& x, int first) {
    Column y;
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = x[first + i];
    return y;
  }
  __device__ static __forceinline__ float get(Row x, int i) { return x[i]; }
};

template <int DT, int DP>
struct HeadTile {
  static constexpr int EL = Ops<DT>::EL, CHUNKS = DP / EL, ROW_BYTES = Ops<DT>::SIZE * DP;
  // A 128-bit read takes sixteen lanes at a time, rows of sixteen different row % 16 here, and a transposing one four rows of 64 bytes: the
  // first must differ in all of row % 16 that one line of the banks holds, the second in the 64-byte group.
  __device__ static constexpr unsigned swizzle(unsigned row) {
    return ROW_BYTES % 256 == 0   ? (row & 3) << 2 | ((row >> 2) & 3)
           : ROW_BYTES == 128 ? (row & 2) << 1 | ((row >> 2) & 3)
                              : (row >> 2) & 3;
  }
};

// Valid rows of sample b: a length beyond the tensor's, or below zero, counts as the nearest that is none.
__device__ __forceinline__ int valid_rows(const int32_t* len, int b, int T) { return len ? min(max(len[b], 0), T) : T; }

// (sample and head, block) of workgroup id; a unit past the last pair comes out at or past a.heads.  With `spread` a pair's blocks go to
// one XCD (id % 8), whose L2 then holds its keys and values.  Pairs come in groups of a.group (to an XCD): the group's block 0, its block 1 ...,
// so that under a causal mask, with the longest as block 0, the units that get a short one last are those that had much before.
__device__ __forceinline__ void attn_unit(const AttnArgs& a, unsigned id, int& pair, int& block) {
  const unsigned i = a.spread ? id >> 3 : id, per_group = (unsigned)(a.group * a.blocks), g = i / per_group, rest = i - g * per_group;
  const unsigned left = (unsigned)(a.spread ? a.heads / 8 + (a.heads % 8 != 0) : a.heads) - g * a.group;
  const unsigned size = left < (unsigned)a.group ? left : (unsigned)a.group;       // of this group
  block = (int)(rest / size);
  pair = (int)(g * a.group + rest - block * size);
  if (a.spread) pair = 8 * pair + (int)(id & 7);
  pair = __builtin_amdgcn_readfirstlane(pair);    // (the divisions run on the vector side)
  block = __builtin_amdgcn_readfirstlane(block);
}

// ROWS rows of a head from memory to LDS, one 16-byte chunk a lane and load, NW waves.  Rows past the descriptor's size and columns from D on
// arrive as zeros.
template <int DT, int DP, int ROWS, int NW>
struct TileLoader {
  typedef HeadTile<DT, DP> H;
  static constexpr int CHUNKS = H::CHUNKS, WAVE_LOADS = ROWS * CHUNKS / 64, LOADS = (WAVE_LOADS + NW - 1) / NW;
  static_assert(WAVE_LOADS * 64 == ROWS * CHUNKS, "whole loads");
  // Every wave makes the same number of loads: where they are more than a tile needs, some are made twice.
  __device__ static int slot(int i, int wave) { return WAVE_LOADS % NW == 0 ? i * NW + wave : (i * NW + wave) % WAVE_LOADS; }
  unsigned off[LOADS];
  uint64_t base;
  unsigned row_bytes;
  __device__ __forceinline__ void init(const void* head, int64_t token_stride, int D, int wave, int lane) {
    base = reinterpret_cast<uint64_t>(head);
    row_bytes = (unsigned)(Ops<DT>::SIZE * token_stride);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const unsigned id = slot(i, wave) * 64 + lane, row = id / CHUNKS, chunk = (id % CHUNKS) ^ H::swizzle(row);
      off[i] = (int)chunk * H::EL < D ? row * row_bytes + chunk * 16 : OOB;
    }
  }
  // Rows row0 .. row0 + ROWS - 1 of which those below `end` are there.
  __device__ __forceinline__ void load(int row0, int end, unsigned lds, int wave) const {
    i32x4 r = make_rsrc(reinterpret_cast<const void*>(base + (uint64_t)row0 * row_bytes), min(max(end - row0, 0), ROWS) * row_bytes);
#pragma unroll
    for (int i = 0; i < 3; ++i) r[i] = __builtin_amdgcn_readfirstlane(r[i]);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) load_to_lds(r, off[i], 0, lds + slot(i, wave) * 1024);
  }
};

// All loads into LDS issued so far have landed, here and (after the barrier) in the other waves; and every wave is through with its
// reads so far.
__device__ __forceinline__ void tiles_landed() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// Where in LDS a lane finds its operands of a tile that begins at `lds`, worked out once: a tile elsewhere is a constant in the instruction.
template <int DT, int DP>
struct TileReader {
  typedef HeadTile<DT, DP> H;
  static constexpr int KS = H::CHUNKS / 2, CB = DP / 32, ROW_BYTES = H::ROW_BYTES, COLUMNS = DT == DP_F32 ? 4 : 2 * CB;
  unsigned row_at[KS], column_at[COLUMNS];
  __device__ __forceinline__ void init(unsigned lds, int lane) {
    const unsigned row = lane & 31, h = lane >> 5;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) row_at[ks] = lds + row * ROW_BYTES + ((2 * ks + h) ^ H::swizzle(row)) * 16;
    if constexpr (DT == DP_F32) {
      // row 8 (e / 4) + 4 h + e % 4 is swizzled by h and by what e alone says: four addresses, the rest is constant
#pragma unroll
      for (int n = 0; n < COLUMNS; ++n) column_at[n] = lds + 4 * h * ROW_BYTES + ((row >> 2) ^ h ^ 2 * n) * 16 + (row & 3) * 4;
    } else {
      const int s = lane & 15, blk = lane >> 4;
      const unsigned first = 4 * (blk >> 1) + (s >> 2);
#pragma unroll
      for (int cb = 0; cb < CB; ++cb)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const unsigned chunk = 4 * cb + 2 * (blk & 1) + ((s & 3) >> 1);
          column_at[2 * cb + i] = lds + (first + 8 * i) * ROW_BYTES + (chunk ^ H::swizzle(first + 8 * i)) * 16 + 8 * (s & 1);
        }
    }
  }
  // Rows row0 + lane % 32 (row0: a multiple of 32), columns 2 EL ks + EL h .. (h = lane / 32) of the tile at byte `tile`.
  __device__ __forceinline__ typename Ops<DT>::Row rows(int tile, int row0, int ks) const {
    return *(__attribute__((address_space(3))) const typename Ops<DT>::Row*)(uintptr_t)(row_at[ks] + tile + row0 * ROW_BYTES);
  }
  // Column 32 cb + lane % 32, rows row0 + 4 h .. + 3 and row0 + 8 + 4 h .. + 3 (row0: of 16).
  __device__ __forceinline__ typename Ops<DT>::Column columns(int tile, int row0, int cb) const {
    if constexpr (DT == DP_F32) {
      f32x8 f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const unsigned fixed = H::swizzle(8 * (e >> 2) + (e & 3));
        f[e] = *(__attribute__((address_space(3))) const float*)(uintptr_t)(column_at[(fixed & 7) >> 1] + tile +
                                                                           (row0 + 8 * (e >> 2) + (e & 3)) * ROW_BYTES +
                                                                           ((8 * cb) ^ (fixed & 8)) * 16);
      }
      return f;
    } else {
      Frag f;
#pragma unroll
      for (int i = 0; i < 2; ++i) f.h[i] = lds_read_tr(column_at[2 * cb + i] + tile + row0 * ROW_BYTES);
      return f.v;
    }
  }
};

// N matrix instructions whose operands are asked for AHEAD instructions before.  The order is fixed here: left to itself the compiler
// reads an operand right before its use and waits for LDS each time.  begin() may come early, with other work behind it.
template <class Operand, int N, int AHEAD_>
struct Stretch {
  static constexpr int AHEAD = AHEAD_ < N ? AHEAD_ : N;
  Operand f[N];
  template <class Read>
  __device__ __forceinline__ void begin(Read read) {
#pragma unroll
    for (int m = 0; m < AHEAD; ++m) f[m] = read(m);
    DP_PIN();
  }
  template <class Read, class Multiply>
  __device__ __forceinline__ void run(Read read, Multiply multiply) {
    DP_PIN();
#pragma unroll
    for (int m = 0; m < N; ++m) {
      if (m + AHEAD < N) f[m + AHEAD] = read(m + AHEAD);
      multiply(m, f[m]);
      DP_PIN();
    }
  }
};

// What these loads bring is there from here on.  (Otherwise the wait for them may come where they are first used, in a loop, and would be one
// for the tiles on their way as well.)
template <class Row, int N>
__device__ __forceinline__ void have(Row (&f)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+v"(f[i]));
}

// The wave's own operand from memory: row `row` (zeros where !there), columns 2 EL ks + EL (lane / 32) ...
template <int DT, int KS>
__device__ __forceinline__ void load_own(typename Ops<DT>::Row (&f)[KS], const typename Ops<DT>::E* head, int64_t token_stride, int row,
                                         bool there, int D, int lane) {
  constexpr int EL = Ops<DT>::EL;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    const int col = 2 * EL * ks + EL * (lane >> 5);
    uint4 w = make_uint4(0, 0, 0, 0);
    if (there && col < D) w = *reinterpret_cast<const uint4*>(head + row * token_stride + col);
    f[ks] = __builtin_bit_cast(typename Ops<DT>::Row, w);
  }
}

// The other half's value (lane ^ 32).
__device__ __forceinline__ float other_half(float x, int lane) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(lane < 32 ? r[1] : r[0]);
}

__device__ __forceinline__ f32x16 zeros16() {
  f32x16 z;
#pragma unroll
  for (int r = 0; r < 16; ++r) z[r] = 0.f;
  return z;
}

// A 32-row result (columns by register, the wave's rows by lane) times f, rounded, to memory: turned in LDS (`lds`: 32 rows of the wave's
// own), so that whole rows leave, 16 bytes a lane.  Rows with there == false get zeros; rows from `rows` on are not in the tensor.
template <int DT, int DP>
__device__ __forceinline__ void store_rows(const f32x16 (&acc)[DP / 32], float f, bool there, typename Ops<DT>::E* head,
                                           int64_t token_stride, int row0, int rows, int D, unsigned lds, int lane) {
  typedef HeadTile<DT, DP> H;
  typedef __attribute__((ext_vector_type(4))) typename Ops<DT>::E E4;         // a lane has four adjacent columns
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
  for (int cb = 0; cb < DP / 32; ++cb)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      E4 y;
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = (typename Ops<DT>::E)(there ? acc[cb][4 * g + i] * f : 0.f);
      const unsigned at = (32 * cb + 8 * g + 4 * (lane >> 5)) * Ops<DT>::SIZE;
      *(__attribute__((address_space(3))) E4*)(uintptr_t)(lds + (lane & 31) * H::ROW_BYTES + ((at / 16) ^ H::swizzle(lane & 31)) * 16 + at % 16) = y;
    }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
  for (int i = 0; i < 32 * H::CHUNKS / 64; ++i) {
    const int id = i * 64 + lane, row = id / H::CHUNKS, chunk = id % H::CHUNKS;
    typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
    const u32x4 w = *(__attribute__((address_space(3))) const u32x4*)(uintptr_t)(lds + row * H::ROW_BYTES + (chunk ^ H::swizzle(row)) * 16);
    if (row0 + row < rows && chunk * H::EL < D) *reinterpret_cast<u32x4*>(head + (row0 + row) * token_stride + chunk * H::EL) = w;
  }
}

// The same result as it is, fp32, to rows of D columns.
template <int DP>
__device__ __forceinline__ void store_partial(const f32x16 (&acc)[DP / 32], bool there, float* head, int row, int rows, int D, int lane) {
  if (row >= rows) return;
#pragma unroll
  for (int cb = 0; cb < DP / 32; ++cb)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int col = 32 * cb + 8 * g + 4 * (lane >> 5);
      f32x4 y;
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = there ? acc[cb][4 * g + i] : 0.f;
      if (col < D) *reinterpret_cast<f32x4*>(head + (int64_t)row * D + col) = y;
    }
}

// Several waves may own the same 32 rows and take the other side's tiles in turn.  In how many floats they hand N values a lane to the first.
constexpr int handed_floats(int n) { return 64 * n; }
template <int N>
__device__ __forceinline__ void hand_over(const f32x16 (&acc)[N], float* to, int lane) {
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int r = 0; r < 16; ++r) to[(16 * n + r) * 64 + lane] = acc[n][r];
}
template <int N>
__device__ __forceinline__ void take_over(f32x16 (&acc)[N], const float* from, int lane) {
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[n][r] += from[(16 * n + r) * 64 + lane];
}

// How many they are: as LDS has room for tiles of 32 rows to each, in two stages.
constexpr int split_waves(int row_bytes) { return row_bytes <= 128 ? 8 : row_bytes <= 256 ? 4 : 2; }
// Whether there are so few rows (of `heads` pairs) that their workgroups leave compute units idle, and so many of the other side that turns are
// worth the joining.  In us, forward and both passes' gradients, one wave's and split: bf16, 8 heads of 64, 1 x 1 query, 4096 keys 59 + 71,
// 20 + 27; 1 head, 4096 tokens 49 + 145, 21 + 50; 8 heads, 2048 tokens 28 + 79, 21 + 54; but 24 heads, 512 tokens 11 + 29, 15 + 41.  fp32, whose tiles take
// eight times as long: 2 x 512 tokens, 8 heads of 128 73 + 239, 58 + 142; 4 x 128, 6 heads of 64 15 + 43, 11 + 25; but 8 x 128, 12 heads 16
// + 49, 20 + 50.
// Such a turn's tile is 32 rows for each wave: not where that many, as far apart as a side (x, y) has them, lie beyond the byte offsets of one
// descriptor.
template <int DT, int DP>
bool split_rows(int64_t heads, int rows, int others, const AttnSide& x, const AttnSide& y) {
  constexpr int64_t TILE_ROWS = 32 * split_waves(HeadTile<DT, DP>::ROW_BYTES);
  if (TILE_ROWS * Ops<DT>::SIZE * (x.token > y.token ? x.token : y.token) > (int64_t)OOB) return false;
  const int64_t workgroups = heads * ((rows + 127) / 128);
  return DT == DP_F32 ? workgroups <= 64 && others > 64 : workgroups <= 128 && others >= 1024;
}
// Queries, which go through keys and values, and keys, which go through queries and their gradients.
template <int DT, int DP>
bool split_queries(const AttnArgs& a) {
  return split_rows<DT, DP>((int64_t)a.B * a.H, a.Tq, a.Tk, a.ks, a.vs);
}
template <int DT, int DP>
bool split_keys(const AttnArgs& a) {
  return split_rows<DT, DP>((int64_t)a.B * a.H_kv * a.parts, a.Tk, a.Tq, a.qs, a.os);
}

// Calls f with the width that rows of D values are padded to.
template <int DT, class F>
auto by_head_width(int D, F f) {
  using std::integral_constant;
  if (D <= 32) return f(integral_constant<int, 32>{});
  if (D <= 64) return f(integral_constant<int, 64>{});
  if constexpr (DT != DP_F32)
    if (D <= 96) return f(integral_constant<int, 96>{});
  return f(integral_constant<int, 128>{});
}

// The scores' gradients of a lane's own row in fp16, times 2^raise, which keeps them below 2 and the largest so far from about 2^-6 on (so that 2^-8 of it
// has all bits and what a smaller one loses is 2^-19 of the largest at most).  It begins beyond need and is lowered where one outgrows it (the
// sums so far with it, exactly); it is taken out of the sums in fp32.  (A gradient of 10^-3, the mean loss of 2048 tokens, would put scores'
// gradients at 10^-7 else: the 2-norm of dq's error 9.4e-4 instead of 3.5e-4.)
struct Raised {
  int raise = 48;                                 // (a value is at most 2^41 as it is)
  __device__ __forceinline__ float factor(int less) const { return ldexpf(1.f, raise - less); }
  // Rounded values of 2 and more, infinities and what is no number among them: their exponents' highest bit.
  __device__ __forceinline__ static bool outgrown(const bf16x8 (&x)[2]) {
    typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
    const u32x4 bits = __builtin_bit_cast(u32x4, x[0]) | __builtin_bit_cast(u32x4, x[1]);
    return __any(((bits[0] | bits[1] | bits[2] | bits[3]) & 0x40004000u) != 0);
  }
  template <int N>
  __device__ __forceinline__ void lower(f32x16& x, f32x16 (&sum)[N], int lane) {
    float top = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) top = fmaxf(top, fabsf(x[r]));
    top = fmaxf(top, other_half(top, lane));
    if (top < 1.9f || !(top < INFINITY)) top = 0.015625f;            // (as it is)
    const int by = -5 - __builtin_amdgcn_frexp_expf(top);
    const float f = ldexpf(1.f, by);
    raise += by;
#pragma unroll
    for (int r = 0; r < 16; ++r) x[r] *= f;
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int r = 0; r < 16; ++r) sum[n][r] *= f;
  }
  template <int N>
  __device__ __forceinline__ void take_out(f32x16 (&sum)[N]) const { lower_by(sum, raise); }
  template <int N>
  __device__ __forceinline__ static void lower_by(f32x16 (&sum)[N], int by) {
    const float f = ldexpf(1.f, -by);
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int r = 0; r < 16; ++r) sum[n][r] *= f;
  }
};

// Calls f with a tile's number and the stage that it lies in, as a constant, for n tiles.
template <class F>
__device__ __forceinline__ void two_stages(int n, F f) {
  for (int t = 0;;) {
    if (t >= n) break;
    f(t++, std::integral_constant<int, 0>{});
    if (t >= n) break;
    f(t++, std::integral_constant<int, 1>{});
  }
}

// Whether some value is an infinity or no number.
template <int N>
__device__ __forceinline__ bool not_finite(const f32x16 (&acc)[N]) {
  float t = 0.f;
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int r = 0; r < 16; ++r) t = fmaf(acc[n][r], 0.f, t);
  return t != 0.f;
}

// ---- One row by one wave, in fp32 on the vector unit: what fp32 rows of no whole 16-byte pieces run on, and what a row is formed by again
// where a value that it does not see (a later token's, under a causal mask) is an infinity or no number and has spoilt its tile's
// products.  A lane takes one of 64 keys for the scores, its row against the wave's own, which lies in LDS; and columns lane and lane + 64
// for the sums.

constexpr int kRowFloats = 256;                   // of LDS to a wave: two own rows

// Products of N rows (a lane's, in memory) with own rows at `own` + 128 n in LDS.  whole: four elements at a time.
template <int N, class E>
__device__ __forceinline__ void dot_rows(float (&s)[N], const E* const (&row)[N], const float* own, int D, bool whole) {
  typedef __attribute__((ext_vector_type(4))) E E4;
#pragma unroll
  for (int n = 0; n < N; ++n) s[n] = 0.f;
  if (whole) {
#pragma unroll 4
    for (int d = 0; d < D; d += 4)
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const E4 y = *reinterpret_cast<const E4*>(row[n] + d);
        const f32x4 x = *reinterpret_cast<const f32x4*>(own + 128 * n + d);
#pragma unroll
        for (int i = 0; i < 4; ++i) s[n] = fmaf(x[i], (float)y[i], s[n]);
      }
  } else {
    for (int d = 0; d < D; ++d)
#pragma unroll
      for (int n = 0; n < N; ++n) s[n] = fmaf(own[128 * n + d], (float)row[n][d], s[n]);
  }
}

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) x = fmaxf(x, __shfl_xor(x, off));
  return x;
}
__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off);
  return x;
}

// acc += sum_j w_j rows[j], j < n <= 64 (w_j in lane j), in order, eight rows in flight.
template <class E>
__device__ __forceinline__ void add_rows(float (&acc)[2], float w, const E* rows, int64_t stride, int n, int D, int lane) {
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const int col = lane + 64 * c;
    if (c > 0 && D <= 64) break;
    const E* p = rows + min(col, D - 1);
    int j = 0;
    for (; j + 8 <= n; j += 8) {
      E x[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) x[q] = p[(j + q) * stride];
#pragma unroll
      for (int q = 0; q < 8; ++q)
        acc[c] = fmaf(__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), j + q)), (float)x[q], acc[c]);
    }
    for (; j < n; ++j) acc[c] = fmaf(__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), j)), (float)p[j * stride], acc[c]);
  }
}

template <class T>
__device__ __forceinline__ void store_row(const float (&acc)[2], float f, T* row, int D, int lane) {
#pragma unroll
  for (int c = 0; c < 2; ++c)
    if (lane + 64 * c < D) row[lane + 64 * c] = (T)(acc[c] * f);
}

template <class E>
struct AttnRows {
  const AttnArgs& a;
  float* own;                                     // the wave's, in LDS
  int b, h, lane, n_q, n_k;
  bool whole;
  __device__ AttnRows(const AttnArgs& args, float* own_, int b_, int h_, int lane_) : a(args), own(own_), b(b_), h(h_), lane(lane_) {
    n_q = valid_rows(a.q_len, b, a.Tq);
    n_k = valid_rows(a.k_len, b, a.Tk);
    const int64_t all = a.D | a.qs.sample | a.qs.token | a.qs.head | a.ks.sample | a.ks.token | a.ks.head | a.vs.sample | a.vs.token |
                        a.vs.head | a.os.sample | a.os.token | a.os.head;
    whole = (all & 3) == 0 && aligned_arrays(a);
  }
  __device__ const E* query(const void* t, const AttnSide& s, int head) const { return (const E*)t + b * s.sample + head * s.head; }
  __device__ int keys_of(int i) const {         // row i sees keys below this
    return i >= n_q ? 0 : a.causal ? min(max(i + n_k - n_q + 1, 0), n_k) : n_k;
  }
  __device__ void keep_own(const E* row, int n) const {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    for (int d = lane; d < a.D; d += 64) own[128 * n + d] = (float)row[d];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }

  __device__ void forward(int i) const {
    const E *q = query(a.q, a.qs, h) + i * a.qs.token, *k = query(a.k, a.ks, h / a.share), *v = query(a.v, a.vs, h / a.share);
    const int n = keys_of(i);
    float most = -INFINITY, total = 0.f, acc[2] = {0.f, 0.f};
    keep_own(q, 0);
    for (int j0 = 0; j0 < n; j0 += 64) {
      const E* const rows[1] = {k + min(j0 + lane, n - 1) * a.ks.token};
      float s[1];
      dot_rows<1, E>(s, rows, own, a.D, whole);
      s[0] = j0 + lane < n ? a.scale2 * s[0] : -INFINITY;
      const float top = fmaxf(most, wave_max(s[0])), ref = top == -INFINITY ? 0.f : top;
      const float p = exp2f(s[0] - ref), fix = exp2f(most - ref);
      most = top;
      total = total * fix + wave_sum(p);
#pragma unroll
      for (int c = 0; c < 2; ++c) acc[c] *= fix;
      add_rows(acc, p, v + j0 * a.vs.token, a.vs.token, min(64, n - j0), a.D, lane);
    }
    store_row(acc, total != 0.f ? 1.f / total : 0.f, (E*)a.out + b * a.os.sample + h * a.os.head + i * a.os.token, a.D, lane);
    if (lane == 0) a.lse[((int64_t)b * a.H + h) * a.Tq + i] = total != 0.f ? most * kLn2 + logf(total) : -INFINITY;
  }

  // Probability, and its score's gradient, of a lane's row against the own rows.
  __device__ void pair(const E* x, const E* y, float lse2, float delta, float& p, float& ds) const {
    const E* const rows[2] = {x, y};
    float s[2];
    dot_rows<2, E>(s, rows, own, a.D, whole);
    p = exp2f(fmaf(a.scale2, s[0], -lse2));
    ds = p * (s[1] - delta);
  }

  __device__ void query_gradient(int i) const {
    const E *q = query(a.q, a.qs, h) + i * a.qs.token, *k = query(a.k, a.ks, h / a.share), *v = query(a.v, a.vs, h / a.share);
    const E *dout = query(a.dout, a.os, h) + i * a.os.token, *o = query(a.o, a.os, h) + i * a.os.token;
    const int n = keys_of(i);
    const int64_t at = ((int64_t)b * a.H + h) * a.Tq + i;
    const float lse = a.lse[at], lse2 = n == 0 || lse == -INFINITY ? INFINITY : lse * kLog2e;
    keep_own(q, 0);
    keep_own(dout, 1);
    float delta[1] = {0.f};                       // formed as do v' is: a row of one key has the same products in both
    if (n > 0) {
      const E* const rows[1] = {o};
      dot_rows<1, E>(delta, rows, own + 128, a.D, whole);
    }
    float acc[2] = {0.f, 0.f};
    for (int j0 = 0; j0 < n; j0 += 64) {
      const int j = min(j0 + lane, n - 1);
      float p, ds;
      pair(k + j * a.ks.token, v + j * a.vs.token, lse2, delta[0], p, ds);
      add_rows(acc, ds, k + j0 * a.ks.token, a.ks.token, min(64, n - j0), a.D, lane);
    }
    store_row(acc, a.scale, (E*)a.dq + b * a.qs.sample + h * a.qs.head + i * a.qs.token, a.D, lane);
    if (lane == 0) {
      a.lse2[at] = lse2 - kGain<E>;
      a.delta[at] = -delta[0];
    }
  }

  // h: a key head, of whose query heads first .. last - 1 count; to partial sums (rows of D values) or, null, to the gradients.
  __device__ void key_gradient(int j, int first, int last, float* dk_part, float* dv_part) const {
    const E *k = query(a.k, a.ks, h) + j * a.ks.token, *v = query(a.v, a.vs, h) + j * a.vs.token;
    float dk[2] = {0.f, 0.f}, dv[2] = {0.f, 0.f};
    const int from = a.causal ? max(j - (n_k - n_q), 0) : 0;
    keep_own(k, 0);
    keep_own(v, 1);
    for (int hq = first; j < n_k && hq < last; ++hq) {
      const E *q = query(a.q, a.qs, hq), *dout = query(a.dout, a.os, hq);
      const int64_t at = ((int64_t)b * a.H + hq) * a.Tq;
      for (int i0 = from; i0 < n_q; i0 += 64) {
        const int i = min(i0 + lane, n_q - 1);
        float p, ds;
        pair(q + i * a.qs.token, dout + i * a.os.token, a.lse2[at + i] + kGain<E>, -a.delta[at + i], p, ds);
        // no gradient of the scores of a row that sees one key (a 16-bit row's delta is not formed as do v' is)
        if (keys_of(i) == 1) ds = 0.f;
        add_rows(dv, p, dout + i0 * a.os.token, a.os.token, min(64, n_q - i0), a.D, lane);
        add_rows(dk, ds, q + i0 * a.qs.token, a.qs.token, min(64, n_q - i0), a.D, lane);
      }
    }
    if (dk_part) {
      store_row(dk, 1.f, dk_part + (int64_t)j * a.D, a.D, lane);
      store_row(dv, 1.f, dv_part + (int64_t)j * a.D, a.D, lane);
      return;
    }
    store_row(dk, a.scale, (E*)a.dk + b * a.ks.sample + h * a.ks.head + j * a.ks.token, a.D, lane);
    store_row(dv, 1.f, (E*)a.dv + b * a.vs.sample + h * a.vs.head + j * a.vs.token, a.D, lane);
  }
};

// Rows of fp32 that the matrix kernels take: 16-byte pieces throughout.
inline bool whole_pieces(const AttnArgs& a) {
  const AttnSide* sides[] = {&a.qs, &a.ks, &a.vs, &a.os};
  int64_t all = a.D;
  for (const AttnSide* s : sides) all |= s->sample | s->token | s->head;
  return all % 4 == 0 && aligned_arrays(a);
}

// Launches `blocks` of a.heads pairs, in runs below the grid's limit.
constexpr int64_t kGroupBytes = 3 << 20;
template <class K>
dp_status launch_attention(K kernel, AttnArgs a, int64_t shared_bytes, int threads, int lds, hipStream_t s) {
  // A pair's blocks stay on one XCD where the pairs fill the eight of them (padded up to a multiple of eight); a group of pairs is what half
  // an L2 cache holds of what their blocks share.
  a.spread = a.blocks > 1 && (a.heads % 8 == 0 || a.heads >= 64);
  const int64_t group = kGroupBytes / (shared_bytes > 0 ? shared_bytes : 1);
  a.group = (int)(group < 1 ? 1 : group > a.heads ? a.heads : group);
  const int64_t n = (int64_t)(a.spread ? (a.heads + 7) / 8 * 8 : a.heads) * a.blocks;
  return launch_in_runs(n, [&](dim3 grid, int first) {
    AttnArgs run = a;
    run.first = (unsigned)first;
    hipLaunchKernelGGL(kernel, grid, dim3(threads), lds, s, run);
  });
}

dp_status launch_attention_forward(const AttnArgs& a, dp_dtype dt, hipStream_t s);
// Rows of the other side that a tile holds in the forward pass, and (a.parts set) in the two backward kernels; 1 where rows are taken one by one.
int attention_forward_tile(const AttnArgs& a, dp_dtype dt);
void attention_backward_tiles(const AttnArgs& a, dp_dtype dt, int& queries, int& keys);
// Sets key_parts and part_keys; floats that they need where key_parts is more than one.
void attention_key_parts(AttnArgs& a, dp_dtype dt);
int64_t attention_key_floats(const AttnArgs& a);
// Workgroups that the query heads of a key head are dealt to in the backward pass, and floats that they need where it is more than one.
int attention_parts(const AttnArgs& a);
int64_t attention_partial_floats(const AttnArgs& a);
dp_status launch_attention_backward(const AttnArgs& a, dp_dtype dt, hipStream_t s);

}  // namespace dpbk
