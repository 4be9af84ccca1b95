// Tiles of products on the 16-bit matrix instructions:  acc[m, n] = sum_s sum_k A_s[m, k] B_s[k, n]  over up to two segments s; and, of values that
// are two fp16 halves h + l each, with all of it but l l'.
//
// A has its terms adjacent ([m][k]); B as well ([n][k], "rows"), or its columns ([k][n]): two sets of them side by side, each with its own
// origin, which is how a gate and its factor meet in one lane ("sets"), or one of values in halves ("split").
//  * 256 x 256 tiles by eight waves of 128 x 64, or 128 x 128 by four of 64 x 64 (two workgroups to a compute unit).  Accumulators and
//    operands of one k-step and the next lie in registers.
//  * memory -> LDS without registers (16 bytes a lane), stages of 64 terms: whole 128-byte lines of [m][k] rows.  (Stages of 32, five of
//    them, took each line in two halves a microsecond apart, and through the first-level cache twice: 4096 x 65536 x 12288 6050 us, two stages of
//    64 with these instructions 5020.)  A has three places in LDS and B two, all of it: B's of a stage is free once its operands are in
//    registers, half a stage before A's, so B's loads have 1.4 stages to land and A's two.
//    Two barriers to a stage of the large tiles: M, behind the last read of B; E, behind the last one of A, where the next stage has landed.
//  * LDS holds [m][64 k] in rows of 128 bytes: a 128-bit read takes sixteen lanes at a time, here sixteen rows at one place of eight, so that
//    place is XORed with row / 2 and all banks are met.  [k][n] rows are of 128 to 1024 bytes; the transposing read takes eight rows of 32
//    bytes at a time, which the XOR by k spreads over all banks.
//  * rows, columns and terms past the end arrive as zeros: by the descriptor's size, or by an offset past it.
//  * Halves: 32 terms are a line of 32 h and 32 l, so a stage is 32 terms of both, and its operands are read once for the three products of
//    a term.  (As three segments of a product, h h', h l' and l h', everything was read one and a half times: A of 60 matrices of 768 rows,
//    340 MB, 267 us.)
// The first operand of an instruction is B's: a lane has one row of the result and four adjacent columns to a register quad.
#pragma once

#include <type_traits>
#include <utility>

#include "dp_internal.h"
#include "lds_dma.h"
#include "tile_order.h"

namespace dpbk {

struct ProductSegment {
  const void *a, *b0, *b1;          // b1: the second set's columns (sets only)
};
constexpr int kProductTerms = 64;   // of a stage
constexpr int kHalfTerms = 32;      // of one of values in halves
struct ProductShape {
  int M, N, K;                      // K: of a segment, in 16-bit values (halves: both); K and N (columns) are multiples of 8
  int terms;                        // columns: rows of B that are there (fewer than A has terms: A has zeros beyond)
  int lda, ldb;                     // 16-bit values from one row (of columns: term) to the next
  int segments;
  int first, stages;                // of all segments' stages one behind the other, those that this tile takes
  ProductSegment s[2];
};

enum ProductB { kRowsOfTerms, kColumnSets, kSplitColumns };
template <int BM_, int WM_, int WN_, ProductB B_, bool HALVES_ = false>
struct ProductTile {
  static constexpr int BM = BM_, BN = BM_, BK = kProductTerms, A_PLACES = 3, B_PLACES = 2, WM = WM_, WN = WN_, NW = WM * WN, NT = 64 * NW;
  static constexpr bool HALVES = HALVES_, SETS = B_ == kColumnSets, SPLIT = B_ == kSplitColumns, ROWS = B_ == kRowsOfTerms;
  static constexpr int WTM = BM / WM, WTN = BN / WN, TM = WTM / 16, TN = WTN / 16;       // 16 x 16 results of a wave
  static constexpr int ROW_BYTES = 2 * BK, A_BYTES = BM * ROW_BYTES, B_BYTES = BN * ROW_BYTES;
  static constexpr int B_AT = A_PLACES * A_BYTES;                              // of B's first place
  static constexpr int TERMS = HALVES ? kHalfTerms : BK;                       // of a stage
  static constexpr int HALF_BYTES = B_BYTES / 2;                               // sets: of one of them
  static constexpr int COL_BYTES = SPLIT ? 4 * BN : BN;                        // columns: a term's, of one set or of both halves
  static constexpr int LDS_BYTES = B_AT + B_PLACES * B_BYTES, LOADS = A_BYTES / (NW * 1024);     // of an operand, wave and stage
  // epilogue: 32 rows of a wave's columns, fp32
  static constexpr int SLAB_PITCH = WTN + 4, SLAB_BYTES = 32 * SLAB_PITCH * 4;
  // columns: the 16-byte place of a term's row is XORed with this
  __device__ static constexpr unsigned spread(unsigned k) {
    return COL_BYTES >= 256 ? (k & 3) << 2 | (k >> 2 & 2) : (k & 2) << 1 | (k >> 2 & 2);
  }
  static_assert(LOADS * NW * 1024 == A_BYTES && LOADS % 2 == 0 && NW * SLAB_BYTES <= LDS_BYTES, "load split, fragments, epilogue");
  static_assert(HALVES != SETS && HALVES >= SPLIT || !HALVES, "what there is");
};
template <ProductB B, bool HALVES = false>
using BigProduct = ProductTile<256, 2, 4, B, HALVES>;
template <ProductB B, bool HALVES = false>
using MidProduct = ProductTile<128, 2, 2, B, HALVES>;

// Memory -> LDS: the stages of A and of B, each a stream of its own.
template <class S>
struct ProductLoads {
  struct Stream {                   // the stage to ask for next: segment, first value or term of it, place in LDS; how many there are
    int seg, k, place, left;
  };
  const ProductShape& p;
  int m0, chunk;
  unsigned n_off, a_pitch, b_pitch, a_bytes, b_bytes, lds_ld;
  unsigned va[S::LOADS], vb[S::LOADS];
  i32x4 ra, rb[2];
  Stream a, b;

  __device__ static __forceinline__ i32x4 scalar(i32x4 r) {
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __builtin_amdgcn_readfirstlane(r[i]);
    return r;
  }
  __device__ static __forceinline__ unsigned scalar(unsigned x) { return __builtin_amdgcn_readfirstlane(x); }
  __device__ static __forceinline__ const char* pick(int seg, const void* first, const void* second) {
    return static_cast<const char*>(seg == 0 ? first : second);                // (an index would put them in memory)
  }
  __device__ __forceinline__ ProductLoads(const ProductShape& shape, int m, const int (&n0)[2], unsigned lds0, int wave, int lane) : p(shape), m0(m) {
    chunk = (lane & 7) ^ ((4 * (wave & 1) + (lane >> 4)) & 7);                 // 16-byte piece of a row's stage
    a_pitch = 2u * p.lda;
    b_pitch = 2u * p.ldb;
    n_off = n0[0];
#pragma unroll
    for (int l = 0; l < S::LOADS; ++l) {
      const unsigned row = 8 * (l * S::NW + wave) + (lane >> 3);
      va[l] = row * a_pitch + chunk * 16;
      if constexpr (S::ROWS) {
        vb[l] = row * b_pitch + chunk * 16;
      } else {
        // 1 KiB of LDS: some terms' rows (of one set), or one
        constexpr int PIECES = S::COL_BYTES / 16, SET_LOADS = S::SETS ? S::LOADS / 2 : S::LOADS;
        const unsigned k = PIECES <= 64 ? (l % SET_LOADS * S::NW + wave) * (64 / PIECES) + lane / PIECES : 0, at = lane % PIECES;
        const unsigned piece = at ^ S::spread(k), value = S::SETS ? n0[l / SET_LOADS] + 8 * piece : 2 * n0[0] + 8 * piece;
        vb[l] = (int)value < (S::SPLIT ? p.ldb : p.N) ? k * b_pitch + 2 * value : OOB;
      }
    }
    a_bytes = (unsigned)imin(p.M - m0, S::BM) * a_pitch;
    b_bytes = S::ROWS ? (unsigned)imax(imin(p.N - n0[0], S::BN), 0) * b_pitch : 0;
    lds_ld = lds0 + wave * 1024;
    const int per = (p.K + S::BK - 1) / S::BK;                                 // stages of a segment
    a.seg = p.first >= per ? 1 : 0;
    a.k = p.first - a.seg * per;
    a.place = 0;
    a.left = p.stages;
    b = a;
    a.k *= S::BK;
    b.k *= S::ROWS ? S::BK : S::TERMS;
    b.place = S::B_AT;
    open_a();
    open_b();
  }
  __device__ __forceinline__ void open_a() {
    ra = make_rsrc(pick(a.seg, p.s[0].a, p.s[1].a) + (uint64_t)m0 * a_pitch, a.left > 0 ? a_bytes : 0);
  }
  __device__ __forceinline__ void open_b() {
    const char* const b0 = pick(b.seg, p.s[0].b0, p.s[1].b0);
    if constexpr (S::ROWS) {
      rb[0] = make_rsrc(b0 + (uint64_t)n_off * b_pitch, b.left > 0 ? b_bytes : 0);
    } else {
      rb[0] = make_rsrc(b0 + (uint64_t)b.k * b_pitch, 0);
      if constexpr (S::SETS) rb[1] = make_rsrc(pick(b.seg, p.s[0].b1, p.s[1].b1) + (uint64_t)b.k * b_pitch, 0);
      open_terms();
    }
  }
  __device__ __forceinline__ void open_terms() {                               // columns: terms b.k .. of the segment that are there
    rb[0][2] = (int)(b.left > 0 ? (unsigned)imax(imin(p.terms - b.k, S::TERMS), 0) * b_pitch : 0);
    if constexpr (S::SETS) rb[1][2] = rb[0][2];
  }
  __device__ __forceinline__ void load_a(int l) {
    load_to_lds(scalar(ra), a.k + 8 * chunk < p.K ? va[l] : OOB, scalar(2u * a.k), scalar(lds_ld + a.place + l * S::NW * 1024));
  }
  __device__ __forceinline__ void load_b(int l) {
    const unsigned to = scalar(lds_ld + b.place + l * S::NW * 1024);
    if constexpr (S::ROWS)
      load_to_lds(scalar(rb[0]), b.k + 8 * chunk < p.K ? vb[l] : OOB, scalar(2u * b.k), to);
    else
      load_to_lds(scalar(rb[S::SETS ? l / (S::LOADS / 2) : 0]), vb[l], 0, to);
  }
  __device__ __forceinline__ void advance_a() {
    a.place = a.place == 2 * S::A_BYTES ? 0 : a.place + S::A_BYTES;
    a.k += S::BK;
    --a.left;
    if (a.k >= p.K || a.left <= 0) {
      a.k = 0;
      ++a.seg;
      open_a();
    }
  }
  __device__ __forceinline__ void advance_b() {
    b.place = 2 * S::B_AT + S::B_BYTES - b.place;
    b.k += S::ROWS ? S::BK : S::TERMS;
    --b.left;
    if (b.left <= 0 || (S::ROWS || !S::HALVES ? b.k >= p.K : 2 * b.k >= p.K)) {
      b.k = 0;
      ++b.seg;
      open_b();
    } else if constexpr (!S::ROWS) {
#pragma unroll
      for (int l = 0; l < (S::SETS ? 2 : 1); ++l) {
        const uint64_t q = ((uint64_t)(uint32_t)rb[l][1] << 32 | (uint32_t)rb[l][0]) + (uint64_t)S::TERMS * b_pitch;
        rb[l][0] = (int)(uint32_t)q;
        rb[l][1] = (int)(uint32_t)(q >> 32);
      }
      open_terms();
    }
  }
  // A 0, B 0, A 1, B 1, A 2; the first two have landed.
  __device__ __forceinline__ void begin() {
#pragma unroll
    for (int q = 0; q < 5; ++q) {
#pragma unroll
      for (int l = 0; l < S::LOADS; ++l) {
        if (q & 1)
          load_b(l);
        else
          load_a(l);
      }
      if (q & 1)
        advance_b();
      else
        advance_a();
    }
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(3 * S::LOADS) : "memory");
  }
};

// LDS -> operands: where a lane finds them.  Part: the k-step of 32 terms, or h and l.
template <class S>
struct ProductReads {
  unsigned a_rd[2], b_rd[2];
  typedef __attribute__((address_space(3))) const bf16x8* Lds;
  __device__ __forceinline__ ProductReads(unsigned lds0, int wave, int lane) {
    const int row = lane & 15, wm = wave / S::WN * S::WTM, wc = wave % S::WN;
#pragma unroll
    for (int part = 0; part < 2; ++part) {
      const unsigned place = (unsigned)((4 * part + (lane >> 4)) ^ (row >> 1)) << 4;
      a_rd[part] = lds0 + (wm + row) * S::ROW_BYTES + place;
      if constexpr (S::ROWS) {
        b_rd[part] = lds0 + S::B_AT + (S::WTN * wc + row) * S::ROW_BYTES + place;
      } else {
        const int k = 8 * (lane >> 4) + (row >> 2);
        // split: blocks of 32 columns, 64 bytes of h and as many of l
        const unsigned piece = (S::SETS ? (unsigned)(S::WTN / 2 * wc) >> 3 : (unsigned)(S::WTN * wc) >> 2) + ((row & 3) >> 1);
        b_rd[part] = lds0 + S::B_AT + (S::SETS ? 32 * part + k : k) * S::COL_BYTES + ((piece ^ S::spread(k)) << 4) + 8 * (row & 1);
      }
    }
  }
  __device__ __forceinline__ bf16x8 a(int x, unsigned base, int part) const { return *(Lds)(uintptr_t)(a_rd[part] + base + x * 16 * S::ROW_BYTES); }
  __device__ __forceinline__ void b(Frag& f, int y, unsigned base, int part) const {
    if constexpr (S::ROWS) {
      f.v = *(Lds)(uintptr_t)(b_rd[part] + base + y * 16 * S::ROW_BYTES);
    } else {
      // 16 columns further are two pieces; h and l, four; in bits that the lane's own piece has as the XOR by k alone left them
      const unsigned at = S::SETS ? ((b_rd[part] + base) ^ (y % (S::TN / 2) << 5)) + y / (S::TN / 2) * S::HALF_BYTES
                                  : (b_rd[part] + base) ^ ((y & 1) << 5 | part << 6 | (y >> 1) << 7);
      f.h[0] = lds_read_tr(at);
      f.h[1] = lds_read_tr(at + 4 * S::COL_BYTES);
    }
  }
};

// The tile at (m0, n0) (sets: of either set n0[0], n0[1]) into acc.  acc[x][y], lane, register r: row 16 x + lane % 16 of the wave's, column
// 16 y + 4 (lane / 16) + r of its WTN: those of the tile from WTN (wave % WN) on, or half as many of each set.
template <class S, bool F16>
__device__ __forceinline__ void product_tile(const ProductShape& p, int m0, const int (&n0)[2], unsigned lds0, f32x4 (&acc)[S::TM][S::TN]) {
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  ProductLoads<S> load(p, m0, n0, lds0, wave, lane);
  const ProductReads<S> read(lds0, wave, lane);
#pragma unroll
  for (int x = 0; x < S::TM; ++x)
#pragma unroll
    for (int y = 0; y < S::TN; ++y) acc[x][y] = f32x4{0.f, 0.f, 0.f, 0.f};
  load.begin();
  unsigned a_base = 0, b_base = 0;
  auto next_bases = [&]() {
    a_base = a_base == 2 * S::A_BYTES ? 0 : a_base + S::A_BYTES;
    b_base = S::B_BYTES - b_base;
    asm("" : "+s"(a_base), "+s"(b_base));
  };
  if constexpr (S::HALVES) {
    // A row of A's operands, h and l, is asked for a row ahead; B's of the next stage, of h and l, within the last row.
    Frag fa[2][2], fb[2][2][S::TN];                                // [row % 2][h, l]; [stage % 2][h, l]
#pragma unroll
    for (int part = 0; part < 2; ++part) {
#pragma unroll
      for (int y = 0; y < S::TN; ++y) read.b(fb[0][part][y], y, 0, part);
      fa[0][part].v = read.a(0, 0, part);
    }
    auto stage = [&](auto turn_tag) {
      constexpr int turn = decltype(turn_tag)::value, LAST = S::TM - 1;
#pragma unroll
      for (int x = 0; x < S::TM; ++x) {
        // M: B's operands are in registers (the last row's reads; two of A's are younger)
        if (x == 1) asm volatile("s_waitcnt lgkmcnt(2)\n\ts_barrier" ::: "memory");
        if (x == LAST) {                                           // E
          asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(2 * S::LOADS) : "memory");
          next_bases();
        }
        DP_PIN();
#pragma unroll
        for (int slot = 0; slot < 3 * S::TN; ++slot) {
          const int product = slot / S::TN, y = slot % S::TN;      // h h, l of B, l of A
          acc[x][y] = mfma16<F16>(fb[turn][product == 1][y].v, fa[x & 1][product == 2].v, acc[x][y]);
          DP_PIN();
          if (slot < 2) fa[~x & 1][slot].v = read.a((x + 1) % S::TM, a_base, slot);
          if (x == LAST && slot >= 2 && slot < 2 + 2 * S::TN) read.b(fb[turn ^ 1][(slot - 2) / S::TN][(slot - 2) % S::TN], (slot - 2) % S::TN, b_base, (slot - 2) / S::TN);
          // loads: B's behind M, A's behind E
          if (x >= 1 && x < LAST) {
            constexpr int SLOTS = (LAST - 1) * 3 * S::TN;
            const int at = (x - 1) * 3 * S::TN + slot;
#pragma unroll
            for (int e = at * S::LOADS / SLOTS; e < (at + 1) * S::LOADS / SLOTS; ++e) {
              load.load_b(e);
              if (e == S::LOADS - 1) load.advance_b();
            }
          }
          if (x == LAST && slot % 3 == 2 && slot / 3 < S::LOADS) {
            load.load_a(slot / 3);
            if (slot / 3 == S::LOADS - 1) load.advance_a();
          }
          DP_PIN();
        }
      }
    };
    for (int st = 0; st < p.stages; st += 2) {                     // (a stage past the last one: zeros)
      asm("" : "+s"(a_base), "+s"(b_base));
      stage(std::integral_constant<int, 0>{});
      stage(std::integral_constant<int, 1>{});
    }
  } else {
    // B's operands of a k-step of 32 and the next; A's, each used by four instructions in a row, AHEAD of their use.
    constexpr int AHEAD = 3;
    Frag fa[4], fb[2][S::TN];
#pragma unroll
    for (int y = 0; y < S::TN; ++y) read.b(fb[0][y], y, 0, 0);
#pragma unroll
    for (int x = 0; x < AHEAD; ++x) fa[x].v = read.a(x, 0, 0);
    // TWO: barriers M and E; else one, of both (small tiles: a few instructions lie between the two).
    constexpr bool TWO = S::TM > 4;
    constexpr int TURN = S::TM - AHEAD;                            // from this row on operands of the next k-step
    for (int st = 0; st < p.stages; ++st) {
      asm("" : "+s"(a_base), "+s"(b_base));
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
        for (int x = 0; x < S::TM; ++x) {
          if (TWO && ks == 1 && x == 1) asm volatile("s_waitcnt lgkmcnt(1)\n\ts_barrier" ::: "memory");      // one of A's is younger
          if (ks == 1 && x == TURN) {
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((TWO ? 2 : 1) * S::LOADS) : "memory");
            next_bases();
          }
          DP_PIN();
#pragma unroll
          for (int y = 0; y < S::TN; ++y) {
            acc[x][y] = mfma16<F16>(fb[ks][y].v, fa[x & 3].v, acc[x][y]);
            DP_PIN();
            if (y == 0) fa[(x + AHEAD) & 3].v = read.a((x + AHEAD) % S::TM, a_base, x >= TURN ? ks ^ 1 : ks);
            constexpr int SLOTS = AHEAD * S::TN;
            const int slot = (x - TURN) * S::TN + y;               // of the last AHEAD rows
            // B's of the next k-step, each behind an instruction that reads none of A's
            if (x >= TURN && y != 0) {
              const int from = (slot - (x - TURN) - 1) * S::TN / (SLOTS - AHEAD), to = (slot - (x - TURN)) * S::TN / (SLOTS - AHEAD);
#pragma unroll
              for (int b = from; b < to; ++b) read.b(fb[ks ^ 1][b], b, b_base, ks ^ 1);
            }
            // loads: B's behind M (or E), A's behind E
            if (TWO && ks == 1 && x >= 1 && x < 1 + S::LOADS && y == 2) {
              load.load_b(x - 1);
              if (x == S::LOADS) load.advance_b();
            }
            if (ks == 1 && x >= TURN) {
              constexpr int LOADS = (TWO ? 1 : 2) * S::LOADS;
#pragma unroll
              for (int e = slot * LOADS / SLOTS; e < (slot + 1) * LOADS / SLOTS; ++e) {
                if (TWO || e >= S::LOADS)
                  load.load_a(e % S::LOADS);
                else
                  load.load_b(e);
              }
              if (slot == SLOTS - 1) {
                if (!TWO) load.advance_b();
                load.advance_a();
              }
            }
            DP_PIN();
          }
        }
      }
    }
  }
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");      // loads past the end
  __syncthreads();
}

// Where a lane's eight columns of a result's rows are in the epilogue: PAIRS, of both sets, else of one.
template <class S, bool PAIRS>
struct ProductPlaces {
  static constexpr int LANES = S::WTN / (PAIRS ? 16 : 8), PASSES = 32 * LANES / 64, HALF = S::WTN / 2, BLOCKS = S::TM / 2;
  int c, set, col, first;           // column of the wave's, set, column within it or within the tile; row
  __device__ __forceinline__ ProductPlaces() {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wc = wave % S::WN;
    c = 8 * (lane % LANES);
    set = S::SETS && !PAIRS ? c / HALF : 0;
    col = S::SETS ? HALF * wc + c % HALF : S::WTN * wc + c;
    first = wave / S::WN * S::WTM + lane / LANES;
  }
  __device__ __forceinline__ int row(int x, int i) const { return first + 32 * x + i * (64 / LANES); }       // of block x, pass i
};

// What load(row, column, set) brings for each place, asked for a block of 32 rows ahead.  (Asked for before the products, where a small tile's fit the
// registers, it came no sooner: 4096 x 1280 x 3456 57.0 us, so 59.2.)
template <class S, bool PAIRS, class Load>
struct ProductAhead {
  typedef ProductPlaces<S, PAIRS> Places;
  Load load;
  decltype(std::declval<Load>()(0, 0, 0)) values[2][Places::PASSES];
  __device__ __forceinline__ explicit ProductAhead(Load l) : load(l) {}
  __device__ __forceinline__ void ask(const Places& at, int x) {
    if (x >= Places::BLOCKS) return;
#pragma unroll
    for (int i = 0; i < Places::PASSES; ++i) values[x & 1][i] = load(at.row(x, i), at.col, at.set);
  }
};
struct Nothing {};
struct NoLoad {
  __device__ Nothing operator()(int, int, int) const { return {}; }
};
template <class S, bool PAIRS>
using NothingAhead = ProductAhead<S, PAIRS, NoLoad>;

// acc's rows to store(row of the tile, column, set, values, ahead's): columns 8 at a time, of both sets where PAIRS (v[0] and v[1]), else of one
// (v[0]).  The wave's 32 rows at a time are turned in LDS, so that whole rows leave.  across(first row, column, values): the same by columns, rows 8
// at a time, where `mirror`.
struct NoMirror {
  __device__ void operator()(int, int, const float (&)[8]) const {}
};
template <class S, bool PAIRS, class Ahead, class Store, class Across = NoMirror>
__device__ __forceinline__ void product_rows(const f32x4 (&acc)[S::TM][S::TN], unsigned lds0, Ahead& ahead, Store store, bool mirror = false,
                                             Across across = {}) {
  typedef ProductPlaces<S, PAIRS> Places;
  const Places at;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / S::WN * S::WTM, wc = wave % S::WN;
  const unsigned slab = lds0 + wave * S::SLAB_BYTES;
  typedef __attribute__((address_space(3))) f32x4* Lds;
  constexpr int PASSES = Places::PASSES, HALF = Places::HALF;
  ahead.ask(at, 0);
#pragma unroll
  for (int x = 0; x < S::TM / 2; ++x) {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int y = 0; y < S::TN; ++y)
        *(Lds)(uintptr_t)(slab + 4 * ((16 * h + (lane & 15)) * S::SLAB_PITCH + 16 * y + 4 * (lane >> 4))) = acc[2 * x + h][y];
    ahead.ask(at, x + 1);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      float v[2][8];
#pragma unroll
      for (int s = 0; s < (PAIRS ? 2 : 1); ++s)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const f32x4 w = *(Lds)(uintptr_t)(slab + 4 * ((at.row(0, i) - wm) * S::SLAB_PITCH + HALF * s + at.c + 4 * h));
#pragma unroll
          for (int e = 0; e < 4; ++e) v[s][4 * h + e] = w[e];
        }
      store(at.row(x, i), at.col, at.set, v, ahead.values[x & 1][i]);
    }
    if (!std::is_same_v<Across, NoMirror> && mirror) {
#pragma unroll
      for (int i = 0; i < S::WTN / 16; ++i) {                      // four lanes have the 32 rows of a column
        const int r = 8 * (lane & 3), column = 16 * i + (lane >> 2);
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
          v[e] = *(__attribute__((address_space(3))) const float*)(uintptr_t)(slab + 4 * ((r + e) * S::SLAB_PITCH + column));
        across(wm + 32 * x + r, S::WTN * wc + column, v);
      }
    }
  }
}

}  // namespace dpbk
