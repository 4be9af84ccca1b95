// Tiles of products on the 16-bit matrix instructions:  acc[m, n] = sum_s sum_k A_s[m, k] B_s[k, n]  over up to three segments s.
//
// A has its terms adjacent ([m][k]); B as well ([n][k], "rows"), or its columns ([k][n], "columns": two sets of them side by side, each with
// its own origin, which is how a gate and its factor meet in one lane).
//  * 256 x 256 tiles by eight waves of 128 x 64, or 128 x 128 by four of 64 x 64 (two workgroups to a compute unit).  Accumulators and
//    operands of one k-step and the next lie in registers.
//  * memory -> LDS without registers (16 bytes a lane), stages of 64 terms: whole 128-byte lines of [m][k] rows.  (Stages of 32, five of
//    them, took each line in two halves a microsecond apart, and through the first-level cache twice: 4096 x 65536 x 12288 6050 us, two stages of
//    64 with these instructions 5020.)  A has three places in LDS and B two, all of it: B's of a stage is free once its operands are in
//    registers, half a stage before A's, so B's loads have 1.4 stages to land and A's two.
//    Two barriers to a stage of the large tiles: M, behind the last read of B; E, behind the last one of A, where the next stage has landed.
//  * LDS holds [m][64 k] in rows of 128 bytes: a 128-bit read takes sixteen lanes at a time, here sixteen rows at one place of eight, so that
//    place is XORed with row / 2 and all banks are met.  [k][n] halves have rows of 256 or 128 bytes; the transposing read takes four
//    rows of 64 bytes at a time, which the XOR by k spreads over the four groups of banks.
//  * rows, columns and terms past the end arrive as zeros: by the descriptor's size, or by an offset past it.
// The first operand of an instruction is B's: a lane has one row of the result and four adjacent columns to a register quad.
#pragma once

#include <type_traits>

#include "dp_internal.h"
#include "lds_dma.h"
#include "tile_order.h"

namespace dpbk {

struct ProductSegment {
  const void *a, *b0, *b1;          // b1: the second set's columns (columns only)
};
constexpr int kProductTerms = 64;   // of a stage
struct ProductShape {
  int M, N, K;                      // K: of a segment; K and N (columns) are multiples of 8
  int terms;                        // columns: rows of B that are there (K or fewer: A has zeros beyond)
  int lda, ldb;                     // elements from one row (of columns: term) to the next
  int segments;
  int first, stages;                // of all segments' stages one behind the other, those that this tile takes
  ProductSegment s[3];
};

template <int BM_, int WM_, int WN_, bool COLUMNS_>
struct ProductTile {
  static constexpr int BM = BM_, BN = BM_, BK = kProductTerms, A_PLACES = 3, B_PLACES = 2, WM = WM_, WN = WN_, NW = WM * WN, NT = 64 * NW;
  static constexpr bool COLUMNS = COLUMNS_;
  static constexpr int WTM = BM / WM, WTN = BN / WN, TM = WTM / 16, TN = WTN / 16;       // 16 x 16 results of a wave
  static constexpr int ROW_BYTES = 2 * BK, A_BYTES = BM * ROW_BYTES, B_BYTES = BN * ROW_BYTES;
  static constexpr int B_AT = A_PLACES * A_BYTES;                              // of B's first place
  static constexpr int HALF_BYTES = B_BYTES / 2, COL_BYTES = BN;               // a term's columns of one set
  static constexpr int LDS_BYTES = B_AT + B_PLACES * B_BYTES, LOADS = A_BYTES / (NW * 1024);     // of an operand, wave and stage
  // epilogue: 32 rows of a wave's columns, fp32
  static constexpr int SLAB_PITCH = WTN + 4, SLAB_BYTES = 32 * SLAB_PITCH * 4;
  // columns: the 16-byte place of a term's row is XORed with this
  __device__ static constexpr unsigned spread(unsigned k) {
    return COL_BYTES == 256 ? (k & 3) << 2 | (k >> 2 & 2) : (k & 2) << 1 | (k >> 2 & 2);
  }
  static_assert(LOADS * NW * 1024 == A_BYTES && LOADS % 2 == 0 && NW * SLAB_BYTES <= LDS_BYTES, "load split, fragments, epilogue");
};
template <bool COLUMNS>
using BigProduct = ProductTile<256, 2, 4, COLUMNS>;
template <bool COLUMNS>
using MidProduct = ProductTile<128, 2, 2, COLUMNS>;

// The tile at (m0, n0) (columns: of either set n0[0], n0[1]) into acc.  acc[x][y], lane, register r: row 16 x + lane % 16 of the wave's, column
// 16 y + 4 (lane / 16) + r of its WTN: those of the tile from WTN (wave % WN) on, or half as many of each set.
template <class S, bool F16>
__device__ __forceinline__ void product_tile(const ProductShape& p, int m0, const int (&n0)[2], unsigned lds0, f32x4 (&acc)[S::TM][S::TN]) {
  constexpr int BK = S::BK;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  // ---- memory -> LDS
  const int chunk = (lane & 7) ^ ((4 * (wave & 1) + (lane >> 4)) & 7);         // 16-byte piece of a row's 64 terms
  const unsigned a_pitch = 2u * p.lda, b_pitch = 2u * p.ldb;
  unsigned va[S::LOADS], vb[S::LOADS];
#pragma unroll
  for (int l = 0; l < S::LOADS; ++l) {
    const unsigned row = 8 * (l * S::NW + wave) + (lane >> 3);
    va[l] = row * a_pitch + chunk * 16;
    if constexpr (S::COLUMNS) {
      constexpr int PIECES = S::COL_BYTES / 16;
      const unsigned k = (l % (S::LOADS / 2) * S::NW + wave) * (1024 / S::COL_BYTES) + lane / PIECES, at = lane % PIECES;
      const unsigned c = at ^ S::spread(k);
      const int col = n0[l / (S::LOADS / 2)] + 8 * (int)c;
      vb[l] = col < p.N ? k * b_pitch + 2u * col : OOB;
    } else {
      vb[l] = row * b_pitch + chunk * 16;
    }
  }
  const unsigned a_bytes = (unsigned)imin(p.M - m0, S::BM) * a_pitch;
  const unsigned b_bytes = S::COLUMNS ? 0 : (unsigned)imax(imin(p.N - n0[0], S::BN), 0) * b_pitch;
  const unsigned lds_ld = lds0 + wave * 1024;
  i32x4 ra, rb[2];
  const int per = (p.K + BK - 1) / BK;                             // stages of a segment
  struct Stream {                                                  // the stage to ask for next: segment, first term, place in LDS; how many there are
    int seg, k, place, left;
  } pa, pb;
  pa.seg = p.first >= per ? p.first >= 2 * per ? 2 : 1 : 0;
  pa.k = (p.first - pa.seg * per) * BK;
  pa.place = 0;
  pa.left = p.stages;
  pb = pa;
  pb.place = S::B_AT;
  auto scalar = [](i32x4 r) {
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __builtin_amdgcn_readfirstlane(r[i]);
    return r;
  };
  auto pick = [&](int seg, const void* first, const void* second, const void* third) {         // (an index would put them in memory)
    return static_cast<const char*>(seg == 0 ? first : seg == 1 ? second : third);
  };
  auto open_a = [&]() {
    ra = make_rsrc(pick(pa.seg, p.s[0].a, p.s[1].a, p.s[2].a) + (uint64_t)m0 * a_pitch, pa.left > 0 ? a_bytes : 0);
  };
  auto open_b = [&]() {
    const char* const b0 = pick(pb.seg, p.s[0].b0, p.s[1].b0, p.s[2].b0);
    if constexpr (S::COLUMNS) {
      rb[0] = make_rsrc(b0 + (uint64_t)pb.k * b_pitch, 0);
      rb[1] = make_rsrc(pick(pb.seg, p.s[0].b1, p.s[1].b1, p.s[2].b1) + (uint64_t)pb.k * b_pitch, 0);
    } else {
      rb[0] = make_rsrc(b0 + (uint64_t)n0[0] * b_pitch, pb.left > 0 ? b_bytes : 0);
    }
  };
  auto open_terms = [&]() {                                        // columns: terms pb.k .. of the segment that are there
    if constexpr (S::COLUMNS) rb[0][2] = rb[1][2] = (int)(pb.left > 0 ? (unsigned)imax(imin(p.terms - pb.k, BK), 0) * b_pitch : 0);
  };
  auto prefetch_a = [&](int l) {
    load_to_lds(scalar(ra), pa.k + 8 * chunk < p.K ? va[l] : OOB, 2u * pa.k, lds_ld + pa.place + l * S::NW * 1024);
  };
  auto prefetch_b = [&](int l) {
    if constexpr (S::COLUMNS)
      load_to_lds(scalar(rb[l / (S::LOADS / 2)]), vb[l], 0, lds_ld + pb.place + l * S::NW * 1024);
    else
      load_to_lds(scalar(rb[0]), pb.k + 8 * chunk < p.K ? vb[l] : OOB, 2u * pb.k, lds_ld + pb.place + l * S::NW * 1024);
  };
  auto advance_a = [&]() {
    pa.place = pa.place == 2 * S::A_BYTES ? 0 : pa.place + S::A_BYTES;
    pa.k += BK;
    --pa.left;
    if (pa.k >= p.K || pa.left <= 0) {
      pa.k = 0;
      ++pa.seg;
      open_a();
    }
  };
  auto advance_b = [&]() {
    pb.place = 2 * S::B_AT + S::B_BYTES - pb.place;
    pb.k += BK;
    if constexpr (S::COLUMNS) {
#pragma unroll
      for (int l = 0; l < 2; ++l) {
        const uint64_t q = ((uint64_t)(uint32_t)rb[l][1] << 32 | (uint32_t)rb[l][0]) + (uint64_t)BK * b_pitch;
        rb[l][0] = (int)(uint32_t)q;
        rb[l][1] = (int)(uint32_t)(q >> 32);
      }
    }
    --pb.left;
    if (pb.k >= p.K || pb.left <= 0) {
      pb.k = 0;
      ++pb.seg;
      open_b();
    }
    open_terms();
  };

  // ---- LDS -> operands
  const int row = lane & 15, wm = wave / S::WN * S::WTM, wc = wave % S::WN;
  unsigned a_rd[2], b_rd[2];
#pragma unroll
  for (int ks = 0; ks < 2; ++ks) {
    const unsigned place = (unsigned)((4 * ks + (lane >> 4)) ^ (row >> 1)) << 4;
    a_rd[ks] = lds0 + (wm + row) * S::ROW_BYTES + place;
    if constexpr (S::COLUMNS) {
      const int k = 8 * (lane >> 4) + (row >> 2);
      const unsigned c = (unsigned)(S::WTN / 2 * wc + 4 * (row & 3)) >> 3;
      b_rd[ks] = lds0 + S::B_AT + (32 * ks + k) * S::COL_BYTES + ((c ^ S::spread(k)) << 4) + 8 * (row & 1);
    } else {
      b_rd[ks] = lds0 + S::B_AT + (S::WTN * wc + row) * S::ROW_BYTES + place;
    }
  }
#pragma unroll
  for (int x = 0; x < S::TM; ++x)
#pragma unroll
    for (int y = 0; y < S::TN; ++y) acc[x][y] = f32x4{0.f, 0.f, 0.f, 0.f};
  // B's operands of a k-step of 32 and the next; A's, each used by four instructions in a row, AHEAD of their use.
  constexpr int AHEAD = 3;
  Frag fa[4], fb[2][S::TN];
  typedef __attribute__((address_space(3))) const bf16x8* Lds;
  auto read_a = [&](int x, unsigned base, int ks) { fa[x & 3].v = *(Lds)(uintptr_t)(a_rd[ks] + base + x * 16 * S::ROW_BYTES); };
  auto read_b = [&](int y, unsigned base, int ks) {
    if constexpr (S::COLUMNS) {
      // 16 columns further within a set are two places, in bits that the lane's own place has as the XOR by k alone left them
      const unsigned at = ((b_rd[ks] + base) ^ (y % (S::TN / 2) << 5)) + y / (S::TN / 2) * S::HALF_BYTES;
      fb[ks][y].h[0] = lds_read_tr(at);
      fb[ks][y].h[1] = lds_read_tr(at + 4 * S::COL_BYTES);
    } else {
      fb[ks][y].v = *(Lds)(uintptr_t)(b_rd[ks] + base + y * 16 * S::ROW_BYTES);
    }
  };

  open_a();
  open_b();
  open_terms();
#pragma unroll
  for (int q = 0; q < 5; ++q) {                                    // A 0, B 0, A 1, B 1, A 2
#pragma unroll
    for (int l = 0; l < S::LOADS; ++l) {
      if (q & 1)
        prefetch_b(l);
      else
        prefetch_a(l);
    }
    if (q & 1)
      advance_b();
    else
      advance_a();
  }
  asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(3 * S::LOADS) : "memory");
#pragma unroll
  for (int y = 0; y < S::TN; ++y) read_b(y, 0, 0);
#pragma unroll
  for (int x = 0; x < AHEAD; ++x) read_a(x, 0, 0);
  // SPLIT: barriers M and E; else one, of both (small tiles: a few instructions lie between the two).
  constexpr bool SPLIT = S::TM > 4;
  constexpr int TURN = S::TM - AHEAD;                              // from this row on operands of the next k-step
  unsigned a_base = 0, b_base = 0;
  for (int st = 0; st < p.stages; ++st) {
    asm("" : "+s"(a_base), "+s"(b_base));
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
      for (int x = 0; x < S::TM; ++x) {
        if (SPLIT && ks == 1 && x == 1) asm volatile("s_waitcnt lgkmcnt(1)\n\ts_barrier" ::: "memory");      // one of A's is younger
        if (ks == 1 && x == TURN) {
          asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((SPLIT ? 2 : 1) * S::LOADS) : "memory");
          a_base = a_base == 2 * S::A_BYTES ? 0 : a_base + S::A_BYTES;
          b_base = S::B_BYTES - b_base;
          asm("" : "+s"(a_base), "+s"(b_base));
        }
        DP_PIN();
#pragma unroll
        for (int y = 0; y < S::TN; ++y) {
          acc[x][y] = mfma16<F16>(fb[ks][y].v, fa[x & 3].v, acc[x][y]);
          DP_PIN();
          if (y == 0) read_a((x + AHEAD) % S::TM, a_base, x >= TURN ? ks ^ 1 : ks);
          constexpr int SLOTS = AHEAD * S::TN;
          const int slot = (x - TURN) * S::TN + y;                 // of the last AHEAD rows
          // B's of the next k-step, each behind an instruction that reads none of A's
          if (x >= TURN && y != 0) {
            const int from = (slot - (x - TURN) - 1) * S::TN / (SLOTS - AHEAD), to = (slot - (x - TURN)) * S::TN / (SLOTS - AHEAD);
#pragma unroll
            for (int b = from; b < to; ++b) read_b(b, b_base, ks ^ 1);
          }
          // loads: B's behind M (or E), A's behind E
          if (SPLIT && ks == 1 && x >= 1 && x < 1 + S::LOADS && y == 2) {
            prefetch_b(x - 1);
            if (x == S::LOADS) advance_b();
          }
          if (ks == 1 && x >= TURN) {
            constexpr int LOADS = (SPLIT ? 1 : 2) * S::LOADS;
#pragma unroll
            for (int e = slot * LOADS / SLOTS; e < (slot + 1) * LOADS / SLOTS; ++e) {
              if (SPLIT || e >= S::LOADS)
                prefetch_a(e % S::LOADS);
              else
                prefetch_b(e);
            }
            if (slot == SLOTS - 1) {
              if (!SPLIT) advance_b();
              advance_a();
            }
          }
          DP_PIN();
        }
      }
    }
  }
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");      // loads past the end
  __syncthreads();
}

// acc's rows to store(row of the tile, column, set, values, ahead): columns 8 at a time, of both sets where PAIRS (v[0] and v[1]), else of one
// (v[0]).  The wave's 32 rows at a time are turned in LDS, so that whole rows leave.  ahead: what load(row, column, set) brought for this place,
// asked for 32 rows before.  across(first row, column, values): the same by columns, rows 8 at a time, where `mirror`.
struct NoMirror {
  __device__ void operator()(int, int, const float (&)[8]) const {}
};
struct Nothing {};
struct NoLoad {
  __device__ Nothing operator()(int, int, int) const { return {}; }
};
template <class S, bool PAIRS, class Load, class Store, class Across = NoMirror>
__device__ __forceinline__ void product_rows(const f32x4 (&acc)[S::TM][S::TN], unsigned lds0, Load load, Store store, bool mirror = false,
                                             Across across = {}) {
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / S::WN * S::WTM, wc = wave % S::WN;
  const unsigned slab = lds0 + wave * S::SLAB_BYTES;
  typedef __attribute__((address_space(3))) f32x4* Lds;
  constexpr int LANES = S::WTN / (PAIRS ? 16 : 8), PASSES = 32 * LANES / 64, HALF = S::WTN / 2;
  const int c = 8 * (lane % LANES), set = S::COLUMNS && !PAIRS ? c / HALF : 0;
  const int col = S::COLUMNS ? HALF * wc + c % HALF : S::WTN * wc + c;       // within a set, or within the tile
  auto row_of = [&](int x, int i) { return 32 * x + i * (64 / LANES) + lane / LANES; };
  decltype(load(0, 0, 0)) ahead[2][PASSES];
#pragma unroll
  for (int i = 0; i < PASSES; ++i) ahead[0][i] = load(wm + row_of(0, i), col, set);
#pragma unroll
  for (int x = 0; x < S::TM / 2; ++x) {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int y = 0; y < S::TN; ++y)
        *(Lds)(uintptr_t)(slab + 4 * ((16 * h + (lane & 15)) * S::SLAB_PITCH + 16 * y + 4 * (lane >> 4))) = acc[2 * x + h][y];
    if (x + 1 < S::TM / 2)
#pragma unroll
      for (int i = 0; i < PASSES; ++i) ahead[(x + 1) & 1][i] = load(wm + row_of(x + 1, i), col, set);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      float v[2][8];
#pragma unroll
      for (int s = 0; s < (PAIRS ? 2 : 1); ++s)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const f32x4 w = *(Lds)(uintptr_t)(slab + 4 * ((row_of(0, i)) * S::SLAB_PITCH + HALF * s + c + 4 * h));
#pragma unroll
          for (int e = 0; e < 4; ++e) v[s][4 * h + e] = w[e];
        }
      store(wm + row_of(x, i), col, set, v, ahead[x & 1][i]);
    }
    if (!std::is_same_v<Across, NoMirror> && mirror) {
#pragma unroll
      for (int i = 0; i < S::WTN / 16; ++i) {                      // four lanes have the 32 rows of a column
        const int r = 8 * (lane & 3), at = 16 * i + (lane >> 2);
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
          v[e] = *(__attribute__((address_space(3))) const float*)(uintptr_t)(slab + 4 * ((r + e) * S::SLAB_PITCH + at));
        across(wm + 32 * x + r, S::WTN * wc + at, v);
      }
    }
  }
}

}  // namespace dpbk
