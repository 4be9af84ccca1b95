// Tiles of products on the 16-bit matrix instructions:  acc[m, n] = sum_s sum_k A_s[m, k] B_s[k, n]  over up to three segments s.
//
// A has its terms adjacent ([m][k]); B as well ([n][k], "rows"), or its columns ([k][n], "columns": two sets of them side by side, each with
// its own origin, which is how a gate and its factor meet in one lane).
//  * 256 x 256 tiles by eight waves of 128 x 64, or 128 x 128 by four of 64 x 64 (two workgroups to a compute unit).  Accumulators and
//    operands of one k-step and the next lie in registers.
//  * memory -> LDS without registers (16 bytes a lane), two stages of 64 terms: whole 128-byte lines of [m][k] rows.  (Stages of 32, five of
//    them, took each line in two halves a microsecond apart, and through the first-level cache twice: 4096 x 65536 x 12288 6050 us.)
//    One barrier to a stage, before its last k-step: the next stage has landed, and the last operands of this one are in registers, so
//    that its place is free; the loads of the stage after the next go out within that k-step and have three more to land.
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
struct ProductShape {
  int M, N, K;                      // K: of a segment; K and N (columns) are multiples of 8
  int terms;                        // columns: rows of B that are there (K or fewer: A has zeros beyond)
  int lda, ldb;                     // elements from one row (of columns: term) to the next
  int segments;
  ProductSegment s[3];
};

template <int BM_, int WM_, int WN_, bool COLUMNS_>
struct ProductTile {
  static constexpr int BM = BM_, BN = BM_, BK = 64, NSTAGE = 2, WM = WM_, WN = WN_, NW = WM * WN, NT = 64 * NW;
  static constexpr bool COLUMNS = COLUMNS_;
  static constexpr int WTM = BM / WM, TM = WTM / 32, TN = 2;
  static constexpr int ROW_BYTES = 2 * BK, A_BYTES = BM * ROW_BYTES, B_BYTES = BN * ROW_BYTES, STAGE_BYTES = A_BYTES + B_BYTES;
  static constexpr int HALF_BYTES = B_BYTES / 2, COL_BYTES = BN;               // a term's columns of one set
  static constexpr int LDS_BYTES = NSTAGE * STAGE_BYTES, LOADS = 4;            // of an operand, wave and stage
  // epilogue: a wave's 32 rows of 64 columns, fp32
  static constexpr int SLAB_PITCH = 68, SLAB_BYTES = 32 * SLAB_PITCH * 4;
  static_assert(BN / WN == 64 && LOADS * NW * 1024 == A_BYTES && NW * SLAB_BYTES <= LDS_BYTES, "load split, fragments, epilogue");
};
template <bool COLUMNS>
using BigProduct = ProductTile<256, 2, 4, COLUMNS>;
template <bool COLUMNS>
using MidProduct = ProductTile<128, 2, 2, COLUMNS>;

// The tile at (m0, n0) (columns: of either set n0[0], n0[1]) into acc.  acc[x][y], lane, register r: row 32 x + lane % 32 of the wave's, column
// 8 (r / 4) + 4 (lane / 32) + r % 4 of its fragment y: column 32 (wave % WN) of set y, or 64 (wave % WN) + 32 y of the tile.
template <class S, bool F16>
__device__ __forceinline__ void product_tile(const ProductShape& p, int m0, const int (&n0)[2], unsigned lds0, f32x16 (&acc)[S::TM][S::TN]) {
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
      const unsigned k = ((l & 1) * S::NW + wave) * (1024 / S::COL_BYTES) + lane / PIECES, at = lane % PIECES;
      const unsigned c = S::COL_BYTES == 256 ? at ^ ((k & 3) << 2) : at ^ ((k & 2) << 1);
      const int col = n0[l >> 1] + 8 * (int)c;
      vb[l] = col < p.N ? k * b_pitch + 2u * col : OOB;
    } else {
      vb[l] = row * b_pitch + chunk * 16;
    }
  }
  const unsigned a_bytes = (unsigned)imin(p.M - m0, S::BM) * a_pitch;
  const unsigned b_bytes = S::COLUMNS ? 0 : (unsigned)imax(imin(p.N - n0[0], S::BN), 0) * b_pitch;
  const unsigned lds_ld = lds0 + wave * 1024;
  i32x4 ra, rb[2];
  int p_seg = 0, p_k = 0, p_stage = 0;                             // of the stage to ask for next; its place
  auto scalar = [](i32x4 r) {
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __builtin_amdgcn_readfirstlane(r[i]);
    return r;
  };
  auto open_segment = [&]() {
    if (p_seg < p.segments) {
      const auto pick = [&](const void* first, const void* second, const void* third) {        // (an index would put them in memory)
        return p_seg == 0 ? first : p_seg == 1 ? second : third;
      };
      const ProductSegment s = {pick(p.s[0].a, p.s[1].a, p.s[2].a), pick(p.s[0].b0, p.s[1].b0, p.s[2].b0), pick(p.s[0].b1, p.s[1].b1, p.s[2].b1)};
      ra = make_rsrc(static_cast<const char*>(s.a) + (uint64_t)m0 * a_pitch, a_bytes);
      if constexpr (S::COLUMNS) {
        rb[0] = make_rsrc(s.b0, 0);
        rb[1] = make_rsrc(s.b1, 0);
      } else {
        rb[0] = make_rsrc(static_cast<const char*>(s.b0) + (uint64_t)n0[0] * b_pitch, b_bytes);
      }
    } else {
      ra[2] = rb[0][2] = 0;
    }
    ra = scalar(ra);
    rb[0] = scalar(rb[0]);
    if constexpr (S::COLUMNS) rb[1] = scalar(rb[1]);
  };
  auto open_block = [&]() {                                        // columns: terms p_k .. of the segment that are there
    if constexpr (S::COLUMNS) {
      const unsigned n = p_seg < p.segments ? (unsigned)imax(imin(p.terms - p_k, BK), 0) * b_pitch : 0;
      rb[0][2] = rb[1][2] = (int)n;
    }
  };
  auto prefetch_a = [&](int l) {
    load_to_lds(scalar(ra), p_k + 8 * chunk < p.K ? va[l] : OOB, 2u * p_k, lds_ld + p_stage + l * S::NW * 1024);
  };
  auto prefetch_b = [&](int l) {
    if constexpr (S::COLUMNS)
      load_to_lds(scalar(rb[l >> 1]), vb[l], 0, lds_ld + p_stage + S::A_BYTES + l * S::NW * 1024);
    else
      load_to_lds(scalar(rb[0]), p_k + 8 * chunk < p.K ? vb[l] : OOB, 2u * p_k, lds_ld + p_stage + S::A_BYTES + l * S::NW * 1024);
  };
  auto prefetch_advance = [&]() {
    p_stage = S::STAGE_BYTES - p_stage;
    p_k += BK;
    if constexpr (S::COLUMNS) {
#pragma unroll
      for (int l = 0; l < 2; ++l) {
        const uint64_t q = ((uint64_t)(uint32_t)rb[l][1] << 32 | (uint32_t)rb[l][0]) + (uint64_t)BK * b_pitch;
        rb[l][0] = (int)(uint32_t)q;
        rb[l][1] = (int)(uint32_t)(q >> 32);
      }
    }
    if (p_k >= p.K) {
      p_k = p_seg + 1 < p.segments ? 0 : p_k;
      ++p_seg;
      open_segment();
    }
    open_block();
  };

  // ---- LDS -> operands
  const int row = lane & 31, sw = (row >> 1) & 7, wm = wave / S::WN * S::WTM, wc = wave % S::WN;
  unsigned a_rd[4], b_rd[4];
#pragma unroll
  for (int ks = 0; ks < 4; ++ks) {
    const unsigned place = (unsigned)((2 * ks + (lane >> 5)) ^ sw) << 4;
    a_rd[ks] = lds0 + (wm + row) * S::ROW_BYTES + place;
    if constexpr (S::COLUMNS) {
      const int blk = lane >> 4, s = lane & 15, k = 8 * (blk >> 1) + (s >> 2);
      const unsigned c = (unsigned)(32 * wc + 16 * (blk & 1) + 4 * (s & 3)) >> 3;
      const unsigned at = S::COL_BYTES == 256 ? c ^ ((k & 3) << 2) : c ^ ((k & 2) << 1);
      b_rd[ks] = lds0 + S::A_BYTES + (16 * ks + k) * S::COL_BYTES + (at << 4) + 8 * (s & 1);
    } else {
      b_rd[ks] = lds0 + S::A_BYTES + (64 * wc + row) * S::ROW_BYTES + place;
    }
  }
#pragma unroll
  for (int x = 0; x < S::TM; ++x)
#pragma unroll
    for (int y = 0; y < S::TN; ++y)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[x][y][r] = 0.f;
  Frag fa[2][S::TM], fb[2][S::TN];
  typedef __attribute__((address_space(3))) const bf16x8* Lds;
  // Items of a k-step's operands in the order in which its matrix instructions need them: B 0, A 0, B 1, A 1 ...
  auto read_frag = [&](int buf, int q, unsigned base, int ks) {
    const bool is_b = q == 0 || q == 2;
    const int i = is_b ? q >> 1 : q == 1 ? 0 : q - 2;
    if (!is_b) {
      fa[buf][i].v = *(Lds)(uintptr_t)(a_rd[ks] + base + i * 32 * S::ROW_BYTES);
    } else if constexpr (S::COLUMNS) {
      const unsigned at = b_rd[ks] + base + i * S::HALF_BYTES;
      fb[buf][i].h[0] = lds_read_tr(at);
      fb[buf][i].h[1] = lds_read_tr(at + 4 * S::COL_BYTES);
    } else {
      fb[buf][i].v = *(Lds)(uintptr_t)(b_rd[ks] + base + i * 32 * S::ROW_BYTES);
    }
  };
  constexpr int ITEMS = S::TM + S::TN, STEPS = S::TM * S::TN;

  const int stages = p.segments * ((p.K + BK - 1) / BK);
  open_segment();
  open_block();
#pragma unroll
  for (int q = 0; q < 2; ++q) {
#pragma unroll
    for (int l = 0; l < S::LOADS; ++l) {
      prefetch_a(l);
      prefetch_b(l);
    }
    prefetch_advance();
    if (q == 0) asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
  }
#pragma unroll
  for (int q = 0; q < ITEMS; ++q) read_frag(0, q, 0, 0);
  unsigned c_base = 0;
  for (int st = 0; st < stages; ++st) {
    asm("" : "+s"(c_base));
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      if (ks == 3) {                                               // the next stage is there, this one's operands are in registers
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        c_base = S::STAGE_BYTES - c_base;
        asm("" : "+s"(c_base));
      }
      DP_PIN();
#pragma unroll
      for (int slot = 0; slot < STEPS; ++slot) {
        const int x = slot / S::TN, y = slot % S::TN;
        acc[x][y] = mfma16<F16>(fb[ks & 1][y].v, fa[ks & 1][x].v, acc[x][y]);
        DP_PIN();
        if (slot < ITEMS) read_frag(~ks & 1, slot, c_base, (ks + 1) & 3);
        if (ks == 3) {
          constexpr int PER = 2 * S::LOADS / STEPS;
#pragma unroll
          for (int e = slot * PER; e < slot * PER + PER; ++e) {
            if (e & 1)
              prefetch_b(e >> 1);
            else
              prefetch_a(e >> 1);
          }
          if (slot == STEPS - 1) prefetch_advance();
        }
        DP_PIN();
      }
    }
  }
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");      // loads past the end
  __syncthreads();
}

// acc's rows to store(row of the tile, first column, values): columns 8 at a time, of both sets where PAIRS (v[0] and v[1]), else of one
// fragment (v[0]).  The wave's 32 rows at a time are turned in LDS, so that whole rows leave.  across(first row, column, values): the same
// by columns, rows 8 at a time, where `mirror`.
struct NoMirror {
  __device__ void operator()(int, int, const float (&)[8]) const {}
};
template <class S, bool PAIRS, class Store, class Across = NoMirror>
__device__ __forceinline__ void product_rows(const f32x16 (&acc)[S::TM][S::TN], unsigned lds0, Store store, bool mirror = false,
                                             Across across = {}) {
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / S::WN * S::WTM, wc = wave % S::WN;
  const unsigned slab = lds0 + wave * S::SLAB_BYTES;
  typedef __attribute__((address_space(3))) f32x4* Lds;
#pragma unroll
  for (int x = 0; x < S::TM; ++x) {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int y = 0; y < S::TN; ++y)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 v = {acc[x][y][4 * g], acc[x][y][4 * g + 1], acc[x][y][4 * g + 2], acc[x][y][4 * g + 3]};
        *(Lds)(uintptr_t)(slab + 4 * ((lane & 31) * S::SLAB_PITCH + 32 * y + 8 * g + 4 * (lane >> 5))) = v;
      }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    constexpr int LANES = PAIRS ? 4 : 8, PASSES = 32 * LANES / 64;
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      const int r = i * (64 / LANES) + lane / LANES, c = 8 * (lane % LANES);
      float v[2][8];
#pragma unroll
      for (int s = 0; s < (PAIRS ? 2 : 1); ++s)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const f32x4 w = *(Lds)(uintptr_t)(slab + 4 * (r * S::SLAB_PITCH + 32 * s + c + 4 * h));
#pragma unroll
          for (int e = 0; e < 4; ++e) v[s][4 * h + e] = w[e];
        }
      // column within a set, or within the tile
      const int col = S::COLUMNS ? 32 * wc + c % 32 : 64 * wc + c;
      store(wm + 32 * x + r, col, S::COLUMNS && !PAIRS ? c / 32 : 0, v);
    }
    if (!std::is_same_v<Across, NoMirror> && mirror) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
          v[e] = *(__attribute__((address_space(3))) const float*)(uintptr_t)(slab + 4 * ((8 * i + e) * S::SLAB_PITCH + lane));
        across(wm + 32 * x + 8 * i, 64 * wc + lane, v);
      }
    }
  }
}

}  // namespace dpbk
