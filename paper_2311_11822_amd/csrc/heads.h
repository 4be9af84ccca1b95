// Launchers of what happens to heads between projection and attention (heads.hip).  They validate nothing.
#pragma once

#include "dp_internal.h"

namespace dpbk {

constexpr int kHeadsMaxWidth = 256;

struct HeadStrides {                 // elements from one sample, token, head to the next
  int64_t sample, token, head;
};
struct HeadsArgs {
  const void* in[2];                 // queries and keys, [1] null: queries alone; in the backward pass of a norm: what was normalised
  const void* dy[2];                 // backward pass of a norm: gradients of the results
  void* out[2];
  const float* gain[2];              // norms; null: ones
  HeadStrides in_stride[2], dy_stride[2], out_stride[2];
  int heads[2];
  int B, T, D;
  int turn, interleaved;             // columns that turn
  float amplitude, eps;
  const double* turns;               // [turn / 2]
  const int32_t *position, *len;     // [B, T], [B]; or null
  float *partial, *kept, *sqnorm;    // backward pass of a norm: [B, chunks, 2, D], [B, 2, D] ([B, 1, D] without keys), [B]; kept may be null
  int chunks, chunk_tokens;          // a sample's tokens by workgroup
  int block_tokens;                  // those whose angles are in LDS at a time
  int lanes;                         // log2 of the lanes of a row
  int back;                          // rotations: the other way round
};
enum HeadsKind { kRotate, kNorm, kNormGrad };

// Fills in chunks, chunk_tokens, block_tokens and lanes; `vec` comes out as the values of an access.
void heads_layout(HeadsArgs& a, dp_dtype dt, HeadsKind kind, int& vec);
dp_status launch_heads(HeadsArgs a, dp_dtype dt, HeadsKind kind, hipStream_t s);

}  // namespace dpbk
