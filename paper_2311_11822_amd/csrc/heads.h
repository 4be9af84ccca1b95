// Launchers of what happens to heads between projection and attention (heads.hip).  They validate nothing.
#pragma once

#include "dp_internal.h"

namespace dpbk {

constexpr int kHeadsMaxWidth = 256, kHeadsMostSamples = 1 << 21;      // (a workgroup to a sample at least, and fewer than 2^32 threads)

struct HeadStrides {                 // elements from one sample, token, head to the next
  int64_t sample, token, head;
};
struct HeadsPlan {                   // a side's work
  int chunks, chunk_tokens;          // a sample's tokens by workgroup
  int block_tokens;                  // those whose angles are in LDS at a time
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
  float *partial, *kept, *sqnorm;    // backward pass of a norm: [B, chunks, D] of each side, [B, 2, D] ([B, 1, D] without keys), [B]; kept may be null
  HeadsPlan plan[2];
  unsigned begin;                    // first workgroup of the keys' side
  int lanes;                         // log2 of the lanes of a row
  int back;                          // rotations: the other way round
};
enum HeadsKind { kRotate, kNorm, kNormGrad };

// Chunks of all samples of a side are no more than this and one more for each.
constexpr int kHeadsChunks = 2048, kHeadsGradChunks = 768;
dp_status launch_heads(HeadsArgs a, dp_dtype dt, HeadsKind kind, hipStream_t s);

}  // namespace dpbk
