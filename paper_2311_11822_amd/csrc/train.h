// Launchers of what stands around the linear layers: layer norms (norm.hip) and the optimizer (adamw.hip).  They validate nothing.
#pragma once

#include "dp_internal.h"

namespace dpbk {

// Rows are held in registers; wider ones are refused.
constexpr int kNormMaxWidth = 32768;

struct NormArgs {
  const void *x, *dy, *add;      // forward: x, add; backward: x, dy, add; add may be null
  void *sum, *out;               // forward: x + add (or null) and y; backward: dx
  const float *gain, *bias;      // either may be null: ones, zeros
  float *mean, *rstd;            // forward: may be null
  float* kept;                   // backward: [B, 2, d], or null
  float* partial;                // backward: [B, chunks, 2, d] where chunks > 1
  float* sqnorm;                 // backward: [B] (with kept)
  int B, T, d;
  float eps;
  int chunks, chunk_rows;        // backward: a sample's rows by workgroup
};

dp_status launch_layer_norm(const NormArgs& a, dp_dtype dt, hipStream_t s);
// Workgroups to a sample; partial sums are needed where they are more than one.
int layer_norm_chunks(dp_dtype dt, int B, int T, int d);
dp_status launch_layer_norm_backward(NormArgs a, dp_dtype dt, hipStream_t s);

// sqnorm[i] = sum_k rows[i, k]^2 (bias.hip).
dp_status launch_row_sqnorm(const float* rows, int B, int p, float* sqnorm, hipStream_t s);

constexpr int kAdamTensors = 128;        // of a launch
constexpr int kAdamScaleBlock = 256;     // values to a scale of the 8-bit states
struct AdamTensor {
  float* param;
  const void* grad;
  void *m, *v;
  float *m_scale, *v_scale;
  void* copy;
  uint64_t n;
  float keep;                            // 1 - lr * weight decay
  int whole;                             // every array begins where its vector accesses may
};
struct AdamArgs {
  int n_tensors;
  unsigned first;                        // number of the launch's first workgroup
  float grad_scale, beta1, beta2, rest1, rest2;      // rest: 1 - beta
  float lr, fix1, fix2, eps;             // fix: 1 / (1 - beta^t)
  uint32_t dither;                       // step * 0x9E3779B1
  unsigned begin[kAdamTensors];          // first workgroup of a tensor
  AdamTensor t[kAdamTensors];
};
// Elements of a workgroup.
constexpr int kAdamChunk = 4096;
dp_status launch_adamw(const AdamArgs& a, int64_t blocks, dp_dtype grad_dt, int state_bits, int copy_dt, hipStream_t s);

}  // namespace dpbk
