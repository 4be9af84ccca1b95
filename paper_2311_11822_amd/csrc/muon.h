// Launcher of the optimizer that orthogonalises its update (muon.hip).  It validates nothing.
#pragma once

#include "dp_internal.h"

namespace dpbk {

constexpr int kMuonGroup = 64;             // tensors of a launch: 6 KiB of kernel arguments
constexpr int kMuonParts = 1024;           // partial sums of a tensor's square, at most
constexpr int kMuonMostSide = 1 << 20, kMuonMostShort = 1 << 16;
constexpr float kMuonMost = 15.f;          // values that 2^12 of still fit fp16

constexpr int kMuonMostIterations = 32;
constexpr int kMuonSmallTiles = 6;         // sixteens of the shorter side of matrices that one workgroup holds

struct MuonTensor {
  float* param;
  const void* grad;
  float* momentum;
  void* copy;
  int rows, cols;
  float keep, rate;                        // 1 - lr * weight decay, lr * scale
};
struct MuonArgs {
  float beta, ahead, grad_scale, eps;      // u = g + ahead m, or m (ahead < 0)
  int iterations;
  const double* coefficients;              // HOST, [iterations][3]
};

// Matrices that one workgroup holds (muon_small.hip), of one run; they use no workspace.
bool muon_is_small(int rows, int cols);
dp_status launch_muon_small(const MuonTensor* tensors, int n, const MuonArgs& a, dp_dtype grad_dt, dp_dtype copy_dt, hipStream_t s);
// Of one run of up to kMuonGroup matrices.
struct MuonLaunches {
  int side, parts;                                     // of a step's tiles, and the workgroups that share one
};
void muon_launches(const MuonTensor* tensors, int n, MuonLaunches (&steps)[3]);                     // A, its polynomial, the update
size_t muon_workspace(const MuonTensor* tensors, int n);
dp_status launch_muon(const MuonTensor* tensors, int n, const MuonArgs& a, dp_dtype grad_dt, dp_dtype copy_dt, void* ws, hipStream_t s);

}  // namespace dpbk
