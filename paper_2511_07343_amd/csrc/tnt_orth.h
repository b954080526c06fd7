// Orthogonalised update: argument block and launchers.  Internal to the library.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace tnt {

constexpr int ORTH_MAX_STEPS = 16;
constexpr int ORTH_PART = 256;  // partial sums of a matrix's norm, at most
constexpr int ORTH_TILE = 64;   // sides of the tiles of the products of large matrices

struct OrthArgs {
  const void* G;
  void* out;
  int64_t gb, gr, ob, orow;  // element strides of matrices and rows
  int n, rows, cols;
  int m, k;      // the shorter and the longer side
  int mp, kp;    // padded (matrices that do not fit one workgroup)
  // row pitches of the planes: 128 bytes past the padded side.  At a pitch of a power of
  // two the rows that a workgroup requests together lie in one channel of the cache
  int lm, lk;
  bool flip;     // rows > cols: the shorter side runs along the columns
  bool bf16;
  int steps;
  float eps, scale;
  float coef[3 * ORTH_MAX_STEPS];
  // workspace of the large form: two fp16 planes each
  int parts;         // of a matrix's norm
  double* part;      // [n][parts]
  _Float16 *X;       // [n][2][mp][lk]
  _Float16 *XT, *XT2;  // [n][2][kp][lm]
  _Float16 *A, *B;   // [n][2][mp][lm]
};

// one workgroup a matrix: fits its registers, and is the faster form
bool orth_small(int n, int m, int k);
hipError_t launch_orth_small(const OrthArgs& a, hipStream_t st);
hipError_t launch_orth_large(const OrthArgs& a, hipStream_t st);

}  // namespace tnt
