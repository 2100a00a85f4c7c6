// Orthogonalised momentum (moe_muon_*): X <- a X + b A X + c A A X with A = X X^T (X^T X where a matrix is taller than wide), a few
// times over, for a batch of matrices.  muon.cu: the passes over single elements; muon_gemm.cu: the products.
//
// How X, A and B = b A + c A A are held.  The products' operands are fp16 (11 significant bits at the rate of bf16), scaled by powers
// of two so that entries of matrices whose singular values are at most 1 or so lie in its range.  X itself is held in two fp16
// numbers, hi + lo / 2048 (22 bits): a product takes hi, the linear term a X both.  What rounding hi costs a product is relative
// to the LARGE singular values, and the linear term is what carries the small ones, by a factor a a step; with hi alone there, what
// 2^-12 of the largest entries adds to a small singular value grows with it: matrices of rank 256 + rounding, 512 x 768, were 6.8e-3
// off in the norm after five steps, with both 1.3e-3 (bf16 operands and X: 5.4e-2).
//
// Once the singular values have come near 1 (from the fourth step on), B's diagonal is near b + c, which a X mostly cancels: there
// three quarters of it move from B to the linear term, X <- (a - s) X + (B + s I) X with s = -3/4 (b + c).  Errors halve: 1.6e-3 ->
// 0.9e-3 on normally distributed matrices.
#pragma once

#include "moe_internal.h"

namespace moe {

constexpr float MUON_SX = 4096.f, MUON_SA = 4096.f, MUON_SB = 1024.f, MUON_SLO = 2048.f;
constexpr int MUON_SHIFT_FROM = 3;   // first step (from 0) with the shifted diagonal

enum MuonProduct : int {
  MUON_GRAM = 0,    // A = X X^T or X^T X
  MUON_POLY = 1,    // B = b A + c A A + s I
  MUON_APPLY = 2,   // X' = (a - s) X + B X or X B
  MUON_LAST = 3,    // the same of the last step: into the caller's tensors
};

// What is done with the last step's X'
struct MuonFinish {
  uint16_t* out;         // bf16 [n][rows][cols], W' or X' itself
  const uint16_t* W;     // W' = keep W - rate X'; NULL: out = X'
  float keep, rate;
  int vec;               // rows of out (and W) are whole 16-byte vectors
};

struct MuonProductArgs {
  CUtensorMap tmA, tmB;        // operands: boxes of 64 k x 128 rows (K-major) or 64 columns x 64 k (MN-major)
  CUtensorMap tmIn0, tmIn1;    // epilogue: boxes of 32 rows x 64 columns of A (POLY) or X hi, X lo (APPLY)
  CUtensorMap tmOut0, tmOut1;  // GRAM, POLY: the product, and mirrored (boxes of 64 x 32, not swizzled); APPLY: X' hi, X' lo
  int n, M, N, K;              // matrices; sizes of the product
  int nt;                      // columns of a tile: 128, 192 or 256
  int ld;                      // GRAM, POLY: elements from row to row of the product
  uint16_t* out;               // GRAM, POLY: the product
  float k_acc, k_in, k_diag;   // factors of the accumulator, of what the epilogue reads, on the diagonal; in the product's scaling
  MuonFinish fin;              // LAST
  DevStatus* status;
  uint64_t budget_ns;
};
// a_mn, b_mn: the operand's rows are the reduction
cudaError_t launch_muon_product(MuonProduct what, bool a_mn, bool b_mn, const MuonProductArgs& a, int num_sms, cudaStream_t s);

struct MuonElemArgs {
  const void* G;        // [n][rows][cols], bf16 or fp32
  int g_fp32;
  const float* M;       // momentum [n][rows][cols]; NULL: u = G
  float* M_out;
  float mu;
  int nesterov;
  long elems;           // rows * cols
  int n, rows, cols, ld;
  int vec;              // matrices and their rows are whole vectors of eight elements
  double* part;         // [n][parts] sums of squares
  int parts;
  float eps;
  uint16_t *hi, *lo;    // X [n][rows][ld]
};
constexpr long MUON_PART = 32768;   // elements of a part
inline long muon_parts(long elems) { return (elems + MUON_PART - 1) / MUON_PART; }
// M_out = mu M + G, u = G + mu M_out (nesterov) or M_out; sums of u's squares
cudaError_t launch_muon_momentum(const MuonElemArgs& a, cudaStream_t s);
// X = u / (norm + eps)
cudaError_t launch_muon_normalize(const MuonElemArgs& a, cudaStream_t s);

}  // namespace moe
