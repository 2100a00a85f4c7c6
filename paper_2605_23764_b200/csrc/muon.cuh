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
// From the fourth step on (MUON_SHIFT) the larger singular values have come near 1.  B's diagonal is near b + c there, which a X mostly cancels:
// three quarters of it move from B to the linear term, X <- (a - s) X + (B + s I) X with s = -3/4 (b + c).  Errors halve: 1.6e-3 -> 0.9e-3
// on normally distributed matrices, five steps.  The product takes s of X's hi alone, so lo enters the linear term with a.
//
// X's lo part is left out of the last steps (MuonArgs::late).  What rounding X to hi adds to a small singular value grows by |a| a step, so a
// step can do without lo where the products of the |a| left, from its own and every later step's to the last's, sum up to MUON_GROWTH: two
// of five steps of (3.4445, -4.7750, 2.0315), 15.3 (0.9e-3 instead of 0.8e-3, 1.8e-3 instead of 1.3e-3 for the rank of 256), never the first three.
// Left out from the fourth step on whatever follows, with the shift's s of hi alone, matrices of rank 64, 256 x 400, were 1.6e-2 off
// after seven such steps and 3.9e-2 after twelve of (1.875, -1.25, 0.375), 1.7e-3 and 1.3e-3 this way.
#pragma once

#include "moe_internal.h"

namespace moe {

constexpr float MUON_SX = 4096.f, MUON_SA = 4096.f, MUON_SB = 1024.f, MUON_SLO = 2048.f;
constexpr int MUON_STEPS_MAX = 16;
constexpr int MUON_SHIFT = 3;          // first step (from 0) with the shifted diagonal
constexpr double MUON_GROWTH = 16.0;   // see above

enum MuonPhase : int {
  MUON_GRAM = 0,    // A = X X^T or X^T X, or sums over parts of the reduction
  MUON_JOIN = 1,    // A from those
  MUON_POLY = 2,    // B = b A + c A A + s I
  MUON_APPLY = 3,   // X' = (a - s) X + s lo + B X or X B; of the last step: into the caller's tensors
};

// A symmetric matrix is stored by blocks of 256 x 256, those on and below the diagonal.
constexpr int MUON_BLOCK = 256;

struct MuonArgs {
  // X, by buffer: K-major operands (128 rows x 64; half a tile's columns x 64), MN-major operand (64 x 64), epilogue boxes (32 rows x 32)
  // of hi and lo; A and B likewise
  CUtensorMap x128[2], x_part[2], x64[2], xhi[2], xlo[2];
  CUtensorMap a128, a_part, a64, abox, b128, b_part, b64, bbox;
  CUtensorMap out, w;          // the caller's tensors by epilogue boxes (vec)
  CUtensorMap part;            // GRAM's sums over parts [tile of a matrix][part][256][nt_tri] in fp32, boxes of 32 x 32
  int n, rows, cols;           // matrices of the batch
  int steps;
  int nt_tri, nt_app;          // columns of a tile: 64, 128 or 256; APPLY's also 192 in wide matrices
  int split, strips;           // parts of GRAM's reduction (1: no JOIN); strips of a tile's rows that JOIN's items are
  const float* part_ptr;
  uint16_t* a_ptr;             // A, rows lda apart
  int lda;
  int sub;                     // matrices whose phases follow one another
  int z0;                      // the batch's first matrix in the caller's tensors
  int late;                    // first step that goes by X's hi part alone
  // factors in the stored scalings; app_in: of X (hi + lo), app_rest: of lo besides (0 without a shift)
  struct Step { float gram_acc, poly_acc, poly_in, poly_diag, app_acc, app_in, app_rest; } step[MUON_STEPS_MAX];
  // the last step's X': out = X', or with W: out = keep W - rate X'
  uint16_t* out_ptr;           // bf16 [rows][cols] of the batch's first matrix
  const uint16_t* w_ptr;       // NULL: none
  float keep, rate;
  int vec;                     // rows of both are whole 16-byte vectors
  int* ctr;                    // [n] finished warps' parts of tiles of each matrix, [n]: next item; zero before the launch
  DevStatus* status;
  uint64_t budget_ns;
};
// One persistent launch for all products of a batch; wide: rows <= cols
cudaError_t launch_muon_products(bool wide, const MuonArgs& a, int num_sms, cudaStream_t s);

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
  int* ctr;             // [n + 1] cleared on the way
};
// Elements of a part, of vectors and of single ones: a few turns of a block's threads (with 32768, 16 matrices 128 x 256 took 10 us longer)
constexpr long MUON_PART_VEC = 8192, MUON_PART_ONE = 2048;
inline long muon_parts(long elems, bool vec) { return (elems + (vec ? MUON_PART_VEC : MUON_PART_ONE) - 1) / (vec ? MUON_PART_VEC : MUON_PART_ONE); }
// M_out = mu M + G, u = G + mu M_out (nesterov) or M_out; sums of u's squares
cudaError_t launch_muon_momentum(const MuonElemArgs& a, cudaStream_t s);
// X = u / (norm + eps)
cudaError_t launch_muon_normalize(const MuonElemArgs& a, cudaStream_t s);

// Small matrices: everything of one in one block (muon_small.cu), no workspace but the status
constexpr int MUON_SMALL_M = 128, MUON_SMALL_L = 384;
inline bool muon_is_small(int rows, int cols) {
  return (rows < cols ? rows : cols) <= MUON_SMALL_M && (rows < cols ? cols : rows) <= MUON_SMALL_L;
}
struct MuonSmallArgs {
  MuonElemArgs e;
  int steps;
  MuonArgs::Step step[MUON_STEPS_MAX];   // app_in: a - s; app_rest: s in steps that are not late
  uint16_t* out;
  const uint16_t* W;    // NULL: out = X'
  float keep, rate;
  int vec;              // rows of everything are whole vectors of eight elements
  DevStatus* status;
  uint64_t budget_ns;
};
cudaError_t launch_muon_small(const MuonSmallArgs& a, cudaStream_t s);

}  // namespace moe
