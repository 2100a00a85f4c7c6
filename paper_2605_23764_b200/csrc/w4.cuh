// Expert weights in 4 bits with a scale -- and a zero point, where there are any -- for each group of 32, 64 or 128 reduction
// elements: w = s (q - z), q and z in 0 .. 15 (z = 8 without zero points), s in bf16.
//
// Layout.  A matrix of R rows (output features) and K columns (reduction) is cut into units of 32 rows x 128 columns, 2 KB each;
// four units below one another (128 rows, one copy for the tensor-core kernel) lie side by side, then the next 128 columns, then the
// next 128 rows.  A unit is cut into quarters of 16 rows x 64 columns (columns slow: first half's two, second half's two).  The 32 lanes of
// a warp own 16 bytes of a quarter side by side: word j of lane 4 g + c holds, of the quarter's columns 16 j .., what the lane is
// given of a 16 x 16 bf16 operand of a matrix instruction -- the pairs of columns {2 c, 2 c + 1} and {2 c + 8, 2 c + 9} of rows g
// and g + 8:
//   pair r (0: row g, first pair; 1: row g + 8, first; 2: row g, second; 3: row g + 8, second)
//   has its even column in bits 4 r + 3 .. 4 r + 6 and its odd column in bits 4 r + 19 .., counted round the word's end,
// so that (word rotated right by 4 r) & 0x00780078 is a pair in the place of the highest mantissa bits of two bf16 numbers: with the
// exponent of 16 they are 16 + q.  (In the lowest bits they would be 128 + q: what is taken off again would be five times as much.)
// The same fragment is what a warp writes to TMEM for 16 lanes x 8 columns (two bf16 each), so matrix-vector and tensor-core kernels
// read one layout.
// Scales [unit][8][groups of a unit][4] bf16 and zero points [..] bytes: lanes 4 g + c need rows {g, g + 8, g + 16, g + 24} of the unit's
// 1, 2 or 4 groups, side by side, in the same order of units.
// Rows of W_gate_up: of 16 rows, 0 .. 7 are gate rows, 8 .. 15 the up rows of the same features (SwiGLU needs no exchange).
// Rows behind the last are codes of value 0 with scale 0, columns behind K codes of value 0.
#pragma once

#include "moe_internal.h"

namespace moe {

constexpr int W4_TILE_ROWS = 32, W4_UNIT_K = 128, W4_UNIT_BYTES = 2048;

struct W4Shape {
  int rows, cols, group, paired;
  __host__ __device__ int row_tiles() const { return (rows + W4_TILE_ROWS - 1) / W4_TILE_ROWS; }   // that hold rows
  __host__ __device__ int stored_tiles() const { return (row_tiles() + 3) & ~3; }
  __host__ __device__ int units() const { return (cols + W4_UNIT_K - 1) / W4_UNIT_K; }   // of a row tile
  __host__ __device__ int unit_groups() const { return W4_UNIT_K / group; }
  // row of the matrix that is row r of tile rt; -1: behind the last
  __host__ __device__ int row_at(int rt, int r) const {
    const int sub = 2 * rt + (r >> 4);   // sixteen rows
    const int i = paired ? (sub * 8 < rows / 2 ? (r & 8 ? rows / 2 : 0) + sub * 8 + (r & 7) : rows) : sub * 16 + (r & 15);
    return i < rows ? i : -1;
  }
};

// The four registers of a 16 x 16 bf16 operand from a word of codes: 16 + q, the codes being the high mantissa bits.
constexpr uint32_t W4_MAGIC = 0x41804180u;
__device__ __forceinline__ uint32_t w4_pair(uint32_t word) {
  uint32_t r;
  asm("lop3.b32 %0, %1, 0x00780078, %2, 0xEA;" : "=r"(r) : "r"(word), "r"(W4_MAGIC));   // (word & mask) | magic
  return r;
}
__device__ __forceinline__ void w4_fragment(uint32_t word, uint32_t (&a)[4]) {
#pragma unroll
  for (int r = 0; r < 4; ++r) a[r] = w4_pair(r < 3 ? word >> (4 * r) : __funnelshift_r(word, word, 12));
}
// Unit ku of row tile rt of a matrix of KU units a row tile.
__host__ __device__ __forceinline__ int64_t w4_unit(int rt, int ku, int KU) { return ((int64_t)(rt >> 2) * KU + ku) * 4 + (rt & 3); }

// 16 + q less 16 + z: a whole number, exact.  A fused multiply-add by one: the subtraction of bf16 pairs is not one instruction here.
__host__ __device__ __forceinline__ uint32_t w4_bias(uint32_t z) { return 0xC180C180u | z * 0x00080008u; }   // - (16 + z), twice
__device__ __forceinline__ uint32_t add_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(0x3F803F80u), "r"(b));
  return r;
}
__device__ __forceinline__ float w4_offset(uint32_t z) { return __uint_as_float(0x41800000u | (z & 0xFu) << 19); }   // 16 + z

// One expert product of the layer over experts with few rows (w4_vec.cu).
struct W4VecArgs {
  const uint4* codes;
  const uint32_t* scales;     // bf16 pairs
  const uint16_t* zeros;      // byte pairs; NULL: 8
  int K, KU, RT, RTS, group;  // reduction, units of a row tile, row tiles of an expert that hold rows, that are stored
  int down;                   // 0: x -> A = w silu(gate) up; 1: A -> Y
  int n_out;                  // features of the result
  const uint16_t* in;         // x [T][in_ld] or A [rows][in_ld]
  int in_ld;
  uint16_t* A;                // rows a_ld apart
  int a_ld;
  float* Y;                   // rows y_ld apart
  int y_ld;
  const int* ids;             // [T][k]
  const float* w;             // [T][k]
  int T, k, kp, E, Ep;
  int* prow_of;               // [T k'] row of the slot, -1: none; the first product fills it for the combine
  int rows_cap, group_rows;   // filled by the launch: staged rows, rows of a pass over an expert's weights
  DevStatus* status;
};
constexpr int W4_VEC_SLOTS = 320;   // T k', at most

// The same for a batch, on the tensor cores (w4_tile.cu): M-blocks of the padded row space, x gathered into it.
struct W4TileArgs {
  CUtensorMap tok[4];         // Xp or A, boxes of 16, 32, 48, 64 rows x 64 columns
  const uint8_t *codes, *scales, *zeros;   // zeros NULL: 8
  int K, KU, RT, RTS, group;
  int ntn;                    // tiles of 256 weight rows
  int down, n_out;
  uint16_t* A;
  int a_ld;
  float* Y;
  int y_ld;
  const float* prow_w;
  const int *mblk_expert, *mb_start, *counts, *meta;
  DevStatus* status;
  uint64_t budget_ns;
};
cudaError_t launch_w4_tile(const W4TileArgs& a, int num_sms, cudaStream_t st, int* launches);

cudaError_t launch_w4_quantize(const uint16_t* W, int n, const W4Shape& s, uint32_t* codes, uint16_t* scales, uint8_t* zeros, cudaStream_t st);
cudaError_t launch_w4_pack(const uint8_t* q, const uint16_t* qs, const uint8_t* qz, int n, const W4Shape& s, uint32_t* codes, uint16_t* scales,
                           uint8_t* zeros, cudaStream_t st);
cudaError_t launch_w4_dequantize(const uint32_t* codes, const uint16_t* scales, const uint8_t* zeros, int n, const W4Shape& s, uint16_t* W, cudaStream_t st);
// rows the vector kernel can stage at reduction K; 0: too long
int w4_vec_rows(int K, int group, bool asym);
cudaError_t launch_w4_vec(W4VecArgs a, int num_sms, cudaStream_t st, int* launches);
// out[t] = sum_j Y[prow_of[t kp + j]], j ascending
cudaError_t launch_w4_combine(const float* Y, int y_ld, const int* prow_of, int T, int d, int kp, uint16_t* out, cudaStream_t st, int* launches);

}  // namespace moe
