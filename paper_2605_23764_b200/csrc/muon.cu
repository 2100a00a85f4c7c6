// The passes over single elements in front of an orthogonalisation (muon.cuh): momentum with the sum of squares, and X = u / norm.
// Both are streams: 10 and 10 bytes an element of a training step (bf16 gradients, fp32 momentum), 2 and 6 of a plain bf16 input.
// Squares are summed in 64 bits in a fixed order, so that neither large nor small gradients leave fp32's range.
#include <cuda_fp16.h>

#include "muon.cuh"
#include "topk.cuh"

namespace moe {

constexpr int MU_ELEM_THREADS = 256;

// eight elements from index i on (vec), or the element i alone in v[0]
template <bool VEC>
__device__ __forceinline__ void muon_load_g(const MuonElemArgs& a, size_t i, float* v) {
  if (a.g_fp32) {
    const float* g = static_cast<const float*>(a.G) + i;
    if (VEC) {
      const float4 x = *reinterpret_cast<const float4*>(g), y = *reinterpret_cast<const float4*>(g + 4);
      v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w; v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
    } else {
      v[0] = *g;
    }
  } else {
    const uint16_t* g = static_cast<const uint16_t*>(a.G) + i;
    if (VEC) {
      const uint4 x = *reinterpret_cast<const uint4*>(g);
      const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
      for (int p = 0; p < 4; ++p) { v[2 * p] = bf16lo(w[p]); v[2 * p + 1] = bf16hi(w[p]); }
    } else {
      v[0] = __uint_as_float((uint32_t)*g << 16);
    }
  }
}
template <bool VEC>
__device__ __forceinline__ void muon_load_f(const float* m, float* v) {
  if (VEC) {
    const float4 x = *reinterpret_cast<const float4*>(m), y = *reinterpret_cast<const float4*>(m + 4);
    v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w; v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
  } else {
    v[0] = *m;
  }
}

template <bool VEC>
__global__ void __launch_bounds__(MU_ELEM_THREADS) muon_momentum_kernel(const MuonElemArgs a) {
  constexpr int N = VEC ? 8 : 1;
  __shared__ double sums[MU_ELEM_THREADS / 32];
  pdl_trigger();
  pdl_wait();
  const int mat = blockIdx.x / a.parts, part = blockIdx.x - mat * a.parts;
  constexpr long PART = VEC ? MUON_PART_VEC : MUON_PART_ONE;
  const long e0 = part * PART, e1 = min(a.elems, e0 + PART);
  const size_t base = (size_t)mat * a.elems;
  if (blockIdx.x == 0)
    for (int i = threadIdx.x; i <= a.n; i += MU_ELEM_THREADS) a.ctr[i] = 0;
  double sum = 0.0;
#pragma unroll 4
  for (long i = e0 + threadIdx.x * N; i < e1; i += MU_ELEM_THREADS * N) {
    float u[N];
    muon_load_g<VEC>(a, base + i, u);
    if (a.M) {
      float m[N];
      muon_load_f<VEC>(a.M + base + i, m);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        m[j] = fmaf(a.mu, m[j], u[j]);
        u[j] = a.nesterov ? fmaf(a.mu, m[j], u[j]) : m[j];
      }
      float* out = a.M_out + base + i;
      if (VEC) {
        *reinterpret_cast<float4*>(out) = make_float4(m[0], m[1], m[2], m[3]);
        *reinterpret_cast<float4*>(out + 4) = make_float4(m[4 % N], m[5 % N], m[6 % N], m[7 % N]);
      } else {
        *out = m[0];
      }
    }
#pragma unroll
    for (int j = 0; j < N; ++j) sum = fma((double)u[j], (double)u[j], sum);
  }
#pragma unroll
  for (int off = 16; off; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
  if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    double t = 0.0;
    for (int w = 0; w < MU_ELEM_THREADS / 32; ++w) t += sums[w];
    a.part[(size_t)mat * a.parts + part] = t;
  }
}

// rows_per: rows of a block
template <bool VEC>
__global__ void __launch_bounds__(MU_ELEM_THREADS) muon_normalize_kernel(const MuonElemArgs a, int rows_per, int blocks_per) {
  constexpr int N = VEC ? 8 : 1;
  __shared__ float factor[2];
  pdl_trigger();
  pdl_wait();
  const int mat = blockIdx.x / blocks_per, blk = blockIdx.x - mat * blocks_per;
  if (threadIdx.x < 32) {
    double sum = 0.0;
    for (int p = threadIdx.x; p < a.parts; p += 32) sum += a.part[(size_t)mat * a.parts + p];
#pragma unroll
    for (int off = 16; off; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
    if (threadIdx.x == 0) {
      const double norm = sqrt(sum) + (double)a.eps;
      const double up = norm < 1e-18 ? 18446744073709551616.0 : 1.0;   // the factor of a tiny norm is beyond fp32
      factor[0] = (float)up;
      factor[1] = norm == 0.0 ? 0.f : (float)((double)MUON_SX / (norm * up));
    }
  }
  __syncthreads();
  const float f0 = factor[0], f1 = factor[1];
  const int r0 = blk * rows_per, nrows = min(a.rows - r0, rows_per);
  const int per_row = (a.cols + N - 1) / N, count = nrows * per_row;
#pragma unroll 4
  for (int i = threadIdx.x; i < count; i += MU_ELEM_THREADS) {
    const int row = i / per_row, col = (i - row * per_row) * N;
    const size_t at = (size_t)mat * a.elems + (size_t)(r0 + row) * a.cols + col;
    float u[N];
    muon_load_g<VEC>(a, at, u);
    if (a.M) {
      float m[N];
      muon_load_f<VEC>(a.M_out + at, m);
#pragma unroll
      for (int j = 0; j < N; ++j) u[j] = a.nesterov ? fmaf(a.mu, m[j], u[j]) : m[j];
    }
    const size_t to = ((size_t)mat * a.rows + r0 + row) * a.ld + col;
    uint16_t h[N], l[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const float x = u[j] * f0 * f1;
      const __half hi = __float2half_rn(x);
      h[j] = __half_as_ushort(hi);
      l[j] = __half_as_ushort(__float2half_rn((x - __half2float(hi)) * MUON_SLO));
    }
    if (VEC) {
#define MOE_PAIR(x, j) ((uint32_t)x[(j) % N] | (uint32_t)x[((j) + 1) % N] << 16)
      *reinterpret_cast<uint4*>(a.hi + to) = make_uint4(MOE_PAIR(h, 0), MOE_PAIR(h, 2), MOE_PAIR(h, 4), MOE_PAIR(h, 6));
      *reinterpret_cast<uint4*>(a.lo + to) = make_uint4(MOE_PAIR(l, 0), MOE_PAIR(l, 2), MOE_PAIR(l, 4), MOE_PAIR(l, 6));
#undef MOE_PAIR
    } else {
      a.hi[to] = h[0];
      a.lo[to] = l[0];
    }
  }
}

cudaError_t launch_muon_momentum(const MuonElemArgs& a, cudaStream_t s) {
  const dim3 grid((unsigned)(a.n * (long)a.parts));
  return a.vec ? launch_dependent(muon_momentum_kernel<true>, grid, dim3(MU_ELEM_THREADS), 0, s, a)
               : launch_dependent(muon_momentum_kernel<false>, grid, dim3(MU_ELEM_THREADS), 0, s, a);
}
cudaError_t launch_muon_normalize(const MuonElemArgs& a, cudaStream_t s) {
  int rows_per = (int)((a.vec ? MUON_PART_VEC : MUON_PART_ONE) / a.cols);
  if (rows_per < 1) rows_per = 1;
  const int blocks_per = (a.rows + rows_per - 1) / rows_per;
  const dim3 grid((unsigned)(a.n * (long)blocks_per));
  return a.vec ? launch_dependent(muon_normalize_kernel<true>, grid, dim3(MU_ELEM_THREADS), 0, s, a, rows_per, blocks_per)
               : launch_dependent(muon_normalize_kernel<false>, grid, dim3(MU_ELEM_THREADS), 0, s, a, rows_per, blocks_per);
}

}  // namespace moe
