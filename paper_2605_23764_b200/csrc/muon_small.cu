// Orthogonalised momentum of small matrices (m <= 128, l <= 384): a block takes one through the whole step, momentum, norm, all
// products and the weights' update, in one launch.
//
// X lies in TMEM in fp32, row i of its m rows on lane i, as V = X S_X S_B, and its fp16 image X S_X in shared memory.  A step is
//   acc = X X^T;  A = acc;  acc = A A;  B = b A + c acc + s I;  V <- (a - s) V + s (V - image), then V += B X on the tensor cores
// so the linear term never leaves fp32 (s (V - image) in steps that are not late: muon.cuh).  The image serves both products: as K-major operands of X X^T, and MN-major as the second of B X.
// Matrices taller than wide are turned while they are staged.  A A and B X sum over the m rows there are, in sixteens.
// Up to 64 rows (MS_LO) A and B are two fp16 numbers each, hi + lo, and both products take lo too: there are few entries for roundings to
// even out over (16 x 16, six steps: 1.4e-3 off in the norm instead of 2.0e-3; 128 x 256: 0.8e-3 instead of 1.2e-3), and their sums stay
// short.  At 128 rows lo would cost 8 us of 31.
//
// What bounds it: latencies, 3.8 us a step of 16 x 128 x 256 (three products of at most 0.3 us with what lies between them; 4.2 us where V's
// rest is added) and 14 us for the loads in front and the stores behind, 10 without momentum and weights: 33 us for five steps.  By the tiles of muon_gemm.cu every phase passes through
// L2 instead, with its stores, signal, poll and loads: 3.7 us.
#include <cuda_fp16.h>

#include "launch_pairs.cuh"
#include "muon.cuh"
#include "topk.cuh"

namespace moe {

constexpr int MS_THREADS = 512, MS_WARPS = MS_THREADS / 32;
constexpr int MS_BOX = 128 * 128;          // 128 rows x 64 columns in fp16, swizzled
constexpr int MS_LO = 64;                  // see above
constexpr int MS_AB = 2 * MS_BOX;          // A's or B's hi, and 128 x 64 elements in fp32 on their way in and out; lo lies behind it

struct MuonSmallShared {
  uint64_t done;           // the products issued last are complete
  uint32_t tmem_base;
  float factor[2];
  double sums[MS_WARPS];
};
static size_t small_smem(int lp) { return 1024 + (size_t)(lp / 64) * MS_BOX + 2 * MS_AB + sizeof(MuonSmallShared); }

// tmem_ld16 the other way round; complete for other readers behind tmem_st_wait() and the fences.
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const float* v) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
      ::"r"(taddr), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "f"(v[8]), "f"(v[9]),
        "f"(v[10]), "f"(v[11]), "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15])
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// hi of two values, and what it leaves of them
__device__ __forceinline__ uint32_t half2_rest(float& x, float& y) {
  const __half2 h = __floats2half2_rn(x, y);
  const float2 f = __half22float2(h);
  x -= f.x;
  y -= f.y;
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t half2_of(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
// element (i, j) of the fp32 staging, a chunk of four columns at a time; 16-byte chunk j of row i of an fp16 box
__device__ __forceinline__ float* stage4(uint8_t* ab, int i, int j4) { return reinterpret_cast<float*>(ab + i * 256 + ((j4 ^ (i & 15)) << 4)); }
__device__ __forceinline__ uint4* box8(uint8_t* box, int i, int j) { return reinterpret_cast<uint4*>(box + i * 128 + ((j ^ (i & 7)) << 4)); }

// The elements of a chunk of 64 of the l columns that one thread moves: `at` in the matrix, row i and column j of X's chunk.
// Vectors of eight lie along the matrix's rows: along j if it is wide, along i if it is tall.
struct SmallSlot { int i, j; long at; bool in; };
template <bool WIDE, bool VEC>
__device__ __forceinline__ SmallSlot small_slot(const MuonElemArgs& e, int chunk, int n) {   // n: 0 .. (VEC ? 1024 : 8192) - 1
  SmallSlot s;
  const int along = VEC ? 8 : 1;
  if (WIDE) {
    const int per = 64 / along;
    s.i = n / per;
    s.j = (n % per) * along;
    const int col = chunk * 64 + s.j;
    s.in = s.i < e.rows && col < e.cols;
    s.at = (long)s.i * e.cols + col;
  } else {
    const int per = 128 / along;
    s.j = n / per;
    s.i = (n % per) * along;
    const int row = chunk * 64 + s.j;
    s.in = row < e.rows && s.i < e.cols;
    s.at = (long)row * e.cols + s.i;
  }
  return s;
}
// eight (or one) elements of 16 or 32 bits
template <bool VEC>
__device__ __forceinline__ void load_bf(const uint16_t* p, float* v) {
  if (VEC) {
    const uint4 x = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int q = 0; q < 4; ++q) { v[2 * q] = bf16lo(w[q]); v[2 * q + 1] = bf16hi(w[q]); }
  } else {
    v[0] = __uint_as_float((uint32_t)*p << 16);
  }
}
template <bool VEC>
__device__ __forceinline__ void load_fp(const float* p, float* v) {
  if (VEC) {
    const float4 x = reinterpret_cast<const float4*>(p)[0], y = reinterpret_cast<const float4*>(p)[1];
    v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w; v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
  } else {
    v[0] = *p;
  }
}

template <bool WIDE, bool VEC>
__global__ void __launch_bounds__(MS_THREADS, 1) muon_small_kernel(const __grid_constant__ MuonSmallArgs a) {
  constexpr int N = VEC ? 8 : 1, SLOTS = (VEC ? 1024 : 8192) / MS_THREADS;   // of a thread and chunk
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const MuonElemArgs& e = a.e;
  const int l = WIDE ? e.cols : e.rows, chunks = (l + 63) / 64, lp = chunks * 64;
  const int rows = WIDE ? e.rows : e.cols, ks = (rows + 15) / 16;
  const bool with_lo = rows <= MS_LO;
  uint8_t* ab = smem + chunks * MS_BOX;
  MuonSmallShared* sh = reinterpret_cast<MuonSmallShared*>(ab + 2 * MS_AB);
  const int warp = warp_index(), lane = threadIdx.x & 31, quad = warp & 3, group = warp >> 2;
  const int row = quad * 32 + lane;   // of X: this thread's TMEM lane
  const WaitCtl wc{a.status, a.budget_ns};
  int cols = 128;                     // of TMEM: V, behind it the accumulator
  while (cols < lp + 128) cols <<= 1;

  if (threadIdx.x == 0) {
    mbar_init(&sh->done, 1);
    mbar_fence_init();
  }
  if (warp == 0) {
    tmem_alloc_cta(&sh->tmem_base, cols);
    tmem_relinquish_cta();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = uniform(sh->tmem_base), acc = tmem + lp, lanes = static_cast<uint32_t>(quad * 32) << 16;
  pdl_trigger();
  pdl_wait();

  // ---------------------------------------------------------------- momentum, u into TMEM, its square
  const size_t base = (size_t)blockIdx.x * e.elems;
  double sum = 0.0;
  for (int c = 0; c < chunks; ++c) {
#pragma unroll 2
    for (int q = 0; q < SLOTS; ++q) {
      const SmallSlot s = small_slot<WIDE, VEC>(e, c, q * MS_THREADS + threadIdx.x);
      float u[N];
#pragma unroll
      for (int i = 0; i < N; ++i) u[i] = 0.f;
      if (s.in) {
        if (e.g_fp32) load_fp<VEC>(static_cast<const float*>(e.G) + base + s.at, u);
        else load_bf<VEC>(static_cast<const uint16_t*>(e.G) + base + s.at, u);
        if (e.M) {
          float m[N];
          load_fp<VEC>(e.M + base + s.at, m);
#pragma unroll
          for (int i = 0; i < N; ++i) {
            m[i] = fmaf(e.mu, m[i], u[i]);
            u[i] = e.nesterov ? fmaf(e.mu, m[i], u[i]) : m[i];
          }
          float* o = e.M_out + base + s.at;
          if (VEC) {
            reinterpret_cast<float4*>(o)[0] = make_float4(m[0], m[1 % N], m[2 % N], m[3 % N]);
            reinterpret_cast<float4*>(o)[1] = make_float4(m[4 % N], m[5 % N], m[6 % N], m[7 % N]);
          } else {
            *o = m[0];
          }
        }
#pragma unroll
        for (int i = 0; i < N; ++i) sum = fma((double)u[i], (double)u[i], sum);
      }
      if (VEC && WIDE) {
        *reinterpret_cast<float4*>(stage4(ab, s.i, s.j / 4)) = make_float4(u[0], u[1 % N], u[2 % N], u[3 % N]);
        *reinterpret_cast<float4*>(stage4(ab, s.i, s.j / 4 + 1)) = make_float4(u[4 % N], u[5 % N], u[6 % N], u[7 % N]);
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) stage4(ab, s.i + i, s.j / 4)[s.j & 3] = u[i];
      }
    }
    __syncthreads();
    float v[16];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float4 x = *reinterpret_cast<const float4*>(stage4(ab, row, group * 4 + q));
      v[4 * q] = x.x; v[4 * q + 1] = x.y; v[4 * q + 2] = x.z; v[4 * q + 3] = x.w;
    }
    tmem_st16(tmem + lanes + c * 64 + group * 16, v);
    __syncthreads();
  }
  tmem_st_wait();
#pragma unroll
  for (int off = 16; off; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
  if (lane == 0) sh->sums[warp] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    double t = 0.0;
    for (int w = 0; w < MS_WARPS; ++w) t += sh->sums[w];
    const double norm = sqrt(t) + (double)e.eps;
    const double up = norm < 1e-18 ? 18446744073709551616.0 : 1.0;   // the factor of a tiny norm is beyond fp32
    sh->factor[0] = (float)up;
    sh->factor[1] = norm == 0.0 ? 0.f : (float)((double)MUON_SX / (norm * up));
  }
  __syncthreads();
  // V = X S_X S_B and its image; a warp's 16 columns of every chunk
  {
    const float f0 = sh->factor[0], f1 = sh->factor[1];
    for (int c = 0; c < chunks; ++c) {
      float v[16];
      const uint32_t at = tmem + lanes + c * 64 + group * 16;
      tmem_ld16(at, v);
      tmem_ld_wait();
#pragma unroll
      for (int q = 0; q < 16; ++q) v[q] = v[q] * f0 * f1;
      uint8_t* box = smem + c * MS_BOX;
      *box8(box, row, 2 * group) = make_uint4(half2_of(v[0], v[1]), half2_of(v[2], v[3]), half2_of(v[4], v[5]), half2_of(v[6], v[7]));
      *box8(box, row, 2 * group + 1) = make_uint4(half2_of(v[8], v[9]), half2_of(v[10], v[11]), half2_of(v[12], v[13]), half2_of(v[14], v[15]));
#pragma unroll
      for (int q = 0; q < 16; ++q) v[q] *= MUON_SB;
      tmem_st16(at, v);
    }
    tmem_st_wait();
  }

  // ---------------------------------------------------------------- the steps
  const uint32_t x_k = smem_desc_lo(smem_u32(smem), 16), x_mn = smem_desc_lo(smem_u32(smem), MS_BOX), ab_k = smem_desc_lo(smem_u32(ab), 16);
  constexpr uint32_t hi = smem_desc_hi(1024), sym = make_idesc_f16(128, 128, 0, 0);
  uint32_t par = 0;
  bool ok = true;
  // every thread: what was written to shared memory and TMEM is there for the products / their result is there for every thread
  auto ready = [&] {
    fence_proxy_async_smem();
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
  };
  auto wait = [&] {
    ok = mbar_wait_warp(&sh->done, par, wc, SITE_TMEM_FULL, blockIdx.x) && ok;
    par ^= 1;
    tc_fence_after_sync();
  };
  for (int k = 0; k < a.steps; ++k) {
    const MuonArgs::Step st = a.step[k];
    ready();
    if (warp == 0) {
      for (int kk = 0; kk < chunks * 4; ++kk) {
        const uint32_t at = x_k + (kk >> 2) * (MS_BOX >> 4) + (kk & 3) * 2;
        tc_mma1_f16_cta(acc, at, at, hi, sym, kk != 0);
      }
      tc_commit_cta(&sh->done);
    }
    // the linear term, beside the products
    const bool rest = st.app_rest != 0.f;
    for (int c = group * 16; c < lp; c += 64) {
      float v[16];
      tmem_ld16(tmem + lanes + c, v);
      tmem_ld_wait();
#pragma unroll
      for (int q = 0; q < 16; ++q) {
        float x = v[q] * st.app_in;
        if (rest) x = fmaf(v[q] - __half2float(__float2half_rn(v[q] * (1.f / MUON_SB))) * MUON_SB, st.app_rest, x);   // what the image lacks of V
        v[q] = x;
      }
      tmem_st16(tmem + lanes + c, v);
    }
    tmem_st_wait();
    wait();
    // columns 32 group .. of the accumulator: half a box of 64
    uint8_t* box = ab + (group >> 1) * MS_BOX;
    const int j0 = (group & 1) * 4;
    float v[32];
    tmem_ld16(acc + lanes + group * 32, v);
    tmem_ld16(acc + lanes + group * 32 + 16, v + 16);
    tmem_ld_wait();
    float A[32];
#pragma unroll
    for (int q = 0; q < 32; ++q) A[q] = v[q] * st.gram_acc;
    // 32 columns of the lane's row into the boxes of hi and lo
    auto put = [&](const float* x) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t h[4], l[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float x0 = x[8 * j + 2 * q], x1 = x[8 * j + 2 * q + 1];
          h[q] = half2_rest(x0, x1);
          l[q] = half2_of(x0, x1);
        }
        *box8(box, row, j0 + j) = make_uint4(h[0], h[1], h[2], h[3]);
        if (with_lo) *box8(box + MS_AB, row, j0 + j) = make_uint4(l[0], l[1], l[2], l[3]);
      }
    };
    put(A);
    if (!with_lo) {   // b A + c A A of one and the same A: with fp32's A in the first of them 1.8e-3 off instead of 1.2e-3 (100 x 120, six steps)
#pragma unroll
      for (int q = 0; q < 32; ++q) A[q] = __half2float(__float2half_rn(A[q]));
    }
    ready();
    if (warp == 0) {
      for (int kk = 0; kk < ks; ++kk) {
        const uint32_t at = ab_k + (kk >> 2) * (MS_BOX >> 4) + (kk & 3) * 2, lo = at + (MS_AB >> 4);
        tc_mma1_f16_cta(acc, at, at, hi, sym, kk != 0);
        if (!with_lo) continue;
        tc_mma1_f16_cta(acc, lo, at, hi, sym, 1);
        tc_mma1_f16_cta(acc, at, lo, hi, sym, 1);
      }
      tc_commit_cta(&sh->done);
    }
    wait();
    tmem_ld16(acc + lanes + group * 32, v);
    tmem_ld16(acc + lanes + group * 32 + 16, v + 16);
    tmem_ld_wait();
    const int diag = row - group * 32;
#pragma unroll
    for (int q = 0; q < 32; ++q) {
      A[q] = fmaf(A[q], st.poly_in, v[q] * st.poly_acc);
      if (diag == q) A[q] += st.poly_diag;
    }
    put(A);
    ready();
    if (warp == 0) {
      for (int c = 0; c < lp; c += 256) {
        const uint32_t idesc = make_idesc_f16(128, min(256, lp - c), 0, 1);
        for (int kk = 0; kk < ks; ++kk) {
          const uint32_t at = ab_k + (kk >> 2) * (MS_BOX >> 4) + (kk & 3) * 2, x = x_mn + (c / 64) * (MS_BOX >> 4) + kk * (2048 >> 4);
          tc_mma1_f16_cta(tmem + c, at, x, hi, idesc, 1);
          if (with_lo) tc_mma1_f16_cta(tmem + c, at + (MS_AB >> 4), x, hi, idesc, 1);
        }
      }
      tc_commit_cta(&sh->done);
    }
    wait();
    if (k + 1 < a.steps)
      for (int c = group * 16; c < lp; c += 64) {   // the image
        float x[16];
        tmem_ld16(tmem + lanes + c, x);
        tmem_ld_wait();
        uint8_t* xb = smem + (c / 64) * MS_BOX;
        uint32_t h[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) h[q] = half2_of(x[2 * q] * (1.f / MUON_SB), x[2 * q + 1] * (1.f / MUON_SB));
        *box8(xb, row, 2 * group) = make_uint4(h[0], h[1], h[2], h[3]);
        *box8(xb, row, 2 * group + 1) = make_uint4(h[4], h[5], h[6], h[7]);
      }
  }

  // ---------------------------------------------------------------- out, or the weights' update, chunk by chunk through the staging
  for (int c = 0; c < chunks; ++c) {
    float v[16];
    tmem_ld16(tmem + lanes + c * 64 + group * 16, v);
    tmem_ld_wait();
    __syncthreads();   // the chunk before has been read
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      constexpr float S = 1.f / (MUON_SX * MUON_SB);
      *reinterpret_cast<float4*>(stage4(ab, row, group * 4 + q)) = make_float4(v[4 * q] * S, v[4 * q + 1] * S, v[4 * q + 2] * S, v[4 * q + 3] * S);
    }
    __syncthreads();
#pragma unroll 2
    for (int q = 0; q < SLOTS; ++q) {
      const SmallSlot s = small_slot<WIDE, VEC>(e, c, q * MS_THREADS + threadIdx.x);
      if (!s.in) continue;
      float x[N], w[N];
      if (VEC && WIDE) {
        const float4 p = *reinterpret_cast<const float4*>(stage4(ab, s.i, s.j / 4)), r = *reinterpret_cast<const float4*>(stage4(ab, s.i, s.j / 4 + 1));
        x[0] = p.x; x[1 % N] = p.y; x[2 % N] = p.z; x[3 % N] = p.w; x[4 % N] = r.x; x[5 % N] = r.y; x[6 % N] = r.z; x[7 % N] = r.w;
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = stage4(ab, s.i + i, s.j / 4)[s.j & 3];
      }
      if (a.W) {
        load_bf<VEC>(a.W + base + s.at, w);
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = fmaf(a.keep, w[i], -a.rate * x[i]);
      }
      uint16_t* o = a.out + base + s.at;
      if (VEC)
        *reinterpret_cast<uint4*>(o) = make_uint4(pack_bf16x2(x[0], x[1 % N]), pack_bf16x2(x[2 % N], x[3 % N]), pack_bf16x2(x[4 % N], x[5 % N]),
                                                  pack_bf16x2(x[6 % N], x[7 % N]));
      else
        *o = (uint16_t)pack_bf16x2(x[0], 0.f);
    }
  }

  if (*reinterpret_cast<volatile int*>(&a.status->abort)) __nanosleep(200000);
  tc_fence_before_sync();
  __syncthreads();
  if (warp == 0) {
    tc_fence_after_sync();
    tmem_dealloc_cta(tmem, cols);
  }
}

template <bool WIDE, bool VEC>
static cudaError_t launch_one(const MuonSmallArgs& a, cudaStream_t s) {
  const int l = WIDE ? a.e.cols : a.e.rows;
  cudaError_t e = opt_in_smem<muon_small_kernel<WIDE, VEC>>((int)small_smem(MUON_SMALL_L));
  if (e != cudaSuccess) return e;
  return launch_dependent(muon_small_kernel<WIDE, VEC>, dim3((unsigned)a.e.n), dim3(MS_THREADS), small_smem((l + 63) / 64 * 64), s, a);
}
cudaError_t launch_muon_small(const MuonSmallArgs& a, cudaStream_t s) {
  if (a.e.rows <= a.e.cols) return a.vec ? launch_one<true, true>(a, s) : launch_one<true, false>(a, s);
  return a.vec ? launch_one<false, true>(a, s) : launch_one<false, false>(a, s);
}

}  // namespace moe
