// The products of an orthogonalising step (muon.cuh) on the tensor cores: fp16 operands, fp32 accumulators, CTA pairs, persistent.
//
// A tile is 256 rows x nt columns of one matrix's product, its accumulator one of two in TMEM, so that a tile's products run beside
// the epilogue of the one before.  Operands come in as they lie: K-major where the reduction is contiguous, MN-major where it is the
// rows (X as the second operand of B X, both of X^T X), so nothing is ever transposed in memory.
//
// GRAM and POLY are symmetric: only tiles that touch the lower triangle are computed (21 of 36 for 1408), and boxes of 32 rows x 64
// columns below the diagonal are stored twice, as they are and mirrored, from a box transposed in shared memory.  Boxes on the
// diagonal are stored element by element, each written once.
//
// Roles per CTA: warp 0 TMA producer, warp 1 MMA issuer (even CTA) and TMEM owner, warps 2-9 epilogue.
#include <cuda_fp16.h>

#include "gemm_tile.cuh"
#include "launch_pairs.cuh"
#include "muon.cuh"
#include "topk.cuh"

namespace moe {

constexpr int MU_STAGES = 5;
constexpr int MU_STAGE_BYTES = A_STAGE_BYTES + HALF_B_BYTES;   // 128 rows of A, up to 128 of the tile's columns
constexpr int MU_EPI_WARPS = 8, MU_THREADS = 32 * (2 + MU_EPI_WARPS);
constexpr int MU_BOX = 32 * 64 * 2;

struct MuonBarriers {
  uint64_t full[MU_STAGES], empty[MU_STAGES];
  uint64_t tmem_full[2], tmem_empty[2];
  uint64_t in_full[MU_EPI_WARPS];
  uint64_t drain;
  uint32_t tmem_base;
};
constexpr size_t MU_SMEM = 1024 + MU_STAGES * MU_STAGE_BYTES + MU_EPI_WARPS * 2 * MU_BOX + sizeof(MuonBarriers);
static_assert(MU_SMEM <= 227 * 1024, "shared memory budget");

struct MuonTile { int mat, m0, n0; };

template <bool TRI>
__host__ __device__ __forceinline__ int muon_row_tiles(const MuonProductArgs& a, int i) {
  const int cols = TRI ? min(256 * (i + 1), a.N) : a.N;
  return (cols + a.nt - 1) / a.nt;
}
template <bool TRI>
__host__ __device__ __forceinline__ int muon_tiles(const MuonProductArgs& a) {   // of one matrix
  const int rows = (a.M + 255) / 256;
  if (!TRI) return rows * muon_row_tiles<TRI>(a, 0);
  int n = 0;
  for (int i = 0; i < rows; ++i) n += muon_row_tiles<TRI>(a, i);
  return n;
}
template <bool TRI>
__device__ __forceinline__ MuonTile muon_decode(const MuonProductArgs& a, int per, int t) {
  MuonTile r;
  r.mat = t / per;
  int q = t - r.mat * per, i = 0;
  if (TRI) {
    for (int c; q >= (c = muon_row_tiles<TRI>(a, i)); ++i) q -= c;
  } else {
    const int c = muon_row_tiles<TRI>(a, 0);
    i = q / c;
    q -= i * c;
  }
  r.m0 = i * 256;
  r.n0 = q * a.nt;
  return r;
}

__device__ __forceinline__ uint32_t pack_h2(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float2 unpack_h2(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2*>(&v)); }

// One box of 32 rows x 64 columns of the accumulator, first row r0 of the matrix (this lane's: r0 + lane), first column c0.
template <int WHAT>
__device__ __forceinline__ void muon_epilogue_box(const MuonProductArgs& a, uint32_t tcol, uint8_t* box0, uint8_t* box1, int mat, int r0, int c0, int lane) {
  float v[64];
#pragma unroll
  for (int q = 0; q < 4; ++q) tmem_ld16(tcol + 16 * q, v + 16 * q);
  tmem_ld_wait();
  const int r = r0 + lane;
  uint8_t* row0 = box0 + lane * 128;
  uint8_t* row1 = box1 + lane * 128;
  if constexpr (WHAT == MUON_GRAM || WHAT == MUON_POLY) {
    uint32_t h[32];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      uint4 in = make_uint4(0, 0, 0, 0);
      if (WHAT == MUON_POLY) in = *reinterpret_cast<uint4*>(row0 + ((j ^ (lane & 7)) << 4));
      const uint32_t w[4] = {in.x, in.y, in.z, in.w};
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        float2 x = make_float2(v[8 * j + 2 * p] * a.k_acc, v[8 * j + 2 * p + 1] * a.k_acc);
        if (WHAT == MUON_POLY) {
          const float2 y = unpack_h2(w[p]);
          x.x = fmaf(y.x, a.k_in, x.x);
          x.y = fmaf(y.y, a.k_in, x.y);
          const int c = c0 + 8 * j + 2 * p;
          if (c == r) x.x += a.k_diag;
          if (c + 1 == r) x.y += a.k_diag;
        }
        h[4 * j + p] = pack_h2(x.x, x.y);
      }
    }
    if (c0 + 63 < r0) {   // below the diagonal: as it is and mirrored
#pragma unroll
      for (int j = 0; j < 8; ++j)
        *reinterpret_cast<uint4*>(row0 + ((j ^ (lane & 7)) << 4)) = make_uint4(h[4 * j], h[4 * j + 1], h[4 * j + 2], h[4 * j + 3]);
      uint16_t* t = reinterpret_cast<uint16_t*>(box1) + lane;
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        t[(2 * i) * 32] = (uint16_t)h[i];
        t[(2 * i + 1) * 32] = (uint16_t)(h[i] >> 16);
      }
      staging_release();
      if (lane == 0) {
        tma_store_3d(&a.tmOut0, c0, r0, mat, box0);
        tma_store_3d(&a.tmOut1, r0, c0, mat, box1);
        tma_store_commit();
      }
    } else if (r < a.M) {
      uint16_t* A = a.out + (size_t)mat * a.M * a.ld;
#pragma unroll
      for (int i = 0; i < 64; ++i) {
        const int c = c0 + i;
        const uint16_t x = (uint16_t)(h[i >> 1] >> (16 * (i & 1)));
        if (c <= r) A[(size_t)r * a.ld + c] = x;
        if (c < r) A[(size_t)c * a.ld + r] = x;
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      uint4* ph = reinterpret_cast<uint4*>(row0 + ((j ^ (lane & 7)) << 4));
      uint4* pl = reinterpret_cast<uint4*>(row1 + ((j ^ (lane & 7)) << 4));
      const uint4 xh = *ph, xl = *pl;
      const uint32_t wh[4] = {xh.x, xh.y, xh.z, xh.w}, wl[4] = {xl.x, xl.y, xl.z, xl.w};
      uint32_t oh[4], ol[4];
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        const float2 yh = unpack_h2(wh[p]), yl = unpack_h2(wl[p]);
        const float x0 = fmaf(fmaf(yl.x, 1.f / MUON_SLO, yh.x), a.k_in, v[8 * j + 2 * p] * a.k_acc);
        const float x1 = fmaf(fmaf(yl.y, 1.f / MUON_SLO, yh.y), a.k_in, v[8 * j + 2 * p + 1] * a.k_acc);
        v[8 * j + 2 * p] = x0;
        v[8 * j + 2 * p + 1] = x1;
        if (WHAT == MUON_APPLY) {
          oh[p] = pack_h2(x0, x1);
          const float2 z = unpack_h2(oh[p]);
          ol[p] = pack_h2((x0 - z.x) * MUON_SLO, (x1 - z.y) * MUON_SLO);
        }
      }
      if (WHAT == MUON_APPLY) {
        *ph = make_uint4(oh[0], oh[1], oh[2], oh[3]);
        *pl = make_uint4(ol[0], ol[1], ol[2], ol[3]);
      }
    }
    if (WHAT == MUON_APPLY) {
      staging_release();
      if (lane == 0) {
        tma_store_3d(&a.tmOut0, c0, r0, mat, box0);
        tma_store_3d(&a.tmOut1, c0, r0, mat, box1);
        tma_store_commit();
      }
    } else {
      staging_release();   // what was read here is overwritten by the next box's loads
      if (r < a.M) {
        const size_t at = ((size_t)mat * a.M + r) * a.N + c0;
        const MuonFinish& f = a.fin;
        if (f.vec) {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (c0 + 8 * j < a.N) {
              float* x = v + 8 * j;
              if (f.W) {
                const uint4 w = *reinterpret_cast<const uint4*>(f.W + at + 8 * j);
                const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                  x[2 * p] = fmaf(f.keep, bf16lo(ww[p]), -f.rate * x[2 * p]);
                  x[2 * p + 1] = fmaf(f.keep, bf16hi(ww[p]), -f.rate * x[2 * p + 1]);
                }
              }
              *reinterpret_cast<uint4*>(f.out + at + 8 * j) =
                  make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
            }
        } else {
#pragma unroll
          for (int i = 0; i < 64; ++i)
            if (c0 + i < a.N) {
              float x = v[i];
              if (f.W) x = fmaf(f.keep, __uint_as_float((uint32_t)f.W[at + i] << 16), -f.rate * x);
              f.out[at + i] = (uint16_t)pack_bf16x2(x, 0.f);
            }
        }
      }
    }
  }
}

template <int WHAT, bool A_MN, bool B_MN>
__global__ void __launch_bounds__(MU_THREADS, 1) muon_product_kernel(const __grid_constant__ MuonProductArgs a) {
  constexpr bool TRI = WHAT == MUON_GRAM || WHAT == MUON_POLY;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* boxes = smem + MU_STAGES * MU_STAGE_BYTES;
  MuonBarriers* bars = reinterpret_cast<MuonBarriers*>(boxes + MU_EPI_WARPS * 2 * MU_BOX);

  const int warp = warp_index(), lane = threadIdx.x & 31;
  const int rank = (int)cluster_ctarank();
  const int pair = blockIdx.x >> 1, npairs = gridDim.x >> 1;
  const WaitCtl wc{a.status, a.budget_ns};

  if (threadIdx.x == 0) {
    for (int s = 0; s < MU_STAGES; ++s) {
      mbar_init(&bars->full[s], 1);
      mbar_init(&bars->empty[s], 1);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(&bars->tmem_full[s], 1);
      mbar_init(&bars->tmem_empty[s], 2 * MU_EPI_WARPS);
    }
    for (int w = 0; w < MU_EPI_WARPS; ++w) mbar_init(&bars->in_full[w], 1);
    mbar_init(&bars->drain, 1);
    mbar_fence_init();
    fence_proxy_async();
    tma_prefetch_desc(&a.tmA);
    tma_prefetch_desc(&a.tmB);
  }
  if (warp == 1) {
    tmem_alloc_pair(&bars->tmem_base, TMEM_COLS);
    tmem_relinquish_pair();
  }
  tc_fence_before_sync();
  __syncthreads();
  cluster_sync_all();
  tc_fence_after_sync();
  const uint32_t tmem_base = uniform(bars->tmem_base);
  pdl_trigger();
  pdl_wait();

  const int per = muon_tiles<TRI>(a), total = a.n * per, nkb = (a.K + BK - 1) / BK;
  const int half = a.nt / 2;   // columns of a tile that one CTA brings in
  if (warp == 0) {
    const int b_boxes = (half + 63) / 64;
    const int bytes = 2 * (A_STAGE_BYTES + (B_MN ? b_boxes * MN_BOX_BYTES : half * BK * 2));
    uint32_t s = 0, par = (1u << MU_STAGES) - 1;
    bool ok = true;
    for (int t = pair; t < total && ok; t += npairs) {
      const MuonTile tl = muon_decode<TRI>(a, per, t);
      const int m0 = uniform(tl.m0 + rank * 128), n0 = uniform(tl.n0 + rank * half), mat = uniform(tl.mat);
      for (int kb = 0; kb < nkb; ++kb) {
        if (!mbar_wait_warp(&bars->empty[s], (par >> s) & 1, wc, SITE_EMPTY, t, 20)) { ok = false; break; }
        uint8_t* st = smem + s * MU_STAGE_BYTES;
        if (rank == 0) mbar_expect_tx_elect(&bars->full[s], bytes);
        if (A_MN) {
          tma_load_3d_pair(st, &a.tmA, m0, kb * BK, mat, &bars->full[s]);
          tma_load_3d_pair(st + MN_BOX_BYTES, &a.tmA, m0 + 64, kb * BK, mat, &bars->full[s]);
        } else {
          tma_load_3d_pair(st, &a.tmA, kb * BK, m0, mat, &bars->full[s]);
        }
        uint8_t* sb = st + A_STAGE_BYTES;
        if (B_MN) {
          tma_load_3d_pair(sb, &a.tmB, n0, kb * BK, mat, &bars->full[s]);
          if (b_boxes > 1) tma_load_3d_pair(sb + MN_BOX_BYTES, &a.tmB, n0 + 64, kb * BK, mat, &bars->full[s]);
        } else {
          tma_load_3d_pair(sb, &a.tmB, kb * BK, n0, mat, &bars->full[s]);
        }
        par ^= 1u << s;
        if (++s == MU_STAGES) s = 0;
      }
    }
  } else if (warp == 1) {
    if (rank == 0) {
      const uint32_t idesc = make_idesc_f16(256, a.nt, A_MN, B_MN);
      constexpr int ASTEP = A_MN ? 2048 >> 4 : 2, BSTEP = B_MN ? 2048 >> 4 : 2;
      const uint32_t a_lo0 = smem_desc_lo(smem_u32(smem), A_MN ? MN_BOX_BYTES : 16);
      const uint32_t b_lo0 = smem_desc_lo(smem_u32(smem + A_STAGE_BYTES), B_MN ? MN_BOX_BYTES : 16);
      uint32_t s = 0, par = 0, acc = 0, acc_par = 3;
      bool ok = true;
      for (int t = pair; t < total && ok; t += npairs) {
        if (!mbar_wait_warp(&bars->tmem_empty[acc], (acc_par >> acc) & 1, wc, SITE_TMEM_EMPTY, t)) { ok = false; break; }
        acc_par ^= 1u << acc;
        tc_fence_after_sync();
        const uint32_t d_tmem = uniform(tmem_base + acc * 256);
        for (int kb = 0; kb < nkb; ++kb) {
          if (!mbar_wait_warp(&bars->full[s], (par >> s) & 1, wc, SITE_FULL, t)) { ok = false; break; }
          par ^= 1u << s;
          tc_fence_after_sync();
          const uint32_t at = s * (MU_STAGE_BYTES >> 4);
          tc_mma4_bf16_pair<ASTEP, BSTEP>(d_tmem, a_lo0 + at, b_lo0 + at, smem_desc_hi(1024), idesc, kb != 0);
          tc_commit_pair(&bars->empty[s]);
          if (++s == MU_STAGES) s = 0;
        }
        if (!ok) break;
        tc_commit_pair(&bars->tmem_full[acc]);
        acc ^= 1;
      }
      if (uniform(!ok || *reinterpret_cast<volatile int*>(&a.status->abort) ? 1 : 0)) {
        tc_commit_pair(&bars->drain);
        const WaitCtl shortwc{a.status, 20ull * 1000 * 1000};
        mbar_wait_warp(&bars->drain, 0, shortwc, SITE_DRAIN, 0);
      }
    }
  } else {
    const int ew = warp - 2, quad = warp & 3;
    uint8_t* box0 = boxes + ew * 2 * MU_BOX;
    uint8_t* box1 = box0 + MU_BOX;
    uint32_t acc = 0, full_par = 0, in_par = 0;
    bool ok = true;
    for (int t = pair; t < total && ok; t += npairs) {
      const MuonTile tl = muon_decode<TRI>(a, per, t);
      const int r0 = tl.m0 + rank * 128 + quad * 32;
      bool up = false;   // the accumulator has been seen complete
      for (int b = (ew >> 2) * 64; b < a.nt && ok; b += 128) {
        const int c0 = tl.n0 + b;
        if (r0 >= a.M || c0 >= a.N || (TRI && c0 > r0 + 31)) break;
        __syncwarp();   // every lane has read the boxes
        if (lane == 0) {
          tma_store_wait_read();
          if (WHAT != MUON_GRAM) {
            mbar_expect_tx(&bars->in_full[ew], WHAT == MUON_POLY ? MU_BOX : 2 * MU_BOX);
            tma_load_3d_thread(box0, &a.tmIn0, c0, r0, tl.mat, &bars->in_full[ew]);
            if (WHAT != MUON_POLY) tma_load_3d_thread(box1, &a.tmIn1, c0, r0, tl.mat, &bars->in_full[ew]);
          }
        }
        __syncwarp();
        if (!up) {
          ok = mbar_wait_warp(&bars->tmem_full[acc], (full_par >> acc) & 1, wc, SITE_TMEM_FULL, t, 100);
          tc_fence_after_sync();
          up = true;
        }
        if (WHAT != MUON_GRAM) {
          ok = mbar_wait_warp(&bars->in_full[ew], in_par, wc, SITE_DEP, t) && ok;
          in_par ^= 1;
        }
        if (!ok) break;
        muon_epilogue_box<WHAT>(a, tmem_base + acc * 256 + b + (static_cast<uint32_t>(quad * 32) << 16), box0, box1, tl.mat, r0, c0, lane);
      }
      if (!up && ok) ok = mbar_wait_warp(&bars->tmem_full[acc], (full_par >> acc) & 1, wc, SITE_TMEM_FULL, t, 100);
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive_leader(&bars->tmem_empty[acc]);
      full_par ^= 1u << acc;
      acc ^= 1;
    }
    if (lane == 0) tma_store_wait_all();
  }

  // ---------------------------------------------------------------- teardown
  if (*reinterpret_cast<volatile int*>(&a.status->abort)) __nanosleep(200000);
  tc_fence_before_sync();
  __syncthreads();
  cluster_sync_all();
  if (warp == 1) {
    tc_fence_after_sync();
    tmem_dealloc_pair(tmem_base, TMEM_COLS);
  }
}

template <int WHAT, bool A_MN, bool B_MN>
static cudaError_t launch_one(const MuonProductArgs& a, int num_sms, cudaStream_t s) {
  static PairLaunchState st;
  const int tiles = a.n * muon_tiles<WHAT == MUON_GRAM || WHAT == MUON_POLY>(a);
  const int sms = 2 * tiles < num_sms ? 2 * tiles : num_sms;
  return launch_on_pairs(st, muon_product_kernel<WHAT, A_MN, B_MN>, a, MU_THREADS, MU_SMEM, sms, s, true);
}

cudaError_t launch_muon_product(MuonProduct what, bool a_mn, bool b_mn, const MuonProductArgs& a, int num_sms, cudaStream_t s) {
  switch (what) {
    case MUON_GRAM: return a_mn ? launch_one<MUON_GRAM, true, true>(a, num_sms, s) : launch_one<MUON_GRAM, false, false>(a, num_sms, s);
    case MUON_POLY: return launch_one<MUON_POLY, false, false>(a, num_sms, s);
    case MUON_APPLY: return b_mn ? launch_one<MUON_APPLY, false, true>(a, num_sms, s) : launch_one<MUON_APPLY, false, false>(a, num_sms, s);
    case MUON_LAST: return b_mn ? launch_one<MUON_LAST, false, true>(a, num_sms, s) : launch_one<MUON_LAST, false, false>(a, num_sms, s);
  }
  return cudaErrorInvalidValue;
}

}  // namespace moe
