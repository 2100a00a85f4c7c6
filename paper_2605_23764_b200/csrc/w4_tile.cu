// The layer's expert products over 4-bit weights on the tensor cores: batches and prompts.
//
//   D_g[f][t] = sum over group g of (q - z)[f][k] x[t][k],   h[f][t] = sum_g s[f][g] D_g[f][t]
//
// Tiles are those of the bf16 operators: 256 weight rows of a CTA pair as accumulator rows, up to 128 rows of an expert as
// accumulator columns, x (or A) by TMA.  The weights are the A operand and are read from TMEM: codes travel as they are (a quarter
// of the bytes of bf16), four warps of each CTA widen them to whole numbers q - z -- exact in bf16 -- and write them to TMEM in the
// fragments that the layout of w4.cuh holds, so they never are in shared memory as bf16.  An accumulator holds one group of the
// reduction; the epilogue warps scale it in fp32 and add it up in registers while the next group is multiplied.  So there is no
// rounding that the formula does not have but that of the activations to bf16 between the two products.
//
// Roles per CTA: warp 0 loads codes, scales and zero points, warp 1 issues the products (even CTA), warp 2 loads rows of x, warps 4-7
// widen, warps 8-15 scale and add up.
#include "gemm_tile.cuh"
#include "launch_pairs.cuh"
#include "topk.cuh"
#include "w4.cuh"

namespace moe {

namespace {

constexpr int WT_THREADS = 512;
constexpr int WT_CODES = 4 * W4_UNIT_BYTES;   // 128 rows x 128 columns
constexpr int WT_CODE_STAGES = 4, WT_SCALE_STAGES = 8, WT_TOK_STAGES = 6, WT_A_STAGES = 2, WT_D_BUFS = 3;
constexpr int WT_TOK_BYTES = 64 * 256;        // half of 128 rows x 128 columns bf16
constexpr int WT_A_COLS = 64;                 // TMEM columns of 128 bf16
constexpr int WT_A_AT = WT_D_BUFS * BLOCK_M;  // behind the accumulators
static_assert(WT_A_AT + WT_A_STAGES * WT_A_COLS <= TMEM_COLS, "TMEM");

struct __align__(8) WtBarriers {
  uint64_t code_full[WT_CODE_STAGES], code_empty[WT_CODE_STAGES];      // in each CTA
  uint64_t scale_full[WT_SCALE_STAGES], scale_empty[WT_SCALE_STAGES];  // in each CTA
  uint64_t tok_full[WT_TOK_STAGES];    // even CTA: both CTAs' rows
  uint64_t tok_empty[WT_TOK_STAGES];   // in each CTA
  uint64_t a_full[WT_A_STAGES];        // even CTA: the widening warps of both
  uint64_t a_empty[WT_A_STAGES];       // in each CTA
  uint64_t d_full[WT_D_BUFS];          // in each CTA
  uint64_t d_empty[WT_D_BUFS];         // even CTA: the epilogue warps of both
  uint64_t drain;
  uint32_t tmem_base;
};

__host__ __device__ constexpr int wt_code_stage(int ng, bool asym) { return WT_CODES + (asym ? 128 * ng : 0); }
__host__ __device__ constexpr size_t wt_smem(int ng, bool asym) {
  return 1024 + (size_t)WT_TOK_STAGES * WT_TOK_BYTES + (size_t)WT_CODE_STAGES * wt_code_stage(ng, asym) + (size_t)WT_SCALE_STAGES * 256 * ng +
         sizeof(WtBarriers);
}
static_assert(wt_smem(4, true) <= 227 * 1024, "shared memory");

__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)), "l"(src), "r"(bytes),
               "r"(smem_u32(bar))
               : "memory");
}
// 16 lanes x 32 columns of TMEM from operand fragments: registers 2 i, 2 i + 1 are rows lane / 4 and lane / 4 + 8 of column 4 i + lane % 4
__device__ __forceinline__ void tmem_st_frag8(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile("tcgen05.st.sync.aligned.16x128b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr), "r"(r[0]),
               "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]),
               "r"(r[13]), "r"(r[14]), "r"(r[15])
               : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// One 16-deep product with the A operand in TMEM.
__device__ __forceinline__ void tc_mma_ts_pair(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred e, p;\n .reg .b64 db;\n elect.sync _|e, 0xffffffff;\n setp.ne.b32 p, %5, 0;\n"
      " mov.b64 db, {%2, %3};\n"
      " @e tcgen05.mma.cta_group::2.kind::f16 [%0], [%1], db, %4, p;\n}" ::"r"(d_tmem), "r"(a_tmem), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate)
      : "memory");
}
// mbar_wait_warp with acquire at cluster scope: what the partner CTA wrote before its arrival is visible
__device__ __forceinline__ bool mbar_wait_cluster_warp(uint64_t* bar, uint32_t parity, const WaitCtl& wc, int site, int tile) {
  const bool ok = mbar_wait_cluster(bar, parity, wc, site, tile);
  return __all_sync(0xffffffffu, ok);
}

struct WtItem { int e, nb, row0, ntok; };   // expert, 256-row weight tile, first row, columns (a multiple of 32)
__device__ __forceinline__ WtItem wt_item(const W4TileArgs& a, int t) {
  WtItem it;
  const int mb = t / a.ntn;
  it.nb = t - mb * a.ntn;
  it.e = a.mblk_expert[mb];
  it.row0 = mb * BLOCK_M;
  const int rows = a.counts[it.e] - (mb - a.mb_start[it.e]) * BLOCK_M;
  it.ntok = min(BLOCK_M, (rows + 31) & ~31);
  return it;
}

// Position in a ring of N slots and the parity to wait for next in it.
template <int N>
struct RingAt {
  int s = 0;
  uint32_t par;
  __device__ __forceinline__ explicit RingAt(uint32_t first) : par(first) {}
  __device__ __forceinline__ void next() {
    if (++s == N) { s = 0; par ^= 1; }
  }
};

}  // namespace

template <bool ASYM, int NG>
__global__ void __launch_bounds__(WT_THREADS, 1) w4_tile_kernel(const __grid_constant__ W4TileArgs a) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* const smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  constexpr int CODE_STAGE = wt_code_stage(NG, ASYM), SCALE_STAGE = 256 * NG;
  uint8_t* const tok_s = smem;
  uint8_t* const code_s = tok_s + WT_TOK_STAGES * WT_TOK_BYTES;
  uint8_t* const scale_s = code_s + WT_CODE_STAGES * CODE_STAGE;
  WtBarriers* const bars = reinterpret_cast<WtBarriers*>(scale_s + WT_SCALE_STAGES * SCALE_STAGE);

  const int warp = warp_index(), lane = threadIdx.x & 31;
  const int rank = (int)cluster_ctarank();
  const int pair = blockIdx.x >> 1, npairs = gridDim.x >> 1;
  const WaitCtl wc{a.status, a.budget_ns};

  if (threadIdx.x == 0) {
    for (int i = 0; i < WT_CODE_STAGES; ++i) { mbar_init(&bars->code_full[i], 1); mbar_init(&bars->code_empty[i], 4); }
    for (int i = 0; i < WT_SCALE_STAGES; ++i) { mbar_init(&bars->scale_full[i], 1); mbar_init(&bars->scale_empty[i], 8); }
    for (int i = 0; i < WT_TOK_STAGES; ++i) { mbar_init(&bars->tok_full[i], 1); mbar_init(&bars->tok_empty[i], 1); }
    for (int i = 0; i < WT_A_STAGES; ++i) { mbar_init(&bars->a_full[i], 8); mbar_init(&bars->a_empty[i], 1); }
    for (int i = 0; i < WT_D_BUFS; ++i) { mbar_init(&bars->d_full[i], 1); mbar_init(&bars->d_empty[i], 16); }
    mbar_init(&bars->drain, 1);
    mbar_fence_init();
    fence_proxy_async();
    for (int i = 0; i < 4; ++i) tma_prefetch_desc(&a.tok[i]);
  }
  if (warp == 1) {
    tmem_alloc_pair(&bars->tmem_base, TMEM_COLS);
    tmem_relinquish_pair();
  }
  tc_fence_before_sync();
  __syncthreads();
  cluster_sync_all();   // both CTAs' barriers exist before anyone signals across the pair
  tc_fence_after_sync();
  const uint32_t tmem_base = uniform(bars->tmem_base);
  pdl_trigger();
  pdl_wait();

  const int total = a.meta[0] * a.ntn, KU = a.KU;
  WtItem cur{}, next{};
  if (pair < total) cur = wt_item(a, pair);
  if (warp == 0) {
    // ---- codes, scales, zero points: lane i < 4 has the i-th 32 rows.  Row tiles behind the last are read again and not stored.
    RingAt<WT_CODE_STAGES> cr(1);
    RingAt<WT_SCALE_STAGES> sr(1);
    bool ok = true;
    for (int t = pair; t < total && ok; t += npairs, cur = next) {
      if (t + npairs < total) next = wt_item(a, t + npairs);
      const int rt = min(cur.nb * 8 + rank * 4 + min(lane, 3), a.RT - 1);
      size_t unit = ((size_t)cur.e * a.RT + rt) * KU;
      for (int ku = 0; ku < KU; ++ku, ++unit) {
        if (!mbar_wait_warp(&bars->code_empty[cr.s], cr.par, wc, SITE_EMPTY, t, 20) ||
            !mbar_wait_warp(&bars->scale_empty[sr.s], sr.par, wc, SITE_EMPTY, t, 20)) { ok = false; break; }
        uint8_t *const cs = code_s + cr.s * CODE_STAGE, *const ss = scale_s + sr.s * SCALE_STAGE;
        if (lane == 0) {
          mbar_expect_tx(&bars->code_full[cr.s], CODE_STAGE);
          mbar_expect_tx(&bars->scale_full[sr.s], SCALE_STAGE);
        }
        __syncwarp();
        if (lane < 4) {
          bulk_load(cs + lane * W4_UNIT_BYTES, a.codes + unit * W4_UNIT_BYTES, W4_UNIT_BYTES, &bars->code_full[cr.s]);
          if (ASYM) bulk_load(cs + WT_CODES + lane * 32 * NG, a.zeros + unit * (32 * NG), 32 * NG, &bars->code_full[cr.s]);
          bulk_load(ss + lane * 64 * NG, a.scales + unit * (64 * NG), 64 * NG, &bars->scale_full[sr.s]);
        }
        cr.next();
        sr.next();
      }
    }
  } else if (warp == 2) {
    // ---- rows of x: this CTA's half, two boxes of 64 columns
    RingAt<WT_TOK_STAGES> tr(1);
    bool ok = true;
    for (int t = pair; t < total && ok; t += npairs, cur = next) {
      if (t + npairs < total) next = wt_item(a, t + npairs);
      const int ntok = uniform(cur.ntok), half = ntok >> 1, row = uniform(cur.row0) + rank * half;
      const CUtensorMap* tm = &a.tok[(half >> 4) - 1];
      for (int ku = 0; ku < KU; ++ku) {
        if (!mbar_wait_warp(&bars->tok_empty[tr.s], tr.par, wc, SITE_EMPTY, t, 20)) { ok = false; break; }
        uint8_t* const ts = tok_s + tr.s * WT_TOK_BYTES;
        if (rank == 0) mbar_expect_tx_elect(&bars->tok_full[tr.s], (uint32_t)ntok * 256);
        tma_load_2d_pair(ts, tm, ku * W4_UNIT_K, row, &bars->tok_full[tr.s]);
        tma_load_2d_pair(ts + half * 128, tm, ku * W4_UNIT_K + 64, row, &bars->tok_full[tr.s]);
        tr.next();
      }
    }
  } else if (warp == 1 && rank == 0) {
    // ---- products
    RingAt<WT_TOK_STAGES> tr(0);
    RingAt<WT_A_STAGES> ar(0);
    RingAt<WT_D_BUFS> dr(1);
    bool ok = true;
    constexpr int STEPS = 8 / NG;   // of 16 columns in a group
    for (int t = pair; t < total && ok; t += npairs, cur = next) {
      if (t + npairs < total) next = wt_item(a, t + npairs);
      const int ntok = uniform(cur.ntok);
      const uint32_t idesc = make_idesc_bf16(2 * BLOCK_M, ntok, 0, 0), box = (uint32_t)(ntok >> 1) * 128 >> 4;
      for (int ku = 0; ku < KU && ok; ++ku) {
        if (!mbar_wait_warp(&bars->tok_full[tr.s], tr.par, wc, SITE_FULL, t) ||
            !mbar_wait_cluster_warp(&bars->a_full[ar.s], ar.par, wc, SITE_FULL, t)) { ok = false; break; }
        const uint32_t b_lo = smem_desc_lo(smem_u32(tok_s + tr.s * WT_TOK_BYTES), 16);
        const uint32_t a_t = tmem_base + WT_A_AT + ar.s * WT_A_COLS;
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          if (!mbar_wait_warp(&bars->d_empty[dr.s], dr.par, wc, SITE_TMEM_EMPTY, t)) { ok = false; break; }
          tc_fence_after_sync();
          const uint32_t d_t = tmem_base + dr.s * BLOCK_M;
#pragma unroll
          for (int j = 0; j < STEPS; ++j) {
            const int k16 = g * STEPS + j;
            tc_mma_ts_pair(d_t, a_t + 8 * k16, b_lo + (k16 >> 2) * box + 2 * (k16 & 3), smem_desc_hi(1024), idesc, j != 0);
          }
          tc_commit_pair(&bars->d_full[dr.s]);
          dr.next();
        }
        tc_commit_pair(&bars->a_empty[ar.s]);
        tc_commit_pair(&bars->tok_empty[tr.s]);
        ar.next();
        tr.next();
      }
    }
    if (uniform(!ok || *reinterpret_cast<volatile int*>(&a.status->abort) ? 1 : 0)) {   // let what was issued end before TMEM is freed
      tc_commit_pair(&bars->drain);
      const WaitCtl shortwc{a.status, 20ull * 1000 * 1000};
      mbar_wait_warp(&bars->drain, 0, shortwc, SITE_DRAIN, 0);
    }
  } else if (warp >= 4 && warp < 8) {
    // ---- codes to whole numbers in TMEM: a warp has the 32 lanes of its quarter
    RingAt<WT_CODE_STAGES> cr(0);
    RingAt<WT_A_STAGES> ar(1);
    const int quad = warp & 3, g = lane >> 2;
    const uint32_t lanes = (uint32_t)(quad * 32) << 16;
    bool ok = true;
    for (int t = pair; t < total && ok; t += npairs) {
      for (int ku = 0; ku < KU; ++ku) {
        if (!mbar_wait_warp(&bars->code_full[cr.s], cr.par, wc, SITE_FULL, t)) { ok = false; break; }
        const uint8_t* const cs = code_s + cr.s * CODE_STAGE + quad * W4_UNIT_BYTES + lane * 16;
        uint4 q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = *reinterpret_cast<const uint4*>(cs + 512 * i);
        uint32_t zp[ASYM ? NG : 1];
        if constexpr (ASYM) {
          const uint32_t* z = reinterpret_cast<const uint32_t*>(code_s + cr.s * CODE_STAGE + WT_CODES + quad * 32 * NG + g * 4 * NG);
#pragma unroll
          for (int i = 0; i < NG; ++i) zp[i] = z[i];
        }
        if (!mbar_wait_warp(&bars->a_empty[ar.s], ar.par, wc, SITE_TMEM_EMPTY, t)) { ok = false; break; }
        tc_fence_after_sync();
        const uint32_t a_t = tmem_base + lanes + WT_A_AT + ar.s * WT_A_COLS;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int s = 0; s < 2; ++s) {   // halves of 64 columns, sixteen rows
            const uint4 w = q[2 * h + s];
            const uint32_t words[4] = {w.x, w.y, w.z, w.w};
            uint32_t v[16];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const int grp = (4 * h + j) * NG / 8;
              const uint32_t z = ASYM ? zp[ASYM ? grp : 0] >> (16 * s) : 0;
              uint32_t f[4];
              w4_fragment(words[j], f);
              const uint32_t lo = ASYM ? w4_bias(z & 0xFFu) : w4_bias(8), hi = ASYM ? w4_bias((z >> 8) & 0xFFu) : w4_bias(8);
#pragma unroll
              for (int r = 0; r < 4; ++r) v[4 * j + r] = add_bf16x2(f[r], r & 1 ? hi : lo);
            }
            tmem_st_frag8(a_t + ((uint32_t)(16 * s) << 16) + 32 * h, v);
          }
        tmem_st_wait();
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive_cluster_addr(smem_u32(&bars->a_full[ar.s]) & PEER_BIT_MASK);
          mbar_arrive_cta(&bars->code_empty[cr.s]);
        }
        cr.next();
        ar.next();
      }
    }
  } else if (warp >= 8) {
    // ---- groups scaled and added up: a thread has a weight row, half of the columns
    RingAt<WT_SCALE_STAGES> sr(0);
    RingAt<WT_D_BUFS> dr(0);
    const int quad = warp & 3, side = (warp - 8) >> 2;
    const uint32_t lanes = (uint32_t)(quad * 32) << 16;
    bool ok = true;
    for (int t = pair; t < total && ok; t += npairs, cur = next) {
      if (t + npairs < total) next = wt_item(a, t + npairs);
      const int cols = uniform(cur.ntok) >> 1, c0 = side * cols;   // 16, 32, 48 or 64 columns
      float acc[64];
#pragma unroll
      for (int i = 0; i < 64; ++i) acc[i] = 0.f;
      for (int ku = 0; ku < KU && ok; ++ku) {
        if (!mbar_wait_warp(&bars->scale_full[sr.s], sr.par, wc, SITE_FULL, t)) { ok = false; break; }
        float sc[NG];
#pragma unroll
        for (int g = 0; g < NG; ++g)
          sc[g] = __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(scale_s + sr.s * SCALE_STAGE + quad * 64 * NG + ((lane & 7) * NG + g) * 8 +
                                                                                (lane >> 3) * 2)
                                  << 16);
        __syncwarp();
        if (lane == 0) mbar_arrive_cta(&bars->scale_empty[sr.s]);
        sr.next();
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          if (!mbar_wait_warp(&bars->d_full[dr.s], dr.par, wc, SITE_TMEM_FULL, t)) { ok = false; break; }
          tc_fence_after_sync();
          const uint32_t d_t = tmem_base + lanes + dr.s * BLOCK_M + c0;
#pragma unroll
          for (int c = 0; c < 4; ++c)
            if (16 * c < cols) {
              float v[16];
              tmem_ld16(d_t + 16 * c, v);
              tmem_ld_wait();
#pragma unroll
              for (int i = 0; i < 16; ++i) acc[16 * c + i] = fmaf(sc[g], v[i], acc[16 * c + i]);
            }
          tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) mbar_arrive_leader(&bars->d_empty[dr.s]);
          dr.next();
        }
      }
      if (!ok) break;
      const int rt = cur.nb * 8 + rank * 4 + quad;   // the warp's 32 rows
      const int rows = cur.row0 + c0;
      if (rt < a.RT) {
        if (a.down) {
          const int feature = rt * 32 + lane;
          if (feature < a.n_out) {
            float* y = a.Y + (size_t)rows * a.y_ld + feature;
#pragma unroll
            for (int i = 0; i < 64; ++i)
              if (i < cols) { *y = acc[i]; y += a.y_ld; }
          }
        } else {
          // lanes 0-7 and 16-23 have gate rows, the others the up rows of the same features: of two columns each takes one
          const bool is_up = lane & 8;
          const int feature = rt * 16 + ((lane >> 4) << 3) + (lane & 7);
          const int row = rows + (is_up ? 1 : 0);
          uint16_t* out = a.A + (size_t)row * a.a_ld + feature;
          const float* w = a.prow_w + row;
#pragma unroll
          for (int i = 0; i < 64; i += 2)
            if (i < cols) {
              const float other = __shfl_xor_sync(0xffffffffu, is_up ? acc[i] : acc[i + 1], 8);
              const float gate = is_up ? other : acc[i], up = is_up ? acc[i + 1] : other;
              const float act = __ldg(w + i) * (gate / (1.0f + __expf(-gate)) * up);
              if (feature < a.n_out) *out = (uint16_t)(pack_bf16x2(act, 0.f) & 0xFFFFu);
              out += 2 * (size_t)a.a_ld;
            }
        }
      }
    }
  }

  // ---------------------------------------------------------------- teardown
  if (*reinterpret_cast<volatile int*>(&a.status->abort)) __nanosleep(200000);
  tc_fence_before_sync();
  __syncthreads();
  cluster_sync_all();   // neither CTA leaves while its partner may still read its shared memory or signal it
  if (warp == 1) {
    tc_fence_after_sync();
    tmem_dealloc_pair(tmem_base, TMEM_COLS);
  }
}

template <bool ASYM, int NG>
static cudaError_t launch_tile(const W4TileArgs& a, int num_sms, cudaStream_t st) {
  static PairLaunchState state;
  return launch_on_pairs(state, w4_tile_kernel<ASYM, NG>, a, WT_THREADS, wt_smem(NG, ASYM), num_sms, st, true);
}

cudaError_t launch_w4_tile(const W4TileArgs& a, int num_sms, cudaStream_t st, int* launches) {
  ++*launches;
  const bool asym = a.zeros != nullptr;
  switch (a.group) {
    case 128: return asym ? launch_tile<true, 1>(a, num_sms, st) : launch_tile<false, 1>(a, num_sms, st);
    case 64: return asym ? launch_tile<true, 2>(a, num_sms, st) : launch_tile<false, 2>(a, num_sms, st);
    default: return asym ? launch_tile<true, 4>(a, num_sms, st) : launch_tile<false, 4>(a, num_sms, st);
  }
}

}  // namespace moe
