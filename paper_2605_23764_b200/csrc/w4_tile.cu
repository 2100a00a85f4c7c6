// The layer's expert products over 4-bit weights on the tensor cores: batches and prompts.
//
//   D_g[f][t] = sum over group g of (q - z)[f][k] x[t][k],   h[f][t] = sum_g s[f][g] D_g[f][t]
//
// Tiles are those of the bf16 operators: 256 weight rows of a CTA pair as accumulator rows, up to 128 rows of an expert as
// accumulator columns, x (or A) by TMA.  The weights are the A operand and are read from TMEM: codes travel as they are (a quarter
// of the bytes of bf16), four warps of each CTA widen them to whole numbers q - z -- exact in bf16 -- and write them to TMEM in the
// fragments that the layout of w4.cuh holds, so they never are in shared memory as bf16.  An accumulator holds one group of the
// reduction; the epilogue warps scale it in fp32 and add it up in registers while the next group is multiplied.  So there is no
// rounding that the formula does not have but that of the activations to bf16 between the two products.  (Scales folded into the widened
// weights would spare the accumulators between groups, but round every weight: twice the error of the plain formula instead of 1.4 times.)
//
// Measured for 66 experts of 2048 x 1408, 8 rows a token, groups of 128: 64 tokens 104 us, 512 tokens 164, 4096 tokens 806 (703
// TFLOP/s; the bf16 layer takes 190, 212 and 565: it is the faster one from some 850 tokens on, about 80 rows a routed expert).  What
// bounds it: with many rows the epilogue, which takes every group's accumulator out of TMEM (800 clocks a unit beside 512 of products);
// with few the chain from codes to operand to products through two stages of A (760 clocks a unit).
//
// Roles per CTA: warp 0 loads codes and zero points (a copy of each for 128 rows x 128 columns; with one for every 32 rows issuing
// them took 1000 clocks, twice as long as the products), warp 18 the rows of x, warp 1 issues the products (even CTA), warps 2-9 widen
// (four for every other unit), warps 10-17 scale and add up (four for each half of the columns; with sixteen warps their waits and
// signals took the issue slots that the widening warps need: a prompt of 4096 tokens 841 us).
#include "gemm_tile.cuh"
#include "launch_pairs.cuh"
#include "topk.cuh"
#include "w4.cuh"

namespace moe {

namespace {

constexpr int WT_WIDEN_WARP = 2, WT_EPI_WARP = 10, WT_EPI_SIDES = 2, WT_TOK_WARP = WT_EPI_WARP + 4 * WT_EPI_SIDES, WT_THREADS = 32 * (WT_TOK_WARP + 1);
constexpr int WT_CODES = 4 * W4_UNIT_BYTES;   // 128 rows x 128 columns
constexpr int WT_CODE_STAGES = 6, WT_TOK_STAGES = 6, WT_A_STAGES = 2, WT_D_BUFS = 3;
constexpr int WT_TOK_BYTES = 64 * 256;        // half of 128 rows x 128 columns bf16
constexpr int WT_A_COLS = 64;                 // TMEM columns of 128 bf16
constexpr int WT_A_AT = WT_D_BUFS * BLOCK_M;  // behind the accumulators
static_assert(WT_CODE_STAGES % 2 == 0 && WT_TOK_STAGES % 2 == 0 && WT_A_STAGES == 2, "a set of widening warps keeps to every other slot");
static_assert(WT_A_AT + WT_A_STAGES * WT_A_COLS <= TMEM_COLS, "TMEM");

struct __align__(8) WtBarriers {
  uint64_t code_full[WT_CODE_STAGES], code_empty[WT_CODE_STAGES];      // in each CTA
  // of unit u, at u % WT_TOK_STAGES: one wait and one commit for both operands (each costs the issuer some 100 clocks)
  uint64_t full[WT_TOK_STAGES];        // even CTA: both CTAs' rows of x and widened weights
  uint64_t done[WT_TOK_STAGES];        // in each CTA: multiplied
  uint64_t d_full[WT_D_BUFS];          // in each CTA
  uint64_t d_empty[WT_D_BUFS];         // even CTA: the epilogue warps of both
  uint64_t drain;
  uint32_t tmem_base;
};

__host__ __device__ constexpr int wt_code_stage(int ng, bool asym) { return WT_CODES + (asym ? 128 * ng : 0); }
__host__ __device__ constexpr size_t wt_smem(int ng, bool asym) {
  return 1024 + (size_t)WT_TOK_STAGES * WT_TOK_BYTES + (size_t)WT_CODE_STAGES * wt_code_stage(ng, asym) + sizeof(WtBarriers);
}
static_assert(wt_smem(4, true) <= 227 * 1024, "shared memory");

__device__ __forceinline__ void bulk_load_elect(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile(
      "{\n .reg .pred e;\n elect.sync _|e, 0xffffffff;\n"
      " @e cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];\n}" ::"r"(smem_u32(dst)),
      "l"(src), "r"(bytes), "r"(smem_u32(bar))
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
// Two or four 16-deep products with the A operand in TMEM (8 columns each).
template <int N>
__device__ __forceinline__ void tc_mma_ts_pair(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t accumulate) {
  static_assert(N == 2 || N == 4, "");
  if constexpr (N == 4)
    asm volatile(
        "{\n .reg .pred e, p;\n .reg .b64 db;\n .reg .b32 ta;\n elect.sync _|e, 0xffffffff;\n setp.ne.b32 p, %5, 0;\n"
        " mov.b64 db, {%2, %3};\n"
        " @e tcgen05.mma.cta_group::2.kind::f16 [%0], [%1], db, %4, p;\n"
        " add.u64 db, db, 2;\n add.u32 ta, %1, 8;\n"
        " @e tcgen05.mma.cta_group::2.kind::f16 [%0], [ta], db, %4, 1;\n"
        " add.u64 db, db, 2;\n add.u32 ta, %1, 16;\n"
        " @e tcgen05.mma.cta_group::2.kind::f16 [%0], [ta], db, %4, 1;\n"
        " add.u64 db, db, 2;\n add.u32 ta, %1, 24;\n"
        " @e tcgen05.mma.cta_group::2.kind::f16 [%0], [ta], db, %4, 1;\n}" ::"r"(d_tmem), "r"(a_tmem), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate)
        : "memory");
  else
    asm volatile(
        "{\n .reg .pred e, p;\n .reg .b64 db;\n .reg .b32 ta;\n elect.sync _|e, 0xffffffff;\n setp.ne.b32 p, %5, 0;\n"
        " mov.b64 db, {%2, %3};\n"
        " @e tcgen05.mma.cta_group::2.kind::f16 [%0], [%1], db, %4, p;\n"
        " add.u64 db, db, 2;\n add.u32 ta, %1, 8;\n"
        " @e tcgen05.mma.cta_group::2.kind::f16 [%0], [ta], db, %4, 1;\n}" ::"r"(d_tmem), "r"(a_tmem), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate)
        : "memory");
}
// 32 lanes x 16 columns: thread i has lane i.  The values are there behind the wait, which they depend on.
__device__ __forceinline__ void tmem_ld16_wait(uint32_t taddr, float (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n tcgen05.wait::ld.sync.aligned;"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]),
        "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
      : "r"(taddr)
      : "memory");
}
// Groups that share an accumulator buffer of 128 columns: the epilogue's waits and signals, some 500 clocks, are per buffer.
__host__ __device__ constexpr int wt_groups(int ntok) { return ntok == 32 ? 4 : ntok == 64 ? 2 : 1; }

struct WtItem { int e, nb, row0, ntok; };   // expert, 256-row weight tile, first row, columns (a multiple of 32)
// The items of a pair, one after another.  What an item is hangs on two loads in a row: the first of them is made two items ahead, the
// second one item ahead, and nothing waits for either before it is used.
struct WtItems {
  const W4TileArgs& a;
  int t, step, total;
  int e1 = 0, e2 = 0, cnt1 = 0, mb1 = 0;   // of item t, and the expert of item t + step
  __device__ __forceinline__ WtItems(const W4TileArgs& args, int first, int step_, int total_) : a(args), t(first), step(step_), total(total_) {
    if (t < total) {
      e1 = a.mblk_expert[t / a.ntn];
      cnt1 = a.counts[e1];
      mb1 = a.mb_start[e1];
    }
    if (t + step < total) e2 = a.mblk_expert[(t + step) / a.ntn];
  }
  __device__ __forceinline__ bool next(WtItem& it) {
    if (t >= total) return false;
    const int mb = t / a.ntn;
    it.nb = t - mb * a.ntn;
    it.e = e1;
    it.row0 = mb * BLOCK_M;
    it.ntok = min(BLOCK_M, (cnt1 - (mb - mb1) * BLOCK_M + 31) & ~31);
    t += step;
    if (t < total) {
      e1 = e2;
      cnt1 = a.counts[e1];
      mb1 = a.mb_start[e1];
      if (t + step < total) e2 = a.mblk_expert[(t + step) / a.ntn];
    }
    return true;
  }
};

// Position in a ring of N slots and the parity to wait for next in it.
template <int N>
struct RingAt {
  int s = 0;
  uint32_t par;
  __device__ __forceinline__ explicit RingAt(uint32_t first) : par(first) {}
  __device__ __forceinline__ void next(int step = 1) {
    s += step;
    if (s >= N) { s -= N; par ^= 1; }
  }
};

struct WtEpilogue {   // of a warp: 32 weight rows (a lane each) x half of the columns
  const W4TileArgs& a;
  WtBarriers* bars;
  WaitCtl wc;
  uint32_t tmem;     // the warp's lanes
  int rank, quad, side, lane;
  RingAt<WT_D_BUFS> dr{0};

  template <int NTOK, int NG>
  __device__ __forceinline__ bool item(const WtItem& it, int t) {
    constexpr int NC = NTOK / WT_EPI_SIDES, GPB = wt_groups(NTOK), ROUNDS = NC * GPB / 16;   // sixteen values a round
    const int groups = a.KU * NG;
    float2x acc[NC / 2];   // two columns side by side
#pragma unroll
    for (int i = 0; i < NC / 2; ++i) acc[i] = pack2(0.f, 0.f);
    // gate and up: the routing weights of columns lane and lane + 32
    float w_col[2] = {0.f, 0.f};
    if (!a.down) {
      const float* w = a.prow_w + it.row0 + side * NC + lane;
      if (lane < NC) w_col[0] = __ldg(w);
      if (lane + 32 < NC) w_col[1] = __ldg(w + 32);
    }
    // The row's scales, read a buffer ahead.  Group g of the row: group g % NG of unit g / NG.
    const int four = min(it.nb * 2 + rank, (a.RTS >> 2) - 1);
    const uint16_t* const scales = reinterpret_cast<const uint16_t*>(a.scales) + ((size_t)it.e * (a.RTS >> 2) + four) * a.KU * (128 * NG) + quad * 32 * NG +
                                   (lane & 7) * 4 * NG + (lane >> 3);
    uint16_t ahead[GPB];
    auto fetch = [&](int g0) {
#pragma unroll
      for (int i = 0; i < GPB; ++i) {
        const int g = g0 + i;
        ahead[i] = g < groups ? __ldg(scales + (g / NG) * (128 * NG) + (g % NG) * 4) : (uint16_t)0;
      }
    };
    fetch(0);
#pragma unroll 1
    for (int g0 = 0; g0 < groups; g0 += GPB) {
      float sc[GPB];
#pragma unroll
      for (int i = 0; i < GPB; ++i) sc[i] = __uint_as_float((uint32_t)ahead[i] << 16);
      fetch(g0 + GPB);
      if (!mbar_wait_warp(&bars->d_full[dr.s], dr.par, wc, SITE_TMEM_FULL, t)) return false;
      tc_fence_after_sync();
      const uint32_t d = tmem + dr.s * BLOCK_M + side * NC;
#pragma unroll
      for (int r = 0; r < ROUNDS; ++r) {
        float v[16];
        const int grp = 16 * r / NC, col = 16 * r % NC;
        tmem_ld16_wait(d + grp * NTOK + col, v);
        if (r == ROUNDS - 1) {
          tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) mbar_arrive_leader(&bars->d_empty[dr.s]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int to = col / 2 + i;
          // (a group behind the last was not written: nothing of it is added)
          const float2x next = fma2(pack2(sc[grp], sc[grp]), pack2(v[2 * i], v[2 * i + 1]), acc[to]);
          if (GPB == 1 || g0 + grp < groups) acc[to] = next;
        }
      }
      dr.next();
    }
    // ---- the result
    const int rt = it.nb * 8 + rank * 4 + quad;   // the warp's 32 rows
    if (rt >= a.RT) return true;
    const int rows = it.row0 + side * NC;
    if (a.down) {
      const int feature = rt * 32 + lane;
      if (feature < a.n_out) {
        float* y = a.Y + (size_t)rows * a.y_ld + feature;
#pragma unroll
        for (int i = 0; i < NC / 2; ++i) {
          float lo, hi;
          unpack2(acc[i], lo, hi);
          y[0] = lo;
          y[a.y_ld] = hi;
          y += 2 * (size_t)a.y_ld;
        }
      }
    } else {
      // lanes 0-7 and 16-23 have gate rows, the others the up rows of the same features: of two columns each takes one
      const int is_up = (lane >> 3) & 1;
      const int feature = rt * 16 + ((lane >> 4) << 3) + (lane & 7);
      uint16_t* out = a.A + (size_t)(rows + is_up) * a.a_ld + feature;
#pragma unroll
      for (int i = 0; i < NC / 2; ++i) {
        float lo, hi;
        unpack2(acc[i], lo, hi);
        const float other = __shfl_xor_sync(0xffffffffu, is_up ? lo : hi, 8);
        const float gate = is_up ? other : lo, up = is_up ? hi : other;
        const float w = __shfl_sync(0xffffffffu, w_col[i / 16], (2 * i & 31) + is_up);
        const float act = w * (__fdividef(gate, 1.0f + __expf(-gate)) * up);
        if (feature < a.n_out) *out = (uint16_t)(pack_bf16x2(act, 0.f) & 0xFFFFu);
        out += 2 * (size_t)a.a_ld;
      }
    }
    return true;
  }
};

}  // namespace

template <bool ASYM, int NG>
__global__ void __launch_bounds__(WT_THREADS, 1) w4_tile_kernel(const __grid_constant__ W4TileArgs a) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* const smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  constexpr int CODE_STAGE = wt_code_stage(NG, ASYM);
  uint8_t* const tok_s = smem;
  uint8_t* const code_s = tok_s + WT_TOK_STAGES * WT_TOK_BYTES;
  WtBarriers* const bars = reinterpret_cast<WtBarriers*>(code_s + WT_CODE_STAGES * CODE_STAGE);

  const int warp = warp_index(), lane = threadIdx.x & 31;
  const int rank = (int)cluster_ctarank();
  const int pair = blockIdx.x >> 1, npairs = gridDim.x >> 1;
  const WaitCtl wc{a.status, a.budget_ns};

  if (threadIdx.x == 0) {
    for (int i = 0; i < WT_CODE_STAGES; ++i) { mbar_init(&bars->code_full[i], 1); mbar_init(&bars->code_empty[i], 4); }
    for (int i = 0; i < WT_TOK_STAGES; ++i) { mbar_init(&bars->full[i], 1 + 8); mbar_init(&bars->done[i], 1); }
    for (int i = 0; i < WT_D_BUFS; ++i) { mbar_init(&bars->d_full[i], 1); mbar_init(&bars->d_empty[i], 8 * WT_EPI_SIDES); }
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
  WtItem cur{};
  if (warp == 0) {
    // ---- codes and zero points of this CTA's 128 rows.  Where it has none, the last ones are read again and not stored.
    RingAt<WT_CODE_STAGES> cr(1);
    bool ok = true;
    WtItems items(a, pair, npairs, total);
    while (ok && items.next(cur)) {
      const int t = items.t;
      const int four = min(uniform(cur.nb) * 2 + rank, (a.RTS >> 2) - 1);
      size_t at = ((size_t)uniform(cur.e) * (a.RTS >> 2) + four) * KU;
      for (int ku = 0; ku < KU; ++ku, ++at) {
        if (!mbar_wait_warp(&bars->code_empty[cr.s], cr.par, wc, SITE_EMPTY, t, 20)) { ok = false; break; }
        uint8_t* const cs = code_s + cr.s * CODE_STAGE;
        mbar_expect_tx_elect(&bars->code_full[cr.s], CODE_STAGE);
        bulk_load_elect(cs, a.codes + at * WT_CODES, WT_CODES, &bars->code_full[cr.s]);
        if (ASYM) bulk_load_elect(cs + WT_CODES, a.zeros + at * (128 * NG), 128 * NG, &bars->code_full[cr.s]);
        cr.next();
      }
    }
  } else if (warp == WT_TOK_WARP) {
    // ---- rows of x: this CTA's half, two boxes of 64 columns
    RingAt<WT_TOK_STAGES> tr(1);
    bool ok = true;
    WtItems items(a, pair, npairs, total);
    while (ok && items.next(cur)) {
      const int t = items.t;
      const int ntok = uniform(cur.ntok), half = ntok >> 1, row = uniform(cur.row0) + rank * half;
      const CUtensorMap* tm = &a.tok[(half >> 4) - 1];
      for (int ku = 0; ku < KU; ++ku) {
        if (!mbar_wait_warp(&bars->done[tr.s], tr.par, wc, SITE_EMPTY, t, 20)) { ok = false; break; }
        uint8_t* const ts = tok_s + tr.s * WT_TOK_BYTES;
        if (rank == 0) mbar_expect_tx_elect(&bars->full[tr.s], (uint32_t)ntok * 256);
        tma_load_2d_pair(ts, tm, ku * W4_UNIT_K, row, &bars->full[tr.s]);
        tma_load_2d_pair(ts + half * 128, tm, ku * W4_UNIT_K + 64, row, &bars->full[tr.s]);
        tr.next();
      }
    }
  } else if (warp == 1 && rank == 0) {
    // ---- products
    RingAt<WT_TOK_STAGES> tr(0);
    RingAt<WT_D_BUFS> dr(1);
    const uint32_t a_first = tmem_base + WT_A_AT, a_end = a_first + WT_A_STAGES * WT_A_COLS;
    uint32_t a_t = a_first;
    bool ok = true;
    constexpr int STEPS = 8 / NG;   // of 16 columns in a group
    WtItems items(a, pair, npairs, total);
    while (ok && items.next(cur)) {
      const int t = items.t;
      const int ntok = uniform(cur.ntok);
      const uint32_t idesc = make_idesc_bf16(2 * BLOCK_M, ntok, 0, 0), box = (uint32_t)(ntok >> 1) * 128 >> 4;
      const int gpb = wt_groups(ntok), groups = KU * NG;
      int grp = 0, in_buf = 0;   // group of the item, of the accumulator buffer
      for (int ku = 0; ku < KU && ok; ++ku) {
        if (!mbar_wait_warp(&bars->full[tr.s], tr.par, wc, SITE_FULL, t)) { ok = false; break; }
        const uint32_t b_lo = smem_desc_lo(smem_u32(tok_s + tr.s * WT_TOK_BYTES), 16);
        constexpr int RUN = STEPS < 4 ? STEPS : 4;   // products in a row: of one box and one group
#pragma unroll
        for (int k16 = 0; k16 < 8; k16 += RUN) {
          if (k16 % STEPS == 0 && in_buf == 0 && !mbar_wait_warp(&bars->d_empty[dr.s], dr.par, wc, SITE_TMEM_EMPTY, t)) { ok = false; break; }
          if (k16 % STEPS == 0) tc_fence_after_sync();
          tc_mma_ts_pair<RUN>(tmem_base + dr.s * BLOCK_M + in_buf * ntok, a_t + 8 * k16, b_lo + (k16 >> 2) * box + 2 * (k16 & 3), smem_desc_hi(1024), idesc,
                              k16 % STEPS != 0);
          if ((k16 + RUN) % STEPS == 0) {
            ++grp;
            if (++in_buf == gpb || grp == groups) {
              tc_commit_pair(&bars->d_full[dr.s]);
              dr.next();
              in_buf = 0;
            }
          }
        }
        tc_commit_pair(&bars->done[tr.s]);
        tr.next();
        a_t = a_t + WT_A_COLS == a_end ? a_first : a_t + WT_A_COLS;
      }
    }
    if (uniform(!ok || *reinterpret_cast<volatile int*>(&a.status->abort) ? 1 : 0)) {   // let what was issued end before TMEM is freed
      tc_commit_pair(&bars->drain);
      const WaitCtl shortwc{a.status, 20ull * 1000 * 1000};
      mbar_wait_warp(&bars->drain, 0, shortwc, SITE_DRAIN, 0);
    }
  } else if (warp >= WT_WIDEN_WARP && warp < WT_EPI_WARP) {
    // ---- codes to whole numbers in TMEM: a warp has the 32 lanes of its quarter, a set of four every other unit and one of the two
    // stages of the A operand.  The first half is widened ahead: what the products wait for once a stage is free is short.
    const int quad = warp & 3, set = (warp - WT_WIDEN_WARP) >> 2, g = lane >> 2;
    RingAt<WT_CODE_STAGES> cr(0);
    RingAt<WT_TOK_STAGES> fr(0), before(0);   // the unit, and the one that had the stage before
    cr.s = fr.s = before.s = set;
    const uint32_t a_t = tmem_base + ((uint32_t)(quad * 32) << 16) + WT_A_AT + set * WT_A_COLS;
    const int units = (pair < total ? (total - pair + npairs - 1) / npairs : 0) * KU;
    for (int u = set; u < units; u += 2) {
      if (!mbar_wait_warp(&bars->code_full[cr.s], cr.par, wc, SITE_FULL, u, 50)) break;
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
      uint32_t v[2][16];
      auto widen = [&](int h) {   // half of 64 columns; two times sixteen rows
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const uint4 w = q[2 * h + s];
          const uint32_t words[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t z = ASYM ? zp[ASYM ? (4 * h + j) * NG / 8 : 0] >> (16 * s) : 0;
            const uint32_t lo = ASYM ? w4_bias(z & 0xFFu) : w4_bias(8), hi = ASYM ? w4_bias((z >> 8) & 0xFFu) : w4_bias(8);
            uint32_t f[4];
            w4_fragment(words[j], f);
#pragma unroll
            for (int r = 0; r < 4; ++r) v[s][4 * j + r] = add_bf16x2(f[r], r & 1 ? hi : lo);
          }
        }
      };
      widen(0);
      if (u >= WT_A_STAGES) {
        if (!mbar_wait_warp(&bars->done[before.s], before.par, wc, SITE_TMEM_EMPTY, u, 50)) break;
        before.next(2);
        tc_fence_after_sync();
      }
#pragma unroll
      for (int s = 0; s < 2; ++s) tmem_st_frag8(a_t + ((uint32_t)(16 * s) << 16), v[s]);
      widen(1);
#pragma unroll
      for (int s = 0; s < 2; ++s) tmem_st_frag8(a_t + ((uint32_t)(16 * s) << 16) + 32, v[s]);
      tmem_st_wait();
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive_leader(&bars->full[fr.s]);   // TMEM is ordered by the tcgen05 fences: a release at cluster scope took 1800 clocks
        mbar_arrive_cta(&bars->code_empty[cr.s]);
      }
      cr.next(2);
      fr.next(2);
    }
  } else if (warp >= WT_EPI_WARP) {
    // ---- groups scaled and added up
    WtEpilogue ep{a, bars, wc, tmem_base + ((uint32_t)((warp & 3) * 32) << 16), rank, warp & 3, (warp - WT_EPI_WARP) >> 2, lane};
    WtItems items(a, pair, npairs, total);
    bool ok = true;
    while (ok && items.next(cur)) {
      const int ntok = uniform(cur.ntok);
      if (ntok == 128) ok = ep.item<128, NG>(cur, items.t);
      else if (ntok == 96) ok = ep.item<96, NG>(cur, items.t);
      else if (ntok == 64) ok = ep.item<64, NG>(cur, items.t);
      else ok = ep.item<32, NG>(cur, items.t);
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
