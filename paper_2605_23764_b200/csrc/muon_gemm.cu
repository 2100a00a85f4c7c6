// The products of an orthogonalisation (muon.cuh) on the tensor cores: one persistent launch for all steps of a batch of matrices.
//
// Items are tiles of 256 rows x 256 columns (fewer where there are not enough of them) of one matrix's product.  The products of a matrix
// follow one another; an item waits until all items of its matrix's product before have been stored (a counter a matrix), which other
// matrices' tiles cover.  CTA pairs take items from a ticket in that order, so whichever pairs are resident make progress.  The accumulator
// is one of two in TMEM: a tile's products run beside the epilogue of the one before.
//
// Operands come in as they lie: K-major where the reduction is contiguous, MN-major where it is the rows (X as the second operand of
// B X, both of X^T X), so nothing is ever transposed in memory.  A, B and their like are symmetric: tiles above the diagonal are neither
// computed nor stored, and an operand's k-blocks that would lie there are read from their mirror image, MN-major -- the instruction
// descriptor changes from k-block to k-block.  (Stored twice, as they are and mirrored, 132 matrices 1408 x 2048 took 18 % longer.)
//
// Where there are few tiles and a long reduction, GRAM sums parts of it and JOIN adds them up in their order (one matrix of 256 x 7168:
// 210 -> 140 us).
//
// What bounds it.  Large batches: power.  The tensor pipe is active 68 to 77 % of the clocks, at 1.4 GHz under the limit; 1.03 to 1.26 PFLOP/s
// of executed products, where batched fp16 products of these shapes by the vendor's library sustain 1.07 and 1.16.  Without an epilogue
// it is 78 to 85 %: a k-block brings 32 KB into an SM and the products read as much, near what shared memory gives in the products' 512 clocks.
// Few matrices: latency, 3.7 us a product from the signal of the one before (poll 0.5, loads 0.8, products and commit 0.6 and up,
// epilogue 0.5 to 2.5, stores and signal 0.8).
//
// Roles per CTA: warp 0 TMA producer, warp 1 MMA issuer (even CTA) or tickets (odd CTA) and TMEM owner, warps 2-9 epilogue.
#include <cuda_fp16.h>
#include <limits.h>

#include "gemm_tile.cuh"
#include "launch_pairs.cuh"
#include "muon.cuh"
#include "topk.cuh"

namespace moe {

constexpr int MU_STAGES = 5;
constexpr int MU_STAGE_BYTES = A_STAGE_BYTES + HALF_B_BYTES;   // 128 rows of A, up to 128 of the tile's columns
constexpr int MU_EPI_WARPS = 8, MU_THREADS = 32 * (2 + MU_EPI_WARPS);
constexpr int MU_BOX = 32 * 32 * 2;          // of the epilogue: 32 rows x 32 columns
constexpr int MU_SLOT = 2 * MU_BOX;          // X hi and lo; as much is 32 x 32 in fp32
constexpr int MU_SLOTS = 3;          // tickets taken ahead
constexpr int MU_DEPS = MU_SLOTS + 1; // items that the loader can be ahead of the epilogue, and one
constexpr int MU_READERS = 19;       // warps of the pair that read a ticket: two loaders, the issuer, sixteen of the epilogues
constexpr int MU_PARTS = 2 * MU_EPI_WARPS;   // signals of a tile

struct MuonBarriers {
  uint64_t full[MU_STAGES], empty[MU_STAGES];
  uint64_t tmem_full[2], tmem_empty[2];
  uint64_t in_full[MU_EPI_WARPS][2];
  uint64_t item_full[MU_SLOTS], item_empty[MU_SLOTS];
  uint64_t dep[MU_DEPS];            // the loader has seen what the item depends on complete
  uint64_t drain;
  uint32_t tmem_base;
  int item[MU_SLOTS];
};
constexpr size_t MU_SMEM = 1024 + MU_STAGES * MU_STAGE_BYTES + MU_EPI_WARPS * 2 * MU_SLOT + sizeof(MuonBarriers);
static_assert(MU_SMEM <= 227 * 1024, "shared memory budget");

struct MuonItem {
  int phase, step, mat, m0, n0, nt;
  int tile, part;   // GRAM, JOIN: of the matrix's symmetric tiles; part of the reduction, strip of the tile
  int need;   // the matrix's counter when the phase before is complete
};

// Tiles of a matrix's phases and how items go through them: `sub` matrices at a time, step by step, phase by phase, matrix by matrix.
struct MuonOrder {
  int blocks, per_block, tri, app, app_cols;   // rows of 256 of a symmetric matrix, tiles across one of its blocks; tiles
  int gram, join, per_step;                    // items
  __host__ __device__ explicit MuonOrder(const MuonArgs& a) {
    const int m = a.rows < a.cols ? a.rows : a.cols;
    blocks = (m + MUON_BLOCK - 1) / MUON_BLOCK;
    per_block = MUON_BLOCK / a.nt_tri;
    tri = per_block * (blocks * (blocks + 1) / 2 - 1) + (m - (blocks - 1) * MUON_BLOCK + a.nt_tri - 1) / a.nt_tri;
    app_cols = (a.cols + a.nt_app - 1) / a.nt_app;
    app = (a.rows + 255) / 256 * app_cols;
    gram = tri * a.split;
    join = a.split > 1 ? tri * a.strips : 0;
    per_step = gram + join + tri + app;
  }
  __host__ __device__ long total(const MuonArgs& a) const { return (long)a.n * a.steps * per_step; }
  __device__ __forceinline__ MuonItem decode(const MuonArgs& a, int t) const {
    MuonItem r;
    const int full = a.sub * a.steps * per_step, g = t / full;
    t -= g * full;
    const int s = min(a.sub, a.n - g * a.sub);   // matrices of this group
    r.step = t / (s * per_step);
    t -= r.step * s * per_step;
    r.need = r.step * per_step;
    int items = gram;   // of a matrix's phase
    r.phase = MUON_GRAM;
    while (t >= s * items) {
      t -= s * items;
      r.need += items;
      ++r.phase;
      items = r.phase == MUON_JOIN ? join : r.phase == MUON_POLY ? tri : app;
    }
    r.need *= MU_PARTS;
    const int q = t / items;
    t -= q * items;
    r.mat = g * a.sub + q;
    r.part = 0;
    int i = 0;
    if (r.phase == MUON_APPLY) {
      i = t / app_cols;
      t -= i * app_cols;
      r.nt = a.nt_app;
    } else {
      if (r.phase != MUON_POLY) {
        const int parts = r.phase == MUON_GRAM ? a.split : a.strips;
        r.part = t % parts;
        t /= parts;
      }
      r.tile = t;
      for (int c = per_block; i + 1 < blocks && t >= c; c += per_block, ++i) t -= c;   // row i: (i + 1) blocks; the last one's end at m
      r.nt = a.nt_tri;
    }
    r.m0 = i * 256;
    r.n0 = t * r.nt;
    return r;
  }
};

__device__ __forceinline__ uint32_t pack_h2(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float2 unpack_h2(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2*>(&v)); }
// 16-byte chunk j of the lane's row of a box, swizzled over 64 bytes
__device__ __forceinline__ uint4* box_chunk(uint8_t* box, int lane, int j) { return reinterpret_cast<uint4*>(box + lane * 64 + ((j ^ (lane >> 1 & 3)) << 4)); }
// the same of 32 columns in fp32, over 128 bytes
__device__ __forceinline__ float4* wide_chunk(uint8_t* slot, int lane, int j) { return reinterpret_cast<float4*>(slot + lane * 128 + ((j ^ (lane & 7)) << 4)); }

// Four 16-deep MMAs of a k-block; the operands' steps (16-byte units) follow how each lies.
__device__ __forceinline__ void tc_mma4_pair_steps(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc, uint32_t accumulate,
                                                   uint32_t a_step, uint32_t b_step) {
  asm volatile(
      "{\n .reg .pred e, p;\n .reg .b64 da, db;\n .reg .b32 a, b;\n elect.sync _|e, 0xffffffff;\n setp.ne.b32 p, %5, 0;\n"
      " mov.b64 da, {%1, %3};\n mov.b64 db, {%2, %3};\n"
      " @e tcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %4, p;\n"
      " add.u32 a, %1, %6;\n add.u32 b, %2, %7;\n mov.b64 da, {a, %3};\n mov.b64 db, {b, %3};\n"
      " @e tcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %4, 1;\n"
      " add.u32 a, a, %6;\n add.u32 b, b, %7;\n mov.b64 da, {a, %3};\n mov.b64 db, {b, %3};\n"
      " @e tcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %4, 1;\n"
      " add.u32 a, a, %6;\n add.u32 b, b, %7;\n mov.b64 da, {a, %3};\n mov.b64 db, {b, %3};\n"
      " @e tcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %4, 1;\n}"
      ::"r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "r"(accumulate), "r"(a_step), "r"(b_step)
      : "memory");
}

// k-blocks [first, end) of an item's products
__device__ __forceinline__ int2 muon_blocks(const MuonArgs& a, const MuonItem& it) {
  const int K = it.phase == MUON_GRAM ? max(a.rows, a.cols) : min(a.rows, a.cols), all = (K + BK - 1) / BK;
  if (it.phase != MUON_GRAM) return make_int2(0, all);
  return make_int2((int)((long)all * it.part / a.split), (int)((long)all * (it.part + 1) / a.split));
}

// Whether the operands' k-block kb lies MN-major: X by its place in the product, a symmetric matrix beyond its stored blocks.
template <bool WIDE>
struct MuonMajors {
  int a_from, b_from;   // first k-block that does
  __device__ explicit MuonMajors(const MuonItem& it) {
    constexpr int NEVER = INT_MAX, BKS = MUON_BLOCK / BK;
    const int a_sym = it.m0 / BK + BKS, b_sym = it.n0 / MUON_BLOCK * BKS + BKS;
    if (it.phase == MUON_GRAM) {
      a_from = b_from = WIDE ? NEVER : 0;
    } else if (it.phase == MUON_POLY) {
      a_from = a_sym;
      b_from = b_sym;
    } else {
      a_from = WIDE ? a_sym : NEVER;
      b_from = WIDE ? 0 : b_sym;
    }
  }
};

// A box of the accumulator: v, 32 columns of the lane's row.
__device__ __forceinline__ void muon_box_gram(const MuonArgs::Step k, float* v, uint8_t* box, int lane) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float* x = v + 8 * j;
    *box_chunk(box, lane, j) = make_uint4(pack_h2(x[0] * k.gram_acc, x[1] * k.gram_acc), pack_h2(x[2] * k.gram_acc, x[3] * k.gram_acc),
                                          pack_h2(x[4] * k.gram_acc, x[5] * k.gram_acc), pack_h2(x[6] * k.gram_acc, x[7] * k.gram_acc));
  }
}
// (All chunks are read before the first is written: the compiler keeps reads behind writes that might meet them, a latency a chunk.)
// diag: the column of v on the lane's diagonal, or none of 0 .. 31
__device__ __forceinline__ void muon_box_poly(const MuonArgs::Step k, float* v, uint8_t* box, int lane, int diag) {
  uint4 in[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) in[j] = *box_chunk(box, lane, j);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t w[4] = {in[j].x, in[j].y, in[j].z, in[j].w};
    uint32_t o[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float2 y = unpack_h2(w[q]);
      float x0 = fmaf(y.x, k.poly_in, v[8 * j + 2 * q] * k.poly_acc), x1 = fmaf(y.y, k.poly_in, v[8 * j + 2 * q + 1] * k.poly_acc);
      if (diag == 8 * j + 2 * q) x0 += k.poly_diag;
      if (diag == 8 * j + 2 * q + 1) x1 += k.poly_diag;
      o[q] = pack_h2(x0, x1);
    }
    *box_chunk(box, lane, j) = make_uint4(o[0], o[1], o[2], o[3]);
  }
}
// X' (in v too) from X hi in box0 and, with LO, lo in box1; written back as hi and, with KEEP, lo
template <bool LO, bool HI_OUT, bool LO_OUT>
__device__ __forceinline__ void muon_box_apply(const MuonArgs::Step k, float* v, uint8_t* box0, uint8_t* box1, int lane) {
  uint4 xh[4], xl[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    xh[j] = *box_chunk(box0, lane, j);
    if (LO) xl[j] = *box_chunk(box1, lane, j);
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t wh[4] = {xh[j].x, xh[j].y, xh[j].z, xh[j].w}, wl[4] = {xl[j].x, xl[j].y, xl[j].z, xl[j].w};
    uint32_t oh[4], ol[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      float2 y = unpack_h2(wh[q]), yl = make_float2(0.f, 0.f);
      if (LO) {
        yl = unpack_h2(wl[q]);
        y.x = fmaf(yl.x, 1.f / MUON_SLO, y.x);
        y.y = fmaf(yl.y, 1.f / MUON_SLO, y.y);
      }
      float x0 = fmaf(y.x, k.app_in, v[8 * j + 2 * q] * k.app_acc), x1 = fmaf(y.y, k.app_in, v[8 * j + 2 * q + 1] * k.app_acc);
      if (LO) {
        x0 = fmaf(yl.x, k.app_rest * (1.f / MUON_SLO), x0);
        x1 = fmaf(yl.y, k.app_rest * (1.f / MUON_SLO), x1);
      }
      v[8 * j + 2 * q] = x0;
      v[8 * j + 2 * q + 1] = x1;
      if (HI_OUT) oh[q] = pack_h2(x0, x1);
      if (LO_OUT) {
        const float2 z = unpack_h2(oh[q]);
        ol[q] = pack_h2((x0 - z.x) * MUON_SLO, (x1 - z.y) * MUON_SLO);
      }
    }
    if (HI_OUT) *box_chunk(box0, lane, j) = make_uint4(oh[0], oh[1], oh[2], oh[3]);
    if (LO_OUT) *box_chunk(box1, lane, j) = make_uint4(ol[0], ol[1], ol[2], ol[3]);
  }
}
// The last step's X' in v: bf16, or the weights' update, into box0; W is in box1, or with `lo` (no late step) still in memory
__device__ __forceinline__ void muon_box_out(const MuonArgs& a, float* v, uint8_t* box0, uint8_t* box1, int lane, bool lo, int mat, int r, int c0) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    float* x = v + 8 * j;
    if (a.w_ptr) {
      uint4 w = make_uint4(0, 0, 0, 0);
      const int c = c0 + 8 * j;
      if (!lo) w = *box_chunk(box1, lane, j);
      else if (r < a.rows && c < a.cols) w = *reinterpret_cast<const uint4*>(a.w_ptr + ((size_t)mat * a.rows + r) * a.cols + c);
      const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        x[2 * q] = fmaf(a.keep, bf16lo(ww[q]), -a.rate * x[2 * q]);
        x[2 * q + 1] = fmaf(a.keep, bf16hi(ww[q]), -a.rate * x[2 * q + 1]);
      }
    }
    *box_chunk(box0, lane, j) = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
  }
}
// The same for rows that are no whole vectors: X' in fp32 through the slot, so that a row's elements are next to one another when they are written
__device__ __forceinline__ void muon_rows_out(const MuonArgs& a, const MuonArgs::Step& k, float* v, uint8_t* slot, bool lo, int lane, int mat, int r0, int c0) {
  if (lo) muon_box_apply<true, false, false>(k, v, slot, slot + MU_BOX, lane);
  else muon_box_apply<false, false, false>(k, v, slot, slot + MU_BOX, lane);
  __syncwarp();   // X has been read
#pragma unroll
  for (int j = 0; j < 8; ++j) *wide_chunk(slot, lane, j) = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
  __syncwarp();
  const int c = c0 + lane;
#pragma unroll 4
  for (int i = 0; i < 32; ++i)
    if (r0 + i < a.rows && c < a.cols) {
      float x = reinterpret_cast<const float*>(wide_chunk(slot, i, lane >> 2))[lane & 3];
      const size_t at = ((size_t)mat * a.rows + r0 + i) * a.cols + c;
      if (a.w_ptr) x = fmaf(a.keep, __uint_as_float((uint32_t)a.w_ptr[at] << 16), -a.rate * x);
      a.out_ptr[at] = (uint16_t)pack_bf16x2(x, 0.f);
    }
}

// JOIN: a strip of a tile's rows from the tile's parts, in their order; w: the warp of the pair.  Read past L1, which may hold an earlier
// step's.
__device__ __forceinline__ void muon_join(const MuonArgs& a, const MuonItem& it, int tri, int w, int lane) {
  const int m = min(a.rows, a.cols), rows = 256 / a.strips, quads = it.nt / 4, row0 = it.part * rows;
  const float scale = a.step[0].gram_acc;
  const size_t step = (size_t)256 * it.nt / 4;
  for (int u = w * 32 + lane; u < rows * quads; u += MU_PARTS * 32) {
    const int row = row0 + u / quads, c = u % quads * 4, r = it.m0 + row;
    if (r >= m) break;
    const float4* p = reinterpret_cast<const float4*>(a.part_ptr + (((size_t)it.mat * tri + it.tile) * a.split * 256 + row) * it.nt + c);
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i = 0; i < a.split; i += 16) {   // all loads of a turn under way together
      float4 x[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) x[j] = i + j < a.split ? __ldcg(p + (i + j) * step) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int j = 0; j < 16; ++j) { s.x += x[j].x; s.y += x[j].y; s.z += x[j].z; s.w += x[j].w; }
    }
    if (it.n0 + c < a.lda)   // columns behind m are room
      *reinterpret_cast<uint2*>(a.a_ptr + ((size_t)it.mat * m + r) * a.lda + it.n0 + c) =
          make_uint2(pack_h2(s.x * scale, s.y * scale), pack_h2(s.z * scale, s.w * scale));
  }
}

// A role's place in the ring of tickets.  The slot of an item is free for another once all have read it -- where a phase has few items
// (SPLIT), once the epilogue is done with it: a pair that took its next item early would keep it from an idle one.
struct MuonTickets {
  uint32_t slot = 0, par = 0;
  // all lanes: the next item; -1 after a failed wait
  __device__ __forceinline__ int next(MuonBarriers* bars, int slots, const WaitCtl& wc, uint32_t sleep_ns, bool keep = false) {
    int t = -1;
    if ((threadIdx.x & 31) == 0) {
      if (mbar_wait_cluster(&bars->item_full[slot], par, wc, SITE_DEP, 0, sleep_ns)) t = *reinterpret_cast<volatile int*>(&bars->item[slot]);
      if (!keep) free(bars, slot);
    }
    if (++slot == (uint32_t)slots) { slot = 0; par ^= 1; }
    return uniform(t);
  }
  __device__ __forceinline__ static void free(MuonBarriers* bars, uint32_t slot) {   // one lane
    mbar_arrive_cluster_addr(map_to_rank(smem_u32(&bars->item_empty[slot]), 1));   // where the tickets are taken
  }
};

// SPLIT: GRAM's reduction is (a.split > 1); VEC: a.vec.  Of their own, so that the usual kernel's epilogue keeps its registers.
template <bool WIDE, bool SPLIT, bool VEC>
__global__ void __launch_bounds__(MU_THREADS, 1) muon_products_kernel(const __grid_constant__ MuonArgs a) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* boxes = smem + MU_STAGES * MU_STAGE_BYTES;
  MuonBarriers* bars = reinterpret_cast<MuonBarriers*>(boxes + MU_EPI_WARPS * 2 * MU_SLOT);

  const int warp = warp_index(), lane = threadIdx.x & 31;
  const int rank = (int)cluster_ctarank();
  const WaitCtl wc{a.status, a.budget_ns};

  if (threadIdx.x == 0) {
    for (int s = 0; s < MU_STAGES; ++s) {
      mbar_init(&bars->full[s], 1);
      mbar_init(&bars->empty[s], 1);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(&bars->tmem_full[s], 1);
      mbar_init(&bars->tmem_empty[s], MU_PARTS);
    }
    for (int w = 0; w < 2 * MU_EPI_WARPS; ++w) mbar_init(&bars->in_full[w >> 1][w & 1], 1);
    for (int s = 0; s < MU_SLOTS; ++s) {
      mbar_init(&bars->item_full[s], 1);
      mbar_init(&bars->item_empty[s], MU_READERS);
    }
    for (int s = 0; s < MU_DEPS; ++s) mbar_init(&bars->dep[s], 1);
    mbar_init(&bars->drain, 1);
    mbar_fence_init();
    fence_proxy_async();
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

  const MuonOrder order(a);
  const int total = (int)order.total(a), slots = SPLIT ? 1 : MU_SLOTS;
  if (warp == 0) {
    MuonTickets tk;
    uint32_t s = 0, par = (1u << MU_STAGES) - 1, dep = 0;
    for (bool ok = true; ok;) {
      const int t = tk.next(bars, slots, wc, 20);
      if (t < 0 || t >= total) break;
      const MuonItem it = order.decode(a, t);
      const MuonMajors<WIDE> mj(it);
      const int half = it.nt / 2, mat = uniform(it.mat), cur = it.step & 1;
      const int m0 = uniform(it.m0 + rank * 128), n0 = uniform(it.n0 + rank * half);
      const int2 blocks = muon_blocks(a, it);
      const int kb0 = uniform(blocks.x), kb1 = uniform(blocks.y);
      // K-major and MN-major maps of both operands
      const CUtensorMap *a_k = &a.a128, *a_mn = &a.a64, *b_k = &a.a_part, *b_mn = &a.a64;
      if (it.phase == MUON_GRAM) {
        a_k = &a.x128[cur];
        b_k = &a.x_part[cur];
        a_mn = b_mn = &a.x64[cur];
      } else if (it.phase == MUON_APPLY) {
        a_k = WIDE ? &a.b128 : &a.x128[cur];
        a_mn = &a.b64;
        b_k = &a.b_part;
        b_mn = WIDE ? &a.x64[cur] : &a.b64;
      }
      int up = 1;
      if (it.need && lane == 0) up = counter_wait(a.ctr + mat, it.need, wc, t, 256) ? 1 : 0;
      if (!uniform(up)) break;
      fence_proxy_async_global();   // what the counter announces was written by other CTAs' stores
      if (lane == 0) mbar_arrive_cta(&bars->dep[dep]);
      if (++dep == MU_DEPS) dep = 0;
      if (SPLIT && it.phase == MUON_JOIN) continue;
      const int b_boxes = (half + 63) / 64;
      for (int kb = kb0; kb < kb1; ++kb) {
        if (!mbar_wait_warp(&bars->empty[s], (par >> s) & 1, wc, SITE_EMPTY, t, 20)) { ok = false; break; }
        uint8_t* st = smem + s * MU_STAGE_BYTES;
        const bool amn = kb >= mj.a_from, bmn = kb >= mj.b_from;
        if (rank == 0) mbar_expect_tx_elect(&bars->full[s], 2 * (A_STAGE_BYTES + (bmn ? b_boxes * MN_BOX_BYTES : half * BK * 2)));
        if (amn) {
          tma_load_3d_pair(st, a_mn, m0, kb * BK, mat, &bars->full[s]);
          tma_load_3d_pair(st + MN_BOX_BYTES, a_mn, m0 + 64, kb * BK, mat, &bars->full[s]);
        } else {
          tma_load_3d_pair(st, a_k, kb * BK, m0, mat, &bars->full[s]);
        }
        uint8_t* sb = st + A_STAGE_BYTES;
        if (bmn) {
          tma_load_3d_pair(sb, b_mn, n0, kb * BK, mat, &bars->full[s]);
          if (b_boxes > 1) tma_load_3d_pair(sb + MN_BOX_BYTES, b_mn, n0 + 64, kb * BK, mat, &bars->full[s]);
        } else {
          tma_load_3d_pair(sb, b_k, kb * BK, n0, mat, &bars->full[s]);
        }
        par ^= 1u << s;
        if (++s == MU_STAGES) s = 0;
      }
    }
  } else if (warp == 1 && rank == 0) {
    MuonTickets tk;
    const uint32_t at0 = smem_u32(smem), bt0 = smem_u32(smem + A_STAGE_BYTES);
    const uint32_t a_lo0[2] = {smem_desc_lo(at0, 16), smem_desc_lo(at0, MN_BOX_BYTES)}, b_lo0[2] = {smem_desc_lo(bt0, 16), smem_desc_lo(bt0, MN_BOX_BYTES)};
    uint32_t s = 0, par = 0, acc = 0, acc_par = 3;
    bool ok = true;
    for (;;) {
      const int t = tk.next(bars, slots, wc, 0);
      if (t < 0) ok = false;
      if (t < 0 || t >= total) break;
      const MuonItem it = order.decode(a, t);
      if (SPLIT && it.phase == MUON_JOIN) continue;
      const MuonMajors<WIDE> mj(it);
      const int2 blocks = muon_blocks(a, it);
      const int kb0 = uniform(blocks.x), kb1 = uniform(blocks.y);
      const uint32_t idesc = uniform(make_idesc_f16(256, it.nt, 0, 0));
      const int a_from = uniform(mj.a_from), b_from = uniform(mj.b_from);
      if (!mbar_wait_warp(&bars->tmem_empty[acc], (acc_par >> acc) & 1, wc, SITE_TMEM_EMPTY, t)) { ok = false; break; }
      acc_par ^= 1u << acc;
      tc_fence_after_sync();
      const uint32_t d_tmem = uniform(tmem_base + acc * 256);
      for (int kb = kb0; kb < kb1; ++kb) {
        if (!mbar_wait_warp(&bars->full[s], (par >> s) & 1, wc, SITE_FULL, t)) { ok = false; break; }
        par ^= 1u << s;
        tc_fence_after_sync();
        const uint32_t at = s * (MU_STAGE_BYTES >> 4), amn = kb >= a_from, bmn = kb >= b_from;
        tc_mma4_pair_steps(d_tmem, (amn ? a_lo0[1] : a_lo0[0]) + at, (bmn ? b_lo0[1] : b_lo0[0]) + at, smem_desc_hi(1024),
                           idesc | amn << 15 | bmn << 16, kb != kb0, amn ? 2048 >> 4 : 2, bmn ? 2048 >> 4 : 2);
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
  } else if (warp == 1) {
    if (lane == 0) {   // the odd CTA's
      uint32_t slot = 0, par = 1;
      for (int t = 0; t < total;) {
        if (!mbar_wait_cluster(&bars->item_empty[slot], par, wc, SITE_EMPTY, t, 50)) break;
        t = atomicAdd(a.ctr + a.n, 1);
        const uint32_t at = smem_u32(&bars->item[slot]), full = smem_u32(&bars->item_full[slot]);
#pragma unroll
        for (uint32_t r = 0; r < 2; ++r) {
          asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(map_to_rank(at, r)), "r"(t) : "memory");
          mbar_arrive_cluster_addr(map_to_rank(full, r));
        }
        if (++slot == (uint32_t)slots) { slot = 0; par ^= 1; }
      }
    }
  } else {
    MuonTickets tk;
    const int ew = warp - 2, quad = warp & 3;
    uint8_t* slots_at = boxes + ew * 2 * MU_SLOT;
    uint32_t sl = 0, in_par = 0;   // slot of the next box, parity of either slot's loads
    uint32_t acc = 0, full_par = 0, dep = 0, dep_par = 0;
    for (bool ok = true; ok;) {
      const int t = tk.next(bars, slots, wc, 100, SPLIT);
      if (t < 0 || t >= total) break;   // (a kept slot is the only one, and nobody waits for it any more)
      const MuonItem it = order.decode(a, t);
      const MuonArgs::Step k = a.step[it.step];   // (a copy: by reference the factors were read again for every chunk, 1.4 us a box)
      const int m = min(a.rows, a.cols), cur = it.step & 1;
      const int M = it.phase == MUON_APPLY ? a.rows : m, N = it.phase == MUON_APPLY ? a.cols : m;
      const bool last = it.phase == MUON_APPLY && it.step + 1 == a.steps;
      const bool lo = it.phase == MUON_APPLY && it.step < a.late, lo_out = it.phase == MUON_APPLY && !last && it.step + 1 < a.late;
      const bool upd = last && !lo && VEC && a.w_ptr;   // W comes with X
      const int r0 = it.m0 + rank * 128 + quad * 32;
      // the loader polls the counter for the CTA
      if (!mbar_wait_warp(&bars->dep[dep], dep_par, wc, SITE_DEP, t, 50)) break;
      if (++dep == MU_DEPS) { dep = 0; dep_par ^= 1; }
      if (SPLIT && it.phase == MUON_JOIN) {
        muon_join(a, it, order.tri, rank * MU_EPI_WARPS + ew, lane);
        fence_proxy_async_global();   // every lane's stores, for the loads to come
        __syncwarp();
        if (lane == 0) {
          if (SPLIT) MuonTickets::free(bars, 0);
          counter_signal(a.ctr + it.mat, 1);
        }
        continue;
      }
      const bool parts = SPLIT && it.phase == MUON_GRAM;
      const bool in = it.phase != MUON_GRAM;   // the box needs A or X
      // this warp's boxes: every other one of its rows, those that lie in the product
      const int b0 = (ew >> 2) * 32, left = min(it.nt, N - it.n0) - b0;
      const int n_boxes = r0 < M && left > 0 ? (left + 63) / 64 : 0;
      auto load = [&](int u, uint32_t s) {   // one lane
        uint8_t* to = slots_at + s * MU_SLOT;
        const int c = it.n0 + b0 + 64 * u;
        fence_proxy_async_global();
        mbar_expect_tx(&bars->in_full[ew][s], lo || upd ? 2 * MU_BOX : MU_BOX);
        tma_load_3d_thread(to, it.phase == MUON_POLY ? &a.abox : &a.xhi[cur], c, r0, it.mat, &bars->in_full[ew][s]);
        if (lo) tma_load_3d_thread(to + MU_BOX, &a.xlo[cur], c, r0, it.mat, &bars->in_full[ew][s]);
        else if (upd) tma_load_3d_thread(to + MU_BOX, &a.w, c, r0, a.z0 + it.mat, &bars->in_full[ew][s]);
      };
      __syncwarp();   // every lane has read the slots
      if (in && n_boxes && lane == 0) {
        tma_store_wait_read();
        load(0, sl);
      }
      bool up = false;   // the accumulator has been seen complete
      for (int u = 0; u < n_boxes; ++u, sl ^= 1) {
        uint8_t *box0 = slots_at + sl * MU_SLOT, *box1 = box0 + MU_BOX;
        const int b = b0 + 64 * u, c0 = it.n0 + b;
        __syncwarp();
        if (lane == 0) {
          if (!in) {
            tma_store_wait_read_but_one();   // this slot's, two boxes ago
          } else if (u + 1 < n_boxes) {      // the next box's loads beside this one
            tma_store_wait_read();
            load(u + 1, sl ^ 1);
          }
        }
        __syncwarp();
        if (!up) {
          if (!mbar_wait_warp(&bars->tmem_full[acc], (full_par >> acc) & 1, wc, SITE_TMEM_FULL, t, 100)) ok = false;
          tc_fence_after_sync();
          up = true;
        }
        if (in) {
          if (!mbar_wait_warp(&bars->in_full[ew][sl], (in_par >> sl) & 1, wc, SITE_FULL, t)) ok = false;
          in_par ^= 1u << sl;
        }
        if (!ok) break;
        float v[32];
        const uint32_t tcol = tmem_base + acc * 256 + b + (static_cast<uint32_t>(quad * 32) << 16);
        tmem_ld16(tcol, v);
        tmem_ld16(tcol + 16, v + 16);
        tmem_ld_wait();
        if (!VEC && last) {
          muon_rows_out(a, k, v, box0, lo, lane, it.mat, r0, c0);
          staging_release();   // the slot was written through; what comes into it next is loaded by TMA
          continue;
        }
        if (parts) {
#pragma unroll
          for (int j = 0; j < 8; ++j) *wide_chunk(box0, lane, j) = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
        } else if (it.phase == MUON_GRAM) {
          muon_box_gram(k, v, box0, lane);
        } else if (it.phase == MUON_POLY) {
          muon_box_poly(k, v, box0, lane, r0 + lane - c0);
        } else if (!last) {
          if (lo_out) muon_box_apply<true, true, true>(k, v, box0, box1, lane);
          else if (lo) muon_box_apply<true, true, false>(k, v, box0, box1, lane);
          else muon_box_apply<false, true, false>(k, v, box0, box1, lane);
        } else if (VEC) {
          if (lo) muon_box_apply<true, false, false>(k, v, box0, box1, lane);
          else muon_box_apply<false, false, false>(k, v, box0, box1, lane);
          muon_box_out(a, v, box0, box1, lane, lo, it.mat, r0 + lane, c0);
        }
        staging_release();
        if (lane == 0 && parts) {
          tma_store_2d(&a.part, b, ((it.mat * order.tri + it.tile) * a.split + it.part) * 256 + rank * 128 + quad * 32, box0);
          tma_store_commit();
        } else if (lane == 0) {
          const CUtensorMap* o = it.phase == MUON_GRAM ? &a.abox : it.phase == MUON_POLY ? &a.bbox : last ? &a.out : &a.xhi[cur ^ 1];
          tma_store_3d(o, c0, r0, last ? a.z0 + it.mat : it.mat, box0);
          if (lo_out) tma_store_3d(&a.xlo[cur ^ 1], c0, r0, it.mat, box1);
          tma_store_commit();
        }
      }
      if (!up && ok && !mbar_wait_warp(&bars->tmem_full[acc], (full_par >> acc) & 1, wc, SITE_TMEM_FULL, t, 100)) ok = false;
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive_leader(&bars->tmem_empty[acc]);
        if (SPLIT) MuonTickets::free(bars, 0);
        if (!last && ok) {   // this warp's part of the tile is stored
          tma_store_wait_all();
          fence_proxy_async_global();
          counter_signal(a.ctr + it.mat, 1);
        }
      }
      full_par ^= 1u << acc;
      acc ^= 1;
    }
    if (lane == 0) tma_store_wait_all();
  }

  // ---------------------------------------------------------------- teardown
  __syncwarp();
  if (*reinterpret_cast<volatile int*>(&a.status->abort)) __nanosleep(200000);
  tc_fence_before_sync();
  __syncthreads();
  cluster_sync_all();
  if (warp == 1) {
    tc_fence_after_sync();
    tmem_dealloc_pair(tmem_base, TMEM_COLS);
  }
}

template <bool WIDE, bool SPLIT, bool VEC>
static cudaError_t launch_one(const MuonArgs& a, int sms, cudaStream_t s) {
  static PairLaunchState st;
  return launch_on_pairs(st, muon_products_kernel<WIDE, SPLIT, VEC>, a, MU_THREADS, MU_SMEM, sms, s, true);
}
template <bool WIDE>
static cudaError_t launch_of(const MuonArgs& a, int sms, cudaStream_t s) {
  if (a.split > 1) return a.vec ? launch_one<WIDE, true, true>(a, sms, s) : launch_one<WIDE, true, false>(a, sms, s);
  return a.vec ? launch_one<WIDE, false, true>(a, sms, s) : launch_one<WIDE, false, false>(a, sms, s);
}
cudaError_t launch_muon_products(bool wide, const MuonArgs& a, int num_sms, cudaStream_t s) {
  const long tiles = MuonOrder(a).total(a);
  const int sms = (int)(2 * tiles < num_sms ? 2 * tiles : num_sms);
  return wide ? launch_of<true>(a, sms, s) : launch_of<false>(a, sms, s);
}

}  // namespace moe
