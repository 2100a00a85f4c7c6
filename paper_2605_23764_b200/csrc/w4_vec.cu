// The layer's expert products over 4-bit weights for experts with a few rows: token generation.
//
//   h[i] = sum_groups s_g sum_k (q - z) x[i][k];   A = w silu(h_gate) h_up;   Y = the same over A;   out[t] = sum_j Y of its slots
//
// What bounds it: the weights' bytes are the floor, the instructions that widen and multiply them what it takes.  33 experts of 7168 x
// 2048, groups of 128: 8 tokens that hit 30 of them 155 to 160 us a call, calls back to back, 4.3 TB/s of codes and scales (an instruction
// a code to widen them on a pipe of half rate, 61 % busy, a product of 16 x 8 x 16 for 256 codes and one more for the sums of x).  One
// token of eight experts of 2048 x 1408: 21 to 23 us, of which reading is 5: three launches, each of the latencies of its ids, first units
// and rows of x.
//
// Every warp streams its share of the units (2 KB) through a ring of its own in shared memory (loads kept in registers instead did not
// overlap: a unit then cost a memory latency, 2.7 TB/s), widens the codes to bf16 16 + q -- a mask and an exponent -- and multiplies 32
// rows by up to 8 rows of x at a time (mma.m16n8k16, which a matrix-vector product needs as a dot-product unit, not for its rate; 32
// rows because the operand rows of x are read from shared memory once for all of them).  A third operand of ones gives the sums of x, of
// which 16 + z is taken off:
//   sum (q - z) x = sum (16 + q) x - (16 + z) sum x,
// exact products, fp32 sums, whose rounding is 2^-23 of some 24 sum |x| a step.  (Of 128 + q it was of 136 sum |x|, and showed in the
// result where x has much in common and most codes are zero points: an error of 3.3e-3 in the norm instead of 2.4e-3.)  A subtraction for
// each pair of codes instead kept the pipe that multiplies at 40 %.  Sums of x made once a segment and given to the chains as their
// first accumulator were no faster.  A group's sum is scaled in fp32: the only rounding to fewer bits on the way is that of A to bf16,
// which the second product takes as operand (as the bf16 layer does).
//
// Split.  Blocks take consecutive row tiles of the hit experts, one block an SM; inside a block the warps share the units (32 rows x 128
// columns) evenly, whatever the tile boundaries: a row tile that several warps have a piece of is put together from shared
// memory in the warps' order.  So few experts and long reductions keep all warps at work, and results do not depend on timing.  Sixteen
// warps: twelve took 7 % longer for the 8 tokens above.  Five slots a ring, or four for twelve warps, were no faster.
#include "launch_pairs.cuh"
#include "topk.cuh"
#include "w4.cuh"

namespace moe {

namespace {

constexpr int VEC_WARPS = 16, VEC_THREADS = 32 * VEC_WARPS;
constexpr int VEC_ROWS = 8;          // rows of x that a pass over an expert's weights takes
constexpr int VEC_SEG_TILES = 16;    // row tiles between two joins
static_assert(VEC_SEG_TILES <= 32, "a lane for each pass that a segment may touch");
constexpr int VEC_DEPTH = 3;         // slots of a warp's ring: two units in flight, 66 KB an SM or more
constexpr int VEC_SMEM = 221 * 1024;
constexpr int VEC_PIECE_BYTES = W4_TILE_ROWS * VEC_ROWS * 4;   // sums of a row tile
constexpr int VEC_ROWS_MOST = 64;    // staged rows, at most
static_assert((1024 + 64) < 0x8000, "an expert and a bit");

__host__ __device__ constexpr int vec_ld(int KU) { return KU * W4_UNIT_K * 2 + 16; }   // bytes from row to row: ldmatrix rows in different banks
__host__ __device__ constexpr int vec_slot(int ng, bool asym) { return W4_UNIT_BYTES + 64 * ng + (asym ? 32 * ng : 0); }   // codes, scales, zero points
__host__ __device__ constexpr size_t vec_fixed_smem(int ng, bool asym) {
  return (size_t)VEC_WARPS * VEC_DEPTH * vec_slot(ng, asym) + (size_t)(VEC_SEG_TILES + VEC_WARPS) * VEC_PIECE_BYTES;
}

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void ldmatrix4(uint32_t addr, uint32_t* r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// the first product of a chain: no accumulator goes in
__device__ __forceinline__ void mma16816_first(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
      : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t lds32(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

static_assert(VEC_THREADS >= W4_VEC_SLOTS, "a slot for each thread");

}  // namespace

// NG groups of 128 / NG columns to a unit.
template <bool ASYM, int NG>
__global__ void __launch_bounds__(VEC_THREADS, 1) w4_vec_kernel(const W4VecArgs a) {
  extern __shared__ __align__(16) uint8_t vsm[];
  __shared__ int slot_e[W4_VEC_SLOTS];
  __shared__ float slot_w[W4_VEC_SLOTS];
  // rows in the order of their experts: slot, token, expert (its top bit: a pass begins); passes over an expert's weights: first row, expert
  __shared__ uint16_t row_slot[W4_VEC_SLOTS], row_t[W4_VEC_SLOTS], row_e[W4_VEC_SLOTS], pass_row[W4_VEC_SLOTS + 1], pass_e[W4_VEC_SLOTS];
  __shared__ int pass_count;
  __shared__ uint8_t tile_from[VEC_SEG_TILES], tile_to[VEC_SEG_TILES];   // warps that have the first and the last piece of a row tile
  constexpr int SLOT = vec_slot(NG, ASYM), PIECE = VEC_PIECE_BYTES / 4, STARTS = 0x8000;
  float* const acc_s = reinterpret_cast<float*>(vsm + VEC_WARPS * VEC_DEPTH * SLOT);   // [VEC_SEG_TILES][32][8]
  float* const head_s = acc_s + VEC_SEG_TILES * PIECE;                                 // [VEC_WARPS][32][8]
  const int ld = vec_ld(a.KU);
  uint8_t* const xs = vsm + vec_fixed_smem(NG, ASYM);                                  // [rows_cap][ld]
  const int warp = warp_index(), lane = threadIdx.x & 31, tid = threadIdx.x, g = lane >> 2, c = lane & 3;

  // The first product waits for what is in front of it here; the second one's ids were complete before the first started,
  // so it waits only where it reads what the first product wrote.
  if (!a.down) {
    pdl_wait();
    pdl_trigger();
  }
  // ---- the slots in order of their experts, by every block for itself: a slot's place is the number of slots in front of it, which
  // 512 / n threads count.  (Scans over the experts, searches and the rows of a segment by one warp took 9000 of 28000 clocks of a call
  // for one token.)
  const int n = a.T * a.kp;
  if (tid < n) {
    const int t = tid / a.kp, j = tid - t * a.kp;
    int e = a.E + j - a.k;
    float w = 1.f;
    if (j < a.k) {
      e = __ldcg(a.ids + t * a.k + j);
      if (!a.down) w = __ldcg(a.w + t * a.k + j);
      if (e < 0 || e >= a.E) {
        e = INT_MAX;   // behind all others
        if (blockIdx.x == 0 && !a.down) note(a.status, /*MOE_ERR_BAD_EXPERT_ID*/ 1, tid);
      }
    }
    slot_e[tid] = e;
    slot_w[tid] = w;
  }
  __syncthreads();
  int rows;   // slots that name an expert
  {
    const int lg = n > 256 ? 0 : min(5, 31 - __clz(VEC_THREADS / n)), i = tid >> lg, part = tid & ((1 << lg) - 1);
    const int e = i < n ? slot_e[i] : INT_MAX;
    int less = 0, rank = 0;
    if (e < INT_MAX)
      for (int j = part; j < n; j += 1 << lg) {
        const int o = slot_e[j];
        less += o < e;
        rank += o == e && j < i;
      }
    for (int off = 1 << lg >> 1; off; off >>= 1) {
      less += __shfl_xor_sync(0xffffffffu, less, off);
      rank += __shfl_xor_sync(0xffffffffu, rank, off);
    }
    const bool mine = i < n && part == 0, there = mine && e < INT_MAX;
    const int at = less + rank;
    if (there) {
      row_slot[at] = (uint16_t)i;
      row_t[at] = (uint16_t)(i / a.kp);
      row_e[at] = (uint16_t)(e | (rank % a.group_rows ? 0 : STARTS));
    }
    if (mine && blockIdx.x == 0 && !a.down) a.prow_of[i] = there ? at : -1;
    rows = __syncthreads_count(there);
  }
  if (warp * 32 < rows) {
    int before = 0;
    uint32_t starts = 0;
    for (int q = 0; q <= warp; ++q) {
      before += __popc(starts);
      starts = __ballot_sync(0xffffffffu, q * 32 + lane < rows && (row_e[q * 32 + lane] & STARTS));
    }
    const int pass = before + __popc(starts & ((1u << lane) - 1u));
    if (starts >> lane & 1) {
      pass_row[pass] = (uint16_t)tid;
      pass_e[pass] = row_e[tid] & (STARTS - 1);
    }
    if (tid == rows - 1) {
      pass_count = before + __popc(starts);
      pass_row[before + __popc(starts)] = (uint16_t)rows;
    }
  }
  __syncthreads();
  const int passes = rows ? pass_count : 0;

  const int tiles = passes * a.RT, share = tiles / (int)gridDim.x, extra = tiles - share * (int)gridDim.x;
  const int t1 = share * ((int)blockIdx.x + 1) + min((int)blockIdx.x + 1, extra);
  // The segment that begins at tile `from`: as many tiles as have room, rows staged once.  Every warp works it out.
  struct Segment { int from, tiles, pass0, rt0, row0, rows; };
  auto plan = [&](int from) {
    Segment sg{from, 0, 0, 0, 0, 0};
    if (from >= t1) return sg;
    sg.pass0 = from / a.RT;
    sg.rt0 = from - sg.pass0 * a.RT;
    sg.row0 = pass_row[sg.pass0];
    const int most = min(t1, from + VEC_SEG_TILES), p = sg.pass0 + lane;
    const bool in = p < passes && p * a.RT < most;
    const int m = __popc(__ballot_sync(0xffffffffu, in && pass_row[in ? p + 1 : 0] - sg.row0 <= a.rows_cap));   // the first m passes
    sg.tiles = min(most, (sg.pass0 + m) * a.RT) - from;
    sg.rows = pass_row[sg.pass0 + m] - sg.row0;
    return sg;
  };

  // ---- a warp's units of a segment
  int units = 0, u0 = 0, u1 = 0, tile = 0, ku = 0, pass = 0, rt = 0;   // of the segment; row tile of it, unit of that; pass, row tile of the expert
  // The stream: from unit to unit of a row tile the addresses grow by four units.
  const uint8_t *f_codes = nullptr, *f_scales = nullptr, *f_zeros = nullptr;
  int f_pass = 0, f_rt = 0, f_left = 0, f_run = 0;   // units to fetch, of them in this row tile
  auto seek = [&](int from) {   // lane l copies 16 bytes at 16 l
    const int64_t unit = (int64_t)pass_e[f_pass] * a.RTS * a.KU + w4_unit(f_rt, from, a.KU);
    f_codes = reinterpret_cast<const uint8_t*>(a.codes) + unit * W4_UNIT_BYTES + lane * 16;
    f_scales = reinterpret_cast<const uint8_t*>(a.scales) + unit * (64 * NG) + lane * 16;
    if (ASYM) f_zeros = reinterpret_cast<const uint8_t*>(a.zeros) + unit * (32 * NG) + lane * 16;
    f_run = min(f_left, a.KU - from);
  };
  const uint32_t ring = smem_u32(vsm) + warp * VEC_DEPTH * SLOT, ring_end = ring + VEC_DEPTH * SLOT;
  auto fetch = [&](uint32_t slot) {
    if (f_run == 0 && f_left > 0) {
      if (++f_rt == a.RT) {
        f_rt = 0;
        ++f_pass;
      }
      seek(0);
    }
    if (f_run > 0) {
      --f_run;
      --f_left;
      const uint32_t to = slot + lane * 16;
#pragma unroll
      for (int h = 0; h < 4; ++h) cp_async16(to + 512 * h, f_codes + 512 * h);
      if (lane < 4 * NG) cp_async16(to + W4_UNIT_BYTES, f_scales);
      if (ASYM && lane < 2 * NG) cp_async16(to + W4_UNIT_BYTES + 64 * NG, f_zeros);
      f_codes += 4 * W4_UNIT_BYTES;
      f_scales += 4 * 64 * NG;
      if (ASYM) f_zeros += 4 * 32 * NG;
    }
    cp_async_commit();
  };
  auto begin = [&](const Segment& sg) {
    units = sg.tiles * a.KU;
    u0 = units * warp / VEC_WARPS;
    u1 = units * (warp + 1) / VEC_WARPS;
    tile = u0 / a.KU;
    ku = u0 - tile * a.KU;
    const int over = (sg.rt0 + tile) / a.RT;
    pass = sg.pass0 + over;
    rt = sg.rt0 + tile - over * a.RT;
    f_pass = pass;
    f_rt = rt;
    f_left = u1 - u0;
    f_run = 0;
    if (u0 < u1) seek(ku);
#pragma unroll
    for (int i = 0; i < VEC_DEPTH - 1; ++i) fetch(ring + i * SLOT);
  };
  // Rows of x, zeros behind K.
  auto stage = [&](const Segment& sg) {
    const int pieces = a.KU * (W4_UNIT_K / 8), full = a.K >> 3;
    const int row_step = VEC_THREADS / pieces, step = VEC_THREADS - row_step * pieces;
    int row = tid / pieces, v = tid - row * pieces;
    while (row < sg.rows) {
      const int at = sg.row0 + row;
      uint8_t* dst = xs + (size_t)row * ld + v * 16;
      if (v < full) cp_async16(smem_u32(dst), a.in + (size_t)(a.down ? at : row_t[at]) * a.in_ld + v * 8);
      else *reinterpret_cast<uint4*>(dst) = make_uint4(0, 0, 0, 0);
      row += row_step;
      v += step;
      if (v >= pieces) { v -= pieces; ++row; }
    }
    cp_async_commit();
  };

  Segment sg = plan(share * (int)blockIdx.x + min((int)blockIdx.x, extra));
  if (sg.tiles > 0) begin(sg);
  if (a.down) {
    pdl_wait();
    pdl_trigger();
  }
  if (sg.tiles > 0) stage(sg);
  while (sg.tiles > 0) {
    cp_async_wait<0>();   // (the first units as well)
    __syncthreads();

    // ---- the products
    float acc[2][4] = {};
    bool began = ku == 0;   // this warp has the tile from its first unit on
    uint32_t x_row = 0;
    auto enter_pass = [&]() {   // operand rows: lane l gives row l % 8 of matrix l / 8; rows that are not there are computed and dropped
      const int first = pass_row[pass], r = min(lane & 7, pass_row[pass + 1] - first - 1);
      x_row = smem_u32(xs + (size_t)(first - sg.row0 + r) * ld) + (lane >> 3) * 16;
    };
    if (u0 < u1) enter_pass();
    uint32_t rd = ring, wr = ring + (VEC_DEPTH - 1) * SLOT;
    for (int u = u0; u < u1;) {
      // the warp's piece of a row tile
      const int n = min(a.KU - ku, u1 - u);
      uint32_t x_addr = x_row + ku * (W4_UNIT_K * 2);
#pragma unroll 1
      for (int i = 0; i < n; ++i) {
        fetch(wr);
        cp_async_wait<VEC_DEPTH - 1>();
        __syncwarp();   // the lanes' copies of scales are everybody's
        uint32_t b[16];
#pragma unroll
        for (int h = 0; h < 4; ++h) ldmatrix4(x_addr + 64 * h, b + 4 * h);
        x_addr += W4_UNIT_K * 2;
        // rows {g, g + 8} and {g + 16, g + 24} of each group
        uint32_t sc[2][NG], zp[ASYM ? NG : 1];
        {
          const uint32_t at = rd + W4_UNIT_BYTES + g * (8 * NG);
          if constexpr (NG == 1) {
            const uint2 v = lds64(at);
            sc[0][0] = v.x; sc[1][0] = v.y;
          } else {
#pragma unroll
            for (int h = 0; h < NG; h += 2) {
              const uint4 v = lds128(at + 8 * h);
              sc[0][h] = v.x; sc[1][h] = v.y; sc[0][h + 1] = v.z; sc[1][h + 1] = v.w;
            }
          }
          if constexpr (ASYM) {
            const uint32_t zat = rd + W4_UNIT_BYTES + 64 * NG + g * (4 * NG);
            if constexpr (NG == 1) {
              zp[0] = lds32(zat);
            } else if constexpr (NG == 2) {
              const uint2 v = lds64(zat);
              zp[0] = v.x; zp[1] = v.y;
            } else {
              const uint4 v = lds128(zat);
              zp[0] = v.x; zp[1] = v.y; zp[2] = v.z; zp[3] = v.w;
            }
          }
        }
        constexpr int STEPS = 8 / NG;   // 16-column steps of a group
        constexpr uint32_t ONES[4] = {0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};
        float part[2][4], sums[4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {   // halves of 64 columns
          const uint4 q0 = lds128(rd + lane * 16 + 1024 * h), q1 = lds128(rd + lane * 16 + 1024 * h + 512);
          const uint32_t words[2][4] = {{q0.x, q0.y, q0.z, q0.w}, {q1.x, q1.y, q1.z, q1.w}};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int at = 4 * h + j, grp = at / STEPS;
            if (at % STEPS == 0) mma16816_first(sums, ONES, b[2 * at], b[2 * at + 1]);
            else mma16816(sums, ONES, b[2 * at], b[2 * at + 1]);
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              uint32_t f[4];
              w4_fragment(words[t][j], f);
              if (at % STEPS == 0) mma16816_first(part[t], f, b[2 * at], b[2 * at + 1]);
              else mma16816(part[t], f, b[2 * at], b[2 * at + 1]);
            }
            if (at % STEPS == STEPS - 1)
#pragma unroll
              for (int t = 0; t < 2; ++t) {
                const float zlo = ASYM ? w4_offset(zp[ASYM ? grp : 0] >> (16 * t)) : 24.f;
                const float zhi = ASYM ? w4_offset(zp[ASYM ? grp : 0] >> (16 * t + 8)) : 24.f;
                const float slo = bf16lo(sc[t][grp]), shi = bf16hi(sc[t][grp]);
                acc[t][0] = fmaf(slo, fmaf(-zlo, sums[0], part[t][0]), acc[t][0]);
                acc[t][1] = fmaf(slo, fmaf(-zlo, sums[1], part[t][1]), acc[t][1]);
                acc[t][2] = fmaf(shi, fmaf(-zhi, sums[0], part[t][2]), acc[t][2]);
                acc[t][3] = fmaf(shi, fmaf(-zhi, sums[1], part[t][3]), acc[t][3]);
              }
          }
        }
        __syncwarp();   // everybody has read the slot that the next copy fills
        wr = rd;
        rd = rd + SLOT == ring_end ? ring : rd + SLOT;
      }
      u += n;
      ku += n;
      if (began && lane == 0) tile_from[tile] = (uint8_t)warp;
      float* const to = began ? acc_s + tile * PIECE : head_s + warp * PIECE;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        *reinterpret_cast<float2*>(to + (16 * t + g) * 8 + 2 * c) = make_float2(acc[t][0], acc[t][1]);
        *reinterpret_cast<float2*>(to + (16 * t + g + 8) * 8 + 2 * c) = make_float2(acc[t][2], acc[t][3]);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[t][i] = 0.f;
      }
      if (ku == a.KU) {
        if (lane == 0) tile_to[tile] = (uint8_t)warp;
        began = true;
        ku = 0;
        ++tile;
        if (++rt == a.RT) {
          rt = 0;
          ++pass;
          if (u < u1) enter_pass();
        }
      }
    }
    // The next segment's first units and rows of x are read while this one is put together.
    const Segment done = sg;
    const int done_units = units;
    sg = plan(done.from + done.tiles);
    if (sg.tiles > 0) begin(sg);
    __syncthreads();
    if (sg.tiles > 0) stage(sg);

    // ---- pieces of a tile in the warps' order, then the result.  Threads: features fastest, 16 (gate and up) or 32 to a tile
    auto total = [&](int tl, int r, int col) {
      float v = acc_s[tl * PIECE + r * 8 + col];
      const int last = tile_to[tl];
      for (int w = tile_from[tl] + 1; w <= last; ++w)
        if (done_units * w / VEC_WARPS < done_units * (w + 1) / VEC_WARPS) v += head_s[w * PIECE + r * 8 + col];
      return v;
    };
    const int lg = a.down ? 5 : 4;
    for (int i = tid; i < done.tiles * VEC_ROWS << lg; i += VEC_THREADS) {
      const int f = i & ((1 << lg) - 1), rest = i >> lg, col = rest / done.tiles, tl = rest - col * done.tiles;
      const int over = (done.rt0 + tl) / a.RT, ps = done.pass0 + over, feature = (done.rt0 + tl - over * a.RT << lg) + f;
      const int at = pass_row[ps] + col;
      if (at >= pass_row[ps + 1] || feature >= a.n_out) continue;
      if (a.down) {
        a.Y[(size_t)at * a.y_ld + feature] = total(tl, f, col);
      } else {
        const int r = (f & 8) * 2 + (f & 7);   // of the two sixteens of rows
        const float gate = total(tl, r, col), up = total(tl, r + 8, col);
        const float act = slot_w[row_slot[at]] * (gate / (1.0f + __expf(-gate)) * up);
        a.A[(size_t)at * a.a_ld + feature] = (uint16_t)(pack_bf16x2(act, 0.f) & 0xFFFFu);
      }
    }
  }
  cp_async_wait<0>();
}

int w4_vec_rows(int K, int group, bool asym) {
  const int ng = W4_UNIT_K / group;
  const long room = (long)VEC_SMEM - (long)vec_fixed_smem(ng, asym);
  const long rows = room / vec_ld((K + W4_UNIT_K - 1) / W4_UNIT_K);
  return (int)(rows < 0 ? 0 : rows < VEC_ROWS_MOST ? rows : VEC_ROWS_MOST);
}

cudaError_t launch_w4_vec(W4VecArgs a, int num_sms, cudaStream_t st, int* launches) {
  const int ng = W4_UNIT_K / a.group;
  const bool asym = a.zeros != nullptr;
  a.rows_cap = w4_vec_rows(a.K, a.group, asym);
  const long slots = (long)a.T * a.kp;
  if (a.rows_cap > slots) a.rows_cap = (int)slots;
  a.group_rows = a.rows_cap < VEC_ROWS ? a.rows_cap : VEC_ROWS;
  const size_t smem = vec_fixed_smem(ng, asym) + (size_t)a.rows_cap * vec_ld(a.KU);
  ++*launches;
#define MOE_W4_VEC(ASYM, NG)                                                                  \
  do {                                                                                        \
    if (cudaError_t e = opt_in_smem<w4_vec_kernel<ASYM, NG>>(VEC_SMEM)) return e;             \
    return launch_dependent(w4_vec_kernel<ASYM, NG>, dim3(num_sms), dim3(VEC_THREADS), smem, st, a); \
  } while (0)
  if (a.group == 32) {
    if (asym) MOE_W4_VEC(true, 4);
    MOE_W4_VEC(false, 4);
  }
  if (a.group == 64) {
    if (asym) MOE_W4_VEC(true, 2);
    MOE_W4_VEC(false, 2);
  }
  if (asym) MOE_W4_VEC(true, 1);
  MOE_W4_VEC(false, 1);
#undef MOE_W4_VEC
}

// ------------------------------------------------------------------------------------------
// Combine over fp32 rows: a thread has eight features of a token.
// ------------------------------------------------------------------------------------------
constexpr int W4_COMBINE_THREADS = 128;
__global__ void __launch_bounds__(W4_COMBINE_THREADS) w4_combine_kernel(const float* __restrict__ Y, int y_ld, const int* __restrict__ prow_of, int T,
                                                                        int d, int kp, uint16_t* __restrict__ out) {
  pdl_wait();
  pdl_trigger();
  const int nvec = d >> 3;
  const int64_t n = (int64_t)T * nvec;
  for (int64_t i = (int64_t)blockIdx.x * W4_COMBINE_THREADS + threadIdx.x; i < n; i += (int64_t)gridDim.x * W4_COMBINE_THREADS) {
    const int t = (int)(i / nvec), v = (int)(i - (int64_t)t * nvec);
    float4 lo = make_float4(0.f, 0.f, 0.f, 0.f), hi = lo;
#pragma unroll 4
    for (int j = 0; j < kp; ++j) {
      const int p = __ldg(prow_of + (size_t)t * kp + j);
      if (p < 0) continue;
      const float4* row = reinterpret_cast<const float4*>(Y + (size_t)p * y_ld) + 2 * v;
      const float4 x = __ldcs(row), y = __ldcs(row + 1);
      lo.x += x.x; lo.y += x.y; lo.z += x.z; lo.w += x.w;
      hi.x += y.x; hi.y += y.y; hi.z += y.z; hi.w += y.w;
    }
    reinterpret_cast<uint4*>(out + (size_t)t * d)[v] =
        make_uint4(pack_bf16x2(lo.x, lo.y), pack_bf16x2(lo.z, lo.w), pack_bf16x2(hi.x, hi.y), pack_bf16x2(hi.z, hi.w));
  }
}

cudaError_t launch_w4_combine(const float* Y, int y_ld, const int* prow_of, int T, int d, int kp, uint16_t* out, cudaStream_t st, int* launches) {
  const int64_t blocks = ((int64_t)T * (d >> 3) + W4_COMBINE_THREADS - 1) / W4_COMBINE_THREADS;
  ++*launches;
  return launch_dependent(w4_combine_kernel, dim3((unsigned)(blocks < 148 * 16 ? blocks : 148 * 16)), dim3(W4_COMBINE_THREADS), 0, st, Y, y_ld, prow_of, T,
                          d, kp, out);
}

}  // namespace moe
