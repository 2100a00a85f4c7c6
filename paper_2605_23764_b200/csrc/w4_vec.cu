// The layer's expert products over 4-bit weights for experts with a few rows: token generation.
//
//   h[i] = sum_groups s_g sum_k (q - z) x[i][k];   A = w silu(h_gate) h_up;   Y = the same over A;   out[t] = sum_j Y of its slots
//
// What bounds it: the weights' bytes, read once.  Every warp streams its share of the row tiles straight into registers (16 bytes
// a lane and tile, eight tiles in flight), widens the codes to bf16 -- q - z is a small whole number, exact -- and multiplies 16 rows
// by up to 8 rows of x at a time (mma.m16n8k16, which a matrix-vector product needs as a dot-product unit, not for its rate).
// A group's sum is scaled in fp32: the only rounding to fewer bits on the way is that of A to bf16.
//
// Split.  Blocks take consecutive row tiles of the hit experts, one block an SM; inside a block the warps share the (row tile, 64
// columns) units evenly, whatever the tile boundaries: a row tile that several warps have a piece of is put together from shared
// memory in the warps' order.  So few experts and long reductions keep all warps at work, and results do not depend on timing.
#include "launch_pairs.cuh"
#include "topk.cuh"
#include "w4.cuh"

namespace moe {

namespace {

constexpr int VEC_WARPS = 16, VEC_THREADS = 32 * VEC_WARPS;
constexpr int VEC_ROWS = 8;          // rows of x that a pass over an expert's weights takes
constexpr int VEC_SEG_TILES = 64;    // row tiles between two joins
constexpr int VEC_SEG_GROUPS = 32;   // passes a segment may touch: a lane each
constexpr int VEC_DEPTH = 8;         // units in flight per warp
constexpr int VEC_SMEM = 222 * 1024;
constexpr int VEC_ROWS_MOST = 64;    // staged rows, at most

__host__ __device__ constexpr int vec_ld(int KB) { return KB * W4_TILE_K * 2 + 16; }   // bytes from row to row: ldmatrix rows in different banks
__host__ __device__ constexpr size_t vec_fixed_smem(int Ep) {
  return (size_t)(VEC_SEG_TILES + VEC_WARPS) * W4_TILE_BYTES + sizeof(int) * (3 * (size_t)Ep + 4);
}

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }
__device__ __forceinline__ void ldmatrix4(uint32_t addr, uint32_t* r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint4 ld_stream(const uint4* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}

// Exclusive scan of v over the block, n <= 3 values a thread; returns the total.
__device__ __forceinline__ int block_scan3(int (&v)[3], int* warp_sums) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int mine = v[0] + v[1] + v[2];
  int run = mine;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const int o = __shfl_up_sync(0xffffffffu, run, off);
    if (lane >= off) run += o;
  }
  if (lane == 31) warp_sums[warp] = run;
  __syncthreads();
  int before = 0, total = 0;
#pragma unroll
  for (int w = 0; w < VEC_WARPS; ++w) {
    const int s = warp_sums[w];
    if (w < warp) before += s;
    total += s;
  }
  __syncthreads();
  int at = before + run - mine;
#pragma unroll
  for (int i = 0; i < 3; ++i) { const int x = v[i]; v[i] = at; at += x; }
  return total;
}
static_assert(3 * VEC_THREADS >= 1024 + 64, "an expert for each scanned value");

}  // namespace

// G32: groups of 32, two to a unit of 64 columns; else a unit lies in one group.
template <bool ASYM, bool G32>
__global__ void __launch_bounds__(VEC_THREADS, 1) w4_vec_kernel(const W4VecArgs a) {
  extern __shared__ __align__(16) uint8_t vsm[];
  __shared__ int warp_sums[VEC_WARPS];
  __shared__ int slot_at[W4_SMALL_SLOTS], slot_e[W4_SMALL_SLOTS];
  // the segment: passes (expert, first staged row, rows), staged rows (row of A / Y, slot's weight)
  __shared__ int sg_e[VEC_SEG_GROUPS], sg_x[VEC_SEG_GROUPS], sg_n[VEC_SEG_GROUPS], seg_end, seg_rows;
  __shared__ int row_p[VEC_ROWS_MOST], row_t[VEC_ROWS_MOST];
  __shared__ float row_w[VEC_ROWS_MOST];
  float* const acc_s = reinterpret_cast<float*>(vsm);                                  // [VEC_SEG_TILES][16][8]
  float* const head_s = acc_s + VEC_SEG_TILES * W4_TILE_BYTES / 4;                     // [VEC_WARPS][16][8]
  int* const cnt = reinterpret_cast<int*>(head_s + VEC_WARPS * W4_TILE_BYTES / 4);     // [Ep] rows of the expert
  int* const first = cnt + a.Ep;                                                       // [Ep] first row of the expert (few slots)
  int* const gstart = first + a.Ep;                                                    // [Ep + 1] first pass of the expert
  const int ld = vec_ld(a.KB);
  uint8_t* const xs = vsm + ((vec_fixed_smem(a.Ep) + 15) & ~size_t(15));               // [rows_cap][ld]
  const int warp = warp_index(), lane = threadIdx.x & 31, tid = threadIdx.x, g = lane >> 2, c = lane & 3;
  const bool small = a.counts == nullptr;

  // The first product waits for what is in front of it here; the second one's ids or layout were complete before the first started,
  // so it waits only where it reads what the first product wrote.
  if (!a.down) {
    pdl_wait();
    pdl_trigger();
  }
  // ---- rows of each expert, passes over each expert's weights
  if (small) {
    const int n = a.T * a.kp;
    for (int e = tid; e < a.Ep; e += VEC_THREADS) cnt[e] = 0;
    __syncthreads();
    int e = -1;
    if (tid < n) {
      const int t = tid / a.kp, j = tid - t * a.kp;
      e = j < a.k ? __ldcg(a.ids + t * a.k + j) : a.E + j - a.k;
      if (j < a.k && (e < 0 || e >= a.E)) e = -1;
      slot_e[tid] = e;
      if (e >= 0) atomicAdd(&cnt[e], 1);
      else if (blockIdx.x == 0 && !a.down) note(a.status, /*MOE_ERR_BAD_EXPERT_ID*/ 1, tid);
    }
    __syncthreads();
    int rank = 0;
    if (e >= 0)
      for (int i = 0; i < tid; ++i) rank += slot_e[i] == e;
    int v[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) v[i] = 3 * tid + i < a.Ep ? cnt[3 * tid + i] : 0;
    block_scan3(v, warp_sums);
#pragma unroll
    for (int i = 0; i < 3; ++i)
      if (3 * tid + i < a.Ep) first[3 * tid + i] = v[i];
    __syncthreads();
    if (tid < n) {
      const int at = e >= 0 ? first[e] + rank : -1;
      if (e >= 0) slot_at[at] = tid;
      if (blockIdx.x == 0 && !a.down) a.prow_of[tid] = at;
    }
  } else {
    for (int e = tid; e < a.Ep; e += VEC_THREADS) {
      const int n = __ldcg(a.counts + e);
      cnt[e] = n <= a.rows_most ? n : 0;
    }
  }
  __syncthreads();
  int passes;
  {
    int v[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) v[i] = 3 * tid + i < a.Ep ? (cnt[3 * tid + i] + a.group_rows - 1) / a.group_rows : 0;
    passes = block_scan3(v, warp_sums);
#pragma unroll
    for (int i = 0; i < 3; ++i)
      if (3 * tid + i < a.Ep) gstart[3 * tid + i] = v[i];
    if (tid == 0) gstart[a.Ep] = passes;
  }
  __syncthreads();

  const int64_t tiles = (int64_t)passes * a.RT;
  int64_t t0 = tiles * blockIdx.x / gridDim.x;
  const int64_t t1 = tiles * (blockIdx.x + 1) / gridDim.x;
  bool waited = !a.down;
  while (t0 < t1) {
    // ---- the segment [t0, te): as many tiles as have room, rows staged once
    const int p0 = (int)(t0 / a.RT);
    if (warp == 0) {
      const int p = p0 + lane;
      const int64_t most = min(t1, t0 + VEC_SEG_TILES);
      const bool in = p < passes && (int64_t)p * a.RT < most;
      int e = 0, i0 = 0, n = 0;
      if (in) {
        int lo = 0, hi = a.Ep;   // gstart[lo] <= p < gstart[hi]
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (gstart[mid] <= p) lo = mid; else hi = mid;
        }
        e = lo;
        i0 = (p - gstart[e]) * a.group_rows;
        n = min(a.group_rows, cnt[e] - i0);
      }
      int run = n;
#pragma unroll
      for (int off = 1; off < 32; off <<= 1) {
        const int o = __shfl_up_sync(0xffffffffu, run, off);
        if (lane >= off) run += o;
      }
      const uint32_t fits = __ballot_sync(0xffffffffu, in && run <= a.rows_cap);
      const int m = __popc(fits);   // the first m passes: their rows ascend
      if (lane < m) {
        const int x = run - n;
        sg_e[lane] = e;
        sg_x[lane] = x;
        sg_n[lane] = n;
        for (int i = 0; i < n; ++i) {
          int slot, p_row;
          if (small) { p_row = first[e] + i0 + i; slot = slot_at[p_row]; }
          else { slot = __ldcg(a.src_of + __ldcg(a.offsets + e) + i0 + i); p_row = __ldcg(a.pad_off + e) + i0 + i; }
          const int t = slot / a.kp, j = slot - t * a.kp;
          row_p[x + i] = p_row;
          row_t[x + i] = a.down ? p_row : t;
          row_w[x + i] = a.down || j >= a.k ? 1.f : __ldcg(a.w + (size_t)t * a.k + j);
        }
        if (lane == m - 1) seg_rows = run;
      }
      if (lane == 0) {
        const int64_t end = min(most, (int64_t)(p0 + m) * a.RT);
        seg_end = (int)(end - t0);
      }
    }
    __syncthreads();
    const int ntiles = seg_end, rt0 = (int)(t0 - (int64_t)p0 * a.RT);
    const int units = ntiles * a.KB;
    const int u0 = (int)((int64_t)units * warp / VEC_WARPS), u1 = (int)((int64_t)units * (warp + 1) / VEC_WARPS);

    // ---- the stream: unit u of the segment is k-tile u % KB of row tile u / KB
    uint4 q[VEC_DEPTH];
    uint32_t sc[VEC_DEPTH][G32 ? 2 : 1];
    uint32_t zp[VEC_DEPTH][ASYM ? (G32 ? 2 : 1) : 1];
    int f_tile = u0 / a.KB, f_kb = u0 - f_tile * a.KB, f_rt, f_pass;   // of the next unit to fetch
    {
      const int at = rt0 + f_tile;
      f_pass = at / a.RT;
      f_rt = at - f_pass * a.RT;
    }
    size_t f_row = 0;   // row tile over all experts
    if (u0 < u1) f_row = (size_t)sg_e[f_pass] * a.RT + f_rt;
    const int glog = a.group == 128 ? 7 : 6;
    auto fetch = [&](int i, bool on) {
      if (!on) return;
      q[i] = ld_stream(a.codes + (f_row * a.KB + f_kb) * 32 + lane);
      const size_t sg = f_row * a.NG + (G32 ? 2 * f_kb : (f_kb * W4_TILE_K) >> glog);
      sc[i][0] = __ldg(a.scales + sg * 8 + g);
      if (G32) sc[i][G32 ? 1 : 0] = __ldg(a.scales + (sg + 1) * 8 + g);
      if (ASYM) {
        zp[i][0] = __ldg(a.zeros + sg * 8 + g);
        if (G32) zp[i][ASYM && G32 ? 1 : 0] = __ldg(a.zeros + (sg + 1) * 8 + g);
      }
      if (++f_kb == a.KB) {
        f_kb = 0;
        ++f_row;
        if (++f_rt == a.RT) {
          f_rt = 0;
          ++f_pass;
          if (f_pass < VEC_SEG_GROUPS) f_row = (size_t)sg_e[f_pass] * a.RT;
        }
      }
    };
#pragma unroll
    for (int i = 0; i < VEC_DEPTH; ++i) fetch(i, u0 + i < u1);

    // ---- the rows of x, zeros behind K
    if (!waited) {
      pdl_wait();
      pdl_trigger();
      waited = true;
    }
    {
      const int pieces = a.KB * (W4_TILE_K / 8), full = a.K >> 3, rows = seg_rows;
      for (int i = tid; i < rows * pieces; i += VEC_THREADS) {
        const int r = i / pieces, v = i - r * pieces;
        uint8_t* dst = xs + (size_t)r * ld + v * 16;
        if (v < full) cp_async16(smem_u32(dst), a.in + (size_t)row_t[r] * a.in_ld + v * 8);
        else *reinterpret_cast<uint4*>(dst) = make_uint4(0, 0, 0, 0);
      }
      cp_async_wait_all();
    }
    __syncthreads();

    // ---- the products
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    int tile = u0 / a.KB, kb = u0 - tile * a.KB;
    bool began = kb == 0;   // this warp has the tile from its first unit on
    uint32_t x_addr = 0;
    int rt = 0, pass = 0;
    auto enter_pass = [&]() {   // operand rows: lane l gives row l % 8 of matrix l / 8; rows that are not there are computed and dropped
      const int r = min(lane & 7, sg_n[pass] - 1);
      x_addr = smem_u32(xs + (size_t)(sg_x[pass] + r) * ld) + (lane >> 3) * 16;
    };
    if (u0 < u1) {
      const int at = rt0 + tile;
      pass = at / a.RT;
      rt = at - pass * a.RT;
      enter_pass();
    }
    auto put = [&](float* to) {
      *reinterpret_cast<float2*>(to + g * 8 + 2 * c) = make_float2(acc[0], acc[1]);
      *reinterpret_cast<float2*>(to + (g + 8) * 8 + 2 * c) = make_float2(acc[2], acc[3]);
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i] = 0.f;
    };
#pragma unroll 1
    for (int u = u0; u < u1; u += VEC_DEPTH) {
#pragma unroll
      for (int i = 0; i < VEC_DEPTH; ++i) {
        if (u + i < u1) {
          uint32_t b[8];
          ldmatrix4(x_addr + kb * (W4_TILE_K * 2), b);
          ldmatrix4(x_addr + kb * (W4_TILE_K * 2) + 64, b + 4);
          const uint32_t words[4] = {q[i].x, q[i].y, q[i].z, q[i].w};
#pragma unroll
          for (int h = 0; h < (G32 ? 2 : 1); ++h) {
            const uint32_t z = ASYM ? zp[i][ASYM && G32 ? h : 0] : 0x0808u;
            const uint32_t blo = w4_bias(z & 0xFFu), bhi = w4_bias(z >> 8);
            float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < (G32 ? 2 : 4); ++j) {
              const int jj = (G32 ? 2 * h : 0) + j;
              uint32_t f[4];
              w4_fragment(words[jj], blo, bhi, f);
              mma16816(part, f, b[2 * jj], b[2 * jj + 1]);
            }
            const float slo = bf16lo(sc[i][G32 ? h : 0]), shi = bf16hi(sc[i][G32 ? h : 0]);
            acc[0] = fmaf(slo, part[0], acc[0]);
            acc[1] = fmaf(slo, part[1], acc[1]);
            acc[2] = fmaf(shi, part[2], acc[2]);
            acc[3] = fmaf(shi, part[3], acc[3]);
          }
          fetch(i, u + i + VEC_DEPTH < u1);
          if (++kb == a.KB) {
            put(began ? acc_s + tile * 128 : head_s + warp * 128);
            began = true;
            kb = 0;
            ++tile;
            if (++rt == a.RT) {
              rt = 0;
              ++pass;
              if (u + i + 1 < u1) enter_pass();
            }
          }
        }
      }
    }
    if (u0 < u1 && kb != 0) put(began ? acc_s + tile * 128 : head_s + warp * 128);
    __syncthreads();

    // ---- pieces of a tile in the warps' order, then the result.  Threads: features fastest, 8 (gate and up) or 16 to a tile
    auto total = [&](int tl, int r, int col) {
      float v = acc_s[tl * 128 + r * 8 + col];
      const int lo = tl * a.KB, hi = lo + a.KB;   // units of the tile
      for (int w = (int)((int64_t)lo * VEC_WARPS / units); w < VEC_WARPS; ++w) {
        const int b0 = (int)((int64_t)units * w / VEC_WARPS), b1 = (int)((int64_t)units * (w + 1) / VEC_WARPS);
        if (b0 >= hi) break;
        if (b0 > lo && b1 > b0) v += head_s[w * 128 + r * 8 + col];
      }
      return v;
    };
    const int per = a.down ? 16 : 8;
    for (int i = tid; i < ntiles * per * VEC_ROWS; i += VEC_THREADS) {
      const int f = i % per, rest = i / per, tl = rest % ntiles, col = rest / ntiles;
      const int at = rt0 + tl, ps = at / a.RT, feature = (at - ps * a.RT) * per + f;
      if (col >= sg_n[ps] || feature >= a.n_out) continue;
      const int xr = sg_x[ps] + col;
      if (a.down) {
        a.Y[(size_t)row_p[xr] * a.y_ld + feature] = total(tl, f, col);
      } else {
        const float gate = total(tl, f, col), up = total(tl, f + 8, col);
        const float act = row_w[xr] * (gate / (1.0f + __expf(-gate)) * up);
        a.A[(size_t)row_p[xr] * a.a_ld + feature] = (uint16_t)(pack_bf16x2(act, 0.f) & 0xFFFFu);
      }
    }
    __syncthreads();
    t0 += ntiles;
  }
  if (!waited) {
    pdl_wait();
    pdl_trigger();
  }
}

int w4_vec_rows(int K) {
  const int KB = (K + W4_TILE_K - 1) / W4_TILE_K;
  const long room = (long)VEC_SMEM - (long)((vec_fixed_smem(1024 + 64) + 15) & ~size_t(15));
  const long rows = room / vec_ld(KB);
  return (int)(rows < VEC_ROWS_MOST ? rows : VEC_ROWS_MOST);
}

cudaError_t launch_w4_vec(W4VecArgs a, int num_sms, cudaStream_t st, int* launches) {
  const size_t fixed = (vec_fixed_smem(a.Ep) + 15) & ~size_t(15);
  a.rows_cap = w4_vec_rows(a.K);
  const long slots = (long)a.T * a.kp;
  if (a.rows_cap > slots) a.rows_cap = (int)slots;
  a.group_rows = a.rows_cap < VEC_ROWS ? a.rows_cap : VEC_ROWS;
  const size_t smem = fixed + (size_t)a.rows_cap * vec_ld(a.KB);
  ++*launches;
#define MOE_W4_VEC(ASYM, G32)                                                                  \
  do {                                                                                         \
    if (cudaError_t e = opt_in_smem<w4_vec_kernel<ASYM, G32>>(VEC_SMEM)) return e;              \
    return launch_dependent(w4_vec_kernel<ASYM, G32>, dim3(num_sms), dim3(VEC_THREADS), smem, st, a); \
  } while (0)
  if (a.group == 32) {
    if (a.zeros) MOE_W4_VEC(true, true);
    MOE_W4_VEC(false, true);
  }
  if (a.zeros) MOE_W4_VEC(true, false);
  MOE_W4_VEC(false, false);
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
