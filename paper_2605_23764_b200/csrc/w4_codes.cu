// Weights into 4 bits, from a checkpoint's natural codes into the layout of w4.cuh, and back to the values they stand for.
// A warp takes 16 rows x 128 columns, half a unit: lanes 16 h + m have columns 8 m .. of rows 2 i + h, and change places with the
// layout's lanes through 1 KB of shared memory.  Bound by the bytes of the matrices.
#include "launch_pairs.cuh"
#include "topk.cuh"
#include "w4.cuh"

namespace moe {

namespace {

constexpr int CODE_WARPS = 8, CODE_LD = 17;   // words of a staged row: 16 of codes, one so that rows fall into different banks

struct CodeTask { int64_t unit; int m, rt, chunk, t; };   // unit of all, matrix, row tile, unit of the tile, upper or lower 16 rows
__device__ __forceinline__ CodeTask code_task(int64_t i, int RTS, int chunks) {
  CodeTask t;
  t.unit = i >> 1;
  t.t = (int)(i & 1);
  const int64_t four = t.unit >> 2, tiles = four / chunks;   // four units, four row tiles
  t.chunk = (int)(four - tiles * chunks);
  t.m = (int)(tiles / (RTS >> 2));
  t.rt = (int)(tiles - (int64_t)t.m * (RTS >> 2)) * 4 + (int)(t.unit & 3);
  return t;
}

// natural words [16][CODE_LD] <-> the lane's words of half b of the unit
__device__ __forceinline__ uint4 gather_words(const uint32_t* st, int b, int lane) {
  const int g = lane >> 2, c8 = (lane & 3) * 8;
  uint32_t out[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int at = 8 * b + 2 * j;
    const uint32_t by[4] = {st[g * CODE_LD + at] >> c8, st[(g + 8) * CODE_LD + at] >> c8, st[g * CODE_LD + at + 1] >> c8,
                            st[(g + 8) * CODE_LD + at + 1] >> c8};
    uint32_t w = 0;
#pragma unroll
    for (int r = 0; r < 4; ++r) w |= (by[r] & 15u) << (4 * r) | ((by[r] >> 4) & 15u) << (16 + 4 * r);
    out[j] = w;
  }
  return make_uint4(out[0], out[1], out[2], out[3]);
}
__device__ __forceinline__ void scatter_words(uint32_t* st, int b, int lane, uint4 v) {
  const int g = lane >> 2, c = lane & 3;
  uint8_t* by = reinterpret_cast<uint8_t*>(st);
  const uint32_t in[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      by[4 * ((g + (r & 1) * 8) * CODE_LD + 8 * b + 2 * j + (r >> 1)) + c] =
          (uint8_t)((in[j] >> (4 * r) & 15u) | (in[j] >> (16 + 4 * r) & 15u) << 4);
}

// bf16 of s (q - z): the product has at most 13 significant bits, so one rounding
__device__ __forceinline__ float code_value(uint32_t q, float s, float z) { return s * ((float)q - z); }

__device__ __forceinline__ float bf16_round(float v) { return __bfloat162float(__float2bfloat16_rn(v)); }

}  // namespace

// ------------------------------------------------------------------------------------------
// QUANT: src = bf16 W [n][rows][cols].  Without zero points s = bf16(max |w| / 7), q = round(w / s) + 8, round to even, q in 0 .. 15;
// with them s = bf16((hi - lo) / 15) over the group's values and zero, z = round(-lo / s), q = round(w / s) + z.  Division as IEEE rounds it.
// else : src = codes [n][rows][cols / 2], the even column in the low half of a byte, with their scales and zero points.
// ------------------------------------------------------------------------------------------
template <bool QUANT>
__global__ void __launch_bounds__(32 * CODE_WARPS) w4_encode_kernel(const void* __restrict__ src, const uint16_t* __restrict__ qs,
                                                                    const uint8_t* __restrict__ qz, int64_t tasks, int chunks, W4Shape s,
                                                                    uint4* __restrict__ codes, uint16_t* __restrict__ scales,
                                                                    uint8_t* __restrict__ zeros) {
  __shared__ uint32_t stage[CODE_WARPS][16 * CODE_LD];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, h = lane >> 4, m = lane & 15;
  uint32_t* const st = stage[warp];
  const int RT = s.stored_tiles(), ng = s.unit_groups(), ng_src = (s.cols + s.group - 1) / s.group;
  const int gl = s.group >> 3;   // lanes of a group
  const bool asym = zeros != nullptr;
  pdl_wait();
  pdl_trigger();
  for (int64_t i = (int64_t)blockIdx.x * CODE_WARPS + warp; i < tasks; i += (int64_t)gridDim.x * CODE_WARPS) {
    const CodeTask t = code_task(i, RT, chunks);
    const int col = t.chunk * 128 + m * 8, grp = t.chunk * ng + m / gl;
    const bool leads = m % gl == 0;
    uint4 in[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const int row = s.row_at(t.rt, 16 * t.t + 2 * q + h);
      in[q] = make_uint4(0, 0, 0, 0);
      if (row >= 0 && col < s.cols) {
        const size_t at = ((size_t)t.m * s.rows + row) * s.cols + col;
        if (QUANT) in[q] = __ldcs(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(src) + at));
        else in[q].x = __ldcs(reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(src) + at / 2));
      }
    }
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const int r = 2 * q + h, row = s.row_at(t.rt, 16 * t.t + r);
      uint32_t word;
      float scale = 0.f, zero = 8.f;
      if (QUANT) {
        float v[8] = {bf16lo(in[q].x), bf16hi(in[q].x), bf16lo(in[q].y), bf16hi(in[q].y), bf16lo(in[q].z), bf16hi(in[q].z), bf16lo(in[q].w), bf16hi(in[q].w)};
        float lo = 0.f, hi = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) { lo = fminf(lo, v[e]); hi = fmaxf(hi, v[e]); }
        for (int off = gl >> 1; off; off >>= 1) {
          lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, off));
          hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, off));
        }
        scale = bf16_round(asym ? __fdiv_rn(hi - lo, 15.f) : __fdiv_rn(fmaxf(hi, -lo), 7.f));
        const float step = scale > 0.f ? scale : 1.f;
        if (asym) zero = fminf(fmaxf(rintf(__fdiv_rn(-lo, step)), 0.f), 15.f);
        word = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float code = fminf(fmaxf(rintf(__fdiv_rn(v[e], step)) + zero, 0.f), 15.f);
          word |= (uint32_t)code << (4 * e);
        }
      } else {
        const bool in_matrix = row >= 0 && t.chunk * 128 + (m / gl) * s.group < s.cols;   // the group has columns
        if (in_matrix) {
          const size_t at = ((size_t)t.m * s.rows + row) * ng_src + grp;
          scale = __uint_as_float((uint32_t)qs[at] << 16);
          if (asym) zero = (float)min((int)qz[at], 15);
        }
        word = row >= 0 && col < s.cols ? in[q].x : (uint32_t)zero * 0x11111111u;
      }
      st[r * CODE_LD + m] = word;
      if (leads) {
        const size_t at = (((size_t)t.unit * 8 + (r & 7)) * ng + m / gl) * 4 + 2 * t.t + (r >> 3);
        scales[at] = (uint16_t)(__float_as_uint(scale) >> 16);
        if (asym) zeros[at] = (uint8_t)zero;
      }
    }
    __syncwarp();
#pragma unroll
    for (int b = 0; b < 2; ++b) codes[((size_t)t.unit * 4 + 2 * b + t.t) * 32 + lane] = gather_words(st, b, lane);
    __syncwarp();
  }
}

__global__ void __launch_bounds__(32 * CODE_WARPS) w4_decode_kernel(const uint4* __restrict__ codes, const uint16_t* __restrict__ scales,
                                                                    const uint8_t* __restrict__ zeros, int64_t tasks, int chunks, W4Shape s,
                                                                    uint16_t* __restrict__ W) {
  __shared__ uint32_t stage[CODE_WARPS][16 * CODE_LD];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, h = lane >> 4, m = lane & 15;
  uint32_t* const st = stage[warp];
  const int RT = s.stored_tiles(), ng = s.unit_groups();
  pdl_wait();
  pdl_trigger();
  for (int64_t i = (int64_t)blockIdx.x * CODE_WARPS + warp; i < tasks; i += (int64_t)gridDim.x * CODE_WARPS) {
    const CodeTask t = code_task(i, RT, chunks);
    const int col = t.chunk * 128 + m * 8, grp = m * 8 / s.group;
    uint4 w[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) w[b] = __ldcs(&codes[((size_t)t.unit * 4 + 2 * b + t.t) * 32 + lane]);
    float sc[8], z[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const int r = 2 * q + h;
      const size_t at = (((size_t)t.unit * 8 + (r & 7)) * ng + grp) * 4 + 2 * t.t + (r >> 3);
      sc[q] = __uint_as_float((uint32_t)scales[at] << 16);
      z[q] = zeros ? (float)zeros[at] : 8.f;
    }
#pragma unroll
    for (int b = 0; b < 2; ++b) scatter_words(st, b, lane, w[b]);
    __syncwarp();
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const int r = 2 * q + h, row = s.row_at(t.rt, 16 * t.t + r);
      const uint32_t word = st[r * CODE_LD + m];
      uint32_t o[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = pack_bf16x2(code_value(word >> (8 * e) & 15u, sc[q], z[q]), code_value(word >> (8 * e + 4) & 15u, sc[q], z[q]));
      if (row >= 0 && col < s.cols) __stcs(reinterpret_cast<uint4*>(W + ((size_t)t.m * s.rows + row) * s.cols + col), make_uint4(o[0], o[1], o[2], o[3]));
    }
    __syncwarp();
  }
}

static dim3 code_grid(int64_t tasks) {
  const int64_t blocks = (tasks + CODE_WARPS - 1) / CODE_WARPS;
  return dim3((unsigned)(blocks < 148 * 8 ? blocks : 148 * 8));
}

cudaError_t launch_w4_quantize(const uint16_t* W, int n, const W4Shape& s, uint32_t* codes, uint16_t* scales, uint8_t* zeros, cudaStream_t st) {
  const int chunks = s.units();
  const int64_t tasks = (int64_t)n * s.stored_tiles() * chunks * 2;
  return launch_dependent(w4_encode_kernel<true>, code_grid(tasks), dim3(32 * CODE_WARPS), 0, st, W, nullptr, nullptr, tasks, chunks, s,
                          reinterpret_cast<uint4*>(codes), scales, zeros);
}
cudaError_t launch_w4_pack(const uint8_t* q, const uint16_t* qs, const uint8_t* qz, int n, const W4Shape& s, uint32_t* codes, uint16_t* scales,
                           uint8_t* zeros, cudaStream_t st) {
  const int chunks = s.units();
  const int64_t tasks = (int64_t)n * s.stored_tiles() * chunks * 2;
  return launch_dependent(w4_encode_kernel<false>, code_grid(tasks), dim3(32 * CODE_WARPS), 0, st, q, qs, qz, tasks, chunks, s,
                          reinterpret_cast<uint4*>(codes), scales, zeros);
}
cudaError_t launch_w4_dequantize(const uint32_t* codes, const uint16_t* scales, const uint8_t* zeros, int n, const W4Shape& s, uint16_t* W, cudaStream_t st) {
  const int chunks = s.units();
  const int64_t tasks = (int64_t)n * s.stored_tiles() * chunks * 2;
  return launch_dependent(w4_decode_kernel, code_grid(tasks), dim3(32 * CODE_WARPS), 0, st, reinterpret_cast<const uint4*>(codes), scales, zeros,
                          tasks, chunks, s, W);
}

}  // namespace moe
