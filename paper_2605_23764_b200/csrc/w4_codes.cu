// Weights into 4 bits, from a checkpoint's natural codes into the layout of w4.cuh, and back to the values they stand for.
// A warp takes 16 rows x 128 columns, half a unit: lanes 16 h + m have columns 8 m .. of rows 2 i + h, and change places with the
// layout's lanes through 1 KB of shared memory.  Measured for 64 matrices of 2816 x 2048, groups of 128: 395 us to quantize (740 MB in,
// 190 MB out: 2.4 TB/s; the instructions of a code -- largest value, product, two roundings, clamp, place -- fill 64 % of the issue slots,
// with four warps a scheduler), 450 with zero points of groups of 64; 218 us to pack, 267 with those (1.7 TB/s); 194 us back
// (4.8 TB/s; three quarters of the issue slots).
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

// Staged words [16 rows][CODE_LD]: word m of a row has columns 8 m .., the even ones in its low half, the odd ones in its high half --
// pair c of the four in bits 4 c .. and 16 + 4 c .., where the layout's lanes want them.
// -> the lane's words of half b of the unit
__device__ __forceinline__ uint4 gather_words(const uint32_t* st, int b, int lane) {
  const int g = lane >> 2, c4 = (lane & 3) * 4;
  uint32_t out[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int at = 8 * b + 2 * j;
    const uint32_t in[4] = {st[g * CODE_LD + at], st[(g + 8) * CODE_LD + at], st[g * CODE_LD + at + 1], st[(g + 8) * CODE_LD + at + 1]};
    uint32_t w = 0;
#pragma unroll
    for (int r = 0; r < 4; ++r) w += ((in[r] >> c4) & 0x000F000Fu) << (4 * r);
    out[j] = __funnelshift_l(w, w, 3);
  }
  return make_uint4(out[0], out[1], out[2], out[3]);
}
// Natural codes (two to a byte, the even column in its low half) to and from such a word.
__device__ __forceinline__ uint32_t squeeze(uint32_t x) {   // the low halves of four bytes side by side
  x &= 0x0F0F0F0Fu;
  x = (x | x >> 4) & 0x00FF00FFu;
  return (x | x >> 8) & 0xFFFFu;
}
__device__ __forceinline__ uint32_t split_word(uint32_t natural) { return squeeze(natural) | squeeze(natural >> 4) << 16; }
// the decoder's way back: natural words
__device__ __forceinline__ void scatter_words(uint32_t* st, int b, int lane, uint4 v) {
  const int g = lane >> 2, c = lane & 3;
  uint8_t* by = reinterpret_cast<uint8_t*>(st);
  uint32_t in[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) in[j] = __funnelshift_r(in[j], in[j], 3);
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
    // ---- scale and zero point of each row's group, known to its lanes
    float scale[8], zero[8], inv[8];
    bool plain = false;   // a scale so small that its reciprocal is none
    if (QUANT) {
      float lo[8], hi[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const uint32_t w[4] = {in[q].x, in[q].y, in[q].z, in[q].w};
        lo[q] = hi[q] = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          lo[q] = fminf(lo[q], fminf(bf16lo(w[e]), bf16hi(w[e])));
          hi[q] = fmaxf(hi[q], fmaxf(bf16lo(w[e]), bf16hi(w[e])));
        }
        if (!asym) hi[q] = fmaxf(hi[q], -lo[q]);
      }
#pragma unroll
      for (int off = 8; off; off >>= 1)
        if (off < gl)
#pragma unroll
          for (int q = 0; q < 8; ++q) {
            if (asym) lo[q] = fminf(lo[q], __shfl_xor_sync(0xffffffffu, lo[q], off));
            hi[q] = fmaxf(hi[q], __shfl_xor_sync(0xffffffffu, hi[q], off));
          }
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        // (hi - lo) / 15 of halves, which are exact: the difference may be beyond fp32
        scale[q] = bf16_round(asym ? __fdiv_rn(__fmaf_rn(0.5f, hi[q], -0.5f * lo[q]), 7.5f) : __fdiv_rn(hi[q], 7.f));
        const float step = scale[q] > 0.f ? scale[q] : 1.f;
        zero[q] = asym ? fminf(fmaxf(rintf(__fdiv_rn(-lo[q], step)), 0.f), 15.f) : 8.f;
        inv[q] = __fdividef(1.0f, step);
        plain |= step < 1e-30f;
      }
    } else {
      const bool in_matrix = t.chunk * 128 + (m / gl) * s.group < s.cols;   // the group has columns
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const int row = s.row_at(t.rt, 16 * t.t + 2 * q + h);
        scale[q] = 0.f;
        zero[q] = 8.f;
        if (in_matrix && row >= 0) {
          const size_t at = ((size_t)t.m * s.rows + row) * ng_src + grp;
          scale[q] = __uint_as_float((uint32_t)qs[at] << 16);
          if (asym) zero[q] = (float)min((int)qz[at], 15);
        }
      }
    }
    const bool exact = QUANT && __any_sync(0xffffffffu, plain);
    // ---- codes
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const int r = 2 * q + h, row = s.row_at(t.rt, 16 * t.t + r);
      uint32_t word;
      if (QUANT) {
        const uint32_t w[4] = {in[q].x, in[q].y, in[q].z, in[q].w};
        if (exact) {
          word = 0;
          const float step = scale[q] > 0.f ? scale[q] : 1.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float v = e & 1 ? bf16hi(w[e >> 1]) : bf16lo(w[e >> 1]);
            const float code = fminf(fmaxf(rintf(__fdiv_rn(v, step)) + zero[q], 0.f), 15.f);
            word += (uint32_t)code << (e & 1 ? 16 + 2 * (e - 1) : 2 * e);
          }
        } else {
          // w / s to the nearest whole number, ties to even, without a division.  Both have 8 significant bits, so w / s is a tie or at
          // least 2^-9 away from one, while w (1 / s) is off by less than 2^-18 (15.1 times the two units of 2^-23 that the reciprocal
          // may be off by): rounded to 2^-11 -- by the sum with 6144 -- it is exactly the tie, or on its side of it.  The sum with
          // 1.5 x 2^23 then leaves the code in the lowest bits.
          constexpr float FINE = 6144.f, WHOLE = 12582912.f;
          uint32_t sum = 0;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float v = e & 1 ? bf16hi(w[e >> 1]) : bf16lo(w[e >> 1]);
            float y = __fadd_rn(__fadd_rn(__fmaf_rn(v, inv[q], FINE), -FINE), WHOLE);   // the whole number
            if (asym) y = fminf(fmaxf(__fadd_rn(y, zero[q]), WHOLE), WHOLE + 15.f);
            sum += __float_as_uint(y) * (1u << (e & 1 ? 16 + 2 * (e - 1) : 2 * e));
          }
          // (the bits above the code, which each of the eight brought along, and the 8 of a code without zero points)
          word = sum - (asym ? 0x4B400000u : 0x4B400000u - 8u) * 0x11111111u;
        }
      } else {
        word = row >= 0 && col < s.cols ? split_word(in[q].x) : (uint32_t)zero[q] * 0x11111111u;
      }
      st[r * CODE_LD + m] = word;
      if (leads) {
        const size_t at = (((size_t)t.unit * 8 + (r & 7)) * ng + m / gl) * 4 + 2 * t.t + (r >> 3);
        scales[at] = (uint16_t)(__float_as_uint(scale[q]) >> 16);
        if (asym) zeros[at] = (uint8_t)zero[q];
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
