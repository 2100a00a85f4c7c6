// Routing by groups of experts with a bias for balance (moe_route_grouped), the gradient of its weights, and the bias' update.
//
//   s_e = sigmoid(l_e) or softmax(l)_e, c_e = s_e + b_e; a group's score is the sum of its one or two largest c; the top_groups
//   groups of the largest scores stay, of their experts the k of the largest c; w = s (of the k over their sum), times scale.
//
// Which experts come out must not hang on a rounding: c is compared as it is in 64 bits, ties go to the lower index.  A warp has a
// token.  It selects in fp32 and looks whether the selection is beyond doubt: the groups kept and those left out, and every
// two neighbours in the order of the k + 1 largest, further apart than fp32 can have moved them (RouteTol).  Where the groups are not,
// theirs are computed in 64 bits, where the experts are not, those of the candidates (one token in a thousand of normally distributed
// logits, one in a hundred of a softmax over 512), and where that does not settle it, as with ties, everything is.  Without a bias the
// experts' order is that of the logits, whose comparison is exact, and so is that of groups by their best expert.
#include <float.h>
#include <limits.h>

#include "launch_pairs.cuh"
#include "moe_internal.h"
#include "topk.cuh"

namespace moe {

constexpr unsigned ALL = 0xffffffffu;

// 2^x to 2 ulp, 1 / x to one, log2 x to 2^-22; results below 2^-126 as 0
__device__ __forceinline__ float ex2_approx(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float rcp_approx(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float lg2_approx(float x) {
  float r;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
constexpr float LOG2E = 1.4426950408889634f;

// How far apart two c, or two groups' scores, are for certain in the order that fp32 gives them.  In units of 2^-23 of the value:
//   2^y of y = -l log2 e is off by 2 and by what y's rounding and that of log2 e move it, ln 2 (0.5 + 0.12) |y| < 0.43 |y|;
//   a sigmoid s = 1 / (1 + 2^y) takes the share 1 - s of that, the addition 0.5 and the reciprocal 1: at most 2.5 for l >= 0, and
//   3.5 + 0.43 y for l < 0, which grows without limit as s falls.  s (3.5 + 0.43 y) falls with s, so no expert's error is above
//   s_max (3.5 + 0.43 y) with the largest score's y, where that is positive; y < log2(1 + 2^y) = -log2 s_max.  One unit more is room for the
//   roundings of the comparison itself and of that logarithm.
//   A softmax score's is at most 2.5 of the largest score's, its sum's 10 (the mean of d = max - logit weighted with e^-d is under
//   ln 1024) and 37 additions' roundings: under 32 of the largest score.
// Doubled, since two values are compared, and rounded up; a group's score has two experts'.
//   The bias adds half an ulp of c, a group's sum the errors of both c and half an ulp of its own: of every value by itself, so that a bias that
//   keeps an expert out, -infinity or -1e9, leaves the others' comparisons what they are (by the largest bias of all, 65536 x 256 took 450 us
//   instead of 66, every token in 64 bits).
struct RouteTol {
  static constexpr float ULP = 1.2e-7f;   // 2^-23, rounded up
  float expert, group;
  __device__ RouteTol(bool sigmoid, float s_max) {
    const float s = s_max * (sigmoid ? fmaf(0.86f * ULP, -lg2_approx(fmaxf(s_max, FLT_MIN)), 9.f * ULP) : 64.f * ULP);
    constexpr float SUBNORMAL = 1e-37f;   // numbers below 2^-126 have steps of their own
    expert = s + SUBNORMAL;
    group = 2.f * s + SUBNORMAL;
  }
  // half an ulp of two values, of the magnitudes' sum or, doubled, of the larger one; infinities have none
  __device__ __forceinline__ static float rounding(float magnitude) { return ULP * fminf(magnitude, FLT_MAX); }
  // a >= b, and so they are for certain
  __device__ __forceinline__ bool settled(float a, float b) const { return a - b > expert + rounding(fmaxf(fabsf(a), fabsf(b))); }
};

__device__ __forceinline__ float warp_max(float x) { return key_float(__reduce_max_sync(ALL, float_key(x))); }
__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
  for (int off = 16; off; off >>= 1) x += __shfl_xor_sync(ALL, x, off);
  return x;
}

// INT_MAX: no expert, below all that there are
__device__ __forceinline__ bool above(double a, int ia, double b, int ib) { return a > b || (a == b && ia < ib) || (ib == INT_MAX && ia != INT_MAX); }
// sigmoid(l) over e^min(top, 0), top the largest l: what a row's sigmoids have in common is taken out, so that none leaves fp32's range
// while its share of the sum does not (logits of -50 and -95: 2.9e-20)
__device__ __forceinline__ float shifted_sigmoid(float l, float top) {
  if (l >= 0.f) return __fdividef(1.f, 1.f + expf(-l));
  return __fdividef(expf(l - fminf(top, 0.f)), 1.f + expf(l));
}

// One token in 64 bits, for the cases that fp32 leaves open.  bias: in shared memory, NULL: none.
struct RouteRow {
  const float* row;
  const float* bias;
  int E, log;   // a lane's experts are 2^log neighbours
  bool sigmoid;
  // Where an expert's bias lies: the lanes' first ones, their second ones, .. (as they come, 16 experts a lane were 16 lanes on a bank)
  __device__ __forceinline__ static int place(int e, int log) { return (e & ((1 << log) - 1)) << 5 | e >> log; }
};
// the softmax's largest logit and sum
__device__ __forceinline__ void row_sum64(const RouteRow& r, int lane, double& mx, double& den) {
  mx = -INFINITY;
  den = 0.0;
  if (r.sigmoid) return;
  for (int e = lane; e < r.E; e += 32) mx = fmax(mx, (double)r.row[e]);
#pragma unroll
  for (int off = 16; off; off >>= 1) mx = fmax(mx, __shfl_xor_sync(ALL, mx, off));
#pragma unroll 4
  for (int e = lane; e < r.E; e += 32) den += exp((double)r.row[e] - mx);
#pragma unroll
  for (int off = 16; off; off >>= 1) den += __shfl_xor_sync(ALL, den, off);
}
__device__ __forceinline__ double choice64(const RouteRow& r, int e, double mx, double den) {
  const double l = (double)r.row[e];
  double s = r.sigmoid ? 1.0 / (1.0 + exp(-l)) : exp(l - mx) / den;
  if (r.bias) s += (double)r.bias[RouteRow::place(e, r.log)];
  return l == -INFINITY ? -INFINITY : isnan(s) ? -DBL_MAX : s;
}

// The groups that stay, as bits.  c: the warp's [E] in shared memory, filled with all experts' c.
__device__ __noinline__ uint32_t exact_groups(RouteRow r, double* c, int n_groups, int top_groups, int group_top, int lane) {
  double mx, den;
  row_sum64(r, lane, mx, den);
  __syncwarp();
#pragma unroll 2
  for (int e = lane; e < r.E; e += 32) c[e] = choice64(r, e, mx, den);
  __syncwarp();
  if (top_groups >= n_groups) return ALL;
  const int gs = r.E / n_groups;
  int span = 32;
  while (span * n_groups > 32) span >>= 1;
  const int g = lane / span;
  double m1 = -INFINITY, m2 = -INFINITY;
  if (g < n_groups)
    for (int j = lane - g * span; j < gs; j += span) {
      const double x = c[g * gs + j];
      m2 = fmax(m2, fmin(m1, x));
      m1 = fmax(m1, x);
    }
  for (int off = span >> 1; off; off >>= 1) {
    const double o1 = __shfl_xor_sync(ALL, m1, off), o2 = __shfl_xor_sync(ALL, m2, off);
    m2 = fmax(fmin(m1, o1), fmax(m2, o2));
    m1 = fmax(m1, o1);
  }
  const double score = __shfl_sync(ALL, group_top == 2 ? m1 + m2 : m1, min(lane * span, 31));
  int rank = 0;
  for (int o = 0; o < n_groups; ++o) {
    const double x = __shfl_sync(ALL, score, o);
    rank += x > score || (x == score && o < lane) ? 1 : 0;
  }
  return __ballot_sync(ALL, lane < n_groups && rank < top_groups);
}

// The order of n <= 32 candidates, a lane each (id); lane j returns the j-th.  order: the warp's, 32 entries of shared memory.
__device__ __noinline__ int exact_order(RouteRow r, int id, int n, int* order, int lane) {
  double mx, den;
  row_sum64(r, lane, mx, den);
  const double c = lane < n ? choice64(r, id, mx, den) : 0.0;
  int rank = 0;
  for (int o = 0; o < n; ++o) {
    const double x = __shfl_sync(ALL, c, o);
    const int i = __shfl_sync(ALL, id, o);
    rank += x > c || (x == c && i < id) ? 1 : 0;
  }
  __syncwarp();
  if (lane < n) order[rank] = id;
  __syncwarp();
  return order[lane < n ? lane : 0];
}

// Everything: the groups, and the k largest of all their experts, round by round.
__device__ __noinline__ int exact_choice(RouteRow r, double* c, int k, int n_groups, int top_groups, int group_top, int lane) {
  const uint32_t kept = exact_groups(r, c, n_groups, top_groups, group_top, lane);
  const int gs = r.E / n_groups;
  uint32_t gone = 0;   // bit i: expert 32 i + lane is taken, or its group is left out
  for (int e = lane, i = 0; e < r.E; e += 32, ++i)
    if (!(kept >> (e / gs & 31) & 1)) gone |= 1u << i;
  int mine = 0;
  for (int j = 0; j < k; ++j) {
    double best = -INFINITY;
    int id = INT_MAX;
    for (int e = lane, i = 0; e < r.E; e += 32, ++i) {
      const double x = r.bias ? c[e] : isnan(r.row[e]) ? -DBL_MAX : (double)r.row[e];   // without a bias the logits' order
      if (!(gone >> i & 1) && above(x, e, best, id)) { best = x; id = e; }
    }
    for (int off = 16; off; off >>= 1) {
      const double ob = __shfl_xor_sync(ALL, best, off);
      const int oi = __shfl_xor_sync(ALL, id, off);
      if (above(ob, oi, best, id)) { best = ob; id = oi; }
    }
    if ((id & 31) == lane) gone |= 1u << (id >> 5);
    if (lane == j) mine = id;
  }
  return mine;
}

constexpr int ROUTE_POOL = 32;   // candidates of a token
template <int NPL>
constexpr int ROUTE_WARPS = NPL <= 8 ? 8 : 4;   // of a block: each has a row in 64 bits in shared memory
// Blocks on an SM: 64 registers a thread, 80 with 512 experts, 255 with 1024.  256 experts in 104 registers: a fifth more time for 65536
// tokens; 512 in 64 or 96: 4 to 9 us more for 16384.
template <int NPL>
constexpr int ROUTE_BLOCKS = NPL <= 8 ? 4 : NPL <= 16 ? 6 : 2;

// the two largest of two pairs, the larger first
__device__ __forceinline__ void top2(float& m1, float& m2, float o1, float o2) {
  m2 = fmaxf(fminf(m1, o1), fmaxf(m2, o2));
  m1 = fmaxf(m1, o1);
}

__device__ __forceinline__ void top2_add(float& m1, float& m2, float x) {
  m2 = fmaxf(m2, fminf(m1, x));
  m1 = fmaxf(m1, x);
}

// A lane has NPL experts: with WHOLE (E = 32 NPL) neighbours, so that a row is read in vectors and a group that is a power of two of lanes
// finds its score by shuffles; otherwise every 32nd, and groups are scanned in shared memory.
//
// What bounds it is instructions, 866 a token of 256 experts in 8 groups with a bias at 76 % of the issue slots (65536 tokens 68 us; 1150 with an IEEE
// division and expf for every expert, which the k chosen ones alone need, and a group found by dividing).  The rounds of a selection over
// all keys go over the lanes' largest; who reaches the last of these finds its rank among a dozen.
template <int NPL, bool WHOLE>
__global__ void __launch_bounds__(32 * ROUTE_WARPS<NPL>, ROUTE_BLOCKS<NPL>) route_groups_kernel(const RouteGroupsArgs a) {
  constexpr int WARPS = ROUTE_WARPS<NPL>;
  constexpr int LOG = !WHOLE ? 0 : NPL == 1 ? 0 : NPL == 2 ? 1 : NPL == 4 ? 2 : NPL == 8 ? 3 : NPL == 16 ? 4 : 5;   // of a lane's neighbours
  extern __shared__ double route_smem[];   // [WARPS][E] doubles, bias [E], counts [E]
  __shared__ uint64_t pool_all[WARPS][ROUTE_POOL];
  const int E = WHOLE ? 32 * NPL : a.E, k = a.k, G = a.n_groups, gs = E / G;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint64_t* pool = pool_all[warp];
  double* c64 = route_smem + (size_t)warp * E;
  float* c32 = reinterpret_cast<float*>(c64);
  float* sbias = reinterpret_cast<float*>(route_smem + (size_t)WARPS * E);
  int* hist = reinterpret_cast<int*>(sbias + E);
  const bool sigmoid = (a.mode & GATE_SIGMOID) != 0, renorm = (a.mode & GATE_RENORM) != 0, pick = a.top_groups < G;
  const bool scored = a.bias || (pick && a.group_top == 2);   // scores decide; otherwise the logits do
  const bool by_lanes = WHOLE && (G & (G - 1)) == 0;          // groups are 32 / G lanes
  auto expert = [&](int i) { return WHOLE ? lane * NPL + i : 32 * i + lane; };
  pdl_trigger();
  pdl_wait();
  for (int e = threadIdx.x; e < E; e += 32 * WARPS) {
    sbias[RouteRow::place(e, LOG)] = a.bias ? a.bias[e] : 0.f;
    hist[e] = 0;
  }
  __syncthreads();
  const int avail = a.top_groups * gs, want = min(k + 1, min(avail, 32));
  int span_log = 5;   // 2^span_log lanes scan a group together
  while (G << span_log > 32) --span_log;
  const int span = 1 << span_log;
  const uint32_t per_gs = ((1u << 20) + gs - 1) / gs;   // e / gs = e per_gs / 2^20, exact for e gs < 2^20
  float bias_reg[NPL <= 8 ? NPL : 1];
  if constexpr (NPL <= 8) {
#pragma unroll
    for (int i = 0; i < NPL; ++i) bias_reg[i] = WHOLE || expert(i) < E ? sbias[32 * i + lane] : 0.f;
  }
  auto bias_of = [&](int i) -> float {
    if constexpr (NPL <= 8) return bias_reg[i];
    else return WHOLE || expert(i) < E ? sbias[32 * i + lane] : 0.f;
  };

  const uint32_t below = (1u << lane) - 1u;

  for (int t = blockIdx.x * WARPS + warp; t < a.T; t += gridDim.x * WARPS) {
    const float* row = a.logits + (size_t)t * E;
    float v[NPL];
    if (WHOLE && NPL % 4 == 0 && a.vec) {
#pragma unroll
      for (int i = 0; i < NPL; i += 4) {
        const float4 x = reinterpret_cast<const float4*>(row + lane * NPL)[i / 4];
        v[i] = x.x; v[i + 1 < NPL ? i + 1 : 0] = x.y; v[i + 2 < NPL ? i + 2 : 0] = x.z; v[i + 3 < NPL ? i + 3 : 0] = x.w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < NPL; ++i) v[i] = WHOLE || expert(i) < E ? row[expert(i)] : -INFINITY;
    }
    float mx = -INFINITY, den = 0.f, s_max = 0.f;
    if (!sigmoid) {
#pragma unroll
      for (int i = 0; i < NPL; ++i) mx = fmaxf(mx, v[i]);
      mx = warp_max(mx);
    }
    bool open = false;   // the token goes through exact_choice
    const RouteRow exact{row, a.bias ? sbias : nullptr, E, LOG, sigmoid};
    if (scored) {
      // v becomes c
      if (sigmoid) {
#pragma unroll
        for (int i = 0; i < NPL; ++i) {
          const float s = rcp_approx(1.f + ex2_approx(-LOG2E * v[i]));
          s_max = fmaxf(s_max, s);
          v[i] = v[i] == -INFINITY ? -INFINITY : s + bias_of(i);
        }
        s_max = warp_max(s_max);
      } else {
        float ex[NPL], sum = 0.f;
#pragma unroll
        for (int i = 0; i < NPL; ++i) {
          ex[i] = WHOLE || expert(i) < E ? ex2_approx(LOG2E * (v[i] - mx)) : 0.f;
          sum += ex[i];
        }
        sum = warp_sum(sum);
        s_max = rcp_approx(sum);
#pragma unroll
        for (int i = 0; i < NPL; ++i)
          v[i] = v[i] == -INFINITY ? -INFINITY : ex[i] * s_max + bias_of(i);
      }
      // NaN among the scores; 32 experts have no lane left for the one behind them
      open = !(s_max <= FLT_MAX) || (a.bias && want <= k && avail > k);
    }
    const RouteTol tol(sigmoid, s_max);
    uint32_t kept = ALL;
    if (pick) {
      // `span` lanes a group: the two largest of their shares, then of one another's
      float m1 = -INFINITY, m2 = -INFINITY;
      if (by_lanes) {
        m1 = v[0];
#pragma unroll
        for (int i = 1; i < NPL; ++i) top2_add(m1, m2, v[i]);
      } else {
        __syncwarp();
#pragma unroll
        for (int i = 0; i < NPL; ++i)
          if (WHOLE || expert(i) < E) c32[expert(i)] = v[i];
        __syncwarp();
        const int g = lane >> span_log;
        if (g < G)
          for (int j = lane & (span - 1); j < gs; j += span) top2_add(m1, m2, c32[g * gs + j]);
      }
      for (int off = span >> 1; off; off >>= 1) top2(m1, m2, __shfl_xor_sync(ALL, m1, off), __shfl_xor_sync(ALL, m2, off));
      const int from = min(lane << span_log, 31);   // from here on lane g has group g
      const float score = __shfl_sync(ALL, a.group_top == 2 ? m1 + m2 : m1, from);
      int rank = 0;
      for (int o = 0; o < G; ++o) {
        const float x = __shfl_sync(ALL, score, o);
        rank += x > score || (x == score && o < lane) ? 1 : 0;
      }
      const bool stays = lane < G && rank < a.top_groups;
      kept = __ballot_sync(ALL, stays);
      if (scored) {
        // the least that a group that stays can have, and the most of one that does not
        const float off = RouteTol::rounding(__shfl_sync(ALL, fabsf(m1) + (a.group_top == 2 ? fabsf(m2) : 0.f), from));
        const float least = key_float(__reduce_min_sync(ALL, stays ? float_key(score - off) : ~0u));
        const float most = key_float(__reduce_max_sync(ALL, lane < G && !stays ? float_key(score + off) : 0u));
        if (!(least - most > tol.group)) kept = exact_groups(exact, c64, G, a.top_groups, a.group_top, lane);
      }
    }
    if (scored && !a.bias) {   // the experts' order is that of the logits, scores were for the groups
#pragma unroll
      for (int i = 0; i < NPL; ++i) v[i] = WHOLE || expert(i) < E ? row[expert(i)] : -INFINITY;
    }
    uint32_t key[NPL];
#pragma unroll
    for (int i = 0; i < NPL; ++i) key[i] = WHOLE || expert(i) < E ? float_key(v[i]) : 0u;
    if (pick) {
      if (by_lanes) {
        const bool in = kept >> (lane >> span_log) & 1;
#pragma unroll
        for (int i = 0; i < NPL; ++i) key[i] = in ? key[i] : 0u;
      } else {
#pragma unroll
        for (int i = 0; i < NPL; ++i) key[i] = kept >> (expert(i) * per_gs >> 20 & 31) & 1 ? key[i] : 0u;
      }
    }
    // a bound that the `want` largest reach and few others: the want-th largest of the lanes' largest
    uint32_t top = lane_max<NPL>(key), bound = 0;
#pragma unroll 1
    for (int j = 0; j < want; ++j) {
      bound = __reduce_max_sync(ALL, top);
      top = top == bound ? 0u : top;
    }
    bound = max(bound, 1u);
    int n = 0;
    __syncwarp();
#pragma unroll
    for (int i = 0; i < NPL; ++i) {
      const bool in = key[i] >= bound;
      const uint32_t all = __ballot_sync(ALL, in);
      const int at = n + __popc(all & below);
      if (in && at < ROUTE_POOL) pool[at] = ((uint64_t)key[i] << 32) | (uint32_t)~expert(i);
      n += __popc(all);
    }
    __syncwarp();
    int mine = 0;
    float val = 0.f;
    const bool few = n >= want && n <= ROUTE_POOL;
    if (few) {
      // each finds its rank among them
      const uint64_t w = lane < n ? pool[lane] : 0;
      int rank = 0;
#pragma unroll 4
      for (int c = 0; c < n; ++c) rank += pool[c] > w ? 1 : 0;
      __syncwarp();
      if (lane < n) pool[rank] = w;
      __syncwarp();
      const uint64_t r = pool[lane < n ? lane : 0];
      mine = (int)~(uint32_t)r;
      val = key_float((uint32_t)(r >> 32));
    } else {
      // many equal ones, or more wanted than lanes have any: round by round
#pragma unroll 1
      for (int j = 0; j < want; ++j) {
        const uint32_t best = __reduce_max_sync(ALL, lane_max<NPL>(key));
        int id = INT_MAX;
#pragma unroll
        for (int i = NPL - 1; i >= 0; --i) id = key[i] == best ? expert(i) : id;
        id = __reduce_min_sync(ALL, id);
#pragma unroll
        for (int i = 0; i < NPL; ++i) key[i] = expert(i) == id ? 0u : key[i];
        if (lane == j) { mine = id; val = key_float(best); }
      }
    }
    if (a.bias) {
      const float next = __shfl_down_sync(ALL, val, 1);
      if (__any_sync(ALL, lane + 1 < want && !tol.settled(val, next))) {
        // the candidates' order is enough where none of the others can be among the k
        const float least = __shfl_sync(ALL, val, k - 1);
        uint32_t rest = 0;
#pragma unroll
        for (int i = 0; i < NPL; ++i) rest = max(rest, key[i] < bound ? key[i] : 0u);
        rest = __reduce_max_sync(ALL, rest);
        if (few && (rest == 0u || tol.settled(least, key_float(rest)))) mine = exact_order(exact, mine, n, reinterpret_cast<int*>(pool), lane);
        else open = true;
      }
    }
    if (open) {
      __syncwarp();
      mine = exact_choice(exact, c64, k, G, a.top_groups, a.group_top, lane);
    }
    const bool on = lane < k;
    const float l = on ? row[mine] : -INFINITY;
    float w;
    if (renorm) {
      const float best = warp_max(l);
      const float e = on && l > -INFINITY ? (sigmoid ? shifted_sigmoid(l, best) : expf(l - best)) : 0.f;
      const float z = warp_sum(e);
      w = z > 0.f ? __fdividef(e, z) : z;   // no finite logit: 0
    } else if (sigmoid) {
      w = 1.f / (1.f + expf(-l));
    } else {
#pragma unroll
      for (int i = 0; i < NPL; ++i) den += WHOLE || expert(i) < E ? expf(row[expert(i)] - mx) : 0.f;
      den = warp_sum(den);
      w = mx == -INFINITY ? 0.f : expf(l - mx) / den;
    }
    if (on) {
      a.topk_ids[(size_t)t * k + lane] = mine;
      a.topk_w[(size_t)t * k + lane] = w * a.scale;
      if (a.counts) atomicAdd(&hist[mine], 1);
    }
  }
  if (a.counts) {
    __syncthreads();
    for (int e = threadIdx.x; e < E; e += 32 * WARPS)
      if (hist[e]) atomicAdd(&a.counts[e], hist[e]);
  }
}

template <int NPL, bool WHOLE>
static cudaError_t launch_groups(const RouteGroupsArgs& a, int num_sms, cudaStream_t s) {
  constexpr int WARPS = ROUTE_WARPS<NPL>;
  const size_t smem = (size_t)a.E * (8 * WARPS + 8);
  int per_sm = 1;
  cudaError_t e = blocks_per_sm<route_groups_kernel<NPL, WHOLE>>(32 * WARPS, (size_t)32 * NPL * (8 * WARPS + 8), &per_sm);
  if (e != cudaSuccess) return e;
  const long blocks = ((long)a.T + WARPS - 1) / WARPS, most = (long)per_sm * num_sms;
  return launch_dependent(route_groups_kernel<NPL, WHOLE>, dim3((unsigned)(blocks < most ? blocks : most)), dim3(32 * WARPS), smem, s, a);
}
template <int NPL>
static cudaError_t launch_groups(const RouteGroupsArgs& a, int num_sms, cudaStream_t s) {
  return a.E == 32 * NPL ? launch_groups<NPL, true>(a, num_sms, s) : launch_groups<NPL, false>(a, num_sms, s);
}

cudaError_t launch_route_groups(const RouteGroupsArgs& a, int num_sms, cudaStream_t s, int* launches) {
  if (a.counts) {
    cudaError_t e = cudaMemsetAsync(a.counts, 0, sizeof(int) * (size_t)a.E, s);
    if (e != cudaSuccess) return e;
  }
  if (a.T == 0) return cudaSuccess;
  ++*launches;
  const int npl = (a.E + 31) / 32;
  return npl <= 1 ? launch_groups<1>(a, num_sms, s) : npl <= 2 ? launch_groups<2>(a, num_sms, s) : npl <= 4 ? launch_groups<4>(a, num_sms, s)
       : npl <= 8 ? launch_groups<8>(a, num_sms, s) : npl <= 16 ? launch_groups<16>(a, num_sms, s) : launch_groups<32>(a, num_sms, s);
}

// ------------------------------------------------------------------------------------------
// Gradient of the weights.  g: the weights' gradients times scale, relative to the first one's where the weights are renormalised (what
// they have in common cancels).
//   renormalised, sigmoid:  d l_j = w_j (1 - s_j) (g_j - sum g w);  softmax: d l_j = w_j (g_j - sum g w)
//   as they are,  sigmoid:  d l_j = g_j s_j (1 - s_j);              softmax: d l_e = p_e ([e = e_j] g_j - sum g p), for all e
// Only the last needs all logits (DENSE, a warp a token); the others read k of them, and the pass is the write of the gradient: KP lanes
// a token, the power of two from k on, zeros ahead of everything that waits for a load.
// ------------------------------------------------------------------------------------------
template <int KP>
__device__ __forceinline__ float part_sum(float x) {
#pragma unroll
  for (int off = KP / 2; off; off >>= 1) x += __shfl_xor_sync(ALL, x, off);
  return x;
}
template <int KP>
__device__ __forceinline__ float part_max(float x) {
#pragma unroll
  for (int off = KP / 2; off; off >>= 1) x = fmaxf(x, __shfl_xor_sync(ALL, x, off));
  return x;
}

template <int KP, bool DENSE>
__global__ void __launch_bounds__(256) route_groups_bwd_kernel(const RouteGroupsBwdArgs a) {
  constexpr int TOKENS = 32 / KP;   // of a warp
  const int lane = threadIdx.x & 31, E = a.E, k = a.k, part = lane / KP, j = lane - part * KP;
  const long t0 = ((long)blockIdx.x * 8 + (threadIdx.x >> 5)) * TOKENS;
  pdl_trigger();
  pdl_wait();
  if (t0 >= a.T) return;
  const long t = t0 + part;
  const bool live = t < a.T && j < k;
  const int id = live ? a.topk_ids[t * k + j] : -1;
  float g = live ? a.d_topk_w[t * k + j] * a.scale : 0.f;
  if (!DENSE && !a.accumulate) {
    const int n = (int)min((long)TOKENS, a.T - t0) * E;
    float* first = a.d_logits + t0 * E;
    if (a.vec)
      for (int e = lane; e < n / 4; e += 32) reinterpret_cast<float4*>(first)[e] = make_float4(0.f, 0.f, 0.f, 0.f);
    else
      for (int e = lane; e < n; e += 32) first[e] = 0.f;
  }
  const float* row = a.logits + t * E;
  float* out = a.d_logits + t * E;
  const bool sigmoid = (a.mode & GATE_SIGMOID) != 0, renorm = (a.mode & GATE_RENORM) != 0;
  const bool have = id >= 0 && id < E;
  if (!have) g = 0.f;
  // the token's lanes; whether any has a gradient (NaN is not 0) -- without one its logits may hold anything
  const unsigned mask = (KP == 32 ? ALL : (1u << (KP & 31)) - 1u) << (part * KP);
  const bool any = __ballot_sync(ALL, g != 0.f) & mask;
  const unsigned has = __ballot_sync(ALL, have) & mask;
  const float l = have && any ? row[id] : -INFINITY;
  float d = 0.f;
  if (!DENSE) {
    if (renorm) {
      const float g0 = __shfl_sync(ALL, g, has ? __ffs(has) - 1 : lane);
      g = have ? g - g0 : 0.f;
      const float top = part_max<KP>(l);
      const bool fin = have && l > -INFINITY;
      const float e = fin ? (sigmoid ? shifted_sigmoid(l, top) : expf(l - top)) : 0.f;
      const float z = part_sum<KP>(have && isnan(l) ? l : e), w = z > 0.f ? e / z : z;
      const float dot = part_sum<KP>(have ? g * w : 0.f);
      d = any && have ? w * (g - dot) : 0.f;
      if (sigmoid && fin) d *= 1.f / (1.f + expf(l));
    } else {
      const float q = expf(-fabsf(l)), r = 1.f / (1.f + q);
      d = any && have && l != -INFINITY ? g * (q * r * r) : 0.f;
    }
  } else {
    float mx = -INFINITY, den = 0.f, dot = 0.f;
    if (any) {
      for (int e = lane; e < E; e += 32) mx = fmaxf(mx, row[e]);
      mx = warp_max(mx);
      if (mx > -INFINITY || isnan(mx)) {
        for (int e = lane; e < E; e += 32) den += expf(row[e] - mx);
        den = warp_sum(den);
        d = have ? g * (expf(l - mx) / den) : 0.f;
        dot = warp_sum(d);
      }
    }
    if (any || !a.accumulate)
      for (int e = lane; e < E; e += 32) {
        const float x = den != 0.f ? -(expf(row[e] - mx) / den) * dot : 0.f;
        out[e] = a.accumulate ? out[e] + x : x;
      }
  }
  // an expert that a token names more than once gets the sum, by its first lane
  const unsigned peers = __match_any_sync(ALL, have ? part * 1024 + id : -1 - lane);
  if (__any_sync(ALL, peers & (peers - 1))) {
    float sum = 0.f;
    for (int i = 0; i < 32; ++i) {
      const float o = __shfl_sync(ALL, d, i);
      sum += peers >> i & 1 ? o : 0.f;
    }
    d = sum;
  }
  __syncwarp();
  if (have && any && lane == __ffs(peers) - 1) out[id] = DENSE || a.accumulate ? out[id] + d : d;
}

template <int KP, bool DENSE>
static cudaError_t launch_groups_bwd(const RouteGroupsBwdArgs& a, cudaStream_t s) {
  constexpr int TOKENS = 8 * (32 / KP);
  return launch_dependent(route_groups_bwd_kernel<KP, DENSE>, dim3((unsigned)(((long)a.T + TOKENS - 1) / TOKENS)), dim3(256), 0, s, a);
}
cudaError_t launch_route_groups_bwd(const RouteGroupsBwdArgs& a, cudaStream_t s, int* launches) {
  if (a.T == 0) return cudaSuccess;
  ++*launches;
  if (!(a.mode & (GATE_SIGMOID | GATE_RENORM))) return launch_groups_bwd<32, true>(a, s);
  return a.k <= 4 ? launch_groups_bwd<4, false>(a, s) : a.k <= 8 ? launch_groups_bwd<8, false>(a, s) : a.k <= 16 ? launch_groups_bwd<16, false>(a, s)
                                                                                                          : launch_groups_bwd<32, false>(a, s);
}

// ------------------------------------------------------------------------------------------
// The bias of the next step: down for experts above the mean count, up for those below.  Whole numbers decide.
// ------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(1024) bias_update_kernel(const float* bias, const int* __restrict__ counts, int n_seq, int E, float rate, float* out) {
  __shared__ long long sums[32];
  const int e = threadIdx.x;
  pdl_trigger();
  pdl_wait();
  long long mine = 0;
  if (e < E)
    for (int s = 0; s < n_seq; ++s) mine += counts[(size_t)s * E + e];
  long long all = mine;
#pragma unroll
  for (int off = 16; off; off >>= 1) all += __shfl_xor_sync(ALL, all, off);
  if ((e & 31) == 0) sums[e >> 5] = all;
  __syncthreads();
  all = 0;
  for (int w = 0; w < (int)blockDim.x / 32; ++w) all += sums[w];
  if (e < E) {
    const long long over = (long long)E * mine;
    out[e] = bias[e] + (all > over ? rate : all < over ? -rate : 0.f);
  }
}

cudaError_t launch_bias_update(const float* bias, const int* counts, int n_seq, int E, float rate, float* out, cudaStream_t s, int* launches) {
  ++*launches;
  return launch_dependent(bias_update_kernel, dim3(1), dim3((E + 31) / 32 * 32), 0, s, bias, counts, n_seq, E, rate, out);
}

}  // namespace moe
