// Routing by groups of experts with a bias for balance (moe_route_grouped), the gradient of its weights, and the bias' update.
//
//   s_e = sigmoid(l_e) or softmax(l)_e, c_e = s_e + b_e; a group's score is the sum of its one or two largest c; the top_groups
//   groups of the largest scores stay, of their experts the k of the largest c; w = s (of the k over their sum), times scale.
//
// Which experts come out must not hang on a rounding: c is compared as it is in 64 bits, ties go to the lower index.  A warp has a
// token.  It selects in fp32 and looks whether the selection is beyond doubt -- every two neighbours in the order of the k + 1
// largest, and the last group kept and the first one left out, further apart than fp32 can have moved them (RouteTol) -- and
// does the token again in 64 bits where it is not: one token in a thousand of normally distributed logits, all that have ties.
// Without a bias the experts' order is that of the logits, whose comparison is exact.
#include <float.h>
#include <limits.h>

#include "launch_pairs.cuh"
#include "moe_internal.h"
#include "topk.cuh"

namespace moe {

constexpr unsigned ALL = 0xffffffffu;

// How far apart two c, or two groups' scores, are for certain in the order that fp32 gives them.  An fp32 sigmoid is off by
// 2 ulp of expf, the addition and the division: 3 x 2^-23 of itself; a softmax score by 2 ulp of expf, its argument's rounding (at most
// 2^-25 of the score's largest value), and a sum of up to 1024 terms along 37 additions: under 2^-18 of itself.  The bias adds half
// an ulp of c, a group's sum the errors of both and half an ulp.  Doubled, since two values are compared, and rounded up.
struct RouteTol {
  float expert, group;
  __device__ RouteTol(bool sigmoid, float s_max, float b_max) {
    const float s = s_max * (sigmoid ? 9.5367432e-7f /* 2^-20 */ : 7.6293945e-6f /* 2^-17 */), c = (s_max + b_max) * 1.1920929e-7f /* 2^-23 */;
    constexpr float SUBNORMAL = 1e-37f;   // numbers below 2^-126 have steps of their own
    expert = s + c + SUBNORMAL;
    group = 2.f * (s + c) + 2.f * c + SUBNORMAL;
  }
};

__device__ __forceinline__ float warp_max(float x) { return key_float(__reduce_max_sync(ALL, float_key(x))); }
__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
  for (int off = 16; off; off >>= 1) x += __shfl_xor_sync(ALL, x, off);
  return x;
}

// INT_MAX: no expert, below all that there are
__device__ __forceinline__ bool above(double a, int ia, double b, int ib) { return a > b || (a == b && ia < ib) || (ib == INT_MAX && ia != INT_MAX); }
// e^-m sigmoid(l) with m = min(the largest l, 0): what the sigmoids of rows of large negative logits have in common is taken out
__device__ __forceinline__ float shifted_sigmoid(float l, float top) {
  const float m = fminf(top, 0.f);
  return 1.f / (expf(m - l) + expf(m));
}

// The selection of one token in 64 bits; lane j < k returns the j-th expert.  c: the warp's [E] in shared memory.
__device__ __noinline__ int route_exact(const RouteGroupsArgs& a, const float* row, const float* bias, double* c, int lane) {
  const int E = a.E, gs = E / a.n_groups;
  double mx = -INFINITY, den = 0.0;
  if (!(a.mode & GATE_SIGMOID)) {
    for (int e = lane; e < E; e += 32) mx = fmax(mx, (double)row[e]);
    for (int off = 16; off; off >>= 1) mx = fmax(mx, __shfl_xor_sync(ALL, mx, off));
    for (int e = lane; e < E; e += 32) den += exp((double)row[e] - mx);
    for (int off = 16; off; off >>= 1) den += __shfl_xor_sync(ALL, den, off);
  }
  for (int e = lane; e < E; e += 32) {
    const double l = (double)row[e];
    double s = (a.mode & GATE_SIGMOID) ? 1.0 / (1.0 + exp(-l)) : exp(l - mx) / den;
    if (bias) s += (double)bias[e];
    c[e] = l == -INFINITY ? -INFINITY : isnan(s) ? -DBL_MAX : s;
  }
  __syncwarp();
  uint32_t kept = ALL;   // groups
  if (a.top_groups < a.n_groups) {
    double m1 = -INFINITY, m2 = -INFINITY;
    if (lane < a.n_groups)
      for (int j = 0; j < gs; ++j) {
        const double x = c[lane * gs + j];
        m2 = fmax(m2, fmin(m1, x));
        m1 = fmax(m1, x);
      }
    const double score = a.group_top == 2 ? m1 + m2 : m1;
    int rank = 0;
    for (int g = 0; g < a.n_groups; ++g) {
      const double o = __shfl_sync(ALL, score, g);
      rank += o > score || (o == score && g < lane) ? 1 : 0;
    }
    kept = __ballot_sync(ALL, lane < a.n_groups && rank < a.top_groups);
  }
  uint32_t gone = 0;   // bit i: expert 32 i + lane is taken, or its group is left out
  for (int e = lane, i = 0; e < E; e += 32, ++i)
    if (!(kept >> (e / gs) & 1)) gone |= 1u << i;
  int mine = 0;
  for (int j = 0; j < a.k; ++j) {
    double best = -INFINITY;
    int id = INT_MAX;
    for (int e = lane, i = 0; e < E; e += 32, ++i) {
      const double x = a.bias ? c[e] : isnan(row[e]) ? -DBL_MAX : (double)row[e];
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

template <int NPL>
constexpr int ROUTE_WARPS = NPL <= 8 ? 8 : 4;   // of a block: each has a row in 64 bits in shared memory

template <int NPL>
__global__ void __launch_bounds__(32 * ROUTE_WARPS<NPL>) route_groups_kernel(const RouteGroupsArgs a) {
  constexpr int WARPS = ROUTE_WARPS<NPL>;
  extern __shared__ double route_smem[];   // [WARPS][E] doubles, bias [E], counts [E]
  __shared__ uint64_t pool[WARPS][TOPK_POOL];
  const int E = a.E, k = a.k, G = a.n_groups, gs = E / G;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  double* c64 = route_smem + (size_t)warp * E;
  float* c32 = reinterpret_cast<float*>(c64);
  float* sbias = reinterpret_cast<float*>(route_smem + (size_t)WARPS * E);
  int* hist = reinterpret_cast<int*>(sbias + E);
  const bool sigmoid = (a.mode & GATE_SIGMOID) != 0, pick = a.top_groups < G;
  const bool scored = a.bias || (pick && a.group_top == 2);   // scores decide; otherwise the logits do
  pdl_trigger();
  pdl_wait();
  for (int e = threadIdx.x; e < E; e += 32 * WARPS) {
    sbias[e] = a.bias ? a.bias[e] : 0.f;
    hist[e] = 0;
  }
  __syncthreads();
  float b[NPL], b_max = 0.f;
  int group[NPL];
#pragma unroll
  for (int i = 0; i < NPL; ++i) {
    const int e = 32 * i + lane;
    b[i] = e < E ? sbias[e] : 0.f;
    group[i] = e / gs;
    b_max = fmaxf(b_max, fabsf(b[i]));
  }
  b_max = warp_max(b_max);
  const int avail = a.top_groups * gs, want = min(k + 1, min(avail, 32));
  int span = 32;   // lanes that scan a group together
  while (span * G > 32) span >>= 1;

  for (int t = blockIdx.x * WARPS + warp; t < a.T; t += gridDim.x * WARPS) {
    const float* row = a.logits + (size_t)t * E;
    float v[NPL], c[NPL];
#pragma unroll
    for (int i = 0; i < NPL; ++i) v[i] = 32 * i + lane < E ? row[32 * i + lane] : -INFINITY;
    float mx = -INFINITY, den = 0.f, s_max = 0.f;
    if (!sigmoid) {
#pragma unroll
      for (int i = 0; i < NPL; ++i) mx = fmaxf(mx, v[i]);
      mx = warp_max(mx);
#pragma unroll
      for (int i = 0; i < NPL; ++i) {
        c[i] = 32 * i + lane < E ? expf(v[i] - mx) : 0.f;
        den += c[i];
      }
      den = warp_sum(den);
      s_max = 1.f / den;
    }
    if (scored) {
      const float inv = s_max;
#pragma unroll
      for (int i = 0; i < NPL; ++i) {
        const float s = sigmoid ? 1.f / (1.f + expf(-v[i])) : c[i] * inv;
        if (sigmoid) s_max = fmaxf(s_max, s);
        c[i] = v[i] == -INFINITY ? -INFINITY : s + b[i];
      }
      if (sigmoid) s_max = warp_max(s_max);
    } else {
#pragma unroll
      for (int i = 0; i < NPL; ++i) c[i] = v[i];
    }
    const RouteTol tol(sigmoid, s_max, b_max);
    // NaN among the scores; 32 experts have no lane left for the one behind them
    bool doubt = scored && (!(s_max <= FLT_MAX) || (a.bias && want <= k && avail > k));
    uint32_t kept = ALL;
    if (pick) {
      __syncwarp();
#pragma unroll
      for (int i = 0; i < NPL; ++i)
        if (32 * i + lane < E) c32[32 * i + lane] = c[i];
      __syncwarp();
      // `span` lanes a group: the two largest of their shares, then of one another's
      const int g = lane / span;
      float m1 = -INFINITY, m2 = -INFINITY;
      if (g < G)
        for (int j = lane - g * span; j < gs; j += span) {
          const float x = c32[g * gs + j];
          m2 = fmaxf(m2, fminf(m1, x));
          m1 = fmaxf(m1, x);
        }
      for (int off = span >> 1; off; off >>= 1) {
        const float o1 = __shfl_xor_sync(ALL, m1, off), o2 = __shfl_xor_sync(ALL, m2, off);
        m2 = fmaxf(fmaxf(m2, o2), fminf(m1, o1));
        m1 = fmaxf(m1, o1);
      }
      // from here on lane g has group g
      const float sum = a.group_top == 2 ? m1 + m2 : m1;
      const float score = __shfl_sync(ALL, sum, min(lane * span, 31));
      int rank = 0;
      for (int o = 0; o < G; ++o) {
        const float x = __shfl_sync(ALL, score, o);
        rank += x > score || (x == score && o < lane) ? 1 : 0;
      }
      const bool in = lane < G && rank < a.top_groups;
      kept = __ballot_sync(ALL, in);
      if (scored) {
        const float low = -warp_max(in ? -score : -INFINITY), high = warp_max(lane < G && !in ? score : -INFINITY);
        doubt |= !(low - high > tol.group);
      }
    }
    uint32_t key[1][NPL];
#pragma unroll
    for (int i = 0; i < NPL; ++i)
      key[0][i] = 32 * i + lane < E && (kept >> (group[i] & 31) & 1) ? float_key(a.bias ? c[i] : v[i]) : 0u;
    int id[1] = {0};
    float val[1] = {0.f};
    warp_topk<NPL, 1>(key, want, lane, pool[warp], id, val);
    if (a.bias) {
      const float next = __shfl_down_sync(ALL, val[0], 1);
      doubt |= lane + 1 < want && !(val[0] - next > tol.expert);
    }
    int mine = id[0];
    if (__any_sync(ALL, doubt)) {
      __syncwarp();
      mine = route_exact(a, row, a.bias ? sbias : nullptr, c64, lane);
      __syncwarp();
    }
    const bool on = lane < k;
    const float l = on ? row[mine] : -INFINITY;
    float w;
    if (a.mode & GATE_RENORM) {
      const float top = warp_max(l);
      const float e = on && l > -INFINITY ? (sigmoid ? shifted_sigmoid(l, top) : expf(l - top)) : 0.f;
      const float z = warp_sum(e);
      w = z > 0.f ? e / z : z;   // no finite logit: 0
    } else {
      w = sigmoid ? 1.f / (1.f + expf(-l)) : mx == -INFINITY ? 0.f : expf(l - mx) / den;
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

template <int NPL>
static cudaError_t launch_groups(const RouteGroupsArgs& a, int num_sms, cudaStream_t s) {
  constexpr int WARPS = ROUTE_WARPS<NPL>;
  const size_t smem = (size_t)a.E * (8 * WARPS + 8);
  int per_sm = 1;
  cudaError_t e = blocks_per_sm<route_groups_kernel<NPL>>(32 * WARPS, (size_t)32 * NPL * (8 * WARPS + 8), &per_sm);
  if (e != cudaSuccess) return e;
  const long blocks = ((long)a.T + WARPS - 1) / WARPS, most = (long)per_sm * num_sms;
  return launch_dependent(route_groups_kernel<NPL>, dim3((unsigned)(blocks < most ? blocks : most)), dim3(32 * WARPS), smem, s, a);
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
// Gradient of the weights, one warp a token.  g: the weights' gradients times scale, relative to the first one's where the weights are
// renormalised (what they have in common cancels).
//   renormalised, sigmoid:  d l_j = w_j (1 - s_j) (g_j - sum g w);  softmax: d l_j = w_j (g_j - sum g w)
//   as they are,  sigmoid:  d l_j = g_j s_j (1 - s_j);              softmax: d l_e = p_e ([e = e_j] g_j - sum g p), for all e
// Only the last needs all logits; the others read k of them, and the pass is the write of the gradient.
// ------------------------------------------------------------------------------------------
template <bool DENSE>
__global__ void __launch_bounds__(256) route_groups_bwd_kernel(const RouteGroupsBwdArgs a) {
  const int lane = threadIdx.x & 31, E = a.E, k = a.k;
  const int t = blockIdx.x * 8 + (threadIdx.x >> 5);
  pdl_trigger();
  pdl_wait();
  if (t >= a.T) return;
  const float* row = a.logits + (size_t)t * E;
  float* out = a.d_logits + (size_t)t * E;
  const bool sigmoid = (a.mode & GATE_SIGMOID) != 0, renorm = (a.mode & GATE_RENORM) != 0;
  const int id = lane < k ? a.topk_ids[(size_t)t * k + lane] : -1;
  const bool have = id >= 0 && id < E;
  float g = have ? a.d_topk_w[(size_t)t * k + lane] * a.scale : 0.f;
  const bool any = __any_sync(ALL, g != 0.f);   // (NaN is not 0)
  float d = 0.f, dot = 0.f, mx = -INFINITY, den = 0.f;
  if (any) {
    const float l = have ? row[id] : -INFINITY;
    if (renorm) {
      const unsigned first = __ffs(__ballot_sync(ALL, have)) - 1;
      const float g0 = __shfl_sync(ALL, g, first);
      g = have ? g - g0 : 0.f;
      const float top = warp_max(l);
      const bool fin = have && l > -INFINITY;
      const float e = fin ? (sigmoid ? shifted_sigmoid(l, top) : expf(l - top)) : 0.f;
      const float z = warp_sum(e), w = z > 0.f ? e / z : z;
      dot = warp_sum(have ? g * w : 0.f);
      d = w * (g - dot);
      if (sigmoid && fin) d *= 1.f / (1.f + expf(l));
    } else if (sigmoid) {
      const float q = expf(-fabsf(l)), r = 1.f / (1.f + q);
      d = have && l > -INFINITY ? g * (q * r * r) : 0.f;
    } else {
      for (int e = lane; e < E; e += 32) mx = fmaxf(mx, row[e]);
      mx = warp_max(mx);
      if (mx > -INFINITY || isnan(mx)) {
        for (int e = lane; e < E; e += 32) den += expf(row[e] - mx);
        den = warp_sum(den);
        d = have ? g * (expf(l - mx) / den) : 0.f;
        dot = warp_sum(d);
      }
    }
    // an expert named more than once gets the sum
    const unsigned peers = __match_any_sync(ALL, have ? id : -1 - lane);
    if (__any_sync(ALL, peers & (peers - 1))) {
      float all = 0.f;
      for (int j = 0; j < k; ++j) {
        const float o = __shfl_sync(ALL, d, j);
        all += peers >> j & 1 ? o : 0.f;
      }
      d = all;
    }
    if (DENSE) {
      const bool some = den != 0.f;
      for (int e = lane; e < E; e += 32) {
        const float x = some ? -(expf(row[e] - mx) / den) * dot : 0.f;
        out[e] = a.accumulate ? out[e] + x : x;
      }
      __syncwarp();
      if (have && lane == __ffs(peers) - 1) out[id] += d;
      return;
    }
    if (a.accumulate) {
      if (have && lane == __ffs(peers) - 1) out[id] += d;
      return;
    }
  } else if (a.accumulate) {
    return;
  }
  if (a.vec)
    for (int e = lane; e < E / 4; e += 32) reinterpret_cast<float4*>(out)[e] = make_float4(0.f, 0.f, 0.f, 0.f);
  else
    for (int e = lane; e < E; e += 32) out[e] = 0.f;
  __syncwarp();
  if (any && have) out[id] = d;
}

cudaError_t launch_route_groups_bwd(const RouteGroupsBwdArgs& a, cudaStream_t s, int* launches) {
  if (a.T == 0) return cudaSuccess;
  ++*launches;
  const dim3 grid((unsigned)(((long)a.T + 7) / 8));
  return a.mode & (GATE_SIGMOID | GATE_RENORM) ? launch_dependent(route_groups_bwd_kernel<false>, grid, dim3(256), 0, s, a)
                                               : launch_dependent(route_groups_bwd_kernel<true>, grid, dim3(256), 0, s, a);
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
