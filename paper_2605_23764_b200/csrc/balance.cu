// The router's balance losses with their gradient, and the per-expert counts they need.
//
//   p[t,e]   = softmax(l[t])_e, or sigmoid(l[t,e]) / sum_e' sigmoid(l[t,e']) in the sigmoid gate mode
//   balance  = 1/n_seq sum_s E/(k n_s) sum_e c[s,e] P[s,e]        c: slots that name e, P: mean of p over the sequence's n_s tokens
//   z        = 1/N sum_t logsumexp(l[t])^2                        over the N tokens of all sequences
//   d balance / d p[t,e] = E c[s,e] / (k n_s^2 n_seq) =: x_e;     d balance / d l = p (x - sum p x)     (sigmoid: times 1 - sigmoid)
//   d z / d l = 2/N logsumexp softmax
// The backward adds the gradient of the routing scores (router.cu has its formulas), so that one pass over the logits gives
// their whole gradient.
//
// A group of LPT lanes holds a token's logits, VPL of them a lane, so that a token costs log2(LPT) shuffles a reduction and few
// experts still fill the warp (8 experts: 32 tokens a warp).  Every warp has a range of consecutive tokens and walks its runs --
// stretches of one sequence.
#include <type_traits>

#include "launch_pairs.cuh"
#include "moe_internal.h"
#include "topk.cuh"

namespace moe {

namespace {

constexpr int BAL_MAX_WARPS = 16;

__device__ __forceinline__ float group_sum(float v, int lpt) {
  for (int off = lpt >> 1; off; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
  return v;
}
__device__ __forceinline__ float group_max(float v, int lpt) {
  for (int off = lpt >> 1; off; off >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, off));
  return v;
}

// First token of sequence s (s = n: one behind the last).  Offsets are the caller's: kept inside the batch.
__device__ __forceinline__ int seq_begin(const int* off, int s, int T) {
  if (!off) return s ? T : 0;
  return min(max(__ldg(off + s), 0), T);
}
// Sequence of token t: -1 in front of the first one, n behind the last.  A warp's 32 probes a round, where a lane's bisection
// would be a chain of dependent reads.
__device__ __forceinline__ int seq_of(const int* off, int n, int T, int t, int lane) {
  if (!off) return 0;
  int lo = 0, len = n + 1;
  while (len > 32) {
    const int step = (len + 31) >> 5;
    const int i = lane * step;
    const int c = __popc(__ballot_sync(0xffffffffu, i < len && seq_begin(off, lo + i, T) <= t));
    if (c == 0) return lo - 1;
    const int at = (c - 1) * step;
    lo += at;
    len = min(step, len - at);
  }
  return lo - 1 + __popc(__ballot_sync(0xffffffffu, lane < len && seq_begin(off, lo + lane, T) <= t));
}

// Value i of lane l of a group stands for expert ((i / VW) LPT + l) VW + i % VW: vectors of VW lie side by side.
template <int LPT, int VW>
__device__ __forceinline__ int expert_at(int i, int l) { return ((i / VW) * LPT + l) * VW + i % VW; }

template <int LPT, int VPL, int VW>
__device__ __forceinline__ void load_row(const float* row, int E, int l, bool on, float (&v)[VPL]) {
#pragma unroll
  for (int i = 0; i < VPL; i += VW) {
    const int e = expert_at<LPT, VW>(i, l);
    if (VW == 4) {
      float4 q = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
      if (on && e < E) q = __ldcs(reinterpret_cast<const float4*>(row + e));
      v[i] = q.x; v[i + 1] = q.y; v[i + 2] = q.z; v[i + 3] = q.w;
    } else {
      v[i] = on && e < E ? __ldcs(row + e) : -INFINITY;
    }
  }
}

// Softmax of a row and its logsumexp.  A row without a finite logit has no probabilities: zeros, and logsumexp counts as 0.
template <int LPT, int VPL>
__device__ __forceinline__ float softmax_row(const float (&v)[VPL], float (&p)[VPL]) {
  float m = v[0];
#pragma unroll
  for (int i = 1; i < VPL; ++i) m = fmaxf(m, v[i]);
  m = group_max(m, LPT);
  if (m == -INFINITY) m = 0.f;
  float den = 0.f;
#pragma unroll
  for (int i = 0; i < VPL; ++i) { p[i] = __expf(v[i] - m); den += p[i]; }
  den = group_sum(den, LPT);
  const float r = den == 0.f ? 0.f : 1.0f / den;
#pragma unroll
  for (int i = 0; i < VPL; ++i) p[i] *= r;
  return den == 0.f ? 0.f : m + logf(den);
}
// Normalised sigmoids; s: the sigmoids themselves (NULL: not wanted).  Below zero sigmoid(l) = exp(l) / (1 + exp(l)), so a row of
// large negative logits is scaled by its largest as a softmax is, and keeps its proportions where every sigmoid underflows.
template <int LPT, int VPL>
__device__ __forceinline__ void sigmoid_row(const float (&v)[VPL], float (&p)[VPL], float* s) {
  float m = v[0];
#pragma unroll
  for (int i = 1; i < VPL; ++i) m = fmaxf(m, v[i]);
  m = fminf(group_max(m, LPT), 0.f);
  const bool low = m < -16.f && m > -INFINITY;
  float den = 0.f;
#pragma unroll
  for (int i = 0; i < VPL; ++i) {
    const float t = __expf(-fabsf(v[i])), sig = v[i] >= 0.f ? 1.0f / (1.0f + t) : t / (1.0f + t);
    if (s) s[i] = sig;
    p[i] = low ? __expf(v[i] - m) / (1.0f + t) : sig;
    den += p[i];
  }
  den = group_sum(den, LPT);
  const float r = den == 0.f ? 0.f : 1.0f / den;
#pragma unroll
  for (int i = 0; i < VPL; ++i) p[i] *= r;
}

}  // namespace

// ------------------------------------------------------------------------------------------
// Forward.  What a warp sums over a run that lies wholly in its range is final.  A run that reaches beyond it leaves a piece: the
// warps' pieces of a block are joined in order in shared memory, the blocks' in order by the block that arrives last.  Sums
// are therefore the same from call to call.
//
// Bound by the read of the logits, at few tokens by the latencies of launch, join and last block.
// ------------------------------------------------------------------------------------------
// A piece in global memory, two a block: of the sequence that began before the block, of the one that goes on behind it.
// [block][2] x {float psum[E]; int count[E]}, then per block {seq of both pieces, tokens of both, loss, z, tokens}
struct BalBlock { int seq[2], n[2]; double loss, z; long long tokens; };

template <int LPT, int VPL, int VW, bool SIG>
__global__ void __launch_bounds__(32 * BAL_MAX_WARPS) balance_fwd_kernel(const BalanceArgs a) {
  constexpr int TPW = 32 / LPT;
  extern __shared__ __align__(16) int bsm[];
  __shared__ int w_seq[2 * BAL_MAX_WARPS], w_n[2 * BAL_MAX_WARPS];
  __shared__ double s_loss[BAL_MAX_WARPS], s_z[BAL_MAX_WARPS];
  __shared__ long long s_tok[BAL_MAX_WARPS];
  __shared__ int s_last;
  const int E = a.E, n = a.n_seq, T = a.T;
  const int warps = blockDim.x >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, l = lane % LPT, grp = lane / LPT;
  int* const hist = bsm + warp * E;                                   // [warps][E]
  float* const w_sum = reinterpret_cast<float*>(bsm + warps * E);     // [warps][2][E]
  int* const w_cnt = bsm + 3 * warps * E;                             // [warps][2][E]
  for (int e = lane; e < E; e += 32) hist[e] = 0;
  if (lane < 2) w_seq[2 * warp + lane] = -1;
  __syncwarp();
  pdl_wait();
  pdl_trigger();

  const int b0 = (int)((long long)T * blockIdx.x / gridDim.x), b1 = (int)((long long)T * (blockIdx.x + 1) / gridDim.x);
  const int wa = b0 + (int)((long long)(b1 - b0) * warp / warps), wb = b0 + (int)((long long)(b1 - b0) * (warp + 1) / warps);
  const float unit = (float)E / ((float)a.k * (float)n);
  double loss = 0.0, zsum = 0.0;
  long long tokens = 0;
  int s = wa < wb ? seq_of(a.seq_offsets, n, T, wa, lane) : n;
  for (int t = wa; t < wb;) {
    // the run [t, end) of sequence s
    const int begins = s >= 0 && s < n ? seq_begin(a.seq_offsets, s, T) : 0;
    int stop = s < n ? seq_begin(a.seq_offsets, s + 1, T) : T;
    if (stop <= t) stop = t + 1;   // (offsets that do not ascend)
    const int end = min(stop, wb);
    if (s >= 0 && s < n) {
      float acc[VPL];
#pragma unroll
      for (int i = 0; i < VPL; ++i) acc[i] = 0.f;
      float z = 0.f;
      int live = 0;
      // a token's row, mask and first id of the lane are read a round ahead
      float v[VPL], next[VPL];
      int next_id = -1;
      bool next_on = false;
      auto fetch = [&](int tt) {
        load_row<LPT, VPL, VW>(a.logits + (size_t)tt * E, E, l, tt < end, next);
        next_on = tt < end && (!a.token_mask || a.token_mask[tt] != 0);
        next_id = tt < end && l < a.k ? a.topk_ids[(size_t)tt * a.k + l] : -1;
      };
      fetch(t + grp);
#pragma unroll 1
      for (int t0 = t; t0 < end; t0 += TPW) {
        const int tt = t0 + grp;
#pragma unroll
        for (int i = 0; i < VPL; ++i) v[i] = next[i];
        const bool on = next_on;
        const int id = next_id;
        fetch(tt + TPW);
        if (on) {
          if (id >= 0 && id < E) atomicAdd(&hist[id], 1);
          for (int j = l + LPT; j < a.k; j += LPT) {
            const int e = a.topk_ids[(size_t)tt * a.k + j];
            if (e >= 0 && e < E) atomicAdd(&hist[e], 1);
          }
        }
        float p[VPL];
        const float lse = softmax_row<LPT, VPL>(v, p);
        if (SIG) sigmoid_row<LPT, VPL>(v, p, nullptr);
        if (on) {
#pragma unroll
          for (int i = 0; i < VPL; ++i) acc[i] += p[i];
          if (l == 0) { z = fmaf(lse, lse, z); ++live; }
        }
      }
      // the groups of the warp
#pragma unroll
      for (int off = LPT; off < 32; off <<= 1) {
#pragma unroll
        for (int i = 0; i < VPL; ++i) acc[i] += __shfl_xor_sync(0xffffffffu, acc[i], off);
      }
      z = group_sum(z, 32);
      live = __reduce_add_sync(0xffffffffu, live);
      zsum += z;
      tokens += live;
      __syncwarp();
      const bool whole = begins >= wa && stop <= wb;
      const int piece = t == wa ? 0 : 1;
      if (!whole && lane == 0) { w_seq[2 * warp + piece] = s; w_n[2 * warp + piece] = live; }
      const float inv = live ? 1.0f / (float)live : 0.f;
      float dot = 0.f;
      if (grp == 0) {
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
          const int e = expert_at<LPT, VW>(i, l);
          if (e < E) {
            const int c = hist[e];
            hist[e] = 0;
            if (whole) {
              a.counts[(size_t)s * E + e] = c;
              a.prob[(size_t)s * E + e] = acc[i] * inv;
              dot = fmaf((float)c * inv, acc[i] * inv, dot);
            } else {
              w_sum[(2 * warp + piece) * E + e] = acc[i];
              w_cnt[(2 * warp + piece) * E + e] = c;
            }
          }
        }
      }
      if (whole) {
        loss += (double)(unit * group_sum(dot, 32));
        if (lane == 0) a.tokens[s] = live;
      }
      __syncwarp();
    }
    t = end;
    if (t < wb) s = seq_of(a.seq_offsets, n, T, t, lane);
  }
  if (lane == 0) { s_loss[warp] = loss; s_z[warp] = zsum; s_tok[warp] = tokens; }
  // sequences without tokens belong to no warp's range
  for (int q = blockIdx.x * warps + warp; q < n; q += gridDim.x * warps)
    if (seq_begin(a.seq_offsets, q, T) >= seq_begin(a.seq_offsets, q + 1, T)) {
      for (int e = lane; e < E; e += 32) {
        a.counts[(size_t)q * E + e] = 0;
        a.prob[(size_t)q * E + e] = 0.f;
      }
      if (lane == 0) a.tokens[q] = 0;
    }
  __syncthreads();

  // ---- the warps' pieces in order: every thread has its experts
  const size_t slot_ints = 2 * (size_t)E;
  BalBlock* const meta = reinterpret_cast<BalBlock*>(a.scratch);
  float* const slots = reinterpret_cast<float*>(meta + gridDim.x);   // [block][2][psum | count]
  double my_loss = 0.0;
  if (threadIdx.x == 0) {
    BalBlock m{{-1, -1}, {0, 0}, 0.0, 0.0, 0};
    for (int w = 0; w < warps; ++w) { m.loss += s_loss[w]; m.z += s_z[w]; m.tokens += s_tok[w]; }
    int q = 0;
    while (q < 2 * warps) {
      if (w_seq[q] < 0) { ++q; continue; }
      const int sq = w_seq[q];
      int live = 0;
      while (q < 2 * warps && (w_seq[q] < 0 || w_seq[q] == sq)) { if (w_seq[q] == sq) live += w_n[q]; ++q; }
      const int begins = seq_begin(a.seq_offsets, sq, T), stop = seq_begin(a.seq_offsets, sq + 1, T);
      if (begins >= b0 && stop <= b1) a.tokens[sq] = live;
      else { const int h = begins < b0 ? 0 : 1; m.seq[h] = sq; m.n[h] = live; }
    }
    meta[blockIdx.x] = m;
  }
  for (int e = threadIdx.x; e < E; e += blockDim.x) {
    int q = 0;
    while (q < 2 * warps) {
      if (w_seq[q] < 0) { ++q; continue; }
      const int sq = w_seq[q];
      float sum = 0.f;
      int cnt = 0, live = 0;
      while (q < 2 * warps && (w_seq[q] < 0 || w_seq[q] == sq)) {
        if (w_seq[q] == sq) { sum += w_sum[q * E + e]; cnt += w_cnt[q * E + e]; live += w_n[q]; }
        ++q;
      }
      const int begins = seq_begin(a.seq_offsets, sq, T), stop = seq_begin(a.seq_offsets, sq + 1, T);
      if (begins >= b0 && stop <= b1) {
        const float inv = live ? 1.0f / (float)live : 0.f;
        a.counts[(size_t)sq * E + e] = cnt;
        a.prob[(size_t)sq * E + e] = sum * inv;
        my_loss += (double)(unit * ((float)cnt * inv) * (sum * inv));
      } else {
        float* at = slots + (2 * (size_t)blockIdx.x + (begins < b0 ? 0 : 1)) * slot_ints;
        at[e] = sum;
        reinterpret_cast<int*>(at)[E + e] = cnt;
      }
    }
  }
  __syncthreads();
  auto block_sum = [&](double v) -> double {   // fixed order; the result in thread 0
    for (int off = 16; off; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
    if (lane == 0) s_loss[warp] = v;
    __syncthreads();
    double r = 0.0;
    if (threadIdx.x == 0)
      for (int w = 0; w < warps; ++w) r += s_loss[w];
    __syncthreads();
    return r;
  };
  my_loss = block_sum(my_loss);
  if (threadIdx.x == 0) meta[blockIdx.x].loss += my_loss;

  // ---- a sequence over several blocks: its pieces in order, by the block whose piece arrives last.  The block that holds its
  // first token has it as second piece and its ticket, the others have it as first piece.
  const int nb = gridDim.x;
  auto block_of = [&](int t) {   // floor(T i / nb) <= t, the largest such i
    int i = (int)((long long)t * nb / T);
    while (i + 1 < nb && (long long)T * (i + 1) / nb <= t) ++i;
    return i;
  };
  auto arrive = [&](int* ticket, int expected) -> bool {   // of the whole block; true: everybody else has been
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) s_last = atomicAdd(ticket, 1) == expected - 1;
    __syncthreads();
    const bool last = s_last != 0;
    if (last) __threadfence();
    return last;
  };
  const int parts = max(1, min(2 * warps, (int)blockDim.x / E));
  auto join = [&](int sq) -> double {   // fills the sequence's outputs; its share of the loss
    const int first = block_of(seq_begin(a.seq_offsets, sq, T)), last = block_of(seq_begin(a.seq_offsets, sq + 1, T) - 1);
    int live = 0;
    for (int q = first + threadIdx.x; q <= last; q += blockDim.x) live += __ldcg(&meta[q].n[q == first ? 1 : 0]);
    live = (int)block_sum((double)live);
    if (threadIdx.x == 0) { s_last = live; a.tokens[sq] = live; }
    // the experts, and ranges of the blocks where threads are left
    const int nq = last - first + 1, part = (int)threadIdx.x / E;
    const bool split = parts > 1;
    const int q0 = first + (split ? (int)((long long)nq * part / parts) : 0), q1 = first + (split ? (int)((long long)nq * (part + 1) / parts) : nq);
    auto sums = [&](int e, float* sum, int* cnt) {
      float v = 0.f;
      int c = 0;
#pragma unroll 8
      for (int q = q0; q < q1; ++q) {
        const float* at = slots + (2 * (size_t)q + (q == first ? 1 : 0)) * slot_ints;
        v += __ldcg(at + e);
        c += __ldcg(reinterpret_cast<const int*>(at) + E + e);
      }
      *sum = v;
      *cnt = c;
    };
    float* const p_sum = w_sum;   // [parts][E]
    int* const p_cnt = w_cnt;
    if (split && part < parts) sums((int)threadIdx.x % E, &p_sum[threadIdx.x], &p_cnt[threadIdx.x]);
    __syncthreads();
    live = s_last;
    const float inv = live ? 1.0f / (float)live : 0.f;
    double share = 0.0;
    for (int e = threadIdx.x; e < E; e += blockDim.x) {
      float sum = 0.f;
      int cnt = 0;
      if (split) {
        for (int q = 0; q < parts; ++q) { sum += p_sum[q * E + e]; cnt += p_cnt[q * E + e]; }
      } else {
        sums(e, &sum, &cnt);
      }
      a.counts[(size_t)sq * E + e] = cnt;
      a.prob[(size_t)sq * E + e] = sum * inv;
      share += (double)(unit * ((float)cnt * inv) * (sum * inv));
    }
    __syncthreads();
    return block_sum(share);
  };
  if (n > 1) {
#pragma unroll 1
    for (int h = 0; h < 2; ++h) {
      __syncthreads();
      const int sq = meta[blockIdx.x].seq[h];
      if (sq < 0) continue;
      const int begins = seq_begin(a.seq_offsets, sq, T), stop = seq_begin(a.seq_offsets, sq + 1, T);
      const int first = block_of(begins), last = block_of(stop - 1);
      if (last <= first || (int)blockIdx.x < first || (int)blockIdx.x > last) continue;   // (offsets that do not ascend)
      if (arrive(a.tickets + 1 + first, last - first + 1)) {
        const double share = join(sq);
        if (threadIdx.x == 0) meta[blockIdx.x].loss += share;
      }
    }
  }
  if (!arrive(a.tickets, nb)) return;

  // ---- the last block of all
  for (int i = threadIdx.x; i <= nb; i += blockDim.x) a.tickets[i] = 0;   // for the next call
  double total = 0.0, total_z = 0.0, total_tokens = 0.0;
  for (int b = threadIdx.x; b < nb; b += blockDim.x) {
    total += __ldcg(&meta[b].loss);
    total_z += __ldcg(&meta[b].z);
    total_tokens += (double)__ldcg(&meta[b].tokens);
  }
  if (n == 1 && nb > 1) {
    const int begins = seq_begin(a.seq_offsets, 0, T), stop = seq_begin(a.seq_offsets, 1, T);
    if (begins < stop && block_of(begins) < block_of(stop - 1)) {
      const double share = join(0);
      if (threadIdx.x == 0) total += share;
    }
  }
  total = block_sum(total);
  total_z = block_sum(total_z);
  total_tokens = block_sum(total_tokens);
  if (threadIdx.x == 0) {
    a.losses[0] = (float)total;
    a.losses[1] = total_tokens > 0.0 ? (float)(total_z / total_tokens) : 0.f;
    a.tokens[n] = (int)total_tokens;
  }
}

// ------------------------------------------------------------------------------------------
// Backward: one read of the logits, one write of the gradient.  The coefficients x of a run stay in registers; what the
// k selected experts get is scattered into a row of shared memory that is zero in between, so an id that a token names twice adds up.
// ------------------------------------------------------------------------------------------
constexpr int BAL_BWD_WARPS = 8;

template <int LPT, int VPL, int VW, bool SIG>
__global__ void __launch_bounds__(32 * BAL_BWD_WARPS) balance_bwd_kernel(const BalanceArgs a) {
  constexpr int TPW = 32 / LPT;
  extern __shared__ __align__(16) float fsm[];
  const int E = a.E, n = a.n_seq, T = a.T, k = a.k;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, l = lane % LPT, grp = lane / LPT;
  constexpr int ROW = LPT * VPL;
  float* const add = fsm + (warp * TPW + grp) * 2 * ROW;   // what the selected experts get
  float* const val = add + ROW;                           // the row's probabilities (sigmoid gate: sigmoids)
#pragma unroll
  for (int i = 0; i < VPL; ++i) add[i * LPT + l] = 0.f;
  __syncwarp();
  pdl_wait();
  pdl_trigger();
  const int gw = blockIdx.x * BAL_BWD_WARPS + warp, nw = gridDim.x * BAL_BWD_WARPS;
  const int wa = (int)((long long)T * gw / nw), wb = (int)((long long)T * (gw + 1) / nw);
  const bool scores = a.d_topk_w != nullptr, renorm = (a.mode & GATE_RENORM) != 0;
  const float g_bal = a.d_losses[0];
  const int total = a.tokens[n];
  const float g_z = total > 0 ? 2.0f * a.d_losses[1] / (float)total : 0.f;
  int s = wa < wb ? seq_of(a.seq_offsets, n, T, wa, lane) : n;
  for (int t = wa; t < wb;) {
    int stop = s < n ? seq_begin(a.seq_offsets, s + 1, T) : T;
    if (stop <= t) stop = t + 1;   // (offsets that do not ascend)
    const int end = min(stop, wb);
    const bool inside = s >= 0 && s < n;
    float x[VPL];
    const float ns = inside ? (float)a.tokens[s] : 0.f;
    const float unit = ns > 0.f ? g_bal * (float)E / ((float)k * (float)n) / ns / ns : 0.f;
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      const int e = expert_at<LPT, VW>(i, l);
      x[i] = inside && e < E ? unit * (float)a.counts[(size_t)s * E + e] : 0.f;
    }
    float v[VPL], next[VPL];
    int next_id = -1;
    float next_g = 0.f;
    bool next_on = false;
    auto fetch = [&](int tt) {
      const bool in = tt < end;
      load_row<LPT, VPL, VW>(a.logits + (size_t)tt * E, E, l, in, next);
      next_on = inside && in && (!a.token_mask || a.token_mask[tt] != 0);
      if (scores) {
        next_id = in && l < k ? a.topk_ids[(size_t)tt * k + l] : -1;
        next_g = in && l < k ? a.d_topk_w[(size_t)tt * k + l] : 0.f;
      }
    };
    fetch(t + grp);
#pragma unroll 1
    for (int t0 = t; t0 < end; t0 += TPW) {
      const int tt = t0 + grp;
#pragma unroll
      for (int i = 0; i < VPL; ++i) v[i] = next[i];
      const bool on = next_on;
      const int id = next_id;
      const float g = next_g;
      fetch(tt + TPW);
      float soft[VPL], p[SIG ? VPL : 1], sig[SIG ? VPL : 1], d[VPL];
      const float lse = softmax_row<LPT, VPL>(v, soft);
      if constexpr (SIG) sigmoid_row<LPT, VPL>(v, p, sig);
      // ---- the scores' share: lane l of the group has the ids l, l + LPT, ..
      auto each = [&](auto body) {
        if (tt < end)
          for (int j = l; j < k; j += LPT) {
            const int e = j == l ? id : a.topk_ids[(size_t)tt * k + j];
            if (e >= 0 && e < E) body(e, j == l ? g : a.d_topk_w[(size_t)tt * k + j]);
          }
      };
      if (scores) {
        if (SIG || renorm) {
#pragma unroll
          for (int i = 0; i < VPL; ++i) {
            const int e = expert_at<LPT, VW>(i, l);
            if (e < E) val[e] = SIG ? sig[SIG ? i : 0] : soft[i];
          }
          __syncwarp();
          float Z = 0.f, dot = 0.f;
          if (renorm) {
            each([&](int e, float) { Z += val[e]; });
            Z = group_sum(Z, LPT);
            const float inv = Z > 0.f ? 1.0f / Z : 0.f;
            each([&](int e, float ge) { dot = fmaf(ge, val[e] * inv, dot); });
            dot = group_sum(dot, LPT);
            each([&](int e, float ge) { const float w = val[e] * inv; atomicAdd(&add[e], w * (ge - dot) * (SIG ? 1.0f - val[e] : 1.0f)); });
          } else {
            each([&](int e, float ge) { atomicAdd(&add[e], ge * val[e] * (1.0f - val[e])); });
          }
        } else {
          each([&](int e, float ge) { atomicAdd(&add[e], ge); });   // joins x: both are gradients of the softmax
        }
        __syncwarp();
      }
      // ---- the whole gradient
      float q[VPL], dot = 0.f;
      const bool joins = scores && !SIG && !renorm;
#pragma unroll
      for (int i = 0; i < VPL; ++i) {
        const int e = expert_at<LPT, VW>(i, l);
        const float more = scores && e < E ? add[e] : 0.f;
        const float xi = (on ? x[i] : 0.f) + (joins ? more : 0.f);
        d[i] = joins ? 0.f : more;
        q[i] = xi;
        dot = fmaf(SIG ? p[SIG ? i : 0] : soft[i], xi, dot);
      }
      dot = group_sum(dot, LPT);
      const float zc = on ? g_z * lse : 0.f;
#pragma unroll
      for (int i = 0; i < VPL; ++i) {
        const float pi = SIG ? p[SIG ? i : 0] * (1.0f - sig[SIG ? i : 0]) : soft[i];
        d[i] = fmaf(pi, q[i] - dot, fmaf(zc, soft[i], d[i]));
      }
      if (scores) {
        __syncwarp();
        each([&](int e, float) { add[e] = 0.f; });
      }
      if (tt < end) {
        float* out = a.d_logits + (size_t)tt * E;
#pragma unroll
        for (int i = 0; i < VPL; i += VW) {
          const int e = expert_at<LPT, VW>(i, l);
          if (e < E) {
            if (VW == 4) *reinterpret_cast<float4*>(out + e) = make_float4(d[i], d[i + (VW > 1 ? 1 : 0)], d[i + (VW > 1 ? 2 : 0)], d[i + (VW > 1 ? 3 : 0)]);
            else out[e] = d[i];
          }
        }
      }
      __syncwarp();
    }
    t = end;
    if (t < wb) s = seq_of(a.seq_offsets, n, T, t, lane);
  }
}

// ------------------------------------------------------------------------------------------
// Lanes a token and values a lane by the number of experts; vectors of four where rows are whole 16-byte pieces.
template <class F>
static cudaError_t with_balance_shape(int E, bool vec, F f) {
#define MOE_BAL_CASE(LPT, VPL) return vec ? f(std::integral_constant<int, LPT>(), std::integral_constant<int, VPL>(), std::integral_constant<int, 4>()) \
                                          : f(std::integral_constant<int, LPT>(), std::integral_constant<int, VPL>(), std::integral_constant<int, 1>())
  if (E <= 8) MOE_BAL_CASE(1, 8);
  if (E <= 32) MOE_BAL_CASE(4, 8);
  if (E <= 64) MOE_BAL_CASE(8, 8);
  if (E <= 128) MOE_BAL_CASE(16, 8);
  if (E <= 256) MOE_BAL_CASE(32, 8);
  if (E <= 512) MOE_BAL_CASE(32, 16);
  MOE_BAL_CASE(32, 32);
#undef MOE_BAL_CASE
}

static bool rows_of_vectors(const void* p, int E) { return E % 4 == 0 && (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

int balance_fwd_blocks(int T, int E) {
  const long bytes = (long)T * E * 4;
  long b = (bytes + BAL_BLOCK_BYTES - 1) / BAL_BLOCK_BYTES;
  if (b > BAL_MAX_BLOCKS) b = BAL_MAX_BLOCKS;
  if (b > T) b = T;
  return b < 1 ? 1 : (int)b;
}
size_t balance_scratch_bytes(int T_max, int E) {
  return (size_t)balance_fwd_blocks(T_max, E) * (sizeof(BalBlock) + 4 * (size_t)E * sizeof(int));
}

cudaError_t launch_balance_fwd(const BalanceArgs& a, cudaStream_t s, int* launches) {
  int warps = BAL_MAX_WARPS;
  while (warps > 4 && 5 * warps * a.E * (int)sizeof(int) > 96 * 1024) warps >>= 1;
  const size_t smem = 5 * (size_t)warps * a.E * sizeof(int);
  const int blocks = balance_fwd_blocks(a.T, a.E);
  return with_balance_shape(a.E, rows_of_vectors(a.logits, a.E), [&](auto lpt, auto vpl, auto vw) -> cudaError_t {
    auto go = [&](auto sig) -> cudaError_t {
      constexpr auto kernel = balance_fwd_kernel<lpt(), vpl(), vw(), sig()>;
      if (smem > 48 * 1024)
        if (cudaError_t e = opt_in_smem<kernel>(100 * 1024)) return e;
      ++*launches;
      return launch_dependent(kernel, dim3(blocks), dim3(warps * 32), smem, s, a);
    };
    return (a.mode & GATE_SIGMOID) ? go(std::true_type()) : go(std::false_type());
  });
}

cudaError_t launch_balance_bwd(const BalanceArgs& a, cudaStream_t s, int* launches) {
  const bool vec = rows_of_vectors(a.logits, a.E) && rows_of_vectors(a.d_logits, a.E);
  return with_balance_shape(a.E, vec, [&](auto lpt, auto vpl, auto vw) -> cudaError_t {
    constexpr size_t smem = 2 * sizeof(float) * (size_t)BAL_BWD_WARPS * 32 * vpl();
    const int per_block = BAL_BWD_WARPS * (32 / lpt());   // tokens of a round
    int blocks = (a.T + per_block - 1) / per_block;
    if (blocks > BAL_BWD_MAX_BLOCKS) blocks = BAL_BWD_MAX_BLOCKS;
    auto go = [&](auto sig) -> cudaError_t {
      constexpr auto kernel = balance_bwd_kernel<lpt(), vpl(), vw(), sig()>;
      if (smem > 48 * 1024)
        if (cudaError_t e = opt_in_smem<kernel>((int)smem)) return e;
      ++*launches;
      return launch_dependent(kernel, dim3(blocks), dim3(32 * BAL_BWD_WARPS), smem, s, a);
    };
    return (a.mode & GATE_SIGMOID) ? go(std::true_type()) : go(std::false_type());
  });
}

}  // namespace moe
