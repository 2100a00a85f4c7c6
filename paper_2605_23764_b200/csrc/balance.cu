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

constexpr int BAL_MAX_WARPS = 32;   // of a forward block: one block an SM, so that few blocks' pieces are to be joined

__device__ __forceinline__ float group_sum(float v, int lpt) {
  for (int off = lpt >> 1; off; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
  return v;
}
// N sums at a time: their shuffles overlap
template <int LPT, int N>
__device__ __forceinline__ void group_sums(float (&v)[N]) {
#pragma unroll
  for (int off = LPT >> 1; off; off >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], off);
}
__device__ __forceinline__ float group_max(float v, int lpt) {
  for (int off = lpt >> 1; off; off >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, off));
  return v;
}

// Sequence offsets: the caller's, kept inside the batch; staged in shared memory where they fit, since they are looked up in turn.
struct SeqTable {
  const int* off;    // NULL: the batch is one sequence
  const int* staged; // NULL: not staged
  int n, T;
  // first token of sequence s (s = n: one behind the last)
  __device__ __forceinline__ int begin(int s) const {
    if (staged) return staged[s];
    if (!off) return s ? T : 0;
    return min(max(__ldg(off + s), 0), T);
  }
  // Sequence of token t: -1 in front of the first one, n behind the last.  A warp's 32 probes a round, where a lane's bisection
  // would be a chain of dependent reads.
  __device__ __forceinline__ int of(int t, int lane) const {
    if (!off) return 0;
    int lo = 0, len = n + 1;
    while (len > 32) {
      const int step = (len + 31) >> 5;
      const int i = lane * step;
      const int c = __popc(__ballot_sync(0xffffffffu, i < len && begin(lo + i) <= t));
      if (c == 0) return lo - 1;
      const int at = (c - 1) * step;
      lo += at;
      len = min(step, len - at);
    }
    return lo - 1 + __popc(__ballot_sync(0xffffffffu, lane < len && begin(lo + lane) <= t));
  }
};
constexpr int BAL_STAGED = 1024;   // offsets in shared memory, at most
// Fills `to` by the whole block (a barrier follows in the caller).
__device__ __forceinline__ void stage_offsets(const BalanceArgs& a, int* to) {
  if (a.seq_offsets && a.n_seq < BAL_STAGED)
    for (int i = threadIdx.x; i <= a.n_seq; i += blockDim.x) to[i] = min(max(__ldg(a.seq_offsets + i), 0), a.T);
}
__device__ __forceinline__ SeqTable seq_table(const BalanceArgs& a, const int* staged) {
  return SeqTable{a.seq_offsets, a.seq_offsets && a.n_seq < BAL_STAGED ? staged : nullptr, a.n_seq, a.T};
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

constexpr float LOG2E = 1.4426950408889634f;
__device__ __forceinline__ float ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

template <int LPT, int VPL>
__device__ __forceinline__ float row_max(const float (&v)[VPL]) {
  float m = v[0];
#pragma unroll
  for (int i = 1; i < VPL; ++i) m = fmaxf(m, v[i]);
  return group_max(m, LPT);
}
// Softmax terms exp(v - max) and -- SIG -- sigmoids of a row before they are normalised: ex, p, inv[0] and inv[1] = 1 / their sums, sig
// the sigmoids themselves (NULL: not wanted); the answer is the row's logsumexp.  A row without a finite logit has no probabilities:
// zeros, and logsumexp counts as 0.  Below zero sigmoid(l) = exp(l) / (1 + exp(l)), so sigmoids of a row of large negative logits are
// scaled by its largest as a softmax is, and keep their proportions where every sigmoid underflows.
template <int LPT, int VPL, bool SIG>
__device__ __forceinline__ float row_terms(const float (&v)[VPL], float (&ex)[VPL], float (&p)[SIG ? VPL : 1], float* sig, float (&inv)[2]) {
  float m = row_max<LPT, VPL>(v);
  const bool low = m < -16.f && m > -INFINITY;
  if (m == -INFINITY) m = 0.f;
  float den[SIG ? 2 : 1] = {};
#pragma unroll
  for (int i = 0; i < VPL; ++i) {
    ex[i] = ex2((v[i] - m) * LOG2E);
    den[0] += ex[i];
    if constexpr (SIG) {
      const float t = ex2(-fabsf(v[i]) * LOG2E), r = __fdividef(1.0f, 1.0f + t), s = v[i] >= 0.f ? r : t * r;
      if (sig) sig[i] = s;
      p[i] = low ? ex[i] * r : s;
      den[1] += p[i];
    }
  }
  group_sums<LPT>(den);
  inv[0] = den[0] == 0.f ? 0.f : __fdividef(1.0f, den[0]);
  if constexpr (SIG) inv[1] = den[1] == 0.f ? 0.f : __fdividef(1.0f, den[1]);
  return den[0] == 0.f ? 0.f : m + __logf(den[0]);
}

}  // namespace

// ------------------------------------------------------------------------------------------
// Forward.  What a warp sums over a run that lies wholly in its range is final.  A run that reaches beyond it leaves a piece: the
// warps' pieces of a block are joined in order in shared memory, the blocks' in order by the block that arrives last.  Sums
// are therefore the same from call to call.
//
// Bound by the chain of latencies behind the read of the logits.  Clocks of the block that ends last, one sequence of 8192 x 256 (16 us):
// first loads 1400, rounds of tokens 8400, the warps' pieces sorted and joined 4900, sums over the block 3000 in all, ticket 3000, the
// blocks' pieces joined by the last one 10700; of 31700.  In 8 sequences (20-22 us) a block that joins two of them spends 19500 of 43100
// there.  65536 x 256 (24.5 us, 2.7 TB/s): rounds 25000 of 49000; sigmoid scores in 97 sequences (35 us) 38000 of 70000.  One block an
// SM: two and four left more pieces to join.  The registers that so many warps leave (64 to 128 a thread) spill 7 to 29 words.
// ------------------------------------------------------------------------------------------
// A piece in global memory, two a block: of the sequence that began before the block, of the one that goes on behind it.
// Per block {seq of both pieces, tokens of both, sums of the block}, then [block][2][E] {sum, count}
__host__ __device__ constexpr int balance_warps_most(int vpl) { return vpl <= 8 ? BAL_MAX_WARPS : vpl <= 16 ? 24 : 16; }   // registers
struct BalBlock { int seq[2], n[2]; double loss, joined, z, tokens; };   // joined: share of the sequence that goes on behind it

template <int LPT, int VPL, int VW, bool SIG>
__global__ void __launch_bounds__(32 * balance_warps_most(VPL)) balance_fwd_kernel(const BalanceArgs a) {
  constexpr int TPW = 32 / LPT;
  extern __shared__ __align__(16) int bsm[];
  __shared__ int offsets[BAL_STAGED];
  __shared__ int w_seq[2 * BAL_MAX_WARPS], w_n[2 * BAL_MAX_WARPS];
  __shared__ double s_sum[3][32];
  // stretches of the warps' pieces that are one sequence: pieces [from, to), where the sum goes (0, 1: that piece of the block; 2: final)
  __shared__ int g_seq[2 * BAL_MAX_WARPS], g_from[2 * BAL_MAX_WARPS + 1], g_n[2 * BAL_MAX_WARPS], g_to[2 * BAL_MAX_WARPS], g_count;
  __shared__ unsigned long long g_valid;
  __shared__ int s_last[3], s_live, b_seq[2];
  const int E = a.E, n = a.n_seq, T = a.T;
  const int warps = blockDim.x >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, l = lane % LPT, grp = lane / LPT;
  int* const hist = bsm + warp * E;                                   // [warps][E]
  float* const w_sum = reinterpret_cast<float*>(bsm + warps * E);     // [warps][2][E]
  int* const w_cnt = bsm + 3 * warps * E;                             // [warps][2][E]
  for (int e = lane; e < E; e += 32) hist[e] = 0;
  if (lane < 2) w_seq[2 * warp + lane] = -1;
  pdl_wait();
  pdl_trigger();

  const int b0 = blockIdx.x * a.chunk, b1 = min(b0 + a.chunk, T), per_warp = (a.chunk + warps - 1) / warps;
  const int wa = min(b0 + warp * per_warp, b1), wb = min(wa + per_warp, b1);
  // A token's row, mask and the lane's first id are read a round ahead, the first ones while the offsets arrive.
  float v[VPL], next[VPL];
  int next_id = -1, next_at = wa;
  bool next_on = false;
  auto fetch = [&](int t0) {
    const int tt = t0 + grp;
    next_at = t0;
    load_row<LPT, VPL, VW>(a.logits + (size_t)tt * E, E, l, tt < wb, next);
    next_on = tt < wb && (!a.token_mask || a.token_mask[tt] != 0);
    next_id = tt < wb && l < a.k ? a.topk_ids[(size_t)tt * a.k + l] : -1;
  };
  fetch(wa);
  stage_offsets(a, offsets);
  __syncthreads();
  const SeqTable seqs = seq_table(a, offsets);
  const float unit = (float)E / ((float)a.k * (float)n);
  double my_loss = 0.0, zsum = 0.0;   // of the thread; of the warp
  int tokens = 0;
  int s = wa < wb ? seqs.of(wa, lane) : n;
  for (int t = wa; t < wb;) {
    // the run [t, end) of sequence s
    const bool inside = s >= 0 && s < n;
    const int begins = inside ? seqs.begin(s) : 0;
    int stop = s < n ? seqs.begin(s + 1) : T;
    if (stop <= t) stop = t + 1;   // (offsets that do not ascend)
    const int end = min(stop, wb);
    if (inside) {
      float acc[VPL];
#pragma unroll
      for (int i = 0; i < VPL; ++i) acc[i] = 0.f;
      float z = 0.f;
      int live = 0;
      if (next_at != t) fetch(t);
#pragma unroll 1
      for (int t0 = t; t0 < end; t0 += TPW) {
        const int tt = t0 + grp;
#pragma unroll
        for (int i = 0; i < VPL; ++i) v[i] = next[i];
        const bool on = next_on && tt < end;
        const int id = next_id;
        fetch(t0 + TPW);
        if (on) {
          if (id >= 0 && id < E) atomicAdd(&hist[id], 1);
          for (int j = l + LPT; j < a.k; j += LPT) {
            const int e = a.topk_ids[(size_t)tt * a.k + j];
            if (e >= 0 && e < E) atomicAdd(&hist[e], 1);
          }
        }
        float ex[VPL], p[SIG ? VPL : 1], inv[2];
        const float lse = row_terms<LPT, VPL, SIG>(v, ex, p, nullptr, inv);
        if (on) {
#pragma unroll
          for (int i = 0; i < VPL; ++i) acc[i] = SIG ? fmaf(p[SIG ? i : 0], inv[1], acc[i]) : fmaf(ex[i], inv[0], acc[i]);
          if (l == 0) { z = fmaf(lse, lse, z); ++live; }
        }
      }
      // the groups of the warp
#pragma unroll
      for (int off = LPT; off < 32; off <<= 1) {
#pragma unroll
        for (int i = 0; i < VPL; ++i) acc[i] += __shfl_xor_sync(0xffffffffu, acc[i], off);
      }
      live = __reduce_add_sync(0xffffffffu, live);
      zsum += (double)group_sum(z, 32);
      tokens += live;
      __syncwarp();
      const bool whole = begins >= wa && stop <= wb;
      const int piece = t == wa ? 0 : 1;
      if (!whole && lane == 0) { w_seq[2 * warp + piece] = s; w_n[2 * warp + piece] = live; }
      const float inv = live ? 1.0f / (float)live : 0.f;
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
              my_loss += (double)(unit * ((float)c * inv) * (acc[i] * inv));
            } else {
              w_sum[(2 * warp + piece) * E + e] = acc[i];
              w_cnt[(2 * warp + piece) * E + e] = c;
            }
          }
        }
      }
      if (whole && lane == 0) a.tokens[s] = live;
      __syncwarp();
    }
    t = end;
    if (t < wb) s = seqs.of(t, lane);
  }
  // sequences without tokens belong to no warp's range
  for (int q = blockIdx.x * warps + warp; q < n; q += gridDim.x * warps)
    if (seqs.begin(q) >= seqs.begin(q + 1)) {
      for (int e = lane; e < E; e += 32) {
        a.counts[(size_t)q * E + e] = 0;
        a.prob[(size_t)q * E + e] = 0.f;
      }
      if (lane == 0) a.tokens[q] = 0;
    }
  __syncthreads();

  // ---- the warps' pieces: which of them are one sequence ..
  BalBlock* const meta = reinterpret_cast<BalBlock*>(a.scratch);
  float2* const slots = reinterpret_cast<float2*>(meta + gridDim.x);
  if (warp == 0) {
    // lane w has both of warp w
    int sq[2], ln[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      sq[h] = lane < warps ? w_seq[2 * lane + h] : -1;
      ln[h] = sq[h] >= 0 ? w_n[2 * lane + h] : 0;
    }
    const uint32_t any = __ballot_sync(0xffffffffu, sq[0] >= 0 || sq[1] >= 0), before = any & ((1u << lane) - 1u);
    const int tail = __shfl_sync(0xffffffffu, sq[1] >= 0 ? sq[1] : sq[0], before ? 31 - __clz(before) : 0);   // of the last lane in front
    int prev = before ? tail : -1;
    int run = ln[0] + ln[1];
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int o = __shfl_up_sync(0xffffffffu, run, off);
      if (lane >= off) run += o;
    }
    const int ahead = run - ln[0] - ln[1];   // tokens of the lanes in front
    bool starts[2];
    uint32_t start[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      starts[h] = sq[h] >= 0 && sq[h] != prev;
      if (sq[h] >= 0) prev = sq[h];
      start[h] = __ballot_sync(0xffffffffu, starts[h]);
    }
    if (lane < 2) b_seq[lane] = -1;
    __syncwarp();
    const int count = __popc(start[0]) + __popc(start[1]);
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (starts[h]) {
        const uint32_t below = (1u << lane) - 1u;
        const int i = __popc(start[0] & (h ? below | (1u << lane) : below)) + __popc(start[1] & below);
        const int begins = seqs.begin(sq[h]), stop = seqs.begin(sq[h] + 1);
        g_seq[i] = sq[h];
        g_from[i] = 2 * lane + h;
        g_n[i] = ahead + (h ? ln[0] : 0);   // tokens in front of it, until all are known
        g_to[i] = begins >= b0 && stop <= b1 ? 2 : begins < b0 ? 0 : 1;
      }
    const int all = __shfl_sync(0xffffffffu, run, 31);
    if (lane == 0) { g_count = count; g_from[count] = 2 * warps; }
    const uint32_t v0 = __ballot_sync(0xffffffffu, sq[0] >= 0), v1 = __ballot_sync(0xffffffffu, sq[1] >= 0);
    if (lane < 2) reinterpret_cast<uint32_t*>(&g_valid)[lane] = lane ? v1 : v0;
    __syncwarp();
    int live[2] = {0, 0};
    for (int i = lane, r = 0; i < count; i += 32, ++r) live[r] = (i + 1 < count ? g_n[i + 1] : all) - g_n[i];
    __syncwarp();
    for (int i = lane, r = 0; i < count; i += 32, ++r) {
      g_n[i] = live[r];
      if (g_to[i] == 2) a.tokens[g_seq[i]] = live[r];
      else { b_seq[g_to[i]] = g_seq[i]; meta[blockIdx.x].n[g_to[i]] = live[r]; }
    }
    __syncwarp();
    if (lane < 2) meta[blockIdx.x].seq[lane] = b_seq[lane];
    if (lane == 0) meta[blockIdx.x].joined = 0.0;
  }
  __syncthreads();
  // .. and their sums in order: every thread has an expert, and a range of the pieces where threads are left
  const int parts = max(1, min(warps / 2, (int)blockDim.x / E)), part = (int)threadIdx.x / E;
  float* const p_sum = reinterpret_cast<float*>(bsm);   // [parts][E], in place of the histograms
  int* const p_cnt = bsm + parts * E;
  // sums over [from, until) of what `at` gives for a piece and an expert, handed to `put`
  auto pieces = [&](int from, int until, auto at, auto put) {
    if (parts == 1) {
      for (int e = threadIdx.x; e < E; e += blockDim.x) {
        float sum = 0.f;
        int cnt = 0;
#pragma unroll 8
        for (int q = from; q < until; ++q) at(q, e, sum, cnt);
        put(e, sum, cnt);
      }
      return;
    }
    const int e = (int)threadIdx.x - part * E, len = (until - from + parts - 1) / parts;
    if (part < parts) {
      float sum = 0.f;
      int cnt = 0;
      const int q0 = min(from + part * len, until), q1 = min(q0 + len, until);
#pragma unroll 16
      for (int q = q0; q < q1; ++q) at(q, e, sum, cnt);
      p_sum[threadIdx.x] = sum;
      p_cnt[threadIdx.x] = cnt;
    }
    __syncthreads();
    if (part == 0) {
      float sum = 0.f;
      int cnt = 0;
      for (int q = 0; q < parts; ++q) { sum += p_sum[q * E + e]; cnt += p_cnt[q * E + e]; }
      put(e, sum, cnt);
    }
    __syncthreads();
  };
  for (int i = 0; i < g_count; ++i) {
    const int sq = g_seq[i], to = g_to[i];
    const float inv = g_n[i] ? 1.0f / (float)g_n[i] : 0.f;
    const uint32_t v0 = (uint32_t)g_valid, v1 = (uint32_t)(g_valid >> 32);
    float2* const slot = slots + (2 * (size_t)blockIdx.x + (to & 1)) * E;
    pieces(g_from[i], g_from[i + 1],
           [&](int q, int e, float& sum, int& cnt) {   // (a piece that is not there holds anything)
             const float x = w_sum[q * E + e];
             const int c = w_cnt[q * E + e];
             const bool there = (q & 1 ? v1 : v0) >> (q >> 1) & 1;
             sum += there ? x : 0.f;
             cnt += there ? c : 0;
           },
           [&](int e, float sum, int cnt) {
             if (to == 2) {
               a.counts[(size_t)sq * E + e] = cnt;
               a.prob[(size_t)sq * E + e] = sum * inv;
               my_loss += (double)(unit * ((float)cnt * inv) * (sum * inv));
             } else {
               __stcg(slot + e, make_float2(sum, __int_as_float(cnt)));
             }
           });
  }

  // ---- a sequence over several blocks: its pieces in order, by the block whose piece arrives last.  The block that holds its
  // first token has it as second piece and its ticket, the others have it as first piece.
  const int nb = gridDim.x;
  auto block_of = [&](int t) { return t / a.chunk; };
  auto join = [&](int sq, double& loss) {   // fills the sequence's outputs and adds the threads' shares of its loss
    const int first = block_of(seqs.begin(sq)), last = block_of(seqs.begin(sq + 1) - 1);
    if (parts == 1) __syncthreads();   // (an earlier join's tokens have been used)
    if (warp == warps - 1) {
      int live = 0;
      for (int q = first + lane; q <= last; q += 32) live += __ldcg(&meta[q].n[q == first ? 1 : 0]);
      live = __reduce_add_sync(0xffffffffu, live);
      if (lane == 0) { s_live = live; a.tokens[sq] = live; }
    }
    if (parts == 1) __syncthreads();   // (else there is one between the sums and their use)
    pieces(first, last + 1,
           [&](int q, int e, float& sum, int& cnt) {
             const float2 x = __ldcg(slots + (2 * (size_t)q + (q == first ? 1 : 0)) * E + e);
             sum += x.x;
             cnt += __float_as_int(x.y);
           },
           [&](int e, float sum, int cnt) {
             const float inv = s_live ? 1.0f / (float)s_live : 0.f;
             a.counts[(size_t)sq * E + e] = cnt;
             a.prob[(size_t)sq * E + e] = sum * inv;
             loss += (double)(unit * ((float)cnt * inv) * (sum * inv));
           });
  };
  // sums over the block, in thread 0; the order is fixed
  auto block_sums = [&](auto& v) {
    constexpr int N = sizeof(v) / sizeof(double);
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int off = 16; off; off >>= 1) v[i] += __shfl_xor_sync(0xffffffffu, v[i], off);
    __syncthreads();
    if (lane == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) s_sum[i][warp] = v[i];
    }
    __syncthreads();
    if (warp == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        v[i] = lane < warps ? s_sum[i][lane] : 0.0;
#pragma unroll
        for (int off = 16; off; off >>= 1) v[i] += __shfl_xor_sync(0xffffffffu, v[i], off);
      }
    }
  };
  if (n > 1 && nb > 1) {
    __threadfence();
    __syncthreads();
    if (threadIdx.x < 2) {
      const int sq = b_seq[threadIdx.x];
      int last_one = 0;
      if (sq >= 0) {
        const int first = block_of(seqs.begin(sq)), last = block_of(seqs.begin(sq + 1) - 1);
        if (last > first && (int)blockIdx.x >= first && (int)blockIdx.x <= last)   // (else offsets that do not ascend)
          last_one = atomicAdd(a.tickets + 1 + first, 1) == last - first;
      }
      s_last[threadIdx.x] = last_one;
    }
    __syncthreads();
    // Which block joins depends on timing, so a sequence's share does not count as this block's: it goes to the sequence's first one.
#pragma unroll 1
    for (int h = 0; h < 2; ++h)
      if (s_last[h]) {
        __threadfence();
        double loss[1] = {0.0};
        join(b_seq[h], loss[0]);
        block_sums(loss);
        if (threadIdx.x == 0) meta[block_of(seqs.begin(b_seq[h]))].joined = loss[0];
      }
  }
  // the warps' z and tokens: lane 0 of each has them still
  double r[3] = {my_loss, lane == 0 ? zsum : 0.0, lane == 0 ? (double)tokens : 0.0};
  block_sums(r);
  auto finish = [&]() {
    if (threadIdx.x == 0) {
      a.losses[0] = (float)r[0];
      a.losses[1] = r[2] > 0.0 ? (float)(r[1] / r[2]) : 0.f;
      a.tokens[n] = (int)r[2];
    }
  };
  if (nb == 1) return finish();
  if (threadIdx.x == 0) {
    BalBlock& m = meta[blockIdx.x];
    m.loss = r[0]; m.z = r[1]; m.tokens = r[2];
  }
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) s_last[2] = atomicAdd(a.tickets, 1) == nb - 1;
  __syncthreads();
  if (!s_last[2]) return;
  __threadfence();

  // ---- the last block of all
  for (int i = threadIdx.x; i <= nb; i += blockDim.x) a.tickets[i] = 0;   // for the next call
  for (int i = 0; i < 3; ++i) r[i] = 0.0;
  for (int b = threadIdx.x; b < nb; b += blockDim.x) {
    r[0] += __ldcg(&meta[b].loss) + __ldcg(&meta[b].joined);
    r[1] += __ldcg(&meta[b].z);
    r[2] += __ldcg(&meta[b].tokens);
  }
  if (n == 1) {
    const int begins = seqs.begin(0), stop = seqs.begin(1);
    if (begins < stop && block_of(begins) < block_of(stop - 1)) join(0, r[0]);
  }
  block_sums(r);
  finish();
}

// ------------------------------------------------------------------------------------------
// Backward: one read of the logits, one write of the gradient.  The coefficients x of a run stay in registers; what the
// k selected experts get is scattered into a row of shared memory that is zero in between, so an id that a token names twice adds up.
// Measured: 8192 x 256 7.3 us; 65536 x 256 34 us (4 TB/s), sigmoid scores in 97 sequences 43: issue slots two thirds full
// (exponentials, reductions), and a quarter of the shared memory's cycles are conflicts over the rows of `val` and `add`, whose lanes
// lie four apart.
// ------------------------------------------------------------------------------------------
constexpr int BAL_BWD_WARPS = 8;

template <int LPT, int VPL, int VW, bool SIG>
__global__ void __launch_bounds__(32 * BAL_BWD_WARPS) balance_bwd_kernel(const BalanceArgs a) {
  constexpr int TPW = 32 / LPT;
  extern __shared__ __align__(16) float fsm[];
  __shared__ int offsets[BAL_STAGED];
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
  // read a round ahead, the first ones while the offsets arrive
  float v[VPL], next[VPL];
  int next_id = -1, next_at = wa;
  float next_g = 0.f;
  bool next_on = false;
  auto fetch = [&](int t0) {
    const int tt = t0 + grp;
    const bool in = tt < wb;
    next_at = t0;
    load_row<LPT, VPL, VW>(a.logits + (size_t)tt * E, E, l, in, next);
    next_on = in && (!a.token_mask || a.token_mask[tt] != 0);
    if (scores) {
      next_id = in && l < k ? a.topk_ids[(size_t)tt * k + l] : -1;
      next_g = in && l < k ? a.d_topk_w[(size_t)tt * k + l] : 0.f;
    }
  };
  fetch(wa);
  const float g_bal = a.d_losses[0], g_zl = a.d_losses[1];
  const int total = a.tokens[n];
  stage_offsets(a, offsets);
  __syncthreads();
  const SeqTable seqs = seq_table(a, offsets);
  const float g_z = total > 0 ? 2.0f * g_zl / (float)total : 0.f;
  int s = wa < wb ? seqs.of(wa, lane) : n;
  for (int t = wa; t < wb;) {
    int stop = s < n ? seqs.begin(s + 1) : T;
    if (stop <= t) stop = t + 1;   // (offsets that do not ascend)
    const int end = min(stop, wb);
    const bool inside = s >= 0 && s < n;
    float x[VPL];
    const float ns = inside ? (float)a.tokens[s] : 0.f;
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      const int e = expert_at<LPT, VW>(i, l);
      x[i] = inside && e < E ? (float)a.counts[(size_t)s * E + e] : 0.f;
    }
    const float unit = ns > 0.f ? g_bal * (float)E / ((float)k * (float)n) / ns / ns : 0.f;
#pragma unroll
    for (int i = 0; i < VPL; ++i) x[i] *= unit;
    if (next_at != t) fetch(t);
#pragma unroll 1
    for (int t0 = t; t0 < end; t0 += TPW) {
      const int tt = t0 + grp;
#pragma unroll
      for (int i = 0; i < VPL; ++i) v[i] = next[i];
      const bool on = next_on && inside;
      const int id = next_id;
      const float g = next_g;
      fetch(t0 + TPW);
      float soft[VPL], p[SIG ? VPL : 1], sig[SIG ? VPL : 1], inv[2];
      const float lse = row_terms<LPT, VPL, SIG>(v, soft, p, sig, inv);
      // p x; of the selected experts v and g v, v = sigmoid or softmax -- the softmax's terms as they are for renormalised scores, which are
      // the same and whose sum has a reciprocal
      float sum[3] = {0.f, 0.f, 0.f};
      const float v_scale = renorm ? 1.0f : inv[0];
#pragma unroll
      for (int i = 0; i < VPL; ++i) {
        const int e = expert_at<LPT, VW>(i, l);
        if (scores && e < E) val[e] = SIG ? sig[SIG ? i : 0] : soft[i] * v_scale;
        soft[i] *= inv[0];
        if constexpr (SIG) p[i] *= inv[1];
        if (on) sum[0] = fmaf(SIG ? p[SIG ? i : 0] : soft[i], x[i], sum[0]);
      }
      // lane l of the group has the ids l, l + LPT, ..
      auto each = [&](auto body) {
        if (tt < end)
          for (int j = l; j < k; j += LPT) {
            const int e = j == l ? id : a.topk_ids[(size_t)tt * k + j];
            if (e >= 0 && e < E) body(e, j == l ? g : a.d_topk_w[(size_t)tt * k + j]);
          }
      };
      float ref = 0.f;
      bool mine = false;   // a score's gradient that is not zero
      if (scores) {
        // renormalised scores do not see what all their gradients have in common: without it nothing cancels, and one expert gets zero
        if (renorm) ref = __shfl_sync(0xffffffffu, id >= 0 && id < E ? g : 0.f, 0, LPT);
        __syncwarp();
        each([&](int e, float ge) { sum[1] += val[e]; sum[2] = fmaf(ge - ref, val[e], sum[2]); mine |= ge != 0.f; });
      }
      const uint32_t arrives = __ballot_sync(0xffffffffu, mine) >> (grp * LPT) & (0xffffffffu >> (32 - LPT));   // for the group's token
      const bool idle = !on && !arrives;
      group_sums<LPT>(sum);
      float dense = sum[0];
      if (scores) {
        if (renorm) {   // w = v / sum v:  w (g - sum g w)
          const float iz = sum[1] > 0.f ? __fdividef(1.0f, sum[1]) : 0.f, dot = sum[2] * iz;
          each([&](int e, float ge) { atomicAdd(&add[e], val[e] * iz * (ge - ref - dot) * (SIG ? 1.0f - val[e] : 1.0f)); });
        } else if (SIG) {
          each([&](int e, float ge) { atomicAdd(&add[e], ge * val[e] * (1.0f - val[e])); });
        } else {        // a gradient of the same softmax as x
          dense += sum[2];
          each([&](int e, float ge) { atomicAdd(&add[e], ge * val[e]); });
        }
        __syncwarp();
      }
      const float zc = on ? g_z * lse : 0.f;
      float d[VPL];
#pragma unroll
      for (int i = 0; i < VPL; ++i) {
        const int e = expert_at<LPT, VW>(i, l);
        const float pi = SIG ? p[SIG ? i : 0] * (1.0f - sig[SIG ? i : 0]) : soft[i];
        d[i] = fmaf(pi, (on ? x[i] : 0.f) - dense, fmaf(zc, soft[i], scores && e < E ? add[e] : 0.f));
      }
      if (scores) {
        __syncwarp();
        each([&](int e, float) { add[e] = 0.f; });
      }
      float* const out = a.d_logits + (size_t)tt * E;
      if (tt < end && idle) {   // whatever its logits hold
        for (int e = l; e < E; e += LPT) out[e] = 0.f;
      } else if (tt < end) {
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
    if (t < wb) s = seqs.of(t, lane);
  }
}

// ------------------------------------------------------------------------------------------
// Lanes a token and values a lane by the number of experts; vectors of four where rows are whole 16-byte pieces.
struct BalShape { int most, lpt, vpl; };   // experts, at most
constexpr BalShape BAL_SHAPES[] = {{8, 1, 8}, {32, 2, 16}, {64, 4, 16}, {128, 8, 16}, {256, 16, 16}, {512, 32, 16}, {1024, 32, 32}};
constexpr int BAL_NUM_SHAPES = sizeof(BAL_SHAPES) / sizeof(BAL_SHAPES[0]);
static BalShape balance_shape(int E) {
  int i = 0;
  while (i + 1 < BAL_NUM_SHAPES && E > BAL_SHAPES[i].most) ++i;
  return BAL_SHAPES[i];
}
template <int I = 0, class F>
static cudaError_t with_balance_shape(int E, bool vec, F f) {
  constexpr BalShape s = BAL_SHAPES[I];
  if constexpr (I + 1 < BAL_NUM_SHAPES)
    if (E > s.most) return with_balance_shape<I + 1>(E, vec, f);
  constexpr std::integral_constant<int, s.lpt> lpt{};
  constexpr std::integral_constant<int, s.vpl> vpl{};
  return vec ? f(lpt, vpl, std::integral_constant<int, 4>()) : f(lpt, vpl, std::integral_constant<int, 1>());
}

static bool rows_of_vectors(const void* p, int E) { return E % 4 == 0 && (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

static int balance_warps(int E) {
  int warps = balance_warps_most(balance_shape(E).vpl);
  while (warps > 4 && 5 * warps * E * (int)sizeof(int) > BAL_SMEM) warps >>= 1;
  return warps;
}
// Tokens of a block: as many blocks as leave every warp a round of tokens, up to one an SM (few tokens are bound by the latencies of
// a round).
static int balance_chunk(int T, int E) {
  const int round = balance_warps(E) * (32 / balance_shape(E).lpt), even = (T + BAL_MAX_BLOCKS - 1) / BAL_MAX_BLOCKS;
  return even > round ? even : round;
}
int balance_fwd_blocks(int T, int E) {
  const int chunk = balance_chunk(T, E);
  return T > chunk ? (T + chunk - 1) / chunk : 1;
}
size_t balance_scratch_bytes(int E) {
  return (size_t)BAL_MAX_BLOCKS * (sizeof(BalBlock) + 4 * (size_t)E * sizeof(int));
}

cudaError_t launch_balance_fwd(BalanceArgs a, cudaStream_t s, int* launches) {
  a.chunk = balance_chunk(a.T, a.E);
  const int warps = balance_warps(a.E);
  const size_t smem = 5 * (size_t)warps * a.E * sizeof(int);
  const int blocks = balance_fwd_blocks(a.T, a.E);
  return with_balance_shape(a.E, rows_of_vectors(a.logits, a.E), [&](auto lpt, auto vpl, auto vw) -> cudaError_t {
    auto go = [&](auto sig) -> cudaError_t {
      constexpr auto kernel = balance_fwd_kernel<lpt(), vpl(), vw(), sig()>;
      if (smem > 32 * 1024)   // (static shared memory counts too)
        if (cudaError_t e = opt_in_smem<kernel>(BAL_SMEM)) return e;
      ++*launches;
      return launch_dependent(kernel, dim3(blocks), dim3(warps * 32), smem, s, a);
    };
    return (a.mode & GATE_SIGMOID) ? go(std::true_type()) : go(std::false_type());
  });
}

cudaError_t launch_balance_bwd(const BalanceArgs& a, int num_sms, cudaStream_t s, int* launches) {
  const bool vec = rows_of_vectors(a.logits, a.E) && rows_of_vectors(a.d_logits, a.E);
  return with_balance_shape(a.E, vec, [&](auto lpt, auto vpl, auto vw) -> cudaError_t {
    constexpr size_t smem = 2 * sizeof(float) * (size_t)BAL_BWD_WARPS * 32 * vpl();
    const int per_block = BAL_BWD_WARPS * (32 / lpt());   // tokens of a round
    int blocks = (a.T + per_block - 1) / per_block;
    auto go = [&](auto sig) -> cudaError_t {
      constexpr auto kernel = balance_bwd_kernel<lpt(), vpl(), vw(), sig()>;
      if (smem > 32 * 1024)   // (static shared memory counts too)
        if (cudaError_t e = opt_in_smem<kernel>((int)smem)) return e;
      int resident = 0;   // one wave: a second one, a third full, cost as much as the first
      if (cudaError_t e = blocks_per_sm<kernel>(32 * BAL_BWD_WARPS, smem, &resident)) return e;
      ++*launches;
      return launch_dependent(kernel, dim3(blocks < resident * num_sms ? blocks : resident * num_sms), dim3(32 * BAL_BWD_WARPS), smem, s, a);
    };
    return (a.mode & GATE_SIGMOID) ? go(std::true_type()) : go(std::false_type());
  });
}

}  // namespace moe
