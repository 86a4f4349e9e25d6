// Balance loss and z-loss of the router, with their gradient with respect to the logits.
//
// The auxiliary losses that LAEP is compared with: the load share of every expert times the
// router's mean probability of it, over the whole batch (as Mixtral's) or sequence by sequence
// (as DeepSeek-V3's; moe_laep.h says how their coefficients carry over). Per sequence s with n_s valid tokens, c[s,e] assignments of them to
// expert e, and E' live experts:
//   p[t,:] = softmax over the live experts of z[t,:],  P[s,e] = mean of p[t,e] over the sequence
//   f[s,e] = c[s,e] E' / (k n_s)                        (1 where the load is even)
//   loss_balance = coef / N * sum_s sum_e f[s,e] P[s,e]  over the N sequences with a valid token
//   loss_z       = z_coef / M * sum_t lse[t]^2           over the M valid tokens
// The counts carry no gradient, so
//   dz[t,e] = p[t,e] (a_s (f[s,e] - sum_i p[t,i] f[s,i]) + b lse[t]),
//   a_s = g0 coef / (N n_s),  b = 2 g1 z_coef / M.
// Since the probabilities of a token sum to one, f - 1 may stand for f there, and does: f - 1 is the
// exact quotient (c E' - k n_s) / (k n_s), while f - sum p f of an almost even load is a small
// difference of numbers near one.
//
// Sums over tokens run in an order that the arguments alone fix: tokens are cut into chunks of equal
// length, a block sums what its chunk has of one sequence into a row of partial sums, and a second kernel adds a
// sequence's rows. Chunk i and sequence s share row i + s: both only grow along the tokens, so
// no two (chunk, sequence) pairs that overlap have the same sum, and chunks + sequences rows suffice.
#include <math.h>

#include <type_traits>

#include "common.cuh"

MOE_DEV_ERR_DECL

namespace {

// The kernels here let the next one start when their blocks end, not when they start: waiting blocks
// of a next kernel take room that this one's blocks still want (47.6 / 44.9 us for the three kernels at
// T=65536, 256 experts; 23.3 / 21.9 at 16384, 64; 15.9 / 14.5 at 37, 64).
constexpr int kMaxWarps = 24;  // of a block: 80 registers a thread, one block per SM
constexpr int kMaxSeqs = 1 << 20;
constexpr int kMaxTokens = 1 << 30;  // (a chunk's last token plus a round of tokens stays an int)

// Tokens that a warp takes at once (with_lanes's lanes per token).
int warp_tokens(int E) { return E <= 16 ? 8 : E <= 64 ? 4 : 2; }
// Tokens per chunk: one block for each of a GB300's 152 SMs, and few rows of partial sums for
// the second kernel; at least eight, the tokens of one to four warps. For the sums at most kMaxRounds rounds of a
// block's warps: a lane adds fp32 numbers one after another, and addends that are nearly equal round the same
// way each time (2,300 rounds of equal tokens, T = 2^26: 3.4e-5 off).
constexpr int kMaxRounds = 80;
int even_chunk(int T) { return std::max(8, T / 152 + (T % 152 != 0)); }
int chunk_tokens(int T, int E) { return std::min(even_chunk(T), kMaxRounds * kMaxWarps * warp_tokens(E)); }
int chunk_count(int T, int chunk) { return T / chunk + (T % chunk != 0); }
int expert_groups(int E) { return (E + 31) / 32; }

// Workspace: the ticket of the last block, then the partial sums.
struct BalanceWs {
  size_t prob;   // fp32 [rows, E]  sums of p
  size_t count;  // int32 [rows, E] assignments
  size_t n;      // int32 [rows]    valid tokens
  size_t zsq;    // fp32 [rows]     sums of lse^2
  size_t part;   // fp32 [n_seq, groups of 32 experts] sums of f P
  size_t zseq;   // fp32 [n_seq]    sums of lse^2
  size_t total;
};
BalanceWs balance_ws(int T, int E, int n_seq) {
  auto up = [](size_t x) { return (x + 255) & ~size_t(255); };
  const size_t rows = size_t(chunk_count(T, chunk_tokens(T, E))) + size_t(n_seq);
  BalanceWs w{};
  size_t off = 256;
  w.prob = off;
  off += up(rows * E * 4);
  w.count = off;
  off += up(rows * E * 4);
  w.n = off;
  off += up(rows * 4);
  w.zsq = off;
  off += up(rows * 4);
  w.part = off;
  off += up(size_t(n_seq) * expert_groups(E) * 4);
  w.zseq = off;
  off += up(size_t(n_seq) * 4);
  w.total = off;
  return w;
}

struct BalanceParams {
  const float *logits;
  const int32_t *topk_idx;
  const uint8_t *active_mask, *token_mask;
  const int32_t *seq_offsets;  // nullptr: one sequence, [0, T)
  int n_seq, T, E, k, chunk;
  float coef, z_coef;
  // partial sums (BalanceWs)
  int *ticket;
  float *w_prob;
  int32_t *w_count, *w_n;
  float *w_zsq, *w_part, *w_zseq;
  // outputs
  float *loss, *prob, *lse;
  int32_t *counts, *n_tokens;
};

// Tokens [*a, *b) of sequence s, inside [0, T].
__device__ __forceinline__ void sequence_range(const int32_t *off, int s, int T, int *a, int *b) {
  *a = off == nullptr ? 0 : min(max(off[s], 0), T);
  *b = off == nullptr ? T : min(max(off[s + 1], 0), T);
}
// The first sequence that ends behind token t (n_seq: none), by a whole warp: 32 offsets a step (a
// binary search's dependent loads were ~1.3 us of a 4 us kernel at 24 sequences).
__device__ __forceinline__ int first_sequence(const int32_t *off, int n_seq, int t, int lane) {
  if (off == nullptr) return 0;
  int lo = 0, len = n_seq;
  while (len > 0) {
    const int step = (len + 31) / 32, last = (lane + 1) * step - 1;  // of this lane's share
    const unsigned behind = __ballot_sync(0xffffffffu, last >= len || off[lo + last + 1] > t);
    if (behind == 0) return lo + len;
    const int skip = (__ffs(behind) - 1) * step;
    lo += skip;
    len = min(step - 1, len - skip);
  }
  return lo;
}

// The larger value, NaN if either is one.
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
template <int LPT> __device__ __forceinline__ float group_max(float v) {
#pragma unroll
  for (int h = LPT / 2; h > 0; h >>= 1) v = max_nan(v, __shfl_xor_sync(0xffffffffu, v, h));
  return v;
}
// 2^x, 2 ulp; results below 2^-126 are zero.
__device__ __forceinline__ float exp2_quick(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
constexpr float kLog2e = 1.44269504088896341f;
template <int LPT> __device__ __forceinline__ float group_sum(float v) {
#pragma unroll
  for (int h = LPT / 2; h > 0; h >>= 1) v += __shfl_xor_sync(0xffffffffu, v, h);
  return v;
}

// Expert of logit i of lane q, LPT lanes sharing a token's row: VEC, runs of four (rows of whole 16-byte
// vectors); else every LPT-th expert.
template <int LPT, bool VEC> __device__ __forceinline__ int expert_of(int q, int i) {
  return VEC ? 4 * (q + LPT * (i / 4)) + i % 4 : q + LPT * i;
}
// Of lane q's experts, those that are live (bit i: logit i): the mask's bytes are loaded when this is made
// and waited for when bits() is called, other loads in between.
template <int LPT, int NI, bool VEC> struct LiveMask {
  uint8_t m[NI];
  __device__ __forceinline__ LiveMask(const uint8_t *active_mask, int E, int q) {
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int e = expert_of<LPT, VEC>(q, i);
      m[i] = e >= E ? 0 : active_mask == nullptr ? 1 : active_mask[e];
    }
  }
  __device__ __forceinline__ unsigned bits() const {
    unsigned live = 0;
#pragma unroll
    for (int i = 0; i < NI; ++i) live |= m[i] != 0 ? 1u << i : 0u;
    return live;
  }
};
// A token's logits of lane q (not `mine`, or past E: not read, and z is left as it is).
template <int LPT, int NI, bool VEC>
__device__ __forceinline__ void load_row(const float *__restrict__ row, int E, int q, bool mine, float (&z)[NI]) {
#pragma unroll
  for (int i = 0; i < NI; i += VEC ? 4 : 1) {
    const int e = expert_of<LPT, VEC>(q, i);
    if (!mine || e >= E) continue;
    if (VEC) {
      const float4 v = __ldg(reinterpret_cast<const float4 *>(row + e));
      z[i] = v.x;
      z[i + 1] = v.y;
      z[i + 2] = v.z;
      z[i + 3] = v.w;
    } else {
      z[i] = __ldg(row + e);
    }
  }
}
// Lanes' live experts of 32.
__device__ __forceinline__ int count_live(const uint8_t *active_mask, int E, int lane) {
  int n = 0;
  for (int e = lane; e < E; e += 32) n += active_mask == nullptr || active_mask[e] != 0;
  return __reduce_add_sync(0xffffffffu, n);
}

// One lane's share of the tokens that a block sums: LPT lanes hold a token's logits, so that a shuffle
// step serves 32 / LPT of them, and the next tokens' logits, mask and experts load while these are summed. What
// counts is instructions per logit (five: the largest, the exponent's argument, 2^x, two sums; 17 with expf,
// a select per logit for masked ones and a NaN test were 27 us of issue at T=65536, 256 experts,
// where the loads take 10): a row is masked only where some expert is (or E leaves lanes over), and what a
// token that does not count holds is computed with and not added.
// The argument's product with log2 e is fused with the subtraction of the largest logit's; that one's
// rounding is common to the row, so it cancels in p and adds |m| 2^-24 to the log-sum-exp. (Not where the largest
// is so large that this would be no small part of an exponent, a row of the type's lowest value, say: see
// exponents. Which of the two a token gets is its own row's matter, not its neighbours' in the warp.)
template <int NI> __device__ __forceinline__ void exponents(float (&z)[NI], float m) {  // 2^((z - m) log2 e)
  const bool far = fabsf(m) > 65536.f && m != -INFINITY;  // (-inf: no token, nothing of it is used)
  const float c = -m * kLog2e;
  if (__any_sync(0xffffffffu, far)) {
#pragma unroll
    for (int i = 0; i < NI; ++i) z[i] = far ? (z[i] - m) * kLog2e : fmaf(z[i], kLog2e, c);
  } else {
#pragma unroll
    for (int i = 0; i < NI; ++i) z[i] = fmaf(z[i], kLog2e, c);
  }
#pragma unroll
  for (int i = 0; i < NI; ++i) z[i] = exp2_quick(z[i]);
}
template <int LPT, int NI, bool VEC> struct TokenSums {
  static constexpr int TPW = 32 / LPT;               // tokens per warp
  static constexpr int IDS = LPT >= 8 ? 1 : 8 / LPT;  // experts of a token per lane
  float next[NI];
  int ids[IDS];
  int t;
  bool counts;
  // sums over the tokens taken
  float acc[NI], zs;
  int n;
  __device__ __forceinline__ void fetch(const BalanceParams &p, int q, int to) {
    const bool in = t < to;
    counts = in && (p.token_mask == nullptr || p.token_mask[t] != 0);
    load_row<LPT, NI, VEC>(p.logits + size_t(t) * p.E, p.E, q, in, next);
#pragma unroll
    for (int j = 0; j < IDS; ++j) ids[j] = in && q + LPT * j < p.k ? p.topk_idx[size_t(t) * p.k + q + LPT * j] : 0;
  }
  // The lane's first token of those from `a` on.
  __device__ __forceinline__ void start(const BalanceParams &p, int q, int lane, int warp, int a, int to) {
    t = a + warp * TPW + lane / LPT;
    fetch(p, q, to);
  }
  // Sums of tokens [a, b) from the first one fetched; their log-sum-exp, and their experts into hist.
  __device__ __forceinline__ void take(const BalanceParams &p, int q, int warp, int warps, int a, int b, unsigned live,
                                       bool masked, int *hist) {
#pragma unroll
    for (int i = 0; i < NI; ++i) acc[i] = 0.f;
    zs = 0.f;
    n = 0;
    // (whole warps stay in the loop: the sums are warp-wide)
    for (int tb = a + warp * TPW; tb < b; tb += warps * TPW) {
      const int now = t;
      const bool valid = counts && now < b;
      float z[NI];
      int id[IDS];
#pragma unroll
      for (int i = 0; i < NI; ++i) z[i] = next[i];
#pragma unroll
      for (int j = 0; j < IDS; ++j) id[j] = ids[j];
      t += warps * TPW;
      fetch(p, q, b);
      if (masked) {
#pragma unroll
        for (int i = 0; i < NI; ++i) z[i] = live >> i & 1 ? z[i] : -INFINITY;
      }
      float m[4], den[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < NI; ++i) m[i % 4] = i < 4 ? z[i] : max_nan(m[i % 4], z[i]);
      m[0] = group_max<LPT>(max_nan(max_nan(m[0], m[1]), max_nan(m[2], m[3])));
      exponents(z, m[0]);
#pragma unroll
      for (int i = 0; i < NI; ++i) den[i % 4] += z[i];
      den[0] = group_sum<LPT>((den[0] + den[1]) + (den[2] + den[3]));
      if (valid && !(m[0] == -INFINITY)) {
        const float r = __fdividef(1.f, den[0]), lse = m[0] + logf(den[0]);
#pragma unroll
        for (int i = 0; i < NI; ++i) acc[i] = fmaf(z[i], r, acc[i]);
        if (q == 0) {
          p.lse[now] = lse;
          zs = fmaf(lse, lse, zs);
          ++n;
        }
#pragma unroll
        for (int j = 0; j < IDS; ++j) {
          if (q + LPT * j >= p.k) continue;
          if (id[j] >= 0 && id[j] < p.E) atomicAdd(&hist[id[j]], 1);
          else dev_flag(&g_dev_err, MOE_DEV_BAD_EXPERT);
        }
      } else if (q == 0 && now < b) {
        p.lse[now] = -INFINITY;
      }
    }
  }
  // The warp's sums into shared memory.
  __device__ __forceinline__ void leave(int q, int lane, float *prob, float *z, int *count) {
#pragma unroll
    for (int i = 0; i < NI; ++i) {
#pragma unroll
      for (int h = LPT; h < 32; h <<= 1) acc[i] += __shfl_xor_sync(0xffffffffu, acc[i], h);
      if (lane < LPT) prob[expert_of<LPT, VEC>(q, i)] = acc[i];
    }
    zs = group_sum<32>(zs);
    n = __reduce_add_sync(0xffffffffu, n);
    if (lane == 0) {
      *z = zs;
      *count = n;
    }
  }
};

// Log-sum-exp of every token and the partial sums of a block's chunk.
template <int LPT, int NI, bool VEC>
__global__ void __launch_bounds__(32 * kMaxWarps, 1) balance_stats_kernel(const BalanceParams p) {
  __shared__ float s_prob[kMaxWarps][256];
  __shared__ int s_hist[256];
  __shared__ int s_n[kMaxWarps];
  __shared__ float s_z[kMaxWarps];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, q = lane % LPT;
  const int threads = blockDim.x, warps = threads >> 5;
  for (int e = tid; e < 256; e += threads) s_hist[e] = 0;
  pdl_wait();
  if (blockIdx.x == 0 && tid == 0) *p.ticket = 0;
  const int t0 = blockIdx.x * p.chunk, t1 = min(p.T, t0 + p.chunk);
  if (t0 >= t1) return;  // (no tokens at all)
  // The loads that do not wait for the sequences start first (the chunk's first tokens are fetched as
  // if they were in one).
  const LiveMask<LPT, NI, VEC> mask(p.active_mask, p.E, q);
  TokenSums<LPT, NI, VEC> sums;
  sums.start(p, q, lane, warp, t0, t1);
  int fetched = t0;
  int s = first_sequence(p.seq_offsets, p.n_seq, t0, lane);
  const unsigned live = mask.bits();
  const bool masked = __any_sync(0xffffffffu, live != (1u << NI) - 1u);
  __syncthreads();
  int cur = t0;
  for (; s < p.n_seq && cur < t1; ++s) {
    int a, b;
    sequence_range(p.seq_offsets, s, p.T, &a, &b);
    if (a >= t1) break;
    a = max(a, cur);
    b = min(b, t1);
    for (int t = cur + tid; t < a; t += threads) p.lse[t] = -INFINITY;  // between sequences
    cur = max(cur, a);
    if (a >= b) continue;
    if (fetched != a) sums.start(p, q, lane, warp, a, b);
    fetched = -1;
    sums.take(p, q, warp, warps, a, b, live, masked, s_hist);
    sums.leave(q, lane, s_prob[warp], &s_z[warp], &s_n[warp]);
    __syncthreads();
    const size_t row = size_t(blockIdx.x) + s;
    for (int e = tid; e < p.E; e += threads) {
      float v = 0.f;
#pragma unroll 8
      for (int w = 0; w < warps; ++w) v += s_prob[w][e];
      p.w_prob[row * p.E + e] = v;
      p.w_count[row * p.E + e] = s_hist[e];
      s_hist[e] = 0;
    }
    if (warp == 0) {
      const float zs = group_sum<32>(lane < warps ? s_z[lane] : 0.f);
      const int n = __reduce_add_sync(0xffffffffu, lane < warps ? s_n[lane] : 0);
      if (lane == 0) {
        p.w_zsq[row] = zs;
        p.w_n[row] = n;
      }
    }
    __syncthreads();
    cur = b;
  }
  for (int t = cur + tid; t < t1; t += threads) p.lse[t] = -INFINITY;  // behind the last sequence
}

// The whole forward call in one block, for few tokens and sequences (see one_block): a launch less.
template <int LPT, int NI, bool VEC>
__global__ void __launch_bounds__(32 * kMaxWarps, 1) balance_one_block_kernel(const BalanceParams p) {
  __shared__ float s_prob[kMaxWarps][256];
  __shared__ int s_hist[256];
  __shared__ int s_n[kMaxWarps];
  __shared__ float s_z[kMaxWarps], s_part[kMaxWarps];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, q = lane % LPT;
  const int threads = blockDim.x, warps = threads >> 5;
  for (int e = tid; e < 256; e += threads) s_hist[e] = 0;
  pdl_wait();
  const LiveMask<LPT, NI, VEC> mask(p.active_mask, p.E, q);
  TokenSums<LPT, NI, VEC> sums;
  sums.start(p, q, lane, warp, 0, p.T);
  int fetched = 0;
  const int live_all = count_live(p.active_mask, p.E, lane);
  const unsigned live = mask.bits();
  const bool masked = __any_sync(0xffffffffu, live != (1u << NI) - 1u);
  __syncthreads();
  int cur = 0, all = 0, seqs = 0;
  float part = 0.f, zsum = 0.f;  // (of thread 0)
  for (int s = 0; s < p.n_seq; ++s) {
    int a, b;
    sequence_range(p.seq_offsets, s, p.T, &a, &b);
    if (p.seq_offsets != nullptr && tid == 0 &&
        (p.seq_offsets[s] < 0 || p.seq_offsets[s + 1] < p.seq_offsets[s] || p.seq_offsets[s + 1] > p.T))
      dev_flag(&g_dev_err, MOE_DEV_BAD_OFFSETS);
    a = max(a, cur);
    for (int t = cur + tid; t < a; t += threads) p.lse[t] = -INFINITY;  // between sequences
    cur = max(cur, a);
    if (a < b) {
      if (fetched != a) sums.start(p, q, lane, warp, a, b);
      fetched = -1;
    }
    sums.take(p, q, warp, warps, a, b, live, masked, s_hist);  // (no token: zeros)
    sums.leave(q, lane, s_prob[warp], &s_z[warp], &s_n[warp]);
    __syncthreads();
    const int n = __reduce_add_sync(0xffffffffu, lane < warps ? s_n[lane] : 0);
    float mine = 0.f;
    for (int e = tid; e < p.E; e += threads) {
      float v = 0.f;
#pragma unroll 8
      for (int w = 0; w < warps; ++w) v += s_prob[w][e];
      const int c = s_hist[e];
      s_hist[e] = 0;
      const float prob = n > 0 ? v / float(n) : 0.f;
      p.counts[size_t(s) * p.E + e] = c;
      p.prob[size_t(s) * p.E + e] = prob;
      if (n > 0) mine += float(int64_t(c) * live_all) / float(int64_t(p.k) * n) * prob;
    }
    mine = group_sum<32>(mine);
    if (lane == 0) s_part[warp] = mine;
    const float zs = group_sum<32>(lane < warps ? s_z[lane] : 0.f);
    __syncthreads();
    const float of_s = group_sum<32>(lane < warps ? s_part[lane] : 0.f);
    if (tid == 0) p.n_tokens[s] = n;
    part += of_s;
    zsum += zs;
    all += n;
    seqs += n > 0;
    cur = max(cur, b);
  }
  for (int t = cur + tid; t < p.T; t += threads) p.lse[t] = -INFINITY;  // behind the last sequence
  if (tid == 0) {
    p.loss[0] = seqs > 0 ? p.coef * (part / float(seqs)) : 0.f;
    p.loss[1] = all > 0 && p.z_coef != 0.f ? p.z_coef * (zsum / float(all)) : 0.f;
    p.n_tokens[p.n_seq] = all;
    p.n_tokens[p.n_seq + 1] = seqs;
  }
}

// Sums of one sequence's rows for 32 experts (blockIdx.x = sequence * groups + group; a warp
// takes every (blockDim.x / 32)th row), its counts, mean probabilities and share of the loss. The
// last block to finish adds the shares, always in the same order. (Sums of few terms are fp32: a chain of
// fp64 additions and quotients took ~10 us here, whatever the size.)
constexpr int kRun = 64;
__global__ void __launch_bounds__(1024) balance_reduce_kernel(const BalanceParams p) {
  __shared__ float s_p[32][33];
  __shared__ int s_c[32][33];
  __shared__ int s_n[32], s_m[32];
  __shared__ float s_d[32], s_z[32];
  __shared__ int s_last;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  pdl_wait();
  const int groups = (p.E + 31) / 32;
  const int s = blockIdx.x / groups, grp = blockIdx.x - s * groups, e = grp * 32 + lane;
  int a, b;
  sequence_range(p.seq_offsets, s, p.T, &a, &b);
  if (p.seq_offsets != nullptr && threadIdx.x == 0 &&
      (p.seq_offsets[s] < 0 || p.seq_offsets[s + 1] < p.seq_offsets[s] || p.seq_offsets[s + 1] > p.T))
    dev_flag(&g_dev_err, MOE_DEV_BAD_OFFSETS);
  const int live_all = warp == 0 ? count_live(p.active_mask, p.E, lane) : 0;
  const int c0 = a / p.chunk, c1 = a < b ? (b - 1) / p.chunk : c0 - 1;  // its chunks
  float v = 0.f, zs = 0.f;
  int c = 0, n = 0;
  // (in runs of kRun rows, whose sums are then added: the number of roundings one after another)
  for (int i = c0 + int(threadIdx.x); i <= c1;) {
    float z = 0.f;
    for (int to = min(c1, i + (kRun - 1) * int(blockDim.x)); i <= to; i += blockDim.x) {
      n += p.w_n[size_t(i) + s];
      z += p.w_zsq[size_t(i) + s];
    }
    zs += z;
  }
  if (e < p.E) {
    for (int i = c0 + warp; i <= c1;) {
      float x = 0.f;
#pragma unroll 8
      for (int to = min(c1, i + (kRun - 1) * warps); i <= to; i += warps) {
        const size_t at = (size_t(i) + s) * p.E + e;
        x += p.w_prob[at];
        c += p.w_count[at];
      }
      v += x;
    }
  }
  s_p[warp][lane] = v;
  s_c[warp][lane] = c;
  n = __reduce_add_sync(0xffffffffu, n);
  zs = group_sum<32>(zs);
  if (lane == 0) {
    s_n[warp] = n;
    s_z[warp] = zs;
  }
  __syncthreads();
  if (warp == 0) {
    v = 0.f;
    c = 0;
#pragma unroll 8
    for (int w = 0; w < warps; ++w) {
      v += s_p[w][lane];
      c += s_c[w][lane];
    }
    n = __reduce_add_sync(0xffffffffu, lane < warps ? s_n[lane] : 0);
    zs = group_sum<32>(lane < warps ? s_z[lane] : 0.f);
    const float prob = n > 0 ? v / float(n) : 0.f;
    float part = 0.f;
    if (e < p.E) {
      p.counts[size_t(s) * p.E + e] = c;
      p.prob[size_t(s) * p.E + e] = prob;
      if (n > 0) part = float(int64_t(c) * live_all) / float(int64_t(p.k) * n) * prob;
    }
    part = group_sum<32>(part);
    if (lane == 0) {
      p.w_part[size_t(s) * groups + grp] = part;
      if (grp == 0) {
        p.n_tokens[s] = n;
        p.w_zseq[s] = zs;
      }
      __threadfence();
      s_last = atomicAdd(p.ticket, 1) == int(gridDim.x) - 1;
    }
  }
  __syncthreads();
  if (!s_last) return;
  __threadfence();
  double part = 0.0, zq = 0.0;  // (up to 2^23 terms)
  int m = 0, seqs = 0;
  for (int i = threadIdx.x; i < p.n_seq * groups; i += blockDim.x) part += double(__ldcg(p.w_part + i));
  for (int i = threadIdx.x; i < p.n_seq; i += blockDim.x) {
    const int ni = __ldcg(p.n_tokens + i);
    m += ni;
    seqs += ni > 0;
    zq += double(__ldcg(p.w_zseq + i));
  }
  const float wpart = group_sum<32>(float(part)), wz = group_sum<32>(float(zq));
  m = __reduce_add_sync(0xffffffffu, m);
  seqs = __reduce_add_sync(0xffffffffu, seqs);
  if (lane == 0) {
    s_d[warp] = wpart;
    s_z[warp] = wz;
    s_n[warp] = m;
    s_m[warp] = seqs;
  }
  __syncthreads();
  if (warp == 0) {
    const float d = group_sum<32>(lane < warps ? s_d[lane] : 0.f), z = group_sum<32>(lane < warps ? s_z[lane] : 0.f);
    m = __reduce_add_sync(0xffffffffu, lane < warps ? s_n[lane] : 0);
    seqs = __reduce_add_sync(0xffffffffu, lane < warps ? s_m[lane] : 0);
    if (lane == 0) {
      p.loss[0] = seqs > 0 ? p.coef * (d / float(seqs)) : 0.f;
      p.loss[1] = m > 0 && p.z_coef != 0.f ? p.z_coef * (z / float(m)) : 0.f;
      p.n_tokens[p.n_seq] = m;
      p.n_tokens[p.n_seq + 1] = seqs;
    }
  }
}

// dz, from the kept log-sum-exp. Its rounding (of a number that may be much larger than one) is
// common to a token's probabilities: dividing by their sum takes it out. A warp walks the sequences of
// its tokens by itself, with the sequence's f - 1 of its experts in registers.
template <int LPT, int NI, bool VEC>
__global__ void __launch_bounds__(32 * kMaxWarps, 1) balance_bwd_kernel(
    const float *__restrict__ logits, const uint8_t *__restrict__ active_mask,
    const int32_t *__restrict__ seq_offsets, int n_seq, int T, int E, int k, int chunk, float coef, float z_coef,
    const int32_t *__restrict__ counts, const int32_t *__restrict__ n_tokens,
    const float *__restrict__ lse, const float *__restrict__ d_loss, float *__restrict__ dz) {
  constexpr int TPW = 32 / LPT;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5, q = lane % LPT;
  pdl_wait();
  const int t0 = blockIdx.x * chunk, t1 = min(T, t0 + chunk);
  if (t0 >= t1) return;
  // as in the sums, the loads that do not wait for the sequences first
  const LiveMask<LPT, NI, VEC> mask(active_mask, E, q);
  int t = t0 + warp * TPW + lane / LPT;
  float l, next[NI] = {};
  auto fetch = [&](int to) {
    l = t < to ? lse[t] : -INFINITY;
    load_row<LPT, NI, VEC>(logits + size_t(t) * E, E, q, t < to, next);
  };
  fetch(t1);
  int fetched = t0;
  const int m = n_tokens[n_seq], seqs = n_tokens[n_seq + 1];
  const float g0 = d_loss != nullptr ? d_loss[0] : 1.f, g1 = d_loss != nullptr ? d_loss[1] : 1.f;
  int s = first_sequence(seq_offsets, n_seq, t0, lane);
  const int live_all = count_live(active_mask, E, lane);
  const unsigned live = mask.bits();
  const bool masked = __any_sync(0xffffffffu, live != (1u << NI) - 1u);
  const float bz = m > 0 ? 2.f * z_coef * g1 / float(m) : 0.f;
  auto zero = [&](int a, int b) {  // rows of tokens in no sequence
    for (int t = a + warp; t < b; t += warps)
      for (int e = lane; e < E; e += 32) dz[size_t(t) * E + e] = 0.f;
  };
  int cur = t0;
  for (; s < n_seq && cur < t1; ++s) {
    int a, b;
    sequence_range(seq_offsets, s, T, &a, &b);
    if (a >= t1) break;
    a = max(a, cur);
    b = min(b, t1);
    zero(cur, a);
    cur = max(cur, a);
    if (a >= b) continue;
    if (fetched != a) {
      t = a + warp * TPW + lane / LPT;
      fetch(b);
    }
    fetched = -1;
    const int n = n_tokens[s];
    const float as = n > 0 && seqs > 0 ? coef * g0 / (float(seqs) * float(n)) : 0.f;
    float f[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      f[i] = 0.f;
      if ((live >> i & 1) && n > 0) {
        const int64_t all = int64_t(k) * n, c = counts[size_t(s) * E + expert_of<LPT, VEC>(q, i)];
        f[i] = float(c * live_all - all) / float(all);
      }
    }
    for (int tb = a + warp * TPW; tb < b; tb += warps * TPW) {
      const int tn = t;
      const float ln = l;
      float z[NI], s0[2] = {0.f, 0.f}, s1[2] = {0.f, 0.f};
#pragma unroll
      for (int i = 0; i < NI; ++i) z[i] = next[i];
      t += warps * TPW;
      fetch(b);
      if (masked) {
#pragma unroll
        for (int i = 0; i < NI; ++i) z[i] = live >> i & 1 ? z[i] : -INFINITY;
      }
      exponents(z, ln);
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        s0[i % 2] += z[i];
        s1[i % 2] = fmaf(z[i], f[i], s1[i % 2]);
      }
      s0[0] = group_sum<LPT>(s0[0] + s0[1]);
      s1[0] = group_sum<LPT>(s1[0] + s1[1]);
      if (tn >= b) continue;
      // p (a f + base), p = z / s0; a token that does not count gets zeros whatever it holds
      const float r = __fdividef(1.f, s0[0]), ar = as * r, base = r * fmaf(bz, ln, -as * (s1[0] * r));
      const bool some = !(ln == -INFINITY);
#pragma unroll
      for (int i = 0; i < NI; ++i) z[i] = some ? z[i] * fmaf(ar, f[i], base) : 0.f;
      float *dst = dz + size_t(tn) * E;
#pragma unroll
      for (int i = 0; i < NI; i += VEC ? 4 : 1) {
        const int e = expert_of<LPT, VEC>(q, i);
        if (e >= E) continue;
        if (VEC) *reinterpret_cast<float4 *>(dst + e) = make_float4(z[i], z[i + 1], z[i + 2], z[i + 3]);
        else dst[e] = z[i];
      }
    }
    cur = b;
  }
  zero(cur, t1);
}

// Warps of a block: enough for its tokens at once, up to what an SM holds.
int block_warps(int tokens, int E) { return std::min(kMaxWarps, (tokens + warp_tokens(E) - 1) / warp_tokens(E)); }
// The forward in one block, a launch less than the two kernels: up to four rounds of its warps' tokens, and three
// sequences, which it takes one after another (~2 us each, where the two kernels take them side by side). Forward and
// backward replayed from a graph, us, two kernels / one block, at 16, 37, 100, 200 tokens of 64 experts:
//   1 sequence   10.4 / 5.9    11.3 / 6.3    11.9 / 7.5    11.9 / 8.0
//   3 sequences  12.9 / 10.5   13.2 / 10.8   13.7 / 12.0   14.1 / 12.6
//   4 sequences  13.3 / 12.4   12.6 / 12.4   12.8 / 14.1   13.8 / 15.3
//   6 sequences  15.8 / 17.0   13.3 / 16.0   13.6 / 18.1   14.2 / 19.2
// and with 256 experts 16.7 / 15.5 for 37 tokens in 3 sequences, 16.9 / 17.8 in 4. In the tokens the two meet at four
// rounds: 11.8 / 9.4 at 384 of 64 experts in 1 sequence, 11.9 / 13.6 in 3.
bool one_block(int T, int E, int n_seq) { return T <= 4 * kMaxWarps * warp_tokens(E) && n_seq <= 3; }
// Lanes per token and logits per lane for E experts; whether a row of logits is whole 16-byte vectors.
template <typename F> void with_lanes(int E, bool vec, F f) {
  auto pick = [&](auto v) {
    using std::integral_constant;
    if (E <= 16) f(integral_constant<int, 4>(), integral_constant<int, 4>(), v);
    else if (E <= 64) f(integral_constant<int, 8>(), integral_constant<int, 8>(), v);
    else if (E <= 128) f(integral_constant<int, 16>(), integral_constant<int, 8>(), v);
    else if (E <= 192) f(integral_constant<int, 16>(), integral_constant<int, 12>(), v);
    else f(integral_constant<int, 16>(), integral_constant<int, 16>(), v);
  };
  if (vec) pick(std::true_type());
  else pick(std::false_type());
}
bool whole_vectors(int E, const void *a, const void *b) { return E % 4 == 0 && moe::aligned16(a) && moe::aligned16(b); }

int check_sizes(const char *fn, int T, int E, int k, int n_seq, const void *seq_offsets, float coef, float z_coef) {
  if (E < 1 || E > 256) return moe::set_error(MOE_ERR_UNSUPPORTED, "%s: E=%d not in [1,256]", fn, E);
  if (k < 1 || k > 8 || k > E) return moe::set_error(MOE_ERR_UNSUPPORTED, "%s: k=%d", fn, k);
  if (T < 0 || T > kMaxTokens || n_seq < 1 || n_seq > kMaxSeqs)
    return moe::set_error(MOE_ERR_ARG, "%s: T=%d n_seq=%d", fn, T, n_seq);
  if (n_seq > 1 && !seq_offsets) return moe::set_error(MOE_ERR_ARG, "%s: n_seq=%d without seq_offsets", fn, n_seq);
  if (!isfinite(coef) || !isfinite(z_coef)) return moe::set_error(MOE_ERR_ARG, "%s: coefficients", fn);
  return MOE_OK;
}

}  // namespace

namespace moe {
MOE_DEV_ERR_DEFINE_READER(balance_dev_error)
}

extern "C" {

size_t moe_balance_workspace_size(int T, int E, int n_seq) {
  if (T < 0 || E <= 0 || n_seq <= 0) return 0;
  return balance_ws(T, E, n_seq).total;
}

int moe_balance_loss(const float *logits, const int32_t *topk_idx, const uint8_t *active_mask,
                     const uint8_t *token_mask, const int32_t *seq_offsets, int n_seq, int T, int E,
                     int k, float coef, float z_coef, float *loss, int32_t *counts, float *prob,
                     int32_t *n_tokens, float *lse, void *ws, size_t ws_bytes, moe_stream_t stream) {
  const char *fn = "moe_balance_loss";
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (int st = check_sizes(fn, T, E, k, n_seq, seq_offsets, coef, z_coef)) return st;
  if (!loss || !counts || !prob || !n_tokens || (T > 0 && (!logits || !topk_idx || !lse)))
    return moe::set_error(MOE_ERR_ARG, "%s: null pointer", fn);
  const BalanceWs w = balance_ws(T, E, n_seq);
  if (!ws || ws_bytes < w.total) return moe::set_error(MOE_ERR_WORKSPACE, "%s: workspace", fn);
  if (!moe::aligned16(ws)) return moe::set_error(MOE_ERR_ARG, "%s: ws alignment", fn);
  char *base = static_cast<char *>(ws);
  BalanceParams p{};
  p.logits = logits;
  p.topk_idx = topk_idx;
  p.active_mask = active_mask;
  p.token_mask = token_mask;
  p.seq_offsets = seq_offsets;
  p.n_seq = n_seq;
  p.T = T;
  p.E = E;
  p.k = k;
  p.chunk = chunk_tokens(T, E);
  p.coef = coef;
  p.z_coef = z_coef;
  p.ticket = reinterpret_cast<int *>(base);
  p.w_prob = reinterpret_cast<float *>(base + w.prob);
  p.w_count = reinterpret_cast<int32_t *>(base + w.count);
  p.w_n = reinterpret_cast<int32_t *>(base + w.n);
  p.w_zsq = reinterpret_cast<float *>(base + w.zsq);
  p.w_part = reinterpret_cast<float *>(base + w.part);
  p.w_zseq = reinterpret_cast<float *>(base + w.zseq);
  p.loss = loss;
  p.prob = prob;
  p.lse = lse;
  p.counts = counts;
  p.n_tokens = n_tokens;
  if (one_block(T, E, n_seq)) {
    const int warps = std::max(8, block_warps(T, E));  // (at least a thread per expert)
    with_lanes(E, whole_vectors(E, logits, logits), [&](auto lpt, auto ni, auto vec) {
      MOE_LAUNCH("balance_one_block", s,
                 moe::launch_dep(balance_one_block_kernel<lpt.value, ni.value, vec.value>, 1, 32 * warps, 0, s, p));
    });
    return moe::launch_status("moe_balance_loss: one block");
  }
  const int chunks = chunk_count(T, p.chunk), grid = std::max(1, chunks), stat_threads = 32 * block_warps(p.chunk, E);
  with_lanes(E, whole_vectors(E, logits, logits), [&](auto lpt, auto ni, auto vec) {
    MOE_LAUNCH("balance_stats", s,
               moe::launch_dep(balance_stats_kernel<lpt.value, ni.value, vec.value>, grid, stat_threads, 0, s, p));
  });
  if (int st = moe::launch_status("moe_balance_loss: token sums")) return st;
  // a warp per ~4 of a sequence's rows, about
  const int rows = chunks / n_seq + 1, threads = 32 * std::max(4, std::min(32, rows / 4));
  MOE_LAUNCH("balance_reduce", s, moe::launch_dep(balance_reduce_kernel, n_seq * expert_groups(E), threads, 0, s, p));
  return moe::launch_status("moe_balance_loss: reduction");
}

int moe_balance_loss_bwd(const float *logits, const uint8_t *active_mask, const int32_t *seq_offsets,
                         int n_seq, int T, int E, int k, float coef, float z_coef,
                         const int32_t *counts, const int32_t *n_tokens, const float *lse,
                         const float *d_loss, float *dz, moe_stream_t stream) {
  const char *fn = "moe_balance_loss_bwd";
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (int st = check_sizes(fn, T, E, k, n_seq, seq_offsets, coef, z_coef)) return st;
  if (T == 0) return MOE_OK;
  if (!logits || !counts || !n_tokens || !lse || !dz) return moe::set_error(MOE_ERR_ARG, "%s: null pointer", fn);
  const int chunk = even_chunk(T);
  with_lanes(E, whole_vectors(E, logits, dz), [&](auto lpt, auto ni, auto vec) {
    MOE_LAUNCH("balance_bwd", s,
               moe::launch_dep(balance_bwd_kernel<lpt.value, ni.value, vec.value>, chunk_count(T, chunk), 32 * block_warps(chunk, E), 0, s, logits,
                               active_mask, seq_offsets, n_seq, T, E, k, chunk, coef, z_coef, counts, n_tokens, lse, d_loss,
                               dz));
  });
  return moe::launch_status("moe_balance_loss_bwd: launch");
}

}  // extern "C"
