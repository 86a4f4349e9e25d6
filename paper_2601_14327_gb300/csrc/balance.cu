// Balance loss and z-loss of the router, with their gradient with respect to the logits.
//
// The auxiliary losses that LAEP is compared with: the load share of every expert times the
// router's mean probability of it, over the whole batch (the Mixtral form) or sequence by sequence
// (the DeepSeek-V3 form). Per sequence s with n_s valid tokens, c[s,e] assignments of them to
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

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxSeqs = 1 << 20;

// Tokens per chunk: four chunks per SM of a GB300 (152), at least a token per warp.
int chunk_tokens(int T) { return std::max(kWarps, (T + 607) / 608); }
int chunk_count(int T) { return (T + chunk_tokens(T) - 1) / chunk_tokens(T); }
int expert_groups(int E) { return (E + 31) / 32; }

// Workspace: the ticket of the last block, then the partial sums.
struct BalanceWs {
  size_t prob;   // fp32 [rows, E]  sums of p
  size_t count;  // int32 [rows, E] assignments
  size_t n;      // int32 [rows]    valid tokens
  size_t zsq;    // fp64 [rows]     sums of lse^2
  size_t part;   // fp64 [n_seq, groups of 32 experts] sums of f P
  size_t zseq;   // fp64 [n_seq]    sums of lse^2
  size_t total;
};
BalanceWs balance_ws(int T, int E, int n_seq) {
  auto up = [](size_t x) { return (x + 255) & ~size_t(255); };
  const size_t rows = size_t(chunk_count(T)) + size_t(n_seq);
  BalanceWs w{};
  size_t off = 256;
  w.prob = off;
  off += up(rows * E * 4);
  w.count = off;
  off += up(rows * E * 4);
  w.n = off;
  off += up(rows * 4);
  w.zsq = off;
  off += up(rows * 8);
  w.part = off;
  off += up(size_t(n_seq) * expert_groups(E) * 8);
  w.zseq = off;
  off += up(size_t(n_seq) * 8);
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
  double *w_zsq, *w_part, *w_zseq;
  // outputs
  float *loss, *prob, *lse;
  int32_t *counts, *n_tokens;
};

// Tokens [*a, *b) of sequence s, inside [0, T].
__device__ __forceinline__ void sequence_range(const int32_t *off, int s, int T, int *a, int *b) {
  *a = off == nullptr ? 0 : min(max(off[s], 0), T);
  *b = off == nullptr ? T : min(max(off[s + 1], 0), T);
}
// The first sequence that ends behind token t (n_seq: none).
__device__ __forceinline__ int first_sequence(const int32_t *off, int n_seq, int T, int t) {
  if (off == nullptr) return 0;
  int lo = 0, hi = n_seq;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (off[mid + 1] > t) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

template <int LPT> __device__ __forceinline__ float group_max(float v) {
#pragma unroll
  for (int h = LPT / 2; h > 0; h >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, h));
  return v;
}
template <int LPT> __device__ __forceinline__ float group_sum(float v) {
#pragma unroll
  for (int h = LPT / 2; h > 0; h >>= 1) v += __shfl_xor_sync(0xffffffffu, v, h);
  return v;
}

// Log-sum-exp of every token and the partial sums of its chunk. LPT lanes share a token, lane q
// holding the logits of experts q + LPT i.
template <int LPT, int NI>
__global__ void __launch_bounds__(kThreads) balance_stats_kernel(const BalanceParams p) {
  __shared__ float s_prob[kWarps][256];
  __shared__ int s_hist[256];
  __shared__ int s_n[kWarps];
  __shared__ float s_z[kWarps];
  __shared__ int s_first;
  constexpr int TPW = 32 / LPT;  // tokens per warp
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, q = lane % LPT;
  for (int e = tid; e < 256; e += kThreads) s_hist[e] = 0;
  pdl_start();
  if (blockIdx.x == 0 && tid == 0) *p.ticket = 0;
  const int t0 = blockIdx.x * p.chunk, t1 = min(p.T, t0 + p.chunk);
  if (t0 >= t1) return;  // (no tokens at all)
  if (tid == 0) s_first = first_sequence(p.seq_offsets, p.n_seq, p.T, t0);
  bool live[NI];
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int e = q + LPT * i;
    live[i] = e < p.E && (p.active_mask == nullptr || p.active_mask[e] != 0);
  }
  __syncthreads();
  int cur = t0;
  for (int s = s_first; s < p.n_seq && cur < t1; ++s) {
    int a, b;
    sequence_range(p.seq_offsets, s, p.T, &a, &b);
    if (a >= t1) break;
    a = max(a, cur);
    b = min(b, t1);
    for (int t = cur + tid; t < a; t += kThreads) p.lse[t] = -INFINITY;  // between sequences
    cur = max(cur, a);
    if (a >= b) continue;
    float acc[NI] = {};
    float zs = 0.f;
    int n = 0;
    // (whole warps stay in the loop: the sums are warp-wide)
    for (int tb = a + warp * TPW; tb < b; tb += kWarps * TPW) {
      const int t = tb + lane / LPT;
      const bool mine = t < b && (p.token_mask == nullptr || p.token_mask[t] != 0);
      float z[NI], m = -INFINITY;
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        z[i] = mine && live[i] ? p.logits[size_t(t) * p.E + q + LPT * i] : -INFINITY;
      }
#pragma unroll
      for (int i = 0; i < NI; ++i) m = z[i] != z[i] ? INFINITY : fmaxf(m, z[i]);  // a NaN stays one in the sum
      m = group_max<LPT>(m);
      float den = 0.f;
      const bool some = m > -INFINITY;
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        z[i] = some ? expf(z[i] - m) : 0.f;
        den += z[i];
      }
      den = group_sum<LPT>(den);
      const float lse = some ? m + logf(den) : -INFINITY;
      if (q == 0 && t < b) p.lse[t] = lse;
      if (some) {
        const float r = 1.f / den;
#pragma unroll
        for (int i = 0; i < NI; ++i) acc[i] = fmaf(z[i], r, acc[i]);
        if (q == 0) {
          zs = fmaf(lse, lse, zs);
          ++n;
        }
        for (int j = q; j < p.k; j += LPT) {
          const int e = p.topk_idx[size_t(t) * p.k + j];
          if (e >= 0 && e < p.E) atomicAdd(&s_hist[e], 1);
          else dev_flag(&g_dev_err, MOE_DEV_BAD_EXPERT);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < NI; ++i) {
#pragma unroll
      for (int h = LPT; h < 32; h <<= 1) acc[i] += __shfl_xor_sync(0xffffffffu, acc[i], h);
      if (lane < LPT) s_prob[warp][q + LPT * i] = acc[i];
    }
    zs = group_sum<32>(zs);
    n = __reduce_add_sync(0xffffffffu, n);
    if (lane == 0) {
      s_z[warp] = zs;
      s_n[warp] = n;
    }
    __syncthreads();
    const size_t row = size_t(blockIdx.x) + s;
    for (int e = tid; e < p.E; e += kThreads) {
      float v = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) v += s_prob[w][e];
      p.w_prob[row * p.E + e] = v;
      p.w_count[row * p.E + e] = s_hist[e];
      s_hist[e] = 0;
    }
    if (tid == 0) {
      double z = 0.0;
      int m = 0;
      for (int w = 0; w < kWarps; ++w) {
        z += double(s_z[w]);
        m += s_n[w];
      }
      p.w_zsq[row] = z;
      p.w_n[row] = m;
    }
    __syncthreads();
    cur = b;
  }
  for (int t = cur + tid; t < t1; t += kThreads) p.lse[t] = -INFINITY;  // behind the last sequence
}

// Sums of one sequence's rows for 32 experts (blockIdx.x = sequence * groups + group; a warp
// takes every (blockDim.x / 32)th row), its counts, mean probabilities and share of the loss. The
// last block to finish adds the shares, always in the same order.
__global__ void __launch_bounds__(1024) balance_reduce_kernel(const BalanceParams p) {
  __shared__ float s_p[32][33];
  __shared__ int s_c[32][33];
  __shared__ int s_n[32];
  __shared__ double s_d[32], s_z[32];
  __shared__ int s_last;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  pdl_start();
  const int groups = (p.E + 31) / 32;
  const int s = blockIdx.x / groups, grp = blockIdx.x - s * groups, e = grp * 32 + lane;
  int a, b;
  sequence_range(p.seq_offsets, s, p.T, &a, &b);
  if (p.seq_offsets != nullptr && threadIdx.x == 0 &&
      (p.seq_offsets[s] < 0 || p.seq_offsets[s + 1] < p.seq_offsets[s] || p.seq_offsets[s + 1] > p.T))
    dev_flag(&g_dev_err, MOE_DEV_BAD_OFFSETS);
  const int c0 = a / p.chunk, c1 = a < b ? (b - 1) / p.chunk : c0 - 1;  // its chunks
  float v = 0.f;
  int c = 0, n = 0;
  double zs = 0.0;
  for (int i = c0 + warp; i <= c1; i += warps) {
    const size_t row = size_t(i) + s;
    if (e < p.E) {
      v += p.w_prob[row * p.E + e];
      c += p.w_count[row * p.E + e];
    }
    if (lane == 0) {
      n += p.w_n[row];
      zs += p.w_zsq[row];
    }
  }
  s_p[warp][lane] = v;
  s_c[warp][lane] = c;
  if (lane == 0) {
    s_n[warp] = n;
    s_z[warp] = zs;
  }
  int live_all = 0;
  for (int i = threadIdx.x; i < p.E; i += blockDim.x)
    live_all += p.active_mask == nullptr || p.active_mask[i] != 0;
  live_all = __reduce_add_sync(0xffffffffu, live_all);
  if (lane == 0) s_last = 0;
  __syncthreads();
  if (lane == 0) atomicAdd(&s_last, live_all);
  __syncthreads();
  live_all = s_last;
  __syncthreads();
  if (warp == 0) {
    v = 0.f;
    c = 0;
    n = 0;
    zs = 0.0;
    for (int w = 0; w < warps; ++w) {
      v += s_p[w][lane];
      c += s_c[w][lane];
      n += s_n[w];
      zs += s_z[w];
    }
    const float prob = n > 0 ? v / float(n) : 0.f;
    double part = 0.0;
    if (e < p.E) {
      p.counts[size_t(s) * p.E + e] = c;
      p.prob[size_t(s) * p.E + e] = prob;
      if (n > 0) part = double(c) * live_all / (double(p.k) * n) * double(prob);
    }
#pragma unroll
    for (int h = 16; h > 0; h >>= 1) part += __shfl_xor_sync(0xffffffffu, part, h);
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
  double part = 0.0;
  zs = 0.0;
  int m = 0, seqs = 0;
  for (int i = threadIdx.x; i < p.n_seq * groups; i += blockDim.x) part += __ldcg(p.w_part + i);
  for (int i = threadIdx.x; i < p.n_seq; i += blockDim.x) {
    const int ni = __ldcg(p.n_tokens + i);
    m += ni;
    seqs += ni > 0;
    zs += __ldcg(p.w_zseq + i);
  }
#pragma unroll
  for (int h = 16; h > 0; h >>= 1) {
    part += __shfl_xor_sync(0xffffffffu, part, h);
    zs += __shfl_xor_sync(0xffffffffu, zs, h);
  }
  m = __reduce_add_sync(0xffffffffu, m);
  seqs = __reduce_add_sync(0xffffffffu, seqs);
  if (lane == 0) {
    s_d[warp] = part;
    s_z[warp] = zs;
    s_n[warp] = m;
    s_c[0][warp] = seqs;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    part = 0.0;
    zs = 0.0;
    m = 0;
    seqs = 0;
    for (int w = 0; w < warps; ++w) {
      part += s_d[w];
      zs += s_z[w];
      m += s_n[w];
      seqs += s_c[0][w];
    }
    p.loss[0] = seqs > 0 ? float(double(p.coef) * part / seqs) : 0.f;
    p.loss[1] = m > 0 ? float(double(p.z_coef) * zs / m) : 0.f;
    p.n_tokens[p.n_seq] = m;
    p.n_tokens[p.n_seq + 1] = seqs;
  }
}

// dz, from the kept log-sum-exp. Its rounding (of a number that may be much larger than one) is
// common to a token's probabilities: dividing by their sum takes it out. A warp walks the sequences of
// its tokens by itself, with the sequence's f - 1 of its experts in registers.
template <int LPT, int NI>
__global__ void __launch_bounds__(kThreads) balance_bwd_kernel(
    const float *__restrict__ logits, const uint8_t *__restrict__ active_mask,
    const int32_t *__restrict__ seq_offsets, int n_seq, int T, int E, int k, int chunk, float coef, float z_coef,
    const int32_t *__restrict__ counts, const int32_t *__restrict__ n_tokens,
    const float *__restrict__ lse, const float *__restrict__ d_loss, float *__restrict__ dz) {
  constexpr int TPW = 32 / LPT;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, q = lane % LPT;
  pdl_start();
  const int t0 = blockIdx.x * chunk, t1 = min(T, t0 + chunk);
  if (t0 >= t1) return;
  int live_all = 0;
  for (int e = lane; e < E; e += 32) live_all += active_mask == nullptr || active_mask[e] != 0;
  live_all = __reduce_add_sync(0xffffffffu, live_all);
  bool live[NI];
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int e = q + LPT * i;
    live[i] = e < E && (active_mask == nullptr || active_mask[e] != 0);
  }
  const int m = n_tokens[n_seq], seqs = n_tokens[n_seq + 1];
  const float g0 = d_loss != nullptr ? d_loss[0] : 1.f, g1 = d_loss != nullptr ? d_loss[1] : 1.f;
  const float bz = m > 0 ? 2.f * z_coef * g1 / float(m) : 0.f;
  auto zero = [&](int a, int b) {  // rows of tokens in no sequence
    for (int t = a + warp; t < b; t += kWarps)
      for (int e = lane; e < E; e += 32) dz[size_t(t) * E + e] = 0.f;
  };
  int cur = t0;
  for (int s = first_sequence(seq_offsets, n_seq, T, t0); s < n_seq && cur < t1; ++s) {
    int a, b;
    sequence_range(seq_offsets, s, T, &a, &b);
    if (a >= t1) break;
    a = max(a, cur);
    b = min(b, t1);
    zero(cur, a);
    cur = max(cur, a);
    if (a >= b) continue;
    const int n = n_tokens[s];
    const float as = n > 0 && seqs > 0 ? coef * g0 / (float(seqs) * float(n)) : 0.f;
    float f[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      f[i] = 0.f;
      if (live[i] && n > 0) {
        const int64_t all = int64_t(k) * n, c = counts[size_t(s) * E + q + LPT * i];
        f[i] = float(c * live_all - all) / float(all);
      }
    }
    for (int tb = a + warp * TPW; tb < b; tb += kWarps * TPW) {
      const int t = tb + lane / LPT;
      const float l = t < b ? lse[t] : -INFINITY;
      const bool some = !(l == -INFINITY);
      float z[NI], s0 = 0.f, s1 = 0.f;
#pragma unroll
      for (int i = 0; i < NI; ++i) z[i] = some && live[i] ? logits[size_t(t) * E + q + LPT * i] : -INFINITY;
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        z[i] = some ? expf(z[i] - l) : 0.f;
        s0 += z[i];
        s1 = fmaf(z[i], f[i], s1);
      }
      s0 = group_sum<LPT>(s0);
      s1 = group_sum<LPT>(s1);
      if (t < b) {
        const float r = some ? 1.f / s0 : 0.f, base = some ? fmaf(bz, l, -as * (s1 * r)) : 0.f;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          const int e = q + LPT * i;
          if (e < E) dz[size_t(t) * E + e] = z[i] * r * fmaf(as, f[i], base);
        }
      }
    }
    cur = b;
  }
  zero(cur, t1);
}

// Lanes per token and logits per lane for E experts.
template <typename F> void with_lanes(int E, F f) {
  if (E <= 16) f(std::integral_constant<int, 4>(), std::integral_constant<int, 4>());
  else if (E <= 32) f(std::integral_constant<int, 8>(), std::integral_constant<int, 4>());
  else if (E <= 64) f(std::integral_constant<int, 16>(), std::integral_constant<int, 4>());
  else if (E <= 128) f(std::integral_constant<int, 32>(), std::integral_constant<int, 4>());
  else if (E <= 192) f(std::integral_constant<int, 32>(), std::integral_constant<int, 6>());
  else f(std::integral_constant<int, 32>(), std::integral_constant<int, 8>());
}

int check_sizes(const char *fn, int T, int E, int k, int n_seq, const void *seq_offsets, float coef, float z_coef) {
  if (E < 1 || E > 256) return moe::set_error(MOE_ERR_UNSUPPORTED, "%s: E=%d not in [1,256]", fn, E);
  if (k < 1 || k > 8 || k > E) return moe::set_error(MOE_ERR_UNSUPPORTED, "%s: k=%d", fn, k);
  if (T < 0 || n_seq < 1 || n_seq > kMaxSeqs)
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
  p.chunk = chunk_tokens(T);
  p.coef = coef;
  p.z_coef = z_coef;
  p.ticket = reinterpret_cast<int *>(base);
  p.w_prob = reinterpret_cast<float *>(base + w.prob);
  p.w_count = reinterpret_cast<int32_t *>(base + w.count);
  p.w_n = reinterpret_cast<int32_t *>(base + w.n);
  p.w_zsq = reinterpret_cast<double *>(base + w.zsq);
  p.w_part = reinterpret_cast<double *>(base + w.part);
  p.w_zseq = reinterpret_cast<double *>(base + w.zseq);
  p.loss = loss;
  p.prob = prob;
  p.lse = lse;
  p.counts = counts;
  p.n_tokens = n_tokens;
  const int grid = std::max(1, chunk_count(T));
  with_lanes(E, [&](auto lpt, auto ni) {
    MOE_LAUNCH("balance_stats", s, moe::launch_dep(balance_stats_kernel<lpt.value, ni.value>, grid, kThreads, 0, s, p));
  });
  if (int st = moe::launch_status("moe_balance_loss: token sums")) return st;
  // few sequences: many warps for a sequence's rows; many: few rows each
  const int threads = n_seq <= 32 ? 1024 : 128;
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
  const int chunk = chunk_tokens(T);
  with_lanes(E, [&](auto lpt, auto ni) {
    MOE_LAUNCH("balance_bwd", s, moe::launch_dep(balance_bwd_kernel<lpt.value, ni.value>, chunk_count(T), kThreads, 0, s,
                                                 logits, active_mask, seq_offsets, n_seq, T, E, k, chunk, coef, z_coef, counts,
                                                 n_tokens, lse, d_loss, dz));
  });
  return moe::launch_status("moe_balance_loss_bwd: launch");
}

}  // extern "C"
