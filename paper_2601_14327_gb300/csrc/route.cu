// Router (fp32 logits, top-k, softmax over the selected experts, histogram),
// the standalone histogram, and the router backward.
//
// Routing indicator E[i,j,l] and per-expert token number: Sec. 3.2, Eq. 1 and
// Algorithm 1 Step 1 of the LAEP paper. Pruned experts receive no token
// (Sec. 4, Table 5): their logit is -inf before the top-k.
#include <cuda_fp16.h>
#include <math.h>

#include "common.cuh"
#include "tc_ptx.cuh"
#include "tmap.cuh"

MOE_DEV_ERR_DECL

namespace {

constexpr int kTopkThreads = 128;
int padded_experts(int E) { return E <= 64 ? 64 : (E <= 128 ? 128 : (E <= 192 ? 192 : 256)); }

__global__ void zero_i32_kernel(int32_t *p, int n) {
  pdl_start();
  for (int i = blockIdx.x * blockDim.x + threadIdx.x; i < n; i += gridDim.x * blockDim.x) p[i] = 0;
}

// ---- logits on the tensor cores ----------------------------------------------
// The fp32 router weight is split into three bf16 terms, W = W_hi + W_mid + W_lo,
// each the bf16 rounding of what the earlier terms leave (the bf16x3 scheme of
// Henry, Tang and Heinecke, "Leveraging the bfloat16 artificial intelligence
// datatype for higher-precision computations", 2019). Three 8-bit significands
// cover the 24 of a normal fp32 weight, every bf16 x bf16 product is exact in
// fp32 and accumulates in fp32 in tensor memory, so the logits carry fp32
// accumulation error only.
//
// One CTA = one or two 128-token tiles x one range of k-blocks (a split of the
// reduction over d when there are fewer tiles than CTA slots). Warp 0 issues the
// TMA loads (x tile + the three weight terms per k-block), warp 1 owns TMEM and
// issues the MMAs, then all four warps read the accumulator (one TMEM lane
// quarter each) and write the partial logits partial[split][t][0..NP). The same
// kernel computes the router weight gradient with the roles changed (see
// route_tc_kernel): 128-feature tiles of x^T, the reduction over tokens.
constexpr int kRtBM = 128;       // tokens per tile (TMEM lanes)
constexpr int kRtBK = 64;        // k-block: 64 bf16 = one 128-byte swizzle row
constexpr int kRtThreads = 128;
constexpr int kRtSms = 152;           // SMs of a GB300: the splits aim to fill them
constexpr int kRtSmemPerSm = 233472;  // shared memory per SM (228 KB)
constexpr int kRtLogitsSplits = 8;
constexpr int kRtDwSplits = 64;
constexpr uint32_t kRtABytes = kRtBM * kRtBK * 2;
constexpr int kRtMaxSmem = 232448;  // opt-in dynamic shared memory per CTA
constexpr uint64_t kRtWaitNs = 2000000000ull;

struct RouteTcParams {
  int M;             // output rows: tokens (logits) or d_model (router weight gradient)
  int MT;            // 128-row tiles per CTA (1 or 2); tile m's accumulator at TMEM column 256*m
  int kb_per_split;  // k-blocks of one split
  int nkb;           // k-blocks of the reduction (over d, or over the padded tokens)
  int NP;            // experts rounded up to 16
  int NE;            // row stride of the partial logits
  int stages;        // shared-memory ring depth
  uint32_t tmem_cols;
  float *partial;
};

// Experts rounded up to the MMA's N granularity, and the matching TMEM allocation.
int route_tc_np(int E) { return (E + 15) / 16 * 16; }
// Terms of the second operand (the weight, or dZ) per MMA. Logits: 1, each k-step adds the hi, mid
// and lo products to one accumulator. x^T dZ: as many as fit along N (256), each with an accumulator of
// its own, added at the end; the x tile is then read from shared memory once (up to 80 experts)
// or twice (up to 128) per k-step instead of three times, and shared memory sets the pace of
// these short-N MMAs: 43 / 31 us at T=16384, d=4096, 64 experts, 47 / 40 us at T=35700, d=2856, 57.
// At least one: the workspace is also sized for expert counts that moe_route and moe_route_bwd
// refuse (E > 256), and the plan divides by this.
int route_dw_group(int NP) { return std::max(1, std::min(3, 256 / NP)); }
uint32_t route_tc_tmem_cols(int c, int MT) {  // c: accumulator columns of one tile
  if (MT == 2) return 512u;
  return c <= 32 ? 32u : (c <= 64 ? 64u : (c <= 128 ? 128u : 256u));
}
uint32_t route_tc_stage_bytes(int NP, int MT) { return uint32_t(MT) * kRtABytes + 3u * uint32_t(NP) * 128u; }
size_t route_tc_smem(int NP, int stages, int MT) {
  return 1024 + size_t(stages) * route_tc_stage_bytes(NP, MT) + size_t(2 * stages + 1) * 8 + 16;
}
// CTAs per SM and ring depth: with one 128-row tile per CTA, two CTAs per SM if a ring of at
// least two stages each fits (more independent x streams per SM: measured faster than one
// CTA with a deeper ring); else one with the deepest ring that fits (0 stages: none of two).
void route_tc_ring(int NP, int MT, int *per_sm, int *stages) {
  *per_sm = MT == 1 && 2 * (route_tc_smem(NP, 2, 1) + 1024) <= size_t(kRtSmemPerSm) ? 2 : 1;
  int st = 0;
  while (st < 8 && (*per_sm == 2 ? 2 * (route_tc_smem(NP, st + 1, 1) + 1024) <= size_t(kRtSmemPerSm)
                                 : int64_t(st + 1) * route_tc_stage_bytes(NP, MT) <= kRtMaxSmem - 2048))
    ++st;
  *stages = st >= 2 ? st : 0;
}

struct RtPlan {
  int MT;  // 128-row tiles per CTA
  int stages, splits, kb_per_split;
};
// Logits, M tokens over K = d. Two tiles per CTA from 97 to 192 experts, where the three weight
// terms of a k-block (3 x NP x 128 bytes) outweigh the 16 KB x tile: two x tiles share each
// weight stage. Splits: enough CTAs to fill the SMs' CTA slots when the tokens give few tiles. The
// plan fixes the order in which a logit's products are summed, and with it the last bits that
// decide a near tie: it is a function of (M, K, NP) alone, and a change of it can route a token
// differently.
RtPlan route_logits_plan(int M, int K, int NP) {
  RtPlan r;
  int per_sm;
  r.MT = NP > 96 && NP <= 192 ? 2 : 1;
  route_tc_ring(NP, r.MT, &per_sm, &r.stages);
  const int rows = kRtBM * r.MT, tiles = std::max(1, (M + rows - 1) / rows);
  const int nkb = (K + kRtBK - 1) / kRtBK;
  const int s = std::max(1, std::min({kRtSms * per_sm / tiles, kRtLogitsSplits, nkb}));
  r.kb_per_split = (nkb + s - 1) / s;
  r.splits = (nkb + r.kb_per_split - 1) / r.kb_per_split;  // every split gets at least one k-block
  return r;
}
// x^T dZ, M = d features over K tokens: the tiles per CTA and splits of the reduction with the
// least estimated time (ns). An SM takes a k-block of a CTA in the longest of its share of the HBM
// rate for the x tiles, its shared-memory traffic (TMA writes, MMA reads) at ~243 B/ns, and, with
// few CTAs, a load's way through the ring (~2.3 us for load, wait and MMA over the stages); a
// split adds its partial sums' write and read. A function of (M, K, NP) alone, so the workspace
// size is too. K > 0. Measured, with the logits' plan (at most 8 splits) / with this one: 30 /
// 12.6 us at T=22360, d=1128, 28 experts (9 tiles: 72 CTAs / 32 splits), 67 / 40 us at T=35700,
// d=2856, 57 experts, 22.9 / 18.0 us at T=3516, d=3328, 167 experts; both 49 us at T=8191, d=7168, 171.
RtPlan route_dw_plan(int M, int K, int NP) {
  const int nkb = (K + kRtBK - 1) / kRtBK;
  const int group = route_dw_group(NP), mmas = (3 + group - 1) / group;
  const int64_t ne = (NP + 31) / 32 * 32;
  RtPlan best{1, 2, 1, nkb};
  int64_t best_ns = INT64_MAX;
  for (int mt = 1; mt <= (M > kRtBM ? 2 : 1); ++mt) {
    int per_sm, stages;
    route_tc_ring(NP, mt, &per_sm, &stages);
    if (stages == 0) continue;
    const int64_t tiles = std::max(1, (M + kRtBM * mt - 1) / (kRtBM * mt));
    const int64_t a = int64_t(mt) * kRtABytes, w = int64_t(3) * NP * 128;
    const int64_t busy = std::max<int64_t>(a * 1000 / 44700, (a + w + mmas * a + mt * w) * 1000 / 243000);
    const int64_t ring = 2300 / stages, slots = int64_t(kRtSms) * per_sm;
    for (int s = 1; s <= std::min(nkb, kRtDwSplits); ++s) {
      const int per = (nkb + s - 1) / s;
      if ((nkb + per - 1) / per != s) continue;  // every split gets at least one k-block
      const int64_t full = tiles * s / slots, rest = tiles * s % slots;
      int64_t ns = full * (per * std::max(per_sm * busy, ring) + 1500);
      if (rest > 0) ns += per * std::max(rest > kRtSms ? 2 * busy : busy, ring) + 1500;
      if (s > 1) ns += s * int64_t(M) * ne * 8 / 4000;
      if (ns < best_ns) {
        best_ns = ns;
        best = {mt, stages, s, per};
      }
    }
  }
  return best;
}

// Router weight gradient: tokens padded to one k-block, and the row stride of its
// partial sums (the epilogue writes 32 columns at a time).
int route_tokens_padded(int T) { return (T + kRtBK - 1) / kRtBK * kRtBK; }
int route_dw_stride(int E) { return (route_tc_np(E) + 31) / 32 * 32; }

// W [d, E] fp32 -> W3 [3][NP][d] bf16 (hi, mid, lo; rows e >= E are zero), by
// 32 x 32 tiles transposed through shared memory. The first blocks also zero the counts that
// the top-k kernel adds to (nullptr: none).
__global__ void route_split_w_kernel(const float *__restrict__ w, int d, int E, int NP,
                                     uint16_t *__restrict__ w3, int32_t *__restrict__ counts) {
  __shared__ float tile[32][33];
  pdl_start();
  if (counts != nullptr && blockIdx.x == 0 && threadIdx.y == 0 && blockIdx.y * 32 + threadIdx.x < E)
    counts[blockIdx.y * 32 + threadIdx.x] = 0;
  const int k0 = blockIdx.x * 32, e0 = blockIdx.y * 32;
  const int tx = threadIdx.x, ty = threadIdx.y;
  for (int i = ty; i < 32; i += 8) {
    const int k = k0 + i, e = e0 + tx;
    tile[i][tx] = (k < d && e < E) ? w[size_t(k) * E + e] : 0.f;
  }
  __syncthreads();
  for (int i = ty; i < 32; i += 8) {
    const int e = e0 + i, k = k0 + tx;
    if (e < NP && k < d) {
      const float v = tile[tx][i];
      const __nv_bfloat16 hi = __float2bfloat16_rn(v);
      const float r1 = v - __bfloat162float(hi);
      const __nv_bfloat16 mid = __float2bfloat16_rn(r1);
      const float r2 = r1 - __bfloat162float(mid);
      const __nv_bfloat16 lo = __float2bfloat16_rn(r2);
      const size_t plane = size_t(NP) * d, at = size_t(e) * d + k;
      w3[at] = __bfloat16_as_ushort(hi);
      w3[plane + at] = __bfloat16_as_ushort(mid);
      w3[2 * plane + at] = __bfloat16_as_ushort(lo);
    }
  }
}

// DW = false: the logits, partial[split][t][e] = x[t, k-range] . W3[e, k-range].
// DW = true: the router weight gradient, partial[split][i][e] = sum over the split's
// tokens t of x[t, i] * dZ[t, e] (A = x^T, read MN-major from x itself as two 64 x 64
// boxes per k-block; B = dZ's three bf16 terms, K-major [3][NP][T padded to 64]).
// G = terms per MMA (see route_dw_group), at compile time: the issuing thread's loop sets the pace
// otherwise (with a bound read from the parameters 110 instead of 79 us at T=32768, 128 experts).
// AHEAD (logits): a stage's next x tile goes to L2 while this one loads (see launch_route_tc).
template <bool DW, int G, bool AHEAD>
__global__ void __launch_bounds__(kRtThreads, 1)
    route_tc_kernel(const __grid_constant__ CUtensorMap tmX,
                    const __grid_constant__ CUtensorMap tmW, const RouteTcParams p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = tc::smem_u32(smem_raw);
  const uint32_t pad = (1024u - (raw & 1023u)) & 1023u;
  const uint32_t b_bytes = uint32_t(p.NP) * 128u;
  const uint32_t a_bytes = uint32_t(p.MT) * kRtABytes;  // the CTA's x tiles of a k-block
  const uint32_t stage_bytes = a_bytes + 3u * b_bytes;
  const int S = p.stages;
  const uint32_t s0 = raw + pad;
  uint64_t *bars = reinterpret_cast<uint64_t *>(smem_raw + pad + size_t(S) * stage_bytes);
  int *misc = reinterpret_cast<int *>(bars + 2 * S + 1);
  volatile int *abort_flag = misc + 1;
  volatile int no_abort = 0;
  const uint32_t bar0 = tc::smem_u32(bars);
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (S + s); };
  const uint32_t done_bar = bar0 + 8u * (2 * S);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int mt = blockIdx.x, split = blockIdx.y;
  const int kb0 = split * p.kb_per_split, nk = min(p.nkb, kb0 + p.kb_per_split) - kb0;
  // Each token tile starts its k-loop at its own offset, so that the CTAs do not all read
  // the same weight tile from L2 at the same time (the order is fixed per tile; without it
  // 88 instead of 71 us at T=26750, d=4296, 61 experts). x^T dZ's feature tiles read slices
  // of the same token rows and stay in step (48 against 51 us at T=35700, d=2856).
  const int rot = !DW && nk > 0 ? int((mt * 7u) % uint32_t(nk)) : 0;
  const uint32_t idesc_g = tc::idesc_bf16_f32(kRtBM, G * p.NP, DW, false);
  const uint32_t idesc_1 = tc::idesc_bf16_f32(kRtBM, p.NP, DW, false);

  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s) {
      tc::mbar_init(full_bar(s), 1);
      tc::mbar_init(empty_bar(s), 1);
    }
    tc::mbar_init(done_bar, 1);
    tc::fence_mbar_init();
    misc[1] = 0;
  }
  if (warp == 0 && lane == 0) {
    tc::tma_prefetch_desc(&tmX);
    tc::tma_prefetch_desc(&tmW);
  }
  if (warp == 1) {
    tc::tmem_alloc(tc::smem_u32(misc), p.tmem_cols);
    tc::tmem_relinquish();
  }
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  const uint32_t tmem_base = static_cast<uint32_t>(misc[0]);
  pdl_start();  // TMEM is allocated; set-up overlaps the end of the previous kernel

  if (warp == 0 && lane == 0) {
    // ---- TMA producer ----
    uint32_t it = 0;
    for (; int(it) < nk; ++it) {
      const int kb = kb0 + (int(it) + rot) % nk;
      const int s = it % S;
      const uint32_t ph = (it / S) & 1u;
      if (!tc::mbar_wait(empty_bar(s), ph ^ 1u, kRtWaitNs, abort_flag)) {
        dev_flag(&g_dev_err, MOE_DEV_WAIT_TIMEOUT);
        *abort_flag = 1;
        break;
      }
      tc::mbar_arrive_expect_tx(full_bar(s), stage_bytes);
      const uint32_t dst = s0 + s * stage_bytes;
      const int k0 = kb * kRtBK;
      for (int m = 0; m < p.MT; ++m) {
        const int row0 = (mt * p.MT + m) * kRtBM;
        const uint32_t am = dst + uint32_t(m) * kRtABytes;
        if (DW) {  // x^T: features row0 .. +127 (two 64-wide boxes) x tokens k0 .. k0+63
          tc::tma_load_2d(am, &tmX, full_bar(s), row0, k0);
          tc::tma_load_2d(am + 64 * 128, &tmX, full_bar(s), row0 + 64, k0);
        } else {
          tc::tma_load_2d(am, &tmX, full_bar(s), k0, row0);
        }
      }
#pragma unroll
      for (int j = 0; j < 3; ++j)
        tc::tma_load_2d(dst + a_bytes + j * b_bytes, &tmW, full_bar(s), k0, j * p.NP);
      if (AHEAD && int(it) + 2 < nk) {
        const int k2 = (kb0 + (int(it) + 2 + rot) % nk) * kRtBK;
        for (int m = 0; m < p.MT; ++m) {
          const int row0 = (mt * p.MT + m) * kRtBM;
          if (row0 < p.M) tc::tma_prefetch_2d(&tmX, k2, row0);
        }
      }
    }
    // every issued load lands before the CTA may exit (also after an abort)
    for (int s = 0; s < S; ++s) {
      if (it > uint32_t(s)) {
        const uint32_t n = (it - 1 - s) / S;
        if (!tc::mbar_wait(full_bar(s), n & 1u, kRtWaitNs, &no_abort))
          dev_flag(&g_dev_err, MOE_DEV_WAIT_TIMEOUT);
      }
    }
  } else if (warp == 1 && lane == 0) {
    // ---- MMA issuer ----
    uint32_t it = 0;
    bool issued = false;
    for (; int(it) < nk; ++it) {
      const int s = it % S;
      const uint32_t ph = (it / S) & 1u;
      if (!tc::mbar_wait(full_bar(s), ph, kRtWaitNs, abort_flag)) {
        dev_flag(&g_dev_err, MOE_DEV_WAIT_TIMEOUT);
        *abort_flag = 1;
        break;
      }
      tc::fence_after_sync();
      const uint32_t a_s = s0 + s * stage_bytes, b_s = a_s + a_bytes;
      // (a descriptor's address field counts 16 bytes: steps are plain additions)
      const uint64_t b0 = tc::smem_desc_sw128(b_s, 16, 1024);
      for (int m = 0; m < p.MT; ++m) {
        const uint32_t am = a_s + uint32_t(m) * kRtABytes, d = tmem_base + uint32_t(m) * 256u;
        const uint64_t a0 = DW ? tc::smem_desc_sw128(am, 8192, 1024) : tc::smem_desc_sw128(am, 16, 1024);
#pragma unroll
        for (int kk = 0; kk < kRtBK / 16; ++kk) {
          const uint64_t ad = a0 + uint64_t(DW ? kk * 128 : kk * 2);
          tc::mma_bf16(d, ad, b0 + uint64_t(kk * 2), idesc_g, (it != 0 || kk != 0) ? 1u : 0u);
#pragma unroll
          for (int j = G; j < 3; ++j)  // terms that did not fit: into the first accumulator
            tc::mma_bf16(d, ad, b0 + uint64_t(kk * 2) + uint64_t(j) * (b_bytes >> 4), idesc_1, 1u);
        }
      }
      tc::mma_commit(empty_bar(s));
      issued = true;
    }
    if (issued) tc::mma_commit(done_bar);
    else *abort_flag = 1;  // nothing to wait for: the epilogue must not wait either
  }
  __syncwarp();

  // ---- epilogue: TMEM lane quarter `warp` -> 32 output rows x NP partial sums ----
  int ok = 0;
  if (lane == 0) {
    ok = tc::mbar_wait(done_bar, 0, kRtWaitNs, abort_flag) ? 1 : 0;
    if (!ok && !*abort_flag) {
      dev_flag(&g_dev_err, MOE_DEV_WAIT_TIMEOUT);
      *abort_flag = 1;
    }
  }
  ok = __shfl_sync(0xffffffffu, ok, 0);
  if (ok) {
    tc::fence_after_sync();
    for (int m = 0; m < p.MT; ++m) {
      const int t = (mt * p.MT + m) * kRtBM + warp * 32 + lane;
      float *dst = p.partial + (size_t(split) * p.M + t) * p.NE;
      for (int c0 = 0; c0 < p.NP; c0 += 32) {
        uint32_t r[32];
        const uint32_t tb = tmem_base + (uint32_t(warp * 32) << 16) + uint32_t(m) * 256u + uint32_t(c0);
        tc::tmem_ld_32x32b_x32(tb, r);
        tc::tmem_ld_wait();
#pragma unroll
        for (int j = 1; j < G; ++j) {
          uint32_t q[32];
          tc::tmem_ld_32x32b_x32(tb + uint32_t(j * p.NP), q);
          tc::tmem_ld_wait();
#pragma unroll
          for (int i = 0; i < 32; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) + __uint_as_float(q[i]));
        }
        if (t < p.M) {
#pragma unroll
          for (int q = 0; q < 8; ++q)
            stg_v4(dst + c0 + 4 * q, make_uint4(r[4 * q], r[4 * q + 1], r[4 * q + 2], r[4 * q + 3]));
        }
      }
    }
  }
  tc::fence_before_sync();
  __syncthreads();
  if (warp == 1) {
    tc::fence_after_sync();
    tc::tmem_dealloc(tmem_base, p.tmem_cols);
  }
}

// The K largest (key, expert) pairs so far, descending; equal keys by ascending expert.
template <int K> struct TopList {
  unsigned key[K];  // order-preserving key of a logit, 0: empty
  int e[K];
  __device__ __forceinline__ TopList() {
#pragma unroll
    for (int s = 0; s < K; ++s) {
      key[s] = 0u;
      e[s] = -1;
    }
  }
  // Experts come in ascending order: a later one passes strictly smaller keys only (the
  // entries from there on move down one slot).
  __device__ __forceinline__ void add(unsigned x, int xe) {
    bool up = false;
#pragma unroll
    for (int s = 0; s < K; ++s) {
      up = up || x > key[s];
      const unsigned lk = up ? key[s] : x;
      const int le = up ? e[s] : xe;
      key[s] = up ? x : key[s];
      e[s] = up ? xe : e[s];
      x = lk;
      xe = le;
    }
  }
  static __device__ __forceinline__ bool before(unsigned ka, int ea, unsigned kb, int eb) {
    return ka > kb || (ka == kb && ea < eb);
  }
  // The K largest of this list and lane ^ `lane_xor`'s: the larger of entry s here and entry
  // K-1-s there are those K, as a bitonic sequence, which log2(K) exchange stages sort.
  __device__ __forceinline__ void merge(int lane_xor) {
    unsigned ok[K];
    int oe[K];
#pragma unroll
    for (int s = 0; s < K; ++s) {
      ok[s] = __shfl_xor_sync(0xffffffffu, key[s], lane_xor);
      oe[s] = __shfl_xor_sync(0xffffffffu, e[s], lane_xor);
    }
#pragma unroll
    for (int s = 0; s < K; ++s) {
      const bool other = before(ok[K - 1 - s], oe[K - 1 - s], key[s], e[s]);
      key[s] = other ? ok[K - 1 - s] : key[s];
      e[s] = other ? oe[K - 1 - s] : e[s];
    }
#pragma unroll
    for (int h = K / 2; h > 0; h >>= 1)
#pragma unroll
      for (int s = 0; s < K; ++s)
        if ((s & h) == 0) {
          const bool sw = before(key[s + h], e[s + h], key[s], e[s]);
          const unsigned ka = key[s], kb = key[s + h];
          const int ea = e[s], eb = e[s + h];
          key[s] = sw ? kb : ka;
          e[s] = sw ? eb : ea;
          key[s + h] = sw ? ka : kb;
          e[s + h] = sw ? ea : eb;
        }
  }
};

// LPT (4 or 16) lanes per token: logits = sum of the split partials (fixed order) + bias, pruned
// experts -inf; top-k (ties to the lower index), softmax over the selected logits,
// per-expert histogram (shared per block, then one global add per expert and block).
// Lane q keeps the K largest logits of experts 4 LPT i + 4 q .. + 3 in registers (~5 K
// instructions per logit, 32 / LPT tokens per instruction), exchanges merge the lists.
// Issue-bound with many tokens: 4 lanes, ~250 warp instructions per token at 128 experts, top-8,
// against ~1,000 for a warp per token with two redux per selected expert: 21 us instead of 40
// at T=32768 (the compares and selects, at half the issue rate, are its bound now). Latency-bound
// with few: 16 lanes, a quarter of the chain per lane.
template <int K, int LPT>
__global__ void __launch_bounds__(kTopkThreads) route_topk_kernel(
    const float *__restrict__ partial, int splits, int NE, const float *__restrict__ logits_in,
    const float *__restrict__ bias, const uint8_t *__restrict__ active_mask, int T, int E, int k,
    float *__restrict__ logits_out, int32_t *__restrict__ topk_idx, float *__restrict__ topk_gate,
    int32_t *__restrict__ counts) {
  __shared__ int hist[256];
  __shared__ __align__(16) float s_bias[256];
  __shared__ uint8_t s_live[256];
  const int tid = threadIdx.x, q = tid % LPT;
  for (int e = tid; e < 256; e += kTopkThreads) hist[e] = 0;
  pdl_start();
  for (int e = tid; e < 256; e += kTopkThreads) {
    s_bias[e] = (bias != nullptr && e < E) ? bias[e] : 0.f;
    s_live[e] = e < E && (active_mask == nullptr || active_mask[e] != 0);
  }
  __syncthreads();
  constexpr int per_block = kTopkThreads / LPT;
  // (whole warps stay in the loop: the merges are warp-wide)
  for (int t0 = blockIdx.x * per_block; t0 < T; t0 += gridDim.x * per_block) {
    const int t = t0 + tid / LPT;
    const bool mine = t < T;
    TopList<K> top;
    // four chunks of four experts at a time, so that their loads (of up to four partials each)
    // are in flight together
    for (int g0 = 0; g0 < E; g0 += 16 * LPT) {
      float z[4][4] = {};
      if (mine) {
        if (logits_in != nullptr) {
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int e = g0 + 4 * (c * LPT + q) + i;
              if (e < E) z[c][i] = logits_in[size_t(t) * E + e];
            }
        } else {
          const float *src = partial + size_t(t) * NE + g0 + 4 * q;
          const size_t plane = size_t(T) * NE;
          for (int y0 = 0; y0 < splits; y0 += 4) {  // summed in order
            float4 v[4][4];
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
              for (int c = 0; c < 4; ++c)
                if (y0 + u < splits && g0 + 4 * (c * LPT + q) < E)
                  v[u][c] = *reinterpret_cast<const float4 *>(src + (y0 + u) * plane + 4 * LPT * c);
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
              for (int c = 0; c < 4; ++c)
                if (y0 + u < splits && g0 + 4 * (c * LPT + q) < E) {
                  z[c][0] += v[u][c].x;
                  z[c][1] += v[u][c].y;
                  z[c][2] += v[u][c].z;
                  z[c][3] += v[u][c].w;
                }
          }
        }
      }
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int e0 = g0 + 4 * (c * LPT + q);
        if (e0 < E) {
          if (logits_in == nullptr && bias != nullptr) {
            const float4 b = *reinterpret_cast<const float4 *>(s_bias + e0);
            z[c][0] += b.x;
            z[c][1] += b.y;
            z[c][2] += b.z;
            z[c][3] += b.w;
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int e = e0 + i;
            float v = z[c][i];
            if (!s_live[e]) v = -INFINITY;
            if (e < E) {
              if (logits_out != nullptr && mine) logits_out[size_t(t) * E + e] = v;
              // a larger float gives a larger key; -0 is taken as +0 so that equal logits tie
              const unsigned u = __float_as_uint(v == 0.f ? 0.f : v);
              top.add((u & 0x80000000u) ? ~u : (u | 0x80000000u), e);
            }
          }
        }
      }
    }
    __syncwarp();
#pragma unroll
    for (int h = 1; h < LPT; h <<= 1) top.merge(h);
    if (!mine) continue;
    // softmax over the selected logits (renormalised top-k), fp32
    float ex[K], den = 0.f, zmax = 0.f;
    bool too_few = false;
#pragma unroll
    for (int s = 0; s < K; ++s) {
      if (s < k) {
        const unsigned m = top.key[s];
        const float v = __uint_as_float((m & 0x80000000u) ? (m & 0x7fffffffu) : ~m);
        if (s == 0) zmax = v;
        ex[s] = expf(v - zmax);
        den += ex[s];
        if (v == -INFINITY) too_few = true;
      }
    }
    if (q == 0 && too_few) dev_flag(&g_dev_err, MOE_DEV_TOO_FEW_LIVE);
#pragma unroll
    for (int s = 0; s < K; ++s) {
      if (s < k && s % LPT == q) {
        topk_idx[size_t(t) * k + s] = top.e[s];
        topk_gate[size_t(t) * k + s] = ex[s] / den;
        if (top.e[s] >= 0) atomicAdd(&hist[top.e[s]], 1);
      }
    }
  }
  __syncthreads();
  if (counts != nullptr)
    for (int e = tid; e < E; e += kTopkThreads)
      if (hist[e]) atomicAdd(&counts[e], hist[e]);
}

// store: the only block of the launch, which writes the counts instead of adding to them.
__global__ void load_stats_kernel(const int32_t *__restrict__ topk_idx, int64_t A, int E, int store,
                                  int32_t *__restrict__ counts) {
  __shared__ int hist[256];
  for (int e = threadIdx.x; e < E; e += blockDim.x) hist[e] = 0;
  __syncthreads();
  pdl_start();
  for (int64_t a = blockIdx.x * int64_t(blockDim.x) + threadIdx.x; a < A;
       a += int64_t(gridDim.x) * blockDim.x) {
    const int e = topk_idx[a];
    if (e >= 0 && e < E)
      atomicAdd(&hist[e], 1);
    else
      dev_flag(&g_dev_err, MOE_DEV_BAD_EXPERT);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < E; e += blockDim.x) {
    if (store) counts[e] = hist[e];
    else if (hist[e]) atomicAdd(&counts[e], hist[e]);
  }
}

// ---- router backward -------------------------------------------------------

// Softmax backward over the selected k, d_logits[t,j] = g_j (dg_j - sum_i g_i dg_i),
// and dZ (the [T, E] logit gradient, zero off the selected experts) as three bf16
// terms, K-major for the tensor cores: dz3[s][e][t] for e < NP, t < Tp (tokens padded
// to 64; the padding is zero). One thread per token and 16 experts (blockIdx.y); the
// y = 0 blocks also write d_logits.
constexpr int kDzExperts = 16;
__global__ void route_bwd_dz_kernel(const int32_t *__restrict__ topk_idx,
                                    const float *__restrict__ gate, const float *__restrict__ dgate,
                                    int T, int Tp, int k, int NP, float *__restrict__ d_logits,
                                    uint16_t *__restrict__ dz3) {
  pdl_start();
  const int t = blockIdx.x * blockDim.x + threadIdx.x;
  if (t >= Tp) return;
  float g[8], dg[8], s = 0.f;
  int ei[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    g[j] = 0.f;
    dg[j] = 0.f;
    ei[j] = -1;
    if (j < k && t < T) {
      g[j] = gate[size_t(t) * k + j];
      dg[j] = dgate[size_t(t) * k + j];
      ei[j] = topk_idx[size_t(t) * k + j];
      s = fmaf(g[j], dg[j], s);
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    g[j] = g[j] * (dg[j] - s);
    if (blockIdx.y == 0 && j < k && t < T) d_logits[size_t(t) * k + j] = g[j];
  }
  const size_t plane = size_t(NP) * Tp;
  const int e0 = blockIdx.y * kDzExperts;
  for (int e = e0; e < min(NP, e0 + kDzExperts); ++e) {
    float v = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (ei[j] == e) v = g[j];  // the k selected experts of a token are distinct
    const __nv_bfloat16 hi = __float2bfloat16_rn(v);
    const float r1 = v - __bfloat162float(hi);
    const __nv_bfloat16 mid = __float2bfloat16_rn(r1);
    const float r2 = r1 - __bfloat162float(mid);
    const __nv_bfloat16 lo = __float2bfloat16_rn(r2);
    const size_t at = size_t(e) * Tp + t;
    dz3[at] = __bfloat16_as_ushort(hi);
    dz3[plane + at] = __bfloat16_as_ushort(mid);
    dz3[2 * plane + at] = __bfloat16_as_ushort(lo);
  }
}

// The same with a dense gradient dz [T, E] beside the selected experts' (topk_idx null: alone): tiles of
// 64 tokens x 64 experts, transposed through shared memory, so that dz is read along its rows and the terms are
// written along theirs, 16 bytes a thread (a thread per token reading 64-byte pieces of its row: 40 us at T=65536,
// 171 experts; 27 now, the bytes alone 17).
constexpr int kDzTile = 64;
__global__ void __launch_bounds__(256) route_bwd_dz_dense_kernel(
    const int32_t *__restrict__ topk_idx, const float *__restrict__ gate, const float *__restrict__ dgate,
    const float *__restrict__ dz, int T, int Tp, int E, int k, int NP, float *__restrict__ d_logits,
    uint16_t *__restrict__ dz3) {
  __shared__ float tile[kDzTile][kDzTile + 1];  // [expert][token]
  pdl_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int t0 = blockIdx.x * kDzTile, e0 = blockIdx.y * kDzTile;
#pragma unroll
  for (int i = 0; i < kDzTile / 8; ++i) {
    const int r = warp + 8 * i, t = t0 + r;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int e = e0 + lane + 32 * h;
      tile[lane + 32 * h][r] = t < T && e < E ? __ldg(dz + size_t(t) * E + e) : 0.f;
    }
  }
  float g[8], dg[8], s = 0.f;
  int ei[8];
  const int t = t0 + tid;
  const bool mine = topk_idx != nullptr && tid < kDzTile && t < T;
  if (mine) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      g[j] = dg[j] = 0.f;
      ei[j] = -1;
      if (j < k) {
        g[j] = gate[size_t(t) * k + j];
        dg[j] = dgate[size_t(t) * k + j];
        ei[j] = topk_idx[size_t(t) * k + j];
        s = fmaf(g[j], dg[j], s);
      }
    }
  }
  __syncthreads();
  if (mine) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float v = g[j] * (dg[j] - s);
      if (blockIdx.y == 0 && j < k) d_logits[size_t(t) * k + j] = v;
      const int e = ei[j] - e0;  // (an id outside [0, E) is left out)
      if (ei[j] >= 0 && ei[j] < E && e >= 0 && e < kDzTile) tile[e][tid] += v;
    }
  }
  __syncthreads();
  const size_t plane = size_t(NP) * Tp;
#pragma unroll
  for (int u = tid; u < kDzTile * (kDzTile / 8); u += 256) {
    const int e = u / 8, c = u % 8 * 8;
    if (e0 + e >= NP) break;
    uint32_t o[3][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint16_t b[3][2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float v = tile[e][c + 2 * i + h];
        const __nv_bfloat16 hi = __float2bfloat16_rn(v);
        const float r1 = v - __bfloat162float(hi);
        const __nv_bfloat16 mid = __float2bfloat16_rn(r1);
        const float r2 = r1 - __bfloat162float(mid);
        b[0][h] = __bfloat16_as_ushort(hi);
        b[1][h] = __bfloat16_as_ushort(mid);
        b[2][h] = __bfloat16_as_ushort(__float2bfloat16_rn(r2));
      }
#pragma unroll
      for (int m = 0; m < 3; ++m) o[m][i] = uint32_t(b[m][0]) | uint32_t(b[m][1]) << 16;
    }
    uint16_t *dst = dz3 + size_t(e0 + e) * Tp + t0 + c;
#pragma unroll
    for (int m = 0; m < 3; ++m) stg_v4(dst + m * plane, make_uint4(o[m][0], o[m][1], o[m][2], o[m][3]));
  }
}

// x^T dZ of the dense router backward on CTA pairs. The tensor core adds to its fp32 accumulator with
// truncation: over the ~2,500 additions of a long split route_tc_kernel's sums come out 4e-5 too small (2-norm,
// T=65536, d=7168, 171 experts; an fp32 product by the library is 5e-6 off), more than the rounding of a dense
// loss gradient may be. Here an accumulator takes kDwFlush k-blocks, while the epilogue warps add the one before to
// their registers, rounding to nearest: 8.8e-7 off. (What is left to grow with T is a chain of T / 256 fp32 additions over
// the number of splits: 2^-24 each of a sum that keeps its sign, 32 at this size.) The tensor pipe sets the time: 275 us there,
// 263 at its measured rate (route_tc_kernel: 291, by shared memory; a pair's M=256 MMA reads each SM's own 128
// features and half of dZ's rows). Two terms of dZ would take 230 us and be 2.5e-6 off, ten times
// what an fp32 product is over 1,000 tokens. Roles as in the grouped GEMMs' pair kernel: warp 0 of each
// CTA loads (its features of x, its half of the terms' rows), one thread of the even CTA issues the MMAs, warps
// 2..9 of each own a TMEM lane quarter and half of the experts.
constexpr int kDwFlush = 4;
constexpr int kDwThreads = 64 + 32 * 8;
struct RouteDwParams {
  int M, NP, NE;         // d, experts rounded up to 16, row stride of the partial sums
  int nkb, kb_per_split; // 64-token k-blocks
  int G;                 // terms per MMA: 3 (each with its own columns) or 1
  int stages;
  uint32_t buf_cols;     // TMEM columns of an accumulator
  float *partial;
  float *dw;             // [M, E], written at once where there is one split (else nullptr)
  int E;
};
uint32_t route_dwp_stage_bytes(int NP) { return kRtBM * kRtBK * 2 + 3u * uint32_t(NP / 2) * 128u; }
int route_dwp_group(int NP) { return 3 * NP <= 256 ? 3 : 1; }
size_t route_dwp_smem(int NP, int stages) {
  return 1024 + size_t(stages) * route_dwp_stage_bytes(NP) + size_t(2 * stages + 5) * 8 + 16;
}
int route_dwp_stages(int NP) { return int(std::min<int64_t>(8, (kRtMaxSmem - 2048) / route_dwp_stage_bytes(NP))); }

__global__ void __launch_bounds__(kDwThreads, 1)
    route_dw_pair_kernel(const __grid_constant__ CUtensorMap tmX, const __grid_constant__ CUtensorMap tmZ,
                         const RouteDwParams p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = tc::smem_u32(smem_raw);
  const uint32_t pad = (1024u - (raw & 1023u)) & 1023u;
  constexpr uint32_t a_bytes = kRtBM * kRtBK * 2;
  const uint32_t half_rows = uint32_t(p.NP / 2), b_term = half_rows * 128u;  // a multiple of 1024
  const uint32_t stage_bytes = a_bytes + 3u * b_term;
  const int S = p.stages;
  const uint32_t s0 = raw + pad;
  uint64_t *bars = reinterpret_cast<uint64_t *>(smem_raw + pad + size_t(S) * stage_bytes);
  int *misc = reinterpret_cast<int *>(bars + 2 * S + 5);
  volatile int *abort_flag = misc + 1;
  volatile int no_abort = 0;
  const uint32_t bar0 = tc::smem_u32(bars);
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (S + s); };
  auto tfull_bar = [&](int a) { return bar0 + 8u * (2 * S + a); };
  auto tempty_bar = [&](int a) { return bar0 + 8u * (2 * S + 2 + a); };
  const uint32_t drain_bar = bar0 + 8u * (2 * S + 4);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = tc::cluster_ctarank();
  const bool leader = rank == 0;
  const int feature0 = int(blockIdx.x) * kRtBM;  // this CTA's features (the pair's are consecutive)
  const int split = blockIdx.y, kb0 = split * p.kb_per_split, nk = min(p.nkb, kb0 + p.kb_per_split) - kb0;

  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s) {
      tc::mbar_init(full_bar(s), 1);
      tc::mbar_init(empty_bar(s), 1);
    }
    for (int a = 0; a < 2; ++a) {
      tc::mbar_init(tfull_bar(a), 1);
      tc::mbar_init(tempty_bar(a), 16);  // the epilogue warps of both CTAs
    }
    tc::mbar_init(drain_bar, 1);
    tc::fence_mbar_init();
    misc[1] = 0;
  }
  if (warp == 1) {
    tc::tmem_alloc_pair(tc::smem_u32(misc), 2 * p.buf_cols);
    tc::tmem_relinquish_pair();
  }
  tc::fence_before_sync();
  __syncthreads();
  tc::cluster_sync();  // barriers of both CTAs initialized before any remote use
  tc::fence_after_sync();
  const uint32_t tmem_base = static_cast<uint32_t>(misc[0]);
  pdl_wait();
  auto fail = [&]() {
    dev_flag(&g_dev_err, MOE_DEV_WAIT_TIMEOUT);
    *abort_flag = 1;
  };

  if (warp == 0) {
    if (lane == 0) {
      const uint32_t full_leader = tc::mapa(full_bar(0), 0);
      uint32_t it = 0;
      for (; int(it) < nk; ++it) {
        const int s = it % S, k0 = (kb0 + int(it)) * kRtBK;
        if (!tc::mbar_wait(empty_bar(s), ((it / S) & 1u) ^ 1u, kRtWaitNs, abort_flag)) { fail(); break; }
        if (leader) tc::mbar_arrive_expect_tx(full_bar(s), 2 * stage_bytes);
        const uint32_t a = s0 + s * stage_bytes, b = a + a_bytes, fb = full_leader + 8u * s;
        // x^T: two 64-feature x 64-token boxes
        tc::tma_load_2d_pair(a, &tmX, fb, feature0, k0);
        tc::tma_load_2d_pair(a + 8192, &tmX, fb, feature0 + 64, k0);
        // the pair's N rows are the even CTA's, then the odd one's: of all three terms, or of each
        if (p.G == 3) {
          tc::tma_load_2d_pair(b, &tmZ, fb, k0, int(rank * 3u * half_rows));
        } else {
#pragma unroll
          for (int j = 0; j < 3; ++j)
            tc::tma_load_2d_pair(b + j * b_term, &tmZ, fb, k0, j * p.NP + int(rank * half_rows));
        }
      }
      if (leader)  // its full barriers count the loads of both CTAs
        for (int s = 0; s < S; ++s)
          if (it > uint32_t(s) && !tc::mbar_wait(full_bar(s), ((it - 1 - s) / S) & 1u, kRtWaitNs, &no_abort)) fail();
    }
  } else if (warp == 1) {
    if (leader && lane == 0) {
      const uint32_t idesc = tc::idesc_bf16_f32(2 * kRtBM, p.G * p.NP, true, false);
      uint32_t it = 0;
      bool ok = true, issued = false;
      for (uint32_t f = 0; int(it) < nk && ok; ++f) {
        const uint32_t a = f & 1u, d = tmem_base + a * p.buf_cols;
        if (!tc::mbar_wait(tempty_bar(a), ((f >> 1) & 1u) ^ 1u, kRtWaitNs, abort_flag)) { fail(); break; }
        tc::fence_after_sync();
        for (int b = 0; b < kDwFlush && int(it) < nk; ++b, ++it) {
          const int s = it % S;
          if (!tc::mbar_wait(full_bar(s), (it / S) & 1u, kRtWaitNs, abort_flag)) { fail(); ok = false; break; }
          tc::fence_after_sync();
          const uint32_t a_s = s0 + s * stage_bytes;
          const uint64_t a0 = tc::smem_desc_sw128(a_s, 8192, 1024), b0 = tc::smem_desc_sw128(a_s + a_bytes, 16, 1024);
#pragma unroll
          for (int kk = 0; kk < kRtBK / 16; ++kk) {  // (a descriptor's address counts 16 bytes)
            tc::mma_bf16_pair(d, a0 + uint64_t(kk * 128), b0 + uint64_t(kk * 2), idesc, (b | kk) != 0 ? 1u : 0u);
            if (p.G == 1) {
              tc::mma_bf16_pair(d, a0 + uint64_t(kk * 128), b0 + uint64_t(kk * 2) + uint64_t(b_term >> 4), idesc, 1u);
              tc::mma_bf16_pair(d, a0 + uint64_t(kk * 128), b0 + uint64_t(kk * 2) + 2 * uint64_t(b_term >> 4), idesc, 1u);
            }
          }
          tc::mma_commit_pair_mc(empty_bar(s), 0x3);
          issued = true;
        }
        if (!ok) break;
        tc::mma_commit_pair_mc(tfull_bar(a), 0x3);
      }
      if (issued) {
        tc::mma_commit_pair(drain_bar);
        if (!tc::mbar_wait(drain_bar, 0, kRtWaitNs, &no_abort)) fail();
      }
    }
  } else {
    const int q = warp & 3, half = (warp - 2) / 4;
    const uint32_t tempty_leader = tc::mapa(tempty_bar(0), 0);
    float acc[128];  // this lane's feature, experts half * NP/2 + c
#pragma unroll
    for (int c = 0; c < 128; ++c) acc[c] = 0.f;
    bool ok = true;
    const uint32_t flushes = uint32_t(nk + kDwFlush - 1) / kDwFlush;
    for (uint32_t f = 0; f < flushes; ++f) {
      const uint32_t a = f & 1u;
      ok = __all_sync(0xffffffffu, tc::mbar_wait(tfull_bar(a), (f >> 1) & 1u, kRtWaitNs, abort_flag));
      if (!ok) { fail(); break; }
      tc::fence_after_sync();
      const uint32_t tb = tmem_base + (uint32_t(q * 32) << 16) + a * p.buf_cols + uint32_t(half) * half_rows;
      // (8 columns at a time: with 16 the 168 registers that ten warps leave a thread do not hold them)
#pragma unroll
      for (int c = 0; c < 128; c += 8) {
        if (uint32_t(c) < half_rows) {
          uint32_t r[8];
          tc::tmem_ld_32x32b_x8(tb + c, r);
          if (p.G == 3) {
            uint32_t r1[8], r2[8];
            tc::tmem_ld_32x32b_x8(tb + c + p.NP, r1);
            tc::tmem_ld_32x32b_x8(tb + c + 2 * p.NP, r2);
            tc::tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 8; ++i)
              acc[c + i] += __uint_as_float(r[i]) + (__uint_as_float(r1[i]) + __uint_as_float(r2[i]));
          } else {
            tc::tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[c + i] += __uint_as_float(r[i]);
          }
        }
      }
      tc::fence_before_sync();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive_remote(tempty_leader + 8u * a);
    }
    const int row = feature0 + q * 32 + lane;
    if (p.dw != nullptr) {
      // The rows go out whole: through the operands' shared memory, which the last MMA has read (an odd
      // stride: a lane owns a row). After an abort nothing is written.
      const int stride = p.E | 1;
      float *s_dw = reinterpret_cast<float *>(smem_raw + pad);
      const int n = min(int(half_rows), p.E - half * int(half_rows));
#pragma unroll
      for (int c = 0; c < 128; ++c)
        if (ok && c < n) s_dw[(q * 32 + lane) * stride + half * half_rows + c] = acc[c];
      asm volatile("bar.sync 1, 256;" ::: "memory");
      for (int r = warp - 2; r < kRtBM; r += 8) {
        if (!ok || feature0 + r >= p.M) break;
        for (int e = lane; e < p.E; e += 32) p.dw[size_t(feature0 + r) * p.E + e] = s_dw[r * stride + e];
      }
    } else if (ok && row < p.M) {
      float *dst = p.partial + (size_t(split) * p.M + row) * p.NE + half * half_rows;
#pragma unroll
      for (int c = 0; c < 128; c += 4)
        if (uint32_t(c) < half_rows) *reinterpret_cast<float4 *>(dst + c) = make_float4(acc[c], acc[c + 1], acc[c + 2], acc[c + 3]);
    }
  }
  tc::fence_before_sync();
  __syncthreads();
  tc::cluster_sync();  // no CTA leaves while its peer may still signal it
  if (warp == 1) {
    tc::fence_after_sync();
    tc::tmem_dealloc_pair(tmem_base, 2 * p.buf_cols);
  }
}

// Splits of the reduction over nkb k-blocks for d features: the least estimated time (ns), a pair's k-block
// in its MMAs, its shared-memory traffic or its share of the HBM rate for x, whole rounds of the 76 pairs with ~3 us of
// filling and draining each, and a split's partial sums written and read. A function of (d, nkb, NP) alone.
// One k-block, or up to kDwFlush of more than 64 experts: one split, which writes the gradient itself; the launch that
// adds the splits costs more than their k-blocks. moe_route_bwd_dense and moe_route_dx, splits / one: 17.2 / 15.6 us at
// 5 tokens, d 424, 8 experts, 19.5 / 18.6 at 60, 7168, 64, 30.6 / 24.2 at 250, 7168, 171, 27.3 / 26.5 at 200, 2872, 225;
// 18.4 / 19.2 at 256, 512, 64, 18.2 / 18.8 at 125, 4280, 8.
int route_dwp_splits(int M, int nkb, int NP) {
  if (nkb == 1 || (nkb <= kDwFlush && NP > 64)) return 1;
  const int64_t tiles = (M + 2 * kRtBM - 1) / (2 * kRtBM), pairs = kRtSms / 2;
  const int64_t a = kRtBM * kRtBK * 2, b = 3 * int64_t(NP / 2) * 128, reads = route_dwp_group(NP) == 3 ? 1 : 3;
  // (MMA: 3 terms x 4 steps of 256 x NP x 16 at a pair's 8,192 multiply-adds a clock, 1.9 GHz)
  const int64_t kb_ns = std::max<int64_t>({a * 1000 / 44700, (a + b + reads * a + b) * 1000 / 243000, int64_t(NP) * 6000 / 1900});
  const int64_t ne = (NP + 31) / 32 * 32;
  int best = 1;
  int64_t best_ns = INT64_MAX;
  for (int r = 1; r <= 8; ++r) {  // the splits that fill r rounds
    const int want = int(std::max<int64_t>(1, std::min<int64_t>({r * pairs / tiles, nkb, kRtDwSplits})));
    const int per = (nkb + want - 1) / want, s = (nkb + per - 1) / per;  // every split gets at least one k-block
    const int64_t ns = (tiles * s + pairs - 1) / pairs * (per * kb_ns + 3000) + s * int64_t(M) * ne * 8 / 4000;
    if (ns < best_ns) {
      best_ns = ns;
      best = s;
    }
  }
  return best;
}

// dw_router[i, e] = sum over the splits, in order, of partial[split][i][e]; four experts per thread,
// four partials in flight.
__global__ void route_dw_reduce_kernel(const float *__restrict__ partial, int splits, int d,
                                       int E, int NE, float *__restrict__ dw_router) {
  pdl_start();
  const int n4 = NE / 4;
  const size_t plane = size_t(d) * n4;
  const float4 *src = reinterpret_cast<const float4 *>(partial);
  for (int idx = blockIdx.x * blockDim.x + threadIdx.x; idx < d * n4; idx += gridDim.x * blockDim.x) {
    const int i = idx / n4, e = 4 * (idx - i * n4);
    if (e >= E) continue;
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    for (int y = 0; y < splits; y += 4) {
      float4 v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (y + u < splits) v[u] = src[(y + u) * plane + idx];
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (y + u < splits) {
          acc[0] += v[u].x;
          acc[1] += v[u].y;
          acc[2] += v[u].z;
          acc[3] += v[u].w;
        }
    }
#pragma unroll
    for (int c = 0; c < 4; ++c)
      if (e + c < E) dw_router[size_t(i) * E + e + c] = acc[c];
  }
}

__global__ void zero_f32_kernel(float *p, int n) {
  pdl_start();
  for (int i = blockIdx.x * blockDim.x + threadIdx.x; i < n; i += gridDim.x * blockDim.x) p[i] = 0.f;
}

// ---- dx = bf16(dx_in + dz W^T) on the tensor cores ------------------------------
// Both factors in half precision: a row of dz [T, E] and a row of W [d, E] (one output column) are each
// scaled by the power of two that brings their largest value into [2^14, 2^15), and split into two terms: 22
// significant bits down to 2^-18 of the row's largest value, an absolute step of 2^-39 of it below. Three products are
// summed, z1 w1 + z2 w1 + z1 w2 (the fourth is 2^-22 of the first); each product is exact, the sum is fp32, and the two
// powers of two are taken out of it exactly. What is lost is ~2^-21 of sum |dz| |W| and the accumulation's truncation,
// where one term of each lost 2^-11 per factor, which shows wherever dx_in and the product cancel. (As good with
// bf16 terms takes six products; tf32 has the bits of one half-precision term.)
//
// HBM-bound up to 64 experts (dx_in read, dx written: 4 bytes per 6 E operations), above by the tensor cores
// beside it. A persistent CTA pair takes
// consecutive 256-token x 256-column tiles, columns first, so that a token block's operand stays in shared memory
// for its whole row of tiles and W's (a few MB) comes from L2, half to each CTA. Warp 0 of each CTA
// issues its operand loads, one thread of the even CTA the MMAs, into two accumulators; warps 2..17 add dx_in. Each
// of those has its own ring of 32-row x 32-column pieces of dx: a piece is loaded by TMA, two pieces
// ahead where there are three, gets the products added in place, and is stored by TMA from there. No piece is touched by
// two warps, so dx_in may be dx.
// T=65536, d=7168: 307 us at up to 64 experts (6.1 TB/s; a copy of dx takes 275), 351 at 128, 389 at 171, 499 at
// 256. One product: 311 / 313 / 317 / 341. MMAs alone take 247 us at 192 experts, 140 clocks each. Tried with one product:
// single SMs, which load all of W's operand, 317 at 171 experts and 400 at 256; eight
// adding warps with pieces of 64 columns 318 and 340; 128-column tiles 416 at 171.
constexpr int kDxBN = 256;
constexpr int kDxEpiWarps = 16;
constexpr int kDxThreads = 64 + 32 * kDxEpiWarps;
constexpr uint32_t kDxABlock = kRtBM * kRtBK * 2, kDxBStage = kDxBN / 2 * kRtBK * 2, kDxSlotBytes = 32 * 32 * 2;

struct RouteDxParams {
  int T, d, NP;  // NP: experts rounded up to 16
  int nkb;       // 64-wide k-blocks
  int n_tiles, tiles, stages;
  int has_in;    // dx_in given
  const float *row_scale, *col_scale;  // what the factors' rows were divided by (col_scale padded to 64)
};

// Pieces of a warp's ring: three up to 128 experts; above, the operands leave room for one beside four to six stages (two
// and two stages at 256 experts: 669 us instead of 499).
int route_dx_slots(int nkb) { return nkb <= 2 ? 3 : 1; }
int route_dx_stages(int nkb, int slots) {
  const int64_t rest = kRtMaxSmem - 2048 - int64_t(2 * nkb) * kDxABlock - int64_t(kDxEpiWarps) * slots * kDxSlotBytes;
  return int(std::min<int64_t>(6, rest / kDxBStage));  // 4 with two or four k-blocks
}
size_t route_dx_smem(int nkb, int stages, int slots) {
  return 1024 + size_t(2 * nkb) * kDxABlock + size_t(stages) * kDxBStage + size_t(kDxEpiWarps) * slots * kDxSlotBytes +
         size_t(2 * stages + 8 + kDxEpiWarps * slots) * 8 + 16;
}

// Rows of W, then rows of dz (E fp32 values each) -> two half-precision terms each [rows][2][NP] and their scales.
__global__ void __launch_bounds__(256) route_dx_split_kernel(const float *__restrict__ w, const float *__restrict__ dz,
                                                             int d, int d_pad, int T, int E, int NP,
                                                             __half *__restrict__ w16, float *__restrict__ col_scale,
                                                             __half *__restrict__ z16, float *__restrict__ row_scale) {
  pdl_start();
  const int lane = threadIdx.x & 31;
  for (int64_t r = int64_t(blockIdx.x) * 8 + (threadIdx.x >> 5); r < int64_t(d_pad) + T; r += int64_t(gridDim.x) * 8) {
    const bool is_w = r < d_pad;
    if (is_w && r >= d) {  // the columns that round d up to whole pieces
      if (lane == 0) col_scale[r] = 0.f;
      continue;
    }
    const int64_t i = is_w ? r : r - d_pad;
    const float *src = (is_w ? w : dz) + size_t(i) * E;
    float v[8];
    uint32_t m = 0;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int e = lane + 32 * u;
      v[u] = e < E ? src[e] : 0.f;
      m = max(m, __float_as_uint(v[u]) & 0x7fffffffu);
    }
    m = __reduce_max_sync(0xffffffffu, m);
    // exponent of the largest value (of a row with an infinity or NaN: as it is; below 2^-111: as 2^-111)
    int e = int(m >> 23);
    e = e == 255 ? 141 : max(e, 16);
    const float up = __uint_as_float(uint32_t(268 - e) << 23);  // 2^(14 - (e - 127))
    __half *dst = (is_w ? w16 : z16) + size_t(i) * (2 * NP);
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (lane + 32 * u < NP) {
        const float y = v[u] * up;
        const __half hi = __float2half_rn(y);
        dst[lane + 32 * u] = hi;
        dst[NP + lane + 32 * u] = __float2half_rn(y - __half2float(hi));
      }
    // (2^24 from one scale to the other: a sum, below 2^38, times dz's alone then stays finite for any dz; a row of W
    // from 2^118 on gets an infinite scale)
    if (lane == 0) (is_w ? col_scale : row_scale)[i] = __uint_as_float(uint32_t(e - 14) << 23) * (is_w ? 0x1p24f : 0x1p-24f);
  }
}

template <int SLOTS>
__global__ void __launch_bounds__(kDxThreads, 1)
    route_dx_kernel(const __grid_constant__ CUtensorMap tmZ, const __grid_constant__ CUtensorMap tmW,
                    const __grid_constant__ CUtensorMap tmIn, const __grid_constant__ CUtensorMap tmOut,
                    const RouteDxParams p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = tc::smem_u32(smem_raw);
  const uint32_t pad = (1024u - (raw & 1023u)) & 1023u;
  const int S = p.stages;
  const uint32_t sA = raw + pad, sB = sA + uint32_t(2 * p.nkb) * kDxABlock, sSlots = sB + uint32_t(S) * kDxBStage;
  const uint32_t bars_off = pad + uint32_t(2 * p.nkb) * kDxABlock + uint32_t(S) * kDxBStage + kDxEpiWarps * SLOTS * kDxSlotBytes;
  uint64_t *bars = reinterpret_cast<uint64_t *>(smem_raw + bars_off);
  int *misc = reinterpret_cast<int *>(bars + 2 * S + 8 + kDxEpiWarps * SLOTS);
  volatile int *abort_flag = misc + 1;
  volatile int no_abort = 0;
  const uint32_t bar0 = tc::smem_u32(bars);
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (S + s); };
  auto tfull_bar = [&](int a) { return bar0 + 8u * (2 * S + a); };
  auto tempty_bar = [&](int a) { return bar0 + 8u * (2 * S + 2 + a); };
  const uint32_t afull_bar = bar0 + 8u * (2 * S + 4), aempty_bar = bar0 + 8u * (2 * S + 5);
  const uint32_t drain_bar = bar0 + 8u * (2 * S + 6);
  auto slot_bar = [&](int w, int s) { return bar0 + 8u * (2 * S + 8 + w * SLOTS + s); };
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr uint32_t IDESC = tc::idesc_f16_f32(2 * kRtBM, kDxBN);
  const uint32_t rank = tc::cluster_ctarank();
  const bool leader = rank == 0;

  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s) {
      tc::mbar_init(full_bar(s), 1);
      tc::mbar_init(empty_bar(s), 1);
    }
    for (int a = 0; a < 2; ++a) {
      tc::mbar_init(tfull_bar(a), 1);
      tc::mbar_init(tempty_bar(a), 2 * kDxEpiWarps);  // of both CTAs
    }
    tc::mbar_init(afull_bar, 1);
    tc::mbar_init(aempty_bar, 1);
    tc::mbar_init(drain_bar, 1);
    for (int w = 0; w < kDxEpiWarps; ++w)
      for (int s = 0; s < SLOTS; ++s) tc::mbar_init(slot_bar(w, s), 1);
    tc::fence_mbar_init();
    misc[1] = 0;
  }
  if (warp == 1) {
    tc::tmem_alloc_pair(tc::smem_u32(misc), 2 * kDxBN);
    tc::tmem_relinquish_pair();
  }
  tc::fence_before_sync();
  __syncthreads();
  tc::cluster_sync();  // barriers of both CTAs initialized before any remote use
  tc::fence_after_sync();
  const uint32_t tmem_base = static_cast<uint32_t>(misc[0]);
  pdl_start();
  const int pair = int(blockIdx.x / 2), pairs = int(gridDim.x / 2);
  const int tile0 = int(int64_t(p.tiles) * pair / pairs), tile1 = int(int64_t(p.tiles) * (pair + 1) / pairs);
  auto fail = [&]() {
    dev_flag(&g_dev_err, MOE_DEV_WAIT_TIMEOUT);
    *abort_flag = 1;
  };

  if (warp == 0) {
    if (lane == 0) {
      const uint32_t full_leader = tc::mapa(full_bar(0), 0), afull_leader = tc::mapa(afull_bar, 0);
      uint32_t it = 0, blocks = 0, s = 0, phase = 1;  // (s = it % S, phase = parity of the round before)
      int m_now = -1;
      bool ok = true;
      for (int tile = tile0; tile < tile1 && ok; ++tile) {
        const int m = tile / p.n_tiles, n = tile - m * p.n_tiles;
        if (m != m_now) {
          if (blocks > 0 && !tc::mbar_wait(aempty_bar, (blocks - 1) & 1u, kRtWaitNs, abort_flag)) { fail(); break; }
          if (leader) tc::mbar_arrive_expect_tx(afull_bar, 4 * uint32_t(p.nkb) * kDxABlock);
          for (int kb = 0; kb < p.nkb; ++kb)
            for (int term = 0; term < 2; ++term)
              tc::tma_load_2d_pair(sA + (2 * kb + term) * kDxABlock, &tmZ, afull_leader, term * p.NP + kb * kRtBK,
                                   (2 * m + int(rank)) * kRtBM);
          ++blocks;
          m_now = m;
        }
        for (int b = 0; b < 2 * p.nkb; ++b, ++it) {  // a k-block's first term, then its second
          if (!tc::mbar_wait(empty_bar(s), phase, kRtWaitNs, abort_flag)) { fail(); ok = false; break; }
          if (leader) tc::mbar_arrive_expect_tx(full_bar(s), 2 * kDxBStage);
          tc::tma_load_2d_pair(sB + s * kDxBStage, &tmW, full_leader + 8u * s, (b & 1) * p.NP + (b >> 1) * kRtBK,
                               n * kDxBN + int(rank) * (kDxBN / 2));
          if (++s == uint32_t(S)) {
            s = 0;
            phase ^= 1u;
          }
        }
      }
      // every issued load lands before the CTAs may exit (the even CTA's barriers count both CTAs')
      if (leader) {
        for (int s = 0; s < S; ++s)
          if (it > uint32_t(s) && !tc::mbar_wait(full_bar(s), ((it - 1 - s) / S) & 1u, kRtWaitNs, &no_abort)) fail();
        if (blocks > 0 && !tc::mbar_wait(afull_bar, (blocks - 1) & 1u, kRtWaitNs, &no_abort)) fail();
      }
    }
  } else if (warp == 1) {
    if (leader && lane == 0) {
      uint32_t blocks = 0, tcount = 0, s = 0, phase = 0;
      const uint64_t a_desc = tc::smem_desc_sw128(sA, 16, 1024), b_desc = tc::smem_desc_sw128(sB, 16, 1024);
      const int last_steps = (p.NP - (p.nkb - 1) * kRtBK) / 16;
      int m_now = -1;
      bool ok = true, issued = false;
      for (int tile = tile0; tile < tile1 && ok; ++tile, ++tcount) {
        const int m = tile / p.n_tiles;
        const uint32_t a = tcount & 1u;
        if (m != m_now) {
          if (!tc::mbar_wait(afull_bar, blocks & 1u, kRtWaitNs, abort_flag)) { fail(); break; }
          ++blocks;
          m_now = m;
        }
        if (!tc::mbar_wait(tempty_bar(a), ((tcount >> 1) & 1u) ^ 1u, kRtWaitNs, abort_flag)) { fail(); break; }
        const uint32_t d = tmem_base + a * kDxBN;
        for (int kb = 0; kb < p.nkb && ok; ++kb) {
          const int steps = kb + 1 < p.nkb ? 4 : last_steps;
          // (descriptors' addresses count 16 bytes; straight code: with the stage from a division and a loop over the
          // steps, issuing took longer than the products)
          const uint64_t ad = a_desc + uint64_t(2 * kb) * (kDxABlock >> 4);
#pragma unroll
          for (int term = 0; term < 2; ++term) {
            if (!tc::mbar_wait(full_bar(s), phase, kRtWaitNs, abort_flag)) { fail(); ok = false; break; }
            tc::fence_after_sync();
            const uint64_t bd = b_desc + uint64_t(s) * (kDxBStage >> 4);
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
              if (kk >= steps) break;
              tc::mma_bf16_pair(d, ad + uint64_t(2 * kk), bd + uint64_t(2 * kk), IDESC, term != 0 || kk != 0 || kb != 0);
              if (term == 0)  // dz's second term
                tc::mma_bf16_pair(d, ad + uint64_t((kDxABlock >> 4) + 2 * kk), bd + uint64_t(2 * kk), IDESC, 1u);
            }
            tc::mma_commit_pair_mc(empty_bar(s), 0x3);
            issued = true;
            if (++s == uint32_t(S)) {
              s = 0;
              phase ^= 1u;
            }
          }
        }
        if (!ok) break;
        tc::mma_commit_pair_mc(tfull_bar(a), 0x3);
        if ((tile + 1) / p.n_tiles != m) tc::mma_commit_pair_mc(aempty_bar, 0x3);  // the token block's last tile
      }
      if (issued) {
        tc::mma_commit_pair(drain_bar);
        if (!tc::mbar_wait(drain_bar, 0, kRtWaitNs, &no_abort)) fail();
      }
    }
  } else {
    const int w = warp - 2, q = warp & 3, part = w / 4;
    const uint32_t tempty_leader = tc::mapa(tempty_bar(0), 0);
    const uint32_t slots = sSlots + uint32_t(w) * (SLOTS * kDxSlotBytes);
    // This warp's pieces: (tile, c), c = 0 or 1, column c * 32 of its quarter of the tile; those that lie
    // wholly past dx are left out. Piece n is in slot n % SLOTS.
    struct Piece {
      int tile, c;
    };
    auto row_of = [&](const Piece &x) { return (x.tile / p.n_tiles * 2 + int(rank)) * kRtBM + q * 32; };
    auto col_of = [&](const Piece &x) { return x.tile % p.n_tiles * kDxBN + part * 64 + x.c * 32; };
    auto inside = [&](const Piece &x) { return row_of(x) < p.T && col_of(x) < p.d; };
    auto next = [&](Piece &x) {  // the piece that follows (tile == tile1: none)
      do {
        x.c ^= 1;
        if (x.c == 0) ++x.tile;
      } while (x.tile < tile1 && !inside(x));
    };
    Piece ahead{tile0 - 1, 1};
    next(ahead);
    uint32_t loads = 0, done = 0;
    auto load = [&]() {  // lane 0: the next piece's dx_in into its slot, which its last store has left
      if (p.has_in && ahead.tile < tile1) {
        const uint32_t s = loads % SLOTS;
        tc::mbar_arrive_expect_tx(slot_bar(w, s), kDxSlotBytes);
        tc::tma_load_2d(slots + s * kDxSlotBytes, &tmIn, slot_bar(w, s), col_of(ahead), row_of(ahead));
        next(ahead);
        ++loads;
      }
    };
    if (lane == 0) {
      load();
      if (SLOTS > 1) load();
    }
    bool ok = true;
    uint32_t tcount = 0;
    for (int tile = tile0; tile < tile1 && ok; ++tile, ++tcount) {
      const uint32_t a = tcount & 1u;
      ok = __all_sync(0xffffffffu, tc::mbar_wait(tfull_bar(a), (tcount >> 1) & 1u, kRtWaitNs, abort_flag));
      if (!ok) { fail(); break; }
      tc::fence_after_sync();
      const int row = (tile / p.n_tiles * 2 + int(rank)) * kRtBM + q * 32 + lane;
      const float rs = row < p.T ? p.row_scale[row] : 0.f;
      for (int c = 0; c < 2; ++c) {
        const Piece x{tile, c};
        if (!inside(x)) continue;
        const uint32_t s = done % SLOTS, slot = slots + s * kDxSlotBytes;
        uint32_t r[32];
        tc::tmem_ld_32x32b_x32(tmem_base + (uint32_t(q * 32) << 16) + a * kDxBN + part * 64 + c * 32, r);
        tc::tmem_ld_wait();
        if (p.has_in) {
          ok = __all_sync(0xffffffffu, tc::mbar_wait(slot_bar(w, s), (done / SLOTS) & 1u, kRtWaitNs, abort_flag));
          if (!ok) { fail(); break; }
        } else {
          if (lane == 0) tc::bulk_wait_read<SLOTS - 1>();  // the slot's last store has read it
          __syncwarp();
        }
        const float *cs = p.col_scale + col_of(x);
        const uint32_t mine = slot + uint32_t(lane) * 64u, sw = (uint32_t(lane) >> 1) & 3u;
#pragma unroll
        for (uint32_t v = 0; v < 4; ++v) {
          const uint32_t at = mine + ((v ^ sw) << 4);  // the 64-byte swizzle
          float f[8];
          if (p.has_in) {
            unpack8(tc::ld_shared_v4(at), f);
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = 0.f;
          }
          const float4 c0 = __ldg(reinterpret_cast<const float4 *>(cs + 8 * v)), c1 = __ldg(reinterpret_cast<const float4 *>(cs + 8 * v + 4));
          const float sc[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w};
#pragma unroll
          for (int i = 0; i < 8; ++i) f[i] = fmaf(__uint_as_float(r[8 * v + i]) * rs, sc[i], f[i]);
          tc::st_shared_v4(at, pack8(f));
        }
        tc::fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          tc::tma_store_2d(&tmOut, slot, col_of(x), row_of(x));
          tc::bulk_commit();
          if (p.has_in) {
            tc::bulk_wait_read<(SLOTS > 1 ? 1 : 0)>();  // the store before this one (with one slot: this one) has left its slot
            load();
          }
        }
        ++done;
      }
      tc::fence_before_sync();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive_remote(tempty_leader + 8u * a);
    }
    if (lane == 0) {
      for (uint32_t n = done; n < loads; ++n)  // (after an abort: loads nothing read)
        if (!tc::mbar_wait(slot_bar(w, n % SLOTS), (n / SLOTS) & 1u, kRtWaitNs, &no_abort)) fail();
      tc::bulk_wait0();
    }
    __syncwarp();
  }
  tc::fence_before_sync();
  __syncthreads();
  tc::cluster_sync();  // no CTA leaves while its peer may still signal it
  if (warp == 1) {
    tc::fence_after_sync();
    tc::tmem_dealloc_pair(tmem_base, 2 * kDxBN);
  }
}

// The regions of route_dx_bytes: W's and dz's rows in half precision, their scales.
int launch_route_dx(const float *dz, const float *w, const uint16_t *dx_in, int T, int d, int E, uint16_t *dx, char *ws,
                    cudaStream_t s) {
  const int NP = route_tc_np(E), d_pad = (d + 63) / 64 * 64;
  __half *w16 = reinterpret_cast<__half *>(ws), *z16 = w16 + size_t(d_pad) * (2 * NP);
  float *col_scale = reinterpret_cast<float *>(z16 + size_t(T) * (2 * NP)), *row_scale = col_scale + d_pad;
  const char *what = "moe_route_dx: factors";
  const int64_t rows = int64_t(d_pad) + T;
  const int grid0 = int(std::min<int64_t>((rows + 7) / 8, int64_t(moe::num_sms()) * 32));
  MOE_LAUNCH("route_dx_split", s, moe::launch_dep(route_dx_split_kernel, grid0, 256, 0, s, w, dz, d, d_pad, T, E, NP, w16,
                                                  col_scale, z16, row_scale));
  if (int st = moe::launch_status(what)) return st;
  what = "moe_route_dx: product";
  RouteDxParams p{};
  p.T = T;
  p.d = d;
  p.NP = NP;
  p.nkb = (NP + kRtBK - 1) / kRtBK;
  p.n_tiles = (d + kDxBN - 1) / kDxBN;
  p.tiles = (T + 2 * kRtBM - 1) / (2 * kRtBM) * p.n_tiles;
  const int slots = route_dx_slots(p.nkb);
  p.stages = route_dx_stages(p.nkb, slots);
  p.has_in = dx_in != nullptr;
  p.row_scale = row_scale;
  p.col_scale = col_scale;
  CUtensorMap mz, mw, mi, mo;
  int st;
  if ((st = moe::make_map(&mz, z16, uint64_t(T), uint64_t(2 * NP), kRtBK, kRtBM, "router dx dz"))) return st;
  if ((st = moe::make_map(&mw, w16, uint64_t(d), uint64_t(2 * NP), kRtBK, kDxBN / 2, "router dx w"))) return st;
  if ((st = moe::make_map(&mo, dx, uint64_t(T), uint64_t(d), 32, 32, "router dx", CU_TENSOR_MAP_SWIZZLE_64B))) return st;
  mi = mo;
  if (dx_in != nullptr &&
      (st = moe::make_map(&mi, dx_in, uint64_t(T), uint64_t(d), 32, 32, "router dx_in", CU_TENSOR_MAP_SWIZZLE_64B)))
    return st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = 2;
  at[0].val.clusterDim.y = 1;
  at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // see moe::launch_dep
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(kDxThreads);
  cfg.stream = s;
  cfg.attrs = at;
  auto kern = slots == 3 ? route_dx_kernel<3> : route_dx_kernel<1>;
  static int fit[2][64] = {};  // pairs at once on each device (one CTA per SM, whatever the sizes)
  int &pairs = fit[slots == 3][moe::device_slot()];
  if (!pairs) {
    cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kRtMaxSmem);
    if (e != cudaSuccess) return moe::cuda_status(e, what);
    cfg.gridDim = dim3(2 * (moe::num_sms() / 2));
    cfg.dynamicSmemBytes = kRtMaxSmem;
    cfg.numAttrs = 1;
    int n = 0;
    e = cudaOccupancyMaxActiveClusters(&n, kern, &cfg);
    if (e != cudaSuccess) return moe::cuda_status(e, what);
    if (n <= 0) return moe::set_error(MOE_ERR_CUDA, "%s: no co-resident CTA pair fits", what);
    pairs = n;
  }
  cfg.gridDim = dim3(2 * std::min(p.tiles, pairs));
  cfg.dynamicSmemBytes = route_dx_smem(p.nkb, p.stages, slots);
  cfg.numAttrs = 2;
  MOE_LAUNCH("route_dx", s, cudaLaunchKernelEx(&cfg, kern, mz, mw, mi, mo, p));
  return moe::launch_status(what);
}

template <bool DW, int G, bool AHEAD = false>
int launch_route_mma(const char *name, dim3 grid, size_t smem, const CUtensorMap &a, const CUtensorMap &b,
                       const RouteTcParams &p, cudaStream_t s, const char *what) {
  static bool attr_set[64] = {};
  bool &set = attr_set[moe::device_slot()];
  if (!set) {
    cudaError_t e = cudaFuncSetAttribute(route_tc_kernel<DW, G, AHEAD>, cudaFuncAttributeMaxDynamicSharedMemorySize, kRtMaxSmem);
    if (e != cudaSuccess) return moe::cuda_status(e, what);
    set = true;
  }
  MOE_LAUNCH(name, s, moe::launch_dep(route_tc_kernel<DW, G, AHEAD>, grid, kRtThreads, smem, s, a, b, p));
  return moe::launch_status(what);
}
// Tensor-core logits: splits W into its three bf16 terms (w3), then one CTA per
// (token tile, split). Returns the number of partial planes written in *splits.
int launch_route_tc(const uint16_t *x, const float *w, int T, int d, int E, int NE, uint16_t *w3,
                    float *partial, int32_t *counts, int *splits_out, cudaStream_t s) {
  const int NP = route_tc_np(E);
  const RtPlan plan = route_logits_plan(T, d, NP);
  const int MT = plan.MT, stages = plan.stages, splits = plan.splits;
  const size_t smem = route_tc_smem(NP, stages, MT);
  dim3 sgrid((d + 31) / 32, (NP + 31) / 32);
  MOE_LAUNCH("route_split_w", s, moe::launch_dep(route_split_w_kernel, sgrid, dim3(32, 8), 0, s, w, d, E, NP, w3, counts));
  if (int st = moe::launch_status("moe_route: split router weight")) return st;
  CUtensorMap mx, mw;
  int st;
  if ((st = moe::make_map(&mx, x, uint64_t(T), uint64_t(d), kRtBK, kRtBM, "router x"))) return st;
  if ((st = moe::make_map(&mw, w3, uint64_t(3 * NP), uint64_t(d), kRtBK, uint32_t(NP), "router w")))
    return st;
  RouteTcParams p;
  p.M = T;
  p.MT = MT;
  p.kb_per_split = plan.kb_per_split;
  p.nkb = (d + kRtBK - 1) / kRtBK;
  p.NP = NP;
  p.NE = NE;
  p.stages = stages;
  p.tmem_cols = route_tc_tmem_cols(NP, MT);
  p.partial = partial;
  dim3 grid((T + kRtBM * MT - 1) / (kRtBM * MT), splits);
  *splits_out = splits;
  // A two-stage ring holds too little to cover an HBM load's way (~1.1 us a k-block), so the x tile
  // of a stage's next use goes to L2 while this one loads: 78.0 / 72.6 us at T=32768, d=4096,
  // 128 experts, 62.2 / 56.3 at 64, 428 / 412 at T=65536, d=7168, 208. Not with more stages (no gain
  // at 28 and 112 experts, 3 stages), nor above 208 experts, where the weights are most of a stage
  // (277 / 283 at T=65536, d=4096, 240), nor where a tile's rows straddle 128-byte lines (36.6 / 45.9
  // at T=16545, d=3336, 49 experts; 30.7 / 32.8 at d=3360), nor over few k-blocks. Further ahead is
  // slower (73.4 us three, 79 eight k-blocks on), and so it is for x^T dZ (40.9 / 47.8 at T=35700,
  // d=2856, 57 experts).
  const bool ahead = stages == 2 && NP <= 208 && plan.kb_per_split >= 16 && d % 64 == 0 &&
                     (reinterpret_cast<uintptr_t>(x) & 127) == 0;
  const char *what = "moe_route: logits";
  return ahead ? launch_route_mma<false, 1, true>("route_logits", grid, smem, mx, mw, p, s, what)
               : launch_route_mma<false, 1, false>("route_logits", grid, smem, mx, mw, p, s, what);
}

int launch_route(const uint16_t *x, const float *w, const float *b, const uint8_t *mask, int T,
                 int d, int E, int k, const float *lin, float *lout, int32_t *idx, float *gate,
                 int32_t *counts, float *partial, uint16_t *w3, cudaStream_t s) {
  int splits = 0;
  const int NE = padded_experts(E);
  if (lin == nullptr)
    if (int st = launch_route_tc(x, w, T, d, E, NE, w3, partial, counts, &splits, s)) return st;
  // at most eight blocks per SM, so that each block's shared histogram sums ~50 tokens'
  // assignments or more before its global atomics (one block per 8 tokens sent 512k atomics to
  // the counters at T=65536, top-8; the heaviest expert's counter took ~60k of them one after
  // another)
  const bool wide = T <= 2048;  // 16 lanes per token: 6.5 against 16 us at T=764, 198 experts, 13 against 7 at T=8192, 64
  const int per_block = kTopkThreads / (wide ? 16 : 4);
  const int grid = int(std::min<int64_t>((int64_t(T) + per_block - 1) / per_block, int64_t(moe::num_sms()) * 8));
  auto launch = [&](auto kern) {
    MOE_LAUNCH("route_topk", s, moe::launch_dep(kern, grid, kTopkThreads, 0, s, partial, splits, NE, lin, b, mask, T, E,
                                                k, lout, idx, gate, counts));
  };
  if (k <= 2) launch(wide ? route_topk_kernel<2, 16> : route_topk_kernel<2, 4>);
  else if (k <= 4) launch(wide ? route_topk_kernel<4, 16> : route_topk_kernel<4, 4>);
  else launch(wide ? route_topk_kernel<8, 16> : route_topk_kernel<8, 4>);
  return moe::launch_status("moe_route: top-k");
}

}  // namespace

namespace moe {
MOE_DEV_ERR_DEFINE_READER(route_dev_error)

size_t route_partial_bytes(int T, int d, int E) {
  if (T <= 0) return 0;
  const int splits = route_logits_plan(T, d, route_tc_np(E)).splits;
  return size_t(splits) * size_t(T) * size_t(padded_experts(E)) * 4;
}
size_t route_w3_bytes(int d, int E) { return size_t(3) * route_tc_np(E) * size_t(d) * 2; }
size_t route_dz3_bytes(int T, int E) {
  return size_t(3) * route_tc_np(E) * size_t(route_tokens_padded(T)) * 2;
}
size_t route_dx_bytes(int T, int d, int E) {
  const size_t rows = size_t(std::max(T, 0)) + size_t((d + 63) / 64 * 64);
  return rows * (size_t(route_tc_np(E)) * 4 + 4);
}
size_t route_dw_partial_bytes(int T, int d, int E) {
  if (T <= 0) return 0;
  const int NP = route_tc_np(E), Tp = route_tokens_padded(T);
  int splits = route_dw_plan(d, Tp, NP).splits;
  if (E <= 256) splits = std::max(splits, route_dwp_splits(d, Tp / kRtBK, NP));  // (moe_route_bwd_dense)
  return size_t(splits) * size_t(d) * size_t(route_dw_stride(E)) * 4;
}
}  // namespace moe

extern "C" {

int moe_route(const uint16_t *x, const float *w_router, const float *bias,
              const uint8_t *active_mask, int T, int d, int E, int k, const float *logits_in,
              float *logits_out, int32_t *topk_idx, float *topk_gate, int32_t *counts, void *ws,
              size_t ws_bytes, moe_stream_t stream) {
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (E < 1 || E > 256) return moe::set_error(MOE_ERR_UNSUPPORTED, "moe_route: E=%d not in [1,256]", E);
  if (k < 1 || k > 8 || k > E) return moe::set_error(MOE_ERR_UNSUPPORTED, "moe_route: k=%d", k);
  if (T < 0 || d <= 0 || d % 8) return moe::set_error(MOE_ERR_ARG, "moe_route: T=%d d=%d", T, d);
  if (T > 0 && (!topk_idx || !topk_gate)) return moe::set_error(MOE_ERR_ARG, "moe_route: null output");
  if (T > 0 && !logits_in && (!x || !w_router))
    return moe::set_error(MOE_ERR_ARG, "moe_route: null x/w_router");
  if (x && !moe::aligned16(x)) return moe::set_error(MOE_ERR_ARG, "moe_route: x not 16-byte aligned");
  float *partial = nullptr;
  uint16_t *w3 = nullptr;
  if (!logits_in && T > 0) {
    const moe::WsLayout L = moe::ws_layout(T, d, E, k, 0);
    if (!ws || ws_bytes < L.total) return moe::set_error(MOE_ERR_WORKSPACE, "moe_route: workspace");
    if (!moe::aligned16(ws)) return moe::set_error(MOE_ERR_ARG, "moe_route: ws alignment");
    partial = reinterpret_cast<float *>(static_cast<char *>(ws) + L.route_partial);
    w3 = reinterpret_cast<uint16_t *>(static_cast<char *>(ws) + L.route_w3);
  }
  if (counts && (logits_in || T == 0)) {  // else zeroed by the kernel that splits w_router
    MOE_LAUNCH("zero_counts", s, moe::launch_dep(zero_i32_kernel, 1, 256, 0, s, counts, E));
    if (int st = moe::launch_status("moe_route: zero counts")) return st;
  }
  if (T == 0) return MOE_OK;
  return launch_route(x, w_router, bias, active_mask, T, d, E, k, logits_in, logits_out, topk_idx, topk_gate, counts,
                      partial, w3, s);
}

int moe_load_stats(const int32_t *topk_idx, int T, int k, int E, int32_t *counts, int accumulate,
                   moe_stream_t stream) {
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (E < 1 || E > 256 || k < 1 || T < 0) return moe::set_error(MOE_ERR_ARG, "moe_load_stats: sizes");
  if (!counts || (T > 0 && !topk_idx)) return moe::set_error(MOE_ERR_ARG, "moe_load_stats: null");
  const int64_t A = int64_t(T) * k;
  if (!accumulate && A <= 8192) {  // one block (8 loads per thread), no launch to zero the counts
    MOE_LAUNCH("load_stats", s, moe::launch_dep(load_stats_kernel, 1, 1024, 0, s, topk_idx, A, E, 1, counts));
    return moe::launch_status("moe_load_stats: launch");
  }
  if (!accumulate) {
    MOE_LAUNCH("zero_counts", s, moe::launch_dep(zero_i32_kernel, 1, 256, 0, s, counts, E));
    if (int st = moe::launch_status("moe_load_stats: zero")) return st;
  }
  if (A == 0) return MOE_OK;
  const int grid = int(std::min<int64_t>((A + 255) / 256, int64_t(moe::num_sms()) * 4));
  MOE_LAUNCH("load_stats", s, moe::launch_dep(load_stats_kernel, grid, 256, 0, s, topk_idx, A, E, 0, counts));
  return moe::launch_status("moe_load_stats: launch");
}

}  // extern "C"

namespace {
// Weight-gradient launch on the tensor cores: partial[split][i][e] over the split's tokens.
int launch_route_dw(const uint16_t *x, const uint16_t *dz3, int T, int d, int E, float *partial,
                    int *splits_out, cudaStream_t s) {
  const int NP = route_tc_np(E), Tp = route_tokens_padded(T);
  const RtPlan plan = route_dw_plan(d, Tp, NP);
  const int MT = plan.MT, stages = plan.stages, splits = plan.splits;
  const size_t smem = route_tc_smem(NP, stages, MT);
  CUtensorMap mx, mz;
  int st;
  // x [T, d] read as 64 features x 64 tokens boxes (features contiguous: MN-major A)
  if ((st = moe::make_map(&mx, x, uint64_t(T), uint64_t(d), 64, kRtBK, "router bwd x"))) return st;
  if ((st = moe::make_map(&mz, dz3, uint64_t(3 * NP), uint64_t(Tp), kRtBK, uint32_t(NP), "router bwd dz")))
    return st;
  RouteTcParams p;
  p.M = d;
  p.MT = MT;
  p.kb_per_split = plan.kb_per_split;
  p.nkb = Tp / kRtBK;
  p.NP = NP;
  p.NE = route_dw_stride(E);
  p.stages = stages;
  p.tmem_cols = route_tc_tmem_cols(route_dw_group(NP) * NP, MT);
  p.partial = partial;
  dim3 grid((d + kRtBM * MT - 1) / (kRtBM * MT), splits);
  *splits_out = splits;
  const char *what = "moe_route_bwd: weight gradient";
  switch (route_dw_group(NP)) {
    case 1: return launch_route_mma<true, 1>("route_bwd_dw", grid, smem, mx, mz, p, s, what);
    case 2: return launch_route_mma<true, 2>("route_bwd_dw", grid, smem, mx, mz, p, s, what);
    default: return launch_route_mma<true, 3>("route_bwd_dw", grid, smem, mx, mz, p, s, what);
  }
}

// As launch_route_dw, on CTA pairs (see route_dw_pair_kernel).
int launch_route_dw_pair(const uint16_t *x, const uint16_t *dz3, int T, int d, int E, float *partial,
                         float *dw_router, int *splits_out, cudaStream_t s) {
  const int NP = route_tc_np(E), Tp = route_tokens_padded(T);
  const char *what = "moe_route_bwd_dense: weight gradient";
  RouteDwParams p{};
  p.M = d;
  p.NP = NP;
  p.NE = route_dw_stride(E);
  p.nkb = Tp / kRtBK;
  const int splits = route_dwp_splits(d, p.nkb, NP);
  p.kb_per_split = (p.nkb + splits - 1) / splits;
  p.G = route_dwp_group(NP);
  p.stages = route_dwp_stages(NP);
  const uint32_t cols = uint32_t(p.G * NP);
  p.buf_cols = cols <= 32 ? 32u : cols <= 64 ? 64u : cols <= 128 ? 128u : 256u;
  p.partial = partial;
  p.dw = splits == 1 ? dw_router : nullptr;
  p.E = E;
  CUtensorMap mx, mz;
  int st;
  if ((st = moe::make_map(&mx, x, uint64_t(T), uint64_t(d), 64, kRtBK, "router bwd x"))) return st;
  if ((st = moe::make_map(&mz, dz3, uint64_t(3 * NP), uint64_t(Tp), kRtBK, uint32_t(p.G * NP / 2), "router bwd dz")))
    return st;
  static bool attr_set[64] = {};
  bool &set = attr_set[moe::device_slot()];
  if (!set) {
    cudaError_t e = cudaFuncSetAttribute(route_dw_pair_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRtMaxSmem);
    if (e != cudaSuccess) return moe::cuda_status(e, what);
    set = true;
  }
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = 2;
  at[0].val.clusterDim.y = 1;
  at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // see moe::launch_dep
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(2 * ((d + 2 * kRtBM - 1) / (2 * kRtBM)), splits);
  cfg.blockDim = dim3(kDwThreads);
  cfg.dynamicSmemBytes = route_dwp_smem(NP, p.stages);
  cfg.stream = s;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  *splits_out = splits;
  MOE_LAUNCH("route_bwd_dw", s, cudaLaunchKernelEx(&cfg, route_dw_pair_kernel, mx, mz, p));
  return moe::launch_status(what);
}
}  // namespace

extern "C" {

static int route_bwd(const char *fn, const uint16_t *x, const int32_t *topk_idx, const float *topk_gate,
                     const float *d_gate, const float *dz, int T, int d, int E, int k, float *d_logits,
                     float *dw_router, void *ws, size_t ws_bytes, cudaStream_t s) {
  if (E < 1 || E > 256 || k < 1 || k > 8 || k > E || T < 0 || d <= 0 || d % 8)
    return moe::set_error(MOE_ERR_ARG, "%s: sizes", fn);
  const bool gates = dz == nullptr || topk_idx || topk_gate || d_gate || d_logits;
  if (!dw_router || (T > 0 && (!x || !ws || (gates && (!topk_idx || !topk_gate || !d_gate || !d_logits)))))
    return moe::set_error(MOE_ERR_ARG, "%s: null pointer", fn);
  if ((x && !moe::aligned16(x)) || (ws && !moe::aligned16(ws)))
    return moe::set_error(MOE_ERR_ARG, "%s: alignment", fn);
  if (T == 0) {
    const int n = d * E;
    MOE_LAUNCH("zero_dw_router", s, moe::launch_dep(zero_f32_kernel, std::min((n + 255) / 256, 1024), 256, 0, s, dw_router, n));
    return moe::launch_status("moe_route_bwd: zero");
  }
  const moe::WsLayout L = moe::ws_layout(T, d, E, k, 0);
  if (ws_bytes < L.total) return moe::set_error(MOE_ERR_WORKSPACE, "%s: workspace", fn);
  uint16_t *dz3 = reinterpret_cast<uint16_t *>(static_cast<char *>(ws) + L.route_dz3);
  float *partial = reinterpret_cast<float *>(static_cast<char *>(ws) + L.route_dw_partial);
  const int NP = route_tc_np(E), Tp = route_tokens_padded(T);
  dim3 zgrid((Tp + 255) / 256, (NP + kDzExperts - 1) / kDzExperts);
  if (dz)
    MOE_LAUNCH("route_bwd_dz", s, moe::launch_dep(route_bwd_dz_dense_kernel, dim3(Tp / kDzTile, (NP + kDzTile - 1) / kDzTile), 256,
                                      0, s, topk_idx, topk_gate, d_gate, dz, T, Tp, E, k, NP, d_logits, dz3));
  else
    MOE_LAUNCH("route_bwd_dz", s, moe::launch_dep(route_bwd_dz_kernel, zgrid, 256, 0, s,
                                      topk_idx, topk_gate, d_gate, T, Tp, k, NP, d_logits, dz3));
  if (int st = moe::launch_status("moe_route_bwd: dz")) return st;
  int splits = 0;
  if (int st = dz ? launch_route_dw_pair(x, dz3, T, d, E, partial, dw_router, &splits, s)
                  : launch_route_dw(x, dz3, T, d, E, partial, &splits, s))
    return st;
  if (dz && splits == 1) return MOE_OK;  // written at once
  const int n = d * (route_dw_stride(E) / 4);
  MOE_LAUNCH("route_bwd_reduce", s, moe::launch_dep(route_dw_reduce_kernel, std::min((n + 255) / 256, 4 * moe::num_sms()), 256, 0, s,
                                        partial, splits, d, E, route_dw_stride(E), dw_router));
  return moe::launch_status("moe_route_bwd: reduce");
}

int moe_route_bwd(const uint16_t *x, const int32_t *topk_idx, const float *topk_gate,
                  const float *d_gate, int T, int d, int E, int k, float *d_logits,
                  float *dw_router, void *ws, size_t ws_bytes, moe_stream_t stream) {
  return route_bwd("moe_route_bwd", x, topk_idx, topk_gate, d_gate, nullptr, T, d, E, k, d_logits, dw_router, ws,
                   ws_bytes, reinterpret_cast<cudaStream_t>(stream));
}

int moe_route_bwd_dense(const uint16_t *x, const int32_t *topk_idx, const float *topk_gate,
                        const float *d_gate, const float *dz, int T, int d, int E, int k,
                        float *d_logits, float *dw_router, void *ws, size_t ws_bytes,
                        moe_stream_t stream) {
  if (T > 0 && !dz) return moe::set_error(MOE_ERR_ARG, "moe_route_bwd_dense: null dz");
  return route_bwd("moe_route_bwd_dense", x, topk_idx, topk_gate, d_gate, dz, T, d, E, k, d_logits, dw_router, ws,
                   ws_bytes, reinterpret_cast<cudaStream_t>(stream));
}

int moe_route_dx(const float *dz, const float *w_router, const uint16_t *dx_in, int T, int d, int E,
                 int k, uint16_t *dx, void *ws, size_t ws_bytes, moe_stream_t stream) {
  const char *fn = "moe_route_dx";
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (E < 1 || E > 256 || k < 1 || k > 8 || T < 0 || d <= 0 || d % 8) return moe::set_error(MOE_ERR_ARG, "%s: sizes", fn);
  if (T == 0) return MOE_OK;
  if (!dz || !w_router || !dx || !ws) return moe::set_error(MOE_ERR_ARG, "%s: null pointer", fn);
  if (!moe::aligned16(dx) || (dx_in && !moe::aligned16(dx_in)) || !moe::aligned16(ws))
    return moe::set_error(MOE_ERR_ARG, "%s: alignment", fn);
  const moe::WsLayout L = moe::ws_layout(T, d, E, k, 0);
  if (ws_bytes < L.total) return moe::set_error(MOE_ERR_WORKSPACE, "%s: workspace", fn);
  return launch_route_dx(dz, w_router, dx_in, T, d, E, dx, static_cast<char *>(ws) + L.route_dx, s);
}

}  // extern "C"
