// Orthogonalised updates (sm_103a): Newton-Schulz products over a stack of matrices, and the step of an
// optimiser around them (momentum, orthogonalised update, weights).
//
//   X0 = U / (|U|_F + eps);  steps times, with n = the short side:
//     A = X X^T (X^T X where there are more rows than columns),  B = b A + c A A,  X <- a X + B X (X B)
//
// Per step 2 n^2 k + 2 n^3 + 2 n^2 k operations as plain products; A and A A are symmetric and only their tiles at
// or above the diagonal are computed (n^2 k + n^3 + 2 n^2 k).
//
// Precision. The products' operands are half precision: X scaled by a power of two near sqrt(max(rows, cols)), which puts
// its entries around 1 (bf16 would round them 8 times coarser: 1e-2 off in the result, against 1.7e-3 for the result's own
// rounding to bf16). X itself is kept in two such terms, hi + lo / 2048 (22 bits), and a X is taken from both in fp32: with
// hi alone the rounding errors fill the directions that U lacks, and every step multiplies them by a = 3.44 (4e-2 off for
// a gradient of rank 16 in 256 x 512). B's diagonal is near b + c in the last steps; what its rounding leaves is kept
// per row and given back in a X (1.7e-3 -> 1.3e-3 off at 512 x 1,792).
#include <cuda_fp16.h>

#include <math.h>
#include <stdlib.h>

#include "common.cuh"

MOE_DEV_ERR_DECL

#include "dense_gemm.cuh"

namespace {

constexpr float kLo = 2048.f;      // lo = (x - hi) * kLo
constexpr float kScaleA = 64.f;    // A and B are stored times this: entries up to ~1,000 fit, normal down to 1e-6
constexpr int kMaxSteps = 16;
constexpr int kParts = 64;         // blocks that a matrix's sums are taken by, at most

__device__ __forceinline__ uint32_t pack_half2(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ float2 unpack_half2(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2 *>(&v)); }

__device__ __forceinline__ void st_shared_f32(uint32_t addr, float v) {
  asm volatile("st.shared.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory");
}
__device__ __forceinline__ float ld_shared_f32(uint32_t addr) {
  float v;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
  return v;
}

// ---------------------------------------------------------------- epilogues of the products

// A = acc * scale, both halves of the symmetric matrix.
struct GramEpi {
  CUtensorMap out;
  float scale;
  int n;

  static constexpr int kChunk = 0;
  static constexpr bool kTrigger = true;

  template <int BN, int kSlots, class Ready> __device__ __forceinline__ void run(dg::Warp &w, Ready ready) const {
    const int row0 = w.row - w.lane;
    if (row0 >= n || !ready()) return;
    const bool mirror = row0 / dg::kTileRows != w.col / dg::kTileRows;
#pragma unroll 1
    for (int c = 0; c < BN / 2; c += 32) {
      const int col = w.col + c;
      if (col >= n) break;
      uint32_t r[32];
      tc::tmem_ld_32x32b_x32(w.tb + c, r);
      tc::tmem_ld_wait();
      uint4 v[4];
      uint32_t *p = reinterpret_cast<uint32_t *>(v);
#pragma unroll
      for (int i = 0; i < 16; ++i)
        p[i] = pack_half2(__uint_as_float(r[2 * i]) * scale, __uint_as_float(r[2 * i + 1]) * scale);
      dg::stage_and_store(&out, w.st, w.lane, v, col, row0, w.z);
      if (mirror) dg::stage_and_store_t(&out, w.st, w.lane, v, col, row0, w.z);
    }
  }
};

// B = b A + c A A, both halves; what the rounding of its diagonal leaves goes to resid [mats, n].
struct PolyEpi {
  CUtensorMap out;
  const uint16_t *a;    // A [mats, n, pitch]
  float *resid;
  float b, c;
  int n, pitch;

  static constexpr int kChunk = 0;
  static constexpr bool kTrigger = true;

  template <int BN, int kSlots, class Ready> __device__ __forceinline__ void run(dg::Warp &w, Ready ready) const {
    const int row0 = w.row - w.lane;
    if (row0 >= n || w.col >= n) return;
    const bool mirror = row0 / dg::kTileRows != w.col / dg::kTileRows;
    const uint16_t *arow = a + (size_t(w.z) * n + min(w.row, n - 1)) * pitch;
    // A's values of a chunk are loaded a chunk ahead, the first while the products still run
    // (pitch is a multiple of 64: 32 columns never leave the row)
    uint4 x[4], nx[4];
    auto load = [&](int col) {
#pragma unroll
      for (int i = 0; i < 4; ++i) nx[i] = *reinterpret_cast<const uint4 *>(arow + col + 8 * i);
    };
    load(w.col);
    if (!ready()) return;
#pragma unroll 1
    for (int cc = 0; cc < BN / 2; cc += 32) {
      const int col = w.col + cc;
      if (col >= n) break;
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = nx[i];
      if (cc + 32 < BN / 2 && col + 32 < n) load(col + 32);
      uint32_t r[32];
      tc::tmem_ld_32x32b_x32(w.tb + cc, r);
      tc::tmem_ld_wait();
      const uint32_t *xa = reinterpret_cast<const uint32_t *>(x);
      uint4 v[4];
      uint32_t *p = reinterpret_cast<uint32_t *>(v);
      float diag = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float2 ai = unpack_half2(xa[i]);
        const float y0 = fmaf(b, ai.x, c * __uint_as_float(r[2 * i])), y1 = fmaf(b, ai.y, c * __uint_as_float(r[2 * i + 1]));
        p[i] = pack_half2(y0, y1);
        const float2 back = unpack_half2(p[i]);
        if (col + 2 * i == w.row) diag = y0 - back.x;
        if (col + 2 * i + 1 == w.row) diag = y1 - back.y;
      }
      if (w.row >= col && w.row < col + 32 && w.row < n) resid[size_t(w.z) * n + w.row] = diag * (1.f / kScaleA);
      dg::stage_and_store(&out, w.st, w.lane, v, col, row0, w.z);
      if (mirror) dg::stage_and_store_t(&out, w.st, w.lane, v, col, row0, w.z);
    }
  }
};

// X <- (a + resid) X + acc: to the next hi and lo, or with LAST to the caller's tensors.
struct Target {
  const int *live;            // the stack's matrices among the caller's; null: first, first + 1, ...
  int first;
  int vec;                    // rows of 16-byte multiples, 16-byte aligned tensors
  float inv;                  // 1 / X's scale
  uint16_t *out;              // orthogonalised [n_mats, rows, cols], or null: weights
  uint16_t *w;
  float *master;              // may be null
  float keep, step;           // w <- keep w - step O
};

template <bool LAST> struct StepEpi {
  CUtensorMap hi, lo;         // X's terms; lo is replaced in place
  CUtensorMap next;           // the new hi, or with LAST and to.vec the caller's bf16 tensor
  const float *resid;         // [mats, rows or cols]
  float a;
  int rows, cols, tall;
  Target to;

  static constexpr int kChunk = 0;
  static constexpr bool kTrigger = true;

  // A chunk of 32 columns at a time: TMA brings its hi and lo into a slot's two buffers (up to kSlots chunks ahead, the
  // first ones while the products still run), every lane changes its row in place, and TMA stores them.
  template <int BN, int kSlots, class Ready> __device__ __forceinline__ void run(dg::Warp &w, Ready ready) const {
    const int row0 = w.row - w.lane;
    if (row0 >= rows || w.col >= cols) return;
    static_assert(kSlots >= 3, "a slot's store is waited for a chunk later");
    const int chunks = min(BN / 64, (cols - w.col + 31) / 32);
    volatile int never = 0;
    const float *res = resid + size_t(w.z) * (tall ? cols : rows);
    const float ar = tall ? a : a + res[min(w.row, rows - 1)];
    // a slot: hi, lo and, where w goes through it, w
    const bool with_w = LAST && to.vec && to.w != nullptr && to.master == nullptr;
    const uint32_t bufs = with_w ? 3 : 2, slots = 2 * kSlots / bufs;
    auto slot = [&](int c) { return (w.st.turn + uint32_t(c)) % slots; };
    auto load = [&](int c) {
      const uint32_t s = slot(c), buf = w.st.base + s * (bufs * dg::kStageBytes), bar = w.st.bar + 8u * s;
      tc::mbar_arrive_expect_tx(bar, bufs * dg::kStageBytes);
      if (with_w) tc::tma_load_3d(buf + 2 * dg::kStageBytes, &next, bar, w.col + 32 * c, row0, caller(w.z));
      tc::tma_load_3d(buf, &hi, bar, w.col + 32 * c, row0, w.z);
      tc::tma_load_3d(buf + dg::kStageBytes, &lo, bar, w.col + 32 * c, row0, w.z);
    };
    // arrival of chunk c (a slot's n-th use is the phase of parity n % 2)
    auto arrived = [&](int c) {
      return tc::mbar_wait(w.st.bar + 8u * slot(c), ((w.st.turn + uint32_t(c)) / slots) & 1u, dg::kWaitLimitNs, &never);
    };
    __syncwarp();
    if (w.lane == 0) {
      tc::bulk_wait_read<0>();  // the last tile's stores have left the slots
      for (int c = 0; c < min(chunks, int(slots)); ++c) load(c);
    }
    if (!ready()) {  // (the loads in flight end before the CTA does)
      if (w.lane == 0)
        for (int c = 0; c < min(chunks, int(slots)); ++c)
          if (!arrived(c)) dev_flag(&g_dev_err, MOE_DEV_WAIT_TIMEOUT);
      return;
    }
#pragma unroll 1
    for (int c = 0; c < chunks; ++c) {
      const int col = w.col + 32 * c;
      const uint32_t sh = w.st.base + slot(c) * (bufs * dg::kStageBytes), sl = sh + dg::kStageBytes;
      const float rc = tall ? a + res[min(col + w.lane, cols - 1)] : 0.f;
      uint32_t r[32];
      tc::tmem_ld_32x32b_x32(w.tb + 32 * c, r);
      if (!arrived(c)) dev_flag(&g_dev_err, MOE_DEV_WAIT_TIMEOUT);
      tc::tmem_ld_wait();
      float x[32];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint4 vh = tc::ld_shared_v4(dg::stage_at(sh, w.lane, q)), vl = tc::ld_shared_v4(dg::stage_at(sl, w.lane, q));
        const uint32_t ph[4] = {vh.x, vh.y, vh.z, vh.w}, pl[4] = {vl.x, vl.y, vl.z, vl.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int j = 8 * q + 2 * i;
          const float2 h = unpack_half2(ph[i]), l = unpack_half2(pl[i]);
          const float a0 = tall ? __shfl_sync(0xffffffffu, rc, j) : ar;
          const float a1 = tall ? __shfl_sync(0xffffffffu, rc, j + 1) : ar;
          x[j] = fmaf(a0, fmaf(l.x, 1.f / kLo, h.x), __uint_as_float(r[j]) * (1.f / kScaleA));
          x[j + 1] = fmaf(a1, fmaf(l.y, 1.f / kLo, h.y), __uint_as_float(r[j + 1]) * (1.f / kScaleA));
        }
      }
      if (!LAST) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          uint32_t oh[4], ol[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int j = 8 * q + 2 * i;
            oh[i] = pack_half2(x[j], x[j + 1]);
            const float2 h = unpack_half2(oh[i]);
            ol[i] = pack_half2((x[j] - h.x) * kLo, (x[j + 1] - h.y) * kLo);
          }
          tc::st_shared_v4(dg::stage_at(sh, w.lane, q), make_uint4(oh[0], oh[1], oh[2], oh[3]));
          tc::st_shared_v4(dg::stage_at(sl, w.lane, q), make_uint4(ol[0], ol[1], ol[2], ol[3]));
        }
      } else {
        finish(w, col, x, sh);
      }
      tc::fence_proxy_async_smem();
      __syncwarp();
      if (w.lane == 0) {
        if (!LAST) {
          tc::tma_store_3d(&next, sh, col, row0, w.z);
          tc::tma_store_3d(&lo, sl, col, row0, w.z);
        } else if (to.vec) {
          tc::tma_store_3d(&next, with_w ? sh + 2 * dg::kStageBytes : sh, col, row0, caller(w.z));
        }
        tc::bulk_commit();
        // the chunk after this one's store in the same slot: loaded once the store has read it, a chunk later
        if (c >= 1 && c - 1 + int(slots) < chunks) {
          tc::bulk_wait_read<1>();
          load(c - 1 + int(slots));
        }
      }
    }
    w.st.turn += uint32_t(chunks);
  }

  __device__ __forceinline__ int caller(int z) const { return to.live != nullptr ? to.live[z] : to.first + z; }

  // The last step's result: to the caller's tensor, by way of the slot at `stage`.
  __device__ __forceinline__ void finish(const dg::Warp &w, int col, float (&x)[32], uint32_t stage) const {
#pragma unroll
    for (int i = 0; i < 32; ++i) x[i] *= to.inv;
    if (to.vec) {  // rows of 16-byte multiples
      // out, or w without master: in the slot's first or third buffer, which TMA stores (and filled with w); with master the
      // row's fp32 values come straight from memory, 128 bytes a lane
      const uint32_t buf = to.out != nullptr ? stage : stage + 2 * dg::kStageBytes;
      float *m = to.master;
      if (m != nullptr) m += (size_t(caller(w.z)) * rows + min(w.row, rows - 1)) * cols + col;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = x[8 * g + i];
        const uint32_t at = dg::stage_at(m != nullptr ? stage : buf, w.lane, g);
        if (m != nullptr) {
          if (col + 8 * g < cols && w.row < rows) {
            float4 *q = reinterpret_cast<float4 *>(m + 8 * g);
            const float4 u = q[0], v = q[1];
            const float o[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = fmaf(to.keep, o[i], -to.step * y[i]);
            q[0] = make_float4(y[0], y[1], y[2], y[3]);
            q[1] = make_float4(y[4], y[5], y[6], y[7]);
          }
        } else if (to.out == nullptr) {
          float o[8];
          unpack8(tc::ld_shared_v4(at), o);
#pragma unroll
          for (int i = 0; i < 8; ++i) y[i] = fmaf(to.keep, o[i], -to.step * y[i]);
        }
        tc::st_shared_v4(at, pack8(y));
      }
      return;
    }
    // Rows of odd length: a lane a column, so that a warp's accesses to memory lie together (a row a lane: ~5,400 cycles a chunk
    // in the place of ~1,300), through 32 x 32 fp32 values, column c of row r at c ^ r: no bank twice in either direction.
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 32; ++i) st_shared_f32(stage + uint32_t(w.lane * 32 + (i ^ w.lane)) * 4u, x[i]);
    __syncwarp();
    const size_t o0 = (size_t(caller(w.z)) * rows + (w.row - w.lane)) * cols + col + w.lane;
    const int here = min(32, rows - (w.row - w.lane));
    if (col + w.lane < cols) {
#pragma unroll 4
      for (int r = 0; r < here; ++r) {
        const size_t at = o0 + size_t(r) * cols;
        float y = ld_shared_f32(stage + uint32_t(r * 32 + (w.lane ^ r)) * 4u);
        if (to.out == nullptr) {
          const float v = to.master != nullptr ? to.master[at] : __uint_as_float(uint32_t(to.w[at]) << 16);
          y = fmaf(to.keep, v, -to.step * y);
          if (to.master != nullptr) to.master[at] = y;
        }
        (to.out != nullptr ? to.out : to.w)[at] = __bfloat16_as_ushort(__float2bfloat16_rn(y));
      }
    }
    __syncwarp();
  }
};

// ---------------------------------------------------------------- small kernels

// With a mask: live[0] = number of matrices that are updated, then their indices in ascending order.
__global__ void muon_live(const uint8_t *__restrict__ mask, int n_mats, int per, int *__restrict__ live) {
  pdl_start();
  const int lane = threadIdx.x;
  int n = 0;
  for (int i0 = 0; i0 < n_mats; i0 += 32) {
    const int i = i0 + lane;
    const bool on = i < n_mats && mask[i / per] != 0;
    const uint32_t b = __ballot_sync(0xffffffffu, on);
    if (on) live[1 + n + __popc(b & ((1u << lane) - 1u))] = i;
    n += __popc(b);
  }
  if (lane == 0) live[0] = n;
}

struct Source {
  const uint16_t *g;     // gradient [n_mats, rows, cols]
  float *m;              // momentum, or null: U = g
  float mu;
  int nesterov;
  int rows, cols, vec;
};

// U of the 8 columns from `col` of matrix row `row` (0 past the row's end). UPDATE: the momentum is new.
template <bool UPDATE>
__device__ __forceinline__ void load_u(const Source &s, size_t row, int col, float (&u)[8]) {
  const size_t o = row * s.cols + col;
  if (s.vec) {
    unpack8(*reinterpret_cast<const uint4 *>(s.g + o), u);
    if (s.m == nullptr) return;
    float4 *pm = reinterpret_cast<float4 *>(s.m + o);
    const float4 a = pm[0], b = pm[1];
    float m[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    if (UPDATE) {
#pragma unroll
      for (int i = 0; i < 8; ++i) m[i] = fmaf(s.mu, m[i], u[i]);
      pm[0] = make_float4(m[0], m[1], m[2], m[3]);
      pm[1] = make_float4(m[4], m[5], m[6], m[7]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = s.nesterov ? fmaf(s.mu, m[i], u[i]) : m[i];
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    u[i] = 0.f;
    if (col + i >= s.cols) continue;
    u[i] = __uint_as_float(uint32_t(s.g[o + i]) << 16);
    if (s.m == nullptr) continue;
    float m = s.m[o + i];
    if (UPDATE) {
      m = fmaf(s.mu, m, u[i]);
      s.m[o + i] = m;
    }
    u[i] = s.nesterov ? fmaf(s.mu, m, u[i]) : m;
  }
}

// Sums of squares of a matrix's U in three scales, so that any fp32 values have a norm: squares of values
// around 1, of small ones times 2^80, of large ones times 2^-80. Block (part, slot).
constexpr float kUp = 1.2089258196146292e24f, kDown = 8.271806125530277e-25f;  // 2^80, 2^-80
__global__ void __launch_bounds__(256) muon_norm(const Source s, const int *__restrict__ live, int first, int parts,
                                                 float *__restrict__ sums) {
  __shared__ float sh[3][8];
  pdl_start();
  const int slot = blockIdx.y;
  if (live != nullptr && first + slot >= live[0]) return;
  const size_t mrow = size_t(live != nullptr ? live[1 + first + slot] : first + slot) * s.rows;
  const int cpr = (s.cols + 7) / 8;
  const int64_t units = int64_t(s.rows) * cpr;
  float t[3] = {};
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < units; i += int64_t(parts) * 256) {
    const int64_t r = i / cpr;
    float u[8], q[3] = {};
    load_u<true>(s, mrow + r, int(i - r * cpr) * 8, u);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float up = u[j] * kUp, down = u[j] * kDown;
      q[0] = fmaf(u[j], u[j], q[0]);
      q[1] = fmaf(up, up, q[1]);
      q[2] = fmaf(down, down, q[2]);
    }
#pragma unroll
    for (int j = 0; j < 3; ++j) t[j] += q[j];
  }
#pragma unroll
  for (int j = 0; j < 3; ++j) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) t[j] += __shfl_down_sync(0xffffffffu, t[j], o);
    if ((threadIdx.x & 31) == 0) sh[j][threadIdx.x >> 5] = t[j];
  }
  __syncthreads();
  if (threadIdx.x < 3) {
    float v = 0.f;
    for (int i = 0; i < 8; ++i) v += sh[threadIdx.x][i];
    sums[(size_t(slot) * kParts + blockIdx.x) * 3 + threadIdx.x] = v;
  }
}

// hi and lo of U * scale / (|U|_F + eps).
__global__ void __launch_bounds__(256) muon_split(const Source s, const int *__restrict__ live, int first, int parts,
                                                  const float *__restrict__ sums, float scale, float eps, int pitch,
                                                  uint16_t *__restrict__ hi, uint16_t *__restrict__ lo) {
  __shared__ float sh[2];
  pdl_start();
  const int slot = blockIdx.y;
  if (live != nullptr && first + slot >= live[0]) return;
  if (threadIdx.x < 32) {
    float t[3] = {};
    for (int i = threadIdx.x; i < parts; i += 32)
#pragma unroll
      for (int j = 0; j < 3; ++j) t[j] += sums[(size_t(slot) * kParts + i) * 3 + j];
#pragma unroll
    for (int j = 0; j < 3; ++j)
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) t[j] += __shfl_down_sync(0xffffffffu, t[j], o);
    if (threadIdx.x == 0) {
      // the plain sum unless it lost squares below (then it is small) or above fp32's range; the norm itself may
      // lie above it, so U and eps are divided as they are scaled
      const int j = t[0] > 1e30f ? 2 : t[0] < 1e-18f ? 1 : 0;
      const float pre = j == 2 ? kDown : j == 1 ? kUp : 1.f;
      sh[0] = pre;
      sh[1] = sqrtf(j == 2 ? t[2] : j == 1 ? t[1] : t[0]) + eps * pre;
    }
  }
  __syncthreads();
  const float pre = sh[0], norm = sh[1];
  const size_t mrow = size_t(live != nullptr ? live[1 + first + slot] : first + slot) * s.rows;
  const int cpr = (s.cols + 7) / 8;
  const int64_t units = int64_t(s.rows) * cpr;
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < units; i += int64_t(gridDim.x) * 256) {
    const int64_t r = i / cpr;
    const int col = int(i - r * cpr) * 8;
    float u[8];
    load_u<false>(s, mrow + r, col, u);
    uint32_t h[4], l[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float x = u[2 * j] * pre / norm * scale, y = u[2 * j + 1] * pre / norm * scale;
      h[j] = pack_half2(x, y);
      const float2 b = unpack_half2(h[j]);
      l[j] = pack_half2((x - b.x) * kLo, (y - b.y) * kLo);
    }
    const size_t o = (size_t(slot) * s.rows + r) * pitch + col;
    stg_v4(hi + o, make_uint4(h[0], h[1], h[2], h[3]));
    stg_v4(lo + o, make_uint4(l[0], l[1], l[2], l[3]));
  }
}

// ---------------------------------------------------------------- host side

inline int64_t up256(int64_t x) { return (x + 255) & ~int64_t(255); }

struct Layout {
  int64_t live, sums, resid, hi0, hi1, lo, a, b, total;
  int pitch, npitch;
};
Layout layout(int n_mats, int rows, int cols, int64_t batch) {
  Layout l{};
  const int64_t n = std::min(rows, cols);
  l.pitch = (cols + 63) / 64 * 64;
  l.npitch = int((n + 63) / 64 * 64);
  int64_t off = 0;
  l.live = off;
  off += up256((int64_t(n_mats) + 1) * 4);
  l.sums = off;
  off += up256(batch * kParts * 3 * 4);
  l.resid = off;
  off += up256(batch * n * 4);
  const int64_t x = up256(batch * rows * l.pitch * 2), a = up256(batch * n * l.npitch * 2);
  l.hi0 = off; off += x;
  l.hi1 = off; off += x;
  l.lo = off; off += x;
  l.a = off; off += a;
  l.b = off; off += a;
  l.total = off;
  return l;
}

bool sizes_ok(int n_mats, int rows, int cols) {
  return n_mats >= 0 && n_mats <= (1 << 20) && rows >= 1 && cols >= 1 && rows <= 16384 && cols <= 16384;
}

int ceil_div(int64_t a, int64_t b) { return int((a + b - 1) / b); }

// Whether a product of so many 256 x 256 tiles at most runs in 256 x 128 tiles (dg::Small).
// MOE_DENSE_SMALL=0 or 1 forces either form (tests and A/B measurements).
bool small_tiles(long long tiles) {
  static const int forced = [] {
    const char *e = getenv("MOE_DENSE_SMALL");
    return e && (e[0] == '0' || e[0] == '1') && e[1] == 0 ? e[0] - '0' : -1;
  }();
  return forced >= 0 ? forced == 1 : tiles <= 76;
}

const float kCoef[3] = {3.4445f, -4.7750f, 2.0315f};

int run(const char *fn, const Source &src, const uint8_t *mask, int n_mats, int per, Target to, const float *coef, int steps,
        float eps, void *ws, size_t ws_bytes, cudaStream_t s) {
  const int rows = src.rows, cols = src.cols;
  if (!sizes_ok(n_mats, rows, cols))
    return moe::set_error(MOE_ERR_ARG, "%s: need 0 <= n_mats <= 2^20, 1 <= rows, cols <= 16384", fn);
  if (per < 1 || n_mats % per != 0)
    return moe::set_error(MOE_ERR_ARG, "%s: n_mats must be a multiple of mats_per_expert >= 1", fn);
  if (steps < 1 || steps > kMaxSteps) return moe::set_error(MOE_ERR_ARG, "%s: need 1 <= steps <= %d", fn, kMaxSteps);
  if (!(eps > 0.f) || !(eps < 1e30f)) return moe::set_error(MOE_ERR_ARG, "%s: eps must be positive and finite", fn);
  if (n_mats == 0) return MOE_OK;
  if (!src.g || (!to.out && !to.w)) return moe::set_error(MOE_ERR_ARG, "%s: null pointer", fn);
  const bool aligned = moe::aligned16(src.g) && moe::aligned16(src.m) && moe::aligned16(to.out) && moe::aligned16(to.w) &&
                       moe::aligned16(to.master);
  if (!aligned) return moe::set_error(MOE_ERR_ARG, "%s: tensors must be 16-byte aligned", fn);
  if (!ws || !moe::aligned16(ws) || ws_bytes < size_t(layout(n_mats, rows, cols, 1).total))
    return moe::set_error(MOE_ERR_WORKSPACE, "%s: workspace of %lld bytes at least, 16-byte aligned, needed", fn,
                          (long long)layout(n_mats, rows, cols, 1).total);
  // as many matrices at a time as the workspace holds
  int batch = 1;
  for (int hi = n_mats; batch < hi;) {
    const int mid = batch + (hi - batch + 1) / 2;
    if (size_t(layout(n_mats, rows, cols, mid).total) <= ws_bytes) batch = mid;
    else hi = mid - 1;
  }
  const Layout l = layout(n_mats, rows, cols, batch);
  uint8_t *base = static_cast<uint8_t *>(ws);
  int *live = reinterpret_cast<int *>(base + l.live);
  float *sums = reinterpret_cast<float *>(base + l.sums), *resid = reinterpret_cast<float *>(base + l.resid);
  uint16_t *x[2] = {reinterpret_cast<uint16_t *>(base + l.hi0), reinterpret_cast<uint16_t *>(base + l.hi1)};
  uint16_t *lo = reinterpret_cast<uint16_t *>(base + l.lo);
  uint16_t *ma = reinterpret_cast<uint16_t *>(base + l.a), *mb = reinterpret_cast<uint16_t *>(base + l.b);
  const bool tall = rows > cols;
  const int n = std::min(rows, cols), k = std::max(rows, cols);
  const float scale = exp2f(floorf(0.5f * log2f(float(k))));
  Source u = src;
  u.vec = cols % 8 == 0;
  to.vec = u.vec;
  to.inv = 1.f / scale;
  int st;
  const int64_t xstep = int64_t(rows) * l.pitch, astep = int64_t(n) * l.npitch;
  CUtensorMap xo[2], lom, ao, bo;
  for (int i = 0; i < 2; ++i)
    if ((st = dg::store_map(&xo[i], x[i], true, batch, rows, cols, l.pitch, xstep, fn))) return st;
  if ((st = dg::store_map(&lom, lo, true, batch, rows, cols, l.pitch, xstep, fn))) return st;
  if ((st = dg::store_map(&ao, ma, true, batch, n, n, l.npitch, astep, fn))) return st;
  if ((st = dg::store_map(&bo, mb, true, batch, n, n, l.npitch, astep, fn))) return st;
  CUtensorMap om = lom;
  if (to.vec && (st = dg::store_map(&om, to.out ? to.out : to.w, false, n_mats, rows, cols, cols, int64_t(rows) * cols, fn)))
    return st;
  const dg::Matrix A = {ma, batch, n, n, l.npitch, astep}, B = {mb, batch, n, n, l.npitch, astep};

  const int64_t units = int64_t(rows) * ((cols + 7) / 8);
  const int parts = int(std::max<int64_t>(1, std::min<int64_t>(kParts, units / 512)));
  const int blocks = int(std::max<int64_t>(1, std::min<int64_t>(1024, units / 512)));
  if (mask) {
    MOE_LAUNCH("muon_live", s, moe::launch_dep(muon_live, 1, 32, 0, s, mask, n_mats, per, live));
    if ((st = moe::launch_status(fn))) return st;
  } else {
    live = nullptr;
  }
  for (int first = 0; first < n_mats; first += batch) {
    const int mats = std::min(batch, n_mats - first);
    // (grid.y holds 65,535 matrices at most)
    for (int f = 0; f < mats; f += 65535) {
      const int m = std::min(65535, mats - f);
      MOE_LAUNCH("muon_norm", s, moe::launch_dep(muon_norm, dim3(parts, m), 256, 0, s, u, live, first + f, parts,
                                                 sums + size_t(f) * kParts * 3));
      if ((st = moe::launch_status(fn))) return st;
      MOE_LAUNCH("muon_split", s, moe::launch_dep(muon_split, dim3(blocks, m), 256, 0, s, u, live, first + f, parts,
                                                  sums + size_t(f) * kParts * 3, scale, eps, l.pitch, x[0] + f * xstep,
                                                  lo + f * xstep));
      if ((st = moe::launch_status(fn))) return st;
    }
    const int nt = ceil_div(n, 256);
    const bool small_sq = small_tiles((long long)mats * nt * (nt + 1) / 2), small_x = small_tiles((long long)mats * nt * ceil_div(k, 256));
    dg::Tiles t = {};
    t.mats = mats; t.live = live; t.first = first; t.splits = 1; t.group = 8;
    for (int i = 0; i < steps; ++i) {
      const float *cf = coef ? coef + 3 * i : kCoef;
      const dg::Matrix X = {x[i & 1], batch, rows, cols, l.pitch, xstep};
      t.sym = 1;
      GramEpi g;
      g.out = ao; g.scale = kScaleA / (scale * scale); g.n = n;
      if (tall) st = small_sq ? dg::product<dg::Small, true, true, true>("muon_gram", X, X, g, t, s, fn)
                              : dg::product<dg::Wide, true, true, true>("muon_gram", X, X, g, t, s, fn);
      else st = small_sq ? dg::product<dg::Small, false, false, true>("muon_gram", X, X, g, t, s, fn)
                         : dg::product<dg::Wide, false, false, true>("muon_gram", X, X, g, t, s, fn);
      if (st) return st;
      PolyEpi p;
      p.out = bo; p.a = ma; p.resid = resid; p.b = cf[1]; p.c = cf[2] / kScaleA; p.n = n; p.pitch = l.npitch;
      st = small_sq ? dg::product<dg::Small, false, false, true>("muon_poly", A, A, p, t, s, fn)
                    : dg::product<dg::Wide, false, false, true>("muon_poly", A, A, p, t, s, fn);
      if (st) return st;
      t.sym = 0;
      auto step = [&](auto e) -> int {
        e.hi = xo[i & 1]; e.lo = lom; e.next = i + 1 < steps ? xo[(i + 1) & 1] : om; e.resid = resid; e.a = cf[0];
        e.rows = rows; e.cols = cols; e.tall = tall; e.to = to;
        e.to.live = live ? live + 1 + first : nullptr; e.to.first = first;
        if (tall)
          return small_x ? dg::product<dg::SmallIO, false, false, true>("muon_step", X, B, e, t, s, fn)
                         : dg::product<dg::WideIO, false, false, true>("muon_step", X, B, e, t, s, fn);
        return small_x ? dg::product<dg::SmallIO, false, true, true>("muon_step", B, X, e, t, s, fn)
                       : dg::product<dg::WideIO, false, true, true>("muon_step", B, X, e, t, s, fn);
      };
      if ((st = i + 1 < steps ? step(StepEpi<false>()) : step(StepEpi<true>()))) return st;
    }
  }
  return MOE_OK;
}

}  // namespace

namespace moe {
MOE_DEV_ERR_DEFINE_READER(muon_dev_error)
}  // namespace moe

extern "C" {

size_t moe_orthogonalize_workspace_size(int n_mats, int rows, int cols, int batch) {
  if (!sizes_ok(n_mats, rows, cols) || batch < 1) return 0;
  return size_t(layout(n_mats, rows, cols, std::min(batch, std::max(n_mats, 1))).total);
}

int moe_orthogonalize(const uint16_t *g, const uint8_t *active_mask, int n_mats, int mats_per_expert, int rows, int cols,
                      const float *coef, int steps, float eps, uint16_t *out, void *ws, size_t ws_bytes,
                      moe_stream_t stream) {
  const Source src = {g, nullptr, 0.f, 0, rows, cols, 0};
  Target to = {};
  to.out = out;
  return run("moe_orthogonalize", src, active_mask, n_mats, mats_per_expert, to, coef, steps, eps, ws, ws_bytes,
             reinterpret_cast<cudaStream_t>(stream));
}

int moe_muon_step(uint16_t *w, float *master, const uint16_t *grad, float *momentum, const uint8_t *active_mask, int n_mats,
                  int mats_per_expert, int rows, int cols, float lr, float weight_decay, float mu, int nesterov, float scale,
                  const float *coef, int steps, float eps, void *ws, size_t ws_bytes, moe_stream_t stream) {
  if (n_mats > 0 && !momentum) return moe::set_error(MOE_ERR_ARG, "moe_muon_step: null momentum");
  const Source src = {grad, momentum, mu, nesterov != 0, rows, cols, 0};
  Target to = {};
  to.w = w;
  to.master = master;
  to.keep = 1.f - lr * weight_decay;
  to.step = lr * scale;
  return run("moe_muon_step", src, active_mask, n_mats, mats_per_expert, to, coef, steps, eps, ws, ws_bytes,
             reinterpret_cast<cudaStream_t>(stream));
}

}  // extern "C"
