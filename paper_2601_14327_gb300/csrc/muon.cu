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

// ---------------------------------------------------------------- epilogues of the products

// A = acc * scale, both halves of the symmetric matrix.
struct GramEpi {
  CUtensorMap out;
  float scale;
  int n;

  template <int BN> __device__ __forceinline__ void run(const dg::Warp &w) const {
    const int row0 = w.row - w.lane;
    if (row0 >= n) return;
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
      dg::stage_and_store(&out, w.stage, w.lane, v, col, row0, w.z);
      if (mirror) dg::stage_and_store_t(&out, w.stage, w.lane, v, col, row0, w.z);
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

  template <int BN> __device__ __forceinline__ void run(const dg::Warp &w) const {
    const int row0 = w.row - w.lane;
    if (row0 >= n) return;
    const bool mirror = row0 / dg::kTileRows != w.col / dg::kTileRows;
    const uint16_t *arow = a + (size_t(w.z) * n + min(w.row, n - 1)) * pitch;
#pragma unroll 1
    for (int cc = 0; cc < BN / 2; cc += 32) {
      const int col = w.col + cc;
      if (col >= n) break;
      uint4 x[4];  // (pitch is a multiple of 64: 32 columns never leave the row)
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const uint4 *>(arow + col + 8 * i);
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
      dg::stage_and_store(&out, w.stage, w.lane, v, col, row0, w.z);
      if (mirror) dg::stage_and_store_t(&out, w.stage, w.lane, v, col, row0, w.z);
    }
  }
};

// X <- (a + resid) X + acc: to the next hi and lo, or with LAST to the caller's tensors.
struct Target {
  const int *live;            // the stack's matrices among the caller's
  int vec;                    // rows of 16-byte multiples, 16-byte aligned tensors
  float inv;                  // 1 / X's scale
  uint16_t *out;              // orthogonalised [n_mats, rows, cols], or null: weights
  uint16_t *w;
  float *master;              // may be null
  float keep, step;           // w <- keep w - step O
};

template <bool LAST> struct StepEpi {
  CUtensorMap hi_out, lo_out;
  const uint16_t *hi, *lo;    // [mats, rows, pitch]
  const float *resid;         // [mats, rows or cols]
  float a;
  int rows, cols, pitch, tall;
  Target to;

  template <int BN> __device__ __forceinline__ void run(const dg::Warp &w) const {
    const int row0 = w.row - w.lane;
    if (row0 >= rows) return;
    const size_t at = (size_t(w.z) * rows + min(w.row, rows - 1)) * pitch;
    const float *res = resid + size_t(w.z) * (tall ? cols : rows);
    const float ar = tall ? a : a + res[min(w.row, rows - 1)];
#pragma unroll 1
    for (int c = 0; c < BN / 2; c += 32) {
      const int col = w.col + c;
      if (col >= cols) break;
      uint4 xh[4], xl[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        xh[i] = *reinterpret_cast<const uint4 *>(hi + at + col + 8 * i);
        xl[i] = *reinterpret_cast<const uint4 *>(lo + at + col + 8 * i);
      }
      const float rc = tall ? a + res[min(col + w.lane, cols - 1)] : 0.f;
      uint32_t r[32];
      tc::tmem_ld_32x32b_x32(w.tb + c, r);
      tc::tmem_ld_wait();
      const uint32_t *ph = reinterpret_cast<const uint32_t *>(xh), *pl = reinterpret_cast<const uint32_t *>(xl);
      float x[32];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float2 h = unpack_half2(ph[i]), l = unpack_half2(pl[i]);
        const float a0 = tall ? __shfl_sync(0xffffffffu, rc, 2 * i) : ar;
        const float a1 = tall ? __shfl_sync(0xffffffffu, rc, 2 * i + 1) : ar;
        x[2 * i] = fmaf(a0, fmaf(l.x, 1.f / kLo, h.x), __uint_as_float(r[2 * i]) * (1.f / kScaleA));
        x[2 * i + 1] = fmaf(a1, fmaf(l.y, 1.f / kLo, h.y), __uint_as_float(r[2 * i + 1]) * (1.f / kScaleA));
      }
      if (!LAST) {
        uint4 vh[4], vl[4];
        uint32_t *oh = reinterpret_cast<uint32_t *>(vh), *ol = reinterpret_cast<uint32_t *>(vl);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          oh[i] = pack_half2(x[2 * i], x[2 * i + 1]);
          const float2 h = unpack_half2(oh[i]);
          ol[i] = pack_half2((x[2 * i] - h.x) * kLo, (x[2 * i + 1] - h.y) * kLo);
        }
        dg::stage_and_store(&hi_out, w.stage, w.lane, vh, col, row0, w.z);
        dg::stage_and_store(&lo_out, w.stage, w.lane, vl, col, row0, w.z);
      } else if (w.row < rows) {
        finish(w, col, x);
      }
    }
  }

  __device__ __forceinline__ void finish(const dg::Warp &w, int col, float (&x)[32]) const {
    const size_t o = (size_t(to.live[w.z]) * rows + w.row) * cols + col;
#pragma unroll
    for (int i = 0; i < 32; ++i) x[i] *= to.inv;
    if (to.vec) {
#pragma unroll
      for (int g = 0; g < 32; g += 8) {
        if (col + g >= cols) break;
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = x[g + i];
        if (to.out != nullptr) {
          stg_v4(to.out + o + g, pack8(y));
          continue;
        }
        float v[8];
        if (to.master != nullptr) {
          const float4 p = *reinterpret_cast<const float4 *>(to.master + o + g), q = *reinterpret_cast<const float4 *>(to.master + o + g + 4);
          v[0] = p.x; v[1] = p.y; v[2] = p.z; v[3] = p.w;
          v[4] = q.x; v[5] = q.y; v[6] = q.z; v[7] = q.w;
        } else {
          unpack8(*reinterpret_cast<const uint4 *>(to.w + o + g), v);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = fmaf(to.keep, v[i], -to.step * y[i]);
        if (to.master != nullptr) {
          *reinterpret_cast<float4 *>(to.master + o + g) = make_float4(v[0], v[1], v[2], v[3]);
          *reinterpret_cast<float4 *>(to.master + o + g + 4) = make_float4(v[4], v[5], v[6], v[7]);
        }
        stg_v4(to.w + o + g, pack8(v));
      }
      return;
    }
#pragma unroll 1
    for (int i = 0; i < 32; ++i) {
      if (col + i >= cols) break;
      float y = 0.f;
#pragma unroll
      for (int j = 0; j < 32; ++j) y = j == i ? x[j] : y;
      if (to.out == nullptr) {
        const float v = to.master != nullptr ? to.master[o + i] : __uint_as_float(uint32_t(to.w[o + i]) << 16);
        y = fmaf(to.keep, v, -to.step * y);
        if (to.master != nullptr) to.master[o + i] = y;
      }
      const uint16_t b = __bfloat16_as_ushort(__float2bfloat16_rn(y));
      (to.out != nullptr ? to.out : to.w)[o + i] = b;
    }
  }
};

// ---------------------------------------------------------------- small kernels

// live[0] = number of matrices that are updated, then their indices in ascending order.
__global__ void muon_live(const uint8_t *__restrict__ mask, int n_mats, int per, int *__restrict__ live) {
  pdl_start();
  const int lane = threadIdx.x;
  int n = 0;
  for (int i0 = 0; i0 < n_mats; i0 += 32) {
    const int i = i0 + lane;
    const bool on = i < n_mats && (mask == nullptr || mask[i / per] != 0);
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
  if (first + slot >= live[0]) return;
  const size_t mrow = size_t(live[1 + first + slot]) * s.rows;
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
  if (first + slot >= live[0]) return;
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
  const size_t mrow = size_t(live[1 + first + slot]) * s.rows;
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
  // tensor maps: X as an operand of both products, for its new values; A, B as operands and results
  CUtensorMap gx[2], px[2], xo[2], lom, am, ao, bm, bo;
  const int64_t xstep = int64_t(rows) * l.pitch, astep = int64_t(n) * l.npitch;
  for (int i = 0; i < 2; ++i) {
    if ((st = dg::operand_map(&gx[i], x[i], true, tall, batch, rows, cols, l.pitch, xstep, 128, fn))) return st;
    if ((st = dg::operand_map(&px[i], x[i], true, !tall, batch, rows, cols, l.pitch, xstep, 128, fn))) return st;
    if ((st = dg::store_map(&xo[i], x[i], true, batch, rows, cols, l.pitch, xstep, fn))) return st;
  }
  if ((st = dg::store_map(&lom, lo, true, batch, rows, cols, l.pitch, xstep, fn))) return st;
  if ((st = dg::operand_map(&am, ma, true, false, batch, n, n, l.npitch, astep, 128, fn))) return st;
  if ((st = dg::store_map(&ao, ma, true, batch, n, n, l.npitch, astep, fn))) return st;
  if ((st = dg::operand_map(&bm, mb, true, false, batch, n, n, l.npitch, astep, 128, fn))) return st;
  if ((st = dg::store_map(&bo, mb, true, batch, n, n, l.npitch, astep, fn))) return st;

  const int64_t units = int64_t(rows) * ((cols + 7) / 8);
  const int parts = int(std::max<int64_t>(1, std::min<int64_t>(kParts, units / 512)));
  const int blocks = int(std::max<int64_t>(1, std::min<int64_t>(1024, units / 512)));
  MOE_LAUNCH("muon_live", s, moe::launch_dep(muon_live, 1, 32, 0, s, mask, n_mats, per, live));
  if ((st = moe::launch_status(fn))) return st;
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
    for (int i = 0; i < steps; ++i) {
      const float *cf = coef ? coef + 3 * i : kCoef;
      const int nt = ceil_div(n, 256);
      {
        GramEpi e;
        e.out = ao; e.scale = kScaleA / (scale * scale); e.n = n;
        const dg::Tiles t = {mats, live, first, nt, nt, ceil_div(k, dg::KB), 1, 1, 8};
        const long long most = (long long)mats * nt * (nt + 1) / 2;
        st = tall ? dg::launch<256, true, true, true>("muon_gram", gx[i & 1], gx[i & 1], e, t, most, s, fn)
                  : dg::launch<256, false, false, true>("muon_gram", gx[i & 1], gx[i & 1], e, t, most, s, fn);
        if (st) return st;
      }
      {
        PolyEpi e;
        e.out = bo; e.a = ma; e.resid = resid; e.b = cf[1]; e.c = cf[2] / kScaleA; e.n = n; e.pitch = l.npitch;
        const dg::Tiles t = {mats, live, first, nt, nt, ceil_div(n, dg::KB), 1, 1, 8};
        if ((st = dg::launch<256, false, false, true>("muon_poly", am, am, e, t, (long long)mats * nt * (nt + 1) / 2, s, fn)))
          return st;
      }
      const dg::Tiles t = {mats, live, first, ceil_div(rows, 256), ceil_div(cols, 256), ceil_div(n, dg::KB), 1, 0, 8};
      const long long most = (long long)mats * t.mt * t.nt;
      auto step = [&](auto e) -> int {
        e.hi_out = xo[(i + 1) & 1]; e.lo_out = lom; e.hi = x[i & 1]; e.lo = lo; e.resid = resid; e.a = cf[0];
        e.rows = rows; e.cols = cols; e.pitch = l.pitch; e.tall = tall; e.to = to;
        e.to.live = live + 1 + first;
        return tall ? dg::launch<256, false, false, true>("muon_step", px[i & 1], bm, e, t, most, s, fn)
                    : dg::launch<256, false, true, true>("muon_step", bm, px[i & 1], e, t, most, s, fn);
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
