// Activation checkpoints in 8 bits (see ckpt.cuh for the format): rows packed and unpacked, unpacked
// into the grouped layout, and the kept pre-activations [A|B] unpacked for the entry points that read
// them in bf16. All of it is bound by HBM: a warp takes a row (or a share of it), every lane 8 consecutive
// columns of it per step, 16 bytes of bf16 or 8 of codes.
#include "ckpt.cuh"

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kAhead = 4;  // steps whose loads are in flight together

// Row and column segment of a warp: nseg warps share a row.
__device__ __forceinline__ bool row_segment(int64_t block, int64_t rows, int nseg, int64_t *r, int *seg) {
  const int64_t w = block * kWarps + int(threadIdx.x >> 5);
  *r = w / nseg;
  *seg = int(w - *r * nseg);
  return *r < rows;
}

// x [rows, cols] -> codes [rows, cols], scales [rows, nblk]. Four lanes hold a block of 32 columns
// (a row's last block may be shorter: its missing values count as zero).
__global__ void __launch_bounds__(kThreads) pack_kernel(const uint16_t *__restrict__ x, int64_t rows, int cols,
                                                        int nseg, uint8_t *__restrict__ q,
                                                        uint8_t *__restrict__ scale) {
  pdl_start();
  const int lane = threadIdx.x & 31;
  int64_t r;
  int seg;
  if (!row_segment(blockIdx.x, rows, nseg, &r, &seg)) return;
  const int nv = cols / 8, step = 32 * nseg, nblk = (cols + ckpt::kBlock - 1) / ckpt::kBlock;
  const uint16_t *src = x + size_t(r) * cols;
  // (whole warps stay in the loop: the largest values are exchanged)
  for (int c0 = 32 * seg; c0 < nv; c0 += kAhead * step) {
    uint4 v[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int c = c0 + u * step + lane;
      v[u] = c < nv ? ldg_nc_v4(src + c * 8) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int c = c0 + u * step + lane;
      float f[8];
      unpack8(v[u], f);
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(f[i]) & 0x7fffffffu);
      m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
      m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
      const uint32_t s = ckpt::scale_byte(m);
      uint2 o = make_uint2(ckpt::kNanCodes, ckpt::kNanCodes);
      if (s != 255u) {
        const float inv = ckpt::scale_inverse(s);
        o.x = ckpt::codes4(f[0], f[1], f[2], f[3], inv);
        o.y = ckpt::codes4(f[4], f[5], f[6], f[7], inv);
      }
      if (c < nv) {
        *reinterpret_cast<uint2 *>(q + size_t(r) * cols + c * 8) = o;
        if ((lane & 3) == 0) scale[size_t(r) * nblk + c / 4] = uint8_t(s);
      }
    }
  }
}

// Rows of codes -> bf16 rows x_out[r] (null: not stored) and the K grouped rows of the row's
// assignments (K = 0: none). Blocks below pad_blocks zero the groups' padding rows.
// The next kernel may start when blocks end, not when they start: its waiting blocks then take the
// SMs' room unevenly, and the few heavy blocks of this one (a row and its copies per warp) land on
// few SMs: with a pack before it 26.9 us a pass against 16.5 at 1,021 rows of 2,048, top-6 (12.5 with four
// warps per row besides).
template <bool GROUPED>
__global__ void __launch_bounds__(kThreads) unpack_kernel(
    const uint8_t *__restrict__ q, const uint8_t *__restrict__ scale, int64_t rows, int cols, int nseg,
    const int32_t *__restrict__ row_of_assignment, int k, int64_t rows_cap, int pad_blocks,
    const int32_t *__restrict__ group_offsets, const int32_t *__restrict__ group_counts,
    uint16_t *__restrict__ x_out, uint16_t *__restrict__ x_perm) {
  pdl_wait();
  const int lane = threadIdx.x & 31;
  if (GROUPED && int(blockIdx.x) < pad_blocks) {
    moe::zero_pad_rows<kWarps>(blockIdx.x, group_offsets, group_counts, cols, rows_cap, x_perm);
    return;
  }
  int64_t r;
  int seg;
  if (!row_segment(int64_t(blockIdx.x) - pad_blocks, rows, nseg, &r, &seg)) return;
  int at[8];
  if (GROUPED) {
    const int mine = lane < k ? row_of_assignment[size_t(r) * k + lane] : -1;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      at[j] = __shfl_sync(0xffffffffu, mine, j);
      if (at[j] >= rows_cap) at[j] = -1;
    }
  }
  const int nv = cols / 8, step = 32 * nseg, nblk = (cols + ckpt::kBlock - 1) / ckpt::kBlock;
  for (int c0 = 32 * seg + lane; c0 < nv; c0 += kAhead * step) {
    uint2 v[kAhead];
    uint32_t s[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int c = c0 + u * step;
      if (c < nv) {
        v[u] = __ldg(reinterpret_cast<const uint2 *>(q + size_t(r) * cols + c * 8));
        s[u] = __ldg(scale + size_t(r) * nblk + c / 4);
      }
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int c = c0 + u * step;
      if (c >= nv) break;
      float f[8];
      const float sc = ckpt::scale_value(s[u]);
      ckpt::values4(v[u].x, sc, f);
      ckpt::values4(v[u].y, sc, f + 4);
      const uint4 o = pack8(f);
      if (x_out != nullptr) stg_v4(x_out + size_t(r) * cols + c * 8, o);
      if (GROUPED) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (j < k && at[j] >= 0) stg_v4(x_perm + size_t(at[j]) * cols + c * 8, o);
      }
    }
  }
}

// Kept [A|B] -> bf16 in the layout of moe_grouped_ffn_fwd's ab_saved, and H = silu(A) * B. A warp takes
// 32 columns of A and the same of B of a 32-row tile, a lane a row, as the GEMM epilogue that kept them. H's rows
// go through shared memory, so that a store instruction writes 8 whole 64-byte row pieces and
// not 32 quarters of one.
__global__ void __launch_bounds__(kThreads) unpack_ab_kernel(const uint8_t *__restrict__ q,
                                                             const uint8_t *__restrict__ scale,
                                                             const int32_t *__restrict__ group_offsets, int E, int F,
                                                             int64_t rows_cap, uint16_t *__restrict__ ab,
                                                             uint16_t *__restrict__ h) {
  __shared__ uint4 s_h[kWarps][32][4];  // 16-byte piece c of row r at (c + r / 2) % 4: no bank conflicts
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, per = F / 32;
  const int64_t w = int64_t(blockIdx.x) * kWarps + warp;
  const int64_t tile = w / per;
  if (tile >= min(int64_t(group_offsets[E]), rows_cap) / 32) return;
  const int c = int(w - tile * per) * 32;
  const size_t row = size_t(tile) * 32 + lane;
  const uint8_t *qa = q + ckpt::ab_code_index(row, c, F), *qb = q + ckpt::ab_code_index(row, F + c, F);
  const uint4 va[2] = {ldg_nc_v4(qa), ldg_nc_v4(qa + 512)}, vb[2] = {ldg_nc_v4(qb), ldg_nc_v4(qb + 512)};
  const float sa = ckpt::scale_value(__ldg(scale + ckpt::ab_scale_index(row, c, F)));
  const float sb = ckpt::scale_value(__ldg(scale + ckpt::ab_scale_index(row, F + c, F)));
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    float fa[8], fb[8], fh[8];
    ckpt::values4(v % 2 ? va[v / 2].z : va[v / 2].x, sa, fa);
    ckpt::values4(v % 2 ? va[v / 2].w : va[v / 2].y, sa, fa + 4);
    ckpt::values4(v % 2 ? vb[v / 2].z : vb[v / 2].x, sb, fb);
    ckpt::values4(v % 2 ? vb[v / 2].w : vb[v / 2].y, sb, fb + 4);
#pragma unroll
    for (int i = 0; i < 8; ++i) fh[i] = silu_f(fa[i]) * fb[i];
    if (ab != nullptr) {
      stg_v4(ab + ab_block_index(row, c + 8 * v, F), pack8(fa));
      stg_v4(ab + ab_block_index(row, F + c + 8 * v, F), pack8(fb));
    }
    s_h[warp][lane][(v + (lane >> 1)) & 3] = pack8(fh);
  }
  if (h == nullptr) return;
  __syncwarp();
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int r = 8 * u + (lane >> 2), v = lane & 3;
    stg_v4(h + (size_t(tile) * 32 + r) * F + c + 8 * v, s_h[warp][r][(v + (r >> 1)) & 3]);
  }
}

// Warps per row: one from 32 warps per SM on, and with fewer rows as many as give that (1,021 rows of
// 2,048: 16.5 us with 8 warps per SM, 12.7 with 16, 12.5 with 32; 32,768 rows of 4,096 the same).
int row_segments(int64_t rows, int cols) {
  const int64_t warps = int64_t(moe::num_sms()) * 32, most = (cols / 8 + 31) / 32;
  return int(std::max<int64_t>(1, std::min(most, warps / std::max<int64_t>(rows, 1))));
}
int64_t row_grid(int64_t rows, int nseg) { return (rows * nseg + kWarps - 1) / kWarps; }

bool aligned8(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 7u) == 0; }

int check_rows(const char *fn, int64_t rows, int cols) {
  if (rows < 0 || rows >= (int64_t(1) << 31) || cols <= 0 || cols % 8)
    return moe::set_error(MOE_ERR_ARG, "%s: rows=%lld cols=%d", fn, (long long)rows, cols);
  return MOE_OK;
}

}  // namespace

extern "C" {

int moe_ckpt_pack(const uint16_t *x, int64_t rows, int cols, uint8_t *q, uint8_t *scale, moe_stream_t stream) {
  const char *fn = "moe_ckpt_pack";
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (int st = check_rows(fn, rows, cols)) return st;
  if (rows == 0) return MOE_OK;
  if (!x || !q || !scale) return moe::set_error(MOE_ERR_ARG, "%s: null pointer", fn);
  if (!moe::aligned16(x) || !aligned8(q)) return moe::set_error(MOE_ERR_ARG, "%s: alignment", fn);
  const int nseg = row_segments(rows, cols);
  MOE_LAUNCH("ckpt_pack", s, moe::launch_dep(pack_kernel, dim3(unsigned(row_grid(rows, nseg))), kThreads, 0, s, x, rows,
                                             cols, nseg, q, scale));
  return moe::launch_status("moe_ckpt_pack: launch");
}

int moe_ckpt_unpack(const uint8_t *q, const uint8_t *scale, int64_t rows, int cols, uint16_t *x, moe_stream_t stream) {
  const char *fn = "moe_ckpt_unpack";
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (int st = check_rows(fn, rows, cols)) return st;
  if (rows == 0) return MOE_OK;
  if (!x || !q || !scale) return moe::set_error(MOE_ERR_ARG, "%s: null pointer", fn);
  if (!moe::aligned16(x) || !aligned8(q)) return moe::set_error(MOE_ERR_ARG, "%s: alignment", fn);
  const int nseg = row_segments(rows, cols);
  MOE_LAUNCH("ckpt_unpack", s, moe::launch_dep(unpack_kernel<false>, dim3(unsigned(row_grid(rows, nseg))), kThreads, 0, s,
                                               q, scale, rows, cols, nseg, nullptr, 0, int64_t(0), 0, nullptr, nullptr, x,
                                               nullptr));
  return moe::launch_status("moe_ckpt_unpack: launch");
}

int moe_ckpt_permute(const uint8_t *q, const uint8_t *scale, const int32_t *row_of_assignment,
                     const int32_t *group_offsets, const int32_t *group_counts, int T, int d, int E, int k,
                     int64_t rows_cap, uint16_t *x, uint16_t *x_perm, moe_stream_t stream) {
  const char *fn = "moe_ckpt_permute";
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (E < 1 || E > 256 || k < 1 || k > 8 || T < 0 || d <= 0 || d % 8)
    return moe::set_error(MOE_ERR_ARG, "%s: sizes T=%d d=%d E=%d k=%d", fn, T, d, E, k);
  if (rows_cap < moe_perm_rows_max(T, k, E))
    return moe::set_error(MOE_ERR_ARG, "%s: rows_cap %lld < %lld", fn, (long long)rows_cap,
                          (long long)moe_perm_rows_max(T, k, E));
  if (rows_cap >= (int64_t(1) << 31)) return moe::set_error(MOE_ERR_UNSUPPORTED, "%s: rows_cap >= 2^31", fn);
  if (T == 0) return MOE_OK;  // no group has a row
  if (!q || !scale || !row_of_assignment || !group_offsets || !group_counts || !x_perm)
    return moe::set_error(MOE_ERR_ARG, "%s: null pointer", fn);
  if (!aligned8(q) || (x && !moe::aligned16(x)) || !moe::aligned16(x_perm))
    return moe::set_error(MOE_ERR_ARG, "%s: alignment", fn);
  const int nseg = row_segments(T, d), pad = E * moe::kPadSplit;
  MOE_LAUNCH("ckpt_permute", s, moe::launch_dep(unpack_kernel<true>, dim3(unsigned(pad + row_grid(T, nseg))), kThreads, 0,
                                                s, q, scale, int64_t(T), d, nseg, row_of_assignment, k, rows_cap, pad,
                                                group_offsets, group_counts, x, x_perm));
  return moe::launch_status("moe_ckpt_permute: launch");
}

int moe_ckpt_unpack_ab(const uint8_t *ab_q, const uint8_t *ab_scale, const int32_t *group_offsets, int E,
                       int F, int64_t rows_cap, uint16_t *ab_saved, uint16_t *h, moe_stream_t stream) {
  const char *fn = "moe_ckpt_unpack_ab";
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (E < 1 || E > 256 || F <= 0 || F % 128 || rows_cap < 128 || rows_cap >= (int64_t(1) << 31))
    return moe::set_error(MOE_ERR_ARG, "%s: sizes E=%d F=%d rows_cap=%lld", fn, E, F, (long long)rows_cap);
  if (!ab_q || !ab_scale || !group_offsets || (!ab_saved && !h))
    return moe::set_error(MOE_ERR_ARG, "%s: null pointer", fn);
  for (const void *p : {static_cast<const void *>(ab_q), static_cast<const void *>(ab_scale),
                        static_cast<const void *>(ab_saved), static_cast<const void *>(h)})
    if (p && !moe::aligned16(p)) return moe::set_error(MOE_ERR_ARG, "%s: alignment", fn);
  const int64_t warps = rows_cap / 32 * (F / 32);
  if (warps / kWarps >= (int64_t(1) << 31) - 1)
    return moe::set_error(MOE_ERR_UNSUPPORTED, "%s: rows_cap=%lld F=%d", fn, (long long)rows_cap, F);
  MOE_LAUNCH("ckpt_unpack_ab", s, moe::launch_dep(unpack_ab_kernel, dim3(unsigned((warps + kWarps - 1) / kWarps)), kThreads, 0,
                                                  s, ab_q, ab_scale, group_offsets, E, F, rows_cap, ab_saved, h));
  return moe::launch_status("moe_ckpt_unpack_ab: launch");
}

}  // extern "C"
