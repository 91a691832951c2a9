// Values in 8 bits (e4m3) with a scale for each block of 128 columns of a row, or of 128 x 128 entries of a table.
//
// The scale is the smallest power of two s with amax <= 448 s (448: the largest e4m3 value), so x / s is exact and the only rounding is
// that to e4m3 (nearest, even); a scale amax / 448 would round twice and give ties to chance.  One read and one write: bound by memory
// (a table of 151,936 x 2,048 bf16: 143 us in short runs, 149 to 158 in long ones, 5.9 to 6.5 TB/s).
// A block with NaN or an infinity has the scale NaN and values NaN.
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "e3.h"

namespace e3 {
namespace {

constexpr int kBlock = 128;

struct QuantParams {
  const void *x;
  uint8_t *q;
  float *scale;
  int64_t rows, cols, x_stride, q_stride, scale_stride;
  int64_t row_blocks, col_blocks;
};

// Eight entries of a row from column c on, as they lie in memory; 0 from `left` on.
template <int DT>
struct Raw {
  uint4 v[DT == 0 ? 2 : 1];
};
template <int DT, bool VEC>
__device__ __forceinline__ Raw<DT> load8(const char *row, int64_t c, int64_t left) {
  Raw<DT> r;
  if (VEC && left >= 8) {
#pragma unroll
    for (int k = 0; k < (DT == 0 ? 2 : 1); ++k) r.v[k] = __ldcs(reinterpret_cast<const uint4 *>(row + c * (DT == 0 ? 4 : 2)) + k);
    return r;
  }
  uint32_t w[8];
  if (DT == 1) {
    const uint16_t *const p = reinterpret_cast<const uint16_t *>(row) + c;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (2 * i < left ? p[2 * i] : 0u) | (2 * i + 1 < left ? (uint32_t)p[2 * i + 1] << 16 : 0u);
  } else {
    const uint32_t *const p = reinterpret_cast<const uint32_t *>(row) + c;
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = i < left ? p[i] : 0u;
  }
#pragma unroll
  for (int k = 0; k < (DT == 0 ? 2 : 1); ++k) r.v[k] = make_uint4(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]);
  return r;
}
template <int DT>
__device__ __forceinline__ float entry(const Raw<DT> &r, int i) {
  const uint4 &v = r.v[DT == 0 ? i >> 2 : 0];
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  if (DT == 0) return __uint_as_float(w[i & 3]);
  return __uint_as_float((i & 1) != 0 ? w[i >> 1] & 0xFFFF0000u : w[i >> 1] << 16);
}
// Largest |x|, as a pattern of fp32: they order like the values, NaN above infinity.
template <int DT>
__device__ __forceinline__ uint32_t most8(const Raw<DT> &r) {
  if (DT == 0) {
    uint32_t m = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(entry(r, i)) & 0x7FFFFFFFu);
    return m;
  }
  const uint32_t m = __vmaxu2(__vmaxu2(r.v[0].x & 0x7FFF7FFFu, r.v[0].y & 0x7FFF7FFFu), __vmaxu2(r.v[0].z & 0x7FFF7FFFu, r.v[0].w & 0x7FFF7FFFu));
  return max(m & 0xFFFF0000u, m << 16);
}
// Scale of a block, and its inverse, from the pattern of its largest |x|.
__device__ __forceinline__ float scale_of(uint32_t most, float &inverse) {
  if (most >= 0x7F800000u) {
    inverse = __uint_as_float(0x7FC00000u);
    return inverse;
  }
  if (most == 0u) {
    inverse = 1.f;
    return 1.f;
  }
  // 448 = 1.75 x 2^8; no scale below the smallest normal number
  int e = (int)(most >> 23) - 8 + ((most & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  if (e < 1) e = 1;
  inverse = __uint_as_float((uint32_t)(254 - e) << 23);
  return __uint_as_float((uint32_t)e << 23);
}
template <int DT>
__device__ __forceinline__ uint32_t four(const Raw<DT> &r, int i, float inverse) {
  const float2 lo = make_float2(entry(r, i) * inverse, entry(r, i + 1) * inverse), hi = make_float2(entry(r, i + 2) * inverse, entry(r, i + 3) * inverse);
  const uint32_t a = __nv_cvt_float2_to_fp8x2(lo, __NV_SATFINITE, __NV_E4M3), b = __nv_cvt_float2_to_fp8x2(hi, __NV_SATFINITE, __NV_E4M3);
  return a | b << 16;
}
template <int DT, bool VEC>
__device__ __forceinline__ void store8(uint8_t *q, int64_t left, const Raw<DT> &r, float inverse) {
  const uint2 w = make_uint2(four(r, 0, inverse), four(r, 4, inverse));
  if (VEC && left >= 8) {
    *reinterpret_cast<uint2 *>(q) = w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < left) q[i] = (uint8_t)((i < 4 ? w.x >> (8 * i) : w.y >> (8 * (i - 4))));
  }
}

__device__ __forceinline__ void wait_for_stream_predecessor() {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
}

// Rows: 16 lanes take a block, a warp two.
constexpr int kRowWarps = 8;
template <int DT, bool VEC>
__global__ void __launch_bounds__(kRowWarps * 32) quantize_rows_kernel(const __grid_constant__ QuantParams p) {
  wait_for_stream_predecessor();
  const int half = threadIdx.x >> 4, lane = threadIdx.x & 15;
  const int64_t item = (int64_t)blockIdx.x * (kRowWarps * 2) + half;
  const int64_t row = item / p.col_blocks, cb = item - row * p.col_blocks;
  const bool live = row < p.rows;
  const int64_t c = cb * kBlock + lane * 8, left = live ? p.cols - c : 0;
  const Raw<DT> v = load8<DT, VEC>(static_cast<const char *>(p.x) + (live ? row : 0) * p.x_stride * (DT == 0 ? 4 : 2), c, left);
  uint32_t most = most8(v);
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
  if (!live) return;
  float inverse;
  const float scale = scale_of(most, inverse);
  if (lane == 0) p.scale[row * p.scale_stride + cb] = scale;
  store8<DT, VEC>(p.q + row * p.q_stride + c, left, v, inverse);
}

// Tables: a CTA takes a block of 128 x 128, 16 lanes a row of it, eight rows each.
constexpr int kTableThreads = 256;
constexpr int kEach = kBlock * 16 / kTableThreads;
template <int DT, bool VEC>
__global__ void __launch_bounds__(kTableThreads, DT == 0 ? 2 : 4) quantize_table_kernel(const __grid_constant__ QuantParams p) {
  __shared__ uint32_t sh[kTableThreads / 32];
  wait_for_stream_predecessor();
  const int sub = threadIdx.x >> 4, lane = threadIdx.x & 15;
  const int64_t item = blockIdx.x, rb = item / p.col_blocks, cb = item - rb * p.col_blocks;
  const int64_t c = cb * kBlock + lane * 8;
  Raw<DT> v[kEach];
  uint32_t most = 0u;
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int64_t row = rb * kBlock + k * (kTableThreads / 16) + sub;
    const bool live = row < p.rows;
    v[k] = load8<DT, VEC>(static_cast<const char *>(p.x) + (live ? row : 0) * p.x_stride * (DT == 0 ? 4 : 2), c, live ? p.cols - c : 0);
  }
#pragma unroll
  for (int k = 0; k < kEach; ++k) most = max(most, most8(v[k]));
  most = __reduce_max_sync(0xffffffffu, most);
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = most;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kTableThreads / 32; ++w) most = max(most, sh[w]);
  float inverse;
  const float scale = scale_of(most, inverse);
  if (threadIdx.x == 0) p.scale[rb * p.scale_stride + cb] = scale;
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int64_t row = rb * kBlock + k * (kTableThreads / 16) + sub;
    if (row < p.rows) store8<DT, VEC>(p.q + row * p.q_stride + c, p.cols - c, v[k], inverse);
  }
}

inline bool misaligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) != 0; }

}  // namespace
}  // namespace e3

extern "C" e3_status e3_quantize(const void *x, e3_dtype dt, int64_t rows, int64_t cols, int64_t row_stride, int32_t block_rows,
                                 uint8_t *q, int64_t q_stride, float *scale, int64_t scale_stride, void *stream) {
  using namespace e3;
  if (dt != E3_F32 && dt != E3_BF16) return E3_ERR_DTYPE;
  const int64_t most = int64_t(1) << 31;
  const int64_t col_blocks = (cols + kBlock - 1) / kBlock;
  if (rows < 0 || rows >= most || cols < 1 || cols >= most || row_stride < cols || q_stride < cols || scale_stride < col_blocks ||
      (block_rows != 1 && block_rows != kBlock))
    return E3_ERR_INVALID_ARG;
  if (rows == 0) return E3_OK;
  if (!x || !q || !scale) return E3_ERR_INVALID_ARG;
  const size_t es = dt == E3_F32 ? 4 : 2;
  if (misaligned(x, es) || misaligned(scale, 4)) return E3_ERR_ALIGNMENT;
  QuantParams p = {};
  p.x = x; p.q = q; p.scale = scale; p.rows = rows; p.cols = cols; p.x_stride = row_stride; p.q_stride = q_stride;
  p.scale_stride = scale_stride; p.col_blocks = col_blocks; p.row_blocks = (rows + block_rows - 1) / block_rows;
  const int64_t items = p.row_blocks * col_blocks, ctas = block_rows == 1 ? (items + 2 * kRowWarps - 1) / (2 * kRowWarps) : items;
  if (ctas >= most) return E3_ERR_INVALID_ARG;
  const bool vec = !misaligned(x, 16) && row_stride * es % 16 == 0 && !misaligned(q, 8) && q_stride % 8 == 0;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)ctas);
  cfg.blockDim = dim3(block_rows == 1 ? kRowWarps * 32 : kTableThreads);
  cfg.stream = static_cast<cudaStream_t>(stream);
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  void (*kern)(QuantParams) =
      block_rows == 1 ? (dt == E3_F32 ? (vec ? quantize_rows_kernel<0, true> : quantize_rows_kernel<0, false>)
                                      : (vec ? quantize_rows_kernel<1, true> : quantize_rows_kernel<1, false>))
                      : (dt == E3_F32 ? (vec ? quantize_table_kernel<0, true> : quantize_table_kernel<0, false>)
                                      : (vec ? quantize_table_kernel<1, true> : quantize_table_kernel<1, false>));
  return cudaLaunchKernelEx(&cfg, kern, p) == cudaSuccess ? E3_OK : E3_ERR_CUDA;
}
