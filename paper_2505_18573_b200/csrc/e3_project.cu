// The vocabulary's projection in 8 bits: logits[r, v] = sum_k sx[r, k] sw[v / 128, k] sum_{i in block k} x[r, i] w[v, i], x and w in e4m3.
//
// The table's rows are the tensor cores' M (128 of them, so that a tile has one table scale per block of 128 columns) and the hidden states'
// rows are N, so that a call of a few rows streams the table through tiles of 128 x 16 and the logits of 32 neighbouring vocabulary entries
// are written by the 32 lanes of a warp.  Persistent CTAs, one per SM: a producer thread keeps a ring of TMA copies (128 x 128 bytes of the
// table and the tokens' 128 bytes each, swizzled) under way, one thread issues the tcgen05 products of a block into one of two accumulators in
// tensor memory, a warp lays out the products of the scales, and one or two warpgroups take the block's sums from there, scale them and add them
// up in fp32 registers.  8-bit products of 128 entries are added in 32 bits by the tensor cores, blocks in fp32 here; the logits are rounded once.
//
// Every wait is bounded: one that runs out marks the call's status word, and the CTA's unfinished logits read NaN.
#include "e3_rows_device.cuh"

#include <cuda.h>

#include <atomic>
#include <mutex>

#include "e3.h"

namespace e3 {
namespace {

constexpr int kTileV = 128;                // vocabulary entries of a tile: rows of the tensor memory
constexpr int kTileK = E3_SCALE_BLOCK;     // bytes of a row per stage: a block of one scale, and the width of the swizzle
constexpr int kScaleGroup = 4;             // blocks whose scales are fetched together
constexpr int kScaleRing = 2 * kScaleGroup;
constexpr int kSmemMost = 200 * 1024;      // of the ring of stages

struct ProjectParams {
  const float *x_scale, *w_scale;
  int64_t x_scale_stride, w_scale_stride;
  void *out;
  int64_t out_stride;
  int32_t *status;
  int rows, V, blocks;  // blocks: of 128 columns
  int row_tiles;
  int64_t tiles;        // row tiles run fastest: neighbours share the table's rows in L2
  u64 wait_ns;
};

// NT: rows of the hidden states in a tile (N of the products).
template <int NT>
struct Plan {
  static constexpr int kGroups = NT > 128 ? 2 : 1;           // warpgroups that take sums
  static constexpr int kSumWarps = 4 * kGroups;
  static constexpr int kCols = NT / kGroups;                 // columns of a thread
  static constexpr int kThreads = (kSumWarps + 3) * 32;      // and a producer, an issuer, a warp for the scales
  static constexpr int kStageBytes = (kTileV + NT) * kTileK;
  static constexpr int kStages = kSmemMost / kStageBytes < 12 ? kSmemMost / kStageBytes : 12;
  static constexpr int kTmemCols = 2 * NT < 32 ? 32 : 2 * NT;
  static constexpr size_t kSmem = (size_t)kStages * kStageBytes + 1024;  // (the ring begins on a 1,024-byte boundary)
};

template <int NT>
struct __align__(16) Shared {
  float scale[kScaleRing][NT];
  u64 full[Plan<NT>::kStages], empty[Plan<NT>::kStages];
  u64 sum_full[2], sum_empty[2];
  u64 scale_full[kScaleRing], scale_empty[kScaleRing];
  u64 drained;
  uint32_t tmem;
  int gave_up;
};

__device__ __forceinline__ void mbar_arrive(u64 *b) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(b)) : "memory");
}
// Waits for a phase; false after the limit, or once another thread of the CTA has given up.
__device__ __forceinline__ bool wait_for(u64 *b, uint32_t parity, int *gave_up, u64 limit) {
  if (mbar_try_wait(b, parity)) return true;
  const u64 t0 = global_ns();
  for (uint32_t it = 1;; ++it) {
    if (mbar_try_wait(b, parity)) return true;
    if ((it & 31u) == 0u && (*(volatile int *)gave_up != 0 || global_ns() - t0 > limit)) {
      *(volatile int *)gave_up = 1;
      return false;
    }
  }
}
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap *map, int x, int y, u64 *bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
               "l"(map), "r"(x), "r"(y), "r"(smem_addr(bar))
               : "memory");
}
// Shared-memory operand of a product: rows of 128 bytes, 128-byte swizzle, eight rows 1,024 bytes apart.
__device__ __forceinline__ u64 operand(uint32_t addr) {
  return (u64)((addr >> 4) & 0x3FFFu) | (u64)1 << 16 | (u64)(1024 >> 4) << 32 | (u64)1 << 46 | (u64)2 << 61;
}
__device__ __forceinline__ void multiply(uint32_t d, u64 a, u64 b, uint32_t form, uint32_t add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a),
      "l"(b), "r"(form), "r"(add)
      : "memory");
}
// Arrives on `bar` once the thread's products so far are done.
__device__ __forceinline__ void commit(u64 *bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar)) : "memory");
}
__device__ __forceinline__ void tmem_load16(uint32_t addr, float (&v)[16]) {
  uint32_t r[16];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(addr));
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_wait(float (&v)[16]) {  // the loaded values may be used behind it
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]), "+f"(v[9]),
                 "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15])::"memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

template <int OUT>
__device__ __forceinline__ void store_logit(void *out, int64_t at, float v) {
  if (OUT == 0) static_cast<float *>(out)[at] = v;
  else static_cast<__nv_bfloat16 *>(out)[at] = __float2bfloat16_rn(v);
}

template <int NT, int OUT>
__global__ void __launch_bounds__(Plan<NT>::kThreads, 1)
    project_kernel(const __grid_constant__ CUtensorMap w_map, const __grid_constant__ CUtensorMap x_map, const __grid_constant__ ProjectParams p) {
  using L = Plan<NT>;
  extern __shared__ unsigned char dyn[];
  __shared__ Shared<NT> sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const uint32_t ring = (smem_addr(dyn) + 1023u) & ~1023u;
  if (tid == 0) {
    for (int i = 0; i < L::kStages; ++i) {
      mbar_init(&sh.full[i], 1);
      mbar_init(&sh.empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.sum_full[i], 1);
      mbar_init(&sh.sum_empty[i], L::kSumWarps);
    }
    for (int i = 0; i < kScaleRing; ++i) {
      mbar_init(&sh.scale_full[i], 32);
      mbar_init(&sh.scale_empty[i], L::kSumWarps);
    }
    mbar_init(&sh.drained, 1);
    sh.gave_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
  }
  if (warp == L::kSumWarps + 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&sh.tmem)), "r"(L::kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    fence_before();
  }
  __syncthreads();
  fence_after();
  const uint32_t tmem = sh.tmem;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");

  if (warp == L::kSumWarps) {
    // ---- producer
    if (lane == 0) {
      uint32_t n = 0;
      bool on = true;
      for (int64_t tile = blockIdx.x; tile < p.tiles && on; tile += gridDim.x) {
        const int tv = (int)(tile / p.row_tiles) * kTileV, tr = (int)(tile % p.row_tiles) * NT;
        for (int k = 0; k < p.blocks && on; ++k, ++n) {
          const uint32_t s = n % L::kStages, round = n / L::kStages;
          on = wait_for(&sh.empty[s], (round & 1u) ^ 1u, &sh.gave_up, p.wait_ns);
          if (!on) break;
          const uint32_t at = ring + s * L::kStageBytes;
          mbar_arrive_expect(&sh.full[s], L::kStageBytes);
          tma_load(at, &w_map, k * kTileK, tv, &sh.full[s]);
          tma_load(at + kTileV * kTileK, &x_map, k * kTileK, tr, &sh.full[s]);
        }
      }
      if (!on) {  // given up: the copies under way still land in this CTA's memory
        for (uint32_t m = n > L::kStages ? n - L::kStages : 0; m < n; ++m) {
          const u64 t0 = global_ns();
          while (!mbar_try_wait(&sh.full[m % L::kStages], (m / L::kStages) & 1u) && global_ns() - t0 < p.wait_ns) {
          }
        }
      }
    }
  } else if (warp == L::kSumWarps + 1) {
    // ---- issuer of the products
    if (lane == 0) {
      // fp32 sums of e4m3 x e4m3, both operands along their rows
      constexpr uint32_t kForm = 1u << 4 | (uint32_t)(NT >> 3) << 17 | (uint32_t)(kTileV >> 4) << 24;
      uint32_t n = 0;
      bool on = true;
      for (int64_t tile = blockIdx.x; tile < p.tiles && on; tile += gridDim.x) {
        for (int k = 0; k < p.blocks && on; ++k, ++n) {
          const uint32_t s = n % L::kStages, round = n / L::kStages, half = n & 1u;
          on = wait_for(&sh.sum_empty[half], ((n >> 1) & 1u) ^ 1u, &sh.gave_up, p.wait_ns) &&
               wait_for(&sh.full[s], round & 1u, &sh.gave_up, p.wait_ns);
          if (!on) break;
          fence_after();
          const uint32_t at = ring + s * L::kStageBytes;
          const u64 a = operand(at), b = operand(at + kTileV * kTileK);
#pragma unroll
          for (int i = 0; i < kTileK / 32; ++i)  // 32 bytes of every row at a time
            multiply(tmem + half * NT, a + (u64)(2 * i), b + (u64)(2 * i), kForm, i > 0);
          commit(&sh.empty[s]);
          commit(&sh.sum_full[half]);
        }
      }
      // products under way (there are some if the CTA has given up) write the tensor memory, and their signals its shared memory
      commit(&sh.drained);
      const u64 t0 = global_ns();
      while (!mbar_try_wait(&sh.drained, 0) && global_ns() - t0 < p.wait_ns) {
      }
    }
  } else if (warp == L::kSumWarps + 2) {
    // ---- products of the scales, four blocks at a time
    constexpr int kEach = (NT + 31) / 32;
    uint32_t n = 0;
    bool on = true;
    for (int64_t tile = blockIdx.x; tile < p.tiles && on; tile += gridDim.x) {
      const int64_t tv = tile / p.row_tiles;
      const int tr = (int)(tile % p.row_tiles) * NT;
      for (int k0 = 0; k0 < p.blocks && on; k0 += kScaleGroup) {
        float sw[kScaleGroup], sx[kScaleGroup][kEach];
#pragma unroll
        for (int k = 0; k < kScaleGroup; ++k) {
          sw[k] = k0 + k < p.blocks ? p.w_scale[tv * p.w_scale_stride + k0 + k] : 0.f;
#pragma unroll
          for (int i = 0; i < kEach; ++i) {
            const int r = tr + i * 32 + lane;
            sx[k][i] = k0 + k < p.blocks && r < p.rows ? p.x_scale[r * p.x_scale_stride + k0 + k] : 0.f;
          }
        }
#pragma unroll
        for (int k = 0; k < kScaleGroup; ++k) {
          if (k0 + k >= p.blocks || !on) break;
          const uint32_t s = n % kScaleRing;
          on = __all_sync(0xffffffffu, wait_for(&sh.scale_empty[s], ((n / kScaleRing) & 1u) ^ 1u, &sh.gave_up, p.wait_ns));
          if (!on) break;
#pragma unroll
          for (int i = 0; i < kEach; ++i)
            if (i * 32 + lane < NT) sh.scale[s][i * 32 + lane] = sx[k][i] * sw[k];
          mbar_arrive(&sh.scale_full[s]);
          ++n;
        }
      }
    }
  } else {
    // ---- sums: a thread has one vocabulary entry and kCols rows
    constexpr int kCols = L::kCols;
    const int group = warp >> 2;
    const uint32_t from = tmem + ((uint32_t)(warp & 3) << 21) + group * kCols;  // (lane 32 (warp mod 4) of the tensor memory)
    uint32_t n = 0;
    bool on = true;
    for (int64_t tile = blockIdx.x; tile < p.tiles; tile += gridDim.x) {
      const int64_t v = (tile / p.row_tiles) * kTileV + (warp & 3) * 32 + lane;
      const int r0 = (int)(tile % p.row_tiles) * NT + group * kCols;
      f2 sum[kCols / 2];
#pragma unroll
      for (int i = 0; i < kCols / 2; ++i) sum[i] = pack2f(0.f, 0.f);
      for (int k = 0; k < p.blocks && on; ++k, ++n) {
        const uint32_t s = n % kScaleRing, half = n & 1u;
        on = __all_sync(0xffffffffu, wait_for(&sh.scale_full[s], (n / kScaleRing) & 1u, &sh.gave_up, p.wait_ns) &&
                                         wait_for(&sh.sum_full[half], (n >> 1) & 1u, &sh.gave_up, p.wait_ns));
        if (!on) break;
        fence_after();
        const uint32_t scale = smem_addr(&sh.scale[s][group * kCols]);
        float t[2][16];
        tmem_load16(from + half * NT, t[0]);
#pragma unroll
        for (int c = 0; c < kCols / 16; ++c) {
          tmem_wait(t[c & 1]);
          if (c + 1 < kCols / 16) tmem_load16(from + half * NT + (c + 1) * 16, t[(c + 1) & 1]);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint4 w = lds128(scale + (uint32_t)(c * 16 + i * 4) * 4u);
            f2 &a = sum[c * 8 + 2 * i], &b = sum[c * 8 + 2 * i + 1];
            a = fma2(pack2f(t[c & 1][4 * i], t[c & 1][4 * i + 1]), pack2f(__uint_as_float(w.x), __uint_as_float(w.y)), a);
            b = fma2(pack2f(t[c & 1][4 * i + 2], t[c & 1][4 * i + 3]), pack2f(__uint_as_float(w.z), __uint_as_float(w.w)), b);
          }
        }
        fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&sh.sum_empty[half]);
          mbar_arrive(&sh.scale_empty[s]);
        }
      }
      if (v < p.V) {
#pragma unroll
        for (int i = 0; i < kCols; ++i) {
          if (r0 + i < p.rows)
            store_logit<OUT>(p.out, (int64_t)(r0 + i) * p.out_stride + v, on ? ((i & 1) != 0 ? sum[i >> 1].y : sum[i >> 1].x) : CUDART_NAN_F);
        }
      }
    }
    if (!on && lane == 0 && p.status != nullptr) atomicOr(p.status, kStatusTimeout);
  }
  fence_before();
  __syncthreads();
  if (warp == L::kSumWarps + 1) {
    __syncwarp();
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(L::kTmemCols));
  }
}

// ---- host side -----------------------------------------------------------------------------------------------------
inline bool misaligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) != 0; }

using Encode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                            const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
Encode encode_function() {
  static std::atomic<void *> known{nullptr};
  void *f = known.load();
  if (f == nullptr) {
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess)
      return nullptr;
    known.store(f);
  }
  return reinterpret_cast<Encode>(f);
}
// [rows, cols] bytes with `stride` bytes from row to row, copied `box` rows by 128 bytes at a time; what lies outside reads 0.
bool make_map(Encode encode, CUtensorMap *map, const void *data, int64_t rows, int64_t cols, int64_t stride, int box) {
  const cuuint64_t size[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)stride};
  const cuuint32_t boxes[2] = {(cuuint32_t)kTileK, (cuuint32_t)box}, steps[2] = {1, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(data), size, strides, boxes, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// SMs of the current device; 0 where that cannot be told.
int sm_count(int &dev) {
  static std::atomic<int> sms[64];
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
  int count = sms[dev].load();
  if (count == 0) {
    if (cudaDeviceGetAttribute(&count, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    sms[dev].store(count);
  }
  return count;
}

struct Call {
  const void *x, *w;
  int64_t x_stride, w_stride, D;
  ProjectParams p;
};

template <int NT, int OUT>
cudaError_t launch(Call &c, cudaStream_t stream) {
  using L = Plan<NT>;
  static std::mutex lock;
  static bool ready[64];
  auto kern = project_kernel<NT, OUT>;
  int dev = 0;
  const int sms = sm_count(dev);
  if (sms == 0) return cudaErrorInvalidDevice;
  {
    std::lock_guard<std::mutex> hold(lock);
    if (!ready[dev]) {
      const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)L::kSmem);
      if (e != cudaSuccess) return e;
      ready[dev] = true;
    }
  }
  const Encode encode = encode_function();
  CUtensorMap w_map, x_map;
  if (encode == nullptr || !make_map(encode, &w_map, c.w, c.p.V, c.D, c.w_stride, kTileV) ||
      !make_map(encode, &x_map, c.x, c.p.rows, c.D, c.x_stride, NT))
    return cudaErrorInvalidValue;
  c.p.row_tiles = (c.p.rows + NT - 1) / NT;
  c.p.tiles = (int64_t)((c.p.V + kTileV - 1) / kTileV) * c.p.row_tiles;
  c.p.wait_ns = kDefaultWaitNs;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(c.p.tiles < sms ? c.p.tiles : sms));
  cfg.blockDim = dim3(L::kThreads);
  cfg.dynamicSmemBytes = L::kSmem;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, w_map, x_map, c.p);
}

template <int OUT>
cudaError_t launch_sized(Call &c, cudaStream_t stream) {
  if (c.p.rows <= 16) return launch<16, OUT>(c, stream);
  if (c.p.rows <= 32) return launch<32, OUT>(c, stream);
  if (c.p.rows <= 64) return launch<64, OUT>(c, stream);
  if (c.p.rows <= 128) return launch<128, OUT>(c, stream);
  return launch<256, OUT>(c, stream);
}

}  // namespace
}  // namespace e3

extern "C" e3_status e3_project_vocab(const uint8_t *x, const float *x_scale, int64_t rows, int64_t x_stride, int64_t x_scale_stride,
                                      const uint8_t *w, const float *w_scale, int64_t V, int64_t w_stride, int64_t w_scale_stride, int64_t D,
                                      void *logits, e3_dtype dt, int64_t row_stride, int32_t *out_status, void *stream) {
  using namespace e3;
  if (dt != E3_F32 && dt != E3_BF16) return E3_ERR_DTYPE;
  const int64_t most = int64_t(1) << 31, blocks = (D + kTileK - 1) / kTileK;
  // (tiles may reach past the last row, coordinates are 32-bit)
  if (rows < 0 || rows >= most - 256 || V < 1 || V >= most - kTileV || D < 1 || D >= most - kTileK || x_stride < D || w_stride < D ||
      x_stride >= (int64_t(1) << 40) || w_stride >= (int64_t(1) << 40) || x_scale_stride < blocks || w_scale_stride < blocks || row_stride < V)
    return E3_ERR_INVALID_ARG;
  if (rows == 0) return E3_OK;
  if (!x || !x_scale || !w || !w_scale || !logits) return E3_ERR_INVALID_ARG;
  if (misaligned(x, 16) || misaligned(w, 16) || x_stride % 16 != 0 || w_stride % 16 != 0 || misaligned(x_scale, 4) || misaligned(w_scale, 4) ||
      misaligned(logits, dt == E3_F32 ? 4 : 2) || misaligned(out_status, 4))
    return E3_ERR_ALIGNMENT;
  Call c = {};
  c.x = x; c.w = w; c.x_stride = x_stride; c.w_stride = w_stride; c.D = D;
  c.p.x_scale = x_scale; c.p.w_scale = w_scale; c.p.x_scale_stride = x_scale_stride; c.p.w_scale_stride = w_scale_stride;
  c.p.out = logits; c.p.out_stride = row_stride; c.p.status = out_status;
  c.p.rows = (int)rows; c.p.V = (int)V; c.p.blocks = (int)blocks;
  cudaStream_t cs = static_cast<cudaStream_t>(stream);
  const cudaError_t e = dt == E3_F32 ? launch_sized<0>(c, cs) : launch_sized<1>(c, cs);
  return e == cudaSuccess ? E3_OK : E3_ERR_CUDA;
}
