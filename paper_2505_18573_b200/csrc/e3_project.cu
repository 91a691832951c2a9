// The vocabulary's projection in 8 bits: logits[r, v] = sum_k sx[r, k] sw[v / 128, k] sum_{i in block k} x[r, i] w[v, i], x and w in e4m3.
//
// Two kernels of the same kind: persistent CTAs, one per SM; a producer thread keeps a ring of TMA copies (a block's 128 bytes of every row of both
// operands, swizzled) under way, one thread issues the tcgen05 products of a block into one of two accumulators in tensor memory, and one or two
// warpgroups take the block's sums from there, scale them and add them up in fp32 registers.  8-bit products of 128 entries are added in 32 bits by
// the tensor cores, blocks in fp32 here; the logits are rounded once.
//   - Up to 64 rows: the table's rows are the tensor cores' M (128 of them: one table scale per tile and block), the hidden states' rows their N, so
//     that the table streams through tiles of 128 x 16, 32 or 64; bound by reading the table (8 rows, a table of 151,936 x 2,048: 54 us, 90 % of the rate
//     of a copy).  A lane has a vocabulary entry, the rows' scales come from shared memory.
//   - More rows: 128 of the hidden states' rows are M and 256 vocabulary entries N.  A lane has a row, so that its scale is one register and the
//     sums cost one multiply-add per entry and block and nothing else (with the other form's scales, four bytes per entry and block from shared
//     memory, a block of 128 x 256 x 128 took 2,200 cycles, the products 512).  Bound by the tensor memory, where the products of a block (512 cycles) and
//     the reads of its sums (256) take turns: 740 to 800 cycles a block; 512 rows, a table of 151,936 x 2,048: 169 us, 1.9 PFLOP/s
//     (190 to 200 in runs of seconds, in which the power limit holds the clock at 1.5 GHz).
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
  uint32_t row_tiles;
  int vectors;          // the logits' rows begin on 16-byte boundaries
  uint32_t tiles;       // row tiles run fastest: neighbours share the table's rows in L2
  u64 wait_ns;
  uint32_t stall;       // test hook: the first CTA's copies of this block (counted over its tiles) are never issued
};
constexpr uint32_t kNoStall = 0xffffffffu;
std::atomic<uint32_t> g_stall{kNoStall};
std::atomic<unsigned long long> g_stall_wait_ns{0};

// NT: rows of the hidden states in a tile (N of the products).
template <int NT>
struct Plan {
  static constexpr int kSumWarps = 4;
  static constexpr int kCols = NT;                           // columns of a thread
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
// Waits for a phase; false after the limit, or once another thread of the CTA has given up.  (The global timer is slow to read: not before some polls.)
template <bool CLUSTER>
__device__ __forceinline__ bool poll(u64 *b, uint32_t parity) {
  if (!CLUSTER) return mbar_try_wait(b, parity);
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(smem_addr(b)), "r"(parity)
      : "memory");
  return ok != 0;
}
template <bool CLUSTER = false>
__device__ __noinline__ bool wait_longer(u64 *b, uint32_t parity, int *gave_up, u64 limit) {
  u64 t0 = 0;
  for (uint32_t it = 0;; ++it) {
    if (poll<CLUSTER>(b, parity)) return true;
    if ((it & 63u) == 63u) {
      const u64 now = global_ns();
      if (t0 == 0) t0 = now;
      if (*(volatile int *)gave_up != 0 || now - t0 > limit) {
        *(volatile int *)gave_up = 1;
        return false;
      }
    }
  }
}
template <bool CLUSTER = false>  // CLUSTER: another CTA of the cluster arrives there
__device__ __forceinline__ bool wait_for(u64 *b, uint32_t parity, int *gave_up, u64 limit) {
  return poll<CLUSTER>(b, parity) || wait_longer<CLUSTER>(b, parity, gave_up, limit);
}
// One lane of the warp, always the same.  Loops whose copies and products one lane issues are run by the whole warp: their operands sit in uniform
// registers, and with a lane's own branch around the loop the compiler has to bring each there by a loop over the lanes (800 cycles a block).
__device__ __forceinline__ bool elected() {
  uint32_t is;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(is));
  return is != 0;
}
template <bool CLUSTER = false>
__device__ __forceinline__ bool wait_as_warp(u64 *b, uint32_t parity, int *gave_up, u64 limit) {
  return __all_sync(0xffffffffu, wait_for<CLUSTER>(b, parity, gave_up, limit));
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
  const uint32_t tmem = __shfl_sync(0xffffffffu, sh.tmem, 0);
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");

  if (warp == L::kSumWarps) {
    // ---- producer
    {
      const uint32_t stall = blockIdx.x == 0 ? p.stall : kNoStall;
      uint32_t n = 0;
      bool on = true;
      for (uint32_t tile = blockIdx.x; tile < p.tiles && on; tile += gridDim.x) {
        const int tv = (int)(tile / p.row_tiles) * kTileV, tr = (int)(tile % p.row_tiles) * NT;
        for (int k = 0; k < p.blocks && on; ++k, ++n) {
          const uint32_t s = n % L::kStages, round = n / L::kStages;
          on = wait_as_warp(&sh.empty[s], (round & 1u) ^ 1u, &sh.gave_up, p.wait_ns);
          if (!on) break;
          const uint32_t at = ring + s * L::kStageBytes;
          if (elected() && n != stall) {
            mbar_arrive_expect(&sh.full[s], L::kStageBytes);
            tma_load(at, &w_map, k * kTileK, tv, &sh.full[s]);
            tma_load(at + kTileV * kTileK, &x_map, k * kTileK, tr, &sh.full[s]);
          }
        }
      }
      if (!on && lane == 0) {  // given up: the copies under way still land in this CTA's memory
        for (uint32_t m = n > L::kStages ? n - L::kStages : 0; m < n; ++m) {
          const u64 t0 = global_ns();
          while (!mbar_try_wait(&sh.full[m % L::kStages], (m / L::kStages) & 1u) && global_ns() - t0 < p.wait_ns) {
          }
        }
      }
    }
  } else if (warp == L::kSumWarps + 1) {
    // ---- issuer of the products
    {
      // fp32 sums of e4m3 x e4m3, both operands along their rows
      constexpr uint32_t kForm = 1u << 4 | (uint32_t)(NT >> 3) << 17 | (uint32_t)(kTileV >> 4) << 24;
      uint32_t n = 0;
      bool on = true;
      for (uint32_t tile = blockIdx.x; tile < p.tiles && on; tile += gridDim.x) {
        for (int k = 0; k < p.blocks && on; ++k, ++n) {
          const uint32_t s = n % L::kStages, round = n / L::kStages, half = n & 1u;
          on = wait_as_warp(&sh.sum_empty[half], ((n >> 1) & 1u) ^ 1u, &sh.gave_up, p.wait_ns) &&
               wait_as_warp(&sh.full[s], round & 1u, &sh.gave_up, p.wait_ns);
          if (!on) break;
          fence_after();
          const uint32_t at = ring + s * L::kStageBytes;
          const u64 a = operand(at), b = operand(at + kTileV * kTileK);
          if (elected()) {
#pragma unroll
            for (int i = 0; i < kTileK / 32; ++i)  // 32 bytes of every row at a time
              multiply(tmem + half * NT, a + (u64)(2 * i), b + (u64)(2 * i), kForm, i > 0);
            commit(&sh.empty[s]);
            commit(&sh.sum_full[half]);
          }
        }
      }
      // products under way (there are some if the CTA has given up) write the tensor memory, and their signals its shared memory
      if (elected()) commit(&sh.drained);
      __syncwarp();
      const u64 t0 = global_ns();
      while (!mbar_try_wait(&sh.drained, 0) && global_ns() - t0 < p.wait_ns) {
      }
    }
  } else if (warp == L::kSumWarps + 2) {
    // ---- products of the scales, four blocks at a time
    constexpr int kEach = (NT + 31) / 32;
    uint32_t n = 0;
    bool on = true;
    for (uint32_t tile = blockIdx.x; tile < p.tiles && on; tile += gridDim.x) {
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
    const uint32_t from = tmem + ((uint32_t)warp << 21);  // (lane 32 warp of the tensor memory)
    uint32_t n = 0;
    bool on = true;
    for (uint32_t tile = blockIdx.x; tile < p.tiles; tile += gridDim.x) {
      const int64_t v = (int64_t)(tile / p.row_tiles) * kTileV + warp * 32 + lane;
      const int r0 = (int)(tile % p.row_tiles) * NT;
      f2 sum[kCols / 2];
#pragma unroll
      for (int i = 0; i < kCols / 2; ++i) sum[i] = pack2f(0.f, 0.f);
      for (int k = 0; k < p.blocks && on; ++k, ++n) {
        const uint32_t s = n % kScaleRing, half = n & 1u;
        on = __all_sync(0xffffffffu, wait_for(&sh.scale_full[s], (n / kScaleRing) & 1u, &sh.gave_up, p.wait_ns) &&
                                         wait_for(&sh.sum_full[half], (n >> 1) & 1u, &sh.gave_up, p.wait_ns));
        if (!on) break;
        fence_after();
        const uint32_t scale = smem_addr(&sh.scale[s][0]);
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

// ---- many rows -----------------------------------------------------------------------------------------------------
namespace wide {

// A tile has 128 rows and 256 vocabulary entries.  The issuing warp needs about 500 cycles a block however wide its products are (two waits, four
// products, a signal), so they are as wide as they can be: 512 cycles.
constexpr int kM = 128, kN = 256;
constexpr int kBuffers = 2;
constexpr int kCols = 128;             // columns of a thread
constexpr int kAhead = 2;              // blocks whose scales are fetched together
constexpr int kSumWarps = 4 * kN / kCols;
constexpr int kThreads = (kSumWarps + 2) * 32;
// A CTA alone has a tile to itself; a pair of CTAs shares the products of 256 rows x 256 entries, each with its own 128 rows of sums and half of the
// entries' operand in its shared memory.
template <bool PAIR>
struct Ring {
  static constexpr int kEntries = PAIR ? kN / 2 : kN;  // of the table, in this CTA
  static constexpr int kStageBytes = (kM + kEntries) * kTileK;
  static constexpr int kStages = PAIR ? 5 : 3;
};
// Finished logits leave through shared memory: 128 bytes of each of a warp's 32 rows at a time, swizzled, which one thread then sends off as a whole while
// the warp goes on (its own loads and stores of them, beside the products' and copies' use of the same memory, took 3,100 cycles a tile).
constexpr int kPieceBytes = 128, kPieces = 32 * kPieceBytes;
constexpr int kOutBytes = 2 * kPieces;  // of a warp
template <bool PAIR>
constexpr size_t kSmem = (size_t)Ring<PAIR>::kStages * Ring<PAIR>::kStageBytes + kSumWarps * kOutBytes + 1024;
static_assert(kSmem<false> + 512 <= 227 * 1024 && kSmem<true> + 512 <= 227 * 1024, "shared memory");

// Where 16 bytes of a row lie (the 128-byte swizzle).
__device__ __forceinline__ uint32_t piece_at(int row, int part) { return (uint32_t)(row * kPieceBytes + ((part ^ (row & 7)) << 4)); }
__device__ __forceinline__ void tma_store(const CUtensorMap *map, int x, int y, uint32_t src) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x), "r"(y), "r"(src) : "memory");
}

template <bool PAIR>
struct Shared {
  u64 full[Ring<PAIR>::kStages], empty[Ring<PAIR>::kStages];  // full, of a pair: in the first CTA, for the copies of both
  u64 sum_full[kBuffers], sum_empty[kBuffers];
  u64 drained;
  uint32_t tmem;
  int gave_up;
};

// 16 columns of the tensor memory; they may be read behind tmem_wait.
__device__ __forceinline__ void tmem_begin16(uint32_t addr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(addr)
      : "memory");
}
__device__ __forceinline__ void tmem_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
// (volatile: stays behind the wait.  Operands that pass through the wait, or leave one block with it, cost a move each.)
__device__ __forceinline__ void add_scaled(u64 &sum, uint32_t lo, uint32_t hi, u64 scale) {
  asm volatile("{ .reg .b64 v; mov.b64 v, {%1, %2}; fma.rn.f32x2 %0, v, %3, %0; }" : "+l"(sum) : "r"(lo), "r"(hi), "l"(scale));
}
__device__ __forceinline__ f2 pair_of(u64 v) { return make_float2(__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32))); }
__device__ __forceinline__ void sts128(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ uint32_t bf16_pair(f2 v) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(v.x, v.y);
  return *reinterpret_cast<const uint32_t *>(&h);
}

// Products of a pair of CTAs: issued by its first one, they read both CTAs' operands and write both CTAs' tensor memory.
__device__ __forceinline__ void multiply_pair(uint32_t d, u64 a, u64 b, uint32_t form, uint32_t add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a),
      "l"(b), "r"(form), "r"(add)
      : "memory");
}
// Arrives on `bar` of both CTAs, or of this one, once the pair's products so far are done.
__device__ __forceinline__ void commit_pair_to_both(u64 *bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_addr(bar)),
               "h"((unsigned short)3)
               : "memory");
}
__device__ __forceinline__ void commit_pair(u64 *bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar)) : "memory");
}
// Shared-memory address of the pair's first CTA.
__device__ __forceinline__ uint32_t in_first(const void *p) {
  uint32_t to;
  asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(to) : "r"(smem_addr(p)));
  return to;
}
// Arrives on the barrier of the pair's first CTA, behind the thread's reads of tensor memory.  (With release at cluster scope the arrival waits
// for the warp's logits under way: 1,500 cycles a block.)
__device__ __forceinline__ void arrive_at_first(u64 *b) { asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(in_first(b)) : "memory"); }
// A copy into this CTA whose bytes count on a barrier of the pair's first CTA.
__device__ __forceinline__ void tma_load_pair(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
               "l"(map), "r"(x), "r"(y), "r"(bar)
               : "memory");
}
__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

template <int OUT, bool PAIR>
__global__ void __launch_bounds__(kThreads, 1)
    project_rows_kernel(const __grid_constant__ CUtensorMap x_map, const __grid_constant__ CUtensorMap w_map, const __grid_constant__ CUtensorMap out_map,
                        const __grid_constant__ ProjectParams p) {
  constexpr int kStages = Ring<PAIR>::kStages, kStageBytes = Ring<PAIR>::kStageBytes;
  constexpr int kRows = PAIR ? 2 * kM : kM;  // of a tile
  extern __shared__ unsigned char dyn[];
  __shared__ Shared<PAIR> sh;
  const uint32_t rank = PAIR ? blockIdx.x & 1u : 0u, first_tile = PAIR ? blockIdx.x >> 1 : blockIdx.x, tile_step = PAIR ? gridDim.x >> 1 : gridDim.x;
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const uint32_t ring = (smem_addr(dyn) + 1023u) & ~1023u;
  if (tid == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(&sh.full[i], 1);
      mbar_init(&sh.empty[i], 1);
    }
    for (int i = 0; i < kBuffers; ++i) {
      mbar_init(&sh.sum_full[i], 1);
      mbar_init(&sh.sum_empty[i], PAIR ? 2 * kSumWarps : kSumWarps);
    }
    mbar_init(&sh.drained, 1);
    sh.gave_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
  }
  if (warp == kSumWarps + 1) {
    if (PAIR) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&sh.tmem)), "r"(kBuffers * kN) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&sh.tmem)), "r"(kBuffers * kN) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    fence_before();
  }
  __syncthreads();
  if (PAIR) cluster_barrier();  // (the other CTA's barriers stand, and its tensor memory is there)
  fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, sh.tmem, 0);
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");

  if (warp == kSumWarps) {
    // ---- producer
    {
      const uint32_t stall = blockIdx.x == 0 ? p.stall : kNoStall;
      uint32_t n = 0;
      bool on = true;
      for (uint32_t tile = first_tile; tile < p.tiles && on; tile += tile_step) {
        const int tv = (int)(tile / p.row_tiles) * kN + (int)rank * Ring<PAIR>::kEntries, tr = (int)(tile % p.row_tiles) * kRows + (int)rank * kM;
        for (int k = 0; k < p.blocks && on; ++k, ++n) {
          const uint32_t s = n % kStages, round = n / kStages;
          on = wait_as_warp(&sh.empty[s], (round & 1u) ^ 1u, &sh.gave_up, p.wait_ns);
          if (!on) break;
          const uint32_t at = ring + s * kStageBytes;
          if (elected() && n != stall) {
            if (PAIR) {
              if (rank == 0) mbar_arrive_expect(&sh.full[s], 2 * kStageBytes);
              const uint32_t bar = in_first(&sh.full[s]);
              tma_load_pair(at, &x_map, k * kTileK, tr, bar);
              tma_load_pair(at + kM * kTileK, &w_map, k * kTileK, tv, bar);
            } else {
              mbar_arrive_expect(&sh.full[s], kStageBytes);
              tma_load(at, &x_map, k * kTileK, tr, &sh.full[s]);
              tma_load(at + kM * kTileK, &w_map, k * kTileK, tv, &sh.full[s]);
            }
          }
        }
      }
      if (!on && lane == 0 && rank != 0) {  // given up: this CTA's copies count in the other; they land well within a millisecond
        const u64 t0 = global_ns();
        while (global_ns() - t0 < 1000000u) {
        }
      }
      if (!on && lane == 0 && rank == 0) {  // the copies under way still land in this CTA's memory (and the other's)
        for (uint32_t m = n > kStages ? n - kStages : 0; m < n; ++m) {
          const u64 t0 = global_ns();
          while (!mbar_try_wait(&sh.full[m % kStages], (m / kStages) & 1u) && global_ns() - t0 < p.wait_ns) {
          }
        }
      }
    }
  } else if (warp == kSumWarps + 1) {
    // ---- issuer of the products
    {
      constexpr uint32_t kForm = 1u << 4 | (uint32_t)(kN >> 3) << 17 | (uint32_t)(kRows >> 4) << 24;
      uint32_t n = 0;
      bool on = true;
      if (rank != 0) on = false;  // (a pair's products are issued by its first CTA)
      for (uint32_t tile = first_tile; tile < p.tiles && on; tile += tile_step) {
        for (int k = 0; k < p.blocks && on; ++k, ++n) {
          const uint32_t s = n % kStages, round = n / kStages, half = n % kBuffers;
          // both waits at once, as a rule there is nothing to wait for
          const uint32_t free_parity = ((n / kBuffers) & 1u) ^ 1u, here_parity = round & 1u;
          const bool free = poll<PAIR>(&sh.sum_empty[half], free_parity), here = poll<PAIR>(&sh.full[s], here_parity);
          if (!__all_sync(0xffffffffu, free && here))
            on = wait_as_warp<PAIR>(&sh.sum_empty[half], free_parity, &sh.gave_up, p.wait_ns) &&
                 wait_as_warp<PAIR>(&sh.full[s], here_parity, &sh.gave_up, p.wait_ns);
          if (!on) break;
          fence_after();
          const uint32_t at = ring + s * kStageBytes;
          const u64 a = operand(at), b = operand(at + kM * kTileK);
          if (elected()) {
#pragma unroll
            for (int i = 0; i < kTileK / 32; ++i) {
              if (PAIR) multiply_pair(tmem + half * kN, a + (u64)(2 * i), b + (u64)(2 * i), kForm, i > 0);
              else multiply(tmem + half * kN, a + (u64)(2 * i), b + (u64)(2 * i), kForm, i > 0);
            }
            if (PAIR) commit_pair_to_both(&sh.sum_full[half]);
            else commit(&sh.sum_full[half]);
          }
        }
      }
      // products under way (there are some if the CTA has given up) write the tensor memory, and their signals its shared memory
      if (rank == 0) {
        if (elected()) {
          if (PAIR) commit_pair(&sh.drained);
          else commit(&sh.drained);
        }
        __syncwarp();
        const u64 t0 = global_ns();
        while (!mbar_try_wait(&sh.drained, 0) && global_ns() - t0 < p.wait_ns) {
        }
      }
    }
  } else {
    // ---- sums: a thread has one row and kCols vocabulary entries
    constexpr int kEsize = OUT == 0 ? 4 : 2, kPieceCols = kPieceBytes / kEsize;
    const int group = warp >> 2, row_of_warp = (int)rank * kM + (warp & 3) * 32;
    const uint32_t from = tmem + ((uint32_t)(warp & 3) << 21) + group * kCols;  // (lane 32 (warp mod 4) of the tensor memory)
    const uint32_t piece = ring + kStages * kStageBytes + warp * kOutBytes;
    uint32_t n = 0;
    bool on = true;
    // scales of kAhead blocks ahead, the next tile's first ones too: the row's, and the table's for these entries (multiplied when they are needed, or
    // the loads would be waited for here)
    float next_x[kAhead], next_w[kAhead];
    const float *sx, *sw, *next_sx, *next_sw;
    auto point_at = [&](uint32_t tile, const float *&sx, const float *&sw) {
      const uint32_t tv = tile / p.row_tiles;
      const int64_t r = (int64_t)(tile - tv * p.row_tiles) * kRows + row_of_warp + lane;
      sx = p.x_scale + (r < p.rows ? r : 0) * p.x_scale_stride;
      const int64_t block = ((int64_t)tv * kN + group * kCols) / E3_SCALE_BLOCK;  // (a tile may reach past the last)
      sw = p.w_scale + (block * E3_SCALE_BLOCK < p.V ? block : 0) * p.w_scale_stride;
    };
    auto fetch = [&](int k0) {
      if (k0 + kAhead <= p.blocks) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          next_x[k] = sx[k0 + k];
          next_w[k] = sw[k0 + k];
        }
      } else {
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          next_x[k] = sx[k0 + k < p.blocks ? k0 + k : 0];
          next_w[k] = sw[k0 + k < p.blocks ? k0 + k : 0];
        }
      }
    };
    static_assert(E3_SCALE_BLOCK % kCols == 0, "one scale of the table a thread and block");
    point_at(first_tile < p.tiles ? first_tile : 0, next_sx, next_sw);
    sx = next_sx;
    sw = next_sw;
    fetch(0);
    for (uint32_t tile = first_tile; tile < p.tiles; tile += tile_step) {
      const int64_t v0 = (int64_t)(tile / p.row_tiles) * kN + group * kCols;
      const int64_t r0 = (int64_t)(tile % p.row_tiles) * kRows + row_of_warp;
      // the next tile's scales are on their way while this one is summed: from memory they take as long as three blocks
      const bool more = tile + tile_step < p.tiles;
      if (more) {
        point_at(tile + tile_step, next_sx, next_sw);
        for (int k = 0; k < p.blocks; k += 32) {
          asm volatile("prefetch.global.L1 [%0];" ::"l"(next_sx + k));
          asm volatile("prefetch.global.L1 [%0];" ::"l"(next_sw + k));
        }
      }
      u64 sum[kCols / 2];
#pragma unroll
      for (int i = 0; i < kCols / 2; ++i) sum[i] = 0ull;
      float scale[kAhead];
#pragma unroll 1
      for (int k = 0; k < p.blocks && on; ++k, ++n) {
        if ((k & (kAhead - 1)) == 0) {
#pragma unroll
          for (int i = 0; i < kAhead; ++i) scale[i] = next_x[i] * next_w[i];
          if (k + kAhead < p.blocks) {
            fetch(k + kAhead);
          } else if (more) {
            sx = next_sx;
            sw = next_sw;
            fetch(0);
          }
        }
        const uint32_t bits = __float_as_uint(scale[0]);
        const u64 c2 = (u64)bits << 32 | bits;
        scale[0] = scale[1];
        const uint32_t half = n % kBuffers;
        on = wait_as_warp<PAIR>(&sh.sum_full[half], (n / kBuffers) & 1u, &sh.gave_up, p.wait_ns);
        if (!on) break;
        // (the products have read their operands too)
        if (warp == 0 && lane == 0) mbar_arrive(&sh.empty[n % kStages]);
        fence_after();
#pragma unroll
        for (int q = 0; q < kCols / 16; ++q) {
          uint32_t t[16];
          tmem_begin16(from + half * kN + q * 16, t);
          tmem_wait();
          if (q + 1 == kCols / 16) {
            fence_before();
            __syncwarp();
            if (lane == 0) {
              if (PAIR) arrive_at_first(&sh.sum_empty[half]);
              else mbar_arrive(&sh.sum_empty[half]);
            }
          }
#pragma unroll
          for (int i = 0; i < 8; ++i) add_scaled(sum[q * 8 + i], t[2 * i], t[2 * i + 1], c2);
        }
      }
      // ---- the tile's logits, two pieces at a time
      if (!on) {
#pragma unroll
        for (int i = 0; i < kCols / 2; ++i) sum[i] = 0x7FC000007FC00000ull;
      }
      const int left = (int)(p.rows - r0 < 32 ? (p.rows > r0 ? p.rows - r0 : 0) : 32);  // rows of this warp
      char *const to = static_cast<char *>(p.out) + (r0 * p.out_stride + v0) * kEsize;
      const int64_t row_bytes = p.out_stride * kEsize;
#pragma unroll
      for (int q = 0; q < kCols / kPieceCols; q += 2) {
        if (p.vectors) {  // (what was sent before has left)
          if (elected()) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
        }
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            uint32_t w[4];
#pragma unroll
            for (int h = 0; h < 4; ++h) {
              if (OUT == 1) {
                w[h] = bf16_pair(pair_of(sum[(q + j) * 32 + i * 4 + h]));
              } else {
                const f2 x = pair_of(sum[(q + j) * 16 + i * 2 + (h >> 1)]);
                w[h] = __float_as_uint((h & 1) != 0 ? x.y : x.x);
              }
            }
            sts128(piece + (uint32_t)(j * kPieces) + piece_at(lane, i), w[0], w[1], w[2], w[3]);
          }
        }
        if (p.vectors) {
          fence_async_smem();
          __syncwarp();
          if (elected()) {
            if (left > 0) {  // (rows and entries behind the last are left out by the copy)
              if (v0 + q * kPieceCols < p.V) tma_store(&out_map, (int)v0 + q * kPieceCols, (int)r0, piece);
              if (v0 + (q + 1) * kPieceCols < p.V) tma_store(&out_map, (int)v0 + (q + 1) * kPieceCols, (int)r0, piece + kPieces);
            }
            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
          }
        } else {  // rows that begin anywhere
          __syncwarp();
#pragma unroll 1
          for (int j = 0; j < 2; ++j) {
#pragma unroll 1
            for (int col = lane; col < kPieceCols; col += 32) {
              if (v0 + (q + j) * kPieceCols + col >= p.V) break;
              char *there = to + ((q + j) * kPieceCols + col) * kEsize;
#pragma unroll 8
              for (int rr = 0; rr < left; ++rr, there += row_bytes) {
                const uint32_t at = piece + (uint32_t)(j * kPieces) + piece_at(rr, col * kEsize >> 4) + (uint32_t)(col * kEsize & 15);
                if (OUT == 0) {
                  *reinterpret_cast<float *>(there) = lds_elem<0>(at);
                } else {
                  unsigned short h;
                  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(h) : "r"(at));
                  *reinterpret_cast<unsigned short *>(there) = h;
                }
              }
            }
          }
        }
      }
    }
    if (p.vectors && elected()) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    __syncwarp();
    if (!on && lane == 0 && p.status != nullptr) atomicOr(p.status, kStatusTimeout);
  }
  fence_before();
  __syncthreads();
  if (PAIR) cluster_barrier();  // (the other CTA's products and signals reach into this one)
  if (warp == kSumWarps + 1) {
    __syncwarp();
    fence_after();
    if (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kBuffers * kN));
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kBuffers * kN));
  }
}

}  // namespace wide

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

// The logits, sent 32 rows by 128 bytes at a time.
bool make_out_map(Encode encode, CUtensorMap *map, void *data, int64_t rows, int64_t cols, int64_t stride, int out) {
  const int es = out == 0 ? 4 : 2;
  const cuuint64_t size[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)(stride * es)};
  const cuuint32_t boxes[2] = {(cuuint32_t)(128 / es), 32}, steps[2] = {1, 1};
  return encode(map, out == 0 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, data, size, strides, boxes, steps,
                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
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
  const int64_t tiles = (int64_t)((c.p.V + kTileV - 1) / kTileV) * c.p.row_tiles;
  if (tiles >= (int64_t)1 << 31) return cudaErrorInvalidValue;
  c.p.tiles = (uint32_t)tiles;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles < sms ? tiles : sms));
  cfg.blockDim = dim3(L::kThreads);
  cfg.dynamicSmemBytes = L::kSmem;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, w_map, x_map, c.p);
}

template <int OUT, bool PAIR>
cudaError_t launch_wide(Call &c, cudaStream_t stream) {
  using R = wide::Ring<PAIR>;
  static std::mutex lock;
  static int held[64];  // CTAs, or pairs of them, that the device holds
  auto kern = wide::project_rows_kernel<OUT, PAIR>;
  int dev = 0;
  const int sms = sm_count(dev);
  if (sms == 0) return cudaErrorInvalidDevice;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = 2;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(wide::kThreads);
  cfg.dynamicSmemBytes = wide::kSmem<PAIR>;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = PAIR ? 2 : 1;
  {
    std::lock_guard<std::mutex> hold(lock);
    if (held[dev] == 0) {
      cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)wide::kSmem<PAIR>);
      if (e != cudaSuccess) return e;
      int n = sms;
      if (PAIR) {
        cudaLaunchConfig_t one = cfg;
        one.gridDim = dim3(2);
        one.attrs = attr + 1;
        one.numAttrs = 1;
        one.stream = nullptr;
        e = cudaOccupancyMaxActiveClusters(&n, kern, &one);
        if (e != cudaSuccess) return e;
        if (n < 1) return cudaErrorInvalidConfiguration;
      }
      held[dev] = n;
    }
  }
  const Encode encode = encode_function();
  CUtensorMap w_map, x_map, out_map = {};
  if (encode == nullptr || !make_map(encode, &w_map, c.w, c.p.V, c.D, c.w_stride, R::kEntries) ||
      !make_map(encode, &x_map, c.x, c.p.rows, c.D, c.x_stride, wide::kM) ||
      (c.p.vectors && !make_out_map(encode, &out_map, c.p.out, c.p.rows, c.p.V, c.p.out_stride, OUT)))
    return cudaErrorInvalidValue;
  const int rows = PAIR ? 2 * wide::kM : wide::kM;
  c.p.row_tiles = (uint32_t)((c.p.rows + rows - 1) / rows);
  const int64_t tiles = (int64_t)((c.p.V + wide::kN - 1) / wide::kN) * c.p.row_tiles;
  if (tiles >= (int64_t)1 << 31) return cudaErrorInvalidValue;
  c.p.tiles = (uint32_t)tiles;
  cfg.gridDim = dim3((unsigned)(tiles < held[dev] ? tiles : held[dev]) * (PAIR ? 2u : 1u));
  return cudaLaunchKernelEx(&cfg, kern, x_map, w_map, out_map, c.p);
}

template <int OUT>
cudaError_t launch_sized(Call &c, cudaStream_t stream) {
  if (c.p.rows <= 16) return launch<16, OUT>(c, stream);
  if (c.p.rows <= 32) return launch<32, OUT>(c, stream);
  if (c.p.rows <= 64) return launch<64, OUT>(c, stream);
  if (c.p.rows <= wide::kM) return launch_wide<OUT, false>(c, stream);
  return launch_wide<OUT, true>(c, stream);
}

}  // namespace
}  // namespace e3

extern "C" e3_status e3_project_vocab(const uint8_t *x, const float *x_scale, int64_t rows, int64_t x_stride, int64_t x_scale_stride,
                                      const uint8_t *w, const float *w_scale, int64_t V, int64_t w_stride, int64_t w_scale_stride, int64_t D,
                                      void *logits, e3_dtype dt, int64_t row_stride, int32_t *out_status, void *stream) {
  using namespace e3;
  if (dt != E3_F32 && dt != E3_BF16) return E3_ERR_DTYPE;
  const int64_t most = int64_t(1) << 31, blocks = (D + kTileK - 1) / kTileK;
  // (tiles of up to 256 may reach past the last row, entry or column, coordinates are 32-bit)
  if (rows < 0 || rows >= most - 256 || V < 1 || V >= most - 256 || D < 1 || D >= most - 256 || x_stride < D || w_stride < D ||
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
  c.p.stall = g_stall.exchange(kNoStall);
  c.p.wait_ns = c.p.stall == kNoStall ? kDefaultWaitNs : g_stall_wait_ns.load();
  c.p.vectors = !misaligned(logits, 16) && row_stride * (dt == E3_F32 ? 4 : 2) % 16 == 0;
  cudaStream_t cs = static_cast<cudaStream_t>(stream);
  const cudaError_t e = dt == E3_F32 ? launch_sized<0>(c, cs) : launch_sized<1>(c, cs);
  return e == cudaSuccess ? E3_OK : E3_ERR_CUDA;
}

extern "C" void e3_test_arm_project_stall(uint32_t block, uint64_t wait_ns) {
  e3::g_stall_wait_ns.store(wait_ns);
  e3::g_stall.store(block);
}
