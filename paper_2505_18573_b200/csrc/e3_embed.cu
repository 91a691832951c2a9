// Embedding of tokens, out[t] = scale E[tok_t], and the gradient of its table, dE[v] = scale sum_{t: tok_t = v} g[t].
//
// The gradient adds in a fixed order and without atomics on floating-point values: the tokens are sorted (stable, by two digits: first by
// the upper one across tiles of tokens, then every bucket by the lower one in one CTA), the sorted positions are cut into segments of equal
// length, and a CTA adds the rows of g of a segment in 32 bits.  A token whose run lies within a segment is finished there; the others
// leave a partial sum per segment, and a last kernel adds those in order.  Rows of tokens that do not occur are zeroed by CTAs of the
// same launch that reads g, so that reads and writes share the memory; few tokens are sorted by counting, in one launch that zeroes too.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math_constants.h>
#include <stdint.h>

#include "e3.h"

namespace e3 {
namespace {

constexpr int kDigitsMost = 1024;    // buckets of the upper digit
constexpr int kLowMost = 12;         // bits of the lower digit
constexpr int kTilesMost = 512;
constexpr int64_t kVMost = int64_t(kDigitsMost) << kLowMost;
constexpr int64_t kDMost = int64_t(65535) * 64;  // (64 columns a CTA, as blockIdx.y)

template <int DT>
struct Elem;
template <>
struct Elem<0> {
  using T = float;
  static constexpr int kVec = 4;
  static __device__ __forceinline__ float get(T v) { return v; }
  static __device__ __forceinline__ T put(float v) { return v; }
};
template <>
struct Elem<1> {
  using T = __nv_bfloat16;
  static constexpr int kVec = 8;
  static __device__ __forceinline__ float get(T v) { return __bfloat162float(v); }
  static __device__ __forceinline__ T put(float v) { return __float2bfloat16_rn(v); }  // one rounding, to nearest even
};

// N consecutive elements as they lie in memory (N = one or two 16-byte vectors of them, or 1).
template <int DT, int N>
struct Raw {
  uint4 v[N / Elem<DT>::kVec];
};
template <int DT>
struct Raw<DT, 1> {
  typename Elem<DT>::T v;
};
template <int DT, int N>
__device__ __forceinline__ Raw<DT, N> load_raw(const typename Elem<DT>::T *p) {
  Raw<DT, N> r;
  if constexpr (N == 1) {
    r.v = *p;
  } else {
#pragma unroll
    for (int k = 0; k < N / Elem<DT>::kVec; ++k) r.v[k] = reinterpret_cast<const uint4 *>(p)[k];
  }
  return r;
}
template <int DT, int N>
__device__ __forceinline__ void values(const Raw<DT, N> &r, float (&x)[N]) {
  if constexpr (N == 1) {
    x[0] = Elem<DT>::get(r.v);
  } else {
#pragma unroll
    for (int k = 0; k < N / Elem<DT>::kVec; ++k) {
      const uint32_t w[4] = {r.v[k].x, r.v[k].y, r.v[k].z, r.v[k].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (DT == 0) {
          x[k * 4 + i] = __uint_as_float(w[i]);
        } else {
          x[k * 8 + 2 * i] = __uint_as_float(w[i] << 16);
          x[k * 8 + 2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
      }
    }
  }
}
template <int DT, int N>
__device__ __forceinline__ void load_n(const typename Elem<DT>::T *p, float (&v)[N]) {
  values<DT, N>(load_raw<DT, N>(p), v);
}
// STREAM: the lines are not to push others out of L2.
template <int DT, int N, bool STREAM = false>
__device__ __forceinline__ void store_n(typename Elem<DT>::T *p, const float (&v)[N]) {
  if constexpr (N == 1) {
    *p = Elem<DT>::put(v[0]);
  } else {
#pragma unroll
    for (int k = 0; k < N; k += Elem<DT>::kVec) {
      uint32_t x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (DT == 0) {
          x[i] = __float_as_uint(v[k + i]);
        } else {
          const __nv_bfloat162 h = __floats2bfloat162_rn(v[k + 2 * i], v[k + 2 * i + 1]);
          x[i] = *reinterpret_cast<const uint32_t *>(&h);
        }
      }
      const uint4 w = make_uint4(x[0], x[1], x[2], x[3]);
      if (STREAM) __stcs(reinterpret_cast<uint4 *>(p + k), w);
      else *reinterpret_cast<uint4 *>(p + k) = w;
    }
  }
}

__device__ __forceinline__ void wait_for_stream_predecessor() {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
}

// ---- lookup ------------------------------------------------------------------------------------------------------
struct EmbedParams {
  const int32_t *tok;
  const void *table;
  void *out;
  int64_t n, V, D, table_stride, out_stride;
  float scale;
  int segs, len;  // a row is cut into this many pieces of `len` vectors (a warp each, all under way at once)
};

constexpr int kEmbedWarps = 8;
constexpr int kEmbedVecs = 8;  // vectors of a lane

// scale times the entries of a vector, rounded once.
template <int DT>
__device__ __forceinline__ uint4 scaled(const uint4 &v, float2 scale) {
  uint32_t w[4] = {v.x, v.y, v.z, v.w};
  if (DT == 0) {
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
      const float2 x = __fmul2_rn(make_float2(__uint_as_float(w[i]), __uint_as_float(w[i + 1])), scale);
      w[i] = __float_as_uint(x.x);
      w[i + 1] = __float_as_uint(x.y);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 x = __fmul2_rn(make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u)), scale);
      const __nv_bfloat162 h = __floats2bfloat162_rn(x.x, x.y);
      w[i] = *reinterpret_cast<const uint32_t *>(&h);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// A warp takes a piece of a row, eight vectors a lane: bound by the two moves of the row through memory, the token's number has to come first.
// 131,072 tokens of 1,536 bf16 entries, a third of them frequent ones: 85 us; with four vectors a lane (a row in two pieces) 101, with 32 registers, which
// eight CTAs an SM leave and which spill, 114.  The rows of frequent tokens stay in L2 if the vectors pass by it (plain stores: 88).  Tokens at random, none
// twice: the copy rate.
template <int DT, int N>
__global__ void __launch_bounds__(kEmbedWarps * 32, 4) embed_kernel(const __grid_constant__ EmbedParams p) {
  using E = Elem<DT>;
  using T = typename E::T;
  wait_for_stream_predecessor();
  const int lane = threadIdx.x & 31;
  for (int seg = blockIdx.y; seg < p.segs; seg += gridDim.y) {
    const int64_t first = (int64_t)seg * p.len, vecs = p.D / N - first;  // of this piece and those behind it
    const int left = (int)(vecs < p.len ? vecs : p.len) - lane;
    for (int64_t t = (int64_t)blockIdx.x * kEmbedWarps + (threadIdx.x >> 5); t < p.n; t += (int64_t)gridDim.x * kEmbedWarps) {
      const int64_t tok = p.tok[t];
      const bool live = (uint64_t)tok < (uint64_t)p.V;
      const T *const row = static_cast<const T *>(p.table) + (live ? tok : 0) * p.table_stride, *const src = row + (first + lane) * N;
      T *const out = static_cast<T *>(p.out) + t * p.out_stride, *const dst = out + (first + lane) * N;
      const float fill = tok == -1 ? 0.f : CUDART_NAN_F;
      if constexpr (N == 1) {
        T v[kEmbedVecs];
#pragma unroll
        for (int k = 0; k < kEmbedVecs; ++k)
          if (live && k * 32 < left) v[k] = src[k * 32];
#pragma unroll
        for (int k = 0; k < kEmbedVecs; ++k)
          if (k * 32 < left) dst[k * 32] = E::put(live ? E::get(v[k]) * p.scale : fill);
      } else {
        uint4 v[kEmbedVecs];
#pragma unroll
        for (int k = 0; k < kEmbedVecs; ++k)
          if (live && k * 32 < left) v[k] = reinterpret_cast<const uint4 *>(src)[k * 32];
        if (live) {
          const float2 scale = make_float2(p.scale, p.scale);
#pragma unroll
          for (int k = 0; k < kEmbedVecs; ++k)
            if (k * 32 < left) __stcs(reinterpret_cast<uint4 *>(dst) + k * 32, scaled<DT>(v[k], scale));
        } else {
          float x[N];
#pragma unroll
          for (int i = 0; i < N; ++i) x[i] = fill;
#pragma unroll 1
          for (int k = 0; k * 32 < left; ++k) store_n<DT, N, true>(dst + k * 32 * N, x);
        }
        // entries behind the last whole vector
        const int64_t e = p.D / N * N + lane;
        if (seg == p.segs - 1 && e < p.D) out[e] = E::put(live ? E::get(row[e]) * p.scale : fill);
      }
    }
  }
}

// ---- sorting -----------------------------------------------------------------------------------------------------
struct SortParams {
  const int32_t *tok;
  int64_t n, V;
  int low;               // bits of the lower digit
  int digits;            // values of the upper one
  int tiles;
  int64_t tile;          // tokens of a tile
  int32_t *counts;       // [tiles][digits]
  int32_t *bases;        // [digits + 1]: first place of every value of the upper digit
  uint2 *pairs;          // by the upper digit: (token, position)
  int32_t *keys, *perm;  // sorted: tokens, positions
  int32_t *start;        // [V + 1]: first sorted position of every token
};

constexpr int kCountThreads = 256;
__global__ void __launch_bounds__(kCountThreads) count_kernel(const __grid_constant__ SortParams p) {
  __shared__ int32_t hist[kDigitsMost];
  for (int d = threadIdx.x; d < p.digits; d += kCountThreads) hist[d] = 0;
  __syncthreads();
  wait_for_stream_predecessor();
  const int64_t lo = blockIdx.x * p.tile, hi = lo + p.tile < p.n ? lo + p.tile : p.n;
  for (int64_t t = lo + threadIdx.x; t < hi; t += kCountThreads) {
    const int64_t tok = p.tok[t];
    if ((uint64_t)tok < (uint64_t)p.V) atomicAdd(&hist[tok >> p.low], 1);
  }
  __syncthreads();
  for (int d = threadIdx.x; d < p.digits; d += kCountThreads) p.counts[(int64_t)blockIdx.x * p.digits + d] = hist[d];
}

// Exclusive sums of x[0..n) in place, by a whole CTA; returns the total.  `sh`: 32 words.
__device__ __forceinline__ int32_t scan_in_place(int32_t *x, int n, int32_t *sh) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  int32_t carry = 0;
  for (int base = 0; base < n; base += (int)blockDim.x) {
    const int i = base + (int)threadIdx.x;
    const int32_t own = i < n ? x[i] : 0;
    int32_t v = own;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int32_t up = __shfl_up_sync(0xffffffffu, v, o);
      if (lane >= o) v += up;
    }
    if (lane == 31) sh[warp] = v;
    __syncthreads();
    if (warp == 0) {
      int32_t s = lane < warps ? sh[lane] : 0;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int32_t up = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += up;
      }
      sh[lane] = s;
    }
    __syncthreads();
    if (i < n) x[i] = carry + v - own + (warp > 0 ? sh[warp - 1] : 0);
    carry += sh[warps - 1];
    __syncthreads();
  }
  return carry;
}

// Places of a warp's entries, 32 at a time and in their order: count[d] is the next place of digit d.
__device__ __forceinline__ int32_t place_of(int32_t *count, int d, bool valid) {
  const int lane = threadIdx.x & 31;
  const uint32_t peers = __match_any_sync(0xffffffffu, valid ? d : -1);
  const int before = __popc(peers & ((1u << lane) - 1u));
  int32_t at = 0;
  if (valid) at = count[d] + before;
  __syncwarp();
  if (valid && before == 0) count[d] += __popc(peers);
  __syncwarp();
  return at;
}

constexpr int kScatterWarps = 16;  // at most: each has its own counters
constexpr int kInHand = 4;  // tokens of a lane that are fetched at once
// Bound by its chain of dependent steps, most of all the tiles' counts of a digit (a thread a digit took 10 us for 64 tiles).
__global__ void __launch_bounds__(kScatterWarps * 32) scatter_kernel(const __grid_constant__ SortParams p) {
  extern __shared__ int32_t dyn[];
  __shared__ int32_t sh[32];
  int32_t *const base = dyn;                // [digits]
  int32_t *const mine = dyn + p.digits;     // [digits]: entries in this tile's predecessors
  int32_t *const hist = dyn + 2 * p.digits; // [warps][digits]
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, threads = blockDim.x, warps = threads >> 5;
  for (int d = threadIdx.x; d < p.digits * (warps + 2); d += threads) dyn[d] = 0;
  wait_for_stream_predecessor();
  __syncthreads();
  // the warps take consecutive parts of the tile
  const int64_t part = p.tile / warps;  // a multiple of 32
  const int64_t lo = blockIdx.x * p.tile + warp * part, hi = lo + part < p.n ? lo + part : p.n;
  int32_t tok[kInHand];
#pragma unroll
  for (int k = 0; k < kInHand; ++k) tok[k] = lo + k * 32 + lane < hi ? p.tok[lo + k * 32 + lane] : -1;
  {  // four groups of threads take a quarter of the tiles each
    const int quarter = (p.tiles + 3) / 4, group = (int)threadIdx.x / (threads / 4);
    const int from = group * quarter, to = from + quarter < p.tiles ? from + quarter : p.tiles;
    for (int d = (int)threadIdx.x % (threads / 4); d < p.digits; d += threads / 4) {
      int32_t before = 0, all = 0;
#pragma unroll 8
      for (int t = from; t < to; ++t) {
        const int32_t c = p.counts[(int64_t)t * p.digits + d];
        if (t < (int)blockIdx.x) before += c;
        all += c;
      }
      atomicAdd(&base[d], all);
      atomicAdd(&mine[d], before);
    }
  }
  int32_t *const own = hist + warp * p.digits;
#pragma unroll
  for (int k = 0; k < kInHand; ++k)
    if ((uint32_t)tok[k] < (uint32_t)p.V) atomicAdd(&own[tok[k] >> p.low], 1);
  for (int64_t t = lo + kInHand * 32 + lane; t < hi; t += 32) {
    const int32_t x = p.tok[t];
    if ((uint32_t)x < (uint32_t)p.V) atomicAdd(&own[x >> p.low], 1);
  }
  __syncthreads();
  const int32_t total = scan_in_place(base, p.digits, sh);
  if (blockIdx.x == 0) {
    for (int d = threadIdx.x; d < p.digits; d += threads) p.bases[d] = base[d];
    if (threadIdx.x == 0) p.bases[p.digits] = total;
  }
  for (int d = threadIdx.x; d < p.digits; d += threads) {
    int32_t at = base[d] + mine[d];
    for (int w = 0; w < warps; ++w) {
      const int32_t c = hist[w * p.digits + d];
      hist[w * p.digits + d] = at;
      at += c;
    }
  }
  __syncthreads();
  auto place = [&](int64_t t, int32_t x) {
    const bool valid = (uint32_t)x < (uint32_t)p.V;
    const int32_t at = place_of(own, x >> p.low, valid);
    if (valid) p.pairs[at] = make_uint2((uint32_t)x, (uint32_t)t);
  };
#pragma unroll
  for (int k = 0; k < kInHand; ++k)
    if (lo + k * 32 < hi) place(lo + k * 32 + lane, tok[k]);
  for (int64_t t0 = lo + kInHand * 32; t0 < hi; t0 += 32) place(t0 + lane, t0 + lane < hi ? p.tok[t0 + lane] : -1);
}

// One CTA sorts one bucket by the lower digit.
constexpr int kBucketWarps = 32;  // at most: each has its own counters
__global__ void __launch_bounds__(kBucketWarps * 32) bucket_kernel(const __grid_constant__ SortParams p) {
  extern __shared__ int32_t dyn[];
  __shared__ int32_t sh[32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5, threads = blockDim.x;
  const int bins = 1 << p.low, bucket = blockIdx.x;
  int32_t *const total = dyn;          // [bins]
  int32_t *const hist = dyn + bins;    // [warps][bins]
  for (int d = threadIdx.x; d < bins * warps; d += threads) hist[d] = 0;
  wait_for_stream_predecessor();
  __syncthreads();
  const int32_t first = p.bases[bucket], count = p.bases[bucket + 1] - first;
  const uint2 *const pairs = p.pairs + first;
  const int32_t part = ((count + warps - 1) / warps + 31) / 32 * 32;
  const int32_t lo = warp * part < count ? warp * part : count, hi = lo + part < count ? lo + part : count;
  int32_t *const own = hist + warp * bins;
  constexpr int kRounds = 8;  // entries of a lane that are fetched at once
  uint2 e[kRounds];
  auto fetch = [&](int32_t from) {
#pragma unroll
    for (int k = 0; k < kRounds; ++k)
      if (from + k * 32 + lane < hi) e[k] = pairs[from + k * 32 + lane];
  };
  for (int32_t i0 = lo; i0 < hi; i0 += 32 * kRounds) {
    fetch(i0);
#pragma unroll
    for (int k = 0; k < kRounds; ++k)
      if (i0 + k * 32 + lane < hi) atomicAdd(&own[e[k].x & (uint32_t)(bins - 1)], 1);
  }
  __syncthreads();
  for (int d = threadIdx.x; d < bins; d += threads) {
    int32_t s = 0;
    for (int w = 0; w < warps; ++w) s += hist[w * bins + d];
    total[d] = s;
  }
  __syncthreads();
  scan_in_place(total, bins, sh);
  for (int d = threadIdx.x; d < bins; d += threads) {
    int32_t at = first + total[d];
    const int64_t v = ((int64_t)bucket << p.low) + d;
    if (v < p.V) p.start[v] = at;
    for (int w = 0; w < warps; ++w) {
      const int32_t c = hist[w * bins + d];
      hist[w * bins + d] = at;
      at += c;
    }
    if (v == p.V - 1) p.start[p.V] = at;
  }
  __syncthreads();
  for (int32_t i0 = lo; i0 < hi; i0 += 32 * kRounds) {
    if (hi - lo > 32 * kRounds) fetch(i0);  // (else they are still there)
#pragma unroll
    for (int k = 0; k < kRounds; ++k) {
      if (i0 + k * 32 >= hi) break;
      const bool valid = i0 + k * 32 + lane < hi;
      const int32_t at = place_of(own, (int)(e[k].x & (uint32_t)(bins - 1)), valid);
      if (valid) {
        p.keys[at] = (int32_t)e[k].x;
        p.perm[at] = (int32_t)e[k].y;
      }
    }
  }
}

constexpr int kZeroRows = 32;  // rows of the table that are looked at together
// Zeroes the rows v0 + b for the bits b of `which`, in 16-byte vectors whatever they begin on, L lanes a row.
template <int L>
__device__ __forceinline__ void zero_rows_by(char *out, int64_t v0, uint32_t which, int64_t D, int64_t stride, int esize) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  const int64_t bytes = D * esize;
  const int l = lane % L;
  for (int b = warp * (32 / L) + lane / L; b < kZeroRows; b += warps * (32 / L)) {
    if ((which >> b & 1u) == 0u) continue;
    char *const row = out + (v0 + b) * stride * esize;
    int64_t head = (16 - (int64_t)(reinterpret_cast<uintptr_t>(row) & 15u)) & 15;
    if (head > bytes) head = bytes;
    const int64_t vecs = (bytes - head) / 16, tail = head + vecs * 16;
    uint4 *const mid = reinterpret_cast<uint4 *>(row + head);
    for (int64_t i = l; i < vecs; i += L) __stcs(mid + i, make_uint4(0u, 0u, 0u, 0u));
#pragma unroll
    for (int i = l; i < 16; i += L) {  // fewer than eight entries before and behind
      const int64_t at = i < 8 ? i * esize : tail + (i - 8) * esize;
      if (i < 8 ? at >= head : at >= bytes) continue;
      if (esize == 4) *reinterpret_cast<uint32_t *>(row + at) = 0u;
      else *reinterpret_cast<uint16_t *>(row + at) = 0;
    }
  }
}

// (A warp a row of 64 bytes took three times as long for a table of 2^22 of them.)
__device__ __forceinline__ void zero_rows(char *out, int64_t v0, uint32_t which, int64_t D, int64_t stride, int esize) {
  if (D * esize > 512) zero_rows_by<32>(out, v0, which, D, stride, esize);
  else if (D * esize > 64) zero_rows_by<8>(out, v0, which, D, stride, esize);
  else zero_rows_by<4>(out, v0, which, D, stride, esize);
}

// ---- few tokens ---------------------------------------------------------------------------------------------------
// Up to kFew tokens are sorted by counting, for each, the tokens that come before it: n / 16 comparisons a thread, and no step waits
// for another CTA's.  The rows of tokens that do not occur are zeroed by CTAs of the same launch, which look through all tokens.
// (3,001 tokens of 1001 fp32 into 33,333 rows: 35 us for the whole gradient, 50 with the three kernels above, whose steps wait for one
// another; zeroing in the summing kernel's launch instead took 44, its row loads queueing behind the stores.  The comparisons grow with n^2: 4,096 tokens 38.8
// us and 41.0, 8,192 56.8 and 47.2; into 151,936 x 1,536 bf16 79.6 and 88.0, 94.0 and 91.5; vectors of 64, whose rows cost little, are level at 3,000 tokens,
// 4,096 28.9 and 22.1.)
constexpr int kFew = 4096;
// A CTA that zeroes looks through the tokens for groups of 32 rows: one, or as many (32 at most) as make up kZeroBytes, or short rows of a large table
// cost more looks than bytes (4,096 tokens, 2^22 rows of 16 fp32: 805 us with one).
constexpr int kZeroGroupsMost = 32, kZeroBytes = 32 * 1024;
constexpr int kRankThreads = 512, kRankEach = 16, kRankTokens = kRankThreads / kRankEach;  // threads that compare for a token, tokens of a CTA
struct FewParams {
  const int32_t *tok;
  int n;
  int64_t V;
  int32_t *keys, *perm, *live;
  // CTAs behind the first rank_ctas zero the rows of tokens that do not occur
  char *out;
  int64_t D, out_stride;
  int esize, rank_ctas, zero_groups;
};
__global__ void __launch_bounds__(kRankThreads) few_kernel(const __grid_constant__ FewParams p) {
  __shared__ __align__(16) int32_t key[kFew];
  const int tid = threadIdx.x;
  wait_for_stream_predecessor();
  if ((int)blockIdx.x >= p.rank_ctas) {
    const int rows = p.zero_groups * kZeroRows;
    const int64_t v0 = (int64_t)((int)blockIdx.x - p.rank_ctas) * rows;
    if (tid < p.zero_groups) key[tid] = 0;  // a bit a row
    __syncthreads();
#pragma unroll 4
    for (int t = tid; t < p.n; t += kRankThreads) {
      const int64_t at = (int64_t)p.tok[t] - v0;
      if ((uint64_t)at < (uint64_t)rows) atomicOr(&key[at >> 5], (int32_t)(1u << (at & 31)));
    }
    __syncthreads();
    for (int g = 0; g < p.zero_groups; ++g) {
      const int64_t v = v0 + g * kZeroRows;
      if (v >= p.V) break;
      const uint32_t there = p.V - v < kZeroRows ? (1u << (p.V - v)) - 1u : 0xffffffffu;
      zero_rows(p.out, v, ~(uint32_t)key[g] & there, p.D, p.out_stride, p.esize);
    }
    return;
  }
  constexpr int32_t kNone = 0x7fffffff;  // tokens outside the vocabulary come last
  const int vecs = (p.n + 63) / 64 * 16;  // of four keys, a multiple of kRankEach
  int valid = 0;
  for (int t = tid; t < vecs * 4; t += kRankThreads) {
    const int32_t x = t < p.n ? p.tok[t] : -1;
    const bool is = (uint32_t)x < (uint32_t)p.V;
    key[t] = is ? x : kNone;
    valid += is;
  }
  __syncthreads();
  const int i = blockIdx.x * kRankTokens + tid / kRankEach;
  const int32_t own = i < p.n ? key[i] : kNone;
  int before = 0;
#pragma unroll 4
  for (int c = tid % kRankEach; c < vecs; c += kRankEach) {
    const int4 k = *reinterpret_cast<const int4 *>(&key[4 * c]);
    const int32_t x[4] = {k.x, k.y, k.z, k.w};
#pragma unroll
    for (int h = 0; h < 4; ++h) before += x[h] < own || (x[h] == own && 4 * c + h < i);
  }
#pragma unroll
  for (int o = 1; o < kRankEach; o <<= 1) before += __shfl_xor_sync(0xffffffffu, before, o);
  if (tid % kRankEach == 0 && own != kNone) {
    p.keys[before] = own;
    p.perm[before] = i;
  }
  if (blockIdx.x == 0) {
    __syncthreads();
    if (tid == 0) key[0] = 0;
    __syncthreads();
    valid = __reduce_add_sync(0xffffffffu, valid);
    if ((tid & 31) == 0) atomicAdd(&key[0], valid);
    __syncthreads();
    if (tid == 0) *p.live = key[0];
  }
}

// ---- sums --------------------------------------------------------------------------------------------------------
struct SumParams {
  const void *g;
  void *out;
  int64_t V, D, g_stride, out_stride;
  float scale;
  int accumulate;
  const int32_t *keys, *perm;
  const int32_t *start;  // nullptr: few tokens, `live` of them
  const int32_t *live;
  float *part;     // [segments][2][D]: of the run that came from the segment before, of the one that goes on behind it
  int64_t segs;
  int seg;         // sorted positions of a segment
};

constexpr int kSegMost = 128;
constexpr int kRowsAhead = 8;  // rows of g under way per thread

template <int DO, int N>
__device__ __forceinline__ void finish(const SumParams &p, int64_t v, int64_t c, const float (&sum)[N]) {
  typename Elem<DO>::T *dst = static_cast<typename Elem<DO>::T *>(p.out) + v * p.out_stride + c;
  float r[N];
  if (p.accumulate) {
#pragma unroll
    for (int i = 0; i < N; ++i) r[i] = fmaf(sum[i], p.scale, Elem<DO>::get(dst[i]));
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) r[i] = sum[i] * p.scale;
  }
  store_n<DO, N>(dst, r);
}

// blockIdx.x: first the segments, then the CTAs that zero rows; blockIdx.y: columns.
template <int DG, int DO, int N>
__global__ void __launch_bounds__(256) sum_kernel(const __grid_constant__ SumParams p) {
  __shared__ int32_t key[kSegMost + 2], row[kSegMost];
  wait_for_stream_predecessor();
  const int64_t c = ((int64_t)blockIdx.y * blockDim.x + threadIdx.x) * N;
  if ((int64_t)blockIdx.x >= p.segs) {
    if (blockIdx.y > 0) return;
    const int64_t v0 = ((int64_t)blockIdx.x - p.segs) * kZeroRows, v = v0 + (threadIdx.x & 31);
    const uint32_t absent = __ballot_sync(0xffffffffu, v < p.V && p.start[v] == p.start[v + 1]);
    zero_rows(static_cast<char *>(p.out), v0, absent, p.D, p.out_stride, DO == 0 ? 4 : 2);
    return;
  }
  const int64_t m = p.start != nullptr ? p.start[p.V] : *p.live;
  const int64_t lo = (int64_t)blockIdx.x * p.seg;
  if (lo >= m) return;
  const int len = (int)(m - lo < p.seg ? m - lo : p.seg);
  for (int i = threadIdx.x; i < len + 2; i += blockDim.x) {  // key[0]: before the segment, key[len + 1]: behind it
    const int64_t at = lo - 1 + i;
    key[i] = at >= 0 && at < m ? p.keys[at] : -1;
    if (i >= 1 && i <= len) row[i - 1] = p.perm[at];
  }
  __syncthreads();
  if (c >= p.D) return;
  const typename Elem<DG>::T *const g = static_cast<const typename Elem<DG>::T *>(p.g) + c;
  float sum[N] = {};
  bool head = key[0] == key[1];  // the run in hand came from the segment before
  for (int i0 = 0; i0 < len; i0 += kRowsAhead) {
    Raw<DG, N> v[kRowsAhead];
#pragma unroll
    for (int k = 0; k < kRowsAhead; ++k)
      if (i0 + k < len) v[k] = load_raw<DG, N>(g + (int64_t)(uint32_t)row[i0 + k] * p.g_stride);
#pragma unroll
    for (int k = 0; k < kRowsAhead; ++k) {
      const int i = i0 + k;
      if (i >= len) break;
      float x[N];
      values<DG, N>(v[k], x);
#pragma unroll
      for (int j = 0; j < N; ++j) sum[j] += x[j];
      const int32_t own = key[i + 1];
      if (own != key[i + 2] || i == len - 1) {
        const bool on = own == key[i + 2];  // goes on behind the segment
        if (head || on) {
          store_n<0, N>(p.part + ((int64_t)blockIdx.x * 2 + (head ? 0 : 1)) * p.D + c, sum);
        } else {
          finish<DO, N>(p, own, c, sum);
        }
#pragma unroll
        for (int j = 0; j < N; ++j) sum[j] = 0.f;
        head = false;
      }
    }
  }
}

// Runs of several segments: the CTA of the segment where one begins adds its parts.  Four groups of threads take a quarter of them each, in order,
// and the quarters are added in order (a token that is 6 % of 131,072 has 60 parts).
constexpr int kJoinGroups = 4;
template <int DO, int N>
__global__ void __launch_bounds__(kJoinGroups * 64) join_kernel(const __grid_constant__ SumParams p) {
  __shared__ float sh[kJoinGroups - 1][64 * N];
  wait_for_stream_predecessor();
  const int64_t lo = (int64_t)blockIdx.x * p.seg, hi = lo + p.seg;
  const int64_t m = p.start != nullptr ? p.start[p.V] : *p.live;
  if (hi >= m) return;  // nothing behind this segment
  const int32_t v = p.keys[hi - 1];
  if (v != p.keys[hi] || (lo > 0 && p.keys[lo - 1] == v)) return;  // no run goes on, or it began before
  const int group = threadIdx.x >> 6, col = threadIdx.x & 63;
  const int64_t c = ((int64_t)blockIdx.y * 64 + col) * N;
  int64_t last;  // segment of the run's end
  if (p.start != nullptr) {
    last = ((int64_t)p.start[v + 1] - 1) / p.seg;
  } else {  // (at most kFew / 32 segments, fewer than the CTA has threads)
    const int64_t at = (int64_t)(blockIdx.x + 1 + threadIdx.x) * p.seg;
    last = blockIdx.x + __syncthreads_count(at < m && p.keys[at] == v);
  }
  const int64_t count = last - blockIdx.x, each = (count + kJoinGroups - 1) / kJoinGroups;
  const int64_t from = blockIdx.x + 1 + group * each, to = from + each < last + 1 ? from + each : last + 1;
  float sum[N] = {};
  if (c < p.D) {
    if (group == 0) load_n<0, N>(p.part + ((int64_t)blockIdx.x * 2 + 1) * p.D + c, sum);
#pragma unroll 8
    for (int64_t s = from; s < to; ++s) {
      float x[N];
      load_n<0, N>(p.part + s * 2 * p.D + c, x);
#pragma unroll
      for (int j = 0; j < N; ++j) sum[j] += x[j];
    }
  }
  if (group > 0) {
#pragma unroll
    for (int j = 0; j < N; ++j) sh[group - 1][col * N + j] = sum[j];
  }
  __syncthreads();
  if (group > 0 || c >= p.D) return;
#pragma unroll
  for (int g = 0; g < kJoinGroups - 1; ++g)
#pragma unroll
    for (int j = 0; j < N; ++j) sum[j] += sh[g][col * N + j];
  finish<DO, N>(p, v, c, sum);
}

// ---- host side ---------------------------------------------------------------------------------------------------
inline bool misaligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) != 0; }
inline size_t esize_of(e3_dtype dt) { return dt == E3_F32 ? 4 : 2; }
inline size_t up16(size_t b) { return (b + 15) / 16 * 16; }

struct BackwardPlan {
  int low, digits, tiles, seg;
  int64_t tile, segs;
  size_t counts, bases, pairs, keys, perm, start, part, bytes;  // offsets into the workspace
};
BackwardPlan backward_plan(int64_t n, int64_t V, int64_t D) {
  BackwardPlan b = {};
  int bits = 1;
  while ((int64_t(1) << bits) < V) ++bits;
  // (every CTA of the second kernel reads the counts of all tiles and digits, and one of the third holds counters for each of its warps)
  b.low = bits - 10 > 9 ? bits - 10 : 9;
  b.digits = (int)((V + (int64_t(1) << b.low) - 1) >> b.low);
  // 2,048 tokens a tile, more where there would be over kTilesMost of them (every CTA of the second kernel reads all counts)
  b.tile = (n + kTilesMost - 1) / kTilesMost;
  b.tile = b.tile < 2048 ? 2048 : (b.tile + 511) / 512 * 512;
  b.tiles = (int)((n + b.tile - 1) / b.tile);
  b.seg = n < 32768 ? 32 : kSegMost;  // few tokens: more CTAs, many: fewer partial sums
  b.segs = (n + b.seg - 1) / b.seg;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += up16(bytes);
    return here;
  };
  b.counts = take((size_t)b.tiles * b.digits * 4);
  b.bases = take((size_t)(b.digits + 1) * 4);
  b.pairs = take((size_t)n * 8);
  b.keys = take((size_t)n * 4);
  b.perm = take((size_t)n * 4);
  b.start = take((size_t)(V + 1) * 4);
  b.part = take((size_t)b.segs * 2 * D * 4);
  b.bytes = at;
  return b;
}

template <class... P, class... A>
cudaError_t launch_behind(void (*kern)(P...), dim3 grid, int threads, size_t smem, cudaStream_t stream, A &&...args) {
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, args...);
}

template <int DG, int DO, int N>
cudaError_t launch_sums(const SumParams &p, dim3 sums, dim3 joins, int threads, cudaStream_t stream) {
  const cudaError_t e = launch_behind(sum_kernel<DG, DO, N>, sums, threads, 0, stream, p);
  return e == cudaSuccess ? launch_behind(join_kernel<DO, N>, joins, kJoinGroups * 64, 0, stream, p) : e;
}

}  // namespace
}  // namespace e3

using namespace e3;

extern "C" e3_status e3_embed_tokens(const int32_t *tok, int64_t n, const void *table, e3_dtype dt, int64_t V, int64_t D,
                                     int64_t table_stride, float scale, void *out, int64_t out_stride, void *stream) {
  if (dt != E3_F32 && dt != E3_BF16) return E3_ERR_DTYPE;
  if (n < 0 || V < 1 || V >= (int64_t(1) << 31) || D < 1 || D >= (int64_t(1) << 31) || table_stride < D || out_stride < D)
    return E3_ERR_INVALID_ARG;
  if (n == 0) return E3_OK;
  if (!tok || !table || !out) return E3_ERR_INVALID_ARG;
  const size_t es = esize_of(dt);
  if (misaligned(tok, 4) || misaligned(table, es) || misaligned(out, es)) return E3_ERR_ALIGNMENT;
  EmbedParams p = {};
  p.tok = tok; p.table = table; p.out = out; p.n = n; p.V = V; p.D = D; p.table_stride = table_stride; p.out_stride = out_stride;
  p.scale = scale;
  // rows that all begin on a 16-byte boundary move in vectors
  const bool vec = !misaligned(table, 16) && !misaligned(out, 16) && table_stride * es % 16 == 0 && out_stride * es % 16 == 0 &&
                   D * (int64_t)es >= 16;
  const int64_t vecs = vec ? D / (int64_t)(16 / es) : D;
  p.segs = (int)((vecs + 32 * kEmbedVecs - 1) / (32 * kEmbedVecs));
  p.len = (int)(((vecs + p.segs - 1) / p.segs + 31) / 32 * 32);
  const int64_t ctas = (n + kEmbedWarps - 1) / kEmbedWarps, most = 0x7fffffff;
  const dim3 grid((unsigned)(ctas < most ? ctas : most), (unsigned)(p.segs < 65535 ? p.segs : 65535));
  const cudaError_t e = launch_behind(dt == E3_F32 ? (vec ? embed_kernel<0, 4> : embed_kernel<0, 1>) : (vec ? embed_kernel<1, 8> : embed_kernel<1, 1>),
                                      grid, kEmbedWarps * 32, 0, static_cast<cudaStream_t>(stream), p);
  return e == cudaSuccess ? E3_OK : E3_ERR_CUDA;
}

extern "C" size_t e3_embed_workspace_bytes(int64_t n, int64_t V, int64_t D) {
  if (n <= 0 || n >= (int64_t(1) << 31) || V < 1 || V > kVMost || D < 1 || D > kDMost) return 0;
  return backward_plan(n, V, D).bytes;
}

extern "C" e3_status e3_embed_tokens_backward(const int32_t *tok, int64_t n, const void *g, e3_dtype dt, int64_t V, int64_t D,
                                              int64_t g_stride, float scale, void *dtable, e3_dtype table_dt,
                                              int64_t dtable_stride, int accumulate, void *workspace, size_t workspace_bytes,
                                              void *stream) {
  if ((dt != E3_F32 && dt != E3_BF16) || (table_dt != E3_F32 && table_dt != E3_BF16)) return E3_ERR_DTYPE;
  if (n < 0 || n >= (int64_t(1) << 31) || V < 1 || V > kVMost || D < 1 || D > kDMost || dtable_stride < D || (n > 0 && g_stride < D))
    return E3_ERR_INVALID_ARG;
  if (n == 0 && accumulate) return E3_OK;
  if (!dtable || (n > 0 && (!tok || !g))) return E3_ERR_INVALID_ARG;
  const size_t es = esize_of(dt), eo = esize_of(table_dt);
  if (misaligned(tok, 4) || misaligned(g, es) || misaligned(dtable, eo) || misaligned(workspace, 16)) return E3_ERR_ALIGNMENT;
  cudaStream_t cs = static_cast<cudaStream_t>(stream);
  if (n == 0) {
    const cudaError_t e = cudaMemset2DAsync(dtable, (size_t)dtable_stride * eo, 0, (size_t)D * eo, (size_t)V, cs);
    return e == cudaSuccess ? E3_OK : E3_ERR_CUDA;
  }
  const BackwardPlan b = backward_plan(n, V, D);
  if (!workspace || workspace_bytes < b.bytes) return E3_ERR_WORKSPACE;
  char *const ws = static_cast<char *>(workspace);

  int32_t *const keys = reinterpret_cast<int32_t *>(ws + b.keys), *const perm = reinterpret_cast<int32_t *>(ws + b.perm);
  int32_t *const live = reinterpret_cast<int32_t *>(ws + b.bases), *const start = reinterpret_cast<int32_t *>(ws + b.start);
  const bool few = n <= kFew;
  cudaError_t e = cudaSuccess;
  if (few) {
    FewParams f = {};
    f.tok = tok; f.n = (int)n; f.V = V; f.keys = keys; f.perm = perm; f.live = live;
    f.out = static_cast<char *>(dtable); f.D = D; f.out_stride = dtable_stride; f.esize = table_dt == E3_BF16 ? 2 : 4;
    const int64_t group = kZeroRows * D * f.esize, groups = kZeroBytes / group;
    f.zero_groups = (int)(groups < 1 ? 1 : (groups > kZeroGroupsMost ? kZeroGroupsMost : groups));
    const int rows = f.zero_groups * kZeroRows;
    const int64_t zero_ctas = accumulate ? 0 : (V + rows - 1) / rows;
    f.rank_ctas = (int)((n + kRankTokens - 1) / kRankTokens);
    e = launch_behind(few_kernel, dim3((unsigned)(f.rank_ctas + zero_ctas)), kRankThreads, 0, cs, f);
  } else {
    SortParams s = {};
    s.tok = tok; s.n = n; s.V = V; s.low = b.low; s.digits = b.digits; s.tiles = b.tiles; s.tile = b.tile;
    s.counts = reinterpret_cast<int32_t *>(ws + b.counts);
    s.bases = reinterpret_cast<int32_t *>(ws + b.bases);
    s.pairs = reinterpret_cast<uint2 *>(ws + b.pairs);
    s.keys = keys; s.perm = perm; s.start = start;
    e = launch_behind(count_kernel, dim3((unsigned)b.tiles), kCountThreads, 0, cs, s);
    if (e == cudaSuccess) {
      const int warps = b.digits <= 640 ? kScatterWarps : kScatterWarps / 2;  // (counters of 46 KB at most)
      e = launch_behind(scatter_kernel, dim3((unsigned)b.tiles), warps * 32, (size_t)(warps + 2) * b.digits * 4, cs, s);
    }
    if (e == cudaSuccess) {
      // as many warps as have their own counters in 46 KB
      int warps = (int)(46 * 1024 / 4 / (1 << b.low)) - 1;
      warps = warps > kBucketWarps ? kBucketWarps : (warps < 1 ? 1 : warps);
      e = launch_behind(bucket_kernel, dim3((unsigned)b.digits), warps * 32, (size_t)(warps + 1) * (1u << b.low) * 4, cs, s);
    }
  }
  if (e != cudaSuccess) return E3_ERR_CUDA;

  SumParams p = {};
  p.g = g; p.out = dtable; p.V = V; p.D = D; p.g_stride = g_stride; p.out_stride = dtable_stride; p.scale = scale;
  p.accumulate = accumulate != 0; p.keys = keys; p.perm = perm; p.start = few ? nullptr : start; p.live = live;
  p.part = reinterpret_cast<float *>(ws + b.part); p.segs = b.segs; p.seg = b.seg;
  // vectors of 16 bytes of the narrower type, if all rows begin on a 16-byte boundary and hold whole vectors
  const int n_vec = dt == E3_BF16 || table_dt == E3_BF16 ? 8 : 4;
  const bool vec = !misaligned(g, 16) && !misaligned(dtable, 16) && g_stride * es % 16 == 0 && dtable_stride * eo % 16 == 0 && D % n_vec == 0;
  const int64_t vecs = vec ? D / n_vec : D;
  const int64_t cols = (vecs + 255) / 256;
  const int threads = (int)(((vecs + cols - 1) / cols + 31) / 32 * 32);
  const dim3 sums((unsigned)(b.segs + (few || accumulate ? 0 : (V + kZeroRows - 1) / kZeroRows)), (unsigned)cols), joins((unsigned)b.segs, (unsigned)((vecs + 63) / 64));
  if (dt == E3_F32 && table_dt == E3_F32)
    e = vec ? launch_sums<0, 0, 4>(p, sums, joins, threads, cs) : launch_sums<0, 0, 1>(p, sums, joins, threads, cs);
  else if (dt == E3_F32)
    e = vec ? launch_sums<0, 1, 8>(p, sums, joins, threads, cs) : launch_sums<0, 1, 1>(p, sums, joins, threads, cs);
  else if (table_dt == E3_F32)
    e = vec ? launch_sums<1, 0, 8>(p, sums, joins, threads, cs) : launch_sums<1, 0, 1>(p, sums, joins, threads, cs);
  else
    e = vec ? launch_sums<1, 1, 8>(p, sums, joins, threads, cs) : launch_sums<1, 1, 1>(p, sums, joins, threads, cs);
  return e == cudaSuccess ? E3_OK : E3_ERR_CUDA;
}
