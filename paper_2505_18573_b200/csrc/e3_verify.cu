// Verification of drafted tokens: which drafts of every sequence are kept, and the token that follows them.
//
// p_j = softmax(z_j / tau) of the target at position j, q_j the draft's distribution there.  Draft d_j is kept iff u_j q_j(d_j) < p_j(d_j);
// at the first position a that is refused the token comes from max(p_a - q_a, 0), behind a sequence whose drafts were all kept from p_a.
//
// Two passes.  verify_rows_kernel takes the rows position by position (every sequence's first row, then every second, ...), a row in parts
// of equal length, one CTA each: the part's largest logit R, Z = sum 2^t and W = sum 2^t (z - R) with t = (z - R) log2(e) / tau.  The CTA that
// comes last to a row joins the parts in their order and decides; rows behind a refused position are not read any more once that is known
// (which changes no result).  draw_kernel gives every sequence a cluster of CTAs that reads the one row (and the draft's) the token comes from.
//
// The token comes from the construction of the blocked sampler with given uniforms, one per block of 256 entries: the block with the largest
// ln(sum r_i) - ln(-ln u_b), then the first entry in it whose prefix sum exceeds v times its sum.  Two tokens are the same only if every
// comparison falls the same way, so each is made with a bound on the error of fp32 sums; what the bound does not settle (a few in
// 10,000) is taken again in fp64, over the whole row.
#include "e3_rows_device.cuh"

#include <cooperative_groups.h>

#include <atomic>

#include "e3.h"

namespace cg = cooperative_groups;

namespace e3 {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kPartsMost = 32;
constexpr int kClusterMost = 8;
constexpr unsigned kAll = 0xffffffffu;
// Relative error of p and q, as sums over a block in fp32 (2^t: 2^-22 and the rounding of t) and through Z.
constexpr float kSumError = 5e-6f;
constexpr float kSumErrorPerBit = 1.5e-7f;  // per factor of two by which the sum, or the draft's own q, lies below 1 (rounding of t)
constexpr double kZError = 1e-5;

enum : int { kKept = 0, kRefused = 1, kInvalid = 2 };

struct VerifyPart {
  float R, Z, W;
  int err;
  int best;  // greedy rows: index of R
  int pad[3];
};
struct VerifyRow {
  double lnZ;
  float R, ent, logp;  // logp: of the draft
  int state, best, pad;
};
static_assert(sizeof(VerifyPart) == 32 && sizeof(VerifyRow) == 32, "records");

struct VerifyParams {
  const char *logits, *draft_logits;
  int64_t row_bytes, draft_row_bytes;
  int64_t n_seq, drafts;  // drafts: of a sequence at most
  int V, blocks;
  const float *temps, *draft_temps, *draft_logp;
  const int32_t *draft_tok, *draft_len;
  const double *uniforms;
  int64_t u_stride;
  int32_t *out_tok, *out_kept;
  float *out_logp, *out_ent;
  int32_t *first, *arrived;  // workspace: first position not kept, parts of a row that have come
  VerifyRow *rows;
  VerifyPart *parts;
  int n_parts, part;  // parts of a row, entries of one
};

__device__ __forceinline__ void wait_for_stream_predecessor() {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
}
__device__ __forceinline__ int length_of(const VerifyParams &p, int64_t b) {
  const int64_t n = p.draft_len != nullptr ? (int64_t)p.draft_len[b] : p.drafts;
  return (int)(n < 0 ? 0 : (n < p.drafts ? n : p.drafts));
}
__device__ __forceinline__ bool usable_uniform(double u) { return u >= 0.0 && u < 1.0; }
__device__ __forceinline__ float max_nan(float a, float b) {
  float m;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(b));
  return m;
}
__device__ __forceinline__ f2 mul2(f2 a, f2 b) { return __fmul2_rn(a, b); }

// What is known of the draft at a position.
enum : int { kNoDraft = 0, kOneHot = 1, kDistribution = 2 };  // kNoDraft: none that can be used; the position is refused, the draw is from p
struct Draft {
  int kind, tok;
  float y, tau;  // its logit, the draft's temperature
  double lnq;
};
template <int DT>
__device__ __forceinline__ Draft draft_of(const VerifyParams &p, int64_t b, int64_t j) {
  Draft d = {kNoDraft, -1, 0.f, 0.f, 0.0};
  const int64_t at = b * p.drafts + j;
  const int tok = p.draft_tok[at];
  if ((uint32_t)tok >= (uint32_t)p.V) return d;
  d.tok = tok;
  if (p.draft_logits == nullptr) {
    d.kind = kOneHot;
    return d;
  }
  d.tau = p.draft_temps != nullptr ? p.draft_temps[b] : p.temps[b];
  if (d.tau == 0.f) {
    d.kind = kOneHot;
    return d;
  }
  d.lnq = (double)p.draft_logp[at];
  d.y = load_elem<DT>(p.draft_logits + at * p.draft_row_bytes, tok);
  if (d.tau > 0.f && d.tau < CUDART_INF_F && fabsf(d.y) < CUDART_INF_F && d.lnq < 1.0) d.kind = kDistribution;
  return d;
}

// ---- first pass ----------------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(256) begin_kernel(const __grid_constant__ VerifyParams p) {
  wait_for_stream_predecessor();
  const int64_t rows = p.n_seq * (p.drafts + 1);
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows; i += (int64_t)gridDim.x * 256) {
    p.arrived[i] = 0;
    if (i < p.n_seq) p.first[i] = INT_MAX;
  }
}

// Entries of a vector outside [0, n) become -inf; the vector's first entry has number e.
template <int DT>
__device__ __forceinline__ uint4 keep_entries(const uint4 &v, int e, int n) {
  constexpr int kE = DT == 0 ? 4 : 8;
  if (e >= 0 && e + kE <= n) return v;
  uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (DT == 0) {
      if (e + i < 0 || e + i >= n) w[i] = 0xFF800000u;
    } else {
      if (e + 2 * i < 0 || e + 2 * i >= n) w[i] = (w[i] & 0xFFFF0000u) | 0xFF80u;
      if (e + 2 * i + 1 < 0 || e + 2 * i + 1 >= n) w[i] = (w[i] & 0xFFFFu) | 0xFF800000u;
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
template <int DT>
__device__ __forceinline__ f2 pair_of(const uint4 &v, int j) {  // entries 2j and 2j + 1
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  if (DT == 1) return pack2f(__uint_as_float(w[j] << 16), __uint_as_float(w[j] & 0xFFFF0000u));
  return pack2f(__uint_as_float(w[2 * j]), __uint_as_float(w[2 * j + 1]));
}
// Largest entry; NaN if one is.
template <int DT>
__device__ __forceinline__ float most_of(const uint4 &v) {
  if (DT == 1) {
    uint32_t a, b;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(v.x), "r"(v.y));
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(b) : "r"(v.z), "r"(v.w));
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(a), "r"(b));
    return max_nan(__uint_as_float(a << 16), __uint_as_float(a & 0xFFFF0000u));
  }
  return max_nan(max_nan(__uint_as_float(v.x), __uint_as_float(v.y)), max_nan(__uint_as_float(v.z), __uint_as_float(v.w)));
}

struct Sums {
  float R, Z, W;
};
// Joins two sums; either may be empty (R = -inf).
__device__ __forceinline__ void join(Sums &a, float R, float Z, float W, float c) {
  const float m = fmaxf(a.R, R);
  if (m == -CUDART_INF_F) return;
  const float da = a.R > -CUDART_INF_F ? fmaxf(a.R - m, -1e30f) : -1e30f, db = R > -CUDART_INF_F ? fmaxf(R - m, -1e30f) : -1e30f;
  const float fa = a.Z > 0.f ? ex2f(da * c) : 0.f, fb = Z > 0.f ? ex2f(db * c) : 0.f;
  a.W = (fa > 0.f ? fa * fmaf(da, a.Z, a.W) : 0.f) + (fb > 0.f ? fb * fmaf(db, Z, W) : 0.f);
  a.Z = fa * a.Z + fb * Z;
  a.R = m;
}

// sum over the row of exp((z - R) / tau) in fp64, of the entries from `from` on in steps of `step`, by one thread.
template <int DT>
__device__ __noinline__ double exact_terms(const char *row, int V, float R, float tau, int from, int step) {
  double s = 0.0;
  for (int i = from; i < V; i += step) s += exp(((double)load_elem<DT>(row, i) - (double)R) / (double)tau);
  return s;
}
__device__ __forceinline__ double block_sum(double v, double *sh /* [warps] */) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kAll, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
  __syncthreads();
  v = 0.0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) v += sh[w];
  return v;
}

template <int DT>
__global__ void __launch_bounds__(kThreads, 4) verify_rows_kernel(const __grid_constant__ VerifyParams p) {
  constexpr int kE = DT == 0 ? 4 : 8;  // entries of a vector
  constexpr int kEsize = DT == 0 ? 4 : 2;
  constexpr int kAhead = 8;            // vectors under way per thread
  __shared__ Sums sh[kWarps];
  __shared__ int sh_best[kWarps], sh_bad[kWarps];
  __shared__ double sh_sum[kWarps];
  __shared__ int sh_flag;
  __shared__ VerifyRow sh_row;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t item = blockIdx.x;
  const int64_t at = item / p.n_parts;
  const int part = (int)(item - at * p.n_parts);
  const int64_t j = at / p.n_seq, b = at - j * p.n_seq, r = b * (p.drafts + 1) + j;
  wait_for_stream_predecessor();
  const int len = length_of(p, b);
  if (j > len) return;
  if (j > 0 && __syncthreads_or(tid == 0 && *(volatile const int32_t *)(p.first + b) < j)) return;

  const char *const row = p.logits + r * p.row_bytes;
  const float tau = p.temps[b];
  const bool greedy = tau == 0.f, usable = greedy || (tau > 0.f && tau < CUDART_INF_F);
  const float c = greedy || !usable ? 0.f : __fdiv_rn(kLog2e, tau);
  const int e0 = part * p.part, n = p.V - e0 < p.part ? p.V - e0 : p.part;
  Sums s = {-CUDART_INF_F, 0.f, 0.f};
  bool bad = !usable || !(c < CUDART_INF_F);
  int best = INT_MAX;
  if (usable) {
    const char *const begin = row + (int64_t)e0 * kEsize;
    const int a = (int)(reinterpret_cast<uintptr_t>(begin) & 15u), skip = a / kEsize;
    const uint4 *const src = reinterpret_cast<const uint4 *>(begin - a);
    const int vecs = (skip + n + kE - 1) / kE;
    f2 Z2 = pack2f(0.f, 0.f), W2 = Z2;
    for (int i0 = tid; i0 < vecs; i0 += kThreads * kAhead) {
      uint4 v[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int i = i0 + k * kThreads;
        if (i < vecs) v[k] = __ldcs(src + i);
      }
      float m = -CUDART_INF_F;
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int i = i0 + k * kThreads;
        if (i < vecs) {
          v[k] = keep_entries<DT>(v[k], i * kE - skip, n);
          m = max_nan(m, most_of<DT>(v[k]));
        }
      }
      bad |= !(m < CUDART_INF_F);
      if (greedy) {
        if (m > s.R) {
          s.R = m;
          best = -1;
        }
        if (best < 0) {  // lowest entry of this round with that logit
#pragma unroll
          for (int k = kAhead - 1; k >= 0; --k) {
            const int i = i0 + k * kThreads;
            if (i < vecs) {
#pragma unroll
              for (int h = kE / 2 - 1; h >= 0; --h) {
                const f2 z = pair_of<DT>(v[k], h);
                if (z.y == m) best = e0 + i * kE - skip + 2 * h + 1;
                if (z.x == m) best = e0 + i * kE - skip + 2 * h;
              }
            }
          }
          if (best < 0) best = INT_MAX;  // (NaN: the row is invalid)
        }
        continue;
      }
      if (!(m > -CUDART_INF_F)) continue;
      if (m > s.R) {
        if (s.R > -CUDART_INF_F) {
          const float d = fmaxf(s.R - m, -1e30f), f = ex2f(d * c);
          const f2 d2 = pack2f(d, d), f2f = pack2f(f, f);
          W2 = mul2(f2f, fma2(d2, Z2, W2));
          Z2 = mul2(f2f, Z2);
        }
        s.R = m;
      }
      const f2 nR = pack2f(-s.R, -s.R), c2 = pack2f(c, c);
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        if (i0 + k * kThreads < vecs) {
#pragma unroll
          for (int h = 0; h < kE / 2; ++h) {
            f2 d = add2(pair_of<DT>(v[k], h), nR);
            d = pack2f(fmaxf(d.x, -1e30f), fmaxf(d.y, -1e30f));  // (-inf: weight 0, and 0 times its distance is 0)
            const f2 t = mul2(d, c2), e = pack2f(ex2f(t.x), ex2f(t.y));
            Z2 = add2(Z2, e);
            W2 = fma2(e, d, W2);
          }
        }
      }
    }
    s.Z = sum2(Z2);
    s.W = sum2(W2);
  }
  // ---- the part's result, joined in a fixed order
  if (greedy) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const float R = __shfl_xor_sync(kAll, s.R, o);
      const int i = __shfl_xor_sync(kAll, best, o);
      if (R > s.R || (R == s.R && i < best)) {
        s.R = R;
        best = i;
      }
    }
  } else {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const float R = __shfl_xor_sync(kAll, s.R, o), Z = __shfl_xor_sync(kAll, s.Z, o), W = __shfl_xor_sync(kAll, s.W, o);
      join(s, R, Z, W, c);
    }
  }
  bad = __any_sync(kAll, bad);
  if (lane == 0) {
    sh[warp] = s;
    sh_best[warp] = best;
    sh_bad[warp] = bad;
  }
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < kWarps; ++w) {
      if (greedy) {
        if (sh[w].R > s.R || (sh[w].R == s.R && sh_best[w] < best)) {
          s.R = sh[w].R;
          best = sh_best[w];
        }
      } else {
        join(s, sh[w].R, sh[w].Z, sh[w].W, c);
      }
      bad |= sh_bad[w] != 0;
    }
    VerifyPart out = {s.R, s.Z, s.W, bad ? 1 : 0, best, {0, 0, 0}};
    p.parts[r * p.n_parts + part] = out;
    __threadfence();
    sh_flag = atomicAdd(p.arrived + r, 1) == p.n_parts - 1;
    __threadfence();
  }
  __syncthreads();
  if (!sh_flag) return;

  // ---- the last CTA of the row: all parts are there
  Draft d = {kNoDraft, -1, 0.f, 0.f, 0.0};
  if (j < len) d = draft_of<DT>(p, b, j);
  if (warp == 0) {
    VerifyPart q = {-CUDART_INF_F, 0.f, 0.f, 0, INT_MAX, {0, 0, 0}};
    if (lane < p.n_parts) {  // (written by other SMs: from L2)
      const int4 *const src = reinterpret_cast<const int4 *>(p.parts + r * p.n_parts + lane);
      const int4 x = __ldcg(src), y = __ldcg(src + 1);
      q.R = __int_as_float(x.x); q.Z = __int_as_float(x.y); q.W = __int_as_float(x.z); q.err = x.w;
      q.best = y.x;
    }
    s = {q.R, q.Z, q.W};
    best = q.best;
    bad = __any_sync(kAll, q.err != 0);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const float R = __shfl_xor_sync(kAll, s.R, o), Z = __shfl_xor_sync(kAll, s.Z, o), W = __shfl_xor_sync(kAll, s.W, o);
      const int i = __shfl_xor_sync(kAll, best, o);
      if (greedy) {
        if (R > s.R || (R == s.R && i < best)) {
          s.R = R;
          best = i;
        }
      } else {
        join(s, R, Z, W, c);
      }
    }
    if (lane == 0) {
      VerifyRow w = {0.0, s.R, 0.f, 0.f, kRefused, best, 0};
      const double u = j < len ? p.uniforms[b * p.u_stride + j] : 0.0;
      bool near = false;
      if (bad || !(s.R > -CUDART_INF_F) || (!greedy && !(s.Z > 0.f)) || !usable_uniform(u)) {
        w.state = kInvalid;
      } else if (greedy) {
        if (d.kind != kNoDraft && d.tok == best && u * exp(d.lnq) < 1.0) w.state = kKept;
      } else {
        w.lnZ = log((double)s.Z);
        w.ent = (float)fmax(w.lnZ - (double)s.W / ((double)s.Z * (double)tau), 0.0);
        if (d.kind != kNoDraft) {
          const double x = ((double)load_elem<DT>(row, d.tok) - (double)s.R) / (double)tau, lp = x - w.lnZ;
          const double ratio = u * exp(d.lnq - lp);  // (a token of probability 0: infinity or, from u = 0, NaN)
          w.logp = (float)lp;
          w.state = ratio < 1.0 ? kKept : kRefused;
          near = fabs(ratio - 1.0) < kZError;
        }
      }
      sh_row = w;
      sh_flag = near;
    }
  }
  __syncthreads();
  if (sh_flag) {  // u q and p are closer than Z is known
    const double total = block_sum(exact_terms<DT>(row, p.V, sh_row.R, tau, tid, kThreads), sh_sum);
    if (tid == 0) {
      sh_row.lnZ = log(total);
      const double lp = ((double)load_elem<DT>(row, d.tok) - (double)sh_row.R) / (double)tau - sh_row.lnZ;
      sh_row.logp = (float)lp;
      sh_row.state = p.uniforms[b * p.u_stride + j] * exp(d.lnq) < exp(lp) ? kKept : kRefused;
    }
  }
  if (tid == 0) {
    p.rows[r] = sh_row;
    if (sh_row.state != kKept) {
      __threadfence();
      atomicMin(p.first + b, (int32_t)j);
    }
  }
}

// ---- second pass ---------------------------------------------------------------------------------------------------
// Leading blocks: the largest lower bound of a score, the two largest upper bounds.
struct Lead {
  float lo, hi1, hi2;
  int lo_b, hi_b, bad;
};
__device__ __forceinline__ void insert(Lead &l, float lo, float hi, int b) {
  if (lo > l.lo) {
    l.lo = lo;
    l.lo_b = b;
  }
  if (hi > l.hi1) {
    l.hi2 = l.hi1;
    l.hi1 = hi;
    l.hi_b = b;
  } else if (hi > l.hi2) {
    l.hi2 = hi;
  }
}
__device__ __forceinline__ void merge(Lead &l, const Lead &o) {
  if (o.lo > l.lo || (o.lo == l.lo && o.lo_b < l.lo_b)) {
    l.lo = o.lo;
    l.lo_b = o.lo_b;
  }
  if (o.hi1 > l.hi1) {
    l.hi2 = fmaxf(l.hi1, o.hi2);
    l.hi1 = o.hi1;
    l.hi_b = o.hi_b;
  } else {
    l.hi2 = fmaxf(l.hi2, o.hi1);
  }
  l.bad |= o.bad;
}
__device__ __forceinline__ Lead no_lead() { return Lead{-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, INT_MAX, INT_MAX, 0}; }

// Gumbel variate -ln(-ln u) of a uniform, good to a few units of fp32.
__device__ __forceinline__ float gumbel_of(double u) {
  const float w = u < 0.5 ? (u > 1e-30 ? -logf((float)u) : (float)-log(u)) : -log1pf((float)(u - 1.0));
  return -logf(w);
}

// The row a token is drawn from.
struct DrawRow {
  const char *z, *y;   // target, draft (kDistribution)
  int V, kind, d;
  float tau, R, y_d, tau_d;
  double lnZ, lnq;
};
// The eight entries from i on (i a multiple of 8; a block's entries of a lane) as vectors, whatever the row's alignment.
template <int DT>
struct Eight {
  uint4 v[DT == 0 ? 2 : 1];
};
template <int DT>
__device__ __forceinline__ Eight<DT> load_eight(const char *row, int V, int i) {
  constexpr int kEsize = DT == 0 ? 4 : 2, N = DT == 0 ? 2 : 1;
  Eight<DT> e;
  const char *const at = row + (int64_t)i * kEsize, *const end = row + (int64_t)V * kEsize;
  const uint32_t a = (uint32_t)(reinterpret_cast<uintptr_t>(at) & 15u);
  const uint4 none = make_uint4(0u, 0u, 0u, 0u);
  if (a == 0u) {
#pragma unroll
    for (int k = 0; k < N; ++k) e.v[k] = at + 16 * k < end ? *reinterpret_cast<const uint4 *>(at + 16 * k) : none;
  } else {
    uint4 x = at < end ? *reinterpret_cast<const uint4 *>(at - a) : none;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const uint4 y = at - a + 16 * (k + 1) < end ? *reinterpret_cast<const uint4 *>(at - a + 16 * (k + 1)) : none;
      e.v[k] = shift_vec(x, y, a);
      x = y;
    }
  }
  return e;
}
template <int DT>
__device__ __forceinline__ float entry(const Eight<DT> &e, int k) {
  const uint4 &v = e.v[DT == 0 ? k >> 2 : 0];
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  if (DT == 0) return __uint_as_float(w[k & 3]);
  return __uint_as_float((k & 1) != 0 ? w[k >> 1] & 0xFFFF0000u : w[k >> 1] << 16);
}

// Weight max(p - q, 0) of an entry in fp64 (q of a logit that is NaN: the entry is not drawn); mass: p.
__device__ __forceinline__ double exact_weight(const DrawRow &w, int kind, int i, float z, float y, double &mass) {
  mass = exp(((double)z - (double)w.R) / (double)w.tau - w.lnZ);
  if (kind == kNoDraft) return mass;
  if (kind == kOneHot) return i == w.d ? 0.0 : mass;
  return fmax(mass - exp(((double)y - (double)w.y_d) / (double)w.tau_d + w.lnq), 0.0);
}

// Draw inside block b by a warp.  False: the fp32 normaliser leaves open which entry it is.
template <int DT>
__device__ __noinline__ bool draw_in(const DrawRow &w, int kind, int b, double u, bool exact, int &tok) {
  const int lane = threadIdx.x & 31, i0 = b * E3_SAMPLE_BLOCK + lane * 8;
  const Eight<DT> z = load_eight<DT>(w.z, w.V, i0);
  Eight<DT> y = z;
  if (kind == kDistribution) y = load_eight<DT>(w.y, w.V, i0);
  double r[8], mass = 0.0, sum = 0.0;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    double m = 0.0;
    r[k] = i0 + k < w.V ? exact_weight(w, kind, i0 + k, entry<DT>(z, k), entry<DT>(y, k), m) : 0.0;
    sum += r[k];
    mass += m;
  }
  double before = sum;  // of the lanes up to this one, then of those before it
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const double up = __shfl_up_sync(kAll, before, o);
    if (lane >= o) before += up;
    mass += __shfl_xor_sync(kAll, mass, o);
  }
  const double total = __shfl_sync(kAll, before, 31), t = u * total;
  before = __shfl_up_sync(kAll, before, 1);
  if (lane == 0) before = 0.0;
  int first = INT_MAX, last = -1;
  bool near = false;
  const double margin = exact || kind != kDistribution ? 0.0 : kZError * mass;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    before += r[k];
    if (r[k] > 0.0) last = i0 + k;
    if (before > t && r[k] > 0.0 && first == INT_MAX) first = i0 + k;
    near |= i0 + k < w.V && fabs(before - t) <= margin && margin > 0.0;
  }
  first = __reduce_min_sync(kAll, first);
  last = __reduce_max_sync(kAll, last);
  tok = first != INT_MAX ? first : last;
  return !__any_sync(kAll, near) && tok >= 0;
}

constexpr int kBlocksAhead[2] = {2, 4};  // blocks under way per warp: fp32, bf16

// Scores of the blocks of this warp (every `step`-th from `from` on), with bounds on their errors.
template <int DT>
__device__ __forceinline__ Lead scan_blocks(const DrawRow &w, int blocks, const double *u, int from, int step) {
  constexpr int kAhead = kBlocksAhead[DT];
  const int lane = threadIdx.x & 31;
  const float c = __fdiv_rn(kLog2e, w.tau), nz = -(float)(w.lnZ / kLn2);
  const float cd = w.kind == kDistribution ? __fdiv_rn(kLog2e, w.tau_d) : 0.f, nq = w.kind == kDistribution ? (float)(w.lnq / kLn2) : 0.f;
  Lead lead = no_lead();
  float g = 0.f;
  int n = 0;
  for (int b0 = from; b0 < blocks; b0 += step * kAhead) {
    Eight<DT> z[kAhead], y[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int b = b0 + k * step;
      if (b < blocks) {
        z[k] = load_eight<DT>(w.z, w.V, b * E3_SAMPLE_BLOCK + lane * 8);
        if (w.kind == kDistribution) y[k] = load_eight<DT>(w.y, w.V, b * E3_SAMPLE_BLOCK + lane * 8);
      }
    }
    if ((n & 31) == 0) {  // the variates of the next 32 blocks, one a lane
      const int64_t b = b0 + (int64_t)lane * step;
      const double ub = b < blocks ? u[b] : 0.5;
      if (!usable_uniform(ub)) lead.bad = 1;
      g = gumbel_of(ub);
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int b = b0 + k * step;
      if (b >= blocks) break;
      const int i0 = b * E3_SAMPLE_BLOCK + lane * 8;
      float r = 0.f, s = 0.f;
#pragma unroll
      for (int h = 0; h < 8; ++h) {
        const float zk = i0 + h < w.V ? entry<DT>(z[k], h) : -CUDART_INF_F;
        const float e = ex2f(fmaf(zk - w.R, c, nz));
        float q = 0.f;
        if (w.kind == kDistribution) q = i0 + h < w.V ? ex2f(fmaf(entry<DT>(y[k], h) - w.y_d, cd, nq)) : 0.f;
        if (w.kind == kOneHot && i0 + h == w.d) q = e;
        r += fmaxf(e - q, 0.f);
        s += e + (q <= 2.f ? q : 2.f);
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        r += __shfl_xor_sync(kAll, r, o);
        s += __shfl_xor_sync(kAll, s, o);
      }
      const float gb = __shfl_sync(kAll, g, (n + k) & 31);
      if (s > 0.f) {
        const float off = s * (kSumError + kSumErrorPerBit * (fmaxf(-lg2f(s), 0.f) + 2.f * fabsf(nq))) + 1e-37f;
        const float hi = logf(r + off) + gb, lo = r > off ? logf(r - off) + gb : -CUDART_INF_F;
        insert(lead, lo - 6e-6f - 5e-7f * fabsf(lo), hi + 6e-6f + 5e-7f * fabsf(hi), b);
      }
    }
    n += kAhead;
  }
  lead.bad = __any_sync(kAll, lead.bad != 0);
  return lead;
}

struct Exact {
  double y;
  int b;
};
// The same in fp64; ties go to the lower block, blocks of weight 0 are left out.
template <int DT>
__device__ __noinline__ Exact scan_exact(const DrawRow &w, int kind, int blocks, const double *u, int from, int step) {
  const int lane = threadIdx.x & 31;
  Exact best = {0.0, INT_MAX};
  for (int b = from; b < blocks; b += step) {
    double r = 0.0, m;
    for (int i = b * E3_SAMPLE_BLOCK + lane; i < w.V && i < (b + 1) * E3_SAMPLE_BLOCK; i += 32)
      r += exact_weight(w, kind, i, load_elem<DT>(w.z, i), kind == kDistribution ? load_elem<DT>(w.y, i) : 0.f, m);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) r += __shfl_xor_sync(kAll, r, o);
    if (r > 0.0) {
      const double y = log(r) - log(-log(u[b]));
      if (best.b == INT_MAX || y > best.y) best = {y, b};
    }
  }
  return best;
}
__device__ __forceinline__ void merge(Exact &a, const Exact &o) {
  if (o.b != INT_MAX && (a.b == INT_MAX || o.y > a.y || (o.y == a.y && o.b < a.b))) a = o;
}

struct DrawShared {
  Lead lead[kWarps], cta;
  Exact exact[kWarps], cta_exact;
  double sum[kWarps], cta_sum;
  int slow, again;
};

template <int DT>
__global__ void __launch_bounds__(kThreads, 3) draw_kernel(const __grid_constant__ VerifyParams p) {
  __shared__ DrawShared sh;
  const cg::cluster_group cluster = cg::this_cluster();
  const int rank = (int)cluster.block_rank(), ctas = (int)cluster.num_blocks();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int64_t b = blockIdx.x / (unsigned)ctas;
  wait_for_stream_predecessor();
  const int len = length_of(p, b);
  const int first = p.first[b], a = first < len ? first : len;
  const int64_t r0 = b * (p.drafts + 1), r = r0 + a;
  const VerifyRow rec = p.rows[r];
  const float tau = p.temps[b];
  if (rank == 0) {
    for (int64_t j = tid; j <= p.drafts; j += kThreads) {
      if (j == a) continue;
      const VerifyRow q = j < a ? p.rows[r0 + j] : VerifyRow{};
      p.out_tok[r0 + j] = j < a ? p.draft_tok[b * p.drafts + j] : -1;
      if (p.out_logp != nullptr) p.out_logp[r0 + j] = j < a ? q.logp : 0.f;
      if (p.out_ent != nullptr) p.out_ent[r0 + j] = j < a ? q.ent : 0.f;
    }
    if (tid == 0) p.out_kept[b] = a;
  }
  auto write = [&](int tok, float logp, float ent) {  // by one thread
    p.out_tok[r] = tok;
    if (p.out_logp != nullptr) p.out_logp[r] = logp;
    if (p.out_ent != nullptr) p.out_ent[r] = ent;
  };
  if (rec.state == kInvalid) {
    if (rank == 0 && tid == 0) write(-1, CUDART_NAN_F, CUDART_NAN_F);
    return;
  }
  if (tau == 0.f) {
    if (rank == 0 && tid == 0) write(rec.best, 0.f, 0.f);
    return;
  }
  DrawRow w = {};
  w.z = p.logits + r * p.row_bytes;
  w.V = p.V; w.tau = tau; w.R = rec.R; w.lnZ = rec.lnZ; w.kind = kNoDraft; w.d = -1;
  if (a < len) {
    const Draft d = draft_of<DT>(p, b, a);
    w.kind = d.kind; w.d = d.tok; w.y_d = d.y; w.tau_d = d.tau; w.lnq = d.lnq;
    w.y = p.draft_logits + (b * p.drafts + a) * p.draft_row_bytes;
  }
  const double *const u = p.uniforms + b * p.u_stride + p.drafts;
  const double u_in = u[p.blocks];
  const int from = warp * ctas + rank, step = ctas * kWarps;
  const Lead own = scan_blocks<DT>(w, p.blocks, u, from, step);
  if (lane == 0) sh.lead[warp] = own;
  __syncthreads();
  if (tid == 0) {
    Lead l = sh.lead[0];
    for (int i = 1; i < kWarps; ++i) merge(l, sh.lead[i]);
    sh.cta = l;
  }
  auto finish = [&](int tok) {  // by one thread
    write(tok, (float)(((double)load_elem<DT>(w.z, tok) - (double)w.R) / (double)w.tau - w.lnZ), rec.ent);
  };
  cluster.sync();
  if (rank == 0 && warp == 0) {
    Lead l = lane < ctas ? *cluster.map_shared_rank(&sh.cta, lane) : no_lead();
#pragma unroll
    for (int o = 1; o < kClusterMost; o <<= 1) {
      Lead q;
      q.lo = __shfl_xor_sync(kAll, l.lo, o);
      q.hi1 = __shfl_xor_sync(kAll, l.hi1, o);
      q.hi2 = __shfl_xor_sync(kAll, l.hi2, o);
      q.lo_b = __shfl_xor_sync(kAll, l.lo_b, o);
      q.hi_b = __shfl_xor_sync(kAll, l.hi_b, o);
      q.bad = __shfl_xor_sync(kAll, l.bad, o);
      merge(l, q);
    }
    const bool bad = __shfl_sync(kAll, l.bad, 0) != 0 || !usable_uniform(u_in);
    const int block = __shfl_sync(kAll, l.lo_b, 0);
    const bool sure = __shfl_sync(kAll, l.lo > -CUDART_INF_F && l.hi_b == l.lo_b && l.lo > l.hi2, 0);
    int tok = -1;
    int slow = 0;
    if (!bad) slow = !(sure && draw_in<DT>(w, w.kind, block, u_in, false, tok));
    if (lane == 0 && bad) write(-1, CUDART_NAN_F, CUDART_NAN_F);
    if (lane == 0 && !bad && !slow) finish(tok);
    if (lane < ctas) *cluster.map_shared_rank(&sh.slow, lane) = slow;
  }
  cluster.sync();
  if (!sh.slow) return;

  // ---- in fp64: the normaliser, then every block; where nothing is left of p - q, from p
  {
    const double part = block_sum(exact_terms<DT>(w.z, p.V, w.R, w.tau, rank * kThreads + tid, ctas * kThreads), sh.sum);
    if (tid == 0) sh.cta_sum = part;
    cluster.sync();
    double total = 0.0;
    for (int i = 0; i < ctas; ++i) total += *cluster.map_shared_rank(&sh.cta_sum, i);
    w.lnZ = log(total);
  }
  int kind = w.kind;
  for (int round = 0; round < 2; ++round) {
    const Exact e = scan_exact<DT>(w, kind, p.blocks, u, from, step);
    __syncthreads();
    if (lane == 0) sh.exact[warp] = e;
    __syncthreads();
    if (tid == 0) {
      Exact x = sh.exact[0];
      for (int i = 1; i < kWarps; ++i) merge(x, sh.exact[i]);
      sh.cta_exact = x;
    }
    cluster.sync();
    if (rank == 0 && warp == 0) {
      Exact x = *cluster.map_shared_rank(&sh.cta_exact, 0);
      for (int i = 1; i < ctas; ++i) merge(x, *cluster.map_shared_rank(&sh.cta_exact, i));
      if (x.b != INT_MAX) {
        int tok = -1;
        draw_in<DT>(w, kind, x.b, u_in, true, tok);
        if (lane == 0) finish(tok);
      } else if (round == 1 && lane == 0) {
        write(-1, CUDART_NAN_F, CUDART_NAN_F);
      }
      if (lane < ctas) *cluster.map_shared_rank(&sh.again, lane) = x.b == INT_MAX && round == 0;
    }
    cluster.sync();
    if (!sh.again) return;
    kind = kNoDraft;
  }
}

// ---- host side -----------------------------------------------------------------------------------------------------
inline bool misaligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) != 0; }
inline size_t up16(size_t b) { return (b + 15) / 16 * 16; }

// Parts of a row: up to 64 KB each, smaller ones down to 8 KB where there are few rows, so that a call has about four CTAs an SM.
constexpr int64_t kCtasWanted = 592;
int part_entries(int64_t rows, int64_t V, int64_t esize, int &parts) {
  const int64_t bytes = V * esize;
  int64_t n = (bytes + 65535) / 65536;
  if (rows * n < kCtasWanted) {
    const int64_t more = kCtasWanted / rows, most = (bytes + 8191) / 8192;
    if (n < (more < most ? more : most)) n = more < most ? more : most;
  }
  if (n > kPartsMost) n = kPartsMost;
  const int64_t part = ((V + n - 1) / n + 255) / 256 * 256;
  parts = (int)((V + part - 1) / part);
  return (int)part;
}

template <class... P, class... A>
cudaError_t launch_behind(void (*kern)(P...), unsigned grid, int cluster, cudaStream_t stream, A &&...args) {
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(kThreads);
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 0 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kern, args...);
}

template <int DT>
cudaError_t launch_verify(const VerifyParams &p, cudaStream_t stream) {
  const int64_t rows = p.n_seq * (p.drafts + 1);
  cudaError_t e = launch_behind(begin_kernel, (unsigned)(rows < 256 * 1024 ? (rows + 255) / 256 : 1024), 0, stream, p);
  if (e == cudaSuccess) e = launch_behind(verify_rows_kernel<DT>, (unsigned)(rows * p.n_parts), 0, stream, p);
  int ctas = kClusterMost;
  while (ctas > 1 && (p.n_seq * ctas > kCtasWanted || p.blocks < ctas * kWarps)) ctas /= 2;
  if (e == cudaSuccess) e = launch_behind(draw_kernel<DT>, (unsigned)(p.n_seq * ctas), ctas, stream, p);
  return e;
}

size_t verify_layout(int64_t rows, size_t &arrived, size_t &records, size_t &parts) {
  arrived = up16((size_t)rows * 4);
  records = arrived + up16((size_t)rows * 4);
  parts = records + (size_t)rows * sizeof(VerifyRow);
  return parts + (size_t)rows * kPartsMost * sizeof(VerifyPart);
}

}  // namespace

size_t verify_workspace_bytes(int64_t rows) {
  size_t a, r, p;
  return verify_layout(rows < 0 ? 0 : rows, a, r, p);
}

}  // namespace e3

extern "C" e3_status e3_verify_drafts(const void *logits, e3_dtype dt, int64_t n_seq, int64_t max_draft, int64_t V, int64_t row_stride,
                                      const float *temps, const int32_t *draft_tok, const int32_t *draft_len,
                                      const void *draft_logits, int64_t draft_stride, const float *draft_temps,
                                      const float *draft_logp, const double *uniforms, int64_t uniform_stride, int32_t *out_tok,
                                      int32_t *out_kept, float *out_logp, float *out_ent, void *workspace, size_t workspace_bytes,
                                      void *stream) {
  using namespace e3;
  if (dt != E3_F32 && dt != E3_BF16) return E3_ERR_DTYPE;
  const int64_t most = int64_t(1) << 31;
  if (n_seq < 0 || n_seq >= most || max_draft < 0 || max_draft >= most || V < 1 || V >= most - E3_SAMPLE_BLOCK || row_stride < V) return E3_ERR_INVALID_ARG;
  const int64_t blocks = (V + E3_SAMPLE_BLOCK - 1) / E3_SAMPLE_BLOCK;
  if (n_seq * (max_draft + 1) >= most / kPartsMost) return E3_ERR_INVALID_ARG;  // (the parts of all rows are one grid)
  if (n_seq == 0) return E3_OK;
  if (!logits || !temps || !uniforms || uniform_stride < max_draft + blocks + 1 || !out_tok || !out_kept || (max_draft > 0 && !draft_tok))
    return E3_ERR_INVALID_ARG;
  if (max_draft == 0) draft_logits = nullptr;
  if (draft_logits && (draft_stride < V || !draft_logp)) return E3_ERR_INVALID_ARG;
  const size_t es = dt == E3_F32 ? 4 : 2;
  if (misaligned(logits, es) || misaligned(draft_logits, es) || misaligned(temps, 4) || misaligned(draft_tok, 4) || misaligned(draft_len, 4) ||
      misaligned(draft_temps, 4) || misaligned(draft_logp, 4) || misaligned(uniforms, 8) || misaligned(out_tok, 4) || misaligned(out_kept, 4) ||
      misaligned(out_logp, 4) || misaligned(out_ent, 4) || misaligned(workspace, 16))
    return E3_ERR_ALIGNMENT;
  const int64_t rows = n_seq * (max_draft + 1);
  size_t arrived, records, parts;
  if (!workspace || workspace_bytes < verify_layout(rows, arrived, records, parts)) return E3_ERR_WORKSPACE;
  char *const ws = static_cast<char *>(workspace);
  VerifyParams p = {};
  p.logits = static_cast<const char *>(logits); p.draft_logits = static_cast<const char *>(draft_logits);
  p.row_bytes = row_stride * (int64_t)es; p.draft_row_bytes = draft_stride * (int64_t)es;
  p.n_seq = n_seq; p.drafts = max_draft; p.V = (int)V; p.blocks = (int)blocks;
  p.temps = temps; p.draft_temps = draft_temps; p.draft_logp = draft_logp; p.draft_tok = draft_tok; p.draft_len = draft_len;
  p.uniforms = uniforms; p.u_stride = uniform_stride;
  p.out_tok = out_tok; p.out_kept = out_kept; p.out_logp = out_logp; p.out_ent = out_ent;
  p.first = reinterpret_cast<int32_t *>(ws); p.arrived = reinterpret_cast<int32_t *>(ws + arrived);
  p.rows = reinterpret_cast<VerifyRow *>(ws + records); p.parts = reinterpret_cast<VerifyPart *>(ws + parts);
  p.part = part_entries(rows, V, (int64_t)es, p.n_parts);
  cudaStream_t cs = static_cast<cudaStream_t>(stream);
  const cudaError_t e = dt == E3_F32 ? launch_verify<0>(p, cs) : launch_verify<1>(p, cs);
  return e == cudaSuccess ? E3_OK : E3_ERR_CUDA;
}
