// Verification of drafted tokens: which drafts of every sequence are kept, and the token that follows them.
//
// p_j = softmax(z_j / tau) of the target at position j, q_j the draft's distribution there.  Draft d_j is kept iff u_j q_j(d_j) < p_j(d_j);
// at the first position a that is refused the token comes from max(p_a - q_a, 0), behind a sequence whose drafts were all kept from p_a.
//
// One pass over the logits and a draw that looks at a few blocks.  verify_rows_kernel takes the rows position by position (every sequence's
// first row, then every second, ...), a row in parts of equal length, one CTA each: the sum of 2^t of every block of 256 entries, t = (z - R) log2(e) /
// tau with a logit R that the warp has met and nothing lies far above, and over the part Z = sum 2^t and W = sum 2^t t.  The CTA that comes last to a row joins the parts
// in their order and decides; rows behind a refused position are not read any more once that is known (which changes no result).
//
// The token comes from the construction of the blocked sampler with given uniforms, one per block: the block with the largest
// ln(sum r_i) - ln(-ln u_b), then the first entry in it whose prefix sum exceeds v times its sum.  r = p needs nothing but the blocks' sums;
// r = p - q is at most p, so draw_kernel takes the block with the largest score of p, and looks at the others whose score of p reaches that
// block's own score: three or four of them as a rule.  (Reading the row and the draft's row again, 512 x 151,936, took 164 us.)
//
// Two tokens are the same only if every comparison falls the same way, so each is made with a bound on the error of fp32 sums; what the
// bound does not settle (one sequence in about 1,000) is taken again in fp64, first with the normaliser at hand.
#include "e3_rows_device.cuh"

#include <mutex>
#include <type_traits>

#include "e3.h"

namespace e3 {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr unsigned kAll = 0xffffffffu;
constexpr float kFarBelow = 3e38f;    // distances below the largest logit are no larger (-inf: weight 0, and 0 times its distance is 0)
constexpr float kFarFrom = 0x1p20f;    // |R log2(e) / tau| from which t is taken from z - R
constexpr float kSoundSum = 0x1p20f;   // a lane's sum from which a higher reference is taken
constexpr int kScoresKept = 2048;  // blocks whose scores of p stay in shared memory
// Blocks that a warp takes in the order of their scores, each found by a look at all of them, which many blocks times long rows would make quadratic; where
// that does not do (next to nothing is left of p - q), all that may lead are looked at one after the other.
constexpr int kInOrder = 128;  // (all blocks of rows of 262,144)
// Relative error of Z, whatever V is: more than 32 parts are added in fp64 (`decide`), so what adds up is a part's own.  A term: 2^t 2^-22, and t's rounding,
// two steps of 2^-24 of |t| < 32 bits (further down lies no mass), 1.6e-6; at most 28 sums one after the other, 2^-24 each, 1.7e-6; 2^-22 and three steps for
// each move to another reference, five in a row of steps, the CTA's and the row's, 2.6e-6.
constexpr double kZError = 6e-6;
// Relative error of sums of p and q over a block in fp32 (2^t: 2^-22, and 13 sums) and through Z.
constexpr float kSumError = 8e-6f;
constexpr float kSumErrorPerBit = 1.5e-7f;  // per factor of two by which the sum, or the draft's own q, lies below 1 (rounding of t)

enum : int { kKept = 0, kRefused = 1, kInvalid = 2, kNear = 3 };  // kNear: u q is closer to p than Z is known; kept for the time being

struct VerifyPart {
  float R, Z, W;
  int err;
  int best;  // greedy rows: index of R
  int pad[3];
};
struct VerifyRow {
  double lnZ, lnq;
  float R, ent, logp, y;  // logp: of the draft; y, lnq, kind, tok: the draft's, for the draw
  int state, best, kind, tok;
};
static_assert(sizeof(VerifyPart) == 32 && sizeof(VerifyRow) == 48, "records");

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
  float2 *sums;       // of every row's blocks: sum of 2^t, the logit R it refers to
  int n_parts, part;  // parts of a row, blocks of one
  u64 by_parts, by_seq;  // for quotients by n_parts and n_seq
};

__device__ __forceinline__ void wait_for_stream_predecessor() {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
}
// The draw's CTAs start once all of the rows' have come this far: what lies before the call is done then.
__device__ __forceinline__ void wait_for_stream_predecessor_first() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
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

// Entries of a vector outside [lo, hi) become -inf, or (FINITE) -1e30, whose product with its weight 0 is 0; the vector's first entry has number e.
template <int DT, bool FINITE>
__device__ __forceinline__ uint4 keep_entries(const uint4 &v, int e, int lo, int hi) {
  constexpr uint32_t kFill = FINITE ? (DT == 0 ? 0xF149F2CAu : 0xF14AF14Au) : (DT == 0 ? 0xFF800000u : 0xFF80FF80u);
  constexpr int kE = DT == 0 ? 4 : 8;
  if (e >= lo && e + kE <= hi) return v;
  uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (DT == 0) {
      if (e + i < lo || e + i >= hi) w[i] = kFill;
    } else {
      if (e + 2 * i < lo || e + 2 * i >= hi) w[i] = (w[i] & 0xFFFF0000u) | (kFill & 0xFFFFu);
      if (e + 2 * i + 1 < lo || e + 2 * i + 1 >= hi) w[i] = (w[i] & 0xFFFFu) | (kFill & 0xFFFF0000u);
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
// Joins the sums of the first N lanes (empty ones: R = -inf, Z = 0) in a fixed order, for all of these lanes.
template <int N>
__device__ __forceinline__ void join_lanes(Sums &s, float c) {
  const float m = dec_float(__reduce_max_sync(kAll, enc_float(s.R)));
  if (m == -CUDART_INF_F) return;
  const float d = fmaxf((s.R - m) * c, -kFarBelow), f = s.Z > 0.f ? ex2f(d) : 0.f;
  s.W = f > 0.f ? f * fmaf(d, s.Z, s.W) : 0.f;
  s.Z *= f;
  s.R = m;
#pragma unroll
  for (int o = N / 2; o > 0; o >>= 1) {
    s.Z += __shfl_xor_sync(kAll, s.Z, o);
    s.W += __shfl_xor_sync(kAll, s.W, o);
  }
}
// Largest logit of the warp and its lowest index.
__device__ __forceinline__ void best_of_warp(float &R, int &best) {
  const float m = dec_float(__reduce_max_sync(kAll, enc_float(R)));
  best = __reduce_min_sync(kAll, R == m ? best : INT_MAX);
  R = m;
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

// Sums over the warp of kB values at once: lane l gets that of value l / (32 / kB).
template <int kB>
__device__ __forceinline__ float warp_sums(float (&v)[kB]) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int n = kB, o = 16; o > 0; o >>= 1) {
    if (n > 1) {
      n >>= 1;
      const bool upper = (lane & o) != 0;
#pragma unroll
      for (int i = 0; i < n; ++i) {
        const float keep = upper ? v[i + n] : v[i], give = upper ? v[i] : v[i + n];
        v[i] = keep + __shfl_xor_sync(kAll, give, o);
      }
    } else {
      v[0] += __shfl_xor_sync(kAll, v[0], o);
    }
  }
  return v[0];
}

__device__ __forceinline__ void copy16(uint32_t dst, const void *src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

template <int DT>
struct Form {
  static constexpr int kEsize = DT == 0 ? 4 : 2;
  static constexpr int kE = 16 / kEsize;              // entries of a vector
  static constexpr int kN = 8 / kE;                   // vectors of a lane in a block
  static constexpr int kStep = DT == 0 ? 2 : 4;       // blocks that a warp takes at a time: 2 KB
  static constexpr int kPartMost = DT == 0 ? 24 : 48;  // blocks that a CTA holds: 24 KB
};
constexpr int kRowWarps = 4, kRowThreads = kRowWarps * 32;
constexpr int kHeld = 8;  // CTAs that an SM holds
// Shared memory of a warp with `blocks` blocks: whole steps (the last one is read as a whole), and a vector behind them for rows that begin anywhere.
template <int DT>
__host__ __device__ constexpr int warp_bytes(int blocks) {
  return (blocks + Form<DT>::kStep - 1) / Form<DT>::kStep * Form<DT>::kStep * E3_SAMPLE_BLOCK * Form<DT>::kEsize + 16;
}
// Waits until at most `later` of the thread's groups of copies are under way.
__device__ __forceinline__ void copies_wait(int later) {
  switch (later) {
    case 0: asm volatile("cp.async.wait_group 0;" ::: "memory"); break;
    case 1: asm volatile("cp.async.wait_group 1;" ::: "memory"); break;
    case 2: asm volatile("cp.async.wait_group 2;" ::: "memory"); break;
    default: asm volatile("cp.async.wait_group 3;" ::: "memory"); break;
  }
}

// Sums of a lane's entries of kStep blocks: z of each, and W over all, t = z c - M.  CAREFUL: t = (z - R) c, and entries far below R (-inf) have
// weight 0 and count as finite.  lone: entries of rows that begin off a vector.
template <int DT, bool CAREFUL>
__device__ __forceinline__ float step_sums(const uint4 (&v)[Form<DT>::kStep][Form<DT>::kN], const float (&lone)[Form<DT>::kStep], bool lones,
                                           float c, float R, float M, float (&z)[Form<DT>::kStep]) {
  constexpr int kE = Form<DT>::kE, kN = Form<DT>::kN, kStep = Form<DT>::kStep;
  const f2 c2 = pack2f(c, c), nR2 = pack2f(-R, -R), nM2 = pack2f(-M, -M);
  f2 W2 = pack2f(0.f, 0.f);
#pragma unroll
  for (int k = 0; k < kStep; ++k) {
    f2 Z2 = pack2f(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < kN; ++i) {
#pragma unroll
      for (int h = 0; h < kE / 2; ++h) {
        f2 t = pair_of<DT>(v[k][i], h);
        if (CAREFUL) {
          t = mul2(add2(t, nR2), c2);
          t = pack2f(fmaxf(t.x, -kFarBelow), fmaxf(t.y, -kFarBelow));
        } else {
          t = fma2(t, c2, nM2);
        }
        const f2 e = pack2f(ex2f(t.x), ex2f(t.y));
        Z2 = add2(Z2, e);
        W2 = fma2(e, t, W2);
      }
    }
    z[k] = sum2(Z2);
  }
  float W = sum2(W2);
  if (lones) {
#pragma unroll
    for (int k = 0; k < kStep; ++k) {
      const float t = fmaxf(CAREFUL ? (lone[k] - R) * c : fmaf(lone[k], c, -M), -kFarBelow), e = ex2f(t);
      z[k] += e;
      W = fmaf(e, t, W);
    }
  }
  return W;
}

// Largest entry of a step; NaN if one is.
template <int DT>
__device__ __forceinline__ float most_of_step(const uint4 (&v)[Form<DT>::kStep][Form<DT>::kN], const float (&lone)[Form<DT>::kStep]) {
  float m = -CUDART_INF_F;
#pragma unroll
  for (int k = 0; k < Form<DT>::kStep; ++k) {
#pragma unroll
    for (int i = 0; i < Form<DT>::kN; ++i) m = max_nan(m, most_of<DT>(v[k][i]));
    m = max_nan(m, lone[k]);
  }
  return m;
}

// A part of a row, by its number: parts of a row run fastest, then sequences, then positions.
struct Place {
  int64_t r, b;
  int j, part;
};
// item / d from m = floor((2^64 - 1) / d) + 1 (0 for d = 1): exact for all 32-bit items, m d lies less than d above 2^64.
inline u64 for_quotients(int64_t d) { return d == 1 ? 0ull : ~0ull / (u64)d + 1ull; }
__device__ __forceinline__ uint32_t quotient(uint32_t item, u64 m) { return m == 0ull ? item : (uint32_t)__umul64hi(m, item); }
__device__ __forceinline__ Place place_of(const VerifyParams &p, uint32_t item) {
  const uint32_t at = quotient(item, p.by_parts), j = quotient(at, p.by_seq), b = at - j * (uint32_t)p.n_seq;
  return Place{(int64_t)b * (p.drafts + 1) + j, (int64_t)b, (int)j, (int)(item - at * (uint32_t)p.n_parts)};
}

// Joins the parts of row r and decides its position, by a warp.
template <int DT>
__device__ __noinline__ void decide(const VerifyParams &p, int64_t r, int64_t b, int j, float tau, float c) {
  const int lane = threadIdx.x & 31;
  const bool greedy = tau == 0.f;
  Draft d = {kNoDraft, -1, 0.f, 0.f, 0.0};
  float zd = 0.f;
  double u = 0.0;
  if (lane == 0 && j < length_of(p, b)) {
    d = draft_of<DT>(p, b, j);
    u = p.uniforms[b * p.u_stride + j];
    if (d.kind != kNoDraft) zd = load_elem<DT>(p.logits + r * p.row_bytes, d.tok);
  }
  float R = -CUDART_INF_F;
  float Z = 0.f, W = 0.f;
  int best = INT_MAX;
  bool bad = false;
  const int4 *const parts = reinterpret_cast<const int4 *>(p.parts + r * p.n_parts);  // (written by other SMs: from L2)
  int4 first = make_int4(0, 0, 0, 0);
  for (int i = lane; i < p.n_parts; i += 32) {
    const int4 x = __ldcg(parts + 2 * i);
    if (i == lane) first = x;
    const float top = __int_as_float(x.x);
    bad |= x.w != 0;
    if (greedy) {
      const int at = __ldcg(&parts[2 * i + 1].x);
      if (top > R || (top == R && at < best)) best = at;
    }
    R = fmaxf(R, top);
  }
  bad = __any_sync(kAll, bad);
  if (greedy) {
    best_of_warp(R, best);
  } else {  // each part moves to the row's reference once, and a lane adds its parts in fp64: no error grows with their number
    R = dec_float(__reduce_max_sync(kAll, enc_float(R)));
    auto add = [&](const int4 &x, auto &to_Z, auto &to_W) {
      using T = std::remove_reference_t<decltype(to_Z)>;
      const float t = fmaxf((__int_as_float(x.x) - R) * c, -kFarBelow), z = __int_as_float(x.y) * ex2f(t);
      if (!(z > 0.f)) return;
      to_Z += (T)z;
      to_W += (T)fmaf(t, z, ex2f(t) * __int_as_float(x.z));
    };
    add(first, Z, W);
    if (p.n_parts > 32) {
      double Z_on = Z, W_on = W;
      for (int i = lane + 32; i < p.n_parts; i += 32) add(__ldcg(parts + 2 * i), Z_on, W_on);
      Z = (float)Z_on;
      W = (float)W_on;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      Z += __shfl_xor_sync(kAll, Z, o);
      W += __shfl_xor_sync(kAll, W, o);
    }
  }
  if (lane != 0) return;
  VerifyRow w = {0.0, d.lnq, R, 0.f, 0.f, d.y, kRefused, best, d.kind, d.tok};
  if (bad || !(R > -CUDART_INF_F) || (!greedy && !(Z > 0.f)) || !usable_uniform(u)) {
    w.state = kInvalid;
  } else if (greedy) {
    if (d.kind != kNoDraft && d.tok == best && u * exp(d.lnq) < 1.0) w.state = kKept;
  } else {
    // c is log2(e) / tau rounded to fp32: that turns t by as much, and ln Z by the mean of t
    const double beta = 1.0 / (double)tau, mean = (double)__fdiv_rn(W, Z) * kLn2, lnZ = log((double)Z);
    w.lnZ = lnZ + (beta / (kLn2 * (double)c) - 1.0) * mean;
    w.ent = (float)fmax(lnZ - mean, 0.0);
    if (d.kind != kNoDraft) {
      const double lp = ((double)zd - (double)R) * beta - w.lnZ;
      const double ratio = u * exp(d.lnq - lp);  // (a token of probability 0: infinity or, from u = 0, NaN)
      w.logp = (float)lp;
      w.state = fabs(ratio - 1.0) < 1.01 * kZError ? kNear : (ratio < 1.0 ? kKept : kRefused);
    }
  }
  p.rows[r] = w;
  if (w.state == kRefused || w.state == kInvalid) {
    __threadfence();
    atomicMin(p.first + b, (int32_t)j);
  }
}

// Bound by the exponentials' and the other instructions' issue (70 for a lane's eight logits; 512 sequences of 3 drafts, 151,936 bf16: issue 70 %, DRAM 48 %,
// 91 us for 356 MB) and by latency: a CTA of four warps takes a part of up to
// 24 KB, all of it under way at once, eight of them an SM.  Larger CTAs wait longer for their last warp and for the decision; warps that run on from part
// to part without a barrier (three steps of 2 KB under way each) were slower for their fences and read a third more rows that were not wanted.
template <int DT>
__global__ void __launch_bounds__(kRowThreads, kHeld) verify_rows_kernel(const __grid_constant__ VerifyParams p) {
  using F = Form<DT>;
  constexpr int kE = F::kE, kN = F::kN, kEsize = F::kEsize, kStep = F::kStep;
  extern __shared__ __align__(16) unsigned char dyn[];
  __shared__ Sums sh[kRowWarps];
  __shared__ int sh_best[kRowWarps], sh_bad[kRowWarps];
  const int lane = threadIdx.x & 31, warp = __shfl_sync(kAll, threadIdx.x >> 5, 0);
  const Place at = place_of(p, blockIdx.x);
  wait_for_stream_predecessor_first();
  const int len = length_of(p, at.b);
  const float tau = p.temps[at.b];
  // (no position before it is refused; all warps see the same)
  if (at.j > len || (at.j > 0 && __syncthreads_or(threadIdx.x == 0 && *(volatile const int32_t *)(p.first + at.b) < at.j))) return;
  const char *const row = p.logits + at.r * p.row_bytes;
  const int skip = (int)(reinterpret_cast<uintptr_t>(row) & 15u) / kEsize;
  const bool greedy = tau == 0.f, usable = greedy || (tau > 0.f && tau < CUDART_INF_F);
  const float c = greedy || !usable ? 0.f : __fdiv_rn(kLog2e, tau);
  // the warp's blocks: `each` of every round of the CTA
  const int round = p.part < F::kPartMost ? p.part : F::kPartMost, each = (round + kRowWarps - 1) / kRowWarps;
  const int begin = at.part * p.part, end = begin + p.part < p.blocks ? begin + p.part : p.blocks;
  const uint32_t mem = smem_addr(dyn) + (uint32_t)(warp * warp_bytes<DT>(each));
  Sums s = {-CUDART_INF_F, 0.f, 0.f};
  float M = CUDART_INF_F, f = 1.f, g = 0.f;  // R c rounded, what that does to t (g = M - R c) and to 2^t
  auto refer_to = [&](float m) {  // refers the sums to the largest m of the warp, if that lies above R
    m = dec_float(__reduce_max_sync(kAll, enc_float(m)));
    if (m > s.R) {
      if (s.R > -CUDART_INF_F) {
        const float d = fmaxf((s.R - m) * c, -kFarBelow), t = ex2f(d);
        s.W = t * fmaf(d, s.Z, s.W);
        s.Z *= t;
      }
      s.R = m;
      M = m * c;
      g = fabsf(M) < kFarFrom ? fmaf(-m, c, M) : 0.f;
      f = ex2f(g);
    }
  };
  bool bad = !usable || !(c < CUDART_INF_F);
  int best = INT_MAX;
  // A lane's entries of a block are 8 consecutive ones of the vectors that begin at the row's last 16-byte boundary: `skip` entries early, so that
  // the first lane leaves out as many and the block's last ones are taken by the first lanes, one each.
#pragma unroll 1
  for (int first = begin + warp * each; first < end; first += kRowWarps * each) {
    const int count = first + each < end ? each : end - first, steps = (count + kStep - 1) / kStep;
    __syncwarp();  // (what lay there has been read)
    {
      const char *src = row - skip * kEsize + (int64_t)first * (E3_SAMPLE_BLOCK * kEsize) + lane * 16;
      const int64_t whole = (int64_t)(p.V - first * E3_SAMPLE_BLOCK + skip) * kEsize;  // bytes up to the row's end
      const int blocks = count * E3_SAMPLE_BLOCK * kEsize + (skip != 0 ? 16 : 0);       // (and the vector behind them)
      int left = (int)(whole < blocks ? whole : blocks) - lane * 16;                    // from this lane's next vector on
      uint32_t dst = mem + (uint32_t)lane * 16u;
      constexpr int kVecs = kStep * kN;
#pragma unroll 1
      for (int k = 0; k < steps; ++k) {
        if (left > 512 * (kVecs - 1)) {
#pragma unroll
          for (int i = 0; i < kVecs; ++i) copy16(dst + (uint32_t)(i * 512), src + i * 512);
        } else {
#pragma unroll
          for (int i = 0; i < kVecs; ++i)
            if (left > i * 512) copy16(dst + (uint32_t)(i * 512), src + i * 512);
        }
        src += kVecs * 512;
        dst += kVecs * 512;
        left -= kVecs * 512;
        if (k == steps - 1 && left > 0 && lane == 0) copy16(dst, src);
        asm volatile("cp.async.commit_group;" ::: "memory");
      }
    }
    float2 *const sums = p.sums + at.r * p.blocks + first;
#pragma unroll 1
    for (int k0 = 0; k0 < count; k0 += kStep) {
      // (rows that begin off a vector: a block's last entries lie in the next block's first vector)
      copies_wait(skip != 0 ? 0 : steps - 1 - k0 / kStep);
      __syncwarp();
      const uint32_t slot = mem + (uint32_t)(k0 * E3_SAMPLE_BLOCK * kEsize);
      uint4 v[kStep][kN];
      float lone[kStep];
      const bool whole = skip == 0 && k0 + kStep <= count && (first + k0 + kStep) * E3_SAMPLE_BLOCK <= p.V;
#pragma unroll
      for (int k = 0; k < kStep; ++k) {
        lone[k] = -1e30f;
#pragma unroll
        for (int i = 0; i < kN; ++i) v[k][i] = lds128(slot + (uint32_t)(((k * 32 + lane) * kN + i) * 16));
      }
      auto cut = [&](auto finite) {  // what is not the blocks' or not the row's
#pragma unroll
        for (int k = 0; k < kStep; ++k) {
          const int lo = (first + k0 + k) * E3_SAMPLE_BLOCK, hi = k0 + k < count ? p.V : 0;
#pragma unroll
          for (int i = 0; i < kN; ++i) v[k][i] = keep_entries<DT, decltype(finite)::value>(v[k][i], lo + lane * 8 + i * kE - skip, lo, hi);
          if (!(lane < skip && lo + E3_SAMPLE_BLOCK - skip + lane < hi)) lone[k] = decltype(finite)::value ? -1e30f : -CUDART_INF_F;
        }
      };
      if (skip != 0) {
#pragma unroll
        for (int k = 0; k < kStep; ++k)
          if (lane < skip) lone[k] = lds_elem<DT>(slot + (uint32_t)(((k + 1) * E3_SAMPLE_BLOCK + lane) * kEsize));
      }
      if (!whole) cut(std::true_type());
      if (greedy) {
        cut(std::false_type());
        const float m = most_of_step<DT>(v, lone);
        bad |= !(m < CUDART_INF_F);
        if (m > s.R) {
          s.R = m;
          best = INT_MAX;
#pragma unroll
          for (int k = 0; k < kStep; ++k) {  // lowest of the lane's entries with that logit (those of later steps have higher numbers)
            const int lo = (first + k0 + k) * E3_SAMPLE_BLOCK;
#pragma unroll
            for (int i = 0; i < kN; ++i) {
#pragma unroll
              for (int h = 0; h < kE / 2; ++h) {
                const f2 z = pair_of<DT>(v[k][i], h);
                const int e = lo + lane * 8 + i * kE - skip + 2 * h;
                if (z.x == m && e < best) best = e;
                if (z.y == m && e + 1 < best) best = e + 1;
              }
            }
            if (lone[k] == m && lo + E3_SAMPLE_BLOCK - skip + lane < best) best = lo + E3_SAMPLE_BLOCK - skip + lane;
          }
        }
        continue;
      }
      float z[kStep], W = 0.f, all = 0.f;
      bool sound = false;
      if (s.R == -CUDART_INF_F) {  // a first reference: the largest logit of one block
        const float m = most_of<DT>(v[0][0]);
        refer_to(m > -1e29f && m < CUDART_INF_F ? m : -CUDART_INF_F);
      }
      if (fabsf(M) < kFarFrom && c > 1e-20f) {  // (there is a reference, and -1e30 lies far below it)
        W = step_sums<DT, false>(v, lone, skip != 0, c, s.R, M, z);
#pragma unroll
        for (int k = 0; k < kStep; ++k) all += z[k];
        sound = !__any_sync(kAll, !(all < kSoundSum) || !(fabsf(W) < kFarBelow));
      }
      if (!sound) {
        // no reference yet, or a logit far above it, NaN or an infinity
        cut(std::false_type());
        float m = most_of_step<DT>(v, lone);
        if (!(m < CUDART_INF_F)) {
          bad = true;
          m = -CUDART_INF_F;
        }
        refer_to(m);
        W = step_sums<DT, true>(v, lone, skip != 0, c, s.R > -CUDART_INF_F ? s.R : 0.f, 0.f, z);
        all = 0.f;
#pragma unroll
        for (int k = 0; k < kStep; ++k) all += z[k];
        s.Z += all;
        s.W += W;
      } else {  // from M, which is rounded, to R c
        s.Z = fmaf(f, all, s.Z);
        s.W = fmaf(f, fmaf(g, all, W), s.W);
      }
      const float sum = warp_sums(z);
      const int k = k0 + lane / (32 / kStep);
      if (lane % (32 / kStep) == 0 && k < count) sums[k] = make_float2(sound ? sum * f : sum, s.R);  // (-inf: nothing but -inf so far)
    }
  }
  // ---- the part's result, joined in a fixed order
  if (greedy) {
    best_of_warp(s.R, best);
  } else {  // (R is that of the warp)
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      s.Z += __shfl_xor_sync(kAll, s.Z, o);
      s.W += __shfl_xor_sync(kAll, s.W, o);
    }
  }
  bad = __any_sync(kAll, bad);
  if (lane == 0) {
    sh[warp] = s;
    sh_best[warp] = best;
    sh_bad[warp] = bad;
  }
  __syncthreads();
  if (warp != 0) return;
  s = lane < kRowWarps ? sh[lane] : Sums{-CUDART_INF_F, 0.f, 0.f};
  best = lane < kRowWarps ? sh_best[lane] : INT_MAX;
  bad = __any_sync(kAll, lane < kRowWarps && sh_bad[lane] != 0);
  if (greedy) best_of_warp(s.R, best);
  else join_lanes<kRowWarps>(s, c);
  int last = 0;
  if (lane == 0) {
    VerifyPart out = {s.R, s.Z, s.W, bad ? 1 : 0, best, {0, 0, 0}};
    p.parts[at.r * p.n_parts + at.part] = out;
    int before;
    asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(before) : "l"(p.arrived + at.r) : "memory");
    last = before == p.n_parts - 1;
  }
  if (__shfl_sync(kAll, last, 0) != 0) decide<DT>(p, at.r, at.b, at.j, tau, c);
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

// Gumbel variate -ln(-ln u) of a uniform, good to a few units of fp32; NaN for one that cannot be used.
__device__ __forceinline__ float gumbel_of(double u) {
  if (!usable_uniform(u)) return CUDART_NAN_F;
  const float w = u < 0.5 ? (u > 1e-30 ? -logf((float)u) : (float)-log(u)) : -log1pf((float)(u - 1.0));
  return -logf(w);
}

// The row a token is drawn from.
struct DrawRow {
  const char *z, *y;      // target, draft (kDistribution)
  int V, kind, d;
  float tau, R, y_d;
  double lnZ, lnq, beta, beta_d;  // (betas: 1 / temperature)
  float c, nz, cd, nq;    // the same for sums in fp32, log2 units
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

// exp((z - R) / tau) in fp64 of all bf16 values of 2^-9 <= |z| < 2^8: a row in bf16 has no others but a few near zero.
constexpr int kExpLow = (127 - 9) << 7, kExps = 17 << 7;  // pattern of 2^-9, patterns up to 2^8
// sum over the row of exp((z - R) / tau) in fp64, a thread's part of it, by the whole CTA.  Bound by one SM's fp64 units, and by the latency of what is not
// under way beside other things: vectors, four sums, no branches but for the few logits that the table does not hold.
template <int DT>
__device__ __noinline__ double exact_terms(const char *row, int V, float R, float tau, double *table /* [2 kExps + 1], bf16 */) {
  constexpr int kAhead = DT == 1 ? 4 : 1;
  const double beta = 1.0 / (double)tau;
  if (DT == 1) {
    __syncthreads();
#pragma unroll 1
    for (int i = threadIdx.x; i < 2 * kExps; i += kThreads) {
      const uint32_t bits = i < kExps ? (uint32_t)(kExpLow + i) : (uint32_t)(kExpLow + i - kExps) | 0x8000u;
      table[i] = exp(((double)__uint_as_float(bits << 16) - (double)R) * beta);
    }
    if (threadIdx.x == 0) table[2 * kExps] = 0.0;
    __syncthreads();
  }
  double s[4] = {};
#pragma unroll 1
  for (int64_t i0 = (int64_t)threadIdx.x * 8; i0 < V; i0 += (int64_t)kThreads * 8 * kAhead) {
    Eight<DT> e[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (i0 + (int64_t)k * kThreads * 8 < V) e[k] = load_eight<DT>(row, V, (int)(i0 + (int64_t)k * kThreads * 8));
    bool others = false;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int64_t i = i0 + (int64_t)k * kThreads * 8;
      const int there = i < V ? (V - i < 8 ? (int)(V - i) : 8) : 0;
      if (DT == 1) {
#pragma unroll
        for (int h = 0; h < 8; ++h) {
          const uint32_t bits = __float_as_uint(entry<DT>(e[k], h)) >> 16, at = (bits & 0x7FFFu) - kExpLow;
          const bool known = at < (uint32_t)kExps && h < there;
          others |= !known && h < there;
          s[h & 3] += table[known ? at + ((bits & 0x8000u) != 0u ? kExps : 0) : 2 * kExps];
        }
      } else {
#pragma unroll
        for (int h = 0; h < 8; ++h) s[h & 3] += h < there ? exp(((double)entry<DT>(e[k], h) - (double)R) * beta) : 0.0;
      }
    }
    if (DT == 1 && others) {
#pragma unroll 1
      for (int n = 0; n < 8 * kAhead; ++n) {
        const int64_t i = i0 + (int64_t)(n >> 3) * kThreads * 8 + (n & 7);
        if (i >= V) continue;
        const float z = load_elem<DT>(row, i);
        if (((__float_as_uint(z) >> 16) & 0x7FFFu) - kExpLow >= (uint32_t)kExps && z > -CUDART_INF_F) s[0] += exp(((double)z - (double)R) * beta);
      }
    }
  }
  return (s[0] + s[1]) + (s[2] + s[3]);
}

// Weight max(p - q, 0) of an entry in fp64 (q of a logit that is NaN: the entry is not drawn).  open: by how much the weight may turn otherwise than in
// proportion where Z is known to kZError, in units of that: a weight p (1 + e) - q is (1 + e) (p - q) and e q more, and one within e p of 0 may come or go.
__device__ __forceinline__ double exact_weight(const DrawRow &w, int kind, int i, float z, float y, double &open) {
  const double mass = exp(((double)z - (double)w.R) * w.beta - w.lnZ);
  open = 0.0;
  if (kind == kNoDraft) return mass;
  if (kind == kOneHot) return i == w.d ? 0.0 : mass;
  const double q = exp(((double)y - (double)w.y_d) * w.beta_d + w.lnq), r = mass - q;
  if (r > 0.0) open = q;
  if (fabs(r) <= 2.0 * kZError * mass) open += 2.0 * mass;
  return r > 0.0 ? r : 0.0;
}

// Draw inside block b by the CTA, an entry a thread (a warp with eight entries a lane took 8 us: the exponentials are in fp64).  False: the fp32
// normaliser leaves open which entry it is.
template <int DT>
__device__ __noinline__ bool draw_in(const DrawRow &w, int kind, int b, double u, bool exact, double *sh /* [2 * warps] */, int &tok) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, i = b * E3_SAMPLE_BLOCK + tid;
  static_assert(kThreads == E3_SAMPLE_BLOCK, "an entry a thread");
  double r = 0.0, open = 0.0;
  if (i < w.V) r = exact_weight(w, kind, i, load_elem<DT>(w.z, i), kind == kDistribution ? load_elem<DT>(w.y, i) : 0.f, open);
  double sum = r;  // of the warp's entries up to this one
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const double up = __shfl_up_sync(kAll, sum, o);
    if (lane >= o) sum += up;
    open += __shfl_xor_sync(kAll, open, o);
  }
  __syncthreads();
  if (lane == 31) {
    sh[warp] = sum;
    sh[kWarps + warp] = open;
  }
  __syncthreads();
  double total = 0.0;
  open = 0.0;
#pragma unroll
  for (int k = 0; k < kWarps; ++k) {
    if (k < warp) sum += sh[k];
    total += sh[k];
    open += sh[kWarps + k];
  }
  const double t = u * total, margin = exact || kind != kDistribution ? 0.0 : 1.01 * kZError * open;
  const bool close = i < w.V && margin > 0.0 && fabs(sum - t) <= margin;
  int first = sum > t && r > 0.0 ? i : INT_MAX, last = r > 0.0 ? i : -1;
  first = __reduce_min_sync(kAll, first);
  last = __reduce_max_sync(kAll, last);
  int *const ints = reinterpret_cast<int *>(sh);
  const bool undecided = __syncthreads_or(close);  // (and the sums have been read)
  if (lane == 0) {
    ints[2 * warp] = first;
    ints[2 * warp + 1] = last;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kWarps; ++k) {
    first = min(first, ints[2 * k]);
    last = max(last, ints[2 * k + 1]);
  }
  __syncthreads();
  tok = first != INT_MAX ? first : last;
  return !undecided && tok >= 0;
}

// Score of block b under p, but for the constant -ln Z (natural logarithms): ln of its sum plus its Gumbel variate.
constexpr float kFlushed = 0x1p-118f;  // what a block's 256 terms may lack in fp32: each that is below 2^-126 reads 0
struct Score {
  float y, off, hi;  // value, bound on its error but for terms that read 0, upper bound
};
__device__ __forceinline__ Score score_of_p(const float2 &s, float gumbel, float R, float tau) {
  const float x = __fdiv_rn(fmaxf(s.y - R, -kFarBelow), tau), y = logf(s.x) + x + gumbel;
  const float off = 1.2e-5f + 2e-6f * (fabsf(x) < 1e3f ? fabsf(x) : 1e3f);
  return Score{y, off, (s.x > 0x1p-94f ? y : logf(s.x + kFlushed) + x + gumbel) + off};
}

// Score of a block with weights p - q, with bounds, by a warp.
template <int DT>
__device__ __forceinline__ void score_block(const DrawRow &w, int b, float gumbel, float &lo, float &hi) {
  const int lane = threadIdx.x & 31, i0 = b * E3_SAMPLE_BLOCK + lane * 8;
  const Eight<DT> z = load_eight<DT>(w.z, w.V, i0);
  Eight<DT> y = z;
  if (w.kind == kDistribution) y = load_eight<DT>(w.y, w.V, i0);
  float r = 0.f, s = 0.f;
#pragma unroll
  for (int h = 0; h < 8; ++h) {
    const float zk = i0 + h < w.V ? entry<DT>(z, h) : -CUDART_INF_F;
    const float e = ex2f(fmaf(zk - w.R, w.c, w.nz));
    float q = 0.f;
    if (w.kind == kDistribution) q = i0 + h < w.V ? ex2f(fmaf(entry<DT>(y, h) - w.y_d, w.cd, w.nq)) : 0.f;
    if (w.kind == kOneHot && i0 + h == w.d) q = e;
    r += fmaxf(e - q, 0.f);
    s += e + (q <= 2.f ? q : 2.f);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    r += __shfl_xor_sync(kAll, r, o);
    s += __shfl_xor_sync(kAll, s, o);
  }
  const float off = s * (kSumError + kSumErrorPerBit * (fmaxf(-lg2f(fmaxf(s, kFlushed)), 0.f) + 2.f * fabsf(w.nq))) + 2.f * kFlushed;
  hi = logf(r + off) + gumbel;
  lo = r > off ? logf(r - off) + gumbel : -CUDART_INF_F;
  hi += 6e-6f + 5e-7f * fabsf(hi);
  lo -= 6e-6f + 5e-7f * fabsf(lo);
}

struct Exact {
  double y;
  int b;
};
// The two leading ones of scores that are known but for a bound.
struct Near {
  double lo, hi1, hi2;
  int lo_b, hi_b;
};
__device__ __forceinline__ Near no_near() { return Near{-CUDART_INF, -CUDART_INF, -CUDART_INF, INT_MAX, INT_MAX}; }
__device__ __forceinline__ void merge(Near &a, const Near &o) {
  if (o.lo > a.lo) {
    a.lo = o.lo;
    a.lo_b = o.lo_b;
  }
  if (o.hi1 > a.hi1) {
    a.hi2 = fmax(a.hi1, o.hi2);
    a.hi1 = o.hi1;
    a.hi_b = o.hi_b;
  } else {
    a.hi2 = fmax(a.hi2, o.hi1);
  }
}
// Score of block b with the weights of `kind` in fp64, by a warp; false: weight 0.  off: what an error of kZError in Z may move it against other blocks'.  A
// block's sum r turns into r (1 + e) + e g with |g| at most the sum of `open`, and ln(1 + e) is common to all blocks.
template <int DT>
__device__ __noinline__ bool exact_score_of(const DrawRow &w, int kind, int b, double u, double &y, double &off) {
  const int lane = threadIdx.x & 31, i0 = b * E3_SAMPLE_BLOCK + lane * 8;
  const Eight<DT> z = load_eight<DT>(w.z, w.V, i0);
  Eight<DT> d = z;
  if (kind == kDistribution) d = load_eight<DT>(w.y, w.V, i0);
  double r = 0.0, g = 0.0, open;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    if (i0 + k < w.V) {
      r += exact_weight(w, kind, i0 + k, entry<DT>(z, k), entry<DT>(d, k), open);
      g += open;
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    r += __shfl_xor_sync(kAll, r, o);
    g += __shfl_xor_sync(kAll, g, o);
  }
  off = 0.0;
  if (!(r > 0.0)) {
    off = g > 0.0 ? CUDART_INF : 0.0;
    return false;
  }
  const double e = 1.01 * kZError * g / r, x = e + kZError;
  off = x < 0.1 ? e + x * x + 1e-12 : CUDART_INF;  // (|ln(1 + x) - x| <= x^2)
  y = log(r) - log(-log(u));
  return true;
}
__device__ __forceinline__ void merge(Exact &a, const Exact &o) {
  if (o.b != INT_MAX && (a.b == INT_MAX || o.y > a.y || (o.y == a.y && o.b < a.b))) a = o;
}
__device__ __forceinline__ Lead lead_of_warp(Lead l) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    Lead q;
    q.lo = __shfl_xor_sync(kAll, l.lo, o);
    q.hi1 = __shfl_xor_sync(kAll, l.hi1, o);
    q.hi2 = __shfl_xor_sync(kAll, l.hi2, o);
    q.lo_b = __shfl_xor_sync(kAll, l.lo_b, o);
    q.hi_b = __shfl_xor_sync(kAll, l.hi_b, o);
    q.bad = __shfl_xor_sync(kAll, l.bad, o);
    merge(l, q);
  }
  return l;
}

struct DrawShared {
  float gumbel[kScoresKept];  // of the first blocks: variates
  union {
    float score[kScoresKept];  // and upper bounds of the scores under p
    double exps[2 * kExps + 1];  // while a row is summed in fp64, and no score is needed
  };
  Lead lead[kWarps], all;
  union {
    Exact exact[kWarps];
    Near close[kWarps];
  };
  double sum[2 * kWarps];
  int reached;  // score of p - q that some block reaches, encoded
};
// The CTA's lead from its warps', for every thread.
__device__ __forceinline__ Lead lead_of_cta(const Lead &l, DrawShared &sh) {
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sh.lead[threadIdx.x >> 5] = l;
  __syncthreads();
  if (threadIdx.x < 32) {
    const Lead all = lead_of_warp(threadIdx.x < kWarps ? sh.lead[threadIdx.x] : no_lead());
    if (threadIdx.x == 0) sh.all = all;
  }
  __syncthreads();
  return sh.all;
}

// A CTA draws for a sequence: a chain of dependent loads, small reductions and code that is met once, so what hangs on the call's inputs alone (the
// variates of all blocks) is done beside the last rows, and what the decision knew of the draft comes with its record.
// CTAS of an SM: 4, or the 2 that calls of few sequences need, with as many registers as the draw asks for (64 sequences of 4 drafts, 151,936 bf16: 43 us
// for the whole call, 45.5 with 4; 512 sequences of 3: 118 us with 2, 114 with 4).
template <int DT, int CTAS>
__global__ void __launch_bounds__(kThreads, CTAS) draw_kernel(const __grid_constant__ VerifyParams p) {
  __shared__ DrawShared sh;
  const int tid = threadIdx.x, warp = __shfl_sync(kAll, tid >> 5, 0), lane = tid & 31;
  const int64_t b = blockIdx.x;
  if (tid == 0) sh.reached = enc_neg_inf();
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  // What the call was given may be read beside the last rows (the rows' CTAs have all begun behind it): the blocks' variates are ready when the sums are.
  const double *const u = p.uniforms + b * p.u_stride + p.drafts;
  const float tau = __ldcg(p.temps + b), tau_d = p.draft_temps != nullptr ? __ldcg(p.draft_temps + b) : tau;
  const double u_in = __ldcg(u + p.blocks);
  const int kept = p.blocks < kScoresKept ? p.blocks : kScoresKept;
  if (tau != 0.f) {
#pragma unroll 1
    for (int i = tid; i < kept; i += kThreads) sh.gumbel[i] = gumbel_of(__ldcg(u + i));
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int len = length_of(p, b);
  const int first = p.first[b];
  int a = first < len ? first : len;
  const int64_t r0 = b * (p.drafts + 1);
  auto exact_total = [&](const char *row, float R) { return block_sum(exact_terms<DT>(row, p.V, R, tau, sh.exps), sh.sum); };
  bool near = false;
  for (int j = tid; j < a; j += kThreads) near |= p.rows[r0 + j].state == kNear;
  VerifyRow rec = p.rows[r0 + a];
  if (__syncthreads_or(near)) {  // positions that wait for a normaliser in fp64, in their order
    for (int j = 0; j < a; ++j) {
      const VerifyRow q = p.rows[r0 + j];
      if (q.state != kNear) continue;
      const char *const row = p.logits + (r0 + j) * p.row_bytes;
      const double lnZ = log(exact_total(row, q.R));
      const double lp = ((double)load_elem<DT>(row, q.tok) - (double)q.R) * (1.0 / (double)tau) - lnZ;
      if (p.uniforms[b * p.u_stride + j] * exp(q.lnq) < exp(lp)) continue;
      a = j;
      rec = q;
      rec.lnZ = lnZ;
      rec.state = kRefused;
    }
  }
  const int64_t r = r0 + a;
  for (int64_t j = tid; j <= p.drafts; j += kThreads) {
    if (j == a) continue;
    const VerifyRow q = j < a ? p.rows[r0 + j] : VerifyRow{};
    p.out_tok[r0 + j] = j < a ? p.draft_tok[b * p.drafts + j] : -1;
    if (p.out_logp != nullptr) p.out_logp[r0 + j] = j < a ? q.logp : 0.f;
    if (p.out_ent != nullptr) p.out_ent[r0 + j] = j < a ? q.ent : 0.f;
  }
  if (tid == 0) p.out_kept[b] = a;
  auto write = [&](int tok, float logp, float ent) {
    if (tid != 0) return;
    p.out_tok[r] = tok;
    if (p.out_logp != nullptr) p.out_logp[r] = logp;
    if (p.out_ent != nullptr) p.out_ent[r] = ent;
  };
  if (rec.state == kInvalid) return write(-1, CUDART_NAN_F, CUDART_NAN_F);
  if (tau == 0.f) return write(rec.best, 0.f, 0.f);
  DrawRow w = {};
  w.z = p.logits + r * p.row_bytes;
  w.V = p.V; w.tau = tau; w.R = rec.R; w.lnZ = rec.lnZ; w.kind = rec.kind; w.d = rec.tok; w.y_d = rec.y; w.lnq = rec.lnq;
  if (w.kind == kDistribution) {
    w.y = p.draft_logits + (b * p.drafts + a) * p.draft_row_bytes;
    w.beta_d = 1.0 / (double)tau_d; w.cd = fminf(__fdiv_rn(kLog2e, tau_d), 3.4e38f);  // (times 0 is 0: logits that tie)
    w.nq = (float)(rec.lnq * (1.0 / kLn2));
  }
  const float2 *const sums = p.sums + r * p.blocks;
  // ---- scores under p: of the draw itself, or upper bounds (a loop of one copy: a CTA runs through most of this once, and waits for its instructions)
  Lead lead = no_lead();
  auto score_at = [&](int i, const float2 &s) { return score_of_p(s, i < kScoresKept ? sh.gumbel[i] : gumbel_of(u[i]), w.R, w.tau); };
  float2 sum = tid < p.blocks ? __ldcg(sums + tid) : make_float2(0.f, 0.f);
#pragma unroll 1
  for (int i = tid; i < p.blocks; i += kThreads) {
    const float2 s = sum;
    if (i + kThreads < p.blocks) sum = __ldcg(sums + i + kThreads);
    const Score y = score_at(i, s);
    lead.bad |= y.y != y.y;
    if (i < kScoresKept) sh.score[i] = y.hi;
    insert(lead, y.y - y.off, y.hi, i);
  }
  w.beta = 1.0 / (double)tau; w.c = __fdiv_rn(kLog2e, tau); w.nz = -(float)(rec.lnZ * (1.0 / kLn2));
  // (the normaliser that the decision had, on every way here: which way a draw takes may hang on which warp was first to reach a score)
  auto finish = [&](int tok) {
    if (tok < 0) return write(-1, CUDART_NAN_F, CUDART_NAN_F);
    if (tid == 0) write(tok, (float)(((double)load_elem<DT>(w.z, tok) - (double)w.R) * w.beta - rec.lnZ), rec.ent);
  };
  lead = lead_of_cta(lead_of_warp(lead), sh);
  if (lead.bad != 0 || !usable_uniform(u_in)) return write(-1, CUDART_NAN_F, CUDART_NAN_F);
  float lnz = (float)w.lnZ;
  const float reached_p = lead.lo - lnz;
  if (w.kind != kNoDraft) {
    // weights p - q: those blocks whose scores of p reach the best known score of p - q
    auto bound = [&](int i) {
      if (i < kScoresKept) return sh.score[i];
      return score_at(i, __ldcg(sums + i)).hi;
    };
    Lead mine = no_lead();
    float last = CUDART_INF_F;  // a warp takes its blocks in the order of their scores of p, highest first
    int last_b = -1;
    for (int taken = 0;; ++taken) {
      if (taken == kInOrder) {
        mine.bad = 1;  // unfinished
        break;
      }
      float most = -CUDART_INF_F;
      int at = INT_MAX;
      for (int i = warp * 32 + lane; i < p.blocks; i += kThreads) {
        const float y = bound(i);
        if ((y < last || (y == last && i > last_b)) && y > most) {
          most = y;
          at = i;
        }
      }
      const float top = dec_float(__reduce_max_sync(kAll, enc_float(most)));
      const int i = __reduce_min_sync(kAll, most == top ? at : INT_MAX);
      // (the two kinds of scores differ by ln Z)
      if (i == INT_MAX || top - lnz + 4e-6f < dec_float(*(volatile int *)&sh.reached)) break;
      float lo, hi;
      score_block<DT>(w, i, i < kScoresKept ? sh.gumbel[i] : gumbel_of(u[i]), lo, hi);
      insert(mine, lo, hi, i);
      if (lane == 0) atomicMax(&sh.reached, enc_float(lo));
      __syncwarp();
      last = top;
      last_b = i;
    }
    lead = lead_of_cta(mine, sh);
  }
  const bool sure = lead.bad == 0 && lead.lo > -CUDART_INF_F && lead.hi_b == lead.lo_b && lead.lo > lead.hi2;
  int tok = -1, chosen = sure ? lead.lo_b : INT_MAX;
  if (sure && draw_in<DT>(w, w.kind, chosen, u_in, false, sh.sum, tok)) return finish(tok);

  // Visits the blocks whose scores of p reach `floor`, a warp each; all blocks where nothing is known to be reached (-inf: a block's score is that too
  // where its uniform is 0, and what fp32 does not hold may have weight).
  auto visit = [&](float floor, auto &&with) {
    for (int i0 = warp * 32; i0 < p.blocks; i0 += kThreads) {
      float hi = -CUDART_INF_F;
      if (i0 + lane < p.blocks) hi = score_at(i0 + lane, __ldcg(sums + i0 + lane)).hi - lnz + 1e-5f;
      uint32_t open = __ballot_sync(kAll, i0 + lane < p.blocks && hi >= floor);
      while (open != 0u) {
        with(i0 + __ffs((int)open) - 1);
        open &= open - 1u;
      }
    }
  };
  if (w.kind == kDistribution) {
    // ---- two blocks that fp32 leaves open: their scores in fp64 with the normaliser at hand, as a rule that settles them
    if (!sure) {
      Near mine = no_near();
      visit(lead.lo, [&](int i) {
        double y, off;
        const bool any = exact_score_of<DT>(w, kDistribution, i, u[i], y, off);
        if (any || off > 0.0) merge(mine, any ? Near{y - off, y + off, -CUDART_INF, i, i} : Near{-CUDART_INF, CUDART_INF, -CUDART_INF, INT_MAX, i});
      });
      __syncthreads();
      if (lane == 0) sh.close[warp] = mine;
      __syncthreads();
      mine = sh.close[0];
      for (int i = 1; i < kWarps; ++i) merge(mine, sh.close[i]);
      if (mine.lo > -CUDART_INF && mine.lo_b == mine.hi_b && mine.lo > mine.hi2) {
        chosen = mine.lo_b;
        if (draw_in<DT>(w, kDistribution, chosen, u_in, false, sh.sum, tok)) return finish(tok);
      }
    }
    // ---- the normaliser in fp64: it counts only beside a q that is not in proportion to p
    w.lnZ = log(exact_total(w.z, w.R));
    lnz = (float)w.lnZ;
    if (chosen != INT_MAX) {
      draw_in<DT>(w, kDistribution, chosen, u_in, true, sh.sum, tok);
      return finish(tok);
    }
  }
  // ---- the blocks that the bounds did not exclude, exactly; where nothing is left of p - q, from p
  int kind = w.kind;
  float floor = kind == kNoDraft ? reached_p - 1e-5f : lead.lo;  // a score that some block reaches (ln Z is in it)
  for (int round = 0; round < 2; ++round) {
    Exact e = {0.0, INT_MAX};
    visit(floor, [&](int i) {
      double y, off;
      if (exact_score_of<DT>(w, kind, i, u[i], y, off)) merge(e, Exact{y, i});
    });
    __syncthreads();
    if (lane == 0) sh.exact[warp] = e;
    __syncthreads();
    e = sh.exact[0];
    for (int i = 1; i < kWarps; ++i) merge(e, sh.exact[i]);
    if (e.b != INT_MAX) {
      draw_in<DT>(w, kind, e.b, u_in, true, sh.sum, tok);
      return finish(tok);
    }
    kind = kNoDraft;
    floor = reached_p - 1e-5f;
  }
  write(-1, CUDART_NAN_F, CUDART_NAN_F);
}

// ---- host side -----------------------------------------------------------------------------------------------------
inline bool misaligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) != 0; }
inline size_t up16(size_t b) { return (b + 15) / 16 * 16; }

// Parts of a row (blocks of one, and their number): what a CTA holds, or as much less as makes a call of few rows fill the SMs, down to a step a warp.
// Calls that fill them many times over take two rounds a CTA, whose set-up, joining and decision cost as much as a round (512 sequences of 3 drafts,
// 151,936 bf16: 108 us, 115 with one, 111 with three; 64 of 4: 44.5, with one 43.5).
constexpr int64_t kCtasHeld = kHeld * 148;
int part_blocks(int64_t rows, int64_t blocks, int most, int least, int &parts) {
  int64_t n = (blocks + most - 1) / most;
  if (rows * n < kCtasHeld) {
    const int64_t each = kCtasHeld / rows, finest = (blocks + least - 1) / least;
    n = each < finest ? (each > n ? each : n) : (finest > n ? finest : n);
  }
  int64_t part = (blocks + n - 1) / n;
  while (rows * ((blocks + part - 1) / part) >= int64_t(1) << 31) part *= 2;
  parts = (int)((blocks + part - 1) / part);
  return (int)part;
}

template <class... P, class... A>
cudaError_t launch_behind(void (*kern)(P...), unsigned grid, int threads, size_t smem, cudaStream_t stream, A &&...args) {
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, args...);
}

template <int DT>
cudaError_t launch_verify(VerifyParams &p, cudaStream_t stream) {
  using F = Form<DT>;
  constexpr int kSmemMost = kRowWarps * warp_bytes<DT>(F::kPartMost / kRowWarps);
  static std::mutex lock;
  static bool ready[64];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  {
    std::lock_guard<std::mutex> hold(lock);
    if (!ready[dev]) {
      e = cudaFuncSetAttribute(verify_rows_kernel<DT>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemMost);
      if (e != cudaSuccess) return e;
      ready[dev] = true;
    }
  }
  const int64_t rows = p.n_seq * (p.drafts + 1);
  const bool many = rows * ((p.blocks + F::kPartMost - 1) / F::kPartMost) >= 8 * kCtasHeld;
  p.part = part_blocks(rows, p.blocks, many ? 2 * F::kPartMost : F::kPartMost, F::kStep * kRowWarps, p.n_parts);
  p.by_parts = for_quotients(p.n_parts);
  p.by_seq = for_quotients(p.n_seq);
  const int round = p.part < F::kPartMost ? p.part : F::kPartMost;
  e = launch_behind(begin_kernel, (unsigned)(rows < 256 * 1024 ? (rows + 255) / 256 : 1024), 256, 0, stream, p);
  if (e == cudaSuccess)
    e = launch_behind(verify_rows_kernel<DT>, (unsigned)(rows * p.n_parts), kRowThreads,
                      (size_t)(kRowWarps * warp_bytes<DT>((round + kRowWarps - 1) / kRowWarps)), stream, p);
  if (e == cudaSuccess) e = launch_behind(p.n_seq <= 2 * 148 ? draw_kernel<DT, 2> : draw_kernel<DT, 4>, (unsigned)p.n_seq, kThreads, 0, stream, p);
  return e;
}

struct Layout {
  size_t arrived, records, parts, sums, bytes;
};
Layout layout(int64_t rows, int64_t blocks) {
  Layout l;
  l.arrived = up16((size_t)rows * 4);
  l.records = l.arrived + up16((size_t)rows * 4);
  l.parts = l.records + (size_t)rows * sizeof(VerifyRow);
  l.sums = l.parts + (size_t)rows * (size_t)((blocks + 7) / 8) * sizeof(VerifyPart);  // (parts of at least eight blocks)
  l.bytes = l.sums + (size_t)rows * (size_t)blocks * sizeof(float2);
  return l;
}

}  // namespace

size_t verify_workspace_bytes(int64_t rows, int64_t V) {
  return rows < 0 || V < 1 ? 0 : layout(rows, (V + E3_SAMPLE_BLOCK - 1) / E3_SAMPLE_BLOCK).bytes;
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
  if (n_seq < 0 || n_seq >= most || max_draft < 0 || max_draft >= most || V < 1 || V >= most - 65536 || row_stride < V) return E3_ERR_INVALID_ARG;
  const int64_t blocks = (V + E3_SAMPLE_BLOCK - 1) / E3_SAMPLE_BLOCK;
  if (n_seq * (max_draft + 1) >= int64_t(1) << 26) return E3_ERR_INVALID_ARG;
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
  const Layout l = layout(rows, blocks);
  if (!workspace || workspace_bytes < l.bytes) return E3_ERR_WORKSPACE;
  char *const ws = static_cast<char *>(workspace);
  VerifyParams p = {};
  p.logits = static_cast<const char *>(logits); p.draft_logits = static_cast<const char *>(draft_logits);
  p.row_bytes = row_stride * (int64_t)es; p.draft_row_bytes = draft_stride * (int64_t)es;
  p.n_seq = n_seq; p.drafts = max_draft; p.V = (int)V; p.blocks = (int)blocks;
  p.temps = temps; p.draft_temps = draft_temps; p.draft_logp = draft_logp; p.draft_tok = draft_tok; p.draft_len = draft_len;
  p.uniforms = uniforms; p.u_stride = uniform_stride;
  p.out_tok = out_tok; p.out_kept = out_kept; p.out_logp = out_logp; p.out_ent = out_ent;
  p.first = reinterpret_cast<int32_t *>(ws); p.arrived = reinterpret_cast<int32_t *>(ws + l.arrived);
  p.rows = reinterpret_cast<VerifyRow *>(ws + l.records); p.parts = reinterpret_cast<VerifyPart *>(ws + l.parts);
  p.sums = reinterpret_cast<float2 *>(ws + l.sums);
  cudaStream_t cs = static_cast<cudaStream_t>(stream);
  const cudaError_t e = dt == E3_F32 ? launch_verify<0>(p, cs) : launch_verify<1>(p, cs);
  return e == cudaSuccess ? E3_OK : E3_ERR_CUDA;
}
