// Scored router (mote_route_scored): logits, softmax or sigmoid scores, a bias that takes part in the choice alone,
// groups of experts, top-k, renormalised and scaled weights.
//
//   l = Wr x + logit_bias;  s = softmax(l) or 1 / (1 + exp(-l));  c = s + select_bias
//   groups: the topk_groups groups with the largest (sum of the two largest c) stay;  the k largest c among them are taken
//
// The choice is the one of exact arithmetic, whatever the order of the sums: scores are computed in fp32 with a bound on
// their error, and a token whose choice lies within the bound has the scores concerned evaluated once more in 64 bits
// (a few tokens in a thousand; see RouteDoubt).  So all paths, batch sizes and splits give the same experts.
//
// Logits: one cluster of CTAs per 16 tokens.  Each warp takes a part of the width and multiplies 16 tokens by all experts with
// warp-level bf16 MMAs; an fp32 router weight is split exactly into three bf16 terms (8 + 8 + 8 significand bits), so every
// product is exact and only the additions round.  The warps' sums meet in shared memory, the CTAs' in distributed shared
// memory (in rank order), and each CTA of the cluster then chooses for its share of the 16 tokens, a warp per token.
#include "mote_common.cuh"
#include "mote_internal.h"
#include "ptx_sm100.cuh"

namespace mote {

// What the selection needs of a router.
struct ScoredRouter {
  const uint16_t* x; int64_t ldx;       // tokens, for the second evaluation
  const void* Wr;                       // [E, d] fp32 or bf16
  const float* logit_bias; const float* select_bias;
  const float* w_norm;                  // largest 2-norm of a router row
  int64_t T;
  int d, E, k, sigmoid, n_groups, topk_groups, renorm, w_f32;
  float scale;
  int32_t* idx; float* w; float* logits;
};

// ------------------------------------------------------------------------------------------------
// Error bounds.  A product is exact, so a logit is off by the roundings of its partial sums.  These are no larger than
// |x|_2 |w|_2 (Cauchy-Schwarz), and the roundings of one sum are a few dozen of 2^-24 of the partial sum each, most of it far
// below that; kLogitEps |x|_2 |w|_2 is some 50 times what was seen.  (What all experts of a token have in common, as the truncation
// of the MMA's additions for operands of one sign, cancels in the comparison.)
// ------------------------------------------------------------------------------------------------
constexpr float kLogitEps = 9.5367432e-07f;            // 2^-20

// order-preserving integer images of floats; never 0, which marks an entry that cannot be taken
__device__ __forceinline__ uint32_t order_key(float v) {
  const uint32_t b = __float_as_uint(v + 0.0f);          // -0 counts as +0
  const uint32_t k = (b & 0x80000000u) ? ~b : b | 0x80000000u;
  return k ? k : 1u;
}
__device__ __forceinline__ uint64_t order_key(double v) {
  const uint64_t b = (uint64_t)__double_as_longlong(v + 0.0);
  const uint64_t k = (b >> 63) ? ~b : b | (1ull << 63);
  return k ? k : 1ull;
}
template <typename F> struct KeyOf { using type = uint32_t; };
template <> struct KeyOf<double> { using type = uint64_t; };

__device__ __forceinline__ uint32_t warp_max_key(uint32_t k) { return __reduce_max_sync(0xffffffffu, k); }
__device__ __forceinline__ uint64_t warp_max_key(uint64_t k) {
  const uint32_t hi = (uint32_t)(k >> 32);
  const uint32_t m = __reduce_max_sync(0xffffffffu, hi);
  const uint32_t lo = __reduce_max_sync(0xffffffffu, hi == m ? (uint32_t)k : 0u);
  return (uint64_t(m) << 32) | lo;
}

// The entry with the largest key of 64 (lane, and lane + 32 in the second slot); equal keys: the lower number.  -1 if all are 0.
template <typename K>
__device__ __forceinline__ int warp_argmax(K k0, K k1) {
  const K m = warp_max_key(k0 > k1 ? k0 : k1);
  if (m == 0) return -1;
  const unsigned b0 = __ballot_sync(0xffffffffu, k0 == m);
  if (b0) return __ffs(b0) - 1;
  return 31 + __ffs(__ballot_sync(0xffffffffu, k1 == m));
}
template <typename F>
__device__ __forceinline__ F entry(F v0, F v1, int e) {
  const F a = __shfl_sync(0xffffffffu, v0, e & 31), b = __shfl_sync(0xffffffffu, v1, e & 31);
  return e < 32 ? a : b;
}
__device__ __forceinline__ double warp_sum_f(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ float warp_sum_f(float v) { return warp_sum(v); }
__device__ __forceinline__ double warp_max_f(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmax(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
__device__ __forceinline__ float warp_max_f(float v) { return warp_max(v); }
__device__ __forceinline__ double exp_f(double v) { return exp(v); }
__device__ __forceinline__ float exp_f(float v) { return expf(v); }

// Chooses the experts of one token from its logits (a warp; lane holds experts lane and lane + 32; s_c: 64 values of the warp's
// own) and, unless a score comparison lies within the error bound, writes them.  F = float: `delta` bounds the error of a
// logit; returned is the set of experts whose logits have to be evaluated again (0: none, the choice stands).  F = double: the
// logits are exact for that purpose, the choice always stands.
template <typename F>
__device__ __forceinline__ uint64_t choose_experts(const ScoredRouter& r, int64_t token, F l0, F l1, float delta, F* s_c, int lane) {
  using K = typename KeyOf<F>::type;
  const int E = r.E, k = r.k;
  const bool v0 = lane < E, v1 = lane + 32 < E;
  const F kNone = F(-INFINITY);
  // scores
  F p0, p1;
  F smax = F(1);
  if (r.sigmoid) {
    p0 = F(1) / (F(1) + exp_f(-l0));
    p1 = F(1) / (F(1) + exp_f(-l1));
  } else {
    const F lm = warp_max_f(v0 ? (v1 ? (l0 > l1 ? l0 : l1) : l0) : kNone);
    p0 = v0 ? exp_f(l0 - lm) : F(0);
    p1 = v1 ? exp_f(l1 - lm) : F(0);
    const F den = warp_sum_f(p0 + p1);
    p0 /= den;
    p1 /= den;
    smax = F(1) / den;
  }
  // what the choice goes by.  Both scores grow with the logit: without a bias and without groups (whose sums need the
  // scores) the logits themselves are compared.
  const bool by_logit = !r.select_bias && r.n_groups == 1;
  F c0 = by_logit ? l0 : p0, c1 = by_logit ? l1 : p1;
  float bias_max = 0.0f;
  if (r.select_bias) {
    const float b0 = v0 ? r.select_bias[lane] : 0.0f, b1 = v1 ? r.select_bias[lane + 32] : 0.0f;
    c0 += b0;
    c1 += b1;
    // an expert barred by -inf takes no part in the rounding of the others
    bias_max = warp_max(fmaxf(fabsf(b0) < INFINITY ? fabsf(b0) : 0.0f, fabsf(b1) < INFINITY ? fabsf(b1) : 0.0f));
  }
  // bound on the error of c: of the logit through the score's slope, of expf and the divisions, of adding the bias
  float tau = 0.0f;
  if (sizeof(F) == 4) {
    tau = by_logit ? delta : r.sigmoid ? 0.25f * delta + 4.8e-7f : float(smax) * (2.0f * delta + 2e-6f);
    tau += 1.2e-7f * bias_max;
  }
  bool doubt_all = false;
  uint64_t eligible = ~0ull;
  if (r.n_groups > 1) {
    const int G = r.n_groups, per = E / G;
    __syncwarp();
    if (v0) s_c[lane] = c0;
    if (v1) s_c[lane + 32] = c1;
    __syncwarp();
    auto group_score = [&](int g) {
      F a = s_c[g * per], b = kNone;
      for (int i = 1; i < per; ++i) {
        const F v = s_c[g * per + i];
        if (v > a) { b = a; a = v; }
        else if (v > b) b = v;
      }
      return per > 1 ? a + b : a;
    };
    const F g0 = lane < G ? group_score(lane) : kNone, g1 = lane + 32 < G ? group_score(lane + 32) : kNone;
    K k0 = lane < G ? order_key(g0) : K(0), k1 = lane + 32 < G ? order_key(g1) : K(0);
    F last = kNone;
    eligible = 0ull;
    for (int j = 0; j < r.topk_groups; ++j) {
      const int g = warp_argmax(k0, k1);
      last = entry(g0, g1, g);
      if (lane == (g & 31)) { if (g < 32) k0 = K(0); else k1 = K(0); }
      eligible |= (per == 64 ? ~0ull : ((1ull << per) - 1ull)) << (g * per);
    }
    if (sizeof(F) == 4) {
      const int g = warp_argmax(k0, k1);
      if (g >= 0 && float(last - entry(g0, g1, g)) <= 4.0f * tau + 2.4e-7f * (fabsf(float(last)) < INFINITY ? fabsf(float(last)) : 0.0f))
        doubt_all = true;
    }
  }
  const bool e0 = v0 && ((eligible >> lane) & 1ull), e1 = v1 && ((eligible >> (lane + 32)) & 1ull);
  K k0 = e0 ? order_key(c0) : K(0), k1 = e1 ? order_key(c1) : K(0);
  int sel[MOTE_MAX_TOPK];
  F sp[MOTE_MAX_TOPK];
  unsigned m0 = 0u, m1 = 0u;                     // experts in doubt
  F sum = F(0);
#pragma unroll
  for (int j = 0; j < MOTE_MAX_TOPK; ++j) {
    if (j < k) {
      const int e = warp_argmax(k0, k1);
      sel[j] = e;
      sp[j] = entry(p0, p1, e);
      sum += sp[j];
      if (lane == (e & 31)) { if (e < 32) k0 = K(0); else k1 = K(0); }
      if (sizeof(F) == 4) {
        // entries still to come that are closer to this one than the errors allow: they and it are in doubt
        const F ce = entry(c0, c1, e);
        const unsigned b0 = __ballot_sync(0xffffffffu, k0 != K(0) && float(ce - c0) <= 2.0f * tau);
        const unsigned b1 = __ballot_sync(0xffffffffu, k1 != K(0) && float(ce - c1) <= 2.0f * tau);
        if (b0 | b1) {
          m0 |= b0; m1 |= b1;
          if (e < 32) m0 |= 1u << e; else m1 |= 1u << (e - 32);
        }
      }
    }
  }
  if (sizeof(F) == 4) {
    const uint64_t all = E == 64 ? ~0ull : (1ull << E) - 1ull;
    uint64_t doubt = (uint64_t(m1) << 32) | m0;
    // scores of a softmax share their denominator: exact differences need every logit
    if (doubt_all || (doubt && !r.sigmoid && !by_logit)) doubt = all;
    if (doubt) return doubt & all;
  }
  if (lane == 0) {
    const F div = r.renorm ? (sum > F(1e-20) ? sum : F(1e-20)) : F(1);
#pragma unroll
    for (int j = 0; j < MOTE_MAX_TOPK; ++j)
      if (j < k) {
        r.idx[token * k + j] = sel[j];
        r.w[token * k + j] = float(sp[j] / div) * r.scale;
      }
  }
  return 0ull;
}

// One logit in 64 bits (a warp).
__device__ __forceinline__ double exact_logit(const ScoredRouter& r, int64_t token, int e, int lane) {
  const uint4* x = reinterpret_cast<const uint4*>(r.x + token * r.ldx);
  double acc = 0.0;
  for (int v = lane; v < r.d / 8; v += 32) {
    const uint4 q = x[v];
    const float xv[8] = {bf16_lo(q.x), bf16_hi(q.x), bf16_lo(q.y), bf16_hi(q.y), bf16_lo(q.z), bf16_hi(q.z), bf16_lo(q.w), bf16_hi(q.w)};
    float wv[8];
    if (r.w_f32) {
      const float4* w = reinterpret_cast<const float4*>(static_cast<const float*>(r.Wr) + int64_t(e) * r.d) + 2 * v;
      const float4 a = w[0], b = w[1];
      wv[0] = a.x; wv[1] = a.y; wv[2] = a.z; wv[3] = a.w; wv[4] = b.x; wv[5] = b.y; wv[6] = b.z; wv[7] = b.w;
    } else {
      const uint4 w = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(r.Wr) + int64_t(e) * r.d)[v];
      wv[0] = bf16_lo(w.x); wv[1] = bf16_hi(w.x); wv[2] = bf16_lo(w.y); wv[3] = bf16_hi(w.y);
      wv[4] = bf16_lo(w.z); wv[5] = bf16_hi(w.z); wv[6] = bf16_lo(w.w); wv[7] = bf16_hi(w.w);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) acc = fma(double(xv[j]), double(wv[j]), acc);
  }
  acc = warp_sum_f(acc);
  return r.logit_bias ? acc + double(r.logit_bias[e]) : acc;
}

// Tokens whose choice is left open by the fp32 scores, kept until all tokens of the CTA are through; then its warps share the
// logits to be evaluated and each token gets its choice in 64 bits.
template <int kTokens>
struct RouteDoubt {
  int n;
  int token[kTokens];                            // number within the CTA's tokens
  uint64_t which[kTokens];
  double l[kTokens][64];
};

// All warps of the CTA; `first` is the token with number 0.
template <int kTokens>
__device__ __forceinline__ void settle_doubts(const ScoredRouter& r, int64_t first, RouteDoubt<kTokens>& q, double (*s_c)[64], int warp,
                                              int n_warps, int lane) {
  __syncthreads();
  const int n = q.n;
  if (n == 0) return;                            // uniform over the CTA
  int item = 0;
  for (int i = 0; i < n; ++i)
    for (uint64_t m = q.which[i]; m; m &= m - 1, ++item)
      if (item % n_warps == warp) {
        const int e = __ffsll((long long)m) - 1;
        const double l = exact_logit(r, first + q.token[i], e, lane);
        if (lane == 0) q.l[i][e] = l;
      }
  __syncthreads();
  for (int i = warp; i < n; i += n_warps) {
    const double l0 = lane < r.E ? q.l[i][lane] : 0.0, l1 = lane + 32 < r.E ? q.l[i][lane + 32] : 0.0;
    (void)choose_experts<double>(r, first + q.token[i], l0, l1, 0.0f, s_c[warp], lane);
  }
}

// The fp32 choice of one token, or its entry among those to be settled.
template <int kTokens>
__device__ __forceinline__ void choose_or_defer(const ScoredRouter& r, int64_t first, int number, float l0, float l1, float x_norm2,
                                                RouteDoubt<kTokens>& q, float* s_c, int lane) {
  const int64_t token = first + number;
  if (r.logits) {
    if (lane < r.E) r.logits[token * r.E + lane] = l0;
    if (lane + 32 < r.E) r.logits[token * r.E + lane + 32] = l1;
  }
  // (the logit bias, and the last rounding)
  const float l_max = warp_max(fmaxf(fabsf(l0) < INFINITY ? fabsf(l0) : 0.0f, fabsf(l1) < INFINITY ? fabsf(l1) : 0.0f));
  const float delta = kLogitEps * sqrtf(x_norm2) * *r.w_norm + 1.2e-7f * l_max;
  const uint64_t doubt = choose_experts<float>(r, token, l0, l1, delta, s_c, lane);
  if (doubt == 0ull) return;
  int slot = 0;
  if (lane == 0) {
    slot = atomicAdd(&q.n, 1);
    q.token[slot] = number;
    q.which[slot] = doubt;
  }
  slot = __shfl_sync(0xffffffffu, slot, 0);
  if (lane < r.E) q.l[slot][lane] = double(l0);
  if (lane + 32 < r.E) q.l[slot][lane + 32] = double(l1);
}

// ------------------------------------------------------------------------------------------------
// Logits by warp-level MMAs
// ------------------------------------------------------------------------------------------------
__device__ __forceinline__ void mma_bf16_k16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// upper halves of two floats -> bf16x2 (first in the low half)
__device__ __forceinline__ uint32_t upper_halves(float a, float b) { return __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x7632); }

__device__ __forceinline__ float ld_cluster_f32(uint32_t addr) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
  return v;
}

constexpr int kScoredWarps = 8;
constexpr int kScoredTokens = 16;

// NE: 8-expert column tiles (ceil(E / 8) rounded up to 1, 2, 4 or 8); kF32: type of the router weights.
// Lane (g, t) = (lane / 4, lane % 4) loads elements [32 * step + 8 * t, + 8) of token rows g and g + 8 and of router rows 8n + g;
// the reduction index may be permuted as long as both operands are.
template <int NE, bool kF32>
__global__ void __launch_bounds__(kScoredWarps * 32) route_scored_kernel(ScoredRouter r, int cluster) {
  __shared__ union {
    float part[kScoredWarps][NE * 4][32];
    struct { RouteDoubt<kScoredTokens> doubt; double c64[kScoredWarps][64]; } late;
  } sh;
  __shared__ float s_logits[kScoredTokens][NE * 8 + 1];
  __shared__ float s_norm[kScoredWarps][kScoredTokens];
  __shared__ float s_xx[kScoredTokens];
  __shared__ float s_c[kScoredWarps][64];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int rank = cluster > 1 ? (int)ptx::cluster_ctarank() : 0;
  const int64_t t0 = int64_t(blockIdx.x / cluster) * kScoredTokens;
  const int d = r.d, E = r.E;
  const int n_steps = (d + 31) / 32;
  const int parts = kScoredWarps * cluster, part = rank * kScoredWarps + warp;
  const int sb = int(int64_t(n_steps) * part / parts), se = int(int64_t(n_steps) * (part + 1) / parts);
  const bool ga = t0 + g < r.T, gb = t0 + g + 8 < r.T;
  const uint16_t* xa = r.x + (ga ? t0 + g : 0) * r.ldx + t * 8;
  const uint16_t* xb = r.x + (gb ? t0 + g + 8 : 0) * r.ldx + t * 8;
  float acc[NE][4];
#pragma unroll
  for (int n = 0; n < NE; ++n) acc[n][0] = acc[n][1] = acc[n][2] = acc[n][3] = 0.0f;
  float xxa = 0.0f, xxb = 0.0f;
  const uint4 kZero = make_uint4(0u, 0u, 0u, 0u);
  pdl_wait();
  constexpr int kAhead = 2;
  uint4 ra[kAhead], rb[kAhead];
#pragma unroll
  for (int i = 0; i < kAhead; ++i) {
    const bool in = sb + i < se && (sb + i) * 32 + t * 8 < d;
    ra[i] = in && ga ? *reinterpret_cast<const uint4*>(xa + (sb + i) * 32) : kZero;
    rb[i] = in && gb ? *reinterpret_cast<const uint4*>(xb + (sb + i) * 32) : kZero;
  }
  for (int s0 = sb; s0 < se; s0 += kAhead) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int s = s0 + i;
      if (s < se) {
        const uint4 ca = ra[i], cb = rb[i];
        {
          const bool in = s + kAhead < se && (s + kAhead) * 32 + t * 8 < d;
          ra[i] = in && ga ? *reinterpret_cast<const uint4*>(xa + (s + kAhead) * 32) : kZero;
          rb[i] = in && gb ? *reinterpret_cast<const uint4*>(xb + (s + kAhead) * 32) : kZero;
        }
        const bool in = s * 32 + t * 8 < d;
#pragma unroll
        for (int n = 0; n < NE; ++n) {
          const bool row = in && n * 8 + g < E;
          if (kF32) {
            float4 w0 = make_float4(0.f, 0.f, 0.f, 0.f), w1 = w0;
            if (row) {
              const float4* wp = reinterpret_cast<const float4*>(static_cast<const float*>(r.Wr) + int64_t(n * 8 + g) * d + s * 32 + t * 8);
              w0 = wp[0];
              w1 = wp[1];
            }
            const float w[8] = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w};
            float hi[8], mid[8], lo[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              hi[j] = __uint_as_float(__float_as_uint(w[j]) & 0xFFFF0000u);
              const float r1 = __fsub_rn(w[j], hi[j]);
              mid[j] = __uint_as_float(__float_as_uint(r1) & 0xFFFF0000u);
              lo[j] = __fsub_rn(r1, mid[j]);
            }
            mma_bf16_k16(acc[n], ca.x, cb.x, ca.y, cb.y, upper_halves(hi[0], hi[1]), upper_halves(hi[2], hi[3]));
            mma_bf16_k16(acc[n], ca.z, cb.z, ca.w, cb.w, upper_halves(hi[4], hi[5]), upper_halves(hi[6], hi[7]));
            mma_bf16_k16(acc[n], ca.x, cb.x, ca.y, cb.y, upper_halves(mid[0], mid[1]), upper_halves(mid[2], mid[3]));
            mma_bf16_k16(acc[n], ca.z, cb.z, ca.w, cb.w, upper_halves(mid[4], mid[5]), upper_halves(mid[6], mid[7]));
            mma_bf16_k16(acc[n], ca.x, cb.x, ca.y, cb.y, upper_halves(lo[0], lo[1]), upper_halves(lo[2], lo[3]));
            mma_bf16_k16(acc[n], ca.z, cb.z, ca.w, cb.w, upper_halves(lo[4], lo[5]), upper_halves(lo[6], lo[7]));
          } else {
            uint4 w = kZero;
            if (row) w = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(r.Wr) + int64_t(n * 8 + g) * d + s * 32 + t * 8);
            mma_bf16_k16(acc[n], ca.x, cb.x, ca.y, cb.y, w.x, w.y);
            mma_bf16_k16(acc[n], ca.z, cb.z, ca.w, cb.w, w.z, w.w);
          }
        }
        const uint32_t wa[4] = {ca.x, ca.y, ca.z, ca.w}, wb[4] = {cb.x, cb.y, cb.z, cb.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          xxa = fmaf(bf16_lo(wa[j]), bf16_lo(wa[j]), fmaf(bf16_hi(wa[j]), bf16_hi(wa[j]), xxa));
          xxb = fmaf(bf16_lo(wb[j]), bf16_lo(wb[j]), fmaf(bf16_hi(wb[j]), bf16_hi(wb[j]), xxb));
        }
      }
    }
  }
#pragma unroll
  for (int o = 1; o < 4; o <<= 1) {
    xxa += __shfl_xor_sync(0xffffffffu, xxa, o);
    xxb += __shfl_xor_sync(0xffffffffu, xxb, o);
  }
  if (t == 0) { s_norm[warp][g] = xxa; s_norm[warp][g + 8] = xxb; }
#pragma unroll
  for (int n = 0; n < NE; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) sh.part[warp][n * 4 + i][lane] = acc[n][i];
  __syncthreads();
  // fragment: value i of column tile n at lane (g, t) is token row g + 8*(i/2), expert 8n + 2t + (i&1)
  for (int v = warp; v < NE * 4; v += kScoredWarps) {
    float z = sh.part[0][v][lane];
#pragma unroll
    for (int w = 1; w < kScoredWarps; ++w) z += sh.part[w][v][lane];
    s_logits[g + 8 * ((v & 3) >> 1)][(v >> 2) * 8 + 2 * t + (v & 1)] = z;
  }
  if (threadIdx.x < kScoredTokens) {
    float z = s_norm[0][threadIdx.x];
#pragma unroll
    for (int w = 1; w < kScoredWarps; ++w) z += s_norm[w][threadIdx.x];
    s_xx[threadIdx.x] = z;
  }
  __syncthreads();                               // sh.part has been read: sh.late may take its place
  if (threadIdx.x == 0) sh.late.doubt.n = 0;
  if (cluster > 1) ptx::cluster_sync();
  else __syncthreads();
  const int share = kScoredTokens / cluster;     // tokens this CTA chooses for
  for (int i = warp; i < share; i += kScoredWarps) {
    const int number = rank * share + i;
    if (t0 + number >= r.T) break;               // whole warp
    float l0 = 0.0f, l1 = 0.0f, xx = 0.0f;
    if (cluster > 1) {
      const uint32_t a0 = ptx::smem_u32(&s_logits[number][lane < NE * 8 ? lane : 0]);
      const uint32_t a1 = ptx::smem_u32(&s_logits[number][(lane + 32) % (NE * 8)]);
      const uint32_t ax = ptx::smem_u32(&s_xx[number]);
      for (int c = 0; c < cluster; ++c) {
        l0 += ld_cluster_f32(ptx::map_to_rank(a0, c));
        if (NE > 4) l1 += ld_cluster_f32(ptx::map_to_rank(a1, c));
        xx += ld_cluster_f32(ptx::map_to_rank(ax, c));
      }
    } else {
      l0 = s_logits[number][lane < NE * 8 ? lane : 0];
      if (NE > 4) l1 = s_logits[number][(lane + 32) % (NE * 8)];
      xx = s_xx[number];
    }
    if (r.logit_bias) {
      if (lane < E) l0 += r.logit_bias[lane];
      if (lane + 32 < E) l1 += r.logit_bias[lane + 32];
    }
    choose_or_defer(r, t0, number, l0, l1, xx, sh.late.doubt, s_c[warp], lane);
  }
  if (cluster > 1) ptx::cluster_sync();          // nobody leaves while its sums are being read
  settle_doubts(r, t0, sh.late.doubt, sh.late.c64, warp, kScoredWarps, lane);
}

// Largest 2-norm of a router row, rounded up.  One CTA; an offline step.
__global__ void __launch_bounds__(1024) router_pack_kernel(const void* __restrict__ Wr, int w_f32, int E, int d, float* __restrict__ norm) {
  __shared__ float s_max[32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  float worst = 0.0f;
  for (int e = warp; e < E; e += 32) {
    double ss = 0.0;
    for (int j = lane; j < d; j += 32) {
      const float w = w_f32 ? static_cast<const float*>(Wr)[int64_t(e) * d + j]
                            : __uint_as_float(uint32_t(static_cast<const uint16_t*>(Wr)[int64_t(e) * d + j]) << 16);
      ss = fma(double(w), double(w), ss);
    }
    worst = fmaxf(worst, __double2float_ru(sqrt(warp_sum_f(ss))));
  }
  if (lane == 0) s_max[warp] = worst;
  __syncthreads();
  if (warp == 0) {
    worst = warp_max(s_max[lane]);
    if (lane == 0) norm[0] = worst;
  }
}

// Pairs of every expert in each block of kRouteBlockTokens tokens, as the block-wise dispatch takes them (a CTA per block).
__global__ void __launch_bounds__(MOTE_MAX_EXPERTS) block_counts_kernel(const int32_t* __restrict__ idx, int64_t P, int E, int k,
                                                                        int32_t* __restrict__ blk_hist, int n_blk) {
  __shared__ int s_idx[kRouteBlockTokens * MOTE_MAX_TOPK];
  pdl_wait();
  const int64_t p0 = int64_t(blockIdx.x) * kRouteBlockTokens * k;
  const int n = (int)min(int64_t(kRouteBlockTokens * k), P - p0);
  for (int i = threadIdx.x; i < n; i += MOTE_MAX_EXPERTS) s_idx[i] = idx[p0 + i];
  __syncthreads();
  const int e = threadIdx.x;
  if (e >= E) return;
  int c = 0;
  for (int i = 0; i < n; ++i) c += s_idx[i] == e ? 1 : 0;
  blk_hist[int64_t(e) * blk_stride(n_blk) + blockIdx.x] = c;
}

mote_status_t launch_block_counts(const int32_t* idx, int64_t T, int E, int k, int32_t* blk_hist, cudaStream_t stream) {
  const int n_blk = (int)((T + kRouteBlockTokens - 1) / kRouteBlockTokens);
  MOTE_CUDA_OK(launch_pdl(block_counts_kernel, dim3(n_blk), dim3(MOTE_MAX_EXPERTS), 0, stream, idx, T * k, E, k, blk_hist, n_blk));
  ++g_launch_count;
  MOTE_LAUNCH_OK();
  return MOTE_OK;
}

static bool router_ok(const mote_router_t* R) {
  return R->d > 0 && R->d % 8 == 0 && R->d <= 32768 && R->E >= 1 && R->E <= MOTE_MAX_EXPERTS && R->k >= 1 && R->k <= R->E &&
         R->k <= MOTE_MAX_TOPK && (R->scoring == MOTE_SCORE_SOFTMAX || R->scoring == MOTE_SCORE_SIGMOID) && R->n_groups >= 1 &&
         R->n_groups <= R->E && R->E % R->n_groups == 0 && R->topk_groups >= 1 && R->topk_groups <= R->n_groups &&
         R->k <= R->topk_groups * (R->E / R->n_groups) && R->scale == R->scale;
}

template <int NE>
static cudaError_t launch_scored(const ScoredRouter& r, unsigned tiles, int cluster, cudaStream_t stream) {
  return r.w_f32 ? launch_ex(route_scored_kernel<NE, true>, dim3(tiles * cluster), dim3(kScoredWarps * 32), 0, stream, true, cluster, r, cluster)
                 : launch_ex(route_scored_kernel<NE, false>, dim3(tiles * cluster), dim3(kScoredWarps * 32), 0, stream, true, cluster, r, cluster);
}

mote_status_t launch_route_scored(const mote_router_t* R, const void* x, int64_t ldx, int64_t T, int32_t* idx, float* w, float* logits,
                                  cudaStream_t stream) {
  ScoredRouter r{};
  r.x = static_cast<const uint16_t*>(x); r.ldx = ldx; r.Wr = R->Wr; r.logit_bias = R->logit_bias; r.select_bias = R->select_bias;
  r.w_norm = static_cast<const float*>(R->packed);
  r.T = T; r.d = R->d; r.E = R->E; r.k = R->k; r.sigmoid = R->scoring == MOTE_SCORE_SIGMOID; r.n_groups = R->n_groups;
  r.topk_groups = R->topk_groups; r.renorm = R->renorm != 0; r.w_f32 = R->w_dtype == MOTE_DTYPE_F32; r.scale = R->scale;
  r.idx = idx; r.w = w; r.logits = logits;
  const unsigned tiles = (unsigned)((T + kScoredTokens - 1) / kScoredTokens);
  int cluster = 1;                               // CTAs that share a tile's width: as many as the SMs allow
  while (cluster < 8 && int64_t(tiles) * cluster * 2 <= device_sm_count()) cluster *= 2;
  const int ne = (R->E + 7) / 8;
  MOTE_CUDA_OK(ne <= 1   ? launch_scored<1>(r, tiles, cluster, stream)
               : ne <= 2 ? launch_scored<2>(r, tiles, cluster, stream)
               : ne <= 4 ? launch_scored<4>(r, tiles, cluster, stream) : launch_scored<8>(r, tiles, cluster, stream));
  ++g_launch_count;
  MOTE_LAUNCH_OK();
  return MOTE_OK;
}

// Argument checks shared by the calls that take a router.
mote_status_t check_router(const mote_router_t* R) {
  if (!R) return MOTE_ERR_NULL;
  if (!router_ok(R)) return MOTE_ERR_SHAPE;
  if (R->w_dtype != MOTE_DTYPE_F32 && R->w_dtype != MOTE_DTYPE_BF16) return MOTE_ERR_DTYPE;
  if (!R->Wr || !R->packed) return MOTE_ERR_NULL;
  if (!aligned16(R->Wr) || (reinterpret_cast<uintptr_t>(R->packed) & 255u) != 0) return MOTE_ERR_ALIGN;
  return MOTE_OK;
}

}  // namespace mote

extern "C" size_t mote_router_pack_bytes(int E, int64_t d, int w_dtype) {
  if (E < 1 || E > MOTE_MAX_EXPERTS || d <= 0 || d % 8 != 0 || d > 32768) return 0;
  if (w_dtype != MOTE_DTYPE_F32 && w_dtype != MOTE_DTYPE_BF16) return 0;
  return 256;
}

extern "C" mote_status_t mote_router_pack(const void* Wr, int w_dtype, int E, int64_t d, void* packed, size_t packed_bytes, void* stream) {
  using namespace mote;
  if (w_dtype != MOTE_DTYPE_F32 && w_dtype != MOTE_DTYPE_BF16) return MOTE_ERR_DTYPE;
  const size_t need = mote_router_pack_bytes(E, d, w_dtype);
  if (need == 0) return MOTE_ERR_SHAPE;
  if (!Wr || !packed) return MOTE_ERR_NULL;
  if (!aligned16(Wr) || (reinterpret_cast<uintptr_t>(packed) & 255u) != 0) return MOTE_ERR_ALIGN;
  if (packed_bytes < need) return MOTE_ERR_WORKSPACE;
  router_pack_kernel<<<1, 1024, 0, static_cast<cudaStream_t>(stream)>>>(Wr, w_dtype == MOTE_DTYPE_F32, E, (int)d, static_cast<float*>(packed));
  MOTE_LAUNCH_OK();
  return MOTE_OK;
}

extern "C" mote_status_t mote_route_scored(const mote_router_t* R, const void* x, int64_t ldx, int64_t T, int32_t* topk_idx, float* topk_w,
                                           float* logits, void* stream) {
  using namespace mote;
  const mote_status_t st = check_router(R);
  if (st) return st;
  if (T < 0 || T > (int64_t(1) << 24) || (T > 1 && ldx < R->d)) return MOTE_ERR_SHAPE;
  if (T == 0) return MOTE_OK;
  if (!x || !topk_idx || !topk_w) return MOTE_ERR_NULL;
  if (!aligned16(x) || (T > 1 && ldx % 8 != 0)) return MOTE_ERR_ALIGN;
  return launch_route_scored(R, x, ldx, T, topk_idx, topk_w, logits, static_cast<cudaStream_t>(stream));
}
