// Scored router (mote_route_scored): logits, softmax or sigmoid scores, a bias that takes part in the choice alone,
// groups of experts, top-k, renormalised and scaled weights.
//
//   l = Wr x + logit_bias;  s = softmax(l) or 1 / (1 + exp(-l));  c = s + select_bias
//   groups: the topk_groups groups with the largest (sum of the two largest c) stay;  the k largest c among them are taken
//
// The choice is the one of exact arithmetic, whatever the order of the sums: scores are computed in fp32 with a bound on
// their error, and a token whose choice lies within the bound has the scores concerned evaluated once more in 64 bits (see
// Doubt; one token in a hundred of normal ones, more where logits lie close together, all where saturated scores make
// more than kMaxBorder groups alike).  So all paths, batch sizes and splits give the same experts.
//
// Logits: one cluster of CTAs per 16 tokens.  Each warp takes a part of the width and multiplies 16 tokens by all experts with
// warp-level bf16 MMAs; an fp32 router weight is split exactly into three bf16 terms (8 + 8 + 8 significand bits), so every
// product is exact and only the additions round.  The warps' sums meet in shared memory, the CTAs' in distributed shared
// memory (in rank order), and each CTA of the cluster then chooses for its share of the 16 tokens.
#include <algorithm>

#include "mote_common.cuh"
#include "mote_internal.h"
#include "ptx_sm100.cuh"
#include "tile_launch.cuh"

namespace mote {

// What the selection needs of a router.
struct ScoredRouter {
  const uint16_t* x; int64_t ldx;       // tokens, for the second evaluation
  const void* Wr;                       // [E, d] fp32 or bf16
  const float* logit_bias; const float* select_bias;
  const float* w_norm;                  // largest 2-norm of a router row
  int64_t T;
  int d, E, k, sigmoid, n_groups, per_group, topk_groups, renorm, w_f32;
  float scale;
  int32_t* idx; float* w; float* logits;
};

// ------------------------------------------------------------------------------------------------
// Error bounds.  A product is exact, so a logit is off by what its additions lose.  Sums are bounded by sum |x_i w_i| <= |x|_2 |w|_2, for the
// parts of the width together too (Cauchy-Schwarz), so a bound relative to a part's own norms holds for the whole.  In units of 2^-24:
//   * A tensor-core instruction brings its 16 products and the sum so far to one scale, cuts each off 25 bits below the largest, and cuts
//     the result to 24 bits (found by sums of 1 and n products of 2^-j, the same for mma.sync and tcgen05): 17 addends of half a
//     unit, a result of two: 10.5 for 16 elements.  The weights' upper terms come last; what the middle and lower ones, 2^-7 and less of
//     the weights, lose on the way is 0.4.
//   * A sum by warp-level MMAs is of 16 elements, and two of them are added (1); one by tcgen05.mma is of 32, two instructions (21), and two
//     of them are added (1).  These sums are added up with compensation (Kahan: 2, however many they are).  The parts of warps and CTAs
//     meet in pairs of floats (Knuth's two-sum: of second order), which become one float where a CTA hands over its part and as the
//     logit: 2.
//   * The addition of logit_bias: 1, and 2 of the bias.
// Products of random signs lose one or two in all.
// ------------------------------------------------------------------------------------------------
constexpr float kUnit = 1.0f / 16777216.0f;
constexpr float kWarpLogitEps = 17.5f * kUnit, kTileLogitEps = 27.0f * kUnit;      // 16.9 and 26.4, and what the norms may be off by

// hi + lo += v, lo being what the additions to hi have lost (exactly, for each).
__device__ __forceinline__ void two_sum(float& hi, float& lo, float v) {
  const float s = __fadd_rn(hi, v), part = __fsub_rn(s, hi);
  lo = __fadd_rn(lo, __fadd_rn(__fsub_rn(hi, __fsub_rn(s, part)), __fsub_rn(v, part)));
  hi = s;
}
__device__ __forceinline__ uint64_t sub_f32x2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(b), "l"(f32x2(-1.0f, -1.0f)), "l"(a));
  return d;
}
// sum += v, two at a time; over: what `sum` holds too much.
__device__ __forceinline__ void compensated_add(uint64_t& sum, uint64_t& over, uint64_t v) {
  const uint64_t y = sub_f32x2(v, over), t = add_f32x2(sum, y);
  over = sub_f32x2(sub_f32x2(t, sum), y);
  sum = t;
}

// order-preserving integer images of floats and doubles; never 0, which marks an entry that cannot be taken
__device__ __forceinline__ uint32_t order_key(float v) {
  const uint32_t b = __float_as_uint(v + 0.0f);          // -0 counts as +0
  const uint32_t k = (b & 0x80000000u) ? ~b : b | 0x80000000u;
  return k ? k : 1u;
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? k & 0x7FFFFFFFu : ~k); }
__device__ __forceinline__ uint64_t order_key(double v) {
  const uint64_t b = (uint64_t)__double_as_longlong(v + 0.0);
  const uint64_t k = (b >> 63) ? ~b : b | (1ull << 63);
  return k ? k : 1ull;
}
__device__ __forceinline__ double warp_sum_f64(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ float finite_abs(float v) { return fabsf(v) < INFINITY ? fabsf(v) : 0.0f; }

// ------------------------------------------------------------------------------------------------
// The choice from fp32 sums: a warp to a token, experts lane and lane + 32 to a lane.  It is a chain of dependent steps, so its latency counts:
// maxima are single warp reductions of integer images of the scores.  Loops stay loops: every SM runs through this code a few times
// only, and fetching it takes time too.  (Four or eight lanes to a token, 16 or 8 experts to a lane: 20 000 cycles a token, and no
// faster for the 64 tokens that a CTA has in a long batch.)
// ------------------------------------------------------------------------------------------------
// Up to 64 entries, two to a lane, the larger one first; key 0: none.
struct Entries {
  uint32_t hi, lo;
  int hi_id, lo_id;
  __device__ __forceinline__ Entries(uint32_t k0, uint32_t k1, int lane) {
    const bool swap = k1 > k0;
    hi = swap ? k1 : k0; hi_id = swap ? lane + 32 : lane;
    lo = swap ? k0 : k1; lo_id = swap ? lane : lane + 32;
  }
  // takes out the one with the largest key (of equal ones any: they are in doubt, but for -inf, whose keys differ)
  __device__ __forceinline__ int take(uint32_t& best, int lane) {
    best = __reduce_max_sync(0xffffffffu, hi);
    const int from = __ffs(__ballot_sync(0xffffffffu, hi == best)) - 1;
    const int id = __shfl_sync(0xffffffffu, hi_id, from);
    if (lane == from) { hi = lo; hi_id = lo_id; lo = 0u; }
    return id;
  }
};
// order_key, and -inf ordered by index (decided, where other equal values are in doubt)
__device__ __forceinline__ uint32_t entry_key(float v, int id) { return order_key(v) - (v == -INFINITY ? (uint32_t)id : 0u); }

constexpr int kMaxBorder = 8;                      // groups at the border that are told apart by the scores concerned

// What is known of a token whose choice the fp32 scores leave open.
struct Doubt {
  int token;                                       // number within the CTA's tokens
  int full;                                        // 1: all logits and the whole choice anew
  uint64_t border, kept;                           // groups too close to the border to tell which stay (none: 0); groups that the fp32 scores keep
  float l_max, inv_den, den_rel;                   // softmax: what is taken off the logits, 1 / denominator and the bound on its relative error
  uint64_t which;                                  // experts whose order is open
  uint64_t settled;                                // experts whose logits are evaluated in 64 bits: those, and the groups'
  uint64_t chosen;                                 // the fp32 choice, six bits each
};

// 1 / x of the special-function unit: 2^-23 off, as the library's e^x is (2 ulp; __expf, whose error grows with |x|, is no faster here).
__device__ __forceinline__ float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float sqrt_approx(float x) {
  float y;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// What a lane holds of the router: the biases and groups of its two experts, and the biases' largest magnitudes over all experts.
struct LaneBias {
  float s0 = 0.0f, s1 = 0.0f, select_max = 0.0f, logit_max = 0.0f;
  int group0 = 0, group1 = 0;
  __device__ __forceinline__ void load(const ScoredRouter& r, int lane) {
    const bool v0 = lane < r.E, v1 = lane + 32 < r.E;
    float l0 = 0.0f, l1 = 0.0f;
    if (r.select_bias) {
      if (v0) s0 = r.select_bias[lane];
      if (v1) s1 = r.select_bias[lane + 32];
    }
    if (r.logit_bias) {
      if (v0) l0 = r.logit_bias[lane];
      if (v1) l1 = r.logit_bias[lane + 32];
    }
    // (an expert barred by -inf takes no part in the rounding of the others)
    group0 = lane / r.per_group;
    group1 = (lane + 32) / r.per_group;
    select_max = warp_max(fmaxf(finite_abs(s0), finite_abs(s1)));
    logit_max = warp_max(fmaxf(finite_abs(l0), finite_abs(l1)));
  }
};

// Chooses for one token (a warp) from its logits l0, l1 (off by up to `delta`) and, unless a comparison lies within the error bound, writes
// the choice.  s_c: 64 floats of the warp's own.  Returned: in `d` what is in doubt (settled = 0: nothing, the choice stands), and the
// scores of the lane's experts.
__device__ __forceinline__ void choose_experts(const ScoredRouter& r, const LaneBias& bias, int64_t token, float l0, float l1, float delta,
                                               float* s_c, Doubt& d, float& p0, float& p1, int lane) {
  const int E = r.E, k = r.k;
  const bool v0 = lane < E, v1 = lane + 32 < E;
  // Both scores grow with the logit: without a bias logits are compared, except for the groups, whose sums need the scores.  Sums of a
  // softmax's are then compared relative to their size (the denominator cancels).
  const bool by_logit = !r.select_bias && r.n_groups == 1, ratios = !r.sigmoid && !r.select_bias;
  float smax = 1.0f;
  d.l_max = d.inv_den = d.den_rel = 0.0f;
  if (r.sigmoid) {
    p0 = rcp_approx(1.0f + expf(-l0));
    p1 = rcp_approx(1.0f + expf(-l1));
  } else {
    const float lm = fmaxf(warp_max(fmaxf(v0 ? l0 : -INFINITY, v1 ? l1 : -INFINITY)), -3.4e38f);      // (all barred: scores of 0)
    p0 = v0 ? expf(l0 - lm) : 0.0f;
    p1 = v1 ? expf(l1 - lm) : 0.0f;
    smax = rcp_approx(fmaxf(warp_sum(p0 + p1), 1.0f));             // (1 is the largest one's part; less where all are barred)
    d.l_max = lm;
    d.inv_den = smax;
    d.den_rel = delta < 1.0f ? delta * (1.0f + delta) + 4e-6f : 1e30f;      // e^delta - 1
    p0 *= smax;
    p1 *= smax;
  }
  const float c0 = (by_logit ? l0 : p0) + bias.s0, c1 = (by_logit ? l1 : p1) + bias.s1;
  // bound on the error of c: of the logit through the score's slope, of expf and the reciprocal, of adding the bias
  float tau = (by_logit ? delta : r.sigmoid ? 0.25f * delta + 4.8e-7f : delta < 0.5f ? smax * (2.0f * delta * (1.0f + 2.0f * delta) + 4e-6f) : 1e30f) + 1.2e-7f * bias.select_max;
  uint32_t k0 = v0 ? entry_key(c0, lane) : 0u, k1 = v1 ? entry_key(c1, lane + 32) : 0u, best;
  d.full = 0;
  d.which = d.settled = 0ull;
  d.border = 0ull;
  if (r.n_groups > 1) {
    const int G = r.n_groups, per = r.per_group;
    __syncwarp();
    s_c[lane] = c0;
    s_c[lane + 32] = c1;
    __syncwarp();
    uint32_t g0 = 0u, g1 = 0u;                     // keys of groups lane and lane + 32
    float second0 = 0.0f, second1 = 0.0f;          // the smaller of the scores that they are made of
#pragma unroll 1
    for (int g = lane; g < G; g += 32) {
      float a = s_c[g * per], b = -INFINITY;
#pragma unroll 4
      for (int m = 1; m < per; ++m) {
        const float v = s_c[g * per + m];
        b = fmaxf(b, fminf(a, v));
        a = fmaxf(a, v);
      }
      const float second = per > 1 ? b : a;
      const uint32_t key = entry_key(per > 1 ? a + b : a, g);
      if (g < 32) { g0 = key; second0 = second; } else { g1 = key; second1 = second; }
    }
    uint64_t kept = 0ull;
    uint32_t last = 0u;
    Entries groups(g0, g1, lane);
#pragma unroll 1
    for (int j = 0; j < r.topk_groups; ++j) kept |= 1ull << groups.take(last, lane);
    if (r.topk_groups < G) {
      groups.take(best, lane);
      const float worst = key_value(last), bound = delta > 1e30f ? 1e30f : delta;     // (infinite for a norm beyond fp32; 0 times it is 0)
      float reach = 4.0f * tau + 2.4e-7f * finite_abs(worst), two_taus = 2.0f * tau;
      if (ratios) {
        // e^x is off by its logit's error and by a few 2^-24 |x| (x: the logit less the largest one), relative to its size; a sum's |x| is
        // that of its larger part, no more than |log(sum / largest score)| + 1 and, weighted, as much again for the smaller part.  The
        // last part: scores too small for fp32.
        const float rel = bound + 1e-6f + 2e-7f * fminf(1.0f - __logf(fmaxf(worst / smax, 1e-38f)), 110.0f);
        reach = rel * (worst + key_value(best)) + 1e-36f;
        two_taus = 0.0f;                           // (the floors below are relative too)
      }
      if (worst - key_value(best) <= reach) {
        // The last group that stays and the first one left out are too close.  Of the groups around the border, the scores that their
        // sums may be made of are evaluated; where those are many: everything.
        const float lo = key_value(best) - reach, hi = worst + reach;
        auto at_border = [&](uint32_t key) { return key != 0u && key_value(key) >= lo && key_value(key) <= hi; };
        d.border = uint64_t(__ballot_sync(0xffffffffu, at_border(g1))) << 32 | __ballot_sync(0xffffffffu, at_border(g0));
        d.kept = kept;
        if (__popcll(d.border) > kMaxBorder) {
          d.full = 1;
        } else {
          const float shrink = ratios ? 1.0f - 2.0f * (bound + 3e-5f) : 1.0f;
          second0 = second0 * shrink - two_taus;   // floors
          second1 = second1 * shrink - two_taus;
          auto part_of = [&](bool there, int g, float c) {
            const float a = __shfl_sync(0xffffffffu, second0, g & 31), b = __shfl_sync(0xffffffffu, second1, g & 31);
            return there && ((d.border >> g) & 1ull) && c >= (g < 32 ? a : b);
          };
          const bool part0 = part_of(v0, bias.group0, c0), part1 = part_of(v1, bias.group1, c1);
          d.settled = uint64_t(__ballot_sync(0xffffffffu, part1)) << 32 | __ballot_sync(0xffffffffu, part0);
        }
      }
    }
    if (!r.select_bias) {
      k0 = v0 ? entry_key(l0, lane) : 0u;
      k1 = v1 ? entry_key(l1, lane + 32) : 0u;
      tau = delta;
    }
    if (!((kept >> bias.group0) & 1ull)) k0 = 0u;
    if (!((kept >> bias.group1) & 1ull)) k1 = 0u;
  }
  // a barred logit comes last, whatever its bias for the choice
  if (l0 == -INFINITY && k0) k0 = entry_key(-INFINITY, lane);
  if (l1 == -INFINITY && k1) k1 = entry_key(-INFINITY, lane + 32);
  // The k largest: lane j keeps the j-th and its key.
  Entries rest(k0, k1, lane);
  uint32_t key = 0u;
  int expert = 0;
#pragma unroll 1
  for (int j = 0; j < k; ++j) {
    const int e = rest.take(best, lane);
    if (lane == j) { key = best; expert = e; }
  }
  // Closer to the choice before than the errors allow?  All choices before that one are larger still; those not taken follow the last one.
  // (equal -inf are decided)
  auto is_near = [&](uint32_t key, uint32_t before) {
    const float c = key_value(key);
    return key != 0u && c > -INFINITY && key_value(before) - c <= 2.0f * tau;
  };
  const uint32_t before = __shfl_up_sync(0xffffffffu, key, 1);
  const bool near = lane > 0 && is_near(key, before), near_hi = is_near(rest.hi, best);
  if (__any_sync(0xffffffffu, near || near_hi) || d.full || d.border) {
    // those experts, and the choices before them
    const int prev = __shfl_up_sync(0xffffffffu, expert, 1), last = __shfl_sync(0xffffffffu, expert, k - 1);
    uint64_t which = 0ull;
    if (near) which |= 1ull << expert | 1ull << prev;
    if (near_hi) which |= 1ull << rest.hi_id | 1ull << last;
    if (is_near(rest.lo, best)) which |= 1ull << rest.lo_id;
    const uint64_t chosen = lane < k ? uint64_t(expert) << (6 * lane) : 0ull;
    auto all_of = [](uint64_t m) {
      return uint64_t(__reduce_or_sync(0xffffffffu, uint32_t(m >> 32))) << 32 | __reduce_or_sync(0xffffffffu, uint32_t(m));
    };
    d.chosen = all_of(chosen);
    d.which = which = all_of(which);
    d.settled |= which;
    if (d.full || !d.settled) { d.full = 1; d.settled = E == 64 ? ~0ull : (1ull << E) - 1ull; }      // (none: NaN)
    return;
  }
  const float a = __shfl_sync(0xffffffffu, p0, expert & 31), b = __shfl_sync(0xffffffffu, p1, expert & 31);
  const float p = lane < k ? (expert < 32 ? a : b) : 0.0f;
  float mul = r.scale;
  if (r.renorm) {
    static_assert(MOTE_MAX_TOPK <= 8, "the choice in lanes 0 to 7");
    float sum = p;
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    mul *= rcp_approx(fmaxf(sum, 1e-20f));
  }
  if (lane < k) {
    r.idx[token * k + lane] = expert;
    r.w[token * k + lane] = p * mul;
  }
}

// A logit in 64 bits, by four warps a quarter each: its latency is what a long batch waits for.
__device__ __forceinline__ void load8_router(const ScoredRouter& r, int e, int v, float (&w)[8]) {
  if (r.w_f32) {
    const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(r.Wr) + int64_t(e) * r.d) + 2 * v;
    const float4 a = p[0], b = p[1];
    w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w; w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
  } else {
    const uint4 q = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(r.Wr) + int64_t(e) * r.d)[v];
    w[0] = bf16_lo(q.x); w[1] = bf16_hi(q.x); w[2] = bf16_lo(q.y); w[3] = bf16_hi(q.y);
    w[4] = bf16_lo(q.z); w[5] = bf16_hi(q.z); w[6] = bf16_lo(q.w); w[7] = bf16_hi(q.w);
  }
}
__device__ __forceinline__ double logit_quarter(const ScoredRouter& r, int64_t token, int e, int quarter, int lane) {
  const uint4* x = reinterpret_cast<const uint4*>(r.x + token * r.ldx);
  const int n_vec = r.d / 8, per = (n_vec + 3) / 4, end = min((quarter + 1) * per, n_vec);
  double acc[4] = {0.0, 0.0, 0.0, 0.0};
#pragma unroll 1
  for (int v0 = quarter * per + lane; v0 < end; v0 += 64) {      // two vectors' loads on their way at a time
    uint4 q[2];
    float w[2][8];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int v = v0 + 32 * i;
      q[i] = make_uint4(0u, 0u, 0u, 0u);
      if (v < end) q[i] = x[v];
      load8_router(r, e, min(v, n_vec - 1), w[i]);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float xv[8] = {bf16_lo(q[i].x), bf16_hi(q[i].x), bf16_lo(q[i].y), bf16_hi(q[i].y),
                           bf16_lo(q[i].z), bf16_hi(q[i].z), bf16_lo(q[i].w), bf16_hi(q[i].w)};
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j & 3] = fma(double(xv[j]), double(w[i][j]), acc[j & 3]);
    }
  }
  return warp_sum_f64((acc[0] + acc[1]) + (acc[2] + acc[3]));
}

// Tokens whose choice is left open by the fp32 scores, kept until all tokens of the CTA are through; then its warps share the logits to be
// evaluated, and a warp settles each token.
template <int kTokens>
struct RouteDoubts {
  int n;
  Doubt d[kTokens];
  float p[kTokens][64];                            // fp32 scores
  double l[kTokens][64];                           // exact logits of the experts in doubt
  double quarter[32];                              // a quarter of a sum from each warp
};

// The whole choice in 64 bits (a warp; lane holds experts lane and lane + 32): slots of the lane's experts, -1 if they are not taken.
__device__ __noinline__ void choose_exactly(const ScoredRouter& r, double l0, double l1, double* s_c, int lane, int& slot0, int& slot1) {
  const int E = r.E;
  const bool v0 = lane < E, v1 = lane + 32 < E;
  double c0 = l0, c1 = l1;
  if (r.select_bias || r.n_groups > 1) {
    if (r.sigmoid) {
      c0 = 1.0 / (1.0 + exp(-l0));
      c1 = 1.0 / (1.0 + exp(-l1));
    } else {
      double lm = fmax(v0 ? l0 : -INFINITY, v1 ? l1 : -INFINITY);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) lm = fmax(lm, __shfl_xor_sync(0xffffffffu, lm, o));
      lm = fmax(lm, -1e300);                       // (all barred: scores of 0)
      c0 = v0 ? exp(l0 - lm) : 0.0;
      c1 = v1 ? exp(l1 - lm) : 0.0;
      const double den = r.select_bias ? fmax(warp_sum_f64(c0 + c1), 1.0) : 1.0;
      c0 /= den;
      c1 /= den;
    }
  }
  if (r.select_bias) {
    if (v0) c0 += double(r.select_bias[lane]);
    if (v1) c1 += double(r.select_bias[lane + 32]);
  }
  // the entry with the largest key of 64, of equal ones the lower
  auto argmax = [&](uint64_t k0, uint64_t k1) {
    const uint64_t key = k0 > k1 ? k0 : k1;
    const uint32_t hi = __reduce_max_sync(0xffffffffu, (uint32_t)(key >> 32));
    const uint32_t lo = __reduce_max_sync(0xffffffffu, (uint32_t)(key >> 32) == hi ? (uint32_t)key : 0u);
    const uint64_t best = uint64_t(hi) << 32 | lo;
    const unsigned b0 = __ballot_sync(0xffffffffu, k0 == best), b1 = __ballot_sync(0xffffffffu, k1 == best);
    return b0 ? __ffs(b0) - 1 : 31 + __ffs(b1);
  };
  uint64_t k0 = v0 ? order_key(c0) : 0ull, k1 = v1 ? order_key(c1) : 0ull;
  if (r.n_groups > 1) {
    const int G = r.n_groups, per = r.per_group;
    __syncwarp();
    s_c[lane] = c0;
    s_c[lane + 32] = c1;
    __syncwarp();
    uint64_t g0 = 0ull, g1 = 0ull;
#pragma unroll 1
    for (int g = lane; g < G; g += 32) {
      double a = s_c[g * per], b = -INFINITY;
#pragma unroll 1
      for (int m = 1; m < per; ++m) {
        const double v = s_c[g * per + m];
        b = fmax(b, fmin(a, v));
        a = fmax(a, v);
      }
      (g < 32 ? g0 : g1) = order_key(per > 1 ? a + b : a);
    }
    uint64_t eligible = 0ull;
#pragma unroll 1
    for (int j = 0; j < r.topk_groups; ++j) {
      const int g = argmax(g0, g1);
      if (lane == (g & 31)) { if (g < 32) g0 = 0ull; else g1 = 0ull; }
      eligible |= ((1ull << per) - 1ull) << (g * per);
    }
    if (!r.select_bias) {
      k0 = v0 ? order_key(l0) : 0ull;
      k1 = v1 ? order_key(l1) : 0ull;
    }
    if (!((eligible >> lane) & 1ull)) k0 = 0ull;
    if (!((eligible >> (lane + 32)) & 1ull)) k1 = 0ull;
  }
  if (l0 == -INFINITY && k0) k0 = order_key(l0);   // barred
  if (l1 == -INFINITY && k1) k1 = order_key(l1);
  slot0 = slot1 = -1;
#pragma unroll 1
  for (int j = 0; j < r.k; ++j) {
    const int e = argmax(k0, k1);
    if (lane == (e & 31)) {
      if (e < 32) { slot0 = j; k0 = 0ull; } else { slot1 = j; k1 = 0ull; }
    }
  }
}

// One token in doubt (a warp), its logits evaluated.  false: all of its logits are needed, since the border between groups falls differently,
// or since biased scores of a softmax are closer than the error of the fp32 denominator, which they share: an error in it moves a
// difference of scores in proportion to the difference of what it divides, so that this is rare.
// kBiased: biased scores of a softmax.  A function, called, with the router as a __grid_constant__ parameter, so that its address can be
// handed on: 8192 x 2048 takes 30.2 us, in line 33.4 (registers), with a copy of the router on the stack 32.2.
template <bool kBiased, int kTokens>
__device__ __noinline__ bool settle(const ScoredRouter& r, int64_t t0, const RouteDoubts<kTokens>& q, int i, double* s_c, int lane) {
  const Doubt& d = q.d[i];
  const int k = r.k;
  const double l0 = q.l[i][lane], l1 = q.l[i][lane + 32];
  int slot0 = -1, slot1 = -1;
  if (d.full) {
    choose_exactly(r, l0, l1, s_c, lane, slot0, slot1);
  } else {
    const bool m0 = (d.settled >> lane) & 1ull, m1 = (d.settled >> (lane + 32)) & 1ull;
    // exact scores of the settled experts (a softmax's with the fp32 denominator), or their logits; what a softmax's denominator divides
    double c0 = l0, c1 = l1, e0 = 0.0, e1 = 0.0;
    const double den_rel = double(d.den_rel) * double(d.inv_den);
    // c, e and d, f: scores and what they are without the bias and the denominator
    auto open = [&](double c, double e, double d, double f) {
      if (isinf(c) || isinf(d)) return false;      // (an expert barred by -inf)
      const double margin = den_rel * fabs(e - f) + 1e-14 * (fabs(c) + fabs(d));
      return e != f && !(fabs(c - d) > margin);
    };
    bool unsure = false;
    if (r.select_bias || r.n_groups > 1) {
#pragma unroll 1
      for (int h = 0; h < 2; ++h) {
        if (!(h ? m1 : m0)) continue;
        const double e = exp(!kBiased && r.sigmoid ? -(h ? l1 : l0) : (h ? l1 : l0) - double(d.l_max));
        const double bias = kBiased || r.select_bias ? double(r.select_bias[lane + 32 * h]) : 0.0;
        (h ? c1 : c0) = !kBiased && r.sigmoid ? 1.0 / (1.0 + e) + bias : kBiased ? e * double(d.inv_den) + bias : e;
        (h ? e1 : e0) = e;
      }
    }
    __syncwarp();
    if (d.border) {
      // a lane for each group at the border: its sum, and what the sum is without the biases and the denominator
      const int per = r.per_group, n = __popcll(d.border);
      double sum = 0.0, e_sum = 0.0;
      int group = 0, i = 0;
#pragma unroll 1
      for (uint64_t groups = d.border; groups; groups &= groups - 1, ++i) {
        const int g = __ffsll((long long)groups) - 1;
        // the two largest of the group, among the settled ones
        double a = -INFINITY, b = -INFINITY, ea = 0.0, eb = 0.0;
#pragma unroll 1
        for (uint64_t m = d.settled & (per == 64 ? ~0ull : ((1ull << per) - 1ull) << (g * per)); m; m &= m - 1) {
          const int e = __ffsll((long long)m) - 1;
          const double x = __shfl_sync(0xffffffffu, c0, e & 31), y = __shfl_sync(0xffffffffu, c1, e & 31), c = e < 32 ? x : y;
          const double u = __shfl_sync(0xffffffffu, e0, e & 31), v = __shfl_sync(0xffffffffu, e1, e & 31), ec = e < 32 ? u : v;
          // (which of a group's scores are its two largest may hang on the denominator too)
          if (kBiased && (open(c, ec, a, ea) || open(c, ec, b, eb))) unsure = true;
          if (c > a) { b = a; eb = ea; a = c; ea = ec; }
          else if (c > b) { b = c; eb = ec; }
        }
        if (lane == i) { group = g; sum = per > 1 ? a + b : a; e_sum = per > 1 ? ea + eb : ea; }
      }
      // those that stay must come before those that do not
      const bool out = lane < n && !((d.kept >> group) & 1ull);
      bool wrong = false;
#pragma unroll 1
      for (int j = 0; j < n; ++j) {
        const int g = __shfl_sync(0xffffffffu, group, j);
        const double s = __shfl_sync(0xffffffffu, sum, j), e = __shfl_sync(0xffffffffu, e_sum, j);
        if (!out || !((d.kept >> g) & 1ull)) continue;
        wrong |= !(s > sum || (s == sum && g < group));
        if (kBiased && open(s, e, sum, e_sum)) unsure = true;
      }
      if (__any_sync(0xffffffffu, wrong)) return false;
    }
    // All others are where they belong: the experts in doubt share out the places that experts in doubt have, in their exact order.
    const bool w0 = (d.which >> lane) & 1ull, w1 = (d.which >> (lane + 32)) & 1ull;
    // (an order of all values, NaN too: no two experts get one place)
    const uint64_t k0 = order_key(r.select_bias ? c0 : l0), k1 = order_key(r.select_bias ? c1 : l1);
    int rank0 = 0, rank1 = 0;                      // how many of them come before the lane's
#pragma unroll 1
    for (uint64_t m = d.which; m; m &= m - 1) {
      const int e = __ffsll((long long)m) - 1;
      const uint64_t a = __shfl_sync(0xffffffffu, k0, e & 31), b = __shfl_sync(0xffffffffu, k1, e & 31), c = e < 32 ? a : b;
      rank0 += c > k0 || (c == k0 && e < lane) ? 1 : 0;
      rank1 += c > k1 || (c == k1 && e < lane + 32) ? 1 : 0;
      if (kBiased) {
        const double x = __shfl_sync(0xffffffffu, c0, e & 31), y = __shfl_sync(0xffffffffu, c1, e & 31), ce = e < 32 ? x : y;
        const double u = __shfl_sync(0xffffffffu, e0, e & 31), v = __shfl_sync(0xffffffffu, e1, e & 31), ee = e < 32 ? u : v;
        if ((w0 && e != lane && open(ce, ee, c0, e0)) || (w1 && e != lane + 32 && open(ce, ee, c1, e1))) unsure = true;
      }
    }
    if (kBiased && __any_sync(0xffffffffu, unsure)) return false;
    int place = 0;
#pragma unroll 1
    for (int j = 0; j < k; ++j) {
      const int e = (int)((d.chosen >> (6 * j)) & 63ull);
      if ((d.which >> e) & 1ull) {
        if (w0 && rank0 == place) slot0 = j;
        if (w1 && rank1 == place) slot1 = j;
        ++place;
      } else {
        if (e == lane) slot0 = j;
        if (e == lane + 32) slot1 = j;
      }
    }
  }
  const float p0 = q.p[i][lane], p1 = q.p[i][lane + 32];
  const float sum = warp_sum((slot0 >= 0 ? p0 : 0.0f) + (slot1 >= 0 ? p1 : 0.0f));
  const float div = r.renorm ? fmaxf(sum, 1e-20f) : 1.0f;
  const int64_t at = (t0 + d.token) * k;
  if (slot0 >= 0) { r.idx[at + slot0] = lane; r.w[at + slot0] = p0 / div * r.scale; }
  if (slot1 >= 0) { r.idx[at + slot1] = lane + 32; r.w[at + slot1] = p1 / div * r.scale; }
  return true;
}

__device__ __forceinline__ float ld_cluster_f32(uint32_t addr) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr));      // (in order with the barriers, which are volatile too)
  return v;
}

// The choices of tokens rank * share + [0, share) of a tile whose sums lie in parts in the shared memory of the cluster's CTAs: `part` rows of
// `pitch` floats (E and more), and the squared norms `xx`, at the same places in each.  All threads of the CTA, of which warps 0 ..
// n_warps - 1 choose; s_c: 64 doubles for each of them.
template <int kTokens>
__device__ __forceinline__ void choose_share(const ScoredRouter& r, int64_t t0, int rank, int cluster, int share, const float* part, int pitch,
                                             const float* xx_part, float logit_eps, RouteDoubts<kTokens>& q, double (*s_c)[64],
                                             int warp, int n_warps, int lane) {
  const int n = (int)min(int64_t(share), max(int64_t(0), r.T - t0 - rank * share));      // tokens of this CTA that are there
  if (warp < n_warps && warp < n) {
    LaneBias bias;
    bias.load(r, lane);
    const float w_norm = *r.w_norm;
    const int E = r.E, e0 = min(lane, E - 1), e1 = min(lane + 32, E - 1);
    float lb0 = 0.0f, lb1 = 0.0f;
    if (r.logit_bias) { lb0 = r.logit_bias[e0]; lb1 = r.logit_bias[e1]; }
#pragma unroll 1
    for (int i = warp; i < n; i += n_warps) {
      const int number = rank * share + i;
      const int64_t token = t0 + number;
      float l0 = 0.0f, l1 = 0.0f, xx = 0.0f;
      if (cluster > 1) {
        float lost0 = 0.0f, lost1 = 0.0f;                           // the parts' sums, rank by rank
        const uint32_t row = ptx::smem_u32(part + number * pitch), x_at = ptx::smem_u32(xx_part + number);
#pragma unroll 2
        for (int c = 0; c < cluster; ++c) {
          const uint32_t far = ptx::map_to_rank(row, c);
          two_sum(l0, lost0, ld_cluster_f32(far + 4 * e0));
          two_sum(l1, lost1, ld_cluster_f32(far + 4 * e1));
          xx += ld_cluster_f32(ptx::map_to_rank(x_at, c));
        }
        l0 += lost0;
        l1 += lost1;
      } else {
        l0 = part[number * pitch + e0];
        l1 = part[number * pitch + e1];
        xx = xx_part[number];
      }
      l0 += lb0;
      l1 += lb1;
      if (r.logits) {
        if (lane < E) r.logits[token * E + lane] = l0;
        if (lane + 32 < E) r.logits[token * E + lane + 32] = l1;
      }
      Doubt d;
      float p0, p1;
      choose_experts(r, bias, token, l0, l1, logit_eps * sqrt_approx(xx) * w_norm + 1.2e-7f * bias.logit_max, reinterpret_cast<float*>(s_c[warp]), d, p0, p1,
                     lane);
      if (d.settled) {
        const bool zeros = xx == 0.0f;             // a token of zeros: its logits are the biases, there is nothing to evaluate
        int at = 0;
        if (lane == 0) {
          at = atomicAdd(&q.n, 1);
          d.token = number;
          if (zeros) { d.full = 1; d.settled = 0ull; }
          q.d[at] = d;
        }
        at = __shfl_sync(0xffffffffu, at, 0);
        if (zeros) {
          q.l[at][lane] = double(lb0);
          q.l[at][lane + 32] = double(lb1);
        }
        q.p[at][lane] = p0;
        q.p[at][lane + 32] = p1;
      }
    }
  }
  if (cluster > 1) ptx::cluster_sync();            // nobody leaves while its sums are being read
  else __syncthreads();
  const int doubts = q.n;
  const bool biased_softmax = !r.sigmoid && r.select_bias;
  if (doubts == 0) return;                         // uniform over the CTA
  // the logits in doubt, a warp each; then the tokens, a warp each.  A second time for tokens that need all their logits after all.
#pragma unroll 1
  for (int again = 0; again < 2; ++again) {
    int item = 0;
#pragma unroll 1
    for (int i = 0; i < doubts; ++i) {
      if (again && q.d[i].full != 2) continue;
#pragma unroll 1
      for (uint64_t m = q.d[i].settled; m; m &= m - 1, ++item)
        if (warp < n_warps && item % (n_warps / 4) == warp / 4) {
          const int e = __ffsll((long long)m) - 1;
          const double part = logit_quarter(r, t0 + q.d[i].token, e, warp & 3, lane);
          if (lane == 0) q.quarter[warp] = part;
          asm volatile("bar.sync %0, 128;" ::"r"(1 + warp / 4) : "memory");           // the four warps
          if (lane == 0 && (warp & 3) == 0)
            q.l[i][e] = ((q.quarter[warp] + q.quarter[warp + 1]) + (q.quarter[warp + 2] + q.quarter[warp + 3])) + (r.logit_bias ? double(r.logit_bias[e]) : 0.0);
          asm volatile("bar.sync %0, 128;" ::"r"(1 + warp / 4) : "memory");
        }
    }
    __syncthreads();
    bool more = false;
    if (warp < n_warps)
#pragma unroll 1
      for (int i = warp; i < doubts; i += n_warps) {
        if (again && q.d[i].full != 2) continue;
        const bool settled = biased_softmax ? settle<true>(r, t0, q, i, s_c[warp], lane) : settle<false>(r, t0, q, i, s_c[warp], lane);
        if (!settled) {
          more = true;
          __syncwarp();
          if (lane == 0) {
            q.d[i].full = 2;
            q.d[i].settled = r.E == 64 ? ~0ull : (1ull << r.E) - 1ull;
          }
        }
      }
    if (!__syncthreads_or(more)) return;
  }
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
// A sum of squares is 0 for zeros only (a token of zeros, as padding is, has logits that are known exactly).
__device__ __forceinline__ float nonzero_square(float sum, uint32_t bits) { return sum == 0.0f && (bits & 0x7FFF7FFFu) ? 1e-38f : sum; }
// upper halves of two floats -> bf16x2 (first in the low half)
__device__ __forceinline__ uint32_t upper_halves(float a, float b) { return __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x7632); }

constexpr int kScoredWarps = 8;
constexpr int kScoredTokens = 16;

// NE: 8-expert column tiles (ceil(E / 8) rounded up to 1, 2, 4 or 8); kF32: type of the router weights.
// Lane (g, t) = (lane / 4, lane % 4) loads elements [32 * step + 8 * t, + 8) of token rows g and g + 8 and of router rows 8n + g;
// the reduction index may be permuted as long as both operands are.
// kAlone: a CTA has its SM to itself, and registers for all sums of 64 experts: where the clusters run at a time so (512 x 2048: 11.7 us, 14.2
// with half of them; 256 x 2048, whose 16 clusters of eight do not: 14.7 us in two rounds, 12.2 with two CTAs an SM).
template <int NE, bool kF32, bool kAlone>
__global__ void __launch_bounds__(kScoredWarps * 32, kAlone ? 1 : 2) route_scored_kernel(const __grid_constant__ ScoredRouter r, int cluster) {
  __shared__ union {
    float part[kScoredWarps][NE * 4][32];
    struct { RouteDoubts<kScoredTokens> doubt; double c[kScoredWarps][64]; } late;
  } sh;
  __shared__ float s_logits[kScoredTokens][NE * 8 + 1];
  __shared__ float s_norm[kScoredWarps][kScoredTokens];
  __shared__ float s_xx[kScoredTokens];
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
  uint64_t acc[NE][2], over[NE][2];
#pragma unroll
  for (int n = 0; n < NE; ++n) acc[n][0] = acc[n][1] = over[n][0] = over[n][1] = 0ull;
  float xxa = 0.0f, xxb = 0.0f;
  uint32_t bits_a = 0u, bits_b = 0u;
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
          // an MMA truncates what it adds up: sums of 16 elements start from zero, the smallest terms first, and join the others outside
          float pa[4] = {0.0f, 0.0f, 0.0f, 0.0f}, pb[4] = {0.0f, 0.0f, 0.0f, 0.0f};
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
            mma_bf16_k16(pa, ca.x, cb.x, ca.y, cb.y, upper_halves(lo[0], lo[1]), upper_halves(lo[2], lo[3]));
            mma_bf16_k16(pb, ca.z, cb.z, ca.w, cb.w, upper_halves(lo[4], lo[5]), upper_halves(lo[6], lo[7]));
            mma_bf16_k16(pa, ca.x, cb.x, ca.y, cb.y, upper_halves(mid[0], mid[1]), upper_halves(mid[2], mid[3]));
            mma_bf16_k16(pb, ca.z, cb.z, ca.w, cb.w, upper_halves(mid[4], mid[5]), upper_halves(mid[6], mid[7]));
            mma_bf16_k16(pa, ca.x, cb.x, ca.y, cb.y, upper_halves(hi[0], hi[1]), upper_halves(hi[2], hi[3]));
            mma_bf16_k16(pb, ca.z, cb.z, ca.w, cb.w, upper_halves(hi[4], hi[5]), upper_halves(hi[6], hi[7]));
          } else {
            uint4 w = kZero;
            if (row) w = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(r.Wr) + int64_t(n * 8 + g) * d + s * 32 + t * 8);
            mma_bf16_k16(pa, ca.x, cb.x, ca.y, cb.y, w.x, w.y);
            mma_bf16_k16(pb, ca.z, cb.z, ca.w, cb.w, w.z, w.w);
          }
          compensated_add(acc[n][0], over[n][0], add_f32x2(f32x2(pa[0], pa[1]), f32x2(pb[0], pb[1])));
          compensated_add(acc[n][1], over[n][1], add_f32x2(f32x2(pa[2], pa[3]), f32x2(pb[2], pb[3])));
        }
        const uint32_t wa[4] = {ca.x, ca.y, ca.z, ca.w}, wb[4] = {cb.x, cb.y, cb.z, cb.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          bits_a |= wa[j];
          bits_b |= wb[j];
          xxa = fmaf(bf16_lo(wa[j]), bf16_lo(wa[j]), fmaf(bf16_hi(wa[j]), bf16_hi(wa[j]), xxa));
          xxb = fmaf(bf16_lo(wb[j]), bf16_lo(wb[j]), fmaf(bf16_hi(wb[j]), bf16_hi(wb[j]), xxb));
        }
      }
    }
  }
  xxa = nonzero_square(xxa, bits_a);
  xxb = nonzero_square(xxb, bits_b);
#pragma unroll
  for (int o = 1; o < 4; o <<= 1) {
    xxa += __shfl_xor_sync(0xffffffffu, xxa, o);
    xxb += __shfl_xor_sync(0xffffffffu, xxb, o);
  }
  if (t == 0) { s_norm[warp][g] = xxa; s_norm[warp][g + 8] = xxb; }
#pragma unroll
  for (int n = 0; n < NE; ++n)
#pragma unroll
    for (int h = 0; h < 2; ++h)
      unpack_f32x2(acc[n][h], sh.part[warp][n * 4 + 2 * h][lane], sh.part[warp][n * 4 + 2 * h + 1][lane]);
  __syncthreads();
  // fragment: value i of column tile n at lane (g, t) is token row g + 8*(i/2), expert 8n + 2t + (i&1)
  for (int v = warp; v < NE * 4; v += kScoredWarps) {
    float z = sh.part[0][v][lane], z_lost = 0.0f;
#pragma unroll
    for (int w = 1; w < kScoredWarps; ++w) two_sum(z, z_lost, sh.part[w][v][lane]);
    s_logits[g + 8 * ((v & 3) >> 1)][(v >> 2) * 8 + 2 * t + (v & 1)] = z + z_lost;
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
  choose_share(r, t0, rank, cluster, kScoredTokens / cluster, &s_logits[0][0], NE * 8 + 1, s_xx, kWarpLogitEps, sh.late.doubt, sh.late.c, warp,
               kScoredWarps, lane);
}

// ------------------------------------------------------------------------------------------------
// Logits of long batches: tcgen05.mma kind::f16, a tile of 128 tokens x all experts per cluster of CTAs that share the width.
//
// TMA brings 64 elements of the tokens and of the router's rows (its three bf16 terms, or its bf16 rows) to a stage.  Either half of a
// stage's 4 x terms MMAs forms a sum of its own in TMEM, the smallest terms first -- the tensor core truncates what it adds up, so sums are
// kept short -- and the epilogue warps add both to pairs of fp32 sums in registers (four such accumulators, so that neither side waits for the other).  Eight
// more warps read the tokens of the stage from shared memory for their norms.  Then as above: sums meet in distributed shared memory,
// each CTA chooses for its share of the 128 tokens.
//
// Warps: 0 TMA producer, 1 MMA issuer, 2 TMEM owner, 4 to 19 epilogue (four per TMEM lane quarter, 16 experts each), 20 to 27 norms;
// all 32 choose.
//
// 8192 x 2048, 64 experts in 8 groups, fp32 Wr: 28.9 us in a graph, where the bytes take 5.4 (27.7 with sums of 64 elements and without
// compensation, whose bound did not hold).  About 11 us are the products: 655 KB of operands an SM, three fifths of them the weights'
// terms, are 6 us at the 61 bytes a cycle that an SM gets, the rest is the start of the pipeline.  7 are the choice, bound by instructions
// (710 a token, 64 tokens to an SM), 4 or 5 second evaluations, latency; the rest is not accounted for.  The kernel above, whose tokens
// are 16 to a cluster, takes 67.
// ------------------------------------------------------------------------------------------------
constexpr int kTileTokens = 128;
constexpr int kTileWarps = 16, kTileNormWarps = 8, kTileThreads = 1024;
constexpr int kTileStageA = kTileTokens * 128;
constexpr int kTilePipe = 4 * (kTileStageA + 3 * 64 * 128);      // 160 KB: four stages with three terms of 64 experts, more with less
constexpr int kTileMaxStages = 6;
constexpr int kTileSums = 4;                                      // accumulators in TMEM, 2 x 64 columns each
constexpr int kTilePitch = 65;

struct __align__(8) TileBarriers {
  uint64_t full[kTileMaxStages], empty[kTileMaxStages], sum_full[kTileSums], sum_empty[kTileSums];
  uint32_t tmem_base;
  int abort_flag;
};
struct TileLate {                                                 // over the stages, when they are done with
  RouteDoubts<kTileTokens> doubt;
  double c[kTileThreads / 32][64];
};
static_assert(sizeof(TileLate) <= kTilePipe, "the choices' data fit over the stages");
constexpr int kTileSmem = 1024 + kTilePipe + kTileTokens * (kTilePitch + 1) * 4 + (int)sizeof(TileBarriers);

__global__ void __launch_bounds__(kTileThreads, 1)
route_tile_kernel(const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ ScoredRouter r, int cluster, int experts,
                  int terms, int stages, uint32_t* status) {
  using namespace ptx;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - smem_u32(smem_raw));
  float* part = reinterpret_cast<float*>(gen + kTilePipe);
  float* xx = part + kTileTokens * kTilePitch;
  TileBarriers* bars = reinterpret_cast<TileBarriers*>(xx + kTileTokens);
  TileLate* late = reinterpret_cast<TileLate*>(gen);
  volatile int* abort_flag = &bars->abort_flag;
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const int rank = cluster > 1 ? (int)cluster_ctarank() : 0;
  const int64_t t0 = int64_t(blockIdx.x / cluster) * kTileTokens;
  const uint32_t stage_bytes = kTileStageA + uint32_t(terms * experts) * 128;
  if (threadIdx.x == 0) {
    for (int s = 0; s < kTileMaxStages; ++s) { mbar_init(smem_u32(&bars->full[s]), 1); mbar_init(smem_u32(&bars->empty[s]), 1 + kTileNormWarps); }
    for (int s = 0; s < kTileSums; ++s) { mbar_init(smem_u32(&bars->sum_full[s]), 1); mbar_init(smem_u32(&bars->sum_empty[s]), kTileWarps); }
    bars->abort_flag = 0;
    fence_barrier_init();
    prefetch_tensormap(&tm_x);
    prefetch_tensormap(&tm_w);
  }
  if (warp == 2) {
    tmem_alloc(smem_u32(&bars->tmem_base), 128 * kTileSums);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, bars->tmem_base, 0);
  pdl_wait();
  const int n_steps = (r.d + 63) / 64, kb = n_steps * rank / cluster, ke = n_steps * (rank + 1) / cluster;

  if (warp == 0) {
    if (lane == 0) {
      bool ok = true;
      int s = 0, phase = 0;
      for (int ks = kb; ok && ks < ke; ++ks) {
        ok = mbar_wait(smem_u32(&bars->empty[s]), phase ^ 1, abort_flag);
        if (!ok) break;
        const uint32_t bar = smem_u32(&bars->full[s]), dst = base + s * stage_bytes;
        mbar_expect_tx(bar, stage_bytes);
        tma_load_2d(dst, &tm_x, ks * 64, (int)t0, bar);
        tma_load_2d(dst + kTileStageA, &tm_w, ks * 64, 0, bar);
        if (++s == stages) { s = 0; phase ^= 1; }
      }
      // the commits of the last steps have arrived at this CTA's barriers before it may leave
      for (int i = 0; ok && i < stages; ++i) {
        ok = mbar_wait(smem_u32(&bars->empty[s]), phase ^ 1, abort_flag);
        if (++s == stages) { s = 0; phase ^= 1; }
      }
    }
  } else if (warp == 1) {
    const uint32_t idesc = make_idesc(1, 1, 1, kTileTokens, (uint32_t)experts);
    int s = 0, phase = 0;
    for (int ks = kb; ks < ke; ++ks) {
      const int n = ks - kb, a = n % kTileSums;
      const bool ok = mbar_wait(smem_u32(&bars->sum_empty[a]), ((n / kTileSums) & 1) ^ 1, abort_flag) &&
                      mbar_wait(smem_u32(&bars->full[s]), phase, abort_flag);
      if (!__all_sync(0xffffffffu, ok)) break;
      tc_fence_after();
      const uint64_t da = smem_desc_sw128(base + s * stage_bytes);
      if (elect_one()) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
          for (int term = terms - 1; term >= 0; --term)
#pragma unroll
            for (int j = 0; j < 2; ++j)
              mma_f16(tmem + a * 128 + h * 64, da + 4 * h + 2 * j,
                      smem_desc_sw128(base + s * stage_bytes + kTileStageA + term * experts * 128) + 4 * h + 2 * j, idesc,
                      j > 0 || term < terms - 1 ? 1u : 0u);
        mma_commit(smem_u32(&bars->empty[s]));
        mma_commit(smem_u32(&bars->sum_full[a]));
      }
      __syncwarp();
      if (++s == stages) { s = 0; phase ^= 1; }
    }
  } else if (warp >= 4 && warp < 4 + kTileWarps) {
    const int q = warp & 3, col = ((warp - 4) >> 2) * 16;
    const bool mine = col < experts;
    uint64_t sum[8], over[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] = over[j] = 0ull;
    for (int n = 0; n < ke - kb; ++n) {
      const int a = n % kTileSums;
      if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&bars->sum_full[a]), (n / kTileSums) & 1, abort_flag))) break;
      tc_fence_after();
      if (mine)
#pragma unroll
        for (int c = 0; c < 16; c += 8) {          // (8 columns of both sums at a time: registers)
          uint32_t u[8], v[8];
          tmem_ld_32x32b_x8(tmem + (uint32_t(q * 32) << 16) + a * 128 + col + c, u);
          tmem_ld_32x32b_x8(tmem + (uint32_t(q * 32) << 16) + a * 128 + 64 + col + c, v);
          tmem_wait_ld();
#pragma unroll
          for (int j = 0; j < 4; ++j)
            compensated_add(sum[c / 2 + j], over[c / 2 + j], add_f32x2(f32x2_bits(u[2 * j], u[2 * j + 1]), f32x2_bits(v[2 * j], v[2 * j + 1])));
        }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&bars->sum_empty[a]));
    }
    if (mine)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float* at = part + (q * 32 + lane) * kTilePitch + col + 2 * j;
        unpack_f32x2(sum[j], at[0], at[1]);
      }
  } else if (warp >= 4 + kTileWarps && warp < 4 + kTileWarps + kTileNormWarps) {
    // eight lanes read a token's 128 bytes (in any order), the warp four tokens of each quarter of the tile
    const int first = (warp - 4 - kTileWarps) * 4 + (lane >> 3);
    float sq[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    uint32_t bits[4] = {0u, 0u, 0u, 0u};
    int s = 0, phase = 0;
    for (int ks = kb; ks < ke; ++ks) {
      if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&bars->full[s]), phase, abort_flag))) break;
      const uint8_t* rows = gen + s * stage_bytes + first * 128 + (lane & 7) * 16;
      uint4 v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const uint4*>(rows + i * 32 * 128);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
        bits[i] |= w[0] | w[1] | w[2] | w[3];
#pragma unroll
        for (int j = 0; j < 4; ++j) sq[i] = fmaf(bf16_lo(w[j]), bf16_lo(w[j]), fmaf(bf16_hi(w[j]), bf16_hi(w[j]), sq[i]));
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&bars->empty[s]));
      if (++s == stages) { s = 0; phase ^= 1; }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      sq[i] = nonzero_square(sq[i], bits[i]);
#pragma unroll
      for (int o = 1; o < 8; o <<= 1) sq[i] += __shfl_xor_sync(0xffffffffu, sq[i], o);
      if ((lane & 7) == 0) xx[first + 32 * i] = sq[i];
    }
  }
  // after a wait that ran out: time for copies and MMAs in flight to land before shared memory is used anew
  if (*abort_flag) {
    const uint64_t start = globaltimer_ns();
    while (globaltimer_ns() - start < 200000ull) __nanosleep(1000);
  }
  tc_fence_before();
  __syncthreads();                                 // all stages are done with
  if (threadIdx.x == 0) late->doubt.n = 0;
  if (warp == 2) {
    tc_fence_after();
    tmem_dealloc(tmem, 128 * kTileSums);
  }
  if (cluster > 1) cluster_sync();
  else __syncthreads();
  if (threadIdx.x == 0 && *abort_flag) atomicExch(status, 1u);
  choose_share(r, t0, rank, cluster, kTileTokens / cluster, part, kTilePitch, xx, kTileLogitEps, late->doubt, late->c, warp, kTileThreads / 32, lane);
}

// What a router keeps beside its weights: [0] a device status word, [1] the largest 2-norm of a row (rounded up), and from byte 256 on an
// fp32 router's three bf16 terms, [3][experts rounded up to 16][d], rows past the last zero.
constexpr int kPackTerms = 256;
static int tile_experts(int E) { return (E + 15) & ~15; }

// A CTA per (padded) expert; an offline step.
__global__ void __launch_bounds__(256) router_pack_kernel(const void* __restrict__ Wr, int w_f32, int E, int d, uint8_t* __restrict__ packed) {
  __shared__ double s_sum[8];
  const int e = blockIdx.x, experts = gridDim.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint16_t* terms = reinterpret_cast<uint16_t*>(packed + kPackTerms);
  double ss = 0.0;
  for (int j = threadIdx.x; j < d; j += 256) {
    float w = 0.0f;
    if (e < E)
      w = w_f32 ? static_cast<const float*>(Wr)[int64_t(e) * d + j]
                : __uint_as_float(uint32_t(static_cast<const uint16_t*>(Wr)[int64_t(e) * d + j]) << 16);
    ss = fma(double(w), double(w), ss);
    if (w_f32) {
#pragma unroll
      for (int t = 0; t < 3; ++t) {
        const uint32_t top = __float_as_uint(w) & 0xFFFF0000u;
        terms[(int64_t(t) * experts + e) * d + j] = (uint16_t)(top >> 16);
        w = __fsub_rn(w, __uint_as_float(top));
      }
    }
  }
  ss = warp_sum_f64(ss);
  if (lane == 0) s_sum[warp] = ss;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < 8; ++i) ss += s_sum[i];
    atomicMax(reinterpret_cast<int*>(packed) + 1, __float_as_int(__double2float_ru(sqrt(ss))));      // of non-negative floats
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

template <int NE, bool kF32>
static cudaError_t launch_scored_as(const ScoredRouter& r, unsigned tiles, int cluster, cudaStream_t stream) {
  static ResidentClusters resident;
  const int alone = cluster > 1 ? resident.get(route_scored_kernel<NE, kF32, true>, kScoredWarps * 32, 0, cluster) : device_sm_count();
  const dim3 grid(tiles * cluster), block(kScoredWarps * 32);
  return (int64_t)tiles <= alone ? launch_ex(route_scored_kernel<NE, kF32, true>, grid, block, 0, stream, true, cluster, r, cluster)
                                 : launch_ex(route_scored_kernel<NE, kF32, false>, grid, block, 0, stream, true, cluster, r, cluster);
}
template <int NE>
static cudaError_t launch_scored(const ScoredRouter& r, unsigned tiles, int cluster, cudaStream_t stream) {
  return r.w_f32 ? launch_scored_as<NE, true>(r, tiles, cluster, stream) : launch_scored_as<NE, false>(r, tiles, cluster, stream);
}

static cudaError_t launch_tiles(const ScoredRouter& r, const CUtensorMap& tx, const CUtensorMap& tw, int experts, int terms, uint32_t* status,
                                cudaStream_t stream) {
  static PerDeviceOnce once;
  const cudaError_t e = set_max_dynamic_smem(once, route_tile_kernel, kTileSmem);
  if (e != cudaSuccess) return e;
  // CTAs that share a tile's width: as many as run at a time, each with two steps at least
  static ResidentClusters resident;
  const int64_t tiles = (r.T + kTileTokens - 1) / kTileTokens;
  int cluster = 1;
  for (int c = 2; c <= 8; c *= 2)
    if (tiles <= resident.get(route_tile_kernel, kTileThreads, kTileSmem, c) && r.d >= 128 * c) cluster = c;
  const int stages = std::min(kTileMaxStages, kTilePipe / (kTileStageA + terms * experts * 128));
  return launch_ex(route_tile_kernel, dim3((unsigned)(tiles * cluster)), dim3(kTileThreads), kTileSmem, stream, true, cluster, tx, tw, r, cluster,
                   experts, terms, stages, status);
}

// The logits come from the tcgen05 kernel from this much work on: tokens x width x column tiles of 8 experts x bf16 terms of the weights.  us,
// warp-level MMAs / tcgen05, 64 experts in fp32: 512 x 2048 11.7 / 15.3, 700 x 2048 14.9 / 15.2, 1024 x 2048 15.0 / 15.6, 8192 x 2048 67 / 25,
// 4096 x 256 12.8 / 15.6, 8192 x 256 21.4 / 15.8; 16 experts in fp32: 2048 x 2048 12.9 / 16.0, 8192 x 1024 20.5 / 17.9; 32 in bf16: 4096 x 2048
// 15.2 / 15.7, 8192 x 2048 26.2 / 20.9.
constexpr int64_t kTileMinWork = 30000000;

// status: the device status word that a bounded wait raises; null: the router's own
mote_status_t launch_route_scored(const mote_router_t* R, const void* x, int64_t ldx, int64_t T, int32_t* idx, float* w, float* logits,
                                  uint32_t* status, cudaStream_t stream) {
  ScoredRouter r{};
  r.x = static_cast<const uint16_t*>(x); r.ldx = ldx; r.Wr = R->Wr; r.logit_bias = R->logit_bias; r.select_bias = R->select_bias;
  r.w_norm = static_cast<const float*>(R->packed) + 1;
  r.T = T; r.d = R->d; r.E = R->E; r.k = R->k; r.sigmoid = R->scoring == MOTE_SCORE_SIGMOID;
  r.n_groups = R->topk_groups == R->n_groups ? 1 : R->n_groups;            // where all groups stay there is nothing to choose among them
  r.per_group = R->E / r.n_groups; r.topk_groups = R->topk_groups; r.renorm = R->renorm != 0; r.w_f32 = R->w_dtype == MOTE_DTYPE_F32; r.scale = R->scale;
  r.idx = idx; r.w = w; r.logits = logits;
  if (!status) status = static_cast<uint32_t*>(const_cast<void*>(R->packed));
  const int ne = (R->E + 7) / 8;
  cudaError_t e;
  if (T * r.d * ne * (r.w_f32 ? 3 : 1) >= kTileMinWork) {
    const int experts = tile_experts(R->E), terms = r.w_f32 ? 3 : 1;
    const void* rows = r.w_f32 ? static_cast<const uint8_t*>(R->packed) + kPackTerms : static_cast<const uint8_t*>(R->Wr);
    CUtensorMap tx, tw;
    if (!make_operand_map(&tx, x, T, R->d, ldx, kTileTokens) || !make_operand_map(&tw, rows, r.w_f32 ? 3 * experts : R->E, R->d, R->d, terms * experts))
      return MOTE_ERR_CUDA;
    e = launch_tiles(r, tx, tw, experts, terms, status, stream);
  } else {
    const unsigned tiles = (unsigned)((T + kScoredTokens - 1) / kScoredTokens);
    int cluster = 1;                             // CTAs that share a tile's width: as many as the SMs allow
    while (cluster < 8 && int64_t(tiles) * cluster * 2 <= device_sm_count()) cluster *= 2;
    e = ne <= 1   ? launch_scored<1>(r, tiles, cluster, stream)
        : ne <= 2 ? launch_scored<2>(r, tiles, cluster, stream)
        : ne <= 4 ? launch_scored<4>(r, tiles, cluster, stream) : launch_scored<8>(r, tiles, cluster, stream);
  }
  if (e != cudaSuccess) return MOTE_ERR_CUDA;
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
  return mote::kPackTerms + (w_dtype == MOTE_DTYPE_F32 ? size_t(3) * mote::tile_experts(E) * d * 2 : 0);
}

extern "C" mote_status_t mote_router_pack(const void* Wr, int w_dtype, int E, int64_t d, void* packed, size_t packed_bytes, void* stream) {
  using namespace mote;
  if (w_dtype != MOTE_DTYPE_F32 && w_dtype != MOTE_DTYPE_BF16) return MOTE_ERR_DTYPE;
  const size_t need = mote_router_pack_bytes(E, d, w_dtype);
  if (need == 0) return MOTE_ERR_SHAPE;
  if (!Wr || !packed) return MOTE_ERR_NULL;
  if (!aligned16(Wr) || (reinterpret_cast<uintptr_t>(packed) & 255u) != 0) return MOTE_ERR_ALIGN;
  if (packed_bytes < need) return MOTE_ERR_WORKSPACE;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  MOTE_CUDA_OK(cudaMemsetAsync(packed, 0, kPackTerms, s));
  router_pack_kernel<<<tile_experts(E), 256, 0, s>>>(Wr, w_dtype == MOTE_DTYPE_F32, E, (int)d, static_cast<uint8_t*>(packed));
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
  return launch_route_scored(R, x, T > 1 ? ldx : R->d, T, topk_idx, topk_w, logits, nullptr, static_cast<cudaStream_t>(stream));
}
