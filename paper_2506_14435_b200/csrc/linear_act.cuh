// What the kernels of mote_linear share: arguments and activations.
#pragma once

#include "mote_common.cuh"
#include "mote_internal.h"

namespace mote {

struct LinearArgs {
  const uint16_t* x; int64_t ldx, T;
  const void* W; const float* w_scale; const float* bias;
  const uint16_t* res; int64_t ldr;
  void* out;
  int64_t N;
  int K, act, out_f32;
  uint32_t* status;                              // device status word, cleared by every call
};

// 2^x and 1/x of the special-function unit: relative errors of 2^-22 and 2^-23.
__device__ __forceinline__ float ex2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp_fast(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// The larger of z and 0; NaN stays NaN.
__device__ __forceinline__ float relu_nan(float z) {
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(z), "f"(0.0f));
  return y;
}
constexpr float kGeluFlat = 16.0f;               // from here on gelu(z) = z in fp32, and for z = inf

// Activations by a few instructions each (with expf, a division and erff the SiLU epilogue of a 4096 x 11008 product took longer than its
// MMAs: 192 us instead of 128).  Relative errors of the results: 2^-21 or so and what the exponents' roundings add, 2^-23 for each unit of |z|
// (SiLU), of the tanh's argument or of z^2 (GELU).
__device__ __forceinline__ float act_silu(float z) { return z * rcp_fast(1.0f + ex2_fast(-1.4426950408889634f * z)); }
__device__ __forceinline__ float act_gelu_tanh(float z) {
  // 0.5 z (1 + tanh u) = z / (1 + exp(-2u)),  u = sqrt(2/pi) (z + 0.044715 z^3)
  const float m = z * fmaf(-0.10294323973f, z * z, -2.3022081985f);       // -2 u log2(e)
  return z * rcp_fast(1.0f + ex2_fast(m));
}
// gelu(z) = max(z, 0) - m e^(-m^2/2) h(m),  m = |z|,  h(m) = erfcx(m / sqrt 2) / 2 as a polynomial in t = 1 / (1 + p m) without constant term:
// p and the coefficients are a least-squares fit to the relative error, weights moved until it is even (Lawson), over m up to 13.2, where the
// second part leaves fp32: 2^-20.9.  So the tail of negative z is right relative to its own size (to 2^-19.9 up to 4, 2^-17 up to 13; by
// an absolute bound on erfc it was off by 5e-4 at -4 and 4e-3 at -6).  The second part is 0 long before kGeluFlat.
constexpr float kGeluP = 0.2636375427246094f;
constexpr float kGelu1 = 0.10501818358898163f, kGelu2 = 0.10782589763402939f, kGelu3 = 0.07952073961496353f, kGelu4 = 0.15098322927951813f,
                kGelu5 = -0.0799214094877243f, kGelu6 = 0.20638196170330048f, kGelu7 = -0.06980885565280914f;
__device__ __forceinline__ float act_gelu(float z) {
  const float mag = fabsf(fminf(z, kGeluFlat));
  const float t = rcp_fast(fmaf(kGeluP, mag, 1.0f));
  float q = fmaf(kGelu7, t, kGelu6);
  q = fmaf(q, t, kGelu5);
  q = fmaf(q, t, kGelu4);
  q = fmaf(q, t, kGelu3);
  q = fmaf(q, t, kGelu2);
  q = fmaf(q, t, kGelu1);
  const float e = ex2_fast(-0.72134752044448170f * mag * mag);           // exp(-z^2 / 2)
  return fmaf(-mag, q * t * e, relu_nan(z));
}
__device__ __forceinline__ float apply_act(float z, int act) {
  switch (act) {
    case MOTE_ACT_RELU: return relu_nan(z);
    case MOTE_ACT_SILU: return act_silu(z);
    case MOTE_ACT_GELU: return act_gelu(z);
    case MOTE_ACT_GELU_TANH: return act_gelu_tanh(z);
  }
  return z;
}
// The same on pairs (fp32x2 instructions), for the tensor-core epilogue, whose few warps have 128 x bn values to finish per tile.
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t both(float v) { return f32x2(v, v); }
__device__ __forceinline__ uint64_t ex2_pair(uint64_t v) {
  float a, b;
  unpack_f32x2(v, a, b);
  return f32x2(ex2_fast(a), ex2_fast(b));
}
__device__ __forceinline__ uint64_t rcp_pair(uint64_t v) {
  float a, b;
  unpack_f32x2(v, a, b);
  return f32x2(rcp_fast(a), rcp_fast(b));
}
__device__ __forceinline__ uint64_t max0_pair(uint64_t v) {
  float a, b;
  unpack_f32x2(v, a, b);
  return f32x2(relu_nan(a), relu_nan(b));
}
__device__ __forceinline__ uint64_t flat_magnitude_pair(uint64_t v) {            // |min(v, kGeluFlat)|
  float a, b;
  unpack_f32x2(v, a, b);
  return f32x2(fabsf(fminf(a, kGeluFlat)), fabsf(fminf(b, kGeluFlat)));
}
// z / (1 + 2^m)
__device__ __forceinline__ uint64_t gated_pair(uint64_t z, uint64_t m) {
  return mul_f32x2(z, rcp_pair(add_f32x2(both(1.0f), ex2_pair(m))));
}
// 16 values, one look at which activation it is
__device__ __forceinline__ void apply_act16(uint64_t (&z)[8], int act) {
  if (act == MOTE_ACT_NONE) return;
  if (act == MOTE_ACT_RELU) {
#pragma unroll
    for (int j = 0; j < 8; ++j) z[j] = max0_pair(z[j]);
  } else if (act == MOTE_ACT_SILU) {
#pragma unroll
    for (int j = 0; j < 8; ++j) z[j] = gated_pair(z[j], mul_f32x2(z[j], both(-1.4426950408889634f)));
  } else if (act == MOTE_ACT_GELU_TANH) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      z[j] = gated_pair(z[j], mul_f32x2(z[j], fma2(mul_f32x2(z[j], both(-0.10294323973f)), z[j], both(-2.3022081985f))));
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {                // act_gelu
      const uint64_t mag = flat_magnitude_pair(z[j]);
      const uint64_t t = rcp_pair(fma2(mag, both(kGeluP), both(1.0f)));
      uint64_t q = fma2(both(kGelu7), t, both(kGelu6));
      q = fma2(q, t, both(kGelu5));
      q = fma2(q, t, both(kGelu4));
      q = fma2(q, t, both(kGelu3));
      q = fma2(q, t, both(kGelu2));
      q = fma2(q, t, both(kGelu1));
      const uint64_t e = ex2_pair(mul_f32x2(mul_f32x2(mag, both(-0.72134752044448170f)), mag));
      z[j] = fma2(mul_f32x2(mag, both(-1.0f)), mul_f32x2(mul_f32x2(q, t), e), max0_pair(z[j]));
    }
  }
}

// The tensor-core product (linear_umma.cu); a.W holds bf16 values, a.w_scale is null where they need no scale.
mote_status_t launch_linear_umma(const LinearArgs& a, cudaStream_t stream);

}  // namespace mote
