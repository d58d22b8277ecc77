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
// MMAs: 192 us instead of 128).  Errors are below 2^-21 of |z|.
__device__ __forceinline__ float act_silu(float z) { return z * rcp_fast(1.0f + ex2_fast(-1.4426950408889634f * z)); }
__device__ __forceinline__ float act_gelu_tanh(float z) {
  // 0.5 z (1 + tanh u) = z / (1 + exp(-2u)),  u = sqrt(2/pi) (z + 0.044715 z^3)
  const float m = z * fmaf(-0.10294323973f, z * z, -2.3022081985f);       // -2 u log2(e)
  return z * rcp_fast(1.0f + ex2_fast(m));
}
__device__ __forceinline__ float act_gelu(float z) {
  // erfc(x) = (a1 t + ... + a5 t^5) exp(-x^2), t = 1 / (1 + p x), x >= 0, to 1.5e-7 (Abramowitz and Stegun, 7.1.26);
  // gelu(z) = max(z, 0) - |z| / 2 erfc(|z| / sqrt 2); the second part is 0 long before kGeluFlat
  const float mag = fabsf(fminf(z, kGeluFlat)), x = mag * 0.70710678118654752f;
  const float t = rcp_fast(fmaf(0.3275911f, x, 1.0f));
  float q = fmaf(1.061405429f, t, -1.453152027f);
  q = fmaf(q, t, 1.421413741f);
  q = fmaf(q, t, -0.284496736f);
  q = fmaf(q, t, 0.254829592f);
  const float e = ex2_fast(-0.72134752044448170f * mag * mag);           // exp(-z^2 / 2)
  return fmaf(-0.5f * mag, q * t * e, relu_nan(z));
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
      const uint64_t t = rcp_pair(fma2(mag, both(0.3275911f * 0.70710678118654752f), both(1.0f)));
      uint64_t q = fma2(both(1.061405429f), t, both(-1.453152027f));
      q = fma2(q, t, both(1.421413741f));
      q = fma2(q, t, both(-0.284496736f));
      q = fma2(q, t, both(0.254829592f));
      const uint64_t e = ex2_pair(mul_f32x2(mul_f32x2(mag, both(-0.72134752044448170f)), mag));
      z[j] = fma2(mul_f32x2(mag, both(-0.5f)), mul_f32x2(mul_f32x2(q, t), e), max0_pair(z[j]));
    }
  }
}

// The tensor-core product (linear_umma.cu); a.W holds bf16 values, a.w_scale is null where they need no scale.
mote_status_t launch_linear_umma(const LinearArgs& a, cudaStream_t stream);

}  // namespace mote
