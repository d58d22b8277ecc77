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

__device__ __forceinline__ float apply_act(float z, int act) {
  switch (act) {
    case MOTE_ACT_RELU: return fmaxf(z, 0.0f);
    case MOTE_ACT_SILU: return z / (1.0f + expf(-z));
    case MOTE_ACT_GELU: return 0.5f * z * (1.0f + erff(z * 0.70710678118654752f));
    case MOTE_ACT_GELU_TANH: {
      // 0.5 z (1 + tanh u) = z / (1 + exp(-2u)),  u = sqrt(2/pi) (z + 0.044715 z^3)
      const float u = 0.79788456080286536f * (z + 0.044715f * z * z * z);
      return z / (1.0f + expf(-2.0f * u));
    }
  }
  return z;
}

// The tensor-core product (linear_umma.cu); a.W holds bf16 values, a.w_scale is null where they need no scale.
mote_status_t launch_linear_umma(const LinearArgs& a, cudaStream_t stream);

}  // namespace mote
