// The norms before and after a block, fused with the block's gate and the residual stream (mote_block_norm):
//
//   p  = y, or  y * rsqrt(mean(y^2) + eps) * post_gain          norm after the block
//   r' = round( residual + scale * act(gate) * p )              gate and residual scale; rounded to the stream's type
//   n  = bf16( r' * rsqrt(mean(r'^2) + eps) * pre_gain )        norm before the next block, of the stored r'
//
// HBM-bound: y and the residual are read once, r' and n written once (8 bytes an element with a bf16 stream, 12 with an
// fp32 one).  A row stays in the registers of its threads between the passes (y and r as packed vectors of 8 elements);
// sums are fp32 in a fixed tree, so a row's result depends on its width alone.
#include "mote_common.cuh"
#include "mote_internal.h"

namespace mote {

struct BlockNormArgs {
  const uint16_t* y; int64_t ldy;
  const void* res; int64_t ldr;          // bf16 or fp32, or null
  const void* gate;                      // or null
  const float* post_gain; const float* pre_gain;
  void* res_out; uint16_t* normed_out;   // either may be null
  int64_t T;
  int64_t gate_tokens;                   // tokens per gate row, 0: one row for all
  int d, gate_cols;                      // gate_cols: 1 or d
  int post_norm, gate_f32, gate_sigmoid;
  float eps, scale;
};

__device__ __forceinline__ void unpack8(const uint4& v, float (&f)[8]) {
  f[0] = bf16_lo(v.x); f[1] = bf16_hi(v.x); f[2] = bf16_lo(v.y); f[3] = bf16_hi(v.y);
  f[4] = bf16_lo(v.z); f[5] = bf16_hi(v.z); f[6] = bf16_lo(v.w); f[7] = bf16_hi(v.w);
}
__device__ __forceinline__ uint4 pack8(const float (&f)[8]) {
  return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
}
__device__ __forceinline__ void load8_f32(const float* p, float (&f)[8]) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}
__device__ __forceinline__ float sigmoid_f32(float g) { return 1.0f / (1.0f + expf(-g)); }

// Sum over the row's `group` threads (whole warps); s: one slot per warp of the CTA, used once.
__device__ __forceinline__ float group_sum(float v, int group, float* s) {
  v = warp_sum(v);
  if (group == 32) return v;
  const int warp = threadIdx.x >> 5, per = group >> 5, first = warp / per * per;
  if ((threadIdx.x & 31) == 0) s[warp] = v;
  __syncthreads();
  float sum = s[first];
  for (int i = 1; i < per; ++i) sum += s[first + i];
  return sum;
}

// kVec: vectors of 8 elements per thread; kResF32: type of the residual stream.  A CTA holds blockDim.x / group rows.
template <int kVec, bool kResF32>
__global__ void __launch_bounds__(512) block_norm_kernel(BlockNormArgs a, int group) {
  __shared__ float s_post[16], s_pre[16];
  const int sub = threadIdx.x / group, tid = threadIdx.x - sub * group;
  const int64_t row = int64_t(blockIdx.x) * (blockDim.x / group) + sub;
  const bool row_ok = row < a.T;         // a CTA's rows meet at its barriers: rows past the end go along without loads
  const int n_vec = a.d / 8;
  pdl_wait();
  uint4 yv[kVec];
  float rf[kVec][8];
  const uint16_t* y = a.y + row * a.ldy;
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    const int v = i * group + tid;
    yv[i] = make_uint4(0u, 0u, 0u, 0u);
    if (row_ok && v < n_vec) yv[i] = reinterpret_cast<const uint4*>(y)[v];
  }
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    const int v = i * group + tid;
#pragma unroll
    for (int j = 0; j < 8; ++j) rf[i][j] = 0.0f;
    if (row_ok && a.res && v < n_vec) {
      if (kResF32) load8_f32(static_cast<const float*>(a.res) + row * a.ldr + v * 8, rf[i]);
      else unpack8(*reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.res) + row * a.ldr + v * 8), rf[i]);
    }
  }
  float mul = a.scale;
  if (a.post_norm) {
    float ss = 0.0f;
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      float f[8];
      unpack8(yv[i], f);
#pragma unroll
      for (int j = 0; j < 8; ++j) ss = fmaf(f[j], f[j], ss);
    }
    mul = rsqrtf(group_sum(ss, group, s_post) / float(a.d) + a.eps) * a.scale;
  }
  int64_t grow = 0;
  if (a.gate && row_ok) {
    grow = a.gate_tokens ? row / a.gate_tokens : 0;
    if (a.gate_cols == 1) {
      float g = a.gate_f32 ? static_cast<const float*>(a.gate)[grow]
                           : __uint_as_float(uint32_t(static_cast<const uint16_t*>(a.gate)[grow]) << 16);
      mul *= a.gate_sigmoid ? sigmoid_f32(g) : g;
    }
  }
  const bool wide_gate = a.gate && a.gate_cols != 1;
  float ss = 0.0f;
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    const int v = i * group + tid;
    if (!row_ok || v >= n_vec) continue;
    float p[8];
    unpack8(yv[i], p);
    if (a.post_norm && a.post_gain) {
      float g[8];
      load8_f32(a.post_gain + v * 8, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) p[j] *= g[j];
    }
    if (wide_gate) {
      float g[8];
      if (a.gate_f32) load8_f32(static_cast<const float*>(a.gate) + grow * a.d + v * 8, g);
      else unpack8(*reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.gate) + grow * a.d + v * 8), g);
#pragma unroll
      for (int j = 0; j < 8; ++j) p[j] *= a.gate_sigmoid ? sigmoid_f32(g[j]) : g[j];
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) rf[i][j] = fmaf(p[j], mul, rf[i][j]);
    if (kResF32) {
      if (a.res_out) {
        float4* o = reinterpret_cast<float4*>(static_cast<float*>(a.res_out) + row * a.d + v * 8);
        o[0] = make_float4(rf[i][0], rf[i][1], rf[i][2], rf[i][3]);
        o[1] = make_float4(rf[i][4], rf[i][5], rf[i][6], rf[i][7]);
      }
    } else {
      const uint4 o = pack8(rf[i]);
      if (a.res_out) *reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.res_out) + row * a.d + v * 8) = o;
      unpack8(o, rf[i]);                 // the norm is that of the stored values
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) ss = fmaf(rf[i][j], rf[i][j], ss);
  }
  if (!a.normed_out) return;
  const float inv = rsqrtf(group_sum(ss, group, s_pre) / float(a.d) + a.eps);
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    const int v = i * group + tid;
    if (!row_ok || v >= n_vec) continue;
    float n[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) n[j] = rf[i][j] * inv;
    if (a.pre_gain) {
      float g[8];
      load8_f32(a.pre_gain + v * 8, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) n[j] *= g[j];
    }
    *reinterpret_cast<uint4*>(a.normed_out + row * a.d + v * 8) = pack8(n);
  }
}

template <int kVec>
static cudaError_t launch_block_norm_vec(const BlockNormArgs& a, bool res_f32, int group, cudaStream_t stream) {
  const int threads = group < 128 ? 128 : group;
  const unsigned grid = (unsigned)((a.T + threads / group - 1) / (threads / group));
  return res_f32 ? launch_pdl(block_norm_kernel<kVec, true>, dim3(grid), dim3(threads), 0, stream, a, group)
                 : launch_pdl(block_norm_kernel<kVec, false>, dim3(grid), dim3(threads), 0, stream, a, group);
}

// [a, a + na) and [b, b + nb) share a byte
static bool overlaps(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t pa = reinterpret_cast<uintptr_t>(a), pb = reinterpret_cast<uintptr_t>(b);
  return a && b && pa < pb + nb && pb < pa + na;
}

}  // namespace mote

extern "C" mote_status_t mote_block_norm(const mote_block_norm_t* N, const void* y, int64_t ldy, const void* residual,
                                         int64_t ldr, const void* gate, int64_t T, void* res_out, void* normed_out,
                                         void* stream) {
  using namespace mote;
  if (!N) return MOTE_ERR_NULL;
  const int64_t d = N->d;
  if (d <= 0 || d % 8 != 0 || d > 32768 || T < 0 || T > (int64_t(1) << 24)) return MOTE_ERR_SHAPE;
  if (!(N->eps >= 0.0f) || N->gate_tokens < 0) return MOTE_ERR_SHAPE;
  if (N->gate_cols != 0 && N->gate_cols != 1 && N->gate_cols != d) return MOTE_ERR_SHAPE;
  if (N->res_dtype != MOTE_DTYPE_F32 && N->res_dtype != MOTE_DTYPE_BF16) return MOTE_ERR_DTYPE;
  if (N->gate_cols && N->gate_dtype != MOTE_DTYPE_F32 && N->gate_dtype != MOTE_DTYPE_BF16) return MOTE_ERR_DTYPE;
  if (T == 0) return MOTE_OK;
  if (!y || (!res_out && !normed_out) || (N->gate_cols && !gate)) return MOTE_ERR_NULL;
  const bool f32 = N->res_dtype == MOTE_DTYPE_F32;
  if (T > 1 && (ldy < d || (residual && ldr < d))) return MOTE_ERR_SHAPE;
  if (T > 1 && (ldy % 8 != 0 || (residual && ldr % (f32 ? 4 : 8) != 0))) return MOTE_ERR_ALIGN;
  const void* ptrs[] = {y, residual, N->gate_cols == d ? gate : nullptr, N->post_gain, N->pre_gain, res_out, normed_out};
  for (const void* p : ptrs)
    if (p && !aligned16(p)) return MOTE_ERR_ALIGN;
  if (N->gate_cols == 1 && (reinterpret_cast<uintptr_t>(gate) & (N->gate_dtype == MOTE_DTYPE_F32 ? 3u : 1u))) return MOTE_ERR_ALIGN;
  // An output may take the place of an input, element by element; any other overlap would be read after it was written.
  const int64_t sy = T > 1 ? ldy : d, sr = T > 1 ? ldr : d;
  const int rb = f32 ? 4 : 2;
  auto bad = [&](const void* out, int out_elem, const void* in, int in_elem, int64_t in_stride) {
    return overlaps(out, size_t(T) * d * out_elem, in, size_t((T - 1) * in_stride + d) * in_elem) &&
           !(out == in && out_elem == in_elem && in_stride == d);
  };
  if (bad(res_out, rb, y, 2, sy) || bad(res_out, rb, residual, rb, sr) || bad(normed_out, 2, y, 2, sy) ||
      bad(normed_out, 2, residual, rb, sr) || overlaps(res_out, size_t(T) * d * rb, normed_out, size_t(T) * d * 2))
    return MOTE_ERR_SHAPE;
  const int64_t gate_rows = !N->gate_cols ? 0 : N->gate_tokens ? (T + N->gate_tokens - 1) / N->gate_tokens : 1;
  const size_t gate_bytes = size_t(gate_rows) * N->gate_cols * (N->gate_dtype == MOTE_DTYPE_F32 ? 4 : 2);
  if (N->gate_cols && (overlaps(res_out, size_t(T) * d * rb, gate, gate_bytes) || overlaps(normed_out, size_t(T) * d * 2, gate, gate_bytes)))
    return MOTE_ERR_SHAPE;
  BlockNormArgs a{};
  a.y = static_cast<const uint16_t*>(y); a.ldy = ldy; a.res = residual; a.ldr = ldr;
  a.gate = N->gate_cols ? gate : nullptr; a.gate_cols = N->gate_cols; a.gate_tokens = N->gate_tokens;
  a.gate_f32 = N->gate_dtype == MOTE_DTYPE_F32; a.gate_sigmoid = N->gate_sigmoid != 0;
  a.post_norm = N->post_norm != 0; a.post_gain = N->post_gain; a.pre_gain = N->pre_gain;
  a.res_out = res_out; a.normed_out = static_cast<uint16_t*>(normed_out);
  a.T = T; a.d = (int)d; a.eps = N->eps; a.scale = N->scale;
  const int n_vec = (int)d / 8;
  // Threads of a row: with rows to fill the GPU, up to four vectors a thread; with few, one.
  int vec = T > 1024 ? 4 : T > 256 ? 2 : 1;
  while (vec * 512 < n_vec) vec *= 2;
  int group = 32;
  while (group * vec < n_vec) group *= 2;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  MOTE_CUDA_OK(vec == 8 ? launch_block_norm_vec<8>(a, f32, group, s)
               : vec == 4 ? launch_block_norm_vec<4>(a, f32, group, s)
               : vec == 2 ? launch_block_norm_vec<2>(a, f32, group, s) : launch_block_norm_vec<1>(a, f32, group, s));
  MOTE_LAUNCH_OK();
  return MOTE_OK;
}
