// The norms before and after a block, fused with the block's gate and the residual stream (mote_block_norm):
//
//   p  = y, or  y * rsqrt(mean(y^2) + eps) * post_gain          norm after the block
//   r' = round( residual + scale * act(gate) * p )              gate and residual scale; rounded to the stream's type
//   n  = bf16( r' * rsqrt(mean(r'^2) + eps) * pre_gain )        norm before the next block, of the stored r'
//
// HBM-bound: y and the residual are read once, r' and n written once (8 bytes an element with a bf16 stream, 12 with an
// fp32 one).  A row stays in the registers of its threads between the passes; sums are fp32 in a fixed tree that goes by the row's
// width alone, so a row's result does not depend on the batch.
//
// 8192 x 2048, norms on both sides, bf16 stream: 28 us, 4 800 GB/s (a plain copy of the same bytes 23).  A row per CTA, weights read for
// each: 42; rows side by side, fp32 instructions one at a time: 36 to 47, at 51 instructions an element.
#include <algorithm>

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
  float eps, scale, inv_d;
};

// Eight elements as four pairs (fp32x2 instructions work on two at a time: the kernel is as much issue- as HBM-bound).
struct Eight { uint64_t p[4]; };
__device__ __forceinline__ uint64_t fma_f32x2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ Eight unpack8(const uint4& v) {
  Eight e;
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) e.p[j] = f32x2_bits(w[j] << 16, w[j] & 0xFFFF0000u);
  return e;
}
__device__ __forceinline__ uint4 pack8(const Eight& e) {
  uint32_t w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    float lo, hi;
    unpack_f32x2(e.p[j], lo, hi);
    w[j] = pack_bf16x2(lo, hi);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ Eight load8_f32(const float* p) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  return Eight{{f32x2(a.x, a.y), f32x2(a.z, a.w), f32x2(b.x, b.y), f32x2(b.z, b.w)}};
}
__device__ __forceinline__ Eight operator*(const Eight& a, const Eight& b) {
  return Eight{{mul_f32x2(a.p[0], b.p[0]), mul_f32x2(a.p[1], b.p[1]), mul_f32x2(a.p[2], b.p[2]), mul_f32x2(a.p[3], b.p[3])}};
}
__device__ __forceinline__ Eight operator*(const Eight& a, float s) {
  const uint64_t b = f32x2(s, s);
  return Eight{{mul_f32x2(a.p[0], b), mul_f32x2(a.p[1], b), mul_f32x2(a.p[2], b), mul_f32x2(a.p[3], b)}};
}
// sum of squares on top of a pair of sums
__device__ __forceinline__ uint64_t add_squares(const Eight& e, uint64_t acc) {
#pragma unroll
  for (int j = 0; j < 4; ++j) acc = fma_f32x2(e.p[j], e.p[j], acc);
  return acc;
}
// By the special-function unit: a few 2^-24 and |g| 2^-24 off.  (A gate for each element, 3088 x 1536: 21.3 us, 26 with expf and a division.)
__device__ __forceinline__ float sigmoid_f32(float g) {
  float e, s;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(-1.4426950408889634f * g));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s) : "f"(1.0f + e));
  return s;
}

// Sum over a row's `group` threads (whole warps; sub: the row's number in the CTA); s: one slot per warp of the CTA.  `group` threads
// meet at a barrier of their own.
__device__ __forceinline__ float group_sum(uint64_t pair, int group, int sub, float* s) {
  float lo, hi;
  unpack_f32x2(pair, lo, hi);
  float v = warp_sum(lo + hi);
  if (group == 32) return v;
  const int warp = threadIdx.x >> 5, per = group >> 5, first = warp / per * per;
  if ((threadIdx.x & 31) == 0) s[warp] = v;
  asm volatile("bar.sync %0, %1;" ::"r"(sub + 1), "r"(group) : "memory");
  v = s[first];
  if (per == 4) {                         // the usual widths: one load
    const float4 q = *reinterpret_cast<const float4*>(s + first);
    return ((q.x + q.y) + q.z) + q.w;
  }
  for (int w = 1; w < per; ++w) v += s[first + w];
  return v;
}

template <bool kF32>
struct Stored8 {                          // 8 elements of the residual stream as they are stored
  uint4 v[kF32 ? 2 : 1];
  __device__ __forceinline__ Eight get() const {
    if (!kF32) return unpack8(v[0]);
    const uint4 a = v[0], b = v[kF32 ? 1 : 0];
    return Eight{{f32x2_bits(a.x, a.y), f32x2_bits(a.z, a.w), f32x2_bits(b.x, b.y), f32x2_bits(b.z, b.w)}};
  }
  __device__ __forceinline__ void put(const Eight& e) {        // rounds to the stored type
    if (!kF32) { v[0] = pack8(e); return; }
    float f[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) unpack_f32x2(e.p[j], f[2 * j], f[2 * j + 1]);
    v[0] = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    v[kF32 ? 1 : 0] = make_uint4(__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7]));
  }
};

// A thread's weights for its columns: post_gain * act(gate) (where the gate has a value for each channel) and pre_gain.  Held in
// registers for kVec <= 2, read where they are used for wider rows.
template <int kVec>
struct ColumnWeights {
  static constexpr bool kHeld = kVec <= 2;
  Eight mix[kHeld ? kVec : 1], pre[kHeld ? kVec : 1];
  int64_t gate_row;                       // the gate row that `mix` holds (-1: none yet)
};
__device__ __forceinline__ Eight acted_gate(const BlockNormArgs& a, Eight g) {
  if (a.gate_sigmoid)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float lo, hi;
      unpack_f32x2(g.p[j], lo, hi);
      g.p[j] = f32x2(sigmoid_f32(lo), sigmoid_f32(hi));
    }
  return g;
}
__device__ __forceinline__ Eight mixed_weights(const BlockNormArgs& a, int64_t gate_row, int col) {
  Eight m;
#pragma unroll
  for (int j = 0; j < 4; ++j) m.p[j] = f32x2(1.0f, 1.0f);
  if (a.post_gain) m = load8_f32(a.post_gain + col);
  if (a.gate_cols > 1)
    m = m * acted_gate(a, a.gate_f32 ? load8_f32(static_cast<const float*>(a.gate) + gate_row * a.d + col)
                                     : unpack8(*reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.gate) + gate_row * a.d + col)));
  return m;
}

__device__ __forceinline__ int64_t gate_row_of(const BlockNormArgs& a, int64_t row) {
  if (a.gate_tokens <= 1) return a.gate_tokens ? row : 0;
  return ((row | a.gate_tokens) >> 32) ? row / a.gate_tokens : int64_t(uint32_t(row) / uint32_t(a.gate_tokens));
}
// A gate's one value for the row.
__device__ __forceinline__ float load_token_gate(const BlockNormArgs& a, int64_t row) {
  if (a.gate_cols != 1 || row >= a.T) return 0.0f;
  const int64_t at = gate_row_of(a, row);
  return a.gate_f32 ? static_cast<const float*>(a.gate)[at] : __uint_as_float(uint32_t(static_cast<const uint16_t*>(a.gate)[at]) << 16);
}

// One row.  Threads of a row that is not there (row >= T) go along as zeros.  gv: the row's own gate vectors, kGate (1: bf16, 2: fp32)
// units of 16 bytes each; kGate = 0: a gate with a value for each channel is read here.  token_gate: the row's one value of another gate.
template <int kVec, bool kF32, int kGate>
__device__ __forceinline__ void norm_row(const BlockNormArgs& a, int64_t row, int group, int sub, int tid, const uint4 (&yv)[kVec],
                                         Stored8<kF32> (&rv)[kVec], const Stored8<kGate == 2> (&gv)[kVec], float token_gate,
                                         ColumnWeights<kVec>& cw, float* s_post, float* s_pre) {
  constexpr bool kHeld = ColumnWeights<kVec>::kHeld;
  const bool live = row < a.T;
  float mul = a.scale;
  const int64_t gate_row = a.gate_cols > 1 && live ? gate_row_of(a, row) : 0;
  if (a.gate_cols == 1) mul *= a.gate_sigmoid ? sigmoid_f32(token_gate) : token_gate;
  if (a.post_norm) {
    uint64_t ss = 0ull;
#pragma unroll
    for (int i = 0; i < kVec; ++i) ss = add_squares(unpack8(yv[i]), ss);
    mul *= rsqrtf(group_sum(ss, group, sub, s_post) * a.inv_d + a.eps);
  }
  const bool weighted = a.post_gain || a.gate_cols > 1;
  const uint64_t mul2 = f32x2(mul, mul);
  const int64_t out_at = row * a.d + tid * 8;
  uint64_t ss = 0ull;
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    const int col = (i * group + tid) * 8;
    if (!live || col >= a.d) continue;
    Eight p = unpack8(yv[i]);
    if (weighted) {
      Eight& m = cw.mix[kHeld ? i : 0];
      if (kGate) {                        // (`mix` holds the gain alone)
        const Eight g = acted_gate(a, gv[i].get());
        p = p * (!a.post_gain ? g : (kHeld ? m : load8_f32(a.post_gain + col)) * g);      // (the products of mixed_weights, in its order)
      } else {
        if (!kHeld || gate_row != cw.gate_row) m = mixed_weights(a, gate_row, col);
        p = p * m;
      }
    }
    Eight x = rv[i].get();
#pragma unroll
    for (int j = 0; j < 4; ++j) x.p[j] = fma_f32x2(p.p[j], mul2, x.p[j]);
    rv[i].put(x);
    if (a.res_out) {
      uint4* o = kF32 ? reinterpret_cast<uint4*>(static_cast<float*>(a.res_out) + out_at + i * group * 8)
                      : reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.res_out) + out_at + i * group * 8);
#pragma unroll
      for (int u = 0; u < (kF32 ? 2 : 1); ++u) o[u] = rv[i].v[u];
    }
    ss = add_squares(rv[i].get(), ss);    // the norm is that of the stored values
  }
  if (live) cw.gate_row = gate_row;
  if (!a.normed_out) return;
  const float inv = rsqrtf(group_sum(ss, group, sub, s_pre) * a.inv_d + a.eps);
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    const int col = (i * group + tid) * 8;
    if (!live || col >= a.d) continue;
    Eight x = rv[i].get() * inv;
    if (a.pre_gain) x = x * (kHeld ? cw.pre[kHeld ? i : 0] : load8_f32(a.pre_gain + col));
    *reinterpret_cast<uint4*>(a.normed_out + out_at + i * group * 8) = pack8(x);
  }
}
template <int kVec, int kGate>
__device__ __forceinline__ void start_weights(const BlockNormArgs& a, int group, int tid, ColumnWeights<kVec>& cw) {
  cw.gate_row = -1;
  if (ColumnWeights<kVec>::kHeld)
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      const int col = min((i * group + tid) * 8, a.d - 8);
      if (a.pre_gain) cw.pre[ColumnWeights<kVec>::kHeld ? i : 0] = load8_f32(a.pre_gain + col);
      if (kGate && a.post_gain) cw.mix[ColumnWeights<kVec>::kHeld ? i : 0] = load8_f32(a.post_gain + col);
    }
}

// A row (or several, of few threads each) per CTA.
template <int kVec, bool kF32>
__global__ void __launch_bounds__(512) block_norm_kernel(BlockNormArgs a, int group) {
  __shared__ __align__(16) float s_post[16], s_pre[16];
  const int sub = threadIdx.x / group, tid = threadIdx.x - sub * group;
  const int64_t row = int64_t(blockIdx.x) * (blockDim.x / group) + sub;
  pdl_wait();
  const float token_gate = load_token_gate(a, row);
  uint4 yv[kVec];
  Stored8<kF32> rv[kVec];
#pragma unroll
  for (int i = 0; i < kVec; ++i) {
    const int col = (i * group + tid) * 8;
    const bool in = row < a.T && col < a.d;
    yv[i] = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int u = 0; u < (kF32 ? 2 : 1); ++u) rv[i].v[u] = make_uint4(0u, 0u, 0u, 0u);
    if (in) yv[i] = *reinterpret_cast<const uint4*>(a.y + row * a.ldy + col);
    if (in && a.res) {
      const uint4* q = reinterpret_cast<const uint4*>(static_cast<const char*>(a.res) + (row * a.ldr + col) * (kF32 ? 4 : 2));
#pragma unroll
      for (int u = 0; u < (kF32 ? 2 : 1); ++u) rv[i].v[u] = q[u];
    }
  }
  ColumnWeights<kVec> cw;
  start_weights<kVec, 0>(a, group, tid, cw);
  const Stored8<false> none[kVec] = {};
  norm_row<kVec, kF32, 0>(a, row, group, sub, tid, yv, rv, none, token_gate, cw, s_post, s_pre);
}

// Many rows: the threads of a row walk over rows.  A thread fetches its own vectors of the rows to come into shared memory
// (cp.async; nobody else reads them, so nothing but its own copies has to be waited for), which keeps loads in flight
// through the sums and barriers of the present row, and it holds its columns' weights all the way.
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
// 16-byte units of a thread's vector: y, the stream's one or two, and those of a gate that has a row for each token.  Four rows ahead where two
// CTAs of them fit an SM.  (8192 x 2048: three stages 32 us, six 29; three CTAs per SM, whose registers spill, 33.)
template <int kVec, bool kF32, int kGate>
struct NormRing {
  static constexpr int kUnits = 1 + (kF32 ? 2 : 1) + kGate;
  static constexpr int kStages = kVec * kUnits <= 6 ? 4 : kVec * kUnits <= 8 ? 3 : 2;
  static constexpr int kStageBytes = kVec * kUnits * 16;                   // per thread
};
template <int kVec, bool kF32, int kGate>
__global__ void __launch_bounds__(256, 2) block_norm_stream_kernel(BlockNormArgs a, int group) {
  using R = NormRing<kVec, kF32, kGate>;
  constexpr int kUnits = R::kUnits, kStages = R::kStages, kResUnits = kF32 ? 2 : 1;
  extern __shared__ uint4 s_ring[];                        // [stage][vector][unit][thread]
  __shared__ __align__(16) float s_post[2][8], s_pre[2][8];
  const int threads = blockDim.x, rows = threads / group;
  const int sub = threadIdx.x / group, tid = threadIdx.x - sub * group;
  const int64_t step = int64_t(gridDim.x) * rows;
  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(s_ring) + threadIdx.x * 16;
  auto fetch = [&](int64_t row, int stage) {
    if (row < a.T) {
      const uint16_t* y = a.y + row * a.ldy + tid * 8;
      const char* res = static_cast<const char*>(a.res) + (row * a.ldr + tid * 8) * (kF32 ? 4 : 2);
      const char* gate = static_cast<const char*>(a.gate) + (row * a.d + tid * 8) * (kGate == 2 ? 4 : 2);
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        if ((i * group + tid) * 8 >= a.d) continue;
        const uint32_t dst = ring + ((stage * kVec + i) * kUnits) * (threads * 16);
        cp_async16(dst, y + i * group * 8);
        if (a.res)
#pragma unroll
          for (int u = 0; u < kResUnits; ++u) cp_async16(dst + (1 + u) * (threads * 16), res + i * group * 8 * (kF32 ? 4 : 2) + u * 16);
#pragma unroll
        for (int u = 0; u < kGate; ++u)
          cp_async16(dst + (1 + kResUnits + u) * (threads * 16), gate + i * group * 8 * (kGate == 2 ? 4 : 2) + u * 16);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  // what no copy fills (past the row's end, no residual) reads as zeros
#pragma unroll
  for (int i = 0; i < kStages * kVec * kUnits; ++i) {
    const int unit = i % kUnits;
    const bool copied = ((i / kUnits % kVec) * group + tid) * 8 < a.d && (unit == 0 || unit > kResUnits || a.res);
    if (!copied) s_ring[i * threads + threadIdx.x] = make_uint4(0u, 0u, 0u, 0u);
  }
  pdl_wait();
  ColumnWeights<kVec> cw;
  start_weights<kVec, kGate>(a, group, tid, cw);
  int64_t row = int64_t(blockIdx.x) * rows + sub;
#pragma unroll
  for (int s = 0; s < kStages - 1; ++s) fetch(row + s * step, s);
  int stage = 0, ahead = kStages - 1, parity = 0;
  float next_gate = load_token_gate(a, row);
  for (; row < a.T; row += step) {                         // all threads of a row together
    const float token_gate = next_gate;
    next_gate = load_token_gate(a, row + step);
    fetch(row + (kStages - 1) * step, ahead);
    asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
    uint4 yv[kVec];
    Stored8<kF32> rv[kVec];
    Stored8<kGate == 2> gv[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      const uint4* from = s_ring + ((stage * kVec + i) * kUnits) * threads + threadIdx.x;
      yv[i] = from[0];
#pragma unroll
      for (int u = 0; u < kResUnits; ++u) rv[i].v[u] = from[(1 + u) * threads];
#pragma unroll
      for (int u = 0; u < kGate; ++u) gv[i].v[u] = from[(1 + kResUnits + u) * threads];
    }
    norm_row<kVec, kF32, kGate>(a, row, group, sub, tid, yv, rv, gv, token_gate, cw, s_post[parity], s_pre[parity]);
    ahead = stage;
    stage = stage + 1 == kStages ? 0 : stage + 1;
    parity ^= 1;
  }
}

template <int kVec>
static cudaError_t launch_block_norm(const BlockNormArgs& a, bool res_f32, int group, cudaStream_t stream) {
  const int rows = std::max(1, 128 / group), threads = rows * group;
  const unsigned grid = (unsigned)((a.T + rows - 1) / rows);
  return res_f32 ? launch_pdl(block_norm_kernel<kVec, true>, dim3(grid), dim3(threads), 0, stream, a, group)
                 : launch_pdl(block_norm_kernel<kVec, false>, dim3(grid), dim3(threads), 0, stream, a, group);
}
template <int kVec, bool kF32, int kGate>
static cudaError_t launch_stream_as(const BlockNormArgs& a, int group, cudaStream_t stream) {
  using R = NormRing<kVec, kF32, kGate>;
  static PerDeviceOnce once;
  const cudaError_t e = set_max_dynamic_smem(once, block_norm_stream_kernel<kVec, kF32, kGate>, R::kStages * R::kStageBytes * 256);
  if (e != cudaSuccess) return e;
  const int rows = std::max(1, 256 / group), threads = rows * group, smem = R::kStages * R::kStageBytes * threads;
  const int64_t blocks = (a.T + rows - 1) / rows;
  const int per_sm = std::max(1, std::min(512 / threads, 220 * 1024 / (smem + 2048)));
  return launch_pdl(block_norm_stream_kernel<kVec, kF32, kGate>, dim3((unsigned)std::min<int64_t>(blocks, device_sm_count() * per_sm)), dim3(threads),
                    smem, stream, a, group);
}
template <int kVec, bool kF32>
static cudaError_t launch_stream_gate(const BlockNormArgs& a, int group, cudaStream_t stream) {
  if (a.gate_cols <= 1 || a.gate_tokens != 1) return launch_stream_as<kVec, kF32, 0>(a, group, stream);
  return a.gate_f32 ? launch_stream_as<kVec, kF32, 2>(a, group, stream) : launch_stream_as<kVec, kF32, 1>(a, group, stream);
}
template <int kVec>
static cudaError_t launch_block_norm_stream(const BlockNormArgs& a, bool res_f32, int group, cudaStream_t stream) {
  return res_f32 ? launch_stream_gate<kVec, true>(a, group, stream) : launch_stream_gate<kVec, false>(a, group, stream);
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
  const int64_t gate_rows = !N->gate_cols ? 0 : N->gate_tokens ? (T - 1) / N->gate_tokens + 1 : 1;
  const void* const read[] = {N->gate_cols ? gate : nullptr, N->post_norm ? N->post_gain : nullptr, N->pre_gain};
  const size_t read_bytes[] = {size_t(gate_rows) * N->gate_cols * (N->gate_dtype == MOTE_DTYPE_F32 ? 4 : 2), size_t(d) * 4, size_t(d) * 4};
  for (int i = 0; i < 3; ++i)
    if (overlaps(res_out, size_t(T) * d * rb, read[i], read_bytes[i]) || overlaps(normed_out, size_t(T) * d * 2, read[i], read_bytes[i]))
      return MOTE_ERR_SHAPE;
  BlockNormArgs a{};
  a.y = static_cast<const uint16_t*>(y); a.ldy = ldy; a.res = residual; a.ldr = ldr;
  a.gate = N->gate_cols ? gate : nullptr; a.gate_cols = N->gate_cols; a.gate_tokens = N->gate_tokens;
  a.gate_f32 = N->gate_dtype == MOTE_DTYPE_F32; a.gate_sigmoid = N->gate_sigmoid != 0;
  a.post_norm = N->post_norm != 0; a.post_gain = N->post_norm ? N->post_gain : nullptr; a.pre_gain = N->pre_gain;
  a.res_out = res_out; a.normed_out = static_cast<uint16_t*>(normed_out);
  a.T = T; a.d = (int)d; a.eps = N->eps; a.scale = N->scale; a.inv_d = 1.0f / float(d);
  const int n_vec = (int)d / 8;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  // Threads of a row, by its width alone, so that a row's sums do not depend on T: two vectors a thread (one in rows of up to 256
  // elements), more where that takes over 256 threads, and up to 512 threads for rows of more than 8192 elements.
  const int most = n_vec <= 1024 ? 256 : 512;
  int vec = n_vec <= 32 ? 1 : 2;
  while (vec * most < n_vec) vec *= 2;
  const int group = ((n_vec + vec - 1) / vec + 31) / 32 * 32;
  if (n_vec <= 1024 && T >= int64_t(device_sm_count()) * 8)            // rows enough to walk over
    e = vec == 4   ? launch_block_norm_stream<4>(a, f32, group, s)
        : vec == 2 ? launch_block_norm_stream<2>(a, f32, group, s) : launch_block_norm_stream<1>(a, f32, group, s);
  else
    e = vec == 8   ? launch_block_norm<8>(a, f32, group, s)
        : vec == 4 ? launch_block_norm<4>(a, f32, group, s)
        : vec == 2 ? launch_block_norm<2>(a, f32, group, s) : launch_block_norm<1>(a, f32, group, s);
  if (e != cudaSuccess) return MOTE_ERR_CUDA;
  MOTE_LAUNCH_OK();
  return MOTE_OK;
}
