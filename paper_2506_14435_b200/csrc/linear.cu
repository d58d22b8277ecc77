// Matrix product with bias, activation and residual in its epilogue (mote_linear):
//
//   out = act( scale_n * (x W^T) + bias ) [+ residual]
//
// W [N, K] is bf16, or the RTN codes of mote_rtn_quant (INT8 / INT4) with one scale per row; fp32 accumulation, one rounding
// to the output's type.
//
// Up to kStreamMaxTokens tokens the product is a weight stream: a CTA owns 16 rows of W, its warps share K, a lane loads 16 bytes of
// one weight row straight into registers (codes are expanded there) and feeds them to warp-level MMAs as the A operand with the
// tokens as the 8-wide B operand.  Every weight byte is read once.
#include <algorithm>

#include "linear_act.cuh"

namespace mote {

__device__ __forceinline__ uint4 ldg_once(const void* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ uint2 ldg_once8(const void* p) {
  uint2 v;
  asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
  return v;
}
__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

constexpr int kStreamWarps = 8;
constexpr int kStreamRows = 16;

// kBits: storage of W.  A step covers 32 (bf16), 64 (INT8) or 64 (INT4, 32 code bytes) elements of K: lane (g, t) = (lane / 4, lane % 4)
// takes elements [step * kStep + t * kLane, + kLane) of weight rows g and g + 8 and of its token column; the reduction index may be
// permuted as long as both operands are.
template <int NT, int kBits>
__global__ void __launch_bounds__(kStreamWarps * 32) linear_stream_kernel(LinearArgs a) {
  constexpr int kLane = kBits == 16 ? 8 : 16, kStep = 4 * kLane;
  constexpr int kAhead = 4;
  __shared__ float s_part[kStreamWarps][NT * 4][32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const unsigned row_tiles = unsigned((a.N + kStreamRows - 1) / kStreamRows);
  const int64_t n0 = int64_t(blockIdx.x % row_tiles) * kStreamRows;
  const int64_t t0 = int64_t(blockIdx.x / row_tiles) * (NT * 8);
  const int n_steps = (a.K + kStep - 1) / kStep;
  const int sb = n_steps * warp / kStreamWarps, se = n_steps * (warp + 1) / kStreamWarps;
  const int64_t row_bytes = int64_t(a.K) * kBits / 8;
  const uint8_t* wa = static_cast<const uint8_t*>(a.W) + min(n0 + g, a.N - 1) * row_bytes + t * (kLane * kBits / 8);
  const uint8_t* wb = static_cast<const uint8_t*>(a.W) + min(n0 + g + 8, a.N - 1) * row_bytes + t * (kLane * kBits / 8);
  const uint16_t* tok[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) tok[n] = t0 + n * 8 + g < a.T ? a.x + (t0 + n * 8 + g) * a.ldx + t * kLane : nullptr;
  // 16 bytes of a weight row, or 8 where they hold the lane's 16 four-bit codes
  auto load_w = [&](const uint8_t* row, int s) {
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (kBits == 4) v = make_uint4(0x88888888u, 0x88888888u, 0u, 0u);      // codes of weight 0
    if (s < se && s * kStep + t * kLane < a.K) {
      if (kBits == 4) {
        const uint2 h = ldg_once8(row + s * (kStep / 2));
        v.x = h.x; v.y = h.y;
      } else {
        v = ldg_once(row + int64_t(s) * (kStep * kBits / 8));
      }
    }
    return v;
  };
  float acc[NT][4];
#pragma unroll
  for (int n = 0; n < NT; ++n) acc[n][0] = acc[n][1] = acc[n][2] = acc[n][3] = 0.0f;
  pdl_wait();
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.status = 0u;
  uint4 qa[kAhead], qb[kAhead];
#pragma unroll
  for (int i = 0; i < kAhead; ++i) { qa[i] = load_w(wa, sb + i); qb[i] = load_w(wb, sb + i); }
  for (int s0 = sb; s0 < se; s0 += kAhead) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int s = s0 + i;
      if (s < se) {
        const uint4 ca = qa[i], cb = qb[i];
        qa[i] = load_w(wa, s + kAhead);
        qb[i] = load_w(wb, s + kAhead);
        const bool in = s * kStep + t * kLane < a.K;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          uint4 x0 = make_uint4(0u, 0u, 0u, 0u), x1 = x0;
          if (tok[n] && in) {
            const uint4* xp = reinterpret_cast<const uint4*>(tok[n] + s * kStep);
            x0 = xp[0];
            if (kBits != 16) x1 = xp[1];
          }
          if (kBits == 16) {
            mma_16816(acc[n], ca.x, cb.x, ca.y, cb.y, x0.x, x0.y);
            mma_16816(acc[n], ca.z, cb.z, ca.w, cb.w, x0.z, x0.w);
          } else {
            const uint32_t xw[8] = {x0.x, x0.y, x0.z, x0.w, x1.x, x1.y, x1.z, x1.w};
            uint32_t ea[8], eb[8];
            if (kBits == 8) {
              const uint32_t pa[4] = {ca.x, ca.y, ca.z, ca.w}, pb[4] = {cb.x, cb.y, cb.z, cb.w};
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                s8x4_to_bf16x2(pa[j], ea[2 * j], ea[2 * j + 1]);
                s8x4_to_bf16x2(pb[j], eb[2 * j], eb[2 * j + 1]);
              }
            } else {
              uint32_t h[4];
              u4x8_to_bf16x2(ca.x, h); ea[0] = h[0]; ea[1] = h[1]; ea[2] = h[2]; ea[3] = h[3];
              u4x8_to_bf16x2(ca.y, h); ea[4] = h[0]; ea[5] = h[1]; ea[6] = h[2]; ea[7] = h[3];
              u4x8_to_bf16x2(cb.x, h); eb[0] = h[0]; eb[1] = h[1]; eb[2] = h[2]; eb[3] = h[3];
              u4x8_to_bf16x2(cb.y, h); eb[4] = h[0]; eb[5] = h[1]; eb[6] = h[2]; eb[7] = h[3];
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) mma_16816(acc[n], ea[2 * j], eb[2 * j], ea[2 * j + 1], eb[2 * j + 1], xw[2 * j], xw[2 * j + 1]);
          }
        }
      }
    }
  }
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) s_part[warp][n * 4 + i][lane] = acc[n][i];
  __syncthreads();
  // value i of token tile n at lane (g, t) is weight row g + 8 * (i / 2), token 8n + 2t + (i & 1); thread -> (token, row) with
  // the rows fastest, so that a token's 16 outputs leave together
  for (int o = threadIdx.x; o < NT * 8 * kStreamRows; o += kStreamWarps * 32) {
    const int row = o & 15, token = o >> 4;
    const int v = (token >> 3) * 4 + (row >> 3) * 2 + (token & 1), l = (row & 7) * 4 + ((token & 7) >> 1);
    const int64_t tt = t0 + token, nn = n0 + row;
    if (tt >= a.T || nn >= a.N) continue;
    float z = s_part[0][v][l];
#pragma unroll
    for (int w = 1; w < kStreamWarps; ++w) z += s_part[w][v][l];
    if (kBits != 16) z *= a.w_scale[nn];
    if (a.bias) z += a.bias[nn];
    z = apply_act(z, a.act);
    if (a.res) z += __uint_as_float(uint32_t(a.res[tt * a.ldr + nn]) << 16);
    if (a.out_f32) static_cast<float*>(a.out)[tt * a.N + nn] = z;
    else static_cast<uint16_t*>(a.out)[tt * a.N + nn] = (uint16_t)(pack_bf16x2(z, 0.0f) & 0xFFFFu);
  }
}

template <int NT>
static cudaError_t launch_stream(const LinearArgs& a, int bits, cudaStream_t stream) {
  const dim3 grid((unsigned)((a.N + kStreamRows - 1) / kStreamRows * ((a.T + NT * 8 - 1) / (NT * 8))));
  const dim3 block(kStreamWarps * 32);
  return bits == 16  ? launch_pdl(linear_stream_kernel<NT, 16>, grid, block, 0, stream, a)
         : bits == 8 ? launch_pdl(linear_stream_kernel<NT, 8>, grid, block, 0, stream, a)
                     : launch_pdl(linear_stream_kernel<NT, 4>, grid, block, 0, stream, a);
}

// RTN codes -> the same integers as bf16, for the tensor-core product; 8 code bytes per thread and step.
__global__ void __launch_bounds__(256) linear_expand_kernel(const uint2* __restrict__ codes, uint4* __restrict__ out, int64_t n_chunks, int bits) {
  pdl_wait();
  const int64_t stride = int64_t(gridDim.x) * blockDim.x;
  for (int64_t i = int64_t(blockIdx.x) * blockDim.x + threadIdx.x; i < n_chunks; i += stride) {
    const uint2 w = codes[i];
    uint32_t e[4], h[4];
    if (bits == 8) {
      s8x4_to_bf16x2(w.x, e[0], e[1]);
      s8x4_to_bf16x2(w.y, e[2], e[3]);
      out[i] = make_uint4(e[0], e[1], e[2], e[3]);
    } else {
      u4x8_to_bf16x2(w.x, e);
      u4x8_to_bf16x2(w.y, h);
      out[2 * i] = make_uint4(e[0], e[1], e[2], e[3]);
      out[2 * i + 1] = make_uint4(h[0], h[1], h[2], h[3]);
    }
  }
}

constexpr int64_t kStreamMaxTokens = 16;

static int linear_bits(const mote_linear_t* L) { return L->bits == 0 ? MOTE_SHARED_BF16 : L->bits; }
static bool linear_shape_ok(const mote_linear_t* L) {
  const int bits = linear_bits(L);
  return (bits == MOTE_SHARED_BF16 || bits == MOTE_SHARED_INT8 || bits == MOTE_SHARED_INT4) && L->N >= 1 && L->N <= (1 << 24) && L->K >= 1 &&
         L->K <= 65536 && L->K % (bits == MOTE_SHARED_BF16 ? 8 : 16) == 0 && L->act >= MOTE_ACT_NONE && L->act <= MOTE_ACT_GELU_TANH;
}
static bool ranges_overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t pa = reinterpret_cast<uintptr_t>(a), pb = reinterpret_cast<uintptr_t>(b);
  return a && b && pa < pb + nb && pb < pa + na;
}

}  // namespace mote

extern "C" size_t mote_linear_workspace_bytes(const mote_linear_t* L, int64_t T_max) {
  using namespace mote;
  if (!L || !linear_shape_ok(L) || T_max < 0 || T_max > (int64_t(1) << 24)) return 0;
  // status word; from kStreamMaxTokens on the codes as bf16
  const bool expands = linear_bits(L) != MOTE_SHARED_BF16 && T_max > kStreamMaxTokens;
  return 256 + (expands ? round_up(size_t(L->N) * L->K * 2, 256) : 0);
}

extern "C" mote_status_t mote_linear(const mote_linear_t* L, const void* x, int64_t ldx, int64_t T, const void* residual, int64_t ldr,
                                     void* out, int out_dtype, void* ws, size_t ws_bytes, void* stream_) {
  using namespace mote;
  if (!L) return MOTE_ERR_NULL;
  if (!linear_shape_ok(L) || T < 0 || T > (int64_t(1) << 24)) return MOTE_ERR_SHAPE;
  if (out_dtype != MOTE_DTYPE_F32 && out_dtype != MOTE_DTYPE_BF16) return MOTE_ERR_DTYPE;
  if (T == 0) return MOTE_OK;
  const int bits = linear_bits(L);
  if (!x || !out || !ws || !L->W || (bits != MOTE_SHARED_BF16 && !L->w_scale)) return MOTE_ERR_NULL;
  if (T > 1 && (ldx < L->K || (residual && ldr < L->N))) return MOTE_ERR_SHAPE;
  const void* ptrs[] = {x, L->W, residual, out, L->bias, L->w_scale};
  for (const void* p : ptrs)
    if (p && !aligned16(p)) return MOTE_ERR_ALIGN;
  if ((T > 1 && ldx % 8 != 0) || (reinterpret_cast<uintptr_t>(ws) & 255u) != 0) return MOTE_ERR_ALIGN;
  if (ws_bytes < mote_linear_workspace_bytes(L, T)) return MOTE_ERR_WORKSPACE;
  const int64_t sx = T > 1 ? ldx : L->K, sr = T > 1 ? ldr : L->N;
  const size_t out_bytes = size_t(T) * L->N * (out_dtype == MOTE_DTYPE_F32 ? 4 : 2);
  // the output may take the residual's place element by element; x is read by every tile
  if (ranges_overlap(out, out_bytes, x, size_t((T - 1) * sx + L->K) * 2)) return MOTE_ERR_SHAPE;
  if (ranges_overlap(out, out_bytes, residual, size_t((T - 1) * sr + L->N) * 2) &&
      !(out == residual && out_dtype == MOTE_DTYPE_BF16 && sr == L->N))
    return MOTE_ERR_SHAPE;
  LinearArgs a{};
  a.x = static_cast<const uint16_t*>(x); a.ldx = sx; a.T = T; a.W = L->W; a.w_scale = L->w_scale; a.bias = L->bias;
  a.res = static_cast<const uint16_t*>(residual); a.ldr = sr; a.out = out; a.N = L->N; a.K = (int)L->K; a.act = L->act;
  a.out_f32 = out_dtype == MOTE_DTYPE_F32; a.status = static_cast<uint32_t*>(ws);
  cudaStream_t stream = static_cast<cudaStream_t>(stream_);
  if (T <= kStreamMaxTokens) {
    MOTE_CUDA_OK(T <= 8 ? launch_stream<1>(a, bits, stream) : launch_stream<2>(a, bits, stream));
    MOTE_LAUNCH_OK();
    return MOTE_OK;
  }
  if (bits == MOTE_SHARED_BF16) {
    a.w_scale = nullptr;
  } else {
    void* expanded = static_cast<char*>(ws) + 256;
    const int64_t n_chunks = L->N * L->K * bits / 64;
    const unsigned grid = (unsigned)std::min<int64_t>((n_chunks + 255) / 256, int64_t(device_sm_count()) * 8);
    MOTE_CUDA_OK(launch_pdl(linear_expand_kernel, dim3(grid), dim3(256), 0, stream, static_cast<const uint2*>(L->W),
                            static_cast<uint4*>(expanded), n_chunks, bits));
    a.W = expanded;
  }
  return launch_linear_umma(a, stream);
}
