// Matrix product with bias, activation and residual in its epilogue (mote_linear):
//
//   out = act( scale_n * (x W^T) + bias ) [+ residual]
//
// W [N, K] is bf16, or the RTN codes of mote_rtn_quant (INT8 / INT4) with one scale per row; fp32 accumulation, one rounding
// to the output's type.  The whole of K (a warp's or a cluster rank's part of it) is left to the tensor cores' accumulators, which cut off what
// lies 25 bits below the largest addend: 3e-6 of a sum of one sign at K = 11008 (mote.h), below a thousandth of a bf16 output's rounding.
// (The router, whose choice hangs on the last bits, takes its sums out every few steps.)
//
// For few tokens the product is a weight stream, bound by HBM and, at these sizes, by how much is in flight: a CTA owns 16 rows
// of W, its warps share K, and asynchronous copies bring weights and tokens to rings in shared memory, from where they feed warp-level
// MMAs, the weights (codes are expanded in registers) as the A operand, the tokens as the 8-wide B operand.  Every weight byte is read once.
// us from a cold L2 (GB/s of weights): 1 x 2048 x 11008 bf16 9.4 (4800), 1 x 11008 x 2048 bf16 10.0 (4530), 8 x 2048 x 11008 INT8 8.7 (2630);
// with loads into registers, four steps ahead, 24 / 12 / 14: they came to one latency a step.
#include <algorithm>

#include "linear_act.cuh"

namespace mote {

// kBytes from global into shared memory, behind the thread's back.
template <int kBytes>
__device__ __forceinline__ void cp_async(uint32_t dst, const void* src) {
  if (kBytes == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

constexpr int kStreamRows = 16;

// What a warp has in flight: a ring of steps in shared memory, filled by asynchronous copies of its own lanes.  A step's units of 16 bytes
// per lane: the weights of rows g and g + 8 (INT4: 8 bytes of each in one unit), and the tokens of each column tile, one unit with bf16
// weights, two with codes, which have twice as many elements to a step.
template <int NT, int kBits, int kWarps>
struct StreamRing {
  static constexpr int kXUnits = kBits == 16 ? 1 : 2;
  static constexpr int kWUnits = kBits == 4 ? 1 : 2;
  static constexpr int kUnits = kWUnits + NT * kXUnits;
  static constexpr int kDepth = kUnits <= 3 ? 8 : kUnits <= 4 ? 6 : 4;     // 8 warps: 96 KB or less, two CTAs per SM
  static constexpr int kBytes = kWarps * kDepth * kUnits * 32 * 16;
};

// kBits: storage of W.  A step covers 32 (bf16), 64 (INT8) or 64 (INT4, 32 code bytes) elements of K: lane (g, t) = (lane / 4, lane % 4)
// takes elements [step * kStep + t * kLane, + kLane) of weight rows g and g + 8 and of its token column; the reduction index may be
// permuted as long as both operands are.  The CTA walks over its row tiles, and the ring runs on from one to the next.
template <int NT, int kBits, int kWarps>
__global__ void __launch_bounds__(kWarps * 32, 16 / kWarps) linear_stream_kernel(LinearArgs a, int n_tiles) {
  using R = StreamRing<NT, kBits, kWarps>;
  constexpr int kLane = kBits == 16 ? 8 : 16, kStep = 4 * kLane;
  const int64_t t0 = int64_t(blockIdx.y) * (NT * 8);             // this CTA's tokens
  a.T -= t0;
  a.x += t0 * a.ldx;
  if (a.res) a.res += t0 * a.ldr;
  a.out = static_cast<char*>(a.out) + t0 * a.N * (a.out_f32 ? 4 : 2);
  extern __shared__ __align__(16) uint8_t s_dyn[];
  __shared__ float s_part[2][kWarps][NT * 4][32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int n_steps = (a.K + kStep - 1) / kStep;
  const int sb = n_steps * warp / kWarps, n = n_steps * (warp + 1) / kWarps - sb;      // this warp's steps
  const int64_t row_bytes = int64_t(a.K) * kBits / 8;
  const uint8_t* w0 = static_cast<const uint8_t*>(a.W) + (sb * kStep + t * kLane) * kBits / 8;
  // With two units a step, a copy takes the four neighbouring units u * 4 + t of a token's eight, 64 bytes in a row (as each lane's own two
  // they would be every other 16 bytes, twice the traffic: 8 x 2048 x 11008, INT8: 13.5 us).  Unit c of token g is kept at c ^ (g & 1), where
  // neither copies nor reads have bank conflicts.
  const uint16_t* tok[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) tok[j] = j * 8 + g < a.T ? a.x + (j * 8 + g) * a.ldx + sb * kStep + t * 8 : nullptr;
  auto x_unit = [&](int j, int c) {              // where unit c of the lane's token is, in units of 16 bytes from the place's start
    return (R::kWUnits + j * R::kXUnits) * 32 + (R::kXUnits == 1 ? g * 4 + c : g * 8 + (c ^ (g & 1)));
  };
  const int warp_base = warp * (R::kDepth * R::kUnits * 32);
  const uint4* ring = reinterpret_cast<const uint4*>(s_dyn) + warp_base;
  const uint32_t ring_addr = (uint32_t)__cvta_generic_to_shared(s_dyn) + warp_base * 16;
  pdl_wait();
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *a.status = 0u;

  // the step that is fetched next: its tile, its number in the warp's share, its place, its rows
  int f_tile = n > 0 ? (int)blockIdx.x : n_tiles, f_step = 0, f_place = 0;
  const uint8_t *fa = nullptr, *fb = nullptr;
  auto fetch = [&]() {
    if (f_tile < n_tiles) {
      if (f_step == 0) {
        const int64_t row = int64_t(f_tile) * kStreamRows + g;
        fa = w0 + min(row, a.N - 1) * row_bytes;
        fb = w0 + min(row + 8, a.N - 1) * row_bytes;
      }
      const uint32_t dst = ring_addr + f_place * (R::kUnits * 512);
      const int k0 = (sb + f_step) * kStep;
      if (k0 + t * kLane < a.K) {
        if (kBits == 4) {
          cp_async<8>(dst + lane * 16, fa);
          cp_async<8>(dst + lane * 16 + 8, fb);
        } else {
          cp_async<16>(dst + lane * 16, fa);
          cp_async<16>(dst + lane * 16 + 512, fb);
        }
      }
#pragma unroll
      for (int j = 0; j < NT; ++j)
        if (tok[j])
#pragma unroll
          for (int u = 0; u < R::kXUnits; ++u)
            if (k0 + (u * 4 + t) * 8 < a.K) cp_async<16>(dst + x_unit(j, u * 4 + t) * 16, tok[j] + f_step * kStep + u * 32);
      fa += kStep * kBits / 8;
      fb += kStep * kBits / 8;
      if (++f_step == n) { f_step = 0; f_tile += gridDim.x; }
      f_place = f_place + 1 == R::kDepth ? 0 : f_place + 1;
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int i = 0; i < R::kDepth - 1; ++i) fetch();
  // The output that this thread finishes: rows fastest, so that a token's 16 outputs leave together.  Value i of token tile j at lane
  // (g, t) is weight row g + 8 * (i / 2), token 8j + 2t + (i & 1).
  const int row = threadIdx.x & 15, token = threadIdx.x >> 4;
  const bool mine = token < NT * 8 && token < a.T;
  const int v = ((token >> 3) % NT) * 4 + (row >> 3) * 2 + (token & 1), l = (row & 7) * 4 + ((token & 7) >> 1);
  static_assert(kWarps * 32 >= NT * 8 * kStreamRows, "an output per thread");
  int place = 0, buf = 0;
  for (int tile = blockIdx.x; tile < n_tiles; tile += gridDim.x, buf ^= 1) {
    const int64_t nn = int64_t(tile) * kStreamRows + row;
    float scale = 1.0f, bias = 0.0f, res = 0.0f;   // on their way while the products are formed
    if (mine && nn < a.N) {
      if (kBits != 16) scale = a.w_scale[nn];
      if (a.bias) bias = a.bias[nn];
      if (a.res) res = __uint_as_float(uint32_t(a.res[token * a.ldr + nn]) << 16);
    }
    float acc[NT][4];
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.0f;
    for (int s = 0; s < n; ++s) {
      __syncwarp();                              // all lanes have read the place that is filled now
      fetch();
      asm volatile("cp.async.wait_group %0;" ::"n"(R::kDepth - 1) : "memory");
      __syncwarp();                              // and all lanes' copies of this step have landed
      const uint4* at = ring + place * (R::kUnits * 32);
      place = place + 1 == R::kDepth ? 0 : place + 1;
      const bool in = (sb + s) * kStep + t * kLane < a.K;                  // places that no copy filled hold anything
      const uint4 kZero = make_uint4(0u, 0u, 0u, 0u);
      const uint4 ca = in ? at[lane] : kZero, cb = in && R::kWUnits > 1 ? at[lane + 32] : kZero;
      uint32_t ea[8], eb[8];
      if (kBits == 8) {
        const uint32_t pa[4] = {ca.x, ca.y, ca.z, ca.w}, pb[4] = {cb.x, cb.y, cb.z, cb.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          s8x4_to_bf16x2(pa[j], ea[2 * j], ea[2 * j + 1]);
          s8x4_to_bf16x2(pb[j], eb[2 * j], eb[2 * j + 1]);
        }
      } else if (kBits == 4) {
        const uint32_t p[4] = {ca.x, ca.y, ca.z, ca.w};                    // two words of row g, two of row g + 8
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          uint32_t h[4];
          u4x8_to_bf16x2(p[j], h);
          ea[4 * j] = h[0]; ea[4 * j + 1] = h[1]; ea[4 * j + 2] = h[2]; ea[4 * j + 3] = h[3];
          u4x8_to_bf16x2(p[2 + j], h);
          eb[4 * j] = h[0]; eb[4 * j + 1] = h[1]; eb[4 * j + 2] = h[2]; eb[4 * j + 3] = h[3];
        }
      }
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const bool live = in && tok[j];
        const uint4 x0 = live ? at[x_unit(j, R::kXUnits * t)] : kZero;
        if (kBits == 16) {
          mma_16816(acc[j], ca.x, cb.x, ca.y, cb.y, x0.x, x0.y);
          mma_16816(acc[j], ca.z, cb.z, ca.w, cb.w, x0.z, x0.w);
        } else {
          const uint4 x1 = live ? at[x_unit(j, R::kXUnits * t + R::kXUnits - 1)] : kZero;
          const uint32_t xw[8] = {x0.x, x0.y, x0.z, x0.w, x1.x, x1.y, x1.z, x1.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) mma_16816(acc[j], ea[2 * i], eb[2 * i], ea[2 * i + 1], eb[2 * i + 1], xw[2 * i], xw[2 * i + 1]);
        }
      }
    }
    // the warps' sums meet; two buffers, so that one barrier a tile is enough
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) s_part[buf][warp][j * 4 + i][lane] = acc[j][i];
    __syncthreads();
    if (mine && nn < a.N) {
      float z = s_part[buf][0][v][l];
#pragma unroll
      for (int w = 1; w < kWarps; ++w) z += s_part[buf][w][v][l];
      if (kBits != 16) z *= scale;
      z = apply_act(z + bias, a.act) + res;
      if (a.out_f32) static_cast<float*>(a.out)[token * a.N + nn] = z;
      else static_cast<uint16_t*>(a.out)[token * a.N + nn] = (uint16_t)(pack_bf16x2(z, 0.0f) & 0xFFFFu);
    }
  }
}

template <int NT, int kBits, int kWarps>
static cudaError_t launch_stream_as(const LinearArgs& a, int tiles, cudaStream_t stream) {
  static PerDeviceOnce once;
  constexpr int smem = StreamRing<NT, kBits, kWarps>::kBytes;
  const cudaError_t e = set_max_dynamic_smem(once, linear_stream_kernel<NT, kBits, kWarps>, smem);
  if (e != cudaSuccess) return e;
  const int groups = (int)((a.T + NT * 8 - 1) / (NT * 8)), slots = std::max(1, device_sm_count() * (16 / kWarps) / groups);
  return launch_pdl(linear_stream_kernel<NT, kBits, kWarps>, dim3(std::min(tiles, slots), groups), dim3(kWarps * 32), smem, stream, a, tiles);
}
template <int NT, int kBits>
static cudaError_t launch_stream_bits(const LinearArgs& a, cudaStream_t stream) {
  // A tile per SM: sixteen warps share its K (1 x 2048 x 11008: 10.4 us with eight).  More tiles: two CTAs of eight warps per SM, whose sums and
  // barriers fall apart in time (16 x 8960 x 1536: 8.3 us, 9.5 with sixteen).
  const int tiles = (int)((a.N + kStreamRows - 1) / kStreamRows);
  const int groups = (int)((a.T + NT * 8 - 1) / (NT * 8));
  return tiles * groups <= device_sm_count() ? launch_stream_as<NT, kBits, 16>(a, tiles, stream) : launch_stream_as<NT, kBits, 8>(a, tiles, stream);
}
template <int NT>
static cudaError_t launch_stream(const LinearArgs& a, int bits, cudaStream_t stream) {
  return bits == 16 ? launch_stream_bits<NT, 16>(a, stream) : bits == 8 ? launch_stream_bits<NT, 8>(a, stream) : launch_stream_bits<NT, 4>(a, stream);
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

static int linear_bits(const mote_linear_t* L) { return L->bits == 0 ? MOTE_SHARED_BF16 : L->bits; }
static bool linear_shape_ok(const mote_linear_t* L) {
  const int bits = linear_bits(L);
  return (bits == MOTE_SHARED_BF16 || bits == MOTE_SHARED_INT8 || bits == MOTE_SHARED_INT4) && L->N >= 1 && L->N <= (1 << 24) && L->K >= 1 &&
         L->K <= 65536 && L->K % (bits == MOTE_SHARED_BF16 ? 8 : 16) == 0 && L->act >= MOTE_ACT_NONE && L->act <= MOTE_ACT_GELU_TANH;
}
// Up to 16 tokens go through the weight stream, two column tiles of them; more in groups of 16, whose weights come from the L2 after the first
// one, while that costs less than the tensor-core product's longer way.  Codes, which that product needs expanded: always for two groups
// (32 x 2048 x 11008, INT8: 17.7 us, expanded 22.2; 2048 x 2048: 5.1, 12.5), for three and four while the groups' products are few
// (64 x 2048 x 2048: 8.3, 12.9; 64 x 1536 x 8960: 22.5, 16.4).  bf16: two and three groups of few products (32 x 2048 x 2048: 5.5, 8.1;
// 48 x 2048 x 2048: 7.7, 8.5; 32 x 1536 x 8960: 12.9, 9.2).
static bool takes_stream(const mote_linear_t* L, int64_t T) {
  const int64_t groups = (T + 15) / 16, work = groups * L->N * L->K;
  if (linear_bits(L) == MOTE_SHARED_BF16) return groups <= 1 || (groups <= 3 && work <= 13000000);
  return groups <= 2 || (groups <= 4 && work <= 40000000);
}
static bool ranges_overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t pa = reinterpret_cast<uintptr_t>(a), pb = reinterpret_cast<uintptr_t>(b);
  return a && b && pa < pb + nb && pb < pa + na;
}

}  // namespace mote

extern "C" size_t mote_linear_workspace_bytes(const mote_linear_t* L, int64_t T_max) {
  using namespace mote;
  if (!L || !linear_shape_ok(L) || T_max < 0 || T_max > (int64_t(1) << 24)) return 0;
  // status word; where the tensor-core product takes over, the codes as bf16
  const bool expands = linear_bits(L) != MOTE_SHARED_BF16 && !takes_stream(L, T_max);
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
  // the output may take the residual's place element by element; x, the weights and the workspace are read by every tile
  const void* const read[] = {x, L->W, bits == MOTE_SHARED_BF16 ? nullptr : L->w_scale, L->bias, ws};
  const size_t read_bytes[] = {size_t((T - 1) * sx + L->K) * 2, size_t(L->N) * L->K * bits / 8, size_t(L->N) * 4, size_t(L->N) * 4,
                               mote_linear_workspace_bytes(L, T)};
  for (int i = 0; i < 5; ++i)
    if (ranges_overlap(out, out_bytes, read[i], read_bytes[i])) return MOTE_ERR_SHAPE;
  if (ranges_overlap(out, out_bytes, residual, size_t((T - 1) * sr + L->N) * 2) &&
      !(out == residual && out_dtype == MOTE_DTYPE_BF16 && sr == L->N))
    return MOTE_ERR_SHAPE;
  LinearArgs a{};
  a.x = static_cast<const uint16_t*>(x); a.ldx = sx; a.T = T; a.W = L->W; a.w_scale = L->w_scale; a.bias = L->bias;
  a.res = static_cast<const uint16_t*>(residual); a.ldr = sr; a.out = out; a.N = L->N; a.K = (int)L->K; a.act = L->act;
  a.out_f32 = out_dtype == MOTE_DTYPE_F32; a.status = static_cast<uint32_t*>(ws);
  cudaStream_t stream = static_cast<cudaStream_t>(stream_);
  if (takes_stream(L, T)) {
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
