// Tensor-core product of mote_linear: out = act( w_scale * (x W^T) + bias ) + residual, tcgen05.mma kind::f16 with TMEM accumulators,
// operands staged in shared memory by TMA.
//
// Tile: 128 tokens (one TMEM lane each; 256 for a pair of CTAs) x bn rows of W (bn a multiple of 16, of 32 for a pair, up to 256); K
// advances 64 elements, 128 bytes of either operand, per pipeline stage, four K = 16 MMAs each.  What lies beyond the tensors is zero
// (TMA fill) and is not stored.
//
// Warp roles: 0 TMA producer, 1 MMA issuer, 2 TMEM owner, 4 to 11 epilogue (two per TMEM lane quarter, which share the tile's columns).
// Three forms:
//   pairs of CTAs (CG = 2)   cta_group::2 MMAs read half of the weight rows from either CTA: a tile of 256 x 256 fetches 32 KB a stage and
//                            SM, two thirds of what two tiles of 128 x 256 do
//   single CTAs (CG = 1)     persistent as the pairs are: two accumulators in TMEM let a tile's epilogue run under the next one's MMAs
//   split along K (kSplit)   a cluster of CTAs shares one tile's K where the tiles are too few for the SMs; the partial sums meet in
//                            distributed shared memory, are added in rank order, and each CTA finishes its share of the columns
//
// Every mbarrier wait is bounded; on expiry the CTA raises the status word and leaves.
#include <cuda.h>

#include <algorithm>
#include <mutex>

#include "linear_act.cuh"
#include "ptx_sm100.cuh"

namespace mote {

using namespace ptx;

constexpr int kLinThreads = 384;
constexpr int kLinEpiFirst = 4, kLinEpiWarps = 8;
constexpr int kLinStageA = 128 * 128;            // 128 rows x 128 bytes
constexpr int kLinMaxStages = 8;
constexpr int kLinPipeBytes = 192 * 1024;
constexpr int kLinPitch = 17;                    // floats per row of an epilogue warp's staging block
constexpr int kLinStaging = kLinEpiWarps * 32 * kLinPitch * 4;

struct LinearTiles {
  int bn, stages, k_steps, splits;
  int n_mt, n_nt;
  int rows_fast;                                 // items: weight tiles (0) or token tiles (1) change fastest
  int a_rows;                                    // rows of the token operand's box
  int vec8, wide;                                // rows of out (and residual) on 16-byte boundaries; out on 32-byte ones
};

struct __align__(8) LinearBarriers {
  uint64_t full[kLinMaxStages], empty[kLinMaxStages], tmem_full[2], tmem_empty[2];
  uint32_t tmem_base;
  int abort_flag;
};
constexpr int kLinSmem = 1024 + kLinPipeBytes + kLinStaging + (int)sizeof(LinearBarriers);

__device__ __forceinline__ void linear_item(const LinearTiles& t, int item, int& mt, int& nt) {
  if (t.rows_fast) { mt = item % t.n_mt; nt = item / t.n_mt; }
  else { nt = item % t.n_nt; mt = item / t.n_nt; }
}

// Finishes 16 neighbouring columns of a warp's 32 rows (lane = row): scale, bias, activation, residual, one rounding.
__device__ __forceinline__ void finish_columns(const LinearArgs& a, const LinearTiles& t, float (&z)[16], int64_t row0, int64_t col, float* stg,
                                               int lane) {
  if (a.w_scale || a.bias) {
    if (col + 16 <= a.N) {                       // col is a multiple of 16, so these vectors are aligned
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        if (a.w_scale) {
          const float4 s = __ldg(reinterpret_cast<const float4*>(a.w_scale + col) + v);
          z[4 * v] *= s.x; z[4 * v + 1] *= s.y; z[4 * v + 2] *= s.z; z[4 * v + 3] *= s.w;
        }
        if (a.bias) {
          const float4 b = __ldg(reinterpret_cast<const float4*>(a.bias + col) + v);
          z[4 * v] += b.x; z[4 * v + 1] += b.y; z[4 * v + 2] += b.z; z[4 * v + 3] += b.w;
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < 16; ++j)
        if (col + j < a.N) {
          if (a.w_scale) z[j] *= __ldg(a.w_scale + col + j);
          if (a.bias) z[j] += __ldg(a.bias + col + j);
        }
    }
  }
  if (a.act != MOTE_ACT_NONE) {
#pragma unroll
    for (int j = 0; j < 16; ++j) z[j] = apply_act(z[j], a.act);
  }
  const int64_t row = row0 + lane;
  if (t.vec8) {                                  // N is a multiple of 8: each half of the 16 columns is inside or outside as a whole
    if (row >= a.T || col >= a.N) return;
    const bool both = col + 16 <= a.N;
    if (a.res) {
      const uint4* rp = reinterpret_cast<const uint4*>(a.res + row * a.ldr + col);
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if (h == 0 || both) {
          const uint4 r = rp[h];
          const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) { z[8 * h + 2 * j] += bf16_lo(w[j]); z[8 * h + 2 * j + 1] += bf16_hi(w[j]); }
        }
    }
    if (a.out_f32) {
      float* o = static_cast<float*>(a.out) + row * a.N + col;
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if (h == 0 || both) {
          if (t.wide) {
            st_global_v8(o + 8 * h, __float_as_uint(z[8 * h]), __float_as_uint(z[8 * h + 1]), __float_as_uint(z[8 * h + 2]), __float_as_uint(z[8 * h + 3]),
                         __float_as_uint(z[8 * h + 4]), __float_as_uint(z[8 * h + 5]), __float_as_uint(z[8 * h + 6]), __float_as_uint(z[8 * h + 7]));
          } else {
            reinterpret_cast<float4*>(o + 8 * h)[0] = make_float4(z[8 * h], z[8 * h + 1], z[8 * h + 2], z[8 * h + 3]);
            reinterpret_cast<float4*>(o + 8 * h)[1] = make_float4(z[8 * h + 4], z[8 * h + 5], z[8 * h + 6], z[8 * h + 7]);
          }
        }
    } else {
      uint16_t* o = static_cast<uint16_t*>(a.out) + row * a.N + col;
      uint32_t p[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) p[j] = pack_bf16x2(z[2 * j], z[2 * j + 1]);
      if (t.wide && both) st_global_v8(o, p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7]);
      else {
        reinterpret_cast<uint4*>(o)[0] = make_uint4(p[0], p[1], p[2], p[3]);
        if (both) reinterpret_cast<uint4*>(o)[1] = make_uint4(p[4], p[5], p[6], p[7]);
      }
    }
    return;
  }
  // rows on any boundary: through shared memory, so that 16 lanes write 16 neighbouring elements of a row
  __syncwarp();
#pragma unroll
  for (int j = 0; j < 16; ++j) stg[lane * kLinPitch + j] = z[j];
  __syncwarp();
  const int64_t c = col + (lane & 15);
#pragma unroll 4
  for (int r = lane >> 4; r < 32; r += 2) {
    if (row0 + r >= a.T || c >= a.N) continue;
    float v = stg[r * kLinPitch + (lane & 15)];
    if (a.res) v += __uint_as_float(uint32_t(a.res[(row0 + r) * a.ldr + c]) << 16);
    if (a.out_f32) static_cast<float*>(a.out)[(row0 + r) * a.N + c] = v;
    else static_cast<uint16_t*>(a.out)[(row0 + r) * a.N + c] = (uint16_t)(pack_bf16x2(v, 0.0f) & 0xFFFFu);
  }
}

struct Ring {
  uint32_t stage = 0, phase = 0;
  __device__ __forceinline__ void next(uint32_t n) {
    if (++stage == n) { stage = 0; phase ^= 1; }
  }
};

template <int CG, bool kSplit>
__global__ void __launch_bounds__(kLinThreads, 1)
linear_umma_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_b, const LinearArgs a, const LinearTiles t) {
  static_assert(CG == 1 || !kSplit, "K is split over single CTAs");
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem_gen = smem_raw + (smem_base - smem_u32(smem_raw));
  const uint32_t stage_b = uint32_t(t.bn / CG) * 128;
  const uint32_t stage_bytes = kLinStageA + stage_b;
  float* staging = reinterpret_cast<float*>(smem_gen + kLinPipeBytes);
  LinearBarriers* bars = reinterpret_cast<LinearBarriers*>(smem_gen + kLinPipeBytes + kLinStaging);
  volatile int* abort_flag = &bars->abort_flag;
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const uint32_t rank = (CG == 2 || kSplit) ? cluster_ctarank() : 0;
  const int per = kSplit ? t.splits : CG;          // CTAs that work on one item
  const int worker = blockIdx.x / per, workers = gridDim.x / per;
  const int n_items = t.n_mt * t.n_nt;
  const int S = t.stages;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kLinMaxStages; ++s) { mbar_init(smem_u32(&bars->full[s]), 1); mbar_init(smem_u32(&bars->empty[s]), 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(smem_u32(&bars->tmem_full[b]), 1); mbar_init(smem_u32(&bars->tmem_empty[b]), kLinEpiWarps * CG); }
    bars->abort_flag = 0;
    fence_barrier_init();
    prefetch_tensormap(&tm_a);
    prefetch_tensormap(&tm_b);
  }
  if (warp == 2) {
    tmem_alloc<CG>(smem_u32(&bars->tmem_base), 512);
    tmem_relinquish<CG>();
  }
  tc_fence_before();
  __syncthreads();
  if (CG == 2) cluster_sync();                     // the other CTA's barriers are initialised
  tc_fence_after();
  const uint32_t tmem_base = __shfl_sync(0xffffffffu, bars->tmem_base, 0);
  pdl_wait();
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.status = 0u;
  // this CTA's steps along K
  const int kb = kSplit ? t.k_steps * (int)rank / t.splits : 0, ke = kSplit ? t.k_steps * ((int)rank + 1) / t.splits : t.k_steps;

  if (warp == 0) {
    if (lane == 0) {
      Ring p;
      bool ok = true;
      for (int item = worker; ok && item < n_items; item += workers) {
        int mt, nt;
        linear_item(t, item, mt, nt);
        const int a_row = (mt * CG + (CG == 2 ? (int)rank : 0)) * 128;
        const int b_row = nt * t.bn + (CG == 2 ? (int)rank * (t.bn / 2) : 0);
        for (int ks = kb; ks < ke; ++ks) {
          if (!mbar_wait(smem_u32(&bars->empty[p.stage]), p.phase ^ 1, abort_flag)) { ok = false; break; }
          uint32_t bar = smem_u32(&bars->full[p.stage]);
          if (CG == 1 || rank == 0) mbar_expect_tx(bar, CG * (uint32_t(t.a_rows) * 128 + stage_b));
          const uint32_t dst = smem_base + p.stage * stage_bytes;
          if (CG == 2) {
            bar = map_to_rank(bar, 0);
            tma_load_2d_pair(dst, &tm_a, ks * 64, a_row, bar);
            tma_load_2d_pair(dst + kLinStageA, &tm_b, ks * 64, b_row, bar);
          } else {
            tma_load_2d(dst, &tm_a, ks * 64, a_row, bar);
            tma_load_2d(dst + kLinStageA, &tm_b, ks * 64, b_row, bar);
          }
          p.next(S);
        }
      }
      // the commits of the last steps have arrived at this CTA's barriers before it may leave
      for (int i = 0; ok && i < S; ++i) {
        ok = mbar_wait(smem_u32(&bars->empty[p.stage]), p.phase ^ 1, abort_flag);
        p.next(S);
      }
    }
  } else if (warp == 1) {
    if (CG == 1 || rank == 0) {
      Ring p;
      const uint32_t idesc = make_idesc(1, 1, 1, 128 * CG, (uint32_t)t.bn);
      int local = 0;
      bool ok = true;
      for (int item = worker; ok && item < n_items; item += workers, ++local) {
        const int buf = local & 1;
        if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&bars->tmem_empty[buf]), ((local >> 1) & 1) ^ 1, abort_flag))) break;
        tc_fence_after();
        uint32_t acc = 0;
        for (int ks = kb; ks < ke; ++ks) {
          if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&bars->full[p.stage]), p.phase, abort_flag))) { ok = false; break; }
          tc_fence_after();
          const uint64_t da = smem_desc_sw128(smem_base + p.stage * stage_bytes);
          const uint64_t db = smem_desc_sw128(smem_base + p.stage * stage_bytes + kLinStageA);
          if (elect_one()) {
#pragma unroll
            for (int j = 0; j < 4; ++j) mma_f16<CG>(tmem_base + buf * 256, da + 2 * j, db + 2 * j, idesc, j > 0 ? 1u : acc);
            mma_commit<CG>(smem_u32(&bars->empty[p.stage]));
          }
          __syncwarp();
          acc = 1;
          p.next(S);
        }
        if (!ok) break;
        if (elect_one()) mma_commit<CG>(smem_u32(&bars->tmem_full[buf]));
        __syncwarp();
      }
    }
  } else if (warp >= kLinEpiFirst && !kSplit) {
    const int q = warp & 3, part = (warp - kLinEpiFirst) >> 2;
    float* stg = staging + (warp - kLinEpiFirst) * 32 * kLinPitch;
    int local = 0;
    for (int item = worker; item < n_items; item += workers, ++local) {
      int mt, nt;
      linear_item(t, item, mt, nt);
      const int buf = local & 1;
      if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&bars->tmem_full[buf]), (local >> 1) & 1, abort_flag))) break;
      tc_fence_after();
      const uint32_t t_row = tmem_base + (uint32_t(q * 32) << 16) + buf * 256;
      const int64_t row0 = int64_t(mt * CG + (CG == 2 ? (int)rank : 0)) * 128 + q * 32;
#pragma unroll 1
      for (int c = part * 16; c < t.bn; c += 32) {
        const int64_t col = int64_t(nt) * t.bn + c;
        if (row0 >= a.T || col >= a.N) continue;   // whole warp
        uint32_t r[16];
        tmem_ld_32x32b_x16(t_row + c, r);
        tmem_wait_ld();
        float z[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) z[j] = __uint_as_float(r[j]);
        finish_columns(a, t, z, row0, col, stg, lane);
        __syncwarp();
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if (CG == 2) mbar_arrive_cluster(map_to_rank(smem_u32(&bars->tmem_empty[buf]), 0));
        else mbar_arrive(smem_u32(&bars->tmem_empty[buf]));
      }
    }
  } else if (warp >= kLinEpiFirst) {
    // this CTA's partial sums: column-major, over the pipeline's stages, which its own MMAs have left
    const int q = warp & 3, part = (warp - kLinEpiFirst) >> 2;
    if (__all_sync(0xffffffffu, mbar_wait(smem_u32(&bars->tmem_full[0]), 0, abort_flag))) {
      tc_fence_after();
      float* sums = reinterpret_cast<float*>(smem_gen);
#pragma unroll 1
      for (int c = part * 16; c < t.bn; c += 32) {
        uint32_t r[16];
        tmem_ld_32x32b_x16(tmem_base + (uint32_t(q * 32) << 16) + c, r);
        tmem_wait_ld();
#pragma unroll
        for (int j = 0; j < 16; ++j) sums[(c + j) * 128 + q * 32 + lane] = __uint_as_float(r[j]);
      }
    }
  }

  if (kSplit) {
    tc_fence_before();
    cluster_sync();
    if (warp >= kLinEpiFirst) {
      const int q = warp & 3, part = (warp - kLinEpiFirst) >> 2;
      float* stg = staging + (warp - kLinEpiFirst) * 32 * kLinPitch;
      int mt, nt;
      linear_item(t, worker, mt, nt);
      const int64_t row0 = int64_t(mt) * 128 + q * 32;
      const int w = t.bn / t.splits;               // columns this CTA finishes, a multiple of 16
#pragma unroll 1
      for (int c = (int)rank * w + part * 16; c < ((int)rank + 1) * w; c += 32) {
        const int64_t col = int64_t(nt) * t.bn + c;
        if (row0 >= a.T || col >= a.N) continue;
        float z[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) z[j] = 0.0f;
        for (int s = 0; s < t.splits; ++s) {
          const uint32_t src = map_to_rank(smem_base + uint32_t(c * 128 + q * 32 + lane) * 4, s);
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            float v;
            asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(src + j * 512) : "memory");
            z[j] += v;
          }
        }
        finish_columns(a, t, z, row0, col, stg, lane);
        __syncwarp();
      }
    }
  }

  // after a wait that ran out: time for copies and MMAs in flight to land before shared memory and TMEM go away
  if (*abort_flag) {
    const uint64_t t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 200000ull) __nanosleep(1000);
  }
  tc_fence_before();
  __syncthreads();
  if (CG == 2 || kSplit) cluster_sync();           // neither CTA's shared memory and TMEM go while another still works with them
  if (warp == 2) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc<CG>(tmem_base, 512);
  }
  if (threadIdx.x == 0 && *abort_flag) atomicExch(a.status, 1u);
  if (CG == 2) cluster_sync();
}

// ------------------------------------------------------------------------------------------------
// Host side
// ------------------------------------------------------------------------------------------------
using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                              const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// bf16 [rows, cols] with a row stride in elements; box [box_rows, 64], 128-byte swizzle
static bool make_operand_map(CUtensorMap* m, const void* base, int64_t rows, int64_t cols, int64_t stride, int box_rows) {
  static EncodeFn fn = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<EncodeFn>(p);
  });
  if (!fn) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)stride * 2};
  const cuuint32_t box[2] = {64, (cuuint32_t)box_rows};
  const cuuint32_t estr[2] = {1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Which form and tile width: the least estimated time, in cycles.
struct LinearForm { int cg, bn, splits; };
static LinearForm pick_form(int64_t T, int64_t N, int k_steps, int sms) {
  LinearForm best{1, 256, 1};
  double best_cost = 1e300;
  auto consider = [&](int cg, int bn, int splits) {
    const int64_t items = ((T + 128 * cg - 1) / (128 * cg)) * ((N + bn - 1) / bn);
    const int64_t workers = std::max(1, sms / (cg * splits));
    const int64_t rounds = (items + workers - 1) / workers;
    const double active = double(std::min(items, workers)) * cg * splits;
    // a step: four MMAs, or the way of its operands from L2 (some 6 KB a cycle for all SMs, 64 bytes for one)
    const double rows = std::min<int64_t>(T, 128);
    const double bytes = rows * 128 + double(bn / cg) * 128;
    const double step = std::max({2.0 * std::max(bn, 64), bytes / 64.0, bytes * active / 6000.0});
    const int steps = (k_steps + splits - 1) / splits;
    const double epilogue = 6.0 * bn / splits + (splits > 1 ? 1500.0 + 4.0 * bn : 0.0);
    const double cost = double(rounds) * steps * step + epilogue + (rounds > 1 ? 200.0 * rounds : 0.0);
    if (cost < best_cost) { best_cost = cost; best = {cg, bn, splits}; }
  };
  const int bn_max = (int)std::min<int64_t>(256, (N + 15) / 16 * 16);
  for (int bn = bn_max; bn >= 16; bn -= 16) consider(1, bn, 1);
  if (T > 128)
    for (int bn = 256; bn >= 64; bn -= 32)
      if (bn - 32 < N) consider(2, bn, 1);
  for (int splits = 2; splits <= 8; splits *= 2)
    for (int bn = 16 * splits; bn <= 256; bn += 16 * splits)
      if (k_steps >= 2 * splits && bn - 16 * splits < N) consider(1, bn, splits);
  return best;
}

template <int CG, bool kSplit>
static cudaError_t launch_form(const CUtensorMap& ta, const CUtensorMap& tb, const LinearArgs& a, const LinearTiles& t, int grid, int cluster,
                               cudaStream_t stream) {
  static PerDeviceOnce once;
  const cudaError_t e = set_max_dynamic_smem(once, linear_umma_kernel<CG, kSplit>, kLinSmem);
  if (e != cudaSuccess) return e;
  return launch_ex(linear_umma_kernel<CG, kSplit>, dim3(grid), dim3(kLinThreads), kLinSmem, stream, true, cluster, ta, tb, a, t);
}

mote_status_t launch_linear_umma(const LinearArgs& a, cudaStream_t stream) {
  const int sms = device_sm_count();
  LinearTiles t{};
  t.k_steps = (a.K + 63) / 64;
  const LinearForm f = pick_form(a.T, a.N, t.k_steps, sms);
  t.bn = f.bn; t.splits = f.splits;
  t.n_mt = (int)((a.T + 128 * f.cg - 1) / (128 * f.cg));
  t.n_nt = (int)((a.N + f.bn - 1) / f.bn);
  if (int64_t(t.n_mt) * t.n_nt > (1ll << 28)) return MOTE_ERR_SHAPE;
  // the smaller operand's tiles change fastest: its whole stays in L2, the larger one is read from HBM once
  t.rows_fast = a.T <= a.N;
  t.a_rows = f.cg == 1 ? (int)std::min<int64_t>(128, (a.T + 7) / 8 * 8) : 128;
  t.stages = std::min(kLinMaxStages, kLinPipeBytes / (kLinStageA + f.bn / f.cg * 128));
  t.vec8 = a.N % 8 == 0 && (!a.res || a.ldr % 8 == 0);
  t.wide = a.N % 16 == 0 && (reinterpret_cast<uintptr_t>(a.out) & 31u) == 0;
  CUtensorMap ta, tb;
  if (!make_operand_map(&ta, a.x, a.T, a.K, a.ldx, t.a_rows) || !make_operand_map(&tb, a.W, a.N, a.K, a.K, f.bn / f.cg)) return MOTE_ERR_CUDA;
  const int items = t.n_mt * t.n_nt;
  const cudaError_t e = f.splits > 1 ? launch_form<1, true>(ta, tb, a, t, items * f.splits, f.splits, stream)
                        : f.cg == 2  ? launch_form<2, false>(ta, tb, a, t, 2 * std::min(items, sms / 2), 2, stream)
                                     : launch_form<1, false>(ta, tb, a, t, std::min(items, sms), 1, stream);
  if (e != cudaSuccess) return MOTE_ERR_CUDA;
  MOTE_LAUNCH_OK();
  return MOTE_OK;
}

}  // namespace mote
