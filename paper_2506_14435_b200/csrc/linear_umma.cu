// Tensor-core product of mote_linear: out = act( w_scale * (x W^T) + bias ) + residual, tcgen05.mma kind::f16 with TMEM accumulators,
// operands staged in shared memory by TMA.
//
// Tile: 128 tokens (one TMEM lane each; 256 for a pair of CTAs) x bn rows of W (bn a multiple of 16, of 32 for a pair, up to 256); K
// advances 64 elements, 128 bytes of either operand, per pipeline stage, four K = 16 MMAs each.  What lies beyond the tensors is zero
// (TMA fill) and is not stored.
//
// Warp roles: 0 TMA producer, 1 MMA issuer, 2 TMEM owner, 4 to 19 epilogue (four per TMEM lane quarter, which share the tile's columns).
// Three forms:
//   pairs of CTAs (CG = 2)   cta_group::2 MMAs read half of the weight rows from either CTA: a tile of 256 x 256 fetches 32 KB a stage and
//                            SM, two thirds of what two tiles of 128 x 256 do
//   single CTAs (CG = 1)     persistent as the pairs are: two accumulators in TMEM let a tile's epilogue run under the next one's MMAs
//   split along K (kSplit)   a cluster of CTAs shares one tile's K where the tiles are too few for the SMs; the partial sums meet in
//                            distributed shared memory, are added in rank order, and each CTA finishes its share of the columns
//
// Every mbarrier wait is bounded; on expiry the CTA raises the status word and leaves.
#include <algorithm>

#include "linear_act.cuh"
#include "ptx_sm100.cuh"
#include "tile_launch.cuh"

namespace mote {

using namespace ptx;

constexpr int kLinEpiFirst = 4, kLinEpiWarps = 16, kLinParts = kLinEpiWarps / 4;
constexpr int kLinThreads = (kLinEpiFirst + kLinEpiWarps) * 32;
constexpr int kLinStageA = 128 * 128;            // 128 rows x 128 bytes
constexpr int kLinMaxStages = 8;
constexpr int kLinPipeBytes = 192 * 1024;         // the stages' share of shared memory; less where rows of out have no alignment:
constexpr int kLinPipeBytesOdd = 148 * 1024;      // the epilogue then puts its rows together in shared memory
constexpr int kLinPitch = 33;                     // words per row of an epilogue warp's block for that: 64 bf16 or 32 fp32 values
constexpr int kLinStaging = kLinEpiWarps * 32 * kLinPitch * 4;

struct LinearTiles {
  int bn, stages, k_steps, splits;
  int n_mt, n_nt;
  int rows_fast;                                 // items: weight tiles (0) or token tiles (1) change fastest
  int a_rows;                                    // rows of the token operand's box
  int wide;                                      // rows of out on 32-byte boundaries
};

struct __align__(8) LinearBarriers {
  uint64_t full[kLinMaxStages], empty[kLinMaxStages], tmem_full[2], tmem_empty[2];
  uint32_t tmem_base;
  int abort_flag;
};
constexpr int kLinColumns = kLinEpiWarps * 2 * 64 * 4;      // scale and bias of an epilogue warp's columns
constexpr int kLinPastPipe = std::max(kLinPipeBytes, kLinPipeBytesOdd + kLinStaging);
constexpr int kLinSmem = 1024 + kLinPastPipe + kLinColumns + (int)sizeof(LinearBarriers);
static_assert(kLinSmem <= 227 * 1024, "shared memory of a CTA");

__device__ __forceinline__ void linear_item(const LinearTiles& t, int item, int& mt, int& nt) {
  if (t.rows_fast) { mt = item % t.n_mt; nt = item / t.n_mt; }
  else { nt = item % t.n_nt; mt = item / t.n_nt; }
}

// Scale and bias of an epilogue warp's `n` (up to 64) columns from col0 on, into its own block; asked for before the accumulator is
// complete.
__device__ __forceinline__ void load_columns(const LinearArgs& a, int64_t col0, int n, float* cols, int lane) {
  __syncwarp();
#pragma unroll
  for (int i = lane; i < 64; i += 32) {
    if (a.w_scale && i < n) cols[i] = __ldg(a.w_scale + col0 + i);
    if (a.bias && i < n) cols[64 + i] = __ldg(a.bias + col0 + i);
  }
  __syncwarp();
}

// The residual of 16 neighbouring columns of a row, where rows lie on 16-byte boundaries.
template <bool kOdd>
__device__ __forceinline__ void load_residual(const LinearArgs& a, int64_t row, int64_t col, uint4 (&r)[2]) {
  if (kOdd || !a.res || row >= a.T) return;
  const uint4* rp = reinterpret_cast<const uint4*>(a.res + row * a.ldr + col);
  if (col < a.N) r[0] = rp[0];
  if (col + 8 < a.N) r[1] = rp[1];
}

// Writes the `n` columns from col on that a warp has put together in its block, 32 rows from row0 on: neighbouring lanes write
// neighbouring elements, on any boundary.
__device__ __forceinline__ void write_rows(const LinearArgs& a, int64_t row0, int64_t col, int n, const uint32_t* stg, int lane) {
  __syncwarp();
  const int rows = (int)min(int64_t(32), a.T - row0);
  if (a.out_f32) {
    float* o = static_cast<float*>(a.out) + row0 * a.N + col + lane;
    const bool in = lane < n;
    const uint32_t* from = stg + lane;
#pragma unroll 8
    for (int r = 0; r < rows; ++r, o += a.N)
      if (in) *o = __uint_as_float(from[r * kLinPitch]);
  } else {
    uint16_t* o = static_cast<uint16_t*>(a.out) + row0 * a.N + col + lane;
    const uint16_t* from = reinterpret_cast<const uint16_t*>(stg) + lane;
    const bool in0 = lane < n, in1 = lane + 32 < n;
#pragma unroll 8
    for (int r = 0; r < rows; ++r, o += a.N) {
      if (in0) o[0] = from[r * 2 * kLinPitch];
      if (in1) o[32] = from[r * 2 * kLinPitch + 32];
    }
  }
  __syncwarp();
}

// Brings the residual of `n` columns from col on, 32 rows from row0 on, to the warp's block, where the rows lie on any boundary: as they will
// be stored, so that a lane takes its row's from where it then puts its results (fp32 results, of twice the size: from the upper half of
// the row, behind the first 16 results).  2-byte loads, neighbouring lanes neighbouring columns (419 x 896 x 9660: 18.7 us; each lane its own
// row's: 25.7).
__device__ __forceinline__ void read_rows(const LinearArgs& a, int64_t row0, int64_t col, int n, uint32_t* stg, int lane) {
  __syncwarp();
  const int rows = (int)min(int64_t(32), a.T - row0);
  const uint16_t* from = a.res + row0 * a.ldr + col + lane;
  uint16_t* to = reinterpret_cast<uint16_t*>(stg + (a.out_f32 ? 16 : 0)) + lane;
  const bool in0 = lane < n, in1 = lane + 32 < n;
#pragma unroll 1
  for (int r = 0; r < rows; r += 4) {
    uint16_t v0[4], v1[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (in0 && r + i < rows) v0[i] = from[(r + i) * a.ldr];
      if (in1 && r + i < rows) v1[i] = from[(r + i) * a.ldr + 32];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (in0) to[(r + i) * 2 * kLinPitch] = v0[i];
      if (in1) to[(r + i) * 2 * kLinPitch + 32] = v1[i];
    }
  }
  __syncwarp();
}

// Finishes 16 neighbouring columns of a warp's 32 rows (lane = row): scale, bias, activation, residual, one rounding.  Stored at once
// where rows lie on 16-byte boundaries, else put at column `at` of the warp's block.
template <bool kOdd>
__device__ __forceinline__ void finish_columns(const LinearArgs& a, const LinearTiles& t, uint64_t (&z)[8], const uint4 (&res)[2], int64_t row0,
                                               int64_t col, const float* cols, uint32_t* stg, int at, int lane) {
  if (a.w_scale) {
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const ulonglong2 s = reinterpret_cast<const ulonglong2*>(cols)[v];
      z[2 * v] = mul_f32x2(z[2 * v], s.x);
      z[2 * v + 1] = mul_f32x2(z[2 * v + 1], s.y);
    }
  }
  if (a.bias) {
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const ulonglong2 b = reinterpret_cast<const ulonglong2*>(cols + 64)[v];
      z[2 * v] = add_f32x2(z[2 * v], b.x);
      z[2 * v + 1] = add_f32x2(z[2 * v + 1], b.y);
    }
  }
  apply_act16(z, a.act);
  const int64_t row = row0 + lane;
  if (a.res) {
    if (!kOdd) {                                 // a half that lies outside is not stored
      const uint32_t w[8] = {res[0].x, res[0].y, res[0].z, res[0].w, res[1].x, res[1].y, res[1].z, res[1].w};
#pragma unroll
      for (int j = 0; j < 8; ++j) z[j] = add_f32x2(z[j], f32x2_bits(w[j] << 16, w[j] & 0xFFFF0000u));
    } else {                                     // (columns and rows that are not there hold anything)
      const uint32_t* w = stg + lane * kLinPitch + (a.out_f32 ? 16 : 0) + at / 2;
#pragma unroll
      for (int j = 0; j < 8; ++j) z[j] = add_f32x2(z[j], f32x2_bits(w[j] << 16, w[j] & 0xFFFF0000u));
    }
  }
  uint32_t w[16];                                // the values as stored: 16 words, or 8 of two bf16 each
  if (a.out_f32) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float lo, hi;
      unpack_f32x2(z[j], lo, hi);
      w[2 * j] = __float_as_uint(lo);
      w[2 * j + 1] = __float_as_uint(hi);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float lo, hi;
      unpack_f32x2(z[j], lo, hi);
      w[j] = pack_bf16x2(lo, hi);
    }
  }
  if (kOdd) {
    if (a.out_f32) {
#pragma unroll
      for (int j = 0; j < 16; ++j) stg[lane * kLinPitch + at + j] = w[j];
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) stg[lane * kLinPitch + at / 2 + j] = w[j];
    }
    return;
  }
  // N is a multiple of 8: each half of the 16 columns is inside or outside as a whole
  if (row >= a.T) return;
  const bool both_in = col + 16 <= a.N;
  if (a.out_f32) {
    float* o = static_cast<float*>(a.out) + row * a.N + col;
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (h == 0 || both_in) {
        const uint32_t* v = w + 8 * h;
        if (t.wide) st_global_v8(o + 8 * h, v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]);
        else {
          reinterpret_cast<uint4*>(o + 8 * h)[0] = make_uint4(v[0], v[1], v[2], v[3]);
          reinterpret_cast<uint4*>(o + 8 * h)[1] = make_uint4(v[4], v[5], v[6], v[7]);
        }
      }
  } else {
    uint16_t* o = static_cast<uint16_t*>(a.out) + row * a.N + col;
    if (t.wide) st_global_v8(o, w[0], w[1], w[2], w[3], w[4], w[5], w[6], w[7]);
    else {
      reinterpret_cast<uint4*>(o)[0] = make_uint4(w[0], w[1], w[2], w[3]);
      if (both_in) reinterpret_cast<uint4*>(o)[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
  }
}

struct Ring {
  uint32_t stage = 0, phase = 0;
  __device__ __forceinline__ void next(uint32_t n) {
    if (++stage == n) { stage = 0; phase ^= 1; }
  }
};

// kOdd: rows of out (or residual) without 16-byte boundaries.  (A kernel of its own: as a branch it costs the others 3 %.)
template <int CG, bool kSplit, bool kOdd>
__global__ void __launch_bounds__(kLinThreads, 1)
linear_umma_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_b, const LinearArgs a, const LinearTiles t) {
  static_assert(CG == 1 || !kSplit, "K is split over single CTAs");
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem_gen = smem_raw + (smem_base - smem_u32(smem_raw));
  const uint32_t stage_b = uint32_t(t.bn / CG) * 128;
  const uint32_t stage_bytes = kLinStageA + stage_b;
  uint32_t* staging = reinterpret_cast<uint32_t*>(smem_gen + kLinPipeBytesOdd);      // kOdd
  float* column_data = reinterpret_cast<float*>(smem_gen + kLinPastPipe);
  LinearBarriers* bars = reinterpret_cast<LinearBarriers*>(smem_gen + kLinPastPipe + kLinColumns);
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
    uint32_t* stg = staging + (warp - kLinEpiFirst) * 32 * kLinPitch;
    float* cols = column_data + (warp - kLinEpiFirst) * 128;
    const int share = (t.bn / kLinParts + 15) & ~15;            // columns of one of the warps of a lane quarter, up to 64
    const int room = a.out_f32 ? 32 : 64;                       // columns that a warp's block holds
    int local = 0;
    for (int item = worker; item < n_items; item += workers, ++local) {
      int mt, nt;
      linear_item(t, item, mt, nt);
      const int buf = local & 1;
      const int64_t row0 = int64_t(mt * CG + (CG == 2 ? (int)rank : 0)) * 128 + q * 32, col0 = int64_t(nt) * t.bn + part * share;
      const uint32_t t_row = tmem_base + (uint32_t(q * 32) << 16) + buf * 256 + part * share;
      // columns of this warp that are there (a warp beyond the last row has none)
      const int n = row0 < a.T ? (int)max(int64_t(0), min(int64_t(min(share, t.bn - part * share)), a.N - col0)) : 0;
      if (n > 0) load_columns(a, col0, n, cols, lane);
      uint4 res[2];
      if (n > 0) load_residual<kOdd>(a, row0 + lane, col0, res);
      const bool block_res = kOdd && a.res;                     // the residual comes through the warp's block
      if (block_res && n > 0) read_rows(a, row0, col0, min(room, n), stg, lane);
      if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&bars->tmem_full[buf]), (local >> 1) & 1, abort_flag))) break;
      tc_fence_after();
      int put = 0;
#pragma unroll 1
      for (int c = 0; c < n; c += 16) {
        if (block_res && put == 0 && c > 0) read_rows(a, row0, col0 + c, min(room, n - c), stg, lane);
        uint32_t r[16];
        tmem_ld_32x32b_x16(t_row + c, r);
        if (c > 0) load_residual<kOdd>(a, row0 + lane, col0 + c, res);
        tmem_wait_ld();
        uint64_t z[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) z[j] = f32x2_bits(r[2 * j], r[2 * j + 1]);
        finish_columns<kOdd>(a, t, z, res, row0, col0 + c, cols + c, stg, put, lane);
        if (kOdd) {
          put += 16;
          if (put == room || c + 16 >= n) {
            write_rows(a, row0, col0 + c + 16 - put, min(put, n - (c + 16 - put)), stg, lane);
            put = 0;
          }
        }
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
      for (int c = part * 16; c < t.bn; c += 16 * kLinParts) {
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
      uint32_t* stg = staging + (warp - kLinEpiFirst) * 32 * kLinPitch;
      float* cols = column_data + (warp - kLinEpiFirst) * 128;
      const int room = a.out_f32 ? 32 : 64;
      int mt, nt;
      linear_item(t, worker, mt, nt);
      const int64_t row0 = int64_t(mt) * 128 + q * 32;
      const int w = t.bn / t.splits;               // columns this CTA finishes, a multiple of 16
      const int share = (w / kLinParts + 15) & ~15;
      const int first = (int)rank * w + part * share;
      const int64_t col0 = int64_t(nt) * t.bn + first;
      const int n = row0 < a.T ? (int)max(int64_t(0), min(int64_t(min(share, w - part * share)), a.N - col0)) : 0;
      if (n > 0) load_columns(a, col0, n, cols, lane);
      int put = 0;
#pragma unroll 1
      for (int c = 0; c < n; c += 16) {
        uint4 res[2];
        load_residual<kOdd>(a, row0 + lane, col0 + c, res);
        if (kOdd && a.res && put == 0) read_rows(a, row0, col0 + c, min(room, n - c), stg, lane);
        uint64_t z[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) z[j] = 0ull;
        for (int s = 0; s < t.splits; ++s) {
          const uint32_t src = map_to_rank(smem_base + uint32_t((first + c) * 128 + q * 32 + lane) * 4, s);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            float lo, hi;
            asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(lo) : "r"(src + j * 1024) : "memory");
            asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(hi) : "r"(src + j * 1024 + 512) : "memory");
            z[j] = add_f32x2(z[j], f32x2(lo, hi));
          }
        }
        finish_columns<kOdd>(a, t, z, res, row0, col0 + c, cols + c, stg, put, lane);
        if (kOdd) {
          put += 16;
          if (put == room || c + 16 >= n) {
            write_rows(a, row0, col0 + c + 16 - put, min(put, n - (c + 16 - put)), stg, lane);
            put = 0;
          }
        }
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
// Which form and tile width: the least estimated time, in cycles.  The estimate's constants were fitted to times of all forms at 79
// sizes (17 to 8192 tokens, 26 to 11008 rows, K 128 to 11008): the form that it names is 0.9 % slower than the best one on average and
// 16 % at worst (2048 x 2048 x 2048: pairs of 256, 18.1 us, single CTAs of 240 15.7).  Times of those runs, one size back to back (as calls among
// others the first two below take 150 and 14.9 us).  Tokens x N x K: 4096 x 11008 x 2048: pairs of 256, 122 us
// (single CTAs 133), 333 x 8960 x 1536: single CTAs of 192, 13.6 us (pairs 16), 64 x 2048 x 2048: tiles of 64 split four ways, 8.4 us (whole 10).
struct LinearForm { int cg, bn, splits; };
static LinearForm pick_form(int64_t T, int64_t N, int k_steps, int sms, const int (&clusters)[9]) {
  LinearForm best{1, 256, 1};
  double best_cost = 1e300;
  auto consider = [&](int cg, int bn, int splits) {
    const int64_t items = ((T + 128 * cg - 1) / (128 * cg)) * ((N + bn - 1) / bn);
    const int64_t workers = splits > 1 ? clusters[splits] : sms / cg;            // items that are worked on at a time
    if (workers < 1) return;
    const double rounds = double((items + workers - 1) / workers);
    const double active = double(std::min(items, workers)) * cg * splits;
    // a step: four MMAs, the way of its operands from L2 (61 bytes a cycle for an SM, 9300 for all of them), or a stage's latency
    const double bytes = double(std::min<int64_t>(T, 128)) * 128 + double(bn / cg) * 128;
    const double step = std::max({2.0 * bn, bytes / 61.0, bytes * active / 9300.0, 420.0});
    const double main = double((k_steps + splits - 1) / splits) * step;
    const double epilogue = 1900.0 + 19.0 * bn / splits + (splits > 1 ? 2800.0 + 28.0 * bn : cg == 2 ? 4000.0 : 0.0);
    const double cost = main + epilogue + (rounds - 1) * (std::max(main, epilogue) + 1000.0);
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

template <int CG, bool kSplit, bool kOdd>
static cudaError_t launch_form(const CUtensorMap& ta, const CUtensorMap& tb, const LinearArgs& a, const LinearTiles& t, int grid, int cluster,
                               cudaStream_t stream) {
  static PerDeviceOnce once;
  const cudaError_t e = set_max_dynamic_smem(once, linear_umma_kernel<CG, kSplit, kOdd>, kLinSmem);
  if (e != cudaSuccess) return e;
  return launch_ex(linear_umma_kernel<CG, kSplit, kOdd>, dim3(grid), dim3(kLinThreads), kLinSmem, stream, true, cluster, ta, tb, a, t);
}

template <bool kOdd>
static cudaError_t launch_any(const LinearForm& f, const CUtensorMap& ta, const CUtensorMap& tb, const LinearArgs& a, const LinearTiles& t, int items,
                              int sms, cudaStream_t stream) {
  return f.splits > 1 ? launch_form<1, true, kOdd>(ta, tb, a, t, items * f.splits, f.splits, stream)
         : f.cg == 2  ? launch_form<2, false, kOdd>(ta, tb, a, t, 2 * std::min(items, sms / 2), 2, stream)
                      : launch_form<1, false, kOdd>(ta, tb, a, t, std::min(items, sms), 1, stream);
}

mote_status_t launch_linear_umma(const LinearArgs& a, cudaStream_t stream) {
  const int sms = device_sm_count();
  LinearTiles t{};
  t.k_steps = (a.K + 63) / 64;
  static PerDeviceOnce split_once;               // its shared-memory limit has to be set before the query
  if (set_max_dynamic_smem(split_once, linear_umma_kernel<1, true, false>, kLinSmem) != cudaSuccess) return MOTE_ERR_CUDA;
  static ResidentClusters resident;
  int clusters[9] = {};
  for (int c = 2; c <= 8; c *= 2) clusters[c] = resident.get(linear_umma_kernel<1, true, false>, kLinThreads, kLinSmem, c);
  const LinearForm f = pick_form(a.T, a.N, t.k_steps, sms, clusters);
  t.bn = f.bn; t.splits = f.splits;
  t.n_mt = (int)((a.T + 128 * f.cg - 1) / (128 * f.cg));
  t.n_nt = (int)((a.N + f.bn - 1) / f.bn);
  if (int64_t(t.n_mt) * t.n_nt > (1ll << 28)) return MOTE_ERR_SHAPE;
  // the smaller operand's tiles change fastest: its whole stays in L2, the larger one is read from HBM once
  t.rows_fast = a.T <= a.N;
  t.a_rows = f.cg == 1 ? (int)std::min<int64_t>(128, (a.T + 7) / 8 * 8) : 128;
  const bool odd = a.N % 8 != 0 || (a.res && a.ldr % 8 != 0);
  t.stages = std::min(kLinMaxStages, (odd ? kLinPipeBytesOdd : kLinPipeBytes) / (kLinStageA + f.bn / f.cg * 128));
  t.wide = a.N % 16 == 0 && (reinterpret_cast<uintptr_t>(a.out) & 31u) == 0;
  CUtensorMap ta, tb;
  if (!make_operand_map(&ta, a.x, a.T, a.K, a.ldx, t.a_rows) || !make_operand_map(&tb, a.W, a.N, a.K, a.K, f.bn / f.cg)) return MOTE_ERR_CUDA;
  const int items = t.n_mt * t.n_nt;
  const cudaError_t e = odd ? launch_any<true>(f, ta, tb, a, t, items, sms, stream) : launch_any<false>(f, ta, tb, a, t, items, sms, stream);
  if (e != cudaSuccess) return MOTE_ERR_CUDA;
  MOTE_LAUNCH_OK();
  return MOTE_OK;
}

}  // namespace mote
