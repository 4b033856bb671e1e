// The tensor-core product behind the operators on raw tensors (vocab_loss.cu, orthogonalize.cu):
//
//     C[z] = epilogue( sum over products (i, j) of  A_i[z] B_j[z]^T )
//
// with A_i [M][K] and B_j [N][K] matrices of 16-bit numbers, K- or MN-major.  An operand is given as NP "pieces" whose
// sum is the operand: one for a bf16 tensor, two fp16 pieces (22 significant bits, operands scaled into fp16's range by
// the caller), three bf16 pieces (24 bits, all of fp32's range).  The products kept are those with i + j < NP (1, 3 or
// 6 of them): the dropped ones are below the last bit kept.  A stage of the ring holds a 64-wide K block of all pieces
// of both operands, so two pieces cost three products but only twice the operand traffic.
//
// Persistent kernel on CTA pairs (cta_group::2), a 256 x 256 tile per pair:
//   warp 0     TMA producer (each CTA brings its 128 rows of A and its 128 columns of B)
//   warp 1     leader: issues the MMAs.  A tensor-memory accumulator is used for `chunk_kb` K blocks and then handed to
//              the epilogue; two of them alternate, so that products run while the other one is collected
//   warps 2-9  epilogue: warp w owns TMEM lanes 32 (w % 4) .. + 31 (rows) and one half of the columns; a thread adds the
//              chunks of its row's 128 columns in registers, rounding to nearest.  The tensor core's own fp32
//              accumulation truncates, which biases a sum of a thousand MMAs by about 2e-5 of its value: short
//              chunks keep that below the last bits that matter (see kChunk*), and since a tile's last chunk is
//              collected like any other, the epilogue of a tile runs under the products of the next one.
// Outputs leave through 4 KB of shared memory per warp and TMA stores, which clip at the tensor's edge; ragged M, N
// and K are the zero fill of the loads and that clip.  A symmetric result is computed on and above the diagonal tiles and
// stored twice, the second time from a transposed box.
// Before a CTA exits, every arrival that the tensor core or the other CTA sends to its barriers has been waited for.
#pragma once

#include "ls_internal.h"
#include "tc_ptx.cuh"

#include <cuda_fp16.h>

namespace ls {
namespace gop {

using namespace ptx;

constexpr int kTile = 256;               // rows and columns of a pair's tile
constexpr int kThreads = 320;            // warp 0 producer, warp 1 MMA issuer, warps 2-9 epilogue
constexpr int kSlice = 128;              // columns of an epilogue thread: the unit of the row statistics
constexpr int kStageBoxBytes = 4096;     // staging of one epilogue warp: 32 rows x 128 bytes

template <int NP>
struct Smem {
  static constexpr int kOperand = 128 * 128;                       // 128 rows (or columns) x 64 numbers
  static constexpr int kStage = 2 * NP * kOperand;
  static constexpr int kStages = NP == 1 ? 6 : NP == 2 ? 3 : 2;
  static constexpr int kRing = kStages * kStage;
  static constexpr int kOut = 8 * kStageBoxBytes;
  static constexpr int kBars = 2 * kStages + 4;
  static constexpr int kTotal = 1024 + kRing + kOut + kBars * 8 + 16;
  static_assert(kTotal <= 227 * 1024, "shared memory budget");
};

enum Epi {
  EPI_F32,        // fp32 C = alpha acc (reduce: C += alpha acc)
  EPI_BF16,       // bf16 C = alpha acc
  EPI_STATS,      // row statistics of exp only
  EPI_STATS_F16,  // statistics, and C = fp16 exp(acc - slice maximum)
  EPI_STATS_F32,  // statistics, and C = fp32 acc
  EPI_PIECES,     // two fp16 pieces of alpha acc + diag I (once or twice, with other factors), optionally mirrored
};

struct Params {
  int m_tiles, n_tiles, batch, splits;   // splits > 1: K is cut, split s writes plane c_z0 + z c_zstep + s
  int num_kb, kb_per_split, chunk_kb;
  int total;                             // tiles of the launch
  int tri;                               // 1: only tiles on or above the diagonal (symmetric C)
  int n_fast;                            // 1: neighbouring pairs take neighbouring columns, else neighbouring rows
  int a_z0, a_zstep, b_z0, b_zstep;      // plane of batch entry z: z0 + z * zstep (+ piece)
  int c_z0, c_zstep;
  int M, N;
  float alpha;
  const float* alpha_dev;                // EPI_F32, EPI_BF16: a further factor of alpha in device memory, or null
  int reduce;                            // EPI_F32: C += instead of C =
  // row statistics: slice t = column / 128 of row r at [t * stat_ld + r]
  float* stat_max;                       // slice maximum * log2(e)
  float* stat_sum;                       // sum over the slice of exp(acc - slice maximum)
  int64_t stat_ld;
  const int32_t* labels;                 // [M]; a label inside the slice gets its logit written to label_logit[row]
  float* label_logit;
  // EPI_PIECES: output i (of n_out) is planes c + 2 i (first piece) and c + 2 i + 1 of the stack
  int n_out;
  float out_alpha[2], out_diag[2];       // out_alpha acc + out_diag on the diagonal
  int mirror;
  int* err;
};

struct Tile { int m, n, split, z; };

__device__ __forceinline__ Tile tile_of(const Params& p, int t) {
  Tile r;
  const int per = p.tri ? p.m_tiles * (p.m_tiles + 1) / 2 : p.m_tiles * p.n_tiles;
  const int q = t / per, i = t - q * per;
  r.z = q / p.splits;
  r.split = q - r.z * p.splits;
  if (p.tri) {
    int n = (int)((sqrtf(8.f * (float)i + 1.f) - 1.f) * 0.5f);
    while ((n + 1) * (n + 2) / 2 <= i) ++n;
    while (n * (n + 1) / 2 > i) --n;
    r.n = n;
    r.m = i - n * (n + 1) / 2;
  } else if (p.n_fast) {
    r.m = i / p.n_tiles;
    r.n = i - r.m * p.n_tiles;
  } else {
    r.n = i / p.m_tiles;
    r.m = i - r.n * p.m_tiles;
  }
  return r;
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ void store_box(const CUtensorMap* m, const void* src, int x, int y, int z) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(
                   reinterpret_cast<uint64_t>(m)),
               "r"(smem_u32(src)), "r"(x), "r"(y), "r"(z)
               : "memory");
}
__device__ __forceinline__ void add_box(const CUtensorMap* m, const void* src, int x, int y, int z) {
  asm volatile("cp.reduce.async.bulk.tensor.3d.global.shared::cta.add.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(
                   reinterpret_cast<uint64_t>(m)),
               "r"(smem_u32(src)), "r"(x), "r"(y), "r"(z)
               : "memory");
}
// the staging box may be written again: the bulk store has read it
__device__ __forceinline__ void box_free(int lane) {
  if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
  __syncwarp();
}
// hand the box over: all lanes have written it
__device__ __forceinline__ void box_send(const CUtensorMap* m, const void* box, int lane, int x, int y, int z, bool add) {
  fence_proxy_async_smem();
  __syncwarp();
  if (lane == 0) {
    if (add) add_box(m, box, x, y, z);
    else store_box(m, box, x, y, z);
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
  }
}

template <int NP, bool F16, bool A_MN, bool B_MN, int EPI>
__global__ void __launch_bounds__(kThreads, 1)
gemm_op_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
               const __grid_constant__ CUtensorMap tmC, const __grid_constant__ CUtensorMap tmCT, const Params p) {
  using L = Smem<NP>;
  constexpr int STAGES = L::kStages;
  constexpr uint32_t IDESC = make_idesc(F16 ? 0u : 1u, A_MN, B_MN, 256, 256);
  constexpr uint32_t TMEM_COLS = 512;

  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint8_t* out_base = smem + L::kRing;
  uint64_t* full = reinterpret_cast<uint64_t*>(out_base + L::kOut);
  uint64_t* empty = full + STAGES;
  uint64_t* acc_full = empty + STAGES;         // [2]
  uint64_t* acc_empty = acc_full + 2;          // [2] leader's: sixteen epilogue warps of the pair
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_empty + 2);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = (int)cluster_ctarank();
  const int pair = (int)(blockIdx.x >> 1), pairs = (int)(gridDim.x >> 1);
  bool failed = false;

  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
    for (int s = 0; s < 2; ++s) { mbar_init(&acc_full[s], 1); mbar_init(&acc_empty[s], 16); }
    fence_mbar_init();
    prefetch_tmap(&tmA);
    prefetch_tmap(&tmB);
    prefetch_tmap(&tmC);
    if (EPI == EPI_PIECES) prefetch_tmap(&tmCT);
  }
  __syncwarp();
  if (warp == 1) {
    tmem_alloc_pair(tmem_slot, TMEM_COLS);
    tmem_relinquish_pair();
  }
  tc_fence_before_sync();
  cluster_sync_all();       // both CTAs' barriers exist before either signals the other
  tc_fence_after_sync();
  const uint32_t tmem_base = *tmem_slot;
  grid_dep_wait();
  grid_dep_launch();

  if (warp == 0) {
    if (elect_one()) {
      const uint64_t pol = l2_policy(0);
      const uint32_t full_leader = map_to_rank(smem_u32(&full[0]), 0);
      int it = 0;
      for (int t = pair; t < p.total && !failed; t += pairs) {
        const Tile tl = tile_of(p, t);
        const int k0 = tl.split * p.kb_per_split;
        const int k1 = min(p.num_kb, k0 + p.kb_per_split);
        const int az = p.a_z0 + tl.z * p.a_zstep, bz = p.b_z0 + tl.z * p.b_zstep;
        const int ma = tl.m * kTile + rank * 128, nb = tl.n * kTile + rank * 128;
        for (int kb = k0; kb < k1; ++kb, ++it) {
          const int s = it % STAGES;
          if (it >= STAGES && !mbar_wait(&empty[s], ((it / STAGES) - 1) & 1)) { atomicExch(p.err, 31); failed = true; break; }
          if (rank == 0) mbar_expect_tx(&full[s], 2 * L::kStage);      // both CTAs' bytes
          const uint32_t bar = full_leader + (uint32_t)(s * 8);
          uint8_t* sa = smem + s * L::kStage;
          uint8_t* sb = sa + NP * L::kOperand;
#pragma unroll
          for (int q = 0; q < NP; ++q) {
            if (A_MN) {
              tma_load_3d_pair(sa + q * L::kOperand, &tmA, bar, ma, kb * 64, az + q, pol);
              tma_load_3d_pair(sa + q * L::kOperand + 8192, &tmA, bar, ma + 64, kb * 64, az + q, pol);
            } else {
              tma_load_3d_pair(sa + q * L::kOperand, &tmA, bar, kb * 64, ma, az + q, pol);
            }
            if (B_MN) {
              tma_load_3d_pair(sb + q * L::kOperand, &tmB, bar, nb, kb * 64, bz + q, pol);
              tma_load_3d_pair(sb + q * L::kOperand + 8192, &tmB, bar, nb + 64, kb * 64, bz + q, pol);
            } else {
              tma_load_3d_pair(sb + q * L::kOperand, &tmB, bar, kb * 64, nb, bz + q, pol);
            }
          }
        }
      }
      // the releases of the last stages arrive here from the leader's tensor core: wait for them before leaving
      for (int s = 0; s < STAGES && s < it && !failed; ++s) {
        const int uses = (it - 1 - s) / STAGES + 1;
        if (!mbar_wait(&empty[s], (uses - 1) & 1)) { atomicExch(p.err, 35); failed = true; }
      }
    }
  } else if (warp == 1) {
    if (rank == 0 && elect_one()) {
      int it = 0, ch = 0;
      for (int t = pair; t < p.total && !failed; t += pairs) {
        const Tile tl = tile_of(p, t);
        const int k0 = tl.split * p.kb_per_split;
        const int nk = min(p.num_kb, k0 + p.kb_per_split) - k0;
        for (int kb = 0; kb < nk; ++kb, ++it) {
          const int in_chunk = kb % p.chunk_kb;
          if (in_chunk == 0 && ch >= 2 && !mbar_wait(&acc_empty[ch & 1], ((ch >> 1) - 1) & 1)) {
            atomicExch(p.err, 32); failed = true; break;
          }
          const int s = it % STAGES;
          if (!mbar_wait(&full[s], (it / STAGES) & 1)) { atomicExch(p.err, 33); failed = true; break; }
          tc_fence_after_sync();
          const uint32_t d_tmem = tmem_base + (uint32_t)((ch & 1) * kTile);
          const uint32_t a_addr = smem_u32(smem + s * L::kStage);
          const uint32_t b_addr = a_addr + NP * L::kOperand;
          bool first = in_chunk == 0;
          // small products first
#pragma unroll
          for (int i = NP - 1; i >= 0; --i)
#pragma unroll
            for (int j = NP - 1 - i; j >= 0; --j)
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const uint64_t da = make_smem_desc(a_addr + i * L::kOperand + (A_MN ? k * 2048 : k * 32), A_MN ? 8192 : 16, 1024);
                const uint64_t db = make_smem_desc(b_addr + j * L::kOperand + (B_MN ? k * 2048 : k * 32), B_MN ? 8192 : 16, 1024);
                mma_bf16_pair(d_tmem, da, db, IDESC, first ? 0u : 1u);
                first = false;
              }
          mma_commit_pair(&empty[s]);
          if (in_chunk == p.chunk_kb - 1 || kb == nk - 1) {
            mma_commit_pair(&acc_full[ch & 1]);
            ++ch;
          }
        }
      }
      // both CTAs' epilogues have let go of the last accumulators
      for (int b = 0; b < 2 && b < ch && !failed; ++b) {
        const int uses = (ch - 1 - b) / 2 + 1;
        if (!mbar_wait(&acc_empty[b], (uses - 1) & 1)) { atomicExch(p.err, 36); failed = true; }
      }
    }
  } else {
    const int q = warp & 3, cs = (warp - 2) >> 2;
    const uint32_t taddr = tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(cs * kSlice);
    uint8_t* box = out_base + (warp - 2) * kStageBoxBytes;
    uint8_t* myrow = box + lane * 128;
    const uint32_t empty_leader = map_to_rank(smem_u32(&acc_empty[0]), 0);
    int ch = 0;
    for (int t = pair; t < p.total && !failed; t += pairs) {
      const Tile tl = tile_of(p, t);
      const int k0 = tl.split * p.kb_per_split;
      const int nk = min(p.num_kb, k0 + p.kb_per_split) - k0;
      const int chunks = (nk + p.chunk_kb - 1) / p.chunk_kb;
      uint32_t acc[4][32];
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 32; ++i) acc[j][i] = 0u;
      for (int c = 0; c < chunks; ++c, ++ch) {
        const int buf = ch & 1;
        if (!__all_sync(0xffffffffu, mbar_wait(&acc_full[buf], (ch >> 1) & 1))) {
          if (lane == 0) atomicExch(p.err, 34);
          failed = true;
          break;
        }
        __syncwarp();
        tc_fence_after_sync();
        const uint32_t at = taddr + (uint32_t)(buf * kTile);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          uint32_t r[16];
          tmem_ld_32x16(at + j * 16, r);
          tmem_ld_wait();
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            uint32_t& sum = acc[j >> 1][(j & 1) * 16 + i];
            sum = __float_as_uint(__uint_as_float(sum) + __uint_as_float(r[i]));
          }
        }
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(empty_leader + (uint32_t)(buf * 8));
        __syncwarp();
      }
      if (failed) break;
      const int wr0 = tl.m * kTile + rank * 128 + q * 32;        // first row of the warp
      const int row = wr0 + lane;
      const int col0 = tl.n * kTile + cs * kSlice;
      const int zc = p.c_z0 + tl.z * p.c_zstep + tl.split;
      if (wr0 >= p.M) continue;                                    // nothing of the warp's rows is inside
      if constexpr (EPI == EPI_STATS || EPI == EPI_STATS_F16 || EPI == EPI_STATS_F32) {
        if (col0 + kSlice > p.N) {                                 // the ragged end (or all) of the last slices
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (col0 + j * 32 + i >= p.N) acc[j][i] = 0xff800000u;
        }
        float mx = -INFINITY;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int i = 0; i < 32; ++i) mx = fmaxf(mx, __uint_as_float(acc[j][i]));
        constexpr float kLog2e = 1.4426950408889634f;
        // (a slice of nothing but -inf: any finite reference gives the zero terms that it has; a finite maximum's reference
        // stays finite)
        const float ref = mx == -INFINITY ? 0.f : mx < 0.f ? fmaxf(mx * kLog2e, -3.4e38f) : mx * kLog2e;
        if (p.labels != nullptr) {
          const int lab = row < p.M ? p.labels[row] - col0 : -1;
          const bool mine = lab >= 0 && lab < kSlice && lab + col0 < p.N;
          if (__any_sync(0xffffffffu, mine)) {
            float zl = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
              for (int i = 0; i < 32; ++i)
                if (lab == j * 32 + i) zl = __uint_as_float(acc[j][i]);
            if (mine) p.label_logit[row] = zl;
          }
        }
        if constexpr (EPI == EPI_STATS_F32) {
          // the logits themselves leave; the exponentials are only summed
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if (col0 + j * 32 >= p.N) continue;
            box_free(lane);
#pragma unroll
            for (int u = 0; u < 8; ++u)
              *reinterpret_cast<uint4*>(myrow + ((u ^ (lane & 7)) << 4)) =
                  make_uint4(acc[j][4 * u], acc[j][4 * u + 1], acc[j][4 * u + 2], acc[j][4 * u + 3]);
            box_send(&tmC, box, lane, col0 + j * 32, wr0, zc, false);
          }
        }
        float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            const float e = ex2(fmaf(__uint_as_float(acc[j][i]), kLog2e, -ref));
            part[i & 3] += e;
            acc[j][i] = __float_as_uint(e);
          }
        if (row < p.M) {
          const int64_t at = (int64_t)(tl.n * 2 + cs) * p.stat_ld + row;
          p.stat_max[at] = mx == -INFINITY ? -INFINITY : ref;
          p.stat_sum[at] = (part[0] + part[1]) + (part[2] + part[3]);
        }
        if constexpr (EPI == EPI_STATS_F16) {
#pragma unroll
          for (int b2 = 0; b2 < 2; ++b2) {
            if (col0 + b2 * 64 >= p.N) continue;
            box_free(lane);
#pragma unroll
            for (int u = 0; u < 8; ++u) {
              uint32_t w[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int i = u * 8 + e * 2;
                __half2 h = __floats2half2_rn(__uint_as_float(acc[b2 * 2 + (i >> 5)][i & 31]),
                                              __uint_as_float(acc[b2 * 2 + ((i + 1) >> 5)][(i + 1) & 31]));
                w[e] = *reinterpret_cast<uint32_t*>(&h);
              }
              *reinterpret_cast<uint4*>(myrow + ((u ^ (lane & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
            }
            box_send(&tmC, box, lane, col0 + b2 * 64, wr0, zc, false);
          }
        }
      }
      const float alpha = (EPI == EPI_F32 || EPI == EPI_BF16) && p.alpha_dev != nullptr ? p.alpha * __ldg(p.alpha_dev) : p.alpha;
      if constexpr (EPI == EPI_F32) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (col0 + j * 32 >= p.N) continue;
          box_free(lane);
#pragma unroll
          for (int u = 0; u < 8; ++u) {
            float4 v;
            v.x = alpha * __uint_as_float(acc[j][4 * u]);
            v.y = alpha * __uint_as_float(acc[j][4 * u + 1]);
            v.z = alpha * __uint_as_float(acc[j][4 * u + 2]);
            v.w = alpha * __uint_as_float(acc[j][4 * u + 3]);
            *reinterpret_cast<float4*>(myrow + ((u ^ (lane & 7)) << 4)) = v;
          }
          box_send(&tmC, box, lane, col0 + j * 32, wr0, zc, p.reduce != 0);
        }
      }
      if constexpr (EPI == EPI_BF16) {
#pragma unroll
        for (int b2 = 0; b2 < 2; ++b2) {
          if (col0 + b2 * 64 >= p.N) continue;
          box_free(lane);
#pragma unroll
          for (int u = 0; u < 8; ++u) {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int i = u * 8 + e * 2;
              __nv_bfloat162 h = __floats2bfloat162_rn(alpha * __uint_as_float(acc[b2 * 2 + (i >> 5)][i & 31]),
                                                       alpha * __uint_as_float(acc[b2 * 2 + ((i + 1) >> 5)][(i + 1) & 31]));
              w[e] = *reinterpret_cast<uint32_t*>(&h);
            }
            *reinterpret_cast<uint4*>(myrow + ((u ^ (lane & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
          }
          box_send(&tmC, box, lane, col0 + b2 * 64, wr0, zc, false);
        }
      }
      if constexpr (EPI == EPI_PIECES) {
        const bool flip = p.mirror != 0 && tl.m != tl.n;
        for (int o = 0; o < p.n_out; ++o) {
          const float alpha_o = p.out_alpha[o], diag_o = p.out_diag[o];
          const int zp = zc + 2 * o;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int c0 = col0 + j * 32;
            if (c0 >= p.N) continue;
            // the first pieces of two columns in a word, and what they leave over: 32 x 32 boxes of 2 KB each
            uint32_t hi[16], lo[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const float v0 = fmaf(alpha_o, __uint_as_float(acc[j][2 * e]), row == c0 + 2 * e ? diag_o : 0.f);
              const float v1 = fmaf(alpha_o, __uint_as_float(acc[j][2 * e + 1]), row == c0 + 2 * e + 1 ? diag_o : 0.f);
              const __half2 h = __floats2half2_rn(v0, v1);
              const float2 f = __half22float2(h);
              const __half2 l = __floats2half2_rn(v0 - f.x, v1 - f.y);
              hi[e] = *reinterpret_cast<const uint32_t*>(&h);
              lo[e] = *reinterpret_cast<const uint32_t*>(&l);
            }
            box_free(lane);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
              uint8_t* at = box + lane * 64 + ((u ^ ((lane >> 1) & 3)) << 4);      // the 64-byte swizzle
              *reinterpret_cast<uint4*>(at) = make_uint4(hi[4 * u], hi[4 * u + 1], hi[4 * u + 2], hi[4 * u + 3]);
              *reinterpret_cast<uint4*>(at + 2048) = make_uint4(lo[4 * u], lo[4 * u + 1], lo[4 * u + 2], lo[4 * u + 3]);
            }
            box_send(&tmC, box, lane, c0, wr0, zp, false);
            box_send(&tmC, box + 2048, lane, c0, wr0, zp + 1, false);
            if (flip) {
              box_free(lane);
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                uint8_t* at = box + 2 * e * 64 + lane * 2;
                *reinterpret_cast<uint16_t*>(at) = (uint16_t)hi[e];
                *reinterpret_cast<uint16_t*>(at + 64) = (uint16_t)(hi[e] >> 16);
                *reinterpret_cast<uint16_t*>(at + 2048) = (uint16_t)lo[e];
                *reinterpret_cast<uint16_t*>(at + 2112) = (uint16_t)(lo[e] >> 16);
              }
              box_send(&tmCT, box, lane, wr0, c0, zp, false);
              box_send(&tmCT, box + 2048, lane, wr0, c0, zp + 1, false);
            }
          }
        }
      }
    }
    if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    tc_fence_before_sync();
  }
  __syncwarp();
  if (failed) {
    // a wait ran out: give the loads in flight time to land before the shared memory is released
    const long long t0 = clock64();
    while (clock64() - t0 < 4000000ll) {}
  }
  // neither CTA leaves (or frees tensor memory) while the other may still signal it
  cluster_sync_all();
  if (warp == 1) {
    tc_fence_after_sync();
    tmem_dealloc_pair(tmem_base, TMEM_COLS);
  }
}

// ---- host side ---------------------------------------------------------------------------------------------------

// A stack of `planes` row-major matrices [rows][cols] of 16-bit or fp32 numbers (row pitch ld, plane pitch `plane`, in
// elements, both 16-byte multiples), read or written in boxes of 128 bytes x box_rows rows with the 128-byte swizzle.
// MAP_F16_S, MAP_F16_T: boxes of 64 bytes x box_rows rows with the 64-byte swizzle, or none (EPI_PIECES' straight and
// transposed stores).
enum MapType { MAP_BF16, MAP_F16, MAP_F32, MAP_F16_S, MAP_F16_T };
int make_stack_map(CUtensorMap* out, const void* base, MapType type, int64_t rows, int64_t cols, int64_t planes, int64_t ld,
                   int64_t plane, int box_rows);
// where a bounded wait that runs out is recorded (one word per device, read by ls_device_status); null on failure
int* device_error_word();

// K blocks per tensor-memory accumulator.  One MMA adds 16 products per element and truncates: 64 (24, 48) MMAs per chunk
// bias a sum of equal signs by about 2e-6 (0.8e-6, 1.5e-6) of its value, and sums of mixed signs by far less.  The row
// statistics of bf16 operands, which leave in fp32, take 32.
constexpr int kChunk1 = 16, kChunk2 = 2, kChunk3 = 2;
constexpr int kPairs = 74;

// Fills in the tile counts and launches.  p.splits, p.M, p.N, p.batch, p.tri, p.n_fast and the epilogue's fields are the
// caller's; K is the contraction length.
template <int NP, bool F16, bool A_MN, bool B_MN, int EPI>
cudaError_t launch(const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& c, const CUtensorMap& ct, Params p, int64_t K,
                   cudaStream_t st) {
  auto kern = gemm_op_kernel<NP, F16, A_MN, B_MN, EPI>;
  static uint64_t configured = 0;        // one bit per device
  cudaError_t e = allow_dynamic_smem(kern, (int)Smem<NP>::kTotal, &configured);
  if (e != cudaSuccess) return e;
  p.m_tiles = (p.M + kTile - 1) / kTile;
  p.n_tiles = (p.N + kTile - 1) / kTile;
  p.num_kb = (int)((K + 63) / 64);
  if (p.splits < 1) p.splits = 1;
  p.kb_per_split = (p.num_kb + p.splits - 1) / p.splits;
  p.splits = (p.num_kb + p.kb_per_split - 1) / p.kb_per_split;       // (callers ask split_count() first: no change here)
  p.chunk_kb = NP == 1 ? (EPI == EPI_F32 || EPI == EPI_BF16 ? kChunk1 : kChunk1 / 2) : NP == 2 ? kChunk2 : kChunk3;
  const int64_t per = p.tri ? (int64_t)p.m_tiles * (p.m_tiles + 1) / 2 : (int64_t)p.m_tiles * p.n_tiles;
  const int64_t total = per * p.splits * p.batch;
  if (total > 2000000000ll) return cudaErrorInvalidValue;
  p.total = (int)total;
  p.err = device_error_word();
  if (p.err == nullptr) return cudaErrorUnknown;
  const unsigned pairs = (unsigned)(total < kPairs ? total : kPairs);
  return launch_dep(kern, dim3(2 * pairs), dim3(kThreads), Smem<NP>::kTotal, st, 2, a, b, c, ct, p);
}

// Into how many parts the contraction is cut when `tiles` output tiles leave pairs idle: enough parts to give each pair
// one, each of at least `least` K blocks.  Always a number that launch() keeps.
inline int split_count(int64_t tiles, int64_t K, int least) {
  const int num_kb = (int)((K + 63) / 64);
  int64_t s = tiles >= kPairs ? 1 : kPairs / tiles;
  if (s > num_kb / least) s = num_kb / least;
  if (s < 1) s = 1;
  const int per = (int)((num_kb + s - 1) / s);
  return (num_kb + per - 1) / per;
}

}  // namespace gop
}  // namespace ls
