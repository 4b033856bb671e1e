// The tensor-core product behind the operators on raw tensors (vocab_loss.cu, orthogonalize.cu):
//
//     C[z] = epilogue( sum over products (i, j) of  A_i[z] B_j[z]^T )
//
// with A_i [M][K] and B_j [N][K] matrices of 16-bit numbers, K- or MN-major.  An operand is given as NP "pieces" whose
// sum is the operand: one for a bf16 tensor, two fp16 pieces (22 significant bits, operands scaled into fp16's range by
// the caller), three bf16 pieces (24 bits, all of fp32's range).  The products kept are those with i + j < NP (1, 3 or
// 6 of them): the dropped ones are below the last bit kept.  The ring's slots hold a 64-wide K block of one piece of both
// operands; a K block's products are issued when its NP slots are there, so two pieces cost three products but only
// twice the operand traffic.
//
// Persistent kernel on CTA pairs (cta_group::2), a 256 x NT tile per pair:
//   warp 0     TMA producer (each CTA brings its 128 rows of A and its NT / 2 columns of B)
//   warp 1     leader: issues the MMAs.  A tensor-memory accumulator is used for `chunk_kb` K blocks and then handed to
//              the epilogue; 512 / NT of them take turns, so that products run while others are collected
//   warps 2-9  epilogue: warp w owns TMEM lanes 32 (w % 4) .. + 31 (rows) and one half of the columns; a thread adds the
//              chunks of its row's NT / 2 columns in registers, rounding to nearest.  The tensor core's own fp32
//              accumulation truncates, which biases a sum of a thousand MMAs by about 2e-5 of its value: short
//              chunks keep that below the last bits that matter (see chunk_of()), and since a tile's last chunk is
//              collected like any other, the epilogue of a tile runs under the products of the next one.
// NT is 256, or 128 where there are too few tiles for the pairs (pick_nt).  Collecting a chunk costs about as much as two K
// blocks: a Newton-Schulz step of eight 2048 x 2048 matrices took 880 us at chunks of two, 780 us at eight, 800 us as they are now.
//
// Outputs leave through boxes of shared memory per warp and TMA stores, which clip at the tensor's edge; ragged M, N
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

constexpr int kTileM = 256;              // rows of a pair's tile
constexpr int kThreads = 320;            // warp 0 producer, warp 1 MMA issuer, warps 2-9 epilogue

// NP: pieces of an operand.  NT: columns of a pair's tile; half of them is a slice, the unit of the row statistics.
template <int NP, int NT>
struct Smem {
  static constexpr int kA = 128 * 128;                             // 128 rows x 64 numbers
  static constexpr int kB = NT / 2 * 128;
  static constexpr int kSlot = kA + kB;
  static constexpr int kSlots = NT == 256 ? 6 : 7;
  static constexpr int kRing = kSlots * kSlot;
  // boxes of an epilogue warp: 32 rows of kBoxRow bytes, kBoxes of them in turn
  static constexpr int kBoxRow = NP == 1 ? 128 : 64;
  static constexpr int kBox = 32 * kBoxRow;
  static constexpr int kBoxes = NP == 1 ? 1 : NT == 256 ? 2 : 3;
  static constexpr int kOut = 8 * kBoxes * kBox;
  static constexpr int kAccs = 512 / NT;
  static constexpr int kBars = 2 * kSlots + 2 * kAccs;
  static constexpr int kTotal = 1024 + kRing + kOut + kBars * 8 + 16;
  static_assert(kTotal <= 227 * 1024, "shared memory budget");
};
constexpr int box_row(int np) { return np == 1 ? 128 : 64; }

enum Epi {
  EPI_F32,        // fp32 C = alpha acc (reduce: C += alpha acc)
  EPI_BF16,       // bf16 C = alpha acc
  EPI_STATS,      // row statistics of exp only
  EPI_STATS_E16,  // statistics, and C = exp(acc - slice maximum) as 16-bit numbers (pack_e16)
  EPI_STATS_F32,  // statistics, and C = fp32 acc
  EPI_PIECES,     // two fp16 pieces of alpha acc + diag I (once or twice, with other factors), optionally mirrored
};

struct Params {
  int m_tiles, n_tiles, batch, splits;   // splits > 1: K is cut, split s writes plane c_z0 + z c_zstep + s
  int num_kb, kb_per_split;
  int chunk_kb;                          // 0: chunk_of()
  int total;                             // tiles of the launch
  int tri;                               // 1: only tiles on or above the diagonal (symmetric C)
  int per, step;                         // tiles of one batch entry and split; 256 / NT
  int fine;                              // EPI_PIECES: 1 cuts the tail's chunks further, see k_order()
  int dominant;                          // where one K block dominates a row's (1) or a column's (2) sum: see k_order()
  int a_box;                             // rows of a box of A's map if not 64 (K-major A with M <= a_box only)
  int n_fast;                            // 1: neighbouring pairs take neighbouring columns, else neighbouring rows
  int a_z0, a_zstep, b_z0, b_zstep;      // plane of batch entry z: z0 + z * zstep (+ piece)
  int c_z0, c_zstep;
  int M, N;
  float alpha;
  const float* alpha_dev;                // EPI_F32, EPI_BF16: further factors of alpha in device memory, one per batch entry, or null
  int reduce;                            // EPI_F32: C += instead of C =
  // row statistics: slice t = column / (NT / 2) of row r at [t * stat_ld + r]
  float* stat_max;                       // slice maximum * log2(e)
  float* stat_sum;                       // sum over the slice of exp(acc - slice maximum)
  int64_t stat_ld, stat_z;               // elements between slices, between batch entries
  const int32_t* labels;                 // [M], label_z apart; the label's logit is written to label_logit[row], and the slice's
  float* label_logit;                    // numbers are those of the other columns
  int64_t label_z;
  // few rows (or null): row-major h [M][dot_d] and W [N][dot_d], dot_hz and dot_wz apart, from which the labels' logits are formed
  // beside the product, see label_dots(); label_lo[row] receives what label_logit[row] leaves over
  const __nv_bfloat16 *dot_h, *dot_w;
  int64_t dot_hz, dot_wz;
  int dot_d;
  float* label_lo;
  unsigned* clear;                       // `batch` words that the launch sets to zero for the next one, or null
  // EPI_PIECES: output i (of n_out) is planes c + 2 i (first piece) and c + 2 i + 1 of the stack
  int n_out;
  float out_alpha[2], out_diag[2];       // out_alpha acc + out_diag on the diagonal (the last output only)
  int mirror;
  int* err;
};

struct Tile { int m, n, split, z; };

__device__ __forceinline__ Tile tile_of(const Params& p, int t) {
  Tile r;
  const int per = p.per;
  const int q = t / per, i = t - q * per;
  r.z = q / p.splits;
  r.split = q - r.z * p.splits;
  if (p.tri) {
    // row block m has the column blocks from its diagonal on: step * m .. n_tiles - 1, step = 256 / NT
    int m = 0, left = i;
    for (int w = p.n_tiles; left >= w; w -= p.step) { left -= w; ++m; }
    r.m = m;
    r.n = m * p.step + left;
  } else if (p.n_fast) {
    r.m = i / p.n_tiles;
    r.n = i - r.m * p.n_tiles;
  } else {
    r.n = i / p.m_tiles;
    r.m = i - r.n * p.m_tiles;
  }
  return r;
}

// The order in which a tile takes its K blocks, and how they are cut into chunks: `first`, first + 1, ... round the end;
// a chunk closes after every chunk_kb blocks, and each of the last `tail` blocks is a chunk of its own.
//
// When A is (nearly) diagonal, one product dominates an element's sum, the one with k = row (dominant = 1; 2: B is, and
// k = column).  Every MMA that follows it in the accumulator truncates it again, a bias that the Newton-Schulz
// iteration amplifies (error of five steps 2.9e-6 at chunks of 2 K blocks, 4.8e-6 at 4, 8.7e-6 at 8).  The blocks with
// the tile's own k therefore come last, each in a chunk of its own, and the others, small sums of mixed signs, first.
// Params::fine: each of the four MMAs of such a block's first pieces has a chunk of its own, because within the block, too, up to three
// MMAs follow the dominant product.
struct KOrder { int first, tail; };
template <int NT>
__device__ __forceinline__ KOrder k_order(const Params& p, const Tile& t) {
  KOrder o{0, 0};
  if (p.dominant != 0) {
    const int width = (p.dominant == 1 ? kTileM : NT) / 64;
    const int from = (p.dominant == 1 ? t.m * kTileM : t.n * NT) / 64;
    const int end = min(from + width, p.num_kb);
    o.tail = max(0, end - from);
    o.first = end == p.num_kb ? 0 : end;
  }
  return o;
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
// The next of a warp's boxes may be written: the bulk store that used it last has read it.
template <int NBOX>
__device__ __forceinline__ void box_free(int lane) {
  if (lane == 0) asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(NBOX - 1) : "memory");
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
// piece u of 16 bytes of this lane's row, as the tensor map's swizzle places it
template <int ROW>
__device__ __forceinline__ uint4* box_piece(uint8_t* box, int lane, int u) {
  return reinterpret_cast<uint4*>(box + lane * ROW + ((ROW == 128 ? u ^ (lane & 7) : u ^ ((lane >> 1) & 3)) << 4));
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<uint32_t*>(&h);
}

// Exponentials, numbers in [0, 1], in 16 bits: they need no sign and no exponent above 0, so there are six bits of exponent and
// ten of mantissa, the precision of fp16 (half a step is 2^-11) down to 2^-62; below, the steps stay 2^-72 (the value is off by
// 2^-63 at most), and zero is zero.  In the bits of an fp32 number that is a subtraction from the exponent and a rounding at
// bit 13; one saturating instruction does both and keeps any other bits (the largest exponential of logits beyond 10^7, NaN)
// inside the 16.  (fp16 itself has 11 bits down to 2^-14 only, 9.7 nats, and nothing below 2^-25.)
constexpr int kE16Bias = 64 << 23;       // subtracted from the bits of an exponential
constexpr float kE16Scale = 18446744073709551616.f;       // 2^64: what unpack_e16() leaves to be multiplied by
__device__ __forceinline__ uint32_t pack_e16(float a, float b) {
  const int x = __viaddmin_s32_relu(__float_as_int(a), 0x1000 - kE16Bias, 0x1FFFFFFF);
  const int y = __viaddmin_s32_relu(__float_as_int(b), 0x1000 - kE16Bias, 0x1FFFFFFF);
  return __byte_perm((uint32_t)x << 3, (uint32_t)y << 3, 0x7632);
}
// the two numbers of a word, divided by kE16Scale (a field of zeros then reads as a number without the implicit bit)
__device__ __forceinline__ float2 unpack_e16(uint32_t w) {
  return make_float2(__uint_as_float((w << 13) & 0x1FFFE000u), __uint_as_float((w >> 3) & 0x1FFFE000u));
}

// The logit of a label is a sum of equal signs where a row is sure of it, which the tensor core's truncation leaves off by 1e-6,
// and with a handful of rows nothing averages the losses.  One warp of a CTA forms it in double while the first tile's products run.
// (Chunks of one K block for all columns instead: a quarter to a third more time.)
__device__ __forceinline__ void label_dots(const Params& p, int lane) {
  for (int i = blockIdx.x; i < p.M * p.batch; i += gridDim.x) {
    const int z = i / p.M, row = i - z * p.M;
    const int y = p.labels[z * p.label_z + row];
    if (y < 0 || y >= p.N) continue;
    const __nv_bfloat16* h = p.dot_h + z * p.dot_hz + (int64_t)row * p.dot_d;
    const __nv_bfloat16* w = p.dot_w + z * p.dot_wz + (int64_t)y * p.dot_d;
    double sum = 0.0;
    if (p.dot_d % 8 == 0) {                  // (rows start on 16-byte boundaries then)
#pragma unroll 4
      for (int k = lane * 8; k < p.dot_d; k += 256) {
        const uint4 a = __ldg(reinterpret_cast<const uint4*>(h + k)), b = __ldg(reinterpret_cast<const uint4*>(w + k));
        const uint32_t u[4] = {a.x, a.y, a.z, a.w}, v[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {        // (products of bf16 numbers are exact in fp32)
          sum += (double)(__uint_as_float(u[e] << 16) * __uint_as_float(v[e] << 16));
          sum += (double)(__uint_as_float(u[e] & 0xFFFF0000u) * __uint_as_float(v[e] & 0xFFFF0000u));
        }
      }
    } else {
#pragma unroll 8
      for (int k = lane; k < p.dot_d; k += 32) sum += (double)(__bfloat162float(h[k]) * __bfloat162float(w[k]));
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) {
      const float hi = (float)sum;
      p.label_logit[z * p.label_z + row] = hi;
      p.label_lo[z * p.label_z + row] = isfinite(hi) ? (float)(sum - (double)hi) : 0.f;
    }
  }
}

template <int NP, int NT, bool F16, bool A_MN, bool B_MN, int EPI>
__global__ void __launch_bounds__(kThreads, 1)
gemm_op_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
               const __grid_constant__ CUtensorMap tmC, const __grid_constant__ CUtensorMap tmCT, const Params p) {
  using L = Smem<NP, NT>;
  constexpr int SLOTS = L::kSlots, ACCS = L::kAccs, HALF = NT / 2;
  constexpr uint32_t IDESC = make_idesc(F16 ? 0u : 1u, A_MN, B_MN, 256, NT);
  constexpr uint32_t TMEM_COLS = 512;

  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint8_t* out_base = smem + L::kRing;
  uint64_t* full = reinterpret_cast<uint64_t*>(out_base + L::kOut);
  uint64_t* empty = full + SLOTS;
  uint64_t* acc_full = empty + SLOTS;          // [ACCS]
  uint64_t* acc_empty = acc_full + ACCS;       // [ACCS] leader's: sixteen epilogue warps of the pair
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_empty + ACCS);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = (int)cluster_ctarank();
  const int pair = (int)(blockIdx.x >> 1), pairs = (int)(gridDim.x >> 1);
  bool failed = false;

  if (threadIdx.x == 0) {
    for (int s = 0; s < SLOTS; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
    for (int s = 0; s < ACCS; ++s) { mbar_init(&acc_full[s], 1); mbar_init(&acc_empty[s], 16); }
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
  if (blockIdx.x == 0 && p.clear != nullptr)
    for (int i = threadIdx.x; i < p.batch; i += kThreads) p.clear[i] = 0u;

  // The loops of warps 0 and 1 run in all lanes (the waits too), so that addresses and descriptors are warp-uniform values;
  // one lane issues.  Slots and accumulators are counted with a place in the ring and the parity of the round.
  if (warp == 0) {
    const bool lead = elect_one();
    const uint64_t pol = l2_policy(0);
    const uint32_t full_leader = map_to_rank(smem_u32(&full[0]), 0);
    int s = 0, round = 0;
    for (int t = pair; t < p.total && !failed; t += pairs) {
      const Tile tl = tile_of(p, t);
      const int k0 = tl.split * p.kb_per_split;
      const int k1 = min(p.num_kb, k0 + p.kb_per_split);
      const int az = p.a_z0 + tl.z * p.a_zstep, bz = p.b_z0 + tl.z * p.b_zstep;
      const int ma = tl.m * kTileM + rank * 128, nb = tl.n * NT + rank * HALF;
      // Boxes wholly outside are left out: zero-filled rows are requests too, all to one place of the L2 (8 rows of 2048 times
      // 32000 took 147 us instead of 36).  What their place holds ends in rows and columns that are not stored.
      auto inside = [](int extent, int from, int most) { return min(max((extent - from + 63) / 64, 0), most); };
      const int a_boxes = inside(p.M, ma, 2), b_boxes = inside(p.N, nb, HALF / 64);
      const uint32_t bytes = (uint32_t)((inside(p.M, tl.m * kTileM, 2) + inside(p.M, tl.m * kTileM + 128, 2)) * p.a_box * 128 +
                                        (inside(p.N, tl.n * NT, HALF / 64) + inside(p.N, tl.n * NT + HALF, HALF / 64)) * 8192);
      const bool whole = a_boxes == 2 && b_boxes == HALF / 64;
      int kb = k0 + k_order<NT>(p, tl).first;
      for (int left = k1 - k0; left > 0 && !failed; --left) {
#pragma unroll
        for (int q = NP - 1; q >= 0; --q) {        // in the order in which the MMAs let go of them
          if (round > 0 && !__all_sync(0xffffffffu, mbar_wait(&empty[s], (round - 1) & 1))) { failed = true; break; }
          if (lead) {
            if (rank == 0) mbar_expect_tx(&full[s], bytes);             // both CTAs'
            const uint32_t bar = full_leader + (uint32_t)(s * 8);
            uint8_t* sa = smem + s * L::kSlot;
            uint8_t* sb = sa + L::kA;
            auto load_a = [&](int c) {
              if (A_MN) tma_load_3d_pair(sa + c * 8192, &tmA, bar, ma + c * 64, kb * 64, az + q, pol);
              else tma_load_3d_pair(sa + c * 8192, &tmA, bar, kb * 64, ma + c * 64, az + q, pol);
            };
            auto load_b = [&](int c) {
              if (B_MN) tma_load_3d_pair(sb + c * 8192, &tmB, bar, nb + c * 64, kb * 64, bz + q, pol);
              else tma_load_3d_pair(sb + c * 8192, &tmB, bar, kb * 64, nb + c * 64, bz + q, pol);
            };
            if (whole) {                               // (unrolled: tests between the loads cost 3 % of a large product)
#pragma unroll
              for (int c = 0; c < 2; ++c) load_a(c);
#pragma unroll
              for (int c = 0; c < HALF / 64; ++c) load_b(c);
            } else {
              for (int c = 0; c < a_boxes; ++c) load_a(c);
              for (int c = 0; c < b_boxes; ++c) load_b(c);
            }
          }
          __syncwarp();
          if (++s == SLOTS) { s = 0; ++round; }
        }
        if (++kb == k1) kb = k0;
      }
    }
    // the releases of the last slots arrive here from the leader's tensor core: wait for them before leaving
    for (int i = 0; i < SLOTS && !failed; ++i) {
      const int uses = round + (i < s ? 1 : 0);
      if (uses > 0 && !__all_sync(0xffffffffu, mbar_wait(&empty[i], (uses - 1) & 1))) failed = true;
    }
    if (failed && lane == 0) atomicExch(p.err, 31);
  } else if (warp == 1) {
    if (rank == 0) {
      const bool lead = elect_one();
      constexpr uint32_t HI = smem_desc_hi(1024);
      const uint32_t a_lo0 = smem_desc_lo(smem_u32(smem), A_MN ? 8192 : 16);
      const uint32_t b_lo0 = smem_desc_lo(smem_u32(smem) + L::kA, B_MN ? 8192 : 16);
      int s = 0, round = 0, acc = 0, acc_round = 0;
      for (int t = pair; t < p.total && !failed; t += pairs) {
        const Tile tl = tile_of(p, t);
        const int k0 = tl.split * p.kb_per_split;
        const int nk = min(p.num_kb, k0 + p.kb_per_split) - k0;
        const int body = nk - k_order<NT>(p, tl).tail;
        int in_chunk = 0;
        for (int kb = 0; kb < nk; ++kb) {
          if (in_chunk == 0 && acc_round > 0 &&
              !__all_sync(0xffffffffu, mbar_wait(&acc_empty[acc], (acc_round - 1) & 1))) { failed = true; break; }
          uint32_t a_lo[NP], b_lo[NP];
          int slot[NP];
          bool got = true;
#pragma unroll
          for (int q = NP - 1; q >= 0; --q) {
            slot[q] = s;
            a_lo[q] = a_lo0 + (uint32_t)(s * (L::kSlot >> 4));
            b_lo[q] = b_lo0 + (uint32_t)(s * (L::kSlot >> 4));
            got = got && mbar_wait(&full[s], round & 1);
            if (++s == SLOTS) { s = 0; ++round; }
          }
          if (!__all_sync(0xffffffffu, got)) { failed = true; break; }
          tc_fence_after_sync();
          const bool fine = EPI == EPI_PIECES && p.fine != 0 && kb >= body;
          const bool last = fine || in_chunk == p.chunk_kb - 1 || kb >= body - 1;
          if (lead) {
            const uint32_t d_tmem = tmem_base + (uint32_t)(acc * NT);
            // small products first; a piece's slot is released after the last product that needs it
            bool begin = in_chunk == 0;
#pragma unroll
            for (int q = NP - 1; q >= 0; --q) {
#pragma unroll
              for (int o = q; o >= 0; --o) {
                if (q + o >= NP) continue;
#pragma unroll
                for (int turn = 0; turn < (q == o ? 1 : 2); ++turn) {
                  const int i = turn == 0 ? q : o, j = turn == 0 ? o : q;
#pragma unroll
                  for (int k = 0; k < 4; ++k) {
                    if (q == 0 && k > 0 && fine) continue;
                    mma_f16_pair_lo(d_tmem, a_lo[i] + (A_MN ? k * 128 : k * 2), b_lo[j] + (B_MN ? k * 128 : k * 2), HI, IDESC,
                                    begin ? 0u : 1u);
                    begin = false;
                  }
                }
              }
              if (q > 0 || !fine) mma_commit_pair(&empty[slot[q]]);
            }
            if (last) mma_commit_pair(&acc_full[acc]);
          }
          __syncwarp();
          ++in_chunk;
          if (last) {
            in_chunk = 0;
            if (++acc == ACCS) { acc = 0; ++acc_round; }
          }
          if (fine) {                        // the other three MMAs of the first pieces
            for (int k = 1; k < 4; ++k) {
              if (acc_round > 0 && !__all_sync(0xffffffffu, mbar_wait(&acc_empty[acc], (acc_round - 1) & 1))) { failed = true; break; }
              tc_fence_after_sync();
              if (lead) {
                mma_f16_pair_lo(tmem_base + (uint32_t)(acc * NT), a_lo[0] + (A_MN ? k * 128 : k * 2), b_lo[0] + (B_MN ? k * 128 : k * 2),
                                HI, IDESC, 0u);
                if (k == 3) mma_commit_pair(&empty[slot[0]]);
                mma_commit_pair(&acc_full[acc]);
              }
              __syncwarp();
              if (++acc == ACCS) { acc = 0; ++acc_round; }
            }
            if (failed) break;
          }
        }
      }
      // both CTAs' epilogues have let go of the last accumulators
      for (int i = 0; i < ACCS && !failed; ++i) {
        const int uses = acc_round + (i < acc ? 1 : 0);
        if (uses > 0 && !__all_sync(0xffffffffu, mbar_wait(&acc_empty[i], (uses - 1) & 1))) failed = true;
      }
      if (failed && lane == 0) atomicExch(p.err, 32);
    }
  } else {
    constexpr int G = HALF / 32;             // groups of 32 columns of a thread
    constexpr int ROW = L::kBoxRow, NBOX = L::kBoxes;
    const int q = warp & 3, cs = (warp - 2) >> 2;
    const uint32_t taddr = tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(cs * HALF);
    uint8_t* boxes = out_base + (warp - 2) * (NBOX * L::kBox);
    int turn = 0;                            // which box is next
    const uint32_t empty_leader = map_to_rank(smem_u32(&acc_empty[0]), 0);
    int buf = 0, round = 0;
    if constexpr (NP == 1 && (EPI == EPI_STATS || EPI == EPI_STATS_E16 || EPI == EPI_STATS_F32)) {
      if (p.dot_h != nullptr && warp == 2) label_dots(p, lane);
    }
    for (int t = pair; t < p.total && !failed; t += pairs) {
      const Tile tl = tile_of(p, t);
      const int k0 = tl.split * p.kb_per_split;
      const int nk = min(p.num_kb, k0 + p.kb_per_split) - k0;
      const int tail = k_order<NT>(p, tl).tail;
      const int chunks = (nk - tail + p.chunk_kb - 1) / p.chunk_kb + tail * (EPI == EPI_PIECES && p.fine != 0 ? 4 : 1);
      uint32_t acc[G][32];
#pragma unroll
      for (int j = 0; j < G; ++j)
#pragma unroll
        for (int i = 0; i < 32; ++i) acc[j][i] = 0u;
      for (int c = 0; c < chunks; ++c) {
        if (!__all_sync(0xffffffffu, mbar_wait(&acc_full[buf], round & 1))) {
          if (lane == 0) atomicExch(p.err, 34);
          failed = true;
          break;
        }
        __syncwarp();
        tc_fence_after_sync();
        const uint32_t at = taddr + (uint32_t)(buf * NT);
        if constexpr (G <= 2) {
          uint32_t r[G][32];
#pragma unroll
          for (int j = 0; j < G; ++j) tmem_ld_32x32(at + j * 32, r[j]);
          tmem_ld_wait();
#pragma unroll
          for (int j = 0; j < G; ++j)
#pragma unroll
            for (int i = 0; i < 32; ++i)
              acc[j][i] = __float_as_uint(__uint_as_float(acc[j][i]) + __uint_as_float(r[j][i]));
        } else {
#pragma unroll
          for (int j = 0; j < 2 * G; ++j) {
            uint32_t r[16];
            tmem_ld_32x16(at + j * 16, r);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              uint32_t& sum = acc[j >> 1][(j & 1) * 16 + i];
              sum = __float_as_uint(__uint_as_float(sum) + __uint_as_float(r[i]));
            }
          }
        }
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive_remote(empty_leader + (uint32_t)(buf * 8));
        __syncwarp();
        if (++buf == ACCS) { buf = 0; ++round; }
      }
      if (failed) break;
      const int wr0 = tl.m * kTileM + rank * 128 + q * 32;       // first row of the warp
      const int row = wr0 + lane;
      const int col0 = tl.n * NT + cs * HALF;
      const int zc = p.c_z0 + tl.z * p.c_zstep + tl.split;
      if (wr0 >= p.M) continue;                                    // nothing of the warp's rows is inside
      auto next_box = [&]() {
        uint8_t* b = boxes + turn * L::kBox;
        turn = turn + 1 == NBOX ? 0 : turn + 1;
        box_free<NBOX>(lane);
        return b;
      };
      if constexpr (EPI == EPI_STATS || EPI == EPI_STATS_E16 || EPI == EPI_STATS_F32) {
        if (col0 + HALF > p.N) {                                   // the ragged end (or all) of the last slices
#pragma unroll
          for (int j = 0; j < G; ++j)
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (col0 + j * 32 + i >= p.N) acc[j][i] = 0xff800000u;
        }
        // A row's label stays out of its statistics: its logit leaves on its own and the combining kernel adds its term, so that
        // 1 - p of a certain row is a sum of small numbers and not what is left of 1.
        if (p.labels != nullptr) {
          const int lab = row < p.M ? p.labels[tl.z * p.label_z + row] - col0 : -1;
          const bool mine = lab >= 0 && lab < HALF && lab + col0 < p.N;
          float zl = 0.f;
#pragma unroll
          for (int j = 0; j < G; ++j) {
            if (!__any_sync(0xffffffffu, mine && lab >> 5 == j)) continue;
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (lab == j * 32 + i) {
                zl = __uint_as_float(acc[j][i]);
                acc[j][i] = 0xff800000u;
              }
          }
          if (mine && p.dot_h == nullptr) p.label_logit[tl.z * p.label_z + row] = zl;
        }
        float mx = -INFINITY;
#pragma unroll
        for (int j = 0; j < G; ++j)
#pragma unroll
          for (int i = 0; i < 32; ++i) mx = fmaxf(mx, __uint_as_float(acc[j][i]));
        constexpr float kLog2e = 1.4426950408889634f;
        // (a slice of nothing but -inf: any finite reference gives the zero terms that it has; a finite maximum's reference
        // stays finite)
        const float ref = mx == -INFINITY ? 0.f : mx < 0.f ? fmaxf(mx * kLog2e, -3.4e38f) : mx * kLog2e;
        if constexpr (EPI == EPI_STATS_F32) {
          // the logits themselves (-inf at the label) leave; the exponentials are only summed
          constexpr int W = ROW / 4;                               // columns of a box
#pragma unroll
          for (int j = 0; j < HALF / W; ++j) {
            if (col0 + j * W >= p.N) continue;
            uint8_t* box = next_box();
#pragma unroll
            for (int u = 0; u < ROW / 16; ++u) {
              const int i = j * W + u * 4;
              *box_piece<ROW>(box, lane, u) =
                  make_uint4(acc[i >> 5][i & 31], acc[i >> 5][(i + 1) & 31], acc[i >> 5][(i + 2) & 31], acc[i >> 5][(i + 3) & 31]);
            }
            box_send(&tmC, box, lane, col0 + j * W, wr0, zc, false);
          }
        }
        float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < G; ++j)
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            const float e = ex2(fmaf(__uint_as_float(acc[j][i]), kLog2e, -ref));
            part[i & 3] += e;
            acc[j][i] = __float_as_uint(e);
          }
        if (row < p.M) {
          const int64_t at = tl.z * p.stat_z + (int64_t)(tl.n * 2 + cs) * p.stat_ld + row;
          p.stat_max[at] = mx == -INFINITY ? -INFINITY : ref;
          p.stat_sum[at] = (part[0] + part[1]) + (part[2] + part[3]);
        }
      }
      if constexpr (EPI == EPI_STATS_E16 || EPI == EPI_BF16) {
        const float alpha = EPI == EPI_BF16 && p.alpha_dev != nullptr ? p.alpha * __ldg(p.alpha_dev + tl.z) : p.alpha;
        constexpr int W = ROW / 2;
#pragma unroll
        for (int j = 0; j < HALF / W; ++j) {
          if (col0 + j * W >= p.N) continue;
          uint8_t* box = next_box();
#pragma unroll
          for (int u = 0; u < ROW / 16; ++u) {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int i = j * W + u * 8 + e * 2;
              const float a = __uint_as_float(acc[i >> 5][i & 31]), b = __uint_as_float(acc[i >> 5][(i + 1) & 31]);
              w[e] = EPI == EPI_BF16 ? pack_bf16(alpha * a, alpha * b) : pack_e16(a, b);
            }
            *box_piece<ROW>(box, lane, u) = make_uint4(w[0], w[1], w[2], w[3]);
          }
          box_send(&tmC, box, lane, col0 + j * W, wr0, zc, false);
        }
      }
      if constexpr (EPI == EPI_F32) {
        const float alpha = p.alpha_dev != nullptr ? p.alpha * __ldg(p.alpha_dev + tl.z) : p.alpha;
        constexpr int W = ROW / 4;
#pragma unroll
        for (int j = 0; j < HALF / W; ++j) {
          if (col0 + j * W >= p.N) continue;
          uint8_t* box = next_box();
#pragma unroll
          for (int u = 0; u < ROW / 16; ++u) {
            const int i = j * W + u * 4;
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = __float_as_uint(alpha * __uint_as_float(acc[i >> 5][(i + e) & 31]));
            *box_piece<ROW>(box, lane, u) = make_uint4(w[0], w[1], w[2], w[3]);
          }
          box_send(&tmC, box, lane, col0 + j * W, wr0, zc, p.reduce != 0);
        }
      }
      if constexpr (EPI == EPI_PIECES) {
        static_assert(EPI != EPI_PIECES || ROW == 64, "boxes of 32 x 32 16-bit numbers");
        const bool flip = p.mirror != 0 && tl.n >= (tl.m + 1) * p.step;          // strictly above the diagonal block
        for (int o = 0; o < p.n_out; ++o) {
          const float alpha_o = p.out_alpha[o];
          const int zp = zc + 2 * o;
          if (p.out_diag[o] != 0.f && row >= col0 && row < col0 + HALF) {
            // + diag I, on the accumulator (only the last output has one, so that it disturbs no other)
            const float d = p.out_diag[o] / alpha_o;
#pragma unroll
            for (int j = 0; j < G; ++j)
#pragma unroll
              for (int i = 0; i < 32; ++i)
                if (row == col0 + j * 32 + i) acc[j][i] = __float_as_uint(__uint_as_float(acc[j][i]) + d);
          }
          __syncwarp();
#pragma unroll
          for (int j = 0; j < G; ++j) {
            const int c0 = col0 + j * 32;
            if (c0 >= p.N) continue;
            // the first pieces of two columns in a word, and what they leave over
            uint32_t hi[16], lo[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const float v0 = alpha_o * __uint_as_float(acc[j][2 * e]);
              const float v1 = alpha_o * __uint_as_float(acc[j][2 * e + 1]);
              const __half2 h = __floats2half2_rn(v0, v1);
              const float2 f = __half22float2(h);
              hi[e] = *reinterpret_cast<const uint32_t*>(&h);
              lo[e] = pack_f16(v0 - f.x, v1 - f.y);
            }
#pragma unroll
            for (int piece = 0; piece < 2; ++piece) {
              uint8_t* box = next_box();
              const uint32_t* w = piece == 0 ? hi : lo;
#pragma unroll
              for (int u = 0; u < 4; ++u)
                *box_piece<ROW>(box, lane, u) = make_uint4(w[4 * u], w[4 * u + 1], w[4 * u + 2], w[4 * u + 3]);
              box_send(&tmC, box, lane, c0, wr0, zp + piece, false);
            }
            if (flip) {
#pragma unroll
              for (int piece = 0; piece < 2; ++piece) {
                uint8_t* box = next_box();
                const uint32_t* w = piece == 0 ? hi : lo;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                  *reinterpret_cast<uint16_t*>(box + 2 * e * 64 + lane * 2) = (uint16_t)w[e];
                  *reinterpret_cast<uint16_t*>(box + (2 * e + 1) * 64 + lane * 2) = (uint16_t)(w[e] >> 16);
                }
                box_send(&tmCT, box, lane, wr0, c0, zp + piece, false);
              }
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
// elements, both 16-byte multiples).  An operand is read in boxes of 64 rows (or box_rows, whole 8s) x 128 bytes with
// the 128-byte swizzle; an output is written in boxes of 32 rows x `row_bytes` (Smem::kBoxRow) with the swizzle of that width, or, transposed, none.
enum MapType { MAP_BF16, MAP_F16, MAP_F32 };
int make_operand_map(CUtensorMap* out, const void* base, MapType type, int64_t rows, int64_t cols, int64_t planes, int64_t ld,
                     int64_t plane, int box_rows = 64);
int make_output_map(CUtensorMap* out, void* base, MapType type, int64_t rows, int64_t cols, int64_t planes, int64_t ld,
                    int64_t plane, int row_bytes, bool transposed = false);
// A bf16 tensor [m][tokens][heads][head_dim] (distances in elements, 16-byte multiples) in boxes of 64 elements of a head x
// box_rows tokens, 128-byte swizzle; coordinates (element, head, token, replica).
int make_heads_map(CUtensorMap* out, const void* base, int64_t head_dim, int64_t heads, int64_t tokens, int64_t m, int64_t row,
                   int64_t replica, int box_rows);
// where a bounded wait that runs out is recorded (one word per device, read by ls_device_status); null on failure
int* device_error_word();

// K blocks per tensor-memory accumulator.  One MMA adds 16 products per element and truncates: 64 MMAs bias a sum of equal
// signs by about 2e-6 of its value, and sums of mixed signs by far less.  One piece: 256 MMAs for results that are rounded to
// bf16 (whose half step is 4e-3), 32 for the row statistics, which leave in fp32, or 16 for a single tile of rows, where the
// bytes of B bound the product and few rows average the losses' errors (2 x 2047 x 50001: 332 us at 32, 369 at 16, loss off by
// 4e-7 and 2e-7; 64 x 32000: 26.5 and 27.1 us).  Two: 16 MMAs of the large product, unless the caller asks for fewer.  Three: 4, for
// 2 % more time than 8, which
// leave the gradient of a cross entropy over 10007 columns off by 6.9e-7, not 2.6e-7.
constexpr int chunk_of(int np, bool stats, int m_tiles) {
  return np == 1 ? (!stats ? 64 : m_tiles > 1 ? 8 : 4) : np == 2 ? 4 : 1;
}
constexpr int kPairs = 74;

// Fills in the tile counts and launches.  p.splits, p.M, p.N, p.batch, p.tri, p.n_fast and the epilogue's fields are the
// caller's; K is the contraction length.
template <int NP, int NT, bool F16, bool A_MN, bool B_MN, int EPI>
cudaError_t launch_nt(const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& c, const CUtensorMap& ct, Params p,
                      int64_t K, cudaStream_t st) {
  auto kern = gemm_op_kernel<NP, NT, F16, A_MN, B_MN, EPI>;
  static uint64_t configured = 0;        // one bit per device
  cudaError_t e = allow_dynamic_smem(kern, (int)Smem<NP, NT>::kTotal, &configured);
  if (e != cudaSuccess) return e;
  p.m_tiles = (p.M + kTileM - 1) / kTileM;
  p.n_tiles = (p.N + NT - 1) / NT;
  p.step = kTileM / NT;
  p.num_kb = (int)((K + 63) / 64);
  if (p.splits < 1) p.splits = 1;
  p.kb_per_split = (p.num_kb + p.splits - 1) / p.splits;
  if (p.dominant != 0 && p.splits > 1) return cudaErrorInvalidValue;     // (the order goes round the whole K)
  p.splits = (p.num_kb + p.kb_per_split - 1) / p.kb_per_split;       // (callers ask pick_cut() first: no change here)
  if (p.chunk_kb == 0) p.chunk_kb = chunk_of(NP, EPI != EPI_F32 && EPI != EPI_BF16, p.m_tiles);
  int64_t per = (int64_t)p.m_tiles * p.n_tiles;
  if (p.tri) {
    per = 0;
    for (int m = 0; m < p.m_tiles; ++m) per += p.n_tiles - m * p.step;
  }
  const int64_t total = per * p.splits * p.batch;
  if (total > 2000000000ll) return cudaErrorInvalidValue;
  if (p.a_box == 0) p.a_box = 64;
  if (p.a_box != 64 && (A_MN || p.M > p.a_box)) return cudaErrorInvalidValue;
  p.per = (int)per;
  p.total = (int)total;
  p.err = device_error_word();
  if (p.err == nullptr) return cudaErrorUnknown;
  const unsigned pairs = (unsigned)(total < kPairs ? total : kPairs);
  return launch_dep(kern, dim3(2 * pairs), dim3(kThreads), Smem<NP, NT>::kTotal, st, 2, a, b, c, ct, p);
}

// How a product is cut: columns of a tile (256 or 128) and parts of the contraction.
struct Cut { int nt, splits; double us; };       // (us: the estimate below)
inline int64_t tile_count(int64_t M, int64_t N, int64_t batch, bool tri, int64_t nt) {
  const int64_t mt = (M + 255) / 256, n = (N + nt - 1) / nt, step = 256 / nt;
  return (tri ? mt * n - step * (mt * (mt - 1) / 2) : mt * n) * batch;
}
// The cut with the least estimated time: rounds of tiles over the pairs at 1.6 GHz, and for several parts 5 us for the
// launch that adds them up and their fp32 sums written and read once at 6 TB/s.  An MMA of 256 x 128 takes about 0.85 of one
// of 256 x 256, not half (its operands come out of shared memory at 64 bytes a clock, 6 KB against 8 KB), so narrow
// tiles pay only where they keep idle pairs busy.  (8192 x 2048 over K = 65536: 256 tiles are four rounds, the last one
// with 34 tiles; two parts are seven half rounds.  The Gram matrices of two 1024 x 4096: 20 tiles; three parts of 22 K blocks.)  At
// least 4 K blocks a part, and always a number of parts that launch() keeps.
inline Cut pick_cut(int64_t M, int64_t N, int64_t batch, bool tri, int64_t K, int np, int most_splits) {
  const int num_kb = (int)((K + 63) / 64);
  const double kb_us = (np == 1 ? 1 : np == 2 ? 3 : 6) * 512 / 1600.0;
  const double results = (double)M * (double)N * (double)batch * (tri ? 0.5 : 1.0);
  Cut best{256, 1, 0.0};
  for (int nt = 256; nt >= 128; nt /= 2) {
    const int64_t tiles = tile_count(M, N, batch, tri, nt);
    for (int s = 1; s <= most_splits && (s == 1 || num_kb / s >= 4); ++s) {
      const int per = (num_kb + s - 1) / s;
      if ((num_kb + per - 1) / per != s) continue;
      const double us = (double)((tiles * s + kPairs - 1) / kPairs) * per * kb_us * (nt == 256 ? 1.0 : 0.85) +
                        (s > 1 ? 5.0 + results * 8.0 * s / 6e6 : 0.0);
      if ((nt == 256 && s == 1) || us < 0.97 * best.us) best = Cut{nt, s, us};
    }
  }
  return best;
}
inline int pick_nt(int64_t M, int64_t N, int64_t batch, bool tri) { return pick_cut(M, N, batch, tri, 64, 1, 1).nt; }
template <int NP, bool F16, bool A_MN, bool B_MN, int EPI>
cudaError_t launch(int nt, const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& c, const CUtensorMap& ct,
                   const Params& p, int64_t K, cudaStream_t st) {
  return nt == 256 ? launch_nt<NP, 256, F16, A_MN, B_MN, EPI>(a, b, c, ct, p, K, st)
                   : launch_nt<NP, 128, F16, A_MN, B_MN, EPI>(a, b, c, ct, p, K, st);
}

}  // namespace gop
}  // namespace ls
