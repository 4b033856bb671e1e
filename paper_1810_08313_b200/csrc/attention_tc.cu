// Attention over packed sequences on the tensor cores: bf16 heads of up to 128 elements (see attention.cuh for the formulas).
//
// Forward.  An SM has two tiles of 128 rows of a head each (rows of S are TMEM lanes), and each passes over the keys in blocks of 128,
// once.  The tensor core works for one tile while the other's softmax runs.  A CTA has
//   a TMA producer: Q, then K and V blocks through a ring
//   a warp for each tile that issues its MMAs: S = Q K^T (operands in shared memory) and O += P V (P in tensor memory)
//   four warps for each tile's softmax, a thread a row: 128 scores in registers, maximum, exponentials, sum, P in bf16 back to
//              tensor memory in two halves, on the first of which PV starts
// Heads of up to 64: a CTA has one tile, and the SM two CTAs, of which one starts and ends while the other works (16 heads of 64,
// two tiles a CTA: 9 % longer for 8192 rows and for 23 packed sequences).  P has a place of its own, and S of the next block is issued
// as soon as this one's is in registers.
// Larger heads: a CTA has both tiles, 256 consecutive rows, and they share every K and V block, which one CTA a tile would draw from
// the L2 faster than it gives them (64 KB a block, twice in the 1700 cycles that two softmaxes take).  S and O fill the tensor memory,
// P takes the place of S, and S of a block is issued when the PV before it is done.  So the two tiles have to stay half a block
// apart: S of a tile waits until the other one is past its maxima.  (16384 rows of 16 heads of 128: without, both end in step, 5 %
// longer; with two threads a row, and twice the warps, 7 %.)
// O stays in tensor memory over all blocks and is rescaled only where a row's maximum has grown by more than 2^8 since its
// reference was taken: P then lies below 2^8 instead of 1, which costs bf16 and fp32 no precision, and most blocks need no
// pass over O.  P is rounded to bf16 (at most 2^-8 of each term, signs at random), its sum is taken before the rounding:
// out is off by 1.8e-3 of its norm, 1.66e-3 of which its own rounding to bf16 is.
// Exponentials are the special-function unit's, 1024 cycles a tile and block.  (A polynomial on the FMA units for three of 16 gains
// nothing, every instruction of a softmax thread being on the critical path: 16384 rows of 16 heads of 128 1011 to 1015 us with
// it, 1009 to 1018 without, 8192 rows of 16 heads of 64 239 and 230, in turn.)
// Bound by the softmax of a tile, 1500 to 1700 cycles a block of the SM (the MMAs take 510 with heads of 64 and 1020 with 128), and in long
// calls by the clock under the power cap: 16384 rows of 16 heads of 128 take 930 to 1070 us with the clock (1.18 to 1.03
// PFLOP/s), 23 packed sequences in 8191 rows of 16 heads of 64 48 to 51 us, with 5700 of a CTA's 18000 cycles before its first block and
// behind its last one.
#include "attention.cuh"

namespace ls {
namespace attn {
namespace {

using namespace ptx;

constexpr int kB = 128;                  // rows of a tile, keys of a block

template <int HD>
struct Fwd {
  static constexpr bool kShared = HD == 128;                // P in the place of S
  static constexpr int kTiles = HD == 128 ? 2 : 1;          // of 128 rows
  static constexpr int kTile = kB * HD * 2;                 // bytes: HD / 64 panels of 128 rows x 128 bytes
  static constexpr int kSlots = 2;                          // of a K and a V block
  static constexpr int kRing = kTiles * kTile;              // offset of the ring, behind Q
  static constexpr int kBars = kRing + kSlots * 2 * kTile;
  static constexpr int kTotal = 1024 + kBars + (2 * kSlots + 14) * 8 + 16;
  // TMEM columns: S, 128 a tile, then O (tile x: + x HD); P, 64 columns, in the place of S, or behind O where that ends early
  static constexpr uint32_t kColumns = kTiles * 256, kO = kTiles * kB, kP = kShared ? 0 : kO + kTiles * HD, kPStep = kShared ? kB : 64;
  static constexpr int kThreads = 32 * (1 + 5 * kTiles), kPerSm = HD == 128 ? 1 : 2;
};

struct FwdMaps { CUtensorMap q, k, v; };

__device__ __forceinline__ float ex2(float x) { return gop::ex2(x); }
__device__ __forceinline__ uint32_t pack2(float a, float b) { return gop::pack_bf16(a, b); }

__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// Of 32 columns, a bit for each one in [from, to].
__device__ __forceinline__ uint32_t visible(int from, int to) {
  return (from > 31 ? 0u : from > 0 ? 0xffffffffu << from : 0xffffffffu) & (to < 0 ? 0u : to < 31 ? (2u << to) - 1 : 0xffffffffu);
}

// key blocks [lo, hi] that the tile of rows from r0 on needs (lo > hi: none)
struct Span { int lo, hi; };
__device__ __forceinline__ Span key_blocks(const Bounds& b, int r0) {
  if (r0 >= b.tokens) return Span{1, 0};
  return Span{b.first_key(r0) / kB, r0 / kB};
}

// Operands are tiles of 128 rows in panels of 64 columns (128 bytes a row, 128-byte swizzle, a panel 16 KB), given by the low words
// of their descriptors: K-major (row = M or N) or MN-major (row = K).
constexpr uint32_t kDescHi = smem_desc_hi(1024);
// (In a cluster, a shared-memory address has the CTA's rank above its 18 bits, where a descriptor has the distance of panels.)
__device__ __forceinline__ uint32_t k_major(uint32_t addr) { return smem_desc_lo(addr & 0x3FFFF, 16); }
__device__ __forceinline__ uint32_t mn_major(uint32_t addr) { return smem_desc_lo(addr & 0x3FFFF, kB * 128); }
// D = A B^T, both K-major, `ksteps` of 16
template <int HD>
__device__ __forceinline__ void product_ss(bool lead, uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, int ksteps) {
#pragma unroll
  for (int k = 0; k < HD / 16; ++k) {
    const uint32_t off = (k >> 2) * (kB * 128 / 16) + (k & 3) * 2;
    mma_f16_if(lead && k < ksteps, d, a + off, b + off, kDescHi, idesc, k > 0);
  }
}
// D += A B, 64 columns of A in bf16 in tensor memory, B their 64 rows, MN-major
__device__ __forceinline__ void product_ts(bool lead, uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool add) {
#pragma unroll
  for (int k = 0; k < 4; ++k) mma_f16_ts_if(lead, d, a + k * 8, b + k * (2048 / 16), kDescHi, idesc, add || k > 0);
}
constexpr uint32_t kHalfRows = 4 * 2048 / 16;              // from the first 64 rows of an MN-major tile to the others

// A bounded wait in a loop whose lanes stay together: every lane waits, and the warp looks at `ok` once a round.  After one that
// ran out no other one waits.
__device__ __forceinline__ void wait(uint64_t* bar, uint32_t parity, bool& ok) {
  if (!mbar_wait(bar, parity, ok ? kSpinLimit : 0)) ok = false;
}

// A tile of 128 rows (tokens) of a head, `panels` of 64 elements.
__device__ __forceinline__ void load_tile(const CUtensorMap* m, uint8_t* dst, uint64_t* bar, int panels, int head, int token, int rep, uint64_t pol) {
  mbar_expect_tx(bar, panels * kB * 128);
  for (int c = 0; c < panels; ++c) tma_load_4d_hint(dst + c * kB * 128, m, bar, c * 64, head, token, rep, pol);
}

// COLS columns from c0 on of this lane's row of a result in tensor memory, times `by`, in bf16 to `row` (of head_dim elements, or null).
// Returns whether they are finite; `any`: there is a result; `zero`: zeros instead.  (Rows leave from registers: by way of
// shared memory and a bulk store the end of a tile took 1000 cycles more, which nothing else runs under.)
template <int COLS>
__device__ __forceinline__ bool result_row(uint32_t ta, int c0, int cols, bool any, bool zero, float by, __nv_bfloat16* row, int head_dim) {
  bool fine = true;
#pragma unroll
  for (int g = 0; g < COLS; g += 32) {
    const int c = c0 + g;
    uint32_t o[32];
    if (c < cols && any) {
      tmem_ld_32x32(ta + c, o);
      tmem_ld_wait();
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (c + u * 8 >= head_dim) continue;
      uint32_t w[4] = {0u, 0u, 0u, 0u};
      if (any && !zero) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x = __uint_as_float(o[u * 8 + 2 * e]) * by, y = __uint_as_float(o[u * 8 + 2 * e + 1]) * by;
          fine = fine && fabsf(x) < INFINITY && fabsf(y) < INFINITY;
          w[e] = pack2(x, y);
        }
      }
      if (row != nullptr) *reinterpret_cast<uint4*>(row + c + u * 8) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
  return fine;
}

template <int HD>
__global__ void __launch_bounds__(Fwd<HD>::kThreads, Fwd<HD>::kPerSm)
attention_tc_kernel(const __grid_constant__ FwdMaps maps, const __grid_constant__ Args a) {
  using L = Fwd<HD>;
  constexpr int SLOTS = L::kSlots, TILES = L::kTiles;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + L::kBars);
  uint64_t* empty = full + SLOTS;
  uint64_t* q_full = empty + SLOTS;      // [2]
  uint64_t* s_full = q_full + 2;         // [2] S of the next block is there, and the PV before it done
  uint64_t* p_half = s_full + 2;         // [half][tile] four warps have left P of the first 64 keys, of the others
  uint64_t* past_max = p_half + 4;       // [2] four warps have a block's maxima
  uint64_t* s_free = past_max + 2;       // [2] four warps have S in registers
  uint64_t* o_done = s_free + 2;        // [2] a PV is done
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(o_done + 2);

  // the rows with the most keys first; heads of a group beside each other
  const int tiles = (int)((a.tokens + TILES * kB - 1) / (TILES * kB));
  const int head = blockIdx.x % a.heads, rest = blockIdx.x / a.heads, rep = rest % a.m;
  const int r0 = (tiles - 1 - rest / a.m) * TILES * kB;
  const int kvh = head / (a.heads / a.kv_heads);
  const int panels = (a.head_dim + 63) / 64;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  bool failed = false;
  if (threadIdx.x == 0) {
    for (int s = 0; s < SLOTS; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], TILES); }
    for (int x = 0; x < 2; ++x) { mbar_init(&q_full[x], 1); mbar_init(&s_full[x], 1); mbar_init(&p_half[x], 4); mbar_init(&p_half[2 + x], 4); mbar_init(&past_max[x], 4); mbar_init(&s_free[x], 4); mbar_init(&o_done[x], 1); }
    fence_mbar_init();
    prefetch_tmap(&maps.k);
    prefetch_tmap(&maps.v);
    // Q is on its way while the tensor memory is allocated and the boundaries are read
    fence_proxy_async_smem();
    grid_dep_wait();
    for (int x = 0; x < TILES; ++x)
      if (r0 + x * kB < a.tokens) load_tile(&maps.q, smem + x * L::kTile, &q_full[x], panels, head, r0 + x * kB, rep, l2_policy(0));
  }
  __syncwarp();
  if (warp == 1) {
    tmem_alloc(tmem_slot, L::kColumns);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = *tmem_slot;
  grid_dep_wait();
  grid_dep_launch();

  const Bounds bounds(a, rep);
  const Span sa = key_blocks(bounds, r0);
  Span sb = TILES == 2 ? key_blocks(bounds, r0 + kB) : Span{1, 0};
  // The second tile never starts before the first one, as its rows lie behind.  Boundaries that do not ascend may say otherwise; the
  // hand-over below counts on it: the pair passes over the blocks from the first tile's on, and each tile waits for the other's maxima.
  if (sa.lo <= sa.hi) sb.lo = max(sb.lo, sa.lo);
  const bool has_a = sa.lo <= sa.hi, has_b = sb.lo <= sb.hi;
  const int lo = has_a ? sa.lo : sb.lo, hi = has_b ? sb.hi : has_a ? sa.hi : lo - 1;

  if (warp == 0) {
    const bool lead = elect_one();
    const uint64_t pol = l2_policy(0);
    // slot t: K of block t and V of the block before
    int s = 0, round = 0;
    for (int j = lo; j <= hi + 1 && lo <= hi && !failed; ++j) {
      if (round > 0 && !__all_sync(0xffffffffu, mbar_wait(&empty[s], (round - 1) & 1))) { failed = true; break; }
      if (lead) {
        uint8_t* dst = smem + L::kRing + s * 2 * L::kTile;
        mbar_expect_tx(&full[s], ((j <= hi) + (j > lo)) * panels * kB * 128);
        for (int c = 0; c < panels && j <= hi; ++c)
          tma_load_4d_hint(dst + c * kB * 128, &maps.k, &full[s], c * 64, kvh, j * kB, rep, pol);
        for (int c = 0; c < panels && j > lo; ++c)
          tma_load_4d_hint(dst + L::kTile + c * kB * 128, &maps.v, &full[s], c * 64, kvh, (j - 1) * kB, rep, pol);
      }
      __syncwarp();
      if (++s == SLOTS) { s = 0; ++round; }
    }
    // Q that no product needs, and the releases of the last slots, arrive here: wait for them before leaving
    for (int x = 0; x < TILES; ++x)
      if (r0 + x * kB < a.tokens && !(x == 0 ? has_a : has_b) && !__all_sync(0xffffffffu, mbar_wait(&q_full[x], 0))) failed = true;
    for (int i = 0; i < SLOTS && !failed; ++i) {
      const int uses = round + (i < s ? 1 : 0);
      if (uses > 0 && !__all_sync(0xffffffffu, mbar_wait(&empty[i], (uses - 1) & 1))) failed = true;
    }
    if (failed && lane == 0) atomicExch(a.err, 41);
  } else if (warp <= TILES) {
    const int x = warp - 1;
    const bool lead = elect_one();
    const int ksteps = (a.head_dim + 15) / 16;
    const uint32_t idesc_s = make_idesc(1, false, false, kB, kB);
    const uint32_t idesc_o = make_idesc(1, false, true, kB, (uint32_t)ksteps * 16);
    constexpr uint32_t T = L::kTile / 16;
    const uint32_t q_lo = k_major(smem_u32(smem)) + x * T, k_lo = k_major(smem_u32(smem) + L::kRing);
    const uint32_t v_lo = mn_major(smem_u32(smem) + L::kRing + L::kTile);
    const uint32_t ts = tmem + x * kB, tp = tmem + L::kP + x * L::kPStep, to = tmem + L::kO + x * HD;
    const int from = x == 0 ? sa.lo : sb.lo, upto = x == 0 ? sa.hi : sb.hi;
    bool ok = true;
    if (from <= upto) wait(&q_full[x], 0, ok);
    int s = 0, round = 0;
    for (int j = lo; j <= hi + 1 && lo <= hi; ++j) {
      const uint32_t turn = (uint32_t)(j - 1 - from) & 1;
      const bool pv = j > from && j <= upto + 1, qk = j >= from && j <= upto;
      wait(&full[s], round & 1, ok);     // (a slot that this tile does not need is let go of in its turn all the same)
      auto scores = [&]() {
        tc_fence_after_sync();
        product_ss<HD>(lead, ts, q_lo, k_lo + s * 2 * T, idesc_s, ksteps);
        mma_commit_if(lead, &s_full[x]);
      };
      if (!L::kShared && qk) {
        if (j > from) wait(&s_free[x], turn, ok);
        scores();
      }
      if (pv) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          wait(&p_half[2 * h + x], turn, ok);
          tc_fence_after_sync();
          product_ts(lead, to, tp + h * 32, v_lo + s * 2 * T + h * kHalfRows, idesc_o, j - 1 > from || h > 0);
        }
        mma_commit_if(lead, &o_done[x]);
      }
      if (L::kShared && qk) {
        // S goes where P lies: the product that reads it has to be complete (products of other shapes or accumulators are not
        // known to keep their order)
        if (pv) wait(&o_done[x], turn, ok);
        // the other tile is past its maximum: its exponentials and this product run together
        const int b = x == 1 ? j : j - 1, b_from = x == 1 ? sa.lo : sb.lo, b_upto = x == 1 ? sa.hi : sb.hi;
        if (b >= b_from && b <= b_upto) wait(&past_max[1 - x], (uint32_t)(b - b_from) & 1, ok);
        scores();
      }
      mma_commit_if(lead, &empty[s]);
      if (++s == SLOTS) { s = 0; ++round; }
      if (!__all_sync(0xffffffffu, ok)) { failed = true; break; }
    }
    if (failed && lane == 0) atomicExch(a.err, 42);
  } else {
    const int x = (warp - 1 - TILES) >> 2, q = warp & 3;
    const Span sp = x == 0 ? sa : sb;
    const int row = r0 + x * kB + q * 32 + lane;
    int start, end;
    bounds.rows(r0 + x * kB + q * 32, &start, &end);
    const uint32_t ts = tmem + ((uint32_t)(q * 32) << 16) + x * kB;
    const uint32_t to = tmem + ((uint32_t)(q * 32) << 16) + L::kO + x * HD;
    const uint32_t tp = tmem + ((uint32_t)(q * 32) << 16) + L::kP + x * L::kPStep;
    const float scale2 = a.scale * kLog2e;
    const int cols = (a.head_dim + 15) / 16 * 16;
    float top = -INFINITY, sum = 0.f;    // the reference of the exponentials (a product, not scaled), and their sum
    bool ok = true;
    for (int j = sp.lo; j <= sp.hi; ++j) {
      wait(&s_full[x], (j - sp.lo) & 1, ok);
      tc_fence_after_sync();
      // columns [from, to_col] are visible; one bit each in a mask of 32
      const int from = start - j * kB, to_col = row - j * kB;
      const bool cut = __any_sync(0xffffffffu, from > 0 || to_col < kB - 1);
      auto hide = [&](int c, uint32_t (&v)[32]) {
        const uint32_t seen = visible(from - c * 32, to_col - c * 32);
        if (__all_sync(0xffffffffu, seen == 0xffffffffu)) return;
#pragma unroll
        for (int i = 0; i < 32; ++i)
          if ((seen >> i & 1) == 0) v[i] = 0xff800000u;
      };
      uint32_t s[4][32];
#pragma unroll
      for (int c = 0; c < 4; ++c) tmem_ld_32x32(ts + c * 32, s[c]);
      tmem_ld_wait();
      if (!L::kShared) {
        tc_fence_before_sync();
        __syncwarp();
        mbar_arrive_if(lane == 0, &s_free[x]);
      }
      if (__builtin_expect(cut, 0)) {
#pragma unroll
        for (int c = 0; c < 4; ++c) hide(c, s[c]);
      }
      // four chains of three-input maxima: one would take them one after another.  A NaN stays.
      float m4[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float m = max3(__uint_as_float(s[0][e]), __uint_as_float(s[0][e + 4]), __uint_as_float(s[0][e]));
#pragma unroll
        for (int i = 8; i < 128; i += 8) m = max3(m, __uint_as_float(s[i >> 5][(i & 31) + e]), __uint_as_float(s[i >> 5][(i & 31) + 4 + e]));
        m4[e] = m;
      }
      const float most = max3(max3(m4[0], m4[1], m4[2]), m4[3], m4[3]);
      if (L::kShared) {
        __syncwarp();
        mbar_arrive_if(lane == 0, &past_max[x]);
      } else if (j > sp.lo) {            // (PV of the block before is long done: O may be rescaled, and P written)
        wait(&o_done[x], (j - 1 - sp.lo) & 1, ok);
        tc_fence_after_sync();
      }
      // (top = -inf: the difference is infinite, and the factor zero; a NaN goes on into the reference)
      const bool far = !((most - top) * scale2 <= 8.f) && !(most == -INFINITY);
      if (__builtin_expect(__any_sync(0xffffffffu, far), 0)) {
        const float next = max3(most, top, top);
        const float keep = next == top ? 1.f : ex2((top - next) * scale2);
        top = next;
        sum *= keep;
        if (j > sp.lo) {
          for (int c = 0; c < cols; c += 16) {
            uint32_t o[16];
            tmem_ld_32x16(to + c, o);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * keep);
            tmem_st_32x16(to + c, o);
          }
        }
      }
      const float ref = top == -INFINITY ? 0.f : top * scale2;
      const uint64_t by2 = two(scale2, scale2), ref2 = two(-ref, -ref);
      uint64_t part[2] = {0, 0};
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        uint32_t p[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const uint64_t t = fma2(two(s[c][2 * i], s[c][2 * i + 1]), by2, ref2);
          float2 e = parts(t);
          e.x = ex2(e.x);
          e.y = ex2(e.y);
          part[i & 1] = add2(part[i & 1], two(e.x, e.y));
          p[i] = pack2(e.x, e.y);
        }
        if (c == 2) {                      // PV may start with the first half of the keys, whose stores are done by now
          tmem_st_wait();
          tc_fence_before_sync();
          __syncwarp();
          mbar_arrive_if(lane == 0, &p_half[x]);
        }
        tmem_st_32x16(tp + c * 16, p);
        if (c == 3) {
          tmem_st_wait();
          tc_fence_before_sync();
          __syncwarp();
          mbar_arrive_if(lane == 0, &p_half[2 + x]);
        }
      }
      const float2 total = parts(add2(part[0], part[1]));
      sum += total.x + total.y;
      if (!__all_sync(0xffffffffu, ok)) { failed = true; break; }
    }
    const bool none = start > row;       // in no sequence, or behind the tensor
    if (sp.lo <= sp.hi && !failed) {
      if (!__all_sync(0xffffffffu, mbar_wait(&o_done[x], (sp.hi - sp.lo) & 1))) failed = true;
      __syncwarp();
      tc_fence_after_sync();
    }
    if (failed) {
      if (lane == 0) atomicExch(a.err, 43);
    } else if (r0 + x * kB + q * 32 < a.tokens) {
      // (scores with a NaN or +inf, or of -inf only, have no softmax)
      const bool has = fabsf(top) < INFINITY;
      const float by = none ? 0.f : has ? 1.f / sum : NAN;
      __nv_bfloat16* dst = row < a.tokens ? head_ptr<__nv_bfloat16>(a.out, rep, head, a.head_dim) + row * a.out.row : nullptr;
      const bool fine = result_row<HD>(to, 0, cols, sp.lo <= sp.hi, none, by, dst, a.head_dim);
      if (row < a.tokens)
        a.lse[((int64_t)rep * a.heads + head) * a.tokens + row] = none ? 0.f : has ? fmaf(top * scale2, kLn2, logf(sum)) : top;
      __syncwarp();
      const uint32_t bad = __ballot_sync(0xffffffffu, !none && has && !fine);
      __syncwarp();
      if (bad != 0u) forward_rows<__nv_bfloat16, HD / 32>(a, rep, head, r0 + x * kB + q * 32, bad);
    }
    tc_fence_before_sync();
  }
  __syncwarp();
  if (failed) {
    // a wait ran out: give the loads in flight time to land before the shared memory is released
    const long long t0 = clock64();
    while (clock64() - t0 < 4000000ll) {}
  }
  __syncthreads();
  if (warp == 1) {
    tc_fence_after_sync();
    tmem_dealloc(tmem, L::kColumns);
  }
}

// ---- backward ----------------------------------------------------------------------------------------------------
//
// Two kernels, so that no sum depends on an order of arrival and dq needs no fp32 copy in memory: seven products of a block
// instead of five, scores and exponentials twice.  Both have a producer warp, a warp that issues the MMAs, and eight warps for
// the elements, two a TMEM quadrant: half 0 has the columns 0-63 of a tile, half 1 the others.  Two documents in 8192 rows of 32
// heads of 128 on 8: 486 and 522 us, 1.19 PFLOP/s of the eight products of what is visible, at the power cap; 9 sequences in 2 x 4095 rows of 8
// heads of 96: 54 and 57 us.

constexpr int kBwdThreads = 320;

// the named barrier of the eight element warps
__device__ __forceinline__ void elements_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

// dq, a tile of 128 rows of one head: S = Q K^T and dP = dO V^T of the next block run while the elements of this one become
// dS = P (dP - D), and dq += dS K follows.  S and dP are free as soon as they are in registers.  A row's dS add up to zero, so what
// its keys have in common cancels, but not in the roundings of dS: it goes to the product in two bf16 pieces (2^-17 of each
// term; with one, dq was off by 2.65e-3 of its norm, 1.66e-3 of which its own rounding is).  D is formed here from dout and
// out, and left for the other kernel.
template <int HD>
struct Dq {
  static constexpr int kTile = kB * HD * 2;
  static constexpr int kK = 3, kV = 2;                      // slots
  static constexpr int kBars = (2 + kK + kV) * kTile;       // behind Q, dO, the K and V slots
  static constexpr int kTotal = 1024 + kBars + kB * 4 + 16 + (2 * kK + 2 * kV + 8) * 8 + 16;
  static constexpr uint32_t kS = 0, kP = 128, kO = 256, kDs = 384;     // (dS: 64 columns of first pieces, 64 of second ones)
};
struct DqMaps { CUtensorMap q, dout, k, v; };

template <int HD>
__global__ void __launch_bounds__(kBwdThreads, 1)
attention_dq_tc_kernel(const __grid_constant__ DqMaps maps, const __grid_constant__ Args a) {
  using L = Dq<HD>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  float* dots = reinterpret_cast<float*>(smem + L::kBars);           // [128]
  uint32_t* bad = reinterpret_cast<uint32_t*>(dots + kB);            // [4]
  uint64_t* k_full = reinterpret_cast<uint64_t*>(bad + 4);
  uint64_t* k_empty = k_full + L::kK;
  uint64_t* v_full = k_empty + L::kK;
  uint64_t* v_empty = v_full + L::kV;
  uint64_t* q_full = v_empty + L::kV;    // [2] Q, dO
  uint64_t* s_full = q_full + 2;         // S and dP of a block
  uint64_t* s_free = s_full + 1;         // eight warps have them in registers
  uint64_t* ds_ready = s_free + 1;       // eight warps have left dS
  uint64_t* done = ds_ready + 1;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(done + 1);
  uint8_t* sk = smem + 2 * L::kTile;
  uint8_t* sv = sk + L::kK * L::kTile;

  const int tiles = (int)((a.tokens + kB - 1) / kB);
  const int head = blockIdx.x % a.heads, rest = blockIdx.x / a.heads, rep = rest % a.m;
  const int r0 = (tiles - 1 - rest / a.m) * kB;
  const int kvh = head / (a.heads / a.kv_heads);
  const int panels = (a.head_dim + 63) / 64, ksteps = (a.head_dim + 15) / 16, cols = ksteps * 16;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  bool failed = false;
  if (threadIdx.x == 0) {
    for (int i = 0; i < L::kK; ++i) { mbar_init(&k_full[i], 1); mbar_init(&k_empty[i], 1); }
    for (int i = 0; i < L::kV; ++i) { mbar_init(&v_full[i], 1); mbar_init(&v_empty[i], 1); }
    mbar_init(&q_full[0], 1);
    mbar_init(&q_full[1], 1);
    mbar_init(s_full, 1);
    mbar_init(s_free, 8);
    mbar_init(ds_ready, 8);
    mbar_init(done, 1);
    fence_mbar_init();
    for (int i = 0; i < 4; ++i) bad[i] = 0u;
    prefetch_tmap(&maps.k);
    prefetch_tmap(&maps.v);
    // Q and dO are on their way while the tensor memory is allocated and the boundaries are read
    fence_proxy_async_smem();
    grid_dep_wait();
    load_tile(&maps.q, smem, &q_full[0], panels, head, r0, rep, l2_policy(0));
    load_tile(&maps.dout, smem + L::kTile, &q_full[1], panels, head, r0, rep, l2_policy(0));
  }
  __syncwarp();
  if (warp == 1) {
    tmem_alloc(tmem_slot, 512);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = *tmem_slot;
  grid_dep_wait();
  grid_dep_launch();

  const Bounds bounds(a, rep);
  const Span sp = key_blocks(bounds, r0);
  const int n = sp.hi - sp.lo + 1;       // blocks (none: n <= 0)

  if (warp == 0) {
    const bool lead = elect_one();
    const uint64_t pol = l2_policy(0);
    for (int i = 0; i < n && !failed; ++i) {
      const int ks = i % L::kK, vs = i % L::kV;
      if (i >= L::kK && !__all_sync(0xffffffffu, mbar_wait(&k_empty[ks], (i / L::kK - 1) & 1))) { failed = true; break; }
      if (lead) load_tile(&maps.k, sk + ks * L::kTile, &k_full[ks], panels, kvh, (sp.lo + i) * kB, rep, pol);
      __syncwarp();
      if (i >= L::kV && !__all_sync(0xffffffffu, mbar_wait(&v_empty[vs], (i / L::kV - 1) & 1))) { failed = true; break; }
      if (lead) load_tile(&maps.v, sv + vs * L::kTile, &v_full[vs], panels, kvh, (sp.lo + i) * kB, rep, pol);
      __syncwarp();
    }
    // tiles that no product needs, and the releases of the last slots, arrive here: wait for them before leaving
    for (int i = 0; i < 2; ++i)
      if (n <= 0 && !__all_sync(0xffffffffu, mbar_wait(&q_full[i], 0))) failed = true;
    for (int i = 0; i < L::kK && i < n && !failed; ++i)
      if (!__all_sync(0xffffffffu, mbar_wait(&k_empty[i], ((n - 1 - i) / L::kK) & 1))) failed = true;
    for (int i = 0; i < L::kV && i < n && !failed; ++i)
      if (!__all_sync(0xffffffffu, mbar_wait(&v_empty[i], ((n - 1 - i) / L::kV) & 1))) failed = true;
    if (failed && lane == 0) atomicExch(a.err, 44);
  } else if (warp == 1) {
    const bool lead = elect_one();
    const uint32_t idesc_s = make_idesc(1, false, false, kB, kB);
    const uint32_t idesc_o = make_idesc(1, false, true, kB, (uint32_t)cols);
    constexpr uint32_t T = L::kTile / 16;
    const uint32_t qb = k_major(smem_u32(smem)), gb = qb + T, kb = k_major(smem_u32(sk)), vb = k_major(smem_u32(sv)), kmn = mn_major(smem_u32(sk));
    bool ok = true;
    auto scores = [&](int i) {           // S and dP of block i
      const int ks = i % L::kK, vs = i % L::kV;
      wait(&k_full[ks], (i / L::kK) & 1, ok);
      if (i == 0) wait(&q_full[0], 0, ok);
      tc_fence_after_sync();
      product_ss<HD>(lead, tmem + L::kS, qb, kb + ks * T, idesc_s, ksteps);
      wait(&v_full[vs], (i / L::kV) & 1, ok);
      if (i == 0) wait(&q_full[1], 0, ok);
      tc_fence_after_sync();
      product_ss<HD>(lead, tmem + L::kP, gb, vb + vs * T, idesc_s, ksteps);
      mma_commit_if(lead, s_full);
      mma_commit_if(lead, &v_empty[vs]);
    };
    if (n > 0) scores(0);
    for (int i = 0; i < n; ++i) {
      if (i + 1 < n) {
        wait(s_free, i & 1, ok);
        scores(i + 1);
      }
      wait(ds_ready, i & 1, ok);
      tc_fence_after_sync();
      const uint32_t ds = tmem + L::kDs, k0 = kmn + (i % L::kK) * T;
#pragma unroll
      for (int e = 0; e < 4; ++e)          // the small pieces first
        product_ts(lead, tmem + L::kO, ds + (e < 2 ? 64 : 0) + (e & 1) * 32, k0 + (e & 1) * kHalfRows, idesc_o, i > 0 || e > 0);
      mma_commit_if(lead, &k_empty[i % L::kK]);
      mma_commit_if(lead && i == n - 1, done);
      if (!__all_sync(0xffffffffu, ok)) break;
    }
    if (!__all_sync(0xffffffffu, ok)) failed = true;
    if (failed && lane == 0) atomicExch(a.err, 45);
  } else {
    const int half = (warp - 2) >> 2, q = warp & 3, r = q * 32 + lane, row = r0 + r;
    const uint32_t lanes = (uint32_t)(q * 32) << 16;
    const int64_t stat = ((int64_t)rep * a.heads + head) * a.tokens + row;
    int start, end;
    bounds.rows(r0 + q * 32, &start, &end);
    const float nl2 = row < a.tokens ? -a.lse[stat] * kLog2e : 0.f;
    {
      // D of 16 rows a warp, a row's 16-byte pieces in neighbouring lanes (a lane to a row, each of its loads would touch 32 lines,
      // and the first block waited 4500 cycles for D)
      constexpr int N = HD / 8, ROWS = 32 / N;
      const int piece = lane % N, e = piece * 8;
      const __nv_bfloat16* g = head_ptr<const __nv_bfloat16>(a.dout, rep, head, a.head_dim) + e;
      const __nv_bfloat16* o = head_ptr<const __nv_bfloat16>(a.out, rep, head, a.head_dim) + e;
      uint4 x[16 / ROWS], y[16 / ROWS];
#pragma unroll
      for (int i = 0; i < 16 / ROWS; ++i) {
        const int64_t at = r0 + q * 32 + half * 16 + i * ROWS + lane / N;
        const bool in = at < a.tokens && e < a.head_dim;
        x[i] = in ? __ldg(reinterpret_cast<const uint4*>(g + at * a.dout.row)) : make_uint4(0u, 0u, 0u, 0u);
        y[i] = in ? __ldg(reinterpret_cast<const uint4*>(o + at * a.out.row)) : make_uint4(0u, 0u, 0u, 0u);
      }
#pragma unroll
      for (int i = 0; i < 16 / ROWS; ++i) {
        const uint32_t u[4] = {x[i].x, x[i].y, x[i].z, x[i].w}, v[4] = {y[i].x, y[i].y, y[i].z, y[i].w};
        float part = 0.f;
#pragma unroll
        for (int f = 0; f < 4; ++f) {
          part = fmaf(__uint_as_float(u[f] << 16), __uint_as_float(v[f] << 16), part);
          part = fmaf(__uint_as_float(u[f] & 0xFFFF0000u), __uint_as_float(v[f] & 0xFFFF0000u), part);
        }
#pragma unroll
        for (int f = N / 2; f > 0; f >>= 1) part += __shfl_xor_sync(0xffffffffu, part, f);
        if (piece == 0) dots[q * 32 + half * 16 + i * ROWS + lane / N] = part;
      }
    }
    elements_sync();
    const float dot = dots[r];
    if (half == 0 && row < a.tokens) a.dot[stat] = dot;
    const float scale2 = a.scale * kLog2e;
    const uint64_t by2 = two(scale2, scale2), less2 = two(nl2, nl2), minus_dot = two(-dot, -dot), minus_one = two(-1.f, -1.f);
    bool ok = true;
    for (int i = 0; i < n; ++i) {
      wait(s_full, i & 1, ok);
      tc_fence_after_sync();
      uint32_t s[2][32], g[2][32];
#pragma unroll
      for (int c = 0; c < 2; ++c) tmem_ld_32x32(tmem + L::kS + lanes + half * 64 + c * 32, s[c]);
#pragma unroll
      for (int c = 0; c < 2; ++c) tmem_ld_32x32(tmem + L::kP + lanes + half * 64 + c * 32, g[c]);
      tmem_ld_wait();
      tc_fence_before_sync();
      __syncwarp();
      mbar_arrive_if(lane == 0, s_free);
      const int at = (sp.lo + i) * kB + half * 64;
      const int from = start - at, to = row - at;          // visible columns [from, to]
      const bool cut = __any_sync(0xffffffffu, from > 0 || to < 63);
#pragma unroll
      for (int c = 0; c < 2; ++c) {
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
          const float2 x = parts(fma2(two(s[c][e], s[c][e + 1]), by2, less2));
          const float2 d = parts(mul2(two(ex2(x.x), ex2(x.y)), add2(two(g[c][e], g[c][e + 1]), minus_dot)));
          g[c][e] = __float_as_uint(d.x);
          g[c][e + 1] = __float_as_uint(d.y);
        }
        if (__builtin_expect(cut, 0)) {
          const uint32_t seen = visible(from - c * 32, to - c * 32);
#pragma unroll
          for (int e = 0; e < 32; ++e)
            if ((seen >> e & 1) == 0) g[c][e] = 0u;
        }
        uint32_t w[16], low[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          w[e] = pack2(__uint_as_float(g[c][2 * e]), __uint_as_float(g[c][2 * e + 1]));
          const float2 rest = parts(fma2(two(w[e] << 16, w[e] & 0xFFFF0000u), minus_one, two(g[c][2 * e], g[c][2 * e + 1])));
          low[e] = pack2(rest.x, rest.y);
        }
        // (dS of the block before has been read)
        if (c == 0 && i > 0) wait(&k_empty[(i - 1) % L::kK], ((i - 1) / L::kK) & 1, ok);
        tmem_st_32x16(tmem + L::kDs + lanes + half * 32 + c * 16, w);
        tmem_st_32x16(tmem + L::kDs + 64 + lanes + half * 32 + c * 16, low);
      }
      tmem_st_wait();
      tc_fence_before_sync();
      __syncwarp();
      mbar_arrive_if(lane == 0, ds_ready);
      if (!__all_sync(0xffffffffu, ok)) break;
    }
    if (n > 0) wait(done, 0, ok);
    if (!__all_sync(0xffffffffu, ok)) failed = true;
    tc_fence_after_sync();
    if (failed && lane == 0) atomicExch(a.err, 46);
    if (!failed) {
      __nv_bfloat16* dst = row < a.tokens ? head_ptr<__nv_bfloat16>(a.dq, rep, head, a.head_dim) + row * a.dq.row : nullptr;
      const bool fine = result_row<HD / 2>(tmem + L::kO + lanes, half * (HD / 2), cols, n > 0, start > row, a.scale, dst, a.head_dim);
      const uint32_t ill = __ballot_sync(0xffffffffu, !fine && row < a.tokens);
      if (ill != 0u && lane == 0) atomicOr(&bad[q], ill);
    }
    elements_sync();
    if (!failed) {
      const uint32_t ill = bad[q] & 0xFFFFu << half * 16;
      if (ill != 0u) dq_rows<__nv_bfloat16, HD / 32>(a, rep, head, r0 + q * 32, ill);
    }
    tc_fence_before_sync();
  }
  __syncwarp();
  if (failed) {
    // a wait ran out: give the loads in flight time to land before the shared memory is released
    const long long t0 = clock64();
    while (clock64() - t0 < 4000000ll) {}
  }
  __syncthreads();
  if (warp == 1) {
    tc_fence_after_sync();
    tmem_dealloc(tmem, 512);
  }
}

// dk and dv, a tile of 128 keys (rows of S^T = K Q^T and dP^T = V dO^T) over all tiles of queries of its group's heads.  The elements
// take turns: while those of P are formed, dk of the step before and the next dP are; while those of dS are, dv of this step and
// the next S.  Heads of 128 fill the tensor memory with S, dP, dk and dv: P takes the place of S there, and dS that of dP, so the
// next S (dP) waits for the product that reads P (dS).  Smaller ones have places of their own for P and dS, which the elements
// fill again when that product is done.  A key is seen by the queries from itself to the end of its sequence.  P and dS are
// one bf16 piece here (2^-8 of each term): a column's terms cancel by no law as a row's dS do, so what the roundings leave is a share
// of the result, 1.6e-3 of its norm beside the 1.66e-3 of its own rounding.
//
// Where there are few tiles of keys, a cluster of `split` CTAs shares a tile's queries.  Each leaves its sums in shared memory, and adds
// up a slice of the columns over all of them, in order (2048 rows of 8 heads on 1 of 128: 16 tiles).
template <int HD>
struct Dkv {
  static constexpr int kTile = kB * HD * 2;
  static constexpr int kQ = 3, kG = 2;                      // slots of Q and dO; the rows' lse and D have two
  static constexpr int kStats = (2 + kQ + kG) * kTile;      // behind K, V, the Q and dO slots
  static constexpr int kBars = kStats + 2 * 2 * kB * 4;
  static constexpr int kTotal = kBars + 16 + (2 * kQ + 2 * kG + 8) * 8 + 16;
  static constexpr bool kShared = HD == 128;                // P and dS in the places of S and dP
  static constexpr uint32_t kS = 0, kDp = 128, kDk = 256, kDv = 256 + HD;
  // the bf16 of P and dS: half h of the columns at + h * kHalf
  static constexpr uint32_t kP = kShared ? kS : 384, kDs = kShared ? kDp : 448, kHalf = kShared ? 64 : 32;
};
struct DkvMaps { CUtensorMap q, dout, k, v; };

template <int HD>
__global__ void __launch_bounds__(kBwdThreads, 1)
attention_dkv_tc_kernel(const __grid_constant__ DkvMaps maps, const __grid_constant__ Args a, const int split) {
  using L = Dkv<HD>;
  extern __shared__ __align__(1024) uint8_t smem[];                  // (no room to round its start up)
  if ((smem_u32(smem) & 1023) != 0) {                                  // (then it is so for every CTA)
    if (threadIdx.x == 0) atomicExch(a.err, 40);
    return;
  }
  float* stats = reinterpret_cast<float*>(smem + L::kStats);         // [slot][-lse * log2(e), -D][128]
  uint32_t* bad = reinterpret_cast<uint32_t*>(smem + L::kBars);      // [4]
  uint64_t* q_full = reinterpret_cast<uint64_t*>(bad + 4);
  uint64_t* q_empty = q_full + L::kQ;
  uint64_t* g_full = q_empty + L::kQ;
  uint64_t* g_empty = g_full + L::kG;
  uint64_t* kv_full = g_empty + L::kG;   // [2] K, V
  uint64_t* st_full = kv_full + 2;       // [2] lse and D
  uint64_t* s_full = st_full + 2;        // S of a step
  uint64_t* dp_full = s_full + 1;
  uint64_t* p_ready = dp_full + 1;       // eight warps have left P
  uint64_t* ds_ready = p_ready + 1;      // ... and dS
  uint64_t* done = ds_ready + 1;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(done + 1);
  uint8_t* sq = smem + 2 * L::kTile;
  uint8_t* sg = sq + L::kQ * L::kTile;

  // the keys with the most queries first
  const int unit = blockIdx.x / split, rank = blockIdx.x % split;
  const int kvh = unit % a.kv_heads, rest = unit / a.kv_heads, rep = rest % a.m;
  const int kt = rest / a.m, k0 = kt * kB, group = a.heads / a.kv_heads;
  const int panels = (a.head_dim + 63) / 64, ksteps = (a.head_dim + 15) / 16, cols = ksteps * 16;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  bool failed = false;
  if (threadIdx.x == 0) {
    for (int i = 0; i < L::kQ; ++i) { mbar_init(&q_full[i], 1); mbar_init(&q_empty[i], 1); }
    for (int i = 0; i < L::kG; ++i) { mbar_init(&g_full[i], 1); mbar_init(&g_empty[i], 1); }
    mbar_init(&kv_full[0], 1);
    mbar_init(&kv_full[1], 1);
    mbar_init(&st_full[0], 1);
    mbar_init(&st_full[1], 1);
    mbar_init(s_full, 1);
    mbar_init(dp_full, 1);
    mbar_init(p_ready, 8);
    mbar_init(ds_ready, 8);
    mbar_init(done, 1);
    fence_mbar_init();
    for (int i = 0; i < 4; ++i) bad[i] = 0u;
    prefetch_tmap(&maps.q);
    prefetch_tmap(&maps.dout);
    // K and V are on their way while the tensor memory is allocated and the boundaries are read
    fence_proxy_async_smem();
    grid_dep_wait();
    load_tile(&maps.k, smem, &kv_full[0], panels, kvh, k0, rep, l2_policy(0));
    load_tile(&maps.v, smem + L::kTile, &kv_full[1], panels, kvh, k0, rep, l2_policy(0));
  }
  __syncwarp();
  if (warp == 1) {
    tmem_alloc(tmem_slot, 512);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = *tmem_slot;
  grid_dep_wait();
  grid_dep_launch();

  const Bounds bounds(a, rep);
  const int end = bounds.last_query((int)min((int64_t)k0 + kB, a.tokens) - 1);
  const int per = end > k0 ? (end - 1) / kB - kt + 1 : 0;            // tiles of queries of a head
  // this CTA's steps of all: tiles of queries, head by head
  const int64_t all = (int64_t)per * group;
  const int first = (int)(all * rank / split), n = (int)(all * (rank + 1) / split) - first;

  if (warp == 0) {
    const bool lead = elect_one();
    const uint64_t pol = l2_policy(0);
    int head = kvh * group + (per > 0 ? first / per : 0), tile = kt + (per > 0 ? first % per : 0);
    for (int i = 0; i < n && !failed; ++i) {
      const int qs = i % L::kQ, gs = i % L::kG;
      if (i >= L::kQ && !__all_sync(0xffffffffu, mbar_wait(&q_empty[qs], (i / L::kQ - 1) & 1))) { failed = true; break; }
      if (lead) load_tile(&maps.q, sq + qs * L::kTile, &q_full[qs], panels, head, tile * kB, rep, pol);
      __syncwarp();
      if (i >= L::kG && !__all_sync(0xffffffffu, mbar_wait(&g_empty[gs], (i / L::kG - 1) & 1))) { failed = true; break; }
      if (lead) load_tile(&maps.dout, sg + gs * L::kTile, &g_full[gs], panels, head, tile * kB, rep, pol);
      __syncwarp();
      // the rows' numbers, into the place of the step before the last, whose elements are done when its Q is let go of
      const int64_t stat = ((int64_t)rep * a.heads + head) * a.tokens;
      float l[kB / 32], d[kB / 32];
#pragma unroll
      for (int e = 0; e < kB / 32; ++e) {
        const int row = tile * kB + e * 32 + lane;
        const bool in = row < a.tokens;
        l[e] = in ? -a.lse[stat + row] * kLog2e : 0.f;
        d[e] = in ? -a.dot[stat + row] : 0.f;
      }
      if (i >= 2 && !__all_sync(0xffffffffu, mbar_wait(&q_empty[(i - 2) % L::kQ], ((i - 2) / L::kQ) & 1))) { failed = true; break; }
      float* st = stats + (i & 1) * 2 * kB;
#pragma unroll
      for (int e = 0; e < kB / 32; ++e) {
        st[e * 32 + lane] = l[e];
        st[kB + e * 32 + lane] = d[e];
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&st_full[i & 1]);
      __syncwarp();
      if (++tile == kt + per) { tile = kt; ++head; }
    }
    // tiles that no product needs, and the releases of the last slots, arrive here: wait for them before leaving
    for (int i = 0; i < 2; ++i)
      if (n <= 0 && !__all_sync(0xffffffffu, mbar_wait(&kv_full[i], 0))) failed = true;
    for (int i = 0; i < L::kQ && i < n && !failed; ++i)
      if (!__all_sync(0xffffffffu, mbar_wait(&q_empty[i], ((n - 1 - i) / L::kQ) & 1))) failed = true;
    for (int i = 0; i < L::kG && i < n && !failed; ++i)
      if (!__all_sync(0xffffffffu, mbar_wait(&g_empty[i], ((n - 1 - i) / L::kG) & 1))) failed = true;
    if (failed && lane == 0) atomicExch(a.err, 47);
  } else if (warp == 1) {
    const bool lead = elect_one();
    const uint32_t idesc_s = make_idesc(1, false, false, kB, kB);
    const uint32_t idesc_o = make_idesc(1, false, true, kB, (uint32_t)cols);
    constexpr uint32_t T = L::kTile / 16;
    const uint32_t kb = k_major(smem_u32(smem)), vb = kb + T, qb = k_major(smem_u32(sq)), gb = k_major(smem_u32(sg));
    const uint32_t qmn = mn_major(smem_u32(sq)), gmn = mn_major(smem_u32(sg));
    bool ok = true;
    auto scores = [&](int i) {
      const int qs = i % L::kQ;
      wait(&q_full[qs], (i / L::kQ) & 1, ok);
      if (i == 0) wait(&kv_full[0], 0, ok);
      tc_fence_after_sync();
      product_ss<HD>(lead, tmem + L::kS, kb, qb + qs * T, idesc_s, ksteps);
      mma_commit_if(lead, s_full);
    };
    auto dots = [&](int i) {
      const int gs = i % L::kG;
      wait(&g_full[gs], (i / L::kG) & 1, ok);
      if (i == 0) wait(&kv_full[1], 0, ok);
      tc_fence_after_sync();
      product_ss<HD>(lead, tmem + L::kDp, vb, gb + gs * T, idesc_s, ksteps);
      mma_commit_if(lead, dp_full);
    };
    if (n > 0) {
      scores(0);
      dots(0);
    }
    for (int i = 0; i < n; ++i) {
      const int qs = i % L::kQ, gs = i % L::kG;
      auto dv = [&]() {
        product_ts(lead, tmem + L::kDv, tmem + L::kP, gmn + gs * T, idesc_o, i > 0);
        product_ts(lead, tmem + L::kDv, tmem + L::kP + L::kHalf, gmn + gs * T + kHalfRows, idesc_o, true);
        mma_commit_if(lead, &g_empty[gs]);
      };
      auto dk = [&]() {
        product_ts(lead, tmem + L::kDk, tmem + L::kDs, qmn + qs * T, idesc_o, i > 0);
        product_ts(lead, tmem + L::kDk, tmem + L::kDs + L::kHalf, qmn + qs * T + kHalfRows, idesc_o, true);
        mma_commit_if(lead, &q_empty[qs]);
        mma_commit_if(lead && i == n - 1, done);
      };
      wait(p_ready, i & 1, ok);
      tc_fence_after_sync();
      if (L::kShared) {
        dv();
        if (i + 1 < n) wait(&g_empty[gs], (i / L::kG) & 1, ok);
        if (i + 1 < n) scores(i + 1);
      } else {
        if (i + 1 < n) scores(i + 1);
        dv();
      }
      wait(ds_ready, i & 1, ok);
      tc_fence_after_sync();
      if (L::kShared) {
        dk();
        if (i + 1 < n) wait(&q_empty[qs], (i / L::kQ) & 1, ok);
        if (i + 1 < n) dots(i + 1);
      } else {
        if (i + 1 < n) dots(i + 1);
        dk();
      }
      if (!__all_sync(0xffffffffu, ok)) break;
    }
    if (!__all_sync(0xffffffffu, ok)) failed = true;
    if (failed && lane == 0) atomicExch(a.err, 48);
  } else {
    const int half = (warp - 2) >> 2, q = warp & 3, r = q * 32 + lane, key = k0 + r;
    const uint32_t lanes = (uint32_t)(q * 32) << 16, mine = lanes + half * 64, left = lanes + half * L::kHalf;
    int start, seq_end;
    bounds.rows(k0 + q * 32, &start, &seq_end);
    const float scale2 = a.scale * kLog2e;
    const uint64_t by2 = two(scale2, scale2);
    int tile = kt + (per > 0 ? first % per : 0);
    bool ok = true;
    for (int i = 0; i < n; ++i) {
      const float* st = stats + (i & 1) * 2 * kB + half * 64;
      const int at = tile * kB + half * 64;
      const int from = key - at, to = seq_end - 1 - at;    // visible columns [from, to]
      const bool cut = __any_sync(0xffffffffu, from > 0 || to < 63);
      const uint32_t seen[2] = {visible(from, to), visible(from - 32, to - 32)};
      float p[64];
      wait(&st_full[i & 1], (i >> 1) & 1, ok);
      wait(s_full, i & 1, ok);
      tc_fence_after_sync();
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        uint32_t s[32], w[16];
        tmem_ld_32x32(tmem + L::kS + mine + c * 32, s);
        tmem_ld_wait();
#pragma unroll
        for (int e = 0; e < 32; e += 4) {
          const ulonglong2 l = *reinterpret_cast<const ulonglong2*>(st + c * 32 + e);
          const float2 x = parts(fma2(two(s[e], s[e + 1]), by2, l.x)), y = parts(fma2(two(s[e + 2], s[e + 3]), by2, l.y));
          p[c * 32 + e] = ex2(x.x);
          p[c * 32 + e + 1] = ex2(x.y);
          p[c * 32 + e + 2] = ex2(y.x);
          p[c * 32 + e + 3] = ex2(y.y);
        }
        if (__builtin_expect(cut, 0)) {
#pragma unroll
          for (int e = 0; e < 32; ++e)
            if ((seen[c] >> e & 1) == 0) p[c * 32 + e] = 0.f;
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) w[e] = pack2(p[c * 32 + 2 * e], p[c * 32 + 2 * e + 1]);
        if (!L::kShared && c == 0 && i > 0) wait(&g_empty[(i - 1) % L::kG], ((i - 1) / L::kG) & 1, ok);
        tmem_st_32x16(tmem + L::kP + left + c * 16, w);
      }
      tmem_st_wait();
      tc_fence_before_sync();
      __syncwarp();
      mbar_arrive_if(lane == 0, p_ready);
      wait(dp_full, i & 1, ok);
      tc_fence_after_sync();
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        uint32_t g[32], w[16];
        tmem_ld_32x32(tmem + L::kDp + mine + c * 32, g);
        tmem_ld_wait();
#pragma unroll
        for (int e = 0; e < 32; e += 4) {
          const ulonglong2 d = *reinterpret_cast<const ulonglong2*>(st + kB + c * 32 + e);
          const float2 x = parts(mul2(two(p[c * 32 + e], p[c * 32 + e + 1]), add2(two(g[e], g[e + 1]), d.x)));
          const float2 y = parts(mul2(two(p[c * 32 + e + 2], p[c * 32 + e + 3]), add2(two(g[e + 2], g[e + 3]), d.y)));
          g[e] = __float_as_uint(x.x);
          g[e + 1] = __float_as_uint(x.y);
          g[e + 2] = __float_as_uint(y.x);
          g[e + 3] = __float_as_uint(y.y);
        }
        if (__builtin_expect(cut, 0)) {    // (0 times NaN)
#pragma unroll
          for (int e = 0; e < 32; ++e)
            if ((seen[c] >> e & 1) == 0) g[e] = 0u;
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) w[e] = pack2(__uint_as_float(g[2 * e]), __uint_as_float(g[2 * e + 1]));
        if (!L::kShared && c == 0 && i > 0) wait(&q_empty[(i - 1) % L::kQ], ((i - 1) / L::kQ) & 1, ok);
        tmem_st_32x16(tmem + L::kDs + left + c * 16, w);
      }
      tmem_st_wait();
      tc_fence_before_sync();
      __syncwarp();
      mbar_arrive_if(lane == 0, ds_ready);
      if (!__all_sync(0xffffffffu, ok)) break;
      if (++tile == kt + per) tile = kt;
    }
    if (n > 0) wait(done, 0, ok);
    if (!__all_sync(0xffffffffu, ok)) failed = true;
    tc_fence_after_sync();
    if (failed && lane == 0) atomicExch(a.err, 49);
    if (split == 1) {
      if (!failed) {
        const bool none = seq_end <= key, in = key < a.tokens;
        __nv_bfloat16* dk = in ? head_ptr<__nv_bfloat16>(a.dk, rep, kvh, a.head_dim) + key * a.dk.row : nullptr;
        __nv_bfloat16* dv = in ? head_ptr<__nv_bfloat16>(a.dv, rep, kvh, a.head_dim) + key * a.dv.row : nullptr;
        bool fine = result_row<HD / 2>(tmem + L::kDk + lanes, half * (HD / 2), cols, n > 0, none, a.scale, dk, a.head_dim);
        fine = result_row<HD / 2>(tmem + L::kDv + lanes, half * (HD / 2), cols, n > 0, none, 1.f, dv, a.head_dim) && fine;
        const uint32_t ill = __ballot_sync(0xffffffffu, !fine && in);
        if (ill != 0u && lane == 0) atomicOr(&bad[q], ill);
      }
      elements_sync();
      if (!failed) {
        const uint32_t ill = bad[q] & 0xFFFFu << half * 16;
        if (ill != 0u) dkv_rows<__nv_bfloat16, HD / 32>(a, rep, kvh, k0 + q * 32, ill, a.dot);
      }
    } else {
      // [dk, dv][column][row], neighbouring lanes beside each other (over K and V, which have to have landed)
      if (n <= 0) {
        wait(&kv_full[0], 0, ok);
        wait(&kv_full[1], 0, ok);
      }
      float* sums = reinterpret_cast<float*>(smem) + r;
#pragma unroll
      for (int g = 0; g < 2 * HD / 32; ++g) {
        const int c = half * HD + g * 16;  // (half 0 has dk, half 1 dv)
        uint32_t o[16];
        if (n > 0 && !failed) {
          tmem_ld_32x16(tmem + L::kDk + lanes + c, o);
          tmem_ld_wait();
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e) o[e] = 0u;
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) sums[(c + e) * kB] = __uint_as_float(o[e]);
      }
    }
    tc_fence_before_sync();
  }
  if (split > 1) {
    __syncwarp();
    cluster_sync_all();
    if (warp >= 2) {
      constexpr int kMost = 8;             // columns at a time
      const int t = (warp - 2) * 32 + lane, r = t & (kB - 1), mat = t >> 7, key = k0 + r;
      const int width = HD / split, from = rank * width;
      int start, seq_end;
      bounds.rows(k0 + (r & ~31), &start, &seq_end);
      const bool none = seq_end <= key;
      const Tensor& d = mat == 0 ? a.dk : a.dv;
      __nv_bfloat16* row = head_ptr<__nv_bfloat16>(d, rep, kvh, a.head_dim) + (int64_t)key * d.row;
      bool fine = true;
      for (int c = from; c < from + width && c < a.head_dim; c += kMost) {
        float v[kMost];
#pragma unroll
        for (int e = 0; e < kMost; ++e) v[e] = 0.f;
        for (int p = 0; p < split; ++p) {
          const uint32_t at = map_to_rank(smem_u32(smem), p) + ((mat * HD + c) * kB + r) * 4;
#pragma unroll
          for (int e = 0; e < kMost; ++e) v[e] += ld_cluster_f32(at + e * kB * 4);
        }
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float by = mat == 0 ? a.scale : 1.f, x = v[2 * e] * by, y = v[2 * e + 1] * by;
          fine = fine && fabsf(x) < INFINITY && fabsf(y) < INFINITY;
          w[e] = none ? 0u : pack2(x, y);
        }
        if (key < a.tokens) *reinterpret_cast<uint4*>(row + c) = make_uint4(w[0], w[1], w[2], w[3]);
      }
      if (!fine && key < a.tokens) atomicOr(&bad[r >> 5], 1u << (r & 31));
    }
    __syncwarp();
    cluster_sync_all();                    // (all columns written, all rows looked at)
    if (warp >= 2 && rank == 0) {
      for (int g = 0; g < 4; ++g) {
        uint32_t ill = 0;
        for (int p = 0; p < split; ++p) ill |= __float_as_uint(ld_cluster_f32(map_to_rank(smem_u32(&bad[g]), p)));
        ill &= 0xFu << (warp - 2) * 4;
        if (ill != 0u) dkv_rows<__nv_bfloat16, HD / 32>(a, rep, kvh, k0 + g * 32, ill, a.dot);
      }
    }
    __syncwarp();
    cluster_sync_all();                    // (nobody's shared memory is read any more)
  }
  __syncwarp();
  if (failed) {
    // a wait ran out: give the loads in flight time to land before the shared memory is released
    const long long t0 = clock64();
    while (clock64() - t0 < 4000000ll) {}
  }
  __syncthreads();
  if (warp == 1) {
    tc_fence_after_sync();
    tmem_dealloc(tmem, 512);
  }
}

// ---- host side ---------------------------------------------------------------------------------------------------

template <int HD>
cudaError_t launch_forward(const FwdMaps& maps, const Args& a, cudaStream_t st) {
  using L = Fwd<HD>;
  static uint64_t done = 0;              // one bit per device
  static_assert(L::kTotal <= 227 * 1024, "shared memory budget");
  const cudaError_t e = allow_dynamic_smem(attention_tc_kernel<HD>, L::kTotal, &done);
  if (e != cudaSuccess) return e;
  const int64_t tiles = (a.tokens + L::kTiles * kB - 1) / (L::kTiles * kB);
  return launch_dep(attention_tc_kernel<HD>, dim3((unsigned)(tiles * a.heads * a.m)), dim3(L::kThreads), L::kTotal, st, 1, maps, a);
}

constexpr int kAlone = 227 * 1024;       // shared memory beside which no other kernel with tensor memory fits

template <int HD>
cudaError_t launch_backward(const DqMaps& dq, const DkvMaps& dkv, const Args& a, cudaStream_t st) {
  static uint64_t done[2] = {0, 0};      // one bit per device
  static_assert(Dq<HD>::kTotal <= 227 * 1024 && Dkv<HD>::kTotal <= 227 * 1024, "shared memory budget");
  cudaError_t e = allow_dynamic_smem(attention_dq_tc_kernel<HD>, Dq<HD>::kTotal, &done[0]);
  if (e == cudaSuccess) e = allow_dynamic_smem(attention_dkv_tc_kernel<HD>, kAlone, &done[1]);
  const int64_t tiles = (a.tokens + kB - 1) / kB;
  if (e == cudaSuccess)
    e = launch_dep(attention_dq_tc_kernel<HD>, dim3((unsigned)(tiles * a.heads * a.m)), dim3(kBwdThreads), Dq<HD>::kTotal, st, 1, dq, a);
  // As many CTAs to a tile of keys, up to eight, as still find an SM.  Those of a cluster have an SM for themselves: a CTA that waited
  // there for another kernel's tensor memory, while that one's cluster waited for a CTA that waits for this one's, would wait for good.
  const int64_t units = tiles * a.kv_heads * a.m;
  int split = 1;
  while (split < 8 && units * split * 2 <= 148) split *= 2;
  if (e == cudaSuccess)
    e = launch_dep(attention_dkv_tc_kernel<HD>, dim3((unsigned)(units * split)), dim3(kBwdThreads), split > 1 ? kAlone : Dkv<HD>::kTotal, st,
                   (unsigned)split, dkv, a, split);
  return e;
}

int head_map(CUtensorMap* map, const Args& a, const Tensor& t, int heads, int box_rows) {
  return gop::make_heads_map(map, t.p, a.head_dim, heads, a.tokens, a.m, t.row, t.replica, box_rows);
}
bool tc_tensor(const Tensor& t) {
  return reinterpret_cast<uintptr_t>(t.p) % 16 == 0 && t.row % 8 == 0 && t.replica % 8 == 0 && t.replica < (1ll << 38);
}

}  // namespace

bool tc_takes(const Args& a, int dtype) {
  if (dtype != LS_DTYPE_BF16 || a.head_dim % 8 != 0 || a.head_dim > 128 || !(a.scale > 0.f)) return false;
  for (const Tensor* t : {&a.q, &a.k, &a.v, &a.out, &a.dout, &a.dq, &a.dk, &a.dv})
    if (t->p != nullptr && !tc_tensor(*t)) return false;
  return true;
}

cudaError_t tc_forward(const Args& a, cudaStream_t st) {
  FwdMaps maps;
  if (head_map(&maps.q, a, a.q, a.heads, kB) != cudaSuccess || head_map(&maps.k, a, a.k, a.kv_heads, kB) != cudaSuccess ||
      head_map(&maps.v, a, a.v, a.kv_heads, kB) != cudaSuccess)
    return cudaErrorInvalidValue;
  return a.head_dim <= 64 ? launch_forward<64>(maps, a, st) : launch_forward<128>(maps, a, st);
}

cudaError_t tc_backward(const Args& a, cudaStream_t st) {
  DqMaps dq;
  DkvMaps dkv;
  if (head_map(&dq.q, a, a.q, a.heads, kB) != cudaSuccess || head_map(&dq.dout, a, a.dout, a.heads, kB) != cudaSuccess ||
      head_map(&dq.k, a, a.k, a.kv_heads, kB) != cudaSuccess || head_map(&dq.v, a, a.v, a.kv_heads, kB) != cudaSuccess)
    return cudaErrorInvalidValue;
  dkv.q = dq.q;
  dkv.dout = dq.dout;
  dkv.k = dq.k;
  dkv.v = dq.v;
  return a.head_dim <= 64 ? launch_backward<64>(dq, dkv, a, st) : launch_backward<128>(dq, dkv, a, st);
}

}  // namespace attn
}  // namespace ls
