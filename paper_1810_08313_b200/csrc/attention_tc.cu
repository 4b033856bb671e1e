// Attention over packed sequences on the tensor cores: bf16 heads of up to 128 elements (see attention.cuh for the formulas).
//
// Forward.  A CTA takes 256 consecutive rows of one head as two tiles of 128 (rows of S are TMEM lanes) and passes over the keys in
// blocks of 128, once:
//   warp 0     TMA producer: both tiles of Q, then K and V blocks through a ring
//   warp 1     issues the MMAs: S = Q K^T (operands in shared memory) and O += P V (P in tensor memory, where it
//              takes the place of S).  Per block and tile: PV of the block before, then S of this one; the tiles alternate, so that
//              the tensor core works for one while the other's softmax runs
//   warps 2-5, 6-9   the softmax of a tile, a thread a row: 128 scores in registers, running maximum, exponentials, sum, P in
//              bf16 back to tensor memory
// A commit arrives when everything issued before it is complete, so S of a block also says that the PV before it is done.
// O stays in tensor memory over all blocks and is rescaled only where a row's maximum has grown by more than 2^8 since its
// reference was taken: P then lies below 2^8 instead of 1, which costs bf16 and fp32 no precision, and most blocks need no
// pass over O.  P is rounded to bf16 (2^-8 of each term, signs at random), its sum is taken before the rounding.
#include "attention.cuh"

namespace ls {
namespace attn {
namespace {

using namespace ptx;

constexpr int kB = 128;                  // rows of a tile, keys of a block
constexpr int kFwdThreads = 320;

template <int HD>
struct Fwd {
  static constexpr int kTile = kB * HD * 2;                 // bytes: HD / 64 panels of 128 rows x 128 bytes
  static constexpr int kSlots = HD == 128 ? 4 : 6;
  static constexpr int kRing = 2 * kTile;                   // offset of the ring, behind Q
  static constexpr int kBars = kRing + kSlots * kTile;
  static constexpr int kTotal = 1024 + kBars + (2 * kSlots + 8) * 8 + 16;
  static constexpr uint32_t kO = 256;                       // first TMEM column of O (tile X: + X HD); S: 0 and 128
};

struct FwdMaps { CUtensorMap q, k, v, out; };

__device__ __forceinline__ float ex2(float x) { return gop::ex2(x); }
__device__ __forceinline__ uint32_t pack2(float a, float b) { return gop::pack_bf16(a, b); }

// key blocks [lo, hi] that the tile of rows from r0 on needs (lo > hi: none)
struct Span { int lo, hi; };
__device__ __forceinline__ Span key_blocks(const Args& a, int rep, int r0) {
  if (r0 >= a.tokens) return Span{1, 0};
  return Span{first_key(a, rep, r0) / kB, r0 / kB};
}

__device__ __forceinline__ void store_heads(const CUtensorMap* m, const void* src, int x, int head, int token, int rep) {
  asm volatile("cp.async.bulk.tensor.4d.global.shared::cta.bulk_group [%0, {%2, %3, %4, %5}], [%1];" ::"l"(
                   reinterpret_cast<uint64_t>(m)),
               "r"(smem_u32(src)), "r"(x), "r"(head), "r"(token), "r"(rep)
               : "memory");
}

template <int HD>
__global__ void __launch_bounds__(kFwdThreads, 1)
attention_tc_kernel(const __grid_constant__ FwdMaps maps, const __grid_constant__ Args a) {
  using L = Fwd<HD>;
  constexpr int PANELS = HD / 64, SLOTS = L::kSlots;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + L::kBars);
  uint64_t* empty = full + SLOTS;
  uint64_t* q_full = empty + SLOTS;      // [2]
  uint64_t* s_full = q_full + 2;         // [2] S of the next block is there, and the PV before it done
  uint64_t* p_ready = s_full + 2;        // [2] four warps have left P
  uint64_t* o_done = p_ready + 2;        // [2] the last PV is done
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(o_done + 2);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  bool failed = false;
  if (threadIdx.x == 0) {
    for (int s = 0; s < SLOTS; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
    for (int x = 0; x < 2; ++x) { mbar_init(&q_full[x], 1); mbar_init(&s_full[x], 1); mbar_init(&p_ready[x], 4); mbar_init(&o_done[x], 1); }
    fence_mbar_init();
    prefetch_tmap(&maps.q);
    prefetch_tmap(&maps.k);
    prefetch_tmap(&maps.v);
    prefetch_tmap(&maps.out);
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

  // the rows with the most keys first; heads of a group beside each other
  const int tiles = (int)((a.tokens + 2 * kB - 1) / (2 * kB));
  const int head = blockIdx.x % a.heads, rest = blockIdx.x / a.heads, rep = rest % a.m;
  const int r0 = (tiles - 1 - rest / a.m) * 2 * kB;
  const int kvh = head / (a.heads / a.kv_heads);
  const Span sa = key_blocks(a, rep, r0), sb = key_blocks(a, rep, r0 + kB);
  const bool has_a = sa.lo <= sa.hi, has_b = sb.lo <= sb.hi;
  const int lo = has_a ? sa.lo : sb.lo, hi = has_b ? sb.hi : sa.hi;        // (lo > hi if neither has any)
  const int panels = (a.head_dim + 63) / 64;

  if (warp == 0) {
    const bool lead = elect_one();
    const uint64_t pol = l2_policy(0);
    if (lead) {
      for (int x = 0; x < 2; ++x) {
        if (!(x == 0 ? has_a : has_b)) continue;
        mbar_expect_tx(&q_full[x], panels * kB * 128);
        for (int c = 0; c < panels; ++c)
          tma_load_4d_hint(smem + x * L::kTile + c * kB * 128, &maps.q, &q_full[x], c * 64, head, r0 + x * kB, rep, pol);
      }
    }
    __syncwarp();
    int s = 0, round = 0;
    for (int j = lo; j <= hi && !failed; ++j) {
      for (int kv = 0; kv < 2; ++kv) {
        if (round > 0 && !__all_sync(0xffffffffu, mbar_wait(&empty[s], (round - 1) & 1))) { failed = true; break; }
        if (lead) {
          uint8_t* dst = smem + L::kRing + s * L::kTile;
          mbar_expect_tx(&full[s], panels * kB * 128);
          for (int c = 0; c < panels; ++c)
            tma_load_4d_hint(dst + c * kB * 128, kv == 0 ? &maps.k : &maps.v, &full[s], c * 64, kvh, j * kB, rep, pol);
        }
        __syncwarp();
        if (++s == SLOTS) { s = 0; ++round; }
      }
    }
    // the releases of the last slots arrive here: wait for them before leaving
    for (int i = 0; i < SLOTS && !failed; ++i) {
      const int uses = round + (i < s ? 1 : 0);
      if (uses > 0 && !__all_sync(0xffffffffu, mbar_wait(&empty[i], (uses - 1) & 1))) failed = true;
    }
    if (failed && lane == 0) atomicExch(a.err, 41);
  } else if (warp == 1) {
    const bool lead = elect_one();
    const int ksteps = (a.head_dim + 15) / 16;
    const uint32_t idesc_s = make_idesc(1, false, false, kB, kB);
    const uint32_t idesc_o = make_idesc(1, false, true, kB, (uint32_t)ksteps * 16);
    const uint32_t base = smem_u32(smem);
    for (int x = 0; x < 2; ++x)
      if ((x == 0 ? has_a : has_b) && !__all_sync(0xffffffffu, mbar_wait(&q_full[x], 0))) failed = true;
    int s = 0, round = 0;
    int vslot = 0;
    for (int j = lo; j <= hi + 1 && lo <= hi && !failed; ++j) {
      const bool has_v = j > lo, has_k = j <= hi;
      if (has_v) {                       // V of the block before
        vslot = s;
        if (!__all_sync(0xffffffffu, mbar_wait(&full[s], round & 1))) { failed = true; break; }
        if (++s == SLOTS) { s = 0; ++round; }
      }
      const int kslot = s;
      if (has_k) {
        if (!__all_sync(0xffffffffu, mbar_wait(&full[s], round & 1))) { failed = true; break; }
        if (++s == SLOTS) { s = 0; ++round; }
      }
      for (int x = 0; x < 2 && !failed; ++x) {
        const Span sp = x == 0 ? sa : sb;
        const uint32_t ts = tmem + x * kB, to = tmem + L::kO + x * HD;
        if (has_v && j - 1 >= sp.lo && j - 1 <= sp.hi) {
          if (!__all_sync(0xffffffffu, mbar_wait(&p_ready[x], (j - 1 - sp.lo) & 1))) { failed = true; break; }
          tc_fence_after_sync();
          if (lead) {
            const uint32_t vb = base + L::kRing + vslot * L::kTile;
#pragma unroll
            for (int k = 0; k < kB / 16; ++k)
              mma_bf16_ts(to, ts + k * 8, make_smem_desc(vb + k * 2048, kB * 128, 1024), idesc_o, j - 1 > sp.lo || k > 0);
            if (j - 1 == sp.hi) mma_commit(&o_done[x]);
          }
          __syncwarp();
        }
        if (has_k && j >= sp.lo && j <= sp.hi) {
          tc_fence_after_sync();
          if (lead) {
            const uint32_t qb = base + x * L::kTile, kb = base + L::kRing + kslot * L::kTile;
            for (int k = 0; k < ksteps; ++k) {
              const uint32_t off = (k >> 2) * (kB * 128) + (k & 3) * 32;
              mma_bf16(ts, make_smem_desc(qb + off, 16, 1024), make_smem_desc(kb + off, 16, 1024), idesc_s, k > 0);
            }
            mma_commit(&s_full[x]);
          }
          __syncwarp();
        }
      }
      if (failed) break;
      if (lead) {
        if (has_v) mma_commit(&empty[vslot]);
        if (has_k) mma_commit(&empty[kslot]);
      }
      __syncwarp();
    }
    if (failed && lane == 0) atomicExch(a.err, 42);
  } else {
    const int x = (warp - 2) >> 2, q = warp & 3;
    const Span sp = x == 0 ? sa : sb;
    const int row = r0 + x * kB + q * 32 + lane;
    const int start = row_start(a, rep, row);
    const uint32_t ts = tmem + ((uint32_t)(q * 32) << 16) + x * kB;
    const uint32_t to = tmem + ((uint32_t)(q * 32) << 16) + L::kO + x * HD;
    const float scale2 = a.scale * kLog2e;
    const int cols = (a.head_dim + 15) / 16 * 16;
    float top = -INFINITY, sum = 0.f;    // the reference of the exponentials (a product, not scaled), and their sum
    for (int j = sp.lo; j <= sp.hi; ++j) {
      if (!__all_sync(0xffffffffu, mbar_wait(&s_full[x], (j - sp.lo) & 1))) { failed = true; break; }
      __syncwarp();
      tc_fence_after_sync();
      uint32_t s[4][32];
#pragma unroll
      for (int c = 0; c < 4; ++c) tmem_ld_32x32(ts + c * 32, s[c]);
      tmem_ld_wait();
      const int from = start - j * kB, to_col = row - j * kB;                // visible columns [from, to_col]
      if (__any_sync(0xffffffffu, from > 0 || to_col < kB - 1)) {
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (c * 32 + i < from || c * 32 + i > to_col) s[c][i] = 0xff800000u;
      }
      float most = -INFINITY;
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int i = 0; i < 32; i += 2)
          most = fmaxf(most, fmaxf(__uint_as_float(s[c][i]), __uint_as_float(s[c][i + 1])));
      // (top = -inf: the difference is infinite, and the factor zero)
      const bool far = most > top && (most - top) * scale2 > 8.f;
      if (__any_sync(0xffffffffu, far)) {
        const float next = fmaxf(most, top);
        const float keep = next > top ? ex2((top - next) * scale2) : 1.f;
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
      float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        uint32_t p[16];
#pragma unroll
        for (int i = 0; i < 32; i += 2) {
          const float e = ex2(fmaf(__uint_as_float(s[c][i]), scale2, -ref)), f = ex2(fmaf(__uint_as_float(s[c][i + 1]), scale2, -ref));
          part[i & 2] += e;
          part[(i & 2) + 1] += f;
          p[i >> 1] = pack2(e, f);
        }
        tmem_st_32x16(ts + c * 16, p);
      }
      sum += (part[0] + part[1]) + (part[2] + part[3]);
      tmem_st_wait();
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(&p_ready[x]);
      __syncwarp();
    }
    const bool none = start > row;       // in no sequence, or behind the tensor
    if (sp.lo <= sp.hi && !failed) {
      if (!__all_sync(0xffffffffu, mbar_wait(&o_done[x], 0))) failed = true;
      __syncwarp();
      tc_fence_after_sync();
    }
    if (failed) {
      if (lane == 0) atomicExch(a.err, 43);
    } else if (r0 + x * kB + q * 32 < a.tokens) {
      // this warp's 32 rows leave through its part of the tile's place for Q
      const float by = none ? 0.f : 1.f / sum;
      bool fine = true;
      uint8_t* box = smem + x * L::kTile + q * 32 * 128;
#pragma unroll
      for (int c = 0; c < PANELS; ++c) {
        if (c * 64 >= a.head_dim) break;
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          uint32_t o[16];
          if (c * 64 + h * 16 < cols && sp.lo <= sp.hi) {
            tmem_ld_32x16(to + c * 64 + h * 16, o);
            tmem_ld_wait();
          }
          uint32_t w[8];
          if (c * 64 + h * 16 < cols && !none) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float e = __uint_as_float(o[2 * i]) * by, f = __uint_as_float(o[2 * i + 1]) * by;
              fine = fine && fabsf(e) < INFINITY && fabsf(f) < INFINITY;
              w[i] = pack2(e, f);
            }
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = 0u;
          }
          *gop::box_piece<128>(box + c * kB * 128, lane, h * 2) = make_uint4(w[0], w[1], w[2], w[3]);
          *gop::box_piece<128>(box + c * kB * 128, lane, h * 2 + 1) = make_uint4(w[4], w[5], w[6], w[7]);
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) {
        for (int c = 0; c < panels; ++c) store_heads(&maps.out, box + c * kB * 128, c * 64, head, r0 + x * kB + q * 32, rep);
        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
      }
      if (row < a.tokens)
        a.lse[((int64_t)rep * a.heads + head) * a.tokens + row] = none ? 0.f : fmaf(top * scale2, kLn2, logf(sum));
      __syncwarp();
      uint32_t bad = __ballot_sync(0xffffffffu, !none && !fine);
      while (bad != 0u) {
        const int r = __ffs(bad) - 1;
        bad &= bad - 1;
        forward_row<__nv_bfloat16>(a, rep, head, r0 + x * kB + q * 32 + r);
      }
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

// ---- host side ---------------------------------------------------------------------------------------------------

template <int HD>
cudaError_t launch_forward(const FwdMaps& maps, const Args& a, cudaStream_t st) {
  static uint64_t done = 0;              // one bit per device
  static_assert(Fwd<HD>::kTotal <= 227 * 1024, "shared memory budget");
  const cudaError_t e = allow_dynamic_smem(attention_tc_kernel<HD>, Fwd<HD>::kTotal, &done);
  if (e != cudaSuccess) return e;
  const int64_t tiles = (a.tokens + 2 * kB - 1) / (2 * kB);
  return launch_dep(attention_tc_kernel<HD>, dim3((unsigned)(tiles * a.heads * a.m)), dim3(kFwdThreads), Fwd<HD>::kTotal, st, 1, maps, a);
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
      head_map(&maps.v, a, a.v, a.kv_heads, kB) != cudaSuccess || head_map(&maps.out, a, a.out, a.heads, 32) != cudaSuccess)
    return cudaErrorInvalidValue;
  return a.head_dim <= 64 ? launch_forward<64>(maps, a, st) : launch_forward<128>(maps, a, st);
}

}  // namespace attn
}  // namespace ls
