// RMS norm of every head of q and k with the rotation by position in the same pass, and its gradient (ls_qk_norm_rope,
// ls_qk_norm_rope_grad).
//
//   xhat = x * rstd,  rstd = 1 / sqrt(mean of x^2 over the head + eps),  z = xhat * w
//   y: the pairs (z_a, z_b) of the first rot_dim elements turned by angle = position * inv_freq[pair], the rest as it is
//   dz: the pairs of dy turned back;  dw = sum over rows and heads of dz * xhat;  t = dz * w,  dx = rstd (t - xhat <t xhat>)
//
// Bound by HBM: every element is read once and written once (backward: two read, one written).  A warp takes a token and all
// its heads (or a part of them, where there are few tokens), so that the angles of a token are formed once: a lane keeps the
// cosine and sine of its four pairs and the eight weights that belong to them in registers, and a head takes head_dim / 8
// lanes, two heads of 128 a warp at a time.  The steps of a warp are one sequence over its tokens, in which the loads are a fixed
// number of steps ahead (as raw words: four registers for eight bf16 numbers), also while the angles of the next token are formed.
// Both elements of a pair lie in one lane, so the turn needs no exchange; the sum over a head is a shuffle.  Angles are formed in
// double and reduced by whole turns there: a position of 10^6 leaves an fp32 angle off by 6e-2, and the reduced one by 1e-10
// before it is rounded to fp32.  Heads or rows that are no whole vectors are read element by element, pair l + 32 i in lane l.
#include "ls_internal.h"
#include "tc_ptx.cuh"

#include <math.h>

namespace ls {
namespace {

using ptx::add2;
using ptx::fma2;
using ptx::mul2;
using ptx::parts;
using ptx::two;

constexpr int kNrMaxDim = 256;
constexpr int kNrWarps = 8;              // of a CTA
// CTAs of an SM.  The forward pass of bf16 vectors has registers for three (16384 x 40 heads of 128: 68 us, 74 with two; 78 with two and loads
// eight steps ahead, 74 with four CTAs and two).  That of fp32 spills with three (4096 x 40 heads of 128: 38 us, 32 with two; 16384
// tokens 119 and 120, in neighbouring pairs 133 and 124), and so does the backward pass (bf16 145 us, 107 with two).
constexpr int nr_per_sm(bool vec, bool grad, bool bf16) { return vec && !grad && bf16 ? 3 : 2; }

struct NrTensor { const void* p; int64_t row, replica; };
struct NrArgs {
  NrTensor x[2], dy[2];                  // q, k
  NrTensor out[2];                       // y, or dx
  const float* w[2];
  int64_t w_stride;
  const double* inv_freq;
  const int32_t* positions;              // [m][tokens]
  float* part;                           // backward: [m][ctas][2][head_dim]
  int64_t tokens;
  int m, heads[2], head_dim, rot_dim;
  int parts_log2;                        // warps that share a token's heads: 1 to 8
  float eps;
};

// Where the four pairs of a lane are.  Vectors: A and B are runs of four elements; pairs are (A_i, B_i), or neighbours.
struct Slots {
  int a, b;                              // first elements of the runs (VEC), or unused
  bool live;                             // the lane has elements
};

// elements of pair p (hd: there is none)
template <bool INTER>
__device__ __forceinline__ void pair_at(int p, int hd, int rot, int& x, int& y) {
  const int half = rot / 2;
  if (p < half) {
    x = INTER ? 2 * p : p;
    y = INTER ? x + 1 : p + half;
  } else {
    x = min(2 * p, hd);
    y = min(2 * p + 1, hd);
  }
}

// A lane's eight elements of a head as they lie in memory: two runs of four, or lo[i] and hi[i] of its pairs.
template <typename T, bool VEC> struct Raw;
template <> struct Raw<float, true> { float4 a, b; };
template <> struct Raw<__nv_bfloat16, true> { uint2 a, b; };
template <typename T> struct Raw<T, false> { T lo[4], hi[4]; };

template <typename T, bool VEC, bool INTER>
__device__ __forceinline__ void raw_load(Raw<T, VEC>& r, const T* p, const Slots& s, int lane, int hd, int rot, bool in) {
  if constexpr (VEC) {
    using V = decltype(r.a);
    r.a = in ? *reinterpret_cast<const V*>(p + s.a) : V{};
    r.b = in ? *reinterpret_cast<const V*>(p + s.b) : V{};
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      int x, y;
      pair_at<INTER>(lane + 32 * i, hd, rot, x, y);
      r.lo[i] = in && x < hd ? p[x] : T(0.f);
      r.hi[i] = in && y < hd ? p[y] : T(0.f);
    }
  }
}
__device__ __forceinline__ void four(const float4& t, float (&v)[4]) { v[0] = t.x; v[1] = t.y; v[2] = t.z; v[3] = t.w; }
__device__ __forceinline__ void four(const uint2& t, float (&v)[4]) {
  v[0] = __uint_as_float(t.x << 16); v[1] = __uint_as_float(t.x & 0xFFFF0000u);
  v[2] = __uint_as_float(t.y << 16); v[3] = __uint_as_float(t.y & 0xFFFF0000u);
}
__device__ __forceinline__ float value(float x) { return x; }
__device__ __forceinline__ float value(__nv_bfloat16 x) { return __bfloat162float(x); }
// A lane's pairs: lo of pairs (0, 1) and (2, 3), then hi of them, two numbers to an operand.
struct Pairs { uint64_t lo[2], hi[2]; };
__device__ __forceinline__ Pairs gather(const float (&lo)[4], const float (&hi)[4]) {
  return Pairs{{two(lo[0], lo[1]), two(lo[2], lo[3])}, {two(hi[0], hi[1]), two(hi[2], hi[3])}};
}
template <bool INTER>
__device__ __forceinline__ Pairs from_runs(const float (&a)[4], const float (&b)[4]) {
  if (INTER) return Pairs{{two(a[0], a[2]), two(b[0], b[2])}, {two(a[1], a[3]), two(b[1], b[3])}};
  return Pairs{{two(a[0], a[1]), two(a[2], a[3])}, {two(b[0], b[1]), two(b[2], b[3])}};
}
// (zeros where the lane has none: its raw words start as zeros and are loaded only where it has)
template <typename T, bool VEC, bool INTER>
__device__ __forceinline__ Pairs raw_pairs(const Raw<T, VEC>& r) {
  if constexpr (VEC) {
    float a[4], b[4];
    four(r.a, a);
    four(r.b, b);
    return from_runs<INTER>(a, b);
  } else {
    float lo[4], hi[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) { lo[i] = value(r.lo[i]); hi[i] = value(r.hi[i]); }
    return gather(lo, hi);
  }
}
__device__ __forceinline__ void store4(float* p, float a, float b, float c, float d) { *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d); }
__device__ __forceinline__ void store4(__nv_bfloat16* p, float a, float b, float c, float d) {
  const __nv_bfloat162 u = __floats2bfloat162_rn(a, b), v = __floats2bfloat162_rn(c, d);
  *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&u), *reinterpret_cast<const uint32_t*>(&v));
}
__device__ __forceinline__ void set(float& p, float x) { p = x; }
__device__ __forceinline__ void set(__nv_bfloat16& p, float x) { p = __float2bfloat16_rn(x); }
template <typename T, bool VEC, bool INTER>
__device__ __forceinline__ void store_pairs(T* p, const Slots& s, int lane, int hd, int rot, const Pairs& v) {
  const float2 l0 = parts(v.lo[0]), l1 = parts(v.lo[1]), h0 = parts(v.hi[0]), h1 = parts(v.hi[1]);
  const float lo[4] = {l0.x, l0.y, l1.x, l1.y}, hi[4] = {h0.x, h0.y, h1.x, h1.y};
  if constexpr (VEC) {
    if (INTER) {
      store4(p + s.a, lo[0], hi[0], lo[1], hi[1]);
      store4(p + s.b, lo[2], hi[2], lo[3], hi[3]);
    } else {
      store4(p + s.a, lo[0], lo[1], lo[2], lo[3]);
      store4(p + s.b, hi[0], hi[1], hi[2], hi[3]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      int x, y;
      pair_at<INTER>(lane + 32 * i, hd, rot, x, y);
      if (x < hd) set(p[x], lo[i]);
      if (y < hd) set(p[y], hi[i]);
    }
  }
}

template <int LPR>
__device__ __forceinline__ float head_sum(float x) {
#pragma unroll
  for (int o = LPR / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

// cosines and sines of this lane's pairs at a position (1 and 0 for pairs that are not turned)
__device__ __forceinline__ void angles(const double (&turns)[4], int position, float (&c)[4], float (&s)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const double t = (double)position * turns[i];
    sincospif(2.f * (float)(t - rint(t)), &s[i], &c[i]);
  }
}

// LPR lanes to a head, 32 / LPR heads of a token at a time, U such steps loaded ahead.
template <typename T, bool VEC, bool INTER, int LPR, bool GRAD>
__global__ void __launch_bounds__(kNrWarps * 32, nr_per_sm(VEC, GRAD, sizeof(T) == 2))
qk_norm_rope_kernel(const __grid_constant__ NrArgs a) {
  constexpr int H = 32 / LPR, U = GRAD && (sizeof(T) == 4 || !VEC) ? 2 : 4;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane / LPR, slot = lane % LPR;
  const int hd = a.head_dim, rot = a.rot_dim, half = rot / 2;
  const int rep = blockIdx.y;
  Slots s{};
  s.live = true;
  if (VEC) {
    s.live = slot * 8 < hd;
    const bool split = !INTER && slot * 4 < half;
    s.a = split ? slot * 4 : slot * 8;
    s.b = split ? half + slot * 4 : slot * 8 + 4;
    if (!s.live) s.a = s.b = 0;
  }
  grid_dep_wait();
  grid_dep_launch();
  __shared__ __align__(16) float weight[2][kNrMaxDim];                  // (read four at a time)
  for (int i = threadIdx.x; i < 2 * kNrMaxDim; i += kNrWarps * 32)
    if ((i & (kNrMaxDim - 1)) < hd) weight[i / kNrMaxDim][i & (kNrMaxDim - 1)] = a.w[i / kNrMaxDim][rep * a.w_stride + (i & (kNrMaxDim - 1))];
  // Units are tokens, or parts of them: the parts of a token go to neighbouring warps, so a warp has the same part of every one.
  const int q_steps = (a.heads[0] + H - 1) / H, steps = q_steps + (a.heads[1] + H - 1) / H;
  const int units = (int)a.tokens << a.parts_log2, stride = (int)gridDim.x * kNrWarps;
  const int first_unit = (int)blockIdx.x * kNrWarps + warp, part = first_unit & ((1 << a.parts_log2) - 1);
  const int from = (int)((int64_t)steps * part >> a.parts_log2), upto = (int)((int64_t)steps * (part + 1) >> a.parts_log2);
  // A place in the warp's sequence: step `from` .. `upto` - 1 of a unit, and where its heads are in one or two tensors.  Steps lie
  // beside each other, so only the first one of q, of k and of a unit is looked up.
  struct Place { int unit, step; const T *p, *p2; };
  auto look_up = [&](Place& w, const NrTensor* a1, const NrTensor* a2) {
    const int t = w.step >= q_steps ? 1 : 0, head = (t ? w.step - q_steps : w.step) * H + sub;
    const int64_t token = w.unit >> a.parts_log2;
    w.p = static_cast<const T*>(a1[t].p) + rep * a1[t].replica + token * a1[t].row + head * hd;
    if (GRAD) w.p2 = static_cast<const T*>(a2[t].p) + rep * a2[t].replica + token * a2[t].row + head * hd;
  };
  auto next = [&](Place& w, const NrTensor* a1, const NrTensor* a2) {
    ++w.step;
    w.p += H * hd;
    if (GRAD) w.p2 += H * hd;
    if (w.step == upto) { w.step = from; w.unit += stride; }
    if (w.step == from || w.step == q_steps) look_up(w, a1, a2);
  };
  // whether this lane has a head there (with whole steps: at every place)
  const bool whole = a.heads[0] % H == 0 && a.heads[1] % H == 0;
  auto has = [&](const Place& w) {
    bool in = w.unit < units && s.live;
    if (!whole) {
      const int t = w.step >= q_steps ? 1 : 0;
      in = in && (t ? w.step - q_steps : w.step) * H + sub < a.heads[t];
    }
    return in;
  };
  Raw<T, VEC> x[U], g[GRAD ? U : 1];
  Place ahead{from < upto ? first_unit : units, from, nullptr, nullptr}, now = ahead;
  look_up(ahead, a.x, a.dy);
  look_up(now, a.out, a.out);
  auto load = [&](Raw<T, VEC>& rx, Raw<T, VEC>& rg) {
    const bool in = has(ahead);
    raw_load<T, VEC, INTER>(rx, ahead.p, s, lane, hd, rot, in);
    if (GRAD) raw_load<T, VEC, INTER>(rg, ahead.p2, s, lane, hd, rot, in);
    next(ahead, a.x, a.dy);
  };
#pragma unroll
  for (int u = 0; u < U; ++u) load(x[u], g[GRAD ? u : 0]);
  double turns[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int p = VEC ? slot * 4 + i : lane + 32 * i;
    turns[i] = p < half && s.live ? a.inv_freq[p] * 0.15915494309189533577 : 0.0;
  }
  Pairs dw[2] = {};
  __syncthreads();
  const float inv = 1.f / (float)hd;
  Pairs cs{};                            // cosines and sines of the pairs, for the unit `angle_of`
  int angle_of = -1;
  while (now.unit < units) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (now.unit >= units) break;
      if (now.unit != angle_of) {
        angle_of = now.unit;
        float c[4], sn[4];
        angles(turns, half > 0 ? a.positions[rep * a.tokens + (now.unit >> a.parts_log2)] : 0, c, sn);
        cs = gather(c, sn);
      }
      const int t = now.step >= q_steps ? 1 : 0;
      const bool in = has(now);
      Pairs v = raw_pairs<T, VEC, INTER>(x[u]), d{};
      if (GRAD) d = raw_pairs<T, VEC, INTER>(g[GRAD ? u : 0]);
      load(x[u], g[GRAD ? u : 0]);
      Pairs w;
      if constexpr (VEC) {
        float va[4], vb[4];
        four(*reinterpret_cast<const float4*>(&weight[t][s.a]), va);
        four(*reinterpret_cast<const float4*>(&weight[t][s.b]), vb);
        w = from_runs<INTER>(va, vb);
      } else {
        float wl[4], wh[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          int e, f;
          pair_at<INTER>(lane + 32 * i, hd, rot, e, f);
          wl[i] = e < hd ? weight[t][e] : 0.f;
          wh[i] = f < hd ? weight[t][f] : 0.f;
        }
        w = gather(wl, wh);
      }
      const float2 sq = parts(fma2(v.lo[0], v.lo[0], fma2(v.lo[1], v.lo[1], fma2(v.hi[0], v.hi[0], mul2(v.hi[1], v.hi[1])))));
      const float rstd = rsqrtf(fmaf(head_sum<LPR>(sq.x + sq.y), inv, a.eps));
      const uint64_t r2 = two(rstd, rstd), minus = two(-1.f, -1.f);
      if (!GRAD) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint64_t p = mul2(mul2(v.lo[i], r2), w.lo[i]), q = mul2(mul2(v.hi[i], r2), w.hi[i]);
          v.lo[i] = fma2(p, cs.lo[i], mul2(mul2(q, minus), cs.hi[i]));
          v.hi[i] = fma2(p, cs.hi[i], mul2(q, cs.lo[i]));
        }
      } else {
        uint64_t along2 = 0;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          v.lo[i] = mul2(v.lo[i], r2);
          v.hi[i] = mul2(v.hi[i], r2);
          const uint64_t p = fma2(d.lo[i], cs.lo[i], mul2(d.hi[i], cs.hi[i]));
          const uint64_t q = fma2(d.hi[i], cs.lo[i], mul2(mul2(d.lo[i], minus), cs.hi[i]));
          if (in) {                        // (outside, eps = 0 makes xhat 0 / 0)
            if (t) {
              dw[1].lo[i] = fma2(p, v.lo[i], dw[1].lo[i]);
              dw[1].hi[i] = fma2(q, v.hi[i], dw[1].hi[i]);
            } else {
              dw[0].lo[i] = fma2(p, v.lo[i], dw[0].lo[i]);
              dw[0].hi[i] = fma2(q, v.hi[i], dw[0].hi[i]);
            }
          }
          d.lo[i] = mul2(p, w.lo[i]);
          d.hi[i] = mul2(q, w.hi[i]);
          along2 = fma2(d.lo[i], v.lo[i], fma2(d.hi[i], v.hi[i], along2));
        }
        const float2 al = parts(along2);
        const float along = -head_sum<LPR>(al.x + al.y) * inv;
        const uint64_t a2 = two(along, along);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          v.lo[i] = mul2(r2, fma2(v.lo[i], a2, d.lo[i]));
          v.hi[i] = mul2(r2, fma2(v.hi[i], a2, d.hi[i]));
        }
      }
      if (in) store_pairs<T, VEC, INTER>(const_cast<T*>(now.p), s, lane, hd, rot, v);
      next(now, a.out, a.out);
    }
  }
  if constexpr (GRAD) {
    // this CTA's part of dw: the lanes that share a pair, then the warps, in order
    __shared__ float sum[kNrWarps][kNrMaxDim];
    float* part = a.part + ((int64_t)rep * gridDim.x + blockIdx.x) * 2 * hd;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const float2 l0 = parts(dw[t].lo[0]), l1 = parts(dw[t].lo[1]), h0 = parts(dw[t].hi[0]), h1 = parts(dw[t].hi[1]);
      float dwl[4] = {l0.x, l0.y, l1.x, l1.y}, dwh[4] = {h0.x, h0.y, h1.x, h1.y};
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int o = LPR; o < 32; o <<= 1) {
          dwl[i] += __shfl_xor_sync(0xffffffffu, dwl[i], o);
          dwh[i] += __shfl_xor_sync(0xffffffffu, dwh[i], o);
        }
        int x, y;
        pair_at<INTER>(VEC ? slot * 4 + i : lane + 32 * i, hd, rot, x, y);
        if (VEC && !INTER && slot * 4 >= half) { x = s.a + i; y = s.b + i; }
        if (sub == 0 && s.live) {
          if (x < hd) sum[warp][x] = dwl[i];
          if (y < hd) sum[warp][y] = dwh[i];
        }
      }
      __syncthreads();
      if ((int)threadIdx.x < hd) {
        float total = 0.f;
#pragma unroll
        for (int w = 0; w < kNrWarps; ++w) total += sum[w][threadIdx.x];
        part[t * hd + threadIdx.x] = total;
      }
    }
  }
}

// dw = sum of the CTAs' parts, every 32nd by one warp, then the warps in order.  (Columns of dw_q and dw_k are one axis.)
__global__ void __launch_bounds__(1024)
qk_norm_fold_kernel(const float* __restrict__ part, int parts, int hd, float* __restrict__ dwq, float* __restrict__ dwk, int64_t stride) {
  __shared__ float slice[32][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
  const int64_t rep = blockIdx.y;
  grid_dep_wait();
  grid_dep_launch();
  float s = 0.f;
  if (col < 2 * hd) {
    const float* p = part + rep * parts * 2 * hd + col;
#pragma unroll 8
    for (int i = warp; i < parts; i += 32) s += __ldcg(p + (int64_t)i * 2 * hd);
  }
  slice[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && col < 2 * hd) {
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) t += slice[i][lane];
    if (col < hd) dwq[rep * stride + col] = t;
    else dwk[rep * stride + col - hd] = t;
  }
}

// ---- host side ---------------------------------------------------------------------------------------------------

// CTAs of a replica: its share of those that are resident, and no more than there are warps' units (tokens, or parts of them) for
unsigned nr_ctas(int m, int64_t units, int per_sm) {
  const int64_t most = (units + kNrWarps - 1) / kNrWarps;
  int64_t n = (148 * per_sm + m - 1) / m;
  n = n > most ? most : n;
  return (unsigned)(n < 1 ? 1 : n);
}

template <typename T, bool VEC, bool INTER, int LPR>
cudaError_t nr_launch(NrArgs& a, bool grad, unsigned ctas, cudaStream_t st) {
  if (grad) return launch_dep(qk_norm_rope_kernel<T, VEC, INTER, LPR, true>, dim3(ctas, (unsigned)a.m), dim3(kNrWarps * 32), 0, st, 1, a);
  return launch_dep(qk_norm_rope_kernel<T, VEC, INTER, LPR, false>, dim3(ctas, (unsigned)a.m), dim3(kNrWarps * 32), 0, st, 1, a);
}
template <typename T, bool INTER>
cudaError_t nr_pick(NrArgs& a, bool vec, bool grad, unsigned ctas, cudaStream_t st) {
  if (!vec) return nr_launch<T, false, INTER, 32>(a, grad, ctas, st);
  const int slots = a.head_dim / 8;
  if (slots <= 4) return nr_launch<T, true, INTER, 4>(a, grad, ctas, st);
  if (slots <= 8) return nr_launch<T, true, INTER, 8>(a, grad, ctas, st);
  if (slots <= 16) return nr_launch<T, true, INTER, 16>(a, grad, ctas, st);
  return nr_launch<T, true, INTER, 32>(a, grad, ctas, st);
}

int nr_check(int m, int64_t tokens, int heads, int kv_heads, int head_dim, int rot_dim, int dtype) {
  if (m < 1 || tokens < 0 || heads < 1 || kv_heads < 1 || head_dim < 1 || rot_dim < 0 || rot_dim > head_dim || rot_dim % 2 != 0)
    return LS_ERR_INVALID_ARG;
  if (dtype != LS_DTYPE_FP32 && dtype != LS_DTYPE_BF16) return LS_ERR_INVALID_ARG;
  if (m > 65535 || tokens > (1ll << 30) || heads > 65536 || kv_heads > 65536 || head_dim > kNrMaxDim) return LS_ERR_TOO_LARGE;
  return LS_OK;
}
bool nr_bad(const NrArgs& a, const NrTensor& t, int heads, int dtype) {
  const int64_t width = (int64_t)heads * a.head_dim;
  if (reinterpret_cast<uintptr_t>(t.p) % (dtype == LS_DTYPE_BF16 ? 2 : 4) != 0) return true;
  if (a.tokens == 0) return false;
  if (t.p == nullptr || (a.tokens > 1 && t.row < width) || t.row > (1ll << 40) / a.tokens) return true;
  return a.m > 1 && t.replica < (a.tokens - 1) * (a.tokens > 1 ? t.row : 0) + width;
}
// runs of four elements need every row of every tensor to start on their boundary, and the pairs to come in fours
bool nr_vec(const NrArgs& a, int dtype, bool grad) {
  if (a.head_dim % 8 != 0 || a.rot_dim % 8 != 0) return false;
  const uintptr_t bytes = dtype == LS_DTYPE_BF16 ? 8 : 16;
  for (int t = 0; t < 2; ++t)
    for (const NrTensor* x : {&a.x[t], &a.out[t], grad ? &a.dy[t] : &a.x[t]})
      if (reinterpret_cast<uintptr_t>(x->p) % bytes != 0 || (a.tokens > 1 && x->row % 4 != 0) || (a.m > 1 && x->replica % 4 != 0))
        return false;
  return true;
}
cudaError_t nr_run(NrArgs& a, int dtype, bool interleaved, bool grad, unsigned ctas, cudaStream_t st) {
  const bool vec = nr_vec(a, dtype, grad);
  if (dtype == LS_DTYPE_BF16)
    return interleaved ? nr_pick<__nv_bfloat16, true>(a, vec, grad, ctas, st) : nr_pick<__nv_bfloat16, false>(a, vec, grad, ctas, st);
  return interleaved ? nr_pick<float, true>(a, vec, grad, ctas, st) : nr_pick<float, false>(a, vec, grad, ctas, st);
}
bool nr_misaligned(const void* p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n != 0; }

}  // namespace
}  // namespace ls

extern "C" int ls_qk_norm_rope(const void* q_dev, const void* k_dev, const float* q_weight_dev, const float* k_weight_dev,
                               const int32_t* positions_dev, const double* inv_freq_dev, int m, int64_t tokens, int heads,
                               int kv_heads, int head_dim, int rot_dim, int interleaved, int64_t q_row, int64_t k_row,
                               int64_t q_stride, int64_t k_stride, int64_t weight_stride, int dtype, float eps, void* q_out_dev,
                               void* k_out_dev, int64_t q_out_row, int64_t k_out_row, int64_t q_out_stride, int64_t k_out_stride,
                               void* cuda_stream) {
  using namespace ls;
  int rc = nr_check(m, tokens, heads, kv_heads, head_dim, rot_dim, dtype);
  if (rc != LS_OK) return rc;
  NrArgs a{};
  a.m = m; a.tokens = tokens; a.heads[0] = heads; a.heads[1] = kv_heads; a.head_dim = head_dim; a.rot_dim = rot_dim; a.eps = eps;
  a.x[0] = NrTensor{q_dev, q_row, q_stride};
  a.x[1] = NrTensor{k_dev, k_row, k_stride};
  a.out[0] = NrTensor{q_out_dev, q_out_row, q_out_stride};
  a.out[1] = NrTensor{k_out_dev, k_out_row, k_out_stride};
  a.w[0] = q_weight_dev; a.w[1] = k_weight_dev; a.w_stride = m > 1 ? weight_stride : 0;
  a.positions = positions_dev; a.inv_freq = inv_freq_dev;
  if (!(eps >= 0.f) || !isfinite(eps) || interleaved < 0 || interleaved > 1 || q_weight_dev == nullptr || k_weight_dev == nullptr ||
      (m > 1 && weight_stride < head_dim) || (rot_dim > 0 && tokens > 0 && (positions_dev == nullptr || inv_freq_dev == nullptr)))
    return LS_ERR_INVALID_ARG;
  for (int t = 0; t < 2; ++t)
    if (nr_bad(a, a.x[t], a.heads[t], dtype) || nr_bad(a, a.out[t], a.heads[t], dtype)) return LS_ERR_INVALID_ARG;
  if (nr_misaligned(q_weight_dev, 4) || nr_misaligned(k_weight_dev, 4) || nr_misaligned(positions_dev, 4) || nr_misaligned(inv_freq_dev, 8))
    return LS_ERR_INVALID_ARG;
  if (tokens == 0) return LS_OK;
  // few tokens: their heads are shared out over several warps, up to eight
  while (a.parts_log2 < 3 && (m * tokens << a.parts_log2) < 148 * 16) ++a.parts_log2;
  const unsigned ctas = nr_ctas(m, tokens << a.parts_log2, nr_per_sm(nr_vec(a, dtype, false), false, dtype == LS_DTYPE_BF16));
  return nr_run(a, dtype, interleaved != 0, false, ctas, static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? LS_OK : LS_ERR_CUDA;
}

extern "C" int ls_qk_norm_rope_grad_ws_bytes(int m, int64_t tokens, int head_dim, size_t* bytes) {
  using namespace ls;
  const int rc = nr_check(m, tokens, 1, 1, head_dim, 0, LS_DTYPE_FP32);
  if (rc != LS_OK) return rc;
  if (bytes == nullptr) return LS_ERR_INVALID_ARG;
  *bytes = (size_t)m * nr_ctas(m, tokens, nr_per_sm(true, true, true)) * 2 * (size_t)head_dim * sizeof(float);
  return LS_OK;
}

extern "C" int ls_qk_norm_rope_grad(const void* dq_out_dev, const void* dk_out_dev, const void* q_dev, const void* k_dev,
                                    const float* q_weight_dev, const float* k_weight_dev, const int32_t* positions_dev,
                                    const double* inv_freq_dev, int m, int64_t tokens, int heads, int kv_heads, int head_dim,
                                    int rot_dim, int interleaved, int64_t dq_out_row, int64_t dk_out_row, int64_t q_row, int64_t k_row,
                                    int64_t dq_out_stride, int64_t dk_out_stride, int64_t q_stride, int64_t k_stride,
                                    int64_t weight_stride, int dtype, float eps, void* dq_dev, void* dk_dev, int64_t dq_row,
                                    int64_t dk_row, int64_t dq_stride, int64_t dk_stride, float* dq_weight_dev, float* dk_weight_dev,
                                    int64_t dweight_stride, void* ws_dev, size_t ws_bytes, void* cuda_stream) {
  using namespace ls;
  int rc = nr_check(m, tokens, heads, kv_heads, head_dim, rot_dim, dtype);
  if (rc != LS_OK) return rc;
  NrArgs a{};
  a.m = m; a.tokens = tokens; a.heads[0] = heads; a.heads[1] = kv_heads; a.head_dim = head_dim; a.rot_dim = rot_dim; a.eps = eps;
  a.dy[0] = NrTensor{dq_out_dev, dq_out_row, dq_out_stride};
  a.dy[1] = NrTensor{dk_out_dev, dk_out_row, dk_out_stride};
  a.x[0] = NrTensor{q_dev, q_row, q_stride};
  a.x[1] = NrTensor{k_dev, k_row, k_stride};
  a.out[0] = NrTensor{dq_dev, dq_row, dq_stride};
  a.out[1] = NrTensor{dk_dev, dk_row, dk_stride};
  a.w[0] = q_weight_dev; a.w[1] = k_weight_dev; a.w_stride = m > 1 ? weight_stride : 0;
  a.positions = positions_dev; a.inv_freq = inv_freq_dev;
  if (!(eps >= 0.f) || !isfinite(eps) || interleaved < 0 || interleaved > 1 || q_weight_dev == nullptr || k_weight_dev == nullptr ||
      dq_weight_dev == nullptr || dk_weight_dev == nullptr || ws_dev == nullptr ||
      (m > 1 && (weight_stride < head_dim || dweight_stride < head_dim)) ||
      (rot_dim > 0 && tokens > 0 && (positions_dev == nullptr || inv_freq_dev == nullptr)))
    return LS_ERR_INVALID_ARG;
  for (int t = 0; t < 2; ++t)
    if (nr_bad(a, a.x[t], a.heads[t], dtype) || nr_bad(a, a.dy[t], a.heads[t], dtype) || nr_bad(a, a.out[t], a.heads[t], dtype))
      return LS_ERR_INVALID_ARG;
  if (nr_misaligned(q_weight_dev, 4) || nr_misaligned(k_weight_dev, 4) || nr_misaligned(positions_dev, 4) ||
      nr_misaligned(inv_freq_dev, 8) || nr_misaligned(dq_weight_dev, 4) || nr_misaligned(dk_weight_dev, 4))
    return LS_ERR_INVALID_ARG;
  size_t need = 0;
  rc = ls_qk_norm_rope_grad_ws_bytes(m, tokens, head_dim, &need);
  if (rc != LS_OK) return rc;
  if (ws_bytes < need || reinterpret_cast<uintptr_t>(ws_dev) % 256 != 0) return LS_ERR_STATE_SIZE;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  a.part = static_cast<float*>(ws_dev);
  const unsigned ctas = nr_ctas(m, tokens, nr_per_sm(true, true, true));
  // (no tokens: the sums are those of no parts)
  if (tokens > 0 && nr_run(a, dtype, interleaved != 0, true, ctas, st) != cudaSuccess) return LS_ERR_CUDA;
  const cudaError_t e = launch_dep(qk_norm_fold_kernel, dim3((unsigned)((2 * head_dim + 31) / 32), (unsigned)m), dim3(1024), 0, st, 1,
                                   static_cast<const float*>(a.part), tokens > 0 ? (int)ctas : 0, head_dim, dq_weight_dev,
                                   dk_weight_dev, dweight_stride);
  return e == cudaSuccess ? LS_OK : LS_ERR_CUDA;
}
