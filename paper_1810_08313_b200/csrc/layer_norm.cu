// Layer norm of the rows of activation matrices and its gradient (ls_layer_norm, ls_layer_norm_grad).
//
//   y = (x - mean) * rstd * w + b            mean, rstd = 1 / sqrt(var + eps) over the d features of a row
//   dx = rstd * (t - <t> - xhat <t xhat>)    t = dy * w, xhat = (x - mean) * rstd, <.> the mean over the row
//   dw = sum over rows of dy * xhat,  db = sum over rows of dy
//
// Both passes are bound by HBM: forward reads x and writes y, backward reads x and dy and writes dx, each once.  The threads
// of a row (a warp, or a CTA) hold it in registers between its reductions, 16 elements each in pieces of 16 bytes.  Short and
// fp32 forward rows are taken all at once, one per warp or CTA (6.7 TB/s for 16384 x 4096 fp32).  bf16 rows and the backward
// pass have more instructions per byte: there a CTA takes every gridDim.x-th row, so that the parameters are read once per
// CTA, the rows come through a ring in shared memory, filled by bulk copies several rows ahead, and the barrier of a
// row's reduction also says that all its threads have read the row, so its place can be filled again (forward 16384 x
// 4096 bf16 4.9 TB/s, 4.0 without; backward 5.1 TB/s, 4.5 with the next row requested into registers).  Rows that are no
// whole 16 bytes are read element by element.
//
// The variance is the mean square of x - mean with the mean already known (two reductions over the registers, no difference
// of large sums).  All statistics are fp32; a bf16 output is rounded once.
//
// Backward: the sums over rows are split over the CTAs.  Every thread keeps dw and db of its own columns in registers
// over all rows its CTA takes, writes them to the workspace once, and a second kernel adds the CTAs' parts in
// index order: fixed order, no atomics.
#include "gemm_op.cuh"

#include "ls_internal.h"

#include <math.h>

namespace ls {
namespace {

constexpr int kLnMaxWidth = 16384;
constexpr size_t kLnRing = 192 * 1024;    // bytes of the rings of an SM
constexpr int kLnSmemMost = 192 * 1024 + 128;               // (holds the two fp32 rows of the largest width)
constexpr int kLnMaxReplicas = 65535;     // grid.y

template <typename T, int VEC> struct Pack;
template <> struct Pack<float, 4> { float4 v; };
template <> struct Pack<float, 1> { float v; };
template <> struct Pack<__nv_bfloat16, 8> { uint4 v; };
template <> struct Pack<__nv_bfloat16, 1> { __nv_bfloat16 v; };

// fp32 numbers as the arithmetic takes them: two at a time (one instruction for both, each rounded as on its own), or one.
// With scalar instructions a row of 4096 bf16 numbers cost 281 (backward 343) instructions a warp, 16 numbers a lane, and
// the issue slots were 56 % busy at 4.6 (5.0) TB/s.
struct F2 { unsigned long long v; };
struct F1 { float v; };
template <int VEC> struct Num { using type = F2; static constexpr int kPer = 2; };
template <> struct Num<1> { using type = F1; static constexpr int kPer = 1; };

__device__ __forceinline__ F2 make2(float a, float b) {
  F2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void parts(F2 a, float* f) { asm("mov.b64 {%0, %1}, %2;" : "=f"(f[0]), "=f"(f[1]) : "l"(a.v)); }
__device__ __forceinline__ void parts(F1 a, float* f) { f[0] = a.v; }
__device__ __forceinline__ void all(F2& r, float a) { r = make2(a, a); }
__device__ __forceinline__ void all(F1& r, float a) { r.v = a; }
__device__ __forceinline__ F2 add(F2 a, F2 b) { F2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ F2 mul(F2 a, F2 b) { F2 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ F2 fma(F2 a, F2 b, F2 c) {
  F2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}
__device__ __forceinline__ F1 add(F1 a, F1 b) { return F1{a.v + b.v}; }
__device__ __forceinline__ F1 mul(F1 a, F1 b) { return F1{a.v * b.v}; }
__device__ __forceinline__ F1 fma(F1 a, F1 b, F1 c) { return F1{fmaf(a.v, b.v, c.v)}; }
__device__ __forceinline__ float total(F2 a) { float f[2]; parts(a, f); return f[0] + f[1]; }
__device__ __forceinline__ float total(F1 a) { return a.v; }

__device__ __forceinline__ void unpack(const Pack<float, 1>& p, F1* f) { f[0].v = p.v; }
__device__ __forceinline__ void unpack(const Pack<__nv_bfloat16, 1>& p, F1* f) { f[0].v = (float)p.v; }
__device__ __forceinline__ void unpack(const Pack<float, 4>& p, F2* f) {
  f[0] = make2(p.v.x, p.v.y);
  f[1] = make2(p.v.z, p.v.w);
}
__device__ __forceinline__ void unpack(const Pack<__nv_bfloat16, 8>& p, F2* f) {
  const uint32_t w[4] = {p.v.x, p.v.y, p.v.z, p.v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = make2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
}
__device__ __forceinline__ void pack(const F1* f, Pack<float, 1>& p) { p.v = f[0].v; }
__device__ __forceinline__ void pack(const F1* f, Pack<__nv_bfloat16, 1>& p) { p.v = (__nv_bfloat16)f[0].v; }
__device__ __forceinline__ void pack(const F2* f, Pack<float, 4>& p) {
  float a[4];
  parts(f[0], a); parts(f[1], a + 2);
  p.v = make_float4(a[0], a[1], a[2], a[3]);
}
__device__ __forceinline__ void pack(const F2* f, Pack<__nv_bfloat16, 8>& p) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a[2];
    parts(f[i], a);
    w[i] = gop::pack_bf16(a[0], a[1]);
  }
  p.v = make_uint4(w[0], w[1], w[2], w[3]);
}
// VEC fp32 parameters
template <int VEC>
__device__ __forceinline__ void load_param(const float* p, typename Num<VEC>::type* f) {
  if constexpr (VEC == 1) {
    f[0].v = __ldg(p);
  } else {
#pragma unroll
    for (int i = 0; i < VEC / 4; ++i) {
      const float4 v = __ldg(reinterpret_cast<const float4*>(p) + i);
      f[2 * i] = make2(v.x, v.y);
      f[2 * i + 1] = make2(v.z, v.w);
    }
  }
}

// Sums over the NT threads of the CTA of N values; every thread receives them.  Consecutive calls alternate between two
// sets of `red`, so one barrier per call is enough.
template <int NT, int N>
__device__ __forceinline__ void row_sum(float (&v)[N], float (*red)[N]) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
  if constexpr (NT > 32) {
    constexpr int W = NT / 32;
    if ((threadIdx.x & 31) == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) red[threadIdx.x >> 5][i] = v[i];
    }
    __syncthreads();
    // every lane takes one warp's sums and the lanes add them up
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = red[threadIdx.x & (W - 1)][i];
#pragma unroll
    for (int o = W / 2; o > 0; o >>= 1)
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
  }
}

struct LnShape {
  int64_t rows;
  int d;
  int64_t x_stride, dy_stride, y_stride, param_stride;   // elements between replicas (y: the output, y or dx)
  float eps, inv_d;
};

// The rows a CTA takes, one after another: NSRC source matrices, `depth` places in shared memory, then their barriers.
template <typename T, int NSRC>
struct Ring {
  uint8_t* base;
  uint64_t* full;
  const T* src[NSRC];
  int d, depth, place, round;
  uint32_t row_bytes;
  bool ok;
  __device__ __forceinline__ Ring(uint8_t* smem, int d_, int depth_) : base(smem), d(d_), depth(depth_), place(0), round(0), ok(true) {
    row_bytes = (uint32_t)d * sizeof(T);
    full = reinterpret_cast<uint64_t*>(smem + (size_t)depth * NSRC * row_bytes);
    if (depth > 0) {
      if (threadIdx.x == 0) {
        for (int i = 0; i < depth; ++i) ptx::mbar_init(&full[i], 1);
        ptx::fence_mbar_init();
      }
      __syncthreads();
    }
  }
  __device__ __forceinline__ void request(int64_t row, int at) {       // thread 0
    ptx::mbar_expect_tx(&full[at], NSRC * row_bytes);
#pragma unroll
    for (int i = 0; i < NSRC; ++i)
      ptx::bulk_load(base + (size_t)(NSRC * at + i) * row_bytes, src[i] + row * d, row_bytes, &full[at]);
  }
  __device__ __forceinline__ void start(int64_t row, int64_t step, int64_t rows) {
    if (threadIdx.x == 0)
      for (int i = 0; i < depth && row + i * step < rows; ++i) request(row + i * step, i);
  }
  // (a wait that runs out is recorded; the caller goes on with whatever is there, so that every barrier is met)
  __device__ __forceinline__ void wait(int* err) {
    if (ok && !ptx::mbar_wait(&full[place], round & 1)) { ok = false; atomicExch(err, 51); }
  }
  __device__ __forceinline__ const uint8_t* row(int i) const { return base + (size_t)(NSRC * place + i) * row_bytes; }
  // after a barrier that follows every thread's reads of the place
  __device__ __forceinline__ void advance(int64_t row, int64_t step, int64_t rows) {
    if (threadIdx.x == 0 && row + depth * step < rows) request(row + depth * step, place);
    if (++place == depth) { place = 0; ++round; }
  }
  // after a wait that ran out: time for the copies in flight to land before the shared memory is released
  __device__ __forceinline__ void finish() const {
    if (!ok) {
      const long long t0 = clock64();
      while (clock64() - t0 < 4000000ll) {}
    }
  }
};

// ---- forward --------------------------------------------------------------------------------------------------
// RING: a persistent grid with the parameters in registers.  Else a row per CTA (NT == 32: a row per warp, four a CTA), all
// rows at once, the parameters read when they are needed; few registers keep enough CTAs resident.
template <typename T, int VEC, int NT, int EPT, bool RING>
__global__ void __launch_bounds__(NT == 32 && !RING ? 128 : NT)
layer_norm_kernel(const T* __restrict__ x, const float* __restrict__ w, const float* __restrict__ b, T* __restrict__ y,
                  float* __restrict__ mean_out, float* __restrict__ rstd_out, const LnShape s, int depth, int* err) {
  using N = typename Num<VEC>::type;
  constexpr int NCH = EPT / VEC, PC = VEC / Num<VEC>::kPer;      // chunks, numbers of a chunk
  constexpr int RPC = NT == 32 && !RING ? 4 : 1;                 // rows of a CTA at a time
  __shared__ float red[2][NT / 32][1];
  extern __shared__ __align__(128) uint8_t dyn[];
  const int tid = RPC > 1 ? threadIdx.x & 31 : threadIdx.x;
  const int64_t g = blockIdx.y;
  Ring<T, 1> ring(dyn, s.d, RING ? depth : 0);
  grid_dep_wait();
  grid_dep_launch();
  const T* xg = x + g * s.x_stride;
  T* yg = y + g * s.y_stride;
  ring.src[0] = xg;
  const int64_t step = (int64_t)gridDim.x * RPC;
  const int64_t row0 = (int64_t)blockIdx.x * RPC + (RPC > 1 ? threadIdx.x >> 5 : 0);
  if (RING) ring.start(row0, step, s.rows);
  N wv[NCH * PC], bv[NCH * PC];
  auto params = [&](int c, int e) {
#pragma unroll
    for (int i = 0; i < PC; ++i) all(bv[c * PC + i], 0.f);
    load_param<VEC>(w + g * s.param_stride + e, wv + c * PC);
    if (b != nullptr) load_param<VEC>(b + g * s.param_stride + e, bv + c * PC);
  };
  if (RING) {
#pragma unroll
    for (int c = 0; c < NCH; ++c)
      if ((c * NT + tid) * VEC < s.d) params(c, (c * NT + tid) * VEC);
  }
  for (int64_t row = row0; row < s.rows; row += step) {
    N v[NCH * PC], acc;
    all(acc, 0.f);
    if (RING) ring.wait(err);
    const T* xr = RING ? reinterpret_cast<const T*>(ring.row(0)) : xg + row * s.d;
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int e = (c * NT + tid) * VEC;
      if (e < s.d) {
        unpack(*reinterpret_cast<const Pack<T, VEC>*>(xr + e), v + c * PC);
#pragma unroll
        for (int i = 0; i < PC; ++i) acc = add(acc, v[c * PC + i]);
      }
    }
    float sum[1] = {total(acc)};
    row_sum<NT, 1>(sum, red[0]);
    if (RING) ring.advance(row, step, s.rows);
    const float mean = sum[0] * s.inv_d;
    N m;
    all(m, -mean);
    all(acc, 0.f);
#pragma unroll
    for (int c = 0; c < NCH; ++c)
      if ((c * NT + tid) * VEC < s.d) {
#pragma unroll
        for (int i = 0; i < PC; ++i) {
          N& u = v[c * PC + i];
          u = add(u, m);
          acc = fma(u, u, acc);
        }
      }
    sum[0] = total(acc);
    row_sum<NT, 1>(sum, red[1]);
    const float rstd = rsqrtf(fmaf(sum[0], s.inv_d, s.eps));
    if (tid == 0) {
      if (mean_out) mean_out[g * s.rows + row] = mean;
      if (rstd_out) rstd_out[g * s.rows + row] = rstd;
    }
    N r;
    all(r, rstd);
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int e = (c * NT + tid) * VEC;
      if (e < s.d) {
        Pack<T, VEC> o;
        if (!RING) params(c, e);
#pragma unroll
        for (int i = 0; i < PC; ++i) v[c * PC + i] = fma(mul(v[c * PC + i], r), wv[c * PC + i], bv[c * PC + i]);
        pack(v + c * PC, o);
        *reinterpret_cast<Pack<T, VEC>*>(yg + row * s.d + e) = o;
      }
    }
  }
  if (RING) ring.finish();
}

// ---- backward -------------------------------------------------------------------------------------------------
// part: [replica][CTA][2][d] fp32, dw then db of the rows the CTA took.
template <typename T, int VEC, int NT, int EPT>
__global__ void __launch_bounds__(NT)
layer_norm_grad_kernel(const T* __restrict__ dy, const T* __restrict__ x, const float* __restrict__ w,
                       const float* __restrict__ mean_in, const float* __restrict__ rstd_in, T* __restrict__ dx,
                       float* __restrict__ part, const LnShape s, int depth, int* err) {
  using N = typename Num<VEC>::type;
  constexpr int NCH = EPT / VEC, PC = VEC / Num<VEC>::kPer;      // chunks, numbers of a chunk
  constexpr bool RING = VEC > 1;
  __shared__ float red[2][NT / 32][2];
  extern __shared__ __align__(128) uint8_t dyn[];
  const int tid = threadIdx.x;
  const int64_t g = blockIdx.y;
  Ring<T, 2> ring(dyn, s.d, RING ? depth : 0);
  grid_dep_wait();
  grid_dep_launch();
  const T* xg = x + g * s.x_stride;
  const T* dyg = dy + g * s.dy_stride;
  T* dxg = dx + g * s.y_stride;
  ring.src[0] = xg;
  ring.src[1] = dyg;
  const int64_t step = gridDim.x;
  if (RING) ring.start(blockIdx.x, step, s.rows);
  N dw[NCH * PC], db[NCH * PC], wv[NCH * PC];
#pragma unroll
  for (int i = 0; i < NCH * PC; ++i) { all(dw[i], 0.f); all(db[i], 0.f); }
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    const int e = (c * NT + tid) * VEC;
    if (e < s.d) load_param<VEC>(w + g * s.param_stride + e, wv + c * PC);
  }
  float nmean = 0.f, nrstd = 0.f;
  if (blockIdx.x < s.rows) {
    nmean = mean_in[g * s.rows + blockIdx.x];
    nrstd = rstd_in[g * s.rows + blockIdx.x];
  }
  int flip = 0;
  for (int64_t row = blockIdx.x; row < s.rows; row += step) {
    const float rstd = nrstd;
    N m, r, st, sx;
    all(m, -nmean);
    all(r, rstd);
    all(st, 0.f);
    all(sx, 0.f);
    if (row + step < s.rows) {                     // the next row's statistics, ahead of this row's barrier
      nmean = mean_in[g * s.rows + row + step];
      nrstd = rstd_in[g * s.rows + row + step];
    }
    N t[NCH * PC], xh[NCH * PC];
    if (RING) ring.wait(err);
    const T* xr = RING ? reinterpret_cast<const T*>(ring.row(0)) : xg + row * s.d;
    const T* dr = RING ? reinterpret_cast<const T*>(ring.row(1)) : dyg + row * s.d;
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int e = (c * NT + tid) * VEC;
      if (e < s.d) {
        unpack(*reinterpret_cast<const Pack<T, VEC>*>(xr + e), xh + c * PC);
        unpack(*reinterpret_cast<const Pack<T, VEC>*>(dr + e), t + c * PC);
      }
    }
#pragma unroll
    for (int c = 0; c < NCH; ++c)
      if ((c * NT + tid) * VEC < s.d) {
#pragma unroll
        for (int i = 0; i < PC; ++i) {
          const int k = c * PC + i;
          xh[k] = mul(add(xh[k], m), r);
          db[k] = add(db[k], t[k]);
          dw[k] = fma(t[k], xh[k], dw[k]);
          t[k] = mul(t[k], wv[k]);
          st = add(st, t[k]);
          sx = fma(t[k], xh[k], sx);
        }
      }
    float sums[2] = {total(st), total(sx)};
    row_sum<NT, 2>(sums, red[flip]);
    flip ^= 1;
    if (RING) ring.advance(row, step, s.rows);
    N c0, c1;
    all(c0, -sums[0] * s.inv_d * rstd);
    all(c1, -sums[1] * s.inv_d * rstd);
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int e = (c * NT + tid) * VEC;
      if (e < s.d) {
        Pack<T, VEC> o;
#pragma unroll
        for (int i = 0; i < PC; ++i) t[c * PC + i] = fma(t[c * PC + i], r, fma(xh[c * PC + i], c1, c0));
        pack(t + c * PC, o);
        *reinterpret_cast<Pack<T, VEC>*>(dxg + row * s.d + e) = o;
      }
    }
  }
  float* pw = part + (g * gridDim.x + blockIdx.x) * 2 * (int64_t)s.d;
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    const int e = (c * NT + tid) * VEC;
    if (e < s.d) {
#pragma unroll
      for (int i = 0; i < PC; ++i) {
        parts(dw[c * PC + i], pw + e + i * Num<VEC>::kPer);
        parts(db[c * PC + i], pw + s.d + e + i * Num<VEC>::kPer);
      }
    }
  }
  if (RING) ring.finish();
}

// dw, db = sum of the CTAs' parts in index order within a slice, then the slices in order: 32 columns per CTA, 32 warps
// take every 32nd part.  (Columns of dw and db are one axis of 2 d.)
__global__ void __launch_bounds__(1024)
layer_norm_fold_kernel(const float* __restrict__ part, int parts, int d, float* __restrict__ dw, float* __restrict__ db,
                       int64_t param_stride) {
  __shared__ float slice[32][33];
  const int lane = threadIdx.x & 31, wp = threadIdx.x >> 5;
  const int64_t g = blockIdx.y;
  const int col = blockIdx.x * 32 + lane;
  grid_dep_wait();
  grid_dep_launch();
  float s = 0.f;
  if (col < 2 * d) {
    const float* p = part + g * parts * 2 * (int64_t)d + col;
#pragma unroll 8
    for (int i = wp; i < parts; i += 32) s += __ldcg(p + (int64_t)i * 2 * d);
  }
  slice[wp][lane] = s;
  __syncthreads();
  if (wp == 0 && col < 2 * d) {
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) t += slice[i][lane];
    if (col < d) dw[g * param_stride + col] = t;
    else if (db != nullptr) db[g * param_stride + col - d] = t;
  }
}

// ---- host side --------------------------------------------------------------------------------------------------

struct LnArgs {
  const void *dy, *x;
  const float *w, *b, *mean, *rstd;
  void *y;                    // forward: y; backward: dx
  float *mean_out, *rstd_out, *part;
  LnShape s;
  int m;
  unsigned ctas;              // per replica
  bool grad;
};

// How a row of d elements is spread over threads, and over which kernel.
struct LnWay {
  int nt, ept;      // threads of a row, elements of a thread
  bool ring;
  int rpc;          // rows of a CTA at a time
};
// Forward: bf16 rows of more than 2 KB through the ring (16384 x 4096: 55 us, 67 us without), others a CTA or a warp each: a
// fp32 row has twice the bytes per instruction, and 16384 x 4096 runs at 6.7 TB/s that way, 5.7 with the ring; a short row
// costs a CTA of the ring more in barriers than it saves.  Backward: always the ring where rows are whole 16-byte pieces.
LnWay ln_way(int d, bool vec, bool bf16, bool grad) {
  LnWay w{};
  if (!vec) {
    w.nt = d <= 128 ? 32 : d <= 1024 ? 256 : d <= 4096 ? 512 : 1024;
    w.ept = d <= 1024 ? 4 : d <= 4096 ? 8 : 16;
  } else if (grad || (bf16 && d > 1024)) {
    w.ring = true;
    w.nt = d <= 512 ? 32 : d <= 1024 ? 64 : d <= 2048 ? 128 : d <= 4096 ? 256 : d <= 8192 ? 512 : 1024;
    w.ept = 16;
  } else {
    w.nt = d <= 1024 ? 32 : d <= 2048 ? 128 : d <= 4096 ? 256 : d <= 8192 ? 512 : 1024;
    w.ept = d > 512 && d <= 1024 ? 32 : 16;
  }
  w.rpc = w.nt == 32 && !grad && !w.ring ? 4 : 1;
  return w;
}
// CTAs of a persistent launch on every SM: 1024 (backward: 512) threads, 16 CTAs at most
int ln_per_sm(int nt, bool grad) {
  const int n = (grad ? 512 : 1024) / nt;
  return n > 16 ? 16 : n < 1 ? 1 : n;
}

template <typename T, int VEC, int NT, int EPT, bool RING>
cudaError_t launch_ln_fwd(const LnArgs& a, int depth, size_t smem, int* err, cudaStream_t st) {
  static uint64_t configured = 0;        // one bit per device
  auto kern = layer_norm_kernel<T, VEC, NT, EPT, RING>;
  if (RING) {
    const cudaError_t e = allow_dynamic_smem(kern, kLnSmemMost, &configured);
    if (e != cudaSuccess) return e;
  }
  return launch_dep(kern, dim3(a.ctas, (unsigned)a.m), dim3(NT == 32 && !RING ? 128 : NT), smem, st, 1,
                    static_cast<const T*>(a.x), a.w, a.b, static_cast<T*>(a.y), a.mean_out, a.rstd_out, a.s, depth, err);
}
template <typename T, int VEC, int NT, int EPT>
cudaError_t launch_ln_grad(const LnArgs& a, int depth, size_t smem, int* err, cudaStream_t st) {
  static uint64_t configured = 0;        // one bit per device
  auto kern = layer_norm_grad_kernel<T, VEC, NT, EPT>;
  const cudaError_t e = allow_dynamic_smem(kern, kLnSmemMost, &configured);
  if (e != cudaSuccess) return e;
  return launch_dep(kern, dim3(a.ctas, (unsigned)a.m), dim3(NT), smem, st, 1, static_cast<const T*>(a.dy),
                    static_cast<const T*>(a.x), a.w, a.mean, a.rstd, static_cast<T*>(a.y), a.part, a.s, depth, err);
}

template <typename T, int VEC>
cudaError_t pick_ln(const LnArgs& a, const LnWay& way, cudaStream_t st) {
  const size_t per_row = (size_t)(a.grad ? 2 : 1) * a.s.d * sizeof(T);
  // the ring: this CTA's share of 192 KB, eight rows at most, and one row where that is more
  size_t depth = 0;
  if (way.ring) {
    depth = kLnRing / (size_t)ln_per_sm(way.nt, a.grad) / per_row;
    depth = depth > 8 ? 8 : depth < 1 ? 1 : depth;
  }
  const size_t smem = depth * per_row + depth * 8;
  int* err = gop::device_error_word();
  if (err == nullptr) return cudaErrorUnknown;
  const int dep = (int)depth, nt = way.nt;
  if constexpr (VEC == 1) {
    if (!a.grad) {
      if (nt == 32) return launch_ln_fwd<T, 1, 32, 4, false>(a, dep, smem, err, st);
      if (nt == 256) return launch_ln_fwd<T, 1, 256, 4, false>(a, dep, smem, err, st);
      if (nt == 512) return launch_ln_fwd<T, 1, 512, 8, false>(a, dep, smem, err, st);
      return launch_ln_fwd<T, 1, 1024, 16, false>(a, dep, smem, err, st);
    }
    if (nt == 32) return launch_ln_grad<T, 1, 32, 4>(a, dep, smem, err, st);
    if (nt == 256) return launch_ln_grad<T, 1, 256, 4>(a, dep, smem, err, st);
    if (nt == 512) return launch_ln_grad<T, 1, 512, 8>(a, dep, smem, err, st);
    return launch_ln_grad<T, 1, 1024, 16>(a, dep, smem, err, st);
  } else {
    if (!a.grad) {
      constexpr bool R = VEC == 8;       // (beyond 1024 columns)
      if (nt == 32 && way.ept == 16) return launch_ln_fwd<T, VEC, 32, 16, false>(a, dep, smem, err, st);
      if (nt == 32) return launch_ln_fwd<T, VEC, 32, 32, false>(a, dep, smem, err, st);
      if (nt == 128) return launch_ln_fwd<T, VEC, 128, 16, R>(a, dep, smem, err, st);
      if (nt == 256) return launch_ln_fwd<T, VEC, 256, 16, R>(a, dep, smem, err, st);
      if (nt == 512) return launch_ln_fwd<T, VEC, 512, 16, R>(a, dep, smem, err, st);
      return launch_ln_fwd<T, VEC, 1024, 16, R>(a, dep, smem, err, st);
    }
    if (nt == 32) return launch_ln_grad<T, VEC, 32, 16>(a, dep, smem, err, st);
    if (nt == 64) return launch_ln_grad<T, VEC, 64, 16>(a, dep, smem, err, st);
    if (nt == 128) return launch_ln_grad<T, VEC, 128, 16>(a, dep, smem, err, st);
    if (nt == 256) return launch_ln_grad<T, VEC, 256, 16>(a, dep, smem, err, st);
    if (nt == 512) return launch_ln_grad<T, VEC, 512, 16>(a, dep, smem, err, st);
    return launch_ln_grad<T, VEC, 1024, 16>(a, dep, smem, err, st);
  }
}

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// 16-byte accesses need every row and every replica of every tensor to start on a 16-byte boundary.
bool ln_vec(const LnArgs& a, int dtype) {
  const int per = dtype == LS_DTYPE_BF16 ? 8 : 4;
  if (a.s.d % per != 0 || !aligned16(a.x) || !aligned16(a.y) || !aligned16(a.w) || !aligned16(a.b) || !aligned16(a.dy)) return false;
  return a.m == 1 || (a.s.x_stride % per == 0 && a.s.y_stride % per == 0 && a.s.dy_stride % per == 0 && a.s.param_stride % 4 == 0);
}
// CTAs of a replica: one per row (or four rows) for a launch that takes all rows at once; else its share of the resident ones,
// at most one per row (backward: four, so that a CTA's part of the sums is paid for).
unsigned replica_ctas(int m, int64_t rows, const LnWay& way, bool grad) {
  if (!grad && !way.ring) return (unsigned)((rows + way.rpc - 1) / way.rpc);
  const int least = grad ? 4 : 1;
  int64_t want = (148 * (int64_t)ln_per_sm(way.nt, grad) + m - 1) / m;
  const int64_t most = (rows + least - 1) / least;
  if (want > most) want = most;
  return (unsigned)(want < 1 ? 1 : want);
}
// the most parts that a backward call of this size may have (whichever way its rows are read)
unsigned most_parts(int m, int64_t rows, int d) {
  const unsigned a = replica_ctas(m, rows, ln_way(d, true, true, true), true);
  const unsigned b = replica_ctas(m, rows, ln_way(d, false, true, true), true);
  return a > b ? a : b;
}
cudaError_t run_ln(LnArgs& a, int dtype, cudaStream_t st) {
  const bool vec = ln_vec(a, dtype), bf16 = dtype == LS_DTYPE_BF16;
  const LnWay way = ln_way(a.s.d, vec, bf16, a.grad);
  a.ctas = replica_ctas(a.m, a.s.rows, way, a.grad);
  if (bf16) return vec ? pick_ln<__nv_bfloat16, 8>(a, way, st) : pick_ln<__nv_bfloat16, 1>(a, way, st);
  return vec ? pick_ln<float, 4>(a, way, st) : pick_ln<float, 1>(a, way, st);
}

int check_ln(int m, int64_t rows, int d, const LnShape& s, int dtype) {
  if (m < 1 || rows < 0 || d < 1) return LS_ERR_INVALID_ARG;
  if (dtype != LS_DTYPE_FP32 && dtype != LS_DTYPE_BF16) return LS_ERR_INVALID_ARG;
  if (d > kLnMaxWidth || m > kLnMaxReplicas || rows > 2147483647ll) return LS_ERR_TOO_LARGE;
  const int64_t n = rows * d;
  if (m > 1 && (s.x_stride < n || s.y_stride < n || s.dy_stride < n || s.param_stride < d)) return LS_ERR_INVALID_ARG;
  return LS_OK;
}
bool misaligned(const void* p, int dtype) { return reinterpret_cast<uintptr_t>(p) % (dtype == LS_DTYPE_BF16 ? 2 : 4) != 0; }
bool misaligned4(const void* p) { return reinterpret_cast<uintptr_t>(p) % 4 != 0; }

}  // namespace
}  // namespace ls

extern "C" int ls_layer_norm(const void* x_dev, const float* weight_dev, const float* bias_dev, int m, int64_t rows, int d,
                             int64_t x_stride, int64_t param_stride, int dtype, float eps, void* y_dev, int64_t y_stride,
                             float* mean_dev, float* rstd_dev, void* cuda_stream) {
  using namespace ls;
  LnArgs a{};
  a.s = LnShape{rows, d, x_stride, y_stride, y_stride, param_stride, eps, 1.f / (float)d};
  int rc = check_ln(m, rows, d, a.s, dtype);
  if (rc != LS_OK) return rc;
  if (weight_dev == nullptr || !(eps >= 0.f) || !isfinite(eps)) return LS_ERR_INVALID_ARG;
  if (rows > 0 && (x_dev == nullptr || y_dev == nullptr)) return LS_ERR_INVALID_ARG;
  if (misaligned(x_dev, dtype) || misaligned(y_dev, dtype) || misaligned4(weight_dev) || misaligned4(bias_dev) ||
      misaligned4(mean_dev) || misaligned4(rstd_dev))
    return LS_ERR_INVALID_ARG;
  if (rows == 0) return LS_OK;
  a.x = x_dev; a.w = weight_dev; a.b = bias_dev; a.y = y_dev; a.mean_out = mean_dev; a.rstd_out = rstd_dev;
  a.m = m; a.grad = false;
  return run_ln(a, dtype, static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? LS_OK : LS_ERR_CUDA;
}

extern "C" int ls_layer_norm_grad_ws_bytes(int m, int64_t rows, int d, size_t* bytes) {
  using namespace ls;
  const int64_t n = rows * (int64_t)d;
  int rc = check_ln(m, rows, d, LnShape{rows, d, n, n, n, d, 0.f, 1.f}, LS_DTYPE_FP32);
  if (rc != LS_OK) return rc;
  if (bytes == nullptr) return LS_ERR_INVALID_ARG;
  *bytes = (size_t)m * most_parts(m, rows, d) * 2 * (size_t)d * sizeof(float);
  return LS_OK;
}

extern "C" int ls_layer_norm_grad(const void* dy_dev, const void* x_dev, const float* weight_dev, const float* mean_dev,
                                  const float* rstd_dev, int m, int64_t rows, int d, int64_t dy_stride, int64_t x_stride,
                                  int64_t param_stride, int dtype, void* dx_dev, int64_t dx_stride, float* dweight_dev,
                                  float* dbias_dev, int64_t dparam_stride, void* ws_dev, size_t ws_bytes,
                                  void* cuda_stream) {
  using namespace ls;
  LnArgs a{};
  a.s = LnShape{rows, d, x_stride, dy_stride, dx_stride, param_stride, 0.f, 1.f / (float)d};
  int rc = check_ln(m, rows, d, a.s, dtype);
  if (rc != LS_OK) return rc;
  if (weight_dev == nullptr || dweight_dev == nullptr || ws_dev == nullptr || (m > 1 && dparam_stride < d))
    return LS_ERR_INVALID_ARG;
  if (rows > 0 && (dy_dev == nullptr || x_dev == nullptr || mean_dev == nullptr || rstd_dev == nullptr || dx_dev == nullptr))
    return LS_ERR_INVALID_ARG;
  if (misaligned(dy_dev, dtype) || misaligned(x_dev, dtype) || misaligned(dx_dev, dtype) || misaligned4(weight_dev) ||
      misaligned4(mean_dev) || misaligned4(rstd_dev) || misaligned4(dweight_dev) || misaligned4(dbias_dev))
    return LS_ERR_INVALID_ARG;
  size_t need = 0;
  rc = ls_layer_norm_grad_ws_bytes(m, rows, d, &need);
  if (rc != LS_OK) return rc;
  if (ws_bytes < need || reinterpret_cast<uintptr_t>(ws_dev) % 256 != 0) return LS_ERR_STATE_SIZE;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  a.dy = dy_dev; a.x = x_dev; a.w = weight_dev; a.mean = mean_dev; a.rstd = rstd_dev; a.y = dx_dev;
  a.part = static_cast<float*>(ws_dev);
  a.m = m; a.grad = true;
  // (no rows: the sums are those of no parts)
  if (rows > 0 && run_ln(a, dtype, st) != cudaSuccess) return LS_ERR_CUDA;
  const cudaError_t e = launch_dep(layer_norm_fold_kernel, dim3((unsigned)((2 * (int64_t)d + 31) / 32), (unsigned)m), dim3(1024),
                                   0, st, 1, static_cast<const float*>(a.part), rows > 0 ? (int)a.ctas : 0, d, dweight_dev,
                                   dbias_dev, dparam_stride);
  return e == cudaSuccess ? LS_OK : LS_ERR_CUDA;
}
