// Layer norm of the rows of activation matrices and its gradient (ls_layer_norm, ls_layer_norm_grad).
//
//   y = (x - mean) * rstd * w + b            mean, rstd = 1 / sqrt(var + eps) over the d features of a row
//   dx = rstd * (t - <t> - xhat <t xhat>)    t = dy * w, xhat = (x - mean) * rstd, <.> the mean over the row
//   dw = sum over rows of dy * xhat,  db = sum over rows of dy
//
// Both passes are bound by HBM: forward reads x and writes y, backward reads x and dy and writes dx, each once.  A row
// therefore stays in registers between its reductions: NT threads (a warp, or a whole CTA) hold EPT elements each, in
// pieces of 16 bytes that a warp reads side by side.  The variance is the mean square of x - mean with the mean
// already known (two reductions over the registers, no difference of large sums).  All statistics are fp32; a bf16
// output is rounded once.
//
// Backward: the sums over rows are split over the CTAs of a persistent grid.  Every thread keeps dw and db of its own
// columns in registers over all rows its CTA takes, writes them to the workspace once, and a second kernel adds the
// CTAs' parts in index order: fixed order, no atomics.  The next row is requested before the reductions of the current
// one, so that the loads do not wait for the two barriers of a row.
#include "ls_internal.h"

#include <math.h>

namespace ls {
namespace {

constexpr int kLnMaxWidth = 16384;
constexpr int kLnMaxReplicas = 65535;     // grid.y

template <typename T, int VEC> struct Pack;
template <> struct Pack<float, 4> { float4 v; };
template <> struct Pack<float, 1> { float v; };
template <> struct Pack<__nv_bfloat16, 8> { uint4 v; };
template <> struct Pack<__nv_bfloat16, 1> { __nv_bfloat16 v; };

template <typename T, int VEC>
__device__ __forceinline__ void unpack(const Pack<T, VEC>& p, float* f) {
  if constexpr (VEC == 1) {
    f[0] = (float)p.v;
  } else if constexpr (VEC == 4) {
    f[0] = p.v.x; f[1] = p.v.y; f[2] = p.v.z; f[3] = p.v.w;
  } else {
    const uint32_t w[4] = {p.v.x, p.v.y, p.v.z, p.v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
}
template <typename T, int VEC>
__device__ __forceinline__ Pack<T, VEC> pack(const float* f) {
  Pack<T, VEC> p;
  if constexpr (VEC == 1) {
    p.v = (T)f[0];
  } else if constexpr (VEC == 4) {
    p.v = make_float4(f[0], f[1], f[2], f[3]);
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      __nv_bfloat162 t = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
      w[i] = *reinterpret_cast<uint32_t*>(&t);
    }
    p.v = make_uint4(w[0], w[1], w[2], w[3]);
  }
  return p;
}
// VEC fp32 parameters
template <int VEC>
__device__ __forceinline__ void load_param(const float* p, float* f) {
  if constexpr (VEC == 1) {
    f[0] = __ldg(p);
  } else {
#pragma unroll
    for (int i = 0; i < VEC / 4; ++i) {
      const float4 v = __ldg(reinterpret_cast<const float4*>(p) + i);
      f[4 * i] = v.x; f[4 * i + 1] = v.y; f[4 * i + 2] = v.z; f[4 * i + 3] = v.w;
    }
  }
}

// Sum of (a, b) over the NT threads that share a row; every one of them receives it.  `red` holds 2 * NT / 32 floats
// per set; consecutive calls alternate between two sets, so one barrier per call is enough.
template <int NT>
__device__ __forceinline__ float2 row_sum(float a, float b, float2* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    a += __shfl_xor_sync(0xffffffffu, a, o);
    b += __shfl_xor_sync(0xffffffffu, b, o);
  }
  if constexpr (NT > 32) {
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = make_float2(a, b);
    __syncthreads();
    a = b = 0.f;
#pragma unroll
    for (int i = 0; i < NT / 32; ++i) {
      const float2 v = red[i];
      a += v.x; b += v.y;
    }
  }
  return make_float2(a, b);
}

struct LnShape {
  int64_t rows;
  int d;
  int64_t x_stride, dy_stride, y_stride, param_stride;   // elements between replicas (y: the output, y or dx)
  float eps;
};

// ---- forward --------------------------------------------------------------------------------------------------
// NT == 32: a warp per row, four rows per CTA.  NT > 32: a CTA per row.
template <typename T, int VEC, int NT, int EPT>
__global__ void __launch_bounds__(NT == 32 ? 128 : NT)
layer_norm_kernel(const T* __restrict__ x, const float* __restrict__ w, const float* __restrict__ b, T* __restrict__ y,
                  float* __restrict__ mean_out, float* __restrict__ rstd_out, const LnShape s) {
  constexpr int NCH = EPT / VEC;
  __shared__ float2 red[2][NT > 32 ? NT / 32 : 1];
  const int tid = NT == 32 ? (threadIdx.x & 31) : threadIdx.x;
  const int64_t row = NT == 32 ? (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5) : (int64_t)blockIdx.x;
  const int64_t g = blockIdx.y;
  grid_dep_wait();
  grid_dep_launch();
  if (row >= s.rows) return;                       // (whole warps: a CTA per row never takes this)
  const T* xr = x + g * s.x_stride + row * s.d;
  float v[EPT];
  float sum = 0.f;
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    const int e = (c * NT + tid) * VEC;
    if (e < s.d) {
      unpack<T, VEC>(*reinterpret_cast<const Pack<T, VEC>*>(xr + e), v + c * VEC);
#pragma unroll
      for (int i = 0; i < VEC; ++i) sum += v[c * VEC + i];
    }
  }
  const float mean = row_sum<NT>(sum, 0.f, red[0]).x / (float)s.d;
  float sq = 0.f;
#pragma unroll
  for (int c = 0; c < NCH; ++c)
    if ((c * NT + tid) * VEC < s.d) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        v[c * VEC + i] -= mean;
        sq = fmaf(v[c * VEC + i], v[c * VEC + i], sq);
      }
    }
  const float var = row_sum<NT>(sq, 0.f, red[1]).x / (float)s.d;
  const float rstd = 1.0f / sqrtf(var + s.eps);
  if (tid == 0) {
    if (mean_out) mean_out[g * s.rows + row] = mean;
    if (rstd_out) rstd_out[g * s.rows + row] = rstd;
  }
  T* yr = y + g * s.y_stride + row * s.d;
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    const int e = (c * NT + tid) * VEC;
    if (e < s.d) {
      float wv[VEC], bv[VEC], o[VEC];
      load_param<VEC>(w + g * s.param_stride + e, wv);
      if (b != nullptr) load_param<VEC>(b + g * s.param_stride + e, bv);
#pragma unroll
      for (int i = 0; i < VEC; ++i) o[i] = fmaf(v[c * VEC + i] * rstd, wv[i], b != nullptr ? bv[i] : 0.f);
      *reinterpret_cast<Pack<T, VEC>*>(yr + e) = pack<T, VEC>(o);
    }
  }
}

// ---- backward -------------------------------------------------------------------------------------------------
// part: [replica][CTA][2][d] fp32, dw then db of the rows the CTA took.  CTA `blockIdx.x` of `gridDim.x` takes every
// gridDim.x-th row (NT == 32: every warp of the grid a row).
template <typename T, int VEC, int NT, int EPT>
__global__ void __launch_bounds__(NT == 32 ? 128 : NT, 1)
layer_norm_grad_kernel(const T* __restrict__ dy, const T* __restrict__ x, const float* __restrict__ w,
                       const float* __restrict__ mean_in, const float* __restrict__ rstd_in, T* __restrict__ dx,
                       float* __restrict__ part, const LnShape s) {
  constexpr int NCH = EPT / VEC;
  constexpr int RPC = NT == 32 ? 4 : 1;            // rows in flight per CTA
  __shared__ float2 red[2][NT > 32 ? NT / 32 : 1];
  extern __shared__ float fold[];                  // NT == 32: [3][2][d] sums of warps 1..3
  const int tid = NT == 32 ? (threadIdx.x & 31) : threadIdx.x;
  const int sub = NT == 32 ? (threadIdx.x >> 5) : 0;
  const int64_t g = blockIdx.y;
  grid_dep_wait();
  grid_dep_launch();
  float dw[EPT], db[EPT];
#pragma unroll
  for (int i = 0; i < EPT; ++i) dw[i] = db[i] = 0.f;
  const T* xg = x + g * s.x_stride;
  const T* dyg = dy + g * s.dy_stride;
  T* dxg = dx + g * s.y_stride;
  const float* wg = w + g * s.param_stride;
  const int64_t step = (int64_t)gridDim.x * RPC;
  int64_t row = (int64_t)blockIdx.x * RPC + sub;
  Pack<T, VEC> px[NCH], pd[NCH];
  float pmean = 0.f, prstd = 0.f;
  if (row < s.rows) {
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int e = (c * NT + tid) * VEC;
      if (e < s.d) {
        px[c] = *reinterpret_cast<const Pack<T, VEC>*>(xg + row * s.d + e);
        pd[c] = *reinterpret_cast<const Pack<T, VEC>*>(dyg + row * s.d + e);
      }
    }
    pmean = mean_in[g * s.rows + row];
    prstd = rstd_in[g * s.rows + row];
  }
  int flip = 0;
  for (; row < s.rows; row += step) {
    const float mean = pmean, rstd = prstd;
    float t[EPT], xh[EPT];
    float st = 0.f, sx = 0.f;
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int e = (c * NT + tid) * VEC;
      if (e < s.d) {
        float wv[VEC];
        load_param<VEC>(wg + e, wv);
        unpack<T, VEC>(px[c], xh + c * VEC);
        unpack<T, VEC>(pd[c], t + c * VEC);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          const int k = c * VEC + i;
          xh[k] = (xh[k] - mean) * rstd;
          db[k] += t[k];
          dw[k] = fmaf(t[k], xh[k], dw[k]);
          t[k] *= wv[i];
          st += t[k];
          sx = fmaf(t[k], xh[k], sx);
        }
      }
    }
    // the next row, before the barriers of this one
    const int64_t next = row + step;
    if (next < s.rows) {
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        const int e = (c * NT + tid) * VEC;
        if (e < s.d) {
          px[c] = *reinterpret_cast<const Pack<T, VEC>*>(xg + next * s.d + e);
          pd[c] = *reinterpret_cast<const Pack<T, VEC>*>(dyg + next * s.d + e);
        }
      }
      pmean = mean_in[g * s.rows + next];
      prstd = rstd_in[g * s.rows + next];
    }
    const float2 sums = row_sum<NT>(st, sx, red[flip]);
    flip ^= 1;
    const float mt = sums.x / (float)s.d, mx = sums.y / (float)s.d;
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int e = (c * NT + tid) * VEC;
      if (e < s.d) {
        float o[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) o[i] = (t[c * VEC + i] - mt - xh[c * VEC + i] * mx) * rstd;
        *reinterpret_cast<Pack<T, VEC>*>(dxg + row * s.d + e) = pack<T, VEC>(o);
      }
    }
  }
  if constexpr (NT == 32) {
    // the four warps' sums, added in warp order
    if (sub > 0) {
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        const int e = (c * NT + tid) * VEC;
        if (e < s.d) {
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            fold[((sub - 1) * 2) * s.d + e + i] = dw[c * VEC + i];
            fold[((sub - 1) * 2 + 1) * s.d + e + i] = db[c * VEC + i];
          }
        }
      }
    }
    __syncthreads();
    if (sub > 0) return;
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int e = (c * NT + tid) * VEC;
      if (e < s.d) {
#pragma unroll
        for (int i = 0; i < VEC; ++i)
#pragma unroll
          for (int r = 0; r < 3; ++r) {
            dw[c * VEC + i] += fold[(r * 2) * s.d + e + i];
            db[c * VEC + i] += fold[(r * 2 + 1) * s.d + e + i];
          }
      }
    }
  }
  float* pw = part + (g * gridDim.x + blockIdx.x) * 2 * (int64_t)s.d;
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    const int e = (c * NT + tid) * VEC;
    if (e < s.d) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        pw[e + i] = dw[c * VEC + i];
        pw[s.d + e + i] = db[c * VEC + i];
      }
    }
  }
}

// dw, db = sum of the CTAs' parts in index order within a slice, then the slices in order: 32 columns per CTA, 16 warps
// take every 16th part.  (Columns of dw and db are one axis of 2 d.)
__global__ void __launch_bounds__(512)
layer_norm_fold_kernel(const float* __restrict__ part, int parts, int d, float* __restrict__ dw, float* __restrict__ db,
                       int64_t param_stride) {
  __shared__ float slice[16][33];
  const int lane = threadIdx.x & 31, wp = threadIdx.x >> 5;
  const int64_t g = blockIdx.y;
  const int col = blockIdx.x * 32 + lane;
  grid_dep_wait();
  grid_dep_launch();
  float s = 0.f;
  if (col < 2 * d) {
    const float* p = part + g * parts * 2 * (int64_t)d + col;
#pragma unroll 4
    for (int i = wp; i < parts; i += 16) s += __ldcg(p + (int64_t)i * 2 * d);
  }
  slice[wp][lane] = s;
  __syncthreads();
  if (wp == 0 && col < 2 * d) {
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) t += slice[i][lane];
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
  unsigned ctas;              // backward: CTAs per replica
  bool grad;
};

template <typename T, int VEC, int NT, int EPT>
cudaError_t launch_ln(const LnArgs& a, cudaStream_t st) {
  if (!a.grad) {
    const int64_t gx = NT == 32 ? (a.s.rows + 3) / 4 : a.s.rows;
    return launch_dep(layer_norm_kernel<T, VEC, NT, EPT>, dim3((unsigned)gx, (unsigned)a.m), dim3(NT == 32 ? 128 : NT), 0,
                      st, 1, static_cast<const T*>(a.x), a.w, a.b, static_cast<T*>(a.y), a.mean_out, a.rstd_out, a.s);
  }
  return launch_dep(layer_norm_grad_kernel<T, VEC, NT, EPT>, dim3(a.ctas, (unsigned)a.m), dim3(NT == 32 ? 128 : NT),
                    NT == 32 ? (size_t)6 * a.s.d * sizeof(float) : 0, st, 1, static_cast<const T*>(a.dy),
                    static_cast<const T*>(a.x), a.w, a.mean, a.rstd, static_cast<T*>(a.y), a.part, a.s);
}

// Threads per row: a warp while its lanes hold the row in 16 (32) elements each, else a CTA of 16 per thread.
template <typename T, int VEC>
cudaError_t pick_ln(const LnArgs& a, cudaStream_t st) {
  const int d = a.s.d;
  if (d <= 512) return launch_ln<T, VEC, 32, 16>(a, st);
  if (d <= 1024) return launch_ln<T, VEC, 32, 32>(a, st);
  if (d <= 2048) return launch_ln<T, VEC, 128, 16>(a, st);
  if (d <= 4096) return launch_ln<T, VEC, 256, 16>(a, st);
  if (d <= 8192) return launch_ln<T, VEC, 512, 16>(a, st);
  return launch_ln<T, VEC, 1024, 16>(a, st);
}

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// 16-byte accesses need every row and every replica of every tensor to start on a 16-byte boundary.
cudaError_t run_ln(const LnArgs& a, int dtype, cudaStream_t st) {
  const int per = dtype == LS_DTYPE_BF16 ? 8 : 4;
  const bool one = a.m == 1;
  const bool vec = a.s.d % per == 0 && (one || (a.s.x_stride % per == 0 && a.s.y_stride % per == 0 && a.s.dy_stride % per == 0 &&
                                                   a.s.param_stride % 4 == 0)) && aligned16(a.x) &&
                   aligned16(a.y) && aligned16(a.w) && aligned16(a.b) && aligned16(a.dy);
  if (dtype == LS_DTYPE_BF16)
    return vec ? pick_ln<__nv_bfloat16, 8>(a, st) : pick_ln<__nv_bfloat16, 1>(a, st);
  return vec ? pick_ln<float, 4>(a, st) : pick_ln<float, 1>(a, st);
}

// CTAs of a replica in the backward kernel: two resident CTAs' worth of rows on every SM over all replicas, never more
// than there are rows (or groups of four rows).
unsigned grad_ctas(int m, int64_t rows, int d) {
  const int64_t units = d <= 1024 ? (rows + 3) / 4 : rows;
  const int64_t per_sm = d <= 2048 ? 4 : d <= 4096 ? 2 : 1;
  int64_t want = (148 * per_sm + m - 1) / m;
  if (want > units) want = units;
  return (unsigned)(want < 1 ? 1 : want);
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
  a.s = LnShape{rows, d, x_stride, y_stride, y_stride, param_stride, eps};
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
  int rc = check_ln(m, rows, d, LnShape{rows, d, n, n, n, d, 0.f}, LS_DTYPE_FP32);
  if (rc != LS_OK) return rc;
  if (bytes == nullptr) return LS_ERR_INVALID_ARG;
  *bytes = (size_t)m * grad_ctas(m, rows, d) * 2 * (size_t)d * sizeof(float);
  return LS_OK;
}

extern "C" int ls_layer_norm_grad(const void* dy_dev, const void* x_dev, const float* weight_dev, const float* mean_dev,
                                  const float* rstd_dev, int m, int64_t rows, int d, int64_t dy_stride, int64_t x_stride,
                                  int64_t param_stride, int dtype, void* dx_dev, int64_t dx_stride, float* dweight_dev,
                                  float* dbias_dev, int64_t dparam_stride, void* ws_dev, size_t ws_bytes,
                                  void* cuda_stream) {
  using namespace ls;
  LnArgs a{};
  a.s = LnShape{rows, d, x_stride, dy_stride, dx_stride, param_stride, 0.f};
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
  a.m = m; a.grad = true; a.ctas = grad_ctas(m, rows, d);
  // (no rows: the sums are those of no parts)
  if (rows > 0 && run_ln(a, dtype, st) != cudaSuccess) return LS_ERR_CUDA;
  const cudaError_t e = launch_dep(layer_norm_fold_kernel, dim3((unsigned)((2 * (int64_t)d + 31) / 32), (unsigned)m), dim3(512),
                                   0, st, 1, static_cast<const float*>(a.part), rows > 0 ? (int)a.ctas : 0, d, dweight_dev,
                                   dbias_dev, dparam_stride);
  return e == cudaSuccess ? LS_OK : LS_ERR_CUDA;
}
