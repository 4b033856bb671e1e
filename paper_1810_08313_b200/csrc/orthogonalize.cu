// Orthogonalisation of matrices by Newton-Schulz products and the momentum step that uses it (ls_orthogonalize,
// ls_muon_step; the update of the Muon optimiser).
//
//   X_0 = U / (|U|_F + 1e-7)
//   X_{k+1} = a X_k + (b A + c A^2) X_k,   A = X_k X_k^T,   (a, b, c) = (3.4445, -4.7750, 2.0315)
//
//             = P_k X_k,  P = a I + A (b I + c A)
// which drives every singular value of U towards 1 (into about [0.7, 1.2]) and leaves the singular vectors alone.  With
// n the shorter and k the longer side the step is two symmetric products of n x n results and one full one.  The side of
// the Gram matrix is the shorter one: A = X X^T and P X for a wide matrix, A = X^T X and X P for a tall one; both
// read X as it lies (K- or MN-major operands), nothing is transposed.
//
// Arithmetic: X, A, C = b I + c A and P are kept as two fp16 pieces (22 bits) scaled by powers of two into fp16's range,
// and every product is three fp16 MMAs (gemm_op.cuh).  bf16 alone would put an error of 2^-9 into each of the fifteen
// products, several times the rounding of a bf16 result; three MMAs of fp16 pieces cost half of three tf32 ones.  Of the
// symmetric products only the tiles on and above the diagonal are computed; the epilogue writes them to both places.
// The multiples of I are added in the epilogues (one launch writes A and C from the same accumulator), so that no
// epilogue reads a matrix.  Bound by the tensor cores: 3 (n^2 k + n^3 + 2 n^2 k) / 2 MMA multiply-adds a step.
#include "gemm_op.cuh"

#include <math.h>

namespace ls {
namespace {

using gop::Params;

constexpr float kNsA = 3.4445f, kNsB = -4.7750f, kNsC = 2.0315f;
constexpr float kNsEps = 1e-7f;
constexpr int kMaxSide = 1 << 15;
constexpr int kMaxSteps = 64;
constexpr int kSumBlocks = 296;        // at most: partial sums of squares of a matrix
// Scales of A, C and P in fp16.  Singular values stay below 1.25, so no entry of A exceeds 1.6, none of C |b| + 1.6 |c| < 8.1,
// and P, whose eigenvalues lie between 0 and a, has none above 3.5.
constexpr float kScaleA = 8192.f, kScaleC = 4096.f, kScaleP = 8192.f;

struct MatArgs {
  const void* g;                       // gradients (or the matrices to orthogonalise)
  float *w, *v;                        // null: ls_orthogonalize
  void* out;
  int m, rows, cols;
  int64_t w_stride, v_stride, g_stride, out_stride;
  float lr, mu;
  int nesterov;
  int64_t ld, plane;                   // pieces of X: row pitch, elements of one piece
  double* partial;                     // [m][kSumBlocks]
  int blocks;                          // partial sums per matrix
  float scale_x;
};

template <typename G>
__device__ __forceinline__ float load_g(const void* g, int64_t i) { return (float)static_cast<const G*>(g)[i]; }

// v <- mu v + g, and the partial sums of squares of U in double
template <typename G, bool MUON>
__global__ void __launch_bounds__(512) ns_momentum_kernel(const MatArgs a) {
  __shared__ double red[16];
  grid_dep_wait();
  grid_dep_launch();
  const int64_t n = (int64_t)a.rows * a.cols;
  const int64_t z = blockIdx.y;
  double s = 0.0;
  for (int64_t i = (int64_t)blockIdx.x * 512 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 512) {
    const float g = load_g<G>(a.g, z * a.g_stride + i);
    float u = g;
    if constexpr (MUON) {
      float* v = a.v + z * a.v_stride + i;
      const float nv = fmaf(a.mu, *v, g);
      *v = nv;
      u = a.nesterov ? fmaf(a.mu, nv, g) : nv;
    }
    s += (double)u * (double)u;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    double t = 0.0;
    for (int i = 0; i < 16; ++i) t += red[i];
    a.partial[z * kSumBlocks + blockIdx.x] = t;
  }
}

// X_0 = U / (|U| + eps) as two scaled pieces
template <typename G, bool MUON>
__global__ void __launch_bounds__(512) ns_start_kernel(const MatArgs a, __half* x) {
  __shared__ float inv_s;
  grid_dep_wait();
  grid_dep_launch();
  const int64_t z = blockIdx.y;
  if (threadIdx.x < 32) {
    double t = 0.0;
    for (int i = threadIdx.x; i < a.blocks; i += 32) t += a.partial[z * kSumBlocks + i];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
    if (threadIdx.x == 0) inv_s = (float)sqrt(t) + kNsEps;
  }
  __syncthreads();
  const float norm = inv_s;
  __half* hi = x + z * 2 * a.plane;
  __half* lo = hi + a.plane;
  const int64_t n = (int64_t)a.rows * a.cols;
  for (int64_t i = (int64_t)blockIdx.x * 512 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 512) {
    const float g = load_g<G>(a.g, z * a.g_stride + i);
    float u = g;
    if constexpr (MUON) {
      const float nv = a.v[z * a.v_stride + i];
      u = a.nesterov ? fmaf(a.mu, nv, g) : nv;
    }
    const float v = u / norm * a.scale_x;
    const __half h = __float2half_rn(v);
    const int64_t r = i / a.cols, at = r * a.ld + (i - r * a.cols);
    hi[at] = h;
    lo[at] = __float2half_rn(v - __half2float(h));
  }
}

// W <- W - step O, or out <- O, from the pieces of the last X
template <typename G, bool MUON>
__global__ void __launch_bounds__(512) ns_finish_kernel(const MatArgs a, const __half* x, float step) {
  grid_dep_wait();
  grid_dep_launch();
  const int64_t z = blockIdx.y;
  const __half* hi = x + z * 2 * a.plane;
  const __half* lo = hi + a.plane;
  const float inv = 1.f / a.scale_x;
  const int64_t n = (int64_t)a.rows * a.cols;
  for (int64_t i = (int64_t)blockIdx.x * 512 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 512) {
    const int64_t r = i / a.cols, at = r * a.ld + (i - r * a.cols);
    const float o = (__half2float(hi[at]) + __half2float(lo[at])) * inv;
    if constexpr (MUON) {
      float* w = a.w + z * a.w_stride + i;
      *w = fmaf(-step, o, *w);
    } else {
      static_cast<G*>(a.out)[z * a.out_stride + i] = (G)o;
    }
  }
}

int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

struct Plan {
  int n, k;                    // shorter and longer side
  bool tall;
  int64_t ld, plane;           // X
  int64_t ldn, plane_n;        // A, C, P
  size_t o_partial, o_x[2], o_ac, o_p, total;
};

Plan make_plan(int m, int rows, int cols) {
  Plan p{};
  p.tall = rows > cols;
  p.n = p.tall ? cols : rows;
  p.k = p.tall ? rows : cols;
  p.ld = round_up(cols, 64);
  p.plane = p.ld * rows;
  p.ldn = round_up(p.n, 64);
  p.plane_n = p.ldn * p.n;
  size_t at = 0;
  auto take = [&at](int64_t bytes) { size_t o = at; at += (size_t)round_up(bytes, 256); return o; };
  p.o_partial = take((int64_t)m * kSumBlocks * 8);
  for (int i = 0; i < 2; ++i) p.o_x[i] = take((int64_t)m * 2 * p.plane * 2);
  p.o_ac = take((int64_t)m * 4 * p.plane_n * 2);
  p.o_p = take((int64_t)m * 2 * p.plane_n * 2);
  p.total = at;
  return p;
}

#define LS_TRY(x)                                   \
  do {                                              \
    if ((x) != cudaSuccess) return LS_ERR_CUDA;     \
  } while (0)

template <typename G, bool MUON>
int run_ns(MatArgs a, int steps, char* ws, cudaStream_t st) {
  const Plan p = make_plan(a.m, a.rows, a.cols);
  a.ld = p.ld; a.plane = p.plane;
  a.partial = reinterpret_cast<double*>(ws + p.o_partial);
  const int64_t n = (int64_t)a.rows * a.cols;
  // entries of X_0 of about 1: the root mean square of a matrix of Frobenius norm 1, inverted; none exceeds 2^14
  a.scale_x = exp2f(floorf(0.5f * log2f((float)n)));
  if (a.scale_x > 16384.f) a.scale_x = 16384.f;
  int64_t blocks = (n + 2047) / 2048, share = 148 * 4 / a.m;
  if (share < 1) share = 1;
  if (blocks > share) blocks = share;
  if (blocks > kSumBlocks) blocks = kSumBlocks;
  a.blocks = (int)blocks;
  __half* x[2] = {reinterpret_cast<__half*>(ws + p.o_x[0]), reinterpret_cast<__half*>(ws + p.o_x[1])};
  const void* ac = ws + p.o_ac;      // [m][A first, second piece, C first, second piece]
  const void* pp = ws + p.o_p;
  const dim3 grid((unsigned)blocks, (unsigned)a.m);
  LS_TRY(launch_dep(ns_momentum_kernel<G, MUON>, grid, dim3(512), 0, st, 1, a));
  LS_TRY(launch_dep(ns_start_kernel<G, MUON>, grid, dim3(512), 0, st, 1, a, x[0]));
  // maps: X as K-major and MN-major operand and as output; A, C and P as K-major operands (they are symmetric) and as
  // outputs, straight and transposed
  CUtensorMap xk[2], xm[2], xo[2], ack, aco, act, pk, po, pt;
  const int64_t m = a.m;
  for (int i = 0; i < 2; ++i) {
    LS_TRY(gop::make_stack_map(&xk[i], x[i], gop::MAP_F16, a.rows, a.cols, 2 * m, p.ld, p.plane, 128));
    LS_TRY(gop::make_stack_map(&xm[i], x[i], gop::MAP_F16, a.rows, a.cols, 2 * m, p.ld, p.plane, 64));
    LS_TRY(gop::make_stack_map(&xo[i], x[i], gop::MAP_F16_S, a.rows, a.cols, 2 * m, p.ld, p.plane, 32));
  }
  LS_TRY(gop::make_stack_map(&ack, ac, gop::MAP_F16, p.n, p.n, 4 * m, p.ldn, p.plane_n, 128));
  LS_TRY(gop::make_stack_map(&aco, ac, gop::MAP_F16_S, p.n, p.n, 4 * m, p.ldn, p.plane_n, 32));
  LS_TRY(gop::make_stack_map(&act, ac, gop::MAP_F16_T, p.n, p.n, 4 * m, p.ldn, p.plane_n, 32));
  LS_TRY(gop::make_stack_map(&pk, pp, gop::MAP_F16, p.n, p.n, 2 * m, p.ldn, p.plane_n, 128));
  LS_TRY(gop::make_stack_map(&po, pp, gop::MAP_F16_S, p.n, p.n, 2 * m, p.ldn, p.plane_n, 32));
  LS_TRY(gop::make_stack_map(&pt, pp, gop::MAP_F16_T, p.n, p.n, 2 * m, p.ldn, p.plane_n, 32));
  int cur = 0;
  for (int s = 0; s < steps; ++s, cur ^= 1) {
    Params g{};
    g.batch = a.m;
    // A = X X^T (wide) or X^T X (tall), and C = b I + c A
    g.M = g.N = p.n; g.tri = g.mirror = 1;
    g.a_zstep = g.b_zstep = 2; g.c_zstep = 4;
    g.n_out = 2;
    const float unit = 1.f / (a.scale_x * a.scale_x);
    g.out_alpha[0] = kScaleA * unit;
    g.out_alpha[1] = kNsC * kScaleC * unit;
    g.out_diag[1] = kNsB * kScaleC;
    if (p.tall) LS_TRY((gop::launch<2, true, true, true, gop::EPI_PIECES>(xm[cur], xm[cur], aco, act, g, p.k, st)));
    else LS_TRY((gop::launch<2, true, false, false, gop::EPI_PIECES>(xk[cur], xk[cur], aco, act, g, p.k, st)));
    // P = a I + A C
    g.a_zstep = g.b_zstep = 4; g.b_z0 = 2; g.c_zstep = 2;
    g.n_out = 1;
    g.out_alpha[0] = kScaleP / (kScaleA * kScaleC);
    g.out_diag[0] = kNsA * kScaleP;
    LS_TRY((gop::launch<2, true, false, false, gop::EPI_PIECES>(ack, ack, po, pt, g, p.n, st)));
    // X <- P X (wide) or X P (tall)
    g.a_zstep = g.b_zstep = g.c_zstep = 2; g.b_z0 = 0;
    g.tri = g.mirror = 0;
    g.M = a.rows; g.N = a.cols;
    g.out_alpha[0] = 1.f / kScaleP;
    g.out_diag[0] = 0.f;
    if (p.tall) LS_TRY((gop::launch<2, true, false, false, gop::EPI_PIECES>(xk[cur], pk, xo[cur ^ 1], xo[cur ^ 1], g, p.n, st)));
    else LS_TRY((gop::launch<2, true, false, true, gop::EPI_PIECES>(pk, xm[cur], xo[cur ^ 1], xo[cur ^ 1], g, p.n, st)));
  }
  const float step = a.lr * sqrtf(fmaxf(1.f, (float)a.rows / (float)a.cols));
  LS_TRY(launch_dep(ns_finish_kernel<G, MUON>, grid, dim3(512), 0, st, 1, a, static_cast<const __half*>(x[cur]), step));
  return LS_OK;
}

int check_sizes(int m, int rows, int cols) {
  if (m < 1 || rows < 1 || cols < 1) return LS_ERR_INVALID_ARG;
  if (m > 65535 || rows > kMaxSide || cols > kMaxSide) return LS_ERR_TOO_LARGE;
  return LS_OK;
}
bool off(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }

int check_ws(int m, int rows, int cols, const void* ws, size_t ws_bytes) {
  if (ws == nullptr) return LS_ERR_INVALID_ARG;
  if (ws_bytes < make_plan(m, rows, cols).total || off(ws, 256)) return LS_ERR_STATE_SIZE;
  return LS_OK;
}

}  // namespace
}  // namespace ls

extern "C" int ls_orthogonalize_ws_bytes(int m, int rows, int cols, size_t* bytes) {
  using namespace ls;
  int rc = check_sizes(m, rows, cols);
  if (rc != LS_OK) return rc;
  if (bytes == nullptr) return LS_ERR_INVALID_ARG;
  *bytes = make_plan(m, rows, cols).total;
  return LS_OK;
}

extern "C" int ls_orthogonalize(const void* u_dev, int m, int rows, int cols, int64_t u_stride, int dtype, int steps,
                                void* out_dev, int64_t out_stride, void* ws_dev, size_t ws_bytes, void* cuda_stream) {
  using namespace ls;
  int rc = check_sizes(m, rows, cols);
  if (rc != LS_OK) return rc;
  if (u_dev == nullptr || out_dev == nullptr || steps < 1 || steps > kMaxSteps) return LS_ERR_INVALID_ARG;
  if (dtype != LS_DTYPE_FP32 && dtype != LS_DTYPE_BF16) return LS_ERR_INVALID_ARG;
  const size_t eb = dtype == LS_DTYPE_BF16 ? 2 : 4;
  if (off(u_dev, eb) || off(out_dev, eb)) return LS_ERR_INVALID_ARG;
  if (m > 1 && (u_stride < (int64_t)rows * cols || out_stride < (int64_t)rows * cols)) return LS_ERR_INVALID_ARG;
  rc = check_ws(m, rows, cols, ws_dev, ws_bytes);
  if (rc != LS_OK) return rc;
  MatArgs a{};
  a.g = u_dev; a.g_stride = u_stride; a.out = out_dev; a.out_stride = out_stride;
  a.m = m; a.rows = rows; a.cols = cols;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  return dtype == LS_DTYPE_BF16 ? run_ns<__nv_bfloat16, false>(a, steps, static_cast<char*>(ws_dev), st)
                                : run_ns<float, false>(a, steps, static_cast<char*>(ws_dev), st);
}

extern "C" int ls_muon_step(float* w_dev, float* v_dev, const void* g_dev, int m, int rows, int cols, int64_t w_stride,
                            int64_t v_stride, int64_t g_stride, int g_dtype, float lr, float momentum, int nesterov, int steps, void* ws_dev,
                            size_t ws_bytes, void* cuda_stream) {
  using namespace ls;
  int rc = check_sizes(m, rows, cols);
  if (rc != LS_OK) return rc;
  if (w_dev == nullptr || v_dev == nullptr || g_dev == nullptr || steps < 1 || steps > kMaxSteps) return LS_ERR_INVALID_ARG;
  if (g_dtype != LS_DTYPE_FP32 && g_dtype != LS_DTYPE_BF16) return LS_ERR_INVALID_ARG;
  if (!isfinite(lr) || !(momentum >= 0.f) || !(momentum < 1.f) || (nesterov != 0 && nesterov != 1)) return LS_ERR_INVALID_ARG;
  if (off(w_dev, 4) || off(v_dev, 4) || off(g_dev, g_dtype == LS_DTYPE_BF16 ? 2 : 4)) return LS_ERR_INVALID_ARG;
  const int64_t n = (int64_t)rows * cols;
  if (m > 1 && (w_stride < n || v_stride < n || g_stride < n)) return LS_ERR_INVALID_ARG;
  rc = check_ws(m, rows, cols, ws_dev, ws_bytes);
  if (rc != LS_OK) return rc;
  MatArgs a{};
  a.g = g_dev; a.g_stride = g_stride; a.w = w_dev; a.v = v_dev; a.w_stride = w_stride; a.v_stride = v_stride;
  a.m = m; a.rows = rows; a.cols = cols; a.lr = lr; a.mu = momentum; a.nesterov = nesterov;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  return g_dtype == LS_DTYPE_BF16 ? run_ns<__nv_bfloat16, true>(a, steps, static_cast<char*>(ws_dev), st)
                                  : run_ns<float, true>(a, steps, static_cast<char*>(ws_dev), st);
}
