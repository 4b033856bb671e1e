// Orthogonalisation of matrices by Newton-Schulz products and the momentum step that uses it (ls_orthogonalize,
// ls_muon_step; the update of the Muon optimiser).
//
//   X_0 = U / (|U|_F + 1e-7)
//   X_{k+1} = a X_k + (b A + c A^2) X_k = P_k X_k,   A = X_k X_k^T,   P = a I + A (b I + c A)
//
// with (a, b, c) = (3.4445, -4.7750, 2.0315), which drives every singular value of U towards 1 (into about [0.7, 1.2]) and
// leaves the singular vectors alone.  With n the shorter and k the longer side the step is two symmetric products of n x n results and one full one.  The side of
// the Gram matrix is the shorter one: A = X X^T and P X for a wide matrix, A = X^T X and X P for a tall one; both
// read X as it lies (K- or MN-major operands), nothing is transposed.
//
// Arithmetic: X, A, C = b I + c A and P are kept as two fp16 pieces (22 bits) scaled by powers of two into fp16's range,
// and every product is three fp16 MMAs (gemm_op.cuh).  bf16 alone would put an error of 2^-9 into each of the fifteen
// products, several times the rounding of a bf16 result; three MMAs of fp16 pieces cost half of three tf32 ones.  Of the
// symmetric products only the tiles on and above the diagonal are computed; the epilogue writes them to both places.
// The multiples of I are added in the epilogues (one launch writes A and C from the same accumulator), so that no
// epilogue reads a matrix.  Bound by the tensor cores: 3 (n^2 k + n^3 + 2 n^2 k) / 2 MMA multiply-adds a step.
//
// Steps taken together: A and P are polynomials of the first A, so they commute and A_{k+1} = A_k P_k P_k.  Two or three steps
// need one A = X X^T and one X <- Q X with Q = P_2 P_1 P_0; each step after the first replaces that pair of products,
// 3 n^2 k multiply-adds, by three symmetric ones more (B = A P, B P, P Q), 3 n^3 / 2.  That pays for matrices longer than wide whose
// products fill the GPU (Plan::group compares both by pick_cut()'s estimates): 2 x 1024 x 4096 513 -> 436 us.  It costs
// accuracy: what the tensor core truncates in A is multiplied by a^2 a step (11.9) before it acts, and every P and Q has
// one large product a row.  Five steps of normal matrices are off by 4e-6 to 8e-6 of their norm, 1e-6 to 3e-6 one at a time, as in
// fp32 arithmetic, so only steps from bf16 numbers, which carry 2e-3, are taken together.
#include "gemm_op.cuh"

#include <math.h>

namespace ls {
namespace {

using gop::Params;

constexpr float kNsA = 3.4445f, kNsB = -4.7750f, kNsC = 2.0315f;
constexpr float kNsEps = 1e-7f;
constexpr int kMaxSide = 1 << 15;
constexpr int kMaxSteps = 64;
constexpr int kSumBlocks = 592;        // at most: partial sums of squares of a matrix
// Scales of A, C and P in fp16.  Singular values stay below 1.25, so no entry of A exceeds 1.6, none of C |b| + 1.6 |c| < 8.1,
// and P, whose eigenvalues lie between 0 and a, has none above 3.5.
constexpr float kScaleA = 8192.f, kScaleC = 4096.f, kScaleP = 8192.f;
// B = A P has no eigenvalue above 1.45; Q, a product of two or three P, none above a^2 = 11.9 or a^3 = 40.9.
constexpr float kScaleB = 8192.f, kScaleQ[2] = {4096.f, 1024.f};
constexpr double kLaunchUs = 6.0;      // what a product costs beside its tiles: first operands, last epilogue

struct MatArgs {
  const void* g;                       // gradients (or the matrices to orthogonalise)
  float *w, *v;                        // null: ls_orthogonalize
  void* out;
  int m, rows, cols;
  int64_t w_stride, v_stride, g_stride, out_stride;
  float lr, mu;
  int nesterov;
  int blocked;                         // w and v lie in 32 x 32 blocks (TileMap), rows and cols multiples of 32
  int64_t ld, plane;                   // pieces of X: row pitch, elements of one piece
  double* partial;                     // [m][kSumBlocks]
  int blocks;                          // partial sums per matrix
  float scale_x;
};

// The element-wise passes take a matrix in units of 512 columns of a row, one warp each; a lane has four groups of four
// consecutive elements, read as 16 (bf16: 8) bytes where rows start on such boundaries (VEC), else one by one.
constexpr int kUnit = 512;
constexpr int kWarps = 8;                // per CTA

template <typename T, bool VEC>
__device__ __forceinline__ void load4(const T* p, int left, float (&f)[4]) {
  if constexpr (VEC && sizeof(T) == 4) {
    const float4 v = *reinterpret_cast<const float4*>(p);
    f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
  } else if constexpr (VEC) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    f[0] = __uint_as_float(v.x << 16); f[1] = __uint_as_float(v.x & 0xFFFF0000u);
    f[2] = __uint_as_float(v.y << 16); f[3] = __uint_as_float(v.y & 0xFFFF0000u);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = i < left ? (float)p[i] : 0.f;
  }
}
template <typename T, bool VEC>
__device__ __forceinline__ void store4(T* p, int left, const float (&f)[4]) {
  if constexpr (VEC && sizeof(T) == 4) {
    *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
  } else if constexpr (VEC) {
    *reinterpret_cast<uint2*>(p) = make_uint2(gop::pack_bf16(f[0], f[1]), gop::pack_bf16(f[2], f[3]));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) if (i < left) p[i] = (T)f[i];
  }
}
// Where four consecutive elements of w and v from (r, c) on start, `at` their place in row-major order.
__device__ __forceinline__ int64_t state_at(const MatArgs& a, int64_t at, int r, int c) {
  return a.blocked ? ((int64_t)(r >> 5) * (a.cols >> 5) + (c >> 5)) * 1024 + (r & 31) * 32 + (c & 31) : at;
}
// For each of this warp's units: load(k, offset, row, column, elements left in the row) for its four groups, then
// use(k, ...) for them, so that the loads of a unit are in flight together.
template <typename L, typename F>
__device__ __forceinline__ void for_units(const MatArgs& a, L load, F use) {
  const int segs = (a.cols + kUnit - 1) / kUnit;
  const int64_t units = (int64_t)a.rows * segs;
  const int lane = threadIdx.x & 31;
  for (int64_t u = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5); u < units; u += (int64_t)gridDim.x * kWarps) {
    const int r = (int)(u / segs), c0 = (int)(u - (int64_t)r * segs) * kUnit + lane * 4;
    const int64_t at = (int64_t)r * a.cols + c0;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (c0 + k * 128 < a.cols) load(k, at + k * 128, r, c0 + k * 128, a.cols - c0 - k * 128);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (c0 + k * 128 < a.cols) use(k, at + k * 128, r, c0 + k * 128, a.cols - c0 - k * 128);
  }
}

// v <- mu v + g, and the partial sums of squares of U in double
template <typename G, bool MUON, bool VEC>
__global__ void __launch_bounds__(32 * kWarps) ns_momentum_kernel(const MatArgs a) {
  __shared__ double red[kWarps];
  grid_dep_wait();
  grid_dep_launch();
  const int64_t z = blockIdx.y;
  const G* gz = static_cast<const G*>(a.g) + z * a.g_stride;
  float* vz = MUON ? a.v + z * a.v_stride : nullptr;
  double s = 0.0;
  float g[4][4], v[4][4];
  for_units(
      a,
      [&](int k, int64_t at, int r, int c, int left) {
        load4<G, VEC>(gz + at, left, g[k]);
        if constexpr (MUON) load4<float, VEC>(vz + state_at(a, at, r, c), left, v[k]);
      },
      [&](int k, int64_t at, int r, int c, int left) {
        if constexpr (MUON) {
#pragma unroll
          for (int i = 0; i < 4; ++i) v[k][i] = fmaf(a.mu, v[k][i], g[k][i]);
          store4<float, VEC>(vz + state_at(a, at, r, c), left, v[k]);
#pragma unroll
          for (int i = 0; i < 4; ++i) g[k][i] = a.nesterov ? fmaf(a.mu, v[k][i], g[k][i]) : v[k][i];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) s += (double)g[k][i] * (double)g[k][i];
      });
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    double t = 0.0;
    for (int i = 0; i < kWarps; ++i) t += red[i];
    a.partial[z * kSumBlocks + blockIdx.x] = t;
  }
}

// X_0 = U / (|U| + eps) as two scaled pieces
template <typename G, bool MUON, bool VEC>
__global__ void __launch_bounds__(32 * kWarps) ns_start_kernel(const MatArgs a, __half* x) {
  __shared__ float norm_s;
  grid_dep_wait();
  grid_dep_launch();
  const int64_t z = blockIdx.y;
  if (threadIdx.x < 32) {
    double t = 0.0;
    for (int i = threadIdx.x; i < a.blocks; i += 32) t += a.partial[z * kSumBlocks + i];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
    if (threadIdx.x == 0) norm_s = (float)sqrt(t) + kNsEps;
  }
  __syncthreads();
  const float norm = norm_s;
  __half* hi = x + z * 2 * a.plane;
  const G* gz = static_cast<const G*>(a.g) + z * a.g_stride;
  const float* vz = MUON ? a.v + z * a.v_stride : nullptr;
  float g[4][4], v[4][4];
  for_units(
      a,
      [&](int k, int64_t at, int r, int c, int left) {
        load4<G, VEC>(gz + at, left, g[k]);
        if constexpr (MUON) load4<float, VEC>(vz + state_at(a, at, r, c), left, v[k]);
      },
      [&](int k, int64_t, int r, int c, int) {
        if constexpr (MUON) {
#pragma unroll
          for (int i = 0; i < 4; ++i) g[k][i] = a.nesterov ? fmaf(a.mu, v[k][i], g[k][i]) : v[k][i];
        }
        float l[4];
        uint32_t hw[2];
#pragma unroll
        for (int i = 0; i < 4; ++i) g[k][i] = g[k][i] / norm * a.scale_x;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const __half2 h = __floats2half2_rn(g[k][2 * i], g[k][2 * i + 1]);
          const float2 f = __half22float2(h);
          l[2 * i] = g[k][2 * i] - f.x; l[2 * i + 1] = g[k][2 * i + 1] - f.y;
          hw[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
        // (rows of X are padded to whole 64 elements: the group past the last column is written as it is)
        __half* o = hi + (int64_t)r * a.ld + c;
        *reinterpret_cast<uint2*>(o) = make_uint2(hw[0], hw[1]);
        *reinterpret_cast<uint2*>(o + a.plane) = make_uint2(gop::pack_f16(l[0], l[1]), gop::pack_f16(l[2], l[3]));
      });
}

// W <- W - step O, or out <- O, from the pieces of the last X
template <typename G, bool MUON, bool VEC>
__global__ void __launch_bounds__(32 * kWarps) ns_finish_kernel(const MatArgs a, const __half* x, float step) {
  grid_dep_wait();
  grid_dep_launch();
  const int64_t z = blockIdx.y;
  const __half* hi = x + z * 2 * a.plane;
  const float inv = 1.f / a.scale_x;
  float* wz = MUON ? a.w + z * a.w_stride : nullptr;
  G* oz = MUON ? nullptr : static_cast<G*>(a.out) + z * a.out_stride;
  uint2 h[4], l[4];
  float w[4][4];
  for_units(
      a,
      [&](int k, int64_t at, int r, int c, int left) {
        const __half* p = hi + (int64_t)r * a.ld + c;
        h[k] = *reinterpret_cast<const uint2*>(p);
        l[k] = *reinterpret_cast<const uint2*>(p + a.plane);
        if constexpr (MUON) load4<float, VEC>(wz + state_at(a, at, r, c), left, w[k]);
      },
      [&](int k, int64_t at, int r, int c, int left) {
        const uint32_t hw[2] = {h[k].x, h[k].y}, lw[2] = {l[k].x, l[k].y};
        float o[4];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&hw[i]));
          const float2 e = __half22float2(*reinterpret_cast<const __half2*>(&lw[i]));
          o[2 * i] = (f.x + e.x) * inv; o[2 * i + 1] = (f.y + e.y) * inv;
        }
        if constexpr (MUON) {
#pragma unroll
          for (int i = 0; i < 4; ++i) w[k][i] = fmaf(-step, o[i], w[k][i]);
          store4<float, VEC>(wz + state_at(a, at, r, c), left, w[k]);
        } else {
          store4<G, VEC>(oz + at, left, o);
        }
      });
}

// The Gram matrix from the parts of a cut contraction: A and C = b I + c A as pieces, on both sides of the diagonal.  A CTA takes a
// block of 64 x 64 on or above it and adds the parts in index order, two columns a thread; the transposed block goes through
// shared memory.
struct FoldArgs {
  const float* part;          // [m][splits] planes of n rows of ldf
  __half* ac;                 // [m] of four planes
  int n, splits;
  int64_t ldf, planef, ldn, plane_n;
  float alpha_a, alpha_c, diag_c;
};
__global__ void __launch_bounds__(256) ns_gram_fold_kernel(const FoldArgs a) {
  __shared__ float tile[64][65];
  grid_dep_wait();
  grid_dep_launch();
  // block of the upper triangle: column block bc, row block br <= bc
  int bc = (int)((sqrtf(8.f * (float)blockIdx.x + 1.f) - 1.f) * 0.5f);
  while ((bc + 1) * (bc + 2) / 2 <= (int)blockIdx.x) ++bc;
  while (bc * (bc + 1) / 2 > (int)blockIdx.x) --bc;
  const int br = (int)blockIdx.x - bc * (bc + 1) / 2;
  const int64_t z = blockIdx.y;
  const int x = (threadIdx.x & 31) * 2, y0 = threadIdx.x >> 5;
  const float* src = a.part + z * a.splits * a.planef;
  __half* out = a.ac + z * 4 * a.plane_n;
  // columns col, col + 1 of row r (rows are padded to whole 64 columns)
  auto put = [&](int r, int col, float v0, float v1) {
    uint32_t* o = reinterpret_cast<uint32_t*>(out + (int64_t)r * a.ldn + col);
    const int64_t plane = a.plane_n / 2;
    auto pieces = [&](uint32_t* at, float u0, float u1) {
      const __half2 h = __floats2half2_rn(u0, u1);
      const float2 f = __half22float2(h);
      at[0] = *reinterpret_cast<const uint32_t*>(&h);
      at[plane] = gop::pack_f16(u0 - f.x, u1 - f.y);
    };
    pieces(o, a.alpha_a * v0, a.alpha_a * v1);
    pieces(o + 2 * plane, fmaf(a.alpha_c, v0, r == col ? a.diag_c : 0.f), fmaf(a.alpha_c, v1, r == col + 1 ? a.diag_c : 0.f));
  };
  const int c = bc * 64 + x;
  float2 v[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) v[k] = make_float2(0.f, 0.f);
  for (int s = 0; s < a.splits; ++s) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int r = br * 64 + y0 + k * 8;
      if (r < a.n && c < a.n) {
        const float2 u = __ldcg(reinterpret_cast<const float2*>(src + s * a.planef + (int64_t)r * a.ldf + c));
        v[k].x += u.x; v[k].y += u.y;
      }
    }
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int r = br * 64 + y0 + k * 8;
    if (r < a.n && c < a.n) put(r, c, v[k].x, v[k].y);
    tile[y0 + k * 8][x] = v[k].x;
    tile[y0 + k * 8][x + 1] = v[k].y;
  }
  if (br == bc) return;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int r = bc * 64 + y0 + k * 8, col = br * 64 + x;        // the transposed place
    if (r < a.n && col < a.n) put(r, col, tile[x][y0 + k * 8], tile[x + 1][y0 + k * 8]);
  }
}

int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

struct Plan {
  int n, k;                    // shorter and longer side
  bool tall;
  int64_t ld, plane;           // X
  int64_t ldn, plane_n;        // A, C, P
  int64_t ldf, planef;         // parts of the Gram matrix
  gop::Cut gram, full, square;   // X X^T, P X and a symmetric product of n x n matrices
  bool group;                    // steps may be taken together
  size_t o_partial, o_x[2], o_ac, o_s, o_gram, total;
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
  p.gram = gop::pick_cut(p.n, p.n, m, true, p.k, 2, 32);
  p.full = gop::pick_cut(rows, cols, m, false, p.n, 2, 1);
  p.square = gop::pick_cut(p.n, p.n, m, true, p.n, 2, 1);
  // (by a tenth: the estimates are no better)
  p.group = p.gram.us + p.full.us + 2 * kLaunchUs > 1.1 * 3 * (p.square.us + kLaunchUs);
  p.o_s = take((int64_t)m * 2 * p.plane_n * 2 * (p.group ? 3 : 1));
  p.ldf = round_up(p.n, 4);
  p.planef = p.ldf * p.n;
  p.o_gram = take(p.gram.splits > 1 ? (int64_t)m * p.gram.splits * p.planef * 4 : 0);
  p.total = at;
  return p;
}

#define LS_TRY(x)                                   \
  do {                                              \
    if ((x) != cudaSuccess) return LS_ERR_CUDA;     \
  } while (0)

bool off(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }

template <typename G, bool MUON, bool VEC>
int run_ns(MatArgs a, int steps, char* ws, cudaStream_t st) {
  const Plan p = make_plan(a.m, a.rows, a.cols);
  a.ld = p.ld; a.plane = p.plane;
  a.partial = reinterpret_cast<double*>(ws + p.o_partial);
  const int64_t n = (int64_t)a.rows * a.cols;
  // entries of X_0 of about 1: the root mean square of a matrix of Frobenius norm 1, inverted; none exceeds 2^14
  a.scale_x = exp2f(floorf(0.5f * log2f((float)n)));
  if (a.scale_x > 16384.f) a.scale_x = 16384.f;
  // (four resident CTAs per SM over all replicas)
  int64_t blocks = ((int64_t)a.rows * ((a.cols + kUnit - 1) / kUnit) + kWarps - 1) / kWarps, share = 148 * 4 / a.m;
  if (share < 1) share = 1;
  if (blocks > share) blocks = share;
  if (blocks > kSumBlocks) blocks = kSumBlocks;
  a.blocks = (int)blocks;
  __half* x[2] = {reinterpret_cast<__half*>(ws + p.o_x[0]), reinterpret_cast<__half*>(ws + p.o_x[1])};
  const bool cut = p.gram.splits > 1, together = p.group && sizeof(G) == 2;
  void* ac = ws + p.o_ac;      // [m][A first, second piece, C first, second piece]
  const dim3 grid((unsigned)blocks, (unsigned)a.m);
  LS_TRY(launch_dep(ns_momentum_kernel<G, MUON, VEC>, grid, dim3(32 * kWarps), 0, st, 1, a));
  LS_TRY(launch_dep(ns_start_kernel<G, MUON, VEC>, grid, dim3(32 * kWarps), 0, st, 1, a, x[0]));
  // maps: X as operand and as output; A and C, and the matrices P, Q, B as operands and as outputs, straight and transposed
  constexpr int kRow = gop::box_row(2);
  CUtensorMap xk[2], xo[2], ack, aco, act, sk[3], so[3], sq[3], gf;
  const int64_t m = a.m;
  for (int i = 0; i < 2; ++i) {
    LS_TRY(gop::make_operand_map(&xk[i], x[i], gop::MAP_F16, a.rows, a.cols, 2 * m, p.ld, p.plane));
    LS_TRY(gop::make_output_map(&xo[i], x[i], gop::MAP_F16, a.rows, a.cols, 2 * m, p.ld, p.plane, kRow));
  }
  LS_TRY(gop::make_operand_map(&ack, ac, gop::MAP_F16, p.n, p.n, 4 * m, p.ldn, p.plane_n));
  LS_TRY(gop::make_output_map(&aco, ac, gop::MAP_F16, p.n, p.n, 4 * m, p.ldn, p.plane_n, kRow));
  LS_TRY(gop::make_output_map(&act, ac, gop::MAP_F16, p.n, p.n, 4 * m, p.ldn, p.plane_n, kRow, true));
  for (int i = 0; i < (together ? 3 : 1); ++i) {
    void* s = ws + p.o_s + (size_t)i * m * 2 * p.plane_n * 2;
    LS_TRY(gop::make_operand_map(&sk[i], s, gop::MAP_F16, p.n, p.n, 2 * m, p.ldn, p.plane_n));
    LS_TRY(gop::make_output_map(&so[i], s, gop::MAP_F16, p.n, p.n, 2 * m, p.ldn, p.plane_n, kRow));
    LS_TRY(gop::make_output_map(&sq[i], s, gop::MAP_F16, p.n, p.n, 2 * m, p.ldn, p.plane_n, kRow, true));
  }
  if (cut)
    LS_TRY(gop::make_output_map(&gf, ws + p.o_gram, gop::MAP_F32, p.n, p.n, m * p.gram.splits, p.ldf, p.planef, kRow));
  // symmetric products of commuting n x n matrices, all of which tend to multiples of I
  auto square = [&](const CUtensorMap& l, int lstep, const CUtensorMap& r, int rstep, int r0, const CUtensorMap& out,
                    const CUtensorMap& out_t, int ostep, Params g) {
    g.batch = a.m; g.M = g.N = p.n; g.tri = g.mirror = 1;
    g.a_zstep = lstep; g.b_zstep = rstep; g.b_z0 = r0; g.c_zstep = ostep;
    g.dominant = 1;
    g.chunk_kb = together ? 2 : 4;          // (together: 2e-5 at chunks of 8 for singular values over six decades, 9e-6 at 2)
    // P of a small matrix (up to three K blocks): few elements average what the MMAs after a row's dominant product truncate, and
    // near singular values of 1 P is what is left of a - 2.7.  1524 x 65 is off by 1.7e-6 without, 1.1e-6 with it, 763 x 189 by 1.5
    // and 0.7 times fp32 arithmetic's error; at 256 x 256 (129 and 142 us) the two errors are alike already.
    g.fine = !together && p.n <= 192;
    return gop::launch<2, true, false, false, gop::EPI_PIECES>(p.square.nt, l, r, out, out_t, g, p.n, st);
  };
  // A, and C = b I + c A, of a product whose operands were scaled
  auto a_and_c = [](float operands) {
    Params g{};
    g.n_out = 2;
    g.out_alpha[0] = kScaleA / operands;
    g.out_alpha[1] = kNsC * kScaleC / operands;
    g.out_diag[1] = kNsB * kScaleC;
    return g;
  };
  auto one = [](float alpha, float diag) {
    Params g{};
    g.n_out = 1;
    g.out_alpha[0] = alpha;
    g.out_diag[0] = diag;
    return g;
  };
  int cur = 0;
  for (int left = steps; left > 0; cur ^= 1) {
    const int group = !together || left == 1 ? 1 : left % 2 == 1 ? 3 : 2;
    left -= group;
    // A = X X^T (wide) or X^T X (tall), and C = b I + c A
    Params g{};
    if (!cut) g = a_and_c(a.scale_x * a.scale_x);
    g.batch = a.m; g.M = g.N = p.n; g.tri = 1;
    g.a_zstep = g.b_zstep = 2;
    // The diagonal is a sum of equal signs, and what it loses moves all singular values the same way: 1524 x 65 is off by 2.5e-6 at
    // chunks of 4 and 1.7e-6 at 1 for the same time.  It no longer shows with many rows, where it costs time (8 x 2048 x 2048: about 1 %).
    g.chunk_kb = p.n <= 512 ? 1 : 4;
    if (cut) {
      g.alpha = 1.f; g.splits = p.gram.splits; g.c_zstep = p.gram.splits;
      if (p.tall) LS_TRY((gop::launch<2, true, true, true, gop::EPI_F32>(p.gram.nt, xk[cur], xk[cur], gf, gf, g, p.k, st)));
      else LS_TRY((gop::launch<2, true, false, false, gop::EPI_F32>(p.gram.nt, xk[cur], xk[cur], gf, gf, g, p.k, st)));
      const float unit = 1.f / (a.scale_x * a.scale_x);
      const FoldArgs f{reinterpret_cast<const float*>(ws + p.o_gram), static_cast<__half*>(ac), p.n, p.gram.splits, p.ldf, p.planef,
                       p.ldn, p.plane_n, kScaleA * unit, kNsC * kScaleC * unit, kNsB * kScaleC};
      const unsigned nb = (unsigned)((p.n + 63) / 64);
      LS_TRY(launch_dep(ns_gram_fold_kernel, dim3(nb * (nb + 1) / 2, (unsigned)a.m), dim3(256), 0, st, 1, f));
    } else {
      g.mirror = 1; g.c_zstep = 4;
      if (p.tall) LS_TRY((gop::launch<2, true, true, true, gop::EPI_PIECES>(p.gram.nt, xk[cur], xk[cur], aco, act, g, p.k, st)));
      else LS_TRY((gop::launch<2, true, false, false, gop::EPI_PIECES>(p.gram.nt, xk[cur], xk[cur], aco, act, g, p.k, st)));
    }
    // P = a I + A C, and Q = the product of the group's P
    const Params make_p = one(kScaleP / (kScaleA * kScaleC), kNsA * kScaleP);
    LS_TRY(square(ack, 4, ack, 4, 2, so[0], sq[0], 2, make_p));
    int ip = 0, iq = 0;
    float scale_q = kScaleP;
    for (int s = 1; s < group; ++s) {
      const int ib = ip == iq ? 1 : 3 - ip - iq;        // neither P nor Q
      LS_TRY(square(ack, 4, sk[ip], 2, 0, so[ib], sq[ib], 2, one(kScaleB / (kScaleA * kScaleP), 0.f)));
      LS_TRY(square(sk[ib], 2, sk[ip], 2, 0, aco, act, 4, a_and_c(kScaleB * kScaleP)));
      ip = ib;
      LS_TRY(square(ack, 4, ack, 4, 2, so[ip], sq[ip], 2, make_p));
      const int in = 3 - ip - iq;
      LS_TRY(square(sk[ip], 2, sk[iq], 2, 0, so[in], sq[in], 2, one(kScaleQ[s - 1] / (kScaleP * scale_q), 0.f)));
      iq = in;
      scale_q = kScaleQ[s - 1];
    }
    // X <- Q X (wide) or X Q (tall)
    g = one(1.f / scale_q, 0.f);
    g.batch = a.m; g.M = a.rows; g.N = a.cols;
    g.a_zstep = g.b_zstep = g.c_zstep = 2;
    g.dominant = p.tall ? 2 : 1;
    // (directions of large singular values are sums over the whole K: 722 x 805 of rank 45 and noise is 1.95 times as far off as fp32
    // arithmetic at chunks of 8 here and in P, 1.2 times at 4; 2 x 2501 x 1000: 464 and 474 us)
    g.chunk_kb = 4;
    if (p.tall) LS_TRY((gop::launch<2, true, false, false, gop::EPI_PIECES>(p.full.nt, xk[cur], sk[iq], xo[cur ^ 1], xo[cur ^ 1], g, p.n, st)));
    else LS_TRY((gop::launch<2, true, false, true, gop::EPI_PIECES>(p.full.nt, sk[iq], xk[cur], xo[cur ^ 1], xo[cur ^ 1], g, p.n, st)));
  }
  const float step = a.lr * sqrtf(fmaxf(1.f, (float)a.rows / (float)a.cols));
  LS_TRY(launch_dep(ns_finish_kernel<G, MUON, VEC>, grid, dim3(32 * kWarps), 0, st, 1, a, static_cast<const __half*>(x[cur]), step));
  return LS_OK;
}

// 16-byte (bf16: 8-byte) accesses need every row and replica of every tensor of the call to start on such a boundary.
template <typename G, bool MUON>
int pick_ns(const MatArgs& a, int steps, char* ws, cudaStream_t st) {
  const size_t e = sizeof(G) * 4;
  bool vec = a.cols % 4 == 0 && !off(a.g, e) && !off(a.out, e) && !off(a.w, 16) && !off(a.v, 16);
  if (a.m > 1) vec = vec && a.g_stride % 4 == 0 && a.out_stride % 4 == 0 && a.w_stride % 4 == 0 && a.v_stride % 4 == 0;
  return vec ? run_ns<G, MUON, true>(a, steps, ws, st) : run_ns<G, MUON, false>(a, steps, ws, st);
}

int check_sizes(int m, int rows, int cols) {
  if (m < 1 || rows < 1 || cols < 1) return LS_ERR_INVALID_ARG;
  if (m > 65535 || rows > kMaxSide || cols > kMaxSide) return LS_ERR_TOO_LARGE;
  return LS_OK;
}

int check_ws(int m, int rows, int cols, const void* ws, size_t ws_bytes) {
  if (ws == nullptr) return LS_ERR_INVALID_ARG;
  if (ws_bytes < make_plan(m, rows, cols).total || off(ws, 256)) return LS_ERR_STATE_SIZE;
  return LS_OK;
}

}  // namespace

int muon_step(float* w_dev, float* v_dev, const void* g_dev, int m, int rows, int cols, int64_t w_stride, int64_t v_stride,
              int64_t g_stride, int g_dtype, float lr, float momentum, int nesterov, int steps, bool blocked, void* ws_dev,
              size_t ws_bytes, cudaStream_t st) {
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
  a.m = m; a.rows = rows; a.cols = cols; a.lr = lr; a.mu = momentum; a.nesterov = nesterov; a.blocked = blocked ? 1 : 0;
  return g_dtype == LS_DTYPE_BF16 ? pick_ns<__nv_bfloat16, true>(a, steps, static_cast<char*>(ws_dev), st)
                                  : pick_ns<float, true>(a, steps, static_cast<char*>(ws_dev), st);
}

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
  return dtype == LS_DTYPE_BF16 ? pick_ns<__nv_bfloat16, false>(a, steps, static_cast<char*>(ws_dev), st)
                                : pick_ns<float, false>(a, steps, static_cast<char*>(ws_dev), st);
}

extern "C" int ls_muon_step(float* w_dev, float* v_dev, const void* g_dev, int m, int rows, int cols, int64_t w_stride,
                            int64_t v_stride, int64_t g_stride, int g_dtype, float lr, float momentum, int nesterov, int steps, void* ws_dev,
                            size_t ws_bytes, void* cuda_stream) {
  return ls::muon_step(w_dev, v_dev, g_dev, m, rows, cols, w_stride, v_stride, g_stride, g_dtype, lr, momentum, nesterov, steps,
                       false, ws_dev, ws_bytes, static_cast<cudaStream_t>(cuda_stream));
}
