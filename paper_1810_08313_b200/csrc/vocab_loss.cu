// Softmax cross entropy of a wide output matrix and its gradient (ls_vocab_loss, ls_vocab_loss_grad).
//
//   z = h W^T  [rows][V];   loss_n = log sum_v exp z_nv - z_n,y(n);   loss = mean of the rows that have a label
//   dz = exp(z - lse) - onehot(y);   dh = dz W / count;   dW = dz^T h / count
//
// The three products are 6 rows V d flops and bound the call; what must not be added to them is traffic of rows x V
// numbers in fp32.  The logits never reach memory in the loss: the product's epilogue reduces every row of a 256 x 256 tile to
// (maximum, sum of exponentials) per slice of half a tile's columns, and a small kernel combines those.  The gradient needs the
// normalised probabilities twice, as an operand of dh (contracted over V) and of dW (contracted over rows), and their
// normaliser only when the last column is known.  Recomputing the logits would cost a third more flops; instead a piece
// of rows (at most 2^29 elements of the piece's probabilities, 1 GiB) keeps exp(z - slice maximum) as 16-bit numbers,
// a streaming pass scales them to dz in bf16 in place (4 bytes a logit against 6 d flops), and both products
// read them.  The number is rounded once more, so it has 11 bits and not bf16's 8: its error (2^-11) disappears under the bf16
// rounding of dz (2^-8), which the tensor cores need and which is of the same size as the rounding of the bf16 results.
// It keeps them down to 2^-62 of the slice's maximum, 43 nats, so that an unlikely column's dz is as accurate as a likely
// one's (pack_e16 in gemm_op.cuh).  The label's logit is no part of any slice: with S the sum of the other columns and e_y the label's
// term, the loss of a row with S < e_y is log1p(S / e_y) and dz at the label -S / (S + e_y), which lose nothing
// however certain the row is (of a rounded log-sum-exp, 1 - p is right to 1e-6 only).  The factor
// scale / count is applied to the fp32 accumulators: in dz it would give every uncertain row the same rounding error
// of 1 / count, where -1 is exact.
//
// fp32 tensors: operands as three bf16 pieces (24 bits) and six products (gemm_op.cuh), logits kept in fp32 for a piece of rows, dz
// in three pieces; sums over several pieces of rows are added into dW by the bulk-copy engine in fp32.  A few rows take the
// CUDA cores instead (vocab_few_*).
//
// The row sums, the loss and every accumulation are fp32 or wider and in a fixed order: results are
// reproducible bit for bit (the atomic counter only picks the CTA that finishes).
#include "gemm_op.cuh"

#include <math.h>

namespace ls {
namespace {

using gop::Params;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ bool has_label(int y, int V) { return y >= 0 && y < V; }

// ---- slices -> log-sum-exp and row loss: 32 rows per CTA, 32 warps take every 32nd slice ------------------------------
// The last CTA to finish also counts the replica's labels (inv_count given: first piece of rows) and takes the mean of its
// row losses (loss given: last piece), in double, thread by thread and then in thread order.  `done` counts the CTAs; the
// product before this launch has cleared it.
// (blockIdx.y: replicas taken together, stat_z and all_rows apart.)
struct CombineArgs {
  const float *stat_max, *stat_sum;
  int64_t stat_ld, stat_z;
  int slices, rows, V;
  const int32_t* labels;          // of the piece
  float* label;                   // the label's logit; replaced by dz at the label
  const float* label_lo;          // what it leaves over, or null
  float *lse, *row_loss;
  float2* norm;                   // fp32 gradient: (reference of the exponentials, their sum) of the piece's rows, or null
  unsigned* done;
  // of the whole replica
  const int32_t* all_labels;
  const float* all_row_loss;
  int64_t all_rows;
  float *inv_count, *loss;
};
__global__ void __launch_bounds__(1024) vocab_combine_kernel(CombineArgs a) {
  __shared__ float smax[32][33], ssum[32][33];
  __shared__ double sum[32];
  __shared__ long long cnt[32];
  __shared__ bool last;
  const int lane = threadIdx.x & 31, wp = threadIdx.x >> 5;
  const int row = blockIdx.x * 32 + lane;
  const int64_t z = blockIdx.y;
  a.stat_max += z * a.stat_z; a.stat_sum += z * a.stat_z;
  a.labels += z * a.all_rows; a.label += z * a.all_rows; a.lse += z * a.all_rows; a.row_loss += z * a.all_rows;
  a.all_labels += z * a.all_rows; a.all_row_loss += z * a.all_rows;
  a.done += z;
  if (a.norm != nullptr) a.norm += z * a.all_rows;
  if (a.label_lo != nullptr) a.label_lo += z * a.all_rows;
  if (a.inv_count != nullptr) a.inv_count += z;
  if (a.loss != nullptr) a.loss += z;
  grid_dep_wait();
  grid_dep_launch();
  int y = -1;
  float zy = 0.f, zy_lo = 0.f;                              // (whatever is there without a label)
  if (wp == 0 && row < a.rows) {
    y = a.labels[row];
    zy = __ldcg(a.label + row);
    if (a.label_lo != nullptr) zy_lo = __ldcg(a.label_lo + row);
  }
  // eight slices at a time, their sixteen loads in flight together
  float m = -INFINITY, s = 0.f;
  if (row < a.rows) {
    for (int t0 = wp; t0 < a.slices; t0 += 8 * 32) {
      float tm[8], ts[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int64_t at = (int64_t)(t0 + i * 32) * a.stat_ld + row;
        const bool in = t0 + i * 32 < a.slices;
        tm[i] = in ? __ldcg(a.stat_max + at) : -INFINITY;
        ts[i] = in ? __ldcg(a.stat_sum + at) : 0.f;
      }
      float top = m;
#pragma unroll
      for (int i = 0; i < 8; ++i) top = fmaxf(top, tm[i]);
      const float ref = top == -INFINITY ? 0.f : top;
      if (m != -INFINITY) s *= gop::ex2(m - ref);               // (only -inf so far: nothing to add, or NaN)
#pragma unroll
      for (int i = 0; i < 8; ++i) s += tm[i] == -INFINITY ? ts[i] : ts[i] * gop::ex2(tm[i] - ref);
      m = top;
    }
  }
  smax[wp][lane] = m; ssum[wp][lane] = s;
  __syncthreads();
  if (wp == 0 && row < a.rows) {
    float M = -INFINITY;
#pragma unroll
    for (int i = 0; i < 32; ++i) M = fmaxf(M, smax[i][lane]);
    float S = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      const float tm = smax[i][lane];
      S += tm == -INFINITY ? ssum[i][lane] : ssum[i][lane] * gop::ex2(tm - M);
    }
    // the label's term, with the larger reference of the two (a NaN stays out of the reference and enters the sum)
    const bool labelled = has_label(y, a.V);
    const float ry = !labelled ? -INFINITY : zy < 0.f && zy != -INFINITY ? fmaxf(zy * kLog2e, -3.4e38f) : zy * kLog2e;
    const float top = fmaxf(M, ry);
    const float ref = top == -INFINITY ? 0.f : top;
    if (M != -INFINITY) S *= gop::ex2(M - ref);
    const double dy = fma((double)zy + (double)zy_lo, (double)kLog2e, -(double)ref);
    const float ey = labelled ? gop::ex2((float)dy) : 0.f;
    const float T = S + ey;
    // T is a sum of 2^(z kLog2e - ref), so that log-sum-exp and row loss are differences in that base, formed in double: rounded,
    // a log-sum-exp of 20 is off by 1e-6, and so would be the loss
    const double log_sum = (double)logf(T) * (1.0 / (double)kLn2);
    a.lse[row] = (float)(((double)ref + log_sum) / (double)kLog2e);
    if (a.norm != nullptr) a.norm[row] = make_float2(ref, T);
    float loss = 0.f;
    if (labelled) {
      loss = S < ey ? log1pf(S / ey) : (float)((log_sum - dy) / (double)kLog2e);
      a.label[row] = -(S / T);
    }
    a.row_loss[row] = loss;
  }
  if (a.inv_count == nullptr && a.loss == nullptr) return;
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) last = atomicAdd(a.done, 1u) == gridDim.x - 1;
  __syncthreads();
  if (!last) return;
  __threadfence();
  double ls = 0.0;
  long long n = 0;
  for (int64_t i = threadIdx.x; i < a.all_rows; i += 1024)
    if (has_label(a.all_labels[i], a.V)) {
      ++n;
      if (a.loss != nullptr) ls += (double)__ldcg(a.all_row_loss + i);
    }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    ls += __shfl_xor_sync(0xffffffffu, ls, o);
    n += __shfl_xor_sync(0xffffffffu, n, o);
  }
  if (lane == 0) { sum[wp] = ls; cnt[wp] = n; }
  __syncthreads();
  if (threadIdx.x == 0) {
    ls = 0.0; n = 0;
    for (int i = 0; i < 32; ++i) { ls += sum[i]; n += cnt[i]; }
    if (a.inv_count != nullptr) *a.inv_count = n > 0 ? (float)(1.0 / (double)n) : 0.f;
    if (a.loss != nullptr) *a.loss = n > 0 ? (float)(ls / (double)n) : 0.f;
  }
}

// ---- exponentials -> dz, eight columns per thread ------------------------------------------------------------------------
// bf16: in place over the 16-bit exponentials.  Rows from `rows` to `pad`, which fill the last K block of dW, become zeros.
// What the launch that forms dz does to a row of h for dW: rows without a label are cleared, so that whatever they hold stays out
// of dW.  h itself is the caller's: where the product read it in place (src given), the other rows are copied into the
// workspace; where it was laid out there already, they stay.
struct HRows {
  const __nv_bfloat16* src;
  __nv_bfloat16* dst;
  int64_t ld, piece;
  int64_t src_z, dst_z;                    // between replicas
  int d, np;
};
__device__ __forceinline__ void h_row(const HRows& h, int64_t z, int row, bool labelled) {
  const int n = (h.d + 7) / 8;             // pieces of 16 bytes (rows of the workspace are padded to whole ones)
  uint4* dst = reinterpret_cast<uint4*>(h.dst + z * h.dst_z + (int64_t)row * h.ld);
  if (!labelled) {
    for (int q = 0; q < h.np; ++q)
      for (int i = threadIdx.x; i < n; i += blockDim.x) dst[q * (h.piece / 8) + i] = make_uint4(0, 0, 0, 0);
  } else if (h.src != nullptr) {
    const uint4* src = reinterpret_cast<const uint4*>(h.src + z * h.src_z + (int64_t)row * h.d);
    for (int i = threadIdx.x; i < n; i += blockDim.x) dst[i] = src[i];
  }
}

// A CTA takes four rows of 2048 columns: a thread's four groups of eight columns lie below one another, in one slice, whose four
// maxima are one load.  (Four groups of one row read as many sectors of the statistics as of a row; 8192 x 65536: 424 us.)
constexpr int kDzCols = 2048, kDzRows = 4;
struct DzStep { int64_t e, out, stat, rows; };          // elements between replicas (blockIdx.z)
__global__ void __launch_bounds__(256)
vocab_dz_bf16_kernel(uint16_t* e, int64_t ld, int rows, int pad, int V, const float* stat_max, int64_t stat_ld, int slice,
                     const int32_t* labels, const float* label_dz, const float* lse, const HRows h, const DzStep by) {
  const int row0 = blockIdx.y * kDzRows;
  const int c = blockIdx.x * kDzCols + threadIdx.x * 8;
  const int64_t z = blockIdx.z;
  e += z * by.e; stat_max += z * by.stat; labels += z * by.rows; label_dz += z * by.rows; lse += z * by.rows;
  grid_dep_wait();
  grid_dep_launch();
  int y[kDzRows];
#pragma unroll
  for (int k = 0; k < kDzRows; ++k) y[k] = row0 + k < rows ? labels[row0 + k] : -1;
#pragma unroll
  for (int k = 0; k < kDzRows; ++k)
    if (k % gridDim.x == blockIdx.x && row0 + k < pad) h_row(h, z, row0 + k, has_label(y[k], V));
  if (c >= V) return;
  uint16_t* at = e + (int64_t)row0 * ld + c;
  // (rows of the statistics beyond the last one exist, padded to whole 256)
  const float4 top4 = __ldg(reinterpret_cast<const float4*>(stat_max + (int64_t)(c / slice) * stat_ld + row0));
  const float top[kDzRows] = {top4.x, top4.y, top4.z, top4.w};
  uint4 u[kDzRows];
  float l[kDzRows];
#pragma unroll
  for (int k = 0; k < kDzRows; ++k)
    if (has_label(y[k], V)) {
      u[k] = *reinterpret_cast<const uint4*>(at + k * ld);
      l[k] = lse[row0 + k];
    }
#pragma unroll
  for (int k = 0; k < kDzRows; ++k) {
    if (row0 + k >= pad) break;
    uint32_t w[4] = {0, 0, 0, 0};
    if (has_label(y[k], V)) {
      const uint32_t in[4] = {u[k].x, u[k].y, u[k].z, u[k].w};
      const float f = gop::ex2(top[k] - l[k] * kLog2e) * gop::kE16Scale;
      float v[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 t = gop::unpack_e16(in[i]);
        v[2 * i] = t.x * f; v[2 * i + 1] = t.y * f;
      }
      const int d = y[k] - c;
      if (d >= 0 && d < 8) {
        const float py = label_dz[row0 + k];
#pragma unroll
        for (int i = 0; i < 8; ++i) if (i == d) v[i] = py;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = gop::pack_bf16(v[2 * i], v[2 * i + 1]);
    }
    *reinterpret_cast<uint4*>(at + k * ld) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// x = p0 + p1 + p2, each piece the bf16 rounding of what is left.  The first piece stays finite: the products pair every
// piece with others that may be zero, and 0 * inf would be a NaN.  An infinite x counts as the largest bf16 number.
__device__ __forceinline__ void split3(float x, __nv_bfloat16 (&p)[3]) {
  const float kMax = 3.3895313892515355e38f;                  // 0x7f7f
  p[0] = isnan(x) ? __float2bfloat16_rn(x) : __float2bfloat16_rn(fminf(fmaxf(x, -kMax), kMax));
  const float r = isinf(x) ? 0.f : x - __bfloat162float(p[0]);
  p[1] = __float2bfloat16_rn(r);
  p[2] = __float2bfloat16_rn(r - __bfloat162float(p[1]));
}

// dz of an fp32 logit: exp(z - lse) as 2^(z log2(e) - M) / S with the reference M that the sum S was formed with.  lse itself, rounded
// at its size, would put an error of 1e-6 at a log-sum-exp of 20 into every number of the row.
struct Norm {
  float ref, inv;
  __device__ __forceinline__ explicit Norm(float2 n) : ref(n.x), inv(1.f / n.y) {}
  __device__ __forceinline__ float p(float z) const { return exp2f(fmaf(z, kLog2e, -ref)) * inv; }
};

// fp32: logits z -> three pieces of dz.
__global__ void __launch_bounds__(256)
vocab_dz_fp32_kernel(const float* z, __nv_bfloat16* out, int64_t ld, int64_t piece, int rows, int V, const int32_t* labels,
                     const float* label_dz, const float2* norm, const HRows h, const DzStep by) {
  const int row = blockIdx.y;
  const int c = (blockIdx.x * 256 + threadIdx.x) * 4;
  const int64_t rep = blockIdx.z;
  z += rep * by.e; out += rep * by.out; labels += rep * by.rows; label_dz += rep * by.rows; norm += rep * by.rows;
  grid_dep_wait();
  grid_dep_launch();
  const int y = row < rows ? labels[row] : -1;
  if (blockIdx.x == 0) h_row(h, rep, row, has_label(y, V));
  if (c >= V) return;
  const int64_t at = (int64_t)row * ld + c;
  float v[4] = {0.f, 0.f, 0.f, 0.f};
  if (has_label(y, V)) {
    const Norm n(norm[row]);
    const float4 u = *reinterpret_cast<const float4*>(z + at);
    v[0] = n.p(u.x); v[1] = n.p(u.y); v[2] = n.p(u.z); v[3] = n.p(u.w);
    const int d = y - c;
    if (d >= 0 && d < 4) {
      const float py = label_dz[row];
#pragma unroll
      for (int i = 0; i < 4; ++i) if (i == d) v[i] = py;
    }
  }
  __nv_bfloat16 p[4][3];
#pragma unroll
  for (int i = 0; i < 4; ++i) split3(v[i], p[i]);
#pragma unroll
  for (int q = 0; q < 3; ++q) {
    uint2 w;
    __nv_bfloat162 a = __halves2bfloat162(p[0][q], p[1][q]), b = __halves2bfloat162(p[2][q], p[3][q]);
    w.x = *reinterpret_cast<uint32_t*>(&a); w.y = *reinterpret_cast<uint32_t*>(&b);
    *reinterpret_cast<uint2*>(out + q * piece + at) = w;
  }
}

// ---- operands into the workspace: rows padded to whole 16 bytes, fp32 cut into three pieces ------------------------------
template <typename T>
__global__ void __launch_bounds__(256)
vocab_pack_kernel(const T* src, int64_t src_z, int64_t rows, int d, __nv_bfloat16* dst, int64_t dst_z, int64_t ld, int64_t piece,
                  bool vec) {
  src += blockIdx.y * src_z;                   // replica
  dst += blockIdx.y * dst_z;
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int PER = F32 ? 4 : 8;
  const int per_row = (d + PER - 1) / PER;
  grid_dep_wait();
  grid_dep_launch();
  const int64_t total = rows * per_row;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / per_row;
    const int c = (int)(i - row * per_row) * PER;
    T v[PER];
    if (vec) {
      *reinterpret_cast<uint4*>(v) = *reinterpret_cast<const uint4*>(src + row * d + c);
    } else {
#pragma unroll
      for (int k = 0; k < PER; ++k) v[k] = c + k < d ? src[row * d + c + k] : (T)0.f;
    }
    if constexpr (F32) {
      __nv_bfloat16 p[4][3];
#pragma unroll
      for (int k = 0; k < 4; ++k) split3(v[k], p[k]);
#pragma unroll
      for (int q = 0; q < 3; ++q) {
        __nv_bfloat162 a = __halves2bfloat162(p[0][q], p[1][q]), b = __halves2bfloat162(p[2][q], p[3][q]);
        *reinterpret_cast<uint2*>(dst + q * piece + row * ld + c) =
            make_uint2(*reinterpret_cast<uint32_t*>(&a), *reinterpret_cast<uint32_t*>(&b));
      }
    } else {
      *reinterpret_cast<uint4*>(dst + row * ld + c) = *reinterpret_cast<const uint4*>(v);
    }
  }
}

// ---- sum of fp32 planes in index order, rounded to the output type --------------------------------------------------------
template <typename T>
__global__ void __launch_bounds__(256)
vocab_fold_kernel(const float* part, int planes, int64_t plane, int64_t ld, int64_t rows, int d, T* out, int64_t out_stride) {
  const int per_row = (d + 3) / 4;
  grid_dep_wait();
  grid_dep_launch();
  part += blockIdx.y * planes * plane;         // replica
  out += blockIdx.y * out_stride;
  const int64_t total = rows * per_row;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / per_row;
    const int c = (int)(i - row * per_row) * 4;
    float4 s = *reinterpret_cast<const float4*>(part + row * ld + c);
    for (int p = 1; p < planes; ++p) {
      const float4 t = *reinterpret_cast<const float4*>(part + p * plane + row * ld + c);
      s.x += t.x; s.y += t.y; s.z += t.z; s.w += t.w;
    }
    const float v[4] = {s.x, s.y, s.z, s.w};
    T* o = out + row * d + c;
#pragma unroll
    for (int k = 0; k < 4; ++k) if (c + k < d) o[k] = (T)v[k];
  }
}

// ---- few rows: CUDA cores (bf16: of the gradient, after the product that gives the logits) ------------------------------
// With a handful of rows W is all there is to read, and products of rows padded to 256 take longer than the FMAs; laying
// an fp32 W out as pieces alone moves 2.5 times its bytes.  Here W is read once for the logits and once more for the
// gradient, whose pass also writes dW (kFewRows says up to where).  The logits' kernel is bound by the latency of its steps, at 3
// to 4 TB/s of W for 8 rows; the gradient's by HBM, 5 TB/s for 8 rows.

// An infinity counts as the largest bf16 number, as it does in split3(); NaN stays.
__device__ __forceinline__ float finite(float x) {
  const float kMax = 3.3895313892515355e38f;
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(x), "f"(-kMax));
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(y), "f"(kMax));
  return y;
}
__device__ __forceinline__ float4 finite(float4 v) { return make_float4(finite(v.x), finite(v.y), finite(v.z), finite(v.w)); }

template <typename T>
__device__ __forceinline__ float few_operand(float x) { return sizeof(T) == 4 ? finite(x) : x; }

struct FewArgs {
  const float *h, *W;
  int64_t h_stride, w_stride;
  int rows, V, d;
  float* z;                       // [replica][rows][ldz] logits, or null
  int64_t ldz;
  float *stat_max, *stat_sum;
  int64_t stat_ld, stat_z;
  const int32_t* labels;
  float* label_logit;
  unsigned* done;                 // cleared for the combining launch
};
// Logits of RT rows and 128 columns per CTA: 32-wide steps of d through a ring of cp.async, a thread has four columns and RT / 4
// rows.  A warp's eight columns and four rows at a time are one shared-memory wavefront each (rows 144 bytes apart).  The
// products of a step are added up by themselves first.
constexpr int kFewCols = 128, kFewStep = 32, kFewPitch = 36, kFewStages = 3;
template <int RT>
constexpr int kFewSmem = kFewStages * (kFewCols + RT) * kFewPitch * 4;

template <bool VEC>
__device__ __forceinline__ void few_copy(float* dst, const float* src, int64_t row, int rows, int d, int k, int piece) {
  // piece: four floats of the step; floats past the row's end, and rows past the last, become zeros
  const bool in = row < rows;
  const float* from = src + (in ? row : 0) * d;
  if constexpr (VEC) {
    const int c = k + piece * 4;
    const int left = in && c < d ? 16 : 0;
    asm volatile("cp.async.cg.shared.global.L2::256B [%0], [%1], 16, %2;" ::"r"(ptx::smem_u32(dst + piece * 4)),
                 "l"(from + (left ? c : 0)), "r"(left) : "memory");
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = k + piece * 4 + i;
      const int left = in && c < d ? 4 : 0;
      asm volatile("cp.async.ca.shared.global.L2::256B [%0], [%1], 4, %2;" ::"r"(ptx::smem_u32(dst + piece * 4 + i)),
                   "l"(from + (left ? c : 0)), "r"(left) : "memory");
    }
  }
}

template <int RT, bool VEC>
__global__ void __launch_bounds__(128) vocab_few_logits_kernel(const FewArgs a) {
  constexpr int RPT = RT / 4;
  extern __shared__ __align__(16) float few[];
  const int lane = threadIdx.x & 31, wp = threadIdx.x >> 5;
  const int tiles = (a.rows + RT - 1) / RT;                     // of rows: neighbouring CTAs read the same columns' rows of W
  const int slice = blockIdx.x / tiles;
  const int row0 = (int)(blockIdx.x - slice * tiles) * RT;
  const int64_t v0 = (int64_t)slice * kFewCols, z = blockIdx.z;
  grid_dep_wait();
  grid_dep_launch();
  if (blockIdx.x == 0 && threadIdx.x == 0) a.done[z] = 0u;
  const float* W = a.W + z * a.w_stride;
  const float* h = a.h + z * a.h_stride;
  const int steps = (a.d + kFewStep - 1) / kFewStep;
  auto load = [&](int s) {
    if (s < steps) {
      float* w = few + (s % kFewStages) * (kFewCols + RT) * kFewPitch;
      float* hs = w + kFewCols * kFewPitch;
#pragma unroll
      for (int i = 0; i < kFewCols / 16; ++i) {
        const int r = i * 16 + (threadIdx.x >> 3);
        few_copy<VEC>(w + r * kFewPitch, W, v0 + r, a.V, a.d, s * kFewStep, threadIdx.x & 7);
      }
#pragma unroll
      for (int i = 0; i < (RT + 15) / 16; ++i) {
        const int r = i * 16 + (threadIdx.x >> 3);
        if (r < RT) few_copy<VEC>(hs + r * kFewPitch, h, row0 + r, a.rows, a.d, s * kFewStep, threadIdx.x & 7);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  const int vl = wp * 32 + (lane & 7), rl = lane >> 3;          // columns vl + 8 i, rows rl + 4 j
  float acc[4][RPT];
  auto pass = [&](auto clamp) {
    for (int s = 0; s < kFewStages - 1; ++s) load(s);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < RPT; ++j) acc[i][j] = 0.f;
    for (int s = 0; s < steps; ++s) {
      asm volatile("cp.async.wait_group %0;" ::"n"(kFewStages - 2) : "memory");
      __syncthreads();                                          // step s is there, and step s - 1 has been read
      load(s + kFewStages - 1);
      const float* w = few + (s % kFewStages) * (kFewCols + RT) * kFewPitch;
      const float* hs = w + kFewCols * kFewPitch;
      float part[4][RPT];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < RPT; ++j) part[i][j] = 0.f;
#pragma unroll
      for (int k = 0; k < kFewStep; k += 4) {
        float4 wv[4], hv[RPT];
#pragma unroll
        for (int i = 0; i < 4; ++i) wv[i] = clamp(*reinterpret_cast<const float4*>(w + (vl + 8 * i) * kFewPitch + k));
#pragma unroll
        for (int j = 0; j < RPT; ++j) hv[j] = clamp(*reinterpret_cast<const float4*>(hs + (rl + 4 * j) * kFewPitch + k));
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < RPT; ++j) {
            float t = part[i][j];
            t = fmaf(wv[i].x, hv[j].x, t);
            t = fmaf(wv[i].y, hv[j].y, t);
            t = fmaf(wv[i].z, hv[j].z, t);
            part[i][j] = fmaf(wv[i].w, hv[j].w, t);
          }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < RPT; ++j) acc[i][j] += part[i][j];
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();
  };
  pass([](float4 v) { return v; });
  // an infinite operand leaves an infinity or a NaN in every sum it enters: only then once more, with operands made finite
  float odd = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < RPT; ++j) odd = isfinite(acc[i][j]) ? odd : 1.f;
  if (__syncthreads_or(odd != 0.f)) pass([](float4 v) { return finite(v); });
  // the tile through shared memory: a warp takes a row's 128 logits, one slice of the statistics
  constexpr int kPitch = kFewCols + 4;
  static_assert(RT * kPitch * 4 <= kFewSmem<RT>, "tile of logits");
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < RPT; ++j) few[(rl + 4 * j) * kPitch + vl + 8 * i] = acc[i][j];
  __syncthreads();
  for (int r = wp; r < RT; r += 4) {
    const int row = row0 + r;
    if (row >= a.rows) break;
    const int64_t c = v0 + lane * 4;
    const float4 t = *reinterpret_cast<const float4*>(few + r * kPitch + lane * 4);
    float v[4] = {t.x, t.y, t.z, t.w};
    const int64_t lab = a.labels[z * a.rows + row] - c;
    float mx = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (c + i >= a.V) v[i] = -INFINITY;
      else if (lab == i) {                                        // no part of the statistics: EPI_STATS
        a.label_logit[z * a.rows + row] = v[i];
        v[i] = -INFINITY;
      }
      mx = fmaxf(mx, v[i]);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    // (the reference stays finite for a finite maximum, and where there is nothing but -inf: EPI_STATS)
    const float ref = mx == -INFINITY ? 0.f : mx < 0.f ? fmaxf(mx * kLog2e, -3.4e38f) : mx * kLog2e;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) sum += gop::ex2(fmaf(v[i], kLog2e, -ref));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) {
      const int64_t at = z * a.stat_z + (int64_t)slice * a.stat_ld + row;
      a.stat_max[at] = mx == -INFINITY ? -INFINITY : ref;
      a.stat_sum[at] = sum;
    }
    if (a.z != nullptr && c < a.V)
      *reinterpret_cast<float4*>(a.z + (z * a.rows + row) * a.ldz + c) = make_float4(v[0], v[1], v[2], v[3]);
  }
}

// z -> dz in place, four columns a thread
__global__ void __launch_bounds__(256)
vocab_few_dz_kernel(float* zz, int64_t ld, int rows, int V, const int32_t* labels, const float* label_dz, const float2* norm) {
  const int64_t at_row = (int64_t)blockIdx.z * rows + blockIdx.y;
  const int c = (blockIdx.x * 256 + threadIdx.x) * 4;
  grid_dep_wait();
  grid_dep_launch();
  if (c >= V) return;
  const int y = labels[at_row];
  float4* at = reinterpret_cast<float4*>(zz + at_row * ld + c);
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  if (has_label(y, V)) {
    const Norm n(norm[at_row]);
    const float4 u = *at;
    o = make_float4(n.p(u.x), n.p(u.y), n.p(u.z), n.p(u.w));
    const int d = y - c;
    if (d >= 0 && d < 4) {
      const float py = label_dz[at_row];
      if (d == 0) o.x = py;
      else if (d == 1) o.y = py;
      else if (d == 2) o.z = py;
      else o.w = py;
    }
  }
  *at = o;
}

// dW = dz^T h and, per block of `block` columns of dz, its part of dh = dz W.  A CTA has 128 (bf16: 256) elements of d, a warp every
// fourth row of W of the block: a lane reads its 16 bytes, adds them times dz to RT rows of dh in registers, and writes the 16
// bytes of dW from RT rows of h in registers.  The warps' sums of dh are added in order.
template <typename T>
struct FewGradArgs {
  const T *h, *W;
  const float* dz;
  int64_t h_stride, w_stride, dw_stride, ldz;
  int rows, V, d, block;
  const int32_t* labels;
  const float* inv;
  float scale;
  T* dW;
  float* part;                    // [replica][block][rows][ldp]
  int64_t ldp;
};
template <typename T, int RT, bool VEC>
__global__ void __launch_bounds__(128) vocab_few_grad_kernel(const FewGradArgs<T> a) {
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int C = F32 ? 4 : 8, kWide = 32 * C;   // elements of a lane, of a CTA
  constexpr int kChunk = 128, kRows = 4;           // columns of dz in shared memory at a time; rows of W that a warp reads at a time
  static_assert(F32 || VEC, "bf16 rows of whole 16 bytes");
  __shared__ __align__(16) float dz[kChunk][RT];
  __shared__ float sum[4][RT][kWide];
  const int lane = threadIdx.x & 31, wp = threadIdx.x >> 5;
  const int64_t z = blockIdx.z;
  const int k0 = blockIdx.x * kWide;
  grid_dep_wait();
  grid_dep_launch();
  const T* W = a.W + z * a.w_stride;
  T* dW = a.dW + z * a.dw_stride;
  const float* zz = a.dz + z * a.rows * a.ldz;
  const float alpha = a.scale * a.inv[z];
  auto col = [&](int i) { return VEC ? k0 + lane * C + i : k0 + i * 32 + lane; };
  float h[RT][C], acc[RT][C];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const bool in = r < a.rows && has_label(a.labels[z * a.rows + (r < a.rows ? r : 0)], a.V);
#pragma unroll
    for (int i = 0; i < C; ++i) {
      h[r][i] = in && col(i) < a.d ? few_operand<T>((float)a.h[z * a.h_stride + (int64_t)r * a.d + col(i)]) : 0.f;
      acc[r][i] = 0.f;
    }
  }
  const int from = blockIdx.y * a.block, to = min(from + a.block, a.V);
  uint4 w[kRows];                                  // as they lie in memory
  auto read = [&](int v0) {                        // rows v0, v0 + 4, ...
#pragma unroll
    for (int q = 0; q < kRows; ++q) {
      const int64_t at = (int64_t)(v0 + q * 4) * a.d;
      const bool in = v0 + q * 4 < to;
      w[q] = make_uint4(0, 0, 0, 0);
      if constexpr (VEC) {
        if (in && col(0) < a.d) w[q] = __ldg(reinterpret_cast<const uint4*>(W + at + col(0)));
      } else {
        uint32_t* e = reinterpret_cast<uint32_t*>(&w[q]);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (in && col(i) < a.d) e[i] = __float_as_uint(__ldg(W + at + col(i)));
      }
    }
  };
  read(from + wp);
  for (int c0 = from; c0 < to; c0 += kChunk) {
    __syncthreads();
    for (int i = threadIdx.x; i < kChunk * RT; i += 128) {
      const int r = i / kChunk, c = i - r * kChunk;
      dz[c][r] = r < a.rows && c0 + c < to ? zz[r * a.ldz + c0 + c] : 0.f;
    }
    __syncthreads();
    for (int c = wp; c < kChunk && c0 + c < to; c += 4 * kRows) {
      uint4 x[kRows];
#pragma unroll
      for (int q = 0; q < kRows; ++q) x[q] = w[q];
      read(c0 + c + 4 * kRows);                    // the next ones, also across chunks
#pragma unroll
      for (int q = 0; q < kRows; ++q) {
        const uint32_t u[4] = {x[q].x, x[q].y, x[q].z, x[q].w};
        float f[C], o[C];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if constexpr (F32) {
            f[i] = few_operand<T>(__uint_as_float(u[i]));
          } else {
            f[2 * i] = __uint_as_float(u[i] << 16);
            f[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
          }
        }
#pragma unroll
        for (int i = 0; i < C; ++i) o[i] = 0.f;
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          const float g = dz[c + q * 4][r];
#pragma unroll
          for (int i = 0; i < C; ++i) {
            acc[r][i] = fmaf(g, f[i], acc[r][i]);
            o[i] = fmaf(g, h[r][i], o[i]);
          }
        }
        const int v = c0 + c + q * 4;
        if (v < to) {
          const int64_t at = (int64_t)v * a.d;
          if constexpr (VEC) {
            uint32_t p[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              if constexpr (F32) p[i] = __float_as_uint(alpha * o[i]);
              else p[i] = gop::pack_bf16(alpha * o[2 * i], alpha * o[2 * i + 1]);
            }
            if (col(0) < a.d) *reinterpret_cast<uint4*>(dW + at + col(0)) = make_uint4(p[0], p[1], p[2], p[3]);
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) if (col(i) < a.d) dW[at + col(i)] = alpha * o[i];
          }
        }
      }
    }
  }
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int i = 0; i < C; ++i) sum[wp][r][VEC ? lane * C + i : i * 32 + lane] = acc[r][i];
  __syncthreads();
  float* part = a.part + (z * gridDim.y + blockIdx.y) * a.rows * a.ldp;
  for (int t = threadIdx.x; t < kWide && k0 + t < a.d; t += 128)
    for (int r = 0; r < a.rows; ++r)
      part[r * a.ldp + k0 + t] = alpha * (((sum[0][r][t] + sum[1][r][t]) + sum[2][r][t]) + sum[3][r][t]);
}

// ---- plan: what a call keeps in its workspace ---------------------------------------------------------------------------------
constexpr int64_t kMaxVocab = 1 << 24, kMaxWidth = 1 << 16;
// At most so many rows go to the CUDA cores.  fp32 loss of 118995 x 1608: 8 rows 229 us, 32 rows 435, 64 rows 810, on the tensor
// cores 790 for any of them (32000 x 2048: 138 us for 32 rows, 257).  fp32 gradient: 8 rows 530 us, 16 rows 830, tensor cores
// 1270.  bf16 gradient of 118992 x 1608: 4 rows 280 us, 8 rows 379, tensor cores 288; dz stays in fp32 here, whose
// rounding to bf16 no other row would average.
constexpr int64_t kFewRows = 32, kFewRowsGrad = 16, kFewRowsGrad16 = 4;
// bf16: up to so many rows the labels' logits are formed on their own (gop::label_dots()).
constexpr int64_t kDotRows = 4;

int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

struct Plan {
  bool f32, grad;
  bool few;             // few rows on the CUDA cores, all replicas at once
  int np;
  int batch;            // replicas taken together: all of them where the rows are one piece and the workspace stays small
  int64_t R;            // rows of a piece
  int64_t pieces;
  int64_t Vp, dp;       // padded row lengths: probabilities, packed operands
  int64_t df;           // padded row length of fp32 sums
  int nt, nt_dh, nt_dw;
  int slices;
  int64_t stat_ld;
  int splits;           // of the contraction over V in dh
  int block;            // few rows: columns of a part
  bool dh_fold, dw_fold;   // dh, dW pass through an fp32 sum in the workspace (several parts, or rows of no whole 16 bytes)
  size_t o_stat, o_logit, o_lse, o_rowloss, o_norm, o_inv, o_done, o_e, o_dz, o_h, o_w, o_dh, o_dw, total;
};

int check_sizes(int m, int64_t rows, int64_t vocab, int d, int dtype) {
  if (m < 1 || rows < 0 || vocab < 1 || d < 1) return LS_ERR_INVALID_ARG;
  if (dtype != LS_DTYPE_FP32 && dtype != LS_DTYPE_BF16) return LS_ERR_INVALID_ARG;
  if (m > 65535 || rows > 2147483647ll || vocab > kMaxVocab || d > kMaxWidth) return LS_ERR_TOO_LARGE;
  return LS_OK;
}

// What m replicas need that are taken `batch` at a time.
Plan replica_plan(Plan p, int m, int batch, int64_t rows, int64_t V, int d) {
  const bool grad = p.grad, lay = p.f32 || d % 8 != 0;
  p.batch = batch;
  p.stat_ld = p.R;
  // tile widths of the three products (a slice of the statistics is half a tile)
  const int64_t most_rows = p.R < rows ? p.R : rows;
  p.nt = gop::pick_nt(most_rows, V, p.batch, false);
  const gop::Cut cut = gop::pick_cut(most_rows, d, batch, false, V, p.np, grad ? 64 : 1);
  p.nt_dh = cut.nt;
  p.splits = cut.splits;
  p.nt_dw = gop::pick_nt(V, d, batch, false);
  p.slices = (int)(2 * ((V + p.nt - 1) / p.nt));
  const bool whole = d % (p.f32 ? 4 : 8) == 0;
  p.dh_fold = grad && (p.splits > 1 || !whole);
  p.dw_fold = grad && (!whole || (!p.f32 && p.pieces > 1));
  size_t at = 0;
  auto take = [&at](int64_t bytes) { size_t o = at; at += (size_t)round_up(bytes, 256); return o; };
  p.o_stat = take(2 * (int64_t)p.batch * p.slices * p.stat_ld * 4);
  p.o_logit = take(m * rows * 8);          // (and what it leaves over)
  p.o_lse = take(m * rows * 4);
  p.o_rowloss = take(m * rows * 4);
  p.o_norm = take(p.f32 && grad ? batch * p.R * 8 : 0);
  p.o_inv = take(m * 4);
  p.o_done = take(4 * (int64_t)p.batch);
  // operands laid out anew: fp32 ones (as pieces), bf16 ones whose rows are no whole 16 bytes, and, for dW, h with the
  // rows that have no label cleared
  p.o_h = take(lay || grad ? batch * p.np * p.R * p.dp * 2 : 0);
  p.o_w = take(lay ? batch * p.np * V * p.dp * 2 : 0);
  if (grad) {
    p.o_e = take(batch * p.R * p.Vp * (p.f32 ? 4 : 2));
    p.o_dz = p.f32 ? take(batch * 3 * p.R * p.Vp * 2) : p.o_e;
    p.o_dh = take(p.dh_fold ? (int64_t)batch * p.splits * p.R * p.df * 4 : 0);
    p.o_dw = take(p.dw_fold ? batch * V * p.df * 4 : 0);
  }
  p.total = at;
  return p;
}

// The parts of dh: about four CTAs an SM, in blocks of whole 64 columns.
Plan few_plan(Plan p, int m, int64_t rows, int64_t V, int d) {
  p.batch = m;
  p.nt = gop::pick_nt(rows, V, m, false);                  // (bf16: the logits are a product of all replicas)
  p.slices = (int)(p.f32 ? (V + kFewCols - 1) / kFewCols : 2 * ((V + p.nt - 1) / p.nt));
  p.stat_ld = round_up(rows, 32);
  const int64_t wide = p.f32 ? 128 : 256, kb = (d + wide - 1) / wide, want = (148 * 4 + kb * m - 1) / (kb * m);
  p.block = (int)round_up((V + want - 1) / want, 64);
  p.splits = (int)((V + p.block - 1) / p.block);
  size_t at = 0;
  auto take = [&at](int64_t bytes) { size_t o = at; at += (size_t)round_up(bytes, 256); return o; };
  p.o_stat = take(2 * (int64_t)m * p.slices * p.stat_ld * 4);
  p.o_logit = take(m * rows * 8);          // (and what it leaves over)
  p.o_lse = take(m * rows * 4);
  p.o_rowloss = take(m * rows * 4);
  p.o_norm = take(m * rows * 8);
  p.o_inv = take(m * 4);
  p.o_done = take(m * 4);
  if (p.grad) {
    p.o_e = take(m * rows * p.Vp * 4);
    p.o_dh = take(m * p.splits * rows * p.df * 4);
  }
  p.total = at;
  return p;
}

Plan make_plan(int m, int64_t rows, int64_t V, int d, int dtype, bool grad) {
  Plan p{};
  p.f32 = dtype == LS_DTYPE_FP32;
  p.grad = grad;
  p.np = p.f32 ? 3 : 1;
  p.Vp = round_up(V, 64);
  p.dp = round_up(d, 8);
  p.df = round_up(d, 4);
  // rows of a piece: the probabilities of a piece of a gradient, or the statistics of a piece of a loss, stay bounded
  const int64_t most = grad ? (p.f32 ? (int64_t)1 << 27 : (int64_t)1 << 29) / p.Vp : ((int64_t)1 << 31) / p.Vp;
  int64_t R = most / 256 * 256;
  if (R < 256) R = 256;
  p.pieces = rows > 0 ? (rows + R - 1) / R : 0;
  p.R = rows > 0 ? round_up((rows + p.pieces - 1) / p.pieces, 256) : 0;
  p.pieces = rows > 0 ? (rows + p.R - 1) / p.R : 0;
  p.few = rows > 0 && (p.f32 ? rows <= (grad ? kFewRowsGrad : kFewRows) : grad && d % 8 == 0 && rows <= kFewRowsGrad16);
  if (p.few) return few_plan(p, m, rows, V, d);
  // All replicas in one set of launches while the workspace of that stays below 512 MB; larger ones fill the GPU by
  // themselves (fp32 gradients, time on the GPU: 2 x 513 x 10007 x 760 381 -> 339 us, 4 x 178 x 21522 x 512 605 -> 397 us).
  if (m > 1 && p.pieces == 1) {
    const Plan all = replica_plan(p, m, m, rows, V, d);
    if (all.total <= (size_t)1 << 29) return all;
  }
  return replica_plan(p, m, 1, rows, V, d);
}

// Rows of a box of an operand with so many rows in all.
int box_rows(int64_t rows) { return rows < 64 ? (int)round_up(rows, 8) : 64; }

unsigned stream_grid(int64_t items) {
  const int64_t g = (items + 255) / 256;
  return (unsigned)(g < 148 * 8 ? (g < 1 ? 1 : g) : 148 * 8);
}

template <typename T>
cudaError_t pack(const T* src, int64_t src_z, int m, int64_t rows, int d, __nv_bfloat16* dst, int64_t dst_z, int64_t ld,
                 int64_t piece, cudaStream_t st) {
  const int per = 16 / sizeof(T);
  const bool vec = d % per == 0 && reinterpret_cast<uintptr_t>(src) % 16 == 0 && (m == 1 || src_z % per == 0);
  return launch_dep(vocab_pack_kernel<T>, dim3(stream_grid(rows * ((d + per - 1) / per)), (unsigned)m), dim3(256), 0, st, 1, src,
                    src_z, rows, d, dst, dst_z, ld, piece, vec);
}

struct VocabArgs {
  const void *h, *W;
  const int32_t* labels;
  int m;
  int64_t rows, V;
  int d;
  int64_t h_stride, w_stride, dh_stride, dw_stride;
  int dtype;
  float scale;
  float *loss, *row_loss, *lse;
  void *dh, *dW;
  char* ws;
};

#define LS_TRY(x)                                   \
  do {                                              \
    if ((x) != cudaSuccess) return LS_ERR_CUDA;     \
  } while (0)

// One replica, or p.batch of them from `rep` on.  T: element type of h, W, dh, dW.  NP: pieces an operand is given in.
template <typename T, int NP>
int run_replica(const VocabArgs& a, const Plan& p, int rep, cudaStream_t st) {
  constexpr bool F32 = NP == 3;
  constexpr int kRow = gop::box_row(NP);
  using bf = __nv_bfloat16;
  const T* h = static_cast<const T*>(a.h) + rep * a.h_stride;
  const T* W = static_cast<const T*>(a.W) + rep * a.w_stride;
  const int32_t* labels = a.labels + rep * a.rows;
  float* stat_max = reinterpret_cast<float*>(a.ws + p.o_stat);
  const int64_t stat_z = p.slices * p.stat_ld;
  float* stat_sum = stat_max + p.batch * stat_z;
  float* logit = reinterpret_cast<float*>(a.ws + p.o_logit) + rep * a.rows;
  float* lse = (a.lse ? a.lse : reinterpret_cast<float*>(a.ws + p.o_lse)) + rep * a.rows;
  float* row_loss = (a.row_loss ? a.row_loss : reinterpret_cast<float*>(a.ws + p.o_rowloss)) + rep * a.rows;
  float* inv = reinterpret_cast<float*>(a.ws + p.o_inv) + rep;
  float2* norm = reinterpret_cast<float2*>(a.ws + p.o_norm);
  unsigned* done = reinterpret_cast<unsigned*>(a.ws + p.o_done);
  bf* hpack = reinterpret_cast<bf*>(a.ws + p.o_h);
  bf* wpack = reinterpret_cast<bf*>(a.ws + p.o_w);
  const int64_t V = a.V;
  const int d = a.d;
  const bool lay = F32 || d % 8 != 0;
  const int nb = p.batch;
  const bool many = nb > 1;
  if (lay) LS_TRY(pack<T>(W, a.w_stride, nb, V, d, wpack, NP * V * p.dp, p.dp, V * p.dp, st));
  const bf* wop = lay ? wpack : reinterpret_cast<const bf*>(W);
  const int64_t wld = lay ? p.dp : d;
  CUtensorMap mw;
  LS_TRY(gop::make_operand_map(&mw, wop, gop::MAP_BF16, V, d, nb * NP, wld, many && !lay ? a.w_stride : V * wld));
  for (int64_t r0 = 0, piece = 0; r0 < a.rows; r0 += p.R, ++piece) {
    const int64_t rn = a.rows - r0 < p.R ? a.rows - r0 : p.R;
    const T* hr = h + r0 * d;
    const int64_t hplane = p.R * p.dp;
    if (lay) LS_TRY(pack<T>(hr, a.h_stride, nb, rn, d, hpack, NP * hplane, p.dp, hplane, st));
    const bf* hop = lay ? hpack : reinterpret_cast<const bf*>(hr);
    const int64_t hld = lay ? p.dp : d;
    CUtensorMap mh, me;
    const int a_box = box_rows(rn);
    LS_TRY(gop::make_operand_map(&mh, hop, gop::MAP_BF16, rn, d, nb * NP, hld, many && !lay ? a.h_stride : hplane, a_box));
    // logits
    Params g{};
    g.batch = nb; g.a_zstep = g.b_zstep = NP; g.c_zstep = 1; g.splits = 1; g.M = (int)rn; g.N = (int)V; g.alpha = 1.f;
    g.stat_max = stat_max; g.stat_sum = stat_sum; g.stat_ld = p.stat_ld; g.stat_z = stat_z; g.label_z = a.rows;
    g.labels = labels + r0; g.label_logit = logit + r0; g.clear = done; g.a_box = a_box;
    float* label_lo = nullptr;
    if (!F32 && a.rows <= kDotRows) {
      label_lo = logit + a.m * a.rows;
      g.dot_h = reinterpret_cast<const bf*>(h); g.dot_w = reinterpret_cast<const bf*>(W);
      g.dot_hz = a.h_stride; g.dot_wz = a.w_stride; g.dot_d = d; g.label_lo = label_lo;
    }
    if (!p.grad) {
      LS_TRY((gop::launch<NP, false, false, false, gop::EPI_STATS>(p.nt, mh, mw, mh, mh, g, d, st)));
    } else {
      constexpr gop::Epi kEpi = F32 ? gop::EPI_STATS_F32 : gop::EPI_STATS_E16;
      LS_TRY(gop::make_output_map(&me, a.ws + p.o_e, F32 ? gop::MAP_F32 : gop::MAP_F16, rn, V, nb, p.Vp, p.R * p.Vp, kRow));
      LS_TRY((gop::launch<NP, false, false, false, kEpi>(p.nt, mh, mw, me, me, g, d, st)));
    }
    CombineArgs cb{};
    cb.stat_max = stat_max; cb.stat_sum = stat_sum; cb.stat_ld = p.stat_ld; cb.stat_z = stat_z; cb.slices = p.slices;
    cb.rows = (int)rn; cb.V = (int)V;
    cb.labels = labels + r0; cb.label = logit + r0; cb.label_lo = label_lo; cb.lse = lse + r0; cb.row_loss = row_loss + r0;
    cb.done = done; cb.all_labels = labels; cb.all_row_loss = row_loss; cb.all_rows = a.rows;
    cb.norm = F32 && p.grad ? norm : nullptr;
    if (p.grad && piece == 0) cb.inv_count = inv;
    if (r0 + p.R >= a.rows) cb.loss = a.loss + rep;
    LS_TRY(launch_dep(vocab_combine_kernel, dim3((unsigned)((rn + 31) / 32), (unsigned)p.batch), dim3(1024), 0, st, 1, cb));
    if (!p.grad) continue;
    // dz
    bf* dz = reinterpret_cast<bf*>(a.ws + p.o_dz);
    const HRows hrows{lay ? nullptr : hop, hpack, p.dp, hplane, a.h_stride, NP * hplane, d, NP};
    const DzStep by{p.R * p.Vp, NP * p.R * p.Vp, stat_z, a.rows};
    // (grid.y is limited to 65535 rows a launch; p.R rows are there, so that the padding is, too)
    const int64_t rp = round_up(rn, 64);
    for (int64_t q0 = 0; q0 < rp; q0 += 65280) {
      const int qn = (int)(rp - q0 < 65280 ? rp - q0 : 65280), ql = (int)(rn - q0 < qn ? rn - q0 : qn);
      const int32_t* ly = labels + r0 + q0;
      HRows hr_q = hrows;
      hr_q.dst += q0 * p.dp;
      if (hr_q.src != nullptr) hr_q.src += q0 * d;
      if (F32) {
        LS_TRY(launch_dep(vocab_dz_fp32_kernel, dim3((unsigned)((V + 1023) / 1024), (unsigned)qn, (unsigned)nb), dim3(256), 0, st, 1,
                          reinterpret_cast<const float*>(a.ws + p.o_e) + q0 * p.Vp, dz + q0 * p.Vp, p.Vp, p.R * p.Vp, ql, (int)V,
                          ly, logit + r0 + q0, norm + q0, hr_q, by));
      } else {
        LS_TRY(launch_dep(vocab_dz_bf16_kernel,
                          dim3((unsigned)((V + kDzCols - 1) / kDzCols), (unsigned)(qn + kDzRows - 1) / kDzRows, (unsigned)nb), dim3(256), 0, st, 1, reinterpret_cast<uint16_t*>(dz) + q0 * p.Vp, p.Vp, ql, qn, (int)V,
                          stat_max + q0, p.stat_ld, p.nt / 2, ly, logit + r0 + q0, lse + r0 + q0, hr_q, by));
      }
    }
    CUtensorMap mz, mzk, mhz, mo;
    LS_TRY(gop::make_operand_map(&mz, dz, gop::MAP_BF16, rp, V, nb * NP, p.Vp, p.R * p.Vp));
    LS_TRY(gop::make_operand_map(&mzk, dz, gop::MAP_BF16, rn, V, nb * NP, p.Vp, p.R * p.Vp, a_box));
    // dh = dz W
    T* dh = static_cast<T*>(a.dh) + rep * a.dh_stride + r0 * d;
    Params gh{};
    gh.batch = nb; gh.a_zstep = gh.b_zstep = NP; gh.c_zstep = 1; gh.splits = p.splits; gh.M = (int)rn; gh.N = d; gh.alpha = a.scale; gh.alpha_dev = inv; gh.n_fast = 1; gh.a_box = a_box;
    if (p.dh_fold) {
      float* part = reinterpret_cast<float*>(a.ws + p.o_dh);
      gh.c_zstep = p.splits;
      LS_TRY(gop::make_output_map(&mo, part, gop::MAP_F32, rn, d, (int64_t)nb * p.splits, p.df, p.R * p.df, kRow));
      LS_TRY((gop::launch<NP, false, false, true, gop::EPI_F32>(p.nt_dh, mzk, mw, mo, mo, gh, V, st)));
      LS_TRY(launch_dep(vocab_fold_kernel<T>, dim3(stream_grid(rn * ((d + 3) / 4)), (unsigned)nb), dim3(256), 0, st, 1,
                        static_cast<const float*>(part), p.splits, p.R * p.df, p.df, rn, d, dh, a.dh_stride));
    } else {
      LS_TRY(gop::make_output_map(&mo, dh, F32 ? gop::MAP_F32 : gop::MAP_BF16, rn, d, nb, d, many ? a.dh_stride : rn * d, kRow));
      LS_TRY((gop::launch<NP, false, false, true, F32 ? gop::EPI_F32 : gop::EPI_BF16>(p.nt_dh, mzk, mw, mo, mo, gh, V, st)));
    }
    // dW (+)= dz^T h, with the rows that have no label cleared
    LS_TRY(gop::make_operand_map(&mhz, hpack, gop::MAP_BF16, rp, d, nb * NP, p.dp, hplane));
    T* dW = static_cast<T*>(a.dW) + rep * a.dw_stride;
    Params gw{};
    gw.batch = nb; gw.a_zstep = gw.b_zstep = NP; gw.c_zstep = 1; gw.splits = 1; gw.M = (int)V; gw.N = d; gw.alpha = a.scale; gw.alpha_dev = inv; gw.n_fast = 1;
    gw.reduce = piece > 0;
    if (p.dw_fold) {
      float* sum = reinterpret_cast<float*>(a.ws + p.o_dw);
      LS_TRY(gop::make_output_map(&mo, sum, gop::MAP_F32, V, d, nb, p.df, V * p.df, kRow));
      LS_TRY((gop::launch<NP, false, true, true, gop::EPI_F32>(p.nt_dw, mz, mhz, mo, mo, gw, rn, st)));
      if (r0 + p.R >= a.rows)
        LS_TRY(launch_dep(vocab_fold_kernel<T>, dim3(stream_grid(V * ((d + 3) / 4)), (unsigned)nb), dim3(256), 0, st, 1,
                          static_cast<const float*>(sum), 1, V * p.df, p.df, V, d, dW, a.dw_stride));
    } else {
      LS_TRY(gop::make_output_map(&mo, dW, F32 ? gop::MAP_F32 : gop::MAP_BF16, V, d, nb, d, many ? a.dw_stride : V * d, kRow));
      LS_TRY((gop::launch<NP, false, true, true, F32 ? gop::EPI_F32 : gop::EPI_BF16>(p.nt_dw, mz, mhz, mo, mo, gw, rn, st)));
    }
  }
  return LS_OK;
}

template <int RT, bool VEC>
cudaError_t launch_few_logits(const FewArgs& f, unsigned m, cudaStream_t st) {
  static uint64_t configured = 0;        // one bit per device
  auto kern = vocab_few_logits_kernel<RT, VEC>;
  const cudaError_t e = allow_dynamic_smem(kern, kFewSmem<RT>, &configured);
  if (e != cudaSuccess) return e;
  const dim3 grid((unsigned)((f.rows + RT - 1) / RT) * (unsigned)((f.V + kFewCols - 1) / kFewCols), 1, m);
  return launch_dep(kern, grid, dim3(128), kFewSmem<RT>, st, 1, f);
}
template <typename T, bool VEC>
int run_few(const VocabArgs& a, const Plan& p, cudaStream_t st) {
  const unsigned m = (unsigned)a.m;
  const int rows = (int)a.rows, V = (int)a.V;
  float* z = p.grad ? reinterpret_cast<float*>(a.ws + p.o_e) : nullptr;
  float* stat_max = reinterpret_cast<float*>(a.ws + p.o_stat);
  const int64_t stat_z = p.slices * p.stat_ld;
  float* stat_sum = stat_max + m * stat_z;
  float* logit = reinterpret_cast<float*>(a.ws + p.o_logit);
  unsigned* done = reinterpret_cast<unsigned*>(a.ws + p.o_done);
  float* label_lo = nullptr;
  if constexpr (sizeof(T) == 4) {
    FewArgs f{};
    f.h = static_cast<const float*>(a.h); f.W = static_cast<const float*>(a.W);
    f.h_stride = a.h_stride; f.w_stride = a.w_stride; f.rows = rows; f.V = V; f.d = a.d;
    f.z = z; f.ldz = p.Vp;
    f.stat_max = stat_max; f.stat_sum = stat_sum; f.stat_ld = p.stat_ld; f.stat_z = stat_z;
    f.labels = a.labels; f.label_logit = logit; f.done = done;
    if (rows <= 8) LS_TRY((launch_few_logits<8, VEC>(f, m, st)));
    else if (rows <= 16) LS_TRY((launch_few_logits<16, VEC>(f, m, st)));
    else LS_TRY((launch_few_logits<32, VEC>(f, m, st)));
  } else {
    CUtensorMap mh, mw, mz;
    const int a_box = box_rows(rows);
    LS_TRY(gop::make_operand_map(&mh, a.h, gop::MAP_BF16, rows, a.d, m, a.d, m > 1 ? a.h_stride : (int64_t)rows * a.d, a_box));
    LS_TRY(gop::make_operand_map(&mw, a.W, gop::MAP_BF16, V, a.d, m, a.d, m > 1 ? a.w_stride : a.V * a.d));
    LS_TRY(gop::make_output_map(&mz, z, gop::MAP_F32, rows, V, m, p.Vp, rows * p.Vp, gop::box_row(1)));
    Params g{};
    g.batch = a.m; g.a_zstep = g.b_zstep = g.c_zstep = 1; g.splits = 1; g.M = rows; g.N = V; g.alpha = 1.f;
    g.stat_max = stat_max; g.stat_sum = stat_sum; g.stat_ld = p.stat_ld; g.stat_z = stat_z; g.label_z = rows;
    g.labels = a.labels; g.label_logit = logit; g.clear = done; g.a_box = a_box;
    label_lo = logit + m * a.rows;
    g.dot_h = reinterpret_cast<const __nv_bfloat16*>(a.h); g.dot_w = reinterpret_cast<const __nv_bfloat16*>(a.W);
    g.dot_hz = a.h_stride; g.dot_wz = a.w_stride; g.dot_d = a.d; g.label_lo = label_lo;
    LS_TRY((gop::launch<1, false, false, false, gop::EPI_STATS_F32>(p.nt, mh, mw, mz, mz, g, a.d, st)));
  }
  CombineArgs cb{};
  cb.stat_max = stat_max; cb.stat_sum = stat_sum; cb.stat_ld = p.stat_ld; cb.stat_z = stat_z; cb.slices = p.slices;
  cb.rows = rows; cb.V = V; cb.labels = cb.all_labels = a.labels; cb.label = logit; cb.label_lo = label_lo;
  cb.lse = a.lse ? a.lse : reinterpret_cast<float*>(a.ws + p.o_lse);
  cb.row_loss = a.row_loss ? a.row_loss : reinterpret_cast<float*>(a.ws + p.o_rowloss);
  cb.all_row_loss = cb.row_loss; cb.all_rows = a.rows; cb.done = done; cb.loss = a.loss;
  float2* norm = reinterpret_cast<float2*>(a.ws + p.o_norm);
  float* inv = reinterpret_cast<float*>(a.ws + p.o_inv);
  if (p.grad) { cb.norm = norm; cb.inv_count = inv; }
  LS_TRY(launch_dep(vocab_combine_kernel, dim3((unsigned)((rows + 31) / 32), m), dim3(1024), 0, st, 1, cb));
  if (!p.grad) return LS_OK;
  LS_TRY(launch_dep(vocab_few_dz_kernel, dim3((unsigned)((V + 1023) / 1024), (unsigned)rows, m), dim3(256), 0, st, 1, z, p.Vp, rows, V,
                    a.labels, static_cast<const float*>(logit), static_cast<const float2*>(norm)));
  FewGradArgs<T> g{};
  g.h = static_cast<const T*>(a.h); g.W = static_cast<const T*>(a.W); g.dz = z;
  g.h_stride = a.h_stride; g.w_stride = a.w_stride; g.dw_stride = a.dw_stride; g.ldz = p.Vp;
  g.rows = rows; g.V = V; g.d = a.d; g.block = p.block; g.labels = a.labels; g.inv = inv; g.scale = a.scale;
  g.dW = static_cast<T*>(a.dW); g.part = reinterpret_cast<float*>(a.ws + p.o_dh); g.ldp = p.df;
  constexpr int kWide = sizeof(T) == 4 ? 128 : 256;
  const dim3 grid((unsigned)((a.d + kWide - 1) / kWide), (unsigned)p.splits, m);
  if (rows <= 4) LS_TRY(launch_dep(vocab_few_grad_kernel<T, 4, VEC>, grid, dim3(128), 0, st, 1, g));
  if constexpr (sizeof(T) == 4) {
    if (rows > 4 && rows <= 8) LS_TRY(launch_dep(vocab_few_grad_kernel<T, 8, VEC>, grid, dim3(128), 0, st, 1, g));
    if (rows > 8) LS_TRY(launch_dep(vocab_few_grad_kernel<T, 16, VEC>, grid, dim3(128), 0, st, 1, g));
  }
  LS_TRY(launch_dep(vocab_fold_kernel<T>, dim3(stream_grid(a.rows * ((a.d + 3) / 4)), m), dim3(256), 0, st, 1,
                    static_cast<const float*>(g.part), p.splits, rows * p.df, p.df, a.rows, a.d, static_cast<T*>(a.dh), a.dh_stride));
  return LS_OK;
}

int run_vocab(const VocabArgs& a, bool grad, size_t ws_bytes, cudaStream_t st) {
  const Plan p = make_plan(a.m, a.rows, a.V, a.d, a.dtype, grad);
  if (ws_bytes < p.total || reinterpret_cast<uintptr_t>(a.ws) % 256 != 0) return LS_ERR_STATE_SIZE;
  const size_t eb = a.dtype == LS_DTYPE_BF16 ? 2 : 4;
  if (a.rows == 0) {
    LS_TRY(cudaMemsetAsync(a.loss, 0, a.m * sizeof(float), st));
    if (grad)
      for (int i = 0; i < a.m; ++i)
        LS_TRY(cudaMemsetAsync(static_cast<char*>(a.dW) + i * a.dw_stride * eb, 0, (size_t)a.V * a.d * eb, st));
    return LS_OK;
  }
  if (p.few && !p.f32) return run_few<__nv_bfloat16, true>(a, p, st);
  if (p.few) return a.d % 4 == 0 ? run_few<float, true>(a, p, st) : run_few<float, false>(a, p, st);
  for (int i = 0; i < a.m; i += p.batch) {
    const int rc = p.f32 ? run_replica<float, 3>(a, p, i, st) : run_replica<__nv_bfloat16, 1>(a, p, i, st);
    if (rc != LS_OK) return rc;
  }
  return LS_OK;
}

bool off(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }

int check_call(const VocabArgs& a, bool grad) {
  int rc = check_sizes(a.m, a.rows, a.V, a.d, a.dtype);
  if (rc != LS_OK) return rc;
  if (a.W == nullptr || a.loss == nullptr || a.ws == nullptr) return LS_ERR_INVALID_ARG;
  if (a.rows > 0 && (a.h == nullptr || a.labels == nullptr)) return LS_ERR_INVALID_ARG;
  const size_t eb = a.dtype == LS_DTYPE_BF16 ? 2 : 4;
  if (off(a.h, eb) || off(a.W, eb) || off(a.labels, 4) || off(a.loss, 4) || off(a.row_loss, 4) || off(a.lse, 4))
    return LS_ERR_INVALID_ARG;
  if (a.m > 1 && (a.h_stride < a.rows * a.d || a.w_stride < a.V * a.d)) return LS_ERR_INVALID_ARG;
  // rows of whole 16 bytes are moved by bulk copies, which start on 16-byte boundaries
  const int per = a.dtype == LS_DTYPE_BF16 ? 8 : 4;
  const bool whole = a.d % per == 0, many = a.m > 1;
  if (whole && (off(a.h, 16) || off(a.W, 16) || (many && (a.h_stride % per != 0 || a.w_stride % per != 0))))
    return LS_ERR_INVALID_ARG;
  if (grad) {
    if (a.dW == nullptr || (a.rows > 0 && a.dh == nullptr) || off(a.dW, eb) || off(a.dh, eb)) return LS_ERR_INVALID_ARG;
    if (a.m > 1 && (a.dh_stride < a.rows * a.d || a.dw_stride < a.V * a.d)) return LS_ERR_INVALID_ARG;
    if (whole && (off(a.dh, 16) || off(a.dW, 16) || (many && (a.dh_stride % per != 0 || a.dw_stride % per != 0))))
      return LS_ERR_INVALID_ARG;
    if (!isfinite(a.scale)) return LS_ERR_INVALID_ARG;
  }
  return LS_OK;
}

}  // namespace
}  // namespace ls

extern "C" int ls_vocab_loss_ws_bytes(int m, int64_t rows, int64_t vocab, int d, int dtype, int grad, size_t* bytes) {
  using namespace ls;
  int rc = check_sizes(m, rows, vocab, d, dtype);
  if (rc != LS_OK) return rc;
  if (bytes == nullptr) return LS_ERR_INVALID_ARG;
  // (few rows take less for a gradient than for a loss, which then runs on other kernels: the gradient's size serves both)
  const size_t loss = make_plan(m, rows, vocab, d, dtype, false).total, both = grad != 0 ? make_plan(m, rows, vocab, d, dtype, true).total : 0;
  *bytes = loss > both ? loss : both;
  return LS_OK;
}

extern "C" int ls_vocab_loss(const void* h_dev, const void* W_dev, const int32_t* labels_dev, int m, int64_t rows,
                             int64_t vocab, int d, int64_t h_stride, int64_t w_stride, int dtype, float* loss_dev,
                             float* row_loss_dev, float* lse_dev, void* ws_dev, size_t ws_bytes, void* cuda_stream) {
  using namespace ls;
  VocabArgs a{};
  a.h = h_dev; a.W = W_dev; a.labels = labels_dev; a.m = m; a.rows = rows; a.V = vocab; a.d = d;
  a.h_stride = h_stride; a.w_stride = w_stride; a.dtype = dtype;
  a.loss = loss_dev; a.row_loss = row_loss_dev; a.lse = lse_dev; a.ws = static_cast<char*>(ws_dev);
  int rc = check_call(a, false);
  return rc != LS_OK ? rc : run_vocab(a, false, ws_bytes, static_cast<cudaStream_t>(cuda_stream));
}

extern "C" int ls_vocab_loss_grad(const void* h_dev, const void* W_dev, const int32_t* labels_dev, int m, int64_t rows,
                                  int64_t vocab, int d, int64_t h_stride, int64_t w_stride, int dtype, float scale,
                                  float* loss_dev, float* row_loss_dev, float* lse_dev, void* dh_dev, int64_t dh_stride,
                                  void* dW_dev, int64_t dw_stride, void* ws_dev, size_t ws_bytes, void* cuda_stream) {
  using namespace ls;
  VocabArgs a{};
  a.h = h_dev; a.W = W_dev; a.labels = labels_dev; a.m = m; a.rows = rows; a.V = vocab; a.d = d;
  a.h_stride = h_stride; a.w_stride = w_stride; a.dh_stride = dh_stride; a.dw_stride = dw_stride; a.dtype = dtype;
  a.scale = scale;
  a.loss = loss_dev; a.row_loss = row_loss_dev; a.lse = lse_dev; a.dh = dh_dev; a.dW = dW_dev;
  a.ws = static_cast<char*>(ws_dev);
  int rc = check_call(a, true);
  return rc != LS_OK ? rc : run_vocab(a, true, ws_bytes, static_cast<cudaStream_t>(cuda_stream));
}
