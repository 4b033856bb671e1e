// What the attention kernels (attention_simt.cu, attention_tc.cu) share: the arguments of a call, where the sequence of a
// row starts and ends, and the rows computed one by one from the formulas.
//
//   s_ij = scale q_i . k_j  for start(i) <= j <= i,   p_i = softmax(s_i),   out_i = sum_j p_ij v_j,   lse_i = log sum_j exp s_ij
//   P_ij = exp(s_ij - lse_i),  D_i = dout_i . out_i,  dS_ij = P_ij (dout_i . v_j - D_i)
//   dq_i = scale sum_j dS_ij k_j,   dk_j = scale sum_i dS_ij q_i,   dv_j = sum_i P_ij dout_i
//
// Tiles are cut out of the packed rows of a replica, whatever sequences they hold: row i attends to the keys from the start of
// its own sequence to itself, so a tile of rows needs the keys from its first row's start on.  Short sequences share tiles, and
// the host needs to know no lengths.
//
// A product of a whole tile multiplies what the mask leaves out by zero, and zero times an infinity or NaN is NaN.  So a row
// of the result that is not finite is computed once more, alone, over the rows that it depends on: a NaN in one sequence, or in
// the rows behind the last one, reaches no other.
#pragma once

#include "gemm_op.cuh"
#include "ls_internal.h"

#include <math.h>

namespace ls {
namespace attn {

struct Tensor {                          // [m][tokens][heads][head_dim]; distances in elements
  void* p;
  int64_t row, replica;
};

struct Args {
  Tensor q, k, v, out, dout, dq, dk, dv;
  float* lse;                            // [m][heads][tokens]
  float* dot;                            // D, the same (backward)
  const int32_t* seq_start;              // [m][n_seqs + 1], or null: one sequence of all tokens
  int64_t tokens;
  int m, heads, kv_heads, head_dim, n_seqs;
  float scale;
  int* err;
};

// The boundaries of a replica's sequences, as a whole warp sees them: up to 32 are loaded once, one a lane, and searched with
// ballots; more are searched 32 at a time.  (A binary search of 24 boundaries is six loads one after another, some 2 us of a CTA
// that has 10 us of work.)  Whatever the boundaries hold, the results stay within the rows.
struct Bounds {
  const int32_t* b;                      // null: one sequence of all rows
  int n, tokens;                         // sequences, rows
  int held;                              // lane l: boundary l, or none

  __device__ __forceinline__ Bounds(const Args& a, int rep) {
    n = a.n_seqs;
    tokens = (int)a.tokens;
    b = a.seq_start == nullptr ? nullptr : a.seq_start + (int64_t)rep * (n + 1);
    const int lane = threadIdx.x & 31;
    held = b != nullptr && lane <= n ? b[lane] : 0x7fffffff;
  }
  __device__ __forceinline__ int at(int i) const { return n < 32 ? __shfl_sync(0xffffffffu, held, i) : b[i]; }
  // the number of boundaries that are <= t (one t for the warp)
  __device__ __forceinline__ int upto(int t) const {
    if (n < 32) return __popc(__ballot_sync(0xffffffffu, held <= t));
    const int lane = threadIdx.x & 31;
    int lo = 0, hi = n + 1;
    while (lo < hi) {
      const int step = (hi - lo + 31) / 32, i = lo + lane * step;
      const int before = __popc(__ballot_sync(0xffffffffu, i < hi && b[min(i, n)] <= t));
      if (step == 1) return lo + before;
      if (before == 0) return lo;
      hi = min(hi, lo + before * step);
      lo += (before - 1) * step + 1;
    }
    return lo;
  }
  // The first key that any row from t on needs (tokens if there is none).
  __device__ __forceinline__ int first_key(int t) const {
    if (b == nullptr) return 0;
    const int s = upto(t) - 1;
    return s >= n ? tokens : min(max(at(max(s, 0)), 0), tokens);
  }
  // The end of the rows that any key up to t is needed by (0 if there is none).
  __device__ __forceinline__ int last_query(int t) const {
    if (b == nullptr) return tokens;
    const int s = upto(t) - 1;
    return s < 0 ? 0 : min(max(at(min(s + 1, n)), 0), tokens);
  }
  // The sequence of row t0 + lane: its rows are [start, end).  In none: start = row + 1, end = row.
  __device__ __forceinline__ void rows(int t0, int* start, int* end) const {
    const int lane = threadIdx.x & 31, t = t0 + lane;
    if (b == nullptr) {
      *start = t < tokens ? 0 : t + 1;
      *end = t < tokens ? tokens : t;
      return;
    }
    // one bit for each of the warp's rows that a boundary after t0 lies at, and the first boundary behind them
    const int c = upto(t0);
    uint32_t starts = 0;
    int next = 0x7fffffff;
    for (int i = c; ; i += 32) {
      const int v = n < 32 ? held : i + lane <= n ? b[i + lane] : 0x7fffffff;
      starts |= __reduce_or_sync(0xffffffffu, v > t0 && v - t0 < 32 ? 1u << (v - t0) : 0u);
      next = min(next, __reduce_min_sync(0xffffffffu, v > t0 && v - t0 >= 32 ? v : 0x7fffffff));
      if (n < 32 || i + 32 > n || next != 0x7fffffff) break;
    }
    const uint32_t upto_me = 0xffffffffu >> (31 - lane);
    const uint32_t mine = starts & upto_me, later = starts & ~upto_me;
    const int before = c > 0 ? at(c - 1) : 0, last = at(n);          // (the whole warp's, so not inside what lanes decide)
    int s = mine != 0u ? t0 + 31 - __clz(mine) : before;
    int e = later != 0u ? t0 + __ffs(later) - 1 : next;
    const bool none = t >= tokens || (mine == 0u && c == 0) || t >= last;
    s = none ? t + 1 : min(max(s, 0), t);
    e = none ? t : min(max(e, t + 1), tokens);
    *start = s;
    *end = e;
  }
};
// The same of one row, for the kernels' rare ways.
__device__ __forceinline__ void row_bounds(const Args& a, int rep, int t, int* start, int* end) {
  const Bounds bounds(a, rep);
  int s, e;
  bounds.rows(t, &s, &e);
  *start = __shfl_sync(0xffffffffu, s, 0);
  *end = __shfl_sync(0xffffffffu, e, 0);
}

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.69314718055994531f;

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

template <typename T>
__device__ __forceinline__ T* head_ptr(const Tensor& t, int rep, int head, int head_dim) {
  return static_cast<T*>(t.p) + rep * t.replica + (int64_t)head * head_dim;
}

// ---- rows by themselves, one warp each: lane l has the elements l, l + 32, ... of a head (256 at most) --------------------
constexpr int kLaneMost = 8;

template <typename T>
__device__ __forceinline__ void lane_load(const T* p, int hd, int lane, float (&x)[kLaneMost]) {
#pragma unroll
  for (int e = 0; e < kLaneMost; ++e) x[e] = lane + 32 * e < hd ? to_f32(p[lane + 32 * e]) : 0.f;
}
template <typename T>
__device__ __forceinline__ void lane_store(T* p, int hd, int lane, const float (&x)[kLaneMost], float by) {
#pragma unroll
  for (int e = 0; e < kLaneMost; ++e)
    if (lane + 32 * e < hd) p[lane + 32 * e] = from_f32<T>(x[e] * by);
}
__device__ __forceinline__ float lane_dot(const float (&x)[kLaneMost], const float (&y)[kLaneMost], int hd, int lane) {
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < kLaneMost; ++e)
    if (lane + 32 * e < hd) s = fmaf(x[e], y[e], s);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  return s;
}

template <typename T>
__device__ __noinline__ void forward_row(const Args& a, int rep, int head, int i) {
  const int lane = threadIdx.x & 31, hd = a.head_dim, kvh = head / (a.heads / a.kv_heads);
  int from, end;
  row_bounds(a, rep, i, &from, &end);
  float q[kLaneMost], x[kLaneMost], acc[kLaneMost] = {};
  lane_load(head_ptr<const T>(a.q, rep, head, hd) + i * a.q.row, hd, lane, q);
  const T* k = head_ptr<const T>(a.k, rep, kvh, hd);
  const T* v = head_ptr<const T>(a.v, rep, kvh, hd);
  float top = -INFINITY, sum = 0.f;
  for (int64_t j = from; j <= i; ++j) {
    lane_load(k + j * a.k.row, hd, lane, x);
    const float s = lane_dot(q, x, hd, lane) * a.scale;
    top = s > top || s != s ? s : top;
    if (top != top) break;
  }
  if (fabsf(top) < INFINITY) {
    for (int64_t j = from; j <= i; ++j) {
      lane_load(k + j * a.k.row, hd, lane, x);
      const float p = expf(lane_dot(q, x, hd, lane) * a.scale - top);
      sum += p;
      lane_load(v + j * a.v.row, hd, lane, x);
#pragma unroll
      for (int e = 0; e < kLaneMost; ++e) acc[e] = fmaf(p, x[e], acc[e]);
    }
  } else {                               // NaN, or infinite scores only: the softmax has no value
#pragma unroll
    for (int e = 0; e < kLaneMost; ++e) acc[e] = NAN;
    sum = NAN;
  }
  lane_store(head_ptr<T>(a.out, rep, head, hd) + i * a.out.row, hd, lane, acc, 1.f / sum);
  if (lane == 0) a.lse[((int64_t)rep * a.heads + head) * a.tokens + i] = fabsf(top) == INFINITY ? top : logf(sum) + top;
}

template <typename T>
__device__ __noinline__ void dq_row(const Args& a, int rep, int head, int i) {
  const int lane = threadIdx.x & 31, hd = a.head_dim, kvh = head / (a.heads / a.kv_heads);
  int from, end;
  row_bounds(a, rep, i, &from, &end);
  const int64_t stat = ((int64_t)rep * a.heads + head) * a.tokens + i;
  float q[kLaneMost], g[kLaneMost], x[kLaneMost], y[kLaneMost], acc[kLaneMost] = {};
  lane_load(head_ptr<const T>(a.q, rep, head, hd) + i * a.q.row, hd, lane, q);
  lane_load(head_ptr<const T>(a.dout, rep, head, hd) + i * a.dout.row, hd, lane, g);
  lane_load(head_ptr<const T>(a.out, rep, head, hd) + i * a.out.row, hd, lane, x);
  const float lse = a.lse[stat], dot = lane_dot(g, x, hd, lane);
  const T* k = head_ptr<const T>(a.k, rep, kvh, hd);
  const T* v = head_ptr<const T>(a.v, rep, kvh, hd);
  for (int64_t j = from; j <= i; ++j) {
    lane_load(k + j * a.k.row, hd, lane, x);
    lane_load(v + j * a.v.row, hd, lane, y);
    const float ds = expf(lane_dot(q, x, hd, lane) * a.scale - lse) * (lane_dot(g, y, hd, lane) - dot);
#pragma unroll
    for (int e = 0; e < kLaneMost; ++e) acc[e] = fmaf(ds, x[e], acc[e]);
  }
  lane_store(head_ptr<T>(a.dq, rep, head, hd) + i * a.dq.row, hd, lane, acc, a.scale);
}

template <typename T>
__device__ __noinline__ void dkv_row(const Args& a, int rep, int kvh, int j) {
  const int lane = threadIdx.x & 31, hd = a.head_dim, group = a.heads / a.kv_heads;
  int start, end;
  row_bounds(a, rep, j, &start, &end);
  float k[kLaneMost], v[kLaneMost], x[kLaneMost], g[kLaneMost], dk[kLaneMost] = {}, dv[kLaneMost] = {};
  lane_load(head_ptr<const T>(a.k, rep, kvh, hd) + j * a.k.row, hd, lane, k);
  lane_load(head_ptr<const T>(a.v, rep, kvh, hd) + j * a.v.row, hd, lane, v);
  for (int head = kvh * group; head < (kvh + 1) * group; ++head) {
    const T* q = head_ptr<const T>(a.q, rep, head, hd);
    const T* d = head_ptr<const T>(a.dout, rep, head, hd);
    const T* o = head_ptr<const T>(a.out, rep, head, hd);
    const float* lse = a.lse + ((int64_t)rep * a.heads + head) * a.tokens;
    for (int64_t i = j; i < end; ++i) {
      lane_load(d + i * a.dout.row, hd, lane, g);
      lane_load(o + i * a.out.row, hd, lane, x);
      const float dot = lane_dot(g, x, hd, lane);
      lane_load(q + i * a.q.row, hd, lane, x);
      const float p = expf(lane_dot(k, x, hd, lane) * a.scale - lse[i]);
      const float ds = p * (lane_dot(g, v, hd, lane) - dot);
#pragma unroll
      for (int e = 0; e < kLaneMost; ++e) {
        dk[e] = fmaf(ds, x[e], dk[e]);
        dv[e] = fmaf(p, g[e], dv[e]);
      }
    }
  }
  lane_store(head_ptr<T>(a.dk, rep, kvh, hd) + j * a.dk.row, hd, lane, dk, a.scale);
  lane_store(head_ptr<T>(a.dv, rep, kvh, hd) + j * a.dv.row, hd, lane, dv, 1.f);
}

// Whether the tensor-core kernels take a call: bf16, heads of whole 16 bytes up to 128 elements, every row on a 16-byte
// boundary (TMA), and a positive scale (the running maximum is that of the products, and what is masked stays -inf).
bool tc_takes(const Args& a, int dtype);
cudaError_t tc_forward(const Args& a, cudaStream_t st);
cudaError_t tc_backward(const Args& a, cudaStream_t st);

}  // namespace attn
}  // namespace ls
