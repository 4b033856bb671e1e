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
// A product of a whole tile multiplies what the mask leaves out by zero, and zero times an infinity or NaN is NaN.  So what is
// not finite in a row of the result, and not so because of a row that it depends on, is computed once more from those rows alone: a
// NaN in one sequence, or in the rows behind the last one, reaches no other.
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

// ---- rows by themselves, a few to a warp: lane l has the elements l, l + 32, ... of a head, L of them ------------------------
// Results that a warp forms together, which share the rows they depend on, and how many of those it reads together: the loads and
// the sums over lanes of one hide those of the others.
template <int L> constexpr int kRows = L > 4 ? 2 : 4;
constexpr int kStep = 2;

template <int L, typename T>
__device__ __forceinline__ void lane_load(const T* p, int hd, int lane, float (&x)[L]) {
#pragma unroll
  for (int e = 0; e < L; ++e) x[e] = lane + 32 * e < hd ? to_f32(p[lane + 32 * e]) : 0.f;
}
// (elements behind the head are zeros)
template <int L>
__device__ __forceinline__ float lane_dot(const float (&x)[L], const float (&y)[L]) {
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < L; ++e) s = fmaf(x[e], y[e], s);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  return s;
}
// rows i, i + 1, ... of a tensor, none from `to` on: the last one again
template <int L, typename T>
__device__ __forceinline__ void lane_rows(const T* p, int64_t row, int i, int to, int hd, int lane, float (&x)[kStep][L]) {
#pragma unroll
  for (int u = 0; u < kStep; ++u) lane_load(p + min(i + u, to - 1) * row, hd, lane, x[u]);
}
// A bit for each element of a stored row that is not finite.
template <int L, typename T>
__device__ __forceinline__ uint32_t lane_ill(const T* p, int hd, int lane) {
  float x[L];
  lane_load(p, hd, lane, x);
  uint32_t ill = 0;
#pragma unroll
  for (int e = 0; e < L; ++e)
    if (!(fabsf(x[e]) < INFINITY)) ill |= 1u << e;
  return ill;
}
template <int L, typename T>
__device__ __forceinline__ void lane_store(T* p, int lane, const float (&x)[L], float by, uint32_t ill) {
#pragma unroll
  for (int e = 0; e < L; ++e)
    if ((ill >> e & 1) != 0) p[lane + 32 * e] = from_f32<T>(x[e] * by);
}
// Whether an element in `ill` is not NaN yet, so that further terms may change it.
template <int L>
__device__ __forceinline__ bool lane_open(const float (&x)[L], uint32_t ill) {
  bool open = false;
#pragma unroll
  for (int e = 0; e < L; ++e) open = open || ((ill >> e & 1) != 0 && x[e] == x[e]);
  return open;
}
// What the rows that a result depends on hold of NaN, +inf and -inf: a bit for each of the lane's columns.  The results of a warp are taken
// in an order in which those of a sequence depend on more and more rows, so that each row is looked at once for all.  (When every
// result was formed again from all of its rows, one NaN in v, in the middle of 16384 rows of 16 heads of 128, took 714 ms, now 14.)
struct Held {
  uint32_t nan = 0, up = 0, down = 0;
  // rows [i, to)
  template <int L, typename T>
  __device__ __forceinline__ void add_rows(const T* p, int64_t row, int i, int to, int hd, int lane) {
    constexpr int N = 4;
    for (; i < to; i += N) {
      float x[N][L];
#pragma unroll
      for (int u = 0; u < N; ++u) lane_load(p + min(i + u, to - 1) * row, hd, lane, x[u]);
#pragma unroll
      for (int u = 0; u < N; ++u)
#pragma unroll
        for (int e = 0; e < L; ++e) {
          if (x[u][e] != x[u][e]) nan |= 1u << e;
          if (x[u][e] == INFINITY) up |= 1u << e;
          if (x[u][e] == -INFINITY) down |= 1u << e;
        }
    }
  }
  // Sums of those rows with positive factors: sets the elements that are not finite for that reason, and returns the others of `ill`.
  template <int L, typename T>
  __device__ __forceinline__ uint32_t mark(T* p, int lane, uint32_t ill) const {
    const uint32_t none = nan | (up & down), all = none | up | down;
#pragma unroll
    for (int e = 0; e < L; ++e)
      if ((ill & all) >> e & 1) p[lane + 32 * e] = from_f32<T>(none >> e & 1 ? NAN : up >> e & 1 ? INFINITY : -INFINITY);
    return ill & ~all;
  }
};

// Rows r0 + the bits of `rows`.  A row whose lse is not finite has no softmax: all of its elements are NaN, and stay so.  Those of the
// others have it as the reference of their exponentials.
template <typename T, int L>
__device__ __noinline__ void forward_rows(const Args& a, int rep, int head, int r0, uint32_t rows) {
  constexpr int R = kRows<L>;
  const int lane = threadIdx.x & 31, hd = a.head_dim, kvh = head / (a.heads / a.kv_heads);
  const T* q = head_ptr<const T>(a.q, rep, head, hd);
  const T* k = head_ptr<const T>(a.k, rep, kvh, hd);
  const T* v = head_ptr<const T>(a.v, rep, kvh, hd);
  T* out = head_ptr<T>(a.out, rep, head, hd);
  Held held;
  int first = -1, next = 0;              // of the keys that were looked at
  while (rows != 0u) {
    float x[R][L], acc[R][L], sum[R], lse[R];
    int from[R], upto[R], lo = 0x7fffffff, hi = 0;
    uint32_t ill[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int i = r0 + max(__ffs(rows) - 1, 0);
      const float l = a.lse[((int64_t)rep * a.heads + head) * a.tokens + i];
      const bool has = rows != 0u && fabsf(l) < INFINITY;
      rows &= rows - 1;
      ill[r] = 0u;
      from[r] = upto[r] = 0;             // [from, upto): its keys
      lse[r] = l;
      sum[r] = 0.f;
#pragma unroll
      for (int e = 0; e < L; ++e) x[r][e] = acc[r][e] = 0.f;
      if (!has) continue;
      int start, end;
      row_bounds(a, rep, i, &start, &end);
      if (start != first) {
        held = Held{};
        first = next = start;
      }
      held.add_rows<L>(v, a.v.row, next, i + 1, hd, lane);
      next = i + 1;
      ill[r] = held.mark<L>(out + i * a.out.row, lane, lane_ill<L>(out + i * a.out.row, hd, lane));
      if (!__any_sync(0xffffffffu, ill[r] != 0u)) continue;
      lane_load(q + i * a.q.row, hd, lane, x[r]);
      from[r] = start;
      upto[r] = i + 1;
      lo = min(lo, start);
      hi = max(hi, i + 1);
    }
    for (int j = lo; j < hi; j += kStep) {
      bool open = false;
#pragma unroll
      for (int r = 0; r < R; ++r) open = open || (upto[r] > j && lane_open(acc[r], ill[r]));
      if (!__any_sync(0xffffffffu, open)) break;
      float kk[kStep][L], vv[kStep][L], s[R][kStep];
      lane_rows(k, a.k.row, j, hi, hd, lane, kk);
      lane_rows(v, a.v.row, j, hi, hd, lane, vv);
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int u = 0; u < kStep; ++u) s[r][u] = lane_dot(x[r], kk[u]);
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int u = 0; u < kStep; ++u)
          if (j + u >= from[r] && j + u < upto[r]) {
            const float p = expf(s[r][u] * a.scale - lse[r]);
            sum[r] += p;
#pragma unroll
            for (int e = 0; e < L; ++e) acc[r][e] = fmaf(p, vv[u][e], acc[r][e]);
          }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) lane_store(out + (upto[r] - 1) * a.out.row, lane, acc[r], 1.f / sum[r], ill[r]);
  }
}

// Rows r0 + the bits of `rows`.  Where lse or D is not finite, neither is any element of the row.
template <typename T, int L>
__device__ __noinline__ void dq_rows(const Args& a, int rep, int head, int r0, uint32_t rows) {
  constexpr int R = kRows<L>;
  const int lane = threadIdx.x & 31, hd = a.head_dim, kvh = head / (a.heads / a.kv_heads);
  const T* q = head_ptr<const T>(a.q, rep, head, hd);
  const T* g = head_ptr<const T>(a.dout, rep, head, hd);
  const T* o = head_ptr<const T>(a.out, rep, head, hd);
  const T* k = head_ptr<const T>(a.k, rep, kvh, hd);
  const T* v = head_ptr<const T>(a.v, rep, kvh, hd);
  T* dq = head_ptr<T>(a.dq, rep, head, hd);
  while (rows != 0u) {
    float x[R][L], y[R][L], acc[R][L], lse[R], dot[R];
    int from[R], upto[R], lo = 0x7fffffff, hi = 0;
    uint32_t ill[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int i = r0 + max(__ffs(rows) - 1, 0);
      lane_load(g + i * a.dout.row, hd, lane, y[r]);
      lane_load(o + i * a.out.row, hd, lane, x[r]);
      lse[r] = a.lse[((int64_t)rep * a.heads + head) * a.tokens + i];
      dot[r] = lane_dot(x[r], y[r]);
      const bool has = rows != 0u && fabsf(lse[r]) < INFINITY && fabsf(dot[r]) < INFINITY;
      rows &= rows - 1;
      lane_load(q + i * a.q.row, hd, lane, x[r]);
      ill[r] = 0u;
      from[r] = upto[r] = 0;
#pragma unroll
      for (int e = 0; e < L; ++e) acc[r][e] = 0.f;
      if (!has) continue;
      int end;
      row_bounds(a, rep, i, &from[r], &end);
      ill[r] = lane_ill<L>(dq + i * a.dq.row, hd, lane);
      upto[r] = i + 1;
      lo = min(lo, from[r]);
      hi = max(hi, i + 1);
    }
    for (int j = lo; j < hi; j += kStep) {
      bool open = false;
#pragma unroll
      for (int r = 0; r < R; ++r) open = open || (upto[r] > j && lane_open(acc[r], ill[r]));
      if (!__any_sync(0xffffffffu, open)) break;
      float kk[kStep][L], vv[kStep][L], s[R][kStep], d[R][kStep];
      lane_rows(k, a.k.row, j, hi, hd, lane, kk);
      lane_rows(v, a.v.row, j, hi, hd, lane, vv);
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int u = 0; u < kStep; ++u) {
          s[r][u] = lane_dot(x[r], kk[u]);
          d[r][u] = lane_dot(y[r], vv[u]);
        }
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int u = 0; u < kStep; ++u)
          if (j + u >= from[r] && j + u < upto[r]) {
            const float ds = expf(s[r][u] * a.scale - lse[r]) * (d[r][u] - dot[r]);
#pragma unroll
            for (int e = 0; e < L; ++e) acc[r][e] = fmaf(ds, kk[u][e], acc[r][e]);
          }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) lane_store(dq + (upto[r] - 1) * a.dq.row, lane, acc[r], a.scale, ill[r]);
  }
}

// Keys k0 + the bits of `rows`, the last one first.  A query whose lse is NaN or -inf leaves nothing finite, one whose D is not finite
// nothing of dk.  dots: every row's D, or null where nobody has left it.
template <typename T, int L>
__device__ __noinline__ void dkv_rows(const Args& a, int rep, int kvh, int k0, uint32_t rows, const float* dots) {
  constexpr int R = L > 2 ? 2 : 4;       // (four keys of 128 elements take more registers than the tiles)
  const int lane = threadIdx.x & 31, hd = a.head_dim, group = a.heads / a.kv_heads;
  const int64_t stats = ((int64_t)rep * a.heads + kvh * group) * a.tokens;
  const T* k = head_ptr<const T>(a.k, rep, kvh, hd);
  const T* v = head_ptr<const T>(a.v, rep, kvh, hd);
  T* to_k = head_ptr<T>(a.dk, rep, kvh, hd);
  T* to_v = head_ptr<T>(a.dv, rep, kvh, hd);
  Held held;                             // of dout
  bool no_p = false, no_ds = false;
  int last = -1, low = 0, low_g = 0;     // of the queries that were looked at, and from where on
  while (rows != 0u) {
    float x[R][L], y[R][L], dk[R][L], dv[R][L];
    int from[R], upto[R], lo = 0x7fffffff, hi = 0;
    uint32_t ill_k[R], ill_v[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int bit = 31 - __clz(rows), j = k0 + max(bit, 0);
      ill_k[r] = ill_v[r] = 0u;
      from[r] = upto[r] = 0;             // [from, upto): its queries
#pragma unroll
      for (int e = 0; e < L; ++e) x[r][e] = y[r][e] = dk[r][e] = dv[r][e] = 0.f;
      if (rows == 0u) continue;
      rows &= ~(1u << bit);
      int start, end;
      row_bounds(a, rep, j, &start, &end);
      if (end != last) {
        held = Held{};
        no_p = no_ds = false;
        last = low = low_g = end;
      }
      for (int h = 0; h < group; ++h)
        for (int i = j; i < low; i += 32) {
          const bool in = i + lane < low;
          const float l = in ? a.lse[stats + h * a.tokens + i + lane] : 0.f, d = dots != nullptr && in ? dots[stats + h * a.tokens + i + lane] : 0.f;
          no_p = __any_sync(0xffffffffu, !(l > -INFINITY)) || no_p;
          no_ds = __any_sync(0xffffffffu, !(fabsf(d) < INFINITY)) || no_ds;
        }
      low = j;
      if (no_p) continue;
      const uint32_t of_k = lane_ill<L>(to_k + j * a.dk.row, hd, lane), of_v = lane_ill<L>(to_v + j * a.dv.row, hd, lane);
      if (dots == nullptr || __any_sync(0xffffffffu, of_v != 0u)) {
        for (int h = 0; h < group; ++h) {
          const T* g = head_ptr<const T>(a.dout, rep, kvh * group + h, hd);
          held.add_rows<L>(g, a.dout.row, j, low_g, hd, lane);
          if (dots != nullptr) continue;
          const T* o = head_ptr<const T>(a.out, rep, kvh * group + h, hd);
          for (int i = j; i < low_g; i += kStep) {
            float gg[kStep][L], oo[kStep][L];
            lane_rows(g, a.dout.row, i, low_g, hd, lane, gg);
            lane_rows(o, a.out.row, i, low_g, hd, lane, oo);
#pragma unroll
            for (int u = 0; u < kStep; ++u) no_ds = !(fabsf(lane_dot(gg[u], oo[u])) < INFINITY) || no_ds;
          }
        }
        low_g = j;
      }
      ill_k[r] = no_ds ? 0u : of_k;
      ill_v[r] = held.mark<L>(to_v + j * a.dv.row, lane, of_v);
      from[r] = j;
      if (!__any_sync(0xffffffffu, (ill_k[r] | ill_v[r]) != 0u)) continue;
      lane_load(k + j * a.k.row, hd, lane, x[r]);
      lane_load(v + j * a.v.row, hd, lane, y[r]);
      upto[r] = end;
      lo = min(lo, j);
      hi = max(hi, end);
    }
    uint32_t any_k = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) any_k |= ill_k[r];
    const bool of_dk = __any_sync(0xffffffffu, any_k != 0u);
    for (int h = 0; h < group; ++h) {
      const T* q = head_ptr<const T>(a.q, rep, kvh * group + h, hd);
      const T* g = head_ptr<const T>(a.dout, rep, kvh * group + h, hd);
      const T* o = head_ptr<const T>(a.out, rep, kvh * group + h, hd);
      const int64_t stat = stats + h * a.tokens;
      for (int i = lo; i < hi; i += kStep) {
        bool open = false;
#pragma unroll
        for (int r = 0; r < R; ++r) open = open || lane_open(dk[r], ill_k[r]) || lane_open(dv[r], ill_v[r]);
        if (!__any_sync(0xffffffffu, open)) break;
        float qq[kStep][L], gg[kStep][L], lse[kStep], dot[kStep];
        lane_rows(q, a.q.row, i, hi, hd, lane, qq);
        lane_rows(g, a.dout.row, i, hi, hd, lane, gg);
#pragma unroll
        for (int u = 0; u < kStep; ++u) {
          lse[u] = a.lse[stat + min(i + u, hi - 1)];
          dot[u] = dots != nullptr ? dots[stat + min(i + u, hi - 1)] : 0.f;
        }
        if (dots == nullptr) {
          float oo[kStep][L];
          lane_rows(o, a.out.row, i, hi, hd, lane, oo);
#pragma unroll
          for (int u = 0; u < kStep; ++u) dot[u] = lane_dot(gg[u], oo[u]);
        }
        float s[R][kStep], d[R][kStep] = {};
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int u = 0; u < kStep; ++u) s[r][u] = lane_dot(x[r], qq[u]);
        if (of_dk) {
#pragma unroll
          for (int r = 0; r < R; ++r)
#pragma unroll
            for (int u = 0; u < kStep; ++u) d[r][u] = lane_dot(y[r], gg[u]);
        }
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int u = 0; u < kStep; ++u)
            if (i + u >= from[r] && i + u < upto[r]) {
              const float p = expf(s[r][u] * a.scale - lse[u]), ds = p * (d[r][u] - dot[u]);
#pragma unroll
              for (int e = 0; e < L; ++e) {
                dk[r][e] = fmaf(ds, qq[u][e], dk[r][e]);
                dv[r][e] = fmaf(p, gg[u][e], dv[r][e]);
              }
            }
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      lane_store(to_k + from[r] * a.dk.row, lane, dk[r], a.scale, ill_k[r]);
      lane_store(to_v + from[r] * a.dv.row, lane, dv[r], 1.f, ill_v[r]);
    }
  }
}

// The larger of two numbers, NaN if one is.
__device__ __forceinline__ float max_nan(float x, float y) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(y));
  return r;
}

// Whether the tensor-core kernels take a call: bf16, heads of whole 16 bytes up to 128 elements, every row on a 16-byte
// boundary (TMA), and a positive scale (the running maximum is that of the products, and what is masked stays -inf).
bool tc_takes(const Args& a, int dtype);
cudaError_t tc_forward(const Args& a, cudaStream_t st);
cudaError_t tc_backward(const Args& a, cudaStream_t st);

}  // namespace attn
}  // namespace ls
